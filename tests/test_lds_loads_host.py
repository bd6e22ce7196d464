"""The built GPU code: no load to LDS reads M0 in the instruction after the one that writes it.

The instruction set asks for one wait state between a scalar write of M0 and a load that takes its
place in LDS from it.  The compiler sees to that for its own code, not inside of inline assembly.
"""
import numpy as np

import paper_1911_08020_amd as darb

#: the words of gfx950 instructions: s_mov_b32 m0, <scalar register or inline constant>, and the first
#: word of global_load_lds_dword / _dwordx3 / _dwordx4 (global segment, opcodes 42, 126, 125; cache
#: bits left out)
MOV_M0, MOV_M0_MASK = 0xBEFC0000, 0xFFFFFF00
LOAD_LDS_MASK = 0xFDFCC000
LOADS = [0xDC008000 | op << 18 for op in (42, 126, 125)]


def adjacent(words):
    """(writes of M0 right before a load to LDS, loads to LDS that have one within three words)."""
    load = np.isin(words & np.uint32(LOAD_LDS_MASK), np.array(LOADS, np.uint32))
    mov = (words & np.uint32(MOV_M0_MASK)) == MOV_M0
    near = mov[:-3] & (load[1:-2] | load[2:-1] | load[3:])
    return int((mov[:-1] & load[1:]).sum()), int(near.sum())


def test_the_search_finds_them():
    plain = [0xBEFC0004, 0xDDF48000, 0x007F0002, 0xBF810000, 0xBF800000]
    waits = [0xBEFC0004, 0xBF800000, 0xDDF48000, 0x007F0002, 0xBF810000]
    assert adjacent(np.array(plain, np.uint32)) == (1, 1)
    assert adjacent(np.array(waits, np.uint32)) == (0, 1)


def test_loads_to_lds_wait_for_m0():
    code = open(darb.LIB_PATH, "rb").read()
    words = np.frombuffer(code[:len(code) // 4 * 4], "<u4")
    at_once, near = adjacent(words)
    assert near > 100, "the library's loads to LDS were not found"
    assert at_once == 0
