"""The 8-bit states on the CPU (in the numpy form that the GPU tests compare with, bit for bit):
the codes' values, the rounding's expectation, and the averages it keeps moving."""
import numpy as np

from tests._adamw import decode, encode, random_bits, random_of

f32 = np.float32


def test_codes_are_fixed_points():
    # the product and the quotient are off by a step of fp32 at most, which the random bits
    # carry to another code once in 2^16 (or 2^15) roundings: not with the middle ones
    for signed, n in ((True, 127), (False, 255)):
        codes = np.arange(1, n + 1, dtype=np.uint8)
        codes = np.concatenate([codes, [n] * (256 - n)]).astype(np.uint8)
        for scale in (1.0, 0.37, 1e-9, 3e20):
            x = decode(codes, np.array([scale], f32), signed)
            assert x[n - 1] == f32(scale)
            c, s = encode(x, np.full(256, 32768, np.int64), signed)
            assert s[0] == f32(scale) and np.array_equal(c, codes)
    assert decode(np.array([0], np.uint8), np.array([5.0], f32), True)[0] == 0


def test_relative_spacing():
    x = decode(np.arange(1, 128, dtype=np.uint8), np.array([1.0], f32), True)
    assert (np.diff(x) / x[:-1] <= 1 / 8).all() and x[0] == f32(1.25 * 2.0 ** -16)
    x = decode(np.arange(1, 256, dtype=np.uint8), np.array([1.0], f32), False)
    assert (np.diff(x) / x[:-1] <= 1 / 16).all() and x[0] == f32(1.125 * 2.0 ** -16)


def test_rounding_is_unbiased():
    rng = np.random.default_rng(0)
    n = 256 * 400
    for signed in (True, False):
        x = (rng.random(n) * 0.9 + 0.05).astype(f32)
        x[::256] = 1.0                                   # the same scale everywhere
        if signed:
            x[1::2] *= -1
        mean = np.zeros(n)
        trials = 60
        for k in range(trials):
            rm, rv = random_of(n, 12345 + 77777 * k)
            mean += decode(*encode(x, rm if signed else rv, signed), signed)
        err = (mean / trials - x) / np.abs(x)
        # a code's spacing is at most 1/8 (1/16): the mean of n * trials roundings is within
        # five standard deviations of nothing
        assert abs(err.mean()) < 5 * (0.125 if signed else 0.0625) / 2 / np.sqrt(n * trials)


def test_random_bits_are_uniform():
    # sequential counters: each bit set half the time, bytes evenly spread, neighbours unrelated
    n = 1 << 20
    for first in (0, 0x6A09E667, 0xFFFF0000):
        h = random_bits(np.arange(n, dtype=np.uint64) + np.uint64(first))
        for bit in range(32):
            share = ((h >> np.uint64(bit)) & np.uint64(1)).mean()
            assert abs(share - 0.5) < 5 * 0.5 / np.sqrt(n), bit
        for half in (h & np.uint64(0xFFFF), h >> np.uint64(16)):
            u = half.astype(np.float64) / 65536 - 0.5
            assert abs((u[1:] * u[:-1]).mean()) < 5 / 12 / np.sqrt(n)
            assert abs((u[256:] * u[:-256]).mean()) < 5 / 12 / np.sqrt(n)
        u, w = ((x.astype(np.float64) / 65536 - 0.5) for x in (h & np.uint64(0xFFFF), h >> np.uint64(16)))
        assert abs((u * w).mean()) < 5 / 12 / np.sqrt(n)


def test_second_moment_follows_a_change():
    # v after the gradient falls to a tenth: rounding to nearest would keep it for ever
    n, b2 = 256 * 64, 0.999
    v = np.full(n, 1.0, f32)
    for t in range(2000):
        v = (v * f32(b2) + f32(0.01) * f32(1 - b2)).astype(f32)
        v = decode(*encode(v, random_of(n, t * 0x6A09E667)[1], False), False)
    want = 0.01 + 0.99 * b2 ** 2000
    assert 0.85 * want < v.mean() < 1.25 * want


def test_zero_small_and_poisoned_blocks():
    x = np.zeros(512, f32)
    x[300] = 1e-37
    c, s = encode(x, np.full(512, 65535, np.int64), False)
    assert (c == 0).all() and (s == 0).all()             # below 2^-120
    x[:] = 1.0
    x[1], x[300] = 1e-12, np.inf
    c, s = encode(x, np.zeros(512, np.int64), False)
    assert c[1] == 1 and s[0] == 1 and np.isnan(s[1])
    assert np.isnan(decode(c, s, False)[256:]).all() and np.isfinite(decode(c, s, False)[:256]).all()
    c, s = encode(x[:256], np.zeros(256, np.int64), True)
    assert c[1] == 0
