"""The AdamW step in numpy: the documented formula, every operation one correctly rounded fp32
operation (numpy's are), and the 8-bit codes."""
import math

import numpy as np

f32 = np.float32
BLOCK = 256


def random_bits(x):
    x = np.asarray(x, np.uint64) & 0xFFFFFFFF
    x ^= x >> np.uint64(16)
    x = x * np.uint64(0x9E3779B9) & np.uint64(0xFFFFFFFF)
    x ^= x >> np.uint64(15)
    x = x * np.uint64(0xB504F333) & np.uint64(0xFFFFFFFF)
    return x ^ (x >> np.uint64(16))


def _blocks(x, fill=0.0):
    n = -(-len(x) // BLOCK) * BLOCK
    return np.concatenate([x, np.full(n - len(x), fill, x.dtype)]).reshape(-1, BLOCK)


def encode(x, random, signed):
    """Codes and scales of x fp32 [n]; ``random``: 16 bits each."""
    shift, low, top = (20, 889, 127) if signed else (19, 1777, 255)
    n = len(x)
    b = _blocks(x.astype(f32))
    r = _blocks(random.astype(np.int64), 0)
    a = np.abs(b).max(1, keepdims=True)                  # NaN wins
    fine = np.isfinite(a)
    dead = ~fine | (a < f32(2.0 ** -120))
    with np.errstate(all="ignore"):
        inv = np.where(dead, f32(0), f32(1) / a)
        q = (np.abs(b) * inv).astype(f32)
    c = ((q.view(np.int32).astype(np.int64) + (r << (shift - 16))) >> shift) - low
    c = np.clip(c, 0, top)
    if signed:
        c = np.where(c > 0, c + 128 * (b < 0), 0)
    else:
        c = np.where(b > 0, np.maximum(c, 1), 0)
    c = np.where(dead, 0, c).reshape(-1)[:n].astype(np.uint8)
    scale = np.where(~fine, f32(np.nan), np.where(a < f32(2.0 ** -120), f32(0), a))
    return c, scale.reshape(-1).astype(f32)


def decode(code, scale, signed):
    shift, low, top = (20, 889, 127) if signed else (19, 1777, 255)
    c = code.astype(np.int64)
    mag = c & top
    x = np.where(mag > 0, (mag + low) << shift, 0).astype(np.int32).view(f32)
    x = (x * np.repeat(scale, BLOCK)[:len(code)]).astype(f32)
    return np.where(c > 127, -x, x).astype(f32) if signed else x


def step(p, g, m, v, t, lr, betas, eps, decay, scale=1.0):
    """p, m, v after step t, fp32."""
    b1, b2 = betas
    rs, size = f32(1 / math.sqrt(1 - b2 ** t)), f32(lr / (1 - b1 ** t))
    with np.errstate(all="ignore"):
        g = (g.astype(f32) * f32(scale)).astype(f32)
        m = m * f32(b1) + g * f32(1 - b1)
        v = v * f32(b2) + (g * g) * f32(1 - b2)
        d = np.sqrt(v) * rs + f32(eps)
        p = p.astype(f32) * f32(1 - lr * decay) - (m / d) * size
    assert p.dtype == m.dtype == v.dtype == f32
    return p, m, v


def seed_of(seed, t, tensor):
    return (seed + t * 0x6A09E667 + tensor * 0xBB67AE85) & 0xFFFFFFFF


def random_of(n, key):
    h = random_bits(np.arange(n, dtype=np.uint64) + np.uint64(key))
    return (h & np.uint64(0xFFFF)).astype(np.int64), (h >> np.uint64(16)).astype(np.int64)
