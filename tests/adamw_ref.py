"""The AdamW update of include/rip.h in numpy: fp32, operation by operation."""
import numpy as np

BLOCK = 32
F = np.float32


def mix(x):
    m = (1 << 64) - 1
    x = ((x ^ (x >> 30)) * 0xBF58476D1CE4E5B9) & m
    x = ((x ^ (x >> 27)) * 0x94D049BB133111EB) & m
    return x ^ (x >> 31)


def key_of(seed, step, replica, segment):
    k = seed
    for c in (step, replica, segment):
        k = mix((k + 0x9E3779B97F4A7C15 * (c + 1)) & ((1 << 64) - 1))
    return k & 0xffffffff


def hashes(n, key):
    return hashes_from(0, n, key)


def hashes_from(first, n, key):
    x = np.arange(first, first + n, dtype=np.uint64)
    x = (x & np.uint64(0xffffffff)) ^ np.uint64(key)
    for shift, mul in ((16, 0x85ebca6b), (13, 0xc2b2ae35)):
        x = ((x ^ (x >> np.uint64(shift))) * np.uint64(mul)) & np.uint64(0xffffffff)
    return (x ^ (x >> np.uint64(16))).astype(np.uint32)


def scalars(step, lr, b1, b2, wd):
    return (F(1.0 - lr * wd), F(lr / (1.0 - b1 ** step)), F(1.0 / np.sqrt(1.0 - b2 ** step)))


def update(w, g, m, v, step, lr, b1, b2, eps, wd, gs):
    """(w, m, v) after a step; all float32 arrays."""
    decay, rate, root = scalars(step, lr, b1, b2, wd)
    with np.errstate(all="ignore"):
        g = F(gs) * g
        m = F(b1) * m + F(1.0 - b1) * g
        v = F(b2) * v + (F(1.0 - b2) * g) * g
        w = w * decay - (rate * m) / (np.sqrt(v) * root + F(eps))
    return w, m, v


def to_bf16(x):
    """float32 values as bf16 bits, to nearest even."""
    b = x.astype(F).view(np.uint32).astype(np.uint64)
    return ((b + 0x7fff + ((b >> 16) & 1)) >> 16).astype(np.uint16)


def blocks(x):
    return np.pad(x, (0, -len(x) % BLOCK)).reshape(-1, BLOCK)


def _exponents(x, top, largest):
    e = np.full(len(x), -126)
    for i, row in enumerate(np.abs(x).max(1)):
        if not np.isfinite(row):
            e[i] = 128                                  # byte 255
        else:
            while e[i] < largest and float(row) > top * 2.0 ** float(e[i]):
                e[i] += 1
    return e


def encode_m(x, h):
    """(codes, exponent bytes) of float32 x with its hashes."""
    x, r = blocks(x), blocks(h & 0xffff).astype(F) / F(65536)
    e = _exponents(x, 127.0, 121)
    with np.errstate(all="ignore"):
        q = np.floor(x * np.exp2(-e.astype(np.float64)).astype(F)[:, None] + r)
        q = np.where(e[:, None] == 128, 0, np.clip(np.nan_to_num(q), -127, 127))
    return q.astype(np.int8).ravel(), (e + 127).astype(np.uint8)


def encode_v(x, h):
    x, r = blocks(x), blocks(h >> 16)
    e = _exponents(x, 31.0 * 2 ** 14, 127)
    with np.errstate(all="ignore"):
        t = (x * np.exp2(-e.astype(np.float64)).astype(F)[:, None]).astype(F)
        low = np.floor(t + r.astype(F) / F(65536))
        # between 2^k and 2^(k+1) codes are 2^(k-4) apart
        k = np.floor(np.log2(np.maximum(t.astype(np.float64), 1)))
        high = np.floor(t / 2 ** (k - 4) + r / 65536.0) - 16 + 16 * (k - 3)
        c = np.where(t < 16, low, high)
        c = np.where(x > 0, np.maximum(c, 1), c)
        c = np.where(e[:, None] == 128, 0, np.nan_to_num(c))
    return c.astype(np.uint8).ravel(), (e + 127).astype(np.uint8)


def _steps(exps):
    with np.errstate(all="ignore"):
        return np.where(exps == 255, np.nan, np.exp2(exps.astype(np.float64) - 127)).astype(F)


def value_m(codes, exps):
    return (codes.reshape(-1, BLOCK).astype(F) * _steps(exps)[:, None]).ravel()


def value_v(codes, exps):
    c = codes.reshape(-1, BLOCK).astype(np.int64)
    x, y = c >> 4, c & 15
    f = np.where(x == 0, y, (16 + y) << np.maximum(x - 1, 0))
    return (f.astype(F) * _steps(exps)[:, None]).ravel()
