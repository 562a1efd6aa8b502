"""AdamW moments in 8 bits, and the step that makes them, in numpy.

Written from the format's definition: the codes' values are tabled and a value's
place among them is searched, in 64 bits (every fp32 value times a power of two
is exact there)."""
import numpy as np

BLOCK = 32


def table(bias):
    """Values of codes 0, 1, ...: 128 of a first moment (bias 7), 256 of a second (bias 23)."""
    c = np.arange(128 if bias == 7 else 256)
    e, f = c // 8, c % 8
    return np.where(e == 0, f / 8 * 2.0 ** (1 - bias), (1 + f / 8) * 2.0 ** (e - float(bias)))


def blocks(x):
    return x.reshape(-1, BLOCK)


def block_bytes(x):
    """b of each block: the largest magnitude times 2^(127 - b) lies in [128, 256), or b = 0."""
    top = np.abs(blocks(x)).max(1).astype(np.float64)
    with np.errstate(all="ignore"):
        b = np.floor(np.log2(np.where(top > 0, top, 2.0 ** -149))).astype(int) - 7 + 127
        # (log2 may round up to the power above)
        b = np.where(top < 2.0 ** (b - 127.0 + 7), b - 1, b)
    return np.where(np.isfinite(top), np.maximum(b, 0), 255)


def encode(x, bias, r=None):
    """(codes of magnitudes, block bytes) of fp32 values x; r: 20 random bits of each, or to the nearest."""
    t = table(bias)
    b = block_bytes(x)
    with np.errstate(all="ignore"):
        y = np.abs(blocks(x)).astype(np.float64) * 2.0 ** (127.0 - b)[:, None]
    y[b == 255] = 0
    low = np.searchsorted(t, y, side="right") - 1
    up = np.minimum(low + 1, len(t) - 1)
    place = (y - t[low]) / np.where(up > low, t[up] - t[low], 1)
    if r is None:
        code = np.where((place > 0.5) | ((place == 0.5) & (low % 2 == 1)), up, low)
    else:
        code = np.where(np.floor(place * 2 ** 20) + blocks(r) >= 2 ** 20, up, low)
    if bias == 23:
        code = np.where((blocks(x) > 0) & (b != 255)[:, None], np.maximum(code, 1), code)
    return code.reshape(-1), b


def decode(code, b, bias):
    v = table(bias)[code.astype(int)].reshape(-1, BLOCK) * 2.0 ** (b.astype(float) - 127)[:, None]
    v[b == 255] = np.nan
    return v.reshape(-1)


def pack(m, v, r=(None, None)):
    """The state that holds moments m and v (fp32, whole blocks): uint8."""
    cm, bm = encode(m, 7, r[0])
    cv, bv = encode(v, 23, r[1])
    sign = np.where((bm != 255)[:, None], blocks(np.signbit(m)) * 128, 0).reshape(-1)
    return np.concatenate([(cm + sign), cv, bm, bv]).astype(np.uint8)


def unpack(state):
    total = len(state) * 16 // 33
    c, cv, b, bv = np.split(state, [total, 2 * total, 2 * total + total // 32])
    m = decode(c & 127, b, 7)
    return np.where(c > 127, -m, m), decode(cv, bv, 23)


def chance(n, seed, step, start=0):
    """20, 20 and 16 random bits of each of n elements from element `start` on."""
    one = np.uint64(0xFFFFFFFF)
    i = np.arange(start, start + n, dtype=np.uint64)

    def times(x, k):
        return x * np.uint64(k) & one

    h = times((i & one) ^ np.uint64(((seed & 0xFFFFFFFF) + step * 0x9E3779B1) & 0xFFFFFFFF), 0x6A09E667)
    h ^= h >> np.uint64(15)
    h = times((h + np.uint64(seed >> 32 & 0xFFFFFFFF) + times(i >> np.uint64(32), 0xBB67AE85)) & one, 0xBB67AE85)
    h ^= h >> np.uint64(13)
    y = times(h, 0x3C6EF373)
    y ^= y >> np.uint64(16)
    return (h >> np.uint64(12)).astype(int), (y >> np.uint64(12)).astype(int), ((h ^ (y << np.uint64(4))) & np.uint64(0xFFFF)).astype(int)


def step32(m, v, g, beta1, beta2, scale):
    """The moments' step in fp32, each product and sum rounded."""
    f = np.float32
    with np.errstate(all="ignore"):
        g = g.astype(f) * f(scale)
        return m.astype(f) * f(beta1) + g * f(1 - beta1), v.astype(f) * f(beta2) + g * g * f(1 - beta2)


def weights64(p, m, v, step, lr, beta1, beta2, eps, decay):
    """The weights' step in 64 bits, and the magnitude of what is taken off."""
    with np.errstate(all="ignore"):
        off = lr * (m.astype(np.float64) / (1 - beta1 ** step)) / (np.sqrt(v.astype(np.float64) / (1 - beta2 ** step)) + eps)
    return p.astype(np.float64) * (1 - lr * decay) - off, np.abs(off)
