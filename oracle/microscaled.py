"""Oracle of 4-bit tiles and table rows: plain numpy in float64, from the
definitions, sharing nothing with the library.

A block is 32 values of the contracted index.  With m the largest magnitude,
e = max(floor(log2 m) - 2, -127), stored as e + 127; a value is the nearest of
0, 0.5, 1, 1.5, 2, 3, 4, 6 times 2^e (codes 0 .. 7, ties to the even code, 8
added for a negative sign); a block that is not finite is stored as 255.
"""
from __future__ import annotations

import math

import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def row_blocks(k: int) -> int:
    if k <= 32:
        return 1
    if k <= 64:
        return 2
    return 4 * -(-k // 128)


def tile_bytes(rows: int, k: int) -> int:
    return -(-17 * rows * row_blocks(k) // 16) * 16


def roles(einsum: str, operand: int):
    """Labels of the operand's rows (those both inputs and W have, then its own
    that W has, in W's order) and of its contracted index (U's order)."""
    ins, w = einsum.replace(" ", "").split("->")
    u, v = ins.split(",")
    own = (u, v)[operand]
    rows = [c for c in w if c in u and c in v] + [c for c in w if c in own and not (c in u and c in v)]
    return own, rows, [c for c in u if c in v and c not in w]


def matrix(einsum: str, operand: int, sizes: dict, tiles: np.ndarray) -> np.ndarray:
    """Tiles [n, elems] as [n, rows, K]; `sizes` are the labels' extents in a tile."""
    own, rows, k = roles(einsum, operand)
    t = np.asarray(tiles).reshape([len(tiles)] + [sizes[c] for c in own])
    # (a label summed inside one operand alone has extent one)
    order = [1 + own.index(c) for c in rows + k] + [1 + i for i, c in enumerate(own) if c not in rows + k]
    return t.transpose([0] + order).reshape(len(tiles), math.prod([sizes[c] for c in rows]),
                                            math.prod([sizes[c] for c in k]))


def encode(x: np.ndarray):
    """[..., K] float64 -> (codes [..., B, 32], scale bytes [..., B])."""
    k = x.shape[-1]
    b = row_blocks(k)
    p = np.zeros(x.shape[:-1] + (32 * b,))
    p[..., :k] = x
    p = p.reshape(x.shape[:-1] + (b, 32))
    codes = np.zeros(p.shape, np.uint8)
    scales = np.zeros(p.shape[:-1], np.uint8)
    for at in np.ndindex(p.shape[:-1]):
        v = p[at]
        if not np.all(np.isfinite(v)):
            scales[at] = 255
            continue
        m = np.abs(v).max()
        e = -127 if m == 0 else max(math.frexp(m)[1] - 1 - 2, -127)
        a = np.abs(v) / 2.0 ** e
        # distance to each magnitude; of two alike the even code
        d = np.abs(a[:, None] - MAGNITUDES[None, :])
        c = d.argmin(1)
        up = np.minimum(c + 1, 7)
        c = np.where((c % 2 == 1) & (d[np.arange(32), up] == d[np.arange(32), c]) & (up > c), up, c)
        codes[at] = c + 8 * np.signbit(v)
        scales[at] = e + 127
    return codes, scales


def pack(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """(codes [n, R, B, 32], scales [n, R, B]) -> uint8 [n, tile_bytes]."""
    n, r, b = scales.shape
    g = min(b, 4)  # groups of four blocks, every row of one before the next
    codes = codes.reshape(n, r, b // g, g, 32).transpose(0, 2, 1, 3, 4)
    scales = scales.reshape(n, r, b // g, g).transpose(0, 2, 1, 3)
    out = np.zeros((n, -(-17 * r * b // 16) * 16), np.uint8)
    c = codes.reshape(n, r * b, 16, 2)
    out[:, :16 * r * b] = (c[..., 0] | (c[..., 1] << 4)).reshape(n, 16 * r * b)
    out[:, 16 * r * b:17 * r * b] = scales.reshape(n, r * b)
    return out


def decode(codes: np.ndarray, scales: np.ndarray, k: int) -> np.ndarray:
    """The values, [..., K] float64."""
    v = MAGNITUDES[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    v = v * s[..., None]
    return v.reshape(v.shape[:-2] + (32 * v.shape[-2],))[..., :k]


def values(einsum: str, operand: int, sizes: dict, tiles: np.ndarray) -> np.ndarray:
    """Tiles [n, elems] after quantising and reading back, in the operand's own order."""
    own, rows, k = roles(einsum, operand)
    m = matrix(einsum, operand, sizes, tiles)
    v = decode(*encode(m), m.shape[-1])
    rest = [c for c in own if c not in rows + k]
    t = v.reshape([len(tiles)] + [sizes[c] for c in rows + k + rest])
    order = [1 + (rows + k + rest).index(c) for c in own]
    return t.transpose([0] + order).reshape(np.asarray(tiles).shape)


def lookup_grad(grad: np.ndarray, ids: np.ndarray, n_rows: int, scale: float):
    """(gradient, sum of magnitudes), float64."""
    total = np.zeros((n_rows, grad.shape[-1]))
    mag = np.zeros_like(total)
    flat, rows = ids.reshape(-1), grad.reshape(-1, grad.shape[-1])
    ok = (flat >= 0) & (flat < n_rows)
    np.add.at(total, flat[ok], rows[ok])
    np.add.at(mag, flat[ok], np.abs(rows[ok]))
    return total * scale, mag * abs(scale)
