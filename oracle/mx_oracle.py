"""Plain fp64 definitions (numpy) of the residual path and of the microscaled formats: the counter-based generator, dropout, packing to
blocks of 32 with a common scale, the residual's addition with its norm and its gradients, the product of packed tensors."""
from __future__ import annotations

import numpy as np

E4M3, E2M1 = 1, 2
BLOCK, PAD = 32, 256
TOP = {E4M3: 8, E2M1: 2}


def numbers(fmt):
    """The format's numbers from 0 up; the index is the code without its sign."""
    if fmt == E2M1:
        return np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    return np.array([m / 8 * 2.0 ** -6 for m in range(8)] + [(1 + m / 8) * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8)][:119])


# ------------------------------------------------------------------ generator and dropout
def philox(counter, key):
    """Philox4x32-10 of counters [4, ...] under a key of two words (Salmon, Moraes, Dror, Shaw 2011, Section 4.3)."""
    c = [np.asarray(w, dtype=np.uint64) for w in counter]
    low, s = np.uint64(0xFFFFFFFF), np.uint64(32)
    k = [int(key[0]), int(key[1])]
    for _ in range(10):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> s) ^ c[1] ^ np.uint64(k[0]), q & low, (p >> s) ^ c[3] ^ np.uint64(k[1]), p & low]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return c


def kept(rows, cols, p, seed, offset):
    """[rows, cols]: whether an element is kept."""
    groups = -(-cols // 8)
    g, r = np.meshgrid(np.arange(groups, dtype=np.uint64), np.arange(rows, dtype=np.uint64))
    one = np.ones_like(g)
    w = philox((g, r, one * np.uint64(offset % 2 ** 32), one * np.uint64(offset // 2 ** 32)), (seed % 2 ** 32, seed // 2 ** 32))
    bits = np.empty((rows, groups, 8), dtype=np.int64)
    for i in range(8):
        bits[:, :, i] = (w[i // 2] >> np.uint64(16 * (i % 2))) & np.uint64(0xFFFF)
    return bits.reshape(rows, -1)[:, :cols] >= threshold(p)


def threshold(p):
    return int(np.rint(p * 65536))


def dropout(x, p, seed, offset):
    t = threshold(p)
    scale = 0.0 if t == 65536 else 65536 / (65536 - t)
    return np.where(kept(*x.shape, p, seed, offset), x, 0.0) * (scale if t < 65536 else 1.0)


# ------------------------------------------------------------------ packing
def _grouped(x):
    rows, k = x.shape
    full = np.zeros((rows, -(-k // PAD) * PAD))
    full[:, :k] = x
    return full.reshape(rows, -1, BLOCK)


def quantise(x, fmt):
    """codes [rows, K] (one a byte, not yet paired) and scale bytes [rows, K / 32] of x [rows, k], K = k rounded up to 256."""
    g = _grouped(np.asarray(x, dtype=np.float64))
    most = np.abs(g).max(axis=2)
    bad = ~np.isfinite(g).all(axis=2)
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.frexp(np.where(bad, 1.0, most))[1] - 1 - TOP[fmt]
    e = np.where(most == 0, -127, np.maximum(e, -127))
    table = numbers(fmt)
    v = np.where(bad[:, :, None], 0.0, g) / np.exp2(e.astype(np.float64))[:, :, None]
    a = np.abs(v)
    up = np.minimum(np.searchsorted(table, a), len(table) - 1)
    down = np.maximum(up - 1, 0)
    to_up, to_down = np.abs(table[up] - a), np.abs(a - table[down])
    code = np.where((to_up < to_down) | ((to_up == to_down) & (up % 2 == 0)), up, down)
    code = code + np.where(np.signbit(v), 128 if fmt == E4M3 else 8, 0)
    code = np.where(bad[:, :, None], 127 if fmt == E4M3 else 7, code)
    return code.reshape(x.shape[0], -1).astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def in_memory(codes, fmt):
    return codes if fmt == E4M3 else (codes[:, 0::2] | (codes[:, 1::2] << 4)).astype(np.uint8)


def from_memory(data, fmt):
    if fmt == E4M3:
        return data
    return np.stack((data & 15, data >> 4), axis=2).reshape(data.shape[0], -1)


def values(codes, scales, k, fmt):
    half = 128 if fmt == E4M3 else 8
    table = numbers(fmt)
    if fmt == E4M3:
        table = np.append(table, np.nan)
    code = codes.astype(np.int64)
    v = table[code % half] * np.where(code >= half, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return (v.reshape(v.shape[0], -1, BLOCK) * s[:, :, None]).reshape(v.shape)[:, :k]


def rounded(x, fmt):
    """The values that a packed x stands for."""
    return values(*quantise(x, fmt), x.shape[1], fmt)


# ------------------------------------------------------------------ residual and norm
def norm(h, g, eps):
    return h / np.sqrt(np.mean(h * h, axis=1, keepdims=True) + eps) * g


def norm_grad(h, g, eps, dxn, dh):
    """-> gradients of h and g"""
    r = 1 / np.sqrt(np.mean(h * h, axis=1, keepdims=True) + eps)
    u = dxn * g
    dx = r * (u - h * r ** 2 * np.mean(u * h, axis=1, keepdims=True))
    return dx + dh, np.sum(dxn * h * r, axis=0)
