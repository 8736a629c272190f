"""CPU oracle of the training operators (TEST INFRASTRUCTURE ONLY): matrices in
e4m3 with a power of two for 128 neighbours of a row, and the norm over a
token's 2n reals with its gradient, in float64."""
from __future__ import annotations

import numpy as np

BLOCK = 128


def _e4m3(code):
    sign, e, m = code >> 7, code >> 3 & 15, code & 7
    if e == 15 and m == 7:
        return np.nan
    v = (1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6
    return -v if sign else v


E4M3 = np.array([_e4m3(c) for c in range(256)])


def round_e4m3(v):
    """float64, magnitudes up to 448 or NaN -> codes: the nearest of the 127
    magnitudes, found among its two neighbours, ties to the even code."""
    v = np.asarray(v, np.float64)
    a = np.abs(np.where(np.isnan(v), 0, v))
    grid = E4M3[:127]
    up = np.clip(np.searchsorted(grid, a), 0, 126)
    down = np.maximum(up - 1, 0)
    du, dd = grid[up] - a, a - grid[down]
    code = np.where((dd < du) | ((dd == du) & (down % 2 == 0)), down, up)
    code = np.where(grid[up] == a, up, code)
    return np.where(np.isnan(v), 127, code + 128 * np.signbit(v)).astype(np.uint8)


def scale_exponent(top):
    """The smallest e in [-117, 119] with top <= 448 * 2^e, found by trying them."""
    e = -117
    while e < 119 and top > 448 * 2.0 ** e:
        e += 1
    return e


def quantize(x):
    """[rows, cols] -> (codes uint8 [rows, cp], scales uint8 [ceil(cols / 512),
    rows, 4]); scale bytes of blocks past cols are 0 here."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    nb = -(-cols // BLOCK)
    codes = np.zeros((rows, nb * BLOCK), np.uint8)
    scales = np.zeros((-(-cols // 512), rows, 4), np.uint8)
    for k in range(nb):
        at = slice(k * BLOCK, min(cols, (k + 1) * BLOCK))
        block = np.where(np.isfinite(x[:, at]), x[:, at], np.nan)
        top = np.nanmax(np.abs(np.c_[block, np.zeros(rows)]), axis=1)
        e = np.array([scale_exponent(t) for t in top])
        codes[:, at] = round_e4m3(np.clip(block / 2.0 ** e[:, None], -448, 448))
        scales[k // 4, :, k % 4] = e + 127
    return codes, scales


def dequantize(codes, scales, cols):
    codes = np.asarray(codes)
    v = E4M3[codes].copy()
    for k in range(codes.shape[1] // BLOCK):
        v[:, k * BLOCK:(k + 1) * BLOCK] *= 2.0 ** (scales[k // 4, :, k % 4].astype(np.float64) - 127)[:, None]
    return v[:, :cols]


def _pairs(v, n):
    """[2n] (real parts', then imaginary parts') -> [n, 2]."""
    return np.asarray(v, np.float64).reshape(2, n).T


def layernorm(x, delta, gain, bias, eps=1e-5, center=True):
    """(h complex64, z float64 [B, n, 2], stats float64 [B, 2])."""
    h = np.asarray(x, np.complex64)
    if delta is not None:
        h = (h + np.asarray(delta, np.complex64)).astype(np.complex64)
    B, n = h.shape
    r = np.stack([h.real, h.imag], -1).astype(np.float64)
    mu = r.mean((1, 2)) if center else np.zeros(B)
    c = r - mu[:, None, None]
    inv = 1 / np.sqrt((c * c).mean((1, 2)) + float(np.float32(eps)))
    z = c * inv[:, None, None] * _pairs(gain, n)
    if bias is not None:
        z = z + _pairs(bias, n)
    return h, z, np.stack([mu, inv], 1)


def layernorm_backward(dz, h, stats, gain, dh=None, center=True):
    """(dx complex128, dgain [2n], dbias [2n]); dz [B, n, 2] reals."""
    h = np.asarray(h)
    n = h.shape[1]
    dz = np.asarray(dz, np.float64)
    mu, inv = (np.asarray(stats, np.float64)[:, i, None, None] for i in (0, 1))
    y = (np.stack([h.real, h.imag], -1).astype(np.float64) - mu) * inv
    w = dz * _pairs(gain, n)
    d = w - y * (w * y).mean((1, 2), keepdims=True)
    if center:
        d = d - w.mean((1, 2), keepdims=True)
    d = d * inv
    dx = d[..., 0] + 1j * d[..., 1]
    if dh is not None:
        dx = dx + np.asarray(dh, np.complex128)
    return dx, (dz * y).sum(0).T.reshape(-1), dz.sum(0).T.reshape(-1)
