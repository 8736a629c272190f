"""CPU oracle of the serving operators (TEST INFRASTRUCTURE ONLY): residual
addition + RMSNorm + int8 activations, the paged cache in microscaled 4-bit
floating point (its number format and byte layout), and causal
Hermitian-score attention of a batch of sequences over it, in float64.

``rms_norm`` and ``hermitian_attention`` of oracle/block.py are the same
operations for one token of one sequence; tests/test_oracle_serving.py holds
the two against each other.
"""
from __future__ import annotations

import numpy as np

from .block import rms_norm

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
TILE = 32


def add_rmsnorm_i8(x, delta, gain, eps=1e-5):
    """(h, z, scale): h = x + delta rounded to complex64, z = RMSNorm(h) in
    float64 [B, n, 2], scale [B] = max |z| / 127; q is z / scale rounded."""
    h = np.asarray(x, np.complex64)
    if delta is not None:
        h = (h + np.asarray(delta, np.complex64)).astype(np.complex64)
    z = rms_norm(h, gain, float(np.float32(eps)))
    z = np.stack([z.real, z.imag], -1)
    return h, z, np.abs(z).reshape(len(z), -1).max(1) / 127


def rotate(x, cos, sin):
    """complex64 x times (cos + i sin), every product and sum rounded once to float32."""
    re, im = x.real.astype(np.float32), x.imag.astype(np.float32)
    return np.stack([re * cos - im * sin, re * sin + im * cos], -1)


def mx_block(values):
    """32 reals -> (codes uint8 [32], e): the nearest of e2m1 * 2^e, found by
    trying all of them (ties to the even code, magnitudes above 6 as 6)."""
    v = np.asarray(values, np.float64)
    top = np.abs(v).max()
    e = -125
    while e < 125 and top > 7 * 2.0 ** e:
        e += 1
    codes = np.zeros(32, np.uint8)
    for i, x in enumerate(v):
        d = np.abs(min(abs(x) / 2.0 ** e, 6.0) - E2M1)
        near = np.flatnonzero(d == d.min())
        codes[i] = (near[0] if len(near) == 1 or near[0] % 2 == 0 else near[1]) + 8 * np.signbit(x)
    return codes, e


def mx_token(k, v):
    """One position's key and value of a head, float32 [dc, 2] each -> their
    code bytes [dc] and scale bytes [nb]."""
    nb = len(k) // 16
    bad = not (np.isfinite(k).all() and np.isfinite(v).all())
    out = []
    for x, is_key in ((k, True), (v, False)):
        codes, scales = np.zeros((nb, 32), np.uint8), np.zeros(nb, np.uint8)
        for b in range(nb):
            block = x[16 * b:16 * b + 16].reshape(32)
            if not np.isfinite(block).all():
                block = np.zeros(32)
            codes[b], e = mx_block(block)
            scales[b] = 255 if bad and is_key else e + 127
        codes = codes.reshape(-1, 2)
        out += [codes[:, 0] | codes[:, 1] << 4, scales]
    return out


def tile_bytes(dc):
    nb = dc // 16
    return 1024 * nb + 64 * (nb if nb <= 2 else -(-nb // 4) * 4)


def layout(dc):
    """Byte offsets in a tile: keys [32, dc], values [32, dc], their scales
    [32, nb] each."""
    nb = dc // 16
    U = 4 if nb % 2 == 0 else 2
    sb = nb if nb <= 2 else -(-nb // 4) * 4
    k, v = np.zeros((TILE, dc), int), np.zeros((TILE, dc), int)
    ks, vs = np.zeros((TILE, nb), int), np.zeros((TILE, nb), int)

    def at(b, g, r, s, byte):  # axes [2 nb / U][g][r][U / 2][s][byte]
        return ((((b // (U // 2) * 4 + g) * 16 + r) * (U // 2) + b % (U // 2)) * 2 + s) * 4 + byte

    for p in range(TILE):
        s, q = p // 16, p % 16
        for c in range(dc):
            b, e = c // 16, c % 16
            k[p, c] = at(b, e // 4, q, s, e % 4)
            v[p, c] = 512 * nb + at(b, q // 4, e, s, q % 4)
        for b in range(nb):
            ks[p, b] = 1024 * nb + p * sb + b
            vs[p, b] = 1024 * nb + 32 * sb + ((q // 4 * 2 + s) * 4 + q % 4) * sb + b
    return k, v, ks, vs


def values_of(codes, scales):
    """Code bytes [.., dc] and scale bytes [.., nb] -> float64 [.., dc, 2]."""
    def half(c):
        return np.where(c & 8, -1.0, 1.0) * E2M1[c & 7]
    scale = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return np.stack([half(codes & 15), half(codes >> 4)], -1) * np.repeat(scale, 16, axis=-1)[..., None]


def read(cache, page_size, kv_heads, dc, pages, length):
    """What a sequence's first `length` positions stand for: (k, v) float64
    [length, kv_heads, dc, 2]; NaN where `pages` names no page."""
    cache = cache.reshape(-1, kv_heads, page_size // TILE, tile_bytes(dc))
    at = layout(dc)
    out = np.full((2, length, kv_heads, dc, 2), np.nan)
    for p in range(length):
        page = pages[p // page_size]
        if not 0 <= page < len(cache):
            continue
        t = cache[page, :, p % page_size // TILE]
        kc, vc, ks, vs = (t[:, a[p % TILE]] for a in at)
        out[0, p], out[1, p] = values_of(kc, ks), values_of(vc, vs)
    return out


def attend(q, k, v, first, scale, present=None):
    """Rows of one sequence: q [n, H, dc, 2], k and v [L, kv_heads, dc, 2];
    row j stands at position first + j.  Returns (out [n, H, dc, 2], the same
    with |v| in place of v, max over positions of scale sum |q||k|)."""
    q = np.asarray(q, np.float64)
    n, H = q.shape[:2]
    L, kv = k.shape[:2]
    out, absolute, most = np.zeros_like(q), np.zeros_like(q), 0.0
    for j in range(n):
        seen = np.arange(L) <= first + j
        if present is not None:
            seen &= present
        if not seen.any():
            continue
        for h in range(H):
            kk, vv = k[seen, h * kv // H], v[seen, h * kv // H]
            s = scale * np.tensordot(kk, q[j, h], 2)
            with np.errstate(invalid="ignore"):
                p = np.exp(s - s.max())
                p /= p.sum()
                out[j, h], absolute[j, h] = np.tensordot(p, vv, 1), np.tensordot(p, np.abs(vv), 1)
            most = max(most, scale * np.tensordot(np.abs(kk), np.abs(q[j, h]), 2).max())
    return out, absolute, most
