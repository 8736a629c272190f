"""The gradient of the training norm (layernorm_backward) where its sums are long
or its tokens far from zero, and the norm near float32's largest numbers, against
oracle/training.py in 64 bits.
Tolerances, from the arithmetic (u = 2^-24, half a step of float32):

sums over   of up to 8192 entries: float32 over at most 64 tokens of a team, 7
tokens      additions to join a block's teams, then double and one rounding: 72 u
            of the sum of |dz y|; of more entries: double, one rounding of a
            block's part and one of the result, 2 u.
far tokens  (|mu| r above 64) y: the difference from the float32 mean is exact or
            rounded once, r and the factor are two more: 3 u |y|, |y| before the
            token's mean of it is taken off; that mean: at most 32 additions of a
            thread, 14 over threads and waves, the factor 1 / 2n and y's own: 50 u
            of the mean of |y|.  Others keep what the mean's rounding moves y by.
"""
import numpy as np
import pytest

from oracle import training as tr
from test_gpu_training import backward_check, dev, grad_inputs, host

pytestmark = pytest.mark.gpu

u = 2.0 ** -24


# ------------------------------------------------- sums over many tokens


def sums_of_one_and_many_small(gpu, B, n, firsts, bf16):
    """dz = 1 in the first `firsts` tokens, 2^-25 in the others; y = 1: float32 sums that begin with a 1 lose every other
    term.  (dgain, dbias), which are both firsts + (B - firsts) 2^-25 in every place."""
    import torch
    import paper_2512_02901_amd as f2
    dz = torch.full((B, n, 2), 2.0 ** -25, dtype=torch.bfloat16 if bf16 else torch.float32, device=gpu)
    dz[:firsts] = 1
    h = torch.full((B, n), 1 + 1j, dtype=torch.complex64, device=gpu)
    stats = torch.tensor([[0.0, 1.0]], device=gpu).repeat(B, 1)
    _, dgain, dbias = f2.layernorm_backward(dz if bf16 else torch.view_as_complex(dz), h, stats,
                                            torch.ones(2 * n, device=gpu), center=False, out=h)
    return host(dgain).astype(np.float64), host(dbias).astype(np.float64), firsts + (B - firsts) * 2.0 ** -25


@pytest.mark.parametrize("B, n", [(1500, 8200), (40, (1 << 19) + 3)])
@pytest.mark.parametrize("bf16", [True, False])
def test_sums_over_many_long_tokens(gpu, B, n, bf16):
    """25 tokens a block, and 40 in the only one; every term is exact: two roundings."""
    *got, want = sums_of_one_and_many_small(gpu, B, n, 1, bf16)
    for g in got:
        assert np.abs(g - want).max() <= 2 * u * want


@pytest.mark.parametrize("B, n, teams", [(1 << 20, 16, 8), (1 << 19, 300, 4), (1 << 18, 700, 2), (1 << 17, 1500, 1), (1 << 16, 3000, 1),
                                         (1 << 16, 5000, 1)])
@pytest.mark.parametrize("bf16", [True, False])
def test_sums_over_many_short_tokens(gpu, B, n, teams, bf16):
    """256 tokens for each team of 256 or 512 blocks; a team adds 64 at most.  Every term is exact."""
    *got, want = sums_of_one_and_many_small(gpu, B, n, teams, bf16)
    for g in got:
        assert np.abs(g - want).max() <= (64 + 7 + 1) * u * want


# ------------------------------------------- many tokens a block, all forms


# Tokens for three steps and more of each team, a last block with fewer and (where a block takes several tokens at a
# time) a last step with fewer: eight, four, two teams, one of one, two and four groups of entries; blocks of two a CU;
# tokens too long for registers, the last in one block.
MANY = [(6203, 130), (3103, 300), (1603, 700), (3001, 700), (1102, 2000), (2103, 1100), (801, 3001), (801, 6000),
        (200, 8200), (131, 9001), (5, (1 << 19) + 1)]


@pytest.mark.parametrize("B, n", MANY)
@pytest.mark.parametrize("bf16", [True, False])
def test_backward_of_many_tokens(gpu, B, n, bf16):
    import torch
    import paper_2512_02901_amd as f2
    center, bias = bf16, (B + bf16) % 2 == 0
    x, stats, gain, dh, dz = grad_inputs(B, n, 34, center, bf16)
    dzd = dz.to(gpu) if bf16 else torch.view_as_complex(dz.to(gpu))
    got = f2.layernorm_backward(dzd, dev(x, gpu), dev(stats, gpu), dev(gain, gpu), dh=dev(dh, gpu), center=center, bias=bias)
    backward_check(got, host(dz), x, stats, gain, dh, center)


@pytest.mark.parametrize("B, n", [(1603, 700), (1102, 2000), (801, 6000), (131, 9001), (5, (1 << 19) + 1)])
@pytest.mark.parametrize("where", ["dh", "h"])
def test_backward_of_many_tokens_in_place(gpu, B, n, where):
    import paper_2512_02901_amd as f2
    x, stats, gain, dh, dz = grad_inputs(B, n, 35, True, True)
    h, d = dev(x, gpu), dev(dh, gpu)
    got = f2.layernorm_backward(dz.to(gpu), h, dev(stats, gpu), dev(gain, gpu), dh=d, out=d if where == "dh" else h)
    assert got[0] is (d if where == "dh" else h)
    backward_check(got, host(dz), x, stats, gain, dh, True)


@pytest.mark.parametrize("n, bf16, bias", [(130, False, False), (300, True, False), (700, False, True), (2000, True, True),
                                           (3001, False, False), (6000, True, False), (9001, False, False)])
def test_backward_of_many_tokens_repeats_its_bits(gpu, n, bf16, bias):
    import torch
    import paper_2512_02901_amd as f2
    B = {130: 6203, 300: 3103, 700: 1603}.get(n, 803)
    x, stats, gain, dh, dz = grad_inputs(B, n, 36, True, bf16)
    args = (dz.to(gpu) if bf16 else torch.view_as_complex(dz.to(gpu)), dev(x, gpu), dev(stats, gpu), dev(gain, gpu))
    got = f2.layernorm_backward(*args, bias=bias)
    backward_check(got, host(dz), x, stats, gain, None, True)
    for _ in range(3):
        again = f2.layernorm_backward(*args, bias=bias)
        assert all(p is None or torch.equal(p, q) for p, q in zip(got, again))


# ------------------------------------------------------- means far from zero


def mean_check(got, dz, h, stats, gain, dh):
    """stats: the means in 64 bits (the kernel was given them in 32), factors that are float32 numbers."""
    B, n = h.shape
    dx, dgain, dbias = tr.layernorm_backward(dz, h, stats, gain, dh, True)
    mu, r = (stats[:, i, None, None] for i in (0, 1))
    y = np.abs((np.stack([h.real, h.imag], -1).astype(np.float64) - mu) * r)
    D = np.abs(mu.astype(np.float32) - mu) * r       # what the mean's rounding moves y by
    far = np.abs(mu) * r > 63.99
    yf = y + D                                       # bounds y as it is before its mean is taken off
    # tokens near zero keep D; in the others y: subtraction, factor, the mean's (3 and 50 roundings)
    E = np.where(far, 3 * u * yf + 50 * u * yf.mean((1, 2), keepdims=True), D + 2 * u * y)
    w = np.abs(dz.astype(np.float64) * np.asarray(gain, np.float64).reshape(2, n).T)
    m1, m2 = w.mean((1, 2), keepdims=True), (w * yf).mean((1, 2), keepdims=True)
    d = np.abs(np.stack([dh.real, dh.imag], -1)).astype(np.float64)
    # the float32 arithmetic's, as of any token, and what y's error makes of y mean(w y)
    tol = u * (2 * d + np.abs(r) * (8 * w + 100 * m1 + 200 * yf * m2))
    tol = tol + np.abs(r) * (E * m2 + yf * (w * E).mean((1, 2), keepdims=True))
    e = host(got[0]).astype(np.complex128) - dx
    err = np.abs(np.stack([e.real, e.imag], -1))
    assert (err <= tol).all(), (err / tol).max()
    a = np.abs(dz).astype(np.float64)
    # dz y is added and dz mean(y) taken off: two additions a token
    ga = ((a * E).sum(0) + (2 * 72 + 3) * u * (a * yf).sum(0)).T.reshape(-1)
    err = np.abs(host(got[1]) - dgain)
    assert (err <= ga).all(), (err / ga).max()
    assert (np.abs(host(got[2]) - dbias) <= 72 * u * a.sum(0).T.reshape(-1)).all()


@pytest.mark.parametrize("B, n", [(6, 33), (50, 130), (21, 300), (700, 300), (9, 700), (5, 1500), (4, 3000), (3, 6000), (7, 9001)])
@pytest.mark.parametrize("bf16", [True, False])
def test_backward_of_tokens_far_from_zero(gpu, B, n, bf16):
    """A mean above its spread by up to 10^6, tokens near zero between them: the mean in float32 is off by up to a
    tenth of the spread."""
    import torch
    import paper_2512_02901_amd as f2
    rng = np.random.default_rng((37, B, n))
    x, _, gain, dh, dz = grad_inputs(B, n, 37, True, bf16)
    part = np.stack([x.real, x.imag], -1)
    offset = np.array([1e4, 0, -1e3, 64, 3e5])[np.arange(B) % 5]
    spread = np.array([1e-2, 1, 0.1, 0.9, 1])[np.arange(B) % 5]
    part = (part * spread[:, None, None] + offset[:, None, None] + 1e-3 * rng.standard_normal((B, 1, 1))).astype(np.float32)
    x = part[..., 0] + 1j * part[..., 1]
    assert x.dtype == np.complex64
    _, _, stats = tr.layernorm(x, None, gain, None, 1e-5, True)
    stats[:, 1] = stats[:, 1].astype(np.float32)
    h, d = dev(x, gpu), dev(dh, gpu)
    dzd = dz.to(gpu) if bf16 else torch.view_as_complex(dz.to(gpu))
    args = dzd, h, dev(stats.astype(np.float32), gpu), dev(gain, gpu)
    got = f2.layernorm_backward(*args, dh=d)
    mean_check(got, host(dz), x, stats, gain, dh)
    again = f2.layernorm_backward(*args, dh=d, out=h)
    assert all(torch.equal(p, q) for p, q in zip(got, again))


# ---------------------------------------------- entries near the largest float32


def large_tokens(n):
    rng = np.random.default_rng((38, n))
    part = (2e38 * rng.standard_normal((6, n, 2))).clip(-3.3e38, 3.3e38).astype(np.float32)
    part[1:3] = 3.3e38
    part[1, 0, 0] = part[2, n - 1, 1] = -3.3e38  # 6.6e38 below the others' mean
    part[3] *= np.float32(2.0 ** -10)
    part[4] = np.float32(3e38) + part[4] * np.float32(2.0 ** -8)
    x = (part[..., 0] + 1j * part[..., 1]).astype(np.complex64)
    gain = (1 + 0.1 * rng.standard_normal(2 * n)).astype(np.float32)
    return x, gain, rng.standard_normal(2 * n).astype(np.float32)


@pytest.mark.parametrize("n", [64, 1000, 3000, 5001, 9001])
@pytest.mark.parametrize("fp8", [False, True])
def test_norm_of_entries_near_the_largest(gpu, n, fp8):
    """Differences from the mean that are no float32, factors that are no normal one.  z: within 8 u (|t| + |bias|) and
    half a step of bf16, or of e4m3 as in the other tests of the norm."""
    import paper_2512_02901_amd as f2
    x, gain, bias = large_tokens(n)
    h, z, s = f2.add_layernorm(dev(x, gpu), dev(gain, gpu), bias=dev(bias, gpu), fp8=fp8)
    _, want, _ = tr.layernorm(x, None, gain, bias)
    b = np.abs(bias).astype(np.float64).reshape(2, n).T
    tol = 8 * u * (np.abs(want - bias.astype(np.float64).reshape(2, n).T) + b)
    v = (host(z.dequantize()).reshape(want.shape) if fp8 else host(z)).astype(np.float64)
    if fp8:
        unit = 2.0 ** (host(z.scales).transpose(1, 0, 2).reshape(len(want), -1).astype(np.float64) - 127)
        unit = np.repeat(unit, 128, 1)[:, :2 * n].reshape(want.shape)
        tol = tol + np.maximum(2.0 ** -4 * (np.abs(want) + tol), 2.0 ** -10 * unit)
    else:
        tol = tol + 2.0 ** -8 * (np.abs(want) + tol)
    assert (np.abs(v - want) <= tol).all()


@pytest.mark.parametrize("n", [64, 300, 700, 1000, 3000, 5001, 9001])
def test_backward_of_entries_near_the_largest(gpu, n):
    """Gradients of gain and bias; dx is r ~ 10^-38 times ordinary numbers, to half a step of 2^-149 more a rounding.
    One entry of 18002 below the others is 67 spreads from zero, so there the mean is the one in 64 bits (far tokens
    above): 50 u of the mean of |y|, y with what the mean's rounding moves it by."""
    import torch
    import paper_2512_02901_amd as f2
    x, gain, _ = large_tokens(n)
    _, _, stats = tr.layernorm(x, None, gain, None)
    s32 = stats.astype(np.float32)
    keep = np.arange(6) != 4  # 2^8 spreads from zero: the mean's rounding counts there
    x, s32, stats = x[keep], s32[keep], stats[keep].astype(np.float64)
    far = np.abs(stats[:, 0]) * stats[:, 1] > 64
    assert far.any() == (n == 9001)
    rounded = np.abs(s32[:, 0] - stats[:, 0]) * s32[:, 1]
    held = np.stack([np.where(far, stats[:, 0], s32[:, 0].astype(np.float64)), s32[:, 1].astype(np.float64)], 1)
    dz = np.random.default_rng((39, n)).standard_normal((5, n, 2)).astype(np.float32)
    got = f2.layernorm_backward(torch.view_as_complex(dev(dz, gpu)), dev(x, gpu), dev(s32, gpu), dev(gain, gpu))
    dx, dgain, dbias = tr.layernorm_backward(dz, x, held, gain)
    y = np.abs((np.stack([x.real, x.imag], -1).astype(np.float64) - held[:, 0, None, None]) * held[:, 1, None, None])
    w = np.abs(dz * gain.reshape(2, n).T).astype(np.float64)
    m1, m2 = w.mean((1, 2), keepdims=True), (w * y).mean((1, 2), keepdims=True)
    e = host(got[0]).astype(np.complex128) - dx
    err = np.abs(np.stack([e.real, e.imag], -1))
    assert (err <= u * s32[:, 1, None, None].astype(np.float64) * (8 * w + 100 * m1 + 100 * y * m2) + 2.0 ** -149).all()
    E = np.where(far, 50 * u * (y.mean((1, 2)) + rounded), 0)[:, None, None]
    ga, ba = (np.abs(dz) * (y + E / (15 * u))).sum(0).T.reshape(-1), np.abs(dz).astype(np.float64).sum(0).T.reshape(-1)
    assert (np.abs(host(got[1]) - dgain) <= 15 * u * ga).all()
    assert (np.abs(host(got[2]) - dbias) <= 12 * u * ba).all()
