"""The rounding of the training norm's outputs, pinned: what add_layernorm stores
is the nearest number of its type to z in 64 bits, oracle/training.py's.

The 8-bit output is formed in double: the sum of a token's 2n values is off by
at most 100 roundings of 2^-53 of the values' mean, r, the two factors and the
bias add a few more, so z is within 2^-45 (|t| + |bias| + r |gain| max|h|), t =
(h - mu) r gain.  A code or a scale byte may differ from the oracle's only where
z that far up or down has it: 2^-40 is taken.  The bf16 output is formed in
float32 from the double difference: within 8 u (|t| + |bias|), u = 2^-24, and
half a step of bf16 where z lies, 2^-8 of its power of two.
"""
import numpy as np
import pytest

from oracle import training as tr
from test_gpu_training import dev, host, norm_inputs, raw

pytestmark = pytest.mark.gpu

u = 2.0 ** -24
SIZES = [(300, 40), (77, 129), (64, 256), (40, 1000), (77, 1500), (30, 2048), (9, 4099), (5, 8192), (3, 9001)]


def inputs(B, n, seed):
    """Ordinary tokens, and some with a mean above their spread or a small size, where eps counts."""
    x, delta, gain, bias = norm_inputs(B, n, seed)
    x[1::5] = x[1::5] * np.float32(1e-2) + np.complex64(100 - 100j)
    x[2::5] *= np.float32(1e-3)
    delta[2::5] *= np.float32(1e-3)
    return x, delta, gain, bias


def interleaved(v, n):
    return np.asarray(v, np.float64).reshape(2, n).T


@pytest.mark.parametrize("B, n", SIZES)
@pytest.mark.parametrize("center", [True, False])
def test_codes_and_scales_of_the_norm(gpu, B, n, center):
    import paper_2512_02901_amd as f2
    x, delta, gain, bias = inputs(B, n, 70)
    for b in (bias, None):
        h, z, _ = f2.add_layernorm(dev(x, gpu), dev(gain, gpu), bias=None if b is None else dev(b, gpu), delta=dev(delta, gpu),
                                   center=center, fp8=True)
        want_h, want, s = tr.layernorm(x, delta, gain, b, 1e-5, center)
        np.testing.assert_array_equal(host(h), want_h)
        add = interleaved(b, n) if b is not None else 0.0
        most = np.maximum(np.abs(want_h.real), np.abs(want_h.imag)).astype(np.float64).max(1)[:, None, None]
        tol = 2.0 ** -40 * (np.abs(want - add) + np.abs(add) + s[:, 1, None, None] * np.abs(interleaved(gain, n)) * most)
        got, scales = raw(z)
        down, up = (tr.quantize((np.sign(want) * (np.abs(want) + k * tol)).reshape(B, 2 * n)) for k in (-1, 1))
        near = (down[0] != up[0]).sum() + (down[1] != up[1]).sum()
        assert near <= 1e-4 * got.size
        assert ((scales == down[1]) | (scales == up[1])).all()
        assert ((got == down[0]) | (got == up[0])).all()


@pytest.mark.parametrize("B, n", SIZES)
@pytest.mark.parametrize("center", [True, False])
def test_bf16_of_the_norm(gpu, B, n, center):
    import paper_2512_02901_amd as f2
    x, delta, gain, bias = inputs(B, n, 71)
    for b in (bias, None):
        _, z, _ = f2.add_layernorm(dev(x, gpu), dev(gain, gpu), bias=None if b is None else dev(b, gpu), delta=dev(delta, gpu),
                                   center=center)
        _, want, _ = tr.layernorm(x, delta, gain, b, 1e-5, center)
        add = interleaved(b, n) if b is not None else 0.0
        tol = 8 * u * (np.abs(want - add) + np.abs(add))
        half = 2.0 ** -8 * 2.0 ** np.floor(np.log2(np.maximum(np.abs(want) + tol, 2.0 ** -126)))
        err = np.abs(host(z).astype(np.float64) - want)
        assert (err <= half + tol).all(), (err / (half + tol)).max()


@pytest.mark.parametrize("n", [64, 300, 1000, 2048, 3001, 5000, 8200])
def test_values_beside_the_midpoints_of_codes(gpu, n):
    """Entries of +-1 +-i, so z is +-r gain; the gains are the float32 numbers around each midpoint of two codes, over r:
    z lies within 2^-22 of a midpoint, and float32 on the way would put many on its other side."""
    import paper_2512_02901_amd as f2
    rng = np.random.default_rng((72, n))
    x = (rng.choice([-1, 1], (4, n)) + 1j * rng.choice([-1, 1], (4, n))).astype(np.complex64)
    r = 1 / np.sqrt(1 + float(np.float32(1e-5)))
    grid = tr.E4M3[8:125]  # normal ones, below 400
    mid = rng.choice((grid[1:] + grid[:-1]) / 2, 2 * n)
    gain = (mid / r).astype(np.float32)
    for _ in range(2):
        gain = np.where(rng.random(2 * n) < 0.5, np.nextafter(gain, np.float32(np.inf) * rng.choice([-1, 1], 2 * n).astype(np.float32)), gain)
    gain[:n][::64] = np.float32(400 / r)  # a block's power of two is 1: 64 entries are 128 reals
    _, z, _ = f2.add_layernorm(dev(x, gpu), dev(gain, gpu), center=False, fp8=True)
    _, want, _ = tr.layernorm(x, None, gain, None, 1e-5, False)
    got, scales = raw(z)
    down, up = (tr.quantize((want * (1 + k * 2.0 ** -40)).reshape(4, 2 * n)) for k in (-1, 1))
    assert (scales[:, :, 0] == 127).all() and (scales == down[1]).all()
    assert (down[0] != up[0]).mean() < 1e-3
    assert ((got == down[0]) | (got == up[0])).all()
    # what these values tell apart: float32 factors, rounded one after the other
    single = (np.float32(r) * gain).reshape(2, n).T[None] * np.sign(np.stack([x.real, x.imag], -1))
    assert (tr.quantize(single.reshape(4, 2 * n))[0] != down[0]).mean() > 0.05
