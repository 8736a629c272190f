"""Pins of oracle/training.py: the 8-bit format against torch's cast and by
hand, the norm against the serving oracle's, its gradient against differences."""
import numpy as np
import pytest

from oracle import serving as sv
from oracle import training as tr


def test_codes_stand_for_what_torch_says():
    import torch
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(tr.E4M3, want)


def test_rounding_is_torchs_at_every_midpoint_and_beside_it():
    import torch
    grid = tr.E4M3[:127]
    mid = (grid[1:] + grid[:-1]) / 2
    v = np.concatenate([grid, mid, np.nextafter(mid, 0), np.nextafter(mid, 500)]).astype(np.float32)
    v = np.concatenate([v, np.nextafter(mid.astype(np.float32), np.float32(0)), np.nextafter(mid.astype(np.float32), np.float32(500))])
    v = v[np.abs(v) <= 448]
    v = np.concatenate([v, -v])
    want = torch.from_numpy(v).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(tr.round_e4m3(v), want)


def test_scale_exponents():
    for top, e in ((0.0, -117), (448.0, 0), (np.nextafter(448.0, 500), 1), (224.0, -1), (1.0, -8), (1.75, -8), (1.76, -7),
                   (2.0 ** -110, -117), (3.4e38, 119), (448 * 2.0 ** 119, 119)):
        assert tr.scale_exponent(top) == e, top


def test_a_matrix_by_hand():
    x = np.zeros((2, 700))
    x[0, 0], x[0, 130], x[1, 699] = 448.0, -3.0, np.nan
    codes, scales = tr.quantize(x)
    assert codes.shape == (2, 768) and scales.shape == (2, 2, 4)
    assert codes[0, 0] == 0x7E and scales[0, 0, 0] == 127
    assert scales[0, 0, 1] == 127 - 7 and tr.E4M3[codes[0, 130]] == -384      # 3 = 384 / 128
    assert codes[1, 699] == 0x7F and scales[1, 1, 1] == 10
    v = tr.dequantize(codes, scales, 700)
    np.testing.assert_array_equal(v, x)


def test_norm_is_the_serving_oracles():
    rng = np.random.default_rng(1)
    B, n = 3, 10
    x = (rng.standard_normal((B, n)) + 1j * rng.standard_normal((B, n))).astype(np.complex64)
    gain = rng.standard_normal(2 * n).astype(np.float32)
    h, z, stats = tr.layernorm(x, x, gain, None, center=False)
    h2, z2, _ = sv.add_rmsnorm_i8(x, x, gain)
    np.testing.assert_array_equal(h, h2)
    np.testing.assert_allclose(z, z2, rtol=1e-12)


@pytest.mark.parametrize("center", [True, False])
def test_gradient_against_differences(center):
    rng = np.random.default_rng(2)
    B, n, eps = 3, 5, 0.125  # exact in float32
    h = (1 + rng.standard_normal((B, n)) + 1j * rng.standard_normal((B, n))).astype(np.complex64)
    gain, bias = rng.standard_normal(2 * n), rng.standard_normal(2 * n)
    dz = rng.standard_normal((B, n, 2))

    def loss(r, gain, bias):
        mu = r.mean((1, 2), keepdims=True) if center else 0.0
        c = r - mu
        z = c / np.sqrt((c * c).mean((1, 2), keepdims=True) + eps) * gain.reshape(2, n).T + bias.reshape(2, n).T
        return (z * dz).sum()

    _, z, stats = tr.layernorm(h, None, gain, bias, eps=eps, center=center)
    r = np.stack([h.real, h.imag], -1).astype(np.float64)
    assert abs(loss(r, gain, bias) - (z * dz).sum()) < 1e-9
    dx, dgain, dbias = tr.layernorm_backward(dz, h, stats, gain, center=center)
    dx = np.stack([dx.real, dx.imag], -1)
    step = 1e-5  # the differences' own error: step^2 times a third derivative, and 1e-16 / step

    def diff(which, i):
        args = [r, gain, bias]
        out = []
        for s in (step, -step):
            a = args[which].copy()
            a.reshape(-1)[i] += s
            out.append(loss(*[a if k == which else v for k, v in enumerate(args)]))
        return (out[0] - out[1]) / (2 * step)

    for which, got in ((0, dx), (1, dgain), (2, dbias)):
        want = np.array([diff(which, i) for i in range(got.size)])
        np.testing.assert_allclose(got.reshape(-1), want, atol=1e-7, rtol=1e-7)
