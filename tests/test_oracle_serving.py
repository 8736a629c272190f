"""The serving oracle (oracle/serving.py) held against facts outside it."""
import numpy as np
import pytest

from oracle import block as ob
from oracle import serving as sv


def test_norm_is_the_block_oracles():
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((3, 20)) + 1j * rng.standard_normal((3, 20))).astype(np.complex64)
    gain = rng.standard_normal(40)
    h, z, scale = sv.add_rmsnorm_i8(x, x, gain)
    np.testing.assert_array_equal(h, 2 * x)
    want = ob.rms_norm(h, gain, float(np.float32(1e-5)))
    np.testing.assert_allclose(z[..., 0] + 1j * z[..., 1], want, rtol=1e-15)
    assert np.abs(z).max() / 127 == scale.max()


@pytest.mark.parametrize("top, e", [(7.0, 0), (np.nextafter(7.0, 8), 1), (14.0, 1), (3.5, -1), (6.0, 0), (3.6, 0), (0.0, -125),
                                    (1e-40, -125), (7 * 2.0 ** -125, -125), (3e38, 125)])
def test_block_exponent(top, e):
    v = np.zeros(32)
    v[5] = -top
    assert sv.mx_block(v)[1] == e


def test_nearest_value_and_ties():
    v = np.zeros(32)
    v[0] = 6.0  # e = 0
    v[1:8] = 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0     # every midpoint: to the even code
    v[8:15] = np.nextafter(v[1:8], 9)
    v[15:22] = -np.nextafter(v[1:8], 0)
    codes, e = sv.mx_block(v)
    assert e == 0 and list(codes[1:8]) == [0, 2, 2, 4, 4, 6, 6]
    assert list(codes[8:15]) == [1, 2, 3, 4, 5, 6, 7] and list(codes[15:22] - 8) == [0, 1, 2, 3, 4, 5, 6]
    v[:] = 7.0
    assert set(sv.mx_block(v)[0]) == {7}  # saturates


def test_error_is_at_most_half_a_step():
    rng = np.random.default_rng(1)
    v = rng.standard_normal((200, 32)) * np.exp(4 * rng.standard_normal((200, 1)))
    for row in v:
        codes, e = sv.mx_block(row)
        got = np.where(codes & 8, -1, 1) * sv.E2M1[codes & 7] * 2.0 ** e
        u = np.abs(row) / 2.0 ** e
        half = np.select([u <= 2, u <= 4], [0.25, 0.5], 1.0)
        assert (np.abs(got - row) / 2.0 ** e <= half).all()


@pytest.mark.parametrize("dc", range(16, 129, 16))
def test_layout_is_a_bijection(dc):
    k, v, ks, vs = sv.layout(dc)
    codes = np.concatenate([k.ravel(), v.ravel()])
    assert sorted(codes) == list(range(64 * dc))
    scales = np.concatenate([ks.ravel(), vs.ravel()])
    assert len(set(scales)) == 4 * dc and scales.min() >= 64 * dc and scales.max() < sv.tile_bytes(dc)
    # bytes of four positions of a value, or four entries of a key, are a dword
    assert (v[1] - v[0] == 1).all() and (v[0] % 4 == 0).all() and (k[:, 1] - k[:, 0] == 1).all() and (k[:, 0] % 4 == 0).all()


def test_attention_is_the_block_oracles():
    rng = np.random.default_rng(2)
    H, dc, L = 3, 16, 11
    q, k, v = rng.standard_normal((1, H, dc, 2)), rng.standard_normal((L, H, dc, 2)), rng.standard_normal((L, H, dc, 2))
    c = lambda t: t[..., 0] + 1j * t[..., 1]  # noqa: E731
    want = ob.hermitian_attention(c(q)[0], c(k).transpose(1, 0, 2), c(v).transpose(1, 0, 2), 9, 2 * dc)
    got, _, _ = sv.attend(q, k, v, 8, (2 * dc) ** -0.5)
    np.testing.assert_allclose(c(got)[0], want, rtol=1e-13)
    # shared key heads are repeated key heads
    q2 = rng.standard_normal((2, 2 * H, dc, 2))
    a = sv.attend(q2, k, v, 5, 0.1)[0]
    b = sv.attend(q2, k.repeat(2, 1), v.repeat(2, 1), 5, 0.1)[0]
    np.testing.assert_allclose(a, b, rtol=1e-13)
    assert (sv.attend(q2, k, v, -2, 0.1)[0] == 0).all()


def test_read_of_missing_pages_and_nan_keys():
    cache = np.zeros((2, 1, 1, sv.tile_bytes(16)), np.uint8)
    k, v = sv.read(cache, 32, 1, 16, [1, -1, 2], 96)
    assert (k[:32] == 0).all() and np.isnan(k[32:]).all() and np.isnan(v[32:]).all()
    x = np.ones((16, 2), np.float32)
    y = x.copy()
    y[3, 1] = np.inf
    kc, ks, vc, vs = sv.mx_token(x, y)
    assert ks[0] == 255 and (vc == 0).all() and vs[0] == 2
    kc, ks, vc, vs = sv.mx_token(y, x)
    assert ks[0] == 255 and sv.values_of(vc, vs).min() == 1.0
