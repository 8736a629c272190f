"""Host-side checks of the serving entry points (no GPU): sizes, and arguments
rejected before anything is launched."""
import ctypes

import pytest

from oracle import serving as sv
from paper_2512_02901_amd import binding
from paper_2512_02901_amd.binding import ERR_NULL, ERR_SHAPE, ERR_UNSUPPORTED, ERR_WORKSPACE, KvBatchDesc, KvCacheDesc

P = ctypes.c_void_p(0x1000)  # never used: every call below is refused first


@pytest.fixture(scope="module")
def lib():
    return binding.load()


def cache(data=0x1000, n_pages=4, page=64, kv=2, dc=64):
    return ctypes.byref(KvCacheDesc(data, n_pages, page, kv, dc, 0))


def batch(pages=0x1000, cu=0x1000, lens=0x1000, n_new=3, n_seqs=2, max_pages=4):
    return ctypes.byref(KvBatchDesc(pages, cu, lens, n_new, n_seqs, max_pages))


@pytest.mark.parametrize("dc", range(16, 129, 16))
def test_cache_bytes(lib, dc):
    assert lib.fairy2i_kv_cache_bytes(5, 96, 3, dc) == 5 * 3 * 3 * sv.tile_bytes(dc)


def test_cache_bytes_refusals(lib):
    f = lib.fairy2i_kv_cache_bytes
    for args in ((0, 32, 1, 16), (1, 16, 1, 16), (1, 33, 1, 16), (1, 32, 0, 16), (1, 32, 1, 8), (1, 32, 1, 20), (1, 32, 1, 144),
                 (1, 1 << 21, 1, 16), (1 << 31, 32, 1, 16), (1, 32, 65536, 16), (-1, 32, 1, 16)):
        assert f(*args) == 0, args


def test_norm_validation(lib):
    f = lib.fairy2i_add_rmsnorm_i8
    assert f(None, P, P, 1e-5, 1, 8, P, P, P, None) == ERR_NULL
    assert f(P, P, None, 1e-5, 1, 8, P, P, P, None) == ERR_NULL
    assert f(P, P, P, 1e-5, 1, 8, P, None, P, None) == ERR_NULL
    assert f(P, P, P, 1e-5, 1, 8, P, P, None, None) == ERR_NULL
    for B, n in ((0, 8), (1, 0), (1 << 31, 8), (1, (1 << 24) + 1)):
        assert f(P, P, P, 1e-5, B, n, P, P, P, None) == ERR_SHAPE
    for eps in (0.0, -1.0, float("inf"), float("nan")):
        assert f(P, P, P, eps, 1, 8, P, P, P, None) == ERR_SHAPE


def common(call):
    """What every call over a cache and a batch refuses."""
    assert call(None, batch()) == ERR_NULL
    assert call(cache(), None) == ERR_NULL
    assert call(cache(data=None), batch()) == ERR_NULL
    for k in ("pages", "cu", "lens"):
        assert call(cache(), batch(**{k: None})) == ERR_NULL
    assert call(cache(dc=40), batch()) == ERR_SHAPE
    assert call(cache(page=40), batch()) == ERR_SHAPE
    for kw in (dict(n_new=0), dict(n_new=(1 << 26) + 1), dict(n_seqs=0), dict(n_seqs=(1 << 20) + 1), dict(max_pages=0),
               dict(max_pages=1 << 25)):
        assert call(cache(), batch(**kw)) == ERR_SHAPE, kw
    assert call(cache(data=0x1008), batch()) == ERR_UNSUPPORTED


def test_append_validation(lib):
    def f(c=None, b=None, q=P, q_ld=256, heads=4, k=P, k_ld=128, v=P, v_ld=128, rope=P, n=16, out=P):
        return lib.fairy2i_kv_append(c, b, q, q_ld, heads, k, k_ld, v, v_ld, rope, n, out, None)
    common(f)
    for kw in (dict(k=None), dict(v=None), dict(rope=None), dict(q=None), dict(out=None)):
        assert f(cache(), batch(), **kw) == ERR_NULL, kw
    for kw in (dict(k_ld=127), dict(v_ld=127), dict(q_ld=255), dict(heads=0), dict(n=0)):
        assert f(cache(), batch(), **kw) == ERR_SHAPE, kw


def test_read_validation(lib):
    def f(c=None, b=None, k=P, v=P):
        return lib.fairy2i_kv_read(c, b, k, v, None)
    common(f)
    assert f(cache(), batch(), k=None) == ERR_NULL
    assert f(cache(), batch(), v=None) == ERR_NULL


def test_attend_validation(lib):
    def f(c=None, b=None, q=P, heads=4, scale=0.1, out=P, ws=P, size=1 << 40):
        return lib.fairy2i_kv_attend(c, b, q, heads, scale, out, ws, size, None)
    common(f)
    assert f(cache(), batch(), q=None) == ERR_NULL
    assert f(cache(), batch(), out=None) == ERR_NULL
    for kw in (dict(heads=0), dict(heads=3), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=1e31)):
        assert f(cache(), batch(), **kw) == ERR_SHAPE, kw
    need = lib.fairy2i_kv_attend_workspace_bytes(cache(), 3, 2, 4)
    assert need > 0
    assert f(cache(), batch(), size=need - 1) == ERR_WORKSPACE
    assert f(cache(), batch(), ws=None) == ERR_WORKSPACE
    assert f(cache(), batch(), ws=ctypes.c_void_p(0x1008)) == ERR_WORKSPACE
    for args in ((0, 2, 4), (3, 0, 4), (3, 2, 3), (3, 2, 0)):
        assert lib.fairy2i_kv_attend_workspace_bytes(cache(), *args) == 0


def test_rope_validation(lib):
    f = lib.fairy2i_rope_table
    assert f(4, 4, 1e4, None, None) == ERR_NULL
    for n, dc, base in ((0, 4, 1e4), (4, 0, 1e4), (4, 4, 0.0), (4, 4, -1.0), (4, 4, float("inf")), ((1 << 30) + 1, 4, 1e4)):
        assert f(n, dc, base, P, None) == ERR_SHAPE


def test_more_work_than_a_launch_takes(lib):
    """2^24 blocks of 256 threads: refused before the launch, which takes fewer than 2^32 threads."""
    def append(c, b, q_ld=16, heads=1, k_ld=512, q=P):
        return lib.fairy2i_kv_append(c, b, q, q_ld, heads, P, k_ld, P, k_ld, P, 16, q, None)
    assert append(cache(dc=16), batch(n_new=1 << 24)) == ERR_UNSUPPORTED
    assert append(cache(dc=16), batch(n_new=1 << 23), q_ld=1040, heads=65) == ERR_UNSUPPORTED
    assert append(cache(kv=8), batch(n_new=1 << 26), q=None) == ERR_UNSUPPORTED
    assert lib.fairy2i_kv_read(cache(kv=8), batch(n_new=1 << 26), P, P, None) == ERR_UNSUPPORTED
