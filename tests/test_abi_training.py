"""Host-side checks of the training entry points (no GPU): sizes, and arguments
rejected before anything is launched."""
import ctypes

import pytest

from paper_2512_02901_amd import binding
from paper_2512_02901_amd.binding import ACT_BF16, ACT_F32, ACT_I8, ERR_DTYPE, ERR_NULL, ERR_SHAPE, ERR_UNSUPPORTED, ERR_WORKSPACE, Fp8Desc

P = ctypes.c_void_p(0x1000)  # never used: every call below is refused first
MOST = 1 << 22


@pytest.fixture(scope="module")
def lib():
    return binding.load()


def mat(rows=4, cols=300, codes=0x1000, scales=0x1000):
    return ctypes.byref(Fp8Desc(codes, scales, rows, cols))


def test_bytes(lib):
    for rows, cols, codes, scales in ((1, 1, 128, 4), (3, 128, 384, 12), (3, 129, 768, 12), (5, 512, 2560, 20), (5, 513, 3200, 40),
                                      (MOST, MOST, 1 << 44, 1 << 37)):
        assert lib.fairy2i_fp8_codes_bytes(rows, cols) == codes
        assert lib.fairy2i_fp8_scales_bytes(rows, cols) == scales
    for rows, cols in ((0, 1), (1, 0), (-1, 4), (MOST + 1, 1), (1, MOST + 1)):
        assert lib.fairy2i_fp8_codes_bytes(rows, cols) == 0
        assert lib.fairy2i_fp8_scales_bytes(rows, cols) == 0


def bad_matrices(call):
    assert call(None) == ERR_NULL
    assert call(mat(codes=None)) == ERR_NULL
    assert call(mat(scales=None)) == ERR_NULL
    for kw in (dict(rows=0), dict(cols=0), dict(rows=-3), dict(rows=MOST + 1), dict(cols=MOST + 1)):
        assert call(mat(**kw)) == ERR_SHAPE, kw
    assert call(mat(codes=0x1008)) == ERR_UNSUPPORTED
    assert call(mat(scales=0x1002)) == ERR_UNSUPPORTED


def test_quantize_validation(lib):
    f = lib.fairy2i_fp8_quantize
    bad_matrices(lambda m: f(P, ACT_F32, MOST + 9, m, None, None))
    bad_matrices(lambda m: f(P, ACT_F32, MOST + 9, None, m, None))
    assert f(None, ACT_F32, 300, mat(), None, None) == ERR_NULL
    assert f(P, ACT_F32, 299, mat(), None, None) == ERR_SHAPE
    assert f(P, ACT_F32, 3, None, mat(), None) == ERR_SHAPE                    # turned: x has 4 columns
    assert f(P, ACT_F32, 300, mat(), mat(), None) == ERR_SHAPE                 # not each other's transpose
    assert f(P, ACT_F32, 300, mat(), mat(rows=300, cols=5), None) == ERR_SHAPE
    for dt in (ACT_I8, -1, 3):
        assert f(P, dt, 300, mat(), None, None) == ERR_DTYPE
    assert f(P, ACT_F32, MOST, mat(rows=1 << 21, cols=1 << 17), None, None) == ERR_UNSUPPORTED  # 2^24 tiles


def test_matrices_that_overlap(lib):
    # 4 x 300: 1536 bytes of codes, 16 of scales; 300 x 4: 38400 and 1200
    a = mat(codes=0x10000, scales=0x20000)
    for codes, scales in ((0x10000, 0x40000), (0x105F0, 0x40000), (0x10000 - 38384, 0x40000), (0x40000, 0x20000),
                          (0x40000, 0x2000C), (0x1FFF0, 0x40000), (0x40000, 0x105FC)):
        b = mat(rows=300, cols=4, codes=codes, scales=scales)
        assert lib.fairy2i_fp8_quantize(P, ACT_F32, 300, a, b, None) == ERR_UNSUPPORTED, (codes, scales)
        assert lib.fairy2i_fp8_transpose(a, b, None) == ERR_UNSUPPORTED, (codes, scales)


def test_transpose_validation(lib):
    f = lib.fairy2i_fp8_transpose
    bad_matrices(lambda m: f(m, mat(), None))
    bad_matrices(lambda m: f(mat(), m, None))
    assert f(mat(), mat(), None) == ERR_SHAPE
    assert f(mat(), mat(rows=300, cols=3), None) == ERR_SHAPE
    assert f(mat(rows=1 << 21, cols=1 << 17), mat(rows=1 << 17, cols=1 << 21), None) == ERR_UNSUPPORTED


def test_dequantize_validation(lib):
    f = lib.fairy2i_fp8_dequantize
    bad_matrices(lambda m: f(m, P, None))
    assert f(mat(), None, None) == ERR_NULL


def test_gemm_validation(lib):
    def f(a=mat(), b=mat(rows=7), c=P, dt=ACT_BF16, ldc=7, acc=0, ws=P, size=1 << 40):
        return lib.fairy2i_gemm_fp8(a, b, c, dt, ldc, acc, ws, size, None)
    bad_matrices(lambda m: f(a=m))
    bad_matrices(lambda m: f(b=m))
    assert f(c=None) == ERR_NULL
    for kw in (dict(b=mat(cols=301)), dict(ldc=6), dict(acc=2), dict(acc=-1)):
        assert f(**kw) == ERR_SHAPE, kw
    assert f(dt=ACT_I8) == ERR_DTYPE
    assert f(a=mat(rows=MOST), b=mat(rows=MOST), ldc=MOST) == ERR_UNSUPPORTED
    need = lib.fairy2i_gemm_fp8_workspace_bytes
    assert need(0, 1, 1) == need(1, 0, 1) == need(1, 1, 0) == need(MOST + 1, 1, 1) == 0
    few = need(3, 64, 8192)  # few tiles over a long axis: split
    assert few > 0 and few % (4 * 3 * 64) == 0
    a, b = mat(rows=3, cols=8192), mat(rows=64, cols=8192)
    assert f(a=a, b=b, ldc=64, size=few - 1) == ERR_WORKSPACE
    assert f(a=a, b=b, ldc=64, ws=None) == ERR_WORKSPACE
    assert f(a=a, b=b, ldc=64, ws=ctypes.c_void_p(0x1002)) == ERR_WORKSPACE


def test_layernorm_validation(lib):
    def f(x=P, delta=P, gain=P, bias=P, eps=1e-5, center=1, B=4, n=150, h=P, z=P, z8=None, stats=P):
        return lib.fairy2i_add_layernorm(x, delta, gain, bias, eps, center, B, n, h, z, z8, stats, None)
    for kw in (dict(x=None), dict(gain=None), dict(stats=None), dict(z=None)):
        assert f(**kw) == ERR_NULL, kw
    for kw in (dict(B=0), dict(B=1 << 31), dict(n=0), dict(n=(1 << 24) + 1), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("inf")),
               dict(eps=float("nan")), dict(center=2), dict(center=-1)):
        assert f(**kw) == ERR_SHAPE, kw
    assert f(z8=mat()) == ERR_UNSUPPORTED
    bad = lambda m: f(z=None, z8=m)  # noqa: E731
    assert bad(mat(codes=None)) == bad(mat(scales=None)) == ERR_NULL
    assert bad(mat(rows=5)) == bad(mat(cols=299)) == bad(mat(rows=0)) == ERR_SHAPE
    assert bad(mat(codes=0x1008)) == bad(mat(scales=0x1001)) == ERR_UNSUPPORTED


def test_layernorm_backward_validation(lib):
    def f(dz=P, dt=ACT_BF16, h=P, stats=P, gain=P, dh=P, center=1, B=600, n=150, dx=P, dgain=P, dbias=P, ws=P, size=1 << 40):
        return lib.fairy2i_layernorm_backward(dz, dt, h, stats, gain, dh, center, B, n, dx, dgain, dbias, ws, size, None)
    for kw in (dict(dz=None), dict(h=None), dict(stats=None), dict(gain=None), dict(dx=None), dict(dgain=None)):
        assert f(**kw) == ERR_NULL, kw
    for kw in (dict(B=0), dict(B=1 << 31), dict(n=0), dict(n=(1 << 24) + 1), dict(center=2)):
        assert f(**kw) == ERR_SHAPE, kw
    assert f(dt=ACT_I8) == ERR_DTYPE
    for B, n in ((600, 150), (5, 9000)):
        need = lib.fairy2i_layernorm_backward_workspace_bytes(B, n)
        assert need > 0
        assert f(B=B, n=n, size=need - 1) == ERR_WORKSPACE
        assert f(B=B, n=n, ws=None) == ERR_WORKSPACE
        assert f(B=B, n=n, ws=ctypes.c_void_p(0x1002)) == ERR_WORKSPACE
    assert lib.fairy2i_layernorm_backward_workspace_bytes(0, 8) == lib.fairy2i_layernorm_backward_workspace_bytes(8, 0) == 0


def test_layernorm_backward_workspace_follows_the_tokens(lib):
    """16 bytes an entry for each block; a block's teams take 64 tokens at most; a launch keeps below 2^32 threads."""
    for n, teams in ((1, 8), (16, 8), (256, 8), (300, 4), (700, 2), (1500, 1), (3000, 1), (8192, 1)):
        for B in (100, 1000, 1 << 14, 1 << 16, 100003, 1 << 20, 1 << 22):
            need = lib.fairy2i_layernorm_backward_workspace_bytes(B, n)
            assert need % (16 * n) == 0
            blocks = max(1, need // (16 * n))
            assert B <= blocks * teams * 64, (B, n)
            assert blocks <= B
        assert lib.fairy2i_layernorm_backward_workspace_bytes((1 << 31) - 1, n) // (16 * n) <= 1 << 22


def test_outputs_that_overlap_inputs(lib):
    # 4 x 300: 1536 bytes of codes, 16 of scales; every call is refused
    def quantize(x, m=mat(codes=0x100000, scales=0x200000), dt=ACT_F32, ld=300):
        return lib.fairy2i_fp8_quantize(ctypes.c_void_p(x), dt, ld, m, None, None)
    for x in (0x100000, 0x1005FC, 0x100000 - 4796, 0x200000, 0x20000C, 0x200000 - 4796):
        assert quantize(x) == ERR_UNSUPPORTED, hex(x)
        turned = mat(300, 4, 0x100000, 0x200000) if x < 0x200000 else mat(300, 4, 0x180000, 0x200000)
        assert lib.fairy2i_fp8_quantize(ctypes.c_void_p(x), ACT_F32, 300, None, turned, None) == ERR_UNSUPPORTED, hex(x)
    # bf16 is half as long; rows far apart meet the matrix with each of them
    assert quantize(0x100000 - 2398, dt=ACT_BF16) == ERR_UNSUPPORTED
    for row in range(4):
        for off in (-1196, 0, 1532):
            assert quantize(0x100000 + off - row * 4 * 0x1000, ld=0x1000) == ERR_UNSUPPORTED, (row, off)
    # one row's distance to the next says nothing; rows further apart than memory is large
    assert quantize(0x100000, m=mat(1, 300, 0x100000, 0x200000), ld=(1 << 63) - 1) == ERR_UNSUPPORTED
    assert quantize(0x100000, ld=(1 << 62)) == ERR_UNSUPPORTED
    out = lambda p: lib.fairy2i_fp8_dequantize(mat(codes=0x100000, scales=0x200000), ctypes.c_void_p(p), None)  # noqa: E731
    for p in (0x100000, 0x1005FE, 0x100000 - 2398, 0x200000 - 2398, 0x20000E):
        assert out(p) == ERR_UNSUPPORTED, hex(p)

    # C is 4 x 7 beside 4 x 300 and 7 x 300 (2688 bytes of codes, 28 of scales)
    a, b = mat(4, 300, 0x100000, 0x200000), mat(7, 300, 0x300000, 0x400000)

    def gemm(c, dt=ACT_F32, ldc=7, x=a, y=b):
        return lib.fairy2i_gemm_fp8(x, y, ctypes.c_void_p(c), dt, ldc, 0, P, 1 << 40, None)
    for c in (0x100000, 0x1005FC, 0x100000 - 108, 0x20000C, 0x300000 - 108, 0x300A7C, 0x400018, 0x400000 - 108):
        assert gemm(c) == ERR_UNSUPPORTED, hex(c)
        assert gemm(c, x=b, y=a, ldc=4) == ERR_UNSUPPORTED, hex(c)
    assert gemm(0x100000 - 54, dt=ACT_BF16) == ERR_UNSUPPORTED
    for row in range(4):
        assert gemm(0x300000 - row * 4 * 0x1000 - 24, ldc=0x1000) == ERR_UNSUPPORTED, row
