"""The serving operators (add_rmsnorm_i8, PagedKv) against oracle/serving.py in
64 bits.  Tolerances, from the arithmetic:

norm    h is one float32 addition: equal.  z * 127 / g takes at most five
        float32 roundings (2^-24 each) of a number up to 127, and r's own
        error drops out of z / g: a q is within 0.5 + 127 * 6 * 2^-24 of the
        exact quotient.  x_scale: r (double, rounded once), h * gain, * r,
        / 127: 4 roundings, 2^-22 relative.
append  the rotation rounds as the oracle's float32 does, and everything after
        is exact: codes and scales are equal, and no other byte changes.
read    exact.
attend  the output is rounded to bf16 once (2^-9 relative) and the weights may
        be (2^-9 each), so an element is within 2^-8 A of the exact one, A =
        sum p |v|; a score's float32 sums are off by at most 2^-19 S, S =
        scale * sum |q||k| (some 2 dc additions), which changes a weight by
        that factor: (2^-8 + 2^-18 S) A in all.  Over all elements the
        roundings are independent: relative L2 at most 2^-8.
"""
import numpy as np
import pytest

from oracle import serving as sv

pytestmark = pytest.mark.gpu


def dev(a, gpu):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to(gpu)


def host(t):
    import torch
    return t.float().cpu().numpy() if t.dtype == torch.bfloat16 else t.cpu().numpy()


def bf16(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).bfloat16()


# -------------------------------------------------------------------- norm


def norm_check(h, q, s, x, delta, gain, eps=1e-5):
    want_h, z, scale = sv.add_rmsnorm_i8(x, delta, gain, eps)
    np.testing.assert_array_equal(host(h), want_h)
    got = host(s).astype(np.float64)
    np.testing.assert_allclose(got, scale, rtol=2.0 ** -22, atol=0)
    unit = np.where(scale > 0, scale, 1)[:, None, None]
    assert np.abs(host(q) - z / unit).max() <= 0.5 + 127 * 6 * 2.0 ** -24
    assert np.abs(host(q)).max() <= 127


def norm_inputs(B, n, seed):
    rng = np.random.default_rng((seed, B, n))
    def c():
        return (rng.standard_normal((B, n)) + 1j * rng.standard_normal((B, n))).astype(np.complex64)
    return c() * np.exp(rng.standard_normal((1, n))).astype(np.float32), c(), (1 + 0.1 * rng.standard_normal(2 * n)).astype(np.float32)


@pytest.mark.parametrize("B, n", [(1, 1), (3, 2), (2, 3), (5, 4), (1, 63), (4, 64), (2, 256), (3, 260), (2, 1001), (77, 1500),
                                  (2, 1024), (9, 2048), (2, 2052), (3, 8192), (2, 8196), (1, 20001), (300, 128)])
@pytest.mark.parametrize("with_delta", [True, False])
def test_norm(gpu, B, n, with_delta):
    import paper_2512_02901_amd as f2
    x, delta, gain = norm_inputs(B, n, 1)
    h, q, s = f2.add_rmsnorm_i8(dev(x, gpu), dev(gain, gpu), delta=dev(delta, gpu) if with_delta else None)
    norm_check(h, q, s, x, delta if with_delta else None, gain)


@pytest.mark.parametrize("n", [1500, 1501, 20000])
@pytest.mark.parametrize("where", ["x", "delta", "offset", "kept"])
def test_norm_in_place_and_at_odd_addresses(gpu, n, where):
    import torch
    import paper_2512_02901_amd as f2
    x, delta, gain = norm_inputs(3, n, 2)
    xd, dd, gd = dev(x, gpu), dev(delta, gpu), dev(gain, gpu)
    if where == "offset":  # 8 bytes past a 16-byte boundary
        buf = torch.empty(3 * n + 1, dtype=torch.complex64, device=gpu)
        buf[1:] = xd.reshape(-1)
        xd = buf[1:].view(3, n)
    h_out = {"x": xd, "delta": dd, "offset": None, "kept": torch.empty_like(xd)}[where]
    q0 = torch.full((3, n, 2), 99, dtype=torch.int8, device=gpu)
    s0 = torch.full((3,), -1.0, device=gpu)
    h, q, s = f2.add_rmsnorm_i8(xd, gd, delta=dd, h_out=h_out, out=(q0, s0))
    assert q is q0 and s is s0 and (h_out is None or h is h_out)
    norm_check(h, q, s, x, delta, gain)


def test_norm_extremes(gpu):
    import paper_2512_02901_amd as f2
    for n in (128, 129):
        x, _, gain = norm_inputs(8, n, 3)
        gain = np.abs(gain)
        x[0] = 0
        x[1] *= 1e30          # the squares overflow float32
        x[2] *= 1e-30         # eps decides
        x[3] = 0
        x[3, 5] = 3.0
        x[4, 7] = np.nan
        x[5, 1] = np.inf
        x[6, 0] = 1j * -np.inf
        h, q, s = f2.add_rmsnorm_i8(dev(x, gpu), dev(gain, gpu))
        ok = [0, 1, 2, 3, 7]
        norm_check(h[ok], q[ok], s[ok], x[ok], None, gain)
        assert np.isnan(host(s)[4:7]).all() and (host(q)[4:7] == 0).all()
        assert (host(q)[0] == 0).all() and host(s)[0] == 0
        h, q, s = f2.add_rmsnorm_i8(dev(x[ok], gpu), dev(0 * gain, gpu))
        assert (host(q) == 0).all() and (host(s) == 0).all()


def test_norm_feeds_the_product(gpu):
    import oracle
    import synth
    import paper_2512_02901_amd as f2
    N, K, B = 96, 256, 21
    A = synth.llama_weight(2 * N, 2 * K, (5, 5))
    U, W = oracle.to_widely_linear(A)
    (cu, su), (cw, sw) = oracle.quantize(U, 2), oracle.quantize(W, 2)
    x, delta, gain = norm_inputs(B, K, 4)
    _, q, s = f2.add_rmsnorm_i8(dev(x, gpu), dev(gain, gpu), delta=dev(delta, gpu))
    y = host(f2.wl_matmul(dev(oracle.pack(cu), gpu), dev(su, gpu), dev(oracle.pack(cw), gpu), dev(sw, gpu), q, s))
    want = oracle.wl_matmul_int8(cu, su, cw, sw, host(q), host(s))
    assert np.linalg.norm(y - want) <= 1e-5 * np.linalg.norm(want)


# ------------------------------------------------------------------- cache


class Batch:
    """Sequences with (new, length) each, on pages in no order."""

    def __init__(self, seqs, kv, dc, page, gpu, seed=0, spare=2):
        rng = np.random.default_rng((seed, kv, dc, page, len(seqs)))
        self.rng, self.seqs, self.kv, self.dc, self.page, self.gpu = rng, seqs, kv, dc, page, gpu
        used = [-(-c // page) for _, c in seqs]
        self.width = max(1, *used) if len(used) > 1 else max(1, used[0])
        self.n_pages = sum(used) + spare
        order = rng.permutation(self.n_pages)
        self.table = np.full((len(seqs), self.width), -1, np.int32)
        at = 0
        for i, u in enumerate(used):
            self.table[i, :u] = order[at:at + u]
            at += u
        self.cu = np.concatenate([[0], np.cumsum([n for n, _ in seqs])]).astype(np.int32)
        self.lens = np.array([c for _, c in seqs], np.int32)
        self.N = int(self.cu[-1])
        self.tile = sv.tile_bytes(dc)
        self.cache = rng.integers(0, 256, self.n_pages * kv * (page // 32) * self.tile, dtype=np.uint8)

    def fill(self, scale=1.0):
        """Values of ordinary size everywhere (codes stay random), garbage past every length."""
        c = self.cache.reshape(self.n_pages, self.kv, self.page // 32, self.tile)
        c[..., 64 * self.dc:] = np.clip(np.round(127 + self.rng.standard_normal(c[..., 64 * self.dc:].shape) * 0.7
                                                 + np.log2(scale)), 2, 252)
        at = np.concatenate([a[..., None] if a.ndim == 1 else a for a in sv.layout(self.dc)], 1)  # [32, bytes]
        for i, (_, length) in enumerate(self.seqs):
            for p in range(length, self.width * self.page):
                page = self.table[i, p // self.page]
                if page >= 0:
                    t = c[page, :, p % self.page // 32]
                    t[:, at[p % 32]] = self.rng.integers(0, 256, (self.kv, at.shape[1])) | 0x80  # NaN and huge scales
        return self

    def dev(self):
        import paper_2512_02901_amd as f2
        self.data = dev(self.cache, self.gpu)
        self.kvc = f2.PagedKv(self.n_pages, self.page, self.kv, self.dc, data=self.data)
        self.t = tuple(dev(a, self.gpu) for a in (self.table, self.cu, self.lens))
        return self.kvc


SEQS = {
    "one": [(1, 1)],
    "first_of_a_page": [(1, 33)],
    "decode": [(1, 7), (1, 64), (1, 65), (1, 1), (1, 95)],
    "ragged": [(5, 5), (0, 0), (3, 40), (0, 12), (37, 64), (2, 97)],
    "long": [(70, 131)],
}


def rope_of(n, dc, gpu):
    import paper_2512_02901_amd as f2
    return f2.rope_table(n, dc, device=gpu)


@pytest.mark.parametrize("dc", [1, 16, 100])
def test_rope_table(gpu, dc):
    got = host(rope_of(5000, dc, gpu)).astype(np.float64)
    angle = np.arange(5000)[:, None] * 10000.0 ** (-np.arange(dc) / dc)
    np.testing.assert_allclose(got[..., 0], np.cos(angle), rtol=0, atol=2.0 ** -24 + 1e-11)
    np.testing.assert_allclose(got[..., 1], np.sin(angle), rtol=0, atol=2.0 ** -24 + 1e-11)


def expect_append(b, k, v, turn):
    """The cache's bytes after an append of k (turned) and v."""
    want = b.cache.copy().reshape(b.n_pages, b.kv, b.page // 32, b.tile)
    at = sv.layout(b.dc)
    for i, (n, length) in enumerate(b.seqs):
        for j in range(n):
            p, row = length - n + j, b.cu[i] + j
            kr = sv.rotate(k[row], turn[p, :, 0], turn[p, :, 1])
            vr = np.stack([v[row].real, v[row].imag], -1)
            page = b.table[i, p // b.page]
            if page < 0 or page >= b.n_pages:
                continue
            for h in range(b.kv):
                t = want[page, h, p % b.page // 32]
                for a, bytes_ in zip((at[0], at[2], at[1], at[3]), sv.mx_token(kr[h], vr[h])):
                    t[a[p % 32]] = bytes_
    return want.reshape(-1)


def random_c(rng, *shape):
    return ((rng.standard_normal(shape) + 1j * rng.standard_normal(shape))
            * np.exp(rng.standard_normal(shape[:-1] + (1,)))).astype(np.complex64)


@pytest.mark.parametrize("seqs", list(SEQS))
@pytest.mark.parametrize("kv, heads, dc, page", [(1, 1, 16, 32), (5, 10, 16, 64), (3, 3, 32, 32), (2, 8, 48, 96), (4, 4, 64, 64),
                                                 (1, 3, 80, 32), (2, 2, 96, 64), (3, 6, 112, 32), (2, 4, 128, 128)])
def test_append(gpu, seqs, kv, heads, dc, page):
    import torch
    b = Batch(SEQS[seqs], kv, dc, page, gpu, seed=1)
    cache = b.dev()
    q, k, v = (random_c(b.rng, b.N, h, dc) for h in (heads, kv, kv))
    rope = rope_of(b.width * page, dc, gpu)
    got_q = cache.append(dev(k, gpu), dev(v, gpu), *b.t, rope, q=dev(q.reshape(b.N, -1), gpu))
    turn = host(rope)
    np.testing.assert_array_equal(host(b.data), expect_append(b, k, v, turn))
    pos = np.concatenate([np.arange(c - n, c) for n, c in b.seqs])
    want_q = sv.rotate(q, turn[pos][:, None, :, 0], turn[pos][:, None, :, 1])
    assert torch.equal(got_q.cpu(), bf16(want_q))
    # and what it reads as
    got_k, got_v = cache.read(*b.t, b.N)
    for i, (n, length) in enumerate(b.seqs):
        want = sv.read(host(b.data), page, kv, dc, b.table[i], length)[:, length - n:]
        np.testing.assert_array_equal(host(got_k)[b.cu[i]:b.cu[i + 1]], want[0])
        np.testing.assert_array_equal(host(got_v)[b.cu[i]:b.cu[i + 1]], want[1])


@pytest.mark.parametrize("kv, heads, dc", [(2, 6, 64), (3, 3, 16), (1, 2, 112)])
def test_append_of_columns_of_one_product(gpu, kv, heads, dc):
    import torch
    b = Batch(SEQS["ragged"], kv, dc, 32, gpu, seed=2)
    x = random_c(b.rng, b.N, (heads + 2 * kv) * dc + 3)
    xd = dev(x, gpu)
    rope = rope_of(b.width * 32, dc, gpu)
    parts = xd[:, 1:-2].split([heads * dc, kv * dc, kv * dc], 1)
    cache = b.dev()
    q0 = cache.append(parts[1], parts[2], *b.t, rope, q=parts[0])
    got = host(b.data)
    b.dev()
    q1 = b.kvc.append(parts[1].contiguous(), parts[2].contiguous(), *b.t, rope, q=parts[0].contiguous())
    np.testing.assert_array_equal(got, host(b.data))
    assert torch.equal(q0, q1)
    # in two calls: the bytes of a position do not depend on its neighbours' call
    b.dev()
    b.kvc.append(parts[1], parts[2], *b.t, rope)
    np.testing.assert_array_equal(got, host(b.data))


def test_append_one_at_a_time(gpu):
    b = Batch([(45, 45)], 3, 32, 32, gpu, seed=3)
    k, v = random_c(b.rng, 45, 3, 32), random_c(b.rng, 45, 3, 32)
    rope = rope_of(64, 32, gpu)
    b.dev().append(dev(k, gpu), dev(v, gpu), *b.t, rope)
    want = host(b.data)
    b.dev()
    for p in range(45):
        b.kvc.append(dev(k[p:p + 1], gpu), dev(v[p:p + 1], gpu), b.t[0], dev(np.array([0, 1], np.int32), gpu),
                     dev(np.array([p + 1], np.int32), gpu), rope)
    np.testing.assert_array_equal(want, host(b.data))


def test_append_extreme_values(gpu):
    b = Batch([(8, 8)], 2, 48, 32, gpu, seed=4)
    k, v = random_c(b.rng, 8, 2, 48), random_c(b.rng, 8, 2, 48)
    k[0] *= 1e37
    v[1] *= 3e37
    k[2] *= 1e-37
    v[2] *= 1e-40
    k[3] = 0
    v[4] = -0.0
    k[5, 0, 3] = np.nan           # head 0 of position 5 only
    v[6, 1, 20] = 1j * np.inf     # block 1 of head 1
    v[7, 0, 0], k[7, 0, 47] = -np.inf, np.inf
    rope = rope_of(32, 48, gpu)
    b.dev().append(dev(k, gpu), dev(v, gpu), *b.t, rope)
    got_k, got_v = (host(t) for t in b.kvc.read(*b.t, 8))
    turn = host(rope)
    for p in range(8):
        for h in range(2):
            kr = sv.rotate(k[p, h], turn[p, :, 0], turn[p, :, 1])
            kc, ks, vc, vs = sv.mx_token(kr, np.stack([v[p, h].real, v[p, h].imag], -1))
            np.testing.assert_array_equal(got_k[p, h], sv.values_of(kc, ks))
            np.testing.assert_array_equal(got_v[p, h], sv.values_of(vc, vs))
    assert np.isnan(got_k[5, 0]).all() and np.isfinite(got_k[5, 1]).all() and np.isfinite(got_v).all()


def test_append_outside_pages_and_table(gpu):
    """Positions without a page, and past the rotation table, are not stored."""
    b = Batch([(50, 50), (3, 20)], 2, 32, 32, gpu, seed=5)
    b.table[0, 1] = -1
    b.table[1, 0] = b.n_pages
    k, v, q = (random_c(b.rng, b.N, 2, 32) for _ in range(3))
    rope = rope_of(30, 32, gpu)
    got = b.dev().append(dev(k, gpu), dev(v, gpu), *b.t, rope, q=dev(q, gpu))
    turn = np.concatenate([host(rope), np.zeros((70, 32, 2), np.float32)])
    want = expect_append(b, k, v, turn).reshape(b.n_pages, 2, 1, -1)
    page = want[b.table[0, 0]]
    old = b.cache.reshape(want.shape)[b.table[0, 0]]
    for a in sv.layout(32):
        page[:, :, a[30:]] = old[:, :, a[30:]]
    np.testing.assert_array_equal(host(b.data), want.reshape(-1))
    bad = np.isnan(host(got)).all((1, 2, 3))
    np.testing.assert_array_equal(bad, np.arange(53) // 10 % 5 >= 3)  # rows 30 .. 49; 50 .. 52 are positions 17 .. 19
    assert not np.isnan(host(got)[~bad]).any()
    rk, rv = b.kvc.read(*b.t, b.N)
    assert np.isnan(host(rk)[32:]).all() and np.isnan(host(rv)[32:]).all()


def test_read_every_scale(gpu):
    b = Batch([(96, 96)], 3, 64, 32, gpu, seed=6)
    k, v = b.dev().read(*b.t, 96)
    want = sv.read(b.cache, 32, 3, 64, b.table[0], 96)
    ks = np.abs(want) < 2.0 ** 126  # the largest scale times 2 and more is past bf16's range
    np.testing.assert_array_equal(np.where(ks[0], host(k), 0), np.where(ks[0], want[0], 0))
    np.testing.assert_array_equal(np.where(ks[1], host(v), 0), np.where(ks[1], want[1], 0))


# --------------------------------------------------------------- attention


def attend_check(b, heads, q, got, scale, nan_rows=()):
    got = host(got).astype(np.float64)
    off = norm = 0.0
    for i, (n, length) in enumerate(b.seqs):
        k, v = sv.read(b.cache, b.page, b.kv, b.dc, b.table[i], length)
        present = ~np.isnan(v).any((1, 2, 3))
        rows = slice(b.cu[i], b.cu[i + 1])
        want, size, most = sv.attend(q[rows], k, v, length - n, scale, present)
        g = got[rows]
        assert np.isfinite(g).all()
        d = np.abs(g - want)
        assert (d <= (2.0 ** -8 + 2.0 ** -18 * most) * size + 1e-37).all(), (i, n, length, (d / (size + 1e-37)).max())
        off += (d ** 2).sum()
        norm += (want ** 2).sum()
    assert off <= 2.0 ** -16 * norm


def queries(b, heads, size=1.0):
    return bf16(b.rng.standard_normal((b.N, heads, b.dc, 2)) * size)


@pytest.mark.parametrize("seqs", list(SEQS))
@pytest.mark.parametrize("kv, heads, dc, page", [(1, 1, 16, 32), (5, 10, 16, 64), (3, 3, 32, 32), (2, 8, 48, 96), (4, 4, 64, 64),
                                                 (1, 17, 64, 32), (1, 3, 80, 32), (2, 2, 96, 64), (1, 6, 112, 32),
                                                 (2, 4, 128, 128), (1, 40, 128, 32)])
def test_attend(gpu, seqs, kv, heads, dc, page):
    b = Batch(SEQS[seqs], kv, dc, page, gpu, seed=7).fill()
    q = queries(b, heads)
    got = b.dev().attend(q.to(gpu), *b.t)
    attend_check(b, heads, q.double().numpy(), got, (2 * dc) ** -0.5)


# several chunks a row and several row tiles; prompts, and single tokens behind long prefixes
LONG = {
    "decode_2000": [(1, 2000)],
    "decode_mixed": [(1, 1500), (0, 0), (1, 1), (1, 3001), (1, 257), (1, 256), (1, 255)],
    "verify": [(5, 1300), (3, 700)],
    "prompt": [(300, 300)],
    "chunk": [(130, 1100), (1, 40), (257, 257)],
}


@pytest.mark.parametrize("seqs", list(LONG))
@pytest.mark.parametrize("kv, heads, dc, page", [(1, 1, 64, 64), (2, 6, 32, 32), (1, 4, 128, 256), (1, 2, 80, 32)])
def test_attend_long(gpu, seqs, kv, heads, dc, page):
    b = Batch(LONG[seqs], kv, dc, page, gpu, seed=8).fill()
    q = queries(b, heads, 2.0)
    got = b.dev().attend(q.to(gpu), *b.t)
    attend_check(b, heads, q.double().numpy(), got, (2 * dc) ** -0.5)


@pytest.mark.parametrize("size, scale", [(0.0, 1.0), (1e-3, 1.0), (100.0, 1.0), (1.0, 1e-30)])
@pytest.mark.parametrize("seqs", ["ragged", "long"])
def test_attend_flat_and_peaked(gpu, seqs, size, scale):
    """Equal weights, and one position taking all."""
    b = Batch(SEQS[seqs], 2, 64, 32, gpu, seed=9).fill()
    q = queries(b, 4, size)
    got = b.dev().attend(q.to(gpu), *b.t, scale=scale)
    attend_check(b, 4, q.double().numpy(), got, scale)


@pytest.mark.parametrize("seqs", [[(6, 40), (1, 33)], [(200, 200), (140, 300)]])
def test_later_nan_reaches_only_those_who_see_it(gpu, seqs):
    """A position that is not finite, appended in the middle of the new ones."""
    import torch
    b = Batch(seqs, 2, 64, 32, gpu, seed=10).fill()
    q = queries(b, 4)
    rope = rope_of(b.width * 32, 64, gpu)
    k, v = random_c(b.rng, b.N, 2, 64), random_c(b.rng, b.N, 2, 64)
    clean = b.dev()
    clean.append(dev(k, gpu), dev(v, gpu), *b.t, rope)
    want = clean.attend(q.to(gpu), *b.t)
    k[3, 0, 5] = np.nan        # row 3, key head 0: query heads 0 and 1
    v[4, 1, 60] = np.inf       # row 4, key head 1: query heads 2 and 3
    clean.append(dev(k, gpu), dev(v, gpu), *b.t, rope)
    got = clean.attend(q.to(gpu), *b.t)
    n0 = seqs[0][0]
    nan = torch.isnan(got).all(-1).all(-1).cpu()
    some = torch.isnan(got).any(-1).any(-1).cpu()
    expect = torch.zeros_like(nan)
    expect[3:n0, :2] = True
    expect[4:n0, 2:] = True
    assert torch.equal(nan, expect) and torch.equal(some, expect)
    assert torch.equal(got.cpu()[~expect], want.cpu()[~expect])


@pytest.mark.parametrize("seqs", [[(1, 90)], [(40, 90)], [(33, 33), (2, 64)]])
def test_missing_pages_are_not_seen(gpu, seqs):
    b = Batch(seqs, 2, 32, 32, gpu, seed=11).fill()
    b.table[0, 0] = -1
    if len(seqs) > 1:
        b.table[1] = b.n_pages  # nothing of it
    q = queries(b, 2)
    got = b.dev().attend(q.to(gpu), *b.t)
    attend_check(b, 2, q.double().numpy(), got, 64 ** -0.5)
    if len(seqs) > 1:
        assert (host(got)[:32] == 0).all() and (host(got)[33:] == 0).all()


def test_rows_longer_than_their_sequence_see_nothing(gpu):
    """len < rows: the rows before position 0 are zero, nothing faults."""
    b = Batch([(40, 40)], 1, 32, 32, gpu, seed=12).fill()
    b.dev()
    q = queries(b, 3)
    short = dev(np.array([10], np.int32), gpu)
    got = host(b.kvc.attend(q.to(gpu), b.t[0], b.t[1], short))
    assert (got[:30] == 0).all() and np.isfinite(got[30:]).all() and (got[30:] != 0).any()
    none = host(b.kvc.attend(q.to(gpu), b.t[0], b.t[1], dev(np.array([-5], np.int32), gpu)))
    assert (none == 0).all()
    far = host(b.kvc.attend(q.to(gpu), b.t[0], b.t[1], dev(np.array([2 ** 31 - 1], np.int32), gpu)))
    assert far.shape == got.shape  # bounded by the pages


def test_numbers_out_of_range_are_bounded(gpu):
    """cu_new past the rows or decreasing, lens and pages of any value: no call reads or writes outside."""
    import torch
    b = Batch([(4, 40), (4, 40), (4, 40)], 2, 32, 32, gpu, seed=13).fill()
    b.dev()
    rope = rope_of(64, 32, gpu)
    q, k, v = (random_c(b.rng, 12, 2, 32) for _ in range(3))
    for cu in ([0, 9, 5, 12], [-7, 4, 2 ** 31 - 1, 3], [12, 0, 12, 0], [5, 5, 5, 5]):
        for lens in ([2 ** 31 - 1, -2 ** 31, 40], [0, 3, 63]):
            t = (b.t[0], dev(np.array(cu, np.int32), gpu), dev(np.array(lens, np.int32), gpu))
            qr = b.kvc.append(dev(k, gpu), dev(v, gpu), *t, rope, q=dev(q, gpu))
            b.kvc.attend(torch.nan_to_num(qr), *t)
            b.kvc.read(*t, 12)
    torch.cuda.synchronize()


def test_past_32_bit_offsets(gpu):
    """Pages above 4 GiB of a cache."""
    import torch
    import paper_2512_02901_amd as f2
    b = Batch([(3, 70)], 2, 64, 32, gpu, seed=14, spare=0).fill()
    n = (5 << 30) // (2 * b.tile)
    data = torch.empty(n * 2 * b.tile, dtype=torch.uint8, device=gpu)
    big = f2.PagedKv(n, 32, 2, 64, data=data)
    far = np.array([[n - 1, n - 7, n - 100]], np.int32)
    small = b.dev()
    for m in range(3):
        data.view(n, -1)[int(far[0, m])] = b.data.view(b.n_pages, -1)[int(b.table[0, m])]
    t = (dev(far, gpu), *b.t[1:])
    rope = rope_of(96, 64, gpu)
    q, k, v = (random_c(b.rng, 3, h, 64) for h in (4, 2, 2))
    outs = [c.append(dev(k, gpu), dev(v, gpu), *tt, rope, q=dev(q, gpu)) for c, tt in ((small, b.t), (big, t))]
    assert torch.equal(outs[0], outs[1])
    assert torch.equal(small.attend(outs[0], *b.t), big.attend(outs[0], *t))
    for x, y in zip(small.read(*b.t, 3), big.read(*t, 3)):
        assert torch.equal(x, y)


def test_repeats_are_equal_and_streams_and_graphs_work(gpu):
    import torch
    b = Batch(LONG["decode_mixed"], 2, 64, 64, gpu, seed=15).fill()
    q = queries(b, 8).to(gpu)
    kv = b.dev()
    want = kv.attend(q, *b.t)
    for _ in range(5):
        assert torch.equal(kv.attend(q, *b.t), want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ws = torch.empty(kv.attend_workspace_bytes(b.N, len(b.seqs), 8), dtype=torch.uint8, device=gpu)
    out = torch.empty_like(q)
    with torch.cuda.stream(side):
        kv.attend(q, *b.t, out=out, workspace=ws)
    side.synchronize()
    assert torch.equal(out, want)
    # a captured step follows what the tensors hold
    rope = rope_of(b.width * 64, 64, gpu)
    k, v, raw = (dev(random_c(b.rng, b.N, h, 64), gpu) for h in (2, 2, 8))
    x, delta, gain = (dev(a, gpu) for a in norm_inputs(b.N, 64, 9))
    h, qi, xs = torch.empty_like(x), torch.empty((b.N, 64, 2), dtype=torch.int8, device=gpu), torch.empty(b.N, device=gpu)
    qr = torch.empty_like(q)

    def step():
        f2.add_rmsnorm_i8(x, gain, delta=delta, h_out=h, out=(qi, xs))
        kv.append(k, v, *b.t, rope, q=raw, q_out=qr)
        kv.attend(qr, *b.t, out=out, workspace=ws)

    import paper_2512_02901_amd as f2
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for shift in (0, 1, 7, 30):
        b.t[2].copy_(dev(np.maximum(b.lens - shift, b.cu[1:] - b.cu[:-1]), gpu))
        raw.mul_(1.0 + shift / 100)
        x.mul_(0.5)
        step()
        torch.cuda.synchronize()
        eager = out.clone(), qi.clone(), xs.clone()
        out.zero_()
        qi.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager[0]) and torch.equal(qi, eager[1]) and torch.equal(xs, eager[2])


# ---------------------------------------------------------------- refusals


def test_refusals(gpu):
    import torch
    import paper_2512_02901_amd as f2
    b = Batch([(2, 5)], 2, 32, 32, gpu, seed=16).fill()
    kv = b.dev()
    rope = rope_of(32, 32, gpu)
    k = torch.zeros((2, 64), dtype=torch.complex64, device=gpu)
    q = torch.zeros((2, 4, 32, 2), dtype=torch.bfloat16, device=gpu)

    def bad(kind, f, *a, **kw):
        with pytest.raises(kind):
            f(*a, **kw)

    for sizes in ((0, 32, 1, 32), (1, 31, 1, 32), (1, 48, 1, 32), (1, 32, 0, 32), (1, 32, 1, 24), (1, 32, 1, 144), (1, 32, 1, 0)):
        bad(ValueError, f2.PagedKv, *sizes)
    bad(ValueError, f2.PagedKv, b.n_pages, 32, 2, 32, data=b.data[:-1])
    bad(TypeError, f2.PagedKv, b.n_pages, 32, 2, 32, data=b.data.view(torch.int8))
    bad(ValueError, kv.append, k[:, :32], k, *b.t, rope)                   # one head
    bad(ValueError, kv.append, k, k[:1], *b.t, rope)                       # rows
    bad(TypeError, kv.append, k.real.contiguous(), k, *b.t, rope)
    bad(ValueError, kv.append, k.conj(), k, *b.t, rope)
    bad(ValueError, kv.append, k.t().contiguous().t(), k, *b.t, rope)      # columns contiguous
    bad(ValueError, kv.append, k[:1].expand(2, 64), k, *b.t, rope)         # rows overlap
    bad(ValueError, kv.append, k, k, *b.t, rope[:, :16])
    bad(ValueError, kv.append, k, k, *b.t, rope, q_out=q)
    bad(ValueError, kv.append, k, k, b.t[0], b.t[1][:1], b.t[2], rope)
    bad(TypeError, kv.append, k, k, b.t[0].long(), b.t[1], b.t[2], rope)
    bad(ValueError, kv.append, k, k, b.t[0].cpu(), b.t[1], b.t[2], rope)
    bad(ValueError, kv.attend, q[:, :3].contiguous(), *b.t)
    bad(ValueError, kv.attend, q[:, :, :16].contiguous(), *b.t)
    bad(TypeError, kv.attend, q.half(), *b.t)
    bad(ValueError, kv.attend, q.transpose(0, 1), *b.t)
    bad(f2.Fairy2iError, kv.attend, q, *b.t, scale=0.0)
    bad(f2.Fairy2iError, kv.attend, q, *b.t, scale=float("nan"))
    bad(f2.Fairy2iError, kv.attend, q[:0], *b.t)
    bad(f2.Fairy2iError, kv.attend, q, *b.t, workspace=torch.empty(64, dtype=torch.uint8, device=gpu))
    bad(ValueError, kv.read, *b.t, 2, out=(q, q))
    x = torch.zeros((2, 8), dtype=torch.complex64, device=gpu)
    g = torch.ones(16, device=gpu)
    bad(ValueError, f2.add_rmsnorm_i8, x, g[:8])
    bad(ValueError, f2.add_rmsnorm_i8, x, g, delta=x[:1])
    bad(TypeError, f2.add_rmsnorm_i8, x.real.contiguous(), g)
    bad(ValueError, f2.add_rmsnorm_i8, x.cpu(), g)
    bad(f2.Fairy2iError, f2.add_rmsnorm_i8, x, g, eps=0.0)
    bad(f2.Fairy2iError, f2.add_rmsnorm_i8, x[:0], g)
    bad(ValueError, f2.rope_table, 0, 4, device=gpu)
    bad(f2.Fairy2iError, f2.rope_table, 4, 4, base=-1.0, device=gpu)


# ------------------------------------------- more than one kernel's own edges


@pytest.mark.parametrize("extra", [0, 1024])
@pytest.mark.parametrize("kv, heads, dc, page", [(1, 2, 48, 32), (2, 2, 64, 96), (1, 3, 64, 32), (1, 2, 32, 64), (1, 1, 112, 32)])
def test_attend_row_tiles_and_rounds(gpu, kv, heads, dc, page, extra):
    """Rows on both sides of 16, 32 and 128 a sequence and in the mean, lengths
    past 64 tiles (2048 positions) and not of whole rounds, some pages missing."""
    b = Batch([(1 + extra, 1 + extra), (150, 2500), (17, 17), (128, 129), (1, 2177), (0, 300), (8, 2049), (33, 33)], kv, dc, page, gpu, seed=17).fill()
    b.table[1, 3] = -1
    b.table[1, -(-2400 // page)] = -1
    b.table[4, 1:5] = b.n_pages
    b.table[7] = -1
    q = queries(b, heads, 1.5)
    got = b.dev().attend(q.to(gpu), *b.t)
    attend_check(b, heads, q.double().numpy(), got, (2 * dc) ** -0.5)
    assert (host(got)[b.cu[7]:] == 0).all()


@pytest.mark.parametrize("n_seqs", [65, 130, 300])
def test_many_sequences(gpu, n_seqs):
    """More sequences than a wave has lanes; some empty, some without rows."""
    rng = np.random.default_rng(n_seqs)
    seqs = [(int(n), int(n + c)) for n, c in zip(rng.integers(0, 3, n_seqs), rng.integers(0, 90, n_seqs))]
    seqs[n_seqs // 2] = (1, 1700)
    b = Batch(seqs, 2, 32, 32, gpu, seed=18).fill()
    k, v, q = random_c(b.rng, b.N, 2, 32), random_c(b.rng, b.N, 2, 32), random_c(b.rng, b.N, 4, 32)
    rope = rope_of(b.width * 32, 32, gpu)
    qr = b.dev().append(dev(k, gpu), dev(v, gpu), *b.t, rope, q=dev(q, gpu))
    np.testing.assert_array_equal(host(b.data), expect_append(b, k, v, host(rope)))
    b.cache = host(b.data)
    got = b.kvc.attend(qr, *b.t)
    attend_check(b, 4, host(qr).astype(np.float64), got, 64 ** -0.5)
    rk, rv = b.kvc.read(*b.t, b.N)
    for i in (0, n_seqs // 2, n_seqs - 1):
        n, length = seqs[i]
        want = sv.read(b.cache, 32, 2, 32, b.table[i], length)[:, length - n:]
        np.testing.assert_array_equal(host(rk)[b.cu[i]:b.cu[i + 1]], want[0])
        np.testing.assert_array_equal(host(rv)[b.cu[i]:b.cu[i + 1]], want[1])


def test_scale_at_the_ends_of_its_range(gpu):
    b = Batch([(3, 300), (20, 40)], 1, 64, 32, gpu, seed=19).fill()
    q = queries(b, 2)
    b.dev()
    for scale in (1e-30, 1e30):
        got = host(b.kvc.attend(q.to(gpu), *b.t, scale=scale))
        assert np.isfinite(got).all()
    flat = b.kvc.attend(q.to(gpu), *b.t, scale=1e-30)
    attend_check(b, 2, q.double().numpy(), flat, 1e-30)
