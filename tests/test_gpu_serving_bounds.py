"""The serving operators at the ends of what their arrays may say: lengths past
the page table, rows past the tensors, positions that nobody stored.  The
expectations are oracle/serving.py's, or a call's own for arrays that name the
same rows and positions; tolerances are tests/test_gpu_serving.py's."""
import numpy as np
import pytest

from oracle import serving as sv
from test_gpu_serving import Batch, attend_check, dev, expect_append, host, queries, random_c, rope_of

pytestmark = pytest.mark.gpu


def same(x, y):
    """Equal bit for bit, a NaN to any NaN."""
    import torch
    return torch.equal(torch.isnan(x), torch.isnan(y)) and torch.equal(torch.nan_to_num(x), torch.nan_to_num(y))


# ------------------------------------------------ lengths past the page table

CAPACITY = 192
PAST = {
    "one_past": [(1, CAPACITY + 1)],
    "three_around": [(3, CAPACITY + 1)],
    "some_past": [(1, CAPACITY), (3, CAPACITY + 2), (1, CAPACITY + 1), (0, CAPACITY + 9), (5, CAPACITY + 300), (2, 7)],
    "prompt": [(CAPACITY + 70, CAPACITY + 70)],
    "prompts": [(150, CAPACITY + 31), (170, 170)],
}


@pytest.mark.parametrize("seqs", list(PAST))
@pytest.mark.parametrize("kv, heads, dc, page", [(3, 3, 16, 32), (2, 4, 32, 64), (1, 2, 48, 96), (2, 4, 64, 32), (1, 4, 128, 192)])
def test_rows_past_the_table_are_left_out(gpu, seqs, kv, heads, dc, page):
    """They are not stored, their q and what is read of them are NaN, and the
    other rows stand where they stand: a call with a wider table without pages there."""
    import torch
    b = Batch(PAST[seqs], kv, dc, page, gpu, seed=31).fill()
    width = CAPACITY // page
    b.table[:, width:] = -1
    b.dev()
    t = (dev(b.table[:, :width], gpu), *b.t[1:])
    rope = rope_of(b.width * page, dc, gpu)
    q, k, v = (random_c(b.rng, b.N, h, dc) for h in (heads, kv, kv))
    got_q = b.kvc.append(dev(k, gpu), dev(v, gpu), *t, rope, q=dev(q, gpu))
    np.testing.assert_array_equal(host(b.data), expect_append(b, k, v, host(rope)))
    pos = np.concatenate([np.arange(c - n, c) for n, c in b.seqs])
    inside = pos < CAPACITY
    nan = np.isnan(host(got_q))
    assert nan[~inside].all() and not nan[inside].any()
    turn = host(rope)
    want_q = sv.rotate(q, turn[pos][:, None, :, 0], turn[pos][:, None, :, 1])
    assert torch.equal(got_q.cpu()[inside], torch.from_numpy(want_q).bfloat16()[inside])
    out = tuple(torch.full((b.N, kv, dc, 2), 7.0, dtype=torch.bfloat16, device=gpu) for _ in range(2))
    b.kvc.read(*t, b.N, out=out)
    for i, (n, length) in enumerate(b.seqs):
        want = sv.read(host(b.data), page, kv, dc, b.table[i], length)[:, length - n:]
        np.testing.assert_array_equal(host(out[0])[b.cu[i]:b.cu[i + 1]], want[0])
        np.testing.assert_array_equal(host(out[1])[b.cu[i]:b.cu[i + 1]], want[1])
    b.cache = host(b.data)
    qb = queries(b, heads)
    attend_check(b, heads, qb.double().numpy(), b.kvc.attend(qb.to(gpu), *t), (2 * dc) ** -0.5)


@pytest.mark.parametrize("length", [2 ** 31 - 1, 2 ** 31 - 2, 2 ** 30 + 64])
def test_far_lengths_touch_nothing(gpu, length):
    """A length that no table holds: nothing is stored, and the rows see all that there is."""
    b = Batch([(40, 64)], 2, 32, 32, gpu, seed=32).fill()
    b.dev()
    t = (*b.t[:2], dev(np.array([length], np.int32), gpu))
    q, k, v = (random_c(b.rng, 40, 2, 32) for _ in range(3))
    rope = rope_of(64, 32, gpu)
    assert np.isnan(host(b.kvc.append(dev(k, gpu), dev(v, gpu), *t, rope, q=dev(q, gpu)))).all()
    np.testing.assert_array_equal(host(b.data), b.cache)
    for x in b.kvc.read(*t, 40):
        assert np.isnan(host(x)).all()
    qb = queries(b, 4)
    got = host(b.kvc.attend(qb.to(gpu), *t)).astype(np.float64)
    k, v = sv.read(b.cache, 32, 2, 32, b.table[0], 64)
    want, size, most = sv.attend(qb.double().numpy(), k, v, 64, 64 ** -0.5)
    assert (np.abs(got - want) <= (2.0 ** -8 + 2.0 ** -18 * most) * size + 1e-37).all()


@pytest.mark.parametrize("cu, rows, as_cu", [([0, 3, 9], 7, [0, 3, 7]), ([-2, 3, 7], 7, [0, 3, 7]),
                                             ([0, 3, 2 ** 31 - 101], 7, [0, 3, 7]), ([0, 140, 300], 290, [0, 140, 290])])
@pytest.mark.parametrize("dc", [32, 64])
def test_rows_past_the_tensors_leave_the_others_in_place(gpu, cu, rows, as_cu, dc):
    """cu_new beyond the rows that q, k and v have: row j of a sequence still stands at lens - rows + j."""
    import torch
    n = [b - a for a, b in zip(as_cu, as_cu[1:])]
    b = Batch([(n[0], n[0] + 20), (n[1], n[1] + 33)], 2, dc, 32, gpu, seed=33).fill()
    q, k, v = (dev(random_c(b.rng, rows, 2, dc), gpu) for _ in range(3))
    rope = rope_of(b.width * 32, dc, gpu)
    results = []
    for starts in (as_cu, cu):
        b.dev()
        lens = (b.lens + (np.array(starts[1:], np.int64) - as_cu[1:])).astype(np.int32)
        t = (b.t[0], dev(np.array(starts, np.int32), gpu), dev(lens, gpu))
        qr = b.kvc.append(k, v, *t, rope, q=q)
        results.append((b.data, qr, b.kvc.attend(qr, *t), *b.kvc.read(*t, rows)))
    for x, y in zip(*results):
        assert same(x, y)
    assert not torch.isnan(results[0][2]).any()


# ----------------------------------------------- positions that nobody stored


@pytest.mark.parametrize("byte", [0xFF, 0xFE, 0xFD])
@pytest.mark.parametrize("seqs, stored", [([(40, 40)], 21), ([(1, 30), (30, 60)], 45), ([(200, 200)], 150), ([(170, 300), (140, 170)], 161)])
@pytest.mark.parametrize("kv, heads, dc, page", [(2, 2, 16, 32), (1, 3, 32, 64), (2, 2, 48, 32), (1, 2, 64, 64), (1, 2, 128, 32)])
def test_unstored_positions_reach_no_earlier_row(gpu, kv, heads, dc, page, seqs, stored, byte):
    """Rows past the rotation table are not stored: what their positions held
    before (codes and scales of NaN and infinities) is not in the rows before them."""
    import torch
    b = Batch(seqs, kv, dc, page, gpu, seed=34)
    b.cache[:] = byte
    b.dev()
    q, k, v = (random_c(b.rng, b.N, h, dc) for h in (heads, kv, kv))
    # what stands before the new rows, then the rows as far as the table goes
    before = [length - n for n, length in seqs]
    rope = rope_of(b.width * page, dc, gpu)
    old = [random_c(b.rng, sum(before), kv, dc) for _ in range(2)]
    cu = np.concatenate([[0], np.cumsum(before)]).astype(np.int32)
    if sum(before):
        b.kvc.append(*(dev(x, gpu) for x in old), b.t[0], dev(cu, gpu), dev(np.array(before, np.int32), gpu), rope)
    qr = b.kvc.append(dev(k, gpu), dev(v, gpu), *b.t, rope[:stored].contiguous(), q=dev(q, gpu))
    got = b.kvc.attend(qr, *b.t)
    pos = np.concatenate([np.arange(c - n, c) for n, c in seqs])
    late = torch.from_numpy(pos >= stored)
    assert late.any() and torch.isnan(got.cpu()[late]).all()
    # the rows that are stored, as a call of their own over the clean cache
    few = [(max(0, min(c, stored) - (c - n)), min(c, max(stored, c - n))) for n, c in seqs]
    b.cache, b.seqs = host(b.data), few
    b.cu = np.concatenate([[0], np.cumsum([n for n, _ in few])]).astype(np.int32)
    attend_check(b, heads, host(qr)[~late.numpy()].astype(np.float64), got.cpu()[~late], (2 * dc) ** -0.5)


# ------------------------------------------------------ a cu_new that decreases


def fenced(n, gpu, pad=1 << 16):
    """n bytes between two runs of `pad` marked ones: (all of them, the n)."""
    import torch
    whole = torch.full((n + 2 * pad,), 0xA5, dtype=torch.uint8, device=gpu)
    return whole, whole[pad:pad + n]


def fences_stand(whole, n):
    pad = (whole.numel() - n) // 2
    return bool((whole[:pad] == 0xA5).all()) and bool((whole[pad + n:] == 0xA5).all())


def test_counts_that_wrap_stay_in_the_workspace(gpu):
    """Half a million times the same 4096 rows (cu_new goes up and down): the work
    counted over the sequences passes 2^31, the last one's numbers with it."""
    import torch
    import paper_2512_02901_amd as f2
    n_seqs, rows, heads, pages = 1 << 20, 4096, 24, 10
    kv = f2.PagedKv(pages, 32, 1, 16, data=torch.zeros(f2.PagedKv.bytes(pages, 32, 1, 16), dtype=torch.uint8, device=gpu))
    cu = torch.zeros(n_seqs + 1, dtype=torch.int32, device=gpu)
    cu[1::2] = rows
    lens = torch.zeros(n_seqs, dtype=torch.int32, device=gpu)
    lens[n_seqs - 2] = 320  # the last one with rows: more than one chunk
    table = torch.arange(pages, dtype=torch.int32, device=gpu).expand(n_seqs, pages).contiguous()
    q = torch.ones((rows, heads, 16, 2), dtype=torch.bfloat16, device=gpu)
    need = kv.attend_workspace_bytes(rows, n_seqs, heads)
    ws, mid = fenced(need, gpu)
    buf, out = fenced(q.numel() * 2, gpu)
    kv.attend(q, table, cu, lens, out=out.view(torch.bfloat16).view(q.shape), workspace=mid)
    assert fences_stand(ws, need) and fences_stand(buf, q.numel() * 2)
    assert (host(kv.data) == 0).all()


# --------------------------------------------------- more than a launch takes


@pytest.mark.parametrize("B, n", [((1 << 24) + 7, 1), ((1 << 26) + 7, 4)])
def test_norm_of_more_tokens_than_a_launch_takes(gpu, B, n):
    """2^32 threads and more: the same tokens over and over give the same results."""
    import torch
    import paper_2512_02901_amd as f2
    few = 4099
    rng = np.random.default_rng(n)
    x = dev(random_c(rng, few, n), gpu)
    gain = dev((1 + 0.1 * rng.standard_normal(2 * n)).astype(np.float32), gpu)
    want = f2.add_rmsnorm_i8(x, gain, delta=x)
    again = -(-B // few)
    many = x.repeat(again, 1)[:B]
    got = f2.add_rmsnorm_i8(many, gain, delta=many)
    for w, g in zip(want, got):
        whole = B // few * few
        assert (g[:whole].view(-1, *w.shape) == w).all()
        assert torch.equal(g[whole:], w[:B - whole])
    del many, got
    torch.cuda.empty_cache()


def test_rope_table_of_more_entries_than_a_launch_takes(gpu):
    import torch
    n, dc = 1 << 20, 4096
    got = rope_of(n, dc, gpu)
    for p in (0, 1, 77777, n // 2, n - 2, n - 1):
        angle = p * 10000.0 ** (-np.arange(dc) / dc)
        # the angle is off by some 2^-51 of itself
        np.testing.assert_allclose(host(got[p]), np.stack([np.cos(angle), np.sin(angle)], -1), rtol=0, atol=2.0 ** -24 + 2.0 ** -30)
    del got
    torch.cuda.empty_cache()


# ------------------------------------------------------ tensors at any element


def placed(t, off):
    """t at `off` elements past a 512-byte boundary."""
    import torch
    buf = torch.empty(t.numel() + off, dtype=t.dtype, device=t.device)
    out = buf[off:].view(t.shape)
    out.copy_(t)
    assert out.is_contiguous() and out.data_ptr() % 512 == off * t.element_size()
    return out


@pytest.mark.parametrize("off", [1, 2, 5])
@pytest.mark.parametrize("seqs", [[(1, 40), (3, 1500)], [(150, 170), (140, 900)]])
@pytest.mark.parametrize("kv, heads, dc", [(2, 4, 32), (1, 4, 64), (1, 2, 128)])
def test_tensors_at_any_element(gpu, kv, heads, dc, seqs, off):
    import torch
    b = Batch(seqs, kv, dc, 32, gpu, seed=35).fill()
    q, k, v = (dev(random_c(b.rng, b.N, h, dc), gpu) for h in (heads, kv, kv))
    rope = rope_of(b.width * 32, dc, gpu)
    b.dev()
    qr = b.kvc.append(k, v, *b.t, rope, q=q)
    want = (b.data, qr, b.kvc.attend(qr, *b.t), *b.kvc.read(*b.t, b.N))
    b.dev()
    got_q = b.kvc.append(placed(k, off), placed(v, off), *b.t, placed(rope, off), q=placed(q, off),
                         q_out=placed(torch.zeros_like(qr), off))
    out = b.kvc.attend(got_q, *b.t, out=placed(torch.zeros_like(qr), off + 1))
    both = tuple(placed(torch.zeros_like(x), off) for x in want[3:])
    b.kvc.read(*b.t, b.N, out=both)
    for x, y in zip(want, (b.data, got_q, out, *both)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("off", [1, 3, 8])
@pytest.mark.parametrize("n", [64, 1500, 77])
def test_norm_into_any_byte(gpu, n, off):
    import torch
    import paper_2512_02901_amd as f2
    rng = np.random.default_rng(n)
    x, gain = dev(random_c(rng, 5, n), gpu), dev(rng.standard_normal(2 * n).astype(np.float32), gpu)
    h, q, s = f2.add_rmsnorm_i8(x, gain, delta=x)
    q0, s0 = placed(torch.zeros_like(q), off), placed(torch.zeros_like(s), off)
    f2.add_rmsnorm_i8(placed(x, off), placed(gain, off), delta=placed(x, off), h_out=placed(h, off), out=(q0, s0))
    assert torch.equal(q, q0) and torch.equal(s, s0)


# ------------------------------------------- numbers of any value, memory around


def in_fences(t, gpu):
    """A copy of t between two marked runs: (all bytes, the copy)."""
    import torch
    whole, mid = fenced(t.numel() * t.element_size(), gpu)
    out = mid.view(t.dtype).view(t.shape)
    out.copy_(t)
    return whole, out


@pytest.mark.parametrize("n, heads, dc", [(4, 2, 32), (4, 4, 64), (150, 2, 48), (150, 2, 16)])
def test_numbers_out_of_range_write_nothing_outside(gpu, n, heads, dc):
    """Whatever cu_new, lens and pages hold: the bytes around every output, around
    the workspace and of pages that no table names stay, and so do the inputs."""
    import torch
    import paper_2512_02901_amd as f2
    b = Batch([(n, 2 * n + 40)] * 3, 2, dc, 32, gpu, seed=36, spare=5).fill()
    N = b.N
    rope = rope_of(b.width * 32, dc, gpu)
    q, k, v = (dev(random_c(b.rng, N, h, dc), gpu) for h in (heads, 2, 2))
    inputs = [x.clone() for x in (q, k, v, rope)]
    qb = torch.zeros((N, heads, dc, 2), dtype=torch.bfloat16, device=gpu)
    kb = torch.zeros((N, 2, dc, 2), dtype=torch.bfloat16, device=gpu)
    named = np.unique(b.table[b.table >= 0])
    spare = np.setdiff1d(np.arange(b.n_pages), named)
    tables = [b.table.copy() for _ in range(2)]
    tables[1][0, ::2], tables[1][0, 1::2] = -1, b.n_pages
    tables[1][1, ::2], tables[1][2, 0] = 2 ** 31 - 1, -2 ** 31
    far = 2 ** 31 - 1
    for cu in ([0, 2 * n + 1, n + 1, 3 * n], [-7, n, far, n - 1], [3 * n, 0, 3 * n, 0], [5, 5, 5, 5], [-far, far, -far, far]):
        for lens in ([far, -far - 1, 40], [0, 3, 63], [b.width * 32 + 1, b.width * 32 - 1, n]):
            for table in tables:
                t = tuple(dev(np.array(a, np.int32), gpu) for a in (table, cu, lens))
                whole, data = in_fences(dev(b.cache, gpu), gpu)
                kv = f2.PagedKv(b.n_pages, 32, 2, dc, data=data)
                w1, q_out = in_fences(qb, gpu)
                qr = kv.append(k, v, *t, rope, q=q, q_out=q_out)
                w2, out = in_fences(qb, gpu)
                need = kv.attend_workspace_bytes(N, 3, heads)
                w3, ws = fenced(need, gpu)
                kv.attend(torch.nan_to_num(qr), *t, out=out, workspace=ws)
                (w4, rk), (w5, rv) = in_fences(kb, gpu), in_fences(kb, gpu)
                kv.read(*t, N, out=(rk, rv))
                for w, size in ((whole, data.numel()), (w1, 2 * qb.numel()), (w2, 2 * qb.numel()), (w3, need),
                                (w4, 2 * kb.numel()), (w5, 2 * kb.numel())):
                    assert fences_stand(w, size), (cu, lens)
                pages = host(data).reshape(b.n_pages, -1)
                np.testing.assert_array_equal(pages[spare], b.cache.reshape(b.n_pages, -1)[spare])
    for x, y in zip((q, k, v, rope), inputs):
        assert torch.equal(x, y)


PLANS = {
    "decode": [(1, 40), (1, 3000), (0, 0), (1, 700)],
    "verify": [(5, 1300), (3, 700)],
    "prompt": [(300, 300)],
    "prompts": [(140, 2000), (200, 260), (1, 900)],
}


@pytest.mark.parametrize("seqs", list(PLANS))
@pytest.mark.parametrize("kv, heads, dc", [(2, 2, 16), (1, 4, 32), (2, 2, 48), (1, 3, 64), (1, 2, 128)])
def test_workspace_and_output_memory(gpu, kv, heads, dc, seqs):
    """A workspace of exactly the bytes asked for, holding anything, and an output
    in q's own memory give what a call of its own gives."""
    import torch
    b = Batch(PLANS[seqs], kv, dc, 32, gpu, seed=37).fill()
    q = queries(b, heads).to(gpu)
    kvc = b.dev()
    want = kvc.attend(q, *b.t)
    need = kvc.attend_workspace_bytes(b.N, len(b.seqs), heads)
    for byte in (0x00, 0x7F, 0xFF):
        whole, ws = fenced(need, gpu)
        ws.fill_(byte)
        whole_out, out = in_fences(q, gpu)
        kvc.attend(out, *b.t, out=out, workspace=ws)
        assert torch.equal(out, want)
        assert fences_stand(whole, need) and fences_stand(whole_out, 2 * q.numel())


# --------------------------------------- plans that short sequences never reach


def sampled_check(b, heads, q, got, scale, every):
    """attend_check's bound for every `every`-th row of each sequence and its last."""
    got = host(got).astype(np.float64)
    for i, (n, length) in enumerate(b.seqs):
        k, v = sv.read(b.cache, b.page, b.kv, b.dc, b.table[i], length)
        for j in sorted({*range(0, n, every), n - 1}):
            want, size, most = sv.attend(q[b.cu[i] + j:b.cu[i] + j + 1], k, v, length - n + j, scale)
            d = np.abs(got[b.cu[i] + j:b.cu[i] + j + 1] - want)
            assert (d <= (2.0 ** -8 + 2.0 ** -18 * most) * size + 1e-37).all(), (i, j)


# more than 64 chunks of 8 tiles a row (a block joins each row); chunks longer than
# the least, by one row block and by two; 336 and 512 items of 128 rows, whose second
# half goes the other way round
@pytest.mark.parametrize("seqs, kv, heads, dc, every", [
    ([(1, 17000)], 1, 2, 64, 1), ([(3, 17111), (1, 20)], 1, 2, 16, 1), ([(1, 16700)], 1, 3, 128, 1), ([(2, 17300)], 1, 1, 48, 1),
    ([(100, 3000)] * 8, 2, 2, 16, 37), ([(1, 8200)] * 2, 17, 17, 16, 1),
    ([(1200, 4000)] * 2, 2, 4, 32, 173),
    ([(700, 700), (600, 650)], 8, 16, 64, 83), ([(2048, 2048)], 8, 8, 64, 293)])
def test_plans_of_long_calls(gpu, seqs, kv, heads, dc, every):
    b = Batch(seqs, kv, dc, 64, gpu, seed=38)
    at = 64 * dc
    c = b.cache.reshape(-1, b.tile)
    c[:, at:] = np.clip(np.round(127 + 0.7 * b.rng.standard_normal(c[:, at:].shape)), 2, 252)
    q = queries(b, heads)
    got = b.dev().attend(q.to(gpu), *b.t)
    sampled_check(b, heads, q.double().numpy(), got, (2 * dc) ** -0.5, every)


# ------------------------------------------------------------------ midpoints


def midpoint_block(e, sign):
    """32 reals of scale 2^e (dtype float32): every midpoint between two e2m1 values, the
    floats next to it, and a largest value that asks for that scale."""
    mid = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], np.float32)
    v = np.concatenate([mid, np.nextafter(mid, np.float32(9)), np.nextafter(mid, np.float32(0)), -mid,
                        np.array([7.0, 6.0, 0.0, -0.0], np.float32)])
    return np.ldexp(v * np.float32(sign), e).astype(np.float32)


@pytest.mark.parametrize("dc", [16, 64, 80])
def test_midpoints_round_to_the_even_code(gpu, dc):
    """Keys at position 0 (turned by nothing) and values, at scales over the whole range."""
    n, nb = 63, dc // 16
    b = Batch([(1, 1)] * n, 2, dc, 32, gpu, seed=39)
    es = np.linspace(-122, 124, n * 2 * nb).astype(int)  # the smallest neighbours stay normal numbers
    x = np.stack([midpoint_block(e, 1 - 2 * (i % 2)) for i, e in enumerate(es)])
    k = x.reshape(n, 2, dc, 2)
    v = x[::-1].reshape(n, 2, dc, 2)
    k, v = (np.ascontiguousarray(t).view(np.complex64)[..., 0] for t in (k, v))
    rope = rope_of(32, dc, gpu)
    assert (host(rope[0]) == [1, 0]).all()
    b.dev().append(dev(k, gpu), dev(v, gpu), *b.t, rope)
    np.testing.assert_array_equal(host(b.data), expect_append(b, k, v, host(rope)))
