"""How exactly attention weighs: its bound against oracle/serving.py in 64 bits, and
that weights of one bf16 number would break it.

Before its rounding to bf16 (2^-8 of itself) an output is off by at most E A, A =
sum p |v|, with S = scale * sum |q||k| over a head's 2 dc reals, L positions:
- a weight enters as two bf16 numbers, of which the second one's rounding is lost:
  2^-8 of 2^-8 of it, 2^-16;
- the weighted sum adds 2 L products and the weights' sum L numbers in float32; 2^-24
  for each addition of either, twice that for the matrix cores' own order: L 2^-21;
- a score adds 2 dc products, dc 2^-22 S with the same allowance; its scale, the
  difference to the reference, their product and the exponential are four
  roundings of a number up to 2 S log2(e) + 8: 2^-20 (S + 3).  A weight changes by that
  factor, and the sum of the weights as well: twice.
"""
import numpy as np
import pytest

from oracle import serving as sv
from test_gpu_serving import Batch, bf16, host, queries


def bound(want, size, most, length, dc):
    E = 2.0 ** -16 + length * 2.0 ** -21 + 2 * (dc * 2.0 ** -22 * most + 2.0 ** -20 * (most + 3))
    return 2.0 ** -8 * np.abs(want) + (1 + 2.0 ** -8) * E * size + 1e-37


CASES = [([(1, 64)], 2, 8, 64), ([(40, 90)], 2, 4, 64), ([(140, 140)], 2, 2, 64), ([(150, 160)], 1, 2, 48),
         ([(17, 60), (3, 33)], 1, 4, 128), ([(140, 150)], 2, 4, 32), ([(5, 100)], 2, 4, 16), ([(300, 300)], 1, 1, 16)]


def batch(seqs, kv, heads, dc, gpu=None):
    b = Batch(seqs, kv, dc, 32, gpu, seed=51).fill()
    return b, queries(b, heads, 0.25)


def exact(b, q, dc):
    for i, (n, length) in enumerate(b.seqs):
        k, v = sv.read(b.cache, b.page, b.kv, dc, b.table[i], length)
        rows = slice(b.cu[i], b.cu[i + 1])
        yield i, rows, k, v, length, sv.attend(q[rows], k, v, length - (b.cu[i + 1] - b.cu[i]), (2 * dc) ** -0.5)


@pytest.mark.gpu
@pytest.mark.parametrize("seqs, kv, heads, dc", CASES)
def test_weights_of_two_parts(gpu, seqs, kv, heads, dc):
    b, q = batch(seqs, kv, heads, dc, gpu)
    got = host(b.dev().attend(q.to(gpu), *b.t)).astype(np.float64)
    for i, rows, _, _, length, (want, size, most) in exact(b, q.double().numpy(), dc):
        assert (np.abs(got[rows] - want) <= bound(want, size, most, length, dc)).all()


@pytest.mark.parametrize("seqs, kv, heads, dc", CASES)
def test_the_bound_tells_one_part_from_two(seqs, kv, heads, dc):
    """The oracle's own sums with its weights rounded to bf16 once, and as two parts."""
    b, q = batch(seqs, kv, heads, dc)
    q = q.double().numpy()
    one_part_in = True
    for i, rows, k, v, length, (want, size, most) in exact(b, q, dc):
        n, scale = rows.stop - rows.start, (2 * dc) ** -0.5
        for parts in (1, 2):
            got = np.zeros_like(want)
            for j in range(n):
                seen = length - n + j + 1
                for h in range(heads):
                    kk, vv = k[:seen, h * kv // heads], v[:seen, h * kv // heads]
                    p = np.exp(scale * np.tensordot(kk, q[rows][j, h], 2))
                    p /= p.max()
                    w = bf16(p).double().numpy()
                    if parts == 2:
                        w += bf16(p - w).double().numpy()
                    got[j, h] = np.tensordot(w, vv, 1) / p.sum()
            got = bf16(got).double().numpy()
            ok = (np.abs(got - want) <= bound(want, size, most, length, dc)).all()
            if parts == 2:
                assert ok
            else:
                one_part_in &= ok
    assert not one_part_in
