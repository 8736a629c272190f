"""The gradient of the training norm (layernorm_backward) where its sums are long.
Tolerances, from the arithmetic (u = 2^-24, half a step of float32):

sums over   of up to 8192 entries: float32 over at most 64 tokens of a team, 7
tokens      additions to join a block's teams, then double and one rounding: 72 u
            of the sum of |dz y|; of more entries: double, one rounding of a
            block's part and one of the result, 2 u.
"""
import numpy as np
import pytest

from test_gpu_training import host

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
