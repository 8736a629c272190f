"""Widely-linear decoder layers serving several sequences at once.

Prompts of different lengths are taken in one pass, then every sequence
generates one position a step.  Between the widely-linear products stand the
serving operators: the residual addition with RMSNorm and int8 activations
(``add_rmsnorm_i8``), and the paged 4-bit cache that turns, stores and attends
(``PagedKv``).  Weights are seeded random matrices, quantised here; there is no
vocabulary: a step's input is the last position's own output.

    python examples/serve_batch.py --layers 4 --n 2048 --heads 32 --kv-heads 8 --prompts 700,33,1024 --steps 16
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2512_02901_amd as f2  # noqa: E402


def widely_linear(N, K, T, gen):
    """(codes_U, scales_U, codes_W, scales_W) of a random real 2N x 2K layer."""
    A = torch.randn(2 * N, 2 * K, generator=gen, device="cuda") * (2 * K) ** -0.5
    U, W = f2.to_widely_linear(A)
    return (*f2.quantize(U, T), *f2.quantize(W, T))


class Layer:
    """One decoder layer; its keys and values live in pages of a cache of its own."""

    def __init__(self, n, n_ff, heads, kv_heads, T, n_pages, page_size, gen):
        self.n, self.heads, self.dc = n, heads, n // heads
        kv = kv_heads * self.dc
        self.w = {name: widely_linear(N, K, T, gen) for name, N, K in
                  (("q", n, n), ("k", kv, n), ("v", kv, n), ("o", n, n), ("gate", n_ff, n), ("up", n_ff, n), ("down", n, n_ff))}
        self.norm_attn, self.norm_mlp = (1 + 0.1 * torch.randn(2 * n, generator=gen, device="cuda") for _ in range(2))
        self.kv = f2.PagedKv(n_pages, page_size, kv_heads, self.dc)

    def __call__(self, h, delta, batch, rope):
        """The residual stream h (updated in place) with delta still to be added
        to it -> the same pair after the layer."""
        _, z, scale = f2.add_rmsnorm_i8(h, self.norm_attn, delta=delta, h_out=h)
        q, k, v = (f2.wl_matmul(*self.w[name], z, scale) for name in "qkv")
        q = self.kv.append(k, v, *batch, rope, q=q)
        o = self.kv.attend(q, *batch).view(-1, self.n, 2)
        a = f2.wl_matmul(*self.w["o"], *f2.quantize_act_int8(o))
        _, z, scale = f2.add_rmsnorm_i8(h, self.norm_mlp, delta=a, h_out=h)
        g, u = (torch.view_as_real(f2.wl_matmul(*self.w[name], z, scale)) for name in ("gate", "up"))
        act = torch.view_as_complex(torch.nn.functional.silu(g) * u)
        return h, f2.wl_matmul(*self.w["down"], *f2.quantize_act_int8(act))


class Server:
    """Layers, and which pages each sequence has."""

    def __init__(self, layers, n, n_ff, heads, kv_heads, T, n_seqs, max_len, page_size=64, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.page_size, max_pages = page_size, -(-max_len // page_size)
        self.layers = [Layer(n, n_ff, heads, kv_heads, T, n_seqs * max_pages, page_size, gen) for _ in range(layers)]
        self.rope = f2.rope_table(max_len, n // heads)
        # pages are handed out as sequences grow; the table holds what they have
        self.free = torch.randperm(n_seqs * max_pages).tolist()
        self.pages = torch.full((n_seqs, max_pages), -1, dtype=torch.int32)
        self.lens = [0] * n_seqs

    def step(self, x, new):
        """x: complex64 [sum(new), n], the rows of new[i] further positions of
        sequence i one after the other -> their outputs."""
        for i, count in enumerate(new):
            for page in range(-(-self.lens[i] // self.page_size), -(-(self.lens[i] + count) // self.page_size)):
                self.pages[i, page] = self.free.pop()
            self.lens[i] += count
        cu = torch.tensor([0, *new]).cumsum(0).int()
        batch = [t.cuda() for t in (self.pages, cu, torch.tensor(self.lens, dtype=torch.int32))]
        h, delta = x.clone(), torch.zeros_like(x)
        for layer in self.layers:
            h, delta = layer(h, delta, batch, self.rope)
        return h + delta


def last_rows(new):
    return torch.tensor(new).cumsum(0).sub(1).cuda()


def run(layers=2, n=512, n_ff=1408, heads=8, kv_heads=4, T=2, prompts=(70, 5, 129), steps=4, seed=0, log=print):
    """Generates `steps` positions behind each prompt, and then takes the same
    positions in one pass through a second server: returns how far the two
    differ (2-norm over 2-norm) in the last step's outputs."""
    dims = dict(layers=layers, n=n, n_ff=n_ff, heads=heads, kv_heads=kv_heads, T=T, n_seqs=len(prompts),
                max_len=max(prompts) + steps + 1, seed=seed)
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    x = torch.randn(sum(prompts), n, dtype=torch.complex64, generator=gen, device="cuda")
    server = Server(**dims)
    seen = [list(part) for part in x.split(list(prompts))]

    def timed(f, what, tokens):
        torch.cuda.synchronize()
        t = time.perf_counter()
        y = f()
        torch.cuda.synchronize()
        log(f"{what}: {tokens} positions in {1e3 * (time.perf_counter() - t):.2f} ms")
        return y

    y = timed(lambda: server.step(x, list(prompts)), "prompts", len(x))[last_rows(prompts)]
    ones = [1] * len(prompts)
    for s in range(steps):
        y = y / y.abs().square().mean(1, keepdim=True).sqrt()
        for rows, row in zip(seen, y):
            rows.append(row)
        y = timed(lambda: server.step(y, ones), f"step {s}", len(y))
    del server
    again = Server(**dims).step(torch.stack([row for rows in seen for row in rows]), [len(rows) for rows in seen])
    want = again[last_rows([len(rows) for rows in seen])]
    off = float((y - want).norm() / want.norm())
    log(f"one position at a time against all at once: {off:.2e}")
    return off


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--n", type=int, default=512, help="complex width")
    ap.add_argument("--n-ff", type=int, default=0, help="complex width of gate and up (2.75 n by default)")
    ap.add_argument("--heads", type=int, default=8)
    ap.add_argument("--kv-heads", type=int, default=4)
    ap.add_argument("--stages", type=int, default=2)
    ap.add_argument("--prompts", default="70,5,129", help="lengths")
    ap.add_argument("--steps", type=int, default=4)
    a = ap.parse_args()
    run(a.layers, a.n, a.n_ff or a.n * 11 // 4 // 64 * 64, a.heads, a.kv_heads, a.stages,
        tuple(int(p) for p in a.prompts.split(",")), a.steps)


if __name__ == "__main__":
    main()
