"""The attention half of a decoder layer on this library alone: q/k/v products of packed matrices, norms and rotation, a 4-bit
cache, attention, o product -- for packed prompts and for token generation.

    python3 -m paper_2412_17560_amd.attention_layer [--hidden 4096] [--heads 32] [--kv-heads 8] [--prompts 700,15,2048] [--tokens 64]

runs prompts of these lengths, then generates tokens for all of them with one captured HIP graph, on random weights, and prints what each
phase took and what the cache holds.
"""
from __future__ import annotations

import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

MOST_ROWS = 16          # of a product


class AttentionLayer:
    """q, k, v, o: packed matrices (gqsa_pack ...); q_norm, k_norm: float16 [head_dim] or None; table: float32 [positions,
    rotary_dim / 2, 2]; cache: from gqsa_cache_create, for k's heads."""

    def __init__(self, q, k, v, o, heads: int, table, cache, q_norm=None, k_norm=None, eps: float = 1e-6):
        self.q, self.k, self.v, self.o = q, k, v, o
        self.heads, self.kv_heads, self.head_dim = heads, cache.kv_heads, cache.head_dim
        self.table, self.cache, self.norms, self.eps = table, cache, (q_norm, k_norm), eps

    def _products(self, handles, x):
        import torch

        import paper_2412_17560_amd as gq
        ys = [torch.empty((x.shape[0], gq.gqsa_info(h)["N"]), dtype=torch.float16, device=x.device) for h in handles]
        for r in range(0, x.shape[0], MOST_ROWS):
            gq.gqsa_gemv_multi(handles, x[r:r + MOST_ROWS], [y[r:r + MOST_ROWS] for y in ys])
        return ys

    def _queries_keys_values(self, x, positions):
        import paper_2412_17560_amd as gq
        q, k, v = self._products([self.q, self.k, self.v], x)
        q = q.view(-1, self.heads, self.head_dim)
        k, v = (t.view(-1, self.kv_heads, self.head_dim) for t in (k, v))
        gq.gqsa_qk_norm_rotate(q, k, positions, self.table, *self.norms, eps=self.eps, q_out=q, k_out=k)
        return q, k, v

    def prompt(self, x, positions, pages, starts, lengths):
        """Rows x [rows, hidden] of packed prompts (sequence b: starts[b] .. starts[b + 1] - 1, all of its lengths[b] tokens)."""
        import paper_2412_17560_amd as gq
        q, k, v = self._queries_keys_values(x, positions)
        gq.gqsa_cache_append(self.cache, k, v, pages, lengths, starts)
        attended = gq.gqsa_prompt_attend(q, k, v, starts, starts)
        return self._products([self.o], attended.view(x.shape[0], self.heads * self.head_dim))[0]

    def step(self, x, positions, pages, lengths):
        """One new row for every sequence; lengths counts it in."""
        import paper_2412_17560_amd as gq
        q, k, v = self._queries_keys_values(x, positions)
        gq.gqsa_cache_append(self.cache, k, v, pages, lengths)
        attended = gq.gqsa_cache_attend(self.cache, q, pages, lengths)
        return self._products([self.o], attended.view(x.shape[0], self.heads * self.head_dim))[0]


def rotary_table(positions: int, rotary_dim: int, theta: float = 10000.0):
    """float32 [positions, rotary_dim / 2, 2] on the device: cosine and sine of position * theta^(-2 i / rotary_dim)."""
    import torch
    i = torch.arange(0, rotary_dim, 2, device="cuda", dtype=torch.float64)
    angle = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * theta ** (-i / rotary_dim)
    return torch.stack([angle.cos(), angle.sin()], dim=-1).float()


def main() -> None:
    p = argparse.ArgumentParser()
    p.add_argument("--hidden", type=int, default=4096)
    p.add_argument("--heads", type=int, default=32)
    p.add_argument("--kv-heads", type=int, default=8)
    p.add_argument("--head-dim", type=int, default=128, choices=(64, 128))
    p.add_argument("--prompts", default="700,15,2048", help="lengths of the prompts (up to 16 of them)")
    p.add_argument("--tokens", type=int, default=64, help="1 or more: a step without the graph, then one replay fewer than this")
    p.add_argument("--sparsity", type=float, default=0.5)
    args = p.parse_args()
    if args.tokens < 1:
        p.error("--tokens must be 1 or more")

    import torch

    import paper_2412_17560_amd as gq

    torch.cuda.set_device(0)
    gen = torch.Generator(device="cuda").manual_seed(0)
    dim, counts = args.head_dim, [int(n) for n in args.prompts.split(",")]
    sizes = [(args.heads * dim, args.hidden), (args.kv_heads * dim, args.hidden), (args.kv_heads * dim, args.hidden), (args.hidden, args.heads * dim)]
    matrices = [gq.gqsa_pack_device(torch.randn(s, generator=gen, device="cuda") / s[1] ** 0.5, 16, 4, args.sparsity) for s in sizes]
    page = 64
    per_sequence = [-(-(n + args.tokens) // page) for n in counts]
    cache = gq.gqsa_cache_create(sum(per_sequence), page, args.kv_heads, dim)
    pages = torch.full((len(counts), max(per_sequence)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(per_sequence):
        pages[b, :n] = torch.arange(at, at + n, dtype=torch.int32, device="cuda")
        at += n
    norms = [torch.ones(dim, dtype=torch.float16, device="cuda") for _ in range(2)]
    layer = AttentionLayer(*matrices, args.heads, rotary_table(max(counts) + args.tokens, dim), cache, *norms)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    def timed(f):
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        f()
        end.record()
        end.synchronize()
        return begin.elapsed_time(end)

    starts = ints([sum(counts[:b]) for b in range(len(counts) + 1)])
    positions = torch.cat([torch.arange(n, device="cuda", dtype=torch.int32) for n in counts])
    lengths = ints(counts)
    x = torch.randn((sum(counts), args.hidden), generator=gen, device="cuda").half()
    layer.prompt(x, positions, pages, starts, lengths)           # (the first call of each kernel loads it)
    ms = timed(lambda: layer.prompt(x, positions, pages, starts, lengths))
    print(f"prompts of {counts}: {sum(counts)} rows in {ms:.2f} ms", flush=True)

    row = torch.randn((len(counts), args.hidden), generator=gen, device="cuda").half()
    place = lengths.clone()
    lengths += 1
    without_graph = layer.step(row, place, pages, lengths)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer.step(row, place, pages, lengths)

    def generate():
        for _ in range(args.tokens - 1):
            graph.replay()
            row.copy_(out)                  # (a model would have the rest of the layer here, and more layers)
            place.add_(1)
            lengths.add_(1)
    ms = timed(generate)
    assert torch.isfinite(out if args.tokens > 1 else without_graph).all()
    info = gq.gqsa_cache_info(cache)
    if args.tokens > 1:
        print(f"{args.tokens - 1} tokens for {len(counts)} sequences: {ms / (args.tokens - 1) * 1e3:.1f} us a step; ", end="")
    print(f"cache {info['device_bytes'] / 2 ** 20:.1f} MiB of {info['token_bytes']} bytes a token and head ({4 * dim} in fp16)", flush=True)


if __name__ == "__main__":
    main()
