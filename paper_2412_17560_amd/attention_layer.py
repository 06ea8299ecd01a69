"""The attention half of a decoder layer on this library alone: q/k/v products of packed matrices, norms and rotation, a 4-bit
cache, attention, o product -- for packed prompts, for token generation, and for steps of several drafted tokens.

    python3 -m paper_2412_17560_amd.attention_layer [--hidden 4096] [--heads 32] [--kv-heads 8] [--prompts 700,15,2048] [--tokens 64] [--drafts 0]

runs prompts of these lengths, then generates tokens for all of them with one captured HIP graph, on random weights, and prints what each
phase took and what the cache holds.  With --drafts each further step takes a tree of that many drafted tokens per sequence, of which those that the target's
probabilities let stand are kept.
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

    def drafts(self, x, positions, pages, lengths, starts, masks):
        """Rows x of drafted trees, the newest tokens of each sequence (lengths counts them in; positions: those before them, and a row's depth), of which each
        sees the tokens before all of them and those that its mask names."""
        import paper_2412_17560_amd as gq
        q, k, v = self._products([self.q, self.k, self.v], x)
        q = q.view(-1, self.heads, self.head_dim)
        k, v = (t.view(-1, self.kv_heads, self.head_dim) for t in (k, v))
        gq.gqsa_cache_append_rotated(self.cache, q, k, v, positions, self.table, pages, lengths, starts, *self.norms, eps=self.eps, q_out=q)
        attended = gq.gqsa_cache_attend_tree(self.cache, q, pages, lengths, starts, masks)
        return self._products([self.o], attended.view(x.shape[0], self.heads * self.head_dim))[0]

    def keep(self, pages, lengths, starts, path, accepted):
        """Of those rows the ones of path become the first accepted + 1 (the caller then lowers lengths to them)."""
        import paper_2412_17560_amd as gq
        gq.gqsa_cache_keep(self.cache, pages, lengths, starts, path, accepted)


def rotary_table(positions: int, rotary_dim: int, theta: float = 10000.0):
    """float32 [positions, rotary_dim / 2, 2] on the device: cosine and sine of position * theta^(-2 i / rotary_dim)."""
    import torch
    i = torch.arange(0, rotary_dim, 2, device="cuda", dtype=torch.float64)
    angle = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * theta ** (-i / rotary_dim)
    return torch.stack([angle.cos(), angle.sin()], dim=-1).float()


def drafted_tree(drafts: int):
    """(parents, depths, masks) of a row and `drafts` tokens behind it, two to a parent, as lists: masks int32 words."""
    parents, depths, sees = [-1] + [(i - 1) // 2 for i in range(1, drafts + 1)], [0], [1]
    for i, p in enumerate(parents[1:], 1):
        depths.append(depths[p] + 1)
        sees.append(sees[p] | 1 << i)
    words = [[s >> 32 * w & 0xFFFFFFFF for w in range(drafts // 32 + 1)] for s in sees]
    return parents, depths, [[w - (w >> 31 << 32) for w in row] for row in words]


class DraftedSteps:
    """Steps of drafted tokens on one layer and random embeddings, whose products with themselves stand for a model's output: a token's likeliest successor is the
    token itself, which is what the tree's first children are (the second: the next number)."""

    def __init__(self, layer, pages, before, drafts: int, vocab: int = 1024):
        """before: int32 [n_seqs] tokens cached."""
        import torch

        import paper_2412_17560_amd as gq
        self.layer, self.pages, self.before = layer, pages, before.clone()
        n, rows = len(before), drafts + 1
        hidden = gq.gqsa_info(layer.o)["N"]
        parents, self.depths, masks = drafted_tree(drafts)
        self.parents = torch.tensor(parents * n, dtype=torch.int32, device="cuda")
        self.depth = torch.tensor(self.depths, dtype=torch.int32, device="cuda")
        self.masks = torch.tensor(masks * n, dtype=torch.int32, device="cuda")
        self.starts = torch.arange(n + 1, dtype=torch.int32, device="cuda") * rows
        # second children, counted along the way from row 0
        added = [0]
        for i in range(1, rows):
            added.append(added[parents[i]] + (i % 2 == 0))
        self.added = torch.tensor(added, device="cuda")
        self.embedding = torch.randn((vocab, hidden), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").half()
        self.last = torch.zeros(n, dtype=torch.int64, device="cuda")
        self.uniforms, self.finals = torch.empty(n * rows, device="cuda"), torch.empty(n, device="cuda")
        self.generated = torch.zeros((), dtype=torch.int64, device="cuda")
        self.verifier = gq.gqsa_verify_create(n, vocab)
        self.rows, self.vocab = rows, vocab

    def step(self):
        """(Can be captured: what it changes stays on the device.)"""
        import torch

        import paper_2412_17560_amd as gq
        tokens = ((self.last[:, None] + self.added) % self.vocab).flatten()
        lengths = self.before + self.rows
        positions = (self.before[:, None] + self.depth).flatten()
        x = self.embedding[tokens]
        y = x + self.layer.drafts(x, positions, self.pages, lengths, self.starts, self.masks)
        target = torch.softmax((y @ self.embedding.T).float() * (8.0 / x.shape[1]), dim=-1)
        self.uniforms.uniform_(), self.finals.uniform_()
        path, out, accepted = gq.gqsa_verify(self.verifier, target, tokens.int(), self.uniforms, self.finals, self.starts, parents=self.parents)
        self.layer.keep(self.pages, lengths, self.starts, path, accepted)
        self.last.copy_(out[(self.starts[:-1] + accepted).long()])
        self.before += accepted + 1
        self.generated += (accepted + 1).sum()
        return y


def main() -> None:
    p = argparse.ArgumentParser()
    p.add_argument("--hidden", type=int, default=4096)
    p.add_argument("--heads", type=int, default=32)
    p.add_argument("--kv-heads", type=int, default=8)
    p.add_argument("--head-dim", type=int, default=128, choices=(64, 128))
    p.add_argument("--prompts", default="700,15,2048", help="lengths of the prompts (up to 16 of them)")
    p.add_argument("--tokens", type=int, default=64, help="1 or more: a step without the graph, then one replay fewer than this")
    p.add_argument("--drafts", type=int, default=0, help="drafted tokens per sequence and step (up to 1000)")
    p.add_argument("--sparsity", type=float, default=0.5)
    args = p.parse_args()
    if args.tokens < 1:
        p.error("--tokens must be 1 or more")
    if not 0 <= args.drafts <= 1000:
        p.error("--drafts must be 0 to 1000")

    import torch

    import paper_2412_17560_amd as gq

    torch.cuda.set_device(0)
    gen = torch.Generator(device="cuda").manual_seed(0)
    dim, counts = args.head_dim, [int(n) for n in args.prompts.split(",")]
    sizes = [(args.heads * dim, args.hidden), (args.kv_heads * dim, args.hidden), (args.kv_heads * dim, args.hidden), (args.hidden, args.heads * dim)]
    matrices = [gq.gqsa_pack_device(torch.randn(s, generator=gen, device="cuda") / s[1] ** 0.5, 16, 4, args.sparsity) for s in sizes]
    page = 64
    most = args.tokens if args.drafts == 0 else args.tokens * (args.drafts.bit_length() + 1) + args.drafts         # (a way has at most bit_length rows behind row 0)
    per_sequence = [-(-(n + most) // page) for n in counts]
    cache = gq.gqsa_cache_create(sum(per_sequence), page, args.kv_heads, dim)
    pages = torch.full((len(counts), max(per_sequence)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(per_sequence):
        pages[b, :n] = torch.arange(at, at + n, dtype=torch.int32, device="cuda")
        at += n
    norms = [torch.ones(dim, dtype=torch.float16, device="cuda") for _ in range(2)]
    layer = AttentionLayer(*matrices, args.heads, rotary_table(max(counts) + most, dim), cache, *norms)

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
    drafted = DraftedSteps(layer, pages, lengths, args.drafts) if args.drafts else None
    lengths += 1
    without_graph = layer.step(row, place, pages, lengths)
    torch.cuda.synchronize()
    if drafted:
        drafted.step()
        torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer.step(row, place, pages, lengths) if drafted is None else drafted.step()

    def generate():
        for _ in range(args.tokens - 1):
            graph.replay()
            if drafted:
                continue
            row.copy_(out)                  # (a model would have the rest of the layer here, and more layers)
            place.add_(1)
            lengths.add_(1)
    ms = timed(generate)
    assert torch.isfinite(out if args.tokens > 1 else without_graph).all()
    info = gq.gqsa_cache_info(cache)
    if drafted:
        print(f"steps of {args.drafts} drafted tokens kept {int(drafted.generated) / (args.tokens * len(counts)):.2f} tokens each")
    if args.tokens > 1:
        print(f"{args.tokens - 1} {'steps' if drafted else 'tokens'} for {len(counts)} sequences: {ms / (args.tokens - 1) * 1e3:.1f} us a step; ", end="")
    print(f"cache {info['device_bytes'] / 2 ** 20:.1f} MiB of {info['token_bytes']} bytes a token and head ({4 * dim} in fp16)", flush=True)


if __name__ == "__main__":
    main()
