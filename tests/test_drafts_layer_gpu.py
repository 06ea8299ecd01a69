"""Drafted steps as they are used: append, attention, verification and the kept rows one after the other, eager and from a captured graph, and as a layer runs
them."""
from __future__ import annotations

import numpy as np
import pytest

import paper_2412_17560_amd as gq
from oracle import attention as ref
from oracle import drafts
from test_attention_gpu import Cached, _table, dev, ints, normal
from test_drafts_gpu import starts_of

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


class Step:
    """One step with everything in buffers that stay; lengths move on by what was kept."""

    def __init__(self, c, counts, heads, vocab, table, weights, parents, masks):
        rows, n = sum(counts), len(counts)
        self.c, self.counts, self.vocab = c, counts, vocab
        self.q = torch.empty((rows, heads, c.dim), dtype=torch.float16, device="cuda")
        self.k, self.v = (torch.empty((rows, c.kv_heads, c.dim), dtype=torch.float16, device="cuda") for _ in range(2))
        self.turned, self.attended = torch.empty_like(self.q), torch.empty_like(self.q)
        self.target, self.uniforms, self.finals = torch.empty((rows, vocab), device="cuda"), torch.empty(rows, device="cuda"), torch.empty(n, device="cuda")
        self.tokens, self.positions, self.path, self.out = (torch.zeros(rows, dtype=torch.int32, device="cuda") for _ in range(4))
        self.accepted = torch.zeros(n, dtype=torch.int32, device="cuda")
        self.starts, self.of, self.pages = dev(starts_of(counts)), ints(*counts), dev(c.pages)
        self.before, self.lengths = ints(*c.lengths()), ints(*([0] * n))
        self.table, self.weights, self.parents, self.masks = dev(table), [dev(w) for w in weights], dev(parents), dev(masks)
        self.verifier = gq.gqsa_verify_create(n, vocab)

    def fill(self, values):
        for name, value in values.items():
            getattr(self, name).copy_(torch.from_numpy(value))

    def run(self):
        torch.add(self.before, self.of, out=self.lengths)
        gq.gqsa_cache_append_rotated(self.c.cache, self.q, self.k, self.v, self.positions, self.table, self.pages, self.lengths, self.starts, *self.weights, q_out=self.turned)
        gq.gqsa_cache_attend_tree(self.c.cache, self.turned, self.pages, self.lengths, self.starts, self.masks, out=self.attended)
        gq.gqsa_verify(self.verifier, self.target, self.tokens, self.uniforms, self.finals, self.starts, parents=self.parents, path=self.path, out=self.out, accepted=self.accepted)
        gq.gqsa_cache_keep(self.c.cache, self.pages, self.lengths, self.starts, self.path, self.accepted)
        self.before.add_(self.accepted).add_(1)

    def results(self):
        lengths = self.before.cpu().numpy()
        starts = dev(starts_of(lengths))
        kv = [torch.empty((int(lengths.sum()), self.c.kv_heads, self.c.dim), dtype=torch.float16, device="cuda") for _ in range(2)]
        gq.gqsa_cache_read(self.c.cache, self.pages, self.before, starts, *kv)
        return [t.cpu().numpy() for t in (self.turned, self.attended, self.path, self.out, self.accepted, self.before, *kv)]


@pytest.mark.parametrize("dim, heads, kv_heads, page, cached, counts, room, vocab", [
    (128, 8, 2, 64, [70, 0, 300], [9, 1, 34], 200, 5000),
    (64, 4, 4, 32, [33, 5], [8, 16], 120, 300),
    (128, 16, 1, 128, [900], [64], 70000, 40000),           # the kernel of many rows: a page table for 70000 tokens
])
def test_steps_one_after_the_other(dim, heads, kv_heads, page, cached, counts, room, vocab):
    """Steps run eagerly are the definition's; the same steps from a captured graph, with the eager ones between its replays, give the same bits."""
    rng = np.random.default_rng(dim + vocab)
    n, rows, steps = len(counts), sum(counts), 4
    twins = [Cached(cached, kv_heads, dim, page, seed=8, room=120, spare=2) for _ in range(2)]
    for c in twins:
        c.pages = np.pad(c.pages, [(0, 0), (0, max(0, room // page - c.pages.shape[1]))], constant_values=-1)
    table, weights = _table(2000, dim // 2), [normal(rng, dim) for _ in range(2)]
    parents = np.concatenate([[-1] + [int(rng.integers(0, i)) for i in range(1, m)] for m in counts]).astype(np.int32)
    starts = starts_of(counts)
    sees = [drafts.ancestors(parents[s:e]) for s, e in zip(starts, starts[1:])]
    masks = np.concatenate([drafts.mask_words(m, 2) for m in sees])
    depth = np.concatenate([m.sum(axis=1) - 1 for m in sees])
    eager, graphed = (Step(c, counts, heads, vocab, table, weights, parents, masks) for c in twins)

    def values(before):
        target = rng.random((rows, vocab)).astype(np.float32) ** 8
        tokens = rng.integers(0, vocab, rows).astype(np.int32)
        for s, e in zip(starts, starts[1:]):
            for i in range(s + 1, e):
                target[s + parents[i], tokens[i]] = vocab / 10         # (so that ways of several rows come about)
        target /= target.sum(axis=1, keepdims=True)
        return dict(q=normal(rng, rows, heads, dim), k=normal(rng, rows, kv_heads, dim), v=normal(rng, rows, kv_heads, dim), target=target.astype(np.float32), tokens=tokens,
                    uniforms=rng.random(rows).astype(np.float32), finals=rng.random(n).astype(np.float32),
                    positions=(np.repeat(before, counts) + depth).astype(np.int32))

    graph, moved = None, 0
    for _ in range(steps):
        c = twins[0]
        now = values(c.lengths())
        eager.fill(now), graphed.fill(now)
        eager.run()
        if graph is None:
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                graphed.run()
        graph.replay()
        got, other = eager.results(), graphed.results()
        assert all(np.array_equal(a, b) for a, b in zip(got, other))
        turned, attended, path, out, accepted, before = got[:6]
        kw = dict(positions=now["positions"], table=table)
        want_q, want_k = (drafts.norm_rotate_rounded(now[x], weight=w, **kw) for x, w in zip("qk", weights))
        assert np.array_equal(turned, want_q)
        for b, (s, e) in enumerate(zip(starts, starts[1:])):
            way, last = drafts.verify(now["target"][s:e], now["tokens"][s:e], now["uniforms"][s:e], now["finals"][b], parents[s:e])
            assert accepted[b] == len(way) - 1 and list(path[s:s + len(way)]) == way and (path[s + len(way):e] == -1).all()
            assert list(out[s:s + len(way)]) == [int(now["tokens"][s + i]) for i in way[1:]] + [last]
            k, v = np.concatenate([c.k[b], want_k[s:e]]), np.concatenate([c.v[b], now["v"][s:e]])
            want, size = drafts.tree_attention(turned[s:e], ref.cache_values(k), ref.cache_values(v), dim ** -0.5, sees[b])
            assert (np.abs(attended[s:e] - want) <= 2e-3 * size + 1e-4).all()
            of = [len(c.k[b]) + i for i in way]
            moved += len(way) - 1
            c.k[b], c.v[b] = (np.concatenate([x[:len(y)], x[of]]) for x, y in ((k, c.k[b]), (v, c.v[b])))
        c.check()
        assert list(before) == list(c.lengths())
    assert moved > 0


@pytest.mark.parametrize("room", [0, 70000])                  # the attention for few rows, and for many
def test_offsets_that_pass_32_bits(room):
    """Pages behind the fourth gigabyte of a cache, rows of queries, results and probabilities 2^28 elements apart."""
    heads, kv_heads, dim, rows, vocab = 64, 1, 128, 9, 3000
    c = Cached([600], kv_heads, dim, 256, seed=12)
    big = gq.gqsa_cache_create(5 * 2 ** 30 // (256 * 160 * kv_heads) + 1, 256, kv_heads, dim)
    n = gq.gqsa_cache_info(big)["n_pages"]
    k, v = c.k[0], c.v[0]
    c.cache, c.n_pages, c.k, c.v = big, n, [k[:0]], [v[:0]]
    c.pages = np.array([[n - 1, 0, n - 2]], np.int32)
    c.append([k], [v])
    wide = np.pad(c.pages, [(0, 0), (0, max(0, room // 256 - 3))], constant_values=-1)
    parents = np.array([-1, 0, 0, 1, 2, 2, 4, 6, 7], np.int32)
    sees = drafts.ancestors(parents)
    table, positions = _table(700, dim // 2), (600 + sees.sum(axis=1) - 1).astype(np.int32)
    apart = torch.empty((rows, 1 << 28), dtype=torch.float16, device="cuda")
    q, out = (apart[:, at:at + heads * dim].view(rows, heads, dim) for at in (0, 1 << 20))
    x, new_k, new_v = normal(c.rng, rows, heads, dim), c.some(rows), c.some(rows)
    q.copy_(dev(x))
    lengths, starts = ints(600 + rows), ints(0, rows)
    gq.gqsa_cache_append_rotated(big, q, dev(new_k), dev(new_v), dev(positions), dev(table), dev(c.pages), lengths, starts, q_out=q)
    want = drafts.norm_rotate_rounded(x, positions, table)
    assert np.array_equal(q.cpu().numpy(), want)
    gq.gqsa_cache_attend_tree(big, q, dev(wide), lengths, starts, dev(drafts.mask_words(sees, 1)), out=out)
    k, v = np.concatenate([k, drafts.norm_rotate_rounded(new_k, positions, table)]), np.concatenate([v, new_v])
    attended, size = drafts.tree_attention(want, ref.cache_values(k), ref.cache_values(v), dim ** -0.5, sees)
    assert (np.abs(out.cpu().numpy() - attended) <= 2e-3 * size + 1e-4).all()
    del q, out, apart
    target = c.rng.random((rows, vocab)).astype(np.float32)
    tokens, uniforms = c.rng.integers(0, vocab, rows).astype(np.int32), np.zeros(rows, np.float32)
    target /= target.sum(axis=1, keepdims=True)
    uniforms[1] = 1.0                                       # the way goes by row 2 and 4 to the last row
    spread = torch.empty((rows, 1 << 28), dtype=torch.float32, device="cuda")[:, :vocab]
    spread.copy_(dev(target))
    path, drawn, accepted = gq.gqsa_verify(gq.gqsa_verify_create(1, vocab), spread, dev(tokens), dev(uniforms), dev(np.array([0.7], np.float32)), starts, parents=dev(parents))
    way, last = drafts.verify(target, tokens, uniforms, np.float32(0.7), parents)
    assert way == [0, 2, 4, 6, 7, 8] and path.tolist() == way + [-1] * 3 and drawn.tolist()[5] == last and accepted.tolist() == [5]
    gq.gqsa_cache_keep(big, dev(c.pages), lengths, starts, path, accepted)
    of = list(range(600)) + [600 + i for i in way]
    c.k, c.v = [k[of]], [v[of]]
    c.check()
    gq.gqsa_cache_free(big)


def test_a_step_on_another_stream_makes_its_arrays_there():
    """All four calls with a stream of their own, also as its number, and with results that the calls allocate."""
    c, d = (Cached([45], 2, 64, 32, seed=2, room=40) for _ in range(2))
    rng, parents, vocab = np.random.default_rng(5), np.array([-1, 0, 0, 2], np.int32), 500
    sees = drafts.ancestors(parents)
    q, k, v = normal(rng, 4, 4, 64), normal(rng, 4, 2, 64), normal(rng, 4, 2, 64)
    target = rng.random((4, vocab)).astype(np.float32)
    tokens, uniforms, finals = rng.integers(0, vocab, 4).astype(np.int32), np.array([0, 1, 0, 0], np.float32), np.array([0.5], np.float32)
    fixed = [dev(a) for a in (q, k, v, drafts.mask_words(sees, 1), target, tokens, uniforms, finals, parents)]
    lengths, starts = ints(49), ints(0, 4)
    other = torch.cuda.Stream()
    results = []
    for x, stream in ((c, None), (d, other), (c, other.cuda_stream)):
        if stream is not None:
            other.wait_stream(torch.cuda.current_stream())
        pages, verifier = dev(x.pages), gq.gqsa_verify_create(1, vocab)
        torch.cuda.synchronize()
        turned, _ = gq.gqsa_cache_append_rotated(x.cache, *fixed[:3], None, dev(_table(64, 32)), pages, lengths, starts, stream=stream)
        attended = gq.gqsa_cache_attend_tree(x.cache, turned, pages, lengths, starts, fixed[3], stream=stream)
        path, out, accepted = gq.gqsa_verify(verifier, *fixed[4:8], starts, parents=fixed[8], stream=stream)
        gq.gqsa_cache_keep(x.cache, pages, lengths, starts, path, accepted, stream=stream)
        kept = gq.gqsa_cache_read(x.cache, pages, ints(48), ints(0, 48), *(torch.empty((48, 2, 64), dtype=torch.float16, device="cuda") for _ in range(2)), stream=stream)
        torch.cuda.synchronize()
        results.append([t.cpu().numpy() for t in (turned, attended, path, out, accepted, *kept)])
    assert list(results[0][2]) == [0, 2, 3, -1]
    for other_results in results[1:]:
        assert all(np.array_equal(a, b) for a, b in zip(results[0], other_results))


def test_drafts_of_a_layer_are_its_steps():
    """A chain that is kept whole leaves what as many steps of one token leave, and each row attends to what the step's row attends to."""
    import gqsa_inputs as gi
    from paper_2412_17560_amd.attention_layer import AttentionLayer, drafted_tree, rotary_table

    hidden, heads, kv_heads, dim, rows = 256, 4, 2, 64, 5
    sizes = [(heads * dim, hidden), (kv_heads * dim, hidden), (kv_heads * dim, hidden), (hidden, heads * dim)]
    matrices = [gq.gqsa_pack(gi.dense_weight(n, k, seed=i), 16, 4, 0.5) for i, (n, k) in enumerate(sizes)]
    caches = [Cached([40, 61], kv_heads, dim, 32, seed=6, room=32) for _ in range(2)]
    layers = [AttentionLayer(*matrices, heads, rotary_table(100, dim), c.cache) for c in caches]
    rng = np.random.default_rng(1)
    x = normal(rng, 2, rows, hidden)
    chain = np.tile([(2 << i) - 1 for i in range(rows)], 2).astype(np.int32)[:, None]
    places = (np.array([40, 61])[:, None] + np.arange(rows)).astype(np.int32)
    y = layers[0].drafts(dev(x.reshape(-1, hidden)), dev(places.flatten()), dev(caches[0].pages), ints(40 + rows, 61 + rows), ints(0, rows, 2 * rows), dev(chain))
    layers[0].keep(dev(caches[0].pages), ints(40 + rows, 61 + rows), ints(0, rows, 2 * rows), dev(np.tile(np.arange(rows), 2).astype(np.int32)), ints(rows - 1, rows - 1))
    got = y.view(2, rows, hidden).cpu().numpy().astype(np.float64)
    for i in range(rows):
        want = layers[1].step(dev(np.ascontiguousarray(x[:, i])), dev(np.ascontiguousarray(places[:, i])), dev(caches[1].pages), ints(41 + i, 62 + i)).cpu().numpy()
        # the same tokens in other blocks: each result is within 2e-3 of its terms' sum, which is more than its value
        assert np.abs(got[:, i] - want).max() <= 4e-3 * np.abs(want).max() + 1e-4
    out = []
    for c in caches:
        kv = [torch.empty((2 * rows, kv_heads, dim), dtype=torch.float16, device="cuda") for _ in range(2)]
        out.append(gq.gqsa_cache_read(c.cache, dev(c.pages), ints(40 + rows, 61 + rows), ints(0, rows, 2 * rows), *kv))
    assert all(torch.equal(a, b) for a, b in zip(*out))
    parents, depths, masks = drafted_tree(40)
    assert np.array_equal(drafts.mask_words(drafts.ancestors(parents), 2), np.array(masks, np.int64).astype(np.int32))
    assert depths == list(drafts.ancestors(parents).sum(axis=1) - 1)


@pytest.mark.parametrize("tokens, drafted, prompts", [(1, 3, "64,3"), (6, 7, "40,3"), (3, 33, "63")])
def test_example_command_with_drafts(monkeypatch, capsys, tokens, drafted, prompts):
    from paper_2412_17560_amd import attention_layer
    monkeypatch.setattr("sys.argv", ["attention_layer", "--hidden", "512", "--heads", "8", "--kv-heads", "2", "--head-dim", "64",
                                     "--prompts", prompts, "--tokens", str(tokens), "--drafts", str(drafted)])
    attention_layer.main()
    printed = capsys.readouterr().out
    assert f"steps of {drafted} drafted tokens kept" in printed and ("us a step" in printed) == (tokens > 1)
