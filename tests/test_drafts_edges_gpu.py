"""Where a decoding step of several drafted tokens could go wrong at the edge of what its calls take: against the definitions in float64, on the GPU."""
from __future__ import annotations

import ctypes as C

import numpy as np
import pytest

import paper_2412_17560_amd as gq
from oracle import attention as ref
from oracle import drafts
from paper_2412_17560_amd import binding
from test_attention_edges_gpu import SMALL, _check_sum_of_small, _sink
from test_attention_gpu import Cached, _check_attended, dev, ints, normal
from test_drafts_gpu import _check_verified, _verify, probabilities, random_tree, roomy, roomy_pages, same, starts_of

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


# ----------------------------------------------------------------------------- a rotation's table without rows
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim, rotary, given", [(64, 32, True), (128, 128, False), (128, 48, True)])
def test_a_table_without_rows(dim, rotary, given, interleaved):
    """No position is in it: what would be rotated is NaN, the rest is normed as ever, and nothing is read of it.  (Through the C call: torch has no address for an
    empty array.  The table begins where an array ends.)"""
    c = Cached([30, 3], 2, dim, 32, seed=dim + rotary, room=10)
    counts, lengths = [5, 1], [35, 4]
    n, starts = sum(counts), starts_of(counts)
    q, k, v, weight = normal(c.rng, n, 3, dim), c.some(n), c.some(n), normal(c.rng, dim)
    held = torch.ones(16 * rotary, device="cuda")
    dq, dk, dv, dw, pages, at, positions = (dev(x) for x in (q, k, v, weight, c.pages, starts, np.arange(-1, n - 1, dtype=np.int32)))
    q_out, k_out, total = torch.zeros_like(dq), torch.zeros_like(dk), ints(*lengths)
    p = [C.c_void_p(t.data_ptr()) for t in (dq, dk, dv, dw, positions, q_out, k_out, pages, total, at)]
    status = binding._lib().gqsa_cache_append_rotated(
        c.cache.ptr, p[0], 3 * dim, dim, 3, p[1], 2 * dim, dim, p[2], 2 * dim, dim, n, p[3], p[3], 1e-5, C.c_void_p(held.data_ptr() + held.numel() * 4), 0, rotary,
        interleaved, p[4] if given else None, p[5], 3 * dim, dim, p[6], 2 * dim, dim, p[7], c.pages.shape[1], p[8], p[9], 2, C.c_void_p(torch.cuda.current_stream().cuda_stream))
    assert status == 0
    want = []
    for x in (q, k):
        y = drafts.norm_rotate_rounded(x, weight=weight, eps=1e-5)
        y[..., :rotary] = np.nan
        want.append(y)
    assert same(q_out.cpu().numpy(), want[0]) and same(k_out.cpu().numpy(), want[1])
    c.k, c.v = ([np.concatenate([a, new[s:e]]) for a, s, e in zip(held, starts, starts[1:])] for held, new in ((c.k, want[1]), (c.v, v)))
    c.check()


# ----------------------------------------------------------------------------- calls without rows
@pytest.mark.parametrize("n_seqs", [0, 1, 3])
@pytest.mark.parametrize("drawn", [False, True])
def test_verify_without_rows(n_seqs, drawn):
    verifier = gq.gqsa_verify_create(3, 40000)
    target = torch.empty((0, 40000), device="cuda")
    finals, accepted = torch.zeros(n_seqs, device="cuda"), torch.full((n_seqs,), 7, dtype=torch.int32, device="cuda")
    for starts in (ints(*[0] * (n_seqs + 1)), None):
        path, out, got = gq.gqsa_verify(verifier, target, ints(), torch.empty(0, device="cuda"), finals, starts, parents=None if drawn else ints(),
                                        draft=target if drawn else None, accepted=accepted.clone())
        assert path.shape == out.shape == (0,) and got.tolist() == [-1] * n_seqs


@pytest.mark.parametrize("n_seqs", [0, 2])
def test_a_layers_drafted_step_without_rows(n_seqs):
    """Nothing is appended, attended, verified or kept, and the cache is what it was."""
    import gqsa_inputs as gi
    from paper_2412_17560_amd.attention_layer import AttentionLayer, rotary_table

    hidden, heads, kv_heads, dim = 256, 4, 2, 64
    sizes = [(heads * dim, hidden), (kv_heads * dim, hidden), (kv_heads * dim, hidden), (hidden, heads * dim)]
    c = Cached([40, 3], kv_heads, dim, 32, room=64)
    layer = AttentionLayer(*[gq.gqsa_pack(gi.dense_weight(n, k, seed=i), 16, 4, 0.5) for i, (n, k) in enumerate(sizes)], heads, rotary_table(64, dim), c.cache)
    pages, lengths, starts = dev(c.pages[:n_seqs]), ints(*[40, 3][:n_seqs]), ints(*[0] * (n_seqs + 1))
    x = torch.empty((0, hidden), dtype=torch.float16, device="cuda")
    assert layer.drafts(x, ints(), pages, lengths, starts, torch.empty((0, 1), dtype=torch.int32, device="cuda")).shape == (0, hidden)
    path, _, accepted = gq.gqsa_verify(gq.gqsa_verify_create(2, 50), torch.empty((0, 50), device="cuda"), ints(), torch.empty(0, device="cuda"),
                                       torch.zeros(n_seqs, device="cuda"), starts, parents=ints())
    layer.keep(pages, lengths, starts, path, accepted)
    c.check()


# ----------------------------------------------------------------------------- rows of a tree that pass the end of the pages
@roomy
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("fit", [12, 7, 1, 0, -3])
def test_a_trees_rows_beyond_the_pages(dim, fit, room):
    """The rows that still have a place are the tokens that append has made of them, and see those before them all; the others have none, and see what their masks name of the
    rest.  The sequence's last two pages are there only, the table's last ones: with room, a table for which the kernel for many rows is taken."""
    n, heads, kv_heads, page, there = 12, 8, 2, 32, 64
    wide = -(-65536 * 32 // (n * heads // 16 * page)) if room else 4
    c = Cached([0], kv_heads, dim, page, seed=fit + dim, room=there)
    pages = np.full((1, wide), -1, np.int32)
    pages[0, -2:] = c.pages[0]
    before = wide * page - fit                                  # tokens before the rows; those that are there are the last 64 of the table's room
    old = there - max(fit, 0)
    k, v = c.some(old + n), c.some(old + n)
    lost = max(-fit, 0)                                         # (of the old ones, appended in a call of their own)
    for at, end, length in ((0, old, before - lost), (old, old + n, before + n)):
        gq.gqsa_cache_append(c.cache, dev(k[at:end]), dev(v[at:end]), dev(pages), ints(length), ints(0, end - at))
    q, sees = normal(c.rng, n, heads, dim), drafts.ancestors(random_tree(c.rng, n, 3))
    out = gq.gqsa_cache_attend_tree(c.cache, dev(q), dev(pages), ints(before + n), ints(0, n), dev(drafts.mask_words(sees, 1))).cpu().numpy()
    seen = sees.copy()
    seen[:, max(fit, 0):] = False
    hk, hv = ref.cache_values(k), ref.cache_values(v)
    want, size = drafts.tree_attention(q, hk, hv, dim ** -0.5, seen)
    _check_attended(out, want, size, old + n, hv)


@roomy
def test_lengths_far_beyond_the_pages(room):
    """Every token that is there lies before the rows, however far."""
    n, heads, dim, page = 12, 32, 64, 32
    wide = -(-65536 * 32 // (n * heads // 16 * page)) if room else 2
    c = Cached([64, 64, 64], 2, dim, page, seed=1)
    pages = np.full((3, wide), -1, np.int32)
    pages[:, -2:] = c.pages
    for b in range(3):
        gq.gqsa_cache_append(c.cache, dev(c.k[b]), dev(c.v[b]), dev(pages[b:b + 1]), ints(wide * page), ints(0, 64))
    q, counts = normal(c.rng, n, heads, dim), [5, 4, 3]
    masks = dev(drafts.mask_words(np.zeros((n, n), bool), 1))
    out = gq.gqsa_cache_attend_tree(c.cache, dev(q), dev(pages), ints(wide * page + 5, 2 ** 31 - 1, 2 ** 31 - 4000), dev(starts_of(counts)), masks).cpu().numpy()
    for b, (s, e) in enumerate(zip(starts_of(counts), starts_of(counts)[1:])):
        hk, hv = ref.cache_values(c.k[b]), ref.cache_values(c.v[b])
        want, size = ref.attention(q[s:e], hk, hv, dim ** -0.5, [64] * (e - s))
        _check_attended(out[s:e], want, size, 64, hv)


# ----------------------------------------------------------------------------- many small weights behind a large one
@roomy
@pytest.mark.parametrize("of_sink", [0.0, 1.0])
@pytest.mark.parametrize("tokens, gap", SMALL)
def test_many_small_weights_of_a_tree(tokens, gap, of_sink, room):
    n = 40
    c = Cached([0], 1, 64, 1024, seed=int(10 * gap), room=tokens)
    q, k, v = _sink(c.rng, tokens, 1, 1, gap, of_sink, rows=n)
    c.append([k], [v])
    pages = roomy_pages(c, n) if room else c.pages
    masks = drafts.mask_words(np.tri(n, dtype=bool), 2)
    out = gq.gqsa_cache_attend_tree(c.cache, dev(q), dev(pages), ints(tokens), ints(0, n), dev(masks), scale=1.0).cpu().numpy()
    hk, hv = ref.cache_values(k), ref.cache_values(v)
    want, size = ref.attention(q, hk, hv, 1.0, [tokens - n + i + 1 for i in range(n)])
    _check_sum_of_small(out, want, size, tokens, hv)


# ----------------------------------------------------------------------------- many children of one row
@pytest.mark.parametrize("n, vocab, distinct", [(65, 300, 300), (200, 300, 40), (200, 5000, 5000), (1024, 3000, 700), (1024, 20000, 20000)])
def test_verify_many_children_of_one_row(n, vocab, distinct):
    """Stars: more children than the 64 rows that are looked at together, with tokens that come again in the same 64 and in later ones; none stands, one stands alone (with a
    token that an earlier one has, or has not), any may.  The second half of them has children of its own in a last star."""
    rng = np.random.default_rng(n + distinct)
    sequences, finals, ends = [], [], []
    for case in range(24):
        target = probabilities(rng, n, vocab)
        tokens = rng.permutation(vocab)[:distinct][rng.integers(0, distinct, n)].astype(np.int32)
        if distinct >= n:
            tokens = rng.permutation(vocab)[:n].astype(np.int32)
        parents = np.zeros(n, np.int32)
        parents[0] = -1
        uniforms = np.ones(n, np.float32)
        if case % 4 == 1:
            uniforms[n - 1 - rng.integers(0, n // 3)] = 0.0
        elif case % 4 == 2:
            uniforms[1 + rng.integers(0, n - 1)] = 0.0
        elif case % 4 == 3:
            uniforms = (0.9 + 0.1 * rng.random(n)).astype(np.float32)
        if case % 8 >= 4:                                      # (a row in the middle, which stands, has all that come behind it)
            middle = n // 2 + int(rng.integers(-3, 4))
            parents[middle + 1:], uniforms[middle] = middle, 0.0
        sequences.append((target, tokens, uniforms, parents, None))
        finals.append(rng.random(dtype=np.float32))
        ends.append(len(drafts.verify(target, tokens, uniforms, finals[-1], parents)[0]))
    assert {1, 2} <= set(ends)
    _check_verified(sequences, finals, _verify(gq.gqsa_verify_create(24, vocab), sequences, finals))


# ----------------------------------------------------------------------------- the command's steps
class _Given(torch.Tensor):
    """Numbers that are what they have been set to."""

    def uniform_(self):
        return self


@pytest.mark.parametrize("count, vocab, cached", [(7, 1024, [40, 3]), (40, 300, [700])])
def test_replayed_drafted_steps_are_the_eager_ones(count, vocab, cached):
    """The command's whole step, torch's products and sums in it, from a captured graph: every replay gives what the eager step gives, with eager steps between them."""
    import gqsa_inputs as gi
    from paper_2412_17560_amd.attention_layer import AttentionLayer, DraftedSteps, rotary_table

    hidden, heads, kv_heads, dim = 256, 4, 2, 64
    sizes = [(heads * dim, hidden), (kv_heads * dim, hidden), (kv_heads * dim, hidden), (hidden, heads * dim)]
    matrices = [gq.gqsa_pack(gi.dense_weight(n, k, seed=i), 16, 4, 0.5) for i, (n, k) in enumerate(sizes)]
    twins = [Cached(cached, kv_heads, dim, 64, seed=3, room=count + 8 * 7) for _ in range(2)]
    eager, graphed = (DraftedSteps(AttentionLayer(*matrices, heads, rotary_table(2000, dim), c.cache), dev(c.pages), ints(*cached), count, vocab) for c in twins)
    for steps in (eager, graphed):
        steps.uniforms, steps.finals = steps.uniforms.as_subclass(_Given), steps.finals.as_subclass(_Given)
    rng, graph, kept = np.random.default_rng(count), None, 0
    for _ in range(7):
        numbers = rng.random(len(cached) * (count + 1), dtype=np.float32), rng.random(len(cached), dtype=np.float32)
        for steps in (eager, graphed):
            steps.uniforms.copy_(dev(numbers[0])), steps.finals.copy_(dev(numbers[1]))
        want = eager.step()
        if graph is None:
            got = graphed.step()                               # (the first call of each kernel loads it)
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                got_by_graph = graphed.step()
        else:
            graph.replay()
            got = got_by_graph
        torch.cuda.synchronize()
        assert torch.equal(want, got) and torch.isfinite(got).all()
        assert all(torch.equal(getattr(eager, name), getattr(graphed, name)) for name in ("before", "last", "generated"))
        kept = int(eager.generated)
    assert kept > 7 * len(cached)                              # (drafted tokens stood)
