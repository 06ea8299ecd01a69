"""Where a decoding step of several drafted tokens could go wrong at the edge of what its calls take: against the definitions in float64, on the GPU."""
from __future__ import annotations

import ctypes as C

import numpy as np
import pytest

import paper_2412_17560_amd as gq
from oracle import attention as ref
from oracle import drafts
from paper_2412_17560_amd import binding
from test_attention_gpu import Cached, _check_attended, dev, ints, normal
from test_drafts_gpu import random_tree, roomy, same, starts_of

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
