"""Where the operators between the q/k/v and the o product could go wrong at the edge of what they take: against float64, on the GPU."""
from __future__ import annotations

import numpy as np
import pytest

import paper_2412_17560_amd as gq
from oracle import attention as ref
from test_attention_gpu import Cached, _check_attended, _check_prompts, _check_rotated, dev, ints, normal

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

LEAST, MOST = -2 ** 31, 2 ** 31 - 1


# ----------------------------------------------------------------------------- arrays on the device that hold anything
def _between(starts, n):
    """The rows of each sequence that are there."""
    return [range(max(a, 0), max(min(b, n), max(a, 0))) for a, b in zip(starts, starts[1:])]


STARTS = [[2, LEAST, 3], [5, LEAST, MOST], [MOST, LEAST, 2], [LEAST, 1, LEAST], [1, -1, LEAST + 1], [MOST, MOST - 1, LEAST]]


@pytest.mark.parametrize("starts", STARTS)
def test_starts_whose_difference_passes_32_bits_cache(starts):
    c = Cached([64, 40], 1, 64, 32, seed=11)
    n = 6
    q = normal(c.rng, n, 2, 64)
    room = torch.full((n + 20, 2, 64), 4.0, dtype=torch.float16, device="cuda")
    gq.gqsa_cache_attend(c.cache, dev(q), dev(c.pages), ints(*c.lengths()), ints(*starts), out=room[10:10 + n])
    kv = torch.full((n + 20, 1, 64), 4.0, dtype=torch.float16, device="cuda")
    kv2 = kv.clone()
    gq.gqsa_cache_read(c.cache, dev(c.pages), ints(*c.lengths()), ints(*starts), kv[10:10 + n], kv2[10:10 + n])
    out, kv, kv2 = (t.cpu().numpy() for t in (room, kv, kv2))
    left = np.ones(n + 20, bool)
    for b, rows in enumerate(_between(starts, n)):
        for i, r in enumerate(rows):
            left[10 + r] = False
            token = len(c.k[b]) - len(rows) + i
            hk, hv = ref.cache_values(c.k[b]), ref.cache_values(c.v[b])
            want, size = ref.attention(q[r:r + 1], hk, hv, 0.125, [token + 1])
            _check_attended(out[10 + r:11 + r], want, size, len(hk), hv)
            assert np.array_equal(kv[10 + r], hk[token]) and np.array_equal(kv2[10 + r], hv[token])
    assert (out[left] == 4).all() and (kv[left] == 4).all() and (kv2[left] == 4).all()
    x = normal(c.rng, n, 1, 64)
    gq.gqsa_cache_append(c.cache, dev(x), dev(x), dev(c.pages), ints(*c.lengths()), ints(*starts))
    for b, rows in enumerate(_between(starts, n)):          # the last tokens are these rows now, everything else is what it was
        if len(rows):
            c.k[b][-len(rows):] = c.v[b][-len(rows):] = x[rows.start:rows.stop]
    c.check()


@pytest.mark.parametrize("heads", [2, 96])          # rows shared by two wavefronts or not
@pytest.mark.parametrize("q_starts, k_starts", [*[(s, [0, 40, 70]) for s in STARTS], *[([0, 4, 6], [10 * v if abs(v) < 9 else v for v in s]) for s in STARTS]])
def test_starts_whose_difference_passes_32_bits_prompts(heads, q_starts, k_starts):
    rng = np.random.default_rng(3)
    n, keys = 6, 70
    q, k, v = normal(rng, n, heads, 64), normal(rng, keys, 1, 64), normal(rng, keys, 1, 64)
    room = torch.full((n + 20, heads, 64), 4.0, dtype=torch.float16, device="cuda")
    gq.gqsa_prompt_attend(dev(q), dev(k), dev(v), ints(*q_starts), ints(*k_starts), out=room[10:10 + n])
    out = room.cpu().numpy()
    left = np.ones(n + 20, bool)
    for rows, seen in zip(_between(q_starts, n), _between(k_starts, keys)):
        if not len(rows):
            continue
        left[10 + rows.start:10 + rows.stop] = False
        at, kb, vb = slice(rows.start, rows.stop), k[seen.start:seen.stop], v[seen.start:seen.stop]
        want, size = ref.attention(q[at], kb, vb, 0.125, [len(seen) - len(rows) + i + 1 for i in range(len(rows))])
        _check_attended(out[10 + rows.start:10 + rows.stop], want, size, len(seen), vb)
    assert (out[left] == 4).all()


# ----------------------------------------------------------------------------- sequences longer than their pages
@pytest.mark.parametrize("dim", [64, 128])
def test_rows_beyond_the_pages_are_left_out(dim):
    """A sequence that outgrows its pages keeps the tokens it has, whatever is appended to it."""
    c = Cached([60, 30], 2, dim, 32, seed=dim)                 # two pages and one: room for 64 and 32 tokens, of a table of two
    x, y = c.some(7), c.some(7)
    pages = dev(c.pages)
    gq.gqsa_cache_append(c.cache, dev(x), dev(y), pages, ints(67, 30), ints(0, 7, 7))
    c.k[0], c.v[0] = np.concatenate([c.k[0], x[:4]]), np.concatenate([c.v[0], y[:4]])
    c.check()
    for length in (65, 68, 96, 97, 64 + 2 ** 20, MOST - 40, MOST):
        gq.gqsa_cache_append(c.cache, dev(x[:1]), dev(y[:1]), pages, ints(length, 30), ints(0, 1, 1))
    gq.gqsa_cache_append(c.cache, dev(x), dev(y), pages, ints(MOST, 30), ints(0, 7, 7))
    gq.gqsa_cache_append(c.cache, dev(x[:2]), dev(y[:2]), pages, ints(65, 100))           # a row per sequence, both beyond
    c.check()
    k, v = (torch.full((7, 2, dim), 3.0, dtype=torch.float16, device="cuda") for _ in range(2))
    gq.gqsa_cache_read(c.cache, pages, ints(67, 30), ints(0, 7, 7), k, v)       # row i: the token that append makes of it
    for got, held in ((k, c.k[0]), (v, c.v[0])):
        got = got.cpu().numpy()
        assert np.array_equal(got[:4], ref.cache_values(held[60:])) and (got[4:] == 0).all()
    gq.gqsa_cache_read(c.cache, pages, ints(MOST, 30), ints(0, 7, 7), k, v)
    assert (k == 0).all() and (v == 0).all()


# ----------------------------------------------------------------------------- steps at the end of the range
def test_steps_whose_largest_value_is_next_to_infinity():
    """low + 15 step just below, at and just above where fp16 rounds to infinity: only the last two take the smaller step."""
    c = Cached([0], 1, 64, 32, room=32)
    x = c.some(8)
    x[:, 0, :32] = 0
    x[:, 0, 1] = 65504
    x[:, 0, 2:20] = (3000 * np.arange(1, 19)).astype(np.float16)
    for i, low in enumerate([-0.0005, -6e-8, 0, 6e-8, 0.0005, -1, -0.00195, 1]):
        x[i, 0, 0] = low
        x[i, 0, 20:32] = max(low, 0)
    c.append([x], [x])
    c.check()


# ----------------------------------------------------------------------------- many small weights behind a large one
def _sink(rng, tokens, kv_heads, q_heads, gap, of_sink, rows=1):
    """A first token that has the weight 1, and many that lie about `gap` below it in the exponent; the first one's value is `of_sink`."""
    q, k, v = np.zeros((rows, q_heads, 64)), np.zeros((tokens, kv_heads, 64)), 1 + 0.25 * rng.standard_normal((tokens, kv_heads, 64))
    q[:, :, 0], k[0, :, 0], v[0] = gap / 15, 15, of_sink
    q[:, :, 32:], k[1:, :, 32:] = rng.standard_normal((rows, q_heads, 32)), 0.05 * rng.standard_normal((tokens - 1, kv_heads, 32))
    return [x.astype(np.float16) for x in (q, k, v)]


def _check_sum_of_small(got, want, size, tokens, values):
    """The largest weight is 2^7 at least, and no less is their sum.  A weight is rounded to fp16, by 2^-11 of it or by 2^-25 (2^-32 of the sum), in the product as
    in the sum; so is the result, once (2^-11 or 2^-25); fp32 scores, exponentials and sums stay below 2^-14 of the size together."""
    error = np.abs(got.astype(np.float64) - want)
    bound = (3 * 2.0 ** -11 + 2.0 ** -14) * size + tokens * 2.0 ** -31 * np.abs(values).max() + 2.0 ** -25
    assert (error <= bound).all(), (error / size).max()


SMALL = [(131072, 17.0), (131072, 17.8), (8192, 17.8), (8192, 15.0), (1000, 14.0)]


@pytest.mark.parametrize("of_sink", [0.0, 1.0])
@pytest.mark.parametrize("tokens, gap", SMALL)
def test_many_small_weights_over_the_cache(tokens, gap, of_sink):
    c = Cached([0], 1, 64, 1024, seed=int(10 * gap), room=tokens)
    q, k, v = _sink(c.rng, tokens, 1, 2, gap, of_sink)
    c.append([k], [v])
    out = gq.gqsa_cache_attend(c.cache, dev(q), dev(c.pages), ints(tokens), scale=1.0).cpu().numpy()
    hk, hv = ref.cache_values(k), ref.cache_values(v)
    want, size = ref.attention(q, hk, hv, 1.0, [tokens])
    _check_sum_of_small(out, want, size, tokens, hv)


@pytest.mark.parametrize("of_sink", [0.0, 1.0])
@pytest.mark.parametrize("tokens, gap", [(8192, 17.8), (8192, 16.0), (30000, 17.4)])
def test_many_small_weights_of_many_sequences_over_the_cache(tokens, gap, of_sink):
    """As many sequences as there are workgroups, so that the large weight's wavefront has many of the small ones too; on the same pages all of them."""
    count = 520
    c = Cached([0], 1, 64, 1024, seed=tokens, room=tokens)
    q, k, v = _sink(c.rng, tokens, 1, 1, gap, of_sink, rows=count)
    c.append([k], [v])
    pages = dev(np.repeat(c.pages, count, axis=0))
    out = gq.gqsa_cache_attend(c.cache, dev(q), pages, ints(*[tokens] * count), scale=1.0).cpu().numpy()
    hk, hv = ref.cache_values(k), ref.cache_values(v)
    want, size = ref.attention(q, hk, hv, 1.0, [tokens] * count)
    _check_sum_of_small(out, want, size, tokens, hv)


@pytest.mark.parametrize("of_sink", [0.0, 1.0])
@pytest.mark.parametrize("tokens, gap, heads", [*[(*s, 2) for s in SMALL], (8192, 17.8, 520), (1000, 14.0, 520)])       # rows shared by two wavefronts or not
def test_many_small_weights_of_a_prompt(tokens, gap, heads, of_sink):
    q, k, v = _sink(np.random.default_rng(heads), tokens, 1, heads, gap, of_sink)
    out = gq.gqsa_prompt_attend(dev(q), dev(k), dev(v), ints(0, 1), ints(0, tokens), scale=1.0).cpu().numpy()
    want, size = ref.attention(q, k, v, 1.0, [tokens])
    _check_sum_of_small(out, want, size, tokens, v)


# ----------------------------------------------------------------------------- infinite values
@pytest.mark.parametrize("heads", [2, 96])          # rows shared by two wavefronts or not
@pytest.mark.parametrize("dim", [64, 128])
def test_infinite_values_of_any_weight(dim, heads):
    """An infinite value that a row sees makes the element infinite and a NaN, or two infinities of different signs, make it NaN, even where the weight is far below
    what 32 bits hold, wherever the key lies among those that the row sees."""
    rng = np.random.default_rng(dim)
    rows = 400
    q, k, v = normal(rng, rows, heads, dim), normal(rng, rows, 1, dim), normal(rng, rows, 1, dim)
    q[:, :, 0], k[:, :, 0] = 8, 0
    low = [3, 70, 71, 200, 390]
    k[low, :, 0] = -400                                        # scores of -3200 and less
    k[low, :, 1:] = 0
    v[3, 0, 5], v[70, 0, 6], v[71, 0, 6], v[70, 0, 7], v[71, 0, 7] = np.inf, -np.inf, -np.inf, np.inf, -np.inf
    v[200, 0, 8], v[390, 0, 9], v[390, 0, 10] = np.nan, -np.inf, np.inf
    v[100, 0, 11] = -np.inf                                    # (of a weight like the others')
    starts = ints(0, rows)
    out = gq.gqsa_prompt_attend(dev(q), dev(k), dev(v), starts, starts, scale=1.0).cpu().numpy()
    special = np.zeros(out.shape, bool)
    for element, first, value in [(5, 3, np.inf), (6, 70, -np.inf), (7, 71, np.nan), (8, 200, np.nan), (9, 390, -np.inf), (10, 390, np.inf), (11, 100, -np.inf)]:
        special[first:, :, element] = True
        assert np.array_equal(out[first:, :, element], np.full((rows - first, heads), value), equal_nan=True), element
    assert (out[70, :, 7] == np.inf).all()
    special[70, :, 7] = True
    finite = np.where(np.isfinite(v), v, 0)
    want = gq.gqsa_prompt_attend(dev(q), dev(k), dev(finite), starts, starts, scale=1.0).cpu().numpy()
    assert np.array_equal(out[~special], want[~special])
    heads_checked = slice(0, 2)
    _check_prompts(want[:, heads_checked], q[:, heads_checked], k, finite, [0, rows], [0, rows], 1.0)


# ----------------------------------------------------------------------------- the example
@pytest.mark.parametrize("tokens, prompts", [(1, "64,3"), (2, "63,64")])
def test_example_command_with_few_tokens(monkeypatch, capsys, tokens, prompts):
    from paper_2412_17560_amd import attention_layer
    monkeypatch.setattr("sys.argv", ["attention_layer", "--hidden", "512", "--heads", "8", "--kv-heads", "2", "--head-dim", "64",
                                     "--prompts", prompts, "--tokens", str(tokens)])
    attention_layer.main()
    printed = capsys.readouterr().out
    assert "prompts of" in printed and "cache" in printed and ("us a step" in printed) == (tokens > 1)


def test_a_layer_without_rows():
    import gqsa_inputs as gi
    from paper_2412_17560_amd.attention_layer import AttentionLayer, rotary_table

    hidden, heads, kv_heads, dim = 256, 4, 2, 64
    sizes = [(heads * dim, hidden), (kv_heads * dim, hidden), (kv_heads * dim, hidden), (hidden, heads * dim)]
    c = Cached([0, 0], kv_heads, dim, 32, room=64)
    layer = AttentionLayer(*[gq.gqsa_pack(gi.dense_weight(n, k, seed=i), 16, 4, 0.5) for i, (n, k) in enumerate(sizes)], heads, rotary_table(64, dim), c.cache)
    x = torch.empty((0, hidden), dtype=torch.float16, device="cuda")
    assert layer.prompt(x, ints(), dev(c.pages), ints(0, 0, 0), ints(0, 0)).shape == (0, hidden)


# ----------------------------------------------------------------------------- more than 64 sequences, and the queries of a layer
@pytest.mark.parametrize("dim, q_heads, kv_heads, count, least", [
    (64, 4, 2, 130, 1), (128, 1, 1, 65, 1), (64, 24, 8, 200, 1),
    (64, 8, 2, 75, 130)])                                      # as long as those whose blocks are mixed, but for their number
def test_prompts_of_many_sequences(dim, q_heads, kv_heads, count, least):
    """More sequences than a wavefront has lanes, some without rows, some without keys, some with an earlier part."""
    rng = np.random.default_rng(count)
    q_rows = [0 if b % 7 == 3 else least + (29 * b) % 70 for b in range(count)]
    q_rows[64] = 150
    k_rows = [0 if b % 11 == 5 else n + (b % 3) * 20 for b, n in enumerate(q_rows)]
    q, k, v = normal(rng, sum(q_rows), q_heads, dim), normal(rng, sum(k_rows), kv_heads, dim), normal(rng, sum(k_rows), kv_heads, dim)
    qs, ks = (np.cumsum([0] + n).astype(np.int32) for n in (q_rows, k_rows))
    out = torch.full(q.shape, 9.0, dtype=torch.float16, device="cuda")
    gq.gqsa_prompt_attend(dev(q), dev(k), dev(v), dev(qs), dev(ks), out=out)
    _check_prompts(out.cpu().numpy(), q, k, v, qs, ks, dim ** -0.5)


def test_queries_that_a_layer_attends_with():
    """What both attentions get are the normed and rotated queries, of the rows' own positions, with the queries' own weights."""
    import gqsa_inputs as gi
    from paper_2412_17560_amd.attention_layer import AttentionLayer, rotary_table

    hidden, heads, kv_heads, dim, counts = 256, 4, 2, 64, [37, 5]
    sizes = [(heads * dim, hidden), (kv_heads * dim, hidden), (kv_heads * dim, hidden), (hidden, heads * dim)]
    c = Cached([0, 0], kv_heads, dim, 32, room=64)
    norms = [normal(c.rng, dim) for _ in range(2)]
    table = rotary_table(64, dim)
    layer = AttentionLayer(*[gq.gqsa_pack(gi.dense_weight(n, k, seed=i), 16, 4, 0.5) for i, (n, k) in enumerate(sizes)], heads, table, c.cache,
                           *map(dev, norms))
    starts = np.cumsum([0] + counts).astype(np.int32)
    positions = np.concatenate([np.arange(n) for n in counts]).astype(np.int32)
    seen = []

    def watch(original, place):
        def call(*args, **kw):
            seen.append(args[place].cpu().numpy().copy())
            return original(*args, **kw)
        return call

    with pytest.MonkeyPatch.context() as m:
        for name, place in (("gqsa_qk_norm_rotate", 0), ("gqsa_prompt_attend", 0), ("gqsa_cache_attend", 1)):
            m.setattr(gq, name, watch(getattr(gq, name), place))
        layer.prompt(dev(normal(c.rng, sum(counts), hidden)), dev(positions), dev(c.pages), dev(starts), ints(*counts))
        layer.step(dev(normal(c.rng, 2, hidden)), ints(*counts), dev(c.pages), ints(*(n + 1 for n in counts)))
    assert len(seen) == 4
    for raw, turned, where in ((seen[0], seen[1], positions), (seen[2], seen[3], np.array(counts))):
        assert np.abs(raw).max() > 0
        _check_rotated(turned, raw, positions=where, table=table.cpu().numpy(), weight=norms[0])
