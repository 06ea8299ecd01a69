"""The operators between the q/k/v and the o product of a decoder layer against float64, on the GPU."""
from __future__ import annotations

import ctypes as C

import numpy as np
import pytest

import paper_2412_17560_amd as gq
from oracle import attention as ref
from paper_2412_17560_amd import binding

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def ints(*values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def normal(rng, *shape):
    return rng.standard_normal(shape).astype(np.float16)


# ----------------------------------------------------------------------------- norm and rotation
def _table(n, half):
    angle = np.arange(n)[:, None] * 10000.0 ** (-np.arange(half) / max(half, 1))
    return np.stack([np.cos(angle), np.sin(angle)], axis=-1).astype(np.float32)


def _check_rotated(got, x, **kw):
    """Rounded once (2^-11 of the result, half a subnormal step), from fp32: no more than 16 roundings (2^-20) of the terms."""
    want, size = ref.norm_rotate(x, **kw)
    error = np.abs(got.astype(np.float64) - want)
    assert (error <= 2.0 ** -11 * np.abs(want) + 2.0 ** -20 * size + 2.0 ** -25).all(), error.max()


@pytest.mark.parametrize("rows, q_heads, k_heads, dim, rotary, interleaved, norm", [
    (1, 32, 32, 128, 128, False, True),
    (1, 1, 1, 16, 16, True, True),
    (3, 5, 2, 64, 32, True, False),
    (7, 28, 4, 64, 64, False, True),
    (5, 3, 1, 80, 32, False, True),          # five runs of 16: lanes without any
    (4, 3, 3, 96, 96, True, True),
    (2, 9, 2, 256, 128, False, True),
    (6, 4, 1, 128, 0, False, True),          # no rotation
    (1500, 14, 2, 128, 64, False, True),     # sets of heads spread over wavefronts, and not all alike
    (9000, 9, 2, 64, 64, True, True),        # a wavefront per row
])
def test_norm_rotate(rows, q_heads, k_heads, dim, rotary, interleaved, norm):
    rng = np.random.default_rng(rows + dim)
    q, k = normal(rng, rows, q_heads, dim), normal(rng, rows, k_heads, dim) * np.float16(5)
    wq, wk = (normal(rng, dim) if norm else None for _ in range(2))
    table = _table(97, rotary // 2) if rotary else None
    positions = rng.integers(0, 97, rows).astype(np.int32)
    got = gq.gqsa_qk_norm_rotate(dev(q), dev(k), dev(positions) if rotary else None, dev(table) if rotary else None,
                                 dev(wq) if norm else None, dev(wk) if norm else None, eps=1e-5, interleaved=interleaved)
    for y, x, w in zip(got, (q, k), (wq, wk)):
        _check_rotated(y.cpu().numpy(), x, positions=positions, table=table, weight=w, eps=1e-5, interleaved=interleaved)


@pytest.mark.parametrize("interleaved", [False, True])
def test_norm_rotate_in_place_in_a_joint_array_and_with_heads_outermost(interleaved):
    rng = np.random.default_rng(5)
    rows, dim = 33, 128
    table, positions = _table(64, 64), rng.integers(0, 64, rows).astype(np.int32)
    weight = normal(rng, dim)
    joint = normal(rng, rows, 12, dim)                                   # 8 query heads, 2 of keys, 2 of values
    y = dev(joint)
    gq.gqsa_qk_norm_rotate(y[:, :8], y[:, 8:10], dev(positions), dev(table), dev(weight), None, interleaved=interleaved,
                           q_out=y[:, :8], k_out=y[:, 8:10])
    got = y.cpu().numpy()
    assert np.array_equal(got[:, 10:], joint[:, 10:])
    _check_rotated(got[:, :8], joint[:, :8], positions=positions, table=table, weight=weight, interleaved=interleaved)
    _check_rotated(got[:, 8:10], joint[:, 8:10], positions=positions, table=table, interleaved=interleaved)
    x = dev(joint.transpose(1, 0, 2)).transpose(0, 1)                    # heads outermost in memory
    into = torch.full((rows, 8, dim + 8), 7.0, dtype=torch.float16, device="cuda")
    out, none = gq.gqsa_qk_norm_rotate(x[:, :8], None, dev(positions), dev(table), dev(weight), interleaved=interleaved,
                                       q_out=into[:, :, :dim])
    assert none is None and (into[:, :, dim:] == 7.0).all()
    assert np.array_equal(out.cpu().numpy(), got[:, :8])                 # the same bits, wherever they lie


def test_norm_rotate_positions_outside_the_table():
    x = np.ones((4, 2, 64), np.float16)
    positions = np.array([0, -1, 9, 8], np.int32)
    y, _ = gq.gqsa_qk_norm_rotate(dev(x), None, dev(positions), dev(_table(9, 16)))
    y = y.cpu().numpy()
    assert np.isfinite(y[[0, 3]]).all() and np.isfinite(y[..., 32:]).all() and np.isnan(y[1:3, :, :32]).all()


def test_norm_of_extremes():
    """The largest and the smallest numbers, a head of zeros, an infinity and a NaN: the sum of squares stays finite, the rest is the formula."""
    x = np.zeros((5, 1, 128), np.float16)
    x[0], x[1], x[3, 0, 7], x[4, 0, 9] = 65504, 6e-8, np.inf, np.nan
    w = np.ones(128, np.float16)
    y, _ = gq.gqsa_qk_norm_rotate(dev(x), None, None, None, dev(w), eps=1e-6)
    y = y.cpu().numpy()
    _check_rotated(y[:3], x[:3], weight=w, eps=1e-6)
    assert np.isnan(y[3, 0, 7]) and (np.delete(y[3, 0], 7) == 0).all() and np.isnan(y[4]).all()


# ----------------------------------------------------------------------------- the cache
class Cached:
    """A cache, and beside it what it should hold."""

    def __init__(self, lengths, kv_heads, dim, page_tokens=32, seed=0, spare=0, room=0):
        self.rng = np.random.default_rng(seed)
        self.kv_heads, self.dim, self.page = kv_heads, dim, page_tokens
        counts = [-(-(n + room) // page_tokens) for n in lengths]
        self.n_pages = max(1, sum(counts)) + spare
        order = self.rng.permutation(self.n_pages).astype(np.int32)
        self.pages = np.full((len(lengths), max([1, *counts])), -1, np.int32)
        at = 0
        for b, c in enumerate(counts):
            self.pages[b, :c] = order[at:at + c]
            at += c
        self.cache = gq.gqsa_cache_create(self.n_pages, page_tokens, kv_heads, dim)
        self.k, self.v = ([np.zeros((0, kv_heads, dim), np.float16) for _ in lengths] for _ in range(2))
        if any(lengths):
            self.append([self.some(n) for n in lengths], [self.some(n) for n in lengths])

    def some(self, n):
        x = self.rng.standard_normal((n, self.kv_heads, self.dim))
        x[..., ::17] *= 6
        return x.astype(np.float16)

    def lengths(self):
        return [len(k) for k in self.k]

    def append(self, ks, vs):
        self.k = [np.concatenate([a, b]) for a, b in zip(self.k, ks)]
        self.v = [np.concatenate([a, b]) for a, b in zip(self.v, vs)]
        starts = np.cumsum([0] + [len(k) for k in ks]).astype(np.int32)
        gq.gqsa_cache_append(self.cache, dev(np.concatenate(ks)), dev(np.concatenate(vs)), dev(self.pages), ints(*self.lengths()), dev(starts))

    def read(self, counts):
        starts = np.cumsum([0] + list(counts)).astype(np.int32)
        k, v = (torch.full((int(starts[-1]), self.kv_heads, self.dim), 3.0, dtype=torch.float16, device="cuda") for _ in range(2))
        gq.gqsa_cache_read(self.cache, dev(self.pages), ints(*self.lengths()), dev(starts), k, v)
        return [[a.cpu().numpy()[s:e] for s, e in zip(starts, starts[1:])] for a in (k, v)]

    def check(self):
        got_k, got_v = self.read(self.lengths())
        for got, held in ((got_k, self.k), (got_v, self.v)):
            for g, x in zip(got, held):
                want = ref.cache_values(x)
                assert np.array_equal(np.isnan(g), np.isnan(want))
                assert np.array_equal(np.nan_to_num(g), np.nan_to_num(want))


@pytest.mark.parametrize("dim, page, kv_heads, lengths", [
    (128, 32, 1, [1]), (64, 32, 3, [31, 0, 33]), (128, 64, 2, [64, 65, 1, 200]), (64, 256, 5, [257, 255, 256]), (128, 4096, 1, [4100])])
def test_cache_holds_what_the_definition_says(dim, page, kv_heads, lengths):
    Cached(lengths, kv_heads, dim, page, seed=dim + len(lengths), spare=2).check()


@pytest.mark.parametrize("dim", [64, 128])
def test_appending_in_pieces_is_appending_at_once(dim):
    c = Cached([5, 0, 40], 2, dim, 32, seed=7, spare=1, room=120)
    for counts in ([1, 1, 1], [0, 30, 26], [1, 0, 33], [63, 2, 1], [1, 1, 1]):
        c.append([c.some(n) for n in counts], [c.some(n) for n in counts])
    c.check()


def test_one_row_per_sequence_needs_no_starts_and_strides_do_not_matter():
    c = Cached([31, 32, 0], 2, 128, 32, seed=3, room=1)
    joint = normal(c.rng, 3, 7, 128)
    c.k, c.v = ([np.concatenate([x, joint[b:b + 1, h:h + 2]]) for b, x in enumerate(held)] for held, h in ((c.k, 2), (c.v, 5)))
    y = dev(joint)
    gq.gqsa_cache_append(c.cache, y[:, 2:4], y[:, 5:7], dev(c.pages), ints(*c.lengths()))
    c.check()


def test_groups_without_width_and_groups_that_are_not_finite():
    c = Cached([0], 1, 128, 32, room=64)
    k, v = c.some(40), c.some(40)
    for x in (k, v):
        x[0, 0, :32] = 2.5                              # all alike
        x[1, 0, 32:64] = 0
        x[2, 0, 5] = np.inf
        x[3, 0, 70], x[33, 0, 127] = np.nan, -np.inf
        x[4, 0, :32] = np.linspace(-65504, 65504, 32).astype(np.float16)
        x[5, 0, :32] = np.arange(32, dtype=np.float16) * np.float16(6e-8)       # steps below the smallest fp16 number
        x[6, 0, 0:32] = (1000 + np.arange(32) % 2).astype(np.float16)
    c.append([k], [v])
    c.check()


def test_reading_rows_that_no_token_stands_behind():
    c = Cached([3, 40], 1, 64, 32, seed=1)
    (a, b), _ = c.read([5, 2])
    assert (a[:2] == 0).all() and np.array_equal(a[2:], ref.cache_values(c.k[0])) and np.array_equal(b, ref.cache_values(c.k[1][-2:]))
    page = c.pages[1, 0]
    c.pages[1, 0] = c.n_pages                           # outside the cache: absent
    (_, b), _ = c.read([1, 40])
    assert (b[:32] == 0).all() and np.array_equal(b[32:], ref.cache_values(c.k[1][32:]))
    more = [c.some(0), c.some(3)]
    c.pages[1, 1] = -5
    gq.gqsa_cache_append(c.cache, dev(more[1]), dev(more[1]), dev(c.pages), ints(3, 43), ints(0, 0, 3))     # written nowhere
    c.pages[1] = page, c.pages[1, 1]
    (_, b), _ = c.read([0, 40])
    assert np.array_equal(b[:32], ref.cache_values(c.k[1][:32])) and (b[32:] == 0).all()


def test_cache_info():
    c = gq.gqsa_cache_create(7, 64, 3, 128)
    info = gq.gqsa_cache_info(c)
    assert info["token_bytes"] == 160 and info["device_bytes"] == 7 * 64 * 3 * 160 and info["page_tokens"] == 64
    gq.gqsa_cache_free(c)
    gq.gqsa_cache_free(c)


def test_a_cache_that_does_not_fit_leaves_no_error_behind():
    with pytest.raises(RuntimeError):
        gq.gqsa_cache_create(2 ** 30, 4096, 1024, 128)
    assert int(torch.ones(5, device="cuda").sum()) == 5
    Cached([40], 1, 64, 32).check()


# ----------------------------------------------------------------------------- attention over the cache
def _check_attended(got, want, size, tokens, values):
    """Each weight and the result are rounded to fp16 (2^-11 each, of what they make up), a weight below the normal range by up to 2^-25 of the
    largest; fp32 scores, exponentials and sums stay below 2^-14 of the size together."""
    error = np.abs(got.astype(np.float64) - want)
    bound = (2.0 ** -10 + 2.0 ** -14) * size + tokens * 2.0 ** -25 * (np.abs(values).max() if values.size else 0) + 2.0 ** -25
    assert (error <= bound).all(), (error - bound).max()


def _attend_all(c, q_rows, q_heads, scale=None, **kw):
    q = [normal(c.rng, n, q_heads, c.dim) for n in q_rows]
    starts = np.cumsum([0] + list(q_rows)).astype(np.int32)
    out = torch.full((int(starts[-1]), q_heads, c.dim), 9.0, dtype=torch.float16, device="cuda")
    got = gq.gqsa_cache_attend(c.cache, dev(np.concatenate(q)), dev(c.pages), ints(*c.lengths()), dev(starts), scale=scale, out=out, **kw)
    assert got is out
    return q, [out.cpu().numpy()[s:e] for s, e in zip(starts, starts[1:])]


def _check_cache(c, q, out, scale=None):
    for qb, got, k, v in zip(q, out, c.k, c.v):
        n, rows = len(k), len(qb)
        hk, hv = ref.cache_values(k), ref.cache_values(v)
        want, size = ref.attention(qb, hk, hv, c.dim ** -0.5 if scale is None else scale, [n - rows + i + 1 for i in range(rows)])
        _check_attended(got, want, size, n, hv)


@pytest.mark.parametrize("dim, page, q_heads, kv_heads, lengths, rows", [
    (128, 32, 1, 1, [1], [1]),
    (128, 32, 4, 4, [31, 32, 33, 0], [1, 1, 1, 1]),            # a sequence without tokens
    (64, 64, 8, 2, [127, 128, 129], [1, 1, 1]),
    (128, 64, 14, 2, [300, 1, 700], [1, 1, 1]),                # seven heads to one
    (64, 32, 16, 1, [513], [1]),                               # sixteen heads to one
    (128, 128, 40, 2, [90, 1000], [1, 1]),                     # twenty: more than one block of rows
    (128, 32, 8, 2, [40, 5, 333, 64], [5, 5, 0, 3]),           # several rows, none, as many as tokens
    (64, 32, 4, 4, [50, 3], [40, 7]),                          # more rows than a block holds; more rows than tokens
    (128, 256, 8, 8, [5000], [2]),                             # split over the length
    (64, 32, 6, 3, [2500, 10, 1200], [1, 4, 17]),
])
def test_attention_over_the_cache(dim, page, q_heads, kv_heads, lengths, rows):
    c = Cached(lengths, kv_heads, dim, page, seed=sum(lengths), spare=1)
    q, out = _attend_all(c, rows, q_heads)
    _check_cache(c, q, out)
    _, again = _attend_all(c, rows, q_heads)                   # (other queries in between)
    starts = np.cumsum([0] + list(rows)).astype(np.int32)
    twice = gq.gqsa_cache_attend(c.cache, dev(np.concatenate(q)), dev(c.pages), ints(*lengths), dev(starts)).cpu().numpy()
    assert np.array_equal(twice, np.concatenate(out))          # the same bits from run to run


@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0])
def test_scales(scale):
    c = Cached([200, 33], 2, 64, 32, seed=9)
    q, out = _attend_all(c, [1, 2], 4, scale=scale)
    _check_cache(c, q, out, scale)


def test_many_sequences():
    lengths = [(7 * b) % 90 for b in range(150)]
    c = Cached(lengths, 1, 64, 32, seed=4)
    q, out = _attend_all(c, [1 if b % 5 else 0 for b in range(150)], 2)
    _check_cache(c, q, out)


@pytest.mark.parametrize("kv_heads, lengths", [
    (1, [131000]),              # one head over all workgroups
    (1, [70001]),
    (8, [16500]),               # heads over 65 of them, the last of which is the next one's first
    (3, [51500]),
    (2, [300, 68000, 900]),
])
def test_one_head_over_many_workgroups(kv_heads, lengths):
    """Equal weights, which are exact, and values that rise along the sequence: a part that is missing, or counted for another, shows."""
    c = Cached([0] * len(lengths), kv_heads, 64, 1024, seed=len(lengths), room=max(lengths))
    k, v = [c.some(n) for n in lengths], [c.some(n) for n in lengths]
    for x in v:
        x += (6 * np.linspace(-1, 1, len(x))[:, None, None] * np.arange(1, kv_heads + 1)[:, None]).astype(np.float16)
    c.append(k, v)
    rows = [1 + b % 2 for b in range(len(lengths))]
    for _ in range(3):                                         # (and leaves nothing behind for the next call)
        q, out = _attend_all(c, rows, 2 * kv_heads, scale=0.0)
        for qb, got, kb, vb in zip(q, out, c.k, c.v):
            n = len(kb)
            want, size = ref.attention(qb, ref.cache_values(kb), ref.cache_values(vb), 0.0, [n - len(qb) + i + 1 for i in range(len(qb))])
            assert (np.abs(got - want) <= (2.0 ** -11 + 2.0 ** -14) * size).all()
    q, out = _attend_all(c, rows, 2 * kv_heads)
    _check_cache(c, q, out)


def test_more_steps_than_workgroups_twice():
    c = Cached([650 + 3 * b for b in range(40)], 8, 64, 32, seed=3)
    q, out = _attend_all(c, [1] * 40, 8)
    _check_cache(c, q, out)


def test_more_pages_than_a_wavefront_holds_at_once():
    """The same 40 pages over and over, in random order, some absent: every workgroup has 65 steps and more of one sequence."""
    n, count = 33000, 130
    c = Cached([1280], 1, 64, 32, seed=15)
    held = [np.concatenate([ref.cache_values(x[0]), np.zeros((32, 1, 64))]).reshape(41, 32, 64) for x in (c.k, c.v)]
    place = {page: i for i, page in enumerate(c.pages[0])}
    table = c.rng.integers(0, c.n_pages, (count, -(-n // 32))).astype(np.int32)
    table[c.rng.random(table.shape) < 0.1] = -1
    q = normal(c.rng, count, 2, 64)
    out = gq.gqsa_cache_attend(c.cache, dev(q), dev(table), ints(*[n - 7 * b for b in range(count)])).cpu().numpy()
    for b in range(0, count, 3):
        at = np.array([place.get(page, 40) for page in table[b]])
        there = np.repeat(at < 40, 32)[:n - 7 * b]
        k, v = (x[at].reshape(-1, 1, 64)[:n - 7 * b][there] for x in held)
        want, size = ref.attention(q[b:b + 1], k, v, 0.125, [len(k)])
        _check_attended(out[b:b + 1], want, size, len(k), v)


def test_one_row_per_sequence_and_strided_queries():
    c = Cached([100, 7], 2, 128, 32, seed=8)
    joint = normal(c.rng, 2, 8, 128)
    y = torch.zeros((4, 2, 128), dtype=torch.float16, device="cuda").transpose(0, 1)       # heads outermost
    gq.gqsa_cache_attend(c.cache, dev(joint)[:, 2:6], dev(c.pages), ints(*c.lengths()), out=y)
    _check_cache(c, [joint[:1, 2:6], joint[1:, 2:6]], [y[:1].cpu().numpy(), y[1:].cpu().numpy()])


def test_scores_that_rise_and_fall_far():
    """The running maximum moves by far more than the slack from tile to tile, upwards and downwards."""
    c = Cached([0], 1, 128, 32, seed=2, room=1000)
    k, v = c.some(1000), c.some(1000)
    k *= (0.2 + 4.0 * np.abs(np.sin(np.arange(1000) / 50.0)))[:, None, None].astype(np.float16)
    c.append([k], [v])
    q, out = _attend_all(c, [3], 4, scale=0.5)
    _check_cache(c, q, out, 0.5)


def test_what_lies_behind_the_last_token_does_not_matter():
    """The pages hold older tokens with NaN and infinities there; and a NaN that a later row may see does not reach an earlier one."""
    c = Cached([0], 2, 128, 64, seed=6, room=128)
    wild = c.some(128)
    wild[60:] = np.nan
    gq.gqsa_cache_append(c.cache, dev(wild), dev(wild), dev(c.pages), ints(128), ints(0, 128))
    c.append([c.some(70)], [c.some(70)])
    q, out = _attend_all(c, [4], 8)
    assert np.isfinite(out[0]).all()
    _check_cache(c, q, out)
    k, v = c.some(3), c.some(3)
    v[1, 0, 40] = np.inf                                       # the second of three new tokens: its group is NaN
    c.append([k], [v])
    q, (out,) = _attend_all(c, [3], 8)
    assert np.isfinite(out[0]).all() and np.isfinite(out[:, 4:]).all()
    assert np.isnan(out[1:, :4, 32:64]).all() and np.isfinite(np.delete(out[1:, :4], np.arange(32, 64), axis=2)).all()
    finite = [np.where(np.isfinite(x), x, 0) for x in c.v]
    want, size = ref.attention(q[0][:1], ref.cache_values(c.k[0]), ref.cache_values(finite[0]), 128 ** -0.5, [71])
    _check_attended(out[:1], want, size, 71, finite[0])


def test_nan_keys_reach_the_rows_that_see_them():
    c = Cached([40], 1, 64, 32, seed=6, room=3)
    k = c.some(3)
    k[1, 0, 3] = np.nan
    c.append([k], [c.some(3)])
    _, (out,) = _attend_all(c, [3], 2)
    assert np.isfinite(out[0]).all() and np.isnan(out[1:]).all()


def test_infinite_queries_are_nan_where_they_see_a_token():
    c = Cached([40, 0, 300], 1, 64, 32, seed=16)
    q = normal(c.rng, 3, 3, 64)
    q[:, 0, 5], q[:, 1, 9] = np.inf, -np.inf
    out = gq.gqsa_cache_attend(c.cache, dev(q), dev(c.pages), ints(*c.lengths())).cpu().numpy()
    assert np.isnan(out[::2, :2]).all() and (out[1] == 0).all()
    _check_cache(c, [x[None, 2:] for x in q], [x[None, 2:] for x in out])


def test_absent_pages_are_absent_tokens():
    c = Cached([300], 2, 64, 32, seed=5)
    c.pages[0, 2], c.pages[0, 5] = -1, c.n_pages
    there = np.ones(300, bool)
    there[64:96] = there[160:192] = False
    q, (out,) = _attend_all(c, [1], 4)
    want, size = ref.attention(q[0], ref.cache_values(c.k[0][there]), ref.cache_values(c.v[0][there]), 64 ** -0.5, [300])
    _check_attended(out, want, size, 300, c.v[0])
    c.pages[:] = -1
    _, (out,) = _attend_all(c, [1], 4)
    assert (out == 0).all()


def test_lengths_and_starts_beyond_their_arrays_stay_inside():
    c = Cached([64, 64], 1, 64, 32, seed=11)
    q = dev(normal(c.rng, 3, 2, 64))
    room = torch.full((5, 2, 64), 4.0, dtype=torch.float16, device="cuda")
    gq.gqsa_cache_attend(c.cache, q, dev(c.pages), ints(10 ** 6, -3), ints(0, 2, 900), out=room[1:4])
    assert (room[0] == 4).all() and (room[4] == 4).all()
    want, size = ref.attention(q[:2].cpu().numpy(), ref.cache_values(c.k[0]), ref.cache_values(c.v[0]), 0.125, [63, 64])
    _check_attended(room[1:3].cpu().numpy(), want, size, 64, c.v[0])
    assert (room[3] == 0).all()
    k = dev(c.some(3))
    gq.gqsa_cache_append(c.cache, k, k, dev(c.pages), ints(10 ** 6, -3), ints(-7, 1, 900))
    torch.cuda.synchronize()


def test_pages_beyond_four_gigabytes():
    """Offsets that pass 32 bits: the last pages of a cache of 5 GB."""
    page_bytes = 256 * 160 * 2
    c = Cached([600], 2, 128, 256, seed=12)
    big = gq.gqsa_cache_create(5 * 2 ** 30 // page_bytes + 1, 256, 2, 128)
    n = gq.gqsa_cache_info(big)["n_pages"]
    c.cache, c.n_pages = big, n
    c.pages[0] = [n - 1, 0, n - 2]
    k, v = c.k[0], c.v[0]
    c.k, c.v = [k[:0]], [v[:0]]
    c.append([k], [v])
    c.check()
    q, out = _attend_all(c, [2], 8)
    _check_cache(c, q, out)
    gq.gqsa_cache_free(big)


def test_decode_steps_in_a_graph_and_on_another_stream():
    """Append and attend, captured once; every replay has new inputs, lengths and pages, with eager work between the replays."""
    c = Cached([37, 5], 2, 128, 32, seed=13, room=70)
    other = torch.cuda.Stream()
    pages, lengths = dev(c.pages), ints(*c.lengths())
    q, k, v = (torch.zeros((2, h, 128), dtype=torch.float16, device="cuda") for h in (8, 2, 2))
    out = torch.zeros_like(q)

    def step():
        gq.gqsa_cache_append(c.cache, k, v, pages, lengths)
        gq.gqsa_cache_attend(c.cache, q, pages, lengths, out=out)
    other.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=other):
        step()
    for i in range(60):
        new = [normal(c.rng, 2, h, 128) for h in (8, 2, 2)]
        for t, x in zip((q, k, v), new):
            t.copy_(dev(x))
        c.k = [np.concatenate([a, new[1][b:b + 1]]) for b, a in enumerate(c.k)]
        c.v = [np.concatenate([a, new[2][b:b + 1]]) for b, a in enumerate(c.v)]
        lengths.copy_(ints(*c.lengths()))
        graph.replay()
        if i % 12 == 0:
            got = out.cpu().numpy()
            _check_cache(c, [new[0][:1], new[0][1:]], [got[:1], got[1:]])
            eager = gq.gqsa_cache_attend(c.cache, q, pages, lengths)
            assert torch.equal(eager, out)
            other.wait_stream(torch.cuda.current_stream())
            elsewhere = gq.gqsa_cache_attend(c.cache, q, pages, lengths, stream=other)
            torch.cuda.current_stream().wait_stream(other)
            assert torch.equal(elsewhere, eager)
    c.check()


# ----------------------------------------------------------------------------- attention over prompts
def _prompts(rng, q_rows, k_rows, q_heads, kv_heads, dim):
    q, k, v = normal(rng, sum(q_rows), q_heads, dim), normal(rng, sum(k_rows), kv_heads, dim), normal(rng, sum(k_rows), kv_heads, dim)
    starts = [np.cumsum([0] + list(n)).astype(np.int32) for n in (q_rows, k_rows)]
    return q, k, v, *starts


def _check_prompts(out, q, k, v, q_starts, k_starts, scale):
    for b in range(len(q_starts) - 1):
        qb, kb, vb = (x[s[b]:s[b + 1]] for x, s in ((q, q_starts), (k, k_starts), (v, k_starts)))
        rows, keys = len(qb), len(kb)
        want, size = ref.attention(qb, kb, vb, scale, [keys - rows + i + 1 for i in range(rows)])
        _check_attended(out[q_starts[b]:q_starts[b + 1]], want, size, keys, vb)


@pytest.mark.parametrize("dim, q_heads, kv_heads, q_rows, k_rows", [
    (128, 1, 1, [1], [1]),
    (64, 2, 1, [15], [15]),
    (128, 4, 2, [63, 64, 65, 0, 1], [63, 64, 65, 0, 1]),
    (64, 3, 3, [127, 128, 129], [127, 128, 129]),
    (128, 8, 1, [300], [300]),                               # heads a multiple of 8
    (128, 7, 1, [33, 200], [33, 200]),
    (64, 4, 4, [1, 40, 130], [100, 41, 500]),                # an earlier part of the prompt in front
    (128, 2, 2, [50, 140, 3], [20, 0, 1]),                   # rows that see no key
])
def test_attention_over_prompts(dim, q_heads, kv_heads, q_rows, k_rows):
    rng = np.random.default_rng(sum(q_rows) + dim)
    q, k, v, qs, ks = _prompts(rng, q_rows, k_rows, q_heads, kv_heads, dim)
    out = torch.full(q.shape, 9.0, dtype=torch.float16, device="cuda")
    args = dev(q), dev(k), dev(v), dev(qs), dev(ks)
    gq.gqsa_prompt_attend(*args, out=out)
    _check_prompts(out.cpu().numpy(), q, k, v, qs, ks, dim ** -0.5)
    assert torch.equal(gq.gqsa_prompt_attend(*args), out)


@pytest.mark.parametrize("dim, q_heads, kv_heads, q_rows, k_rows", [
    (64, 64, 4, [300, 130], [300, 500]),
    (128, 96, 32, [200, 1, 70], [260, 300, 40]),
    (128, 270, 2, [129], [200]),
    (64, 64, 2, [300, 5, 0, 130, 700], [300, 400, 0, 20, 701]),       # blocks of the sequences mixed
    (128, 80, 8, [10, 400, 129, 128, 60, 257], [600, 400, 140, 128, 50, 257]),
    (64, 33, 3, [150 + (37 * b) % 200 for b in range(40)], [180 + (37 * b) % 200 for b in range(40)]),
])
def test_attention_over_prompts_with_many_heads(dim, q_heads, kv_heads, q_rows, k_rows):
    rng = np.random.default_rng(q_heads)
    q, k, v, qs, ks = _prompts(rng, q_rows, k_rows, q_heads, kv_heads, dim)
    out = gq.gqsa_prompt_attend(dev(q), dev(k), dev(v), dev(qs), dev(ks)).cpu().numpy()
    _check_prompts(out, q, k, v, qs, ks, dim ** -0.5)


@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0])
def test_prompt_scales(scale):
    q, k, v, qs, ks = _prompts(np.random.default_rng(1), [70, 9], [70, 20], 2, 1, 64)
    k *= (0.2 + np.abs(np.sin(np.arange(90) / 9.0)))[:, None, None].astype(np.float16)
    out = gq.gqsa_prompt_attend(dev(q), dev(k), dev(v), dev(qs), dev(ks), scale=scale).cpu().numpy()
    _check_prompts(out, q, k, v, qs, ks, scale)


def test_prompts_in_a_joint_array_and_with_heads_outermost():
    rng = np.random.default_rng(3)
    joint = normal(rng, 150, 12, 128)                        # 8 query heads, 2 of keys, 2 of values
    starts = np.array([0, 100, 150], np.int32)
    y = dev(joint)
    out = torch.zeros((8, 150, 128), dtype=torch.float16, device="cuda").transpose(0, 1)
    gq.gqsa_prompt_attend(y[:, :8], y[:, 8:10], y[:, 10:], dev(starts), dev(starts), out=out)
    _check_prompts(out.cpu().numpy(), joint[:, :8], joint[:, 8:10], joint[:, 10:], starts, starts, 128 ** -0.5)
    z = dev(joint.transpose(1, 0, 2)).transpose(0, 1)
    assert torch.equal(gq.gqsa_prompt_attend(z[:, :8], z[:, 8:10], z[:, 10:], dev(starts), dev(starts)), out)


@pytest.mark.parametrize("dim", [64, 128])
def test_keys_and_values_that_a_row_does_not_see_have_no_effect(dim):
    """NaN and infinities in other sequences and in later tokens of the row's own: the rows ahead of them keep their bits."""
    rng = np.random.default_rng(dim)
    q, k, v, qs, ks = _prompts(rng, [90, 150], [90, 170], 4, 2, dim)
    clean = gq.gqsa_prompt_attend(dev(q), dev(k), dev(v), dev(qs), dev(ks)).cpu().numpy()
    k2, v2 = k.copy(), v.copy()
    k2[90 + 120] = np.nan                                    # seen from row 100 of the second sequence on
    v2[90 + 60, 0, 5], v2[90 + 61, 1, 7] = np.inf, np.nan    # from rows 40 and 41 on
    v2[88, 1, 3] = -np.inf                                   # row 88 of the first
    out = gq.gqsa_prompt_attend(dev(q), dev(k2), dev(v2), dev(qs), dev(ks)).cpu().numpy()
    touched = np.zeros(q.shape, bool)
    touched[90 + 100:] = True
    touched[90 + 40:, :2, 5] = touched[90 + 41:, 2:, 7] = True
    touched[88:90, 2:, 3] = True
    assert np.array_equal(out[~touched], clean[~touched])
    assert not np.isfinite(out[touched]).any()
    assert (out[88:90, 2:, 3] == -np.inf).all() and (out[90 + 40:90 + 100, :2, 5] == np.inf).all()


def test_prompt_scores_of_infinity():
    """All scores of a row -infinity, or one +infinity: NaN, as the formula's; some -infinity: weights of 0."""
    q, k, v, qs, ks = _prompts(np.random.default_rng(5), [3, 200], [2, 200], 2, 1, 64)
    q, k = np.abs(q) + np.float16(0.1), np.abs(k) + np.float16(0.1)
    k[0, 0, 7] = k[2, 0, 3] = k[100, 0, 1] = -np.inf
    out = gq.gqsa_prompt_attend(dev(q), dev(k), dev(v), dev(qs), dev(ks)).cpu().numpy()
    assert (out[0] == 0).all() and np.isnan(out[1]).all() and np.isnan(out[3]).all()
    for r, at in [(2, [1]), *[(3 + r, [2 + i for i in range(r + 1) if i not in (0, 98)]) for r in (1, 60, 98, 99, 199)]]:
        want, size = ref.attention(q[r:r + 1], k[at], v[at], 0.125, [len(k[at])])
        _check_attended(out[r:r + 1], want, size, len(k[at]), v[at])
    k[np.isinf(k)] = 1
    q[50, 0, 3] = np.inf
    out = gq.gqsa_prompt_attend(dev(q), dev(k), dev(v), dev(qs), dev(ks)).cpu().numpy()
    assert np.isnan(out[50, 0]).all() and np.isfinite(np.delete(out.reshape(-1, 64), 100, axis=0)).all()


@pytest.mark.parametrize("dim", [64, 128])
def test_what_a_row_does_not_see_with_many_heads(dim):
    rng = np.random.default_rng(dim + 1)
    q, k, v, qs, ks = _prompts(rng, [90, 150], [90, 170], 96, 2, dim)
    clean = gq.gqsa_prompt_attend(dev(q), dev(k), dev(v), dev(qs), dev(ks)).cpu().numpy()
    k2, v2 = k.copy(), v.copy()
    k2[90 + 160, 0] = np.nan                                 # seen from row 140 of the second sequence on
    v2[90 + 60, 0, 5], v2[90 + 61, 1, 7], v2[90 + 130, 1, 7] = np.inf, -np.inf, np.inf      # from rows 40, 41 and 110 on
    out = gq.gqsa_prompt_attend(dev(q), dev(k2), dev(v2), dev(qs), dev(ks)).cpu().numpy()
    touched = np.zeros(q.shape, bool)
    touched[90 + 140:, :48] = touched[90 + 40:, :48, 5] = touched[90 + 41:, 48:, 7] = True
    assert np.array_equal(out[~touched], clean[~touched])
    assert np.isnan(out[90 + 140:, :48]).all() and (out[90 + 40:90 + 140, :48, 5] == np.inf).all()
    assert (out[90 + 41:90 + 110, 48:, 7] == -np.inf).all() and np.isnan(out[90 + 110:, 48:, 7]).all()


def test_prompt_starts_beyond_their_arrays_stay_inside():
    rng = np.random.default_rng(0)
    q, k, v, _, _ = _prompts(rng, [40], [40], 2, 1, 64)
    room = torch.full((60, 2, 64), 4.0, dtype=torch.float16, device="cuda")
    gq.gqsa_prompt_attend(dev(q), dev(k), dev(v), ints(-9, 30, 10 ** 6), ints(-9, 30, 10 ** 6), out=room[10:50])
    out = room.cpu().numpy()
    assert (out[:10] == 4).all() and (out[50:] == 4).all()
    _check_prompts(out[10:50], q, k, v, [0, 30, 40], [0, 30, 40], 0.125)


def test_prompts_without_any_key():
    q = dev(normal(np.random.default_rng(2), 5, 4, 64))
    for k in (torch.zeros((0, 2, 64), dtype=torch.float16, device="cuda"), torch.zeros(0, dtype=torch.float16, device="cuda").as_strided((0, 2, 64), (0, 0, 0))):
        out = gq.gqsa_prompt_attend(q, k, k, ints(0, 3, 5), ints(0, 0, 0), out=torch.ones_like(q))
        assert (out == 0).all()


def test_prompt_through_the_cache_is_the_prompt():
    """A prompt's second part attends to the first as the cache gives it back: the same as the plain attention over those values."""
    c = Cached([200], 2, 128, 64, seed=21)
    (k,), (v,) = c.read([200])
    q = normal(c.rng, 70, 8, 128)
    out = gq.gqsa_prompt_attend(dev(q), dev(k), dev(v), ints(0, 70), ints(0, 200)).cpu().numpy()
    _check_prompts(out, q, ref.cache_values(c.k[0]), ref.cache_values(c.v[0]), [0, 70], [0, 200], 128 ** -0.5)


def test_no_rows_is_no_work():
    lib = binding._lib()
    c = gq.gqsa_cache_create(1, 32, 1, 64)
    assert lib.gqsa_cache_attend(c.ptr, None, 0, 0, 1, 0, None, 1, None, None, 1, 1.0, None, 0, 0, None) == 0
    empty = torch.empty((0, 1, 64), dtype=torch.float16, device="cuda")
    gq.gqsa_cache_append(c, empty, empty, ints(0).view(1, 1), ints(0), ints(0, 0))
    assert gq.gqsa_prompt_attend(empty, empty, empty, ints(0, 0), ints(0, 0)).shape == (0, 1, 64)
    assert gq.gqsa_qk_norm_rotate(empty, None, None, None)[0].shape == (0, 1, 64)
    assert isinstance(c.ptr, C.c_void_p)


@pytest.mark.parametrize("change, status", [
    (dict(q=None), 1), (dict(out=None), 1), (dict(pages=None), 1), (dict(lengths=None), 1), (dict(q_heads=3), 2), (dict(q_heads=0), 2),
    (dict(rows=-1), 2), (dict(rows=2), 2), (dict(n_seqs=0), 2), (dict(max_pages=0), 2), (dict(q_heads=2048), 3), (dict(n_seqs=65537), 3),
    (dict(max_pages=(1 << 20) + 1), 3), (dict(scale=float("inf")), 4), (dict(q_row=4), 8), (dict(lengths_off=2), 8), (dict(out_off=8), 8)])
def test_cache_attend_refuses(change, status):
    c = gq.gqsa_cache_create(1, 32, 2, 64)
    x = torch.zeros(1024, dtype=torch.float16, device="cuda").data_ptr()
    a = dict(q=x, q_row=256, q_head=64, q_heads=4, rows=1, pages=x, max_pages=1, lengths=x, starts=None, n_seqs=1, scale=0.1, out=x, out_row=256,
             out_head=64)
    change = dict(change)
    a["lengths"] += change.pop("lengths_off", 0)
    a["out"] += change.pop("out_off", 0)
    assert binding._lib().gqsa_cache_attend(c.ptr, *{**a, **change}.values(), None) == status


@pytest.mark.parametrize("change, status", [
    (dict(k=None), 1), (dict(v=None), 1), (dict(pages=None), 1), (dict(rows=-1), 2), (dict(rows=3), 2), (dict(n_seqs=0), 2), (dict(k_row=-64), 2),
    (dict(v_head=60), 8), (dict(n_seqs=65537), 3)])
def test_cache_copies_refuse(change, status):
    c = gq.gqsa_cache_create(1, 32, 2, 64)
    x = torch.zeros(1024, dtype=torch.float16, device="cuda").data_ptr()
    a = dict(k=x, k_row=128, k_head=64, v=x, v_row=128, v_head=64, rows=1, pages=x, max_pages=1, lengths=x, starts=None, n_seqs=1)
    for copy in (binding._lib().gqsa_cache_append, binding._lib().gqsa_cache_read):
        assert copy(c.ptr, *{**a, **change}.values(), None) == status


def test_the_binding_refuses():
    c = gq.gqsa_cache_create(2, 32, 2, 64)
    x, pages, one = (torch.zeros(s, dtype=d, device="cuda") for s, d in (((1, 2, 64), torch.float16), ((1, 2), torch.int32), ((1,), torch.int32)))
    for call in (lambda: gq.gqsa_cache_append(c, x[:, :1], x, pages, one), lambda: gq.gqsa_cache_append(c, x.float(), x.float(), pages, one),
                 lambda: gq.gqsa_cache_append(c, x, x, pages.long(), one), lambda: gq.gqsa_cache_append(c, x, x, pages[0], one),
                 lambda: gq.gqsa_cache_attend(c, x[..., :32], pages, one), lambda: gq.gqsa_cache_attend(c, x, pages, one, out=x[:, :1]),
                 lambda: gq.gqsa_cache_attend(c, x, pages, one, row_starts=one), lambda: gq.gqsa_cache_attend(c, x.cpu(), pages, one),
                 lambda: gq.gqsa_cache_attend(c, x.transpose(1, 2), pages, one), lambda: gq.gqsa_prompt_attend(x, x, x[..., :32], one, one),
                 lambda: gq.gqsa_prompt_attend(x, x, x, one, pages[0]), lambda: gq.gqsa_qk_norm_rotate(x, x[0], None, None),
                 lambda: gq.gqsa_qk_norm_rotate(x, None, None, torch.zeros((3, 32, 2), device="cuda")),
                 lambda: gq.gqsa_qk_norm_rotate(x, None, None, None, x[0, 0, :32])):
        with pytest.raises(ValueError):
            call()


# ----------------------------------------------------------------------------- all of it together
def test_layer_of_prompts_and_steps():
    """Products, norms, rotation, cache and attention as a decoder layer runs them: every stage against the definition, from the stage's own inputs."""
    import gqsa_inputs as gi
    import oracle
    from paper_2412_17560_amd.attention_layer import AttentionLayer, rotary_table

    hidden, heads, kv_heads, dim, counts = 256, 4, 2, 64, [37, 5]
    sizes = [(heads * dim, hidden), (kv_heads * dim, hidden), (kv_heads * dim, hidden), (hidden, heads * dim)]
    weights = [gi.dense_weight(n, k, seed=i) for i, (n, k) in enumerate(sizes)]
    packed = [oracle.pack(w, 16, 4, sparsity=0.5) for w in weights]
    c = Cached([0, 0], kv_heads, dim, 32, room=64)
    norms = [dev(normal(c.rng, dim)) for _ in range(2)]
    table = rotary_table(64, dim)
    layer = AttentionLayer(*[gq.gqsa_pack(w, 16, 4, 0.5) for w in weights], heads, table, c.cache, *norms)
    seen = {}

    def watch(name, original):
        def call(*args, **kw):
            inputs = [a.cpu().numpy().copy() if torch.is_tensor(a) else a for a in args]
            out = original(*args, **kw)
            seen[name] = inputs, out
            return out
        return call

    starts = np.cumsum([0] + counts).astype(np.int32)
    positions = np.concatenate([np.arange(n) for n in counts]).astype(np.int32)
    with pytest.MonkeyPatch.context() as m:
        for name in ("gqsa_qk_norm_rotate", "gqsa_cache_append", "gqsa_prompt_attend", "gqsa_cache_attend"):
            m.setattr(gq, name, watch(name, getattr(gq, name)))
        x = normal(c.rng, sum(counts), hidden)
        y = layer.prompt(dev(x), dev(positions), dev(c.pages), dev(starts), ints(*counts))
        prompt_seen = dict(seen)
        row = normal(c.rng, 2, hidden)
        z = layer.step(dev(row), ints(*counts), dev(c.pages), ints(*(n + 1 for n in counts)))

    def product(p, a):
        return np.stack([r for r in oracle.gemv(p, a)])

    for seen_now, rows, where in ((prompt_seen, x, positions), (seen, row, np.array(counts))):
        q, k = seen_now["gqsa_qk_norm_rotate"][0][:2]
        for got, p in ((q, packed[0]), (k, packed[1])):
            want = product(p, rows).reshape(got.shape)
            assert np.abs(got - want).max() <= 2e-3 * np.abs(want).max()
        turned = seen_now["gqsa_cache_append"][0][1]
        _check_rotated(turned, k, positions=where, table=table.cpu().numpy(), weight=norms[1].cpu().numpy())
    new = [(s["gqsa_cache_append"][0][1], s["gqsa_cache_append"][0][2]) for s in (prompt_seen, seen)]
    c.k, c.v = ([np.concatenate([new[0][i][starts[b]:starts[b + 1]], new[1][i][b:b + 1]]) for b in range(2)] for i in (0, 1))
    c.check()
    q, k, v = prompt_seen["gqsa_prompt_attend"][0][:3]
    attended = prompt_seen["gqsa_prompt_attend"][1].cpu().numpy()
    _check_prompts(attended, q, k, v, starts, starts, dim ** -0.5)
    step_q, step_out = seen["gqsa_cache_attend"][0][1], seen["gqsa_cache_attend"][1].cpu().numpy()
    _check_cache(c, [step_q[:1], step_q[1:]], [step_out[:1], step_out[1:]])
    for got, a in ((y, attended), (z, step_out)):
        want = product(packed[3], a.reshape(len(a), -1))
        assert np.abs(got.cpu().numpy() - want).max() <= 2e-3 * np.abs(want).max()


def test_example_command(monkeypatch, capsys):
    from paper_2412_17560_amd import attention_layer
    monkeypatch.setattr("sys.argv", ["attention_layer", "--hidden", "512", "--heads", "8", "--kv-heads", "2", "--head-dim", "64",
                                     "--prompts", "40,3", "--tokens", "5"])
    attention_layer.main()
    printed = capsys.readouterr().out
    assert "prompts of [40, 3]: 43 rows" in printed and "4 tokens for 2 sequences" in printed
