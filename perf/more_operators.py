"""A decoding step of several drafted tokens over the 4-bit cache, as cases that are timed one by one.

  append   queries and keys normed and rotated, keys and values into the cache on the way (gqsa_cache_append_rotated), and what the
           cache then stands for, read back (gqsa_cache_read)
  tree     attention of the newest rows over their cache, each row over the tokens before them all and those of its own ancestors
           in a tree of drafted tokens (gqsa_cache_attend_tree)
  verify   which drafted tokens the target's probabilities let stand, and the token behind them (gqsa_verify)
  keep     a tree's rows appended, the accepted ones made neighbours (gqsa_cache_keep), and the rows read back

Activations are fp16, probabilities fp32.  A tree's rows lie parents first; row 0 is the last token that is certain.

Norms: r = fp32(1 / sqrt(mean(x^2) + eps)) from 64 bits; x * (r * w), the rotation's products, its sum and its difference are one fp32
operation each, then one rounding to fp16: every rounding is given, as the 4-bit codes hang on the last bit.
The cache holds groups of 32 channels of one token and head: `low` = the least of them, `step` = fp16((greatest - low) / 15),
codes = min(15, round((x - low) / step)) (0 where step is 0), every operation a single fp32 operation; a code stands for
the fp16 number nearest to low + code * step.

Verification.  Row i of a sequence (token x, parent g) is accepted if u_i d < p, p = target[g][x], d = draft[i][x] where the tokens were
drawn from `draft` (a chain), else d = 1 less the target's probabilities of the children of g before i.  From row 0 on the first accepted child
follows.  Where none is, the next token is the first whose running sum of weights passes v times their sum; weights: target[g] less draft[i] of the
rejected row i, where that is positive, or target[g] without the tokens of g's children, or where those leave nothing target[g] itself.  Sums and products
are in 64 bits.
"""
from __future__ import annotations

import random

import numpy as np
import torch

own = False         # False: plain torch; True: the framework's operators

DEVICE = "cuda:0"
GROUP = 32
EPS = 1e-6
THETA = 10000.0


def _append(name, sequences, cached, new, q_heads, kv_heads, head_dim=128, rotary_dim=128, interleaved=False, norm=True, page_tokens=64,
            ragged=False):
    return {"name": name, "kind": "append", "sequences": sequences, "cached": cached, "new": new, "q_heads": q_heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "rotary_dim": rotary_dim, "interleaved": interleaved, "norm": norm, "page_tokens": page_tokens, "ragged": ragged}


def _tree(name, sequences, cached, new, q_heads, kv_heads, width=8, head_dim=128, page_tokens=64, ragged=False):
    return {"name": name, "kind": "tree", "sequences": sequences, "cached": cached, "new": new, "q_heads": q_heads, "kv_heads": kv_heads,
            "width": width, "head_dim": head_dim, "page_tokens": page_tokens, "ragged": ragged}


def _verify(name, sequences, new, vocabulary, drawn, width=1, truncated=False, ragged=False):
    return {"name": name, "kind": "verify", "sequences": sequences, "new": new, "vocabulary": vocabulary, "drawn": drawn, "width": width,
            "truncated": truncated, "ragged": ragged}


def _keep(name, sequences, cached, new, kv_heads, width=8, head_dim=128, page_tokens=64, ragged=False):
    return {"name": name, "kind": "keep", "sequences": sequences, "cached": cached, "new": new, "kv_heads": kv_heads, "width": width,
            "head_dim": head_dim, "page_tokens": page_tokens, "ragged": ragged}


def listed():
    return [
        # token generation, one sequence, a head of keys for every query head (hidden size 4096): launch and call overhead
        _append("append_step_b1", 1, 143, 1, 32, 32),
        # packed pieces of prompts of different lengths, small heads, half of the channels rotated in neighbouring pairs, no norms
        _append("append_ragged", 7, 200, 501, 28, 4, head_dim=64, rotary_dim=32, interleaved=True, norm=False, page_tokens=32, ragged=True),
        # a long prompt goes into the cache
        _append("append_prompt", 1, 0, 8192, 32, 8, page_tokens=128),
        # one short sequence and eight drafted tokens: launch and waits
        _tree("tree_b1_short", 1, 143, 8, 32, 32, width=3),
        # a few sequences of very different lengths, small heads, up to 13 drafted tokens
        _tree("tree_ragged", 7, 16003, 13, 28, 4, width=4, head_dim=64, page_tokens=32, ragged=True),
        # a batch of 16 with trees of 64: as many rows over each head of the cache as a block of a prompt has
        _tree("tree_b16", 16, 4096, 64, 32, 8, page_tokens=128),
        # one very long sequence, a tree of 16: split over its length
        _tree("tree_b1_long", 1, 131072, 16, 64, 8, width=5, page_tokens=256),
        # one sequence, four tokens of a chain that were drawn from the draft's probabilities
        _verify("verify_chain_b1", 1, 5, 32000, True),
        # a batch of 64 of these, the largest vocabulary here
        _verify("verify_chain_b64", 64, 5, 128256, True),
        # trees of the draft's most likely tokens, the target's probabilities cut off below
        _verify("verify_tree_b16", 16, 64, 128256, False, width=8, truncated=True),
        # one sequence, every head of keys for itself
        _keep("keep_b1", 1, 700, 8, 32, width=3),
        # a batch with larger trees
        _keep("keep_b16", 16, 2000, 64, 8, ragged=True),
    ]


def _log_uniform(rng, low, high):
    return max(1, int(round(low * (high / low) ** rng.random())))


HEADS = [(32, 32), (32, 8), (64, 8), (40, 40), (40, 8), (28, 4), (14, 2), (12, 12), (16, 1)]     # (queries, keys)
MOST_APPENDED = 8192 * 40 * 128         # elements of new queries and keys
MOST_CACHED = 131072 * 8 * 128          # elements of the keys that are attended to
MOST_SCORES = 16 * 32 * 64 * 4160       # (row, head, token) triples
MOST_PROBABILITIES = 16 * 64 * 128256


def draw(rng):
    """One more case of the ranges: one sequence to 64, an empty cache to a very long one, 1 row to 128 (of prompts 8192), 12 to 64 heads of 64 or
    128 channels, 1000 to 128256 tokens in the vocabulary."""
    kind = rng.choice(["append", "append", "tree", "tree", "tree", "verify", "verify", "keep"])
    q_heads, kv_heads = rng.choice(HEADS)
    head_dim = rng.choice([64, 128, 128])
    page_tokens = rng.choice([32, 64, 64, 128, 256])
    ragged = rng.random() < 0.6
    cached = _log_uniform(rng, 1, 4000) - 1
    if kind == "append":
        sequences = _log_uniform(rng, 1, 32)
        new = _log_uniform(rng, 1, max(1, MOST_APPENDED // (sequences * (q_heads + kv_heads) * head_dim)))
        case = _append("", sequences, cached, new, q_heads, kv_heads, head_dim, rng.choice([head_dim, head_dim, head_dim // 2]),
                       rng.random() < 0.3, rng.random() < 0.7, page_tokens, ragged)
    elif kind == "tree":
        sequences, new = _log_uniform(rng, 1, 64), _log_uniform(rng, 1, 128)
        most = min(MOST_CACHED // (sequences * kv_heads * head_dim), MOST_SCORES // (sequences * q_heads * new)) - new
        while most < 1:
            sequences, new = max(1, sequences // 2), max(1, new // 2)
            most = min(MOST_CACHED // (sequences * kv_heads * head_dim), MOST_SCORES // (sequences * q_heads * new)) - new
        cached = _log_uniform(rng, 1, min(131072, most)) - 1
        case = _tree("", sequences, cached, new, q_heads, kv_heads, rng.choice([1, 2, 4, 8, 16]), head_dim, page_tokens, ragged)
    elif kind == "verify":
        drawn = rng.random() < 0.5
        sequences, new = _log_uniform(rng, 1, 64), _log_uniform(rng, 1, 9 if drawn else 128)
        vocabulary = _log_uniform(rng, 1000, min(128256, max(1000, MOST_PROBABILITIES // (sequences * new * (2 if drawn else 1)))))
        case = _verify("", sequences, new, vocabulary, drawn, 1 if drawn else rng.choice([1, 2, 4, 8, 16]), rng.random() < 0.5, ragged)
    else:
        case = _keep("", _log_uniform(rng, 1, 64), cached, _log_uniform(rng, 1, 128), kv_heads, rng.choice([1, 2, 4, 8, 16]), head_dim, page_tokens, ragged)
    del case["name"]
    return case


# --------------------------------------------------------------------------- lengths and trees, which belong to the case and not to the seed
def _spread(case, longest, salt):
    """One length per sequence: all `longest`, or, ragged, the first one that and the others 1 to that (none where that is 0)."""
    if not case["ragged"] or longest == 0:
        return [longest] * case["sequences"]
    rng = random.Random(case["sequences"] * 1000003 + longest * 7 + salt)
    return [longest] + [rng.randint(1, longest) for _ in range(case["sequences"] - 1)]


def _counts(case):
    """(new rows, tokens in the cache with them) of every sequence."""
    new = _spread(case, case["new"], 0)
    return new, [n + c for n, c in zip(new, _spread(case, case.get("cached", 0), 1))]


def _parents(case):
    """The parent of every row, within its sequence; -1: none.  One of the `width` rows before it."""
    rng = random.Random(case["new"] * 31 + case["width"])
    return [[-1] + [max(0, i - 1 - rng.randrange(case["width"])) for i in range(1, n)] for n in _counts(case)[0]]


def _ancestors(parents):
    """For every row, itself and the rows above it, as a whole number with a bit for each."""
    out = []
    for i, p in enumerate(parents):
        out.append((out[p] if p >= 0 else 0) | 1 << i)
    return out


def _masks(case):
    """int32 [rows, words]: bit i % 32 of word i / 32 says whether the row sees row i of its sequence."""
    every = [m for parents in _parents(case) for m in _ancestors(parents)]
    words = -(-case["new"] // 32)
    return np.array([[m >> 32 * w & 0xFFFFFFFF for w in range(words)] for m in every], np.uint32).view(np.int32)


def _starts(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


# --------------------------------------------------------------------------- inputs, made on the GPU
def _generator(seed):
    return torch.Generator(device=DEVICE).manual_seed(seed)


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEVICE).to(torch.float16)


def _keys(gen, tokens, heads, dim):
    """Keys as models have them: a few channels of every head are larger than the others."""
    k = torch.randn((tokens, heads, dim), generator=gen, device=DEVICE)
    gain = torch.where(torch.rand((heads, dim), generator=gen, device=DEVICE) < 0.03, 3.0, 1.0)
    return k.mul_(gain).to(torch.float16)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def _inputs_cache(case, seed):
    """Keys and values of all tokens of all sequences one behind the other, the queries of the new ones, and a table of pages in no order, with a
    few pages that belong to nobody."""
    gen = _generator(seed)
    new, total = _counts(case)
    k = _keys(gen, sum(total), case["kv_heads"], case["head_dim"])
    v = _normal(gen, sum(total), case["kv_heads"], case["head_dim"])
    q = _normal(gen, sum(new), case["q_heads"], case["head_dim"]) if "q_heads" in case else None
    page = case["page_tokens"]
    counts = [-(-t // page) for t in total]
    n_pages = sum(counts) + 3
    order = torch.randperm(n_pages, generator=gen, device=DEVICE).to(torch.int32)
    pages = torch.full((len(total), max(counts)), -1, dtype=torch.int32, device=DEVICE)
    for b, (c, at) in enumerate(zip(counts, _starts(counts))):
        pages[b, :c] = order[at: at + c]
    return gen, k, v, q, pages, n_pages


def _inputs_rotation(case, gen):
    """Weights, table, positions (a token's place in its sequence)."""
    weights = [(1.0 + 0.1 * torch.randn(case["head_dim"], generator=gen, device=DEVICE)).to(torch.float16) for _ in range(2)] if case["norm"] else [None, None]
    new, total = _counts(case)
    half = case["rotary_dim"] // 2
    angle = torch.arange(max(total), device=DEVICE, dtype=torch.float64)[:, None] * THETA ** (-torch.arange(half, device=DEVICE, dtype=torch.float64) / half)
    table = torch.stack([angle.cos(), angle.sin()], dim=-1).float()
    positions = torch.cat([torch.arange(t - n, t, device=DEVICE, dtype=torch.int32) for n, t in zip(new, total)])
    return weights, table, positions


def _inputs_verify(case, seed):
    """The target's probabilities behind every row; the tokens, drawn from the draft's probabilities or its most likely ones; random numbers."""
    gen = _generator(seed)
    new = _counts(case)[0]
    starts, parents, size = _starts(new), _parents(case), case["vocabulary"]
    logits = torch.randn((sum(new), size), generator=gen, device=DEVICE)
    likely = torch.randint(0, size, (sum(new), 16), generator=gen, device=DEVICE)
    logits.scatter_add_(1, likely, 12.0 * torch.rand(likely.shape, generator=gen, device=DEVICE))
    above = torch.tensor([s + max(p, 0) for s, own_parents in zip(starts, parents) for p in own_parents], device=DEVICE)
    draft, tokens = None, torch.zeros(sum(new), dtype=torch.int64, device=DEVICE)
    if case["drawn"]:
        draft = torch.softmax(logits[above] + 0.7 * torch.randn(logits.shape, generator=gen, device=DEVICE), dim=-1)
        tokens = torch.multinomial(draft, 1, generator=gen).squeeze(1)
    else:
        most = min(size, max(2, case["width"]) + 1)
        ranked = torch.topk(logits + 0.7 * torch.randn(logits.shape, generator=gen, device=DEVICE), most, dim=-1).indices
        rank = [sum(p == own_parents[i] for p in own_parents[:i]) % most for own_parents in parents for i in range(len(own_parents))]
        tokens = ranked[above, torch.tensor(rank, device=DEVICE)]
    target = torch.softmax(logits, dim=-1)
    if case["truncated"]:
        target = torch.where(target < 2e-5, torch.zeros_like(target), target)
        target /= target.sum(dim=-1, keepdim=True)
    uniforms = torch.rand(sum(new), generator=gen, device=DEVICE)
    finals = torch.rand(len(new), generator=gen, device=DEVICE)
    return target, draft, tokens.to(torch.int32), uniforms, finals


def _accepted_paths(case, seed):
    """A way down from row 0 for every sequence: (rows on it, one behind the other and -1 behind them, and how many there are behind row 0)."""
    rng = random.Random(seed)
    path, accepted = [], []
    for parents in _parents(case):
        way, ends = [], [i for i in range(len(parents)) if i not in parents[i + 1:]]
        row = rng.choice(ends)
        while row >= 0:
            way.append(row)
            row = parents[row]
        way = way[::-1][: rng.randint(1, len(way))]
        path += way + [-1] * (len(parents) - len(way))
        accepted.append(len(way) - 1)
    return path, accepted


def prepare(case, seed):
    kind = case["kind"]
    new, total = _counts(case)
    state = {"case": case, "new": new, "total": total, "row_starts": _ints(_starts(new))}
    if kind == "verify":
        target, draft, tokens, uniforms, finals = _inputs_verify(case, seed)
        parents = None if case["drawn"] else _ints([p for own_parents in _parents(case) for p in own_parents])
        state |= {"target": target, "draft": draft, "tokens": tokens, "uniforms": uniforms, "finals": finals, "parents": parents,
                  "out": [torch.empty_like(tokens), torch.empty_like(tokens), torch.empty(len(new), dtype=torch.int32, device=DEVICE)]}
        if own:
            import paper_2412_17560_amd as gq
            state["verifier"] = gq.gqsa_verify_create(len(new), case["vocabulary"])
        return state

    gen, k, v, q, pages, n_pages = _inputs_cache(case, seed)
    state |= {"pages": pages, "lengths": _ints(total), "q": q}
    at = _starts(total)
    filled = total
    if kind == "append":
        state["weights"], state["table"], state["positions"] = _inputs_rotation(case, gen)
    if kind == "tree":
        state["masks"] = torch.from_numpy(_masks(case)).to(DEVICE)
        state["out"] = torch.empty_like(q)
    else:                # what is there already, and the new rows
        filled = [t - n for n, t in zip(new, total)]
        rows = torch.cat([torch.arange(a + f, a + t, device=DEVICE) for a, f, t in zip(at, filled, total)])
        earlier = torch.cat([torch.arange(a, a + f, device=DEVICE) for a, f in zip(at, filled)])
        state["k"], state["v"] = k[rows].contiguous(), v[rows].contiguous()
        k, v = k[earlier].contiguous(), v[earlier].contiguous()
        state["read"] = [torch.empty_like(state["k"]), torch.empty_like(state["v"])]
        state["q_out"] = torch.empty_like(q) if q is not None else None
    if kind == "keep":
        path, accepted = _accepted_paths(case, seed)
        state["path"], state["accepted"] = _ints(path), _ints(accepted)
    if own:
        import paper_2412_17560_amd as gq
        state["cache"] = gq.gqsa_cache_create(n_pages, case["page_tokens"], case["kv_heads"], case["head_dim"])
        if k.shape[0]:
            gq.gqsa_cache_append(state["cache"], k, v, pages, _ints(filled), _ints(_starts(filled)))
    else:
        shape = (n_pages * case["page_tokens"], case["kv_heads"])
        state["pool"] = [{"codes": torch.zeros((*shape, case["head_dim"] // 2), dtype=torch.uint8, device=DEVICE),
                          "low": torch.zeros((*shape, case["head_dim"] // GROUP), dtype=torch.float16, device=DEVICE),
                          "step": torch.zeros((*shape, case["head_dim"] // GROUP), dtype=torch.float16, device=DEVICE)} for _ in range(2)]
        if k.shape[0]:
            count = _ints(filled).long()
            sequence = torch.repeat_interleave(torch.arange(len(filled), device=DEVICE), count)
            token = torch.arange(k.shape[0], device=DEVICE) - _ints(_starts(filled)).long()[sequence]
            for pool, x in zip(state["pool"], (k, v)):
                _plain_store(pool, _slots(state, sequence, token), x)
    return state


# --------------------------------------------------------------------------- the plain forms
def _slots(state, sequence, token):
    """Where the pool holds these tokens."""
    page = state["case"]["page_tokens"]
    return state["pages"][sequence, token // page].long() * page + token % page


def _new_rows(state):
    """(sequence, number in the sequence, token) of every new row."""
    starts = state["row_starts"].long()
    count = starts[1:] - starts[:-1]
    row = torch.arange(state["row_starts"].shape[0] - 1, device=DEVICE)
    sequence = torch.repeat_interleave(row, count, output_size=sum(state["new"]))
    number = torch.arange(sequence.shape[0], device=DEVICE) - starts[sequence]
    token = number if "lengths" not in state else state["lengths"].long()[sequence] - count[sequence] + number
    return sequence, number, token


def _plain_store(pool, slots, x):
    g = x.float().view(x.shape[0], x.shape[1], -1, GROUP)
    low = g.amin(dim=-1, keepdim=True)
    # (a quotient of two tensors is one division; a tensor over a number may be a product with the number's inverse)
    step = ((g.amax(dim=-1, keepdim=True) - low) / torch.full_like(low, 15.0)).half()
    whole = step.float()
    codes = torch.where(whole > 0, torch.round((g - low) / torch.where(whole > 0, whole, torch.ones_like(whole))), torch.zeros_like(g))
    codes = codes.clamp_(0.0, 15.0).to(torch.uint8).view(x.shape)
    pool["codes"][slots] = codes[..., 0::2] | (codes[..., 1::2] << 4)
    pool["low"][slots] = low.half().squeeze(-1)
    pool["step"][slots] = step.squeeze(-1)


def _plain_load(pool, slots):
    """fp32 values of the cached tokens: codes, fp16 numbers nearest to low + code * step."""
    packed = pool["codes"][slots]
    codes = torch.stack([packed & 15, packed >> 4], dim=-1).float().flatten(-2).unflatten(-1, (-1, GROUP))
    values = pool["low"][slots].float().unsqueeze(-1) + codes * pool["step"][slots].float().unsqueeze(-1)
    return values.half().float().flatten(-2)


def _plain_rotate(x, weight, cos, sin, case):
    """fp32 operations one by one; only the norm's factor is computed in 64 bits, as codes hang on its last bit."""
    y = x.float()
    if weight is not None:
        factor = (x.double().square().mean(dim=-1, keepdim=True) + float(np.float32(EPS))).sqrt().reciprocal().float()
        y = y * (factor * weight.float())
    r = case["rotary_dim"]
    turned, rest = y[..., :r], y[..., r:]
    if case["interleaved"]:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2)
    else:
        a, b = turned[..., : r // 2], turned[..., r // 2:]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)
    return torch.cat([turned, rest], dim=-1).half()


def _plain_tree(state):
    """All sequences at once, padded to the longest."""
    case = state["case"]
    heads, kv_heads, dim = case["q_heads"], case["kv_heads"], case["head_dim"]
    per, n_seqs, rows, tokens = heads // kv_heads, case["sequences"], max(state["new"]), max(state["total"])
    sequence, number, _ = _new_rows(state)
    every = torch.arange(tokens, device=DEVICE)
    lengths = state["lengths"].long()
    before = lengths - (state["row_starts"][1:] - state["row_starts"][:-1]).long()
    there = every < lengths[:, None]
    slots = torch.where(there, _slots(state, torch.arange(n_seqs, device=DEVICE)[:, None], every.expand(n_seqs, tokens)), torch.zeros_like(there, dtype=torch.int64))
    k, v = (_plain_load(pool, slots).masked_fill_(~there[:, :, None, None], 0.0).transpose(1, 2) for pool in state["pool"])     # [seqs, kv heads, tokens, D]
    bits = (state["masks"].long()[:, :, None] >> torch.arange(32, device=DEVICE) & 1).flatten(1).bool()                          # [all rows, 32 words]
    behind = every[None, :] - before[sequence][:, None]
    seen = torch.where(behind < 0, True, torch.gather(bits, 1, behind.clamp(0, bits.shape[1] - 1)) & (behind < bits.shape[1])) & there[sequence]
    allowed = torch.zeros((n_seqs, rows, tokens), dtype=torch.bool, device=DEVICE)
    allowed[sequence, number] = seen
    q = torch.zeros((n_seqs, rows, heads, dim), device=DEVICE)
    q[sequence, number] = state["q"].float()
    q = q.view(n_seqs, rows, kv_heads, per, dim).permute(0, 2, 3, 1, 4).reshape(n_seqs, kv_heads, per * rows, dim)
    s = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(dim ** -0.5).view(n_seqs, kv_heads, per, rows, tokens)
    s.masked_fill_(~allowed[:, None, None], float("-inf"))
    s = s.sub_(s.amax(dim=-1, keepdim=True).clamp(min=-1e30)).exp_()
    s = s.div_(s.sum(dim=-1, keepdim=True).clamp(min=1e-30)).view(n_seqs, kv_heads, per * rows, tokens)
    o = torch.matmul(s, v.contiguous()).view(n_seqs, kv_heads, per, rows, dim).permute(0, 3, 1, 2, 4).reshape(n_seqs, rows, heads, dim)
    return o[sequence, number].half()


def _plain_verify(state):
    """All sequences at once, padded to the most rows: [sequences, rows]."""
    case = state["case"]
    n_seqs, rows = case["sequences"], max(state["new"])
    sequence, number, _ = _new_rows(state)
    first = state["row_starts"].long()[:-1, None]
    target = state["target"]
    each = torch.arange(rows, device=DEVICE)

    def padded(x, fill):
        out = torch.full((n_seqs, rows), fill, dtype=x.dtype, device=DEVICE)
        out[sequence, number] = x
        return out
    there = padded(torch.ones_like(sequence, dtype=torch.bool), False)
    parent = (each - 1).expand(n_seqs, rows) if state["parents"] is None else padded(state["parents"].long(), -1)
    parent = torch.where(there, parent, torch.full_like(parent, -1))
    token, uniform = padded(state["tokens"].long(), 0), padded(state["uniforms"].double(), 2.0)
    p = target[first + parent.clamp(min=0), token].double()
    sibling = (parent[:, :, None] == parent[:, None, :]) & (each[:, None] > each) & (parent >= 0)[:, :, None]      # before: [sequences, row, other row]
    if case["drawn"]:
        left = state["draft"][first + torch.where(there, each, 0), token].double()
    else:       # (of siblings with the same token the first counts)
        again = (sibling & (token[:, :, None] == token[:, None, :])).any(dim=-1)
        p = torch.where(again, torch.zeros_like(p), p)
        left = 1.0 - (sibling * p[:, None, :]).sum(dim=-1)
    accepted = (uniform * left < p) & (parent >= 0)
    # on the way: row 0, and the first accepted children of rows that are on it; in steps of twice as many rows at a time
    on = accepted & ~(sibling & accepted[:, None, :]).any(dim=-1)
    on[:, 0] = there[:, 0]
    up = parent.clamp(min=0)
    for _ in range((rows - 1).bit_length()):
        on &= torch.gather(on, 1, up)
        up = torch.gather(up, 1, up)
    path = torch.where(on, each, rows).sort(dim=1).values
    path = torch.cat([torch.where(path < rows, path, -1), torch.full_like(path[:, :1], -1)], dim=1)
    count = (path >= 0).sum(dim=1) - 1
    row = path.amax(dim=1)
    weights = target[first[:, 0] + row].double()
    if case["drawn"]:
        last = row + 1 >= there.sum(dim=1)
        less = state["draft"][first[:, 0] + torch.where(last, row, row + 1)].double()
        weights = torch.where(last[:, None], weights, (weights - less).clamp(min=0.0))
    else:
        child = parent == row[:, None]
        weights[torch.arange(n_seqs, device=DEVICE)[:, None].expand_as(child)[child], token[child]] = 0.0
    nothing = ~(weights > 0).any(dim=1, keepdim=True)
    weights = torch.where(nothing, target[first[:, 0] + row].double(), weights)
    sums = weights.cumsum(dim=1)
    drawn = torch.searchsorted(sums, (state["finals"].double() * sums[:, -1])[:, None], right=True)[:, 0]
    last_of = torch.where(weights > 0, torch.arange(weights.shape[1], device=DEVICE), -1).amax(dim=1)
    drawn = torch.minimum(drawn, last_of)
    out = torch.where(path[:, 1:] > 0, torch.gather(token, 1, path[:, 1:].clamp(min=0, max=rows - 1)), -1)
    out = torch.where(each == count[:, None], drawn[:, None], out)
    return [path[sequence, number].int(), out[sequence, number].int(), count.int()]


def _plain(state):
    case, kind = state["case"], state["case"]["kind"]
    if kind == "verify":
        return _plain_verify(state)
    if kind == "tree":
        return _plain_tree(state)
    sequence, number, token = _new_rows(state)
    slots = _slots(state, sequence, token)
    k, out = state["k"], []
    if kind == "append":
        turn = state["table"][state["positions"].long()].unsqueeze(1)
        q, k = (_plain_rotate(x, w, turn[..., 0], turn[..., 1], case) for x, w in zip((state["q"], k), state["weights"]))
        out = [q]
    for pool, x in zip(state["pool"], (k, state["v"])):
        _plain_store(pool, slots, x)
    if kind == "keep":
        kept = state["path"] >= 0
        at = _slots(state, sequence[kept], token[kept])
        of = _slots(state, sequence[kept], token[kept] - number[kept] + state["path"][kept].long())
        for pool in state["pool"]:
            for part in pool.values():
                part[at] = part[of]
    return out + [_plain_load(pool, slots).half() for pool in state["pool"]]


# --------------------------------------------------------------------------- one pass
def run(state):
    if not own:
        return _plain(state)
    import paper_2412_17560_amd as gq
    case, kind = state["case"], state["case"]["kind"]
    if kind == "verify":
        return list(gq.gqsa_verify(state["verifier"], state["target"], state["tokens"], state["uniforms"], state["finals"], state["row_starts"],
                                   parents=state["parents"], draft=state["draft"], path=state["out"][0], out=state["out"][1], accepted=state["out"][2]))
    where = (state["pages"], state["lengths"], state["row_starts"])
    if kind == "tree":
        return gq.gqsa_cache_attend_tree(state["cache"], state["q"], *where, state["masks"], out=state["out"])
    if kind == "append":
        q, _ = gq.gqsa_cache_append_rotated(state["cache"], state["q"], state["k"], state["v"], state["positions"], state["table"], *where,
                                            *state["weights"], eps=EPS, interleaved=case["interleaved"], q_out=state["q_out"])
        return [q, *gq.gqsa_cache_read(state["cache"], *where, *state["read"])]
    gq.gqsa_cache_append(state["cache"], state["k"], state["v"], *where)
    gq.gqsa_cache_keep(state["cache"], *where, state["path"], state["accepted"])
    return list(gq.gqsa_cache_read(state["cache"], *where, *state["read"]))


# --------------------------------------------------------------------------- the definitions in float64
def _to_half(x):
    """float64 to fp16 in one rounding, and back: by way of fp32, where odd last bits keep the result that a second rounding would lose."""
    near = x.float()
    lost = near.double() != x
    bits = near.view(torch.int32)
    towards_zero = torch.where(near.double().abs() > x.abs(), bits - 1, bits)
    return torch.where(lost, towards_zero | 1, bits).view(torch.float32).half().double()


def _exact_held(x):
    """float64 values that the cache stands for.  The fp32 roundings of the definition are kept: a difference or quotient of fp32 numbers taken in
    float64 and rounded to fp32 is the fp32 one."""
    g = x.double().unflatten(-1, (-1, GROUP))
    low = g.min(dim=-1, keepdim=True).values
    step = ((g.max(dim=-1, keepdim=True).values - low).float().double() / 15.0).float().half().double()
    ratio = ((g - low).float().double() / step).float().double()
    codes = torch.where(step > 0, ratio.round().clamp(max=15.0), torch.zeros_like(g))
    return _to_half(low + codes * step).flatten(-2)


def _exact_rotated(x, w, table, positions, case):
    """Two results: with the definition's fp32 roundings and the one to fp16 (what the cache is made of), and without any."""
    x = x.double()
    r, both = case["rotary_dim"], []
    first = torch.arange(0, r, 2, device=DEVICE) if case["interleaved"] else torch.arange(r // 2, device=DEVICE)
    second = first + (1 if case["interleaved"] else r // 2)
    for rounded in (lambda t: t.float().double(), lambda t: t):
        y = x.clone()
        if w is not None:
            root = rounded(1.0 / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + float(np.float32(EPS))).sqrt())
            y = rounded(x * rounded(root * w.double()))
        c, s = (table[positions.long()][:, None, :, i].double() for i in (0, 1))
        a, b = y[..., first], y[..., second]
        z = y.clone()
        z[..., first] = rounded(rounded(a * c) - rounded(b * s))
        z[..., second] = rounded(rounded(a * s) + rounded(b * c))
        both.append(z)
    return both[0].half(), both[1]


def _exact_verify(case, seed):
    target, draft, tokens, uniforms, finals = _inputs_verify(case, seed)
    tokens, uniforms, finals = tokens.tolist(), uniforms.tolist(), finals.tolist()
    new = _counts(case)[0]
    paths, outs, counts = [], [], []
    for b, (start, parents) in enumerate(zip(_starts(new), _parents(case))):
        row, path = 0, [0]
        while True:
            children, mass, followed = [i for i, p in enumerate(parents) if p == row and i > row], 1.0, None
            tried = set()
            for i in children:
                x = tokens[start + i]
                p = float(target[start + row, x])
                if case["drawn"]:
                    stands = uniforms[start + i] * float(draft[start + i, x]) < p
                else:
                    stands = x not in tried and uniforms[start + i] * mass < p
                    mass -= 0.0 if x in tried else p
                tried.add(x)
                if stands:
                    followed = i
                    break
            if followed is None:
                break
            row = followed
            path.append(row)
        weights = target[start + row].cpu().numpy().astype(np.float64)
        if case["drawn"]:
            if children:
                weights = np.maximum(weights - draft[start + children[0]].cpu().numpy().astype(np.float64), 0.0)
        else:
            weights[sorted(tried)] = 0.0
        if not (weights > 0).any():
            weights = target[start + row].cpu().numpy().astype(np.float64)
        sums = np.cumsum(weights)
        drawn = min(int(np.searchsorted(sums, finals[b] * sums[-1], side="right")), int(np.flatnonzero(weights > 0)[-1]))
        pad = [-1] * (len(parents) - len(path))
        paths += path + pad
        outs += [tokens[start + i] for i in path[1:]] + [drawn] + pad
        counts.append(len(path) - 1)
    return [torch.tensor(x, dtype=torch.int32) for x in (paths, outs, counts)]


def exact(case, seed):
    """What run() returns for these inputs, in float64."""
    kind = case["kind"]
    if kind == "verify":
        return _exact_verify(case, seed)
    gen, k, v, q, _, _ = _inputs_cache(case, seed)
    new, total = _counts(case)
    row, at = _starts(new), _starts(total)
    if kind != "tree":
        rows = torch.cat([torch.arange(a + t - n, a + t, device=DEVICE) for a, n, t in zip(at, new, total)])
        k, v = k[rows], v[rows]
        if kind == "append":
            weights, table, positions = _inputs_rotation(case, gen)
            return [_exact_rotated(q, weights[0], table, positions, case)[1],
                    _exact_held(_exact_rotated(k, weights[1], table, positions, case)[0]), _exact_held(v)]
        held = [_exact_held(k), _exact_held(v)]
        path, accepted = _accepted_paths(case, seed)
        of = torch.tensor([row[b] + (path[row[b] + i] if i <= accepted[b] else i) for b in range(len(new)) for i in range(new[b])], device=DEVICE)
        return [x[of] for x in held]
    out = torch.empty(q.shape, dtype=torch.float64, device=DEVICE)
    per, scale = case["q_heads"] // case["kv_heads"], case["head_dim"] ** -0.5
    for b, parents in enumerate(_parents(case)):
        n, t = new[b], total[b]
        sees = torch.ones((n, t), dtype=torch.bool)
        sees[:, t - n:] = torch.tensor([[bool(m >> i & 1) for i in range(n)] for m in _ancestors(parents)])
        sees = sees.to(DEVICE)
        for h in range(case["kv_heads"]):
            kh, vh = (_exact_held(x[at[b]:at[b + 1], h]) for x in (k, v))
            for i in range(h * per, (h + 1) * per):
                s = (q[row[b]:row[b + 1], i].double() @ kh.t()) * scale
                top = torch.where(sees, s, torch.full_like(s, -1e300)).max(dim=1, keepdim=True).values
                p = torch.where(sees, torch.exp(s - top), torch.zeros_like(s))
                out[row[b]:row[b + 1], i] = (p @ vh) / p.sum(dim=1, keepdim=True)
    return out


# --------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    """Inputs and outputs once each.  A cached group of 32 values is 16 bytes of codes, 2 of low, 2 of step."""
    kind = case["kind"]
    new, total = _counts(case)
    if kind == "verify":        # one row a sequence of the target's probabilities, and of the draft's; six numbers a drafted row
        rows = len(new) * case["vocabulary"] * (2 if case["drawn"] else 1)
        return {"bytes": 4 * rows + 28 * sum(new) + 8 * len(new), "flops": 2 * rows}
    d = case["head_dim"]
    elements = sum(new) * case["kv_heads"] * d
    if kind == "append":        # read, held, given back; queries read and written; the table's rows
        turned = sum(new) * (case["q_heads"] + case["kv_heads"]) * d
        return {"bytes": 8 * elements + 4 * elements * 20 // 32 + 4 * sum(new) * case["q_heads"] * d + sum(new) * (4 + 4 * case["rotary_dim"]),
                "flops": 7 * turned + 16 * elements}
    if kind == "keep":
        return {"bytes": 8 * elements + 4 * elements * 20 // 32, "flops": 16 * elements}
    pairs = sum(n * (t - n) + sum(m.bit_count() for m in _ancestors(parents)) for n, t, parents in zip(new, total, _parents(case)))
    return {"bytes": 4 * sum(new) * case["q_heads"] * d + 2 * sum(total) * case["kv_heads"] * d * 20 // 32 + 4 * sum(new) * -(-case["new"] // 32),
            "flops": 4 * d * case["q_heads"] * pairs}
