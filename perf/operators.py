"""The operators between the q/k/v products and the o product of a decoder layer, as cases that are timed one by one.

  rotate   norms of the queries and keys of each head and the rotation by position, in one pass (gqsa_qk_norm_rotate)
  append   new keys and values into a paged 4-bit cache, and what the cache then stands for, read back (gqsa_cache_append,
           gqsa_cache_read: the way from a cached prefix to the attention of a later part of the prompt)
  attend   attention of the newest rows of some sequences over their cache (gqsa_cache_attend)
  prompt   causal attention over packed prompts with grouped heads (gqsa_prompt_attend)

Everything is fp16, as the activations of the framework's products are; sums and softmax are in fp32.

The cache holds groups of 32 channels of one token and head: `low` = the least of them, `step` = fp16((greatest - low) / 15),
codes = min(15, round((x - low) / step)) (0 where step is 0), every operation a single fp32 operation; a code stands for
the fp16 number nearest to low + code * step.
"""
from __future__ import annotations

import random

import torch

own = False         # False: plain torch in 32 bits; True: the framework's operators

DEVICE = "cuda:0"
GROUP = 32
EPS = 1e-6
THETA = 10000.0


def _rotate(name, tokens, q_heads, k_heads, head_dim=128, rotary_dim=128, interleaved=False, norm=True, fused=True):
    return {"name": name, "kind": "rotate", "tokens": tokens, "q_heads": q_heads, "k_heads": k_heads, "head_dim": head_dim,
            "rotary_dim": rotary_dim, "interleaved": interleaved, "norm": norm, "fused": fused}


def _append(name, sequences, cached, new, kv_heads, head_dim=128, page_tokens=64, ragged=False):
    return {"name": name, "kind": "append", "sequences": sequences, "cached": cached, "new": new, "kv_heads": kv_heads,
            "head_dim": head_dim, "page_tokens": page_tokens, "ragged": ragged}


def _attend(name, sequences, longest, q_heads, kv_heads, rows=1, head_dim=128, page_tokens=64, ragged=False):
    return {"name": name, "kind": "attend", "sequences": sequences, "longest": longest, "q_heads": q_heads, "kv_heads": kv_heads,
            "rows": rows, "head_dim": head_dim, "page_tokens": page_tokens, "ragged": ragged}


def _prompt(name, sequences, longest, q_heads, kv_heads, prefix=0, head_dim=128, ragged=False):
    return {"name": name, "kind": "prompt", "sequences": sequences, "longest": longest, "q_heads": q_heads, "kv_heads": kv_heads,
            "prefix": prefix, "head_dim": head_dim, "ragged": ragged}


def listed():
    return [
        # token generation, one sequence, a head of its own for every query (hidden size 4096): launch and call overhead
        _rotate("rotate_decode_b1", 1, 32, 32),
        # a long prompt of the widest layers here (hidden size 8192, 64 heads, 8 for keys), slices of one q/k/v array
        _rotate("rotate_prompt_gqa", 8192, 64, 8),
        # an odd number of tokens, small heads, half of the channels rotated in neighbouring pairs, no norms, arrays of their own
        _rotate("rotate_partial_ragged", 1237, 28, 4, head_dim=64, rotary_dim=32, interleaved=True, norm=False, fused=False),
        # one token for each of 16 sequences: the step ahead of a decoding step's attention
        _append("append_decode_b16", 16, 700, 1, 8),
        # a long prompt goes into the cache
        _append("append_prompt", 1, 0, 8192, 8, page_tokens=128),
        # token generation, one sequence: 15 tokens of prompt and 128 generated ones
        _attend("attend_b1_short", 1, 143, 32, 32),
        # a batch of 16, every query head with keys of its own, equal lengths: the bytes of the cache
        _attend("attend_b16_mha", 16, 4096, 32, 32, page_tokens=128),
        # a few sequences of very different lengths, grouped heads, five candidate tokens each
        _attend("attend_gqa_ragged_rows5", 8, 16003, 32, 8, rows=5, ragged=True),
        # one very long sequence: split over its length
        _attend("attend_b1_long", 1, 131072, 64, 8, page_tokens=256),
        # a short question
        _prompt("prompt_short", 1, 15, 32, 32),
        # packed prompts of different lengths
        _prompt("prompt_packed_ragged", 7, 2500, 40, 8, ragged=True),
        # one long prompt, grouped heads: the matrix cores
        _prompt("prompt_long", 1, 8192, 32, 8),
    ]


def _log_uniform(rng, low, high, multiple=1):
    v = low * (high / low) ** rng.random()
    return max(multiple, int(round(v / multiple)) * multiple)


HEADS = [(32, 32), (32, 8), (64, 8), (40, 40), (40, 8), (28, 4), (14, 2), (12, 12), (16, 1)]     # (queries, keys)
MOST_ROTATED = 8192 * 72 * 128          # elements of q and k together
MOST_APPENDED = 8192 * 8 * 128          # elements of the new keys
MOST_CACHED = 16 * 4096 * 32 * 128      # elements of the keys that are attended to
MOST_PAIRS = 8192 * 8193 // 2 * 32 * 128    # allowed (query row, key) pairs times head_dim


def draw(rng):
    """One more case of the ranges: one token to thousands, one sequence to 64, 12 to 64 heads of 64 or 128 channels."""
    kind = rng.choice(["rotate", "append", "attend", "attend", "prompt", "prompt"])
    q_heads, kv_heads = rng.choice(HEADS)
    head_dim = rng.choice([64, 128, 128])
    page_tokens = rng.choice([32, 64, 64, 128, 256])
    ragged = rng.random() < 0.6
    if kind == "rotate":
        tokens = _log_uniform(rng, 1, min(16384, MOST_ROTATED // ((q_heads + kv_heads) * head_dim)))
        case = _rotate("", tokens, q_heads, kv_heads, head_dim, rng.choice([head_dim, head_dim, head_dim // 2]),
                       rng.random() < 0.3, rng.random() < 0.7, rng.random() < 0.5)
    elif kind == "append":
        sequences = _log_uniform(rng, 1, 32)
        case = _append("", sequences, _log_uniform(rng, 1, 2000) - 1,
                       _log_uniform(rng, 1, max(1, MOST_APPENDED // (sequences * kv_heads * head_dim))), kv_heads, head_dim, page_tokens, ragged)
    elif kind == "attend":
        sequences = _log_uniform(rng, 1, 64)
        longest = _log_uniform(rng, 1, min(131072, MOST_CACHED // (sequences * kv_heads * head_dim)))
        case = _attend("", sequences, longest, q_heads, kv_heads, rng.choice([1, 1, 1, 2, 3, 4, 8]), head_dim, page_tokens, ragged)
    else:
        sequences = _log_uniform(rng, 1, 32)
        prefix = rng.choice([0, 0, 0, _log_uniform(rng, 1, 2000)])
        longest = _log_uniform(rng, 1, 8192)
        case = _prompt("", sequences, longest, q_heads, kv_heads, prefix, head_dim, ragged)
        while _pairs(case) * q_heads * head_dim > MOST_PAIRS:
            case["longest"] = max(1, int(case["longest"] * 0.8))
            case["prefix"] = int(case["prefix"] * 0.8)
    del case["name"]
    return case


# --------------------------------------------------------------------------- lengths, which belong to the case and not to the seed
def _spread(case, longest):
    """One length per sequence: all `longest`, or, ragged, the first one that and the others 1 to that."""
    if not case["ragged"]:
        return [longest] * case["sequences"]
    rng = random.Random(case["sequences"] * 1000003 + longest)
    return [longest] + [rng.randint(1, longest) for _ in range(case["sequences"] - 1)]


def _new_and_total(case):
    """(new rows, tokens in the cache or in front of the last row with the new ones) of every sequence."""
    if case["kind"] == "append":
        new = _spread(case, case["new"])
        before = _spread(case, case["cached"]) if case["cached"] else [0] * case["sequences"]
        return new, [n + c for n, c in zip(new, before)]
    if case["kind"] == "attend":
        total = _spread(case, case["longest"])
        return [min(case["rows"], t) for t in total], total
    new = _spread(case, case["longest"])
    return new, [n + case["prefix"] for n in new]


def _starts(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


def _pairs(case):
    """(row, token) pairs of one query head that the causal mask leaves."""
    return sum(n * (t - n) + n * (n + 1) // 2 for n, t in zip(*_new_and_total(case)))


# --------------------------------------------------------------------------- inputs, made on the GPU
def _generator(seed):
    return torch.Generator(device=DEVICE).manual_seed(seed)


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEVICE).to(torch.float16)


def _keys(gen, tokens, heads, dim):
    """Keys as models have them: a few channels of every head are much larger than the others."""
    k = torch.randn((tokens, heads, dim), generator=gen, device=DEVICE)
    gain = torch.where(torch.rand((heads, dim), generator=gen, device=DEVICE) < 0.03, 6.0, 1.0)
    return k.mul_(gain).to(torch.float16)


def _inputs_rotate(case, seed):
    gen = _generator(seed)
    t, d = case["tokens"], case["head_dim"]
    heads = case["q_heads"] + 2 * case["k_heads"]
    qkv = _normal(gen, t, heads, d)
    q, k = qkv[:, : case["q_heads"]], qkv[:, case["q_heads"]: case["q_heads"] + case["k_heads"]]
    if not case["fused"]:
        q, k = q.contiguous(), k.contiguous()
    first = int(torch.randint(0, 4096, (1,), generator=gen, device=DEVICE))
    weights = [(1.0 + 0.1 * torch.randn(d, generator=gen, device=DEVICE)).to(torch.float16) for _ in range(2)]
    half = case["rotary_dim"] // 2
    angle = torch.arange(4096 + t, device=DEVICE, dtype=torch.float64)[:, None] * THETA ** (
        -torch.arange(half, device=DEVICE, dtype=torch.float64) / half)
    table = torch.stack([angle.cos(), angle.sin()], dim=-1).float()
    positions = torch.arange(first, first + t, device=DEVICE, dtype=torch.int32)
    return q, k, positions, table, weights if case["norm"] else [None, None]


def _inputs_cache(case, seed):
    """Keys and values of all tokens of all sequences one behind the other, the rows' starts, the lengths, and a table of
    pages in no order, with a few pages that belong to nobody."""
    gen = _generator(seed)
    new, total = _new_and_total(case)
    k = _keys(gen, sum(total), case["kv_heads"], case["head_dim"])
    v = _normal(gen, sum(total), case["kv_heads"], case["head_dim"])
    page = case["page_tokens"]
    counts = [-(-t // page) for t in total]
    n_pages = sum(counts) + 3
    order = torch.randperm(n_pages, generator=gen, device=DEVICE).to(torch.int32)
    pages = torch.full((len(total), max(counts)), -1, dtype=torch.int32, device=DEVICE)
    for b, (c, at) in enumerate(zip(counts, _starts(counts))):
        pages[b, :c] = order[at: at + c]
    q = _normal(gen, sum(new), case["q_heads"], case["head_dim"]) if case["kind"] == "attend" else None
    return k, v, q, pages, n_pages, new, total


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def _rows_of(parts):
    """Indices of the rows [start, end) of the parts, one behind the other."""
    return torch.cat([torch.arange(a, b, device=DEVICE) for a, b in parts])


def prepare(case, seed):
    kind = case["kind"]
    if kind == "rotate":
        q, k, positions, table, weights = _inputs_rotate(case, seed)
        out = [torch.empty((case["tokens"], x.shape[1], case["head_dim"]), dtype=torch.float16, device=DEVICE) for x in (q, k)]
        return {"case": case, "q": q, "k": k, "positions": positions, "table": table, "weights": weights, "out": out}
    if kind == "prompt":
        gen = _generator(seed)
        new, total = _new_and_total(case)
        q = _normal(gen, sum(new), case["q_heads"], case["head_dim"])
        k = _keys(gen, sum(total), case["kv_heads"], case["head_dim"])
        v = _normal(gen, sum(total), case["kv_heads"], case["head_dim"])
        return {"case": case, "q": q, "k": k, "v": v, "new": new, "total": total, "q_starts": _ints(_starts(new)),
                "k_starts": _ints(_starts(total)), "out": torch.empty_like(q)}

    k, v, q, pages, n_pages, new, total = _inputs_cache(case, seed)
    state = {"case": case, "q": q, "pages": pages, "new": new, "total": total, "lengths": _ints(total), "row_starts": _ints(_starts(new))}
    at = _starts(total)
    if kind == "append":        # what is there already, and the new rows
        filled = [t - n for n, t in zip(new, total)]
        rows = _rows_of([(a + f, a + t) for a, f, t in zip(at, filled, total)])
        state["k"], state["v"] = k[rows].contiguous(), v[rows].contiguous()
        earlier = _rows_of([(a, a + f) for a, f in zip(at, filled)])
        k, v = k[earlier].contiguous(), v[earlier].contiguous()
        if own:
            state["read"] = [torch.empty_like(state["k"]), torch.empty_like(state["v"])]
    else:
        filled = total
        state["out"] = torch.empty_like(q)
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
            slots = _slots(case, pages, [(0, f) for f in filled])
            for pool, x in zip(state["pool"], (k, v)):
                _plain_store(pool, slots, x)
    return state


# --------------------------------------------------------------------------- the plain forms
def _slots(case, pages, spans):
    """Where the pool holds the tokens [first, end) of each sequence."""
    page = case["page_tokens"]
    out = []
    for b, (first, end) in enumerate(spans):
        token = torch.arange(first, end, device=DEVICE)
        out.append(pages[b].long()[token // page] * page + token % page)
    return torch.cat(out)


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
    """fp32 values of the cached rows: codes, fp16 numbers nearest to low + code * step."""
    packed = pool["codes"][slots]
    codes = torch.stack([packed & 15, packed >> 4], dim=-1).float()
    codes = codes.view(packed.shape[0], packed.shape[1], -1, GROUP)
    values = pool["low"][slots].float().unsqueeze(-1) + codes * pool["step"][slots].float().unsqueeze(-1)
    return values.half().float().view(packed.shape[0], packed.shape[1], -1)


def _plain_rotate(x, weight, cos, sin, case):
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + EPS) * weight.float()
    r = case["rotary_dim"]
    turned, rest = x[..., :r], x[..., r:]
    if case["interleaved"]:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2)
    else:
        a, b = turned[..., : r // 2], turned[..., r // 2:]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)
    return torch.cat([turned, rest], dim=-1).half()


MOST_SCORES = 1 << 29       # scores held at once


def _plain_attention(q, k, v, scale):
    """q [rows, heads, D], k and v [tokens, kv heads, D] in fp32; the last row sees every token, the one before one fewer."""
    rows, heads, dim = q.shape
    tokens, kv_heads = k.shape[:2]
    per = heads // kv_heads
    blocked = torch.arange(tokens, device=DEVICE) > torch.arange(rows, device=DEVICE)[:, None] + (tokens - rows)
    out = torch.empty_like(q)
    width = max(1, min(kv_heads, MOST_SCORES // max(1, per * rows * tokens)))
    for h in range(0, kv_heads, width):
        kh, vh = k[:, h:h + width].transpose(0, 1), v[:, h:h + width].transpose(0, 1)
        n = kh.shape[0]
        qh = q[:, h * per:(h + n) * per].transpose(0, 1).reshape(n, per * rows, dim)
        s = torch.matmul(qh, kh.transpose(1, 2).contiguous()).mul_(scale).view(n, per, rows, tokens)
        s.masked_fill_(blocked, float("-inf"))
        s = s.sub_(s.amax(dim=-1, keepdim=True)).exp_()
        s = s.div_(s.sum(dim=-1, keepdim=True)).view(n, per * rows, tokens)
        o = torch.matmul(s, vh.contiguous()).view(n * per, rows, dim)
        out[:, h * per:(h + n) * per] = o.transpose(0, 1)
    return out


def _plain(state):
    case, kind = state["case"], state["case"]["kind"]
    if kind == "rotate":
        turn = state["table"][state["positions"].long()].unsqueeze(1)
        return [_plain_rotate(x, w, turn[..., 0], turn[..., 1], case) for x, w in zip((state["q"], state["k"]), state["weights"])]
    new, total = state["new"], state["total"]
    if kind == "append":
        slots = _slots(case, state["pages"], [(t - n, t) for n, t in zip(new, total)])
        for pool, x in zip(state["pool"], (state["k"], state["v"])):
            _plain_store(pool, slots, x)
        return [_plain_load(pool, slots).half() for pool in state["pool"]]
    scale = case["head_dim"] ** -0.5
    row, out = _starts(new), []
    if kind == "attend":
        for b, t in enumerate(total):
            slots = _slots({**case}, state["pages"][b:b + 1], [(0, t)])
            k, v = (_plain_load(pool, slots) for pool in state["pool"])
            out.append(_plain_attention(state["q"][row[b]:row[b + 1]].float(), k, v, scale).half())
    else:
        at = _starts(total)
        for b in range(len(new)):
            q, k, v = (x[s[b]:s[b + 1]].float() for x, s in ((state["q"], row), (state["k"], at), (state["v"], at)))
            out.append(_plain_attention(q, k, v, scale).half())
    return torch.cat(out)


# --------------------------------------------------------------------------- one pass
def run(state):
    if not own:
        return _plain(state)
    import paper_2412_17560_amd as gq
    case, kind = state["case"], state["case"]["kind"]
    if kind == "rotate":
        return list(gq.gqsa_qk_norm_rotate(state["q"], state["k"], state["positions"], state["table"], *state["weights"], eps=EPS,
                                           interleaved=case["interleaved"], q_out=state["out"][0], k_out=state["out"][1]))
    if kind == "append":
        gq.gqsa_cache_append(state["cache"], state["k"], state["v"], state["pages"], state["lengths"], state["row_starts"])
        gq.gqsa_cache_read(state["cache"], state["pages"], state["lengths"], state["row_starts"], *state["read"])
        return state["read"]
    if kind == "attend":
        return gq.gqsa_cache_attend(state["cache"], state["q"], state["pages"], state["lengths"], state["row_starts"], out=state["out"])
    return gq.gqsa_prompt_attend(state["q"], state["k"], state["v"], state["q_starts"], state["k_starts"], out=state["out"])


# --------------------------------------------------------------------------- the definitions in float64
def _exact_held(x):
    """float64 values that the cache stands for.  The two fp32 roundings of the definition are kept: a difference or quotient
    of fp32 numbers taken in float64 and rounded to fp32 is the fp32 one."""
    g = x.double().unflatten(-1, (-1, GROUP))
    low = g.min(dim=-1, keepdim=True).values
    step = ((g.max(dim=-1, keepdim=True).values - low).float().double() / 15.0).float().half().double()
    ratio = ((g - low).float().double() / step).float().double()
    codes = torch.where(step > 0, ratio.round().clamp(max=15.0), torch.zeros_like(g))
    held = low + codes * step
    near = held.float()                 # to fp16 by way of fp32: where that rounds twice, odd last bits keep the result
    lost = held != near.double()
    bits = near.view(torch.int32)
    towards_zero = torch.where(near.double().abs() > held.abs(), bits - 1, bits)
    odd = torch.where(lost, towards_zero | 1, bits).view(torch.float32)
    return odd.half().double().flatten(-2)


def _exact_head(q, k, v, scale):
    """One query head [rows, D] over keys and values [tokens, D], a slab of rows at a time."""
    rows, tokens = q.shape[0], k.shape[0]
    out = torch.empty_like(q)
    slab = max(1, (1 << 26) // tokens)
    for r in range(0, rows, slab):
        s = (q[r:r + slab] @ k.t()) * scale
        seen = tokens - rows + 1 + torch.arange(r, r + s.shape[0], device=q.device)
        allowed = torch.arange(tokens, device=q.device).expand_as(s) < seen[:, None]
        top = torch.where(allowed, s, torch.full_like(s, -1e300)).max(dim=1, keepdim=True).values
        p = torch.where(allowed, torch.exp(s - top), torch.zeros_like(s))
        out[r:r + slab] = (p @ v) / p.sum(dim=1, keepdim=True)
    return out


def exact(case, seed):
    """What run() returns for these inputs, in float64."""
    kind = case["kind"]
    if kind == "rotate":
        q, k, positions, table, weights = _inputs_rotate(case, seed)
        r, results = case["rotary_dim"], []
        for x, w in zip((q, k), weights):
            x = x.double().clone()
            if w is not None:
                x = x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt() * w.double()
            first = torch.arange(0, r, 2, device=DEVICE) if case["interleaved"] else torch.arange(r // 2, device=DEVICE)
            second = first + (1 if case["interleaved"] else r // 2)
            z = torch.complex(x[..., first], x[..., second]) * torch.view_as_complex(table[positions.long()].double())[:, None]
            x[..., first], x[..., second] = z.real, z.imag
            results.append(x)
        return results
    scale = case["head_dim"] ** -0.5
    new, total = _new_and_total(case)
    row, at = _starts(new), _starts(total)
    if kind == "prompt":
        gen = _generator(seed)
        q = _normal(gen, sum(new), case["q_heads"], case["head_dim"])
        k = _keys(gen, sum(total), case["kv_heads"], case["head_dim"])
        v = _normal(gen, sum(total), case["kv_heads"], case["head_dim"])
    else:
        k, v, q = _inputs_cache(case, seed)[:3]
        if kind == "append":
            rows = torch.cat([torch.arange(a + t - n, a + t, device=DEVICE) for a, n, t in zip(at, new, total)])
            return [_exact_held(k[rows]), _exact_held(v[rows])]
    out = torch.empty(q.shape, dtype=torch.float64, device=DEVICE)
    per = case["q_heads"] // case["kv_heads"]
    for h in range(case["kv_heads"]):
        kh, vh = (_exact_held(x[:, h]) if kind == "attend" else x[:, h].double() for x in (k, v))
        for b in range(len(new)):
            for i in range(h * per, (h + 1) * per):
                out[row[b]:row[b + 1], i] = _exact_head(q[row[b]:row[b + 1], i].double(), kh[at[b]:at[b + 1]], vh[at[b]:at[b + 1]], scale)
    return out


# --------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    """Inputs and outputs once each.  A cached group of 32 values is 16 bytes of codes, 2 of low, 2 of step."""
    kind, d = case["kind"], case["head_dim"]
    if kind == "rotate":
        elements = case["tokens"] * (case["q_heads"] + case["k_heads"]) * d
        return {"bytes": 4 * elements + case["tokens"] * (4 + 4 * case["rotary_dim"]) + (4 * d if case["norm"] else 0),
                "flops": (7 if case["norm"] else 3) * elements}
    new, total = _new_and_total(case)
    if kind == "append":        # the new rows read, held, and given back from what is held
        elements = 2 * sum(new) * case["kv_heads"] * d
        return {"bytes": 4 * elements + 2 * elements * 20 // 32, "flops": 8 * elements}
    ends = 4 * sum(new) * case["q_heads"] * d
    flops = 4 * d * case["q_heads"] * _pairs(case)
    if kind == "attend":
        return {"bytes": ends + 2 * sum(total) * case["kv_heads"] * d * 20 // 32 + 4 * sum(-(-t // case["page_tokens"]) for t in total), "flops": flops}
    return {"bytes": ends + 4 * sum(total) * case["kv_heads"] * d, "flops": flops}
