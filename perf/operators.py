"""What the speed of the attention operators is measured on: the 4-bit cache of keys and values
(written, read back, attended to) and the attention of a prompt with a sliding window and sinks.

Activations are matrices of features x tokens with the tokens innermost, as the linear layers of this
library take and leave them; head h owns rows h * head_dim and up.  A case is a dict of plain values:

* ``kind`` "store": ``tokens`` columns of new keys and values are quantised into the cache at slots all over
  its pages, and the same slots are read back.
* ``kind`` "cache": ``batch`` sequences with ``queries`` new tokens each attend to the cache, which holds
  up to ``length`` tokens of each, the new ones among them.
* ``kind`` "prompt": ``batch`` sequences of up to ``length`` tokens attend to themselves, keys and values in 16 bits.

``ragged`` spreads the sequences' lengths below ``length`` by up to that many per cent, ``window`` 0 is none.
A key at position j is visible from position p if j <= p and (no window, or p - j < window, or j < sinks).
A block of 32 features of one token and head shares a scale 2^e, e = floor(log2(largest magnitude)) - 2, and its
values are rounded to a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times the scale, ties to the even code.
"""
import math
import random

import torch

own = False
DEVICE = "cuda:0"
DTYPE = {"f16": torch.float16, "bf16": torch.bfloat16}
MOST_FLOPS = 1.0e12            # of a drawn case: what the largest listed ones have
MOST_BYTES = 6.8e8
MOST_SCORES = 4.0e9            # the same with all scores before a query counted, those outside the window too


def _store(name, tokens, heads, head_dim, page, fmt):
    return dict(name=name, kind="store", tokens=tokens, heads=heads, head_dim=head_dim, page=page, fmt=fmt)


def _cache(name, batch, queries, length, ragged, q_heads, heads, head_dim, page, window, sinks, fmt):
    return dict(name=name, kind="cache", batch=batch, queries=queries, length=length, ragged=ragged, q_heads=q_heads,
                heads=heads, head_dim=head_dim, page=page, window=window, sinks=sinks, fmt=fmt)


def _prompt(name, batch, length, ragged, q_heads, heads, head_dim, window, sinks, fmt):
    return dict(name=name, kind="prompt", batch=batch, length=length, ragged=ragged, q_heads=q_heads, heads=heads,
                head_dim=head_dim, window=window, sinks=sinks, fmt=fmt)


def listed():
    return [
        # a decoding step of 64 sequences: one token each
        _store("store_step", 64, 8, 128, 64, "f16"),
        # the prompts of a batch, token count as it comes, the heads of Transformer-big (1024 features)
        _store("store_prompt", 8191, 16, 64, 32, "bf16"),
        # long documents taken in at once
        _store("store_large", 65536, 8, 128, 128, "f16"),
        # one user, one token, a short conversation: latency is all that counts
        _cache("decode_single", 1, 1, 1023, 0, 16, 16, 64, 32, 0, 0, "f16"),
        # a serving batch of different lengths, grouped heads over the 8192 features of the largest layer
        _cache("decode_batch", 64, 1, 4096, 80, 64, 8, 128, 64, 0, 0, "bf16"),
        # few users with very long contexts: the work has to be split along the context
        _cache("decode_long", 2, 1, 131071, 10, 64, 8, 128, 128, 0, 0, "f16"),
        # many sequences of a model that looks back over a window and keeps the first tokens
        _cache("decode_window", 128, 1, 16384, 50, 16, 16, 64, 64, 1024, 4, "bf16"),
        # a few drafted tokens of every sequence checked at once
        _cache("draft_check", 24, 5, 3001, 60, 64, 8, 128, 32, 0, 0, "f16"),
        # a long prompt taken in by chunks: 1024 more tokens on top of what the cache holds
        _cache("chunk", 4, 1024, 9000, 40, 64, 8, 128, 64, 0, 0, "bf16"),
        # a sentence
        _prompt("prompt_short", 1, 77, 0, 16, 16, 64, 0, 0, "f16"),
        # long prompts of different lengths, grouped heads
        _prompt("prompt_batch", 4, 4096, 25, 64, 8, 128, 0, 0, "bf16"),
        # documents under a window with sinks, the heads of Transformer-big
        _prompt("prompt_window", 2, 16384, 5, 16, 16, 64, 1024, 4, "f16"),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    while True:
        case = _draw(rng)
        w = work(case)
        scores = work({**case, "window": 0})["flops"] / 4 / case["head_dim"] if case["kind"] != "store" else 0
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES and scores <= MOST_SCORES:
            return case


def _draw(rng):
    kind = rng.choice(["store", "cache", "cache", "cache", "prompt", "prompt"])
    fmt = rng.choice(["f16", "bf16"])
    heads, group, head_dim = rng.choice([1, 2, 4, 8, 16]), rng.choice([1, 2, 4, 5, 8]), rng.choice([64, 64, 96, 128, 128])
    page = rng.choice([32, 64, 128])
    window, sinks = rng.choice([(0, 0), (0, 0), (_spread(rng, 32, 4096), rng.choice([0, 1, 4, 33]))])
    ragged = rng.choice([0, 10, 50, 90])
    if kind == "store":
        return _store("", _spread(rng, 1, 65536), heads, head_dim, page, fmt)
    if kind == "cache":
        queries = rng.choice([1, 1, 1, rng.randint(2, 8), _spread(rng, 9, 2048)])
        length = max(queries, _spread(rng, 16, 131072))
        return _cache("", _spread(rng, 1, 128), queries, length, ragged, heads * group, heads, head_dim, page, window, sinks, fmt)
    return _prompt("", _spread(rng, 1, 32), _spread(rng, 16, 16384), ragged, heads * group, heads, head_dim, window, sinks, fmt)


def _lengths(case):
    """Tokens of every sequence; the first has the full length."""
    rng = random.Random("%(batch)d %(length)d %(ragged)d" % case)
    least = case.get("queries", 1)
    return [max(least, case["length"] - (rng.randrange(case["length"] * case["ragged"] // 100 + 1) if i else 0))
            for i in range(case["batch"])]


def _visible(p, case):
    """How many keys a query at position p sees."""
    if not case["window"]:
        return p + 1
    first = max(0, p - case["window"] + 1)
    return p + 1 - first + min(case["sinks"], first)


def _pairs(first, last, case):
    """Sum of _visible over the positions first..last-1, for any of them."""
    w = case["window"]
    steady = max(first, min(last, w + case["sinks"])) if w else last
    return sum(_visible(p, case) for p in range(first, steady)) + (last - steady) * (_visible(last, case) if steady < last else 0)


def work(case):
    heads, D = case["heads"], case["head_dim"]
    if case["kind"] == "store":
        values = 2 * case["tokens"] * heads * D
        # in, out, the cache written and read: 17 bytes for 32 values
        return {"bytes": values * 2 * 2 + 2 * values * 17 // 32 + 8 * case["tokens"], "flops": 2 * values}
    lengths = _lengths(case)
    if case["kind"] == "prompt":
        tokens = sum(lengths)
        pairs = sum(_pairs(0, n, case) for n in lengths)
        return {"bytes": tokens * D * 2 * (2 * case["q_heads"] + 2 * heads), "flops": 4 * D * case["q_heads"] * pairs}
    nq = case["queries"]
    pairs = sum(_pairs(n - nq, n, case) for n in lengths)
    # what any of a sequence's queries sees is read once
    seen = 0
    for n in lengths:
        first = max(0, n - nq - case["window"] + 1) if case["window"] else 0
        seen += n - first + min(case["sinks"], first)
    return {"bytes": seen * heads * D * 2 * 17 // 32 + case["batch"] * nq * D * case["q_heads"] * 4,
            "flops": 4 * D * case["q_heads"] * pairs}


# ---- inputs

def _keys_values(case, tokens, gen):
    """New keys and values: keys with a few strong features, as trained ones have, values without."""
    rows, dtype = case["heads"] * case["head_dim"], DTYPE[case["fmt"]]
    gain = torch.exp(0.5 * torch.randn(rows, 1, device=DEVICE, generator=gen))
    k = (torch.randn(rows, tokens, device=DEVICE, generator=gen) * gain).to(dtype)
    v = torch.randn(rows, tokens, device=DEVICE, generator=gen).to(dtype)
    return k, v


def _query(case, tokens, gen):
    return torch.randn(case["q_heads"] * case["head_dim"], tokens, device=DEVICE, generator=gen).to(DTYPE[case["fmt"]])


def _pages(case, lengths, seed):
    """Pages of all sequences in no particular order: (pages in all, table of every sequence's pages)."""
    each = [-(-n // case["page"]) for n in lengths]
    pages = sum(each)
    order = list(range(pages))
    random.Random(seed).shuffle(order)
    table, at = [], 0
    for n in each:
        table.append(order[at:at + n] + [-1] * (max(each) - n))
        at += n
    return pages, torch.tensor(table, dtype=torch.int32)


def _new_cache(case, pages):
    """The library's cache, or what the plain form keeps: two codes a byte and a scale byte for 32."""
    heads, D = case["heads"], case["head_dim"]
    if own:
        from paper_2203_05016_amd import binding
        return binding.KVCache(pages, case["page"], heads, D, DTYPE[case["fmt"]], DEVICE)
    slots = pages * case["page"]
    return {name: (torch.zeros(slots, heads, D // 2, dtype=torch.uint8, device=DEVICE),
                   torch.zeros(slots, heads, D // 32, dtype=torch.uint8, device=DEVICE)) for name in "kv"}


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    state = {"case": case}
    if case["kind"] == "store":
        pages = -(-case["tokens"] // case["page"]) + 1
        state["cache"] = _new_cache(case, pages)
        state["k"], state["v"] = _keys_values(case, case["tokens"], gen)
        order = torch.randperm(pages * case["page"], device=DEVICE, generator=gen)[:case["tokens"]]
        if case["tokens"] >= case["page"]:        # prompts fill whole pages, in order
            first = torch.randperm(pages, device=DEVICE, generator=gen) * case["page"]
            order = (first[:, None] + torch.arange(case["page"], device=DEVICE)).flatten()[:case["tokens"]]
        state["slots"] = order.to(torch.int32)
        return state
    lengths = _lengths(case)
    state["lengths"] = lengths
    if case["kind"] == "prompt":
        state["starts"] = torch.tensor([0] + lengths, dtype=torch.int32).cumsum(0, dtype=torch.int32).to(DEVICE)
        state["q"] = _query(case, sum(lengths), gen)
        state["k"], state["v"] = _keys_values(case, sum(lengths), gen)
        return state
    pages, table = _pages(case, lengths, seed)
    state["cache"] = _new_cache(case, pages)
    state["table"] = table.to(DEVICE)
    state["size"] = torch.tensor(lengths, dtype=torch.int32, device=DEVICE)
    state["starts"] = None
    if case["queries"] > 1:
        state["starts"] = (torch.arange(case["batch"] + 1, device=DEVICE) * case["queries"]).to(torch.int32)
    state["q"] = _query(case, case["batch"] * case["queries"], gen)
    for b, n in enumerate(lengths):
        k, v = _keys_values(case, n, gen)
        slots = _slots_of(case, table[b].to(DEVICE), n)
        if own:
            state["cache"].write(k, v, slots)
        else:
            _plain_write(case, state["cache"], k, v, slots)
    return state


def _slots_of(case, pages, length):
    at = torch.arange(length, device=DEVICE)
    return (pages[at // case["page"]].long() * case["page"] + at % case["page"]).to(torch.int32)


# ---- the calls

def run(state):
    case = state["case"]
    if not own:
        return _plain(case, state)
    from paper_2203_05016_amd import binding
    if case["kind"] == "store":
        state["cache"].write(state["k"], state["v"], state["slots"])
        return state["cache"].read(state["slots"])
    if case["kind"] == "prompt":
        return binding.window_attention(state["q"], state["k"], state["v"], case["head_dim"], state["starts"],
                                        max_tokens=max(state["lengths"]), window=case["window"], sinks=case["sinks"])
    return state["cache"].attention(state["q"], state["table"], state["size"], starts=state["starts"],
                                    max_queries=case["queries"], max_length=max(state["lengths"]),
                                    window=case["window"], sinks=case["sinks"])


# ---- the plain forms: elementary operations in 32 bits

def _quantise(x):
    """(tokens, heads, D) in 32 bits -> two codes a byte, scale bytes."""
    blocks = x.unflatten(-1, (-1, 32))
    largest = blocks.abs().amax(-1, keepdim=True)
    exponent = (torch.frexp(largest).exponent - 3).clamp(min=-126)
    exponent = torch.where(largest > 0, exponent, torch.full_like(exponent, -126))
    a = torch.ldexp(blocks.abs(), -exponent)
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5))
    code = torch.where(torch.isfinite(largest), code + 8 * torch.signbit(blocks), 0).to(torch.uint8).flatten(-2)
    scale = torch.where(torch.isfinite(largest), exponent + 127, 255).squeeze(-1).to(torch.uint8)
    return code[..., 0::2] | code[..., 1::2] << 4, scale


def _dequantise(packed, scale):
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float32, device=packed.device)
    grid = torch.cat([grid, -grid])
    code = torch.stack([packed & 15, packed >> 4], -1).flatten(-2)
    value = torch.ldexp(grid[code.int()].unflatten(-1, (-1, 32)), (scale.int() - 127).unsqueeze(-1))
    return torch.where((scale == 255).unsqueeze(-1), torch.nan, value).flatten(-2)


def _plain_write(case, cache, k, v, slots):
    for name, x in (("k", k), ("v", v)):
        x = x.float().view(case["heads"], case["head_dim"], -1).permute(2, 0, 1)
        codes, scales = _quantise(x)
        cache[name][0][slots.long()] = codes
        cache[name][1][slots.long()] = scales


def _plain_read(cache, name, slots):
    codes, scales = cache[name]
    return _dequantise(codes[slots.long()], scales[slots.long()])          # (tokens, heads, D)


def _needed(first, last, case):
    """The keys that queries at positions first..last-1 need: the first s, and from lo to last."""
    lo = max(0, first - case["window"] + 1) if case["window"] else 0
    return min(case["sinks"], lo), lo


def _positions(first, last, case):
    s, lo = _needed(first, last, case)
    return torch.cat([torch.arange(s, device=DEVICE), torch.arange(lo, last, device=DEVICE)])


def _attend(q, k, v, first, case):
    """q (Hq, n, D) at positions first and up, k and v (H, keys, D) at the positions these need, in 32 bits."""
    heads, keys, D = k.shape
    group, n = q.shape[0] // heads, q.shape[1]
    out = torch.empty_like(q)
    s0, lo0 = _needed(first, first + n, case)
    step = max(1, (1 << 28) // (q.shape[0] * keys))
    if case["window"]:
        step = min(step, max(256, case["window"]))
    for i in range(0, n, step):
        part = q[:, i:i + step]
        m = part.shape[1]
        s, lo = _needed(first + i, first + i + m, case)
        begin, end = lo - lo0 + s0, first + i + m - lo0 + s0
        kc, vc = (torch.cat([x[:, :s], x[:, begin:end]], 1) if s else x[:, begin:end].contiguous() for x in (k, v))
        p = torch.arange(first + i, first + i + m, device=q.device)[:, None]
        j = _positions(first + i, first + i + m, case)[None]
        seen = j <= p
        if case["window"]:
            seen &= (p - j < case["window"]) | (j < case["sinks"])
        score = torch.matmul(part.reshape(heads, group * m, D), kc.transpose(1, 2).contiguous()) * (D ** -0.5)
        score = score.view(heads, group, m, -1).masked_fill_(~seen, -torch.inf)
        score = (score - score.amax(-1, keepdim=True)).exp_()
        total = score.sum(-1, keepdim=True)
        o = torch.matmul(score.view(heads, group * m, -1), vc).view(heads, group, m, D) / total
        out[:, i:i + m] = o.reshape(heads * group, m, D)
    return out


def _by_head(x, D):
    return x.view(-1, D, x.shape[-1]).transpose(1, 2).float()              # (heads, tokens, D)


def _plain(case, state):
    D, dtype = case["head_dim"], DTYPE[case["fmt"]]
    if case["kind"] == "store":
        _plain_write(case, state["cache"], state["k"], state["v"], state["slots"])
        return tuple(_plain_read(state["cache"], name, state["slots"]).flatten(1).t().to(dtype).contiguous() for name in "kv")
    out = torch.empty_like(state["q"])
    at = 0
    for b, n in enumerate(state["lengths"]):
        nq = n if case["kind"] == "prompt" else case["queries"]
        q = _by_head(state["q"][:, at:at + nq], D)
        if case["kind"] == "prompt":
            k, v = _by_head(state["k"][:, at:at + n], D), _by_head(state["v"][:, at:at + n], D)
        else:
            at_pages = _positions(n - nq, n, case)
            slots = state["table"][b].long()[at_pages // case["page"]] * case["page"] + at_pages % case["page"]
            k, v = (_plain_read(state["cache"], name, slots).transpose(0, 1) for name in "kv")
        o = _attend(q, k.contiguous(), v.contiguous(), n - nq, case)
        out[:, at:at + nq] = o.transpose(1, 2).reshape(-1, nq).to(dtype)
        at += nq
    return out


# ---- the definition in 64 bits

def _nearest(x):
    """What the cache holds of (rows, tokens): the nearest value its blocks can hold, in 64 bits."""
    blocks = x.double().view(-1, 32, x.shape[-1])
    largest = blocks.abs().amax(1, keepdim=True)
    scale = torch.exp2(torch.floor(torch.log2(largest.clamp(min=2.0 ** -140))).sub(2).clamp(min=-126))
    ratio, best, off = blocks.abs() / scale, torch.zeros_like(blocks), None
    # even codes first: of two values as near, the one seen first stays
    for value in (0.0, 1.0, 2.0, 4.0, 0.5, 1.5, 3.0, 6.0):
        d = (ratio - value).abs()
        if off is None:
            off = d
        else:
            best, off = torch.where(d < off, value, best), torch.minimum(d, off)
    return (torch.copysign(best, blocks) * scale).view(x.shape)


def exact(case, seed):
    if work(case)["flops"] > 1.0e13:
        return None
    D = case["head_dim"]
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    if case["kind"] == "store":
        k, v = _keys_values(case, case["tokens"], gen)
        return _nearest(k), _nearest(v)
    lengths = _lengths(case)
    prompt = case["kind"] == "prompt"
    q = _query(case, sum(lengths) if prompt else case["batch"] * case["queries"], gen)
    if prompt:
        keys, values = _keys_values(case, sum(lengths), gen)
    out, at = torch.empty(q.shape, dtype=torch.float64, device=DEVICE), 0
    for n in lengths:
        if prompt:
            nq, k, v = n, keys[:, at:at + n].double(), values[:, at:at + n].double()
        else:
            nq, (k, v) = case["queries"], (_nearest(x) for x in _keys_values(case, n, gen))
        group = case["q_heads"] // case["heads"]
        position = torch.arange(n - nq, n, device=DEVICE)
        for head in range(case["q_heads"]):
            kh, vh = (x[head // group * D:head // group * D + D] for x in (k, v))
            qh = q[head * D:head * D + D, at:at + nq].double()
            for i in range(0, nq, 2048):
                p = position[i:i + 2048]
                s = kh.t().contiguous() @ qh[:, i:i + 2048].contiguous() / math.sqrt(D)          # keys x queries
                j = torch.arange(n, device=DEVICE).unsqueeze(1)
                hidden = j > p
                if case["window"]:
                    hidden |= (j <= p - case["window"]) & (j >= case["sinks"])
                weight = torch.softmax(s.masked_fill(hidden, -math.inf), 0)
                out[head * D:head * D + D, at + i:at + i + len(p)] = vh.contiguous() @ weight
        at += nq
    return out
