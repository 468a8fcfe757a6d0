"""What the speed of the operators around a shared cache is measured on: norms of queries and keys with the rotation by
position, attention of sequences that share prefixes, and the bookkeeping of the cache's pages.

Activations are matrices of features x tokens with the tokens innermost, as the linear layers of this
library take and leave them; head h owns rows h * head_dim and up.  A case is a dict of plain values:

* ``kind`` "rotate": ``tokens`` columns of queries and keys.  Every head's column is divided by the root of its mean square (``norm``)
  and multiplied by weights, then its first 2 * ``pairs`` features are turned, in pairs of neighbours (``interleaved``) or of
  the two halves, by position * frequency; the pairs are dealt to ``axes`` rows of positions, one behind the other.
* ``kind`` "shared": ``prefixes`` prefixes of up to ``prefix`` tokens, each shared by ``batch`` sequences with up to ``length`` tokens of their own,
  the last ``queries`` of which attend to the prefix and to their own tokens up to themselves, all in the 4-bit cache.
* ``kind`` "extend": ``batch`` sequences of up to ``length`` tokens get up to ``count`` more: pages, and the slots to write them to.
* ``kind`` "fork": ``batch`` sequences, in families of ``family``, continue what a member of the family has; pages that are not yet full
  are copied for all but the first that continues them.  What nothing continues is given up.
* ``kind`` "compact": the pages of ``batch`` sequences, ``live`` per cent of the cache, move to its front.

``ragged`` spreads lengths below the longest by up to that many per cent.  Free pages are taken from the lowest up.  A block of 32 features
of one token and head shares a scale 2^e, e = floor(log2(largest magnitude)) - 2, and its
values are rounded to a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times the scale, ties to the even code.
"""
import math
import random

import numpy as np
import torch

own = False
DEVICE = "cuda:0"
DTYPE = {"f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-6
MOST_FLOPS = 5.5e11            # of a drawn case: what the largest listed ones have
MOST_BYTES = 3.0e8
MOST_CACHE = 6.0e8             # bytes of a cache whose pages are moved
MOST_SCORES = 1.1e9            # of the attention's plain form


def _rotate(name, tokens, q_heads, heads, head_dim, pairs, axes, norm, interleaved, furthest, fmt):
    return dict(name=name, kind="rotate", tokens=tokens, q_heads=q_heads, heads=heads, head_dim=head_dim, pairs=pairs, axes=axes,
                norm=norm, interleaved=interleaved, furthest=furthest, fmt=fmt)


def _shared(name, prefixes, batch, prefix, length, ragged, queries, q_heads, heads, head_dim, page, fmt):
    return dict(name=name, kind="shared", prefixes=prefixes, batch=batch, prefix=prefix, length=length, ragged=ragged, queries=queries,
                q_heads=q_heads, heads=heads, head_dim=head_dim, page=page, fmt=fmt)


def _extend(name, batch, length, count, ragged, page, pages):
    return dict(name=name, kind="extend", batch=batch, length=length, count=count, ragged=ragged, page=page, pages=pages)


def _fork(name, batch, family, length, ragged, heads, head_dim, page, pages):
    return dict(name=name, kind="fork", batch=batch, family=family, length=length, ragged=ragged, heads=heads, head_dim=head_dim,
                page=page, pages=pages)


def _compact(name, batch, live, heads, head_dim, page, pages):
    return dict(name=name, kind="compact", batch=batch, live=live, heads=heads, head_dim=head_dim, page=page, pages=pages)


def listed():
    return [
        # a decoding step of 64 sequences, grouped heads over the 8192 features of the largest layer
        _rotate("rotate_step", 64, 64, 8, 128, 64, 1, True, False, 131072, "bf16"),
        # prompts with images among the text: positions in time, height and width, token count as it comes
        _rotate("rotate_images", 8191, 64, 8, 128, 64, 3, True, False, 32768, "bf16"),
        # four answers to one short question: latency is all that counts
        _shared("shared_small", 1, 4, 601, 40, 50, 1, 16, 16, 64, 32, "f16"),
        # a decoding step of a serving batch whose requests all begin with the same instructions
        _shared("shared_step", 1, 64, 8001, 512, 90, 1, 64, 8, 128, 64, "bf16"),
        # 8 answers each to 16 long questions, three drafted tokens of every answer checked at once
        _shared("shared_drafts", 16, 8, 4096, 300, 60, 3, 32, 8, 96, 32, "f16"),
        # requests of ordinary length taken in at once behind a long document they are about
        _shared("shared_prompts", 1, 8, 4096, 512, 0, 512, 64, 8, 128, 64, "bf16"),
        # one more token of 64 sequences: most need no page
        _extend("extend_step", 64, 4096, 1, 80, 64, 8192),
        # 256 prompts are given their pages
        _extend("extend_prompts", 256, 64, 8192, 70, 32, 65536),
        # a step of a search with four beams
        _fork("fork_beams", 4, 4, 700, 0, 16, 64, 32, 128),
        # the same for 64 requests at once, 8 beams each
        _fork("fork_batch", 512, 8, 2000, 60, 8, 128, 32, 16000),
        # a small cache with a third of its pages in use
        _compact("compact_small", 8, 33, 16, 64, 32, 200),
        # half of a large one's sequences have ended
        _compact("compact_large", 128, 50, 8, 128, 64, 8000),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _page_bytes(case):
    scales = 2 if case["head_dim"] == 64 else 4
    return case["heads"] * case["page"] * (case["head_dim"] + 2 * scales)


def draw(rng):
    while True:
        case = _draw(rng)
        w = work(case)
        cache = case["pages"] * _page_bytes(case) if case["kind"] in ("fork", "compact") else 0
        scores = w["flops"] / 4 / case["head_dim"] if case["kind"] == "shared" else 0
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES and cache <= MOST_CACHE and scores <= MOST_SCORES:
            return case


def _draw(rng):
    kind = rng.choice(["rotate", "rotate", "shared", "shared", "shared", "extend", "fork", "compact"])
    fmt = rng.choice(["f16", "bf16"])
    heads, group, head_dim = rng.choice([1, 2, 4, 8, 16]), rng.choice([1, 2, 4, 5, 8]), rng.choice([64, 64, 96, 128, 128])
    page = rng.choice([32, 64, 128])
    ragged = rng.choice([0, 10, 50, 90])
    if kind == "rotate":
        pairs = rng.choice([head_dim // 2, head_dim // 2, head_dim // 4, rng.randint(3, head_dim // 2)])
        return _rotate("", _spread(rng, 1, 16384), heads * group, heads, head_dim, pairs, rng.choice([1, 1, 2, 3]), rng.random() < 0.8,
                       rng.random() < 0.3, _spread(rng, 64, 1048576), fmt)
    if kind == "shared":
        queries = rng.choice([1, 1, 1, rng.randint(2, 8), _spread(rng, 9, 512)])
        return _shared("", rng.choice([1, 1, 1, _spread(rng, 2, 16)]), _spread(rng, 1, 64), _spread(rng, 32, 32768),
                       max(queries, _spread(rng, 1, 2048)), ragged, queries, heads * group, heads, head_dim, page, fmt)
    if kind == "extend":
        batch, length, count = _spread(rng, 1, 512), _spread(rng, 1, 8192), rng.choice([1, 1, rng.randint(2, 16), _spread(rng, 17, 8192)])
        return _extend("", batch, length, count, ragged, page, batch * (-(-(length + count) // page)) + rng.randint(0, 4096))
    if kind == "fork":
        family = _spread(rng, 1, 16)
        batch, length = family * _spread(rng, 1, 64), _spread(rng, 1, 8192)
        return _fork("", batch, family, length, ragged, heads, head_dim, page, batch * (-(-length // page) + 1) + rng.randint(0, 100))
    return _compact("", _spread(rng, 1, 128), rng.randint(5, 95), heads, head_dim, page, _spread(rng, 16, 8192))


def _lengths(batch, length, ragged, least=0):
    """Tokens of every sequence; the first has the full length."""
    rng = random.Random("%d %d %d" % (batch, length, ragged))
    return [max(least, length - (rng.randrange(length * ragged // 100 + 1) if i else 0)) for i in range(batch)]


def _tokens_of(case):
    """Of a "shared" case: tokens of every prefix, and every sequence's own."""
    return (_lengths(case["prefixes"], case["prefix"], case["ragged"]),
            _lengths(case["prefixes"] * case["batch"], case["length"], case["ragged"], case["queries"]))


def work(case):
    kind = case["kind"]
    if kind == "rotate":
        values = case["tokens"] * case["head_dim"] * (case["q_heads"] + case["heads"])
        return {"bytes": 4 * values + 4 * case["axes"] * case["tokens"], "flops": 8 * values}
    if kind == "shared":
        prefix, own_tokens = _tokens_of(case)
        nq, D = case["queries"], case["head_dim"]
        pairs = sum(nq * case["batch"] * n for n in prefix) + sum(nq * n - nq * (nq - 1) // 2 for n in own_tokens)
        return {"bytes": (sum(prefix) + sum(own_tokens)) * case["heads"] * D * 2 * 17 // 32 + len(own_tokens) * nq * D * case["q_heads"] * 4,
                "flops": 4 * D * case["q_heads"] * pairs}
    if kind == "extend":
        lengths, counts = _extend_numbers(case)
        held = sum(-(-(n + c) // case["page"]) for n, c in zip(lengths, counts))
        return {"bytes": 8 * held + 8 * case["pages"] + 4 * sum(counts) + 16 * case["batch"], "flops": held + case["pages"] + sum(counts)}
    if kind == "fork":
        lengths, parents = _fork_numbers(case)
        entries = sum(-(-lengths[b] // case["page"]) for b in parents)
        copies = sum(1 for i, b in enumerate(parents) if b in parents[:i] and lengths[b] % case["page"])
        return {"bytes": 8 * entries + 8 * case["pages"] + 12 * case["batch"] + 2 * copies * _page_bytes(case), "flops": 2 * entries + case["pages"]}
    rows, moved = _compact_numbers(case)
    entries = sum(len(r) for r in rows)
    return {"bytes": 8 * entries + 8 * case["pages"] + 2 * moved * _page_bytes(case), "flops": entries + case["pages"]}


# ---- inputs: what the host knows of a case, and what lies on the GPU

def _extend_numbers(case):
    lengths = _lengths(case["batch"], case["length"], case["ragged"])
    return lengths, _lengths(case["batch"], case["count"], case["ragged"])[::-1]


def _fork_numbers(case):
    """Lengths, the same in all of a family, and whom every sequence continues: what a search has after it has picked the best."""
    rng = random.Random("%(batch)d %(family)d %(length)d" % case)
    family = case["family"]
    each = _lengths(case["batch"] // family, case["length"], case["ragged"], 1)
    return ([each[b // family] for b in range(case["batch"])],
            [b - b % family + min(rng.randrange(family), rng.randrange(family)) for b in range(case["batch"])])


def _compact_numbers(case):
    """Pages of every sequence, and how many pages have to move."""
    rng = random.Random("%(batch)d %(live)d %(pages)d" % case)
    live = max(1, case["pages"] * case["live"] // 100)
    pages = rng.sample(range(case["pages"]), live)
    batch = min(case["batch"], live)
    return [pages[b::batch] for b in range(batch)], sum(1 for p in pages if p >= live)


def _filled(rows, width):
    return [list(r) + [-1] * (width - len(r)) for r in rows]


def _int32(values):
    return torch.tensor(values, dtype=torch.int32).to(DEVICE)


def _keys_values(case, tokens, gen):
    """New keys and values: keys with a few strong features, as trained ones have, values without."""
    rows, dtype = case["heads"] * case["head_dim"], DTYPE[case["fmt"]]
    gain = torch.exp(0.5 * torch.randn(rows, 1, device=DEVICE, generator=gen))
    k = (torch.randn(rows, tokens, device=DEVICE, generator=gen) * gain).to(dtype)
    v = torch.randn(rows, tokens, device=DEVICE, generator=gen).to(dtype)
    return k, v


def _query(case, gen):
    columns = case["prefixes"] * case["batch"] * case["queries"]
    return torch.randn(case["q_heads"] * case["head_dim"], columns, device=DEVICE, generator=gen).to(DTYPE[case["fmt"]])


def _rotate_inputs(case, gen):
    """Queries and keys as one projection leaves them, weights near one, positions of a batch of prompts."""
    dtype, D, n = DTYPE[case["fmt"]], case["head_dim"], case["tokens"]
    gain = torch.exp(0.5 * torch.randn((case["q_heads"] + case["heads"]) * D, 1, device=DEVICE, generator=gen))
    x = (torch.randn(len(gain), n, device=DEVICE, generator=gen) * gain).to(dtype)
    weights = [(1 + 0.1 * torch.randn(D, device=DEVICE, generator=gen)).to(dtype) if case["norm"] else None for _ in range(2)]
    first = torch.randint(0, max(1, case["furthest"] - n + 1), (1,), device=DEVICE, generator=gen)
    steps = torch.arange(n, device=DEVICE)
    rows = [first + steps, first + steps // 32 % 32, first + steps % 32][:case["axes"]]       # time, height, width
    positions = torch.stack(rows).to(torch.int32)
    frequencies = torch.tensor([10000.0 ** (-i / case["pairs"]) for i in range(case["pairs"])], dtype=torch.float64).to(DEVICE)
    axes = _int32([i * case["axes"] // case["pairs"] for i in range(case["pairs"])])
    return dict(x=x, weights=weights, positions=positions, frequencies=frequencies, axes=axes)


def _cache_bytes(case, gen):
    return torch.randint(0, 256, (case["pages"], _page_bytes(case)), dtype=torch.uint8, device=DEVICE, generator=gen)


def _page_order(pages, seed):
    order = list(range(pages))
    random.Random(seed).shuffle(order)
    return order


def _page_state(case, seed):
    """Table, lengths and uses as lists of an "extend", "fork" or "compact" case."""
    kind, page = case["kind"], case["page"]
    if kind == "compact":
        rows, _ = _compact_numbers(case)
        order = _page_order(len(rows), seed)
        rows = [rows[i] for i in order]
        lengths, width = [len(r) * page for r in rows], max(len(r) for r in rows)
    else:
        lengths = (_extend_numbers if kind == "extend" else _fork_numbers)(case)[0]
        order, rows = _page_order(case["pages"], seed), []
        family = case.get("family", 1)
        for b, n in enumerate(lengths):
            shared = n // page * 3 // 4 if b % family else 0       # the beams of a search share most of what they have
            rows.append((rows[b - b % family][:shared] if shared else []) + [order.pop() for _ in range(-(-n // page) - shared)])
        width = -(-(case["length"] + case.get("count", 0)) // page)
    uses = [0] * case["pages"]
    for r in rows:
        for p in r:
            uses[p] += 1
    return _filled(rows, width), lengths, uses


def _slots_of(case, pages, length):
    at = torch.arange(length, device=DEVICE)
    return (pages[at // case["page"]].long() * case["page"] + at % case["page"]).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    state = {"case": case}
    if case["kind"] == "rotate":
        state.update(_rotate_inputs(case, gen))
        state["q"], state["k"] = state.pop("x").split([case["q_heads"] * case["head_dim"], case["heads"] * case["head_dim"]])
        return state
    if case["kind"] == "shared":
        return _prepare_shared(case, seed, gen, state)
    table, lengths, uses = _page_state(case, seed)
    state["table"], state["lengths"], state["uses"] = _int32(table), _int32(lengths), _int32(uses)
    if case["kind"] == "extend":
        counts = _extend_numbers(case)[1]
        state["counts"], state["tokens"] = _int32(counts), sum(counts)
    if case["kind"] == "fork":
        state["parents"] = _int32(_fork_numbers(case)[1])
    if case["kind"] != "extend":
        state["data"] = _cache_bytes(case, gen)
    if own:
        from paper_2203_05016_amd import binding
        state["cache"] = binding.KVCache(case["pages"], case["page"], case.get("heads", 1), case.get("head_dim", 64), torch.float16, DEVICE)
        if case["kind"] != "extend":
            state["cache"].data.copy_(state.pop("data"))
    return state


def _prepare_shared(case, seed, gen, state):
    prefix, own_tokens = _tokens_of(case)
    state["prefix"], state["own"] = prefix, own_tokens
    each = [-(-n // case["page"]) for n in prefix + own_tokens]
    order = _page_order(sum(each), seed)
    rows = [[order.pop() for _ in range(n)] for n in each]
    state["prefix_table"] = _int32(_filled(rows[:len(prefix)], max(each[:len(prefix)])))
    state["table"] = _int32(_filled(rows[len(prefix):], max(each[len(prefix):])))
    state["prefix_size"], state["size"] = _int32(prefix), _int32(own_tokens)
    state["members"] = _int32([g * case["batch"] for g in range(len(prefix) + 1)]) if len(prefix) > 1 else None
    state["starts"] = _int32([b * case["queries"] for b in range(len(own_tokens) + 1)]) if case["queries"] > 1 else None
    heads, D = case["heads"], case["head_dim"]
    if own:
        from paper_2203_05016_amd import binding
        state["cache"] = binding.KVCache(sum(each), case["page"], heads, D, DTYPE[case["fmt"]], DEVICE)
    else:
        slots = sum(each) * case["page"]
        state["cache"] = {name: (torch.zeros(slots, heads, D // 2, dtype=torch.uint8, device=DEVICE),
                                 torch.zeros(slots, heads, D // 32, dtype=torch.uint8, device=DEVICE)) for name in "kv"}
    state["q"] = _query(case, gen)
    for i, n in enumerate(prefix + own_tokens):
        k, v = _keys_values(case, n, gen)
        slots = _slots_of(case, _int32(rows[i]), n)
        if own:
            state["cache"].write(k, v, slots)
        else:
            _plain_write(case, state["cache"], k, v, slots)
    return state


# ---- the calls

def run(state):
    case = state["case"]
    kind = case["kind"]
    if not own:
        return {"rotate": _plain_rotate, "shared": _plain_shared, "extend": _plain_extend, "fork": _plain_fork, "compact": _plain_compact}[kind](case, state)
    from paper_2203_05016_amd import binding
    if kind == "rotate":
        return binding.norm_rotate(state["q"], state["k"], case["head_dim"], state["positions"], state["frequencies"],
                                   axes=state["axes"] if case["axes"] > 1 else None, q_weight=state["weights"][0], k_weight=state["weights"][1],
                                   eps=EPS, norm=case["norm"], interleaved=case["interleaved"])
    cache = state["cache"]
    if kind == "shared":
        return cache.shared_attention(state["q"], state["prefix_table"], state["prefix_size"], state["table"], state["size"],
                                      members=state["members"], starts=state["starts"], max_queries=case["queries"],
                                      max_length=max(state["own"]), max_prefix=max(state["prefix"]), max_sharing=case["batch"] * case["queries"])
    if kind == "extend":
        return cache.extend(state["table"], state["lengths"], state["uses"], state["counts"], state["tokens"])
    if kind == "fork":
        return cache.fork(state["table"], state["lengths"], state["uses"], state["parents"]) + (cache.data,)
    return cache.compact(state["table"], state["uses"]) + (cache.data,)


# ---- the plain forms: elementary operations in 32 bits, angles in 64, whole numbers

def _plain_rotate(case, state):
    D, R, dtype = case["head_dim"], 2 * case["pairs"], DTYPE[case["fmt"]]
    angle = state["positions"][state["axes"].long()].double() * state["frequencies"][:, None]            # (pairs, tokens)
    cos, sin = angle.cos().float(), angle.sin().float()
    out = []
    for x, weight in zip((state["q"], state["k"]), state["weights"]):
        y = x.float().view(-1, D, x.shape[-1])
        if case["norm"]:
            y = y / ((y * y).mean(1, keepdim=True) + EPS).sqrt() * weight.float()[:, None]
        a, b = (y[:, 0:R:2], y[:, 1:R:2]) if case["interleaved"] else (y[:, :R // 2], y[:, R // 2:R])
        turned = (a * cos - b * sin, a * sin + b * cos)
        turned = torch.stack(turned, 2).flatten(1, 2) if case["interleaved"] else torch.cat(turned, 1)
        out.append(torch.cat([turned, y[:, R:]], 1).view_as(x).to(dtype))
    return tuple(out)


def _quantise(x):
    """(tokens, heads, D) in 32 bits -> two codes a byte, scale bytes."""
    blocks = x.unflatten(-1, (-1, 32))
    largest = blocks.abs().amax(-1, keepdim=True)
    exponent = (torch.frexp(largest).exponent - 3).clamp(min=-126)
    exponent = torch.where(largest > 0, exponent, torch.full_like(exponent, -126))
    a = torch.ldexp(blocks.abs(), -exponent)
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5))
    code = (code + 8 * torch.signbit(blocks)).to(torch.uint8).flatten(-2)
    return code[..., 0::2] | code[..., 1::2] << 4, (exponent + 127).squeeze(-1).to(torch.uint8)


def _plain_write(case, cache, k, v, slots):
    for name, x in (("k", k), ("v", v)):
        codes, scales = _quantise(x.float().view(case["heads"], case["head_dim"], -1).permute(2, 0, 1))
        cache[name][0][slots.long()] = codes
        cache[name][1][slots.long()] = scales


def _plain_read(cache, name, slots):
    codes, scales = (x[slots.long()] for x in cache[name])
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float32, device=DEVICE)
    code = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    value = torch.cat([grid, -grid])[code.int()].unflatten(-1, (-1, 32))
    return torch.ldexp(value, (scales.int() - 127).unsqueeze(-1)).flatten(-2).transpose(0, 1).contiguous()    # (heads, tokens, D)


def _plain_shared(case, state):
    heads, D, nq = case["heads"], case["head_dim"], case["queries"]
    out, group = torch.empty_like(state["q"]), case["q_heads"] // heads
    for g, shared in enumerate(state["prefix"]):
        slots = _slots_of(case, state["prefix_table"][g], shared)
        prefix = [_plain_read(state["cache"], name, slots) for name in "kv"]
        for b in range(g * case["batch"], (g + 1) * case["batch"]):
            n = state["own"][b]
            slots = _slots_of(case, state["table"][b], n)
            k, v = (torch.cat([x, _plain_read(state["cache"], name, slots)], 1) for x, name in zip(prefix, "kv"))
            q = state["q"][:, b * nq:(b + 1) * nq].float().view(heads, group, D, nq).transpose(2, 3).reshape(heads, group * nq, D)
            score = torch.matmul(q, k.transpose(1, 2).contiguous()) * D ** -0.5
            position = torch.arange(shared + n - nq, shared + n, device=DEVICE)
            hidden = torch.arange(shared + n, device=DEVICE) > position[:, None]
            score = score.view(heads, group, nq, -1).masked_fill_(hidden, -torch.inf)
            weight = (score - score.amax(-1, keepdim=True)).exp_()
            o = torch.matmul(weight.view(heads, group * nq, -1), v).view(heads, group, nq, D) / weight.sum(-1, keepdim=True)
            out[:, b * nq:(b + 1) * nq] = o.transpose(2, 3).reshape(-1, nq).to(out.dtype)
    return out


def _held(lengths, page):
    return (lengths.long() + page - 1) // page


def _free_pages(uses, most):
    """The free pages from the lowest up, -1 past the last: `most` entries."""
    free = uses == 0
    place = torch.where(free, free.cumsum(0) - 1, most).clamp(max=most)
    found = torch.full((most + 1,), -1, dtype=torch.int64, device=DEVICE)
    found.scatter_(0, place, torch.arange(len(uses), device=DEVICE))
    return torch.where(torch.arange(most, device=DEVICE) < free.sum(), found[:most], -1)


def _plain_extend(case, state):
    page, table, lengths, counts = case["page"], state["table"], state["lengths"].long(), state["counts"].long()
    before, after = _held(lengths, page), _held(lengths + counts, page)
    base = (after - before).cumsum(0) - (after - before)
    fresh = _free_pages(state["uses"], case["pages"])
    j = torch.arange(table.shape[1], device=DEVICE)[None]
    new = (j >= before[:, None]) & (j < after[:, None])
    taken = fresh[(base[:, None] + j - before[:, None]).clamp(0, case["pages"] - 1)]
    table = torch.where(new, taken, torch.where(j < before[:, None], table.long(), -1))
    uses = state["uses"].long().index_add(0, table.clamp(min=0).flatten(), (new & (table >= 0)).long().flatten())
    starts = torch.cat([torch.zeros_like(counts[:1]), counts.cumsum(0)])
    column = torch.arange(state["tokens"], device=DEVICE)
    row = torch.searchsorted(starts, column, right=True) - 1
    at = lengths[row] + column - starts[row]
    slots = table[row, at // page] * page + at % page
    return tuple(x.to(torch.int32) for x in (table, lengths + counts, uses, slots, starts))


def _plain_fork(case, state):
    page, pages, table, lengths, parents = case["page"], case["pages"], state["table"].long(), state["lengths"].long(), state["parents"].long()
    batch = len(parents)
    j = torch.arange(table.shape[1], device=DEVICE)[None]
    uses = state["uses"].long().index_add(0, table.clamp(min=0).flatten(), -(table >= 0).long().flatten())
    children = torch.where(parents[:, None] == torch.arange(batch, device=DEVICE), torch.arange(batch, device=DEVICE)[:, None], batch)
    first = children.amin(0)[parents] == torch.arange(batch, device=DEVICE)
    now, size = table[parents], lengths[parents]
    is_open = (j == (size // page)[:, None]) & (size % page != 0)[:, None]
    copied = is_open & ~first[:, None]
    uses = uses.index_add(0, now.clamp(min=0).flatten(), ((now >= 0) & ~copied).long().flatten())
    needs = copied.any(1)
    fresh = _free_pages(uses, batch)[(needs.cumsum(0) - 1).clamp(min=0)]
    source = torch.where(is_open, now, 0).sum(1)
    target = torch.where(needs, fresh, source)
    state["data"][target] = state["data"][source]
    now = torch.where(copied, fresh[:, None], now)
    uses = uses.index_add(0, fresh.clamp(min=0), needs.long())
    return now.to(torch.int32), size.to(torch.int32), uses.to(torch.int32), state["data"]


def _plain_compact(case, state):
    pages, uses, table = case["pages"], state["uses"].long(), state["table"].long()
    live, page = uses != 0, torch.arange(case["pages"], device=DEVICE)
    front = page < live.sum()
    moves, holes = live & ~front, ~live & front
    # the n-th page to move goes to the n-th hole
    source = torch.full((pages + 1,), 0, device=DEVICE).scatter_(0, torch.where(moves, moves.cumsum(0) - 1, pages), page)
    target = torch.full((pages + 1,), 0, device=DEVICE).scatter_(0, torch.where(holes, holes.cumsum(0) - 1, pages), page)
    goes = torch.where(moves, target[(moves.cumsum(0) - 1).clamp(min=0)], page)
    comes = torch.where(holes, source[(holes.cumsum(0) - 1).clamp(min=0)], page)
    state["data"].copy_(state["data"][comes])
    uses = torch.where(front, uses[comes], 0)
    table = torch.where(table >= 0, goes[table.clamp(min=0)], table)
    return table.to(torch.int32), uses.to(torch.int32), state["data"]


# ---- the definitions in 64 bits

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
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    kind = case["kind"]
    if kind == "rotate":
        return _exact_rotate(case, _rotate_inputs(case, gen))
    if kind == "shared":
        return _exact_shared(case, gen)
    table, lengths, uses = _page_state(case, seed)
    if kind == "extend":
        return tuple(_int32(x) for x in _exact_extend(case, table, lengths, uses))
    data = _cache_bytes(case, gen)
    if kind == "fork":
        numbers, copies = _exact_fork(case, table, lengths, uses)
    else:
        numbers, copies = _exact_compact(table, uses)
    for source, target in copies:
        data[target].copy_(data[source])
    return tuple(_int32(x) for x in numbers) + (data,)


def _exact_rotate(case, given):
    """Every pair as a complex number times e^(i angle)."""
    D, R, out = case["head_dim"], 2 * case["pairs"], []
    first = [2 * i if case["interleaved"] else i for i in range(case["pairs"])]
    second = [i + (1 if case["interleaved"] else case["pairs"]) for i in first]
    turn = torch.polar(torch.ones_like(given["frequencies"])[:, None],
                       given["frequencies"][:, None] * given["positions"].double()[given["axes"].long()])
    at = 0
    for heads, weight in zip((case["q_heads"], case["heads"]), given["weights"]):
        x = given["x"][at:at + heads * D].double().view(heads, D, -1)
        at += heads * D
        if case["norm"]:
            x = x * torch.rsqrt(x.square().sum(1, keepdim=True) / D + EPS) * weight.double().view(1, D, 1)
        z = torch.complex(x[:, first].contiguous(), x[:, second].contiguous()) * turn
        y = x.clone()
        y[:, first], y[:, second] = z.real, z.imag
        out.append(y.view(heads * D, -1))
    return tuple(out)


def _exact_shared(case, gen):
    D, nq, group = case["head_dim"], case["queries"], case["q_heads"] // case["heads"]
    prefix, own_tokens = _tokens_of(case)
    q = _query(case, gen)
    held = [[_nearest(x) for x in _keys_values(case, n, gen)] for n in prefix + own_tokens]
    out = torch.empty(q.shape, dtype=torch.float64, device=DEVICE)
    for b, n in enumerate(own_tokens):
        g = b // case["batch"]
        k, v = (torch.cat([x, y], 1) for x, y in zip(held[g], held[len(prefix) + b]))
        hidden = torch.arange(prefix[g] + n, device=DEVICE)[:, None] > prefix[g] + n - nq + torch.arange(nq, device=DEVICE)
        for head in range(case["q_heads"]):
            rows = slice(head // group * D, head // group * D + D)
            s = k[rows].t().contiguous() @ q[head * D:head * D + D, b * nq:(b + 1) * nq].double() / math.sqrt(D)      # keys x queries
            out[head * D:head * D + D, b * nq:(b + 1) * nq] = v[rows].contiguous() @ torch.softmax(s.masked_fill(hidden, -math.inf), 0)
    return out


def _exact_extend(case, table, lengths, uses):
    page, counts = case["page"], _extend_numbers(case)[1]
    free = iter([p for p, n in enumerate(uses) if n == 0])
    slots, starts = [], [0]
    for b, count in enumerate(counts):
        for j in range(-(-lengths[b] // page), -(-(lengths[b] + count) // page)):
            table[b][j] = next(free)
            uses[table[b][j]] = 1
        slots += [table[b][at // page] * page + at % page for at in range(lengths[b], lengths[b] + count)]
        starts.append(len(slots))
    return table, [n + c for n, c in zip(lengths, counts)], uses, slots, starts


def _exact_fork(case, table, lengths, uses):
    page, parents = case["page"], _fork_numbers(case)[1]
    uses = np.array(uses)
    rows, seen, wanting, copies = [], set(), [], []
    for row in table:
        np.subtract.at(uses, [p for p in row if p >= 0], 1)
    for i, b in enumerate(parents):
        rows.append(list(table[b]))
        named = [p for p in rows[i] if p >= 0]
        if b in seen and lengths[b] % page:
            wanting.append((i, lengths[b] // page))
            named.remove(rows[i][lengths[b] // page])
        seen.add(b)
        np.add.at(uses, named, 1)
    free = np.flatnonzero(uses == 0)
    for (i, j), p in zip(wanting, free.tolist()):
        copies.append((rows[i][j], p))
        rows[i][j] = p
        uses[p] = 1
    return (rows, [lengths[b] for b in parents], uses.tolist()), copies


def _exact_compact(table, uses):
    live = [p for p, n in enumerate(uses) if n]
    count, now, goes = len(live), [0] * len(uses), {}
    holes = iter([p for p in range(count) if uses[p] == 0])
    for p in live:
        goes[p] = p if p < count else next(holes)
        now[goes[p]] = uses[p]
    return ([[goes.get(p, p) for p in row] for row in table], now), [(p, to) for p, to in goes.items() if p != to]
