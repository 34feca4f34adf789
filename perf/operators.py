"""The paged-pool operators' calls that are timed: their inputs, one pass of
each in plain torch and through the package, the work a pass cannot do without,
and their results in 64 bits.

A pool of equal pages holds the keys and values of the sequences that a model
is answering.  Four operators work on it:

  tables   page_tables and slot_map: a step's pages placed, given back and
           refused, from the sequences' new lengths, and the new tokens' slots;
  write    cache_write: rows of keys and values to their slots;
  attend   tree_attention: drafted trees, single tokens or pieces of prompts
           against the pool;
  step     all of them, as a decoding step with drafts runs them.

Lengths are spread over a case's range (evenly in their logarithm) and dealt
out to the requests in an order that the seed makes, so that the work of a case
does not depend on the seed.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
E4M3 = torch.float8_e4m3fn
E4M3_MAX = 448.0
FREE, EVICTABLE, PINNED = 0, 1, 2


# ---------------------------------------------------------------------------
# The cases
# ---------------------------------------------------------------------------

def _tables(requests, page, lo, hi, grow, fresh, done, slack):
    return {"op": "tables", "requests": requests, "page": page, "lo": lo, "hi": hi, "grow": grow,
            "fresh": fresh, "done": done, "slack": slack}


def _write(tokens, heads, dim, dtype, cache, page, pages, skipped):
    return {"op": "write", "tokens": tokens, "kv_heads": heads, "dim": dim, "dtype": dtype,
            "cache": cache, "page": page, "pages": pages, "skipped": skipped}


def _attend(requests, lo, hi, t_lo, t_hi, tree, q_heads, kv_heads, dim, dtype, cache, page):
    return {"op": "attend", "requests": requests, "lo": lo, "hi": hi, "t_lo": t_lo, "t_hi": t_hi,
            "tree": tree, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype,
            "cache": cache, "page": page}


def _step(*a):
    return dict(_attend(*a), op="step")


def listed():
    cases = {
        # a few interactive sequences, each one token longer
        "tables_few": _tables(8, 16, 100, 2000, 1, 0.0, 0.0, 0.10),
        # a busy server's step: drafts accepted, prompts admitted, sequences done
        "tables_batch": _tables(512, 16, 64, 16000, 8, 0.05, 0.05, 0.10),
        # a pool that fills up while prompts queue: the last of them are refused
        "tables_full": _tables(4096, 16, 64, 16000, 4, 0.10, 0.05, -0.01),
        # the tokens of one decoding step of 64 sequences
        "write_step": _write(64, 8, 128, "bf16", "same", 16, 4096, 0),
        # prompts into a cache of 8-bit values, some tokens' slots not granted
        "write_prompts": _write(65536, 8, 128, "bf16", "e4m3", 16, 8192, 5),
        # one token each for four short conversations of a small model
        "attend_few": _attend(4, 100, 700, 1, 1, False, 16, 16, 64, "fp16", "same", 16),
        # one token each for a ragged batch
        "attend_tokens": _attend(64, 500, 16000, 1, 1, False, 32, 8, 128, "bf16", "same", 16),
        # one long document, a chain of eight drafted tokens
        "attend_long": _attend(1, 260001, 260001, 8, 8, False, 64, 8, 128, "fp16", "same", 64),
        # drafted trees of a batch
        "attend_trees": _attend(16, 1000, 8000, 64, 64, True, 32, 8, 128, "bf16", "same", 16),
        # drafted trees of all sizes over 8-bit keys and values
        "attend_trees_e4m3": _attend(48, 300, 12000, 1, 40, True, 32, 4, 128, "bf16", "e4m3", 32),
        # pieces of prompts, the first of them with nothing cached
        "attend_prompts": _attend(4, 0, 12000, 1000, 2048, False, 32, 8, 128, "bf16", "same", 16),
        # a whole decoding step with drafted trees
        "step_trees": _step(64, 200, 4000, 12, 12, True, 32, 8, 128, "bf16", "same", 16),
    }
    return [dict(c, name=name) for name, c in cases.items()]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tables", "tables", "write", "attend", "attend", "attend", "attend", "step"])
    page = rng.choice([8, 16, 16, 24, 32, 64, 128])
    if op == "tables":
        requests = _log(rng, 1, 4096)
        hi = min(_log(rng, 20, 64000), (1 << 26) // requests)
        return _tables(requests, page, max(1, hi // rng.choice([2, 20, 200])), max(2, hi),
                       rng.choice([1, 1, 4, 16]), rng.choice([0.0, 0.05, 0.15]),
                       rng.choice([0.0, 0.05, 0.3]), rng.choice([0.3, 0.05, 0.0, -0.02]))
    dim = rng.choice([64, 96, 128, 128, 128, 256])
    dtype, cache = rng.choice(["bf16", "bf16", "fp16"]), rng.choice(["same", "same", "e4m3"])
    kv_heads = rng.choice([1, 2, 4, 8, 8])
    if op == "write":
        tokens = min(_log(rng, 1, 1 << 16), (1 << 26) // (kv_heads * dim))
        pages = -(-tokens * rng.choice([2, 5]) // page) + rng.randrange(1, 50)
        return _write(tokens, kv_heads, dim, dtype, cache, page, pages, rng.choice([0, 0, 3, 7]))
    q_heads = kv_heads * rng.choice([1, 2, 4, 7, 8])
    requests, t_hi = _log(rng, 1, 256), 1
    kind = rng.choice(["token", "token", "tree", "tree", "chain", "prompt"])
    if op == "step":
        kind = rng.choice(["token", "tree"])
    if kind in ("tree", "chain"):
        t_hi = _log(rng, 2, 100)
    elif kind == "prompt":
        requests, t_hi = _log(rng, 1, 16), _log(rng, 64, 1500)
    # no more cached bytes, and no more products, than the largest listed cases
    hi = min(_log(rng, 16, 200000), (1 << 28) // (requests * kv_heads * dim))
    hi = max(1, min(hi, (1 << 35) // (requests * t_hi * q_heads * dim) - t_hi))
    lo = max(1, hi // rng.choice([1, 3, 30]))
    t_lo = max(1, t_hi // rng.choice([1, 2, 10]))
    make = _step if op == "step" else _attend
    return make(requests, lo, hi, t_lo, t_hi, kind == "tree", q_heads, kv_heads, dim, dtype,
                cache, page)


def _spread(lo, hi, n):
    """n whole numbers from lo to hi, evenly in their logarithm."""
    a, b = math.log(lo + 1 if n > 1 else hi + 1), math.log(hi + 1)
    return [int(round(math.exp(a + (b - a) * i / max(1, n - 1)))) - 1 for i in range(n)]


def _roles(case):
    """Cached and new lengths of a tables case, in the order before the seed's."""
    old, new = [], []
    for i, n in enumerate(_spread(case["lo"], case["hi"], case["requests"])):
        x = (i * 0.6180339887) % 1.0
        fresh, done = x < case["fresh"], x > 1.0 - case["done"]
        old.append(0 if fresh else max(n, 1))
        new.append(max(n, 1) if fresh else 0 if done else max(n, 1) + 1 + i % case["grow"])
    return old, new


def _pages(lengths, page):
    return sum(-(-n // page) for n in lengths)


def _tables_sizes(case):
    """Pages of the pool, columns of the table, new tokens."""
    old, new = _roles(case)
    page = case["page"]
    most = _pages([max(a, b) for a, b in zip(old, new)], page)
    pages = max(_pages(old, page) + 1, int(most * (1 + case["slack"])))
    pages += pages // 20  # other owners' pages
    cols = -(-max(max(old), max(new)) // page)
    return pages, cols, sum(max(0, b - a) for a, b in zip(old, new))


def _attend_sizes(case):
    """Cached lengths and new tokens of each request before the seed's order."""
    B = case["requests"]
    lens = _spread(case["lo"], case["hi"], B)
    trees = [case["t_lo"] + (case["t_hi"] - case["t_lo"]) * i // max(1, B - 1) for i in range(B)]
    if B > 1:
        trees = trees[B // 3:] + trees[:B // 3]
    return lens, trees


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _ints(values, dtype=torch.int64):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _offsets(counts):
    off = counts.new_zeros(counts.numel() + 1)
    off[1:] = torch.cumsum(counts, 0)
    return off


def _deal(gen, old, cols, page, pages, others):
    """Pages dealt out at random to sequences of the lengths `old`: the pool's
    kinds, the table and how many entries of each row are in use."""
    held = (old + page - 1) // page
    order = torch.randperm(pages, generator=gen, device="cuda")
    j = torch.arange(cols, device="cuda")[None]
    first = torch.cumsum(held, 0) - held
    at = (first[:, None] + j).clamp(max=pages - 1)
    table = torch.where(j < held[:, None], order[at], -1).to(torch.int32)
    used = int(held.sum())
    kind = torch.zeros(pages, dtype=torch.uint8, device="cuda")
    kind[order[:used]] = PINNED
    rest = order[used:used + others]
    kind[rest] = 1 + (torch.arange(rest.numel(), device="cuda") % 2).to(torch.uint8)
    return kind, table, held.to(torch.int32)


def _rows(gen, n, heads, dim, dtype):
    return torch.randn(n, heads, dim, generator=gen, device="cuda", dtype=dtype)


def _head_scales(gen, heads):
    """Scales with which about four standard deviations fill e4m3's range."""
    u = torch.rand(heads, generator=gen, device="cuda")
    return (0.8 + 0.4 * u) * (4.0 / E4M3_MAX)


def _cache(gen, case, pages):
    """The pool's keys and values, and the 8-bit types' scales."""
    shape, dtype = (pages, case["page"], case["kv_heads"], case["dim"]), DTYPES[case["dtype"]]
    kv, scales = [], []
    for _ in range(2):
        x = torch.randn(shape, generator=gen, device="cuda", dtype=dtype)
        if case["cache"] == "e4m3":
            s = _head_scales(gen, case["kv_heads"])
            x = (x.float() / s[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(E4M3)
            scales.append(s)
        kv.append(x)
    return kv, scales or [None, None]


def _parents(gen, off, n):
    """Trees as drafting grows them: each token's parent is one of the eight
    tokens before it, or it starts a branch of its own (-1)."""
    t = torch.arange(n, device="cuda")
    b = torch.searchsorted(off, t, right=True) - 1
    i = t - off[b]
    back = torch.floor(torch.rand(n, generator=gen, device="cuda") * 8).to(torch.int64)
    return (i - 1 - torch.minimum(back, i)).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case, "op": case["op"], "page": case["page"]}
    page = case["page"]
    if case["op"] == "tables":
        pages, cols, tokens = _tables_sizes(case)
        old, new = (_ints(x) for x in _roles(case))
        order = torch.randperm(old.numel(), generator=gen, device="cuda")
        old, new = old[order], new[order]
        s["kind"], s["table"], s["held"] = _deal(gen, old, cols, page, pages, pages // 21)
        s["lengths"], s["tokens"] = new, tokens
        s["offsets"] = _offsets((new - old).clamp(min=0))
        return s
    dtype = DTYPES[case["dtype"]]
    if case["op"] == "write":
        n, slots = case["tokens"], case["pages"] * page
        (s["k_cache"], s["v_cache"]), (s["k_scale"], s["v_scale"]) = _cache(gen, case, case["pages"])
        s["k"], s["v"] = (_rows(gen, n, case["kv_heads"], case["dim"], dtype) for _ in range(2))
        # whole pages at random places, in order inside a page
        order = torch.randperm(case["pages"], generator=gen, device="cuda")
        t = torch.arange(n, device="cuda")
        s["slots"] = order[t // page] * page + t % page
        if case["skipped"]:
            s["slots"][torch.randperm(n, generator=gen, device="cuda")[:n * case["skipped"] // 100]] = -1
        return s
    lens, trees = _attend_sizes(case)
    B, n = case["requests"], sum(trees)
    s["longest"], s["widest"], s["tokens"] = max(lens), max(trees), n
    order = torch.randperm(B, generator=gen, device="cuda")
    s["lengths"], counts = _ints(lens)[order], _ints(trees)[order]
    s["offsets"] = _offsets(counts)
    cols = max(1, -(-(max(lens) + max(trees)) // page))
    pages = _pages([a + b for a, b in zip(lens, trees)], page)
    pages += pages // 16 + 1
    s["kind"], s["table"], s["held"] = _deal(gen, s["lengths"], cols, page, pages, pages // 32)
    (s["k_cache"], s["v_cache"]), (s["k_scale"], s["v_scale"]) = _cache(gen, case, pages)
    s["q"] = 1.5 * _rows(gen, n, case["q_heads"], case["dim"], dtype)
    s["k"], s["v"] = (_rows(gen, n, case["kv_heads"], case["dim"], dtype) for _ in range(2))
    s["parents"] = _parents(gen, s["offsets"], n) if case["tree"] else None
    s["scale"] = case["dim"] ** -0.5
    if case["op"] == "step":
        # half of each tree's tokens are accepted (at least one), in their order
        taken = (counts + 1) // 2
        s["taken_offsets"] = _offsets(taken)
        s["taken"] = sum((t + 1) // 2 for t in trees)
        t = torch.arange(s["taken"], device="cuda")
        b = torch.searchsorted(s["taken_offsets"], t, right=True) - 1
        s["rows"] = s["offsets"][b] + 2 * (t - s["taken_offsets"][b])
        s["new_lengths"] = s["lengths"] + taken
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(s):
    if own:
        return _run_own(s)
    if s["op"] == "tables":
        return _plain_tables(s, s["lengths"], s["offsets"], s["tokens"])
    if s["op"] == "write":
        return _plain_write(s, s["k"], s["v"], s["slots"])
    out = _plain_attend(s)
    if s["op"] == "attend":
        return out
    placed = _plain_tables(s, s["new_lengths"], s["taken_offsets"], s["taken"])
    return [out, *placed, *_plain_write(s, s["k"][s["rows"]], s["v"][s["rows"]], placed[-1])]


def _run_own(s):
    import paper_2311_00591_amd as coop
    if s["op"] == "write":
        return coop.cache_write(s["k"], s["v"], s["slots"], s["k_cache"], s["v_cache"],
                                k_scale=s["k_scale"], v_scale=s["v_scale"])
    if s["op"] == "tables":
        return _own_tables(coop, s, s["lengths"], s["offsets"], s["tokens"])
    out = coop.tree_attention(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"],
                              s["lengths"], s["offsets"], s["parents"], scale=s["scale"],
                              k_scale=s["k_scale"], v_scale=s["v_scale"])
    if s["op"] == "attend":
        return out
    placed = _own_tables(coop, s, s["new_lengths"], s["taken_offsets"], s["taken"])
    return [out, *placed,
            *coop.cache_write(s["k"][s["rows"]], s["v"][s["rows"]], placed[-1], s["k_cache"],
                              s["v_cache"], k_scale=s["k_scale"], v_scale=s["v_scale"])]


def _own_tables(coop, s, lengths, offsets, tokens):
    table, held, kind, status, free = coop.page_tables(s["kind"], s["table"], s["held"], lengths,
                                                       s["page"])
    slots = coop.slot_map(table, held, lengths, offsets, tokens, s["page"], kind.numel())
    return [table, held, kind, status, free, slots]


def _plain_tables(s, lengths, offsets, tokens):
    kind, table, page = s["kind"].clone(), s["table"], s["page"]
    pages, (B, cols) = kind.numel(), table.shape
    held, j = s["held"].to(torch.int64), torch.arange(cols, device="cuda")[None]
    need = (lengths + page - 1) // page
    wide = need > cols
    need = torch.where(wide, held, need)
    # pages given back: the entries past what a sequence still needs (the one
    # place past the pool's end takes what is not given back)
    back = (j >= need[:, None]) & (j < held[:, None])
    grown = torch.cat([kind, kind.new_zeros(1)])
    grown[torch.where(back, table, pages).to(torch.int64)] = FREE
    kind = grown[:pages]
    # pages taken: the lowest free ones, in the requests' order
    count = (need - held).clamp(min=0)
    upto = torch.cumsum(count, 0)
    is_free = kind == FREE
    rank = torch.cumsum(is_free, 0)
    free = rank[-1]
    granted = (count == 0) | (upto <= free)
    now = torch.where(granted, need, held)
    by_rank = torch.full((pages + 1,), -1, dtype=torch.int64, device="cuda")
    by_rank[torch.where(is_free, rank - 1, pages)] = torch.arange(pages, device="cuda")
    new = (j >= held[:, None]) & (j < now[:, None])
    at = (upto - count)[:, None] + j - held[:, None]
    page_of = by_rank[torch.where(new, at, pages)]
    table = torch.where(new, page_of, torch.where(j < now[:, None], table, -1)).to(torch.int32)
    taken = torch.where(granted, count, 0).sum()
    kind = torch.where(is_free & (rank <= taken), PINNED, kind).to(torch.uint8)
    status = (~granted).any().to(torch.int32) + 2 * wide.any().to(torch.int32)
    # the new tokens' slots
    t = torch.arange(tokens, device="cuda")
    b = (torch.searchsorted(offsets, t, right=True) - 1).clamp(max=B - 1)
    pos = lengths[b] - offsets[b + 1] + t
    col = pos.clamp(min=0) // page
    at = table[b, col.clamp(max=cols - 1)].to(torch.int64)
    good = (pos >= 0) & (col < now[b]) & (t < offsets[B])
    slots = torch.where(good, at * page + pos % page, -1)
    return [table, now.to(torch.int32), kind, status.view(1), (free - taken).view(1), slots]


def _store(x, scale, dtype):
    if scale is None:
        return x
    return (x.float() / scale[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(dtype)


def _bytes(x):
    """8-bit numbers as bytes, which indexing takes."""
    return x.view(torch.uint8) if x.dtype == E4M3 else x


def _put(x, cache, scale, rows, slots):
    _bytes(cache).view(-1, *cache.shape[2:])[slots] = _bytes(_store(x[rows], scale, cache.dtype))
    return cache


def _plain_write(s, k, v, slots):
    rows = (slots >= 0).nonzero().squeeze(1)
    return [_put(k, s["k_cache"], s["k_scale"], rows, slots[rows]),
            _put(v, s["v_cache"], s["v_scale"], rows, slots[rows])]


def _cached(cache, scale, page, place):
    """The rows at (page, place) in 32 bits."""
    x = _bytes(cache)[page, place].view(cache.dtype).float()
    return x if scale is None else x * scale[:, None]


def _closure(reach, steps):
    """Ancestors within 2**steps generations, from those within one."""
    return reach if steps == 0 else _closure((reach @ reach).clamp(max=1.0), steps - 1)


def _plain_attend(s):
    case, off, lens, page = s["case"], s["offsets"], s["lengths"], s["page"]
    Hq, Hk, D, B = case["q_heads"], case["kv_heads"], case["dim"], case["requests"]
    L, T, G = s["longest"], s["widest"], Hq // Hk
    t, c = torch.arange(T, device="cuda"), torch.arange(L, device="cuda")
    here = t[None] < (off[1:] - off[:-1])[:, None]
    row = torch.where(here, off[:-1, None] + t[None], 0)
    pages = s["table"][:, c // page].clamp(min=0).to(torch.int64)
    keys, values = (
        torch.cat([_cached(cache, scale, pages, (c % page).expand(B, L)), new[row].float()], 1)
        .transpose(1, 2).contiguous()
        for cache, scale, new in ((s["k_cache"], s["k_scale"], s["k"]),
                                  (s["v_cache"], s["v_scale"], s["v"])))
    # which of its request's keys each token sees
    if s["parents"] is None:
        seen = (t[None, :] <= t[:, None]).expand(B, T, T)
    else:
        up = torch.where(here, s["parents"][row].to(torch.int64), -1)
        reach = ((up[:, :, None] == t) | (t[:, None] == t)).float()
        seen = _closure(reach, max(1, (T - 1).bit_length())) > 0
    seen = seen & here[:, None, :]
    seen = torch.cat([(c[None] < lens[:, None])[:, None].expand(B, T, L), seen], 2)
    q = s["q"][row].float().view(B, T, Hk, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hk, T * G, D)
    score = ((q @ keys.transpose(2, 3)) * s["scale"]).view(B, Hk, T, G, L + T)
    score = score.masked_fill(~seen[:, None, :, None], -math.inf)
    p = torch.exp(score - score.amax(-1, keepdim=True).clamp(min=-1e30))
    total = p.sum(-1, keepdim=True)
    p = (p / total.clamp(min=1e-30)).view(B, Hk, T * G, L + T)
    out = (p @ values).view(B, Hk, T, G, D).permute(0, 2, 1, 3, 4).reshape(B, T, Hq, D)
    flat = torch.arange(s["tokens"], device="cuda")
    b = torch.searchsorted(off, flat, right=True) - 1
    return out[b, flat - off[b]].to(s["q"].dtype)


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def _tables_work(pages, cols, B, tokens):
    # kinds and rows in and out, lengths and counts in, counts out, offsets in, slots out
    return {"bytes": 2 * pages + 8 * B * cols + 16 * B + 12 + 8 * (B + 1) + 8 * tokens,
            "flops": pages + B * cols + tokens}


def _write_work(case, tokens, written):
    row = 2 * case["kv_heads"] * case["dim"]
    e4m3 = case["cache"] == "e4m3"
    return {"bytes": 8 * tokens + written * row * (2 + (1 if e4m3 else 2)),
            "flops": written * row if e4m3 else 0}


def work(case):
    if case["op"] == "tables":
        pages, cols, tokens = _tables_sizes(case)
        return _tables_work(pages, cols, case["requests"], tokens)
    if case["op"] == "write":
        n = case["tokens"]
        return _write_work(case, n, n - n * case["skipped"] // 100)
    lens, trees = _attend_sizes(case)
    n, row = sum(trees), case["kv_heads"] * case["dim"]
    qrow = case["q_heads"] * case["dim"]
    size = 1 if case["cache"] == "e4m3" else 2
    # cached and new keys and values, queries and outputs, table entries,
    # lengths and offsets; a tree's pairs are counted as a chain's only where
    # it is one
    moved = sum(lens) * 2 * row * size + n * 2 * row * 2 + 2 * n * qrow * 2
    moved += 4 * _pages(lens, case["page"]) + 16 * case["requests"] + (4 * n if case["tree"] else 0)
    # (order is the seed's, but the same for lengths and trees)
    pairs = sum(a * t + (t if case["tree"] else t * (t + 1) // 2) for a, t in zip(lens, trees))
    w = {"bytes": moved, "flops": 4 * qrow * pairs}
    if case["op"] == "step":
        taken = sum((t + 1) // 2 for t in trees)
        cols = max(1, -(-(max(lens) + max(trees)) // case["page"]))
        pages = _pages([a + b for a, b in zip(lens, trees)], case["page"])
        pages += pages // 16 + 1
        for more in (_tables_work(pages, cols, case["requests"], taken),
                     _write_work(case, taken, taken)):
            w = {k: w[k] + more[k] for k in w}
    return w


# ---------------------------------------------------------------------------
# The same in 64 bits, request by request
# ---------------------------------------------------------------------------

def _nearest_e4m3(x):
    """The nearest multiple of e4m3's step at x (ties to even), at most 448."""
    x = x.clamp(-E4M3_MAX, E4M3_MAX)
    exponent = torch.frexp(x)[1] - 1
    step = torch.exp2((exponent.clamp(min=-6) - 3).to(torch.float64))
    return torch.round(x / step) * step


def _exact_write(s, k, v, slots):
    out = []
    for x, cache, scale in ((k, s["k_cache"], s["k_scale"]), (v, s["v_cache"], s["v_scale"])):
        rows = cache.to(torch.float64).view(-1, *cache.shape[2:])
        good, x = slots >= 0, x.to(torch.float64)
        if scale is not None:
            x = _nearest_e4m3(x / scale.to(torch.float64)[:, None])
        rows[slots[good]] = x[good]
        out.append(rows.view(cache.shape))
    return out


def _exact_slots(s):
    """A step's slots, one request after the other (none gives pages back)."""
    page, first = s["page"], s["taken_offsets"].tolist()
    free = [p for p, k in enumerate(s["kind"].tolist()) if k == FREE]
    held, table = s["held"].tolist(), s["table"].tolist()
    slots = []
    for b, n in enumerate(s["new_lengths"].tolist()):
        row = table[b][:held[b]]
        more = -(-n // page) - held[b]
        if more <= len(free):
            row, free = row + free[:more], free[more:]
        else:
            free = []
        for pos in range(n - (first[b + 1] - first[b]), n):
            slots.append(row[pos // page] * page + pos % page if pos // page < len(row) else -1)
    return _ints(slots)


def _exact_attend(s):
    case, page = s["case"], s["page"]
    Hq, Hk, D = case["q_heads"], case["kv_heads"], case["dim"]
    G = Hq // Hk
    off, lens, table = s["offsets"].tolist(), s["lengths"].tolist(), s["table"].tolist()
    parents = s["parents"].tolist() if s["parents"] is not None else None
    out = torch.empty(s["tokens"], Hq, D, dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        lo, hi = off[b], off[b + 1]
        T = hi - lo
        used = table[b][:-(-n // page)]
        kv = []
        for cache, scale, new in ((s["k_cache"], s["k_scale"], s["k"]),
                                  (s["v_cache"], s["v_scale"], s["v"])):
            old = [cache[p:p + 1] for p in used]
            if old:
                old = torch.cat([x.view(torch.uint8) if scale is not None else x for x in old])
                old = old.view(cache.dtype).to(torch.float64).reshape(-1, Hk, D)[:n]
                old = old if scale is None else old * scale.to(torch.float64)[:, None]
                kv.append(torch.cat([old, new[lo:hi].to(torch.float64)]))
            else:
                kv.append(new[lo:hi].to(torch.float64))
        hidden = torch.ones(T, T, dtype=torch.bool)
        for i in range(T):
            if parents is None:
                hidden[i, :i + 1] = False
            else:
                j = i
                while j >= 0:
                    hidden[i, j] = False
                    j = parents[lo + j]
        hidden = hidden.cuda()
        for h in range(Hq):
            key, value = kv[0][:, h // G], kv[1][:, h // G]
            x = s["q"][lo:hi, h].to(torch.float64) @ key.t() * s["scale"]
            x[:, n:][hidden] = -math.inf
            out[lo:hi, h] = torch.softmax(x, -1) @ value
    return out


def exact(case, seed):
    if case["op"] == "tables":
        return None  # whole numbers
    s = prepare(case, seed)
    if case["op"] == "write":
        return _exact_write(s, s["k"], s["v"], s["slots"])
    out = _exact_attend(s)
    if case["op"] == "attend":
        return out
    return [out, None, None, None, None, None, None,
            *_exact_write(s, s["k"][s["rows"]], s["v"][s["rows"]], _exact_slots(s))]
