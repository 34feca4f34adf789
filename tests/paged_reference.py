"""The paged-pool operators from their definitions: whole numbers one request
after the other, attention one token and head at a time in 64 bits.  Shares
nothing with the package."""
import numpy as np
import torch

E4M3_MAX = 448.0


def page_tables(kind, table, held, lengths, page_size, taken=2):
    """(table, held, kind, status, free) as numpy arrays."""
    kind, table = np.asarray(kind).astype(np.uint8), np.asarray(table).astype(np.int32)
    rows, cols = table.shape
    held = [min(max(int(h), 0), cols) for h in held]
    need = [-(-(int(n) % 2**64) // page_size) for n in lengths]
    status = 2 if any(n > cols for n in need) else 0
    for b in range(rows):
        if need[b] <= cols and need[b] < held[b]:
            for p in table[b, need[b]:held[b]]:
                if 0 <= p < len(kind):
                    kind[p] = 0
            held[b] = need[b]
    free = [p for p in range(len(kind)) if kind[p] == 0]
    full = False
    for b in range(rows):
        if need[b] > cols or need[b] <= held[b]:
            continue
        more = need[b] - held[b]
        full = full or more > len(free)
        if full:
            status |= 1
            continue
        table[b, held[b]:need[b]] = free[:more]
        kind[free[:more]] = taken
        free, held[b] = free[more:], need[b]
    for b in range(rows):
        table[b, held[b]:] = -1
    return table, np.array(held, dtype=np.int32), kind, status, len(free)


def slot_map(table, held, lengths, offsets, num_tokens, page_size, num_pages):
    rows, cols = table.shape
    out = np.full(num_tokens, -1, dtype=np.int64)
    for b in range(rows):
        n = int(offsets[b + 1]) - int(offsets[b])
        for i in range(n):
            pos = int(lengths[b]) - n + i
            if pos < 0:
                continue
            c = pos // page_size
            if c < min(max(int(held[b]), 0), cols) and 0 <= table[b, c] < num_pages:
                out[int(offsets[b]) + i] = int(table[b, c]) * page_size + pos % page_size
    return out


def e4m3_values():
    """Every finite e4m3 number, from its bits."""
    v = []
    for bits in range(256):
        e, m = (bits >> 3) & 15, bits & 7
        if e == 15 and m == 7:
            continue
        x = m * 2.0**-9 if e == 0 else (8 + m) * 2.0**(e - 10)
        v.append((-1) ** (bits >> 7) * x)
    return np.array(sorted(set(v)))


def seen(parents, i):
    """The tokens that token i of a tree sees, None if it is void."""
    if parents is None:
        return list(range(i + 1))
    void = lambda j: not (parents[j] == -1 or 0 <= parents[j] < j)
    if void(i):
        return None
    out = [i]
    while parents[out[-1]] >= 0 and not void(parents[out[-1]]):
        out.append(parents[out[-1]])
    return out


def attention(q, k, v, k_cache, v_cache, table, lengths, offsets, parents, scale, k_scale=None,
              v_scale=None, only=None):
    """out, and how far a result of q's type may be from it, both [tokens,
    q_heads, dim] in 64 bits; rows of no request are NaN, and so are tokens not
    in `only` (request-local numbers) where it is given.

    With u = eps / 2 of the type (half a step, relative) and w the exact
    weights, A = sum_j w_j |v_j|:
      the result's own rounding                            u |out|
      the weights' rounding before the products            u A
      a score's error d changes its weight by e^d - 1, and the sum that
      divides by as much: 2 d A, d = 2^-24 ((dim + 4) S + 4 |s|) with S the sum
      of |q_i k_i| scale over a row of at most dim terms (each 32-bit addition
      is off by 2^-24 of the partial sum), |s| for e^s by way of 2^x
      32-bit sums over n tokens: 2 n 2^-24 A, and as many roundings again when
      a running maximum changes, at most once for each 16 tokens
      e^x itself: 2^-21
    16-bit floats below 2^-14 have a fixed step of 2^-24 (weights are at most
    one before the division, and one of them is one): 2^-25 sum_j |v_j| and
    2^-25; numbers of bfloat16 and e4m3 are not that small here."""
    dtype = q.dtype
    u = torch.finfo(dtype).eps / 2
    f64 = lambda t: t.to(torch.float64).cpu().numpy()
    q, k, v = f64(q), f64(k), f64(v)
    kc, vc = f64(k_cache.float()), f64(v_cache.float())
    if k_scale is not None:
        kc, vc = kc * f64(k_scale)[:, None], vc * f64(v_scale)[:, None]
    pages, page = kc.shape[:2]
    table, lengths, offsets = (t.cpu().numpy() for t in (table, lengths, offsets))
    parents = parents.cpu().numpy() if parents is not None else None
    n, hq, dim = q.shape
    group = hq // k.shape[1]
    out, tol = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    for b in range(len(lengths)):
        lo, hi = int(offsets[b]), int(offsets[b + 1])
        count = min(int(lengths[b]), table.shape[1] * page)
        at = [(int(table[b, j // page]), j % page) for j in range(count)]
        at = [(p, o) for p, o in at if 0 <= p < pages]
        p, o = [x[0] for x in at], [x[1] for x in at]
        own = None if parents is None else parents[lo:hi].tolist()
        for i in range(hi - lo) if only is None else only:
            tokens = seen(own, i)
            if tokens is None:
                out[lo + i] = tol[lo + i] = 0
                continue
            rows = [lo + j for j in tokens]
            for h in range(hq):
                g = h // group
                key = np.concatenate([kc[p, o, g], k[rows, g]]) if p else k[rows, g]
                val = np.concatenate([vc[p, o, g], v[rows, g]]) if p else v[rows, g]
                with np.errstate(all="ignore"):
                    s = key @ q[lo + i, h] * scale
                    w = np.exp(s - s.max())
                    total = w.sum()
                    w /= total
                    out[lo + i, h] = w @ val
                    a = w @ np.abs(val)
                    d = 2.0**-24 * ((dim + 4) * abs(scale) * (np.abs(key) @ np.abs(q[lo + i, h])).max()
                                    + 4 * np.abs(s).max())
                    t = u * np.abs(out[lo + i, h]) + (u + 2 * d + 2.25 * len(s) * 2.0**-24 + 2.0**-21) * a
                    if dtype == torch.float16:
                        t += 2.0**-25 * (np.abs(val).sum(0) / total + 1)
                    tol[lo + i, h] = t
    return out, tol
