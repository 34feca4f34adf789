"""The paged-pool operators on the GPU against their plain reference."""
import sys

import numpy as np
import pytest

import paged_reference as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16, FP16, E4M3 = torch.bfloat16, torch.float16, torch.float8_e4m3fn
DEV = "cuda"


def _coop():
    import paper_2311_00591_amd as coop
    return coop


def _announce(label):
    print(f"[gpu case] paged: {label}", flush=True)
    sys.stdout.flush()


def _ints(a, dtype=torch.int64):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV, dtype)


# ---------------------------------------------------------------------------
# Block tables and slot maps
# ---------------------------------------------------------------------------

def _random_tables(rng, pages, rows, cols, page, free=0.6, tight=1.0):
    """Rows that hold some of the pages that are not free, and new lengths
    that ask for about `tight` times the free ones."""
    kind = (rng.random(pages) > free).astype(np.uint8) * 2
    busy = rng.permutation(np.flatnonzero(kind))
    held = np.zeros(rows, dtype=np.int64)
    table = np.full((rows, cols), -1, dtype=np.int32)
    for b in range(rows):
        h = int(min(rng.integers(0, cols + 1), len(busy)))
        h = h if rng.random() < 0.8 else 0
        table[b, :h], busy, held[b] = busy[:h], busy[h:], h
    kind[rng.permutation(busy)[:len(busy) // 2]] = 1
    most = max(1.0, tight * 2 * (kind == 0).sum() / max(rows, 1))
    lengths = np.where(rng.random(rows) < 0.3, (held * rng.random(rows)).astype(np.int64),
                       np.minimum(held + (most * rng.random(rows)).astype(np.int64), cols)) * page
    lengths = np.maximum(lengths - rng.integers(0, page, rows), 0)
    lengths[rng.random(rows) < 0.05] = cols * page + 1  # more than a row can list
    return kind, table, held, lengths


def _check_tables(got, want):
    table, held, kind, status, free = got
    assert np.array_equal(held.cpu().numpy(), want[1])
    assert np.array_equal(table.cpu().numpy(), want[0])
    assert np.array_equal(kind.cpu().numpy(), want[2])
    assert (status.item(), free.item()) == want[3:]


@pytest.mark.parametrize("pages, rows, cols, page, free, tight", [
    (1, 1, 1, 1, 1.0, 1.0), (64, 1, 70, 16, 0.5, 2.0), (63, 5, 1, 16, 0.5, 0.5),
    (1000, 7, 130, 16, 0.6, 0.4), (4096, 64, 33, 7, 0.3, 1.5), (4097, 300, 20, 16, 0.9, 0.5),
    (20000, 1500, 9, 128, 0.5, 1.1), (131072, 512, 60, 16, 0.6, 0.9), (131072, 513, 60, 16, 0.6, 0.9), (131073, 9, 800, 16, 0.2, 1.0),
    (5000, 1000, 40, 48, 0.95, 0.1), (70000, 40, 2500, 16, 0.7, 0.7),
    (300001, 1025, 400, 1, 0.8, 0.9)])
def test_page_tables(pages, rows, cols, page, free, tight):
    coop = _coop()
    _announce(f"tables {pages} pages, {rows} x {cols}, page {page}")
    rng = np.random.default_rng(pages + rows)
    for taken in (1, 2):
        kind, table, held, lengths = _random_tables(rng, pages, rows, cols, page, free, tight)
        want = ref.page_tables(kind, table, held, lengths, page, taken)
        given = [_ints(kind, torch.uint8), _ints(table, torch.int32), _ints(held, torch.int32),
                 _ints(lengths)]
        before = [t.clone() for t in given]
        _check_tables(coop.page_tables(*given, page, taken=taken), want)
        assert all(torch.equal(x, y) for x, y in zip(given, before))
        # in place, and one of the three only
        k, t, h, n = (x.clone() for x in given)
        _check_tables(coop.page_tables(k, t, h, n, page, taken=taken, out=(t, h, k)), want)
        assert torch.equal(n, given[3])
        k, t, h, n = (x.clone() for x in given)
        out = (torch.full_like(t, 99), h, torch.full_like(k, 7))
        _check_tables(coop.page_tables(k, t, h, n, page, taken=taken, out=out), want)
        assert torch.equal(k, given[0]) and torch.equal(t, given[1])


def test_page_tables_edges():
    coop = _coop()
    _announce("tables, edges")
    i32 = dict(dtype=torch.int32, device=DEV)
    u8 = dict(dtype=torch.uint8, device=DEV)
    i64 = dict(dtype=torch.int64, device=DEV)
    # no requests; no pages; no columns
    got = coop.page_tables(torch.tensor([0, 1, 0], **u8), torch.zeros((0, 3), **i32),
                           torch.zeros(0, **i32), torch.zeros(0, **i64), 16)
    assert got[2].tolist() == [0, 1, 0] and (got[3].item(), got[4].item()) == (0, 2)
    got = coop.page_tables(torch.zeros(0, **u8), torch.full((2, 3), -1, **i32),
                           torch.zeros(2, **i32), torch.tensor([0, 5], **i64), 16)
    assert got[1].tolist() == [0, 0] and (got[3].item(), got[4].item()) == (1, 0)
    got = coop.page_tables(torch.zeros(4, **u8), torch.zeros((2, 0), **i32), torch.zeros(2, **i32),
                           torch.tensor([0, 5], **i64), 16)
    assert got[1].tolist() == [0, 0] and (got[3].item(), got[4].item()) == (2, 4)
    # pages out of range are not given back; counts out of range are limited; a
    # length with its top bit set is a long one
    kind = torch.tensor([2, 2, 0, 2], **u8)
    table = torch.tensor([[7, 1, -3], [3, 3, 0], [0, -1, -1]], **i32)
    held = torch.tensor([9, 3, -2], **i32)
    got = coop.page_tables(kind, table, held, torch.tensor([0, 1, -1], **i64), 4)
    want = ref.page_tables(kind.tolist(), table.tolist(), held.tolist(), [0, 1, -1], 4)
    _check_tables(got, want)
    assert got[2].tolist() == [0, 0, 0, 0] and got[3].item() == 2


@pytest.mark.parametrize("rows, cols, page, most", [
    (1, 1, 1, 1), (3, 40, 16, 20), (70, 9, 7, 30), (500, 60, 128, 700), (5000, 3, 16, 3)])
def test_slot_map(rows, cols, page, most):
    coop = _coop()
    _announce(f"slots {rows} x {cols}, page {page}")
    rng = np.random.default_rng(rows * cols)
    pages = 2 * cols + 5
    table = rng.integers(0, pages, (rows, cols)).astype(np.int32)
    table[rng.random((rows, cols)) < 0.02] = -1
    table[rng.random((rows, cols)) < 0.02] = pages
    held = rng.integers(-1, cols + 2, rows)
    lengths = rng.integers(0, cols * page + 2, rows)
    count = np.where(rng.random(rows) < 0.3, 0, rng.integers(0, most + 1, rows))
    offsets = np.concatenate([[0], np.cumsum(count)])
    for n in (int(offsets[-1]), int(offsets[-1]) + 300):  # a padded batch
        want = ref.slot_map(table, held, lengths, offsets, n, page, pages)
        got = coop.slot_map(_ints(table, torch.int32), _ints(held, torch.int32), _ints(lengths),
                            _ints(offsets), n, page, pages)
        assert np.array_equal(got.cpu().numpy(), want)


# ---------------------------------------------------------------------------
# Cache writes
# ---------------------------------------------------------------------------

def _pool(rng, pages, page, heads, dim, dtype, order="pages", scales=False):
    """A pool of random numbers as [pages, page, heads, dim]: contiguous, heads
    outside places, or keys and values side by side."""
    g = torch.Generator().manual_seed(int(rng.integers(1 << 30)))
    shape = (pages, page, heads, dim)
    x = [torch.randn(shape, generator=g) for _ in range(2)]
    s = [None, None]
    if dtype == E4M3:
        s = [torch.rand(heads, generator=g) * 0.02 + 0.005 for _ in range(2)]
        x = [(a / b[:, None]).clamp(-448, 448) for a, b in zip(x, s)]
        s = [b.to(DEV) for b in s]
    x = [a.to(dtype).to(DEV) for a in x]
    raw = [a.view(torch.uint8) if dtype == E4M3 else a for a in x]
    if order == "heads":
        raw = [a.transpose(1, 2).contiguous().transpose(1, 2) for a in raw]
    elif order == "pairs":
        both = torch.stack(raw, 2).contiguous()
        raw = [both[:, :, 0], both[:, :, 1]]
    return [a.view(dtype) for a in raw], s


@pytest.mark.parametrize("dtype, cache", [(BF16, BF16), (FP16, FP16), (BF16, E4M3), (FP16, E4M3)])
@pytest.mark.parametrize("tokens, pages, page, heads, dim, order", [
    (1, 1, 1, 1, 64, "pages"), (37, 9, 7, 3, 80, "heads"), (300, 40, 16, 8, 128, "pairs"),
    (5000, 300, 32, 2, 256, "pages"), (65, 100, 1, 5, 16, "heads")])
def test_cache_write(dtype, cache, tokens, pages, page, heads, dim, order):
    coop = _coop()
    _announce(f"write {tokens} tokens, {heads} x {dim}, {dtype} to {cache}, {order}")
    rng = np.random.default_rng(tokens + dim)
    (kc, vc), (ks, vs) = _pool(rng, pages, page, heads, dim, cache, order)
    slots = rng.permutation(pages * page)[:tokens]
    slots = np.concatenate([slots, np.full(tokens - len(slots), -1)])
    slots[rng.random(tokens) < 0.1] = -1
    slots[rng.random(tokens) < 0.05] = pages * page
    # rows of a fused projection: strided, not contiguous
    fused = torch.from_numpy(rng.standard_normal((tokens, 3 * heads, dim))).to(DEV, dtype)
    k, v = fused[:, heads:2 * heads], fused[:, 2 * heads:]
    before = [a.clone() for a in (kc, vc)]
    got = coop.cache_write(k, v, _ints(slots), kc, vc, k_scale=ks, v_scale=vs)
    assert got[0] is kc and got[1] is vc
    good = np.flatnonzero((slots >= 0) & (slots < pages * page))
    for new, old, x, s in ((kc, before[0], k, ks), (vc, before[1], v, vs)):
        want = old.float().cpu().reshape(-1, heads, dim).clone()
        rows = x.float().cpu()[good]
        if cache == E4M3:
            rows = (rows / s.cpu()[:, None]).clamp(-448, 448).to(E4M3).float()
        want[slots[good]] = rows
        assert torch.equal(new.float().cpu().reshape(-1, heads, dim), want)


def test_cache_write_rounds_to_the_nearest_of_all_e4m3_numbers():
    coop = _coop()
    _announce("write, every step of e4m3")
    v = ref.e4m3_values()
    mid = (v[1:] + v[:-1]) / 2
    x = np.concatenate([v, mid, np.nextafter(mid.astype(np.float16), np.float16(np.inf)),
                        np.nextafter(mid.astype(np.float16), np.float16(-np.inf)), [449, 6e4, -6e4],
                        [0.0, -0.0, np.inf, -np.inf]])
    x = np.concatenate([x, np.zeros(-len(x) % 16)])
    x = torch.from_numpy(x).to(FP16).view(1, -1, 16)
    heads = x.shape[1]
    kc, vc = (torch.zeros((1, 1, heads, 16), dtype=torch.uint8, device=DEV).view(E4M3) for _ in "kv")
    one, two = torch.ones(heads, device=DEV), torch.full((heads,), 0.5, device=DEV)
    coop.cache_write(x.to(DEV), x.to(DEV), _ints([0]), kc, vc, k_scale=one, v_scale=two)
    for cache, scale in ((kc, 1.0), (vc, 0.5)):
        want = np.clip(x.double().numpy().ravel() / scale, -448, 448)
        got = cache.float().cpu().numpy().ravel().astype(np.float64)
        dist = np.abs(v[None] - want[:, None])
        assert np.array_equal(np.abs(got - want), dist.min(1))
        # ties go to the even one, whose last bit is zero
        bits = cache.view(torch.uint8).cpu().numpy().ravel()
        tie = (dist == dist.min(1, keepdims=True)).sum(1) > 1
        assert tie.sum() > 100 and not (bits[tie] & 1).any()
    nan = torch.full((1, 1, 16), float("nan"), dtype=BF16, device=DEV)
    kc, vc = (torch.zeros((1, 1, 1, 16), dtype=torch.uint8, device=DEV).view(E4M3) for _ in "kv")
    coop.cache_write(nan, nan, _ints([0]), kc, vc, k_scale=one[:1], v_scale=one[:1])
    assert kc.float().isnan().all() and vc.float().isnan().all()


# ---------------------------------------------------------------------------
# Attention
# ---------------------------------------------------------------------------

def _trees(rng, counts, kind):
    """parents of all tokens: None, a chain written out, random trees, or
    trees with void tokens."""
    if kind is None:
        return None
    out = []
    for n in counts:
        i = np.arange(n)
        if kind == "chain":
            p = i - 1
        else:
            p = i - 1 - np.minimum((rng.random(n) * 6).astype(np.int64), i)
            if kind == "void":
                bad = rng.random(n) < 0.2
                p = np.where(bad, rng.choice([-2, 5000, -2**31, 2**31 - 1], n), p)
                p[n // 2:n // 2 + 1] = n // 2  # its own parent
        out.append(p)
    return _ints(np.concatenate(out) if out else np.zeros(0), torch.int32)


def _attention_inputs(seed, lengths, counts, q_heads, heads, dim, dtype, cache, page, tree,
                      order="pages", padding=0, cols=None, spread=1.0):
    rng = np.random.default_rng(seed)
    held = [-(-n // page) for n in lengths]
    pages = sum(held) + 3
    cols = cols or max(held + [1]) + 1
    (kc, vc), (ks, vs) = _pool(rng, pages, page, heads, dim, cache, order)
    perm = rng.permutation(pages)
    table = np.full((len(lengths), cols), -1, dtype=np.int32)
    for b, h in enumerate(held):
        table[b, :h], perm = perm[:h], perm[h:]
    n = sum(counts) + padding
    fused = torch.from_numpy(rng.standard_normal((n, q_heads + 2 * heads, dim)) * spread).to(DEV, dtype)
    parents = _trees(rng, counts, tree)
    if parents is not None and padding:
        parents = torch.cat([parents, parents.new_full((padding,), -1)])
    return dict(q=fused[:, :q_heads], k=fused[:, q_heads:q_heads + heads],
                v=fused[:, q_heads + heads:], k_cache=kc, v_cache=vc, table=_ints(table, torch.int32),
                lengths=_ints(lengths), token_offsets=_ints(np.concatenate([[0], np.cumsum(counts)])),
                parents=parents, k_scale=ks, v_scale=vs)


def _check_attention(a, got, scale=None):
    scale = a["q"].shape[2] ** -0.5 if scale is None else scale
    want, tol = ref.attention(a["q"], a["k"], a["v"], a["k_cache"], a["v_cache"], a["table"],
                              a["lengths"], a["token_offsets"], a["parents"], scale, a["k_scale"],
                              a["v_scale"])
    used = int(a["token_offsets"][-1])
    got = got.double().cpu().numpy()[:used]
    want, tol = want[:used], tol[:used]
    assert np.array_equal(np.isnan(got), np.isnan(want))
    fine = ~np.isnan(want)
    off = np.abs(got - want)[fine]
    worst = (off / np.maximum(tol[fine], 1e-300)).max() if off.size else 0.0
    print(f"  worst error {worst:.3f} of what rounding allows", flush=True)
    assert (off <= tol[fine]).all(), worst


CASES = [
    # lengths, counts, q_heads, heads, dim, page
    ([1], [1], 1, 1, 64, 16), ([0], [1], 4, 4, 64, 16), ([0, 5, 0], [0, 1, 3], 6, 2, 128, 16),
    ([15, 16, 17, 63, 64, 65], [1] * 6, 8, 1, 128, 16), ([1000, 3, 300], [1, 1, 1], 32, 8, 128, 16),
    ([130, 0, 517], [9, 17, 64], 8, 2, 128, 16), ([257, 31], [1, 40], 6, 6, 96, 7),
    ([700, 20], [65, 3], 14, 2, 64, 32), ([333], [130], 4, 2, 256, 64), ([90, 91], [2, 31], 4, 1, 80, 1),
    ([2100], [3], 5, 1, 112, 1000), ([40] * 70, [1 + i % 3 for i in range(70)], 4, 2, 64, 8)]


@pytest.mark.parametrize("dtype, cache", [(BF16, BF16), (FP16, FP16), (BF16, E4M3), (FP16, E4M3)])
@pytest.mark.parametrize("tree", [None, "tree", "void"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_tree_attention(case, tree, dtype, cache):
    coop = _coop()
    lengths, counts, q_heads, heads, dim, page = CASES[case]
    order = ("pages", "heads", "pairs")[case % 3]
    _announce(f"attention {lengths[:6]} + {counts[:6]}, {q_heads}/{heads} x {dim}, {dtype} {cache}, "
              f"{tree}, {order}")
    a = _attention_inputs(case, lengths, counts, q_heads, heads, dim, dtype, cache, page, tree, order,
                          padding=3 if case % 2 else 0)
    n = a["q"].shape[0]
    out = torch.full((n, q_heads, dim), 7.0, dtype=dtype, device=DEV)
    got = coop.tree_attention(**a, out=out)
    assert got is out
    _check_attention(a, got)
    assert (got[sum(counts):] == 7).all()  # rows of no request


@pytest.mark.parametrize("dim", [8, 24, 40, 72, 104, 136, 192, 200, 248])
def test_tree_attention_head_sizes(dim):
    coop = _coop()
    _announce(f"attention, heads of {dim}")
    for counts, dtype in (([1, 1], BF16), ([7, 33], FP16)):
        a = _attention_inputs(dim, [77, 200], counts, 4, 2, dim, dtype, dtype, 16, "tree")
        _check_attention(a, coop.tree_attention(**a))


@pytest.mark.parametrize("counts, q_heads, heads", [
    ([1], 64, 2), ([1, 2], 48, 3), ([5], 71, 1), ([16], 16, 16), ([200], 3, 1), ([1] * 33, 16, 1)])
def test_tree_attention_head_sharing(counts, q_heads, heads):
    coop = _coop()
    _announce(f"attention, {q_heads} query heads on {heads}, {counts[:3]}")
    a = _attention_inputs(q_heads, [150] * len(counts), counts, q_heads, heads, 64, BF16, BF16, 16,
                          "tree")
    _check_attention(a, coop.tree_attention(**a, scale=0.3), 0.3)


@pytest.mark.parametrize("lengths, counts, q_heads, heads, dim, page", [
    ([90, 0, 300, 70], [150, 3, 201, 61], 4, 2, 128, 16), ([64, 1], [130, 111], 2, 1, 104, 7),
    ([1100], [129], 2, 1, 128, 24), ([20, 40] * 35, [12 + i % 20 for i in range(70)], 8, 1, 128, 16),
    ([0, 500], [700, 530], 1, 1, 120, 64)])
@pytest.mark.parametrize("tree", [None, "tree", "void"])
@pytest.mark.parametrize("dtype, cache", [(BF16, BF16), (FP16, FP16), (BF16, E4M3)])
def test_tree_attention_many_rows(lengths, counts, q_heads, heads, dim, page, tree, dtype, cache):
    coop = _coop()
    dim += 8 if cache == E4M3 and dim % 16 else 0  # (rows start at multiples of 16 bytes)
    _announce(f"attention, many rows: {lengths[:4]} + {counts[:4]}, {dtype} {cache}, {tree}")
    a = _attention_inputs(dim, lengths, counts, q_heads, heads, dim, dtype, cache, page, tree,
                          padding=5)
    out = torch.full((sum(counts) + 5, q_heads, dim), 7.0, dtype=dtype, device=DEV)
    _check_attention(a, coop.tree_attention(**a, out=out))
    assert (out[sum(counts):] == 7).all()


@pytest.mark.parametrize("lengths, counts, heads, page", [
    ([20000], [1], 1, 16), ([9000, 12], [2, 2], 2, 24), ([5000, 0, 1, 4000], [33, 1, 70, 5], 1, 64)])
@pytest.mark.parametrize("dtype, cache", [(BF16, BF16), (FP16, E4M3)])
def test_tree_attention_long(lengths, counts, heads, page, dtype, cache):
    coop = _coop()
    _announce(f"attention, long: {lengths} + {counts}")
    a = _attention_inputs(5, lengths, counts, 2 * heads, heads, 128, dtype, cache, page, "tree")
    _check_attention(a, coop.tree_attention(**a))


@pytest.mark.parametrize("requests, longest, width, q_heads, heads", [
    (64, 9000, 1, 32, 8), (8, 5000, 40, 16, 4), (100, 2000, 3, 8, 8), (3, 3500, 700, 8, 2),
    (70, 900, 100, 16, 4)])
def test_tree_attention_fills_the_device(requests, longest, width, q_heads, heads):
    """Many workgroups at once: every run gives the same bits, and rows picked
    at random are right."""
    coop = _coop()
    _announce(f"attention, {requests} requests up to {longest} + {width}")
    rng = np.random.default_rng(requests)
    lengths = rng.integers(1, longest, requests).tolist()
    counts = rng.integers(1, width + 1, requests).tolist()
    dim, page = 128, 16
    a = _attention_inputs(requests, lengths, counts, q_heads, heads, dim, BF16, BF16, page,
                          "tree" if width < 100 else None)
    got = coop.tree_attention(**a)
    for _ in range(4):
        assert torch.equal(coop.tree_attention(**a), got)
    offsets = np.concatenate([[0], np.cumsum(counts)])
    for b in rng.permutation(requests)[:3]:
        lo, hi = offsets[b], offsets[b + 1]
        one = {**a, "table": a["table"][b:b + 1], "lengths": a["lengths"][b:b + 1],
               "token_offsets": _ints([0, hi - lo])}
        pick = sorted({0, hi - lo - 1})
        for n in "qkv":
            one[n] = a[n][lo:hi]
        if a["parents"] is not None:
            one["parents"] = a["parents"][lo:hi]
        want, tol = ref.attention(one["q"], one["k"], one["v"], a["k_cache"], a["v_cache"], one["table"],
                                  one["lengths"], one["token_offsets"], one["parents"], dim ** -0.5,
                                  only=pick)
        off = np.abs(got[lo:hi].double().cpu().numpy() - want)[pick]
        assert (off <= tol[pick]).all(), (b, (off / tol[pick]).max())


def test_tree_attention_long_chain_written_out():
    """parents of a chain give what parents=None gives, bit for bit."""
    coop = _coop()
    _announce("attention, chains")
    a = _attention_inputs(9, [10, 0, 300], [1, 300, 129], 4, 2, 64, BF16, BF16, 16, "chain")
    got = coop.tree_attention(**a)
    assert torch.equal(got, coop.tree_attention(**{**a, "parents": None}))
    _check_attention(a, got)


def test_tree_attention_large_scores():
    """Scores far apart, where all weights but one vanish, and far from zero."""
    coop = _coop()
    _announce("attention, large scores")
    for dtype in (BF16, FP16):
        a = _attention_inputs(3, [200, 40], [5, 20], 4, 2, 64, dtype, dtype, 16, "tree", spread=6.0)
        _check_attention(a, coop.tree_attention(**a, scale=1.0), 1.0)
        _check_attention(a, coop.tree_attention(**a, scale=0.0), 0.0)
        _check_attention(a, coop.tree_attention(**a, scale=-0.5), -0.5)


@pytest.mark.parametrize("counts, dim", [
    ([1, 1, 1], 64), ([6, 30, 2], 64), ([70, 3, 64], 64), ([70, 3, 64], 128), ([140, 130, 75], 128),
    ([140, 130, 75], 104), ([9, 130, 75], 256)])
@pytest.mark.parametrize("dtype, cache", [(BF16, BF16), (FP16, FP16), (BF16, E4M3)])
def test_tree_attention_sees_nothing_that_is_masked(counts, dim, dtype, cache):
    """NaN and infinities in places past the lengths, on pages that are not in
    the pool, in other requests' rows and in other branches."""
    coop = _coop()
    dim += 8 if cache == E4M3 and dim % 16 else 0  # (rows start at multiples of 16 bytes)
    _announce(f"attention, NaN in masked places, {counts} x {dim}")
    lengths, page = [37, 0, 90], 16
    a = _attention_inputs(11, lengths, counts, 4, 2, dim, dtype, cache, page, "tree", padding=2)
    nan = float("nan")
    for name in ("k_cache", "v_cache"):
        c = a[name].float()
        used = torch.zeros(c.shape[:2], dtype=torch.bool, device=DEV)
        for b, n in enumerate(lengths):
            for j in range(n):
                used[a["table"][b, j // page], j % page] = True
        c[~used] = nan
        a[name] = c.to(cache)
    a["table"][2, 1] = 10**6   # tokens on these pages do not count
    a["table"][2, 3] = -5
    k, v = a["k"].clone(), a["v"].clone()
    k[-2:], v[-2:] = nan, float("inf")
    first = 0
    for n in counts:  # the last token is a leaf of its own: no other token sees it
        if n > 1:
            k[first + n - 1], v[first + n - 1, :, ::2] = float("inf"), nan
            v[first + n - 1, :, 1::2] = float("-inf")
        first += n
    a["k"], a["v"] = k, v
    got = coop.tree_attention(**a)
    last = np.cumsum(counts)[np.array(counts) > 1] - 1
    assert got[last].isnan().all()
    keep = np.setdiff1d(np.arange(sum(counts)), last)
    assert got[keep].isfinite().all()
    want, tol = ref.attention(a["q"], a["k"], a["v"], a["k_cache"], a["v_cache"], a["table"],
                              a["lengths"], a["token_offsets"], a["parents"], dim ** -0.5,
                              a["k_scale"], a["v_scale"])
    assert (np.abs(got.double().cpu().numpy()[keep] - want[keep]) <= tol[keep]).all()


def test_tree_attention_counts_infinite_values_that_are_seen():
    """An infinite value is passed on to the tokens that see it, in its own
    place of the row only, and not a number to those where two signs meet."""
    coop = _coop()
    _announce("attention, infinite values")
    a = _attention_inputs(13, [20], [4], 2, 1, 64, BF16, BF16, 16, "tree")
    a["parents"] = _ints([-1, 0, 0, 2], torch.int32)
    v = a["v"].clone()
    v[0, 0, 3], v[2, 0, 3], v[1, 0, 5] = float("inf"), float("-inf"), float("inf")
    a["v"] = v
    got = coop.tree_attention(**a).float().cpu()
    assert (got[:2, :, 3] == float("inf")).all() and got[2:, :, 3].isnan().all()
    assert (got[1, :, 5] == float("inf")).all() and got[[0, 2, 3]][:, :, 5].isfinite().all()
    rest = [i for i in range(64) if i not in (3, 5)]
    assert got[:, :, rest].isfinite().all()


def test_lengths_past_the_table_and_padded_requests():
    coop = _coop()
    _announce("attention, lengths past the table")
    a = _attention_inputs(15, [48, 48, 5], [2, 1, 0], 4, 2, 64, BF16, BF16, 16, None, cols=3)
    want = coop.tree_attention(**a)
    _check_attention(a, want)
    a["lengths"][0] = 10**15
    a["lengths"][1] = -1
    assert torch.equal(coop.tree_attention(**a), want)


def test_empty_calls():
    coop = _coop()
    _announce("empty calls")
    a = _attention_inputs(1, [5], [2], 4, 2, 64, BF16, BF16, 16, None)
    none = {**a, **{n: a[n][:0] for n in "qkv"}, "token_offsets": a["token_offsets"] * 0}
    assert coop.tree_attention(**none).shape == (0, 4, 64)
    out = torch.full((2, 4, 64), 3.0, dtype=BF16, device=DEV)
    coop.tree_attention(**{**a, "table": a["table"][:0], "lengths": a["lengths"][:0],
                           "token_offsets": a["token_offsets"][:1]}, out=out)
    assert (out == 3).all()
    empty = {**a, "k_cache": a["k_cache"][:0], "v_cache": a["v_cache"][:0]}
    got = coop.tree_attention(**empty)
    _check_attention({**empty, "lengths": a["lengths"] * 0}, got)
    assert coop.slot_map(a["table"], a["lengths"].int(), a["lengths"], a["token_offsets"], 0, 16,
                         4).shape == (0,)
    coop.cache_write(a["k"][:0], a["v"][:0], _ints(np.zeros(0)), a["k_cache"], a["v_cache"])
    coop.cache_write(a["k"], a["v"], _ints([0, 1]), a["k_cache"][:0], a["v_cache"][:0])


# ---------------------------------------------------------------------------
# Refusals of the binding
# ---------------------------------------------------------------------------

def test_refusals():
    coop = _coop()
    a = _attention_inputs(1, [5], [2], 4, 2, 64, BF16, BF16, 16, "tree")

    def bad(error, match, **kw):
        with pytest.raises(error, match=match):
            coop.tree_attention(**{**a, **kw})

    bad(TypeError, "q must be", q=a["q"].float())
    bad(TypeError, "k must be", k=a["k"].half())
    bad(ValueError, "shape", v=a["v"][:1])
    bad(ValueError, "share", q=a["q"][:, :3])
    bad(TypeError, "k_cache", k_cache=a["k_cache"].half(), v_cache=a["v_cache"].half())
    bad(ValueError, "one shape", v_cache=a["v_cache"][:, :8])
    bad(ValueError, "no k_scale", k_scale=torch.ones(2, device=DEV))
    bad(ValueError, "needs k_scale", k_cache=a["k_cache"].to(E4M3), v_cache=a["v_cache"].to(E4M3))
    bad(TypeError, "table must", table=a["table"].long())
    bad(ValueError, "token_offsets must", token_offsets=a["token_offsets"][:1])
    bad(ValueError, "expected", lengths=a["lengths"].cpu())
    bad(TypeError, "parents must", parents=a["parents"].long())
    bad(ValueError, "contiguous", k_cache=a["k_cache"].transpose(2, 3).contiguous().transpose(2, 3))
    bad(ValueError, "16 bytes", q=torch.zeros(2 * 4 * 64 + 1, dtype=BF16, device=DEV)[1:].view(2, 4, 64))
    bad(ValueError, "workspace", workspace=torch.zeros(4, dtype=torch.uint8, device=DEV)[::2])
    bad(ValueError, "out must", out=torch.zeros((2, 4, 65), dtype=BF16, device=DEV))
    with pytest.raises(coop.CoopError):
        coop.tree_attention(**_attention_inputs(1, [5], [2], 2, 2, 264, BF16, BF16, 16, None))
    kind = torch.zeros(4, dtype=torch.uint8, device=DEV)
    t, h, n = a["table"], torch.ones(1, dtype=torch.int32, device=DEV), a["lengths"]
    for args, kw, match in (((kind, t, h, n, 0), {}, "page_size"),
                            ((kind, t, h, n, 16), dict(taken=0), "taken"),
                            ((kind, t, h[:0], n, 16), {}, "held"),
                            ((kind, t, h, n, 16), dict(out=(t, h, kind[:2])), "out"),
                            ((torch.zeros(200000, dtype=torch.uint8, device=DEV), t, h, n, 16),
                             dict(workspace=kind), "workspace")):
        with pytest.raises(ValueError, match=match):
            coop.page_tables(*args, **kw)
    both = torch.zeros(2 * t.numel(), dtype=torch.int32, device=DEV)
    with pytest.raises(coop.CoopError):  # overlaps its input in part
        coop.page_tables(kind, both[:t.numel()].view_as(t), h, n, 16,
                         out=(both[1:t.numel() + 1].view_as(t), h.clone(), kind.clone()))
    with pytest.raises(ValueError, match="num_tokens"):
        coop.slot_map(t, h, n, a["token_offsets"], -1, 16, 4)
    with pytest.raises(ValueError, match="slots"):
        coop.cache_write(a["k"], a["v"], _ints([0]), a["k_cache"], a["v_cache"])


# ---------------------------------------------------------------------------
# Streams, graphs, and the operators together
# ---------------------------------------------------------------------------

def test_another_stream():
    coop = _coop()
    _announce("another stream")
    a = _attention_inputs(21, [300, 20], [3, 9], 8, 2, 128, BF16, BF16, 16, "tree")
    want = coop.tree_attention(**a)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        got = coop.tree_attention(**a, stream=side.cuda_stream)
        side.synchronize()
        assert torch.equal(got, want)
    with torch.cuda.stream(side):
        got = coop.tree_attention(**a)
    side.synchronize()
    assert torch.equal(got, want)


def test_two_streams_at_once():
    """Calls of two streams that run at the same time, with a workspace each."""
    coop = _coop()
    _announce("two streams")
    a = [_attention_inputs(41, [9000, 4000, 2500], [9, 9, 20], 8, 2, 128, BF16, BF16, 16, "tree"),
         _attention_inputs(42, [3000] * 70, [2] * 70, 8, 4, 64, FP16, FP16, 16, None)]
    want = [coop.tree_attention(**x) for x in a]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in a]
    calls = [coop.TreeAttention(**x) for x in a]
    torch.cuda.synchronize()
    for _ in range(10):
        for call, stream in zip(calls, streams):
            call.launch(stream.cuda_stream)
    torch.cuda.synchronize()
    for call, x in zip(calls, want):
        assert torch.equal(call.out, x)


@pytest.mark.parametrize("requests, tokens", [(3, 5), (80, 1), (3, 150)])
def test_attention_captured_and_replayed(requests, tokens):
    """Replays take their lengths, trees and tables from the device."""
    coop = _coop()
    _announce(f"attention of {requests} requests captured")
    made = [_attention_inputs(50 + i, [(i + 1) * 100 + 7 * b for b in range(requests)],
                              [tokens] * requests, 4, 2, 128, BF16, BF16, 16, tree, cols=80)
            for i, tree in enumerate(("tree", "chain", "void"))]
    pages = max(x["k_cache"].shape[0] for x in made)
    a = {n: torch.zeros_like(x) for n, x in made[0].items() if x is not None}
    for n in ("k_cache", "v_cache"):
        a[n] = torch.zeros((pages, *a[n].shape[1:]), dtype=BF16, device=DEV)
    a["table"].fill_(-1)
    a["parents"].fill_(-1)
    coop.tree_attention(**a)  # (loads the kernels)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = coop.tree_attention(**a)
    for x in made + made[:1]:
        for n, to in a.items():
            to[:x[n].shape[0]].copy_(x[n])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, coop.tree_attention(**x))
    _check_attention(made[0], out)


@pytest.mark.parametrize("counts", [[1, 2, 1], [30, 9, 25], [200, 3, 180]])
@pytest.mark.parametrize("cache", [BF16, E4M3])
def test_keys_and_values_laid_out_apart(counts, cache):
    """Other strides for the keys than for the values, and pages that two
    requests share: the same bits as from one plain layout."""
    coop = _coop()
    _announce(f"keys and values laid out apart, {counts}")
    a = _attention_inputs(61, [130, 50, 130], counts, 6, 3, 128, BF16, cache, 16, "tree")
    a["table"][2] = a["table"][0]
    want = coop.tree_attention(**a)
    _check_attention(a, want)
    raw = a["k_cache"].view(torch.uint8 if cache == E4M3 else torch.int16)
    a["k_cache"] = raw.transpose(1, 2).contiguous().transpose(1, 2).view(cache)
    assert a["k_cache"].stride() != a["v_cache"].stride()
    assert torch.equal(coop.tree_attention(**a), want)


@pytest.mark.parametrize("cache", [BF16, E4M3])
def test_pools_past_32_bits(cache):
    """Pools of more than 2^32 elements for each of keys and values."""
    coop = _coop()
    pages, page, heads, dim = 300_000, 16, 8, 128
    assert pages * page * heads * dim > 2**32
    _announce(f"a pool past 32 bits, {cache}")
    raw = torch.uint8 if cache == E4M3 else BF16
    far = (torch.empty((pages, page, heads, dim), dtype=raw, device=DEV).view(cache),
           torch.empty((heads, pages, page, dim), dtype=raw, device=DEV).permute(1, 2, 0, 3).view(cache))
    near = tuple(torch.empty((16, page, heads, dim), dtype=raw, device=DEV).view(cache) for _ in "kv")
    where = [299_999, 5, 150_000, 262_143, 262_144, 262_145, 131_071, 131_072, 280_000, 0, 299_998, 77]
    scales = {}
    if cache == E4M3:
        scales = {n: torch.full((heads,), 0.01, device=DEV) for n in ("k_scale", "v_scale")}
    g = torch.Generator(device=DEV).manual_seed(1)
    k, v = (torch.randn((192, heads, dim), generator=g, device=DEV, dtype=BF16) for _ in "kv")
    place = torch.arange(192, device=DEV)
    coop.cache_write(k, v, place, *near, **scales)
    coop.cache_write(k, v, _ints(where)[place // page] * page + place % page, *far, **scales)
    for x, y in zip(far, near):
        got = torch.stack([x[p].contiguous().view(torch.uint8) for p in where])
        assert torch.equal(got, y[:12].view(torch.uint8).view_as(got))
    lengths = _ints([100, 80])
    table = torch.full((2, 8), -1, dtype=torch.int32, device=DEV)
    table[0, :7], table[1, :5] = _ints(range(7), torch.int32), _ints(range(7, 12), torch.int32)
    moved = torch.where(table < 0, table, _ints(where, torch.int32)[table.clamp(min=0)])
    for n in (1, 9, 80):
        q = torch.randn((2 * n, 2 * heads, dim), generator=g, device=DEV, dtype=BF16)
        k, v = (torch.randn((2 * n, heads, dim), generator=g, device=DEV, dtype=BF16) for _ in "kv")
        offsets = _ints([0, n, 2 * n])
        want = coop.tree_attention(q, k, v, *near, table, lengths, offsets, **scales)
        assert torch.equal(coop.tree_attention(q, k, v, *far, moved, lengths, offsets, **scales), want)


class _Server:
    """Sequences in a pool, a decoding step with drafted trees at a time, on
    the package and on the reference."""

    def __init__(self, seed, rows=6, pages=60, cols=12, page=8, heads=2, q_heads=4, dim=64):
        self.rng = np.random.default_rng(seed)
        self.rows, self.page, self.heads, self.q_heads, self.dim = rows, page, heads, q_heads, dim
        self.width = 4  # drafted tokens a row and step
        self.kind = torch.zeros(pages, dtype=torch.uint8, device=DEV)
        self.table = torch.full((rows, cols), -1, dtype=torch.int32, device=DEV)
        self.held = torch.zeros(rows, dtype=torch.int32, device=DEV)
        self.lengths = torch.zeros(rows, dtype=torch.int64, device=DEV)
        self.k_cache, self.v_cache = (torch.full((pages, page, heads, dim), float("nan"), dtype=BF16,
                                                 device=DEV) for _ in "kv")
        self.n = rows * self.width
        self.offsets = _ints(np.arange(rows + 1) * self.width)
        self.new_lengths = torch.zeros_like(self.lengths)
        self.order = torch.zeros(self.n, dtype=torch.int64, device=DEV)
        self.taken_offsets = torch.zeros(rows + 1, dtype=torch.int64, device=DEV)
        self.parents = torch.zeros(self.n, dtype=torch.int32, device=DEV)
        self.q = torch.zeros((self.n, q_heads, dim), dtype=BF16, device=DEV)
        self.k, self.v = (torch.zeros((self.n, heads, dim), dtype=BF16, device=DEV) for _ in "kv")
        self.out = torch.zeros_like(self.q)

    def inputs(self):
        """Draws a step: trees, rows, and the accepted path of each tree (its
        first branch), or a sequence that ends."""
        rng, w = self.rng, self.width
        parents = np.tile([-1, 0, 0, 1], self.rows)
        self.parents.copy_(_ints(parents, torch.int32))
        for t in (self.q, self.k, self.v):
            t.copy_(torch.from_numpy(rng.standard_normal(tuple(t.shape))))
        done = rng.random(self.rows) < 0.1
        path = [0, 1, 3]
        took = np.where(done, 0, rng.integers(1, 4, self.rows))
        order = [b * w + path[i] for b in range(self.rows) for i in range(took[b])]
        self.order.zero_()
        self.order[:len(order)] = _ints(order)
        self.taken_offsets.copy_(_ints(np.concatenate([[0], np.cumsum(took)])))
        lengths = self.lengths.cpu().numpy()
        self.new_lengths.copy_(_ints(np.where(done, 0, np.minimum(lengths + took, 90))))

    def step(self, coop):
        """What a program captures: attention over the pool, pages and slots
        for the accepted tokens, their rows written."""
        coop.tree_attention(self.q, self.k, self.v, self.k_cache, self.v_cache, self.table,
                            self.lengths, self.offsets, self.parents, out=self.out)
        _, _, _, self.status, self.free = coop.page_tables(
            self.kind, self.table, self.held, self.new_lengths, self.page,
            out=(self.table, self.held, self.kind))
        self.slots = coop.slot_map(self.table, self.held, self.new_lengths, self.taken_offsets,
                                   self.n, self.page, self.kind.numel())
        coop.cache_write(self.k[self.order], self.v[self.order], self.slots, self.k_cache,
                         self.v_cache)

    def want(self):
        kept = ("q", "k", "v", "k_cache", "v_cache", "table", "lengths", "parents", "held", "kind",
                "new_lengths", "taken_offsets", "order")
        return {n: getattr(self, n).clone() for n in kept}

    def check(self, was):
        a = {n: was[n] for n in ("q", "k", "v", "k_cache", "v_cache", "table", "lengths", "parents")}
        _check_attention({**a, "token_offsets": self.offsets, "k_scale": None, "v_scale": None},
                         self.out)
        want = ref.page_tables(was["kind"].cpu(), was["table"].cpu(), was["held"].cpu(),
                               was["new_lengths"].cpu(), self.page)
        _check_tables((self.table, self.held, self.kind, self.status, self.free), want)
        slots = ref.slot_map(want[0], want[1], was["new_lengths"].cpu(),
                             was["taken_offsets"].cpu(), self.n, self.page, len(want[2]))
        assert np.array_equal(self.slots.cpu().numpy(), slots)
        good = np.flatnonzero(slots >= 0)
        for x, cache, old in ((was["k"], self.k_cache, was["k_cache"]),
                              (was["v"], self.v_cache, was["v_cache"])):
            rows = old.view(-1, self.heads, self.dim).clone()
            rows[_ints(slots[good])] = x[was["order"]][_ints(good)]
            assert torch.equal(rows.view(torch.int16), cache.view(-1, self.heads, self.dim).view(torch.int16))
        # a row that could not grow keeps its length
        grown = self.held.long() * self.page >= self.new_lengths
        self.lengths.copy_(torch.where(grown, self.new_lengths, self.lengths))


def test_steps_together():
    coop = _coop()
    _announce("decoding steps together")
    s = _Server(31)
    for _ in range(25):
        s.inputs()
        was = s.want()
        s.step(coop)
        torch.cuda.synchronize()
        s.check(was)
    assert int(s.lengths.max()) > 3 * s.page


def test_steps_captured_and_replayed():
    coop = _coop()
    _announce("decoding steps captured")
    s = _Server(32)
    s.inputs()
    s.step(coop)   # (loads the kernels)
    s = _Server(33)
    s.inputs()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.step(coop)
    torch.cuda.synchronize()
    for i in range(12):
        if i:
            s.inputs()
        was = s.want()
        graph.replay()
        torch.cuda.synchronize()
        s.check(was)
        eager = coop.tree_attention(was["q"], was["k"], was["v"], was["k_cache"], was["v_cache"],
                                    was["table"], was["lengths"], s.offsets, was["parents"])
        assert torch.equal(eager, s.out)


def test_pools_of_pages_are_pools():
    """The window search and first fit on the same kinds: which adjacent pages
    to evict for a block of six pages, once none is free."""
    coop = _coop()
    _announce("window search on pages")
    kind = torch.tensor([2, 1, 1, 1, 1, 1, 1, 2, 0, 0], dtype=torch.uint8, device=DEV)
    table = torch.full((1, 4), -1, dtype=torch.int32, device=DEV)
    held = torch.zeros(1, dtype=torch.int32, device=DEV)
    table, held, kind, status, free = coop.page_tables(kind, table, held, _ints([20]), 16,
                                                       taken=coop.COOP_EVICTABLE)
    assert kind.tolist() == [2, 1, 1, 1, 1, 1, 1, 2, 1, 1] and free.item() == 0
    size = torch.full((10,), 4096, dtype=torch.int64, device=DEV)
    cost = _ints([0, 9, 1, 1, 5, 1, 1, 0, 3, 3])
    seg = _ints([0, 10])
    got = coop.window_search(size, cost, kind, seg, _ints([2 * 4096]), _ints([0, 1]))
    assert got.tolist() == [[2, 4, 2]]
    kind[2:4] = coop.COOP_FREE
    assert coop.first_fit(size, kind, seg, _ints([4096]), _ints([0, 1])).tolist() == [2]
    table, held, kind, status, free = coop.page_tables(kind, table, held, _ints([60]), 16)
    assert table.tolist() == [[8, 9, 2, 3]] and status.item() == 0
