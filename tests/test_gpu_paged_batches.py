"""Batches as a server has them: single tokens beside a long piece of a prompt,
and pages that the window search takes back from sequences."""
import sys

import numpy as np
import pytest

import paged_reference as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn
DEV = "cuda"


def _coop():
    import paper_2311_00591_amd as coop
    return coop


def _announce(label):
    print(f"[gpu case] paged: {label}", flush=True)
    sys.stdout.flush()


def _ints(a, dtype=torch.int64):
    return torch.tensor(np.asarray(a), device=DEV).to(dtype)


@pytest.mark.parametrize("counts, at, cache", [
    ([1] * 63 + [1024], 63, BF16),     # the mean calls for wide tiles: single tokens on them
    ([1] * 255 + [2048], 100, BF16),   # and for narrow ones: a prompt on them
    ([1] * 40 + [700], 0, E4M3), ([1] * 7 + [900], 3, E4M3), ([1, 1, 1, 3000], 3, BF16)])
def test_a_prompt_among_single_tokens(counts, at, cache):
    """Every row is within what rounding allows (a few of the prompt's, all of
    the single tokens), wherever the prompt stands."""
    coop = _coop()
    n = len(counts)
    counts = counts[:-1][:at] + counts[-1:] + counts[:-1][at:]
    _announce(f"attention, {n - 1} single tokens and a piece of {max(counts)}, {cache}")
    rng = np.random.default_rng(n)
    q_heads, heads, dim, page = 8, 2, 128, 16
    lengths = rng.integers(1, 200, n)
    held = -(-lengths // page)
    pages = int(held.sum()) + 1
    g = torch.Generator().manual_seed(n)
    pool = [torch.randn((pages, page, heads, dim), generator=g) for _ in "kv"]
    scales = [None, None]
    if cache == E4M3:
        scales = [torch.full((heads,), 0.01), torch.full((heads,), 0.02)]
        pool = [x / s[:, None] for x, s in zip(pool, scales)]
        scales = [s.to(DEV) for s in scales]
    k_cache, v_cache = (x.to(cache).to(DEV) for x in pool)
    table = np.full((n, int(held.max())), -1)
    order = rng.permutation(pages)
    for b, h in enumerate(held):
        table[b, :h], order = order[:h], order[h:]
    total = sum(counts)
    q, k, v = (torch.randn((total, h, dim), generator=g).to(DEV, BF16) for h in (q_heads, heads, heads))
    table, lengths = _ints(table, torch.int32), _ints(lengths)
    offsets = np.concatenate([[0], np.cumsum(counts)])
    got = coop.tree_attention(q, k, v, k_cache, v_cache, table, lengths, _ints(offsets),
                              k_scale=scales[0], v_scale=scales[1])
    for b, c in enumerate(counts):
        pick = [0] if c == 1 else [0, 1, c // 2, c - 1]
        lo, hi = offsets[b], offsets[b + 1]
        want, tol = ref.attention(q[lo:hi], k[lo:hi], v[lo:hi], k_cache, v_cache, table[b:b + 1],
                                  lengths[b:b + 1], _ints([0, c]), None, dim ** -0.5, scales[0],
                                  scales[1], only=pick)
        mine, want, tol = got[lo:hi].double().cpu().numpy()[pick], want[pick], tol[pick]
        # (a few of the pool's numbers are past e4m3's range, and not numbers there)
        assert np.array_equal(np.isnan(mine), np.isnan(want))
        fine = ~np.isnan(want)
        worst = (np.abs(mine - want)[fine] / tol[fine]).max()
        assert worst <= 1, (b, worst)


def test_pages_that_are_evicted_leave_their_rows():
    """Pages that the window search picks belong to rows.  A sequence gives
    them back by page_tables: it is cut to the tokens before its first page
    that goes (what it loses is computed again when it comes back); in the same
    call the waiting sequence has them, and no page is in two rows."""
    coop = _coop()
    _announce("evicted pages leave their rows")
    page, evictable = 16, coop.COOP_EVICTABLE
    kind = torch.zeros(12, dtype=torch.uint8, device=DEV)
    table = torch.full((4, 8), -1, dtype=torch.int32, device=DEV)
    held = torch.zeros(4, dtype=torch.int32, device=DEV)
    lengths = _ints([5 * page, 4 * page - 3, 3 * page, 0])
    table, held, kind, status, free = coop.page_tables(kind, table, held, lengths, page, taken=evictable)
    assert kind.tolist() == [1] * 12 and (status.item(), free.item()) == (0, 0)
    wanted = lengths.clone()
    wanted[3] = 2 * page  # waits for two pages
    same = coop.page_tables(kind, table, held, wanted, page, taken=evictable)
    assert same[3].item() == 1 and same[1].tolist() == held.tolist()
    cost = _ints([9, 9, 9, 9, 9, 8, 8, 1, 1, 7, 7, 7])
    start, end, _ = coop.window_search(torch.full((12,), 4096, dtype=torch.int64, device=DEV), cost, kind,
                                       _ints([0, 12]), _ints([2 * 4096]), _ints([0, 1])).tolist()[0]
    assert (start, end) == (7, 9)
    gone = (table >= start) & (table < end)
    first = torch.where(gone.any(1), gone.int().argmax(1), held)  # the first page that goes
    cut = torch.where(first < held, first * page, wanted)
    table, held, kind, status, free = coop.page_tables(kind, table, held, cut, page, taken=evictable,
                                                       out=(table, held, kind))
    assert (status.item(), free.item()) == (0, 0) and held.tolist() == [5, 2, 3, 2]
    entries = table[table >= 0]
    assert entries.numel() == 12 == entries.unique().numel()
    assert table[1].tolist() == [5, 6] + [-1] * 6 and table[3, :2].tolist() == [7, 8]


def test_a_long_row_that_is_refused_takes_no_longer_than_one_that_is_granted():
    """A prompt that finds too few pages leaves its row's entries empty, a
    wavefront at a time: one thread took 23 times as long as granting 16000."""
    coop = _coop()
    _announce("a long row refused")
    cols = 16000
    kind = torch.full((100000,), 2, dtype=torch.uint8, device=DEV)
    kind[:cols - 1] = 0
    table = torch.full((4, cols), 77, dtype=torch.int32, device=DEV)
    held = torch.tensor([0, 0, 3, 0], dtype=torch.int32, device=DEV)
    took = []
    for need in (cols - 1, cols):
        lengths = torch.tensor([0, need, 1, 0], device=DEV)
        call = coop.PageTables(kind, table, held, lengths, 1)
        want = ref.page_tables(kind.cpu(), table.cpu(), held.cpu(), lengths.cpu(), 1)
        got = [t.clone() for t in call()]
        for t, x in zip(got, want):
            assert np.array_equal(t.cpu().numpy().ravel(), np.ravel(x))
        best = np.inf
        for _ in range(6):
            start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            start.record()
            for _ in range(10):
                call.launch()
            end.record()
            torch.cuda.synchronize()
            best = min(best, start.elapsed_time(end) * 100)
        took.append(best)
    print(f"  granted {took[0]:.1f} us, refused {took[1]:.1f} us", flush=True)
    assert took[1] < 4 * took[0]
