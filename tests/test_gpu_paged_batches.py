"""Batches as a server has them."""
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda"


def _coop():
    import paper_2311_00591_amd as coop
    return coop


def _announce(label):
    print(f"[gpu case] paged: {label}", flush=True)
    sys.stdout.flush()


def _ints(a, dtype=torch.int64):
    return torch.tensor(np.asarray(a), device=DEV).to(dtype)


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
