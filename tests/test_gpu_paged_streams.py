"""Paged-pool calls on other streams than the one that they were made on."""
import sys
import time

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
DEV = "cuda"


def _coop():
    import paper_2311_00591_amd as coop
    return coop


def _announce(label):
    print(f"[gpu case] paged: {label}", flush=True)
    sys.stdout.flush()


@pytest.fixture(scope="module")
def busy():
    """Enqueues some 150 ms of products on the current stream; returns an event
    behind them."""
    a = torch.zeros((8192, 8192), dtype=BF16, device=DEV)
    out = torch.empty_like(a)
    torch.mm(a, a, out=out)
    torch.cuda.synchronize()

    def enqueue(n=60):
        for _ in range(n):
            torch.mm(a, a, out=out)
        return torch.cuda.current_stream().record_event()

    start = time.perf_counter()
    enqueue(20).synchronize()
    took = (time.perf_counter() - start) / 20
    return lambda: enqueue(int(0.15 / took) + 1)


def _attention():
    g = torch.Generator(device=DEV).manual_seed(1)
    rnd = lambda *s: torch.randn(s, generator=g, device=DEV, dtype=BF16)
    return dict(q=rnd(8, 8, 128), k=rnd(8, 2, 128), v=rnd(8, 2, 128), k_cache=rnd(40, 16, 2, 128),
                v_cache=rnd(40, 16, 2, 128),
                table=torch.randperm(40, generator=g, device=DEV).to(torch.int32).view(2, 20),
                lengths=torch.tensor([300, 77], device=DEV),
                token_offsets=torch.tensor([0, 3, 8], device=DEV))


def _memory_of(t):
    return t.data_ptr(), t.untyped_storage().nbytes()


def _taken_while(event, memory):
    """Allocates and overwrites as much as `memory` says, many times over, on
    the current stream; whether any of it was that memory, and whether `event`
    was still ahead."""
    hit = []
    for at, size in memory:
        for t in [torch.empty(size, dtype=torch.uint8, device=DEV) for _ in range(4)]:
            t.fill_(0xff)
            hit.append(t.data_ptr() < at + size and at < t.data_ptr() + size)
    return any(hit), not event.query()


def test_the_default_stream_by_its_handle(busy):
    """stream=0 names the default stream, while another one is current: memory
    of a dropped call is not handed out before the default stream is done."""
    coop = _coop()
    _announce("the default stream's handle")
    a = _attention()
    want = coop.tree_attention(**a)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    copy = torch.empty_like(want)
    ahead = busy()
    with torch.cuda.stream(side):
        call = coop.TreeAttention(**a)
        call.launch(torch.cuda.default_stream().cuda_stream)
        memory = [_memory_of(call.out), _memory_of(call.workspace)]
        with torch.cuda.stream(torch.cuda.default_stream()):
            copy.copy_(call.out)
        del call
        taken, waiting = _taken_while(ahead, memory)
    assert waiting and not taken
    torch.cuda.synchronize()
    assert torch.equal(copy, want)


def test_memory_is_waited_for(busy):
    """Results and workspaces come from the allocator for the stream that is
    current, where work on what was there before may be under way: a call on
    another stream starts behind it, a later launch there does not wait again."""
    coop = _coop()
    _announce("other streams wait for the memory")
    a = _attention()
    want = coop.tree_attention(**a)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    ahead = busy()
    got = coop.tree_attention(**a, stream=side.cuda_stream)
    done = side.record_event()
    time.sleep(0.01)
    early = done.query()
    assert not ahead.query() and not early
    torch.cuda.synchronize()
    assert torch.equal(got, want)

    call = coop.TreeAttention(**a)
    call.launch()
    torch.cuda.synchronize()
    call.out.zero_()
    ahead = busy()
    with torch.cuda.stream(side):
        call.launch()
    done = side.record_event()
    time.sleep(0.01)
    early = done.query()
    assert not ahead.query() and not early
    torch.cuda.synchronize()
    assert torch.equal(call.out, want)

    call.out.zero_()
    torch.cuda.synchronize()
    ahead = busy()
    call.launch(side.cuda_stream)
    side.record_event().synchronize()
    assert not ahead.query()
    torch.cuda.synchronize()
    assert torch.equal(call.out, want)


def test_memory_is_kept_for_the_stream_that_uses_it(busy):
    """A call made on one stream, launched while another is current and
    dropped: its memory is not handed out before that stream is done."""
    coop = _coop()
    _announce("memory kept for another stream")
    a = _attention()
    want = coop.tree_attention(**a)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    copy = torch.empty_like(want)
    call = coop.TreeAttention(**a)
    memory = [_memory_of(call.out), _memory_of(call.workspace)]
    with torch.cuda.stream(side):
        ahead = busy()
        call.launch()
        copy.copy_(call.out)
    del call
    taken, waiting = _taken_while(ahead, memory)
    assert waiting and not taken
    torch.cuda.synchronize()
    assert torch.equal(copy, want)


def test_prepared_calls_are_captured_on_another_stream():
    """A call made before the capture, on the stream that was current then."""
    coop = _coop()
    _announce("a prepared call captured")
    a = _attention()
    want = coop.tree_attention(**a)
    call = coop.TreeAttention(**a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call.launch()
    for _ in range(4):
        call.out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(call.out, want)
        assert torch.equal(coop.tree_attention(**a), want)
    # and eagerly on a third one afterwards
    side = torch.cuda.Stream()
    call.out.zero_()
    call.launch(side.cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(call.out, want)


def test_a_branch_of_a_capture():
    """A call on a second stream of the capture, which the first one joins."""
    coop = _coop()
    _announce("a branch of a capture")
    a = _attention()
    want = coop.tree_attention(**a)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = coop.tree_attention(**a, stream=side.cuda_stream)
        torch.cuda.current_stream().wait_stream(side)
        twice = got + got
    for _ in range(4):
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(twice, want + want)


def test_inputs_are_kept_for_the_stream_that_reads_them(busy):
    """Inputs that are dropped with the call, made for it alone (accepted
    tokens' rows): their memory is not handed out before they were read."""
    coop = _coop()
    _announce("inputs kept for another stream")
    g = torch.Generator(device=DEV).manual_seed(2)
    k, v = (torch.randn((64, 8, 128), generator=g, device=DEV, dtype=BF16) for _ in "kv")
    k_cache, v_cache = (torch.zeros((8, 16, 8, 128), device=DEV, dtype=BF16) for _ in "kv")
    picked = torch.randperm(64, generator=g, device=DEV)
    slots = torch.arange(64, device=DEV)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        ahead = busy()
    rows = [k[picked], v[picked], slots + 64]
    memory = [_memory_of(t) for t in rows]
    coop.cache_write(*rows, k_cache, v_cache, stream=side.cuda_stream)
    del rows
    taken, waiting = _taken_while(ahead, memory)
    assert waiting and not taken
    torch.cuda.synchronize()
    for cache, x in ((k_cache, k), (v_cache, v)):
        assert torch.equal(cache.view(128, 8, 128)[64:], x[picked]) and not cache[:4].any()


def test_empty_calls_on_another_stream():
    """Tensors without memory have none to wait for or to keep."""
    coop = _coop()
    _announce("empty calls on another stream")
    a = _attention()
    side = torch.cuda.Stream()
    stream = side.cuda_stream
    none = {**a, **{n: a[n][:0] for n in "qkv"}, "token_offsets": a["token_offsets"] * 0}
    assert coop.tree_attention(**none, stream=stream).shape == (0, 8, 128)
    empty = torch.zeros(0, dtype=torch.int64, device=DEV)
    coop.cache_write(a["k"][:0], a["v"][:0], empty, a["k_cache"], a["v_cache"], stream=stream)
    assert coop.slot_map(a["table"], a["lengths"].int(), a["lengths"], a["token_offsets"], 0, 16, 40,
                         stream=stream).shape == (0,)
    got = coop.page_tables(torch.zeros(3, dtype=torch.uint8, device=DEV), a["table"][:0, :0],
                           empty.int(), empty, 16, stream=stream)
    side.synchronize()
    assert (got[3].item(), got[4].item()) == (0, 3)
