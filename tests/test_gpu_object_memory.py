"""Buffers that the objects over the caller's tensors own: they stay theirs while calls that use them are still running, and
while a captured graph can still be replayed."""
import numpy as np
import pytest

from paper_2606_07665_b200 import workloads as W
from tests.test_gpu_q4 import Case, bits, dev

pytestmark = pytest.mark.gpu

LENS = [5000, 100, 3000]
WAIT = 1_000_000_000                  # cycles that the side stream is busy before the call: half a second


@pytest.fixture(scope="module")
def rt():
    import torch
    from paper_2606_07665_b200 import build, runner
    build.build()
    torch.cuda.set_device(0)
    return runner


def place(*tensors):
    return [(t.data_ptr(), t.numel() * t.element_size()) for t in tensors]


def overlap(a, b):
    return any(x < y + m and y < x + n for x, n in a for y, m in b)


def handed_out(buffers):
    """Whether the allocator gives any of these places (address, bytes) to new tensors of the current stream."""
    import torch
    return overlap(buffers, place(*[torch.empty(n, dtype=torch.uint8, device="cuda") for _, n in buffers for _ in range(8)]))


def attention(rt, kind):
    """(object, its one call that takes a stream)"""
    import torch
    c = Case(rt, 70, LENS, 8, 2, 64, 16, 32)
    kw = dict(lens_host=c.lens, num_splits=5, row_order=[0, 2, 1])
    q = dev(bits(c.rng, 3, 8, 64))
    if kind == "q4":
        h = rt.Q4DecodeStep(c.upload(rt), dev(c.table), dev(c.lens), 8, **kw)
    else:
        kv = [dev(bits(c.rng, c.num_pages, 16, 2, 64)) for _ in range(2)]
        h = rt.PagedAttention(*kv, dev(c.table.clip(0)), dev(c.lens), 8, **kw)
    out = torch.empty_like(q)
    return h, lambda stream: h.attention(q, out=out, stream=stream), out


@pytest.mark.parametrize("kind", ["q4", "bf16"])
@pytest.mark.parametrize("how", ["stream", "handle", "current"])
@pytest.mark.parametrize("end", ["plan", "drop"])
def test_buffers_outlive_the_calls_that_use_them(rt, kind, how, end):
    import torch
    h, call, out = attention(rt, kind)
    call(None)
    torch.cuda.synchronize()
    want = out.clone()
    out.zero_()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(WAIT)
        if how == "current":
            call(None)
    if how != "current":
        call(side.cuda_stream if how == "handle" else side)
    old = place(h.workspace, h.row_order) + (place(h.status_flag) if end == "drop" else [])
    if end == "plan":
        h.plan(lens_host=LENS, num_splits=7, row_order=[2, 0, 1])
        assert not overlap(old, place(h.workspace, h.row_order))
    else:
        call = None
        h = None
    early = handed_out(old)
    busy = not side.query()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    if not busy:
        pytest.skip("the side stream was done too early for this test to say anything")
    assert not early
    if end == "plan":
        call(None)                     # another split count, so other low bits
        torch.cuda.synchronize()
        assert bool(((out.view(torch.bfloat16).double() - want.view(torch.bfloat16).double()).abs() < 0.05).all())


def test_pages_and_cache_buffers_outlive_the_calls_that_use_them(rt):
    import torch
    cache = rt.Q4Cache.empty(64, 16, 2, 64, 32)
    table = torch.arange(32, dtype=torch.int32, device="cuda").reshape(4, 8)
    lens, refs = torch.tensor([40, -1, -1, -1], dtype=torch.int32, device="cuda"), torch.zeros(64, dtype=torch.int32, device="cuda")
    refs[:3] = 1
    pages = rt.CachePages(cache.pools, table, lens, refs, 16)
    pairs = torch.tensor([[0, 1]], dtype=torch.int32, device="cuda")
    k = torch.ones(8, 2, 64, dtype=torch.bfloat16, device="cuda")
    start, off = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.tensor([0, 8, 8, 8, 8], dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    pages.fork(pairs)                   # a kernel's first launch waits for the device
    pages.release(pairs[0, 1:])
    cache.store(k, k, table, start, off)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(WAIT)
        pages.fork(pairs)
        cache.store(k, k, table, start, off)
    old = place(pages.workspace, pages.status_flag, cache.status_flag, cache.k_codes, cache.v_codes, cache.params)
    pages = cache = None
    early = handed_out(old)
    busy = not side.query()
    torch.cuda.synchronize()
    if not busy:
        pytest.skip("the side stream was done too early for this test to say anything")
    assert not early


@pytest.mark.parametrize("kind", ["q4", "bf16"])
@pytest.mark.parametrize("warm", [False, True])
def test_a_captured_graph_keeps_the_plan_that_it_was_captured_under(rt, kind, warm):
    import torch
    h, call, out = attention(rt, kind)
    side = torch.cuda.Stream()
    if warm:                            # the usual way: a call on the stream of the capture before it
        call(side)
        torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call(None)
    old = place(h.workspace, h.row_order)
    for n in (7, 3):
        h.plan(lens_host=LENS, num_splits=n, row_order=[2, 0, 1])
        assert not overlap(old, place(h.workspace, h.row_order))
    torch.cuda.synchronize()
    assert not handed_out(old)
    call(None)
    torch.cuda.synchronize()
    want = out.clone()
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert bool(((out.view(torch.bfloat16).double() - want.view(torch.bfloat16).double()).abs() < 0.05).all())


def test_a_capture_is_noticed_on_a_stream_that_is_not_the_current_one(rt):
    import torch
    h, call, out = attention(rt, "q4")
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    call(b)
    torch.cuda.synchronize()
    want = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=a):
        b.wait_stream(a)
        call(b.cuda_stream)             # the fork of the capture, by its handle
        a.wait_stream(b)
    old = place(h.workspace, h.row_order)
    h.plan(lens_host=LENS, num_splits=7, row_order=[2, 0, 1])
    torch.cuda.synchronize()
    assert not overlap(old, place(h.workspace, h.row_order)) and not handed_out(old)
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_plans_in_a_loop_do_not_pile_up(rt):
    # without captured graphs nothing old is kept
    import torch
    h, call, out = attention(rt, "q4")
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    for i in range(50):
        call(None)
        h.plan(lens_host=LENS, num_splits=5, row_order=[0, 2, 1])
    torch.cuda.synchronize()
    assert torch.cuda.memory_allocated() <= before + 4096
