"""Waits of the layer for few tokens: what workgroups do about shares that others have not done."""
import contextlib

import pytest

from test_gpu_layer_few import FORMS, SOFT, Layer

pytestmark = pytest.mark.gpu


@contextlib.contextmanager
def waits(polls, workgroups=0):
    import paper_2605_05888_amd as hub
    lib = hub.load_library()
    lib.moe_few_test_waits(polls, workgroups)
    try:
        yield
    finally:
        lib.moe_few_test_waits(-1, 0)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("N", [3, 21, 64])
def test_shares_that_are_taken_over_at_once_give_the_same_bits(form, N):
    import torch
    t = Layer(form, N, 192, 12, 3, 256, SOFT)
    first = t.call().clone()
    routed = t.idx.clone(), t.wt.clone()
    with waits(0):
        for _ in range(3):
            t.ws.fill_(0xFF)
            t.out.fill_(0)
            t.idx[:N] = -1
            again = t.call()
            torch.cuda.synchronize()
            assert torch.equal(first.view(torch.uint8), again.view(torch.uint8))
            assert torch.equal(routed[0], t.idx) and torch.equal(routed[1], t.wt)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("N,H,F", [(3, 192, 1024), (40, 512, 640)])
@pytest.mark.parametrize("workgroups", [1, 7, 100, 200])
def test_a_call_with_few_workgroups_does_the_others_shares_in_parallel(form, N, H, F, workgroups):
    """As where other work holds the compute units.  The waits of one share after the other, 33 ms each, took seconds; together
    they take one wait, and a few turns."""
    import torch
    print("workgroups", form, N, H, F, workgroups, flush=True)
    t = Layer(form, N, H, 12, 3, F, SOFT)
    first = t.call().clone()
    routed = t.idx.clone(), t.wt.clone()
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    with waits(-1, workgroups):
        for _ in range(2):
            t.ws.fill_(0xFF)
            t.out.fill_(0)
            t.idx[:N] = -1
            start.record()
            again = t.call()
            end.record()
            torch.cuda.synchronize()
            assert torch.equal(first.view(torch.uint8), again.view(torch.uint8))
            assert torch.equal(routed[0], t.idx) and torch.equal(routed[1], t.wt)
    print("ms", start.elapsed_time(end), flush=True)
    assert start.elapsed_time(end) < 100.0


def test_calls_on_several_streams_do_not_wait_for_each_other_for_long():
    """Four streams of calls whose workgroups are on the device in part: a call is some tens of microseconds, and waits of 33 ms
    for a share made it as many milliseconds."""
    import time
    import torch
    layers = [Layer("bf16", n, 1024, 32, 4, 512, SOFT, seed=n) for n in (1, 1, 2, 5)]
    streams = [torch.cuda.Stream() for _ in layers]
    want = [t.call().clone() for t in layers]
    torch.cuda.synchronize()
    calls = 40
    for turn in range(2):
        start = time.perf_counter()
        for _ in range(calls):
            for t, st in zip(layers, streams):
                with torch.cuda.stream(st):
                    t.call()
        torch.cuda.synchronize()
        ms = (time.perf_counter() - start) / calls * 1e3
        print("ms", ms, flush=True)
    assert ms < 5.0
    for t, w in zip(layers, want):
        assert torch.equal(t.out[:t.N], w)
