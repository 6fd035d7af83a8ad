"""Waits of the layer for few tokens: what workgroups do about shares that others have not done."""
import contextlib

import pytest

from test_gpu_layer_few import FORMS, SOFT, Layer

pytestmark = pytest.mark.gpu


@contextlib.contextmanager
def waits(polls):
    import paper_2605_05888_amd as hub
    lib = hub.load_library()
    lib.moe_few_test_waits(polls)
    try:
        yield
    finally:
        lib.moe_few_test_waits(-1)


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
