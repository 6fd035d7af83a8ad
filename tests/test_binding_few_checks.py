"""The binding's checks of the layer's workspace: what would send a kernel to memory it cannot or must not write (no GPU needed)."""
import types

import pytest
import torch

from paper_2605_05888_amd import binding


def tensor(shape, dtype, device=0, dense=True, cuda=True):
    n = 1
    for s in shape:
        n *= s
    return types.SimpleNamespace(shape=shape, dtype=dtype, is_cuda=cuda, is_contiguous=lambda: dense, dim=lambda: len(shape),
                                 device=types.SimpleNamespace(index=device), data_ptr=lambda: 0x1000, numel=lambda: n, element_size=lambda: 1)


class Library:
    def __getattr__(self, name):
        return lambda *args: self.calls.append((name, args)) or 0

    def __init__(self):
        self.calls = []


@pytest.fixture
def library(monkeypatch):
    lib = Library()
    monkeypatch.setattr(binding, "_lib", lib)
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    return lib


def call(q4, ws):
    b16, u8 = torch.bfloat16, torch.uint8
    N, H, E, K, F = 2, 64, 4, 2, 128
    x, W_r, out = tensor((N, H), b16), tensor((H, E), torch.float32), tensor((N, H), b16)
    idx, w = tensor((N, K), torch.int32), tensor((N, K), torch.float32)
    if q4:
        pairs = [(tensor((E, r, c // 2), u8), tensor((E, r, c // 32), u8)) for r, c in ((F, H), (F, H), (H, F))]
        binding.moe_layer_few_q4(x, W_r, None, K, 0, *pairs, binding.Q4_FP4, 32, idx, w, out, ws)
    else:
        weights = [tensor((E, r, c), b16) for r, c in ((F, H), (F, H), (H, F))]
        binding.moe_layer_few(x, W_r, None, K, 0, *weights, idx, w, out, ws)


@pytest.mark.parametrize("q4", [False, True])
def test_a_workspace_of_the_current_device_is_passed_on(library, q4):
    call(q4, tensor((4096,), torch.uint8))
    call(q4, None)  # (the library says what it needs)
    assert [args[-3:-1] for _, args in library.calls] == [(0x1000, 4096), (None, 0)]


@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("wrong", [dict(cuda=False), dict(dense=False), dict(device=1)])
def test_another_workspace_is_refused(library, q4, wrong):
    with pytest.raises(TypeError, match="ws"):
        call(q4, tensor((4096,), torch.uint8, **wrong))
    assert library.calls == []
