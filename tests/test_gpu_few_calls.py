"""Calls of the decoding operators that a program may make and that their sizes do not show: tensors that begin anywhere a row may,
captured conversions and products, several threads."""
import threading

import numpy as np
import pytest

import few_reference as ref
import moe_inputs as mi
from test_gpu_layer_few import FORMS, SOFT, Layer
from test_gpu_q4 import FORMATS, dev, random_q4

pytestmark = pytest.mark.gpu


def moved(t, bytes_):
    """The same values in memory that begins `bytes_` past a line's start."""
    import torch
    n = bytes_ // t.element_size()
    room = torch.empty(t.numel() + n + 64, dtype=t.dtype, device=t.device)
    v = room[n:n + t.numel()].view(t.shape)
    v.copy_(t)
    assert v.data_ptr() % 128 == bytes_ and v.is_contiguous()
    return v


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("N", [2, 11, 37])
@pytest.mark.parametrize("by", [16, 48, 112])
def test_layer_of_tensors_that_begin_inside_a_line(form, N, by):
    import torch
    t = Layer(form, N, 320, 6, 3, 448, SOFT, np.zeros(6))
    want = t.call().clone()
    t.d["w"] = [tuple(moved(a, by) for a in p) if isinstance(p, tuple) else moved(p, by) for p in t.d["w"]]
    for k in ("x", "W_r", "bias"):
        t.d[k] = moved(t.d[k], by)
    t.out, t.idx, t.wt = (moved(a, by) for a in (t.out, t.idx, t.wt))
    t.out[:N].fill_(0)
    assert torch.equal(t.call(), want)
    assert bool((t.out[N] == -7).all() and (t.idx[N] == -7).all() and (t.wt[N] == -7).all())


def chain(hub, w, x, codes, scales, back, y, fmt, group):
    hub.moe_quantize_q4(w, fmt, group, codes, scales)
    hub.moe_dequantize_q4(codes, scales, fmt, group, back)
    hub.moe_matvec_q4(x, None, codes, scales, fmt, group, y)


def operands(rng, rows, cols, M, fmt, group):
    import torch
    w = dev(mi.f32_to_bf16_bits(rng.standard_normal((1, rows, cols)).astype(np.float32)))
    x = dev(mi.f32_to_bf16_bits(rng.standard_normal((M, cols)).astype(np.float32)))
    codes, scales = (dev(a) for a in random_q4(rng, (1, rows, cols), fmt, group))
    return w, x, codes, scales, torch.zeros_like(w), torch.zeros((M, rows), dtype=torch.bfloat16, device="cuda:0")


@pytest.mark.parametrize("fmt,group", FORMATS)
def test_captured_conversions_and_products(fmt, group):
    import torch
    import paper_2605_05888_amd as hub
    a = operands(np.random.default_rng(group), 264, 448, 5, fmt, group)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        chain(hub, *a, fmt, group)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        chain(hub, *a, fmt, group)
    for turn in range(4):
        a[0].copy_(a[0].roll(turn, 1))
        chain(hub, *a, fmt, group)
        want = [t.clone() for t in a[2:]]
        for t in a[2:]:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        for t, v in zip(a[2:], want):
            assert torch.equal(t, v), turn


def test_calls_of_several_threads():
    """Each thread with a stream, tensors and a workspace of its own."""
    import torch
    import paper_2605_05888_amd as hub
    hub.load_library()
    jobs = [(Layer(form, n, 512, 16, 2, 256, SOFT, seed=n), torch.cuda.Stream()) for n, form in ((1, "bf16"), (9, (ref.FP4, 32)), (40, (ref.INT4, 64)), (5, "f32"))]
    want = [t.call().clone() for t, _ in jobs]
    torch.cuda.synchronize()
    failed = []

    def work(job, w):
        try:
            t, stream = job
            torch.cuda.set_device(0)
            with torch.cuda.stream(stream):
                for _ in range(20):
                    t.out.fill_(0)
                    t.call()
                    if not torch.equal(t.out[:t.N], w):
                        failed.append(t.form)
        except Exception as e:  # (of a thread: to the test)
            failed.append(repr(e))

    threads = [threading.Thread(target=work, args=a) for a in zip(jobs, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed
