"""Activations of the largest and smallest bf16 numbers against a 64-bit reference, and rows of what is not finite beside others."""
import numpy as np
import pytest

import few_close
import few_reference as ref
import moe_inputs as mi
from test_gpu_layer_few import FORMS, SOFT, Layer
from test_gpu_q4 import FORMATS, dev, host

pytestmark = pytest.mark.gpu

MOST = 0x7F7F  # the largest bf16 number


def large(rng, shape):
    """bf16 bits of numbers from 2^118 up, either sign."""
    return (rng.integers(245 << 7, 255 << 7, shape) | rng.integers(0, 2, shape) << 15).astype(np.uint16)


def small_scales(rng, shape, fmt):
    """Scales from 2^-125 to 2^-122: a code's value times a large activation is about one."""
    if fmt == ref.FP4:
        return rng.integers(2, 5, shape, dtype=np.uint8)
    return (rng.integers(2 << 7, 5 << 7, shape) | rng.integers(0, 2, shape) << 15).astype(np.uint16)


@pytest.mark.parametrize("fmt,group", FORMATS)
@pytest.mark.parametrize("M", [1, 4, 13, 40])
@pytest.mark.parametrize("cols,rows", [(64, 24), (320, 136)])
def test_products_of_the_largest_activations(fmt, group, M, cols, rows):
    import torch
    import paper_2605_05888_amd as hub
    print("large", fmt, group, M, cols, rows, flush=True)
    rng = np.random.default_rng([fmt, group, M, cols])
    codes = rng.integers(0, 256, (1, rows, cols // 2), dtype=np.uint8)
    codes[0, :3] = np.array([0x00, 0x88, 0xFF], np.uint8)[:, None]  # one code all along a row
    scales = small_scales(rng, (1, rows, -(-cols // group)), fmt)
    x = large(rng, (M, cols))
    x[M // 2] = MOST  # its sums over a group are the largest there are
    y = torch.zeros((M, rows), dtype=torch.bfloat16, device="cuda:0")
    hub.moe_matvec_q4(dev(x), None, dev(codes), dev(scales), fmt, group, y)
    want, err = ref.product(ref.f64(x), ref.values(codes[0], scales[0], fmt, group), few_close.held(codes[0], scales[0], fmt, group))
    ref.check(host(y), want, err + ref.HALF["bf16"] * (np.abs(want) + err), "large")


@pytest.mark.parametrize("fmt,group", FORMATS)
@pytest.mark.parametrize("M", [2, 13, 40])
def test_products_of_the_smallest_activations(fmt, group, M):
    """Normal numbers up to 2^-120; with scales of about 2^110 their products are ordinary numbers."""
    import torch
    import paper_2605_05888_amd as hub
    print("small", fmt, group, M, flush=True)
    rng = np.random.default_rng([fmt, group, M])
    cols, rows = 192, 40
    codes = rng.integers(0, 256, (1, rows, cols // 2), dtype=np.uint8)
    at = rng.integers(235, 240, (1, rows, -(-cols // group)))
    scales = at.astype(np.uint8) if fmt == ref.FP4 else (at << 7).astype(np.uint16)
    x = (rng.integers(1 << 7, 7 << 7, (M, cols)) | rng.integers(0, 2, (M, cols)) << 15).astype(np.uint16)
    y = torch.zeros((M, rows), dtype=torch.bfloat16, device="cuda:0")
    hub.moe_matvec_q4(dev(x), None, dev(codes), dev(scales), fmt, group, y)
    want, err = ref.product(ref.f64(x), ref.values(codes[0], scales[0], fmt, group), few_close.held(codes[0], scales[0], fmt, group))
    ref.check(host(y), want, err + ref.HALF["bf16"] * (np.abs(want) + err), "small")


class CloseLayer(Layer):
    def matrix(self, which):
        w = self.w[which]
        return lambda e: (ref.values(w[0][e], w[1][e], *self.form), few_close.held(w[0][e], w[1][e], *self.form))


@pytest.mark.parametrize("form", FORMATS)
@pytest.mark.parametrize("N,H,E,K,F", [(1, 64, 4, 2, 64), (6, 192, 5, 2, 128), (20, 320, 3, 2, 192), (50, 128, 2, 1, 64)])
def test_layer_of_the_largest_activations(form, N, H, E, K, F):
    print("large layer", form, N, H, E, K, F, flush=True)
    rng = np.random.default_rng([N, H, form[1]])
    x = mi.bf16_bits_to_f32(large(rng, (N, H)))
    W_r = (rng.standard_normal((H, E)) * 2.0 ** -124).astype(np.float32)
    t = CloseLayer(form, N, H, E, K, F, SOFT, x=x, W_r=W_r)
    for which in range(2):  # gate, up
        t.w[which] = (t.w[which][0], small_scales(rng, t.w[which][1].shape, form[0]))
    t.on_device()
    t.check()


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("N", [3, 12, 30, 40])
@pytest.mark.parametrize("bad", ["large", "inf", "nan"])
def test_a_token_of_what_is_not_finite_leaves_the_others_their_bits(form, N, bad):
    """Every token goes to every expert, so that the lists are the same."""
    import torch
    H, E, F = (132, 2, 100) if form == "f32" else (192, 2, 320)
    t = Layer(form, N, H, E, E, F)
    want = t.call().clone()
    x = t.d["x"].clone()
    x[1, 5] = {"large": 3.3e38, "inf": float("inf"), "nan": float("nan")}[bad]
    x[1, 6] = -x[1, 5]
    t.d["x"] = x
    got = t.call()
    rest = [n for n in range(N) if n != 1]
    assert bool(torch.isfinite(got[rest].float()).all())
    assert torch.equal(got[rest], want[rest])


@pytest.mark.parametrize("fmt,group", FORMATS)
@pytest.mark.parametrize("M", [3, 12, 40])
def test_products_of_what_is_not_finite_stay_in_their_row(fmt, group, M):
    import torch
    import paper_2605_05888_amd as hub
    rng = np.random.default_rng(M)
    rows, cols = 56, 448
    codes = dev(rng.integers(0, 256, (1, rows, cols // 2), dtype=np.uint8))
    scales = rng.integers(117, 125, (1, rows, -(-cols // group)))
    scales = dev(scales.astype(np.uint8) if fmt == ref.FP4 else (scales << 7).astype(np.uint16))
    x = dev(mi.f32_to_bf16_bits(rng.standard_normal((M, cols)).astype(np.float32)))
    y = [torch.zeros((M, rows), dtype=torch.bfloat16, device="cuda:0") for _ in range(2)]
    hub.moe_matvec_q4(x, None, codes, scales, fmt, group, y[0])
    x[1, 7], x[1, 300], x[1, 301] = float("nan"), float("inf"), -float("inf")
    hub.moe_matvec_q4(x, None, codes, scales, fmt, group, y[1])
    rest = [m for m in range(M) if m != 1]
    assert bool(torch.isfinite(y[1][rest].float()).all()) and torch.equal(y[0][rest], y[1][rest])
    assert bool(torch.isnan(y[1][1].float()).all())
