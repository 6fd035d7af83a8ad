"""Conversions of very many short rows, whose last scale covers fewer columns than its group."""
import numpy as np
import pytest

import few_reference as ref
from test_gpu_q4 import host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols,group", [(360_000_000, 64, 128), (5, 64, 128), (1001, 64, 64), (77, 192, 128)])
def test_rows_that_end_inside_a_group(rows, cols, group):
    import torch
    import paper_2605_05888_amd as hub
    print("rows", rows, cols, group, flush=True)
    w = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda:0")
    some = min(rows, 40)
    w[-some:] = torch.randn((some, cols), device="cuda:0").to(torch.bfloat16)
    tail = w[-some:].clone()
    codes = torch.full((rows, cols // 2), 0x11, dtype=torch.uint8, device="cuda:0")
    scales = torch.full((rows, -(-cols // group)), -3.0, dtype=torch.bfloat16, device="cuda:0")
    hub.moe_quantize_q4(w, ref.INT4, group, codes, scales)
    want_c, want_s = ref.quantize(ref.f64(host(tail)), ref.INT4, group)
    assert np.array_equal(host(scales[-some:]), want_s) and np.array_equal(host(codes[-some:]), want_c)
    assert bool((codes[:-some] == 0x88).all()) and bool((scales[:-some] == 0).all())
    w.fill_(5.0)
    hub.moe_dequantize_q4(codes, scales, ref.INT4, group, w)
    back = ref.values(want_c, want_s, ref.INT4, group)
    assert (np.abs(ref.f64(host(w[-some:])) - back) <= 2.0 ** -8 * np.abs(back)).all()
    assert bool((w[:-some] == 0).all())
