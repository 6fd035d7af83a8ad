"""Segment offsets that break their contract: rows outside x and y are neither read nor written."""
import numpy as np
import pytest

import few_reference as ref
import moe_inputs as mi
from test_gpu_q4 import dev, host, random_q4

pytestmark = pytest.mark.gpu

M, ROWS, COLS, BEHIND = 21, 48, 192, 9  # x and y lie between rows of their own kind, so that nothing else can be hit


def product(seg, fmt, group):
    import torch
    import paper_2605_05888_amd as hub
    print("offsets", seg, fmt, group, flush=True)
    rng = np.random.default_rng(len(seg))
    E = len(seg) - 1
    codes, scales = random_q4(rng, (E, ROWS, COLS), fmt, group)
    x = mi.f32_to_bf16_bits(rng.standard_normal((M + 2 * BEHIND, COLS)).astype(np.float32))
    y = torch.full((M + 2 * BEHIND, ROWS), 7.0, dtype=torch.bfloat16, device="cuda:0")
    hub.moe_matvec_q4(dev(x)[BEHIND:BEHIND + M], dev(np.array(seg, np.int32)), dev(codes), dev(scales), fmt, group, y[BEHIND:BEHIND + M])
    got = host(y)
    assert (ref.f64(got[:BEHIND]) == 7.0).all() and (ref.f64(got[BEHIND + M:]) == 7.0).all()
    return x[BEHIND:BEHIND + M], got[BEHIND:BEHIND + M], codes, scales


@pytest.mark.parametrize("fmt,group", [(ref.FP4, 32), (ref.INT4, 64)])
@pytest.mark.parametrize("seg", [[-5, 3, 10, M + 7], [-9, -1, M, M + 1], [M + 2, M + 5, M + 9]])
def test_offsets_outside_count_as_the_nearer_end(seg, fmt, group):
    x, got, codes, scales = product(seg, fmt, group)
    at = np.clip(seg, 0, M)
    for e in range(len(seg) - 1):
        m = slice(at[e], at[e + 1])
        want, err = ref.product(ref.f64(x)[m], ref.values(codes[e], scales[e], fmt, group), ref.most(codes[e], scales[e], fmt, group))
        if want.size:
            ref.check(got[m], want, err + ref.HALF["bf16"] * (np.abs(want) + err), (seg, e))
    assert (ref.f64(got[:at[0]]) == 7.0).all() and (ref.f64(got[at[-1]:]) == 7.0).all()


@pytest.mark.parametrize("seg", [[0, M, 4, M], [M, 0, M, 0], [M + 8, 2, -3, 5], [0] + [M, 0] * 40])
def test_offsets_that_decrease_touch_nothing_outside(seg):
    product(seg, ref.FP4, 32)
