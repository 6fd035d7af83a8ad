"""That the checks by blocks fail for what a kernel with a missing part would give, at the sizes of the GPU tests."""
import numpy as np
import pytest

import few_close
import few_reference as ref
import moe_inputs as mi
from test_gpu_q4 import random_q4


def refused(got, want, dtype="bf16"):
    return bool((few_close.off(got, want) >= few_close.LIMIT[dtype]).any())


def bf16(v):
    return ref.f64(mi.f32_to_bf16_bits(v.astype(np.float32)))


@pytest.mark.parametrize("fmt,group", [(ref.FP4, 32), (ref.INT4, 32), (ref.INT4, 128)])
@pytest.mark.parametrize("N,H,E,K,F", [(1, 2048, 8, 4, 1408), (5, 576, 40, 5, 128), (8, 7168, 9, 2, 64), (4, 64, 6, 2, 8192),
                                       (20, 7168, 5, 2, 128), (3, 8256, 4, 2, 64), (2, 33024, 2, 1, 64), (64, 256, 4, 2, 448)])
def test_layer(fmt, group, N, H, E, K, F):
    rng = np.random.default_rng([N, H, E, F])
    w = [random_q4(rng, s, fmt, group) for s in ((E, F, H), (E, F, H), (E, H, F))]
    x = bf16(rng.standard_normal((N, H)))
    idx = np.stack([rng.choice(E, K, replace=False) for _ in range(N)])
    weight = np.full((N, K), 1.0 / K)

    def layer(lost_h=(0, 0), lost_f=(0, 0)):
        def of(which, lost):
            def matrix(e):
                v = ref.values(w[which][0][e], w[which][1][e], fmt, group)
                v[:, lost[0]:lost[1]] = 0.0
                return v, np.abs(v)
            return matrix
        return ref.layer(x, idx, weight, of(0, lost_h), of(1, (0, 0)), of(2, lost_f), "bf16")[0]

    want = layer()
    assert not refused(bf16(want), want)  # (one rounding of the two)
    assert refused(np.zeros_like(want), want) and refused(-want, want)
    assert refused(layer(lost_h=(H - 64, H)), want) and refused(layer(lost_f=(0, 64)), want)
    one = want.copy()
    one[N // 2, H - 64 + np.argmax(np.abs(one[N // 2, H - 64:]))] = 0.0  # a column of its size or more
    assert refused(one, want)
    part = want.copy()
    part[:, :16] = part[:, 16:32]  # another tile's columns
    assert refused(part, want)


@pytest.mark.parametrize("fmt,group", [(ref.FP4, 32), (ref.INT4, 32), (ref.INT4, 64), (ref.INT4, 128)])
@pytest.mark.parametrize("M,cols,rows", [(1, 16384, 40), (3, 2880, 1000), (16, 4096, 520), (40, 64, 88)])
def test_products(fmt, group, M, cols, rows):
    rng = np.random.default_rng([M, cols, rows])
    codes, scales = random_q4(rng, (rows, cols), fmt, group)
    x, v = bf16(rng.standard_normal((M, cols))), ref.values(codes, scales, fmt, group)
    want = x @ v.T
    assert not refused(bf16(want), want)
    assert refused(np.zeros_like(want), want) and refused(-want, want)
    v[:, cols - 64:] = 0.0  # a line
    assert refused(x @ v.T, want)
