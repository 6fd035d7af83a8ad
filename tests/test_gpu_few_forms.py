"""The decoding operators in every form that sizes choose: wide down tiles, several rounds of them, wide panels of products, long
reductions; against a 64-bit reference by blocks of a row, which one missing line, column or part is enough to fail."""
import numpy as np
import pytest

import few_close
import few_reference as ref
import moe_inputs as mi
from test_gpu_layer_few import FORMS, SHAPES, SIGM, SOFT, Layer
from test_gpu_q4 import FORMATS, dev, host, random_q4

pytestmark = pytest.mark.gpu


class CloseLayer(Layer):
    def check(self):
        super().check()
        got = host(self.out[:self.N])
        idx, w = host(self.idx[:self.N]), ref.f64(host(self.wt[:self.N]))
        want, bound = ref.layer(ref.f64(self.x), idx, w, *[self.matrix(i) for i in range(3)], self.dtype)
        ref.check(got, want, bound, "out")
        few_close.check(got, want, self.dtype, "out")

    def matrix(self, which):
        if not isinstance(self.form, tuple):
            return super().matrix(which)
        w = self.w[which]
        return lambda e: (ref.values(w[0][e], w[1][e], *self.form), few_close.held(w[0][e], w[1][e], *self.form))


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("N,H,E,K,F,mode,bias", [s for s in SHAPES if s[1] >= 64])
def test_layer_by_blocks(form, N, H, E, K, F, mode, bias):
    print("layer", form, N, H, E, K, F, mode, bias, flush=True)
    b = np.random.default_rng(E).standard_normal(E) if bias else None
    CloseLayer(form, N, H, E, K, F, mode, b).check()


# more than 4096 columns have down tiles of more than 16, more than 8192 (4096 with many rows: 64 x 32) a second round of them
WIDE = [(20, 7168, 5, 2, 128), (33, 4160, 6, 2, 64), (64, 5760, 3, 1, 192), (3, 8256, 4, 2, 64), (40, 8320, 3, 2, 192),
        (64, 4160, 32, 32, 64), (64, 12352, 4, 3, 64), (2, 33024, 2, 1, 64), (17, 16448, 2, 2, 320)]


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("N,H,E,K,F", WIDE)
def test_layer_with_wide_down_tiles_and_rounds_of_them(form, N, H, E, K, F):
    print("wide", form, N, H, E, K, F, flush=True)
    CloseLayer(form, N, H, E, K, F, SIGM).check()


@pytest.mark.parametrize("N,H,E,K,F", [(7, 4100, 4, 2, 36), (30, 8196, 3, 2, 100), (64, 6148, 2, 2, 68)])
def test_layer_fp32_odd_sizes_with_wide_down_tiles(N, H, E, K, F):
    print("wide f32", N, H, E, K, F, flush=True)
    CloseLayer("f32", N, H, E, K, F, SOFT).check()


PRODUCTS = [
    # rows of each segment (None: one matrix for all M rows), M, cols, rows of W; panels of 32 rows from 4096 on in all
    ([1, 3, 10, 40, 0, 17, 33, 4], 0, 64, 5768), ([1, 3, 10, 40, 0, 17, 33, 4], 0, 320, 5768),
    ([2, 70, 0, 9, 16, 1, 5, 12], 0, 2880, 5768), ([4] * 30 + [20, 50], 0, 832, 1096), ([1] * 64, 0, 192, 520),
    (None, 1, 448, 32776), (None, 3, 2880, 33000), (None, 16, 192, 32800), (None, 64, 704, 16384), (None, 200, 320, 4104),
    # panels of 16
    (None, 1, 16384, 40), (None, 17, 14336, 24), (None, 40, 8192, 16), ([3, 0, 18], 0, 7168, 48),
]


@pytest.mark.parametrize("fmt,group", FORMATS)
@pytest.mark.parametrize("counts,M,cols,rows", PRODUCTS)
def test_products_by_blocks(fmt, group, counts, M, cols, rows):
    import torch
    import paper_2605_05888_amd as hub
    print("products", fmt, group, counts, M, cols, rows, flush=True)
    rng = np.random.default_rng(cols + rows + M + group)
    E, seg = 1, None
    if counts is not None:
        E = len(counts)
        seg = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        M = int(seg[-1])
    codes, scales = random_q4(rng, (E, rows, cols), fmt, group)
    x = mi.f32_to_bf16_bits(rng.standard_normal((M, cols)).astype(np.float32))
    y = torch.full((M + 1, rows), 7.0, dtype=torch.bfloat16, device="cuda:0")
    hub.moe_matvec_q4(dev(x), None if seg is None else dev(seg), dev(codes), dev(scales), fmt, group, y[:M])
    got, at = host(y), [0, M] if seg is None else seg
    for e in range(E):
        m = slice(at[e], at[e + 1])
        if at[e] == at[e + 1]:
            continue
        for lo in range(0, rows, 4096):
            r = slice(lo, lo + 4096)
            want, err = ref.product(ref.f64(x)[m], ref.values(codes[e][r], scales[e][r], fmt, group),
                                    few_close.held(codes[e][r], scales[e][r], fmt, group))
            ref.check(got[m, r], want, err + ref.HALF["bf16"] * (np.abs(want) + err), (e, lo))
            few_close.check(got[m, r], want, "bf16", (e, lo))
    assert (ref.f64(got[M]) == 7.0).all()
