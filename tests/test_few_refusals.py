"""The decoding operators (moe_few.h) without a GPU: symbols, workspace sizes, refusals before anything is launched."""
import ctypes
import os
import re

import pytest

import paper_2605_05888_amd as hub

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 0x1000  # a fake, well-aligned, never-dereferenced pointer: every case below fails validation first
BIG = 1 << 30


def test_every_declared_function_is_exported_and_bound():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "moe_few.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(moe_[a-z0-9_]+)\s*\(", text))
    assert names == {"moe_layer_few", "moe_layer_few_q4", "moe_matvec_q4", "moe_quantize_q4", "moe_dequantize_q4"}
    lib = hub.load_library()
    assert names == set(hub.exported_few_symbols())
    for n in names:
        assert hasattr(lib, n) and hasattr(hub, n), n


def test_headers_compile_as_c(tmp_path):
    import subprocess
    src = tmp_path / "t.c"
    src.write_text('#include "moe_few.h"\nint main(void) { return MOE_Q4_FP4 + (MOE_FEW_TOKENS != %d); }\n' % hub.FEW_TOKENS)
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-c", str(src), "-o",
                    str(tmp_path / "t.o")], check=True)


def test_workspace_sizes():
    n = hub.workspace_bytes(hub.OP_LAYER_FEW, N=64, H=4096, E=8, K=2, F=14336, dtype=hub.BF16)
    assert 64 * 2 * 14336 * 2 <= n < 16 << 20
    assert hub.workspace_bytes(hub.OP_LAYER_FEW, N=5, H=516, E=12, K=3, F=1028, dtype=hub.F32) >= 15 * 1028 * 4
    good = dict(N=4, H=64, E=8, K=2, F=64, dtype=hub.BF16)
    assert hub.workspace_bytes(hub.OP_LAYER_FEW, **good) > 0
    for bad in (dict(N=-1), dict(N=65), dict(H=0), dict(F=0), dict(H=1 << 21), dict(E=0), dict(E=2048), dict(K=0), dict(K=33),
                dict(dtype=7)):
        assert hub.workspace_bytes(hub.OP_LAYER_FEW, **{**good, **bad}) == 0, bad


def few(x=A, dtype=hub.BF16, N=4, H=64, W_r=A, bias=None, E=8, K=2, mode=0, F=64, wg=A, wu=A, wd=A, idx=A, w=A, out=A, ws=A,
        ws_bytes=BIG):
    return hub.load_library().moe_layer_few(x, dtype, N, H, W_r, bias, E, K, mode, F, wg, wu, wd, idx, w, out, ws, ws_bytes, None)


def few_q4(x=A, dtype=hub.BF16, N=4, H=64, W_r=A, bias=None, E=8, K=2, mode=0, F=64, fmt=hub.Q4_FP4, group=32, gc=A, gs=A, uc=A,
           us=A, dc=A, ds=A, idx=A, w=A, out=A, ws=A, ws_bytes=BIG):
    return hub.load_library().moe_layer_few_q4(x, dtype, N, H, W_r, bias, E, K, mode, F, fmt, group, gc, gs, uc, us, dc, ds, idx,
                                               w, out, ws, ws_bytes, None)


def matvec(x=A, dtype=hub.BF16, M=4, cols=64, rows=64, E=2, seg=A, fmt=hub.Q4_FP4, group=32, codes=A, scales=A, y=A):
    return hub.load_library().moe_matvec_q4(x, dtype, M, cols, rows, E, seg, fmt, group, codes, scales, y, None)


def quantize(w=A, dtype=hub.BF16, rows=4, cols=64, fmt=hub.Q4_FP4, group=32, codes=A, scales=A):
    return hub.load_library().moe_quantize_q4(w, dtype, rows, cols, fmt, group, codes, scales, None)


def dequantize(w=A, dtype=hub.BF16, rows=4, cols=64, fmt=hub.Q4_FP4, group=32, codes=A, scales=A):
    return hub.load_library().moe_dequantize_q4(codes, scales, fmt, group, rows, cols, w, dtype, None)


LAYER = [
    (dict(dtype=5), -2, "dtype"), (dict(N=-1), -1, "N"), (dict(N=65), -2, "MOE_FEW_TOKENS"), (dict(K=0), -1, "K"),
    (dict(K=9), -1, "K"), (dict(E=64, K=33), -2, "MOE_MAX_TOPK"), (dict(E=1025), -2, "MOE_MAX_EXPERTS"), (dict(E=0, K=0), -1, "E"),
    (dict(mode=2), -1, "score_mode"), (dict(H=0), -1, "H"), (dict(H=60), -1, "16"), (dict(H=96), -2, "multiples of 64"),
    (dict(F=96), -2, "multiples of 64"), (dict(F=0), -1, "F"), (dict(H=1 << 21), -2, "2^21"), (dict(F=1 << 21), -2, "2^21"),
    (dict(x=None), -1, "NULL"), (dict(x=A + 8), -1, "aligned"), (dict(W_r=None), -1, "NULL"), (dict(bias=A + 4), -1, "aligned"),
    (dict(idx=None), -1, "NULL"), (dict(w=None), -1, "NULL"), (dict(out=None), -1, "NULL"), (dict(out=A + 2), -1, "aligned"),
    (dict(ws=None), -3, "workspace"), (dict(ws_bytes=100), -3, "workspace"), (dict(ws=A + 16), -1, "128-byte"),
]


@pytest.mark.parametrize("change,code,word", LAYER + [
    (dict(wg=None), -1, "NULL"), (dict(wu=A + 1), -1, "aligned"), (dict(wd=None), -1, "NULL"),
    (dict(dtype=hub.F32, H=6), -1, "16"), (dict(dtype=hub.F32, F=6), -1, "16")])
def test_layer_few_refuses(change, code, word):
    assert few(**change) == code
    assert word in hub.last_error()


@pytest.mark.parametrize("change,code,word", LAYER + [
    (dict(dtype=hub.F32), -2, "BF16"), (dict(fmt=2), -1, "format"), (dict(group=16), -2, "group"), (dict(group=64), -2, "group"),
    (dict(fmt=hub.Q4_INT4, group=256), -2, "group"), (dict(gc=None), -1, "NULL"), (dict(gs=None), -1, "NULL"),
    (dict(uc=None), -1, "NULL"), (dict(us=A + 1), -1, "aligned"), (dict(dc=A + 8), -1, "aligned"), (dict(ds=None), -1, "NULL")])
def test_layer_few_q4_refuses(change, code, word):
    assert few_q4(**change) == code
    assert word in hub.last_error()


@pytest.mark.parametrize("change,code,word", [
    (dict(dtype=5), -2, "dtype"), (dict(dtype=hub.F32), -2, "BF16"), (dict(M=-1), -1, "M"), (dict(M=1 << 31), -1, "M"),
    (dict(cols=0), -1, "cols"), (dict(cols=96), -2, "multiple of 64"), (dict(cols=1 << 21), -1, "cols"), (dict(rows=0), -1, "rows"),
    (dict(rows=4), -1, "16"), (dict(rows=1 << 27), -1, "rows"), (dict(E=0), -1, "E_local"), (dict(E=65536), -1, "E_local"),
    (dict(seg=None), -1, "seg_offsets"), (dict(fmt=-1), -1, "format"), (dict(group=128), -2, "group"), (dict(x=None), -1, "NULL"),
    (dict(codes=None), -1, "NULL"), (dict(scales=A + 2), -1, "aligned"), (dict(y=None), -1, "NULL")])
def test_matvec_q4_refuses(change, code, word):
    assert matvec(**change) == code
    assert word in hub.last_error()


@pytest.mark.parametrize("call", [quantize, dequantize])
@pytest.mark.parametrize("change,code,word", [
    (dict(dtype=5), -2, "dtype"), (dict(rows=-1), -1, "rows"), (dict(rows=1 << 30), -1, "2^36"), (dict(cols=0), -1, "cols"),
    (dict(cols=32), -2, "multiple of 64"), (dict(fmt=3), -1, "format"), (dict(group=64), -2, "group"), (dict(w=None), -1, "NULL"),
    (dict(codes=A + 4), -1, "aligned"), (dict(scales=None), -1, "NULL")])
def test_conversions_refuse(call, change, code, word):
    assert call(**change) == code
    assert word in hub.last_error()


def test_empty_inputs_are_successful_noops():
    assert few(N=0, x=None, wg=None, out=None, ws=None, ws_bytes=0) == 0
    assert few_q4(N=0, x=None, gc=None, out=None, ws=None, ws_bytes=0) == 0
    assert matvec(M=0, x=None, seg=None, y=None) == 0
    assert quantize(rows=0, w=None, codes=None) == 0 and dequantize(rows=0, w=None, codes=None) == 0
    assert hub.last_error() == ""


def test_the_binding_refuses_host_tensors_and_wrong_shapes():
    import torch
    x = torch.zeros((2, 64), dtype=torch.bfloat16)
    c, s = torch.zeros((1, 64, 32), dtype=torch.uint8), torch.zeros((1, 64, 2), dtype=torch.uint8)
    with pytest.raises(TypeError, match="device tensor"):
        hub.moe_matvec_q4(x, None, c, s, hub.Q4_FP4, 32, torch.zeros_like(x))
    with pytest.raises(TypeError, match="matrix"):
        hub.moe_matvec_q4(x[0], None, c, s, hub.Q4_FP4, 32, x)
    with pytest.raises(TypeError, match="device tensor"):
        hub.moe_quantize_q4(x, hub.Q4_FP4, 32, c[0, :2], s[0, :2])
    with pytest.raises(TypeError, match="matrix"):
        hub.moe_dequantize_q4(c[0, 0], s[0, 0], hub.Q4_FP4, 32, x[0])
    idx, w = torch.zeros((2, 1), dtype=torch.int32), torch.zeros((2, 1))
    with pytest.raises(TypeError, match="device tensor"):
        hub.moe_layer_few(x, torch.zeros((64, 4)), None, 1, 0, c, c, c, idx, w, x, None)
    with pytest.raises(TypeError, match="dtype"):
        hub.moe_layer_few(x.half(), torch.zeros((64, 4)), None, 1, 0, c, c, c, idx, w, x, None)
