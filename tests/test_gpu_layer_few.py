"""The whole layer for a few tokens against a 64-bit reference, and its routing against moe_route, bit for bit."""
import numpy as np
import pytest

import few_reference as ref
import moe_inputs as mi
import oracle
from test_gpu_q4 import FORMATS, dev, host, random_q4

pytestmark = pytest.mark.gpu

SOFT, SIGM = oracle.SOFTMAX_TOPK, oracle.SIGMOID_TOPK


class Layer:
    """Inputs on both sides; form: "bf16", "f32", or (format, group)."""

    def __init__(self, form, N, H, E, K, F, mode=SOFT, bias=None, seed=0, x=None, W_r=None):
        rng = np.random.default_rng([seed, N, H, E, K, F])
        self.form, self.N, self.H, self.E, self.K, self.F, self.mode = form, N, H, E, K, F, mode
        self.dtype = "f32" if form == "f32" else "bf16"
        x = rng.standard_normal((N, H)).astype(np.float32) if x is None else x.astype(np.float32)
        self.x = x if form == "f32" else mi.f32_to_bf16_bits(x)
        self.W_r = (rng.standard_normal((H, E)) * H ** -0.5).astype(np.float32) if W_r is None else W_r
        self.bias = None if bias is None else np.asarray(bias, np.float32)
        if isinstance(form, tuple):
            self.w = [random_q4(rng, s, *form) for s in ((E, F, H), (E, F, H), (E, H, F))]
        else:
            w = [(rng.standard_normal(s) * s[2] ** -0.5).astype(np.float32) for s in ((E, F, H), (E, F, H), (E, H, F))]
            self.w = w if form == "f32" else [mi.f32_to_bf16_bits(a) for a in w]
        self.on_device()

    def on_device(self):
        import torch
        import paper_2605_05888_amd as hub
        self.d = dict(x=dev(self.x), W_r=dev(self.W_r), bias=None if self.bias is None else dev(self.bias),
                      w=[tuple(dev(a) for a in p) if isinstance(p, tuple) else dev(p) for p in self.w])
        n = hub.workspace_bytes(hub.OP_LAYER_FEW, N=self.N, H=self.H, E=self.E, K=self.K, F=self.F,
                                dtype=hub.F32 if self.form == "f32" else hub.BF16)
        self.ws = torch.full((n + 64,), 0xFF, dtype=torch.uint8, device="cuda:0")
        self.idx = torch.full((self.N + 1, self.K), -7, dtype=torch.int32, device="cuda:0")
        self.wt = torch.full((self.N + 1, self.K), -7.0, dtype=torch.float32, device="cuda:0")
        self.out = torch.full((self.N + 1, self.H), -7.0, dtype=self.d["x"].dtype, device="cuda:0")

    def call(self, ws=None, out=None):
        import paper_2605_05888_amd as hub
        ws = self.ws[:-64] if ws is None else ws
        out = self.out[:self.N] if out is None else out
        args = (self.d["x"], self.d["W_r"], self.d["bias"], self.K, self.mode, *self.d["w"])
        tail = (self.idx[:self.N], self.wt[:self.N], out, ws)
        if isinstance(self.form, tuple):
            hub.moe_layer_few_q4(*args, *self.form, *tail)
        else:
            hub.moe_layer_few(*args, *tail)
        return out

    def matrix(self, which):
        w = self.w[which]
        if isinstance(self.form, tuple):
            return lambda e: (ref.values(w[0][e], w[1][e], *self.form), ref.most(w[0][e], w[1][e], *self.form))
        return lambda e: (ref.f64(w[e]), np.abs(ref.f64(w[e])))

    def check(self):
        import torch
        import paper_2605_05888_amd as hub
        self.call()
        torch.cuda.synchronize()
        idx, wt, lg = oracle.route(self.x, self.W_r, self.bias, self.K, self.mode)
        assert np.array_equal(host(self.idx[:self.N]), idx)
        # moe_route's own weights, bit for bit
        i2, w2 = torch.empty_like(self.idx[:self.N]), torch.empty_like(self.wt[:self.N])
        ws = torch.empty(self.N * self.E * 4 + 16, dtype=torch.uint8, device="cuda:0")
        hub.moe_route(self.d["x"], self.d["W_r"], self.d["bias"], self.K, self.mode, i2, w2, None, ws)
        assert torch.equal(i2, self.idx[:self.N])
        assert torch.equal(w2.view(torch.int32), self.wt[:self.N].view(torch.int32))
        want, bound = ref.layer(ref.f64(self.x), idx, ref.f64(host(w2)), *[self.matrix(i) for i in range(3)], self.dtype)
        ref.check(host(self.out[:self.N]), want, bound, "out")
        # nothing behind the outputs or the workspace is touched
        assert bool((self.out[self.N] == -7).all() and (self.idx[self.N] == -7).all() and (self.wt[self.N] == -7).all())
        assert bool((self.ws[-64:] == 0xFF).all())


FORMS = ["bf16", "f32", *FORMATS]
SHAPES = [
    # N, H, E, K, F, mode, bias
    (1, 64, 1, 1, 64, SOFT, False), (1, 2048, 64, 4, 1408, SOFT, False), (2, 128, 8, 2, 256, SOFT, True),
    (3, 320, 12, 3, 192, SIGM, False), (5, 576, 40, 5, 128, SIGM, True), (16, 448, 256, 8, 64, SIGM, True),
    (17, 128, 16, 16, 192, SOFT, False), (33, 64, 100, 7, 320, SOFT, True), (64, 256, 4, 2, 448, SOFT, False),
    (64, 128, 3, 1, 128, SOFT, False), (64, 64, 1024, 32, 64, SIGM, False), (48, 192, 17, 3, 64, SOFT, True),
    (8, 7168, 9, 2, 64, SOFT, False), (4, 64, 6, 2, 8192, SOFT, False),
]


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("N,H,E,K,F,mode,bias", SHAPES)
def test_layer(form, N, H, E, K, F, mode, bias):
    print("layer", form, N, H, E, K, F, mode, bias, flush=True)
    b = np.random.default_rng(E).standard_normal(E) if bias else None
    Layer(form, N, H, E, K, F, mode, b).check()


@pytest.mark.parametrize("N,H,E,K,F", [(1, 4, 2, 1, 4), (3, 12, 5, 2, 20), (5, 516, 12, 3, 1028), (20, 36, 3, 3, 68), (64, 100, 7, 2, 132)])
def test_layer_fp32_odd_sizes(N, H, E, K, F):
    print("layer f32", N, H, E, K, F, flush=True)
    Layer("f32", N, H, E, K, F).check()


@pytest.mark.parametrize("form", ["bf16", "f32", (ref.FP4, 32), (ref.INT4, 64)])
def test_routing_where_it_can_go_wrong(form):
    """Equal logits, masked experts, one expert for all, overflowed logits."""
    rng = np.random.default_rng(3)
    H, E, K, F = 128, 24, 3, 64
    print("ties", flush=True)
    Layer(form, 7, H, E, K, F, W_r=np.zeros((H, E), np.float32)).check()
    Layer(form, 7, H, E, K, F, SIGM, x=rng.integers(-2, 3, (7, H)), W_r=rng.integers(-1, 2, (H, E)).astype(np.float32)).check()
    print("masked", flush=True)
    b = np.full(E, -np.inf)
    b[[3, 11, 19, 20]] = [0.5, -0.5, 1.0, 0.0]
    Layer(form, 18, H, E, K, F, bias=b).check()
    b = rng.standard_normal(E)
    b[::2] = -3.4e38
    Layer(form, 5, H, E, K, F, SIGM, bias=b).check()
    print("one expert", flush=True)
    b = np.zeros(E)
    b[9] = 100.0
    Layer(form, 64, H, E, 1, F, bias=b).check()
    Layer(form, 64, H, E, 2, F, SIGM, bias=b).check()


def test_masked_experts_beyond_the_picks_and_overflow_keep_the_picks_distinct():
    """Fewer experts than K left by the mask: the picks are still K distinct experts, as moe_route's are."""
    import torch
    import paper_2605_05888_amd as hub
    for bias in (np.r_[np.full(10, -np.inf), 0.25, 0.5], np.full(12, -np.inf), np.r_[np.nan, np.zeros(11)]):
        t = Layer("bf16", 9, 128, 12, 4, 64, bias=bias)
        t.call()
        i2, w2 = torch.empty_like(t.idx[:9]), torch.empty_like(t.wt[:9])
        hub.moe_route(t.d["x"], t.d["W_r"], t.d["bias"], 4, SOFT, i2, w2, None, torch.empty(9 * 12 * 4, dtype=torch.uint8, device="cuda:0"))
        assert torch.equal(i2, t.idx[:9]) and torch.equal(w2.view(torch.int32), t.wt[:9].view(torch.int32))
        assert all(len(set(r)) == 4 for r in host(i2).tolist())


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("N,K", [(2, 1), (9, 4), (40, 3)])
def test_what_is_not_finite_in_a_row_of_down_stays_in_its_column(form, N, K):
    """Weights (4 bits: scales) of some rows are infinite, NaN or of the largest size: the other columns keep their bits, also
    where a row ends inside a cache line and the next one begins there."""
    import torch
    H, F = (132, 100) if form == "f32" else (192, 320)
    t = Layer(form, N, H, 6, K, F)
    want = t.call().clone()
    rows = [0, 5, 21, 64, 65, 101, H - 1]
    bad = (0x7F80, 0x7FC0, 0xFF80, 0x7F7F)
    codes = t.w[2][0] if isinstance(form, tuple) else t.w[2]
    scales = t.w[2][1] if isinstance(form, tuple) else None
    for j, r in enumerate(rows):
        if form == "f32":
            codes[:, r] = (np.inf, np.nan, -np.inf, 3.4e38)[j % 4]
        elif form == "bf16":
            codes[:, r] = bad[j % 4]
        elif form[0] == ref.FP4:
            codes[:, r], scales[:, r] = 0x77, 254
        else:
            scales[:, r] = bad[j % 4]
    t.on_device()
    got = t.call()
    rest = [h for h in range(H) if h not in rows]
    assert bool(torch.isfinite(got[:, rest].float()).all())
    assert torch.equal(got[:, rest], want[:, rest])
    assert not bool(torch.isfinite(got[:, rows[:3]].float()).any())


@pytest.mark.parametrize("form", FORMS)
def test_equal_calls_give_equal_bits_whatever_the_workspace_held(form):
    import torch
    t = Layer(form, 21, 512, 32, 4, 384, SOFT)
    first = t.call().clone()
    for fill in (0, 0x3F, 0xFF):
        t.ws.fill_(fill)
        t.out.fill_(0)
        assert torch.equal(t.call(), first), fill


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("N", [3, 21, 64])
def test_shares_that_others_take_over_give_the_same_bits(form, N, monkeypatch):
    """Without patience every workgroup does itself what it finds missing, beside the owner: the same values, twice."""
    import torch
    t = Layer(form, N, 192, 12, 3, 256, SOFT)
    first = t.call().clone()
    routed = t.idx.clone(), t.wt.clone()
    monkeypatch.setenv("MOE_FEW_PATIENCE", "0")
    for _ in range(3):
        t.ws.fill_(0xFF)
        t.out.fill_(0)
        t.idx[:N] = -1
        again = t.call()
        torch.cuda.synchronize()
        assert torch.equal(first.view(torch.uint8), again.view(torch.uint8))
        assert torch.equal(routed[0], t.idx) and torch.equal(routed[1], t.wt)


@pytest.mark.parametrize("form", ["bf16", "f32", (ref.FP4, 32), (ref.INT4, 64)])
@pytest.mark.parametrize("N,E,K", [(1, 4, 2), (12, 8, 2), (64, 8, 2)])
def test_calls_that_follow_each_other_on_one_workspace(form, N, E, K):
    """Other tokens meet the same weights in the same workspace, without a wait between the calls: nothing of an earlier
    call's activation, read by another part of the chip, is seen."""
    import torch
    t = Layer(form, N, 1024, E, K, 512)
    xs = [t.d["x"]] + [torch.randn_like(t.d["x"]) for _ in range(2)]
    want = []
    for x in xs:
        t.d["x"] = x
        want.append(t.call(ws=torch.zeros_like(t.ws[:-64]), out=torch.empty_like(t.out[:N])))
    torch.cuda.synchronize()
    got = []
    for turn in range(30):
        t.d["x"] = xs[turn * turn % 3 if turn % 5 else 2]
        got.append((turn * turn % 3 if turn % 5 else 2, t.call(out=torch.empty_like(t.out[:N]))))
    torch.cuda.synchronize()
    for which, out in got:
        assert torch.equal(out.view(torch.uint8), want[which].view(torch.uint8))


@pytest.mark.parametrize("form", ["bf16", (ref.FP4, 32)])
def test_two_graphs_that_share_a_workspace(form):
    """Captured, replayed several times with eager work between; each replay takes what x holds then."""
    import torch
    a, b = Layer(form, 3, 512, 16, 2, 256, seed=1), Layer(form, 40, 512, 16, 2, 256, seed=2)
    ws = b.ws[:-64]
    want = [t.call(ws).clone() for t in (a, b)]
    graphs = []
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for t in (a, b):
            t.call(ws)
    torch.cuda.synchronize()
    for t in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            t.call(ws)
        graphs.append(g)
    for turn in range(4):
        for t, g, w in zip((a, b), graphs, want):
            t.out.fill_(0)
            g.replay()
            assert torch.equal(t.out[:t.N], w), turn
        ws.fill_(turn * 17)
        torch.cuda.synchronize()
    x = a.d["x"].clone()
    a.d["x"].copy_(x.flip(0))
    graphs[0].replay()
    assert torch.equal(a.out[:3], want[0].flip(0))
    a.d["x"].copy_(x)


@pytest.mark.parametrize("form", ["bf16", "f32", (ref.FP4, 32), (ref.INT4, 128)])
def test_calls_on_several_streams_at_once(form):
    import torch
    layers = [Layer(form, n, 1024, 32, 4, 512, seed=n) for n in (1, 9, 30, 64)]
    want = [t.call().clone() for t in layers]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in layers]
    for turn in range(6):
        for t in layers:
            t.out.fill_(0)
        torch.cuda.synchronize()
        for t, st in zip(layers, streams):
            with torch.cuda.stream(st):
                for _ in range(5):
                    t.call()
        torch.cuda.synchronize()
        for t, w in zip(layers, want):
            assert torch.equal(t.out[:t.N], w), (turn, t.N)


def test_decoding_with_quantised_experts_as_a_program_does():
    """Weights quantised when the model is loaded; prefill with the library's bf16 path on the weights taken back, then
    single tokens with the 4-bit layer: both compute with the same weights, so they agree within bf16's rounding."""
    import torch
    import gpu_layer as G
    import paper_2605_05888_amd as hub
    rng = np.random.default_rng(11)
    N, H, E, K, F = 70, 256, 16, 2, 192
    x = dev(mi.f32_to_bf16_bits(rng.standard_normal((N, H)).astype(np.float32)))
    W_r = dev((rng.standard_normal((H, E)) * H ** -0.5).astype(np.float32))
    for fmt, group in FORMATS:
        packed, back = [], []
        for s in ((E, F, H), (E, F, H), (E, H, F)):
            w = dev(mi.f32_to_bf16_bits((rng.standard_normal(s) * s[2] ** -0.5).astype(np.float32)))
            codes = torch.empty((*s[:2], s[2] // 2), dtype=torch.uint8, device="cuda:0")
            n = -(-s[2] // group)
            scales = torch.empty((*s[:2], n), dtype=torch.uint8 if fmt == ref.FP4 else torch.bfloat16, device="cuda:0")
            hub.moe_quantize_q4(w, fmt, group, codes, scales)
            hub.moe_dequantize_q4(codes, scales, fmt, group, w)
            packed.append((codes, scales))
            back.append(w)
        idx, wt, _ = G.gpu_route(x, W_r, None, K, SOFT)
        lay = G.gpu_layout(idx, E, 1)
        y = G.gpu_ffn(G.gpu_permute(x, K, lay), lay["expert_offsets"], *back)
        prefill = G.gpu_combine(y, K, lay["slot_of_row"], wt)
        out = torch.empty_like(x)
        for n0, n1 in [(0, 1), (1, 2), (2, 6), (6, 70)]:
            ws = torch.empty(hub.workspace_bytes(hub.OP_LAYER_FEW, N=n1 - n0, H=H, E=E, K=K, F=F), dtype=torch.uint8, device="cuda:0")
            i2 = torch.empty((n1 - n0, K), dtype=torch.int32, device="cuda:0")
            w2 = torch.empty((n1 - n0, K), dtype=torch.float32, device="cuda:0")
            hub.moe_layer_few_q4(x[n0:n1], W_r, None, K, SOFT, *packed, fmt, group, i2, w2, out[n0:n1], ws)
            assert torch.equal(i2, idx[n0:n1]) and torch.equal(w2, wt[n0:n1])
        # 2^-8 each for a, y and out in the one, a and out in the other (relative to the largest row term); INT4 weights
        # are rounded once more on the way back to bf16: three products
        d, p = (out.double() - prefill.double()).norm(), prefill.double().norm()
        assert float(d / p) < (5 + (3 if fmt == ref.INT4 else 0)) * 2.0 ** -8
