"""The operators of decoding with few tokens and with 4-bit expert weights, as timed cases.

A case is one pass of one of four programs:

``layer``
    a whole MoE layer (gating, expert FFN, combine) for a handful of tokens, expert weights in bf16 or fp32.
``layer_q4``
    the same layer with the experts' weights held in 4 bits.
``matvec_q4``
    products of a few rows with 4-bit matrices: one matrix, or the rows of several experts' segments.
``requantize_q4``
    a matrix taken into 4 bits and back: what a program does once per weight when it loads a model, and again
    where a long prefill wants bf16 weights.

4-bit formats: ``fp4`` is a sign, two exponent bits and one mantissa bit under a power-of-two scale for 32
columns; ``int4`` is a whole number from -8 to 7 under a bf16 scale for a group of columns.  Sizes are those of
the workload table in ``moe_inputs``; drawn cases spread over the token counts and over generic shapes.
"""
import math

import torch

own = False

# hidden size, experts, top-K, expert FFN size, score mode, Zipf exponent of the experts' popularity (0: uniform)
SHAPES = {
    "mixtral": (4096, 8, 2, 14336, "softmax", 0.0),
    "gptoss": (2880, 128, 4, 2880, "softmax", 1.0),
    "dsv3": (7168, 256, 8, 2048, "sigmoid", 0.0),
    "qwen2moe": (2048, 64, 4, 1408, "softmax", 0.0),
    "phi35moe": (4096, 16, 2, 6400, "softmax", 0.0),
}


def _layer(N, H, E, K, F, score, zipf, dtype="bf16"):
    return {"kind": "layer", "N": N, "H": H, "E": E, "K": K, "F": F, "score": score, "zipf": zipf, "dtype": dtype}


def _layer_q4(N, H, E, K, F, score, zipf, fmt, group):
    return {"kind": "layer_q4", "N": N, "H": H, "E": E, "K": K, "F": F, "score": score, "zipf": zipf,
            "dtype": "bf16", "fmt": fmt, "group": group}


def _matvec_q4(M, cols, rows, E, fmt, group):
    return {"kind": "matvec_q4", "M": M, "cols": cols, "rows": rows, "E": E, "fmt": fmt, "group": group}


def _requantize_q4(rows, cols, dtype, fmt, group):
    return {"kind": "requantize_q4", "rows": rows, "cols": cols, "dtype": dtype, "fmt": fmt, "group": group}


def listed():
    return [
        # one sequence being decoded: launches and latency
        dict(_layer(1, *SHAPES["qwen2moe"]), name="layer_one_token"),
        # a decoding batch over many experts, most of them with one or two rows: their weights stream
        dict(_layer(16, *SHAPES["dsv3"]), name="layer_batch_16_many_experts"),
        # the largest batch over few large experts, each with about 16 rows
        dict(_layer(64, *SHAPES["mixtral"]), name="layer_batch_64_few_experts"),
        # single precision, odd sizes
        dict(_layer(5, 516, 12, 3, 1028, "softmax", 0.0, "fp32"), name="layer_fp32_odd"),
        # 4-bit weights: one token, a skewed batch, many experts with coarse groups, full rows
        dict(_layer_q4(1, *SHAPES["gptoss"], "fp4", 32), name="layer_fp4_one_token"),
        dict(_layer_q4(37, *SHAPES["gptoss"], "fp4", 32), name="layer_fp4_batch_37"),
        dict(_layer_q4(8, *SHAPES["dsv3"], "int4", 128), name="layer_int4_batch_8_many_experts"),
        dict(_layer_q4(64, *SHAPES["mixtral"], "int4", 64), name="layer_int4_batch_64_few_experts"),
        # a projection of one token beside the experts, and segments of uneven length (some empty) of an
        # expert-parallel rank's received rows
        dict(_matvec_q4(1, 4096, 4096, 1, "fp4", 32), name="matvec_fp4_one_row"),
        dict(_matvec_q4(203, 2880, 5768, 32, "int4", 32), name="matvec_int4_segments"),
        # a large expert's matrix, and a small odd one
        dict(_requantize_q4(14336, 4096, "bf16", "fp4", 32), name="requantize_fp4"),
        dict(_requantize_q4(1001, 1088, "fp32", "int4", 128), name="requantize_int4_fp32_odd"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _format(rng):
    return rng.choice([("fp4", 32), ("fp4", 32), ("int4", 32), ("int4", 64), ("int4", 128)])


def draw(rng):
    kind = rng.choice(["layer", "layer", "layer_q4", "layer_q4", "layer_q4", "matvec_q4", "matvec_q4", "requantize_q4"])
    if kind == "matvec_q4":
        E = rng.choice([1, 1, _log_int(rng, 2, 64)])
        cols, rows = 64 * _log_int(rng, 1, 128), 8 * _log_int(rng, 2, 2048)
        while E * rows * cols > 1 << 31:
            E //= 2
        return _matvec_q4(_log_int(rng, 1, 64 if E == 1 else 512), cols, rows, E, *_format(rng))
    if kind == "requantize_q4":
        fmt, group = _format(rng)
        return _requantize_q4(_log_int(rng, 1, 14336), 64 * _log_int(rng, 1, 64), rng.choice(["bf16", "fp32"]), fmt, group)
    N = _log_int(rng, 1, 64)
    if rng.random() < 0.5:
        H, E, K, F, score, zipf = SHAPES[rng.choice(sorted(SHAPES))]
    else:
        E = _log_int(rng, 4, 256)
        H, F, K = 64 * _log_int(rng, 2, 112), 64 * _log_int(rng, 2, 112), rng.randint(1, min(E, 8))
        score, zipf = rng.choice(["softmax", "sigmoid"]), rng.choice([0.0, 0.0, 1.0])
        while E * H * F > 256 * 7168 * 2048:
            E = max(K, E // 2)
            F = max(64, F // 128 * 64)
    while min(E, N * K) * H * F > 96 * 7168 * 2048: # weights of the experts that get a row
        N -= 1
    if kind == "layer":
        if rng.random() < 0.25 and E * H * F < 1 << 27:
            return _layer(N, H - 4 * rng.randint(0, 8), E, K, F - 4 * rng.randint(0, 8), score, zipf, "fp32")
        return _layer(N, H, E, K, F, score, zipf)
    return _layer_q4(N, H, E, K, F, score, zipf, *_format(rng))


# ---- inputs ----------------------------------------------------------------------------------------------------
def _normal(g, shape, std, dtype):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)


def _popularity_bias(g, E, zipf):
    """Router bias whose logits make the experts' popularity follow Zipf's law: log-popularity at Gumbel scale."""
    rank = torch.randperm(E, generator=g, device="cuda").double() + 1.0
    return (-math.sqrt(6.0) / math.pi * zipf * rank.log()).float()


def _tokens(g, case, W_r, bias, dtype):
    """Normal tokens whose K picks, in their order, stand clear of rounding: two logits that are nearer to each other
    than 32-bit sums of them are exact have no one right order, so such a token is drawn again."""
    N, H, K = case["N"], case["H"], case["K"]
    x = _normal(g, (N, H), 1.0, dtype)
    for _ in range(20):
        logits = x.double() @ W_r.double()
        if bias is not None:
            logits = logits + bias.double()
        top = logits.sort(dim=1, descending=True).values[:, :K + 1]
        near = (top[:, :-1] - top[:, 1:] < 1e-4).any(dim=1)
        if not bool(near.any()):
            break
        x = torch.where(near[:, None], _normal(g, (N, H), 1.0, dtype), x)
    return x


def _bytes(g, shape):
    n = math.prod(shape)
    words = torch.empty((n + 3) // 4, dtype=torch.int32, device="cuda").random_(-2 ** 31, 2 ** 31, generator=g)
    return words.view(torch.uint8)[:n].view(shape)


def _q4(g, shape, std, fmt, group):
    """Codes and scales as quantised normal weights of this deviation have them: fp4 codes come out about equally
    often (rms 2.9), int4 ones heaped around zero (rms 3.3)."""
    *lead, cols = shape
    codes = _bytes(g, (*lead, cols // 2))
    if fmt == "fp4":
        scales = (torch.randint(0, 2, (*lead, cols // 32), generator=g, device="cuda", dtype=torch.uint8)
                  + (126 + round(math.log2(std / 2.9))))
        return codes, scales
    codes = codes.bitwise_and_(0x77).add_(_bytes(g, codes.shape).bitwise_and_(0x77)).add_(_bytes(g, codes.shape).bitwise_and_(0x11))
    scales = torch.empty((*lead, -(-cols // group)), dtype=torch.bfloat16, device="cuda")
    return codes, scales.uniform_(0.7 * std / 3.3, 1.3 * std / 3.3, generator=g)


def _code(case):
    import paper_2605_05888_amd as hub
    return hub.Q4_FP4 if case["fmt"] == "fp4" else hub.Q4_INT4


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = {"case": case}
    if case["kind"] == "requantize_q4":
        rows, cols, group = case["rows"], case["cols"], case["group"]
        dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        s["w"] = _normal(g, (rows, cols), cols ** -0.5, dt)
        s["w"][rows // 2] = 0.0 # a row of zeros, as pruned weights have
        s["codes"] = torch.empty((rows, cols // 2), dtype=torch.uint8, device="cuda")
        s["scales"] = (torch.empty((rows, cols // 32), dtype=torch.uint8, device="cuda") if case["fmt"] == "fp4" else
                       torch.empty((rows, -(-cols // group)), dtype=torch.bfloat16, device="cuda"))
        s["back"] = torch.empty_like(s["w"])
        return s
    if case["kind"] == "matvec_q4":
        M, cols, rows, E = case["M"], case["cols"], case["rows"], case["E"]
        s["codes"], s["scales"] = _q4(g, (E, rows, cols), cols ** -0.5, case["fmt"], case["group"])
        s["x"] = _normal(g, (M, cols), 1.0, torch.bfloat16)
        s["seg"] = None
        if E > 1: # each row goes to an expert by chance, every seventh expert is without any
            to = torch.randint(0, E, (M,), generator=g, device="cuda")
            to = torch.where(to % 7 == 3, (to + 1) % E, to)
            counts = torch.bincount(to, minlength=E)
            s["seg"] = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32)
        s["y"] = torch.empty((M, rows), dtype=torch.bfloat16, device="cuda")
        return s
    N, H, E, K, F = (case[k] for k in "NHEKF")
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    s["W_r"] = _normal(g, (H, E), H ** -0.5, torch.float32)
    s["bias"] = _popularity_bias(g, E, case["zipf"]) if case["zipf"] else None
    s["x"] = _tokens(g, case, s["W_r"], s["bias"], dt)
    if case["kind"] == "layer_q4":
        s["gate"] = _q4(g, (E, F, H), H ** -0.5, case["fmt"], case["group"])
        s["up"] = _q4(g, (E, F, H), H ** -0.5, case["fmt"], case["group"])
        s["down"] = _q4(g, (E, H, F), F ** -0.5, case["fmt"], case["group"])
    else:
        s["gate"] = _normal(g, (E, F, H), H ** -0.5, dt)
        s["up"] = _normal(g, (E, F, H), H ** -0.5, dt)
        s["down"] = _normal(g, (E, H, F), F ** -0.5, dt)
    s["topk_idx"] = torch.empty((N, K), dtype=torch.int32, device="cuda")
    s["topk_w"] = torch.empty((N, K), dtype=torch.float32, device="cuda")
    s["out"] = torch.empty((N, H), dtype=dt, device="cuda")
    return s


# ---- the framework's calls ---------------------------------------------------------------------------------------
def _run_own(s):
    import paper_2605_05888_amd as hub
    case = s["case"]
    if case["kind"] == "requantize_q4":
        hub.moe_quantize_q4(s["w"], _code(case), case["group"], s["codes"], s["scales"])
        hub.moe_dequantize_q4(s["codes"], s["scales"], _code(case), case["group"], s["back"])
        return s["back"]
    if case["kind"] == "matvec_q4":
        hub.moe_matvec_q4(s["x"], s["seg"], s["codes"], s["scales"], _code(case), case["group"], s["y"])
        return s["y"]
    if "ws" not in s: # a program keeps its workspace
        n = hub.workspace_bytes(hub.OP_LAYER_FEW, N=case["N"], H=case["H"], E=case["E"], K=case["K"], F=case["F"],
                                dtype=hub.BF16 if case["dtype"] == "bf16" else hub.F32)
        s["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    score = hub.SCORE_SIGMOID_TOPK if case["score"] == "sigmoid" else hub.SCORE_SOFTMAX_TOPK
    if case["kind"] == "layer_q4":
        hub.moe_layer_few_q4(s["x"], s["W_r"], s["bias"], case["K"], score, s["gate"], s["up"], s["down"], _code(case),
                             case["group"], s["topk_idx"], s["topk_w"], s["out"], s["ws"])
    else:
        hub.moe_layer_few(s["x"], s["W_r"], s["bias"], case["K"], score, s["gate"], s["up"], s["down"], s["topk_idx"],
                          s["topk_w"], s["out"], s["ws"])
    return {"out": s["out"], "topk_idx": s["topk_idx"], "topk_w": s["topk_w"]}


# ---- plain forms: elementary operations in 32 bits ---------------------------------------------------------------
_FP4 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0)


def _two_to(e):
    """2^e in 32 bits for whole numbers e from -126 to 127, exactly."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _values(codes, scales, fmt, group):
    """fp32 values of codes [..., cols / 2] under their scales."""
    both = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2)
    cols = both.shape[-1]
    if fmt == "fp4":
        v = torch.tensor(_FP4, dtype=torch.float32, device=codes.device)[both.int()]
        scale = _two_to(scales.int() - 127)
        group = 32
    else:
        v = both.float() - 8.0
        scale = scales.float()
    return v * scale.repeat_interleave(group, dim=-1)[..., :cols]


def _weights(w, case, picked=None):
    """fp32 matrices of the picked experts, or of all."""
    if case["kind"] == "layer_q4":
        codes, scales = w if picked is None else (w[0][picked], w[1][picked])
        return _values(codes, scales, case["fmt"], case["group"])
    return (w if picked is None else w[picked]).float()


def _route(s):
    """Picks and their weights; in 64 bits, so that the picks are those of the exact logits."""
    case = s["case"]
    logits = s["x"].double() @ s["W_r"].double()
    if s["bias"] is not None:
        logits = logits + s["bias"].double()
    v, idx = torch.sort(logits, dim=1, descending=True, stable=True)
    v, idx = v[:, :case["K"]], idx[:, :case["K"]]
    score = 1.0 / (1.0 + torch.exp(-v)) if case["score"] == "sigmoid" else torch.exp(v - v[:, :1])
    return idx, (score / score.sum(dim=1, keepdim=True)).float()


def _plain_layer(s):
    case = s["case"]
    N, E, K, H = (case[k] for k in "NEKH")
    idx, w = _route(s)
    x = s["x"].float()
    if N * K < E: # the picked experts' matrices, one per row
        e = idx.flatten()
        rows = x.repeat_interleave(K, dim=0).unsqueeze(2)
        gate = torch.bmm(_weights(s["gate"], case, e), rows)
        up = torch.bmm(_weights(s["up"], case, e), rows)
        a = gate / (1.0 + torch.exp(-gate)) * up
        y = torch.bmm(_weights(s["down"], case, e), a).view(N, K, H)
    else: # every expert on every token
        gate = torch.matmul(x, _weights(s["gate"], case).transpose(1, 2))
        up = torch.matmul(x, _weights(s["up"], case).transpose(1, 2))
        a = gate / (1.0 + torch.exp(-gate)) * up
        y = torch.matmul(a, _weights(s["down"], case).transpose(1, 2)) # [E, N, H]
        y = y[idx, torch.arange(N, device=idx.device).unsqueeze(1)]
    out = (y * w.unsqueeze(2)).sum(dim=1).to(s["x"].dtype)
    return {"out": out, "topk_idx": idx.int(), "topk_w": w}


def _plain_matvec(s):
    case = s["case"]
    x = s["x"].float()
    if s["seg"] is None:
        return (x @ _values(s["codes"][0], s["scales"][0], case["fmt"], case["group"]).t()).to(torch.bfloat16)
    m = torch.arange(case["M"], device="cuda")
    e = torch.searchsorted(s["seg"][1:].long(), m, right=True)
    if case["M"] < 2 * case["E"]:
        W = _values(s["codes"][e], s["scales"][e], case["fmt"], case["group"])
        return torch.bmm(W, x.unsqueeze(2)).squeeze(2).to(torch.bfloat16)
    W = _values(s["codes"], s["scales"], case["fmt"], case["group"])
    return torch.matmul(x, W.transpose(1, 2))[e, m].to(torch.bfloat16) # [E, M, rows] -> [M, rows]


def _plain_requantize(s):
    case, w = s["case"], s["w"]
    rows, cols = w.shape
    group = case["group"]
    v = torch.nn.functional.pad(w.float(), (0, -cols % group)).view(rows, -1, group)
    most = v.abs().amax(dim=2, keepdim=True)
    if case["fmt"] == "fp4":
        exponent = ((most.view(torch.int32) >> 23) - 129).clamp(min=-126) # of the largest, less the grid's own 2
        m = v.abs() * _two_to(-exponent)
        m = (0.5 * (m > 0.25) + 0.5 * (m >= 0.75) + 0.5 * (m > 1.25) + 0.5 * (m >= 1.75) + (m > 2.5).float() + (m >= 3.5).float()
             + 2.0 * (m > 5.0))
        back = m * _two_to(exponent) * torch.sign(v)
    else: # quotients next to a border between two codes, in 64 bits
        q, e = torch.frexp(most.double() / 7.0)
        scale = torch.round(q * 256.0) * _two_to(e - 8).double()
        code = torch.round(v.double() / torch.where(scale == 0, torch.ones_like(scale), scale)).clamp(-8, 7)
        back = (code * scale).float()
    return back.reshape(rows, -1)[:, :cols].to(w.dtype)


def run(s):
    if own:
        return _run_own(s)
    kind = s["case"]["kind"]
    return _plain_requantize(s) if kind == "requantize_q4" else _plain_matvec(s) if kind == "matvec_q4" else _plain_layer(s)


# ---- the definition in 64 bits -------------------------------------------------------------------------------------
def _exact_matrix(w, fmt=None, group=0):
    """One matrix in 64 bits; 4-bit ones byte by byte: the low half is the even column."""
    if fmt is None:
        return w.double()
    codes, scales = w
    rows, half = codes.shape
    out = torch.empty((rows, 2 * half), dtype=torch.float64, device=codes.device)
    for part in range(2):
        c = codes.int() // 16 if part else codes.int() % 16
        if fmt == "fp4":
            sign, exponent, mantissa = c // 8, c // 2 % 4, c % 2
            mag = torch.where(exponent == 0, 0.5 * mantissa.double(), (1.0 + 0.5 * mantissa.double()) * (1 << exponent).double() / 2.0)
            out[:, part::2] = torch.where(sign == 1, -mag, mag)
        else:
            out[:, part::2] = c.double() - 8.0
    col = torch.arange(2 * half, device=codes.device)
    if fmt == "fp4":
        return out * ((scales.long() + 896) << 52).view(torch.float64)[:, col // 32]
    return out * scales.double()[:, col // group]


def _exact_layer(s):
    case = s["case"]
    fmt, group = case.get("fmt"), case.get("group", 0)
    of = (lambda w, e: _exact_matrix((w[0][e], w[1][e]), fmt, group)) if fmt else (lambda w, e: _exact_matrix(w[e]))
    N, E, K = case["N"], case["E"], case["K"]
    x = s["x"].double()
    logits = x.matmul(s["W_r"].double())
    if s["bias"] is not None:
        logits += s["bias"].double()
    # an expert's rank is the number of experts that go before it
    e = torch.arange(E, device="cuda")
    before = (logits.unsqueeze(1) > logits.unsqueeze(2)) | ((logits.unsqueeze(1) == logits.unsqueeze(2)) & (e < e.unsqueeze(1)))
    rank = before.sum(dim=2)
    idx = torch.empty((N, K), dtype=torch.int64, device="cuda")
    n_of, e_of = (rank < K).nonzero(as_tuple=True)
    idx[n_of, rank[n_of, e_of]] = e_of
    picked = logits.gather(1, idx)
    score = torch.sigmoid(picked) if case["score"] == "sigmoid" else torch.exp(picked - picked.max(dim=1, keepdim=True).values)
    w = score / score.sum(dim=1, keepdim=True)
    out = torch.zeros_like(x)
    for expert in idx.unique().tolist():
        n, k = (idx == expert).nonzero(as_tuple=True)
        rows = x[n]
        gate, up = rows @ of(s["gate"], expert).t(), rows @ of(s["up"], expert).t()
        y = (gate * torch.sigmoid(gate) * up) @ of(s["down"], expert).t()
        out[n] += y * w[n, k].unsqueeze(1)
    return {"out": out, "topk_idx": idx.int(), "topk_w": w}


def _unit(v):
    """The largest power of two that is not above v, in 64 bits; 1 for zeros."""
    return ((torch.where(v > 0, v, torch.ones_like(v)).view(torch.int64) >> 52) << 52).view(torch.float64)


def _exact_requantize(s):
    case, w = s["case"], s["w"].double()
    rows, cols = w.shape
    back = torch.zeros_like(w)
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device="cuda")
    for c in range(0, cols, case["group"]):
        part = w[:, c:c + case["group"]]
        most = part.abs().max(dim=1, keepdim=True).values
        if case["fmt"] == "fp4":
            scale = _unit(most) / 4.0
            m = (part.abs() / scale).clamp(max=6.0)
            far = (m.unsqueeze(2) - grid).abs()
            near = far.min(dim=2, keepdim=True).values
            # of two grid values equally near, the one with an even place
            place = torch.where(far == near, torch.arange(8, device="cuda"), 8)
            low, high = place.min(dim=2).values, torch.where(far == near, torch.arange(8, device="cuda"), -1).max(dim=2).values
            back[:, c:c + case["group"]] = grid[torch.where(low % 2 == 0, low, high)] * scale * torch.sign(part)
        else:
            unit = _unit(most / 7.0) / 128.0
            scale = torch.round(most / 7.0 / unit) * unit
            q = torch.where(scale > 0, part / scale, torch.zeros_like(part))
            back[:, c:c + case["group"]] = torch.round(q).clamp(-8.0, 7.0) * scale
    return back


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "requantize_q4":
        return _exact_requantize(s)
    if case["kind"] == "matvec_q4":
        x = s["x"].double()
        y = torch.zeros((case["M"], case["rows"]), dtype=torch.float64, device="cuda")
        seg = [0, case["M"]] if s["seg"] is None else s["seg"].tolist()
        for e in range(case["E"]):
            if seg[e + 1] > seg[e]:
                W = _exact_matrix((s["codes"][e], s["scales"][e]), case["fmt"], case["group"])
                y[seg[e]:seg[e + 1]] = x[seg[e]:seg[e + 1]] @ W.t()
        return y
    return _exact_layer(s)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------
def _bytes_per_weight(case):
    if "fmt" not in case:
        return 2.0 if case["dtype"] == "bf16" else 4.0
    return 0.5 + (1.0 / 32 if case["fmt"] == "fp4" else 2.0 / case["group"])


def _touched(case):
    """Expected number of experts that get at least one row."""
    E, N, K = case["E"], case["N"], case["K"]
    if not case["zipf"]:
        return E * (1.0 - (1.0 - K / E) ** N)
    g = torch.Generator()
    g.manual_seed(0)
    rank = torch.arange(1, E + 1, dtype=torch.float64)
    z = torch.randn((4096, E), generator=g, dtype=torch.float64) - math.sqrt(6.0) / math.pi * case["zipf"] * rank.log()
    share = torch.bincount(z.topk(K, dim=1).indices.flatten(), minlength=E) / 4096.0
    return float((1.0 - (1.0 - share) ** N).sum())


def work(case):
    if case["kind"] == "requantize_q4":
        w = 2 if case["dtype"] == "bf16" else 4
        n = case["rows"] * case["cols"]
        return {"bytes": n * (2 * w + 2 * _bytes_per_weight(case)), "flops": 4 * n}
    if case["kind"] == "matvec_q4":
        M, cols, rows, E = case["M"], case["cols"], case["rows"], case["E"]
        full = 1.0
        if E > 1: # share of the experts that get a row
            able = E - len(range(3, E, 7))
            full = able / E * (1.0 - (1.0 - 1.0 / able) ** M)
        return {"bytes": E * full * rows * cols * _bytes_per_weight(case) + 2 * M * (cols + rows), "flops": 2 * M * cols * rows}
    N, H, E, K, F = (case[k] for k in "NHEKF")
    b = 2 if case["dtype"] == "bf16" else 4
    nbytes = 4 * H * E + 2 * N * H * b + 8 * N * K + _touched(case) * 3 * H * F * _bytes_per_weight(case)
    return {"bytes": nbytes, "flops": 2 * N * H * E + 6 * N * K * H * F}
