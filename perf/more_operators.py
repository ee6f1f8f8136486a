"""The 8-bit layer's performance cases: activations in 8 bits a token, and their product with 8-bit weights.

Where a layer's weights are held in 8 bits with a scale for each output channel, its inputs can be held in 8 bits with a scale for each
token, and the projections are products of whole numbers.  A layer then needs, each an operator here ("op"):

  norm     rtn_norm_rows: the residual's addition and the root-mean-square norm, in 16 bits or quantised, before qkv and gate_up
  gated    rtn_gated_rows: the activation of the gate times the other half, in 16 bits or quantised, before down
  rows     rtn_quantize_rows: what attention gives, quantised, before o
  linear   rtn_linear_w8a8: the projections

Layers are those of bench.py (hidden sizes 4096, 8192, 16384; feed-forward widths 14336, 28672, 53248) and generic ones of other sizes.
Quantised rows are returned as the values that they stand for, in the input's type, beside their scales.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}

# What a drawn case may cost at most: the largest listed ones (the prompts through gate_up, the 405b decode step).
MOST_FLOPS = 1.93e12
MOST_BYTES = 1.76e9


def _norm(name, **kw):
    return {"name": name, "op": "norm", "type": "fp16", "rows": 16, "dim": 4096, "residual": True, "bits": 8, "pad": 0, **kw}


def _gated(name, **kw):
    return {"name": name, "op": "gated", "type": "fp16", "rows": 16, "dim": 14336, "activation": "silu", "bits": 8, "pad": 0, **kw}


def _rows(name, **kw):
    return {"name": name, "op": "rows", "type": "fp16", "rows": 16, "dim": 4096, "pad": 0, **kw}


def _linear(name, **kw):
    return {"name": name, "op": "linear", "type": "fp16", "rows": 1, "out": 4096, "dim": 4096, **kw}


def listed():
    return [
        # a decode step of 16 sequences of the 8b layer
        _norm("norm_decode_8b_16"),
        # prompts of an odd number of tokens through a norm whose reader wants 16 bits, rows that are part of wider ones
        _norm("norm_d5120_1897_16bit", type="bf16", rows=1897, dim=5120, residual=False, bits=16, pad=64),
        # the prompts of the 70b layer
        _norm("norm_prefill_70b", rows=8192, dim=8192),
        # verification of five drafted tokens in the 8b layer
        _gated("gated_verify_8b_5", rows=5),
        # the prompts of the 70b layer
        _gated("gated_prefill_70b", type="bf16", rows=4096, dim=28672),
        # attention's output in a decode step of a batch of 64 of the 70b layer, and over prompts in the 405b layer
        _rows("rows_decode_70b_64", rows=64, dim=8192),
        _rows("rows_prefill_405b_3001", type="bf16", rows=3001, dim=16384),
        # the smallest call: one token through the 8b layer's qkv
        _linear("linear_8b_qkv_1", out=6144),
        # eight tokens through the largest matrix
        _linear("linear_405b_gate_up_8", rows=8, out=106496, dim=16384),
        # a decode batch of 64 through a matrix that is long along the sums
        _linear("linear_70b_down_64", type="bf16", rows=64, out=8192, dim=28672),
        # a short ragged prompt batch through the smallest matrix
        _linear("linear_8b_o_217", rows=217),
        # prompts through the 8b layer's widest matrix
        _linear("linear_8b_gate_up_8192", type="bf16", rows=8192, out=28672),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["norm", "norm", "gated", "rows", "linear", "linear", "linear", "linear"])
        kw = {"type": rng.choice(["fp16", "bf16"]), "rows": _log_int(rng, 1, 8192)}
        if op == "linear":
            c = _linear("", out=16 * _log_int(rng, 8, 3584), dim=256 * _log_int(rng, 2, 112), **kw)
        else:
            dim = 8 * _log_int(rng, 16, 3584)
            kw.update(dim=dim, pad=rng.choice([0, 0, 8, 8 * rng.randint(1, 256)]))
            if op == "norm":
                c = _norm("", residual=rng.random() < 0.7, bits=rng.choice([8, 8, 16]), **kw)
            elif op == "gated":
                c = _gated("", activation=rng.choice(["silu", "silu", "gelu_tanh"]), bits=rng.choice([8, 8, 16]), **kw)
            else:
                c = _rows("", **kw)
        del c["name"]
        w = work(c)
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES:
            return c


def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(rows, width, pad, dtype, g, outliers=False):
    """Normal values in rows `pad` elements further apart than they are wide; with outliers, one channel in 64 is larger, up to ten times."""
    out = torch.empty((rows, width + pad), dtype=dtype, device=DEV)
    many = max(1, (1 << 27) // (width + pad))
    for i in range(0, rows, many):
        out[i:i + many] = torch.randn((min(many, rows - i), width + pad), generator=g, device=DEV)
    if outliers:
        at = torch.randperm(width, generator=g, device=DEV)[:max(1, width // 64)]
        out[:, at] *= torch.linspace(2, 10, len(at), device=DEV).to(dtype)
    return out[:, :width]


def _codes(n, g, spread):
    """Whole numbers of -127 .. 127 as rounded normal values have them."""
    out = torch.empty(n, dtype=torch.int8, device=DEV)
    for i in range(0, n, 1 << 27):
        m = min(1 << 27, n - i)
        out[i:i + m] = torch.randn(m, generator=g, device=DEV).mul_(spread).round_().clamp_(-127, 127)
    return out


def prepare(case, seed):
    g = _generator(seed)
    M, K = case["rows"], case["dim"]
    state = {"case": case}
    if case["op"] == "linear":
        N, dtype = case["out"], TYPES[case["type"]]
        state["q"] = _codes(M * K, g, 26.0).view(M, K)
        state["q_scales"] = torch.rand(M, generator=g, device=DEV).mul_(0.03).add_(0.02)
        # what rtn_quantize(W, 8, 0) leaves: codes + 128 in tiles of 16 rows x 64 columns (independent values, so any order of them), fp16 scales
        state["qweight"] = (_codes(N * K, g, 29.0).view(torch.uint8) ^ 128)
        state["scales"] = torch.randn((N, 1), generator=g, device=DEV).mul_(0.1).add_(1.0).abs_().mul_(7e-4).half()
        state["out"] = torch.empty((M, N), dtype=dtype, device=DEV)
        # (a workspace of the most that a call of this size may ask for)
        state["workspace"] = torch.empty(64 << 20, dtype=torch.uint8, device=DEV)
        return state
    dtype = TYPES[case["type"]]
    state["x"] = _normal(M, K * (2 if case["op"] == "gated" else 1), case["pad"], dtype, g, outliers=True)
    if case["op"] == "norm":
        state["weight"] = _normal(1, K, 0, torch.float32, g)[0].mul(0.1).add_(1.0).to(dtype)
        state["residual"] = _normal(M, K, 0, dtype, g, outliers=True) if case["residual"] else None
        state["sum"] = torch.empty((M, K), dtype=dtype, device=DEV) if case["residual"] else None
    state["out"] = torch.empty((M, K), dtype=dtype, device=DEV)
    state["q"] = torch.empty((M, K), dtype=torch.int8, device=DEV)
    state["q_scales"] = torch.empty(M, dtype=torch.float32, device=DEV)
    return state


def run(state):
    return _run_linear(state) if state["case"]["op"] == "linear" else _run_rows(state)


def _run_linear(state):
    if own:
        import paper_2505_15909_amd as rtn
        return [rtn.rtn_linear_w8a8(state["q"], state["q_scales"], state["qweight"], state["scales"], out=state["out"], workspace=state["workspace"])]
    N, K = state["case"]["out"], state["case"]["dim"]
    q, S, out = state["q"].float(), state["q_scales"][:, None], state["out"]
    # a tile's bytes stand [quarter of 8 columns][row][half of 32 columns][column]
    tiles = state["qweight"].view(N // 16, K // 64, 4, 16, 2, 8)
    many = max(1, (1 << 28) // (16 * K))
    for i in range(0, N // 16, many):
        w = tiles[i:i + many].permute(0, 3, 1, 4, 2, 5).reshape(-1, K).float() - 128.0
        n = slice(16 * i, 16 * i + w.shape[0])
        out[:, n] = (torch.matmul(q, w.t()) * S * state["scales"][n, 0].float()).to(out.dtype)
    return [out]


def _run_rows(state):
    case, x, out, q, scales = state["case"], state["x"], state["out"], state["q"], state["q_scales"]
    op, quantised = case["op"], case.get("bits", 8) == 8
    got = {}
    if own:
        import paper_2505_15909_amd as rtn
        to = (q, scales) if quantised else out
        if op == "norm":
            rtn.rtn_norm_rows(x, state["weight"], residual=state["residual"], eps=1e-6, quantize=quantised, residual_out=state["sum"], out=to)
        elif op == "gated":
            rtn.rtn_gated_rows(x, activation=case["activation"], quantize=quantised, out=to)
        else:
            rtn.rtn_quantize_rows(x, out=to)
        if quantised:
            rtn.rtn_dequantize_rows(q, scales, out=out)
    else:
        if op == "norm":
            h = x.float()
            if state["residual"] is not None:
                state["sum"].copy_(h + state["residual"].float())
                h = state["sum"].float()
            y = h * torch.rsqrt(h.square().mean(-1, keepdim=True) + 1e-6) * state["weight"].float()
        elif op == "gated":
            a, b = x[:, :case["dim"]].float(), x[:, case["dim"]:].float()
            z = a if case["activation"] == "silu" else a * (1.0 + 0.044715 * a * a) * math.sqrt(8 / math.pi)
            y = a / (1.0 + torch.exp(-z)) * b
        else:
            y = x.float()
        if quantised:
            scales.copy_(y.abs().amax(-1) / 127.0)
            q.copy_(torch.round(torch.where(scales > 0, 1.0 / scales, 0.0)[:, None] * y))
            y = q.float() * scales[:, None]
        out.copy_(y)
    got["out"] = out
    if quantised:
        got["scales"] = scales
    if state.get("sum") is not None:
        got["sum"] = state["sum"]
    return got


def work(case):
    M, K = case["rows"], case["dim"]
    if case["op"] == "linear":
        N = case["out"]
        return {"bytes": N * K + 2 * N + M * K + 4 * M + 2 * M * N, "flops": 2 * M * N * K}
    given = {"norm": 4 if case.get("residual") else 1, "gated": 2, "rows": 1}[case["op"]]
    # the input, the sum read and written, the weight; what goes out, in 16 bits or in 8 with a scale a row
    moved = {"norm": 2 * M * K * (3 if case.get("residual") else 1) + 2 * K, "gated": 4 * M * K, "rows": 2 * M * K}[case["op"]]
    return {"bytes": moved + (2 * M * K if case.get("bits", 8) == 16 else M * K + 4 * M), "flops": M * K * (given + 4)}


def exact(case, seed):
    """The outputs in 64 bits from the definitions: the product over the bytes of each row of weights by their places, the rows in blocks."""
    s = prepare(case, seed)
    M, K = case["rows"], case["dim"]
    if case["op"] == "linear":
        N = case["out"]
        out = torch.empty((M, N), dtype=torch.float64, device=DEV)
        col = torch.arange(K, device=DEV)
        place = col // 64 * 1024 + col % 32 // 8 * 256 + col % 64 // 32 * 8 + col % 8      # of a column's byte, from the tile row's start, for row 0
        a = s["q"].double()
        for i in range(0, N, 2048):
            row = torch.arange(i, min(N, i + 2048), device=DEV)
            at = (row // 16 * (16 * K) + row % 16 * 16)[:, None] + place[None]
            w = s["qweight"][at].double().sub_(128).mul_(s["scales"][i:i + 2048].double())
            out[:, i:i + 2048] = torch.matmul(a, w.t().contiguous())
        return [out.mul_(s["q_scales"].double()[:, None])]
    x, got = s["x"], {"out": torch.empty((M, K), dtype=torch.float64, device=DEV)}
    if case.get("bits", 8) == 8:
        got["scales"] = torch.empty(M, dtype=torch.float64, device=DEV)
    if case.get("residual"):
        got["sum"] = torch.empty((M, K), dtype=torch.float64, device=DEV)
    many = max(1, (1 << 26) // K)
    for i in range(0, M, many):
        r = slice(i, min(M, i + many))
        if case["op"] == "gated":
            a, b = x[r].double().split(K, dim=1)
            gate = torch.sigmoid(a) * a if case["activation"] == "silu" else 0.5 * a * (1 + torch.tanh((2 / math.pi) ** 0.5 * (a + 0.044715 * a ** 3)))
            y = gate * b
        else:
            y = x[r].double()
            if case.get("residual"):
                got["sum"][r] = y + s["residual"][r].double()
                y = got["sum"][r].to(x.dtype).double()               # the sum is held in the type, and its norm taken of what is held
            if case["op"] == "norm":
                y = y / ((y ** 2).sum(1, keepdim=True) / K + 1e-6).sqrt() * s["weight"].double()
        if "scales" in got:
            step = y.abs().max(1).values / 127
            got["scales"][r] = step
            y = torch.round(y / step[:, None]) * step[:, None]
        got["out"][r] = y
    return got
