"""The 8-bit layer: rows quantised on the way (rtn_norm_rows, rtn_gated_rows, rtn_quantize_rows), their values (rtn_dequantize_rows) and their product with
8-bit weights (rtn_linear_w8a8), against plain implementations in 64 bits; and what the entry points refuse.

Tolerances.  u is the unit roundoff of the element type (2^-11 fp16, 2^-8 bf16), e = 2^-24 that of fp32; fp16 results below the normal range are off by
up to 2^-25.
  Codes of plain and normed rows are exact: the values (x, or h w with two significands of at most 11 bits) and the largest of them are exact in fp32, and
  max * (1 / 127), its reciprocal and the value times that are one IEEE operation each, which NumPy's fp32 does alike; then to the nearest, ties to even.  So are plain scales.
  The norm's factor: a thread adds up to 64 squares, then 6 steps over lanes and 15 over wavefronts: the sum is off by at most 86 e, its square root by half of that;
  mean, rsqrt (one unit = 2 e), and two roundings behind it: 43 + 1 + 2 + 2, bounded by 50 e.
  The gate: gelu's z comes from two constants and five operations, each e, so that it is off by at most 7 e |z| (silu's z is exact), which exp carries over; exp's own error
  2 e, 1 + exp, the quotient and the product with b 1 e each, and 3 e to spare: (8 + 7 |z|) e relative.  Below z = -87.33 the divisor is beyond
  2^126 and its reciprocal below the normal range, so that results of up to 87.4 / 2^126 < 2^-119 of |b| may vanish.
  The product: the sum is exact; it and its two products with scales are rounded in fp32: 3 e, and then u."""
import numpy as np
import pytest
import torch

import paper_2505_15909_amd as rtn
from oracle import rtn_oracle as O

lib = rtn._lib
FAKE = 0x1000
DEV = "cuda:0"
UNIT = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -120}
E = 2.0 ** -24
TYPES = [torch.float16, torch.bfloat16]
NULL, SHAPE, ALIGN, CONFIG = 1, 4, 5, 7


# ---- refusals (no GPU: arguments are checked before any launch) --------------------------------------------------------------------

def _norm(x=FAKE, rows=0, stride=64, dim=64, dtype=0, res=None, rs=64, res_out=None, ros=64, w=FAKE, eps=1e-6, out=FAKE, q=None, s=None):
    return lib.rtn_norm_rows(x, rows, stride, dim, dtype, res, rs, res_out, ros, w, eps, out, q, s, None)


def _gated(x=FAKE, rows=0, stride=128, dim=64, dtype=0, act=0, out=FAKE, q=None, s=None):
    return lib.rtn_gated_rows(x, rows, stride, dim, dtype, act, out, q, s, None)


def _quant(x=FAKE, rows=0, stride=64, dim=64, dtype=0, q=FAKE, s=FAKE):
    return lib.rtn_quantize_rows(x, rows, stride, dim, dtype, q, s, None)


def _dequant(q=FAKE, s=FAKE, rows=0, dim=64, dtype=0, out=FAKE):
    return lib.rtn_dequantize_rows(q, s, rows, dim, dtype, out, None)


def _linear(q=FAKE, s=FAKE, M=0, w=FAKE, ws=FAKE, N=64, K=512, dtype=0, C=FAKE, work=None, n=0):
    return lib.rtn_linear_w8a8(q, s, M, w, ws, N, K, dtype, C, work, n, None)


ROWS = [({"rows": -1}, SHAPE), ({"rows": (1 << 20) + 1}, SHAPE), ({"dim": 0}, SHAPE), ({"dim": 60}, SHAPE), ({"dim": 65544, "stride": 1 << 18}, SHAPE),
        ({"dtype": 2}, CONFIG), ({"rows": 1, "x": None}, NULL), ({"x": FAKE + 8}, ALIGN), ({}, 0)]


@pytest.mark.parametrize("kw,status", ROWS + [({"stride": 56}, SHAPE), ({"stride": 68}, ALIGN), ({"rows": 1, "w": None}, NULL), ({"w": FAKE + 2}, ALIGN),
                                              ({"rows": 1, "out": None}, NULL), ({"rows": 1, "q": FAKE, "s": FAKE}, NULL), ({"rows": 1, "out": None, "q": FAKE}, NULL),
                                              ({"rows": 1, "res": FAKE}, NULL), ({"rows": 1, "res_out": FAKE}, NULL), ({"res": FAKE, "res_out": FAKE, "rs": 56}, SHAPE),
                                              ({"res": FAKE, "res_out": FAKE, "ros": 68}, ALIGN), ({"res": FAKE + 2, "res_out": FAKE}, ALIGN),
                                              ({"eps": -1e-6}, CONFIG), ({"eps": float("nan")}, CONFIG), ({"eps": 0.0}, 0), ({"out": FAKE + 8}, ALIGN)])
def test_norm_refusals(kw, status):
    assert _norm(**kw) == status


@pytest.mark.parametrize("kw,status", ROWS + [({"stride": 120}, SHAPE), ({"stride": 132}, ALIGN), ({"act": 2}, CONFIG), ({"act": -1}, CONFIG), ({"rows": 1, "out": None}, NULL),
                                              ({"out": None, "q": FAKE, "s": FAKE + 2}, ALIGN), ({"act": 1}, 0)])
def test_gated_refusals(kw, status):
    assert _gated(**kw) == status


@pytest.mark.parametrize("kw,status", ROWS + [({"stride": 56}, SHAPE), ({"rows": 1, "q": None}, NULL), ({"rows": 1, "s": None}, NULL), ({"q": FAKE + 4}, ALIGN), ({"q": FAKE + 8}, 0), ({"s": FAKE + 2}, ALIGN)])
def test_quantize_refusals(kw, status):
    assert _quant(**kw) == status


@pytest.mark.parametrize("kw,status", [({"rows": -1}, SHAPE), ({"dim": 4}, SHAPE), ({"dtype": -1}, CONFIG), ({"rows": 1, "out": None}, NULL), ({"rows": 1, "s": None}, NULL),
                                       ({"q": FAKE + 4}, ALIGN), ({"out": FAKE + 8}, ALIGN), ({}, 0)])
def test_dequantize_refusals(kw, status):
    assert _dequant(**kw) == status


@pytest.mark.parametrize("kw,status", [({"M": 1, "q": None}, NULL), ({"M": 1, "s": None}, NULL), ({"M": 1, "w": None}, NULL), ({"M": 1, "ws": None}, NULL), ({"M": 1, "C": None}, NULL),
                                       ({"M": -1}, SHAPE), ({"M": (1 << 20) + 1}, SHAPE), ({"N": 24}, SHAPE), ({"N": 0}, SHAPE), ({"K": 128}, SHAPE), ({"K": 1 << 17}, SHAPE),
                                       ({"N": 16448, "K": 130816}, SHAPE), ({"M": 1 << 20, "N": 1 << 22, "K": 256}, SHAPE), ({"dtype": 2}, CONFIG), ({"q": FAKE + 8}, ALIGN), ({"w": FAKE + 8}, ALIGN), ({"ws": FAKE + 2}, ALIGN),
                                       ({"C": FAKE + 8}, ALIGN), ({"work": FAKE + 8}, ALIGN), ({"s": FAKE + 2}, ALIGN), ({}, 0)])
def test_linear_refusals(kw, status):
    assert _linear(**kw) == status


@pytest.mark.parametrize("M,N,K", [(0, 64, 512), (1, 24, 512), (1, 64, 128), (-1, 64, 512), (1, 64, 1 << 17)])
def test_no_workspace_for_what_is_refused(M, N, K):
    assert rtn.rtn_linear_w8a8_workspace_nbytes(M, N, K) == 0


@pytest.mark.parametrize("M", [1, 5, 16, 17, 64, 200, 1000, 1 << 20])
@pytest.mark.parametrize("N,K", [(16, 256), (16, 130816), (4096, 4096), (1024, 16384), (106496, 16384)])
def test_workspaces_stay_within_their_bound(M, N, K):
    assert 0 <= rtn.rtn_linear_w8a8_workspace_nbytes(M, N, K) <= 64 << 20


def test_binding_refuses_what_is_not_on_the_gpu():
    x = torch.zeros(2, 64, dtype=torch.float16)
    q, s = torch.zeros(2, 64, dtype=torch.int8), torch.zeros(2)
    for call in (lambda: rtn.rtn_norm_rows(x, x[0]), lambda: rtn.rtn_gated_rows(x), lambda: rtn.rtn_quantize_rows(x), lambda: rtn.rtn_dequantize_rows(q, s),
                 lambda: rtn.rtn_linear_w8a8(q, s, q.view(torch.uint8).view(-1), x[:, :1])):
        with pytest.raises(ValueError):
            call()


def test_native_calls_leave_what_they_do_not_take():
    from paper_2505_15909_amd import binding
    x, w = torch.zeros(2, 64, dtype=torch.float16), torch.zeros(64, dtype=torch.float16)
    q, s = torch.zeros(2, 64, dtype=torch.int8), torch.zeros(2)
    for call, args in ((binding._native.norm_rows, (x, w, None, 1e-6, False, None, x)), (binding._native.gated_rows, (x, 0, False, x[:, :32])),
                       (binding._native.quantize_rows, (x, (q, s))), (binding._native.dequantize_rows, (q, s, x)),
                       (binding._native.linear_w8a8, (q, s, q.view(torch.uint8).view(-1), x[:, :1], x, x))):
        assert call(*args) is None                           # (nothing of it is on a GPU)
        assert call(*args[:-1]) is None
        assert call(*[None] * len(args)) is None


# ---- rows ---------------------------------------------------------------------------------------------------------------------------

def _matrix(M, K, pad, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(M, K + pad, generator=g) * scale
    x[:, ::61] *= 9.0
    return x.to(dtype).to(DEV)[:, :K]


def _bordered(M, K, dtype):
    """An output with a row on each side that has to stay as it is."""
    whole = torch.full((M + 2, K), 77, dtype=dtype, device=DEV)
    return whole, whole[1:M + 1]


def _sides_are_left(*wholes):
    for w in wholes:
        assert (w[0] == 77).all() and (w[-1] == 77).all()


def _codes(v, most):
    """rne(v * (1 / scale)), scale = most * (1 / 127), of values that fp32 holds, in its steps."""
    step = np.where(most == 0, 1, most).astype(np.float32) * (np.float32(1) / np.float32(127))
    inv = np.where(most < 2.0 ** -100, np.float32(0), np.float32(1) / step).astype(np.float32)
    return np.rint(v.astype(np.float32) * inv[:, None])


def _f64(t):
    return t.double().cpu().numpy()


DIMS = [8, 16, 72, 512, 520, 2048, 2056, 4096, 5120, 8192, 8200, 14336, 16384, 16392, 28672, 32776, 53248, 65536]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K", DIMS)
def test_plain_rows_are_exact(rtn, K, dtype):
    for M, pad in ((1, 0), (5, 24), (258 if K <= 520 else 9, 0)):
        x = _matrix(M, K, pad, dtype, K + M)
        if M > 4:
            x[1] = 0
            x[2] = 0
            x[2, K // 2] = -3.0                              # one value
            x[3] = (x[3].double() * 2.0 ** -20).to(dtype)    # (subnormal in fp16)
        wq, q = _bordered(M, K, torch.int8)
        ws, s = _bordered(M, 1, torch.float32)
        got = rtn.rtn_quantize_rows(x, out=(q, s.view(M)))
        assert got[0] is q
        v = _f64(x)
        most = np.abs(v).max(1)
        assert np.array_equal(q.cpu().numpy(), _codes(v, most))
        assert np.array_equal(s.view(M).cpu().numpy(), most.astype(np.float32) * (np.float32(1) / np.float32(127)))
        _sides_are_left(wq, ws)
        for to in TYPES:
            wo, o = _bordered(M, K, to)
            rtn.rtn_dequantize_rows(q, s.view(M), out=o)
            want = (torch.from_numpy(q.cpu().numpy() * s.cpu().numpy())).to(to)        # (the exact product of 8 and 24 bits, in fp32 rounded once more)
            assert torch.equal(o.cpu(), want)
            _sides_are_left(wo)


def _norm_reference(x, residual, w, eps, dtype):
    h = x if residual is None else (x.double() + residual.double()).to(dtype)
    v = _f64(h) * _f64(w)
    mean = (_f64(h) ** 2).mean(1) + eps
    return h, v, np.where(mean == 0, 0, 1 / np.sqrt(np.where(mean == 0, 1, mean)))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K", DIMS)
@pytest.mark.parametrize("added", [False, True])
def test_normed_rows(rtn, K, added, dtype):
    for M, pad in ((1, 8), (6, 0), (131 if K <= 520 else 7, 40)):
        x = _matrix(M, K, pad, dtype, K + M + 1)
        w = (1 + 0.2 * _matrix(1, K, 0, dtype, 3)[0]).to(dtype)
        r = _matrix(M, K, 16, dtype, K + M + 2, 2.0) if added else None
        if M > 1:
            x[1] = 0
            if added:
                r[1] = 0
        h, v, factor = _norm_reference(x, r, w, 1e-5, dtype)
        y = v * factor[:, None]
        wo, o = _bordered(M, K, dtype)
        wr, ro = _bordered(M, K, dtype)
        rtn.rtn_norm_rows(x, w, residual=r, eps=1e-5, residual_out=ro if added else None, out=o)
        bound = (UNIT[dtype] + 50 * E) * np.abs(y) + TINY[dtype]
        assert (np.abs(_f64(o) - y) <= bound).all()
        if added:
            assert torch.equal(ro, h)
        _sides_are_left(wo, wr)
        wq, q = _bordered(M, K, torch.int8)
        ws, s = _bordered(M, 1, torch.float32)
        before = None if r is None else r.clone()
        rtn.rtn_norm_rows(x, w, residual=r, eps=1e-5, quantize=True, out=(q, s.view(M)))
        if added:                                            # in place where no other place is given
            assert torch.equal(r, h) and not torch.equal(before, r)
        most = np.abs(v).max(1)
        assert np.array_equal(q.cpu().numpy(), _codes(v, most))
        S = most * factor / 127
        assert (np.abs(_f64(s)[:, 0] - S) <= 52 * E * S).all()
        _sides_are_left(wq, ws)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_norm_without_eps_and_in_place_of_x(rtn, dtype):
    x, w = _matrix(4, 264, 0, dtype, 1), torch.ones(264, dtype=dtype, device=DEV)
    x[2] = 0
    y = rtn.rtn_norm_rows(x, w, eps=0.0)
    assert (y[2] == 0).all() and torch.isfinite(y).all()
    q, s = rtn.rtn_norm_rows(x, w, eps=0.0, quantize=True)
    assert (q[2] == 0).all() and s[2] == 0
    r, keep = _matrix(4, 264, 0, dtype, 2), x.clone()
    rtn.rtn_norm_rows(x, w, residual=r, residual_out=x)
    assert torch.equal(x, (keep.double() + r.double()).to(dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("activation", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("K", DIMS)
def test_gated_rows(rtn, K, activation, dtype):
    for M, pad in ((1, 0), (5, 8), (70 if K <= 520 else 6, 0)):
        x = _matrix(M, 2 * K, pad, dtype, K + M + 3, 2.0)
        if M > 1:
            x[1, :K] = 0
            x[2, K:] = 0
            x[3, :8] = torch.tensor([-100.0, 100.0, -12.0, 12.0, -0.0, 30.0, -30.0, 1e-3], device=DEV).to(dtype)
        a, b = _f64(x)[:, :K], _f64(x)[:, K:]
        z = a if activation == "silu" else a * np.sqrt(8 / np.pi) * (1 + 0.044715 * a * a)
        with np.errstate(over="ignore"):
            v = a / (1 + np.exp(-z)) * b
        rel = (8 + 7 * np.abs(z)) * E
        wo, o = _bordered(M, K, dtype)
        rtn.rtn_gated_rows(x, activation, out=o)
        assert (np.abs(_f64(o) - v) <= (UNIT[dtype] + rel) * np.abs(v) + TINY[dtype] + 2.0 ** -119 * np.abs(b)).all()
        _sides_are_left(wo)
        wq, q = _bordered(M, K, torch.int8)
        ws, s = _bordered(M, 1, torch.float32)
        rtn.rtn_gated_rows(x, activation, quantize=True, out=(q, s.view(M)))
        _sides_are_left(wq, ws)
        most = np.abs(v).max(1)
        off = (rel * np.abs(v)).max(1) + 2.0 ** -119 * np.abs(b).max(1)                # of any value, and so of the largest
        assert (np.abs(_f64(s)[:, 0] * 127 - most) <= off + 2 * E * most).all()
        some = most > 0
        assert (q.cpu().numpy()[~some] == 0).all() and (s.cpu().numpy()[~some] == 0).all()
        step = (most / 127)[some, None]
        far = np.abs(q.cpu().numpy()[some] - v[some] / step)
        assert (far <= 0.5 + 2 * off[some, None] / step + 127 * 4 * E).all()


@pytest.mark.gpu
@pytest.mark.parametrize("activation", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("dtype", TYPES)
def test_gate_of_any_magnitude(rtn, dtype, activation):
    most = torch.finfo(dtype).max
    a = torch.tensor([-0.0, 0.0, 2.0 ** -24, -5.5, -10.0, -10.25, -16.0, -80.0, -87.0, -87.5, -88.0, -88.5, -89.0, -104.0, -1e4, -6e4, 6e4, 200.0] +
                     [s * m for s in (1, -1) for m in (most, most / 3, most ** 0.5, most ** 0.25, most ** 0.125)] + [20.0] * 4, device=DEV).to(dtype)
    for up in (1.0, -2.0 ** 10):
        b = torch.full_like(a, up)
        b[a.abs().float() > most / 2 ** 12] = 0.5            # (what leaves the type is not asked for)
        x, y = _f64(a), _f64(b)
        z = x if activation == "silu" else x * np.sqrt(8 / np.pi) * (1 + 0.044715 * x * x)
        with np.errstate(over="ignore"):
            v = x / (1 + np.exp(-z)) * y
        got = _f64(rtn.rtn_gated_rows(torch.cat([a, b])[None], activation)[0])
        rel = (8 + 7 * np.minimum(np.abs(z), 88)) * E        # beyond, the exponential is 0 or its reciprocal is
        assert (np.abs(got - v) <= (UNIT[dtype] + rel) * np.abs(v) + TINY[dtype] + 2.0 ** -119 * np.abs(y)).all()


@pytest.mark.gpu
def test_small_rows_and_rows_that_are_not_finite_stay_by_themselves(rtn):
    x = torch.randn(5, 512, device=DEV).bfloat16()
    x[1] = 2.0 ** -101
    x[2, 7] = float("nan")
    x[3, 9] = float("inf")
    clean = x.clone()
    clean[2:4] = 0
    w = torch.ones(512, dtype=torch.bfloat16, device=DEV)
    both = torch.cat([x, x], 1)
    clean2 = torch.cat([clean, clean], 1)
    for a, b in ((rtn.rtn_quantize_rows(x), rtn.rtn_quantize_rows(clean)), (rtn.rtn_norm_rows(x, w, quantize=True), rtn.rtn_norm_rows(clean, w, quantize=True)),
                 (rtn.rtn_gated_rows(both, quantize=True), rtn.rtn_gated_rows(clean2, quantize=True))):
        for at in (0, 1, 4):
            assert torch.equal(a[0][at], b[0][at]) and torch.equal(a[1][at], b[1][at])
    q, s = rtn.rtn_quantize_rows(x)
    assert (q[1] == 0).all() and s[1] == 0
    assert not torch.isfinite(s[2:4]).any()                  # such a row does not pass for one of zeros


@pytest.mark.gpu
def test_no_rows(rtn):
    x = torch.empty(0, 256, dtype=torch.float16, device=DEV)
    assert rtn.rtn_quantize_rows(x)[0].shape == (0, 256)
    assert rtn.rtn_norm_rows(x, torch.ones(256, dtype=torch.float16, device=DEV)).shape == (0, 256)
    assert rtn.rtn_gated_rows(x).shape == (0, 128)
    q, s = torch.empty(0, 256, dtype=torch.int8, device=DEV), torch.empty(0, device=DEV)
    assert rtn.rtn_dequantize_rows(q, s).shape == (0, 256)
    W = torch.randn(32, 256, device=DEV).half()
    assert rtn.rtn_linear_w8a8(q, s, *rtn.rtn_quantize(W, 8, 0)).shape == (0, 32)


# ---- the product --------------------------------------------------------------------------------------------------------------------

def _problem(M, N, K, seed, full=False):
    r = np.random.RandomState(seed)
    low = -128 if full else -127
    q = r.randint(low, 128, (M, K)).astype(np.int8)
    w = np.clip(np.rint(r.standard_normal((N, K)) * 40), -128, 127).astype(np.int8)
    w[0, :] = -128
    s = (r.rand(M) * 0.02 + 0.001).astype(np.float32)
    ws = (r.rand(N, 1) * 1e-4 + 1e-5).astype(np.float16)
    qw = torch.from_numpy(O.pack_gfx950(w, 8)).to(DEV).view(-1)
    return q, s, w, ws, [torch.from_numpy(q).to(DEV), torch.from_numpy(s).to(DEV), qw, torch.from_numpy(ws).to(DEV)]


def _product(q, s, w, ws):
    total = torch.from_numpy(q).to(DEV).double() @ torch.from_numpy(w).to(DEV).double().t().contiguous()          # below 2^53: exact
    return total.cpu().numpy() * (s.astype(np.float64)[:, None] * ws.astype(np.float64)[:, 0][None])


def _near(got, want, dtype):
    return (np.abs(_f64(got) - want) <= (UNIT[dtype] + 3 * E * (1 + UNIT[dtype])) * np.abs(want) + TINY[dtype]).all()


SIZES = [(16, 256), (48, 512), (272, 768), (1040, 1280), (256, 4096), (4096, 1024), (640, 5376), (16, 28672)]


@pytest.mark.gpu
@pytest.mark.parametrize("N,K", SIZES)
@pytest.mark.parametrize("M", [1, 3, 16, 17, 31, 33, 64, 65, 100, 127, 128, 129, 200, 256, 257, 300, 520])
def test_product(rtn, M, N, K):
    *given, args = _problem(M, N, K, M + N + K, full=True)
    want = _product(*given)
    for dtype in TYPES:
        whole, out = _bordered(M, N, dtype)
        assert rtn.rtn_linear_w8a8(*args, out=out) is out
        assert _near(out, want, dtype)
        _sides_are_left(whole)
        for n in (0, 4 * M * N * 2, 4 * M * N * 3 + 16):     # sums of whole numbers: the same bits however they are split
            ws = torch.full((max(n, 16) // 16 * 16,), 255, dtype=torch.uint8, device=DEV)
            assert torch.equal(rtn.rtn_linear_w8a8(*args, dtype=dtype, workspace=ws), out)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(1, 512, 28672), (16, 1024, 8192), (64, 1024, 8192), (64, 8192, 28672), (217, 1024, 8192), (1024, 1024, 2048), (33, 4112, 16384)])
def test_workspaces_are_not_left(rtn, M, N, K):
    """The splits fit what is given, to the byte, and nothing behind it is touched: all that is asked for, and 16 bytes less than each number of parts takes."""
    *given, args = _problem(M, N, K, 7)
    out = rtn.rtn_linear_w8a8(*args)
    assert _near(out, _product(*given), torch.float16)
    need = rtn.rtn_linear_w8a8_workspace_nbytes(M, N, K)
    for n in [need] + [4 * M * N * k - 16 for k in (1, 2, 3, 4, 8)]:
        buffer = torch.full((n + 4096,), 77, dtype=torch.uint8, device=DEV)
        assert torch.equal(rtn.rtn_linear_w8a8(*args, workspace=buffer[:n]), out)
        assert (buffer[n:] == 77).all()


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 40, 130])
def test_sums_up_to_the_last_of_32_bits(rtn, M):
    K = 130816                                               # 2^14 K = 2^31 - 2^22
    q, w = np.full((M, K), -128, np.int8), np.full((32, K), -128, np.int8)
    w[16:] = 127
    s, ws = np.full(M, 2.0 ** -20, np.float32), np.full((32, 1), 2.0 ** -10, np.float16)
    args = [torch.from_numpy(q).to(DEV), torch.from_numpy(s).to(DEV), torch.from_numpy(O.pack_gfx950(w, 8)).to(DEV).view(-1), torch.from_numpy(ws).to(DEV)]
    out = rtn.rtn_linear_w8a8(*args)
    assert torch.equal(out[:, :16], torch.full_like(out[:, :16], float(K * 2 ** 14) * 2.0 ** -30))
    assert _near(out, _product(q, s, w, ws), torch.float16)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(1, 6144, 4096), (16, 4096, 14336), (64, 10240, 8192), (217, 4096, 4096), (1500, 4096, 2048), (2049, 2064, 1024)])
@pytest.mark.parametrize("flags", [0, 1])
def test_product_of_what_the_quantisers_give(rtn, M, N, K, flags):
    g = torch.Generator(device=DEV).manual_seed(M + N)
    W, x = torch.randn(N, K, generator=g, device=DEV).mul_(0.02).half(), torch.randn(M, K, generator=g, device=DEV).half()
    q, s = rtn.rtn_quantize_rows(x)
    qw, ws = rtn.rtn_quantize(W, 8, 0, flags)
    out = rtn.rtn_linear_w8a8(q, s, qw, ws)
    codes = rtn.rtn_unpack(qw, N, K, 8)
    want = (q.double() @ codes.double().t().contiguous()) * (s.double()[:, None] * ws.double()[:, 0][None])
    assert _near(out, _f64(want), torch.float16)
    # and what it stands for: each side is off by at most half a step
    true = x.double() @ W.double().t().contiguous()
    slack = (s.double() / 2)[:, None] * W.double().abs().sum(1)[None] + x.double().abs().sum(1)[:, None] * ws.double()[:, 0][None] * (0.5 if flags == 0 else 1.0) + \
        K * s.double()[:, None] * ws.double()[:, 0][None]
    assert ((want - true).abs() <= slack).all()


@pytest.mark.gpu
def test_offsets_beyond_32_bits(rtn):
    """Rows, codes and results whose offsets pass 32 bits: the last rows are what a call of their own gives."""
    M, K = 70001, 40960
    x = torch.empty(M, K, dtype=torch.bfloat16, device=DEV)
    x[:-3] = 1.0
    x[-3:] = torch.randn(3, K, device=DEV)
    w = torch.randn(K, device=DEV).bfloat16()
    q, s = rtn.rtn_quantize_rows(x)
    few = rtn.rtn_quantize_rows(x[-3:])
    assert torch.equal(q[-3:], few[0]) and torch.equal(s[-3:], few[1]) and (q[M // 2] == 127).all()
    assert torch.equal(rtn.rtn_dequantize_rows(q, s, torch.bfloat16)[-3:], rtn.rtn_dequantize_rows(*few, torch.bfloat16))
    few = rtn.rtn_gated_rows(x[-3:], quantize=True)
    got = rtn.rtn_gated_rows(x, quantize=True)
    assert torch.equal(got[0][-3:], few[0]) and torch.equal(got[1][-3:], few[1])
    r = x[-3:].clone()
    y = rtn.rtn_norm_rows(r.clone(), w, residual=r)
    assert torch.equal(rtn.rtn_norm_rows(x, w, residual=x)[-3:], y) and torch.equal(x[-3:], r)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(80001, 28672, 256), (1 << 20, 16, 4096), (1 << 20, 272, 2304)])
def test_products_whose_offsets_pass_32_bits(rtn, M, N, K):
    *_, (qe, se, qw, ws) = _problem(5, N, K, 3)
    q, s = torch.ones(M, K, dtype=torch.int8, device=DEV), torch.ones(M, device=DEV)
    q[-5:], s[-5:] = qe, se
    out = rtn.rtn_linear_w8a8(q, s, qw, ws)
    assert torch.equal(out[-5:], rtn.rtn_linear_w8a8(qe, se, qw, ws))
    assert torch.equal(out[M // 2], out[0]) and torch.equal(out[:1], rtn.rtn_linear_w8a8(q[:1], s[:1], qw, ws))


# ---- together, on streams, in graphs ------------------------------------------------------------------------------------------------

def _layer(rtn, seed, H=512, F=1280, heads=4, kv=2, D=128):
    g = torch.Generator(device=DEV).manual_seed(seed)
    shapes = {"qkv": ((heads + 2 * kv) * D, H), "o": (H, heads * D), "gate_up": (2 * F, H), "down": (H, F)}
    w = {n: rtn.rtn_quantize(torch.randn(s, generator=g, device=DEV).mul_(0.03).half(), 8, 0) for n, s in shapes.items()}
    norms = [torch.randn(H, generator=g, device=DEV).mul_(0.1).add_(1).half() for _ in range(2)]
    angle = torch.arange(64, device=DEV)[:, None] * (10000.0 ** (-torch.arange(0, D, 2, device=DEV) / D))[None]
    return w, norms, torch.cat([angle.cos(), angle.sin()], 1).float(), (heads, kv, D)


def _pass(rtn, layer, x, residual, plan):
    """A layer on new tokens, in 8 bits throughout: what a user's program calls."""
    w, norms, rope, (heads, kv, D) = layer
    cache, table, positions, slots, seq, start, most = plan
    q = rtn.rtn_norm_rows(x, norms[0], residual=residual, quantize=True)
    qkv = rtn.rtn_linear_w8a8(*q, *w["qkv"])
    queries = rtn.rtn_rope_cache(qkv, heads, rope, positions, slots, cache)
    a = rtn.rtn_paged_attention(queries, cache, table, seq, start, most)
    x = rtn.rtn_linear_w8a8(*rtn.rtn_quantize_rows(a.view(a.shape[0], -1)), *w["o"])
    q = rtn.rtn_norm_rows(x, norms[1], residual=residual, quantize=True)
    up = rtn.rtn_linear_w8a8(*q, *w["gate_up"])
    return rtn.rtn_linear_w8a8(*rtn.rtn_gated_rows(up, quantize=True), *w["down"])


def _plan(rtn, T, kv, D):
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)                     # noqa: E731
    cache = rtn.PagedCache(*(torch.zeros(4, kv, 16, D, dtype=torch.float16, device=DEV) for _ in range(2)))
    return cache, ints([[2, 0, 1, 3]]), ints(range(T)), ints([[2, 0, 1, 3][t // 16] * 16 + t % 16 for t in range(T)]), ints([T]), ints([0, T]), T


def _pass_64(rtn, layer, x, residual):
    """The same layer from the weights' values in 64 bits, with the activations in 8 bits a token as the calls hold them, 16 bits between the calls."""
    w, norms, rope, (heads, kv, D) = layer
    value = {n: rtn.rtn_dequantize(q, s, K, 8, 0).double() for (n, (q, s)), K in zip(w.items(), (512, heads * D, 512, 1280))}

    def held(v):
        S = v.abs().amax(1, keepdim=True) / 127
        return torch.round(v / S) * S

    def norm(h, n):
        return h / (h.square().mean(1, keepdim=True) + 1e-6).sqrt() * n.double()

    h = (x.double() + residual.double()).half().double()
    qkv = (held(norm(h, norms[0])) @ value["qkv"].t().contiguous()).half().double().view(-1, heads + 2 * kv, D)
    T = len(qkv)
    c, s = rope[:T].double()[:, None].chunk(2, -1)
    a, b = qkv[:, :heads + kv].chunk(2, -1)
    turned = torch.cat([a * c - b * s, b * c + a * s], -1).half().double()
    out = torch.empty(T, heads, D, dtype=torch.float64, device=DEV)
    for i in range(heads):
        k, v = turned[:, heads + i // (heads // kv)], qkv[:, heads + kv + i // (heads // kv)]
        score = (turned[:, i] @ k.t().contiguous()) / D ** 0.5
        out[:, i] = torch.softmax(score.masked_fill(torch.ones(T, T, device=DEV).triu(1).bool(), -np.inf), -1) @ v.contiguous()
    x = (held(out.view(T, -1).half().double()) @ value["o"].t().contiguous()).half()
    h = (x.double() + h).half().double()
    up = (held(norm(h, norms[1])) @ value["gate_up"].t().contiguous()).half().double()
    a, b = up.chunk(2, 1)
    return held(a / (1 + torch.exp(-a)) * b) @ value["down"].t().contiguous(), h


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 5, 40])
def test_a_layer_in_8_bits(rtn, T):
    """Each call of the two chains is held to its own bound above; over the chain a difference in the last place of 16 bits may turn a code by one.  A turned code moves an output by
    a step in one of K terms: relative to the sum's size (amax / 127) / (rms sqrt(K)), under 0.05 / sqrt(512) = 0.0022, and at most one code in eight is near enough to a border
    (2^-11 of 127 steps, both ways) to turn, four times over: 2e-3 sqrt(512 / 8) = 0.018 a projection, all of them together under 0.04."""
    layer = _layer(rtn, T)
    x, r = torch.randn(T, 512, device=DEV).half(), torch.randn(T, 512, device=DEV).half()
    want, h = _pass_64(rtn, layer, x, r.clone())
    got = _pass(rtn, layer, x, r, _plan(rtn, T, 2, 128))
    assert (got.double() - want).norm() <= 0.04 * want.norm()
    assert (r.double() - h).norm() <= 0.04 * h.norm()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 20])
def test_a_layer_captured_and_replayed(rtn, T):
    layer = _layer(rtn, T + 50)
    x, r = torch.randn(T, 512, device=DEV).half(), torch.randn(T, 512, device=DEV).half()
    plan = _plan(rtn, T, 2, 128)
    start = r.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _pass(rtn, layer, x, r, plan)                        # (also what the allocator wants to have seen)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _pass(rtn, layer, x, r, plan)
    for k in range(4):
        x.copy_(torch.randn(T, 512, device=DEV))
        r.copy_(start * (k + 1))
        graph.replay()
        torch.cuda.synchronize()
        got, held = out.clone(), r.clone()
        r.copy_(start * (k + 1))
        want = _pass(rtn, layer, x, r, plan)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(held, r)


@pytest.mark.gpu
def test_calls_on_two_streams_at_once(rtn):
    streams = [torch.cuda.Stream() for _ in range(2)]
    work = []
    for i in range(2):
        *given, args = _problem(40 + 100 * i, 512, 4096, i)
        x = _matrix(700, 4096, 0, torch.float16, i)
        need = rtn.rtn_linear_w8a8_workspace_nbytes(40 + 100 * i, 512, 4096)
        work.append((args, _product(*given), x, torch.empty(max(16, need), dtype=torch.uint8, device=DEV)))
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                args, _, x, ws = work[i]
                got[i].append((rtn.rtn_linear_w8a8(*args, workspace=ws), rtn.rtn_quantize_rows(x)))
    torch.cuda.synchronize()
    for i in range(2):
        q, s = rtn.rtn_quantize_rows(work[i][2])
        for out, (a, b) in got[i]:
            assert _near(out, work[i][1], torch.float16) and torch.equal(a, q) and torch.equal(b, s)


@pytest.mark.gpu
def test_binding_checks(rtn):
    x, w = torch.randn(4, 512, device=DEV).half(), torch.randn(32, 512, device=DEV).half()
    q, s = rtn.rtn_quantize_rows(x)
    qw, ws = rtn.rtn_quantize(w, 8, 0)
    refused = [lambda: rtn.rtn_quantize_rows(x.float()), lambda: rtn.rtn_quantize_rows(x[0]), lambda: rtn.rtn_quantize_rows(x.t()),
               lambda: rtn.rtn_quantize_rows(x, out=(q[:2], s)), lambda: rtn.rtn_quantize_rows(x, out=(q, s.half())), lambda: rtn.rtn_norm_rows(x, w[0].float()),
               lambda: rtn.rtn_norm_rows(x, w[0, :256]), lambda: rtn.rtn_norm_rows(x, w[0], residual=x[:2]), lambda: rtn.rtn_norm_rows(x, w[0], residual_out=x.clone()),
               lambda: rtn.rtn_norm_rows(x, w[0], residual=x.bfloat16()), lambda: rtn.rtn_norm_rows(x, w[0], out=x.bfloat16()), lambda: rtn.rtn_gated_rows(x, "relu"),
               lambda: rtn.rtn_gated_rows(x, out=x), lambda: rtn.rtn_dequantize_rows(q, s[:2]), lambda: rtn.rtn_dequantize_rows(q, s, torch.float32),
               lambda: rtn.rtn_linear_w8a8(q, s, qw[:-1], ws), lambda: rtn.rtn_linear_w8a8(q, s, qw, ws.float()), lambda: rtn.rtn_linear_w8a8(q, s, qw, ws.view(-1)),
               lambda: rtn.rtn_linear_w8a8(q, s[:3], qw, ws), lambda: rtn.rtn_linear_w8a8(q[:, ::2], s, qw, ws), lambda: rtn.rtn_linear_w8a8(q, s, qw, ws, dtype=torch.float32),
               lambda: rtn.rtn_linear_w8a8(q, s, qw, ws, out=torch.empty(4, 16, dtype=torch.float16, device=DEV)),
               lambda: rtn.rtn_linear_w8a8(q, s, qw, ws, workspace=torch.empty(64)), lambda: rtn.rtn_linear_w8a8(q, s, qw, ws, workspace=torch.empty(64, 2, device=DEV).t())]
    for call in refused:
        with pytest.raises(ValueError):
            call()
    with pytest.raises(rtn.RtnError):
        rtn.rtn_quantize_rows(torch.randn(4, 516, device=DEV).half())
    with pytest.raises(rtn.RtnError):
        rtn.rtn_quantize_rows(torch.randn(4, 516, device=DEV).half()[:, :512])           # rows that begin between two pieces
    one = torch.randn(1, 516, device=DEV).half()[:, :512]    # of one row, the stride says nothing
    assert torch.equal(rtn.rtn_quantize_rows(one)[0], rtn.rtn_quantize_rows(one.clone())[0])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_native_calls_and_python_give_the_same(rtn, dtype, monkeypatch):
    """With outputs given a call is read in native code: the same results, and the same refusals from the Python code that it leaves them to."""
    from paper_2505_15909_amd import binding
    x, r, w = _matrix(5, 512, 8, dtype, 1), _matrix(5, 512, 0, dtype, 2), _matrix(1, 512, 0, dtype, 3)[0]
    W = torch.randn(64, 512, device=DEV).half()
    qw = rtn.rtn_quantize(W, 8, 0)
    work = torch.empty(1 << 20, dtype=torch.uint8, device=DEV)

    def calls(out, half, codes, sums):
        yield rtn.rtn_norm_rows(x, w, out=out), out
        yield rtn.rtn_norm_rows(x, w, residual=r, residual_out=sums, quantize=True, out=codes), codes
        yield rtn.rtn_quantize_rows(x, out=codes), codes
        yield rtn.rtn_dequantize_rows(*codes, out=out), out
        yield rtn.rtn_linear_w8a8(*codes, *qw, out=half[:, :64].contiguous(), workspace=work), None
        yield rtn.rtn_gated_rows(x, "gelu_tanh", out=half), half
        short = codes[0][:, :256].contiguous(), codes[1]
        yield rtn.rtn_gated_rows(x, quantize=True, out=short), short

    def results():
        buffers = torch.empty(5, 512, dtype=dtype, device=DEV), torch.empty(5, 256, dtype=dtype, device=DEV), \
            (torch.empty(5, 512, dtype=torch.int8, device=DEV), torch.empty(5, device=DEV)), torch.empty(5, 512, dtype=dtype, device=DEV)
        got = []
        for y, given in calls(*buffers):
            assert given is None or y is given or all(a is b for a, b in zip(y, given))
            got += [t.clone() for t in (y if isinstance(y, tuple) else (y,))]
        return got + [buffers[3].clone()]

    native = results()
    taken = []
    for name in ("norm_rows", "gated_rows", "quantize_rows", "dequantize_rows", "linear_w8a8"):
        call = getattr(binding._native, name)
        monkeypatch.setattr(binding._native, name, lambda *a, call=call: taken.append(call(*a)) or taken[-1])
    again = results()
    assert taken == [0] * 7
    monkeypatch.setattr(binding, "_native", None)
    python = results()
    for a, b, c in zip(native, again, python):
        assert torch.equal(a, b) and torch.equal(a, c)
    half = torch.empty(5, 256, dtype=dtype, device=DEV)
    monkeypatch.undo()
    for call in (lambda: rtn.rtn_norm_rows(x, w, out=half), lambda: rtn.rtn_norm_rows(x, w.float(), out=torch.empty_like(r)), lambda: rtn.rtn_gated_rows(x, "relu", out=half),
                 lambda: rtn.rtn_gated_rows(x[:, :511], out=half), lambda: rtn.rtn_quantize_rows(x, out=(half, half)),
                 lambda: rtn.rtn_norm_rows(x, w, residual_out=r, out=torch.empty_like(r))):
        with pytest.raises(ValueError):
            call()
