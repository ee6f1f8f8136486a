"""The paged cache at the ends of its ranges: what test_paged_cache.py's sizes do not reach.  Against 64 bits, with bounds that do not grow with
the parameter under test.

u is the unit roundoff of the element type (2^-11 fp16, 2^-8 bf16).  With w_j the softmax weights, an output's error is at most
  u |o| + (1.125 u + e) sum_j w_j |v_j|  (the result's rounding, the weights' rounding, and e, the relative error of a weight: twice the score's)
plus, in fp16, what weights below its normal range lose.  Scores are sums of D products in fp32: 2 * 2^-23 * (D / 4) * sum |q k| scale."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from tests.test_paged_cache import DEV, SHAPE, UNIT, _attend, _attention_case, _attention_reference, _cache, _plan_case, _plan_reference, _rope, _run_plan, _same_plan, lib


# ---- capped scores: softcap tanh(s / softcap) ------------------------------------------------------------------------------------------
#
# The cap's own error is relative to the score.  From |x| = 1/5 on (x = s / softcap) tanh x is 1 - 2 / (e^2x + 1), whose last subtraction leaves at most
# 13 * 2^-23 of the result for exp and reciprocal of an ulp each; below, a series, a few roundings.  16 * 2^-23 |score| covers both.

def _check_capped(rtn, dtype, lens, softcap, D=128, scale=None, zero_query=False):
    q, k, v, table, seq, start = _attention_case(dtype, lens, 4, 2, D, 16, seed=int(math.log10(softcap)) + 60)
    if zero_query:
        q[::2] = 0
    out = torch.full(q.shape, float("nan"), dtype=dtype, device=DEV)
    rtn.rtn_paged_attention(q, rtn.PagedCache(k, v), table, seq, start, max(n for _, n in lens), scale=scale, softcap=softcap, out=out)
    s = D ** -0.5 if scale is None else scale
    want, mass, _ = _attention_reference(q, k, v, table, lens, s, softcap, 0)
    _, _, err = _attention_reference(q, k, v, table, lens, s, 0.0, 0)      # (the products' share, without the cap)
    largest = float((q.double().abs().amax(0).sum(-1).max() * k.double().nan_to_num().abs().max()) * s)      # no score is above it
    err = err + 2 * 16 * 2.0 ** -23 * min(softcap, largest)
    u = UNIT[dtype]
    bound = 1.01 * u * want.abs() + (1.125 * u + err) * mass + 2.0 ** -24
    assert torch.isfinite(out).all()
    for exact in [want] + ([_attention_reference(q, k, v, table, lens, s, 0.0, 0)[0]] if softcap >= 1e8 else []):     # (from there on the cap is none)
        over = (out.cpu().double() - exact).abs() - bound
        assert (over <= 0).all(), float(over.max())


CAPPED = {"decode": [(6, 1), (0, 1), (40, 1)], "drafts": [(3, 9), (17, 4)], "tiles": [(5, 70), (0, 40), (33, 1)]}


@pytest.mark.gpu
@pytest.mark.parametrize("lens", sorted(CAPPED))
@pytest.mark.parametrize("softcap", [1e3, 1e4, 1e5, 1e6, 1e8, 1e20, 1e38])
def test_large_caps_are_as_exact_as_none(rtn, lens, softcap):
    for dtype, D in ((torch.float16, 128), (torch.float16, 64), (torch.bfloat16, 256)):
        _check_capped(rtn, dtype, CAPPED[lens], softcap, D)


@pytest.mark.gpu
@pytest.mark.parametrize("lens", sorted(CAPPED))
@pytest.mark.parametrize("softcap", [1e-45, 1e-39, 1e-30, 1e-3, 0.3, 2.0])
def test_small_caps(rtn, lens, softcap):
    """Down to the smallest that fp32 has, where scale / softcap is beyond its range; a score of zero stays zero."""
    for dtype, D in ((torch.float16, 128), (torch.float16, 64), (torch.bfloat16, 256)):
        _check_capped(rtn, dtype, CAPPED[lens], softcap, D, zero_query=True)


@pytest.mark.gpu
@pytest.mark.parametrize("lens", sorted(CAPPED))
def test_scores_across_the_cap(rtn, lens):
    """Scores from far below to far above the cap, through the change of formula."""
    for softcap, scale in ((4.0, 0.5), (20.0, 1.0), (50.0, 2.0)):
        _check_capped(rtn, torch.float16, CAPPED[lens], softcap, 64, scale=scale)


# ---- weights far below the largest -----------------------------------------------------------------------------------------------------
#
# One key that takes nearly all the weight, with a V of zero, before n like ones with V of one: the result is what the small weights come to.  In fp16
# the weights are multiplied by 2^15 (few rows) or, whose weights may be 2^4 times those of the largest score yet seen, by 2^11 (many rows): a weight has
# an error of u of itself, or 2^-25 below the normal range, 2^-40 or 2^-36 of the largest.

@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("new,lost", [(1, 40), (7, 40), (70, 36)])
@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("nats", [5.0, 14.0, 15.0, 16.0, 17.0, 18.0])
def test_many_small_weights_beside_a_large_one(rtn, dtype, D, new, lost, split, nats):
    """In one piece, all of them beside the large one, and split, where every part has a maximum of its own."""
    n, ps, Hq = 32768, 256, 4
    pages = -(-(n + new) // ps)
    k, v = (torch.full((pages, 1, ps, D), x, dtype=dtype, device=DEV) for x in (0.0, 1.0))
    k[0, 0, 0], v[0, 0, 0] = 1.0, 0.0
    q = torch.ones(new, Hq, D, dtype=dtype, device=DEV)
    table = torch.arange(pages, dtype=torch.int32, device=DEV)[None]
    seq, start = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([n + new], [0, new]))
    out = rtn.rtn_paged_attention(q, rtn.PagedCache(k, v), table, seq, start, new, scale=nats / D,
                                  workspace=None if split else torch.empty(0, dtype=torch.uint8, device=DEV))
    small = torch.arange(n, n + new, dtype=torch.float64) * math.exp(-nats)        # the token at position p sees p like keys
    want = (small / (1 + small))[:, None, None]
    u = UNIT[dtype]
    e = 4 * 2.0 ** -23 * (D / 4) * nats + 2.0 ** -20
    bound = (1.01 * u + 1.125 * u + e) * want + (0.0 if dtype is torch.bfloat16 else (n + new) * 2.0 ** -lost + 2.0 ** -25)
    over = ((out.cpu().double() - want).abs() / bound).max()
    assert over <= 1, (float(over), float(out.float().mean()), float(want.mean()))


# ---- scale ---------------------------------------------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("lens", sorted(CAPPED))
@pytest.mark.parametrize("softcap", [0.0, 3e38])
def test_largest_scale_with_scores_of_zero(rtn, lens, softcap):
    """A scale, or a cap, that fp32 holds and its product with log2 e does not: scores of zero are zero, the result the mean of what is seen."""
    q, k, v, table, seq, start = _attention_case(torch.float16, CAPPED[lens], 4, 2, 128, 16)
    q.zero_()
    out = rtn.rtn_paged_attention(q, rtn.PagedCache(k, v), table, seq, start, max(n for _, n in CAPPED[lens]), scale=3.4e38, softcap=softcap)
    want, mass, _ = _attention_reference(q, k, v, table, CAPPED[lens], 1.0, 0.0, 0)
    u = UNIT[torch.float16]
    assert ((out.cpu().double() - want).abs() <= 1.01 * u * want.abs() + (1.125 * u + 2.0 ** -20) * mass + 2.0 ** -24).all()


# ---- the plan's status -----------------------------------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("what", ["negative", "most_negative", "above", "far_above", "all"])
def test_plan_says_everything_that_does_not_fit(rtn, what, in_place):
    """The bits of the status do not depend on one another: a free count out of range, and too few pages for the step."""
    step, cached, table, free, count, ps, max_tokens = _plan_case(11, 40, 16, 20, 200, 60, 0.2, 3)
    step = np.where(step < 0, 1, step).astype(np.int32)        # (nothing comes back)
    if what == "negative":
        count = -1
    elif what == "most_negative":
        count = -2 ** 31
    elif what == "above":                                     # a stack of three, said to hold four, for a step that needs more
        free, count = free[:3].copy(), 4
    elif what == "far_above":
        count = 2 ** 31 - 1
    else:
        count, cached[7], step[9], max_tokens = -5, -3, 2 ** 30, 7
    case = (step, cached, table, free, count, ps, max_tokens)
    want = _plan_reference(*case)
    assert want[5] & 8 and bool(want[5] & 1) == (what != "far_above")
    _same_plan(_run_plan(case, in_place), want)


@pytest.mark.gpu
@pytest.mark.parametrize("back,need,status", [(0, 4096, 1 | 4), (4096, 0, 8), (2048, 2048, 8 | 1 | 4), (4095, 1, 8)])
def test_plan_sums_that_pass_32_bits(rtn, back, need, status):
    """4096 requests of 2^20 + 4 pages: the pages given back or needed come to 2^32 + 16384, which is not 16384."""
    B, ps, blocks = 4096, 16, 2 ** 20 + 8
    ends = torch.arange(B, device=DEV) < back
    cached = torch.where(ends, 2 ** 24 + 64, 0).to(torch.int32)
    step = torch.where(ends, -1, 2 ** 24 + 128 if back else 2 ** 24 + 64).to(torch.int32)
    table = torch.empty(B, blocks, dtype=torch.int32, device=DEV)
    free, count, lens = torch.zeros(30000, dtype=torch.int32, device=DEV), torch.tensor([100 if back else 20000], dtype=torch.int32, device=DEV), cached.clone()
    plan = rtn.rtn_cache_plan(step, lens, table, free, count, ps, 2 ** 25)
    assert back + need == B and int(plan.status) == status
    assert torch.equal(plan.seq_lens, cached) and int(plan.free_count) == int(count) and not plan.query_start.any() and (plan.slots == -1).all()


# ---- workspaces ----------------------------------------------------------------------------------------------------------------------

class OnGpu(torch.Tensor):
    """A host tensor that says it is on the GPU: the binding's checks run without one."""
    is_cuda = property(lambda self: True)


def _on_gpu(*shape, dtype=torch.float16):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)


@pytest.fixture
def launches(monkeypatch):
    """The binding without a GPU and without native code: what would have been launched, none of it launched."""
    from paper_2505_15909_amd import binding
    seen = []

    class Library:
        def __getattr__(self, name):
            return getattr(real, name) if name.endswith("nbytes") else lambda *a: seen.append((name, a)) or 0

    real = binding._lib
    monkeypatch.setattr(binding, "_lib", Library())
    monkeypatch.setattr(binding, "_native", None)
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    return seen


WORKSPACES = {"on the host": lambda t: torch.zeros(4096, dtype=torch.uint8), "strided": lambda t: t(4096, dtype=torch.uint8)[::2],
              "expanded": lambda t: t(1, dtype=torch.uint8).expand(1 << 20), "transposed": lambda t: t(64, 64, dtype=torch.float32).t()}


@pytest.mark.parametrize("what", sorted(WORKSPACES))
def test_attention_refuses_a_workspace_that_is_not_one_piece_on_the_gpu(launches, what):
    import paper_2505_15909_amd as rtn
    q, ints = _on_gpu(2, 4, 128), lambda *n: _on_gpu(*n, dtype=torch.int32)
    cache = rtn.PagedCache(_on_gpu(4, 2, 16, 128), _on_gpu(4, 2, 16, 128))
    for out in (None, _on_gpu(2, 4, 128)):
        with pytest.raises(ValueError, match="workspace"):
            rtn.rtn_paged_attention(q, cache, ints(2, 3), ints(2), ints(3), 1, out=out, workspace=WORKSPACES[what](_on_gpu))
    assert not launches
    rtn.rtn_paged_attention(q, cache, ints(2, 3), ints(2), ints(3), 1, out=q, workspace=_on_gpu(4096, dtype=torch.uint8))
    assert [name for name, _ in launches] == ["rtn_paged_attention"]


@pytest.mark.gpu
@pytest.mark.parametrize("what", sorted(WORKSPACES))
def test_native_attention_leaves_such_a_workspace_to_be_refused(rtn, what):
    q, k, v, table, seq, start = _attention_case(torch.float16, CAPPED["drafts"], 4, 2, 128, 16)
    with pytest.raises(ValueError, match="workspace"):
        rtn.rtn_paged_attention(q, rtn.PagedCache(k, v), table, seq, start, 9, out=torch.empty_like(q),
                                workspace=WORKSPACES[what](lambda *n, dtype: torch.zeros(*n, dtype=dtype, device=DEV)))


# ---- launches ------------------------------------------------------------------------------------------------------------------------

def test_calls_that_no_launch_takes_are_refused():
    """A launch has fewer than 2^32 threads: more heads, or tiles, are refused before it.  (Nothing here is near to launching: no sizes that fit.)"""
    cache = lambda D, H: _cache(head_dim=D, kv_heads=H, token_stride=D, head_stride=16 * D, page_stride=16 * D * H)
    for D in (64, 128, 256):                                   # head_dim / 8 threads a head
        heads = 2 ** 35 // D // 2 ** 21                        # with 2^21 tokens exactly 2^32 threads
        assert _rope(tokens=2 ** 21, heads=heads - 16, stride=heads * D, rotary=64, cache=cache(D, 8)) == SHAPE
        assert _rope(tokens=2 ** 21, heads=heads + 16, stride=(heads + 32) * D, rotary=64, cache=cache(D, 8)) == SHAPE
    for new in (1, 2 ** 20):
        assert _attend(tokens=2 ** 20, heads=65536, stride=65536 * 64, cache=cache(64, 1024), B=1, new=new) == SHAPE
        assert _attend(tokens=2 ** 20, heads=1024, stride=1024 * 64, cache=cache(64, 1024), B=65536, new=new) == SHAPE
    assert _attend(tokens=2 ** 20 + 1) == SHAPE
    size = lambda tokens: lib.rtn_paged_attention_workspace_nbytes(tokens, 2, 4, _cache(), 1)
    assert size(2 ** 20) > 0 and size(2 ** 20 + 1) == 0


# ---- numbers that C's int does not hold ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("n", [2 ** 31 - 1, 2 ** 31, 2 ** 32 + 4, 2 ** 63 - 1, 2 ** 64 + 5])
def test_wide_windows_and_bounds_do_not_wrap(launches, n):
    import paper_2505_15909_amd as rtn
    q, ints = _on_gpu(2, 4, 128), lambda *n: _on_gpu(*n, dtype=torch.int32)
    cache, ws = rtn.PagedCache(_on_gpu(4, 2, 16, 128), _on_gpu(4, 2, 16, 128)), _on_gpu(4096, dtype=torch.uint8)
    rtn.rtn_paged_attention(q, cache, ints(2, 3), ints(2), ints(3), n, window=n, workspace=ws)
    (_, args), = launches
    assert C.c_int(args[11]).value == C.c_int(args[14]).value == 2 ** 31 - 1
    rtn.rtn_paged_attention(q, cache, ints(2, 3), ints(2), ints(3), 1, window=-2 ** 32 + n % 2 ** 32, workspace=ws)
    assert (C.c_int(launches[1][1][14]).value < 0) == (-2 ** 32 + n % 2 ** 32 < 0)
    assert rtn.rtn_paged_attention_workspace_nbytes(100, 2, 4, cache, n) == rtn.rtn_paged_attention_workspace_nbytes(100, 2, 4, cache, 100) > 0


def test_page_sizes_that_no_int_holds_are_refused(launches):
    import paper_2505_15909_amd as rtn
    ints = lambda *n: _on_gpu(*n, dtype=torch.int32)
    out = rtn.CachePlan(ints(2), ints(3), ints(8), ints(8), ints(1), ints(1))
    for page_size in (2 ** 32 + 16, -2 ** 32 + 16, 2 ** 64 + 16, -16):
        with pytest.raises(ValueError, match="page_size"):
            rtn.rtn_cache_plan(ints(2), ints(2), ints(2, 3), ints(4), ints(1), page_size, 8, out=out)
    assert not launches


@pytest.mark.gpu
def test_native_attention_leaves_wide_windows_to_be_clipped(rtn):
    q, k, v, table, seq, start = _attention_case(torch.float16, CAPPED["tiles"], 4, 2, 128, 16)
    cache = rtn.PagedCache(k, v)
    ws = torch.empty(rtn.rtn_paged_attention_workspace_nbytes(q.shape[0], 3, 4, cache, 70), dtype=torch.uint8, device=DEV)
    want = rtn.rtn_paged_attention(q, cache, table, seq, start, 70, workspace=ws).clone()
    assert torch.equal(rtn.rtn_paged_attention(q, cache, table, seq, start, 70, window=2 ** 32 + 4, workspace=ws, out=torch.empty_like(q)), want)


@pytest.mark.gpu
@pytest.mark.parametrize("ps", [16, 256])
@pytest.mark.parametrize("page", [-1, 2 ** 27, 2 ** 28 + 5, 2 ** 31 - 1, -2 ** 31])
def test_pages_that_no_slot_names_are_not_written(rtn, ps, page):
    """page * page_size beyond 31 bits is no slot of another page."""
    ints = lambda *n: torch.tensor(n, dtype=torch.int32, device=DEV)
    largest = 2 ** 31 // ps - 1                                # its slots are the last that there are
    plan = rtn.rtn_cache_plan(ints(3, 2, 1), ints(0, ps - 1, 0), ints(-7, -7, page, -7, -7, -7).view(3, 2), ints(9, 9, largest, page, page), ints(5), ps, 6)
    assert int(plan.status) == 0 and int(plan.free_count) == 2 and plan.positions.tolist() == [0, 1, 2, ps - 1, ps, 0]
    assert (plan.slots[:5] < 0).all() and int(plan.slots[5]) == largest * ps
