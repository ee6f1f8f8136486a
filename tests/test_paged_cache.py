"""The paged KV cache: block tables and slots (rtn_cache_plan), norms and rotation with the cache write (rtn_rope_cache), attention over the
pages (rtn_paged_attention), against plain implementations in 64 bits; and what the entry points refuse.

Tolerances.  u is the unit roundoff of the element type (2^-11 fp16, 2^-8 bf16).
  Rotation: computed in fp32 and rounded once: |error| <= u |y| + 4 fp32 roundings of a term up to sqrt(2) max(|a|, |b|); with a bound of
  16 * 2^-24 * (|a c| + |b s|) on those, plus the smallest subnormal's half in fp16.
  Attention: the weights p <= 1 are rounded to the element type, each off by u p and at most 2^-25 in fp16 below its normal range, before
  the products with V; scores and sums are fp32.  With w_j the softmax weights, |error| <= u |o| + u sum_j w_j |v_j| (1 + 1/8) + n 2^-25
  max|v| / (the row's sum >= 1) + e_s sum_j w_j |v_j|, where e_s bounds the scores' error: 2 * 2^-23 * (D / 4) * sum |q k| scale
  summed in fp32, a bound of 2 e_s on the relative change of a weight."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2505_15909_amd as rtn

lib = rtn._lib
FAKE = 0x1000
DEV = "cuda:0"
UNIT = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


# ---- refusals (no GPU: arguments are checked before any launch) --------------------------------------------------------------------

def _cache(**kw):
    d = dict(dev_k=FAKE, dev_v=FAKE, pages=8, page_size=16, kv_heads=2, head_dim=128, dtype=0, page_stride=2 * 16 * 128, head_stride=16 * 128, token_stride=128)
    d.update(kw)
    return C.byref(rtn.rtn_kv_cache(**d))


def _plan(step=FAKE, cached=FAKE, B=4, ps=16, table=FAKE, stride=8, blocks=8, free=FAKE, pool=8, count=FAKE, seq=FAKE, start=FAKE, pos=FAKE, slots=FAKE,
          tokens=16, count_out=FAKE, status=FAKE):
    return lib.rtn_cache_plan(step, cached, B, ps, table, stride, blocks, free, pool, count, seq, start, pos, slots, tokens, count_out, status, None)


def _rope(qkv=FAKE, tokens=0, stride=8 * 128, heads=4, rope=FAKE, rotary=128, positions_n=16, interleaved=0, pos=FAKE, slots=FAKE, qn=None, kn=None,
          eps=1e-6, cache=None, out=FAKE):
    return lib.rtn_rope_cache(qkv, tokens, stride, heads, rope, rotary, positions_n, interleaved, pos, slots, qn, kn, eps, cache or _cache(), out, None)


def _attend(q=FAKE, tokens=0, stride=4 * 128, heads=4, cache=None, table=FAKE, tstride=8, blocks=8, seq=FAKE, start=FAKE, B=2, new=1, scale=0.1, cap=0.0,
            window=0, out=FAKE, ws=None, wsn=0):
    return lib.rtn_paged_attention(q, tokens, stride, heads, cache or _cache(), table, tstride, blocks, seq, start, B, new, scale, cap, window, out, ws, wsn, None)


NULL, SHAPE, ALIGN, CONFIG = 1, 4, 5, 7


@pytest.mark.parametrize("kw,status", [({"step": None}, NULL), ({"table": None}, NULL), ({"pos": None}, NULL), ({"status": None}, NULL), ({"B": 0}, SHAPE),
                                       ({"B": 4097}, SHAPE), ({"ps": 24}, SHAPE), ({"ps": 8}, SHAPE), ({"ps": 512}, SHAPE), ({"stride": 7}, SHAPE),
                                       ({"blocks": 0}, SHAPE), ({"pool": 0}, SHAPE), ({"tokens": -1}, SHAPE), ({"tokens": 1 << 30}, SHAPE),
                                       ({"seq": FAKE + 2}, ALIGN), ({"slots": FAKE + 1}, ALIGN)])
def test_plan_refusals(kw, status):
    assert _plan(**kw) == status


@pytest.mark.parametrize("kw,status", [({"dev_k": None}, NULL), ({"dtype": 2}, CONFIG), ({"head_dim": 96}, SHAPE), ({"page_size": 48}, SHAPE),
                                       ({"kv_heads": 0}, SHAPE), ({"pages": 0}, SHAPE), ({"pages": 1 << 28}, SHAPE), ({"token_stride": 120}, SHAPE),
                                       ({"token_stride": 132}, ALIGN), ({"page_stride": 4100}, ALIGN), ({"page_stride": -4096}, SHAPE),
                                       ({"token_stride": 1 << 27}, SHAPE), ({"dev_v": FAKE + 8}, ALIGN)])
def test_cache_refusals(kw, status):
    assert _rope(cache=_cache(**kw)) == status
    assert _attend(cache=_cache(**kw)) == status
    assert lib.rtn_paged_attention_workspace_nbytes(4, 2, 4, _cache(**kw), 1) == 0


@pytest.mark.parametrize("kw,status", [({"tokens": 1, "qkv": None}, NULL), ({"tokens": 1, "out": None}, NULL), ({"tokens": -1}, SHAPE), ({"heads": 0}, SHAPE),
                                       ({"rotary": 4}, SHAPE), ({"rotary": 136}, SHAPE), ({"rotary": 60}, SHAPE), ({"positions_n": 0}, SHAPE),
                                       ({"stride": 7 * 128}, SHAPE), ({"stride": 8 * 128 + 4}, ALIGN), ({"qkv": FAKE + 8}, ALIGN), ({"qn": FAKE + 2}, ALIGN),
                                       ({"rope": FAKE + 4}, ALIGN), ({"slots": FAKE + 2}, ALIGN), ({"eps": -1.0}, CONFIG), ({"eps": float("nan")}, CONFIG),
                                       ({"interleaved": 2}, CONFIG), ({}, 0)])
def test_rope_refusals(kw, status):
    assert _rope(**kw) == status


@pytest.mark.parametrize("kw,status", [({"tokens": 1, "q": None}, NULL), ({"table": None}, NULL), ({"start": None}, NULL), ({"heads": 3}, SHAPE),
                                       ({"heads": 130}, SHAPE), ({"tokens": -1}, SHAPE), ({"tokens": (1 << 24) + 1}, SHAPE), ({"B": 0}, SHAPE),
                                       ({"stride": 3 * 128}, SHAPE), ({"stride": 516}, ALIGN), ({"blocks": 0}, SHAPE), ({"tstride": 7}, SHAPE), ({"new": 0}, SHAPE),
                                       ({"scale": 0.0}, CONFIG), ({"scale": float("nan")}, CONFIG), ({"scale": float("inf")}, CONFIG), ({"cap": -1.0}, CONFIG),
                                       ({"window": -1}, CONFIG), ({"q": FAKE + 8}, ALIGN), ({"ws": FAKE + 8}, ALIGN), ({"seq": FAKE + 1}, ALIGN), ({}, 0)])
def test_attention_refusals(kw, status):
    assert _attend(**kw) == status


def test_sizes_beyond_the_offsets_are_refused():
    assert _attend(cache=_cache(page_stride=1 << 40, pages=1 << 26)) == SHAPE
    assert _rope(cache=_cache(head_stride=1 << 50)) == SHAPE
    assert _rope(tokens=1 << 24, heads=128, stride=132 * 128) == SHAPE


def test_binding_refuses_what_is_not_as_described():
    cpu = torch.zeros(4, 2, 16, 128, dtype=torch.float16)
    with pytest.raises(ValueError):
        rtn.PagedCache(cpu, cpu)
    ints = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        rtn.rtn_cache_plan(ints, ints, ints[None], ints, ints[:1], 16, 16)


# ---- plan ----------------------------------------------------------------------------------------------------------------------------

def _plan_reference(step, cached, table, free, count, ps, max_tokens):
    """One request after the other, with a stack."""
    B, width = table.shape
    step, cached = [int(s) for s in step], [int(c) for c in cached]
    status, tokens, need, back = 0, 0, 0, 0
    for s, c in zip(step, cached):
        if c < 0 or -(-c // ps) > width:
            status |= 8
        elif s < 0:
            back += -(-c // ps)
        else:
            fits = -(-(c + s) // ps) <= width
            status |= 0 if fits else 2
            status |= 4 if s > max_tokens else 0
            if fits and s <= max_tokens:
                tokens += s
                need += -(-(c + s) // ps) - -(-c // ps)
    if count < 0 or count > len(free) or count + back - need > len(free):
        status |= 8
    if count + back - need < 0:
        status |= 1
    if tokens > max_tokens:
        status |= 4
    table, free = table.copy(), free.copy()
    positions, slots = np.full(max_tokens, -1, np.int32), np.full(max_tokens, -1, np.int32)
    if status:
        return np.array(cached, np.int32), np.zeros(B + 1, np.int32), positions, slots, count, status, table, free
    stack = list(free[:count])
    for b in range(B):
        if step[b] < 0:
            stack += list(table[b, :-(-cached[b] // ps)])
    seq, start, at = [], [0], 0
    for b in range(B):
        if step[b] < 0:
            seq.append(0)
        else:
            for j in range(-(-cached[b] // ps), -(-(cached[b] + step[b]) // ps)):
                table[b, j] = stack.pop()
            for p in range(cached[b], cached[b] + step[b]):
                positions[at], slots[at] = p, table[b, p // ps] * ps + p % ps
                at += 1
            seq.append(cached[b] + step[b])
        start.append(at)
    if len(stack) > count:
        free[count:len(stack)] = stack[count:]
    return np.array(seq, np.int32), np.array(start, np.int32), positions, slots, len(stack), 0, table, free


def _plan_case(seed, B, ps, width, longest, most_new, p_end, spare, padding=3):
    rng = np.random.default_rng(seed)
    cached = rng.integers(0, longest + 1, B)
    step = np.where(rng.random(B) < p_end, -1 - rng.integers(0, 3, B), rng.integers(0, most_new + 1, B))
    used = -(-cached // ps)
    pages = rng.permutation(int(used.sum()) + 4096).astype(np.int32)
    table = np.full((B, width), -7, np.int32)
    at = 0
    for b in range(B):
        table[b, :used[b]] = pages[at:at + used[b]]
        at += used[b]
    grow = sum(-(-(c + s) // ps) - -(-c // ps) for c, s in zip(cached, step) if s >= 0)
    back = sum(-(-c // ps) for c, s in zip(cached, step) if s < 0)
    count = max(0, grow - back + spare)
    free = np.full(count + back + 5, -9, np.int32)
    free[:count] = np.resize(pages[at:], count)
    return step.astype(np.int32), cached.astype(np.int32), table, free, count, ps, int(max(0, step.clip(0).sum())) + padding


def _run_plan(case, in_place=False, stride_extra=0):
    step, cached, table, free, count, ps, max_tokens = case
    dev = [torch.from_numpy(a.copy()).to(DEV) for a in (step, cached)]
    wide = torch.full((table.shape[0], table.shape[1] + stride_extra), -11, dtype=torch.int32, device=DEV)
    t = wide[:, :table.shape[1]]
    t.copy_(torch.from_numpy(table))
    f, c = torch.from_numpy(free.copy()).to(DEV), torch.tensor([count], dtype=torch.int32, device=DEV)
    out = rtn.CachePlan.empty(len(step), max_tokens, DEV)
    for x in out:
        x.fill_(-77)
    if in_place:
        out = out._replace(seq_lens=dev[1], free_count=c)
    p = rtn.rtn_cache_plan(dev[0], dev[1], t, f, c, ps, max_tokens, out=out)
    torch.cuda.synchronize()
    assert (wide[:, table.shape[1]:] == -11).all()
    return [x.cpu().numpy() for x in (p.seq_lens, p.query_start, p.positions, p.slots)] + [int(p.free_count), int(p.status), t.cpu().numpy(), f.cpu().numpy()]


def _same_plan(got, want):
    for g, w, name in zip(got, want, ("seq_lens", "query_start", "positions", "slots", "free_count", "status", "block_table", "free_pages")):
        assert np.array_equal(g, w), name


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,ps,longest,most_new,p_end,spare", [(1, 16, 0, 1, 0.0, 0), (1, 16, 40, 0, 0.0, 0), (1, 32, 100, 0, 1.0, 0), (64, 16, 500, 1, 0.1, 4),
                                                               (300, 16, 200, 40, 0.2, 0), (257, 64, 3000, 5, 0.5, 2), (5, 16, 30, 3000, 0.0, 1),
                                                               (4096, 16, 100, 3, 0.3, 7), (1000, 256, 900, 1, 0.9, 0)])
def test_plan_matches_a_stack(rtn, B, ps, longest, most_new, p_end, spare, in_place):
    width = -(-(longest + most_new) // ps) + 1
    for seed in range(3):
        case = _plan_case(seed, B, ps, width, longest, most_new, p_end, spare)
        want = _plan_reference(*case)
        assert want[5] == 0
        _same_plan(_run_plan(case, in_place, stride_extra=seed), want)


@pytest.mark.gpu
@pytest.mark.parametrize("what", ["pages", "table", "tokens", "one_step", "cached", "negative", "count", "pool", "sum"])
def test_plan_that_does_not_fit_changes_nothing(rtn, what):
    step, cached, table, free, count, ps, max_tokens = _plan_case(5, 40, 16, 20, 200, 60, 0.1, 3)
    if what == "pages":
        count = max(0, count - 4)
    elif what == "table":
        table = table[:, :int((-(-cached // ps)).max())].copy()
        step[np.argmax(cached)] = 1000
        max_tokens += 1000
    elif what == "tokens":
        max_tokens -= 4
    elif what == "one_step":
        step[step >= 0] = 2 ** 31 - 1
    elif what == "cached":
        cached[7] = 16 * 20 + 1
    elif what == "negative":
        cached[7] = -1
    elif what == "count":
        count = len(free) + 1
    elif what == "pool":
        step[:] = -1
        free = free[:3].copy()
        count = 2
    else:
        step, max_tokens = np.full(40, 60, np.int32), 40 * 60 - 1
        table = np.concatenate([table, np.full((40, 8), -7, np.int32)], 1)
    case = (step, cached, table, free, count, ps, max_tokens)
    want = _plan_reference(*case)
    assert want[5] != 0
    _same_plan(_run_plan(case), want)
    _same_plan(_run_plan(case, in_place=True), want)


# ---- rotation and cache write --------------------------------------------------------------------------------------------------------

def _pools(pages, H, ps, D, dtype, layout, seed, fill=None):
    g = torch.Generator().manual_seed(seed)
    shape = (pages, H, ps, D) if layout == "head" else (pages, ps, H, D)
    pools = []
    for _ in range(2):
        x = torch.randn(shape, generator=g) if fill is None else torch.full(shape, fill)
        x = x.to(dtype).to(DEV)
        pools.append(x if layout == "head" else x.transpose(1, 2))
    return pools


def _rotated(x, weight, rope, positions, rotary, interleaved, eps):
    """float64; also the bound on the fp32 terms."""
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight.double()
    y, size = x.clone(), x.abs()
    cs = rope.double()[positions.long()]
    for i in range(rotary // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rotary // 2)
        c, s = cs[:, i][:, None], cs[:, rotary // 2 + i][:, None]
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
        size[..., a] = x[..., a].abs() * c.abs() + x[..., b].abs() * s.abs()
        size[..., b] = x[..., b].abs() * c.abs() + x[..., a].abs() * s.abs()
    return y, size


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("T,Hq,Hk,D,rotary,interleaved,norm,ps,layout,extra", [
    (1, 32, 8, 128, 128, False, False, 16, "head", 0), (7, 5, 5, 64, 64, False, True, 16, "token", 0), (33, 8, 1, 256, 256, True, True, 64, "head", 8),
    (300, 3, 3, 128, 64, False, True, 32, "token", 64), (129, 28, 4, 64, 8, True, False, 256, "head", 0), (65, 2, 1, 256, 104, False, True, 128, "token", 16),
    (2, 128, 8, 128, 128, True, True, 16, "head", 8), (40, 1, 1, 64, 56, False, False, 16, "head", 0)])
def test_rope_cache(rtn, dtype, T, Hq, Hk, D, rotary, interleaved, norm, ps, layout, extra):
    g = torch.Generator().manual_seed(T * 7 + D)
    wide = torch.randn(T, (Hq + 2 * Hk) * D + extra, generator=g).to(dtype).to(DEV)
    qkv = wide[:, :(Hq + 2 * Hk) * D]
    longest = 700
    rope = torch.randn(longest, rotary, generator=g).to(DEV)           # (any table: only the formula is under test)
    positions = torch.randint(0, longest, (T,), generator=g).to(torch.int32)
    pages = -(-T // ps) + 3
    slots = torch.randperm(pages * ps, generator=g)[:T].to(torch.int32)
    slots[T // 2] = -1 if T > 1 else slots[T // 2]                       # a padded row
    if T > 4:
        slots[3] = pages * ps                                              # out of the pool: not written
    k, v = _pools(pages, Hk, ps, D, dtype, layout, 3)
    k0, v0 = k.clone().cpu(), v.clone().cpu()
    qn, kn = ((1 + 0.1 * torch.randn(D, generator=g)).to(dtype).to(DEV) if norm else None for _ in range(2))
    cache = rtn.PagedCache(k, v)
    out = rtn.rtn_rope_cache(qkv, Hq, rope, positions.to(DEV), slots.to(DEV), cache, qn, kn, eps=1e-5, interleaved=interleaved)
    torch.cuda.synchronize()
    x = qkv.cpu().view(T, Hq + 2 * Hk, D) if extra == 0 else qkv.cpu().reshape(T, Hq + 2 * Hk, D)
    u = UNIT[dtype]

    def close(got, want, size):
        bound = u * want.abs() + 16 * 2.0 ** -24 * size * (1 + u) + 2.0 ** -25
        assert ((got.double() - want).abs() <= bound).all(), float(((got.double() - want).abs() - bound).max())

    want, size = _rotated(x[:, :Hq], None if qn is None else qn.cpu(), rope.cpu(), positions, rotary, interleaved, 1e-5)
    close(out.cpu(), want, size)
    want, size = _rotated(x[:, Hq:Hq + Hk], None if kn is None else kn.cpu(), rope.cpu(), positions, rotary, interleaved, 1e-5)
    kc, vc = k.cpu(), v.cpu()
    untouched = torch.ones(pages, ps, dtype=torch.bool)
    for t in range(T):
        s = int(slots[t])
        if 0 <= s < pages * ps:
            close(kc[s // ps, :, s % ps], want[t], size[t])
            assert torch.equal(vc[s // ps, :, s % ps], x[t, Hq + Hk:])
            untouched[s // ps, s % ps] = False
    assert torch.equal(kc.transpose(1, 2)[untouched], k0.transpose(1, 2)[untouched])
    assert torch.equal(vc.transpose(1, 2)[untouched], v0.transpose(1, 2)[untouched])


@pytest.mark.gpu
def test_rope_cache_of_no_tokens_and_positions_beyond_the_table(rtn):
    k, v = _pools(2, 2, 16, 128, torch.float16, "head", 1)
    cache = rtn.PagedCache(k, v)
    rope = torch.randn(5, 128, device=DEV)
    none = torch.empty(0, dtype=torch.int32, device=DEV)
    assert rtn.rtn_rope_cache(torch.empty(0, 8 * 128, dtype=torch.float16, device=DEV), 4, rope, none, none, cache).shape == (0, 4, 128)
    qkv = torch.randn(2, 8 * 128, device=DEV).half()
    far = torch.tensor([-3, 99], dtype=torch.int32, device=DEV)
    ends = torch.tensor([0, 4], dtype=torch.int32, device=DEV)
    slots = torch.tensor([0, 17], dtype=torch.int32, device=DEV)
    assert torch.equal(rtn.rtn_rope_cache(qkv, 4, rope, far, slots, cache), rtn.rtn_rope_cache(qkv, 4, rope, ends, slots, cache))


# ---- attention -----------------------------------------------------------------------------------------------------------------------

def _attention_case(dtype, lens, Hq, Hk, D, ps, layout="head", seed=0, padding=0, fill_unused=float("nan"), scale_q=1.0, extra=0):
    """lens: (cached, new) of each request.  Slots that hold no token are filled with `fill_unused`."""
    g = torch.Generator().manual_seed(seed)
    counts = [-(-(c + n) // ps) for c, n in lens]
    pages = sum(counts) + 2
    k, v = _pools(pages, Hk, ps, D, dtype, layout, seed + 1)
    order = torch.randperm(pages, generator=g).to(torch.int32)
    width = max(counts) + 1
    table = torch.full((len(lens), width), 2 ** 30, dtype=torch.int32)
    at, held = 0, torch.zeros(pages, ps, dtype=torch.bool)
    for b, (c, n) in enumerate(lens):
        table[b, :counts[b]] = order[at:at + counts[b]]
        at += counts[b]
        for j in range(counts[b]):
            held[table[b, j], :min(ps, c + n - j * ps)] = True
    for pool in (k, v):
        pool.transpose(1, 2)[~held.to(DEV)] = fill_unused
    T = sum(n for _, n in lens) + padding
    q = (torch.randn(T, Hq * D + extra, generator=g) * scale_q).to(dtype).to(DEV)[:, :Hq * D].unflatten(1, (Hq, D))
    start = torch.tensor([0] + list(np.cumsum([n for _, n in lens])), dtype=torch.int32, device=DEV)
    seq = torch.tensor([c + n for c, n in lens], dtype=torch.int32, device=DEV)
    return q, k, v, table.to(DEV), seq, start


def _attention_reference(q, k, v, table, lens, scale, softcap, window):
    """(result, bound) in float64, request by request, on the CPU."""
    q, k, v, table = q.cpu().double(), k.cpu(), v.cpu(), table.cpu().long()
    T, Hq, D = q.shape
    Hk, ps = k.shape[1], k.shape[2]
    out, mass, err = torch.zeros(T, Hq, D, dtype=torch.float64), torch.zeros(T, Hq, D, dtype=torch.float64), torch.zeros(T, Hq, 1, dtype=torch.float64)
    at = 0
    for b, (c, n) in enumerate(lens):
        if c + n > 0 and n > 0:
            lo = max(0, (c + 1 - window) // ps) if window else 0
            key = torch.arange(lo * ps, c + n)
            kb, vb = (x[table[b, lo:-(-(c + n) // ps)]].transpose(0, 1).reshape(Hk, -1, D)[:, :len(key)].double() for x in (k, v))
            pos = torch.arange(c, c + n)[:, None]
            hidden = (key[None] > pos) | ((pos - key[None] >= window) if window else torch.zeros(1, 1, dtype=torch.bool))
            for h in range(Hq):
                hk = h // (Hq // Hk)
                s = q[at:at + n, h] @ kb[hk].T * scale
                size = (q[at:at + n, h].abs() @ kb[hk].abs().T * scale).masked_fill(hidden, 0.0).amax(-1, keepdim=True)
                if softcap:
                    s = softcap * torch.tanh(s / softcap)
                    size = size + softcap
                w = torch.softmax(s.masked_fill(hidden, -np.inf), -1)
                out[at:at + n, h] = w @ vb[hk]
                mass[at:at + n, h] = w @ vb[hk].abs()
                err[at:at + n, h] = 4 * 2.0 ** -23 * (D / 4) * size + 2.0 ** -20
        at += n
    return out, mass, err


def _check_attention(rtn, dtype, lens, Hq, Hk, D, ps, layout="head", softcap=0.0, window=0, seed=0, padding=0, scale=None, scale_q=1.0, extra=0, max_new=None,
                     workspace=None):
    q, k, v, table, seq, start = _attention_case(dtype, lens, Hq, Hk, D, ps, layout, seed, padding, scale_q=scale_q, extra=extra)
    cache = rtn.PagedCache(k, v)
    out = torch.full(q.shape, float("nan"), dtype=dtype, device=DEV)
    bound_new = max_new or max(1, max(n for _, n in lens))
    rtn.rtn_paged_attention(q, cache, table, seq, start, bound_new, scale=scale, softcap=softcap, window=window, out=out, workspace=workspace)
    torch.cuda.synchronize()
    want, mass, err = _attention_reference(q, k, v, table, lens, D ** -0.5 if scale is None else scale, softcap, window)
    u = UNIT[dtype]
    longest = max(c + n for c, n in lens)
    bound = u * want.abs() * 1.01 + (1.125 * u + err) * mass + longest * 2.0 ** -25 * 6.0 / max(1, longest) ** 0.5 + 2.0 ** -24
    over = (out.cpu().double() - want).abs() - bound
    assert torch.isfinite(out).all()
    assert (over <= 0).all(), (float(over.max()), over.argmax())
    return out


LENGTHS = {"one": [(0, 1)], "decode": [(0, 1), (15, 1), (16, 1), (31, 1), (32, 1), (126, 1), (127, 1), (500, 1), (1000, 1)],
           "long": [(4999, 1), (3, 1)], "drafts": [(0, 5), (100, 3), (2, 4), (333, 5), (64, 1)], "chunk": [(70, 40), (0, 129), (1, 16)],
           "empty": [(0, 0), (5, 1), (20, 0), (0, 3), (0, 0)], "mixed": [(0, 200), (400, 1), (17, 1), (250, 66), (9, 1)]}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("lens", sorted(LENGTHS))
@pytest.mark.parametrize("Hq,Hk,D,ps,layout", [(8, 2, 128, 16, "head"), (8, 1, 64, 32, "token"), (3, 3, 256, 64, "head"), (14, 2, 128, 128, "token"),
                                               (40, 2, 64, 256, "head"), (16, 1, 256, 16, "token")])
def test_attention(rtn, dtype, lens, Hq, Hk, D, ps, layout):
    _check_attention(rtn, dtype, LENGTHS[lens], Hq, Hk, D, ps, layout, seed=len(lens))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("lens", ["decode", "chunk", "drafts", "mixed", "long"])
@pytest.mark.parametrize("softcap,window", [(30.0, 0), (0.0, 1), (0.0, 16), (0.0, 37), (5.0, 100), (0.0, 5000)])
def test_attention_with_capped_scores_and_windows(rtn, dtype, lens, softcap, window):
    for Hq, Hk, D, ps in ((8, 2, 128, 16), (4, 2, 256, 32), (6, 1, 64, 64)):
        _check_attention(rtn, dtype, LENGTHS[lens], Hq, Hk, D, ps, softcap=softcap, window=window, seed=window)


@pytest.mark.gpu
@pytest.mark.parametrize("lens", ["decode", "mixed", "chunk"])
def test_attention_of_strided_queries_and_padded_batches(rtn, lens):
    out = _check_attention(rtn, torch.float16, LENGTHS[lens], 8, 2, 128, 16, extra=64)
    padded = _check_attention(rtn, torch.float16, LENGTHS[lens], 8, 2, 128, 16, padding=9)
    assert (padded[-9:] == 0).all() and out.shape[0] == padded.shape[0] - 9


@pytest.mark.gpu
@pytest.mark.parametrize("lens", ["decode", "mixed"])
def test_attention_with_sharp_and_flat_softmaxes(rtn, lens):
    _check_attention(rtn, torch.float16, LENGTHS[lens], 8, 2, 128, 16, scale_q=12.0)
    _check_attention(rtn, torch.bfloat16, LENGTHS[lens], 8, 2, 128, 16, scale=1e-4)


@pytest.mark.gpu
@pytest.mark.parametrize("lens", ["decode", "mixed", "chunk", "long"])
def test_attention_does_not_depend_on_the_bound_or_the_workspace(rtn, lens):
    """A wrong bound and no workspace cost time only."""
    none = torch.empty(0, dtype=torch.uint8, device=DEV)
    for kw in ({"max_new": 1}, {"max_new": 100000}, {"workspace": none}):
        _check_attention(rtn, torch.float16, LENGTHS[lens], 8, 2, 128, 16, **kw)


@pytest.mark.gpu
def test_attention_gives_zeros_where_nothing_is_seen(rtn):
    """Lengths below the number of new tokens: the first of them have no position."""
    q, k, v, table, seq, start = _attention_case(torch.float16, [(0, 6), (30, 1)], 8, 2, 128, 16)
    seq = seq.clone()
    seq[0] = 2
    out = torch.full(q.shape, float("nan"), dtype=q.dtype, device=DEV)
    rtn.rtn_paged_attention(q, rtn.PagedCache(k, v), table, seq, start, 6, out=out)
    want, mass, err = _attention_reference(q[4:], k, v, table, [(0, 2), (30, 1)], 128 ** -0.5, 0.0, 0)
    assert (out[:4] == 0).all()
    assert ((out[4:].cpu().double() - want).abs() <= 2.0 ** -10 * (want.abs() + mass) + 1e-5).all()


@pytest.mark.gpu
def test_attention_reads_no_page_outside_the_window(rtn):
    """Table entries of pages that have left every window may be stale, and the pages hold anything."""
    q, k, v, table, seq, start = _attention_case(torch.float16, [(400, 1), (300, 20)], 8, 2, 128, 16, seed=4)
    cache = rtn.PagedCache(k, v)
    a = rtn.rtn_paged_attention(q, cache, table, seq, start, 20, window=50).clone()
    first = [(400 - 49) // 16, (300 - 49) // 16]
    for b, n in enumerate(first):
        for pool in (k, v):
            pool[table[b, :n].long()] = float("nan")
        table[b, :n] = torch.tensor([-1, 2 ** 30, -2 ** 31, 7777] * 10, dtype=torch.int32, device=DEV)[:n]
    b = rtn.rtn_paged_attention(q, cache, table, seq, start, 20, window=50)
    assert torch.equal(a, b) and torch.isfinite(a).all()


@pytest.mark.gpu
def test_attention_and_rope_run_on_the_current_stream_and_replay(rtn):
    """A step captured in a graph -- plan in place, rotation with the cache write, attention -- replayed while the requests grow, against
    the same step by step."""
    B, Hq, Hk, D, ps, steps = 5, 8, 2, 128, 16, 40
    g = torch.Generator().manual_seed(0)
    rope = torch.randn(256, D, generator=g).to(DEV)
    inputs = torch.randn(steps, B, (Hq + 2 * Hk) * D, generator=g).half().to(DEV)
    results = []
    for captured in (False, True):
        k, v = (torch.zeros(40, Hk, ps, D, dtype=torch.float16, device=DEV) for _ in range(2))
        cache = rtn.PagedCache(k, v)
        table = torch.full((B, 8), -1, dtype=torch.int32, device=DEV)
        free = torch.randperm(40, generator=torch.Generator().manual_seed(1)).to(torch.int32).to(DEV)
        count = torch.tensor([40], dtype=torch.int32, device=DEV)
        lens = torch.tensor([0, 0, 0, 0, 0], dtype=torch.int32, device=DEV)
        step = torch.ones(B, dtype=torch.int32, device=DEV)
        plan = rtn.CachePlan.empty(B, B, DEV)._replace(seq_lens=lens, free_count=count)
        x = torch.empty_like(inputs[0])
        out = torch.empty(B, Hq, D, dtype=torch.float16, device=DEV)
        ws = torch.empty(max(16, rtn.rtn_paged_attention_workspace_nbytes(B, B, Hq, cache, 1)), dtype=torch.uint8, device=DEV)
        qbuf = torch.empty_like(out)

        def one():
            rtn.rtn_cache_plan(step, lens, table, free, count, ps, B, out=plan)
            rtn.rtn_rope_cache(x, Hq, rope, plan.positions, plan.slots, cache, out=qbuf)
            rtn.rtn_paged_attention(qbuf, cache, table, plan.seq_lens, plan.query_start, 1, out=out, workspace=ws)

        seen, graph = [], None
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for i in range(steps):
                x.copy_(inputs[i])
                if i == 17:
                    step[2] = -1                             # a request ends, and begins anew
                elif i == 18:
                    step[2] = 1
                if captured and graph is None and i == 2:
                    side.synchronize()
                    graph = torch.cuda.CUDAGraph()
                    with torch.cuda.graph(graph, stream=side):
                        one()
                if graph is not None:
                    graph.replay()
                else:
                    one()
                assert int(plan.status) == 0
                n = int(plan.query_start[-1])
                seen.append(out[:n].clone())
                torch.randn(1000, device=DEV).sum()           # the program's own work between replays
        side.synchronize()
        results.append(seen)
        assert lens.tolist() == [40, 40, 22, 40, 40]
    for a, b in zip(*results):
        assert torch.equal(a, b)


# ---- many requests, large pools, streams, the binding's two ways -----------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("B", [64, 65, 200, 300, 1100])
@pytest.mark.parametrize("chunks,window", [(0, 0), (3, 0), (3, 40)])
def test_attention_of_many_requests(rtn, B, chunks, window):
    """Up to 64 requests a wavefront finds its piece by itself, above a workgroup does, from 257 with several requests a thread."""
    rng = np.random.default_rng(B + chunks)
    lens = [(int(rng.integers(0, 90)), int(rng.integers(20, 60)) if i % (B // max(chunks, 1)) == 1 and chunks else int(rng.integers(0, 4))) for i in range(B)]
    lens[B // 2] = (3000, 1)
    _check_attention(rtn, torch.float16, lens, 4, 2, 64, 16, window=window, seed=B)


@pytest.mark.gpu
@pytest.mark.parametrize("Hq,Hk,new", [(64, 1, 1), (64, 1, 2), (7, 7, 70), (1, 1, 65), (30, 10, 3), (33, 1, 5)])
def test_attention_of_head_layouts(rtn, Hq, Hk, new):
    _check_attention(rtn, torch.bfloat16, [(300, new), (0, new), (77, max(1, new - 1))], Hq, Hk, 128, 32, seed=new)


@pytest.mark.gpu
@pytest.mark.parametrize("lens", ["long", "mixed", "chunk"])
def test_attention_with_every_size_of_workspace_is_right_and_repeats(rtn, lens):
    """Less workspace: fewer pieces.  The same workspace: the same bits."""
    args = _attention_case(torch.float16, LENGTHS[lens], 8, 2, 128, 16, seed=9)
    q, k, v, table, seq, start = args
    cache, new = rtn.PagedCache(k, v), max(n for _, n in LENGTHS[lens])
    full = rtn.rtn_paged_attention_workspace_nbytes(q.shape[0], len(LENGTHS[lens]), 8, cache, new)
    assert full > 0
    want, mass, err = _attention_reference(q, k, v, table, LENGTHS[lens], 128 ** -0.5, 0.0, 0)
    for nbytes in (0, 4096, full // 100 // 16 * 16, full // 7 // 16 * 16, full // 2 // 16 * 16, full):
        outs = []
        for _ in range(2):
            ws = torch.full((max(nbytes, 1),), 0xFF, dtype=torch.uint8, device=DEV)[:nbytes]      # (NaN patterns: nothing in it is read before it is written)
            outs.append(rtn.rtn_paged_attention(q, cache, table, seq, start, new, workspace=ws))
        assert torch.equal(outs[0], outs[1])
        assert ((outs[0].cpu().double() - want).abs() <= 2.0 ** -11 * (1.01 * want.abs() + 1.125 * mass) + err * mass + 6 * 2.0 ** -25 * 5000 ** -0.5 + 2.0 ** -24).all(), nbytes


@pytest.mark.gpu
def test_pools_beyond_32_bit_offsets(rtn):
    """Pages whose elements lie beyond 2^32 bytes and 2^31 elements of a pool: rotation writes there, attention reads there."""
    Hk, ps, D = 8, 16, 128
    pages = (2 ** 32 // 2 + 2 ** 28) // (Hk * ps * D)                  # 2^31 + 2^28 elements, 4.8 GB a pool
    k, v = (torch.zeros(pages, Hk, ps, D, dtype=torch.float16, device=DEV) for _ in range(2))
    cache = rtn.PagedCache(k, v)
    g = torch.Generator().manual_seed(3)
    ids = torch.tensor([pages - 1, 5, pages - 7, pages // 2 + 1], dtype=torch.int32)
    n, Hq = 60, 16
    qkv = torch.randn(n, (Hq + 2 * Hk) * D, generator=g).half().to(DEV)
    rope = torch.cat([torch.ones(64, D // 2), torch.zeros(64, D // 2)], 1).to(DEV)      # (no rotation)
    pos = torch.arange(n, dtype=torch.int32)
    slots = ids[pos.long() // ps] * ps + pos % ps
    q = rtn.rtn_rope_cache(qkv, Hq, rope, pos.to(DEV), slots.to(torch.int32).to(DEV), cache)
    heads = qkv.view(n, Hq + 2 * Hk, D)
    assert torch.equal(q, heads[:, :Hq])
    for pool, at in ((k, Hq), (v, Hq + Hk)):
        assert torch.equal(pool[ids.long().to(DEV)].transpose(1, 2).reshape(-1, Hk, D)[:n], heads[:, at:at + Hk])
    seq, start = torch.tensor([n], dtype=torch.int32, device=DEV), torch.tensor([0, n], dtype=torch.int32, device=DEV)
    far = rtn.rtn_paged_attention(q, cache, ids[None].to(DEV), seq, start, n)
    near = [torch.zeros(8, Hk, ps, D, dtype=torch.float16, device=DEV) for _ in range(2)]
    for pool, small in ((k, near[0]), (v, near[1])):
        small[:4] = pool[ids.long().to(DEV)]
    assert torch.equal(far, rtn.rtn_paged_attention(q, rtn.PagedCache(*near), torch.arange(4, dtype=torch.int32, device=DEV)[None], seq, start, n))


@pytest.mark.gpu
def test_native_calls_are_the_python_calls(rtn, monkeypatch):
    """The three calls by way of native code and by way of ctypes: the same launches, so the same bits; both on the stream that is current."""
    from paper_2505_15909_amd import binding
    if binding._native is None:
        pytest.skip("the native part of the binding is not built")
    q, k, v, table, seq, start = _attention_case(torch.bfloat16, LENGTHS["mixed"], 8, 2, 128, 16, layout="token")
    qkv = torch.randn(50, 12 * 128, device=DEV).bfloat16()
    rope = torch.randn(64, 96, device=DEV)
    norm = torch.rand(128, device=DEV).bfloat16()
    pos = torch.arange(50, dtype=torch.int32, device=DEV)
    case = _plan_case(1, 90, 16, 30, 200, 50, 0.2, 3)
    results, stream = [], torch.cuda.Stream()
    torch.cuda.synchronize()
    for native in (True, False):
        if not native:
            monkeypatch.setattr(binding, "_native", None)
        with torch.cuda.stream(stream):
            kk, vv = k.clone(), v.clone()
            cache = rtn.PagedCache(kk, vv)
            ws = torch.empty(rtn.rtn_paged_attention_workspace_nbytes(q.shape[0], 5, 8, cache, 200), dtype=torch.uint8, device=DEV)
            out = torch.empty_like(q)
            rtn.rtn_paged_attention(q, cache, table, seq, start, 200, softcap=20.0, window=100, out=out, workspace=ws)
            rot = rtn.rtn_rope_cache(qkv, 8, rope, pos, pos + 3, cache, norm, norm, eps=1e-5, interleaved=True, out=torch.empty(50, 8, 128, dtype=torch.bfloat16, device=DEV))
            plan = _run_plan(case)
        stream.synchronize()
        results.append([out, rot, kk.nan_to_num(), vv.nan_to_num()] + [torch.as_tensor(x) for x in plan])
    for a, b in zip(*results):
        assert torch.equal(a, b)
    # what is not plain goes to the Python code, and is refused there
    with pytest.raises(ValueError):
        rtn.rtn_paged_attention(q.float(), rtn.PagedCache(k, v), table, seq, start, 200, out=torch.empty_like(q), workspace=results[0][0])
    with pytest.raises(ValueError):
        rtn.rtn_rope_cache(qkv, 8, rope.half(), pos, pos, rtn.PagedCache(k, v), out=results[0][1])
    with pytest.raises(rtn.RtnError):
        rtn.rtn_rope_cache(qkv, 8, rope[:, :60].contiguous(), pos, pos, rtn.PagedCache(k, v), out=results[0][1])


@pytest.mark.gpu
def test_attention_block_with_quantised_projections(rtn):
    """The calls as a layer makes them: quantised QKV projection, rotation with the cache write, attention, quantised output projection, over two
    steps (a prompt, then a token), against the same in float64 on the dequantised weights."""
    from paper_2505_15909_amd import synth
    B, Hq, Hk, D, ps, hidden, bits, g = 3, 8, 2, 64, 16, 512, 4, 128
    Wqkv, Wo = synth.normal_weight((Hq + 2 * Hk) * D, hidden, 0.05, 1, DEV), synth.normal_weight(hidden, Hq * D, 0.05, 2, DEV)
    packed = [rtn.rtn_quantize(w, bits, g) for w in (Wqkv, Wo)]
    dense = [rtn.rtn_dequantize(*w, K, bits, g).cpu().double() for w, K in zip(packed, (hidden, Hq * D))]
    angle = torch.arange(64)[:, None] * 10000.0 ** (-torch.arange(0, D, 2) / D)[None]
    rope = torch.cat([angle.cos(), angle.sin()], 1).float().to(DEV)
    k, v = (torch.zeros(16, Hk, ps, D, dtype=torch.float16, device=DEV) for _ in range(2))
    cache = rtn.PagedCache(k, v)
    table = torch.full((B, 4), -1, dtype=torch.int32, device=DEV)
    free, count = torch.randperm(16, device=DEV).to(torch.int32), torch.tensor([16], dtype=torch.int32, device=DEV)
    lens, K64, V64 = torch.zeros(B, dtype=torch.int32, device=DEV), [None] * B, [None] * B
    for seed, new in ((3, [17, 5, 30]), (4, [1, 1, 1])):
        T = sum(new)
        x = synth.activation(T, hidden, seed, DEV)
        plan = rtn.rtn_cache_plan(torch.tensor(new, dtype=torch.int32, device=DEV), lens, table, free, count, ps, T)
        qkv = rtn.rtn_linear(x, *packed[0], bits, g)
        q = rtn.rtn_rope_cache(qkv, Hq, rope, plan.positions, plan.slots, cache)
        att = rtn.rtn_paged_attention(q, cache, table, plan.seq_lens, plan.query_start, max(new))
        out = rtn.rtn_linear(att.view(T, Hq * D), *packed[1], bits, g)
        assert int(plan.status) == 0
        lens, count = plan.seq_lens, plan.free_count
        y = (x.cpu().double() @ dense[0].T).view(T, -1, D)
        positions, at, ref = plan.positions.cpu(), 0, torch.zeros(T, Hq, D, dtype=torch.float64)
        rot, _ = _rotated(y[:, :Hq + Hk], None, rope.cpu(), positions, D, False, 1e-6)
        for b, n in enumerate(new):
            s = slice(at, at + n)
            K64[b] = rot[s, Hq:] if K64[b] is None else torch.cat([K64[b], rot[s, Hq:]])
            V64[b] = y[s, Hq + Hk:] if V64[b] is None else torch.cat([V64[b], y[s, Hq + Hk:]])
            for h in range(Hq):
                sc = rot[s, h] @ K64[b][:, h // 4].T * D ** -0.5
                sc = sc.masked_fill(torch.arange(len(K64[b]))[None] > positions[s][:, None], -np.inf)
                ref[s, h] = torch.softmax(sc, -1) @ V64[b][:, h // 4]
            at += n
        ref = ref.reshape(T, -1) @ dense[1].T
        # fp16 roundings of qkv, queries, keys, weights, attention and result: a few 2^-11 of the norms
        assert (out.cpu().double() - ref).norm() <= 6 * 2.0 ** -11 * ref.norm()


@pytest.mark.gpu
@pytest.mark.parametrize("lens", ["decode", "mixed"])
def test_attention_in_windows_wider_than_any_length(rtn, lens):
    """The widest window is no window, also where a length is below the number of new tokens."""
    q, k, v, table, seq, start = _attention_case(torch.float16, LENGTHS[lens], 8, 2, 128, 16, seed=2)
    cache, new = rtn.PagedCache(k, v), max(n for _, n in LENGTHS[lens])
    seq = seq.clone()
    seq[0] = max(1, int(seq[0]) - 3)
    none = rtn.rtn_paged_attention(q, cache, table, seq, start, new)
    for window in (2 ** 31 - 1, 2 ** 30, 2 ** 30 - 1):
        assert torch.equal(rtn.rtn_paged_attention(q, cache, table, seq, start, new, window=window), none)


@pytest.mark.gpu
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("Hq,Hk,lens", [(4, 2, [(700, 1)]), (6, 2, [(900, 1)]), (14, 2, [(600, 1), (2000, 1)]), (10, 2, [(5000, 2)]), (10, 2, [(3000, 11)]), (8, 1, [(4000, 9)])])
def test_attention_joins_any_number_of_rows(rtn, D, Hq, Hk, lens):
    """Rows and parts that do not divide one another: a tile's rows are shared by as many workgroups as it has parts."""
    _check_attention(rtn, torch.float16, lens, Hq, Hk, D, 16, seed=Hq)
