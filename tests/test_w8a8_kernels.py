"""The 8-bit layer's product, kernel by kernel: what the compiler made of the counted waits, by the code of the built library; which kernel a call takes, by a
small host program around the plan (tests/host/w8a8_plan_driver.cpp); and every kernel, in every way in which a call can reach it, against a product in 64 bits.  The tolerance is that of
tests/test_w8a8.py: the sum is exact, it and its two products with scales are rounded in fp32 and then to the type."""
import bisect
import math
import os
import random
import re
import subprocess

import pytest
import torch

from tests.test_host_plans import PKG, ROOT, _code_objects
from tests.test_w8a8 import DEV, E, TINY, TYPES, UNIT, _bordered, _sides_are_left

STREAM, BLOCK, TILE = range(3)
WORKSPACE = 64 << 20


def _events(tools, code_object, named):
    """Of the kernels with this in their name, what matters for their loads, in the order of the code: {kernel: [(address, kind, value)]} with loads into
    LDS ("D"), other loads ("W"), stores ("X"), waits with the number of them that may be on their way behind, barriers, branches with their targets, ends,
    and where lanes are switched off, with the register that keeps them, and on again."""
    with open(code_object, "rb") as f:
        if named.encode() not in f.read():
            return {}
    text = subprocess.run([f"{tools}/llvm-objdump", "-d", "--no-show-raw-insn", code_object], check=True, capture_output=True, text=True, timeout=300).stdout
    kernels, code, base = {}, None, 0
    for line in text.split("\n"):
        what, _, where = line.strip().partition("//")
        what = what.strip()
        if where == "":
            start = re.match(r"([0-9a-f]+) <(\S+)>:", what)
            if start:
                base, code = int(start[1], 16), kernels.setdefault(start[2], []) if named in start[2] else None
        elif code is not None:
            address = int(where.split(":")[0], 16)
            if what.startswith(("buffer_", "global_", "flat_", "scratch_")):
                code.append((address, "D" if what.endswith(" lds") else "W" if "load" in what else "X", None))
            elif what.startswith("s_waitcnt") and "vmcnt" in what:
                code.append((address, "wait", int(re.search(r"vmcnt\((\d+)\)", what)[1])))
            elif what.startswith("s_barrier"):
                code.append((address, "barrier", None))
            elif what.startswith(("s_branch", "s_cbranch")):
                target = re.search(r"<\S+?(?:\+0x([0-9a-f]+))?>\s*$", where)
                code.append((address, what.split()[0], base + int(target[1] or "0", 16)))
            elif what.startswith("s_endpgm"):
                code.append((address, "end", None))
            elif "saveexec" in what:
                code.append((address, "save", what.split()[1].rstrip(",")))
            elif re.match(r"\S+ exec,", what):
                code.append((address, "exec", what.split()[3] if what.startswith("s_or_b64 exec, exec, ") else None))
    return kernels


def _faulty_barriers(code, loads_to_lds, each):
    """Follows every way through a block kernel.  A request is `loads_to_lds` loads into LDS (D) and the loads of its weights into registers (W), `each` in
    all; barrier k says that request k has landed, so that what is on its way there has to be whole requests behind that one.  Returns the barriers, by
    address, with anything else on its way.  (While no lane is switched off, `execnz` is every
    wavefront's way and `execz` none's.)"""
    addresses = [a for a, _, _ in code]
    request = "D" * loads_to_lds + "W" * (each - loads_to_lds)
    todo, seen, wrong = [(0, "", 0, "")], set(), {}
    while todo:
        i, flying, ahead, kept = todo.pop()                 # ahead: loads into LDS of requests that no barrier has spoken for
        while (i, flying, ahead, kept) not in seen:
            seen.add((i, flying, ahead, kept))
            address, kind, value = code[i]
            if kind in "DWX":
                flying, ahead = flying + kind, ahead + (kind == "D")
            elif kind == "wait":
                flying = flying[max(0, len(flying) - value):]
            elif kind == "barrier":
                if flying and (flying != request * (len(flying) // each) or len(flying) // each >= ahead // loads_to_lds):
                    wrong[address] = (flying, ahead // loads_to_lds)
                ahead = max(0, ahead - loads_to_lds)
            elif kind == "end":
                break
            elif kind == "save":                             # kept: the register with the lanes that a wavefront began with, while some are off
                kept = kept or value
            elif kind == "exec":
                kept = "" if value == kept else kept or "none"
            elif kept or kind != "s_cbranch_execz":
                todo.append((bisect.bisect_left(addresses, value), flying, ahead, kept))
                if kind == "s_branch" or (not kept and kind == "s_cbranch_execnz"):
                    break
            i += 1
    return wrong


def test_block_kernels_wait_for_whole_requests(tmp_path):
    """A load that the compiler drops, adds or moves among those that a wait counts would leave a wavefront reading LDS that has not been written: on every way through every block
    kernel the loads behind a counted wait are the requests that it counts."""
    tools, objects = _code_objects(tmp_path)
    kernels = {}
    for o in objects:
        kernels.update(_events(tools, o, "w8a8_block_kernel"))
    assert len(kernels) >= 38
    wrong = {}
    for name, code in kernels.items():
        mb, nt, wk = map(int, re.search(r"ILi\d+ELi(\d+)ELi(\d+)ELi(\d+)E", name).groups())
        assert {"D", "W", "barrier", "end"} <= {kind for _, kind, _ in code}
        bad = _faulty_barriers(code, mb * wk // 4, mb * wk // 4 + 2 * nt)
        if bad:
            wrong[name] = bad
    assert not wrong, wrong


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    """plan([(M, N, K, bytes of workspace)]) -> the table of shapes [(kind, mb, nt, wk, depth)], [(shape, split, workgroups along N, along M)]"""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("no hipcc")
    exe = str(tmp_path_factory.mktemp("w8a8") / "plan")
    subprocess.run([hipcc, "-O1", "-std=c++17", "--offload-arch=gfx950", "-x", "hip", "-o", exe, os.path.join(ROOT, "tests", "host", "w8a8_plan_driver.cpp")],
                   check=True, capture_output=True, timeout=600)

    def ask(problems):
        out = subprocess.run([exe], input="".join("%d %d %d %d\n" % p for p in problems), check=True, capture_output=True, text=True, timeout=600).stdout
        return [[tuple(map(int, line.split())) for line in part.strip().split("\n")] for part in out.split("\n\n")]

    return ask


PROMPTS = [(M, N, K) for N, K in ((4096, 4096), (6144, 4096), (5120, 5120), (4096, 8192), (12288, 2048)) for M in (2576, 3000, 4112, 5000, 6144, 8192)]


def test_prompts_take_the_tile_kernels(plan):
    """Block kernels take 1.2 to 1.4 times as long there."""
    shapes, plans = plan([p + (WORKSPACE,) for p in PROMPTS])
    for problem, (shape, *_) in zip(PROMPTS, plans):
        assert shapes[shape][0] == TILE, problem


@pytest.mark.parametrize("sweep,mean", [("w8a8_sweep_results.txt", 0.02), ("w8a8_sweep_heldout.txt", 0.03)])
def test_picks_are_near_the_fastest_launch_measured(plan, sweep, mean):
    """Over the sweeps that are kept (which leave out what takes more than 1.6 times as long as the fastest): how far the plan's launch is behind, on the mean of
    logarithms; a split that was not measured counts as the slower of its neighbours."""
    problems = []
    for line in open(os.path.join(PKG, "tuning", sweep)):
        if not line.startswith("#"):
            head, *cells = line.split(" | ")
            times = {tuple(map(int, c.split()[0].split("/"))): float(c.split()[1].rstrip("*")) for c in cells}
            problems.append((tuple(map(int, head.split())), times))
    assert len(problems) > 700
    behind = []
    for (problem, times), (shape, split, *_) in zip(problems, plan([p + (WORKSPACE,) for p, _ in problems])[1]):
        near = [(shape, split)] if split not in (5, 7) or (shape, split) in times else [(shape, split - 1), (shape, split + 1)]
        took = [times[n] for n in near if n in times]
        assert took, (problem, shape, split)
        behind.append(math.log(max(took) / min(times.values())))
    assert sum(behind) / len(behind) <= mean


# M, N, K and MiB of workspace: calls that between them reach all that _reached tells apart (the CPU test below says when the plan has moved away from them).
SIZES = [
    (1, 16, 256, 64), (1, 16, 3840, 64), (1, 16, 4864, 4), (1, 16, 5888, 64), (1, 16, 8448, 4), (1, 4144, 1792, 4), (1, 4240, 2816, 64), (1, 8208,
    768, 64), (1, 82640, 2816, 64), (2, 528, 7424, 64), (2, 9008, 15872, 64), (2, 16800, 8960, 64), (2, 25184, 6912, 64), (3, 16, 34816, 0), (3,
    32912, 4864, 4), (7, 8288, 13056, 4), (7, 8416, 2816, 64), (8, 8848, 2304, 0), (11, 16, 2816, 4), (12, 16, 4352, 64), (12, 41520, 256, 64), (15,
    2064, 10496, 64), (17, 16, 2816, 64), (17, 736, 5632, 4), (17, 1056, 12800, 64), (17, 1136, 6912, 64), (17, 2096, 256, 4), (17, 24656, 1024, 64),
    (17, 25056, 256, 64), (17, 27168, 768, 4), (18, 16, 3584, 64), (18, 16, 12800, 64), (18, 2576, 8704, 64), (18, 65552, 256, 64), (19, 57456, 512,
    4), (20, 16, 1792, 4), (20, 2752, 11520, 64), (29, 16, 10752, 0), (33, 2720, 12544, 0), (33, 4608, 2560, 64), (33, 16416, 256, 64), (33, 51856,
    2304, 64), (34, 16, 16128, 0), (34, 1680, 8704, 64), (35, 576, 6400, 64), (35, 16976, 7168, 64), (36, 3088, 49408, 64), (36, 16544, 5632, 64),
    (40, 5312, 7424, 64), (53, 208, 4352, 4), (61, 688, 48896, 64), (62, 4464, 256, 0), (63, 1056, 39680, 4), (65, 8800, 1536, 0), (65, 9328, 3840,
    64), (65, 11392, 4608, 64), (66, 1712, 19712, 64), (66, 2128, 15872, 64), (66, 3024, 11520, 0), (66, 4160, 11776, 64), (66, 19392, 1792, 0), (66,
    84000, 512, 64), (67, 4752, 7168, 64), (67, 8416, 512, 64), (67, 17232, 2048, 64), (67, 49744, 512, 4), (69, 3136, 20736, 4), (69, 14912, 2304,
    4), (69, 66144, 1024, 64), (70, 16944, 8448, 64), (71, 880, 6400, 64), (73, 8448, 1280, 64), (103, 8304, 5632, 64), (128, 17232, 8192, 64), (129,
    16, 256, 64), (129, 16, 512, 4), (129, 16, 2560, 64), (129, 16, 2816, 64), (129, 65872, 512, 64), (130, 1648, 256, 64), (130, 66224, 256, 64),
    (131, 10912, 14336, 64), (131, 33808, 1024, 0), (131, 68448, 768, 64), (132, 16, 8960, 64), (132, 5600, 28672, 64), (132, 13168, 2560, 64), (133,
    2976, 15104, 64), (133, 65792, 1024, 0), (136, 11872, 2304, 4), (136, 33936, 768, 64), (137, 33296, 512, 64), (137, 34128, 256, 64), (137, 65952,
    1792, 64), (137, 66672, 1280, 4), (151, 1968, 21248, 4), (221, 1312, 13056, 4), (259, 32848, 1024, 64), (259, 32976, 256, 64), (266, 34176, 1792,
    0), (268, 33264, 1536, 4), (270, 32832, 1280, 64), (275, 33136, 512, 64), (282, 33280, 768, 64), (410, 33424, 1536, 64), (829, 48, 24320, 64),
    (1326, 48, 5888, 64), (1585, 16, 23808, 64), (1686, 16, 10496, 64), (2725, 80, 6144, 64), (2793, 80, 32512, 64), (3101, 16, 7936, 4), (4187, 208,
    5632, 64), (5926, 80, 11776, 64), (6004, 144, 7424, 64), (6077, 272, 9984, 64), (8202, 16, 512, 64), (8219, 80, 256, 64), (8268, 48, 512, 0),
    (8513, 272, 768, 64), (8625, 272, 1024, 4), (8689, 272, 256, 4), (8709, 80, 5632, 4), (8913, 208, 2560, 0)
]


def _ceil(a, b):
    return -(-a // b)


def _reached(problem, plan, shapes):
    """What a call tries of its kernel: split or not, one row tile or several (and whether their weights fit the L2s); the numbers of steps with their remainders, of
    tiles in one round and in several; rows and columns that end inside a workgroup's."""
    (M, N, K, _), (shape, split, XB, YB) = problem, plan
    kind, mb, nt, wk, depth = shapes[shape]
    rows, columns, unit = ((16 * mb, 16 * nt, 64), (16 * mb, 128 * nt // max(1, wk), 128), (32 * mb, 256, 256))[kind]
    reached = {("launch", shape, split > 1, YB > 1, kind == BLOCK and YB > 1 and N * K > 32 << 20)}
    units = K // unit
    for u in {units * (z + 1) // split - units * z // split for z in range(split)}:
        if kind == STREAM:                                   # tiles of a wavefront
            reached |= {("steps", shape, n if n <= 2 * depth else 2 * depth + 1 + n % depth) for n in {max(0, _ceil(u - w, wk)) for w in range(wk)}}
        elif kind == BLOCK:
            steps = _ceil(u, wk)
            reached.add(("steps", shape, steps if steps < 4 else 4 + steps % 3, u % wk != 0))
        else:
            reached.add(("steps", shape, 2 * u if u <= 4 else 10 + 2 * u % 6, XB * YB * split <= 256))
    return reached | ({("rows end inside", shape)} if M % rows else set()) | ({("columns end inside", shape)} if N % columns else set())


def test_the_sizes_below_reach_every_kernel_in_every_way(plan):
    r = random.Random(11)

    def spread(lo, hi):
        return int(round(math.exp(r.uniform(math.log(lo), math.log(hi)))))

    calls = [(spread(1, 9000), 16 * spread(1, 6656), 256 * spread(1, 208), r.choice([WORKSPACE] * 4 + [0, 4 << 20])) for _ in range(40000)]
    calls = [c for c in calls if c[1] * c[2] < 0x7FFF0000]
    own = [(M, N, K, mib << 20) for M, N, K, mib in SIZES]
    shapes, plans = plan(own + calls)
    there = set().union(*(_reached(c, p, shapes) for c, p in zip(own, plans)))
    assert {k[1] for k in there} == set(range(len(shapes)))                             # and no shape that no call takes
    assert {(k[1], k[2]) for k in there if k[0] == "launch"} >= {(i, split) for i, s in enumerate(shapes) for split in (False, True) if s[0] != STREAM}
    missing = {}
    for c, p in zip(calls, plans[len(own):]):
        for k in _reached(c, p, shapes) - there:
            missing.setdefault(k, c)
    assert not missing, missing


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K,mib", SIZES)
def test_every_kernel_in_every_way(rtn, M, N, K, mib):
    g = torch.Generator(device=DEV).manual_seed(M + N + K)
    q = torch.randint(-128, 128, (M, K), generator=g, device=DEV, dtype=torch.int8)
    qweight = torch.randint(0, 256, (N * K,), generator=g, device=DEV, dtype=torch.uint8)
    row_scales = torch.rand(M, generator=g, device=DEV) * 0.02 + 0.001
    scales = (torch.rand(N, 1, generator=g, device=DEV) * 1e-4 + 1e-5).half()
    want = q.double() @ rtn.rtn_unpack(qweight, N, K, 8).view(N, K).double().t().contiguous()             # below 2^53: exact
    want *= row_scales.double()[:, None] * scales.double()[:, 0][None]
    workspace = torch.empty(max(16, mib << 20), dtype=torch.uint8, device=DEV)
    for dtype in TYPES:
        whole, out = _bordered(M, N, dtype)
        rtn.rtn_linear_w8a8(q, row_scales, qweight, scales, out=out, workspace=workspace)
        assert ((out.double() - want).abs() <= (UNIT[dtype] + 3 * E * (1 + UNIT[dtype])) * want.abs() + TINY[dtype]).all()
        _sides_are_left(whole)
