"""The 8-bit layer's product, kernel by kernel: what the compiler made of the counted waits, by the code of the built library, and which kernel a call takes, by a
small host program around the plan (tests/host/w8a8_plan_driver.cpp); neither needs a GPU."""
import bisect
import math
import os
import re
import subprocess

import pytest

from tests.test_host_plans import PKG, ROOT, _code_objects

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
    assert len(kernels) >= 44
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
    """plan([(M, N, K, bytes of workspace)]) -> [(shape, kind, split, workgroups along N, along M)]"""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("no hipcc")
    exe = str(tmp_path_factory.mktemp("w8a8") / "plan")
    subprocess.run([hipcc, "-O1", "-std=c++17", "--offload-arch=gfx950", "-x", "hip", "-o", exe, os.path.join(ROOT, "tests", "host", "w8a8_plan_driver.cpp")],
                   check=True, capture_output=True, timeout=600)

    def ask(problems):
        out = subprocess.run([exe], input="".join("%d %d %d %d\n" % p for p in problems), check=True, capture_output=True, text=True, timeout=600).stdout.split("\n")
        return [tuple(map(int, line.split())) for line in out if line]

    return ask


PROMPTS = [(M, N, K) for N, K in ((4096, 4096), (6144, 4096), (5120, 5120), (4096, 8192), (12288, 2048)) for M in (2576, 3000, 4112, 5000, 6144, 8192)]


def test_prompts_take_the_tile_kernels(plan):
    """Block kernels take 1.2 to 1.4 times as long there."""
    for problem, (_, kind, *_) in zip(PROMPTS, plan([p + (WORKSPACE,) for p in PROMPTS])):
        assert kind == TILE, problem


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
    for (problem, times), (shape, _, split, *_) in zip(problems, plan([p + (WORKSPACE,) for p, _ in problems])):
        near = [(shape, split)] if split not in (5, 7) or (shape, split) in times else [(shape, split - 1), (shape, split + 1)]
        took = [times[n] for n in near if n in times]
        assert took, (problem, shape, split)
        behind.append(math.log(max(took) / min(times.values())))
    assert sum(behind) / len(behind) <= mean
