"""The 8-bit layer's product, kernel by kernel: what the compiler made of the counted waits, by the code of the built library (no GPU)."""
import bisect
import re
import subprocess

from tests.test_host_plans import _code_objects


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
