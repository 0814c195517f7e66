"""The kernels of int8 products hand a stage of x over at a barrier, after a counted s_waitcnt vmcnt(n) that leaves the n youngest
loads in flight.  The count is right only if that many loads were sent after the stage's: those to LDS stay where they are,
but loads to registers that nothing reads are dropped by the compiler, and loads that no scheduling barrier parts change places.
So the built code is walked here, with any number of stages, and the waits at the barriers alone have to do: where
the compiler puts others, which it may move, is left out.  CPU only."""
import os
import re
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_21712_amd", "csrc")
HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
LOAD = re.compile(r"(buffer|global|flat|scratch)_(load|store|atomic)")


def assembly(name, out):
    from paper_2606_21712_amd import build
    path = str(out / (name + ".s"))
    subprocess.run([HIPCC, *build.HIP_FLAGS, "-S", "--cuda-device-only", os.path.join(CSRC, name), "-o", path], check=True,
                   capture_output=True)
    with open(path) as f:
        return f.read()


def kernels(text, name):
    """{template arguments: instructions} of every instance of a kernel."""
    found = {}
    for part in re.split(r"^(?=_Z\S+:)", text, flags=re.M):
        m = re.match(r"_Z\S*\d" + name + r"I([^_]*?)EEv\S*:", part)
        if m:
            args = tuple(int(a) for a in re.findall(r"L[bi](\d+)E", m.group(1) + "E"))
            found[args] = events(part.split(".Lfunc_end")[0])
    return found


def events(text):
    """What matters of a kernel: labels, branches, loads to LDS and others, waits for loads, barriers, ends."""
    out = []
    for line in text.splitlines():
        t = line.split(";")[0].strip()
        if m := re.match(r"(\.LBB\w+):", t):
            out.append(("label", m.group(1)))
        elif m := re.match(r"s_(cbranch\w+|branch)\s+(\.LBB\w+)", t):
            out.append(("branch" if m.group(1) == "branch" else "either", m.group(2)))
        elif LOAD.match(t):
            out.append(("lds",) if re.search(r"\blds\b", t) else ("reg",))
        elif m := re.match(r"s_waitcnt\b.*vmcnt\((\d+)\)", t):
            out.append(("wait", int(m.group(1))))
        elif re.match(r"s_waitcnt\b|s_setprio|s_nop", t):
            pass
        elif t.startswith("s_barrier"):
            out.append(("barrier",))
        elif t.startswith("s_endpgm"):
            out.append(("end",))
        elif t and not t.startswith("."):
            out.append(("other",))
    # of the waits, those that a barrier follows
    return [e for i, e in enumerate(out) if e[0] != "other" and (e[0] != "wait" or out[i + 1:i + 2] == [("barrier",)])]


def walks(code, rounds=3):
    """Every way from the first load to LDS to the last load to LDS or barrier, loops taken up to `rounds` times."""
    at = {e[1]: i for i, e in enumerate(code) if e[0] == "label"}
    nexts = []
    for i, e in enumerate(code):
        n = [] if e[0] in ("end", "branch") else [i + 1]
        nexts.append([j for j in n + ([at[e[1]]] if e[0] in ("branch", "either") else []) if j < len(code)])
    ahead = {i for i, e in enumerate(code) if e[0] in ("lds", "barrier")}     # from where one of these is reached
    while more := {i for i, n in enumerate(nexts) if i not in ahead and any(j in ahead for j in n)}:
        ahead |= more
    stack = [(next(i for i, e in enumerate(code) if e[0] == "lds"), [], {})]
    while stack:
        i, way, seen = stack.pop()
        while i in ahead:
            way.append(code[i])
            if len(nexts[i]) == 2:
                back = [j for j in nexts[i] if j <= i]
                count = seen.get(i, 0)
                choices = [j for j in nexts[i] if j > i or count < rounds]
                seen = {**seen, i: count + 1} if back else seen
                for j in choices[1:]:
                    stack.append((j, list(way), seen))
                i = choices[0]
            else:
                i = nexts[i][0]
        yield way


def late(way, each):
    """(stage, steps) where a stage of `each` loads may still be on its way when the barrier before its reads is passed.
    Barrier 0 stands before the first step, barrier b in step b - 1: it hands over stage b, if there is one."""
    sent, barriers, pending, bad = 0, 0, [], []
    steps = sum(e[0] == "barrier" for e in way) - 1
    for e in way:
        if e[0] == "lds":
            pending.append(sent // each)
            sent += 1
        elif e[0] == "reg":
            pending.append(None)
        elif e[0] == "wait":
            pending = pending[len(pending) - e[1]:] if len(pending) > e[1] else pending
        elif e[0] == "barrier":
            if barriers in pending:
                bad.append((barriers, steps))
            barriers += 1
    return bad


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="needs hipcc")
def test_direct_kernels_wait_for_the_next_stage(tmp_path):
    found = kernels(assembly("int8_gemm.hip", tmp_path), "int8_direct_kernel")
    assert {a[1:3] for a in found} == {(2, 2), (4, 2), (6, 2), (8, 2), (10, 4)} and len(found) >= 26
    bad = {}
    for args, code in found.items():
        rows, ring = args[1], args[3]
        ways = list(walks(code))
        assert len({sum(e[0] == "barrier" for e in w) for w in ways}) > 2 * ring          # from no step to some rounds of the ring
        missing = sorted({b for w in ways for b in late(w, rows // 2)})
        if missing:
            bad[args] = missing
    assert not bad, bad


def test_the_walk_finds_late_stages():
    """Stages of two loads in a ring of three: one wait that is right, and the same one load too lax."""
    first = [("lds",)] * 2 + [("reg",)] + [("lds",)] * 2 + [("reg",)]
    step = [("reg",), ("wait", 0), ("barrier",)]
    for n, bad in ((4, []), (5, [(0, 1)])):
        assert late(first + [("wait", n), ("barrier",)] + step, 2) == bad
    assert late(first + [("wait", 4), ("barrier",), ("wait", 2), ("barrier",), ("wait", 0), ("barrier",)], 2) == [(1, 2)]
    assert late(first + [("wait", 4), ("barrier",), ("wait", 1), ("barrier",), ("wait", 0), ("barrier",)], 2) == []


def test_first_stages_of_the_large_tiles_are_pinned():
    """The wait before the first reads counts the loads of the second stage as the youngest.  They go to other LDS
    objects, so the scheduler may send them among the first stage's unless a barrier of its own stands between."""
    with open(os.path.join(CSRC, "int8_large.hip")) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    first = [m for m in re.finditer(r"issue_([xw])\(\1(\d), (\d), (\d)\);", text)]
    assert [(m.group(1), m.group(2), m.group(4)) for m in first] == [
        ("x", "0", "0"), ("x", "0", "1"), ("w", "0", "0"), ("w", "0", "1"), ("x", "1", "0"), ("x", "1", "1"), ("w", "1", "0")]
    for a, b in zip(first, first[1:]):
        if a.group(2) != b.group(2):
            assert "__builtin_amdgcn_sched_barrier(0);" in text[a.end():b.start()]
