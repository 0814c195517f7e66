"""The rule that picks the kernel of a product of 8-bit codes (csrc/launch_rules.h), evaluated on the host.  CPU only."""
import os
import random
import shutil
import subprocess

import pytest

from int8_forms import FORMS, STREAMED

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2606_21712_amd", "csrc")
NAMES = ["few1", "few2", "few2x32", "32x128", "64x128", "96x128", "128x128", "160x256", "192x256", "256x256"]
MOST_T, MOST_N, MOST_K, MOST_OUT = 1 << 20, 1 << 24, 131056, 1 << 37

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")


@pytest.fixture(scope="session")
def plan(tmp_path_factory):
    """plan([(T, N, K, gated, compute units)]) -> [(form, parts, tiles, part_bytes, stream)]."""
    exe = str(tmp_path_factory.mktemp("plan") / "int8_plan")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, os.path.join(HERE, "native", "int8_plan.cpp"),
                    "-o", exe], check=True)

    def ask(cases):
        r = subprocess.run([exe], input="\n".join(" ".join(map(str, c)) for c in cases) + "\n", capture_output=True,
                           text=True, check=True)
        out = [[int(v) for v in line.split()] for line in r.stdout.splitlines()]
        assert len(out) == len(cases)
        return [(NAMES[o[0]], *o[1:]) for o in out]
    return ask


def test_sizes_reach_their_kernels(plan):
    """What the GPU tests run, runs on the kernel that their table says; together they reach every kernel."""
    got = plan([f[2:] for f in FORMS])
    assert [g[:2] for g in got] == [f[:2] for f in FORMS]
    assert all(not g[4] for g in got)
    for gated in (0, 1):
        seen = {f[:2] for f in FORMS if f[5] == gated}
        assert seen >= {(n, 1) for n in NAMES[gated:]}
        assert seen >= {(n, p) for n in NAMES[3:7] for p in (2, 4)} and {("32x128", 8), ("64x128", 8)} <= seen
    got = plan([f[2:] for f in STREAMED])
    assert [g[0] for g in got] == [f[0] for f in STREAMED] and all(g[4] for g in got)
    assert {(f[0], f[5]) for f in STREAMED} >= {(n, g) for n in NAMES[1:7] for g in (0, 1)} | {("few1", 0)}


def test_launches_fit(plan):
    """Over all that the checks let through: fewer than 2^32 threads, parts of a stage at least, a workspace that
    stays small, few-row kernels and streaming loads only where they are meant."""
    r = random.Random(5)
    cases = [(MOST_T, MOST_OUT // MOST_T, 16, g, c) for g in (0, 1) for c in (1, 256)]
    cases += [(T, N, K, g, 256) for T in (1, 16, 128, 4096, MOST_T) for N in (1, 4096, MOST_N) for K in (16, MOST_K) for g in (0, 1)
              if T * N <= MOST_OUT]
    for _ in range(20000):
        T, N, K = (int(m ** r.random()) for m in (MOST_T, MOST_N, MOST_K // 16))
        if T * N <= MOST_OUT:
            cases.append((T, N, 16 * K, r.randint(0, 1), r.choice((1, 7, 64, 256, 304))))
    for c, (form, parts, tiles, part_bytes, stream) in zip(cases, plan(cases)):
        T, N, K, gated, cus = c
        stages = -(-K // 128)
        assert 1 <= parts <= min(8, stages), c
        if form.startswith("few"):
            assert T <= 128 and parts == 1 and -(-N // 16) * 512 < 1 << 32 and not (gated and form == "few1"), c
        else:
            rows, wrows = map(int, form.split("x"))
            assert tiles == -(-T // rows) * -(-N // (wrows // (1 + gated))) and tiles * parts < 1 << 24, c
            assert part_bytes == tiles * rows * wrows * 4, c
            assert parts == 1 or (parts * part_bytes <= 1 << 30 and parts * tiles <= 4 * 4 * cus), c
        assert not stream or (T <= 128 and N * K * (1 + gated) >= 64 << 20), c


# (T, N, K, gated): the kernel, where it was measured to be the fastest
LINES = [
    ((1, 4096, 14336, 0), "few1"), ((8, 2048, 7168, 1), "few2"), ((128, 3576, 10368, 1), "128x128"),
    ((700, 1408, 2816, 1), "64x128"), ((333, 6145, 4096, 0), "96x128"), ((1000, 4096, 4096, 0), "128x128"),
    ((2003, 4608, 7168, 0), "160x256"), ((16384, 4096, 14336, 0), "256x256"), ((8192, 14336, 4096, 1), "256x256"),
]


@pytest.mark.parametrize("case,form", LINES)
def test_lines(plan, case, form):
    assert plan([(*case, 256)])[0][0] == form


def test_launches_fit_whatever_the_budget(plan):
    """A budget may say more compute units than any device has: launches stay under 2^32 threads, the joins' (16 rows
    of a tile a workgroup of 256) among them."""
    r = random.Random(6)
    cases = []
    for _ in range(5000):
        T, N, K = (int(m ** r.random()) for m in (MOST_T, MOST_N, MOST_K // 16))
        if T * N <= MOST_OUT:
            cases.append((T, N, 16 * K, r.randint(0, 1), r.choice((1 << 12, 1 << 20, (1 << 31) - 1))))
    cases += [(MOST_T, 4096, MOST_K, g, (1 << 31) - 1) for g in (0, 1)] + [(2048, MOST_N, MOST_K, 0, (1 << 31) - 1)]
    for c, (form, parts, tiles, part_bytes, stream) in zip(cases, plan(cases)):
        assert tiles * parts * 256 < 1 << 32, c
        if parts > 1:
            assert tiles * (int(form.split("x")[0]) // 16) * 256 < 1 << 32 and parts * part_bytes < 1 << 63, c
