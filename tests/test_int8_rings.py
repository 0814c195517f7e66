"""Every end of a ring that the rule for products of 8-bit codes can lead to is run by a GPU test.  CPU only."""
import math
import random
import shutil

import pytest

from int8_forms import FORMS
from int8_rings import ENDS, ends
from test_int8_plan import plan          # noqa: F401 (a fixture)

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")


def keys(form, parts, K, gated):
    return {(form, gated, parts > 1, e) for e in ends(form, parts, K)}


def test_sizes_reach_their_kernels(plan):                                   # noqa: F811
    assert [g[:2] for g in plan([f[2:] for f in ENDS])] == [f[:2] for f in ENDS]


def test_every_end_is_run(plan):                                            # noqa: F811
    """Over sizes of all kinds at 256 compute units: the kernel, whether it is gated, whether its tiles are cut along k, and
    the steps it ends on."""
    r = random.Random(7)

    def between(lo, hi):
        return round(math.exp(r.uniform(math.log(lo), math.log(hi))))
    cases = []
    for _ in range(100000):
        T = between(*r.choice([(1, 20000), (1, 20000), (1, 1200), (100, 300)]))
        cases.append((T, between(16, 60000), 16 * between(1, r.choice([200, 8190])), r.randint(0, 1), 256))
    run = {k for f in FORMS + ENDS for k in keys(f[0], f[1], f[4], f[5])}
    met = {}
    for c, p in zip(cases, plan(cases)):
        for k in keys(p[0], p[1], c[2], c[3]):
            met.setdefault(k, c)
    assert len(met) > 150
    assert not {k: c for k, c in met.items() if k not in run}
