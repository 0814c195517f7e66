"""The dense half of a layer in 8-bit integers at the ends of what its contract promises."""
from __future__ import annotations

import pytest
import torch

import paper_2606_21712_amd as moe
from gpu_util import log
from test_gpu_int8 import BF, check_join, gen, join

pytestmark = pytest.mark.gpu


def signs(T, H, seed):
    return torch.randint(0, 2, (T, H), generator=gen(seed)) * 2.0 - 1.0


def short_and_long_rows(H):
    """(rows, eps): the shortest rows that are promised, all elements or one of them at 2^-50, any row where eps
    holds it up, and the longest, whose squares sum to 2^127."""
    u = torch.rand(4, H, generator=gen(H)) + 1
    small = u * 2.0 ** -50 * signs(4, H, 1)
    one = u * 2.0 ** -64 * signs(4, H, 2)
    one[:, H // 3] = 2.0 ** -50
    tiny = u * 2.0 ** -90 * signs(4, H, 3)
    tiny[0] = 2.0 ** -126
    long = signs(4, H, 4) * 2.0 ** 63.5 / H ** 0.5
    return [(small, 0.0), (one, 0.0), (tiny, 2.0 ** -100), (long, 0.0), (long, 1e30)]


@pytest.mark.parametrize("H", [256, 4096, 7168, 32768])
@pytest.mark.parametrize("int8", [False, True])
def test_norms_of_the_shortest_and_longest_rows(H, int8):
    for i, (rows, eps) in enumerate(short_and_long_rows(H)):
        log(f"[gpu] norm_join: rows at the ends of fp32's squares, H={H} int8={int8} {i}")
        w = (1 + 0.3 * torch.randn(H, generator=gen(5))).to(BF)
        for x in (rows.to(BF), rows):
            args = (x, None, None, None, False, 1.0, w, 0.0, eps, int8)
            check_join(join(*args), *args)
        x = torch.randn(4, H, generator=gen(6)).to(BF)
        args = (x, rows.to(BF), w, None, False, 0.5, True, 0.0, eps, int8)       # as a block's output
        check_join(join(*args), *args)
