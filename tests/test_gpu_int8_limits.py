"""The dense half of a layer in 8-bit integers at the ends of what its contract promises."""
from __future__ import annotations

import pytest
import torch

import paper_2606_21712_amd as moe
from gpu_util import log
from test_gpu_int8 import BF, bits, check_join, gen, join, random_int8, sums

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


def forms():
    """Rows, channels and columns that run on every kind of kernel: few rows, small tiles whole and in parts, large tiles."""
    return [(5, 40, 256), (30, 3003, 1040), (90, 260, 1040), (150, 520, 8208), (700, 6000, 2064), (3000, 4100, 4112)]


@pytest.mark.parametrize("T,N,K", forms())
def test_scales_are_applied_one_after_the_other(T, N, K):
    """The token's scale first, bit for bit, also where the product of the scales lies under the smallest fp32 number."""
    log(f"[gpu] matmul int8: order of the scales, {T} x {N} x {K}")
    x, _ = random_int8(T, K, 1)
    w, _ = random_int8(N, K, 2)
    s = sums(x, w)
    for a, b in ((2.0 ** -75, 2.0 ** -75), (2.0 ** -40, 2.0 ** 50), (2.0 ** 20, 2.0 ** -140)):
        y = moe.moe_matmul_int8(x.cuda(), torch.full((T,), a).cuda(), moe.moe_pack_int8(w.cuda(), torch.full((N,), b).cuda()))
        want = (s.float() * torch.tensor(a) * torch.tensor(b)).to(BF)
        assert torch.equal(bits(y.cpu()), bits(want)), (a, b)
