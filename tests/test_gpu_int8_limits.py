"""The dense half of a layer in 8-bit integers at the ends of what its contract promises."""
from __future__ import annotations

import pytest
import torch

import paper_2606_21712_amd as moe
from gpu_util import log
from int8_rings import ENDS
from test_gpu_int8 import BF, bits, budget, check_join, check_product, gated_tolerance, gen, join, random_int8, sums      # noqa: F401 (budget is a fixture)

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


@pytest.mark.parametrize("form,parts,T,N,K,gated,cus", ENDS)
def test_every_end_of_a_ring(budget, form, parts, T, N, K, gated, cus):            # noqa: F811
    log(f"[gpu] int8 {form} in {parts}: {T} x {N} x {K} gated={gated}")
    budget(cus)
    check_product(T, N, K, gated)


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


@pytest.mark.parametrize("T,F,K", forms())
def test_gated_products_keep_rows_and_channels_apart(T, F, K):
    """A token's NaN scale shows in its row alone, a channel's infinite or NaN scale in its channel alone."""
    log(f"[gpu] gated int8: scales that are not finite, {T} x {F} x {K}")
    x, sx = random_int8(T, K, 5)
    (wg, sg), (wu, su) = random_int8(F, K, 6), random_int8(F, K, 7)
    run = lambda: moe.moe_gated_int8(x.cuda(), sx.cuda(), moe.moe_pack_int8(wg.cuda(), sg.cuda()),
                                     moe.moe_pack_int8(wu.cuda(), su.cuda())).cpu()
    want = run()
    sx[1], sg[3], su[17], sg[F - 1] = float("nan"), float("inf"), float("-inf"), float("nan")
    h = run()
    rows, channels = torch.arange(T) != 1, torch.ones(F, dtype=torch.bool)
    channels[[3, 17, F - 1]] = False
    assert h[1].isnan().all() and h[:, F - 1].isnan().all()
    assert not h[rows][:, 3].isfinite().any()
    assert torch.equal(bits(h[rows][:, channels]), bits(want[rows][:, channels])) and want.isfinite().all()


@pytest.mark.parametrize("T", [15, 30, 100, 1000, 3000])
def test_gated_products_of_gates_far_out(T):
    """Gates from -100 to 100 with an up projection of 5000.  The quotient 1 / (1 + exp(-g)) is taken as 0 below the smallest
    normal fp32 number, 2^-126: from g = -87.3 down h is off by up to 2^-126 |g u|, there and nowhere else."""
    log(f"[gpu] gated int8: gates far out, T={T}")
    F, K = 520, 64
    x = torch.zeros(T, K, dtype=torch.int8)
    x[:, 0] = 1
    sx = torch.linspace(0.5, 1.0, T)
    wg, wu = torch.zeros(F, K, dtype=torch.int8), torch.zeros(F, K, dtype=torch.int8)
    wg[:, 0] = (torch.arange(F) % 255 - 127).to(torch.int8)
    wu[:, 0] = 125
    sg, su = torch.full((F,), 100 / 127), torch.full((F,), 40.0)
    h = moe.moe_gated_int8(x.cuda(), sx.cuda(), moe.moe_pack_int8(wg.cuda(), sg.cuda()), moe.moe_pack_int8(wu.cuda(), su.cuda()))
    g, u = (sums(x, w) * sx.double()[:, None] * s.double() for w, s in ((wg, sg), (wu, su)))
    ref = g * torch.sigmoid(g) * u
    far = g < -87.3
    tol = gated_tolerance(g, u * 0, ref) + far * 2.0 ** -126 * (g * u).abs()      # u * 0: without the room for far gates
    assert far.any() and (g > 87.3).any()
    assert ((h.cpu().double() - ref).abs() <= tol).all()


@pytest.mark.parametrize("T", [1, 40, 300])
def test_gated_products_at_their_largest_sums(T):
    """All codes -128 and K as long as it may be: both sums are 2^31 - 2^18, times 2^-31 just under 1."""
    log(f"[gpu] gated int8: largest sums, T={T}")
    K, F = 131056, 48
    x = torch.full((T, K), -128, dtype=torch.int8, device="cuda")
    w = moe.moe_pack_int8(torch.full((F, K), -128, dtype=torch.int8, device="cuda"), torch.full((F,), 2.0 ** -15, device="cuda"))
    h = moe.moe_gated_int8(x, torch.full((T,), 2.0 ** -16, device="cuda"), w, w).cpu().double()
    g = torch.full((T, F), K * 2.0 ** 14 * 2.0 ** -31, dtype=torch.float64)
    ref = g * torch.sigmoid(g) * g
    assert ((h - ref).abs() <= gated_tolerance(g, g, ref)).all()


def test_a_projection_repeats_itself():
    """A norm join to codes and the product on them, over and over between other work and on two streams at once: the
    same bits every time."""
    log("[gpu] norm_join and matmul int8: repeats")
    T, N, H = 2003, 4608, 7168
    g = gen(9)
    x, y = (torch.randn(T, H, generator=g).to(BF).cuda() for _ in range(2))
    gate, pre = (torch.randn(H, generator=g).to(BF).cuda() for _ in range(2))
    w = moe.moe_pack_int8(*(t.cuda() for t in random_int8(N, H, 10)))

    def project():
        xo, z, s = moe.moe_norm_join(x, y, gate=gate, pre=pre, int8=True)
        return xo, z, s, moe.moe_matmul_int8(z, s, w)
    want = project()
    noise = torch.randn(4096, 4096, device="cuda")
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for i in range(6):
        noise = noise * 1.0001
        for st in streams:
            with torch.cuda.stream(st):
                got.append(project())
    torch.cuda.synchronize()
    for one in got:
        assert all(torch.equal(bits(a), bits(b)) for a, b in zip(one, want))
