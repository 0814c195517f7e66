"""The operators for few sequences: every variant of the attention kernel, batches of more sequences than a wavefront
looks over at once, and roundings as few as their contracts say."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2606_21712_amd as moe
from gpu_util import log
from test_gpu_few import inputs, layer64, route64
from test_gpu_kv8 import HostCache, attention64, filled, i32

pytestmark = pytest.mark.gpu


@pytest.fixture
def budget():
    yield moe.set_cu_budget
    moe.set_cu_budget(0)


def plan(B, Hq, Hkv, D, new, length, window, cus):
    """The plan of an attention call, restated: rows of a tile, and whether tiles are cut."""
    rows, seen = new * (Hq // Hkv), min(length, window + new) if window else length

    def tiles(of):
        return B * Hkv * -(-rows // of)

    chunks = -(-seen // 64)
    if tiles(16) * chunks <= 8 * cus:
        of = 16
    elif rows > 16 and (rows <= 64 or tiles(32) * chunks <= 12 * cus):
        of = 32
    else:
        of = 16 if rows <= 16 else 128
    return of, tiles(of) < 2 * cus and seen > (1024 if D <= 128 or of == 128 else 512)


@pytest.mark.parametrize("window", [0, 1100])
@pytest.mark.parametrize("cus,cut", [(3, False), (12, True)])
@pytest.mark.parametrize("new,rows", [(1, 16), (9, 32), (40, 128)])
@pytest.mark.parametrize("page", [16, 32, 64, 96])       # pages of whole steps of 64 or of 32 tokens, and of neither
@pytest.mark.parametrize("D", [64, 128, 256])
def test_variants(budget, D, page, new, rows, cus, cut, window):
    """Head sizes, rows of a tile, kinds of pages, tiles whole and cut.  The bound: probabilities and outputs are
    rounded to bf16, 2^-8 of a number at most."""
    log(f"[gpu] attention variants D={D} page={page} new={new} cus={cus} window={window}")
    lens, Hq, Hkv = [1500, 40, 700], 8, 2
    assert plan(3, Hq, Hkv, D, new, max(lens), window, cus) == (rows, cut)
    rng = np.random.default_rng(D + page + new)
    host, table = filled(lens, Hkv, D, page, rng)
    q = torch.from_numpy(rng.standard_normal((3 * new, Hq, D)).astype(np.float32)).to(torch.bfloat16)
    budget(cus)
    out = moe.moe_kv8_attention(q.cuda(), host.device(), i32(table), i32(lens), i32([0, new, 2 * new, 3 * new]), new,
                                max(lens), window=window).cpu().double().numpy()
    ref, mag = attention64(q.double().numpy(), host, table, lens, [new] * 3, window, D ** -0.5)
    err = np.abs(out - ref)
    assert (err <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2e-5) * mag).all()
    # A rounding to bf16 is off by 1.66e-3 in the square mean (steps of 2^-7, over the logarithms of a mantissa: the
    # root of 2^-14 / 12 (1 - 1/4) / (2 ln 2)), one of independent probabilities in their weighted sum by no more
    # than that of its terms, the root of sum (p v)^2 <= |out| here, where values have random signs.  Both: 2.35e-3.
    # One such rounding more, of the same size, would make it 2.88e-3; 5000 numbers and more keep to 5%.
    assert np.linalg.norm(err) <= 1.05 * 2.35e-3 * np.linalg.norm(ref)


@pytest.mark.parametrize("B", [65, 130, 300])
@pytest.mark.parametrize("longest", [0, 4000])           # whole, and cut into parts
def test_many_sequences(B, longest):
    """More sequences than lanes: some of length 0, some without rows, long ones past the first 64."""
    log(f"[gpu] attention B={B} longest={longest}")
    rng = np.random.default_rng(B + longest)
    lens = [int(n) for n in rng.integers(1, 200, B)]
    new = [int(n) for n in rng.integers(0, 3, B)]
    for i in range(7, B, 10):
        lens[i] = 0
    for i in (3, B - 2):
        lens[i], new[i] = max(lens[i], longest), 1
    new = [n if lens[i] == 0 else min(n, lens[i]) for i, n in enumerate(new)]
    host, table = filled(lens, 1, 64, 16, rng)
    q = torch.from_numpy(rng.standard_normal((sum(new), 2, 64)).astype(np.float32)).to(torch.bfloat16)
    assert plan(B, 2, 1, 64, 2, max(lens), 0, 256)[1] == (longest > 0)
    out = moe.moe_kv8_attention(q.cuda(), host.device(), i32(table), i32(lens), i32(np.cumsum([0] + new)), 2,
                                max(lens)).cpu().double().numpy()
    ref, mag = attention64(q.double().numpy(), host, table, lens, new, 0, 0.125)
    assert (np.abs(out - ref) <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2e-5) * mag).all()
    none = np.repeat([n == 0 for n in lens], new)
    assert none.any() and not out[none].any()


@pytest.mark.parametrize("D,page", [(64, 16), (128, 64), (256, 16)])
def test_small_elements_of_a_query(D, page):
    """Elements far below a query row's largest: off by 2^-17 of that at most.  They are chosen so that each is off by
    that much, one half up and one down, against keys of opposite signs; two tokens' probabilities show it."""
    log(f"[gpu] attention: small elements of a query D={D}")
    half = (D - 2) // 2
    q = torch.zeros(1, 1, D, dtype=torch.float64)
    q[0, 0, 0] = 1.0                                        # the largest, 2^7 of the row's units
    q[0, 0, 2:2 + half] = (2.0 ** -4 + 2.0 ** -10) / 128
    q[0, 0, 2 + half:] = (2.0 ** -4 + 3 * 2.0 ** -10) / 128
    assert torch.equal(q.to(torch.bfloat16).double(), q)
    host = HostCache(1, 1, page, D)
    one = int(torch.ones(1).to(torch.float8_e4m3fn).view(torch.uint8))
    host.ke[0, 0, 0] = host.ve[0, 0, 0] = 127
    host.k[0, 0, 0, 2:2 + half], host.k[0, 0, 0, 2 + half:] = one, one | 0x80
    host.v[0, 0, 0, :, 0] = one                             # out: the first token's probability
    scale = 2.0 ** 16 / D
    out = moe.moe_kv8_attention(q.to(torch.bfloat16).cuda(), host.device(), i32([[0]]), i32([2]), i32([0, 1]), 1, 2,
                                scale=scale).cpu().double()
    score = float(q[0, 0, 2:2 + half].sum() - q[0, 0, 2 + half:].sum()) * scale
    got = torch.log(out / (1 - out))
    # the probability is rounded to bf16 twice, 2^-8 each
    assert ((got - score).abs() <= 2.0 ** -17 * (D - 2) * scale + 4 * 2.0 ** -8 / (1 - out)).all()


@pytest.mark.parametrize("T,H,E,k,F,Fs", [(3, 512, 8, 2, 1024, 0), (8, 1024, 16, 4, 512, 256), (16, 768, 32, 4, 640, 0)])
def test_one_rounding(T, H, E, k, F, Fs):
    """h keeps 16 significant bits and sums are fp32, so that y is the rounded value of the formula but where that
    lies next to a tie.  Before its rounding y is off by some 1e-5 of its own size (h by 2^-17 of its terms,
    silu's reciprocal and exponential by as much), against steps of 2^-8 to 2^-7: some 1% of the elements, those far
    below the others' size among them.  With h in bf16 it would be off by 1.7e-3, and a third would differ."""
    log(f"[gpu] few: one rounding T={T} H={H} F={F}")
    x, logits, shapes, r = inputs(T, H, E, k, F, Fs, T)
    w = [(torch.randn(s, generator=r) * s[2] ** -0.5).to(torch.bfloat16) for s in shapes]
    y = moe.moe_few_tokens(x.cuda(), logits.cuda(), k, *[t.cuda() for t in w])[0].cpu()
    ids, gate = route64(logits, k, 1)
    ref, _ = layer64(x, ids, gate, [t.double() for t in w])
    off = y != ref.to(torch.bfloat16)
    assert off.float().mean() <= 0.04
    assert ((y.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 1e-4 * ref.square().mean().sqrt()).all()
