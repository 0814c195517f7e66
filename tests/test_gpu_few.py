"""The layer for few tokens against 64 bits, in bf16 and 4-bit weights, and against MoELayer."""
from __future__ import annotations

import pytest
import torch

import paper_2606_21712_amd as moe
from gpu_util import log, weight_tol
from test_gpu_int4 import dense64, random_int4, standard

pytestmark = pytest.mark.gpu


def route64(logits, k, renorm):
    """Ids (ties to the lower expert) and gate weights in 64 bits."""
    top, ids = torch.sort(logits, dim=1, descending=True, stable=True)
    p = torch.softmax(logits.double(), 1).gather(1, ids[:, :k])
    return ids[:, :k], p / p.sum(1, keepdim=True) if renorm else p


def layer64(x, ids, gate, w):
    """y, and the bound of the bf16 roundings: h to 2^-9 of each value, y to 2^-9."""
    x = x.double()

    def swiglu(rows, ws, scale):
        g, u = rows @ ws[0].T, rows @ ws[1].T
        h = scale * (g * torch.sigmoid(g) * u)
        return h @ ws[2].T, h.abs() @ ws[2].abs().T

    y = torch.zeros_like(x)
    mag = torch.zeros_like(x)
    for e in range(w[0].shape[0]):
        t, j = torch.where(ids == e)
        if len(t):
            a, b = swiglu(x[t], [m[e] for m in w[:3]], gate[t, j, None])
            y[t] += a
            mag[t] += b
    if len(w) > 3:
        a, b = swiglu(x, [m[0] for m in w[3:]], 1.0)
        y += a
        mag += b
    # the fp32 sums and the hardware reciprocal and exponential in silu: some 1e-5 of the terms
    return y, 2.0 ** -8 * y.abs() + (2.0 ** -9 + 2e-5) * mag


def inputs(T, H, E, k, F, Fs, seed):
    r = torch.Generator().manual_seed(seed)
    x = torch.randn(T, H, generator=r).to(torch.bfloat16)
    logits = torch.randn(T, E, generator=r)
    if T > 1:
        logits[1] = logits[1].round()               # ties
    shapes = [(E, F, H), (E, F, H), (E, H, F)] + ([(1, Fs, H), (1, Fs, H), (1, H, Fs)] if Fs else [])
    return x, logits, shapes, r


CASES = [  # T, H, E, k, F, Fs, renorm
    (1, 64, 1, 1, 64, 0, 1), (1, 256, 8, 2, 512, 0, 1), (2, 64, 4, 4, 128, 64, 0), (3, 448, 8, 2, 192, 0, 0),
    (5, 256, 60, 4, 320, 256, 1), (8, 1024, 64, 8, 128, 128, 1), (13, 320, 64, 16, 64, 0, 0), (16, 512, 65, 5, 192, 64, 1),
    (16, 256, 256, 16, 64, 0, 1), (15, 2112, 16, 1, 1088, 0, 1), (7, 704, 129, 8, 256, 448, 0),
]


@pytest.mark.parametrize("T,H,E,k,F,Fs,renorm", CASES)
def test_bf16(T, H, E, k, F, Fs, renorm):
    log(f"[gpu] few bf16 T={T} H={H} E={E} k={k} F={F} Fs={Fs} renorm={renorm}")
    x, logits, shapes, r = inputs(T, H, E, k, F, Fs, T + H)
    w = [(torch.randn(s, generator=r) * s[2] ** -0.5).to(torch.bfloat16) for s in shapes]
    y, ids, gate = moe.moe_few_tokens(x.cuda(), logits.cuda(), k, *[t.cuda() for t in w], renormalize=renorm)
    ids64, gate64 = route64(logits, k, renorm)
    assert torch.equal(ids.cpu().long(), ids64)
    assert ((gate.cpu().double() - gate64).abs() <= weight_tol(k, E)).all()
    ref, bound = layer64(x, ids64, gate64, [t.double() for t in w])
    assert ((y.cpu().double() - ref).abs() <= bound).all()


@pytest.mark.parametrize("T,H,E,k,F,Fs,renorm", CASES)
@pytest.mark.parametrize("g", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
def test_int4(T, H, E, k, F, Fs, renorm, g, zeros):
    if any(n % g for n in (H, F, Fs)):
        H, F, Fs = (-(-n // g) * g for n in (H, F, Fs))
    log(f"[gpu] few int4 T={T} H={H} E={E} k={k} F={F} Fs={Fs} g={g} zeros={zeros}")
    x, logits, shapes, _ = inputs(T, H, E, k, F, Fs, T + F)
    dev, ref_w = [], []
    for i, s in enumerate(shapes):
        one = [random_int4(s[1], s[2], g, zeros, 100 * i + e) for e in range(s[0])]
        q, sc = (torch.stack([o[j] for o in one]) for j in (0, 1))
        z = torch.stack([o[2] for o in one]) if zeros else None
        dev.append(moe.moe_pack_int4(standard(q).cuda(), sc.cuda(), None if z is None else z.cuda(), g))
        ref_w.append(torch.stack([dense64(*o, g) for o in one]))
    y, ids, gate = moe.moe_few_tokens(x.cuda(), logits.cuda(), k, *dev, renormalize=renorm)
    ids64, gate64 = route64(logits, k, renorm)
    assert torch.equal(ids.cpu().long(), ids64)
    ref, bound = layer64(x, ids64, gate64, ref_w)
    # the group sums carry codes as 128 + q: fp32 roundings of sums some 30 times the terms
    extra = 1e-3 * ref.square().mean().sqrt()
    assert ((y.cpu().double() - ref).abs() <= bound + extra).all()


@pytest.mark.parametrize("T,H,E,k,F,Fs", [(1, 256, 8, 2, 512, 0), (16, 1024, 64, 8, 256, 256)])
def test_like_the_layer(T, H, E, k, F, Fs):
    """MoELayerFew and MoELayer on the same inputs: equal routing, outputs within two roundings of h
    and y each; a smaller batch through the same object."""
    log(f"[gpu] few against MoELayer T={T}")
    x, logits, shapes, r = inputs(T, H, E, k, F, Fs, 9)
    w = [(torch.randn(s, generator=r) * s[2] ** -0.5).to(torch.bfloat16).cuda() for s in shapes]
    few, whole = moe.MoELayerFew(T, H, E, k, F, Fs), moe.MoELayer(T, H, E, k, F, Fs, gather=True)
    y = few.run(x.cuda(), logits.cuda(), *w).clone()
    ref = whole.run(x.cuda(), logits.cuda(), *w)
    assert torch.equal(few.topk_ids, whole.topk_ids) and torch.equal(few.topk_weights, whole.topk_weights)
    assert (y - ref).float().norm() <= 3 * 2.0 ** -9 * ref.float().norm()
    half = max(1, T // 2)
    # other tokens' experts change the order of the sums: fp32 roundings, then one of bf16 at most
    part = few.run(x[:half].cuda(), logits[:half].cuda(), *w)
    assert (part - y[:half]).float().norm() <= 2.0 ** -8 * y[:half].float().norm()
    assert torch.equal(few.topk_ids, whole.topk_ids[:half])


def test_odd_logits():
    """Infinite and NaN logits leave the call inside its buffers and the other tokens as they are."""
    log("[gpu] few: non-finite logits")
    x, logits, shapes, r = inputs(4, 128, 8, 2, 64, 0, 1)
    w = [(torch.randn(s, generator=r) * s[2] ** -0.5).to(torch.bfloat16).cuda() for s in shapes]
    y, ids, _ = moe.moe_few_tokens(x.cuda(), logits.cuda(), 2, *w)
    bad = logits.clone()
    bad[1] = float("nan")
    bad[2] = -float("inf")
    bad[1].view(torch.int32)[:4] = -1               # a NaN with every bit set
    y2, ids2, _ = moe.moe_few_tokens(x.cuda(), bad.cuda(), 2, *w)
    for t in (0, 3):                                # the sums' order may differ
        assert (y[t] - y2[t]).float().norm() <= 2.0 ** -8 * y[t].float().norm()
    assert ((ids2 >= 0) & (ids2 < 8)).all() and (ids2[:, 0] != ids2[:, 1]).all()


def test_graph_and_stream():
    """Captured and replayed with other work between, and on another stream: the eager bits."""
    log("[gpu] few: graph")
    x, logits, shapes, r = inputs(6, 256, 16, 4, 128, 128, 5)
    w = [(torch.randn(s, generator=r) * s[2] ** -0.5).to(torch.bfloat16).cuda() for s in shapes]
    layer = moe.MoELayerFew(6, 256, 16, 4, 128, 128)
    xd, ld = x.cuda(), logits.cuda()
    g = moe.LayerGraph(layer, xd, ld, *w)
    for i in range(4):
        xd.copy_(torch.randn(6, 256, generator=r).to(torch.bfloat16))
        ld.copy_(torch.randn(6, 16, generator=r))
        want = layer.run(xd, ld, *w).clone()
        layer.y.zero_()
        torch.cuda.synchronize()
        assert torch.equal(g.replay(), want), i
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    y = layer.run(xd, ld, *w, stream=st)
    torch.cuda.synchronize()
    assert torch.equal(y, want)


def test_refusals():
    x, logits, shapes, r = inputs(4, 128, 8, 2, 64, 0, 1)
    w = [torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in shapes]
    xd, ld = x.cuda(), logits.cuda()
    with pytest.raises(ValueError):
        moe.MoELayerFew(17, 128, 8, 2, 64)
    with pytest.raises(moe.MoEError) as e:
        moe.moe_few_tokens(xd.repeat(5, 1), ld.repeat(5, 1), 2, *w)
    assert e.value.status == 2
    with pytest.raises(ValueError):
        moe.moe_few_tokens(xd, ld, 2, w[0], w[1], w[1])
    with pytest.raises(TypeError):
        moe.moe_few_tokens(xd.float(), ld, 2, *w)
    with pytest.raises(TypeError):
        moe.moe_few_tokens(xd, ld, 2, w[0], moe.quantize_weights_int4(w[1], 64), w[2])
    with pytest.raises(moe.MoEError) as e:
        moe.moe_few_tokens(xd, ld, 2, *w, ws=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 3
    y, ids, _ = moe.moe_few_tokens(xd[:0], ld[:0], 2, *w)
    assert y.shape == (0, 128)
