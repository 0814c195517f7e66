"""The operators for few sequences where their launch rules turn: the rules count work against the
compute units, so a small budget of these brings every variant to small inputs.  References and bounds are those
of the operators' own tests."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2606_21712_amd as moe
from gpu_util import log
from test_gpu_few import inputs, layer64, route64
from test_gpu_int4 import dense64, on_gpu, random_int4, standard
from test_gpu_kv8 import HostCache, angles, attention64, filled, i32

pytestmark = pytest.mark.gpu


@pytest.fixture
def budget():
    yield moe.set_cu_budget
    moe.set_cu_budget(0)


# ---------------------------------------------------------------- 4-bit products
@pytest.mark.parametrize("cus", [1, 5, 12, 0])        # 13 row tiles: four, two and one share a workgroup's x
@pytest.mark.parametrize("T", [1, 16, 17, 32, 33, 70])
@pytest.mark.parametrize("N,K,g,zeros", [(203, 1120, 32, True), (205, 1088, 64, False), (196, 1280, 128, True)])
def test_matvec(budget, cus, T, N, K, g, zeros):
    log(f"[gpu] matvec rules cus={cus} T={T} {N}x{K} g={g}")
    q, s, z = random_int4(N, K, g, zeros, N)
    x = torch.randn(T, K, generator=torch.Generator().manual_seed(T)).to(torch.bfloat16)
    budget(cus)
    y = moe.moe_matvec_int4(x.cuda(), on_gpu(q, s, z, g)).cpu().double()
    ref = x.double() @ dense64(q, s, z, g).T
    assert ((y - ref).abs() <= 2.0 ** -8 * ref.abs() + 1e-3 * ref.square().mean().sqrt()).all()


# ---------------------------------------------------------------- the layer for few tokens
@pytest.mark.parametrize("cus", [1, 8, 64, 0])
@pytest.mark.parametrize("T,H,E,k,F,Fs", [(16, 256, 64, 8, 512, 128), (3, 512, 24, 8, 1024, 0), (9, 128, 8, 2, 2048, 2048),
                                          (8, 1024, 16, 4, 192, 64)])
def test_few(budget, cus, T, H, E, k, F, Fs):
    """Long down axes that are cut into parts, and units of the first kernel that a workgroup takes in
    turn."""
    log(f"[gpu] few rules cus={cus} T={T} H={H} E={E} k={k} F={F} Fs={Fs}")
    x, logits, shapes, r = inputs(T, H, E, k, F, Fs, T + F)
    w = [(torch.randn(s, generator=r) * s[2] ** -0.5).to(torch.bfloat16) for s in shapes]
    budget(cus)
    y, ids, _ = moe.moe_few_tokens(x.cuda(), logits.cuda(), k, *[t.cuda() for t in w])
    again, _, _ = moe.moe_few_tokens(x.cuda(), logits.cuda(), k, *[t.cuda() for t in w])
    assert torch.equal(y, again)
    ids64, gate64 = route64(logits, k, 1)
    assert torch.equal(ids.cpu().long(), ids64)
    ref, bound = layer64(x, ids64, gate64, [t.double() for t in w])
    assert ((y.cpu().double() - ref).abs() <= bound).all()


@pytest.mark.parametrize("cus", [1, 16, 0])
@pytest.mark.parametrize("T,H,E,k,F,Fs,g", [(16, 256, 32, 4, 512, 128, 64), (2, 512, 24, 8, 1024, 0, 128),
                                            (9, 192, 8, 2, 1600, 320, 32)])
def test_few_int4(budget, cus, T, H, E, k, F, Fs, g):
    log(f"[gpu] few int4 rules cus={cus} T={T} H={H} E={E} k={k} F={F} Fs={Fs} g={g}")
    x, logits, shapes, _ = inputs(T, H, E, k, F, Fs, T + F)
    dev, ref_w = [], []
    for i, s in enumerate(shapes):
        one = [random_int4(s[1], s[2], g, True, 100 * i + e) for e in range(s[0])]
        q, sc, z = (torch.stack([o[j] for o in one]) for j in range(3))
        dev.append(moe.moe_pack_int4(standard(q).cuda(), sc.cuda(), z.cuda(), g))
        ref_w.append(torch.stack([dense64(*o, g) for o in one]))
    budget(cus)
    y, ids, _ = moe.moe_few_tokens(x.cuda(), logits.cuda(), k, *dev)
    ids64, gate64 = route64(logits, k, 1)
    assert torch.equal(ids.cpu().long(), ids64)
    ref, bound = layer64(x, ids64, gate64, ref_w)
    assert ((y.cpu().double() - ref).abs() <= bound + 1e-3 * ref.square().mean().sqrt()).all()


# ---------------------------------------------------------------- attention
@pytest.mark.parametrize("cus", [1, 3, 12, 0])        # tiles of 128, 32 and 16 rows; whole and cut
@pytest.mark.parametrize("lens,new,Hq,Hkv,D,page,window", [
    ([300, 40], [70, 33], 4, 1, 128, 16, 0),
    ([1300, 7], [40, 5], 6, 2, 64, 64, 0),
    ([1200], [30], 8, 1, 256, 32, 0),
    ([1100, 1250], [9, 2], 8, 2, 128, 64, 0),
    ([1400, 30], [60, 30], 4, 1, 128, 128, 300),
    ([1500, 1, 16], [1, 1, 1], 8, 2, 128, 16, 0),
])
def test_attention(budget, cus, lens, new, Hq, Hkv, D, page, window):
    log(f"[gpu] attention rules cus={cus} lens={lens} new={new} Hq={Hq} Hkv={Hkv} D={D} page={page} window={window}")
    rng = np.random.default_rng(sum(lens) + D)
    host, table = filled(lens, Hkv, D, page, rng)
    q = torch.from_numpy(rng.standard_normal((sum(new), Hq, D)).astype(np.float32)).to(torch.bfloat16)
    scale = D ** -0.5
    budget(cus)
    out = moe.moe_kv8_attention(q.cuda(), host.device(), i32(table), i32(lens), i32(np.cumsum([0] + new)), max(new),
                                max(lens), window=window).cpu().double().numpy()
    ref, mag = attention64(q.double().numpy(), host, table, lens, new, window, scale)
    assert (np.abs(out - ref) <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2e-5) * mag).all()


def test_rows_outside():
    """Rows that cu_tokens puts before the first or after the last are left out, of the cache and the output."""
    log("[gpu] rows outside")
    rng = np.random.default_rng(5)
    dev = HostCache(3, 1, 16, 64).device()
    x = torch.from_numpy(rng.standard_normal((4, 1, 64)).astype(np.float32)).to(torch.bfloat16)
    cs = angles(64, 64)
    table, lens, cu = i32([[0], [1], [2]]), i32([3, 2, 4]), i32([-2, 1, 3, 7])   # the last has row 3 and three past it
    q = moe.moe_kv8_append(x.cuda(), x.cuda(), x.cuda(), torch.from_numpy(cs).cuda(), dev, table, lens, cu)
    out = torch.full((4, 1, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    moe.moe_kv8_attention(q, dev, table, lens, cu, 4, 4, out=out)
    torch.cuda.synchronize()
    codes = dev.k_codes.cpu().numpy()[:, 0]
    assert not codes[0, :2].any() and codes[0, 2].any()          # positions 0, 1: rows -2, -1
    assert codes[1, :2].any(1).all() and not codes[1, 2:].any()
    assert codes[2, 0].any() and not codes[2, 1:].any()
    assert (out != 7.0).any(-1).all()


# ---------------------------------------------------------------- another stream than the current one
@pytest.mark.parametrize("call", ["matvec", "few", "attention"])
def test_buffers_of_the_call_s_stream(call):
    """What a call on a given stream allocates is not memory that the current stream still reads."""
    log(f"[gpu] buffers on another stream: {call}")
    gen = torch.Generator(device="cuda").manual_seed(3)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16)

    if call == "matvec":
        x, w = normal(8, 256), moe.quantize_weights_int4(normal(2048, 256), 64)
        size, run = 8 * 2048 * 2, lambda st: moe.moe_matvec_int4(x, w, stream=st)
    elif call == "few":
        x, logits, w = normal(8, 256), normal(8, 8).float(), (normal(8, 512, 256), normal(8, 512, 256), normal(8, 256, 512))
        size = moe.moe_few_tokens_workspace_bytes(8, 256, 2, 512)
        run = lambda st: moe.moe_few_tokens(x, logits, 2, *w, stream=st)[0]  # noqa: E731
    else:
        host, table = filled([3000, 2000], 1, 64, 64, np.random.default_rng(1))
        cache, args = host.device(), (i32(table), i32([3000, 2000]), i32([0, 1, 2]), 1, 3000)
        q = normal(2, 4, 64)
        size = moe.moe_kv8_attention_workspace_bytes(2, 2, 4, 1, 64, 1, 3000)
        run = lambda st: moe.moe_kv8_attention(q, cache, *args, stream=st)  # noqa: E731
    assert size > 0
    want = run(None).clone()
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    busy = torch.full((size,), 77, dtype=torch.uint8, device="cuda")
    copy = torch.empty_like(busy)
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)              # some 50 ms
    copy.copy_(busy)
    del busy                                    # its memory is the current stream's next block of this size
    got = run(st)
    torch.cuda.synchronize()
    assert torch.equal(want, got)
    assert (copy == 77).all()
