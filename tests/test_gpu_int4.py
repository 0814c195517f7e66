"""4-bit weights on the GPU: quantizing and packing against plain implementations bit for bit,
products with few rows against 64 bits."""
from __future__ import annotations

import pytest
import torch

import paper_2606_21712_amd as moe
from gpu_util import log

pytestmark = pytest.mark.gpu
GROUPS = (32, 64, 128)


def quantize_plain(w, g, zeros):
    """The definition, in fp32 on the host: codes 0..15 [N, K], scales, zeros."""
    N, K = w.shape
    v = w.float().reshape(N, K // g, g)
    lo, hi = v.amin(2).clamp_max(0), v.amax(2).clamp_min(0)
    s = ((hi - lo) / 15 if zeros else torch.maximum(hi, 0 - lo) / 7).to(torch.bfloat16)
    f = s.float()
    z = torch.where(f > 0, torch.round(-lo / f).clamp_max(15), torch.zeros_like(f)) if zeros else torch.full_like(f, 8)
    q = torch.where(f[..., None] > 0, torch.round(v / f[..., None]) + z[..., None], z[..., None]).clamp(0, 15)
    return q.reshape(N, K).to(torch.uint8), s, z.to(torch.uint8) if zeros else None


def standard(q):
    return q[..., 0::2] | (q[..., 1::2] << 4)


def pack_plain(q, s, z, g):
    """The packed layout, element by element from its description."""
    N, K = q.shape
    Np, Kp = -(-N // 16) * 16, -(-K // 128) * 128
    full = torch.full((Np, Kp), 8, dtype=torch.uint8)
    full[:N, :K] = q
    # [row tile, row, column tile, word j, lane group, column in the word]
    t = full.reshape(Np // 16, 16, Kp // 128, 4, 4, 8).permute(0, 2, 4, 1, 3, 5)
    # nibble p holds column 2 p, or 2 (p - 4) + 1
    t = t[..., [0, 2, 4, 6, 1, 3, 5, 7]]
    codes = (t[..., 0::2] | (t[..., 1::2] << 4)).reshape(-1)

    def spread(v, fill):
        out = torch.full((Np, Kp // g), fill, dtype=v.dtype)
        out[:N, :K // g] = v
        return out.reshape(Np // 16, 4, 4, Kp // 128, 128 // g).permute(0, 3, 1, 4, 2).reshape(-1)

    s = spread(s, 0).view(torch.int16).int()
    if z is not None:                                # words: the scale above, 128 + z in bf16 below
        s = (s << 16) | (spread(z, 8).float() + 128).to(torch.bfloat16).view(torch.int16).int()
    else:
        s = s.to(torch.int16)
    return codes, s.view(torch.uint8)


def random_int4(N, K, g, zeros, seed):
    r = torch.Generator().manual_seed(seed)
    q = torch.randint(0, 16, (N, K), generator=r, dtype=torch.uint8)
    s = (torch.rand((N, K // g), generator=r) + 0.5).mul(K ** -0.5 / 4).to(torch.bfloat16)
    z = torch.randint(0, 16, (N, K // g), generator=r, dtype=torch.uint8) if zeros else None
    return q, s, z


def on_gpu(q, s, z, g):
    return moe.moe_pack_int4(standard(q).cuda(), s.cuda(), None if z is None else z.cuda(), g)


def dense64(q, s, z, g):
    zz = 8.0 if z is None else z.double().repeat_interleave(g, 1)
    return (q.double() - zz) * s.double().repeat_interleave(g, 1)


@pytest.mark.parametrize("g", GROUPS)
@pytest.mark.parametrize("zeros", [False, True])
def test_quantize(g, zeros):
    """Codes, scales and zero points as the definition gives them, a group of zeros, one of one sign and
    one with an outlier among them."""
    log(f"[gpu] quantize int4 g={g} zeros={zeros}")
    w = torch.randn(37, 3 * g, generator=torch.Generator().manual_seed(g)).to(torch.bfloat16)
    w[0, :g] = 0
    w[1, :g] = w[1, :g].abs()
    w[2, g:2 * g] = -w[2, g:2 * g].abs()
    w[3, 5] = 1000.0
    codes, s, z = moe.moe_quantize_int4(w.cuda(), g, zeros)
    q_ref, s_ref, z_ref = quantize_plain(w, g, zeros)
    assert torch.equal(s.cpu().view(torch.int16), s_ref.view(torch.int16))
    assert torch.equal(codes.cpu(), standard(q_ref))
    assert z is None if not zeros else torch.equal(z.cpu(), z_ref)


@pytest.mark.parametrize("N,K,g", [(16, 128, 32), (1, 32, 32), (17, 64, 64), (100, 384, 128), (33, 352, 32),
                                   (5, 192, 64)])
@pytest.mark.parametrize("zeros", [False, True])
def test_pack(N, K, g, zeros):
    log(f"[gpu] pack int4 {N}x{K} g={g} zeros={zeros}")
    q, s, z = random_int4(N, K, g, zeros, N + K)
    w = on_gpu(q, s, z, g)
    codes, scales = pack_plain(q, s, z, g)
    assert torch.equal(w.codes.cpu(), codes)
    assert torch.equal(w.scales.cpu(), scales)
    # a tensor of several matrices is the matrices one after the other
    w2 = moe.moe_pack_int4(torch.stack([standard(q)] * 3).cuda(), torch.stack([s] * 3).cuda(),
                           None if z is None else torch.stack([z] * 3).cuda(), g)
    assert torch.equal(w2.codes, w.codes.repeat(3)) and torch.equal(w2.scales, w.scales.repeat(3))
    assert w2.shape == (3, N, K)


@pytest.mark.parametrize("T", [1, 2, 5, 15, 16, 17, 31, 33, 48, 64, 65, 130])
@pytest.mark.parametrize("N,K,g", [(1, 32, 32), (16, 128, 128), (100, 1024, 64), (203, 1120, 32), (1003, 2048, 128),
                                   (4096, 256, 64), (64, 16384, 128)])
def test_matvec(T, N, K, g):
    """Against 64 bits: one bf16 rounding (2^-9), and the fp32 sums.  A group's sum holds products of up
    to 143 |x|: their fp32 roundings, K of them in a random walk, stay under 1e-3 of the result's size
    (sqrt(K) 2^-24 143 against 4.6 for every unit of scale: 1.1e-3 worst at K = 16384 if all were of
    the largest sum's size; partial sums are smaller)."""
    zeros = (N + K) % 3 != 0
    log(f"[gpu] matvec int4 T={T} {N}x{K} g={g} zeros={zeros}")
    q, s, z = random_int4(N, K, g, zeros, T + N)
    x = torch.randn(T, K, generator=torch.Generator().manual_seed(T)).to(torch.bfloat16)
    y = moe.moe_matvec_int4(x.cuda(), on_gpu(q, s, z, g)).cpu().double()
    ref = x.double() @ dense64(q, s, z, g).T
    rms = ref.square().mean().sqrt()
    assert ((y - ref).abs() <= 2.0 ** -8 * ref.abs() + 1e-3 * rms).all()
    assert (y - ref).norm() <= (2.0 ** -9 + 2e-4) * ref.norm()


def test_matvec_streams_and_repeat():
    """The same bits on another stream, on a second call, and with the output given."""
    log("[gpu] matvec int4 streams")
    q, s, z = random_int4(500, 1024, 64, True, 3)
    w = on_gpu(q, s, z, 64)
    x = torch.randn(7, 1024).to(torch.bfloat16).cuda()
    y0 = moe.moe_matvec_int4(x, w)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    y1 = torch.empty_like(y0)
    moe.moe_matvec_int4(x, w, y=y1, stream=st)
    torch.cuda.synchronize()
    assert torch.equal(y0, y1)
    assert moe.moe_matvec_int4(x[:0], w).shape == (0, 500)


def test_refusals():
    x = torch.zeros(2, 128, dtype=torch.bfloat16, device="cuda")
    w = on_gpu(*random_int4(16, 128, 32, False, 0), 32)
    with pytest.raises(TypeError):
        moe.moe_matvec_int4(x.float(), w)
    with pytest.raises(ValueError):
        moe.moe_matvec_int4(x[:, :64], w)
    with pytest.raises(ValueError):
        moe.moe_matvec_int4(x.cpu(), w)
    with pytest.raises(ValueError):
        moe.moe_matvec_int4(x, w, y=torch.zeros(2, 15, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(moe.MoEError) as e:
        moe.moe_quantize_int4(torch.zeros(4, 96, dtype=torch.bfloat16, device="cuda"), 64)
    assert e.value.status == 1
    with pytest.raises(ValueError):
        moe.moe_pack_int4(torch.zeros(4, 64, dtype=torch.uint8, device="cuda"),
                          torch.zeros(4, 3, dtype=torch.bfloat16, device="cuda"), None, 32)
