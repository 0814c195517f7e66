"""The paged 8-bit cache on the GPU: appending against the definition code for code, attention
against 64 bits."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

import paper_2606_21712_amd as moe
from gpu_util import log

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn


# ---------------------------------------------------------------- the definition on the host
def exponent(amax):
    """Smallest s with amax <= 448 2^s, in [-127, 127]."""
    if amax == 0 or amax < 2.0 ** -126:
        return -127
    s = math.ceil(math.log2(min(float(amax), 3.4028234663852886e38) / 448.0) - 1e-9)
    while amax > 448.0 * 2.0 ** s and s < 127:
        s += 1
    while s > -127 and amax <= 448.0 * 2.0 ** (s - 1):
        s -= 1
    return max(-127, min(127, s))


def to_codes(v, s):
    """fp32 values -> E4M3 codes of v 2^-s, saturated."""
    x = torch.from_numpy(np.asarray(v, np.float32)) * torch.tensor(2.0 ** -s if s >= -127 else 0.0)
    return x.clamp(-448, 448).to(F8).view(torch.uint8).numpy()


def from_codes(c):
    return torch.from_numpy(np.ascontiguousarray(c)).view(F8).float().numpy()


class HostCache:
    def __init__(self, pages, heads, page, dim):
        self.k = np.zeros((pages, heads, page, dim), np.uint8)
        self.v = np.zeros((pages, heads, page // 16, dim, 16), np.uint8)
        self.ke = np.zeros((pages, heads, page // 16), np.uint8)
        self.ve = np.zeros((pages, heads, page // 16), np.uint8)
        self.page = page

    def append(self, k, v, table, first, n):
        """k, v fp32 [n, heads, dim] of positions first .. first + n - 1 of one sequence."""
        for blk in range(first // 16, (first + n - 1) // 16 + 1):
            pg, b = int(table[blk * 16 // self.page]), blk * 16 % self.page // 16
            lo, hi = max(first, blk * 16), min(first + n, blk * 16 + 16)
            for h in range(k.shape[1]):
                for new, codes, exps in ((k, self.k[pg, h, b * 16:b * 16 + 16], self.ke),
                                         (v, self.v[pg, h, b].T, self.ve)):
                    x = new[lo - first:hi - first, h]
                    fin = x[~np.isnan(x)]
                    s = exponent(np.abs(fin).max() if fin.size else 0.0)
                    if lo > blk * 16:
                        old = int(exps[pg, h, b]) - 127
                        s = max(s, old)
                        if s != old:
                            codes[:lo - blk * 16] = to_codes(from_codes(codes[:lo - blk * 16]), s - old)
                    codes[lo - blk * 16:hi - blk * 16] = to_codes(x, s)
                    codes[hi - blk * 16:] = 0
                    exps[pg, h, b] = s + 127

    def values(self, table, n, h):
        """K and V of one sequence and head in 64 bits, [n, dim]."""
        blocks = [(int(table[i * 16 // self.page]), i * 16 % self.page // 16) for i in range(-(-n // 16))]
        k = [from_codes(self.k[p, h, b * 16:b * 16 + 16]).astype(np.float64) * 2.0 ** (int(self.ke[p, h, b]) - 127)
             for p, b in blocks]
        v = [from_codes(self.v[p, h, b]).astype(np.float64).T * 2.0 ** (int(self.ve[p, h, b]) - 127) for p, b in blocks]
        dim = self.k.shape[3]
        return (np.concatenate(k)[:n], np.concatenate(v)[:n]) if blocks else (np.zeros((0, dim)), np.zeros((0, dim)))

    def device(self):
        return moe.KVCache8(*(torch.from_numpy(t.copy()).cuda() for t in (self.k, self.v, self.ke, self.ve)))

    def same(self, c):
        for a, b in ((self.ke, c.k_exps), (self.ve, c.v_exps), (self.k, c.k_codes), (self.v, c.v_codes)):
            if not np.array_equal(a, b.cpu().numpy()):
                return False
        return True


def rotate(x, pos, cs, interleaved):
    """x fp32 [n, heads, dim], each operation rounded to fp32."""
    rot = cs.shape[1]
    half = rot // 2
    c, s = cs[pos][:, None, :half], cs[pos][:, None, half:]
    y = x.copy()
    ia = np.arange(0, rot, 2) if interleaved else np.arange(half)
    ib = ia + 1 if interleaved else ia + half
    a, b = x[..., ia], x[..., ib]
    y[..., ia] = a * c - b * s
    y[..., ib] = a * s + b * c
    return y


def angles(n, rot):
    f = 10000.0 ** (-np.arange(0, rot, 2) / max(rot, 1))
    a = np.arange(n)[:, None] * f
    return np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)


def tables(lens, page, rng, spare=2):
    per = [max(1, -(-n // page)) for n in lens]
    order = rng.permutation(sum(per) + spare)
    t = np.full((len(lens), max(per)), -1, np.int32)
    at = 0
    for b, p in enumerate(per):
        t[b, :p] = order[at:at + p]
        at += p
    return t, sum(per) + spare


def i32(a):
    return torch.from_numpy(np.asarray(a, np.int32)).cuda()


# ---------------------------------------------------------------- append
APPEND = [  # steps of (new tokens of each sequence), Hq, Hkv, D, page, rot, interleaved
    ([[1]], 1, 1, 64, 16, 64, False),
    ([[5, 1, 16], [1, 1, 1], [20, 0, 33], [1, 1, 1]], 4, 2, 128, 32, 128, False),
    ([[100], [1], [1], [40]], 8, 8, 64, 64, 32, True),
    ([[17, 3], [14, 12], [1, 2]], 6, 2, 256, 16, 256, True),
    ([[1, 2, 3, 4, 5, 6, 7], [9, 8, 7, 6, 5, 4, 3]], 5, 1, 128, 128, 64, False),
    ([[31, 1], [2, 2]], 2, 2, 128, 48, 0, False),
    ([[3] * 70, [14] * 70], 2, 1, 64, 16, 64, False),
]


@pytest.mark.parametrize("steps,Hq,Hkv,D,page,rot,inter", APPEND)
def test_append(steps, Hq, Hkv, D, page, rot, inter):
    """Cache bytes equal to the definition's after every step, exponents that grow in a block
    among them; queries to one bf16 rounding of the fp32 rotation."""
    B = len(steps[0])
    log(f"[gpu] append B={B} steps={len(steps)} Hq={Hq} Hkv={Hkv} D={D} page={page} rot={rot}")
    rng = np.random.default_rng(D + B + page)
    lens = [sum(s[b] for s in steps) for b in range(B)]
    table, pages = tables(lens, page, rng)
    host = HostCache(pages, Hkv, page, D)
    dev = host.device()
    cs = angles(max(lens) + 1, rot)
    have = [0] * B
    for i, new in enumerate(steps):
        T = sum(new)
        # sizes that grow from step to step: held codes are rescaled
        qkv = torch.from_numpy(rng.standard_normal((T, Hq + 2 * Hkv, D)).astype(np.float32) * 4.0 ** i).to(torch.bfloat16)
        qkv[0, Hq, 0] = 0
        f = qkv.float().numpy()
        pos = np.concatenate([np.arange(have[b], have[b] + new[b]) for b in range(B)]).astype(int)
        kr, qr = rotate(f[:, Hq:Hq + Hkv], pos, cs, inter), rotate(f[:, :Hq], pos, cs, inter)
        cu = np.concatenate([[0], np.cumsum(new)])
        for b in range(B):
            if new[b]:
                host.append(kr[cu[b]:cu[b + 1]], f[cu[b]:cu[b + 1], Hq + Hkv:], table[b], have[b], new[b])
                have[b] += new[b]
        g = qkv.cuda()
        args = (g[:, :Hq], g[:, Hq:Hq + Hkv], g[:, Hq + Hkv:], torch.from_numpy(cs).cuda(), dev, i32(table), i32(have),
                i32(cu))
        q = moe.moe_kv8_append(*args, interleaved=inter)
        torch.cuda.synchronize()
        assert host.same(dev), f"step {i}"
        assert torch.equal(q.cpu(), torch.from_numpy(qr).to(torch.bfloat16))
        moe.moe_kv8_append(*args, interleaved=inter)             # again: nothing changes
        torch.cuda.synchronize()
        assert host.same(dev), f"step {i}, repeated"


@pytest.mark.parametrize("kind", ["zeros", "tiny", "huge", "inf", "nan", "edge"])
def test_append_values(kind):
    """Blocks of zeros, subnormal and largest values, infinities and NaN, and maxima on both sides of
    448 2^s."""
    log(f"[gpu] append values {kind}")
    n, Hkv, D, page = 21, 1, 64, 16
    rng = np.random.default_rng(1)
    v = rng.standard_normal((n, 3, D)).astype(np.float32)
    if kind == "zeros":
        v[:] = 0
    elif kind == "tiny":
        v *= 1e-38
    elif kind == "huge":
        v *= 1e37
    elif kind == "inf":
        v[2, 1:, 3], v[18, 1:, 5] = np.inf, -np.inf
    elif kind == "nan":
        v[4, 1:, 7], v[20, 1:, 9] = np.nan, np.nan
    else:
        v = np.clip(v, -1, 1)
        v[0, 1, 0], v[17, 1, 0] = 448 * 2.0 ** -3, -450 * 2.0 ** -3      # bf16 has 450
        v[1, 2, 0], v[16, 2, 0] = -448.0, 450.0
    t = torch.from_numpy(v).to(torch.bfloat16)
    f = t.float().numpy()
    host = HostCache(3, Hkv, page, D)
    dev = host.device()
    table = np.array([[2, 0]], np.int32)
    host.append(f[:, 1:2], f[:, 2:3], table[0], 0, n)
    g = t.cuda()
    moe.moe_kv8_append(g[:, :1], g[:, 1:2], g[:, 2:3], torch.zeros((1, 0), device="cuda"), dev, i32(table), i32([n]),
                       i32([0, n]))
    torch.cuda.synchronize()
    for a, b in ((host.ke, dev.k_exps), (host.ve, dev.v_exps)):
        assert np.array_equal(a, b.cpu().numpy())
    for a, b in ((host.k, dev.k_codes), (host.v, dev.v_codes)):
        a, b = from_codes(a), from_codes(b.cpu().numpy())
        assert np.array_equal(a, b, equal_nan=True)


def test_append_inactive():
    """A sequence of length 0 with a row, pages outside the cache and columns outside the table:
    nothing is written for them."""
    log("[gpu] append inactive")
    rng = np.random.default_rng(3)
    host = HostCache(4, 2, 16, 64)
    for t in (host.k, host.v, host.ke, host.ve):
        t[:] = rng.integers(0, 100, t.shape)
    dev = host.device()
    x = torch.randn(4, 2, 64).to(torch.bfloat16).cuda()
    table = i32([[0], [-1], [4], [3]])
    moe.moe_kv8_append(x, x, x, torch.zeros((64, 64), device="cuda"), dev, table, i32([0, 1, 1, 17]), i32([0, 1, 2, 3, 4]))
    torch.cuda.synchronize()
    assert host.same(dev)


# ---------------------------------------------------------------- attention
def filled(lens, Hkv, D, page, rng, poison=True):
    """A cache with random codes and exponents.  Places after a sequence's end hold NaN codes."""
    table, pages = tables(lens, page, rng)
    host = HostCache(pages, Hkv, page, D)
    if poison:
        host.k[:], host.v[:] = 0x7F, 0xFF
        host.ke[:], host.ve[:] = 254, 254
    for b, n in enumerate(lens):
        for blk in range(-(-n // 16)):
            p, i = int(table[b, blk * 16 // page]), blk * 16 % page // 16
            m = min(16, n - blk * 16)
            c = torch.from_numpy(rng.standard_normal((2, Hkv, m, D)).astype(np.float32) * 100).clamp(-448, 448)
            c = c.to(F8).view(torch.uint8).numpy()
            host.k[p, :, i * 16:i * 16 + m] = c[0]
            host.v[p, :, i, :, :m] = c[1].transpose(0, 2, 1)
            host.ke[p, :, i] = rng.integers(127 - 9, 127 - 5, Hkv)
            host.ve[p, :, i] = rng.integers(127 - 12, 127 - 4, Hkv)
    return host, table


def attention64(q, host, table, lens, new, window, scale):
    """out and, for the bounds, sum p |v|."""
    T, Hq, D = q.shape
    Hkv = host.k.shape[1]
    out, mag = np.zeros((T, Hq, D)), np.zeros((T, Hq, D))
    row = 0
    for b, n in enumerate(lens):
        for h in range(Hkv):
            k, v = host.values(table[b], n, h)
            for i in range(new[b]):
                p = n - new[b] + i
                lo = max(0, p - window + 1) if window else 0
                if p < lo:
                    continue
                for j in range(Hq // Hkv):
                    x = k[lo:p + 1] @ q[row + i, h * (Hq // Hkv) + j] * scale
                    w = np.exp(x - x.max())
                    w /= w.sum()
                    out[row + i, h * (Hq // Hkv) + j] = w @ v[lo:p + 1]
                    mag[row + i, h * (Hq // Hkv) + j] = w @ np.abs(v[lo:p + 1])
        row += new[b]
    return out, mag


ATTEND = [  # lens, new, Hq, Hkv, D, page, window
    ([1], [1], 1, 1, 64, 16, 0),
    ([17], [1], 4, 1, 128, 16, 0),
    ([64, 65, 63, 128], [1, 1, 1, 1], 8, 2, 128, 64, 0),
    ([5000, 33, 1, 700], [1, 1, 1, 1], 8, 2, 128, 32, 0),
    ([900, 20], [1, 1], 16, 1, 256, 16, 0),
    ([300, 300], [1, 1], 20, 1, 64, 48, 0),
    ([40, 9, 200], [3, 9, 0], 4, 2, 128, 16, 0),
    ([70, 500], [70, 5], 5, 1, 64, 64, 0),
    ([333], [100], 4, 2, 128, 128, 0),
    ([260, 90], [200, 90], 2, 2, 256, 16, 0),
    ([600], [130], 8, 2, 64, 32, 100),
    ([2000, 50], [1, 1], 4, 4, 128, 64, 37),
    ([150], [60], 3, 1, 128, 16, 1),
    ([1030], [1], 6, 2, 128, 16, 500),
]


@pytest.mark.parametrize("lens,new,Hq,Hkv,D,page,window", ATTEND)
def test_attention(lens, new, Hq, Hkv, D, page, window):
    """Bounds: probabilities and the output are rounded to bf16 (2^-9 of sum p |v|, 2^-9 of the
    result); scores of up to some 30 carry fp32 sums of D products, 1e-5 of the probabilities.  What
    lies past a sequence's end is NaN."""
    log(f"[gpu] attention lens={lens} new={new} Hq={Hq} Hkv={Hkv} D={D} page={page} window={window}")
    rng = np.random.default_rng(len(lens) + D + sum(lens))
    host, table = filled(lens, Hkv, D, page, rng)
    T = sum(new)
    q = torch.from_numpy(rng.standard_normal((T, Hq, D)).astype(np.float32)).to(torch.bfloat16)
    cu = np.concatenate([[0], np.cumsum(new)])
    dev = host.device()
    out = moe.moe_kv8_attention(q.cuda(), dev, i32(table), i32(lens), i32(cu), max(new), max(lens), window=window)
    torch.cuda.synchronize()
    ref, mag = attention64(q.double().numpy(), host, table, lens, new, window, D ** -0.5)
    err = np.abs(out.cpu().double().numpy() - ref)
    assert (err <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2e-5) * mag).all()
    assert host.same(dev)
    # another plan (the longest length is a hint), and the call again: the same to the joins' roundings
    more = moe.moe_kv8_attention(q.cuda(), dev, i32(table), i32(lens), i32(cu), max(new) + 3, 1, window=window)
    err = np.abs(more.cpu().double().numpy() - ref)
    assert (err <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2e-5) * mag).all()
    again = moe.moe_kv8_attention(q.cuda(), dev, i32(table), i32(lens), i32(cu), max(new), max(lens), window=window)
    assert torch.equal(out.view(torch.int16), again.view(torch.int16))


@pytest.mark.parametrize("B,G", [(1, 1), (3, 4), (40, 2)])
def test_attention_splits(B, G):
    """Long and short sequences in one plan: parts without tokens, and rows that see nothing."""
    log(f"[gpu] attention splits B={B} G={G}")
    rng = np.random.default_rng(B)
    lens = [int(n) for n in rng.integers(1, 300, B)]
    lens[0] = 4000
    if B > 2:
        lens[1], lens[2] = 0, 1
    host, table = filled(lens, 2, 64, 16, rng)
    q = torch.randn(B, 2 * G, 64, generator=torch.Generator().manual_seed(B)).to(torch.bfloat16)
    out = moe.moe_kv8_attention(q.cuda(), host.device(), i32(table), i32(lens), i32(range(B + 1)), 1, max(lens))
    ref, mag = attention64(q.double().numpy(), host, table, lens, [1] * B, 0, 0.125)
    err = np.abs(out.cpu().double().numpy() - ref)
    assert (err <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2e-5) * mag).all()
    if B > 2:
        assert (out[1] == 0).all()


@pytest.mark.parametrize("D,new", [(64, 20), (128, 5), (256, 20)])
def test_nan_reaches_those_who_see_it(D, new):
    """A NaN in a new token's key, or in one dimension of its value: NaN (at least there) for the rows that see
    the token, no change for others."""
    log(f"[gpu] attention NaN D={D} new={new}")
    rng = np.random.default_rng(D)
    lens = [100]
    host, table = filled(lens, 1, D, 16, rng)
    q = torch.from_numpy(rng.standard_normal((new, 2, D)).astype(np.float32)).to(torch.bfloat16).cuda()
    args = (i32(table), i32(lens), i32([0, new]), new, 100)
    clean = moe.moe_kv8_attention(q, host.device(), *args)
    bad_at = 100 - new + new // 2                                # position of the bad token
    p, b, i = int(table[0, bad_at // 16]), 0, bad_at % 16
    for what in ("v", "k"):
        h2 = HostCache(*host.k.shape[:2], 16, D)
        h2.k, h2.v, h2.ke, h2.ve = host.k.copy(), host.v.copy(), host.ke, host.ve
        if what == "v":
            h2.v[p, 0, b, 3, i] = 0xFF
        else:
            h2.k[p, 0, i, 5] = 0x7F
        out = moe.moe_kv8_attention(q, h2.device(), *args)
        seen = new // 2
        assert torch.equal(out[:seen], clean[:seen]), what
        assert (out[seen:].isnan() if what == "k" else out[seen:, :, 3].isnan()).all(), what


def test_large_offsets():
    """A page whose codes begin past 2^31 bytes: keys and values of a short sequence there."""
    log("[gpu] offsets past 32 bits")
    pages, Hkv, page, D = 33000, 4, 128, 128                     # 2.2e9 bytes of codes each
    cache = moe.KVCache8.empty(pages, Hkv, D, page)
    last = pages - 1
    n = 100
    rng = np.random.default_rng(0)
    kv = torch.from_numpy(rng.standard_normal((n, 4, 3, D)).astype(np.float32)).to(torch.bfloat16)
    g = kv.cuda()
    table = i32([[last]])
    q, k, v = (g[:, :, i].contiguous() for i in range(3))
    qr = moe.moe_kv8_append(q, k, v, torch.from_numpy(angles(n, D)).cuda(), cache, table, i32([n]), i32([0, n]))
    host = HostCache(1, Hkv, page, D)
    f = kv.float().numpy()
    host.append(rotate(f[:, :, 1], np.arange(n), angles(n, D), False), f[:, :, 2], [0], 0, n)
    assert np.array_equal(host.k[0, :, :n], cache.k_codes[last, :, :n].cpu().numpy())
    assert np.array_equal(host.v[0, :, :6], cache.v_codes[last, :, :6].cpu().numpy())
    out = moe.moe_kv8_attention(qr, cache, table, i32([n]), i32([0, n]), n, n)
    ref, mag = attention64(qr.double().cpu().numpy(), host, [[0]], [n], [n], 0, D ** -0.5)
    assert (np.abs(out.cpu().double().numpy() - ref) <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2e-5) * mag).all()


def test_graph():
    """Append and attention captured together and replayed as the sequences grow: the eager bits."""
    log("[gpu] kv8 graph")
    B, Hq, Hkv, D, page = 3, 4, 2, 128, 16
    rng = np.random.default_rng(11)
    table, pages = tables([80] * B, page, rng)
    caches = [moe.KVCache8.empty(pages, Hkv, D, page) for _ in range(2)]
    for c in caches:
        for t in (c.k_codes, c.v_codes, c.k_exps, c.v_exps):
            t.zero_()
    cs = torch.from_numpy(angles(128, D)).cuda()
    tab, lens, cu = i32(table), i32([0, 14, 40]), i32(range(B + 1))
    qkv = torch.zeros((B, Hq + 2 * Hkv, D), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(max(1, moe.moe_kv8_attention_workspace_bytes(B, B, Hq, Hkv, D, 1, 80)), dtype=torch.uint8, device="cuda")
    q_out, out = (torch.empty((B, Hq, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))

    def step(c):
        moe.moe_kv8_append(qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], cs, c, tab, lens, cu, q_out=q_out)
        return moe.moe_kv8_attention(q_out, c, tab, lens, cu, 1, 80, out=out, ws=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(caches[0])
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(caches[0])
    for i in range(5):
        qkv.copy_(torch.from_numpy(rng.standard_normal(qkv.shape).astype(np.float32) * 2 ** i))
        if i:
            lens += 1
        want = step(caches[1]).clone()
        out.fill_(7.0)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
        assert torch.equal(caches[0].v_codes, caches[1].v_codes) and torch.equal(caches[0].k_exps, caches[1].k_exps)


def test_refusals():
    c = moe.KVCache8.empty(4, 2, 64, 16)
    x = torch.zeros((2, 2, 64), dtype=torch.bfloat16, device="cuda")
    tab, lens, cu = i32([[0], [1]]), i32([1, 1]), i32([0, 1, 2])
    cs = torch.zeros((16, 64), device="cuda")
    for bad in (dict(q=x.float()), dict(k=x[:, :1]), dict(v=x[:1]), dict(lens=i32([1])), dict(cs=cs.double()),
                dict(tab=tab.long()), dict(q=x.transpose(1, 2).contiguous().transpose(1, 2))):
        a = dict(q=x, k=x, v=x, cs=cs, tab=tab, lens=lens, cu=cu)
        a.update(bad)
        with pytest.raises((ValueError, TypeError)):
            moe.moe_kv8_append(a["q"], a["k"], a["v"], a["cs"], c, a["tab"], a["lens"], a["cu"])
    with pytest.raises(moe.MoEError) as e:
        moe.moe_kv8_append(x, x, x, torch.zeros((16, 24), device="cuda"), c, tab, lens, cu)
    assert e.value.status == 1
    with pytest.raises(moe.MoEError) as e:
        moe.moe_kv8_append(x[:, :1], x, x, cs, c, tab, lens, cu)          # 1 query head for 2 kv heads
    assert e.value.status == 1
    with pytest.raises(ValueError):
        moe.KVCache8.empty(4, 2, 64, 16).__class__(c.k_codes, c.v_codes[:3], c.k_exps, c.v_exps)
    with pytest.raises(ValueError):
        moe.moe_kv8_attention(x[..., :32], c, tab, lens, cu, 1, 1)
    with pytest.raises(moe.MoEError) as e:
        moe.moe_kv8_attention(x, c, tab, lens, cu, 0, 1)
    assert e.value.status == 1
    big = moe.moe_kv8_attention_workspace_bytes(2, 2, 2, 2, 64, 1, 100000)
    assert big > 0
    with pytest.raises(moe.MoEError) as e:
        moe.moe_kv8_attention(x, c, tab, lens, cu, 1, 100000, ws=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 3
    with pytest.raises(moe.MoEError) as e:
        moe.moe_kv8_attention(torch.zeros((2, 2, 96), dtype=torch.bfloat16, device="cuda"),
                              moe.KVCache8.empty(4, 2, 96, 16), tab, lens, cu, 1, 1)
    assert e.value.status == 2
    assert moe.moe_kv8_attention(x[:0], c, tab, lens, i32([0, 0, 0]), 1, 1).shape == (0, 2, 64)
