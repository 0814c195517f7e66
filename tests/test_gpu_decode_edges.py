"""The operators for few sequences where they meet what they must leave alone: rows of another batch size, sequences
without rows, values that no row sees, weights of experts that a token did not choose."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2606_21712_amd as moe
from gpu_util import log
from test_gpu_few import inputs
from test_gpu_kv8 import HostCache, angles, attention64, filled, i32, rotate

pytestmark = pytest.mark.gpu


@pytest.fixture
def budget():
    yield moe.set_cu_budget
    moe.set_cu_budget(0)


# ---------------------------------------------------------------- graphs of one layer
def test_graphs_of_several_sizes():
    """Two batch sizes captured from one layer, and eager runs of a third between the replays: each replay returns
    the rows of its own size."""
    log("[gpu] few: graphs of several sizes")
    H, E, k, F = 256, 16, 4, 128
    x, logits, shapes, r = inputs(12, H, E, k, F, 0, 5)
    w = [(torch.randn(s, generator=r) * s[2] ** -0.5).to(torch.bfloat16).cuda() for s in shapes]
    layer = moe.MoELayerFew(12, H, E, k, F)
    x, logits = x.cuda(), logits.cuda()
    sizes = (3, 12)
    xs, ls = [x[:n].clone() for n in sizes], [logits[:n].clone() for n in sizes]
    graphs = [moe.LayerGraph(layer, a, b, *w) for a, b in zip(xs, ls)]
    for i in range(6):
        g = i % 2
        xs[g].copy_(torch.randn(xs[g].shape, generator=r).to(torch.bfloat16))
        ls[g].copy_(torch.randn(ls[g].shape, generator=r))
        want = layer.run(xs[g], ls[g], *w).clone()
        ids, wts = layer.topk_ids.clone(), layer.topk_weights.clone()
        layer.run(x[:7 + i % 3], logits[:7 + i % 3], *w)
        torch.cuda.synchronize()
        y = graphs[g].replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want), i
        assert torch.equal(graphs[g].topk_ids, ids) and torch.equal(graphs[g].topk_weights, wts), i


# ---------------------------------------------------------------- sequences that bring no rows
def test_append_without_rows():
    """A sequence with no new rows is left as it is, what lies past its end too; one whose page another sequence
    appends to in the same call does not touch it."""
    log("[gpu] append without rows")
    rng = np.random.default_rng(8)
    Hkv, page, D = 2, 16, 128
    host = HostCache(5, Hkv, page, D)
    host.k[:], host.v[:] = (rng.integers(0, 0x7E, t.shape) for t in (host.k, host.v))
    host.ke[:], host.ve[:] = 120, 121
    cs = angles(64, D)

    def append(table, lens, new):
        x = torch.from_numpy(rng.standard_normal((sum(new), 3 * Hkv, D)).astype(np.float32)).to(torch.bfloat16)
        dev = host.device()
        cu = np.concatenate([[0], np.cumsum(new)])
        g = x.cuda()
        moe.moe_kv8_append(g[:, :Hkv], g[:, Hkv:2 * Hkv], g[:, 2 * Hkv:], torch.from_numpy(cs).cuda(), dev, i32(table),
                           i32(lens), i32(cu))
        torch.cuda.synchronize()
        f = x.float().numpy()
        for b, n in enumerate(new):
            if n:
                rows = slice(cu[b], cu[b + 1])
                first = lens[b] - n
                host.append(rotate(f[rows, Hkv:2 * Hkv], np.arange(first, lens[b]), cs, False), f[rows, 2 * Hkv:],
                            table[b], first, n)
        assert host.same(dev)

    append([[0, 1], [2, 3]], [21, 13], [0, 3])          # codes lie past the first one's 21 tokens
    append([[2, 3], [2, 3], [2, 3]], [7, 19, 30], [0, 19, 0])   # the page is now the second one's


# ---------------------------------------------------------------- values that no row of a tile, or not every one, sees
def bound(ref, mag):
    """Probabilities and outputs rounded to bf16, 2^-8 at most each; fp32 scores, 1e-5 of the probabilities."""
    return 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2e-5) * mag


WINDOWS = [  # lens, new, Hq, Hkv, D, page, window: tiles of 16, 32 and 128 rows
    ([700, 300], [1, 1], 8, 2, 128, 16, 40), ([700, 90], [1, 1], 4, 1, 64, 64, 100), ([500], [1], 4, 4, 256, 16, 17),
    ([500], [3], 8, 1, 256, 64, 30), ([900, 700], [9, 6], 8, 2, 128, 64, 70), ([800], [12], 4, 1, 64, 16, 50),
    ([900], [8], 8, 1, 256, 16, 33), ([1100, 600], [90, 70], 4, 2, 128, 64, 130), ([1000], [200], 2, 1, 64, 16, 90),
    ([700], [150], 4, 2, 256, 64, 100), ([640], [128], 4, 1, 128, 16, 1),
]


@pytest.mark.parametrize("cus", [1, 0])
@pytest.mark.parametrize("codes,exps", [(0xFF, 254), (0x7E, 254), (0x38, 255), (0x00, 255), (0x7E, 247)])
@pytest.mark.parametrize("lens,new,Hq,Hkv,D,page,window", WINDOWS)
def test_before_the_window(budget, cus, codes, exps, lens, new, Hq, Hkv, D, page, window):
    """Blocks before every row's window hold anything, and pages before it have left the table; so do the places of
    a block that the first row's window begins in."""
    log(f"[gpu] before the window cus={cus} {codes:#x} {exps} lens={lens} new={new} D={D} page={page} window={window}")
    rng = np.random.default_rng(sum(lens) + D)
    host, table = filled(lens, Hkv, D, page, rng)
    # one page more, in front: what -1 is read as
    for name in ("k", "v", "ke", "ve"):
        t = getattr(host, name)
        setattr(host, name, np.concatenate([np.full_like(t[:1], codes if len(name) == 1 else exps), t]))
    table = np.where(table >= 0, table + 1, -1)
    for b, n in enumerate(lens):
        low = max(0, n - new[b] - window + 1)                   # the first token that a row sees
        for blk in range(low // 16 + 1):
            p, i = int(table[b, blk * 16 // page]), blk * 16 % page // 16
            m = min(16, low - blk * 16)
            if m == 16:
                host.k[p, :, i * 16:i * 16 + 16], host.v[p, :, i] = codes, codes
                host.ke[p, :, i], host.ve[p, :, i] = exps, exps
            elif m > 0:
                host.k[p, :, i * 16:i * 16 + m], host.v[p, :, i, :, :m] = 0x7F, 0xFF
        table[b, :low // page] = -1
    q = torch.from_numpy(rng.standard_normal((sum(new), Hq, D)).astype(np.float32)).to(torch.bfloat16)
    budget(cus)
    for most in (max(lens), 1):                                 # cut into parts, where few are; whole
        out = moe.moe_kv8_attention(q.cuda(), host.device(), i32(table), i32(lens), i32(np.cumsum([0] + new)), max(new),
                                    most, window=window).cpu().double().numpy()
        with np.errstate(all="ignore"):
            ref, mag = attention64(q.double().numpy(), host, table, lens, new, window, D ** -0.5)
        assert (np.abs(out - ref) <= bound(ref, mag)).all()


@pytest.mark.parametrize("cus", [1, 0])
@pytest.mark.parametrize("D,Hq,new,window,page", [(128, 2, 6, 0, 16), (64, 4, 40, 20, 64), (128, 2, 100, 0, 64),
                                                  (256, 1, 100, 30, 16), (256, 4, 6, 9, 64)])
def test_infinite_value(budget, cus, D, Hq, new, window, page):
    """A value that no finite bf16 number holds (an infinity that was appended is 448 2^120) makes the rows that see
    its token infinite or NaN, and no others."""
    log(f"[gpu] infinite value cus={cus} D={D} new={new} window={window} page={page}")
    rng = np.random.default_rng(D + new)
    n, at = 200, 200 - new // 2 - 1                             # length, position of the token
    host, table = filled([n], 1, D, page, rng)
    p, i = int(table[0, at // page]), at % page // 16
    # its block's other values: under 2^114, whose sums times probabilities of up to 2^8 fp32 holds
    host.ve[p, 0, i] = 247
    host.v[p, 0, i] = rng.integers(0, 8, host.v[p, 0, i].shape)
    host.v[p, 0, i, :, at % 16] = 0x7E
    q = torch.from_numpy(rng.standard_normal((new, Hq, D)).astype(np.float32)).to(torch.bfloat16)
    budget(cus)
    out = moe.moe_kv8_attention(q.cuda(), host.device(), i32(table), i32([n]), i32([0, new]), new, n,
                                window=window).cpu().double().numpy()
    ref, mag = attention64(q.double().numpy(), host, table, [n], [new], window, D ** -0.5)
    pos = np.arange(n - new, n)
    sees = (pos >= at) & ((pos - at < window) if window else True)
    assert sees.any() and not sees.all()
    assert (np.abs(out - ref) <= bound(ref, mag))[~sees].all()
    assert not np.isfinite(out[sees]).any()


def test_append_rotates_without_a_page():
    """New tokens that have no page in the cache are not written; their queries are rotated all the same."""
    log("[gpu] append: queries of tokens without a page")
    rng = np.random.default_rng(4)
    D, Hq, Hkv = 64, 4, 2
    x = torch.from_numpy(rng.standard_normal((23, Hq + 2 * Hkv, D)).astype(np.float32)).to(torch.bfloat16)
    cs = angles(64, D)
    host = HostCache(2, Hkv, 16, D)
    dev = host.device()
    table, lens, cu = i32([[-1, -1], [2, 0], [1, 0]]), i32([1, 20, 34]), i32([0, 1, 21, 23])
    q_out = torch.full((23, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    g = x.cuda()
    moe.moe_kv8_append(g[:, :Hq], g[:, Hq:Hq + Hkv], g[:, Hq + Hkv:], torch.from_numpy(cs).cuda(), dev, table, lens, cu,
                       q_out=q_out)
    torch.cuda.synchronize()
    pos = np.concatenate([[0], np.arange(20), [32, 33]])        # the last two are past the table's columns
    f = x.float().numpy()
    assert torch.equal(q_out.cpu(), torch.from_numpy(rotate(f[:, :Hq], pos, cs, False)).to(torch.bfloat16))
    host.append(rotate(f[17:21, Hq:Hq + Hkv], pos[17:21], cs, False), f[17:21, Hq + Hkv:], [1, 0], 16, 4)
    assert host.same(dev)


# ---------------------------------------------------------------- the layer for few tokens
@pytest.mark.parametrize("int4", [False, True])
@pytest.mark.parametrize("cus", [8, 0])
@pytest.mark.parametrize("T,H,F,Fs", [(1, 128, 64, 0), (7, 256, 512, 64), (8, 6144, 64, 0), (13, 256, 1024, 0),
                                      (16, 448, 128, 128)])
def test_weights_of_other_experts(budget, cus, T, H, F, Fs, int4):
    """Weights that are not finite reach the tokens that chose their expert, and no others."""
    log(f"[gpu] few: non-finite weights int4={int4} cus={cus} T={T} H={H} F={F} Fs={Fs}")
    E, k, bad = 8, 2, 3
    x, logits, shapes, r = inputs(T, H, E, k, F, Fs, T + H)
    w = [(torch.randn(s, generator=r) * s[2] ** -0.5).to(torch.bfloat16) for s in shapes]
    logits[:, bad] = -9.0
    logits[0, bad] = 9.0                                        # the first token alone chooses it
    x, logits = x.cuda(), logits.cuda()
    budget(cus)

    def run(spoil):
        ws = [t.clone() for t in w]
        if not int4:
            for i, (n, c) in enumerate(spoil):
                if n is not None:
                    ws[2][bad, n, c] = (float("inf"), float("nan"))[i % 2]
            return moe.moe_few_tokens(x, logits, k, *[t.cuda() for t in ws])[0]
        std = [moe.moe_quantize_int4(t.cuda(), 32, True) for t in ws]
        for i, (n, c) in enumerate(spoil):
            if n is not None:
                std[2][1][bad, n, c // 32] = (float("inf"), float("nan"))[i % 2]
        return moe.moe_few_tokens(x, logits, k, *[moe.moe_pack_int4(*s, 32) for s in std])[0]

    clean = run([])
    y = run([(5, 3), (17, F - 1), (H - 1, F // 2)])
    assert torch.equal(y[1:], clean[1:])
    hit = torch.zeros(H, dtype=torch.bool, device="cuda")
    hit[[5, 17, H - 1]] = True
    assert not y[0, hit].isfinite().any() and torch.equal(y[0, ~hit], clean[0, ~hit])
    assert clean.isfinite().all()


@pytest.mark.parametrize("T", [2, 12])
def test_h_beyond_bf16(T):
    """An h above the largest bf16 number is infinite, as in MoELayer: its token's y is infinite where that has a
    sign, the other tokens' is finite."""
    log(f"[gpu] few: h beyond bf16 T={T}")
    H = F = 64
    x = torch.zeros(T, H, dtype=torch.bfloat16)
    x[:, 0] = 1.0
    x[0, 0] = 1e20
    wg, wu, wd = (torch.zeros(1, 64, 64, dtype=torch.bfloat16) for _ in range(3))
    wg[0, 0, 0] = wu[0, 0, 0] = 1.0
    wg[0, 1, 0] = wu[0, 1, 0] = 1.8e-1                          # 3.24e38: finite, and rounds to a finite number
    wd[0, :, 0] = torch.where(torch.arange(H) % 2 == 0, 1.0, -1.0)
    logits = torch.zeros(T, 1)
    args = [t.cuda() for t in (x, logits, wg, wu, wd)]
    y = moe.moe_few_tokens(args[0], args[1], 1, *args[2:])[0]
    ref = moe.MoELayer(T, H, 1, 1, F, gather=True).run(*args)
    assert torch.equal(y, ref) and y[0].isinf().all() and y[1:].isfinite().all()


@pytest.mark.parametrize("int4", [False, True])
def test_one_expert_without_its_axis(int4):
    """Weights of a single expert as matrices, F other than H."""
    log(f"[gpu] few: 2-D weights int4={int4}")
    T, H, F, Fs = 5, 128, 320, 64
    x, logits, shapes, r = inputs(T, H, 1, 1, F, Fs, 2)
    w = [(torch.randn(s, generator=r) * s[2] ** -0.5).to(torch.bfloat16).cuda() for s in shapes]
    if int4:
        w = [moe.quantize_weights_int4(t, 32) for t in w]
        flat = [moe.Int4(t.codes, t.scales, t.zeros, t.shape[1:], t.group) for t in w]
    else:
        flat = [t[0] for t in w]
    x, logits = x.cuda(), logits.cuda()
    want = moe.moe_few_tokens(x, logits, 1, *w)
    got = moe.moe_few_tokens(x, logits, 1, *flat)
    assert all(torch.equal(a, b) for a, b in zip(want, got))


# ---------------------------------------------------------------- 4-bit weights
def test_quantize_largest():
    """A group that spans more than the largest fp32 number has a finite scale."""
    log("[gpu] quantize int4: largest values")
    w = torch.zeros(2, 64, dtype=torch.bfloat16)
    top = torch.finfo(torch.bfloat16).max
    w[0, 0], w[0, 1], w[0, 2] = top, -top, 0.5 * top
    w[1, 3] = -top
    codes, s, z = moe.moe_quantize_int4(w.cuda(), 64, True)
    lo, hi = w.double().amin(1).clamp_max(0), w.double().amax(1).clamp_min(0)
    assert torch.equal(s.cpu()[:, 0], ((hi - lo) / 15).to(torch.bfloat16))
    f = s.cpu().double()
    zero = torch.round(-lo[:, None] / f).clamp_max(15)
    q = (torch.round(w.double() / f) + zero).clamp(0, 15).to(torch.uint8)
    assert torch.equal(z.cpu().double(), zero) and torch.equal(codes.cpu(), q[:, 0::2] | (q[:, 1::2] << 4))


# ---------------------------------------------------------------- the compute-unit budget
@pytest.mark.parametrize("cus,H,T,F", [(8, 64, 3, 4096), (24, 128, 8, 2048), (40, 192, 16, 2048), (0, 256, 2, 8192)])
def test_down_parts_keep_to_the_budget(budget, cus, H, T, F):
    """The down projection's parts, of which each writes its sums to the workspace, are two workgroups a compute unit
    at most, one group of 16 columns more aside."""
    log(f"[gpu] few: parts cus={cus} H={H} T={T} F={F}")
    E, k = 8, 2
    x, logits, shapes, r = inputs(T, H, E, k, F, 0, H)
    w = [(torch.randn(s, generator=r) * s[2] ** -0.5).to(torch.bfloat16).cuda() for s in shapes]
    ws = torch.full((moe.moe_few_tokens_workspace_bytes(T, H, k, F),), 0xAB, dtype=torch.uint8, device="cuda")
    budget(cus)
    moe.moe_few_tokens(x.cuda(), logits.cuda(), k, *w, ws=ws)
    torch.cuda.synchronize()
    sums = ws[-(-T * k * F * 4 // 256) * 256:].view(torch.int32)
    sums = sums[:sums.numel() // (T * H) * (T * H)].view(-1, T * H)
    parts = int((sums != 0xABABABAB - 2 ** 32).any(1).sum())
    groups = H // 16
    units = cus or torch.cuda.get_device_properties(0).multi_processor_count
    assert 1 < parts and (parts - 1) * groups < 2 * units


def test_table_of_many_columns():
    """A block table with place for more tokens than can be counted in 32 bits for all tiles: the long sequence is not
    cut, its output is the same to the rounding of the probabilities."""
    log("[gpu] attention: a table of 400 million tokens")
    rng = np.random.default_rng(6)
    D, page, cols, B = 64, 1 << 18, 1536, 400
    lens = [3000] + [int(n) for n in rng.integers(1, 40, B - 1)]
    cache = moe.KVCache8.empty(1, 1, D, page)
    for t in (cache.k_codes, cache.v_codes):
        t.copy_(torch.from_numpy(rng.integers(0, 0x58, t.shape, dtype=np.uint8)))
    cache.k_exps.fill_(127 - 6)
    cache.v_exps.fill_(127 - 6)
    q = torch.from_numpy(rng.standard_normal((B, 1, D)).astype(np.float32)).to(torch.bfloat16).cuda()
    wide = torch.full((B, cols), -1, dtype=torch.int32, device="cuda")
    wide[:, 0] = 0
    args = i32(lens), i32(range(B + 1)), 1, max(lens)
    a = moe.moe_kv8_attention(q, cache, wide, *args)
    b = moe.moe_kv8_attention(q, cache, wide[:, :1].contiguous(), *args)
    torch.cuda.synchronize()
    assert torch.equal(a[1:], b[1:])
    assert (a[0] - b[0]).float().norm() <= 2.0 ** -7 * b[0].float().norm() and b[0].float().norm() > 0
