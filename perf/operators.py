"""Performance cases of the decode step for a few sequences: the tail of a batch, where a
handful of long sequences is left and all the time goes into weights and cache.

A case is a dict of plain values, its "kind" one of

    few       the whole MoE layer for at most 16 tokens: MoELayerFew.run
              weights "bf16" or "int4" (group scales, optionally zero points)
    matvec    moe_matvec_int4: a few rows times a 4-bit matrix with group scales
    append    moe_kv8_append: position rotation of q and k, keys and values quantised into
              the paged 8-bit cache
    attend    moe_kv8_attention: attention of the new tokens over that cache

The cache holds E4M3 codes with one power-of-two exponent for each block of 16 tokens and
kv head.  k_codes [pages, Hkv, page, D]; v_codes [pages, Hkv, page / 16, D, 16] (tokens of a
block innermost); exponents u8 [pages, Hkv, page / 16], 127 + s.

Sequences of a case: B of them; sequence b brings n_b new tokens and then holds len_b.
"ragged" spreads both below their maxima.

Every input is drawn on the GPU from the seed alone.
"""
from __future__ import annotations

import math
import random

import torch

own = False     # True: run() makes the framework's calls, False: the plain form
DEV = "cuda"
BLOCK = 16      # tokens that share an exponent


# --------------------------------------------------------------------------- the cases
def _few(name, weights, T, H, E, k, F, Fs=0, group=128, zeros=False, renorm=1):
    c = dict(name=name, kind="few", weights=weights, T=T, H=H, E=E, k=k, F=F, Fs=Fs, renorm=renorm)
    if weights == "int4":
        c.update(group=group, zeros=zeros)
    return c


def _matvec(name, T, N, K, group, zeros):
    return dict(name=name, kind="matvec", T=T, N=N, K=K, group=group, zeros=zeros)


def _append(name, B, new, length, Hq, Hkv, D, page, rot, interleaved=False, ragged=False):
    return dict(name=name, kind="append", B=B, new=new, length=length, Hq=Hq, Hkv=Hkv, D=D, page=page, rot=rot,
                interleaved=interleaved, ragged=ragged)


def _attend(name, B, new, length, Hq, Hkv, D, page, window=0, ragged=False):
    return dict(name=name, kind="attend", B=B, new=new, length=length, Hq=Hq, Hkv=Hkv, D=D, page=page, window=window,
                ragged=ragged)


def listed():
    return [
        # The tiny layer, one token: launches and latency are all there is.
        _few("few_tiny_1", "bf16", 1, 256, 8, 2, 512),
        # The last sequence of a batch on the Mixtral shape: two experts' weights for one token.
        _few("few_mixtral_1", "bf16", 1, 4096, 8, 2, 14336),
        # Eight sequences left on the fine-grained DeepSeek shape with its shared expert.
        _few("few_deepseek_8", "bf16", 8, 7168, 64, 8, 2048, 2048),
        # 4-bit experts on the memory-constrained shape, an odd number of sequences.
        _few("few_int4_memconstrained_13", "int4", 13, 4096, 64, 4, 4096, group=64, zeros=True),
        # Attention's output projection for one token: 8 MB of codes.
        _matvec("matvec_1_4096x4096", 1, 4096, 4096, 128, False),
        # A dense gate/up projection (2 x 14336 rows) for a small batch.
        _matvec("matvec_8_28672x4096", 8, 28672, 4096, 64, True),
        # Odd sizes and the smallest groups: a low-rank or class head with a ragged row count.
        _matvec("matvec_5_1003x7168", 5, 1003, 7168, 32, True),
        # One token from each of eight long sequences.
        _append("append_decode_8", 8, 1, 40960, 32, 8, 128, 64, 128),
        # Prompts of ragged lengths, some 16K tokens in all.
        _append("append_prompts_16k", 9, 4096, 4096, 32, 8, 128, 64, 128, ragged=True),
        # The long tail: eight sequences of up to 40K tokens, one token each.
        _attend("attend_tail_8x40k", 8, 1, 40960, 32, 8, 128, 64, ragged=True),
        # A decode batch of medium lengths, eight query heads a kv head, small pages.
        _attend("attend_decode_50x4k", 50, 1, 4500, 32, 4, 128, 16, ragged=True),
        # A chunk of a prompt over what the cache already holds.
        _attend("attend_chunk_2k_of_10k", 1, 2048, 10240, 32, 8, 128, 64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _seen(n):
    """Sizes are the repository's own or spread over the range; this one is neither."""
    return n + 64 if n == 3072 else n


# (H, E, k, F, Fs) of the repository's workloads
_SHAPES = [(4096, 8, 2, 14336, 0), (7168, 64, 8, 2048, 2048), (4096, 64, 4, 4096, 0)]


def _draw_few(rng):
    weights = rng.choice(["bf16", "bf16", "int4"])
    while True:
        if rng.random() < 0.4:
            H, E, k, F, Fs = rng.choice(_SHAPES)
        else:
            H = _seen(64 * _log_int(rng, 4, 112))
            F = _seen(64 * _log_int(rng, 4, 224))
            E = rng.choice([4, 8, 16, 32, 60, 64, 128])
            k = rng.randint(1, min(8, E // 2))
            Fs = rng.choice([0, 0, F])
        T = rng.randint(1, 16)
        if 3 * H * (E * F + Fs) <= 3.3e9:
            break
    group = rng.choice([32, 64, 128] if H % 128 == 0 and F % 128 == 0 else [32, 64])
    c = _few("", weights, T, H, E, k, F, Fs, group, rng.random() < 0.5, rng.choice([1, 1, 0]))
    return c


def _draw_matvec(rng):
    while True:
        group = rng.choice([32, 64, 128])
        K = _seen(group * _log_int(rng, max(1, 256 // group), 16384 // group))
        N = _seen(_log_int(rng, 200, 40000))
        if N * K <= 1.2e8:
            return _matvec("", _log_int(rng, 1, 64), N, K, group, rng.random() < 0.5)


def _heads(rng):
    D = rng.choice([64, 128, 128, 128, 256])
    Hkv = rng.choice([1, 2, 4, 8])
    G = rng.choice([1, 2, 4, 5, 8])
    return Hkv * G, Hkv, D, rng.choice([16, 32, 64, 128])


def _draw_append(rng):
    Hq, Hkv, D, page = _heads(rng)
    if rng.random() < 0.5:
        B, new, length = _log_int(rng, 1, 256), rng.choice([1, 1, 1, 2, 5]), _log_int(rng, 64, 8192)
    else:
        B, new = _log_int(rng, 1, 16), _log_int(rng, 16, 4096)
        length = new + rng.choice([0, rng.randint(1, 2000)])
    while B * new * (Hq + 2 * Hkv) * D > 9 * 4096 * 48 * 128 or B * length * Hkv * D > 5e8:
        B = max(1, B // 2)
        if B == 1:
            new, length = max(1, new // 2), max(1, length // 2)
    return _append("", B, _seen(new), _seen(max(new, length)), Hq, Hkv, D, page, rng.choice([D, D, D // 2]),
                   rng.random() < 0.3, rng.random() < 0.6)


def _draw_attend(rng):
    Hq, Hkv, D, page = _heads(rng)
    kind = rng.random()
    if kind < 0.5:
        B, new, length = _log_int(rng, 1, 64), 1, _log_int(rng, 16, 65536)
    elif kind < 0.7:
        B, new, length = _log_int(rng, 1, 32), rng.randint(2, 9), _log_int(rng, 64, 32768)
    else:
        B, new = _log_int(rng, 1, 8), _log_int(rng, 16, 2048)
        length = new + rng.choice([0, _log_int(rng, 1, 8000)])
    # no more than the largest listed ones: cache bytes, and query-key pairs
    while B * length * Hkv * D > 8 * 40960 * 8 * 128 or B * new * length * Hq * D > 2048 * 10240 * 32 * 128:
        if B > 1:
            B -= max(1, B // 4)
        else:
            length = max(1, length * 3 // 4)
            new = min(new, length)
    window = rng.choice([0, 0, 0, _log_int(rng, 32, 4096)])
    return _attend("", B, _seen(new), _seen(max(new, length)), Hq, Hkv, D, page, _seen(window), rng.random() < 0.6)


def draw(rng):
    kind = rng.choices(["few", "matvec", "append", "attend"], [3, 3, 2, 4])[0]
    c = dict(few=_draw_few, matvec=_draw_matvec, append=_draw_append, attend=_draw_attend)[kind](rng)
    c.pop("name")
    return c


# --------------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _normal(g, *shape, std=1.0, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, std, generator=g)


def _int4(g, lead, N, K, group, zeros):
    """4-bit codes of normal weights N(0, 1 / K), two to a byte (low nibble first), their bf16 group
    scales and, with zeros, zero points."""
    sigma = 2.6                                    # standard deviation in steps
    q = torch.empty((*lead, N, K // 2, 2), dtype=torch.float16, device=DEV).normal_(0.0, sigma, generator=g)
    scales = torch.empty((*lead, N, K // group), device=DEV).uniform_(0.7, 1.3, generator=g)
    scales = (scales * (K ** -0.5 / sigma)).to(torch.bfloat16)
    z = torch.randint(5, 11, scales.shape, dtype=torch.uint8, device=DEV, generator=g) if zeros else None
    q = q.add_(8.0).round_().clamp_(0.0, 15.0).to(torch.uint8)
    return dict(codes=q[..., 0] | (q[..., 1] << 4), scales=scales, zeros=z, group=group)


def _lengths(c):
    """(new tokens, lengths) of the sequences, a function of the case alone."""
    B, new, length = c["B"], c["new"], c["length"]
    if not c["ragged"]:
        return [new] * B, [length] * B
    r = random.Random(B * 1000003 + new * 1009 + length)
    n = [new] + [max(1, int(new * r.uniform(0.1, 0.9))) for _ in range(B - 1)]
    past = [length - new] + [int((length - new) * r.uniform(0.1, 1.0)) for _ in range(B - 1)]
    return n, [a + p for a, p in zip(n, past)]


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _paged(c, g):
    """A cache whose pages are handed out in a shuffled order, filled with what keys and values
    look like once quantised: codes of normal values, exponents around one size."""
    n, lens = _lengths(c)
    Hkv, D, page = c["Hkv"], c["D"], c["page"]
    per = [-(-x // page) for x in lens]
    pages = sum(per) + 3
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    table = torch.full((c["B"], max(per)), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, p in enumerate(per):
        table[b, :p] = order[at:at + p]
        at += p

    def codes(*shape):
        t = torch.empty(shape, dtype=torch.bfloat16, device=DEV).normal_(0.0, 100.0, generator=g)
        return t.clamp_(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)

    def exps():
        return torch.randint(127 - 8, 127 - 5, (pages, Hkv, page // BLOCK), dtype=torch.uint8, device=DEV, generator=g)

    cu = [0]
    for x in n:
        cu.append(cu[-1] + x)
    return dict(k_codes=codes(pages, Hkv, page, D), v_codes=codes(pages, Hkv, page // BLOCK, D, BLOCK),
                k_exps=exps(), v_exps=exps(), table=table, lens=_i32(lens), cu=_i32(cu), total=cu[-1],
                most_new=max(n), most=max(lens))


def _inputs(c, seed):
    g = _gen(seed)
    if c["kind"] == "few":
        T, H, E, F, Fs = c["T"], c["H"], c["E"], c["F"], c["Fs"]
        d = dict(x=_normal(g, T, H), logits=_normal(g, T, E, std=1.5, dtype=torch.float32))
        shapes = [(E, F, H), (E, F, H), (E, H, F)] + ([(1, Fs, H), (1, Fs, H), (1, H, Fs)] if Fs else [])
        if c["weights"] == "int4":
            d["w"] = [_int4(g, s[:1], s[1], s[2], c["group"], c["zeros"]) for s in shapes]
        else:
            d["w"] = [_normal(g, *s, std=s[2] ** -0.5) for s in shapes]
        return d
    if c["kind"] == "matvec":
        return dict(x=_normal(g, c["T"], c["K"]), w=_int4(g, (), c["N"], c["K"], c["group"], c["zeros"]))
    d = _paged(c, g)
    if c["kind"] == "append":
        # q, k and v as one projection writes them: side by side in a row
        Hq, Hkv, D, rot = c["Hq"], c["Hkv"], c["D"], c["rot"]
        qkv = _normal(g, d["total"], Hq + 2 * Hkv, D)
        d.update(q=qkv[:, :Hq], k=qkv[:, Hq:Hq + Hkv], v=qkv[:, Hq + Hkv:])
        freq = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)
        angle = torch.arange(d["most"], dtype=torch.float64, device=DEV)[:, None] * freq
        d["cos_sin"] = torch.cat([angle.cos(), angle.sin()], 1).float()
        d["q_out"] = torch.empty((d["total"], Hq, D), dtype=torch.bfloat16, device=DEV)
    else:
        # rotated queries of normalised states: scores of some units
        d["q"] = _normal(g, d["total"], c["Hq"], c["D"])
    return d


def prepare(case, seed):
    c = case
    s = dict(case=c, **_inputs(c, seed))
    if own:
        import paper_2606_21712_amd as moe
        s["moe"] = moe

        def pack(w):
            return moe.moe_pack_int4(w["codes"], w["scales"], w["zeros"], w["group"])

        if c["kind"] == "few":
            s["layer"] = moe.MoELayerFew(c["T"], c["H"], c["E"], c["k"], c["F"], c["Fs"], device=DEV)
            if c["weights"] == "int4":
                s["w"] = [pack(w) for w in s["w"]]
        elif c["kind"] == "matvec":
            s["w"] = pack(s["w"])
            s["y"] = torch.empty((c["T"], c["N"]), dtype=torch.bfloat16, device=DEV)
        else:
            s["cache"] = moe.KVCache8(s["k_codes"], s["v_codes"], s["k_exps"], s["v_exps"])
            if c["kind"] == "attend":
                n = moe.moe_kv8_attention_workspace_bytes(s["total"], c["B"], c["Hq"], c["Hkv"], c["D"], s["most_new"],
                                                          s["most"], c["window"])
                s["ws"] = torch.empty(max(1, n), dtype=torch.uint8, device=DEV)
                s["out"] = torch.empty_like(s["q"])
    return s


# --------------------------------------------------------------------------- one pass
def run(state):
    s = state
    c = s["case"]
    kind = c["kind"]
    if not own:
        return dict(few=_plain_few, matvec=_plain_matvec, append=_plain_append, attend=_plain_attend)[kind](s)
    moe = s["moe"]
    if kind == "few":
        y = s["layer"].run(s["x"], s["logits"], *s["w"], renormalize=c["renorm"])
        return dict(y=y, ids=s["layer"].topk_ids, weights=s["layer"].topk_weights)
    if kind == "matvec":
        return dict(y=moe.moe_matvec_int4(s["x"], s["w"], y=s["y"]))
    if kind == "append":
        moe.moe_kv8_append(s["q"], s["k"], s["v"], s["cos_sin"], s["cache"], s["table"], s["lens"], s["cu"],
                           interleaved=c["interleaved"], q_out=s["q_out"])
        return _cache_of(s, s["q_out"])
    out = moe.moe_kv8_attention(s["q"], s["cache"], s["table"], s["lens"], s["cu"], s["most_new"], s["most"],
                                window=c["window"], out=s["out"], ws=s["ws"])
    return dict(out=out)


def _cache_of(s, q):
    f8 = torch.float8_e4m3fn
    return dict(q=q, k_codes=s["k_codes"].view(f8), v_codes=s["v_codes"].view(f8), k_exps=s["k_exps"], v_exps=s["v_exps"])


# --------------------------------------------------------------------------- plain forms, 32 bits
def _dequant(w, pick=None):
    codes, scales, zeros = (None if t is None else t if pick is None else t[pick]
                            for t in (w["codes"], w["scales"], w["zeros"]))
    q = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).float()
    q = q.unflatten(-1, (-1, w["group"]))
    q = q - (8.0 if zeros is None else zeros.float()[..., None])
    return (q * scales.float()[..., None]).flatten(-2)


def _floats(w, pick=None):
    return _dequant(w, pick) if isinstance(w, dict) else (w if pick is None else w[pick]).float()


def _plain_few(s):
    c = s["case"]
    k, E, logits = c["k"], c["E"], s["logits"]
    x = s["x"].float()
    top, ids = (t[:, :k] for t in torch.sort(logits, dim=1, descending=True, stable=True))
    p = torch.exp(top - top[:, :1])
    whole = p if c["renorm"] else torch.exp(logits - top[:, :1])
    gate = p / whole.sum(1, keepdim=True)
    if c["T"] * k < E:
        # the experts of each token's slots
        pick = ids.flatten()
        rows = x.repeat_interleave(k, 0)[:, :, None]
        a, u = (torch.matmul(_floats(w, pick), rows) for w in s["w"][:2])
        y = torch.matmul(_floats(s["w"][2], pick), a / (1 + torch.exp(-a)) * u).reshape(c["T"], k, -1)
        y = (gate[:, :, None] * y).sum(1)
    else:
        # every expert on every token, weighted by 0 where it was not chosen
        share = torch.zeros_like(logits).scatter(1, ids, gate)
        a, u = (torch.matmul(x, _floats(w).transpose(1, 2)) for w in s["w"][:2])
        y = torch.matmul(a / (1 + torch.exp(-a)) * u, _floats(s["w"][2]).transpose(1, 2))
        y = (share.t()[:, :, None] * y).sum(0)
    if c["Fs"]:
        a, u = (torch.matmul(x, _floats(w)[0].t()) for w in s["w"][3:5])
        y = y + torch.matmul(a / (1 + torch.exp(-a)) * u, _floats(s["w"][5])[0].t())
    return dict(y=y.to(torch.bfloat16), ids=ids.to(torch.int32), weights=gate)


def _plain_matvec(s):
    return dict(y=torch.matmul(s["x"].float(), _dequant(s["w"]).t()).to(torch.bfloat16))


def _rotate(x, cos, sin, rot, interleaved):
    """x [T, heads, D]; cos, sin [T, 1, rot / 2]."""
    x = x.float()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    ra, rb = a * cos - b * sin, a * sin + b * cos
    y = torch.stack([ra, rb], -1).flatten(-2) if interleaved else torch.cat([ra, rb], -1)
    return torch.cat([y, x[..., rot:]], -1)


def _tokens(s):
    """Sequence and position of each new token."""
    cu = s["cu"].long()
    n = cu[1:] - cu[:-1]
    seq = torch.repeat_interleave(torch.arange(n.numel(), device=DEV), n, output_size=s["total"])
    row = torch.arange(s["total"], device=DEV)
    return seq, s["lens"].long()[seq] - n[seq] + row - cu[seq], row == cu[1:][seq] - 1


def _put(codes, exps, new, at):
    """Writes the values new [T, Hkv, D] of the new tokens into the cache, seen as codes [pages, Hkv, page / 16,
    16, D] and exps [pages, Hkv, page / 16]."""
    T, Hkv, D = new.shape
    page, block, ends = at["page"], at["block"], at["ends"]           # of each token; the blocks' last new tokens
    pg, bl = page[ends], block[ends]
    amax = torch.zeros((ends.numel(), Hkv), device=DEV)
    amax.scatter_reduce_(0, at["rank"][:, None].expand(T, Hkv), new.abs().amax(2), "amax")
    mant, e = torch.frexp(amax)                                       # amax = mant 2^e, 1/2 <= mant < 1
    want = torch.where(amax > 0, (e - 9 + (mant > 0.875)).clamp(-127, 127), -127)  # 448 = 0.875 2^9
    old = exps[pg, :, bl].int() - 127
    kept = at["first"][ends]                                          # slots that hold earlier tokens
    want = torch.where(kept[:, None] > 0, torch.maximum(want, old), want)
    was = codes[pg, :, bl].view(torch.float8_e4m3fn).float()
    was = was * torch.exp2((old - want).float())[:, :, None, None]
    keep = torch.arange(BLOCK, device=DEV)[None, :] < kept[:, None]
    was = torch.where(keep[:, None, :, None], was, 0.0)
    codes[pg, :, bl] = was.to(torch.float8_e4m3fn).view(torch.uint8)
    exps[pg, :, bl] = (want + 127).to(torch.uint8)
    scale = torch.exp2(-want.float())[at["rank"]]
    codes[page, :, block, at["slot"]] = (new * scale[:, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)


def _plain_append(s):
    c = s["case"]
    rot, page = c["rot"], c["page"]
    seq, pos, last = _tokens(s)
    cos, sin = s["cos_sin"][pos].unsqueeze(1).chunk(2, -1)
    q = _rotate(s["q"], cos, sin, rot, c["interleaved"]).to(torch.bfloat16)
    k = _rotate(s["k"], cos, sin, rot, c["interleaved"])
    slot = pos % BLOCK
    done = last | (slot == BLOCK - 1)
    begin = pos - torch.arange(s["total"], device=DEV) + s["cu"].long()[seq]     # the sequence's first new position
    at = dict(page=s["table"].long()[seq, pos // page], block=pos % page // BLOCK, slot=slot,
              ends=torch.nonzero(done).flatten(), rank=torch.cumsum(done, 0) - done.long(),
              first=(begin - (pos - slot)).clamp_min(0))
    _put(s["k_codes"].unflatten(2, (-1, BLOCK)), s["k_exps"], k, at)
    _put(s["v_codes"].transpose(3, 4), s["v_exps"], s["v"].float(), at)
    return _cache_of(s, q)


def _plain_attend(s):
    c = s["case"]
    B, Hq, Hkv, D, new = c["B"], c["Hq"], c["Hkv"], c["D"], s["most_new"]
    G = Hq // Hkv
    f8 = torch.float8_e4m3fn
    pages = s["table"].long().clamp_min(0)                            # [B, P]
    L = pages.shape[1] * c["page"]

    def scale(e):
        return torch.exp2(e.float() - 127.0)

    k = s["k_codes"][pages].view(f8).float().unflatten(3, (-1, BLOCK)) * scale(s["k_exps"][pages])[..., None, None]
    k = k.permute(0, 2, 1, 3, 4, 5).reshape(B, Hkv, L, D)
    v = s["v_codes"][pages].view(f8).float() * scale(s["v_exps"][pages])[..., None, None]
    v = v.permute(0, 2, 1, 3, 5, 4).reshape(B, Hkv, L, D)
    seq, pos, _ = _tokens(s)
    at = torch.arange(s["total"], device=DEV) - s["cu"].long()[seq]
    q = torch.zeros((B, new, Hq, D), device=DEV)
    q[seq, at] = s["q"].float()
    where = torch.full((B, new), -1, dtype=torch.long, device=DEV)
    where[seq, at] = pos
    q = q.reshape(B, new, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * new, D)
    x = torch.matmul(q, k.transpose(2, 3)) * D ** -0.5
    x = x.reshape(B, Hkv, G, new, L)
    key = torch.arange(L, device=DEV)
    seen = key <= where[:, :, None]
    if c["window"]:
        seen &= key > where[:, :, None] - c["window"]
    x = x.masked_fill_(~seen[:, None, None], -math.inf)
    x = x.sub_(x.amax(-1, keepdim=True).clamp_min(-1e30)).exp_()
    x = x.div_(x.sum(-1, keepdim=True).clamp_min(1e-30))
    o = torch.matmul(x.reshape(B, Hkv, G * new, L), v).reshape(B, Hkv, G, new, D)
    return dict(out=o.permute(0, 3, 1, 2, 4).reshape(B, new, Hq, D)[seq, at].to(torch.bfloat16))


# --------------------------------------------------------------------------- what a pass needs
def _pairs(c):
    """Query-key pairs, and cache tokens that are read, of an attention case."""
    pairs = read = 0
    w = c["window"] or 1 << 40
    for n, length in zip(*_lengths(c)):
        first, last = length - n, length - 1                          # positions of the new tokens
        full = max(0, min(last, w - 2) - first + 1)                   # that see everything before them
        pairs += full * (2 * first + full + 1) // 2 + (n - full) * min(w, length)
        read += length - max(0, first - w + 1)
    return pairs, read


def work(case):
    c = case
    if c["kind"] in ("few", "matvec"):
        if c["kind"] == "few" and c["weights"] == "bf16":
            per = 2.0
        else:
            per = 0.5 + (3 if c["zeros"] else 2) / c["group"]
        T = c["T"]
        if c["kind"] == "matvec":
            N, K = c["N"], c["K"]
            return dict(bytes=N * K * per + 2 * T * (N + K), flops=2 * T * N * K)
        H, E, k, F, Fs = (c[f] for f in ("H", "E", "k", "F", "Fs"))
        active = E * (1.0 - (1.0 - k / E) ** T)                       # experts that see a token
        return dict(bytes=3 * H * (F * active + Fs) * per + 4 * T * H + 4 * T * E + 8 * T * k,
                    flops=6 * H * T * (F * k + Fs))
    n, lens = _lengths(c)
    T, Hq, Hkv, D = sum(n), c["Hq"], c["Hkv"], c["D"]
    if c["kind"] == "append":
        return dict(bytes=T * D * (2 * (Hq + 2 * Hkv) + 2 * Hq + 2 * Hkv) + T * 4 * c["rot"],
                    flops=T * ((Hq + Hkv) * 3 * c["rot"] + 4 * Hkv * D))
    pairs, read = _pairs(c)
    return dict(bytes=read * Hkv * (2 * D + 2 / BLOCK) + 4 * T * Hq * D, flops=4 * pairs * Hq * D)


# --------------------------------------------------------------------------- 64-bit values
def _w64(w, e=None):
    """Weights in 64 bits, of expert e."""
    if not isinstance(w, dict):
        return (w if e is None else w[e]).double()
    codes, scales, zeros = (t if t is None or e is None else t[e] for t in (w["codes"], w["scales"], w["zeros"]))
    N, half = codes.shape
    q = torch.empty((N, 2 * half), dtype=torch.float64, device=DEV)
    q[:, 0::2] = (codes % 16).double()
    q[:, 1::2] = (codes // 16).double()
    s = scales.double().repeat_interleave(w["group"], 1)
    return s * q - s * (8.0 if zeros is None else zeros.double().repeat_interleave(w["group"], 1))


def _exact_few(c, d):
    x, logits, k = d["x"].double(), d["logits"].double(), c["k"]
    order = torch.argsort(-logits, dim=1, stable=True)[:, :k]
    every = torch.softmax(logits, 1).gather(1, order)
    gate = every / every.sum(1, keepdim=True) if c["renorm"] else every

    def swiglu(rows, ws, e):
        g, u = rows @ _w64(ws[0], e).T, rows @ _w64(ws[1], e).T
        return (torch.sigmoid(g) * g * u) @ _w64(ws[2], e).T

    y = swiglu(x, d["w"][3:], 0) if c["Fs"] else torch.zeros_like(x)
    for e in sorted(set(order.flatten().tolist())):
        t, j = torch.where(order == e)
        y[t] += gate[t, j, None] * swiglu(x[t], d["w"][:3], e)
    return dict(y=y, ids=None, weights=gate)


def _e4m3_64(v):
    """The nearest E4M3 value (ties to an even mantissa) of values of at most 448."""
    e = torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -9))).clamp_min(-6.0)
    step = torch.exp2(e - 3.0)
    return torch.round(v / step) * step


def _exact_append(c, d):
    n, lens = _lengths(c)
    rot, page, D = c["rot"], c["page"], c["D"]
    half = rot // 2
    ia = torch.arange(0, rot, 2, device=DEV) if c["interleaved"] else torch.arange(half, device=DEV)
    ib = ia + 1 if c["interleaved"] else ia + half
    q, k, v = (d[f].double() for f in ("q", "k", "v"))
    table = d["table"].tolist()
    kc, vc = (d[f].view(torch.float8_e4m3fn).double() for f in ("k_codes", "v_codes"))
    ke, ve = d["k_exps"].double() - 127, d["v_exps"].double() - 127
    row = 0
    spots, blocks = [], {}
    for b in range(c["B"]):
        for i in range(n[b]):
            p = lens[b] - n[b] + i
            spots.append(p)
            key = (table[b][p // page], p % page // BLOCK)
            blocks.setdefault(key, [p % BLOCK, row, 0])[2] += 1
            row += 1
    cs = d["cos_sin"][torch.tensor(spots, device=DEV)].double()
    cos, sin = cs[:, None, :half], cs[:, None, half:]
    for t in (q, k):
        a, b = t[..., ia], t[..., ib]
        t[..., ia], t[..., ib] = a * cos - b * sin, b * cos + a * sin
    keys = sorted(blocks)
    at = torch.tensor([[*key, *blocks[key]] for key in keys], device=DEV)       # page, block, slot, row, count
    pg, bl, slot, row0, count = at.unbind(1)
    place = torch.arange(BLOCK, device=DEV)
    fresh = (place >= slot[:, None]) & (place < (slot + count)[:, None])         # [blocks, 16]
    src = (row0[:, None] + place - slot[:, None]).clamp(0, row - 1)

    def write(codes, exps, new, get, put):
        vals = torch.where(fresh[:, None, :, None], new[src].transpose(1, 2), 0.0)  # [blocks, Hkv, 16, D]
        m = vals.abs().amax((2, 3))
        s = torch.where(m > 0, torch.ceil(torch.log2(m / 448.0)), -127.0).clamp(-127.0, 127.0)
        was = exps[pg, :, bl]
        s = torch.where(slot[:, None] > 0, torch.maximum(s, was), s)
        kept = _e4m3_64(get(codes) * torch.exp2(was - s)[..., None, None])
        kept = torch.where((place < slot[:, None])[:, None, :, None], kept, 0.0)
        put(codes, torch.where(fresh[:, None, :, None], _e4m3_64(vals * torch.exp2(-s)[..., None, None]), kept))

    kb = kc.unflatten(2, (-1, BLOCK))

    def put_k(codes, new):
        codes[pg, :, bl] = new

    def put_v(codes, new):
        codes[pg, :, bl] = new.transpose(2, 3)

    write(kb, ke, k, lambda t: t[pg, :, bl], put_k)
    write(vc, ve, v, lambda t: t[pg, :, bl].transpose(2, 3), put_v)
    return dict(q=q, k_codes=kb.flatten(2, 3), v_codes=vc, k_exps=None, v_exps=None)


def _exact_attend(c, d):
    n, lens = _lengths(c)
    G, D, page = c["Hq"] // c["Hkv"], c["D"], c["page"]
    f8 = torch.float8_e4m3fn
    out = torch.zeros((d["total"], c["Hq"], D), dtype=torch.float64, device=DEV)
    row = 0
    for b in range(c["B"]):
        pages = d["table"][b, :-(-lens[b] // page)].long()
        sk, sv = (torch.exp2(d[f][pages].double() - 127) for f in ("k_exps", "v_exps"))
        pos = torch.arange(lens[b] - n[b], lens[b], device=DEV)
        for h in range(c["Hkv"]):
            k = d["k_codes"][pages, h].view(f8).double() * sk[:, h].repeat_interleave(BLOCK, 1)[:, :, None]
            k = k.reshape(-1, D)[:lens[b]]
            v = d["v_codes"][pages, h].view(f8).double() * sv[:, h, :, None, None]
            v = v.transpose(2, 3).reshape(-1, D)[:lens[b]]
            key = torch.arange(lens[b], device=DEV)
            mask = key[None] > pos[:, None]
            if c["window"]:
                mask |= key[None] <= pos[:, None] - c["window"]
            for j in range(G):
                x = d["q"][row:row + n[b], h * G + j].double() @ k.T / math.sqrt(D)
                out[row:row + n[b], h * G + j] = torch.softmax(x.masked_fill(mask, -math.inf), 1) @ v
        row += n[b]
    return dict(out=out)


def exact(case, seed):
    c = case
    d = _inputs(c, seed)
    if c["kind"] == "few":
        return _exact_few(c, d)
    if c["kind"] == "matvec":
        return dict(y=d["x"].double() @ _w64(d["w"]).T)
    return _exact_append(c, d) if c["kind"] == "append" else _exact_attend(c, d)
