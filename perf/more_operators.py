"""Performance cases of the dense half of a transformer layer in 8-bit integers: what runs before,
after and beside the MoE layer.

A case is a dict of plain values, its "kind" one of

    norm      moe_norm_join: a block's output normalised, gated, scaled and added to the stream,
              and the stream normalised for the next block
    quantize  moe_quantize_int8: bf16 rows to 8-bit codes with a scale for each row
    matmul    moe_matmul_int8: product of codes with scales for each row of both operands
    gated     moe_gated_int8: both projections of a gated feed-forward block, activation and product
    project   moe_norm_join giving codes, then moe_matmul_int8 on them: a block's first projection

Codes are -127..127, scales fp32.  Weights are row-major codes [N, K] with a scale for each row; the
framework packs them once.  Every input is drawn on the GPU from the seed alone.
"""
from __future__ import annotations

import math

import torch

own = False     # True: run() makes the framework's calls, False: the plain form
DEV = "cuda"
EPS = 1e-6


# --------------------------------------------------------------------------- the cases
def _norm(name, T, H, post, gate, alpha=1.0, stream="bf16"):
    return dict(name=name, kind="norm", T=T, H=H, post=post, gate=gate, alpha=alpha, stream=stream)


def _quantize(name, T, K):
    return dict(name=name, kind="quantize", T=T, K=K)


def _matmul(name, T, N, K, bias=False):
    return dict(name=name, kind="matmul", T=T, N=N, K=K, bias=bias)


def _gated(name, T, F, K):
    return dict(name=name, kind="gated", T=T, F=F, K=K)


def _project(name, T, N, H, post=True, gate="none", alpha=1.0):
    return dict(name=name, kind="project", T=T, N=N, H=H, post=post, gate=gate, alpha=alpha)


def listed():
    return [
        # One token between two blocks: a launch and its latency.
        _norm("norm_1x4096", 1, 4096, True, "none"),
        # A prompt's rows after a shared expert, gated by a sigmoid for each token.
        _norm("norm_9001x7168", 9001, 7168, True, "token", alpha=0.5),
        # The last sequences' activations.
        _quantize("quantize_9x7168", 9, 7168),
        # h of a wide feed-forward block on its way to the down projection.
        _quantize("quantize_8192x14336", 8192, 14336),
        # The down projection for one token: 59 MB of weights.
        _matmul("matmul_1_4096x14336", 1, 4096, 14336),
        # Queries, keys and values of a middling batch in one projection with a bias, an odd number of channels.
        _matmul("matmul_333_6145x4096", 333, 6145, 4096, bias=True),
        # The down projection for a large batch.
        _matmul("matmul_16384_4096x14336", 16384, 4096, 14336),
        # A shared expert for the last eight sequences.
        _gated("gated_8_2048x7168", 8, 2048, 7168),
        # A narrow feed-forward block for a ragged batch.
        _gated("gated_700_1408x2816", 700, 1408, 2816),
        # The wide feed-forward block on a large batch.
        _gated("gated_8192_14336x4096", 8192, 14336, 4096),
        # One token from the end of a block to the next one's queries, keys and values.
        _project("project_1_6144x4096", 1, 6144, 4096),
        # The same for a prompt, without a norm after the block, with a learned gate for each channel.
        _project("project_2003_4608x7168", 2003, 4608, 7168, post=False, gate="channel"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _rows(rng):
    lo, hi = rng.choice([(1, 64), (1, 64), (65, 1024), (1025, 16384)])
    return _log_int(rng, lo, hi)


_GATES = ["none", "none", "channel", "token", "full"]


def _draw_norm(rng):
    while True:
        T, H = _rows(rng), 8 * _log_int(rng, 32, 2048)
        if T * H <= 9001 * 7168:
            return _norm("", T, H, rng.random() < 0.6, rng.choice(_GATES), rng.choice([1.0, 0.5, 0.22]),
                         rng.choice(["bf16", "bf16", "f32"]))


def _draw_quantize(rng):
    while True:
        T, K = _rows(rng), 16 * _log_int(rng, 16, 1024)
        if T * K <= 8192 * 14336:
            return _quantize("", T, K)


def _draw_matmul(rng):
    while True:
        T, N, K = _rows(rng), _log_int(rng, 100, 30000), 16 * _log_int(rng, 16, 1024)
        if T * N * K <= 16384 * 4096 * 14336 and N * K <= 1.2e8 and T * N <= 1.2e8:
            return _matmul("", T, N, K, rng.random() < 0.4)


def _draw_gated(rng):
    while True:
        T, F, K = _rows(rng), 16 * _log_int(rng, 16, 1024), 16 * _log_int(rng, 16, 512)
        if T * F * K <= 8192 * 14336 * 4096 and F * K <= 6e7 and T * F <= 1.2e8:
            return _gated("", T, F, K)


def _draw_project(rng):
    while True:
        T, N, H = _rows(rng), _log_int(rng, 256, 20000), 16 * _log_int(rng, 16, 512)
        if T * N * H <= 8192 * 14336 * 4096 and N * H <= 1.2e8 and T * N <= 1.2e8 and T * H <= 9001 * 7168:
            return _project("", T, N, H, rng.random() < 0.6, rng.choice(_GATES), rng.choice([1.0, 0.5]))


def draw(rng):
    kind = rng.choices(["norm", "quantize", "matmul", "gated", "project"], [2, 2, 3, 3, 2])[0]
    c = dict(norm=_draw_norm, quantize=_draw_quantize, matmul=_draw_matmul, gated=_draw_gated,
             project=_draw_project)[kind](rng)
    c.pop("name")
    return c


# --------------------------------------------------------------------------- inputs
def _normal(g, *shape, std=1.0, mean=0.0, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(mean, std, generator=g)


def _codes(g, rows, K):
    """Codes and scales of normal rows: the largest of a row at 127, the others as far below as normal values lie."""
    q = _normal(g, rows, K, std=127 / 3.9, dtype=torch.float32).round_().clamp_(-127, 127)
    s = torch.empty(rows, device=DEV).uniform_(0.7, 1.3, generator=g)
    return q.to(torch.int8), s


def _weights(g, N, K):
    q, s = _codes(g, N, K)
    return dict(codes=q, scales=s * (K ** -0.5 * 3.9 / 127))          # of weights N(0, 1 / K)


def _activations(g, T, K):
    q, s = _codes(g, T, K)
    return dict(codes=q, scales=s * (3.9 / 127))


def _stream(c, g):
    """The residual stream with some large channels, a block's output, its gate and the norms' weights."""
    T, H = c["T"], c["H"]
    wide = torch.where(torch.rand(H, device=DEV, generator=g) < 0.01, 20.0, 2.0)
    x = _normal(g, T, H, dtype=torch.float32) * wide
    d = dict(x=x if c.get("stream") == "f32" else x.to(torch.bfloat16), y=_normal(g, T, H),
             w_pre=_normal(g, H, std=0.2, mean=1.0), w_post=_normal(g, H, std=0.2, mean=1.0) if c["post"] else None)
    shape = dict(none=None, channel=(1, H), token=(T, 1), full=(T, H))[c["gate"]]
    d["gate"] = None if shape is None else _normal(g, *shape)
    return d


def _inputs(c, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    kind = c["kind"]
    if kind == "norm":
        return _stream(c, g)
    if kind == "quantize":
        # rows of h: products of two normal values, of sizes that differ from row to row
        h = _normal(g, c["T"], c["K"]) * _normal(g, c["T"], c["K"])
        return dict(src=h * torch.empty((c["T"], 1), device=DEV).uniform_(0.2, 3.0, generator=g).to(torch.bfloat16))
    if kind == "matmul":
        return dict(x=_activations(g, c["T"], c["K"]), w=_weights(g, c["N"], c["K"]),
                    bias=_normal(g, c["N"]) if c["bias"] else None)
    if kind == "gated":
        return dict(x=_activations(g, c["T"], c["K"]), w_gate=_weights(g, c["F"], c["K"]),
                    w_up=_weights(g, c["F"], c["K"]))
    return dict(**_stream(c, g), w=_weights(g, c["N"], c["H"]))


def prepare(case, seed):
    c = case
    s = dict(case=c, **_inputs(c, seed))
    if own:
        import paper_2606_21712_amd as moe
        s["moe"] = moe

        def buffer(*shape, dtype=torch.bfloat16):
            return torch.empty(shape, dtype=dtype, device=DEV)

        def pack(w):
            return moe.moe_pack_int8(w["codes"], w["scales"])

        kind, T = c["kind"], c["T"]
        if kind in ("norm", "project"):
            s["x_out"] = torch.empty_like(s["x"])
            s["z"] = buffer(T, c["H"], dtype=torch.bfloat16 if kind == "norm" else torch.int8)
            s["z_scales"] = None if kind == "norm" else buffer(T, dtype=torch.float32)
        if kind == "quantize":
            s["codes"], s["scales"] = buffer(T, c["K"], dtype=torch.int8), buffer(T, dtype=torch.float32)
        if kind in ("matmul", "project"):
            s["w"] = pack(s["w"])
            s["out"] = buffer(T, c["N"])
            s["ws"] = buffer(max(1, moe.moe_matmul_int8_workspace_bytes(T, c["N"], s["w"].shape[1])), dtype=torch.uint8)
        if kind == "gated":
            s["w_gate"], s["w_up"] = pack(s["w_gate"]), pack(s["w_up"])
            s["out"] = buffer(T, c["F"])
            s["ws"] = buffer(max(1, moe.moe_gated_int8_workspace_bytes(T, c["F"], c["K"])), dtype=torch.uint8)
    return s


# --------------------------------------------------------------------------- one pass
def run(state):
    s = state
    c = s["case"]
    kind = c["kind"]
    if not own:
        return dict(norm=_plain_norm, quantize=_plain_quantize, matmul=_plain_matmul, gated=_plain_gated,
                    project=_plain_project)[kind](s)
    moe = s["moe"]
    if kind == "quantize":
        codes, scales = moe.moe_quantize_int8(s["src"], codes=s["codes"], scales=s["scales"])
        return dict(codes=codes, scales=scales)
    if kind == "matmul":
        return dict(y=moe.moe_matmul_int8(s["x"]["codes"], s["x"]["scales"], s["w"], bias=s["bias"], y=s["out"],
                                          ws=s["ws"]))
    if kind == "gated":
        return dict(h=moe.moe_gated_int8(s["x"]["codes"], s["x"]["scales"], s["w_gate"], s["w_up"], h=s["out"],
                                         ws=s["ws"]))
    x, z, scales = moe.moe_norm_join(s["x"], s["y"], post=s["w_post"], gate=s["gate"], sigmoid=c["gate"] == "token",
                                     alpha=c["alpha"], pre=s["w_pre"], eps=EPS, int8=kind == "project",
                                     x_out=s["x_out"], z=s["z"], scales=s["z_scales"])
    if kind == "norm":
        return dict(x=x, z=z)
    return dict(x=x, y=moe.moe_matmul_int8(z, scales, s["w"], y=s["out"], ws=s["ws"]))


# --------------------------------------------------------------------------- plain forms, 32 bits
def _rms(v, w):
    return v * torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS) * w.float()


def _join(s):
    c = s["case"]
    j = s["y"].float()
    if c["post"]:
        j = _rms(j, s["w_post"])
    if s["gate"] is not None:
        g = s["gate"].float()
        j = (1 / (1 + torch.exp(-g)) if c["gate"] == "token" else g) * j
    x = s["x"].float() + c["alpha"] * j
    return x, _rms(x, s["w_pre"])


def _plain_norm(s):
    x, z = _join(s)
    return dict(x=x.to(s["x"].dtype), z=z.to(torch.bfloat16))


def _to_codes(v):
    """Codes and scales of the rows of v.  The two quotients are taken in 64 bits and rounded, which gives
    the correctly rounded fp32 quotient whatever the device's fp32 division does."""
    m = v.abs().amax(-1, keepdim=True).double()
    inverse = torch.where(m > 0, 127 / m, 0.0).float()
    return torch.round(v * inverse).to(torch.int8), (m / 127).float().squeeze(-1)


def _plain_quantize(s):
    codes, scales = _to_codes(s["src"].float())
    return dict(codes=codes, scales=scales)


def _product(codes, scales, w):
    return torch.matmul(codes.float(), w["codes"].float().t()) * scales[:, None] * w["scales"]


def _plain_matmul(s):
    y = _product(s["x"]["codes"], s["x"]["scales"], s["w"])
    if s["bias"] is not None:
        y = y + s["bias"].float()
    return dict(y=y.to(torch.bfloat16))


def _plain_gated(s):
    g, u = (_product(s["x"]["codes"], s["x"]["scales"], s[w]) for w in ("w_gate", "w_up"))
    return dict(h=(g / (1 + torch.exp(-g)) * u).to(torch.bfloat16))


def _plain_project(s):
    x, z = _join(s)
    return dict(x=x.to(s["x"].dtype), y=_product(*_to_codes(z), s["w"]).to(torch.bfloat16))


# --------------------------------------------------------------------------- what a pass needs
def work(case):
    c = case
    T = c["T"]
    if c["kind"] == "quantize":
        return dict(bytes=T * (3 * c["K"] + 4), flops=3 * T * c["K"])
    if c["kind"] == "matmul":
        N, K = c["N"], c["K"]
        return dict(bytes=(T + N) * (K + 4) + 2 * T * N + (2 * N if c["bias"] else 0), flops=2 * T * N * K)
    if c["kind"] == "gated":
        F, K = c["F"], c["K"]
        return dict(bytes=(T + 2 * F) * (K + 4) + 2 * T * F, flops=4 * T * F * K)
    H = c["H"]
    gate = dict(none=0, channel=2 * H, token=2 * T, full=2 * T * H)[c["gate"]]
    both = (8 if c.get("stream") == "f32" else 4) * T * H + 2 * T * H + gate + (4 if c["post"] else 2) * H
    if c["kind"] == "norm":
        return dict(bytes=both + 2 * T * H, flops=12 * T * H)
    N = c["N"]
    return dict(bytes=both + N * (H + 4) + 2 * T * N, flops=2 * T * N * H + 12 * T * H)


# --------------------------------------------------------------------------- 64-bit values
def _scaled64(m):
    return m["codes"].double() * m["scales"].double().unsqueeze(1)


def _stream64(c, d):
    y = d["y"].double()
    if c["post"]:
        y = y / (y.square().sum(1, keepdim=True) / c["H"] + EPS).sqrt() * d["w_post"].double()
    if c["gate"] == "token":
        y = torch.sigmoid(d["gate"].double()) * y
    elif c["gate"] != "none":
        y = d["gate"].double() * y
    x = torch.add(d["x"].double(), y, alpha=c["alpha"])
    return x, x / (x.square().sum(1, keepdim=True) / c["H"] + EPS).sqrt() * d["w_pre"].double()


def exact(case, seed):
    c = case
    d = _inputs(c, seed)
    if c["kind"] == "quantize":
        return dict(codes=None, scales=d["src"].abs().double().max(1).values / 127)
    if c["kind"] == "matmul":
        y = _scaled64(d["x"]) @ _scaled64(d["w"]).T
        return dict(y=y if d["bias"] is None else y + d["bias"].double())
    if c["kind"] == "gated":
        x = _scaled64(d["x"])
        return dict(h=torch.nn.functional.silu(x @ _scaled64(d["w_gate"]).T) * (x @ _scaled64(d["w_up"]).T))
    x, z = _stream64(c, d)
    if c["kind"] == "norm":
        return dict(x=x, z=z)
    step = z.abs().max(1, keepdim=True).values / 127
    return dict(x=x, y=(torch.round(z / step) * step) @ _scaled64(d["w"]).T)
