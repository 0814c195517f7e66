"""examples/decode_step.py: one layer of it against 64 bits, and its tokens."""
from __future__ import annotations

import importlib.util
import os

import numpy as np
import pytest
import torch

import paper_2606_21712_amd as moe
from gpu_util import log
from test_gpu_kv8 import HostCache, attention64, i32, rotate

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "decode_step.py")
    spec = importlib.util.spec_from_file_location("decode_step", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def dense(w):
    """A packed Int4 weight in 64 bits: products with the identity, 64 columns at a time."""
    K = w.shape[-1]
    eye = torch.eye(K, dtype=torch.bfloat16, device="cuda")
    mats = 1 if len(w.shape) == 2 else w.shape[0]
    cb, sb = w.codes.numel() // mats, w.scales.numel() // mats
    one = [moe.Int4(w.codes[i * cb:(i + 1) * cb], w.scales[i * sb:(i + 1) * sb], w.zeros, w.shape[-2:], w.group)
           for i in range(mats)]
    d = torch.stack([torch.cat([moe.moe_matvec_int4(eye[i:i + 64], m) for i in range(0, K, 64)]).T for m in one])
    return (d if len(w.shape) == 3 else d[0]).double().cpu()


def test_layer(example):
    """Bound: bf16 roundings, 2^-9 each, of some ten values on the way; twice that in the rms."""
    log("[gpu] decode example layer")
    H, Hq, Hkv, D, E, k, F = 256, 4, 2, 64, 8, 2, 256
    gen = torch.Generator(device="cuda").manual_seed(1)
    layer = example.Layer(H, Hq, Hkv, D, E, k, F, 6, 16, 2, 48, gen)
    table, cs = i32([[3, 1, 5], [0, 2, 4]]), torch.zeros(48, D, device="cuda")
    cs[:, :D // 2] = torch.cos(torch.arange(48, device="cuda")[:, None] * 0.3)
    cs[:, D // 2:] = torch.sin(torch.arange(48, device="cuda")[:, None] * 0.3)
    lens, new = [11, 5], [11, 5]
    x = torch.randn(16, H, generator=gen, device="cuda").to(torch.bfloat16)
    y = layer(x, cs, table, i32(lens), i32([0, 11, 16])).double().cpu()

    def norm(t):
        return t * torch.rsqrt(t.square().mean(-1, keepdim=True) + 1e-6)

    x = x.double().cpu()
    qkv = (norm(x) @ dense(layer.qkv).T).view(16, Hq + 2 * Hkv, D)
    pos = np.concatenate([np.arange(n) for n in lens])
    q = rotate(qkv[:, :Hq].numpy(), pos, cs.cpu().numpy(), False)
    host = HostCache(6, Hkv, 16, D)                             # the cache as the layer left it
    for to, t in ((host.k, layer.cache.k_codes), (host.v, layer.cache.v_codes), (host.ke, layer.cache.k_exps),
                  (host.ve, layer.cache.v_exps)):
        to[:] = t.cpu().numpy()
    a, _ = attention64(q, host, table.cpu().numpy(), lens, new, 0, D ** -0.5)
    x = x + torch.from_numpy(a).view(16, Hq * D) @ dense(layer.o).T
    h = norm(x)
    p = (h @ layer.router.double().cpu().T).gather(1, layer.moe.topk_ids.cpu().long())
    gate = torch.softmax(p, 1)
    w = [dense(t) for t in layer.experts]
    for t in range(16):
        for j in range(k):
            e = int(layer.moe.topk_ids[t, j])
            g, u = w[0][e] @ h[t], w[1][e] @ h[t]
            x[t] += gate[t, j] * (w[2][e] @ (g * torch.sigmoid(g) * u))
    assert (y - x).square().mean().sqrt() <= 20 * 2.0 ** -9 * x.square().mean().sqrt()


def test_tokens(example):
    """Greedy tokens lie in the vocabulary and are those of a second run, over a cache that has been used."""
    log("[gpu] decode example tokens")
    model = example.Model(layers=2, H=256, Hq=4, Hkv=2, D=64, E=8, k=2, F=256, vocab=500, page=16, max_seqs=3,
                          max_len=64)
    prompts = [[1, 2, 3], list(range(40)), [9] * 17]
    out = model.generate(prompts, 8)
    assert out.shape == (3, 8) and int(out.min()) >= 0 and int(out.max()) < 500
    assert torch.equal(out, model.generate(prompts, 8))
