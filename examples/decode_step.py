"""A small MoE transformer that decodes a few sequences greedily on the operators for a batch's last
sequences: 4-bit projections (moe_matvec_int4), the paged 8-bit cache (moe_kv8_append,
moe_kv8_attention) and the MoE layer for few tokens (MoELayerFew).  Weights are random.

    python examples/decode_step.py [--layers 4] [--sequences 4] [--prompt 40] [--new 64]

Prompts go in by chunks of 16 tokens, as many as the MoE layer takes at once, then each step takes one
token of every sequence; decoding does not synchronize."""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2606_21712_amd as moe  # noqa: E402


def rms_norm(x):
    f = x.float()
    return (f * torch.rsqrt(f.square().mean(-1, keepdim=True) + 1e-6)).to(torch.bfloat16)


class Layer:
    """Attention and the MoE layer, each on the normalised stream and added to it."""

    def __init__(self, H, Hq, Hkv, D, E, k, F, pages, page, max_seqs, max_len, gen, device="cuda"):
        self.heads = (Hq, Hkv, D)
        self.max_new, self.max_len = moe.FEW_TOKENS, max_len

        def weights(*shape):
            return (torch.randn(shape, generator=gen, device=device) * shape[-1] ** -0.5).to(torch.bfloat16)

        def int4(*shape):
            return moe.quantize_weights_int4(weights(*shape), group=64, zeros=True)

        self.qkv, self.o = int4((Hq + 2 * Hkv) * D, H), int4(H, Hq * D)
        self.router = weights(E, H).float()
        self.experts = int4(E, F, H), int4(E, F, H), int4(E, H, F)
        self.cache = moe.KVCache8.empty(pages, Hkv, D, page, device)
        self.moe = moe.MoELayerFew(moe.FEW_TOKENS, H, E, k, F, device=device)
        # one workspace for every step: the largest bounds, passed each time, and either number of sequences
        self.ws = torch.empty(max(moe.moe_kv8_attention_workspace_bytes(moe.FEW_TOKENS, B, Hq, Hkv, D, self.max_new,
                                                                        max_len) for B in range(1, max_seqs + 1)) + 1,
                              dtype=torch.uint8, device=device)

    def __call__(self, x, cos_sin, table, lens, cu):
        Hq, Hkv, D = self.heads
        T = x.shape[0]
        qkv = moe.moe_matvec_int4(rms_norm(x), self.qkv).view(T, Hq + 2 * Hkv, D)
        q = moe.moe_kv8_append(qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], cos_sin, self.cache, table, lens, cu)
        a = moe.moe_kv8_attention(q, self.cache, table, lens, cu, self.max_new, self.max_len, ws=self.ws)
        x = x + moe.moe_matvec_int4(a.view(T, Hq * D), self.o)
        h = rms_norm(x)
        return x + self.moe.run(h, h.float() @ self.router.T, *self.experts)


class Model:
    def __init__(self, layers=4, H=1024, Hq=16, Hkv=4, D=64, E=16, k=2, F=1024, vocab=4096, page=64, max_seqs=8,
                 max_len=1024, seed=0, device="cuda"):
        gen = torch.Generator(device=device).manual_seed(seed)
        self.per_seq = -(-max_len // page)
        if max_seqs > moe.FEW_TOKENS:
            raise ValueError(f"at most {moe.FEW_TOKENS} sequences")
        self.max_seqs, self.max_len = max_seqs, max_len
        self.layers = [Layer(H, Hq, Hkv, D, E, k, F, max_seqs * self.per_seq, page, max_seqs, max_len, gen, device)
                       for _ in range(layers)]
        self.embed, self.head = (torch.randn((vocab, H), generator=gen, device=device).to(torch.bfloat16)
                                 for _ in range(2))
        f = 10000.0 ** (-torch.arange(0, D, 2, device=device) / D)
        a = torch.arange(max_len, device=device)[:, None] * f
        self.cos_sin = torch.cat([a.cos(), a.sin()], 1).contiguous()
        # the pages of all sequences, in no order
        order = torch.randperm(max_seqs * self.per_seq, generator=gen, device=device).int()
        self.table = order.view(max_seqs, self.per_seq).contiguous()

    def step(self, tokens, seqs, lens, cu):
        """Logits of the rows: tokens [T], of the sequences `seqs` [B], whose lengths with these tokens are lens
        [B] i32 and whose rows cu [B + 1] i32; all on the GPU."""
        x = self.embed[tokens]
        table = self.table.index_select(0, seqs)
        for layer in self.layers:
            x = layer(x, self.cos_sin, table, lens, cu)
        return rms_norm(x) @ self.head.T

    def generate(self, prompts, new):
        """prompts: lists of tokens; the tokens decoded after each, [B, new]."""
        dev = self.embed.device

        def i32(v):
            return torch.tensor(v, dtype=torch.int32, device=dev)

        B, seqs = len(prompts), torch.arange(len(prompts), device=dev)
        if B > self.max_seqs or max(len(p) for p in prompts) + new > self.max_len:
            raise ValueError("too many sequences, or too long")
        last = []
        for b, p in enumerate(prompts):                      # chunked prefill
            for i in range(0, len(p), moe.FEW_TOKENS):
                chunk = p[i:i + moe.FEW_TOKENS]
                logits = self.step(torch.tensor(chunk, device=dev), seqs[b:b + 1], i32([i + len(chunk)]), i32([0, len(chunk)]))
            last.append(logits[-1].argmax())
        out = [torch.stack(last)]
        lens, cu = i32([len(p) for p in prompts]), i32(range(B + 1))
        for _ in range(new - 1):                             # one token of every sequence
            lens = lens + 1
            out.append(self.step(out[-1], seqs, lens, cu).argmax(-1))
        return torch.stack(out, 1)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, n in (("layers", 4), ("sequences", 4), ("prompt", 40), ("new", 64)):
        ap.add_argument("--" + name, type=int, default=n)
    a = ap.parse_args(argv)
    model = Model(layers=a.layers, max_seqs=a.sequences, max_len=a.prompt + a.sequences + a.new)
    prompts = [[(7 * b + 13 * i) % 4096 for i in range(a.prompt + b)] for b in range(a.sequences)]
    model.generate(prompts, 2)                               # first use of everything
    torch.cuda.synchronize()
    t = time.perf_counter()
    out = model.generate(prompts, a.new)
    torch.cuda.synchronize()
    print(f"{a.sequences} sequences, {a.new} tokens each in {time.perf_counter() - t:.3f} s")
    for b, row in enumerate(out.tolist()):
        print(b, row[:12], "..." if len(row) > 12 else "")
    return out


if __name__ == "__main__":
    main()
