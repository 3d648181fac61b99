"""Decode steps of a batch that shares a prompt: the decoder layer's operators (``Ops``) around the sparse FFN (``Ffn``).

A layer of the stack is

    h = rms(x) w1;  q, k, v = 8-bit projection of h;  rotate q and k, append k and v to the paged cache
    o = attention over the shared prompt's pages and the sequence's own
    x = x + rms(8-bit projection of o) w2            (norm after the block, gated residual update)
    x = x + sparse_ffn(x)                            (predict, select, the selected blocks alone)

The prompt runs through the layers once, in chunks, as one sequence whose FFN is the same sparse step; its pages then
serve every request.  Weights are random (the recipe of ``lsgen``): this shows the calls, it does not write text.

    python examples/decode_batch.py [--batch 8] [--prompt 200] [--steps 16]
"""
import argparse
import os
import sys
import time
from dataclasses import dataclass

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import lsgen  # noqa: E402
import paper_2609_03079_amd as lsffn  # noqa: E402

PAGE = 16


@dataclass
class Shape:
    layers: int = 2
    d: int = 1024
    heads: int = 8
    kv: int = 2
    dim: int = 128
    d_ff: int = 2816
    block: int = 32
    max_len: int = 512   # prompt and sequence together


def quantised(n, k, seed):
    """An [n, k] weight N(0, 1/k) in 8-bit integers with a scale for each row."""
    g = torch.Generator().manual_seed(seed)
    w = torch.randn((n, k), generator=g) / k ** 0.5
    s = w.abs().amax(1) / 127
    return (w / s[:, None]).round().to(torch.int8).cuda(), s.cuda()


class Decoder:
    """A stack of layers with its caches, for up to 8 tokens a step (the FFN's batch)."""

    def __init__(self, shape: Shape, batch: int, dtype=torch.bfloat16, seed=0):
        s, self.shape, self.batch, self.dtype = shape, shape, batch, dtype
        cfg = lsgen.CONFIGS["llama2_7b_ffn"].with_(n_layers=s.layers, d_model=s.d, d_ff=s.d_ff, block=s.block, rank=s.d // 4, seed=seed + 1)
        self.ops = lsffn.Ops()
        self.ffn = lsffn.Ffn(n_layers=s.layers, d_model=s.d, d_ff=s.d_ff, block=s.block, rank=cfg.rank, max_batch=8, dtype=cfg.dtype, act=cfg.act)
        self.keep = cfg.k
        self.layers = []
        pages = (batch + 1) * (s.max_len // PAGE)
        g = torch.Generator().manual_seed(seed)
        for l in range(s.layers):
            self.ffn.ls_ffn_set_layer(l, lsgen.layer_weights(cfg, l))
            w_qkv, s_qkv = quantised((s.heads + 2 * s.kv) * s.dim, s.d, seed + 10 * l + 1)
            w_o, s_o = quantised(s.d, s.heads * s.dim, seed + 10 * l + 2)
            norms = [(1 + 0.1 * torch.randn(s.d, generator=g)).to(dtype).cuda() for _ in range(2)]
            k, v = (torch.empty((pages, s.kv, PAGE, s.dim), dtype=dtype, device="cuda") for _ in range(2))
            self.layers.append((w_qkv, s_qkv, w_o, s_o, *norms, k, v))
        inv = 1e4 ** (-torch.arange(0, s.dim, 2, dtype=torch.float64) / s.dim)
        angle = torch.arange(s.max_len, dtype=torch.float64)[:, None] * inv
        self.table = torch.cat([angle.cos(), angle.sin()], 1).float().cuda()
        per = s.max_len // PAGE
        self.prompt_pages = torch.arange(per, dtype=torch.int32, device="cuda")
        self.pages = torch.arange(per, (batch + 1) * per, dtype=torch.int32, device="cuda").view(batch, per)
        self.prompt_len = 0

    def buffers(self, T):
        s, empty = self.shape, lambda *a: torch.empty(a, dtype=self.dtype, device="cuda")
        nb = s.d_ff // s.block
        return {"h": empty(T, s.d), "qkv": empty(T, (s.heads + 2 * s.kv) * s.dim), "q": empty(T, s.heads, s.dim), "o": empty(T, s.heads, s.dim),
                "y": empty(T, s.d), "x": [torch.empty((T, s.d), device="cuda") for _ in range(2)], "scores": torch.empty((T, nb), device="cuda"),
                "idx": torch.zeros(nb, dtype=torch.int32, device="cuda"), "count": torch.zeros(1, dtype=torch.int32, device="cuda")}

    def run(self, x, b, positions, slots, pages, lens, max_len, prefix_len, n_q):
        """The layers on T tokens x (fp32 [T, d]); returns x after the last."""
        s, T = self.shape, x.shape[0]
        for l, (w_qkv, s_qkv, w_o, s_o, w1, w2, k_cache, v_cache) in enumerate(self.layers):
            self.ops.ls_norm_residual(x, pre_norm=True, pre_weight=w1, h=b["h"])
            self.ops.ls_linear_i8(b["h"], w_qkv, s_qkv, b["qkv"])
            q, k, v = (t.view(T, -1, s.dim) for t in b["qkv"].split([s.heads * s.dim, s.kv * s.dim, s.kv * s.dim], 1))
            self.ops.ls_kv_append(k_cache, v_cache, k, v, positions, slots, self.table, q=q, q_out=b["q"])
            self.ops.ls_attend(b["q"], k_cache, v_cache, pages, lens, b["o"], n_q=n_q, max_len=max_len, prefix_pages=self.prompt_pages,
                               prefix_len=prefix_len, scale=s.dim ** -0.5)
            self.ops.ls_linear_i8(b["o"].view(T, -1), w_o, s_o, b["y"])
            self.ops.ls_norm_residual(x, y=b["y"], post_norm=True, post_weight=w2, x_out=b["x"][0])
            cap = min(s.d_ff // s.block, T * self.keep)
            self.ffn.ls_predict(l, b["x"][0], T, b["scores"])
            self.ffn.ls_select_blocks(b["scores"], T, lsffn.LS_SEL_TOPK, self.keep, 0.0, 1, cap, b["idx"], b["count"])
            self.ffn.ls_sparse_ffn_step(l, b["x"][0], T, b["idx"], b["count"], 0, cap, b["x"][1])
            x = b["x"][1]
        return x

    def prompt(self, x):
        """Runs the shared prompt x [n, d] through the layers, 8 tokens at a time, into its pages."""
        n, pages = x.shape[0], self.prompt_pages[None]
        for start in range(0, n, 8):
            T = min(8, n - start)
            at = torch.arange(start, start + T, dtype=torch.int32, device="cuda")
            # as one sequence without a prefix, whose last T tokens are the queries
            self.run(x[start:start + T].contiguous(), self.buffers(T), at, at, pages, torch.tensor([start + T], dtype=torch.int32, device="cuda"),
                     start + T, 0, T)
        self.prompt_len = n

    def step(self, x, b, lens):
        """One token x [batch, d] for each sequence; lens: int32 [batch], the sequence's tokens before it."""
        slots = self.pages.gather(1, (lens // PAGE).long()[:, None])[:, 0] * PAGE + lens % PAGE
        out = self.run(x, b, self.prompt_len + lens, slots, self.pages, lens + 1, self.shape.max_len - self.prompt_len, self.prompt_len, 1)
        lens.add_(1)
        return out

    def close(self):
        self.ops.close()
        self.ffn.close()


def main():
    p = argparse.ArgumentParser()
    p.add_argument("--batch", type=int, default=8)
    p.add_argument("--prompt", type=int, default=200)
    p.add_argument("--steps", type=int, default=16)
    a = p.parse_args()
    shape = Shape()
    if not 1 <= a.batch <= 8 or a.prompt < 0 or a.prompt + a.steps + 1 > shape.max_len:
        p.error(f"a batch of 1 to 8, and prompt and steps within {shape.max_len} positions")
    model = Decoder(shape, a.batch)
    g = torch.Generator().manual_seed(7)
    model.prompt(torch.randn((a.prompt, shape.d), generator=g).cuda())
    b, lens = model.buffers(a.batch), torch.zeros(a.batch, dtype=torch.int32, device="cuda")
    x = torch.randn((a.steps + 1, a.batch, shape.d), generator=g).cuda()
    model.step(x[0], b, lens)
    torch.cuda.synchronize()
    t = time.perf_counter()
    for i in range(a.steps):
        out = model.step(x[i + 1], b, lens)
    model.ffn.ls_ffn_sync()
    t = (time.perf_counter() - t) / a.steps
    print(f"{a.batch} sequences behind {a.prompt} shared tokens, {shape.layers} layers: {t * 1e6:.0f} us a step; |x| {float(out.norm(dim=1).mean()):.3f}")
    model.close()


if __name__ == "__main__":
    main()
