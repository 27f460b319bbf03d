"""One sequence decoded token by token through a small random decoder: every
projection a dual-sparse SpMSpV, and around them the library's other operators:
the block norm with its gate and residual, the 4-bit key/value cache with its
attention, and sampling.

    python examples/decode_step.py [--tokens N] [--layers L] [--eager]

Weights are random, N(0, 0.02) under a 50 % unstructured mask; there is nothing
to read in the tokens.  A step runs entirely on the GPU (positions, lengths and
the chosen token are device values), so it is captured once as a HIP graph and
replayed; --eager issues it call by call.  Rotary positions and the gated
activation of the feed-forward block are plain torch.
"""
from __future__ import annotations

import argparse
import dataclasses
import math
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_01536_amd as celty  # noqa: E402


@dataclasses.dataclass
class Config:
    layers: int = 2
    heads: int = 8
    kv_heads: int = 2
    head_dim: int = 128
    ffn: int = 2816
    vocabulary: int = 32000
    page_tokens: int = 32
    max_tokens: int = 512
    weight_sparsity: float = 0.5
    tau: float = 0.6            # of the normalised activations, about 45 % inactive
    tau_inner: float = 0.01     # of attention's output and the feed-forward block's
    residual_scale: float = 0.5

    @property
    def hidden(self) -> int:
        return self.heads * self.head_dim


class Layer:
    """A decoder layer's encoded matrices and norm weights; q, k and v, and gate
    and up, are stacked, so a layer is four products."""

    def __init__(self, cfg: Config, rng: np.random.Generator, device):
        qkv = (cfg.heads + 2 * cfg.kv_heads) * cfg.head_dim
        self.dense = {}

        def matrix(name, rows, cols):
            w = (rng.standard_normal((rows, cols), dtype=np.float32) * 0.02).astype(np.float16)
            mask = (rng.random((rows, cols), dtype=np.float32) >= cfg.weight_sparsity).astype(np.uint8)
            self.dense[name] = np.where(mask, w, np.float16(0))
            return celty.celty_encode(w, mask, celty.default_tile_rows(rows, cols)).to_device(device)

        self.qkv = matrix("qkv", qkv, cfg.hidden)
        self.out = matrix("out", cfg.hidden, cfg.heads * cfg.head_dim)
        self.gate_up = matrix("gate_up", 2 * cfg.ffn, cfg.hidden)
        self.down = matrix("down", cfg.hidden, cfg.ffn)

        def vector(scale):
            return torch.from_numpy((1 + scale * rng.standard_normal(cfg.hidden)).astype(np.float16)).to(device)
        # weights of the norms before attention and feed-forward, after them, and the blocks' gates
        self.w_attn, self.w_ffn, self.w_attn_post, self.w_ffn_post = (vector(0.1) for _ in range(4))
        self.g_attn, self.g_ffn = vector(0.05), vector(0.05)


class Decoder:
    def __init__(self, cfg: Config, seed: int = 0, device="cuda"):
        self.cfg, self.device = cfg, torch.device(device)
        rng = np.random.default_rng(seed)
        self.layers = [Layer(cfg, rng, self.device) for _ in range(cfg.layers)]
        h, V = cfg.hidden, cfg.vocabulary
        self.embedding = torch.from_numpy(rng.standard_normal((V, h), dtype=np.float32).astype(np.float16)).to(device)
        head = (rng.standard_normal((V, h), dtype=np.float32) * 0.05).astype(np.float16)
        mask = (rng.random((V, h), dtype=np.float32) >= cfg.weight_sparsity).astype(np.uint8)
        self.head_dense = np.where(mask, head, np.float16(0))
        self.head = celty.celty_encode(head, mask, celty.default_tile_rows(V, h)).to_device(device)
        self.w_last = torch.ones(h, dtype=torch.float16, device=device)

        def half(*shape):
            return torch.empty(*shape, dtype=torch.float16, device=device)
        H, K, D = cfg.heads, cfg.kv_heads, cfg.head_dim
        self.h = torch.zeros(1, h, device=device)                     # the residual stream, fp32
        self.x, self.y = half(1, h), half(1, h)                       # a block's input and output
        self.qkv, self.q, self.attended = half(H + 2 * K, D), half(1, H, D), half(1, H, D)
        self.k, self.gate_up, self.act = half(1, K, D), half(2, cfg.ffn), half(cfg.ffn)
        self.logits, self.noise = half(1, V), torch.empty(1, V, device=device)
        self.token = torch.zeros(1, dtype=torch.int32, device=device)
        # one workspace for the largest product: calls of one stream follow each other
        mats = [m for l in self.layers for m in (l.qkv, l.out, l.gate_up, l.down)] + [self.head]
        self.ws = torch.zeros(max(celty.celty_spmspv_workspace_bytes(m.M, m.K, m.R) for m in mats), dtype=torch.uint8, device=device)
        # the cache: a layer's pages in any order, named by its row of the table
        pages = -(-cfg.max_tokens // cfg.page_tokens)
        self.kv_len = torch.zeros(1, dtype=torch.int32, device=device)
        self.caches, self.seqs = [], []
        for _ in self.layers:
            self.caches.append(celty.Kv4Cache(pages, K, D, cfg.page_tokens, device))
            table = torch.from_numpy(rng.permutation(pages).astype(np.int32)).to(device).view(1, -1)
            self.seqs.append(celty.Kv4Seqs(table, self.kv_len))
        self.ws_attn = celty.new_kv4_workspace(self.caches[0], self.seqs[0], 1, H)
        self.ws_sample = celty.new_sample_workspace(self.logits)
        f = dict(dtype=torch.float32, device=device)
        self.filters = dict(temperature=torch.full((1,), 0.8, **f), top_p=torch.full((1,), 0.95, **f),
                            top_k=torch.full((1,), 50, dtype=torch.int32, device=device))
        angle = torch.arange(cfg.max_tokens, **f)[:, None] * 10000.0 ** (-torch.arange(D // 2, **f) / (D // 2))[None]
        self.cos, self.sin = angle.cos(), angle.sin()

    def _rotate(self, x):
        """x [heads, D] at the current position (rotary, halves paired)."""
        at = (self.kv_len - 1).long()
        c, s = self.cos[at], self.sin[at]
        a, b = x.float().chunk(2, dim=-1)
        return torch.cat([a * c - b * s, a * s + b * c], dim=-1)

    def step(self) -> None:
        """self.token in, the next token out; everything stays on the GPU.  At most
        max_tokens steps after a reset."""
        cfg, H, K = self.cfg, self.cfg.heads, self.cfg.kv_heads
        self.kv_len.add_(1)
        self.h.copy_(self.embedding[self.token.long()])
        block, post, gate = None, None, None     # the block whose output is still to be added
        for layer, cache, seqs in zip(self.layers, self.caches, self.seqs):
            celty.celty_block_norm(self.h, block, self.h, self.x, w_pre=layer.w_attn, w_post=post, gate=gate,
                                   alpha=cfg.residual_scale)
            celty.celty_spmspv(layer.qkv, self.x, cfg.tau, self.qkv, self.ws)
            self.q[0].copy_(self._rotate(self.qkv[:H]))
            self.k[0].copy_(self._rotate(self.qkv[H:H + K]))
            celty.celty_kv4_append(cache, seqs, self.k, self.qkv[H + K:].unsqueeze(0))
            celty.celty_kv4_attention(cache, seqs, self.q, self.attended, self.ws_attn)
            celty.celty_spmspv(layer.out, self.attended, cfg.tau_inner, self.y, self.ws)
            celty.celty_block_norm(self.h, self.y, self.h, self.x, w_pre=layer.w_ffn, w_post=layer.w_attn_post,
                                   gate=layer.g_attn, alpha=cfg.residual_scale)
            celty.celty_spmspv(layer.gate_up, self.x, cfg.tau, self.gate_up, self.ws)
            torch.mul(torch.nn.functional.silu(self.gate_up[0]), self.gate_up[1], out=self.act)
            celty.celty_spmspv(layer.down, self.act, cfg.tau_inner, self.y, self.ws)
            block, post, gate = self.y, layer.w_ffn_post, layer.g_ffn
        celty.celty_block_norm(self.h, block, None, self.x, w_pre=self.w_last, w_post=post, gate=gate, alpha=cfg.residual_scale)
        celty.celty_spmspv(self.head, self.x, cfg.tau, self.logits, self.ws)
        self.noise.exponential_()
        celty.celty_sample(self.logits, self.noise, self.token, self.ws_sample, **self.filters)

    def reset(self, token: int) -> None:
        self.kv_len.zero_()
        self.token.fill_(token)

    def capture(self) -> torch.cuda.CUDAGraph:
        """The step as a graph; the state is then as after reset to the present token."""
        token = self.token.clone()
        self.kv_len.zero_()   # the step below must find room
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            self.step()   # torch's own kernels are loaded outside of the capture
        torch.cuda.current_stream().wait_stream(side)
        self.kv_len.zero_()
        self.token.copy_(token)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            self.step()
        return graph


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--tokens", type=int, default=64)
    p.add_argument("--layers", type=int, default=2)
    p.add_argument("--seed", type=int, default=0)
    p.add_argument("--eager", action="store_true")
    args = p.parse_args()
    cfg = Config(layers=args.layers)
    if not 1 <= args.tokens <= cfg.max_tokens:
        p.error(f"--tokens must be between 1 and {cfg.max_tokens}")
    torch.manual_seed(args.seed)
    decoder = Decoder(cfg, args.seed)
    advance = decoder.step if args.eager else decoder.capture().replay
    decoder.reset(1)
    torch.cuda.synchronize()
    start, tokens = time.perf_counter(), []
    for _ in range(args.tokens):
        advance()
        tokens.append(decoder.token.clone())
    torch.cuda.synchronize()
    us = (time.perf_counter() - start) / args.tokens * 1e6
    print(f"{args.tokens} tokens, {cfg.layers} layers of {cfg.hidden}: {us:.0f} us a token")
    print(" ".join(str(int(t)) for t in tokens))


if __name__ == "__main__":
    main()
