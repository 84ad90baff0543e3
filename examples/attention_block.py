"""The attention half of a served transformer block in W4A4KV4, from the library's operators: what stands between two residual
streams, for prompts and for decode steps, on one paged INT4 cache.

    x, residual -> basq_add_rms_norm -> W4A4 qkv projection -> basq_rope_append -> basq_paged_attention -> W4A4 output projection

Random weights; run on one GPU:

    python examples/attention_block.py --prompts 700,33,257 --steps 32
"""
from __future__ import annotations

import argparse
import math
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2506_15689_amd import binding as B  # noqa: E402

CLIP = 0.9


class Linear:
    """A W4A4 rotated linear layer without a bias: weights quantised once, kept in the layouts of decode and of prompts."""

    def __init__(self, W: torch.Tensor):
        N, K = W.shape
        dev = W.device
        self.N, self.K = N, K
        rotated = torch.empty_like(W)
        B.basq_rotate_weights(W, K, rotated, torch.empty(N * K, device=dev))
        codes, self.scale, self.zero, self.sum = B.alloc_weight_buffers(N, K, dev)
        B.basq_quantize_weights(rotated, codes, self.scale, self.zero, self.sum)
        self.bias = torch.empty(N, device=dev)
        self.fp6 = B.alloc_fp6_buffer(N, K, dev)
        B.basq_prepare_weights(codes, self.scale, self.zero, None, None, self.sum, self.bias, self.fp6)
        self.streamed = torch.empty(B.basq_decode_bytes(N, K), dtype=torch.uint8, device=dev)
        B.basq_pack_decode(codes, self.streamed)
        self.workspace = None

    def __call__(self, x: torch.Tensor) -> torch.Tensor:
        M = x.shape[0]
        need = B.basq_workspace_bytes(M, self.K, self.N)
        if self.workspace is None or self.workspace.nbytes < need:
            self.workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
        y = torch.empty((M, self.N), dtype=torch.bfloat16, device=x.device)
        B.basq_linear_fused(x, self.K, None, None, CLIP, CLIP, self.streamed, self.scale, self.zero, self.sum, self.bias, y,
                            self.workspace, Wq6=self.fp6, w_layout=B.BASQ_W_DECODE16, N=self.N)
        return y


class Cache:
    """A pool of pages and which of them each sequence has; the books are kept on the host."""

    def __init__(self, pages: int, kv_heads: int, head_dim: int, page_size: int, most: int, device="cuda"):
        self.pages = B.alloc_kv_cache(pages, kv_heads, head_dim, page_size, device)
        self.page_size, self.most = page_size, most
        self.free = list(range(pages))
        self.of = []                                             # pages of each sequence
        self.lengths = []

    def new(self) -> int:
        self.of.append([])
        self.lengths.append(0)
        return len(self.of) - 1

    def grow(self, seq: int, tokens: int):
        """Room for more tokens: (their positions, their slots)."""
        return self.grow_all([seq], tokens)

    def grow_all(self, seqs, tokens: int):
        """Room for as many tokens of each sequence, one sequence behind the other; or, with an exception, of none."""
        if len(set(seqs)) != len(seqs):
            raise ValueError("a sequence is named twice")
        lengths = [self.lengths[s] + tokens for s in seqs]
        for s, n in zip(seqs, lengths):
            if n > self.most:
                raise ValueError(f"sequence {s} is longer than {self.most} tokens")
        missing = [-(-n // self.page_size) - len(self.of[s]) for s, n in zip(seqs, lengths)]
        if sum(missing) > len(self.free):
            raise MemoryError("no free page")
        positions, slots = [], []
        for s, n, pages in zip(seqs, lengths, missing):
            self.of[s] += [self.free.pop() for _ in range(pages)]
            at = range(self.lengths[s], n)
            positions += at
            slots += [self.of[s][t // self.page_size] * self.page_size + t % self.page_size for t in at]
            self.lengths[s] = n
        return positions, slots

    def table(self, seqs):
        """(page table, lengths) of some sequences, on the GPU."""
        width = -(-self.most // self.page_size)
        rows = [self.of[s] + [-1] * (width - len(self.of[s])) for s in seqs]
        dev = self.pages.device
        return (torch.tensor(rows, dtype=torch.int32, device=dev), torch.tensor([self.lengths[s] for s in seqs], dtype=torch.int32, device=dev))


class AttentionBlock:
    def __init__(self, heads: int, kv_heads: int, head_dim: int, cache: Cache, *, eps: float = 1e-5, base: float = 500000.0, seed: int = 0,
                 device="cuda"):
        hidden = heads * head_dim
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        weights = lambda n, k: (torch.randn((n, k), generator=g, device=device) / math.sqrt(k)).to(torch.bfloat16)  # noqa: E731
        self.heads, self.kv_heads, self.head_dim, self.cache, self.eps = heads, kv_heads, head_dim, cache, eps
        self.norm = (1 + 0.1 * torch.randn(hidden, generator=g, device=device)).to(torch.bfloat16)
        self.w_qkv, self.w_out = weights((heads + 2 * kv_heads) * head_dim, hidden), weights(hidden, hidden)
        self.qkv, self.out = Linear(self.w_qkv), Linear(self.w_out)
        self.cos_sin = torch.empty((cache.most, head_dim), device=device)
        B.basq_rope_table(self.cos_sin, base)
        self.workspace = None

    def __call__(self, x: torch.Tensor, residual: torch.Tensor, seqs, tokens: int):
        """The next `tokens` tokens of each sequence: x, residual bf16 [len(seqs) * tokens, hidden] -> (output, the residual stream
        with x added)."""
        dev = x.device
        heads, kv_heads, D = self.heads, self.kv_heads, self.head_dim
        positions, slots = (torch.tensor(n, dtype=torch.int32, device=dev) for n in self.cache.grow_all(seqs, tokens))
        table, lengths = self.cache.table(seqs)
        longest = max(self.cache.lengths[s] for s in seqs)

        h, stream = torch.empty_like(x), torch.empty_like(x)
        B.basq_add_rms_norm(x, residual, self.norm, self.eps, h, stream)
        qkv = self.qkv(h).view(x.shape[0], heads + 2 * kv_heads, D)
        q = qkv[:, :heads]                                       # turned in place
        B.basq_rope_append(q, qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:], positions, self.cos_sin, slots, self.cache.pages,
                           CLIP, CLIP, q)
        need = B.basq_paged_attention_workspace_bytes(len(seqs), tokens, heads, kv_heads, D, longest)
        if need and (self.workspace is None or self.workspace.nbytes < need):
            self.workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        attended = torch.empty_like(h)
        B.basq_paged_attention(q, self.cache.pages, table, lengths, longest, 1.0 / math.sqrt(D), attended.view(-1, heads, D),
                               self.workspace, q_len=tokens)
        return self.out(attended), stream


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--prompts", default="700,33,257", help="tokens of each prompt")
    ap.add_argument("--steps", type=int, default=32, help="tokens decoded behind each")
    ap.add_argument("--heads", type=int, default=32)
    ap.add_argument("--kv-heads", type=int, default=8)
    ap.add_argument("--page-size", type=int, default=64)
    a = ap.parse_args()
    D = 128
    prompts = [int(p) for p in a.prompts.split(",")]
    most = max(prompts) + a.steps
    cache = Cache(sum(-(-(p + a.steps) // a.page_size) for p in prompts), a.kv_heads, D, a.page_size, most)
    block = AttentionBlock(a.heads, a.kv_heads, D, cache)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    tokens = lambda n: torch.randn((n, a.heads * D), generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    seqs = [cache.new() for _ in prompts]
    for s, p in zip(seqs, prompts):
        y, stream = block(tokens(p), tokens(p), [s], p)
        print(f"prompt {s}: {p} tokens, output rms {y.float().pow(2).mean().sqrt():.3f}")
    torch.cuda.synchronize()
    began = time.perf_counter()
    for _ in range(a.steps):
        y, stream = block(tokens(len(seqs)), tokens(len(seqs)), seqs, 1)
    torch.cuda.synchronize()
    spent = time.perf_counter() - began
    print(f"{a.steps} decode steps of {len(seqs)} sequences: {1e6 * spent / a.steps:.0f} us each, output rms {y.float().pow(2).mean().sqrt():.3f}; "
          f"cache {cache.pages.nbytes / 1e6:.1f} MB, {cache.pages.nbytes / (len(cache.pages) * a.page_size):.0f} bytes a token")


if __name__ == "__main__":
    main()
