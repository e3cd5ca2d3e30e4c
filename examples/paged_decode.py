"""Decode with a bounded cache: one attention layer of a Llama-3-8B-shaped model
serves a batch of sequences from a paged key-value cache that eviction by
accumulated attention weight keeps within a budget.

    python examples/paged_decode.py [--batch 16] [--prompt 4000] [--tokens 512]
                                    [--budget 4096] [--slack 256]

Per token: the fused QKV projection (torch), then append (norm of queries and
keys, rotation, store), attention over the cache with the rows' weights, and the
output projection (torch); the whole step is one CUDA graph.  Whenever the cache
has grown `slack` rows past the budget, the rows to keep move to the other half of
the pool and the next graph reads them there.  Weights and inputs are random.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2602_01762_gb300 import PagedAttention, rope_table  # noqa: E402


class Layer:
    """One attention layer with its cache: two block tables over one pool."""

    def __init__(self, batch, budget, slack, max_positions, *, hidden=4096, n_q_heads=32, n_kv_heads=8, head_dim=128, page=16,
                 sinks=4, recent=512, seed=0):
        dev, bf16, i32 = "cuda", torch.bfloat16, torch.int32
        gen = torch.Generator(device=dev).manual_seed(seed)
        self.B, self.Hq, self.Hkv, self.D, self.budget, self.sinks, self.recent = batch, n_q_heads, n_kv_heads, head_dim, budget, sinks, min(recent, budget - sinks)
        pages = -(-(budget + slack) // page)
        n = 2 * batch * pages
        heads = n_q_heads + 2 * n_kv_heads
        self.w_qkv = torch.randn(heads * head_dim, hidden, generator=gen, device=dev, dtype=bf16) * hidden ** -0.5
        self.w_o = torch.randn(hidden, n_q_heads * head_dim, generator=gen, device=dev, dtype=bf16) * hidden ** -0.5
        self.g_q, self.g_k = (torch.ones(head_dim, device=dev, dtype=bf16) * 1.5 for _ in range(2))
        self.k_pages, self.v_pages = (torch.zeros(n, n_kv_heads, page, head_dim, device=dev, dtype=bf16) for _ in range(2))
        self.weights = torch.zeros(n, n_kv_heads, page, device=dev)
        tables = torch.randperm(n, generator=gen, device=dev).to(i32).view(2, batch, pages).contiguous()
        self.kv_len, self.pos = torch.zeros(batch, dtype=i32, device=dev), torch.zeros(batch, dtype=i32, device=dev)
        self.rope = rope_table(max_positions, head_dim, 500000.0)
        self.kept = torch.empty(batch, n_kv_heads, budget, dtype=i32, device=dev)
        self.att = PagedAttention(n_q_heads=n_q_heads, n_kv_heads=n_kv_heads, head_dim=head_dim, page_size=page, max_batch=batch,
                                  max_pages=pages, track_weights=True)
        self.caches = [self.att.cache(self.k_pages, self.v_pages, t, self.kv_len, weights=self.weights) for t in tables]
        self.at = 0                                      # the half of the pool in use
        self.x = torch.zeros(batch, 1, hidden, device=dev, dtype=bf16)
        self.q_out = torch.empty(batch, 1, n_q_heads, head_dim, device=dev, dtype=bf16)
        self.out = torch.empty(batch, n_q_heads, head_dim, device=dev, dtype=bf16)
        self.y = torch.empty(batch, hidden, device=dev, dtype=bf16)
        self.graphs = {}

    def rows(self, x):
        qkv = torch.matmul(x, self.w_qkv.T)
        q, k, v = qkv.split([self.Hq * self.D, self.Hkv * self.D, self.Hkv * self.D], -1)
        return (t.unflatten(-1, (-1, self.D)) for t in (q, k, v))

    def prompt(self, x, lengths):
        """Stores the prompts x [B, n, hidden], lengths[b] rows each."""
        q, k, v = self.rows(x)
        self.att.append(self.caches[self.at], q, k, v, torch.empty_like(q, memory_format=torch.contiguous_format), self.rope, g_q=self.g_q,
                        g_k=self.g_k, pos=self.pos, n_new=lengths)
        self.kv_len += lengths
        self.pos += lengths

    def _step(self):
        q, k, v = self.rows(self.x)
        self.att.append(self.caches[self.at], q, k, v, self.q_out, self.rope, g_q=self.g_q, g_k=self.g_k, pos=self.pos)
        self.att.attend(self.caches[self.at], self.q_out.view(self.B, self.Hq, self.D), self.out)
        torch.matmul(self.out.view(self.B, -1), self.w_o.T, out=self.y)
        self.kv_len += 1
        self.pos += 1

    def step(self):
        """One token of every sequence: x in, y out."""
        if self.at in self.graphs:
            self.graphs[self.at].replay()
            return self.y
        self._step()                                     # a half's first token; the next ones replay what is captured here
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=stream):
            self._step()
        self.graphs[self.at] = graph
        return self.y

    def evict(self):
        """Keeps the budget's rows, in the other half of the pool."""
        self.att.evict(self.caches[self.at], self.caches[1 - self.at], self.kept, sinks=self.sinks, recent=self.recent)
        self.at = 1 - self.at


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("batch", 16), ("prompt", 4000), ("tokens", 512), ("budget", 4096), ("slack", 256), ("hidden", 4096)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args(argv)
    if a.prompt > a.budget + a.slack:
        ap.error("the prompt has to fit budget + slack")
    layer = Layer(a.batch, a.budget, a.slack, a.prompt + a.tokens + 1, hidden=a.hidden)
    gen = torch.Generator(device="cuda").manual_seed(1)
    lengths = torch.randint(max(1, a.prompt // 2), a.prompt + 1, (a.batch,), generator=gen, device="cuda", dtype=torch.int32)
    lengths[0] = a.prompt
    layer.prompt(torch.randn(a.batch, a.prompt, a.hidden, generator=gen, device="cuda", dtype=torch.bfloat16), lengths)
    longest, evictions = a.prompt, 0                     # the host knows the lengths without asking the device
    torch.cuda.synchronize()
    begin = time.perf_counter()
    for _ in range(a.tokens):
        if longest == a.budget + a.slack:
            layer.evict()
            longest, evictions = a.budget, evictions + 1
        layer.x.copy_(torch.randn(a.batch, 1, a.hidden, generator=gen, device="cuda", dtype=torch.bfloat16))
        layer.step()
        longest += 1
    flags = layer.att.status()
    seconds = time.perf_counter() - begin
    if flags:
        raise RuntimeError(f"device error word {flags:#x}")
    kept = int(layer.kv_len.max())
    print(f"{a.tokens} tokens of {a.batch} sequences in {seconds * 1e3:.1f} ms ({seconds / a.tokens * 1e6:.1f} us a step, capture included), "
          f"{evictions} evictions, longest cache {kept} rows, positions up to {int(layer.pos.max())}")
    return layer, evictions


if __name__ == "__main__":
    main()
