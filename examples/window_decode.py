"""Decode with a sliding window over a cache held in 8 bits: one attention layer of a
Llama-3-8B-shaped model serves a batch of sequences of any length from a pool that
holds a window of their rows and a few first ones.

    python examples/window_decode.py [--batch 16] [--prompt 1000] [--tokens 2048]
                                     [--window 1024] [--sinks 4] [--cache e4m3]

Per token: the fused QKV projection (torch), then append (norm of queries and keys,
rotation, rows quantised into the cache), attention over the window and the sinks,
and the output projection (torch); the whole step is one CUDA graph.  Attention
follows no block-table entry of a page without a row that it sees, so each sequence
gets its pages back in turn: the table's columns run on, the pages they name repeat.
Weights and inputs are random.
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
    """One attention layer with its cache, a ring of pages for each sequence."""

    def __init__(self, batch, window, sinks, max_positions, *, cache="e4m3", hidden=4096, n_q_heads=32, n_kv_heads=8, head_dim=128, page=16,
                 seed=0):
        dev, bf16, i32 = "cuda", torch.bfloat16, torch.int32
        gen = torch.Generator(device=dev).manual_seed(seed)
        self.B, self.Hq, self.Hkv, self.D, self.page, self.window, self.sinks = batch, n_q_heads, n_kv_heads, head_dim, page, window, sinks
        heads = n_q_heads + 2 * n_kv_heads
        self.w_qkv = torch.randn(heads * head_dim, hidden, generator=gen, device=dev, dtype=bf16) * hidden ** -0.5
        self.w_o = torch.randn(hidden, n_q_heads * head_dim, generator=gen, device=dev, dtype=bf16) * hidden ** -0.5
        self.g_q, self.g_k = (torch.ones(head_dim, device=dev, dtype=bf16) * 1.5 for _ in range(2))
        # pages of the sinks, then a ring that holds a window wherever it begins
        first, ring, columns = -(-sinks // page), -(-window // page) + 1, -(-max_positions // page)
        self.held = first + ring
        owned = torch.randperm(batch * self.held, generator=gen, device=dev).to(i32).view(batch, self.held)
        turn = torch.arange(columns, device=dev)
        table = owned[:, torch.where(turn < self.held, turn, first + (turn - first) % ring)].contiguous()
        codes = torch.float8_e4m3fn if cache == "e4m3" else torch.int8
        shape = (batch * self.held, n_kv_heads, page, head_dim)
        self.k_pages, self.v_pages = (torch.zeros(shape, device=dev, dtype=torch.int8).view(codes) for _ in range(2))
        self.k_scales, self.v_scales = (torch.zeros(*shape[:2], 1, device=dev) for _ in range(2))
        self.kv_len = torch.zeros(batch, dtype=i32, device=dev)
        self.rope = rope_table(max_positions, head_dim, 500000.0)
        self.att = PagedAttention(n_q_heads=n_q_heads, n_kv_heads=n_kv_heads, head_dim=head_dim, page_size=page, max_batch=batch,
                                  max_pages=columns)
        self.cache = self.att.cache(self.k_pages, self.v_pages, table, self.kv_len, k_scales=self.k_scales, v_scales=self.v_scales)
        self.x = torch.zeros(batch, 1, hidden, device=dev, dtype=bf16)
        self.q_out = torch.empty(batch, 1, n_q_heads, head_dim, device=dev, dtype=bf16)
        self.out = torch.empty(batch, n_q_heads, head_dim, device=dev, dtype=bf16)
        self.y = torch.empty(batch, hidden, device=dev, dtype=bf16)
        self.graph = None

    def rows(self, x):
        qkv = torch.matmul(x, self.w_qkv.T)
        q, k, v = qkv.split([self.Hq * self.D, self.Hkv * self.D, self.Hkv * self.D], -1)
        return (t.unflatten(-1, (-1, self.D)) for t in (q, k, v))

    def prompt(self, x, lengths):
        """Stores the prompts x [B, n, hidden], lengths[b] rows each; n rows fit the pages of a sequence."""
        if x.shape[1] > self.held * self.page:
            raise ValueError(f"a prompt of {x.shape[1]} rows needs a larger window than {self.window}")
        q, k, v = self.rows(x)
        self.att.append(self.cache, q, k, v, torch.empty_like(q, memory_format=torch.contiguous_format), self.rope, g_q=self.g_q, g_k=self.g_k,
                        n_new=lengths)
        self.kv_len += lengths

    def _step(self):
        q, k, v = self.rows(self.x)
        self.att.append(self.cache, q, k, v, self.q_out, self.rope, g_q=self.g_q, g_k=self.g_k)
        self.att.attend(self.cache, self.q_out.view(self.B, self.Hq, self.D), self.out, window=self.window, sinks=self.sinks)
        torch.matmul(self.out.view(self.B, -1), self.w_o.T, out=self.y)
        self.kv_len += 1

    def step(self):
        """One token of every sequence: x in, y out."""
        if self.graph is not None:
            self.graph.replay()
            return self.y
        self._step()                                     # the first token; the next ones replay what is captured here
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=stream):
            self._step()
        self.graph = graph
        return self.y


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("batch", 16), ("prompt", 1000), ("tokens", 2048), ("window", 1024), ("sinks", 4), ("hidden", 4096)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--cache", choices=("e4m3", "int8"), default="e4m3")
    a = ap.parse_args(argv)
    layer = Layer(a.batch, a.window, a.sinks, a.prompt + a.tokens + 1, cache=a.cache, hidden=a.hidden)
    gen = torch.Generator(device="cuda").manual_seed(1)
    lengths = torch.randint(max(1, a.prompt // 2), a.prompt + 1, (a.batch,), generator=gen, device="cuda", dtype=torch.int32)
    layer.prompt(torch.randn(a.batch, a.prompt, a.hidden, generator=gen, device="cuda", dtype=torch.bfloat16), lengths)
    torch.cuda.synchronize()
    begin = time.perf_counter()
    for _ in range(a.tokens):
        layer.x.copy_(torch.randn(a.batch, 1, a.hidden, generator=gen, device="cuda", dtype=torch.bfloat16))
        layer.step()
    flags = layer.att.status()
    seconds = time.perf_counter() - begin
    if flags:
        raise RuntimeError(f"device error word {flags:#x}")
    print(f"{a.tokens} tokens of {a.batch} sequences in {seconds * 1e3:.1f} ms ({seconds / a.tokens * 1e6:.1f} us a step, capture included), "
          f"sequences up to {int(layer.kv_len.max())} rows on {layer.held} pages of {layer.page} each")
    return layer


if __name__ == "__main__":
    main()
