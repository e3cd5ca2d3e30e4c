"""Calls on an 8-bit cache one after the other, none waited for: each starts while the one
before is still running, and has to find what that one wrote."""
from __future__ import annotations

import pytest
import torch

from .test_gpu_paged_codes import rng

pytestmark = pytest.mark.gpu


class Steps:
    """Dense norm and rotation, then rows of its queries and keys quantised, read back, attended to, twice over."""

    def __init__(self, B, n, Hq, Hkv, D, page, r, dtype, codes):
        import paper_2602_01762_gb300 as p
        dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        g = rng(7)
        cols = -(-2 * n // page) + 1
        self.B, self.n, self.h = B, n, p.PagedAttention(n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, dtype=dtype, page_size=page, max_batch=B, max_pages=cols)
        table = torch.randperm(B * cols, generator=g).to(torch.int32).view(B, cols).cuda()
        pages = [torch.zeros(B * cols, Hkv, page, D, dtype=torch.uint8, device="cuda").view(codes) for _ in range(2)]
        self.scales = [torch.zeros(B * cols, Hkv, page // r, device="cuda") for _ in range(2)]
        self.raw = [x.view(torch.uint8) for x in pages]
        self.kv_len = torch.zeros(B, dtype=torch.int32, device="cuda")
        self.cache = self.h.cache(*pages, table, self.kv_len, k_scales=self.scales[0], v_scales=self.scales[1])
        self.x = [torch.zeros(B, n, H, D, dtype=dt, device="cuda") for H in (Hq, Hkv, Hkv)]
        self.mid = [torch.zeros_like(t) for t in self.x[:2]]
        self.q_out = torch.zeros_like(self.x[0])
        self.rows = [torch.zeros(B, 2 * n, Hkv, D, dtype=dt, device="cuda") for _ in range(2)]
        self.out, self.out2 = (torch.zeros(B, Hq, D, dtype=dt, device="cuda") for _ in range(2))
        self.count = torch.zeros(B, dtype=torch.int32, device="cuda")
        self.rope, self.pos = p.rope_table(2 * n, D), torch.zeros(B, dtype=torch.int32, device="cuda")
        self.gain = torch.ones(D, dtype=dt, device="cuda") * 1.25

    def all(self):
        return [*self.raw, *self.scales, *self.mid, self.q_out, *self.rows, self.out, self.out2, self.kv_len]

    def clear(self):
        for t in self.all():
            t.zero_()

    def run(self, wait=lambda: None):
        h, c = self.h, self.cache
        for i in range(2):
            h.qk_norm_rope(self.x[0], self.x[1], *self.mid, self.rope, self.pos, g_q=self.gain, g_k=self.gain)
            wait()
            h.append(c, self.mid[0], self.mid[1], self.x[2], self.q_out if i else self.mid[0], self.rope, n_new=self.count)   # first over its own input
            wait()
            h.attend(c, self.mid[0][:, 0].contiguous(), self.out if i else self.out2, added=self.n)
            wait()
            self.kv_len += self.count
            wait()
            h.read(c, *self.rows, n_rows=self.kv_len)
            wait()
            h.attend(c, self.q_out[:, 0].contiguous(), self.out if i else self.out2, added=0, window=100, sinks=5)
            wait()


@pytest.mark.parametrize("codes", [torch.float8_e4m3fn, torch.int8])
@pytest.mark.parametrize("B,n,Hq,Hkv,D,page,r,dtype", [(8, 700, 32, 8, 128, 16, 16, "bf16"), (8, 900, 2, 1, 64, 16, 1, "bf16"), (4, 1500, 6, 3, 128, 16, 16, "f32"),
                                                       (16, 5, 8, 2, 64, 16, 4, "f32"), (3, 1, 8, 8, 128, 64, 64, "bf16")])
def test_calls_that_follow_each_other(codes, B, n, Hq, Hkv, D, page, r, dtype):
    """Waited for one by one, on a stream, and as a graph replayed: the same bits."""
    s = Steps(B, n, Hq, Hkv, D, page, r, dtype, codes)
    g = rng(B)
    inputs = [([torch.randn(t.shape, generator=g).to(t.dtype).cuda() * (1 + i) for t in s.x], torch.randint(max(0, n - 40), n + 1, (B,), generator=g).to(torch.int32).cuda())
              for i in range(3)]

    def go(run, given):
        s.clear()
        for a, b in zip(s.x, given[0]):
            a.copy_(b)
        s.count.copy_(given[1])
        run()
        return [t.clone() for t in s.all()]

    want = [go(lambda: s.run(torch.cuda.synchronize), x) for x in inputs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        go(s.run, inputs[0])
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
    for turn in range(6):
        for i, x in enumerate(inputs):
            for run in (s.run, graph.replay):
                got = go(run, x)
                assert all(torch.equal(a, b) for a, b in zip(got, want[i])), (turn, i, run, [torch.equal(a, b) for a, b in zip(got, want[i])])
    assert s.h.status() == 0
    s.h.close()
