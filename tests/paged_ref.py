"""Plain 64-bit forms of the paged-cache operators, written from their formulas
(numpy-style loops over sequences and heads), and the bounds within which the
kernels' arithmetic has to stay.

u = 2^-24 is half an fp32 ulp.  Bounds are first-order, with room of two or more:

* scores: a D-term fp32 sum, D u scale sum |q k|, and the base-2 scaling, 4 u |z|:
  ``ez`` below, an absolute error of z, so a relative one of exp(z) (twice: once in
  the probability, once in the sum it is divided by).
* probabilities: exp2 and the rescaling of running sums, 2^-20 together; as a pair
  of bf16 values 2^-17 more.
* a bf16 result adds half an ulp, 2^-9 of itself.
"""
import numpy as np
import torch

U = 2.0 ** -24


def gather(pages, table_row, n):
    """Rows 0..n of one sequence, [Hkv, n, ...], from [n_pages, Hkv, page, ...] (float64)."""
    page = pages.shape[2]
    used = table_row[: -(-n // page)].long()
    x = pages[used].double() if n else pages[:0].double()
    return x.transpose(0, 1).reshape(pages.shape[1], -1, *pages.shape[3:])[:, :n]


def attend(q, k_pages, v_pages, table, lens, scale):
    """out, lse, per-row weights (list of [Hkv, n]) and the bounds of each."""
    B, Hq, D = q.shape
    Hkv = k_pages.shape[1]
    G = Hq // Hkv
    bf16 = q.dtype == torch.bfloat16
    out = torch.zeros(B, Hq, D, dtype=torch.float64, device=q.device)
    lse = torch.full((B, Hq), -float("inf"), dtype=torch.float64, device=q.device)
    tol_out, tol_lse = torch.zeros_like(out), torch.ones_like(lse)
    weights, tol_w = [], []
    for b, n in enumerate(lens):
        k, v = gather(k_pages, table[b], n), gather(v_pages, table[b], n)
        w = torch.zeros(Hkv, n, dtype=torch.float64, device=q.device)
        tw = torch.zeros_like(w)
        for h in range(Hkv if n else 0):
            qh = q[b, h * G:(h + 1) * G].double()
            z = qh @ k[h].T * scale
            m = z.amax(1, keepdim=True)
            e = torch.exp(z - m)
            s = e.sum(1, keepdim=True)
            p = e / s
            ez = 2 * D * U * scale * (qh.abs() @ k[h].abs().T).amax(1) + 8 * U * z.abs().amax(1)   # [G]
            rel = 2.0 ** -20 + 4 * ez + (2.0 ** -16 if bf16 else 0.0)
            sl = slice(h * G, (h + 1) * G)
            out[b, sl] = p @ v[h]
            tol_out[b, sl] = rel[:, None] * (p @ v[h].abs()) + (2.0 ** -8 * out[b, sl].abs() if bf16 else 0.0)
            lse[b, sl] = (m + torch.log(s))[:, 0]
            tol_lse[b, sl] = 2 * ez + 2.0 ** -20 + 4 * U * lse[b, sl].abs()
            w[h] = p.sum(0)
            tw[h] = ((2.0 ** -19 + 4 * ez)[:, None] * p).sum(0)
        weights.append(w)
        tol_w.append(tw)
    return out, lse, weights, tol_out, tol_lse, tol_w


def norm_rope(x, g, rope, pos, eps):
    """Rows [n, H, D] at positions pos..; result and its fp32 bound."""
    n, _, D = x.shape
    x = x.double()
    if g is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * g.double()
    t = rope[pos:pos + n].double()
    c, s = t[:, 0, None], t[:, 1, None]
    a, b = x[..., :D // 2], x[..., D // 2:]
    size = torch.cat([a.abs() * c.abs() + b.abs() * s.abs(), b.abs() * c.abs() + a.abs() * s.abs()], -1)
    # the mean of D squares (D u / 2 at worst), the root, four products and a sum
    return torch.cat([a * c - b * s, b * c + a * s], -1), (D / 2 + 16) * U * size


def norm_rope_grad(x, g, dy, rope, pos, eps):
    """dx, dg and their fp32 bounds for rows [n, H, D]."""
    n, _, D = x.shape
    x, dy = x.double(), dy.double()
    t = rope[pos:pos + n].double()
    c, s = t[:, 0, None], t[:, 1, None]
    a, b = dy[..., :D // 2], dy[..., D // 2:]
    dz = torch.cat([a * c + b * s, b * c - a * s], -1)
    size = torch.cat([a.abs() * c.abs() + b.abs() * s.abs(), b.abs() * c.abs() + a.abs() * s.abs()], -1)
    if g is None:
        return dz, None, 8 * U * size, None
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    nrm = x * r
    dn, dn_size = dz * g.double(), size * g.double().abs()
    dx = r * (dn - nrm * (dn * nrm).mean(-1, keepdim=True))
    dx_size = r * (dn_size + nrm.abs() * (dn_size * nrm.abs()).mean(-1, keepdim=True))
    # chains of at most a few hundred additions per lane, warp and CTA
    return dx, (dz * nrm).sum((0, 1)), (2 * D + 32) * U * dx_size, (512 + D) * U * (size * nrm.abs()).sum((0, 1))


def kept_rows(w, length, budget, sinks, recent):
    """Slots that eviction keeps for one (sequence, KV head); w numpy [length]."""
    if length <= budget:
        return np.arange(length)
    mid = np.arange(sinks, length - recent)
    v = w[sinks:length - recent].astype(np.float64)
    best = sorted(mid.tolist(), key=lambda i: (np.isnan(v[i - sinks]), -v[i - sinks] if v[i - sinks] == v[i - sinks] else 0.0, i))
    return np.sort(np.concatenate([np.arange(sinks), np.array(best[:budget - sinks - recent], dtype=np.int64),
                                   np.arange(length - recent, length)]).astype(np.int64))


def within(got, want, tol, what=""):
    got, want = got.double(), want.double()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    bad = ~same & ~((got - want).abs() <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} beyond the bound, worst " \
                          f"{float(((got - want).abs() / tol)[bad].max()) if bad.any() else 0:.3g} of it"
