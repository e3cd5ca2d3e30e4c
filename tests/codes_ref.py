"""Plain 64-bit forms of the paged cache held in 8 bits and of windowed attention
(loops over sequences, heads and blocks, written from the formulas).

A block's scale is the smallest power of two s >= 2^-126 with max |x| <= M s over its
new rows, or what it was if that is larger; a code is x / s to the nearest of the
format, ties to even.
"""
import math

import torch

from .paged_ref import U

MOST = {"e4m3": 448.0, "int8": 127.0}
TYPE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def nearest(y, fmt):
    """The format's nearest value to y (64 bits, within its range), ties to even."""
    if fmt == "int8":
        return torch.round(y)
    # four significant bits; steps of 2^-9 below 2^-6
    _, e = torch.frexp(y)
    step = torch.exp2((e - 4).clamp(min=-9).double())
    return torch.where(y == 0, y, torch.round(y / step) * step)


def scale_of(top, fmt):
    if top == 0:
        return 0.0
    e = max(math.ceil(math.log2(top / MOST[fmt])) + 1, -126)
    while e > -126 and top <= math.ldexp(MOST[fmt], e - 1):
        e -= 1
    return math.ldexp(1.0, e)


def codes_of(pages):
    """Codes as values, on the host, in 64 bits."""
    return pages.cpu().to(torch.float32).double()


def values(pages, scales):
    """[n_pages, Hkv, page, D] in 64 bits, on the host."""
    r = pages.shape[2] // scales.shape[2]
    return codes_of(pages) * scales.cpu().double().repeat_interleave(r, 2)[..., None]


def store(codes, scales, table, lens, x, counts, fmt):
    """codes [n_pages, Hkv, page, D] and scales (64 bits, host, changed in place) after
    rows x[b, :counts[b]] (64 bits) went behind the lens[b] rows of each sequence."""
    page, r = codes.shape[2], codes.shape[2] // scales.shape[2]
    for b, (n, new) in enumerate(zip(lens, counts)):
        for first in range(n // r * r, n + new, r):
            p, row = int(table[b, first // page]), first % page
            lo, hi = max(first, n), min(first + r, n + new)
            if lo >= hi:
                continue
            for h in range(codes.shape[1]):
                rows = x[b, lo - n:hi - n, h]
                s = scale_of(float(rows.abs().max()), fmt)
                if first < n:
                    was = float(scales[p, h, row // r])
                    if s > was:
                        old = codes[p, h, row:row + n - first]
                        codes[p, h, row:row + n - first] = nearest(old * (was / s), fmt)
                    else:
                        s = was
                scales[p, h, row // r] = s
                codes[p, h, row + lo - first:row + hi - first] = nearest(rows / s, fmt) if s else 0.0


def seen(n, window, sinks):
    j = torch.arange(n)
    return j if window is None else j[(j < sinks) | (j >= n - window)]


def attend(q, k_values, v_values, table, lens, scale, window=None, sinks=0, v_scales=None):
    """out, lse, weights (list of [Hkv, rows]) and the bounds of out, lse and weights, as
    paged_ref.attend's, of pages of values (64 bits, host).  What 8-bit caches have
    besides is within them: weights of two fp16 parts (bf16) add 2^-22 of themselves,
    of 2^-16, of three 2^-24, of 2^-20.  With ``v_scales`` (those of v_values' blocks) the bound of out has their
    floor too: fp16 ends at steps of 2^-24, the head's largest weight p s is at least
    2^12 of them over its base (2^13, and one bit for the base's whole number), so two
    parts leave 2^-25 / 2^12 of it for each row's code, 2^-36 with room."""
    q, table = q.cpu(), table.cpu()
    B, Hq, D = q.shape
    Hkv, page = k_values.shape[1:3]
    G, bf16 = Hq // Hkv, q.dtype == torch.bfloat16
    out, lse = torch.zeros(B, Hq, D, dtype=torch.float64), torch.full((B, Hq), -float("inf"), dtype=torch.float64)
    tol_out, tol_lse, weights, tol_w = torch.zeros_like(out), torch.ones_like(lse), [], []
    for b, n in enumerate(lens):
        j = seen(n, window, sinks)
        w = torch.zeros(Hkv, len(j), dtype=torch.float64)
        tw = torch.zeros_like(w)
        if len(j):
            at = table[b].long()[j // page]
            k, v = k_values[at, :, j % page].double(), v_values[at, :, j % page].double()
        for h in range(Hkv if len(j) else 0):
            sl = slice(h * G, (h + 1) * G)
            qh = q[b, sl].double()
            z = qh @ k[:, h].T * scale
            m = z.amax(1, keepdim=True)
            e = torch.exp(z - m)
            s = e.sum(1, keepdim=True)
            p = e / s
            ez = 2 * D * U * scale * (qh.abs() @ k[:, h].abs().T).amax(1) + 8 * U * z.abs().amax(1)
            rel = 2.0 ** -20 + 4 * ez + (2.0 ** -16 if bf16 else 0.0)
            out[b, sl] = p @ v[:, h]
            tol_out[b, sl] = rel[:, None] * (p @ v[:, h].abs()) + (2.0 ** -8 * out[b, sl].abs() if bf16 else 0.0)
            if v_scales is not None:
                vs = v_scales[at, h, j % page * v_scales.shape[2] // page].cpu().double()
                code = torch.where(vs[:, None] > 0, v[:, h] / vs[:, None], 0.0)
                tol_out[b, sl] += 2.0 ** -36 * (p * vs).amax(1, keepdim=True) * code.abs().sum(0)
            lse[b, sl] = (m + torch.log(s))[:, 0]
            tol_lse[b, sl] = 2 * ez + 2.0 ** -20 + 4 * U * lse[b, sl].abs()
            w[h] = p.sum(0)
            tw[h] = ((2.0 ** -19 + 4 * ez)[:, None] * p).sum(0)
        weights.append(w)
        tol_w.append(tw)
    return out, lse, weights, tol_out, tol_lse, tol_w
