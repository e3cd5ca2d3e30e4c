"""What an append to a cache held in 8 bits stored, against the formula: every code
between the formats' nearest to the ends of the interval in which the fp32 key lies,
scales likewise, earlier rows of a block that grew, and all other codes and scales
untouched."""
import torch

from . import codes_ref as ref
from .paged_ref import norm_rope


def interleaved_sizes(g, B, n, Hkv, r):
    """Factors of rows [B, n, Hkv, 1], powers of two: neighbouring rows, the halves of a block and neighbouring blocks
    differ by up to 2^10, so that a maximum of other rows or of another block makes another scale."""
    i = torch.arange(n)
    half, block = i * 2 // max(r, 1) % 2, i // max(r, 1) % 3
    e = torch.randint(-2, 3, (B, n, Hkv), generator=g) + (5 * half - 4 * block)[None, :, None]
    return torch.exp2(e.double())[..., None]


def keys(x, gain, rope, pos, eps):
    """Normed and rotated rows x [n, H, D] of one sequence in 64 bits, on the host, and the fp32 bound of each."""
    y, tol = norm_rope(x, gain, rope, pos, eps)
    return y.cpu(), tol.cpu()


def scales_of(top, fmt):
    return torch.tensor([ref.scale_of(float(t), fmt) for t in top.flatten()], dtype=torch.float64).view(top.shape)


def check_stored(before, after, table, lens, rows, counts, fmt, what):
    """before, after: (codes, scales) in 64 bits on the host; rows[b]: (values [counts[b], Hkv, D], bound of each)."""
    codes0, scales0 = before
    codes, scales = after
    n_pages, Hkv, page, D = codes.shape
    blocks = scales.shape[2]
    r = page // blocks
    own_rows = torch.zeros(n_pages, page, dtype=torch.bool)      # rows that may have changed
    own_blocks = torch.zeros(n_pages, blocks, dtype=torch.bool)
    for b, (n, c) in enumerate(zip(lens, counts)):
        if c == 0:
            continue
        first = n // r * r
        slot = torch.arange(first, -(-(n + c) // r) * r)
        at = table[b].long()[slot // page]
        new = (slot >= n) & (slot < n + c)
        x, t = (torch.zeros(len(slot), Hkv, D, dtype=torch.float64) for _ in range(2))
        x[new], t[new] = (y.double() for y in rows[b])
        top = x.abs().view(-1, r, Hkv, D).amax((1, 3))
        off = t.view(-1, r, Hkv, D).amax((1, 3))
        lo, hi = scales_of((top - off).clamp(min=0), fmt), scales_of(top + off, fmt)
        got = scales[at[::r], :, (slot[::r] % page) // r]         # [blocks, Hkv]
        was = torch.zeros_like(got)
        if first < n:
            was[0] = scales0[at[0], :, int(slot[0]) % page // r]
        ok = (got == torch.maximum(was, lo)) | (got == torch.maximum(was, hi))
        assert ok.all(), f"{what}: sequence {b}, {int((~ok).sum())} scales of {ok.numel()}"
        s = got.repeat_interleave(r, 0)[..., None]
        held = codes[at, :, slot % page]
        per = torch.where(s > 0, s, 1.0)
        most = ref.MOST[fmt]
        low, high = (ref.nearest(((x + d) / per).clamp(-most, most), fmt) for d in (-t, t))
        good = (held >= low) & (held <= high)
        bad = ~good[new]
        assert not bad.any(), f"{what}: sequence {b}, {int(bad.sum())} codes of {bad.numel()} outside their interval"
        if first < n:                    # earlier rows, rounded again where the scale grew
            k = n - first
            want = codes0[at[:k], :, slot[:k] % page]
            ratio = torch.where(got[0] > was[0], was[0] / torch.where(got[0] > 0, got[0], 1.0), 1.0)[None, :, None]
            assert torch.equal(held[:k], ref.nearest(want * ratio, fmt)), f"{what}: earlier rows of sequence {b}"
        used = slot < n + c
        own_rows[at[used], slot[used] % page] = True
        own_blocks[at, slot % page // r] = True
    same = (codes == codes0) | own_rows[:, None, :, None]
    assert same.all(), f"{what}: codes of other rows"
    same = (scales == scales0) | own_blocks[:, None]
    assert same.all(), f"{what}: scales of other blocks"
