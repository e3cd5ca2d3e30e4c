"""Performance cases of the paged key-value cache held in 8 bits and of windowed
attention: keys and values quantised as they are written (with the per-head norm
and rotation before), rows read back, attention of one new token over such a cache,
and attention of one new token to a sliding window and a few first rows (sinks)
over a cache of either kind.

An 8-bit cache holds codes, e4m3 or int8, and one fp32 scale for each block of
``scale_rows`` rows of a page and KV head; a row's value is its code times its
block's scale.  What writes rows gives their block the smallest power of two that
keeps its largest value within the codes' range, never less than what the block's
earlier rows have; if it grows, those rows' codes are rounded anew.

``run`` computes a case either in plain torch operations in 32 bits (``own`` is
false) or through this package's operators (``own`` is true); ``exact`` gives the
same results in 64 bits.
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-5
THETA = 500000.0

# heads: (query heads, key-value heads, head dimension) of the drafter shapes
TINY = dict(q_heads=4, kv_heads=4, head_dim=64)
MID = dict(q_heads=8, kv_heads=2, head_dim=128)
L3_8B = dict(q_heads=32, kv_heads=8, head_dim=128)
L2_7B = dict(q_heads=32, kv_heads=32, head_dim=128)
L3_70B = dict(q_heads=64, kv_heads=8, head_dim=128)
# two grouped layouts beside them: an odd group, and more heads per key than a tile of eight
ODD_GROUP = dict(q_heads=24, kv_heads=8, head_dim=64)
WIDE_GROUP = dict(q_heads=16, kv_heads=1, head_dim=128)


def listed():
    return [
        # one user's chat turn in its first paragraphs: the call is all latency
        dict(name="attend-b1-short", op="attend", **L3_8B, dtype="bf16", cache="e4m3", scale_rows=16, batch=1, min_len=517, max_len=517, page=16),
        # fp32 queries of the mid shape, pages that are no multiple of a tile, three scales a page
        dict(name="attend-b3-f32", op="attend", **MID, dtype="f32", cache="int8", scale_rows=8, batch=3, min_len=411, max_len=2999, page=24),
        # a mixed batch: one sequence has just begun, others are thousands of tokens in; a scale for every row
        dict(name="attend-b16-ragged", op="attend", **L3_8B, dtype="bf16", cache="int8", scale_rows=1, batch=16, min_len=1, max_len=8192, page=16),
        # a full server: many long sequences over eight query heads per key head
        dict(name="attend-b64-long", op="attend", **L3_70B, dtype="bf16", cache="e4m3", scale_rows=32, batch=64, min_len=6001, max_len=16384, page=32),
        # one document of 131072 tokens: one sequence has to fill the whole GPU
        dict(name="attend-b1-128k", op="attend", **L3_8B, dtype="bf16", cache="e4m3", scale_rows=16, batch=1, min_len=131071, max_len=131071, page=16),
        # the decode step's rows of a batch, in blocks that hold earlier rows, and those blocks read back
        dict(name="append-b16-token", op="append", **L3_8B, dtype="bf16", cache="e4m3", scale_rows=16, batch=16, min_new=1, max_new=1, max_len=2047, page=16, gains=True),
        # ragged prompts of up to 2048 tokens stored behind what the cache already holds, and read back for the
        # prompt's own attention
        dict(name="append-b8-prompt", op="append", **L3_8B, dtype="bf16", cache="int8", scale_rows=16, batch=8, min_new=1021, max_new=2048, max_len=777, page=16, gains=True),
        # a short fp32 row range read back, from the middle of a page on
        dict(name="read-b1-f32", op="read", **MID, dtype="f32", cache="int8", scale_rows=24, batch=1, min_rows=67, max_rows=67, max_len=411, page=24),
        # prefixes of up to 16384 rows read back for the attention of a prompt's next part
        dict(name="read-b4-prefix", op="read", **L3_8B, dtype="bf16", cache="e4m3", scale_rows=64, batch=4, min_rows=9001, max_rows=16384, max_len=16384, page=64),
        # a decode batch of 1000 to 65536 rows that attends to its last 1024 and four sinks
        dict(name="window-b16", op="window", **L3_8B, dtype="bf16", cache="same", scale_rows=0, batch=16, min_len=1000, max_len=65536, page=16, window=1024, sinks=4),
        # the same of many sequences over an 8-bit cache, with a window of 4096
        dict(name="window-b64-e4m3", op="window", **L3_70B, dtype="bf16", cache="e4m3", scale_rows=16, batch=64, min_len=2049, max_len=16384, page=16, window=4096, sinks=16),
        # one sequence of the tiny fp32 shape, a window that is no multiple of anything
        dict(name="window-b1-f32", op="window", **TINY, dtype="f32", cache="same", scale_rows=0, batch=1, min_len=1999, max_len=1999, page=16, window=333, sinks=1),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "append", "append", "read", "window", "window"])
    heads = dict(rng.choice([TINY, MID, L3_8B, L3_8B, L2_7B, L3_70B, ODD_GROUP, WIDE_GROUP]))
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    page = rng.choice([8, 16, 16, 24, 32, 64, 128])
    cache = rng.choice(["e4m3", "int8", "same"] if op == "window" else ["e4m3", "int8"])
    rows = 0 if cache == "same" else rng.choice([1, page, page, page // 2, page // 4])
    case = dict(op=op, **heads, dtype=dtype, cache=cache, scale_rows=rows, batch=_log(rng, 1, 96), page=page)
    if op in ("attend", "window"):
        top = _log(rng, 1, 131072)
        case.update(max_len=top, min_len=rng.randint(max(1, top // 5), top))
        if op == "window":
            case.update(window=_log(rng, 1, 8192), sinks=rng.choice([0, 1, 4, 16, 130]))
    elif op == "append":
        new = rng.choice([1, 1, _log(rng, 1, 4096)])
        case.update(max_new=new, min_new=rng.randint(max(1, new // 3), new), max_len=_log(rng, 1, 4096), gains=rng.random() < 0.7)
    else:
        top = _log(rng, 1, 65536)
        case.update(max_len=top, max_rows=rng.randint(max(1, top // 2), top))
        case["min_rows"] = rng.randint(max(1, case["max_rows"] // 3), case["max_rows"])
    # no drawn case moves more bytes (nor keeps a larger pool) than the largest listed one
    while work(case)["bytes"] > 1.2e9 or _pool_rows(case) * case["kv_heads"] * case["head_dim"] > 1e9:
        if case["batch"] > 1:
            case["batch"] = (case["batch"] + 1) // 2
        else:
            for k in ("max_new", "min_new", "max_len", "min_len", "max_rows", "min_rows"):
                if case.get(k, 0) > 1:
                    case[k] = case[k] // 2
    return case


# ------------------------------------------------------------------ sizes

def _size(case):
    return 2 if case["dtype"] == "bf16" else 4


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _spread(lo, hi, n):
    """n whole numbers from hi down to lo."""
    return [hi - (hi - lo) * i // max(1, n - 1) for i in range(n)]


def _up(a, b):
    return -(-a // b)


def _table_pages(case):
    rows = case["max_len"] + (case["max_new"] + case["scale_rows"] if case["op"] == "append" else 0)
    return _up(rows, case["page"])


def _pool_rows(case):
    return case["batch"] * _table_pages(case) * case["page"]


def _visible(case, n):
    return min(n, case["window"] + case["sinks"]) if case["op"] == "window" else n


def work(case):
    es, D, Hq, Hkv, B, R = _size(case), case["head_dim"], case["q_heads"], case["kv_heads"], case["batch"], case["scale_rows"]
    cs = es if case["cache"] == "same" else 1

    def cache_bytes(n):  # K and V of n rows, their scales and block-table entries
        return 2 * n * Hkv * D * cs + (8 * Hkv * _up(n, R) if R else 0) + 4 * _up(n, case["page"])

    if case["op"] in ("attend", "window"):
        lens = [_visible(case, n) for n in _spread(case["min_len"], case["max_len"], B)]
        return {"bytes": sum(cache_bytes(n) for n in lens) + 2 * B * Hq * D * es + 4 * B * Hq + 4 * B, "flops": 4 * sum(lens) * Hq * D}
    if case["op"] == "append":
        # rows of queries, keys and values and their angles; queries and codes written; the rows of their blocks read back
        n = sum(_spread(case["min_new"], case["max_new"], B))
        back = n + sum(L % R for L in _spread(case["max_len"] // 2, case["max_len"], B))
        return {"bytes": n * ((2 * Hq + 2 * Hkv) * D * es + D * 4) + cache_bytes(n) + cache_bytes(back) + 2 * back * Hkv * D * es,
                "flops": 12 * n * (Hq + 2 * Hkv) * D}
    n = sum(_spread(case["min_rows"], case["max_rows"], B))
    return {"bytes": cache_bytes(n) + 2 * n * Hkv * D * es, "flops": 2 * n * Hkv * D}


# ----------------------------------------------------------------- inputs

_handles = {}


def _handle(case, max_pages):
    """The operators' handle, kept per geometry and capacity as a program keeps it."""
    from paper_2602_01762_gb300 import PagedAttention
    key = (case["q_heads"], case["kv_heads"], case["head_dim"], case["dtype"], case["batch"], max_pages, case["page"])
    if key not in _handles:
        if len(_handles) > 40:
            _handles.clear()
        _handles[key] = PagedAttention(n_q_heads=key[0], n_kv_heads=key[1], head_dim=key[2], dtype=key[3], max_batch=key[4],
                                       max_pages=max_pages, page_size=key[6], rms_eps=EPS, device=0)
    return _handles[key]


def _rope(positions, D):
    """cos and sin of position * theta^(-2j/D), computed in 64 bits, kept in 32: [positions, 2, D/2]."""
    a = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * (
        THETA ** (-torch.arange(0, D, 2, dtype=torch.float64, device="cuda") / D))
    return torch.stack([torch.cos(a), torch.sin(a)], 1).float().contiguous()


def prepare(case, seed):
    dev, dt = "cuda", _dtype(case)
    gen = torch.Generator(device=dev).manual_seed(seed)
    B, Hq, Hkv, D, op = case["batch"], case["q_heads"], case["kv_heads"], case["head_dim"], case["op"]
    page, R, kind = case["page"], case["scale_rows"], case["cache"]

    def normal(*shape, scale=1.0, dtype=dt):
        return torch.randn(shape, generator=gen, device=dev, dtype=dtype).mul_(scale)

    def shuffled(values):
        order = torch.randperm(len(values), generator=gen, device=dev)
        return torch.tensor(values, dtype=torch.int32, device=dev)[order].contiguous()

    def pages():
        """Rows of normal values about 1 in size, as they are or as codes and the scales of their blocks."""
        shape = (n_pages, Hkv, page, D)
        if kind == "same":
            return normal(*shape), None
        # blocks of different sizes: what is 1 is 128, 64 or 32 steps of e4m3's 2, 16, 32 or 64 of int8
        scales = torch.exp2(torch.randint(-8 if kind == "e4m3" else -6, -5 if kind == "e4m3" else -3, (n_pages, Hkv, page // R),
                                          generator=gen, device=dev).float())
        if kind == "e4m3":
            return normal(*shape, scale=120.0, dtype=torch.bfloat16).clamp_(-448, 448).to(torch.float8_e4m3fn), scales
        return normal(*shape, scale=36.0, dtype=torch.bfloat16).round_().clamp_(-127, 127).to(torch.int8), scales

    s = {"case": case, "B": B, "Hq": Hq, "Hkv": Hkv, "D": D, "G": Hq // Hkv, "dt": dt, "scale": D ** -0.5, "page": page, "R": R,
         "kind": kind}
    max_pages = _table_pages(case)
    n_pages = B * max_pages
    s["k_pages"], s["k_scales"] = pages()
    s["v_pages"], s["v_scales"] = pages()
    s["table"] = torch.randperm(n_pages, generator=gen, device=dev).to(torch.int32).view(B, max_pages)
    if op == "append":
        n = case["max_new"]
        s["n_new"] = shuffled(_spread(case["min_new"], n, B))
        s["kv_len"] = shuffled(_spread(case["max_len"] // 2, case["max_len"], B))
        s["pos"] = s["kv_len"] + 5  # five rows were evicted earlier
        s["rope"] = _rope(case["max_len"] + n + 5, D)
        qkv = normal(B, n, (Hq + 2 * Hkv) * D, scale=1.2)  # one projection's rows: queries, keys, values
        s["q"] = qkv[:, :, :Hq * D].unflatten(-1, (Hq, D))
        s["k"] = qkv[:, :, Hq * D:(Hq + Hkv) * D].unflatten(-1, (Hkv, D))
        s["v"] = qkv[:, :, (Hq + Hkv) * D:].unflatten(-1, (Hkv, D))
        s["g_q"], s["g_k"] = (normal(D, scale=0.1) + 1 for _ in range(2)) if case["gains"] else (None, None)
        s["q_out"] = torch.zeros(B, n, Hq, D, dtype=dt, device=dev)
        # the new rows and those before them in their first block
        s["start"] = s["kv_len"] // R * R
        s["n_rows"] = s["kv_len"] - s["start"] + s["n_new"]
        rows = _up(n + R - 1, R) * R
    elif op == "read":
        rows = case["max_rows"]
        s["kv_len"] = shuffled([case["max_len"]] * B)
        s["n_rows"] = shuffled(_spread(case["min_rows"], rows, B))
        s["start"] = torch.minimum(shuffled([7 * b for b in range(B)]), s["kv_len"] - s["n_rows"])
    else:
        s["kv_len"] = shuffled(_spread(case["min_len"], case["max_len"], B)) - 1  # committed rows; the new token's row follows
        s["q"] = normal(B, Hq, D, scale=1.3)  # normed and rotated queries; the cache holds normed and rotated keys
        s["out"], s["lse"] = torch.empty(B, Hq, D, dtype=dt, device=dev), torch.empty(B, Hq, device=dev)
        s["window"], s["sinks"] = case.get("window"), case.get("sinks", 0)
    if op in ("append", "read"):
        s["k_rows"], s["v_rows"] = (torch.zeros(B, rows, Hkv, D, dtype=dt, device=dev) for _ in range(2))
    if own:
        h = s["h"] = _handle(case, max_pages)
        s["cache"] = h.cache(s["k_pages"], s["v_pages"], s["table"], s["kv_len"], k_scales=s["k_scales"], v_scales=s["v_scales"])
    return s


# -------------------------------------------------------------- plain forms

def _rotate(x, cos, sin):
    a, b = x.chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _norm_rope(x, g, cos, sin):
    x = x.float()
    if g is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * g.float()
    return _rotate(x, cos, sin)


def _power_of_two(top, kind):
    """The smallest power of two, from 2^-126 on, that holds values up to `top` in the codes' range; 0 for 0."""
    part, e = torch.frexp(top)  # top = part 2^e, part in [1/2, 1)
    e = e - 9 + (part > 0.875) if kind == "e4m3" else e - 7 + (part > 127 / 128)  # 448 = 7/8 2^9
    return torch.where(top > 0, torch.ldexp(torch.ones_like(top), e.clamp(min=-126)), torch.zeros_like(top))


def _codes(x, kind):
    return x.to(torch.float8_e4m3fn) if kind == "e4m3" else torch.round(x).to(torch.int8)


def _store(s, pages, scales, x):
    """Quantises new rows x [B, n, Hkv, D] into their blocks; the values of the blocks' rows."""
    B, R, page, kind = s["B"], s["R"], s["page"], s["kind"]
    raw = pages.view(torch.uint8)
    j = torch.arange(s["k_rows"].shape[1], device="cuda")
    slot = s["start"][:, None].long() + j
    at, off = s["table"].long().gather(1, slot // page), slot % page
    before = (s["kv_len"] - s["start"])[:, None].long()
    new, used = (j >= before) & (j < s["n_rows"][:, None]), j < s["n_rows"][:, None]
    i = (j - before).clamp(0, x.shape[1] - 1)
    x = torch.where(new[:, :, None, None], x.gather(1, i[:, :, None, None].expand(-1, -1, *x.shape[2:])), torch.zeros((), device="cuda"))

    def of_blocks(t):
        return t.unflatten(1, (-1, R))

    def of_rows(t):
        return t.repeat_interleave(R, 1)

    top = of_blocks(x.abs()).amax((2, 4))  # [B, blocks, Hkv]
    was = scales[at, :, off // R]
    old = torch.where(of_blocks(j < before).any(2)[..., None], of_blocks(was)[:, :, 0], torch.zeros((), device="cuda"))
    scale = torch.maximum(old, _power_of_two(top, kind))
    per = torch.where(scale > 0, scale, torch.ones_like(scale))
    codes = pages[at, :, off].float() if kind == "int8" else raw[at, :, off].view(torch.float8_e4m3fn).float()
    codes = torch.where(new[..., None, None], x / of_rows(per)[..., None], codes * of_rows(old / per)[..., None])
    codes = _codes(codes, kind)
    raw[at, :, off] = torch.where(used[..., None, None], codes.view(torch.uint8), raw[at, :, off])
    scales[at, :, off // R] = torch.where(of_rows(of_blocks(used).any(2))[..., None], of_rows(scale), was)
    return torch.where(used[..., None, None], codes.float() * of_rows(scale)[..., None], torch.zeros((), device="cuda")).to(s["dt"])


def _plain_append(s):
    n = s["q"].shape[1]
    i = torch.arange(n, device="cuda")
    cs = s["rope"][s["pos"][:, None].long() + i]
    cos, sin = cs[:, :, None, 0], cs[:, :, None, 1]
    ok = (i < s["n_new"][:, None])[:, :, None, None]
    s["q_out"].copy_(torch.where(ok, _norm_rope(s["q"], s["g_q"], cos, sin).to(s["dt"]), s["q_out"]))
    s["k_rows"].copy_(_store(s, s["k_pages"], s["k_scales"], _norm_rope(s["k"], s["g_k"], cos, sin)))
    s["v_rows"].copy_(_store(s, s["v_pages"], s["v_scales"], s["v"].float()))
    return {"q": s["q_out"], "k_rows": s["k_rows"], "v_rows": s["v_rows"]}


def _values(s, pages, scales, at, off):
    """Rows `off` of pages `at`, [..., Hkv, D] in 32 bits."""
    x = (pages[at, :, off] if pages.dtype != torch.float8_e4m3fn else pages.view(torch.uint8)[at, :, off].view(pages.dtype)).float()
    return x if scales is None else x.mul_(scales[at, :, off // s["R"]][..., None])


def _plain_read(s):
    i = torch.arange(s["k_rows"].shape[1], device="cuda")
    ok = i < s["n_rows"][:, None]
    slot = torch.where(ok, s["start"][:, None].long() + i, torch.zeros((), dtype=torch.int64, device="cuda"))
    at, off = s["table"].long().gather(1, slot // s["page"]), slot % s["page"]
    k, v = _values(s, s["k_pages"], s["k_scales"], at, off), _values(s, s["v_pages"], s["v_scales"], at, off)
    s["k_rows"].copy_(torch.where(ok[..., None, None], k.to(s["dt"]), s["k_rows"]))
    s["v_rows"].copy_(torch.where(ok[..., None, None], v.to(s["dt"]), s["v_rows"]))
    return {"k_rows": s["k_rows"], "v_rows": s["v_rows"]}


def _plain_attend(s):
    B, Hkv, G, D = s["B"], s["Hkv"], s["G"], s["D"]
    L = s["kv_len"][:, None].long() + 1
    if s["window"] is None:
        slot = torch.arange(s["table"].shape[1] * s["page"], device="cuda").expand(B, -1)
        valid = slot < L
    else:  # the sinks, then the window's rows behind them
        i = torch.arange(s["sinks"] + s["window"], device="cuda")
        slot = torch.where(i < s["sinks"], i, L - s["window"] + i - s["sinks"])
        valid = (slot < L) & ((i < s["sinks"]) | (slot >= s["sinks"]))
        slot = torch.where(valid, slot, torch.zeros_like(slot))
    at, off = s["table"].long().gather(1, slot // s["page"]), slot % s["page"]
    z = torch.matmul(s["q"].float().view(B, Hkv, G, D), _values(s, s["k_pages"], s["k_scales"], at, off).permute(0, 2, 3, 1)) * s["scale"]
    z = torch.where(valid[:, None, None], z, torch.full((), -math.inf, device="cuda"))
    m = z.amax(-1, keepdim=True)
    p = torch.exp(z - m)
    total = p.sum(-1, keepdim=True)
    v = _values(s, s["v_pages"], s["v_scales"], at, off).transpose(1, 2)
    v = torch.where(valid[:, None, :, None], v, torch.zeros((), device="cuda"))
    out = torch.matmul(p / total, v).view(B, s["Hq"], D).to(s["dt"])
    return {"out": out, "lse": (m + torch.log(total)).view(B, s["Hq"])}


_PLAIN = {"append": _plain_append, "read": _plain_read, "attend": _plain_attend, "window": _plain_attend}


# ------------------------------------------------------- the package's operators

def _own_append(s):
    s["h"].append(s["cache"], s["q"], s["k"], s["v"], s["q_out"], s["rope"], g_q=s["g_q"], g_k=s["g_k"], pos=s["pos"], n_new=s["n_new"])
    s["h"].read(s["cache"], s["k_rows"], s["v_rows"], start=s["start"], n_rows=s["n_rows"])
    return {"q": s["q_out"], "k_rows": s["k_rows"], "v_rows": s["v_rows"]}


def _own_read(s):
    s["h"].read(s["cache"], s["k_rows"], s["v_rows"], start=s["start"], n_rows=s["n_rows"])
    return {"k_rows": s["k_rows"], "v_rows": s["v_rows"]}


def _own_attend(s):
    s["h"].attend(s["cache"], s["q"], s["out"], lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


def _own_window(s):
    s["h"].attend(s["cache"], s["q"], s["out"], lse=s["lse"], window=s["window"], sinks=s["sinks"])
    return {"out": s["out"], "lse": s["lse"]}


_OWN = {"append": _own_append, "read": _own_read, "attend": _own_attend, "window": _own_window}


def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["op"]](state)


# ------------------------------------------------------------------ 64 bits

def _norm_rope64(x, g, rope, pos):
    """Rows x [n, H, D] at positions pos.. in 64 bits, as a product with complex phases."""
    x = x.double()
    if g is not None:
        x = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * g.double()
    t = rope[pos:pos + x.shape[0]].double()
    h = x.shape[-1] // 2
    z = torch.complex(x[..., :h].contiguous(), x[..., h:].contiguous()) * torch.complex(t[:, 0], t[:, 1])[:, None]
    return torch.cat([z.real, z.imag], -1)


def _held64(x, stored, scale, R, kind):
    """Rows x [n, Hkv, D] (values) as their blocks hold them: the first `stored` of them were there
    before, with the first block's scale [Hkv]."""
    n = x.shape[0]
    x = torch.cat([x, x.new_zeros(-n % R, *x.shape[1:])]).unflatten(0, (-1, R))  # [blocks, R, Hkv, D]
    new = torch.arange(x.shape[0] * R, device=x.device).view(-1, R, 1, 1) >= stored
    top = torch.where(new, x.abs(), 0.0).amax((1, 3))
    s = torch.where(top > 0, torch.exp2(torch.ceil(torch.log2(top / (448 if kind == "e4m3" else 127)))), 0.0)
    if stored:
        s[0] = torch.maximum(s[0], scale)
    s = s[:, None, :, None]
    y = x / torch.where(s > 0, s, 1.0)
    # e4m3 has four significant bits and steps of 2^-9 at least
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3) if kind == "e4m3" else 1.0
    return (torch.round(y / step) * step * s).flatten(0, 1)[:n]


def exact(case, seed):
    s = prepare(case, seed)
    B, Hq, Hkv, D, G, page = s["B"], s["Hq"], s["Hkv"], s["D"], s["G"], s["page"]
    table, lens = s["table"].cpu().numpy().astype(np.int64), s["kv_len"].cpu().numpy()

    def rows_of(name, b, slots):
        """Rows `slots` of sequence b: [rows, Hkv, D]."""
        at, off = torch.from_numpy(table[b, slots // page]).cuda(), torch.from_numpy(slots % page).cuda()
        pages, scales = s[name + "_pages"], s[name + "_scales"]
        if scales is None:
            return pages[at, :, off].double()
        codes = pages.view(torch.uint8)[at, :, off].view(pages.dtype).double()
        return codes * scales.repeat_interleave(s["R"], 2)[at, :, off].double()[..., None]

    if case["op"] in ("append", "read"):
        got = {n: torch.zeros(s[n].shape, dtype=torch.float64, device="cuda") for n in ("k_rows", "v_rows")}
        start, count = s["start"].cpu().numpy(), s["n_rows"].cpu().numpy()
        if case["op"] == "append":
            got["q"] = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        for b in range(B):
            first, m = int(start[b]), int(count[b])
            stored = int(lens[b]) - first if case["op"] == "append" else m
            rows = {name: rows_of(name, b, np.arange(first, first + stored)) for name in ("k", "v")}
            if case["op"] == "append":
                n, pos, page_of = m - stored, int(s["pos"][b]), table[b, first // page]
                got["q"][b, :n] = _norm_rope64(s["q"][b, :n], s["g_q"], s["rope"], pos)
                new = {"k": _norm_rope64(s["k"][b, :n], s["g_k"], s["rope"], pos), "v": s["v"][b, :n].double()}
                for name in rows:
                    scale = s[name + "_scales"][page_of, :, first % page // s["R"]].double()
                    rows[name] = _held64(torch.cat([rows[name], new[name]]), stored, scale, s["R"], s["kind"])
            for name in rows:
                got[name + "_rows"][b, :m] = rows[name]
        return got

    out, lse = torch.empty(B, Hq, D, dtype=torch.float64, device="cuda"), torch.empty(B, Hq, dtype=torch.float64, device="cuda")
    for b in range(B):
        n = int(lens[b]) + 1
        slots = np.arange(n)
        if s["window"] is not None:
            slots = slots[(slots < s["sinks"]) | (slots >= n - s["window"])]
        k, v = rows_of("k", b, slots), rows_of("v", b, slots)
        for h in range(Hkv):
            z = k[:, h] @ s["q"][b, h * G:(h + 1) * G].double().T * s["scale"]  # [rows, G]
            lse[b, h * G:(h + 1) * G] = torch.logsumexp(z, 0)
            out[b, h * G:(h + 1) * G] = torch.softmax(z, 0).T @ v[:, h]
    return {"out": out, "lse": lse}
