"""Performance cases of the paged-cache operators: the per-head norm of queries
and keys with the position rotation (stored into a paged key-value cache, or
dense with its gradient), the attention of one new token over such a cache, and
eviction from it by accumulated attention weight.

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
        dict(name="attend-b1-short", op="attend", **L3_8B, dtype="bf16", batch=1, min_len=517, max_len=517, page=16, weights=False),
        # fp32 reference serving of the mid shape, pages that are no multiple of a tile, weights kept for eviction
        dict(name="attend-b3-f32", op="attend", **MID, dtype="f32", batch=3, min_len=411, max_len=2999, page=24, weights=True),
        # a mixed batch: one sequence has just begun, others are thousands of tokens in; weights kept for eviction
        dict(name="attend-b16-ragged", op="attend", **L3_8B, dtype="bf16", batch=16, min_len=1, max_len=8192, page=16, weights=True),
        # multi-head (ungrouped) layers at the bench's batch 8 and context
        dict(name="attend-b8-mha", op="attend", **L2_7B, dtype="bf16", batch=8, min_len=2048, max_len=4096, page=64, weights=False),
        # a full server: many long sequences over eight query heads per key head
        dict(name="attend-b64-long", op="attend", **L3_70B, dtype="bf16", batch=64, min_len=6001, max_len=16384, page=32, weights=False),
        # one document of 131072 tokens: one sequence has to fill the whole GPU
        dict(name="attend-b1-128k", op="attend", **L3_8B, dtype="bf16", batch=1, min_len=131071, max_len=131071, page=16, weights=False),
        # the decode step's rows at batch 1: a few KB, latency alone
        dict(name="append-b1-token", op="append", **L3_8B, dtype="bf16", batch=1, max_new=1, min_new=1, max_len=2047, page=16, gains=True),
        # ragged prompts of up to 2048 tokens stored behind what the cache already holds
        dict(name="append-b8-prompt", op="append", **L3_8B, dtype="bf16", batch=8, max_new=2048, min_new=1021, max_len=777, page=16, gains=True),
        # forward and backward of the tiny fp32 shape over a 64-row prompt
        dict(name="grad-b1-f32", op="grad", **TINY, dtype="f32", batch=1, max_new=64, min_new=64),
        # forward and backward of a training batch: 16384 rows, some sequences shorter than the batch's length
        dict(name="grad-b4-train", op="grad", **L3_8B, dtype="bf16", batch=4, max_new=4096, min_new=3001),
        # a decode batch that has run 255 tokens over its budget of 4096
        dict(name="evict-b16-steady", op="evict", **L3_8B, dtype="bf16", batch=16, min_len=3900, max_len=4351, page=16, budget=4096, sinks=4, recent=512),
        # a long prompt cut down to 4096 rows at once
        dict(name="evict-b1-prompt", op="evict", **L3_8B, dtype="bf16", batch=1, min_len=65537, max_len=65537, page=64, budget=4096, sinks=16, recent=1024),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "append", "grad", "evict", "evict"])
    heads = dict(rng.choice([TINY, MID, L3_8B, L3_8B, L2_7B, L3_70B, ODD_GROUP, WIDE_GROUP]))
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    batch = _log(rng, 1, 96)
    page = rng.choice([8, 16, 16, 24, 32, 64, 128])
    case = dict(op=op, **heads, dtype=dtype, batch=batch)
    if op == "attend":
        top = _log(rng, 1, 131072)
        case.update(max_len=top, min_len=rng.randint(max(1, top // 5), top), page=page, weights=rng.random() < 0.4)
    elif op == "append":
        new = rng.choice([1, 1, _log(rng, 1, 4096)])
        case.update(max_new=new, min_new=rng.randint(max(1, new // 3), new), max_len=_log(rng, 1, 4096), page=page,
                    gains=rng.random() < 0.7)
    elif op == "grad":
        new = _log(rng, 1, 8192)
        case.update(max_new=new, min_new=rng.randint(max(1, new // 2), new))
    else:
        top = _log(rng, 48, 100000)
        budget = max(16, int(top * rng.uniform(0.1, 0.97)))
        case.update(max_len=top, min_len=rng.randint(max(1, top // 2), top), page=page, budget=budget,
                    sinks=rng.randint(0, budget // 8), recent=rng.randint(0, budget // 2))
    # no drawn case moves more bytes (nor keeps a larger pool) than the largest listed ones
    while work(case)["bytes"] > 1.2e9 or case["batch"] * case.get("max_len", 1) * case["kv_heads"] * case["head_dim"] > 6e8:
        if case["batch"] > 1:
            case["batch"] = (case["batch"] + 1) // 2
        else:
            for k in ("max_new", "min_new", "max_len", "min_len", "budget", "sinks", "recent"):
                if k in case and (k in ("sinks", "recent") or case[k] > 1):
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


def work(case):
    es, D, Hq, Hkv, B = _size(case), case["head_dim"], case["q_heads"], case["kv_heads"], case["batch"]
    if case["op"] == "attend":
        lens = _spread(case["min_len"], case["max_len"], B)
        n = sum(lens)
        b = 2 * n * Hkv * D * es + 2 * B * Hq * D * es + 4 * sum(_up(x, case["page"]) for x in lens) + 4 * B + 4 * B * Hq
        return {"bytes": b + (8 * n * Hkv if case["weights"] else 0), "flops": 4 * n * Hq * D}
    if case["op"] == "append":
        n = sum(_spread(case["min_new"], case["max_new"], B))
        return {"bytes": 2 * n * (Hq + 2 * Hkv) * D * es + n * Hkv * 4 + n * D * 4, "flops": 8 * n * (Hq + Hkv) * D}
    if case["op"] == "grad":
        n = sum(_spread(case["min_new"], case["max_new"], B))
        full = B * case["max_new"]
        # forward: read and write; backward: read gradient and input, write the gradient (zeros past a sequence's rows too)
        return {"bytes": (4 * n + full) * (Hq + Hkv) * D * es + 2 * n * D * 4, "flops": 30 * n * (Hq + Hkv) * D}
    lens = _spread(case["min_len"], case["max_len"], B)
    kept = sum(min(x, case["budget"]) for x in lens)
    read = sum(x for x in lens if x > case["budget"])
    return {"bytes": kept * Hkv * (4 * D * es + 8) + read * Hkv * 4 + B * Hkv * case["budget"] * 4, "flops": 8 * read * Hkv}


# ----------------------------------------------------------------- inputs

_handles = {}


def _handle(case, max_pages, page):
    """The operators' handle, kept per geometry and capacity as a program keeps it."""
    from paper_2602_01762_gb300 import PagedAttention
    key = (case["q_heads"], case["kv_heads"], case["head_dim"], case["dtype"], case["batch"], max_pages, page, bool(case.get("weights")))
    if key not in _handles:
        if len(_handles) > 40:
            _handles.clear()
        _handles[key] = PagedAttention(
            n_q_heads=key[0], n_kv_heads=key[1], head_dim=key[2], dtype=key[3], max_batch=key[4], max_pages=max_pages,
            page_size=page, track_weights=key[7], rms_eps=EPS, device=0)
    return _handles[key]


def _rope(positions, D):
    """cos and sin of position * theta^(-2j/D), computed in 64 bits, kept in 32: [positions, 2, D/2]."""
    a = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * (
        THETA ** (-torch.arange(0, D, 2, dtype=torch.float64, device="cuda") / D))
    return torch.stack([torch.cos(a), torch.sin(a)], 1).float().contiguous()


def prepare(case, seed):
    dev, dt = "cuda", _dtype(case)
    gen = torch.Generator(device=dev).manual_seed(seed)
    B, Hq, Hkv, D = case["batch"], case["q_heads"], case["kv_heads"], case["head_dim"]
    op = case["op"]

    def normal(*shape, scale=1.0, dtype=dt):
        return torch.randn(shape, generator=gen, device=dev, dtype=dtype).mul_(scale)

    def shuffled(values):
        order = torch.randperm(len(values), generator=gen, device=dev)
        return torch.tensor(values, dtype=torch.int32, device=dev)[order].contiguous()

    s = {"case": case, "B": B, "Hq": Hq, "Hkv": Hkv, "D": D, "G": Hq // Hkv, "dt": dt, "scale": D ** -0.5}
    if op == "grad":
        n = case["max_new"]
        qkv = normal(B, n, (Hq + 2 * Hkv) * D, scale=0.7)  # one projection's rows: queries, keys, values
        s["q"] = qkv[:, :, :Hq * D].unflatten(-1, (Hq, D))
        s["k"] = qkv[:, :, Hq * D:(Hq + Hkv) * D].unflatten(-1, (Hkv, D))
        s["n_new"] = shuffled(_spread(case["min_new"], n, B))
        s["pos"] = shuffled([7 * b for b in range(B)])
        s["rope"] = _rope(n + 7 * B, D)
        s["g_q"], s["g_k"] = (normal(D, scale=0.1) + 1 for _ in range(2))
        s["dq_out"], s["dk_out"] = normal(B, n, Hq, D, scale=0.02), normal(B, n, Hkv, D, scale=0.02)
        s["q_out"], s["k_out"] = torch.zeros(B, n, Hq, D, dtype=dt, device=dev), torch.zeros(B, n, Hkv, D, dtype=dt, device=dev)
        s["dq"], s["dk"] = torch.empty_like(s["q_out"]), torch.empty_like(s["k_out"])
        s["dg_q"], s["dg_k"] = (torch.empty(D, device=dev) for _ in range(2))
        if own:
            s["h"] = _handle(case, 1, 16)
        return s

    page = s["page"] = case["page"]
    n_new = case["max_new"] if op == "append" else 0
    rows = case["max_len"] + n_new
    max_pages = s["max_pages"] = _up(rows, page)
    spare = _up(case["budget"], page) if op == "evict" else 0
    n_pages = B * (max_pages + spare)
    s["k_pages"], s["v_pages"] = normal(n_pages, Hkv, page, D), normal(n_pages, Hkv, page, D)
    table = torch.randperm(n_pages, generator=gen, device=dev).to(torch.int32).view(B, max_pages + spare)
    s["table"] = table[:, :max_pages].contiguous()
    weights = None
    if op == "append":
        s["n_new"] = shuffled(_spread(case["min_new"], n_new, B))
        s["kv_len"] = shuffled(_spread(case["max_len"] // 2, case["max_len"], B))
        s["pos"] = s["kv_len"] + 5  # five rows were evicted earlier
        s["rope"] = _rope(rows + 5, D)
        qkv = normal(B, n_new, (Hq + 2 * Hkv) * D, scale=1.4)
        s["q"] = qkv[:, :, :Hq * D].unflatten(-1, (Hq, D))
        s["k"] = qkv[:, :, Hq * D:(Hq + Hkv) * D].unflatten(-1, (Hkv, D))
        s["v"] = qkv[:, :, (Hq + Hkv) * D:].unflatten(-1, (Hkv, D))
        s["g_q"], s["g_k"] = (normal(D, scale=0.1) + 1 for _ in range(2)) if case["gains"] else (None, None)
        s["q_out"] = torch.zeros(B, n_new, Hq, D, dtype=dt, device=dev)
        weights = torch.rand(n_pages, Hkv, page, generator=gen, device=dev)
    elif op == "attend":
        s["kv_len"] = shuffled(_spread(case["min_len"], case["max_len"], B)) - 1  # committed rows; the new token's row follows
        s["q"] = normal(B, Hq, D, scale=1.3)  # normed and rotated queries; the cache holds normed and rotated keys
        s["out"], s["lse"] = torch.empty(B, Hq, D, dtype=dt, device=dev), torch.empty(B, Hq, device=dev)
        if case["weights"]:
            weights = torch.rand(n_pages, Hkv, page, generator=gen, device=dev)
    else:
        s["kv_len"] = shuffled(_spread(case["min_len"], case["max_len"], B))
        s["budget"], s["sinks"], s["recent"] = case["budget"], case["sinks"], case["recent"]
        s["table_to"] = table[:, max_pages:].contiguous()
        s["kept"] = torch.empty(B, Hkv, case["budget"], dtype=torch.int32, device=dev)
        s["len_to"] = torch.empty(B, dtype=torch.int32, device=dev)
        # a few heavy rows, a long tail, and rows that got nothing (their weights tie)
        weights = torch.rand(n_pages, Hkv, page, generator=gen, device=dev).pow_(8).mul_(40)
        weights.mul_(weights > 1e-6)
    s["weights"] = weights
    if own:
        h = s["h"] = _handle(case, max(max_pages, spare), page)
        s["cache"] = h.cache(s["k_pages"], s["v_pages"], s["table"], s["kv_len"], weights=weights)
        if op == "evict":
            s["cache_to"] = h.cache(s["k_pages"], s["v_pages"], s["table_to"], s["len_to"], weights=weights)
    return s


# -------------------------------------------------------------- plain forms

def _rotate(x, cos, sin):
    a, b = x.chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _rows(s):
    """(valid rows, row index i, cos, sin) of a [B, n] block of new rows."""
    n = s["q"].shape[1]
    i = torch.arange(n, device="cuda")
    cs = s["rope"][s["pos"][:, None].long() + i]
    return (i < s["n_new"][:, None]), i, cs[:, :, None, 0], cs[:, :, None, 1]


def _norm_rope(x, g, cos, sin):
    x = x.float()
    if g is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * g.float()
    return _rotate(x, cos, sin)


def _plain_append(s):
    valid, i, cos, sin = _rows(s)
    ok = valid[:, :, None, None]
    slot = s["kv_len"][:, None].long() + i
    page, off = s["table"].long().gather(1, slot // s["page"]), slot % s["page"]
    s["q_out"].copy_(torch.where(ok, _norm_rope(s["q"], s["g_q"], cos, sin).to(s["dt"]), s["q_out"]))
    k = _norm_rope(s["k"], s["g_k"], cos, sin).to(s["dt"])
    s["k_pages"][page, :, off] = torch.where(ok, k, s["k_pages"][page, :, off])
    s["v_pages"][page, :, off] = torch.where(ok, s["v"], s["v_pages"][page, :, off])
    w = s["weights"][page, :, off]
    s["weights"][page, :, off] = torch.where(ok[..., 0], torch.zeros_like(w), w)
    return {"q": s["q_out"], "k_pages": s["k_pages"], "v_pages": s["v_pages"], "weights": s["weights"]}


def _backward(x, g, dy, ok, cos, sin):
    """Gradients of the norm and rotation of one tensor: its rows' and its gain's."""
    x, dy, g = x.float(), dy.float(), g.float()
    dz = torch.where(ok, _rotate(dy, cos, -sin), torch.zeros((), device="cuda"))
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    n = x * r
    dn = dz * g
    return r * (dn - n * (dn * n).mean(-1, keepdim=True)), (dz * n).sum((0, 1, 2))


def _plain_grad(s):
    valid, _, cos, sin = _rows(s)
    ok = valid[:, :, None, None]
    s["q_out"].copy_(torch.where(ok, _norm_rope(s["q"], s["g_q"], cos, sin).to(s["dt"]), s["q_out"]))
    s["k_out"].copy_(torch.where(ok, _norm_rope(s["k"], s["g_k"], cos, sin).to(s["dt"]), s["k_out"]))
    dq, dg_q = _backward(s["q"], s["g_q"], s["dq_out"], ok, cos, sin)
    dk, dg_k = _backward(s["k"], s["g_k"], s["dk_out"], ok, cos, sin)
    return {"q": s["q_out"], "k": s["k_out"], "dq": dq.to(s["dt"]), "dk": dk.to(s["dt"]), "dg_q": dg_q, "dg_k": dg_k}


def _gather(pages, table):
    """[n_pages, Hkv, page, ...] by a table [B, P] -> [B, Hkv, P * page, ...]"""
    return pages[table.long()].transpose(1, 2).flatten(2, 3)


def _plain_attend(s):
    B, Hkv, G, D = s["B"], s["Hkv"], s["G"], s["D"]
    k = _gather(s["k_pages"], s["table"]).float()
    slot = torch.arange(k.shape[2], device="cuda")
    valid = slot <= s["kv_len"][:, None]
    z = torch.matmul(s["q"].float().view(B, Hkv, G, D), k.transpose(2, 3)) * s["scale"]
    del k
    z = torch.where(valid[:, None, None], z, torch.full((), -math.inf, device="cuda"))
    m = z.amax(-1, keepdim=True)
    p = torch.exp(z - m)
    total = p.sum(-1, keepdim=True)
    p = p / total
    v = torch.where(valid[:, None, :, None], _gather(s["v_pages"], s["table"]), torch.zeros((), dtype=s["dt"], device="cuda"))
    out = torch.matmul(p, v.float()).view(B, s["Hq"], D).to(s["dt"])
    lse = (m + torch.log(total)).view(B, s["Hq"])
    if s["weights"] is None:
        return {"out": out, "lse": lse}
    page, off = s["table"].long()[:, slot // s["page"]], (slot % s["page"]).expand(B, -1)
    s["weights"][page, :, off] += torch.where(valid[:, None], p.sum(2), torch.zeros((), device="cuda")).transpose(1, 2)
    return {"out": out, "lse": lse, "weights": s["weights"]}


def _plain_evict(s):
    budget = s["budget"]
    w = _gather(s["weights"], s["table"])
    slot = torch.arange(w.shape[2], device="cuda")
    L = s["kv_len"][:, None]
    keep = (slot < s["sinks"]) | (slot >= L - s["recent"])
    inf = torch.full((), math.inf, device="cuda")
    w = torch.where(keep[:, None], inf, w)
    w = torch.where((slot < L)[:, None], w, -inf)
    order = torch.sort(w, dim=-1, descending=True, stable=True).indices[..., :budget]
    if order.shape[-1] < budget:  # a budget above the table's rows
        order = torch.cat([order, order.new_full((*order.shape[:2], budget - order.shape[-1]), w.shape[2])], -1)
    j = torch.arange(budget, device="cuda")
    kept = torch.where(order < L[..., None], order, w.shape[2])
    kept = torch.sort(kept, dim=-1).values
    ok = j < torch.clamp(L, max=budget)  # [B, budget]
    ok = ok[:, None]
    at = torch.where(ok, kept, torch.zeros_like(kept))
    B, Hkv = kept.shape[:2]
    head = torch.arange(Hkv, device="cuda")[:, None]
    page = s["table"].long()[:, None].expand(B, Hkv, -1).gather(2, at // s["page"])
    to = s["table_to"].long()[:, j // s["page"]][:, None].expand(B, Hkv, -1)
    off = (j % s["page"]).expand(B, Hkv, -1)
    k, v, wt = s["k_pages"], s["v_pages"], s["weights"]
    k[to, head, off] = torch.where(ok[..., None], k[page, head, at % s["page"]], k[to, head, off])
    v[to, head, off] = torch.where(ok[..., None], v[page, head, at % s["page"]], v[to, head, off])
    wt[to, head, off] = torch.where(ok, wt[page, head, at % s["page"]], wt[to, head, off])
    s["len_to"].copy_(torch.clamp(s["kv_len"], max=budget))
    s["kept"].copy_(torch.where(ok, kept, torch.full_like(kept, -1)))
    return {"kept": s["kept"], "kv_len": s["len_to"], "k_pages": k, "v_pages": v, "weights": wt}


_PLAIN = {"append": _plain_append, "grad": _plain_grad, "attend": _plain_attend, "evict": _plain_evict}


# ------------------------------------------------------- the package's operators

def _own_append(s):
    s["h"].append(s["cache"], s["q"], s["k"], s["v"], s["q_out"], s["rope"], g_q=s["g_q"], g_k=s["g_k"], pos=s["pos"], n_new=s["n_new"])
    return {"q": s["q_out"], "k_pages": s["k_pages"], "v_pages": s["v_pages"], "weights": s["weights"]}


def _own_grad(s):
    h = s["h"]
    h.qk_norm_rope(s["q"], s["k"], s["q_out"], s["k_out"], s["rope"], s["pos"], g_q=s["g_q"], g_k=s["g_k"], n_new=s["n_new"])
    h.qk_norm_rope_backward(s["dq_out"], s["dk_out"], s["q"], s["k"], s["dq"], s["dk"], s["rope"], s["pos"], g_q=s["g_q"],
                            g_k=s["g_k"], dg_q=s["dg_q"], dg_k=s["dg_k"], n_new=s["n_new"])
    return {"q": s["q_out"], "k": s["k_out"], "dq": s["dq"], "dk": s["dk"], "dg_q": s["dg_q"], "dg_k": s["dg_k"]}


def _own_attend(s):
    s["h"].attend(s["cache"], s["q"], s["out"], lse=s["lse"])
    if s["weights"] is None:
        return {"out": s["out"], "lse": s["lse"]}
    return {"out": s["out"], "lse": s["lse"], "weights": s["weights"]}


def _own_evict(s):
    s["h"].evict(s["cache"], s["cache_to"], s["kept"], sinks=s["sinks"], recent=s["recent"])
    return {"kept": s["kept"], "kv_len": s["len_to"], "k_pages": s["k_pages"], "v_pages": s["v_pages"], "weights": s["weights"]}


_OWN = {"append": _own_append, "grad": _own_grad, "attend": _own_attend, "evict": _own_evict}


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


def _grad64(x, g, dy, rope, pos):
    """Row and gain gradients by automatic differentiation of the 64-bit forward."""
    with torch.enable_grad():
        x, g = x.double().requires_grad_(), g.double().requires_grad_()
        return torch.autograd.grad(_norm_rope64(x, g, rope, pos), (x, g), dy.double())


def exact(case, seed):
    s = prepare(case, seed)
    B, Hq, Hkv, D, G = s["B"], s["Hq"], s["Hkv"], s["D"], s["G"]
    if case["op"] == "grad":
        q, k, dq, dk = (torch.zeros(s[n].shape, dtype=torch.float64, device="cuda") for n in ("q", "k", "q", "k"))
        dg_q, dg_k = (torch.zeros(D, dtype=torch.float64, device="cuda") for _ in range(2))
        for b in range(B):
            n, pos = int(s["n_new"][b]), int(s["pos"][b])
            for x, g, dy, y, dx, dg in ((s["q"], s["g_q"], s["dq_out"], q, dq, dg_q), (s["k"], s["g_k"], s["dk_out"], k, dk, dg_k)):
                y[b, :n] = _norm_rope64(x[b, :n], g, s["rope"], pos)
                a, c = _grad64(x[b, :n], g, dy[b, :n], s["rope"], pos)
                dx[b, :n] = a
                dg += c
        return {"q": q, "k": k, "dq": dq, "dk": dk, "dg_q": dg_q, "dg_k": dg_k}

    page, table = case["page"], s["table"].cpu().numpy().astype(np.int64)

    def rows_of(b, pages, n):
        """Rows 0..n of sequence b: [Hkv, n, ...]."""
        at = torch.from_numpy(table[b, :_up(n, page)]).cuda()
        return pages.index_select(0, at).transpose(0, 1).reshape(Hkv, -1, *pages.shape[3:])[:, :n]

    if case["op"] == "append":
        q, kp, vp, w = s["q_out"].double(), s["k_pages"].double(), s["v_pages"].double(), s["weights"].double()
        for b in range(B):
            n, pos, L = int(s["n_new"][b]), int(s["pos"][b]), int(s["kv_len"][b])
            slots = np.arange(L, L + n)
            at, off = torch.from_numpy(table[b, slots // page]).cuda(), torch.from_numpy(slots % page).cuda()
            q[b, :n] = _norm_rope64(s["q"][b, :n], s["g_q"], s["rope"], pos)
            kp[at, :, off] = _norm_rope64(s["k"][b, :n], s["g_k"], s["rope"], pos)
            vp[at, :, off] = s["v"][b, :n].double()
            w[at, :, off] = 0
        return {"q": q, "k_pages": kp, "v_pages": vp, "weights": w}

    if case["op"] == "attend":
        out, lse = torch.empty(B, Hq, D, dtype=torch.float64, device="cuda"), torch.empty(B, Hq, dtype=torch.float64, device="cuda")
        w = s["weights"].double() if case["weights"] else None
        for b in range(B):
            n = int(s["kv_len"][b]) + 1
            k, v = rows_of(b, s["k_pages"], n), rows_of(b, s["v_pages"], n)
            for h in range(Hkv):
                z = k[h].double() @ s["q"][b, h * G:(h + 1) * G].double().T * s["scale"]  # [n, G]
                lse[b, h * G:(h + 1) * G] = torch.logsumexp(z, 0)
                p = torch.softmax(z, 0)
                out[b, h * G:(h + 1) * G] = p.T @ v[h].double()
                if w is not None:
                    at = torch.arange(n, device="cuda")
                    pg = s["table"][b].long()[at // page]
                    w[pg, h, at % page] += p.sum(1)
        return {"out": out, "lse": lse} if w is None else {"out": out, "lse": lse, "weights": w}

    # eviction: the rows' order by weight, then slot, sequence by sequence
    budget, sinks, recent = case["budget"], case["sinks"], case["recent"]
    kept = np.full((B, Hkv, budget), -1, dtype=np.int64)
    lens = s["kv_len"].cpu().numpy()
    kp, vp, w = s["k_pages"].double(), s["v_pages"].double(), s["weights"].double()
    for b in range(B):
        L = int(lens[b])
        wb = rows_of(b, s["weights"], L).cpu().numpy()
        for h in range(Hkv):
            if L <= budget:
                keep = np.arange(L)
            else:
                mid = np.arange(sinks, L - recent)
                best = mid[np.lexsort((mid, -wb[h, sinks:L - recent].astype(np.float64)))][:budget - sinks - recent]
                keep = np.sort(np.concatenate([np.arange(sinks), best, np.arange(L - recent, L)]))
            kept[b, h, :len(keep)] = keep
            src, j = torch.from_numpy(keep).cuda(), torch.arange(len(keep), device="cuda")
            pg, to = s["table"][b].long()[src // page], s["table_to"][b].long()[j // page]
            for pool, whole in ((kp, s["k_pages"]), (vp, s["v_pages"]), (w, s["weights"])):
                pool[to, h, j % page] = whole[pg, h, src % page].double()
    return {"kept": kept, "kv_len": np.minimum(lens, budget), "k_pages": kp, "v_pages": vp, "weights": w}
