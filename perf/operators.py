"""The work of the paged cache's operators: rows that are normalised and rotated, rows that enter the pages, attention of new
tokens over the pages, each in a plain form (elementary torch operations in 32 bits, angles in 64) and, where ``own`` is set,
as the calls of ``paper_2602_08686_amd.binding`` that a serving program makes.

``listed()`` names the cases, ``draw(rng)`` gives another one of the same ranges, ``prepare`` makes what a program has in hand
before the call, ``run`` is one pass, ``work`` what a pass cannot do without, ``exact`` the results in 64 bits from the
definition.

Three kinds of case:
  rotate   RMS norm of every head of the new queries and keys and their position rotation, dense outputs
  append   the same on the way into a paged cache, values copied beside the keys; or a plain copy of retained rows into lists
           that differ by head
  attend   attention of a chunk of new tokens (causal among themselves), or of one token per sequence, over the pages
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-6


def _case(name, kind, dtype, batch, q_heads, kv_heads, d, new, **kw):
    """new: tokens per sequence in the call; ragged: fewer of them for most sequences (a padded batch); length: rows of the
    longest list behind the call; varied: shorter lists beside it; by_head: a list for every KV head, pages of one head."""
    c = {"kind": kind, "dtype": dtype, "batch": batch, "q_heads": q_heads, "kv_heads": kv_heads, "d": d, "new": new, "ragged": False,
         "token_major": True}
    if kind != "attend":
        c.update(norm=True, rot_dim=d, pairing="halves")
    if kind != "rotate":
        c.update(length=new, varied=False, page=64, by_head=False, pool_token_major=False)
    if kind == "append":
        c.update(with_q=True)
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one decoding step's rows of a batch of 16, at far positions: the smallest, all latency
        _case("rotate_step_b16", "rotate", "bf16", 16, 32, 8, 128, 1),
        # the rows of a whole 32k prompt, as the projections leave them (token by token)
        _case("rotate_prompt_32k", "rotate", "bf16", 1, 32, 8, 128, 32768),
        # f32, a padded batch of odd lengths, a quarter of each row rotated in neighbouring pairs, no norm
        _case("rotate_f32_ragged", "rotate", "f32", 3, 4, 4, 64, 1021, ragged=True, norm=False, rot_dim=16, pairing="neighbours",
              token_major=False),
        # one decoding step of a batch of 16 into pages of 16 rows, queries in the same call
        _case("append_step_b16", "append", "bf16", 16, 32, 8, 128, 1, length=32769, varied=True, page=16),
        # a chunk of a prompt behind a long cache, padded batch of two
        _case("append_chunk_4k", "append", "bf16", 2, 32, 8, 128, 4099, ragged=True, length=20011, varied=True, norm=False),
        # the rows that retention kept (nominal budget 512, lists that differ by head) into pages of one head: a plain copy
        _case("append_kept_b16", "append", "bf16", 16, 32, 8, 128, 544, ragged=True, length=544, page=32, by_head=True, norm=False,
              rot_dim=0, with_q=False, token_major=False),
        # one layer of a decoding step over the retained rows of a batch of 16, a list for every head
        _case("attend_step_kept_b16", "attend", "bf16", 16, 32, 8, 128, 1, length=544, varied=True, page=32, by_head=True),
        # the same over whole 32k prompts, batch 4
        _case("attend_step_32k", "attend", "bf16", 4, 32, 8, 128, 1, length=32768, page=16),
        # a few drafted tokens per sequence, groups of seven heads, ragged lists
        _case("attend_draft_9k", "attend", "bf16", 8, 28, 4, 128, 5, length=9001, varied=True, page=16, pool_token_major=True),
        # a chunk of 2048 tokens at the end of a 32k prompt: most arithmetic
        _case("attend_chunk_2k_32k", "attend", "bf16", 1, 32, 8, 128, 2048, length=32768, page=64),
        # whole prompts of up to 4k tokens, a model without grouped queries
        _case("attend_prompt_4k", "attend", "bf16", 2, 32, 32, 128, 4096, ragged=True, length=4096, page=128),
        # a short f32 prompt in chunks of 200
        _case("attend_f32_1k", "attend", "f32", 1, 4, 4, 64, 200, length=1024, page=16),
    ]


# what bounds a drawn case: query-key pairs over all heads, rows that are moved, rows of the caches
MOST_PAIRS = 32 * 2048 * 32768
MOST_ROWS = 32768 * 40
MOST_CACHE = 4 * 8 * 32768


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "append", "attend", "attend"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    d = rng.choice([64, 128, 128])
    q_heads, kv_heads = rng.choice([(32, 8), (32, 32), (28, 4), (16, 2), (8, 1), (12, 4), (5, 5), (40, 8)])
    while True:
        batch = _log_uniform(rng, 1, 32)
        new = 1 if rng.random() < 0.35 else _log_uniform(rng, 2, 8192)
        length = max(new, _log_uniform(rng, 17, 65536))
        if kind != "attend":
            if batch * new * (q_heads + kv_heads) <= MOST_ROWS and batch * kv_heads * length <= MOST_CACHE:
                break
        elif batch * q_heads * new * length * (4 if dtype == "f32" else 1) <= MOST_PAIRS and batch * kv_heads * length <= MOST_CACHE:
            break
    kw = {"ragged": new > 1 and rng.random() < 0.5, "token_major": rng.random() < 0.7}
    if kind != "attend":
        kw.update(norm=rng.random() < 0.6, rot_dim=rng.choice([d, d, d // 2, 16, 48]), pairing=rng.choice(["halves", "neighbours"]))
    if kind != "rotate":
        kw.update(length=length, varied=rng.random() < 0.6, page=rng.choice([1, 8, 16, 16, 32, 64, 128, 256]), by_head=rng.random() < 0.3,
                  pool_token_major=rng.random() < 0.4)
    if kind == "append":
        kw.update(with_q=rng.random() < 0.6)
        if rng.random() < 0.3:
            kw.update(norm=False, rot_dim=0)
    return _case(None, kind, dtype, batch, q_heads, kv_heads, d, new, **kw)


def _units(c):
    """Lists of the case: (batch, KV head) each."""
    return c["batch"] * c["kv_heads"]


def _counts(c):
    """[batch, kv_heads] new tokens: the same for a sequence's heads, or (retained rows) different ones."""
    n = c["new"]
    if not c["ragged"]:
        return np.full((c["batch"], c["kv_heads"]), n, np.int32)
    each = c.get("by_head") and not c.get("with_q", True)
    i = np.arange(_units(c)).reshape(c["batch"], -1) if each else np.arange(c["batch"])[:, None].repeat(c["kv_heads"], 1)
    return (n - (i * 41 % 97) * (n // 2) // 97).astype(np.int32)


def _lengths(c):
    """[batch, kv_heads] rows of each list behind the call, at least the new ones."""
    n, counts = c["length"], _counts(c)
    if not c["varied"]:
        return counts + (n - c["new"])
    i = np.arange(_units(c)).reshape(c["batch"], -1) if c["by_head"] else np.arange(c["batch"])[:, None].repeat(c["kv_heads"], 1)
    return (counts + (n - c["new"]) * (1.0 - (i * 37 % 89) / 120.0)).astype(np.int32)


def _rows(g, c, heads, scale=1.0):
    """[batch, heads, new, d] of the case's type, token by token in memory or head by head."""
    t = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    shape = (c["batch"], c["new"], heads, c["d"]) if c["token_major"] else (c["batch"], heads, c["new"], c["d"])
    x = (torch.randn(shape, generator=g, device="cuda") * scale).to(t)
    return x.transpose(1, 2) if c["token_major"] else x


def _pages(g, c, s, filled):
    """The pools, the lists of page numbers (in no order, none twice) and the lengths."""
    lengths, page, Hkv = _lengths(c), c["page"], c["kv_heads"]
    lists = lengths if c["by_head"] else lengths.max(1, keepdims=True)
    per_list = -(-lists // page)
    n_pages, most = int(per_list.sum()) + 3, int(per_list.max())
    ids = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    first = np.concatenate([[0], np.cumsum(per_list.ravel())[:-1]]).reshape(per_list.shape)
    at = torch.from_numpy(first[..., None] + np.minimum(np.arange(most), per_list[..., None] - 1)).to("cuda")
    table = ids[at.long()]
    s["table"] = table.contiguous() if c["by_head"] else table[:, 0].contiguous()
    t = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    heads = 1 if c["by_head"] else Hkv
    for name in ("k_pages", "v_pages"):
        shape = (n_pages, page, heads, c["d"]) if c["pool_token_major"] else (n_pages, heads, page, c["d"])
        x = torch.randn(shape, generator=g, device="cuda") if filled else torch.zeros(shape, device="cuda")
        if filled and name == "k_pages":   # one row in twenty stands out, as keys do that many queries look for
            x *= torch.where(torch.rand(shape[:3] + (1,), generator=g, device="cuda") < 0.05, 2.0, 1.0)
        x = x.to(t)
        x = x.transpose(1, 2) if c["pool_token_major"] else x
        s[name] = x.expand(-1, Hkv, -1, -1)   # pages of one head: every head finds its own by its list
    s["length"] = torch.from_numpy(lengths).to("cuda")


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    s = {"case": c, "q": None, "k": None, "count": None, "q_out": None}
    if c["kind"] != "append" or c["with_q"]:
        s["q"] = _rows(g, c, c["q_heads"], 2.0)
    if c["kind"] != "attend":
        s["k"] = _rows(g, c, c["kv_heads"])
        half = c["rot_dim"] // 2
        s["inv_freq"] = (1e6 ** (-torch.arange(half, dtype=torch.float64) / max(half, 1))).float().to("cuda")
        for name in ("q_weight", "k_weight"):
            s[name] = (0.75 + 0.5 * torch.rand(c["d"], generator=g, device="cuda")).to(t) if c["norm"] else None
    if c["ragged"]:
        s["count"] = torch.from_numpy(_counts(c)).to("cuda")
    if c["kind"] == "rotate":   # prompts that are continued: each sequence from a position of its own
        start = torch.randint(0, 131072, (c["batch"], 1), generator=g, device="cuda")
        s["positions"] = (start + torch.arange(c["new"], device="cuda")).to(torch.int32)
        s["q_out"] = torch.zeros(c["batch"], c["q_heads"], c["new"], c["d"], dtype=t, device="cuda")
        s["k_out"] = torch.zeros(c["batch"], c["kv_heads"], c["new"], c["d"], dtype=t, device="cuda")
        return s
    _pages(g, c, s, filled=c["kind"] == "attend")
    if c["kind"] == "append":   # positions of the prompt, which retention leaves behind the rows' places in their lists
        s["v"] = _rows(g, c, c["kv_heads"])
        start = s["length"][:, :1] + torch.randint(0, 4096, (c["batch"], 1), generator=g, device="cuda")
        s["positions"] = (start + torch.arange(c["new"], device="cuda")).to(torch.int32)
        if c["with_q"]:
            s["q_out"] = torch.zeros(c["batch"], c["q_heads"], c["new"], c["d"], dtype=t, device="cuda")
        return s
    s["out"] = torch.zeros(c["batch"], c["new"], c["q_heads"], c["d"], dtype=t, device="cuda").transpose(1, 2)
    s["lse"] = torch.zeros(c["batch"], c["q_heads"], c["new"], device="cuda")
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------------
def _new_rows(s, heads):
    """[batch, heads, new] whether the row is one of the call's."""
    c, n = s["case"], s["case"]["new"]
    if s["count"] is None:
        return torch.ones(c["batch"], heads, n, dtype=torch.bool, device="cuda")
    each = s["count"].repeat_interleave(heads // c["kv_heads"], 1)
    return torch.arange(n, device="cuda") < each[..., None]


def _plain_transform(s, x, weight):
    c, x = s["case"], x.float()
    if c["norm"]:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
    r = c["rot_dim"]
    if r == 0:
        return x
    angle = s["positions"].double()[..., None] * s["inv_freq"].double()
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    if c["pairing"] == "halves":
        a, b = x[..., : r // 2], x[..., r // 2: r]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned, x[..., r:]], -1)


def _places(s, slot):
    """Page and row of `slot` [batch, kv_heads, ...] in the lists."""
    c, table = s["case"], s["table"]
    if table.dim() == 2:
        table = table[:, None].expand(-1, c["kv_heads"], -1)
    page = torch.gather(table, 2, (slot // c["page"]).flatten(2)).view(slot.shape)
    return page.long(), slot % c["page"]


def _plain_rotate(s):
    for x, w, out in ((s["q"], s["q_weight"], s["q_out"]), (s["k"], s["k_weight"], s["k_out"])):
        out.copy_(torch.where(_new_rows(s, x.shape[1])[..., None], _plain_transform(s, x, w).to(out.dtype), out))
    return {"q_out": s["q_out"], "k_out": s["k_out"]}


def _plain_append(s):
    c = s["case"]
    count = c["new"] if s["count"] is None else s["count"][..., None]
    slot = (s["length"][..., None] - count + torch.arange(c["new"], device="cuda")).long()
    here = _new_rows(s, c["kv_heads"])
    page, row = _places(s, torch.where(here, slot, 0))
    head = torch.arange(c["kv_heads"], device="cuda")[None, :, None].expand_as(page)
    at = tuple(x[here] for x in (page, head, row))
    for pool, x in ((s["k_pages"], _plain_transform(s, s["k"], s["k_weight"])), (s["v_pages"], s["v"])):
        base = pool[:, :1] if c["by_head"] else pool   # pages of one head
        base[(at[0], torch.zeros_like(at[1]) if c["by_head"] else at[1], at[2])] = x[here].to(pool.dtype)
    got = {n: s[n][:, :1] if c["by_head"] else s[n] for n in ("k_pages", "v_pages")}
    if c["with_q"]:
        new = _plain_transform(s, s["q"], s["q_weight"]).to(s["q_out"].dtype)
        s["q_out"].copy_(torch.where(_new_rows(s, c["q_heads"])[..., None], new, s["q_out"]))
        got["q_out"] = s["q_out"]
    return got


def _plain_attend(s):
    c = s["case"]
    batch, Hkv, G, n, T = c["batch"], c["kv_heads"], c["q_heads"] // c["kv_heads"], c["new"], c["length"]
    j = torch.arange(T, device="cuda")
    there = j < s["length"][..., None]
    page, row = _places(s, torch.where(there, j, 0))
    head = torch.arange(Hkv, device="cuda")[None, :, None]
    k, v = (torch.where(there[..., None], s[m][page, head, row].float(), 0.0) for m in ("k_pages", "v_pages"))
    count = torch.full_like(s["length"], n) if s["count"] is None else s["count"]
    sees = (s["length"] - count)[..., None] + torch.arange(n, device="cuda") + 1   # rows that query i sees
    q = s["q"].float().reshape(batch, Hkv, G * n, c["d"])
    z = torch.matmul(q, k.transpose(-1, -2).contiguous()).view(batch, Hkv, G, n, T) * (1.0 / math.sqrt(c["d"]))
    z = torch.where(j < sees[:, :, None, :, None], z, -math.inf)
    top = z.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    w = torch.exp(z - top)
    del z
    total = w.sum(-1, keepdim=True)
    out = torch.matmul(w.view(batch, Hkv, G * n, T), v).view(batch, Hkv, G, n, c["d"]) / torch.where(total == 0, 1.0, total)
    lse = (top + torch.log(total))[..., 0]
    here = _new_rows(s, c["q_heads"])
    s["out"].copy_(torch.where(here[..., None], out.reshape(batch, -1, n, c["d"]).to(s["out"].dtype), s["out"]))
    s["lse"].copy_(torch.where(here, lse.reshape(batch, -1, n), s["lse"]))
    return {"out": s["out"], "lse": s["lse"]}


# ---- the framework's calls ------------------------------------------------------------------------------------------------
def _handles(s):
    """What a serving program keeps over its steps: the descriptions of the call's tensors and of the pools, the workspace."""
    from paper_2602_08686_amd import binding as B

    c = s["case"]
    h = {"B": B, "params": B.step_params(q=s["q"], k=s.get("k"), v=s.get("v"), n_q_heads=c["q_heads"], n_kv_heads=c["kv_heads"])}
    if c["kind"] != "attend":
        pairing = B.PAIR_HALVES if c["pairing"] == "halves" else B.PAIR_NEIGHBOURS
        h["rotation"] = B.make_rotation(c["rot_dim"], pairing=pairing, norm=c["norm"], norm_eps=EPS)
    if c["kind"] != "rotate":
        h["pages"] = B.pages_for(s["k_pages"], s["v_pages"], s["table"])
    if c["kind"] == "attend":
        need = B.ckv_paged_workspace_bytes(h["params"], c["length"])
        h["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    s["handles"] = h
    return h


def run(state):
    s, kind = state, state["case"]["kind"]
    if not own:
        return {"rotate": _plain_rotate, "append": _plain_append, "attend": _plain_attend}[kind](s)
    h = s.get("handles") or _handles(s)
    B = h["B"]
    if kind == "rotate":
        B.ckv_norm_rotate(h["params"], h["rotation"], s["q"], s["k"], s["positions"], s["inv_freq"], s["q_weight"], s["k_weight"],
                          s["q_out"], s["k_out"], count=s["count"])
        return {"q_out": s["q_out"], "k_out": s["k_out"]}
    if kind == "append":
        B.ckv_paged_append(h["params"], h["rotation"], h["pages"], s["k"], s["v"], s["k_pages"], s["v_pages"], s["table"], s["length"],
                           count=s["count"], positions=s["positions"], inv_freq=s["inv_freq"], k_weight=s["k_weight"],
                           q=s["q"], q_weight=s["q_weight"], q_out=s["q_out"])
        got = {n: s[n][:, :1] if s["case"]["by_head"] else s[n] for n in ("k_pages", "v_pages")}
        if s["q_out"] is not None:
            got["q_out"] = s["q_out"]
        return got
    B.ckv_paged_attention(h["params"], h["pages"], s["q"], s["k_pages"], s["v_pages"], s["table"], s["length"], s["case"]["length"],
                          s["out"], s["lse"], h["workspace"], count=s["count"])
    return {"out": s["out"], "lse": s["lse"]}


def work(case):
    """Every input byte that the results depend on read once, every output byte written once; the visible query-key pairs'
    two products."""
    c = case
    e = 4 if c["dtype"] == "f32" else 2
    G, d = c["q_heads"] // c["kv_heads"], c["d"]
    counts = _counts(c).astype(np.float64)
    new = counts.sum()   # rows of K
    if c["kind"] == "rotate":
        return {"bytes": 2 * new * (1 + G) * d * e + 4 * c["batch"] * c["new"], "flops": 0.0}
    lengths = _lengths(c).astype(np.float64)
    if c["kind"] == "append":
        heads = 2 + (G if c["with_q"] else 0)
        return {"bytes": 2 * new * heads * d * e + 4 * c["batch"] * c["new"] + 4 * _units(c), "flops": 0.0}
    lists = lengths.size if c["by_head"] else c["batch"]
    pairs = G * (counts * (lengths - counts) + counts * (counts + 1) / 2).sum()
    table = 4.0 * lists * lengths.mean() / c["page"]
    return {"bytes": 2 * lengths.sum() * d * e + new * G * (2 * d * e + 4) + table + 4 * _units(c), "flops": 4.0 * d * pairs}


# ---- 64 bits --------------------------------------------------------------------------------------------------------------
def _transform64(s, x, weight):
    """The rotation as a product of complex numbers."""
    c, x, r = s["case"], x.double(), s["case"]["rot_dim"]
    if c["norm"]:
        x = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * weight.double()
    if r == 0:
        return x
    front = x[..., :r].unflatten(-1, (2, r // 2)).transpose(-1, -2) if c["pairing"] == "halves" else x[..., :r].unflatten(-1, (r // 2, 2))
    angle = s["positions"].double()[:, None, :, None] * s["inv_freq"].double()
    front = torch.view_as_real(torch.view_as_complex(front.contiguous()) * torch.polar(torch.ones_like(angle), angle))
    front = front.transpose(-1, -2).flatten(-2) if c["pairing"] == "halves" else front.flatten(-2)
    return torch.cat([front, x[..., r:]], -1)


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    counts, G = _counts(c), c["q_heads"] // c["kv_heads"]
    if c["kind"] == "rotate":
        out = {}
        for n, heads in (("q", c["q_heads"]), ("k", c["kv_heads"])):
            x = _transform64(s, s[n], s[n + "_weight"])
            for b in range(c["batch"]):
                x[b, :, counts[b, 0]:] = 0.0
            out[n + "_out"] = x
        return out
    lengths, table, page = _lengths(c), s["table"].cpu().numpy(), c["page"]
    if _units(c) > 600:
        return None   # a list at a time takes too long
    lists = lambda b, g: table[b, g] if c["by_head"] else table[b]  # noqa: E731
    if c["kind"] == "append":
        out = {}
        for n, x in (("k_pages", _transform64(s, s["k"], s["k_weight"])), ("v_pages", s["v"].double())):
            pool = torch.zeros_like(s[n][:, :1] if c["by_head"] else s[n], dtype=torch.float64)
            for b in range(c["batch"]):
                for g in range(c["kv_heads"]):
                    slot = np.arange(lengths[b, g] - counts[b, g], lengths[b, g])
                    ids, row = torch.from_numpy(lists(b, g)[slot // page]).long().cuda(), torch.from_numpy(slot % page).cuda()
                    pool[ids, 0 if c["by_head"] else g, row] = x[b, g, : counts[b, g]]
            out[n] = pool
        if c["with_q"]:
            x = _transform64(s, s["q"], s["q_weight"])
            for b in range(c["batch"]):
                for h in range(c["q_heads"]):
                    x[b, h, counts[b, h // G]:] = 0.0
            out["q_out"] = x
        return out
    out = torch.zeros(c["batch"], c["q_heads"], c["new"], c["d"], dtype=torch.float64, device="cuda")
    lse = torch.zeros(c["batch"], c["q_heads"], c["new"], dtype=torch.float64, device="cuda")
    for b in range(c["batch"]):
        for g in range(c["kv_heads"]):
            m, T = int(counts[b, g]), int(lengths[b, g])
            slot = np.arange(T)
            ids, row = torch.from_numpy(lists(b, g)[slot // page]).long().cuda(), torch.from_numpy(slot % page).cuda()
            k, v = s["k_pages"][ids, g, row].double(), s["v_pages"][ids, g, row].double()
            hidden = torch.ones(m, T, dtype=torch.bool, device="cuda").triu(T - m + 1)
            for h in range(g * G, (g + 1) * G):
                z = (s["q"][b, h, :m].double() @ k.t()).div_(math.sqrt(c["d"])).masked_fill_(hidden, -math.inf)
                lse[b, h, :m] = torch.logsumexp(z, 1)
                out[b, h, :m] = torch.softmax(z, 1) @ v
    return {"out": out, "lse": lse}
