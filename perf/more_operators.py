"""The work of drafted trees over a paged cache and of the pages' lists, each in a plain form (elementary torch operations in 32 bits) and,
where ``own`` is set, as the calls of ``paper_2602_08686_amd.binding`` that a serving program makes.

``listed()`` names the cases, ``draw(rng)`` gives another one of the same ranges, ``prepare`` makes what a program has in hand
before the call, ``run`` is one pass, ``work`` what a pass cannot do without, ``exact`` the results in 64 bits from the
definition.

Kinds of case:
  masks    a tree of drafted tokens, given by parents: which tokens each of them sees (a bit each), and their positions
  attend   attention of such tokens over the pages: every row in front of the drafted ones, and the token's own path
  compact  rows of a list that stay, moved together inside the pages: an accepted path, or what the retention step chose
  copy     whole pages of both pools
  fork     lists that become copies of others (beams, several answers to a prompt) and get pages of their own for what follows
  step     pages that rejected tokens leave are given back, pages for the next ones are taken
"""
import math

import numpy as np
import torch

own = False


def _attend(name, dtype, batch, q_heads, kv_heads, d, new, length, page, **kw):
    """new: drafted tokens per sequence; ragged: fewer of them for most sequences (a padded batch); length: rows of the longest list
    behind the call, the drafted ones included; varied: shorter lists beside it; by_head: a list for every KV head, pages of one head."""
    c = dict(kind="attend", dtype=dtype, batch=batch, q_heads=q_heads, kv_heads=kv_heads, d=d, new=new, length=length, page=page, ragged=False,
             varied=False, by_head=False, pool_token_major=False, token_major=True)
    c.update(kw)
    return dict(c, name=name) if name else c


def _compact(name, dtype, batch, kv_heads, d, new, kept, length, page, **kw):
    """The last `new` rows of each list, of which up to `kept` stay; each_head: every KV head keeps rows of its own."""
    c = dict(kind="compact", dtype=dtype, batch=batch, kv_heads=kv_heads, d=d, new=new, kept=kept, length=length, page=page, each_head=False,
             varied=False, by_head=False, pool_token_major=False)
    c.update(kw)
    return dict(c, name=name) if name else c


def _copy(name, dtype, kv_heads, d, page, pairs, **kw):
    """skipped: one pair in so many names no page (a list that has nothing to copy), 0 none."""
    c = dict(kind="copy", dtype=dtype, kv_heads=kv_heads, d=d, page=page, pairs=pairs, skipped=0, pool_token_major=False)
    c.update(kw)
    return dict(c, name=name) if name else c


def _lists(name, kind, batch, kv_heads, length, page, new, **kw):
    """Lists of up to `length` rows, the first `common` per cent of their pages the same ones; new: rows to come."""
    c = dict(kind=kind, batch=batch, kv_heads=kv_heads, length=length, page=page, new=new, common=25, by_head=False)
    c.update(kw)
    return dict(c, name=name) if name else c


def _masks(name, batch, new):
    c = dict(kind="masks", batch=batch, new=new)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a step's trees of 24 drafted tokens, batch 16: the smallest, all latency
        _masks("masks_step_b16", 16, 24),
        # wide drafts of a large batch
        _masks("masks_b64_n1000", 64, 1000),
        # a layer's verification over the rows that retention kept, a list for every head
        _attend("tree_kept_b16", "bf16", 16, 32, 8, 128, 16, 560, 32, varied=True, by_head=True),
        # 60 drafted tokens over whole 32k prompts: the cache's bytes and the arithmetic weigh alike
        _attend("tree_32k_b4", "bf16", 4, 32, 8, 128, 60, 32768, 16),
        # f32, groups of seven heads, a padded batch of odd lengths
        _attend("tree_f32_ragged", "f32", 3, 14, 2, 64, 33, 1501, 16, ragged=True, varied=True, pool_token_major=True),
        # several hundred tokens, most of whose pairs among themselves are masked
        _attend("tree_500_b2", "bf16", 2, 32, 8, 128, 500, 4099, 64),
        # the accepted path of a step's trees, the same for all heads
        _compact("compact_path_b16", "bf16", 16, 8, 128, 60, 7, 20011, 16, varied=True),
        # the rows of 32k prompts that retention kept (nominal budget 512, chosen by head), in place
        _compact("compact_kept_32k", "bf16", 4, 8, 128, 32768, 544, 32768, 16, each_head=True),
        # a page for each of 32 lists that write into a shared one, every other pair empty
        _copy("copy_shared_b32", "bf16", 8, 128, 16, 32, skipped=2),
        # a cache's pages into another part of the pool
        _copy("copy_1000", "bf16", 8, 128, 64, 1000),
        # 32 beams of 32k rows reordered, each about to write a token
        _lists("fork_beams_b32", "fork", 32, 8, 32768, 16, 1),
        # a step of 64 sequences: surplus pages back, pages for 60 drafted tokens
        _lists("step_b64", "step", 64, 8, 9001, 16, 60),
    ]


# what bounds a drawn case: query-key pairs over all heads, values in the pools, entries of the lists
MOST_PAIRS = 4 * 32 * 60 * 32768
MOST_POOL = 4 * 8 * 32768 * 128
MOST_ENTRIES = 32 * 2048
MOST_MASK = 64 * 1000 * 1000


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["masks", "attend", "attend", "attend", "compact", "compact", "copy", "fork", "step"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    d = rng.choice([64, 128, 128])
    q_heads, kv_heads = rng.choice([(32, 8), (32, 32), (28, 4), (16, 2), (8, 1), (12, 4), (5, 5), (40, 8)])
    page = rng.choice([1, 8, 16, 16, 32, 64, 128, 256])
    while True:
        batch = _log_uniform(rng, 1, 64)
        length = _log_uniform(rng, 17, 65536)
        if kind == "masks":
            new = _log_uniform(rng, 1, 1024)
            if batch * new * new <= MOST_MASK:
                return _masks(None, batch, new)
        elif kind == "attend":
            new = 1 if rng.random() < 0.05 else _log_uniform(rng, 2, 512)
            length = max(length, new)
            if batch * q_heads * new * length * (4 if dtype == "f32" else 1) <= MOST_PAIRS and batch * kv_heads * length * d <= MOST_POOL:
                return _attend(None, dtype, batch, q_heads, kv_heads, d, new, length, page, ragged=rng.random() < 0.5, varied=rng.random() < 0.6,
                               by_head=rng.random() < 0.3, pool_token_major=rng.random() < 0.4, token_major=rng.random() < 0.7)
        elif kind == "compact":
            new = min(length, _log_uniform(rng, 2, 512)) if rng.random() < 0.5 else length
            if batch * kv_heads * length * d <= MOST_POOL:
                return _compact(None, dtype, batch, kv_heads, d, new, _log_uniform(rng, 1, new), length, page, each_head=new == length,
                                varied=new < length and rng.random() < 0.6, by_head=rng.random() < 0.3, pool_token_major=rng.random() < 0.4)
        elif kind == "copy":
            pairs = _log_uniform(rng, 1, 4096)
            if 2 * pairs * page * kv_heads * d <= MOST_POOL:
                return _copy(None, dtype, kv_heads, d, page, pairs, skipped=rng.choice([0, 0, 2, 5]), pool_token_major=rng.random() < 0.4)
        else:
            by_head, page = rng.random() < 0.3, max(page, 8)
            if batch * (kv_heads if by_head else 1) * (length // page + 1) <= MOST_ENTRIES:
                return _lists(None, kind, batch, kv_heads, length, page, _log_uniform(rng, 1, 256), common=rng.choice([0, 25, 90]), by_head=by_head)


# ---- inputs ---------------------------------------------------------------------------------------------------------------
def _vary(c, n):
    """[batch, kv_heads] numbers up to n: the same for a sequence's heads, or where heads have lists of their own different ones."""
    each = c["by_head"]
    i = np.arange(c["batch"] * c["kv_heads"]).reshape(c["batch"], -1) if each else np.arange(c["batch"])[:, None].repeat(c["kv_heads"], 1)
    return (n * (1.0 - (i * 37 % 89) / 120.0)).astype(np.int32)


def _counts(c):
    """[batch, kv_heads] new tokens of each sequence."""
    i = np.arange(c["batch"])[:, None].repeat(c["kv_heads"], 1) if c.get("ragged") else np.zeros((c["batch"], c["kv_heads"]), np.int64)
    return (c["new"] - (i * 41 % 97) * (c["new"] // 2) // 97).astype(np.int32)


def _lengths(c):
    """[batch, kv_heads] rows of each list, the new ones included."""
    counts, old = _counts(c), c["length"] - c["new"]
    return counts + (_vary(c, old) if c["varied"] else old)


def _type(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _pool(g, c, n_pages, one_head=False):
    heads = 1 if one_head else c["kv_heads"]
    shape = (n_pages, c["page"], heads, c["d"]) if c["pool_token_major"] else (n_pages, heads, c["page"], c["d"])
    x = torch.randn(shape, generator=g, device="cuda").to(_type(c))
    return (x.transpose(1, 2) if c["pool_token_major"] else x).expand(-1, c["kv_heads"], -1, -1)


def _paged(g, c, s):
    """The pools, the lists of page numbers (in no order, none twice) and the lengths."""
    lengths = _lengths(c)
    lists = lengths if c["by_head"] else lengths.max(1, keepdims=True)
    per_list = -(-lists // c["page"])
    n_pages, most = int(per_list.sum()) + 3, int(per_list.max())
    ids = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    first = np.concatenate([[0], np.cumsum(per_list.ravel())[:-1]]).reshape(per_list.shape)
    at = torch.from_numpy(first[..., None] + np.minimum(np.arange(most), per_list[..., None] - 1)).to("cuda")
    table = ids[at.long()]
    s["table"] = table.contiguous() if c["by_head"] else table[:, 0].contiguous()
    for name in ("k_pages", "v_pages"):
        s[name] = _pool(g, c, n_pages, c["by_head"])
    s["length"] = torch.from_numpy(lengths).to("cuda")


def _parents(g, batch, new):
    """A step's drafts: a few first tokens, each followed by some; a token's parent is one of those shortly before it."""
    i = torch.arange(new, device="cuda")
    back = 1 + (torch.rand(batch, new, generator=g, device="cuda") * max(1, new // 6)).long()
    return (i - back).clamp(min=-1).to(torch.int32)


def _prepare_lists(g, c, s):
    """Lists with common first pages, how many entries name each page, and what is to happen to them."""
    spare = -(-c["new"] // c["page"])
    rows = _vary(c, c["length"]) if c["by_head"] else _vary(c, c["length"])[:, :1]
    held = -(-rows // c["page"]) + (np.arange(rows.size).reshape(rows.shape) % (spare + 2) if c["kind"] == "step" else 0)
    most = int((-(-(rows + c["new"]) // c["page"])).max()) + spare + 2
    common = np.minimum(rows // c["page"], int(rows.min()) // c["page"] * c["common"] // 100)
    n_common = int(common.max())
    each = held - common
    first = n_common + np.concatenate([[0], np.cumsum(each.ravel())[:-1]]).reshape(each.shape)
    e = np.arange(most)
    at = np.where(e < common[..., None], e, np.where(e < held[..., None], first[..., None] + e - common[..., None], -1))
    used = n_common + int(each.sum())
    n_pages = used + rows.size * (spare + 2) + (int(held.sum()) if c["kind"] == "fork" else 0) // 4 + 7
    ids = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    at = torch.from_numpy(at).to("cuda")
    table = torch.where(at >= 0, ids[at.clamp(min=0)], -1).to(torch.int32)
    s["table"] = (table if c["by_head"] else table[:, 0]).contiguous()
    s["length"] = torch.from_numpy(np.broadcast_to(rows, (c["batch"], c["kv_heads"])).copy()).to("cuda")
    flat = s["table"].flatten()
    refs = torch.bincount(flat[flat >= 0].long(), minlength=n_pages)
    if c["kind"] == "fork":   # the lists of the step before, which the new ones take the place of
        before = torch.randint(0, c["batch"], (c["batch"],), generator=g, device="cuda")
        s["table_out"] = s["table"][before].contiguous()
        flat = s["table_out"].flatten()
        refs += torch.bincount(flat[flat >= 0].long(), minlength=n_pages)
        s["parent"] = torch.randint(0, c["batch"], (c["batch"],), generator=g, device="cuda").to(torch.int32)
        s["parent"][c["batch"] // 2 + 1::7] = -1   # answers that are complete
        s["length_out"] = torch.zeros_like(s["length"])
    s["refs"] = refs.to(torch.int32)
    s["taken"] = _bits(refs > 0)
    s["end"] = s["length"] + c["new"]
    s["copy"] = torch.zeros(rows.size * 2, 2, dtype=torch.int32, device="cuda")
    s["result"] = torch.zeros(2, dtype=torch.int32, device="cuda")
    s["n_pages"] = n_pages


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    kind = c["kind"]
    if kind in ("fork", "step"):
        _prepare_lists(g, c, s)
    elif kind == "copy":
        n = c["pairs"]
        ids = torch.randperm(2 * n + 3, generator=g, device="cuda").to(torch.int32)
        s["table"] = ids[None]   # of one list with every page
        s["copy"] = ids[:2 * n].view(n, 2).contiguous()
        if c["skipped"]:
            s["copy"][::c["skipped"]] = -1
        for name in ("k_pages", "v_pages"):
            s[name] = _pool(g, c, 2 * n + 3)
    elif kind == "masks":
        words = -(-c["new"] // 64)
        s["parent"] = _parents(g, c["batch"], c["new"])
        s["start"] = torch.randint(0, 131072, (c["batch"],), generator=g, device="cuda").to(torch.int32)
        s["sees"] = torch.zeros(c["batch"], c["new"], words, dtype=torch.int64, device="cuda")
        s["positions"] = torch.zeros(c["batch"], c["new"], dtype=torch.int32, device="cuda")
    else:
        _paged(g, c, s)
        s["count"] = torch.from_numpy(_counts(c)).to("cuda")
    if kind == "attend":
        shape = (c["batch"], c["new"], c["q_heads"], c["d"]) if c["token_major"] else (c["batch"], c["q_heads"], c["new"], c["d"])
        q = (torch.randn(shape, generator=g, device="cuda") * 2.0).to(_type(c))
        s["q"] = q.transpose(1, 2) if c["token_major"] else q
        s["sees"] = _words(_paths(_parents(g, c["batch"], c["new"])))
        s["out"] = torch.zeros(c["batch"], c["new"], c["q_heads"], c["d"], dtype=_type(c), device="cuda").transpose(1, 2)
        s["lse"] = torch.zeros(c["batch"], c["q_heads"], c["new"], device="cuda")
    elif kind == "compact":
        # ascending numbers among the last rows: the first ones of a path, or positions all over the prompt and its last rows
        n, kept = c["new"], c["kept"]
        lists = (c["batch"], c["kv_heads"]) if c["each_head"] else (c["batch"],)
        order = torch.rand(*lists, n, generator=g, device="cuda")
        if c["each_head"]:
            order[..., n - kept // 8:] += 1.0
        s["idx"] = order.topk(kept).indices.sort(-1).values.to(torch.int32)
        fewer = torch.randint(0, kept // 2 + 1, lists, generator=g, device="cuda")
        stay = (kept - fewer).to(torch.int32)
        s["kept"] = (stay if c["each_head"] else stay[:, None].expand(-1, c["kv_heads"])).contiguous()
        s["length_out"] = torch.zeros_like(s["length"])
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------------
def _bits(flags):
    """Truth values as words of 32 bits."""
    f = torch.nn.functional.pad(flags.long(), (0, -flags.numel() % 32)).view(-1, 32)
    x = (f << torch.arange(32, device="cuda")).sum(-1)
    return torch.where(x >= 1 << 31, x - (1 << 32), x).to(torch.int32)


def _words(paths):
    """[batch, n, n] truth values as words of 64 bits along the last axis."""
    f = torch.nn.functional.pad(paths.long(), (0, -paths.shape[-1] % 64)).unflatten(-1, (-1, 64))
    return (f << torch.arange(64, device="cuda")).sum(-1)


def _paths(parent):
    """[batch, n, n] whether token j is token i or on its way to the root: steps to the parent, then twice as many, and so on."""
    n = parent.shape[1]
    i = torch.arange(n, device="cuda")
    up = ((parent[..., None] == i) | (i[:, None] == i)).float()
    for _ in range(max(1, (n - 1).bit_length())):
        up = (torch.matmul(up, up) > 0).float()
    return up > 0


def _plain_masks(s):
    paths = _paths(s["parent"])
    s["sees"].copy_(_words(paths))
    s["positions"].copy_(s["start"][:, None] + paths.sum(-1).to(torch.int32) - 1)
    return {"sees": s["sees"], "positions": s["positions"]}


def _places(s, slot):
    """Page and row of `slot` [batch, kv_heads, ...] in the lists."""
    c, table = s["case"], s["table"]
    if table.dim() == 2:
        table = table[:, None].expand(-1, c["kv_heads"], -1)
    page = torch.gather(table, 2, (slot // c["page"]).flatten(2)).view(slot.shape)
    return page.long(), slot % c["page"]


def _plain_attend(s):
    c = s["case"]
    batch, Hkv, G, n, T = c["batch"], c["kv_heads"], c["q_heads"] // c["kv_heads"], c["new"], c["length"]
    j = torch.arange(T, device="cuda")
    there = j < s["length"][..., None]
    page, row = _places(s, torch.where(there, j, 0))
    head = torch.arange(Hkv, device="cuda")[None, :, None]
    k, v = (torch.where(there[..., None], s[m][page, head, row].float(), 0.0) for m in ("k_pages", "v_pages"))
    i = torch.arange(n, device="cuda")
    paths = ((s["sees"][..., None] >> torch.arange(64, device="cuda")) & 1).flatten(2)[..., :n] != 0   # [batch, n, n]
    paths &= i <= i[:, None]
    t = j - (s["length"] - s["count"])[..., None]   # [batch, Hkv, T] drafted token of the row
    drafted = (t >= 0) & (t < s["count"][..., None])
    at = t.clamp(0, n - 1)[:, :, None].expand(-1, -1, n, -1)
    sees = torch.gather(paths[:, None].expand(-1, Hkv, -1, -1), 3, at)
    sees = torch.where(drafted[:, :, None], sees, (t < 0)[:, :, None])
    q = s["q"].float().reshape(batch, Hkv, G * n, c["d"])
    z = torch.matmul(q, k.transpose(-1, -2).contiguous()).view(batch, Hkv, G, n, T) * (1.0 / math.sqrt(c["d"]))
    z = torch.where(sees[:, :, None], z, -math.inf)
    top = z.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    w = torch.exp(z - top)
    del z
    total = w.sum(-1, keepdim=True)
    out = torch.matmul(w.view(batch, Hkv, G * n, T), v).view(batch, Hkv, G, n, c["d"]) / torch.where(total == 0, 1.0, total)
    lse = (top + torch.log(total))[..., 0]
    here = (i < s["count"][..., None]).repeat_interleave(G, 1)
    s["out"].copy_(torch.where(here[..., None], out.reshape(batch, -1, n, c["d"]).to(s["out"].dtype), s["out"]))
    s["lse"].copy_(torch.where(here, lse.reshape(batch, -1, n), s["lse"]))
    return {"out": s["out"], "lse": s["lse"]}


def _moved(s):
    """The call's outputs of `compact`, whole."""
    return {**{m: s[m][:, :1] if s["case"]["by_head"] else s[m] for m in ("k_pages", "v_pages")}, "length_out": s["length_out"]}


def _plain_compact(s):
    c = s["case"]
    idx = s["idx"] if c["each_head"] else s["idx"][:, None].expand(-1, c["kv_heads"], -1)
    first = (s["length"] - s["count"])[..., None]
    r = torch.arange(c["kept"], device="cuda").expand(idx.shape)
    stays = r < s["kept"][..., None]
    page, row = _places(s, torch.where(stays, first + idx, 0).long())
    to_page, to_row = _places(s, torch.where(stays, first + r, 0).long())
    head = torch.zeros_like(page) if c["by_head"] else torch.arange(c["kv_heads"], device="cuda")[None, :, None].expand_as(page)
    for m in ("k_pages", "v_pages"):
        pool = s[m][:, :1] if c["by_head"] else s[m]
        rows = pool[page[stays], head[stays], row[stays]]
        pool[to_page[stays], head[stays], to_row[stays]] = rows
    s["length_out"].copy_(first[..., 0] + s["kept"])
    return _moved(s)


def _plain_copy(s):
    fine = s["copy"].min(-1).values >= 0
    src, dst = s["copy"][fine].long().unbind(-1)
    for m in ("k_pages", "v_pages"):
        s[m][dst] = s[m][src]
    return {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _named(table, n_pages):
    """How many entries name each page."""
    flat = table.flatten().long()
    nowhere = n_pages + torch.arange(flat.numel(), device="cuda")   # a place for each entry that names none
    one = torch.ones_like(flat, dtype=torch.int32)
    return torch.zeros(n_pages + flat.numel(), dtype=torch.int32, device="cuda").index_add_(0, torch.where(flat >= 0, flat, nowhere), one)[:n_pages]


def _plain_reserve(s, table, first, end):
    """Rows first .. end - 1 of each list get pages that no other entry names; nothing happens where the pages do not suffice."""
    c, n_pages = s["case"], s["n_pages"]
    if table.dim() == 2:
        first, end = first.amin(1), end.amax(1)
    e = torch.arange(table.shape[-1], device="cuda")
    asked = (e >= first[..., None] // c["page"]) & (e * c["page"] < end[..., None]) & (end > first)[..., None]
    flat, asked = table.flatten().long(), asked.flatten()
    there, order = flat >= 0, torch.arange(flat.numel(), device="cuda")
    nowhere, places = n_pages + order, n_pages + flat.numel()   # a place for each entry that takes no part
    refs = torch.where(there, s["refs"][flat.clamp(min=0)], 0)
    shared = asked & there & (refs > 1)
    at = torch.where(shared, flat, nowhere)
    wanted = torch.zeros(places, dtype=torch.int32, device="cuda").index_add_(0, at, shared.int())
    last = torch.zeros(places, dtype=torch.long, device="cuda").scatter_reduce_(0, at, order, "amax")
    leaves = shared & ~((wanted[at] >= refs) & (last[at] == order))   # where all who share a page write it, the last one keeps it
    need = asked & (~there | leaves)
    free = torch.argsort((s["refs"] > 0).int(), stable=True)
    missing = torch.maximum(need.sum() - (s["refs"] == 0).sum(), leaves.sum() - s["copy"].shape[0]).clamp(min=0)
    fine = missing == 0
    new = free[(need.cumsum(0) - 1).clamp(0, n_pages - 1)]
    need, leaves = need & fine, leaves & fine
    room = s["copy"].shape[0]
    pairs = torch.full((room + flat.numel(), 2), -1, dtype=torch.int32, device="cuda")
    pairs[torch.where(leaves, leaves.cumsum(0) - 1, room + order)] = torch.stack([flat, new], -1).int()
    s["copy"].copy_(pairs[:room])
    one = torch.ones_like(flat, dtype=torch.int32)
    refs = torch.nn.functional.pad(s["refs"], (0, flat.numel()))
    refs.index_add_(0, torch.where(leaves, flat, nowhere), -one).index_add_(0, torch.where(need, new, nowhere), one)
    s["refs"].copy_(refs[:n_pages])
    s["taken"].copy_(_bits(s["refs"] > 0))
    table.copy_(torch.where(need, new, flat).view(table.shape))
    s["result"].copy_(torch.stack([missing, leaves.sum()]))


def _plain_fork(s):
    parent, out = s["parent"].long(), s["table_out"]
    goes_on = parent >= 0
    new = torch.where(goes_on.view(-1, *[1] * (out.dim() - 1)), s["table"][parent.clamp(min=0)], -1)
    s["refs"] += _named(new, s["n_pages"]) - _named(out, s["n_pages"])
    s["taken"].copy_(_bits(s["refs"] > 0))
    out.copy_(new)
    s["length_out"].copy_(torch.where(goes_on[:, None], s["length"][parent.clamp(min=0)], 0))
    _plain_reserve(s, out, s["length_out"], s["length_out"] + s["case"]["new"])
    return _listed_state(s, out)


def _plain_step(s):
    c, table = s["case"], s["table"]
    keep = s["length"] if table.dim() == 3 else s["length"].amax(1)
    surplus = torch.arange(table.shape[-1], device="cuda") >= ((keep + c["page"] - 1) // c["page"])[..., None]
    s["refs"] -= _named(torch.where(surplus, table, -1), s["n_pages"])
    table.copy_(torch.where(surplus, -1, table))
    _plain_reserve(s, table, s["length"], s["end"])
    return _listed_state(s, table)


def _listed_state(s, table):
    got = {m: s[m] for m in ("refs", "taken", "copy", "result")}
    if "length_out" in s:
        got["length_out"] = s["length_out"]
    return dict(got, table=table)


# ---- the framework's calls ------------------------------------------------------------------------------------------------
def _handles(s):
    """What a serving program keeps over its steps: the descriptions of the call's tensors and of the pools, the workspace."""
    from paper_2602_08686_amd import binding as B

    c = s["case"]
    h = {"B": B}
    if c["kind"] in ("fork", "step"):
        h["lists"] = B.lists_for(s["table"], n_kv_heads=c["kv_heads"], n_pages=s["n_pages"], page_rows=c["page"])
    elif c["kind"] != "masks":
        h["pages"] = B.pages_for(s["k_pages"], s["v_pages"], s["table"])
        if c["kind"] != "attend":
            h["params"] = B.pool_params(s["k_pages"], s["table"])
        else:
            h["params"] = B.step_params(q=s["q"], n_q_heads=c["q_heads"], n_kv_heads=c["kv_heads"])
            need = B.ckv_paged_workspace_bytes(h["params"], c["length"])
            h["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    s["handles"] = h
    return h


def run(state):
    s, kind = state, state["case"]["kind"]
    if not own:
        return {"masks": _plain_masks, "attend": _plain_attend, "compact": _plain_compact, "copy": _plain_copy, "fork": _plain_fork,
                "step": _plain_step}[kind](s)
    h = s.get("handles") or _handles(s)
    B = h["B"]
    if kind == "masks":
        B.ckv_tree_sees(s["parent"], s["start"], s["sees"], s["positions"])
        return {"sees": s["sees"], "positions": s["positions"]}
    if kind == "attend":
        B.ckv_paged_tree_attention(h["params"], h["pages"], s["q"], s["k_pages"], s["v_pages"], s["table"], s["length"], s["case"]["length"],
                                   s["sees"], s["out"], s["lse"], h["workspace"], count=s["count"])
        return {"out": s["out"], "lse": s["lse"]}
    if kind == "compact":
        B.ckv_paged_compact(h["params"], h["pages"], s["k_pages"], s["v_pages"], s["table"], s["length"], s["idx"], s["kept"], s["length_out"],
                            count=s["count"])
        return _moved(s)
    if kind == "copy":
        B.ckv_pages_copy(h["params"], h["pages"], s["k_pages"], s["v_pages"], s["copy"])
        return {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    if kind == "fork":
        B.ckv_pages_fork(h["lists"], s["table"], s["parent"], s["table_out"], s["refs"], s["taken"], s["length"], s["length_out"])
        B.ckv_pages_reserve(h["lists"], s["table_out"], s["length_out"], s["length_out"] + s["case"]["new"], s["refs"], s["taken"], s["copy"],
                            s["result"])
        return _listed_state(s, s["table_out"])
    B.ckv_pages_free(h["lists"], s["table"], s["length"], s["refs"], s["taken"])
    B.ckv_pages_reserve(h["lists"], s["table"], s["length"], s["end"], s["refs"], s["taken"], s["copy"], s["result"])
    return _listed_state(s, s["table"])


def work(case):
    """Every input byte that the results depend on read once, every output byte written once; two products for every drafted token and
    row in front of the drafts, and for the token itself."""
    c, kind = case, case["kind"]
    if kind == "masks":
        return {"bytes": c["batch"] * (c["new"] * (8 * -(-c["new"] // 64) + 8) + 4), "flops": 0.0}
    if kind in ("fork", "step"):
        lists = c["batch"] * (c["kv_heads"] if c["by_head"] else 1)
        new = c["new"] // c["page"] + 1
        if kind == "step":   # the last entries of each list and what is known of the free pages
            return {"bytes": float(lists * (4 * new * 4 + 8)), "flops": 0.0}
        return {"bytes": float(lists * (4 * 4 * (0.63 * c["length"] / c["page"] + new) + 12)), "flops": 0.0}   # lists read, written, two counts an entry
    e = 4 if c["dtype"] == "f32" else 2
    if kind == "copy":
        pairs = c["pairs"] - (-(-c["pairs"] // c["skipped"]) if c["skipped"] else 0)
        return {"bytes": 4.0 * max(pairs, 0.01) * c["page"] * c["kv_heads"] * c["d"] * e + 8 * c["pairs"], "flops": 0.0}
    if kind == "compact":
        rows = c["batch"] * c["kv_heads"] * (c["kept"] - c["kept"] // 4)
        return {"bytes": 4.0 * rows * c["d"] * e + 4 * rows, "flops": 0.0}
    G, d = c["q_heads"] // c["kv_heads"], c["d"]
    counts, lengths = _counts(c).astype(np.float64), _lengths(c).astype(np.float64)
    pairs = G * (counts * (lengths - counts) + counts).sum()
    lists = lengths.size if c["by_head"] else c["batch"]
    table = 4.0 * lists * lengths.mean() / c["page"]
    mask = 8.0 * c["batch"] * c["new"] * -(-c["new"] // 64)
    return {"bytes": 2 * lengths.sum() * d * e + counts.sum() * G * (2 * d * e + 4) + table + mask + 4 * lengths.size, "flops": 4.0 * d * pairs}


# ---- 64 bits --------------------------------------------------------------------------------------------------------------
def _exact_masks(c, s):
    parent, start, n = s["parent"].tolist(), s["start"].tolist(), c["new"]
    words = -(-n // 64)
    sees, positions = np.zeros((c["batch"], n, words), np.uint64), np.zeros((c["batch"], n), np.int64)
    for b in range(c["batch"]):
        rows = []
        for i in range(n):
            rows.append((rows[parent[b][i]] if parent[b][i] >= 0 else 0) | 1 << i)
            sees[b, i] = np.frombuffer(rows[i].to_bytes(8 * words, "little"), np.uint64)
            positions[b, i] = start[b] + bin(rows[i]).count("1") - 1
    return {"sees": sees.view(np.int64), "positions": positions}


def _exact_rows(c, s, b, g, rows):
    """Pages, the pool's head and rows in the pages of the list's rows (a numpy array)."""
    table = s["table"].cpu().numpy()
    ids = (table[b, g] if c["by_head"] else table[b])[rows // c["page"]]
    return torch.from_numpy(ids).long().cuda(), 0 if c["by_head"] else g, torch.from_numpy(rows % c["page"]).cuda()


def _exact_attend(c, s):
    counts, lengths, G, n = _counts(c), _lengths(c), c["q_heads"] // c["kv_heads"], c["new"]
    words = s["sees"].cpu().numpy().view(np.uint64)
    out = torch.zeros(c["batch"], c["q_heads"], n, c["d"], dtype=torch.float64, device="cuda")
    lse = torch.zeros(c["batch"], c["q_heads"], n, dtype=torch.float64, device="cuda")
    for b in range(c["batch"]):
        bits = np.unpackbits(words[b].view(np.uint8), axis=1, bitorder="little")[:, :n] != 0
        for g in range(c["kv_heads"]):
            m, T = int(counts[b, g]), int(lengths[b, g])
            at = _exact_rows(c, s, b, g, np.arange(T))
            k, v = s["k_pages"][at].double(), s["v_pages"][at].double()
            hidden = np.concatenate([np.zeros((m, T - m), bool), ~np.tril(bits[:m, :m])], 1)
            hidden = torch.from_numpy(hidden).cuda()
            for h in range(g * G, (g + 1) * G):
                z = (s["q"][b, h, :m].double() @ k.t()).div_(math.sqrt(c["d"])).masked_fill_(hidden, -math.inf)
                lse[b, h, :m] = torch.logsumexp(z, 1)
                out[b, h, :m] = torch.softmax(z, 1) @ v
    return {"out": out, "lse": lse}


def _exact_compact(c, s):
    counts, lengths, kept, idx = _counts(c), _lengths(c), s["kept"].cpu().numpy(), s["idx"].cpu().numpy()
    got = {m: (s[m][:, :1] if c["by_head"] else s[m]).double() for m in ("k_pages", "v_pages")}
    for b in range(c["batch"]):
        for g in range(c["kv_heads"]):
            first, m = int(lengths[b, g] - counts[b, g]), int(kept[b, g])
            chosen = (idx[b, g] if c["each_head"] else idx[b])[:m].astype(np.int64)
            src, dst = _exact_rows(c, s, b, g, first + chosen), _exact_rows(c, s, b, g, first + np.arange(m))
            for name, pool in got.items():
                pool[dst] = s[name][src].double()
    return dict(got, length_out=torch.from_numpy(lengths - counts + kept))


def _exact_lists(c, s):
    """Lists, counts and free pages, an entry after the other."""
    lists = (s["table_out"] if c["kind"] == "fork" else s["table"]).cpu().numpy()
    shape, refs, rows = lists.shape, s["refs"].tolist(), s["length"].cpu().numpy()
    lists = lists.reshape(c["batch"], -1, shape[-1]).tolist()
    if c["kind"] == "fork":
        old, parent = s["table"].cpu().numpy().reshape(c["batch"], -1, shape[-1]).tolist(), s["parent"].tolist()
        for b in range(c["batch"]):
            for g, entries in enumerate(lists[b]):
                for p in entries:
                    refs[p] -= p >= 0
                lists[b][g] = list(old[parent[b]][g]) if parent[b] >= 0 else [-1] * shape[-1]
                for p in lists[b][g]:
                    refs[p] += p >= 0
        rows = np.array([rows[p] if p >= 0 else 0 * rows[0] for p in parent])
    ranges = []
    for b in range(c["batch"]):
        for g, entries in enumerate(lists[b]):
            first = int(rows[b, g])
            if c["kind"] == "step":
                for e in range(-(-first // c["page"]), shape[-1]):
                    refs[entries[e]] -= entries[e] >= 0
                    entries[e] = -1
            ranges += [(b, g, e) for e in range(first // c["page"], min(-(-(first + c["new"]) // c["page"]), shape[-1]))]
    wanted = {}
    for b, g, e in ranges:
        p = lists[b][g][e]
        if p >= 0 and refs[p] > 1:
            wanted.setdefault(p, []).append((b, g, e))
    leaves = {x for p, who in wanted.items() for x in (who[:-1] if len(who) >= refs[p] else who)}
    need = [x for x in ranges if x in leaves or lists[x[0]][x[1]][x[2]] < 0]
    free = [p for p, r in enumerate(refs) if r == 0]
    room = s["copy"].shape[0]
    missing = max(len(need) - len(free), len(leaves) - room, 0)
    copy = []
    if not missing:
        for (b, g, e), p in zip(need, free):
            before = lists[b][g][e]
            if before >= 0:
                copy.append((before, p))
                refs[before] -= 1
            refs[p] = 1
            lists[b][g][e] = p
    held = np.array(refs) > 0
    taken = np.packbits(np.pad(held, (0, -held.size % 32)), bitorder="little").view(np.int32)
    got = {"table": np.array(lists, np.int64).reshape(shape), "refs": np.array(refs, np.int64), "taken": taken.astype(np.int64),
           "copy": np.array(copy + [(-1, -1)] * (room - len(copy)), np.int64), "result": np.array([missing, len(copy)])}
    return dict(got, length_out=rows.astype(np.int64)) if c["kind"] == "fork" else got


def exact(case, seed):
    c, kind = case, case["kind"]
    if kind in ("attend", "compact") and c["batch"] * c["kv_heads"] > 600:
        return None   # a list at a time takes too long
    s = prepare(c, seed)
    if kind == "copy":
        got = {m: s[m].double() for m in ("k_pages", "v_pages")}
        for src, dst in s["copy"].tolist():
            if src >= 0:
                for m, pool in got.items():
                    pool[dst] = s[m][src].double()
        return got
    return {"masks": _exact_masks, "attend": _exact_attend, "compact": _exact_compact}.get(kind, _exact_lists)(c, s)
