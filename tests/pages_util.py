"""Trees of drafted tokens, rows and pages that move, lists that share pages: cases and their results (numpy, from the definitions in include/ckv.h),
shared by the tests on the host CPU and on the GPU. Tolerances of attention are paged_util's, whose derivation does not depend on which rows a token
sees; everything else is whole numbers or bit copies."""
import pathlib
import subprocess

import numpy as np

import cpu_build as cpu
import paged_util as u


# ---- the library for the host CPU -------------------------------------------------------------------------------------------
def build_cpu(where):
    """As cpu_build.build, with the sources under test here."""
    objs, procs = [], []
    csrc = cpu.ROOT / "paper_2602_08686_amd" / "csrc"
    names = ("ckv_api", "ckv_rows", "ckv_paged", "ckv_paged_rows", "ckv_paged_tree", "ckv_tree", "ckv_moves", "ckv_lists")
    for src in [csrc / (n + ".hip") for n in names] + [cpu.HERE / "emulator.cpp"]:
        objs.append(str(pathlib.Path(where) / (src.name + ".o")))
        procs.append(subprocess.Popen([cpu.CXX, "-x", "c++", "-std=c++17", "-O1", "-fPIC", "-w", "-fsanitize=bounds", "-fsanitize-trap=bounds",
                                       f"-I{cpu.HERE}", f"-I{cpu.ROOT / 'include'}", f"-I{csrc}", "-c", str(src), "-o", objs[-1]]))
    assert [p.wait() for p in procs] == [0] * len(procs)
    lib = str(pathlib.Path(where) / "libckv_pages_cpu.so")
    subprocess.run([cpu.CXX, "-shared", "-fPIC", *objs, "-o", lib], check=True)
    return lib


# ---- trees ------------------------------------------------------------------------------------------------------------------
def parents(kind, batch, n, seed=0):
    rng, i = np.random.default_rng(seed + n), np.arange(n)
    if kind == "chain":
        p = np.tile(i - 1, (batch, 1))
    elif kind == "star":      # all follow the first
        p = np.tile(np.where(i > 0, 0, -1), (batch, 1))
    elif kind == "roots":
        p = np.full((batch, n), -1)
    elif kind == "odd":       # values that are no earlier token make a root
        p = rng.integers(-3, n + 3, (batch, n))
        p[:, ::5] = np.resize([2 ** 31 - 1, -2 ** 31, n], p[:, ::5].shape)
    else:
        p = i - 1 - (rng.random((batch, n)) * max(1, n // 6)).astype(int)
    return p.astype(np.int32)


def paths(parent):
    """[batch, n, n] whether token i sees token j, and the depth."""
    batch, n = parent.shape
    sees = np.zeros((batch, n, n), bool)
    for b, i in np.ndindex(batch, n):
        if 0 <= parent[b, i] < i:
            sees[b, i] = sees[b, parent[b, i]]
        sees[b, i, i] = True
    return sees, sees.sum(-1) - 1


def words(sees):
    """Truth values [..., n] as [..., ceil(n/64)] words."""
    pad = -sees.shape[-1] % 64
    bits = np.concatenate([sees, np.zeros(sees.shape[:-1] + (pad,), bool)], -1)
    return np.ascontiguousarray(np.packbits(bits, axis=-1, bitorder="little")).view(np.int64)


def tree_case(kind="random", **kw):
    c = u.case(**kw)
    sees, _ = paths(parents(kind if kind not in ("empty", "noise") else "random", c["batch"], c["n"], seed=c["seed"]))
    rng = np.random.default_rng(c["n"])
    if kind == "empty":      # some tokens without a bit, their own among them
        sees[:, ::3] = False
    elif kind == "noise":    # any words: bits of later tokens are not looked at
        sees = rng.random(sees.shape) < 0.4
    return dict(c, sees=sees)


def attention(c, s):
    """out, its tolerance, lse, its tolerance; rows that are not the call's are NaN."""
    n, G, d = u.new_counts(c), c["Hq"] // c["Hkv"], c["d"]
    scale = float(np.float32(c["scale"])) or 1.0 / np.sqrt(d)
    n_rows = c["n_rows"] or s["table"].shape[-1] * c["page"]
    shape = (c["batch"], c["Hq"], c["n"])
    out, out_tol = np.full(shape + (d,), np.nan), np.zeros(shape + (d,))
    lse, lse_tol = np.full(shape, np.nan), np.zeros(shape)
    half = u.H8 if c["dtype"] == "bf16" else 0.0
    for b, g in np.ndindex(n.shape):
        length, count, h0 = max(int(c["lengths"][b, g]), 0), int(n[b, g]), 0 if c["by_head"] else g
        rows = [u.place(c, s, b, g, j) for j in range(min(length, n_rows))]
        there = np.array([r is not None for r in rows], bool)
        at = np.array([r if r is not None else (0, 0) for r in rows], int).reshape(-1, 2)
        k, v = (u.values(s[m][at[:, 0], h0, at[:, 1]]).astype(np.float64) for m in ("k_pages", "v_pages"))
        t = np.arange(len(rows)) - (length - count)   # new token of a row
        for i in range(count):
            seen = there & ((t < 0) | ((t <= i) & c["sees"][b, i, np.clip(t, 0, c["n"] - 1)]))
            kk, vv = k[seen], v[seen]
            for h in range(g * G, (g + 1) * G):
                if not seen.any():
                    out[b, h, i], lse[b, h, i] = 0.0, -np.inf
                    continue
                q = u.values(s["q"])[b, h, i].astype(np.float64)
                with np.errstate(invalid="ignore", over="ignore"):
                    z = scale * (kk @ q)
                    top = z.max()
                    w = np.exp(z - top)
                    lse[b, h, i] = top + np.log(w.sum())
                    w /= w.sum()
                    out[b, h, i] = (w[:, None] * vv).sum(0)
                    e = (d + 4) * u.H24 * scale * (np.abs(kk) @ np.abs(q)).max()
                    size = (w[:, None] * np.abs(vv)).sum(0)
                    lse_tol[b, h, i] = e + (len(z) + 16) * u.H24 + 2 * u.H24 * abs(lse[b, h, i])
                    out_tol[b, h, i] = (2 * e + (len(z) + 16) * 2 * u.H24 + half) * size + (half or u.H24) * np.abs(out[b, h, i])
    return out, out_tol, lse, lse_tol


def fine(c):
    """A bf16 case, its results and the bound on them with weights that are off by 2^-16 of themselves at most (two bf16 terms: each is off by 2^-8 of what
    it stands for), in place of one rounding to bf16: attention()'s without its 2^-8 of sum_j w_j |v_j|."""
    s = u.make(c)
    want, tol, lse, lse_tol = attention(c, s)
    plain = dict(s, v_pages=u.stored(np.abs(u.values(np.ascontiguousarray(s["v_pages"]))), c["dtype"]))
    size = np.nan_to_num(attention(c, plain)[0])   # sum_j w_j |v_j|; no rows of the call: 0
    return s, want, tol - (u.H8 - 2.0 ** -16) * size, lse, lse_tol


TREES = [
    tree_case(n=1, lengths=((1, 1), (2, 70), (0, 5))),
    tree_case(n=16, heads=(8, 2), lengths=((90, 60), (16, 17)), by_head=True, page=32),
    tree_case("chain", n=5, heads=(7, 1), lengths=((333,), (5,), (3,)), page=8),                  # the last: fewer rows than tokens
    tree_case("star", n=64, heads=(1, 1), lengths=((64,), (100,)), counts=((64,), (33,)), page=16),  # two tiles of few columns
    tree_case(n=33, heads=(14, 2), d=64, lengths=((100, 100), (45, 45)), counts=((33, 33), (12, 12)), page=16),
    tree_case(n=70, heads=(8, 2), lengths=((70, 70), (300, 290)), counts=((70, 70), (33, 33)), pool_token_major=True),
    tree_case("roots", n=40, heads=(4, 1), lengths=((40,),), page=1),                              # a token sees itself alone
    tree_case("empty", n=20, heads=(2, 1), lengths=((20,), (90,)), page=16),                       # rows that see nothing
    tree_case("empty", n=130, heads=(3, 1), d=64, lengths=((130,), (500,)), page=64),
    tree_case("noise", n=140, heads=(3, 1), d=64, lengths=((200,),), page=128, token_major=False),
    tree_case("noise", n=30, heads=(2, 1), lengths=((100,),), page=16),
    tree_case(n=30, heads=(2, 2), d=64, lengths=((1500, 300),), by_head=True, page=32, n_rows=1400),  # a bound below the length
    tree_case(dtype="f32", n=9, heads=(2, 1), lengths=((200,), (64,)), counts=((9,), (2,)), page=16, scale=0.2),
    tree_case("noise", dtype="f32", n=100, heads=(4, 2), d=64, lengths=((180, 180),), counts=((100, 100),), page=4),   # eight words of few columns' tiles
    tree_case("empty", dtype="f32", n=256, heads=(1, 1), d=64, lengths=((300,),), page=16),
    tree_case(dtype="f32", n=260, heads=(1, 1), d=64, lengths=((270,),), page=16),
    tree_case("noise", dtype="f32", n=140, heads=(2, 1), lengths=((170,),), page=32),
    tree_case(n=3, heads=(4, 1), lengths=((2500,),), page=16),                                      # chunks joined in the launch
    tree_case(n=12, heads=(4, 1), lengths=((1203,),), counts=((11,),), page=16),                    # chunks and a merge
    tree_case("chain", n=257, heads=(2, 1), lengths=((1400,), (257,)), page=16),                    # tiles, chunks along the rows
]

# Those that reach the kernels' other instances, on the GPU: eight waves where the tiles fill the chip or the rows are more than the caches hold.
MANY = [
    tree_case(n=24, heads=(32, 8), lengths=((544, 300, 60, 33, 100, 544, 31, 32),) * 3, by_head=True, page=32),
    tree_case(n=60, heads=(8, 2), lengths=((5000, 5000), (3003, 3003)), page=16),
    tree_case("noise", n=25, heads=(7, 1), lengths=((9001,), (40,), (2000,)), counts=((25,), (13,), (25,)), page=16, pool_token_major=True),
    tree_case("empty", n=300, heads=(4, 1), lengths=((1000,), (300,)), page=64),
    tree_case(n=257, heads=(32, 32), lengths=tuple((257 + 100 * b,) * 32 for b in range(4)), page=16),
    tree_case("noise", n=600, heads=(2, 1), d=64, lengths=((2000,),), counts=((590,),), page=128),
    tree_case("noise", dtype="f32", n=300, heads=(4, 1), lengths=((1100,),), page=16),
    tree_case("empty", dtype="f32", n=64, heads=(4, 1), lengths=((3000,), (70,)), page=8),
    tree_case(dtype="f32", d=64, n=8, heads=(4, 2), lengths=((100, 37),), by_head=True, page=16),
    tree_case("noise", d=64, n=20, heads=(2, 1), lengths=((333,), (21,)), page=4),
    tree_case("noise", d=64, n=257, heads=(32, 32), lengths=tuple((257 + 60 * b,) * 32 for b in range(4)), page=32),
    tree_case(dtype="f32", n=257, heads=(32, 32), lengths=tuple((257 + 40 * b,) * 32 for b in range(4)), page=32),
    tree_case("empty", dtype="f32", d=64, n=257, heads=(32, 32), lengths=((257,) * 32, (300,) * 32, (20,) * 32, (257,) * 32),
              counts=((257,) * 32, (257,) * 32, (257,) * 32, (3,) * 32), page=16),
]


# ---- rows that move ---------------------------------------------------------------------------------------------------------
def chosen(c, cap, kept, each_head, seed=0):
    """idx [batch, (Hkv,) cap] ascending among the last rows, kept [batch, Hkv]; places behind a list's numbers hold what must not be read."""
    rng = np.random.default_rng(seed + cap)
    counts = np.maximum(c["lengths"], 0) if c["counts"] is None else np.clip(c["counts"], 0, np.maximum(c["lengths"], 0))
    lists = counts if each_head else counts.min(1, keepdims=True)
    idx = np.full(lists.shape + (cap,), -2 ** 31, np.int32)
    stay = np.zeros(lists.shape, np.int32)
    for at in np.ndindex(lists.shape):
        m = min(int(kept), int(lists[at]), cap)
        idx[at][:m] = np.sort(rng.permutation(int(lists[at]))[:m])
        stay[at] = m
    return (idx if each_head else idx[:, 0]), np.array(np.broadcast_to(stay, counts.shape))


def compacted(c, s, idx, kept):
    """Pools (as stored) and length_out."""
    lengths = np.maximum(c["lengths"], 0)
    counts = lengths if c["counts"] is None else np.clip(c["counts"], 0, lengths)
    pools = {m: np.array(s[m]) for m in ("k_pages", "v_pages")}
    out = np.zeros_like(lengths)
    cap = idx.shape[-1]
    for b, g in np.ndindex(lengths.shape):
        mine, first = (idx[b, g] if idx.ndim == 3 else idx[b]), int(lengths[b, g] - counts[b, g])
        m = min(max(int(kept[b, g]), 0), int(counts[b, g]), cap)
        out[b, g] = first + m
        for r in range(m):
            if not 0 <= mine[r] < counts[b, g]:
                continue
            src, dst = u.place(c, s, b, g, first + int(mine[r])), u.place(c, s, b, g, first + r)
            if src is not None and dst is not None:
                h = 0 if c["by_head"] else g
                for name, pool in pools.items():
                    pool[dst[0], h, dst[1]] = s[name][src[0], h, src[1]]
    return pools, out


# (case, cap, kept, each_head)
MOVES = [
    (u.case(n=1, lengths=((200, 200), (77, 77)), counts=((60, 60), (24, 24)), page=16), 7, 7, False),        # an accepted path
    (u.case(n=1, lengths=((90, 90), (5, 5), (0, 0)), counts=((0, 0), (5, 5), (3, 3)), page=8), 6, 4, False),   # nothing new; a short list; none
    (u.case(n=1, heads=(4, 4), lengths=((300, 200, 1, 33),), by_head=True, page=32), 150, 140, True),         # rows chosen by head
    (u.case(n=1, heads=(2, 2), lengths=((700, 700), (650, 650)), page=64, pool_token_major=True), 300, 290, True),
    (u.case(n=1, heads=(1, 1), d=64, lengths=((1900,),), page=1), 1800, 1790, True),                           # nearly all: several rounds
    (u.case(dtype="f32", n=1, heads=(3, 3), lengths=((600, 600, 600),), page=128), 599, 500, True),
    (u.case(dtype="f32", n=1, heads=(2, 2), d=64, lengths=((40, 40), (9, 9)), counts=((20, 20), (9, 9)), page=4), 64, 20, False),
    (u.case(n=1, heads=(2, 1), lengths=((1000,),), page=16), 1000, 1000, True),                                # all rows stay
    (u.case(n=1, heads=(2, 1), lengths=((100,),), page=16), 1, 1, True),
]


# ---- lists ------------------------------------------------------------------------------------------------------------------
class Lists:
    """Lists, counts and free pages, an entry after the other."""

    def __init__(self, tables, n_pages, page):
        """tables: every table whose entries the counts hold, as [batch, heads, max_pages]."""
        self.n_pages, self.page, self.refs = n_pages, page, np.zeros(n_pages, np.int32)
        for t in tables:
            for p in t.ravel():
                self.hold(p)

    def there(self, p):
        return 0 <= p < self.n_pages

    def hold(self, p):
        if self.there(p):
            self.refs[p] += 1

    def drop(self, p):
        if self.there(p):
            self.refs[p] -= 1

    def taken(self):
        held = np.concatenate([self.refs > 0, np.zeros(-self.n_pages % 32, bool)])
        return np.packbits(held, bitorder="little").view(np.int32)

    def fork(self, table, parent, out):
        for b in range(len(out)):
            for g in range(out.shape[1]):
                for e in range(out.shape[2]):
                    self.drop(out[b, g, e])
        for b in range(len(out)):
            alive = 0 <= parent[b] < len(table)
            out[b] = table[parent[b]] if alive else -1
            out[b][(out[b] < 0) | (out[b] >= self.n_pages)] = -1
            for p in out[b].ravel():
                self.hold(p)

    def free(self, table, keep):
        batch, heads, most = table.shape
        for b, h in np.ndindex(batch, heads):
            rows = 0 if keep is None else max(0, int(keep[b, h] if heads > 1 else keep[b].max()))
            for e in range(-(-rows // self.page), most):
                self.drop(table[b, h, e])
                table[b, h, e] = -1

    def reserve(self, table, first, end, n_copy):
        """(copy, result)"""
        batch, heads, most = table.shape
        asked = []
        for b, h in np.ndindex(batch, heads):
            ranges = [(max(int(first[b, g]), 0), int(end[b, g])) for g in ([h] if heads > 1 else range(first.shape[1]))]
            ranges = [r for r in ranges if r[1] > r[0]]
            if ranges:
                f, e = min(r[0] for r in ranges), max(r[1] for r in ranges)
                asked += [(b, h, i) for i in range(f // self.page, min(-(-e // self.page), most))]
        who = {}
        for at in asked:
            if self.there(table[at]) and self.refs[table[at]] > 1:
                who.setdefault(int(table[at]), []).append(at)
        leave = {at for p, all_ in who.items() for at in (all_[:-1] if len(all_) == self.refs[p] else all_)}
        need = [at for at in asked if at in leave or not self.there(table[at])]
        free = np.flatnonzero(self.refs == 0)
        copy = np.full((n_copy, 2), -1, np.int32)
        missing = max(len(need) - len(free), len(leave) - n_copy, 0)
        if missing:
            return copy, np.array([missing, 0], np.int32)
        pair = 0
        for at, p in zip(need, free):
            if at in leave:
                copy[pair] = table[at], p
                pair += 1
                self.drop(table[at])
            table[at] = p
            self.hold(p)
        return copy, np.array([0, pair], np.int32)


def list_case(batch=3, heads=1, Hkv=2, page=16, most=6, n_pages=60, lengths=None, common=1, seed=0, bad=False):
    """Lists of pages, the first `common` of which all lists share, and rows that they hold [batch, Hkv]."""
    rng = np.random.default_rng(seed + batch)
    if lengths is None:
        lengths = rng.integers(0, (most - 1) * page + 1, (batch, Hkv))
    lengths = np.array(lengths, np.int32)
    rows = lengths if heads > 1 else lengths.max(1, keepdims=True)
    ids, at = rng.permutation(n_pages), common
    table = np.full((batch, heads, most), -1, np.int32)
    for b, h in np.ndindex(batch, heads):
        held = -(-int(rows[b, h]) // page)
        own = max(0, held - common)
        table[b, h, :min(common, held)] = ids[:min(common, held)]
        table[b, h, common:common + own] = ids[at:at + own]
        at += own
    if bad:
        table[0, 0, -1], table[-1, -1, -1] = n_pages + 5, -7
    return dict(batch=batch, heads=heads, Hkv=Hkv, page=page, most=most, n_pages=n_pages, lengths=lengths, table=table)


LISTS = [
    list_case(),
    list_case(batch=1, Hkv=1, most=1, n_pages=1, lengths=[[0]], common=0),
    list_case(batch=5, heads=3, Hkv=3, page=4, most=9, n_pages=200, seed=3),
    list_case(batch=4, Hkv=1, page=1, most=300, n_pages=1300, seed=4, common=0),
    list_case(batch=2, Hkv=4, page=64, most=700, n_pages=1500, seed=5, common=100, bad=True),
    list_case(batch=300, heads=4, Hkv=4, page=8, most=3, n_pages=4001, seed=6, common=1),     # more lists than threads
    list_case(batch=2, Hkv=2, page=2, most=1500, n_pages=40000, seed=7, common=0, lengths=[[3, 3], [2500, 2500]]),
]
