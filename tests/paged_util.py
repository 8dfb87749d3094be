"""Cases of the paged cache's calls and their results in 64 bits (numpy, from the definitions in include/ckv.h), shared by the tests on
the host CPU and on the GPU.

Tolerances, from the arithmetic: a rounding to bf16 is off by 2^-8 of the value at most, to fp32 by 2^-24.
  rows       sums of d squares, a root, a quotient, two products and a sum: (d + 16) 2^-24 of the pair's length and a turn's rounding
             (2^-24 turns: 2 pi 2^-24 of it); in bf16 one rounding more, 2^-8 of the value
  logits     d products summed: (d + 4) 2^-24 of scale * sum |q_c k_c|, call it e of the row; lse: e + (rows + 16) 2^-24 + 2^-23 |lse|
             (the exponential's unit, the sum's additions)
  out        with A = sum_j w_j |v_j|: weights off by 2 e + (rows + 16) 2^-23 of themselves, in bf16 by 2^-8 more (their rounding)
             and the output's rounding, 2^-8 of it (2^-24 in f32)"""
import ctypes

import numpy as np

from paper_2602_08686_amd import binding as B

H8, H24 = 2.0 ** -8, 2.0 ** -24


def to_bf16(x):
    """fp32 -> bf16 bits, to the nearest, ties to even (finite values and infinities; NaN stays one)."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32)
    r = ((u + 0x7fff + ((u >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where(np.isnan(x), np.uint16(0x7fc0), r)


def from_bf16(b):
    return (b.astype(np.uint32) << 16).view(np.float32)


def stored(x, dtype):
    """The array as it is kept: bits of bf16 (uint16), or fp32."""
    return to_bf16(x) if dtype == "bf16" else np.ascontiguousarray(x, np.float32)


def values(x):
    return from_bf16(x) if x.dtype == np.uint16 else x


def case(dtype="bf16", d=128, heads=(8, 2), n=1, lengths=((40, 40),), counts=None, page=16, by_head=False, token_major=True,
         pool_token_major=False, norm=False, rot_dim=0, pairing=B.PAIR_HALVES, spare=2, seed=0, scale=0.0, n_rows=None):
    lengths = np.array(lengths, np.int32)
    return dict(dtype=dtype, d=d, Hq=heads[0], Hkv=heads[1], n=n, lengths=lengths, batch=len(lengths), page=page, by_head=by_head,
                counts=None if counts is None else np.array(counts, np.int32), token_major=token_major, pool_token_major=pool_token_major,
                norm=norm, rot_dim=rot_dim, pairing=pairing, spare=spare, seed=seed, scale=scale, n_rows=n_rows)


def new_counts(c):
    full = np.full((c["batch"], c["Hkv"]), c["n"], np.int32)
    return full if c["counts"] is None else np.clip(c["counts"], 0, c["n"])


def rows_of(rng, c, heads, scale=1.0):
    """Logical [batch, heads, n, d] view of an array that lies token by token or head by head."""
    shape = (c["batch"], c["n"], heads, c["d"]) if c["token_major"] else (c["batch"], heads, c["n"], c["d"])
    x = stored(scale * rng.standard_normal(shape, dtype=np.float32), c["dtype"])
    return x.transpose(0, 2, 1, 3) if c["token_major"] else x


def make(c):
    """Everything a call may take, as numpy arrays; pools as logical [n_pages, Hkv or 1, page, d] views."""
    rng = np.random.default_rng(c["seed"] + c["d"] + 7 * c["n"])
    s = {"q": rows_of(rng, c, c["Hq"], 2.0), "k": rows_of(rng, c, c["Hkv"]), "v": rows_of(rng, c, c["Hkv"])}
    lists = np.maximum(c["lengths"], 0) if c["by_head"] else np.maximum(c["lengths"], 0).max(1, keepdims=True)
    per_list = -(-lists // c["page"])
    n_pages, most = int(per_list.sum()) + c["spare"], max(1, int(per_list.max()))
    ids = rng.permutation(n_pages).astype(np.int32)
    table, at = np.zeros(lists.shape + (most,), np.int32), 0
    for b, h in np.ndindex(lists.shape):
        k = per_list[b, h]
        table[b, h, :k] = ids[at:at + k]
        table[b, h, k:] = -1
        at += k
    s["table"] = table if c["by_head"] else np.ascontiguousarray(table[:, 0])
    heads = 1 if c["by_head"] else c["Hkv"]
    for name in ("k_pages", "v_pages"):
        shape = (n_pages, c["page"], heads, c["d"]) if c["pool_token_major"] else (n_pages, heads, c["page"], c["d"])
        x = stored(rng.standard_normal(shape, dtype=np.float32), c["dtype"])
        s[name] = x.transpose(0, 2, 1, 3) if c["pool_token_major"] else x
    s["positions"] = (rng.integers(0, 200000, (c["batch"], 1)) + np.arange(c["n"])).astype(np.int32)
    half = c["rot_dim"] // 2
    s["inv_freq"] = (1e4 ** (-np.arange(half) / max(half, 1))).astype(np.float32)
    for name in ("q_weight", "k_weight"):
        s[name] = stored(0.5 + rng.random(c["d"], np.float32), c["dtype"]) if c["norm"] else None
    return s


def params(c, s):
    strides = {f"{n}_stride": [x // s[n].itemsize for x in s[n].strides[:3]] for n in ("q", "k", "v")}
    return B.make_params(batch=c["batch"], n_q_heads=c["Hq"], n_kv_heads=c["Hkv"], head_dim=c["d"], seq_len=c["n"], window=1,
                         dtype=c["dtype"], pool=B.POOL_NONE, pool_kernel=1, budget=1, cap=1, softmax_scale=c["scale"], **strides)


def pages(c, s):
    p = B.CkvPages()
    p.page_rows, p.n_pages, p.max_pages = c["page"], s["k_pages"].shape[0], s["table"].shape[-1]
    for name, arr in (("k_pages", p.k_stride), ("v_pages", p.v_stride)):
        x = s[name]
        for i in range(3):
            arr[i] = 0 if i == 1 and c["by_head"] else x.strides[i] // x.itemsize
    p.table_stride[0] = s["table"].strides[0] // 4
    p.table_stride[1] = s["table"].strides[1] // 4 if c["by_head"] else 0
    return p


def rotation(c):
    return B.make_rotation(c["rot_dim"], pairing=c["pairing"], norm=c["norm"], norm_eps=1e-5)


# ---- results ----------------------------------------------------------------------------------------------------------------
def transform(c, s, x, weight):
    """(result, tolerance) of rows x [batch, heads, n, d] in 64 bits."""
    x, r, d = values(x).astype(np.float64), c["rot_dim"], c["d"]
    if not c["norm"] and r == 0:
        return x, np.zeros_like(x)
    if c["norm"]:
        w = 1.0 if weight is None else values(weight).astype(np.float64)
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + np.float32(1e-5)) * w
    y, size = x.copy(), np.abs(x)
    if r:
        angle = s["positions"].astype(np.float64)[:, None, :, None] * s["inv_freq"].astype(np.float64)
        cos, sin = np.cos(angle), np.sin(angle)
        i, j = (slice(0, r // 2), slice(r // 2, r)) if c["pairing"] == B.PAIR_HALVES else (slice(0, r, 2), slice(1, r, 2))
        a, b = x[..., i], x[..., j]
        y[..., i], y[..., j] = a * cos - b * sin, b * cos + a * sin
        size[..., i] = size[..., j] = np.abs(a) + np.abs(b)
    tol = ((d + 16) + 7) * H24 * size + (H8 if c["dtype"] == "bf16" else H24) * np.abs(y)
    return y, tol


def place(c, s, b, g, row):
    """(page, row in it) of a list's row, or None where nothing is."""
    lists = s["table"][b, g] if c["by_head"] else s["table"][b]
    if not 0 <= row < lists.size * c["page"]:
        return None
    page = int(lists[row // c["page"]])
    return (page, row % c["page"]) if 0 <= page < s["k_pages"].shape[0] else None


def appended(c, s):
    """Pools and tolerances behind the append, in 64 bits; the rows that it does not write keep their values."""
    n = new_counts(c)
    k, tol = transform(c, s, s["k"], s["k_weight"])
    kp, vp = (values(s[m]).astype(np.float64) for m in ("k_pages", "v_pages"))
    kt = np.zeros_like(kp)
    for b, g in np.ndindex(n.shape):
        for i in range(n[b, g]):
            at = place(c, s, b, g, max(int(c["lengths"][b, g]), 0) - int(n[b, g]) + i)
            if at is not None:
                h = 0 if c["by_head"] else g
                kp[at[0], h, at[1]], kt[at[0], h, at[1]] = k[b, g, i], tol[b, g, i]
                vp[at[0], h, at[1]] = values(s["v"])[b, g, i]
    return kp, kt, vp


def attention(c, s):
    """out, its tolerance, lse, its tolerance; rows that are not the call's are NaN."""
    n, G, d = new_counts(c), c["Hq"] // c["Hkv"], c["d"]
    scale = float(np.float32(c["scale"])) or 1.0 / np.sqrt(d)
    n_rows = c["n_rows"] or s["table"].shape[-1] * c["page"]
    shape = (c["batch"], c["Hq"], c["n"])
    out, out_tol = np.full(shape + (d,), np.nan), np.zeros(shape + (d,))
    lse, lse_tol = np.full(shape, np.nan), np.zeros(shape)
    bf16 = c["dtype"] == "bf16"
    for b, g in np.ndindex(n.shape):
        length, count, h0 = max(int(c["lengths"][b, g]), 0), int(n[b, g]), 0 if c["by_head"] else g
        rows = [place(c, s, b, g, j) for j in range(min(length, n_rows))]
        there = np.array([r is not None for r in rows], bool)
        at = np.array([r if r is not None else (0, 0) for r in rows], int).reshape(-1, 2)
        k, v = (values(s[m][at[:, 0], h0, at[:, 1]]).astype(np.float64) for m in ("k_pages", "v_pages"))
        if count and len(rows) and there.all() and length >= count and np.isfinite(k).all() and np.isfinite(v).all():
            # nothing out of the ordinary: all tokens of a head at once
            seen = np.arange(len(rows)) <= (length - count + np.arange(count))[:, None]
            for h in range(g * G, (g + 1) * G):
                q = values(s["q"])[b, h, :count].astype(np.float64)
                z = np.where(seen, scale * (q @ k.T), -np.inf)
                top = z.max(1, keepdims=True)
                w = np.exp(z - top)
                total = w.sum(1, keepdims=True)
                w /= total
                lse[b, h, :count], out[b, h, :count] = (top + np.log(total))[:, 0], w @ v
                e = (d + 4) * H24 * scale * np.where(seen, np.abs(q) @ np.abs(k).T, 0.0).max(1)
                many = seen.sum(1) + 16
                lse_tol[b, h, :count] = e + many * H24 + 2 * H24 * np.abs(lse[b, h, :count])
                out_tol[b, h, :count] = ((2 * e + many * 2 * H24 + (H8 if bf16 else 0.0))[:, None] * (w @ np.abs(v))
                                         + (H8 if bf16 else H24) * np.abs(out[b, h, :count]))
            continue
        for h in range(g * G, (g + 1) * G):
            for i in range(count):
                sees = there & (np.arange(len(rows)) <= length - count + i)
                if not sees.any():
                    out[b, h, i], lse[b, h, i] = 0.0, -np.inf
                    continue
                q = values(s["q"])[b, h, i].astype(np.float64)
                kk, vv = k[sees], v[sees]
                with np.errstate(invalid="ignore", over="ignore"):
                    z = scale * (kk @ q)
                    top = z.max()
                    w = np.exp(z - top)
                    lse[b, h, i] = top + np.log(w.sum())
                    w /= w.sum()
                    out[b, h, i] = (w[:, None] * vv).sum(0)
                    e = (d + 4) * H24 * scale * (np.abs(kk) @ np.abs(q)).max()
                    lse_tol[b, h, i] = e + (len(z) + 16) * H24 + 2 * H24 * abs(lse[b, h, i])
                    size = (w[:, None] * np.abs(vv)).sum(0)
                    out_tol[b, h, i] = (2 * e + (len(z) + 16) * 2 * H24 + (H8 if bf16 else 0.0)) * size + (H8 if bf16 else H24) * np.abs(out[b, h, i])
    return out, out_tol, lse, lse_tol


def check(got, want, tol, what):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    finite = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{what}: NaN in other places"
    assert np.array_equal(got[~finite & ~np.isnan(want)], want[~finite & ~np.isnan(want)]), f"{what}: infinities"
    off = np.abs(got[finite] - want[finite]) - tol[finite]
    assert off.size == 0 or off.max() <= 0, f"{what}: {(off > 0).sum()} of {off.size} off, worst by {off.max():.3e} more than allowed"


A, N = B.PAIR_HALVES, B.PAIR_NEIGHBOURS
ROWS = [
    case(norm=True, rot_dim=128, lengths=((40, 40), (7, 7))),                                     # a step
    case(d=64, heads=(5, 5), n=9, lengths=((9,) * 5, (30,) * 5), counts=((9,) * 5, (4,) * 5), norm=True, rot_dim=64, pairing=N),
    case(dtype="f32", d=64, heads=(4, 2), n=37, lengths=((60, 61),), counts=((37, 12),), rot_dim=16, token_major=False, page=8),
    case(dtype="f32", heads=(3, 1), n=3, lengths=((3,), (3,), (0,)), counts=((3,), (0,), (3,)), norm=True, rot_dim=24, pairing=N, page=1),
    case(heads=(7, 1), n=65, lengths=((130,),), norm=True, rot_dim=0, page=64, pool_token_major=True),        # norm only
    case(heads=(2, 2), n=20, lengths=((50, 20), (21, 99)), counts=((20, 20), (3, 17)), by_head=True, page=16),  # plain copies
    case(dtype="f32", heads=(2, 2), n=5, lengths=((5, 5),), page=2, pool_token_major=True),
    case(d=64, heads=(6, 3), n=33, lengths=((1000, 1000, 1000),), rot_dim=48, page=256),
    case(heads=(8, 2), n=4, lengths=((2, 9), (-3, 4)), counts=((4, 9), (4, -1)), rot_dim=128, page=4),  # rows before the list, odd counts
    case(d=64, heads=(40, 40), n=2, lengths=((2,) * 40,), norm=True, rot_dim=64, pairing=N, page=2),     # a workgroup for each head
    case(heads=(18, 2), n=3, lengths=((3, 3),), norm=True, rot_dim=64, page=8, token_major=False),       # more queries than are in flight together
]

ATTEND = [
    case(n=1, lengths=((1, 1), (2, 700), (0, 5))),
    case(n=1, heads=(4, 4), lengths=((544, 130, 3, 64),), by_head=True, page=32),
    case(n=5, heads=(7, 1), lengths=((333,), (5,), (3,)), page=8),                    # the last: tokens that see no row
    case(n=70, heads=(8, 2), lengths=((70, 70), (300, 290)), counts=((70, 70), (33, 33)), pool_token_major=True),
    case(n=1, heads=(40, 1), lengths=((129,),), page=64),
    case(n=140, heads=(3, 1), d=64, lengths=((200,),), page=128, token_major=False),
    case(n=33, heads=(5, 5), d=64, lengths=((33, 40, 70, 33, 64),), by_head=True, page=1),
    case(dtype="f32", n=1, heads=(4, 2), d=64, lengths=((100, 3), (33, 32))),
    case(dtype="f32", n=50, heads=(4, 2), d=64, lengths=((80, 80),), counts=((50, 50),), page=4),
    case(dtype="f32", n=9, heads=(2, 1), lengths=((200,), (64,)), counts=((9,), (2,)), page=16, scale=0.2),
    case(n=1, heads=(4, 1), lengths=((2500,),), page=16),                             # several workgroups along the rows
    case(n=3, heads=(2, 1), d=64, lengths=((1500,), (64,)), page=32, n_rows=1400),      # a bound below the length
    case(dtype="f32", n=260, heads=(1, 1), d=64, lengths=((270,),), page=16),            # f32 beyond the columns that share rows
    case(n=40, heads=(3, 1), d=64, lengths=((45,), (40,)), counts=((40,), (0,)), page=16),  # a sequence without new tokens
]
