"""The paged cache's kernels on the host CPU, where an access out of bounds ends a child process instead of a GPU: norm and rotation,
the append, attention over pages against 64 bits, with page numbers that are none, pools that end at a page without
access, and infinities and NaN where nobody looks."""
import ctypes

import numpy as np
import pytest

import cpu_build as cpu
import paged_util as u
from paper_2602_08686_amd import binding as B
from test_cpu_build import in_child, lib_path  # noqa: F401  (the library, built once for this module)

pytestmark = pytest.mark.skipif(cpu.CXX is None, reason="no clang++ for the host")
ref = ctypes.byref


def _at_fence(x):
    """The same array, strides and all, with its last byte before a page without access."""
    if x is None:
        return None
    order = sorted(range(x.ndim), key=lambda i: -x.strides[i])
    base = np.ascontiguousarray(x.transpose(order))
    mem = cpu.fenced(base.nbytes)
    mem[:] = base.view(np.uint8).ravel()
    return mem.view(base.dtype).reshape(base.shape).transpose(np.argsort(order))


def _fenced(s):
    return {n: _at_fence(x) for n, x in s.items()}


def _blank(c, heads, dtype=None):
    shape = (c["batch"], heads, c["n"], c["d"])
    x = cpu.fenced(int(np.prod(shape)) * (2 if c["dtype"] == "bf16" else 4)).view(np.uint16 if c["dtype"] == "bf16" else np.float32)
    x[:] = 0x4110 if c["dtype"] == "bf16" else 9.0   # nine
    return x.reshape(shape)


def _rows_case(path, c):
    lib = cpu.load(path)
    s = _fenced(u.make(c))
    p, rot = u.params(c, s), u.rotation(c)
    n, G = u.new_counts(c), c["Hq"] // c["Hkv"]
    count = None if c["counts"] is None else _at_fence(c["counts"])
    P = cpu.ptr
    q_out, k_out = _blank(c, c["Hq"]), _blank(c, c["Hkv"])
    st = lib.ckv_norm_rotate(ref(p), ref(rot), P(s["q"]), P(s["k"]), P(s["positions"]), P(s["inv_freq"]), P(s["q_weight"]),
                             P(s["k_weight"]), P(count), P(q_out), P(k_out), None)
    assert st == B.CKV_OK, st

    def dense(got, x, weight, heads, what):
        want, tol = u.transform(c, s, x, weight)
        new = np.arange(c["n"]) < np.repeat(n, heads // c["Hkv"], 1)[..., None]
        u.check(u.values(got), np.where(new[..., None], want, 9.0), np.where(new[..., None], tol, 0.0), what)

    dense(q_out, s["q"], s["q_weight"], c["Hq"], "q_out")
    dense(k_out, s["k"], s["k_weight"], c["Hkv"], "k_out")
    # into pages, some of which are not there
    for bad in (False, True):
        t = dict(s, table=s["table"].copy())
        if bad:
            t["table"].ravel()[::3] = np.resize([-1, s["k_pages"].shape[0], 1 << 30, -(1 << 31)], t["table"].ravel()[::3].size)
        t = _fenced(t)
        kp, kt, vp = u.appended(c, t)
        q_out = _blank(c, c["Hq"])
        with_q = not bad
        st = lib.ckv_paged_append(ref(p), ref(rot) if c["norm"] or c["rot_dim"] else None, ref(u.pages(c, t)), P(t["q"] if with_q else None),
                                  P(t["k"]), P(t["v"]), P(t["positions"]), P(t["inv_freq"]), P(t["q_weight"]), P(t["k_weight"]),
                                  P(t["table"]), P(_at_fence(c["lengths"])), P(count), P(t["k_pages"]), P(t["v_pages"]),
                                  P(q_out if with_q else None), None)
        assert st == B.CKV_OK, st
        u.check(u.values(t["k_pages"]), kp, kt, "k_pages")
        u.check(u.values(t["v_pages"]), vp, np.zeros_like(vp), "v_pages")
        if with_q:
            dense(q_out, t["q"], t["q_weight"], c["Hq"], "q_out of the append")


@pytest.mark.parametrize("c", u.ROWS, ids=range(len(u.ROWS)))
def test_rows_are_transformed_and_find_their_pages(lib_path, c):  # noqa: F811
    in_child(_rows_case, lib_path, c)


def _attend(lib, c, s, out_stride=None, with_lse=True):
    P, p = cpu.ptr, u.params(c, s)
    n_rows = c["n_rows"] or s["table"].shape[-1] * c["page"]
    out = _blank(c, c["Hq"])
    lse = np.full((c["batch"], c["Hq"], c["n"]), 9.0, np.float32)
    need = lib.ckv_paged_workspace_bytes(ref(p), n_rows)
    ws = cpu.fenced(need) if need else None
    st = lib.ckv_paged_attention(ref(p), ref(u.pages(c, s)), P(s["q"]), P(s["k_pages"]), P(s["v_pages"]), P(s["table"]),
                                 P(_at_fence(c["lengths"])), P(None if c["counts"] is None else _at_fence(c["counts"])), n_rows, P(out),
                                 out_stride, P(lse if with_lse else None), P(ws), ctypes.c_size_t(need), None)
    assert st == B.CKV_OK, st
    return u.values(out), lse


def _check_attention(c, s, out, lse):
    want, tol, wl, lt = u.attention(c, s)
    old = np.arange(c["n"]) >= np.repeat(u.new_counts(c), c["Hq"] // c["Hkv"], 1)[..., None]
    u.check(out, np.where(old[..., None], 9.0, want), tol, "out")
    u.check(lse, np.where(old, 9.0, wl), lt, "lse")


def _attend_case(path, c):
    lib = cpu.load(path)
    s = _fenced(u.make(c))
    _check_attention(c, s, *_attend(lib, c, s))


@pytest.mark.parametrize("c", u.ATTEND, ids=range(len(u.ATTEND)))
def test_attention_over_pages(lib_path, c):  # noqa: F811
    in_child(_attend_case, lib_path, c)


def _attend_odd(path, c, kind):
    lib = cpu.load(path)
    s = u.make(c)
    n_pages = s["k_pages"].shape[0]
    if kind == "bad_pages":   # numbers that are none, one of them the list's first
        t = s["table"].reshape(-1, s["table"].shape[-1])
        t[0, 0] = n_pages
        t[-1, t.shape[1] // 2] = -7
    else:                      # what nobody sees is not finite; what is seen now and then, too
        seen = np.zeros(s["k_pages"].shape[:3], bool)
        new = np.zeros_like(seen)
        n = u.new_counts(c)
        for b, g in np.ndindex(n.shape):
            length = int(c["lengths"][b, g])
            for row in range(length):
                at = u.place(c, s, b, g, row)
                seen[at[0], 0 if c["by_head"] else g, at[1]] = True
                new[at[0], 0 if c["by_head"] else g, at[1]] |= row >= length - 2 and n[b, g] > 2  # not seen by the first new ones
        for m in ("k_pages", "v_pages"):
            x = u.values(s[m]).copy()
            x[~seen] = np.nan
            if kind == "beyond":
                pass
            elif kind == "masked_infinity":
                x[new] = np.inf if m == "v_pages" else x[new]
            elif kind == "masked_nan":
                x[new] = np.nan
            elif kind == "one_component":
                x[new, 3] = -np.inf if m == "v_pages" else x[new, 3]
                x[new, 5] = np.nan if m == "v_pages" else x[new, 5]
            s[m] = u.stored(x, c["dtype"]) if x.flags["C_CONTIGUOUS"] else u.stored(x.transpose(0, 2, 1, 3), c["dtype"]).transpose(0, 2, 1, 3)
    s = _fenced(s)
    _check_attention(c, s, *_attend(lib, c, s))


@pytest.mark.parametrize("kind", ["bad_pages", "beyond", "masked_infinity", "masked_nan", "one_component"])
@pytest.mark.parametrize("i", [1, 2, 3, 6, 8, 9, 10])
def test_what_is_not_seen_has_no_influence(lib_path, i, kind):  # noqa: F811
    in_child(_attend_odd, lib_path, u.ATTEND[i], kind)


def _to_the_last_row(path, c):
    """One list, its pages in the pool's order: the pool's memory ends with the list's last row, whose page goes on."""
    lib = cpu.load(path)
    s = u.make(c)
    s["table"] = np.arange(s["table"].size, dtype=np.int32).reshape(s["table"].shape)
    pg = u.pages(c, s)
    s = _fenced(s)
    rows = int(c["lengths"][0, 0])
    for m in ("k_pages", "v_pages"):
        flat = s[m].reshape(-1, c["d"])[:rows]
        s["short_" + m] = _at_fence(np.ascontiguousarray(flat))
    P, p = cpu.ptr, u.params(c, s)
    out, lse = _blank(c, c["Hq"]), np.full((1, c["Hq"], c["n"]), 9.0, np.float32)
    need = lib.ckv_paged_workspace_bytes(ref(p), rows)
    ws = cpu.fenced(need) if need else None
    st = lib.ckv_paged_attention(ref(p), ref(pg), P(s["q"]), P(s["short_k_pages"]), P(s["short_v_pages"]), P(s["table"]),
                                 P(c["lengths"]), None, rows, P(out), None, P(lse), P(ws), ctypes.c_size_t(need), None)
    assert st == B.CKV_OK, st
    _check_attention(c, s, u.values(out), lse)


@pytest.mark.parametrize("dtype,d,heads,n,length", [("bf16", 128, 4, 1, 33), ("bf16", 64, 2, 20, 70), ("f32", 64, 1, 3, 101), ("f32", 128, 2, 40, 41),
                                                    ("bf16", 128, 8, 1, 1601), ("bf16", 128, 4, 9, 65)])
def test_no_row_behind_the_length_is_read(lib_path, dtype, d, heads, n, length):  # noqa: F811
    in_child(_to_the_last_row, lib_path, u.case(dtype=dtype, d=d, heads=(heads, 1), n=n, lengths=((length,),), page=64, spare=0))
