"""Lists in which a few rows of V or of K are out of the ordinary, for the tests of attention over pages on the host CPU and on the GPU. The first
component of every query is one and softmax_scale is one, so that the first component of a row of K is its logit but for some tenths."""
import numpy as np

import paged_util as u

INF, NAN = np.inf, np.nan


def make(c, rows, v_all=None):
    """rows: {row: (logit or None, {component of V: value})}, planted in every list. v_all: what all of V is otherwise."""
    s = u.make(c)
    x = {m: u.values(np.ascontiguousarray(s[m])).copy() for m in ("q", "k_pages", "v_pages")}
    x["q"][..., 1:] *= 0.02
    x["q"][..., 0] = 1.0
    x["k_pages"][..., 0] = 0.0
    if v_all is not None:
        x["v_pages"][:] = v_all
    for b, g in np.ndindex(c["batch"], c["Hkv"]):
        for row, (logit, v) in rows.items():
            page, at = u.place(c, s, b, g, row)
            h = 0 if c["by_head"] else g
            if logit is not None:
                x["k_pages"][page, h, at, 0] = logit
            for d, value in v.items():
                x["v_pages"][page, h, at, d] = value
    for m in x:
        s[m] = u.stored(x[m], c["dtype"])
    return s


def _case(length, **kw):
    heads = kw.pop("heads", (2, 1))
    return u.case(heads=heads, lengths=((length,) * heads[1],), scale=1.0, spare=0, **kw)


# The kernel for few columns: a wave takes every eighth (f32 rows of 512 bytes: every fourth) block of 32 rows; the one for many columns: stages of 64 rows.
FEW = [
    _case(600, page=16),
    _case(600, d=64, n=3, page=8),
    _case(250, dtype="f32", d=64, page=16, heads=(1, 1)),
    _case(250, dtype="f32", n=3, page=4),
    _case(2500, page=64),                                   # chunks, joined in the same launch
    _case(2500, n=20, page=64),                             # chunks, joined by a kernel of their own
]
MANY = [
    _case(300, n=70, heads=(1, 1), page=16),
    _case(300, n=140, heads=(1, 1), d=64, page=32),
    _case(400, dtype="f32", n=300, heads=(1, 1), d=64, page=16),
    _case(1200, n=70, heads=(1, 1), page=64),               # chunks
]
LOST = {INF: 3, NAN: 5, -INF: 7}                            # component of V by what it holds
BAD = {d: value for value, d in LOST.items()}


def earlier(c, near, far, logit):
    """Row `near` of V is not finite and row `far` outweighs it by `logit`; component 9 has infinities of both signs, in rows of their own."""
    return make(c, {near: (None, dict(BAD)), near + 1: (None, {9: INF}), near + 2: (None, {9: -INF}), far: (logit, {})})


def high(c, rise, value, sign, infinite):
    """All of V at +-value, near the type's largest: every weighted mean is finite, the sums of weights times V are not. rise: logits grow with the
    row, so that the softmax's reference keeps moving. infinite: one row holds an infinity and a NaN beside it."""
    rng = np.random.default_rng(1)
    rows = int(c["lengths"].max())
    v = {r: {0: value if sign == "same" or rng.random() < 0.7 else -value, **({} if not (infinite and r == 7) else {3: INF, 5: NAN})} for r in range(rows)}
    return make(c, {r: (rise * r, x) for r, x in v.items()}, v_all=value)


HIGH = [(0.0, 1e37, "same", False), (0.02, 3e38, "same", False), (0.25, 3e38, "mixed", False), (-0.02, 2e38, "mixed", True)]


def fine(c):
    """Lists as they are, and the bound on the result with weights that are off by 2^-16 of themselves at most (two bf16 terms: each is off by 2^-8 of
    what it stands for), in place of one rounding to bf16: paged_util's without its 2^-8 of sum_j w_j |v_j|."""
    s = u.make(c)
    want, tol, lse, lse_tol = u.attention(c, s)
    plain = dict(s, v_pages=u.stored(np.abs(u.values(np.ascontiguousarray(s["v_pages"]))), c["dtype"]))
    size = u.attention(c, plain)[0]   # sum_j w_j |v_j|
    return s, want, tol - (u.H8 - 2.0 ** -16) * size, lse, lse_tol


FINE = [u.case(n=1, lengths=((600, 31), (33, 1000))), u.case(n=9, heads=(7, 1), d=64, lengths=((900,), (16,)), page=64), u.case(n=4, lengths=((3000, 2900),)),
        u.case(n=1, heads=(4, 1), lengths=((2500,),))]


def no_logit(c, minus_infinity):
    """Rows whose logit is -infinity, V infinite or NaN beside it; or the same rows so far below the others that they weigh nothing in 64 bits either, V
    finite: the results are the same."""
    rows = {4: {3: INF}, 40: {3: NAN, 5: -INF}, 41: {}}
    return make(c, {r: (-INF, v) if minus_infinity else (-800.0, {}) for r, v in rows.items()})
