"""Attention of trees over pages, on the GPU, of values that are not finite or nearly so (paged_values makes them, pages_util the results in 64 bits)."""
import numpy as np
import pytest
import torch

import paged_values as pv
import pages_util as v
from test_gpu_paged import host
from test_gpu_pages import attend, check, tree_on_gpu
import paged_util as u

pytestmark = pytest.mark.gpu
# ... and lists that two groups of waves share out, in one chunk and in several
TREES = [dict(c, sees=v.paths(v.parents("random", c["batch"], c["n"]))[0]) for c in pv.FEW + pv.MANY
         + [u.case(n=90, heads=(2, 1), lengths=((700,),), scale=1.0, spare=0, page=16), u.case(n=200, d=64, heads=(2, 1), lengths=((5000,),), scale=1.0, spare=0, page=64)]]


def _run(c, s):
    out, lse = attend(c, tree_on_gpu(c, s))
    torch.cuda.synchronize()
    check(c, s, out, lse)


@pytest.mark.parametrize("near,far,logit", [(5, 133, 300.0), (5, 40, 120.0), (133, 5, 300.0), (150, 70, 90.0)])
@pytest.mark.parametrize("c", TREES, ids=range(len(TREES)))
def test_what_is_seen_and_not_finite_stays(c, near, far, logit):
    """A row far above in the logits does not take away an infinity or a NaN of a row before it."""
    if far >= int(c["lengths"].min()) - c["n"]:
        far = 100
    _run(c, pv.earlier(c, near, far, logit))


@pytest.mark.parametrize("far_away", [False, True])
@pytest.mark.parametrize("c", TREES, ids=range(len(TREES)))
def test_drafted_tokens_that_are_not_finite(c, far_away):
    """What a drafted token holds touches those behind it in the tree alone, in both halves of a list's rows."""
    first = int(c["lengths"].min()) - c["n"]
    rows = {first + t: (None, dict(pv.BAD) if t % 2 else {9: pv.INF}) for t in range(0, c["n"], 3)}
    if far_away:
        rows[2] = (200.0, {})
    _run(c, pv.make(c, rows))


@pytest.mark.parametrize("rise,value,sign,infinite", pv.HIGH)
@pytest.mark.parametrize("c", TREES, ids=range(len(TREES)))
def test_a_mean_of_large_values_is_finite(c, rise, value, sign, infinite):
    _run(c, pv.high(c, rise, value, sign, infinite))


def _fine(c, entries=0):
    """entries: of a list at least, as in a call that is planned for long lists."""
    s, want, tol, want_lse, lse_tol = v.fine(c)
    more = max(0, entries - s["table"].shape[-1])
    s["table"] = np.concatenate([s["table"], np.full(s["table"].shape[:-1] + (more,), -1, np.int32)], -1)
    out, lse = attend(c, tree_on_gpu(c, s))
    torch.cuda.synchronize()
    old = np.arange(c["n"]) >= np.repeat(u.new_counts(c), c["Hq"] // c["Hkv"], 1)[..., None]
    u.check(host(out), np.where(old[..., None], 9.0, want), tol, "out")
    u.check(host(lse), np.where(old, 9.0, want_lse), lse_tol, "lse")


@pytest.mark.parametrize("c", [c for c in v.TREES + v.MANY if c["dtype"] == "bf16" and c["Hq"] * c["n"] < 8000], ids=lambda c: f"{c['Hq']}x{c['n']}")
def test_trees_lose_nothing_to_the_weights(c):
    _fine(c)


@pytest.mark.parametrize("kw,rows", [
    (dict(n=60, heads=(16, 4), lengths=((2500, 60, 700, 61),), by_head=True), 65536),
    (dict(kind="empty", n=60, d=64, heads=(16, 4), lengths=((1500,) * 4,), counts=((31,) * 4,)), 131072),
    (dict(kind="noise", n=250, heads=(4, 4), lengths=((900,) * 4,), pool_token_major=True), 70000)])
def test_tiles_of_256_columns_in_chunks(kw, rows):
    _fine(v.tree_case(**dict(dict(page=16), **kw)), rows // 16)
