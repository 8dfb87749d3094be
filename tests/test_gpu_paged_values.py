"""Attention over pages, on the GPU, of values that are not finite or nearly so (paged_values makes them, paged_util the results in 64 bits)."""
import pytest
import torch

import paged_util as u
import paged_values as pv
from test_gpu_paged import attend, check_attention, host, on_gpu

pytestmark = pytest.mark.gpu


def _run(c, s):
    out, lse = attend(c, on_gpu(c, s))
    torch.cuda.synchronize()
    check_attention(c, s, out, lse)


@pytest.mark.parametrize("near,far,logit", [(5, 133, 300.0), (5, 261, 100.0), (5, 40, 120.0), (70, 150, 300.0), (133, 5, 300.0), (150, 70, 90.0)])
@pytest.mark.parametrize("c", pv.FEW + pv.MANY, ids=range(len(pv.FEW + pv.MANY)))
def test_what_is_seen_and_not_finite_stays(c, near, far, logit):
    """A row far above in the logits does not take away an infinity or a NaN of a row before it."""
    if far >= int(c["lengths"].min()) - c["n"]:
        far = 100
    _run(c, pv.earlier(c, near, far, logit))


@pytest.mark.parametrize("rise,value,sign,infinite", pv.HIGH)
@pytest.mark.parametrize("c", pv.FEW + pv.MANY, ids=range(len(pv.FEW + pv.MANY)))
def test_a_mean_of_large_values_is_finite(c, rise, value, sign, infinite):
    _run(c, pv.high(c, rise, value, sign, infinite))


@pytest.mark.parametrize("c", pv.FINE, ids=range(len(pv.FINE)))
def test_few_columns_lose_nothing_to_the_weights(c):
    s, want, tol, want_lse, lse_tol = pv.fine(c)
    out, lse = attend(c, on_gpu(c, s))
    torch.cuda.synchronize()
    u.check(host(out), want, tol, "out")
    u.check(host(lse), want_lse, lse_tol, "lse")


@pytest.mark.parametrize("c", [pv.FEW[0], pv.FEW[3], pv.FEW[5], pv.MANY[0], pv.MANY[2]], ids=range(5))
def test_a_row_with_a_logit_of_minus_infinity_is_not_seen(c):
    out, lse = attend(c, on_gpu(c, pv.no_logit(c, True)))
    torch.cuda.synchronize()
    check_attention(c, pv.no_logit(c, False), out, lse)
