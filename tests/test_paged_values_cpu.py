"""Attention over pages, on the host CPU, of values that are not finite or nearly so: the result is the definition's whatever the order of the rows."""
import pytest

import cpu_build as cpu
import paged_util as u
import paged_values as pv
from test_cpu_build import in_child, lib_path  # noqa: F401
from test_paged_cpu import _attend, _check_attention, _fenced

pytestmark = pytest.mark.skipif(cpu.CXX is None, reason="no clang++ for the host")


def _run(path, c, make, *args):
    lib = cpu.load(path)
    s = _fenced(make(c, *args))
    _check_attention(c, s, *_attend(lib, c, s))


@pytest.mark.parametrize("near,far", [(5, 133), (5, 261), (5, 40), (70, 150), (133, 5), (150, 70)])
@pytest.mark.parametrize("c", pv.FEW + pv.MANY, ids=range(len(pv.FEW + pv.MANY)))
def test_what_is_seen_and_not_finite_stays(lib_path, c, near, far):  # noqa: F811
    """A row far above in the logits does not take away an infinity or a NaN of a row before it."""
    if far >= int(c["lengths"].min()) - c["n"]:
        far = 100
    in_child(_run, lib_path, c, pv.earlier, near, far, 300.0)


@pytest.mark.parametrize("rise,value,sign,infinite", pv.HIGH)
@pytest.mark.parametrize("c", pv.FEW + pv.MANY, ids=range(len(pv.FEW + pv.MANY)))
def test_a_mean_of_large_values_is_finite(lib_path, c, rise, value, sign, infinite):  # noqa: F811
    in_child(_run, lib_path, c, pv.high, rise, value, sign, infinite)


def _fine(path, c):
    lib = cpu.load(path)
    s, want, tol, want_lse, lse_tol = pv.fine(c)
    out, lse = _attend(lib, c, _fenced(s))
    u.check(out, want, tol, "out")
    u.check(lse, want_lse, lse_tol, "lse")


@pytest.mark.parametrize("c", pv.FINE, ids=range(len(pv.FINE)))
def test_few_columns_lose_nothing_to_the_weights(lib_path, c):  # noqa: F811
    in_child(_fine, lib_path, c)


def _no_logit(path, c):
    lib = cpu.load(path)
    _check_attention(c, pv.no_logit(c, False), *_attend(lib, c, _fenced(pv.no_logit(c, True))))


@pytest.mark.parametrize("c", [pv.FEW[0], pv.FEW[3], pv.FEW[5], pv.MANY[0], pv.MANY[2]], ids=range(5))
def test_a_row_with_a_logit_of_minus_infinity_is_not_seen(lib_path, c):  # noqa: F811
    in_child(_no_logit, lib_path, c)
