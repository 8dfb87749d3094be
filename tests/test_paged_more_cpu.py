"""On the host CPU: every instance of the paged cache's kernels that a call can reach, and the plans of long calls' rows, are reached by the tests' cases;
those that the shorter cases leave out are run here too."""
import ctypes
import re

import numpy as np
import pytest

import cpu_build as cpu
import paged_more as more
import paged_util as u
from paper_2602_08686_amd import binding as B
from test_cpu_build import in_child, lib_path  # noqa: F401
from test_gpu_paged import LONG
from test_paged_cpu import _attend_case, _rows_case

pytestmark = pytest.mark.skipif(cpu.CXX is None, reason="no clang++ for the host")
AT = ctypes.c_void_p(4096)   # no kernel runs: nothing is there


def _launched(lib):
    """(kernel, its template arguments by name, grid) of the launches since the last call."""
    out = []
    for line in lib.emu_launched().decode().splitlines():
        kernel, where, x, y = line.split("|")
        kernel, own = re.match(r"\((\w+)<(.*)>\)", kernel).groups()
        given = dict(re.findall(r"(\w+) = (\w+)", where[where.index("["):]))
        out.append((kernel, tuple(given.get(a, a) for a in own.replace(" ", "").split(",")), (int(x), int(y))))
    return out


def _attention_launches(lib, c):
    s = u.make(c)
    p, n_rows = u.params(c, s), c["n_rows"] or s["table"].shape[-1] * c["page"]
    need = lib.ckv_paged_workspace_bytes(ctypes.byref(p), n_rows)
    st = lib.ckv_paged_attention(ctypes.byref(p), ctypes.byref(u.pages(c, s)), AT, AT, AT, AT, AT, None, n_rows, AT, None, None, AT,
                                 ctypes.c_size_t(need), None)
    assert st == B.CKV_OK
    return _launched(lib)


def _rows_launches(lib, c, paged):
    s = u.make(c)
    p, rot = u.params(c, s), u.rotation(c)
    if paged:
        st = lib.ckv_paged_append(ctypes.byref(p), ctypes.byref(rot), ctypes.byref(u.pages(c, s)), AT, AT, AT, AT, AT, None, None, AT, AT, None, AT, AT, AT,
                                  None)
    else:
        st = lib.ckv_norm_rotate(ctypes.byref(p), ctypes.byref(rot), AT, AT, AT, AT, None, None, None, AT, AT, None)
    assert st == B.CKV_OK
    return _launched(lib)


def _all_instances(path):
    lib = cpu.load(path)
    lib.emu_set_dry(1)
    lib.emu_launched()
    got = {x[:2] for c in u.ATTEND + LONG + more.MANY for x in _attention_launches(lib, c)}
    got |= {x[:2] for c in u.ROWS + more.ROWS for paged in (False, True) for x in _rows_launches(lib, c, paged)}
    types = [(t, d) for t in "01" for d in ("64", "128")]   # f32, bf16; forms of rows: copied, halves, neighbours
    want = {("paged_tile_kernel", (t, d, w)) for t, d in types for w in "48"} | {("paged_merge_kernel", x) for x in types}
    want |= {("paged_rows_kernel", (t, d, "4" if (t, d) == ("0", "128") else "8", stream)) for t, d in types for stream in ("true", "false")}
    want |= {("rows_kernel", (t, d, form, paged)) for t, d in types for form in "012" for paged in ("true", "false")}
    assert got == want, (want - got, got - want)


def test_every_instance_is_reached(lib_path):  # noqa: F811
    in_child(_all_instances, lib_path)


def _long_plans(path):
    """Tokens and KV heads of a workgroup, read off the grids."""
    lib = cpu.load(path)
    lib.emu_set_dry(1)
    lib.emu_launched()
    reached = []
    for c in more.ROWS:
        for paged in (False, True):
            (_, _, (x, y)), = _rows_launches(lib, c, paged)
            blocks = x // c["batch"]
            tokens = next(t for t in (1, 2, 4, 8) if -(-c["n"] // t) == blocks)
            heads = max(h for h in range(1, 33) if -(-c["Hkv"] // h) == y)
            heads = min(heads, c["Hkv"])
            reached.append((c["dtype"], paged, tokens, c["n"] % tokens > 0, c["Hkv"] % heads > 0, tokens * heads > 256 // (c["d"] // 8)))
    for dtype in ("bf16", "f32"):
        for paged in (False, True):
            mine = [r[2:] for r in reached if r[:2] == (dtype, paged)]
            # several tokens, a block that is not full, a group of heads that is not, more (token, head)s than go abreast
            assert any(r[0] > 1 for r in mine) and any(r[1] for r in mine) and any(r[2] for r in mine) and any(r[3] for r in mine), mine
    assert {1, 2, 4, 8} <= {r[2] for r in reached}


def test_long_calls_share_out_tokens_and_heads(lib_path):  # noqa: F811
    in_child(_long_plans, lib_path)


@pytest.mark.parametrize("c", [more.ROWS[i] for i in (1, 4, 5, 7, 8, 9, 10)], ids=(1, 4, 5, 7, 8, 9, 10))   # the others take a minute here
def test_rows_are_transformed_and_find_their_pages(lib_path, c):  # noqa: F811
    in_child(_rows_case, lib_path, c)


@pytest.mark.parametrize("c", [c for c in more.MANY if c["batch"] * c["Hkv"] < 128], ids=range(sum(c["batch"] * c["Hkv"] < 128 for c in more.MANY)))
def test_attention_over_pages(lib_path, c):  # noqa: F811
    in_child(_attend_case, lib_path, c)
