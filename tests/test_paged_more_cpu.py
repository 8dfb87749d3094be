"""On the host CPU: every instance of the paged attention's kernels that a call can reach is reached by the tests' cases; those that the shorter cases leave out are run here too."""
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
from test_paged_cpu import _attend_case

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


def _all_instances(path):
    lib = cpu.load(path)
    lib.emu_set_dry(1)
    lib.emu_launched()
    got = {x[:2] for c in u.ATTEND + LONG + more.MANY for x in _attention_launches(lib, c)}
    types = [(t, d) for t in "01" for d in ("64", "128")]   # f32, bf16
    want = {("paged_tile_kernel", (t, d, w)) for t, d in types for w in "48"} | {("paged_merge_kernel", x) for x in types}
    want |= {("paged_rows_kernel", (t, d, "4" if (t, d) == ("0", "128") else "8", stream)) for t, d in types for stream in ("true", "false")}
    assert got == want, (want - got, got - want)


def test_every_instance_is_reached(lib_path):  # noqa: F811
    in_child(_all_instances, lib_path)


@pytest.mark.parametrize("c", [c for c in more.MANY if c["batch"] * c["Hkv"] < 128], ids=range(sum(c["batch"] * c["Hkv"] < 128 for c in more.MANY)))
def test_attention_over_pages(lib_path, c):  # noqa: F811
    in_child(_attend_case, lib_path, c)
