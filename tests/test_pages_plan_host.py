"""How calls of ckv_paged_tree_attention are shared out over the chip, from sizes alone: the plan of the library's sources, compiled for the host."""
import ctypes
import os
import subprocess

import pytest

import cpu_build as cpu
import pages_util as v

pytestmark = pytest.mark.skipif(cpu.CXX is None, reason="no clang++ for the host")
CUS = 256

SOURCE = """
#include "ckv_pages.h"
extern "C" void plan(int batch, int heads, int kv_heads, int n, int d, int esize, int rows, int tree, long long *out) {
  ckv::Shape s{};
  s.Bz = batch, s.Hq = heads, s.Hkv = kv_heads, s.G = heads / kv_heads, s.T = n, s.d = d, s.esize = esize;
  const ckv::PagedPlan p = ckv::plan_paged(s, rows, tree != 0);
  const long long all[] = {p.by_rows, p.tile_cols, p.col_tiles, p.n_chunks, p.halves, p.workgroups};
  for (int i = 0; i < 6; ++i) out[i] = all[i];
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    where = tmp_path_factory.mktemp("plan")
    lib = v.build_cpu(where)
    (where / "plan.cpp").write_text(SOURCE)
    so = str(where / "plan.so")
    subprocess.run([cpu.CXX, "-x", "c++", "-std=c++17", "-O1", "-fPIC", "-w", "-shared", f"-I{cpu.HERE}", f"-I{cpu.ROOT / 'include'}",
                    f"-I{cpu.ROOT / 'paper_2602_08686_amd' / 'csrc'}", str(where / "plan.cpp"), "-x", "none", lib, f"-Wl,-rpath,{where}", "-o", so], check=True)
    call = ctypes.CDLL(so, mode=os.RTLD_LAZY).plan   # entry points whose kernels are not part of this build stay unresolved

    def of(batch, heads, kv_heads, n, rows, d=128, esize=2, tree=True):
        out = (ctypes.c_longlong * 6)()
        call(batch, heads, kv_heads, n, d, esize, rows, tree, out)
        return dict(zip(("by_rows", "cols", "col_tiles", "chunks", "halves", "workgroups"), out))
    return of


@pytest.mark.parametrize("batch,heads,kv_heads,n,rows,d,workgroups", [(1, 8, 1, 32, 131072, 128, 128), (1, 16, 2, 32, 65536, 128, 256),
                                                                      (1, 24, 3, 32, 50000, 128, 252), (1, 16, 2, 32, 131072, 64, 256)])
def test_few_long_lists_keep_the_chip_busy(plan, batch, heads, kv_heads, n, rows, d, workgroups):
    """A list has at most 64 chunks: with one to three lists tiles of 256 columns would leave half of the CUs idle."""
    p = plan(batch, heads, kv_heads, n, rows, d)
    assert (p["cols"], p["halves"], p["workgroups"]) == (128, 1, workgroups)


def test_wide_tiles_leave_three_quarters_of_the_waves_busy(plan):
    wide = 0
    for lists in range(1, 400):
        for rows in (700, 3000, 9001, 33000, 131072, 1 << 20):
            for cols in (100, 200, 250, 500, 760, 2000):
                for d in (64, 128):
                    p = plan(1, lists, lists, cols, rows, d)   # a head a list: a column a token
                    narrow, tiles = lists * -(-cols // 128), lists * -(-cols // 256)
                    if p["cols"] != 256 or tiles >= CUS:
                        continue
                    wide += 1
                    most = min(64, -(-rows // 512))
                    other = narrow * min(CUS // narrow, most) if narrow <= CUS else narrow / 2   # of eight waves
                    assert 4 * p["workgroups"] >= 3 * other, (lists, rows, cols, d, p)
                    assert rows // p["chunks"] * d >= 1000 * 128, (lists, rows, cols, d, p)
    assert wide > 1000
    for d, rows in ((128, 65536), (64, 131072)):   # as the kernels' tests have it
        assert (plan(1, 16, 4, 60, rows, d)["cols"], plan(1, 4, 4, 250, rows, d)["cols"]) == (256, 256)
    assert plan(4, 32, 8, 60, 32768)["cols"] == 256 and plan(4, 32, 8, 60, 4096)["cols"] == 128


def test_the_causal_order_has_no_tiles_of_its_own(plan):
    for args in ((4, 32, 8, 60, 32768), (1, 8, 1, 32, 131072), (2, 32, 8, 500, 4099)):
        p = plan(*args, tree=False)
        assert p["cols"] == 128 and not p["halves"]
