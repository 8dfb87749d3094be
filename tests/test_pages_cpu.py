"""Trees of drafted tokens, rows and pages that move and lists that share pages on the host CPU, where an access out of bounds ends a child process
instead of a GPU: against results in 64 bits, with page numbers that are none, memory that ends at a page without access, and infinities and NaN
where nobody looks."""
import ctypes
import re

import numpy as np
import pytest

import cpu_build as cpu
import paged_util as u
import paged_values as pv
import pages_util as v
from paper_2602_08686_amd import binding as B
from test_cpu_build import in_child
from test_paged_cpu import _at_fence, _blank, _fenced

pytestmark = pytest.mark.skipif(cpu.CXX is None, reason="no clang++ for the host")
ref, P = ctypes.byref, cpu.ptr


@pytest.fixture(scope="module")
def lib_path(tmp_path_factory):
    return v.build_cpu(tmp_path_factory.mktemp("pages_cpu"))


# ---- trees ------------------------------------------------------------------------------------------------------------------
def _sees(path, kind, batch, n):
    lib = cpu.load(path)
    parent = _at_fence(v.parents(kind, batch, n))
    start = _at_fence(np.arange(batch, dtype=np.int32) * 1000 - 5)
    sees, depth = v.paths(parent)
    for with_positions in (True, False):
        words, positions = _at_fence(np.full((batch, n, -(-n // 64)), 9, np.int64)), _at_fence(np.full((batch, n), 9, np.int32))
        st = lib.ckv_tree_sees(batch, n, P(parent), P(start if with_positions else None), P(words), P(positions if with_positions else None), None)
        assert st == B.CKV_OK
        assert np.array_equal(words, v.words(sees))
        assert np.array_equal(positions, start[:, None] + depth if with_positions else np.full((batch, n), 9))


@pytest.mark.parametrize("kind", ["chain", "star", "roots", "odd", "random"])
@pytest.mark.parametrize("batch,n", [(1, 1), (3, 2), (2, 63), (1, 64), (2, 65), (3, 130), (1, 257), (1, 700)])
def test_tokens_see_their_paths(lib_path, kind, batch, n):
    in_child(_sees, lib_path, kind, batch, n)


@pytest.mark.parametrize("kind", ["star", "odd", "random"])
@pytest.mark.parametrize("batch,n", [(2, 1025), (1, 2500)])
def test_long_trees_that_branch(lib_path, kind, batch, n):
    in_child(_sees, lib_path, kind, batch, n)


def test_the_longest_path(lib_path):
    in_child(_sees, lib_path, "chain", 1, 4096)


def _attend(lib, c, s, lse=True):
    p = u.params(c, s)
    n_rows = c["n_rows"] or s["table"].shape[-1] * c["page"]
    out, to = _blank(c, c["Hq"]), np.full((c["batch"], c["Hq"], c["n"]), 9.0, np.float32)
    need = lib.ckv_paged_workspace_bytes(ref(p), n_rows)
    ws = cpu.fenced(need) if need else None
    st = lib.ckv_paged_tree_attention(ref(p), ref(u.pages(c, s)), P(s["q"]), P(s["k_pages"]), P(s["v_pages"]), P(s["table"]),
                                      P(_at_fence(c["lengths"])), P(None if c["counts"] is None else _at_fence(c["counts"])), n_rows,
                                      P(_at_fence(v.words(c["sees"]))), P(out), None, P(to if lse else None), P(ws), ctypes.c_size_t(need), None)
    assert st == B.CKV_OK, st
    return u.values(out), to


def _check(c, s, out, lse):
    want, tol, wl, lt = v.attention(c, s)
    old = np.arange(c["n"]) >= np.repeat(u.new_counts(c), c["Hq"] // c["Hkv"], 1)[..., None]
    u.check(out, np.where(old[..., None], 9.0, want), tol, "out")
    u.check(lse, np.where(old, 9.0, wl), lt, "lse")


def _tree(path, c):
    lib, s = cpu.load(path), _fenced(u.make(c))
    _check(c, s, *_attend(lib, c, s))


@pytest.mark.parametrize("i", range(len(v.TREES)))
def test_attention_of_trees(lib_path, i):
    in_child(_tree, lib_path, v.TREES[i])


def _tree_fine(path, c, entries=0):
    s, want, tol, wl, lt = v.fine(c)
    more = max(0, entries - s["table"].shape[-1])   # a call that is planned for long lists
    s["table"] = np.concatenate([s["table"], np.full(s["table"].shape[:-1] + (more,), -1, np.int32)], -1)
    out, lse = _attend(cpu.load(path), c, _fenced(s))
    old = np.arange(c["n"]) >= np.repeat(u.new_counts(c), c["Hq"] // c["Hkv"], 1)[..., None]
    u.check(out, np.where(old[..., None], 9.0, want), tol, "out")
    u.check(lse, np.where(old, 9.0, wl), lt, "lse")


@pytest.mark.parametrize("i", [1, 4, 5, 8, 9, 18, 19])
def test_trees_lose_nothing_to_the_weights(lib_path, i):
    in_child(_tree_fine, lib_path, v.TREES[i])


@pytest.mark.parametrize("d,rows", [(128, 65536), (64, 131072)])
def test_tiles_of_256_columns_in_chunks(lib_path, d, rows):
    in_child(_tree_fine, lib_path, v.tree_case("empty", n=60, d=d, heads=(16, 4), lengths=((150, 60, 70, 400),), by_head=True, page=16), rows // 16)


def _tree_odd(path, c, kind):
    lib, s = cpu.load(path), u.make(c)
    if kind == "bad_pages":
        t = s["table"].reshape(-1, s["table"].shape[-1])
        t[0, 0] = s["k_pages"].shape[0]
        t[-1, t.shape[1] // 2] = -7
    else:   # rows of drafted tokens, which few tokens see, are not finite
        rng = np.random.default_rng(3)
        for m in ("k_pages", "v_pages"):
            x = np.array(u.values(s[m]))
            for b, g in np.ndindex(c["lengths"].shape):
                length, count = int(c["lengths"][b, g]), int(u.new_counts(c)[b, g])
                for row in range(max(0, length - count), length):
                    at = u.place(c, s, b, g, row)
                    if rng.random() < 0.3:
                        h = 0 if c["by_head"] else g
                        if kind == "nan":
                            x[at[0], h, at[1]] = np.nan
                        elif m == "v_pages":
                            x[at[0], h, at[1], ::3] = np.inf
                            x[at[0], h, at[1], 1] = -np.inf
            s[m] = u.stored(x, c["dtype"])
    s = _fenced(s)
    _check(c, s, *_attend(lib, c, s))


@pytest.mark.parametrize("kind", ["bad_pages", "nan", "infinity"])
@pytest.mark.parametrize("i", [1, 4, 5, 8, 12, 15, 18])
def test_what_a_token_does_not_see_has_no_influence(lib_path, i, kind):
    in_child(_tree_odd, lib_path, v.TREES[i], kind)


def _tree_values(path, c, kind):
    first = int(c["lengths"].min()) - c["n"]
    if kind == "high":
        s = pv.high(c, 0.25, 3e38, "mixed", True)
    elif kind == "earlier":
        s = pv.earlier(c, 5, 133, 300.0)
    else:
        s = pv.make(c, {first + t: (None, dict(pv.BAD) if t % 2 else {9: pv.INF}) for t in range(0, c["n"], 3)})
    s = _fenced(s)
    _check(c, s, *_attend(cpu.load(path), c, s))


@pytest.mark.parametrize("kind", ["high", "earlier", "drafted"])
@pytest.mark.parametrize("c", [pv.FEW[0], pv.FEW[3], pv.MANY[0], pv.MANY[3]], ids=range(4))
def test_values_that_are_not_finite_or_nearly_so(lib_path, c, kind):
    in_child(_tree_values, lib_path, dict(c, sees=v.paths(v.parents("random", c["batch"], c["n"]))[0]), kind)


def _causal(path):
    """A chain is the causal order: for few columns, whose kernel is the same but for the mask, the same bits as the call without a tree."""
    lib = cpu.load(path)
    for i in (2, 12, 17):
        c = v.TREES[i]
        c = dict(c, sees=v.paths(v.parents("chain", c["batch"], c["n"]))[0])
        s = _fenced(u.make(c))
        got = _attend(lib, c, s)
        p, n_rows = u.params(c, s), s["table"].shape[-1] * c["page"]
        out, lse = _blank(c, c["Hq"]), np.full((c["batch"], c["Hq"], c["n"]), 9.0, np.float32)
        need = lib.ckv_paged_workspace_bytes(ref(p), n_rows)
        st = lib.ckv_paged_attention(ref(p), ref(u.pages(c, s)), P(s["q"]), P(s["k_pages"]), P(s["v_pages"]), P(s["table"]), P(c["lengths"]), P(c["counts"]),
                                     n_rows, P(out), None, P(lse), P(cpu.fenced(need) if need else None), ctypes.c_size_t(need), None)
        assert st == B.CKV_OK and np.array_equal(got[0], u.values(out)) and np.array_equal(got[1], lse)


def test_a_chain_is_the_causal_order(lib_path):
    in_child(_causal, lib_path)


def _all_instances(path):
    """(kernel, its template arguments) of the launches that the tests' cases make."""
    lib = cpu.load(path)
    lib.emu_set_dry(1)
    lib.emu_launched()
    got = set()
    at = ctypes.c_void_p(4096)   # no kernel runs: nothing is there
    for c in v.TREES + v.MANY:
        s = u.make(c)
        p, n_rows = u.params(c, s), c["n_rows"] or s["table"].shape[-1] * c["page"]
        need = lib.ckv_paged_workspace_bytes(ref(p), n_rows)
        assert lib.ckv_paged_tree_attention(ref(p), ref(u.pages(c, s)), at, at, at, at, at, None, n_rows, at, at, None, None, at, ctypes.c_size_t(need),
                                            None) == B.CKV_OK
        for line in lib.emu_launched().decode().splitlines():
            kernel, own = re.match(r"\((\w+)<(.*)>\)", line.split("|")[0]).groups()
            where = line.split("|")[1]
            given = dict(re.findall(r"(\w+) = (\w+)", where[where.index("["):]))
            got.add((kernel, tuple(given.get(a, a) for a in own.replace(" ", "").split(","))))
    types = [(t, d) for t in "01" for d in ("64", "128")]   # f32, bf16
    want = {("tree_tile_kernel", (t, d, w, "1")) for t, d in types for w in "48"} | {("tree_tile_kernel", ("1", d, "8", "2")) for d in ("64", "128")}
    want |= {("tree_rows_kernel", (t, d, "4" if (t, d) == ("0", "128") else "8", stream)) for t, d in types for stream in ("true", "false")}
    want |= {("paged_merge_kernel", x) for x in types}
    assert got == want, (sorted(want - got), sorted(got - want))


def test_every_instance_is_reached(lib_path):
    in_child(_all_instances, lib_path)


# ---- rows and pages that move -------------------------------------------------------------------------------------------------
def _same(got, want, what):
    assert np.array_equal(np.ascontiguousarray(got).view(np.uint8), np.ascontiguousarray(want).view(np.uint8)), what


def _compact(path, c, cap, kept, each_head, bad):
    lib, s = cpu.load(path), u.make(c)
    if bad:
        t = s["table"].reshape(-1, s["table"].shape[-1])
        t[0, 0], t[-1, t.shape[1] // 2] = s["k_pages"].shape[0], -7
    idx, stay = v.chosen(c, cap, kept, each_head)
    if bad:
        idx.reshape(-1, cap)[:, cap // 2] = -1
        idx.reshape(-1, cap)[:, -1] = 1 << 30
        stay[0, 0], stay[-1, -1] = 1 << 30, -4
    want, length_out = v.compacted(c, s, idx, stay)
    p, s = u.params(c, s), _fenced(s)
    strides = None if each_head and not bad else (ctypes.c_int64 * 2)(idx.strides[0] // 4, idx.strides[1] // 4 if each_head else 0)
    got = _at_fence(np.full_like(c["lengths"], 9))
    st = lib.ckv_paged_compact(ref(p), ref(u.pages(c, s)), P(s["table"]), P(_at_fence(c["lengths"])),
                               P(None if c["counts"] is None else _at_fence(c["counts"])), P(_at_fence(idx)), strides, cap, P(_at_fence(stay)),
                               P(s["k_pages"]), P(s["v_pages"]), P(got), None)
    assert st == B.CKV_OK, st
    for m in ("k_pages", "v_pages"):
        _same(s[m], want[m], m)
    assert np.array_equal(got, length_out)


@pytest.mark.parametrize("bad", [False, True])
@pytest.mark.parametrize("i", range(len(v.MOVES)))
def test_rows_that_stay_move_together(lib_path, i, bad):
    in_child(_compact, lib_path, *v.MOVES[i], bad)


def _compact_odd(path):
    """Lengths behind the lists' pages, by a little and by far, and below zero: rows that are on a page move, nothing else is touched."""
    lib = cpu.load(path)
    base = u.case(n=1, lengths=((96, 90),), page=16)
    for lengths, counts in (((200, 97), None), ((2 ** 31 - 1, 130), None), ((120, 100), (60, 20)), ((2 ** 31 - 1, 2 ** 31 - 20), (40, 2 ** 31 - 1)), ((-3, -2 ** 31), (5, 9))):
        c = dict(base, lengths=np.array([lengths], np.int32), counts=None if counts is None else np.array([counts], np.int32))
        s = u.make(base)
        idx = np.sort(np.random.default_rng(4).permutation(150)[:40]).astype(np.int32)[None]
        kept = np.array([[40, 33]], np.int32)
        want, length_out = v.compacted(c, s, idx, kept)
        s, got = _fenced(s), _at_fence(np.full_like(c["lengths"], 9))
        st = lib.ckv_paged_compact(ref(u.params(base, s)), ref(u.pages(base, s)), P(s["table"]), P(_at_fence(c["lengths"])),
                                   P(None if counts is None else _at_fence(c["counts"])), P(_at_fence(idx)), (ctypes.c_int64 * 2)(40, 0), 40,
                                   P(_at_fence(kept)), P(s["k_pages"]), P(s["v_pages"]), P(got), None)
        assert st == B.CKV_OK
        for m in ("k_pages", "v_pages"):
            _same(s[m], want[m], m)
        assert np.array_equal(got, length_out)


def test_lengths_that_no_list_has(lib_path):
    in_child(_compact_odd, lib_path)


def _copy(path, c, pairs):
    lib, s = cpu.load(path), u.make(c)
    n = s["k_pages"].shape[0]
    ids = np.random.default_rng(1).permutation(n)[:2 * pairs].reshape(-1, 2).astype(np.int32)
    odd = np.array([[-1, -1], [0, n], [n, 0], [3, 3], [-1, 2]], np.int32)   # nothing to copy
    copy = np.concatenate([odd[:2], ids, odd[2:]])
    want = {m: np.array(s[m]) for m in ("k_pages", "v_pages")}
    for x in want.values():
        x[ids[:, 1]] = x[ids[:, 0]]
    p, s = u.params(c, s), _fenced(s)
    st = lib.ckv_pages_copy(ref(p), ref(u.pages(c, s)), P(_at_fence(copy)), len(copy), P(s["k_pages"]), P(s["v_pages"]), None)
    assert st == B.CKV_OK
    for m in ("k_pages", "v_pages"):
        _same(s[m], want[m], m)


@pytest.mark.parametrize("kw,pairs", [
    (dict(lengths=((300, 300),), page=16), 8), (dict(lengths=((60, 60),), page=64, pool_token_major=True, spare=7), 4),
    (dict(heads=(3, 3), lengths=((40, 30, 20),), page=1), 40), (dict(heads=(4, 4), lengths=((90, 90, 90, 90),), page=32, by_head=True), 5),
    (dict(dtype="f32", d=64, heads=(5, 5), lengths=((90,) * 5,), page=8), 5), (dict(dtype="f32", lengths=((600, 600),), page=256, spare=9), 5)])
def test_pages_are_copied(lib_path, kw, pairs):
    in_child(_copy, lib_path, u.case(**kw), pairs)


# ---- lists ------------------------------------------------------------------------------------------------------------------
class _State:
    """A table, counts and bits at fences, beside what they are to be."""

    def __init__(self, c, tables):
        self.c, self.want = c, v.Lists(tables, c["n_pages"], c["page"])
        self.refs, self.taken = _at_fence(self.want.refs.copy()), _at_fence(self.want.taken())
        self.l = B.CkvLists(c["batch"], c["Hkv"], c["n_pages"], c["page"], c["most"], 0)
        self.l.table_stride[0], self.l.table_stride[1] = c["heads"] * c["most"], c["most"] if c["heads"] > 1 else 0

    def check(self, table, want):
        assert np.array_equal(table, want), "table"
        assert np.array_equal(self.refs, self.want.refs), "refs"
        assert np.array_equal(self.taken, self.want.taken()), "taken"


def _lists(path, c):
    lib = cpu.load(path)
    rng = np.random.default_rng(2)
    table, out = _at_fence(c["table"].copy()), _at_fence(c["table"][rng.integers(0, c["batch"], c["batch"])].copy())
    s = _State(c, [c["table"], out])
    parent = _at_fence(rng.integers(-1, c["batch"] + 1, c["batch"]).astype(np.int32))
    lengths, length_out = _at_fence(c["lengths"]), _at_fence(np.full_like(c["lengths"], 9))
    # lists become copies
    want_out, want = out.copy(), table.copy()
    s.want.fork(want, parent, want_out)
    for _ in range(2):   # the second time nothing changes
        assert lib.ckv_pages_fork(ref(s.l), P(table), P(parent), P(out), P(s.refs), P(s.taken), P(lengths), P(length_out), None) == B.CKV_OK
        s.check(out, want_out)
    alive = (parent >= 0) & (parent < c["batch"])
    assert np.array_equal(length_out, np.where(alive[:, None], c["lengths"][np.where(alive, parent, 0)], 0))
    assert lib.ckv_pages_fork(ref(s.l), P(table), P(parent), P(out), P(s.refs), P(s.taken), None, None, None) == B.CKV_OK
    s.check(out, want_out)
    # the former lists go
    s.want.free(want, None)
    assert lib.ckv_pages_free(ref(s.l), P(table), None, P(s.refs), P(s.taken), None) == B.CKV_OK
    s.check(table, want)
    # a few rows more for each of the copies: pages of their own, copies of shared ones; with too few places for pairs nothing happens
    for more, places in ((1, 0), (1, 3 * c["batch"] * c["heads"]), (2 * c["page"] + 1, 2 * c["batch"] * c["heads"] * 3)):
        first, end = _at_fence(length_out.copy()), _at_fence((length_out + more * (rng.random(length_out.shape) < 0.8)).astype(np.int32))
        copy, result = _at_fence(np.full((places, 2), 9, np.int32)) if places else None, _at_fence(np.full(2, 9, np.int32))
        want_copy, want_result = s.want.reserve(want_out, first, end, places)
        st = lib.ckv_pages_reserve(ref(s.l), P(out), P(first), P(end), P(s.refs), P(s.taken), P(copy), places, P(result), None)
        assert st == B.CKV_OK
        s.check(out, want_out)
        assert np.array_equal(result, want_result) and (copy is None or np.array_equal(copy, want_copy)), (result, want_result)
    # all rows are to be written, from the first on; odd bounds
    first, end = np.full_like(c["lengths"], -5), np.full_like(c["lengths"], 2 ** 31 - 1)
    first[0], end[0] = 7, 3
    want_copy, want_result = s.want.reserve(want_out, first, end, 4000)
    copy, result = _at_fence(np.full((4000, 2), 9, np.int32)), _at_fence(np.full(2, 9, np.int32))
    assert lib.ckv_pages_reserve(ref(s.l), P(out), P(_at_fence(first)), P(_at_fence(end)), P(s.refs), P(s.taken), P(copy), 4000, P(result), None) == B.CKV_OK
    s.check(out, want_out)
    assert np.array_equal(result, want_result) and np.array_equal(copy, want_copy)
    # back to fewer rows
    keep = (c["lengths"] * rng.random(c["lengths"].shape)).astype(np.int32) - 1
    s.want.free(want_out, keep)
    assert lib.ckv_pages_free(ref(s.l), P(out), P(_at_fence(keep)), P(s.refs), P(s.taken), None) == B.CKV_OK
    s.check(out, want_out)


@pytest.mark.parametrize("i", range(len(v.LISTS)))
def test_lists_share_get_and_give_back_pages(lib_path, i):
    in_child(_lists, lib_path, v.LISTS[i])


def _most_pages(path):
    lib, n = cpu.load(path), 2 ** 31 - 1
    l = B.CkvLists(1, 1, n, 16, 4, 0)
    l.table_stride[0] = l.table_stride[1] = 4
    table, copy, result = _at_fence(np.full((1, 4), -1, np.int32)), _at_fence(np.full((1, 2), 9, np.int32)), _at_fence(np.full(2, 9, np.int32))
    refs, taken = np.zeros(n, np.int32), np.zeros(2 ** 26, np.uint32)   # only what is written takes memory
    first, end = _at_fence(np.zeros((1, 1), np.int32)), _at_fence(np.full((1, 1), 40, np.int32))
    taken[0] = 0xfffffffd
    refs[0] = refs[2:32] = 1
    assert lib.ckv_pages_reserve(ref(l), P(table), P(first), P(end), P(refs), P(taken), P(copy), 1, P(result), None) == B.CKV_OK
    assert table.tolist() == [[1, 32, 33, -1]] and result.tolist() == [0, 0] and copy.tolist() == [[-1, -1]]
    assert taken[:2].tolist() == [2 ** 32 - 1, 3] and refs[[1, 32, 33]].tolist() == [1, 1, 1]


def test_as_many_pages_as_an_int32_holds(lib_path):
    in_child(_most_pages, lib_path)
