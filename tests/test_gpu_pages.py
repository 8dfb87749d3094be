"""Trees of drafted tokens, rows and pages that move and lists that share pages on the GPU, against results in 64 bits (pages_util holds the definitions);
a serving loop of all of them, eager, on streams of its own and replayed from graphs."""
import numpy as np
import pytest
import torch

import paged_util as u
import pages_util as v
from paper_2602_08686_amd import binding as B
from test_gpu_paged import DEV, gpu, host, nines, on_gpu

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


# ---- trees ------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["chain", "star", "roots", "odd", "random"])
@pytest.mark.parametrize("batch,n", [(1, 1), (16, 24), (3, 64), (2, 65), (3, 300), (2, 1000)])
def test_tokens_see_their_paths(kind, batch, n):
    parent = v.parents(kind, batch, n)
    sees, depth = v.paths(parent)
    start = np.arange(batch, dtype=np.int32) * 70000 - 5
    words, positions = (torch.full(s, 9, dtype=t, device=DEV) for s, t in (((batch, n, -(-n // 64)), torch.int64), ((batch, n), torch.int32)))
    B.ckv_tree_sees(ints(parent), ints(start), words, positions)
    alone = torch.full_like(words, 9)
    B.ckv_tree_sees(ints(parent), None, alone)
    torch.cuda.synchronize()
    assert np.array_equal(words.cpu(), v.words(sees)) and torch.equal(alone, words)
    assert np.array_equal(positions.cpu(), start[:, None] + depth)


@pytest.mark.parametrize("kind", ["star", "odd", "random"])
@pytest.mark.parametrize("batch,n", [(2, 1025), (1, 2500), (1, 4096)])
def test_long_trees_that_branch(kind, batch, n):
    parent = v.parents(kind, batch, n)
    sees, depth = v.paths(parent)
    words, positions = torch.full((batch, n, -(-n // 64)), 9, dtype=torch.int64, device=DEV), torch.full((batch, n), 9, dtype=torch.int32, device=DEV)
    B.ckv_tree_sees(ints(parent), ints(np.arange(batch, dtype=np.int32)), words, positions)
    torch.cuda.synchronize()
    assert np.array_equal(words.cpu(), v.words(sees)) and np.array_equal(positions.cpu(), np.arange(batch)[:, None] + depth)


def test_the_longest_path():
    parent = v.parents("chain", 2, 4096)
    words = torch.zeros(2, 4096, 64, dtype=torch.int64, device=DEV)
    positions = torch.zeros(2, 4096, dtype=torch.int32, device=DEV)
    B.ckv_tree_sees(ints(parent), ints(np.zeros(2, np.int32)), words, positions)
    torch.cuda.synchronize()
    assert np.array_equal(positions.cpu()[1], np.arange(4096))
    assert np.array_equal(words.cpu()[1], v.words(np.tril(np.ones((4096, 4096), bool))))


def attend(c, t, out=None, lse=None, stream=None):
    out = nines(c, c["Hq"]) if out is None else out
    lse = torch.full((c["batch"], c["Hq"], c["n"]), 9.0, device=DEV) if lse is None else lse
    B.ckv_paged_tree_attention(t["params"], t["pages"], t["q"], t["k_pages"], t["v_pages"], t["table"], t["length"], t["n_rows"], t["sees"], out, lse,
                               t["ws"], count=t["count"], stream=stream)
    return out, lse


def tree_on_gpu(c, s):
    return dict(on_gpu(c, s), sees=ints(v.words(c["sees"])))


def check(c, s, out, lse):
    want, tol, wl, lt = v.attention(c, s)
    old = np.arange(c["n"]) >= np.repeat(u.new_counts(c), c["Hq"] // c["Hkv"], 1)[..., None]
    u.check(host(out), np.where(old[..., None], 9.0, want), tol, "out")
    u.check(host(lse), np.where(old, 9.0, wl), lt, "lse")


LONG = v.MANY


@pytest.mark.parametrize("i", range(len(v.TREES) + len(LONG)))
def test_attention_of_trees(i):
    c = (v.TREES + LONG)[i]
    s = u.make(c)
    t = tree_on_gpu(c, s)
    out, lse = attend(c, t)
    torch.cuda.synchronize()
    check(c, s, out, lse)
    again = attend(c, t)
    wide = nines(c, c["Hq"]).transpose(1, 2).contiguous().transpose(1, 2)   # token by token, and without lse
    B.ckv_paged_tree_attention(t["params"], t["pages"], t["q"], t["k_pages"], t["v_pages"], t["table"], t["length"], t["n_rows"], t["sees"], wide, None,
                               t["ws"], count=t["count"])
    torch.cuda.synchronize()
    assert torch.equal(again[0], out) and torch.equal(again[1], lse) and torch.equal(wide, out)


@pytest.mark.parametrize("i", [2, 5, 12, 19])
def test_a_chain_is_the_causal_order(i):
    """Few columns (the first and the third case): the same kernel but for the mask, and the same bits. Many: the calls share the rows out differently,
    so that the same terms are added in another order; both are held to 64 bits, with tolerances that hold for any order of the sums."""
    c = v.TREES[i]
    c = dict(c, sees=v.paths(v.parents("chain", c["batch"], c["n"]))[0])
    s = u.make(c)
    t = tree_on_gpu(c, s)
    out, lse = attend(c, t)
    causal, also = nines(c, c["Hq"]), torch.full_like(lse, 9.0)
    B.ckv_paged_attention(t["params"], t["pages"], t["q"], t["k_pages"], t["v_pages"], t["table"], t["length"], t["n_rows"], causal, also, t["ws"],
                          count=t["count"])
    torch.cuda.synchronize()
    check(c, s, out, lse)
    check(c, s, causal, also)
    assert i in (5, 19) or torch.equal(out, causal) and torch.equal(lse, also)


@pytest.mark.parametrize("kind", ["bad_pages", "nan", "infinity"])
@pytest.mark.parametrize("i", [1, 4, 5, 8, 12, 15, 18, 19, 20, 22])
def test_what_a_token_does_not_see_has_no_influence(i, kind):
    c = (v.TREES + LONG)[i]
    s = u.make(c)
    if kind == "bad_pages":
        table = s["table"].reshape(-1, s["table"].shape[-1])
        table[0, 0], table[-1, table.shape[1] // 2] = s["k_pages"].shape[0], -7
    else:
        rng = np.random.default_rng(3)
        for m in ("k_pages", "v_pages"):
            x = np.array(u.values(s[m]))
            for b, g in np.ndindex(c["lengths"].shape):
                length, count = int(c["lengths"][b, g]), int(u.new_counts(c)[b, g])
                for row in range(max(0, length - count), length):
                    at, h = u.place(c, s, b, g, row), 0 if c["by_head"] else g
                    if rng.random() < 0.3:
                        if kind == "nan":
                            x[at[0], h, at[1]] = np.nan
                        elif m == "v_pages":
                            x[at[0], h, at[1], ::3], x[at[0], h, at[1], 1] = np.inf, -np.inf
            s[m] = u.stored(x, c["dtype"])
    t = tree_on_gpu(c, s)
    out, lse = attend(c, t)
    torch.cuda.synchronize()
    check(c, s, out, lse)


@pytest.mark.parametrize("n,d", [(60, 128), (2, 128), (20, 64), (80, 64)])
def test_a_bound_far_above_the_lengths(n, d):
    """A call that was planned for long lists (a graph, say) on short ones, down to none."""
    for lengths, counts in ((((n + 40, n + 9),), ((n, n),)), (((1, 1),), ((1, 1),)), (((0, 0),), ((n, 0),)), (((700, 2),), ((n, 2),)), (((9000, n),), ((n, n),))):
        c = v.tree_case("random", n=n, d=d, heads=(8, 2), lengths=lengths, counts=counts, page=16)
        s = u.make(c)
        s["table"] = np.concatenate([s["table"], np.full((1, 16000 - s["table"].shape[1]), -1, np.int32)], 1)
        t = tree_on_gpu(c, s)
        assert t["n_rows"] == 256000 and t["ws"] is not None
        out, lse = attend(c, t)
        torch.cuda.synchronize()
        check(c, dict(s, table=s["table"][:, :600]), out, lse)


def test_lengths_behind_the_bound_and_below_zero():
    """Lists that say they are longer than the call looks, by a little and by far: none of the drafted tokens' rows is seen, or some are."""
    c = v.tree_case("random", n=30, heads=(4, 2), lengths=((300, 280),), page=16)
    s = u.make(c)
    for lengths, n_rows in (((300, 280), 290), ((300, 280), 271), ((2 ** 31 - 1, 280), 280), ((-5, -2 ** 31), 300)):
        d = dict(c, lengths=np.array([lengths], np.int32), n_rows=n_rows)
        t = tree_on_gpu(dict(c, n_rows=n_rows), s)
        t["length"] = ints(d["lengths"])
        out, lse = attend(d, t)
        torch.cuda.synchronize()
        want = v.attention(dict(d, lengths=np.minimum(d["lengths"], 1 << 20)), s)   # (rows behind the bound are not looked at)
        u.check(host(out), want[0], want[1], "out")
        u.check(host(lse), want[2], want[3], "lse")


# ---- rows and pages that move -------------------------------------------------------------------------------------------------
def same(got, want, what):
    want = gpu(np.ascontiguousarray(want))
    kind = torch.int16 if want.dtype == torch.bfloat16 else torch.int32
    assert torch.equal(got.contiguous().view(kind), want.view(kind)), what


MOVES = v.MOVES + [
    (u.case(n=1, heads=(8, 8), lengths=((5000,) * 8,) * 2, page=16), 600, 544, True),
    (u.case(n=1, heads=(2, 2), lengths=((9000, 9000),), page=64), 8000, 7900, True),                       # many rounds
    (u.case(dtype="f32", n=1, heads=(2, 2), lengths=((6000, 5000),), by_head=True, page=128, pool_token_major=True), 5500, 4900, True),
    (u.case(n=1, heads=(8, 8), lengths=tuple((20011 - 97 * b,) * 8 for b in range(4)), counts=((60,) * 8,) * 4, page=16), 12, 9, False),
]


@pytest.mark.parametrize("i", range(len(MOVES)))
def test_rows_that_stay_move_together(i):
    c, cap, kept, each_head = MOVES[i]
    s = u.make(c)
    idx, stay = v.chosen(c, cap, kept, each_head)
    want, length_out = v.compacted(c, s, idx, stay)
    t = on_gpu(c, s)
    got = torch.full_like(t["length"], 9)
    B.ckv_paged_compact(B.pool_params(t["k_pages"], t["table"]), t["pages"], t["k_pages"], t["v_pages"], t["table"], t["length"], ints(idx), ints(stay), got,
                        count=t["count"])
    torch.cuda.synchronize()
    for m in ("k_pages", "v_pages"):
        same(t[m + "_all"], want[m], m)
    assert np.array_equal(got.cpu(), length_out)


@pytest.mark.parametrize("kw,pairs", [
    (dict(lengths=((300, 300),), page=16), 8), (dict(lengths=((60, 60),), page=64, pool_token_major=True, spare=7), 4),
    (dict(heads=(3, 3), lengths=((40, 30, 20),), page=1), 40), (dict(heads=(4, 4), lengths=((90, 90, 90, 90),), page=32, by_head=True), 5),
    (dict(dtype="f32", d=64, heads=(5, 5), lengths=((90,) * 5,), page=8), 5), (dict(dtype="f32", lengths=((600, 600),), page=256, spare=9), 5),
    (dict(lengths=((40000, 40000),), page=16), 1200)])
def test_pages_are_copied(kw, pairs):
    c = u.case(**kw)
    s = u.make(c)
    n = s["k_pages"].shape[0]
    ids = np.random.default_rng(1).permutation(n)[:2 * pairs].reshape(-1, 2).astype(np.int32)
    odd = np.array([[-1, -1], [0, n], [n, 0], [3, 3], [-1, 2]], np.int32)
    t = on_gpu(c, s)
    B.ckv_pages_copy(t["params"], t["pages"], t["k_pages"], t["v_pages"], ints(np.concatenate([odd[:2], ids, odd[2:]])))
    B.ckv_pages_copy(t["params"], t["pages"], t["k_pages"], t["v_pages"], torch.zeros(0, 2, dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    for m in ("k_pages", "v_pages"):
        want = np.array(s[m])
        want[ids[:, 1]] = want[ids[:, 0]]
        same(t[m + "_all"], want, m)


def test_pages_and_rows_far_apart_in_a_large_pool():
    """Beyond 2^32 bytes and 2^31 elements of the pools."""
    d, page, n_pages = 128, 64, 270000                      # 4.4 GB a pool
    pools = [torch.zeros(n_pages, 1, page, d, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    for x in pools:
        x[n_pages - 1] = torch.randn(1, page, d, device=DEV).bfloat16()
    table = ints(np.array([[n_pages - 1, 0, n_pages - 2]], np.int32))
    p, pages = B.pool_params(pools[0], table), B.pages_for(*pools, table)
    keep = [x[n_pages - 1].clone() for x in pools]
    B.ckv_pages_copy(p, pages, *pools, ints(np.array([[n_pages - 1, n_pages - 2]], np.int32)))
    idx = ints(np.arange(128, 138, dtype=np.int32)[None])   # rows of the last page to the front
    length_out = ints(np.zeros((1, 1), np.int32))
    B.ckv_paged_compact(p, pages, *pools, table, ints(np.array([[150]], np.int32)), idx, ints(np.array([[10]], np.int32)), length_out)
    torch.cuda.synchronize()
    for x, k in zip(pools, keep):
        assert torch.equal(x[n_pages - 2], k) and torch.equal(x[n_pages - 1, 0, :10], k[0, :10]) and not x[1:n_pages - 2].any()
    assert length_out.item() == 10


# ---- lists ------------------------------------------------------------------------------------------------------------------
class State:
    """Counts and bits on the GPU beside what they are to be."""

    def __init__(self, c, tables):
        self.want = v.Lists(tables, c["n_pages"], c["page"])
        self.refs, self.taken = ints(self.want.refs), ints(self.want.taken())

    def check(self, table, want):
        assert np.array_equal(table.cpu().numpy().reshape(want.shape), want), "table"
        assert np.array_equal(self.refs.cpu(), self.want.refs), "refs"
        assert np.array_equal(self.taken.cpu(), self.want.taken()), "taken"


LISTS = v.LISTS + [v.list_case(batch=32, heads=1, Hkv=8, page=16, most=2050, n_pages=70000, seed=8, common=500)]


@pytest.mark.parametrize("i", range(len(LISTS)))
def test_lists_share_get_and_give_back_pages(i):
    c, rng = LISTS[i], np.random.default_rng(2)
    former = c["table"][rng.integers(0, c["batch"], c["batch"])]
    shape = c["table"].shape if c["heads"] > 1 else (c["batch"], c["most"])
    table, out = ints(c["table"].reshape(shape)), ints(former.reshape(shape))
    lists = B.lists_for(table, n_kv_heads=c["Hkv"], n_pages=c["n_pages"], page_rows=c["page"])
    s = State(c, [c["table"], former])
    parent = rng.integers(-1, c["batch"] + 1, c["batch"]).astype(np.int32)
    length, length_out = ints(c["lengths"]), ints(np.full_like(c["lengths"], 9))
    want, want_out = c["table"].copy(), former.copy()
    s.want.fork(want, parent, want_out)
    for _ in range(3):
        B.ckv_pages_fork(lists, table, ints(parent), out, s.refs, s.taken, length, length_out)
        s.check(out, want_out)
    alive = (parent >= 0) & (parent < c["batch"])
    rows = np.where(alive[:, None], c["lengths"][np.where(alive, parent, 0)], 0)
    assert np.array_equal(length_out.cpu(), rows)
    s.want.free(want, None)
    B.ckv_pages_free(lists, table, None, s.refs, s.taken)
    s.check(table, want)
    result = ints(np.full(2, 9, np.int32))
    for more, places in ((1, 0), (1, 3 * c["batch"] * c["heads"]), (2 * c["page"] + 1, 6 * c["batch"] * c["heads"])):
        end = (rows + more * (rng.random(rows.shape) < 0.8)).astype(np.int32)
        copy = ints(np.full((places, 2), 9, np.int32)) if places else None
        want_copy, want_result = s.want.reserve(want_out, rows, end, places)
        B.ckv_pages_reserve(lists, out, length_out, ints(end), s.refs, s.taken, copy, result)
        s.check(out, want_out)
        assert np.array_equal(result.cpu(), want_result) and (copy is None or np.array_equal(copy.cpu(), want_copy))
    first, end = np.full_like(rows, -5), np.full_like(rows, 2 ** 31 - 1)
    first[0], end[0] = 7, 3
    copy = ints(np.full((4000, 2), 9, np.int32))
    want_copy, want_result = s.want.reserve(want_out, first, end, 4000)
    B.ckv_pages_reserve(lists, out, ints(first), ints(end), s.refs, s.taken, copy, result)
    s.check(out, want_out)
    assert np.array_equal(result.cpu(), want_result) and np.array_equal(copy.cpu(), want_copy)
    keep = (c["lengths"] * rng.random(rows.shape)).astype(np.int32) - 1
    s.want.free(want_out, keep)
    B.ckv_pages_free(lists, out, ints(keep), s.refs, s.taken)
    s.check(out, want_out)
