"""The entry points of trees, of rows and pages that move and of lists of pages refuse on the host what they cannot do, before anything would be launched."""
import ctypes
import re

import pytest
import torch

from paper_2602_08686_amd import binding as B
from test_abi_host import HEADER
from test_paged_host import AT, ODD, _pages, _params

ref = ctypes.byref
ALSO = ctypes.c_void_p(8192)


def _tree(**kw):
    g = lambda n, d=AT: kw.get(n, d)  # noqa: E731
    return B.load().ckv_paged_tree_attention(ref(g("p", _params())), ref(kw.get("pages", _pages())) if kw.get("pages", 1) else None, g("q"), g("kp"),
                                             g("vp"), g("table"), g("length"), None, kw.get("n_rows", 800), g("sees"), g("out"), kw.get("os"),
                                             g("lse", None), g("ws"), kw.get("ws_bytes", 1 << 40), None)


def _sees(batch=2, n=5, parent=AT, start=AT, sees=AT, positions=ALSO):
    return B.load().ckv_tree_sees(batch, n, parent, start, sees, positions, None)


def _compact(**kw):
    g = lambda n, d=AT: kw.get(n, d)  # noqa: E731
    return B.load().ckv_paged_compact(ref(g("p", _params())), ref(kw.get("pages", _pages())) if kw.get("pages", 1) else None, g("table"), g("length"),
                                      g("count", None), g("idx"), kw.get("stride"), kw.get("cap", 9), g("kept"), g("kp"), g("vp"),
                                      g("length_out", ALSO), None)


def _copy(**kw):
    g = lambda n, d=AT: kw.get(n, d)  # noqa: E731
    return B.load().ckv_pages_copy(ref(g("p", _params())), ref(kw.get("pages", _pages())) if kw.get("pages", 1) else None, g("copy"), kw.get("n", 3),
                                   g("kp"), g("vp"), None)


def _lists(**kw):
    l = B.CkvLists(3, 2, 100, 16, 50, 0)
    l.table_stride[0], l.table_stride[1] = 100, 50
    for name, value in kw.items():
        if isinstance(value, tuple):
            getattr(l, name)[value[0]] = value[1]
        else:
            setattr(l, name, value)
    return l


def _fork(l=None, **kw):
    g = lambda n, d=AT: kw.get(n, d)  # noqa: E731
    return B.load().ckv_pages_fork(ref(l) if l is not None else None, g("table"), g("parent"), g("out", ALSO), g("refs"), g("taken"), g("length"),
                                   g("length_out", ALSO), None)


def _reserve(l=None, **kw):
    g = lambda n, d=AT: kw.get(n, d)  # noqa: E731
    return B.load().ckv_pages_reserve(ref(l) if l is not None else None, g("table"), g("first"), g("end"), g("refs"), g("taken"), g("copy"),
                                      kw.get("n", 4), g("result"), None)


def _free(l=None, **kw):
    g = lambda n, d=AT: kw.get(n, d)  # noqa: E731
    return B.load().ckv_pages_free(ref(l) if l is not None else None, g("table"), g("keep"), g("refs"), g("taken"), None)


def test_struct_layout_matches_the_header():
    text = re.sub(r"/\*.*?\*/", "", HEADER.read_text(), flags=re.S)
    body = text[:text.index("} ckv_lists;")].rsplit("typedef struct {", 1)[1]
    assert re.findall(r"\b([a-z_]+)(?:\[\d\])?;", body) == [f[0] for f in B.CkvLists._fields_]
    assert ctypes.sizeof(B.CkvLists) == 24 + 16


def test_trees_are_refused():
    for kw in (dict(batch=0), dict(n=0), dict(parent=None), dict(sees=None), dict(start=None), dict(sees=ctypes.c_void_p(4100)), dict(positions=AT)):
        assert _sees(**kw) == B.CKV_EINVAL, kw
    assert _sees(n=4097) == B.CKV_EUNSUPPORTED
    assert _sees(batch=1 << 20, n=4096) == B.CKV_EUNSUPPORTED and _sees(batch=(1 << 22) + 1, n=1) == B.CKV_EUNSUPPORTED   # a launch's workgroups


def test_outputs_that_lie_where_other_workgroups_read():
    """Wholly or in part: a sequence's positions, a list's length are written while another one's inputs have still to be read."""
    at = lambda n: ctypes.c_void_p(1 << 16 | 4 * n)  # noqa: E731
    far = ctypes.c_void_p(1 << 20)
    for n, batch in ((5, 2), (700, 3)):
        assert _sees(batch, n, far, at(0), AT, at(0)) == B.CKV_EINVAL                                             # positions where start is
        for k in (1 - batch, batch * n - 1):
            assert _sees(batch, n, far, at(batch + k), AT, at(batch)) == B.CKV_EINVAL                              # ... its last, its first entry
        for k in (1 - batch * n, 0, batch * n - 1):
            assert _sees(batch, n, at(3 * batch * n + k), far, AT, at(3 * batch * n)) == B.CKV_EINVAL               # where parent is
    for name in ("length", "count", "kept"):
        for k in (-3, 0, 3):                                                                                       # of 2 x 2 entries
            assert _compact(**{name: at(8 + k)}, length_out=at(8)) == B.CKV_EINVAL, name
    l = _lists()
    for k in (-5, 0, 5):                                                                                           # of 3 x 2
        assert _fork(l, length=at(8 + k), length_out=at(8)) == B.CKV_EINVAL
    for k in (-2, 0, 5):
        assert _fork(l, parent=at(8 + k), length_out=at(8)) == B.CKV_EINVAL


def test_tree_attention_refuses():
    for name in ("q", "kp", "vp", "table", "length", "out", "sees"):
        assert _tree(**{name: None}) == B.CKV_EINVAL, name
    for name in ("q", "kp", "vp", "out"):
        assert _tree(**{name: ODD}) == B.CKV_EINVAL, name
    assert _tree(sees=ctypes.c_void_p(4100)) == B.CKV_EINVAL
    assert _tree(pages=None) == B.CKV_EINVAL
    assert _tree(n_rows=0) == B.CKV_EINVAL and _tree(n_rows=801) == B.CKV_EINVAL
    assert _tree(p=_params(d=80)) == B.CKV_EUNSUPPORTED
    assert _tree(p=_params(n=65537, n_q_heads=2)) == B.CKV_EUNSUPPORTED
    assert _tree(os=(ctypes.c_int64 * 3)(4096, 512, 64)) == B.CKV_EINVAL
    p, pages = _params(n=40), _pages(max_pages=1 << 12)
    need = B.ckv_paged_workspace_bytes(p, 1 << 16)
    call = lambda **kw: _tree(p=p, pages=pages, n_rows=1 << 16, **kw)  # noqa: E731
    assert need > 0 and call(ws=None) == B.CKV_EWORKSPACE and call(ws_bytes=need // 4) == B.CKV_EWORKSPACE
    assert call(ws=ctypes.c_void_p(4096 + 16)) == B.CKV_EWORKSPACE


def test_compact_refuses():
    for name in ("table", "length", "idx", "kept", "kp", "vp", "length_out"):
        assert _compact(**{name: None}) == B.CKV_EINVAL, name
    assert _compact(kp=ODD) == B.CKV_EINVAL and _compact(vp=ODD) == B.CKV_EINVAL
    assert _compact(pages=None) == B.CKV_EINVAL and _compact(cap=0) == B.CKV_EINVAL
    assert _compact(length_out=AT) == B.CKV_EINVAL                                    # the lengths that are read
    for name in ("length", "count", "kept"):
        assert _compact(**{name: ALSO}) == B.CKV_EINVAL, name                         # what is written
    assert _compact(stride=(ctypes.c_int64 * 2)(-1, 0)) == B.CKV_EINVAL and _compact(stride=(ctypes.c_int64 * 2)(9, -9)) == B.CKV_EINVAL
    assert _compact(p=_params(d=96)) == B.CKV_EUNSUPPORTED
    assert _compact(p=_params(batch=(1 << 16) + 1, n_q_heads=4)) == B.CKV_EUNSUPPORTED   # a launch's workgroups
    assert _compact(pages=_pages(page_rows=24)) == B.CKV_EUNSUPPORTED and _compact(pages=_pages(k_stride=(2, 64))) == B.CKV_EINVAL


def test_rows_of_one_head_under_one_list_do_not_move():
    """Every head would move the same rows, the second one those that the first has moved."""
    one = dict(table_stride=(1, 0))
    assert _compact(pages=_pages(k_stride=(1, 0), v_stride=(1, 0), **one)) == B.CKV_EINVAL
    assert _compact(pages=_pages(k_stride=(1, 0), **one)) == B.CKV_EINVAL and _compact(pages=_pages(v_stride=(1, 0), **one)) == B.CKV_EINVAL
    for fine in (dict(k_stride=(1, 0), table_stride=(1, 50)), one):   # lists of their own; pages that hold every head: as far as the next refusal
        assert _compact(pages=_pages(page_rows=24, **fine)) == B.CKV_EUNSUPPORTED, fine


def test_copy_refuses():
    for name in ("copy", "kp", "vp"):
        assert _copy(**{name: None}) == B.CKV_EINVAL, name
    assert _copy(kp=ODD) == B.CKV_EINVAL and _copy(n=-1) == B.CKV_EINVAL and _copy(pages=None) == B.CKV_EINVAL
    assert _copy(n=0) == B.CKV_OK                                                      # nothing to launch
    assert _copy(pages=_pages(page_rows=12)) == B.CKV_EUNSUPPORTED and _copy(p=_params(d=32)) == B.CKV_EUNSUPPORTED
    assert _copy(n=1 << 30) == B.CKV_EUNSUPPORTED                                      # more workgroups than a launch has
    assert _copy(pages=_pages(page_rows=1 << 16, max_pages=1), p=_params(n_q_heads=4096, n_kv_heads=4096)) == B.CKV_EUNSUPPORTED


@pytest.mark.parametrize("bad,status", [
    (dict(batch=0), B.CKV_EINVAL), (dict(n_kv_heads=0), B.CKV_EINVAL), (dict(n_pages=0), B.CKV_EINVAL), (dict(page_rows=0), B.CKV_EINVAL),
    (dict(max_pages=0), B.CKV_EINVAL), (dict(reserved=1), B.CKV_EINVAL), (dict(table_stride=(0, -1)), B.CKV_EINVAL),
    (dict(table_stride=(1, -50)), B.CKV_EINVAL), (dict(table_stride=(1, 49)), B.CKV_EINVAL), (dict(table_stride=(0, 49)), B.CKV_EINVAL),
    (dict(page_rows=24), B.CKV_EUNSUPPORTED), (dict(page_rows=1 << 17), B.CKV_EUNSUPPORTED), (dict(max_pages=1 << 28, table_stride=(1, 0)), B.CKV_EINVAL),
    (dict(batch=1 << 28), B.CKV_EUNSUPPORTED), (dict(batch=(1 << 21) + 1, max_pages=1), B.CKV_EUNSUPPORTED),
])
def test_lists_are_refused(bad, status):
    l = _lists(**bad)
    assert _fork(l) == status and _reserve(l) == status and _free(l) == status


def test_calls_on_lists_refuse():
    l = _lists()
    assert _fork() == B.CKV_EINVAL and _reserve() == B.CKV_EINVAL and _free() == B.CKV_EINVAL
    for name in ("table", "parent", "out", "refs", "taken", "length", "length_out"):
        assert _fork(l, **{name: None}) == B.CKV_EINVAL, name                            # length without its output, too
    assert _fork(l, out=AT) == B.CKV_EINVAL and _fork(l, length_out=AT) == B.CKV_EINVAL  # in place
    assert _fork(l, parent=ALSO) == B.CKV_EINVAL
    for name in ("table", "first", "end", "refs", "taken", "copy", "result"):
        assert _reserve(l, **{name: None}) == B.CKV_EINVAL, name
    assert _reserve(l, n=-1) == B.CKV_EINVAL and _reserve(l, n=1 << 30) == B.CKV_EUNSUPPORTED
    for name in ("table", "refs", "taken"):
        assert _free(l, **{name: None}) == B.CKV_EINVAL, name


def test_helpers_describe_tensors():
    table = torch.zeros(3, 2, 50, dtype=torch.int32)
    l = B.lists_for(table, n_kv_heads=2, n_pages=100, page_rows=16)
    assert bytes(l) == bytes(_lists())
    l = B.lists_for(table[:, 0], n_kv_heads=8, n_pages=100, page_rows=16)
    assert (l.n_kv_heads, list(l.table_stride)) == (8, [100, 0])
    l = B.lists_for(table[:1, :1], n_kv_heads=1, n_pages=100, page_rows=16)              # axes of one entry
    assert list(l.table_stride) == [50, 50]
    for bad in (lambda: B.lists_for(table.long(), n_kv_heads=2, n_pages=9, page_rows=1), lambda: B.lists_for(table, n_kv_heads=3, n_pages=9, page_rows=1),
                lambda: B.lists_for(table[..., ::2], n_kv_heads=2, n_pages=9, page_rows=1), lambda: B.lists_for(table[0, 0], n_kv_heads=1, n_pages=9, page_rows=1),
                lambda: B.pool_params(torch.zeros(4, 2, 64), table), lambda: B.pool_params(torch.zeros(4, 2, 16, 64), table[0, 0])):
        with pytest.raises(ValueError):
            bad()
    p = B.pool_params(torch.zeros(7, 5, 16, 64, dtype=torch.bfloat16), table)
    assert (p.batch, p.n_q_heads, p.n_kv_heads, p.head_dim, p.dtype) == (3, 5, 5, 64, B.CKV_BF16)
    refs, taken = B.page_counts(70, device="cpu")
    assert refs.shape == (70,) and taken.shape == (3,) and not refs.any() and not taken.any()
