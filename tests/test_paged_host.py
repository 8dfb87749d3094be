"""The paged cache's entry points refuse on the host what they cannot do, before anything would be launched."""
import ctypes
import re

import pytest
import torch

import paged_util as u
from paper_2602_08686_amd import binding as B
from test_abi_host import HEADER

ref = ctypes.byref
AT = ctypes.c_void_p(4096)     # never dereferenced: validation fails first
ODD = ctypes.c_void_p(4104)


def _params(n=4, dtype=torch.bfloat16, d=128, **kw):
    base = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=d, seq_len=n, window=1, dtype=dtype, pool=B.POOL_NONE, pool_kernel=1,
                budget=1, cap=1)
    base.update(kw)
    return B.make_params(**base)


def _pages(**kw):
    p = B.CkvPages(16, 100, 50, 0)
    for arr in (p.k_stride, p.v_stride):
        arr[0], arr[1], arr[2] = 2 * 16 * 128, 16 * 128, 128
    p.table_stride[0] = 50
    for name, value in kw.items():
        if isinstance(value, tuple):
            getattr(p, name)[value[0]] = value[1]
        else:
            setattr(p, name, value)
    return p


def _rotate(**kw):
    g = lambda n, d=AT: kw.get(n, d)  # noqa: E731
    return B.load().ckv_norm_rotate(ref(g("p", _params())), None if g("rot") is None else ref(g("rot", B.make_rotation(128, norm=True))),
                                    g("q"), g("k"), g("pos"), g("freq"), g("qw", None), g("kw", None), None, g("q_out"), g("k_out"), None)


def _append(**kw):
    g = lambda n, d=AT: kw.get(n, d)  # noqa: E731
    rot = kw.get("rot", B.make_rotation(128))
    return B.load().ckv_paged_append(ref(g("p", _params())), None if rot is None else ref(rot), ref(kw.get("pages", _pages())) if kw.get("pages", 1) else None,
                                     g("q"), g("k"), g("v"), g("pos"), g("freq"), g("qw", None), g("kw", None), g("table"), g("length"), None,
                                     g("kp"), g("vp"), g("q_out"), None)


def _attend(**kw):
    g = lambda n, d=AT: kw.get(n, d)  # noqa: E731
    return B.load().ckv_paged_attention(ref(g("p", _params())), ref(kw.get("pages", _pages())) if kw.get("pages", 1) else None, g("q"), g("kp"),
                                        g("vp"), g("table"), g("length"), None, kw.get("n_rows", 800), g("out"), kw.get("os"), g("lse", None),
                                        g("ws"), kw.get("ws_bytes", 1 << 40), None)


def test_struct_layouts_match_the_header():
    text = re.sub(r"/\*.*?\*/", "", HEADER.read_text(), flags=re.S)
    for name, struct, size in (("ckv_pages", B.CkvPages, 16 + 64), ("ckv_rotation", B.CkvRotation, 16)):
        body = text[:text.index(f"}} {name};")].rsplit("typedef struct {", 1)[1]
        assert re.findall(r"\b([a-z_]+)(?:\[\d\])?;", body) == [f[0] for f in struct._fields_]
        assert ctypes.sizeof(struct) == size


def test_norm_rotate_refuses():
    for name in ("q", "k", "q_out", "k_out"):
        assert _rotate(**{name: None}) == B.CKV_EINVAL        # an input without its output or the other way round
        assert _rotate(**{name: ODD}) == B.CKV_EINVAL
    assert _rotate(q=None, q_out=None, k=None, k_out=None) == B.CKV_EINVAL
    assert _rotate(pos=None) == B.CKV_EINVAL and _rotate(freq=None) == B.CKV_EINVAL
    assert _rotate(qw=ODD) == B.CKV_EINVAL and _rotate(kw=ODD) == B.CKV_EINVAL
    assert B.load().ckv_norm_rotate(ref(_params()), None, AT, AT, AT, AT, None, None, None, AT, AT, None) == B.CKV_EINVAL
    for bad in (dict(rot_dim=-8), dict(rot_dim=136), dict(rot_dim=9), dict(rot_dim=64, pairing=2), dict(rot_dim=64, norm_eps=-1.0),
                dict(rot_dim=64, norm_eps=float("nan")), dict(rot_dim=64, norm_eps=float("inf"))):
        assert _rotate(rot=B.make_rotation(**bad)) == B.CKV_EINVAL, bad
    assert _rotate(rot=B.CkvRotation(64, 0, 2, 1e-6)) == B.CKV_EINVAL
    assert _rotate(rot=B.make_rotation(12)) == B.CKV_EUNSUPPORTED
    assert _rotate(p=_params(d=96)) == B.CKV_EUNSUPPORTED
    assert _rotate(p=_params(q_stride=(4096, 1024, 100))) == B.CKV_EINVAL
    assert _rotate(p=_params(n=1 << 24, batch=32, n_q_heads=2)) == B.CKV_EUNSUPPORTED   # more workgroups than a launch has


@pytest.mark.parametrize("bad,status", [
    (dict(page_rows=0), B.CKV_EINVAL), (dict(n_pages=0), B.CKV_EINVAL), (dict(max_pages=0), B.CKV_EINVAL), (dict(reserved=1), B.CKV_EINVAL),
    (dict(k_stride=(0, -4096)), B.CKV_EINVAL), (dict(v_stride=(1, 2050)), B.CKV_EINVAL), (dict(k_stride=(2, 64)), B.CKV_EINVAL),
    (dict(v_stride=(0, 0)), B.CKV_EINVAL), (dict(table_stride=(0, -1)), B.CKV_EINVAL), (dict(table_stride=(1, -1)), B.CKV_EINVAL),
    (dict(page_rows=24), B.CKV_EUNSUPPORTED), (dict(page_rows=1 << 17), B.CKV_EUNSUPPORTED),
    (dict(page_rows=1 << 16, max_pages=1 << 15), B.CKV_EUNSUPPORTED),
])
def test_pages_are_refused(bad, status):
    assert _append(pages=_pages(**bad)) == status
    assert _attend(pages=_pages(**bad)) == status


def test_append_refuses():
    for name in ("k", "v", "table", "length", "kp", "vp", "q_out"):
        assert _append(**{name: None}) == B.CKV_EINVAL, name
    assert _append(q=None) == B.CKV_EINVAL                     # q_out without q
    for name in ("q", "k", "v", "kp", "vp", "q_out"):
        assert _append(**{name: ODD}) == B.CKV_EINVAL, name
    assert _append(pages=None) == B.CKV_EINVAL
    assert _append(pos=None) == B.CKV_EINVAL and _append(freq=None) == B.CKV_EINVAL
    assert _append(rot=B.make_rotation(20)) == B.CKV_EUNSUPPORTED
    assert _append(p=_params(n=1 << 24, batch=32, n_q_heads=2)) == B.CKV_EUNSUPPORTED


def test_attention_refuses():
    for name in ("q", "kp", "vp", "table", "length", "out"):
        assert _attend(**{name: None}) == B.CKV_EINVAL, name
    for name in ("q", "kp", "vp", "out"):
        assert _attend(**{name: ODD}) == B.CKV_EINVAL, name
    assert _attend(pages=None) == B.CKV_EINVAL
    assert _attend(n_rows=0) == B.CKV_EINVAL and _attend(n_rows=801) == B.CKV_EINVAL     # 50 pages of 16 rows
    assert _attend(pages=_pages(max_pages=1 << 21), n_rows=(1 << 24) + 1) == B.CKV_EUNSUPPORTED
    stride = lambda *s: (ctypes.c_int64 * 3)(*s)  # noqa: E731
    assert _attend(os=stride(4096, 512, 64)) == B.CKV_EINVAL                             # tokens would lie over one another
    assert _attend(os=stride(4096, 0, 128)) == B.CKV_EINVAL and _attend(os=stride(4096, 516, 128)) == B.CKV_EINVAL
    assert _attend(p=_params(d=80)) == B.CKV_EUNSUPPORTED
    assert _attend(p=_params(softmax_scale=-1.0)) == B.CKV_EINVAL
    assert _attend(p=_params(n=1 << 22, batch=32, n_q_heads=64, n_kv_heads=64), pages=_pages(max_pages=1 << 19), n_rows=1 << 23) == B.CKV_EUNSUPPORTED


def test_attention_workspace():
    p, pages = _params(n=1), _pages(max_pages=1 << 12)
    need = B.ckv_paged_workspace_bytes(p, 1 << 16)
    assert need > 0 and need % 256 == 0
    call = lambda **kw: _attend(p=p, pages=pages, n_rows=1 << 16, **kw)  # noqa: E731
    assert call(ws=None) == B.CKV_EWORKSPACE and call(ws_bytes=need // 2) == B.CKV_EWORKSPACE
    assert call(ws=ctypes.c_void_p(4096 + 16)) == B.CKV_EWORKSPACE
    assert B.ckv_paged_workspace_bytes(p, 0) == 0 and B.ckv_paged_workspace_bytes(p, (1 << 24) + 1) == 0
    assert B.ckv_paged_workspace_bytes(_params(d=96), 100) == 0
    assert B.ckv_paged_workspace_bytes(p, 1) == 0              # one workgroup finishes a short list
    for n in (1, 2, 17, 300, 5000):                            # bounded: as much as some hundred workgroups leave
        for rows in (1, 100, 5000, 1 << 20):
            assert B.ckv_paged_workspace_bytes(_params(n=n), rows) <= 512 << 20


def test_helpers_describe_tensors():
    c = u.case(n=3, lengths=((20, 20), (5, 5)), page=4, pool_token_major=True)
    s = u.make(c)
    t = {n: torch.from_numpy(x.view("int16") if x.dtype == "uint16" else x) if x is not None else None for n, x in s.items()}
    t = {n: x.view(torch.bfloat16) if x is not None and x.dtype == torch.int16 else x for n, x in t.items()}
    p, want = B.step_params(q=t["q"], k=t["k"], v=t["v"], n_q_heads=8, n_kv_heads=2), u.params(c, s)
    for f, _ in B.CkvParams._fields_:
        got, w = getattr(p, f), getattr(want, f)
        assert (list(got) == list(w)) if hasattr(got, "__len__") else got == w, f
    got, w = B.pages_for(t["k_pages"], t["v_pages"], t["table"]), u.pages(c, s)
    assert bytes(got) == bytes(w)
    with pytest.raises(ValueError):
        B.step_params(n_q_heads=8, n_kv_heads=2)
    with pytest.raises(ValueError):
        B.step_params(q=t["q"], k=t["k"][:, :, :2], n_q_heads=8, n_kv_heads=2)
    with pytest.raises(ValueError):
        B.step_params(q=t["q"], n_q_heads=4, n_kv_heads=2)
    with pytest.raises(ValueError):
        B.pages_for(t["k_pages"], t["v_pages"], t["table"].long())
    with pytest.raises(ValueError):
        B.pages_for(t["k_pages"], t["v_pages"][:, :1], t["table"])
    # one token per sequence: whatever stride torch gives the axis, the library gets one that it takes
    one = torch.zeros(2, 8, 128, dtype=torch.bfloat16)[:, :, None]
    assert B.step_params(q=one.as_strided(one.shape, (1024, 128, 1, 1)), n_q_heads=8, n_kv_heads=2).q_stride[2] == 128


def test_an_output_without_a_contiguous_last_axis_is_refused():
    p, pages = B.CkvParams(), B.CkvPages()
    for out in (torch.empty(1, 4, 128, 3).transpose(2, 3), torch.empty(4, 6, 128)[:, ::2]):
        with pytest.raises(ValueError):
            B.ckv_paged_attention(p, pages, None, None, None, None, None, 1, out)
