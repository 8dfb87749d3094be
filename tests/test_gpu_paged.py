"""The paged cache's calls on the GPU against 64 bits (paged_util holds the definitions and the tolerances), and a prompt's way through all of
them: norm and rotation, the append, chunked attention whose lse feeds the retention step, the kept rows into lists of their own,
decoding over those."""
import ctypes

import numpy as np
import pytest
import torch

import paged_util as u
from paper_2602_08686_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"


def gpu(x):
    """A numpy array on the GPU, its layout kept."""
    if x is None:
        return None
    order = sorted(range(x.ndim), key=lambda i: -x.strides[i])
    base = np.ascontiguousarray(x.transpose(order))
    t = torch.from_numpy(base.view(np.int16) if base.dtype == np.uint16 else base.copy()).to(DEV)
    t = t.view(torch.bfloat16) if base.dtype == np.uint16 else t
    return t.permute(*np.argsort(order).tolist())


def host(t):
    return t.detach().float().cpu().numpy()


def on_gpu(c, s):
    t = {n: gpu(x) for n, x in s.items()}
    for m in ("k_pages", "v_pages"):
        t[m + "_all"] = t[m]
        t[m] = t[m].expand(-1, c["Hkv"], -1, -1)
    t["length"], t["count"] = gpu(c["lengths"]), gpu(c["counts"])
    t["params"] = B.step_params(q=t["q"], k=t["k"], v=t["v"], n_q_heads=c["Hq"], n_kv_heads=c["Hkv"], softmax_scale=c["scale"])
    t["pages"] = B.pages_for(t["k_pages"], t["v_pages"], t["table"])
    t["n_rows"] = c["n_rows"] or s["table"].shape[-1] * c["page"]
    need = B.ckv_paged_workspace_bytes(t["params"], t["n_rows"])
    t["ws"] = torch.full((need,), 0xFF, dtype=torch.uint8, device=DEV) if need else None   # NaN wherever it is read too early
    return t


def nines(c, heads):
    return torch.full((c["batch"], heads, c["n"], c["d"]), 9.0, dtype=torch.bfloat16 if c["dtype"] == "bf16" else torch.float32, device=DEV)


def attend(c, t, out=None, lse=None, stream=None):
    out = nines(c, c["Hq"]) if out is None else out
    lse = torch.full((c["batch"], c["Hq"], c["n"]), 9.0, device=DEV) if lse is None else lse
    B.ckv_paged_attention(t["params"], t["pages"], t["q"], t["k_pages"], t["v_pages"], t["table"], t["length"], t["n_rows"], out, lse,
                          t["ws"], count=t["count"], stream=stream)
    return out, lse


def check_attention(c, s, out, lse):
    want, tol, wl, lt = u.attention(c, s)
    old = np.arange(c["n"]) >= np.repeat(u.new_counts(c), c["Hq"] // c["Hkv"], 1)[..., None]
    u.check(host(out), np.where(old[..., None], 9.0, want), tol, "out")
    u.check(host(lse), np.where(old, 9.0, wl), lt, "lse")


@pytest.mark.parametrize("c", u.ROWS, ids=range(len(u.ROWS)))
def test_rows_are_transformed_and_find_their_pages(c):
    s = u.make(c)
    t, rot, n = on_gpu(c, s), u.rotation(c), u.new_counts(c)

    def dense(got, x, weight, what):
        heads = x.shape[1]
        want, tol = u.transform(c, s, x, weight)
        new = (np.arange(c["n"]) < np.repeat(n, heads // c["Hkv"], 1)[..., None])[..., None]
        u.check(host(got), np.where(new, want, 9.0), np.where(new, tol, 0.0), what)

    q_out, k_out = nines(c, c["Hq"]), nines(c, c["Hkv"])
    B.ckv_norm_rotate(t["params"], rot, t["q"], t["k"], t["positions"], t["inv_freq"], t["q_weight"], t["k_weight"], q_out, k_out,
                      count=t["count"])
    torch.cuda.synchronize()
    dense(q_out, s["q"], s["q_weight"], "q_out")
    dense(k_out, s["k"], s["k_weight"], "k_out")
    for with_q in (True, False):
        t = on_gpu(c, s)
        kp, kt, vp = u.appended(c, s)
        q_out = nines(c, c["Hq"])
        B.ckv_paged_append(t["params"], rot if c["norm"] or c["rot_dim"] else None, t["pages"], t["k"], t["v"], t["k_pages"], t["v_pages"],
                           t["table"], t["length"], count=t["count"], positions=t["positions"], inv_freq=t["inv_freq"],
                           k_weight=t["k_weight"], q=t["q"] if with_q else None, q_weight=t["q_weight"], q_out=q_out if with_q else None)
        torch.cuda.synchronize()
        u.check(host(t["k_pages_all"]), kp, kt, "k_pages")
        u.check(host(t["v_pages_all"]), vp, np.zeros_like(vp), "v_pages")
        if with_q:
            dense(q_out, s["q"], s["q_weight"], "q_out of the append")


LONG = [
    u.case(n=1, lengths=((9000, 8000), (1, 4097)), page=16),
    u.case(n=1, heads=(32, 8), lengths=((544, 300, 60, 33, 100, 544, 31, 32),) * 3, by_head=True, page=32),
    u.case(n=16, heads=(4, 4), lengths=((5000, 4000, 17, 16),), page=64, by_head=True),
    u.case(n=8, heads=(7, 1), lengths=((3001,), (8,)), page=16, pool_token_major=True),
    u.case(n=3, heads=(8, 1), d=64, lengths=((4100,), (100,)), page=8),
    u.case(n=257, heads=(4, 1), lengths=((700,),), page=32),
    u.case(n=300, heads=(2, 2), d=64, lengths=((300, 300), (555, 411)), counts=((300, 300), (1, 1)), page=256),
    u.case(n=520, heads=(1, 1), lengths=((1500,),), page=16),
    u.case(n=66, heads=(64, 64), d=64, lengths=(tuple(range(66, 130)),) * 4, page=16, by_head=True),    # tiles of eight waves
    u.case(n=17, heads=(32, 8), lengths=tuple((17 + 31 * b,) * 8 for b in range(32)), page=32),
    u.case(n=600, heads=(8, 8), d=64, lengths=((600,) * 8,) * 8, counts=((600,) * 8,) * 7 + ((5,) * 8,), page=64),
    u.case(dtype="f32", n=1, heads=(8, 2), lengths=((5000, 30),), page=16),
    u.case(dtype="f32", n=130, heads=(2, 1), d=64, lengths=((900,),), page=64),
    u.case(dtype="f32", n=20, heads=(6, 2), lengths=((2100, 40),), by_head=True, page=1),
]


@pytest.mark.parametrize("c", u.ATTEND + LONG, ids=range(len(u.ATTEND) + len(LONG)))
def test_attention_over_pages(c):
    s = u.make(c)
    t = on_gpu(c, s)
    out, lse = attend(c, t)
    torch.cuda.synchronize()
    check_attention(c, s, out, lse)
    again = attend(c, t)
    torch.cuda.synchronize()
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)   # the same bits
    # token by token, as the layer that follows takes it, and without lse
    wide = nines(c, c["Hq"]).transpose(1, 2).contiguous().transpose(1, 2)
    B.ckv_paged_attention(t["params"], t["pages"], t["q"], t["k_pages"], t["v_pages"], t["table"], t["length"], t["n_rows"], wide, None,
                          t["ws"], count=t["count"])
    torch.cuda.synchronize()
    assert torch.equal(wide, out)


@pytest.mark.parametrize("kind", ["bad_pages", "beyond", "masked_infinity", "masked_nan", "one_component"])
@pytest.mark.parametrize("c", [u.ATTEND[2], u.ATTEND[3], u.ATTEND[8], u.ATTEND[10]] + LONG[:6] + [LONG[8]], ids=range(11))
def test_what_is_not_seen_has_no_influence(c, kind):
    s = u.make(c)
    if kind == "bad_pages":
        table = s["table"].reshape(-1, s["table"].shape[-1])
        table[0, 0], table[-1, table.shape[1] // 2] = s["k_pages"].shape[0], -7
    else:
        seen = np.zeros(s["k_pages"].shape[:3], bool)
        new, n = np.zeros_like(seen), u.new_counts(c)
        for b, g in np.ndindex(n.shape):
            length = int(c["lengths"][b, g])
            for row in range(length):
                at = u.place(c, s, b, g, row)
                seen[at[0], 0 if c["by_head"] else g, at[1]] = True
                new[at[0], 0 if c["by_head"] else g, at[1]] |= row >= length - 2 and n[b, g] > 2  # not seen by the first new ones
        for m in ("k_pages", "v_pages"):
            x = u.values(np.ascontiguousarray(s[m])).copy()
            x[~seen] = np.nan
            if kind == "masked_infinity" and m == "v_pages":
                x[new] = np.inf
            elif kind == "masked_nan":
                x[new] = np.nan
            elif kind == "one_component" and m == "v_pages":
                x[new, 3], x[new, 5] = -np.inf, np.nan
            s[m] = u.stored(x, c["dtype"])
    t = on_gpu(c, s)
    out, lse = attend(c, t)
    torch.cuda.synchronize()
    check_attention(c, s, out, lse)


def test_queries_or_keys_alone_and_slices_of_one_projection():
    """q, k and v as slices of what one projection leaves (token by token, their heads side by side), queries alone, keys alone."""
    c = u.case(n=5, heads=(6, 2), lengths=((9, 9), (40, 40)), norm=True, rot_dim=32, page=8)
    s = u.make(c)
    d, n = c["d"], c["n"]
    fused = torch.zeros(2, n, 10 * d + 64, dtype=torch.bfloat16, device=DEV)
    part = {"q": fused[..., :6 * d].unflatten(-1, (6, d)), "k": fused[..., 6 * d:8 * d].unflatten(-1, (2, d)), "v": fused[..., 8 * d:10 * d].unflatten(-1, (2, d))}
    part = {m: x.transpose(1, 2) for m, x in part.items()}
    for m, x in part.items():
        x.copy_(gpu(s[m]))
    t, rot = on_gpu(c, s), u.rotation(c)
    for m in ("q", "k"):
        p = B.step_params(**{m: part[m]}, n_q_heads=6, n_kv_heads=2)
        out = nines(c, part[m].shape[1])
        q, k = (part[m], None) if m == "q" else (None, part[m])
        B.ckv_norm_rotate(p, rot, q, k, t["positions"], t["inv_freq"], t["q_weight"], t["k_weight"], out if q is not None else None,
                          out if k is not None else None)
        torch.cuda.synchronize()
        want, tol = u.transform(c, s, s[m], s[m + "_weight"])
        u.check(host(out), want, tol, m)
    p = B.step_params(**part, n_q_heads=6, n_kv_heads=2)
    B.ckv_paged_append(p, rot, t["pages"], part["k"], part["v"], t["k_pages"], t["v_pages"], t["table"], t["length"], positions=t["positions"],
                       inv_freq=t["inv_freq"], k_weight=t["k_weight"])
    torch.cuda.synchronize()
    kp, kt, vp = u.appended(c, s)
    u.check(host(t["k_pages_all"]), kp, kt, "k_pages")
    u.check(host(t["v_pages_all"]), vp, np.zeros_like(vp), "v_pages")
    out, lse = nines(c, 6), torch.full((2, 6, n), 9.0, device=DEV)
    B.ckv_paged_attention(p, t["pages"], part["q"], t["k_pages"], t["v_pages"], t["table"], t["length"], t["n_rows"], out, lse, t["ws"])
    torch.cuda.synchronize()
    check_attention(c, dict(s, **{m: u.stored(host(t[m + "_all"]), "bf16") for m in ("k_pages", "v_pages")}), out, lse)


def test_pages_that_two_lists_share():
    """Two sequences with a common beginning: the same pages in both lists, pages of their own behind."""
    c = u.case(n=3, heads=(4, 2), lengths=((70, 70), (90, 90)), page=16)
    s = u.make(c)
    s["table"][1, :4] = s["table"][0, :4]
    t = on_gpu(c, s)
    out, lse = attend(c, t)
    torch.cuda.synchronize()
    check_attention(c, s, out, lse)


@pytest.mark.parametrize("n,length", [(1, 300), (3, 3000), (40, 500)])
def test_a_page_several_times_in_a_list(n, length):
    c = u.case(n=n, heads=(4, 2), lengths=((length, length),), page=16)
    s = u.make(c)
    s["table"][0, 1::2] = s["table"][0, 0]
    t = on_gpu(c, s)
    out, lse = attend(c, t)
    torch.cuda.synchronize()
    check_attention(c, s, out, lse)


def test_a_bound_far_above_the_lengths():
    """A call that was planned for long lists (a graph, say) on short ones, down to none: shared out, merged and empty all the same."""
    for lengths in (((40, 40),), ((1, 1),), ((0, 0),), ((700, 2),)):
        c = u.case(n=2, heads=(8, 2), lengths=lengths, counts=(tuple(min(2, x) for x in lengths[0]),), page=16)
        s = u.make(c)
        s["table"] = np.concatenate([s["table"], np.full((1, 4000 - s["table"].shape[1]), -1, np.int32)], 1)
        t = on_gpu(c, s)
        assert t["n_rows"] == 64000 and t["ws"] is not None
        out, lse = attend(c, t)
        torch.cuda.synchronize()
        check_attention(c, s, out, lse)


def test_lists_far_apart_in_a_large_pool():
    """Rows beyond 2^32 bytes and beyond 2^31 elements of the pools; a list whose pages are the last ones."""
    d, page, n_pages = 128, 64, 270000                      # 4.4 GB a pool
    k_pages = torch.zeros(n_pages, 1, page, d, dtype=torch.bfloat16, device=DEV)
    v_pages = torch.zeros_like(k_pages)
    c = u.case(n=2, heads=(4, 1), d=d, lengths=((150,),), page=page, spare=0)
    s = u.make(c)
    ids = torch.tensor([[n_pages - 1, 0, n_pages - 2]], dtype=torch.int32, device=DEV)
    for i, p in enumerate(s["table"][0]):
        k_pages[ids[0, i]], v_pages[ids[0, i]] = gpu(s["k_pages"])[int(p)], gpu(s["v_pages"])[int(p)]
    t = on_gpu(c, s)
    t.update(k_pages=k_pages, v_pages=v_pages, table=ids, pages=B.pages_for(k_pages, v_pages, ids))
    out, lse = attend(c, t)
    torch.cuda.synchronize()
    check_attention(c, s, out, lse)
    B.ckv_paged_append(t["params"], None, t["pages"], t["k"], t["v"], k_pages, v_pages, ids, t["length"])
    torch.cuda.synchronize()
    assert torch.equal(k_pages[n_pages - 2, 0, 150 - 128 - 2:150 - 128], t["k"][0, 0])
    assert torch.equal(v_pages[n_pages - 2, 0, 150 - 128 - 2:150 - 128], t["v"][0, 0])


@pytest.mark.parametrize("c", [LONG[0], LONG[3], LONG[7]], ids=range(3))
def test_calls_on_several_streams_and_from_a_graph(c):
    """A step (append, attention) on streams of its own that overlap, and replayed from a graph with other inputs in the same places."""
    s = u.make(dict(c, norm=True, rot_dim=64))
    c = dict(c, norm=True, rot_dim=64)
    rot = u.rotation(c)
    other = u.make(dict(c, seed=5))

    def fresh():
        t = on_gpu(c, s)
        t["q_out"], t["out"], t["lse"] = nines(c, c["Hq"]), nines(c, c["Hq"]), torch.full((c["batch"], c["Hq"], c["n"]), 9.0, device=DEV)
        return t

    def step(t, stream=None):
        B.ckv_paged_append(t["params"], rot, t["pages"], t["k"], t["v"], t["k_pages"], t["v_pages"], t["table"], t["length"], count=t["count"],
                           positions=t["positions"], inv_freq=t["inv_freq"], k_weight=t["k_weight"], q=t["q"], q_weight=t["q_weight"],
                           q_out=t["q_out"], stream=stream)
        B.ckv_paged_attention(t["params2"], t["pages"], t["q_out"], t["k_pages"], t["v_pages"], t["table"], t["length"], t["n_rows"],
                              t["out"], t["lse"], t["ws"], count=t["count"], stream=stream)

    def load(t, which):
        for n in ("q", "k", "v"):
            t[n].copy_(gpu(which[n]))
        t["out"].fill_(9.0)

    def made():
        t = fresh()
        t["params2"] = B.step_params(q=t["q_out"], n_q_heads=c["Hq"], n_kv_heads=c["Hkv"], softmax_scale=c["scale"])
        return t

    want = []
    for which in (s, other):
        t = made()
        load(t, which)
        torch.cuda.synchronize()
        step(t)
        torch.cuda.synchronize()
        want.append([t[n].clone() for n in ("out", "lse", "q_out", "k_pages_all", "v_pages_all")])
    streams, ts = [torch.cuda.Stream() for _ in range(3)], [made() for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(3):
        for st, t in zip(streams, ts):
            step(t, st)
    torch.cuda.synchronize()
    for t in ts:
        for n, w in zip(("out", "lse", "q_out", "k_pages_all", "v_pages_all"), want[0]):
            assert torch.equal(t[n], w), n
    t = made()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(t)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(t)
    for rep in range(4):
        load(t, (s, other)[rep % 2])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for n, w in zip(("out", "lse", "q_out"), want[rep % 2]):
            assert torch.equal(t[n], w), (n, rep)
        (t["out"].float().sum() + t["lse"].sum()).item()


def test_a_graph_on_growing_lists():
    """A decoding step captured once, its lengths counted on between the replays: from an empty list over one chunk's rows to several."""
    Bz, Hq, Hkv, d, page, cap = 2, 8, 2, 128, 16, 8192
    g = torch.Generator(device=DEV).manual_seed(9)
    kp, vp = (torch.randn(Bz * cap // page, Hkv, page, d, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    ids = torch.randperm(Bz * cap // page, generator=g, device=DEV).to(torch.int32).view(Bz, -1)
    q = torch.randn(Bz, Hq, 1, d, generator=g, device=DEV).to(torch.bfloat16)
    p, pages = B.step_params(q=q, n_q_heads=Hq, n_kv_heads=Hkv), B.pages_for(kp, vp, ids)
    length, out, lse = torch.zeros(Bz, Hkv, dtype=torch.int32, device=DEV), torch.empty_like(q), torch.empty(Bz, Hq, 1, device=DEV)
    need = B.ckv_paged_workspace_bytes(p, cap)
    ws = [torch.full((need,), 0xFF, dtype=torch.uint8, device=DEV) for _ in range(2)]
    call = lambda o, l, w: B.ckv_paged_attention(p, pages, q, kp, vp, ids, length, cap, o, l, w)  # noqa: E731
    call(out, lse, ws[0])
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):   # two graphs that share a workspace, replayed in turn
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(out, lse, ws[0])
        graphs.append(graph)
    for i, n in enumerate((0, 1, 31, 33, 300, 1025, 2047, 5000, 8192, 64, 8191)):
        length.fill_(n)
        length[0, 1] = max(n - 7, 0)
        out.fill_(9.0)
        o, l = torch.empty_like(out), torch.empty_like(lse)
        torch.cuda.synchronize()
        graphs[i % 2].replay()
        call(o, l, ws[1])
        torch.cuda.synchronize()
        assert torch.equal(out, o) and torch.equal(lse, l), n
        for b, h in ((0, 0), (0, 7), (1, 4)):
            m = int(length[b, h // 4])
            rows = torch.arange(m, device=DEV)
            k, v = (t[ids[b, rows // page].long(), h // 4, rows % page].double() for t in (kp, vp))
            z = k @ q[b, h, 0].double() / d ** 0.5
            assert m == 0 and float(l[b, h, 0]) == -float("inf") or abs(float(l[b, h, 0]) - float(torch.logsumexp(z, 0))) < 2e-5
            w = torch.softmax(z, 0)
            ref, size = w @ v, w @ v.abs()
            assert ((o[b, h, 0].double() - ref).abs() <= 2.0 ** -8 * (size + ref.abs()) + 1e-4 * size).all()


def test_a_prompt_through_all_of_it():
    """Two prompts in chunks: rows into pages, attention of each chunk, and beside it dense keys for the retention step, which takes the last
    window's lse from the attention; the kept rows move into lists that differ by head, and tokens are decoded over them."""
    Bz, Hq, Hkv, d, T, W, budget, page = 2, 8, 2, 128, 900, 32, 200, 16
    g = torch.Generator(device=DEV).manual_seed(3)
    rnd = lambda *shape: torch.randn(*shape, generator=g, device=DEV).to(torch.bfloat16)  # noqa: E731
    x = {"q": rnd(Bz, T, Hq, d).transpose(1, 2), "k": rnd(Bz, T, Hkv, d).transpose(1, 2), "v": rnd(Bz, T, Hkv, d).transpose(1, 2)}
    qw, kw = (1 + 0.1 * rnd(d).float()).to(torch.bfloat16), (1 + 0.1 * rnd(d).float()).to(torch.bfloat16)
    freq = (1e4 ** (-torch.arange(d // 2, device=DEV) / (d // 2))).float()
    pos = torch.arange(T, device=DEV, dtype=torch.int32).expand(Bz, T).contiguous()
    rot = B.make_rotation(d, norm=True)
    # dense, at once
    q, k = torch.empty(Bz, Hq, T, d, dtype=torch.bfloat16, device=DEV), torch.empty(Bz, Hkv, T, d, dtype=torch.bfloat16, device=DEV)
    p_all = B.step_params(**x, n_q_heads=Hq, n_kv_heads=Hkv)
    B.ckv_norm_rotate(p_all, rot, x["q"], x["k"], pos, freq, qw, kw, q, k)
    v = x["v"].contiguous()
    # by chunks, over pages
    per = -(-T // page)
    ids = torch.randperm(Bz * per, generator=g, device=DEV).to(torch.int32).view(Bz, per)
    kp, vp = (torch.full((Bz * per, page, Hkv, d), float("nan"), dtype=torch.bfloat16, device=DEV).transpose(1, 2) for _ in range(2))
    pages = B.pages_for(kp, vp, ids)
    out, lse = torch.empty(Bz, Hq, T, d, dtype=torch.bfloat16, device=DEV), torch.empty(Bz, Hq, T, device=DEV)
    at = 0
    for n in (400, 1, 333, 166):
        part = {m: t[:, :, at:at + n] for m, t in x.items()}
        p = B.step_params(**part, n_q_heads=Hq, n_kv_heads=Hkv)
        length = torch.full((Bz, Hkv), at + n, dtype=torch.int32, device=DEV)
        qn, o, l = torch.empty(Bz, Hq, n, d, dtype=torch.bfloat16, device=DEV), torch.empty(Bz, Hq, n, d, dtype=torch.bfloat16, device=DEV), torch.empty(Bz, Hq, n, device=DEV)
        B.ckv_paged_append(p, rot, pages, part["k"], part["v"], kp, vp, ids, length, positions=pos[:, at:at + n].contiguous(), inv_freq=freq,
                           k_weight=kw, q=part["q"], q_weight=qw, q_out=qn)
        assert torch.equal(qn, q[:, :, at:at + n])
        pq = B.step_params(q=qn, n_q_heads=Hq, n_kv_heads=Hkv)
        need = B.ckv_paged_workspace_bytes(pq, at + n)
        B.ckv_paged_attention(pq, pages, qn, kp, vp, ids, length, at + n, o, l, torch.empty(need, dtype=torch.uint8, device=DEV) if need else None)
        out[:, :, at:at + n], lse[:, :, at:at + n] = o, l
        at += n
    z = torch.matmul(q.double(), k.double().repeat_interleave(Hq // Hkv, 1).transpose(-1, -2).contiguous()) / d ** 0.5
    z = z.masked_fill(torch.ones(T, T, dtype=torch.bool, device=DEV).triu(1), -float("inf"))
    ref = torch.softmax(z, -1) @ v.double().repeat_interleave(Hq // Hkv, 1)
    # weights rounded to bf16 and the output too: 2^-8 of sum w |v| and of the value
    size = torch.softmax(z, -1) @ v.double().abs().repeat_interleave(Hq // Hkv, 1)
    assert ((out.double() - ref).abs() <= 2.0 ** -8 * (size + ref.abs()) + 1e-4 * size).all()
    torch.testing.assert_close(lse.double(), torch.logsumexp(z, -1), rtol=0, atol=2e-5)
    # retention with the attention's lse and with its own
    P = T - W
    rp = B.params_for(q[:, :, P:], k, v, pool=B.POOL_AVG, pool_kernel=7, budget=budget, cap=T)
    tables = {"w_head": torch.ones(1, Hq, device=DEV), "head_share": torch.tensor([[0.3, 0.7]], device=DEV)}
    bufs = [B.LayerBuffers(rp, DEV) for _ in range(2)]
    for buf, given in zip(bufs, (lse[:, :, P:].contiguous(), None)):
        B.retention_layer(rp, q[:, :, P:], k, v, tables, buf, lse=given, fused_utility=True)
    torch.testing.assert_close(bufs[0].utility, bufs[1].utility, rtol=1e-4, atol=1e-6)
    buf = bufs[0]
    kept = buf.count
    assert kept[0, 0] != kept[0, 1]
    # the kept rows into pages of one head; tokens decoded over them
    steps, per = 5, -(-(int(kept.max()) + 5) // page)
    ids = torch.randperm(Bz * Hkv * per, generator=g, device=DEV).to(torch.int32).view(Bz, Hkv, per)
    kp, vp = (torch.full((Bz * Hkv * per, 1, page, d), float("nan"), dtype=torch.bfloat16, device=DEV).expand(-1, Hkv, -1, -1) for _ in range(2))
    pages = B.pages_for(kp, vp, ids)
    B.ckv_paged_append(B.step_params(k=buf.k_out, v=buf.v_out, n_q_heads=Hq, n_kv_heads=Hkv), None, pages, buf.k_out, buf.v_out, kp, vp, ids,
                       kept, count=kept)
    keys, vals = ([[t[b, h, :int(kept[b, h])] for h in range(Hkv)] for b in range(Bz)] for t in (buf.k_out, buf.v_out))
    length = kept.clone()
    for step in range(steps):
        one = {"q": rnd(Bz, Hq, 1, d), "k": rnd(Bz, Hkv, 1, d), "v": rnd(Bz, Hkv, 1, d)}
        p = B.step_params(**one, n_q_heads=Hq, n_kv_heads=Hkv)
        length += 1
        where = torch.full((Bz, 1), T + step, dtype=torch.int32, device=DEV)
        qn, o, l = torch.empty_like(one["q"]), torch.empty_like(one["q"]), torch.empty(Bz, Hq, 1, device=DEV)
        B.ckv_paged_append(p, rot, pages, one["k"], one["v"], kp, vp, ids, length, positions=where, inv_freq=freq, k_weight=kw, q=one["q"],
                           q_weight=qw, q_out=qn)
        kn, unused = torch.empty_like(one["k"]), torch.empty_like(one["q"])
        B.ckv_norm_rotate(p, rot, one["q"], one["k"], where, freq, qw, kw, unused, kn)
        n_rows = int(length.max())
        need = B.ckv_paged_workspace_bytes(p, n_rows)
        B.ckv_paged_attention(p, pages, qn, kp, vp, ids, length, n_rows, o, l, torch.empty(need, dtype=torch.uint8, device=DEV) if need else None)
        for b in range(Bz):
            for h in range(Hkv):
                keys[b][h], vals[b][h] = torch.cat([keys[b][h], kn[b, h]]), torch.cat([vals[b][h], one["v"][b, h]])
                for hq in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                    zz = keys[b][h].double() @ qn[b, hq, 0].double() / d ** 0.5
                    w = torch.softmax(zz, 0)
                    ref, size = w @ vals[b][h].double(), w @ vals[b][h].double().abs()
                    assert ((o[b, hq, 0].double() - ref).abs() <= 2.0 ** -8 * (size + ref.abs()) + 1e-4 * size).all()
                    assert abs(float(l[b, hq, 0]) - float(torch.logsumexp(zz, 0))) < 2e-5
    # the same lists through the compact-cache form, for the rows that came with the retention step
    need = max(B.ckv_decode_workspace_bytes(rp, 1, T), 256)
    o32, l32 = torch.empty(Bz, Hq, 1, d, device=DEV), torch.empty(Bz, Hq, 1, device=DEV)
    B.ckv_decode_attention(rp, qn, buf.k_out, buf.v_out, kept, o32, l32, torch.empty(need, dtype=torch.uint8, device=DEV))
    B.ckv_paged_attention(p, pages, qn, kp, vp, ids, kept, int(kept.max()), o, l, torch.empty(1 << 24, dtype=torch.uint8, device=DEV))
    torch.testing.assert_close(l, l32, rtol=0, atol=2e-5)
    assert ((o.float() - o32).abs() <= 2.0 ** -7 * (o32.abs() + 1.0)).all()
