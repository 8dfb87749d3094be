"""Pages, trees and lists as a serving program uses them together: prompts retained in place, answers forked from them, trees of drafted tokens verified and
their accepted paths kept, step after step, eager, replayed from a graph and on several streams."""
import numpy as np
import pytest
import torch

import pages_util as v
from paper_2602_08686_amd import binding as B
from test_gpu_pages import ints

pytestmark = pytest.mark.gpu
DEV = "cuda"


def i32(*shape):
    return torch.zeros(*shape, dtype=torch.int32, device=DEV)


class Server:
    """Slots for sequences over one pair of pools; lists for every KV head (pages of one head) or for a sequence (pages of all heads)."""

    def __init__(self, slots, Hq, Hkv, d, page, most, n_pages, n, by_head, seed=0):
        self.slots, self.Hq, self.Hkv, self.d, self.page, self.n, self.by_head = slots, Hq, Hkv, d, page, n, by_head
        self.g = torch.Generator(device=DEV).manual_seed(seed)
        heads = 1 if by_head else Hkv
        self.k, self.v = (torch.full((n_pages, heads, page, d), float("nan"), dtype=torch.bfloat16, device=DEV).expand(-1, Hkv, -1, -1) for _ in range(2))
        shape = (slots, Hkv, most) if by_head else (slots, most)
        self.table, self.other = (torch.full(shape, -1, dtype=torch.int32, device=DEV) for _ in range(2))
        self.refs, self.taken = B.page_counts(n_pages)
        self.lists = B.lists_for(self.table, n_kv_heads=Hkv, n_pages=n_pages, page_rows=page)
        self.pages = B.pages_for(self.k, self.v, self.table)
        self.length, self.next = i32(slots, Hkv), i32(slots, Hkv)
        self.copy, self.result = i32(4 * slots * Hkv, 2), i32(2)
        self.pool = B.pool_params(self.k, self.table)
        self.freq = (1e4 ** (-torch.arange(d // 2, device=DEV) / (d // 2))).float()
        self.rot = B.make_rotation(d)
        rnd = lambda heads: torch.zeros(slots, heads, n, d, dtype=torch.bfloat16, device=DEV)  # noqa: E731
        self.q, self.kn, self.vn, self.qr = rnd(Hq), rnd(Hkv), rnd(Hkv), rnd(Hq)
        self.params = B.step_params(q=self.q, k=self.kn, v=self.vn, n_q_heads=Hq, n_kv_heads=Hkv)
        self.out, self.lse = rnd(Hq), torch.zeros(slots, Hq, n, device=DEV)
        self.parent, self.sees, self.pos = i32(slots, n), torch.zeros(slots, n, -(-n // 64), dtype=torch.int64, device=DEV), i32(slots, n)
        self.start, self.count, self.path, self.kept = i32(slots), i32(slots, Hkv), i32(slots, n), i32(slots, Hkv)
        self.n_rows = most * page
        need = B.ckv_paged_workspace_bytes(self.params, self.n_rows)
        self.ws = torch.full((need,), 0xFF, dtype=torch.uint8, device=DEV) if need else None

    def room(self, first, end):
        """Pages of their own for rows first .. end - 1, the shared ones' contents with them."""
        B.ckv_pages_reserve(self.lists, self.table, first, end, self.refs, self.taken, self.copy, self.result)
        B.ckv_pages_copy(self.pool, self.pages, self.k, self.v, self.copy)

    def verify(self):
        """A tree of drafted tokens in the rows' own pages, and what they see."""
        self.next.copy_(self.length + self.count)
        self.room(self.length, self.next)
        B.ckv_tree_sees(self.parent, self.start, self.sees, self.pos)
        B.ckv_paged_append(self.params, self.rot, self.pages, self.kn, self.vn, self.k, self.v, self.table, self.next, count=self.count, positions=self.pos,
                           inv_freq=self.freq, q=self.q, q_out=self.qr)
        B.ckv_paged_tree_attention(self.params, self.pages, self.qr, self.k, self.v, self.table, self.next, self.n_rows, self.sees, self.out, self.lse,
                                   self.ws, count=self.count)

    def accept(self):
        """The accepted paths stay, what they leave of the pages goes back."""
        B.ckv_paged_compact(self.pool, self.pages, self.k, self.v, self.table, self.next, self.path, self.kept, self.length, count=self.count)
        B.ckv_pages_free(self.lists, self.table, self.length, self.refs, self.taken)
        self.start.add_(self.kept[:, 0])

    def rows(self, b, h, upto):
        r = torch.arange(upto, device=DEV)
        list_ = (self.table[b, h] if self.by_head else self.table[b])[r // self.page].long()
        assert (list_ >= 0).all()
        return (t[list_, h, r % self.page] for t in (self.k, self.v))

    def agree(self, tables=None):
        """Counts and bits are what the tables say."""
        want = v.Lists([t.cpu().numpy() for t in (tables or [self.table])], self.refs.numel(), self.page)
        assert np.array_equal(self.refs.cpu(), want.refs) and np.array_equal(self.taken.cpu(), want.taken())


def drafts(s, rng, kind="random"):
    """New tokens, their trees, counts, and the paths that will be accepted, as if the model had spoken."""
    for t in (s.q, s.kn, s.vn):
        t.copy_(torch.randn(t.shape, generator=s.g, device=DEV))
    parent = v.parents(kind, s.slots, s.n, seed=int(rng.integers(1000)))
    counts = rng.integers(1, s.n + 1, s.slots)
    path, kept = np.full((s.slots, s.n), -1, np.int32), np.zeros(s.slots, np.int32)
    for b in range(s.slots):
        i, way = int(rng.integers(0, counts[b])), []
        while i >= 0:
            way.append(i)
            i = int(parent[b, i])
        kept[b] = len(way)
        path[b, :kept[b]] = way[::-1]
    s.parent.copy_(ints(parent))
    s.count.copy_(ints(counts.astype(np.int32))[:, None].expand(-1, s.Hkv))
    s.path.copy_(ints(path))
    s.kept.copy_(ints(kept)[:, None].expand(-1, s.Hkv))
    return parent, counts, path, kept


@pytest.mark.parametrize("by_head,n,heads,d", [(True, 12, (8, 2), 128), (False, 30, (14, 2), 64), (False, 70, (8, 2), 128)])
def test_answers_from_retained_prompts(by_head, n, heads, d):
    Hq, Hkv = heads
    G, page, T, W = Hq // Hkv, 16, 700, 32
    slots, rng = 5, np.random.default_rng(n)
    s = Server(slots, Hq, Hkv, d, page, most=64, n_pages=slots * Hkv * 64 if by_head else slots * 64, n=n, by_head=by_head)
    # a prompt in slot 0 and one in slot 1, a third slot empty, ...
    x = {m: torch.randn(slots, heads_, T, d, generator=s.g, device=DEV).bfloat16() for m, heads_ in (("q", Hq), ("k", Hkv), ("v", Hkv))}
    there = torch.zeros(slots, Hkv, dtype=torch.int32, device=DEV)
    there[0], there[1] = T, T - 133
    p = B.step_params(k=x["k"], v=x["v"], n_q_heads=Hq, n_kv_heads=Hkv)
    s.room(i32(slots, Hkv), there)
    B.ckv_paged_append(p, None, s.pages, x["k"], x["v"], s.k, s.v, s.table, there, count=there)
    s.agree()
    assert s.result.tolist() == [0, 0]
    # the retention step over the dense rows says which stay; they move inside the pages, and beside them
    rp = B.params_for(x["q"][:, :, T - W:], x["k"], x["v"], pool=B.POOL_AVG, pool_kernel=7, budget=200, cap=T)
    buf = B.LayerBuffers(rp, DEV)
    tables = {"w_head": torch.ones(1, Hq, device=DEV), "head_share": torch.tensor([[0.3, 0.7]], device=DEV) if by_head else None}
    B.retention_layer(rp, x["q"][:, :, T - W:], x["k"], x["v"], tables, buf, fused_utility=True)
    kept = buf.count.clone()
    kept[1:] = 0           # (the second prompt is shorter than what the retention step saw: it keeps nothing here)
    B.ckv_paged_compact(s.pool, s.pages, s.k, s.v, s.table, there, buf.idx, kept, s.length)
    B.ckv_pages_free(s.lists, s.table, s.length, s.refs, s.taken)
    s.agree()
    logical = {}
    for h in range(Hkv):
        m = int(kept[0, h])
        keys, vals = s.rows(0, h, m)
        assert torch.equal(keys, buf.k_out[0, h, :m]) and torch.equal(vals, buf.v_out[0, h, :m]), h
        logical[h] = (keys.clone(), vals.clone())
    held = int((s.refs > 0).sum())
    # every slot becomes an answer to the first prompt: no page more than before
    B.ckv_pages_fork(s.lists, s.table, i32(slots), s.other, s.refs, s.taken, s.length, s.next)
    s.agree([s.table, s.other])
    B.ckv_pages_free(s.lists, s.table, None, s.refs, s.taken)
    s.table, s.other = s.other, s.table
    s.pages, s.lists = B.pages_for(s.k, s.v, s.table), B.lists_for(s.table, n_kv_heads=Hkv, n_pages=s.refs.numel(), page_rows=page)
    s.length.copy_(s.next)
    s.agree()
    assert int((s.refs > 0).sum()) == held and (s.length == kept[0]).all()
    s.start.fill_(T)
    cache = [[logical[h] for h in range(Hkv)] for _ in range(slots)]
    for step in range(4):
        parent, counts, path, accepted = drafts(s, rng)
        sees, depth = v.paths(parent)
        s.verify()
        s.agree()
        missing, copies = s.result.tolist()
        partial = (kept[0] % page != 0).sum().item() if by_head else int(int(kept[0].max()) % page != 0 or bool((kept[0] < kept[0].max()).any()))
        if step == 0 and partial:
            assert copies > 0   # what the answers share and write into has been copied, but for the last one
        assert missing == 0
        # keys as they are in the cache: turned by the positions start + depth
        turned, unused = torch.empty_like(s.kn), torch.empty_like(s.qr)
        B.ckv_norm_rotate(s.params, s.rot, s.q, s.kn, s.pos, s.freq, None, None, unused, turned)
        assert torch.equal(s.pos.cpu(), s.start.cpu()[:, None] + torch.from_numpy(depth).int())
        for b in range(slots):
            m = int(counts[b])
            seen = torch.from_numpy(sees[b, :m, :m]).to(DEV)
            for h in range(Hkv):
                keys, vals = (torch.cat([old, new[b, h, :m]]) for old, new in zip(cache[b][h], (turned, s.vn)))
                got = s.rows(b, h, int(s.next[b, h]))
                assert all(torch.equal(a, c) for a, c in zip(got, (keys, vals))), (step, b, h)
                mask = torch.cat([torch.ones(m, len(cache[b][h][0]), dtype=torch.bool, device=DEV), seen], 1)
                for hq in range(h * G, (h + 1) * G):
                    z = (s.qr[b, hq, :m].double() @ keys.double().t() / d ** 0.5).masked_fill(~mask, -float("inf"))
                    w = torch.softmax(z, 1)
                    want, size = w @ vals.double(), w @ vals.double().abs()
                    # weights rounded to bf16 and the output too: 2^-8 of sum w |v| and of the value; logits and sums in fp32
                    assert ((s.out[b, hq, :m].double() - want).abs() <= 2.0 ** -8 * (size + want.abs()) + 1e-4 * size).all()
                    assert (s.lse[b, hq, :m].double() - torch.logsumexp(z, 1)).abs().max() < 2e-5
                way = torch.from_numpy(path[b, :accepted[b]]).long().to(DEV)
                cache[b][h] = tuple(torch.cat([old, new[b, h][way]]) for old, new in zip(cache[b][h], (turned, s.vn)))
        s.accept()
        s.agree()
        for b in range(slots):
            for h in range(Hkv):
                upto = len(cache[b][h][0])
                assert int(s.length[b, h]) == upto
                assert all(torch.equal(a, c) for a, c in zip(s.rows(b, h, upto), cache[b][h])), (step, b, h)
        if step == 1:   # two answers go on from the third, one ends
            who = [2, 1, 2, -1, 4]
            B.ckv_pages_fork(s.lists, s.table, ints(np.array(who, np.int32)), s.other, s.refs, s.taken, s.length, s.next)
            B.ckv_pages_free(s.lists, s.table, None, s.refs, s.taken)
            s.table, s.other = s.other, s.table
            s.pages = B.pages_for(s.k, s.v, s.table)
            s.length.copy_(s.next)
            start = s.start.tolist()
            s.start.copy_(ints(np.array([start[w] if w >= 0 else 0 for w in who], np.int32)))
            none = tuple(torch.zeros(0, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
            cache = [[cache[w][h] if w >= 0 else none for h in range(Hkv)] for w in who]
            s.agree()
    B.ckv_pages_free(s.lists, s.table, None, s.refs, s.taken)
    assert not s.refs.any() and not s.taken.any()


def _state(s):
    return [t.clone() for t in (s.k[:, :1] if s.by_head else s.k, s.v[:, :1] if s.by_head else s.v, s.table, s.refs, s.taken, s.length, s.start, s.out, s.lse, s.sees,
                                s.pos, s.copy, s.result)]


def _same(a, b, what):
    for i, (x, y) in enumerate(zip(a, b)):
        assert torch.equal(x.view(torch.int16) if x.dtype == torch.bfloat16 else x, y.view(torch.int16) if y.dtype == torch.bfloat16 else y), (what, i)


def _begin(s, rows):
    """Sequences of some rows, two of them sharing their pages."""
    for t in (s.k, s.v):
        t = t[:, :1] if s.by_head else t
        t.copy_(torch.randn(t.shape, generator=s.g, device=DEV))
    end = ints(np.broadcast_to(np.asarray(rows, np.int32)[:, None], (s.slots, s.Hkv)).copy())
    B.ckv_pages_reserve(s.lists, s.other, i32(s.slots, s.Hkv), end, s.refs, s.taken, s.copy, s.result)
    parent = np.arange(s.slots, dtype=np.int32)
    parent[-1] = 0
    B.ckv_pages_fork(s.lists, s.other, ints(parent), s.table, s.refs, s.taken, end, s.length)
    B.ckv_pages_free(s.lists, s.other, None, s.refs, s.taken)
    s.start.copy_(s.length[:, 0])


@pytest.mark.parametrize("by_head,n,heads,d", [(True, 12, (8, 2), 128), (False, 33, (14, 2), 64), (False, 80, (8, 2), 128)])
def test_steps_replayed_from_a_graph(by_head, n, heads, d):
    """One graph of a whole step, replayed with other tokens, trees and lists that grow, against eager steps of a server of its own."""
    servers = [Server(4, *heads, d, 16, most=80, n_pages=4 * heads[1] * 100, n=n, by_head=by_head) for _ in range(2)]
    eager, replayed = servers
    for s in servers:
        _begin(s, [700, 30, 5, 0])

    def step(s):
        s.verify()
        s.accept()

    trial = Server(4, *heads, d, 16, most=80, n_pages=4 * heads[1] * 100, n=n, by_head=by_head)   # a step before the capture
    _begin(trial, [700, 30, 5, 0])
    drafts(trial, np.random.default_rng(0))
    step(trial)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(replayed)
    rngs = [np.random.default_rng(5) for _ in servers]
    for rep in range(6):
        for s, rng in zip(servers, rngs):
            drafts(s, rng, kind=("random", "chain", "star")[rep % 3])
        torch.cuda.synchronize()
        step(eager)
        graph.replay()
        torch.cuda.synchronize()
        _same(_state(replayed), _state(eager), rep)
        replayed.agree()
        (replayed.out.float().sum() + replayed.refs.sum()).item()   # eager library work between the replays


def test_servers_on_streams_of_their_own():
    make = lambda i: Server(4, 8, 2, 128, 16, most=80, n_pages=900, n=(16, 60, 90)[i], by_head=i == 0, seed=i)  # noqa: E731
    want = []
    for i in range(3):
        s = make(i)
        _begin(s, [900, 30, 300, 0])
        drafts(s, np.random.default_rng(i))
        torch.cuda.synchronize()
        for _ in range(3):
            s.verify()
            s.accept()
        torch.cuda.synchronize()
        want.append(_state(s))
    servers, streams = [make(i) for i in range(3)], [torch.cuda.Stream() for _ in range(3)]
    for i, s in enumerate(servers):
        _begin(s, [900, 30, 300, 0])
        drafts(s, np.random.default_rng(i))
    torch.cuda.synchronize()
    for _ in range(3):
        for s, stream in zip(servers, streams):
            with torch.cuda.stream(stream):
                s.verify()
                s.accept()
    torch.cuda.synchronize()
    for i, s in enumerate(servers):
        _same(_state(s), want[i], i)


def test_too_few_pages_change_nothing():
    s = Server(3, 4, 2, 64, 16, most=40, n_pages=60, n=8, by_head=False)
    _begin(s, [400, 300, 0])                        # 25 + 19 pages, the third shares the first's
    before = [t.clone() for t in (s.table, s.refs, s.taken)]
    B.ckv_pages_reserve(s.lists, s.table, s.length, s.length + 200, s.refs, s.taken, s.copy, s.result)
    torch.cuda.synchronize()
    assert s.result[0].item() > 0 and s.result[1].item() == 0 and (s.copy == -1).all()
    for a, b in zip(before, (s.table, s.refs, s.taken)):
        assert torch.equal(a, b)
    need = s.result[0].item()
    B.ckv_pages_free(s.lists, s.table, ints(np.array([[400] * 2, [0] * 2, [0] * 2], np.int32)), s.refs, s.taken)   # two answers give way
    free = int((s.refs == 0).sum())
    end = s.length.clone()
    end[0] += 200
    B.ckv_pages_reserve(s.lists, s.table, s.length, torch.where(torch.arange(3, device=DEV)[:, None] == 0, end, 0).int(), s.refs, s.taken, s.copy, s.result)
    s.agree()
    assert s.result.tolist() == [0, 0] and need > 0 and free >= 13
