"""The paged cache's calls as a server makes them: prompts in chunks, decode steps, eviction, freed pages given to a new
sequence, decode again; each call against the plain form on what the cache holds then.  A decode step in a graph; two
caches on two streams."""
import math

import pytest
import torch

import paged_plain as plain
from paper_2511_06029_amd import lethe as L

pytestmark = pytest.mark.gpu
DEV = "cuda"


class Server:
    """Layers of one model over a paged cache: pages are handed out and taken back on the host."""

    def __init__(self, layers, seqs, HQ, HK, D, page, pages, most, dtype="bf16", seed=0):
        self.c = L.LethePagedCache.allocate(layers, seqs, pages, page, most, HQ, HK, D, dtype)
        self.g = torch.Generator().manual_seed(seed)
        self.free = torch.randperm(pages, generator=self.g).tolist()
        self.n = [[0] * seqs for _ in range(layers)]
        self.table = torch.full((layers, seqs, most), -1, dtype=torch.int32)
        self.inv_freq = (10000.0 ** (-torch.arange(D // 2).double() / (D // 2))).float()
        self.sections = [D // 2 - 2 * (D // 8), D // 8, D // 8]

    def reserve(self, l, b, rows):
        have, need = -(-self.n[l][b] // self.c.page_size), -(-(self.n[l][b] + rows) // self.c.page_size)
        for i in range(have, need):
            self.table[l, b, i] = self.free.pop()
        self.n[l][b] += rows
        self.c.page_table.copy_(self.table)

    def release(self, l, b, rows):
        """Pages past the first ones that `rows` rows take."""
        for i in range(-(-rows // self.c.page_size), -(-self.n[l][b] // self.c.page_size)):
            self.free.append(int(self.table[l, b, i]))
            self.table[l, b, i] = -1
        self.n[l][b] = rows
        self.c.page_table.copy_(self.table)

    def rows(self, what, l, b):
        r = torch.arange(self.n[l][b])
        page, off = self.table[l, b].long()[r // self.c.page_size], r % self.c.page_size
        return getattr(self.c, what).cpu()[page, :, off].transpose(0, 1).contiguous()

    def tokens(self, lens):
        rows = sum(lens)
        c = self.c
        qkv = torch.randn((rows, c.HQ + 2 * c.HK, c.D), generator=self.g).to(c.tdtype)
        axis = torch.randint(0, 5000, (3, rows), generator=self.g).int()
        start = torch.tensor([sum(lens[:b]) for b in range(len(lens))], dtype=torch.int64)
        return qkv, axis, start, torch.tensor(lens, dtype=torch.int32)

    def forward(self, l, qkv, axis, start, lens, gamma):
        """Append and attend one layer, checked."""
        c = self.c
        most, kv = int(lens.max()), max(self.n[l]) + int(lens.max())
        before = [self.n[l][b] for b in range(c.B)]
        for b in range(c.B):
            self.reserve(l, b, int(lens[b]))
        seen = c.seen[l].tolist()
        dev = qkv.to(DEV)
        q = torch.zeros((len(qkv), c.HQ, c.D), dtype=c.tdtype, device=DEV)
        out = torch.zeros_like(q)
        s, n = start.to(DEV), lens.to(DEV)
        rot = L.Rotary(self.inv_freq.to(DEV), axis.to(DEV), self.sections)
        L.paged_append(c, l, dev[:, :c.HQ], dev[:, c.HQ:c.HQ + c.HK], dev[:, c.HQ + c.HK:], s, n, most, rot, q)
        held = [(self.rows("k", l, b), self.rows("v", l, b), self.rows("score", l, b)) for b in range(c.B)]
        L.paged_attn_score(c, l, q, s, n, most, kv, gamma, 0.0, 0.0, out, c.attn_workspace(len(qkv), most, kv))
        torch.cuda.synchronize()
        assert int(c.dev_status[0]) == 0
        assert c.len[l].tolist() == [before[b] + int(lens[b]) for b in range(c.B)]
        turned, size = plain.rotate(qkv[:, :c.HQ + c.HK], axis, self.inv_freq, self.sections, False)
        near = plain.rounding(turned, size, c.tdtype)
        for b, (K, V, score) in enumerate(held):
            ql, at = int(lens[b]), int(start[b])
            if ql == 0:
                continue
            new = turned[at:at + ql, c.HQ:].transpose(0, 1)
            assert torch.all((K[:, before[b]:].double() - new).abs() <= near[at:at + ql, c.HQ:].transpose(0, 1))
            assert self.rows("pos", l, b)[0, before[b]:].tolist() == list(range(seen[b], seen[b] + ql))
            qb = q[at:at + ql].cpu()
            ref, size, snew, stol, worst = plain.attend(qb, K, V, score, gamma, 1 / math.sqrt(c.D), 0.0)
            tol = plain.out_tolerance(ref, size, worst, c.tdtype, float(V.float().abs().sum(1).max()))
            assert torch.all((out[at:at + ql].cpu().double() - ref).abs() <= tol)
            assert torch.all((self.rows("score", l, b).double() - snew).abs() <= stol)

    def evict(self, budget, recent, sink):
        c = self.c
        was = {(l, b): {x: self.rows(x, l, b) for x in ("k", "v", "score", "pos")} for l in range(c.L) for b in range(c.B)}
        t = torch.tensor(budget, dtype=torch.int32).t().contiguous()  # [seqs][layers]
        L.paged_evict(c, t.to(DEV), recent, sink, c.evict_workspace(), max_kv_len=max(map(max, self.n)))
        torch.cuda.synchronize()
        assert int(c.dev_status[0]) == 0
        for (l, b), old in was.items():
            n = self.n[l][b]
            for h in range(c.HK):
                place, k = plain.evict(n, budget[l][b], recent, sink, old["score"][h], old["pos"][h])
                place = torch.tensor(place, dtype=torch.long)
                for x in old:
                    assert torch.equal(self.rows(x, l, b)[h], old[x][h][place]), (l, b, h, x)
            assert int(c.len[l, b]) == min(n, budget[l][b])
            self.release(l, b, min(n, budget[l][b]))


@pytest.mark.parametrize("HQ,HK,D,page,dtype", [(4, 2, 64, 16, "bf16"), (6, 1, 128, 32, "f16")])
def test_serving(HQ, HK, D, page, dtype):
    layers, seqs = 2, 3
    s = Server(layers, seqs, HQ, HK, D, page, 64, 24, dtype)
    # Prompts, one of them in two chunks; the third sequence is not there yet.
    for lens, gamma in (([70, 40, 0], 1.0), ([33, 1, 0], 1.0)):
        batch = s.tokens(lens)
        for l in range(layers):
            s.forward(l, *batch, gamma)
    for step in range(3):
        batch = s.tokens([1, 1, 0])
        for l in range(layers):
            s.forward(l, *batch, 0.9)
    s.evict([[50, 44, 0], [30, 20, 0]], 16, 2)
    # The freed pages hold a new sequence's prompt while the others decode.
    for lens in ([1, 1, 150], [1, 0, 1], [1, 1, 1]):
        batch = s.tokens(lens)
        for l in range(layers):
            s.forward(l, *batch, 0.9)
    s.evict([[50, 45, 60], [25, 22, 90]], 8, 0)
    for step in range(2):
        batch = s.tokens([1, 1, 1])
        for l in range(layers):
            s.forward(l, *batch, 0.9)
    # Everything goes, and the sequences start again.
    s.evict([[0, 0, 0], [0, 0, 0]], 8, 8)
    assert len(s.free) == 64
    s.forward(0, *s.tokens([5, 1, 17]), 1.0)


def step_buffers(c, rows, seed):
    g = torch.Generator().manual_seed(seed)
    t = {"qkv": torch.randn((rows, c.HQ + 2 * c.HK, c.D), generator=g).to(c.tdtype).to(DEV),
         "axis": torch.zeros((1, rows), dtype=torch.int32, device=DEV),
         "q": torch.zeros((rows, c.HQ, c.D), dtype=c.tdtype, device=DEV),
         "start": torch.arange(rows, dtype=torch.int64, device=DEV),
         "lens": torch.ones(rows, dtype=torch.int32, device=DEV)}
    t["out"] = torch.zeros_like(t["q"])
    t["rot"] = L.Rotary((10.0 ** -torch.arange(c.D // 2).float()).to(DEV), t["axis"], [c.D // 2])
    t["ws"] = c.attn_workspace(rows, 1, c.max_pages * c.page_size)
    return t


def decode(c, t, stream=None):
    for l in range(c.L):
        x = t["qkv"]
        L.paged_append(c, l, x[:, :c.HQ], x[:, c.HQ:c.HQ + c.HK], x[:, c.HQ + c.HK:], t["start"], t["lens"], 1, t["rot"],
                       t["q"], stream=stream)
        L.paged_attn_score(c, l, t["q"], t["start"], t["lens"], 1, c.max_pages * c.page_size, 0.9, 0.0, 0.0, t["out"],
                           t["ws"], stream=stream)


def filled_cache(seed, seqs=3):
    pool = plain.Pool(2, seqs, [[100] * seqs] * 2, 8, 2, 128, "bf16", 16, seed)
    g = torch.Generator().manual_seed(seed)
    for l in range(2):
        for b in range(seqs):
            K = torch.randn((2, 20 + 9 * b, 128), generator=g)
            pool.put(l, b, K, -K, torch.rand((2, 20 + 9 * b), generator=g), torch.arange(20 + 9 * b).expand(2, -1))
    return pool.cache


def test_decode_steps_in_a_graph_with_eviction_between():
    """A captured step of two layers appends and attends anew at every replay; eager calls and eviction in between."""
    a, b = filled_cache(3), filled_cache(3)
    ta, tb = step_buffers(a, 3, 5), step_buffers(b, 3, 5)
    keep = {x: getattr(a, x).clone() for x in ("k", "v", "score", "pos", "len", "seen")}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        decode(a, ta)
    for x in keep:
        getattr(a, x).copy_(keep[x])
    wa = a.evict_workspace()
    for i in range(6):
        ta["axis"].fill_(50 + i)
        tb["axis"].fill_(50 + i)
        ta["qkv"].mul_(-1)
        tb["qkv"].mul_(-1)
        graph.replay()
        decode(b, tb)
        torch.cuda.synchronize()
        assert torch.equal(ta["out"], tb["out"]) and torch.equal(ta["q"], tb["q"])
        if i % 2:
            budget = torch.full((3, 2), 24, dtype=torch.int32, device=DEV)
            L.paged_evict(a, budget, 4, 1, wa)
            L.paged_evict(b, budget, 4, 1, b.evict_workspace())
        for x in keep:
            assert torch.equal(getattr(a, x), getattr(b, x)), (i, x)
    assert int(a.dev_status[0]) == 0 and a.seen.tolist() == [[26, 35, 44]] * 2


@pytest.mark.parametrize("q_lens", [[1, 1], [20, 3]])
def test_a_pool_past_four_gib(q_lens):
    """Pages whose rows lie past 2^32 bytes: the same bits as the same pages at the front of a small pool."""
    HQ, HK, D, page, lens = 8, 2, 128, 64, [700, 90]
    pool = plain.Pool(1, 2, [[n + q for n, q in zip(lens, q_lens)]], HQ, HK, D, "bf16", page, 21)
    g = torch.Generator().manual_seed(21)
    for b, n in enumerate(lens):
        pool.put(0, b, torch.randn((HK, n, D), generator=g), torch.randn((HK, n, D), generator=g),
                 torch.rand((HK, n), generator=g), torch.arange(n).expand(HK, n))
    small = pool.cache
    first = 2 ** 32 // (2 * HK * page * D) + 7
    big = L.LethePagedCache.allocate(1, 2, first + small.num_pages, page, small.max_pages, HQ, HK, D)
    for x in ("k", "v", "score", "pos"):
        getattr(big, x)[first:].copy_(getattr(small, x))
    big.len.copy_(small.len)
    big.seen.copy_(small.seen)
    big.page_table.copy_(torch.where(small.page_table >= 0, small.page_table + first, small.page_table))
    rows, most, kv = sum(q_lens), max(q_lens), 800
    qkv = torch.randn((rows, HQ + 2 * HK, D), generator=g).bfloat16().to(DEV)
    start = torch.tensor([0, q_lens[0]], device=DEV)
    ql = torch.tensor(q_lens, dtype=torch.int32, device=DEV)
    budget = torch.tensor([[300], [60]], dtype=torch.int32, device=DEV)
    outs = []
    for c in (small, big):
        out = torch.zeros((rows, HQ, D), dtype=c.tdtype, device=DEV)
        L.paged_append(c, 0, None, qkv[:, HQ:HQ + HK], qkv[:, HQ + HK:], start, ql, most, None, None)
        L.paged_attn_score(c, 0, qkv[:, :HQ].contiguous(), start, ql, most, kv, 0.9, 0.0, 0.0, out,
                           c.attn_workspace(rows, most, kv))
        L.paged_evict(c, budget, 16, 2, c.evict_workspace())
        outs.append(out)
    torch.cuda.synchronize()
    assert int(small.dev_status[0]) == 0 and int(big.dev_status[0]) == 0
    assert torch.equal(*outs) and big.len.tolist() == [[300, 60]]
    for x in ("k", "v", "score", "pos"):
        assert torch.equal(getattr(big, x)[first:], getattr(small, x)), x
        assert not torch.any(getattr(big, x)[:8]), x


def test_two_caches_on_two_streams():
    caches = [filled_cache(7), filled_cache(8)]
    alone = [filled_cache(7), filled_cache(8)]
    buffers = [step_buffers(c, 3, 9 + i) for i, c in enumerate(caches)]
    streams = [torch.cuda.Stream() for _ in caches]
    torch.cuda.synchronize()
    for _ in range(5):
        for c, t, s in zip(caches, buffers, streams):
            decode(c, t, stream=s)
    torch.cuda.synchronize()
    for i, c in enumerate(alone):
        t = step_buffers(c, 3, 9 + i)
        for _ in range(5):
            decode(c, t)
        torch.cuda.synchronize()
        assert torch.equal(t["out"], buffers[i]["out"])
        for x in ("k", "v", "score", "pos", "len", "seen"):
            assert torch.equal(getattr(c, x), getattr(caches[i], x)), x
