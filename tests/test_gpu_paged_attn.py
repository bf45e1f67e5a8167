"""lethe_paged_attn_score against the plain form in 64 bits: one query and many, mixed batches, every group size, caps,
scores, pages of every kind, infinities and NaN where no query looks, pages out of range, streams and graphs."""
import math

import pytest
import torch

import paged_plain as plain
from paper_2511_06029_amd import lethe as L

pytestmark = pytest.mark.gpu
DEV = "cuda"


def filled(lens, HQ, HK, D, dtype, page, seed, layers=1, layer=0, fill=float("nan")):
    """A pool whose layer `layer` holds rows of random contents; what no row owns is `fill`."""
    g = torch.Generator().manual_seed(seed)
    pool = plain.Pool(layers, len(lens), [lens] * layers, HQ, HK, D, dtype, page, seed, fill=fill)
    T = pool.dtype
    rows = []
    for b, n in enumerate(lens):
        K = (torch.randn((HK, n, D), generator=g) * (0.5 + 2 * torch.rand((HK, n, 1), generator=g))).to(T)
        V = torch.randn((HK, n, D), generator=g).to(T)
        s = torch.rand((HK, n), generator=g)
        pool.put(layer, b, K, V, s, torch.arange(n).expand(HK, n))
        rows.append((K, V, s))
    return pool, rows, g


def batch(q_lens, gap=0):
    starts, at = [], gap
    for q in q_lens:
        starts.append(at)
        at += q + gap
    return torch.tensor(starts, dtype=torch.int64, device=DEV), torch.tensor(q_lens, dtype=torch.int32, device=DEV), at


def check(pool, rows, q, q_start, q_lens, out, gamma, scale, cap, layer=0):
    for b, (K, V, s) in enumerate(rows):
        n, ql, at = K.shape[1], q_lens[b], int(q_start[b])
        got = pool.get("score", layer, b, n)
        if ql == 0:
            assert torch.equal(got, s), "scores of sequence %d without queries" % b
            continue
        ref, size, new, stol, worst = plain.attend(q[at:at + ql].cpu(), K, V, s, gamma, scale, cap)
        tol = plain.out_tolerance(ref, size, worst, pool.dtype, float(V.float().abs().nan_to_num(posinf=0.0).sum(1).max()))
        o = out[at:at + ql].cpu().double()
        assert torch.equal(torch.isfinite(o), torch.isfinite(ref)), "sequence %d: infinities" % b
        fine = torch.isfinite(ref)
        err = (o - ref).abs()[fine] - tol[fine]
        assert fine.sum() == 0 or err.max() <= 0, "sequence %d: out off by %.3g over its bound" % (b, err.max())
        if gamma:
            assert torch.all((got.double() - new).abs() <= stol), "sequence %d: scores" % b
        else:
            assert torch.equal(got, s)


def run(lens, q_lens, HQ, HK, D, dtype="bf16", page=16, gamma=0.9, cap=0.0, scale=0.0, gap=0, seed=0, loose=False,
        layers=1, layer=0):
    pool, rows, g = filled(lens, HQ, HK, D, dtype, page, seed, layers, layer)
    q_start, q_len, total = batch(q_lens, gap)
    q = torch.randn((total, HQ, D), generator=g).to(pool.dtype).to(DEV)
    out = torch.full_like(q, 77.0)
    most = (2 ** 31 - 1, 2 ** 31 - 1) if loose else (max(q_lens), max(lens))
    ws = pool.cache.attn_workspace(total, *most)
    L.paged_attn_score(pool.cache, layer, q, q_start, q_len, *most, gamma, scale, cap, out, ws)
    torch.cuda.synchronize()
    assert int(pool.cache.dev_status[0]) == 0
    check(pool, rows, q, q_start, q_lens, out, gamma, scale or 1 / math.sqrt(D), cap, layer)
    mine = torch.zeros(total, dtype=torch.bool)
    for b, ql in enumerate(q_lens):
        mine[int(q_start[b]):int(q_start[b]) + ql] = True
    assert torch.all(out.cpu()[~mine] == 77.0)
    return pool, out


EDGES = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 128, 129, 700]


@pytest.mark.parametrize("HQ,HK,D,dtype,page", [
    (1, 1, 64, "bf16", 16), (4, 2, 128, "f16", 16), (9, 3, 64, "f16", 32), (32, 8, 128, "bf16", 64),
    (5, 1, 128, "bf16", 128), (12, 2, 64, "bf16", 16), (28, 4, 128, "f16", 256), (8, 1, 64, "bf16", 1024)])
@pytest.mark.parametrize("gamma,cap", [(0.0, 0.0), (0.9, 0.0), (1.0, 5.0)])
def test_one_query(HQ, HK, D, dtype, page, gamma, cap):
    run(EDGES, [1] * len(EDGES), HQ, HK, D, dtype, page, gamma, cap, gap=1)


def test_one_query_with_sequences_that_have_none():
    run([40, 0, 70, 5, 0, 300], [1, 0, 0, 1, 0, 1], 4, 2, 64, gamma=0.5)
    run([40, 0, 70], [0, 0, 0], 4, 2, 64, gamma=0.5)


@pytest.mark.parametrize("B", [65, 300])
def test_one_query_of_many_sequences(B):
    run([1 + (37 * b) % 211 for b in range(B)], [1 if b % 5 else 0 for b in range(B)], 4, 2, 64, page=16, gamma=0.99)


def test_one_query_over_long_rows():
    run([40000, 3, 9001], [1, 1, 1], 8, 1, 128, "bf16", 16, 0.99, seed=3)
    run([70001], [1], 4, 4, 64, "f16", 64, 1.0, seed=4)


@pytest.mark.parametrize("HQ,HK,D,dtype,page", [
    (2, 2, 64, "bf16", 16), (8, 4, 128, "f16", 32), (9, 3, 128, "bf16", 16), (16, 4, 64, "f16", 64),
    (5, 1, 64, "f16", 16), (6, 1, 128, "bf16", 128), (14, 2, 64, "bf16", 512), (8, 1, 128, "f16", 16)])
@pytest.mark.parametrize("gamma,cap", [(0.0, 0.0), (1.0, 0.0), (0.9, 5.0)])
def test_few_columns(HQ, HK, D, dtype, page, gamma, cap):
    """Every number of queries whose columns (queries times group) number 16 at most, none among them."""
    most = 16 * HK // HQ
    q_lens = [min(n, 1 + i % most) if i % 5 else 0 for i, n in enumerate(EDGES)]
    q_lens[-1] = most
    run(EDGES, q_lens, HQ, HK, D, dtype, page, gamma, cap, gap=1)


def test_few_columns_over_long_rows():
    run([40000, 3, 9001], [2, 2, 1], 8, 1, 128, "bf16", 16, 0.99, seed=3)
    run([12000], [16], 4, 4, 64, "f16", 64, 1.0, seed=4)


@pytest.mark.parametrize("HQ,HK,D,dtype,page", [
    (2, 2, 64, "bf16", 16), (6, 3, 128, "f16", 32), (9, 3, 128, "bf16", 16), (16, 4, 128, "bf16", 64),
    (5, 1, 64, "f16", 16), (6, 1, 128, "bf16", 128), (14, 2, 64, "bf16", 512), (8, 1, 128, "f16", 16)])
@pytest.mark.parametrize("gamma,cap", [(0.0, 0.0), (1.0, 0.0), (0.9, 5.0)])
def test_chunks(HQ, HK, D, dtype, page, gamma, cap):
    """Mixed batch: one query, none, few, many; whole prompts and chunks after cached rows."""
    lens = [300, 64, 0, 33, 129, 200, 1, 65, 500]
    q_lens = [1, 64, 0, 7, 129, 0, 1, 2, 131]
    run(lens, q_lens, HQ, HK, D, dtype, page, gamma, cap, gap=1)


def test_few_queries_over_long_rows():
    """Key ranges of their own blocks, several windows of page numbers."""
    run([9000, 2500, 700], [5, 130, 1], 8, 2, 128, "bf16", 16, 1.0, seed=5)
    run([20000], [2], 4, 1, 64, "f16", 64, 0.9, cap=20.0, seed=6)


@pytest.mark.parametrize("B", [70, 300])
def test_chunks_of_many_sequences(B):
    """Lists that no longer fit one entry a thread, and the planning block's larger forms."""
    lens = [1 + 37 * i % 90 for i in range(B)]
    q_lens = [min(n, 9 + i % 23) if i % 4 else i % 3 for i, n in enumerate(lens)]
    run(lens, [min(n, q) for n, q in zip(lens, q_lens)], 6, 2, 64, "bf16", 16, 0.9, seed=9)


def test_as_many_key_ranges_as_a_tile_can_have():
    run([20000], [6], 4, 1, 64, "f16", 64, 0.9, cap=20.0, seed=7)
    run([4700, 2100, 300], [40, 9, 6], 4, 1, 128, "bf16", 16, 1.0, seed=8)


@pytest.mark.parametrize("cap", [1e-38, 1e-6, 1024.0])
def test_smallest_and_largest_caps(cap):
    run([100, 65], [1, 1], 4, 2, 64, cap=cap)
    run([100, 65], [30, 1], 4, 2, 64, "f16", cap=cap)


def test_layers_and_loose_bounds():
    run([100, 17], [1, 1], 4, 2, 64, layers=3, layer=2, loose=True)
    run([100, 17], [40, 1], 4, 2, 64, layers=3, layer=1, loose=True)


def test_given_scale_and_large_logits():
    run([333, 50], [1, 1], 4, 2, 128, scale=1.5, gamma=1.0)
    run([333, 50], [60, 3], 4, 2, 128, scale=1.5, gamma=1.0)


@pytest.mark.parametrize("q_lens", [[1, 1], [4, 3], [5, 40]])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_values_that_no_query_attends_stay_out(q_lens, dtype):
    """NaN and infinities in later rows reach the queries that attend them and no others."""
    HQ, HK, D = 8, 2, 128
    pool, rows, g = filled([90, 200], HQ, HK, D, dtype, 16, 11)
    q_start, q_len, total = batch(q_lens)
    q = torch.randn((total, HQ, D), generator=g).to(pool.dtype).to(DEV)
    new = []
    for b, (K, V, s) in enumerate(rows):
        n = K.shape[1]
        V = V.clone()
        if q_lens[b] > 1:  # only the last queries attend these
            V[0, n - 1] = float("inf")
            V[1, n - 2, 5] = float("nan")
            V[1, n - 3, 7] = float("-inf")  # with three queries, every one of them attends this
        pool.put(0, b, K, V, s, torch.arange(n).expand(HK, n))
        new.append((K, V, s))
    out = torch.zeros_like(q)
    ws = pool.cache.attn_workspace(total, max(q_lens), 200)
    L.paged_attn_score(pool.cache, 0, q, q_start, q_len, max(q_lens), 200, 0.9, 0.0, 0.0, out, ws)
    torch.cuda.synchronize()
    check(pool, new, q, q_start, q_lens, out, 0.9, 1 / math.sqrt(D), 0.0)


@pytest.mark.parametrize("q_lens", [[1, 1, 1], [3, 8, 1], [3, 30, 1]])
def test_rows_on_pages_out_of_range_are_not_attended(q_lens):
    HQ, HK, D, lens = 4, 2, 64, [100, 77, 20]
    pool, rows, g = filled(lens, HQ, HK, D, "bf16", 16, 12)
    q_start, q_len, total = batch(q_lens)
    q = torch.randn((total, HQ, D), generator=g).bfloat16().to(DEV)
    gone = {0: (32, 48), 1: (0, 16), 2: (0, 20)}
    c = pool.cache
    c.page_table[0, 0, 2] = -1
    c.page_table[0, 1, 0] = c.num_pages
    c.page_table[0, 2, :2] = 2 ** 31 - 1
    out = torch.full_like(q, 9.0)
    ws = c.attn_workspace(total, max(q_lens), 100)
    L.paged_attn_score(c, 0, q, q_start, q_len, max(q_lens), 100, 0.5, 0.0, 0.0, out, ws)
    torch.cuda.synchronize()
    assert int(c.dev_status[0]) == L.DEV_BAD_LAYOUT
    for b, (K, V, s) in enumerate(rows):
        a, e = gone[b]
        left = [r for r in range(lens[b]) if not a <= r < e]
        at, ql = int(q_start[b]), q_lens[b]
        if not left:
            assert torch.all(out[at:at + ql] == 0)
            continue
        assert left[-1] >= lens[b] - ql or ql == 1  # the newest rows are there
        ref, size, snew, stol, worst = plain.attend(q[at:at + ql].cpu(), K[:, left], V[:, left], s[:, left], 0.5,
                                                    1 / math.sqrt(D), 0.0)
        tol = plain.out_tolerance(ref, size, worst, pool.dtype, 0.0)
        assert torch.all((out[at:at + ql].cpu().double() - ref).abs() <= tol)
        got = pool.get("score", 0, b, lens[b])
        assert torch.all((got[:, left].double() - snew).abs() <= stol)
        assert torch.equal(got[:, a:e], s[:, a:e])


def test_refused_sequences_leave_the_others_alone():
    lens = [50, 60, 70, 80, 90]
    for q_lens in ([1, 1, 1, 1, 1], [3, 9, 2, 5, 20]):
        pool, rows, g = filled(lens, 4, 2, 64, "f16", 16, 13)
        q_start, q_len, total = batch(q_lens)
        q = torch.randn((total, 4, 64), generator=g).half().to(DEV)
        out = torch.full_like(q, 9.0)
        c = pool.cache
        q_len[0] = -1
        c.len[0, 1] = 4000
        q_start[2] = total
        c.len[0, 3] = 0
        ws = c.attn_workspace(total, max(q_lens), 90)
        L.paged_attn_score(c, 0, q, q_start, q_len, max(q_lens), 90, 0.5, 0.0, 0.0, out, ws)
        torch.cuda.synchronize()
        assert int(c.dev_status[0]) == L.DEV_BAD_LAYOUT
        at = int(q_start[4])
        assert torch.all(out[:at] == 9.0)
        for b in range(4):
            assert torch.equal(pool.get("score", 0, b, lens[b]), rows[b][2])
        q_lens = [0, 0, 0, 0, q_lens[4]]
        check(pool, rows, q, q_start, q_lens, out, 0.5, 1 / 8, 0.0)


@pytest.mark.parametrize("q_lens", [[1, 1, 1], [1, 200, 33]])
def test_same_bits_on_a_stream_and_in_a_graph(q_lens):
    """Repeated calls, a side stream and replays of a captured call give the same bits; each replay attends what the
    cache holds then."""
    pool, rows, g = filled([3000, 400, 33], 8, 2, 128, "bf16", 16, 14)
    c = pool.cache
    q_start, q_len, total = batch(q_lens)
    q = torch.randn((total, 8, 128), generator=g).bfloat16().to(DEV)
    ws = c.attn_workspace(total, max(q_lens), 3000)
    score0 = c.score.clone()

    def call(out, w):
        L.paged_attn_score(c, 0, q, q_start, q_len, max(q_lens), 3000, 0.9, 0.0, 0.0, out, w)

    def eager(w):
        out = torch.zeros_like(q)
        c.score.copy_(score0)
        call(out, w)
        torch.cuda.synchronize()
        return out, c.score.clone()

    want, wscore = eager(ws)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got, gscore = eager(c.attn_workspace(total, max(q_lens), 3000))
    assert torch.equal(got, want) and torch.equal(gscore.nan_to_num(), wscore.nan_to_num())
    out = torch.zeros_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out, ws)
    for i in range(4):
        q.mul_(-1 if i % 2 else 1)
        want, wscore = eager(c.attn_workspace(total, max(q_lens), 3000))
        c.score.copy_(score0)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(c.score.nan_to_num(), wscore.nan_to_num())
