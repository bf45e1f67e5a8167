"""lethe_paged_evict against the plain form: the kept rows, their places, bits, scores and tokens, exactly."""
import pytest
import torch

import paged_plain as plain
from paper_2511_06029_amd import lethe as L

pytestmark = pytest.mark.gpu
DEV = "cuda"


def tokens(n, HK, g, kind):
    """Distinct tokens of n rows a head, and how many were ever appended."""
    if kind == "fresh":  # nothing evicted yet
        return torch.arange(n).expand(HK, n).contiguous(), n
    top = {"holes": 3 * n + 7, "wide": 70000 + 2 * n}[kind]
    return torch.stack([torch.randperm(top, generator=g)[:n] for _ in range(HK)]), top


def scores(n, HK, g, kind):
    s = torch.rand((HK, n), generator=g)
    if kind == "ties":
        return (s * 6).floor() / 4
    if kind == "flat":
        return torch.full((HK, n), 0.25)
    if kind == "odd":  # zeros of both signs, negatives, infinities, NaN
        x = torch.tensor([0.0, -0.0, -1.5, float("inf"), float("-inf"), float("nan"), 1e-42, 2.0])
        return x[(s * 8).long().clamp(max=7)]
    return torch.exp(8 * s)


def run(lens, budgets, recent, sink, HK=2, D=64, page=16, dtype="bf16", stok="holes", sscore="spread", seed=1, layers=1,
        table=None):
    B = len(lens)
    g = torch.Generator().manual_seed(seed)
    room = [[max(n, 1) for n in lens]] * layers
    if table:
        room = [[max(n, 1) if b else table * page for b, n in enumerate(lens)]] * layers
    pool = plain.Pool(layers, B, room, 2 * HK, HK, D, dtype, page, seed)
    c = pool.cache
    want = {}
    for l in range(layers):
        for b, n in enumerate(lens):
            K, V = torch.randn((HK, n, D), generator=g), torch.randn((HK, n, D), generator=g)
            pos, seen = tokens(n, HK, g, stok)
            s = scores(n, HK, g, sscore)
            pool.put(l, b, K, V, s, pos, seen)
            want[l, b] = (K.to(pool.dtype), V.to(pool.dtype), s, pos)
    budget = torch.tensor([[budgets[b] - 3 * l for l in range(layers)] for b in range(B)], dtype=torch.int32)
    L.paged_evict(c, budget.to(DEV), recent, sink, c.evict_workspace())
    torch.cuda.synchronize()
    assert int(c.dev_status[0]) == 0
    for (l, b), (K, V, s, pos) in want.items():
        n = lens[b]
        got = {x: pool.get(x, l, b, n) for x in ("k", "v", "score", "pos")}
        for h in range(HK):
            place, k = plain.evict(n, int(budget[b, l]), recent, sink, s[h], pos[h])
            place = torch.tensor(place, dtype=torch.long)
            assert int(c.len[l, b]) == k
            assert torch.equal(got["pos"][h].long(), pos[h][place]), (l, b, h)
            assert torch.equal(got["score"][h].view(torch.int32), s[h][place].contiguous().view(torch.int32))
            assert torch.equal(got["k"][h], K[h][place]) and torch.equal(got["v"][h], V[h][place])
    return pool


@pytest.mark.parametrize("stok", ["fresh", "holes", "wide"])
@pytest.mark.parametrize("sscore", ["spread", "ties", "flat", "odd"])
def test_lengths(stok, sscore):
    """Lengths around waves, blocks and pages; budgets of none, some, all and more."""
    lens = [0, 1, 2, 16, 63, 64, 65, 255, 256, 257, 1000, 2049]
    budgets = [0, 0, 1, 9, 64, 20, 64, -5, 255, 100, 500, 1700]
    run(lens, budgets, 16, 4, stok=stok, sscore=sscore)
    run(lens, budgets, 0, 0, stok=stok, sscore=sscore, page=64, D=128, dtype="f16", HK=3)


@pytest.mark.parametrize("recent,sink", [(0, 0), (32, 0), (0, 7), (1000, 0), (40, 1000), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_held_rows(recent, sink):
    run([300, 77, 1500], [100, 50, 900], recent, sink, stok="holes")
    run([300, 77, 1500], [100, 50, 900], recent, sink, stok="fresh", sscore="ties")


def test_layers_with_budgets_of_their_own():
    run([200, 90, 333], [150, 91, 60], 16, 2, layers=5, HK=4, D=128)


@pytest.mark.parametrize("sscore", ["spread", "ties"])
def test_long_segments(sscore):
    """More rows than the registers of 256 threads (8192) and of 1024 (32768) hold."""
    run([9000, 40], [2500, 17], 64, 4, HK=1, sscore=sscore, page=64)
    run([40000, 3000], [30000, 17], 64, 4, HK=1, sscore=sscore, page=16, stok="wide")
    run([8192, 8193], [100, 8000], 64, 4, HK=1, sscore=sscore, page=1024, stok="wide")


def test_room_beyond_the_lengths():
    """Tables with room for far more rows than are live, their further entries naming no page."""
    run([50, 3], [20, 1], 4, 1, table=600)


def test_kept_set_is_that_of_the_contiguous_selection():
    """Rows in token order: the kept tokens are lethe_rasr_select's rows."""
    n, HK, D, k = 700, 2, 64, 300
    g = torch.Generator().manual_seed(3)
    s = torch.rand((HK, n), generator=g)
    s[:, ::7] = 0.5
    pool = plain.Pool(1, 1, [[n]], 4, HK, D, "bf16", 32, 4)
    pool.put(0, 0, torch.zeros((HK, n, D)), torch.zeros((HK, n, D)), s, torch.arange(n).expand(HK, n))
    cache = L.LetheCache(1, [n], 4, HK, D, device=DEV)
    cache.score[0, :HK * n] = s.reshape(-1).to(DEV)
    cache.len[0, 0] = n
    budget = torch.tensor([[k]], dtype=torch.int32, device=DEV)
    keep = torch.zeros((1, cache.rows_per_layer), dtype=torch.uint8, device=DEV)
    L.rasr_select(cache, budget, 32, 4, keep)
    L.paged_evict(pool.cache, budget, 32, 4, pool.cache.evict_workspace())
    torch.cuda.synchronize()
    pos = pool.get("pos", 0, 0, k)
    for h in range(HK):
        assert sorted(pos[h].tolist()) == keep[0, h * n:(h + 1) * n].nonzero().flatten().tolist()


def test_refused_sequences_leave_the_others_alone():
    lens, HK, D = [60, 60, 60, 60], 2, 64
    g = torch.Generator().manual_seed(9)
    pool = plain.Pool(1, 4, [lens], 4, HK, D, "bf16", 16, 2)
    data = []
    for b, n in enumerate(lens):
        K = torch.randn((HK, n, D), generator=g)
        s = torch.rand((HK, n), generator=g)
        pool.put(0, b, K, K + 1, s, torch.arange(n).expand(HK, n))
        data.append((K.bfloat16(), s))
    c = pool.cache
    c.page_table[0, 0, 2] = -1          # a live page out of range
    c.page_table[0, 1, 3] = c.num_pages
    c.len[0, 2] = 65                    # more than its table holds
    before = {x: getattr(c, x).clone() for x in ("k", "v", "score", "pos")}
    L.paged_evict(c, torch.full((4, 1), 25, dtype=torch.int32, device=DEV), 4, 0, c.evict_workspace())
    torch.cuda.synchronize()
    assert int(c.dev_status[0]) == L.DEV_BAD_LAYOUT
    assert c.len.tolist() == [[60, 60, 65, 25]]
    changed = torch.zeros(c.score.shape, dtype=torch.bool)
    pg, off = pool.slots(0, 3, 60)
    changed[pg, :, off] = True
    for x in before:
        assert torch.equal(getattr(c, x).cpu()[~changed], before[x].cpu()[~changed])
    for h in range(HK):
        place, _ = plain.evict(60, 25, 4, 0, data[3][1][h], torch.arange(60))
        assert torch.equal(pool.get("k", 0, 3, 60)[h], data[3][0][h][torch.tensor(place)])
