"""lethe_paged_append against the plain form in 64 bits: rotation with one to four axes, both pairings, partial
rotation, strided inputs, ragged chunks, pages of every kind, refused sequences."""
import pytest
import torch

import paged_plain as plain
from paper_2511_06029_amd import lethe as L

pytestmark = pytest.mark.gpu
DEV = "cuda"


def batch(lens, first_row=0, gap=0):
    """q_start and q_len of consecutive chunks, `gap` rows of no sequence between them."""
    starts, at = [], first_row
    for q in lens:
        starts.append(at)
        at += q + gap
    return (torch.tensor(starts, dtype=torch.int64), torch.tensor(lens, dtype=torch.int32), at)


CASES = [
    # dtype, D, HQ, HK, page, cached rows, new rows, sections, adjacent, packed, gap
    ("bf16", 128, 32, 8, 16, [1111], [1], [64], False, True, 0),
    ("bf16", 128, 8, 8, 64, [0, 5, 64, 63], [1, 1, 1, 1], [64], True, False, 2),
    ("f16", 64, 4, 2, 16, [0, 17, 3, 40], [33, 0, 1, 16], [8, 12, 12], False, True, 1),
    ("bf16", 128, 28, 4, 32, [200, 31, 0], [100, 257, 2], [16, 24, 24], False, True, 0),
    ("f16", 128, 5, 1, 1024, [1000, 1], [30, 1100], [0, 0, 32], True, False, 3),
    ("bf16", 64, 9, 3, 128, [1, 127, 128, 129, 0], [1, 2, 1, 0, 9], [4, 4, 0, 0], False, True, 0),
    ("f16", 64, 16, 2, 16, [7], [4000], [16, 8, 4, 4], True, True, 0),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s-D%d-%d/%d-page%d" % c[:5])
def test_append(case):
    dtype, D, HQ, HK, page, cached, new, sections, adjacent, packed, gap = case
    T = plain.DTYPES[dtype]
    g = torch.Generator().manual_seed(sum(cached) + D + page)
    B = len(cached)
    q_start, q_len, rows = batch(new, first_row=gap, gap=gap)
    qkv = torch.randn((rows, HQ + 2 * HK, D), generator=g).to(T)
    half = sum(sections)
    axis_pos = torch.randint(-50, 3000, (len(sections), rows), generator=g).int()
    axis_pos[0] += 1000000  # far positions: an fp32 product would lose the angle
    inv_freq = (10000.0 ** (-torch.arange(half).double() / half)).float()
    for layer in (0, 1):
        pool = plain.Pool(2, B, [[n + m for n, m in zip(cached, new)]] * 2, HQ, HK, D, dtype, page, 3 + layer,
                          fill=float("nan"))
        c = pool.cache
        c.len.copy_(torch.tensor([cached] * 2))
        c.seen.copy_(torch.tensor([[n + 11 for n in cached]] * 2))
        before = {x: getattr(c, x).clone() for x in ("k", "v", "score", "pos")}
        dev = qkv.to(DEV)
        parts = (dev[:, :HQ], dev[:, HQ:HQ + HK], dev[:, HQ + HK:])
        if not packed:
            parts = tuple(x.contiguous() for x in parts)
        q_out = torch.full((rows, HQ, D), 99.0, dtype=T, device=DEV)
        rotary = L.Rotary(inv_freq.to(DEV), axis_pos.to(DEV), sections, adjacent)
        L.paged_append(c, layer, *parts, q_start.to(DEV), q_len.to(DEV), max(new), rotary, q_out)
        torch.cuda.synchronize()
        assert int(c.dev_status[0]) == 0
        rot, size = plain.rotate(qkv[:, :HQ + HK], axis_pos, inv_freq, sections, adjacent)
        tol = plain.rounding(rot, size, T)
        written = torch.zeros(c.score.shape, dtype=torch.bool)
        for b in range(B):
            rs = slice(int(q_start[b]), int(q_start[b]) + new[b])
            assert torch.all((q_out[rs].cpu().double() - rot[rs, :HQ]).abs() <= tol[rs, :HQ])
            n = cached[b] + new[b]
            K, V = pool.get("k", layer, b, n)[:, cached[b]:], pool.get("v", layer, b, n)[:, cached[b]:]
            assert torch.all((K.transpose(0, 1).double() - rot[rs, HQ:]).abs() <= tol[rs, HQ:])
            assert torch.equal(V.transpose(0, 1), qkv[rs, HQ + HK:])
            assert torch.all(pool.get("score", layer, b, n)[:, cached[b]:] == 0)
            want = cached[b] + 11 + torch.arange(new[b])
            assert torch.equal(pool.get("pos", layer, b, n)[:, cached[b]:].long(), want.expand(HK, -1))
            pg, off = pool.slots(layer, b, n)
            written[pg[cached[b]:], :, off[cached[b]:]] = True
        # Rows of no sequence, other rows and the other layer stay as they were.
        mine = torch.zeros(rows, dtype=torch.bool)
        for b in range(B):
            mine[int(q_start[b]):int(q_start[b]) + new[b]] = True
        assert torch.all(q_out.cpu()[~mine] == 99.0)
        for x in before:
            a, z = getattr(c, x).cpu()[~written], before[x].cpu()[~written]
            assert torch.equal(a.nan_to_num(nan=5.0), z.nan_to_num(nan=5.0)), x
        want = torch.tensor([cached] * 2)
        want[layer] += torch.tensor(new)
        assert torch.equal(c.len.cpu().long(), want) and torch.equal(c.seen.cpu().long() - 11, want)


def test_without_rotation_in_place_and_without_queries():
    pool = plain.Pool(1, 2, [[40, 40]], 8, 2, 64, "bf16", 16, 1)
    c = pool.cache
    q_start, q_len, rows = batch([3, 20])
    g = torch.Generator().manual_seed(2)
    q = torch.randn((rows, 8, 64), generator=g).bfloat16().to(DEV)
    k, v = (torch.randn((rows, 2, 64), generator=g).bfloat16().to(DEV) for _ in range(2))
    was = q.clone()
    L.paged_append(c, 0, q, k, v, q_start.to(DEV), q_len.to(DEV), 20, None, q)
    assert torch.equal(q, was)
    L.paged_append(c, 0, None, k, v, q_start.to(DEV), q_len.to(DEV), 64, None, None)
    torch.cuda.synchronize()
    assert c.len.tolist() == [[6, 40]] and int(c.dev_status[0]) == 0
    assert torch.equal(pool.get("k", 0, 1, 40), k[3:].cpu().repeat(2, 1, 1).transpose(0, 1))
    # In place, rotated: the same as out of place.
    rot = L.Rotary(torch.rand(32, device=DEV), torch.arange(rows, device=DEV, dtype=torch.int32)[None], [32])
    out = torch.zeros_like(q)
    q_len.fill_(0)
    q_len[1] = 0
    L.paged_append(c, 0, q, k, v, q_start.to(DEV), torch.tensor([0, 0], dtype=torch.int32, device=DEV), 1, rot, out)
    torch.cuda.synchronize()
    assert torch.all(out == 0) and c.len.tolist() == [[6, 40]]


@pytest.mark.parametrize("lens", [[1, 1, 1, 1, 1, 1], [5, 9, 17, 3, 2, 6]])
def test_refused_sequences_leave_the_others_alone(lens):
    """Overflow, a page out of range, a length out of range, a negative chunk: flagged and skipped."""
    B = 6
    pool = plain.Pool(1, B, [[32] * B], 4, 2, 64, "f16", 16, 5)
    c = pool.cache
    c.len.copy_(torch.tensor([[14, 32, 3, 99, 4, 8]]))
    c.seen.copy_(torch.tensor([[14, 40, 3, 99, 4, 8]]))
    c.page_table[0, 2, 0] = c.num_pages
    q_start, q_len, rows = batch(lens)
    q_len[4] = -1
    g = torch.Generator().manual_seed(7)
    q = torch.randn((rows, 4, 64), generator=g).half().to(DEV)
    k, v = (torch.randn((rows, 2, 64), generator=g).half().to(DEV) for _ in range(2))
    before = c.k.clone()
    out = torch.zeros_like(q)
    L.paged_append(c, 0, q, k, v, q_start.to(DEV), q_len.to(DEV), max(lens), None, out)
    torch.cuda.synchronize()
    assert int(c.dev_status[0]) == L.DEV_APPEND_OVERFLOW | L.DEV_BAD_LAYOUT
    assert c.len.tolist() == [[14 + lens[0], 32, 3, 99, 4, 8 + lens[5]]]
    for b, n0 in ((0, 14), (5, 8)):
        rs = slice(int(q_start[b]), int(q_start[b]) + lens[b])
        assert torch.equal(pool.get("k", 0, b, n0 + lens[b])[:, n0:].transpose(0, 1), k[rs].cpu())
        assert torch.equal(out[rs].cpu(), q[rs].cpu())
        pg, off = pool.slots(0, b, n0 + lens[b])
        before[pg[n0:].to(DEV), :, off[n0:].to(DEV)] = c.k[pg[n0:].to(DEV), :, off[n0:].to(DEV)]
    assert torch.equal(c.k, before)
