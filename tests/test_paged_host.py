"""Host checks of the paged cache's calls: what they refuse before anything reaches the device, and workspace sizes."""
import ctypes
import math

import pytest
import torch

import paged_plain as plain
from paper_2511_06029_amd import lethe as L

FAKE = 0x10000  # never dereferenced: every call below fails validation first
BIG = 1 << 50


def make(**kw):
    c = L.CPagedCache(FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 1000, 16, 64, 2, 4, 32, 8, 128, L.BF16, FAKE)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def rotary(**kw):
    r = L.CRotary(FAKE, FAKE, 128, 3, (ctypes.c_int32 * 4)(16, 24, 24, 0), 0)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def append(c, layer=0, q=FAKE, qs=4096, k=FAKE, ks=1024, v=FAKE, vs=1024, start=FAKE, length=FAKE, rows=4, most=1,
           rot=None, out=FAKE):
    return L.load().lethe_paged_append(ctypes.byref(c), layer, q, qs, k, ks, v, vs, start, length, rows, most,
                                       None if rot is None else ctypes.byref(rot), out, None)


def attn(c, layer=0, q=FAKE, start=FAKE, length=FAKE, rows=4, most=1, kv=100, gamma=0.9, scale=0.0, cap=0.0, out=FAKE,
         ws=FAKE, wsb=BIG):
    return L.load().lethe_paged_attn_score(ctypes.byref(c), layer, q, start, length, rows, most, kv, gamma, scale, cap,
                                           out, ws, wsb, None)


def evict(c, budget=FAKE, recent=1, sink=0, kv=100, ws=FAKE, wsb=BIG):
    return L.load().lethe_paged_evict(ctypes.byref(c), budget, recent, sink, kv, ws, wsb, None)


@pytest.mark.parametrize("field,value,want", [
    ("k", None, L.ERR_INVALID), ("v", None, L.ERR_INVALID), ("len", None, L.ERR_INVALID),
    ("page_table", None, L.ERR_INVALID), ("dev_status", None, L.ERR_INVALID), ("score", None, L.ERR_INVALID),
    ("k", FAKE + 8, L.ERR_INVALID), ("v", FAKE + 2, L.ERR_INVALID),
    ("num_pages", 0, L.ERR_INVALID), ("page_size", 0, L.ERR_INVALID), ("max_pages", 0, L.ERR_INVALID),
    ("num_layers", 0, L.ERR_INVALID), ("num_seqs", 0, L.ERR_INVALID), ("num_kv_heads", 0, L.ERR_INVALID),
    ("num_q_heads", 30, L.ERR_INVALID), ("dtype", 7, L.ERR_INVALID), ("dtype", L.F32, L.ERR_UNSUPPORTED),
    ("head_dim", 96, L.ERR_UNSUPPORTED), ("num_q_heads", 72, L.ERR_UNSUPPORTED), ("num_seqs", 1025, L.ERR_UNSUPPORTED),
    ("num_layers", 257, L.ERR_UNSUPPORTED), ("page_size", 8, L.ERR_UNSUPPORTED), ("page_size", 48, L.ERR_UNSUPPORTED),
    ("page_size", 2048, L.ERR_UNSUPPORTED), ("num_pages", 1 << 24, L.ERR_UNSUPPORTED),
    ("max_pages", 1 << 27, L.ERR_UNSUPPORTED)])
def test_cache_validation(field, value, want):
    c = make(**{field: value})
    assert append(c) == want and attn(c) == want and evict(c) == want
    if want == L.ERR_UNSUPPORTED or value == 0:
        lib = L.load()
        assert lib.lethe_paged_attn_workspace_bytes(ctypes.byref(c), 4, 1, 100) == 0
        assert lib.lethe_paged_evict_workspace_bytes(ctypes.byref(c)) == 0


def test_the_other_calls_refuse_the_paged_type():
    c = L.CCache(FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 4096, 2, 4, 32, 8, 128, L.F16, FAKE, FAKE)
    assert L.load().lethe_score_flush(ctypes.byref(c), None) == L.ERR_INVALID


def test_append_arguments():
    c = make()
    for kw in (dict(layer=-1), dict(layer=2), dict(k=None), dict(v=None), dict(start=None), dict(length=None),
               dict(q=None), dict(out=None), dict(q=FAKE + 4), dict(k=FAKE + 8), dict(v=FAKE + 8), dict(out=FAKE + 8),
               dict(qs=4095), dict(qs=4100), dict(ks=1000), dict(ks=1028), dict(vs=0), dict(vs=-1024), dict(rows=-1),
               dict(most=-1)):
        assert append(c, **kw) == L.ERR_INVALID, kw
    assert append(c, rows=1 << 30) == L.ERR_UNSUPPORTED
    assert append(make(pos=None)) == L.ERR_INVALID and append(make(seen=None)) == L.ERR_INVALID
    bad = (ctypes.c_int32 * 4)(16, 24, 25, 0)
    less = (ctypes.c_int32 * 4)(80, -16, 0, 0)
    for kw in (dict(inv_freq=None), dict(axis_pos=None), dict(rot_dim=0), dict(rot_dim=24), dict(rot_dim=144),
               dict(num_axes=0), dict(num_axes=5), dict(sections=bad), dict(sections=less), dict(adjacent=2)):
        assert append(c, rot=rotary(**kw)) == L.ERR_INVALID, kw


def test_attention_arguments():
    c = make()
    for kw in (dict(layer=-1), dict(layer=2), dict(q=None), dict(start=None), dict(length=None), dict(out=None),
               dict(ws=None), dict(q=FAKE + 8), dict(out=FAKE + 8), dict(ws=FAKE + 16), dict(rows=-1), dict(most=-1),
               dict(kv=-1), dict(gamma=-0.1), dict(gamma=1.1), dict(gamma=math.nan), dict(scale=math.nan),
               dict(scale=math.inf), dict(cap=-1.0), dict(cap=math.nan), dict(cap=math.inf)):
        assert attn(c, **kw) == L.ERR_INVALID, kw
    assert attn(c, cap=1024.5) == L.ERR_UNSUPPORTED and attn(c, cap=1024.0, wsb=0) == L.ERR_WORKSPACE
    assert attn(make(score=None)) == L.ERR_INVALID
    for most in (1, 4):
        need = L.load().lethe_paged_attn_workspace_bytes(ctypes.byref(c), 4, most, 100)
        assert need > 0 and attn(c, most=most, wsb=need - 1) == L.ERR_WORKSPACE
    huge = make(num_seqs=1024, max_pages=1 << 26)
    assert L.load().lethe_paged_attn_workspace_bytes(ctypes.byref(huge), 4, 1, 2 ** 31 - 1) == 0
    assert attn(huge, kv=2 ** 31 - 1) == L.ERR_UNSUPPORTED
    wide = make(num_seqs=1024, num_q_heads=8192, num_kv_heads=8192)
    assert L.load().lethe_paged_attn_workspace_bytes(ctypes.byref(wide), 4, 1, 16) == 0


def test_eviction_arguments():
    c = make()
    for kw in (dict(budget=None), dict(recent=-1), dict(sink=-1), dict(kv=-1), dict(ws=None), dict(ws=FAKE + 8)):
        assert evict(c, **kw) == L.ERR_INVALID, kw
    assert evict(make(pos=None)) == L.ERR_INVALID and evict(make(seen=None)) == L.ERR_INVALID
    need = L.load().lethe_paged_evict_workspace_bytes(ctypes.byref(c))
    assert need >= 1000 * 8 * 16 * 8 and evict(c, wsb=need - 1) == L.ERR_WORKSPACE


def test_tensors_of_another_shape_or_type():
    pool = plain.Pool(1, 2, [[20, 20]], 4, 2, 64, "bf16", 16, 1, device="cpu")
    c = pool.cache
    start, length = torch.zeros(2, dtype=torch.int64), torch.zeros(2, dtype=torch.int32)
    q, kv = torch.zeros((3, 4, 64), dtype=torch.bfloat16), torch.zeros((3, 2, 64), dtype=torch.bfloat16)

    def refused(fn):
        with pytest.raises(L.LetheError) as e:
            fn()
        assert e.value.status == L.ERR_INVALID

    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    for args in ((q.float(), kv, kv, q), (q, kv[:, :1], kv, q), (q, kv, kv[:2], q), (q, kv.transpose(0, 1), kv, q),
                 (q, kv, kv, q[:2]), (q, kv, kv, q.half()), (q[:, :, ::2], kv, kv, q)):
        refused(lambda: L.paged_append(c, 0, args[0], args[1], args[2], start, length, 1, None, args[3]))
    refused(lambda: L.paged_append(c, 0, q, kv, kv, start.int(), length, 1, None, q))
    refused(lambda: L.paged_append(c, 0, q, kv, kv, start, length[:1], 1, None, q))
    short = L.Rotary(torch.zeros(32), torch.zeros((1, 2), dtype=torch.int32), [32])
    refused(lambda: L.paged_append(c, 0, q, kv, kv, start, length, 1, short, q))
    refused(lambda: L.paged_attn_score(c, 0, q.half(), start, length, 1, 20, 1.0, 0.0, 0.0, q, ws))
    refused(lambda: L.paged_attn_score(c, 0, q, start, length, 1, 20, 1.0, 0.0, 0.0, q[:2], ws))
    refused(lambda: L.paged_attn_score(c, 0, q, start, length.long(), 1, 20, 1.0, 0.0, 0.0, q, ws))
    refused(lambda: L.paged_evict(c, torch.zeros((1, 2), dtype=torch.int32), 0, 0, ws))
    refused(lambda: L.paged_evict(c, torch.zeros((2, 1), dtype=torch.int64), 0, 0, ws))
    refused(lambda: L.Rotary(torch.zeros(32).double(), torch.zeros((1, 2), dtype=torch.int32), [32]))
    refused(lambda: L.Rotary(torch.zeros(32), torch.zeros((1, 2), dtype=torch.int64), [32]))
    refused(lambda: L.Rotary(torch.zeros(32), torch.zeros((2, 2), dtype=torch.int32), [32]))
    refused(lambda: L.LethePagedCache(c.k, c.v.half(), c.score, c.pos, c.len, c.seen, c.page_table, 4))
    refused(lambda: L.LethePagedCache(c.k, c.v, c.score, c.pos, c.len, c.seen[:, :1], c.page_table, 4))
    with pytest.raises(L.LetheError) as e:
        L.LethePagedCache(c.k, c.v, c.score, c.pos, c.len, c.seen, c.page_table, 18)
    assert e.value.status == L.ERR_UNSUPPORTED


def test_tensors_on_another_device():
    pool = plain.Pool(1, 2, [[20, 20]], 4, 2, 64, "bf16", 16, 1, device="cpu")
    c = pool.cache
    bf16, i32, i64 = torch.bfloat16, torch.int32, torch.int64
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    append = [torch.zeros((3, 4, 64), dtype=bf16), torch.zeros((3, 2, 64), dtype=bf16),
              torch.zeros((3, 2, 64), dtype=bf16), torch.zeros(2, dtype=i64), torch.zeros(2, dtype=i32),
              torch.zeros(32), torch.zeros((1, 3), dtype=i32), torch.zeros((3, 4, 64), dtype=bf16)]
    attend = [append[0], append[3], append[4], append[7], ws]
    prune = [torch.zeros((2, 1), dtype=i32), ws]

    def do_append(q, k, v, start, length, freq, axis, out):
        L.paged_append(c, 0, q, k, v, start, length, 1, L.Rotary(freq, axis, [32]), out)

    def do_attend(q, start, length, out, w):
        L.paged_attn_score(c, 0, q, start, length, 1, 20, 1.0, 0.0, 0.0, out, w)

    for fn, tensors in ((do_append, append), (do_attend, attend), (lambda b, w: L.paged_evict(c, b, 0, 0, w), prune)):
        for i in range(len(tensors)):
            args = [t.to("meta") if i == j else t for j, t in enumerate(tensors)]
            with pytest.raises(L.LetheError) as e:
                fn(*args)
            assert e.value.status == L.ERR_INVALID
    for fn in (lambda w: do_attend(*attend[:4], w), lambda w: L.paged_evict(c, prune[0], 0, 0, w)):
        with pytest.raises(L.LetheError) as e:
            fn(ws[::2])
        assert e.value.status == L.ERR_INVALID


def test_plain_eviction_is_a_permutation_of_the_rule():
    """The plain form the GPU tests compare with: kept tokens against a direct ranking, movers only from the tail."""
    g = torch.Generator().manual_seed(4)
    for n, k, r, s in ((1, 0, 0, 0), (10, 4, 2, 1), (50, 20, 30, 5), (50, 20, 5, 30), (64, 63, 0, 0), (8, 9, 1, 1)):
        pos = torch.randperm(3 * n, generator=g)[:n]
        score = (torch.rand(n, generator=g) * 5).floor()
        place, m = plain.evict(n, k, r, s, score, pos)
        assert m == min(n, k) and place[m:] == list(range(m, n))
        kept = sorted(place[:m])
        assert len(set(kept)) == m
        assert all(p == d or p >= m for d, p in enumerate(place[:m]))
        age = torch.argsort(pos).tolist()
        r, s = min(r, m), min(s, m - min(r, m))
        assert set(age[:s]) <= set(kept) and set(age[n - r:]) <= set(kept)
        rest = [j for j in age[s:n - r]]
        best = sorted(rest, key=lambda j: (-float(score[j]), int(pos[j])))[:m - r - s]
        if m < n:
            assert set(kept) == set(age[:s]) | set(age[n - r:]) | set(best)
