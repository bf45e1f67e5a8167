"""The paged cache's calls in plain torch on the CPU, in 64 bits, and the layout helpers of their tests.

A segment's rows are held densely here ([rows][D] per (layer, sequence, KV head)); ``Pool`` scatters them over randomly
placed pages of a LethePagedCache and gathers them back, page by page in Python.
"""
import math

import torch

from paper_2511_06029_amd import lethe as L

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


class Pool:
    """A paged cache whose tables name pages in random order, with `spare` unused pages around them."""

    def __init__(self, layers, seqs, room, HQ, HK, D, dtype, page, seed, device="cuda", spare=3, fill=0.0):
        g = torch.Generator().manual_seed(seed)
        self.g, self.HK, self.D, self.page, self.dtype = g, HK, D, page, DTYPES[dtype]
        used = [[-(-room[l][b] // page) for b in range(seqs)] for l in range(layers)]
        P = sum(map(sum, used)) + spare
        most = max(1, max(map(max, used)))
        ids = torch.randperm(P, generator=g).tolist()
        self.table = torch.full((layers, seqs, most), -1, dtype=torch.int32)
        for l in range(layers):
            for b in range(seqs):
                for i in range(used[l][b]):
                    self.table[l, b, i] = ids.pop()
        rows = (P, HK, page)
        dev = lambda t: t.to(device)  # noqa: E731
        self.cache = L.LethePagedCache(
            dev(torch.full(rows + (D,), fill, dtype=self.dtype)), dev(torch.full(rows + (D,), fill, dtype=self.dtype)),
            dev(torch.full(rows, fill)), dev(torch.full(rows, -7, dtype=torch.int32)),
            dev(torch.zeros((layers, seqs), dtype=torch.int32)), dev(torch.zeros((layers, seqs), dtype=torch.int32)),
            dev(self.table), HQ)

    def slots(self, l, b, n):
        """(page, row in page) of a sequence's first n rows."""
        r = torch.arange(n)
        return self.table[l, b].long()[r // self.page], r % self.page

    def put(self, l, b, K, V, score, pos, seen=None):
        """Rows of a segment from K, V [HK][n][D], score and pos [HK][n]."""
        c, n = self.cache, K.shape[1]
        page, off = self.slots(l, b, n)
        dev = c.k.device
        page, off = page.to(dev), off.to(dev)
        c.k[page, :, off] = K.transpose(0, 1).to(self.dtype).to(dev)
        c.v[page, :, off] = V.transpose(0, 1).to(self.dtype).to(dev)
        c.score[page, :, off] = score.t().float().to(dev)
        c.pos[page, :, off] = pos.t().int().to(dev)
        c.len[l, b] = n
        c.seen[l, b] = n if seen is None else seen

    def get(self, what, l, b, n):
        """[HK][n](...) rows of a segment, on the CPU."""
        page, off = self.slots(l, b, n)
        return getattr(self.cache, what).cpu()[page, :, off].transpose(0, 1).contiguous()


def rotate(x, axis_pos, inv_freq, sections, adjacent):
    """x [rows][heads][D] in float64; returns the rotated values and, per element, |a| + |b| of its pair."""
    x = x.double()
    half = sum(sections)
    axis = [a for a, m in enumerate(sections) for _ in range(m)]
    y, size = x.clone(), x.abs().clone()
    for j in range(half):
        i0, i1 = (2 * j, 2 * j + 1) if adjacent else (j, j + half)
        t = axis_pos[axis[j]].double() * inv_freq[j].double()
        c, s = torch.cos(t)[:, None], torch.sin(t)[:, None]
        a, b = x[:, :, i0], x[:, :, i1]
        y[:, :, i0], y[:, :, i1] = a * c - b * s, b * c + a * s
        size[:, :, i0] = size[:, :, i1] = a.abs() + b.abs()
    return y, size


def rounding(ref, size, dtype):
    """Half a step of the result; the pair's fp32 products and the angle's fraction (2^-25 of a turn) before it."""
    fi = torch.finfo(dtype)
    return fi.eps / 2 * ref.abs() * 1.001 + size * 2.0 ** -20 + fi.smallest_normal * fi.eps / 2


def attend(q, K, V, score, gamma, scale, cap):
    """q [ql][HQ][D], K and V [HK][n][D], score [HK][n]: out [ql][HQ][D], new scores [HK][n], and the bounds of their
    errors but for the roundings to the storage type: out's in units of sum p |v|, given with it."""
    ql, HQ, D = q.shape
    HK, n, _ = K.shape
    G = HQ // HK
    q, K, V = q.double(), K.double(), V.double()
    out = torch.zeros((ql, HQ, D), dtype=torch.float64)
    size = torch.zeros((ql, HQ, D), dtype=torch.float64)
    new = gamma * score.double() if gamma else score.double().clone()
    tol = gamma * score.double().abs() * 2.0 ** -22
    far = torch.arange(n)[None, :] > torch.arange(n - ql, n)[:, None]
    worst = 0.0
    for h in range(HK):
        for g in range(G):
            x = q[:, h * G + g] @ K[h].t() * scale
            # fp32 sums of D exact products, in any order: each of D additions is off by half a step of the sum of
            # absolute values at most.
            dx = (q[:, h * G + g].abs() @ K[h].abs().t() * scale) * (D * 2.0 ** -24) + x.abs() * 2.0 ** -22
            if cap:
                x = cap * torch.tanh(x / cap)
                dx = dx + cap * 2.0 ** -20  # exp2 and reciprocal of one step each, near 1, times 2 cap
            x = x.masked_fill(far, -math.inf)
            p = torch.softmax(x, dim=1)
            ok = torch.where(far, 0.0, dx).masked_fill(torch.isnan(dx), 0.0)
            rel = 2.0 * ok.max().item() + 2.0 ** -20  # of a weight: its exponent's error and the maximum's
            worst = max(worst, rel)
            pv = torch.where(far[:, :, None], 0.0, p[:, :, None] * V[h][None]) if not torch.isfinite(V[h]).all() else None
            out[:, h * G + g] = p @ V[h] if pv is None else pv.sum(1)
            size[:, h * G + g] = p @ V[h].abs() if pv is None else pv.abs().sum(1)
            if gamma:
                new[h] += p.sum(0)
                tol[h] += p.sum(0) * (rel + (ql * G) * 2.0 ** -24) + 2.0 ** -40
    return out, size, new, tol, worst


def out_tolerance(out, size, worst, dtype, vmax):
    """Half a step of the result, half a step of every weight, and the weights' own error; fp16 weights below 2^-14 of
    the largest are on a fixed grid of 2^-24."""
    half = torch.finfo(dtype).eps / 2
    tol = half * out.abs() + (1.02 * half + worst) * size + 2.0 ** -30
    if dtype == torch.float16:
        tol = tol + 2.0 ** -25 * vmax
    return tol


def evict(n, k, recent, sink, score, pos):
    """One segment: the row that lies at each of the n places afterwards (places past k keep theirs)."""
    place = list(range(n))
    k = max(k, 0)
    if k >= n:
        return place, n
    r = min(recent, k)
    s = min(sink, k - r)
    age = sorted(range(n), key=lambda j: int(pos[j]))
    held = set(age[:s]) | set(age[n - r:])

    def order(j):
        v = float(score[j])
        return (1, 0.0, int(pos[j])) if math.isnan(v) else (0, -v, int(pos[j]))

    rest = sorted((j for j in range(n) if j not in held), key=order)
    kept = held | set(rest[:k - r - s])
    holes = [j for j in range(k) if j not in kept]
    movers = [j for j in range(k, n) if j in kept]
    for d, m in zip(holes, movers):
        place[d] = m
    assert len(holes) == len(movers) and len(kept) == k
    return place, k
