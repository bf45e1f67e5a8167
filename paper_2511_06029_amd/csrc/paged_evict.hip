// Eviction from a paged cache by accumulated weight, gfx950.
//
// A segment's kept set is a rank test on (score, token); its places are the
// rows before the budget.  Kept rows already there stay, so the rows that move
// are the kept ones beyond the budget, into the places of evicted ones: at
// most min(k, n - k) rows, where order-preserving compaction moves every row
// after the first evicted one (four fifths of 2500 rows kept, 20% of them
// evicted evenly: 400 moves instead of 2000).  Tokens, not places, say which
// rows are new, so the order of places is free.
//
//  1. select_kernel, one block a segment: keys and tokens are read once into
//     registers (up to 32 rows a thread), the thresholds found by radix
//     selection, the two lists (evicted before the budget, kept beyond it)
//     ranked by ballots and one scan, and written as pairs.
//     With many segments its block moves the rows too.
//  2. move_kernel: the pairs' rows, 16 bytes a lane, spread over the chip, and
//     the new lengths; or length_kernel, the lengths alone.
// Bound by the moved rows' bytes: a steady round (2048 segments of 2500 rows, a
// fifth going) moves 0.9 GB in 215 us, selection included; 512 segments of
// 16384 rows to 30% move 1.9 GB in 400 us, 4.8 TB/s, a copy's rate, after 61 us
// of selection.
#include <algorithm>

#include "device_common.h"
#include "paged_internal.h"
#include "radix_select.h"

namespace lethe {

namespace {

constexpr unsigned kEvWhole = 1024;  // segments from which on their blocks move the rows too
constexpr int kEvUnit = 8;    // rows whose loads leave together

// One (layer, sequence) of an eviction.
struct EvSeq {
  int lb, b, n, k, seen;
  const int32_t* table;
};

__device__ inline EvSeq ev_seq(const PagedEvictArgs& a, int lb) {
  EvSeq s;
  s.lb = lb;
  s.b = lb % a.c.B;
  s.n = a.c.len[lb];
  s.k = max(a.budget[(long long)s.b * a.L + lb / a.c.B], 0);
  s.seen = a.c.seen[lb];
  s.table = a.c.table + (long long)lb * a.c.max_pages;
  return s;
}

template <int NT, int REGS>
struct EvShared : RadixShared {
  int pages[NT * REGS / 16];
  int count[2][REGS * (NT / kWave)];  // evicted / kept rows of a wave's 64, then their sums before it
  uint32_t red[2][NT / kWave];
  long long scan_tmp[NT / kWave + 1];
  int total[2];
};

template <int NT, int REGS>
__device__ inline uint2 block_sum2(uint32_t x, uint32_t y, EvShared<NT, REGS>& sh) {
  for (int o = kWave / 2; o > 0; o >>= 1) {
    x += (uint32_t)__shfl_xor(x, o);
    y += (uint32_t)__shfl_xor(y, o);
  }
  const int w = threadIdx.x / kWave;
  if ((threadIdx.x & (kWave - 1)) == 0) {
    sh.red[0][w] = x;
    sh.red[1][w] = y;
  }
  __syncthreads();
  uint2 t = make_uint2(0, 0);
  for (int i = 0; i < NT / kWave; ++i) {
    t.x += sh.red[0][i];
    t.y += sh.red[1][i];
  }
  __syncthreads();
  return t;
}

// The lists of a segment with k < n whose pages are valid.  kRegs: n <= REGS
// NT, keys and tokens in registers and the table in shared memory; otherwise
// every pass reads them again.
template <int NT, int REGS, bool kRegs>
__device__ void select_segment(const PagedEvictArgs& a, const EvSeq& s, int h, EvShared<NT, REGS>& sh, int32_t* count) {
  const int tid = threadIdx.x, lane = tid & (kWave - 1), w = tid / kWave;
  const int n = s.n, shift = a.c.page_shift, mask = (1 << shift) - 1;
  auto place = [&](int j) {
    const int page = kRegs ? sh.pages[j >> shift] : s.table[j >> shift];
    return page_row(a.c, page, h) + (j & mask);
  };
  uint32_t key[REGS];
  int tok[REGS];
  if constexpr (kRegs) {
#pragma unroll
    for (int u0 = 0; u0 < REGS; u0 += kEvUnit) {
      if (u0 * NT < n) {
        int at[kEvUnit];
        float v[kEvUnit];
#pragma unroll
        for (int u = 0; u < kEvUnit; ++u) at[u] = place(min((u0 + u) * NT + tid, n - 1));
#pragma unroll
        for (int u = 0; u < kEvUnit; ++u) {
          v[u] = a.c.score[at[u]];
          tok[u0 + u] = a.c.pos[at[u]];
        }
#pragma unroll
        for (int u = 0; u < kEvUnit; ++u) key[u0 + u] = order_key(v[u]);
      }
    }
  }
  // fn(key, token, row) for this thread's rows.
  auto each = [&](const auto& fn) {
    if constexpr (kRegs) {
#pragma unroll
      for (int u0 = 0; u0 < REGS; u0 += kEvUnit) {
        if (u0 * NT < n) {
#pragma unroll
          for (int u = 0; u < kEvUnit; ++u) {
            const int j = (u0 + u) * NT + tid;
            if (j < n) fn(key[u0 + u], tok[u0 + u], j);
          }
        }
      }
    } else {
      for (long long j0 = 0; j0 < n; j0 += kEvUnit * NT) {
        int at[kEvUnit], t[kEvUnit];
        float v[kEvUnit];
#pragma unroll
        for (int u = 0; u < kEvUnit; ++u) at[u] = place((int)min(j0 + u * NT + tid, (long long)n - 1));
#pragma unroll
        for (int u = 0; u < kEvUnit; ++u) {
          v[u] = a.c.score[at[u]];
          t[u] = a.c.pos[at[u]];
        }
#pragma unroll
        for (int u = 0; u < kEvUnit; ++u)
          if (j0 + u * NT + tid < n) fn(order_key(v[u]), t[u], (int)(j0 + u * NT + tid));
      }
    }
  };
  // The m-th largest value(key, token) over the rows that cand(key, token)
  // takes; need and have: how many rows with that value are among the m
  // largest, and how many have it.
  uint32_t need = 0, have = 0;
  auto select = [&](uint32_t m, int top, const auto& cand, const auto& value) {
    uint32_t t = 0;
    auto count_digits = [&](uint32_t* hist, int sft, uint32_t prefix, uint32_t pmask) {
      each([&](uint32_t ky, int tk, int) {
        const uint32_t x = value(ky, tk);
        if (cand(ky, tk) && (x & pmask) == prefix) atomicAdd(&hist[(x >> sft) & 255u], 1u);
      });
    };
    radix_select<NT>(count_digits, m, sh, &t, &need, &have, top);
    return t;
  };

  // Held rows: tokens from first_new on and up to last_old.  While no held
  // token has been evicted they are the tokens from seen - r and below s.
  const int k = s.k, r = min(a.recent, k), o = min(a.sink, k - r), m = k - r - o;
  const int age_top = s.seen > (1 << 24) ? 24 : s.seen > (1 << 16) ? 16 : s.seen > (1 << 8) ? 8 : 0;
  int first_new = r > 0 ? s.seen - r : 0x7fffffff, last_old = o - 1;
  {
    uint32_t cn = 0, co = 0;
    each([&](uint32_t, int tk, int) {
      cn += tk >= first_new ? 1u : 0u;
      co += tk <= last_old ? 1u : 0u;
    });
    const uint2 c = block_sum2<NT, REGS>(cn, co, sh);
    auto all = [](uint32_t, int) { return true; };
    if (c.x != (uint32_t)r) first_new = (int)select(r, age_top, all, [](uint32_t, int tk) { return (uint32_t)tk; });
    if (c.y != (uint32_t)o)
      last_old = s.seen - 1 - (int)select(o, age_top, all, [&](uint32_t, int tk) { return (uint32_t)(s.seen - 1 - tk); });
  }
  // The others: keys above `limit`, and those equal to it up to token `tie`.
  uint32_t limit = 0xffffffffu;  // above every key
  int tie = 0x7fffffff;
  if (m > 0) {
    auto other = [&](uint32_t, int tk) { return tk < first_new && tk > last_old; };
    limit = select(m, 24, other, [](uint32_t ky, int) { return ky; });
    // The search may end early, at the lowest key of its digit: every key from
    // there on is kept.
    if (need != have) {
      const uint32_t lim = limit;
      tie = s.seen - 1 -
            (int)select(need, age_top, [&](uint32_t ky, int tk) { return other(ky, tk) && ky == lim; },
                        [&](uint32_t, int tk) { return (uint32_t)(s.seen - 1 - tk); });
    }
  }
  const bool open = tie == 0x7fffffff;
  auto kept = [&](uint32_t ky, int tk) {
    return tk >= first_new || tk <= last_old || (m > 0 && (open ? ky >= limit : ky > limit || (ky == limit && tk <= tie)));
  };
  // List entries, in row order: destination i is the i-th evicted row before
  // k, source i the i-th kept row from k on.
  if constexpr (kRegs) {
    constexpr int NW = NT / kWave;
    uint32_t out = 0, in = 0;  // bit u: row u of this thread is listed
#pragma unroll
    for (int u0 = 0; u0 < REGS; u0 += kEvUnit) {
#pragma unroll
      for (int u = u0; u < u0 + kEvUnit; ++u) {
        const int j = u * NT + tid;
        bool hole = false, mover = false;
        if (u0 * NT < n) {
          const bool kp = kept(key[u], tok[u]);
          hole = j < k && !kp;
          mover = j >= k && j < n && kp;
        }
        const unsigned long long bh = __ballot(hole), bm = __ballot(mover);
        out |= hole ? 1u << u : 0u;
        in |= mover ? 1u << u : 0u;
        if (lane == 0) {
          sh.count[0][u * NW + w] = __popcll(bh);
          sh.count[1][u * NW + w] = __popcll(bm);
        }
      }
    }
    __syncthreads();
    if (w < 2) {  // NT >= 128: one wave a list
      constexpr int per = REGS * NW / kWave;
      int v[per], sum = 0;
#pragma unroll
      for (int i = 0; i < per; ++i) {
        v[i] = sh.count[w][lane * per + i];
        sum += v[i];
      }
      const int incl = wave_incl_scan_i32(sum);
      int before = incl - sum;
#pragma unroll
      for (int i = 0; i < per; ++i) {
        sh.count[w][lane * per + i] = before;
        before += v[i];
      }
      if (lane == kWave - 1) sh.total[w] = incl;
    }
    __syncthreads();
    const int moves = min(sh.total[0], sh.total[1]);  // equal where tokens are distinct
#pragma unroll
    for (int u = 0; u < REGS; ++u) {
      if (u * NT < n) {
        const bool hole = (out >> u) & 1u, mover = (in >> u) & 1u;
        const unsigned long long below = (1ull << lane) - 1ull;
        const int ih = sh.count[0][u * NW + w] + __popcll(__ballot(hole) & below);
        const int im = sh.count[1][u * NW + w] + __popcll(__ballot(mover) & below);
        const int j = u * NT + tid;
        if (hole && ih < moves) a.moves[place(ih)].x = place(j);
        if (mover && im < moves) a.moves[place(im)].y = place(j);
      }
    }
    if (tid == 0) *count = moves;
  } else {
    // Two passes, so that no entry goes past the shorter list.
    long long carry = 0, bound = 0;
    for (int pass = 0; pass < 2; ++pass) {
      carry = 0;
      for (long long j0 = 0; j0 < n; j0 += NT) {
        const long long j = j0 + tid;
        bool hole = false, mover = false;
        int at = 0;
        if (j < n) {
          at = place((int)j);
          const bool kp = kept(order_key(a.c.score[at]), a.c.pos[at]);
          hole = j < k && !kp;
          mover = j >= k && kp;
        }
        long long total;
        const long long x = carry + block_excl_scan<NT>((hole ? 1ll : 0ll) + (mover ? 1ll << 32 : 0ll), sh.scan_tmp, &total);
        if (pass == 1) {
          const int ih = (int)(x & 0xffffffffll), im = (int)(x >> 32);
          if (hole && ih < bound) a.moves[place(ih)].x = at;
          if (mover && im < bound) a.moves[place(im)].y = at;
        }
        carry += total;
      }
      bound = min(carry & 0xffffffffll, carry >> 32);
    }
    if (tid == 0) *count = (int)bound;
  }
}

// Moves of a segment by a block of NT threads, one of `parts` that take turns.
template <int D, int NT>
__device__ inline void move_rows(const PagedEvictArgs& a, const int32_t* table, int h, int moves, int part, int parts) {
  constexpr int LPR = D / 8;        // lanes a row: 16 bytes each
  constexpr int RPB = NT / LPR;     // rows of a block at a time
  constexpr int U = 4;              // times that, loads before the first store
  typedef unsigned u32x4_t __attribute__((ext_vector_type(4)));
  const int shift = a.c.page_shift, mask = (1 << shift) - 1;
  const int sub = threadIdx.x / LPR, piece = threadIdx.x % LPR;
  for (long long i0 = (long long)part * RPB * U; i0 < moves; i0 += (long long)parts * RPB * U) {
    int2 e[U];
    u32x4_t kr[U], vr[U];
    float sc[U];
    int tk[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = (int)min(i0 + u * RPB + sub, (long long)moves - 1);
      e[u] = a.moves[page_row(a.c, table[i >> shift], h) + (i & mask)];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      kr[u] = reinterpret_cast<const u32x4_t*>(a.c.k)[(long long)e[u].y * LPR + piece];
      vr[u] = reinterpret_cast<const u32x4_t*>(a.c.v)[(long long)e[u].y * LPR + piece];
      sc[u] = a.c.score[e[u].y];
      tk[u] = a.c.pos[e[u].y];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i0 + u * RPB + sub < moves) {
        reinterpret_cast<u32x4_t*>(a.c.k)[(long long)e[u].x * LPR + piece] = kr[u];
        reinterpret_cast<u32x4_t*>(a.c.v)[(long long)e[u].x * LPR + piece] = vr[u];
        if (piece == 0) {
          a.c.score[e[u].x] = sc[u];
          a.c.pos[e[u].x] = tk[u];
        }
      }
    }
  }
}

// One block a segment.  D > 0: it moves the rows too (len is left to
// length_kernel: another head's block may still have to read it).
template <int NT, int REGS, int D>
__global__ __launch_bounds__(NT) void select_kernel(PagedEvictArgs a) {
  __shared__ EvShared<NT, REGS> sh;
  __shared__ int moves;
  const int h = blockIdx.x % a.c.HK;
  const EvSeq s = ev_seq(a, blockIdx.x / a.c.HK);
  int32_t* const count = a.count + blockIdx.x;
  bool bad = s.n < 0 || s.n > a.max_kv || s.seen < s.n;
  const int pages = bad ? 0 : (int)(((long long)s.n + (1 << a.c.page_shift) - 1) >> a.c.page_shift);
  for (int i = threadIdx.x; i < pages; i += NT) {
    const int page = s.table[i];
    bad = bad || page < 0 || page >= a.c.num_pages;
    if (i < NT * REGS / 16) sh.pages[i] = page;
  }
  bad = __syncthreads_or(bad);
  if (bad || s.k >= s.n) {
    if (threadIdx.x == 0) {
      if (bad) atomicOr(a.c.dev_status, LETHE_DEV_BAD_LAYOUT);
      *count = kEvictNone;
    }
    return;
  }
  if (s.n <= REGS * NT)
    select_segment<NT, REGS, true>(a, s, h, sh, &moves);
  else
    select_segment<NT, REGS, false>(a, s, h, sh, &moves);
  if (threadIdx.x == 0) *count = moves;
  if constexpr (D > 0) {
    __threadfence_block();
    __syncthreads();
    move_rows<D, NT>(a, s.table, h, moves, 0, 1);
  }
}

// blockIdx.x = segment * parts + part.
template <int D>
__global__ __launch_bounds__(256) void move_kernel(PagedEvictArgs a, int parts) {
  const int seg = blockIdx.x / parts, part = blockIdx.x % parts;
  const int moves = a.count[seg];
  if (moves == kEvictNone) return;
  const int h = seg % a.c.HK, lb = seg / a.c.HK;
  const EvSeq s = ev_seq(a, lb);  // len: written below by one block of the sequence, not used here
  move_rows<D, 256>(a, s.table, h, moves, part, parts);
  if (h == 0 && part == 0 && threadIdx.x == 0) a.c.len[lb] = s.k;
}

__global__ __launch_bounds__(256) void length_kernel(PagedEvictArgs a) {
  const int lb = blockIdx.x * 256 + threadIdx.x;
  if (lb < a.L * a.c.B && a.count[(long long)lb * a.c.HK] != kEvictNone) a.c.len[lb] = ev_seq(a, lb).k;
}

template <int NT, int REGS>
lethe_status launch(const PagedEvictArgs& a, unsigned segs, hipStream_t s) {
  // Blocks that move what they have ranked overlap the two, if they are many
  // (a fifth of 2500 rows going: 2048 segments 246 us against 261 in two
  // launches, 1024 129 against 134, 512 74 both, 128 34 against 28).
  const bool whole = segs >= kEvWhole;
  if (whole) {
    const auto kernel = a.D == 128 ? select_kernel<NT, REGS, 128> : select_kernel<NT, REGS, 64>;
    hipLaunchKernelGGL(kernel, dim3(segs), dim3(NT), 0, s, a);
    if (hipGetLastError() != hipSuccess) return LETHE_ERR_HIP;
    hipLaunchKernelGGL(length_kernel, dim3((a.L * a.c.B + 255) / 256), dim3(256), 0, s, a);
    return hipGetLastError() == hipSuccess ? LETHE_OK : LETHE_ERR_HIP;
  }
  hipLaunchKernelGGL((select_kernel<NT, REGS, 0>), dim3(segs), dim3(NT), 0, s, a);
  if (hipGetLastError() != hipSuccess) return LETHE_ERR_HIP;
  // Enough blocks to fill the chip however few the segments are, but no more
  // than a segment's largest number of moves has use for.
  const long long most = (a.max_kv / 2 + 63) / 64;
  const int parts = (int)std::max(1LL, std::min({most, 4096LL / segs, 1024LL}));
  const auto kernel = a.D == 128 ? move_kernel<128> : move_kernel<64>;
  hipLaunchKernelGGL(kernel, dim3(segs * parts), dim3(256), 0, s, a, parts);
  return hipGetLastError() == hipSuccess ? LETHE_OK : LETHE_ERR_HIP;
}


}  // namespace

lethe_status launch_paged_evict(const PagedEvictArgs& a, hipStream_t s) {
  const long long segs = (long long)a.L * a.c.B * a.c.HK;
  if (segs * 1024 > 0xffffffffLL) return LETHE_ERR_UNSUPPORTED;  // threads of a launch stay below 2^32
  // The fewest threads that hold the rows.
  if (a.max_kv <= 16 * 256) return launch<256, 16>(a, (unsigned)segs, s);
  if (a.max_kv <= 16 * 512) return launch<512, 16>(a, (unsigned)segs, s);
  if (a.max_kv <= 24 * 1024) return launch<1024, 24>(a, (unsigned)segs, s);
  return launch<1024, 32>(a, (unsigned)segs, s);
}

}  // namespace lethe
