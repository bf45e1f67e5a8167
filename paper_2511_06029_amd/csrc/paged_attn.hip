// Causal attention of a batch's newest rows over a paged cache, with the
// importance update of Eq. 5 / Eq. 2, gfx950.
//
// The q_len queries of a sequence and the G query heads of a KV group are the
// columns of one product: column c is query c / G, head c % G, so a group's
// keys and values are read once for all of them whatever G and q_len are.
//
// Up to 16 columns (one query, or a few), bound by the rows' bytes:
//  1. decode_kernel: the rows of every (sequence, KV head) cut into chunks of
//     like length, one block each; a wavefront takes 32 rows at a time on
//     16x16x32 products.  Writes a chunk's (max, sum, output) and, for the
//     scores, the rows' logits.
//  2. finish_kernel: joins a segment's chunks and turns the logits into
//     weights once the segment's max and sum are known.
//  128 users over 200 to 12000 rows, 8 KV heads, 1.54 GB: 289 + 28 us, 4.8 TB/s
//  (256 us without scores, 6.0 TB/s; a read stream reaches 6.2).
//
// More columns, bound by the products (sequences with few decode beside them):
//  1. plan_kernel (one block): cuts every (sequence, 128 columns) into key
//     ranges of like work and orders them, longest first.
//  2. tile_kernel: flash attention forward of 128 columns over a key range,
//     32 columns a wavefront on 32x32x16 products, keys and values shared by
//     the block's four wavefronts through LDS.
//  3. join_kernel: where a tile's keys were cut.
//  4. seed_kernel (with scores): key-major second pass, the columns' final
//     max and sum at hand, in a fixed order without atomics.
//  Eight prompts of 2048 rows, 32 query heads: 9 + 366 + 5 + 217 us, the tiles
//  at 0.76 PFLOP/s; over 32768 rows 1.04 (0.86 capped; a large library product
//  reaches 1.2).
#include <algorithm>

#include "paged_internal.h"
#include "paged_mma.h"

namespace lethe {

namespace {

constexpr int kThreads = 256;
constexpr int kNumWaves = kThreads / kWave;
constexpr float kNegBig = -1.0e30f;

// Sizes of sequence b as this call sees them; ok: they fit together.
struct AttnSeq {
  int n, ql;
  long long q0;
  bool ok;
};

__device__ inline AttnSeq attn_seq(const PagedAttnArgs& a, int b) {
  AttnSeq s;
  s.n = a.c.len[b];
  s.ql = a.q_len[b];
  s.q0 = a.q_start[b];
  s.ok = s.n >= 0 && s.n <= a.max_kv && s.ql >= 0 && s.ql <= s.n && s.ql <= a.max_q && s.q0 >= 0 &&
         s.q0 + s.ql <= a.q_rows;
  return s;
}

// Rows are addressed in granules of 16, which lie in one page whatever its
// size: pool row of granule `g` (its rows 16 g ..), or -1 (flagged) where the
// page is out of range.
__device__ inline int granule_row(const PagedView& c, int b, int h, int g) {
  const int row = 16 * g;
  const int page = c.table[(long long)b * c.max_pages + (row >> c.page_shift)];
  if (page < 0 || page >= c.num_pages) {
    atomicOr(c.dev_status, LETHE_DEV_BAD_LAYOUT);
    return -1;
  }
  return page_row(c, page, h) + (row & ((1 << c.page_shift) - 1));
}

// Base-2 logits are A v + B of a value v of the raw product x: x itself
// (A = scale, B = 0), or, capped, 1 / (1 + exp(2 x / cap)), which falls as x
// grows: cap tanh(x / cap) = cap - 2 cap v.
template <bool kCap>
struct Logit {
  float A, B, cap_in;
  __device__ inline explicit Logit(const PagedAttnArgs& a)
      : A(kCap ? -2.0f * a.cap_log2 : a.scale_log2), B(kCap ? a.cap_log2 : 0.0f), cap_in(a.cap_in) {}
  __device__ inline float value(float x) const {
    return kCap ? __builtin_amdgcn_rcpf(1.0f + hw_exp2(x * cap_in)) : x;
  }
  // The value of a masked logit, and the value of the larger logit.
  static constexpr float kMasked = kCap ? INFINITY : -INFINITY;
  static __device__ inline float larger(float u, float v) { return kCap ? fminf(u, v) : fmaxf(u, v); }
  __device__ inline float logit(float v) const { return kCap ? fmaf(A, v, B) : A * v; }
  // exp2(logit(v) - m) from shift = B - m.
  __device__ inline float weight(float v, float shift) const { return hw_exp2(fmaf(A, v, shift)); }
};

// Query of column c, c / G (columns stay below 2^28: exact).
__device__ inline int query_of(const PagedAttnArgs& a, int c) { return a.G == 1 ? c : (int)__umulhi((unsigned)c, a.g_magic); }

__device__ inline float max_halves(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// 16 bytes a lane from `base + off` into LDS: lane l's land at dst + 16 l.
__device__ inline void load_lds(const char* p, lds_char* dst) {
  __builtin_amdgcn_global_load_lds((global_cvoid*)p, (lds_void*)dst, 16, 0, 0);
}

// The same for bytes that nothing else of the launch reads: they leave L2 early.
__device__ inline void load_lds_nt(const char* p, lds_char* dst) {
  __builtin_amdgcn_global_load_lds((global_cvoid*)p, (lds_void*)dst, 16, 0, 2);
}

// Waits until at most N vector-memory operations are on their way (expcnt and
// lgkmcnt left free).
template <int N>
__device__ inline void wait_vmem_but() {
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14));
}
__device__ inline void wait_vmem() { wait_vmem_but<0>(); }

// A barrier without __syncthreads' wait for every load on its way: LDS reads
// are done, and of the loads those that the caller has waited for.
__device__ inline void barrier_only() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// ---------------------------------------------------------------------------
// Few columns
// ---------------------------------------------------------------------------
constexpr int kFewCols = 16;
__device__ inline bool few_cols(const PagedAttnArgs& a, int ql) { return ql > 0 && ql <= kFewCols / a.G; }
// Columns that a call's partials and logits have room for.
__host__ __device__ inline int room_cols(int max_q, int G) { return max_q > kFewCols / G ? kFewCols / G * G : max_q * G; }
constexpr int kDecStep = 32;        // rows a wavefront takes at a time
constexpr int kDecMaxChunks = 64;   // of a segment
constexpr int kDecChunkSteps = 14;  // steps of a chunk, where there are enough
constexpr int kDecLeastSteps = 4;   // one a wavefront
constexpr int kDecMinBlocks = 512, kDecMaxBlocks = 4096;
constexpr int kFinUnit = 4 * kThreads;  // rows that a finishing block takes at a time, four a thread
constexpr long long kFinBlocks = 4096;  // about as many finishing blocks as there should be

__host__ __device__ inline long long dec_blocks(long long steps) {
  const long long nb = steps / kDecChunkSteps;
  return nb < kDecMinBlocks ? kDecMinBlocks : nb > kDecMaxBlocks ? kDecMaxBlocks : nb;
}
// Steps of a chunk, of `all` steps over the call's segments, and chunks of a
// segment.
__host__ __device__ inline int dec_chunk_steps(long long all) {
  const long long per = (all + dec_blocks(all) - 1) / dec_blocks(all);
  return (int)(per < kDecLeastSteps ? kDecLeastSteps : per);
}
__host__ __device__ inline int dec_chunks(int steps, int per) {
  const int nch = (steps + per - 1) / per;
  return nch < kDecMaxChunks ? nch : kDecMaxChunks;
}
// Floats of a chunk's partial: (max, sum) and output of every column.
__host__ __device__ inline int dec_part(int cols, int D) { return (cols * (D + 2) + 31) / 32 * 32; }

struct DecChunk {
  int b, h, c, nch, n, ql;
  int first;               // block index of the segment's chunk 0
  long long row0;          // rows of the segments before it, rounded up to steps: its logits start at row0 room_cols
  long long q0;
};

// The chunk that block `idx` works on.  Every wave derives the same map: 64
// sequences at a time, lane l holding sequence 64 r + l.  seg >= 0 asks for
// chunk 0 of that segment (b HK + h) instead.
template <int R>
__device__ inline bool dec_chunk(const PagedAttnArgs& a, int idx, int seg, DecChunk& ck) {
  const int lane = threadIdx.x & (kWave - 1);
  int steps[R], rows[R], queries[R];
  int total = 0;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int b = kWave * r + lane;
    steps[r] = rows[r] = queries[r] = 0;
    if (b < a.c.B) {
      const AttnSeq s = attn_seq(a, b);
      if (s.ok && few_cols(a, s.ql)) {
        queries[r] = s.ql;
        rows[r] = s.n;
        steps[r] = (s.n + kDecStep - 1) / kDecStep;
      } else if (!s.ok && blockIdx.x == 0 && threadIdx.x < kWave) {
        atomicOr(a.c.dev_status, LETHE_DEV_BAD_LAYOUT);
      }
    }
    total += steps[r];
  }
  for (int o = kWave / 2; o > 0; o >>= 1) total += __shfl_xor(total, o);
  const int per = dec_chunk_steps((long long)total * a.c.HK);
  int blocks0 = 0;
  long long steps0 = 0;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int nch = dec_chunks(steps[r], per);
    const int incl = wave_incl_scan_i32(nch * a.c.HK);
    const int sincl = wave_incl_scan_i32(steps[r]);
    const int sum = __builtin_amdgcn_readlane(incl, kWave - 1);
    const bool mine = seg >= 0 ? seg / a.c.HK / kWave == r : idx < blocks0 + sum;
    if (mine) {
      const int l = seg >= 0 ? seg / a.c.HK % kWave : (int)__builtin_ctzll(__ballot(blocks0 + incl > idx));
      ck.b = kWave * r + l;
      ck.nch = __builtin_amdgcn_readlane(nch, l);
      ck.n = __builtin_amdgcn_readlane(rows[r], l);
      ck.ql = __builtin_amdgcn_readlane(queries[r], l);
      const int st = __builtin_amdgcn_readlane(steps[r], l);
      if (ck.nch == 0) return false;
      const int at = blocks0 + __builtin_amdgcn_readlane(incl, l) - ck.nch * a.c.HK;
      ck.h = seg >= 0 ? seg % a.c.HK : (idx - at) / ck.nch;
      ck.c = seg >= 0 ? 0 : (idx - at) % ck.nch;
      ck.first = at + ck.h * ck.nch;
      ck.row0 = ((steps0 + __builtin_amdgcn_readlane(sincl, l) - st) * a.c.HK + (long long)ck.h * st) * kDecStep;
      ck.q0 = a.q_start[ck.b];
      return true;
    }
    blocks0 += sum;
    steps0 += __builtin_amdgcn_readlane(sincl, kWave - 1);
  }
  return false;
}

template <int D>
struct DecCfg {
  static constexpr int KK = D / 32;          // k-steps of 32 over the head dim
  static constexpr int NT = D / 16;          // output tiles of 16 dims
  static constexpr int ROWB = D * 2;
  static constexpr int LPR = ROWB / 16;      // lanes a row for V loads
  static constexpr int VLOADS = kDecStep * LPR / kWave;
  // V load u carries rows u + VLOADS j into block u; the blocks' padding
  // spreads the rows of one transposing read over the LDS banks.
  static constexpr int VBLK = kWave * 16 + 32;
  static constexpr int VTILE = VLOADS * VBLK;
  static __device__ constexpr int vaddr(int r, int c) { return (r % VLOADS) * VBLK + (r / VLOADS) * ROWB + c; }
};

struct DecWs {
  float* part;
  float* logit;
  long long logit_rows;
};
// Whether the workspace has room for the segment's logits: always, unless
// tables share pages, which a call that updates scores does not allow.
__device__ inline bool dec_room(const DecWs& ws, const DecChunk& ck) {
  return ck.row0 + (ck.n + kDecStep - 1) / kDecStep * kDecStep <= ws.logit_rows;
}

// One chunk by a block of kThreads; its partial goes to slot `slot`.  tile(w):
// LDS of wave w, DecCfg::VTILE bytes.  kOne: sequences have one query, which
// attends every row (the masks of several cost registers that the loop spills).
template <typename T, int D, bool kCap, bool kOne, class Tile>
__device__ inline void decode_chunk(const PagedAttnArgs& a, const DecWs& ws, const DecChunk& ck, long long slot,
                                    const Tile& tile, float2 (&wave_ml)[kNumWaves][kFewCols]) {
  using Cfg = DecCfg<D>;
  using M = Mma<T>;
  constexpr int KK = Cfg::KK, NT = Cfg::NT, ROWB = Cfg::ROWB, LPR = Cfg::LPR, VLOADS = Cfg::VLOADS;
  const int tid = threadIdx.x;
  const int lane = tid & (kWave - 1);
  const int w = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int g4 = lane >> 4, s = lane & 15;
  const int n = ck.n, cols = kOne ? a.G : ck.ql * a.G;
  const int full = n - ck.ql;                 // rows up to it are attended by every column
  const int query = kOne ? 0 : query_of(a, s);
  const int lim = full + query;               // last row of column s
  const int steps = (n + kDecStep - 1) / kDecStep;
  const int first = (int)((long long)steps * ck.c / ck.nch), end = (int)((long long)steps * (ck.c + 1) / ck.nch);
  lds_char* const vb = (lds_char*)tile(w);

  // Queries as the B operand of S^T = K Q^T: lane (g4, s) holds
  // Q[column s][dims 32 kk + 8 g4 ..], columns past the last zero.
  typename M::x8 qb[KK];
  {
    const char* q = (const char*)a.q + ((ck.q0 + query) * a.c.HQ + ck.h * a.G + s - query * a.G) * (long long)ROWB;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
      qb[kk] = s < cols ? *reinterpret_cast<const typename M::x8*>(q + 64 * kk + 16 * g4) : mma_zero<T>();
  }

  // Granules of this wave's next 32 steps, two a step: lane 2 i + g holds
  // granule g of its i-th step from `base`.
  int ids = -1;
  bool bad = false;
  auto load_ids = [&](int step) {
    const int st = step + kNumWaves * (lane >> 1);
    const int g = min(2 * st + (lane & 1), (n - 1) >> 4);
    ids = granule_row(a.c, ck.b, ck.h, g);
    bad = __any(ids < 0);
  };
  typename M::x8 kr[2][KK];
  int g0 = 0, g1 = 0;
  auto granules = [&](int i) {
    g0 = __builtin_amdgcn_readlane(ids, 2 * i);
    g1 = __builtin_amdgcn_readlane(ids, 2 * i + 1);
  };
  // Rows past the last one read that one instead; a granule out of range
  // reads the pool's first rows.  Whole steps take two addresses for K (the
  // granules', the same for every lane) and one for V.
  auto row_of = [&](int base, int r) {
    r = min(r, n - 1 - base);
    return (long long)(max(r < 16 ? g0 : g1, 0) + (r & 15)) * ROWB;
  };
  auto load_k = [&](int base) {
    if (base + kDecStep <= n) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const char* p = a.c.k + (long long)max(t ? g1 : g0, 0) * ROWB;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk)
          kr[t][kk] = *reinterpret_cast<const typename M::x8*>(p + (unsigned)(s * ROWB + 16 * g4) + 64 * kk);
      }
    } else {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const char* p = a.c.k + row_of(base, 16 * t + s) + 16 * g4;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) kr[t][kk] = *reinterpret_cast<const typename M::x8*>(p + 64 * kk);
      }
    }
  };
  const int vrow = VLOADS * (lane / LPR);  // + u for load u; lanes of the upper half have granule 1
  auto load_v = [&](int base) {
    if (base + kDecStep <= n) {
      const char* p = a.c.v + (long long)(max(lane < kWave / 2 ? g0 : g1, 0) + (vrow & 15)) * ROWB + 16 * (lane % LPR);
#pragma unroll
      for (int u = 0; u < VLOADS; ++u) load_lds_nt(p + u * ROWB, vb + u * Cfg::VBLK);
    } else {
#pragma unroll
      for (int u = 0; u < VLOADS; ++u)
        load_lds(a.c.v + row_of(base, u + vrow) + 16 * (lane % LPR), vb + u * Cfg::VBLK);
    }
  };

  float m = kNegBig, l = 0.0f;
  mma_f32x4_t o[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) o[nt] = mma_f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  const Logit<kCap> lg(a);
  // Logits, [step][column][row of the step]: a step's lie side by side.
  float* const logit = a.gamma > 0.0f && dec_room(ws, ck) && s < cols
                           ? ws.logit + ck.row0 * room_cols(a.max_q, a.G) + s * kDecStep + 4 * g4
                           : nullptr;

  int step = first + w, i = 0;
  if (step < end) {
    load_ids(step);
    granules(0);
    load_k(step * kDecStep);
    load_v(step * kDecStep);
  }
  while (step < end) {
    const int base = step * kDecStep;
    const int next = step + kNumWaves;
    const bool b0 = bad && g0 < 0, b1 = bad && g1 < 0;  // of this step
    // Rows of the step that take no part (wave-uniform).
    uint32_t dead = (n - base < kDecStep ? ~0u << (n - base) : 0u) | (b0 ? 0xffffu : 0u) | (b1 ? 0xffff0000u : 0u);
    mma_f32x4_t x[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      x[t] = mma_f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) x[t] = M::mma16(kr[t][kk], qb[kk], x[t]);
    }
    if (next < end) {
      if (++i == kWave / 2) {
        load_ids(next);
        i = 0;
      }
      granules(i);
      load_k(next * kDecStep);
    }
    // Logits of rows base + 16 t + 4 g4 + r for column s.
    const bool edge = !kOne && base + kDecStep - 1 > full;  // some columns do not attend some rows
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        x[t][r] = lg.logit(lg.value(x[t][r]));
        if (dead && ((dead >> (16 * t + 4 * g4 + r)) & 1u)) x[t][r] = -INFINITY;
        if (edge && base + 16 * t + 4 * g4 + r > lim) x[t][r] = -INFINITY;
      }
    if (logit) {
#pragma unroll
      for (int t = 0; t < 2; ++t) *reinterpret_cast<mma_f32x4_t*>(logit + (long long)base * cols + 16 * t) = x[t];
    }
    float mx = fmaxf(fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[0][2], x[0][3])),
                     fmaxf(fmaxf(x[1][0], x[1][1]), fmaxf(x[1][2], x[1][3])));
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    const float mnew = fmaxf(m, mx);
    const float corr = hw_exp2(m - mnew);
    m = mnew;
    float psum = 0.0f;
    typename M::x8 p;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float e = hw_exp2(x[j >> 2][j & 3] - mnew);
      psum += e;
      p[j] = (T)e;
    }
    l = l * corr + psum;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) o[nt] *= corr;
    // V^T operand through the transposing LDS read: lane s of group g4 points
    // at row 4 g4 + s / 4 (and 16 more), column 16 nt + 4 (s % 4); its slots
    // j < 4 are rows 4 g4 + j, the others 16 + 4 g4 + j - 4, as p's.
    const int rsub = 4 * g4 + (s >> 2);
    auto operand = [&](int nt) {
      const int col = (16 * nt + 4 * (s & 3)) * 2;
      const typename M::x4 a0 = M::read_tr(vb + Cfg::vaddr(rsub, col)), a1 = M::read_tr(vb + Cfg::vaddr(rsub + 16, col));
      return __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    uint32_t apart = 0;
    if (edge && full + 1 < n) {
      // Rows that only some columns attend stay out of the products where they
      // hold an infinity or NaN, and are added one by one.
      const int r0 = max(full + 1 - base, 0), r1 = min(n - base, kDecStep);
      for (int x0 = r0 * LPR; x0 < r1 * LPR; x0 += kWave) {
        const int i = min(x0 + lane, r1 * LPR - 1);
        const uint4 v = *reinterpret_cast<const uint4*>(tile(w) + Cfg::vaddr(i / LPR, 16 * (i % LPR)));
        unsigned long long hit = __ballot(M::odd(v));
        while (hit) {  // rare
          apart |= 1u << (min(x0 + (int)__builtin_ctzll(hit), r1 * LPR - 1) / LPR);
          hit &= hit - 1;
        }
      }
      apart &= ~dead;
      dead |= apart;
    }
    if (!dead) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) o[nt] = M::mma16(operand(nt), p, o[nt]);
    } else {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        typename M::x8 av = operand(nt);
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if ((dead >> (16 * (j >> 2) + 4 * g4 + (j & 3))) & 1u) av[j] = (T)0.0f;
        o[nt] = M::mma16(av, p, o[nt]);
      }
      if (apart) {
#pragma unroll 1
        while (apart) {
          const int r = (int)__builtin_ctz(apart);
          apart &= apart - 1;
          float mine = 0.0f;  // an index would put p in scratch memory
#pragma unroll
          for (int j = 0; j < 8; ++j) mine = j == 4 * (r >> 4) + (r & 3) ? (float)p[j] : mine;
          const float pr = __shfl(mine, 16 * ((r >> 2) & 3) + s);
          if (base + r <= lim) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int x = 0; x < 4; ++x)
                o[nt][x] = fmaf(pr, (float)*reinterpret_cast<const T*>(tile(w) + Cfg::vaddr(r, 2 * (16 * nt + 4 * g4 + x))),
                                o[nt][x]);
          }
        }
      }
    }
    if (next < end) {
      // The tile's reads are done (their results are in the products above).
      __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
      load_v(next * kDecStep);
    }
    step = next;
  }

  // Lane groups hold different rows of the same columns.
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  // The waves' parts of the chunk, joined in LDS: outputs transposed through
  // this wave's own V tile, [column][dim].
  if (g4 == 0 && s < cols) wave_ml[w][s] = make_float2(m, l);
  static_assert(Cfg::VTILE >= kFewCols * D * 4, "a wave's outputs fit its V tile");
  wait_vmem();
  __builtin_amdgcn_s_waitcnt(0xc07f);
  if (s < cols) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
      *(__attribute__((address_space(3))) mma_f32x4_t*)(vb + (s * D + 16 * nt + 4 * g4) * 4) = o[nt];
  }
  __syncthreads();
  float* const part = ws.part + slot * dec_part(room_cols(a.max_q, a.G), D);
  for (int x = tid; x < cols * D; x += kThreads) {
    const int c = x / D;
    float mm = wave_ml[0][c].x;
#pragma unroll
    for (int v = 1; v < kNumWaves; ++v) mm = fmaxf(mm, wave_ml[v][c].x);
    float sum = 0.0f, lsum = 0.0f;
#pragma unroll
    for (int v = 0; v < kNumWaves; ++v) {
      const float f = hw_exp2(wave_ml[v][c].x - mm);
      sum = fmaf(f, *reinterpret_cast<const float*>(tile(v) + x * 4), sum);
      lsum = fmaf(f, wave_ml[v][c].y, lsum);
    }
    part[2 * cols + x] = sum;
    if (x % D == 0) *reinterpret_cast<float2*>(part + 2 * c) = make_float2(mm, lsum);
  }
}

template <typename T, int D, bool kCap, int R, bool kOne>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(kOne ? 3 : 2))) void decode_kernel(PagedAttnArgs a, DecWs ws) {
  __shared__ __attribute__((aligned(16))) char vtiles[kNumWaves * DecCfg<D>::VTILE];
  __shared__ float2 wave_ml[kNumWaves][kFewCols];
  DecChunk ck;
  if (!dec_chunk<R>(a, blockIdx.x, -1, ck)) return;
  decode_chunk<T, D, kCap, kOne>(a, ws, ck, blockIdx.x, [&](int w) { return vtiles + w * DecCfg<D>::VTILE; }, wave_ml);
}

// What is left of a segment with few columns: y = 0: its output, y > 0: the
// scores of its rows from (y - 1) span on.  Every block joins the chunks'
// statistics.
template <typename T, int D, int R>
__device__ inline void finish_segment(const PagedAttnArgs& a, const DecWs& ws, int span, int seg, long long y) {
  __shared__ float factor[kFewCols][kDecMaxChunks];  // what a chunk's output counts
  __shared__ float2 stat[kFewCols];                  // max, 1 / sum
  const int tid = threadIdx.x, lane = tid & (kWave - 1), w = tid / kWave;
  DecChunk ck;
  if (!dec_chunk<R>(a, -1, seg, ck)) return;
  const long long r0 = (y - 1) * span;
  if (y > 0 && r0 >= ck.n) return;
  const int cols = ck.ql * a.G, room = room_cols(a.max_q, a.G), pstride = dec_part(room, D);
  const float* const part = ws.part + (long long)ck.first * pstride;
  for (int c = w; c < cols; c += kNumWaves) {
    const float2 ml = lane < ck.nch ? *reinterpret_cast<const float2*>(part + (long long)lane * pstride + 2 * c)
                                    : make_float2(kNegBig, 0.0f);
    const float mm = wave_max(ml.x);
    const float f = hw_exp2(ml.x - mm);
    const float sum = wave_sum(f * ml.y);
    const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;  // no row at all: 0
    factor[c][lane] = f * inv;
    if (lane == 0) stat[c] = make_float2(mm, inv);
  }
  __syncthreads();
  if (y == 0) {
    for (int x = tid; x < cols * D; x += kThreads) {
      const int c = x / D, query = query_of(a, c);
      const float* const po = part + 2 * cols + x;
      float sum = 0.0f;
      for (int i0 = 0; i0 < ck.nch; i0 += 8) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = po[(long long)min(i0 + i, ck.nch - 1) * pstride];
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fmaf(i0 + i < ck.nch ? factor[c][i0 + i] : 0.0f, v[i], sum);
      }
      ((T*)a.out)[((ck.q0 + query) * a.c.HQ + ck.h * a.G + c - query * a.G) * D + x % D] = (T)sum;
    }
    return;
  }
  if (!dec_room(ws, ck)) {
    if (tid == 0) atomicOr(a.c.dev_status, LETHE_DEV_BAD_LAYOUT);
    return;
  }
  const float* const logit = ws.logit + ck.row0 * room;
  const int mask = (1 << a.c.page_shift) - 1;
  const int end = (int)min(r0 + span, (long long)ck.n);
  // Four rows a thread: their scores lie side by side (a page holds whole
  // granules of 16).
  for (int r = (int)r0 + 4 * tid; r < end; r += kFinUnit) {
    const int page = a.c.table[(long long)ck.b * a.c.max_pages + (r >> a.c.page_shift)];
    const float* const xr = logit + (long long)(r / kDecStep) * cols * kDecStep + r % kDecStep;
    mma_f32x4_t sum = mma_f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    for (int c0 = 0; c0 < cols; c0 += 8) {
      mma_f32x4_t x[8];
#pragma unroll
      for (int c = 0; c < 8; ++c)
        if (c0 + c < cols) x[c] = *reinterpret_cast<const mma_f32x4_t*>(xr + (c0 + c) * kDecStep);
#pragma unroll
      for (int c = 0; c < 8; ++c)
        if (c0 + c < cols) {
#pragma unroll
          for (int i = 0; i < 4; ++i) sum[i] = fmaf(hw_exp2(x[c][i] - stat[c0 + c].x), stat[c0 + c].y, sum[i]);
        }
    }
    if (page < 0 || page >= a.c.num_pages) continue;
    float* const sp = a.c.score + page_row(a.c, page, ck.h) + (r & mask);
    if (r + 4 <= end) {
      mma_f32x4_t old = *reinterpret_cast<const mma_f32x4_t*>(sp);
#pragma unroll
      for (int i = 0; i < 4; ++i) old[i] = fmaf(a.gamma, old[i], sum[i]);
      *reinterpret_cast<mma_f32x4_t*>(sp) = old;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (r + i < end) sp[i] = fmaf(a.gamma, sp[i], sum[i]);
    }
  }
}

template <typename T, int D, int R>
__global__ __launch_bounds__(kThreads) void finish_kernel(PagedAttnArgs a, DecWs ws, int span) {
  finish_segment<T, D, R>(a, ws, span, blockIdx.x, blockIdx.y);
}

// ---------------------------------------------------------------------------
// More columns
// ---------------------------------------------------------------------------
constexpr int kTileWaves = 4;     // of a block, 32 columns each
constexpr int kTileThreads = kWave * kTileWaves;
constexpr int kTileCols = 32 * kTileWaves;
constexpr int kKeyStep = 64;      // keys of a step
// Keys of a range at least: 3 sequences of 80 queries over 1200 rows take 25.5 us,
// 29.7 with 512 and 23.6 with 128; 66 of 9 over 370 62.6 and 65.4 with 128.
constexpr int kLeastKeys = 256;
constexpr int kChip = 256;        // CUs
constexpr int kLongRange = 2048;  // keys from which on two blocks a CU are aimed at
constexpr int kMaxSplit = 64;     // ranges of a tile
constexpr int kJoinCols = 16;     // columns of a joining block
constexpr float kLag = 8.0f;      // of a running maximum, base 2
constexpr int kBuckets = 1024;    // of the lists' order, by length

struct PlanHead {
  int items, splits, seeds;  // entries of the lists
  int wide;                  // seed blocks of kSeedWide keys instead of kSeedNarrow
};
// Keys of a seeding block; below this many wide ones, one a CU, the narrow ones
// are used (2048 queries over 8192 rows, 256 wide blocks: 427 us, 469 narrow; two
// prompts of 250 to 500 queries beside 30 decoding users, 130: 122 narrow, 134
// wide).
constexpr int kSeedWide = 256, kSeedNarrow = 64, kSeedFill = 256;
constexpr int kSeedGrid = 2048;  // seeding blocks launched, at most
// One tile and key range, or (splits) one tile with several ranges, or one
// chunk of a sequence with few columns.  An entry has its sequence's sizes, so
// that the block that takes it waits for one read before those of its rows.
constexpr int kNoTile = -1, kChunkItem = -2;
struct alignas(16) PlanItem {
  int b, tile;
  int range;   // in the split list, how many; of a chunk, its number and, from bit 8 on, how many the segment has
  int slot;    // of its partial, -1: the only range; of a chunk, the chunks of one head before the sequence
  int steps0;  // of a chunk, the steps of one head before the sequence
  int keys;    // of a range
  int n, ql;
  long long q0;
};
struct alignas(16) PlanSeed {
  int b, block;  // of seed keys
  int n, ql;
  long long q0;
};

struct TileWs {
  PlanHead* head;
  PlanItem* items;
  PlanItem* splits;
  PlanSeed* seeds;
  float2* stat;      // [q_rows][HQ] max (base 2), 1 / sum
  float2* part_ml;   // [slots][HK][kTileCols]
  float* part_o;     // [slots][HK][kTileCols][D]
  int max_items, max_slots, max_seeds;
};

__device__ inline int tile_count(int cols) { return (cols + kTileCols - 1) / kTileCols; }
// One past the last key that columns up to `last` attend.
__device__ inline int key_end(const AttnSeq& s, int last, int G) { return s.n - s.ql + min(last / G, s.ql - 1) + 1; }

// Exclusive prefix sums of K values a thread and their totals, over a block of
// NT threads.
template <int K, int NT>
__device__ inline void scan_all(int (&v)[K], int (&total)[K], int (&tmp)[8][NT / kWave]) {
  const int lane = threadIdx.x & (kWave - 1), w = threadIdx.x / kWave;
  int own[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    own[k] = v[k];
    v[k] = wave_incl_scan_i32(v[k]);
    if (lane == kWave - 1) tmp[k][w] = v[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < K; ++k) {
    int before = 0, all = 0;
#pragma unroll
    for (int i = 0; i < NT / kWave; ++i) {
      const int x = tmp[k][i];
      before += i < w ? x : 0;
      all += x;
    }
    total[k] = all;
    v[k] += before - own[k];
  }
  __syncthreads();
}

// Sum of a float over the block, the same for every thread.
template <int NT>
__device__ inline float sum_all(float v, float (&tmp)[NT / kWave]) {
  v = group_sum<kWave>(v);
  if ((threadIdx.x & (kWave - 1)) == 0) tmp[threadIdx.x / kWave] = v;
  __syncthreads();
  float all = 0.0f;
#pragma unroll
  for (int i = 0; i < NT / kWave; ++i) all += tmp[i];
  __syncthreads();
  return all;
}

// NT threads, one a sequence at least: 256 where they are enough (4 chunks of 40
// to 100 queries 31.7 us, 33.5 with 1024, whose waves each read every wave's
// partial sums).
template <int NT>
__global__ __launch_bounds__(NT) void plan_kernel(PagedAttnArgs a, TileWs ws) {
  __shared__ int scan_tmp[8][NT / kWave];
  __shared__ float sum_tmp[NT / kWave];
  // By sequence: rows and queries, first entry of its in the three lists,
  // first partial, steps before it (few columns), keys of a range.
  __shared__ int rows_of[NT], queries_of[NT], item0[NT], split0[NT];
  __shared__ int seed0[NT], slot0[NT], steps0[NT], keys_of[NT];
  __shared__ long long query0[NT];
  __shared__ int hist[kBuckets];
  const int tid = threadIdx.x;
  AttnSeq s{0, 0, 0, true};
  if (tid < a.c.B) s = attn_seq(a, tid);
  if (!s.ok) {
    atomicOr(a.c.dev_status, LETHE_DEV_BAD_LAYOUT);
    s.n = s.ql = 0;
  }
  rows_of[tid] = s.n;
  queries_of[tid] = s.ql;
  query0[tid] = s.q0;
  const bool few = few_cols(a, s.ql), many = s.ql > 0 && !few;
  const int tiles = many ? tile_count(s.ql * a.G) : 0;
  const int steps = few ? (s.n + kDecStep - 1) / kDecStep : 0;
  const int wide_seeds = many ? (s.n + kSeedWide - 1) / kSeedWide : 0;
  int v1[2] = {steps, wide_seeds}, t1[2];
  scan_all<2, NT>(v1, t1, scan_tmp);
  steps0[tid] = v1[0];
  const int chunks = dec_chunks(steps, dec_chunk_steps((long long)t1[0] * a.c.HK));
  const float work = sum_all<NT>((float)tiles * (float)s.n, sum_tmp) * (float)a.c.HK;
  // Ranges of like length: two blocks a CU, if the ranges are long (512 queries
  // over 32768 rows: 307 us against 370 with one); else one, for a tile that is
  // not cut needs no joining (two prompts of 500 queries over 1700 rows beside
  // 30 decoding users: 131 us against 156 with two).
  const float want = fmaxf(fmaxf((float)kLeastKeys, work / (2.0f * kChip)), fminf(work / kChip, (float)kLongRange));
  const int ranges = max(1, min(kMaxSplit, (int)((float)s.n / want + 0.5f)));
  const int keys = (int)((((long long)s.n + ranges - 1) / ranges + kKeyStep - 1) / kKeyStep * kKeyStep);
  keys_of[tid] = keys;
  const bool wide = (long long)t1[1] * a.c.HK >= kSeedFill;
  const int seed_keys = wide ? kSeedWide : kSeedNarrow;
  const int seed_blocks = !(a.gamma > 0.0f) || !many ? 0 : (s.n + seed_keys - 1) / seed_keys;
  int v2[5] = {tiles * ranges + chunks, ranges > 1 ? tiles : 0, ranges > 1 ? tiles * ranges : 0, chunks, seed_blocks}, t2[5];
  scan_all<5, NT>(v2, t2, scan_tmp);
  const float count = sum_all<NT>((float)tiles * (float)ranges + (float)chunks, sum_tmp);  // also where t2[0] would not hold it
  item0[tid] = v2[0];
  split0[tid] = v2[1];
  slot0[tid] = chunks ? v2[3] : v2[2];
  seed0[tid] = v2[4];
  // More work than the bounds allow: rows of q that belong to two sequences.
  const bool over = count > 1.5e9f || t2[0] > ws.max_items || t2[2] > ws.max_slots || t2[4] > ws.max_seeds;
  const int items = over ? 0 : t2[0], seeds = over ? 0 : t2[4];
  if (tid == 0) {
    if (over) atomicOr(a.c.dev_status, LETHE_DEV_BAD_LAYOUT);
    *ws.head = PlanHead{items, over ? 0 : t2[1], seeds, wide ? 1 : 0};
  }
  __syncthreads();
  // The sequence that entry i of a list belongs to (empty ones share a start).
  auto sequence = [&](const int (&first)[NT], int i) {
    int lo = 0, hi = a.c.B;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (first[mid] <= i)
        lo = mid;
      else
        hi = mid;
    }
    return lo;
  };
  // Item i and the keys it works on.
  auto item = [&](int i, PlanItem& it) {
    const int b = sequence(item0, i);
    const int n = rows_of[b], ql = queries_of[b];
    const int mine = (b + 1 < NT ? item0[b + 1] : items) - item0[b];
    it.b = b;
    it.n = n;
    it.ql = ql;
    it.q0 = query0[b];
    it.keys = keys_of[b];
    if (few_cols(a, ql)) {
      it.tile = kChunkItem;
      it.range = (i - item0[b]) | mine << 8;
      it.slot = slot0[b];
      it.steps0 = steps0[b];
      return max(n / mine, 1);
    }
    const int per = it.keys;
    const int nr = mine / tile_count(ql * a.G);
    it.steps0 = 0;
    it.tile = (i - item0[b]) / nr;
    it.range = (i - item0[b]) % nr;
    it.slot = nr > 1 ? slot0[b] + i - item0[b] : -1;
    const int end = key_end(AttnSeq{n, ql, 0, true}, kTileCols * it.tile + kTileCols - 1, a.G);
    const long long from = (long long)it.range * per;
    if (it.range == 0 && nr > 1) {
      PlanItem sp = it;
      sp.range = (int)((end + per - 1) / per);
      sp.slot = slot0[b] + it.tile * nr;
      ws.splits[split0[b] + it.tile] = sp;
    }
    return from >= end ? 0 : (int)(min((long long)end, from + per) - from);
  };
  // Key block i of the seeding pass and the column tiles it meets.
  auto seed = [&](int i, PlanSeed& x) {
    const int b = sequence(seed0, i);
    x = PlanSeed{b, i - seed0[b], rows_of[b], queries_of[b], query0[b]};
    return (int)(((long long)x.ql * a.G + 31) / 32 - (long long)max(0, x.block * seed_keys - (x.n - x.ql)) * a.G / 32);
  };
  // A list's entries, longest first (the order within a bucket does not
  // matter), unless each has a CU of its own.  A thread's only entry is formed
  // once.
  auto emit = [&](int count, const auto& entry, const auto& store) {
    if ((long long)count * a.c.HK <= kChip) {
      for (int i = tid; i < count; i += NT) {
        entry(i);
        store(i);
      }
      return;
    }
    constexpr int PER = kBuckets / NT;
#pragma unroll
    for (int x = 0; x < PER; ++x) hist[NT * x + tid] = 0;
    __syncthreads();
    int bin = 0;
    for (int i = tid; i < count; i += NT) {
      bin = kBuckets - 1 - min(entry(i), kBuckets - 1);
      atomicAdd(&hist[bin], 1);
    }
    __syncthreads();
    int own[PER], v[1] = {0}, unused[1];
#pragma unroll
    for (int x = 0; x < PER; ++x) {
      own[x] = hist[PER * tid + x];
      v[0] += own[x];
    }
    scan_all<1, NT>(v, unused, scan_tmp);
#pragma unroll
    for (int x = 0; x < PER; ++x) {
      hist[PER * tid + x] = v[0];
      v[0] += own[x];
    }
    __syncthreads();
    for (int i = tid; i < count; i += NT) {
      if (count > NT) bin = kBuckets - 1 - min(entry(i), kBuckets - 1);
      store(atomicAdd(&hist[bin], 1));
    }
    __syncthreads();
  };
  PlanItem it;
  emit(
      items, [&](int i) {
        const int keyn = item(i, it);
        if (keyn == 0) it.tile = kNoTile;
        return (keyn + kKeyStep - 1) / kKeyStep;
      },
      [&](int at) { ws.items[at] = it; });
  PlanSeed sd;
  emit(
      seeds, [&](int i) { return seed(i, sd); }, [&](int at) { ws.seeds[at] = sd; });
}

template <int D>
struct TileCfg {
  static constexpr int KS = D / 16;          // k-steps of 16 over the head dim
  static constexpr int NT = D / 32;          // output tiles of 32 dims
  static constexpr int ROWB = D * 2;
  static constexpr int CH = ROWB / 16;       // 16-byte pieces of a row
  // K tiles: piece c of row r at 16-byte slot r CH + (c ^ (r mod CH)), so the
  // rows that an operand read touches fall in different LDS banks.
  static constexpr int KTILE = kKeyStep * ROWB;
  static constexpr int KPW = KTILE / (kTileThreads * 16);  // loads of a wave
  static __device__ constexpr int kslot(int r, int c) { return r * CH + (c ^ (r % CH)); }
  // V tiles: load u (one wavefront) carries rows u + VLOADS j into block u.
  static constexpr int VLOADS = kKeyStep * CH / kWave;
  static constexpr int VPW = VLOADS / kTileWaves;
  static constexpr int VBLK = kWave * 16 + 64;
  static constexpr int VTILE = VLOADS * VBLK;
  static __device__ constexpr int vaddr(int r, int c) { return (r % VLOADS) * VBLK + (r / VLOADS) * ROWB + c; }
};

// Order for the compiler's scheduler: N LDS reads next; one product and N
// vector instructions next.
template <int N>
__device__ inline void sched_reads() {
  __builtin_amdgcn_sched_group_barrier(0x100, N, 0);
}
template <int N>
__device__ inline void sched_product() {
  __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
  __builtin_amdgcn_sched_group_barrier(0x402, N, 0);
}

template <typename T, int D, bool kCap>
__global__ __launch_bounds__(kTileThreads) __attribute__((amdgpu_waves_per_eu(2))) void tile_kernel(PagedAttnArgs a, TileWs ws, DecWs dec) {
  using Cfg = TileCfg<D>;
  using M = Mma<T>;
  constexpr int KS = Cfg::KS, NT = Cfg::NT, ROWB = Cfg::ROWB, CH = Cfg::CH, STEP = kKeyStep;
  constexpr int KPW = Cfg::KPW, VPW = Cfg::VPW;
  // Separate arrays, so that the compiler can tell a read of one tile from
  // the direct loads that fill another.
  __shared__ __attribute__((aligned(16))) char kt0[Cfg::KTILE];
  __shared__ __attribute__((aligned(16))) char kt1[Cfg::KTILE];
  __shared__ __attribute__((aligned(16))) char vt0[Cfg::VTILE];
  __shared__ __attribute__((aligned(16))) char vt1[Cfg::VTILE];
  const int tid = threadIdx.x;
  const int lane = tid & (kWave - 1);
  const int w = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int hh = lane >> 5;  // lane half
  const int s = lane & 31;   // column
  const int h = blockIdx.x % a.c.HK;
  const int at = blockIdx.x / a.c.HK;
  const PlanItem it = ws.items[at];  // read beside the list's length
  if (at >= ws.head->items || it.tile == kNoTile) return;
  const int b = it.b, G = a.G, HQ = a.c.HQ;
  const AttnSeq sq{it.n, it.ql, it.q0, true};
  if (it.tile == kChunkItem) {
    __shared__ float2 wave_ml[kNumWaves][kFewCols];
    DecChunk ck;
    ck.b = b;
    ck.h = h;
    ck.c = it.range & 255;
    ck.nch = it.range >> 8;
    ck.n = sq.n;
    ck.ql = sq.ql;
    ck.first = it.slot * a.c.HK + h * ck.nch;
    ck.row0 = ((long long)it.steps0 * a.c.HK + (long long)h * ((sq.n + kDecStep - 1) / kDecStep)) * kDecStep;
    ck.q0 = sq.q0;
    static_assert(Cfg::KTILE >= DecCfg<D>::VTILE && kTileThreads == kThreads, "a wave's tile fits a K tile");
    decode_chunk<T, D, kCap, false>(a, dec, ck, ck.first + ck.c,
                             [&](int v) { return v & 2 ? (v & 1 ? vt1 : vt0) : (v & 1 ? kt1 : kt0); }, wave_ml);
    return;
  }
  const int cols = sq.ql * G, first = sq.n - sq.ql;
  const int ks = it.range * it.keys;
  // Keys [ks, kend) of this wave and of the block; rows up to `full` are
  // attended by each of the wave's columns.
  const int range_end = (int)min((long long)ks + it.keys, (long long)sq.n);
  const int c0 = kTileCols * it.tile + 32 * w;
  const bool active = c0 < cols;
  const int kend_blk = min(range_end, key_end(sq, kTileCols * it.tile + kTileCols - 1, G));
  const int kend = active ? min(range_end, key_end(sq, c0 + 31, G)) : 0;
  const int full = first + c0 / G;
  const int nsteps = (kend_blk - ks + STEP - 1) / STEP;
  const int own = kend > ks ? (kend - ks + STEP - 1) / STEP : 0;
  const int col = c0 + s;
  const int query = query_of(a, col);
  const int pos = first + query;  // this lane's last key
  const Logit<kCap> lg(a);

  // Queries as the B operand of S^T = K Q^T: lane (hh, s) holds
  // Q[column s][dims 16 kk + 8 hh ..].
  typename M::x8 qb[KS];
  {
    const char* q = (const char*)a.q + ((sq.q0 + query) * HQ + h * G + col - query * G) * (long long)ROWB;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk)
      qb[kk] = col < cols ? *reinterpret_cast<const typename M::x8*>(q + 32 * kk + 16 * hh) : mma_zero<T>();
  }

  // Granules of 16 steps at a time: lane l holds granule l of the window; even
  // windows in ids0, odd ones in ids1, the next one asked for ahead.
  const int glast = (kend_blk - 1) >> 4;
  int ids0 = -1, ids1 = -1;
  bool bad = false;
  auto load_ids = [&](int window, int& ids) {
    ids = granule_row(a.c, b, h, min((ks >> 4) + kWave * window + lane, glast));
    bad = bad || __any(ids < 0);
  };
  auto granule = [&](int st, int g) {
    return __builtin_amdgcn_readlane((st >> 4) & 1 ? ids1 : ids0, 4 * (st & 15) + g);
  };
  // This wave's share of a step's tiles.  Rows past the last key of the block
  // (final step only) read that key instead; a granule out of range the
  // pool's first rows.
  const int krow = (kWave * w + lane) / CH;
  const int kpiece = 16 * ((lane % CH) ^ (krow % CH));
  auto issue_k = [&](int st, char* tile) {
    const int j0 = ks + st * STEP;
    if (j0 >= kend_blk) return;
    lds_char* kl = (lds_char*)tile + kWave * 16 * w;
    const int last = kend_blk - 1 - j0;
#pragma unroll
    for (int k = 0; k < KPW; ++k) {
      constexpr int RPL = kTileThreads / CH;          // rows between a wave's loads
      const int g = (RPL * k + kWave / CH * w) >> 4;  // uniform: a load stays in a granule
      if (last >= STEP - 1) {
        const char* p = a.c.k + (long long)max(granule(st, g), 0) * ROWB;
        load_lds(p + (unsigned)((krow & 15) * ROWB + kpiece), kl + kWave * 16 * kTileWaves * k);
      } else {
        const int r = min(krow + RPL * k, last);
        const char* p = a.c.k + (long long)max(granule(st, min(g, last >> 4)), 0) * ROWB;
        load_lds(p + (unsigned)((r & 15) * ROWB + kpiece), kl + kWave * 16 * kTileWaves * k);
      }
    }
  };
  const int vrow = w + Cfg::VLOADS * (lane / CH);  // + 4 a load; granule lane / 16
  auto issue_v = [&](int st, char* tile) {
    const int j0 = ks + st * STEP;
    if (j0 >= kend_blk) return;
    lds_char* vl = (lds_char*)tile + Cfg::VBLK * w;
    const int last = kend_blk - 1 - j0;
    const int i0 = granule(st, 0), i1 = granule(st, 1), i2 = granule(st, 2), i3 = granule(st, 3);
    if (last >= STEP - 1) {
      const int g = lane >> 4;
      const int row = max(g < 2 ? (g == 0 ? i0 : i1) : (g == 2 ? i2 : i3), 0);
      const char* p = a.c.v + (long long)row * ROWB + (vrow & 15) * ROWB + 16 * (lane % CH);
#pragma unroll
      for (int k = 0; k < VPW; ++k) load_lds(p + k * kTileWaves * ROWB, vl + Cfg::VBLK * kTileWaves * k);
    } else {
#pragma unroll
      for (int k = 0; k < VPW; ++k) {
        const int r = min(vrow + kTileWaves * k, last);
        const int g = r >> 4;
        const int row = max(g < 2 ? (g == 0 ? i0 : i1) : (g == 2 ? i2 : i3), 0) + (r & 15);
        load_lds(a.c.v + (long long)row * ROWB + 16 * (lane % CH), vl + Cfg::VBLK * kTileWaves * k);
      }
    }
  };

  float m = kNegBig, l = 0.0f, corr = 1.0f;
  bool grown = false;
  mma_f32x16_t o[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[nt][r] = 0.0f;
  // S^T of a step: lane (hh, s), register r of sub-tile t: key j0 + 32 t +
  // 8 (r / 4) + 4 hh + r % 4, column s.
  mma_f32x16_t sa[2], sb[2];
  auto qk = [&](mma_f32x16_t& x, const char* kt, int t, int kk) {
    x = M::mma32(*reinterpret_cast<const typename M::x8*>(kt + 16 * Cfg::kslot(32 * t + s, 2 * kk + hh)), qb[kk],
                 kk == 0 ? mma_f32x16_t{} : x);
  };
  // Rows of step st on pages out of range, as bits of its granules.
  auto bad_granules = [&](int st) {
    unsigned x = 0;
    if (bad) {
#pragma unroll
      for (int g = 0; g < 4; ++g) x |= (granule(st, g) < 0 ? 1u : 0u) << g;
    }
    return x;
  };
  // A step is plain where every one of its rows counts for every column.
  auto plain = [&](int st) { return ks + st * STEP + STEP - 1 <= full && ks + (st + 1) * STEP <= kend && !bad; };
  auto col_max = [&](const mma_f32x16_t (&x)[2]) {
    float mx = lg.larger(x[0][0], x[1][0]);
#pragma unroll
    for (int r = 1; r < 16; ++r) mx = lg.larger(lg.larger(mx, x[0][r]), x[1][r]);
    return mx;
  };
  auto capped = [&](mma_f32x16_t& x) {
    if constexpr (kCap) {
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = lg.value(x[r]);
    }
  };
  // Masks step st's logits, whose largest over all its rows has value mx, and
  // moves the running maximum.
  auto settle = [&](mma_f32x16_t (&x)[2], int st, float mx) {
    if (!plain(st)) {
      asm volatile("");  // keeps the mask behind a branch
      const int j0 = ks + st * STEP;
      const int lim = min(pos, kend - 1) - j0 - 4 * hh;
      const unsigned bg = bad_granules(st);
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (32 * t + 8 * (r >> 2) + (r & 3) > lim || ((bg >> (2 * t + (r >> 3))) & 1u)) x[t][r] = lg.kMasked;
      mx = col_max(x);
    }
    // The running maximum follows only where it would fall behind by more
    // than kLag: weights then stay below 2^kLag, which the sums and both
    // storage types hold with the same relative error, and the outputs are
    // rescaled a few times a tile (following each maximum: in nearly every
    // step, since one of 32 columns finds a new one).
    const float top = max_halves(lg.logit(mx));
    grown = __any(top > m + kLag);
    if (grown) {
      const float mnew = fmaxf(m, top);
      corr = hw_exp2(m - mnew);
      m = mnew;
    }
  };
  auto rescale = [&]() {
    if (grown) {
      l *= corr;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[nt][r] *= corr;
    }
  };
  // Weights of keys 16 mm .. + 15 in the order of the V^T operand: slot j is
  // key 4 hh + j (j < 4) or 8 + 4 hh + j - 4.  They are rounded to the
  // storage type, as the output is; the sum is of the unrounded ones.
  float psum[2];
  auto half_weights = [&](const mma_f32x16_t (&x)[2], int mm, int half) {
    typename M::x4 p;
#pragma unroll
    for (int j = 0; j < 4; j += 2) {
      const float pa = lg.weight(x[mm >> 1][8 * (mm & 1) + 4 * half + j], lg.B - m);
      const float pb = lg.weight(x[mm >> 1][8 * (mm & 1) + 4 * half + j + 1], lg.B - m);
      psum[0] += pa;
      psum[1] += pb;
      const typename M::x2 r = __builtin_convertvector((mma_f32x2_t{pa, pb}), typename M::x2);
      p[j] = r[0];
      p[j + 1] = r[1];
    }
    return p;
  };
  auto joined = [&](const typename M::x4& u, const typename M::x4& v) {
    return __builtin_shufflevector(u, v, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  auto weights = [&](const mma_f32x16_t (&x)[2], int mm) {
    const typename M::x4 u = half_weights(x, mm, 0);
    return joined(u, half_weights(x, mm, 1));
  };
  // V^T operand of keys 16 mm .. and dims 32 nt ..: lane i of a 16-lane group
  // points at row 4 hh + i / 4 (and 8 more), 4 columns from
  // 32 nt + 16 (group mod 2) + 4 (i mod 4).
  auto v_operand = [&](const char* vtile, int mm, int nt) {
    const lds_char* vt = (const lds_char*)vtile;
    const int vr = 16 * mm + 4 * hh + ((lane & 15) >> 2);
    const int c = (32 * nt + 16 * ((lane >> 4) & 1) + 4 * (lane & 3)) * 2;
    const typename M::x4 a0 = M::read_tr(vt + Cfg::vaddr(vr, c)), a1 = M::read_tr(vt + Cfg::vaddr(vr + 8, c));
    return __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  // A plain step that is not this wave's last: weights and P V of step st,
  // whose logits are in sx, among S^T of step st + 1 (K runs one tile ahead of
  // V).  In eight parts of four products each, S^T and P V in turn; a part's
  // operands are read while the part before it runs.  The matrix and the
  // vector units work side by side where a few vector instructions follow each
  // product (a product of 32 cycles and six of them: 34 to 37; products in a
  // row leave the vector units idle), so the weights are spread over the parts
  // and the compiler is given the order.
  auto body = [&](int st, mma_f32x16_t (&sx)[2], mma_f32x16_t (&sn)[2], const char* knext, const char* vcur) {
    constexpr int KQ = KS / 4;  // k-steps of a part
    rescale();
    psum[0] = psum[1] = 0.0f;
    typename M::x8 kf[KQ][2], vf[NT];
    auto read_k = [&](int part) {
#pragma unroll
      for (int kk = 0; kk < KQ; ++kk)
#pragma unroll
        for (int t = 0; t < 2; ++t)
          kf[kk][t] = *reinterpret_cast<const typename M::x8*>(knext + 16 * Cfg::kslot(32 * t + s, 2 * (KQ * part + kk) + hh));
    };
    read_k(0);
    sched_reads<2 * KQ>();
    typename M::x4 pa = half_weights(sx, 0, 0);
    float mx = 0.0f;
#pragma unroll
    for (int mm = 0; mm < 4; ++mm) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) vf[nt] = v_operand(vcur, mm, nt);
#pragma unroll
      for (int kk = 0; kk < KQ; ++kk)
#pragma unroll
        for (int t = 0; t < 2; ++t)
          sn[t] = M::mma32(kf[kk][t], qb[KQ * mm + kk], mm == 0 && kk == 0 ? mma_f32x16_t{} : sn[t]);
      const typename M::x8 p = joined(pa, half_weights(sx, mm, 1));
      sched_reads<2 * NT>();
#pragma unroll
      for (int i = 0; i < 2 * KQ; ++i) {
        if (mm == 0)
          sched_product<28 / (2 * KQ)>();
        else
          sched_product<16 / (2 * KQ)>();
      }
      if (mm < 3) {
        read_k(mm + 1);
        pa = half_weights(sx, mm + 1, 0);
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) o[nt] = M::mma32(vf[nt], p, o[nt]);
      if (mm < 3) {
        sched_reads<2 * KQ>();
#pragma unroll
        for (int i = 0; i < NT; ++i) sched_product<16 / NT>();
      }
    }
    capped(sn[0]);
    capped(sn[1]);
    mx = col_max(sn);
    l += psum[0] + psum[1];
    // Sums and maximum stay among the products.
    asm volatile("" : "+v"(l) : "v"(mx));
#pragma unroll
    for (int i = 0; i < NT; ++i) sched_product<24 / NT>();
    settle(sn, st + 1, mx);
  };
  // Rows of a step that some columns do not attend must not meet them in a
  // product where they hold an infinity or NaN (0 times either is NaN).  Bits
  // of the rows to leave out: those that no column of the wave attends, and
  // of those that only some do the ones that hold such a value, which
  // `apart` gets.
  auto left_out = [&](int st, const char* vcur, unsigned long long& apart) {
    const int j0 = ks + st * STEP;
    const unsigned bg = bad_granules(st);
    unsigned long long z = kend - j0 < STEP ? ~0ull << (kend - j0) : 0ull;
#pragma unroll
    for (int g = 0; g < 4; ++g)
      if ((bg >> g) & 1u) z |= 0xffffull << (16 * g);
    apart = 0;
    const int r0 = max(full + 1 - j0, 0), r1 = min(kend - j0, STEP);  // attended by some columns only
    for (int x0 = r0 * CH; x0 < r1 * CH; x0 += kWave) {
      const int x = min(x0 + lane, r1 * CH - 1);
      const uint4 v = *reinterpret_cast<const uint4*>(vcur + Cfg::vaddr(x / CH, 16 * (x % CH)));
      unsigned long long hit = __ballot(M::odd(v));
      while (hit) {  // rare
        const int i = (int)__builtin_ctzll(hit);
        apart |= 1ull << (min(x0 + i, r1 * CH - 1) / CH);
        hit &= hit - 1;
      }
    }
    apart &= ~z;
    return z | apart;
  };
  // Any other step: S^T of the next one is not interleaved.
  auto careful = [&](int st, const char* vcur) {
    rescale();
    psum[0] = psum[1] = 0.0f;
    unsigned long long apart;
    const unsigned long long z = left_out(st, vcur, apart);
    typename M::x8 p[4];
#pragma unroll
    for (int mm = 0; mm < 4; ++mm) {
      const unsigned zg = (unsigned)(z >> (16 * mm)) & 0xffffu;
      p[mm] = mma_zero<T>();
      if (zg == 0xffffu && apart == 0) continue;  // no row of these counts
      p[mm] = weights(sa, mm);
      if (zg == 0) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) o[nt] = M::mma32(v_operand(vcur, mm, nt), p[mm], o[nt]);
      } else {
        const unsigned zl = zg >> (4 * hh);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          typename M::x8 av = v_operand(vcur, mm, nt);
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if ((zl >> (8 * (j >> 2) + (j & 3))) & 1u) av[j] = (T)0.0f;
          o[nt] = M::mma32(av, p[mm], o[nt]);
        }
      }
    }
    l += psum[0] + psum[1];
    if (apart) {
      // Their contributions one by one, to the columns that attend them.
#pragma unroll 1
      while (apart) {
        const int r = (int)__builtin_ctzll(apart);
        apart &= apart - 1;
        float mine = 0.0f;  // an index would put p in scratch memory
#pragma unroll
        for (int x = 0; x < 32; ++x) mine = x == 8 * (r >> 4) + 4 * ((r >> 3) & 1) + (r & 3) ? (float)p[x >> 3][x & 7] : mine;
        const float other = __shfl_xor(mine, 32);
        const float pr = ((r >> 2) & 1) == hh ? mine : other;
        if (pos >= ks + st * STEP + r) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int x = 0; x < 16; ++x) {
              const int d = 32 * nt + 8 * (x >> 2) + 4 * hh + (x & 3);
              o[nt][x] = fmaf(pr, (float)*reinterpret_cast<const T*>(vcur + Cfg::vaddr(r, 2 * d)), o[nt][x]);
            }
        }
      }
    }
  };

  // At step st, K of step st + 2 and V of step st + 1 are on their way into
  // the tiles that step st - 1 has read.  Each wave waits for its own loads;
  // the barrier makes every wave's visible and says that those tiles are free.
  auto advance = [&](int st, char* kfill, char* vfill) {
    wait_vmem();
    barrier_only();
    issue_k(st + 2, kfill);
    issue_v(st + 1, vfill);
    if ((st & 15) == 0 && st > 0) {
      if ((st >> 4) & 1)
        load_ids((st >> 4) + 1, ids0);
      else
        load_ids((st >> 4) + 1, ids1);
    }
  };
  load_ids(0, ids0);
  load_ids(1, ids1);
  issue_k(0, kt0);
  issue_k(1, kt1);
  issue_v(0, vt0);
  wait_vmem();
  barrier_only();
  auto alone = [&](int st, const char* kt) {
#pragma unroll
    for (int kk = 0; kk < KS; ++kk)
#pragma unroll
      for (int t = 0; t < 2; ++t) qk(sa[t], kt, t, kk);
    capped(sa[0]);
    capped(sa[1]);
    settle(sa, st, col_max(sa));
  };
  if (own > 0) alone(0, kt0);
  // Steps before `lead` are plain and not the last.  A page out of range
  // further on ends them early.
  const int lead = min(own - 1, (min(full, kend - 1) + 1 - ks) / STEP);
  int st = 0;
  while (st < lead && !bad) {
    advance(st, kt0, vt1);
    body(st, sa, sb, kt1, vt0);
    if (++st >= lead || bad) break;
    advance(st, kt1, vt0);
    body(st, sb, sa, kt0, vt1);
    ++st;
  }
  if (st & 1) {
    sa[0] = sb[0];
    sa[1] = sb[1];
  }
  for (; st < own; ++st) {
    advance(st, (st & 1) ? kt1 : kt0, (st & 1) ? vt0 : vt1);
    careful(st, (st & 1) ? vt1 : vt0);
    if (st + 1 < own) alone(st + 1, (st & 1) ? kt0 : kt1);
  }
  for (; st < nsteps; ++st) advance(st, (st & 1) ? kt1 : kt0, (st & 1) ? vt0 : vt1);
  if (!active) return;

  // l is split over the two lane halves of a column; m is common.
  l += __shfl_xor(l, 32);
  if (it.slot >= 0) {
    const long long pc = ((long long)it.slot * a.c.HK + h) * kTileCols + 32 * w + s;
    if (hh == 0) ws.part_ml[pc] = make_float2(m, l);
    float* const po = ws.part_o + pc * D;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        *reinterpret_cast<float4*>(po + 32 * nt + 2 * r + 4 * hh) = make_float4(o[nt][r], o[nt][r + 1], o[nt][r + 2], o[nt][r + 3]);
    return;
  }
  if (col >= cols) return;
  const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;  // no row at all: 0
  const long long orow = (sq.q0 + query) * HQ + h * G + col - query * G;
  T* const out = (T*)a.out + orow * D;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      const mma_f32x4_t f = mma_f32x4_t{o[nt][r], o[nt][r + 1], o[nt][r + 2], o[nt][r + 3]} * inv;
      *reinterpret_cast<typename M::x4*>(out + 32 * nt + 2 * r + 4 * hh) = __builtin_convertvector(f, typename M::x4);
    }
  if (hh == 0 && a.gamma > 0.0f) ws.stat[orow] = make_float2(m, inv);
}

// Tiles whose keys were cut (the first `tiles` blocks: entry of the split list,
// KV head and kJoinCols columns, 16 lanes each), then the segments with few
// columns.  Few bytes and a chain of reads: a lane reads the statistics of
// every 16th range, and the outputs of eight ranges are asked for at once (16
// queries over 60000 rows: 64 us less than with one range after the other).
template <typename T, int D, int R>
__global__ __launch_bounds__(kThreads) void join_kernel(PagedAttnArgs a, TileWs ws, DecWs dec, unsigned tiles, int span) {
  if (blockIdx.x >= tiles) {
    const unsigned segs = (unsigned)(a.c.B * a.c.HK), i = blockIdx.x - tiles;
    finish_segment<T, D, R>(a, dec, span, (int)(i % segs), i / segs);
    return;
  }
  const int unit = blockIdx.x / (kTileCols / kJoinCols), G = a.G;
  const int entry = unit / a.c.HK, h = unit % a.c.HK;
  const PlanItem it = ws.splits[entry];  // read beside the list's length
  if (entry >= ws.head->splits) return;
  const AttnSeq sq{it.n, it.ql, it.q0, true};
  constexpr int EL = D / 16;  // dims of a lane
  constexpr int ML = kMaxSplit / 16;
  const int x = threadIdx.x % 16, c = kJoinCols * (blockIdx.x % (kTileCols / kJoinCols)) + threadIdx.x / 16;
  const int col = kTileCols * it.tile + c;
  if (col >= sq.ql * G) return;  // whole groups of 16 lanes
  const long long p0 = ((long long)it.slot * a.c.HK + h) * kTileCols + c;
  const long long ps = (long long)a.c.HK * kTileCols;
  float2 ml[ML];
  float m = kNegBig;
#pragma unroll
  for (int k = 0; k < ML; ++k) {
    const int r = 16 * k + x;
    ml[k] = r < it.range ? ws.part_ml[p0 + r * ps] : make_float2(kNegBig, 0.0f);
    m = fmaxf(m, ml[k].x);
  }
#pragma unroll
  for (int k = 8; k > 0; k >>= 1) m = fmaxf(m, __shfl_xor(m, k));
  float l = 0.0f, f[ML];
#pragma unroll
  for (int k = 0; k < ML; ++k) {
    f[k] = hw_exp2(ml[k].x - m);
    l = fmaf(f[k], ml[k].y, l);
  }
  l = group_sum<16>(l);
  const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
  float o[EL];
#pragma unroll
  for (int e = 0; e < EL; ++e) o[e] = 0.0f;
#pragma unroll
  for (int k = 0; k < ML; ++k)
    for (int r0 = 16 * k; r0 < min(it.range, 16 * k + 16); r0 += 8) {
      float4 v[8][EL / 4];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float4* const po = reinterpret_cast<const float4*>(ws.part_o + (p0 + min(r0 + i, it.range - 1) * ps) * D);
#pragma unroll
        for (int e = 0; e < EL / 4; ++e) v[i][e] = po[x + 16 * e];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float g = __shfl(f[k], r0 % 16 + i, 16);
        if (r0 + i < it.range) {
#pragma unroll
          for (int e = 0; e < EL / 4; ++e) {
            o[4 * e] = fmaf(g, v[i][e].x, o[4 * e]);
            o[4 * e + 1] = fmaf(g, v[i][e].y, o[4 * e + 1]);
            o[4 * e + 2] = fmaf(g, v[i][e].z, o[4 * e + 2]);
            o[4 * e + 3] = fmaf(g, v[i][e].w, o[4 * e + 3]);
          }
        }
      }
    }
  const int query = query_of(a, col);
  const long long orow = (sq.q0 + query) * a.c.HQ + h * G + col - query * G;
  typedef typename Mma<T>::x4 x4;
#pragma unroll
  for (int e = 0; e < EL / 4; ++e) {
    const mma_f32x4_t y = mma_f32x4_t{o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]} * inv;
    reinterpret_cast<x4*>((T*)a.out + orow * D)[x + 16 * e] = __builtin_convertvector(y, x4);
  }
  if (x == 0 && a.gamma > 0.0f) ws.stat[orow] = make_float2(m, inv);
}

// Second pass, key-major.  A block is KW waves of 32 NS keys each times IG
// groups of waves; group ig takes the column tiles ig, ig + IG, ... of 32
// columns and keeps its own double-buffered query tile.  Bound by vector
// instructions: a weight takes a multiply-add, an exp2 and a multiply-add
// against 8 matrix-core cycles a lane, so the rest is kept small (64 keys a
// wave share a tile's reads, addresses move by constants) and the products of
// the next tile run among the weights of this one.  Blocks of four waves, two a
// CU, so that one's beginning runs beside the other's weights (109 sequences of
// 44 to 59 queries over 1428 to 4873 rows, D 64, three rounds a block: 244 us, 304
// with one block of eight waves; 16 queries over 60000 rows 108, 136).  Where the
// blocks of 256 keys do not fill the chip, 64 keys and two groups.
constexpr int kSeedThreads = 256;

template <typename T, int D, bool kCap, int NS, int KW, int IG>
__device__ inline void seed_block(const PagedAttnArgs& a, const TileWs& ws, const PlanSeed& sq, int h, int kblk0, char* const buf0,
                                  char* const buf1, float* const sums) {
  using Cfg = TileCfg<D>;
  using M = Mma<T>;
  constexpr int KS = Cfg::KS, ROWB = Cfg::ROWB, CH = Cfg::CH;
  constexpr int KEYS = 32 * NS * KW;  // of a block
  constexpr int QTILE = 32 * ROWB;
  constexpr int LPW = QTILE / (kWave * 16) / KW;  // loads of a wave
  static_assert(LPW >= 1, "a tile gives every wave of a group a load");
  static_assert(KW * IG * kWave == kSeedThreads, "every wave has keys and a group");
  const int tid = threadIdx.x;
  const int lane = tid & (kWave - 1);
  const int w = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int kw = w % KW, ig = w / KW;
  const int hh = lane >> 5, s = lane & 31;
  const int b = sq.b, G = a.G, HQ = a.c.HQ, cols = sq.ql * G, first = sq.n - sq.ql;
  const int j0w = kblk0 + 32 * NS * kw;

  // This wave's keys as the A operand (row 32 t + s, dims 16 kk + 8 hh ..).
  typename M::x8 kr[NS][KS];
#pragma unroll
  for (int t = 0; t < NS; ++t) {
    const int row = min(j0w + 32 * t + s, sq.n - 1);
    const int gr = granule_row(a.c, b, h, row >> 4);
    const char* p = a.c.k + (long long)(max(gr, 0) + (row & 15)) * ROWB;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) kr[t][kk] = *reinterpret_cast<const typename M::x8*>(p + 32 * kk + 16 * hh);
  }

  // Column tiles holding a query at or after the block's first key.  A lane's
  // place in its group's next tile, for each of its loads and for its
  // column's statistics: row of q and head, and the head alone.
  const int it0 = (int)((long long)max(0, kblk0 - first) * G / 32);
  const int nitems = (cols + 31) / 32 - it0;
  struct Place {
    long long at;
    int head;
  };
  auto place = [&](int c) {
    const int qi = query_of(a, c);
    return Place{(sq.q0 + qi) * HQ + h * G + c - qi * G, c - qi * G};
  };
  constexpr int kAdvance = 32 * IG;
  const int dq = kAdvance / G, dh = kAdvance % G;
  auto move = [&](Place& x) {
    x.at += dq * HQ + dh;
    x.head += dh;
    const bool wrap = x.head >= G;
    x.at += wrap ? HQ - G : 0;
    x.head -= wrap ? G : 0;
  };
  const int qrow = (kWave * kw + lane) / CH;                   // + 64 KW / CH a load
  Place pl[LPW], ps = place(32 * (it0 + ig) + s);
#pragma unroll
  for (int k = 0; k < LPW; ++k) pl[k] = place(32 * (it0 + ig) + qrow + k * (kWave * KW / CH));
  int left = cols - 32 * (it0 + ig);  // columns from the group's next tile on
  float2 st_next = make_float2(0.0f, 0.0f);
  auto issue = [&](char* buf) {
#pragma unroll
    for (int k = 0; k < LPW; ++k) {
      const int r = qrow + k * (kWave * KW / CH);
      if (r < left)
        load_lds((const char*)a.q + pl[k].at * ROWB + 16 * ((lane % CH) ^ (r % CH)), (lds_char*)buf + ig * QTILE + kWave * 16 * (kw + KW * k));
      move(pl[k]);
    }
    if (s < left) st_next = ws.stat[ps.at];
    move(ps);
    left -= kAdvance;
  };
  const Logit<kCap> lg(a);
  float acc[NS][16];
#pragma unroll
  for (int t = 0; t < NS; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[t][r] = 0.0f;
  auto product = [&](mma_f32x16_t (&x)[NS], const char* buf) {
    const char* qt = buf + ig * QTILE;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) {
      const typename M::x8 q = *reinterpret_cast<const typename M::x8*>(qt + 16 * Cfg::kslot(s, 2 * kk + hh));
#pragma unroll
      for (int t = 0; t < NS; ++t) x[t] = M::mma32(kr[t][kk], q, kk == 0 ? mma_f32x16_t{} : x[t]);
    }
  };
  // The weights of an item, whose products are in x, among the products of the
  // next one, whose queries are in `buf`.  Columns past the last have whatever
  // lies in their place; no product mixes columns.
  auto step = [&](int item, mma_f32x16_t (&x)[NS], float2 qs, mma_f32x16_t (&xn)[NS], const char* buf) {
    const int c0 = 32 * (it0 + item);
    const float shift = lg.B - qs.x;
    if (item < nitems && first + query_of(a, c0) >= j0w + 32 * NS - 1 && c0 + 32 <= cols) {
      product(xn, buf);
#pragma unroll
      for (int t = 0; t < NS; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[t][r] = fmaf(lg.weight(lg.value(x[t][r]), shift), qs.y, acc[t][r]);
    } else {
      // A masked weight is left out, whatever its column's statistics hold.
      const int lim = c0 + s < cols ? first + query_of(a, c0 + s) - j0w - 4 * hh : -1;
#pragma unroll
      for (int t = 0; t < NS; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float p = lg.weight(lg.value(x[t][r]), shift) * qs.y;
          acc[t][r] += 32 * t + 8 * (r >> 2) + (r & 3) > lim ? 0.0f : p;
        }
      product(xn, buf);
    }
  };
  // Round x: the products of item x + 1 need its queries (asked for two rounds
  // ago); those of item x + 2 go where item x's were.
  const int rounds = (nitems + IG - 1) / IG;
  float2 qs0, qs1;
  mma_f32x16_t xa[NS], xb[NS];
  issue(buf0);
  qs0 = st_next;
  issue(buf1);
  qs1 = st_next;
  wait_vmem();
  barrier_only();
  product(xa, buf0);
  for (int x = 0; x < rounds; x += 2) {
    wait_vmem();
    barrier_only();
    issue(buf0);
    step(x * IG + ig, xa, qs0, xb, buf1);
    qs0 = st_next;
    if (x + 1 >= rounds) break;
    wait_vmem();
    barrier_only();
    issue(buf1);
    step((x + 1) * IG + ig, xb, qs1, xa, buf0);
    qs1 = st_next;
  }
  // Sum over the 32 columns: each exchange halves the keys a lane holds, until
  // lane s holds key register s / 2.
#pragma unroll
  for (int t = 0; t < NS; ++t) {
#pragma unroll
    for (int half = 8; half >= 1; half /= 2) {
      const bool up = (s & (2 * half)) != 0;
#pragma unroll
      for (int r = 0; r < half; ++r) {
        const float mine = up ? acc[t][r + half] : acc[t][r];
        const float give = up ? acc[t][r] : acc[t][r + half];
        acc[t][r] = mine + __shfl_xor(give, 2 * half);
      }
    }
    const float v = acc[t][0] + __shfl_xor(acc[t][0], 1);
    const int r = s >> 1;
    if ((s & 1) == 0) sums[ig * KEYS + 32 * (NS * kw + t) + 8 * (r >> 2) + 4 * hh + (r & 3)] = v;
  }
  __syncthreads();
  const int j = kblk0 + tid;
  if (tid < KEYS && j < sq.n) {
    const int gr = granule_row(a.c, b, h, j >> 4);
    if (gr >= 0) {
      float* const sp = a.c.score + gr + (j & 15);
      float t = sums[tid];
#pragma unroll
      for (int x = 1; x < IG; ++x) t += sums[x * KEYS + tid];
      *sp = fmaf(a.gamma, *sp, t);
    }
  }
}

template <typename T, int D, bool kCap>
__global__ __launch_bounds__(kSeedThreads) __attribute__((amdgpu_waves_per_eu(2))) void seed_kernel(PagedAttnArgs a, TileWs ws) {
  constexpr int QTILE = 32 * TileCfg<D>::ROWB;
  __shared__ __attribute__((aligned(16))) char buf0[2 * QTILE];
  __shared__ __attribute__((aligned(16))) char buf1[2 * QTILE];
  __shared__ float sums[kSeedWide];
  static_assert(kSeedWide >= 2 * kSeedNarrow, "both forms' sums fit");
  const PlanHead head = *ws.head;
  for (int i = blockIdx.x; i < head.seeds * a.c.HK; i += gridDim.x) {
    const PlanSeed x = ws.seeds[i / a.c.HK];
    const int h = i % a.c.HK;
    if (head.wide)
      seed_block<T, D, kCap, 2, 4, 1>(a, ws, x, h, x.block * kSeedWide, buf0, buf1, sums);
    else
      seed_block<T, D, kCap, 1, 2, 2>(a, ws, x, h, x.block * kSeedNarrow, buf0, buf1, sums);
    __syncthreads();  // the buffers are free
  }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
struct Sizes {
  int max_q, max_kv, R;
  long long dec_grid;
  long long items, slots, tiles;
  size_t total;
  DecWs dec;
  TileWs tile;
};

// Grid sizes and the workspace's parts (their addresses from `ws` on).  The
// bounds may be loose: no sequence that passes the checks has more queries
// than there are query rows, or more rows than its table holds.
bool sizes(Sizes& z, int64_t q_rows, int max_q, long long max_kv, int B, int HQ, int HK, int D, int64_t pool_rows, char* ws) {
  const int G = HQ / HK;
  if (q_rows > (1LL << 28) / G) return false;  // columns stay below 2^28
  z.max_q = (int)std::min<int64_t>(max_q, q_rows);
  z.max_kv = (int)max_kv;
  if (z.max_kv == 0) z.max_q = 0;
  z.R = B <= kWave ? 1 : B <= 4 * kWave ? 4 : 16;
  const long long steps = (z.max_kv + kDecStep - 1LL) / kDecStep * B;
  if (steps * HK > 0x7fffffffLL) return false;
  char* p = ws;
  auto part = [&](size_t bytes) {
    char* const at = p;
    p += align_up(bytes, 256);
    return at;
  };
  // Threads of a launch stay below 2^32 (the largest are the joining ones).
  if ((4LL * B * HK + 8LL * HK + 32768) * kThreads > 0xffffffffLL) return false;
  z.dec_grid = std::min(dec_blocks(steps * HK), steps * HK / kDecLeastSteps) + (long long)B * HK;
  z.dec.logit_rows = std::min(steps * kDecStep, pool_rows + (long long)B * kDecStep) * HK;
  const int room = room_cols(z.max_q, G);
  z.dec.part = (float*)part((size_t)z.dec_grid * dec_part(room, D) * 4);
  z.dec.logit = (float*)part((size_t)z.dec.logit_rows * room * 4);
  if (z.max_q > kFewCols / G) {
    // Every sequence with queries rounds up to whole tiles.
    z.tiles = q_rows * G / kTileCols + std::min<int64_t>(B, q_rows);
    z.items = z.tiles + 2 * kChip / HK + 1 + z.dec_grid / HK + 1;
    z.slots = z.max_kv <= kLeastKeys ? 0 : std::min<long long>(4LL * kChip / HK + 2, z.tiles * std::min<long long>(kMaxSplit, (z.max_kv + kLeastKeys - 1) / kLeastKeys));
    z.tile.max_items = (int)std::min(z.items, 0x7fffffffLL);
    z.tile.max_slots = (int)z.slots;
    // Key blocks of sequences with many columns; narrow ones only where the
    // wide ones are fewer than kSeedFill, four to a wide one at most.
    const long long wide = std::min<int64_t>(B, q_rows / 2) * ((z.max_kv + kSeedWide - 1LL) / kSeedWide);
    const long long seeds = std::max(wide, std::min(4 * wide, 4LL * kSeedFill / HK + 4));
    if (seeds * HK > 0x7fffffffLL) return false;
    z.tile.max_seeds = (int)seeds;
    z.tile.head = (PlanHead*)part(sizeof(PlanHead));
    z.tile.items = (PlanItem*)part((size_t)z.items * sizeof(PlanItem));
    z.tile.splits = (PlanItem*)part((size_t)z.items * sizeof(PlanItem));
    z.tile.seeds = (PlanSeed*)part((size_t)seeds * sizeof(PlanSeed));
    z.tile.stat = (float2*)part((size_t)q_rows * HQ * sizeof(float2));
    z.tile.part_ml = (float2*)part((size_t)z.slots * HK * kTileCols * sizeof(float2));
    z.tile.part_o = (float*)part((size_t)z.slots * HK * kTileCols * D * 4);
    if (z.items * HK * kTileThreads > 0xffffffffLL) return false;
  }
  z.total = (size_t)(p - ws);
  return true;
}

// Finishing blocks of a segment: one for its output, and with scores one for
// every `span` rows (each repeats the map and the statistics).
unsigned finish_blocks(const PagedAttnArgs& a, int& span) {
  const long long units = std::max(1LL, (a.max_kv + kFinUnit - 1LL) / kFinUnit);
  const long long per = std::max(1LL, units * a.c.B * a.c.HK / kFinBlocks);
  span = (int)std::min(per * kFinUnit, 0x40000000LL);
  return 1u + (a.gamma > 0.0f ? (unsigned)((units + per - 1) / per) : 0u);
}

template <typename T, int D, bool kCap, int R>
lethe_status launch_few(const PagedAttnArgs& a, const Sizes& z, hipStream_t s) {
  const auto kernel = z.max_q <= 1 ? decode_kernel<T, D, kCap, R, true> : decode_kernel<T, D, kCap, R, false>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)z.dec_grid), dim3(kThreads), 0, s, a, z.dec);
  if (hipGetLastError() != hipSuccess) return LETHE_ERR_HIP;
  int span;
  const unsigned y = finish_blocks(a, span);
  hipLaunchKernelGGL((finish_kernel<T, D, R>), dim3(a.c.B * a.c.HK, y), dim3(kThreads), 0, s, a, z.dec, span);
  return hipGetLastError() == hipSuccess ? LETHE_OK : LETHE_ERR_HIP;
}

template <typename T, int D, bool kCap, int R>
lethe_status launch_form(const PagedAttnArgs& a, const Sizes& z, hipStream_t s) {
  if (z.max_q <= kFewCols / a.G) return launch_few<T, D, kCap, R>(a, z, s);
  constexpr int plan_threads = R == 16 ? 1024 : 256;
  hipLaunchKernelGGL(plan_kernel<plan_threads>, dim3(1), dim3(plan_threads), 0, s, a, z.tile);
  if (hipGetLastError() != hipSuccess) return LETHE_ERR_HIP;
  hipLaunchKernelGGL((tile_kernel<T, D, kCap>), dim3((unsigned)(z.items * a.c.HK)), dim3(kTileThreads), 0, s, a, z.tile,
                     z.dec);
  if (hipGetLastError() != hipSuccess) return LETHE_ERR_HIP;
  // A cut tile has two slots at least.
  int span;
  const unsigned y = finish_blocks(a, span);
  const unsigned tiles = (unsigned)(std::min(z.tiles, z.slots / 2) * a.c.HK * (kTileCols / kJoinCols));
  hipLaunchKernelGGL((join_kernel<T, D, R>), dim3(tiles + (unsigned)(a.c.B * a.c.HK) * y), dim3(kThreads), 0, s, a, z.tile,
                     z.dec, tiles, span);
  if (hipGetLastError() != hipSuccess) return LETHE_ERR_HIP;
  if (!(a.gamma > 0.0f)) return LETHE_OK;
  const unsigned blocks = (unsigned)std::min<long long>((long long)z.tile.max_seeds * a.c.HK, kSeedGrid);
  hipLaunchKernelGGL((seed_kernel<T, D, kCap>), dim3(blocks), dim3(kSeedThreads), 0, s, a, z.tile);
  return hipGetLastError() == hipSuccess ? LETHE_OK : LETHE_ERR_HIP;
}

template <typename T, int D>
lethe_status launch_cap(const PagedAttnArgs& a, const Sizes& z, hipStream_t s) {
  const bool cap = a.cap_log2 > 0.0f;
  if (z.R == 1) return cap ? launch_form<T, D, true, 1>(a, z, s) : launch_form<T, D, false, 1>(a, z, s);
  if (z.R == 4) return cap ? launch_form<T, D, true, 4>(a, z, s) : launch_form<T, D, false, 4>(a, z, s);
  return cap ? launch_form<T, D, true, 16>(a, z, s) : launch_form<T, D, false, 16>(a, z, s);
}

}  // namespace

size_t paged_attn_ws_bytes(int64_t q_rows, int max_q, long long max_kv, int B, int HQ, int HK, int D, int64_t pool_rows) {
  Sizes z{};
  return sizes(z, q_rows, max_q, max_kv, B, HQ, HK, D, pool_rows, nullptr) ? std::max<size_t>(z.total, 256) : 0;
}

lethe_status launch_paged_attn(const PagedAttnArgs& args, lethe_dtype dt, int D, int64_t pool_rows, hipStream_t s) {
  Sizes z{};
  if (!sizes(z, args.q_rows, args.max_q, args.max_kv, args.c.B, args.c.HQ, args.c.HK, D, pool_rows, args.ws))
    return LETHE_ERR_UNSUPPORTED;
  PagedAttnArgs a = args;
  a.max_q = z.max_q;
  a.max_kv = z.max_kv;
  if (dt == LETHE_BF16) return D == 128 ? launch_cap<__bf16, 128>(a, z, s) : launch_cap<__bf16, 64>(a, z, s);
  return D == 128 ? launch_cap<_Float16, 128>(a, z, s) : launch_cap<_Float16, 64>(a, z, s);
}

}  // namespace lethe
