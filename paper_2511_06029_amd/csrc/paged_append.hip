// Append to a paged cache: rotation of queries and keys, and the new rows'
// way into their pages, gfx950.
//
// A block takes kRows or fewer consecutive rows of q / k_new / v_new, whatever
// sequences they belong to.  It finds each row's sequence (every thread looks
// at some sequences' row ranges), checks the sequence, forms the rows' sines
// and cosines once in shared memory, and then copies: an item is 16 elements
// of one head of one row (two 16-byte pieces, the two halves of eight pairs),
// neighbouring lanes on neighbouring pieces.  Bytes bound it: each element is
// read once and written once (8 sequences of 1500 to 2048 rows of 48 heads, 347
// MB: 77 us, 4.6 TB/s, a large copy reaching 4.8); one row is a chain of four
// reads (4.6 us).  Eight rows a block share the search and the sines; one a
// block while the rows do not fill the chip.
//
// The angle is a position times a frequency, reduced to a turn's fraction in
// 64 bits (a position of 10^6 leaves an fp32 product no more than two decimal
// digits of the angle); sine and cosine of the fraction in 32 bits, the
// rotation in 32 bits, one rounding to the storage type.
#include <algorithm>

#include "device_common.h"
#include "paged_internal.h"

namespace lethe {

namespace {

constexpr int kAppThreads = 256;
constexpr int kAppRows = 8;      // rows of a block, at most
constexpr int kMaxPairs = 64;    // head_dim / 2
constexpr double kInvTwoPi = 0.15915494309189533577;

// Eight elements of a 16-bit type.
template <typename T>
struct Eight {
  typedef T vec_t __attribute__((ext_vector_type(8)));
  typedef float f32_t __attribute__((ext_vector_type(8)));
  static __device__ inline f32_t widen(const uint4& r) { return __builtin_convertvector(__builtin_bit_cast(vec_t, r), f32_t); }
  static __device__ inline uint4 narrow(const f32_t& f) { return __builtin_bit_cast(uint4, __builtin_convertvector(f, vec_t)); }
};

// Whether the new rows of sequence b fit the cache; *bits gets what is wrong.
// n and tok: rows and tokens before them.  All threads of the block call it.
__device__ inline bool append_fits(const PagedView& c, int b, int ql, int& n, int& tok, int* bits) {
  n = c.len[b];
  tok = c.seen[b];
  const long long room = (long long)c.max_pages << c.page_shift;
  if (n < 0 || n > room || tok < 0 || (long long)tok + ql > 0x7fffffffLL) {
    *bits = LETHE_DEV_BAD_LAYOUT;
    return false;
  }
  if (n + (long long)ql > room) {
    *bits = LETHE_DEV_APPEND_OVERFLOW;
    return false;
  }
  bool bad = false;
  if (ql > 0) {
    const int last = (n + ql - 1) >> c.page_shift;
    for (int i = (n >> c.page_shift) + (int)threadIdx.x; i <= last; i += kAppThreads) {
      const int page = c.table[(long long)b * c.max_pages + i];
      bad = bad || page < 0 || page >= c.num_pages;
    }
  }
  if (__syncthreads_or(bad)) {
    *bits = LETHE_DEV_BAD_LAYOUT;
    return false;
  }
  return true;
}

__device__ inline bool range_ok(const PagedAppendArgs& a, long long qs, int ql) {
  return ql >= 0 && ql <= a.max_q && qs >= 0 && qs + ql <= a.q_rows;
}

template <typename T, int D>
__global__ __launch_bounds__(kAppThreads) void append_kernel(PagedAppendArgs a, int rows) {
  constexpr int CH = D / 8;      // 16-byte pieces of a row
  constexpr int IT = D / 16;     // items of a head
  __shared__ int seq[kAppRows];          // sequence of a row, -1: none
  __shared__ int row_n[kAppRows];        // its row in the cache, -1: not appended
  __shared__ int row_tok[kAppRows];
  __shared__ float2 turn[kAppRows][kMaxPairs];  // cos, sin
  const int tid = threadIdx.x;
  const long long r0 = (long long)blockIdx.x * rows;
  const int nr = (int)min((long long)rows, a.q_rows - r0);  // no rows at all: one block, for the flags
  if (tid < kAppRows) seq[tid] = row_n[tid] = -1;
  __syncthreads();
  for (int b = tid; b < a.c.B; b += kAppThreads) {
    const long long qs = a.q_start[b];
    const int ql = a.q_len[b];
    if (!range_ok(a, qs, ql)) {
      if (blockIdx.x == 0) atomicOr(a.c.dev_status, LETHE_DEV_BAD_LAYOUT);
      continue;
    }
    for (long long r = max(qs, r0); r < min(qs + ql, r0 + nr); ++r) seq[r - r0] = b;
  }
  __syncthreads();
  for (int i = 0, before = -1, n = 0, tok = 0; i < nr; ++i) {
    const int b = seq[i];
    if (b < 0) continue;  // the same for every thread
    if (b != before) {
      int bits = 0;
      before = b;
      if (!append_fits(a.c, b, a.q_len[b], n, tok, &bits)) {
        n = -1;
        if (tid == 0) atomicOr(a.c.dev_status, bits);
      }
    }
    if (tid == 0 && n >= 0) {
      const int j = (int)(r0 + i - a.q_start[b]);
      row_n[i] = n + j;
      row_tok[i] = tok + j;
    }
  }
  const int half = a.rot / 2;
  for (int x = tid; x < nr * half; x += kAppThreads) {
    const int i = x / half, j = x % half;
    if (seq[i] < 0) continue;
    int axis = 0;
    while (axis + 1 < a.axes && j >= a.ends[axis]) ++axis;
    const double turns = (double)a.axis_pos[(long long)axis * a.q_rows + r0 + i] * (double)a.inv_freq[j] * kInvTwoPi;
    float s, c;
    sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
    turn[i][j] = make_float2(c, s);
  }
  __syncthreads();

  // One row's items: queries, keys, values, in that order.
  const int heads_q = a.q ? a.c.HQ : 0;
  const int items = (heads_q + 2 * a.c.HK) * IT;
  for (int x = tid; x < nr * items; x += kAppThreads) {
    const int i = x / items;
    int head = x % items / IT;
    const int it = x % IT;
    if (seq[i] < 0) continue;
    const bool is_q = head < heads_q;
    const bool is_v = !is_q && head >= heads_q + a.c.HK;
    head -= is_q ? 0 : is_v ? heads_q + a.c.HK : heads_q;
    const long long r = r0 + i;
    const T* src;
    T* dst;
    if (is_q) {
      src = (const T*)a.q + r * a.q_stride + head * D;
      dst = (T*)a.q_out + (r * a.c.HQ + head) * D;
    } else {
      const int n = row_n[i];
      if (n < 0) continue;
      const int page = a.c.table[(long long)seq[i] * a.c.max_pages + (n >> a.c.page_shift)];
      const long long row = page_row(a.c, page, head) + (n & ((1 << a.c.page_shift) - 1));
      src = is_v ? (const T*)a.v_new + r * a.v_stride + head * D : (const T*)a.k_new + r * a.k_stride + head * D;
      dst = (T*)(is_v ? a.c.v : a.c.k) + row * D;
      if (is_v && it == 0) {
        a.c.score[row] = 0.0f;
        a.c.pos[row] = row_tok[i];
      }
    }
    // Pieces of the item: the two halves of eight pairs, or two neighbours
    // (adjacent pairs, elements that are not rotated, values).
    const int rot_items = is_v ? 0 : a.rot / 16;
    const bool turned = it < rot_items;
    const bool split = turned && !a.adjacent;
    const int c0 = split ? it : 2 * it;
    const int c1 = split ? it + rot_items : 2 * it + 1;
    uint4 p0 = reinterpret_cast<const uint4*>(src)[c0], p1 = reinterpret_cast<const uint4*>(src)[c1];
    if (turned) {
      auto x0 = Eight<T>::widen(p0), x1 = Eight<T>::widen(p1);
      if (split) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float2 t = turn[i][8 * it + j];
          const float u = x0[j], w = x1[j];
          x0[j] = u * t.x - w * t.y;
          x1[j] = w * t.x + u * t.y;
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 t0 = turn[i][8 * it + j], t1 = turn[i][8 * it + 4 + j];
          const float u0 = x0[2 * j], w0 = x0[2 * j + 1], u1 = x1[2 * j], w1 = x1[2 * j + 1];
          x0[2 * j] = u0 * t0.x - w0 * t0.y;
          x0[2 * j + 1] = w0 * t0.x + u0 * t0.y;
          x1[2 * j] = u1 * t1.x - w1 * t1.y;
          x1[2 * j + 1] = w1 * t1.x + u1 * t1.y;
        }
      }
      p0 = Eight<T>::narrow(x0);
      p1 = Eight<T>::narrow(x1);
    }
    static_assert(CH == 2 * IT, "an item is two pieces");
    reinterpret_cast<uint4*>(dst)[c0] = p0;
    reinterpret_cast<uint4*>(dst)[c1] = p1;
  }
  // A sequence of one new row lies in this block alone, whose reads of its
  // length are done; longer ones are left to advance_kernel.
  if (a.max_q <= 1 && tid < nr && row_n[tid] >= 0) {
    a.c.len[seq[tid]] = row_n[tid] + 1;
    a.c.seen[seq[tid]] = row_tok[tid] + 1;
  }
}

// len and seen of sequences with several new rows, once the rows are written:
// one block a sequence, with the checks of append_kernel.
__global__ __launch_bounds__(kAppThreads) void advance_kernel(PagedAppendArgs a) {
  const int b = blockIdx.x;
  const int ql = a.q_len[b];
  if (!range_ok(a, a.q_start[b], ql) || ql == 0) return;
  int n, tok, bits = 0;
  if (!append_fits(a.c, b, ql, n, tok, &bits)) return;
  if (threadIdx.x == 0) {
    a.c.len[b] = n + ql;
    a.c.seen[b] = tok + ql;
  }
}

template <typename T, int D>
lethe_status launch(const PagedAppendArgs& a, hipStream_t s) {
  // One row a block until the blocks fill the chip, then up to kAppRows.
  const int rows = (int)std::max<int64_t>(1, std::min<int64_t>(kAppRows, a.q_rows / 1024));
  const int64_t blocks = std::max<int64_t>(1, (a.q_rows + rows - 1) / rows);
  if (blocks * kAppThreads > 0xffffffffLL) return LETHE_ERR_UNSUPPORTED;
  hipLaunchKernelGGL((append_kernel<T, D>), dim3((unsigned)blocks), dim3(kAppThreads), 0, s, a, rows);
  if (hipGetLastError() != hipSuccess) return LETHE_ERR_HIP;
  if (a.max_q > 1) {
    hipLaunchKernelGGL(advance_kernel, dim3(a.c.B), dim3(kAppThreads), 0, s, a);
    if (hipGetLastError() != hipSuccess) return LETHE_ERR_HIP;
  }
  return LETHE_OK;
}

}  // namespace

lethe_status launch_paged_append(const PagedAppendArgs& a, lethe_dtype dt, int D, hipStream_t s) {
  if (dt == LETHE_BF16) return D == 128 ? launch<__bf16, 128>(a, s) : launch<__bf16, 64>(a, s);
  return D == 128 ? launch<_Float16, 128>(a, s) : launch<_Float16, 64>(a, s);
}

}  // namespace lethe
