// What the paged cache's sources share: the layer view that the kernels get,
// row addressing, and the launch functions.
#pragma once

#include "lethe_internal.h"

namespace lethe {

// One layer of a paged cache.
struct PagedView {
  char* k;               // the pools, seen as rows of D elements
  char* v;
  float* score;
  int32_t* pos;
  int32_t* len;          // [B], the layer's
  int32_t* seen;         // [B]
  const int32_t* table;  // [B][max_pages]
  int32_t num_pages, page_shift, max_pages, B, HQ, HK;
  int32_t* dev_status;
};

// Pool row of head h's first row in a page (num_pages * HK * page_size < 2^31).
__host__ __device__ inline int page_row(const PagedView& p, int page, int h) {
  return (page * p.HK + h) << p.page_shift;
}

struct PagedAppendArgs {
  PagedView c;
  const void* q;
  const void* k_new;
  const void* v_new;
  int64_t q_stride, k_stride, v_stride;  // elements between rows
  const int64_t* q_start;
  const int32_t* q_len;
  int64_t q_rows;
  int32_t max_q;
  const float* inv_freq;    // null: no rotation
  const int32_t* axis_pos;
  int32_t rot, adjacent, axes;
  int32_t ends[LETHE_MAX_AXES];  // pair index after each axis' last
  void* q_out;
};

lethe_status launch_paged_append(const PagedAppendArgs& a, lethe_dtype dt, int D, hipStream_t s);

struct PagedAttnArgs {
  PagedView c;
  const void* q;
  const int64_t* q_start;
  const int32_t* q_len;
  int64_t q_rows;
  int32_t max_q, max_kv, G;
  uint32_t g_magic;  // 2^32 / G, rounded up (G > 1)
  float scale_log2;  // softmax scale * log2(e)
  float cap_in;      // softcap > 0: 2 * scale * log2(e) / softcap
  float cap_log2;    // softcap * log2(e), 0 for none
  float gamma;       // 0: scores are left alone
  void* out;
  char* ws;
};

// 0 where the sizes are too large for the launches.
size_t paged_attn_ws_bytes(int64_t q_rows, int max_q, long long max_kv, int B, int HQ, int HK, int D, int64_t pool_rows);
lethe_status launch_paged_attn(const PagedAttnArgs& a, lethe_dtype dt, int D, int64_t pool_rows, hipStream_t s);

struct PagedEvictArgs {
  PagedView c;           // layer 0: len, seen and table hold every layer
  int32_t L, D;
  const int32_t* budget; // [B][L]
  int32_t recent, sink, max_kv;
  int32_t* count;        // [L][B][HK] moves of a segment, or kEvict* codes
  int2* moves;           // (destination, source) pool rows: a segment's i-th at the place of its row i
};

constexpr int32_t kEvictNone = -1;  // nothing changes: the budget has room, or a bad layout

lethe_status launch_paged_evict(const PagedEvictArgs& a, hipStream_t s);

}  // namespace lethe
