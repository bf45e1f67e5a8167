// Host side of the paged cache's calls: argument validation, workspace sizing
// and launch dispatch.  Every check runs before any HIP call.
#include <float.h>
#include <math.h>

#include "paged_internal.h"

using namespace lethe;

namespace {

lethe_status check_desc(const lethe_paged_cache* c) {
  if (!c) return LETHE_ERR_INVALID;
  if (c->num_layers < 1 || c->num_seqs < 1 || c->num_q_heads < 1 || c->num_kv_heads < 1) return LETHE_ERR_INVALID;
  if (c->num_pages < 1 || c->page_size < 1 || c->max_pages < 1) return LETHE_ERR_INVALID;
  if (c->num_q_heads % c->num_kv_heads != 0) return LETHE_ERR_INVALID;
  if (c->dtype != LETHE_BF16 && c->dtype != LETHE_F16 && c->dtype != LETHE_F32) return LETHE_ERR_INVALID;
  if (c->dtype == LETHE_F32) return LETHE_ERR_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128) return LETHE_ERR_UNSUPPORTED;
  if (c->num_q_heads / c->num_kv_heads > 8) return LETHE_ERR_UNSUPPORTED;
  if (c->num_seqs > kMaxSeqs || c->num_layers > kMaxLayers) return LETHE_ERR_UNSUPPORTED;
  if (c->page_size < 16 || c->page_size > 1024 || (c->page_size & (c->page_size - 1))) return LETHE_ERR_UNSUPPORTED;
  // Row numbers of the pool and of a sequence are int32.
  if (c->num_pages > 0x7fffffffLL / c->page_size / c->num_kv_heads) return LETHE_ERR_UNSUPPORTED;
  if (c->max_pages > 0x7fffffff / c->page_size) return LETHE_ERR_UNSUPPORTED;
  return LETHE_OK;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// Sizes plus the device pointers that every call needs.
lethe_status check_cache(const lethe_paged_cache* c) {
  const lethe_status st = check_desc(c);
  if (st != LETHE_OK) return st;
  if (!c->k || !c->v || !c->len || !c->page_table || !c->dev_status) return LETHE_ERR_INVALID;
  if (!aligned16(c->k) || !aligned16(c->v)) return LETHE_ERR_INVALID;
  return LETHE_OK;
}

PagedView view(const lethe_paged_cache* c, int layer) {
  PagedView p;
  p.k = (char*)c->k;
  p.v = (char*)c->v;
  p.score = c->score;
  p.pos = c->pos;
  p.len = c->len + (size_t)layer * c->num_seqs;
  p.seen = c->seen ? c->seen + (size_t)layer * c->num_seqs : nullptr;
  p.table = c->page_table + (size_t)layer * c->num_seqs * c->max_pages;
  p.num_pages = (int32_t)c->num_pages;
  p.page_shift = __builtin_ctz((unsigned)c->page_size);
  p.max_pages = c->max_pages;
  p.B = c->num_seqs;
  p.HQ = c->num_q_heads;
  p.HK = c->num_kv_heads;
  p.dev_status = c->dev_status;
  return p;
}

// A capped logit is cap - 2 cap / (1 + exp(2 x / cap)): it is off by a few
// roundings of cap, whatever its size.
constexpr float kMaxCap = 1024.0f;

int64_t pool_rows(const lethe_paged_cache* c) { return c->num_pages * c->page_size; }

// A loose bound: no table holds more rows.
int32_t most_rows(const lethe_paged_cache* c, int32_t max_kv_len) {
  const int32_t room = c->max_pages * c->page_size;
  return max_kv_len < room ? max_kv_len : room;
}

lethe_status check_bounds(int64_t q_rows, int32_t max_q_len) {
  if (q_rows < 0 || max_q_len < 0) return LETHE_ERR_INVALID;
  return q_rows > 0x7fffffffLL / LETHE_MAX_AXES ? LETHE_ERR_UNSUPPORTED : LETHE_OK;
}

lethe_status check_rotary(const lethe_rotary* r, int head_dim) {
  if (!r) return LETHE_OK;
  if (!r->inv_freq || !r->axis_pos) return LETHE_ERR_INVALID;
  if (r->num_axes < 1 || r->num_axes > LETHE_MAX_AXES) return LETHE_ERR_INVALID;
  if (r->rot_dim < 16 || r->rot_dim > head_dim || r->rot_dim % 16) return LETHE_ERR_INVALID;
  if (r->adjacent != 0 && r->adjacent != 1) return LETHE_ERR_INVALID;
  int64_t pairs = 0;
  for (int a = 0; a < r->num_axes; ++a) {
    if (r->sections[a] < 0) return LETHE_ERR_INVALID;
    pairs += r->sections[a];
  }
  return pairs == r->rot_dim / 2 ? LETHE_OK : LETHE_ERR_INVALID;
}

size_t evict_count_bytes(const lethe_paged_cache* c) {
  return align_up((size_t)c->num_layers * c->num_seqs * c->num_kv_heads * sizeof(int32_t), 256);
}
// One (destination, source) entry a pool row: the i-th move of a segment is
// kept at the place of its row i, so the pool bounds the list whatever the
// tables could hold.
size_t evict_ws_bytes(const lethe_paged_cache* c) {
  return evict_count_bytes(c) + (size_t)c->num_pages * c->num_kv_heads * c->page_size * sizeof(int2);
}

}  // namespace

extern "C" {

lethe_status lethe_paged_append(const lethe_paged_cache* c, int32_t layer, const void* q, int64_t q_stride,
                                const void* k_new, int64_t k_stride, const void* v_new, int64_t v_stride,
                                const int64_t* q_start, const int32_t* q_len, int64_t q_rows, int32_t max_q_len,
                                const lethe_rotary* rotary, void* q_out, hipStream_t stream) {
  lethe_status st = check_cache(c);
  if (st != LETHE_OK) return st;
  if (!c->score || !c->pos || !c->seen) return LETHE_ERR_INVALID;
  if (layer < 0 || layer >= c->num_layers) return LETHE_ERR_INVALID;
  if (!q_start || !q_len || (q_rows != 0 && (!k_new || !v_new || (q == nullptr) != (q_out == nullptr))))
    return LETHE_ERR_INVALID;
  if (!aligned16(q) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(q_out)) return LETHE_ERR_INVALID;
  st = check_bounds(q_rows, max_q_len);
  if (st != LETHE_OK) return st;
  const int64_t D = c->head_dim;
  if ((q && (q_stride < c->num_q_heads * D || q_stride % 8)) || k_stride < c->num_kv_heads * D || k_stride % 8 ||
      v_stride < c->num_kv_heads * D || v_stride % 8)
    return LETHE_ERR_INVALID;
  st = check_rotary(rotary, c->head_dim);
  if (st != LETHE_OK) return st;
  PagedAppendArgs a;
  a.c = view(c, layer);
  a.q = q;
  a.k_new = k_new;
  a.v_new = v_new;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.q_start = q_start;
  a.q_len = q_len;
  a.q_rows = q_rows;
  a.max_q = max_q_len;
  a.inv_freq = rotary ? rotary->inv_freq : nullptr;
  a.axis_pos = rotary ? rotary->axis_pos : nullptr;
  a.rot = rotary ? rotary->rot_dim : 0;
  a.adjacent = rotary ? rotary->adjacent : 0;
  a.axes = rotary ? rotary->num_axes : 0;
  for (int x = 0, end = 0; x < LETHE_MAX_AXES; ++x) a.ends[x] = x < a.axes ? end += rotary->sections[x] : end;
  a.q_out = q_out;
  return launch_paged_append(a, c->dtype, c->head_dim, stream);
}

size_t lethe_paged_attn_workspace_bytes(const lethe_paged_cache* c, int64_t q_rows, int32_t max_q_len,
                                        int32_t max_kv_len) {
  if (check_desc(c) != LETHE_OK || check_bounds(q_rows, max_q_len) != LETHE_OK || max_kv_len < 0) return 0;
  return paged_attn_ws_bytes(q_rows, max_q_len, most_rows(c, max_kv_len), c->num_seqs, c->num_q_heads, c->num_kv_heads, c->head_dim,
                             pool_rows(c));
}

lethe_status lethe_paged_attn_score(const lethe_paged_cache* c, int32_t layer, const void* q,
                                    const int64_t* q_start, const int32_t* q_len, int64_t q_rows, int32_t max_q_len,
                                    int32_t max_kv_len, float gamma, float softmax_scale, float softcap, void* out,
                                    void* ws, size_t ws_bytes, hipStream_t stream) {
  lethe_status st = check_cache(c);
  if (st != LETHE_OK) return st;
  if (layer < 0 || layer >= c->num_layers) return LETHE_ERR_INVALID;
  if (!q_start || !q_len || !ws || (q_rows != 0 && (!q || !out))) return LETHE_ERR_INVALID;
  if (!aligned16(q) || !aligned16(out)) return LETHE_ERR_INVALID;
  if (((uintptr_t)ws & 255) != 0) return LETHE_ERR_INVALID;
  if (max_kv_len < 0) return LETHE_ERR_INVALID;
  if (!(gamma >= 0.0f && gamma <= 1.0f)) return LETHE_ERR_INVALID;  // also rejects NaN
  if (gamma > 0.0f && (!c->score || !aligned16(c->score))) return LETHE_ERR_INVALID;
  if (isnan(softmax_scale) || isinf(softmax_scale)) return LETHE_ERR_INVALID;
  if (!(softcap >= 0.0f) || isinf(softcap)) return LETHE_ERR_INVALID;
  if (softcap > kMaxCap) return LETHE_ERR_UNSUPPORTED;
  st = check_bounds(q_rows, max_q_len);
  if (st != LETHE_OK) return st;
  if (ws_bytes < lethe_paged_attn_workspace_bytes(c, q_rows, max_q_len, max_kv_len)) return LETHE_ERR_WORKSPACE;
  const float scale = softmax_scale > 0.0f ? softmax_scale : 1.0f / sqrtf((float)c->head_dim);
  constexpr float kLog2e = 1.4426950408889634f;
  PagedAttnArgs a;
  a.c = view(c, layer);
  a.q = q;
  a.q_start = q_start;
  a.q_len = q_len;
  a.q_rows = q_rows;
  a.max_q = max_q_len;
  a.max_kv = most_rows(c, max_kv_len);
  a.G = c->num_q_heads / c->num_kv_heads;
  a.g_magic = a.G > 1 ? (uint32_t)((0xffffffffULL + a.G) / a.G) : 0u;
  a.scale_log2 = scale * kLog2e;
  // Finite, so that a product of 0 stays 0 under the smallest caps.
  a.cap_in = softcap > 0.0f ? fminf(2.0f * scale * kLog2e / softcap, FLT_MAX) : 0.0f;
  a.cap_log2 = softcap * kLog2e;
  a.gamma = gamma;
  a.out = out;
  a.ws = (char*)ws;
  return launch_paged_attn(a, c->dtype, c->head_dim, pool_rows(c), stream);
}

size_t lethe_paged_evict_workspace_bytes(const lethe_paged_cache* c) {
  return check_desc(c) == LETHE_OK ? evict_ws_bytes(c) : 0;
}

lethe_status lethe_paged_evict(const lethe_paged_cache* c, const int32_t* budget, int32_t recent, int32_t sink,
                               int32_t max_kv_len, void* ws, size_t ws_bytes, hipStream_t stream) {
  const lethe_status st = check_cache(c);
  if (st != LETHE_OK) return st;
  if (!c->score || !c->pos || !c->seen || !budget || recent < 0 || sink < 0 || max_kv_len < 0)
    return LETHE_ERR_INVALID;
  if (!ws || ((uintptr_t)ws & 255) != 0) return LETHE_ERR_INVALID;
  if (ws_bytes < evict_ws_bytes(c)) return LETHE_ERR_WORKSPACE;
  PagedEvictArgs a;
  a.c = view(c, 0);
  a.L = c->num_layers;
  a.D = c->head_dim;
  a.budget = budget;
  a.recent = recent;
  a.sink = sink;
  a.max_kv = most_rows(c, max_kv_len);
  a.count = (int32_t*)ws;
  a.moves = (int2*)((char*)ws + evict_count_bytes(c));
  return launch_paged_evict(a, stream);
}

}  // extern "C"
