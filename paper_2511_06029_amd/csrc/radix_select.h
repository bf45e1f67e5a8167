// Exact selection of the m-th best 32-bit key by a block.
#pragma once

#include "device_common.h"

namespace lethe {

// A float's bits as a word whose unsigned order is the float order.
__device__ inline uint32_t order_key(float f) {
  uint32_t u = __float_as_uint(f);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0u;  // NaN ranks last
  if (u == 0x80000000u) u = 0u;                      // -0 ties with +0
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

struct RadixShared {
  uint32_t hist[2][256];
  uint32_t digit, need, count;
};

// MSB-first radix select over candidates that `count_digits(hist, shift,
// prefix, pmask)` counts by the 8-bit digit at `shift` (those whose bits under
// pmask equal prefix): key T of the m-th best (m >= 1), how many candidates
// with key T belong to the best m, and how many have it; all threads get the
// three.  A digit whose candidates are all needed ends the search: T is then
// the lowest key of that digit, and the two counts are equal.  With keys that
// spread (accumulated attention) two or three of the four passes run.  `top`: the shift
// of the first digit, for keys that have no bit above it (24: 32-bit keys).
// Bound by latency: two barriers a pass, the next histogram cleared while the
// first wave searches this one (five barriers and always four passes took 91 us
// for the 32768 segments of a batch-128 round, 1024 to 65536 rows at shares of
// 2% to 20%; this, 79 us).
template <int NT, class CountFn>
__device__ void radix_select(const CountFn& count_digits, uint32_t m, RadixShared& sh, uint32_t* T_out,
                             uint32_t* need_out, uint32_t* count_out, int top = 24) {
  const int tid = threadIdx.x;
  uint32_t prefix = 0, pmask = 0, need = m, count = 0;
  if (tid < 256) sh.hist[0][tid] = 0;
  __syncthreads();
  int cur = 0;
  for (int shift = top; shift >= 0; shift -= 8, cur ^= 1) {
    count_digits(sh.hist[cur], shift, prefix, pmask);
    __syncthreads();
    if (tid < kWave) {
      // suffix[d] = matching keys whose digit is >= d: four bins a lane; the
      // digit is the largest one whose suffix reaches need.
      const uint32_t h0 = sh.hist[cur][4 * tid], h1 = sh.hist[cur][4 * tid + 1];
      const uint32_t h2 = sh.hist[cur][4 * tid + 2], h3 = sh.hist[cur][4 * tid + 3];
      const uint32_t tot = h0 + h1 + h2 + h3;
      uint32_t incl = tot;  // sum over lanes tid .. 63
      for (int o = 1; o < kWave; o <<= 1) {
        const uint32_t v = __shfl_down(incl, o);
        if (tid + o < kWave) incl += v;
      }
      const uint32_t s4 = incl - tot, s3 = s4 + h3, s2 = s3 + h2, s1 = s2 + h1;
      if (incl >= need && s4 < need) {
        const int d = s3 >= need ? 3 : s2 >= need ? 2 : s1 >= need ? 1 : 0;
        sh.digit = (uint32_t)(4 * tid + d);
        sh.need = need - (d == 3 ? s4 : d == 2 ? s3 : d == 1 ? s2 : s1);
        sh.count = d == 3 ? h3 : d == 2 ? h2 : d == 1 ? h1 : h0;
      }
    }
    // The other histogram, for the next pass (by the last threads: the first
    // wave is busy).
    if (tid >= NT - 256) sh.hist[cur ^ 1][tid - (NT - 256)] = 0;
    __syncthreads();
    prefix |= sh.digit << shift;
    pmask |= 255u << shift;
    need = sh.need;
    count = sh.count;
    if (need == count) break;
  }
  *T_out = prefix;
  *need_out = need;
  *count_out = count;
}

}  // namespace lethe
