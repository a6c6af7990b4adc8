// cache_common.cuh — the paged key-value cache as the device sees it.
#pragma once

#include "avits_common.cuh"

namespace avits {

// n / p for 0 <= n < 2^31 by a multiplication (Granlund and Montgomery,
// "Division by invariant integers using multiplication"): with s = ceil(log2 p)
// and m = floor(2^32 (2^s - p) / p) + 1, n / p = (hi32(n m) + n) >> s.
struct FastDiv {
  uint32_t m, s, p;
  static FastDiv of(int p) {
    FastDiv f;
    f.p = (uint32_t)p;
    f.s = 0;
    while ((1ull << f.s) < (unsigned long long)p) ++f.s;
    f.m = (uint32_t)((((1ull << f.s) - (uint64_t)p) << 32) / (uint64_t)p + 1ull);
    return f;
  }
  __device__ __forceinline__ int div(int n) const {
    return (int)((__umulhi((uint32_t)n, m) + (uint32_t)n) >> s);
  }
};

// Cached tokens of sequence b.  A length outside [0, max_len] is cut to it:
// nothing past the table's promised part is ever followed.
__device__ __forceinline__ int cache_len(const avits_kv_cache& c, int b) {
  const int n = c.lens[b];
  return min(max(n, 0), c.max_len);
}
__device__ __forceinline__ void check_cache_len(const avits_kv_cache& c, int b, unsigned int* st) {
  const int n = c.lens[b];
  if (n < 0 || n > c.max_len) raise_status(st, AVITS_ERR_PAGE);
}

// Page number of table column col of sequence b, -1 (and the status word) when
// it is not a page of the pool.
__device__ __forceinline__ int checked_page(const avits_kv_cache& c, int page, unsigned int* st) {
  if ((unsigned)page < (unsigned)c.num_pages) return page;
  raise_status(st, AVITS_ERR_PAGE);
  return -1;
}

// The sequence of token t: the number of b in [1, B] with cu[b] <= t, found in
// rounds of 32 probes.  B or more: past the last sequence.
__device__ __forceinline__ int sequence_of(const int32_t* cu, int B, int t, int lane) {
  int lo = 0, n = B;            // the answer lies in [lo, lo + n]
  while (n > 0) {
    const int step = (n + 31) / 32;
    const int at = lo + min((lane + 1) * step, n);     // in [lo+1, lo+n]
    const unsigned below = __ballot_sync(0xffffffffu, cu[at] <= t);
    const int k = __popc(below);                        // probes at or below t
    if (step == 1) return lo + min(k, n);
    const int from = lo + min(k * step, n);
    if (k == 32) return from;
    n = min(step - 1, lo + n - from);
    lo = from;
  }
  return lo;
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// 16 bytes read once: not kept in L1.
__device__ __forceinline__ uint4 ld_once(const void* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}

}  // namespace avits
