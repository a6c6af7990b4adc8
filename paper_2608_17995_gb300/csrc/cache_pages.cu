// cache_pages.cu — what moves a paged key-value cache's tokens: new ones into
// their pages, and eviction by accumulated attention weight.  Both move whole
// token rows of 16-byte pieces; the bytes bound them.
#include <cooperative_groups.h>

#include "cache_common.cuh"
#include "avits_internal.h"

namespace cg = cooperative_groups;

namespace avits {
namespace {

// ----------------------------------------------------------------- append --
// One warp per new token: its first pieces are on their way while the sequence is
// found by a search of cu_new 32 ways at a time, and the place from the length;
// then the token's Hkv rows of keys and of values go there.  A step's 64 tokens take
// 2.3 us, a launch and three dependent reads (2.7 with 8 warps to a CTA); prompts are
// bound by HBM, 43 us where their bytes take 36 at a copy's rate.
constexpr int kAppendThreads = 128;

struct Append {
  avits_kv_cache c;
  FastDiv page, pieces;     // pieces: 16-byte pieces of a row
  const char* k_new;
  const char* v_new;
  const int32_t* cu;
  int64_t k_st, k_sh, v_st, v_sh;   // bytes
  int T, es;
  unsigned int* status;
};

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

__global__ void __launch_bounds__(kAppendThreads)
cache_append_kernel(const __grid_constant__ Append a) {
  pdl_wait_then_trigger();
  const int lane = threadIdx.x & 31;
  const int t = blockIdx.x * (kAppendThreads / 32) + (threadIdx.x >> 5);
  if (t >= a.T) return;
  const char* kn = a.k_new + t * a.k_st;
  const char* vn = a.v_new + t * a.v_st;
  const int n = a.c.Hkv * (int)a.pieces.p;
  constexpr int kDeep = 4;
  uint4 k[kDeep], v[kDeep];
  auto load = [&](int i0) {
#pragma unroll
    for (int r = 0; r < kDeep; ++r) {
      const int i = i0 + 32 * r;
      if (i < n) {
        const int h = a.pieces.div(i), c = i - h * (int)a.pieces.p;
        k[r] = ld_once(kn + h * a.k_sh + c * 16);
        v[r] = ld_once(vn + h * a.v_sh + c * 16);
      }
    }
  };
  load(lane);
  const int b = sequence_of(a.cu, a.c.B, t, lane);
  if (b >= a.c.B) return;
  // by the length as it is: cut to max_len, it would put tokens past the capacity over
  // cached ones
  const int len = a.c.lens[b];
  if (len > a.c.max_len && lane == 0) raise_status(a.status, AVITS_ERR_PAGE);
  const int64_t place = (int64_t)len - ((int64_t)a.cu[b + 1] - t);
  if (place < 0 || place >= min(len, a.c.max_len)) {
    if (lane == 0) raise_status(a.status, AVITS_ERR_PAGE);
    return;
  }
  const int j = (int)place, col = a.page.div(j), slot = j - col * a.c.page_size;
  if (a.c.acc)
    for (int h = lane; h < a.c.Hkv; h += 32)
      a.c.acc[(int64_t)b * a.c.acc_sb + (int64_t)h * a.c.acc_sh + j] = 0.f;
  const int page = a.c.block_table[(int64_t)b * a.c.table_sb + col];
  if ((unsigned)page >= (unsigned)a.c.num_pages) {
    if (lane == 0) raise_status(a.status, AVITS_ERR_PAGE);
    return;
  }
  char* kp = static_cast<char*>(a.c.k_pages) + ((int64_t)page * a.c.k_sp + slot * a.c.k_st) * a.es;
  char* vp = static_cast<char*>(a.c.v_pages) + ((int64_t)page * a.c.v_sp + slot * a.c.v_st) * a.es;
  for (int i0 = lane; i0 < n; i0 += 32 * kDeep) {
    if (i0 != lane) load(i0);
#pragma unroll
    for (int r = 0; r < kDeep; ++r) {
      const int i = i0 + 32 * r;
      if (i < n) {
        const int h = a.pieces.div(i), c = i - h * (int)a.pieces.p;
        *reinterpret_cast<uint4*>(kp + h * a.c.k_sh * a.es + c * 16) = k[r];
        *reinterpret_cast<uint4*>(vp + h * a.c.v_sh * a.es + c * 16) = v[r];
      }
    }
  }
}

// ------------------------------------------------------------------ evict --
// Selection: a cluster of CTAs per (b, KV head), each with a contiguous part
// of the row, a thread with runs of 8 or 16 weights in registers, seen as 32-bit
// keys whose order is the weights' order.  The keep-th largest key by radix digits
// of 8 bits: each CTA counts its digits and adds the counts to the first CTA's
// table (distributed shared memory), from which every CTA finds the digit.  Then
// the keys above it, and of the equal ones the lowest places, in order: a scan over
// the runs, CTAs included, gives each its first rank.
//
// The cost is latency: a barrier over a cluster takes 1-2 thousand cycles, one of
// a CTA a tenth of it, and counting goes with a CTA's keys.  8 rows of 1024 keys
// take 4 us, of 4096 5, of 131072 20; 192 of up to 4096 keys 12.
constexpr int kSelMaxThreads = 1024;
constexpr int kSelMaxCluster = 8;

struct Evict {
  avits_kv_cache src, dst;
  int keep, sinks, recent;
  int part;            // keys per CTA, a multiple of 16
  int32_t* idx;
  unsigned int* status;
};

__device__ __forceinline__ uint32_t order_of(float s) {
  if (s != s) return 0u;
  const float c = (s == 0.0f) ? 0.0f : s;
  const uint32_t u = __float_as_uint(c);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// Sums of two counts over the threads before this one, and over all.
__device__ __forceinline__ void block_scan(uint32_t x, uint32_t y, uint2* s_warp, int lane, int w,
                                           int warps, uint32_t& bx, uint32_t& by, uint32_t& tx,
                                           uint32_t& ty) {
  uint32_t ix = x, iy = y;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t ux = __shfl_up_sync(0xffffffffu, ix, o), uy = __shfl_up_sync(0xffffffffu, iy, o);
    if (lane >= o) {
      ix += ux;
      iy += uy;
    }
  }
  if (lane == 31) s_warp[w] = make_uint2(ix, iy);
  __syncthreads();
  // every warp scans the warps' counts itself
  const uint2 own = lane < warps ? s_warp[lane] : make_uint2(0u, 0u);
  uint32_t wx = own.x, wy = own.y;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t ux = __shfl_up_sync(0xffffffffu, wx, o), uy = __shfl_up_sync(0xffffffffu, wy, o);
    if (lane >= o) {
      wx += ux;
      wy += uy;
    }
  }
  tx = __shfl_sync(0xffffffffu, wx, 31);
  ty = __shfl_sync(0xffffffffu, wy, 31);
  bx = __shfl_sync(0xffffffffu, wx - own.x, w) + ix - x;
  by = __shfl_sync(0xffffffffu, wy - own.y, w) + iy - y;
}

template <int kRun>
__global__ void __launch_bounds__(kSelMaxThreads)
cache_select_kernel(const __grid_constant__ Evict a) {
  __shared__ __align__(16) uint32_t s_total[4][256];   // of the cluster, in its first CTA
  __shared__ __align__(16) uint32_t s_hist[2][256];    // of this CTA
  __shared__ uint32_t s_pick[3];      // digit, how many of it are needed, whether all are
  __shared__ uint2 s_count[kSelMaxCluster];   // the CTAs' keys above, and equal to, the threshold
  __shared__ uint2 s_warp[2][32];
  cg::cluster_group cluster = cg::this_cluster();
  const int ncta = (int)cluster.num_blocks(), me = (int)cluster.block_rank();
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, threads = blockDim.x;
  for (int i = tid; i < 1024; i += threads) (&s_total[0][0])[i] = 0u;
  for (int i = tid; i < 512; i += threads) (&s_hist[0][0])[i] = 0u;
  // the first CTA's table is zero once this barrier is waited for
  if (ncta > 1) cluster.barrier_arrive();
  pdl_wait();
  const int bh = blockIdx.x / ncta;
  const int b = bh / a.src.Hkv, h = bh - b * a.src.Hkv;
  if (h == 0 && me == 0 && tid == 0) check_cache_len(a.src, b, a.status);
  const int n = cache_len(a.src, b), m = min(n, a.keep);
  const float* acc = a.src.acc + (int64_t)b * a.src.acc_sb + (int64_t)h * a.src.acc_sh;
  int32_t* idx = a.idx + (int64_t)bh * a.keep;
  if (h == 0 && me == 0 && tid == 0) a.dst.lens[b] = m;
  // all of them, and the places past the kept ones: the same for every CTA
  if (n <= a.keep) {
    for (int i = me * threads + tid; i < a.keep; i += ncta * threads) idx[i] = i < n ? i : -1;
    if (ncta > 1) cluster.barrier_wait();
    return;   // the whole cluster takes this way
  }
  const int lo = min(n, me * a.part), hi = min(n, lo + a.part);
  const int last = n - a.recent, stripe = threads * kRun;
  const bool vec = (reinterpret_cast<uintptr_t>(acc) & 15u) == 0;   // lo is a multiple of 4
  uint32_t k[kRun];
  int here;                // keys of the run that are in the part: the first ones
  // this thread's run of a stripe; a part of one stripe is read once, here
  auto load_keys = [&](int j0) {
    float x[kRun];
    here = min(max(hi - j0, 0), kRun);
    if (vec && here == kRun) {
#pragma unroll
      for (int i = 0; i < kRun; i += 4) {
        const float4 p = *reinterpret_cast<const float4*>(acc + j0 + i);
        x[i] = p.x; x[i + 1] = p.y; x[i + 2] = p.z; x[i + 3] = p.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < kRun; ++i) x[i] = i < here ? acc[j0 + i] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < kRun; ++i)       // the first and the last ones stand above all
      k[i] = j0 + i < a.sinks || j0 + i >= last ? 0xFFFFFFFFu : order_of(x[i]);
  };
  const int j1 = lo + tid * kRun;
  const bool again = hi - lo > stripe;
  load_keys(j1);
  __syncthreads();

  uint32_t prefix = 0u, mask = 0u, need = (uint32_t)a.keep;
#pragma unroll 1
  for (int pass = 0; pass < 4; ++pass) {
    const int shift = 24 - 8 * pass;
    uint32_t* hist = s_hist[pass & 1];
    // (the first digit is one of few; a table per group of lanes was no faster, nor
    // where all weights are equal)
    for (int j0 = j1; j0 < hi; j0 += stripe) {
      if (again) load_keys(j0);
#pragma unroll
      for (int i = 0; i < kRun; ++i)
        if (i < here && (k[i] & mask) == prefix) atomicAdd(&hist[(k[i] >> shift) & 255u], 1u);
    }
    __syncthreads();
    if (ncta > 1) {
      if (pass == 0) cluster.barrier_wait();
      uint32_t* to = cluster.map_shared_rank(s_total[pass], 0);
      for (int i = tid; i < 256; i += threads)
        if (hist[i]) atomicAdd(&to[i], hist[i]);
      cluster.sync();
    }
    if (w == 0) {
      // lane l adds up digits 255 - 8 l down to 248 - 8 l; then lanes 0-7 take one
      // digit each of those that hold the needed one
      const uint32_t* table = ncta > 1 ? cluster.map_shared_rank(s_total[pass], 0) : hist;
      const uint4* at = reinterpret_cast<const uint4*>(table) + 2 * (31 - lane);
      const uint4 p = at[0], q = at[1];
      const uint32_t sum = ((p.x + p.y) + (p.z + p.w)) + ((q.x + q.y) + (q.z + q.w));
      uint32_t upto = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += y;
      }
      const int from = __ffs(__ballot_sync(0xffffffffu, upto >= need)) - 1;
      const uint32_t rest = need - __shfl_sync(0xffffffffu, upto - sum, from);
      const int digit = 255 - 8 * from - (lane & 7);
      const uint32_t c = table[digit];
      uint32_t to = c;
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, to, o);
        if (lane >= o) to += y;
      }
      if (lane < 8 && to - c < rest && rest <= to) {
        s_pick[0] = (uint32_t)digit;
        s_pick[1] = rest - (to - c);
        s_pick[2] = to == rest;
      }
    } else if (pass > 0) {
      // the other table was last read two barriers ago
      for (int i = tid - 32; i < 256; i += threads - 32) s_hist[(pass & 1) ^ 1][i] = 0u;
    }
    __syncthreads();
    prefix |= s_pick[0] << shift;
    mask |= 255u << shift;
    need = s_pick[1];
    if (s_pick[2]) break;     // the digit is taken whole: no ties to count
  }
  // taken: (key & mask) above the prefix, and of the equal ones the first `need`
  const int warps = threads >> 5;
  uint32_t above = 0u, equal = 0u;
  for (int j0 = j1; j0 < hi; j0 += stripe) {
    if (again) load_keys(j0);
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
      above += i < here && (k[i] & mask) > prefix;
      equal += i < here && (k[i] & mask) == prefix;
    }
  }
  uint32_t bx, by, tx, ty;      // of the threads before, of all
  block_scan(above, equal, s_warp[0], lane, w, warps, bx, by, tx, ty);
  uint32_t base_a = 0u, base_e = 0u;      // of the CTAs before this one
  if (ncta > 1) {
    // told to every CTA, so that nothing of this one is read after the barrier
    if (tid < ncta) cluster.map_shared_rank(s_count, tid)[me] = make_uint2(tx, ty);
    cluster.sync();
    for (int r = 0; r < me; ++r) {
      base_a += s_count[r].x;
      base_e += s_count[r].y;
    }
  }
  int par = 1;
  for (int s0 = lo; s0 < hi; s0 += stripe, par ^= 1) {      // the same for all threads
    const int j0 = s0 + tid * kRun;
    if (again) {
      load_keys(j0);
      above = equal = 0u;
#pragma unroll
      for (int i = 0; i < kRun; ++i) {
        above += i < here && (k[i] & mask) > prefix;
        equal += i < here && (k[i] & mask) == prefix;
      }
      block_scan(above, equal, s_warp[par], lane, w, warps, bx, by, tx, ty);
    }
    uint32_t ra = base_a + bx, re = base_e + by;
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
      const uint32_t kk = k[i] & mask;
      if (i < here) {
        if (kk > prefix || (kk == prefix && re < need)) idx[ra + min(re, need)] = j0 + i;
        ra += kk > prefix;
        re += kk == prefix;
      }
    }
    base_a += tx;
    base_e += ty;
  }
  pdl_trigger();
}

// Copy: a block takes rows of one (b, head), 8 KB of keys and values.  First
// where each row lies on both sides, and its weight, then the 16-byte pieces flat
// over the threads, neighbouring lanes on neighbouring pieces, 4 to a thread at
// once, so that a block's bytes are all on their way before the first is stored.
// HBM bounds it: 24 x 8 heads x 1024 rows of 512 bytes 30 us (27.4 at a copy's rate),
// 8 x 16384 22 (19.8).  Larger blocks leave calls of few rows on few SMs: 16 KB (256
// threads) 24 x <= 4096 41.7 us a call, 8 x 512 rows 7.2; 32 KB 42.1 and 7.8; 8 KB
// 41.2 and 7.2; 8 KB as 2 pieces to each of 256 threads 43.4 and 7.2.
constexpr int kCopyThreads = 128;
constexpr int kCopyDeep = 4;
constexpr int kCopyPieces = kCopyThreads * kCopyDeep;
constexpr int kCopyRows = kCopyPieces / 2;       // of a block, at most: rows of one piece

struct Copy {
  avits_kv_cache src, dst;
  FastDiv spage, dpage, pieces;
  int keep, es, blocks, rows;      // blocks: per (b, head); rows: of a block
  const int32_t* idx;
  unsigned int* status;
};

__global__ void __launch_bounds__(kCopyThreads)
cache_copy_kernel(const __grid_constant__ Copy a) {
  __shared__ const char* s_from[2 * kCopyRows];    // [row][keys, values]
  __shared__ char* s_to[2 * kCopyRows];            // nullptr: a page out of range
  pdl_wait();
  const int bh = blockIdx.x / a.blocks, part = blockIdx.x - bh * a.blocks;
  const int b = bh / a.src.Hkv, h = bh - b * a.src.Hkv, tid = threadIdx.x;
  const int m = min(cache_len(a.src, b), a.keep), r0 = part * a.rows;
  const int rows = min(a.rows, m - r0);
  if (rows <= 0) return;
  const int32_t* idx = a.idx + (int64_t)bh * a.keep;
  const float* acc = a.src.acc + (int64_t)b * a.src.acc_sb + (int64_t)h * a.src.acc_sh;
  float* acc2 = a.dst.acc + (int64_t)b * a.dst.acc_sb + (int64_t)h * a.dst.acc_sh;
  const int32_t* ts = a.src.block_table + (int64_t)b * a.src.table_sb;
  const int32_t* td = a.dst.block_table + (int64_t)b * a.dst.table_sb;
  for (int i = tid; i < rows; i += kCopyThreads) {
    const int r = r0 + i, cd = a.dpage.div(r), pd = td[cd];
    const int j = idx[r], cs = a.spage.div(j), ps = ts[cs];
    acc2[r] = acc[j];
    const int ss = j - cs * a.src.page_size, sd = r - cd * a.dst.page_size;
    const bool ok = (unsigned)ps < (unsigned)a.src.num_pages &&
                    (unsigned)pd < (unsigned)a.dst.num_pages;
    if (!ok) raise_status(a.status, AVITS_ERR_PAGE);
    s_from[2 * i] = static_cast<const char*>(a.src.k_pages) +
                    (ps * a.src.k_sp + ss * a.src.k_st + h * a.src.k_sh) * a.es;
    s_from[2 * i + 1] = static_cast<const char*>(a.src.v_pages) +
                        (ps * a.src.v_sp + ss * a.src.v_st + h * a.src.v_sh) * a.es;
    s_to[2 * i] = !ok ? nullptr
                      : static_cast<char*>(a.dst.k_pages) +
                            (pd * a.dst.k_sp + sd * a.dst.k_st + h * a.dst.k_sh) * a.es;
    s_to[2 * i + 1] = !ok ? nullptr
                          : static_cast<char*>(a.dst.v_pages) +
                                (pd * a.dst.v_sp + sd * a.dst.v_st + h * a.dst.v_sh) * a.es;
  }
  __syncthreads();
  const int count = rows * 2 * (int)a.pieces.p;
  uint4 x[kCopyDeep];
  char* to[kCopyDeep];
#pragma unroll
  for (int q = 0; q < kCopyDeep; ++q) {
    const int i = tid + q * kCopyThreads;
    to[q] = nullptr;
    if (i < count) {
      const int half = a.pieces.div(i), at = (i - half * (int)a.pieces.p) * 16;
      if (s_to[half]) {
        to[q] = s_to[half] + at;
        x[q] = ld_once(s_from[half] + at);
      }
    }
  }
#pragma unroll
  for (int q = 0; q < kCopyDeep; ++q)
    if (to[q]) *reinterpret_cast<uint4*>(to[q]) = x[q];
  // here and not at the start: blocks that only wait cost the ones that work (24 x <=
  // 4096 tokens 41.2 us with both kernels' triggers at the start, 40.8 so)
  pdl_trigger();
}

}  // namespace

cudaError_t launch_cache_append(const avits_kv_cache& c, const void* k_new, const void* v_new,
                                int T, const int32_t* cu, int64_t k_st, int64_t k_sh, int64_t v_st,
                                int64_t v_sh, unsigned int* status, cudaStream_t s) {
  Append a{};
  a.c = c;
  a.es = c.dt == AVITS_BF16 ? 2 : 4;
  a.page = FastDiv::of(c.page_size);
  a.pieces = FastDiv::of(c.d * a.es / 16);
  a.k_new = static_cast<const char*>(k_new);
  a.v_new = static_cast<const char*>(v_new);
  a.cu = cu;
  a.k_st = k_st * a.es; a.k_sh = k_sh * a.es; a.v_st = v_st * a.es; a.v_sh = v_sh * a.es;
  a.T = T;
  a.status = status;
  const cudaError_t e = prefer_max_shared<cache_append_kernel>();
  if (e != cudaSuccess) return e;
  constexpr int kWarps = kAppendThreads / 32;
  return launch_pdl(cache_append_kernel, dim3((unsigned)((T - 1) / kWarps + 1)),
                    dim3(kAppendThreads), 0, s, a);
}

cudaError_t launch_cache_evict(const avits_kv_cache& src, const avits_kv_cache& dst, int keep,
                               int sinks, int recent, int32_t* idx, int num_sms,
                               unsigned int* status, cudaStream_t s) {
  Evict a{};
  a.src = src;
  a.dst = dst;
  a.keep = keep;
  a.sinks = sinks;
  a.recent = recent;
  a.idx = idx;
  a.status = status;
  // CTAs of a row: while there are SMs for them, as many as leave 4096 keys to each
  // (whole calls, 8 rows of 4096 keys: 9.5 us, with 2048 each 10.9; of 16384: 15.2, with
  // 8192 each 17.0, on one CTA 18.1).  Past 16 keys to a thread, which are read again
  // at each digit, a row is cut whatever the SMs.  Threads have runs of 8 keys (8 x 1024:
  // 7.0 us, of 16 8.3) while 1024 of them reach (8 x 131072: 42.8 with 16, 52.3 with 8).
  const long long bh = (long long)src.B * src.Hkv;
  int ncta = 1;
  while (ncta < kSelMaxCluster && (int64_t)ncta * 4096 < src.max_len &&
         (bh * ncta * 2 <= num_sms || (int64_t)ncta * kSelMaxThreads * 16 < src.max_len))
    ncta *= 2;
  a.part = ((src.max_len + ncta - 1) / ncta + 15) / 16 * 16;
  const int run = a.part <= 8 * kSelMaxThreads ? 8 : 16;
  int threads = (a.part / run + 31) / 32 * 32;
  threads = threads < 64 ? 64 : threads > kSelMaxThreads ? kSelMaxThreads : threads;
  const auto kernel = run == 8 ? cache_select_kernel<8> : cache_select_kernel<16>;
  cudaError_t e = run == 8 ? prefer_max_shared<cache_select_kernel<8>>()
                           : prefer_max_shared<cache_select_kernel<16>>();
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(src.B * src.Hkv * ncta));
  cfg.blockDim = dim3((unsigned)threads);
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)ncta;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  e = cudaLaunchKernelEx(&cfg, kernel, a);
  if (e != cudaSuccess) return e;
  Copy c{};
  c.src = src;
  c.dst = dst;
  c.es = src.dt == AVITS_BF16 ? 2 : 4;
  c.spage = FastDiv::of(src.page_size);
  c.dpage = FastDiv::of(dst.page_size);
  c.pieces = FastDiv::of(src.d * c.es / 16);
  c.keep = keep;
  c.idx = idx;
  c.status = status;
  c.rows = kCopyPieces / (2 * (src.d * c.es / 16));
  c.blocks = (keep + c.rows - 1) / c.rows;
  e = prefer_max_shared<cache_copy_kernel>();
  if (e != cudaSuccess) return e;
  return launch_pdl(cache_copy_kernel, dim3((unsigned)(src.B * src.Hkv * c.blocks)),
                    dim3(kCopyThreads), 0, s, c);
}

}  // namespace avits
