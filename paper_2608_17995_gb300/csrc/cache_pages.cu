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
// One warp per new token: the sequence by a search of cu_new 32 ways at a time,
// the place from the length, then the token's Hkv rows of keys and of values.
constexpr int kAppendThreads = 256;

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
  const int b = sequence_of(a.cu, a.c.B, t, lane);
  if (b >= a.c.B) return;
  if (a.c.lens[b] > a.c.max_len && lane == 0) raise_status(a.status, AVITS_ERR_PAGE);
  const int len = cache_len(a.c, b);
  const int64_t place = (int64_t)len - ((int64_t)a.cu[b + 1] - t);
  if (place < 0 || place >= len) {
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
  const char* kn = a.k_new + t * a.k_st;
  const char* vn = a.v_new + t * a.v_st;
  const int n = a.c.Hkv * (int)a.pieces.p;
  constexpr int kDeep = 4;
  for (int i0 = lane; i0 < n; i0 += 32 * kDeep) {
    uint4 k[kDeep], v[kDeep];
#pragma unroll
    for (int r = 0; r < kDeep; ++r) {
      const int i = i0 + 32 * r;
      if (i < n) {
        const int h = a.pieces.div(i), c = i - h * (int)a.pieces.p;
        k[r] = ld_once(kn + h * a.k_sh + c * 16);
        v[r] = ld_once(vn + h * a.v_sh + c * 16);
      }
    }
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
// of the row as 32-bit keys whose order is the weights' order (in shared memory
// where they fit).  The keep-th largest key by radix digits of 8 bits: each CTA
// counts its digits, every CTA of the cluster adds up the counts through
// distributed shared memory.  Then the keys above it, and of the equal ones
// the lowest places, are written in order: a thread owns a contiguous run, and
// one scan over runs, CTAs included, gives its first rank.
constexpr int kSelThreads = 512;
constexpr int kSelMaxKeys = 40960;   // keys of a CTA in shared memory (padded by 1/32)

struct Evict {
  avits_kv_cache src, dst;
  int keep, sinks, recent;
  int part;            // keys per CTA
  int run;             // keys per thread
  int in_smem;
  int32_t* idx;
  unsigned int* status;
};

__device__ __forceinline__ uint32_t order_of(float s) {
  if (s != s) return 0u;
  const float c = (s == 0.0f) ? 0.0f : s;
  const uint32_t u = __float_as_uint(c);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ int padded(int i) { return i + (i >> 5); }

__global__ void __launch_bounds__(kSelThreads)
cache_select_kernel(const __grid_constant__ Evict a) {
  extern __shared__ uint32_t s_key[];
  __shared__ uint32_t s_hist[2][256];
  __shared__ uint32_t s_warp[kSelThreads / 32];
  __shared__ uint32_t s_pick[2];      // digit and how many of it are needed
  __shared__ uint32_t s_count[2];     // this CTA's keys above, and equal to, the threshold
  cg::cluster_group cluster = cg::this_cluster();
  pdl_wait_then_trigger();
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  const int ncta = (int)cluster.num_blocks(), me = (int)cluster.block_rank();
  const int bh = blockIdx.x / ncta;
  const int b = bh / a.src.Hkv, h = bh - b * a.src.Hkv;
  if (h == 0 && me == 0 && tid == 0) check_cache_len(a.src, b, a.status);
  const int n = cache_len(a.src, b), m = min(n, a.keep);
  const float* acc = a.src.acc + (int64_t)b * a.src.acc_sb + (int64_t)h * a.src.acc_sh;
  float* acc2 = a.dst.acc + (int64_t)b * a.dst.acc_sb + (int64_t)h * a.dst.acc_sh;
  int32_t* idx = a.idx + (int64_t)bh * a.keep;
  if (h == 0 && me == 0 && tid == 0) a.dst.lens[b] = m;
  // all of them, and the places past the kept ones: the same for every CTA
  if (n <= a.keep) {
    for (int i = me * kSelThreads + tid; i < a.keep; i += ncta * kSelThreads) {
      idx[i] = i < n ? i : -1;
      if (i < n) acc2[i] = acc[i];
    }
    return;   // the whole cluster takes this way
  }
  const int lo = min(n, me * a.part), hi = min(n, lo + a.part);
  const int last = n - a.recent;
  auto key_at = [&](int j) {     // the first and the last ones stand above all
    return j < a.sinks || j >= last ? 0xFFFFFFFFu : order_of(acc[j]);
  };
  auto key = [&](int j) { return a.in_smem ? s_key[padded(j - lo)] : key_at(j); };
  if (a.in_smem)
    for (int j = lo + tid; j < hi; j += kSelThreads) s_key[padded(j - lo)] = key_at(j);

  uint32_t prefix = 0u, mask = 0u, need = (uint32_t)a.keep;
  bool all = false;     // the threshold's whole digit is taken: no ties to count
#pragma unroll 1
  for (int pass = 0; pass < 4; ++pass) {
    const int shift = 24 - 8 * pass;
    uint32_t* hist = s_hist[pass & 1];
    for (int i = tid; i < 256; i += kSelThreads) hist[i] = 0u;
    __syncthreads();
    for (int j = lo + tid; j < hi; j += kSelThreads) {
      const uint32_t k = key(j);
      if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & 255u], 1u);
    }
    cluster.sync();
    // suffix sums of the cluster's counts: thread t < 256 has digit 255 - t
    uint32_t mine = 0u;
    if (tid < 256)
      for (int r = 0; r < ncta; ++r) mine += cluster.map_shared_rank(hist, r)[255 - tid];
    uint32_t inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t y = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += y;
    }
    if (lane == 31) s_warp[w] = inc;
    __syncthreads();
    if (tid < 256) {
      for (int i = 0; i < w; ++i) inc += s_warp[i];
      const uint32_t above = inc - mine;
      if (above < need && need <= inc) {
        s_pick[0] = 255u - tid;
        s_pick[1] = need - above;
        s_count[0] = mine == need - above ? 1u : 0u;
      }
    }
    __syncthreads();
    prefix |= s_pick[0] << shift;
    mask |= 255u << shift;
    need = s_pick[1];
    all = s_count[0] != 0u;
    if (all) break;
  }
  // taken: (key & mask) above the prefix, and of the equal ones the first `need`
  // (all of them where the digit is taken whole)
  const int r0 = lo + tid * a.run, r1 = min(hi, r0 + a.run);
  uint32_t above = 0u, equal = 0u;
  for (int j = r0; j < r1; ++j) {
    const uint32_t k = key(j) & mask;
    above += k > prefix;
    equal += k == prefix;
  }
  uint32_t ia = above, ie = equal;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t ya = __shfl_up_sync(0xffffffffu, ia, o), ye = __shfl_up_sync(0xffffffffu, ie, o);
    if (lane >= o) {
      ia += ya;
      ie += ye;
    }
  }
  __shared__ uint32_t s_a[kSelThreads / 32], s_e[kSelThreads / 32];
  if (lane == 31) {
    s_a[w] = ia;
    s_e[w] = ie;
  }
  __syncthreads();
  uint32_t before_a = ia - above, before_e = ie - equal, sum_a = 0u, sum_e = 0u;
  for (int i = 0; i < kSelThreads / 32; ++i) {
    if (i < w) {
      before_a += s_a[i];
      before_e += s_e[i];
    }
    sum_a += s_a[i];
    sum_e += s_e[i];
  }
  if (tid == 0) {
    s_count[0] = sum_a;
    s_count[1] = sum_e;
  }
  cluster.sync();
  for (int r = 0; r < me; ++r) {
    const uint32_t* other = cluster.map_shared_rank(s_count, r);
    before_a += other[0];
    before_e += other[1];
  }
  for (int j = r0; j < r1; ++j) {
    const uint32_t k = key(j) & mask;
    const bool take = k > prefix || (k == prefix && before_e < need);
    if (take) {
      const uint32_t rank = before_a + min(before_e, need);
      idx[rank] = j;
      acc2[rank] = acc[j];
    }
    before_a += k > prefix;
    before_e += k == prefix;
  }
  cluster.sync();   // no CTA leaves while another reads its counts
}

// Copy: the kept rows, each of Hkv * 2 * pieces 16-byte pieces, flat over the
// threads so that neighbouring lanes read neighbouring pieces of a row.
constexpr int kCopyThreads = 256;
constexpr int kCopyDeep = 4;

struct Copy {
  avits_kv_cache src, dst;
  FastDiv spage, dpage, pieces;
  int keep, es, blocks;      // blocks: per (b, head)
  const int32_t* idx;
  unsigned int* status;
};

__global__ void __launch_bounds__(kCopyThreads)
cache_copy_kernel(const __grid_constant__ Copy a) {
  pdl_wait_then_trigger();
  const int bh = blockIdx.x / a.blocks, part = blockIdx.x - bh * a.blocks;
  const int b = bh / a.src.Hkv, h = bh - b * a.src.Hkv;
  const int m = min(cache_len(a.src, b), a.keep);
  const int32_t* idx = a.idx + (int64_t)bh * a.keep;
  const int32_t* ts = a.src.block_table + (int64_t)b * a.src.table_sb;
  const int32_t* td = a.dst.block_table + (int64_t)b * a.dst.table_sb;
  const int per = 2 * (int)a.pieces.p;
  const int rows = kCopyThreads * kCopyDeep / per;        // rows of a block, >= 8
  const int r0 = part * rows, count = min(rows, m - r0) * per;
  uint4 x[kCopyDeep];
  char* to[kCopyDeep];
#pragma unroll
  for (int q = 0; q < kCopyDeep; ++q) {
    const int i = threadIdx.x + q * kCopyThreads;
    to[q] = nullptr;
    if (i < count) {
      const int half = a.pieces.div(i), row = half >> 1, c = i - half * (int)a.pieces.p;
      const int r = r0 + row, j = idx[r];
      const int cs = a.spage.div(j), cd = a.dpage.div(r);
      const int ps = ts[cs], pd = td[cd];
      if ((unsigned)ps < (unsigned)a.src.num_pages && (unsigned)pd < (unsigned)a.dst.num_pages) {
        const int ss = j - cs * a.src.page_size, sd = r - cd * a.dst.page_size;
        const bool is_v = half & 1;
        const int64_t so = is_v ? ps * a.src.v_sp + ss * a.src.v_st + h * a.src.v_sh
                                : ps * a.src.k_sp + ss * a.src.k_st + h * a.src.k_sh;
        const int64_t dof = is_v ? pd * a.dst.v_sp + sd * a.dst.v_st + h * a.dst.v_sh
                                 : pd * a.dst.k_sp + sd * a.dst.k_st + h * a.dst.k_sh;
        const char* from =
            static_cast<const char*>(is_v ? a.src.v_pages : a.src.k_pages) + so * a.es + c * 16;
        to[q] = static_cast<char*>(is_v ? a.dst.v_pages : a.dst.k_pages) + dof * a.es + c * 16;
        x[q] = ld_once(from);
      } else {
        raise_status(a.status, AVITS_ERR_PAGE);
      }
    }
  }
#pragma unroll
  for (int q = 0; q < kCopyDeep; ++q)
    if (to[q]) *reinterpret_cast<uint4*>(to[q]) = x[q];
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
  return launch_pdl(cache_append_kernel, dim3((unsigned)((T + kWarps - 1) / kWarps)),
                    dim3(kAppendThreads), 0, s, a);
}

cudaError_t launch_cache_evict(const avits_kv_cache& src, const avits_kv_cache& dst, int keep,
                               int sinks, int recent, int32_t* idx, unsigned int* status,
                               cudaStream_t s) {
  Evict a{};
  a.src = src;
  a.dst = dst;
  a.keep = keep;
  a.sinks = sinks;
  a.recent = recent;
  a.idx = idx;
  a.status = status;
  // CTAs per row: 4096 keys each, up to the 8 of a portable cluster
  int ncta = 1;
  while (ncta < 8 && (int64_t)ncta * 4096 < src.max_len) ncta *= 2;
  a.part = (src.max_len + ncta - 1) / ncta;
  a.run = (a.part + kSelThreads - 1) / kSelThreads;
  a.in_smem = a.part <= kSelMaxKeys;
  const size_t smem = a.in_smem ? (size_t)(a.part + a.part / 32 + 1) * 4 : 0;
  cudaError_t e =
      prefer_max_shared<cache_select_kernel, (kSelMaxKeys + kSelMaxKeys / 32 + 1) * 4>();
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(src.B * src.Hkv * ncta));
  cfg.blockDim = dim3(kSelThreads);
  cfg.dynamicSmemBytes = smem;
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
  e = cudaLaunchKernelEx(&cfg, cache_select_kernel, a);
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
  const int rows = kCopyThreads * kCopyDeep / (2 * (src.d * c.es / 16));
  c.blocks = (keep + rows - 1) / rows;
  e = prefer_max_shared<cache_copy_kernel>();
  if (e != cudaSuccess) return e;
  return launch_pdl(cache_copy_kernel, dim3((unsigned)(src.B * src.Hkv * c.blocks)),
                    dim3(kCopyThreads), 0, s, c);
}

}  // namespace avits
