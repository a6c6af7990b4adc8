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
// of the row, seen as 32-bit keys whose order is the weights' order and kept in
// shared memory where they fit.  The keep-th largest key by radix digits of 8
// bits: each CTA counts its digits, one warp of every CTA adds up the cluster's
// counts through distributed shared memory.  Then the keys above it, and of the
// equal ones the lowest places, in order: a thread owns a contiguous run, one scan
// over runs, CTAs included, gives its first rank, and the CTA's places go out
// through a list in shared memory, side by side.
constexpr int kSelMaxThreads = 1024;
constexpr int kSelMaxKeys = 32768;   // of a CTA in shared memory

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

__host__ __device__ __forceinline__ int padded(int i) { return i + (i >> 5); }

__global__ void __launch_bounds__(kSelMaxThreads)
cache_select_kernel(const __grid_constant__ Evict a) {
  extern __shared__ uint32_t s_key[];                // [padded(part)], then the list
  __shared__ __align__(16) uint32_t s_hist[2][256];
  __shared__ uint32_t s_pick[3];      // digit, how many of it are needed, whether all are
  __shared__ uint32_t s_count[2];     // this CTA's keys above, and equal to, the threshold
  __shared__ uint32_t s_a[32], s_e[32];
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, threads = blockDim.x;
  for (int i = tid; i < 512; i += threads) (&s_hist[0][0])[i] = 0u;
  pdl_wait_then_trigger();
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
    for (int i = me * threads + tid; i < a.keep; i += ncta * threads) {
      idx[i] = i < n ? i : -1;
      if (i < n) acc2[i] = acc[i];
    }
    return;   // the whole cluster takes this way
  }
  const int lo = min(n, me * a.part), hi = min(n, lo + a.part);
  const int last = n - a.recent;
  auto key_of = [&](int j, float x) {     // the first and the last ones stand above all
    return j < a.sinks || j >= last ? 0xFFFFFFFFu : order_of(x);
  };
  if (a.in_smem) {
    constexpr int kDeep = 8;      // loads on their way at once
    for (int j0 = lo + tid; j0 < hi; j0 += kDeep * threads) {
      float x[kDeep];
#pragma unroll
      for (int i = 0; i < kDeep; ++i) x[i] = acc[min(j0 + i * threads, hi - 1)];
#pragma unroll
      for (int i = 0; i < kDeep; ++i)
        if (j0 + i * threads < hi)
          s_key[padded(j0 + i * threads - lo)] = key_of(j0 + i * threads, x[i]);
    }
  }
  auto key = [&](int j) { return a.in_smem ? s_key[padded(j - lo)] : key_of(j, acc[j]); };
  __syncthreads();

  uint32_t prefix = 0u, mask = 0u, need = (uint32_t)a.keep;
#pragma unroll 1
  for (int pass = 0; pass < 4; ++pass) {
    const int shift = 24 - 8 * pass;
    uint32_t* hist = s_hist[pass & 1];
    if (pass == 0) {
      // the top digits are few: one count per digit and warp
      for (int j0 = lo; j0 < hi; j0 += threads) {
        const int j = j0 + tid;
        const uint32_t d = j < hi ? key(j) >> 24 : 256u;
        const unsigned same = __match_any_sync(0xffffffffu, d);
        if (j < hi && lane == __ffs(same) - 1) atomicAdd(&hist[d], (uint32_t)__popc(same));
      }
    } else {
#pragma unroll 4
      for (int j = lo + tid; j < hi; j += threads) {
        const uint32_t k = key(j);
        if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & 255u], 1u);
      }
    }
    cluster.sync();
    // the other table was last read before this barrier
    for (int i = tid; i < 256; i += threads) s_hist[(pass & 1) ^ 1][i] = 0u;
    if (w == 0) {
      // lane l: digits 255 - 8 l down to 248 - 8 l, over the cluster
      uint32_t c[8] = {};
      for (int r = 0; r < ncta; ++r) {
        const uint4* other =
            reinterpret_cast<const uint4*>(cluster.map_shared_rank(hist, r)) + 2 * (31 - lane);
        const uint4 x = other[0], y = other[1];
        c[7] += x.x; c[6] += x.y; c[5] += x.z; c[4] += x.w;
        c[3] += y.x; c[2] += y.y; c[1] += y.z; c[0] += y.w;
      }
      uint32_t sum = 0u;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += c[i];
      uint32_t above = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, above, o);
        if (lane >= o) above += y;
      }
      above -= sum;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (above < need && need <= above + c[i]) {
          s_pick[0] = 255u - 8u * lane - i;
          s_pick[1] = need - above;
          s_pick[2] = c[i] == need - above;
        }
        above += c[i];
      }
    }
    __syncthreads();
    prefix |= s_pick[0] << shift;
    mask |= 255u << shift;
    need = s_pick[1];
    if (s_pick[2]) break;     // the digit is taken whole: no ties to count
  }
  // taken: (key & mask) above the prefix, and of the equal ones the first `need`
  const int r0 = lo + tid * a.run, r1 = min(hi, r0 + a.run);
  uint32_t above = 0u, equal = 0u;
#pragma unroll 4
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
  if (lane == 31) {
    s_a[w] = ia;
    s_e[w] = ie;
  }
  __syncthreads();
  // every warp scans the warps' counts itself
  const int warps = threads >> 5;
  uint32_t wa = lane < warps ? s_a[lane] : 0u, we = lane < warps ? s_e[lane] : 0u;
  const uint32_t own_a = wa, own_e = we;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t ya = __shfl_up_sync(0xffffffffu, wa, o), ye = __shfl_up_sync(0xffffffffu, we, o);
    if (lane >= o) {
      wa += ya;
      we += ye;
    }
  }
  const uint32_t sum_a = __shfl_sync(0xffffffffu, wa, 31), sum_e = __shfl_sync(0xffffffffu, we, 31);
  uint32_t before_a = __shfl_sync(0xffffffffu, wa - own_a, w) + ia - above;
  uint32_t before_e = __shfl_sync(0xffffffffu, we - own_e, w) + ie - equal;
  uint32_t base_a = 0u, base_e = 0u;      // of the CTAs before this one
  if (ncta > 1) {
    if (tid == 0) {
      s_count[0] = sum_a;
      s_count[1] = sum_e;
    }
    cluster.sync();
    for (int r = 0; r < me; ++r) {
      const uint32_t* other = cluster.map_shared_rank(s_count, r);
      base_a += other[0];
      base_e += other[1];
    }
  }
  // ranks: of the row, from the CTA's first on
  const uint32_t base = base_a + min(base_e, need);
  const uint32_t count = base_a + sum_a + min(base_e + sum_e, need) - base;
  uint16_t* list = reinterpret_cast<uint16_t*>(s_key + padded(a.part) + 1);
  before_a += base_a;
  before_e += base_e;
  for (int j = r0; j < r1; ++j) {
    const uint32_t k = key(j) & mask;
    if (k > prefix || (k == prefix && before_e < need)) {
      const uint32_t rank = before_a + min(before_e, need);
      if (a.in_smem) {
        list[rank - base] = (uint16_t)(j - lo);
      } else {
        idx[rank] = j;
        acc2[rank] = acc[j];
      }
    }
    before_a += k > prefix;
    before_e += k == prefix;
  }
  if (a.in_smem) {
    __syncthreads();
#pragma unroll 4
    for (uint32_t i = tid; i < count; i += threads) {
      const int j = lo + list[i];
      idx[base + i] = j;
      acc2[base + i] = acc[j];
    }
  }
  if (ncta > 1) cluster.sync();   // no CTA leaves while another reads its counts
}

// Copy: a block takes rows of one (b, head), 32 KB of keys and values.  First
// where each row lies on both sides, then the 16-byte pieces flat over the
// threads, neighbouring lanes on neighbouring pieces, 8 to a thread at once.
constexpr int kCopyThreads = 256;
constexpr int kCopyDeep = 8;
constexpr int kCopyPieces = kCopyThreads * kCopyDeep;
constexpr int kCopyRows = 256;       // of a block, at most

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
  pdl_wait_then_trigger();
  const int bh = blockIdx.x / a.blocks, part = blockIdx.x - bh * a.blocks;
  const int b = bh / a.src.Hkv, h = bh - b * a.src.Hkv, tid = threadIdx.x;
  const int m = min(cache_len(a.src, b), a.keep), r0 = part * a.rows;
  const int rows = min(a.rows, m - r0);
  if (rows <= 0) return;
  const int32_t* idx = a.idx + (int64_t)bh * a.keep;
  const int32_t* ts = a.src.block_table + (int64_t)b * a.src.table_sb;
  const int32_t* td = a.dst.block_table + (int64_t)b * a.dst.table_sb;
  for (int i = tid; i < rows; i += kCopyThreads) {
    const int r = r0 + i, cd = a.dpage.div(r), pd = td[cd];
    const int j = idx[r], cs = a.spage.div(j), ps = ts[cs];
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
  // CTAs of a row: enough for 4096 keys each, and while there are SMs for all of
  // them down to 512, up to the 8 of a portable cluster
  const long long bh = (long long)src.B * src.Hkv;
  int ncta = 1;
  while (ncta < 8 && ((int64_t)ncta * 4096 < src.max_len ||
                      (bh * ncta * 2 <= num_sms && (int64_t)ncta * 512 < src.max_len)))
    ncta *= 2;
  a.part = (src.max_len + ncta - 1) / ncta;
  int threads = 128;
  while (threads < kSelMaxThreads && threads * 4 < a.part) threads *= 2;
  a.run = (a.part + threads - 1) / threads;
  a.in_smem = a.part <= kSelMaxKeys;
  const size_t smem = a.in_smem ? (size_t)(padded(a.part) + 1) * 4 + (size_t)a.part * 2 + 4 : 0;
  cudaError_t e = prefer_max_shared<cache_select_kernel,
                                    (kSelMaxKeys + kSelMaxKeys / 32 + 2) * 4 + kSelMaxKeys * 2>();
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(src.B * src.Hkv * ncta));
  cfg.blockDim = dim3((unsigned)threads);
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
  c.rows = kCopyPieces / (2 * (src.d * c.es / 16));
  if (c.rows > kCopyRows) c.rows = kCopyRows;
  c.blocks = (keep + c.rows - 1) / c.rows;
  e = prefer_max_shared<cache_copy_kernel>();
  if (e != cudaSuccess) return e;
  return launch_pdl(cache_copy_kernel, dim3((unsigned)(src.B * src.Hkv * c.blocks)),
                    dim3(kCopyThreads), 0, s, c);
}

}  // namespace avits
