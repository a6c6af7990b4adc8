// cache_shared.cu — attention of one new token per sequence over a prefix that its group
// shares and its own cached tokens.
//
// For sequence b of group g and its query head h, over the keys j of both:
//   x_j = scale q . k_j,  lse = log sum_j exp x_j,  o = sum_j exp(x_j - lse) v_j
// The sum splits: each part of the keys leaves its maximum m, its sum l of
// exp(x - m) and its O = sum exp(x - m) v, and parts are joined by
//   M = max m,  o = sum_parts exp(m - M) O / sum_parts exp(m - M) l.
//
// A prefix is read once for all sequences of its group: the query heads of all of them
// that share a KV head are the rows of one product.  Three kernels: parts of the prefixes,
// parts of the own tokens beside it, and the join.
#include "cache_line.cuh"

namespace avits {
namespace {

using namespace cache;

constexpr int kJoinThreads = 256;

size_t up16(size_t n) { return (n + 15) / 16 * 16; }

// One line of tiles: how it is cut and what it leaves.
struct Line {
  int rows, groups, D, tile, grid, least;
  int box;                     // prefixes on the tensor cores: tokens of a copy; else 0
  long long units, tiles;      // at most
  size_t rec, pml, po, base, end;
};

int width_of(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

constexpr int kPrefixLeast = 2;

void cut(Line& l, const avits_kv_cache& c, int num_sms) {
  const bool bf = c.dt == AVITS_BF16;
  l.D = width_of(c.d);
  l.tile = l.box ? kPrefixTile : bf ? 16 : 8;
  const int longest = (c.max_len + l.tile - 1) / l.tile, few = l.box ? kPrefixLeast : kWarps;
  l.tiles = l.units * longest;
  l.least = longest < few ? longest : few;
  const long long most = (l.tiles + l.least - 1) / l.least;
  long long full = (long long)num_sms * (l.box ? kPrefixCtas : line_ctas(l.D, l.rows, bf));
  if (full > kMaxGrid) full = kMaxGrid;
  l.grid = (int)(most < full ? (most > 0 ? most : 1) : full);
}

// Rows of a unit for groups of n query heads that share a KV head.
int rows_of(bool bf, int D, long long n) {
  return !bf ? (n <= 4 ? 4 : 8) : n <= 8 ? 8 : n <= 16 || D == 256 ? 16 : 32;
}

struct Shape {
  Line own, pre;
  size_t total;
};

Shape shape_of(const CacheSharedCall& s, int num_sms) {
  const avits_kv_cache &c = s.cache, &p = s.prefix;
  const bool bf = c.dt == AVITS_BF16;
  const int G = s.H / c.Hkv, D = width_of(c.d);
  Shape x{};
  x.own.rows = rows_of(bf, D, G);
  x.own.groups = (G + x.own.rows - 1) / x.own.rows;
  x.own.units = (long long)c.B * c.Hkv * x.own.groups;
  x.pre.box = prefix_tc_box(p);
  x.pre.rows = x.pre.box ? kPrefixRows : rows_of(bf, D, ((long long)c.B + p.B - 1) / p.B * G);
  x.pre.groups = 0;
  x.pre.units = c.Hkv * ((long long)c.B * G / x.pre.rows + p.B);
  cut(x.own, c, num_sms);
  cut(x.pre, p, num_sms);
  size_t at = 0;
  for (Line* l : {&x.own, &x.pre}) {
    const size_t parts = (size_t)(l->units + l->grid) * l->rows;
    l->rec = at;
    l->pml = l->rec + up16((size_t)l->units * sizeof(int2));
    l->po = l->pml + up16(parts * sizeof(float2));
    l->base = l->po + up16(parts * c.d * sizeof(float));
    at = l->base + up16(((size_t)p.B + 1) * sizeof(int));
  }
  x.total = at;
  return x;
}

CacheAttn args_of(const CacheSharedCall& s, const avits_kv_cache& c, const Line& l,
                  unsigned int* status) {
  char* ws = static_cast<char*>(s.ws);
  CacheAttn a{};
  a.c = c;
  a.page = FastDiv::of(c.page_size);
  a.q = s.q;
  a.o = s.o;
  a.q_sb = s.q_sb; a.q_sh = s.q_sh; a.o_sb = s.o_sb; a.o_sh = s.o_sh;
  a.lse = s.lse;
  a.H = s.H;
  a.G = s.H / c.Hkv;
  a.rows = l.rows;
  a.groups = l.groups;
  a.tile = l.tile;
  a.grid = l.grid;
  a.least = l.least;
  a.box = l.box;
  a.scale2 = s.scale * kLog2e;
  a.rec = reinterpret_cast<int2*>(ws + l.rec);
  a.pml = reinterpret_cast<float2*>(ws + l.pml);
  a.po = reinterpret_cast<float*>(ws + l.po);
  a.base = reinterpret_cast<int*>(ws + l.base);
  a.start = s.group_start;
  a.seqs = s.cache.B;
  a.most = (int)l.units;
  a.status = status;
  return a;
}

// -------------------------------------------------------------------- join --
// The parts of one row: own ones, then the prefix's.
struct Parts {
  int own, n_own, pre, n_pre;      // first slots, times rows plus the row
  int own_step, pre_step;          // rows
  __device__ __forceinline__ int count() const { return n_own + n_pre; }
};

__device__ __forceinline__ float2 ml_of(const CacheAttn& o, const CacheAttn& p, const Parts& x,
                                        int k) {
  return k < x.n_own ? o.pml[x.own + k * x.own_step]
                     : p.pml[x.pre + (k - x.n_own) * x.pre_step];
}
// Columns 4 col .. of a part.  From the tensor cores a part lies as [d / 4][128 rows][4],
// so that a thread per row writes it in whole lines.
__device__ __forceinline__ float4 o_of(const CacheAttn& o, const CacheAttn& p, const Parts& x, int k,
                                       int col) {
  const int d4 = o.c.d / 4;
  if (k < x.n_own)
    return reinterpret_cast<const float4*>(o.po)[(int64_t)(x.own + k * x.own_step) * d4 + col];
  const int at = x.pre + (k - x.n_own) * x.pre_step;
  const float4* po = reinterpret_cast<const float4*>(p.po);
  if (p.rows != kPrefixRows) return po[(int64_t)at * d4 + col];
  return po[(int64_t)(at / kPrefixRows) * d4 * kPrefixRows + col * kPrefixRows + at % kPrefixRows];
}

// Block (b, hk, some of its query heads): threads lie over the heads, their columns, and
// the parts.
template <typename T>
__global__ void __launch_bounds__(kJoinThreads)
cache_join_kernel(const __grid_constant__ CacheAttn o, const __grid_constant__ CacheAttn p,
                  int heads) {
  __shared__ float4 s_sum[kJoinThreads];
  __shared__ Parts s_parts[kJoinThreads];
  __shared__ float2 s_ml[kJoinThreads];
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  const int b = blockIdx.x / o.c.Hkv, hk = blockIdx.x - b * o.c.Hkv;
  const int g0 = blockIdx.y * heads, n = min(heads, o.G - g0);
  pdl_wait_then_trigger();
  if (tid < n) {
    Parts x{0, 0, 0, 0, o.rows, p.rows};
    const int gq = g0 + tid;
    if (cache_len(o.c, b) > 0) {
      const int rg = gq / o.rows;
      const int2 rec = o.rec[(b * o.c.Hkv + hk) * o.groups + rg];
      x.own = rec.x * o.rows + gq - rg * o.rows;
      x.n_own = rec.y;
    }
    // the last group that starts at b or before it
    int lo = 0, hi = p.c.B - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (p.start[mid] <= b) lo = mid; else hi = mid - 1;
    }
    const int2 m = members_of(p.start, p.seqs, lo);
    if (b >= m.x && b < m.y && p.base[p.c.B] && cache_len(p.c, lo) > 0) {
      const int row = (b - m.x) * o.G + gq, rg = row / p.rows;
      const int all = ((m.y - m.x) * o.G + p.rows - 1) / p.rows;
      const int2 rec = p.rec[p.base[lo] + hk * all + rg];
      x.pre = rec.x * p.rows + row - rg * p.rows;
      x.n_pre = rec.y;
    }
    s_parts[tid] = x;
  }
  __syncthreads();
  for (int r = w; r < n; r += kJoinThreads / 32) {
    const Parts x = s_parts[r];
    float top = -INFINITY, l = 0.f;
    for (int k = lane; k < x.count(); k += 32) {
      const float2 y = ml_of(o, p, x, k);
      const float mn = fmaxf(top, y.x), ref = mn == -INFINITY ? 0.f : mn;
      l = l * ex2(top - ref) + y.y * ex2(y.x - ref);
      top = mn;
    }
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) {
      const float tx = __shfl_xor_sync(0xffffffffu, top, s);
      const float lx = __shfl_xor_sync(0xffffffffu, l, s);
      const float mn = fmaxf(top, tx), ref = mn == -INFINITY ? 0.f : mn;
      l = l * ex2(top - ref) + lx * ex2(tx - ref);
      top = mn;
    }
    if (lane == 0) {
      s_ml[r] = norm_of(top, l);
      if (o.lse) o.lse[(int64_t)b * o.H + hk * o.G + g0 + r] = lse2_of(top, l) * kLn2;
    }
  }
  __syncthreads();
  const int d4 = o.c.d / 4, items = n * d4, lanes = kJoinThreads / items;
  const int sub = tid / items, it = tid - sub * items, col = it / n, r = it - col * n;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  float2 norm = make_float2(0.f, 0.f);
  if (sub < lanes) {
    const Parts x = s_parts[r];
    norm = s_ml[r];
    for (int k = sub; k < x.count(); k += lanes) {
      const float4 y = o_of(o, p, x, k, col);
      const float f = ex2(ml_of(o, p, x, k).x - norm.x);
      v.x = fmaf(f, y.x, v.x); v.y = fmaf(f, y.y, v.y);
      v.z = fmaf(f, y.z, v.z); v.w = fmaf(f, y.w, v.w);
    }
  }
  if (lanes > 1) {
    s_sum[tid] = v;
    __syncthreads();
    if (sub != 0) return;
    for (int k = 1; k < lanes; ++k) {
      const float4 y = s_sum[k * items + it];
      v.x += y.x; v.y += y.y; v.z += y.z; v.w += y.w;
    }
  }
  if (sub != 0) return;
  T* out = static_cast<T*>(o.o) + (int64_t)b * o.o_sb + (int64_t)(hk * o.G + g0 + r) * o.o_sh +
           col * 4;
  store_elem(out, 0, v.x * norm.y);
  store_elem(out, 1, v.y * norm.y);
  store_elem(out, 2, v.z * norm.y);
  store_elem(out, 3, v.w * norm.y);
}

template <typename T>
cudaError_t launch_join(const CacheAttn& o, const CacheAttn& p, cudaStream_t s) {
  const int fit = kJoinThreads / (o.c.d / 4), heads = o.G < fit ? o.G : fit;
  const cudaError_t e = prefer_max_shared<cache_join_kernel<T>>();
  if (e != cudaSuccess) return e;
  return launch_pdl(cache_join_kernel<T>,
                    dim3((unsigned)(o.c.B * o.c.Hkv), (unsigned)((o.G + heads - 1) / heads)),
                    dim3(kJoinThreads), 0, s, o, p, heads);
}

template <int kForm>
cudaError_t launch_parts(CacheAttn& a, int D, cudaStream_t s) {
  return by_rows(a, D, [&](auto rows) {
    using Rows = decltype(rows);
    CUtensorMap mk{}, mv{};
    map_cache<Rows>(a, &mk, &mv);
    constexpr auto kernel = cache_line_kernel<Rows, kForm>;
    const cudaError_t e = prefer_max_shared<kernel, smem_bytes<Rows>(kWarps)>();
    if (e != cudaSuccess) return e;
    return launch_pdl(kernel, dim3(a.grid), dim3(kThreads), smem_bytes<Rows>(kWarps), s, mk, mv, a);
  });
}

}  // namespace

bool cache_shared_sizes_ok(const CacheSharedCall& s) {
  const avits_kv_cache& c = s.cache;
  if (s.H / c.Hkv > kMaxGroup || (long long)c.B * s.H >= (1ll << 30)) return false;
  const Shape x = shape_of(s, 1);
  if ((long long)c.B * c.Hkv >= (1ll << 31) - 1) return false;
  for (const Line* l : {&x.own, &x.pre})
    if (l->tiles >= (1ll << 30) || (l->units + kMaxGrid) * l->rows >= (1ll << 31)) return false;
  return true;
}

size_t cache_shared_workspace(const CacheSharedCall& s, int num_sms) {
  return shape_of(s, num_sms).total;
}

cudaError_t launch_cache_shared(const CacheSharedCall& s, int num_sms, unsigned int* status,
                                cudaStream_t stream) {
  const Shape x = shape_of(s, num_sms);
  CacheAttn own = args_of(s, s.cache, x.own, status), pre = args_of(s, s.prefix, x.pre, status);
  cudaError_t e = x.pre.box ? launch_prefix_tc(pre, stream)
                          : launch_parts<kGroup>(pre, x.pre.D, stream);
  if (e == cudaSuccess) e = launch_parts<kOwn>(own, x.own.D, stream);
  if (e != cudaSuccess) return e;
  return s.cache.dt == AVITS_BF16 ? launch_join<__nv_bfloat16>(own, pre, stream)
                                  : launch_join<float>(own, pre, stream);
}

}  // namespace avits
