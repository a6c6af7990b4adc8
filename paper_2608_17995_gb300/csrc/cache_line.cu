// cache_line.cu — the cache attention on one line of tiles: a kernel over equal
// pieces of it, and a second one that joins what was cut and sums the weights.
#include "cache_line.cuh"

namespace avits {
namespace cache {
namespace {

// ---------------------------------------------------------- second kernel --
// Block (unit, row), or, where there are many units, (CTA of the first kernel,
// rows): O of that unit, or of the one whose first of several pieces was that
// CTA's.  Block (b, hk, 512 keys or more): their weights.  What a block reads waits
// for as little as can be: parts and logits are on their way while the row's maximum and
// sum are put together.
constexpr int kFinishThreads = 128;
constexpr int kWeightKeys = 4 * kFinishThreads;

// Part of piece k of a unit: the first one's is given, the following CTAs' are
// their first.
__device__ __forceinline__ int part_of(int slot, int k) {
  return k == 0 ? slot : ((slot >> 1) + k) * 2;
}

// Maximum and sum of row r over a unit's pieces, in a whole warp.
__device__ __forceinline__ float2 join_rows(const CacheAttn& a, int slot, int pieces, int r,
                                            int lane) {
  constexpr int kDeep = 4;
  float top = -INFINITY, l = 0.f;
  for (int k0 = lane; k0 < pieces; k0 += 32 * kDeep) {
    float2 x[kDeep];
#pragma unroll
    for (int i = 0; i < kDeep; ++i) {
      const int k = k0 + 32 * i;
      x[i] = k < pieces ? a.pml[part_of(slot, k) * a.rows + r] : make_float2(-INFINITY, 0.f);
    }
    float mn = top;
#pragma unroll
    for (int i = 0; i < kDeep; ++i) mn = fmaxf(mn, x[i].x);
    const float ref = mn == -INFINITY ? 0.f : mn;
    l *= ex2(top - ref);                                  // a NaN stays one
#pragma unroll
    for (int i = 0; i < kDeep; ++i) l = fmaf(ex2(x[i].x - ref), x[i].y, l);
    top = mn;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float tx = __shfl_xor_sync(0xffffffffu, top, o);
    const float lx = __shfl_xor_sync(0xffffffffu, l, o);
    const float mn = fmaxf(top, tx), ref = mn == -INFINITY ? 0.f : mn;
    l = l * ex2(top - ref) + lx * ex2(tx - ref);
    top = mn;
  }
  return make_float2(top, l);
}

// The same in one thread, for few pieces.
__device__ __forceinline__ float2 join_rows_serial(const CacheAttn& a, int slot, int pieces,
                                                   int r) {
  float top = -INFINITY, l = 0.f;
  for (int k0 = 0; k0 < pieces; k0 += kFewPieces) {
    float2 x[kFewPieces];
#pragma unroll
    for (int i = 0; i < kFewPieces; ++i)
      x[i] = k0 + i < pieces ? a.pml[part_of(slot, k0 + i) * a.rows + r]
                             : make_float2(-INFINITY, 0.f);
    float mn = top;
#pragma unroll
    for (int i = 0; i < kFewPieces; ++i) mn = fmaxf(mn, x[i].x);
    const float ref = mn == -INFINITY ? 0.f : mn;
    l *= ex2(top - ref);
#pragma unroll
    for (int i = 0; i < kFewPieces; ++i) l = fmaf(ex2(x[i].x - ref), x[i].y, l);
    top = mn;
  }
  return make_float2(top, l);
}

// kWide: `at0` is a unit and r0 one of its rows, threads lie over 32 of its columns
// (from c0) and over its pieces; else at0 is a CTA of the first kernel and threads
// lie over whole rows from r0 on, each going through its row's pieces.
constexpr int kWideCols = 8;     // of 4

template <typename T, bool kWide>
__device__ __forceinline__ void join_block(const CacheAttn& a, int at0, int r0, int c0) {
  __shared__ float4 s_sum[kFinishThreads];
  const int tid = threadIdx.x, units = a.c.Hkv * a.groups;
  int4 own;
  if (kWide) {
    const int len = cache_len(a.c, at0 / units);
    const int2 rec = a.rec[at0];
    if (len == 0) return;
    own = make_int4(rec.y > 1 ? at0 : -1, rec.x, rec.y, 0);
  } else {
    own = a.own[at0];
  }
  if (own.x < 0) return;
  const int b = own.x / units, u = own.x - b * units, hk = u / a.groups;
  const int d4 = kWide ? kWideCols : a.c.d / 4, lanes = kFinishThreads / d4;
  const int sub = tid / d4, col = c0 + tid - sub * d4;
  const int r = kWide ? r0 : r0 + sub, step = kWide ? lanes : 1;
  const int row = (u - hk * a.groups) * a.rows + r, h = hk * a.G + row;
  const bool mine = sub < lanes && r < a.rows && row < a.G && col < a.c.d / 4;
  const int pieces = mine ? own.z : 0, k1 = kWide ? sub : 0;
  constexpr int kDeep = 8;
  float4 x[kDeep];
  float mx[kDeep];
  auto load = [&](int k0) {
#pragma unroll
    for (int i = 0; i < kDeep; ++i) {
      const int k = k0 + i * step;
      if (k < pieces) {
        const int at = part_of(own.y, k) * a.rows + r;
        x[i] = *reinterpret_cast<const float4*>(a.po + (int64_t)at * a.c.d + col * 4);
        mx[i] = a.pml[at].x;
      }
    }
  };
  load(k1);
  const float2 ml = kWide ? (row < a.G ? join_rows(a, own.y, own.z, r, tid & 31)
                                       : make_float2(-INFINITY, 0.f))
                          : join_rows_serial(a, own.y, pieces, r);
  if (mine && k1 == 0 && col == 0 && a.lse)
    a.lse[(int64_t)b * a.H + h] = lse2_of(ml.x, ml.y) * kLn2;
  const float2 norm = norm_of(ml.x, ml.y);
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int k0 = k1; k0 < pieces; k0 += kDeep * step) {
    if (k0 != k1) load(k0);
#pragma unroll
    for (int i = 0; i < kDeep; ++i)
      if (k0 + i * step < pieces) {
        const float f = ex2(mx[i] - norm.x);     // from -inf: 0
        v.x = fmaf(f, x[i].x, v.x); v.y = fmaf(f, x[i].y, v.y);
        v.z = fmaf(f, x[i].z, v.z); v.w = fmaf(f, x[i].w, v.w);
      }
  }
  if (kWide) {
    s_sum[tid] = v;
    __syncthreads();
    if (sub != 0) return;
    for (int k = 1; k < lanes; ++k) {
      const float4 y = s_sum[k * d4 + tid];
      v.x += y.x; v.y += y.y; v.z += y.z; v.w += y.w;
    }
  }
  if (!mine) return;
  T* out = static_cast<T*>(a.o) + (int64_t)b * a.o_sb + (int64_t)h * a.o_sh + col * 4;
  store_elem(out, 0, v.x * norm.y);
  store_elem(out, 1, v.y * norm.y);
  store_elem(out, 2, v.z * norm.y);
  store_elem(out, 3, v.w * norm.y);
}

// `parts` parts of kSpan runs of 512 keys, kRows rows at a time.  First the length
// and where the rows' pieces are; then everything else of the first part at once:
// logits, old weights, pieces.
template <int kSpan, int kRows>
__device__ __forceinline__ void weights_block(const CacheAttn& a, int bh, int part, int parts) {
  __shared__ float2 s_norm[kMaxGroup];
  const int b = bh / a.c.Hkv, hk = bh - b * a.c.Hkv, tid = threadIdx.x, w = tid >> 5;
  int jb = part * (kSpan * kWeightKeys);
  const int2* recs = a.rec + bh * a.groups;
  const int len = cache_len(a.c, b);
  int2 rec = recs[0];
  if (jb >= len) return;
  const float* lg = a.logits + ((int64_t)b * a.H + hk * a.G) * a.ld;
  float* acc = a.c.acc + (int64_t)b * a.c.acc_sb + (int64_t)hk * a.c.acc_sh;
  const bool vec = (reinterpret_cast<uintptr_t>(acc) & 15u) == 0;
  float4 x[kSpan][kRows];
  float old[kSpan][4];
  auto load = [&](int r0) {
#pragma unroll
    for (int g = 0; g < kSpan; ++g) {
      const int j = jb + g * kWeightKeys + tid * 4;
#pragma unroll
      for (int r = 0; r < kRows; ++r)
        if (j < len && r0 + r < a.G)
          x[g][r] = *reinterpret_cast<const float4*>(lg + (int64_t)(r0 + r) * a.ld + j);
    }
  };
  auto load_old = [&]() {
#pragma unroll
    for (int g = 0; g < kSpan; ++g) {
      const int j = jb + g * kWeightKeys + tid * 4;
#pragma unroll
      for (int k = 0; k < 4; ++k) old[g][k] = 0.f;
      if (a.add) {
        if (vec && j + 4 <= len) {
          const float4 y = *reinterpret_cast<const float4*>(acc + j);
          old[g][0] = y.x; old[g][1] = y.y; old[g][2] = y.z; old[g][3] = y.w;
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (j + k < len) old[g][k] = acc[j + k];
        }
      }
    }
  };
  load(0);
  load_old();
  const int step = a.few ? kFinishThreads : kFinishThreads / 32;
  for (int r = a.few ? tid : w; r < a.G; r += step) {
    const int rg = a.groups == 1 ? 0 : r / a.rows;
    if (rg > 0) rec = recs[rg];
    const int row = r - rg * a.rows;
    float2 norm;
    if (rec.y == 1) {
      norm = a.norm[(int64_t)b * a.H + hk * a.G + r];
    } else {
      const float2 ml = a.few ? join_rows_serial(a, rec.x, rec.y, row)
                              : join_rows(a, rec.x, rec.y, row, tid & 31);
      norm = norm_of(ml.x, ml.y);
    }
    if (a.few || (tid & 31) == 0) s_norm[r] = norm;
  }
  __syncthreads();
  const int end = min(len, jb + parts * (kSpan * kWeightKeys));
#pragma unroll 1
  for (;;) {
    float s[kSpan][4] = {};
    for (int r0 = 0; r0 < a.G; r0 += kRows) {
      if (r0 > 0) load(r0);
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        if (r0 + r < a.G) {
          const float2 norm = s_norm[r0 + r];
#pragma unroll
          for (int g = 0; g < kSpan; ++g) {
            s[g][0] = fmaf(ex2(x[g][r].x - norm.x), norm.y, s[g][0]);
            s[g][1] = fmaf(ex2(x[g][r].y - norm.x), norm.y, s[g][1]);
            s[g][2] = fmaf(ex2(x[g][r].z - norm.x), norm.y, s[g][2]);
            s[g][3] = fmaf(ex2(x[g][r].w - norm.x), norm.y, s[g][3]);
          }
        }
      }
    }
#pragma unroll
    for (int g = 0; g < kSpan; ++g) {
      const int j = jb + g * kWeightKeys + tid * 4;
#pragma unroll
      for (int k = 0; k < 4; ++k) s[g][k] = fmaf(s[g][k], a.wmean, old[g][k]);
      if (vec && j + 4 <= len) {
        *reinterpret_cast<float4*>(acc + j) = make_float4(s[g][0], s[g][1], s[g][2], s[g][3]);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (j + k < len) acc[j + k] = s[g][k];
      }
    }
    jb += kSpan * kWeightKeys;
    if (jb >= end) return;
    load(0);
    load_old();
  }
}

// Runs of 512 keys that a block of weights takes: small groups have few logits (40
// heads of one row to a group, 1500 keys: 50.5 us with 2 runs, 51.6 with 1; 2 KV heads
// with 24 rows each: 49.7 and 47.3).
inline int weight_span(int G) { return G > 2 ? 1 : 2; }

// The blocks of the second kernel: weights, `weights` blocks per (b, hk) of `parts`
// parts each, then joins.
struct Finish {
  int blocks, weights, parts;      // blocks: of weights, in all
  int rows, cols;                  // join blocks of a unit: row groups, column groups
};

template <typename T>
__global__ void __launch_bounds__(kFinishThreads, 6)
cache_finish_kernel(const __grid_constant__ CacheAttn a, Finish f) {
  pdl_wait_then_trigger();
  int i = blockIdx.x;
  if (i < f.blocks) {
    const int bh = i / f.weights, part = (i - bh * f.weights) * f.parts;
    if (a.G > 2) weights_block<1, 8>(a, bh, part, f.parts);
    else weights_block<2, 2>(a, bh, part, f.parts);
    return;
  }
  i -= f.blocks;
  if (a.few) {
    join_block<T, false>(a, i / f.rows, i % f.rows * (kFinishThreads / (a.c.d / 4)), 0);
  } else {
    const int col = i % f.cols, row = i / f.cols;
    join_block<T, true>(a, row / f.rows, row % f.rows, col * kWideCols);
  }
}

template <typename Rows>
cudaError_t launch_rows(CacheAttn& a, int num_sms, cudaStream_t s) {
  CUtensorMap mk{}, mv{};
  map_cache<Rows>(a, &mk, &mv);
  constexpr auto kernel = cache_line_kernel<Rows, kWhole>;
  cudaError_t e = prefer_max_shared<kernel, smem_bytes<Rows>(kWarps)>();
  if (e != cudaSuccess) return e;
  e = launch_pdl(kernel, dim3(a.grid), dim3(kThreads), smem_bytes<Rows>(kWarps), s, mk, mv, a);
  if (e != cudaSuccess) return e;
  const int bh = a.c.B * a.c.Hkv, d4 = a.c.d / 4;
  Finish f{};
  if (a.score) {
    // one part to a block, or two where there would be more blocks than are resident
    // at once (131072 keys: 61.0 us with two, 62.6 with one); four in a row took
    // longer again (48 x <= 4096: 98 us, with two 90)
    const int run = weight_span(a.G) * kWeightKeys, parts = (a.c.max_len + run - 1) / run;
    f.parts = parts > 1 && (long long)bh * parts > 6ll * num_sms ? 2 : 1;
    f.weights = (parts + f.parts - 1) / f.parts;
    f.blocks = bh * f.weights;
  }
  const int lanes = kFinishThreads / d4;
  f.rows = a.few ? (a.rows + lanes - 1) / lanes : a.rows;
  f.cols = a.few ? 1 : (d4 + kWideCols - 1) / kWideCols;
  const int joins = (a.few ? a.grid : bh * a.groups) * f.rows * f.cols;
  constexpr auto finish = cache_finish_kernel<typename Rows::T>;
  e = prefer_max_shared<finish>();
  if (e != cudaSuccess) return e;
  return launch_pdl(finish, dim3((unsigned)(f.blocks + joins)), dim3(kFinishThreads), 0, s, a, f);
}

}  // namespace

cudaError_t launch_line(CacheAttn& a, int D, int num_sms, cudaStream_t s) {
  return by_rows(a, D, [&](auto rows) { return launch_rows<decltype(rows)>(a, num_sms, s); });
}

}  // namespace cache
}  // namespace avits
