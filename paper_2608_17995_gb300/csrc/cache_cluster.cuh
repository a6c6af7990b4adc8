// cache_cluster.cuh — the cache attention of shorter sequences: a cluster of CTAs per unit.
#pragma once

#include <cooperative_groups.h>

#include "cache_line.cuh"

namespace cg = cooperative_groups;

namespace avits {
namespace cache {
namespace {

// kAlone: avits_cache_attention in one launch.  For shared prefixes:
//   kBoth   a prefix's tokens and then the sequence's own, in one launch; every sequence
//           reads its prefix by itself (from L2)
//   kParts  the own tokens, a CTA for each run of a unit's tiles (a.least of them, a.grid runs to
//           a unit), as parts to be joined, beside the kernel before, which goes over the
//           prefixes and has waited for what both read: the last CTA waits for it, for the join
enum ClusterForm { kAlone = 0, kBoth = 1, kParts = 2 };

template <int kForm>
struct Beside {};
template <>
struct Beside<kBoth> {
  CUtensorMap mk, mv;
  CacheAttn p;
};

template <typename Rows>
constexpr int cluster_smem(int warps, int rows, int keys) {   // keys: logits' row stride, 0: none
  return smem_bytes<Rows>(warps) + Rows::kR * Rows::D * 4 + rows * keys * 4;
}
// The row stride of `keys` logits: 8 more than a multiple of 32, which spreads
// the rows over the banks.
inline int logit_stride(int keys) { return (keys + 23) / 32 * 32 + 8; }

// CTAs to an SM that the registers have to allow: parts of 8 rows need no more than 128.
template <typename Rows, int W, int kForm>
constexpr int cluster_min() {
  return kForm == kParts && Rows::kBf16 && Rows::D <= 128 && Rows::kR == 8
             ? 16 / W : cluster_ctas(Rows::D, Rows::kR, W);
}

// A cluster of CTAs per unit, each with an equal run of its
// tiles and their logits in shared memory.  The CTAs' maxima, sums and O meet
// through distributed shared memory; then every CTA writes a slice of O and the
// weights of its own keys.  No workspace, no second kernel.
template <typename Rows, int W, int kForm>
__global__ void __launch_bounds__(32 * W, cluster_min<Rows, W, kForm>())
cache_cluster_kernel(const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
                     const __grid_constant__ CacheAttn a, int stride,
                     const __grid_constant__ Beside<kForm> x) {
  using T = typename Rows::T;
  constexpr int D = Rows::D, kR = Rows::kR, kTile = Rows::kTile, NS = stages<Rows>();
  constexpr int kMaxCluster = 8, kCta = 32 * W;
  extern __shared__ __align__(1024) char smem[];
  __shared__ float2 s_ml[W][Rows::kBufRows];
  __shared__ float2 s_mine[kR];                  // this CTA's maximum and sum of a row
  __shared__ float s_f[kMaxCluster][kR];
  __shared__ float2 s_norm[kR];
  __shared__ int s_free[W];
  __shared__ uint64_t s_full[W][NS];
  __shared__ uint32_t s_mask[W][NS];
  cg::cluster_group cluster = cg::this_cluster();
  const int ncta = kForm == kParts ? a.grid : (int)cluster.num_blocks();
  // The shuffle tells the compiler that a warp's w is one value, so that its tiles'
  // shuffles and products are in no divergent code (8 x <= 2000 with 32
  // rows to a unit 22.0 us without it, 21.3 with).
  const int tid = threadIdx.x, w = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int unit = blockIdx.x / ncta;
  const int me = kForm == kParts ? (int)blockIdx.x - unit * ncta : (int)cluster.block_rank();
  const int units = a.c.Hkv * a.groups;
  const OwnUnits all{units, a.groups};
  const int b = unit / units, u = unit - b * units;
  const int hk = u / a.groups, row0 = (u - hk * a.groups) * kR;
  const int h0 = hk * a.G + row0, rows_here = min(kR, a.G - row0);
  if (lane < NS) mbar_init(&s_full[w][lane], a.box ? 1 : 32);   // a warp's barriers are its own
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  before_copies();
  __syncwarp();
  if (tid == 0 && a.box) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&mk));
    asm volatile("prefetch.tensormap [%0];" ::"l"(&mv));
  }
  if (kForm != kParts) pdl_wait();
  pdl_trigger();
  if (u == 0 && me == 0 && tid == 0) check_cache_len(a.c, b, a.status);
  const int len = cache_len(a.c, b);
  int g = 0, len_p = 0, nt_p = 0;        // the prefix
  if constexpr (kForm == kBoth) {
    const CacheAttn& p = x.p;
    const int each = (p.c.B + 31) / 32, g0 = min(p.c.B, lane * each);
    g = group_of(p.start, p.c.B, b);
    const int2 m = members_of(p.start, p.seqs, g);
    const int n = cache_len(p.c, g);              // all of these reads at once
    const bool rise = __all_sync(0xffffffffu, groups_ok(p, g0, min(p.c.B, g0 + each)));
    if (rise && b >= m.x && b < m.y) len_p = n;
    nt_p = tiles_of(p, len_p);
    if (blockIdx.x == 0 && w == 0) {
      for (int y = lane; y < p.c.B; y += 32) check_cache_len(p.c, y, a.status);
      if (!rise && lane == 0) raise_status(a.status, AVITS_ERR_PAGE);
    }
  }
  if (kForm == kParts && me * a.least * kTile >= len) {
    if (blockIdx.x == gridDim.x - 1) pdl_wait();
    return;
  }
  if (len + len_p == 0) {      // the whole cluster
    if (me == 0)
      for (int i = tid; i < rows_here * a.c.d; i += kCta) {
        const int r = i / a.c.d;
        store_elem(static_cast<T*>(a.o), (int64_t)b * a.o_sb + (int64_t)(h0 + r) * a.o_sh +
                   (i - r * a.c.d), 0.f);
        if (a.lse && i == r * a.c.d) a.lse[(int64_t)b * a.H + h0 + r] = -INFINITY;
      }
    return;
  }
  const int nt = nt_p + tiles_of(a, len), run = kForm == kParts ? a.least : (nt + ncta - 1) / ncta;
  const int t0 = min(nt, me * run), mine = min(nt, t0 + run) - t0;
  char* ring = smem + w * NS * Rows::kStage;
  char* s_q = smem + W * NS * Rows::kStage;
  char* s_w = s_q + Rows::kQBytes + w * Rows::kWarpBytes;
  float* s_o = reinterpret_cast<float*>(smem + smem_bytes<Rows>(W));
  float* s_lg = s_o + kR * D;
  const int all_mine = (mine - w + W - 1) / W;
  // of this warp's tiles, those of the prefix
  const int n_p = kForm == kBoth ? max(0, (min(mine, nt_p - t0) - w + W - 1) / W) : 0;
  Cursor cur{b, u, t0 + w + n_p * W - nt_p, nt - nt_p, len, all_mine - n_p, -1};
  if (cur.left > 0) cur.look_up<kTile>(a, lane);
  Cursor cur_p{g, u, t0 + w, nt_p, len_p, n_p, -1};
  if constexpr (kForm == kBoth)
    if (cur_p.left > 0) cur_p.look_up<kTile>(x.p, lane);
  constexpr int kQEach = (Rows::kQPieces + kCta - 1) / kCta;
  uint4 q[kQEach];
#pragma unroll
  for (int k = 0; k < kQEach; ++k)
    if (tid + k * kCta < Rows::kQPieces)
      q[k] = Rows::load_q(a, QRows{b, h0, rows_here, 0, 0}, tid + k * kCta);
  int fill = 0, use = 0;
  uint32_t phase = 0;
  int late = 0;         // a copy did not come in time: the others get little more
  auto issue = [&]() {
    if constexpr (kForm == kBoth) {
      if (cur_p.left > 0) {
        copy_tile<Rows, W>(x.mk, x.mv, x.p, cur_p, ring + fill * Rows::kStage, &s_full[w][fill],
                           &s_mask[w][fill], all, lane);
        fill = fill + 1 == NS ? 0 : fill + 1;
        return;
      }
    }
    if (cur.left > 0)
      copy_tile<Rows, W>(mk, mv, a, cur, ring + fill * Rows::kStage, &s_full[w][fill],
                         &s_mask[w][fill], all, lane);
    fill = fill + 1 == NS ? 0 : fill + 1;
  };
#pragma unroll 1
  for (int i = 0; i < NS - 1; ++i) issue();
#pragma unroll
  for (int k = 0; k < kQEach; ++k)
    if (tid + k * kCta < Rows::kQPieces) Rows::store_q(s_q, tid + k * kCta, q[k]);
  __syncthreads();
  Rows rows;
  rows.reset();
  const int lrow = Rows::logit_row(lane);
#pragma unroll 1
  for (int t = w; t < mine; t += W) {
    __syncwarp();
    issue();
    late |= !mbar_wait_bounded(&s_full[w][use], phase, nullptr, a.status,
                               late ? kLateNs : kWaitLimitNs);
    __syncwarp();
    const unsigned here = s_mask[w][use];
    if (here != (1u << kTile) - 1u)
      clear_rows<Rows>(ring + use * Rows::kStage, here, lane);
    one_tile(rows, a, ring + use * Rows::kStage, s_q, s_w, here,
             s_lg + lrow * stride + t * kTile, stride, rows_here, lane);
    if (++use == NS) {
      use = 0;
      phase ^= 1u;
    }
  }
  // this CTA's rows over its warps
#pragma unroll
  for (int part = 0; part < Rows::kM; ++part) {
    __syncwarp();
    rows.put(part, s_ml[w], reinterpret_cast<float*>(ring + fill * Rows::kStage), lane);
    if (lane == 0) s_free[w] = (w * NS + fill) * Rows::kStage;
    __syncthreads();
    for (int i = tid; i < Rows::kBufRows * (D / 4); i += kCta) {
      const int r = i / (D / 4), d = (i - r * (D / 4)) * 4, row = part * 16 + r;
      if (row >= rows_here || d >= a.c.d) continue;
      float top = -INFINITY, l = 0.f;
#pragma unroll
      for (int k = 0; k < W; ++k) top = fmaxf(top, s_ml[k][r].x);
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < W; ++k) {
        const float2 ml = s_ml[k][r];
        const float4 x = *reinterpret_cast<const float4*>(smem + s_free[k] + o_at(r, d, D) * 4);
        const float f = ml.x == -INFINITY ? 0.f : ex2(ml.x - top);
        v.x = fmaf(f, x.x, v.x); v.y = fmaf(f, x.y, v.y);
        v.z = fmaf(f, x.z, v.z); v.w = fmaf(f, x.w, v.w);
        l = fmaf(f, ml.y, l);
      }
      if (kForm == kParts) {
        *reinterpret_cast<float4*>(a.po + ((int64_t)blockIdx.x * kR + row) * a.c.d + d) = v;
        if (d == 0) a.pml[blockIdx.x * kR + row] = make_float2(top, l);
        continue;
      }
      *reinterpret_cast<float4*>(s_o + row * D + d) = v;
      if (d == 0) s_mine[row] = make_float2(top, l);
    }
    __syncthreads();
  }
  if (kForm == kParts) {
    if (tid == 0 && me == 0) a.rec[unit] = make_int2(blockIdx.x, (nt + run - 1) / run);
    if (blockIdx.x == gridDim.x - 1) pdl_wait();
    return;
  }
  cluster.sync();
  // over the CTAs: a row's maximum and sum, and what each CTA's O counts in it
  if (tid < rows_here) {
    float2 x[kMaxCluster];
    float top = -INFINITY, l = 0.f;
#pragma unroll
    for (int k = 0; k < kMaxCluster; ++k) {
      x[k] = make_float2(-INFINITY, 0.f);
      if (k < ncta) x[k] = cluster.map_shared_rank(s_mine, k)[tid];
      top = fmaxf(top, x[k].x);
    }
    const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int k = 0; k < kMaxCluster; ++k) l = fmaf(ex2(x[k].x - ref), x[k].y, l);
    const float2 norm = norm_of(top, l);
#pragma unroll
    for (int k = 0; k < kMaxCluster; ++k) s_f[k][tid] = ex2(x[k].x - ref) * norm.y;
    s_norm[tid] = norm;
    if (me == 0 && a.lse) a.lse[(int64_t)b * a.H + h0 + tid] = lse2_of(top, l) * kLn2;
  }
  __syncthreads();
  const int d4 = a.c.d / 4;
  for (int i = me * kCta + tid; i < rows_here * d4; i += ncta * kCta) {
    const int r = i / d4, d = (i - r * d4) * 4;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int k = 0; k < ncta; ++k) {
      const float4 x =
          *reinterpret_cast<const float4*>(cluster.map_shared_rank(s_o, k) + r * D + d);
      const float f = s_f[k][r];
      v.x = fmaf(f, x.x, v.x); v.y = fmaf(f, x.y, v.y);
      v.z = fmaf(f, x.z, v.z); v.w = fmaf(f, x.w, v.w);
    }
    T* out = static_cast<T*>(a.o) + (int64_t)b * a.o_sb + (int64_t)(h0 + r) * a.o_sh + d;
    store_elem(out, 0, v.x);
    store_elem(out, 1, v.y);
    store_elem(out, 2, v.z);
    store_elem(out, 3, v.w);
  }
  if (kForm == kAlone && a.score) {
    const int j0 = t0 * kTile, n = min(len - j0, mine * kTile);
    float* acc = a.c.acc + (int64_t)b * a.c.acc_sb + (int64_t)hk * a.c.acc_sh + j0;
    for (int j = tid; j < n; j += kCta) {
      const float old = a.add ? acc[j] : 0.f;
      float s = 0.f;
#pragma unroll 8
      for (int r = 0; r < rows_here; ++r) {
        const float2 norm = s_norm[r];
        s = fmaf(ex2(s_lg[r * stride + j] - norm.x), norm.y, s);
      }
      acc[j] = fmaf(s, a.wmean, old);
    }
  }
  cluster.sync();      // no CTA leaves while another reads its O
}

template <typename Rows, int W, int kForm>
cudaError_t launch_rows(const CUtensorMap& mk, const CUtensorMap& mv, const CacheAttn& a, int ncta,
                        int max_len, const Beside<kForm>& x, cudaStream_t s) {
  constexpr auto kernel = cache_cluster_kernel<Rows, W, kForm>;
  const cudaError_t e = prefer_max_shared<kernel, kMaxDynamic>();
  if (e != cudaSuccess) return e;
  const int tiles = (max_len + a.tile - 1) / a.tile;
  const int stride = a.score ? logit_stride((tiles + ncta - 1) / ncta * a.tile) : 0;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(a.c.B * a.c.Hkv * a.groups * (kForm == kParts ? a.grid : ncta)));
  cfg.blockDim = dim3(32 * W);
  cfg.dynamicSmemBytes = (size_t)cluster_smem<Rows>(W, a.G < a.rows ? a.G : a.rows, stride);
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)ncta;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = kForm == kParts ? 1 : 2;
  return cudaLaunchKernelEx(&cfg, kernel, mk, mv, a, stride, x);
}

}  // namespace
}  // namespace cache
}  // namespace avits
