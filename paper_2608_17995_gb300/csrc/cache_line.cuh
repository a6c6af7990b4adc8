// cache_line.cuh — attention on one line of tiles: the kernel over equal pieces of it.
#pragma once

#include "cache_tiles.cuh"

namespace avits {
namespace cache {
namespace {

// Whether the groups of prefixes [g0, g1) rise within the batch.
__device__ __forceinline__ bool groups_ok(const CacheAttn& a, int g0, int g1) {
  bool ok = true;
  for (int g = g0; g < g1; ++g) {
    const int x = a.start[g], y = a.start[g + 1];
    ok = ok && x >= 0 && x <= y && y <= a.seqs;
  }
  return ok;
}

// The last group that starts at sequence b or before it.
__device__ __forceinline__ int group_of(const int32_t* start, int groups, int b) {
  int lo = 0, hi = groups - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (start[mid] <= b) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// kWhole: avits_cache_attention's first kernel.  Units that lie in one piece are finished.
// The others leave every piece of a unit as a part: part (unit + CTA) of the line, which
// has one more at each unit's and each CTA's border.
//   kOwn    a batch's own tokens, beside the kernel before, which goes over the prefixes and
//           has waited for what both read: it is waited for at the end, for the join
//   kGroup  prefixes, whose rows are the query heads of all sequences of a group; the
//           kernel behind it may start beside it
enum LineForm { kWhole = 0, kOwn = 1, kGroup = 2 };

template <typename Rows, int kForm>
constexpr int line_min() {
  return kForm == kOwn ? own_ctas(Rows::D, Rows::kR, Rows::kBf16)
                       : line_ctas(Rows::D, Rows::kR, Rows::kBf16);
}

template <typename Rows, int kForm>
__global__ void __launch_bounds__(kThreads, line_min<Rows, kForm>())
cache_line_kernel(const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
                  const __grid_constant__ CacheAttn a) {
  using T = typename Rows::T;
  constexpr int D = Rows::D, kR = Rows::kR, kTile = Rows::kTile, NS = stages<Rows>();
  extern __shared__ __align__(1024) char smem[];
  __shared__ float2 s_ml[2][kWarps][Rows::kBufRows];
  __shared__ int s_free[2][kWarps];
  __shared__ uint64_t s_full[kWarps][NS];
  __shared__ uint32_t s_mask[kWarps][NS];
  // The shuffle tells the compiler that a warp's w is one value, so that its tiles'
  // shuffles and products are in no divergent code (2 KV heads with 24 rows
  // each, 32 x <= 6000, 47.1 us without it, 46.5 with).
  const int tid = threadIdx.x, w = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  if (lane < NS) mbar_init(&s_full[w][lane], a.box ? 1 : 32);   // a warp's barriers are its own
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  before_copies();
  __syncwarp();
  if (tid == 0 && a.box) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&mk));
    asm volatile("prefetch.tensormap [%0];" ::"l"(&mv));
  }
  if (kForm != kOwn) pdl_wait();
  if (kForm == kGroup) pdl_trigger();

  // sequences without cached tokens
  for (int b = kForm == kWhole ? blockIdx.x : a.c.B; b < a.c.B; b += gridDim.x) {
    if (cache_len(a.c, b) > 0) continue;
    for (int i = tid; i < a.H * a.c.d; i += kThreads) {
      const int h = i / a.c.d;
      store_elem(static_cast<T*>(a.o), (int64_t)b * a.o_sb + (int64_t)h * a.o_sh + (i - h * a.c.d),
                 0.f);
      if (a.lse && i == h * a.c.d) a.lse[(int64_t)b * a.H + h] = -INFINITY;
    }
  }

  // where this CTA's piece of the line of tiles begins: every warp scans the
  // lengths, a lane a contiguous run of them
  const int B = a.c.B;
  const auto all = [&] {
    if constexpr (kForm == kGroup) return GroupUnits{};
    else return OwnUnits{a.c.Hkv * a.groups, a.groups};
  }();
  const int each = (B + 31) / 32, b0 = min(B, lane * each), b1 = min(B, b0 + each);
  int sum = 0, usum = 0;          // tiles; units
  for (int b = b0; b < b1; ++b) {
    const int n = all.of(a, b);
    sum += tiles_of(a, cache_len(a.c, b)) * n;
    usum += n;
    if (blockIdx.x == 0 && w == 0) check_cache_len(a.c, b, a.status);
  }
  int inc = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += y;
  }
  int total = __shfl_sync(0xffffffffu, inc, 31);
  int ubase = 0;                  // first unit of a sequence
  if (kForm == kGroup) {
    int uinc = usum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, uinc, o);
      if (lane >= o) uinc += y;
    }
    ubase = uinc - usum;
    // groups that do not rise could be more units than there is room for: no prefix is read
    const bool rise = __all_sync(0xffffffffu, groups_ok(a, b0, b1));
    if (blockIdx.x == 0 && w == 0) {
      for (int b = b0, at = ubase; b < b1; at += all.of(a, b++)) a.base[b] = at;
      if (lane == 0) {
        a.base[B] = rise;
        if (!rise) raise_status(a.status, AVITS_ERR_PAGE);
      }
    }
    if (!rise) total = 0;
  }
  const int per = max(a.least, (total + a.grid - 1) / a.grid);
  const int first = blockIdx.x * per;
  if (first >= total) {
    if (kForm == kWhole && tid == 0) a.own[blockIdx.x] = make_int4(-1, 0, 0, 0);
    if (kForm == kOwn) pdl_wait();
    return;
  }
  int sb = b0, soff = first - (inc - sum);
  const bool here_lane = soff >= 0 && soff < sum;
  if (here_lane)
    for (;; ++sb) {
      const int un = all.of(a, sb), n = tiles_of(a, cache_len(a.c, sb)) * un;
      if (soff < n) break;
      soff -= n;
      ubase += un;
    }
  const int src = __ffs(__ballot_sync(0xffffffffu, here_lane)) - 1;
  sb = __shfl_sync(0xffffffffu, sb, src);
  soff = __shfl_sync(0xffffffffu, soff, src);
  ubase = kForm == kGroup ? __shfl_sync(0xffffffffu, ubase, src) : sb * (a.c.Hkv * a.groups);
  char* ring = smem + w * NS * Rows::kStage;
  char* s_q = smem + kWarps * NS * Rows::kStage;
  char* s_w = s_q + Rows::kQBytes + w * Rows::kWarpBytes;

  int left = min(per, total - first), b = sb;
  int len = cache_len(a.c, b), nt = tiles_of(a, len);
  int u = soff / nt, t0 = soff - u * nt;
  Cursor cur{b, u, t0 + w, nt, len, (left - w + kWarps - 1) / kWarps, -1};
  if (cur.left > 0) {
    cur.settle(a, all);
    cur.look_up<kTile>(a, lane);
  }
  auto rows_of = [&](int bb, int uu) {
    if constexpr (kForm == kGroup) {
      const int2 m = members_of(a.start, a.seqs, bb);
      const int n = (m.y - m.x) * a.G, rg = (n + kR - 1) / kR, hk = uu / rg, r0 = (uu - hk * rg) * kR;
      return QRows{m.x, hk * a.G, min(kR, n - r0), r0, a.G};
    } else {
      const int hk = a.groups == 1 ? uu : uu / a.groups, row0 = (uu - hk * a.groups) * kR;
      return QRows{bb, hk * a.G + row0, min(kR, a.G - row0), 0, 0};
    }
  };
  // stage `fill` is the free one: the tile after the last issued goes there
  int fill = 0, use = 0;
  uint32_t phase = 0;
  int late = 0;         // a copy did not come in time: the others get little more
  auto issue = [&]() {
    if (cur.left > 0)
      copy_tile<Rows, kWarps>(mk, mv, a, cur, ring + fill * Rows::kStage, &s_full[w][fill],
                              &s_mask[w][fill], all, lane);
    fill = fill + 1 == NS ? 0 : fill + 1;
  };
  constexpr int kQEach = (Rows::kQPieces + kThreads - 1) / kThreads;
  uint4 nq[kQEach];
  {
    const QRows h = rows_of(b, u);
#pragma unroll
    for (int k = 0; k < kQEach; ++k)
      if (tid + k * kThreads < Rows::kQPieces)
        nq[k] = Rows::load_q(a, h, tid + k * kThreads);
  }
#pragma unroll 1
  for (int i = 0; i < NS - 1; ++i) issue();
#pragma unroll
  for (int k = 0; k < kQEach; ++k)
    if (tid + k * kThreads < Rows::kQPieces) Rows::store_q(s_q, tid + k * kThreads, nq[k]);
  __syncthreads();      // Q is there

  int f0 = 0, seg = 0;
  int4 own = make_int4(-1, 0, 0, 0);
  Rows rows;
  while (left > 0) {
    const int t1 = min(nt, t0 + left);
    const QRows h = rows_of(b, u);
    // the next unit, and its Q on the way
    int nb = b, nu = u + 1, nlen = len, nnt = nt, nbase = ubase;
    const int after = left - (t1 - t0);
    if (after > 0) {
      int un = all.of(a, nb);
      if (nu == un) {
        nu = 0;
        do {
          nbase += un;
          nlen = cache_len(a.c, ++nb);
          nnt = tiles_of(a, nlen);
          un = all.of(a, nb);
        } while (nnt == 0 || un == 0);
      }
      const QRows nh = rows_of(nb, nu);
#pragma unroll
      for (int k = 0; k < kQEach; ++k)
        if (tid + k * kThreads < Rows::kQPieces)
          nq[k] = Rows::load_q(a, nh, tid + k * kThreads);
    }
    rows.reset();
    const int lrow = Rows::logit_row(lane);
    const bool score = kForm == kWhole && a.score;
    float* lg = score ? a.logits + ((int64_t)b * a.H + h.h0 + lrow) * a.ld : nullptr;
#pragma unroll 1
    for (int t = t0 + ((w - f0) & (kWarps - 1)); t < t1; t += kWarps) {
      __syncwarp();
      issue();
      late |= !mbar_wait_bounded(&s_full[w][use], phase, nullptr, a.status,
                                 late ? kLateNs : kWaitLimitNs);
      __syncwarp();
      const unsigned here = s_mask[w][use];
      if (here != (1u << kTile) - 1u)
        clear_rows<Rows>(ring + use * Rows::kStage, here, lane);
      one_tile(rows, a, ring + use * Rows::kStage, s_q, s_w, here,
               score ? lg + t * kTile : nullptr, a.ld, h.rows, lane);
      if (++use == NS) {
        use = 0;
        phase ^= 1u;
      }
    }
    // the warps meet: each leaves its rows in the free stage of its ring
    const bool whole = t0 == 0 && t1 == nt;
    const int slot = kForm == kWhole ? 2 * blockIdx.x + (seg == 0 ? 0 : 1)
                                     : ubase + u + (int)blockIdx.x;
#pragma unroll
    for (int part = 0; part < Rows::kM; ++part) {
      const int par = (seg * Rows::kM + part) & 1;
      __syncwarp();
      rows.put(part, s_ml[par][w], reinterpret_cast<float*>(ring + fill * Rows::kStage), lane);
      if (lane == 0) s_free[par][w] = (w * NS + fill) * Rows::kStage;
      __syncthreads();
      if (part == 0 && after > 0) {
#pragma unroll
        for (int k = 0; k < kQEach; ++k)
          if (tid + k * kThreads < Rows::kQPieces) Rows::store_q(s_q, tid + k * kThreads, nq[k]);
      }
      for (int i = tid; i < Rows::kBufRows * (D / 4); i += kThreads) {
        const int r = i / (D / 4), d = (i - r * (D / 4)) * 4, row = part * 16 + r;
        if (row >= h.rows || d >= a.c.d) continue;
        float top = -INFINITY, l = 0.f;
#pragma unroll
        for (int k = 0; k < kWarps; ++k) top = fmaxf(top, s_ml[par][k][r].x);
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < kWarps; ++k) {
          const float2 ml = s_ml[par][k][r];
          const float4 x = *reinterpret_cast<const float4*>(smem + s_free[par][k] +
                                                            o_at(r, d, D) * 4);
          const float f = ml.x == -INFINITY ? 0.f : ex2(ml.x - top);
          v.x = fmaf(f, x.x, v.x); v.y = fmaf(f, x.y, v.y);
          v.z = fmaf(f, x.z, v.z); v.w = fmaf(f, x.w, v.w);
          l = fmaf(f, ml.y, l);
        }
        const int hh = h.h0 + row;
        if (kForm == kWhole && whole) {
          const float2 norm = norm_of(top, l);
          const float inv = norm.y;
          T* out = static_cast<T*>(a.o) + (int64_t)b * a.o_sb + (int64_t)hh * a.o_sh + d;
          store_elem(out, 0, v.x * inv);
          store_elem(out, 1, v.y * inv);
          store_elem(out, 2, v.z * inv);
          store_elem(out, 3, v.w * inv);
          if (d == 0) {
            if (a.score) a.norm[(int64_t)b * a.H + hh] = norm;
            if (a.lse) a.lse[(int64_t)b * a.H + hh] = lse2_of(top, l) * kLn2;
          }
        } else {
          *reinterpret_cast<float4*>(a.po + ((int64_t)slot * kR + row) * a.c.d + d) = v;
          if (d == 0) a.pml[slot * kR + row] = make_float2(top, l);
        }
      }
      before_copies();
      __syncthreads();     // the free stages are free again
    }
    if (t0 == 0) {
      const int T0 = first + f0, c1 = (T0 + nt - 1) / per;
      const int pieces = c1 - (int)blockIdx.x + 1;
      const int unit = ubase + u;
      if (pieces > 1) own = make_int4(unit, slot, pieces, 0);
      if (tid == 0 && (kForm != kWhole || a.score || !a.few)) a.rec[unit] = make_int2(slot, pieces);
    }
    ++seg;
    f0 += t1 - t0;
    left = after;
    b = nb; u = nu; len = nlen; nt = nnt; t0 = 0; ubase = nbase;
  }
  if (kForm == kOwn) pdl_wait();
  if (kForm == kWhole && tid == 0) a.own[blockIdx.x] = own;
  // The joining kernel's blocks come onto the SMs only now: let go at the start, they
  // cost this kernel more than they gained (14 x <= 2286 in fp32, 3 CTAs to an SM, 52
  // us for 34; 131072 keys 58.5 for 56.4; launched without overlap 58.8).
  if (kForm != kGroup) pdl_trigger();
}

}  // namespace
}  // namespace cache
}  // namespace avits
