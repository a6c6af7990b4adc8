// cache_prefix_tc.cu — parts of the attention over shared prefixes on the tensor cores
// (bf16, widths up to 128): the query heads of all of a group's sequences that share a KV
// head are the rows of one product.
//
// Unit: (group, KV head, 128 kT rows), kT = 1 or 2 row tiles.  All tiles of 64 keys of all
// units form one line, cut into equal pieces, one per CTA.  kT = 1: two CTAs share an SM, so
// that one's exponentials run while the other's products do; kT = 2: one CTA, whose two row
// tiles do that with one copy of the keys and values.  Roles of the warps:
//   0          loads keys and values through a ring of tiles (TMA, a box per page or part
//              of one; what lies past the prefix or outside the pool comes as zeros)
//   1 .. kT    issue a row tile's products: S(j+1) = Q K(j+1)^T, then O += P(j) V(j) as soon
//              as P(j) is written, so that S is a tile ahead
//   then 4 kT  one row to a thread: the running maximum (moved when a tile's passes it by
//              2^8: O is rescaled then), exponentials, the fp32 sum, P to tensor memory over S
// P enters the product in two bf16 parts, the weight cut to 8 bits and the rest, for an error
// of 2^-16 of a weight.  (In one part the error of O against 64 bits would be 1.4 times that of
// its own rounding.)  The rest is taken of w (1 + 2^-20), so that it is above zero wherever w is
// and an infinite value meets no zero; O is divided by 1 + 2^-20 at the end.
//
// Tensor memory of a row tile (256 columns): S of two tiles (64 columns each; P's parts over it,
// 32 columns each), O behind them.
//
// What bounds it, at 128 x 32768 (1024 rows of a KV head, 86 us for the call, 87 with one row
// tile): 2230 clocks for a tile of 256 rows, of which the products alone, issued without a pause by
// the two warps, are 1773 (a product of S, 64 columns, takes 48 clocks: its 6 KB of operands at 128
// bytes a clock, where its arithmetic is 32; one of P V, 128 columns with P in tensor memory, 64) and
// a softmax warp's work 2000 (535 instructions, of which 64 exponentials, for 64 keys of 32 rows, two
// such warps to a scheduler).  The pipe's counter, 68 % over the whole kernel, counts the arithmetic:
// 1536 clocks of 2230.  Neither side alone is the bound, but the chain of S, softmax and P V over
// two row tiles: without the rests' products 82 us, without the rests 77, without copies 85.  What did
// not help: S of 128 keys at a time, or Q in tensor memory (96 and 109 us: no room for a second S),
// two threads to a row (94), one warp that issues for both row tiles (120), registers moved to the
// softmax warps (90).  Shorter
// prefixes are start and end: groups and lengths 1.2 us, first page numbers 0.7, Q and the first
// tiles 2.5; a part out 2.
#include "cache_line.cuh"

namespace avits {
namespace cache {
namespace {

using namespace tc;

constexpr int kBM = 128, kBN = 64;
constexpr int kColO = 2 * kBN;
constexpr float kRise = 8.f;               // log2: a maximum that passes the reference by more
constexpr float kUp = 1.f + 0x1p-20f;      // moves it
constexpr int kMaxStages = 8;
constexpr int kOutBytes = kBM * 16 * 4;    // 16 columns of O

// kT row tiles of 128 share the ring of keys and values.
template <int D, int kT>
struct Pre {
  static constexpr int kCB = D / 64;
  static constexpr int kTileBytes = kCB * kBN * 128;
  static constexpr int kQBytes = kCB * kBM * 128;        // of a row tile
  static constexpr int kStages = kT == 2 ? (D == 128 ? 6 : 8) : (D == 128 ? 4 : 8);
  static constexpr int kRows = kT * kBM;
  static constexpr int kThreads = 32 * (1 + kT + 4 * kT);
  static constexpr int kTmemCols = 256;                  // of a row tile
  static constexpr uint32_t kIdescS = idesc_bf16(kBM, kBN, false);
  static constexpr uint32_t kIdescPV = idesc_bf16(kBM, D, true);
};

struct TileBars {      // of a row tile
  uint64_t q_full, q_empty, o_full, o_empty, drain;
  uint64_t s_full[2], p_full[2], pv_done[2];
};
template <int kT>
struct PreBars {
  TileBars tile[kT];
  uint64_t kv_full[kMaxStages], kv_empty[kMaxStages];
  uint32_t tmem_base;
  int abort;
};

template <int D, int kT>
constexpr int pre_smem() {
  using C = Pre<D, kT>;
  return kT * (C::kQBytes + kOutBytes) + C::kStages * C::kTileBytes + (int)sizeof(PreBars<kT>);
}
// One row tile: two CTAs to an SM, of 228 KB with 1 KB of each block's kept by the system.
static_assert(2 * (pre_smem<128, 1>() + 1024) <= 228 * 1024, "two CTAs to an SM");
static_assert(pre_smem<128, 2>() <= 227 * 1024, "the opt-in limit");

// A CTA's piece of the line, segment by segment.
template <int kRows>
struct Walk {
  int g, u, t0, t1, nt, len, left, ubase, per;
  int seq, n;            // the group's first sequence, and the rows of a KV head

  __device__ __forceinline__ int units(const CacheAttn& a) const {
    return a.c.Hkv * ((n + kRows - 1) / kRows);
  }
  __device__ __forceinline__ void look(const CacheAttn& a) {
    const int2 m = members_of(a.start, a.seqs, g);
    seq = m.x;
    n = (m.y - m.x) * a.G;
    len = cache_len(a.c, g);
    nt = tiles_of(a, len);
  }
  // false: this CTA has none
  __device__ __forceinline__ bool begin(const CacheAttn& a, int lane) {
    const int B = a.c.B, each = (B + 31) / 32;
    const int b0 = min(B, lane * each), b1 = min(B, b0 + each);
    int sum = 0, usum = 0;
    bool ok = true;
    Walk mine{};                         // of the lane's last group
    for (mine.g = b0; mine.g < b1; ++mine.g) {
      mine.look(a);
      const int x = a.start[mine.g], y = a.start[mine.g + 1];
      ok = ok && x >= 0 && x <= y && y <= a.seqs;
      sum += mine.nt * mine.units(a);
      usum += mine.units(a);
    }
    int inc = sum, uinc = usum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, inc, o), z = __shfl_up_sync(0xffffffffu, uinc, o);
      if (lane >= o) {
        inc += y;
        uinc += z;
      }
    }
    const int total = __shfl_sync(0xffffffffu, inc, 31);
    int base = uinc - usum;
    // groups that do not rise could be more units than there is room for: no prefix is read
    const bool rise = __all_sync(0xffffffffu, ok);
    if (blockIdx.x == 0 && threadIdx.x < 32) {
      Walk x{};
      x.ubase = base;
      for (x.g = b0; x.g < b1; ++x.g) {
        x.look(a);
        a.base[x.g] = x.ubase;
        x.ubase += x.units(a);
        check_cache_len(a.c, x.g, a.status);
      }
      if (lane == 0) {
        a.base[B] = rise;
        if (!rise) raise_status(a.status, AVITS_ERR_PAGE);
      }
    }
    per = max(a.least, (total + a.grid - 1) / a.grid);
    const int first = blockIdx.x * per;
    if (!rise || first >= total) return false;
    int off = first - (inc - sum);
    const bool here = off >= 0 && off < sum;
    mine.g = b0;
    if (here && each > 1)
      for (;; ++mine.g) {
        mine.look(a);
        const int un = mine.units(a), tiles = mine.nt * un;
        if (off < tiles) break;
        off -= tiles;
        base += un;
      }
    const int src = __ffs(__ballot_sync(0xffffffffu, here)) - 1;
    g = __shfl_sync(0xffffffffu, mine.g, src);
    seq = __shfl_sync(0xffffffffu, mine.seq, src);
    n = __shfl_sync(0xffffffffu, mine.n, src);
    len = __shfl_sync(0xffffffffu, mine.len, src);
    off = __shfl_sync(0xffffffffu, off, src);
    ubase = __shfl_sync(0xffffffffu, base, src);
    left = min(per, total - first);
    nt = tiles_of(a, len);
    u = off / nt;
    t0 = off - u * nt;
    t1 = min(nt, t0 + left);
    return true;
  }
  __device__ __forceinline__ bool next(const CacheAttn& a) {
    left -= t1 - t0;
    if (left <= 0) return false;
    if (++u == units(a)) {
      u = 0;
      do {
        ubase += units(a);
        ++g;
        look(a);
      } while (nt == 0 || n == 0);
    }
    t0 = 0;
    t1 = min(nt, left);
    return true;
  }
  // rows of the unit's row tile t
  __device__ __forceinline__ QRows rows(const CacheAttn& a, int t) const {
    const int rg = (n + kRows - 1) / kRows, hk = u / rg, r0 = (u - hk * rg) * kRows + t * kBM;
    return QRows{seq, hk * a.G, max(0, min(kBM, n - r0)), r0, a.G};
  }
};

__device__ __forceinline__ void bar_arrive(int id, int count) {
  asm volatile("barrier.cta.arrive %0, %1;" ::"r"(id), "r"(count) : "memory");
}

// (c0, c1) += (a0, a1) * b.
__device__ __forceinline__ void fma2(float a0, float a1, float b, float& c0, float& c1) {
  asm("{\n\t.reg .b64 a, b, c;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %4};\n\t"
      "mov.b64 c, {%0, %1};\n\tfma.rn.f32x2 c, a, b, c;\n\tmov.b64 {%0, %1}, c;\n\t}"
      : "+f"(c0), "+f"(c1)
      : "f"(a0), "f"(a1), "f"(b));
}

template <int D, int kT>
// Two row tiles: at most 128 registers (86 us for 128 x 32768, 88 with 161).
__global__ void __launch_bounds__(kT == 2 ? 512 : Pre<D, kT>::kThreads, 3 - kT)
cache_prefix_kernel(const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
                    const __grid_constant__ CacheAttn a) {
  using C = Pre<D, kT>;
  extern __shared__ __align__(1024) char smem[];
  char* sKV = smem + kT * C::kQBytes;
  char* sOut = sKV + C::kStages * C::kTileBytes;
  PreBars<kT>* bars = reinterpret_cast<PreBars<kT>*>(sOut + kT * kOutBytes);
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&mk));
    asm volatile("prefetch.tensormap [%0];" ::"l"(&mv));
    for (int t = 0; t < kT; ++t) {
      TileBars& x = bars->tile[t];
      mbar_init(&x.q_full, 4);
      mbar_init(&x.q_empty, 1);
      mbar_init(&x.o_full, 1);
      mbar_init(&x.o_empty, 4);
      mbar_init(&x.drain, 1);
      for (int i = 0; i < 2; ++i) {
        mbar_init(&x.s_full[i], 1);
        mbar_init(&x.p_full[i], 4);
        mbar_init(&x.pv_done[i], 1);
      }
    }
    for (int i = 0; i < C::kStages; ++i) {
      mbar_init(&bars->kv_full[i], 1);
      mbar_init(&bars->kv_empty[i], kT);      // a commit per row tile
    }
    bars->abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_shared();
  }
  // what this call reads may come from the kernel before; the next one may start beside it
  pdl_wait();
  pdl_trigger();
  Walk<C::kRows> seg;
  if (!seg.begin(a, lane)) return;         // the whole CTA
  volatile int* abort_flag = &bars->abort;
  uint32_t tmem = 0;
  if (warp == 0) {
    bar_arrive(1, C::kThreads);            // its copies need no tensor memory
    __syncwarp();
  } else {
    if (warp == 1) tmem_alloc(&bars->tmem_base, kT * C::kTmemCols);
    fence_before();
    bar_sync(1, C::kThreads);
    fence_after();
    tmem = bars->tmem_base;
  }

  if (warp == 0) {
    // --------------------------------------------------------- producer --
    bool ok = true;
    int loads = 0;
    const int boxes = kBN / a.box;
    do {
      const int hk = seg.rows(a, 0).h0 / a.G;
      // the box of a tile that this lane brings: its page and place in it
      auto page_of = [&](int t) {
        const int j = t * kBN + lane * a.box;
        return lane < boxes && t < seg.t1 && j < seg.len
                   ? a.c.block_table[(int64_t)seg.g * a.c.table_sb + a.page.div(j)]
                   : -1;
      };
      auto load = [&](const CUtensorMap* map, int page, int t) {
        const int st = loads % C::kStages;
        ok = mbar_wait_bounded(&bars->kv_empty[st], ((uint32_t)(loads / C::kStages) & 1u) ^ 1u,
                               abort_flag, a.status);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) return;
        ++loads;
        if (lane == 0) mbar_arrive_expect_tx(&bars->kv_full[st], C::kTileBytes);
        __syncwarp();
        if (lane < boxes) {
          const int j = t * kBN + lane * a.box, place = j - a.page.div(j) * a.c.page_size;
          char* to = sKV + st * C::kTileBytes + lane * a.box * 128;
#pragma unroll
          for (int cb = 0; cb < C::kCB; ++cb)
            tma_load_4d(to + cb * (kBN * 128), map, cb * 64, hk, place, page, &bars->kv_full[st]);
        }
        __syncwarp();
      };
      int entry = page_of(seg.t0), v_page = -1;
      // in the order of the products: K(0), K(1), V(0), K(2), V(1), ...
      for (int t = seg.t0; t <= seg.t1 && ok; ++t) {
        int page = -1;
        if (t < seg.t1) {
          const int j = t * kBN + lane * a.box;
          if (lane < boxes && j < seg.len) page = checked_page(a.c, entry, a.status);
          entry = page_of(t + 1);
          load(&mk, page, t);
        }
        if (ok && t > seg.t0) load(&mv, v_page, t - 1);
        v_page = page;
      }
    } while (ok && seg.next(a));
    if (!ok)       // the copies in flight land before the CTA leaves
      for (int i = loads > C::kStages ? loads - C::kStages : 0; i < loads; ++i)
        mbar_wait_bounded(&bars->kv_full[i % C::kStages], (uint32_t)(i / C::kStages) & 1u, nullptr,
                          a.status);
  } else if (warp <= kT) {
    // --------------------------------------------------------- products --
    const int rt = warp - 1;
    TileBars* const tb = &bars->tile[rt];
    tmem += (uint32_t)(rt * C::kTmemCols);
    const uint32_t q_lo = sw128_desc_lo(smem + rt * C::kQBytes), kv_lo = sw128_desc_lo(sKV);
    const uint32_t v_lo0 = sw128_mn_desc_lo(sKV, kBN * 128), d_hi = sw128_desc_hi();
    bool ok = true;
    int loads = 0, tile = 0, n_seg = 0;
    auto wait = [&](uint64_t* bar, int phase) {
      if (ok) ok = mbar_wait_bounded(bar, (uint32_t)(phase & 1), abort_flag, a.status);
    };
    auto issue_s = [&](int at, bool last) {      // at: the tile's number
      const int st = loads % C::kStages;
      wait(&bars->kv_full[st], loads / C::kStages);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) return;
      ++loads;
      fence_after();
      if (elect_one()) {
        const uint32_t k_lo = kv_lo + (uint32_t)((st * C::kTileBytes) >> 4);
        const uint32_t tS = tmem + (uint32_t)((at & 1) * kBN);
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
          mma_ss(tS, q_lo + (uint32_t)(((kk >> 2) * (kBM * 128) + (kk & 3) * 32) >> 4),
                 k_lo + (uint32_t)(((kk >> 2) * (kBN * 128) + (kk & 3) * 32) >> 4), d_hi, C::kIdescS,
                 kk > 0 ? 1u : 0u);
        mma_commit(&tb->s_full[at & 1]);
        mma_commit(&bars->kv_empty[st]);
        if (last) mma_commit(&tb->q_empty);
      }
      __syncwarp();
    };
    do {
      const int n = seg.t1 - seg.t0;
      wait(&tb->q_full, n_seg);
      ok = __all_sync(0xffffffffu, ok);
      if (ok) issue_s(tile, n == 1);
      for (int j = 0; j < n && ok; ++j, ++tile) {
        // S(j+1) over P(j-1), whose product is before it in the pipe
        if (j + 1 < n) issue_s(tile + 1, j + 2 == n);
        if (!ok) break;
        const int st = loads % C::kStages;
        if (j == 0 && n_seg > 0) wait(&tb->o_empty, n_seg - 1);
        wait(&bars->kv_full[st], loads / C::kStages);
        wait(&tb->p_full[tile & 1], tile >> 1);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        ++loads;
        fence_after();
        if (elect_one()) {
          const uint32_t tP = tmem + (uint32_t)((tile & 1) * kBN), tO = tmem + (uint32_t)kColO;
          const uint32_t v_lo = v_lo0 + (uint32_t)((st * C::kTileBytes) >> 4);
#pragma unroll
          for (int kk = 0; kk < kBN / 16; ++kk) {
            const uint32_t v_at = v_lo + (uint32_t)((kk * 16 * 128) >> 4);
            mma_ts(tO, tP + (uint32_t)(kk * 8), v_at, d_hi, C::kIdescPV, j > 0 || kk > 0 ? 1u : 0u);
            mma_ts(tO, tP + (uint32_t)(32 + kk * 8), v_at, d_hi, C::kIdescPV, 1u);
          }
          mma_commit(&bars->kv_empty[st]);
          mma_commit(&tb->pv_done[tile & 1]);
          if (j + 1 == n) mma_commit(&tb->o_full);
        }
        __syncwarp();
      }
      ++n_seg;
    } while (ok && seg.next(a));
    // everything issued has completed before tensor memory is given back
    if (elect_one()) mma_commit(&tb->drain);
    __syncwarp();
    mbar_wait_bounded(&tb->drain, 0, nullptr, a.status);
  } else {
    // ------------------------------------------------ softmax, epilogue --
    const int quad = warp & 3, row = quad * 32 + lane;
    const int rt = (warp - 1 - kT) >> 2, part = (int)threadIdx.x - 32 * (1 + kT) - 128 * rt;
    TileBars* const tb = &bars->tile[rt];
    char* const sQ = smem + rt * C::kQBytes;
    char* const sO = sOut + rt * kOutBytes;
    tmem += (uint32_t)(rt * C::kTmemCols);
    const uint32_t lanes = (uint32_t)(quad * 32) << 16;
    const uint32_t tO = tmem + lanes + (uint32_t)kColO;
    bool ok = true;
    int tile = 0, n_seg = 0, loads = 0;
    auto wait = [&](uint64_t* bar, int phase) {
      ok = ok && *abort_flag == 0 &&
           mbar_wait_bounded(bar, (uint32_t)(phase & 1), abort_flag, a.status);
      ok = __all_sync(0xffffffffu, ok);      // what follows are accesses of a whole warp
      return ok;
    };
    // Q of a unit in the swizzled layout of the product: a warp brings its 32 rows, all
    // loads at once.  (A row to a thread, 16 bytes at a time, took 5 us for 128 rows.)
    auto put_q = [&](const QRows& h) {
      constexpr int kC = D / 8, kSide = 32 / kC, kSteps = 32 / kSide;   // pieces, rows at once
      const int c = lane % kC, side = lane / kC;
      const int64_t mine = row < h.rows ? h.at(a, row) : 0;
      const uint16_t* q = static_cast<const uint16_t*>(a.q);
      const bool vec = __all_sync(0xffffffffu, (reinterpret_cast<uintptr_t>(q + mine) & 15u) == 0);
      uint4 x[kSteps];
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        const int r = i * kSide + side;
        const uint16_t* from = q + __shfl_sync(0xffffffffu, mine, r) + c * 8;
        x[i] = make_uint4(0u, 0u, 0u, 0u);
        if (quad * 32 + r < h.rows && c * 8 < a.c.d) {
          if (vec) {
            x[i] = *reinterpret_cast<const uint4*>(from);
          } else {
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = (uint32_t)from[2 * k] | ((uint32_t)from[2 * k + 1] << 16);
            x[i] = make_uint4(w[0], w[1], w[2], w[3]);
          }
        }
      }
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        const int r = quad * 32 + i * kSide + side;
        *reinterpret_cast<uint4*>(sQ + (c >> 3) * (kBM * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4)) =
            x[i];
      }
      fence_async_shared();
      __syncwarp();
      if (lane == 0) mbar_arrive(&tb->q_full);
    };
    QRows h = seg.rows(a, rt);
    put_q(h);
    bool more = true;
    while (more) {
      const int n = seg.t1 - seg.t0;
      const int slot = seg.ubase + seg.u + (int)blockIdx.x;
      if (seg.t0 == 0 && part == 0 && rt == 0) {
        // pieces of this unit: this CTA's and those of the CTAs that the rest reaches
        const int over = seg.nt - seg.left;
        a.rec[seg.ubase + seg.u] =
            make_int2(slot, over <= 0 ? 1 : 1 + (over + seg.per - 1) / seg.per);
      }
      // Which keys of a tile are there: those below the length whose page is one of the pool.  Each
      // warp looks that up by itself, a tile ahead: told by the producer through a barrier, it
      // cost 250 clocks of a tile's 2200.
      auto entry_of = [&](int t) {
        const int at = t * kBN + lane * a.box;
        return lane * a.box < kBN && t < seg.t1 && at < seg.len
                   ? a.c.block_table[(int64_t)seg.g * a.c.table_sb + a.page.div(at)]
                   : -1;
      };
      int entry = entry_of(seg.t0);
      float m = -INFINITY, l = 0.f;
      for (int j = 0; j < n; ++j, ++tile) {
        const uint32_t tS = tmem + lanes + (uint32_t)((tile & 1) * kBN);
        const int t = seg.t0 + j;
        const bool page_ok = (unsigned)entry < (unsigned)a.c.num_pages;
        unsigned long long mask = ~0ull;
        if ((t + 1) * kBN > seg.len || !__all_sync(0xffffffffu, page_ok || lane * a.box >= kBN)) {
          unsigned long long bits = 0;
          const int at = t * kBN + lane * a.box, here = min(a.box, seg.len - at);
          if (page_ok && lane * a.box < kBN)
            bits = (here >= 64 ? ~0ull : (1ull << here) - 1ull) << (lane * a.box);
          mask = (unsigned long long)__reduce_or_sync(0xffffffffu, (unsigned)(bits >> 32)) << 32 |
                 __reduce_or_sync(0xffffffffu, (unsigned)bits);
        }
        entry = entry_of(t + 1);
        if (!wait(&tb->s_full[tile & 1], tile >> 1)) break;
        fence_after();
        uint32_t r0[32], r1[32];
        tmem_ld64_wait(tS, r0, r1);
        if (mask != ~0ull) {
          const uint32_t m0 = (uint32_t)mask, m1 = (uint32_t)(mask >> 32);
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            if (!((m0 >> e) & 1u)) r0[e] = 0xff800000u;
            if (!((m1 >> e) & 1u)) r1[e] = 0xff800000u;
          }
        }
        float t4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int e = 0; e < 32; ++e)
          t4[e & 3] = max3(t4[e & 3], __uint_as_float(r0[e]), __uint_as_float(r1[e]));
        const float top = fmaxf(fmaxf(t4[0], t4[1]), fmaxf(t4[2], t4[3])) * a.scale2;
        const bool up = top > m + kRise || (m == -INFINITY && top > m);
        if (__any_sync(0xffffffffu, up)) {
          const float mn = up ? top : m, f = up ? avits::ex2(m - mn) : 1.f;
          m = mn;
          l *= f;
          if (j > 0) {
            if (!wait(&tb->pv_done[(tile - 1) & 1], (tile - 1) >> 1)) break;
            fence_after();
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
              uint32_t x[32];
              tmem_ld32_wait(tO + (uint32_t)c, x);
#pragma unroll
              for (int e = 0; e < 32; ++e) x[e] = __float_as_uint(__uint_as_float(x[e]) * f);
              tmem_st32(tO + (uint32_t)c, x);
            }
          }
        }
        const float nm = m == -INFINITY ? 0.f : -m;
        float s4[4] = {0.f, 0.f, 0.f, 0.f};
        // Half of the tile at a time (registers): of keys 2e, 2e + 1 the weights cut to bf16 and
        // their rests, to columns e and 32 + e.
        auto half = [&](const uint32_t (&r)[32], int at) {
          uint32_t hi[16], lo[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            float x0, x1;
            ffma2(__uint_as_float(r[2 * e]), __uint_as_float(r[2 * e + 1]), a.scale2, nm, x0, x1);
            x0 = avits::ex2(x0);
            x1 = avits::ex2(x1);
            fadd2(s4[2 * (e & 1)], s4[2 * (e & 1) + 1], x0, x1);
            hi[e] = __byte_perm(__float_as_uint(x0), __float_as_uint(x1), 0x7632);
            float y0 = __uint_as_float((__float_as_uint(x0) & 0xffff0000u) ^ 0x80000000u);
            float y1 = __uint_as_float((__float_as_uint(x1) & 0xffff0000u) ^ 0x80000000u);
            fma2(x0, x1, kUp, y0, y1);
            lo[e] = pack_bf16x2(y0, y1);
          }
          tmem_st16(tS + (uint32_t)at, hi);
          tmem_st16(tS + 32u + (uint32_t)at, lo);
        };
        half(r0, 0);
        half(r1, 16);
        l += (s4[0] + s4[1]) + (s4[2] + s4[3]);
        tmem_wait_st();
        if (mask != ~0ull) {
          // values that are not there: a weight of zero times a NaN is one
          const int v_at = loads + (j + 1 < n ? 2 * j + 2 : 2 * n - 1), st = v_at % C::kStages;
          if (!wait(&bars->kv_full[st], v_at / C::kStages)) break;
          char* v = sKV + st * C::kTileBytes;
          for (int i = part; i < kBN * C::kCB * 8; i += 128) {
            const int key = i / (C::kCB * 8), c = i - key * (C::kCB * 8);
            if (!((mask >> key) & 1ull))
              *reinterpret_cast<uint4*>(v + (c >> 3) * (kBN * 128) + key * 128 +
                                        (((c & 7) ^ (key & 7)) << 4)) = make_uint4(0u, 0u, 0u, 0u);
          }
          fence_async_shared();
        }
        fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&tb->p_full[tile & 1]);
      }
      if (!ok) break;
      loads += 2 * n;
      const int rows = h.rows;
      more = seg.next(a);
      if (more) {      // the next unit's Q, while the last product runs
        if (!wait(&tb->q_empty, n_seg)) break;
        h = seg.rows(a, rt);
        put_q(h);
      }
      if (!wait(&tb->o_full, n_seg)) break;
      fence_after();
      // O by 16 columns through shared memory, so that a row's go out as whole sectors
#pragma unroll 1
      for (int c = 0; c < D; c += 32) {
        uint32_t x[32];
        tmem_ld32_wait(tO + (uint32_t)c, x);
        if (c + 32 >= D) {        // O has been read
          fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&tb->o_empty);
        }
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          float4* buf = reinterpret_cast<float4*>(sO);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            buf[row * 4 + (e ^ ((row >> 1) & 3))] =
                make_float4(__uint_as_float(x[16 * hf + 4 * e]) * (1.f / kUp),
                            __uint_as_float(x[16 * hf + 4 * e + 1]) * (1.f / kUp),
                            __uint_as_float(x[16 * hf + 4 * e + 2]) * (1.f / kUp),
                            __uint_as_float(x[16 * hf + 4 * e + 3]) * (1.f / kUp));
          __syncwarp();
          const int col = lane & 3, at = c + 16 * hf + col * 4;
          if (at < a.c.d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int r = quad * 32 + i * 8 + (lane >> 2);
              if (r < rows)
                *reinterpret_cast<float4*>(a.po + ((int64_t)slot * C::kRows + rt * kBM + r) * a.c.d + at) =
                    buf[r * 4 + (col ^ ((r >> 1) & 3))];
            }
          __syncwarp();
        }
      }
      if (row < rows) a.pml[slot * C::kRows + rt * kBM + row] = make_float2(m, l);
      ++n_seg;
    }
  }
  fence_before();
  __syncthreads();
  if (warp == 1) {
    fence_after();
    tmem_dealloc(bars->tmem_base, kT * C::kTmemCols);
  }
}

template <int D, int kT>
cudaError_t launch_width(const CacheAttn& a, cudaStream_t s) {
  CUtensorMap mk{}, mv{};
  using Rows = RowsBf16<D, 8>;
  const avits_kv_cache& c = a.c;
  if (!map_pages<Rows>(&mk, c.k_pages, c.k_sp, c.k_st, c.k_sh, c, a.box) ||
      !map_pages<Rows>(&mv, c.v_pages, c.v_sp, c.v_st, c.v_sh, c, a.box))
    return cudaErrorInvalidValue;
  constexpr auto kernel = cache_prefix_kernel<D, kT>;
  const cudaError_t e = prefer_max_shared<kernel, pre_smem<D, kT>()>();
  if (e != cudaSuccess) return e;
  return launch_pdl(kernel, dim3(a.grid), dim3(Pre<D, kT>::kThreads), pre_smem<D, kT>(), s, mk, mv, a);
}

}  // namespace

int prefix_tc_box(const avits_kv_cache& c) {
  if (c.dt != AVITS_BF16 || c.d > 128 || c.page_size % 8 || !encode_fn()) return 0;
  // what a tensor map takes; a stride of an axis of one entry is never used
  const int64_t n[3] = {c.num_pages, c.page_size, c.Hkv};
  const int64_t st[2][3] = {{c.k_sp, c.k_st, c.k_sh}, {c.v_sp, c.v_st, c.v_sh}};
  for (int i = 0; i < 2; ++i)
    for (int x = 0; x < 3; ++x)
      if (n[x] > 1 && (st[i][x] <= 0 || st[i][x] >= (1ll << 39))) return 0;
  int box = kBN;
  while (c.page_size % box) box /= 2;
  return box;
}

cudaError_t launch_prefix_tc(const CacheAttn& a, cudaStream_t s) {
  if (a.rows == kBM) return a.c.d <= 64 ? launch_width<64, 1>(a, s) : launch_width<128, 1>(a, s);
  return a.c.d <= 64 ? launch_width<64, 2>(a, s) : launch_width<128, 2>(a, s);
}

}  // namespace cache
}  // namespace avits
