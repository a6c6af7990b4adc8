// cache_attention.cu — attention of one new token per sequence over a paged
// key-value cache, with the weight each cached token got.
//
// For sequence b, KV head hk and the G query heads h that share it:
//   x_hj = scale q_h . k_j,  lse_h = log sum_j exp x_hj,  o_h = sum_j exp(x_hj - lse_h) v_j,
//   acc_j (+)= weight mean_h exp(x_hj - lse_h)
// Every key and value is read once, so HBM bounds it: 4 G operations per bf16
// element of K and V.
//
// Split.  A sequence's keys are cut into tiles; all tiles of all units (b, hk,
// row group) form one line, cut into equal pieces, one per CTA, so that uneven
// lengths and few heads load the SMs alike.  A CTA finds its piece by a scan of
// the lengths.  Its warps take the piece's tiles in turn, each with a running
// maximum, sum and O in registers and a ring of tiles of its own in shared
// memory, filled by TMA copies that run ahead over unit borders; the warps meet
// once per unit.  A unit that lies in one piece is finished there; of the others
// each piece leaves its maximum, sum and O, and a second kernel joins them, in the
// pieces' order.  The weights need the whole row's lse: the first kernel leaves the
// logits (fp32), the second sums exp(x - lse) over the group's heads, in a fixed
// order.
//
// Shorter sequences take one launch: a cluster of CTAs per unit, whose logits
// stay in shared memory.
#include <cooperative_groups.h>

#include "cache_common.cuh"
#include "avits_internal.h"
#include "tc_common.cuh"

namespace cg = cooperative_groups;

namespace avits {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kMinTiles = 4;      // tiles of the smallest piece: one per warp
constexpr int kMaxGrid = 1024;
constexpr unsigned long long kLateNs = 1000ull * 1000ull;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct CacheAttn {
  avits_kv_cache c;
  FastDiv page;
  const void* q;
  void* o;
  int64_t q_sb, q_sh, o_sb, o_sh;
  float* lse;
  int H, G;
  int rows;         // rows (query heads) of a unit
  int groups;       // units per KV head: ceil(G / rows)
  int tile;         // keys per tile
  int grid;         // CTAs of the first kernel
  int box;          // tokens of a TMA box; 0: rows come by 16-byte copies
  int score;        // weights wanted: logits are kept
  int few;          // units have few pieces each
  float scale2;     // scale * log2(e)
  float wmean;      // weight / G
  int add;
  // workspace
  int2* rec;        // [B units] first part of a unit and its pieces; one: it is in lse2
  int4* own;        // [grid] unit whose first piece is the CTA's, of several: (unit or -1,
                    // first part, pieces); read where units have few pieces
  float* lse2;      // [B,H] log2-domain lse of rows finished in one piece
  float2* pml;      // [2 grid][rows] maximum and sum of a piece's row
  float* po;        // [2 grid][rows][d] its O
  float* logits;    // [B,H,ld] log2-domain logits (weights wanted)
  int64_t ld;
  unsigned int* status;
};

__device__ __forceinline__ int tiles_of(const CacheAttn& a, int len) {
  return (len + a.tile - 1) / a.tile;
}

// 16 bytes from global to shared memory; zeros where !ok (nothing is read).
__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool ok) {
  const int n = ok ? 16 : 0;
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n));
}
// `bar` gets this thread's arrival when its 16-byte copies so far are done.
__device__ __forceinline__ void cp_arrive(uint64_t* bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar))
               : "memory");
}
// Orders this thread's accesses of shared memory before later bulk copies into it.
__device__ __forceinline__ void before_copies() {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

// A warp's place on the line of tiles: what it copies next.
struct Cursor {
  int b, u, t;      // sequence, unit in it, tile in the unit
  int nt, len;
  int left;         // tiles still to come
  int entry;        // table entry: of this lane's key, or of its box, of that tile

  __device__ __forceinline__ void settle(const CacheAttn& a, int units) {
    while (t >= nt) {
      t -= nt;
      if (++u == units) {
        u = 0;
        do {
          len = cache_len(a.c, ++b);
          nt = tiles_of(a, len);
        } while (nt == 0);
      }
    }
  }
  template <int kTile>
  __device__ __forceinline__ void look_up(const CacheAttn& a, int lane) {
    const int j = t * kTile + (a.box ? lane * a.box & (kTile - 1) : lane & (kTile - 1));
    entry = j < len ? a.c.block_table[(int64_t)b * a.c.table_sb + a.page.div(j)] : -1;
  }
};

// Copies the cursor's tile to `dst`, keys then values, and steps on.  `mask` gets
// a bit for each key that is there (below the length, its page in range).  A tile
// lies as columns of 128 bytes: in bf16 [D / 64][16 rows][128 bytes] with the
// 16-byte pieces of row r at c ^ (r % 8) (TMA's 128-byte swizzle, for ldmatrix),
// in fp32 plain rows.  By TMA where boxes of 16 or 8 tokens never cross a page:
// what lies outside the tensors (columns past the width, a page out of range)
// comes as zeros.  Else by 16-byte copies, a row's pieces side by side, zeros past
// the width.  So the products run over whole widths of 64, 128 or 256 unchecked.
template <typename Rows>
__device__ __forceinline__ void copy_tile(const CUtensorMap& mk, const CUtensorMap& mv,
                                          const CacheAttn& a, Cursor& cur, char* dst, uint64_t* bar,
                                          uint32_t* mask, int units, int lane) {
  constexpr int kTile = Rows::kTile, kEs = sizeof(typename Rows::T), D = Rows::D;
  const int hk = a.groups == 1 ? cur.u : cur.u / a.groups;
  const int j0 = cur.t * kTile;
  unsigned ok;
  if (a.box) {
    const int jb = j0 + (lane * a.box & (kTile - 1));
    const int page = jb < cur.len ? checked_page(a.c, cur.entry, a.status) : -1;
    int p0 = page, p1 = page;        // one box: the same page in all lanes
    const int n = cur.len - j0;
    ok = n >= kTile ? (1u << kTile) - 1u : (1u << n) - 1u;
    if (a.box == kTile) {
      if (page < 0) ok = 0u;
    } else {
      p0 = __shfl_sync(0xffffffffu, page, 0);
      p1 = __shfl_sync(0xffffffffu, page, 1);
      if (p0 < 0) ok &= ~((1u << a.box) - 1u);
      if (p1 < 0) ok &= (1u << a.box) - 1u;
    }
    if (tc::elect_one()) {
      mbar_arrive_expect_tx(bar, Rows::kStage);
#pragma unroll 1
      for (int at = 0; at < kTile; at += a.box) {
        const int jj = j0 + at, slot = jj - a.page.div(jj) * a.c.page_size, pg = at ? p1 : p0;
#pragma unroll
        for (int c = 0; c < Rows::kCols; ++c) {
          char* to = dst + c * Rows::kColBytes + at * Rows::kColPitch;
          tc::tma_load_4d(to, &mk, c * Rows::kColWidth, hk, slot, pg, bar);
          tc::tma_load_4d(to + Rows::kStage / 2, &mv, c * Rows::kColWidth, hk, slot, pg, bar);
        }
      }
    }
  } else {
    constexpr int kPieces = D * kEs / 16;
    constexpr int kSide = kPieces < 32 ? 32 / kPieces : 1;       // rows side by side
    constexpr int kSteps = kPieces < 32 ? 1 : kPieces / 32;      // steps along a row
    const int side = kPieces < 32 ? lane / kPieces : 0;
    const int piece = kPieces < 32 ? lane % kPieces : lane;
    const int some = a.c.d * kEs / 16;
    const int j = j0 + (lane & (kTile - 1));
    const int page = j < cur.len ? checked_page(a.c, cur.entry, a.status) : -1;
    ok = __ballot_sync(0xffffffffu, page >= 0) & ((1u << kTile) - 1u);
    const int slot = j - a.page.div(j) * a.c.page_size;
    // lanes below 16 hold the key's offset, the others the value's
    const int64_t off = page < 0 ? 0
                        : lane < 16
                            ? (int64_t)page * a.c.k_sp + (int64_t)slot * a.c.k_st + hk * a.c.k_sh
                            : (int64_t)page * a.c.v_sp + (int64_t)slot * a.c.v_st + hk * a.c.v_sh;
#pragma unroll
    for (int i = 0; i < kTile / kSide; ++i) {
      const int row = i * kSide + side;
      const int64_t ko = __shfl_sync(0xffffffffu, off, row) * kEs;
      const int64_t vo = __shfl_sync(0xffffffffu, off, row + 16) * kEs;
#pragma unroll
      for (int st = 0; st < kSteps; ++st) {
        const int c = piece + 32 * st;
        const bool there = ((ok >> row) & 1u) && c < some;
        const uint32_t to = smem_u32(dst) + Rows::piece_at(row, c);
        cp16(to, static_cast<const char*>(a.c.k_pages) + ko + c * 16, there);
        cp16(to + Rows::kStage / 2, static_cast<const char*>(a.c.v_pages) + vo + c * 16, there);
      }
    }
    cp_arrive(bar);
  }
  if (lane == 0) *mask = ok;
  if (--cur.left > 0) {
    cur.t += kWarps;
    cur.settle(a, units);
    cur.look_up<kTile>(a, lane);
  }
}

// A tile that has come: value rows that are not there are set to zero, since a
// weight of zero times a NaN is one.
template <typename Rows>
__device__ __forceinline__ void clear_rows(char* st, unsigned mask, int lane) {
  constexpr int kPieces = Rows::D * (int)sizeof(typename Rows::T) / 16;
  for (int i = lane; i < Rows::kTile * kPieces; i += 32) {
    const int row = i / kPieces, c = i - row * kPieces;
    if (!((mask >> row) & 1u))
      *reinterpret_cast<uint4*>(st + Rows::kStage / 2 + Rows::piece_at(row, c)) =
          make_uint4(0u, 0u, 0u, 0u);
  }
  before_copies();
  __syncwarp();
}

// The place of O's column d of a row in a warp's buffer (bank conflicts).
__device__ __forceinline__ int o_at(int row, int d, int D) {
  return row * D + ((((d >> 3) ^ (row & 7)) << 3) | (d & 7));
}

// ------------------------------------------------------------------ bf16 --
// m16n8k16, heads in the rows.  kR = 8 heads or fewer: the weights enter P V as
// two bf16 parts (value and rest, 16 significant bits together), the value in
// rows 0-7 and the rest in rows 8-15, which are free.  kR = 16, 32: one or two
// row tiles, the rest in a second product.  Either way O is as exact as with
// weights in fp32.
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                         uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
      "{%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ void ldsm2(uint32_t& r0, uint32_t& r1, uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x2.shared.b16 {%0,%1}, [%2];"
               : "=r"(r0), "=r"(r1)
               : "r"(at)
               : "memory");
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

template <int D_, int kR_>
struct RowsBf16 {
  using T = __nv_bfloat16;
  static constexpr int D = D_, kR = kR_;
  static constexpr bool kSplit8 = kR == 8;
  static constexpr int kM = kR == 32 ? 2 : 1;      // row tiles
  static constexpr int kTile = 16;
  static constexpr bool kBf16 = true;
  static constexpr int kStage = 2 * kTile * D * 2;
  static constexpr int kCols = D / 64, kColWidth = 64, kColPitch = 128;
  static constexpr int kColBytes = kTile * kColPitch;
  static constexpr int kQBytes = kR * D * 2;
  static constexpr int kQPieces = kQBytes / 16;
  static constexpr int kBufRows = kR < 16 ? kR : 16;     // rows of O in a free stage
  static constexpr int kWarpBytes = 0;

  float m[kM][2], l[kM][2];        // of rows g and g + 8 of a row tile
  float o[kM][D / 8][4];

  // 16-byte piece c of a row of a tile
  __device__ static __forceinline__ int piece_at(int row, int c) {
    return (c >> 3) * kColBytes + row * kColPitch + (((c & 7) ^ (row & 7)) << 4);
  }

  // 16 bytes of Q: piece i of the unit's rows
  __device__ static __forceinline__ uint4 load_q(const CacheAttn& a, int b, int h0, int rows,
                                                 int i) {
    const int row = i / (D / 8), d = (i % (D / 8)) * 8;
    uint32_t w[4] = {0u, 0u, 0u, 0u};
    if (row < rows && d < a.c.d) {
      const uint16_t* q = static_cast<const uint16_t*>(a.q) + (int64_t)b * a.q_sb +
                          (int64_t)(h0 + row) * a.q_sh + d;
      if ((reinterpret_cast<uintptr_t>(q) & 15u) == 0) return *reinterpret_cast<const uint4*>(q);
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] = (uint32_t)q[2 * k] | ((uint32_t)q[2 * k + 1] << 16);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ static __forceinline__ void store_q(char* sq, int i, const uint4& v) {
    const int row = i / (D / 8), c = i % (D / 8);
    *reinterpret_cast<uint4*>(sq + (c >> 3) * kR * 128 + row * 128 +
                              (((c & 7) ^ (row & 7)) << 4)) = v;
  }

  __device__ __forceinline__ void reset() {
#pragma unroll
    for (int mt = 0; mt < kM; ++mt) {
      m[mt][0] = m[mt][1] = -INFINITY;
      l[mt][0] = l[mt][1] = 0.f;
#pragma unroll
      for (int j = 0; j < D / 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[mt][j][e] = 0.f;
    }
  }

  // one tile; lg: the logits of row g of row tile 0 at the tile's first key
  __device__ __forceinline__ void tile(const CacheAttn& a, uint32_t kt, const char* sq, char*,
                                       uint32_t mask, float* lg, int64_t ld, int rows, int lane) {
    const int g = lane >> 2, t = lane & 3, r8 = lane & 7;
    float s[kM][2][4] = {};
    {
      const int krow = r8 + ((lane >> 4) << 3), kc = (lane >> 3) & 1;
      const int qrow = kSplit8 ? r8 : r8 + (((lane >> 3) & 1) << 3);
      const int qc = kSplit8 ? (lane >> 3) & 1 : lane >> 4;
      const uint32_t kx = (kc ^ r8) << 4, qx = (qc ^ r8) << 4;
      const uint32_t kat = kt + krow * 128, qat = smem_u32(sq) + qrow * 128;
#pragma unroll
      for (int st = 0; st < D / 16; ++st) {
        uint32_t k[4];
        ldsm4(k, kat + (st >> 2) * kColBytes + (kx ^ ((st & 3) << 5)));
#pragma unroll
        for (int mt = 0; mt < kM; ++mt) {
          uint32_t q[4] = {0u, 0u, 0u, 0u};
          const uint32_t at = qat + (st >> 2) * kR * 128 + mt * 16 * 128 + (qx ^ ((st & 3) << 5));
          if (kSplit8) ldsm2(q[0], q[2], at); else ldsm4(q, at);
          mma16816(s[mt][0], q[0], q[1], q[2], q[3], k[0], k[1]);
          mma16816(s[mt][1], q[0], q[1], q[2], q[3], k[2], k[3]);
        }
      }
    }
    // keys 2t, 2t+1 (s[.][0]) and 8+2t, 9+2t (s[.][1]); rows g (e 0, 1), g + 8 (e 2, 3)
    uint32_t p[kM][4], r[kM][4];     // A fragments of the weights and their rests
    bool raise = false;
    float top[kM][2];
#pragma unroll
    for (int mt = 0; mt < kM; ++mt) {
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[mt][n][e] *= a.scale2;
      if (mask != (1u << kTile) - 1u) {
        const unsigned here = mask >> (2 * t);
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!((here >> (8 * n + (e & 1))) & 1u)) s[mt][n][e] = -INFINITY;
      }
      if (a.score) {
#pragma unroll
        for (int hf = 0; hf < (kSplit8 ? 1 : 2); ++hf) {
          const int row = mt * 16 + hf * 8 + g;
          if (row < rows) {
            float2* to = reinterpret_cast<float2*>(lg + (mt * 16 + hf * 8) * ld + 2 * t);
            to[0] = make_float2(s[mt][0][2 * hf], s[mt][0][2 * hf + 1]);
            to[4] = make_float2(s[mt][1][2 * hf], s[mt][1][2 * hf + 1]);
          }
        }
      }
#pragma unroll
      for (int hf = 0; hf < (kSplit8 ? 1 : 2); ++hf) {
        float x = fmaxf(fmaxf(s[mt][0][2 * hf], s[mt][0][2 * hf + 1]),
                        fmaxf(s[mt][1][2 * hf], s[mt][1][2 * hf + 1]));
        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
        top[mt][hf] = x;
        raise |= x > m[mt][hf];
      }
    }
    if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
      for (int mt = 0; mt < kM; ++mt) {
        float f[2] = {1.f, 1.f};
#pragma unroll
        for (int hf = 0; hf < (kSplit8 ? 1 : 2); ++hf) {
          const float mn = fmaxf(m[mt][hf], top[mt][hf]);
          f[hf] = mn == m[mt][hf] ? 1.f : ex2(m[mt][hf] - mn);   // from -inf: 0
          m[mt][hf] = mn;
          l[mt][hf] *= f[hf];
        }
        if (kSplit8) f[1] = f[0];
#pragma unroll
        for (int j = 0; j < D / 8; ++j) {
          o[mt][j][0] *= f[0];
          o[mt][j][1] *= f[0];
          o[mt][j][2] *= f[1];
          o[mt][j][3] *= f[1];
        }
      }
    }
#pragma unroll
    for (int mt = 0; mt < kM; ++mt) {
#pragma unroll
      for (int hf = 0; hf < (kSplit8 ? 1 : 2); ++hf) {
        const float ref = m[mt][hf] == -INFINITY ? 0.f : m[mt][hf];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          const float x0 = ex2(s[mt][n][2 * hf] - ref), x1 = ex2(s[mt][n][2 * hf + 1] - ref);
          l[mt][hf] += x0 + x1;
          const uint32_t both = pack_bf16(x0, x1);
          const uint32_t rest = pack_bf16(x0 - bf16_lo(both), x1 - bf16_hi(both));
          p[mt][2 * n + hf] = both;
          if (kSplit8) p[mt][2 * n + 1] = rest; else r[mt][2 * n + hf] = rest;
        }
      }
    }
    {
      const int vrow = r8 + (((lane >> 3) & 1) << 3), vc = lane >> 4;
      const uint32_t vx = (vc ^ r8) << 4, vat = kt + kStage / 2 + vrow * 128;
#pragma unroll
      for (int j = 0; j < D / 16; ++j) {
        uint32_t v[4];
        ldsm4t(v, vat + (j >> 2) * kColBytes + (vx ^ ((j & 3) << 5)));
#pragma unroll
        for (int mt = 0; mt < kM; ++mt) {
          mma16816(o[mt][2 * j], p[mt][0], p[mt][1], p[mt][2], p[mt][3], v[0], v[1]);
          mma16816(o[mt][2 * j + 1], p[mt][0], p[mt][1], p[mt][2], p[mt][3], v[2], v[3]);
          if (!kSplit8) {
            mma16816(o[mt][2 * j], r[mt][0], r[mt][1], r[mt][2], r[mt][3], v[0], v[1]);
            mma16816(o[mt][2 * j + 1], r[mt][0], r[mt][1], r[mt][2], r[mt][3], v[2], v[3]);
          }
        }
      }
    }
  }

  // rows [16 part, 16 part + kBufRows) of this warp: (maximum, sum), and O
  __device__ __forceinline__ void put(int part, float2* ml, float* buf, int lane) {
    const int g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int mt = 0; mt < kM; ++mt) {
      if (mt != part) continue;
#pragma unroll
      for (int hf = 0; hf < (kSplit8 ? 1 : 2); ++hf) {
        float x = l[mt][hf];
        x += __shfl_xor_sync(0xffffffffu, x, 1);
        x += __shfl_xor_sync(0xffffffffu, x, 2);
        if (t == 0) ml[g + 8 * hf] = make_float2(m[mt][hf], x);
      }
#pragma unroll
      for (int j = 0; j < D / 8; ++j) {
        const float* x = o[mt][j];
        if (kSplit8) {
          *reinterpret_cast<float2*>(buf + o_at(g, 8 * j + 2 * t, D)) =
              make_float2(x[0] + x[2], x[1] + x[3]);
        } else {
          *reinterpret_cast<float2*>(buf + o_at(g, 8 * j + 2 * t, D)) = make_float2(x[0], x[1]);
          *reinterpret_cast<float2*>(buf + o_at(g + 8, 8 * j + 2 * t, D)) =
              make_float2(x[2], x[3]);
        }
      }
    }
  }
};

// ------------------------------------------------------------------ fp32 --
// CUDA cores in fp32, 8 heads.  Q K^T: 8 lanes to a key (16-byte pieces of its
// row), 4 keys at a time; a lane's partial dot products of the 8 heads are
// summed over the 8 lanes by halving, which leaves head lane % 8 with the lane.
// P V: a lane owns columns of O and reads the weights from shared memory.
template <int D_, int>
struct RowsF32 {
  using T = float;
  static constexpr int D = D_, kR = 8;
  static constexpr int kTile = 8;
  static constexpr bool kBf16 = false;
  static constexpr int kStage = 2 * kTile * D * 4;
  static constexpr int kCols = 1, kColWidth = 0, kColPitch = D * 4, kColBytes = 0;
  static constexpr int kQBytes = kR * D * 4;
  static constexpr int kQPieces = kQBytes / 16;
  static constexpr int kBufRows = kR, kM = 1;
  static constexpr int kWarpBytes = kTile * 8 * 4;
  static constexpr int kKeysPerV = D >= 128 ? 1 : 128 / D;   // value rows read side by side
  static constexpr int kV = D >= 128 ? D / 128 : 1;

  float m, l;            // of row lane % 8; l: this lane's keys only until the end
  float o[8][kV][4];

  __device__ static __forceinline__ int piece_at(int row, int c) { return row * kColPitch + c * 16; }

  __device__ static __forceinline__ uint4 load_q(const CacheAttn& a, int b, int h0, int rows,
                                                 int i) {
    const int row = i / (D / 4), d = (i % (D / 4)) * 4;
    if (row >= rows || d >= a.c.d) return make_uint4(0u, 0u, 0u, 0u);
    const uint32_t* q = static_cast<const uint32_t*>(a.q) + (int64_t)b * a.q_sb +
                        (int64_t)(h0 + row) * a.q_sh + d;
    return make_uint4(q[0], q[1], q[2], q[3]);
  }
  __device__ static __forceinline__ void store_q(char* sq, int i, const uint4& v) {
    reinterpret_cast<uint4*>(sq)[i] = v;
  }

  __device__ __forceinline__ void reset() {
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int g = 0; g < 8; ++g)
#pragma unroll
      for (int c = 0; c < kV; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[g][c][e] = 0.f;
  }

  __device__ __forceinline__ void tile(const CacheAttn& a, uint32_t, const char* sq, char* sw,
                                       uint32_t mask, float* lg, int rows, int lane,
                                       const char* st) {
    const int kg = lane >> 3, t8 = lane & 7;
    const float* q = reinterpret_cast<const float*>(sq);
    const float* kt = reinterpret_cast<const float*>(st);
    const float* vt = kt + kTile * D;
    float* sp = reinterpret_cast<float*>(sw);
    // a lane's keys: 2 kg, 2 kg + 1
    float s[2][8] = {};
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      const int d = c * 32 + t8 * 4;
      const float4 k0 = *reinterpret_cast<const float4*>(kt + (2 * kg) * D + d);
      const float4 k1 = *reinterpret_cast<const float4*>(kt + (2 * kg + 1) * D + d);
#pragma unroll
      for (int g = 0; g < 8; ++g) {
        const float4 qv = *reinterpret_cast<const float4*>(q + g * D + d);
        s[0][g] = fmaf(qv.x, k0.x, fmaf(qv.y, k0.y, fmaf(qv.z, k0.z, fmaf(qv.w, k0.w, s[0][g]))));
        s[1][g] = fmaf(qv.x, k1.x, fmaf(qv.y, k1.y, fmaf(qv.z, k1.z, fmaf(qv.w, k1.w, s[1][g]))));
      }
    }
    float x[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float h4[4], h2[2];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float mine = (t8 & 4) ? s[i][j + 4] : s[i][j], give = (t8 & 4) ? s[i][j] : s[i][j + 4];
        h4[j] = mine + __shfl_xor_sync(0xffffffffu, give, 4);
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float mine = (t8 & 2) ? h4[j + 2] : h4[j], give = (t8 & 2) ? h4[j] : h4[j + 2];
        h2[j] = mine + __shfl_xor_sync(0xffffffffu, give, 2);
      }
      const float mine = (t8 & 1) ? h2[1] : h2[0], give = (t8 & 1) ? h2[0] : h2[1];
      const float dot = mine + __shfl_xor_sync(0xffffffffu, give, 1);
      x[i] = (mask >> (2 * kg + i)) & 1u ? dot * a.scale2 : -INFINITY;
    }
    if (a.score && t8 < rows)
      *reinterpret_cast<float2*>(lg + 2 * kg) = make_float2(x[0], x[1]);
    float top = fmaxf(x[0], x[1]);
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
    if (__any_sync(0xffffffffu, top > m)) {
      const float mn = fmaxf(m, top);
      const float f = mn == m ? 1.f : ex2(m - mn);
      m = mn;
      l *= f;
#pragma unroll
      for (int g = 0; g < 8; ++g) {
        const float fg = __shfl_sync(0xffffffffu, f, g);
#pragma unroll
        for (int c = 0; c < kV; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[g][c][e] *= fg;
      }
    }
    const float ref = m == -INFINITY ? 0.f : m;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float p = ex2(x[i] - ref);
      l += p;
      sp[(2 * kg + i) * 8 + t8] = p;
    }
    __syncwarp();
    const int sub = kKeysPerV == 1 ? 0 : lane / (32 / kKeysPerV);
    const int col = kKeysPerV == 1 ? lane * 4 : (lane % (32 / kKeysPerV)) * 4;
#pragma unroll
    for (int j = 0; j < kTile / kKeysPerV; ++j) {
      const int key = j * kKeysPerV + sub;
      const float4* pp = reinterpret_cast<const float4*>(sp + key * 8);
      const float4 pa = pp[0], pb = pp[1];
      const float p[8] = {pa.x, pa.y, pa.z, pa.w, pb.x, pb.y, pb.z, pb.w};
#pragma unroll
      for (int c = 0; c < kV; ++c) {
        const float4 v = *reinterpret_cast<const float4*>(vt + key * D + col + c * 128);
#pragma unroll
        for (int g = 0; g < 8; ++g) {
          o[g][c][0] = fmaf(p[g], v.x, o[g][c][0]);
          o[g][c][1] = fmaf(p[g], v.y, o[g][c][1]);
          o[g][c][2] = fmaf(p[g], v.z, o[g][c][2]);
          o[g][c][3] = fmaf(p[g], v.w, o[g][c][3]);
        }
      }
    }
  }
  __device__ __forceinline__ void put(int, float2* ml, float* buf, int lane) {
    float x = l;
    x += __shfl_xor_sync(0xffffffffu, x, 8);
    x += __shfl_xor_sync(0xffffffffu, x, 16);
    if (lane < 8) ml[lane] = make_float2(m, x);
#pragma unroll
    for (int g = 0; g < 8; ++g)
#pragma unroll
      for (int c = 0; c < kV; ++c) {
        float4 v = make_float4(o[g][c][0], o[g][c][1], o[g][c][2], o[g][c][3]);
        if (kKeysPerV > 1) {
          v.x += __shfl_xor_sync(0xffffffffu, v.x, 16);
          v.y += __shfl_xor_sync(0xffffffffu, v.y, 16);
          v.z += __shfl_xor_sync(0xffffffffu, v.z, 16);
          v.w += __shfl_xor_sync(0xffffffffu, v.w, 16);
          if (lane >= 16) continue;
        }
        *reinterpret_cast<float4*>(buf + o_at(g, lane * 4 + c * 128, D)) = v;
      }
  }
};

// ----------------------------------------------------------- first kernel --
// Stages of a warp's ring, and CTAs that share an SM: on the line of tiles, and
// with a cluster per unit.
template <typename Rows>
constexpr int stages() { return 2; }
constexpr int line_ctas(int D, int rows) { return D > 128 ? 1 : rows > 8 || D == 128 ? 2 : 4; }
constexpr int cluster_ctas(int D, int rows) { return D > 128 ? 1 : rows > 8 ? 2 : 3; }
template <typename Rows>
constexpr int smem_bytes() {
  return kWarps * stages<Rows>() * Rows::kStage + Rows::kQBytes + kWarps * Rows::kWarpBytes;
}

template <typename Rows>
__device__ __forceinline__ void one_tile(Rows& r, const CacheAttn& a, const char* st, const char* sq,
                                         char* sw, uint32_t mask, float* lg, int64_t ld, int rows,
                                         int lane) {
  if constexpr (Rows::kBf16)
    r.tile(a, smem_u32(st), sq, sw, mask, lg, ld, rows, lane);
  else
    r.tile(a, 0u, sq, sw, mask, lg, rows, lane, st);
}

template <typename Rows>
__global__ void __launch_bounds__(kThreads, line_ctas(Rows::D, Rows::kR))
cache_attention_kernel(const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
                       const __grid_constant__ CacheAttn a) {
  using T = typename Rows::T;
  constexpr int D = Rows::D, kR = Rows::kR, kTile = Rows::kTile, NS = stages<Rows>();
  extern __shared__ __align__(1024) char smem[];
  __shared__ float2 s_ml[2][kWarps][Rows::kBufRows];
  __shared__ int s_free[2][kWarps];
  __shared__ uint64_t s_full[kWarps][NS];
  __shared__ uint32_t s_mask[kWarps][NS];
  const int tid = threadIdx.x, w = tid >> 5, lane = tid & 31;
  if (lane < NS) mbar_init(&s_full[w][lane], a.box ? 1 : 32);   // a warp's barriers are its own
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  before_copies();
  __syncwarp();
  if (tid == 0 && a.box) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&mk));
    asm volatile("prefetch.tensormap [%0];" ::"l"(&mv));
  }
  pdl_wait_then_trigger();

  // sequences without cached tokens
  for (int b = blockIdx.x; b < a.c.B; b += gridDim.x) {
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
  const int B = a.c.B, units = a.c.Hkv * a.groups;
  const int each = (B + 31) / 32, b0 = min(B, lane * each), b1 = min(B, b0 + each);
  int sum = 0;
  for (int b = b0; b < b1; ++b) {
    sum += tiles_of(a, cache_len(a.c, b)) * units;
    if (blockIdx.x == 0 && w == 0) check_cache_len(a.c, b, a.status);
  }
  int inc = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += y;
  }
  const int total = __shfl_sync(0xffffffffu, inc, 31);
  const int per = max(kMinTiles, (total + a.grid - 1) / a.grid);
  const int first = blockIdx.x * per;
  if (first >= total) {
    if (tid == 0) a.own[blockIdx.x] = make_int4(-1, 0, 0, 0);
    return;
  }
  int sb = b0, soff = first - (inc - sum);
  const bool here_lane = soff >= 0 && soff < sum;
  if (here_lane)
    for (;; ++sb) {
      const int n = tiles_of(a, cache_len(a.c, sb)) * units;
      if (soff < n) break;
      soff -= n;
    }
  const int src = __ffs(__ballot_sync(0xffffffffu, here_lane)) - 1;
  sb = __shfl_sync(0xffffffffu, sb, src);
  soff = __shfl_sync(0xffffffffu, soff, src);
  char* ring = smem + w * NS * Rows::kStage;
  char* s_q = smem + kWarps * NS * Rows::kStage;
  char* s_w = s_q + Rows::kQBytes + w * Rows::kWarpBytes;

  int left = min(per, total - first), b = sb;
  int len = cache_len(a.c, b), nt = tiles_of(a, len);
  int u = soff / nt, t0 = soff - u * nt;
  Cursor cur{b, u, t0 + w, nt, len, (left - w + kWarps - 1) / kWarps, -1};
  if (cur.left > 0) {
    cur.settle(a, units);
    cur.look_up<kTile>(a, lane);
  }
  auto h_of = [&](int uu) {      // first query head of a unit, its rows
    const int hk = a.groups == 1 ? uu : uu / a.groups, row0 = (uu - hk * a.groups) * kR;
    return make_int2(hk * a.G + row0, min(kR, a.G - row0));
  };
  // stage `fill` is the free one: the tile after the last issued goes there
  int fill = 0, use = 0;
  uint32_t phase = 0;
  int late = 0;         // a copy did not come in time: the others get little more
  auto issue = [&]() {
    if (cur.left > 0)
      copy_tile<Rows>(mk, mv, a, cur, ring + fill * Rows::kStage, &s_full[w][fill], &s_mask[w][fill],
                      units, lane);
    fill = fill + 1 == NS ? 0 : fill + 1;
  };
  constexpr int kQEach = (Rows::kQPieces + kThreads - 1) / kThreads;
  uint4 nq[kQEach];
  {
    const int2 h = h_of(u);
#pragma unroll
    for (int k = 0; k < kQEach; ++k)
      if (tid + k * kThreads < Rows::kQPieces)
        nq[k] = Rows::load_q(a, b, h.x, h.y, tid + k * kThreads);
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
    const int2 h = h_of(u);
    // the next unit, and its Q on the way
    int nb = b, nu = u + 1, nlen = len, nnt = nt;
    const int after = left - (t1 - t0);
    if (after > 0) {
      if (nu == units) {
        nu = 0;
        do {
          nlen = cache_len(a.c, ++nb);
          nnt = tiles_of(a, nlen);
        } while (nnt == 0);
      }
      const int2 nh = h_of(nu);
#pragma unroll
      for (int k = 0; k < kQEach; ++k)
        if (tid + k * kThreads < Rows::kQPieces)
          nq[k] = Rows::load_q(a, nb, nh.x, nh.y, tid + k * kThreads);
    }
    rows.reset();
    const int lrow = Rows::kBf16 ? lane >> 2 : lane & 7;
    float* lg = a.score ? a.logits + ((int64_t)b * a.H + h.x + lrow) * a.ld : nullptr;
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
               a.score ? lg + t * kTile : nullptr, a.ld, h.y, lane);
      if (++use == NS) {
        use = 0;
        phase ^= 1u;
      }
    }
    // the warps meet: each leaves its rows in the free stage of its ring
    const bool whole = t0 == 0 && t1 == nt;
    const int slot = 2 * blockIdx.x + (seg == 0 ? 0 : 1);
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
        if (row >= h.y || d >= a.c.d) continue;
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
        const int hh = h.x + row;
        if (whole) {
          const float inv = l > 0.f ? 1.f / l : (l != l ? l : 0.f);
          T* out = static_cast<T*>(a.o) + (int64_t)b * a.o_sb + (int64_t)hh * a.o_sh + d;
          store_elem(out, 0, v.x * inv);
          store_elem(out, 1, v.y * inv);
          store_elem(out, 2, v.z * inv);
          store_elem(out, 3, v.w * inv);
          if (d == 0) {
            const float e = l > 0.f ? top + log2f(l) : (l != l ? l : -INFINITY);
            if (a.score) a.lse2[(int64_t)b * a.H + hh] = e;
            if (a.lse) a.lse[(int64_t)b * a.H + hh] = e * kLn2;
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
      if (pieces > 1) own = make_int4(b * units + u, slot, pieces, 0);
      if (tid == 0 && (a.score || !a.few)) a.rec[b * units + u] = make_int2(slot, pieces);
    }
    ++seg;
    f0 += t1 - t0;
    left = after;
    b = nb; u = nu; len = nlen; nt = nnt; t0 = 0;
  }
  if (tid == 0) a.own[blockIdx.x] = own;
}

// ---------------------------------------------------------- one launch --
// Shorter sequences: a cluster of CTAs per unit, each with an equal run of its
// tiles and their logits in shared memory.  The CTAs' maxima, sums and O meet
// through distributed shared memory; then every CTA writes a slice of O and the
// weights of its own keys.  No workspace, no second kernel.
template <typename Rows>
constexpr int cluster_smem(int rows, int keys) {   // keys: logits' row stride, 0: none
  return smem_bytes<Rows>() + Rows::kR * Rows::D * 4 + rows * keys * 4;
}
// The row stride of `keys` logits: 8 more than a multiple of 32, which spreads
// the rows over the banks.
inline int logit_stride(int keys) { return (keys + 23) / 32 * 32 + 8; }

template <typename Rows>
__global__ void __launch_bounds__(kThreads, cluster_ctas(Rows::D, Rows::kR))
cache_cluster_kernel(const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
                     const __grid_constant__ CacheAttn a, int stride) {
  using T = typename Rows::T;
  constexpr int D = Rows::D, kR = Rows::kR, kTile = Rows::kTile, NS = stages<Rows>();
  constexpr int kMaxCluster = 8;
  extern __shared__ __align__(1024) char smem[];
  __shared__ float2 s_ml[kWarps][Rows::kBufRows];
  __shared__ float2 s_mine[kR];                  // this CTA's maximum and sum of a row
  __shared__ float s_f[kMaxCluster][kR], s_e[kR];
  __shared__ int s_free[kWarps];
  __shared__ uint64_t s_full[kWarps][NS];
  __shared__ uint32_t s_mask[kWarps][NS];
  cg::cluster_group cluster = cg::this_cluster();
  const int ncta = (int)cluster.num_blocks(), me = (int)cluster.block_rank();
  const int tid = threadIdx.x, w = tid >> 5, lane = tid & 31;
  const int unit = blockIdx.x / ncta, units = a.c.Hkv * a.groups;
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
  pdl_wait_then_trigger();
  if (u == 0 && me == 0 && tid == 0) check_cache_len(a.c, b, a.status);
  const int len = cache_len(a.c, b);
  if (len == 0) {      // the whole cluster
    if (me == 0)
      for (int i = tid; i < rows_here * a.c.d; i += kThreads) {
        const int r = i / a.c.d;
        store_elem(static_cast<T*>(a.o), (int64_t)b * a.o_sb + (int64_t)(h0 + r) * a.o_sh +
                   (i - r * a.c.d), 0.f);
        if (a.lse && i == r * a.c.d) a.lse[(int64_t)b * a.H + h0 + r] = -INFINITY;
      }
    return;
  }
  const int nt = tiles_of(a, len), run = (nt + ncta - 1) / ncta;
  const int t0 = min(nt, me * run), mine = min(nt, t0 + run) - t0;
  char* ring = smem + w * NS * Rows::kStage;
  char* s_q = smem + kWarps * NS * Rows::kStage;
  char* s_w = s_q + Rows::kQBytes + w * Rows::kWarpBytes;
  float* s_o = reinterpret_cast<float*>(smem + smem_bytes<Rows>());
  float* s_lg = s_o + kR * D;
  Cursor cur{b, u, t0 + w, nt, len, (mine - w + kWarps - 1) / kWarps, -1};
  if (cur.left > 0) cur.look_up<kTile>(a, lane);
  constexpr int kQEach = (Rows::kQPieces + kThreads - 1) / kThreads;
  uint4 q[kQEach];
#pragma unroll
  for (int k = 0; k < kQEach; ++k)
    if (tid + k * kThreads < Rows::kQPieces)
      q[k] = Rows::load_q(a, b, h0, rows_here, tid + k * kThreads);
  int fill = 0, use = 0;
  uint32_t phase = 0;
  int late = 0;         // a copy did not come in time: the others get little more
  auto issue = [&]() {
    if (cur.left > 0)
      copy_tile<Rows>(mk, mv, a, cur, ring + fill * Rows::kStage, &s_full[w][fill], &s_mask[w][fill],
                      units, lane);
    fill = fill + 1 == NS ? 0 : fill + 1;
  };
#pragma unroll 1
  for (int i = 0; i < NS - 1; ++i) issue();
#pragma unroll
  for (int k = 0; k < kQEach; ++k)
    if (tid + k * kThreads < Rows::kQPieces) Rows::store_q(s_q, tid + k * kThreads, q[k]);
  __syncthreads();
  Rows rows;
  rows.reset();
  const int lrow = Rows::kBf16 ? lane >> 2 : lane & 7;
#pragma unroll 1
  for (int t = w; t < mine; t += kWarps) {
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
    for (int i = tid; i < Rows::kBufRows * (D / 4); i += kThreads) {
      const int r = i / (D / 4), d = (i - r * (D / 4)) * 4, row = part * 16 + r;
      if (row >= rows_here || d >= a.c.d) continue;
      float top = -INFINITY, l = 0.f;
#pragma unroll
      for (int k = 0; k < kWarps; ++k) top = fmaxf(top, s_ml[k][r].x);
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < kWarps; ++k) {
        const float2 ml = s_ml[k][r];
        const float4 x = *reinterpret_cast<const float4*>(smem + s_free[k] + o_at(r, d, D) * 4);
        const float f = ml.x == -INFINITY ? 0.f : ex2(ml.x - top);
        v.x = fmaf(f, x.x, v.x); v.y = fmaf(f, x.y, v.y);
        v.z = fmaf(f, x.z, v.z); v.w = fmaf(f, x.w, v.w);
        l = fmaf(f, ml.y, l);
      }
      *reinterpret_cast<float4*>(s_o + row * D + d) = v;
      if (d == 0) s_mine[row] = make_float2(top, l);
    }
    __syncthreads();
  }
  cluster.sync();
  // over the CTAs: a row's lse, and what each CTA's O counts in it
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
    const float inv = l > 0.f ? 1.f / l : (l != l ? l : 0.f);
#pragma unroll
    for (int k = 0; k < kMaxCluster; ++k) s_f[k][tid] = ex2(x[k].x - ref) * inv;
    const float e = l > 0.f ? top + log2f(l) : (l != l ? l : -INFINITY);
    s_e[tid] = e == -INFINITY ? INFINITY : e;     // nothing to attend to: no weight
    if (me == 0 && a.lse) a.lse[(int64_t)b * a.H + h0 + tid] = e * kLn2;
  }
  __syncthreads();
  const int d4 = a.c.d / 4;
  for (int i = me * kThreads + tid; i < rows_here * d4; i += ncta * kThreads) {
    const int r = i / d4, d = (i - r * d4) * 4;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int k = 0; k < ncta; ++k) {
      const float4 x = *reinterpret_cast<const float4*>(cluster.map_shared_rank(s_o, k) + r * D + d);
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
  if (a.score) {
    const int j0 = t0 * kTile, n = min(len - j0, mine * kTile);
    float* acc = a.c.acc + (int64_t)b * a.c.acc_sb + (int64_t)hk * a.c.acc_sh + j0;
    for (int j = tid; j < n; j += kThreads) {
      const float old = a.add ? acc[j] : 0.f;
      float s = 0.f;
#pragma unroll 8
      for (int r = 0; r < rows_here; ++r) s += ex2(s_lg[r * stride + j] - s_e[r]);
      acc[j] = fmaf(s, a.wmean, old);
    }
  }
  cluster.sync();      // no CTA leaves while another reads its O
}

// ---------------------------------------------------------- second kernel --
// Block (unit, row), or, where there are many units, (CTA of the first kernel,
// rows): O of that unit, or of the one whose first of several pieces was that
// CTA's.  Block (b, hk, 512 keys or more): their weights.  What a block reads waits
// for as little as can be: parts and logits are on their way while the row's lse
// is put together.
constexpr int kFinishThreads = 128;
constexpr int kWeightKeys = 4 * kFinishThreads;
constexpr int kMaxGroup = 256;
constexpr int kFewPieces = 8;

// Part of piece k of a unit: the first one's is given, the following CTAs' are
// their first.
__device__ __forceinline__ int part_of(int slot, int k) { return k == 0 ? slot : ((slot >> 1) + k) * 2; }

// log2-domain lse of row r over a unit's pieces, in a whole warp.
__device__ __forceinline__ float join_lse(const CacheAttn& a, int slot, int pieces, int r,
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
  return l > 0.f ? top + log2f(l) : (l != l ? l : -INFINITY);
}

// The same in one thread, for few pieces.
__device__ __forceinline__ float join_lse_serial(const CacheAttn& a, int slot, int pieces, int r) {
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
  return l > 0.f ? top + log2f(l) : (l != l ? l : -INFINITY);
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
  const float e = kWide ? (row < a.G ? join_lse(a, own.y, own.z, r, tid & 31) : 0.f)
                        : join_lse_serial(a, own.y, pieces, r);
  if (mine && k1 == 0 && col == 0 && a.lse) a.lse[(int64_t)b * a.H + h] = e * kLn2;
  const float none = e != e ? e : 0.f;
  float4 v = make_float4(none, none, none, none);
  if (e != -INFINITY) {
    for (int k0 = k1; k0 < pieces; k0 += kDeep * step) {
      if (k0 != k1) load(k0);
#pragma unroll
      for (int i = 0; i < kDeep; ++i)
        if (k0 + i * step < pieces) {
          const float f = ex2(mx[i] - e);     // from -inf: 0
          v.x = fmaf(f, x[i].x, v.x); v.y = fmaf(f, x[i].y, v.y);
          v.z = fmaf(f, x[i].z, v.z); v.w = fmaf(f, x[i].w, v.w);
        }
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
  store_elem(out, 0, v.x);
  store_elem(out, 1, v.y);
  store_elem(out, 2, v.z);
  store_elem(out, 3, v.w);
}

// `parts` parts of kSpan runs of 512 keys, kRows rows at a time.  First the length
// and where the rows' pieces are; then everything else of the first part at once:
// logits, old weights, pieces.
template <int kSpan, int kRows>
__device__ __forceinline__ void weights_block(const CacheAttn& a, int bh, int part, int parts) {
  __shared__ float s_e[kMaxGroup];
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
    const float e = rec.y == 1 ? a.lse2[(int64_t)b * a.H + hk * a.G + r]
                    : a.few    ? join_lse_serial(a, rec.x, rec.y, row)
                               : join_lse(a, rec.x, rec.y, row, tid & 31);
    if (a.few || (tid & 31) == 0) s_e[r] = e == -INFINITY ? INFINITY : e;   // no weight there
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
          const float e = s_e[r0 + r];
#pragma unroll
          for (int g = 0; g < kSpan; ++g) {
            s[g][0] += ex2(x[g][r].x - e);
            s[g][1] += ex2(x[g][r].y - e);
            s[g][2] += ex2(x[g][r].z - e);
            s[g][3] += ex2(x[g][r].w - e);
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

// Runs of 512 keys that a block of weights takes: small groups have few logits.
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

// How a call is cut: the widths 64, 128 and 256 have kernels of their own; a
// unit has 8 rows (fp32), or 8, 16 or 32 by the group's size (bf16), so that a
// tile in shared memory serves all the heads that share it (256 columns: 16 at
// most, by registers).
struct Shape {
  int G, D, rows, groups, tile, grid;
  int cluster;      // CTAs of a unit's cluster; 0: the line of tiles
  long long tiles;
};

constexpr int kMaxDynamic = 220 * 1024;
constexpr int kClusterKeys = 512;       // of a CTA
constexpr int kClusterLogits = 8192;    // rows times keys of a CTA

int cluster_of(const avits_kv_cache& c, const Shape& s, bool score, int num_sms) {
  if (score && s.groups > 1) return 0;      // a unit has not all the heads of a weight
  const int rows = s.G < s.rows ? s.G : s.rows;
  const long long units = (long long)c.B * c.Hkv * s.groups;
  auto fits = [&](int n) {
    const int64_t keys = ((int64_t)c.max_len + n - 1) / n;
    return keys <= (score || n > 1 ? kClusterKeys : 2 * kClusterKeys) && (!score || keys * rows <= kClusterLogits);
  };
  int n = 1;
  while (n < 8 && !fits(n)) n *= 2;
  if (!fits(n) || units * n >= (1 << 30)) return 0;
  const long long resident = (long long)num_sms * (s.D > 128 ? 1 : 2);
  if (n > 1 && units * n > resident) return 0;
  while (n < 8 && units * n * 2 <= resident && c.max_len > n * 64) n *= 2;
  if (units * n < num_sms && c.max_len > n * 256) return 0;
  return n;
}

Shape shape_of(const avits_kv_cache& c, int H, bool score, int num_sms) {
  Shape s;
  const bool bf = c.dt == AVITS_BF16;
  s.G = H / c.Hkv;
  s.D = c.d <= 64 ? 64 : c.d <= 128 ? 128 : 256;
  s.rows = !bf || s.G <= 8 ? 8 : s.G <= 16 || s.D == 256 ? 16 : 32;
  s.groups = (s.G + s.rows - 1) / s.rows;
  s.tile = bf ? 16 : 8;
  s.tiles = (long long)c.B * c.Hkv * s.groups * ((c.max_len + s.tile - 1) / s.tile);
  const long long most = (s.tiles + kMinTiles - 1) / kMinTiles;
  long long full = (long long)num_sms * line_ctas(s.D, s.rows);
  if (full > kMaxGrid) full = kMaxGrid;
  s.grid = (int)(most < full ? (most > 0 ? most : 1) : full);
  s.cluster = cluster_of(c, s, score, num_sms);
  return s;
}

size_t up16(size_t n) { return (n + 15) / 16 * 16; }

struct Layout {
  size_t rec, own, lse2, pml, po, logits, total;
  int64_t ld;
};

Layout layout_of(const avits_kv_cache& c, int H, const Shape& s, bool score) {
  Layout l;
  const size_t nrow = s.rows;
  l.ld = ((int64_t)c.max_len + 15) / 16 * 16;
  l.rec = 0;
  l.own = up16((size_t)c.B * c.Hkv * s.groups * 8);
  l.lse2 = l.own + up16((size_t)s.grid * 16);
  l.pml = l.lse2 + up16((size_t)c.B * H * 4);
  l.po = l.pml + up16((size_t)2 * s.grid * nrow * 8);
  l.logits = l.po + up16((size_t)2 * s.grid * nrow * c.d * 4);
  l.total = l.logits + (score ? (size_t)c.B * H * l.ld * 4 : 0);
  return l;
}

// Tensor map of the pages: boxes of `box` tokens of one head and page, in columns
// of 128 bytes with the 128-byte swizzle (bf16) or whole rows (fp32).
template <typename Rows>
bool map_pages(CUtensorMap* map, const void* pages, int64_t sp, int64_t st, int64_t sh,
               const avits_kv_cache& c, int box) {
  const tc::EncodeTiledFn fn = tc::encode_fn();
  if (!fn) return false;
  constexpr int64_t es = sizeof(typename Rows::T);
  // a dimension of extent 1 has a stride that is never used
  const int64_t row = c.d * es;
  const cuuint64_t dims[4] = {(cuuint64_t)c.d, (cuuint64_t)c.Hkv, (cuuint64_t)c.page_size,
                              (cuuint64_t)c.num_pages};
  const int64_t str[3] = {c.Hkv > 1 ? sh * es : row, c.page_size > 1 ? st * es : row,
                          c.num_pages > 1 ? sp * es : row};
  cuuint64_t strides[3];
  for (int i = 0; i < 3; ++i) {
    if (str[i] <= 0 || str[i] >= (1ll << 40)) return false;
    strides[i] = (cuuint64_t)str[i];
  }
  const cuuint32_t width = Rows::kBf16 ? 64 : Rows::D;
  const cuuint32_t shape[4] = {width, 1, (cuuint32_t)box, 1}, step[4] = {1, 1, 1, 1};
  return fn(map, Rows::kBf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32,
            4, const_cast<void*>(pages), dims, strides, shape, step,
            CU_TENSOR_MAP_INTERLEAVE_NONE,
            Rows::kBf16 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE,
            row >= 256 ? CU_TENSOR_MAP_L2_PROMOTION_L2_256B : CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The maps, and a.box: 0 where the pages' layout has none.
template <typename Rows>
void map_cache(CacheAttn& a, CUtensorMap* mk, CUtensorMap* mv) {
  const avits_kv_cache& c = a.c;
  const int box = c.page_size % Rows::kTile == 0 ? Rows::kTile : c.page_size % 8 == 0 ? 8 : 0;
  a.box = box && map_pages<Rows>(mk, c.k_pages, c.k_sp, c.k_st, c.k_sh, c, box) &&
                  map_pages<Rows>(mv, c.v_pages, c.v_sp, c.v_st, c.v_sh, c, box)
              ? box
              : 0;
}

template <typename Rows>
cudaError_t launch_cluster(const CUtensorMap& mk, const CUtensorMap& mv, const CacheAttn& a,
                           int ncta, cudaStream_t s) {
  constexpr auto kernel = cache_cluster_kernel<Rows>;
  const cudaError_t e = prefer_max_shared<kernel, kMaxDynamic>();
  if (e != cudaSuccess) return e;
  const int tiles = (a.c.max_len + a.tile - 1) / a.tile;
  const int stride = a.score ? logit_stride((tiles + ncta - 1) / ncta * a.tile) : 0;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(a.c.B * a.c.Hkv * a.groups * ncta));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = (size_t)cluster_smem<Rows>(a.G < a.rows ? a.G : a.rows, stride);
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
  return cudaLaunchKernelEx(&cfg, kernel, mk, mv, a, stride);
}

template <typename Rows>
cudaError_t launch_rows(CacheAttn& a, int ncta, int num_sms, cudaStream_t s) {
  CUtensorMap mk{}, mv{};
  map_cache<Rows>(a, &mk, &mv);
  if (ncta > 0) return launch_cluster<Rows>(mk, mv, a, ncta, s);
  constexpr auto kernel = cache_attention_kernel<Rows>;
  cudaError_t e = prefer_max_shared<kernel, smem_bytes<Rows>()>();
  if (e != cudaSuccess) return e;
  e = launch_pdl(kernel, dim3(a.grid), dim3(kThreads), smem_bytes<Rows>(), s, mk, mv, a);
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

template <template <int, int> class Rows, int kR>
cudaError_t launch_width(CacheAttn& a, int D, int ncta, int num_sms, cudaStream_t s) {
  if (D == 64) return launch_rows<Rows<64, kR>>(a, ncta, num_sms, s);
  if (D == 128) return launch_rows<Rows<128, kR>>(a, ncta, num_sms, s);
  if constexpr (kR <= 16) return launch_rows<Rows<256, kR>>(a, ncta, num_sms, s);
  return cudaErrorInvalidValue;
}

}  // namespace

bool cache_attention_sizes_ok(const avits_kv_cache& c, int H) {
  if (H / c.Hkv > kMaxGroup) return false;
  const Shape s = shape_of(c, H, false, 1);
  return s.tiles < (1ll << 30) && (long long)c.B * H < (1ll << 30);
}

size_t cache_attention_workspace(const avits_kv_cache& c, int H, bool score, int num_sms) {
  const Shape s = shape_of(c, H, score, num_sms);
  return s.cluster > 0 ? 0 : layout_of(c, H, s, score).total;
}

cudaError_t launch_cache_attention(const CacheAttnCall& call, int num_sms, unsigned int* status,
                                   cudaStream_t s) {
  const avits_kv_cache& c = call.cache;
  const bool score = call.weights != AVITS_WEIGHTS_NONE;
  const Shape sh = shape_of(c, call.H, score, num_sms);
  const Layout l = layout_of(c, call.H, sh, score);
  char* ws = static_cast<char*>(call.ws);
  CacheAttn a{};
  a.c = c;
  a.page = FastDiv::of(c.page_size);
  a.q = call.q;
  a.o = call.o;
  a.q_sb = call.q_sb; a.q_sh = call.q_sh; a.o_sb = call.o_sb; a.o_sh = call.o_sh;
  a.lse = call.lse;
  a.H = call.H;
  a.G = sh.G;
  a.rows = sh.rows;
  a.groups = sh.groups;
  a.tile = sh.tile;
  a.grid = sh.grid;
  a.score = score;
  a.few = (long long)c.B * c.Hkv * sh.groups * kFewPieces > sh.grid;
  a.scale2 = call.scale * kLog2e;
  a.wmean = call.weight / (float)sh.G;
  a.add = call.weights == AVITS_WEIGHTS_ADD;
  a.rec = reinterpret_cast<int2*>(ws + l.rec);
  a.own = reinterpret_cast<int4*>(ws + l.own);
  a.lse2 = reinterpret_cast<float*>(ws + l.lse2);
  a.pml = reinterpret_cast<float2*>(ws + l.pml);
  a.po = reinterpret_cast<float*>(ws + l.po);
  a.logits = reinterpret_cast<float*>(ws + l.logits);
  a.ld = l.ld;
  a.status = status;
  if (c.dt != AVITS_BF16) return launch_width<RowsF32, 8>(a, sh.D, sh.cluster, num_sms, s);
  if (sh.rows == 8) return launch_width<RowsBf16, 8>(a, sh.D, sh.cluster, num_sms, s);
  if (sh.rows == 16) return launch_width<RowsBf16, 16>(a, sh.D, sh.cluster, num_sms, s);
  return launch_width<RowsBf16, 32>(a, sh.D, sh.cluster, num_sms, s);
}

}  // namespace avits
