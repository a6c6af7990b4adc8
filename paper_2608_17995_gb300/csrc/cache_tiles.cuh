// cache_tiles.cuh — what the two forms of the cache attention share: a tile of
// keys and values in shared memory, the copies that bring it, and the arithmetic
// of a row tile of heads with it (bf16: tensor cores, fp32: CUDA cores).
#pragma once

#include "cache_common.cuh"
#include "avits_internal.h"
#include "tc_common.cuh"

namespace avits {
namespace cache {

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kMaxGrid = 1024;
constexpr int kMaxGroup = 256;        // query heads of a KV head
// Units of that many pieces or fewer are joined by a thread per four columns, which
// goes through the pieces, longer ones by threads that lie over the pieces.  Serial
// and spread: 48 x <= 4096 85 and 102 us, 40 x 24 heads x <= 1500 50.5 and 67, one of
// 131072 61.9 and 55.2 (4 KV heads), 8 heads of 30000 54.1 and 45.5.  32 x <= 6000 with
// 2 KV heads has 4.6 pieces to a unit: 47 and 63, so that 4 is too low a border.
constexpr int kFewPieces = 8;
constexpr int kMaxDynamic = 220 * 1024;
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
  int least;        // tiles of the smallest piece
  int box;          // tokens of a TMA box; 0: rows come by 16-byte copies
  int score;        // weights wanted: logits are kept
  int few;          // units have kFewPieces pieces or fewer each, by and large
  float scale2;     // scale * log2(e)
  float wmean;      // weight / G
  int add;
  // workspace
  int2* rec;        // [B units] first part of a unit and its pieces; one: it is in norm
  int4* own;        // [grid] unit whose first piece is the CTA's, of several: (unit or -1,
                    // first part, pieces); read where units have few pieces
  float2* norm;     // [B,H] of rows finished in one piece (see norm_of)
  float2* pml;      // [2 grid][rows] maximum and sum of a piece's row
  float* po;        // [2 grid][rows][d] its O
  float* logits;    // [B,H,ld] log2-domain logits (weights wanted)
  int64_t ld;
  unsigned int* status;
  // attention over prefixes that groups of sequences share: the prefixes' cache is c, and
  const int32_t* start;   // [c.B + 1] first sequence of each group
  int seqs;               // sequences of the batch
  int* base;              // [c.B + 1] first unit of each group; the last: 1 if the groups rise
};

// Sequences [x, y) of group g.
__device__ __forceinline__ int2 members_of(const int32_t* start, int seqs, int g) {
  const int x = min(max(start[g], 0), seqs), y = min(max(start[g + 1], 0), seqs);
  return make_int2(x, max(x, y));
}

// A sequence's units.  Its own tokens: each KV head's row groups, the same number in every
// sequence.
struct OwnUnits {
  int n, groups;
  __device__ __forceinline__ int of(const CacheAttn&, int) const { return n; }
  __device__ __forceinline__ int head(const CacheAttn&, int, int u) const {
    return groups == 1 ? u : u / groups;
  }
};
// A prefix: each KV head's row groups over the query heads of all members.
struct GroupUnits {
  __device__ __forceinline__ static int row_groups(const CacheAttn& a, int g) {
    const int2 m = members_of(a.start, a.seqs, g);
    return ((m.y - m.x) * a.G + a.rows - 1) / a.rows;
  }
  __device__ __forceinline__ int of(const CacheAttn& a, int g) const {
    return a.c.Hkv * row_groups(a, g);
  }
  __device__ __forceinline__ int head(const CacheAttn& a, int g, int u) const {
    return u / row_groups(a, g);
  }
};

// A row's maximum and sum -> what a weight is: exp2(x - .x) times .y.  Not exp2(x - lse):
// a step of lse is up to 2^-24 |lse|, an error that all weights of a row would share,
// while a maximum is one of the logits and the differences from it are as exact as they
// are.  A row without keys has weights of zero, a row with a NaN NaN.
__device__ __forceinline__ float2 norm_of(float top, float l) {
  return make_float2(top == -INFINITY ? 0.f : top, l > 0.f ? 1.f / l : (l != l ? l : 0.f));
}
// Its lse in the log2 domain.
__device__ __forceinline__ float lse2_of(float top, float l) {
  return l > 0.f ? top + log2f(l) : (l != l ? l : -INFINITY);
}

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

  template <typename Units>
  __device__ __forceinline__ void settle(const CacheAttn& a, const Units& units) {
    while (t >= nt) {
      t -= nt;
      if (++u == units.of(a, b)) {
        u = 0;
        do {
          len = cache_len(a.c, ++b);
          nt = tiles_of(a, len);
        } while (nt == 0 || units.of(a, b) == 0);
      }
    }
  }
  template <int kTile>
  __device__ __forceinline__ void look_up(const CacheAttn& a, int lane) {
    const int j = t * kTile + (a.box ? lane * a.box & (kTile - 1) : lane & (kTile - 1));
    entry = j < len ? a.c.block_table[(int64_t)b * a.c.table_sb + a.page.div(j)] : -1;
  }
};

// A unit's rows: query heads h0 .. of sequence b, or, G > 0, rows of a group: row r is head
// h0 + (r0 + r) % G of sequence b + (r0 + r) / G.
struct QRows {
  int b, h0, rows, r0, G;
  __device__ __forceinline__ int64_t at(const CacheAttn& a, int row) const {
    if (G == 0) return (int64_t)b * a.q_sb + (int64_t)(h0 + row) * a.q_sh;
    const int x = (r0 + row) / G;
    return (int64_t)(b + x) * a.q_sb + (int64_t)(h0 + r0 + row - x * G) * a.q_sh;
  }
};

// Copies the cursor's tile to `dst`, keys then values, and steps on by kStep.  `mask` gets
// a bit for each key that is there (below the length, its page in range).  A tile
// lies as columns of 128 bytes: in bf16 [D / 64][16 rows][128 bytes] with the
// 16-byte pieces of row r at c ^ (r % 8) (TMA's 128-byte swizzle, for ldmatrix),
// in fp32 plain rows.  By TMA where boxes of 16 or 8 tokens never cross a page:
// what lies outside the tensors (columns past the width, a page out of range)
// comes as zeros.  Else by 16-byte copies, a row's pieces side by side, zeros past
// the width.  So the products run over whole widths of 64, 128 or 256 unchecked.
// 48 x <= 1024 took 32.7 us by TMA and 35.3 by 16-byte copies, 40 x 24 heads of width
// 64 54.2 and 58.4: a copy costs a warp instructions per row, a box one.
template <typename Rows, int kStep, typename Units>
__device__ __forceinline__ void copy_tile(const CUtensorMap& mk, const CUtensorMap& mv,
                                          const CacheAttn& a, Cursor& cur, char* dst, uint64_t* bar,
                                          uint32_t* mask, const Units& units, int lane) {
  constexpr int kTile = Rows::kTile, kEs = sizeof(typename Rows::T), D = Rows::D;
  const int hk = units.head(a, cur.b, cur.u);
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
    cur.t += kStep;
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
// two bf16 parts (value and rest, 16 significant bits and a sign together: off by
// 2^-17 of a weight at most, where a bf16 O is rounded by 2^-8), the value in
// rows 0-7 and the rest in rows 8-15, which are free.  kR = 16, 32: one or two
// row tiles, the rest in a second product.
//
// The rest may be negative or zero, so that its product with an infinite value of V
// is no part of the result: the value's product alone has it, and its NaN.  kR = 8: the
// rest's sum is added where the value's is finite.  kR = 16, 32, whose products share
// their sums: the second one takes V cut to the finite range (two instructions to a
// register of V: 32 sequences of 714-6000 with 24 heads to each of 2 KV heads 34.1 us,
// 33.0 without them; 16 heads of width 256 39.0 and 37.8).
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
// Infinities and NaN of two bf16 as finite numbers (min and max give the other
// operand for a NaN).
__device__ __forceinline__ uint32_t finite_bf16(uint32_t x) {
  uint32_t y;
  asm("{\n\t.reg .b32 t;\n\tmax.bf16x2 t, %1, %2;\n\tmin.bf16x2 %0, t, %3;\n\t}"
      : "=r"(y)
      : "r"(x), "r"(0xFF7FFF7Fu), "r"(0x7F7F7F7Fu));
  return y;
}
// The sum of a row's two parts.
__device__ __forceinline__ float both_parts(float value, float rest) {
  return fabsf(value) < INFINITY ? value + rest : value;
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

  // row of the logits that a lane keeps
  __device__ static __forceinline__ int logit_row(int lane) { return lane >> 2; }
  // 16-byte piece c of a row of a tile
  __device__ static __forceinline__ int piece_at(int row, int c) {
    return (c >> 3) * kColBytes + row * kColPitch + (((c & 7) ^ (row & 7)) << 4);
  }

  // 16 bytes of Q: piece i of the unit's rows
  __device__ static __forceinline__ uint4 load_q(const CacheAttn& a, const QRows& u, int i) {
    const int row = i / (D / 8), d = (i % (D / 8)) * 8;
    uint32_t w[4] = {0u, 0u, 0u, 0u};
    if (row < u.rows && d < a.c.d) {
      const uint16_t* q = static_cast<const uint16_t*>(a.q) + u.at(a, row) + d;
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
        }
        if (!kSplit8) {
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = finite_bf16(v[i]);
#pragma unroll
          for (int mt = 0; mt < kM; ++mt) {
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
              make_float2(both_parts(x[0], x[2]), both_parts(x[1], x[3]));
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
// CUDA cores in fp32, kR = 8 heads, or 4: every head of a row tile is multiplied,
// also those past the group's.  Q K^T: 8 lanes to a key (16-byte pieces of its
// row), 4 keys at a time; a lane's partial dot products of the heads are summed
// over the 8 lanes by halving, which leaves a head with each lane (8) or with two
// lanes (4).  P V: a lane owns columns of O and reads the weights from shared
// memory.
template <int D_, int kR_>
struct RowsF32 {
  using T = float;
  static constexpr int D = D_, kR = kR_;
  static constexpr int kTwin = 8 / kR;       // lanes that hold the same head
  static constexpr int kTile = 8;
  static constexpr bool kBf16 = false;
  static constexpr int kStage = 2 * kTile * D * 4;
  static constexpr int kCols = 1, kColWidth = 0, kColPitch = D * 4, kColBytes = 0;
  static constexpr int kQBytes = kR * D * 4;
  static constexpr int kQPieces = kQBytes / 16;
  static constexpr int kBufRows = kR, kM = 1;
  static constexpr int kWarpBytes = kTile * kR * 4;
  static constexpr int kKeysPerV = D >= 128 ? 1 : 128 / D;   // value rows read side by side
  static constexpr int kV = D >= 128 ? D / 128 : 1;

  float m, l;            // of row lane % 8 / kTwin; l: this lane's keys only until the end
  float o[kR][kV][4];

  __device__ static __forceinline__ int logit_row(int lane) { return (lane & 7) / kTwin; }
  __device__ static __forceinline__ int piece_at(int row, int c) {
    return row * kColPitch + c * 16;
  }

  __device__ static __forceinline__ uint4 load_q(const CacheAttn& a, const QRows& u, int i) {
    const int row = i / (D / 4), d = (i % (D / 4)) * 4;
    if (row >= u.rows || d >= a.c.d) return make_uint4(0u, 0u, 0u, 0u);
    const uint32_t* q = static_cast<const uint32_t*>(a.q) + u.at(a, row) + d;
    return make_uint4(q[0], q[1], q[2], q[3]);
  }
  __device__ static __forceinline__ void store_q(char* sq, int i, const uint4& v) {
    reinterpret_cast<uint4*>(sq)[i] = v;
  }

  __device__ __forceinline__ void reset() {
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int g = 0; g < kR; ++g)
#pragma unroll
      for (int c = 0; c < kV; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[g][c][e] = 0.f;
  }

  __device__ __forceinline__ void tile(const CacheAttn& a, uint32_t, const char* sq, char* sw,
                                       uint32_t mask, float* lg, int rows, int lane,
                                       const char* st) {
    const int kg = lane >> 3, t8 = lane & 7, row = t8 / kTwin;
    const float* q = reinterpret_cast<const float*>(sq);
    const float* kt = reinterpret_cast<const float*>(st);
    const float* vt = kt + kTile * D;
    float* sp = reinterpret_cast<float*>(sw);
    // a lane's keys: 2 kg, 2 kg + 1
    float s[2][kR] = {};
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      if (c * 32 >= a.c.d) break;
      const int d = c * 32 + t8 * 4;
      const float4 k0 = *reinterpret_cast<const float4*>(kt + (2 * kg) * D + d);
      const float4 k1 = *reinterpret_cast<const float4*>(kt + (2 * kg + 1) * D + d);
#pragma unroll
      for (int g = 0; g < kR; ++g) {
        const float4 qv = *reinterpret_cast<const float4*>(q + g * D + d);
        s[0][g] = fmaf(qv.x, k0.x, fmaf(qv.y, k0.y, fmaf(qv.z, k0.z, fmaf(qv.w, k0.w, s[0][g]))));
        s[1][g] = fmaf(qv.x, k1.x, fmaf(qv.y, k1.y, fmaf(qv.z, k1.z, fmaf(qv.w, k1.w, s[1][g]))));
      }
    }
    float x[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      // half of the heads go to the lane whose bit is the other
      auto halve = [&](float (&v)[kR], int n, int bit) {
#pragma unroll
        for (int j = 0; j < kR / 2; ++j)
          if (j < n) {
            const float mine = (t8 & bit) ? v[j + n] : v[j], give = (t8 & bit) ? v[j] : v[j + n];
            v[j] = mine + __shfl_xor_sync(0xffffffffu, give, bit);
          }
      };
      halve(s[i], kR / 2, 4);
      halve(s[i], kR / 4, 2);
      if (kR == 8)
        halve(s[i], 1, 1);
      else
        s[i][0] += __shfl_xor_sync(0xffffffffu, s[i][0], 1);
      const float dot = s[i][0];
      x[i] = (mask >> (2 * kg + i)) & 1u ? dot * a.scale2 : -INFINITY;
    }
    if (a.score && row < rows && t8 % kTwin == 0)
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
      for (int g = 0; g < kR; ++g) {
        const float fg = __shfl_sync(0xffffffffu, f, g * kTwin);
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
      if (t8 % kTwin == 0) sp[(2 * kg + i) * kR + row] = p;
    }
    __syncwarp();
    const int sub = kKeysPerV == 1 ? 0 : lane / (32 / kKeysPerV);
    const int col = kKeysPerV == 1 ? lane * 4 : (lane % (32 / kKeysPerV)) * 4;
#pragma unroll
    for (int j = 0; j < kTile / kKeysPerV; ++j) {
      const int key = j * kKeysPerV + sub;
      float p[kR];
#pragma unroll
      for (int g = 0; g < kR; g += 4) {
        const float4 pa = *reinterpret_cast<const float4*>(sp + key * kR + g);
        p[g] = pa.x; p[g + 1] = pa.y; p[g + 2] = pa.z; p[g + 3] = pa.w;
      }
#pragma unroll
      for (int c = 0; c < kV; ++c) {
        const float4 v = *reinterpret_cast<const float4*>(vt + key * D + col + c * 128);
#pragma unroll
        for (int g = 0; g < kR; ++g) {
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
    if (lane < 8 && lane % kTwin == 0) ml[lane / kTwin] = make_float2(m, x);
#pragma unroll
    for (int g = 0; g < kR; ++g)
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

// ------------------------------------------------------------- geometry --
// Stages of a warp's ring, and CTAs that share an SM: on the line of tiles, and
// with a cluster per unit.  More CTAs hide more of each other's starts, ends and
// arithmetic, fewer cut the line into fewer pieces to join; more stages than two
// were no faster wherever the shared memory had room for them.  On the line:
//   bf16, width 128: 2 CTAs 131072 keys 55.8 us, with 3 58.1; 48 x <= 4096 without
//     weights 78.1 and 79.0, but 48 x <= 1024 with weights 34.3 and 31.4; 3 stages
//     of 2 CTAs 59.1 for 131072 keys, where 2 stages took 57.0
//   width 64: 4 CTAs, chosen when the kernels held fewer registers (50.3 us and 50.8 with
//     3 for 40 x 24 heads x <= 1500).  As the kernels are, 3 would serve bf16 better
//     (53.8 and 54.7; 48 x <= 4096 53.8 and 55.1; 131072 keys 35.3 and 36.5; 8 x <= 6000
//     18.6 and 20.1) and fp32 as well (24 x <= 3000 35.3 and 35.0)
//   fp32, width 128, whose arithmetic is on the CUDA cores: 3 CTAs 14 x <= 2286 34.2,
//     28 x <= 9904 of 16 heads to a group 166, with 2 40.9 and 192; but 30000 keys of
//     one head to a group 46.3 and 45.3
template <typename Rows>
constexpr int stages() { return 2; }
constexpr int line_ctas(int D, int rows, bool bf16) {
  return D > 128 ? 1 : bf16 && rows > 8 ? 2 : D <= 64 ? 4 : bf16 ? 2 : 3;
}
// Own tokens beside shared prefixes on the line, 8 rows of width 128: 3 CTAs (16 sequences of
// 4096 beside 8000 52.3 us, with 2 55.2; one of 60000 beside 20000 73.6 and 71.9).
constexpr int own_ctas(int D, int rows, bool bf16) {
  return bf16 && rows == 8 && D == 128 ? 3 : line_ctas(D, rows, bf16);
}
// A cluster's CTAs hold to what their registers allow without spills.
constexpr int cluster_ctas(int D, int rows, int warps) {
  return (D > 128 ? 4 : rows > 8 ? 8 : 12) / warps;
}
template <typename Rows>
constexpr int smem_bytes(int warps) {
  return warps * stages<Rows>() * Rows::kStage + Rows::kQBytes + warps * Rows::kWarpBytes;
}

template <typename Rows>
__device__ __forceinline__ void one_tile(Rows& r, const CacheAttn& a, const char* st,
                                         const char* sq, char* sw, uint32_t mask, float* lg,
                                         int64_t ld, int rows, int lane) {
  if constexpr (Rows::kBf16)
    r.tile(a, smem_u32(st), sq, sw, mask, lg, ld, rows, lane);
  else
    r.tile(a, 0u, sq, sw, mask, lg, rows, lane, st);
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

// f(Rows<width, rows>()) of the call's type, width and rows.  256 columns have at
// most 16 rows.
template <typename F>
cudaError_t by_rows(const CacheAttn& a, int D, F f) {
  if (a.c.dt != AVITS_BF16) {
    switch (a.rows + D) {
      case 64 + 4: return f(RowsF32<64, 4>());
      case 128 + 4: return f(RowsF32<128, 4>());
      case 256 + 4: return f(RowsF32<256, 4>());
      case 64 + 8: return f(RowsF32<64, 8>());
      case 128 + 8: return f(RowsF32<128, 8>());
      default: return f(RowsF32<256, 8>());
    }
  }
  switch (a.rows + D) {
    case 64 + 8: return f(RowsBf16<64, 8>());
    case 128 + 8: return f(RowsBf16<128, 8>());
    case 256 + 8: return f(RowsBf16<256, 8>());
    case 64 + 16: return f(RowsBf16<64, 16>());
    case 128 + 16: return f(RowsBf16<128, 16>());
    case 256 + 16: return f(RowsBf16<256, 16>());
    case 64 + 32: return f(RowsBf16<64, 32>());
    default: return f(RowsBf16<128, 32>());
  }
}

// The launchers of the two forms, by width (64, 128, 256) and rows of a unit.
cudaError_t launch_line(CacheAttn& a, int D, int num_sms, cudaStream_t s);
cudaError_t launch_cluster(CacheAttn& a, int D, int ncta, int warps, cudaStream_t s);

// Shared prefixes: own tokens as parts, a CTA of `warps` warps per unit; prefix and own tokens in
// one launch, a cluster of ncta CTAs per unit.
cudaError_t launch_own_parts(CacheAttn& a, int D, int warps, cudaStream_t s);
cudaError_t launch_both(CacheAttn& a, const CacheAttn& p, int D, int ncta, cudaStream_t s);

// Prefixes on the tensor cores: units of 128 rows on two CTAs to an SM, or of 256 on one, tiles
// of 64 keys.  prefix_tc_box: tokens of a copy, 0 where the type, the width or the pages' layout
// is not theirs.
constexpr int kPrefixRows = 128, kPrefixTile = 64;
int prefix_tc_box(const avits_kv_cache& c);
cudaError_t launch_prefix_tc(const CacheAttn& a, cudaStream_t s);

}  // namespace cache
}  // namespace avits
