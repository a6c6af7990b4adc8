// cache_attention.cu — attention of one new token per sequence over a paged
// key-value cache, with the weight each cached token got.
//
// For sequence b, KV head hk and the G query heads h that share it:
//   x_hj = scale q_h . k_j,  lse_h = log sum_j exp x_hj,  o_h = sum_j exp(x_hj - lse_h) v_j,
//   acc_j (+)= weight mean_h exp(x_hj - lse_h)
// Every key and value is read once, so HBM bounds it: 4 G operations per bf16
// element of K and V.
//
// Split.  A sequence's keys are cut into tiles of 16; all tiles of all (b, hk,
// row group) form one line, cut into equal pieces, one per CTA, so that uneven
// lengths and few heads load the SMs alike.  A CTA finds its piece by a scan of
// the lengths.  Inside a piece each warp takes tiles of its own with a running
// maximum, sum and O in registers; the warps meet once per (b, hk) at the end.
// A (b, hk) that lies in one piece is finished there; of the others each piece
// leaves its maximum, sum and O, and the second kernel joins them.
//
// The weights need the whole row's lse: the first kernel leaves the logits
// (fp32), the second sums exp(x - lse) over the group's heads, in a fixed order.
#include "cache_common.cuh"
#include "avits_internal.h"

namespace avits {
namespace {

constexpr int kTile = 16;         // keys per tile
constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kMinTiles = 4;      // tiles of the smallest piece: one per warp
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
  int rt;           // row tiles of 8 heads side by side in a CTA (1, 2 or 4)
  int groups;       // row groups (units) per KV head: ceil(G / (8 rt))
  int grid;         // CTAs of the first kernel
  float scale2;     // scale * log2(e)
  float wmean;      // weight / G
  int add;
  // workspace
  int* starts;      // [B+1] first tile of a sequence on the line
  float* lse2;      // [B,H] log2-domain lse of rows finished in one piece
  float2* pml;      // [2 grid][8 rt] maximum and sum of a piece's row
  float* po;        // [2 grid][8 rt][d] its O
  float* logits;    // [B,H,ld] log2-domain logits (weights wanted)
  int64_t ld;
  unsigned int* status;
};

__device__ __forceinline__ int tiles_of(const CacheAttn& a, int b) {
  return (cache_len(a.c, b) + kTile - 1) / kTile;
}

// The piece's row: what the CTA's warps agree on for one (b, hk, row group).
struct Unit {
  int b, hk, row0;    // first row (query head of the group) of this warp's row tile
  int rows;           // rows of this warp's tile (<= 8; <= 0: nothing to do)
  int len;
};

// Rows' pages of one tile: lane l holds the page and the place of key l % 16.
struct TileKeys {
  int page, slot;
};

__device__ __forceinline__ int table_entry(const CacheAttn& a, const int32_t* table, int tile,
                                           int len, int lane) {
  const int j = tile * kTile + (lane & 15);
  return j < len ? table[a.page.div(j)] : -1;
}
__device__ __forceinline__ TileKeys tile_keys(const CacheAttn& a, int entry, int tile, int len,
                                              int lane) {
  const int j = tile * kTile + (lane & 15);
  TileKeys t;
  t.slot = j - a.page.div(j) * a.c.page_size;
  t.page = j < len ? checked_page(a.c, entry, a.status) : -1;
  return t;
}

// ------------------------------------------------------------------ bf16 --
// m16n8k16 with the 8 heads of a row tile in rows 0-7.  The product over d may
// take d in any order, the same for Q and K, and O's columns may come in any
// order: a lane loads 16 bytes of a key's row and 16 bytes of a value's row
// straight into operand registers, no shared memory in between.  The weights
// enter P V as two bf16 parts (value and rest, 16 significant bits together),
// the rest in rows 8-15 that are free: O is as exact as with fp32 weights.
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                         uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
      "{%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

template <int D, bool kScore>
struct RowsBf16 {
  static constexpr int kC = D / 32;     // 16-byte pieces of a key's row per lane
  static constexpr int kV = D / 64;     // of a value's row
  static constexpr int kQBytes = D / 16 * 32 * 8;   // Q fragments of a row tile
  static constexpr int kWarpBytes = 0;
  static constexpr int kStride = D + 4; // row stride of the CTA's O buffer

  float m, l;
  float o[kV][8][4];

  // Q's fragments of one row tile: per step of 16 d values and lane, the pairs
  // a lane multiplies with the two words of its key piece.
  __device__ static void stage_q(const CacheAttn& a, const Unit& u, char* sq, int lane) {
    const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(a.q) + (int64_t)u.b * a.q_sb;
    const int g = lane >> 2, t = lane & 3;
    const bool ok = g < u.rows;
    const __nv_bfloat16* row = q + (int64_t)(u.hk * a.G + u.row0 + (ok ? g : 0)) * a.q_sh;
    uint2* out = reinterpret_cast<uint2*>(sq);
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      const int d0 = (s >> 1) * 32 + t * 8 + (s & 1) * 4;
      uint32_t w[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int dd = d0 + 2 * i;
        uint32_t x = 0u;
        if (ok && dd < a.c.d)
          x = (uint32_t)__bfloat16_as_ushort(row[dd]) |
              ((uint32_t)__bfloat16_as_ushort(row[dd + 1]) << 16);
        w[i] = x;
      }
      out[s * 32 + lane] = make_uint2(w[0], w[1]);
    }
  }

  __device__ __forceinline__ void reset() {
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int c = 0; c < kV; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[c][j][e] = 0.f;
  }

  __device__ __forceinline__ void load_k(const CacheAttn& a, const TileKeys& tk,
                                         const __nv_bfloat16* kb, uint4 (&k)[2][kC], int lane) {
    const int g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const int page = __shfl_sync(0xffffffffu, tk.page, g + 8 * n);
      const int slot = __shfl_sync(0xffffffffu, tk.slot, g + 8 * n);
      const __nv_bfloat16* row = kb + (int64_t)page * a.c.k_sp + (int64_t)slot * a.c.k_st;
#pragma unroll
      for (int c = 0; c < kC; ++c) {
        k[n][c] = make_uint4(0u, 0u, 0u, 0u);
        if (page >= 0 && c * 32 + t * 8 < a.c.d) {
          const void* p = row + c * 32 + t * 8;
          k[n][c] = a.rt == 1 ? ld_once(p) : ld_shared_by_warps(p);
        }
      }
    }
  }

  __device__ __forceinline__ void run(const CacheAttn& a, const Unit& u, const char* sq, char*,
                                      int tile, int t1, int step, int lane) {
    reset();
    const int g = lane >> 2, t = lane & 3;
    const int32_t* table = a.c.block_table + (int64_t)u.b * a.c.table_sb;
    const __nv_bfloat16* kb =
        static_cast<const __nv_bfloat16*>(a.c.k_pages) + (int64_t)u.hk * a.c.k_sh;
    const __nv_bfloat16* vb =
        static_cast<const __nv_bfloat16*>(a.c.v_pages) + (int64_t)u.hk * a.c.v_sh;
    float* lg = kScore ? a.logits + ((int64_t)u.b * a.H + u.hk * a.G + u.row0 + g) * a.ld : nullptr;
    const bool keep_logits = kScore && g < u.rows;
    const uint2* qf = reinterpret_cast<const uint2*>(sq);
    if (tile >= t1) return;
    uint4 k[2][kC];
    TileKeys tk = tile_keys(a, table_entry(a, table, tile, u.len, lane), tile, u.len, lane);
    load_k(a, tk, kb, k, lane);
    for (; tile < t1; tile += step) {
      // this tile's values, and the next one's page numbers, on their way
      uint4 v[4][kV];
      bool live[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = 2 * t + (i & 1) + 8 * (i >> 1);
        const int page = __shfl_sync(0xffffffffu, tk.page, key);
        const int slot = __shfl_sync(0xffffffffu, tk.slot, key);
        live[i] = page >= 0;
        const __nv_bfloat16* row = vb + (int64_t)page * a.c.v_sp + (int64_t)slot * a.c.v_st;
#pragma unroll
        for (int c = 0; c < kV; ++c) {
          v[i][c] = make_uint4(0u, 0u, 0u, 0u);
          if (live[i] && c * 64 + g * 8 < a.c.d) {
            const void* p = row + c * 64 + g * 8;
            v[i][c] = a.rt == 1 ? ld_once(p) : ld_shared_by_warps(p);
          }
        }
      }
      const int next = tile + step;
      const int entry = next < t1 ? table_entry(a, table, next, u.len, lane) : -1;
      float s[2][4] = {};
#pragma unroll
      for (int c = 0; c < kC; ++c) {
        const uint2 q0 = qf[(2 * c) * 32 + lane], q1 = qf[(2 * c + 1) * 32 + lane];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          mma16816(s[n], q0.x, 0u, q0.y, 0u, k[n][c].x, k[n][c].y);
          mma16816(s[n], q1.x, 0u, q1.y, 0u, k[n][c].z, k[n][c].w);
        }
      }
      if (next < t1) {
        tk = tile_keys(a, entry, next, u.len, lane);
        load_k(a, tk, kb, k, lane);
      }
      // keys 2t, 2t+1 (s[0]) and 8+2t, 9+2t (s[1]) of row g
      float x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = live[i] ? s[i >> 1][i & 1] * a.scale2 : -INFINITY;
      if (keep_logits) {
        float2* to = reinterpret_cast<float2*>(lg + (int64_t)tile * kTile + 2 * t);
        to[0] = make_float2(x[0], x[1]);
        to[4] = make_float2(x[2], x[3]);
      }
      float top = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      if (__any_sync(0xffffffffu, top > m)) {
        const float mn = fmaxf(m, top);
        const float f = mn == m ? 1.f : ex2(m - mn);   // m = -inf: 0
        m = mn;
        l *= f;
#pragma unroll
        for (int c = 0; c < kV; ++c)
#pragma unroll
          for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[c][j][e] *= f;
      }
      const float ref = m == -INFINITY ? 0.f : m;
      float p[4], r[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[i] = ex2(x[i] - ref);
        l += p[i];
        r[i] = p[i] - __bfloat162float(__float2bfloat16_rn(p[i]));
      }
      const uint32_t a0 = pack_bf16(p[0], p[1]), a2 = pack_bf16(p[2], p[3]);
      const uint32_t a1 = pack_bf16(r[0], r[1]), a3 = pack_bf16(r[2], r[3]);
#pragma unroll
      for (int c = 0; c < kV; ++c) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t v0 = (&v[0][c].x)[w], v1 = (&v[1][c].x)[w];
          const uint32_t v2 = (&v[2][c].x)[w], v3 = (&v[3][c].x)[w];
          mma16816(o[c][2 * w], a0, a1, a2, a3, __byte_perm(v0, v1, 0x5410),
                   __byte_perm(v2, v3, 0x5410));
          mma16816(o[c][2 * w + 1], a0, a1, a2, a3, __byte_perm(v0, v1, 0x7632),
                   __byte_perm(v2, v3, 0x7632));
        }
      }
    }
    l += __shfl_xor_sync(0xffffffffu, l, 1);
    l += __shfl_xor_sync(0xffffffffu, l, 2);
  }

  // (maximum, sum) of the warp's rows, one lane per row
  __device__ __forceinline__ void put_ml(float2* ml, int lane) const {
    if ((lane & 3) == 0) ml[lane >> 2] = make_float2(m, l);
  }
  // O times f(row) into the CTA's buffer
  __device__ __forceinline__ void put_o(float* buf, const float* f, int lane) const {
    const int g = lane >> 2, t = lane & 3;
    const float fr = f[g];
#pragma unroll
    for (int c = 0; c < kV; ++c) {
      float4* to = reinterpret_cast<float4*>(buf + g * kStride + c * 64 + 16 * t);
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float4 x;
          float* px = &x.x;
#pragma unroll
          for (int j = 0; j < 4; ++j) px[j] = (o[c][4 * h + j][e] + o[c][4 * h + j][e + 2]) * fr;
          to[2 * e + h] = x;
        }
    }
  }
};

// ------------------------------------------------------------------ fp32 --
// CUDA cores in fp32.  Q K^T: 8 lanes to a key (16-byte pieces of its row), 4
// keys at a time; a lane's partial dot products of the 8 heads are summed over
// the 8 lanes by halving, which leaves head lane % 8 with the lane.  P V: a
// lane owns columns of O and reads the weights from shared memory.
template <int D, bool kScore>
struct RowsF32 {
  static constexpr int kC = D / 32;
  static constexpr int kKeysPerV = D >= 128 ? 1 : 128 / D;   // value rows read side by side
  static constexpr int kV = D >= 128 ? D / 128 : 1;
  static constexpr int kBlock = kC < 4 ? kC : 4;             // pieces of a key in registers
  static constexpr int kQBytes = 8 * D * 4;
  static constexpr int kWarpBytes = kTile * 8 * 4;
  static constexpr int kStride = D + 4;

  float m, l;            // of row lane % 8; l: this lane's keys only until the end
  float o[8][kV][4];

  __device__ static void stage_q(const CacheAttn& a, const Unit& u, char* sq, int lane) {
    const float* q = static_cast<const float*>(a.q) + (int64_t)u.b * a.q_sb;
    float* out = reinterpret_cast<float*>(sq);
#pragma unroll 1
    for (int g = 0; g < 8; ++g) {
      const float* row = q + (int64_t)(u.hk * a.G + u.row0 + (g < u.rows ? g : 0)) * a.q_sh;
      for (int d = lane; d < D; d += 32) out[g * D + d] = g < u.rows && d < a.c.d ? row[d] : 0.f;
    }
  }

  __device__ __forceinline__ void run(const CacheAttn& a, const Unit& u, const char* sq, char* sw,
                                      int tile, int t1, int step, int lane) {
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int g = 0; g < 8; ++g)
#pragma unroll
      for (int c = 0; c < kV; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[g][c][e] = 0.f;
    const int kg = lane >> 3, t8 = lane & 7;
    const int32_t* table = a.c.block_table + (int64_t)u.b * a.c.table_sb;
    const float* kb = static_cast<const float*>(a.c.k_pages) + (int64_t)u.hk * a.c.k_sh;
    const float* vb = static_cast<const float*>(a.c.v_pages) + (int64_t)u.hk * a.c.v_sh;
    const float* q = reinterpret_cast<const float*>(sq);
    float* sp = reinterpret_cast<float*>(sw);
    float* lg = kScore ? a.logits + ((int64_t)u.b * a.H + u.hk * a.G + u.row0 + t8) * a.ld : nullptr;
    const bool keep_logits = kScore && t8 < u.rows;
    for (; tile < t1; tile += step) {
      const TileKeys tk = tile_keys(a, table_entry(a, table, tile, u.len, lane), tile, u.len, lane);
      // a lane's keys: kg*4 .. kg*4+3
      const float* row[4];
      bool live[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int page = __shfl_sync(0xffffffffu, tk.page, kg * 4 + i);
        const int slot = __shfl_sync(0xffffffffu, tk.slot, kg * 4 + i);
        live[i] = page >= 0;
        row[i] = kb + (int64_t)page * a.c.k_sp + (int64_t)slot * a.c.k_st;
      }
      float s[4][8] = {};
#pragma unroll 1
      for (int cb = 0; cb < kC; cb += kBlock) {
        float4 k[4][kBlock];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int c = 0; c < kBlock; ++c) {
            const int d = (cb + c) * 32 + t8 * 4;
            k[i][c] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (live[i] && d < a.c.d) {
              const uint4 w = ld_shared_by_warps(row[i] + d);
              k[i][c] = make_float4(__uint_as_float(w.x), __uint_as_float(w.y),
                                    __uint_as_float(w.z), __uint_as_float(w.w));
            }
          }
#pragma unroll
        for (int g = 0; g < 8; ++g)
#pragma unroll
          for (int c = 0; c < kBlock; ++c) {
            const float4 qv =
                *reinterpret_cast<const float4*>(q + g * D + (cb + c) * 32 + t8 * 4);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              s[i][g] = fmaf(qv.x, k[i][c].x, fmaf(qv.y, k[i][c].y,
                        fmaf(qv.z, k[i][c].z, fmaf(qv.w, k[i][c].w, s[i][g]))));
          }
      }
      float x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
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
        x[i] = live[i] ? dot * a.scale2 : -INFINITY;
      }
      if (keep_logits)
        *reinterpret_cast<float4*>(lg + (int64_t)tile * kTile + kg * 4) =
            make_float4(x[0], x[1], x[2], x[3]);
      float top = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
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
      for (int i = 0; i < 4; ++i) {
        const float p = ex2(x[i] - ref);
        l += p;
        sp[(kg * 4 + i) * 8 + t8] = p;
      }
      __syncwarp();
      const int sub = kKeysPerV == 1 ? 0 : lane / (32 / kKeysPerV);
      const int col = kKeysPerV == 1 ? lane * 4 : (lane % (32 / kKeysPerV)) * 4;
#pragma unroll 1
      for (int j0 = 0; j0 < kTile; j0 += 8) {
        float4 v[8 / kKeysPerV][kV];
#pragma unroll
        for (int j = 0; j < 8 / kKeysPerV; ++j) {
          const int key = j0 + j * kKeysPerV + sub;
          const int page = __shfl_sync(0xffffffffu, tk.page, key);
          const int slot = __shfl_sync(0xffffffffu, tk.slot, key);
          const float* vr = vb + (int64_t)page * a.c.v_sp + (int64_t)slot * a.c.v_st;
#pragma unroll
          for (int c = 0; c < kV; ++c) {
            v[j][c] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (page >= 0 && col + c * 128 < a.c.d) {
              const uint4 w = ld_shared_by_warps(vr + col + c * 128);
              v[j][c] = make_float4(__uint_as_float(w.x), __uint_as_float(w.y),
                                    __uint_as_float(w.z), __uint_as_float(w.w));
            }
          }
        }
#pragma unroll
        for (int j = 0; j < 8 / kKeysPerV; ++j) {
          const float4* pp =
              reinterpret_cast<const float4*>(sp + (j0 + j * kKeysPerV + sub) * 8);
          const float4 pa = pp[0], pb = pp[1];
          const float p[8] = {pa.x, pa.y, pa.z, pa.w, pb.x, pb.y, pb.z, pb.w};
#pragma unroll
          for (int g = 0; g < 8; ++g)
#pragma unroll
            for (int c = 0; c < kV; ++c) {
              o[g][c][0] = fmaf(p[g], v[j][c].x, o[g][c][0]);
              o[g][c][1] = fmaf(p[g], v[j][c].y, o[g][c][1]);
              o[g][c][2] = fmaf(p[g], v[j][c].z, o[g][c][2]);
              o[g][c][3] = fmaf(p[g], v[j][c].w, o[g][c][3]);
            }
        }
      }
    }
    l += __shfl_xor_sync(0xffffffffu, l, 8);
    l += __shfl_xor_sync(0xffffffffu, l, 16);
    if (kKeysPerV > 1) {
#pragma unroll
      for (int g = 0; g < 8; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          o[g][0][e] += __shfl_xor_sync(0xffffffffu, o[g][0][e], 16);
    }
  }

  __device__ __forceinline__ void put_ml(float2* ml, int lane) const {
    if (lane < 8) ml[lane] = make_float2(m, l);
  }
  __device__ __forceinline__ void put_o(float* buf, const float* f, int lane) const {
    if (kKeysPerV > 1 && lane >= 16) return;
#pragma unroll
    for (int g = 0; g < 8; ++g)
#pragma unroll
      for (int c = 0; c < kV; ++c) {
        const float fr = f[g];
        *reinterpret_cast<float4*>(buf + g * kStride + lane * 4 + c * 128) = make_float4(
            o[g][c][0] * fr, o[g][c][1] * fr, o[g][c][2] * fr, o[g][c][3] * fr);
      }
  }
};

// ----------------------------------------------------------- first kernel --
template <typename Rows>
constexpr size_t smem_bytes(int rt) {
  return (size_t)kWarps * 8 * Rows::kStride * 4 + (size_t)rt * Rows::kQBytes +
         (size_t)kWarps * Rows::kWarpBytes;
}

template <typename T, int D, typename Rows, int kMinCtas>
__global__ void __launch_bounds__(kThreads, kMinCtas)
cache_attention_kernel(const __grid_constant__ CacheAttn a) {
  extern __shared__ __align__(16) char smem[];
  __shared__ float2 s_ml[kWarps][8];
  __shared__ float s_f[kWarps][8];
  __shared__ int s_scan[kWarps], s_b, s_off;
  const int tid = threadIdx.x, w = tid >> 5, lane = tid & 31;
  pdl_wait_then_trigger();

  // where this CTA's piece of the line of tiles begins
  const int B = a.c.B, units = a.c.Hkv * a.groups;
  const int each = (B + kThreads - 1) / kThreads;
  const int b0 = min(B, tid * each), b1 = min(B, b0 + each);
  int sum = 0;
  for (int b = b0; b < b1; ++b) {
    sum += tiles_of(a, b) * units;
    if (blockIdx.x == 0) check_cache_len(a.c, b, a.status);
  }
  int inc = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += y;
  }
  if (lane == 31) s_scan[w] = inc;
  __syncthreads();
  int total = 0, before = inc - sum;
#pragma unroll
  for (int i = 0; i < kWarps; ++i) {
    if (i < w) before += s_scan[i];
    total += s_scan[i];
  }
  if (blockIdx.x == 0) {
    int at = before;
    for (int b = b0; b < b1; ++b) {
      a.starts[b] = at;
      at += tiles_of(a, b) * units;
    }
    if (tid == 0) a.starts[B] = total;
  }
  const int per = max(kMinTiles, (total + a.grid - 1) / a.grid);
  const int first = blockIdx.x * per;
  if (first >= total) return;
  if (before <= first && first < before + sum) {
    int at = before, b = b0;
    for (;; ++b) {
      const int n = tiles_of(a, b) * units;
      if (first < at + n) break;
      at += n;
    }
    s_b = b;
    s_off = first - at;
  }
  __syncthreads();

  float* s_o = reinterpret_cast<float*>(smem);
  char* s_q = smem + kWarps * 8 * Rows::kStride * 4;
  char* s_w = s_q + a.rt * Rows::kQBytes + w * Rows::kWarpBytes;
  int left = min(per, total - first), b = s_b, off = s_off;
  const int rt = w & (a.rt - 1), step = kWarps / a.rt, lead = w / a.rt;
  bool is_first = true;
  Rows rows;
  while (left > 0) {
    Unit u;
    u.len = cache_len(a.c, b);
    const int nt = (u.len + kTile - 1) / kTile;
    if (nt == 0) {
      ++b;
      continue;
    }
    const int unit = off / nt, t0 = off - unit * nt, t1 = min(nt, t0 + left);
    const int rg = unit % a.groups;
    u.b = b;
    u.hk = unit / a.groups;
    u.row0 = (rg * a.rt + rt) * 8;
    u.rows = a.G - u.row0;
    if (lead == 0) Rows::stage_q(a, u, s_q + rt * Rows::kQBytes, lane);
    __syncthreads();   // Q is there; everybody is done with the last unit's buffers
    rows.run(a, u, s_q + rt * Rows::kQBytes, s_w, t0 + lead, u.rows > 0 ? t1 : 0, step, lane);
    rows.put_ml(s_ml[w], lane);
    __syncthreads();
    if (lane < 8) {   // this warp's rows relative to the row's maximum over the warps
      float top = -INFINITY;
      for (int i = rt; i < kWarps; i += a.rt) top = fmaxf(top, s_ml[i][lane].x);
      const float mine = s_ml[w][lane].x;
      s_f[w][lane] = mine == -INFINITY ? 0.f : ex2(mine - top);
    }
    __syncwarp();
    rows.put_o(s_o + w * 8 * Rows::kStride, s_f[w], lane);
    __syncthreads();
    // sum over the warps, and out: finished, or as this piece's part
    const bool whole = t0 == 0 && t1 == nt;
    const int slot = 2 * blockIdx.x + (is_first ? 0 : 1);
    const int nrow = 8 * a.rt;
    for (int i = tid; i < nrow * (D / 4); i += kThreads) {
      const int r = i / (D / 4), d = (i - r * (D / 4)) * 4, r8 = r & 7, wr = r >> 3;
      const int row = rg * nrow + r;
      if (row >= a.G || d >= a.c.d) continue;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      float top = -INFINITY, l = 0.f;
      for (int k = wr; k < kWarps; k += a.rt) {
        const float4 x = *reinterpret_cast<const float4*>(s_o + (k * 8 + r8) * Rows::kStride + d);
        v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
        top = fmaxf(top, s_ml[k][r8].x);
        l += s_f[k][r8] * s_ml[k][r8].y;
      }
      const int h = u.hk * a.G + row;
      if (whole) {
        const float inv = l > 0.f ? 1.f / l : (l != l ? l : 0.f);
        T* out = static_cast<T*>(a.o) + (int64_t)b * a.o_sb + (int64_t)h * a.o_sh + d;
        store_elem(out, 0, v.x * inv);
        store_elem(out, 1, v.y * inv);
        store_elem(out, 2, v.z * inv);
        store_elem(out, 3, v.w * inv);
        if (d == 0) {
          const float e = l > 0.f ? top + log2f(l) : (l != l ? l : -INFINITY);
          a.lse2[(int64_t)b * a.H + h] = e;
          if (a.lse) a.lse[(int64_t)b * a.H + h] = e * kLn2;
        }
      } else {
        *reinterpret_cast<float4*>(a.po + ((int64_t)slot * nrow + r) * a.c.d + d) = v;
        if (d == 0) a.pml[slot * nrow + r] = make_float2(top, l);
      }
    }
    is_first = false;
    left -= t1 - t0;
    off += t1 - t0;
    if (off == nt * units) {
      ++b;
      off = 0;
    }
  }
}

// ---------------------------------------------------------- second kernel --
// Block (b, hk, part): the lse of the group's rows from their pieces, the
// weights of the part's keys, and O of the rows part, part + parts, ...
constexpr int kJoinThreads = 256;
constexpr int kMaxGroup = 256;

template <typename T>
__global__ void __launch_bounds__(kJoinThreads)
cache_join_kernel(const __grid_constant__ CacheAttn a, int parts, int keys, int score) {
  __shared__ float s_lse2[kMaxGroup];
  __shared__ float4 s_sum[kJoinThreads];
  pdl_wait_then_trigger();
  const int tid = threadIdx.x, w = tid >> 5, lane = tid & 31;
  const int bh = blockIdx.x / parts, part = blockIdx.x - bh * parts;
  const int b = bh / a.c.Hkv, hk = bh - b * a.c.Hkv;
  const int len = cache_len(a.c, b), nt = (len + kTile - 1) / kTile;
  const int nrow = 8 * a.rt, d4 = a.c.d / 4;
  if (nt == 0) {
    for (int r = part; r < a.G; r += parts) {
      const int h = hk * a.G + r;
      T* out = static_cast<T*>(a.o) + (int64_t)b * a.o_sb + (int64_t)h * a.o_sh;
      for (int d = tid; d < a.c.d; d += kJoinThreads) store_elem(out, d, 0.f);
      if (a.lse && tid == 0) a.lse[(int64_t)b * a.H + h] = -INFINITY;
    }
    return;
  }
  const int per = max(kMinTiles, (a.starts[a.c.B] + a.grid - 1) / a.grid);
  const int start = a.starts[b];
  for (int r = w; r < a.G; r += kJoinThreads / 32) {
    const int rg = r / nrow, T0 = start + (hk * a.groups + rg) * nt, T1 = T0 + nt;
    const int c0 = T0 / per, c1 = (T1 - 1) / per;
    const int h = hk * a.G + r;
    float e;
    if (c0 == c1) {
      e = a.lse2[(int64_t)b * a.H + h];
    } else {
      float top = -INFINITY, l = 0.f;
      for (int c = c0 + lane; c <= c1; c += 32) {
        const int slot = 2 * c + (c == c0 && T0 != c0 * per ? 1 : 0);
        const float2 x = a.pml[slot * nrow + (r - rg * nrow)];
        const float mn = fmaxf(top, x.x), ref = mn == -INFINITY ? 0.f : mn;
        l = l * ex2(top - ref) + x.y * ex2(x.x - ref);   // a NaN stays one
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
      e = l > 0.f ? top + log2f(l) : (l != l ? l : -INFINITY);
      if (a.lse && lane == 0 && r % parts == part) a.lse[(int64_t)b * a.H + h] = e * kLn2;
    }
    if (lane == 0) s_lse2[r] = e;
  }
  __syncthreads();
  if (score) {
    const int j1 = min(len, (part + 1) * keys);
    float* acc = a.c.acc + (int64_t)b * a.c.acc_sb + (int64_t)hk * a.c.acc_sh;
    const float* lg = a.logits + ((int64_t)b * a.H + hk * a.G) * a.ld;
    for (int j = part * keys + tid; j < j1; j += kJoinThreads) {
      float s = 0.f;
      for (int r = 0; r < a.G; ++r) {
        const float e = s_lse2[r];
        // nothing to attend to (every page out of range): no weight
        s += e == -INFINITY ? 0.f : ex2(lg[(int64_t)r * a.ld + j] - e);
      }
      s *= a.wmean;
      acc[j] = a.add ? acc[j] + s : s;
    }
  }
  // O of the rows that were cut
  for (int r = part; r < a.G; r += parts) {
    const int rg = r / nrow, T0 = start + (hk * a.groups + rg) * nt, T1 = T0 + nt;
    const int c0 = T0 / per, c1 = (T1 - 1) / per;
    if (c0 == c1) continue;
    const float e = s_lse2[r];
    const int h = hk * a.G + r, rr = r - rg * nrow;
    const int lanes = kJoinThreads / d4, col = tid % d4, sub = tid / d4;
    const float none = e != e ? e : 0.f;
    float4 v = make_float4(none, none, none, none);
    if (sub < lanes && e != -INFINITY) {
      for (int c = c0 + sub; c <= c1; c += lanes) {
        const int slot = 2 * c + (c == c0 && T0 != c0 * per ? 1 : 0);
        const float mx = a.pml[slot * nrow + rr].x;
        if (mx == -INFINITY) continue;
        const float f = ex2(mx - e);
        const float4 x =
            *reinterpret_cast<const float4*>(a.po + ((int64_t)slot * nrow + rr) * a.c.d + col * 4);
        v.x = fmaf(f, x.x, v.x); v.y = fmaf(f, x.y, v.y);
        v.z = fmaf(f, x.z, v.z); v.w = fmaf(f, x.w, v.w);
      }
    }
    __syncthreads();
    s_sum[tid] = v;
    __syncthreads();
    if (sub == 0) {
      for (int k = 1; k < lanes; ++k) {
        const float4 x = s_sum[k * d4 + col];
        v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
      }
      T* out = static_cast<T*>(a.o) + (int64_t)b * a.o_sb + (int64_t)h * a.o_sh + col * 4;
      store_elem(out, 0, v.x);
      store_elem(out, 1, v.y);
      store_elem(out, 2, v.z);
      store_elem(out, 3, v.w);
    }
  }
}

constexpr int ctas_per_sm(int D) { return D <= 128 ? 3 : 2; }

int padded_d(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

struct Shape {
  int G, rt, groups, grid;
  long long tiles;
};

Shape shape_of(const avits_kv_cache& c, int H, int num_sms) {
  Shape s;
  s.G = H / c.Hkv;
  s.rt = s.G <= 8 ? 1 : s.G <= 16 ? 2 : 4;
  s.groups = (s.G + 8 * s.rt - 1) / (8 * s.rt);
  s.tiles = (long long)c.B * c.Hkv * s.groups * ((c.max_len + kTile - 1) / kTile);
  const long long most = (s.tiles + kMinTiles - 1) / kMinTiles;
  const long long full = (long long)num_sms * ctas_per_sm(padded_d(c.d));
  s.grid = (int)(most < full ? (most > 0 ? most : 1) : full);
  return s;
}

size_t up16(size_t n) { return (n + 15) / 16 * 16; }

struct Layout {
  size_t starts, lse2, pml, po, logits, total;
  int64_t ld;
};

Layout layout_of(const avits_kv_cache& c, int H, const Shape& s, bool score) {
  Layout l;
  const size_t nrow = 8 * s.rt;
  l.ld = (c.max_len + kTile - 1) / kTile * (int64_t)kTile;
  l.starts = 0;
  l.lse2 = up16(((size_t)c.B + 1) * 4);
  l.pml = l.lse2 + up16((size_t)c.B * H * 4);
  l.po = l.pml + up16((size_t)2 * s.grid * nrow * 8);
  l.logits = l.po + up16((size_t)2 * s.grid * nrow * c.d * 4);
  l.total = l.logits + (score ? (size_t)c.B * H * l.ld * 4 : 0);
  return l;
}

template <typename T, int D, typename Rows>
cudaError_t launch_rows(const CacheAttn& a, cudaStream_t s) {
  constexpr int kCtas = ctas_per_sm(D);
  constexpr auto kernel = cache_attention_kernel<T, D, Rows, kCtas>;
  const cudaError_t e = prefer_max_shared<kernel, (int)smem_bytes<Rows>(4)>();
  if (e != cudaSuccess) return e;
  return launch_pdl(kernel, dim3(a.grid), dim3(kThreads), smem_bytes<Rows>(a.rt), s, a);
}

template <typename T, template <int, bool> class Rows>
cudaError_t launch_typed(const CacheAttn& a, bool score, cudaStream_t s) {
  cudaError_t e;
  switch (padded_d(a.c.d)) {
    case 64:
      e = score ? launch_rows<T, 64, Rows<64, true>>(a, s) : launch_rows<T, 64, Rows<64, false>>(a, s);
      break;
    case 128:
      e = score ? launch_rows<T, 128, Rows<128, true>>(a, s)
                : launch_rows<T, 128, Rows<128, false>>(a, s);
      break;
    default:
      e = score ? launch_rows<T, 256, Rows<256, true>>(a, s)
                : launch_rows<T, 256, Rows<256, false>>(a, s);
  }
  if (e != cudaSuccess) return e;
  constexpr auto join = cache_join_kernel<T>;
  e = prefer_max_shared<join>();
  if (e != cudaSuccess) return e;
  // parts of a (b, hk): as many as its keys' weights or its rows' joins are
  // worth, about two blocks per SM in all
  const long long bh = (long long)a.c.B * a.c.Hkv;
  const int most = score ? (a.c.max_len + kJoinThreads - 1) / kJoinThreads : a.G;
  long long parts = (304 + bh - 1) / bh;
  parts = parts < most ? parts : most;
  if (score && (a.c.max_len + parts - 1) / parts > 4096) parts = (a.c.max_len + 4095) / 4096;
  if (parts < 1) parts = 1;
  const int keys = (int)((a.c.max_len + parts - 1) / parts);
  return launch_pdl(join, dim3((unsigned)(bh * parts)), dim3(kJoinThreads), 0, s, a, (int)parts,
                    keys, score ? 1 : 0);
}

}  // namespace

bool cache_attention_sizes_ok(const avits_kv_cache& c, int H) {
  if (H / c.Hkv > kMaxGroup) return false;
  const Shape s = shape_of(c, H, 1);
  return s.tiles < (1ll << 30) && (long long)c.B * H < (1ll << 30);
}

size_t cache_attention_workspace(const avits_kv_cache& c, int H, bool score, int num_sms) {
  return layout_of(c, H, shape_of(c, H, num_sms), score).total;
}

cudaError_t launch_cache_attention(const CacheAttnCall& call, int num_sms, unsigned int* status,
                                   cudaStream_t s) {
  const avits_kv_cache& c = call.cache;
  const bool score = call.weights != AVITS_WEIGHTS_NONE;
  const Shape sh = shape_of(c, call.H, num_sms);
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
  a.rt = sh.rt;
  a.groups = sh.groups;
  a.grid = sh.grid;
  a.scale2 = call.scale * kLog2e;
  a.wmean = call.weight / (float)sh.G;
  a.add = call.weights == AVITS_WEIGHTS_ADD;
  a.starts = reinterpret_cast<int*>(ws + l.starts);
  a.lse2 = reinterpret_cast<float*>(ws + l.lse2);
  a.pml = reinterpret_cast<float2*>(ws + l.pml);
  a.po = reinterpret_cast<float*>(ws + l.po);
  a.logits = reinterpret_cast<float*>(ws + l.logits);
  a.ld = l.ld;
  a.status = status;
  return c.dt == AVITS_BF16 ? launch_typed<__nv_bfloat16, RowsBf16>(a, score, s)
                            : launch_typed<float, RowsF32>(a, score, s);
}

}  // namespace avits
