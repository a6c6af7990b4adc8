// rotate.cuh — norm of each head and rotation by position, queries and keys in one
// pass; in a second form keys and values go straight to their places in a paged cache.
//
// For a head's vector x of d values at position p:
//   y = x / sqrt(mean x^2 + eps) * w                       (or y = x)
//   (y_a, y_b) of pair i -> m (y_a cos t - y_b sin t, y_b cos t + y_a sin t),
//   t = 2 pi p f_i, pairs (2i, 2i+1) or (i, i + rot/2), i < rot/2; the rest stays.
// All in fp32, rounded once.  Angles: f_i is a 64-bit binary fraction of a turn, so that
// p f_i mod 1 is the low 64 bits of an integer product, exact for the f_i given; its top
// 32 bits become an fp32 angle in [-pi, pi).  No table of cosines is read, and far
// positions add nothing but p times the error of f_i (avits_rotary_frequencies computes them
// in fp64, off by up to 2^-53: p 2^-53 turns).
//
// Bytes bound it: q and k once in, once out.  A row's 16-byte pieces lie over 4 to 32
// lanes, two to a lane, chosen so that a pair's halves are in one lane; a warp has
// one token and some of its rows, for which its lanes hold cosines and sines.
#pragma once

#include "cache_common.cuh"
#include "avits_internal.h"

namespace avits {
namespace rotate {

constexpr int kRotThreads = 128;
constexpr int kRotWarps = kRotThreads / 32;
constexpr int kDeep = 3;       // steps whose rows are under way at once

// What a lane reads and writes at once: E values, 16 bytes, or 8 or 4 where that is what
// halves are whole numbers of.
template <int kBytes>
struct Word;
template <>
struct Word<16> {
  using V = uint4;
  __device__ static V zero() { return make_uint4(0u, 0u, 0u, 0u); }
  __device__ static uint32_t at(const V& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
  __device__ static V of(const uint32_t (&w)[4]) { return make_uint4(w[0], w[1], w[2], w[3]); }
  // memory that this kernel may write again in place: no read-only path
  __device__ static V load(const void* p) {
    V v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p));
    return v;
  }
};
template <>
struct Word<8> {
  using V = uint2;
  __device__ static V zero() { return make_uint2(0u, 0u); }
  __device__ static uint32_t at(const V& v, int i) { return i == 0 ? v.x : v.y; }
  __device__ static V of(const uint32_t (&w)[2]) { return make_uint2(w[0], w[1]); }
  __device__ static V load(const void* p) {
    V v;
    asm volatile("ld.global.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
    return v;
  }
};
template <>
struct Word<4> {
  using V = uint32_t;
  __device__ static V zero() { return 0u; }
  __device__ static uint32_t at(const V& v, int) { return v; }
  __device__ static V of(const uint32_t (&w)[1]) { return w[0]; }
  __device__ static V load(const void* p) {
    V v;
    asm volatile("ld.global.L1::no_allocate.u32 %0, [%1];" : "=r"(v) : "l"(p));
    return v;
  }
};

template <typename T, int kBytes>
struct Piece {
  static constexpr int E = kBytes / (int)sizeof(T), kWords = kBytes / 4;
  using W = Word<kBytes>;
  using V = typename W::V;
  __device__ static void unpack(const V& v, float (&x)[E]) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      const uint32_t w = W::at(v, i);
      if constexpr (sizeof(T) == 2) {
        x[2 * i] = bf16_lo(w);
        x[2 * i + 1] = bf16_hi(w);
      } else {
        x[i] = __uint_as_float(w);
      }
    }
  }
  __device__ static V pack(const float (&x)[E]) {
    uint32_t w[kWords];
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      if constexpr (sizeof(T) == 2) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&v);
      } else {
        w[i] = __float_as_uint(x[i]);
      }
    }
    return W::of(w);
  }
};

// cos and sin of p f turns, times m.  bf16: the fast functions, off by 2^-21 in
// [-pi, pi] where the result is rounded by 2^-9 of itself.
template <typename T>
__device__ __forceinline__ void turn(uint64_t f, int p, float m, float& c, float& s) {
  const int hi = (int)(uint32_t)((f * (uint64_t)(int64_t)p) >> 32);
  const float x = (float)hi * 0x1p-31f;        // half turns
  if constexpr (sizeof(T) == 2) {
    __sincosf(x * 3.14159265358979f, &s, &c);
  } else {
    sincospif(x, &s, &c);
  }
  c *= m;
  s *= m;
}

// Two values to an instruction.
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 o;
  asm("{\n\t.reg .b64 a, b;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
      "mul.rn.f32x2 a, a, b;\n\tmov.b64 {%0, %1}, a;\n\t}"
      : "=f"(o.x), "=f"(o.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return o;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 o;
  asm("{\n\t.reg .b64 a, b, c;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
      "mov.b64 c, {%6, %7};\n\tfma.rn.f32x2 a, a, b, c;\n\tmov.b64 {%0, %1}, a;\n\t}"
      : "=f"(o.x), "=f"(o.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return o;
}

enum { kPairs = 0, kHalves = 1, kHalvesAny = 2 };

struct Rotate {
  RotateCall r;
  int parts;                       // warps of a token
  int q_steps, k_steps, steps;     // of a token: rows in groups of 32 / lanes; in all
  int pieces;                      // of a row
  int first[4];                    // first pair of each axis (axes past the last: none)
  float inv_d;
  FastDiv seq, part, page;         // tokens of a sequence, warps of a token, tokens of a page
  unsigned int* status;
};

// kLanes to a row, pieces of kBytes.
template <typename T, int kForm, bool kAppend, int kLanes, int kBytes>
__global__ void __launch_bounds__(kRotThreads)
norm_rotate_kernel(const __grid_constant__ Rotate a) {
  using Piece = Piece<T, kBytes>;
  using V = typename Piece::V;
  constexpr int E = Piece::E, kAngles = kForm == kHalvesAny ? 2 * E : E, kPer = 32 / kLanes;
  extern __shared__ float s_rows[];
  const RotateCall& r = a.r;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int unit = blockIdx.x * kRotWarps + warp;
  pdl_wait_then_trigger();
  const int t = a.part.div(unit), part = unit - t * a.parts;
  if (t >= r.tokens) return;
  const int b = kAppend ? 0 : a.seq.div(t), n = kAppend ? t : t - b * r.N;
  int64_t k_at = 0, v_at = 0;          // elements: where the token's keys and values go
  if (kAppend) {
    const int64_t slot = r.slots[t];
    if (slot < 0) return;              // padding
    const avits_kv_cache& c = r.cache;
    if (slot >= (int64_t)c.num_pages * c.page_size) {
      if (lane == 0 && part == 0) raise_status(a.status, AVITS_ERR_PAGE);
      return;
    }
    const int64_t page = slot >> 31 ? slot / c.page_size : a.page.div((int)slot);
    const int at = (int)(slot - page * c.page_size);
    k_at = page * c.k_sp + at * c.k_st;
    v_at = page * c.v_sp + at * c.v_st;
    if (c.acc && part == 0) {
      const int sb = r.seq[t], j = r.place[t];
      if ((unsigned)sb < (unsigned)c.B && (unsigned)j < (unsigned)c.max_len) {
        for (int h = lane; h < c.Hkv; h += 32)
          c.acc[(int64_t)sb * c.acc_sb + (int64_t)h * c.acc_sh + j] = 0.f;
      } else if (lane == 0) {
        raise_status(a.status, AVITS_ERR_PAGE);
      }
    }
  }
  // this lane's two pieces of a row
  const int sub = lane % kLanes, g = lane / kLanes, half = r.rot.rot / 2;
  int pa = sub, pb = sub + kLanes;
  if (kForm == kHalves) {
    const int turned = half / E, rest = (a.pieces - 2 * turned + 1) / 2;
    if (sub < turned) {
      pb = sub + turned;
    } else {
      pa = sub - turned < rest ? turned + sub : a.pieces;      // 2 turned + (sub - turned)
      pb = pa + rest;
    }
  }
  const bool ha = pa < a.pieces, hb = pb < a.pieces && ha;

  // The token's rows in steps of kPer: queries, then keys, then an append's values.  A warp
  // takes steps s0 .. s1-1 of them all.
  const int each = (a.steps + a.parts - 1) / a.parts;
  const int s0 = part * each, s1 = min(a.steps, s0 + each);
  if (s0 >= s1) return;
  // Step st: its rows are queries (0), keys (1) or values (2), this lane's is `row` of them.
  auto kind_of = [&](int st) {
    return st < a.q_steps ? 0 : !kAppend || st < a.q_steps + a.k_steps ? 1 : 2;
  };
  auto row_of = [&](int st, int kind) {
    return (st - (kind == 0 ? 0 : kind == 1 ? a.q_steps : a.q_steps + a.k_steps)) * kPer + g;
  };
  const T* q_in = static_cast<const T*>(r.q) + (int64_t)b * r.q_str[0] + (int64_t)n * r.q_str[1];
  const T* k_in = static_cast<const T*>(r.k) + (int64_t)b * r.k_str[0] + (int64_t)n * r.k_str[1];
  const T* v_in = kAppend ? static_cast<const T*>(r.v) + (int64_t)n * r.v_st : nullptr;
  T* q_out = static_cast<T*>(r.q_out) + (int64_t)b * r.qo_str[0] + (int64_t)n * r.qo_str[1];
  T* k_out = kAppend ? static_cast<T*>(r.cache.k_pages) + k_at
                     : static_cast<T*>(r.k_out) + (int64_t)b * r.ko_str[0] + (int64_t)n * r.ko_str[1];
  // A ring of kDeep steps' rows.  Lanes without a piece keep the zeros, lanes past the rows
  // what they had (it stays in their row's lanes).
  V va[kDeep], vb[kDeep];
#pragma unroll
  for (int k = 0; k < kDeep; ++k) va[k] = vb[k] = Piece::W::zero();
  auto load = [&](V& x, V& y, int st) {
    if (st >= s1) return;
    const int kind = kind_of(st), row = row_of(st, kind);
    if (row >= (kind == 0 ? r.H : r.Hkv)) return;
    const T* in = kind == 0   ? q_in + row * r.q_str[2]
                  : kind == 1 ? k_in + row * r.k_str[2]
                              : v_in + row * r.v_sh;
    if (ha) x = Piece::W::load(in + pa * E);
    if (hb) y = Piece::W::load(in + pb * E);
  };
  // the first rows are on their way while the angles are computed
#pragma unroll
  for (int k = 0; k < kDeep; ++k) load(va[k], vb[k], s0 + k);

  // The pair of angle e; each of the kPer groups of lanes, which hold the same pairs, computes
  // its share of the angles and hands it on.
  auto pair_of = [&](int e) {
    if (kForm == kHalves) return pa * E + e;
    if (kForm == kPairs) return e < E / 2 ? pa * (E / 2) + e : pb * (E / 2) + e - E / 2;
    const int x = e < E ? pa * E + e : pb * E + e - E;
    return x < half ? x : x < 2 * half ? x - half : half;
  };
  float cs[kAngles], sn[kAngles];
#pragma unroll
  for (int e = 0; e < kAngles; ++e) {
    cs[e] = 1.f;
    sn[e] = 0.f;
  }
  if (half > 0) {
    const int32_t* at = r.positions + (int64_t)b * r.pos_sb + (int64_t)n * r.pos_sn;
    int p[4] = {at[0], 0, 0, 0};
    if (r.rot.axes > 1)
      for (int x = 1; x < r.rot.axes; ++x) p[x] = at[x];
    constexpr int kShare = (kAngles + kPer - 1) / kPer;
    float c[kShare], s[kShare];
#pragma unroll
    for (int y = 0; y < kShare; ++y) {
      c[y] = 1.f;
      s[y] = 0.f;
      int i = half;
#pragma unroll
      for (int z = 0; z < kPer; ++z)
        if (y * kPer + z < kAngles && g == z) i = pair_of(y * kPer + z);
      if (i < half) {
        int x = p[0];
        if (r.rot.axes > 1)
          x = i >= a.first[3] ? p[3] : i >= a.first[2] ? p[2] : i >= a.first[1] ? p[1] : p[0];
        turn<T>(r.rot.freq[i], x, r.rot.magnitude, c[y], s[y]);
      }
    }
#pragma unroll
    for (int e = 0; e < kAngles; ++e) {
      const int from = sub + (e % kPer) * kLanes;
      cs[e] = kPer == 1 ? c[e / kPer] : __shfl_sync(0xffffffffu, c[e / kPer], from);
      sn[e] = kPer == 1 ? s[e / kPer] : __shfl_sync(0xffffffffu, s[e / kPer], from);
    }
  }
  const bool whole = 2 * half == r.d;

  float2 wa[E / 2], wb[E / 2];       // weights of the lane's pieces, of rows of kind `last`
  int last = -1;
  bool weighed = false;
#pragma unroll 1
  for (int st0 = s0; st0 < s1; st0 += kDeep) {
#pragma unroll
    for (int k = 0; k < kDeep; ++k) {
      const int st = st0 + k;
      if (st >= s1) break;
      const int kind = kind_of(st), row = row_of(st, kind);
      const bool live = row < (kind == 0 ? r.H : r.Hkv);
      T* out = kind == 0   ? q_out + row * r.qo_str[2]
               : kind == 1 ? k_out + row * (kAppend ? r.cache.k_sh : r.ko_str[2])
                           : static_cast<T*>(r.cache.v_pages) + v_at + row * r.cache.v_sh;
      if (kAppend && kind == 2) {          // a value: as it came
        if (live && ha) *reinterpret_cast<V*>(out + pa * E) = va[k];
        if (live && hb) *reinterpret_cast<V*>(out + pb * E) = vb[k];
        load(va[k], vb[k], st + kDeep);
        continue;
      }
      if (kind != last) {
        last = kind;
        const T* w = static_cast<const T*>(kind == 0 ? r.q_weight : r.k_weight);
        weighed = w != nullptr;
        if (weighed) {
          float x0[E], x1[E];
#pragma unroll
          for (int e = 0; e < E; ++e) x0[e] = x1[e] = 1.f;
          if (ha) Piece::unpack(__ldg(reinterpret_cast<const V*>(w + pa * E)), x0);
          if (hb) Piece::unpack(__ldg(reinterpret_cast<const V*>(w + pb * E)), x1);
#pragma unroll
          for (int e = 0; e < E / 2; ++e) {
            wa[e] = make_float2(x0[2 * e], x0[2 * e + 1]);
            wb[e] = make_float2(x1[2 * e], x1[2 * e + 1]);
          }
        }
      }
      {
        float fu[E], fv[E];
        Piece::unpack(va[k], fu);
        Piece::unpack(vb[k], fv);
        load(va[k], vb[k], st + kDeep);
        float2 u[E / 2], v[E / 2];
#pragma unroll
        for (int e = 0; e < E / 2; ++e) {
          u[e] = make_float2(fu[2 * e], fu[2 * e + 1]);
          v[e] = make_float2(fv[2 * e], fv[2 * e + 1]);
        }
        if (r.norm) {
          float2 q0 = mul2(u[0], u[0]), q1 = mul2(v[0], v[0]);
#pragma unroll
          for (int e = 1; e < E / 2; ++e) {
            q0 = fma2(u[e], u[e], q0);
            q1 = fma2(v[e], v[e], q1);
          }
          float sum = (q0.x + q0.y) + (q1.x + q1.y);
#pragma unroll
          for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
          const float f = rsqrtf(fmaf(sum, a.inv_d, r.eps));
          const float2 f2 = make_float2(f, f);
#pragma unroll
          for (int e = 0; e < E / 2; ++e) {
            u[e] = mul2(u[e], f2);
            v[e] = mul2(v[e], f2);
          }
          if (weighed) {
#pragma unroll
            for (int e = 0; e < E / 2; ++e) {
              u[e] = mul2(u[e], wa[e]);
              v[e] = mul2(v[e], wb[e]);
            }
          }
        }
        // in place of u and v; the rest of a head is no pair: an infinity in one of its values
        // leaves the others alone
        if (kForm == kHalves) {
          if (pa * E < half) {
#pragma unroll
            for (int e = 0; e < E / 2; ++e) {
              const float2 c = make_float2(cs[2 * e], cs[2 * e + 1]);
              const float2 s = make_float2(sn[2 * e], sn[2 * e + 1]);
              const float2 nv = make_float2(-v[e].x, -v[e].y);
              const float2 o = fma2(nv, s, mul2(u[e], c));
              v[e] = fma2(u[e], s, mul2(v[e], c));
              u[e] = o;
            }
          }
        } else if (kForm == kPairs) {
#pragma unroll
          for (int e = 0; e < E / 2; ++e) {
            if (whole || pair_of(e) < half)
              u[e] = make_float2(fmaf(-u[e].y, sn[e], u[e].x * cs[e]),
                                 fmaf(u[e].x, sn[e], u[e].y * cs[e]));
            if (whole || pair_of(E / 2 + e) < half)
              v[e] = make_float2(fmaf(-v[e].y, sn[E / 2 + e], v[e].x * cs[E / 2 + e]),
                                 fmaf(v[e].x, sn[E / 2 + e], v[e].y * cs[E / 2 + e]));
          }
        } else if (half > 0) {
          // the other value of a pair is in another lane
          float* mine = s_rows + (warp * kPer + g) * r.d;
          __syncwarp();
#pragma unroll
          for (int e = 0; e < E / 2; ++e) {
            if (ha) *reinterpret_cast<float2*>(mine + pa * E + 2 * e) = u[e];
            if (hb) *reinterpret_cast<float2*>(mine + pb * E + 2 * e) = v[e];
          }
          __syncwarp();
          auto other = [&](float y, bool there, int i, int e) {
            if (!there || i >= 2 * half) return y;
            const float o = mine[i < half ? i + half : i - half];
            return fmaf(i < half ? -o : o, sn[e], y * cs[e]);
          };
#pragma unroll
          for (int e = 0; e < E / 2; ++e) {
            u[e] = make_float2(other(u[e].x, ha, pa * E + 2 * e, 2 * e),
                               other(u[e].y, ha, pa * E + 2 * e + 1, 2 * e + 1));
            v[e] = make_float2(other(v[e].x, hb, pb * E + 2 * e, E + 2 * e),
                               other(v[e].y, hb, pb * E + 2 * e + 1, E + 2 * e + 1));
          }
        }
#pragma unroll
        for (int e = 0; e < E / 2; ++e) {
          fu[2 * e] = u[e].x;
          fu[2 * e + 1] = u[e].y;
          fv[2 * e] = v[e].x;
          fv[2 * e + 1] = v[e].y;
        }
        if (live && ha) *reinterpret_cast<V*>(out + pa * E) = Piece::pack(fu);
        if (live && hb) *reinterpret_cast<V*>(out + pb * E) = Piece::pack(fv);
      }
    }
  }
}

template <typename T, int kForm, bool kAppend, int kLanes, int kBytes = 16>
cudaError_t launch_lanes(const Rotate& a, int grid, cudaStream_t s) {
  constexpr auto kernel = norm_rotate_kernel<T, kForm, kAppend, kLanes, kBytes>;
  const cudaError_t e = prefer_max_shared<kernel>();
  if (e != cudaSuccess) return e;
  const size_t smem = kForm == kHalvesAny
                          ? (size_t)kRotWarps * (32 / kLanes) * a.r.d * sizeof(float) : 0;
  return launch_pdl(kernel, dim3((unsigned)grid), dim3(kRotThreads), smem, s, a);
}

// How a call's rows lie over lanes (launch_norm_rotate).
struct Cut {
  int form, bytes, lanes, grid;
};

template <typename T, int kForm, bool kAppend>
cudaError_t launch_form(const Rotate& a, const Cut& c, cudaStream_t s) {
  if constexpr (kForm == kHalves) {
    if (c.bytes == 8)
      return c.lanes <= 16 ? launch_lanes<T, kForm, kAppend, 16, 8>(a, c.grid, s)
                           : launch_lanes<T, kForm, kAppend, 32, 8>(a, c.grid, s);
    if constexpr (sizeof(T) == 2)
      if (c.bytes == 4)
        return c.lanes <= 16 ? launch_lanes<T, kForm, kAppend, 16, 4>(a, c.grid, s)
                             : launch_lanes<T, kForm, kAppend, 32, 4>(a, c.grid, s);
  }
  if (c.lanes <= 4) return launch_lanes<T, kForm, kAppend, 4>(a, c.grid, s);
  if (c.lanes <= 8) return launch_lanes<T, kForm, kAppend, 8>(a, c.grid, s);
  if (sizeof(T) == 2 || c.lanes <= 16) return launch_lanes<T, kForm, kAppend, 16>(a, c.grid, s);
  if constexpr (sizeof(T) == 4) return launch_lanes<T, kForm, kAppend, 32>(a, c.grid, s);
  return cudaErrorInvalidValue;
}

template <typename T>
cudaError_t launch_type(const Rotate& a, bool append, const Cut& c, cudaStream_t s) {
  if (append) {
    if (c.form == kPairs) return launch_form<T, kPairs, true>(a, c, s);
    if (c.form == kHalves) return launch_form<T, kHalves, true>(a, c, s);
    return launch_form<T, kHalvesAny, true>(a, c, s);
  }
  if (c.form == kPairs) return launch_form<T, kPairs, false>(a, c, s);
  if (c.form == kHalves) return launch_form<T, kHalves, false>(a, c, s);
  return launch_form<T, kHalvesAny, false>(a, c, s);
}

cudaError_t launch_f32(const Rotate& a, bool append, const Cut& c, cudaStream_t s);

}  // namespace rotate
}  // namespace avits
