// rotate.cu — norm of each head and rotation by position, queries and keys in one
// pass; in a second form keys and values go straight to their places in a paged cache.
//
// For a head's vector x of d values at position p:
//   y = x / sqrt(mean x^2 + eps) * w                       (or y = x)
//   (y_a, y_b) of pair i -> m (y_a cos t - y_b sin t, y_b cos t + y_a sin t),
//   t = 2 pi p f_i, pairs (2i, 2i+1) or (i, i + rot/2), i < rot/2; the rest stays.
// All in fp32, rounded once.  Angles: f_i is a 64-bit binary fraction of a turn, so that
// p f_i mod 1 is the low 64 bits of an integer product, off by p 2^-65 turns; its top
// 32 bits become an fp32 angle in [-pi, pi).  No table of cosines is read, and far
// positions are as exact as near ones.
//
// Bytes bound it: q and k once in, once out.  A row's 16-byte pieces lie over 1 to 32
// lanes, two to a lane, chosen so that a pair's halves are in one lane; a warp has
// one token and some of its rows, for which its lanes hold cosines and sines.
#include "cache_common.cuh"
#include "avits_internal.h"

namespace avits {
namespace {

constexpr int kRotThreads = 128;
constexpr int kRotWarps = kRotThreads / 32;

template <typename T>
struct Piece;
template <>
struct Piece<__nv_bfloat16> {
  static constexpr int E = 8;
  __device__ static void unpack(const uint4& w, float (&x)[8]) {
    x[0] = bf16_lo(w.x); x[1] = bf16_hi(w.x); x[2] = bf16_lo(w.y); x[3] = bf16_hi(w.y);
    x[4] = bf16_lo(w.z); x[5] = bf16_hi(w.z); x[6] = bf16_lo(w.w); x[7] = bf16_hi(w.w);
  }
  __device__ static uint32_t two(float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
  }
  __device__ static uint4 pack(const float (&x)[8]) {
    return make_uint4(two(x[0], x[1]), two(x[2], x[3]), two(x[4], x[5]), two(x[6], x[7]));
  }
};
template <>
struct Piece<float> {
  static constexpr int E = 4;
  __device__ static void unpack(const uint4& w, float (&x)[4]) {
    x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y);
    x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
  }
  __device__ static uint4 pack(const float (&x)[4]) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]),
                      __float_as_uint(x[3]));
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

// 16 bytes that this kernel may write again in place: no read-only path.
__device__ __forceinline__ uint4 ld_piece(const void* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}

enum { kPairs = 0, kHalves = 1, kHalvesAny = 2 };

struct Rotate {
  RotateCall r;
  int lanes;         // of a row: 1 .. 32
  int steps;         // of a token: rows in groups of 32 / lanes
  int parts;         // warps of a token
  int pieces;        // of a row
  int first[4];      // first pair of each axis (axes past the last: none)
  FastDiv seq, part, page;     // tokens of a sequence, warps of a token, tokens of a page
  unsigned int* status;
};

template <typename T, int kForm, bool kAppend>
__global__ void __launch_bounds__(kRotThreads)
norm_rotate_kernel(const __grid_constant__ Rotate a) {
  constexpr int E = Piece<T>::E, kAngles = kForm == kHalvesAny ? 2 * E : E;
  extern __shared__ float s_rows[];
  const RotateCall& r = a.r;
  const int w = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int unit = blockIdx.x * kRotWarps + w;
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
  const int sub = lane & (a.lanes - 1), half = r.rot.rot / 2;
  int pa, pb;
  if (kForm == kHalves) {
    const int turned = half / E;
    pa = sub < turned ? sub : turned + sub;            // 2 turned + (sub - turned)
    pb = sub < turned ? sub + turned : pa + (a.pieces - 2 * turned + 1) / 2;
    if (sub >= turned && sub - turned >= (a.pieces - 2 * turned + 1) / 2) pa = a.pieces;
  } else {
    pa = sub;
    pb = sub + a.lanes;
  }
  const bool ha = pa < a.pieces, hb = pb < a.pieces && ha;
  // the pair of angle e
  auto pair_of = [&](int e) {
    if (kForm == kHalves) return pa * E + e;
    if (kForm == kPairs) return e < E / 2 ? pa * (E / 2) + e : pb * (E / 2) + e - E / 2;
    const int x = e < E ? pa * E + e : pb * E + e - E;
    return x < half ? x : x - half;
  };
  float cs[kAngles], sn[kAngles];
  {
    int p[4] = {0, 0, 0, 0};
    if (half > 0) {
      const int32_t* at = r.positions + (int64_t)b * r.pos_sb + (int64_t)n * r.pos_sn;
      for (int x = 0; x < r.rot.axes; ++x) p[x] = at[x];
    }
#pragma unroll
    for (int e = 0; e < kAngles; ++e) {
      const int i = pair_of(e);
      cs[e] = 1.f;
      sn[e] = 0.f;
      const bool mine = kForm == kHalvesAny ? (e < E ? pa * E + e : pb * E + e - E) < 2 * half
                        : kForm == kPairs ? (e < E / 2 ? ha : hb) && i < half
                                          : i < half;
      if (mine) {
        const int x = i >= a.first[3] ? p[3] : i >= a.first[2] ? p[2] : i >= a.first[1] ? p[1] : p[0];
        turn<T>(r.rot.freq[i], x, r.rot.magnitude, cs[e], sn[e]);
      }
    }
  }
  // A row of this lane: what it reads, writes and is multiplied by.
  const int per = 32 / a.lanes, heads = r.H + r.Hkv, rows = heads + (kAppend ? r.Hkv : 0);
  const int g = lane / a.lanes;
  struct Row {
    const T* in;
    T* out;
    const T* w;
    bool turned;
  };
  auto row_of = [&](int i) {
    Row x{nullptr, nullptr, nullptr, true};
    if (i < r.H) {
      x.in = static_cast<const T*>(r.q) + (int64_t)b * r.q_str[0] + (int64_t)n * r.q_str[1] +
             (int64_t)i * r.q_str[2];
      x.out = static_cast<T*>(r.q_out) + (int64_t)b * r.qo_str[0] + (int64_t)n * r.qo_str[1] +
              (int64_t)i * r.qo_str[2];
      x.w = static_cast<const T*>(r.q_weight);
    } else if (i < heads) {
      const int h = i - r.H;
      x.in = static_cast<const T*>(r.k) + (int64_t)b * r.k_str[0] + (int64_t)n * r.k_str[1] +
             (int64_t)h * r.k_str[2];
      x.out = kAppend ? static_cast<T*>(r.cache.k_pages) + k_at + (int64_t)h * r.cache.k_sh
                      : static_cast<T*>(r.k_out) + (int64_t)b * r.ko_str[0] +
                            (int64_t)n * r.ko_str[1] + (int64_t)h * r.ko_str[2];
      x.w = static_cast<const T*>(r.k_weight);
    } else if (i < rows) {
      const int h = i - heads;
      x.in = static_cast<const T*>(r.v) + (int64_t)n * r.v_st + (int64_t)h * r.v_sh;
      x.out = static_cast<T*>(r.cache.v_pages) + v_at + (int64_t)h * r.cache.v_sh;
      x.turned = false;
    }
    return x;
  };
  const int each = (a.steps + a.parts - 1) / a.parts;
  const int s0 = part * each, s1 = min(a.steps, s0 + each);
  const uint4 none = make_uint4(0u, 0u, 0u, 0u);
  Row row = row_of(s0 * per + g);
  uint4 va = none, vb = none;
  if (s0 < s1 && row.in) {
    if (ha) va = ld_piece(row.in + pa * E);
    if (hb) vb = ld_piece(row.in + pb * E);
  }
  for (int st = s0; st < s1; ++st) {
    const Row cur = row;
    const uint4 ca = va, cb = vb;
    row = Row{nullptr, nullptr, nullptr, true};
    if (st + 1 < s1) {
      row = row_of((st + 1) * per + g);
      if (row.in) {
        if (ha) va = ld_piece(row.in + pa * E);
        if (hb) vb = ld_piece(row.in + pb * E);
      }
    }
    float x[E], y[E];
    Piece<T>::unpack(ca, x);
    Piece<T>::unpack(cb, y);
    if (r.norm) {
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if (ha) sum = fmaf(x[e], x[e], sum);
        if (hb) sum = fmaf(y[e], y[e], sum);
      }
      for (int o = a.lanes >> 1; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      const float f = rsqrtf(sum / (float)r.d + r.eps);
      float wa[E], wb[E];
#pragma unroll
      for (int e = 0; e < E; ++e) wa[e] = wb[e] = 1.f;
      if (cur.w) {
        if (ha) Piece<T>::unpack(__ldg(reinterpret_cast<const uint4*>(cur.w + pa * E)), wa);
        if (hb) Piece<T>::unpack(__ldg(reinterpret_cast<const uint4*>(cur.w + pb * E)), wb);
      }
#pragma unroll
      for (int e = 0; e < E; ++e) {
        x[e] = x[e] * f * wa[e];
        y[e] = y[e] * f * wb[e];
      }
    }
    float ox[E], oy[E];
    if (kForm == kHalves) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        // the rest of a head is no pair: an infinity in one value leaves the other alone
        const bool turns = pa * E < half;
        ox[e] = turns ? x[e] * cs[e] - y[e] * sn[e] : x[e];
        oy[e] = turns ? y[e] * cs[e] + x[e] * sn[e] : y[e];
      }
    } else if (kForm == kPairs) {
#pragma unroll
      for (int e = 0; e < E / 2; ++e) {
        const bool ta = pair_of(e) < half, tb = pair_of(E / 2 + e) < half;
        const float x0 = x[2 * e], x1 = x[2 * e + 1], y0 = y[2 * e], y1 = y[2 * e + 1];
        ox[2 * e] = ta ? x0 * cs[e] - x1 * sn[e] : x0;
        ox[2 * e + 1] = ta ? x1 * cs[e] + x0 * sn[e] : x1;
        oy[2 * e] = tb ? y0 * cs[E / 2 + e] - y1 * sn[E / 2 + e] : y0;
        oy[2 * e + 1] = tb ? y1 * cs[E / 2 + e] + y0 * sn[E / 2 + e] : y1;
      }
    } else {
      // the other value of a pair is in another lane
      float* mine = s_rows + (w * per + g) * r.d;
      __syncwarp();
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if (ha) mine[pa * E + e] = x[e];
        if (hb) mine[pb * E + e] = y[e];
      }
      __syncwarp();
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int i = pa * E + e, j = pb * E + e;
        const float xo = ha && i < 2 * half ? mine[i < half ? i + half : i - half] : 0.f;
        const float yo = hb && j < 2 * half ? mine[j < half ? j + half : j - half] : 0.f;
        ox[e] = x[e] * cs[e] + (i < half ? -xo : xo) * sn[e];
        oy[e] = y[e] * cs[E + e] + (j < half ? -yo : yo) * sn[E + e];
      }
    }
    if (cur.in) {
      const bool keep = kAppend && !cur.turned;        // a value: as it came
      if (ha) *reinterpret_cast<uint4*>(cur.out + pa * E) = keep ? ca : Piece<T>::pack(ox);
      if (hb) *reinterpret_cast<uint4*>(cur.out + pb * E) = keep ? cb : Piece<T>::pack(oy);
    }
  }
}

template <typename T, int kForm, bool kAppend>
cudaError_t launch_form(const Rotate& a, int grid, cudaStream_t s) {
  constexpr auto kernel = norm_rotate_kernel<T, kForm, kAppend>;
  const cudaError_t e = prefer_max_shared<kernel>();
  if (e != cudaSuccess) return e;
  const size_t smem = kForm == kHalvesAny
                          ? (size_t)kRotWarps * (32 / a.lanes) * a.r.d * sizeof(float) : 0;
  return launch_pdl(kernel, dim3((unsigned)grid), dim3(kRotThreads), smem, s, a);
}

template <typename T>
cudaError_t launch_type(const Rotate& a, int form, bool append, int grid, cudaStream_t s) {
  if (append) {
    if (form == kPairs) return launch_form<T, kPairs, true>(a, grid, s);
    if (form == kHalves) return launch_form<T, kHalves, true>(a, grid, s);
    return launch_form<T, kHalvesAny, true>(a, grid, s);
  }
  if (form == kPairs) return launch_form<T, kPairs, false>(a, grid, s);
  if (form == kHalves) return launch_form<T, kHalves, false>(a, grid, s);
  return launch_form<T, kHalvesAny, false>(a, grid, s);
}

}  // namespace

cudaError_t launch_norm_rotate(const RotateCall& call, bool append, int num_sms,
                               unsigned int* status, cudaStream_t s) {
  Rotate a{};
  a.r = call;
  const int E = call.dt == AVITS_BF16 ? 8 : 4;
  a.pieces = call.d / E;
  const int half = call.rot.rot / 2;
  const int form = call.rot.interleaved ? kPairs : half % E == 0 ? kHalves : kHalvesAny;
  // lanes of a row: two pieces each; halves that turn and a rest are paired apart
  const int need = form == kHalves ? half / E + (a.pieces - 2 * (half / E) + 1) / 2
                                   : (a.pieces + 1) / 2;
  a.lanes = 1;
  while (a.lanes < need) a.lanes *= 2;
  const int per = 32 / a.lanes, rows = call.H + call.Hkv * (append ? 2 : 1);
  a.steps = (rows + per - 1) / per;
  // a warp for each token, or several where tokens are too few to fill the SMs
  a.parts = 1;
  while (a.parts < a.steps && (long long)call.tokens * a.parts < 16ll * num_sms) a.parts *= 2;
  if (a.parts > a.steps) a.parts = a.steps;
  a.first[0] = 0;
  for (int x = 1; x < 4; ++x)
    a.first[x] = x < call.rot.axes ? a.first[x - 1] + call.rot.sections[x - 1] : 1 << 30;
  a.seq = FastDiv::of(call.N);
  a.part = FastDiv::of(a.parts);
  a.page = FastDiv::of(append ? call.cache.page_size : 1);
  a.status = status;
  const long long units = (long long)call.tokens * a.parts;
  const int grid = (int)((units + kRotWarps - 1) / kRotWarps);
  return call.dt == AVITS_BF16 ? launch_type<__nv_bfloat16>(a, form, append, grid, s)
                               : launch_type<float>(a, form, append, grid, s);
}

}  // namespace avits
