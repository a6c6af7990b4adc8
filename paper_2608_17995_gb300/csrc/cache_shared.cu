// cache_shared.cu — attention of one new token per sequence over a prefix that its group
// shares and its own cached tokens.
//
// For sequence b of group g and its query head h, over the keys j of both:
//   x_j = scale q . k_j,  lse = log sum_j exp x_j,  o = sum_j exp(x_j - lse) v_j
// The sum splits: each part of the keys leaves its maximum m, its sum l of
// exp(x - m) and its O = sum exp(x - m) v, and parts are joined by
//   M = max m,  o = sum_parts exp(m - M) O / sum_parts exp(m - M) l.
//
// A prefix is read for many sequences of its group at once: the query heads of all of them
// that share a KV head are the rows of one product.  Three kernels: parts of the prefixes,
// parts of the own tokens beside it, and the join.  How often a prefix is read (again mostly
// from L2):
//   bf16, widths to 128, pages of a multiple of 8 tokens   once per 128 or 256 rows
//   bf16, other pages or strides                           once per 8, 16 or 32 rows
//   bf16, wider                                            once per 8 or 16 rows
//   fp32                                                   once per 4 or 8 rows
//   both short, one launch over them                       once per sequence, per those rows
// 64 sequences of 4 query heads to each of 8 KV heads on 8192 + 512 tokens: width 128 37 us, width
// 256 172 (its bytes at a copy's rate 39), fp32 of width 128 411 (39); 12 groups of 8 on up to 3001 +
// 700 53, 133 (88), 198 (88).
//
// What bounds it: the prefixes' bytes and the own ones, while a group has up to about 128
// rows of a KV head; products and softmax in turn beyond (a tile of 64 keys by 128 rows is 8
// products of 64 columns for S, 48 clocks each, and 8 of 128 for the two parts of P, 64 each: 887
// clocks on the pipe of the 1115 that it takes; cache_prefix_tc.cu).  Of a call's time
// much is start and end: lengths, pages and the first tiles in turn 5 us, parts out and joined
// 6.  With 8 KV heads of 4 query heads, width 128, in us and (bytes at a copy's rate): 8
// sequences on 517 tokens 8.9 (0.7), 64 on 8192 with up to 512 of their own 37 (16), 12 groups
// of 8 on up to 3001 53 (36); 128 sequences of 4 x 8 heads on 32768 86 (36 of products).
#include <algorithm>

#include "cache_line.cuh"

namespace avits {
namespace {

using namespace cache;

constexpr int kJoinThreads = 128, kJoinHeads = 64;

size_t up16(size_t n) { return (n + 15) / 16 * 16; }

// One line of tiles: how it is cut and what it leaves.
struct Line {
  int rows, groups, D, tile, grid, least;
  int box;                     // prefixes on the tensor cores: tokens of a copy; else 0
  long long units, tiles;      // at most
  size_t rec, pml, po, base, end;
};

int width_of(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

// Pieces of a prefix on the tensor cores: short ones cost a start and a part each, and the SMs
// that get none go over own tokens meanwhile.  64 sequences on 8192 tokens took 42 us in
// 152 pieces of 7 tiles (of 256 rows), 37 in 103 of 10, 41 in 76; 160 in 4 groups on 2000 57 and
// 52.  Where a whole call has few tiles, they are cut finer.  Of 128 rows: 8 tiles where a unit
// has many pieces to join (11 sequences on 46000 24.7, of 4 tiles 28.8; 8 on 16000 27.0, of 5
// 28.3), else 5 (64 in 16 groups on up to 1000 23.7, of 8 29.8; 70 in 24 on 1282 22.0 and 27.3).
constexpr int kManyTiles = 160;      // of a unit
int piece_tiles(long long tiles, int longest, bool two, int num_sms) {
  const int most = two ? 10 : longest > kManyTiles ? 8 : 5;
  const long long share = tiles * 38 / (25ll * num_sms * (two ? 1 : 2));      // 100 and 200 on 152 SMs
  return (int)(share < 2 ? 2 : share > most ? most : share);
}
// Units of groups of prefixes with units of so many rows.
long long units_at_most(const avits_kv_cache& c, const avits_kv_cache& p, int G, int rows) {
  return c.Hkv * ((long long)c.B * G / rows + p.B);
}

void cut(Line& l, const avits_kv_cache& c, int num_sms) {
  const bool bf = c.dt == AVITS_BF16;
  l.D = width_of(c.d);
  l.tile = l.box ? kPrefixTile : bf ? 16 : 8;
  const int longest = (c.max_len + l.tile - 1) / l.tile;
  l.tiles = l.units * longest;
  const int few = l.box ? piece_tiles(l.tiles, longest, l.rows > kPrefixRows, num_sms) : kWarps;
  l.least = longest < few ? longest : few;
  const long long most = (l.tiles + l.least - 1) / l.least;
  const int ctas = l.box      ? 2 * kPrefixRows / l.rows
                   : l.groups ? own_ctas(l.D, l.rows, bf)      // groups: of own tokens
                              : line_ctas(l.D, l.rows, bf);
  long long full = (long long)num_sms * ctas;
  if (full > kMaxGrid) full = kMaxGrid;
  l.grid = (int)(most < full ? (most > 0 ? most : 1) : full);
}

// Rows of a unit for groups of n query heads that share a KV head.
int rows_of(bool bf, int D, long long n) {
  return !bf ? (n <= 4 ? 4 : 8) : n <= 8 ? 8 : n <= 16 || D == 256 ? 16 : 32;
}

// Rows of a unit on the tensor cores, for groups of n rows of a KV head.  Two row tiles to a CTA
// leave room on its SM for a CTA of own tokens, and SMs without a piece to more: taken where the
// tiles come in pairs, there are own tokens for the rest, and the prefix is one or the pieces fit
// the SMs at once.  It takes more own tokens where one prefix's pieces are few and run from one
// unit into the next (a second start and end in some CTAs), and for long prefixes at width 64,
// whose own tokens are half the bytes.  us, 128 and 256 rows, 8 KV heads of width 128, 64 sequences:
//   own       100          200          300          400          512          2000
//   on 1000                22.2  20.9   26.2  25.2   29.4  28.1   33.1  31.5
//      2000   23.8* 27.7*  25.5  29.3   28.7  30.6   32.0  32.1   36.3  33.4   79.0  73.8
//      4000                26.9  34.7   31.4  35.9   34.6  37.8   39.1  39.6
//      8192                33.9  36.0   38.4  36.9   42.7  37.6   47.2  40.8          (* own 50)
//     16000                41.5  42.4   45.7  46.2   49.7  49.6   54.3  54.6
// 63 tiles in pieces of 7, 4 KV heads of 512 rows on 4000 + 600 30.6 and 26.9.  128 sequences on 3000
// + 150 38.0 and 36.3, 5500 + 150 41.6 and 42.2, 8192 + 256 54.6 and 55.6, 16000 + 200 65.4 and 64.8; 4
// KV heads of 1024 rows on 32768 + 200 84.8 and 84.9, + 300 88.5 and 87.6.  Three prefixes 96 x (8000 +
// 300) 60.3 and 64.6.  Width 64: 128 x (12174 + 622) of 2 KV heads 30.0 and 33.7, 128 x (6618 + 640)
// of 4 27.4 and 23.3, 256 x (1389 + 149) of 4 24.6 and 23.6.  An odd tile: 324 rows on 30145 59.9 and
// 70.2, 1136 on 16837 123 and 132.  Of 230 drawn sizes the choice costs 0.6 % on average, more than 5
// on 8 of them and at most 11 (three uneven groups of width 64; 256 x (800 + 61)).
constexpr int kAtOnce = 10, kMuchOwn = 862, kMoreOwn = 1536;      // tiles, keys of KV heads: to an SM
constexpr int kShortTiles = 40;
int prefix_rows(const avits_kv_cache& c, const avits_kv_cache& p, int G, long long n, int num_sms) {
  const long long tiles = (n + kPrefixRows - 1) / kPrefixRows, pairs = (tiles + 1) / 2;
  if (tiles < 2 || 40 * pairs > 21 * tiles) return kPrefixRows;
  const int longest = (p.max_len + kPrefixTile - 1) / kPrefixTile;
  const long long all = pairs * c.Hkv * p.B * longest, own = (long long)c.B * c.Hkv * c.max_len;
  if (p.B > 1 && all > (long long)kAtOnce * num_sms) return kPrefixRows;
  long long much = kMuchOwn;
  if (p.B == 1) {
    const long long at_most = units_at_most(c, p, G, 2 * kPrefixRows) * longest;
    const int piece = piece_tiles(at_most, longest, true, num_sms);
    if (longest % piece != 0 && 5 * ((all + piece - 1) / piece) < 2ll * num_sms) much = kMoreOwn;
  }
  if (c.d <= 64 && longest > kShortTiles) much = std::max(much, 2ll * kMuchOwn);
  return own < much * num_sms ? kPrefixRows : 2 * kPrefixRows;
}

// CTAs of a unit's cluster that goes over prefix and own tokens in one launch, 0 where parts
// are faster: where the keys do not fit a cluster, where reading the prefix for every
// sequence costs more than two launches, or where the units are many.  us, one launch and
// parts, 8 KV heads of width 128 (prefix + own tokens):
//   4 x (900 + 700)   10.1  16.4    48 x (256 + 120)   13.1  15.7   (50 MB read again)
//   16 x (900 + 120)  14.8  17.7    48 x (512 + 120)   16.9  15.2   (100 MB)
//   16 x (512 + 700)  16.5  16.5    128 x (64 + 120)   25.6  21.8   (1024 units)
//   fp32, 16 x (512 + 120) 19.6 20.6, 16 x (900 + 120) 27.8 23.6    (67 and 118 MB)
constexpr long long kAgainBytes = 64ll << 20;
constexpr int kManyUnits = 4;      // to an SM

int both_of(const CacheSharedCall& s, const Line& own, int num_sms) {
  const long long units = own.units, keys = (long long)s.cache.max_len + s.prefix.max_len;
  // CTAs at once.  3 to an SM do not all find a place as clusters of 8: 448 of them took 15.3 us
  // where 224 in clusters of 4 took 10.8, but 384 7.7 and 192 8.2.
  const long long resident = own.D > 128   ? num_sms
                             : own.rows > 8 ? 2ll * num_sms
                                            : 8ll * num_sms / 3;
  auto fits = [&](int n) { return (keys + n - 1) / n <= (n > 1 ? 512 : 1024); };
  int n = 1;
  while (n < 8 && !fits(n)) n *= 2;
  if (!fits(n) || (n > 1 && units * n > resident) || units > (long long)kManyUnits * num_sms) return 0;
  const int es = s.cache.dt == AVITS_BF16 ? 2 : 4;
  if (units * s.prefix.max_len * 2 * s.cache.d * es > kAgainBytes) return 0;
  while (n < 8 && units * n * 2 <= resident && keys > n * 64) n *= 2;
  if (units * n < num_sms && keys > n * 256) return 0;
  return n;
}

// Own tokens: runs of 256 or 512 keys, a CTA each, up to kOwnLong or where the runs are few;
// else they lie on a line.  us, line and runs (the longer of the two kinds): 48 x (3000 + 1000) of
// 128 heads 62.5 and 61.5, 64 x (8192 + 512) 46 and 41, 48 x (8000 + 2000) 75.4 and 74.8; by the
// number of runs 40 (1 x (500 + 2500)) 16.6 and 13.5, 256 (1 x (8000 + 16000)) 35.5 and 32.1, 384
// (4 x (500 + 6000)) 28.3 and 20.8, 640 (16 x (500 + 2500)) 35.9 and 31.7, 944 (1 x (20000 +
// 60000)) 74.5 and 85, 1024 (4 x (8000 + 16000)) 54.3 and 57.2, 1536 (16 x (8000 + 6000)) 67.5 and
// 69.8.  Width 256: two warps to a CTA (88.8, with four 111.6).
constexpr int kOwnShort = 1024, kOwnLong = 2048;
constexpr int kFewRuns = 5;        // to an SM

struct Shape {
  Line own, pre;
  int both;         // CTAs of a cluster that goes over prefix and own tokens; 0: parts
  int warps;        // of a run's CTA where own tokens are short; 0: the line of tiles
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
  // rows of a group's KV head, by and large
  const long long rows = ((long long)c.B + p.B - 1) / p.B * G;
  x.pre.rows = x.pre.box ? prefix_rows(c, p, G, rows, num_sms) : rows_of(bf, D, rows);
  x.pre.units = units_at_most(c, p, G, x.pre.rows);
  cut(x.own, c, num_sms);
  cut(x.pre, p, num_sms);
  x.both = both_of(s, x.own, num_sms);
  // runs of a unit
  const int longest = (c.max_len + x.own.tile - 1) / x.own.tile, run = c.max_len <= kOwnShort ? 16 : 32;
  const int runs = (longest + run - 1) / run;
  if (c.max_len <= kOwnLong || x.own.units * runs <= (long long)kFewRuns * num_sms) {
    x.warps = D > 128 ? 2 : 4;
    x.own.least = run;
    x.own.grid = runs;
  }
  size_t at = 0;
  for (Line* l : {&x.own, &x.pre}) {
    const size_t parts =
        (size_t)(l == &x.own && x.warps ? l->units * l->grid : l->units + l->grid) * l->rows;
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

// Part k of a row: its maximum and sum, and columns 4 col .. of its O.
__device__ __forceinline__ void part_of(const CacheAttn& o, const CacheAttn& p, const Parts& x, int k,
                                        int col, float4& v, float2& ml) {
  const bool own = k < x.n_own;
  const int at = own ? x.own + k * x.own_step : x.pre + (k - x.n_own) * x.pre_step;
  v = reinterpret_cast<const float4*>(own ? o.po : p.po)[(int64_t)at * (o.c.d / 4) + col];
  ml = (own ? o.pml : p.pml)[at];
}

// Block (b, hk, some of its query heads): threads lie over the heads, their columns, and
// the parts, kDeep of which a thread has under way at once.
template <typename T>
__global__ void __launch_bounds__(kJoinThreads, 6)
cache_join_kernel(const __grid_constant__ CacheAttn o, const __grid_constant__ CacheAttn p,
                  int heads) {
  __shared__ float4 s_sum[kJoinThreads];
  __shared__ float2 s_ml[kJoinThreads];
  __shared__ Parts s_parts[kJoinHeads];
  const int tid = threadIdx.x;
  const int b = blockIdx.x / o.c.Hkv, hk = blockIdx.x - b * o.c.Hkv;
  const int g0 = blockIdx.y * heads, n = min(heads, o.G - g0);
  // what was there before this call: the group, lengths
  const int gq = g0 + tid, rg = gq / o.rows;
  int len = 0, lo = 0, len_p = 0;
  int2 m = make_int2(0, 0);
  if (tid < n) {
    len = cache_len(o.c, b);
    lo = group_of(p.start, p.c.B, b);
    m = members_of(p.start, p.seqs, lo);
    len_p = cache_len(p.c, lo);
  }
  pdl_wait_then_trigger();
  if (tid < n) {
    Parts x{0, 0, 0, 0, o.rows, p.rows};
    const int row = (b - m.x) * o.G + gq, rgp = row / p.rows;
    const int all = ((m.y - m.x) * o.G + p.rows - 1) / p.rows;
    const int2 own = o.rec[(b * o.c.Hkv + hk) * o.groups + rg];     // of an empty one: not used
    if (p.base[p.c.B] && b >= m.x && b < m.y && len_p > 0) {
      const int2 rec = p.rec[p.base[lo] + hk * all + rgp];
      x.pre = rec.x * p.rows + row - rgp * p.rows;
      x.n_pre = rec.y;
    }
    if (len > 0) {
      x.own = own.x * o.rows + gq - rg * o.rows;
      x.n_own = own.y;
    }
    s_parts[tid] = x;
  }
  __syncthreads();
  constexpr int kDeep = 8;
  const int d4 = o.c.d / 4, items = n * d4, lanes = kJoinThreads / items;
  const int sub = tid / items, it = tid - sub * items, r = it / d4, col = it - r * d4;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  float top = -INFINITY, l = 0.f;
  if (sub < lanes) {
    const Parts x = s_parts[r];
    for (int k0 = sub; k0 < x.count(); k0 += lanes * kDeep) {
      float4 y[kDeep];
      float2 ml[kDeep];
#pragma unroll
      for (int i = 0; i < kDeep; ++i) {
        const int k = k0 + i * lanes;
        y[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        ml[i] = make_float2(-INFINITY, 0.f);
        if (k < x.count()) part_of(o, p, x, k, col, y[i], ml[i]);
      }
      float mn = top;
#pragma unroll
      for (int i = 0; i < kDeep; ++i) mn = fmaxf(mn, ml[i].x);
      const float ref = mn == -INFINITY ? 0.f : mn, f0 = ex2(top - ref);
      l *= f0;
      v.x *= f0; v.y *= f0; v.z *= f0; v.w *= f0;
#pragma unroll
      for (int i = 0; i < kDeep; ++i) {
        const float f = ex2(ml[i].x - ref);      // from -inf: 0
        l = fmaf(f, ml[i].y, l);
        v.x = fmaf(f, y[i].x, v.x); v.y = fmaf(f, y[i].y, v.y);
        v.z = fmaf(f, y[i].z, v.z); v.w = fmaf(f, y[i].w, v.w);
      }
      top = mn;
    }
  }
  if (lanes > 1) {
    s_sum[tid] = v;
    s_ml[tid] = make_float2(top, l);
    __syncthreads();
    if (sub != 0) return;
    float mn = top;
    for (int k = 1; k < lanes; ++k) mn = fmaxf(mn, s_ml[k * items + it].x);
    const float ref = mn == -INFINITY ? 0.f : mn, f0 = ex2(top - ref);
    l *= f0;
    v.x *= f0; v.y *= f0; v.z *= f0; v.w *= f0;
    for (int k = 1; k < lanes; ++k) {
      const float2 ml = s_ml[k * items + it];
      const float4 y = s_sum[k * items + it];
      const float f = ex2(ml.x - ref);
      l = fmaf(f, ml.y, l);
      v.x = fmaf(f, y.x, v.x); v.y = fmaf(f, y.y, v.y);
      v.z = fmaf(f, y.z, v.z); v.w = fmaf(f, y.w, v.w);
    }
    top = mn;
  }
  if (sub != 0) return;
  const int h = hk * o.G + g0 + r;
  if (col == 0 && o.lse) o.lse[(int64_t)b * o.H + h] = lse2_of(top, l) * kLn2;
  const float inv = norm_of(top, l).y;
  T* out = static_cast<T*>(o.o) + (int64_t)b * o.o_sb + (int64_t)h * o.o_sh + col * 4;
  store_elem(out, 0, v.x * inv);
  store_elem(out, 1, v.y * inv);
  store_elem(out, 2, v.z * inv);
  store_elem(out, 3, v.w * inv);
}

template <typename T>
cudaError_t launch_join(const CacheAttn& o, const CacheAttn& p, cudaStream_t s) {
  // heads of a block: a thread for each four of their columns
  const int fit = kJoinThreads / (o.c.d / 4), most = fit < kJoinHeads ? fit : kJoinHeads;
  const int heads = o.G < most ? o.G : most;
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

bool cache_shared_sizes_ok(const CacheSharedCall& s, int num_sms) {
  const avits_kv_cache& c = s.cache;
  if (s.H / c.Hkv > kMaxGroup || (long long)c.B * s.H >= (1ll << 30)) return false;
  const Shape x = shape_of(s, num_sms);
  for (const Line* l : {&x.own, &x.pre}) {
    const long long parts = l == &x.own && x.warps ? l->units * l->grid : l->units + kMaxGrid;
    if (l->tiles >= (1ll << 30) || parts * l->rows >= (1ll << 31)) return false;
  }
  return (long long)c.B * c.Hkv < (1ll << 31) - 1;
}

size_t cache_shared_workspace(const CacheSharedCall& s, int num_sms) {
  return shape_of(s, num_sms).total;
}

cudaError_t launch_cache_shared(const CacheSharedCall& s, int num_sms, unsigned int* status,
                                cudaStream_t stream) {
  const Shape x = shape_of(s, num_sms);
  CacheAttn own = args_of(s, s.cache, x.own, status), pre = args_of(s, s.prefix, x.pre, status);
  if (x.both) return launch_both(own, pre, x.own.D, x.both, stream);
  cudaError_t e = x.pre.box ? launch_prefix_tc(pre, stream)
                            : launch_parts<kGroup>(pre, x.pre.D, stream);
  if (e == cudaSuccess)
    e = x.warps ? launch_own_parts(own, x.own.D, x.warps, stream)
                : launch_parts<kOwn>(own, x.own.D, stream);
  if (e != cudaSuccess) return e;
  return s.cache.dt == AVITS_BF16 ? launch_join<__nv_bfloat16>(own, pre, stream)
                                  : launch_join<float>(own, pre, stream);
}

}  // namespace avits
