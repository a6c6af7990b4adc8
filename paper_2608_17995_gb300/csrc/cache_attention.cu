// cache_attention.cu — attention of one new token per sequence over a paged
// key-value cache, with the weight each cached token got.
//
// For sequence b, KV head hk and the G query heads h that share it:
//   x_hj = scale q_h . k_j,  lse_h = log sum_j exp x_hj,  o_h = sum_j exp(x_hj - lse_h) v_j,
//   acc_j (+)= weight mean_h exp(x_hj - lse_h)
// A key or a value is 2 G operations to an element, so HBM bounds it where the heads of a
// KV head fit one unit (below), whose keys and values are read once.  Larger groups
// are several units, each of which copies the tiles again; L2 has part of them (28 x
// 1180-9904 in fp32, 16 heads in two units of 8: 220 MB from HBM for 155 MB of keys and
// values).
//
// The products are m16n8k16 of mma.sync, heads in the rows, 8 to 32 of them.  tcgen05
// has at least 64 rows: heads there would leave half of them and more empty, keys there
// and heads in the columns (8 and more) would fit, but P would pass through shared
// memory and O be rescaled in TMEM.  It was not tried: the tensor pipe does not bound
// these calls (15 % busy with 8 rows, 27 % with 32), and one warp's tiles need no other
// warp.
//
// Measured, against the time of the call's bytes at a copy's rate: 48 sequences of
// 409-4096 tokens, 32 heads over 8 of width 128, with weights 85 us (floor 68), without
// 77 (67); one of 131072, 32 over 4, 56 (40); 40 of up to 1500, 24 heads of width 64, 53
// (36); one of 517 tokens 5.5 (0.3).  These have max_len as the longest length.  The
// grids, the form and the logits' workspace go by max_len: with 32 times as much the
// first takes 130 us, the one of 517 tokens 7.8, and without weights there is no
// difference.
//
// Split.  A sequence's keys are cut into tiles; all tiles of all units (b, hk,
// row group) form one line, cut into equal pieces, one per CTA, so that uneven
// lengths and few heads load the SMs alike.  A CTA finds its piece by a scan of
// the lengths.  Its warps take the piece's tiles in turn, each with a running
// maximum, sum and O in registers and a ring of tiles of its own in shared
// memory, filled by TMA copies that run ahead over unit borders; the warps meet
// once per unit.  A unit that lies in one piece is finished there; of the others
// each piece leaves its maximum, sum and O, and a second kernel joins them, in the
// pieces' order.  The weights need the whole row's maximum and sum: the first kernel
// leaves the logits (fp32), the second sums exp(x - maximum) / sum over the group's
// heads, in a fixed order.
//
// Shorter sequences take one launch: a cluster of CTAs per unit, whose logits
// stay in shared memory.
#include "cache_tiles.cuh"

namespace avits {
namespace {

using namespace cache;

// How a call is cut: the widths 64, 128 and 256 have kernels of their own; a
// unit has 4 or 8 rows (fp32), or 8, 16 or 32 (bf16), by the group's size, so that
// a tile in shared memory serves all the heads that share it (256 columns: 16 at
// most, by registers).  In fp32 the CUDA cores multiply every row of a unit, so that
// 4 rows pay where the group has no more.
struct Shape {
  int G, D, rows, groups, tile, grid;
  int least;        // tiles of the smallest piece on the line
  int cluster;      // CTAs of a unit's cluster; 0: the line of tiles
  int warps;        // of a CTA of the cluster
  long long tiles;
};

constexpr int kClusterKeys = 512;       // of a CTA
constexpr int kClusterLogits = 8192;    // rows times keys of a CTA

// CTAs of a unit's cluster, 0 where the line of tiles is faster.  A cluster pays
// where the second launch would cost much beside the keys, and loses where units
// are too few to fill the SMs, or too many or too uneven to be resident at once.
// us, cluster and line (8 KV heads of width 128 with weights, if nothing is said):
//   1 x 517    6.1   8.4       1 x 4096, 4 KV heads  12.9  10.4
//   4 x 1024   7.6  12.6       16 x 2048             30.8  27.9
//   4 x 4096  16.9  21.2       48 x 1024             38.5  32.9, without 25.7  30.2
//   16 x 512   9.3  12.8       96 x 1000, without    63.9  70.1
//                              16 x 2000, width 256  33    28.2
// With weights a CTA has its keys' logits in shared memory, so that keys past 512
// would cost residency.
int cluster_of(const avits_kv_cache& c, const Shape& s, bool score, int num_sms) {
  if (score && s.groups > 1) return 0;      // a unit has not all the heads of a weight
  const int rows = s.G < s.rows ? s.G : s.rows;
  const long long units = (long long)c.B * c.Hkv * s.groups;
  auto fits = [&](int n) {
    const int64_t keys = ((int64_t)c.max_len + n - 1) / n;
    return keys <= (score || n > 1 ? kClusterKeys : 2 * kClusterKeys) &&
           (!score || keys * rows <= kClusterLogits);
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

// Warps of a unit's one CTA.  Where the units are more than two rounds of 4-warp
// CTAs, CTAs of 2 warps, of which twice as many share an SM, wait for their first
// copies beside more of each other: 1464 units of up to 271 keys 43.3 -> 32.6 us,
// 1368 of 119 25.0 -> 22.1 (768 of 100: 13.9 and 13.7).  With few tiles to a unit
// 1 warp: 1152 units of 8 keys 13.8 (4), 10.1 (2), 5.7; 1896 of 90 30.7, 24.5, 23.5,
// but 1368 of 119 29.7.  In fp32, whose O and Q are twice as wide, it never paid.
int warps_of(const avits_kv_cache& c, const Shape& s, int tiles, int num_sms) {
  const long long units = (long long)c.B * c.Hkv * s.groups;
  if (units <= 2ll * num_sms * cluster_ctas(s.D, s.rows, kWarps)) return kWarps;
  return c.dt == AVITS_BF16 && s.rows <= 16 && tiles <= 4 ? 1 : 2;
}

Shape shape_of(const avits_kv_cache& c, int H, bool score, int num_sms) {
  Shape s;
  const bool bf = c.dt == AVITS_BF16;
  s.G = H / c.Hkv;
  s.D = c.d <= 64 ? 64 : c.d <= 128 ? 128 : 256;
  s.rows = !bf ? (s.G <= 4 ? 4 : 8) : s.G <= 8 ? 8 : s.G <= 16 || s.D == 256 ? 16 : 32;
  s.groups = (s.G + s.rows - 1) / s.rows;
  s.tile = bf ? 16 : 8;
  s.tiles = (long long)c.B * c.Hkv * s.groups * ((c.max_len + s.tile - 1) / s.tile);
  // one tile for each warp, where a sequence has that many
  const int longest = (c.max_len + s.tile - 1) / s.tile;
  s.least = longest < kWarps ? longest : kWarps;
  const long long most = (s.tiles + s.least - 1) / s.least;
  long long full = (long long)num_sms * line_ctas(s.D, s.rows, bf);
  if (full > kMaxGrid) full = kMaxGrid;
  s.grid = (int)(most < full ? (most > 0 ? most : 1) : full);
  s.cluster = cluster_of(c, s, score, num_sms);
  s.warps = s.cluster == 1 ? warps_of(c, s, longest, num_sms) : kWarps;
  return s;
}

size_t up16(size_t n) { return (n + 15) / 16 * 16; }

struct Layout {
  size_t rec, own, norm, pml, po, logits, total;
  int64_t ld;
};

Layout layout_of(const avits_kv_cache& c, int H, const Shape& s, bool score) {
  Layout l;
  const size_t nrow = s.rows;
  l.ld = ((int64_t)c.max_len + 15) / 16 * 16;
  l.rec = 0;
  l.own = up16((size_t)c.B * c.Hkv * s.groups * 8);
  l.norm = l.own + up16((size_t)s.grid * 16);
  l.pml = l.norm + up16((size_t)c.B * H * 8);
  l.po = l.pml + up16((size_t)2 * s.grid * nrow * 8);
  l.logits = l.po + up16((size_t)2 * s.grid * nrow * c.d * 4);
  l.total = l.logits + (score ? (size_t)c.B * H * l.ld * 4 : 0);
  return l;
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
  a.least = sh.least;
  a.score = score;
  a.few = (long long)c.B * c.Hkv * sh.groups * kFewPieces > sh.grid;
  a.scale2 = call.scale * kLog2e;
  a.wmean = call.weight / (float)sh.G;
  a.add = call.weights == AVITS_WEIGHTS_ADD;
  a.rec = reinterpret_cast<int2*>(ws + l.rec);
  a.own = reinterpret_cast<int4*>(ws + l.own);
  a.norm = reinterpret_cast<float2*>(ws + l.norm);
  a.pml = reinterpret_cast<float2*>(ws + l.pml);
  a.po = reinterpret_cast<float*>(ws + l.po);
  a.logits = reinterpret_cast<float*>(ws + l.logits);
  a.ld = l.ld;
  a.status = status;
  return sh.cluster > 0 ? cache::launch_cluster(a, sh.D, sh.cluster, sh.warps, s)
                        : cache::launch_line(a, sh.D, num_sms, s);
}

}  // namespace avits
