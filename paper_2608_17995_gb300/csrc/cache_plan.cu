// cache_plan.cu — a step's changes of length become pages: taken from and given
// back to the list of free ones, with the block tables and a place for every new row.
//
// With n0 a sequence's length, c its change, n1 = max(n0 + c, 0), p(n) = ceil(n / page):
//   c < 0   columns p(n1) .. p(n0)-1 of its table go behind the free pages
//   c > 0   columns p(n0) .. p(n1)-1 come from the list's end; new row i of the
//           sequence, place j = n0 + i, has slot table[j / page] * page + j % page
// Ranks (which page, which row) are sums over the sequences before it: two scans,
// since the pages taken may be ones given back by a later sequence.
//
// The bytes are few (a step of 256 sequences 25 KB), so that latency is all: one CTA
// scans and moves pages, a second kernel over all SMs writes the rows where they are
// many.
#include "cache_common.cuh"
#include "avits_internal.h"

namespace avits {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWarps = kPlanThreads / 32;
constexpr int kRowThreads = 256;
constexpr int kOwnPages = 4;      // pages that a thread moves alone; more, and its warp does
constexpr int kFewRows = 4096;    // rows that the first kernel's CTA writes itself

struct Plan {
  CachePlanCall p;
  FastDiv page;
  int rows_here;
  unsigned int* status;
};

__device__ __forceinline__ int pages_of(const Plan& a, int n) {
  return a.page.div(n + a.p.cache.page_size - 1);
}

// Sums of x over the threads before this one, and over all; a barrier at each end.
__device__ __forceinline__ long long block_scan(long long x, long long* s_warp, int tid,
                                                long long& total) {
  const int lane = tid & 31, w = tid >> 5;
  long long inc = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += y;
  }
  __syncthreads();
  if (lane == 31) s_warp[w] = inc;
  __syncthreads();
  long long own = s_warp[lane], run = own;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, run, o);
    if (lane >= o) run += y;
  }
  total = __shfl_sync(0xffffffffu, run, 31);
  return __shfl_sync(0xffffffffu, run - own, w) + inc - x;
}
static_assert(kPlanWarps == 32, "block_scan reads one sum per lane");

// f(column, rank) for a sequence's columns col .. col+n-1, ranks from `rank` on: the
// first few by its thread, the others by the warp (all of it calls this).
template <typename F>
__device__ __forceinline__ void over_pages(int b, int col, int n, long long rank, int lane, F f) {
  const int own = min(n, kOwnPages);
  for (int i = 0; i < own; ++i) f(b, col + i, rank + i);
  unsigned more = __ballot_sync(0xffffffffu, n > own);
  while (more) {
    const int l = __ffs(more) - 1;
    more &= more - 1;
    const int bl = __shfl_sync(0xffffffffu, b, l), cl = __shfl_sync(0xffffffffu, col, l);
    const int nl = __shfl_sync(0xffffffffu, n, l);
    const long long rl = __shfl_sync(0xffffffffu, rank, l);
    for (int i = kOwnPages + lane; i < nl; i += 32) f(bl, cl + i, rl + i);
  }
}

// Row t of the step.  place[cu[b]], of a sequence's first row, is there already: -1 if
// it got no pages.
__device__ __forceinline__ void write_row(const Plan& a, const int32_t* cu, int t) {
  const CachePlanCall& p = a.p;
  int lo = 0, hi = p.cache.B;            // sequences whose rows end at t or before it
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (cu[mid + 1] <= t) lo = mid + 1; else hi = mid;
  }
  const int b = lo;
  int64_t slot = -1;
  int place = -1, pos = -1, seq = -1;
  const int head = b < p.cache.B ? cu[b] : 0;
  if (b < p.cache.B) place = p.place[head];
  if (place >= 0) {
    place += t - head;
    seq = b;
    pos = place + (p.pos_base ? p.pos_base[b] : 0);
    const int col = a.page.div(place);
    const int page = p.cache.block_table[(int64_t)b * p.cache.table_sb + col];
    if ((unsigned)page < (unsigned)p.cache.num_pages)
      slot = (int64_t)page * p.cache.page_size + (place - col * p.cache.page_size);
    else
      raise_status(a.status, AVITS_ERR_PAGE);
  }
  p.slots[t] = slot;
  p.seq[t] = seq;
  if (b >= p.cache.B || t != head) p.place[t] = place;
  if (p.pos) p.pos[t] = pos;
}

__global__ void __launch_bounds__(kPlanThreads)
cache_plan_kernel(const __grid_constant__ Plan a) {
  __shared__ long long s_warp[32];
  __shared__ int s_taken;
  const CachePlanCall& p = a.p;
  const avits_kv_cache& c = p.cache;
  int32_t* table = const_cast<int32_t*>(c.block_table);
  const int tid = threadIdx.x, lane = tid & 31;
  if (tid == 0) s_taken = 0;
  pdl_wait_then_trigger();
  const int each = (c.B + kPlanThreads - 1) / kPlanThreads;
  const int b0 = min(c.B, tid * each), mine = min(c.B, b0 + each) - b0;
  const int had = *p.free_count;
  const int count = min(max(had, 0), c.num_pages);
  if (tid == 0 && had != count) raise_status(a.status, AVITS_ERR_PAGE);

  struct Item {
    int n0, n1, rows, give;     // n1: wanted; give: pages given back
    bool ok;                    // a length in range, and one that fits the table
  };
  auto item = [&](int b) {
    Item x;
    x.n0 = p.lens[b];
    const int ch = p.change[b];
    const int64_t n1 = (int64_t)x.n0 + ch;
    x.rows = max(ch, 0);
    x.ok = x.n0 >= 0 && x.n0 <= c.max_len && n1 <= c.max_len;
    x.n1 = x.ok ? (int)max(n1, (int64_t)0) : x.n0;
    x.give = x.ok && ch < 0 ? pages_of(a, x.n0) - pages_of(a, x.n1) : 0;
    return x;
  };

  long long rows = 0, give = 0, all_rows, all_give;
  for (int i = 0; i < mine; ++i) {
    const Item x = item(b0 + i);
    rows += x.rows;
    give += x.give;
  }
  rows = block_scan(rows, s_warp, tid, all_rows);
  give = block_scan(give, s_warp, tid, all_give);
  if (tid == 0 && count + all_give > c.num_pages) raise_status(a.status, AVITS_ERR_PAGE);
  const int avail = (int)min(count + all_give, (long long)c.num_pages);

  // pages given back; what is needed, now that the rows before each sequence are known
  long long need = 0, all_need, row = rows;
  for (int i = 0; i < each; ++i) {
    Item x{};
    const int b = b0 + i;
    if (i < mine) {
      x = item(b);
      row += x.rows;
      if (x.ok && x.rows > 0 && row <= p.T) need += pages_of(a, x.n1) - pages_of(a, x.n0);
    }
    over_pages(b, x.give > 0 ? pages_of(a, x.n1) : 0, x.give, count + give, lane,
               [&](int bb, int col, long long at) {
                 if (at < c.num_pages) p.free_pages[at] = table[(int64_t)bb * c.table_sb + col];
               });
    give += x.give;
  }
  need = block_scan(need, s_warp, tid, all_need);      // its barriers: the list is complete

  int taken = 0;
  row = rows;
  for (int i = 0; i < each; ++i) {
    const int b = b0 + i;
    int n = 0, col = 0;
    long long rank = 0;
    if (i < mine) {
      const Item x = item(b);
      const long long before = row;
      row += x.rows;
      bool ok = x.ok && (x.rows == 0 || row <= p.T);
      if (ok && x.rows > 0) {
        col = pages_of(a, x.n0);
        n = pages_of(a, x.n1) - col;
        rank = need;
        need += n;
        if (n > 0 && need > avail) {
          ok = false;
          n = 0;
        }
        if (n > 0) taken = (int)need;
      }
      if (!ok) raise_status(a.status, AVITS_ERR_PAGE);
      c.lens[b] = ok ? x.n1 : x.n0;
      p.cu_new[b + 1] = (int)min(row, (long long)p.T);
      if (x.rows > 0 && before < p.T) p.place[before] = ok ? x.n0 : -1;
    }
    over_pages(b, col, n, rank, lane, [&](int bb, int cc, long long at) {
      table[(int64_t)bb * c.table_sb + cc] = p.free_pages[avail - 1 - at];
    });
  }
  taken = __reduce_max_sync(0xffffffffu, taken);
  if (lane == 0) atomicMax(&s_taken, taken);
  __syncthreads();
  if (tid == 0) {
    *p.free_out = avail - s_taken;
    p.cu_new[0] = 0;
  }
  if (!a.rows_here) return;
  __syncthreads();
  for (int t = tid; t < p.T; t += kPlanThreads) write_row(a, p.cu_new, t);
}

__global__ void __launch_bounds__(kRowThreads)
cache_plan_rows_kernel(const __grid_constant__ Plan a) {
  pdl_wait_then_trigger();
  const int t = blockIdx.x * kRowThreads + threadIdx.x;
  if (t < a.p.T) write_row(a, a.p.cu_new, t);
}

}  // namespace

cudaError_t launch_cache_plan(const CachePlanCall& call, unsigned int* status, cudaStream_t s) {
  Plan a{};
  a.p = call;
  a.page = FastDiv::of(call.cache.page_size);
  a.rows_here = call.T <= kFewRows;
  a.status = status;
  cudaError_t e = prefer_max_shared<cache_plan_kernel>();
  if (e != cudaSuccess) return e;
  e = launch_pdl(cache_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, a);
  if (e != cudaSuccess || a.rows_here) return e;
  e = prefer_max_shared<cache_plan_rows_kernel>();
  if (e != cudaSuccess) return e;
  return launch_pdl(cache_plan_rows_kernel, dim3((call.T + kRowThreads - 1) / kRowThreads),
                    dim3(kRowThreads), 0, s, a);
}

}  // namespace avits
