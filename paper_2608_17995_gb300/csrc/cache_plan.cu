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
// The bytes are few (a step of 256 sequences 25 KB), so that latency is all: one CTA, a
// thread to a sequence, scans and moves pages; what is more than a few pages or rows of a
// sequence is shared out among the block's threads.  Where the rows are many, a second kernel over
// all SMs writes them.  A step of 256 sequences takes 5.0 us, 96 prompts with 108000 rows and 7000
// pages 8.9: the chain lengths, scan, list, scan, list, table.
#include "cache_common.cuh"
#include "avits_internal.h"

namespace avits {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kRowThreads = 128;
// Pages, and rows, of a sequence that a thread moves alone; more go to several threads.  us with
// up to 4, 8 and 16 rows alone: 128 sequences of 8 tokens 4.5, 5.5 and 5.5; 64 of 16 4.3, 4.3, 7.0.
constexpr int kOwnPages = 2;
constexpr int kOwnRows = 4;
// log2 of the fewest threads that share such a sequence's rows (4, 8 and 16 threads: 113 of 9
// tokens 5.1, 5.8 and 7.1 us; 60 of 17 5.0, 5.0, 5.9) and its pages (a warp; 96 prompts of 7000
// pages 8.9, with 4 threads 9.7).
constexpr int kRowBits = 2, kPageBits = 5;
// Rows that the first kernel's CTA writes itself: threads lie over sequences and rows evenly, so
// that the number of rows decides, however they lie in sequences.  us, so and by the second
// kernel: 256 sequences of 1, 2 and 4 tokens 3.6 and 6.4, 4.0 and 6.8, 4.8 and 6.8; 102 of 10 5.1
// and 6.0; 8 of 128 4.3 and 5.8; one of 512 4.0 and 5.6, of 1024 4.3 and 5.7; 255 of one beside one
// of 700 5.0 and 7.0.  Past the border both win somewhere: 150 of 10 6.6 and 6.0, 300 of 5 7.3 and
// 6.8, 200 of 10 6.7 and 6.1, 256 of 8 6.1 and 6.2, one of 2048 4.9 and 5.6, of 4096 6.2 and 5.7, 8
// of 900 9.1 and 6.0.
constexpr int kFewRows = 1024;

struct Plan {
  CachePlanCall p;
  FastDiv page;
  int rows_here;
  unsigned int* status;
};

__device__ __forceinline__ int pages_of(const Plan& a, int n) {
  return a.page.div(n + a.p.cache.page_size - 1);
}

// Sums of x and y over the threads before this one, and over all.  The caller has a barrier
// between two of these.
__device__ __forceinline__ longlong2 block_scan(longlong2 x, longlong2* s_warp, longlong2& total) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, warps = blockDim.x >> 5;
  longlong2 inc = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, inc.x, o), z = __shfl_up_sync(0xffffffffu, inc.y, o);
    if (lane >= o) {
      inc.x += y;
      inc.y += z;
    }
  }
  if (lane == 31) s_warp[w] = inc;
  __syncthreads();
  const longlong2 own = lane < warps ? s_warp[lane] : make_longlong2(0, 0);
  longlong2 run = own;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, run.x, o), z = __shfl_up_sync(0xffffffffu, run.y, o);
    if (lane >= o) {
      run.x += y;
      run.y += z;
    }
  }
  total = make_longlong2(__shfl_sync(0xffffffffu, run.x, 31), __shfl_sync(0xffffffffu, run.y, 31));
  return make_longlong2(__shfl_sync(0xffffffffu, run.x - own.x, w) + inc.x - x.x,
                        __shfl_sync(0xffffffffu, run.y - own.y, w) + inc.y - x.y);
}
static_assert(kPlanThreads == 32 * 32, "block_scan reads one sum per lane");

// Row t: token `place` of sequence b on page `page`; place < 0: padding.
__device__ __forceinline__ void put_row(const Plan& a, int t, int b, int place, int col, int page) {
  const CachePlanCall& p = a.p;
  int64_t slot = -1;
  if (place >= 0) {
    if ((unsigned)page < (unsigned)p.cache.num_pages)
      slot = (int64_t)page * p.cache.page_size + (place - col * p.cache.page_size);
    else
      raise_status(a.status, AVITS_ERR_PAGE);
  }
  p.slots[t] = slot;
  p.seq[t] = place >= 0 ? b : -1;
  p.place[t] = place;
  if (p.pos) p.pos[t] = place >= 0 ? place + (p.pos_base ? p.pos_base[b] : 0) : -1;
}
__device__ __forceinline__ void put_row(const Plan& a, int t, int b, int place) {
  const int col = place >= 0 ? a.page.div(place) : 0;
  const int page =
      place >= 0 ? a.p.cache.block_table[(int64_t)b * a.p.cache.table_sb + col] : -1;
  put_row(a, t, b, place, col, page);
}

// put(i, get(i)) for i < n by threads `at` of `all`, four reads on their way at once.
template <typename Get, typename Put>
__device__ __forceinline__ void by_four(int n, int at, int all, Get get, Put put) {
  for (int i0 = at; i0 < n; i0 += 4 * all) {
    int v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i0 + all * k < n) v[k] = get(i0 + all * k);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i0 + all * k < n) put(i0 + all * k, v[k]);
  }
}

// A sequence's part of the plan that several threads do.
struct Big {
  int b, col, n;             // pages: columns col .. col+n-1, ranks from `rank` on
  int row, rows, place;      // rows, from `row` on; the first one's place, -1: padding
  long long rank;
};

__global__ void __launch_bounds__(kPlanThreads)
cache_plan_kernel(const __grid_constant__ Plan a) {
  __shared__ longlong2 s_warp[2][32];
  __shared__ int s_taken, s_big;
  __shared__ Big s_list[kPlanThreads];
  const CachePlanCall& p = a.p;
  const avits_kv_cache& c = p.cache;
  int32_t* table = const_cast<int32_t*>(c.block_table);
  const int tid = threadIdx.x, lane = tid & 31, step = blockDim.x;
  if (tid == 0) s_taken = s_big = 0;
  pdl_wait_then_trigger();
  const int had = *p.free_count;
  const int count = min(max(had, 0), c.num_pages);
  if (tid == 0 && had != count) raise_status(a.status, AVITS_ERR_PAGE);

  struct Item {
    int n0, n1, rows, give;     // n1: wanted; give: pages given back
    bool ok;                    // a length in range, and one that fits the table
  };
  auto item = [&](int b) {
    Item x{0, 0, 0, 0, true};
    if (b >= c.B) return x;
    x.n0 = p.lens[b];
    const int ch = p.change[b];
    const int64_t n1 = (int64_t)x.n0 + ch;
    x.rows = max(ch, 0);
    x.ok = x.n0 >= 0 && x.n0 <= c.max_len && n1 <= c.max_len;
    x.n1 = x.ok ? (int)max(n1, (int64_t)0) : x.n0;
    x.give = x.ok && ch < 0 ? pages_of(a, x.n0) - pages_of(a, x.n1) : 0;
    return x;
  };
  // What the list holds, the block's threads shared out among its entries, a power of two of
  // them to each, 2^least or more: f(entry, thread of so many).  Between two barriers.
  auto over_list = [&](int least, auto f) {
    __syncthreads();
    const int n = s_big;
    const int bits = n > 0 ? max(least, __clz(n - 1) - 1 - __clz(step)) : least;
    for (int e = tid >> bits; e < n; e += step >> bits)
      f(s_list[e], tid & ((1 << bits) - 1), 1 << bits);
    __syncthreads();
    if (tid == 0) s_big = 0;
  };

  // Pages given back, `step` sequences at a time.
  Item x = item(tid);
  longlong2 at = make_longlong2(0, 0), sum;     // rows and pages given back before the chunk
  longlong2 mine = block_scan(make_longlong2(x.rows, x.give), s_warp[0], sum);
  for (int b0 = 0;;) {
    const long long rank = count + at.y + mine.y;
    const int b = b0 + tid, col = x.give > 0 ? pages_of(a, x.n1) : 0;
    const bool big = x.give > kOwnPages;
    if (big) s_list[atomicAdd(&s_big, 1)] = Big{b, col, x.give, 0, 0, 0, rank};
    for (int i = 0; !big && i < x.give; ++i)
      if (rank + i < c.num_pages) p.free_pages[rank + i] = table[(int64_t)b * c.table_sb + col + i];
    over_list(kPageBits, [&](const Big& y, int thread, int all) {
      const int32_t* from = table + (int64_t)y.b * c.table_sb + y.col;
      by_four(y.n, thread, all, [&](int i) { return from[i]; },
              [&](int i, int v) {
                if (y.rank + i < c.num_pages) p.free_pages[y.rank + i] = v;
              });
    });
    at.x += sum.x;
    at.y += sum.y;
    b0 += step;
    if (b0 >= c.B) break;
    x = item(b0 + tid);
    mine = block_scan(make_longlong2(x.rows, x.give), s_warp[0], sum);
  }
  const long long all_give = at.y, all_rows = at.x;
  if (tid == 0 && count + all_give > c.num_pages) raise_status(a.status, AVITS_ERR_PAGE);
  const int avail = (int)min(count + all_give, (long long)c.num_pages);

  // Pages taken, and rows.
  const bool once = c.B <= step;      // else the rows before a chunk's sequences are summed again
  longlong2 before = make_longlong2(0, 0);
  long long chunk_rows = 0;
  int taken = 0;
  for (int b0 = 0; b0 < c.B; b0 += step) {
    const int b = b0 + tid;
    if (!once) {
      x = item(b);
      __syncthreads();
      mine = block_scan(make_longlong2(x.rows, 0), s_warp[0], sum);
      chunk_rows = sum.x;
    }
    const long long row = before.x + mine.x;
    bool ok = x.ok && (x.rows == 0 || row + x.rows <= p.T);
    int col = 0, n = 0;
    // of the first row, if that page is there already
    const int col0 = x.rows > 0 && x.n0 >= 0 ? a.page.div(x.n0) : 0;
    int page = -1;
    if (ok && x.rows > 0) {
      col = pages_of(a, x.n0);
      n = pages_of(a, x.n1) - col;
      if (col0 < col) page = table[(int64_t)b * c.table_sb + col0];
    }
    const longlong2 need = block_scan(make_longlong2(n, 0), s_warp[1], sum);
    const long long rank = before.y + need.x;
    if (n > 0 && rank + n > avail) {
      ok = false;
      n = 0;
    }
    if (n > 0) taken = (int)(rank + n);
    const bool rows_in = x.rows > 0 && row < p.T;
    const int rows = rows_in ? (int)min((long long)x.rows, p.T - row) : 0;
    if (b < c.B) {
      if (!ok) raise_status(a.status, AVITS_ERR_PAGE);
      c.lens[b] = ok ? x.n1 : x.n0;
      p.cu_new[b + 1] = (int)min(row + x.rows, (long long)p.T);
    }
    const bool big = n > kOwnPages || (a.rows_here && rows > kOwnRows);
    if (big) {
      s_list[atomicAdd(&s_big, 1)] =
          Big{b, col, n, (int)row, rows, ok ? x.n0 : -1, rank};
    } else {
      int got[kOwnPages];
#pragma unroll
      for (int i = 0; i < kOwnPages; ++i) {
        got[i] = -1;
        if (i < n) {
          got[i] = p.free_pages[avail - 1 - (rank + i)];
          table[(int64_t)b * c.table_sb + col + i] = got[i];
        }
      }
      if (a.rows_here) {
        for (int i = 0; i < rows; ++i) {
          const int place = ok ? x.n0 + i : -1, at_col = ok ? a.page.div(place) : 0;
          int on = page;          // of column col0, the only one that was there before
#pragma unroll
          for (int k = 0; k < kOwnPages; ++k)
            if (k < n && at_col == col + k) on = got[k];
          put_row(a, (int)row + i, b, place, at_col, on);
        }
      } else if (rows > 0) {
        p.place[row] = ok ? x.n0 : -1;
      }
    }
    // rows read new pages from the free list, so that they wait for no other thread's table entries
    over_list(a.rows_here ? kRowBits : kPageBits, [&](const Big& y, int thread, int all) {
      int32_t* to = table + (int64_t)y.b * c.table_sb + y.col;
      const int32_t* from = p.free_pages + (avail - 1 - y.rank);
      by_four(y.n, thread, all, [&](int i) { return from[-(int64_t)i]; },
              [&](int i, int v) { to[i] = v; });
      if (a.rows_here) {
        auto page_of = [&](int i) {
          if (y.place < 0) return -1;
          const int k = a.page.div(y.place + i) - y.col;
          return k >= 0 ? from[-(int64_t)k] : to[k];
        };
        by_four(y.rows, thread, all, page_of, [&](int i, int v) {
          const int place = y.place >= 0 ? y.place + i : -1;
          put_row(a, y.row + i, y.b, place, place >= 0 ? a.page.div(place) : 0, v);
        });
      } else if (thread == 0 && y.rows > 0) {
        p.place[y.row] = y.place;
      }
    });
    before.x += chunk_rows;
    before.y += sum.x;
  }
  taken = __reduce_max_sync(0xffffffffu, taken);
  if (lane == 0) atomicMax(&s_taken, taken);
  __syncthreads();
  if (tid == 0) {
    *p.free_out = avail - s_taken;
    p.cu_new[0] = 0;
  }
  if (a.rows_here)
    for (long long t = min(all_rows, (long long)p.T) + tid; t < p.T; t += step) put_row(a, (int)t, 0, -1);
}

// Rows by many CTAs.  place[cu[b]], of a sequence's first row, is there already: -1 if it
// got no pages.
__global__ void __launch_bounds__(kRowThreads)
cache_plan_rows_kernel(const __grid_constant__ Plan a) {
  const CachePlanCall& p = a.p;
  const int32_t* cu = p.cu_new;
  const int t = blockIdx.x * kRowThreads + threadIdx.x, lane = threadIdx.x & 31, B = p.cache.B;
  pdl_wait_then_trigger();
  int b = sequence_of(cu, B, t - lane, lane);      // of the warp's first row
  if (t >= p.T) return;
  for (int i = 0; i < 4 && b < B && cu[b + 1] <= t; ++i) ++b;
  if (b < B && cu[b + 1] <= t) {
    int top = B;
    while (b < top) {
      const int mid = (b + top) >> 1;
      if (cu[mid + 1] <= t) b = mid + 1; else top = mid;
    }
  }
  const int head = b < B ? cu[b] : t, first = b < B ? p.place[head] : -1;
  if (b < B && t == head) {       // its place is there: other rows read it
    const int col = first >= 0 ? a.page.div(first) : 0;
    const int page = first >= 0 ? p.cache.block_table[(int64_t)b * p.cache.table_sb + col] : -1;
    put_row(a, t, b, first, col, page);
    return;
  }
  put_row(a, t, b, first >= 0 ? first + (t - head) : -1);
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
  int threads = 512;
  while (threads < call.cache.B && threads < kPlanThreads) threads *= 2;
  e = launch_pdl(cache_plan_kernel, dim3(1), dim3(threads), 0, s, a);
  if (e != cudaSuccess || a.rows_here) return e;
  e = prefer_max_shared<cache_plan_rows_kernel>();
  if (e != cudaSuccess) return e;
  return launch_pdl(cache_plan_rows_kernel, dim3((call.T + kRowThreads - 1) / kRowThreads),
                    dim3(kRowThreads), 0, s, a);
}

}  // namespace avits
