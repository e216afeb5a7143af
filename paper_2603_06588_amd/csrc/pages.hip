// Pages of the paged cache shared between sequences: fork (share, reorder, cut back, free), append (allocate, copy shared
// last pages) and compact (move live pages to the front).  Everything is decided on the device from the tables and
// the reference counts; the host sees none of them, so each call is a fixed sequence of launches.
//
// Bookkeeping is bound by launches and by trips to memory, the data by its bandwidth: a copied page is read once and
// written once, by workgroups that take one piece of one page in one cache at a time.
// Which page is the k-th free (or live) one is a sum over all pages.  It is taken in two launches: the first lists the free pages of every
// chunk of kChunk pages and counts them; every workgroup of the second adds the chunks' counts up for itself and then looks a page up
// by its number.  (With a launch in between that hands the pages out the step after a fork of 512 rows took 34 us instead of 24.)
#include "../../include/hook_api.h"
#include "hook_device.h"

#include <algorithm>

namespace hook {
namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 2048;          // pages of a workgroup, eight to a thread
constexpr int kPer = kChunk / kThreads;
constexpr int kRowChunk = 1024;       // table entries of a workgroup, one to a thread in fork and four in compact
constexpr int kTooMany = 0x3fffffff;  // "needs" of a row that the table cannot hold: more than any cache has

struct RowPlan {
  int start;   // first table entry that gets a new page
  int tail;    // page to be copied into the first of them, or -1
  int len;     // tokens that the row holds before the call
  int grow;    // tokens that it is to hold more
};

struct PagesParams {
  int S, mb, nb, rows;
  const int *table, *lens, *refs;
  int *table_out, *lens_out, *refs_out, *status;
  const int *src, *keep, *cu;
  int *page_map, *num_live;
  // scratch
  int nc;            // chunks
  int* counts;       // [nc] free pages of a chunk
  int* free_list;    // [nc, kChunk] the free pages of each chunk
  int* live_list;    // [nc, kChunk] the live ones (compact)
  int* order;        // [nb] a live page's number among those of its chunk, or -1 - a free one's (compact)
  int* need;         // [S] new pages of a row (append)
  RowPlan* plan;     // [S] (append)
  // data
  int ncaches, heads;
  int row_chunks;    // 16-byte pieces of a token row of one head
  int keep_lines;    // the caches fit the last-level cache (compact)
};

// The caches travel as an argument of their own, of two lengths: a launch with 2 KB of arguments costs the host more than one with 256 bytes
// (append of 64 rows in 8 caches 11.6 us a call with the long list, 11.2 with the short one).
constexpr int kFewCaches = 32;
template <int N> struct CacheList {
  void* cache[N];
};

// Sum over the workgroup, in every thread; `sh` holds one value per wave.
__device__ __forceinline__ long long block_sum(long long x, long long* sh) {
#pragma unroll
  for (int m = 32; m > 0; m >>= 1) x += __shfl_xor(x, m, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = x;
  __syncthreads();
  x = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) x += sh[w];
  return x;
}

// Sum of x over the threads before this one; the whole sum in *all.
__device__ __forceinline__ int block_scan(int x, int* sh, int* all) {
  const int in = wave_scan(x), wave = threadIdx.x >> 6;
  __syncthreads();
  if ((threadIdx.x & 63) == 63) sh[wave] = in;
  __syncthreads();
  int before = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    if (w < wave) before += sh[w];
    sum += sh[w];
  }
  *all = sum;
  return before + in - x;
}

__device__ __forceinline__ void report(const PagesParams& p, int bits) {
  if (bits) atomicOr(p.status, bits);
}

__device__ __forceinline__ int pages_of(int len) { return (int)(((long long)len + kBlock - 1) / kBlock); }

// A length as it counts: inside [0, what a table row holds].
__device__ __forceinline__ int length_of(int len, int mb, int* bits) {
  const long long most = (long long)mb * kBlock;
  if (len < 0) { *bits |= HOOK_PAGES_BAD_LENGTH; return 0; }
  if (len > most) { *bits |= HOOK_PAGES_BAD_LENGTH; return (int)most; }
  return len;
}

// ---- fork -----------------------------------------------------------------------------------------------

__global__ __launch_bounds__(kThreads) void k_pages_copy_counts(const int* from, int* to, int n) {
  const int i = blockIdx.x * kThreads + threadIdx.x;
  if (i < n) to[i] = from[i];
}

// Row of the old table that new row r comes from (-1: none) and the tokens that it takes over.
__device__ __forceinline__ int2 origin_of(const PagesParams& p, int r, int* bits) {
  const int from = p.src[r];
  int len = 0;
  if (from >= 0 && from < p.S) {
    len = length_of(p.lens[from], p.mb, bits);
    if (p.keep) len = min(len, max(p.keep[r], 0));
  } else if (from != -1) {
    *bits |= HOOK_PAGES_BAD_ROW;
  }
  return make_int2(from, len);
}

constexpr int kForkThreads = 1024;
constexpr int kCols = 8;
constexpr int kLanes = kForkThreads / kCols;      // rows at a time
constexpr int kBatch = 4096;                      // rows whose origin and length are fetched together
constexpr int kSlots = 2048, kProbes = 8;
constexpr int kCounters = 512;                    // workgroups that count, two for each compute unit; they take turns over longer rows

// Two kinds of workgroups.  The last ones copy kRowChunk entries of a new row from the row it comes from.  Each of the first
// takes kCols columns of both tables and counts the entries of the new rows up and those of the old rows down.  Pages
// that rows share lie in the same column of each of them, so the changes are summed up in shared memory first (open addressing; a page
// that finds no place goes to memory at once), and what is left of them goes to the counts by one atomic per page.  64 rows of 4000-32000
// tokens shared out to 512 and back: 16.6 us, with an atomic per entry 27.7; 16 columns at 512 threads 38.7, 4 17.1.
template <bool TURNS>      // tables of more columns than the workgroups of one turn take
__global__ __launch_bounds__(kForkThreads) void k_pages_fork(const PagesParams p, int chunks) {
  const int tid = threadIdx.x;
  int bits = 0;
  const int counters = min((p.mb + kCols - 1) / kCols, kCounters);
  if ((int)blockIdx.x >= counters) {
    const int b = blockIdx.x - counters, row = b / chunks, e0 = (b - row * chunks) * kRowChunk;
    const int2 o = origin_of(p, row, &bits);
    if (e0 == 0 && tid == 0) p.lens_out[row] = o.y;
    const int held = pages_of(o.y);
#pragma unroll
    for (int u = 0; u < kRowChunk / kForkThreads; ++u) {
      const int e = e0 + u * kForkThreads + tid;
      if (e >= held) continue;
      const int page = p.table[(size_t)o.x * p.mb + e];
      if ((unsigned)page >= (unsigned)p.nb) bits |= HOOK_PAGES_BAD_PAGE;
      p.table_out[(size_t)row * p.mb + e] = page;
    }
    report(p, bits);
    return;
  }
  __shared__ int key[kSlots], change[kSlots];
  __shared__ int2 origin[kBatch];      // row of the old table, held pages
  __shared__ int heir[kBatch];
  __shared__ int longest;
  const int lane = tid / kCols, total = p.rows + p.S;
  auto held_by = [&](int r) {
    const int2 o = r < p.rows ? origin_of(p, r, &bits) : make_int2(r - p.rows, length_of(p.lens[r - p.rows], p.mb, &bits));
    return make_int2(o.x, pages_of(o.y));
  };
  if (tid == 0) longest = 0;
  for (int i = tid; i < kSlots; i += kForkThreads) { key[i] = -1; change[i] = 0; }
  __syncthreads();
  int most = 0;
  for (int r = tid; r < total; r += kForkThreads) {
    const int2 o = held_by(r);
    if (r < kBatch) { origin[r] = o; heir[r] = p.rows; }
    if (TURNS) most = max(most, o.y);
  }
  if (TURNS) {
    most = wave_max(most);
    if ((tid & 63) == 0) atomicMax(&longest, most);
  }
  __syncthreads();
  const int columns = TURNS ? longest : p.mb;
  // A row that a new one takes over with all its pages is counted neither down nor up for that one.  (512 rows of 4000 tokens in another
  // order 12.5 -> 4.6 us, 2000 rows of 600, more pages than slots, 60 -> 6.9.)
  if (total <= kBatch) {
    for (int r = tid; r < p.rows; r += kForkThreads)
      if (origin[r].y > 0 && origin[r].y == origin[p.rows + origin[r].x].y) atomicMin(&heir[origin[r].x], r);
    __syncthreads();
    for (int i = tid; i < p.S; i += kForkThreads)
      if (heir[i] < p.rows) origin[heir[i]].y = origin[p.rows + i].y = 0;
    __syncthreads();
  }
  auto count = [&](int page, int by) {
    if ((unsigned)page >= (unsigned)p.nb) { bits |= HOOK_PAGES_BAD_PAGE; return; }
    unsigned slot = ((unsigned)page * 2654435769u) >> 21;      // 11 bits: kSlots
    for (int probe = 0; probe < kProbes; ++probe) {
      const int had = atomicCAS(&key[slot], -1, page);
      if (had == -1 || had == page) { atomicAdd(&change[slot], by); return; }
      slot = (slot + 1) % kSlots;
    }
    atomicAdd(&p.refs_out[page], by);
  };
  for (int c0 = blockIdx.x * kCols; c0 < columns; c0 += counters * kCols) {
    const int col = c0 + tid % kCols;
    for (int r0 = 0; r0 < total; r0 += kBatch) {
      const int rows = min(kBatch, total - r0);
      if (total > kBatch) {
        __syncthreads();
        for (int i = tid; i < rows; i += kForkThreads) origin[i] = held_by(r0 + i);
        __syncthreads();
      }
      constexpr int kAhead = 4;
      for (int i0 = lane; i0 < rows; i0 += kAhead * kLanes) {
        int page[kAhead];
        bool held[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          const int i = i0 + u * kLanes;
          const int2 o = i < rows ? origin[i] : make_int2(-1, 0);
          held[u] = col < o.y;
          if (held[u]) page[u] = p.table[(size_t)o.x * p.mb + col];
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
          if (held[u]) count(page[u], r0 + i0 + u * kLanes < p.rows ? 1 : -1);
      }
    }
    __syncthreads();
    for (int i = tid; i < kSlots; i += kForkThreads) {
      if (change[i] != 0) atomicAdd(&p.refs_out[key[i]], change[i]);
      if (TURNS) { key[i] = -1; change[i] = 0; }
    }
    if (!TURNS) break;
    __syncthreads();
  }
  report(p, bits);
}

// ---- the pages by number, for append and compact ----------------------------------------------------------

// A chunk: its free pages are listed and counted, and for a compaction the live ones too.
template <bool LIVE>
__device__ __forceinline__ void list_chunk(const PagesParams& p, int chunk, int* sh) {
  const int tid = threadIdx.x, first = chunk * kChunk + tid * kPer;
  int r[kPer], n = 0, count;
#pragma unroll
  for (int u = 0; u < kPer; ++u) r[u] = first + u < p.nb ? p.refs[first + u] : 1;
#pragma unroll
  for (int u = 0; u < kPer; ++u) n += r[u] <= 0;
  int frees = block_scan(n, sh, &count), lives = tid * kPer - frees;
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    if (first + u >= p.nb) break;
    if (p.refs_out != p.refs) p.refs_out[first + u] = r[u];
    if (LIVE) p.order[first + u] = r[u] <= 0 ? -1 - frees : lives;
    if (r[u] <= 0) p.free_list[(size_t)chunk * kChunk + frees++] = first + u;
    else if (LIVE) p.live_list[(size_t)chunk * kChunk + lives++] = first + u;
    else ++lives;
  }
  if (tid == 0) p.counts[chunk] = count;
}

// What a workgroup knows of all chunks: free pages before every segment of them (one chunk to a segment up to kThreads chunks).
struct Ranks {
  int before[kThreads + 1];
};

__device__ __forceinline__ int chunks_per_segment(const PagesParams& p) { return (p.nc + kThreads - 1) / kThreads; }

__device__ __forceinline__ void load_ranks(const PagesParams& p, Ranks& ranks, int* sh) {
  const int tid = threadIdx.x, per = chunks_per_segment(p);
  int n = 0, all;
  for (int c = tid * per; c < min((tid + 1) * per, p.nc); ++c) n += p.counts[c];
  ranks.before[tid] = block_scan(n, sh, &all);
  if (tid == 0) ranks.before[kThreads] = all;
  __syncthreads();
}

__device__ __forceinline__ int frees_before(const PagesParams& p, const Ranks& ranks, int chunk) {
  const int per = chunks_per_segment(p), seg = chunk / per;
  int n = ranks.before[seg];
  for (int c = seg * per; c < chunk; ++c) n += p.counts[c];
  return n;
}

// The k-th free page, or the k-th live one (0 is the lowest).
template <bool LIVE>
__device__ __forceinline__ int page_by_number(const PagesParams& p, const Ranks& ranks, int k) {
  const int per = chunks_per_segment(p);
  auto before = [&](int seg) {
    const int n = ranks.before[seg];
    return LIVE ? (int)min((long long)seg * per * kChunk, (long long)p.nb) - n : n;
  };
  int lo = 0, hi = kThreads;      // the last segment with no more than k before it
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (before(mid) <= k) lo = mid; else hi = mid;
  }
  int c = lo * per;
  k -= before(lo);
  for (; per > 1 && c + 1 < p.nc; ++c) {
    const int n = LIVE ? kChunk - p.counts[c] : p.counts[c];
    if (k < n) break;
    k -= n;
  }
  return (LIVE ? p.live_list : p.free_list)[(size_t)c * kChunk + k];
}

// ---- append ---------------------------------------------------------------------------------------------

// What row i writes: its length, its new tokens, and whether the first of them goes into a page that is partly filled.
__device__ __forceinline__ bool appends(const PagesParams& p, int i, int* len, int* n, int* bits) {
  *len = length_of(p.lens[i], p.mb, bits);
  const long long m = (long long)p.cu[i + 1] - p.cu[i];
  if (m < 0) *bits |= HOOK_PAGES_BAD_LENGTH;
  *n = m < 0 ? 0 : m > kTooMany ? kTooMany : (int)m;
  return *n > 0 && *len % kBlock != 0;
}

__device__ __forceinline__ int last_page(const PagesParams& p, int i, int len) { return p.table[(size_t)i * p.mb + len / kBlock]; }

// Workgroups below nc list the free pages of a chunk; in the others a wave plans a row: it looks through the rows before its own
// for those that leave the same last page, kRowsAhead rows to a lane at a time (one at a time, 512 rows took eight times two trips
// to memory one after the other: 8.0 us instead of 5.5).
__global__ __launch_bounds__(kThreads) void k_pages_plan(const PagesParams p) {
  __shared__ int sh[kThreads / 64];
  if ((int)blockIdx.x < p.nc) {
    list_chunk<false>(p, blockIdx.x, sh);
    return;
  }
  const int lane = threadIdx.x & 63, i = (blockIdx.x - p.nc) * (kThreads / 64) + (threadIdx.x >> 6);
  if (i >= p.S) return;
  int bits = 0, len, n;
  const bool writes = appends(p, i, &len, &n, &bits);
  int tail = -1;
  if (writes) {
    const int page = last_page(p, i, len);
    if ((unsigned)page >= (unsigned)p.nb) {
      bits |= HOOK_PAGES_BAD_PAGE;
    } else {
      constexpr int kRowsAhead = 4;
      int holders = p.refs[page];
      for (int j0 = 0; holders > 1 && j0 < i; j0 += 64 * kRowsAhead) {
        int at[kRowsAhead];
        bool partly[kRowsAhead];
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u) {
          const int j = j0 + u * 64 + lane;
          int n_j, ignored = 0;
          partly[u] = j < i && appends(p, j, &at[u], &n_j, &ignored);
        }
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u) {
          const bool leaves = partly[u] && last_page(p, j0 + u * 64 + lane, at[u]) == page;
          holders -= __popcll(__ballot(leaves));
        }
      }
      if (holders > 1) tail = page;
    }
  }
  if (lane == 0) {
    const bool fits = (long long)len + n <= (long long)p.mb * kBlock;
    RowPlan plan;
    plan.start = pages_of(len) - (tail >= 0);
    plan.tail = tail;
    plan.len = len;
    plan.grow = n;
    p.plan[i] = plan;
    p.need[i] = !fits ? kTooMany : n > 0 ? pages_of(len + n) - plan.start : 0;
    report(p, bits);
  }
}

constexpr int kInFlight = 4;      // 16-byte pieces of a thread in flight

// A workgroup takes a row and every `groups`-th cache.  The first of a row's writes its table entries, its length and the counts of
// its pages; all of them copy the token rows of the page that the row leaves.
template <int N>
__global__ __launch_bounds__(kThreads) void k_pages_append(const PagesParams p, int groups, const CacheList<N> list) {
  __shared__ Ranks ranks;
  __shared__ long long sh[kThreads / 64];
  __shared__ int shi[kThreads / 64];
  const int tid = threadIdx.x, row = blockIdx.x / groups, group = blockIdx.x - row * groups;
  const RowPlan plan = p.plan[row];
  if (group > 0 && plan.tail < 0) return;
  long long before = 0, total = 0;      // pages needed by the rows before this one, and by all
  for (int i = tid; i < p.S; i += kThreads) {
    const int n = p.need[i];
    total += n;
    if (i < row) before += n;
  }
  load_ranks(p, ranks, shi);
  total = block_sum(total, sh);
  const bool fits = total <= ranks.before[kThreads];
  if (group == 0) {
    if (p.table_out != p.table) {
      const int held = pages_of(plan.len), copied = fits && plan.tail >= 0 ? plan.start : -1;
      for (int e = tid; e < held; e += kThreads)
        if (e != copied) p.table_out[(size_t)row * p.mb + e] = p.table[(size_t)row * p.mb + e];
    }
    if (tid == 0) {
      p.lens_out[row] = fits ? plan.len + plan.grow : plan.len;
      if (!fits && row == 0) report(p, HOOK_PAGES_FULL);
      if (fits && plan.tail >= 0) atomicSub(&p.refs_out[plan.tail], 1);
    }
  }
  if (!fits) return;
  const int first = (int)block_sum(before, sh);
  if (group == 0) {
    const int need = p.need[row];
    for (int k = tid; k < need; k += kThreads) {
      const int page = page_by_number<false>(p, ranks, first + k);
      p.table_out[(size_t)row * p.mb + plan.start + k] = page;
      p.refs_out[page] = 1;
    }
  }
  if (plan.tail < 0) return;
  const int to = page_by_number<false>(p, ranks, first);
  const unsigned run = plan.len % kBlock * p.row_chunks, head = kBlock * p.row_chunks;      // 16-byte pieces copied and held of a head
  const size_t page = (size_t)p.heads * head;
  const unsigned pieces = p.heads * run;
  for (int c = group; c < p.ncaches; c += groups) {
    uint4* const cache = static_cast<uint4*>(list.cache[c]);
    const uint4* const src = cache + (size_t)plan.tail * page;
    uint4* const dst = cache + (size_t)to * page;
    for (unsigned x0 = tid; x0 < pieces; x0 += kInFlight * kThreads) {
      uint4 v[kInFlight];
      unsigned at[kInFlight];
#pragma unroll
      for (int u = 0; u < kInFlight; ++u) {
        const unsigned x = x0 + u * kThreads, h = x / run;
        at[u] = h * head + (x - h * run);
        if (x < pieces) v[u] = src[at[u]];      // (a last page was written not long ago)
      }
#pragma unroll
      for (int u = 0; u < kInFlight; ++u)
        if (x0 + u * kThreads < pieces) store_stream16(&dst[at[u]], v[u]);
    }
  }
}

// ---- compact --------------------------------------------------------------------------------------------

__global__ __launch_bounds__(kThreads) void k_pages_list(const PagesParams p) {
  __shared__ int sh[kThreads / 64];
  list_chunk<true>(p, blockIdx.x, sh);
}

// Three kinds of workgroups: the data, the map and the counts, and the table rows.  With `live` live pages, `moves` of them at or above
// number `live`, the moving pages are the last `moves` live ones and the holes the first `moves` free ones.
template <int N>
__global__ __launch_bounds__(kThreads) void k_pages_move(const PagesParams p, int movers, int mappers, int chunks, const CacheList<N> list) {
  __shared__ Ranks ranks;
  __shared__ int shi[kThreads / 64];
  const int tid = threadIdx.x;
  load_ranks(p, ranks, shi);
  const int live = p.nb - ranks.before[kThreads];
  int moves = 0;
  if (live < p.nb) {
    const int chunk = live / kChunk, order = p.order[live];
    moves = frees_before(p, ranks, chunk) + (order < 0 ? -1 - order : live - chunk * kChunk - order);
  }
  const int stay = live - moves;
  int b = blockIdx.x;
  if (b < movers) {
    // A piece of a page to the workgroup, or one to each of its waves where a page is less than the workgroup moves at a time (7000 pages
    // of 4 KB in 8 caches: 45 and 26 us; 8192 of 32 KB 202 and 205)
    const int page = p.heads * kBlock * p.row_chunks, threads = page >= kThreads * kInFlight ? kThreads : 64, lane = tid & (threads - 1);
    const int size = threads * kInFlight, pieces = (page + size - 1) / size, each = kThreads / threads;
    // (the pages of one cache are moved one after the other, so that workgroups that run together work on neighbours)
    const long long items = (long long)moves * p.ncaches * pieces;
    for (long long x = (long long)b * each + tid / threads; x < items; x += (long long)movers * each) {
      const long long rest = x / pieces;
      const int piece = (int)(x - rest * pieces), c = (int)(rest / moves), k = (int)(rest - (long long)c * moves);
      uint4* const cache = static_cast<uint4*>(list.cache[c]);
      const uint4* const src = cache + (size_t)page_by_number<true>(p, ranks, stay + k) * page;
      uint4* const dst = cache + (size_t)page_by_number<false>(p, ranks, k) * page;
      uint4 v[kInFlight];
#pragma unroll
      for (int u = 0; u < kInFlight; ++u) {
        const int at = piece * size + u * threads + lane;
        if (at < page) v[u] = p.keep_lines ? src[at] : load_stream16(&src[at]);
      }
#pragma unroll
      for (int u = 0; u < kInFlight; ++u) {
        const int at = piece * size + u * threads + lane;
        if (at < page) store_stream16(&dst[at], v[u]);
      }
    }
    return;
  }
  b -= movers;
  // the page that takes over what page `page` holds, or -1 for a free one
  auto moved = [&](int page) {
    const int order = p.order[page];
    if (order < 0) return -1;
    if (page < live) return page;
    const int chunk = page / kChunk, number = chunk * kChunk - frees_before(p, ranks, chunk) + order;
    return page_by_number<false>(p, ranks, number - stay);
  };
  if (b < mappers) {
    const int page = b * kThreads + tid;
    if (b == 0 && tid == 0) *p.num_live = live;
    if (page >= p.nb) return;
    const int to = moved(page);
    p.page_map[page] = to;
    if (to >= 0 && to != page) {      // (counts of a moving page and of its hole are read and written by this thread alone)
      p.refs_out[to] = p.refs[page];
      p.refs_out[page] = 0;
    }
    return;
  }
  b -= mappers;
  const int row = b / chunks, e0 = (b % chunks) * kRowChunk;
  int bits = 0;
  const int held = pages_of(length_of(p.lens[row], p.mb, &bits));
#pragma unroll
  for (int u = 0; u < kRowChunk / kThreads; ++u) {
    const int e = e0 + u * kThreads + tid;
    if (e >= held) continue;
    int page = p.table[(size_t)row * p.mb + e];
    const int to = (unsigned)page < (unsigned)p.nb ? moved(page) : -1;
    if (to < 0) bits |= HOOK_PAGES_BAD_PAGE;
    else page = to;
    p.table_out[(size_t)row * p.mb + e] = page;
  }
  report(p, bits);
}

// ---- host side ------------------------------------------------------------------------------------------

inline size_t align16(size_t x) { return (x + 15) / 16 * 16; }

struct Scratch {
  size_t plan, need, counts, free_list, live_list, order, bytes;
};

Scratch scratch_of(int S, int nb) {
  Scratch s;
  const size_t nc = ((size_t)nb + kChunk - 1) / kChunk;
  s.plan = 0;
  s.need = align16(sizeof(RowPlan) * (size_t)S);
  s.counts = s.need + align16(4 * (size_t)S);
  s.free_list = s.counts + align16(4 * nc);
  s.live_list = s.free_list + 4 * nc * kChunk;
  s.order = s.live_list + 4 * nc * kChunk;
  s.bytes = s.order + align16(4 * (size_t)nb);
  return s;
}

bool sizes_ok(const hook_pages_args* a) { return a->num_seqs >= 0 && a->max_blocks_per_seq > 0 && a->num_blocks > 0; }

bool sizes_supported(const hook_pages_args* a) {
  return a->block_size == HOOK_BLOCK_SIZE && a->max_blocks_per_seq <= (1 << 26) && a->num_blocks < kTooMany && a->num_seqs <= (1 << 26);
}

// Whether [a, a + n) and [b, b + m) share a byte.
bool overlap(const void* a, size_t n, const void* b, size_t m) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + m && y < x + n;
}

// Two int32 arrays of n entries: the same array, or nothing in common.
bool same_or_apart(const void* a, const void* b, size_t n) { return a == b || !overlap(a, 4 * n, b, 4 * n); }

long long row_chunks_of(const hook_pages_args* a) { return (a->max_blocks_per_seq + kRowChunk - 1) / kRowChunk; }

PagesParams params_of(const hook_pages_args* a) {
  PagesParams p{};
  p.S = a->num_seqs; p.mb = a->max_blocks_per_seq; p.nb = a->num_blocks; p.rows = a->num_rows;
  p.table = a->block_table; p.lens = a->seq_lens; p.refs = a->ref_counts;
  p.table_out = a->block_table_out; p.lens_out = a->seq_lens_out; p.refs_out = a->ref_counts_out; p.status = a->status;
  p.src = a->src_rows; p.keep = a->src_lens; p.cu = a->cu_q_lens;
  p.page_map = a->page_map; p.num_live = a->num_live;
  return p;
}

// What append and compact check alike; fills in scratch and caches.
hook_status prepare(const hook_pages_args* a, PagesParams* p) {
  if (a->num_caches < 0 || (a->num_caches > 0 && (a->num_kv_heads <= 0 || a->row_bytes <= 0))) return HOOK_ERR_SHAPE;
  if (a->num_caches > HOOK_PAGES_MAX_CACHES) return HOOK_ERR_UNSUPPORTED;
  if (a->num_caches > 0) {
    if (a->row_bytes % 16 != 0 || a->row_bytes > (1 << 20) || (long long)a->num_kv_heads * a->row_bytes > (1ll << 27)) return HOOK_ERR_UNSUPPORTED;
    if (!a->caches) return HOOK_ERR_NULL;
    for (int c = 0; c < a->num_caches; ++c) {
      if (!a->caches[c]) return HOOK_ERR_NULL;
      if (reinterpret_cast<uintptr_t>(a->caches[c]) % 16 != 0) return HOOK_ERR_UNSUPPORTED;
    }
    p->heads = a->num_kv_heads;
    p->row_chunks = (int)(a->row_bytes / 16);
  }
  p->ncaches = a->num_caches;
  const Scratch s = scratch_of(a->num_seqs, a->num_blocks);
  if (!a->workspace || a->workspace_bytes < s.bytes || reinterpret_cast<uintptr_t>(a->workspace) % 16 != 0) return HOOK_ERR_WORKSPACE;
  char* ws = static_cast<char*>(a->workspace);
  p->nc = (a->num_blocks + kChunk - 1) / kChunk;
  p->plan = reinterpret_cast<RowPlan*>(ws + s.plan);
  p->need = reinterpret_cast<int*>(ws + s.need);
  p->counts = reinterpret_cast<int*>(ws + s.counts);
  p->free_list = reinterpret_cast<int*>(ws + s.free_list);
  p->live_list = reinterpret_cast<int*>(ws + s.live_list);
  p->order = reinterpret_cast<int*>(ws + s.order);
  return HOOK_OK;
}

template <int N> CacheList<N> list_of(const hook_pages_args* a) {
  CacheList<N> list{};
  for (int c = 0; c < a->num_caches; ++c) list.cache[c] = a->caches[c];
  return list;
}

}  // namespace
}  // namespace hook

extern "C" {

size_t hook_pages_workspace_bytes(const hook_pages_args* a) {
  if (!a || a->num_seqs < 0 || a->num_blocks <= 0) return 0;
  return hook::scratch_of(a->num_seqs, a->num_blocks).bytes;
}

hook_status hook_pages_fork(const hook_pages_args* a) {
  using namespace hook;
  if (!a) return HOOK_ERR_NULL;
  if (!sizes_ok(a) || a->num_rows < 0) return HOOK_ERR_SHAPE;
  if (!sizes_supported(a)) return HOOK_ERR_UNSUPPORTED;
  const long long chunks = row_chunks_of(a);
  const int columns = (a->max_blocks_per_seq + kCols - 1) / kCols;
  const long long workgroups = a->num_rows * chunks + std::min(columns, kCounters);
  if (a->num_rows > (1 << 26) || !grid_fits(workgroups, kForkThreads)) return HOOK_ERR_UNSUPPORTED;
  const bool no_rows = a->num_rows == 0 && a->num_seqs == 0;
  if (no_rows && a->ref_counts == a->ref_counts_out) return HOOK_OK;
  if (!a->ref_counts || !a->ref_counts_out || !a->status) return HOOK_ERR_NULL;
  if (a->num_seqs > 0 && (!a->block_table || !a->seq_lens)) return HOOK_ERR_NULL;
  if (a->num_rows > 0 && (!a->src_rows || !a->block_table_out || !a->seq_lens_out)) return HOOK_ERR_NULL;
  const size_t mb = (size_t)a->max_blocks_per_seq;
  if (a->num_seqs > 0 && a->num_rows > 0 &&
      (overlap(a->block_table, 4 * mb * a->num_seqs, a->block_table_out, 4 * mb * a->num_rows) ||
       overlap(a->seq_lens, 4 * (size_t)a->num_seqs, a->seq_lens_out, 4 * (size_t)a->num_rows)))
    return HOOK_ERR_SHAPE;
  if (!same_or_apart(a->ref_counts, a->ref_counts_out, (size_t)a->num_blocks)) return HOOK_ERR_SHAPE;
  hipStream_t st = static_cast<hipStream_t>(a->stream);
  const PagesParams p = params_of(a);
  if (p.refs != p.refs_out) {
    hipLaunchKernelGGL(k_pages_copy_counts, dim3((unsigned)((p.nb + kThreads - 1) / kThreads)), dim3(kThreads), 0, st, p.refs, p.refs_out, p.nb);
    if (hipGetLastError() != hipSuccess) return HOOK_ERR_LAUNCH;
  }
  if (no_rows) return HOOK_OK;
  const dim3 grid((unsigned)workgroups);
  if (columns > kCounters) hipLaunchKernelGGL(k_pages_fork<true>, grid, dim3(kForkThreads), 0, st, p, (int)chunks);
  else hipLaunchKernelGGL(k_pages_fork<false>, grid, dim3(kForkThreads), 0, st, p, (int)chunks);
  return hipGetLastError() == hipSuccess ? HOOK_OK : HOOK_ERR_LAUNCH;
}

hook_status hook_pages_append(const hook_pages_args* a) {
  using namespace hook;
  if (!a) return HOOK_ERR_NULL;
  if (!sizes_ok(a)) return HOOK_ERR_SHAPE;
  if (!sizes_supported(a)) return HOOK_ERR_UNSUPPORTED;
  if (!a->ref_counts || !a->ref_counts_out || !a->status) return HOOK_ERR_NULL;
  if (a->num_seqs > 0 && (!a->block_table || !a->seq_lens || !a->block_table_out || !a->seq_lens_out || !a->cu_q_lens)) return HOOK_ERR_NULL;
  const size_t entries = (size_t)a->max_blocks_per_seq * a->num_seqs;
  if (!same_or_apart(a->block_table, a->block_table_out, entries) || !same_or_apart(a->seq_lens, a->seq_lens_out, (size_t)a->num_seqs) ||
      !same_or_apart(a->ref_counts, a->ref_counts_out, (size_t)a->num_blocks))
    return HOOK_ERR_SHAPE;
  PagesParams p = params_of(a);
  const hook_status checked = prepare(a, &p);
  if (checked != HOOK_OK) return checked;
  // a workgroup per row and cache while those are few, then caches take turns
  int groups = p.ncaches > 0 ? p.ncaches : 1;
  while (groups > 1 && (long long)groups * p.S > 4096) groups = (groups + 1) / 2;
  const int waves = kThreads / 64;
  if (!grid_fits((long long)p.S * groups, kThreads)) return HOOK_ERR_UNSUPPORTED;
  if (p.S == 0 && p.refs == p.refs_out) return HOOK_OK;
  hipStream_t st = static_cast<hipStream_t>(a->stream);
  hipLaunchKernelGGL(k_pages_plan, dim3((unsigned)(p.nc + (p.S + waves - 1) / waves)), dim3(kThreads), 0, st, p);
  if (hipGetLastError() != hipSuccess) return HOOK_ERR_LAUNCH;
  const dim3 grid((unsigned)(p.S * groups));
  if (p.S == 0) return HOOK_OK;
  if (p.ncaches <= kFewCaches) hipLaunchKernelGGL(k_pages_append<kFewCaches>, grid, dim3(kThreads), 0, st, p, groups, list_of<kFewCaches>(a));
  else hipLaunchKernelGGL(k_pages_append<HOOK_PAGES_MAX_CACHES>, grid, dim3(kThreads), 0, st, p, groups, list_of<HOOK_PAGES_MAX_CACHES>(a));
  return hipGetLastError() == hipSuccess ? HOOK_OK : HOOK_ERR_LAUNCH;
}

hook_status hook_pages_compact(const hook_pages_args* a) {
  using namespace hook;
  if (!a) return HOOK_ERR_NULL;
  if (!sizes_ok(a)) return HOOK_ERR_SHAPE;
  if (!sizes_supported(a)) return HOOK_ERR_UNSUPPORTED;
  if (!a->ref_counts || !a->ref_counts_out || !a->status || !a->page_map || !a->num_live) return HOOK_ERR_NULL;
  if (a->num_seqs > 0 && (!a->block_table || !a->seq_lens || !a->block_table_out)) return HOOK_ERR_NULL;
  const size_t entries = (size_t)a->max_blocks_per_seq * a->num_seqs;
  if (!same_or_apart(a->block_table, a->block_table_out, entries) || !same_or_apart(a->ref_counts, a->ref_counts_out, (size_t)a->num_blocks))
    return HOOK_ERR_SHAPE;
  PagesParams p = params_of(a);
  const hook_status checked = prepare(a, &p);
  if (checked != HOOK_OK) return checked;
  const long long chunks = row_chunks_of(a);
  const int mappers = (p.nb + kThreads - 1) / kThreads, movers = p.ncaches > 0 ? 1024 : 0;
  // Ordinary loads where all caches together fit 256 MB of last-level cache, streaming ones otherwise: 8 caches of 512 pages of 32 KB 16.7 and
  // 18.2 us, of 8192 pages 218 and 205.
  p.keep_lines = (long long)p.ncaches * p.nb * p.heads * kBlock * p.row_chunks * 16 <= (256ll << 20);
  if (!grid_fits(movers + mappers + p.S * chunks, kThreads)) return HOOK_ERR_UNSUPPORTED;
  hipStream_t st = static_cast<hipStream_t>(a->stream);
  hipLaunchKernelGGL(k_pages_list, dim3((unsigned)p.nc), dim3(kThreads), 0, st, p);
  if (hipGetLastError() != hipSuccess) return HOOK_ERR_LAUNCH;
  const dim3 grid((unsigned)(movers + mappers + p.S * chunks));
  if (p.ncaches <= kFewCaches)
    hipLaunchKernelGGL(k_pages_move<kFewCaches>, grid, dim3(kThreads), 0, st, p, movers, mappers, (int)chunks, list_of<kFewCaches>(a));
  else
    hipLaunchKernelGGL(k_pages_move<HOOK_PAGES_MAX_CACHES>, grid, dim3(kThreads), 0, st, p, movers, mappers, (int)chunks, list_of<HOOK_PAGES_MAX_CACHES>(a));
  return hipGetLastError() == hipSuccess ? HOOK_OK : HOOK_ERR_LAUNCH;
}

}  // extern "C"
