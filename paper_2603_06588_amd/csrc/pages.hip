// Pages of the paged cache shared between sequences: fork (share, reorder, cut back, free), append (allocate, copy shared
// last pages) and compact (move live pages to the front).  Everything is decided on the device from the tables and
// the reference counts; the host sees none of them, so each call is a fixed sequence of launches.
//
// Bookkeeping is bound by launches and by trips to memory, the data by its bandwidth: a copied page is read once and
// written once, by workgroups that take one piece of one page in one cache at a time.
// Sums over pages (which is the k-th free one) are taken in two steps: a launch counts every chunk of kChunk pages, and each
// workgroup of the next one adds up the counts before its own chunk for itself, which saves a launch in between.
#include "../../include/hook_api.h"
#include "hook_device.h"

namespace hook {
namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 2048;          // pages of a workgroup, eight to a thread
constexpr int kPer = kChunk / kThreads;
constexpr int kRowChunk = 1024;       // table entries of a workgroup, four to a thread
constexpr int kTooMany = 0x3fffffff;  // "needs" of a row that the table cannot hold: more than any cache has

struct RowPlan {
  int need;    // new pages
  int start;   // first table entry that gets one
  int tail;    // page to be copied into the first of them, or -1
  int len;     // tokens that the row holds before the call
};

struct PagesParams {
  int S, mb, nb, rows;
  const int *table, *lens, *refs;
  int *table_out, *lens_out, *refs_out, *status;
  const int *src, *keep, *cu;
  int *page_map, *num_live;
  // scratch
  int nc;            // chunks
  int* counts;       // [nc] free (append) or live (compact) pages of a chunk
  RowPlan* plan;     // [S]
  int *order, *movers, *holes, *moves;
  // data
  int ncaches, heads;
  int row_chunks;    // 16-byte pieces of a token row of one head
  void* cache[HOOK_PAGES_MAX_CACHES];
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

// A workgroup takes kRowChunk entries of one row.  As a row of the new table it copies them from the row it comes from; as a row of the
// old one it adds to the count of each of its pages the new rows that hold it less one (itself).  New rows hold a
// row's pages up to a cut of their own: the cuts are counted in shared memory, and a page at entry e has as many new holders as
// there are cuts behind e.
__global__ __launch_bounds__(kThreads) void k_pages_fork(const PagesParams p, int chunks) {
  __shared__ int cuts[kRowChunk + 1];
  __shared__ int sh[kThreads / 64];
  const int tid = threadIdx.x, row = blockIdx.x / chunks, e0 = (blockIdx.x % chunks) * kRowChunk;
  int bits = 0;
  if (row < p.rows) {
    const int from = p.src[row];
    int len = 0;
    if (from >= 0 && from < p.S) {
      len = length_of(p.lens[from], p.mb, &bits);
      if (p.keep) len = min(len, max(p.keep[row], 0));
    } else if (from != -1) {
      bits |= HOOK_PAGES_BAD_ROW;
    }
    if (e0 == 0 && tid == 0) p.lens_out[row] = len;
    const int held = pages_of(len);
#pragma unroll
    for (int u = 0; u < kRowChunk / kThreads; ++u) {
      const int e = e0 + u * kThreads + tid;
      if (e < held) p.table_out[(size_t)row * p.mb + e] = p.table[(size_t)from * p.mb + e];
    }
  }
  if (row < p.S) {
    const int len = length_of(p.lens[row], p.mb, &bits), held = pages_of(len);
    if (e0 < held) {      // (the same for the whole workgroup)
      for (int i = tid; i <= kRowChunk; i += kThreads) cuts[i] = 0;
      __syncthreads();
      for (int j = tid; j < p.rows; j += kThreads)
        if (p.src[j] == row) {
          const int cut = pages_of(p.keep ? min(len, max(p.keep[j], 0)) : len) - e0;
          if (cut > 0) atomicAdd(&cuts[min(cut, kRowChunk)], 1);
        }
      __syncthreads();
      // a thread owns four entries in a row; cuts[x] > 0 for x > e counts
      const int at = tid * (kRowChunk / kThreads);
      int mine[kRowChunk / kThreads], sum = 0;
#pragma unroll
      for (int u = 0; u < kRowChunk / kThreads; ++u) { mine[u] = cuts[at + u + 1]; sum += mine[u]; }
      int all;
      const int before = block_scan(sum, sh, &all);
      int behind = all - before;      // cuts at at + 1 and behind
#pragma unroll
      for (int u = 0; u < kRowChunk / kThreads; ++u) {
        const int e = e0 + at + u, change = behind - 1;
        behind -= mine[u];
        if (e < held) {
          const int page = p.table[(size_t)row * p.mb + e];
          if ((unsigned)page >= (unsigned)p.nb) bits |= HOOK_PAGES_BAD_PAGE;
          else if (change != 0) atomicAdd(&p.refs_out[page], change);
        }
      }
    }
  }
  report(p, bits);
}

// ---- counting, shared by append and compact ---------------------------------------------------------------

// Counts of this thread's eight pages; entries past the last page read as `past`.
__device__ __forceinline__ void chunk_refs(const int* refs, int nb, int chunk, int past, int (&r)[kPer]) {
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    const int page = chunk * kChunk + threadIdx.x * kPer + u;
    r[u] = page < nb ? refs[page] : past;
  }
}

// Chunk counts before `chunk` and all of them.
__device__ __forceinline__ long long counts_before(const PagesParams& p, int chunk, long long* sh, long long* all) {
  long long before = 0, sum = 0;
  for (int c = threadIdx.x; c < p.nc; c += kThreads) {
    const int n = p.counts[c];
    sum += n;
    if (c < chunk) before += n;
  }
  *all = block_sum(sum, sh);
  return block_sum(before, sh);
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

// Workgroups below nc count the free pages of a chunk; in the others a wave plans a row: it looks through the rows before its own
// for those that leave the same last page.
__global__ __launch_bounds__(kThreads) void k_pages_plan(const PagesParams p) {
  __shared__ long long sh[kThreads / 64];
  if ((int)blockIdx.x < p.nc) {
    int r[kPer], n = 0;
    chunk_refs(p.refs, p.nb, blockIdx.x, 1, r);
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const int page = blockIdx.x * kChunk + threadIdx.x * kPer + u;
      n += r[u] <= 0;
      if (p.refs_out != p.refs && page < p.nb) p.refs_out[page] = r[u];
    }
    const long long sum = block_sum(n, sh);
    if (threadIdx.x == 0) p.counts[blockIdx.x] = (int)sum;
    return;
  }
  const int lane = threadIdx.x & 63, i = (blockIdx.x - p.nc) * (kThreads / 64) + (threadIdx.x >> 6);
  if (i >= p.S) return;
  int bits = 0, len, n;
  const bool writes = appends(p, i, &len, &n, &bits);
  int tail = -1;
  if (writes && len < (long long)p.mb * kBlock) {
    const int page = last_page(p, i, len);
    if ((unsigned)page >= (unsigned)p.nb) {
      bits |= HOOK_PAGES_BAD_PAGE;
    } else {
      int holders = p.refs[page];
      for (int j0 = 0; holders > 1 && j0 < i; j0 += 64) {
        const int j = j0 + lane;
        bool leaves = false;
        if (j < i) {
          int len_j, n_j, ignored = 0;
          leaves = appends(p, j, &len_j, &n_j, &ignored) && last_page(p, j, len_j) == page;
        }
        holders -= __popcll(__ballot(leaves));
      }
      if (holders > 1) tail = page;
    }
  }
  if (lane == 0) {
    const bool fits = (long long)len + n <= (long long)p.mb * kBlock;
    RowPlan plan;
    plan.start = pages_of(len) - (tail >= 0);
    plan.need = !fits ? kTooMany : n > 0 ? pages_of(len + n) - plan.start : 0;
    plan.tail = tail;
    plan.len = len;
    p.plan[i] = plan;
    report(p, bits);
  }
}

// Workgroups below nc hand out the free pages of a chunk; in the others kRowChunk table entries of a row are carried over, and the first of
// a row's also writes its length and takes a copied page's holder away.
__global__ __launch_bounds__(kThreads) void k_pages_assign(const PagesParams p, int chunks) {
  __shared__ long long sh[kThreads / 64];
  __shared__ int shi[kThreads / 64];
  __shared__ int freed[kChunk];
  __shared__ long long ends[kThreads];      // pages needed up to and with a row of the tile
  const int tid = threadIdx.x, b = blockIdx.x;
  long long need = 0, all;
  for (int i = tid; i < p.S; i += kThreads) need += p.plan[i].need;
  need = block_sum(need, sh);
  const long long base = counts_before(p, b, sh, &all);
  const bool fits = need <= all;
  if (b < p.nc) {
    if (!fits) {
      if (b == 0 && tid == 0) report(p, HOOK_PAGES_FULL);
      return;
    }
    if (base >= need) return;
    int r[kPer], n = 0, count;
    chunk_refs(p.refs, p.nb, b, 1, r);
#pragma unroll
    for (int u = 0; u < kPer; ++u) n += r[u] <= 0;
    int at = block_scan(n, shi, &count);
#pragma unroll
    for (int u = 0; u < kPer; ++u)
      if (r[u] <= 0) freed[at++] = b * kChunk + tid * kPer + u;
    __syncthreads();
    const long long end = base + count < need ? base + count : need;      // pages base .. end - 1 of those handed out lie here
    long long carry = 0;
    for (int i0 = 0; i0 < p.S && carry < end; i0 += kThreads) {
      const int i = i0 + tid;
      int tile;
      const int mine = i < p.S ? p.plan[i].need : 0;
      const int before = block_scan(mine, shi, &tile);      // (a tile needs no more than there are pages)
      ends[tid] = carry + before + mine;
      __syncthreads();
      const long long lo = base > carry ? base : carry, hi = end < carry + tile ? end : carry + tile;
      for (long long k = lo + tid; k < hi; k += kThreads) {
        int a = 0, z = kThreads - 1;      // first row with ends > k
        while (a < z) {
          const int mid = (a + z) >> 1;
          if (ends[mid] > k) z = mid; else a = mid + 1;
        }
        const RowPlan plan = p.plan[i0 + a];
        const int e = plan.start + (int)(k - (ends[a] - plan.need)), page = freed[k - base];
        p.table_out[(size_t)(i0 + a) * p.mb + e] = page;
        p.refs_out[page] = 1;
      }
      carry += tile;
      __syncthreads();
    }
    return;
  }
  const int row = (b - p.nc) / chunks, e0 = ((b - p.nc) % chunks) * kRowChunk;
  const RowPlan plan = p.plan[row];
  if (p.table_out != p.table) {
    const int held = pages_of(plan.len), copied = fits && plan.tail >= 0 ? plan.start : -1;
#pragma unroll
    for (int u = 0; u < kRowChunk / kThreads; ++u) {
      const int e = e0 + u * kThreads + tid;
      if (e < held && e != copied) p.table_out[(size_t)row * p.mb + e] = p.table[(size_t)row * p.mb + e];
    }
  }
  if (e0 == 0 && tid == 0) {
    p.lens_out[row] = fits ? plan.len + max(p.cu[row + 1] - p.cu[row], 0) : plan.len;
    if (plan.tail >= 0) {
      if (fits) atomicSub(&p.refs_out[plan.tail], 1);
      else p.plan[row].tail = -1;      // nothing is copied
    }
  }
}

// The first token rows of the pages that rows leave: a workgroup takes one row and every `groups`-th cache.
__global__ __launch_bounds__(kThreads) void k_pages_copy_tails(const PagesParams p, int groups) {
  const int row = blockIdx.x / groups;
  const RowPlan plan = p.plan[row];
  if (plan.tail < 0) return;
  const int to = p.table_out[(size_t)row * p.mb + plan.start];
  const int run = plan.len % kBlock * p.row_chunks, head = kBlock * p.row_chunks;      // 16-byte pieces copied and held of a head
  const size_t page = (size_t)p.heads * head;
  for (int c = blockIdx.x % groups; c < p.ncaches; c += groups) {
    uint4* const cache = static_cast<uint4*>(p.cache[c]);
    const uint4* const src = cache + (size_t)plan.tail * page;
    uint4* const dst = cache + (size_t)to * page;
    for (int x = threadIdx.x; x < p.heads * run; x += kThreads) {
      const int h = x / run, at = h * head + (x - h * run);
      dst[at] = src[at];
    }
  }
}

// ---- compact --------------------------------------------------------------------------------------------

__global__ __launch_bounds__(kThreads) void k_pages_count_live(const PagesParams p) {
  __shared__ long long sh[kThreads / 64];
  int r[kPer], n = 0;
  chunk_refs(p.refs, p.nb, blockIdx.x, 0, r);
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    const int page = blockIdx.x * kChunk + threadIdx.x * kPer + u;
    n += r[u] > 0;
    if (p.refs_out != p.refs && page < p.nb) p.refs_out[page] = r[u];
  }
  const long long sum = block_sum(n, sh);
  if (threadIdx.x == 0) p.counts[blockIdx.x] = (int)sum;
}

// Ranks the pages that move and the holes that they move to.  order[page]: rank among the moving pages, -1 (a live page that
// stays) or -2 (free).
__global__ __launch_bounds__(kThreads) void k_pages_rank(const PagesParams p) {
  __shared__ long long sh[kThreads / 64];
  __shared__ int shi[kThreads / 64];
  const int tid = threadIdx.x, b = blockIdx.x;
  long long all;
  const long long base = counts_before(p, b, sh, &all);
  const int live = (int)all;
  // live pages below `live`: those of the chunks before the one that `live` lies in, and some of that one's
  const int border = live / kChunk;
  long long below = 0;
  for (int c = tid; c < border && c < p.nc; c += kThreads) below += p.counts[c];
  if (border < p.nc) {
    int r[kPer];
    chunk_refs(p.refs, p.nb, border, 0, r);
#pragma unroll
    for (int u = 0; u < kPer; ++u) below += r[u] > 0 && border * kChunk + tid * kPer + u < live;
  }
  below = block_sum(below, sh);
  int r[kPer], n = 0, count;
  chunk_refs(p.refs, p.nb, b, 0, r);
#pragma unroll
  for (int u = 0; u < kPer; ++u) n += r[u] > 0;
  int rank = (int)base + block_scan(n, shi, &count);      // live pages before this one
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    const int page = b * kChunk + tid * kPer + u;
    if (page >= p.nb) break;
    int order = -2;
    if (r[u] > 0) {
      order = -1;
      if (page >= live) {
        order = rank - (int)below;
        p.movers[order] = page;
      } else {
        p.page_map[page] = page;
      }
      ++rank;
    } else {
      if (page < live) p.holes[page - rank] = page;
      p.page_map[page] = -1;
    }
    p.order[page] = order;
  }
  if (b == 0 && tid == 0) {
    *p.moves = live - (int)below;
    *p.num_live = live;
  }
}

constexpr int kMoveInFlight = 4;
constexpr int kPiece = kThreads * kMoveInFlight;      // 16-byte pieces of a page that a workgroup moves at a time

// Three kinds of workgroups: counts and map of the moved pages, table rows, and the data.
__global__ __launch_bounds__(kThreads) void k_pages_move(const PagesParams p, int fixers, int chunks, int movers) {
  const int tid = threadIdx.x;
  int b = blockIdx.x;
  if (b < movers) {
    const int moves = *p.moves;
    const int page = p.heads * kBlock * p.row_chunks, pieces = (page + kPiece - 1) / kPiece;
    const long long items = (long long)moves * p.ncaches * pieces;
    for (long long x = b; x < items; x += movers) {
      const int piece = (int)(x % pieces);
      const long long rest = x / pieces;
      const int c = (int)(rest % p.ncaches), k = (int)(rest / p.ncaches);
      uint4* const cache = static_cast<uint4*>(p.cache[c]);
      const uint4* const src = cache + (size_t)p.movers[k] * page;
      uint4* const dst = cache + (size_t)p.holes[k] * page;
      uint4 v[kMoveInFlight];
#pragma unroll
      for (int u = 0; u < kMoveInFlight; ++u) {
        const int at = piece * kPiece + u * kThreads + tid;
        if (at < page) v[u] = load_stream16(&src[at]);
      }
#pragma unroll
      for (int u = 0; u < kMoveInFlight; ++u) {
        const int at = piece * kPiece + u * kThreads + tid;
        if (at < page) store_stream16(&dst[at], v[u]);
      }
    }
    return;
  }
  b -= movers;
  if (b < fixers) {
    const int k = b * kThreads + tid;
    if (k < *p.moves) {
      const int from = p.movers[k], to = p.holes[k];
      p.page_map[from] = to;
      p.refs_out[to] = p.refs[from];      // (a moving page's count is read and written by this thread alone)
      p.refs_out[from] = 0;
    }
    return;
  }
  b -= fixers;
  const int row = b / chunks, e0 = (b % chunks) * kRowChunk;
  int bits = 0;
  const int held = pages_of(length_of(p.lens[row], p.mb, &bits));
#pragma unroll
  for (int u = 0; u < kRowChunk / kThreads; ++u) {
    const int e = e0 + u * kThreads + tid;
    if (e >= held) continue;
    int page = p.table[(size_t)row * p.mb + e];
    if ((unsigned)page >= (unsigned)p.nb) {
      bits |= HOOK_PAGES_BAD_PAGE;
    } else {
      const int order = p.order[page];
      if (order >= 0) page = p.holes[order];
      else if (order == -2) bits |= HOOK_PAGES_BAD_PAGE;
    }
    p.table_out[(size_t)row * p.mb + e] = page;
  }
  report(p, bits);
}

// ---- host side ------------------------------------------------------------------------------------------

inline size_t align16(size_t x) { return (x + 15) / 16 * 16; }

struct Scratch {
  size_t plan, counts, moves, order, movers, holes, bytes;
};

Scratch scratch_of(int S, int nb) {
  Scratch s;
  const size_t nc = ((size_t)nb + kChunk - 1) / kChunk;
  s.plan = 0;
  s.moves = align16(sizeof(RowPlan) * (size_t)S);
  s.counts = s.moves + 16;
  s.order = s.counts + align16(4 * nc);
  s.movers = s.order + align16(4 * (size_t)nb);
  s.holes = s.movers + align16(4 * ((size_t)nb / 2 + 1));
  s.bytes = s.holes + align16(4 * ((size_t)nb / 2 + 1));
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
      p->cache[c] = a->caches[c];
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
  p->moves = reinterpret_cast<int*>(ws + s.moves);
  p->counts = reinterpret_cast<int*>(ws + s.counts);
  p->order = reinterpret_cast<int*>(ws + s.order);
  p->movers = reinterpret_cast<int*>(ws + s.movers);
  p->holes = reinterpret_cast<int*>(ws + s.holes);
  return HOOK_OK;
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
  const long long rows = a->num_rows > a->num_seqs ? a->num_rows : a->num_seqs, chunks = row_chunks_of(a);
  if (!grid_fits(rows * chunks)) return HOOK_ERR_UNSUPPORTED;
  if (rows == 0) return HOOK_OK;
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
  hipLaunchKernelGGL(k_pages_fork, dim3((unsigned)(rows * chunks)), dim3(kThreads), 0, st, p, (int)chunks);
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
  const long long chunks = row_chunks_of(a);
  // a workgroup per row and cache while those are few, then caches take turns
  int groups = p.ncaches;
  while (groups > 1 && (long long)groups * p.S > 8192) groups = (groups + 1) / 2;
  if (!grid_fits(p.nc + (long long)p.S * chunks) || !grid_fits((long long)p.S * (groups > 0 ? groups : 1))) return HOOK_ERR_UNSUPPORTED;
  hipStream_t st = static_cast<hipStream_t>(a->stream);
  const int waves = kThreads / 64;
  hipLaunchKernelGGL(k_pages_plan, dim3((unsigned)(p.nc + (p.S + waves - 1) / waves)), dim3(kThreads), 0, st, p);
  if (hipGetLastError() != hipSuccess) return HOOK_ERR_LAUNCH;
  hipLaunchKernelGGL(k_pages_assign, dim3((unsigned)(p.nc + p.S * chunks)), dim3(kThreads), 0, st, p, (int)chunks);
  if (hipGetLastError() != hipSuccess) return HOOK_ERR_LAUNCH;
  if (p.S > 0 && groups > 0) hipLaunchKernelGGL(k_pages_copy_tails, dim3((unsigned)(p.S * groups)), dim3(kThreads), 0, st, p, groups);
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
  const int fixers = (p.nb / 2 + kThreads) / kThreads, movers = p.ncaches > 0 ? 2048 : 0;
  if (!grid_fits(movers + fixers + p.S * chunks)) return HOOK_ERR_UNSUPPORTED;
  hipStream_t st = static_cast<hipStream_t>(a->stream);
  hipLaunchKernelGGL(k_pages_count_live, dim3((unsigned)p.nc), dim3(kThreads), 0, st, p);
  if (hipGetLastError() != hipSuccess) return HOOK_ERR_LAUNCH;
  hipLaunchKernelGGL(k_pages_rank, dim3((unsigned)p.nc), dim3(kThreads), 0, st, p);
  if (hipGetLastError() != hipSuccess) return HOOK_ERR_LAUNCH;
  hipLaunchKernelGGL(k_pages_move, dim3((unsigned)(movers + fixers + p.S * chunks)), dim3(kThreads), 0, st, p, fixers, (int)chunks, movers);
  return hipGetLastError() == hipSuccess ? HOOK_OK : HOOK_ERR_LAUNCH;
}

}  // extern "C"
