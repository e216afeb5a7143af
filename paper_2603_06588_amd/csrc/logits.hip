// Penalties for repeated tokens, a bias list and a grammar mask on rows of logits.
//
// Bound by memory: a row is read once and written once.  A workgroup takes a range of one row's tokens, requests its logits and
// its mask, counts the row's history into shared memory while they come, lays the logits into shared memory too, lets one thread per
// token that occurred or is biased replace that token's logit there, and writes the range with barred tokens at -infinity.
// Only one token in many has a value to compute.  Looking every token's count up on the way out took nearly every wave through the
// divisions for the sake of one lane (256 x 131072 bf16 logits, 4250 tokens of history each: 93 us); writing the few values over the range
// in memory afterwards cost more than laying the range into shared memory (64 us).
// The counts take 16 bits (the top one: in the prompt), so that eight waves find room on every SIMD, and 32, half a range at a time, for a
// history of more generated tokens than 15 bits count.  Counts are whole numbers, a token's last bias entry is the one with the
// largest number, and every touched token is replaced by one thread: the order of the atomics changes nothing.
#include "../../include/hook_api.h"
#include "hook_device.h"

namespace hook {
namespace {

struct LogitsParams {
  int R, V;
  const char* logits;
  char* out;
  long long stride, out_stride;     // bytes
  int history_len, bias_len, masks, words;
  const int *history, *cu_history, *prompt_lens;
  const float *repetition, *frequency, *presence;
  const int *cu_bias, *bias_ids;
  const float* bias_values;
  const unsigned* mask;
  const int* mask_rows;
};

template <int BYTES> struct RawOf;
template <> struct RawOf<16> { typedef u32x4 type; };
template <> struct RawOf<4> { typedef unsigned int type; };
template <> struct RawOf<2> { typedef unsigned short type; };

template <typename E, int W> struct Vec {
  E e[W];
};

// The entries [cu[row], cu[row + 1]) of a list of n.
__device__ __forceinline__ void list_of(const int* cu, int row, int n, int* begin, int* end) {
  *begin = min(max(cu[row], 0), n);
  *end = min(max(cu[row + 1], *begin), n);
}

// What a workgroup knows about its row.
struct Row {
  int begin, generated, end;     // its history, and where the generated part of that begins
  int bias0, bias_end;           // its bias list
  float rep, freq, pres;
};

template <typename E, int kRange, int NT> struct Shared {
  unsigned count[kRange / 2];
  E tile[kRange];
  unsigned done[kRange / 32];         // bit per token: replaced with its bias
  unsigned bias_token[NT];            // tokens of the bias entries in the range, by hash, and the last entry of each
  int bias_last[NT];
  unsigned short listed[kRange / 8];  // tokens that got a count; with more than these the whole range is looked through instead
  int num_listed;
};

// Replaces the logits in the tile, whose first token is s0, that the history or a bias touches.  `lay` lays the logits into the tile.
template <bool WIDE, typename E, int kRange, int NT, typename F>
__device__ __forceinline__ void adjust(const LogitsParams& p, const Row& r, Shared<E, kRange, NT>& sh, unsigned s0, E* tile, F&& lay) {
  constexpr int kSpan = WIDE ? kRange / 2 : kRange, kListed = kRange / 8;
  static_assert((NT & (NT - 1)) == 0, "slots by a mask");
  constexpr unsigned kNoToken = 0xFFFFFFFFu, kPrompt = WIDE ? 0x80000000u : 0x8000u;
  const int tid = threadIdx.x;
  auto count_of = [&](unsigned at) { return WIDE ? sh.count[at] : (sh.count[at >> 1] >> (16 * (at & 1))) & 0xFFFFu; };
  if (tid == 0) sh.num_listed = 0;
  for (int i = tid; i < kRange / 8; i += NT) reinterpret_cast<uint4*>(sh.count)[i] = make_uint4(0u, 0u, 0u, 0u);
  for (int i = tid; i < kRange / 32; i += NT) sh.done[i] = 0;
  __syncthreads();
  constexpr int kAhead = 2;      // entries of a thread in flight
  for (int j0 = r.begin + tid; j0 < r.end; j0 += kAhead * NT) {
    unsigned at[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) at[u] = j0 + u * NT < r.end ? (unsigned)p.history[j0 + u * NT] - s0 : 0xFFFFFFFFu;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (at[u] >= (unsigned)kSpan) continue;
      const int shift = WIDE ? 0 : 16 * (at[u] & 1);
      unsigned* const c = &sh.count[WIDE ? at[u] : at[u] >> 1];
      const unsigned before = j0 + u * NT < r.generated ? atomicOr(c, kPrompt << shift) : atomicAdd(c, 1u << shift);
      if ((WIDE ? before : (before >> shift) & 0xFFFFu) == 0) {
        const int k = atomicAdd(&sh.num_listed, 1);
        if (k < kListed) sh.listed[k] = (unsigned short)at[u];
      }
    }
  }
  lay();
  __syncthreads();
  auto replace = [&](unsigned at, bool biased, float bias) {
    const unsigned w = count_of(at), n = w & (kPrompt - 1);
    float x = (float)tile[at];
    if (w != 0) x = x > 0.0f ? x / r.rep : x * r.rep;
    if (n != 0) x = (x - (float)n * r.freq) - r.pres;
    if (biased) x += bias;
    tile[at] = (E)x;
  };
  // From the list's end, NT entries at a time: of the entries that name a token the last one counts.  They find it in a hash table with as many
  // slots as there can be entries (13 x 1384 fp32 logits with 300 entries a row 6.2 us; comparing them with each other 12.6).
  for (int j1 = r.bias_end; j1 > r.bias0; j1 -= NT) {
    sh.bias_token[tid] = kNoToken;
    sh.bias_last[tid] = -1;
    const int j = j1 - 1 - tid;
    const unsigned at = j >= r.bias0 ? (unsigned)p.bias_ids[j] - s0 : kNoToken;
    const bool mine = at < (unsigned)kSpan && ((sh.done[at >> 5] >> (at & 31)) & 1u) == 0;
    const float value = mine ? p.bias_values[j] : 0.0f;
    unsigned slot = at * 2654435769u >> 16 & (NT - 1);
    __syncthreads();
    if (mine) {
      for (;; slot = (slot + 1) & (NT - 1)) {      // (NT slots, at most NT entries: there is one)
        const unsigned had = atomicCAS(&sh.bias_token[slot], kNoToken, at);
        if (had == kNoToken || had == at) break;
      }
      atomicMax(&sh.bias_last[slot], j);
    }
    __syncthreads();
    if (mine && sh.bias_last[slot] == j) {
      replace(at, true, value);
      atomicOr(&sh.done[at >> 5], 1u << (at & 31));
    }
    __syncthreads();
  }
  auto penalise = [&](unsigned at) {
    if (((sh.done[at >> 5] >> (at & 31)) & 1u) == 0) replace(at, false, 0.0f);
  };
  if (sh.num_listed <= kListed) {
    for (int i = tid; i < sh.num_listed; i += NT) penalise(sh.listed[i]);
  } else {
    for (int at = tid; at < kSpan; at += NT)
      if (count_of((unsigned)at) != 0) penalise((unsigned)at);
  }
  __syncthreads();
}

// W: elements of a load.  Each of the NT threads takes VPT loads of the range; the i-th of thread t starts at element
// (i * NT + t) * W of it.  Ranges are counted from the 16-byte border before the row's first token (`skew` elements before it), so
// rows of any vocabulary are read and written by aligned loads and stores of 16 bytes but for their first and last few tokens.
template <typename E, int W, int NT, int VPT>
__global__ __launch_bounds__(NT) void k_steer_logits(const LogitsParams p, int ranges, int turn) {
  typedef typename RawOf<sizeof(E) * W>::type Raw;
  constexpr int kRange = NT * VPT * W;
  static_assert(kRange <= 65536, "tokens are listed by 16 bits");
  __shared__ __align__(16) Shared<E, kRange, NT> sh;
  // A row's ranges lie on one XCD (workgroups go round the eight of them), whose cache then holds its history for all of them; with
  // fewer rows than XCDs every range goes where it comes.
  const int tid = threadIdx.x, slot = blockIdx.x >> turn, part = slot / ranges, row = (part << turn) + (blockIdx.x & ((1 << turn) - 1));
  const int r0 = (slot - part * ranges) * kRange;
  if (row >= p.R) return;
  const E* const in = reinterpret_cast<const E*>(p.logits + row * p.stride);
  E* const out = reinterpret_cast<E*>(p.out + row * p.out_stride);
  const int skew = (int)(reinterpret_cast<uintptr_t>(in) / sizeof(E) % W), token0 = r0 - skew;
  const int m = p.mask ? (p.mask_rows ? p.mask_rows[row] : row) : -1;
  const bool masked = m >= 0 && m < p.masks;
  const unsigned* const mask = p.mask + (masked ? (size_t)m * p.words : 0);
  unsigned allowed[VPT];                   // bits of the loads' tokens
  if (masked)
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int e = token0 + (i * NT + tid) * W, word = e >> 5;      // (below 0 where a row's first load begins before it)
      const unsigned lo = e >= 0 && e < p.V ? mask[word] : 0u;
      unsigned hi = 0u;
      if ((e & 31) + W > 32 && e + W > 0 && word + 1 < p.words) hi = mask[word + 1];
      allowed[i] = (unsigned)((((unsigned long long)hi << 32) | lo) >> (e & 31));
    }
  Raw raw[VPT];
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int e = token0 + (i * NT + tid) * W;
    // A load whose tokens are all barred is left out: 256 x 131072 bf16 with 2000 tokens of history each take 25.5 us where a grammar allows one
    // token in 2000 (29.2 with all loads), 28.4 and 28.9 where it allows a quarter or all.
    raw[i] = Raw{};
    if (masked && (allowed[i] & ((1u << W) - 1u)) == 0) continue;
    if (e >= 0 && e + W <= p.V) {
      raw[i] = __builtin_nontemporal_load(reinterpret_cast<const Raw*>(in + e));
    } else {      // the row's first or last tokens, fewer than a load
      Vec<E, W> v;
#pragma unroll
      for (int u = 0; u < W; ++u) v.e[u] = e + u >= 0 && e + u < p.V ? in[e + u] : (E)0.0f;
      __builtin_memcpy(&raw[i], &v, sizeof v);
    }
  }
  Row r{};
  r.rep = p.repetition ? p.repetition[row] : 1.0f;
  r.freq = p.frequency ? p.frequency[row] : 0.0f;
  r.pres = p.presence ? p.presence[row] : 0.0f;
  if (p.history && (r.rep != 1.0f || r.freq != 0.0f || r.pres != 0.0f)) list_of(p.cu_history, row, p.history_len, &r.begin, &r.end);
  if (p.cu_bias) list_of(p.cu_bias, row, p.bias_len, &r.bias0, &r.bias_end);
  r.generated = r.begin + (p.prompt_lens ? min(max(p.prompt_lens[row], 0), r.end - r.begin) : 0);

  auto write = [&](int i, Raw from) {
    const int e = token0 + (i * NT + tid) * W;
    Vec<E, W> v;
    __builtin_memcpy(&v, &from, sizeof v);
    if (masked)
#pragma unroll
      for (int u = 0; u < W; ++u)
        if (((allowed[i] >> u) & 1u) == 0) v.e[u] = (E)-__builtin_inff();
    if (e >= 0 && e + W <= p.V) {
      Raw x;
      __builtin_memcpy(&x, &v, sizeof x);
      __builtin_nontemporal_store(x, reinterpret_cast<Raw*>(out + e));
    } else {
#pragma unroll
      for (int u = 0; u < W; ++u)
        if (e + u >= 0 && e + u < p.V) out[e + u] = v.e[u];
    }
  };
  if (r.begin == r.end && r.bias0 == r.bias_end) {
#pragma unroll
    for (int i = 0; i < VPT; ++i) write(i, raw[i]);
    return;
  }
  auto lay = [&]() {
#pragma unroll
    for (int i = 0; i < VPT; ++i) reinterpret_cast<Raw*>(sh.tile)[i * NT + tid] = raw[i];
  };
  if (r.end - r.generated <= 0x7FFF) {
    adjust<false, E, kRange, NT>(p, r, sh, (unsigned)token0, sh.tile, lay);
  } else {
    adjust<true, E, kRange, NT>(p, r, sh, (unsigned)token0, sh.tile, lay);
    adjust<true, E, kRange, NT>(p, r, sh, (unsigned)(token0 + kRange / 2), sh.tile + kRange / 2, []() {});
  }
#pragma unroll
  for (int i = 0; i < VPT; ++i) write(i, reinterpret_cast<const Raw*>(sh.tile)[i * NT + tid]);
}

template <typename E, int W, int NT, int VPT>
hook_status launch_range(const LogitsParams& p, hipStream_t st) {
  const bool on_border = (reinterpret_cast<uintptr_t>(p.logits) | (uintptr_t)p.stride) % 16 == 0;      // else a row may begin W - 1 elements behind one
  const int ranges = (p.V + (on_border ? 0 : W - 1) + NT * VPT * W - 1) / (NT * VPT * W);
  const int turn = p.R >= 8 ? 3 : 0;
  const long long workgroups = (((long long)p.R + (1 << turn) - 1) >> turn << turn) * ranges;
  if (!grid_fits(workgroups, NT)) return HOOK_ERR_UNSUPPORTED;
  hipLaunchKernelGGL((k_steer_logits<E, W, NT, VPT>), dim3((unsigned)workgroups), dim3(NT), 0, st, p, ranges, turn);
  return hipGetLastError() == hipSuccess ? HOOK_OK : HOOK_ERR_LAUNCH;
}

}  // namespace
}  // namespace hook

extern "C" hook_status hook_steer_logits(const hook_steer_logits_args* a) {
  using namespace hook;
  if (!a) return HOOK_ERR_NULL;
  if (a->num_rows < 0 || a->vocab < 0 || a->logits_stride < 0 || a->out_stride < 0 || a->history_len < 0 || a->bias_len < 0 || a->num_masks < 0)
    return HOOK_ERR_SHAPE;
  if (a->dtype != HOOK_BF16 && a->dtype != HOOK_F32) return HOOK_ERR_UNSUPPORTED;
  if (a->history_len > (1 << 30) || a->bias_len > (1 << 30)) return HOOK_ERR_UNSUPPORTED;      // (entries are counted on past the end)
  if (a->vocab > (1 << 30)) return HOOK_ERR_UNSUPPORTED;
  if (a->num_rows == 0 || a->vocab == 0) return HOOK_OK;
  const long long stride = a->logits_stride ? a->logits_stride : a->vocab, out_stride = a->out_stride ? a->out_stride : a->vocab;
  if (stride > (1ll << 40) || out_stride > (1ll << 40)) return HOOK_ERR_UNSUPPORTED;
  if (stride < a->vocab || out_stride < a->vocab || (a->out == a->logits && stride != out_stride)) return HOOK_ERR_SHAPE;
  if (!a->logits || !a->out) return HOOK_ERR_NULL;
  if (a->history_len > 0 && (!a->history || !a->cu_history)) return HOOK_ERR_NULL;
  const bool biases = a->bias_len > 0;
  if (biases && (!a->cu_bias || !a->bias_ids || !a->bias_values)) return HOOK_ERR_NULL;
  const uintptr_t esize = a->dtype == HOOK_BF16 ? 2 : 4;
  const uintptr_t from = reinterpret_cast<uintptr_t>(a->logits), to = reinterpret_cast<uintptr_t>(a->out);
  if ((from | to) % esize != 0) return HOOK_ERR_UNSUPPORTED;

  LogitsParams p{};
  p.R = a->num_rows; p.V = a->vocab;
  p.logits = static_cast<const char*>(a->logits); p.out = static_cast<char*>(a->out);
  p.stride = stride * (long long)esize; p.out_stride = out_stride * (long long)esize;
  p.history_len = a->history_len; p.bias_len = a->bias_len; p.masks = a->num_masks; p.words = (a->vocab + 31) / 32;
  p.history = a->history_len > 0 ? a->history : nullptr;
  p.cu_history = a->cu_history; p.prompt_lens = a->prompt_lens;
  p.repetition = a->repetition; p.frequency = a->frequency; p.presence = a->presence;
  p.cu_bias = biases ? a->cu_bias : nullptr; p.bias_ids = a->bias_ids; p.bias_values = a->bias_values;
  p.mask = a->mask; p.mask_rows = a->mask_rows;
  hipStream_t st = static_cast<hipStream_t>(a->stream);
  // Loads of 16 bytes where a row's input and output lie alike to the borders of those, else of one element.  1024 threads of two loads
  // (ranges of 16384 and 8192 tokens) against 256 and 512: 256 x 131072 bf16 36, 49 and 39 us, 128 x 131072 fp32 33, 46 and 38; four
  // rows 6 us with each of them.
  const bool wide = from % 16 == to % 16 && (uintptr_t)stride * esize % 16 == (uintptr_t)out_stride * esize % 16;
  if (esize == 2) return wide ? launch_range<__bf16, 8, 1024, 2>(p, st) : launch_range<__bf16, 1, 512, 16>(p, st);
  return wide ? launch_range<float, 4, 1024, 2>(p, st) : launch_range<float, 1, 512, 8>(p, st);
}
