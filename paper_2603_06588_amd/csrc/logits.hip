// Penalties for repeated tokens, a bias list and a grammar mask on rows of logits.
//
// Bound by memory: a row is read once and written once.  A workgroup takes a range of one row's tokens.  It counts the row's
// history into shared memory, one word per token of the range (bit 31: in the prompt; below: occurrences among the generated
// tokens), notes the last bias entry of each token in a second word where there are biases, and then passes over
// the range once.  All counts are whole numbers and the last entry is a maximum, so the order of the atomics changes nothing.
// The logits are requested before the history is counted, so the trips to memory overlap.
#include "../../include/hook_api.h"
#include "hook_device.h"

namespace hook {
namespace {

constexpr unsigned kInPrompt = 0x80000000u;

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

// W: elements of a load.  Each of the NT threads takes VPT loads of the range; the i-th of thread t starts at element
// (i * NT + t) * W of it.
template <typename E, int W, int NT, int VPT, bool BIAS>
__global__ __launch_bounds__(NT) void k_steer_logits(const LogitsParams p, int ranges) {
  typedef typename RawOf<sizeof(E) * W>::type Raw;
  constexpr int kRange = NT * VPT * W;
  __shared__ unsigned count[kRange];
  __shared__ int biased[BIAS ? kRange : 1];
  const int tid = threadIdx.x, row = blockIdx.x / ranges, r0 = (blockIdx.x - row * ranges) * kRange;
  const char* const in = p.logits + row * p.stride;
  char* const out = p.out + row * p.out_stride;
  Raw raw[VPT];
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int e = r0 + (i * NT + tid) * W;
    if (e + W <= p.V) raw[i] = __builtin_nontemporal_load(reinterpret_cast<const Raw*>(in + (size_t)e * sizeof(E)));
  }
  // bits of the loads' tokens
  const int m = p.mask ? (p.mask_rows ? p.mask_rows[row] : row) : -1;
  const bool masked = m >= 0 && m < p.masks;
  unsigned allowed[VPT];
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int e = r0 + (i * NT + tid) * W;
    allowed[i] = 0xFFFFFFFFu;
    if (masked && e < p.V) allowed[i] = p.mask[(size_t)m * p.words + (e >> 5)] >> (e & 31);
  }
  const float rep = p.repetition ? p.repetition[row] : 1.0f, freq = p.frequency ? p.frequency[row] : 0.0f;
  const float pres = p.presence ? p.presence[row] : 0.0f;
  const bool counts = p.history != nullptr && (rep != 1.0f || freq != 0.0f || pres != 0.0f);

  for (int i = tid; i < kRange; i += NT) {
    count[i] = 0;
    if (BIAS) biased[i] = 0;
  }
  __syncthreads();
  if (counts) {
    int begin, end;
    list_of(p.cu_history, row, p.history_len, &begin, &end);
    const int generated = begin + (p.prompt_lens ? min(max(p.prompt_lens[row], 0), end - begin) : 0);
    for (int j = begin + tid; j < end; j += NT) {
      const unsigned at = (unsigned)p.history[j] - (unsigned)r0;
      if (at < (unsigned)kRange) {
        if (j < generated) atomicOr(&count[at], kInPrompt);
        else atomicAdd(&count[at], 1u);
      }
    }
  }
  int bias0 = 0;
  if (BIAS) {
    int end;
    list_of(p.cu_bias, row, p.bias_len, &bias0, &end);
    for (int j = bias0 + tid; j < end; j += NT) {
      const unsigned at = (unsigned)p.bias_ids[j] - (unsigned)r0;
      if (at < (unsigned)kRange) atomicMax(&biased[at], j - bias0 + 1);
    }
  }
  __syncthreads();

  auto adjusted = [&](E logit, int at, bool barred) {
    const unsigned c = count[at];
    const int b = BIAS ? biased[at] : 0;
    if (c == 0 && b == 0 && !barred) return logit;
    float x = (float)logit;
    if (c != 0) {
      x = x > 0.0f ? x / rep : x * rep;
      const unsigned n = c & ~kInPrompt;
      if (n != 0) x = (x - (float)n * freq) - pres;
    }
    if (b != 0) x += p.bias_values[bias0 + b - 1];
    return (E)(barred ? -__builtin_inff() : x);
  };
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int at = (i * NT + tid) * W, e = r0 + at;
    if (e + W <= p.V) {
      Vec<E, W> v;
      __builtin_memcpy(&v, &raw[i], sizeof v);
#pragma unroll
      for (int u = 0; u < W; ++u) v.e[u] = adjusted(v.e[u], at + u, ((allowed[i] >> u) & 1u) == 0);
      Raw r;
      __builtin_memcpy(&r, &v, sizeof r);
      __builtin_nontemporal_store(r, reinterpret_cast<Raw*>(out + (size_t)e * sizeof(E)));
    } else {
      for (int u = 0; e + u < p.V; ++u)      // the row's last tokens, fewer than a load
        reinterpret_cast<E*>(out)[e + u] = adjusted(reinterpret_cast<const E*>(in)[e + u], at + u, ((allowed[i] >> u) & 1u) == 0);
    }
  }
}

template <typename E, int W, int NT, int VPT>
hipError_t launch_range(const LogitsParams& p, hipStream_t st) {
  const int ranges = (p.V + NT * VPT * W - 1) / (NT * VPT * W);
  const dim3 grid((unsigned)(p.R * ranges));
  if (p.cu_bias) hipLaunchKernelGGL((k_steer_logits<E, W, NT, VPT, true>), grid, dim3(NT), 0, st, p, ranges);
  else hipLaunchKernelGGL((k_steer_logits<E, W, NT, VPT, false>), grid, dim3(NT), 0, st, p, ranges);
  return hipGetLastError();
}

}  // namespace
}  // namespace hook

extern "C" hook_status hook_steer_logits(const hook_steer_logits_args* a) {
  using namespace hook;
  if (!a) return HOOK_ERR_NULL;
  if (a->num_rows < 0 || a->vocab < 0 || a->logits_stride < 0 || a->out_stride < 0 || a->history_len < 0 || a->bias_len < 0 || a->num_masks < 0)
    return HOOK_ERR_SHAPE;
  if (a->dtype != HOOK_BF16 && a->dtype != HOOK_F32) return HOOK_ERR_UNSUPPORTED;
  if (a->vocab > (1 << 30) || !grid_fits((long long)a->num_rows * (a->vocab / 4096 + 1))) return HOOK_ERR_UNSUPPORTED;
  if (a->num_rows == 0 || a->vocab == 0) return HOOK_OK;
  const long long stride = a->logits_stride ? a->logits_stride : a->vocab, out_stride = a->out_stride ? a->out_stride : a->vocab;
  if (stride < a->vocab || out_stride < a->vocab || (a->out == a->logits && stride != out_stride)) return HOOK_ERR_SHAPE;
  if (!a->logits || !a->out) return HOOK_ERR_NULL;
  if (a->history_len > 0 && (!a->history || !a->cu_history)) return HOOK_ERR_NULL;
  const bool biases = a->bias_len > 0;
  if (biases && (!a->cu_bias || !a->bias_ids || !a->bias_values)) return HOOK_ERR_NULL;
  const uintptr_t esize = a->dtype == HOOK_BF16 ? 2 : 4;
  const uintptr_t grain = reinterpret_cast<uintptr_t>(a->logits) | reinterpret_cast<uintptr_t>(a->out) | (uintptr_t)stride * esize | (uintptr_t)out_stride * esize;
  if (grain % esize != 0) return HOOK_ERR_UNSUPPORTED;

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
  const bool wide = grain % 16 == 0;
  hipError_t e;
  if (esize == 2) e = wide ? launch_range<__bf16, 8, 256, 2>(p, st) : launch_range<__bf16, 1, 256, 16>(p, st);
  else e = wide ? launch_range<float, 4, 256, 4>(p, st) : launch_range<float, 1, 256, 16>(p, st);
  return e == hipSuccess ? HOOK_OK : HOOK_ERR_LAUNCH;
}
