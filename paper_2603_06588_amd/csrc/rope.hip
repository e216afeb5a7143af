// Rotary positions of queries and keys (up to four axes), and with a cache the write of the rotated keys and of the values
// into its pages.  Per pair (x1, x2) of a head and its angle a:  (x1 cos a - x2 sin a, x2 cos a + x1 sin a).
//
// Bound by memory: every element is read once and written once (keys twice where both outputs are asked for).  The angles
// of a token are the same in all its heads, so a workgroup takes a token, lets one wave compute its cosines and sines
// once into shared memory (a lane per pair) while another finds the token's slot in the cache, and then walks the token's heads
// by units of two vectors of what one load carries: the two halves of as many pairs, or neighbouring pairs in each.  The
// first units are requested before the angles are computed.
// 16384 tokens of 64 query and 8 key and value heads of 128 into the cache: 120 us, 5.9 TB/s (two tokens to a workgroup 123, four 137;
// threads 128 / 512: 127 / 139); 8000 tokens of 32 and 8: 40 us, neighbouring pairs 39, 8-bit cache 43.
#include "../../include/hook_api.h"
#include "kv_write_device.h"

namespace hook {
namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeInFlight = 2;      // units that a thread requests together (one and three: 123 and 122 us)

struct RopeParams {
  int T, Hq, Hk, Hv, d, pairs;        // Hk, Hv: 0 where k is not rotated, or no cache is written
  int axes, axis_pairs[HOOK_ROPE_MAX_AXES], cyclic;
  float magnitude, sign;
  const int* positions;
  const float* inv_freq;
  const char *q, *k, *v;
  char *q_out, *k_out;
  long long q_stride, k_stride, v_stride, q_out_stride, k_out_stride;   // bytes
  // the cache
  int num_seqs, max_blocks, num_blocks, kv8;
  const int *block_table, *seq_lens, *cu;
  char *k_cache, *v_cache;
  const float *k_scale, *v_scale;
};

template <int BYTES> struct RawOf;
template <> struct RawOf<16> { typedef u32x4 type; };
template <> struct RawOf<8> { typedef u32x2 type; };
template <> struct RawOf<4> { typedef unsigned int type; };
template <> struct RawOf<2> { typedef unsigned short type; };
template <> struct RawOf<1> { typedef unsigned char type; };

template <typename E, int W> struct Vec {
  E e[W];
};

template <typename E, int W>
__device__ __forceinline__ Vec<E, W> load_vec(const char* p) {
  typedef typename RawOf<sizeof(E) * W>::type Raw;
  const Raw r = __builtin_nontemporal_load(reinterpret_cast<const Raw*>(p));
  Vec<E, W> v;
  __builtin_memcpy(&v, &r, sizeof v);
  return v;
}

template <typename E, int W>
__device__ __forceinline__ void store_vec(char* p, const Vec<E, W>& v) {
  typedef typename RawOf<sizeof(E) * W>::type Raw;
  Raw r;
  __builtin_memcpy(&r, &v, sizeof r);
  __builtin_nontemporal_store(r, reinterpret_cast<Raw*>(p));
}

// W values as E4M3 bytes: what the cache write stores for them (kv_write_device.h)
template <typename E, int W>
__device__ __forceinline__ void store_e4m3(char* p, const Vec<E, W>& v, float scale) {
  Vec<unsigned char, W> b;
#pragma unroll
  for (int i = 0; i < W; i += 2) {
    const float lo = fp8_prescale((float)v.e[i], scale), hi = W > 1 ? fp8_prescale((float)v.e[W > 1 ? i + 1 : 0], scale) : 0.0f;
    const int two = __builtin_amdgcn_cvt_pk_fp8_f32(lo, hi, 0, false);
    b.e[i] = (unsigned char)(two & 0xFF);
    if constexpr (W > 1) b.e[i + 1] = (unsigned char)((two >> 8) & 0xFF);
  }
  typedef typename RawOf<W>::type Raw;
  Raw r;
  __builtin_memcpy(&r, &b, sizeof r);
  *reinterpret_cast<Raw*>(p) = r;
}

// Largest i in [0, n) with cu[i] <= row, by all lanes of a wave: each trip to memory leaves one 64th of the sequences.
__device__ __forceinline__ int find_sequence(const int* cu, int n, int row, int lane) {
  int lo = 0;
  while (n > 1) {
    const int stride = (n + 63) >> 6, i = lane * stride;
    const unsigned long long below = __ballot(i < n && cu[lo + min(i, n - 1)] <= row);
    const int k = max(__popcll(below) - 1, 0);
    lo += k * stride;
    n = min(stride, n - k * stride);
  }
  return lo;
}

template <typename E, int W, bool NEIGHBOURS>
__global__ __launch_bounds__(kRopeThreads) void k_rope(const RopeParams p, int parts) {
  __shared__ float sh_cos[HOOK_ROPE_MAX_DIM / 2], sh_sin[HOOK_ROPE_MAX_DIM / 2];
  __shared__ long long sh_row;        // blk * Hkv * 16 + slot of the token in the cache, or -1
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int t = blockIdx.x / parts, part = blockIdx.x - t * parts;
  const int units = (p.d + 2 * W - 1) / (2 * W);                // of a head: the turned ones, then the rest of it
  const int total = (p.Hq + p.Hk + p.Hv) * units;
  const int turned = p.pairs / W;

  Vec<E, W> x[kRopeInFlight][2];
  // where unit e of the token lies: head (queries, keys, values in a row) and the elements of its two vectors
  struct Unit { int h, a, b; };                                 // b < 0: the head ends inside the unit
  auto unit = [&](int e) {
    Unit u;
    u.h = e / units;
    const int c = e - u.h * units;
    // the unit's vectors lie apart rather than side by side, so that neighbouring lanes load neighbouring vectors
    if (NEIGHBOURS && W == 1 && u.h < p.Hq + p.Hk) {
      u.a = 2 * c;
      u.b = u.a + 1;
    } else if (NEIGHBOURS || u.h >= p.Hq + p.Hk) {
      u.a = c * W;
      u.b = (units + c) * W;
    } else if (c < turned) {
      u.a = c * W;
      u.b = p.pairs + c * W;
    } else {                                                    // behind both halves
      u.a = (turned + c) * W;
      u.b = (units + c) * W;
    }
    if (u.b + W > p.d) u.b = -1;
    return u;
  };
  auto request = [&](int e0) {
#pragma unroll
    for (int i = 0; i < kRopeInFlight; ++i) {
      const int e = e0 + i * kRopeThreads * parts;
      if (e >= total) break;
      const Unit u = unit(e);
      const char* src;
      if (u.h < p.Hq) src = p.q + t * p.q_stride + (size_t)u.h * p.d * sizeof(E);
      else if (u.h < p.Hq + p.Hk) src = p.k + t * p.k_stride + (size_t)(u.h - p.Hq) * p.d * sizeof(E);
      else src = p.v + t * p.v_stride + (size_t)(u.h - p.Hq - p.Hk) * p.d * sizeof(E);
      x[i][0] = load_vec<E, W>(src + (size_t)u.a * sizeof(E));
      if (u.b >= 0) x[i][1] = load_vec<E, W>(src + (size_t)u.b * sizeof(E));
    }
  };
  const int first = part * kRopeThreads + tid;
  request(first);

  if (wave == 0) {
    for (int c = lane; c < p.pairs; c += 64) {
      int axis = 0;
      if (p.cyclic) {
        const int a = c % p.axes;
        axis = c / p.axes < p.axis_pairs[a] ? a : 0;
      } else {
        for (int a = 0, end = 0; a + 1 < p.axes; ++a) {
          end += p.axis_pairs[a];
          if (c >= end) axis = a + 1;
        }
      }
      // the angle in half turns, reduced to [-1, 1] in fp64: positions of a million still leave 30 bits of it
      double turns = (double)p.positions[(size_t)axis * p.T + t] * ((double)p.inv_freq[c] * 0.15915494309189533577);
      turns -= __builtin_rint(turns);
      float sn, cs;
      sincospif(2.0f * (float)turns, &sn, &cs);
      sh_cos[c] = cs * p.magnitude;
      sh_sin[c] = sn * p.sign;
    }
  } else if (wave == 1 && p.Hv > 0) {
    const int i = find_sequence(p.cu, p.num_seqs, t, lane);
    if (lane == 0) {
      const int begin = p.cu[i], n = p.cu[i + 1] - begin, L = p.seq_lens[i], at = t - begin;
      long long r = -1;
      if (begin >= 0 && at >= 0 && at < n && n <= L) {
        const int pos = L - n + at;
        if ((pos >> 4) < p.max_blocks) {
          const int blk = p.block_table[(size_t)i * p.max_blocks + (pos >> 4)];
          if ((unsigned)blk < (unsigned)p.num_blocks) r = (long long)blk * p.Hv * kBlock + (pos & 15);
        }
      }
      sh_row = r;
    }
  }
  __syncthreads();

  for (int e0 = first; e0 < total; e0 += kRopeInFlight * kRopeThreads * parts) {
    if (e0 != first) request(e0);
#pragma unroll
    for (int i = 0; i < kRopeInFlight; ++i) {
      const int e = e0 + i * kRopeThreads * parts;
      if (e >= total) break;
      const Unit u = unit(e);
      const bool value = u.h >= p.Hq + p.Hk, key = !value && u.h >= p.Hq;
      auto turn = [&](E& lo, E& hi, int c) {
        const float a = (float)lo, b = (float)hi, cs = sh_cos[c], sn = sh_sin[c];
        lo = (E)(a * cs - b * sn);
        hi = (E)(b * cs + a * sn);
      };
      if (!value) {
        if constexpr (NEIGHBOURS && W > 1) {
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const int at = half == 0 ? u.a : u.b;
            if (at < 0 || at >= 2 * p.pairs) continue;
#pragma unroll
            for (int j = 0; j < W; j += 2) turn(x[i][half].e[j], x[i][half].e[j + 1], (at + j) / 2);
          }
        } else if (NEIGHBOURS ? u.a < 2 * p.pairs : u.a < p.pairs) {
#pragma unroll
          for (int j = 0; j < W; ++j) turn(x[i][0].e[j], x[i][1].e[j], NEIGHBOURS ? u.a / 2 : u.a + j);
        }
      }
      char* dst = nullptr;
      if (!value && !key) dst = p.q_out + t * p.q_out_stride + (size_t)u.h * p.d * sizeof(E);
      else if (key && p.k_out) dst = p.k_out + t * p.k_out_stride + (size_t)(u.h - p.Hq) * p.d * sizeof(E);
      if (dst) {
        store_vec<E, W>(dst + (size_t)u.a * sizeof(E), x[i][0]);
        if (u.b >= 0) store_vec<E, W>(dst + (size_t)u.b * sizeof(E), x[i][1]);
      }
      if (p.Hv > 0 && (value || key) && sh_row >= 0) {
        const int g = value ? u.h - p.Hq - p.Hk : u.h - p.Hq;
        const size_t row = (size_t)(sh_row + (long long)g * kBlock) * p.d;
        char* cache = value ? p.v_cache : p.k_cache;
        if (p.kv8) {
          const float scale = value ? p.v_scale[g] : p.k_scale[g];
          store_e4m3<E, W>(cache + row + u.a, x[i][0], scale);
          if (u.b >= 0) store_e4m3<E, W>(cache + row + u.b, x[i][1], scale);
        } else {
          store_vec<E, W>(cache + (row + u.a) * sizeof(E), x[i][0]);
          if (u.b >= 0) store_vec<E, W>(cache + (row + u.b) * sizeof(E), x[i][1]);
        }
      }
    }
  }
}

template <typename E, int W, bool NEIGHBOURS>
hipError_t launch_width(const RopeParams& p, hipStream_t st) {
  const int units = (p.d + 2 * W - 1) / (2 * W);
  const long long per_token = (long long)(p.Hq + p.Hk + p.Hv) * units;
  // Few tokens: a token's heads are cut over several workgroups, one round of units each, to be spread over the chip (2000 tokens of 32 and
  // 8 heads 14.8 us so, 12.0 with a workgroup each; 1000 tokens 8.5 with either, where the launch counts).
  const int parts = p.T >= 600 ? 1 : (int)((per_token + kRopeThreads - 1) / kRopeThreads);
  hipLaunchKernelGGL((k_rope<E, W, NEIGHBOURS>), dim3((unsigned)(p.T * parts)), dim3(kRopeThreads), 0, st, p, parts);
  return hipGetLastError();
}

template <typename E, bool NEIGHBOURS>
hipError_t launch_rope(const RopeParams& p, int width, hipStream_t st) {
  if constexpr (sizeof(E) == 2)
    if (width == 8) return launch_width<E, 8, NEIGHBOURS>(p, st);
  if (width >= 4) return launch_width<E, 4, NEIGHBOURS>(p, st);
  if (width == 2) return launch_width<E, 2, NEIGHBOURS>(p, st);
  return launch_width<E, 1, NEIGHBOURS>(p, st);
}

}  // namespace
}  // namespace hook

extern "C" hook_status hook_rope(const hook_rope_args* a) {
  using namespace hook;
  if (!a) return HOOK_ERR_NULL;
  if (a->num_tokens < 0 || a->num_q_heads < 0 || a->num_kv_heads < 0 || a->head_dim <= 0 || a->rotary_dim < 0 ||
      a->rotary_dim > a->head_dim || a->q_stride < 0 || a->k_stride < 0 || a->v_stride < 0 || a->q_out_stride < 0 || a->k_out_stride < 0)
    return HOOK_ERR_SHAPE;
  if (a->dtype != HOOK_BF16 && a->dtype != HOOK_F32) return HOOK_ERR_UNSUPPORTED;
  if (a->head_dim > HOOK_ROPE_MAX_DIM || a->rotary_dim % 2 != 0 || a->num_q_heads > 65536 || a->num_kv_heads > 65536 || a->num_tokens > (1 << 30)) return HOOK_ERR_UNSUPPORTED;
  if (a->layout != HOOK_ROPE_HALVES && a->layout != HOOK_ROPE_NEIGHBOURS) return HOOK_ERR_SHAPE;
  if (a->axis_order != HOOK_ROPE_BLOCKED && a->axis_order != HOOK_ROPE_CYCLIC) return HOOK_ERR_SHAPE;
  if (a->num_axes < 1 || a->num_axes > HOOK_ROPE_MAX_AXES) return HOOK_ERR_SHAPE;
  const int pairs = a->rotary_dim / 2;
  long long sum = 0;
  for (int i = 0; i < a->num_axes; ++i) {
    const int n = a->axis_pairs[i];
    if (n < 0) return HOOK_ERR_SHAPE;
    if (a->axis_order == HOOK_ROPE_CYCLIC && i > 0 && n > 0 && i + (long long)a->num_axes * (n - 1) >= pairs) return HOOK_ERR_SHAPE;
    sum += n;
  }
  if (sum != pairs) return HOOK_ERR_SHAPE;
  const bool cache = a->k_cache != nullptr || a->v_cache != nullptr;
  const int esize = a->dtype == HOOK_BF16 ? 2 : 4;
  const bool has_q = a->q != nullptr && a->num_q_heads > 0, has_k = a->k != nullptr && a->num_kv_heads > 0;
  const long long qw = (long long)a->num_q_heads * a->head_dim, kw = (long long)a->num_kv_heads * a->head_dim;
  auto stride = [](int64_t given, long long width) { return given ? (long long)given : width; };
  const long long qs = stride(a->q_stride, qw), ks = stride(a->k_stride, kw), vs = stride(a->v_stride, kw);
  const long long qos = stride(a->q_out_stride, qw), kos = stride(a->k_out_stride, kw);
  for (long long x : {qs, ks, vs, qos, kos})
    if (x > (1ll << 40)) return HOOK_ERR_UNSUPPORTED;
  if ((has_q && (qs < qw || qos < qw)) || (has_k && (ks < kw || kos < kw)) || (cache && vs < kw)) return HOOK_ERR_SHAPE;
  if ((has_q && a->q_out == a->q && qs != qos) || (has_k && a->k_out == a->k && ks != kos)) return HOOK_ERR_SHAPE;
  bool kv8 = false;
  if (cache) {
    if (a->num_seqs < 0 || a->max_blocks_per_seq <= 0 || a->num_blocks <= 0) return HOOK_ERR_SHAPE;
    if (a->kv_dtype != HOOK_KV_SAME && a->kv_dtype != HOOK_KV_FP8_E4M3) return HOOK_ERR_SHAPE;
    kv8 = a->kv_dtype == HOOK_KV_FP8_E4M3;
    if (a->block_size != HOOK_BLOCK_SIZE || (kv8 && a->dtype != HOOK_BF16) || a->max_blocks_per_seq > (1 << 26)) return HOOK_ERR_UNSUPPORTED;
  }
  if (a->num_tokens == 0 || (!has_q && !has_k && !cache)) return HOOK_OK;
  if (has_q && !a->q_out) return HOOK_ERR_NULL;
  if (has_k && !a->k_out && !cache) return HOOK_ERR_NULL;
  if (pairs > 0 && (!a->positions || !a->inv_freq)) return HOOK_ERR_NULL;
  if (cache) {
    if (!has_k || !a->v || !a->k_cache || !a->v_cache || !a->block_table || !a->seq_lens || !a->cu_q_lens) return HOOK_ERR_NULL;
    if (kv8 && (!a->k_scale || !a->v_scale)) return HOOK_ERR_NULL;
    if (a->num_seqs == 0) return HOOK_ERR_SHAPE;      // tokens of no sequence
  }

  RopeParams p{};
  p.T = a->num_tokens;
  p.Hq = has_q ? a->num_q_heads : 0;
  p.Hk = has_k ? a->num_kv_heads : 0;
  p.Hv = cache ? a->num_kv_heads : 0;
  p.d = a->head_dim;
  p.pairs = pairs;
  p.axes = a->num_axes;
  for (int i = 0; i < a->num_axes; ++i) p.axis_pairs[i] = a->axis_pairs[i];
  p.cyclic = a->axis_order == HOOK_ROPE_CYCLIC;
  p.magnitude = a->magnitude != 0.0f ? a->magnitude : 1.0f;
  p.sign = a->inverse ? -p.magnitude : p.magnitude;
  p.positions = a->positions;
  p.inv_freq = a->inv_freq;
  p.q = static_cast<const char*>(a->q);
  p.k = static_cast<const char*>(a->k);
  p.v = static_cast<const char*>(a->v);
  p.q_out = static_cast<char*>(a->q_out);
  p.k_out = static_cast<char*>(a->k_out);
  p.q_stride = qs * esize; p.k_stride = ks * esize; p.v_stride = vs * esize;
  p.q_out_stride = qos * esize; p.k_out_stride = kos * esize;
  if (cache) {
    p.num_seqs = a->num_seqs; p.max_blocks = a->max_blocks_per_seq; p.num_blocks = a->num_blocks; p.kv8 = kv8 ? 1 : 0;
    p.block_table = a->block_table; p.seq_lens = a->seq_lens; p.cu = a->cu_q_lens;
    p.k_cache = static_cast<char*>(a->k_cache); p.v_cache = static_cast<char*>(a->v_cache);
    p.k_scale = a->k_scale; p.v_scale = a->v_scale;
  }
  // Elements that one load carries: the largest power of two, up to 16 bytes, that divides heads, pairs, strides and addresses
  // (an 8-bit cache's rows are addressed by single bytes, so by elements).
  uintptr_t grain = 16;
  auto divides = [&](uintptr_t bytes) { grain |= bytes; };
  divides((uintptr_t)a->head_dim * esize);
  divides((uintptr_t)pairs * esize);
  if (has_q) { divides((uintptr_t)a->q); divides((uintptr_t)a->q_out); divides((uintptr_t)p.q_stride); divides((uintptr_t)p.q_out_stride); }
  if (has_k) {
    divides((uintptr_t)a->k);
    divides((uintptr_t)p.k_stride);
    if (a->k_out) { divides((uintptr_t)a->k_out); divides((uintptr_t)p.k_out_stride); }
  }
  if (cache) {
    divides((uintptr_t)a->v);
    divides((uintptr_t)p.v_stride);
    divides((uintptr_t)a->k_cache * (kv8 ? 2 : 1));
    divides((uintptr_t)a->v_cache * (kv8 ? 2 : 1));
  }
  const int bytes = (int)(grain & (~grain + 1));
  if (bytes < esize) return HOOK_ERR_UNSUPPORTED;
  const int width = bytes / esize;
  const long long units = (a->head_dim + 2 * width - 1) / (2 * width), per_token = (p.Hq + p.Hk + p.Hv) * units;
  if (per_token > (1 << 27) || !grid_fits((per_token / kRopeThreads + 1) * p.T)) return HOOK_ERR_UNSUPPORTED;
  hipStream_t st = static_cast<hipStream_t>(a->stream);
  const bool nb = a->layout == HOOK_ROPE_NEIGHBOURS;
  const hipError_t e = a->dtype == HOOK_BF16 ? (nb ? launch_rope<__bf16, true>(p, width, st) : launch_rope<__bf16, false>(p, width, st))
                                             : (nb ? launch_rope<float, true>(p, width, st) : launch_rope<float, false>(p, width, st));
  return e == hipSuccess ? HOOK_OK : HOOK_ERR_LAUNCH;
}
