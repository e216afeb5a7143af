// Rotary positions of queries and keys (up to four axes), and with a cache the write of the rotated keys and of the values
// into its pages.  Per pair (x1, x2) of a head and its angle a:  (x1 cos a - x2 sin a, x2 cos a + x1 sin a).
//
// Bound by memory: every element is read once and written once (keys twice where both outputs are asked for).  The angles
// of a token are the same in all its heads, so a workgroup takes a token, lets one wave compute its cosines and sines
// once into shared memory (a lane per pair) while another finds the token's slot in the cache, and then walks the token's heads
// by units of two vectors of what one load carries: the two halves of as many pairs, or neighbouring pairs in each.  The
// first units are requested before the angles are computed.
// 16384 tokens of 64 query and 8 key and value heads of 128 into the cache: 120 us, 5.9 TB/s (two tokens to a workgroup 123, four 137;
// threads 128 / 512: 127 / 139); 8000 tokens of 32 and 8: 40 us, neighbouring pairs 39, 8-bit cache 45.
#include "../../include/hook_api.h"
#include "kv_write_device.h"

namespace hook {
namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeInFlight = 2;      // units that a thread requests together (one and three: 123 and 122 us)

struct RopeParams {
  int T, Hq, Hk, Hv, d, pairs;        // Hk, Hv: 0 where k is not rotated, or no cache is written
  int axes, axis_pairs[HOOK_ROPE_MAX_AXES], cyclic;
  int q_apart, k_apart;               // the output is not the input
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

template <typename E, int W> struct Vec {
  E e[W];
};

// W elements at an address that is a multiple of 16 bytes (ALIGNED), or of one element alone.
template <typename E, int W, bool ALIGNED> struct RawOf {
  typedef unsigned int type __attribute__((ext_vector_type(sizeof(E) * W / 4), aligned(ALIGNED ? sizeof(E) * W : sizeof(E))));
};

// The first n of W elements (all of them where ALIGNED).
template <typename E, int W, bool ALIGNED>
__device__ __forceinline__ Vec<E, W> load_vec(const char* p, int n) {
  typedef typename RawOf<E, W, ALIGNED>::type Raw;
  Vec<E, W> v;
  if (ALIGNED || n == W) {
    const Raw r = __builtin_nontemporal_load(reinterpret_cast<const Raw*>(p));
    __builtin_memcpy(&v, &r, sizeof v);
  } else {
#pragma unroll
    for (int j = 0; j < W; ++j) v.e[j] = j < n ? reinterpret_cast<const E*>(p)[j] : (E)0.0f;
  }
  return v;
}

template <typename E, int W, bool ALIGNED>
__device__ __forceinline__ void store_vec(char* p, const Vec<E, W>& v, int n) {
  typedef typename RawOf<E, W, ALIGNED>::type Raw;
  if (ALIGNED || n == W) {
    Raw r;
    __builtin_memcpy(&r, &v, sizeof v);
    if (ALIGNED) __builtin_nontemporal_store(r, reinterpret_cast<Raw*>(p));      // (parts of lines are to meet in the cache: 68 us -> 63)
    else *reinterpret_cast<Raw*>(p) = r;
  } else {
#pragma unroll
    for (int j = 0; j < W; ++j)
      if (j < n) reinterpret_cast<E*>(p)[j] = v.e[j];
  }
}

// The same as E4M3 bytes: what the cache write stores for them (kv_write_device.h)
template <typename E, int W, bool ALIGNED>
__device__ __forceinline__ void store_e4m3(char* p, const Vec<E, W>& v, float scale, int n) {
  typedef unsigned int Raw __attribute__((ext_vector_type(W / 4), aligned(ALIGNED ? W : 1)));
  Raw r;
#pragma unroll
  for (int i = 0; i < W / 4; ++i) {
    int four = 0;
    four = __builtin_amdgcn_cvt_pk_fp8_f32(fp8_prescale((float)v.e[4 * i], scale), fp8_prescale((float)v.e[4 * i + 1], scale), four, false);
    four = __builtin_amdgcn_cvt_pk_fp8_f32(fp8_prescale((float)v.e[4 * i + 2], scale), fp8_prescale((float)v.e[4 * i + 3], scale), four, true);
    r[i] = (unsigned)four;
  }
  if (ALIGNED || n == W) {
    *reinterpret_cast<Raw*>(p) = r;
  } else {
#pragma unroll
    for (int j = 0; j < W; ++j)
      if (j < n) p[j] = (char)(r[j / 4] >> (8 * (j % 4)));
  }
}

// Units of a head: the turned pairs, then the rest of it, two vectors at a time.
__host__ __device__ __forceinline__ int vectors_of(int elements, int width) { return (elements + width - 1) / width; }
__host__ __device__ __forceinline__ int units_of(int d, int pairs, int width, bool neighbours) {
  return neighbours ? (vectors_of(d, width) + 1) / 2 : vectors_of(pairs, width) + (vectors_of(d - 2 * pairs, width) + 1) / 2;
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

// ALIGNED: pairs and heads are whole vectors, and every vector lies at a multiple of 16 bytes.  Otherwise vectors lie anywhere (the
// memory takes them at any address) and the last one of the pairs, of what is behind them and of a head may be a part of one.  Such a
// part is moved back to be a whole one, whose first elements another thread computes alike, unless those are turned in place or
// there are not as many (8000 tokens of 32 + 8 heads with 25 pairs into the cache, halves: 62 us, 88 with parts by elements;
// neighbours 51).  What goes to and from memory is the same as with whole vectors (83 + 82 MB without the cache).
template <typename E, int W, bool NEIGHBOURS, bool ALIGNED>
__global__ __launch_bounds__(kRopeThreads) void k_rope(const RopeParams p, int parts) {
  __shared__ float sh_cos[HOOK_ROPE_MAX_DIM / 2], sh_sin[HOOK_ROPE_MAX_DIM / 2];
  __shared__ long long sh_row;        // blk * Hkv * 16 + slot of the token in the cache, or -1
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int t = blockIdx.x / parts, part = blockIdx.x - t * parts;
  const int units = units_of(p.d, p.pairs, W, NEIGHBOURS), value_units = (vectors_of(p.d, W) + 1) / 2;
  const int turning = (p.Hq + p.Hk) * units, total = turning + p.Hv * value_units;

  Vec<E, W> x[kRopeInFlight][2];
  // where unit e of the token lies: head (queries, keys, values in a row), the elements that its two vectors begin with and how many
  // of each there are; c is the first pair of a turned unit of halves
  struct Unit { int h, a, b, n, m; bool turned; };
  auto unit = [&](int e) {
    Unit u;
    u.turned = false;
    bool apart = true;
    int c, lo = 0, half;              // unit of a part of the head that begins at lo and has its second vectors half of them further
    if (e >= turning) {
      u.h = p.Hq + p.Hk + (e - turning) / value_units;
      c = (e - turning) % value_units;
      half = value_units;
    } else {
      u.h = e / units;
      c = e - u.h * units;
      half = units;
      apart = u.h < p.Hq ? p.q_apart : p.k_apart;
      if (!NEIGHBOURS) {
        const int turned = vectors_of(p.pairs, W);
        if (c < turned) {
          u.turned = true;
          u.a = c * W;
          if (!ALIGNED && apart && p.pairs >= W) u.a = min(u.a, p.pairs - W);
          u.b = p.pairs + u.a;
          u.n = u.m = ALIGNED ? W : min(W, p.pairs - u.a);
          return u;
        }
        c -= turned;
        half = units - turned;
        lo = 2 * p.pairs;
      }
    }
    // the vectors lie apart rather than side by side, so that neighbouring lanes load neighbouring vectors
    u.a = lo + c * W;
    u.b = lo + (half + c) * W;
    u.n = ALIGNED ? W : min(W, p.d - u.a);
    u.m = ALIGNED ? (u.b < p.d ? W : 0) : max(0, min(W, p.d - u.b));
    // (neighbouring pairs stay whole only where the head has an even number of elements)
    if (!ALIGNED && apart && p.d - lo >= W && !(NEIGHBOURS && p.d % 2 != 0)) {
      if (u.n < W) { u.a = p.d - W; u.n = W; }
      if (u.m > 0 && u.m < W) { u.b = p.d - W; u.m = W; }
    }
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
      x[i][0] = load_vec<E, W, ALIGNED>(src + (size_t)u.a * sizeof(E), u.n);
      if (u.m > 0) x[i][1] = load_vec<E, W, ALIGNED>(src + (size_t)u.b * sizeof(E), u.m);
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
      // the angle in turns, reduced to [-1/2, 1/2] in fp64: positions of a million still leave 30 bits of it.  What fp32 loses of that goes
      // into the sine and cosine to first order (fp32 outputs 4.0e-8 off 64 bits without, 2.9e-8 with it).
      double turns = (double)p.positions[(size_t)axis * p.T + t] * ((double)p.inv_freq[c] * 0.15915494309189533577);
      turns -= __builtin_rint(turns);
      float sn, cs;
      const float most = (float)turns, rest = 6.2831853f * (float)(turns - (double)most);
      sincospif(2.0f * most, &sn, &cs);
      sh_cos[c] = (cs - sn * rest) * p.magnitude;
      sh_sin[c] = (sn + cs * rest) * p.sign;
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
      if constexpr (NEIGHBOURS) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int at = half == 0 ? u.a : u.b;
          if (value || at >= 2 * p.pairs) continue;
#pragma unroll
          for (int j = 0; j < W; j += 2)
            if (ALIGNED || at + j < 2 * p.pairs) turn(x[i][half].e[j], x[i][half].e[j + 1], (at + j) / 2);
        }
      } else if (u.turned) {
#pragma unroll
        for (int j = 0; j < W; ++j)
          if (ALIGNED || j < u.n) turn(x[i][0].e[j], x[i][1].e[j], u.a + j);
      }
      char* dst = nullptr;
      if (!value && !key) dst = p.q_out + t * p.q_out_stride + (size_t)u.h * p.d * sizeof(E);
      else if (key && p.k_out) dst = p.k_out + t * p.k_out_stride + (size_t)(u.h - p.Hq) * p.d * sizeof(E);
      if (dst) {
        store_vec<E, W, ALIGNED>(dst + (size_t)u.a * sizeof(E), x[i][0], u.n);
        if (u.m > 0) store_vec<E, W, ALIGNED>(dst + (size_t)u.b * sizeof(E), x[i][1], u.m);
      }
      if (p.Hv > 0 && (value || key) && sh_row >= 0) {
        const int g = value ? u.h - p.Hq - p.Hk : u.h - p.Hq;
        const size_t row = (size_t)(sh_row + (long long)g * kBlock) * p.d;
        char* cache = value ? p.v_cache : p.k_cache;
        if (p.kv8) {
          const float scale = value ? p.v_scale[g] : p.k_scale[g];
          store_e4m3<E, W, ALIGNED>(cache + row + u.a, x[i][0], scale, u.n);
          if (u.m > 0) store_e4m3<E, W, ALIGNED>(cache + row + u.b, x[i][1], scale, u.m);
        } else {
          store_vec<E, W, ALIGNED>(cache + (row + u.a) * sizeof(E), x[i][0], u.n);
          if (u.m > 0) store_vec<E, W, ALIGNED>(cache + (row + u.b) * sizeof(E), x[i][1], u.m);
        }
      }
    }
  }
}

// Workgroups to a token.  Few tokens: a token's heads are cut over several of them, one round of units each, to be spread over the chip; many fill it
// with one each, whose angles and slot are then found once.  Cut / whole, launches of a graph on the same tensors, 128 elements into the cache:
//   tokens         64         256        500        600        700        1000         2000
//   32 + 8 heads   3.2 / 3.9  3.8 / 4.2  4.9 / 4.9  5.2 / 5.1  6.1 / 5.1   8.1 / 5.4   13.1 / 9.9  us
//   64 + 8 heads   3.2 / 4.7  4.3 / 5.5  5.9 / 6.0  7.0 / 7.5  8.5 / 7.9  10.5 / 9.3   17.7 / 15.9
// A token of no more units than a workgroup has threads (8 + 1 heads) is not cut on either side.
long long parts_of(const RopeParams& p, int width, bool neighbours) {
  const long long per_token = (long long)(p.Hq + p.Hk) * units_of(p.d, p.pairs, width, neighbours) + (long long)p.Hv * ((vectors_of(p.d, width) + 1) / 2);
  return p.T >= 600 ? 1 : (per_token + kRopeThreads - 1) / kRopeThreads;
}

template <typename E, bool NEIGHBOURS, bool ALIGNED>
hipError_t launch_rope(const RopeParams& p, hipStream_t st) {
  constexpr int W = 16 / sizeof(E);
  const long long parts = parts_of(p, W, NEIGHBOURS);
  hipLaunchKernelGGL((k_rope<E, W, NEIGHBOURS, ALIGNED>), dim3((unsigned)(p.T * parts)), dim3(kRopeThreads), 0, st, p, (int)parts);
  return hipGetLastError();
}

template <typename E>
hipError_t launch_rope(const RopeParams& p, bool neighbours, bool aligned, hipStream_t st) {
  if (neighbours) return aligned ? launch_rope<E, true, true>(p, st) : launch_rope<E, true, false>(p, st);
  return aligned ? launch_rope<E, false, true>(p, st) : launch_rope<E, false, false>(p, st);
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
  p.q_apart = a->q_out != a->q;
  p.k_apart = a->k_out != a->k;
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
  // Whether heads, halves, strides and addresses are all multiples of 16 bytes (of 8 in an 8-bit cache, whose rows take half of that).
  uintptr_t grain = 0;
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
  if (grain % esize != 0) return HOOK_ERR_UNSUPPORTED;
  const bool neighbours = a->layout == HOOK_ROPE_NEIGHBOURS, aligned = grain % 16 == 0;
  // (an upper bound of the units of a token: one to a vector)
  if ((long long)(p.Hq + p.Hk + p.Hv) * (a->head_dim * esize / 16 + 3) > (1 << 27) || !grid_fits(p.T * parts_of(p, 16 / esize, neighbours), kRopeThreads))
    return HOOK_ERR_UNSUPPORTED;
  hipStream_t st = static_cast<hipStream_t>(a->stream);
  const hipError_t e = a->dtype == HOOK_BF16 ? launch_rope<__bf16>(p, neighbours, aligned, st) : launch_rope<float>(p, neighbours, aligned, st);
  return e == hipSuccess ? HOOK_OK : HOOK_ERR_LAUNCH;
}
