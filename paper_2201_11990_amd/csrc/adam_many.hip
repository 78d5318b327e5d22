// The optimizer step over many tensors at once, with the moments in fp32 or in 8 bits, and the squared norm of all their gradients.
//
// A model's parameters are a few large tensors and many small ones (gains, biases), and a launch for each is what the small ones cost.
// Here the addresses and sizes of up to kStepTensors tensors travel in the launch's arguments (no table in device memory, nothing to copy before the
// call), every tensor is cut into chunks of 4096 elements, and a workgroup finds its chunk's tensor with a ballot over where they begin.
//
// States in 8 bits: e4m3 codes of m and of r = sqrt(v), with one fp32 scale each to a block of 256 elements, which is what a wave takes at 4
// elements a lane, so that a block's largest magnitude is one reduction over the wave.  r and not v: a code's range (2^-9 .. 448 times the scale) then spans
// 10 decades of v, and a step is at most 1/8 of r as it is of m.  Codes are rounded up with the probability of the part of a step that is left: rounded to
// nearest, a moment whose change in a step is below half a code (beta2 = 0.95 takes 5 % of v, 2.5 % of r; a code is 6 to 12 % wide) would never move.
// The mean of r is kept, that of r^2 is not: larger by r's variance, which is at most (a code's step d) (the change of r) while that is less than a step, so v settles at most
// d / r E|g^2 / v - 1| / 2 too high for the gradients, and as much again for a scale that moves: 1/8 (0.97 + 1) / 2 = 12.5 % at most for
// normally distributed gradients and roots of a code's full precision (above 2^-14 of their block's largest).  Measured, even and uneven blocks: 2.6 and 2.2 % at
// beta2 = 0.95, 4.8 and 4.7 at 0.99, 5.5 and 5.8 at 0.999; steps are 0.7 to 1.3 % short.  Rounding r up by the odds of squares would keep v's mean and lose r's, which is what an update divides by.
//
// Both are bound by HBM: 122 M parameters in fp32 (30 bytes each) 620 us, 5.9 TB/s; 243 M in 8 bits with bf16 gradients (16 bytes) 660 us, 5.9 TB/s; their norms 75 and 77 us,
// 6.4 and 6.3 TB/s (a copy of 2 GiB: 4.7 to 4.9 TB/s without the hint that goes past the caches).
#include <algorithm>
#include <new>
#include <type_traits>

#include "adam.h"

namespace mtnlg {

namespace {

constexpr int kBlock = 256;                // elements that share a scale
constexpr int kChunk = 4096;               // elements of a workgroup's turn: 4 vectors of 4 a thread
constexpr int kTurns = kChunk / 1024;
constexpr int kStepTensors = 56, kNormTensors = 160;   // per launch: what 4 KB of arguments hold
constexpr int kNormBlocks = 2048;          // partial sums at most
constexpr uint32_t kOnce = 32;             // chunks up to which one workgroup takes all, two to a wave
constexpr int32_t kMostTensors = 1 << 16;

struct StepTensor {
  float *p;
  void *m, *v;
  float *m_scale, *v_scale;
  const void *g;
  bf16 *w;
  int64_t count_decay;                 // twice the count, and whether weight decay applies
  uint32_t first_chunk, first_block;   // of this launch; of the call
  __host__ __device__ __forceinline__ int64_t count() const { return count_decay >> 1; }
};
struct StepArgs {
  AdamArgs a;
  uint32_t key_lo, key_hi, chunks;
  int32_t tensors;
  const float *sqnorm;
  StepTensor of[kStepTensors];
};
static_assert(sizeof(StepArgs) <= 4096, "arguments of a launch");

struct NormTensor {
  const void *g;
  int64_t count;
  uint32_t first_chunk, pad;
};
struct NormArgs {
  uint32_t chunks;
  int32_t tensors;
  NormTensor of[kNormTensors];
};
static_assert(sizeof(NormArgs) + 32 <= 4096, "arguments of a launch");

// Few chunks, each named on the host: a wave's first wait is for its own entry
struct NormChunk {
  const void *g;
  int64_t count;   // elements from g on, at most kChunk
};
struct NormOnceArgs {
  uint32_t chunks;
  NormChunk of[kOnce];
};

// the tensor that chunk c is of: the last one that begins at it or before.  Every lane looks at some of the tensors: one load's latency, where a
// binary search through 64 of them waits for six
template <int MOST, typename A>
__device__ __forceinline__ int tensor_of(const A &a, uint32_t c) {
  const int lane = threadIdx.x & 63;
  int n = 0;
#pragma unroll
  for (int i = 0; i < MOST; i += 64) {
    const int k = i + lane < MOST ? i + lane : MOST - 1;
    n += __builtin_popcountll(__builtin_amdgcn_ballot_w64(i + lane < a.tensors && a.of[k].first_chunk <= c));
  }
  return __builtin_amdgcn_readfirstlane(n - 1);
}

// What passes once goes past the caches: reading 500 MB without the hint reached 5.7 TB/s, with it 6.9.
typedef __attribute__((ext_vector_type(4))) short i16x4;
template <typename E>
__device__ __forceinline__ f32x4 stream4(const E *p) {
  if constexpr (sizeof(E) == 4) {
    return __builtin_nontemporal_load(reinterpret_cast<const f32x4 *>(p));
  } else {
    const bf16x4 t = __builtin_bit_cast(bf16x4, __builtin_nontemporal_load(reinterpret_cast<const i16x4 *>(p)));
    return f32x4{(float)t[0], (float)t[1], (float)t[2], (float)t[3]};
  }
}
// elements i .. i + 3 of n (zeros beyond), aligned for one access; WHOLE: all of them are there
template <bool WHOLE, typename E>
__device__ __forceinline__ f32x4 load_some(const E *p, int64_t i, int64_t n) {
  if (WHOLE || i + 4 <= n) return stream4(p + i);
  f32x4 r = {};
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (i + e < n) r[e] = to_f32(p[i + e]);
  return r;
}
template <bool WHOLE, typename E>
__device__ __forceinline__ void store_some(E *p, int64_t i, int64_t n, f32x4 x) {
  if (WHOLE || i + 4 <= n) {
    if constexpr (sizeof(E) == 4) __builtin_nontemporal_store(x, reinterpret_cast<f32x4 *>(p + i));
    else __builtin_nontemporal_store(__builtin_bit_cast(i16x4, (bf16x4{(bf16)x[0], (bf16)x[1], (bf16)x[2], (bf16)x[3]})), reinterpret_cast<i16x4 *>(p + i));
    return;
  }
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (i + e < n) p[i + e] = from_f32<E>(x[e]);
}
// four codes
template <bool WHOLE>
__device__ __forceinline__ uint32_t load_codes(const uint8_t *p, int64_t i, int64_t n) {
  if (WHOLE || i + 4 <= n) return __builtin_nontemporal_load(reinterpret_cast<const uint32_t *>(p + i));
  uint32_t r = 0;
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (i + e < n) r |= (uint32_t)p[i + e] << (8 * e);
  return r;
}
template <bool WHOLE>
__device__ __forceinline__ void store_codes(uint8_t *p, int64_t i, int64_t n, uint32_t x) {
  if (WHOLE || i + 4 <= n) {
    __builtin_nontemporal_store(x, reinterpret_cast<uint32_t *>(p + i));
    return;
  }
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (i + e < n) p[i + e] = (uint8_t)(x >> (8 * e));
}
__device__ __forceinline__ f32x4 decode(uint32_t codes) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
  return f32x4{lo[0], lo[1], hi[0], hi[1]};
}

// 32 random bits for element e of a block: products, shifts and exclusive ors on the step's two words, the block's number and e.
__device__ __forceinline__ uint32_t block_key(uint32_t block, uint32_t lo, uint32_t hi) {
  uint32_t k = block * 0x9E3779B1u + lo;
  k = (k ^ (k >> 15)) * 0x510E527Fu;
  return (k ^ (k >> 13)) ^ hi;
}
__device__ __forceinline__ uint32_t element_bits(uint32_t key, uint32_t e) {
  uint32_t h = key + e * 0x3C6EF373u;
  h = (h ^ (h >> 16)) * 0x6A09E667u;
  h = (h ^ (h >> 15)) * 0xBB67AE85u;
  return h ^ (h >> 16);
}

// Codes of four quotients, rounded up where the part of a step that is left and u make a whole one: the conversion instruction adds the upper 20 bits of a
// random word to what the code leaves of the value, below 2^-6 too, where a step is 2^-9.  Those bits are of u = (16 random bits + 1/2) / 2^16.
__device__ __forceinline__ uint32_t encode(const float (&y)[4], const uint32_t (&u)[4]) {
  int w = __builtin_amdgcn_cvt_sr_fp8_f32(y[0], (int)u[0], 0, 0);
  w = __builtin_amdgcn_cvt_sr_fp8_f32(y[1], (int)u[1], w, 1);
  w = __builtin_amdgcn_cvt_sr_fp8_f32(y[2], (int)u[2], w, 2);
  return (uint32_t)__builtin_amdgcn_cvt_sr_fp8_f32(y[3], (int)u[3], w, 3);
}
// the largest of 64 lanes' values that are not negative, in all of them: within rows of 16 lanes, from row to row, from the last lane
__device__ __forceinline__ float wave_most(float x) {
  auto step = [&](auto ctrl) {
    x = fmaxf(x, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xF, 0xF, false)));
  };
  step(std::integral_constant<int, 0x111>{});   // row_shr 1, 2, 4, 8
  step(std::integral_constant<int, 0x112>{});
  step(std::integral_constant<int, 0x114>{});
  step(std::integral_constant<int, 0x118>{});
  step(std::integral_constant<int, 0x142>{});   // row_bcast 15, 31
  step(std::integral_constant<int, 0x143>{});
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}
// scale of a block with this largest magnitude
__device__ __forceinline__ float scale_of(float most) { return most > 0.0f ? fmaxf(most * (1.0f / 448.0f), 0x1p-126f) : 1.0f; }

// The four elements of a thread at i
template <bool EIGHT, typename G, bool WHOLE>
struct Turn {
  f32x4 p, g, m, v;
  uint32_t mc, vc;
  float ms, vs;
  // whether the wave has elements of this turn
  static __device__ __forceinline__ bool any(int64_t i, int64_t n) { return WHOLE || i - (threadIdx.x & 63) * 4 < n; }
  __device__ __forceinline__ void load(const StepTensor &t, int64_t n, int64_t i) {
    if (!any(i, n)) return;
    p = load_some<WHOLE>(t.p, i, n);
    g = load_some<WHOLE>(static_cast<const G *>(t.g), i, n);
    if constexpr (EIGHT) {
      mc = load_codes<WHOLE>(static_cast<const uint8_t *>(t.m), i, n);
      vc = load_codes<WHOLE>(static_cast<const uint8_t *>(t.v), i, n);
      ms = t.m_scale[i / kBlock];
      vs = t.v_scale[i / kBlock];
    } else {
      m = load_some<WHOLE>(static_cast<const float *>(t.m), i, n);
      v = load_some<WHOLE>(static_cast<const float *>(t.v), i, n);
    }
  }
  __device__ __forceinline__ void step(const StepArgs &s, const StepTensor &t, int64_t n, float wd, float coef, int64_t i) {
    if (!any(i, n)) return;
    if constexpr (EIGHT) {
      // What leads to codes and scales rounds operation by operation, so that a state follows from its inputs alone, whatever is contracted or
      // approximated elsewhere; the update takes the same root and the hardware's reciprocal (1 ulp).
#pragma clang fp contract(off)
      const AdamArgs &a = s.a;
      const float root_c2 = sqrtf(a.inv_c2), new_m = 1.0f - a.beta1, new_v = 1.0f - a.beta2;
      f32x4 r = decode(vc);
      m = decode(mc);
      float mm = 0.0f, rm = 0.0f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float ge = g[e] * coef, old = r[e] * vs;
        m[e] = (m[e] * ms) * a.beta1 + ge * new_m;
        r[e] = sqrtf((old * old) * a.beta2 + (ge * new_v) * ge);
        const float update = m[e] * a.inv_c1 * __builtin_amdgcn_rcpf(__builtin_fmaf(r[e], root_c2, a.eps));
        p[e] = __builtin_fmaf(-a.lr, __builtin_fmaf(wd, p[e], update), p[e]);
        mm = fmaxf(mm, fabsf(m[e]));
        rm = fmaxf(rm, r[e]);
      }
      const int64_t b = i / kBlock;
      ms = scale_of(wave_most(mm));
      vs = scale_of(wave_most(rm));
      const float mi = 1.0f / ms, ri = 1.0f / vs;
      const uint32_t key = block_key(__builtin_amdgcn_readfirstlane(t.first_block + (uint32_t)b), s.key_lo, s.key_hi);
      float ym[4], yr[4];
      uint32_t um[4], ur[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t h = element_bits(key, (threadIdx.x & 63) * 4 + e);
        um[e] = (h << 16) | 0x8000u;
        ur[e] = (h & 0xFFFF0000u) | 0x8000u;
        const float y = m[e] * mi;   // (comparisons that let NaN through)
        ym[e] = y > 448.0f ? 448.0f : y < -448.0f ? -448.0f : y;
        // one step at least of a root that is not zero: what lies below it has the code of it, however it is rounded
        const float q = r[e] * ri, least = r[e] > 0.0f ? 0x1p-9f : 0.0f;
        yr[e] = q < least ? least : q > 448.0f ? 448.0f : q;
      }
      mc = encode(ym, um);
      vc = encode(yr, ur);
      store_codes<WHOLE>(static_cast<uint8_t *>(t.m), i, n, mc);
      store_codes<WHOLE>(static_cast<uint8_t *>(t.v), i, n, vc);
      if ((threadIdx.x & 63) == 0) {
        t.m_scale[b] = ms;
        t.v_scale[b] = vs;
      }
    } else {
      AdamArgs a = s.a;
      a.wd = wd;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float pe = p[e], me = m[e], ve = v[e];
        adam_one(a, coef, g[e], pe, me, ve);
        p[e] = pe;
        m[e] = me;
        v[e] = ve;
      }
      store_some<WHOLE>(static_cast<float *>(t.m), i, n, m);
      store_some<WHOLE>(static_cast<float *>(t.v), i, n, v);
    }
    store_some<WHOLE>(t.p, i, n, p);
    if (t.w != nullptr) store_some<WHOLE>(t.w, i, n, p);
  }
};

template <bool EIGHT, typename G>
__global__ __launch_bounds__(256) void adam_many_kernel(StepArgs s) {
  float coef = 1.0f;
  if (s.sqnorm != nullptr) {
    const float sq = s.sqnorm[0];
    if (!(fabsf(sq) < INFINITY)) return;   // a gradient that is not finite: the step is left out
    if (s.a.max_norm > 0.0f) coef = fminf(1.0f, s.a.max_norm / (sqrtf(sq) + 1e-6f));
  }
  for (uint32_t c = blockIdx.x; c < s.chunks; c += gridDim.x) {
    const StepTensor &t = s.of[tensor_of<kStepTensors>(s, c)];
    const int64_t n = t.count(), base = (int64_t)(c - t.first_chunk) * kChunk, first = base + threadIdx.x * 4;
    const float wd = (t.count_decay & 1) ? s.a.wd : 0.0f;
    auto chunk = [&](auto whole) {   // all loads of a chunk at once
      Turn<EIGHT, G, decltype(whole)::value> turn[kTurns];
#pragma unroll
      for (int u = 0; u < kTurns; ++u) turn[u].load(t, n, first + u * 1024);
#pragma unroll
      for (int u = 0; u < kTurns; ++u) turn[u].step(s, t, n, wd, coef, first + u * 1024);
    };
    if (base + kChunk <= n) chunk(std::true_type{});
    else chunk(std::false_type{});
  }
}

// The squares of `left` elements of a chunk (p and left the same in all lanes), this thread's share of THREADS: 16 bytes a load, past the caches; vectors
// that do not lie within the chunk as a whole are outside the descriptor and arrive as zeros, and what is left of the last one is read an element a lane
template <typename G, int THREADS>
__device__ __forceinline__ double squares(const G *p, int left) {
  constexpr int W = 16 / sizeof(G), TURNS = kChunk / (W * THREADS), NONTEMPORAL = 2;
  const int lane = threadIdx.x % THREADS;
  const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<G *>(p), 0, left / W * 16, 0x00020000);
  f32x4 raw[TURNS];
#pragma unroll
  for (int u = 0; u < TURNS; ++u)
    raw[u] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, (u * THREADS + lane) * 16, 0, NONTEMPORAL));
  const float rest = lane < left % W ? to_f32(p[left / W * W + lane]) : 0.0f;
  double s = (double)rest * rest;
#pragma unroll
  for (int u = 0; u < TURNS; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float x = raw[u][e];
      if constexpr (sizeof(G) == 4) {
        s += (double)x * x;
      } else {   // two bf16 values, the upper halves of fp32 ones
        const uint32_t w = __builtin_bit_cast(uint32_t, x);
        const float lo = __builtin_bit_cast(float, w << 16), hi = __builtin_bit_cast(float, w & 0xFFFF0000u);
        s += (double)lo * lo;
        s += (double)hi * hi;
      }
    }
  return s;
}
// partial[block] = the squares of chunks block, block + grid, ..., added to what launches before left in the first `have`
template <typename G>
__global__ __launch_bounds__(256) void norm_many_kernel(NormArgs s, double *__restrict__ partial, int have) {
  double sum = 0.0;
  for (uint32_t c = blockIdx.x; c < s.chunks; c += gridDim.x) {
    const NormTensor &t = s.of[tensor_of<kNormTensors>(s, c)];
    const int64_t base = (int64_t)(c - t.first_chunk) * kChunk, left = t.count - base;
    sum += squares<G, 256>(static_cast<const G *>(t.g) + base, left < kChunk ? (int)left : kChunk);
  }
  sum = workgroup_sum<256>(sum);
  if (threadIdx.x == 0) partial[blockIdx.x] = (int)blockIdx.x < have ? partial[blockIdx.x] + sum : sum;
}
__global__ __launch_bounds__(256) void norm_many_sum(int blocks, const double *__restrict__ partial, float *__restrict__ out, int accumulate) {
  double s = 0.0;
#pragma unroll
  for (int i = 0; i < kNormBlocks / 256; ++i) {
    const int b = i * 256 + threadIdx.x;
    s += b < blocks ? partial[b] : 0.0;
  }
  s = workgroup_sum<256>(s);
  if (threadIdx.x == 0) out[0] = (float)(accumulate ? (double)out[0] + s : s);
}
// Few elements: the launches are the time, so there is one
template <typename G>
__global__ __launch_bounds__(1024) void norm_many_once(NormOnceArgs s, float *__restrict__ out, int accumulate) {
  double sum = 0.0;
#pragma unroll 1
  for (uint32_t c = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); c < s.chunks; c += 16)
    sum += squares<G, 64>(static_cast<const G *>(s.of[c].g), (int)s.of[c].count);
  sum = workgroup_sum<1024>(sum);
  if (threadIdx.x == 0) out[0] = (float)(accumulate ? (double)out[0] + sum : sum);
}

// Bytes that a call reads or writes.
struct Span {
  uintptr_t from, to;
  bool written;
};
// Whether no byte that is written is of two spans.  Sorted by merging the runs that are there already: tensors of a kind mostly lie in the order in
// which the call names them (112 tensors, seven spans each: 30 us with std::sort).  other: room for n more.
bool spans_apart(Span *s, Span *other, int64_t n) {
  auto run_end = [&](int64_t i) {
    for (++i; i < n && s[i - 1].from <= s[i].from; ++i) {}
    return i;
  };
  auto before = [](const Span &a, const Span &b) { return a.from < b.from; };
  while (run_end(0) < n) {
    for (int64_t i = 0; i < n;) {
      const int64_t mid = run_end(i), end = mid < n ? run_end(mid) : n;
      std::merge(s + i, s + mid, s + mid, s + end, other + i, before);
      i = end;
    }
    std::swap(s, other);
  }
  uintptr_t any = 0, written = 0;   // ends of the spans so far, of the written ones
  for (int64_t i = 0; i < n; ++i) {
    if (s[i].from < (s[i].written ? any : written)) return false;
    any = std::max(any, s[i].to);
    if (s[i].written) written = std::max(written, s[i].to);
  }
  return true;
}

int64_t blocks_of(int64_t count) { return (count + kBlock - 1) / kBlock; }

// Which elements a tensor may have: their blocks are counted in 32 bits
bool count_ok(int64_t count) { return count > 0 && count <= (int64_t)1 << 39; }

// Two words of random numbers' key
void step_keys(uint64_t seed, int32_t step, uint32_t *lo, uint32_t *hi) {
  uint64_t s = seed * 0x9E3779B97F4A7C15ull + (uint64_t)step;
  s = (s ^ (s >> 32)) * 0xBB67AE8584CAA73Bull;
  s = (s ^ (s >> 29)) * 0x6A09E667F3BCC909ull;
  s ^= s >> 32;
  *lo = (uint32_t)s;
  *hi = (uint32_t)(s >> 32);
}

}  // namespace

}  // namespace mtnlg

using namespace mtnlg;

extern "C" {

size_t mtnlg_grad_sqnorm_many_workspace(void) { return kNormBlocks * sizeof(double); }

int mtnlg_grad_sqnorm_many(int32_t tensors, const mtnlg_adam_tensor *of, int grad_dtype, void *workspace, size_t workspace_bytes, float *sqnorm,
                           int accumulate, void *stream) {
  if (!of || !workspace || !sqnorm) return MTNLG_NULL_POINTER;
  if (tensors <= 0 || (grad_dtype != MTNLG_F32 && grad_dtype != MTNLG_BF16)) return MTNLG_INVALID_ARG;
  if (tensors > kMostTensors) return MTNLG_UNSUPPORTED_SHAPE;
  if (((uintptr_t)workspace & 7) || ((uintptr_t)sqnorm & 3)) return MTNLG_INVALID_ARG;
  if (workspace_bytes < mtnlg_grad_sqnorm_many_workspace()) return MTNLG_WORKSPACE_TOO_SMALL;
  const bool f32 = grad_dtype == MTNLG_F32;
  for (int32_t i = 0; i < tensors; ++i) {
    if (!of[i].grad) return MTNLG_NULL_POINTER;
    if (of[i].count <= 0 || ((uintptr_t)of[i].grad & (f32 ? 15 : 7))) return MTNLG_INVALID_ARG;
    if (!count_ok(of[i].count)) return MTNLG_UNSUPPORTED_SHAPE;
    // what is written lies on no gradient
    const uintptr_t from = (uintptr_t)of[i].grad, to = from + (uintptr_t)(of[i].count * (f32 ? 4 : 2));
    if (((uintptr_t)sqnorm < to && from < (uintptr_t)sqnorm + 4) || ((uintptr_t)workspace < to && from < (uintptr_t)workspace + kNormBlocks * sizeof(double)))
      return MTNLG_INVALID_ARG;
  }
  if ((uintptr_t)sqnorm < (uintptr_t)workspace + kNormBlocks * sizeof(double) && (uintptr_t)workspace < (uintptr_t)sqnorm + 4) return MTNLG_INVALID_ARG;
  hipStream_t st = (hipStream_t)stream;
  LaunchScope scope(MTNLG_K_ELEMENTWISE, st);
  NormOnceArgs once;
  once.chunks = 0;
  int32_t named = 0;
  for (; named < tensors && once.chunks + (of[named].count + kChunk - 1) / kChunk <= kOnce; ++named)
    for (int64_t at = 0; at < of[named].count; at += kChunk)
      once.of[once.chunks++] = NormChunk{(const char *)of[named].grad + at * (f32 ? 4 : 2), std::min<int64_t>(of[named].count - at, kChunk)};
  if (named == tensors) {
    if (f32) norm_many_once<float><<<1, 1024, 0, st>>>(once, sqnorm, accumulate ? 1 : 0);
    else norm_many_once<bf16><<<1, 1024, 0, st>>>(once, sqnorm, accumulate ? 1 : 0);
    return check_launch();
  }
  int have = 0;
  for (int32_t i = 0; i < tensors;) {
    NormArgs s;
    uint64_t chunks = 0;
    int32_t k = 0;
    for (; i + k < tensors && k < kNormTensors && chunks < ((uint64_t)1 << 31); ++k) {
      s.of[k] = NormTensor{of[i + k].grad, of[i + k].count, (uint32_t)chunks, 0};
      chunks += (uint64_t)(of[i + k].count + kChunk - 1) / kChunk;
    }
    s.chunks = (uint32_t)chunks;   // (a tensor has up to 2^27)
    s.tensors = k;
    const int grid = chunks < kNormBlocks ? (int)chunks : kNormBlocks;
    if (f32) norm_many_kernel<float><<<grid, 256, 0, st>>>(s, (double *)workspace, have);
    else norm_many_kernel<bf16><<<grid, 256, 0, st>>>(s, (double *)workspace, have);
    MTNLG_TRY(check_launch());
    have = std::max(have, grid);
    i += k;
  }
  norm_many_sum<<<1, 256, 0, st>>>(have, (const double *)workspace, sqnorm, accumulate ? 1 : 0);
  return check_launch();
}

int mtnlg_adam_step_many(const mtnlg_adam_many_desc *desc, const mtnlg_adam_tensor *of, const float *sqnorm, void *stream) {
  if (!desc || !of) return MTNLG_NULL_POINTER;
  const bool eight = desc->state_bits == 8, f32 = desc->grad_dtype == MTNLG_F32;
  if (desc->tensors <= 0 || !adam_desc_ok(desc->adam) || (!eight && desc->state_bits != 32) || (!f32 && desc->grad_dtype != MTNLG_BF16))
    return MTNLG_INVALID_ARG;
  if (desc->tensors > kMostTensors) return MTNLG_UNSUPPORTED_SHAPE;
  if ((uintptr_t)sqnorm & 3) return MTNLG_INVALID_ARG;
  uint64_t blocks = 0;
  for (int32_t i = 0; i < desc->tensors; ++i) {
    const mtnlg_adam_tensor &t = of[i];
    if (!t.master || !t.m || !t.v || !t.grad || (eight && (!t.m_scale || !t.v_scale))) return MTNLG_NULL_POINTER;
    const uintptr_t states = (uintptr_t)t.m | (uintptr_t)t.v;
    if (t.count <= 0 || ((uintptr_t)t.master & 15) || ((uintptr_t)t.grad & (f32 ? 15 : 7)) || ((uintptr_t)t.weight_bf16 & 7) ||
        (states & (eight ? 3 : 15)) || (eight && (((uintptr_t)t.m_scale | (uintptr_t)t.v_scale) & 3)))
      return MTNLG_INVALID_ARG;
    if (!count_ok(t.count)) return MTNLG_UNSUPPORTED_SHAPE;
    blocks += (uint64_t)blocks_of(t.count);
  }
  if (blocks > 0xFFFFFFFFull) return MTNLG_UNSUPPORTED_SHAPE;
  {
    const size_t most = (size_t)desc->tensors * 7 + 1;
    Span *spans = new (std::nothrow) Span[2 * most];
    if (!spans) return MTNLG_HIP_ERROR;
    int64_t n = 0;
    auto add = [&](auto place, int64_t bytes, bool written, bool scales = false) {   // of every tensor
      for (int32_t i = 0; i < desc->tensors; ++i)
        if (const uintptr_t p = (uintptr_t)place(of[i]))
          spans[n++] = Span{p, p + (uintptr_t)((scales ? blocks_of(of[i].count) : of[i].count) * bytes), written};
    };
    using T = const mtnlg_adam_tensor &;
    add([](T t) { return t.master; }, 4, true);
    add([](T t) { return t.m; }, eight ? 1 : 4, true);
    add([](T t) { return t.v; }, eight ? 1 : 4, true);
    add([](T t) { return t.weight_bf16; }, 2, true);
    add([](T t) { return t.grad; }, f32 ? 4 : 2, false);
    if (eight) {
      add([](T t) { return t.m_scale; }, 4, true, true);
      add([](T t) { return t.v_scale; }, 4, true, true);
    }
    if (sqnorm) spans[n++] = Span{(uintptr_t)sqnorm, (uintptr_t)sqnorm + 4, false};
    const bool apart = spans_apart(spans, spans + most, n);
    delete[] spans;
    if (!apart) return MTNLG_INVALID_ARG;
  }
  hipStream_t st = (hipStream_t)stream;
  LaunchScope scope(MTNLG_K_ELEMENTWISE, st);
  StepArgs s;
  s.a = adam_args(desc->adam);
  if (eight) s.a.eps = fmaxf(s.a.eps, 0x1p-126f);   // what it is added to is multiplied with by its reciprocal: finite
  s.sqnorm = sqnorm;
  step_keys(desc->seed, desc->adam.step, &s.key_lo, &s.key_hi);
  uint32_t block = 0;
  for (int32_t i = 0; i < desc->tensors;) {
    uint64_t chunks = 0;
    int32_t k = 0;
    for (; i + k < desc->tensors && k < kStepTensors && chunks < ((uint64_t)1 << 31); ++k) {
      const mtnlg_adam_tensor &t = of[i + k];
      s.of[k] = StepTensor{t.master, t.m, t.v, t.m_scale, t.v_scale, t.grad, (bf16 *)t.weight_bf16, t.count * 2 + (t.decay ? 1 : 0), (uint32_t)chunks, block};
      chunks += (uint64_t)(t.count + kChunk - 1) / kChunk;
      block += (uint32_t)blocks_of(t.count);
    }
    s.chunks = (uint32_t)chunks;
    s.tensors = k;
    const unsigned grid = (unsigned)std::min<uint64_t>(chunks, 1u << 20);
    if (eight && f32) adam_many_kernel<true, float><<<grid, 256, 0, st>>>(s);
    else if (eight) adam_many_kernel<true, bf16><<<grid, 256, 0, st>>>(s);
    else if (f32) adam_many_kernel<false, float><<<grid, 256, 0, st>>>(s);
    else adam_many_kernel<false, bf16><<<grid, 256, 0, st>>>(s);
    MTNLG_TRY(check_launch());
    i += k;
  }
  return MTNLG_OK;
}

}  // extern "C"
