// The gate of the gated feed-forward block: an activation of fp32 values, and its slope.
#pragma once
#include "common.h"

namespace mtnlg {

__device__ __forceinline__ float nan_of_inf(float x, float y) { return __builtin_fmaf(x, 0.0f, y); }   // y, or NaN where x is not finite
// FAST: hardware exp2 and reciprocal (1 ulp each), for results that round to bf16: silu(x) = x s, s = 1 / (1 + exp(-x)), silu' = s + x s (1 - s) with 1 - s = exp(-x) s;
// GeLU's tanh form likewise (gelu_sigmoid_f).  Relative error: some 1e-7 for the operations and 1e-7 times the exponential's exponent, whose argument is rounded: at |x| < 5
// 3.4e-7 (SiLU), 2.3e-6 (tanh), 1.5e-6 (erf), and below 1e-5 wherever a value is more than 1e-32, a four-hundredth of the rounding to bf16.  x is clamped where both have reached their
// limits to 1e-32, so that exp(-x) s and powers of x stay finite and large negative values give no multiple of themselves; by comparisons, which let NaN through, and to a value
// that an infinity makes NaN: an infinite x (sums that pass the largest value) gives what the formulas give in floating point, so that it is seen in the results: inf act(inf), NaN
// at -inf (-inf times 0) and in the slope at either, whose second term is infinity times 0.
template <bool FAST, int KIND>
__device__ __forceinline__ void gate_one(float x, float &a, float &slope) {
  if constexpr (KIND == MTNLG_GATE_SILU) {
    if constexpr (FAST) {
      const float c = x < -80.0f ? nan_of_inf(x, -80.0f) : x, e = __builtin_amdgcn_exp2f(c * -1.4426950408889634f), s = __builtin_amdgcn_rcpf(1.0f + e);
      a = c * s;
      slope = s + a * (e * s);
    } else {
      const float s = 1.0f / (1.0f + expf(-x));
      a = x * s;
      slope = s + a * (1.0f - s);
    }
  } else if constexpr (KIND == MTNLG_GATE_GELU_TANH) {
    constexpr float K = 2.0f * 0.79788456080286536f, D3 = K * 3.0f * 0.044715f;   // 2 u' = K + D3 x^2
    if constexpr (FAST) {
      const float lo = x < -10.0f ? nan_of_inf(x, -10.0f) : x, c = lo > 10.0f ? 10.0f : lo, c2 = c * c;
      float e;
      const float s = gelu_sigmoid_f(c, c2, e);
      a = lo * s;
      slope = nan_of_inf(x, s) + (c * (K + D3 * c2)) * (e * s) * s;
    } else {
      // s and 1 - s from exp(-|2 u|), which is at most 1: neither is a difference.  (1 + tanh u) / 2 has 24 bits below 1 and not below s: at -5 the value had two of its own left
      const float w = K * (x + 0.044715f * x * x * x), t = expf(-fabsf(w)), d = 1.0f / (1.0f + t), td = t * d, s = w < 0.0f ? td : d;
      const float lo = x < -12.0f ? -12.0f : x, c = lo > 12.0f ? 12.0f : lo;   // (beyond, t is 0)
      a = x * s;
      slope = nan_of_inf(x, s) + (c * (K + D3 * c * c)) * (td * d);
    }
  } else if constexpr (FAST) {
    // The normal distribution's tail below -|x| as exp(-x^2 / 2) t P(t), t = 1 / (1 + 0.44 |x| / sqrt 2): P of degree 7 fitted here to the least relative error
    // over |x| <= 14 (1.8e-7 in exact arithmetic), so nothing cancels for negative x.  16 instructions, where the library's erf made the product that carries it take 140 us longer
    // forward and backward (6331 tokens, F 5456).
    constexpr float C[8] = {0.124110477f, 0.12443559f, 0.108656778f, 0.107906111f, -0.0100903258f, 0.148343735f, -0.13897401f, 0.0356117356f};
    const float t = __builtin_amdgcn_rcpf(1.0f + 0.311126984f * fabsf(x)), e = __builtin_amdgcn_exp2f(x * x * -0.72134752f);
    float tail = C[7];
#pragma unroll
    for (int i = 6; i >= 0; --i) tail = tail * t + C[i];
    tail *= t * e;
    const float cdf = x < 0.0f ? tail : 1.0f - tail;
    a = x * cdf;
    slope = cdf + x * (e * 0.39894228f);
  } else {
    // the tail by erfc: (1 + erf) / 2 cancels for negative x as 1 + tanh does
    const float tail = 0.5f * erfcf(fabsf(x) * 0.70710678118654752f), cdf = x < 0.0f ? tail : 1.0f - tail;
    a = x * cdf;
    slope = cdf + x * (expf(-0.5f * x * x) * 0.39894228f);
  }
}
// a[i] = act(x[i]), slope[i] = act'(x[i]); the kind is the same in all lanes and is looked at once for the N values
template <bool FAST, int N>
__device__ __forceinline__ void gate_of(int kind, const float (&x)[N], float (&a)[N], float (&slope)[N]) {
  if (kind == MTNLG_GATE_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) gate_one<FAST, MTNLG_GATE_SILU>(x[i], a[i], slope[i]);
  } else if (kind == MTNLG_GATE_GELU_TANH) {
#pragma unroll
    for (int i = 0; i < N; ++i) gate_one<FAST, MTNLG_GATE_GELU_TANH>(x[i], a[i], slope[i]);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) gate_one<FAST, MTNLG_GATE_GELU_ERF>(x[i], a[i], slope[i]);
  }
}

// What a product of the block does with its results, in the place of the other epilogues (EpiArgs: aux is z [M, 2 F], flags the kind):
//   GATE_FWD  N = 2 F columns of z, in fours (gate, gate, other, other): act(gate) * other to C [M, F], z to aux (nullable)
//   GATE_BWD  N = F columns of dg: with z from aux, dz to C [M, 2 F]
enum gate_mode { GATE_NONE = 0, GATE_FWD = 1, GATE_BWD = 2 };
// Row of w_fc1 [2 F, h] that column n of GATE_FWD's product takes: so every lane of a matrix instruction's result holds both parts of two columns
__device__ __forceinline__ int64_t gate_row(int64_t n, int64_t F) { return (n >> 2) * 2 + (n & 1) + ((n & 2) ? F : 0); }

template <typename E>
__device__ __forceinline__ void put4(E *p, f32x4 x) {
  if constexpr (sizeof(E) == 4) *reinterpret_cast<f32x4 *>(p) = x;
  else *reinterpret_cast<bf16x4 *>(p) = bf16x4{(bf16)x[0], (bf16)x[1], (bf16)x[2], (bf16)x[3]};
}
typedef __attribute__((ext_vector_type(2))) float gate_f32x2;
template <typename E>
__device__ __forceinline__ void put2(E *p, float x, float y) {
  if constexpr (sizeof(E) == 4) *reinterpret_cast<gate_f32x2 *>(p) = gate_f32x2{x, y};
  else *reinterpret_cast<bf16x2 *>(p) = bf16x2{(bf16)x, (bf16)y};
}
// Four consecutive columns of row m at column n of such a product
template <typename E, int MODE>
__device__ __forceinline__ void gate_epilogue4(const EpiArgs &ea, void *C, int64_t N, int64_t m, int64_t n, f32x4 v) {
  constexpr bool FAST = sizeof(E) == 2;
  if constexpr (MODE == GATE_FWD) {
    const int64_t F = N / 2, c = n / 2;
    if (ea.aux != nullptr) {
      E *z = static_cast<E *>(ea.aux) + m * N + c;
      put2(z, v[0], v[1]);
      put2(z + F, v[2], v[3]);
    }
    const float x[2] = {v[0], v[1]};
    float a[2], slope[2];
    gate_of<FAST>((int)ea.flags, x, a, slope);
    put2(static_cast<E *>(C) + m * F + c, a[0] * v[2], a[1] * v[3]);
  } else {
    const E *z = static_cast<const E *>(ea.aux) + m * 2 * N + n;
    const f32x4 g = load4(z), u = load4(z + N);
    const float x[4] = {g[0], g[1], g[2], g[3]};
    float a[4], slope[4];
    gate_of<FAST>((int)ea.flags, x, a, slope);
    f32x4 da, db;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      da[e] = v[e] * u[e] * slope[e];
      db[e] = v[e] * a[e];
    }
    E *dz = static_cast<E *>(C) + m * 2 * N + n;
    put4(dz, da);
    put4(dz + N, db);
  }
}

}  // namespace mtnlg
