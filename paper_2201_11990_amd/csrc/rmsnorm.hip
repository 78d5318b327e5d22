// Root-mean-square norm (Zhang and Sennrich, "Root mean square layer normalization", 2019) with the residual's addition before it:
//   s = x [+ residual] (stored, in the storage type),  r = 1 / sqrt(mean(s^2) + eps),  out = s r gamma,
// the same with the result in 8 bits (e4m3) and a scale to every row or every so many columns, and the backward pass
//   dn = dout gamma,  n = s r,  dx = dres + r (dn - n mean(dn n)),  dgamma = sum over rows of dout n.
// All bound by memory: every matrix is read or written once, a row stays in registers between its reduction and its result.  2048 rows of 20480 columns, bf16, with residuals: forward
// 336 MB in 58 us; backward 336 MB, and 21 MB of sums of dgamma written and read, in 77 and 6 us.  8192 rows of 2048 columns to 8 bits with a scale to 128 columns: 118 MB in 23 us.
#include "common.h"

namespace mtnlg {

namespace {

constexpr int MAX_COLUMNS = 32768;
constexpr float E4M3_MOST = 448.0f, SCALE_LEAST = 0x1p-126f;

// How a row is shared out: W waves to a row (1 up to 1024 columns, 4 up to 4096, then 16), NV pieces of 8 columns to a lane.  One wave needs no barrier, several have more of a row
// in flight and start few rows sooner.  Median us of forward and backward, bf16 with a residual, inputs in no cache: 2048 columns with one wave / four: 300 rows 8.5 and 12.2 / 7.0 and 11.2,
// 1024 rows 10.7 and 16.3 / 9.9 and 15.7, 8192 rows 40 and 59 / 41 and 54; 8192 columns with four / sixteen: 64 rows 8.9 and 12.3 / 7.7 and 12.4, 2048 rows 41 and 65 / 42 and 57,
// 8192 rows 125 and 158 / 126 and 153.
template <int W> constexpr int threads_of() { return W < 4 ? 256 : 64 * W; }

// Sum over the W waves of a row; the same in every lane.
template <int W>
__device__ __forceinline__ float row_sum(float v, float *lds) {
  v = wave_sum(v);
  if constexpr (W > 1) {
    __syncthreads();   // lds may still be read from the last time
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll
    for (int i = 0; i < W; ++i) v += lds[i];
  }
  return v;
}
template <int W>
__device__ __forceinline__ float row_max(float v, float *lds) {
  v = wave_max(v);
  if constexpr (W > 1) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int i = 1; i < W; ++i) v = fmaxf(v, lds[i]);
  }
  return v;
}

struct NormArgs {
  int64_t rows;
  int h;
  const void *x, *residual, *gamma;
  void *xsum, *out;
  float eps;
  float *rstd, *scale;
  int columns, scales;   // 8 bits: columns that share a scale (0: the row), scales of a row
};

// y to the nearest value of e4m3, beyond 448 to 448 (NaN stays NaN).  The instruction rounds to nearest even.
__device__ __forceinline__ unsigned e4m3_of4(float a, float b, float c, float d) {
  auto within = [](float y) { return y > E4M3_MOST ? E4M3_MOST : y < -E4M3_MOST ? -E4M3_MOST : y; };
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(within(a), within(b), 0, false);
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(within(c), within(d), w, true);
}

// y / scale, correctly rounded: codes are of quotients by the scale that is stored, and next to a border between two codes a product with a rounded reciprocal has the other
// one.  Both are taken relative to the power of two in the scale (exact), so that nothing below overflows or loses bits that a code shows; the product with the
// mantissa's reciprocal is corrected by its remainder (Markstein, "Computation of elementary functions on the IBM RISC System/6000 processor", 1990).  8192 rows of
// 2048 columns to 8 bits: 26.0 us a call, 25.4 with products by 448 / m, 26.8 with eight divisions.
struct QuotientBy {
  float toward, mantissa, inverse;
  __device__ __forceinline__ explicit QuotientBy(float scale) {   // normal, or infinite: quotients of what is finite are 0 then
    const unsigned bits = __float_as_uint(scale);
    toward = __uint_as_float(bits < 0x7F800000u ? 0x7F000000u - (bits & 0x7F800000u) : 0);
    mantissa = __uint_as_float((bits & 0x7FFFFFu) | 0x3F800000u);
    inverse = 1.0f / mantissa;
  }
  __device__ __forceinline__ float operator()(float y) const {
    const float x = y * toward, q = x * inverse;
    return fmaf(fmaf(-q, mantissa, x), inverse, q);
  }
};

template <typename E, int W, int NV, bool E4M3>
__global__ __launch_bounds__(threads_of<W>()) void rmsnorm_fwd_kernel(NormArgs a) {
  __shared__ float red[16];
  constexpr int LANES = 64 * W, ROWS = threads_of<W>() / LANES;
  const int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES;
  if (ROWS > 1 && row >= a.rows) return;   // whole waves
  const int at = threadIdx.x % LANES, nvec = a.h / 8;
  const E *x = static_cast<const E *>(a.x) + row * a.h, *res = static_cast<const E *>(a.residual) + row * a.h;
  Raw8<E> xv[NV], rv[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int j = at + i * LANES;
    if (j < nvec) {
      xv[i].load(x + 8 * j);
      if (a.residual) rv[i].load(res + 8 * j);
    }
  }
  float v[NV][8], sum = 0.0f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int j = at + i * LANES;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[i][e] = j < nvec ? xv[i][e] : 0.0f;
    if (j < nvec && a.residual) {
      // what is normalised is the sum as it is stored, which the backward pass is given
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = to_f32(from_f32<E>(v[i][e] + rv[i][e]));
      store8(static_cast<E *>(a.xsum) + row * a.h + 8 * j, v[i]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += v[i][e] * v[i][e];
  }
  const float r = 1.0f / sqrtf(row_sum<W>(sum, red) / (float)a.h + a.eps);
  if (at == 0) a.rstd[row] = r;
  const E *gamma = static_cast<const E *>(a.gamma);
  float most = 0.0f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int j = at + i * LANES;
    if (j < nvec) {
      float g[8];
      load8(gamma + 8 * j, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[i][e] = v[i][e] * r * g[e];
        most = fmaxf(most, fabsf(v[i][e]));
      }
      if constexpr (!E4M3) store8(static_cast<E *>(a.out) + row * a.h + 8 * j, v[i]);
    }
  }
  if constexpr (E4M3) {
    if (a.columns == 0) most = row_max<W>(most, red);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int j = at + i * LANES;
      float m = most;
      if (a.columns != 0) {   // columns is 8 times a power of two up to 64: lanes that share a scale lie side by side
        m = 0.0f;
        if (j < nvec) {
#pragma unroll
          for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(v[i][e]));
        }
        for (int off = 1; off < a.columns / 8; off *= 2) m = fmaxf(m, __shfl_xor(m, off, 64));
      }
      if (j >= nvec) continue;
      const float scale = m > 0.0f ? fmaxf(m / E4M3_MOST, SCALE_LEAST) : 1.0f;
      const QuotientBy by(scale);
      const int first = a.columns ? 8 * j % a.columns : j;
      if (first == 0) a.scale[row * a.scales + (a.columns ? 8 * j / a.columns : 0)] = scale;
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = by(v[i][e]);
      *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(a.out) + row * a.h + 8 * j) =
          uint2{e4m3_of4(y[0], y[1], y[2], y[3]), e4m3_of4(y[4], y[5], y[6], y[7])};
    }
  }
}

// Rows of a launch: 16 waves to each would pass 2^32 work items from 2^22 on.
constexpr int64_t LAUNCHED_ROWS = 1 << 21;

template <typename E, bool E4M3>
int fwd_launch(const NormArgs &all, hipStream_t st) {
  const int nvec = all.h / 8;
  LaunchScope scope(MTNLG_K_LN_FWD, st);
  for (int64_t first = 0; first < all.rows; first += LAUNCHED_ROWS) {
    NormArgs a = all;
    a.rows = all.rows - first < LAUNCHED_ROWS ? all.rows - first : LAUNCHED_ROWS;
    a.x = static_cast<const E *>(all.x) + first * all.h;
    if (all.residual) {
      a.residual = static_cast<const E *>(all.residual) + first * all.h;
      a.xsum = static_cast<E *>(all.xsum) + first * all.h;
    }
    a.out = static_cast<char *>(all.out) + first * all.h * (E4M3 ? 1 : sizeof(E));
    a.rstd = all.rstd + first;
    if (E4M3) a.scale = all.scale + first * all.scales;
#define RMS(W, NV) \
  rmsnorm_fwd_kernel<E, W, NV, E4M3><<<(unsigned)((a.rows + threads_of<W>() / (64 * W) - 1) / (threads_of<W>() / (64 * W))), threads_of<W>(), 0, st>>>(a)
    if (nvec <= 64) RMS(1, 1);
    else if (nvec <= 128) RMS(1, 2);
    else if (nvec <= 256) RMS(4, 1);
    else if (nvec <= 512) RMS(4, 2);
    else if (nvec <= 1024) RMS(16, 1);
    else if (nvec <= 2048) RMS(16, 2);
    else if (nvec <= 3 * 1024) RMS(16, 3);
    else RMS(16, 4);
#undef RMS
    MTNLG_TRY(check_launch());
  }
  return MTNLG_OK;
}

// ------------------------------------------------------------------ backward
// as loaded, not as eight floats (the compiler else widens them once, for all rows)
__device__ __forceinline__ void keep(Raw8<bf16> &r) { asm volatile("" : "+v"(r.v)); }
__device__ __forceinline__ void keep(Raw8<float> &) {}

typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
// the lane's number, worked out where it stands
__device__ __forceinline__ int lane_of() {
  int lane;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(lane));
  return lane;
}

struct NormBwdArgs {
  int64_t rows;
  int h;
  const void *x, *gamma, *dout, *dres;
  const float *rstd;
  void *dx;
  float *partial;   // [workgroups][h]: the workgroup's rows of dgamma
};

// A workgroup takes every gridDim.x-th row (of each of its ROWS groups of waves) and sums its share of dgamma in registers.  The next row is requested before the
// present one is reduced, so that the loads of a row travel behind the barriers of the other.  Rows up to 8192 columns; longer ones have no registers for a row ahead.
template <typename E, int W, int NV>
__global__ __launch_bounds__(threads_of<W>()) void rmsnorm_bwd_kernel(NormBwdArgs a) {
  constexpr int LANES = 64 * W, ROWS = threads_of<W>() / LANES;
  __shared__ float red[16];
  __shared__ __attribute__((aligned(16))) float side[ROWS > 1 ? (ROWS - 1) * LANES * NV * 8 : 1];
  const int at = threadIdx.x % LANES, group = ROWS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / LANES), nvec = a.h / 8;
  const int64_t step = (int64_t)gridDim.x * ROWS;
  struct Row { Raw8<E> x[NV], dout[NV], dres[NV]; };
  float dg[NV][8] = {};
  const bool with_dres = a.dres != nullptr;
  auto request = [&](int64_t row, Row &to) __attribute__((always_inline)) {
    if (row >= a.rows) return;
    const int64_t from = row * a.h + 8 * at;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (at + i * LANES < nvec) {
        to.x[i].load(static_cast<const E *>(a.x) + from + 8 * LANES * i);
        to.dout[i].load(static_cast<const E *>(a.dout) + from + 8 * LANES * i);
        if (with_dres) to.dres[i].load(static_cast<const E *>(a.dres) + from + 8 * LANES * i);
      }
    }
  };
  int64_t row = (int64_t)blockIdx.x * ROWS + group;
  Row next;
  request(row, next);
  // gamma stays in registers: a load of it behind the next row's would be waited for after them
  Raw8<E> gamma[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (at + i * LANES < nvec) gamma[i].load(static_cast<const E *>(a.gamma) + 8 * at + 8 * LANES * i);
  // the same number of turns for all waves of a row's group; a group without a row left has none
  for (; row < a.rows; row += step) {
    const float r = a.rstd[row];
    const Row now = next;
    request(row + step, next);
    float dot = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (at + i * LANES < nvec) {
        keep(gamma[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float n = now.x[i][e] * r;
          dot += now.dout[i][e] * gamma[i][e] * n;
          dg[i][e] += now.dout[i][e] * n;
        }
      }
      __builtin_amdgcn_sched_barrier(0);   // eight columns at a time: all of them in fp32 at once do not fit beside the next row
    }
    const float mean = row_sum<W>(dot, red) / (float)a.h;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (at + i * LANES < nvec) {
        float o[8];
        keep(gamma[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          o[e] = r * (now.dout[i][e] * gamma[i][e] - now.x[i][e] * r * mean);
          if (with_dres) o[e] += now.dres[i][e];
        }
        store8(static_cast<E *>(a.dx) + row * a.h + 8 * at + 8 * LANES * i, o);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  if constexpr (ROWS > 1) {   // the groups' sums, in their order
    if (group > 0) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 8; e += 4)
          *reinterpret_cast<f32x4 *>(side + (((group - 1) * NV + i) * 2 + e / 4) * LANES * 4 + at * 4) = f32x4{dg[i][e], dg[i][e + 1], dg[i][e + 2], dg[i][e + 3]};
    }
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int s = 0; s < ROWS - 1; ++s)
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) dg[i][e] += side[((s * NV + i) * 2 + e / 4) * LANES * 4 + at * 4 + e % 4];
  }
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (at + i * LANES < nvec) store8(a.partial + (int64_t)blockIdx.x * a.h + 8 * (at + i * LANES), dg[i]);
}

// Rows of more than 8192 columns, 16 waves to a row.  The next row comes into LDS by DMA while the present one is in registers: every wave brings what it reads itself, so that
// no barrier stands between.  PRE: of x, dout and dres those that LDS has room for (the others are loaded with their row).  Where dres is not ahead its place is taken before the next
// row's DMA goes out, since memory operations are waited for in their order; dx goes out by buffer stores, of which every wave has the same number (what lies past the
// row is dropped), so that the next row can be waited for and they not.
template <typename E, int NV, int PRE>
__global__ __launch_bounds__(1024) void rmsnorm_bwd_wide_kernel(NormBwdArgs a) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ float red[16];
  constexpr int ES = sizeof(E), HALVES = ES / 2, SEG = 64 * 8 * ES, STORES = NV * HALVES;   // SEG: a wave's bytes of a piece
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool with_dres = a.dres != nullptr;
  const uint32_t bytes = (uint32_t)a.h * ES;
  char *const mine = smem + wave * (PRE * NV * SEG);
  const uint32_t lds0 = lds_address(mine);
  const char *const from[3] = {static_cast<const char *>(a.x), static_cast<const char *>(a.dout), static_cast<const char *>(a.dres)};
  auto fetch = [&](int64_t row) {
    const uint32_t here = (uint32_t)(wave * SEG + lane_of() * 16);   // worked out where it stands: no registers for offsets across the loop
#pragma unroll
    for (int m = 0; m < PRE; ++m) {
      if (m == 2 && !with_dres) continue;
      const dma_rsrc_t rs = dma_rsrc(from[m] + row * bytes, __builtin_amdgcn_readfirstlane(bytes));
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int k = 0; k < HALVES; ++k) dma16(rs, lds0 + (m * NV + i) * SEG + k * 1024, here + i * 16 * SEG + k * 1024);
    }
  };
  auto column = [&](int i) { return (i * 1024 + wave * 64 + lane) * 8; };
  auto take = [&](int m, int i, int64_t row) {
    Raw8<E> r{};
    if (m < PRE) r.load(reinterpret_cast<const E *>(mine + (m * NV + i) * SEG) + lane * 8);
    else if (column(i) < a.h) r.load(reinterpret_cast<const E *>(from[m]) + row * a.h + column(i));
    return r;
  };
  auto sum_over = [&](float v) {   // of the row, without waiting for memory
    v = wave_sum(v);
    asm volatile("s_barrier" ::: "memory");   // read the last time
    if (lane == 0) red[wave] = v;
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    v = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) v += red[i];
    return v;
  };
  Raw8<E> gamma[NV];
  float dg[NV][8] = {};
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    gamma[i] = Raw8<E>{};
    if (column(i) < a.h) gamma[i].load(static_cast<const E *>(a.gamma) + column(i));
  }
  // rstd by scalar loads, which are counted apart: a vector load behind the next row's DMA would be waited for with it
  const auto rstd = (const __attribute__((address_space(4))) float *)a.rstd;
  int64_t row = blockIdx.x;
  fetch(row);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  for (; row < a.rows; row += gridDim.x) {
    const float r = rstd[row];
    Raw8<E> x[NV], d[NV], res[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      x[i] = take(0, i, row);
      d[i] = take(1, i, row);
      if (with_dres) res[i] = take(2, i, row);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {   // here, before the next row's go out
      keep(x[i]);
      keep(d[i]);
      keep(res[i]);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (row + gridDim.x < a.rows) fetch(row + gridDim.x);
    float dot = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      keep(gamma[i]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float n = x[i][e] * r;
        dot += d[i][e] * gamma[i][e] * n;
        dg[i][e] += d[i][e] * n;
      }
      __builtin_amdgcn_sched_barrier(0);   // eight columns at a time: no registers for all of them in fp32
    }
    const float mean = sum_over(dot) / (float)a.h;
    const int col = (wave * 64 + lane_of()) * 8 * ES;
    const auto out = __builtin_amdgcn_make_buffer_rsrc(static_cast<char *>(a.dx) + row * bytes, 0, (int)bytes, 0x00020000);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      E o[8];
      keep(gamma[i]);
      keep(x[i]);
      keep(d[i]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float v = r * (d[i][e] * gamma[i][e] - x[i][e] * r * mean);
        if (with_dres) v += res[i][e];
        o[e] = from_f32<E>(v);
      }
#pragma unroll
      for (int k = 0; k < HALVES; ++k) {
        u32x4 v;
        __builtin_memcpy(&v, o + k * (16 / ES), 16);
        __builtin_amdgcn_raw_buffer_store_b128(v, out, col + i * 1024 * 8 * ES + k * 16, 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(STORES) : "memory");   // the next row's have landed
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int col = (i * 1024 + wave * 64 + lane_of()) * 8;
    if (col < a.h) store8(a.partial + (int64_t)blockIdx.x * a.h + col, dg[i]);
  }
}
template <typename E, int NV> constexpr int wide_ahead() { return 3 * NV * 16 * 64 * 8 * (int)sizeof(E) <= 156 * 1024 ? 3 : 2 * NV * 16 * 64 * 8 * (int)sizeof(E) <= 156 * 1024 ? 2 : 1; }
template <typename E, int NV>
int bwd_wide_launch(const NormBwdArgs &a, unsigned groups, hipStream_t st) {
  constexpr int PRE = wide_ahead<E, NV>(), lds = PRE * NV * 16 * 64 * 8 * (int)sizeof(E);
  static unsigned long long attr_done = 0;
  int device;
  if (!attr_is_set(attr_done, &device)) {
    if (hipFuncSetAttribute((const void *)rmsnorm_bwd_wide_kernel<E, NV, PRE>, hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess) return MTNLG_HIP_ERROR;
    attr_mark_set(attr_done, device);
  }
  rmsnorm_bwd_wide_kernel<E, NV, PRE><<<groups, 1024, lds, st>>>(a);
  return check_launch();
}

// dgamma from the workgroups' sums: 32 columns to a workgroup, 8 lanes across them, 32 down; a fixed order
template <typename O>
__global__ __launch_bounds__(256) void rmsnorm_dgamma_kernel(int rows, int h, const float *__restrict__ partial, O *__restrict__ dgamma, int accumulate) {
  __shared__ f32x4 side[32][8];
  const int lane = threadIdx.x % 8, down = threadIdx.x / 8, col = blockIdx.x * 32 + lane * 4;
  f32x4 s = {};
  if (col < h) {
#pragma unroll 4
    for (int i = down; i < rows; i += 32) s += *reinterpret_cast<const f32x4 *>(partial + (int64_t)i * h + col);
  }
  side[down][lane] = s;
  __syncthreads();
  if (down > 0 || col >= h) return;
  for (int i = 1; i < 32; ++i) s += side[i][lane];
#pragma unroll
  for (int e = 0; e < 4; ++e) dgamma[col + e] = from_f32<O>(accumulate ? to_f32(dgamma[col + e]) + s[e] : s[e]);
}

// Workgroups of the row kernel: as many as run at once; for fewer rows one to four (a wave) or two (four waves), whose sums of dgamma are added up before they are written (1024 rows of 2048
// columns, four waves: 18.9 us with one row, 15.7 with two, 15.6 with four; 512 rows 13.0, 13.0, 14.2).
int waves_of(int h) { return h <= 1024 ? 1 : h <= 4096 ? 4 : 16; }
int64_t bwd_groups(int64_t rows, int h) {
  const int w = waves_of(h);
  const int64_t most = w == 16 ? 256 : 1024, each = w == 1 ? 4 : w == 4 ? 2 : 1, want = (rows + each - 1) / each;
  return want < most ? want : most;
}

template <typename E>
int bwd_launch(const NormBwdArgs &a, void *dgamma, int grad_f32, int accumulate, hipStream_t st) {
  const int nvec = a.h / 8;
  const unsigned groups = (unsigned)bwd_groups(a.rows, a.h);
  LaunchScope scope(MTNLG_K_LN_BWD, st);
#define RMS(W, NV) rmsnorm_bwd_kernel<E, W, NV><<<groups, threads_of<W>(), 0, st>>>(a)
  if (nvec <= 64) RMS(1, 1);
  else if (nvec <= 128) RMS(1, 2);
  else if (nvec <= 256) RMS(4, 1);
  else if (nvec <= 512) RMS(4, 2);
  else if (nvec <= 1024) RMS(16, 1);
  else MTNLG_TRY((nvec <= 2048 ? bwd_wide_launch<E, 2>(a, groups, st) : nvec <= 3 * 1024 ? bwd_wide_launch<E, 3>(a, groups, st) : bwd_wide_launch<E, 4>(a, groups, st)));
#undef RMS
  MTNLG_TRY(check_launch());
  const unsigned blocks = (a.h + 31) / 32;
  if (grad_f32) rmsnorm_dgamma_kernel<float><<<blocks, 256, 0, st>>>((int)groups, a.h, a.partial, (float *)dgamma, accumulate);
  else rmsnorm_dgamma_kernel<E><<<blocks, 256, 0, st>>>((int)groups, a.h, a.partial, (E *)dgamma, accumulate);
  return check_launch();
}

int check_norm(int dtype, int64_t T, int64_t h) {
  if (dtype != MTNLG_F32 && dtype != MTNLG_BF16) return MTNLG_INVALID_ARG;
  if (T <= 0 || h <= 0) return MTNLG_INVALID_ARG;
  if (h % 8 || h > MAX_COLUMNS || T > 0x7FFFFFFF) return MTNLG_UNSUPPORTED_SHAPE;
  return MTNLG_OK;
}
bool unaligned(std::initializer_list<const void *> ps) {
  for (const void *p : ps)
    if ((uintptr_t)p & 15) return true;
  return false;
}

}  // namespace

}  // namespace mtnlg

using namespace mtnlg;

extern "C" {

int mtnlg_rmsnorm_fwd(int dtype, int64_t T, int64_t h, const void *x, const void *residual, const void *gamma, float eps, void *xsum, void *out,
                      float *rstd, void *stream) {
  if (!x || !gamma || !out || !rstd || (residual && !xsum)) return MTNLG_NULL_POINTER;
  MTNLG_TRY(check_norm(dtype, T, h));
  if (!(eps >= 0.0f && eps < INFINITY) || unaligned({x, residual, gamma, xsum, out}) || ((uintptr_t)rstd & 3)) return MTNLG_INVALID_ARG;
  if (residual && out == xsum) return MTNLG_INVALID_ARG;   // the sum would be lost
  const NormArgs a{T, (int)h, x, residual, gamma, xsum, out, eps, rstd, nullptr, 0, 0};
  return dtype == MTNLG_F32 ? fwd_launch<float, false>(a, (hipStream_t)stream) : fwd_launch<bf16, false>(a, (hipStream_t)stream);
}

int mtnlg_rmsnorm_fwd_e4m3(int dtype, int64_t T, int64_t h, const void *x, const void *residual, const void *gamma, float eps, int32_t columns,
                           void *xsum, void *out, float *scale, float *rstd, void *stream) {
  if (!x || !gamma || !out || !rstd || !scale || (residual && !xsum)) return MTNLG_NULL_POINTER;
  MTNLG_TRY(check_norm(dtype, T, h));
  if (!(eps >= 0.0f && eps < INFINITY) || unaligned({x, residual, gamma, xsum}) || ((uintptr_t)out & 7) || (((uintptr_t)rstd | (uintptr_t)scale) & 3))
    return MTNLG_INVALID_ARG;
  if (columns != 0 && (columns < 8 || columns > 512 || (columns & (columns - 1)))) return MTNLG_INVALID_ARG;
  const NormArgs a{T, (int)h, x, residual, gamma, xsum, out, eps, rstd, scale, columns, columns ? (int)((h + columns - 1) / columns) : 1};
  return dtype == MTNLG_F32 ? fwd_launch<float, true>(a, (hipStream_t)stream) : fwd_launch<bf16, true>(a, (hipStream_t)stream);
}

size_t mtnlg_rmsnorm_bwd_workspace(int64_t T, int64_t h) {
  if (check_norm(MTNLG_F32, T, h) != MTNLG_OK) return 0;
  return (size_t)bwd_groups(T, (int)h) * h * sizeof(float);
}

int mtnlg_rmsnorm_bwd(int dtype, int64_t T, int64_t h, const void *x, const void *gamma, const float *rstd, const void *dout, const void *dres,
                      void *dx, void *dgamma, int grad_f32, int accumulate, void *workspace, size_t workspace_bytes, void *stream) {
  if (!x || !gamma || !rstd || !dout || !dx || !dgamma || !workspace) return MTNLG_NULL_POINTER;
  MTNLG_TRY(check_norm(dtype, T, h));
  if (unaligned({x, gamma, dout, dres, dx, dgamma, workspace}) || ((uintptr_t)rstd & 3)) return MTNLG_INVALID_ARG;
  if (workspace_bytes < mtnlg_rmsnorm_bwd_workspace(T, h)) return MTNLG_WORKSPACE_TOO_SMALL;
  const NormBwdArgs a{T, (int)h, x, gamma, dout, dres, rstd, dx, (float *)workspace};
  return dtype == MTNLG_F32 ? bwd_launch<float>(a, dgamma, grad_f32, accumulate ? 1 : 0, (hipStream_t)stream)
                            : bwd_launch<bf16>(a, dgamma, grad_f32, accumulate ? 1 : 0, (hipStream_t)stream);
}

}  // extern "C"
