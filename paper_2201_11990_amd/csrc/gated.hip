// Gated feed-forward block: z = x w_fc1^T, g = act(z_a) * z_b, y = g w_fc2^T and its adjoint.
#include <algorithm>

#include "common.h"

namespace mtnlg {

namespace {

// The activation of fp32 x and its slope
__device__ __forceinline__ void gate_of(int kind, float x, float &a, float &da) {
  if (kind == MTNLG_GATE_SILU) {
    const float s = 1.0f / (1.0f + expf(-x));
    a = x * s;
    da = s * (1.0f + x * (1.0f - s));
  } else {
    a = gelu_f(x, kind == MTNLG_GATE_GELU_ERF);
    da = gelu_grad_f(x, kind == MTNLG_GATE_GELU_ERF);
  }
}

template <typename E>
__global__ __launch_bounds__(256) void gate_fwd_kernel(int64_t T, int64_t F, int kind, const float *__restrict__ zf, E *__restrict__ z, E *__restrict__ g) {
  const int64_t n = T * (F / 8);
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < n; i += gridDim.x * 256ll) {
    const int64_t t = i / (F / 8), c = i % (F / 8) * 8;
    float a[8], b[8];
    load8(zf + t * 2 * F + c, a);
    load8(zf + t * 2 * F + F + c, b);
    if (z != nullptr) {
      store8(z + t * 2 * F + c, a);
      store8(z + t * 2 * F + F + c, b);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float v, d;
      gate_of(kind, a[e], v, d);
      a[e] = v * b[e];
    }
    store8(g + t * F + c, a);
  }
}
template <typename E>
__global__ __launch_bounds__(256) void gate_bwd_kernel(int64_t T, int64_t F, int kind, const E *__restrict__ z, const float *__restrict__ dg, E *__restrict__ dz) {
  const int64_t n = T * (F / 8);
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < n; i += gridDim.x * 256ll) {
    const int64_t t = i / (F / 8), c = i % (F / 8) * 8;
    float a[8], b[8], d[8];
    load8(z + t * 2 * F + c, a);
    load8(z + t * 2 * F + F + c, b);
    load8(dg + t * F + c, d);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float v, s;
      gate_of(kind, a[e], v, s);
      a[e] = d[e] * b[e] * s;
      b[e] = d[e] * v;
    }
    store8(dz + t * 2 * F + c, a);
    store8(dz + t * 2 * F + F + c, b);
  }
}

struct Sizes {
  int64_t T, h, F;
  int dtype, gate;
  size_t es, gemm_ws, inner;
};
int sizes_of(const mtnlg_gated_desc *d, Sizes *s) {
  if (!d) return MTNLG_NULL_POINTER;
  if ((d->dtype != MTNLG_F32 && d->dtype != MTNLG_BF16) || d->gate < MTNLG_GATE_SILU || d->gate > MTNLG_GATE_GELU_ERF || d->tokens <= 0 ||
      d->hidden <= 0 || d->ffn <= 0 || (d->flags & ~(MTNLG_ACCUMULATE_WGRAD | MTNLG_WGRAD_FP32)))
    return MTNLG_INVALID_ARG;
  if (d->tokens > GEMM_GENERIC_MAX_ROWS || d->hidden % 8 || d->hidden > 32768 || d->ffn % 8 || d->ffn > (1 << 20)) return MTNLG_UNSUPPORTED_SHAPE;
  *s = Sizes{d->tokens, d->hidden, d->ffn, d->dtype, d->gate, d->dtype == MTNLG_F32 ? (size_t)4 : 2, 0, 0};
  auto need = [&](int layout, int64_t M, int64_t N, int64_t K) { s->gemm_ws = std::max(s->gemm_ws, mtnlg_gemm_workspace(s->dtype, layout, M, N, K)); };
  need(MTNLG_GEMM_NT, s->T, 2 * s->F, s->h);
  need(MTNLG_GEMM_NT, s->T, s->h, s->F);
  need(MTNLG_GEMM_NN, s->T, s->F, s->h);
  need(MTNLG_GEMM_NN, s->T, s->h, 2 * s->F);
  need(MTNLG_GEMM_TN, 2 * s->F, s->h, s->T);
  need(MTNLG_GEMM_TN, s->h, s->F, s->T);
  s->gemm_ws = align_up(s->gemm_ws, 256);
  s->inner = align_up((size_t)(s->T * 2 * s->F) * 4, 256);
  return MTNLG_OK;
}

struct Bytes {
  const void *p;
  size_t n;
};
// Whether what is written lies on nothing else (null pointers aside)
bool lies_apart(const Bytes *out, int outs, const Bytes *in, int ins) {
  auto on = [](const Bytes &a, const Bytes &b) { return a.p && b.p && (uintptr_t)a.p < (uintptr_t)b.p + b.n && (uintptr_t)b.p < (uintptr_t)a.p + a.n; };
  for (int i = 0; i < outs; ++i) {
    for (int j = 0; j < i; ++j)
      if (on(out[i], out[j])) return false;
    for (int j = 0; j < ins; ++j)
      if (on(out[i], in[j])) return false;
  }
  return true;
}

unsigned grid_of(const Sizes &s) { return (unsigned)std::min<int64_t>((s.T * (s.F / 8) + 255) / 256, 8192); }

}  // namespace

}  // namespace mtnlg

using namespace mtnlg;

extern "C" {

size_t mtnlg_gated_ffn_workspace(const mtnlg_gated_desc *desc) {
  Sizes s;
  return sizes_of(desc, &s) == MTNLG_OK ? s.gemm_ws + s.inner : 0;
}

int mtnlg_gated_ffn_fwd(const mtnlg_gated_desc *desc, const void *x, const void *w_fc1, const void *w_fc2, void *z, void *g, void *y,
                        void *workspace, size_t workspace_bytes, void *stream) {
  Sizes s;
  MTNLG_TRY(sizes_of(desc, &s));
  const size_t need = mtnlg_gated_ffn_workspace(desc);
  if (!x || !w_fc1 || !w_fc2 || !g || !y || (need && !workspace)) return MTNLG_NULL_POINTER;
  if (((uintptr_t)x | (uintptr_t)w_fc1 | (uintptr_t)w_fc2 | (uintptr_t)z | (uintptr_t)g | (uintptr_t)y | (uintptr_t)workspace) & 15) return MTNLG_INVALID_ARG;
  const size_t th = s.T * s.h * s.es, tf = s.T * s.F * s.es, w = s.h * s.F * s.es;
  const Bytes out[] = {{z, 2 * tf}, {g, tf}, {y, th}, {workspace, need}}, in[] = {{x, th}, {w_fc1, 2 * w}, {w_fc2, w}};
  if (!lies_apart(out, 4, in, 3)) return MTNLG_INVALID_ARG;
  if (workspace_bytes < need) return MTNLG_WORKSPACE_TOO_SMALL;
  hipStream_t st = (hipStream_t)stream;
  float *zf = (float *)((char *)workspace + s.gemm_ws);
  MTNLG_TRY(mtnlg_gemm(s.dtype, MTNLG_GEMM_NT, s.T, 2 * s.F, s.h, x, w_fc1, zf, nullptr, nullptr, MTNLG_EPI_OUT_F32, workspace, s.gemm_ws, stream));
  {
    LaunchScope scope(MTNLG_K_GELU, st);
    if (s.dtype == MTNLG_F32) gate_fwd_kernel<float><<<grid_of(s), 256, 0, st>>>(s.T, s.F, s.gate, zf, (float *)z, (float *)g);
    else gate_fwd_kernel<bf16><<<grid_of(s), 256, 0, st>>>(s.T, s.F, s.gate, zf, (bf16 *)z, (bf16 *)g);
    MTNLG_TRY(check_launch());
  }
  return mtnlg_gemm(s.dtype, MTNLG_GEMM_NT, s.T, s.h, s.F, g, w_fc2, y, nullptr, nullptr, 0, workspace, s.gemm_ws, stream);
}

int mtnlg_gated_ffn_bwd(const mtnlg_gated_desc *desc, const void *x, const void *w_fc1, const void *w_fc2, const void *z, const void *g,
                        const void *dy, void *dz, void *dx, void *dw_fc1, void *dw_fc2, void *workspace, size_t workspace_bytes, void *stream) {
  Sizes s;
  MTNLG_TRY(sizes_of(desc, &s));
  const size_t need = mtnlg_gated_ffn_workspace(desc);
  if (!x || !w_fc1 || !w_fc2 || !z || !g || !dy || !dz || (need && !workspace)) return MTNLG_NULL_POINTER;
  if (((uintptr_t)x | (uintptr_t)w_fc1 | (uintptr_t)w_fc2 | (uintptr_t)z | (uintptr_t)g | (uintptr_t)dy | (uintptr_t)dz | (uintptr_t)dx |
       (uintptr_t)dw_fc1 | (uintptr_t)dw_fc2 | (uintptr_t)workspace) & 15)
    return MTNLG_INVALID_ARG;
  const bool wide = (desc->flags & MTNLG_WGRAD_FP32) != 0;
  const size_t th = s.T * s.h * s.es, tf = s.T * s.F * s.es, w = s.h * s.F * s.es, dw = s.h * s.F * (wide ? 4 : s.es);
  const Bytes out[] = {{dz, 2 * tf}, {dx, th}, {dw_fc1, 2 * dw}, {dw_fc2, dw}, {workspace, need}};
  const Bytes in[] = {{x, th}, {w_fc1, 2 * w}, {w_fc2, w}, {z, 2 * tf}, {g, tf}, {dy, th}};
  if (!lies_apart(out, 5, in, 6)) return MTNLG_INVALID_ARG;
  if (workspace_bytes < need) return MTNLG_WORKSPACE_TOO_SMALL;
  hipStream_t st = (hipStream_t)stream;
  const uint32_t epi = ((desc->flags & MTNLG_ACCUMULATE_WGRAD) ? (uint32_t)MTNLG_EPI_ACCUMULATE : 0u) | (wide ? (uint32_t)MTNLG_EPI_OUT_F32 : 0u);
  float *dg = (float *)((char *)workspace + s.gemm_ws);
  MTNLG_TRY(mtnlg_gemm(s.dtype, MTNLG_GEMM_NN, s.T, s.F, s.h, dy, w_fc2, dg, nullptr, nullptr, MTNLG_EPI_OUT_F32, workspace, s.gemm_ws, stream));
  {
    LaunchScope scope(MTNLG_K_GELU, st);
    if (s.dtype == MTNLG_F32) gate_bwd_kernel<float><<<grid_of(s), 256, 0, st>>>(s.T, s.F, s.gate, (const float *)z, dg, (float *)dz);
    else gate_bwd_kernel<bf16><<<grid_of(s), 256, 0, st>>>(s.T, s.F, s.gate, (const bf16 *)z, dg, (bf16 *)dz);
    MTNLG_TRY(check_launch());
  }
  if (dw_fc2) MTNLG_TRY(mtnlg_gemm(s.dtype, MTNLG_GEMM_TN, s.h, s.F, s.T, dy, g, dw_fc2, nullptr, nullptr, epi, workspace, s.gemm_ws, stream));
  if (dx) MTNLG_TRY(mtnlg_gemm(s.dtype, MTNLG_GEMM_NN, s.T, s.h, 2 * s.F, dz, w_fc1, dx, nullptr, nullptr, 0, workspace, s.gemm_ws, stream));
  if (dw_fc1) MTNLG_TRY(mtnlg_gemm(s.dtype, MTNLG_GEMM_TN, 2 * s.F, s.h, s.T, dz, x, dw_fc1, nullptr, nullptr, epi, workspace, s.gemm_ws, stream));
  return MTNLG_OK;
}

}  // extern "C"
