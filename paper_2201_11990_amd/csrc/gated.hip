// Gated feed-forward block: z = x w_fc1^T, g = act(z_a) * z_b, y = g w_fc2^T and its adjoint, as matrix products that carry the activation:
//   forward   x w_fc1^T (act(gate) * other in the epilogue), g w_fc2^T
//   backward  dw_fc2 = dy^T g, dy w_fc2 (the activation's backward in the epilogue: dz), dx = dz w_fc1, dw_fc1 = dz^T x
// Bound by the matrix pipes from some hundred tokens on: 6 T h F operations forward and 12 backward, with z written and read once.  In small calls
// the products of one weight matrix's backward are one launch (gemm_wave.hip), so a step of 61 tokens is four: 25 us in fp32 (h 520, F 344), 39 in the seven that it was.
#include <algorithm>

#include "gated.h"

namespace mtnlg {

namespace {

struct Sizes {
  int64_t T, h, F;
  int dtype, gate;
  size_t es, gemm_ws;
};
int sizes_of(const mtnlg_gated_desc *d, Sizes *s) {
  if (!d) return MTNLG_NULL_POINTER;
  if ((d->dtype != MTNLG_F32 && d->dtype != MTNLG_BF16) || d->gate < MTNLG_GATE_SILU || d->gate > MTNLG_GATE_GELU_ERF || d->tokens <= 0 ||
      d->hidden <= 0 || d->ffn <= 0 || (d->flags & ~(MTNLG_ACCUMULATE_WGRAD | MTNLG_WGRAD_FP32)))
    return MTNLG_INVALID_ARG;
  if (d->tokens > GEMM_GENERIC_MAX_ROWS || d->hidden % 8 || d->hidden > 32768 || d->ffn % 8 || d->ffn > (1 << 20)) return MTNLG_UNSUPPORTED_SHAPE;
  // 32-bit offsets reach both halves of w_fc1 from a tile's first row
  if ((int64_t)d->hidden * d->ffn > (d->dtype == MTNLG_F32 ? ((int64_t)1 << 30) - (1 << 22) : ((int64_t)1 << 31) - (1 << 23))) return MTNLG_UNSUPPORTED_SHAPE;
  // a launch is of less than 2^32 work items: in parts, 512 to a tile of 128 x 128 (what bf16 takes for so many columns has fewer, and memory ends before)
  if (d->dtype == MTNLG_F32 && ((d->tokens + 127) / 128) * ((2 * (int64_t)d->ffn + 127) / 128) >= (int64_t)1 << 23) return MTNLG_UNSUPPORTED_SHAPE;
  *s = Sizes{d->tokens, d->hidden, d->ffn, d->dtype, d->gate, d->dtype == MTNLG_F32 ? (size_t)4 : 2, 0};
  auto need = [&](int layout, int64_t M, int64_t N, int64_t K) { s->gemm_ws = std::max(s->gemm_ws, mtnlg_gemm_workspace(s->dtype, layout, M, N, K)); };
  need(MTNLG_GEMM_NT, s->T, 2 * s->F, s->h);
  need(MTNLG_GEMM_NT, s->T, s->h, s->F);
  need(MTNLG_GEMM_NN, s->T, s->F, s->h);
  need(MTNLG_GEMM_NN, s->T, s->h, 2 * s->F);
  need(MTNLG_GEMM_TN, 2 * s->F, s->h, s->T);
  need(MTNLG_GEMM_TN, s->h, s->F, s->T);
  if (s->dtype == MTNLG_BF16)
    s->gemm_ws = std::max({s->gemm_ws, gated_split_workspace(s->T, s->h, s->F), gated_split_workspace(s->T, s->h, 2 * s->F),
                           gated_split_workspace(s->T, 2 * s->F, s->h), gated_split_workspace(s->T, s->F, s->h)});
  s->gemm_ws = align_up(s->gemm_ws, 256);
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

// Whether a bf16 product is estimated to be fastest on tiles that are cut along K (rows that do not begin at whole lines cost the 32 and 64 tiles of
// gemm_wave.hip a third more than their estimate)
bool cut_along_k(const Sizes &s, int layout, int64_t M, int64_t N, int64_t K) {
  const double split = gated_split_time(M, N, K, s.gemm_ws);
  return split < gemm_time(s.dtype, layout, M, N, K, s.gemm_ws) && !gemm_wave_pick(s.dtype, layout, M, N, K, split / (K % 64 ? 1.35 : 1.0)) &&
         (int64_t)128 * (2 * K + N) * 2 < ((int64_t)1 << 31);   // (what 32-bit offsets reach, with room)
}
// One of the two products that carry the activation, on the kernel that is estimated to be the fastest
double gated_time(const Sizes &s, int mode) {
  const int layout = mode == GATE_FWD ? MTNLG_GEMM_NT : MTNLG_GEMM_NN;
  const int64_t N = mode == GATE_FWD ? 2 * s.F : s.F;
  return s.dtype == MTNLG_F32 ? gemm_parts_time(s.T, N, s.h) : gemm_mfma_time(layout, s.T, N, s.h, s.gemm_ws);
}
int gated_pick(const Sizes &s, int mode) {
  const int layout = mode == GATE_FWD ? MTNLG_GEMM_NT : MTNLG_GEMM_NN;
  const int64_t N = mode == GATE_FWD ? 2 * s.F : s.F;
  if (s.dtype == MTNLG_BF16 && mode == GATE_FWD && gated_tokens_takes(s.T, N, s.h)) return GATED_TOKENS;
  if (s.dtype == MTNLG_BF16 && cut_along_k(s, layout, s.T, N, s.h)) return GATED_STREAM + GATED_SPLIT;
  if (const int tile = gemm_wave_pick(s.dtype, layout, s.T, N, s.h, gated_time(s, mode))) return tile == 32 ? GATED_WAVE_32 : GATED_WAVE_64;
  return s.dtype == MTNLG_F32 ? (int)GATED_PARTS : GATED_STREAM + gemm_mfma_pick_tile(layout, s.T, N, s.h, s.gemm_ws);
}
int gated_product(const Sizes &s, int mode, int kernel, const void *A, const void *B, void *z, void *C, void *ws, hipStream_t st) {
  if (kernel == GATED_TOKENS) return gated_tokens_fwd(s.gate, s.T, s.h, s.F, A, B, z, C, st);
  if (kernel == GATED_WAVE_32 || kernel == GATED_WAVE_64)
    return gated_wave(s.dtype, mode, s.gate, s.T, s.h, s.F, A, B, z, C, kernel == GATED_WAVE_32 ? 32 : 64, st);
  if (kernel == GATED_PARTS) return gated_parts(mode, s.gate, s.T, s.h, s.F, A, B, z, C, st);
  return mode == GATE_FWD ? gated_mfma_fwd(s.gate, s.T, s.h, s.F, A, B, z, C, kernel - GATED_STREAM, ws, s.gemm_ws, st)
                          : gated_mfma_bwd(s.gate, s.T, s.h, s.F, A, B, z, C, kernel - GATED_STREAM, ws, s.gemm_ws, st);
}

// The tile of a launch of both products of a weight's backward (of sizes [M, N, K]), 0 where launches of their own are estimated to be faster; the estimate does not
// know of rows that begin amid lines, which cost long launches a third (7473 tokens, h 2680, F 560: 144 us for what two launches take 112 for)
int one_launch(const Sizes &s, double nn_time, const int64_t (&nn)[3], const int64_t (&tn)[3]) {
  auto call = [](const int64_t (&n)[3]) { return GemmCall{n[0], n[1], n[2], nullptr, nullptr, nullptr, nullptr, 0}; };   // (all matrices are aligned)
  const double tn_time = gemm_time(s.dtype, MTNLG_GEMM_TN, tn[0], tn[1], tn[2], s.gemm_ws);
  const double less = s.dtype == MTNLG_BF16 && (s.h % 64 || s.F % 64) && nn_time + tn_time > 50.0 ? 1.0 / 1.35 : 1.0;
  return gemm_wave_group_tile(s.dtype, call(nn), call(tn), 0, 0, 0, nn_time * less, tn_time * less);
}

// The kernel of a product: z and g, y, dz, dx; with_dw: of a backward one whose weight's gradient is wanted too
enum Product { TO_G = 0, TO_Y, TO_DZ, TO_DX };
int path_of(const Sizes &s, int product, bool with_dw) {
  if (with_dw && product >= TO_DZ) {
    const int tile = product == TO_DZ ? one_launch(s, gated_time(s, GATE_BWD), {s.T, s.F, s.h}, {s.h, s.F, s.T})
                                      : one_launch(s, gemm_time(s.dtype, MTNLG_GEMM_NN, s.T, s.h, 2 * s.F, s.gemm_ws), {s.T, s.h, 2 * s.F}, {2 * s.F, s.h, s.T});
    if (tile) return tile == 32 ? GATED_GROUP_32 : GATED_GROUP_64;
  }
  if (product == TO_G || product == TO_DZ) return gated_pick(s, product == TO_G ? GATE_FWD : GATE_BWD);
  if (s.dtype == MTNLG_F32) return GATED_PLAIN;
  if (product == TO_Y && gated_tokens_takes(s.T, s.h, s.F)) return GATED_TOKENS;
  const bool cut = product == TO_Y ? cut_along_k(s, MTNLG_GEMM_NT, s.T, s.h, s.F) : cut_along_k(s, MTNLG_GEMM_NN, s.T, s.h, 2 * s.F);
  return cut ? GATED_STREAM + GATED_SPLIT : (int)GATED_PLAIN;
}

}  // namespace

int gated_path(const mtnlg_gated_desc *desc, int product, int with_dw) {
  Sizes s;
  MTNLG_TRY(sizes_of(desc, &s));
  return path_of(s, product, with_dw != 0);
}

}  // namespace mtnlg

using namespace mtnlg;

extern "C" {

size_t mtnlg_gated_ffn_workspace(const mtnlg_gated_desc *desc) {
  Sizes s;
  return sizes_of(desc, &s) == MTNLG_OK ? s.gemm_ws : 0;
}

int mtnlg_gated_ffn_fwd(const mtnlg_gated_desc *desc, const void *x, const void *w_fc1, const void *w_fc2, void *z, void *g, void *y,
                        void *workspace, size_t workspace_bytes, void *stream) {
  Sizes s;
  MTNLG_TRY(sizes_of(desc, &s));
  const size_t need = s.gemm_ws;
  if (!x || !w_fc1 || !w_fc2 || !g || !y || (need && !workspace)) return MTNLG_NULL_POINTER;
  if (((uintptr_t)x | (uintptr_t)w_fc1 | (uintptr_t)w_fc2 | (uintptr_t)z | (uintptr_t)g | (uintptr_t)y | (uintptr_t)workspace) & 15) return MTNLG_INVALID_ARG;
  const size_t th = s.T * s.h * s.es, tf = s.T * s.F * s.es, w = s.h * s.F * s.es;
  const Bytes out[] = {{z, 2 * tf}, {g, tf}, {y, th}, {workspace, need}}, in[] = {{x, th}, {w_fc1, 2 * w}, {w_fc2, w}};
  if (!lies_apart(out, 4, in, 3)) return MTNLG_INVALID_ARG;
  if (workspace_bytes < need) return MTNLG_WORKSPACE_TOO_SMALL;
  hipStream_t st = (hipStream_t)stream;
  MTNLG_TRY(gated_product(s, GATE_FWD, path_of(s, TO_G, false), x, w_fc1, z, g, workspace, st));
  const int to_y = path_of(s, TO_Y, false);
  if (to_y == GATED_TOKENS) return gated_tokens_out(s.T, s.h, s.F, g, w_fc2, y, st);
  if (to_y != GATED_PLAIN) return gated_split(MTNLG_GEMM_NT, s.T, s.h, s.F, g, w_fc2, y, workspace, s.gemm_ws, st);
  return mtnlg_gemm(s.dtype, MTNLG_GEMM_NT, s.T, s.h, s.F, g, w_fc2, y, nullptr, nullptr, 0, workspace, s.gemm_ws, stream);
}

int mtnlg_gated_ffn_bwd(const mtnlg_gated_desc *desc, const void *x, const void *w_fc1, const void *w_fc2, const void *z, const void *g,
                        const void *dy, void *dz, void *dx, void *dw_fc1, void *dw_fc2, void *workspace, size_t workspace_bytes, void *stream) {
  Sizes s;
  MTNLG_TRY(sizes_of(desc, &s));
  const size_t need = s.gemm_ws;
  if (!x || !w_fc1 || !w_fc2 || !z || !g || !dy || !dz || (need && !workspace)) return MTNLG_NULL_POINTER;
  if (((uintptr_t)x | (uintptr_t)w_fc1 | (uintptr_t)w_fc2 | (uintptr_t)z | (uintptr_t)g | (uintptr_t)dy | (uintptr_t)dz | (uintptr_t)dx |
       (uintptr_t)dw_fc1 | (uintptr_t)dw_fc2 | (uintptr_t)workspace) & 15)
    return MTNLG_INVALID_ARG;
  const bool wide = s.dtype == MTNLG_BF16 && (desc->flags & MTNLG_WGRAD_FP32) != 0;
  const size_t th = s.T * s.h * s.es, tf = s.T * s.F * s.es, w = s.h * s.F * s.es, dw = s.h * s.F * (wide ? 4 : s.es);
  const Bytes out[] = {{dz, 2 * tf}, {dx, th}, {dw_fc1, 2 * dw}, {dw_fc2, dw}, {workspace, need}};
  const Bytes in[] = {{x, th}, {w_fc1, 2 * w}, {w_fc2, w}, {z, 2 * tf}, {g, tf}, {dy, th}};
  if (!lies_apart(out, 5, in, 6)) return MTNLG_INVALID_ARG;
  if (workspace_bytes < need) return MTNLG_WORKSPACE_TOO_SMALL;
  hipStream_t st = (hipStream_t)stream;
  const uint32_t epi = ((desc->flags & MTNLG_ACCUMULATE_WGRAD) ? (uint32_t)MTNLG_EPI_ACCUMULATE : 0u) | (wide ? (uint32_t)MTNLG_EPI_OUT_F32 : 0u);
  auto gemm = [&](int layout, const GemmCall &c) {
    return mtnlg_gemm(s.dtype, layout, c.M, c.N, c.K, c.A, c.B, c.C, nullptr, nullptr, c.epi, workspace, s.gemm_ws, stream);
  };
  const GemmCall to_dz{s.T, s.F, s.h, dy, w_fc2, dz, const_cast<void *>(z), (uint32_t)s.gate}, to_dw2{s.h, s.F, s.T, dy, g, dw_fc2, nullptr, epi};
  const int dz_path = path_of(s, TO_DZ, dw_fc2 != nullptr);
  if (dz_path == GATED_GROUP_32 || dz_path == GATED_GROUP_64) {
    MTNLG_TRY(gated_wave_group(s.dtype, to_dz, to_dw2, dz_path == GATED_GROUP_32 ? 32 : 64, st));
  } else {
    if (dw_fc2) MTNLG_TRY(gemm(MTNLG_GEMM_TN, to_dw2));
    MTNLG_TRY(gated_product(s, GATE_BWD, dz_path, dy, w_fc2, const_cast<void *>(z), dz, workspace, st));
  }
  const GemmCall to_dx{s.T, s.h, 2 * s.F, dz, w_fc1, dx, nullptr, 0}, to_dw1{2 * s.F, s.h, s.T, dz, x, dw_fc1, nullptr, epi};
  if (dx) {
    const int dx_path = path_of(s, TO_DX, dw_fc1 != nullptr);
    if (dx_path == GATED_GROUP_32 || dx_path == GATED_GROUP_64)
      return gemm_wave_group(s.dtype, to_dx, to_dw1, ColumnSums{}, dx_path == GATED_GROUP_32 ? 32 : 64, st);
    if (dx_path != GATED_PLAIN) MTNLG_TRY(gated_split(MTNLG_GEMM_NN, s.T, s.h, 2 * s.F, dz, w_fc1, dx, workspace, s.gemm_ws, st));
    else MTNLG_TRY(gemm(MTNLG_GEMM_NN, to_dx));
  }
  if (dw_fc1) MTNLG_TRY(gemm(MTNLG_GEMM_TN, to_dw1));
  return MTNLG_OK;
}

}  // extern "C"
