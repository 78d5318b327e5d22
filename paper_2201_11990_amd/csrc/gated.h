// Launchers of the gated feed-forward block's products that carry its activation (gate.h: what they do with their results).
#pragma once
#include "gate.h"

namespace mtnlg {

// Kernels that the block's products go to; of GATED_STREAM on with a gemm_tile, or GATED_SPLIT, added: 128 x 128, each cut along K (gated_split_time)
enum gated_kernel { GATED_PLAIN = 0, GATED_TOKENS, GATED_WAVE_32, GATED_WAVE_64, GATED_PARTS, GATED_GROUP_32, GATED_GROUP_64, GATED_STREAM = 16 };
constexpr int GATED_SPLIT = 8;

// The kernel that one of the block's products goes to: 0 z and g, 1 y, 2 dz, 3 dx (GATED_PLAIN: one of mtnlg_gemm's); with_dw: the gradient of the weight that dz or dx is
// worked out with is wanted too.  Negative: a status
int gated_path(const mtnlg_gated_desc *desc, int product, int with_dw);

// tile: a gemm_tile, or GATED_SPLIT
int gated_mfma_fwd(int kind, int64_t T, int64_t h, int64_t F, const void *x, const void *w_fc1, void *z, void *g, int tile, void *ws, size_t ws_bytes,
                   hipStream_t stream);
int gated_mfma_bwd(int kind, int64_t T, int64_t h, int64_t F, const void *dy, const void *w_fc2, const void *z, void *dz, int tile, void *ws,
                   size_t ws_bytes, hipStream_t stream);

// mode: GATE_FWD (A x, B w_fc1, C g) or GATE_BWD (A dy, B w_fc2, C dz); tile: 32 or 64
bool gated_wave_takes(int dtype, int64_t h, int64_t F);
int gated_wave(int dtype, int mode, int kind, int64_t T, int64_t h, int64_t F, const void *A, const void *B, void *z, void *C, int tile,
               hipStream_t stream);
int gated_wave_group(int dtype, const GemmCall &nn, const GemmCall &tn, int tile, hipStream_t stream);   // nn: the one with the gate's backward
int gated_parts(int mode, int kind, int64_t T, int64_t h, int64_t F, const void *A, const void *B, void *z, void *C, hipStream_t stream);

// few tokens, bf16: forward's products (N, K: rows and columns of the weights)
bool gated_tokens_takes(int64_t T, int64_t N, int64_t K);
int gated_tokens_fwd(int kind, int64_t T, int64_t h, int64_t F, const void *x, const void *w_fc1, void *z, void *g, hipStream_t stream);
int gated_tokens_out(int64_t T, int64_t h, int64_t F, const void *g, const void *w_fc2, void *y, hipStream_t stream);

// C = A B^T (NT) or A B (NN), bf16, on 128 x 128 tiles that are split along K where they leave compute units idle
size_t gated_split_workspace(int64_t M, int64_t N, int64_t K);
double gated_split_time(int64_t M, int64_t N, int64_t K, size_t ws_bytes);
int gated_split(int layout, int64_t M, int64_t N, int64_t K, const void *A, const void *B, void *C, void *ws, size_t ws_bytes, hipStream_t stream);

}  // namespace mtnlg
