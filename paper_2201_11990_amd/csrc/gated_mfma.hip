// The two products of the gated feed-forward block that carry its activation, bf16, on the streaming kernel (gemm_stream.h): x w_fc1^T with
// act(gate) * other in the epilogue, and dy w_fc2 with the activation's backward.  z is written once and read once, dg never stored: 8192 tokens, h 2048, F 8192
// take 1897 us forward and backward (1304 TFLOP/s; with both in fp32 through memory and launches of their own for the activation 2246).  What bounds these two there: the matrix
// pipes (busy 65 and 49 % of the time; 80 in the products without the activation), and then HBM, which the epilogues of a round's tiles ask for all at once: 402 MB of z and g out cost some
// 55 us of 440, 536 MB of z in and dz out 97 of 289.
#include <math.h>

#include "gated.h"
#include "gemm_stream.h"

namespace mtnlg {

namespace {

template <bool BT, int EPI>
int launch_tile(int tile, const GemmArgs &g, void *ws, size_t ws_bytes, hipStream_t st) {
  switch (tile) {
    case GEMM_TILE_STREAM_256x256: return launch_stream<256, 256, 2, 4, 0, false, BT, false, EPI>(g, ws, ws_bytes, st);
    case GEMM_TILE_STREAM_256x320: return launch_stream<256, 320, 2, 4, 0, false, BT, false, EPI>(g, ws, ws_bytes, st);
    case GEMM_TILE_RAGGED_256: return launch_stream<256, 256, 2, 4, 0, false, BT, true, EPI>(g, ws, ws_bytes, st);
    case GEMM_TILE_RAGGED_128: return launch_stream<128, 128, 2, 2, 0, false, BT, true, EPI>(g, ws, ws_bytes, st);
    case GEMM_TILE_RAGGED_128_DEEP: return launch_stream<128, 128, 2, 2, 4, false, BT, true, EPI>(g, ws, ws_bytes, st);
    case GATED_SPLIT: return launch_stream<128, 128, 2, 2, 4, false, BT, true, EPI, true>(g, ws, ws_bytes, st);
    default: return MTNLG_UNSUPPORTED_SHAPE;
  }
}

}  // namespace

int gated_mfma_fwd(int kind, int64_t T, int64_t h, int64_t F, const void *x, const void *w_fc1, void *z, void *g, int tile, void *ws, size_t ws_bytes,
                   hipStream_t stream) {
  const GemmArgs a{T, 2 * F, h, (const bf16 *)x, (const bf16 *)w_fc1, h, h, g, F, EpiArgs{nullptr, z, (uint32_t)kind}, 0, 0, 0, 0, 1, 0, nullptr};
  LaunchScope scope(MTNLG_K_GEMM_NT, stream);
  return launch_tile<false, EPI_GATE_FWD>(tile, a, ws, ws_bytes, stream);
}

int gated_mfma_bwd(int kind, int64_t T, int64_t h, int64_t F, const void *dy, const void *w_fc2, const void *z, void *dz, int tile, void *ws,
                   size_t ws_bytes, hipStream_t stream) {
  const GemmArgs a{T, F, h, (const bf16 *)dy, (const bf16 *)w_fc2, h, F, dz, 2 * F, EpiArgs{nullptr, const_cast<void *>(z), (uint32_t)kind}, 0, 0, 0, 0, 1, 0,
                   nullptr};
  LaunchScope scope(MTNLG_K_GEMM_NN, stream);
  return launch_tile<true, EPI_GATE_BWD>(tile, a, ws, ws_bytes, stream);
}

// Products of few row and column tiles with long sums (of some hundred tokens, w_fc2's and dx from both halves of dz above all): on 128 x 128 tiles of which
// each is cut along K, so that all compute units have one.  us, 2048 columns, K 5464, 130 / 300 / 777 tokens: 22 / 28 / 40 against 22 / 30 / 52 on the tiles
// that mtnlg_gemm has for them; 4096 columns, K 11264, 100 / 200 tokens 29 / 39 against 43 / 44.
static SplitPlan split_plan(int64_t M, int64_t N, int64_t K, size_t ws_bytes) {
  return plan_split(((M + 127) / 128) * ((N + 127) / 128), (int)((K + BK - 1) / BK), 128, 128, ws_bytes);
}
size_t gated_split_workspace(int64_t M, int64_t N, int64_t K) { return split_plan(M, N, K, 0).workspace; }
// Estimated microseconds (fitted to 40 products of 70 to 1024 tokens, K 2816 to 11264: within 20 %), infinite for problems that are not cut as a whole
double gated_split_time(int64_t M, int64_t N, int64_t K, size_t ws_bytes) {
  const SplitPlan p = split_plan(M, N, K, ws_bytes);
  return p.tail > 0 && p.whole == 0 ? 11.0 + 0.42 * p.part_slabs + 0.03 * p.tail * p.split : INFINITY;
}
int gated_split(int layout, int64_t M, int64_t N, int64_t K, const void *A, const void *B, void *C, void *ws, size_t ws_bytes, hipStream_t stream) {
  const bool bt = layout == MTNLG_GEMM_NN;
  const GemmArgs a{M, N, K, (const bf16 *)A, (const bf16 *)B, K, bt ? N : K, C, N, EpiArgs{nullptr, nullptr, 0}, 0, 0, 0, 0, 1, 0, nullptr};
  LaunchScope scope(MTNLG_K_GEMM_NT + layout, stream);
  return bt ? launch_stream<128, 128, 2, 2, 4, false, true, true, EPI_FLAGS, true>(a, ws, ws_bytes, stream)
            : launch_stream<128, 128, 2, 2, 4, false, false, true, EPI_FLAGS, true>(a, ws, ws_bytes, stream);
}

}  // namespace mtnlg
