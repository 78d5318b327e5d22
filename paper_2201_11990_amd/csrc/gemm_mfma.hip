// bf16 GEMM on the gfx950 matrix cores, fp32 accumulate:  C[M,N] = op(A) * op(B).
//
// One kernel, gemm_stream_kernel: v_mfma_f32_16x16x32_bf16, both operands moved global -> LDS by DMA through a ring of stages
// with the loads spread over the slab, transposing LDS reads for row-contiguous operands.  Described at its definition.
//   256 x 256 and 256 x 320 tiles on 2 x 4 waves for aligned problems (M a multiple of 256, N of the tile width, K of 64 --
//   every GEMM of the MT-NLG slice); 256 x 256 with ragged edges; 128 x 128 on 2 x 2 waves with ragged edges and short or
//   deep rings, for problems with too few large tiles to fill the chip.
// gemm_mfma_pick_tile chooses per problem.  Ragged problems: any M, N a multiple of 8, K a multiple of 8 where an operand
// is K-contiguous and anything in the weight-gradient form, whose M is a multiple of 8 (16-byte accesses never straddle
// a row's end).
//
// Workgroups are numbered so that the 8 XCDs (workgroup id mod 8) each own a contiguous run of
// column-major tiles: neighbours in an XCD's L2 share A and B panels.
#include "gemm_stream.h"

namespace mtnlg {

namespace {

// Relative cost per FLOP of the wider streaming tile against 256 x 256 (measured on the MT-NLG slice's shapes).
constexpr double GEMM_COST_256x320 = 0.97;

template <bool AT, bool BT>
int launch_tile(int tile, const GemmArgs &g, void *ws, size_t ws_bytes, hipStream_t st) {
  switch (tile) {
    case GEMM_TILE_STREAM_256x256: return launch_stream<256, 256, 2, 4, 0, AT, BT, false>(g, ws, ws_bytes, st);
    case GEMM_TILE_STREAM_256x320: return launch_stream<256, 320, 2, 4, 0, AT, BT, false>(g, ws, ws_bytes, st);
    case GEMM_TILE_RAGGED_256: return launch_stream<256, 256, 2, 4, 0, AT, BT, true>(g, ws, ws_bytes, st);
    case GEMM_TILE_RAGGED_128: return launch_stream<128, 128, 2, 2, 0, AT, BT, true>(g, ws, ws_bytes, st);
    case GEMM_TILE_RAGGED_128_DEEP: return launch_stream<128, 128, 2, 2, 4, AT, BT, true>(g, ws, ws_bytes, st);
    default: return MTNLG_INVALID_ARG;
  }
}

// Estimated microseconds of a problem with nk 64-k slabs on each kind of tile: fits to measurements between 256 and 8192
// rows and columns, K 256 to 8192, weights not in the caches, one MI355X.
//   256 x 256: 1.45 us a slab and 8 per round of 256 tiles; a last round split along K has fewer slabs, and its fp32
//     partial tiles (256 KB each, written and read once) cost 0.05 us apiece.  256 x 320: 25 % more area at 0.97 of the
//     cost per FLOP.
//   128 x 128: twice the L2 -> LDS bytes per FLOP, which bounds it, so it is for problems with too few large tiles.  Short
//     rings: two workgroups a compute unit, 1.0 us a slab for a full round of 512; a lone workgroup (0.88) waits for its
//     DMA.  Rings of four stages: one workgroup a unit, 0.53 us a slab.
// Measured (us; 256 x 256, split along K where that pays / 128 x 128 / with deep rings): 2048^3 42 / 28 / 21,
// 1024 x 6144 x 2048 46 / 37 / 42, 2048 x 8192 x 2048 48 / 59 / 67, 256 x 960 x 512 13 / 9.3 / 7.5.  2048 x 2048 x 8192 75 / 71 / 62 (TN 75 / 70 / 65), where the estimates tie
// (71.2 and 72.3 for the first and last) and take the first: a slab of the deep rings is dearer here than it measures at long K (4096: 32 against 38 estimated).
double time_256(int64_t tiles, int nk, bool can_split, size_t ws_bytes) {
  const double slab = 1.45, round = 8.0;
  if (can_split) {
    const SplitPlan p = plan_split(tiles, nk, 256, 256, ws_bytes);
    if (p.tail > 0)
      return (double)(p.whole / 256) * (slab * nk + round) + slab * p.part_slabs + round + 4.0 + 0.05 * p.tail * p.split;
  }
  return (double)((tiles + 255) / 256) * (slab * nk + round);
}
double time_128(int64_t tiles, int nk) {
  const int64_t full = tiles / 512, rest = tiles % 512;
  return (double)full * (1.0 * nk + 6.0) + (rest == 0 ? 0.0 : rest <= 256 ? 0.88 * nk + 2.0 : 1.0 * nk + 6.0);
}
double time_128_deep(int64_t tiles, int nk) { return (double)((tiles + 255) / 256) * (0.53 * nk + 4.5); }

}  // namespace

// Which tile shape takes a problem: the least estimated time among those whose DMA reaches the operands, -1 if none does.  A last
// round is split along K if its partial tiles fit the workspace.
static int pick_tile(int layout, int64_t M, int64_t N, int64_t K, size_t ws_bytes, double &best) {
  best = 1e300;
  if (M <= 0 || N <= 0 || K <= 0) return -1;
  const int nk = (int)((K + BK - 1) / BK);
  const bool at = layout == MTNLG_GEMM_TN, bt = layout != MTNLG_GEMM_NT;
  int pick = -1;
  auto offer = [&](int tile, int bm, int bn, double t) {
    if (t < best && tile_reaches(at, bt, M, N, K, bm, bn)) { best = t; pick = tile; }
  };
  auto tiles = [&](int64_t bm, int64_t bn) { return ((M + bm - 1) / bm) * ((N + bn - 1) / bn); };
  const bool aligned = K % BK == 0 && M % 256 == 0;
  offer(aligned && N % 256 == 0 ? GEMM_TILE_STREAM_256x256 : GEMM_TILE_RAGGED_256, 256, 256,
        time_256(tiles(256, 256), nk, true, ws_bytes));
  if (aligned && N % 320 == 0)
    offer(GEMM_TILE_STREAM_256x320, 256, 320, time_256(tiles(256, 320), nk, false, 0) * 1.25 * GEMM_COST_256x320);
  offer(GEMM_TILE_RAGGED_128, 128, 128, time_128(tiles(128, 128), nk));
  offer(GEMM_TILE_RAGGED_128_DEEP, 128, 128, time_128_deep(tiles(128, 128), nk));
  return pick;
}
int gemm_mfma_pick_tile(int layout, int64_t M, int64_t N, int64_t K, size_t ws_bytes) {
  double t;
  return pick_tile(layout, M, N, K, ws_bytes, t);
}
double gemm_mfma_time(int layout, int64_t M, int64_t N, int64_t K, size_t ws_bytes) {
  double t;
  const int tile = pick_tile(layout, M, N, K, ws_bytes, t);
  return tile == GEMM_TILE_RAGGED_128 ? t + 1.5 : t;   // its few-slab launches take that much longer than the choice between tiles needs to know
}

// Room for the partial tiles of a 256 x 256 tiling's split last round.  What callers size their scratch by, so it
// does not follow every choice of gemm_mfma_pick_tile: a problem that another tile takes may use none of it.  Aligned
// problems of a width that only 320 divides, and those that 256 x 320 tiles cover in less area of whole rounds, ask for none
// (with more than is asked for, 256 x 960 x 8192 would be split on ragged 256 x 256 tiles: estimated 37 us, 72 without).
size_t gemm_mfma_workspace_bytes(int64_t M, int64_t N, int64_t K) {
  if (M <= 0 || N <= 0 || K <= 0) return 0;
  const int64_t tiles256 = ((M + 255) / 256) * ((N + 255) / 256);
  const SplitPlan plan = plan_split(tiles256, (int)((K + BK - 1) / BK), 256, 256, 0);
  if (K % BK == 0 && M % 256 == 0 && N % 320 == 0) {
    const int64_t tiles320 = (M / 256) * (N / 320);
    if (N % 256 || (double)((tiles320 + 255) / 256) * 1.25 * GEMM_COST_256x320 < (double)tiles256 / 256 + 0.15) return 0;
  }
  return plan.workspace;
}

int gemm_mfma_bf16(int layout, int64_t M, int64_t N, int64_t K, const void *A, const void *B, void *C,
                   const void *bias, void *aux, uint32_t epi, void *ws, size_t ws_bytes, hipStream_t stream,
                   int prof_class, int tile) {
  if ((layout != MTNLG_GEMM_TN && K % 8) || N % 8) return MTNLG_UNSUPPORTED_SHAPE;   // rows of 16-byte units
  const bool at = layout == MTNLG_GEMM_TN, bt = layout != MTNLG_GEMM_NT;
  if (at && M % 8) return MTNLG_UNSUPPORTED_SHAPE;
  if (((uintptr_t)A | (uintptr_t)B | (uintptr_t)C | (uintptr_t)bias | (uintptr_t)aux) & 3) return MTNLG_UNSUPPORTED_SHAPE;   // DMA: whole dwords
  GemmArgs g;
  g.M = M; g.N = N; g.K = K;
  g.A = (const bf16 *)A; g.B = (const bf16 *)B;
  g.lda = at ? M : K;
  g.ldb = bt ? N : K;
  g.C = C; g.ldc = N;
  g.ea = EpiArgs{bias, aux, epi};
  g.tiles_m = g.tiles_n = g.per_xcd = 0;
  g.whole_tiles = 0; g.split = 1; g.part_slabs = 0; g.partial = nullptr;
  if (tile < 0)
    tile = gemm_mfma_pick_tile(layout, M, N, K, ws != nullptr ? ws_bytes : 0);
  if (tile < 0) return MTNLG_UNSUPPORTED_SHAPE;
  LaunchScope scope(prof_class >= 0 ? prof_class : MTNLG_K_GEMM_NT + layout, stream);
  if (!at && !bt) return launch_tile<false, false>(tile, g, ws, ws_bytes, stream);
  if (!at && bt) return launch_tile<false, true>(tile, g, ws, ws_bytes, stream);
  return launch_tile<true, true>(tile, g, ws, ws_bytes, stream);
}

}  // namespace mtnlg
