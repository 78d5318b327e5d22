// The gated feed-forward block's products for few tokens (a model in use: the next token of some sequences), bf16: x [T, K] by weights [N, K].
//
// Every weight is used for at most 64 tokens, so its way from memory is all (h 20480, F 10240: 1.26 GB).  A workgroup has TN rows of weights and all
// tokens; its eight waves take every eighth slab of 64 k each, through stages of their own that DMA fills with whole 128-byte lines past the caches, so nothing
// waits for another wave before the sums meet in LDS, where they are added in wave order.  One token takes 122 us by 20480 x 20480 (6.9 TB/s) and 62 by
// 20480 x 10240; without the hint that goes past the caches 139 and 71, with fragments straight from memory to registers, 16 rows x 64 bytes an instruction, 180 and 87.
// The tokens come from the caches, once for every TN rows: what that costs beside the weights (28 % of their time times T / TN), and compute units that
// others wait for, is what the choice of TN goes by.  us by 20480 x 20480 / 20480 x 10240, 24 tokens, TN 32 / 48 / 80 / 96: 163 / 150 / 136 / 143, 84 / 78 / 75 / 79 (80: 256
// workgroups); on the 32 x 32 tiles of gemm_wave.hip 169 and 94.
#include <algorithm>

#include "gated.h"
#include "slab.h"

namespace mtnlg {

namespace {

constexpr int WAVES = 8;

struct TokenArgs {
  int T, N, K;
  const bf16 *x, *w;
  bf16 *out;
  EpiArgs ea;
};

// LDS of a wave: its stages, and then its partial tile
template <int NX, int TN, int STAGES>
constexpr int wave_bytes() {
  constexpr int stages = STAGES * (8 * NX + TN) * 128, tile = (NX + 1) / 2 * (TN / 16) * 1024;
  return stages > tile ? stages : tile;
}

// NX: groups of 8 tokens
template <int NX, int TN, int STAGES, int GATE>
__global__ __launch_bounds__(64 * WAVES) void gated_tokens_kernel(TokenArgs a) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  using SX = Slab<bf16, 8 * NX, false>;
  using SW = Slab<bf16, TN, false, GATE == GATE_FWD>;
  constexpr int MB = (NX + 1) / 2, NB = TN / 16, STAGE = SX::BYTES + SW::BYTES, SK = SX::SK, PENDING = (STAGES - 1) * (SX::NI + SW::NI);
  constexpr int MINE = wave_bytes<NX, TN, STAGES>();
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n0 = blockIdx.x * TN;
  const bf16 *W = a.w + (int64_t)(GATE == GATE_FWD ? n0 / 2 : n0) * a.K;
  const SX sx(a.K, a.T, lane);
  const SW sw(a.K, a.N - n0, lane, a.N / 2);
  char *const mine = smem + wave * MINE;
  const uint32_t lds = lds_address(mine);
  const int slabs = (a.K + SK - 1) / SK;
  // slab s into a stage; past the last one zeros, which no memory is read for (the wait below counts every stage's DMAs)
  auto fetch = [&](int s, int stage) {
    const int64_t k0 = (int64_t)(s < slabs ? s : slabs) * SK;
    sw.template fetch<true>(W, a.K, n0, k0, a.K, lds + stage * STAGE, lane);
    sx.fetch(a.x, a.K, 0, k0, a.K, lds + stage * STAGE + SW::BYTES, lane);
  };
  f32x4 acc[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < STAGES; ++i) fetch(wave + i * WAVES, i);
  int stage = 0;
  for (int s = wave; s < slabs; s += WAVES) {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(PENDING) : "memory");   // this wave's slab has landed
    Frag16<TN, false> wf;
    Frag16<16 * MB, false> xf;   // (beyond 8 NX tokens whatever lies behind the stage: the sums of those rows are not stored)
    wf.read(mine + stage * STAGE, lane);
    xf.read(mine + stage * STAGE + SW::BYTES, lane);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // ... and left the stage
    fetch(s + STAGES * WAVES, stage);
    stage = stage + 1 == STAGES ? 0 : stage + 1;
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)   // weights first: a lane ends up with four consecutive columns of one token
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf.v[j][kk], xf.v[i][kk], acc[i][j], 0, 0, 0);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  f32x4 *red = reinterpret_cast<f32x4 *>(smem);
  constexpr int PITCH = MINE / 16;   // vectors between two waves
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) red[wave * PITCH + (i * NB + j) * 64 + lane] = acc[i][j];
  __syncthreads();
#pragma unroll 1
  for (int v = wave; v < MB * NB; v += WAVES) {
    f32x4 sum = red[v * 64 + lane];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) sum += red[i * PITCH + v * 64 + lane];
    const int m = v / NB * 16 + r, n = n0 + v % NB * 16 + 4 * g;
    if (m < a.T && n < a.N) {
      if constexpr (GATE == GATE_FWD) gate_epilogue4<bf16, GATE_FWD>(a.ea, a.out, a.N, m, n, sum);
      else put4(a.out + (int64_t)m * a.N + n, sum);
    }
  }
}

template <int NX, int TN, int STAGES, int GATE>
int launch(const TokenArgs &a, hipStream_t st) {
  constexpr int smem = WAVES * wave_bytes<NX, TN, STAGES>() + NX % 2 * 1024;   // (odd: the last stage is read past its end)
  if constexpr (smem > 160 * 1024) {
    return MTNLG_UNSUPPORTED_SHAPE;
  } else {
    static unsigned long long attr_done = 0;
    int device;
    if (!attr_is_set(attr_done, &device)) {
      if (hipFuncSetAttribute((const void *)gated_tokens_kernel<NX, TN, STAGES, GATE>, hipFuncAttributeMaxDynamicSharedMemorySize, smem) != hipSuccess)
        return MTNLG_HIP_ERROR;
      attr_mark_set(attr_done, device);
    }
    gated_tokens_kernel<NX, TN, STAGES, GATE><<<(unsigned)((a.N + TN - 1) / TN), 64 * WAVES, smem, st>>>(a);
    return check_launch();
  }
}

// Tokens in the stages of a workgroup: so many groups of 8
int token_groups(int64_t T) { return T <= 8 ? 1 : T <= 16 ? 2 : T <= 32 ? 4 : T <= 48 ? 6 : 8; }

// Rows of weights to a workgroup, of 16 times 1 .. 6 the one with the least of: the tokens' share; stages that few slabs a wave leave waiting for memory
// (16384 x 2048 by 16 tokens, four slabs a wave: 64 rows 15.4 us, 16 rows 15.1, 32 rows 14.6); compute units that have more workgroups than others, half of
// which the memory's time hides where all workgroups are on the chip at once.
int rows_of(int64_t T, int64_t N, int64_t K) {
  const int nx = token_groups(T);
  int pick = 16;
  double best = 1e300;
  for (int tn = 16; tn <= 96; tn += 16) {
    const int bytes = WAVES * 128 * std::max(8 * nx + tn, (nx + 1) / 2 * (tn / 16) * 8);
    if (bytes > 160 * 1024) continue;
    const int64_t wgs = (N + tn - 1) / tn, most = (wgs + 255) / 256;
    const double uneven = (double)(most * 256) / (double)wgs, slabs = (double)K / (64 * WAVES);
    const double cost = (1.0 + 0.28 * (double)T / tn + 0.015 * tn / std::max(slabs, 1.0)) *
                        (most * bytes <= 160 * 1024 ? 1.0 + 0.4 * (uneven - 1.0) : uneven);
    if (cost < best) { best = cost; pick = tn; }
  }
  return pick;
}

template <int NX, int GATE>
int launch_rows(const TokenArgs &a, hipStream_t st) {
  switch (rows_of(a.T, a.N, a.K)) {
    // a second stage pays where a wave has many slabs, or the tokens are next to nothing (one and two stages: 2048 x 8192, one token 12.7 / 10.2 us; 16384 x 2048, 16 tokens 15.1 / 15.6)
    case 16: return a.T <= 8 || a.K >= 8 * 64 * WAVES ? launch<NX, 16, 2, GATE>(a, st) : launch<NX, 16, 1, GATE>(a, st);
    case 32: return launch<NX, 32, 1, GATE>(a, st);
    case 48: return launch<NX, 48, 1, GATE>(a, st);
    case 64: return launch<NX, 64, 1, GATE>(a, st);
    case 80: return launch<NX, 80, 1, GATE>(a, st);
    default: return launch<NX, 96, 1, GATE>(a, st);
  }
}
template <int GATE>
int launch_tokens(const TokenArgs &a, hipStream_t st) {
  switch (token_groups(a.T)) {
    case 1: return launch_rows<1, GATE>(a, st);
    case 2: return launch_rows<2, GATE>(a, st);
    case 4: return launch_rows<4, GATE>(a, st);
    case 6: return launch_rows<6, GATE>(a, st);
    default: return launch_rows<8, GATE>(a, st);
  }
}

}  // namespace

// Whether a product by T tokens belongs here: up to 32 always, up to 64 where many rows of weights are long or do not begin at whole lines (us, here / on
// gemm_wave.hip's tiles: 20480 x 10240 by 48 tokens 81 / 114, 16384 x 2048 17.5 / 17.6, 20160 x 2040 by 57 tokens 29 / 47; 2048 x 8192 by 48 19.3 / 17.2).
bool gated_tokens_takes(int64_t T, int64_t N, int64_t K) {
  return (T <= 32 || (T <= 64 && N >= 4096 && (N * K >= (int64_t)1 << 25 || K % 64))) && (96 + N / 2) * K * 2 < (int64_t)RECORDS - 256;
}

int gated_tokens_fwd(int kind, int64_t T, int64_t h, int64_t F, const void *x, const void *w_fc1, void *z, void *g, hipStream_t stream) {
  LaunchScope scope(MTNLG_K_GEMM_NT, stream);
  return launch_tokens<GATE_FWD>(TokenArgs{(int)T, (int)(2 * F), (int)h, (const bf16 *)x, (const bf16 *)w_fc1, (bf16 *)g, EpiArgs{nullptr, z, (uint32_t)kind}},
                                 stream);
}
int gated_tokens_out(int64_t T, int64_t h, int64_t F, const void *g, const void *w_fc2, void *y, hipStream_t stream) {
  LaunchScope scope(MTNLG_K_GEMM_NT, stream);
  return launch_tokens<GATE_NONE>(TokenArgs{(int)T, (int)h, (int)F, (const bf16 *)g, (const bf16 *)w_fc2, (bf16 *)y, EpiArgs{nullptr, nullptr, 0}}, stream);
}

}  // namespace mtnlg
