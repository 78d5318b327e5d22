// Attention over packed sequences with grouped heads, backward, bf16 (packed_fwd.hip: forward).
//
//   D = da . a (of a row):  dP = da v^T,  dS = P o (dP - D),  dq = scale dS k;  of a head of keys, summed over the query heads that share it:
//   dk = scale sum dS^T q,  dv = sum P^T da
//
// Two kernels, in the order of attention_bwd.hip: dq (and D), which owns rows (token, head of the group) as the forward kernel does and streams K and V, and dk / dv, which owns
// keys and streams Q and dO of one head of the group after the other.  No atomics: where the keys alone leave units idle, the tiles of a block of keys (of all heads of the group, one
// head after the other) are dealt out in parts to several workgroups, whose sums packed.hip adds up in their order.  Keys that no query sees get zeros.
//
// P and dS round to bf16 before the products that sum them up (2^-8 of each term at most, as each result once more), since as three bf16 parts that keep all bits those products would be three times as long; D and
// all sums are fp32.  D is worked out from the stored a, which is rounded: forward keeps no other.  All in all dq and dk are off by 0.0025 to 0.0031 of their norm, 0.0017 of that by their own
// rounding.  (The dense kernels round P and dS at heads of 64, 128 and 160 only, and cut them into parts at others: 1024 keys, heads of 72 to 256, dq off by 0.0018 there and 0.0025 here.)
//
// Seven products, of which two (S and dP) are taken in both kernels: one kernel for all would add up either dq or dk and dv through atomics, whose
// order changes results, or through memory (a part of dq to every block of keys).  Four sequences of 384 to 9001 tokens, 32 heads of 128 on 8: dq 1110 us, 1.2 PFLOP/s, bound by the matrix
// pipes, which are busy 75 % of the time; dk / dv 1850 us, 0.95 PFLOP/s, 53 %, not by one thing alone.  Without its fragments' reads, DMA, exponentials and the exchange that loop took 1332 us of 2020, without one of the
// first two 1790 to 1850, without one of the others 1870 to 1970: nothing of it stands out.  Eight of 77 to 2048, 16 heads on 4: 98 and 160 us, pipes busy 47 and 41 %; 2501 and 1589 tokens, 16 heads of 160: 98 and 128 us, 46 and 44 %.
#include "packed.h"

namespace mtnlg {

namespace {

// ------------------------------------------------------------------ dq (and D)
constexpr int DQ_THREADS = 256;
template <int D> constexpr int dq_per_unit() { return D <= 160 ? 2 : 1; }
// SPLIT 2: 64 rows to a workgroup, waves 0, 1 take the first 32 keys of every tile, waves 2, 3 the last 32; SPLIT 1: 128 rows.
template <int D, int SPLIT>
__global__ __launch_bounds__(DQ_THREADS, dq_per_unit<D>()) void packed_dq_kernel(PackedBwdArgs w) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  using P = Elem<bf16, D>;
  using T = typename P::T;
  constexpr int OWNED = 128 / SPLIT;
  constexpr int K1 = D / 16, CB = D / 32, STAGE = 2 * T::BYTES;
  constexpr int SUBS = SPLIT == 2 ? 1 : 2;                // 32-row parts of a tile that a wave takes
  constexpr int N1 = 3 * K1, NF = D == 160 ? 5 : D == 64 ? 4 : 6, PF = NF - 1;   // steps of a part: K1 for S, K1 for dP, K1 for dq
  static_assert(N1 % NF == 0, "fragment buffers");
  const int lane = threadIdx.x & 63, h = lane >> 5, r = w.group, d = w.d;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int j = blockIdx.x % w.kv_heads;
  Span s;
  unsigned at;
  if (!find_piece(w.where, blockIdx.x / w.kv_heads, [&](const Span &s) { return (unsigned)((s.lq * r + OWNED - 1) / OWNED); }, s, at)) return;
  const int count = (s.lq * r + OWNED - 1) / OWNED, shift = s.lk - s.lq, block = count - 1 - at;   // falling work
  const int rows = s.lq * r, block0 = block * OWNED, last_row = min(block0 + OWNED, rows) - 1;
  const int end = max(0, min(s.lk, last_row / r + shift + 1)), ntiles = (end + 63) / 64;   // keys that the block sees

  const int part = SPLIT == 2 ? wave >> 1 : 0;
  const int own0 = block0 + (SPLIT == 2 ? wave & 1 : wave) * 32, mine = own0 + (lane & 31), row = min(mine, rows - 1);
  const int tok = row / r, g = row - tok * r, head = j * r + g;
  const int limit = min(tok + shift, s.lk - 1);
  const int least = __builtin_amdgcn_readfirstlane(limit), most = own0 < rows ? __builtin_amdgcn_readlane(limit, 31) : -1;
  const float f = w.scale * kLog2e;
  typename P::Lane ln(lane);
  ln.n0 += part * T::ROWS32;
  ln.t0 += part * T::ROWS32;
  const uint32_t smem_addr = lds_address(smem);

  constexpr int IPW = 2 * T::NI;
  const int half = wave >> 1;   // waves 0, 1 bring 32 rows each of K, waves 2, 3 of V
  const Heads &mat = half ? w.v : w.k;
  const int row0 = 32 * (wave & 1);
  RowWalk stream(row_at<bf16>(mat, s.k0 + row0, j, 0), end - row0, (uint32_t)(mat.token * 2), 64);   // from the wave's rows on
  const uint32_t dst0 = smem_addr + half * T::BYTES + (wave & 1) * (2 * T::NI * 1024);
  uint32_t dma_off[T::NI];   // of 16 rows: the next 16 lie the same in a descriptor of their own
#pragma unroll
  for (int i = 0; i < T::NI; ++i) dma_off[i] = T::dma_offset(stream.pitch, 0, lane, i, d);
  constexpr int ISSUE_STEPS = IPW / 2;   // (one tile ahead: it is waited for in the same iteration)
  auto issue_step = [&](int step, int st) {
#pragma unroll
    for (int i = 0; i < IPW; ++i)
      if (i >= (step ? dma_by<IPW, ISSUE_STEPS>(step - 1) : 0) && i < dma_by<IPW, ISSUE_STEPS>(step))
        dma16<Spread::value>(stream.tile<16>(16 * (i / T::NI)), dst0 + st * STAGE + i * 1024, dma_off[i % T::NI]);
  };
#pragma unroll
  for (int i = 0; i < IPW; ++i) dma16<Burst::value>(stream.tile<16>(16 * (i / T::NI)), dst0 + i * 1024, dma_off[i % T::NI]);
  stream.advance<64>();
  bf16x8 of0[K1], of1[K1];   // own rows of q and da: columns 16 kk + 8 h .. + 7
  float dsum = 0.0f;
  {
    const bf16 *qrow = row_at<bf16>(w.q, s.q0 + tok, j, g), *drow = row_at<bf16>(w.da, s.q0 + tok, j, g), *arow = row_at<bf16>(w.a, s.q0 + tok, j, g);
    bf16x8 av[K1];
#pragma unroll
    for (int kk = 0; kk < K1; ++kk) {
      av[kk] = row_unit<bf16, D>(arow, kk, h, d);
      of1[kk] = row_unit<bf16, D>(drow, kk, h, d);
      of0[kk] = row_unit<bf16, D>(qrow, kk, h, d);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int kk = 0; kk < K1; ++kk) {
      dsum = P::dot(av[kk], of1[kk], dsum);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  dsum += __shfl_xor(dsum, 32, 64);
  const int64_t stat = (int64_t)head * w.where.q_tokens + s.q0 + tok;
  if (mine < rows && h == 0 && part == 0) w.D[stat] = -dsum;   // as dP's accumulators start
  float lsf = w.lse[stat];
  lsf = lsf == -INFINITY ? INFINITY : lsf * kLog2e;   // a row that sees nothing: weights of 0
  float dneg = -dsum;
#pragma unroll
  for (int kk = 0; kk < K1; ++kk) {
    arrive(of0[kk]);
    arrive(of1[kk]);
  }
  arrive(lsf);
  arrive(dneg);
  f32x16 acc[CB];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) acc[cb] = f32x16{};
  bool redo = false;       // the wave has met keys that are not finite where a mask hides some
  wait_and_barrier<0>();   // tile 0 landed everywhere

  bf16x8 fr[NF];
  f32x16 sc, pc;   // pc accumulates dP - D
  bf16x8 x[2];
  auto load = [&](int i, const char *Kt) {   // the fragment of step i, of the tile in stage Kt
    const int sub = i / N1, r = i % N1;
    const char *k = Kt + sub * T::ROWS32;
    bf16x8 &v = fr[i % NF];
    if (r < K1) v = T::nat32(k, ln, r);
    else if (r < 2 * K1) v = T::nat32(k + T::BYTES, ln, r - K1);
    else v = T::tr32(k, ln, (r - 2 * K1) / 2, r % 2);
  };
#pragma unroll
  for (int i = 0; i < PF; ++i) load(i, smem);
  __builtin_amdgcn_sched_barrier(0);

  int cur = 0;
  auto tile = [&](auto TAKEN, auto MASKED, auto STAGE_OF, int it) __attribute__((always_inline)) {   // TAKEN: parts, SUBS or the first only; STAGE_OF: -1 as it comes
    constexpr int N = decltype(TAKEN)::value * N1;
    constexpr int FIXED = decltype(STAGE_OF)::value;
    if constexpr (FIXED < 0) ln.here();
    const int now = FIXED < 0 ? cur : FIXED, next = now ^ 1;   // stages of tiles it, it + 1
    const char *const K = smem + now * STAGE;
    auto step = [&](auto I) __attribute__((always_inline)) {
      constexpr int i = decltype(I)::value, sub = i / N1, r = i % N1;
      const int key0 = it * 64 + 32 * (part + sub);
      if (r == 0) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          sc[e] = 0.0f;
          pc[e] = dneg;
        }
      }
      // the vector work: weights over dP, dS^T = P^T o (dP^T - D) behind it
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        if (r == K1 + e * K1 / 16) sc[e] = fast_exp2(fmaf(sc[e], f, -lsf));
        if (r == 2 * K1) pc[e] *= sc[e];
      }
      if (r == 2 * K1) {
        if constexpr (decltype(MASKED)::value) {
          const int seen = limit - key0 - 4 * (lane_here() >> 5);
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (8 * (e / 4) + e % 4 > seen) pc[e] = 0.0f;
          redo |= rows_not_finite<bf16, D>(K + sub * T::ROWS32, ln);
        }
        x[0] = P::weights(pc, 0);
        x[1] = P::weights(pc, 1);
      }
      if (i == N - PF) wait_and_barrier<0>();   // all of tile `it` has been read; tile it + 1 landed everywhere
      load((i + PF) % N, smem + (i + PF < N ? now : next) * STAGE);
      if (i < ISSUE_STEPS) issue_step(i, next);
      const bf16x8 &v = fr[i % NF];
      if constexpr (r < K1) sc = MFMA32(v, of0[r], sc);
      else if constexpr (r < 2 * K1) pc = MFMA32(v, of1[r - K1], pc);
      else acc[(r - 2 * K1) / 2] = MFMA32(v, x[r % 2], acc[(r - 2 * K1) / 2]);
      __builtin_amdgcn_sched_barrier(0);
    };
    for_each_step(step, std::make_integer_sequence<int, N>{});
    stream.advance<64>();
    cur = next;
  };
  // 32-key parts with a key that a row of the wave sees, and of those the first ones, which all rows see whole: a loop without masks for them, which has fewer values
  // to keep.  The parts after them are passed over.
  auto parts_of = [&](int keys) { return SPLIT == 2 ? (keys / 32 + 1 - part) / 2 : keys / 32; };
  const int visible = max(0, parts_of(most + 32)), whole = parts_of(min(least, most) + 1) / SUBS;
  int it = 0;
  using Any = std::integral_constant<int, -1>;
  if constexpr (D <= 128) {   // in pairs, with the stages known (packed_fwd.hip): 1145 us, 1120 so; wider heads have no registers for it (heads of 160: 97 us, 112 so)
    for (; it + 1 < whole; it += 2) {
      tile(std::integral_constant<int, SUBS>{}, std::false_type{}, std::integral_constant<int, 0>{}, it);
      tile(std::integral_constant<int, SUBS>{}, std::false_type{}, std::integral_constant<int, 1>{}, it + 1);
    }
  }
  for (; it < whole; ++it) tile(std::integral_constant<int, SUBS>{}, std::false_type{}, Any{}, it);
  for (; it < visible / SUBS; ++it) tile(std::integral_constant<int, SUBS>{}, std::true_type{}, Any{}, it);
  if constexpr (SUBS == 2) {
    if (visible % 2) tile(std::integral_constant<int, 1>{}, std::true_type{}, Any{}, it++);
  }
  for (; it < ntiles; ++it) {   // passed over: its share of a later tile, and the barrier
#pragma unroll
    for (int i = 0; i < IPW; ++i) dma16<Burst::value>(stream.tile<16>(16 * (i / T::NI)), dst0 + (cur ^ 1) * STAGE + i * 1024, dma_off[i % T::NI]);
    wait_and_barrier<0>();
    stream.advance<64>();
    cur ^= 1;
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");   // the look-ahead tiles, which nobody uses

  // SPLIT 2: the two waves with the same rows each hand over half of their column blocks' elements (q 0, 1 or 2, 3) and finish the other half
  f32x4 *slots = reinterpret_cast<f32x4 *>(smem) + lane_here();
  if constexpr (SPLIT == 2) {
    int *const bad = reinterpret_cast<int *>(smem + 2 * 4 * CB * 1024);
    __syncthreads();   // the rings are no longer read
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int q = 0; q < 2; ++q) slots[((wave * CB + cb) * 2 + q) * 64] = part ? quarter_of(acc[cb], q) : quarter_of(acc[cb], 2 + q);
    if (lane_here() == 0) bad[wave] = redo;
    __syncthreads();
    redo |= __builtin_amdgcn_readfirstlane(bad[wave ^ 2]) != 0;
  }
  if (own0 >= rows) return;
  // where the row lies, worked out once more: registers less across the loop
  const int last = own0 + (lane_here() & 31), out_row = min(last, rows - 1), out_tok = out_row / r, out_g = out_row - out_tok * r, out_h = lane_here() >> 5;
  bf16 *const out = row_at<bf16>(w.dq, s.q0 + out_tok, j, out_g);
  if (redo) {   // key by key, without matrix instructions (packed_fwd.hip: why)
    if (part) return;
    float sum[K1][8];
#pragma unroll
    for (int kk = 0; kk < K1; ++kk)
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[kk][e] = 0.0f;
    const bf16 *qrow = row_at<bf16>(w.q, s.q0 + out_tok, j, out_g), *drow = row_at<bf16>(w.da, s.q0 + out_tok, j, out_g);
#pragma unroll 1
    for (int key = 0; key <= most; ++key) {
      const bf16 *kr = row_at<bf16>(w.k, s.k0 + key, j, 0), *vr = row_at<bf16>(w.v, s.k0 + key, j, 0);
      float sk = 0.0f, dp = 0.0f;
#pragma unroll
      for (int kk = 0; kk < K1; ++kk) {
        sk = P::dot(row_unit<bf16, D>(kr, kk, out_h, d), row_unit<bf16, D>(qrow, kk, out_h, d), sk);
        dp = P::dot(row_unit<bf16, D>(vr, kk, out_h, d), row_unit<bf16, D>(drow, kk, out_h, d), dp);
        __builtin_amdgcn_sched_barrier(0);   // few reads at once: no registers for more
      }
      sk += __shfl_xor(sk, 32, 64);
      dp += __shfl_xor(dp, 32, 64);
      if (key > out_tok + shift) continue;
      const float ds = fast_exp2(fmaf(sk, f, -lsf)) * (dp + dneg);
#pragma unroll
      for (int kk = 0; kk < K1; ++kk) {
        const bf16x8 k = row_unit<bf16, D>(kr, kk, out_h, d);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[kk][e] = fmaf(ds, (float)k[e], sum[kk][e]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (last >= rows) return;
#pragma unroll
    for (int kk = 0; kk < K1; ++kk)
#pragma unroll
      for (int e = 0; e < 8; e += 4)
        if (16 * kk + 8 * out_h < d) put4(out + 16 * kk + 8 * out_h + e, f32x4{sum[kk][e], sum[kk][e + 1], sum[kk][e + 2], sum[kk][e + 3]} * w.scale);
    return;
  }
  if (last >= rows) return;
  auto put = [&](int cb, int q, f32x4 v) {   // columns 32 cb + 8 q + 4 h .. + 3
    const int col = 32 * cb + 8 * q + 4 * out_h;
    if (col < d) put4(out + col, v * w.scale);
  };
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) {
    if constexpr (SPLIT == 2) {
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const f32x4 other = slots[(((wave ^ 2) * CB + cb) * 2 + q) * 64];
        if (part) put(cb, 2 + q, quarter_of(acc[cb], 2 + q) + other);
        else put(cb, q, quarter_of(acc[cb], q) + other);
      }
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) put(cb, q, quarter_of(acc[cb], q));
    }
  }
}

// ------------------------------------------------------------------ dk and dv
// Eight waves, two to a SIMD, in pairs (roles 0 and 1) of which each owns 32 keys and takes 32 rows of a tile: role 0 forms S and P and accumulates dv,
// role 1 forms dP and dS and accumulates dk.  P goes to role 1 through LDS in fp32.  The second product runs one tile behind, so that one barrier a tile serves the exchange as well.
// D up to 128: a workgroup owns 64 keys and takes tiles of 64 rows; the two pairs of a group of keys take one half each and are merged through LDS at the end.
// Wider ones: 128 keys and tiles of 32 rows (64 x 192 do not fit three times).  Both ways, median us, 64 / 128 keys: eight sequences of 77 to 2048 tokens, 16 heads of 128 on 4:
// 186 / 180 and 15 for the join of its tiles' parts, which 64 keys do without; four of 384 to 9001, 32 heads of 128 on 8: 1970 / 2051; 17, 64 and 130 tokens, 4 heads of
// 64 on 2: 13 / 17; 2501 and 1589 tokens, 16 heads of 160: 139 / 133.
template <int D> struct Dkv {
  static constexpr int OWNED = D <= 128 ? 64 : 128, PARTS = 128 / OWNED, PAIRS = 4, THREADS = 128 * PAIRS;
  static constexpr int ROWS = 32 * PARTS, GROUPS = OWNED / 32;
  static constexpr int MATRIX = ROWS * D * 2, STAGE = 2 * MATRIX + 512;   // Q tile, dO tile, 256 bytes each of lse and -D
  static constexpr int XCHG = PAIRS * 4096;                               // P of a tile
  static constexpr int RING = 4 * STAGE + 2 * XCHG <= 160 * 1024 ? 4 : 3, AHEAD = RING - 2;   // tiles in LDS, and fetched ahead
  static constexpr int BYTES = RING * STAGE + 2 * XCHG;
  static_assert(BYTES <= 160 * 1024, "");
};

template <int D>
__global__ __launch_bounds__(Dkv<D>::THREADS) void packed_dkv_kernel(PackedBwdArgs w) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  using P = Elem<bf16, D>;
  using T = typename P::T;
  using L = Dkv<D>;
  constexpr int OWNED = L::OWNED, PARTS = L::PARTS, PAIRS = L::PAIRS;
  constexpr int K1 = D / 16, CB = D / 32, STAGE = L::STAGE, RING = L::RING, AHEAD = L::AHEAD, ROWS = L::ROWS;
  constexpr int N = 2 * K1, NF = D == 128 ? 8 : D == 160 ? 10 : 4, PF = D == 128 ? 5 : D == 160 ? 6 : NF - 1;   // steps of a tile: K1 for the first product, K1 for the second of the tile before
  constexpr int HAND_OVER = N - PF;
  static_assert(N % NF == 0 && HAND_OVER >= K1, "");
  const int lane = threadIdx.x & 63, h = lane >> 5, r = w.group, d = w.d;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int j = blockIdx.x % w.kv_heads;
  Span s;
  unsigned at;
  if (!find_piece(w.where, blockIdx.x / w.kv_heads, [&](const Span &s) { return (unsigned)((s.lk + OWNED - 1) / OWNED * w.splits); }, s, at)) return;
  const int split = at % w.splits, block0 = (int)(at / w.splits) * OWNED, shift = s.lk - s.lq;
  const int part = PARTS == 2 ? wave >> 1 & 1 : 0, role = wave / PAIRS;
  const int own0 = block0 + (wave & (L::GROUPS - 1)) * 32, mine = own0 + (lane & 31), key = min(mine, s.lk - 1);
  const int first = max(0, block0 - shift) / ROWS * ROWS, tiles = s.lq > first ? (s.lq - first + ROWS - 1) / ROWS : 0;   // of a head: from the first query that sees the block on
  // The workgroup's part of the tiles of all heads of the group, one head after the other: n from tile t0 of head g0 on.
  const int n0 = (int)((int64_t)r * tiles * split / w.splits), n = (int)((int64_t)r * tiles * (split + 1) / w.splits) - n0;
  const int g0 = tiles ? n0 / tiles : 0, t0 = n0 - g0 * tiles;
  const float f = w.scale * kLog2e;
  typename P::Lane ln(lane);
  const uint32_t smem_addr = lds_address(smem);

  // The waves of role 0 bring the Q tile, those of role 1 the dO tile (bands of 16 rows, NI instructions each, dealt out over them; what does not come out even is brought twice), and
  // every wave the tile's lse values (even waves) or -D values (odd ones): all issue the same number of memory operations, which the counted waits rely on.
  constexpr int ALL = ROWS / 16 * T::NI, IPW = (ALL + PAIRS - 1) / PAIRS, OPS = IPW + 1;
  const int half = wave / PAIRS;
  const Heads &mat = half ? w.da : w.q;
  const uint32_t pitch = (uint32_t)(mat.token * 2);
  auto instruction = [&](int i) { return (wave % PAIRS + PAIRS * i) % ALL; };
  uint32_t dma_off[IPW];
#pragma unroll
  for (int i = 0; i < IPW; ++i) dma_off[i] = T::dma_offset(pitch, instruction(i) / T::NI, lane, instruction(i) % T::NI, d);
  auto rows_at = [&](int g, int row) { return RowWalk(row_at<bf16>(mat, s.q0 + row, j, g), s.lq - row, pitch, ROWS); };
  auto stats_at = [&](int g, int row) { return RowWalk((wave & 1 ? w.D : w.lse) + ((int64_t)(j * r + g) * w.where.q_tokens + s.q0 + row), s.lq - row, 4, ROWS); };
  RowWalk stream = rows_at(g0, first + t0 * ROWS), stats = stats_at(g0, first + t0 * ROWS);
  int to_come = tiles - t0, g_in = g0;   // tiles of the head g_in that have not been fetched
  auto issue_one = [&](auto tag, int st, int i) {   // i == IPW: the statistics (with tiles of 32 rows those of the next tile as well, unused)
    constexpr int TAG = decltype(tag)::value;
    const uint32_t stage = smem_addr + st * STAGE;
    if (i == IPW) dma4<TAG>(stats.tile<64>(), stage + 2 * L::MATRIX + (wave & 1) * 256, lane * 4);
    else dma16<TAG>(stream.tile<ROWS>(), stage + half * L::MATRIX + instruction(i < IPW ? i : 0) * 1024, dma_off[i < IPW ? i : 0]);
  };
  auto advance = [&] {
    stream.advance<ROWS>();
    stats.advance<ROWS>();
    if (--to_come == 0 && g_in + 1 < r) {   // the next head of the group
      to_come = tiles;
      stream = rows_at(++g_in, first);
      stats = stats_at(g_in, first);
    }
  };
  auto issue_tile = [&](int st) {
#pragma unroll
    for (int i = 0; i < OPS; ++i) issue_one(Burst{}, st, i);
    advance();
  };
  constexpr int ISSUE_STEPS = AHEAD == 1 ? (OPS + 1) / 2 : N - PF;   // (one tile ahead: it is waited for in the same iteration)
  auto issue_step = [&](int step, int st) {
#pragma unroll
    for (int i = 0; i < OPS; ++i)
      if (i >= (step ? dma_by<OPS, ISSUE_STEPS>(step - 1) : 0) && i < dma_by<OPS, ISSUE_STEPS>(step)) issue_one(Spread{}, st, i);
  };
  bool redo = false;   // the wave has met rows that are not finite where a mask hides some
  f32x16 acc[CB];      // dv (role 0) or dk (role 1)
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) acc[cb] = f32x16{};
  if (n > 0) {
#pragma unroll
    for (int t = 0; t < AHEAD; ++t) issue_tile(t);   // (past the last tile: rows past the end, zeros)
  }
  bf16x8 of[K1];   // own rows of K (role 0) or V
  {
    const bf16 *own = row_at<bf16>(role ? w.v : w.k, s.k0 + key, j, 0);
#pragma unroll
    for (int kk = 0; kk < K1; ++kk) of[kk] = row_unit<bf16, D>(own, kk, h, d);
#pragma unroll
    for (int kk = 0; kk < K1; ++kk) arrive(of[kk]);
  }
  // the loop, once for each role
  f32x4 *const xchg = reinterpret_cast<f32x4 *>(smem + RING * STAGE) + wave % PAIRS * 256 + lane;   // 4 x 64 of the pair
  auto run = [&](auto ROLE) __attribute__((always_inline)) {
    constexpr int me = decltype(ROLE)::value;
    ln.n0 += part * T::ROWS32;
    ln.t0 += part * T::ROWS32;
    constexpr int FIRST_AT = me ? L::MATRIX : 0, SECOND_AT = me ? 0 : L::MATRIX;   // S from Q, then dv from dO; dP from dO, then dk from Q
    int cur = 0, last = 0, odd = 0;   // stages of the tile and of the one before (of the first: its own); P's buffer
    auto after = [](int cur, int n) { return cur + n >= RING ? cur + n - RING : cur + n; };   // stage of tile it + n
    bf16x8 fr[NF];
    f32x16 sc, prev = {};   // S and P (role 0); dP - D of this tile and of the one before
    bf16x8 x[2], xn[2];     // the second product's operand: what is in use, and (role 0) the next
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[t][e] = (bf16)0.0f;
    auto load = [&](int r, const char *t) {   // the fragment of step r, from stage t
      if (r < K1) fr[r % NF] = T::nat32(t + FIRST_AT, ln, r);
      else fr[r % NF] = T::tr32(t + SECOND_AT, ln, (r - K1) / 2, r % 2);
    };
    auto take = [&](int buffer, f32x16 &p) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 v = xchg[buffer * (L::XCHG / 16) + q * 64];
#pragma unroll
        for (int e = 0; e < 4; ++e) p[4 * q + e] = v[e];
      }
    };
    // the first tile has none before it.  Its products are with zeros, P among them: LDS holds what was there before
    if constexpr (me == 1) {
#pragma unroll
      for (int q = 0; q < 4; ++q) xchg[(odd ^ 1) * (L::XCHG / 16) + q * 64] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    wait_and_barrier<(AHEAD - 1) * OPS>();   // tile 0 landed everywhere
    redo |= rows_not_finite<bf16, D>(smem + SECOND_AT, ln);   // whose rows those zeros meet
#pragma unroll
    for (int i = 0; i < PF; ++i) load(i, smem);
    __builtin_amdgcn_sched_barrier(0);
    int row = first + t0 * ROWS + 32 * part, left = tiles - t0;   // the tile's first query (of this part), tiles of the head from it on
    int row_before = row;                        // ... of the tile before
    // element e: query row + 8 (e / 4) + 4 h + e % 4; not seen: before the own key, or past the end
    auto hide = [&](int row, f32x16 &v) {
      int lo = mine - shift - row - 4 * h, hi = s.lq - row - 4 * h;
      asm volatile("" : "+v"(lo), "+v"(hi));   // known here only: the compiler else does all this for every tile and drops the results
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int q = 8 * (e / 4) + e % 4;
        if (q < lo || q >= hi) v[e] = 0.0f;
      }
    };
    auto masked = [&](int row) { return row + shift < own0 + 31 || row + 32 > s.lq; };   // wave-uniform
    auto tile = [&](auto STAGE_OF) __attribute__((always_inline)) {   // STAGE_OF: -1 as it comes
      constexpr int FIXED = decltype(STAGE_OF)::value;
      if constexpr (FIXED < 0) ln.here();
      const int at = FIXED < 0 ? cur : FIXED, next = after(at, 1), nn = after(at, AHEAD);
      const char *const now = smem + at * STAGE, *const before = smem + (FIXED < 0 ? last : after(at, RING - 1)) * STAGE;
      const float *stat = reinterpret_cast<const float *>(now + 2 * L::MATRIX) + 32 * part + 4 * h;
      f32x16 ls, p;
      if constexpr (me == 0) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4 v = *reinterpret_cast<const f32x4 *>(stat + 8 * q);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            ls[4 * q + e] = v[e];
            sc[4 * q + e] = 0.0f;
          }
        }
      } else {
        take(odd ^ 1, p);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4 v = *reinterpret_cast<const f32x4 *>(stat + 64 + 8 * q);
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[4 * q + e] = v[e];
        }
      }
      auto step = [&](auto I) __attribute__((always_inline)) {
        constexpr int r = decltype(I)::value;
        if constexpr (me == 0) {
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (r == K1 + e * (HAND_OVER - K1) / 16) sc[e] = fast_exp2(fmaf(sc[e], f, -ls[e] * kLog2e));
          if (r == HAND_OVER) {
            if (masked(row)) {
              hide(row, sc);
              redo |= rows_not_finite<bf16, D>(now + SECOND_AT, ln);
            }
#pragma unroll
            for (int t = 0; t < 2; ++t) xn[t] = P::weights(sc, t);
#pragma unroll
            for (int q = 0; q < 4; ++q) xchg[odd * (L::XCHG / 16) + q * 64] = quarter_of(sc, q);
          }
        } else {
          // dS of the tile before, over this one's first product's steps
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (r == 2 + e * (K1 - 2) / 16) prev[e] *= p[e];
          if (r == K1) {
            if (masked(row_before)) {   // (before the first tile there is none: this looks at the first)
              hide(row_before, prev);
              redo |= rows_not_finite<bf16, D>(before + SECOND_AT, ln);
            }
#pragma unroll
            for (int t = 0; t < 2; ++t) x[t] = P::weights(prev, t);
          }
        }
        if (r == N - PF) wait_and_barrier<(AHEAD - 1) * OPS>();   // all that this iteration reads has been read, and all it hands over is written; tile it + 1 landed everywhere
        load((r + PF) % N, r + PF >= N ? smem + next * STAGE : r + PF < K1 ? now : before);
        if (r < ISSUE_STEPS) issue_step(r, nn);
        const bf16x8 &v = fr[r % NF];
        if constexpr (r < K1) sc = MFMA32(v, of[r], sc);
        else acc[(r - K1) / 2] = MFMA32(v, x[r % 2], acc[(r - K1) / 2]);
        __builtin_amdgcn_sched_barrier(0);
      };
      for_each_step(step, std::make_integer_sequence<int, N>{});
      if constexpr (me == 0) {
        x[0] = xn[0];
        x[1] = xn[1];
      } else {
        prev = sc;
      }
      advance();
      row_before = row;
      row += ROWS;
      if (--left == 0) {
        left = tiles;
        row = first + 32 * part;
      }
      last = at;
      cur = next;
      odd ^= 1;
    };
    using Any = std::integral_constant<int, -1>;
    int it = 1;
    tile(Any{});
    // a round of the ring at a time, with the stages known (packed_fwd.hip): four sequences of 384 to 9001 tokens, 32 heads of 128 on 8, 2030 us one by one, 1910 so; heads of 160: 133 and
    // 129.  Heads of 192 have no registers for it (505 us, 680 so).
    if constexpr (D <= 160) {
      for (; it + RING <= n; it += RING) for_each_step([&](auto I) __attribute__((always_inline)) { tile(std::integral_constant<int, (decltype(I)::value + 1) % RING>{}); }, std::make_integer_sequence<int, RING>{});
    }
    for (; it < n; ++it) tile(Any{});
    // the second product of the last tile
    const char *const before = smem + last * STAGE;
    if constexpr (me == 1) {
      f32x16 p;
      take(odd ^ 1, p);
#pragma unroll
      for (int e = 0; e < 16; ++e) prev[e] *= p[e];
      if (masked(row_before)) {
        hide(row_before, prev);
        redo |= rows_not_finite<bf16, D>(before + SECOND_AT, ln);
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) x[t] = P::weights(prev, t);
    }
    bf16x8 v[4];
    pipelined<K1, 3>([&](int i) { v[i & 3] = T::tr32(before + SECOND_AT, ln, i / 2, i % 2); },
                     [&](int i) { acc[i / 2] = MFMA32(v[i & 3], x[i % 2], acc[i / 2]); }, [](int) {});
  };
  if (n > 0) {
    if (role == 0) run(std::integral_constant<int, 0>{});
    else run(std::integral_constant<int, 1>{});
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");   // the look-ahead tiles, which nobody uses

  // Two parts: of the two waves with the same rows and role each hands over half of its columns and finishes the other half
  f32x4 *slots = reinterpret_cast<f32x4 *>(smem) + lane;
  if constexpr (PARTS == 2) {
    int *const bad = reinterpret_cast<int *>(smem + 8 * CB * 2 * 1024);
    static_assert(PAIRS == 4 && 8 * CB * 2 * 1024 + 64 <= L::BYTES, "");
    __syncthreads();   // the rings are no longer read
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int q = 0; q < 2; ++q) slots[((wave * CB + cb) * 2 + q) * 64] = part ? quarter_of(acc[cb], q) : quarter_of(acc[cb], 2 + q);
    if (lane == 0) bad[wave] = redo;
    __syncthreads();
    redo |= __builtin_amdgcn_readfirstlane(bad[wave ^ 2]) != 0;
  }
  if (own0 >= s.lk) return;
  const float mul = role ? w.scale : 1.0f;
  float *const partial = w.part + (((int64_t)split * w.where.k_tokens + s.k0 + key) * w.kv_heads + j) * (2 * d) + role * d;
  bf16 *const out = row_at<bf16>(role ? w.dk : w.dv, s.k0 + key, j, 0);
  auto put = [&](int col, f32x4 v) {
    if (col >= d) return;
    if (w.splits > 1) *reinterpret_cast<f32x4 *>(partial + col) = v * mul;
    else put4(out + col, v * mul);
  };
  if (redo) {   // query by query, without matrix instructions (packed_fwd.hip: why)
    if (part) return;
    float sum[K1][8];
#pragma unroll
    for (int kk = 0; kk < K1; ++kk)
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[kk][e] = 0.0f;
    const bf16 *kr = row_at<bf16>(w.k, s.k0 + key, j, 0), *vr = row_at<bf16>(w.v, s.k0 + key, j, 0);
#pragma unroll 1
    for (int it = n0; it < n0 + n; ++it) {
      const int g = it / tiles, q0 = first + (it - g * tiles) * ROWS;
#pragma unroll 1
      for (int q = q0; q < min(q0 + ROWS, s.lq); ++q) {
        const bf16 *qr = row_at<bf16>(w.q, s.q0 + q, j, g), *dr = row_at<bf16>(w.da, s.q0 + q, j, g);
        float sk = 0.0f, dpk = 0.0f;
#pragma unroll
        for (int kk = 0; kk < K1; ++kk) {
          sk = P::dot(row_unit<bf16, D>(qr, kk, h, d), row_unit<bf16, D>(kr, kk, h, d), sk);
          dpk = P::dot(row_unit<bf16, D>(dr, kk, h, d), row_unit<bf16, D>(vr, kk, h, d), dpk);
          __builtin_amdgcn_sched_barrier(0);   // few reads at once: no registers for more
        }
        sk += __shfl_xor(sk, 32, 64);
        dpk += __shfl_xor(dpk, 32, 64);
        if (q + shift < mine) continue;
        const int64_t stat = (int64_t)(j * r + g) * w.where.q_tokens + s.q0 + q;
        float weight = fast_exp2(fmaf(sk, f, -w.lse[stat] * kLog2e));
        if (role) weight *= dpk + w.D[stat];
#pragma unroll
        for (int kk = 0; kk < K1; ++kk) {
          const bf16x8 v = row_unit<bf16, D>(role ? qr : dr, kk, h, d);
#pragma unroll
          for (int e = 0; e < 8; ++e) sum[kk][e] = fmaf(weight, (float)v[e], sum[kk][e]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    if (mine >= s.lk) return;
#pragma unroll
    for (int kk = 0; kk < K1; ++kk)
#pragma unroll
      for (int e = 0; e < 8; e += 4) put(16 * kk + 8 * h + e, f32x4{sum[kk][e], sum[kk][e + 1], sum[kk][e + 2], sum[kk][e + 3]});
    return;
  }
  if (mine >= s.lk) return;
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) {
    if constexpr (PARTS == 2) {
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const f32x4 other = slots[(((wave ^ 2) * CB + cb) * 2 + q) * 64];
        if (part) put(32 * cb + 8 * (2 + q) + 4 * h, quarter_of(acc[cb], 2 + q) + other);
        else put(32 * cb + 8 * q + 4 * h, quarter_of(acc[cb], q) + other);
      }
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) put(32 * cb + 8 * q + 4 * h, quarter_of(acc[cb], q));
    }
  }
}

template <int D>
int bwd_launch(const PackedBwdArgs &w, int owned, int64_t pieces, int64_t key_pieces, hipStream_t st) {
  constexpr int merge = 4 * (D / 32) * 2048 + 64, ring = 4 * Tile<D>::BYTES, smem = ring > merge ? ring : merge;
  static unsigned long long attr_done = 0;
  int device;
  if (!attr_is_set(attr_done, &device)) {
    MTNLG_TRY(set_lds(packed_dq_kernel<D, 1>, smem));
    if constexpr (packed_dq_places(D) > 0) MTNLG_TRY(set_lds(packed_dq_kernel<D, 2>, smem));
    MTNLG_TRY(set_lds(packed_dkv_kernel<D>, Dkv<D>::BYTES));
    attr_mark_set(attr_done, device);
  }
  const unsigned blocks = (unsigned)(pieces * w.kv_heads), key_blocks = (unsigned)(key_pieces * w.splits * w.kv_heads);
  if constexpr (packed_dq_places(D) > 0) {
    if (owned == 64) packed_dq_kernel<D, 2><<<blocks, DQ_THREADS, smem, st>>>(w);
  }
  if (owned == 128) packed_dq_kernel<D, 1><<<blocks, DQ_THREADS, smem, st>>>(w);
  MTNLG_TRY(check_launch());
  packed_dkv_kernel<D><<<key_blocks, Dkv<D>::THREADS, Dkv<D>::BYTES, st>>>(w);
  return check_launch();
}

}  // namespace

int packed_dkv_tuned_owned(int d) {
  return packed_tuned_by_size(d, [&](auto D) { return Dkv<decltype(D)::value>::OWNED; });
}

int packed_bwd_tuned(const PackedBwdArgs &w, int owned, int64_t pieces, int64_t key_pieces, hipStream_t st) {
  return packed_tuned_by_size(w.d, [&](auto D) { return bwd_launch<decltype(D)::value>(w, owned, pieces, key_pieces, st); });
}

}  // namespace mtnlg
