// Causal softmax attention over packed sequences with grouped heads, forward, bf16 in, fp32 softmax and sums, on the gfx950 matrix cores.
//
//   query t of a sequence of lq queries and lk keys sees its keys 0 .. t + lk - lq:
//   S = scale q k^T,  P = softmax of the keys that are seen,  a = P v,  lse = log sum exp S;  no key seen: a = 0, lse = -inf
//
// A workgroup owns 64 or 128 rows of one head of keys, rows being (token, head of the group) with the head fastest: the query heads that share keys share every tile of
// them, and a single token's heads fill one block.  K and V stream through LDS past the own rows in tiles of 64; the products are those of attention_mfma.hip (the
// streamed tile as A operand, 32 own rows to a wave as B, P from one product to the next in registers, fragments read a few steps ahead across the end of a tile).
// Calls of few rows cut the keys into chunks, whose results packed.hip joins.
//
// P rounds to bf16 before its product (2^-8 of each term at most, as the result once more): as three bf16 parts that keep all bits that product would be three times as long.  Scores, maxima, sums and results are fp32.
// (packed_bwd.hip: where the dense kernels do not round.)
//
// Bound by the matrix and vector pipes alike: 64 keys and 128 rows of 128 are 32 MFMAs and 168 vector instructions to a wave, 34 of them exponentials at a quarter of
// the rate.  Four sequences of 384 to 9001 tokens, 32 heads of 128 on 8: 869 us, 1.04 PFLOP/s of what is not masked, matrix pipes busy 59 % of the time (a large product of the
// library reaches 1.2 PFLOP/s on this card); eight of 77 to 2048, 16 heads on 4: 73 us, 0.67 PFLOP/s, 39 %, since pieces are short; 2501 and 1589 tokens, 16 heads of 160: 71 us.
// Single tokens read K and V once: 32 of them over 64 to 15872 keys, 425 MB in 88 us, 4.8 TB/s, and 8 us for the join.
#include "packed.h"

namespace mtnlg {

namespace {

constexpr int WAVES = 4;
// Two workgroups to a compute unit where registers and LDS allow.
template <int D> constexpr int per_unit() { return D <= 160 ? 2 : 1; }

// A wave's rows once more without matrix instructions, key by key: where a tile that a mask crosses holds an infinity or NaN, zero weights would carry it to rows that
// do not see it.  Lanes (l, l + 32) share a row, each has the 16-byte units of one parity.
template <int D>
struct RowByRow {
  using P = Elem<bf16, D>;
  float o[P::K1][8], m = -INFINITY, l = 0.0f;
  __device__ __forceinline__ void run(const PackedFwdArgs &w, const Span &s, int j, const bf16 *qrow, int begin, int most, int limit, int h) {
    const float c = w.scale * kLog2e;
#pragma unroll
    for (int kk = 0; kk < P::K1; ++kk)
#pragma unroll
      for (int e = 0; e < 8; ++e) o[kk][e] = 0.0f;
#pragma unroll 1
    for (int key = begin; key <= most; ++key) {
      const bf16 *kr = row_at<bf16>(w.k, s.k0 + key, j, 0), *vr = row_at<bf16>(w.v, s.k0 + key, j, 0);
      float sc = 0.0f;
#pragma unroll
      for (int kk = 0; kk < P::K1; ++kk) {
        sc = P::dot(row_unit<bf16, D>(kr, kk, h, w.d), row_unit<bf16, D>(qrow, kk, h, w.d), sc);
        __builtin_amdgcn_sched_barrier(0);   // few reads at once: no registers for more
      }
      sc += __shfl_xor(sc, 32, 64);
      if (key > limit) continue;
      const float mn = fmaxf(m, sc), ref = mn == -INFINITY ? 0.0f : mn;
      const float alpha = m == mn ? 1.0f : fast_exp2((m - mn) * c), p = fast_exp2(fmaf(sc, c, -ref * c));
      l = l * alpha + p;
      m = mn;
#pragma unroll
      for (int kk = 0; kk < P::K1; ++kk) {
        const bf16x8 v = row_unit<bf16, D>(vr, kk, h, w.d);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[kk][e] = o[kk][e] * alpha + p * (float)v[e];
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
};

// SPLIT 2: 64 rows to a workgroup, waves 0, 1 take the first 32 keys of every tile, waves 2, 3 the last 32, each with a maximum and a sum of its own, merged through LDS at the
// end.  SPLIT 1: 128 rows.
template <int D, int SPLIT>
__global__ __launch_bounds__(64 * WAVES, per_unit<D>()) void packed_fwd_kernel(PackedFwdArgs w) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  using P = Elem<bf16, D>;
  using T = typename P::T;
  constexpr int ROWS = WAVES / SPLIT, OWNED = 32 * ROWS;   // waves with rows of their own
  constexpr int K1 = D / 16, CB = D / 32, STAGE = 2 * T::BYTES;
  constexpr int SUBS = SPLIT == 2 ? 1 : 2;                // 32-key parts of a tile that a wave takes
  constexpr int N1 = 2 * K1, NF = D == 160 ? 5 : D == 96 ? 6 : 4, PF = NF - 1;   // steps of a part: K1 for S, K1 for O
  static_assert(N1 % NF == 0, "fragment buffers");
  const int lane = threadIdx.x & 63, h = lane >> 5, r = w.group, d = w.d;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int j = blockIdx.x % w.kv_heads;
  const bool chunked = w.chunk > 0;
  auto chunks_of = [&](const Span &s) { return chunked ? min((int)(((unsigned)max(s.lk, 1) + w.chunk - 1) / w.chunk), w.chunks) : 1; };   // (unsigned: the sum may pass 2^31)
  Span s;
  unsigned at;
  if (!find_piece(w.where, blockIdx.x / w.kv_heads, [&](const Span &s) { return (unsigned)((s.lq * r + OWNED - 1) / OWNED * chunks_of(s)); }, s, at)) return;
  const int nc = chunks_of(s), count = (s.lq * r + OWNED - 1) / OWNED, shift = s.lk - s.lq;
  const int chunk = at % nc, block = count - 1 - at / nc;   // falling work
  const int rows = s.lq * r, block0 = block * OWNED, last_row = min(block0 + OWNED, rows) - 1;
  const int begin = chunk * w.chunk;
  int end = min(s.lk, last_row / r + shift + 1);   // keys that the block sees
  if (chunked && chunk + 1 < nc) end = min(end, begin + w.chunk);
  if (chunked && end <= begin && chunk > 0) return;
  const int ntiles = end > begin ? (end - begin + 63) / 64 : 0;

  const int part = SPLIT == 2 ? wave / ROWS : 0, other = SPLIT == 2 ? wave ^ ROWS : wave;   // the wave with the same rows
  const int own0 = block0 + wave % ROWS * 32, mine = own0 + (lane & 31), row = min(mine, rows - 1);
  const int tok = row / r, g = row - tok * r;
  const int limit = min(tok + shift, end - 1);   // the last key here that the row sees
  // uniform over the wave: the least and the most of its rows, none if it has no row
  const int least = __builtin_amdgcn_readfirstlane(limit), most = own0 < rows ? __builtin_amdgcn_readlane(limit, 31) : begin - 1;
  const float c = w.scale * kLog2e;
  typename P::Lane ln(lane);
  ln.n0 += part * T::ROWS32;
  ln.t0 += part * T::ROWS32;
  const uint32_t smem_addr = lds_address(smem);

  // waves 0, 1 bring 32 rows each of K, waves 2, 3 of V
  constexpr int IPW = 2 * T::NI;
  const int half = wave >> 1, band = 2 * (wave & 1);
  const Heads &mat = half ? w.v : w.k;
  RowWalk stream(row_at<bf16>(mat, s.k0 + begin + 16 * band, j, 0), end - begin - 16 * band, (uint32_t)(mat.token * 2), 64);   // from the wave's rows on
  uint32_t dma_off[T::NI];   // of 16 rows: the next 16 lie the same in a descriptor of their own
#pragma unroll
  for (int i = 0; i < T::NI; ++i) dma_off[i] = T::dma_offset(stream.pitch, 0, lane, i, d);
  const uint32_t dst0 = smem_addr + half * T::BYTES + band * (T::NI * 1024);
  constexpr int ISSUE_STEPS = IPW / 2;   // (one tile ahead: it is waited for in the same iteration)
  auto issue_step = [&](int step, int st) {
#pragma unroll
    for (int i = 0; i < IPW; ++i)
      if (i >= (step ? dma_by<IPW, ISSUE_STEPS>(step - 1) : 0) && i < dma_by<IPW, ISSUE_STEPS>(step))
        dma16<Spread::value>(stream.tile<16>(16 * (i / T::NI)), dst0 + st * STAGE + i * 1024, dma_off[i % T::NI]);
  };
  bf16x8 qf[K1];   // own rows: columns 16 kk + 8 h .. + 7
#pragma unroll
  for (int i = 0; i < IPW; ++i) dma16<Burst::value>(stream.tile<16>(16 * (i / T::NI)), dst0 + i * 1024, dma_off[i % T::NI]);
  stream.advance<64>();
  {
    const bf16 *qrow = row_at<bf16>(w.q, s.q0 + tok, j, g);
#pragma unroll
    for (int kk = 0; kk < K1; ++kk) qf[kk] = row_unit<bf16, D>(qrow, kk, h, d);
  }
#pragma unroll
  for (int kk = 0; kk < K1; ++kk) arrive(qf[kk]);
  f32x16 o[CB];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) o[cb] = f32x16{};
  float m = -INFINITY, l = 0.0f;   // l: this lane's share of the row sum
  bool redo = false;               // the wave has met values that are not finite where a mask hides some
  wait_and_barrier<0>();           // tile 0 landed everywhere

  bf16x8 fr[NF];
  f32x16 sc;
  bf16x8 x[2];
  auto load = [&](int i, const char *Kt) {   // the fragment of step i, of the tile in stage Kt
    const int sub = i / N1, r = i % N1;
    const char *k = Kt + sub * T::ROWS32;
    if (r < K1) fr[i % NF] = T::nat32(k, ln, r);
    else fr[i % NF] = T::tr32(k + T::BYTES, ln, (r - K1) / 2, r % 2);
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
    const char *const V = smem + now * STAGE + T::BYTES;
    auto step = [&](auto I) __attribute__((always_inline)) {
      constexpr int i = decltype(I)::value, sub = i / N1, r = i % N1;
      const int key0 = begin + it * 64 + 32 * (part + sub);
      if (r == 0) sc = f32x16{};
      if (r == K1) {
        // element e: key key0 + 8 (e / 4) + 4 h + e % 4
        if constexpr (decltype(MASKED)::value) {
          const int seen = limit - key0 - 4 * (lane_here() >> 5);
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (8 * (e / 4) + e % 4 > seen) sc[e] = -INFINITY;
          redo |= rows_not_finite<bf16, D>(V + sub * T::ROWS32, ln);
        }
        // m: the running maximum of the raw scores; it follows when the row maximum has outgrown it by more than 2^8 in the exponent's units (any reference gives the
        // same sums; this one keeps p <= 256 and makes rescaling O rare), and in the first tile, where a weight of 1, which does not round, is the largest.
        float mx = sc[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) mx = fmaxf(mx, sc[e]);
        mx = pair_max(mx);
        const float m_new = mx * c > m * c + (sub == 1 && it == 0 ? 0.0f : 8.0f) ? mx : m;
        const float ref = m_new == -INFINITY ? 0.0f : m_new;
        const float mc = ref * c;
        float rs = 0.0f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          sc[e] = fast_exp2(fmaf(sc[e], c, -mc));
          rs += sc[e];
        }
        const float alpha = m == m_new ? 1.0f : fast_exp2((m - m_new) * c);
        l = l * alpha + rs;
        m = m_new;
        if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {   // a reference maximum moved: rescale O
#pragma unroll
          for (int cb = 0; cb < CB; ++cb) o[cb] *= alpha;
        }
        x[0] = P::weights(sc, 0);
        x[1] = P::weights(sc, 1);
      }
      if (i == N - PF) wait_and_barrier<0>();   // all of tile `it` has been read; tile it + 1 landed everywhere
      load((i + PF) % N, smem + (i + PF < N ? now : next) * STAGE);
      if (i < ISSUE_STEPS) issue_step(i, next);
      const bf16x8 &v = fr[i % NF];
      if constexpr (r < K1) sc = MFMA32(v, qf[r], sc);
      else o[(r - K1) / 2] = MFMA32(v, x[r % 2], o[(r - K1) / 2]);
      __builtin_amdgcn_sched_barrier(0);
    };
    for_each_step(step, std::make_integer_sequence<int, N>{});
    stream.advance<64>();
    cur = next;
  };
  // 32-key parts with a key that a row of the wave sees, and of those the first ones, which all rows see whole: a loop without masks for them, which has fewer values
  // to keep.  The parts after them are passed over.
  auto parts_of = [&](int keys) { return SPLIT == 2 ? (keys / 32 + 1 - part) / 2 : keys / 32; };
  const int visible = max(0, parts_of(most - begin + 32)), whole = parts_of(min(least, most) - begin + 1) / SUBS;
  int it = 0;
  using Any = std::integral_constant<int, -1>;
  // In pairs, with the stages known: fragments' addresses are registers and constants, 17 % fewer vector instructions (four sequences of 384 to 9001 tokens, 32 heads of 128 on 8: 905 us
  // tile by tile, 869 so).  Not where 128 rows of 96 would need 187 registers then, not 168, and two workgroups share a unit in place of three (2501 and 1589 tokens, 32 heads: 77 us, 79 so).
  if constexpr (D != 96 || SPLIT == 2) {
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
  for (; it < ntiles; ++it) {   // passed over: its share of the next tile, and the barrier
#pragma unroll
    for (int i = 0; i < IPW; ++i) dma16<Burst::value>(stream.tile<16>(16 * (i / T::NI)), dst0 + (cur ^ 1) * STAGE + i * 1024, dma_off[i % T::NI]);
    wait_and_barrier<0>();
    stream.advance<64>();
    cur ^= 1;
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");   // the look-ahead tiles, which nobody uses

  l += __shfl_xor(l, 32, 64);
  // lane, own row and where it lies, worked out once more: registers less across the loop
  const int out_lane = lane_here(), out_h = out_lane >> 5, last = own0 + (out_lane & 31), out_row = min(last, rows - 1), out_tok = out_row / r, out_g = out_row - out_tok * r;
  if constexpr (SPLIT == 2) {   // the part's results relative to the larger of the two maxima
    f32x4 *slots = reinterpret_cast<f32x4 *>(smem) + out_lane;
    float *const stat = reinterpret_cast<float *>(smem + 2 * WAVES * CB * 1024);   // maximum and sum of each wave
    int *const bad = reinterpret_cast<int *>(stat + WAVES * 128);
    __syncthreads();   // the rings are no longer read
    stat[wave * 128 + out_lane] = m;
    stat[wave * 128 + 64 + out_lane] = l;
    if (out_lane == 0) bad[wave] = redo;
    __syncthreads();
    redo |= __builtin_amdgcn_readfirstlane(bad[other]) != 0;
    const float mo = stat[other * 128 + out_lane], lo = stat[other * 128 + 64 + out_lane], both = fmaxf(m, mo), ref = both == -INFINITY ? 0.0f : both;
    auto relative = [&](float x) { return fast_exp2((x - ref) * c); };
    const float mul = relative(m);
    l = part ? fmaf(l, mul, lo * relative(mo)) : fmaf(lo, relative(mo), l * mul);
    m = both;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) o[cb] *= mul;
    // the two waves with the same rows each hand over half of their column blocks' elements (q 0, 1 or 2, 3) and finish the other half
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int q = 0; q < 2; ++q) slots[((wave * CB + cb) * 2 + q) * 64] = part ? quarter_of(o[cb], q) : quarter_of(o[cb], 2 + q);
    __syncthreads();
  }
  if (own0 >= rows) return;
  const int head = j * r + out_g;
  const int64_t id = (int64_t)(s.q0 + out_tok) * ((int64_t)w.kv_heads * r) + head, place = chunk * ((int64_t)w.where.q_tokens * w.kv_heads * r) + id;
  bf16 *const out = row_at<bf16>(w.a, s.q0 + out_tok, j, out_g);
  float *const to = w.part + place * d, *const out_lse = w.lse + (int64_t)head * w.where.q_tokens + s.q0 + out_tok;
  const bool none = out_tok + shift < 0;   // the row sees no key
  auto statistics = [&](float m, float l) {
    if (chunked) *reinterpret_cast<float2 *>(w.stat + 2 * place) = float2{m, l};
    else *out_lse = none ? -INFINITY : plus_log(product_of(m, w.scale), l);
  };
  if (redo) {
    if (part) return;
    RowByRow<D> again;
    again.run(w, s, j, row_at<bf16>(w.q, s.q0 + out_tok, j, out_g), begin, most, min(out_tok + shift, end - 1), out_h);
    if (last >= rows) return;
    const float inv = none ? 0.0f : 1.0f / again.l;
#pragma unroll
    for (int kk = 0; kk < K1; ++kk) {
      const int col = 16 * kk + 8 * out_h;
      if (col >= d) continue;
#pragma unroll
      for (int e = 0; e < 8; e += 4) {
        const f32x4 v = {again.o[kk][e], again.o[kk][e + 1], again.o[kk][e + 2], again.o[kk][e + 3]};
        if (chunked) *reinterpret_cast<f32x4 *>(to + col + e) = v;
        else put4(out + col + e, v * inv);
      }
    }
    if (out_h == 0) statistics(again.m, again.l);
    return;
  }
  if (last >= rows) return;
  const float inv = none ? 0.0f : 1.0f / l;
  auto put = [&](int cb, int q, f32x4 sum) {   // columns 32 cb + 8 q + 4 out_h .. + 3
    const int col = 32 * cb + 8 * q + 4 * out_h;
    if (col >= d) return;
    if (chunked) *reinterpret_cast<f32x4 *>(to + col) = sum;
    else put4(out + col, sum * inv);
  };
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) {
    if constexpr (SPLIT == 2) {
      const f32x4 *slots = reinterpret_cast<const f32x4 *>(smem) + out_lane;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const f32x4 rest = slots[((other * CB + cb) * 2 + q) * 64];
        if (part) put(cb, 2 + q, quarter_of(o[cb], 2 + q) + rest);
        else put(cb, q, quarter_of(o[cb], q) + rest);
      }
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) put(cb, q, quarter_of(o[cb], q));
    }
  }
  if (out_h == 0 && part == 0) statistics(m, l);
}

template <int D, int SPLIT>
int fwd_launch(const PackedFwdArgs &w, int64_t blocks, hipStream_t st) {
  constexpr int merge = SPLIT == 2 ? WAVES * (2 * (D / 32) * 1024 + 512) + 64 : 0, ring = 4 * Tile<D>::BYTES, smem = ring > merge ? ring : merge;
  static unsigned long long attr_done = 0;
  int device;
  if (!attr_is_set(attr_done, &device)) {
    MTNLG_TRY(set_lds(packed_fwd_kernel<D, SPLIT>, smem));
    attr_mark_set(attr_done, device);
  }
  packed_fwd_kernel<D, SPLIT><<<(unsigned)blocks, 64 * WAVES, smem, st>>>(w);
  return check_launch();
}

}  // namespace

int packed_fwd_tuned(const PackedFwdArgs &w, int owned, int64_t blocks, hipStream_t st) {
  return packed_tuned_by_size(w.d, [&](auto D) {
    constexpr int d = decltype(D)::value;
    return owned == 64 ? fwd_launch<d, 2>(w, blocks, st) : fwd_launch<d, 1>(w, blocks, st);
  });
}

}  // namespace mtnlg
