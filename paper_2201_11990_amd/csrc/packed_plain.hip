// Attention over packed sequences in the order of its formulas, without a schedule of its own: fp32 on v_mfma_f32_32x32x2_f32 with P and dS in fp32, and bf16
// of head sizes above 192 (packed_fwd.hip, packed_bwd.hip: the others).
//
// fp32 instructions take 64 cycles on the matrix pipes: a workgroup alone on a unit takes 6.6 us for 64 keys of 96 columns, 5.1 of them MFMAs.  Small calls are bound by how
// their pieces come out: 1536 tokens in 4 documents, 8 heads of 96 on 4, in chunks: forward 36 us and 10 for the join, dq 53 and 8, dk / dv 59 and 8, pipes busy 45 to 52 % of the time.
#include "packed.h"

namespace mtnlg {

namespace {

// ------------------------------------------------------------------ forward
// rows of a tile: what 160 KB of LDS hold twice of K and V, and two workgroups of each
template <typename E> constexpr int tile_rows() { return sizeof(E) == 2 ? 64 : 32; }
template <typename E, int D> constexpr int fwd_stage() { return 2 * tile_rows<E>() * D * (int)sizeof(E); }
template <typename E, int D> constexpr int fwd_per_unit() { return 2 * 2 * fwd_stage<E, D>() <= 160 * 1024 ? 2 : 1; }

template <typename E, int D>
__global__ __launch_bounds__(256, (fwd_per_unit<E, D>())) void plain_fwd_kernel(PackedFwdArgs w) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  using P = Elem<E, D>;
  constexpr int TR = tile_rows<E>(), K1 = P::K1, CB = D / 32, MATRIX = TR * D * (int)sizeof(E), STAGE = 2 * MATRIX, SUB = 2 * P::BAND;
  constexpr int OWNED = 128, SUBS = TR / 32;
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
  const int rows = s.lq * r, block0 = block * OWNED;
  const int last_row = min(block0 + OWNED, rows) - 1;
  const int begin = chunk * w.chunk;
  int end = min(s.lk, last_row / r + shift + 1);   // keys that the block sees
  if (chunked && chunk + 1 < nc) end = min(end, begin + w.chunk);
  if (chunked && end <= begin && chunk > 0) return;
  const int ntiles = end > begin ? (end - begin + TR - 1) / TR : 0;

  const int own0 = block0 + wave * 32, mine = own0 + (lane & 31), row = min(mine, rows - 1);
  const int tok = row / r, g = row - tok * r;
  const int limit = min(tok + shift, end - 1);   // the last key here that the row sees
  // uniform over the wave: the least and the most of its rows, -1 if it has none
  const int least = __builtin_amdgcn_readfirstlane(limit), most = own0 < rows ? __builtin_amdgcn_readlane(limit, 31) : -1;

  const RowStream ks{reinterpret_cast<const char *>(row_at<E>(w.k, s.k0 + begin, j, 0)), end - begin, (uint32_t)(w.k.token * sizeof(E))};
  const RowStream vs{reinterpret_cast<const char *>(row_at<E>(w.v, s.k0 + begin, j, 0)), end - begin, (uint32_t)(w.v.token * sizeof(E))};
  // waves 0, 1 bring K, waves 2, 3 V
  constexpr int IPW = TR / 32 * P::NI;
  const int half = wave >> 1, band = (wave & 1) * (TR / 32);
  const uint32_t pitch = half ? vs.pitch : ks.pitch;
  uint32_t dma_off[IPW];
#pragma unroll
  for (int i = 0; i < IPW; ++i) dma_off[i] = P::dma_offset(pitch, band + i / P::NI, lane, i % P::NI, d);
  const uint32_t dst0 = lds_address(smem) + half * MATRIX + band * P::BAND;
  auto issue = [&](int t) {
    const dma_rsrc_t rs = half ? vs.tile<TR>(t) : ks.tile<TR>(t);
#pragma unroll
    for (int i = 0; i < IPW; ++i) dma16<Burst::value>(rs, dst0 + (t & 1) * STAGE + i * 1024, dma_off[i]);
  };
  if (ntiles > 0) issue(0);
  typename P::Unit qf[K1];
  const E *qrow = row_at<E>(w.q, s.q0 + tok, j, g);
#pragma unroll
  for (int kk = 0; kk < K1; ++kk) qf[kk] = row_unit<E, D>(qrow, kk, h, d);
#pragma unroll
  for (int kk = 0; kk < K1; ++kk) arrive(qf[kk]);

  constexpr bool EXACT = sizeof(E) == 4;
  const float c = w.scale * kLog2e, f = EXACT ? w.scale : c;
  const typename P::Lane ln(lane);
  f32x16 o[CB];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) o[cb] = f32x16{};
  float m = -INFINITY, l = 0.0f;
  for (int it = 0; it < ntiles; ++it) {
    wait_and_barrier<0>();   // tile it landed everywhere, and the other stage is free
    if (it + 1 < ntiles) issue(it + 1);
#pragma unroll
    for (int sub = 0; sub < SUBS; ++sub) {
      const int key0 = begin + it * TR + 32 * sub;
      if (key0 > most) continue;   // nothing that a row of the wave sees
      const char *K = smem + (it & 1) * STAGE + sub * SUB, *V = K + MATRIX;
      f32x16 sc = {};
#pragma unroll
      for (int kk = 0; kk < K1; ++kk) sc = P::mma(P::unit(K, ln, kk), qf[kk], sc);
      const bool masked = key0 + 31 > least;
      if (masked) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (key0 + 8 * (e / 4) + 4 * h + e % 4 > limit) sc[e] = -INFINITY;
      }
      // The reference maximum follows when the row maximum has outgrown it by more than 2^8: any reference gives the same sums, this one makes rescaling rare.
      float mx = sc[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) mx = fmaxf(mx, sc[e]);
      mx = pair_max(mx);
      const float m_new = mx * c > m * c + (it == 0 ? 0.0f : 8.0f) ? mx : m;
      const float ref = m_new == -INFINITY ? 0.0f : m_new;
      const float shifted = EXACT ? product_of(ref, w.scale) : ref * c;
      float rs = 0.0f;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        sc[e] = weight_of<E>(sc[e], f, shifted);
        rs += sc[e];
      }
      const float alpha = m == m_new ? 1.0f : EXACT ? exact_exp(product_of(m, w.scale) - shifted) : fast_exp2((m - m_new) * c);
      l = l * alpha + rs;
      m = m_new;
      if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) o[cb] *= alpha;
      }
      if (masked && rows_not_finite<E, D>(V, ln)) {
        add_seen_rows<E, D>(o, sc, V, [&](int row) { return key0 + row <= limit; });
      } else {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const typename P::Weights x = P::weights(sc, t);
#pragma unroll
          for (int cb = 0; cb < CB; ++cb) o[cb] = P::mma_rows(P::column(V, ln, cb, t), x, o[cb]);
        }
      }
    }
  }
  l += __shfl_xor(l, 32, 64);
  if (mine >= rows) return;
  const int head = j * r + g;
  if (chunked) {
    const int64_t id = (int64_t)(s.q0 + tok) * ((int64_t)w.kv_heads * r) + head, at = chunk * ((int64_t)w.where.q_tokens * w.kv_heads * r) + id;
    float *const to = w.part + at * d;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int col = 32 * cb + 8 * q + 4 * h;
        if (col < d) *reinterpret_cast<f32x4 *>(to + col) = quarter_of(o[cb], q);
      }
    if (h == 0) *reinterpret_cast<float2 *>(w.stat + 2 * at) = float2{m, l};
    return;
  }
  const bool none = tok + shift < 0;   // the row sees no key
  const float inv = none ? 0.0f : 1.0f / l;
  E *const to = row_at<E>(w.a, s.q0 + tok, j, g);
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int col = 32 * cb + 8 * q + 4 * h;
      if (col < d) put4(to + col, quarter_of(o[cb], q) * inv);
    }
  if (h == 0) w.lse[(int64_t)head * w.where.q_tokens + s.q0 + tok] = none ? -INFINITY : plus_log(product_of(m, w.scale), l);
}

template <typename E, int D>
int fwd_launch(const PackedFwdArgs &w, int64_t blocks, hipStream_t st) {
  constexpr int smem = 2 * fwd_stage<E, D>();
  static unsigned long long attr_done = 0;
  int device;
  if (!attr_is_set(attr_done, &device)) {
    MTNLG_TRY(set_lds(plain_fwd_kernel<E, D>, smem));
    attr_mark_set(attr_done, device);
  }
  plain_fwd_kernel<E, D><<<(unsigned)blocks, 256, smem, st>>>(w);
  return check_launch();
}

// ------------------------------------------------------------------ backward: dq and D
template <typename E> constexpr int dq_rows() { return sizeof(E) == 2 ? 64 : 32; }
template <typename E, int D> constexpr int dq_stage() { return 2 * dq_rows<E>() * D * (int)sizeof(E); }
// own rows of q and da, and results, take D * sizeof(E) / 2 + D / 2 registers and more
template <typename E, int D> constexpr int dq_per_unit() { return 2 * 2 * dq_stage<E, D>() <= 160 * 1024 && D * (int)sizeof(E) <= 384 ? 2 : 1; }

template <typename E, int D>
__global__ __launch_bounds__(256, (dq_per_unit<E, D>())) void plain_dq_kernel(PackedBwdArgs w) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  using P = Elem<E, D>;
  constexpr int TR = dq_rows<E>(), K1 = P::K1, CB = D / 32, MATRIX = TR * D * (int)sizeof(E), STAGE = 2 * MATRIX, SUB = 2 * P::BAND;
  constexpr int OWNED = 128, SUBS = TR / 32;
  const int lane = threadIdx.x & 63, h = lane >> 5, r = w.group, d = w.d;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int j = blockIdx.x % w.kv_heads;
  Span s;
  unsigned at;
  const bool chunked = w.chunk > 0;
  auto chunks_of = [&](const Span &s) { return chunked ? min((int)(((unsigned)max(s.lk, 1) + w.chunk - 1) / w.chunk), w.chunks) : 1; };   // (unsigned: the sum may pass 2^31)
  if (!find_piece(w.where, blockIdx.x / w.kv_heads, [&](const Span &s) { return (unsigned)((s.lq * r + OWNED - 1) / OWNED * chunks_of(s)); }, s, at)) return;
  const int nc = chunks_of(s), count = (s.lq * r + OWNED - 1) / OWNED, shift = s.lk - s.lq;
  const int chunk = at % nc, block = count - 1 - at / nc;   // falling work
  const int rows = s.lq * r, block0 = block * OWNED, last_row = min(block0 + OWNED, rows) - 1;
  const int begin = chunk * w.chunk;
  int end = min(s.lk, last_row / r + shift + 1);   // keys that the block sees
  if (chunked && chunk + 1 < nc) end = min(end, begin + w.chunk);
  if (chunked && end <= begin && chunk > 0) return;
  const int ntiles = end > begin ? (end - begin + TR - 1) / TR : 0;

  const int own0 = block0 + wave * 32, mine = own0 + (lane & 31), row = min(mine, rows - 1);
  const int tok = row / r, g = row - tok * r, head = j * r + g;
  const int limit = min(tok + shift, end - 1);   // the last key here that the row sees
  const int least = __builtin_amdgcn_readfirstlane(limit), most = own0 < rows ? __builtin_amdgcn_readlane(limit, 31) : -1;

  const RowStream ks{reinterpret_cast<const char *>(row_at<E>(w.k, s.k0 + begin, j, 0)), end - begin, (uint32_t)(w.k.token * sizeof(E))};
  const RowStream vs{reinterpret_cast<const char *>(row_at<E>(w.v, s.k0 + begin, j, 0)), end - begin, (uint32_t)(w.v.token * sizeof(E))};
  constexpr int IPW = TR / 32 * P::NI;
  const int half = wave >> 1, band = (wave & 1) * (TR / 32);
  const uint32_t pitch = half ? vs.pitch : ks.pitch;
  uint32_t dma_off[IPW];
#pragma unroll
  for (int i = 0; i < IPW; ++i) dma_off[i] = P::dma_offset(pitch, band + i / P::NI, lane, i % P::NI, d);
  const uint32_t dst0 = lds_address(smem) + half * MATRIX + band * P::BAND;
  auto issue = [&](int t) {
    const dma_rsrc_t rs = half ? vs.tile<TR>(t) : ks.tile<TR>(t);
#pragma unroll
    for (int i = 0; i < IPW; ++i) dma16<Burst::value>(rs, dst0 + (t & 1) * STAGE + i * 1024, dma_off[i]);
  };
  if (ntiles > 0) issue(0);
  typename P::Unit qf[K1], df[K1];   // own rows of q and da
  float dsum = 0.0f;
  {
    const E *qrow = row_at<E>(w.q, s.q0 + tok, j, g), *drow = row_at<E>(w.da, s.q0 + tok, j, g), *arow = row_at<E>(w.a, s.q0 + tok, j, g);
#pragma unroll
    for (int kk = 0; kk < K1; ++kk) {
      qf[kk] = row_unit<E, D>(qrow, kk, h, d);
      df[kk] = row_unit<E, D>(drow, kk, h, d);
      dsum = P::dot(row_unit<E, D>(arow, kk, h, d), df[kk], dsum);
    }
  }
  dsum += __shfl_xor(dsum, 32, 64);
  constexpr bool EXACT = sizeof(E) == 4;
  const int64_t stat = (int64_t)head * w.where.q_tokens + s.q0 + tok;
  if (mine < rows && h == 0 && chunk == 0) w.D[stat] = dsum;
  float lse = w.lse[stat];
  lse = lse == -INFINITY ? INFINITY : EXACT ? lse : lse * kLog2e;   // a row that sees nothing: weights of 0
#pragma unroll
  for (int kk = 0; kk < K1; ++kk) {
    arrive(qf[kk]);
    arrive(df[kk]);
  }
  arrive(lse);

  const float f = EXACT ? w.scale : w.scale * kLog2e;
  const typename P::Lane ln(lane);
  f32x16 acc[CB];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) acc[cb] = f32x16{};
  for (int it = 0; it < ntiles; ++it) {
    wait_and_barrier<0>();
    if (it + 1 < ntiles) issue(it + 1);
#pragma unroll
    for (int sub = 0; sub < SUBS; ++sub) {
      const int key0 = begin + it * TR + 32 * sub;
      if (key0 > most) continue;
      const char *K = smem + (it & 1) * STAGE + sub * SUB, *V = K + MATRIX;
      f32x16 sc = {}, pc = {};
#pragma unroll
      for (int kk = 0; kk < K1; ++kk) sc = P::mma(P::unit(K, ln, kk), qf[kk], sc);
#pragma unroll
      for (int kk = 0; kk < K1; ++kk) pc = P::mma(P::unit(V, ln, kk), df[kk], pc);
#pragma unroll
      for (int e = 0; e < 16; ++e) pc[e] = weight_of<E>(sc[e], f, lse) * (pc[e] - dsum);
      const bool masked = key0 + 31 > least;
      if (masked) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (key0 + 8 * (e / 4) + 4 * h + e % 4 > limit) pc[e] = 0.0f;
      }
      if (masked && rows_not_finite<E, D>(K, ln)) {
        add_seen_rows<E, D>(acc, pc, K, [&](int row) { return key0 + row <= limit; });
      } else {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const typename P::Weights x = P::weights(pc, t);
#pragma unroll
          for (int cb = 0; cb < CB; ++cb) acc[cb] = P::mma_rows(P::column(K, ln, cb, t), x, acc[cb]);
        }
      }
    }
  }
  if (mine >= rows) return;
  if (chunked) {
    float *const to = w.dq_part + (chunk * ((int64_t)w.where.q_tokens * w.kv_heads * r) + (int64_t)(s.q0 + tok) * ((int64_t)w.kv_heads * r) + head) * d;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int col = 32 * cb + 8 * q + 4 * h;
        if (col < d) *reinterpret_cast<f32x4 *>(to + col) = quarter_of(acc[cb], q);
      }
    return;
  }
  E *const to = row_at<E>(w.dq, s.q0 + tok, j, g);
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int col = 32 * cb + 8 * q + 4 * h;
      if (col < d) put4(to + col, quarter_of(acc[cb], q) * w.scale);
    }
}

// ------------------------------------------------------------------ dk and dv
// Waves in pairs, each of 32 keys: one wave forms S and P and sums up dv, the other dP and dS and dk, so that either holds one of K and V and one of the results.  P goes to
// the second through LDS in fp32.
template <typename E, int D> struct Dkv {
  static constexpr int PAIRS = D * (int)sizeof(E) <= 512 && D <= 192 ? 4 : 2;   // registers: 8 waves have 256 each
  static constexpr int OWNED = 32 * PAIRS, THREADS = 128 * PAIRS, WAVES = 2 * PAIRS;
  static constexpr int MATRIX = 32 * D * (int)sizeof(E), STAGE = 2 * MATRIX + 512, LDS = 2 * STAGE + PAIRS * 4096;
};

template <typename E, int D>
__global__ __launch_bounds__((Dkv<E, D>::THREADS)) void plain_dkv_kernel(PackedBwdArgs w) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  using P = Elem<E, D>;
  using L = Dkv<E, D>;
  constexpr int K1 = P::K1, CB = D / 32, WAVES = L::WAVES;
  const int lane = threadIdx.x & 63, h = lane >> 5, r = w.group, d = w.d;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int j = blockIdx.x % w.kv_heads;
  Span s;
  unsigned at;
  if (!find_piece(w.where, blockIdx.x / w.kv_heads, [&](const Span &s) { return (unsigned)((s.lk + L::OWNED - 1) / L::OWNED * w.splits); }, s, at)) return;
  const int split = at % w.splits, block0 = (int)(at / w.splits) * L::OWNED, shift = s.lk - s.lq;
  const int role = wave / L::PAIRS, pair = wave % L::PAIRS;
  const int own0 = block0 + pair * 32, mine = own0 + (lane & 31), key = min(mine, s.lk - 1);
  const int first = max(0, block0 - shift) / 32, tiles = s.lq > first * 32 ? (s.lq - first * 32 + 31) / 32 : 0;   // of a head: from the first query that sees the block on
  // the workgroup's part of the tiles of all heads of the group, one head after the other: n from tile t0 of head g0 on
  const int n0 = (int)((int64_t)r * tiles * split / w.splits), n = (int)((int64_t)r * tiles * (split + 1) / w.splits) - n0;
  const int g0 = tiles ? n0 / tiles : 0, t0 = n0 - g0 * tiles;

  // two matrices of two bands, NI instructions each, dealt out over the waves
  constexpr int ALL = 4 * P::NI, IPW = (ALL + WAVES - 1) / WAVES;
  const uint32_t qp = (uint32_t)(w.q.token * sizeof(E)), dp = (uint32_t)(w.da.token * sizeof(E));
  uint32_t dma_off[IPW];
#pragma unroll
  for (int i = 0; i < IPW; ++i) {
    const int k = wave + WAVES * i, second = k / (2 * P::NI), in = k % (2 * P::NI);
    dma_off[i] = P::dma_offset(second ? dp : qp, in / P::NI, lane, in % P::NI, d);
  }
  const uint32_t lds0 = lds_address(smem);
  int ig = g0, it_of = t0;   // what is issued next
  auto issue = [&](int stage) {
    const int row0 = (first + it_of) * 32;
    const RowStream qs{reinterpret_cast<const char *>(row_at<E>(w.q, s.q0 + row0, j, ig)), s.lq - row0, qp};
    const RowStream ds{reinterpret_cast<const char *>(row_at<E>(w.da, s.q0 + row0, j, ig)), s.lq - row0, dp};
    const dma_rsrc_t rq = qs.tile<32>(0), rd = ds.tile<32>(0);
#pragma unroll
    for (int i = 0; i < IPW; ++i) {
      const int k = wave + WAVES * i, second = k / (2 * P::NI), in = k % (2 * P::NI);
      if (ALL % WAVES == 0 || k < ALL) dma16<Burst::value>(second ? rd : rq, lds0 + stage * L::STAGE + second * L::MATRIX + in * 1024, dma_off[i]);
    }
    if (wave < 2) {   // lse and D of the rows
      const int64_t from = (int64_t)(j * r + ig) * w.where.q_tokens + s.q0 + row0;
      const int left = min(s.lq - row0, 64);
      dma4<Burst::value>(dma_rsrc((wave ? w.D : w.lse) + from, __builtin_amdgcn_readfirstlane((uint32_t)left * 4)), lds0 + stage * L::STAGE + 2 * L::MATRIX + wave * 256, lane * 4);
    }
    if (++it_of == tiles) {
      it_of = 0;
      ++ig;
    }
  };
  if (n > 0) issue(0);
  typename P::Unit of[K1];   // own rows of K (role 0) or V
  {
    const E *own = row_at<E>(role ? w.v : w.k, s.k0 + key, j, 0);
#pragma unroll
    for (int kk = 0; kk < K1; ++kk) of[kk] = row_unit<E, D>(own, kk, h, d);
#pragma unroll
    for (int kk = 0; kk < K1; ++kk) arrive(of[kk]);
  }
  constexpr bool EXACT = sizeof(E) == 4;
  const float f = EXACT ? w.scale : w.scale * kLog2e;
  const typename P::Lane ln(lane);
  f32x16 acc[CB];   // dv (role 0) or dk
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) acc[cb] = f32x16{};
  f32x4 *const xchg = reinterpret_cast<f32x4 *>(smem + 2 * L::STAGE) + pair * 256 + lane;
  int t = t0;
  for (int it = 0; it < n; ++it) {
    wait_and_barrier<0>();
    if (it + 1 < n) issue((it + 1) & 1);
    const char *stage = smem + (it & 1) * L::STAGE, *Q = stage, *dO = stage + L::MATRIX;
    const int row0 = (first + t) * 32;   // tile's first query
    if (++t == tiles) t = 0;
    const bool seen = row0 + 31 + shift >= own0 && own0 < s.lk;   // by a key of the pair
    const bool masked = row0 + shift < own0 + 31 || row0 + 31 >= s.lq;
    // element e: query row0 + 8 (e / 4) + 4 h + e % 4; sees the own key?
    auto sees = [&](int row) { return row0 + row + shift >= mine && row0 + row < s.lq; };
    f32x16 sc = {};
    if (seen) {
      const char *from = role ? dO : Q;
#pragma unroll
      for (int kk = 0; kk < K1; ++kk) sc = P::mma(P::unit(from, ln, kk), of[kk], sc);
      if (role == 0) {
        const float *stat = reinterpret_cast<const float *>(stage + 2 * L::MATRIX) + 4 * h;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4 v = *reinterpret_cast<const f32x4 *>(stat + 8 * q);
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[4 * q + e] = weight_of<E>(sc[4 * q + e], f, EXACT ? v[e] : v[e] * kLog2e);
        }
        if (masked) {
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (!sees(8 * (e / 4) + 4 * h + e % 4)) sc[e] = 0.0f;
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) xchg[q * 64] = quarter_of(sc, q);
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (!seen) continue;
    const char *with = role ? Q : dO;
    if (role == 1) {
      const float *stat = reinterpret_cast<const float *>(stage + 2 * L::MATRIX + 256) + 4 * h;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 p = xchg[q * 64], v = *reinterpret_cast<const f32x4 *>(stat + 8 * q);
#pragma unroll
        for (int e = 0; e < 4; ++e) sc[4 * q + e] = p[e] * (sc[4 * q + e] - v[e]);
      }
      if (masked) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (!sees(8 * (e / 4) + 4 * h + e % 4)) sc[e] = 0.0f;
      }
    }
    if (masked && rows_not_finite<E, D>(with, ln)) {
      add_seen_rows<E, D>(acc, sc, with, sees);
    } else {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const typename P::Weights x = P::weights(sc, u);
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) acc[cb] = P::mma_rows(P::column(with, ln, cb, u), x, acc[cb]);
      }
    }
  }
  if (mine >= s.lk) return;
  const float mul = role ? w.scale : 1.0f;
  if (w.splits > 1) {
    float *const to = w.part + (((int64_t)split * w.where.k_tokens + s.k0 + mine) * w.kv_heads + j) * (2 * d) + role * d;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int col = 32 * cb + 8 * q + 4 * h;
        if (col < d) *reinterpret_cast<f32x4 *>(to + col) = quarter_of(acc[cb], q) * mul;
      }
    return;
  }
  E *const to = row_at<E>(role ? w.dk : w.dv, s.k0 + mine, j, 0);
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int col = 32 * cb + 8 * q + 4 * h;
      if (col < d) put4(to + col, quarter_of(acc[cb], q) * mul);
    }
}

template <typename E, int D>
int bwd_launch(const PackedBwdArgs &w, int64_t pieces, int64_t key_pieces, hipStream_t st) {
  constexpr int smem = 2 * dq_stage<E, D>();
  static unsigned long long attr_done = 0;
  int device;
  if (!attr_is_set(attr_done, &device)) {
    MTNLG_TRY(set_lds(plain_dq_kernel<E, D>, smem));
    MTNLG_TRY(set_lds(plain_dkv_kernel<E, D>, Dkv<E, D>::LDS));
    attr_mark_set(attr_done, device);
  }
  plain_dq_kernel<E, D><<<(unsigned)(pieces * w.kv_heads), 256, smem, st>>>(w);
  MTNLG_TRY(check_launch());
  plain_dkv_kernel<E, D><<<(unsigned)(key_pieces * w.splits * w.kv_heads), Dkv<E, D>::THREADS, Dkv<E, D>::LDS, st>>>(w);
  return check_launch();
}

template <typename F>
int by_size(int dtype, int d, F &&f) {
  if (dtype == MTNLG_F32) return packed_by_size(d, [&](auto D) { return f(0.0f, D); });
  return f((bf16)0.0f, std::integral_constant<int, 256>{});
}

}  // namespace

int packed_fwd_plain(int dtype, const PackedFwdArgs &w, int64_t blocks, hipStream_t st) {
  return by_size(dtype, w.d, [&](auto e, auto D) { return fwd_launch<decltype(e), decltype(D)::value>(w, blocks, st); });
}

int packed_bwd_plain(int dtype, const PackedBwdArgs &w, int64_t pieces, int64_t key_pieces, hipStream_t st) {
  return by_size(dtype, w.d, [&](auto e, auto D) { return bwd_launch<decltype(e), decltype(D)::value>(w, pieces, key_pieces, st); });
}

int packed_dkv_plain_owned(int dtype, int d) {
  return by_size(dtype, d, [&](auto e, auto D) { return Dkv<decltype(e), decltype(D)::value>::OWNED; });
}

}  // namespace mtnlg
