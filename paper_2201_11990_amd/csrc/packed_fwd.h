// Causal softmax attention over packed sequences with grouped heads, forward.
//
//   query t of a sequence of lq queries and lk keys sees its keys 0 .. t + lk - lq:
//   S = scale q k^T,  P = softmax of the keys that are seen,  a = P v,  lse = log sum exp S;  no key seen: a = 0, lse = -inf
//
// A workgroup owns 64 or 128 rows of one head of keys, rows being (token, head of the group) with the head fastest: the query heads that share keys share every tile of
// them, and a token's position decides how much a row sees.  K and V stream through LDS past the own rows (attention_mfma.hip: the order of the products).
#pragma once
#include "packed.h"

namespace mtnlg {

namespace {

// rows of a tile: what 160 KB of LDS hold twice of K and V, and two workgroups of each
template <typename E> constexpr int tile_rows() { return sizeof(E) == 2 ? 64 : 32; }
template <typename E, int D> constexpr int fwd_stage() { return 2 * tile_rows<E>() * D * (int)sizeof(E); }
template <typename E, int D> constexpr int fwd_per_unit() { return 2 * 2 * fwd_stage<E, D>() <= 160 * 1024 ? 2 : 1; }

// SPLIT 2: 64 rows to a workgroup, waves 0, 1 take the first 32 keys of every tile, waves 2, 3 the last; SPLIT 1: 128 rows
template <typename E, int D, int SPLIT>
__global__ __launch_bounds__(256, (fwd_per_unit<E, D>())) void packed_fwd_kernel(PackedFwdArgs w) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  using P = Elem<E, D>;
  constexpr int TR = tile_rows<E>(), K1 = P::K1, CB = D / 32, MATRIX = TR * D * (int)sizeof(E), STAGE = 2 * MATRIX, SUB = 2 * P::BAND;
  constexpr int OWNED = 128 / SPLIT, SUBS = TR / 32 / SPLIT;
  static_assert(SUBS >= 1, "");
  const int lane = threadIdx.x & 63, h = lane >> 5, r = w.group, d = w.d;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int j = blockIdx.x % w.kv_heads;
  const bool chunked = w.chunk > 0;
  auto chunks_of = [&](const Span &s) { return chunked ? min((max(s.lk, 1) + w.chunk - 1) / w.chunk, w.chunks) : 1; };
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

  const int part = SPLIT == 2 ? wave >> 1 : 0, rows_of = SPLIT == 2 ? wave & 1 : wave;
  const int own0 = block0 + rows_of * 32, mine = own0 + (lane & 31), row = min(mine, rows - 1);
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
      const int key0 = begin + it * TR + 32 * (part + sub);
      if (key0 > most) continue;   // nothing that a row of the wave sees
      const char *K = smem + (it & 1) * STAGE + (part + sub) * SUB, *V = K + MATRIX;
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
  if constexpr (SPLIT == 2) {   // the two halves of the keys, relative to the larger of the maxima
    f32x4 *slots = reinterpret_cast<f32x4 *>(smem) + lane;
    float *const stat = reinterpret_cast<float *>(smem + 4 * CB * 2048);
    const int other = wave ^ 2;
    __syncthreads();   // the stages are no longer read
    stat[wave * 128 + lane] = m;
    stat[wave * 128 + 64 + lane] = l;
    __syncthreads();
    const float mo = stat[other * 128 + lane], lo = stat[other * 128 + 64 + lane], both = fmaxf(m, mo), ref = both == -INFINITY ? 0.0f : both;
    auto relative = [&](float x) { return EXACT ? exact_exp(product_of(x, w.scale) - product_of(ref, w.scale)) : fast_exp2((x - ref) * c); };
    const float mul = relative(m);
    l = part ? fmaf(l, mul, lo * relative(mo)) : fmaf(lo, relative(mo), l * mul);
    m = both;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) o[cb] *= mul;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int q = 0; q < 2; ++q) slots[((wave * CB + cb) * 2 + q) * 64] = part ? quarter_of(o[cb], q) : quarter_of(o[cb], 2 + q);
    __syncthreads();
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const f32x4 rest = slots[((other * CB + cb) * 2 + q) * 64];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (part) o[cb][8 + 4 * q + e] += rest[e];
          else o[cb][4 * q + e] += rest[e];
        }
      }
  }
  if (mine >= rows) return;
  const int head = j * r + g;
  constexpr int FROM = 0, TO = 4;
  if (chunked) {
    const int64_t id = (int64_t)(s.q0 + tok) * ((int64_t)w.kv_heads * r) + head, at = chunk * ((int64_t)w.where.q_tokens * w.kv_heads * r) + id;
    float *const to = w.part + at * d;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int q = FROM; q < TO; ++q) {
        const int col = 32 * cb + 8 * q + 4 * h;
        if (col < d && (SPLIT == 1 || q / 2 == part)) *reinterpret_cast<f32x4 *>(to + col) = quarter_of(o[cb], q);
      }
    if (h == 0 && part == 0) *reinterpret_cast<float2 *>(w.stat + 2 * at) = float2{m, l};
    return;
  }
  const bool none = tok + shift < 0;   // the row sees no key
  const float inv = none ? 0.0f : 1.0f / l;
  E *const to = row_at<E>(w.a, s.q0 + tok, j, g);
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int q = FROM; q < TO; ++q) {
      const int col = 32 * cb + 8 * q + 4 * h;
      if (col < d && (SPLIT == 1 || q / 2 == part)) put4(to + col, quarter_of(o[cb], q) * inv);
    }
  if (h == 0 && part == 0) w.lse[(int64_t)head * w.where.q_tokens + s.q0 + tok] = none ? -INFINITY : plus_log(product_of(m, w.scale), l);
}

template <typename E, int D, int SPLIT>
int fwd_launch(const PackedFwdArgs &w, int64_t blocks, hipStream_t st) {
  constexpr int CB = D / 32, merge = SPLIT == 2 ? 4 * (CB * 2048 + 512) : 0, ring = 2 * fwd_stage<E, D>(), smem = ring > merge ? ring : merge;
  static unsigned long long attr_done = 0;
  int device;
  if (!attr_is_set(attr_done, &device)) {
    MTNLG_TRY(set_lds(packed_fwd_kernel<E, D, SPLIT>, smem));
    attr_mark_set(attr_done, device);
  }
  packed_fwd_kernel<E, D, SPLIT><<<(unsigned)blocks, 256, smem, st>>>(w);
  return check_launch();
}

}  // namespace

}  // namespace mtnlg
