// What the kernels of attention over packed sequences with grouped heads share (packed_fwd.hip, packed_bwd.hip): where a sequence lies, tiles of either
// element type in LDS and the streams that fill them, fragments, products with masked rows that are not finite.
#pragma once
#include "attention_tiles.h"

namespace mtnlg {

struct Sequences {
  const int32_t *q_offsets, *k_offsets, *q_lengths, *k_lengths;
  int count, q_tokens, k_tokens;
};
struct PackedShape {
  int dtype, heads, kv_heads, group, d;
  float scale;
  Sequences where;
  int max_q, max_k;
};
int packed_shape(const mtnlg_packed_desc *desc, PackedShape *S);   // checks the descriptor

// A matrix of heads on the device, strides in elements.
struct Heads {
  void *base;
  int64_t token, group, head;
};
struct PackedFwdArgs {
  Sequences where;
  int kv_heads, group, d, chunk, chunks;   // chunk: keys that a workgroup takes at most (0: all); chunks: how many of those there are at most
  float scale;
  Heads q, k, v, a;
  float *lse;
  float *part, *stat;   // of chunks: results relative to a maximum, and the maximum and the sum of each row
};

struct PackedBwdArgs {
  Sequences where;
  int kv_heads, group, d, splits;   // splits: parts of a dk / dv workgroup's tiles
  float scale;
  Heads q, k, v, a, da, dq, dk, dv;
  const float *lse;
  float *D, *part;
  int chunk, chunks;   // packed_plain.hip: keys that a dq workgroup takes at most (0: all), how many of those there are at most
  float *dq_part;      // of chunks
};

// Head sizes up to which bf16 has kernels of its own (packed_fwd.hip, packed_bwd.hip); others and fp32: packed_plain.hip.
constexpr int PACKED_TUNED = 192;
inline bool packed_tuned(int dtype, int d) { return dtype == MTNLG_BF16 && d <= PACKED_TUNED; }
// Rows of a workgroup of the forward pass and of dq: 128, and 64 (a pair of waves to 32 rows, each with half of a tile's keys) while 128 would leave some of the
// places for workgroups, two to a unit or one, empty.  2501 and 1589 tokens, median us with 64 / 128: forward, 480 workgroups of 128 at heads of 128: 61 / 61, 384: 44 / 59;
// heads of 192, 384: 73 / 64, 256: 52 / 62.  dq, dk and dv, heads of 128, 480: 194 / 188, 384: 145 / 157; heads of 192, 384: 265 / 251, 256: 174 / 183; heads of 160: 324 / 266
// at 480 and 111 / 98 at 32 (64 keep twice as much in scratch memory), so always 128.
constexpr int packed_fwd_places(int d) { return d <= 160 ? 512 : 256; }
constexpr int packed_dq_places(int d) { return d <= 128 ? 512 : d <= 160 ? 0 : 256; }
// owned: rows of a workgroup (plain: 128); blocks, pieces: workgroups, of all heads of keys and of one
int packed_fwd_tuned(const PackedFwdArgs &w, int owned, int64_t blocks, hipStream_t st);
int packed_fwd_plain(int dtype, const PackedFwdArgs &w, int64_t blocks, hipStream_t st);
int packed_bwd_tuned(const PackedBwdArgs &w, int owned, int64_t pieces, int64_t key_pieces, hipStream_t st);
int packed_bwd_plain(int dtype, const PackedBwdArgs &w, int64_t pieces, int64_t key_pieces, hipStream_t st);
int packed_dkv_plain_owned(int dtype, int d);   // keys of a workgroup of dk / dv
int packed_dkv_tuned_owned(int d);              // ... of the tuned kernels

namespace {

// ------------------------------------------------------------------ sequences
struct Span { int q0, lq, k0, lk; };   // first rows and lengths

// Whatever the arrays hold, what comes out lies inside the matrices.
__device__ __forceinline__ void part_of(const int32_t *offsets, const int32_t *lengths, int tokens, int i, int &first, int &length) {
  const int a = offsets[i], b = offsets[i + 1];
  first = a < 0 ? 0 : a > tokens ? tokens : a;
  const int last = b < first ? first : b > tokens ? tokens : b;
  length = last - first;
  if (lengths != nullptr) {
    const int n = lengths[i];
    length = n < 0 ? 0 : n < length ? n : length;
  }
}
__device__ __forceinline__ Span span_of(const Sequences &s, int i) {
  Span p;
  part_of(s.q_offsets, s.q_lengths, s.q_tokens, i, p.q0, p.lq);
  part_of(s.k_offsets, s.k_lengths, s.k_tokens, i, p.k0, p.lk);
  return p;
}

// Which sequence holds the place-th piece of work, and which of the sequence's pieces it is (at): count(span) says how many a sequence has.  Lengths are known
// on the device only, so every wave looks for itself.  Up to 32 sequences, the ones with the most keys come first: what is left over at the end of a call are
// the pieces of short ones.  More: a lane counts a few consecutive sequences, a sum over the lanes before it finds the lane, and again inside that lane's sequences.
// False: fewer pieces than places.  Median us, longest first / as they come (one run of each kind of length): documents of 32 to 2048 tokens, 16 heads of 128 on 4, forward and backward,
// 8: 43 and 147 / 49 and 160, 16: 50 and 180 / 60 and 212, 24: 84 and 282 / 91 and 317, 32: 64 and 207 / 62 and 202, 40: 101 and 334 / 100 and 348, 64: 143 and 480 / 127 and 452;
// single tokens over 64 to 16384 keys, 32 heads of 128 on 8, 16: 53 / 51, 24: 86 / 88, 32: 96 / 95, 40: 140 / 136, 64: 171 / 165.  Counting costs each wave a turn to a sequence.
template <typename Count>
__device__ __forceinline__ bool find_piece(const Sequences &s, unsigned place, Count &&count, Span &found, unsigned &at) {
  if (s.count <= 32) {
    const int i = threadIdx.x & 63;
    unsigned mine = 0, before = 0;
    int keys = -1;
    if (i < s.count) {
      const Span p = span_of(s, i);
      mine = count(p);
      keys = p.lk;
    }
    for (int o = 0; o < s.count; ++o) {
      const int other = __builtin_amdgcn_readlane(keys, o);
      const unsigned n = (unsigned)__builtin_amdgcn_readlane((int)mine, o);
      before += other > keys || (other == keys && o < i) ? n : 0;
    }
    const uint64_t holds = __builtin_amdgcn_ballot_w64(place >= before && place - before < mine);
    if (holds == 0) return false;
    const int l = __builtin_ctzll(holds);
    found = span_of(s, l);
    at = place - (unsigned)__builtin_amdgcn_readlane((int)before, l);
    return true;
  }
  const int lane = threadIdx.x & 63;
  int first = 0, n = s.count;
  unsigned before = 0;
  while (true) {
    const int per = (n + 63) / 64, lo = first + lane * per, hi = lo + per < first + n ? lo + per : first + n;
    unsigned mine = 0;
    for (int i = lo; i < hi; ++i) mine += count(span_of(s, i));
    unsigned upto = mine;
#pragma unroll
    for (int off = 1; off < 64; off *= 2) {
      const unsigned t = __shfl_up(upto, off, 64);
      if (lane >= off) upto += t;
    }
    upto += before;
    const uint64_t holds = __builtin_amdgcn_ballot_w64(place < upto);
    if (holds == 0) return false;
    const int l = __builtin_ctzll(holds);
    before = (unsigned)__builtin_amdgcn_readlane((int)(upto - mine), l);
    first += l * per;
    if (per == 1) break;
    n = per < n - l * per ? per : n - l * per;
  }
  found = span_of(s, __builtin_amdgcn_readfirstlane(first));
  at = place - before;
  return true;
}

template <typename E>
__device__ __forceinline__ E *row_at(const Heads &m, int64_t token, int group, int head) {
  return static_cast<E *>(m.base) + token * m.token + group * m.group + head * m.head;
}

// Rows of a matrix from one on: what tile number t of TR rows has, rows past the end as zeros.
struct RowStream {
  const char *base;
  int rows;
  uint32_t pitch;
  template <int TR>
  __device__ __forceinline__ dma_rsrc_t tile(int t) const {
    int left = rows - t * TR;
    left = left < 0 ? 0 : left < TR ? left : TR;
    return dma_rsrc(base + (int64_t)t * TR * pitch, __builtin_amdgcn_readfirstlane((uint32_t)left * pitch));
  }
};

// The same as a walk from tile to tile in scalar registers (the compiler clamps and multiplies on the vector unit).
struct RowWalk {
  uint64_t base;
  int rows;
  uint32_t pitch, step;   // bytes of a row, of a tile
  __device__ __forceinline__ RowWalk(const void *first, int n, uint32_t pitch_, int tile_rows) {
    const uint64_t a = (uint64_t)first;
    base = ((uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(a >> 32)) << 32) | (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)a);
    rows = __builtin_amdgcn_readfirstlane(n);
    pitch = __builtin_amdgcn_readfirstlane(pitch_);
    step = pitch * (uint32_t)tile_rows;
  }
  template <int TR>
  __device__ __forceinline__ dma_rsrc_t tile(int row = 0) const {   // TR rows, from a row of the present tile on
    uint32_t records;
    asm("s_max_i32 %0, %1, 0\n\ts_min_i32 %0, %0, %2\n\ts_mul_i32 %0, %0, %3" : "=&s"(records) : "s"(rows - row), "n"(TR), "s"(pitch) : "scc");
    return dma_rsrc((const void *)(base + (uint32_t)row * pitch), records);
  }
  template <int TR>
  __device__ __forceinline__ void advance() {
    base += step;
    rows -= TR;
  }
};

// ------------------------------------------------------------------ element types
// Tiles hold rows as in memory, d columns filled up with zeros to D, 16-byte units permuted by row.  A step of a first product (contracting over columns) is one
// 16-byte piece of a row: 16 columns of bf16 (one MFMA), 8 of fp32 (four).  A step of a second product (contracting over 16 rows of the tile) is a 32-column block: one MFMA
// of bf16, eight of fp32.  Blocks of either come out as C[tile row 8 (i / 4) + 4 (lane / 32) + i % 4][own row lane % 32], i < 16.
template <typename E, int D> struct Elem;

template <int D>
struct Elem<bf16, D> {
  using T = Tile<D, true>;
  using Lane = typename T::Lane32;
  using Unit = bf16x8;
  using Column = bf16x8;
  using Weights = bf16x8;
  static constexpr int K1 = D / 16, UNIT = 8, NI = T::NI, BAND = T::ROWS16;   // BAND: bytes of 16 rows, NI of a wave's DMA instructions
  static __device__ __forceinline__ uint32_t dma_offset(uint32_t pitch, int band, int lane, int i, int d) { return T::dma_offset(pitch, band, lane, i, d); }
  static __device__ __forceinline__ Unit unit(const char *t, const Lane &ln, int kk) { return T::nat32(t, ln, kk); }
  static __device__ __forceinline__ Column column(const char *t, const Lane &ln, int cb, int half) { return T::tr32(t, ln, cb, half); }
  static __device__ __forceinline__ f32x16 mma(const Unit &a, const Unit &b, f32x16 c) { return MFMA32(a, b, c); }
  static __device__ __forceinline__ f32x16 mma_rows(const Column &a, const Weights &b, f32x16 c) { return MFMA32(a, b, c); }
  // P and dS round to bf16: relative to themselves, as the results they enter do once more
  static __device__ __forceinline__ Weights weights(const f32x16 &v, int half) {
    Weights w;
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = (bf16)v[8 * half + e];
    return w;
  }
  // columns 32 cb + 8 q + 4 h .. + 3 of a tile's row
  static __device__ __forceinline__ f32x4 row4(const char *t, int row, int cb, int q, int h) {
    return load4(reinterpret_cast<const bf16 *>(t + T::off(row, 4 * cb + q) + 8 * h));
  }
  static __device__ __forceinline__ float not_finite(const Unit &u, float z) {   // NaN if any is an infinity or NaN
#pragma unroll
    for (int i = 0; i < 8; i += 2) z = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{u[i], u[i + 1]}, bf16x2{(bf16)0.0f, (bf16)0.0f}, z, false);
    return z;
  }
  static __device__ __forceinline__ float dot(const Unit &a, const Unit &b, float s) {
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf((float)a[e], (float)b[e], s);
    return s;
  }
};

template <int D>
struct Elem<float, D> {
  static constexpr int K1 = D / 8, UNIT = 4, UPR = D / 4, NI = D / 16, BAND = 16 * UPR * 16;
  static constexpr bool WIDE = UPR % 16 == 0;   // a row is a multiple of 256 bytes
  using Unit = f32x4;
  typedef __attribute__((ext_vector_type(8))) float Column;
  using Weights = Column;
  // 16-byte reads of 16 rows that differ in their low four bits fall on all banks, 4-byte reads of 32 consecutive columns in two rows that are 4 apart too
  static __device__ __forceinline__ int mask(int row) { return WIDE ? (row & 3) | (row >> 3 & 1) << 2 | (row >> 2 & 1) << 3 : row >> 1 & 7; }
  static __device__ __forceinline__ int off(int row, int u) { return (row * UPR + (u ^ mask(row))) * 16; }
  static __device__ __forceinline__ uint32_t dma_offset(uint32_t pitch, int band, int lane, int i, int d) {
    const int p = i * 64 + lane, r = 16 * band + p / UPR, u = (p % UPR) ^ mask(r);
    return u * 4 < d ? r * pitch + u * 16 : 0xFFFFFFF0u;
  }
  struct Lane {
    uint32_t n0, t0;
    __device__ __forceinline__ explicit Lane(int lane) {
      const int h = lane >> 5, c = lane & 31;
      n0 = (uint32_t)off(c, h);
      t0 = (uint32_t)(4 * h * UPR * 16 + (((c >> 2) ^ (WIDE ? h << 3 : h << 1)) * 16) + (c & 3) * 4);
    }
    __device__ __forceinline__ void here() { asm volatile("" : "+v"(n0), "+v"(t0)); }
  };
  static __device__ __forceinline__ Unit unit(const char *t, const Lane &ln, int kk) {
    const uint32_t at = WIDE ? (ln.n0 ^ ((kk & 7) * 32)) + (kk >> 3) * 256 : (ln.n0 ^ ((kk & 3) * 32)) + (kk >> 2) * 128;
    return *reinterpret_cast<const Unit *>(t + at);
  }
  static __device__ __forceinline__ Column column(const char *t, const Lane &ln, int cb, int half) {
    Column v;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int rows = (16 * half + 8 * (i >> 2) + (i & 3)) * UPR * 16;
      const uint32_t at = WIDE ? (ln.t0 ^ (((cb & 1) << 3 | (i & 3) | (i >> 2 & 1) << 2) * 16)) + (cb >> 1) * 256
                               : (ln.t0 ^ (((i >> 1 & 1) | (i >> 2 & 1) << 2) * 16)) + cb * 128;
      v[i] = *reinterpret_cast<const float *>(t + at + rows);
    }
    return v;
  }
  static __device__ __forceinline__ f32x16 mma(const Unit &a, const Unit &b, f32x16 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ f32x16 mma_rows(const Column &a, const Weights &b, f32x16 c) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ Weights weights(const f32x16 &v, int half) {
    Weights w;
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = v[8 * half + e];
    return w;
  }
  static __device__ __forceinline__ f32x4 row4(const char *t, int row, int cb, int q, int h) {
    return *reinterpret_cast<const f32x4 *>(t + off(row, 8 * cb + 2 * q + h));
  }
  static __device__ __forceinline__ float not_finite(const Unit &u, float z) {
#pragma unroll
    for (int i = 0; i < 4; ++i) z = fmaf(u[i], 0.0f, z);
    return z;
  }
  static __device__ __forceinline__ float dot(const Unit &a, const Unit &b, float s) {
#pragma unroll
    for (int e = 0; e < 4; ++e) s = fmaf(a[e], b[e], s);
    return s;
  }
};

// Piece kk of a row in memory (columns 2 UNIT kk + UNIT h .. ), zeros past d
template <typename E, int D>
__device__ __forceinline__ typename Elem<E, D>::Unit row_unit(const E *row, int kk, int h, int d) {
  using P = Elem<E, D>;
  const int col = (2 * kk + h) * P::UNIT;
  typename P::Unit v = {};
  if (col < d) v = *reinterpret_cast<const typename P::Unit *>(row + col);
  return v;
}

// e^(s scale - shift): bf16 by one multiplication (f and shift have the factor log2 e), fp32 rounded as the scale and e^x are
template <typename E>
__device__ __forceinline__ float weight_of(float s, float f, float shift) { return weight<sizeof(E) == 4>(s, f, shift); }

// Whether 32 rows of a tile hold an infinity or NaN: asked where a mask hides some of them from some of the wave's rows, whose weights there are zeros
// (0 x inf would be NaN in rows that do not depend on it).
template <typename E, int D>
__device__ __forceinline__ bool rows_not_finite(const char *t, typename Elem<E, D>::Lane ln) {
  float z = 0.0f;
  ln.here();   // (as above: not for every tile)
#pragma unroll
  for (int kk = 0; kk < Elem<E, D>::K1; ++kk) {
    z = Elem<E, D>::not_finite(Elem<E, D>::unit(t, ln, kk), z);
    if (kk % 4 == 3) __builtin_amdgcn_sched_barrier(0);
  }
  return __builtin_amdgcn_ballot_w64(z != 0.0f) != 0;
}
// Then the product with 32 rows of the tile is taken row by row, from the weights w of those rows R that the own row sees.
template <typename E, int D, typename Seen>
__device__ __forceinline__ void add_seen_rows(f32x16 (&acc)[D / 32], const f32x16 &w, const char *t, Seen &&seen) {
  const int lane = threadIdx.x & 63, h = lane >> 5;
#pragma unroll 1
  for (int row = 0; row < 32; ++row) {
    const int at = 4 * (row >> 3) + (row & 3);
    float p = w[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) p = at == e ? w[e] : p;
    p = __shfl(p, (lane & 31) + 32 * (row >> 2 & 1), 64);
    if (!seen(row)) continue;
#pragma unroll
    for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 v = Elem<E, D>::row4(t, row, cb, q, h);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[cb][4 * q + e] = fmaf(p, v[e], acc[cb][4 * q + e]);
        __builtin_amdgcn_sched_barrier(0);   // no registers for more reads at once
      }
  }
}

// a result's columns 32 cb + 8 q + 4 h .. + 3
template <typename E>
__device__ __forceinline__ void put4(E *p, f32x4 v) {
  if constexpr (sizeof(E) == 4) *reinterpret_cast<f32x4 *>(p) = v;
  else *reinterpret_cast<bf16x4 *>(p) = bf16x4{(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3]};
}

// ------------------------------------------------------------------ host side
// (one token: its stride is never taken but as the bound of what a tile reads)
inline Heads heads_of(const mtnlg_heads *m, int64_t tokens, int d) { return Heads{m->data, tokens == 1 ? d : m->token, m->group, m->head}; }

// Pieces of `rows` rows that all sequences together can have, each of up to `most` of which all have `total`
inline int64_t pieces_bound(int64_t total, int64_t most, int count, int rows) {
  const int64_t by_total = total / rows + count, by_most = (int64_t)count * ((most + rows - 1) / rows);
  return by_total < by_most ? by_total : by_most;
}

template <typename F>
int packed_tuned_by_size(int d, F &&f) {
  if (d <= 64) return f(std::integral_constant<int, 64>{});
  if (d <= 96) return f(std::integral_constant<int, 96>{});
  if (d <= 128) return f(std::integral_constant<int, 128>{});
  if (d <= 160) return f(std::integral_constant<int, 160>{});
  return f(std::integral_constant<int, 192>{});
}
template <typename F>
int packed_by_size(int d, F &&f) {   // head sizes in tiles of the next multiple of 32 columns that there are kernels for
  return d <= PACKED_TUNED ? packed_tuned_by_size(d, f) : f(std::integral_constant<int, 256>{});
}

}  // namespace

}  // namespace mtnlg
