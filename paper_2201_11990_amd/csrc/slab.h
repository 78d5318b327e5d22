// A wave's slab of an operand in LDS, 128 bytes of k in each of some rows, brought by DMA, and the fragments that matrix instructions take from it:
// what the kernels share whose waves each take slabs of their own (gemm_wave.hip, gated_tokens.hip).
#pragma once
#include "gate.h"

namespace mtnlg {

namespace {

constexpr uint32_t RECORDS = 0xFFFFFFE0u, OUTSIDE = 0xFFFFFFF0u;   // bytes a descriptor covers at most; an offset beyond

typedef __attribute__((ext_vector_type(8))) short i16x8;
typedef __attribute__((ext_vector_type(4))) short i16x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((address_space(3))) i16x4 *lds_i16x4_ptr;

// One operand's slab in a wave's LDS: TB rows x 128 bytes of K.
//   K-contiguous: [TB rows][8 units of 16 bytes], unit c of row r at c ^ (r & 7).
//   Row-contiguous ([k][row] in memory): [k][TB rows], the units of a k-row permuted so that the reads below spread over the banks:
//     bf16 (transposing reads: 16 lanes take 4 k-rows x 32 bytes) by bits 1 and 3 of k; fp32, 32 rows: neighbouring k-rows
//     swap places where bit 2 of k is set; fp32, 64 rows: 256-byte k-rows need nothing.
// PAIRED: rows of the weights in pairs of both halves (gate.h), `half` rows apart.
template <typename E, int TB, bool ROWC, bool PAIRED = false>
struct Slab {
  static constexpr int ES = sizeof(E), EPU = 16 / ES, SK = 128 / ES;   // element size, elements of a unit, k of a slab
  static constexpr int NI = TB / 8;          // DMA instructions (1 KB each)
  static constexpr int UPR = TB / EPU;       // row-contiguous: units of a k-row
  static constexpr int BYTES = TB * 128;
  static __device__ __forceinline__ int mask(int k) {
    if constexpr (ES == 4) return 0;
    else if constexpr (TB == 64) return (k & 2) | ((k >> 1) & 4);
    else return (k >> 2) & 2;
  }
  static __device__ __forceinline__ int place(int k) { return ES == 4 && TB == 32 ? k ^ ((k >> 2) & 1) : k; }   // (its own inverse)

  uint32_t off[NI];   // byte offsets of this lane's units from the slab's first element; rows past the edge lie outside
  __device__ __forceinline__ Slab(int64_t ld, int64_t rows_left, int lane, int64_t half = 0) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      if constexpr (!ROWC) {
        const int row = 8 * i + (lane >> 3), c = (lane & 7) ^ (lane >> 3);
        off[i] = row < rows_left ? (uint32_t)((PAIRED ? gate_row(row, half) * ld : row * ld) * ES + c * 16) : OUTSIDE;
      } else {
        const int q = 64 * i + lane, k = place(q / UPR), u = (q % UPR) ^ mask(k);
        off[i] = u * EPU < rows_left ? (uint32_t)(k * ld * ES + u * 16) : OUTSIDE;
      }
    }
  }
  // ONCE: past the caches
  // the slab at k0 into LDS; first: element (first row of the tile, k = 0); what lies past K arrives as zeros
  template <bool ONCE = false>
  __device__ __forceinline__ void fetch(const E *first, int64_t ld, int64_t row0, int64_t k0, int64_t K, uint32_t lds, int lane) const {
    if constexpr (!ROWC) {
      const dma_rsrc_t rs = dma_rsrc(first + k0, RECORDS);
      const bool inside = k0 + ((lane & 7) ^ (lane >> 3)) * EPU < K;
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        if constexpr (ONCE) dma16_once(rs, lds + i * 1024, inside ? off[i] : OUTSIDE);
        else dma16(rs, lds + i * 1024, inside ? off[i] : OUTSIDE);
      }
    } else {
      const int64_t left = ((K - k0) * ld - row0) * ES;   // to the end of the matrix
      const dma_rsrc_t rs = dma_rsrc(first + k0 * ld, left < RECORDS ? (uint32_t)left : RECORDS);
#pragma unroll
      for (int i = 0; i < NI; ++i) dma16(rs, lds + i * 1024, off[i]);
    }
  }
};

// bf16: fragments of all blocks and both k-steps of a slab.  Lane l = 16 g + r holds row 16 b + r, k = 32 kk + 8 g .. + 7.
template <int TB, bool ROWC>
struct Frag16 {
  bf16x8 v[TB / 16][2];
  __device__ __forceinline__ void read(const char *stage, int lane) {
    using S = Slab<bf16, TB, ROWC>;
    const int g = lane >> 4, r = lane & 15;
#pragma unroll
    for (int b = 0; b < TB / 16; ++b)
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        if constexpr (!ROWC) {
          v[b][kk] = *reinterpret_cast<const bf16x8 *>(stage + (16 * b + r) * 128 + (((kk * 4 + g) ^ (r & 7)) << 4));
        } else {   // lane 16 g + L supplies the address of k-row 8 g + L / 4 (+ 4), rows 4 (L % 4) .. + 3 of the block
          const int u = 2 * b + ((r & 3) >> 1), k = 32 * kk + 8 * g + (r >> 2);
          const char *p = stage + k * (TB * 2) + ((u ^ S::mask(k)) << 4) + (r & 1) * 8;
          const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_ptr)p);
          const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_ptr)(p + 4 * (TB * 2)));
          const i16x8 t = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
          v[b][kk] = __builtin_bit_cast(bf16x8, t);
        }
      }
  }
};

}  // namespace

}  // namespace mtnlg
