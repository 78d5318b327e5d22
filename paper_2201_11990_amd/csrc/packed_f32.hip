// Attention over packed sequences, fp32 (packed_fwd.h, packed_bwd.h): the same kernels on v_mfma_f32_32x32x2_f32, P and dS in fp32.
#include "packed_bwd.h"
#include "packed_fwd.h"

namespace mtnlg {

int packed_fwd_f32(const PackedFwdArgs &w, int64_t blocks, hipStream_t st) {
  return packed_by_size(w.d, [&](auto D) { return fwd_launch<float, decltype(D)::value, 1>(w, blocks, st); });
}

int packed_bwd_f32(const PackedBwdArgs &w, int64_t pieces, int64_t key_pieces, hipStream_t st) {
  return packed_by_size(w.d, [&](auto D) { return bwd_launch<float, decltype(D)::value>(w, 128, pieces, key_pieces, st); });
}

}  // namespace mtnlg
