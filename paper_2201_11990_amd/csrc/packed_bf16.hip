// Attention over packed sequences, bf16 (packed_fwd.h, packed_bwd.h).
#include "packed_bwd.h"
#include "packed_fwd.h"

namespace mtnlg {

int packed_fwd_bf16(const PackedFwdArgs &w, int owned, int64_t blocks, hipStream_t st) {
  return packed_by_size(w.d, [&](auto D) {
    constexpr int d = decltype(D)::value;
    return owned == 64 ? fwd_launch<bf16, d, 2>(w, blocks, st) : fwd_launch<bf16, d, 1>(w, blocks, st);
  });
}

int packed_bwd_bf16(const PackedBwdArgs &w, int owned, int64_t pieces, int64_t key_pieces, hipStream_t st) {
  return packed_by_size(w.d, [&](auto D) { return bwd_launch<bf16, decltype(D)::value>(w, owned, pieces, key_pieces, st); });
}

int packed_dkv_owned(int dtype, int d) {
  return packed_by_size(d, [&](auto D) {
    constexpr int n = decltype(D)::value;
    return dtype == MTNLG_F32 ? Dkv<float, n>::OWNED : Dkv<bf16, n>::OWNED;
  });
}

}  // namespace mtnlg
