// Instances of the product kernel that only the head loss uses: logits reduced or
// turned into their gradient in the epilogue (both operands k-contiguous), dh
// accumulated in fp32 over pieces of the vocabulary (k-strided B), and the head's
// gradient in bf16 (both operands k-strided).
#include "gemm_tile.h"

namespace ls {

hipError_t gemm_head(const GemmArgs& a, GemmTile t, hipStream_t s) {
  if (a.b_kcontig) {
    if (a.epi == EPI_LSE)
      return t == TILE_256 ? launch<true, true, EPI_LSE, 256, 256>(a, s) : launch_narrow<true, true, EPI_LSE>(a, t, s);
    if (a.epi == EPI_DZ)
      return t == TILE_256 ? launch<true, true, EPI_DZ, 256, 256>(a, s) : launch_narrow<true, true, EPI_DZ>(a, t, s);
  } else if (a.a_kcontig) {
    switch (t) {
      case TILE_256: return launch<true, false, EPI_F32, 256, 256>(a, s);
      case TILE_256x192: return launch<true, false, EPI_F32, 256, 192>(a, s);
      default: return launch_narrow<true, false, EPI_F32>(a, t, s);
    }
  } else if (a.epi == EPI_BF16) {
    switch (t) {
      case TILE_256: return launch<false, false, EPI_BF16, 256, 256>(a, s);
      case TILE_256x192: return launch<false, false, EPI_BF16, 256, 192>(a, s);
      default: return launch_narrow<false, false, EPI_BF16>(a, t, s);
    }
  } else if (a.epi == EPI_PART && t == TILE_256) {
    return launch<false, false, EPI_PART, 256, 256>(a, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace ls
