// Instances of the product kernel that only the head loss uses: logits reduced or
// turned into their gradient in the epilogue (both operands k-contiguous), dh
// summed in fp32 over pieces of the vocabulary (k-strided B), and the head's
// gradient, in fp32 or bf16 (both operands k-strided).
#include "gemm_tile.h"

namespace ls {

hipError_t gemm_head(const GemmArgs& a, GemmTile t, hipStream_t s) {
  switch (a.epi) {
    case EPI_LSE:
      return t == TILE_256 ? launch<true, true, EPI_LSE, 256, 256>(a, s) : launch_narrow<true, true, EPI_LSE>(a, t, s);
    case EPI_DZ:
      return t == TILE_256 ? launch<true, true, EPI_DZ, 256, 256>(a, s) : launch_narrow<true, true, EPI_DZ>(a, t, s);
    case EPI_DH:
      switch (t) {
        case TILE_256: return launch<true, false, EPI_DH, 256, 256>(a, s);
        case TILE_256x192: return launch<true, false, EPI_DH, 256, 192>(a, s);
        default: return launch_narrow<true, false, EPI_DH>(a, t, s);
      }
    case EPI_DE:
      switch (t) {
        case TILE_256: return launch<false, false, EPI_DE, 256, 256>(a, s);
        case TILE_256x192: return launch<false, false, EPI_DE, 256, 192>(a, s);
        default: return launch_narrow<false, false, EPI_DE>(a, t, s);
      }
    case EPI_DE16:
      switch (t) {
        case TILE_256: return launch<false, false, EPI_DE16, 256, 256>(a, s);
        case TILE_256x192: return launch<false, false, EPI_DE16, 256, 192>(a, s);
        default: return launch_narrow<false, false, EPI_DE16>(a, t, s);
      }
    case EPI_PART:
      return t == TILE_256 && !a.a_kcontig ? launch<false, false, EPI_PART, 256, 256>(a, s) : hipErrorInvalidValue;
    default: return hipErrorInvalidValue;
  }
}

}  // namespace ls
