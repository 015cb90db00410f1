// Instances of the product kernel that only the log probabilities use: logits reduced to
// what log-sum-exp, entropy and top alternatives need, or turned into their gradient (both
// operands k-contiguous).
#include "gemm_tile.h"

namespace ls {

hipError_t gemm_logprob(const GemmArgs& a, GemmTile t, hipStream_t s) {
  switch (a.epi) {
    case EPI_STAT:
      return t == TILE_256 ? launch<true, true, EPI_STAT, 256, 256>(a, s) : launch_narrow<true, true, EPI_STAT>(a, t, s);
    case EPI_DLP:
      return t == TILE_256 ? launch<true, true, EPI_DLP, 256, 256>(a, s) : launch_narrow<true, true, EPI_DLP>(a, t, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace ls
