// Backward of attention with modified scores: float operands.
#include "scored_bwd.hpp"

namespace mea {

template hipError_t launch_scored_bwd<float>(const ScoredBwdParams&, int, hipStream_t);

}  // namespace mea
