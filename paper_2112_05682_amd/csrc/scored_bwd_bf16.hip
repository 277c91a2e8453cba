// Backward of attention with modified scores: __bf16 operands.
#include "scored_bwd.hpp"

namespace mea {

template hipError_t launch_scored_bwd<__bf16>(const ScoredBwdParams&, int, hipStream_t);

}  // namespace mea
