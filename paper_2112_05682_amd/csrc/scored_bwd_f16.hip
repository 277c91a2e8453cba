// Backward of attention with modified scores: _Float16 operands.
#include "scored_bwd.hpp"

namespace mea {

template hipError_t launch_scored_bwd<_Float16>(const ScoredBwdParams&, int, hipStream_t);

}  // namespace mea
