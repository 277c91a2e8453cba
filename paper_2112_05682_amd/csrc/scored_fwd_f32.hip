// Forward of attention with modified scores: float operands.
#include "scored_fwd.hpp"

namespace mea {

template hipError_t launch_stream<float>(const StreamParams&, int, int, hipStream_t);
template hipError_t launch_stream_pair<float>(const StreamParams&, const StreamParams&, int, int, int, hipStream_t);
template hipError_t launch_scored_combine<float>(const StreamParams&, int, int, hipStream_t);

}  // namespace mea
