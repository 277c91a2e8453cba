// Forward of attention with modified scores: __bf16 operands.
#include "scored_fwd.hpp"

namespace mea {

template hipError_t launch_stream<__bf16>(const StreamParams&, int, int, hipStream_t);
template hipError_t launch_stream_pair<__bf16>(const StreamParams&, const StreamParams&, int, int, int, hipStream_t);
template hipError_t launch_scored_combine<__bf16>(const StreamParams&, int, int, hipStream_t);

}  // namespace mea
