// Forward of attention with modified scores: _Float16 operands.
#include "scored_fwd.hpp"

namespace mea {

template hipError_t launch_stream<_Float16>(const StreamParams&, int, int, hipStream_t);
template hipError_t launch_stream_pair<_Float16>(const StreamParams&, const StreamParams&, int, int, int, hipStream_t);
template hipError_t launch_scored_combine<_Float16>(const StreamParams&, int, int, hipStream_t);

}  // namespace mea
