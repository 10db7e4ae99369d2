// Streaming attention kernels for fp16 storage.
#include "stream_kernels.hpp"

namespace dm {

template void stream_fwd<half_t>(const StreamArgs&, bool, hipStream_t);
template void stream_bwd<half_t>(const StreamArgs&, hipStream_t);

}  // namespace dm
