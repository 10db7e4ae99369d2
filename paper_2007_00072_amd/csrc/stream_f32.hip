// Streaming attention kernels for float32 storage.
#include "stream_kernels.hpp"

namespace dm {

template void stream_fwd<float>(const StreamArgs&, bool, hipStream_t);
template void stream_bwd<float>(const StreamArgs&, hipStream_t);

}  // namespace dm
