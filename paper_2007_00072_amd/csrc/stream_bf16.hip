// Streaming attention kernels for bf16 storage.
#include "stream_kernels.hpp"

namespace dm {

template void stream_fwd<bf16_t>(const StreamArgs&, bool, hipStream_t);
template void stream_bwd<bf16_t>(const StreamArgs&, hipStream_t);

}  // namespace dm
