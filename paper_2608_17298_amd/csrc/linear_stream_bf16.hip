// Streaming kernels of the linear layer in bf16.
#include "linear_stream.h"

namespace gart {

template hipError_t stream_forward<bf16>(const LinearArgs&, hipStream_t);
template hipError_t stream_backward<bf16>(const LinearArgs&, float*, hipStream_t);

}  // namespace gart
