// Streaming kernels of the linear layer in float.
#include "linear_stream.h"

namespace gart {

template hipError_t stream_forward<float>(const LinearArgs&, hipStream_t);
template hipError_t stream_backward<float>(const LinearArgs&, float*, hipStream_t);

}  // namespace gart
