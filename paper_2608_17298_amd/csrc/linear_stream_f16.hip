// Streaming kernels of the linear layer in f16.
#include "linear_stream.h"

namespace gart {

template hipError_t stream_forward<f16>(const LinearArgs&, hipStream_t);
template hipError_t stream_backward<f16>(const LinearArgs&, float*, hipStream_t);

}  // namespace gart
