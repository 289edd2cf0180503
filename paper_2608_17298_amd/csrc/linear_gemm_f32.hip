// Tiled products and few-row kernels of the linear layer in float.
#include "linear_gemm.h"
#include "linear_rows.h"

namespace gart {

template hipError_t gemm_forward<float>(const LinearArgs&, hipStream_t);
template hipError_t gemm_backward<float>(const LinearArgs&, hipStream_t);
template hipError_t rows_forward<float>(const LinearArgs&, hipStream_t);
template hipError_t rows_dz<float>(const LinearArgs&, void*, int64_t, int64_t, hipStream_t);

}  // namespace gart
