// Tiled products and few-row kernels of the linear layer in f16.
#include "linear_gemm.h"
#include "linear_rows.h"

namespace gart {

template hipError_t gemm_forward<f16>(const LinearArgs&, hipStream_t);
template hipError_t gemm_backward<f16>(const LinearArgs&, hipStream_t);
template hipError_t rows_forward<f16>(const LinearArgs&, hipStream_t);
template hipError_t rows_dz<f16>(const LinearArgs&, void*, int64_t, int64_t, hipStream_t);

}  // namespace gart
