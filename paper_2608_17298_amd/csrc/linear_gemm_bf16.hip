// Tiled products and few-row kernels of the linear layer in bf16.
#include "linear_gemm.h"
#include "linear_rows.h"

namespace gart {

template hipError_t gemm_forward<bf16>(const LinearArgs&, hipStream_t);
template hipError_t gemm_backward<bf16>(const LinearArgs&, hipStream_t);
template hipError_t rows_forward<bf16>(const LinearArgs&, hipStream_t);
template hipError_t rows_dz<bf16>(const LinearArgs&, void*, int64_t, int64_t, hipStream_t);

}  // namespace gart
