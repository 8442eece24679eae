// Products of quantised matrices, A in E5M2, B in E5M2 (kernel: gemm_fp8.h).
#include "gemm_fp8.h"

namespace t5mi {

hipError_t launch_gemm_fp8_55(const Fp8Gemm& g, hipStream_t st) { return launch_fp8_types<T5_E5M2, T5_E5M2>(g, st); }

}  // namespace t5mi
