// The head's matrix products on tiles of 64 x 128, for few rows (head_gemm_kernel.h)
#include "head_gemm_kernel.h"

namespace capscaps {

hipError_t launch_head_gemm_few_rows(const HeadGemm& g, HeadEnd end, hipStream_t st) { return launch_end<64, 128, 1, 6>(g, end, st); }

}  // namespace capscaps
