// The head's matrix products on tiles of 256 x 256, one workgroup on a CU (head_gemm_kernel.h)
#include "head_gemm_kernel.h"

namespace capscaps {

hipError_t launch_head_gemm_256(const HeadGemm& g, HeadEnd end, hipStream_t st) { return launch_end<256, 256, 2, 4>(g, end, st); }

}  // namespace capscaps
