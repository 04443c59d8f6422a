// The head's matrix products on tiles of 128 x 256, two workgroups on a CU (head_gemm_kernel.h)
#include "head_gemm_kernel.h"

namespace capscaps {

hipError_t launch_head_gemm_half(const HeadGemm& g, HeadEnd end, hipStream_t st) { return launch_end<128, 256, 2, 3>(g, end, st); }

}  // namespace capscaps
