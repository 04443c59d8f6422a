// The head's matrix products on tiles of 128 x 128 (head_gemm_kernel.h)
#include "head_gemm_kernel.h"

namespace capscaps {

hipError_t launch_head_gemm_128(const HeadGemm& g, HeadEnd end, hipStream_t st) { return launch_end<128, 128, 2, 4>(g, end, st); }
hipError_t launch_head_gemm_pair_128(const HeadGemm& a, const HeadGemm& b, hipStream_t st) { return launch_pair<128, 128, 2, 4>(a, b, st); }

}  // namespace capscaps
