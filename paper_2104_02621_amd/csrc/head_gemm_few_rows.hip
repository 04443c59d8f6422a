// The head's matrix products on tiles of 64 x 128, for few rows (head_gemm_kernel.h)
#include "head_gemm_kernel.h"

namespace capscaps {

hipError_t launch_head_gemm_few_rows(const HeadGemm& g, HeadEnd end, hipStream_t st) { return launch_end<64, 128, 1, 6>(g, end, st); }
hipError_t launch_head_gemm_pair_few_rows(const HeadGemm& a, const HeadGemm& b, hipStream_t st) { return launch_pair<64, 128, 1, 6>(a, b, st); }

}  // namespace capscaps
