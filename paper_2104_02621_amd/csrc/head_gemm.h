// Internal: the matrix products of a linear head over many classes (head_gemm.hip), for head_loss.hip.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/capscaps.h"

namespace capscaps {

constexpr int HEAD_K = 32;        // contracted values of a stage; rows are padded with zeros to a multiple
constexpr int HEAD_PRODUCTS = 6;  // fp32 operands: products of their bf16 terms

// out[m][n] = sum over k of a[m][k] * b[n][k].  Rows of a and b are whole 16-byte vectors at 16-byte addresses, zeros from the
// contracted length up to a multiple of HEAD_K; fp32 operands lie there as three bf16 terms one after another (`plane` values each).
struct HeadGemm {
    const void *a, *b;
    long long lda, ldb;        // bytes from row to row
    long long m_rows, n_rows;  // rows that may be read (beyond them: zeros)
    const int* m_count;        // NULL, or how many of the m rows count, in device memory
    const int* k_count;        // NULL, or how many contracted values count, in device memory
    long long k;
    int plane_a, plane_b;  // bytes of a term of fp32 operands
    int dtype;
    // out: fp32 (out_dtype) or 16 bits; parts of the contracted length go to copies `out_split` elements apart
    void* out;
    long long ldo, out_split;
    int out_dtype, splits;
    bool accumulate;      // add to what is there (fp32, one part)
    const float* scale;   // NULL, or what to multiply by, in device memory
};

// tile shapes
enum HeadTile { HEAD_TILE_256 = 0, HEAD_TILE_128 = 1, HEAD_TILE_FEW_ROWS = 2 };
struct HeadTileShape {
    int m, n;
};
inline HeadTileShape head_tile_shape(int tile)
{
    return tile == HEAD_TILE_256 ? HeadTileShape{256, 256} : tile == HEAD_TILE_128 ? HeadTileShape{128, 128} : HeadTileShape{64, 256};
}
hipError_t launch_head_gemm(const HeadGemm& g, int tile, hipStream_t st);

}  // namespace capscaps
