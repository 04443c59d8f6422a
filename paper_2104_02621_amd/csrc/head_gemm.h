// Internal: the matrix products of a linear head over many classes (head_gemm_kernel.h), for head_loss.hip.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/capscaps.h"

namespace capscaps {

constexpr int HEAD_K = 32;        // contracted values of a stage; rows are padded with zeros to a multiple
constexpr int HEAD_PRODUCTS = 6;  // fp32 operands: products of their bf16 terms

// What a product's tiles become
enum HeadEnd {
    HEAD_OUT = 0,       // out[m][n], or a part of it
    HEAD_STATS = 1,     // the largest of a row's logits, and the sum of exp(logit - largest)
    HEAD_GRADIENT = 2,  // coef exp(logit - lse), as operands of the products that follow, and its sums over rows
};

struct HeadStat {
    float top, sum;
};

// z[m][n] = sum over k of a[m][k] * b[n][k].  Rows of a and b are whole 16-byte vectors at 16-byte addresses, zeros from the
// contracted length up to a multiple of HEAD_K; fp32 operands lie there as three bf16 terms one after another (`plane` bytes each).
struct HeadGemm {
    const void *a, *b;
    long long lda, ldb;        // bytes from row to row
    long long m_rows, n_rows;  // rows that may be read (beyond them: zeros)
    const int* m_count;        // NULL, or how many of the m rows count, in device memory
    const int* k_count;        // NULL, or how many contracted values count, in device memory
    long long k;
    int plane_a, plane_b;
    int dtype;
    // HEAD_OUT: fp32 (out_dtype) or 16 bits; parts of the contracted length go to copies `out_split` elements apart
    void* out;
    long long ldo, out_split;
    int out_dtype, splits;
    bool accumulate;     // add to what is there (fp32, one part)
    const float* scale;  // NULL, or what to multiply by, in device memory
    // the others: logit = (z + bias[n]) * inv_tau
    const float* bias;  // or NULL
    float inv_tau;
    HeadStat* stats;  // [first_part + n / head_stat_columns(tile)][m_rows]
    int first_part;
    const float *coef, *lse;  // of row m, and of row rows_of[m]
    const int* rows_of;
    unsigned short *gn, *gt;        // [m][terms][ldn] and [n][terms][ldt]
    long long ldn, ldt;
    float* sums;  // NULL, or [m / head_sum_rows(tile)][ldn]
};

// tile shapes, the columns of a statistic and the rows of a sum over rows (those of a wave)
enum HeadTile { HEAD_TILE_256 = 0, HEAD_TILE_HALF = 1, HEAD_TILE_128 = 2, HEAD_TILE_FEW_ROWS = 3 };
struct HeadTileShape {
    int m, n, stat_columns, sum_rows, per_cu;
};
inline HeadTileShape head_tile_shape(int tile)
{
    switch (tile) {
        case HEAD_TILE_256: return {256, 256, 128, 128, 1};
        case HEAD_TILE_HALF: return {128, 256, 128, 64, 2};
        case HEAD_TILE_128: return {128, 128, 64, 64, 2};
        default: return {64, 256, 64, 64, 2};
    }
}
hipError_t launch_head_gemm_256(const HeadGemm& g, HeadEnd end, hipStream_t st);
hipError_t launch_head_gemm_half(const HeadGemm& g, HeadEnd end, hipStream_t st);
hipError_t launch_head_gemm_128(const HeadGemm& g, HeadEnd end, hipStream_t st);
hipError_t launch_head_gemm_few_rows(const HeadGemm& g, HeadEnd end, hipStream_t st);
inline hipError_t launch_head_gemm(const HeadGemm& g, int tile, HeadEnd end, hipStream_t st)
{
    return tile == HEAD_TILE_256    ? launch_head_gemm_256(g, end, st)
           : tile == HEAD_TILE_HALF ? launch_head_gemm_half(g, end, st)
           : tile == HEAD_TILE_128  ? launch_head_gemm_128(g, end, st)
                                    : launch_head_gemm_few_rows(g, end, st);
}

}  // namespace capscaps
