// Internal: the matrix products of a linear head over many classes (head_gemm_kernel.h), for head_loss.hip.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/capscaps.h"

namespace capscaps {

constexpr int HEAD_K = 32;        // contracted values of a stage; operands are padded with zeros to a multiple

// Terms of a value of the m side, and the products of terms that a contraction is made of: 1; 2, a 16-bit rounding and that of
// what it leaves over, where the n side has one; 3, fp32 values as bf16 terms on both sides (bf16_split.h)
inline int head_products(int terms) { return terms == 3 ? 6 : terms; }

// An operand in blocks: 16 rows of a stage, 1 KB, in the order in which they lie in LDS, so that one copy of a wave is one
// run of memory.  (Copies of 64 bytes from each of 16 rows make half as wide requests of the L2, of which a CU has only so
// many on their way: a product of 8192 x 2048 x 32768 runs at 700 TFLOP/s so on tiles of 256 x 256, and at 1450 with
// blocks.)
// `stages`: those of a row block, the terms one after another.  Offset of value k of a row, in values:
__host__ __device__ inline long long head_block_at(long long row, long long k, long long stages)
{
    const long long block = (row >> 4) * stages + (k >> 5);
    const int r = (int)(row & 15), chunk = (int)(k >> 3) & 3;
    return block * 512 + r * 32 + ((chunk ^ (r >> 2)) << 3) + (int)(k & 7);
}
inline long long head_block_values(long long rows, long long stages) { return (rows + 15) / 16 * stages * 512; }

// What a product's tiles become
enum HeadEnd {
    HEAD_OUT = 0,       // out[m][n], or a part of it
    HEAD_STATS = 1,     // the largest of a row's logits, and the sum of exp(logit - largest)
    HEAD_GRADIENT = 2,  // coef exp(logit - lse), as operands of the products that follow, and its sums over rows
};

struct HeadStat {
    float top, sum;
};

// z[m][n] = sum over k of a[m][k] * b[n][k], both in blocks; or b as rows (16 bits, whole stages, whole 16-byte vectors).
struct HeadGemm {
    const void *a, *b;
    long long stages_a, stages_b;  // stages of a row block, all terms together; b as rows: 0
    long long ldb;                 // b as rows: bytes from row to row
    long long m_rows, n_rows;
    const int* m_count;        // NULL, or how many of the m rows count, in device memory
    const int* k_count;        // NULL, or how many contracted values count, in device memory
    long long k;
    int plane_a, plane_b;  // stages of a term
    int terms, dtype;      // terms of a; fp32: 3
    // HEAD_OUT: fp32 (out_dtype) or 16 bits; parts of the contracted length go to copies `out_split` elements apart
    void* out;
    long long ldo, out_split;
    int out_dtype, splits;
    bool accumulate;     // add to what is there (fp32, one part)
    bool whole_vectors;  // set by the launcher: rows of out are whole 16-byte vectors, 256 of them within 32 bits
    const float* scale;  // NULL, or what to multiply by, in device memory
    // the others: logit = (z + bias[n]) * inv_tau
    const float* bias;  // or NULL
    float inv_tau;
    HeadStat* stats;  // [n / stat_columns][m_rows]
    const float *coef, *lse;  // of row m, and of row rows_of[m]
    const int* rows_of;
    unsigned short *gn, *gt;  // rows m and rows n, in blocks of planes_n and planes_t stages a term
    int planes_n, planes_t, grad_terms;
    float* sums;  // NULL, or [m / sum_rows][planes_n * HEAD_K]
};

// tile shapes, the columns of a statistic and the rows of a sum over rows (those of a wave), workgroups of a CU
enum HeadTile { HEAD_TILE_256 = 0, HEAD_TILE_128 = 1, HEAD_TILE_FEW_ROWS = 2 };
struct HeadTileShape {
    int m, n, stat_columns, sum_rows, per_cu;
};
inline HeadTileShape head_tile_shape(int tile)
{
    switch (tile) {
        case HEAD_TILE_256: return {256, 256, 128, 128, 1};
        case HEAD_TILE_128: return {128, 128, 64, 64, 2};
        default: return {64, 128, 32, 64, 2};
    }
}
hipError_t launch_head_gemm_256(const HeadGemm& g, HeadEnd end, hipStream_t st);
hipError_t launch_head_gemm_128(const HeadGemm& g, HeadEnd end, hipStream_t st);
hipError_t launch_head_gemm_few_rows(const HeadGemm& g, HeadEnd end, hipStream_t st);
inline hipError_t launch_head_gemm(const HeadGemm& g, int tile, HeadEnd end, hipStream_t st)
{
    return tile == HEAD_TILE_256   ? launch_head_gemm_256(g, end, st)
           : tile == HEAD_TILE_128 ? launch_head_gemm_128(g, end, st)
                                   : launch_head_gemm_few_rows(g, end, st);
}
// Two products on the same tiles (not those of 256 x 256) in one launch, for HEAD_OUT
hipError_t launch_head_gemm_pair_128(const HeadGemm& a, const HeadGemm& b, hipStream_t st);
hipError_t launch_head_gemm_pair_few_rows(const HeadGemm& a, const HeadGemm& b, hipStream_t st);
inline hipError_t launch_head_gemm_pair(const HeadGemm& a, const HeadGemm& b, int tile, hipStream_t st)
{
    return tile == HEAD_TILE_128        ? launch_head_gemm_pair_128(a, b, st)
           : tile == HEAD_TILE_FEW_ROWS ? launch_head_gemm_pair_few_rows(a, b, st)
                                        : hipErrorInvalidValue;
}

}  // namespace capscaps
