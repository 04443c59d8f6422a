// The losses of a linear head over many classes, forward and backward: softmax cross entropy, and distillation from a
// teacher's top logits.  With x the rows, W the classes' weights and z = x W^T + bias, q = softmax(z / tau),
//
//     loss = tau^2 sum_k t_k (log t_k - log q_k)         g = dloss tau (q - sum_k t_k onehot_k)
//     dx = g W        dW = g^T x        dbias = sum over rows of g
//
// where t are the shares of the row's entries k: one entry with t = 1 for the cross entropy (tau = 1).
//
// z is T x V values, far more than x and W for many classes; it is computed by pieces of the classes, once in each
// direction, and never kept whole.  A piece of g is rounded to the operands' 16 bits (fp32: three bf16 terms) for the
// two products that read it, which takes a relative error of half a step to each term of sums over classes or rows, as
// the storage type of a gradient anywhere else does.  Where rows or classes are few (up to 256) a row of dweight or dx
// hangs on few values of g, whose error would be that row's: g is two terms there, the rounding and that of what it
// leaves over.  One term makes dx and dW some 1.4 times as far off as rounding them alone does; a caller who wants no more than that
// asks for two, whose products are twice as long (8192 rows of 2048 bf16 values, 100003 classes: 8.4 -> 13.9 ms; 509 rows of 1024 fp16
// values, 10007 classes: 88 -> 110 us).  It is scaled so that the largest row's dloss is 2^13 to 2^14: fp16, whose smallest step is 2^-24, then
// holds shares down to 1e-11 of it.
//
// Rows that are left out (no class for a target, no entry) take no part at all: the rows that are kept are counted and gathered on
// the device first, and the products run over these.  So what stands in the others does not matter, and they cost nothing.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "bf16_split.h"
#include "conv_shape.h"
#include "head_gemm.h"
#include "row_vectors.h"

namespace capscaps {
namespace {

constexpr int THREADS = 256;
constexpr int MOST_TOP = 1024;
constexpr int STATS_CHUNK = 16384;  // classes of a row whose statistics a workgroup joins
constexpr int FEW = 256;  // rows or classes whose gradients are two terms of 16 bits
// (256 rows of an operand are within a signed 32-bit offset: rows of up to 2^20 values of three terms)
constexpr long long MOST_ROWS = 1 << 20, MOST_PIECE = 1 << 20;
constexpr long long MOST_TILES = 1 << 23;  // of a launch
// (logits that are written in parts and then read: a row by a workgroup)
constexpr int MOST_IN_PARTS = 16384;
constexpr long long PIECE_BYTES = 1ll << 30;  // of a piece's logits, and of its gradients

// What both directions of both losses are given
struct Head {
    long long rows, classes;
    int width, dtype, top;
    float tau;
    bool wide_index;  // 64-bit indices
    const void *x, *weight;
    long long x_stride, weight_stride;
    const float* bias;
    const void* index;  // [rows][top]
    long long index_stride;
    const void* teacher;  // [rows][top] logits, NULL: cross entropy
    long long teacher_stride;
    int teacher_dtype;
    // in the workspace
    int *keep, *rows_of, *pos, *count, *boundless;  // see rows_kernel
    float *share, *entropy, *coef;
};

__device__ __forceinline__ long long index_of(const Head& H, long long row, int k)
{
    const long long at = row * H.index_stride + k;
    const long long v = H.wide_index ? static_cast<const long long*>(H.index)[at] : static_cast<const int*>(H.index)[at];
    return v >= 0 && v < H.classes ? v : -1;
}
__device__ __forceinline__ float share_of(const Head& H, long long row, int k)
{
    return H.teacher != nullptr ? H.share[row * H.top + k] : 1.0f;
}
__device__ __forceinline__ bool finite(float v) { return __builtin_fabsf(v) < __builtin_inff(); }
__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) v = __builtin_fmaxf(v, __shfl_xor(v, k));
    return v;
}

// share = softmax over the row's entries of the teacher's logits / tau, entropy = sum share log(share), keep: whether there is
// an entry that counts.  A wave for a row.
__global__ void __launch_bounds__(THREADS) teacher_kernel(Head H)
{
    const int lane = threadIdx.x & 63;
    const float inv = 1.0f / H.tau;
    for (long long r = blockIdx.x * 4ll + (threadIdx.x >> 6); r < H.rows; r += gridDim.x * 4ll) {
        float top = -__builtin_inff();
        bool nan = false;
        for (int k = lane; k < H.top; k += 64)
            if (index_of(H, r, k) >= 0) {
                const float l = load_element(H.teacher, r * H.teacher_stride + k, H.teacher_dtype) * inv;
                nan |= l != l;
                top = __builtin_fmaxf(top, l);
            }
        top = wave_max(top);
        nan = __any(nan);
        const bool some = nan || top > -__builtin_inff();
        float s = 0.0f;
        for (int k = lane; k < H.top; k += 64)
            if (some && index_of(H, r, k) >= 0)
                s += expf(load_element(H.teacher, r * H.teacher_stride + k, H.teacher_dtype) * inv - top);
        s = lanes_sum(s, 64);
        const float log_s = logf(s);
        float entropy = 0.0f;
        for (int k = lane; k < H.top; k += 64) {
            float t = 0.0f;
            if (some && index_of(H, r, k) >= 0) {
                const float l = load_element(H.teacher, r * H.teacher_stride + k, H.teacher_dtype) * inv - top;
                t = expf(l) / s;
                if (t != 0.0f) entropy += t * (l - log_s);  // (and where it is NaN)
            }
            H.share[r * H.top + k] = t;
        }
        entropy = lanes_sum(entropy, 64);
        if (lane == 0) {
            H.entropy[r] = entropy;
            H.keep[r] = some ? 1 : 0;
        }
    }
}

// The rows that are kept, in their order: rows_of[i], pos[row] (-1: left out), count[0]; coef[i] = dloss tau times a scale,
// count[1] the bits of one over it; boundless: the i whose coef is infinite or NaN, in any order, count[2] of them.  One workgroup.
__global__ void __launch_bounds__(1024) rows_kernel(Head H, const float* dloss, long long dloss_stride)
{
    __shared__ int sums[16];
    __shared__ float tops[16];
    __shared__ int found;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (threadIdx.x == 0) found = 0;
    auto kept = [&](long long r) {
        return r < H.rows && (H.teacher != nullptr ? H.keep[r] != 0 : index_of(H, r, 0) >= 0);
    };
    float scale = 1.0f;
    if (dloss != nullptr) {
        // (the largest that is finite: a row whose dloss is not says nothing about how the others are rounded)
        float top = 0.0f;
        for (long long r = threadIdx.x; r < H.rows; r += 1024)
            if (kept(r)) {
                const float d = __builtin_fabsf(dloss[r * dloss_stride] * H.tau);
                if (finite(d)) top = __builtin_fmaxf(top, d);
            }
        top = wave_max(top);
        if (lane == 0) tops[wave] = top;
        __syncthreads();
        top = 0.0f;
        for (int k = 0; k < 16; ++k) top = __builtin_fmaxf(top, tops[k]);
        float back = 1.0f;
        if (top >= 1e-33f && H.dtype != CAPSCAPS_FP32) {
            // just below 2^14: the values that weigh most, those of the largest dloss at an entry of a row that has not been
            // learnt, then have the longest mantissas, whose rounding is half that of the shortest
            scale = 16352.0f / top;
            back = top * (1.0f / 16352.0f);
        } else if (top > 0.0f) {
            int e = 127 + 13 - (int)(__builtin_bit_cast(unsigned, top) >> 23);
            e = e > 126 ? 126 : e;
            scale = __builtin_bit_cast(float, (unsigned)(127 + e) << 23);
            back = __builtin_bit_cast(float, (unsigned)(127 - e) << 23);
        }
        if (threadIdx.x == 0) H.count[1] = __builtin_bit_cast(int, back);
    }
    int before = 0;
    for (long long at = 0; at < H.rows; at += 1024) {
        const long long r = at + threadIdx.x;
        const bool mine = kept(r);
        const unsigned long long mask = __builtin_amdgcn_ballot_w64(mine);
        if (lane == 0) sums[wave] = __builtin_popcountll(mask);
        __syncthreads();
        int i = before + __builtin_popcountll(mask & ((1ull << lane) - 1));
        for (int k = 0; k < 16; ++k) {
            if (k < wave) i += sums[k];
            before += sums[k];
        }
        __syncthreads();
        if (r < H.rows) H.pos[r] = mine ? i : -1;
        if (mine) {
            H.rows_of[i] = (int)r;
            if (dloss != nullptr) {
                const float coef = dloss[r * dloss_stride] * H.tau * scale;
                H.coef[i] = coef;
                if (!finite(coef)) H.boundless[atomicAdd(&found, 1)] = i;
            }
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        H.count[0] = before;
        if (dloss != nullptr) H.count[2] = found;
    }
}

// ---------------------------------------------------------------------------------------- operands
// 16 bytes at an element's address
typedef Words<4, 2>::at Vector2;
typedef float4v Vector4 __attribute__((aligned(4)));

// Eight values of a row as a product's operand: one 16-byte vector, or one in each of three terms (`stages` of a term)
template <bool TERMS>
__device__ __forceinline__ void put_operand(unsigned short* to, long long row, long long k, long long stages,
                                            const unsigned short* raw, const float* f)
{
    to += head_block_at(row, k, (TERMS ? 3 : 1) * stages);
    if constexpr (!TERMS) {
        chunk_t c;
        __builtin_memcpy(&c, raw, 16);
        *reinterpret_cast<chunk_t*>(to) = c;
    } else {
        unsigned short t[3][8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float xs = f[j] * SPLIT_SCALE;
            t[0][j] = round_to_16(xs, 1);
            // (what is not finite, or 2^104 and more, makes its sums NaN or infinite)
            const bool out = (t[0][j] & 0x7f80u) == 0x7f80u;
            const float r1 = out ? 0.0f : xs - low_half(t[0][j]);
            t[1][j] = round_to_16(r1, 1);
            t[2][j] = round_to_16(r1 - low_half(t[1][j]), 1);
        }
#pragma unroll
        for (int p = 0; p < 3; ++p) {
            chunk_t c;
            __builtin_memcpy(&c, t[p], 16);
            *reinterpret_cast<chunk_t*>(to + p * stages * 512) = c;
        }
    }
}

// Eight gradients as an operand of `terms` (16 bits: 1 or 2; fp32: 3)
template <bool TERMS>
__device__ __forceinline__ void put_gradients(unsigned short* to, long long row, long long k, long long stages, int terms, int dtype,
                                              const float* f)
{
    unsigned short raw[8];
    if constexpr (TERMS) {
        put_operand<true>(to, row, k, stages, raw, f);
    } else {
        to += head_block_at(row, k, terms * stages);
        float left[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) left[j] = f[j];
        for (int p = 0; p < terms; ++p) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                raw[j] = round_to_16(left[j], dtype == CAPSCAPS_FP16 ? 2 : 1);
                left[j] -= dtype == CAPSCAPS_FP16 ? Element<CAPSCAPS_FP16>::get(raw[j]) : Element<CAPSCAPS_BF16>::get(raw[j]);
            }
            chunk_t c;
            __builtin_memcpy(&c, raw, 16);
            *reinterpret_cast<chunk_t*>(to + p * stages * 512) = c;
        }
    }
}

// Rows of `from` (rows_of[i], those that count) as an operand; zeros past the columns and the rows.  A wave writes a block.
template <bool TERMS>
__global__ void __launch_bounds__(THREADS) pack_kernel(const void* from, long long stride, int columns, long long rows,
                                                       const int* rows_of, const int* count, unsigned short* to,
                                                       long long stages)
{
    const long long kept = count != nullptr ? *count : rows, blocks = (kept + 15) / 16 * stages;
    const int lane = threadIdx.x & 63;
    for (long long b = blockIdx.x * 4ll + (threadIdx.x >> 6); b < blocks; b += gridDim.x * 4ll) {
        const long long rb = b / stages, i = rb * 16 + (lane >> 2);
        const int c = (int)(b - rb * stages) * HEAD_K + ((lane & 3) ^ (lane >> 4)) * 8;
        unsigned short raw[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        float f[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (i < kept) {
            const long long at = (rows_of != nullptr ? rows_of[i] : i) * stride + c;
            if (c + 8 <= columns) {
                if constexpr (TERMS) {
                    const Vector4 *p = reinterpret_cast<const Vector4*>(static_cast<const float*>(from) + at);
                    const float4v u = p[0], v = p[1];
#pragma unroll
                    for (int j = 0; j < 4; ++j) f[j] = u[j], f[4 + j] = v[j];
                } else {
                    const chunk_t u = *reinterpret_cast<const Vector2*>(static_cast<const unsigned short*>(from) + at);
                    __builtin_memcpy(raw, &u, 16);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (c + j < columns) {
                        if constexpr (TERMS)
                            f[j] = static_cast<const float*>(from)[at + j];
                        else
                            raw[j] = static_cast<const unsigned short*>(from)[at + j];
                    }
            }
        }
        put_operand<TERMS>(to, i, c, stages, raw, f);
    }
}

// Columns of `from` as an operand that contracts its rows (rows_of[i], those that count); zeros past them.  And, where
// `straight` is not NULL, what pack_kernel makes of it.  Tiles of 64 x 64.
struct Across {
    const void* from;
    long long stride, rows, stages, straight_stages;
    const int *rows_of, *count;
    unsigned short *to, *straight;
    int columns;
    unsigned blocks;
};
template <bool TERMS>
using AcrossTile = std::conditional_t<TERMS, float, unsigned short>[64][TERMS ? 65 : 66];
template <bool TERMS>
__device__ __forceinline__ void pack_across(const Across& A, unsigned block0, AcrossTile<TERMS>& tile)
{
    typedef std::conditional_t<TERMS, float, unsigned short> E;
    long long kept = A.rows;
    if (A.count != nullptr && *A.count < kept) kept = *A.count;
    const long long used = (kept + HEAD_K - 1) / HEAD_K;  // stages that are read
    const int across = (A.columns + 63) / 64;
    const long long tiles = (used + 1) / 2 * across;
    for (long long b = block0; b < tiles; b += A.blocks) {
        const long long i0 = b / across * 64;
        const int c0 = (int)(b % across) * 64;
        constexpr int PER = 16 / sizeof(E), ROW = 64 / PER;  // values of a vector, vectors of a tile's row
        if (c0 + 64 <= A.columns) {
#pragma unroll
            for (int u = 0; u < 64 * ROW / THREADS; ++u) {
                const int t = u * THREADS + threadIdx.x, i = t / ROW, c = t % ROW * PER;
                chunk_t v = {0, 0, 0, 0};
                if (i0 + i < kept) {
                    const long long row = A.rows_of != nullptr ? A.rows_of[i0 + i] : i0 + i;
                    v = *reinterpret_cast<const typename Words<4, sizeof(E)>::at*>(static_cast<const E*>(A.from) + row * A.stride + c0 + c);
                }
                E e[PER];
                __builtin_memcpy(e, &v, 16);
#pragma unroll
                for (int j = 0; j < PER; ++j) tile[i][c + j] = e[j];
            }
        } else {
#pragma unroll 8
            for (int u = 0; u < 16; ++u) {
                const int t = u * THREADS + threadIdx.x, i = t >> 6, c = t & 63;
                E v = 0;
                if (i0 + i < kept && c0 + c < A.columns) {
                    const long long row = A.rows_of != nullptr ? A.rows_of[i0 + i] : i0 + i;
                    v = static_cast<const E*>(A.from)[row * A.stride + c0 + c];
                }
                tile[i][c] = v;
            }
        }
        __syncthreads();
        for (int t = threadIdx.x; t < 64 * 8; t += THREADS) {
            // (a wave: a block)
            const int block = t >> 6, c = (block >> 1) * 16 + ((t & 63) >> 2);
            const int i = (block & 1) * HEAD_K + ((t & 3) ^ ((t & 63) >> 4)) * 8;
            if (c0 + c < (A.columns + 15) / 16 * 16 && i0 + i < used * HEAD_K) {
                unsigned short raw[8];
                float f[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if constexpr (TERMS)
                        f[j] = tile[i + j][c];
                    else
                        raw[j] = tile[i + j][c];
                }
                put_operand<TERMS>(A.to, c0 + c, i0 + i, A.stages, raw, f);
            }
        }
        if (A.straight != nullptr)
            for (int t = threadIdx.x; t < 64 * 8; t += THREADS) {
                const int block = t >> 6, i = (block >> 1) * 16 + ((t & 63) >> 2);
                const int c = (block & 1) * HEAD_K + ((t & 3) ^ ((t & 63) >> 4)) * 8;
                if (i0 + i < (kept + 15) / 16 * 16 && c0 + c < A.straight_stages * HEAD_K) {
                    unsigned short raw[8];
                    float f[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        if constexpr (TERMS)
                            f[j] = tile[i][c + j];
                        else
                            raw[j] = tile[i][c + j];
                    }
                    put_operand<TERMS>(A.straight, i0 + i, c0 + c, A.straight_stages, raw, f);
                }
            }
        __syncthreads();
    }
}

// Of up to two tensors, each by workgroups of its own (0: none), and zeros to `clear`
template <bool TERMS>
__global__ void __launch_bounds__(THREADS) pack_transposed_kernel(Across a, Across b, long long* clear, long long n)
{
    __shared__ AcrossTile<TERMS> tile;
    const unsigned both = a.blocks + b.blocks;
    if (blockIdx.x < a.blocks)
        pack_across<TERMS>(a, blockIdx.x, tile);
    else if (blockIdx.x < both)
        pack_across<TERMS>(b, blockIdx.x - a.blocks, tile);
    else
        for (long long t = (blockIdx.x - both) * (long long)THREADS + threadIdx.x; t < n; t += (gridDim.x - both) * (long long)THREADS)
            clear[t] = 0;
}

// ---------------------------------------------------------------------------------------- few rows of fp32
// Up to 64 rows of fp32 are multiplied by the fp32 matrix instructions with the weights read once, as they lie: written out as
// three terms and read by six products they would move five times the bytes, and large weights are all that counts here.
// 50000 classes of 4096 values: 1 row 255 us forward and 622 back, by terms 958 and 2948; 40 rows 402 and 951, by terms 996 and 3254.
// (Which heads take these kernels: few_of_fp32.)
constexpr int FEW_FP32 = 64;

__device__ __forceinline__ float4v load_four(const float* p, long long left)
{
    if (left >= 4) return *reinterpret_cast<const Vector4*>(p);
    float4v v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < 3; ++k)
        if (k < left) v[k] = p[k];
    return v;
}

// z[part][row][class] of T tiles of 16 rows.  A wave: 32 classes, which are the instruction's rows; a lane holds four values of the
// contracted width of its class and of its row in each tile, taken up one by one (their order does not matter).
template <int T>
__global__ void __launch_bounds__(THREADS) few_logits_kernel(Head H, float* z, long long ldz, int splits, long long split)
{
    const int lane = threadIdx.x & 63, at = lane & 15, kq = (lane >> 4) * 4;
    const int kept = *H.count, part = blockIdx.x % splits;
    const long long n0 = (long long)(blockIdx.x / splits) * 128 + (threadIdx.x >> 6) * 32;
    const int steps = (H.width + 15) / 16, per = (steps + splits - 1) / splits;
    const int begin = part * per, end = begin + per < steps ? begin + per : steps;
    const float *w[2], *x[T];
    bool has_w[2], has_x[T];
#pragma unroll
    for (int a = 0; a < 2; ++a) {
        const long long n = n0 + a * 16 + at;
        has_w[a] = n < H.classes;
        w[a] = static_cast<const float*>(H.weight) + (has_w[a] ? n : 0) * H.weight_stride + kq;
    }
#pragma unroll
    for (int t = 0; t < T; ++t) {
        has_x[t] = t * 16 + at < kept;
        x[t] = static_cast<const float*>(H.x) + (has_x[t] ? (long long)H.rows_of[t * 16 + at] : 0) * H.x_stride + kq;
    }
    float4v acc[2][T];
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int t = 0; t < T; ++t) acc[a][t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    const float4v none = {0.0f, 0.0f, 0.0f, 0.0f};
    float4v wv[2], xv[T];
    auto load = [&](int step) {
        const int k = step * 16, left = step < end ? H.width - k - kq : 0;
#pragma unroll
        for (int a = 0; a < 2; ++a) wv[a] = has_w[a] ? load_four(w[a] + k, left) : none;
#pragma unroll
        for (int t = 0; t < T; ++t) xv[t] = has_x[t] ? load_four(x[t] + k, left) : none;
    };
    load(begin);
    for (int step = begin; step < end; ++step) {
        float4v wn[2], xn[T];
#pragma unroll
        for (int a = 0; a < 2; ++a) wn[a] = wv[a];
#pragma unroll
        for (int t = 0; t < T; ++t) xn[t] = xv[t];
        load(step + 1);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int t = 0; t < T; ++t) acc[a][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(wn[a][j], xn[t][j], acc[a][t], 0, 0, 0);
    }
#pragma unroll
    for (int a = 0; a < 2; ++a) {
        const long long n = n0 + a * 16 + kq;
#pragma unroll
        for (int t = 0; t < T; ++t)
            if (n < H.classes && t * 16 + at < kept) *reinterpret_cast<float4v*>(z + part * split + (t * 16 + at) * ldz + n) = acc[a][t];
    }
}

// dx[part][row][column] = sum over a part's classes of g[row][class] W[class][column].  A wave: 64 columns, of which a lane loads four
// neighbouring ones of a class at a time; columns 4 i + c are the rows of one instruction.
template <int T>
__global__ void __launch_bounds__(THREADS) few_rows_kernel(Head H, const float* g, long long ldg, float* dx, long long ld, int splits,
                                                           long long split)
{
    const int lane = threadIdx.x & 63, at = lane & 15, kq = (lane >> 4) * 4;
    const int kept = *H.count, part = blockIdx.x % splits;
    const int h0 = (blockIdx.x / splits) * 256 + (threadIdx.x >> 6) * 64, left = H.width - h0 - at * 4;
    const int steps = (int)((H.classes + 15) / 16), per = (steps + splits - 1) / splits;
    const int begin = part * per, end = begin + per < steps ? begin + per : steps;
    float4v acc[4][T];
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int t = 0; t < T; ++t) acc[c][t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    const float4v none = {0.0f, 0.0f, 0.0f, 0.0f};
    const float* const w = static_cast<const float*>(H.weight) + h0 + at * 4;
    float4v wv[4], gv[T];
    auto load = [&](int step) {
        const long long n = step * 16ll + kq;
        const bool some = step < end;
#pragma unroll
        for (int q = 0; q < 4; ++q) wv[q] = some && n + q < H.classes && left > 0 ? load_four(w + (n + q) * H.weight_stride, left) : none;
#pragma unroll
        for (int t = 0; t < T; ++t)
            gv[t] = some && t * 16 + at < kept ? load_four(g + (t * 16 + at) * ldg + n, H.classes - n) : none;
    };
    load(begin);
    for (int step = begin; step < end; ++step) {
        float4v wn[4], gn[T];
#pragma unroll
        for (int q = 0; q < 4; ++q) wn[q] = wv[q];
#pragma unroll
        for (int t = 0; t < T; ++t) gn[t] = gv[t];
        load(step + 1);
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int t = 0; t < T; ++t) acc[c][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(wn[q][c], gn[t][q], acc[c][t], 0, 0, 0);
    }
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int h = h0 + (kq + r) * 4;
            if (t * 16 + at < kept && h < H.width)  // (rows of dx are whole vectors)
                *reinterpret_cast<float4v*>(dx + part * split + (t * 16 + at) * ld + h) =
                    float4v{acc[0][t][r], acc[1][t][r], acc[2][t][r], acc[3][t][r]};
        }
}

// ---------------------------------------------------------------------------------------- forward
typedef HeadStat Stat;
__device__ __forceinline__ Stat join(const Stat& a, const Stat& b)
{
    const float top = __builtin_fmaxf(a.top, b.top);
    // (nothing but -infinity so far: no sum)
    const float fa = a.top == top ? 1.0f : __expf(a.top - top), fb = b.top == top ? 1.0f : __expf(b.top - top);
    return {top, (a.sum > 0.0f || a.sum != a.sum ? a.sum * fa : 0.0f) + (b.sum > 0.0f || b.sum != b.sum ? b.sum * fb : 0.0f)};
}
__device__ __forceinline__ Stat wave_join(Stat s)
{
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) s = join(s, {__shfl_xor(s.top, k), __shfl_xor(s.sum, k)});
    return s;
}

// The sum of what lies at `from` in each of `splits` parts, four on their way at a time
template <typename V>
__device__ __forceinline__ V sum_of_parts(const float* from, long long split, int splits)
{
    V sum = {};
    int p = 0;
    for (; p + 4 <= splits; p += 4) {
        V v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = *reinterpret_cast<const V*>(from + (p + q) * split);
        __builtin_amdgcn_sched_barrier(0);  // (the compiler would wait for each before it asks for the next)
#pragma unroll
        for (int q = 0; q < 4; ++q) sum += v[q];
    }
    for (; p < splits; ++p) sum += *reinterpret_cast<const V*>(from + p * split);
    return sum;
}

// stats[chunk][i] of logits that lie in parts.  A workgroup for STATS_CHUNK classes of a row.
__global__ void __launch_bounds__(THREADS) stats_kernel(Head H, const float* z, long long ldz, int splits, long long split,
                                                        Stat* stats)
{
    __shared__ Stat joined[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const float inv = 1.0f / H.tau;
    const long long kept = *H.count;
    const int chunks = (int)((H.classes + STATS_CHUNK - 1) / STATS_CHUNK);
    for (long long t = blockIdx.x; t < kept * chunks; t += gridDim.x) {
        const long long i = t / chunks, first = t % chunks * STATS_CHUNK;
        const long long end = first + STATS_CHUNK < H.classes ? first + STATS_CHUNK : H.classes;
        Stat s = {-__builtin_inff(), 0.0f};
        for (long long c = first + threadIdx.x; c < end; c += THREADS) {
            float v = sum_of_parts<float>(z + i * ldz + c, split, splits);
            if (H.bias != nullptr) v += H.bias[c];
            v *= inv;
            if (v != v)
                s.sum = v;
            else if (v > -__builtin_inff())
                s = join(s, {v, 1.0f});
        }
        s = wave_join(s);
        if (lane == 0) joined[wave] = s;
        __syncthreads();
        if (threadIdx.x == 0) stats[t % chunks * H.rows + i] = join(join(joined[0], joined[1]), join(joined[2], joined[3]));
        __syncthreads();
    }
}

// z of entries k0 to k0 + 3 of row r (0 where they do not count), from the operands in fp32: to picked[r][k].  By a wave, or where there are
// few by a workgroup (LANES); what it waits for is the weights' rows, which lie anywhere.
template <int LANES>
__device__ __forceinline__ void pick_entries(const Head& H, long long r, int k0, float* picked, float (*parts)[4])
{
    const int lane = threadIdx.x & (LANES - 1);
    long long cls[4];
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < 4; ++j) cls[j] = k0 + j < H.top ? index_of(H, r, k0 + j) : -1;
    const long long xa = r * H.x_stride;
    if (H.dtype != CAPSCAPS_FP32) {
        const unsigned short *x = static_cast<const unsigned short*>(H.x) + xa, *w = static_cast<const unsigned short*>(H.weight);
#pragma unroll 2
        for (int c = lane * 8; c + 8 <= H.width; c += LANES * 8) {
            const chunk_t a = *reinterpret_cast<const Vector2*>(x + c);
            chunk_t b[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (cls[j] >= 0) b[j] = *reinterpret_cast<const Vector2*>(w + cls[j] * H.weight_stride + c);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (cls[j] >= 0)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        if (H.dtype == CAPSCAPS_BF16) {
                            s[j] = __builtin_fmaf(low_half(a[q]), low_half(b[j][q]), s[j]);
                            s[j] = __builtin_fmaf(high_half(a[q]), high_half(b[j][q]), s[j]);
                        } else {
                            const half2v u = __builtin_bit_cast(half2v, (unsigned)a[q]), v = __builtin_bit_cast(half2v, (unsigned)b[j][q]);
                            s[j] = __builtin_fmaf((float)u[0], (float)v[0], s[j]);
                            s[j] = __builtin_fmaf((float)u[1], (float)v[1], s[j]);
                        }
                    }
        }
    }
    for (int c = (H.dtype != CAPSCAPS_FP32 ? H.width & ~7 : 0) + lane; c < H.width; c += LANES) {  // (16 bits: the rest)
        const float a = load_element(H.x, xa + c, H.dtype);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (cls[j] >= 0) s[j] = __builtin_fmaf(a, load_element(H.weight, cls[j] * H.weight_stride + c, H.dtype), s[j]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        s[j] = lanes_sum(s[j], 64);
        if constexpr (LANES > 64) {
            if ((lane & 63) == 0) parts[lane >> 6][j] = s[j];
            __syncthreads();
            s[j] = (parts[0][j] + parts[1][j]) + (parts[2][j] + parts[3][j]);
        }
        if (cls[j] >= 0 && H.bias != nullptr) s[j] += H.bias[cls[j]];
        if (lane == 0 && k0 + j < H.top) picked[r * H.top + k0 + j] = s[j];
    }
}

// ... of all rows that are kept (3686 rows of 64 entries, 2048 bf16 values wide: 138 us, 7 TB/s of rows of the weights out of the caches)
template <bool WIDE>
__global__ void __launch_bounds__(THREADS) pick_kernel(Head H, float* picked)
{
    constexpr int LANES = WIDE ? THREADS : 64, PER = THREADS / LANES;
    __shared__ float parts[4][4];
    const long long kept = *H.count, quads = (H.top + 3) / 4;
    for (long long t = blockIdx.x * (long long)PER + threadIdx.x / LANES; t < kept * quads; t += gridDim.x * (long long)PER) {
        pick_entries<LANES>(H, H.rows_of[t / quads], (int)(t % quads) * 4, picked, parts);
        if constexpr (WIDE) __syncthreads();
    }
}

// The parts of the statistics of ROWS rows from i0 on (lane & (ROWS - 1) is a lane's), joined by a workgroup: to joined[row] for
// the first ROWS threads, after the barrier that ends this
template <int ROWS>
__device__ __forceinline__ Stat join_parts(const Stat* stats, long long stride, int parts, long long i0, int rows, Stat (*waves)[ROWS])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Stat s = {-__builtin_inff(), 0.0f};
    if ((lane & (ROWS - 1)) < rows)
        for (int p = threadIdx.x / ROWS; p < parts; p += THREADS / ROWS) s = join(s, stats[p * stride + i0 + (lane & (ROWS - 1))]);
#pragma unroll
    for (int k = ROWS; k < 64; k <<= 1) s = join(s, {__shfl_xor(s.top, k), __shfl_xor(s.sum, k)});
    if (lane < ROWS) waves[wave][lane] = s;
    __syncthreads();
    if (threadIdx.x < ROWS) s = join(join(waves[0][lane], waves[1][lane]), join(waves[2][lane], waves[3][lane]));
    return s;
}

// A piece's parts, and what the pieces before it left in part 0 (`more`), joined into part 0
template <int ROWS>
__global__ void __launch_bounds__(THREADS) fold_kernel(Head H, Stat* stats, int parts, bool more)
{
    __shared__ Stat waves[4][ROWS];
    const int kept = *H.count;
    for (long long i0 = blockIdx.x * (long long)ROWS; i0 < kept; i0 += gridDim.x * (long long)ROWS) {
        const int rows = kept - i0 < ROWS ? (int)(kept - i0) : ROWS;
        Stat s = join_parts<ROWS>(stats + H.rows, H.rows, parts, i0, rows, waves);
        if (threadIdx.x < rows) {
            if (more) s = join(stats[i0 + threadIdx.x], s);
            stats[i0 + threadIdx.x] = s;
        }
        __syncthreads();
    }
}

// loss, lse, logq of all rows, from stats[part][i] and the entries' z: picked[r][k], which logq takes the place of where it is wanted;
// computed here, of rows with four entries at most, which spares a launch; or of logits that lie in parts.
// A workgroup for ROWS of the rows that are kept, and for the zeros of as many that are not (eight: whole 64-byte pieces of a
// part's statistics; one where rows are few).
enum Entries { PICKED, PICK, PARTS };
struct Parts {
    const float* z;
    long long ld, split;
    int splits;
};
template <int ROWS, int ENTRIES>
__global__ void __launch_bounds__(THREADS) loss_kernel(Head H, const Stat* stats, int parts, float* picked, Parts logits, float* loss,
                                                       float* lse, float* logq)
{
    static_assert(ROWS == 1 || ENTRIES != PICK);
    __shared__ Stat joined[4][ROWS];
    __shared__ float lses[ROWS], sums[4][ROWS], products[4][4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const float inv = 1.0f / H.tau;
    const int kept = *H.count;
    for (long long i0 = blockIdx.x * (long long)ROWS; i0 < H.rows; i0 += gridDim.x * (long long)ROWS) {
        for (int t = threadIdx.x; t < ROWS * H.top; t += THREADS) {
            const long long r = i0 + t / H.top;
            if (r < H.rows && H.pos[r] < 0) {
                if (t % H.top == 0) loss[r] = 0.0f, lse[r] = 0.0f;
                if (logq != nullptr) logq[r * H.top + t % H.top] = 0.0f;
            }
        }
        if (i0 >= kept) continue;
        const int rows = kept - i0 < ROWS ? (int)(kept - i0) : ROWS;
        if constexpr (ENTRIES == PICK) pick_entries<THREADS>(H, H.rows_of[i0], 0, picked, products);
        const Stat s = join_parts<ROWS>(stats, H.rows, parts, i0, rows, joined);
        if (threadIdx.x < ROWS) {
            lses[lane] = s.top + logf(s.sum);
        }
        __syncthreads();
        // (lane's row and every 256 / ROWS-th entry)
        float cross = 0.0f;
        if ((lane & (ROWS - 1)) < rows) {
            const long long r = H.rows_of[i0 + (lane & (ROWS - 1))];
            for (int k = threadIdx.x / ROWS; k < H.top; k += THREADS / ROWS) {
                float l = 0.0f;
                const long long cls = index_of(H, r, k);
                if (cls >= 0) {
                    float z = 0.0f;
                    if constexpr (ENTRIES == PARTS) {
                        z = sum_of_parts<float>(logits.z + (i0 + (lane & (ROWS - 1))) * logits.ld + cls, logits.split, logits.splits);
                        if (H.bias != nullptr) z += H.bias[cls];
                    } else {
                        z = picked[r * H.top + k];
                    }
                    // (no class is more likely than certain; z and lse come from sums of their own, and the difference of their roundings
                    // may say so of a class that the row has learnt)
                    l = z * inv - lses[lane & (ROWS - 1)];
                    l = l > 0.0f ? 0.0f : l;
                    const float t = share_of(H, r, k);
                    if (t != 0.0f) cross += t * l;
                }
                if (logq != nullptr) logq[r * H.top + k] = l;
            }
        }
#pragma unroll
        for (int k = ROWS; k < 64; k <<= 1) cross += __shfl_xor(cross, k);
        if (lane < ROWS) sums[wave][lane] = cross;
        __syncthreads();
        if (threadIdx.x < rows) {
            const long long r = H.rows_of[i0 + lane];
            const float entropy = H.teacher != nullptr ? H.entropy[r] : 0.0f;
            loss[r] = H.tau * H.tau * (entropy - ((sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane])));
            lse[r] = lses[lane];
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------------------- backward
// A piece's gradients without the entries' shares: g = coef exp(z - lse), as operands, rows innermost (gt) and classes
// innermost (gn), and their sums over 64 rows but the boundless ones (sums[row tile][class], for the bias).  Tiles of 64 x 64.
template <bool TERMS>
__global__ void __launch_bounds__(THREADS) gradient_kernel(Head H, const float* lse, const float* z, long long ldz, int splits,
                                                           long long split, long long first, int classes, unsigned short* gn,
                                                           int padded_classes, unsigned short* gt, long long padded_rows,
                                                           int terms, float* sums, float* raw)
{
    __shared__ float tile[64][65], part[4][64];
    const float inv = 1.0f / H.tau;
    const long long kept = *H.count;
    const bool boundless = H.count[2] > 0;
    const int across = (padded_classes + 63) / 64;
    const long long tiles = (padded_rows + 63) / 64 * across;
    for (long long b = blockIdx.x; b < tiles; b += gridDim.x) {
        const long long i0 = b / across * 64;
        const int c0 = (int)(b % across) * 64;
        if (i0 >= (kept + HEAD_K - 1) / HEAD_K * HEAD_K) continue;
        // (four columns a thread, of four rows, a part of all at a time: what it waits for is their loads)
        const int c = c0 + (threadIdx.x & 15) * 4;
        float4v v[4];
        float all[4], coef[4];
        bool mine[4];
        const float* from[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const long long i = i0 + u * 16 + (threadIdx.x >> 4);
            mine[u] = i < kept && c < classes;
            v[u] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
            from[u] = z + (mine[u] ? i : i0) * ldz + (mine[u] ? c : 0);  // (rows are a multiple of 32 long)
            all[u] = lse[H.rows_of[mine[u] ? i : 0]], coef[u] = H.coef[mine[u] ? i : 0];
        }
        auto add = [&](int p, auto COUNT) {
            constexpr int N = decltype(COUNT)::value;
            float4v more[N][4];
#pragma unroll
            for (int q = 0; q < N; ++q)
#pragma unroll
                for (int u = 0; u < 4; ++u) more[q][u] = *reinterpret_cast<const float4v*>(from[u] + (p + q) * split);
            __builtin_amdgcn_sched_barrier(0);  // (all on their way before the first is waited for)
#pragma unroll
            for (int q = 0; q < N; ++q)
#pragma unroll
                for (int u = 0; u < 4; ++u) v[u] += more[q][u];
        };
        int p = 0;
        for (; p + 4 <= splits; p += 4) add(p, std::integral_constant<int, 4>());
        for (; p < splits; ++p) add(p, std::integral_constant<int, 1>());
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool in = c + j < classes;
            const float b = H.bias != nullptr && in ? H.bias[first + c + j] : 0.0f;
#pragma unroll
            for (int u = 0; u < 4; ++u)
                tile[u * 16 + (threadIdx.x >> 4)][(threadIdx.x & 15) * 4 + j] =
                    mine[u] && in ? coef[u] * expf(__builtin_fmaf(v[u][j] + b, inv, -all[u])) : 0.0f;
        }
        if (raw != nullptr)  // (where the first part's logits were, which only this thread reads)
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (mine[u]) {
                    const float* const g = tile[u * 16 + (threadIdx.x >> 4)] + (threadIdx.x & 15) * 4;
                    *reinterpret_cast<float4v*>(raw + (from[u] - z)) = float4v{g[0], g[1], g[2], g[3]};
                }
        __syncthreads();
        for (int t = threadIdx.x; t < 2 * 64 * 8; t += THREADS) {
            const bool across_rows = t >= 64 * 8;
            const int a = (t & 511) >> 3, k = (t & 7) * 8;
            float f[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = across_rows ? tile[k + j][a] : tile[a][k + j];
            if (across_rows) {
                if (c0 + a < classes && i0 + k < padded_rows)
                    put_gradients<TERMS>(gt, c0 + a, i0 + k, padded_rows / HEAD_K, terms, H.dtype, f);
            } else if (i0 + a < kept && c0 + k < padded_classes) {
                put_gradients<TERMS>(gn, i0 + a, c0 + k, padded_classes / HEAD_K, terms, H.dtype, f);
            }
        }
        if (sums != nullptr) {  // (a wave for sixteen rows)
            const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const long long row = i0 + wave * 16 + i;
                if (!boundless || row >= kept || finite(H.coef[row])) s += tile[wave * 16 + i][lane];
            }
            part[wave][lane] = s;
            __syncthreads();
            if (wave == 0 && c0 + lane < classes)
                sums[b / across * padded_classes + c0 + lane] = (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]);
        }
        __syncthreads();
    }
}

// ... with them: g = coef (exp(logq) - share) at the rows' entries in the piece.  An index that comes twice is one
// entry with both shares, written by the first.  `taken`: sums of coef share over rows for each class, as whole numbers of
// 2^-24 (their order does not matter then), those of boundless rows left out; where a share is NaN the class's sum over the first rows
// is made NaN instead.  A wave for a row; 4 us for few rows (a launch's time), 35 to 39 for 3686 rows of 64 entries.
template <bool TERMS>
__global__ void __launch_bounds__(THREADS) entries_kernel(Head H, const float* loss, const float* logq, long long first,
                                                          int classes, unsigned short* gn, int padded_classes,
                                                          unsigned short* gt, long long padded_rows, int terms, long long* taken,
                                                          float* sums, float* raw, long long ldr)
{
    const int lane = threadIdx.x & 63;
    const long long kept = *H.count;
    for (long long i = blockIdx.x * 4ll + (threadIdx.x >> 6); i < kept; i += gridDim.x * 4ll) {
        const long long r = H.rows_of[i];
        for (int k = lane; k < H.top; k += 64) {
            const long long cls = index_of(H, r, k), c = cls - first;
            if (cls < 0 || c < 0 || c >= classes) continue;
            float t = share_of(H, r, k);
            bool again = false;
            for (int j = 0; j < H.top && !again; ++j) {
                if (j == k || index_of(H, r, j) != cls) continue;
                if (j < k)
                    again = true;
                else
                    t += share_of(H, r, j);
            }
            if (again) continue;
            const float q = expf(logq != nullptr ? logq[r * H.top + k] : -loss[r]);
            const float g = H.coef[i] * (q - t);
            if (raw != nullptr) raw[i * ldr + c] = g;
            unsigned short v[3];
            if constexpr (TERMS) {
                const float xs = g * SPLIT_SCALE;
                v[0] = round_to_16(xs, 1);
                const float r1 = (v[0] & 0x7f80u) == 0x7f80u ? 0.0f : xs - low_half(v[0]);
                v[1] = round_to_16(r1, 1);
                v[2] = round_to_16(r1 - low_half(v[1]), 1);
            } else {
                v[0] = round_to_16(g, H.dtype == CAPSCAPS_FP16 ? 2 : 1);
                v[1] = round_to_16(g - (H.dtype == CAPSCAPS_FP16 ? Element<CAPSCAPS_FP16>::get(v[0]) : Element<CAPSCAPS_BF16>::get(v[0])),
                                   H.dtype == CAPSCAPS_FP16 ? 2 : 1);
            }
#pragma unroll
            for (int p = 0; p < (TERMS ? 3 : 2); ++p) {
                if (p >= terms) break;
                gn[head_block_at(i, c, terms * (padded_classes / HEAD_K)) + p * (padded_classes / HEAD_K) * 512ll] = v[p];
                gt[head_block_at(c, i, terms * (padded_rows / HEAD_K)) + p * (padded_rows / HEAD_K) * 512] = v[p];
            }
            if (taken != nullptr && finite(H.coef[i])) {
                if (t != t) {
                    sums[c] = t;
                } else {
                    const long long whole = (long long)__builtin_rintf(H.coef[i] * t * 0x1p24f);
                    atomicAdd(reinterpret_cast<unsigned long long*>(taken + cls), (unsigned long long)whole);
                }
            }
        }
    }
}

// dbias of a piece: the sums over rows less the shares, and the boundless rows' gradients (infinite or NaN all of them) from the
// operand that contracts rows, where they are whole
struct Bias {
    const float* sums;
    const long long* taken;
    const int* boundless;
    const unsigned short* gt;
    long long stages;  // of gt, all terms
    float* dbias;
    long long first;
    int padded_classes, tile_rows, classes;
    unsigned blocks;
};
__device__ __forceinline__ void bias_of(const Bias& B, const int* count, int dtype, unsigned block)
{
    const int c = block * THREADS + threadIdx.x;
    if (c >= B.classes) return;
    const long long tiles = (*count + B.tile_rows - 1) / B.tile_rows;
    double s = 0.0;
    long long t = 0;
    for (; t + 8 <= tiles; t += 8) {
        float v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = B.sums[(t + q) * B.padded_classes + c];
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int q = 0; q < 8; ++q) s += v[q];
    }
    for (; t < tiles; ++t) s += B.sums[t * B.padded_classes + c];
    s -= (double)B.taken[B.first + c] * 0x1p-24;
    for (int k = 0; k < count[2]; ++k) {
        const unsigned short g = B.gt[head_block_at(c, B.boundless[k], B.stages)];
        s += dtype == CAPSCAPS_FP16 ? Element<CAPSCAPS_FP16>::get(g) : Element<CAPSCAPS_BF16>::get(g);
    }
    B.dbias[B.first + c] = (float)(s * __builtin_bit_cast(float, count[1]));
}

// out[r][c] = one over the scale times the sum of `splits` parts of sums[pos[r]][c] (pos NULL: r), 0 where a row is left out
struct Finish {
    const int* pos;
    const float* sums;
    long long ld, split, rows;
    int splits, columns;
    void* out;
    unsigned blocks;
};
__device__ __forceinline__ void finish(const Finish& F, const int* count, int dtype, unsigned block)
{
    const float scale = __builtin_bit_cast(float, count[1]);
    const int vecs = (F.columns + 3) / 4;
    const long long all = F.rows * vecs;
    const bool none = *count == 0;  // (nothing was added up then)
    for (long long t = block * (long long)THREADS + threadIdx.x; t < all; t += (long long)F.blocks * THREADS) {
        const long long r = t / vecs;
        const int c = (int)(t - r * vecs) * 4;
        const long long i = F.pos != nullptr ? F.pos[r] : r;
        float4v v = {0, 0, 0, 0};
        if (i >= 0 && !none) {
            v = sum_of_parts<float4v>(F.sums + i * F.ld + c, F.split, F.splits);
            v *= scale;
        }
        const long long at = r * F.columns + c;
        if ((F.columns & 3) == 0 && dtype == CAPSCAPS_FP32) {
            typedef float at4 __attribute__((ext_vector_type(4), aligned(4)));
            *reinterpret_cast<at4*>(static_cast<float*>(F.out) + at) = v;
        } else if ((F.columns & 3) == 0) {
            typedef unsigned u2 __attribute__((ext_vector_type(2)));
            typedef u2 at2 __attribute__((aligned(2)));
            const int kind = dtype == CAPSCAPS_FP16 ? 2 : 1;
            const u2 w = {round_to_16(v[0], kind) | (unsigned)round_to_16(v[1], kind) << 16,
                          round_to_16(v[2], kind) | (unsigned)round_to_16(v[3], kind) << 16};
            *reinterpret_cast<at2*>(static_cast<unsigned short*>(F.out) + at) = w;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c + j < F.columns) store_element(F.out, at + j, v[j], dtype);
        }
    }
}

// Gradients from their sums: of up to two tensors and the bias, each by workgroups of its own (0: none)
__global__ void __launch_bounds__(THREADS) finish_kernel(const int* count, Finish a, Finish b, Bias c, int dtype)
{
    if (blockIdx.x < a.blocks)
        finish(a, count, dtype, blockIdx.x);
    else if (blockIdx.x < a.blocks + b.blocks)
        finish(b, count, dtype, blockIdx.x - a.blocks);
    else
        bias_of(c, count, dtype, blockIdx.x - a.blocks - b.blocks);
}

// ---------------------------------------------------------------------------------------- host
long long round_up(long long v, long long to) { return (v + to - 1) / to * to; }
int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }
unsigned blocks_for(long long work, long long per) { return (unsigned)std::max<long long>(1, std::min<long long>((work + per - 1) / per, 1 << 20)); }

// Tile and parts of a product: the least of an estimate in units of a 256 x 256 tile's stage on a CU (1024 matrix
// cycles, 0.7 us at the clock that large products run at).  A tile begins and ends in the time of some stages; parts are written and added up at memory speed.
struct Pick {
    int tile, splits;
};
struct Product {
    long long m, n, k;
    int terms;
    bool may_split;
    double part_us;  // what parts cost besides their bytes
    long long stages() const { return std::max<long long>(1, (k + HEAD_K - 1) / HEAD_K) * head_products(terms); }
};
// A product on these tiles in `parts`: rounds' worth of workgroups, units that one takes, and that joining the parts takes
struct Estimate {
    bool can;
    double load, tile, join;
};
Estimate estimate(const Product& P, int tile, int parts)
{
    const HeadTileShape s = head_tile_shape(tile);
    const double tiles = (double)((P.m + s.m - 1) / s.m) * (double)((P.n + s.n - 1) / s.n);
    // time of a stage of as many tiles as a CU holds, and stages' time to begin and end
    const double cost = tile == HEAD_TILE_256 ? 1.0 : tile == HEAD_TILE_128 ? 0.75 : 0.5;
    const double ends = tile == HEAD_TILE_256 ? 24 : 8;
    Estimate E{};
    E.can = tiles * parts <= MOST_TILES && (parts == 1 || (P.may_split && P.stages() / parts >= 8));
    E.load = tiles * parts / (256.0 * s.per_cu);
    E.tile = ((double)((P.stages() + parts - 1) / parts) + ends) * cost;
    E.join = parts > 1 ? ((double)P.m * P.n * 8 * parts / 4e6 + P.part_us) / 0.7 : 0.0;
    return E;
}
double rounds_of(double load) { return load <= 4 ? std::max(1.0, (double)(long long)(load + 0.999)) : load; }
int more_parts(int parts) { return parts < 4 ? parts + 1 : parts * 2; }

Pick pick_tile(const Product& P, double* units = nullptr)
{
    Pick best{HEAD_TILE_128, 1};
    double least = 1e300;
    for (const int tile : {HEAD_TILE_256, HEAD_TILE_128, HEAD_TILE_FEW_ROWS})
        for (int parts = 1; parts <= 64; parts = more_parts(parts)) {
            const Estimate E = estimate(P, tile, parts);
            if (!E.can) continue;
            const double t = rounds_of(E.load) * E.tile + E.join;
            if (t < least) least = t, best = {tile, parts};
        }
    if (units != nullptr) *units += least;
    return best;
}

// ... of two products in one launch, whose workgroups share the CUs
struct Two {
    Pick a, b;
};
Two pick_two(const Product& A, const Product& B, double* units)
{
    Two best{{HEAD_TILE_128, 1}, {HEAD_TILE_128, 1}};
    double least = 1e300;
    for (const int tile : {HEAD_TILE_128, HEAD_TILE_FEW_ROWS})
        for (int pa = 1; pa <= 16; pa = more_parts(pa))
            for (int pb = 1; pb <= 16; pb = more_parts(pb)) {
                const Estimate a = estimate(A, tile, pa), b = estimate(B, tile, pb);
                if (!a.can || !b.can) continue;
                const double load = a.load + b.load;
                const double t = rounds_of(load) * (a.load * a.tile + b.load * b.tile) / load;
                const double all = std::max(t, std::max(a.tile, b.tile)) + a.join + b.join;
                if (all < least) least = all, best = {{tile, pa}, {tile, pb}};
            }
    *units = least;
    return best;
}

int check_head(const capscaps_head* h, bool distill)
{
    if (h == nullptr || h->rows < 0 || h->rows > MOST_ROWS || h->width < 1 || h->classes < 1) return CAPSCAPS_EINVAL;
    if (h->width > (1 << 20) || h->classes > (1 << 26) || !known_dtype(h->dtype)) return CAPSCAPS_EINVAL;
    if (h->index_bits != 32 && h->index_bits != 64) return CAPSCAPS_EINVAL;
    if (h->top < 1 || h->top > MOST_TOP) return CAPSCAPS_EINVAL;
    if (!(h->temperature >= 1e-6f && h->temperature <= 1e6f)) return CAPSCAPS_EINVAL;
    if (h->gradient_terms < 0 || h->gradient_terms > 2) return CAPSCAPS_EINVAL;
    if (distill ? !known_dtype(h->teacher_dtype) : h->top != 1 || h->temperature != 1.0f) return CAPSCAPS_EINVAL;
    return CAPSCAPS_OK;
}

// Whether up to 64 rows of fp32 are multiplied as they lie (few_logits_kernel, few_rows_kernel).  Backward that pays from 16 MB of weights
// on for each of up to three tiles of 16 rows.  Times by terms and so, us: 1 row, 6.1 MB (12000 classes of 128 values) 53 and 51, 16.1 (6000 of
// 672) 75 and 69, 32.3 (12000 of 672) 101 and 78; 40 rows, 4.8 MB (444 of 2680) 55 and 99, 32.3 MB 110 and 112, 53.8 MB (20000 of 672) 154 and 131; 64
// rows, 1.2 MB (444 of 672) 44 and 110, 32.3 MB 116 and 123, 53.8 MB 156 and 147.  Forward the logits' own way to memory and back counts,
// where the other path keeps them in registers (past 16384 classes) or the rows are short: 1 row, 20000 classes of 64 values 29 and 41, of 672 (53.8 MB)
// 63 and 69, 40000 of 400 (64 MB) 76 and 56; 16000 of 128 values 31 and 40, of 256 61 and 47; 40 rows 33 and 47, 63 and 55, 40000 of
// 400 77 and 78; 1216 classes of 64 values 29 and 26, of 4096 52 and 36.
bool few_of_fp32(const capscaps_head& A, bool backward)
{
    if (A.dtype != CAPSCAPS_FP32 || A.rows > FEW_FP32 || A.classes > MOST_PIECE || A.classes > (1ll << 38) / A.width) return false;
    const long long bytes = 4ll * A.classes * A.width;
    if (backward) return bytes >= 16000000ll * std::min(3, std::max(1, ceil_div(A.rows, 16)));
    if (A.classes <= MOST_IN_PARTS) return A.classes <= 4096 || A.width >= 256;
    return bytes >= 60000000;
}

// The workspace, piece by piece
struct Layout {
    char* base;
    size_t at = 0;
    template <typename T>
    T* take(long long n)
    {
        T* p = reinterpret_cast<T*>(base + at);
        at = (at + (size_t)std::max<long long>(n, 1) * sizeof(T) + 255) / 256 * 256;
        return p;
    }
};

struct Plan {
    int terms, padded;  // terms of an operand's value, contracted width
    int grad_terms;     // ... of a gradient
    bool in_parts;      // logits in parts: few enough to lie in memory
    bool few;           // few rows of fp32
    long long piece;    // classes of a piece
    int pieces, stat_parts;
    long long padded_rows;
    Pick z, dx, dw;
    bool pair;  // dx and dweight in one launch
    bool distill, backward;
    size_t bytes;
    // the workspace
    unsigned short *x, *xt, *w, *wt, *gn, *gt;
    float *logits, *dx_sums, *dw_sums, *bias_sums;
    Stat* stats;  // [part][rows]; several pieces: part 0 of all, the others of a piece
    float* picked;
    long long* taken;
};

bool vectors_of(const void* p, long long stride, int dtype)
{
    const int per = dtype == CAPSCAPS_FP32 ? 4 : 8;
    return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && stride % per == 0;
}

// (sizes and addresses in one; the addresses mean nothing where `base` is NULL, and the sizes do not depend on the operands' places)
Plan make_plan(const capscaps_head& A, bool distill, bool backward, void* base, Head* H)
{
    Plan P{};
    P.distill = distill, P.backward = backward;
    P.terms = A.dtype == CAPSCAPS_FP32 ? 3 : 1;
    P.grad_terms = P.terms == 3 ? 3 : A.gradient_terms > 0 ? A.gradient_terms : A.rows <= FEW || A.classes <= FEW ? 2 : 1;
    P.padded = (int)round_up(A.width, HEAD_K);
    P.padded_rows = round_up(std::max<long long>(A.rows, 1), HEAD_K);
    const long long rows = std::max<long long>(A.rows, 1);
    // a piece's weights as operands, and its gradients
    const long long per_class = 2ll * std::max<long long>(P.terms * P.padded, backward ? P.grad_terms * rows : 0);
    P.piece = std::max<long long>(256, std::min(MOST_PIECE, PIECE_BYTES / per_class / 256 * 256));
    P.piece = std::min(P.piece, MOST_TILES / ((rows + 255) / 256) * 256);  // (a launch of tiles of 256 x 256)
    P.piece = std::min<long long>(round_up(A.classes, HEAD_K), P.piece);
    // (a piece's statistics: 8 bytes for as few as 32 classes of a row)
    if (!backward) P.piece = std::min(P.piece, std::max<long long>(256, PIECE_BYTES / 8 / rows * 32 / 256 * 256));
    P.few = few_of_fp32(A, backward);
    if (P.few) P.piece = round_up(A.classes, HEAD_K);
    P.pieces = (int)((A.classes + P.piece - 1) / P.piece);
    const long long most = std::min<long long>(P.piece, A.classes);
    P.z = pick_tile({rows, most, A.width, P.terms, P.pieces == 1 && A.classes <= MOST_IN_PARTS && rows * P.piece * 64 * 4 <= PIECE_BYTES, 6.0});
    // (of few rows: four to eight workgroups on a CU, parts of at least 256 values)
    if (P.few) P.z.splits = (int)std::min<long long>(std::max(1, A.width / 256), std::max<long long>(1, 2048 / ceil_div(A.classes, 128)));
    P.in_parts = P.few || P.z.splits > 1;
    P.stat_parts = P.in_parts ? ceil_div(most, STATS_CHUNK) : ceil_div(most, head_tile_shape(P.z.tile).stat_columns);  // of a piece
    Layout L{static_cast<char*>(base)};
    Head unused;
    Head& W = H != nullptr ? *H : unused;
    W.count = L.take<int>(3);
    W.rows_of = L.take<int>(A.rows);
    W.pos = L.take<int>(A.rows);
    W.keep = distill ? L.take<int>(A.rows) : nullptr;
    W.share = distill ? L.take<float>(A.rows * A.top) : nullptr;
    W.entropy = distill ? L.take<float>(A.rows) : nullptr;
    const long long stages = (long long)P.terms * P.padded / HEAD_K;
    P.x = L.take<unsigned short>(head_block_values(rows, stages));
    P.w = L.take<unsigned short>(P.few ? 0 : head_block_values(most, stages));
    P.logits = P.in_parts ? L.take<float>(rows * P.piece * P.z.splits) : nullptr;
    if (!backward) {
        P.stats = L.take<Stat>(rows * (P.stat_parts + (P.pieces > 1)));
        P.picked = distill ? nullptr : L.take<float>(rows);
        P.bytes = L.at;
        return P;
    }
    W.coef = L.take<float>(A.rows);
    W.boundless = L.take<int>(A.rows);
    const Product dx{rows, A.width, P.piece, P.grad_terms, P.pieces == 1, 0.0};  // (several: added up piece after piece)
    const Product dw{most, A.width, rows, P.grad_terms, true, 3.0};
    double apart = 0.0, together = 0.0;
    P.dx = pick_tile(dx, &apart), P.dw = pick_tile(dw, &apart);
    if (P.few) {
        P.dx.splits = (int)std::min<long long>(std::max<long long>(1, A.classes / 256), std::max(1, 1024 / ceil_div(A.width, 256)));
    } else if (P.pieces == 1) {
        const Two two = pick_two(dx, dw, &together);
        if (together < apart) P.pair = true, P.dx = two.a, P.dw = two.b;
    }
    const long long ld = round_up(A.width, 4);
    const long long row_stages = P.terms * P.padded_rows / HEAD_K, class_stages = P.terms * round_up(P.piece, HEAD_K) / HEAD_K;
    P.xt = L.take<unsigned short>(head_block_values(A.width, row_stages));
    P.wt = L.take<unsigned short>(P.few ? 0 : head_block_values(A.width, class_stages));
    P.gn = L.take<unsigned short>(head_block_values(rows, class_stages / P.terms * P.grad_terms));
    P.gt = L.take<unsigned short>(head_block_values(most, row_stages / P.terms * P.grad_terms));
    P.dx_sums = L.take<float>(rows * ld * P.dx.splits);
    P.dw_sums = P.dw.splits > 1 ? L.take<float>(most * ld * P.dw.splits) : nullptr;
    P.bias_sums = L.take<float>((rows + 63) / 64 * P.piece);
    P.taken = L.take<long long>(A.classes);
    P.bytes = L.at;
    return P;
}

template <typename K, typename... Args>
hipError_t run(K kernel, unsigned blocks, unsigned threads, hipStream_t st, Args... args)
{
    kernel<<<dim3(blocks), dim3(threads), 0, st>>>(args...);
    return hipGetLastError();
}
#define CAPSCAPS_TRY(call)                                        \
    do {                                                          \
        const hipError_t err_ = (call);                           \
        if (err_ != hipSuccess) return status_from_hip(err_);     \
    } while (0)

hipError_t pack(const Plan& P, const void* from, long long stride, int columns, long long rows, const Head* kept, int dtype,
                unsigned short* to, hipStream_t st)
{
    const int* rows_of = kept != nullptr ? kept->rows_of : nullptr;
    const int* count = kept != nullptr ? kept->count : nullptr;
    const long long stages = P.padded / HEAD_K;
    const unsigned blocks = blocks_for((rows + 15) / 16 * stages, 4);
    return P.terms == 3 ? run(pack_kernel<true>, blocks, THREADS, st, from, stride, columns, rows, rows_of, count, to, stages)
                        : run(pack_kernel<false>, blocks, THREADS, st, from, stride, columns, rows, rows_of, count, to, stages);
}
Across across_of(const Plan& P, const void* from, long long stride, int columns, long long rows, const Head* kept, unsigned short* to,
                 long long padded, unsigned short* straight)
{
    Across A{};
    A.from = from, A.stride = stride, A.columns = columns, A.rows = rows;
    if (kept != nullptr) A.rows_of = kept->rows_of, A.count = kept->count;
    A.to = to, A.stages = padded / HEAD_K;
    A.straight = straight, A.straight_stages = P.padded / HEAD_K;
    A.blocks = blocks_for((padded + 63) / 64 * ((columns + 63) / 64), 1);
    return A;
}

const void* weight_at(const Head& H, long long cls)
{
    return static_cast<const char*>(H.weight) + cls * H.weight_stride * (long long)element_bytes(H.dtype);
}

hipError_t few_logits(const Head& H, const Plan& P, hipStream_t st)
{
    const auto kernel = H.rows <= 16   ? few_logits_kernel<1>
                        : H.rows <= 32 ? few_logits_kernel<2>
                        : H.rows <= 48 ? few_logits_kernel<3>
                                       : few_logits_kernel<4>;
    return run(kernel, (unsigned)(ceil_div(H.classes, 128) * P.z.splits), THREADS, st, H, P.logits, P.piece, P.z.splits, H.rows * P.piece);
}
hipError_t few_rows(const Head& H, const Plan& P, long long ld, hipStream_t st)
{
    const auto kernel = H.rows <= 16   ? few_rows_kernel<1>
                        : H.rows <= 32 ? few_rows_kernel<2>
                        : H.rows <= 48 ? few_rows_kernel<3>
                                       : few_rows_kernel<4>;
    return run(kernel, (unsigned)(ceil_div(H.width, 256) * P.dx.splits), THREADS, st, H, (const float*)P.logits, P.piece, P.dx_sums, ld,
               P.dx.splits, H.rows * ld);
}

// The rows that count
int begin(const Head& H, const Plan& P, const float* dloss, long long dloss_stride, hipStream_t st)
{
    if (P.distill) CAPSCAPS_TRY(run(teacher_kernel, blocks_for(H.rows, 4), THREADS, st, H));
    CAPSCAPS_TRY(run(rows_kernel, 1, 1024, st, H, dloss, dloss_stride));
    return CAPSCAPS_OK;
}

// The product of x and a piece's weights, for launch_head_gemm with an end of the caller's; `across`: NULL, or what the caller packs
// before it, the weights as an operand that contracts classes
int logits_of(const Head& H, const Plan& P, long long first, long long classes, Across* across, HeadGemm& g, hipStream_t st)
{
    g = HeadGemm{};
    const int stages = P.padded / HEAD_K;
    g.a = P.x, g.stages_a = (long long)P.terms * stages;
    // Weights are read in place where they can be (16 bits, whole vectors, whole stages, rows near enough for 32-bit
    // offsets): the product of 6144 rows with 32768 classes of 4096 values takes 1212 us so and 1161 with a copy in blocks, which
    // itself takes 120 (4 bytes a value at 4.5 TB/s): as much for 15000 rows.
    if (P.terms == 1 && H.rows < 15000 && H.width % HEAD_K == 0 && vectors_of(H.weight, H.weight_stride, H.dtype) &&
        H.weight_stride <= (1 << 21)) {
        g.b = weight_at(H, first), g.ldb = H.weight_stride * 2;
    } else {
        if (across == nullptr) CAPSCAPS_TRY(pack(P, weight_at(H, first), H.weight_stride, H.width, classes, nullptr, H.dtype, P.w, st));
        g.b = P.w, g.stages_b = g.stages_a;
    }
    if (across != nullptr)
        *across = across_of(P, weight_at(H, first), H.weight_stride, H.width, classes, nullptr, P.wt, round_up(classes, HEAD_K),
                            g.b == P.w ? P.w : nullptr);
    g.m_rows = H.rows, g.n_rows = classes, g.m_count = H.count, g.k = H.width;
    g.plane_a = g.plane_b = stages;
    g.terms = P.terms;
    g.dtype = H.dtype, g.splits = P.z.splits;
    if (P.in_parts) {
        g.out = P.logits, g.ldo = P.piece, g.out_split = H.rows * P.piece, g.out_dtype = CAPSCAPS_FP32;
    } else {
        g.bias = H.bias != nullptr ? H.bias + first : nullptr;
        g.inv_tau = 1.0f / H.tau;
    }
    return CAPSCAPS_OK;
}

int forward(const Head& H, const Plan& P, float* loss, float* lse, float* logq, hipStream_t st)
{
    if (H.rows == 0) return CAPSCAPS_OK;
    const bool few = H.rows < 512;
    int rc = begin(H, P, nullptr, 0, st);
    if (rc != CAPSCAPS_OK) return rc;
    if (!P.few) CAPSCAPS_TRY(pack(P, H.x, H.x_stride, H.width, H.rows, &H, H.dtype, P.x, st));
    for (int piece = 0; piece < P.pieces; ++piece) {
        const long long first = piece * P.piece, classes = std::min<long long>(P.piece, H.classes - first);
        HeadGemm g;
        if (P.few) {
            CAPSCAPS_TRY(few_logits(H, P, st));
        } else {
            rc = logits_of(H, P, first, classes, nullptr, g, st);
            if (rc != CAPSCAPS_OK) return rc;
            g.stats = P.pieces > 1 ? P.stats + H.rows : P.stats;
            CAPSCAPS_TRY(launch_head_gemm(g, P.z.tile, P.in_parts ? HEAD_OUT : HEAD_STATS, st));
        }
        if (P.in_parts)
            CAPSCAPS_TRY(run(stats_kernel, blocks_for(H.rows * P.stat_parts, 1), THREADS, st, H, (const float*)P.logits, P.piece, P.z.splits,
                             H.rows * P.piece, P.stats));
        if (P.pieces > 1)
            CAPSCAPS_TRY(run(few ? fold_kernel<1> : fold_kernel<8>, blocks_for(H.rows, few ? 1 : 8), THREADS, st, H, P.stats,
                             ceil_div(classes, head_tile_shape(P.z.tile).stat_columns), piece > 0));
    }
    // (the entries' z: where logq goes, or in the workspace)
    float* const picked = logq != nullptr ? logq : P.picked;
    const long long quads = H.rows * ((H.top + 3) / 4);
    const bool pick = !P.in_parts && few && H.top <= 4;
    if (!P.in_parts && !pick)
        CAPSCAPS_TRY(run(quads < 1024 ? pick_kernel<true> : pick_kernel<false>, blocks_for(quads, quads < 1024 ? 1 : 4), THREADS, st, H, picked));
    const auto kernel = P.in_parts ? (few ? loss_kernel<1, PARTS> : loss_kernel<8, PARTS>)
                        : pick     ? loss_kernel<1, PICK>
                                   : (few ? loss_kernel<1, PICKED> : loss_kernel<8, PICKED>);
    const Parts logits{P.logits, P.piece, H.rows * P.piece, P.z.splits};
    CAPSCAPS_TRY(run(kernel, blocks_for(H.rows, few ? 1 : 8), THREADS, st, H, (const Stat*)P.stats, P.pieces > 1 ? 1 : P.stat_parts, picked,
                     logits, loss, lse, logq));
    return CAPSCAPS_OK;
}

struct Gradients {
    const float *loss, *lse, *logq, *dloss;
    long long dloss_stride;
    void *dx, *dweight;
    float* dbias;
};

template <bool TERMS>
int backward_pieces(const Head& H, const Plan& P, const Gradients& G, hipStream_t st)
{
    const long long ld = round_up(H.width, 4);
    const float* scale = reinterpret_cast<const float*>(H.count + 1);
    const int size = (int)element_bytes(H.dtype);
    // (with the first piece's weights: x both ways, and zeros for what entries take of the bias' gradient)
    Across x_across{};
    if (G.dweight != nullptr)
        x_across = across_of(P, H.x, H.x_stride, H.width, H.rows, &H, P.xt, P.padded_rows, P.x);
    else if (!P.few)
        CAPSCAPS_TRY(pack(P, H.x, H.x_stride, H.width, H.rows, &H, H.dtype, P.x, st));
    unsigned clear = G.dbias != nullptr ? blocks_for(H.classes, THREADS) : 0;
    for (int piece = 0; piece < P.pieces; ++piece) {
        const long long first = piece * P.piece, classes = std::min<long long>(P.piece, H.classes - first);
        HeadGemm z;
        Across w_across{};
        if (!P.few) {
            const int rc = logits_of(H, P, first, classes, G.dx != nullptr ? &w_across : nullptr, z, st);
            if (rc != CAPSCAPS_OK) return rc;
        }
        if (x_across.blocks + w_across.blocks + clear > 0)
            CAPSCAPS_TRY(run(pack_transposed_kernel<TERMS>, x_across.blocks + w_across.blocks + clear, THREADS, st, x_across, w_across, P.taken,
                             H.classes));
        x_across.blocks = clear = 0;
        const int padded = (int)round_up(classes, HEAD_K);
        float* const sums = G.dbias != nullptr ? P.bias_sums : nullptr;
        if (P.in_parts) {
            CAPSCAPS_TRY(P.few ? few_logits(H, P, st) : launch_head_gemm(z, P.z.tile, HEAD_OUT, st));
            const long long tiles = (P.padded_rows + 63) / 64 * ((padded + 63) / 64);
            CAPSCAPS_TRY(run(gradient_kernel<TERMS>, blocks_for(tiles, 1), THREADS, st, H, G.lse, (const float*)P.logits, P.piece,
                             P.z.splits, H.rows * P.piece, first, (int)classes, P.gn, padded, P.gt, P.padded_rows, P.grad_terms, sums, P.few ? P.logits : nullptr));
        } else {
            z.coef = H.coef, z.lse = G.lse, z.rows_of = H.rows_of;
            z.gn = P.gn, z.gt = P.gt, z.planes_n = padded / HEAD_K, z.planes_t = (int)(P.padded_rows / HEAD_K), z.sums = sums;
            z.grad_terms = P.grad_terms;
            CAPSCAPS_TRY(launch_head_gemm(z, P.z.tile, HEAD_GRADIENT, st));
        }
        CAPSCAPS_TRY(run(entries_kernel<TERMS>, blocks_for(H.rows, 4), THREADS, st, H, G.loss, G.logq, first, (int)classes, P.gn,
                         padded, P.gt, P.padded_rows, P.grad_terms, G.dbias != nullptr ? P.taken : nullptr, sums, P.few ? P.logits : nullptr,
                         P.piece));
        Bias bias{};
        if (G.dbias != nullptr)
            bias = {P.bias_sums, P.taken, H.boundless, P.gt, P.grad_terms * (P.padded_rows / HEAD_K), G.dbias, first, padded,
                    P.in_parts ? 64 : head_tile_shape(P.z.tile).sum_rows, (int)classes, blocks_for(classes, THREADS)};
        HeadGemm x{}, w{};
        Finish dx{}, dw{};
        if (G.dx != nullptr) {
            x.a = P.gn, x.b = P.wt;
            x.plane_a = x.plane_b = padded / HEAD_K, x.terms = P.grad_terms;
            x.stages_a = (long long)P.grad_terms * x.plane_a, x.stages_b = (long long)P.terms * x.plane_b;
            x.m_rows = H.rows, x.n_rows = H.width, x.m_count = H.count, x.k = classes;
            x.dtype = H.dtype, x.out = P.dx_sums, x.ldo = ld, x.out_split = H.rows * ld, x.out_dtype = CAPSCAPS_FP32;
            x.splits = P.dx.splits, x.accumulate = piece > 0;
            if (piece == P.pieces - 1)
                dx = {H.pos, P.dx_sums, ld, H.rows * ld, H.rows, P.dx.splits, H.width, G.dx, blocks_for(H.rows * (ld / 4), THREADS)};
        }
        if (G.dweight != nullptr) {
            char* out = static_cast<char*>(G.dweight) + first * H.width * size;
            w.a = P.gt, w.b = P.xt;
            w.plane_a = w.plane_b = (int)(P.padded_rows / HEAD_K), w.terms = P.grad_terms;
            w.stages_a = (long long)P.grad_terms * w.plane_a, w.stages_b = (long long)P.terms * w.plane_b;
            w.m_rows = classes, w.n_rows = H.width, w.k = H.rows, w.k_count = H.count;
            w.dtype = H.dtype, w.splits = P.dw.splits;
            const bool direct = P.dw.splits == 1;
            w.out = direct ? out : (void*)P.dw_sums;
            w.ldo = direct ? H.width : ld, w.out_split = classes * ld, w.out_dtype = direct ? H.dtype : CAPSCAPS_FP32;
            if (direct)
                w.scale = scale;
            else
                dw = {nullptr, P.dw_sums, ld, classes * ld, classes, P.dw.splits, H.width, out, blocks_for(classes * (ld / 4), THREADS)};
        }
        if (P.pair && G.dx != nullptr && G.dweight != nullptr) {
            CAPSCAPS_TRY(launch_head_gemm_pair(x, w, P.dx.tile, st));
        } else {
            if (G.dx != nullptr) CAPSCAPS_TRY(P.few ? few_rows(H, P, ld, st) : launch_head_gemm(x, P.dx.tile, HEAD_OUT, st));
            if (G.dweight != nullptr) CAPSCAPS_TRY(launch_head_gemm(w, P.dw.tile, HEAD_OUT, st));
        }
        const unsigned blocks = dx.blocks + dw.blocks + bias.blocks;
        if (blocks > 0) CAPSCAPS_TRY(run(finish_kernel, blocks, THREADS, st, (const int*)H.count, dx, dw, bias, H.dtype));
    }
    return CAPSCAPS_OK;
}

__global__ void __launch_bounds__(THREADS) zero_kernel(unsigned short* p, long long n)
{
    for (long long t = blockIdx.x * (long long)THREADS + threadIdx.x; t < n; t += (long long)gridDim.x * THREADS) p[t] = 0;
}

int backward(const Head& H, const Plan& P, const Gradients& G, hipStream_t st)
{
    if (H.rows == 0) {  // (sums over no rows)
        const long long n = H.classes * H.width * (long long)(element_bytes(H.dtype) / 2);
        if (G.dweight != nullptr)
            CAPSCAPS_TRY(run(zero_kernel, blocks_for(n, THREADS), THREADS, st, static_cast<unsigned short*>(G.dweight), n));
        if (G.dbias != nullptr)
            CAPSCAPS_TRY(run(zero_kernel, blocks_for(H.classes * 2, THREADS), THREADS, st, reinterpret_cast<unsigned short*>(G.dbias), H.classes * 2));
        return CAPSCAPS_OK;
    }
    const int rc = begin(H, P, G.dloss, G.dloss_stride, st);
    if (rc != CAPSCAPS_OK) return rc;
    return P.terms == 3 ? backward_pieces<true>(H, P, G, st) : backward_pieces<false>(H, P, G, st);
}

bool misaligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

// The head of a call; false where something about it is wrong
bool make_head(const capscaps_head& A, const capscaps_head_tensors& T, bool distill, Head& H)
{
    const size_t size = element_bytes(A.dtype), index = A.index_bits / 8;
    if (T.weight == nullptr || misaligned(T.weight, size) || misaligned(T.bias, 4)) return false;
    if (A.rows > 0 && (T.x == nullptr || T.index == nullptr || misaligned(T.x, size) || misaligned(T.index, index))) return false;
    constexpr long long far = 1ll << 40;
    if (T.x_stride < 0 || T.x_stride > far || T.weight_stride < 0 || T.weight_stride > far || T.index_stride < 0 ||
        T.index_stride > far)
        return false;
    if (distill) {
        if (T.teacher_stride < 0 || T.teacher_stride > far) return false;
        if (A.rows > 0 && (T.teacher == nullptr || misaligned(T.teacher, element_bytes(A.teacher_dtype)))) return false;
    } else if (T.teacher != nullptr) {
        return false;
    }
    H = Head{};
    H.rows = A.rows, H.classes = A.classes, H.width = A.width, H.dtype = A.dtype, H.top = A.top, H.tau = A.temperature;
    H.wide_index = A.index_bits == 64;
    H.x = T.x, H.weight = T.weight, H.bias = T.bias, H.index = T.index, H.teacher = T.teacher;
    H.x_stride = T.x_stride, H.weight_stride = T.weight_stride, H.index_stride = T.index_stride;
    H.teacher_stride = T.teacher_stride, H.teacher_dtype = A.teacher_dtype;
    return true;
}

int run_forward(const capscaps_head* head, const capscaps_head_fwd_args* args, bool distill, void* workspace,
                size_t workspace_bytes, void* stream)
{
    const int rc = check_head(head, distill);
    if (rc != CAPSCAPS_OK) return rc;
    if (args == nullptr) return CAPSCAPS_EINVAL;
    Head H;
    if (!make_head(*head, args->tensors, distill, H)) return CAPSCAPS_EINVAL;
    if (head->rows > 0 && (args->loss == nullptr || args->lse == nullptr || (distill && args->logq == nullptr)))
        return CAPSCAPS_EINVAL;
    if (misaligned(args->loss, 4) || misaligned(args->lse, 4) || misaligned(args->logq, 4) || (!distill && args->logq != nullptr))
        return CAPSCAPS_EINVAL;
    const Plan P = make_plan(*head, distill, false, workspace, &H);
    if (workspace == nullptr || workspace_bytes < P.bytes) return CAPSCAPS_EWORKSPACE;
    if (misaligned(workspace, 16)) return CAPSCAPS_EINVAL;
    return forward(H, P, args->loss, args->lse, args->logq, static_cast<hipStream_t>(stream));
}

int run_backward(const capscaps_head* head, const capscaps_head_bwd_args* args, bool distill, void* workspace,
                 size_t workspace_bytes, void* stream)
{
    const int rc = check_head(head, distill);
    if (rc != CAPSCAPS_OK) return rc;
    if (args == nullptr) return CAPSCAPS_EINVAL;
    Head H;
    if (!make_head(*head, args->tensors, distill, H)) return CAPSCAPS_EINVAL;
    const capscaps_head_bwd_args& A = *args;
    if (head->rows > 0 && (A.lse == nullptr || A.dloss == nullptr || (distill ? A.logq : A.loss) == nullptr)) return CAPSCAPS_EINVAL;
    if ((A.dx == nullptr || head->rows == 0) && A.dweight == nullptr && A.dbias == nullptr) return head->rows == 0 && A.dx != nullptr ? CAPSCAPS_OK : CAPSCAPS_EINVAL;
    if (A.dloss_stride < 0 || A.dloss_stride > (1ll << 40)) return CAPSCAPS_EINVAL;
    const size_t size = element_bytes(head->dtype);
    for (const void* p : {(const void*)A.loss, (const void*)A.lse, (const void*)A.logq, (const void*)A.dloss, (const void*)A.dbias})
        if (misaligned(p, 4)) return CAPSCAPS_EINVAL;
    if (misaligned(A.dx, size) || misaligned(A.dweight, size)) return CAPSCAPS_EINVAL;
    const Plan P = make_plan(*head, distill, true, workspace, &H);
    if (workspace == nullptr || workspace_bytes < P.bytes) return CAPSCAPS_EWORKSPACE;
    if (misaligned(workspace, 16)) return CAPSCAPS_EINVAL;
    const Gradients G{A.loss, A.lse, distill ? A.logq : nullptr, A.dloss, A.dloss_stride, A.dx, A.dweight, A.dbias};
    return backward(H, P, G, static_cast<hipStream_t>(stream));
}

}  // namespace
}  // namespace capscaps

using namespace capscaps;

extern "C" {

size_t capscaps_class_loss_workspace_bytes(const capscaps_head* head, int backward)
{
    return check_head(head, false) == CAPSCAPS_OK ? make_plan(*head, false, backward != 0, nullptr, nullptr).bytes : 0;
}
size_t capscaps_distill_loss_workspace_bytes(const capscaps_head* head, int backward)
{
    return check_head(head, true) == CAPSCAPS_OK ? make_plan(*head, true, backward != 0, nullptr, nullptr).bytes : 0;
}
int capscaps_class_loss_fwd(const capscaps_head* head, const capscaps_head_fwd_args* args, void* workspace,
                            size_t workspace_bytes, void* stream)
{
    return run_forward(head, args, false, workspace, workspace_bytes, stream);
}
int capscaps_class_loss_bwd(const capscaps_head* head, const capscaps_head_bwd_args* args, void* workspace,
                            size_t workspace_bytes, void* stream)
{
    return run_backward(head, args, false, workspace, workspace_bytes, stream);
}
int capscaps_distill_loss_fwd(const capscaps_head* head, const capscaps_head_fwd_args* args, void* workspace,
                              size_t workspace_bytes, void* stream)
{
    return run_forward(head, args, true, workspace, workspace_bytes, stream);
}
int capscaps_distill_loss_bwd(const capscaps_head* head, const capscaps_head_bwd_args* args, void* workspace,
                              size_t workspace_bytes, void* stream)
{
    return run_backward(head, args, true, workspace, workspace_bytes, stream);
}

}  // extern "C"
