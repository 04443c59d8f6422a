// Group norm with its activation, channels last, forward and backward.
//
// x [images][positions][width]; the width is cut into groups of neighbouring columns, and a group of an image, its
// columns at all positions, is normalised by its own mean and variance:
//
//     a = (x - mean) * rstd * weight + bias        y = act(a)
//
// backward, with xn = (x - mean) * rstd and da = dy * act'(a):
//
//     dx = rstd * (da * weight - mean(da * weight) - xn * mean(da * weight * xn))      (means over the group)
//     dweight = sum over images and positions of da * xn          dbias = the same of da
//
// Bound: HBM, with 12 (24) operations a value far below what the vector units do meanwhile.
//
// A lane holds vectors of V neighbouring columns (16 bytes of x where the columns allow it) of some positions, the
// same columns at each; a workgroup takes a slab of columns: one group, some whole ones, or a part of one.
// Two forms.  Resident: a slab of whole groups at all positions of an image fits a workgroup's registers; each value
// is read once, and the variance is taken about the mean, as in the formula.  In two passes: a workgroup takes a
// share of the positions, the shares' means and sums of squared distances from them (about a lane's first value of
// the column, then about its mean so far, which keeps the squares small whatever the mean) are joined, and a second
// pass writes the result.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "conv_shape.h"
#include "row_vectors.h"

namespace capscaps {
namespace {

constexpr int CUS = 256;
constexpr int RESIDENT = 1024, RESIDENT_BACK = 512;  // threads of a workgroup at most, forward and backward
constexpr int SHARED = 256;    // ... in two passes
constexpr int MOST_BLOCKS = 1 << 22;


struct GroupPlan {
    int v, items;            // columns of a vector; vectors a lane holds (0: two passes)
    int threads, rows, vecs; // rows * vecs lanes work: a row is a position's columns of the slab
    int slab, slabs;         // columns, slabs of an image
    int whole;               // groups of a slab (0: a slab is a part of a group)
    int parts;               // slabs of a group, where it is cut
    int fold;                // columns of a vector that are of one group: V, or 1 where vectors straddle groups
    long long shares, per;   // two passes: shares of an image's positions, positions of a share; resident: workgroups of a slab
    long long blocks;
};

struct GroupCall {
    capscaps_group_norm G;
    GroupPlan P;
    int columns;  // of a group
    const char *x, *dy;
    char* out;  // y or dx
    const float *weight, *bias;
    float *mean, *rstd;
    long long x_stride, dy_stride, out_stride;
    float* partial;
};

// V values of a type as they lie in memory, at any element's address
template <int DT, int V>
struct Packed {
    static constexpr int SIZE = DT == CAPSCAPS_FP32 ? 4 : 2, BYTES = V * SIZE, WORDS = (BYTES + 3) / 4;
    unsigned w[WORDS];
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int k = 0; k < WORDS; ++k) w[k] = 0;
    }
    __device__ __forceinline__ void load(const char* p)
    {
        if constexpr (BYTES == 2) {
            w[0] = *reinterpret_cast<const unsigned short*>(p);
        } else if constexpr (WORDS == 1) {
            const typename Words<1, SIZE>::type r = *reinterpret_cast<const typename Words<1, SIZE>::at*>(p);
            w[0] = r[0];
        } else {
            const typename Words<WORDS, SIZE>::type r = *reinterpret_cast<const typename Words<WORDS, SIZE>::at*>(p);
#pragma unroll
            for (int k = 0; k < WORDS; ++k) w[k] = r[k];
        }
    }
    // From here on the values are taken out of their words again (kept as fp32 from one phase to the next they fill twice
    // the registers, and fewer workgroups of a CU run)
    __device__ __forceinline__ void hold()
    {
#pragma unroll
        for (int k = 0; k < WORDS; ++k) asm volatile("" : "+v"(w[k]));
    }
    __device__ __forceinline__ float value(int k) const  // (k is a constant after unrolling)
    {
        if constexpr (DT == CAPSCAPS_FP32) return __builtin_bit_cast(float, w[k]);
        if constexpr (DT == CAPSCAPS_BF16)
            return __builtin_bit_cast(float, (k & 1) ? (w[k / 2] & 0xffff0000u) : (w[k / 2] << 16));
        return Element<CAPSCAPS_FP16>::get((unsigned short)((k & 1) ? (w[k / 2] >> 16) : (w[k / 2] & 0xffffu)));
    }
};
template <int DT, int V>
__device__ __forceinline__ void store_values(char* p, const float* f)
{
    if constexpr (DT == CAPSCAPS_FP32 && V == 1) {
        *reinterpret_cast<float*>(p) = f[0];
    } else if constexpr (DT != CAPSCAPS_FP32 && V == 1) {
        *reinterpret_cast<unsigned short*>(p) = Element<DT>::put(f[0]);
    } else if constexpr (DT != CAPSCAPS_FP32 && V == 2) {
        typedef unsigned at __attribute__((aligned(2)));
        *reinterpret_cast<at*>(p) = Element<DT>::put(f[0]) | (unsigned)Element<DT>::put(f[1]) << 16;
    } else {
        typedef Raw<DT, V> R;
        __builtin_nontemporal_store(pack<DT, V>(f).w, reinterpret_cast<typename R::Whole*>(p));
    }
}

// act(a), and act'(a)  (v_rcp_f32 is off by one unit in the last place)
__device__ __forceinline__ float act_value(int act, float a)
{
    if (act == CAPSCAPS_ACT_LINEAR) return a;
    const float q = __builtin_amdgcn_rcpf(1.0f + __expf(-a));
    return act == CAPSCAPS_ACT_SIGMOID ? q : a * q;
}
__device__ __forceinline__ float act_slope(int act, float a)
{
    if (act == CAPSCAPS_ACT_LINEAR) return 1.0f;
    const float q = __builtin_amdgcn_rcpf(1.0f + __expf(-a)), p = 1.0f - q;
    return q * (act == CAPSCAPS_ACT_SIGMOID ? p : __builtin_fmaf(a, p, 1.0f));
}

// Consecutive workgroups go to the eight XCDs in turn; neighbouring slabs share lines of memory, so each XCD takes a
// run of them.
__device__ __forceinline__ long long by_xcd(long long block, long long blocks)
{
    const long long span = blocks & ~7ll;
    return block < span ? (block & 7) * (span >> 3) + (block >> 3) : block;
}

template <int V>
__device__ __forceinline__ void load_columns(float* f, const float* p, long long at, float none)
{
#pragma unroll
    for (int k = 0; k < V; ++k) f[k] = p != nullptr ? p[at + k] : none;
}

// What a table of the slab's groups holds for a lane's columns: one value where a vector is of one group
template <int V, bool FOLD>
struct OfGroups {
    float f[FOLD ? 1 : V];
    __device__ __forceinline__ OfGroups(const float* table, int c, int columns, float factor = 1.0f)
    {
#pragma unroll
        for (int k = 0; k < (FOLD ? 1 : V); ++k) f[k] = table[(c * V + k) / columns] * factor;
    }
    __device__ __forceinline__ float operator[](int k) const { return f[FOLD ? 0 : k]; }
};

template <int V>
__device__ __forceinline__ void put_columns(float* to, const float* f)  // (to LDS, at a multiple of V)
{
    if constexpr (V % 4 == 0) {
        typedef float four __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int k = 0; k < V; k += 4) *reinterpret_cast<four*>(to + k) = four{f[k], f[k + 1], f[k + 2], f[k + 3]};
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k) to[k] = f[k];
    }
}

// Sums over each group of a slab of what the working lanes hold for their columns (summed first where a vector is of
// one group): to total[group], read after the barrier that ends this.
template <int V, bool FOLD>
__device__ __forceinline__ void group_totals(const GroupPlan& P, const float* f, int q, int c, float* lds,
                                             float* total)
{
    constexpr int per = FOLD ? 1 : V;                    // values of a lane
    const int row = P.vecs * per, mine = row / P.whole;  // ... of a position, and of a group of it
    if (q < P.rows) {
        if constexpr (FOLD) {
            float s = f[0];
#pragma unroll
            for (int k = 1; k < V; ++k) s += f[k];
            lds[q * row + c] = s;
        } else {
            put_columns<V>(lds + q * row + c * V, f);
        }
    }
    __syncthreads();
    const int lane = threadIdx.x & 63, waves = P.threads >> 6;
    for (int g = threadIdx.x >> 6; g < P.whole; g += waves) {
        float s = 0.0f;
        for (int t = lane; t < P.rows * mine; t += 64) {
            const int at = P.whole == 1 ? t : t / mine * row + g * mine + t % mine;
            s += lds[at];
        }
        s = lanes_sum(s, 64);
        if (lane == 0) total[g] = s;
    }
    __syncthreads();
}

// ---------------------------------------------------------------------------------------- resident
// Registers hold the slab from its load to its store; the sums cross lanes twice through LDS.  64 images of 256 positions of
// 4096 values, fp32 to bf16, take 68 us (5.9 TB/s), 64 positions of one image 5.8 us (latency).
template <int XD, int YD, int V, int I, bool FOLD>
__global__ void __launch_bounds__(RESIDENT) group_fwd_resident_kernel(GroupCall C)
{
    extern __shared__ __attribute__((aligned(16))) float lds[];
    const GroupPlan& P = C.P;
    typedef Packed<XD, V> X;
    constexpr int YB = YD == CAPSCAPS_FP32 ? 4 : 2;
    float* total = lds + P.rows * P.vecs * (FOLD ? 1 : V);
    const int q = threadIdx.x / P.vecs, c = threadIdx.x - q * P.vecs;
    const float m = 1.0f / ((float)C.G.positions * (float)C.columns);
    const long long b = by_xcd(blockIdx.x, gridDim.x);
    const int slab = (int)(b % P.slabs);
    const long long col = (long long)slab * P.slab + c * V;
    const int positions = (int)C.G.positions;
    // a lane's vectors: positions q, q + rows, ...
    const int mine = q < P.rows && q < positions ? (positions - q + P.rows - 1) / P.rows : 0;
    float w[V], bias[V];
    load_columns<V>(w, mine ? C.weight : nullptr, col, 1.0f);
    load_columns<V>(bias, mine ? C.bias : nullptr, col, 0.0f);
    const long long x_step = P.rows * C.x_stride * X::SIZE, y_step = P.rows * C.out_stride * YB;
    for (long long n = b / P.slabs; n < C.G.images; n += P.shares) {
        const char* x = C.x + ((n * positions + q) * C.x_stride + col) * X::SIZE;
        X v[I];
#pragma unroll
        for (int i = 0; i < I; ++i) {
            v[i].clear();
            if (i < mine) v[i].load(x + i * x_step);
        }
        float s[V];
#pragma unroll
        for (int k = 0; k < V; ++k) s[k] = 0.0f;
#pragma unroll
        for (int i = 0; i < I; ++i)
#pragma unroll
            for (int k = 0; k < V; ++k) s[k] += v[i].value(k);
        group_totals<V, FOLD>(P, s, q, c, lds, total);
        const OfGroups<V, FOLD> mean(total, c, C.columns, m);
        const long long stat = n * C.G.groups + (long long)slab * P.whole;
        if (C.mean != nullptr)
            for (int g = threadIdx.x; g < P.whole; g += P.threads) C.mean[stat + g] = total[g] * m;
#pragma unroll
        for (int k = 0; k < V; ++k) s[k] = 0.0f;
#pragma unroll
        for (int i = 0; i < I; ++i) {
            v[i].hold();
            if (i < mine)
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    const float d = v[i].value(k) - mean[k];
                    s[k] = __builtin_fmaf(d, d, s[k]);
                }
        }
        __syncthreads();  // (everybody has read the totals)
        group_totals<V, FOLD>(P, s, q, c, lds, total);
        if (C.rstd != nullptr)
            for (int g = threadIdx.x; g < P.whole; g += P.threads)
                C.rstd[stat + g] = 1.0f / __builtin_sqrtf(total[g] * m + C.G.eps);
        OfGroups<V, FOLD> rstd(total, c, C.columns, m);
#pragma unroll
        for (int k = 0; k < (FOLD ? 1 : V); ++k) rstd.f[k] = 1.0f / __builtin_sqrtf(rstd.f[k] + C.G.eps);
#pragma unroll
        for (int k = 0; k < V; ++k) s[k] = w[k] * rstd[k];
        char* y = C.out + ((n * positions + q) * C.out_stride + col) * YB;
#pragma unroll
        for (int i = 0; i < I; ++i) {
            v[i].hold();
            if (i < mine) {
                float f[V];
#pragma unroll
                for (int k = 0; k < V; ++k)
                    f[k] = act_value(C.G.act, __builtin_fmaf(v[i].value(k) - mean[k], s[k], bias[k]));
                store_values<YD, V>(y + i * y_step, f);
            }
        }
        __syncthreads();  // (... and the totals of the squares)
    }
}

// What one value adds to the sums over its column, and what dx takes of it
struct GroupBack {
    float xn, da;
};
__device__ __forceinline__ GroupBack group_back(int act, float x, float dy, float mean, float rstd, float w, float bias)
{
    GroupBack k;
    k.xn = (x - mean) * rstd;
    k.da = dy * act_slope(act, __builtin_fmaf(k.xn, w, bias));
    return k;
}

// partial[workgroup of the slab][2][width]: sums of da * xn and of da over its images.  What bounds it besides HBM is the
// exponential and the quotient of act': da is kept for the second use of it.  A workgroup takes one image after the other, the
// next one's values on their way while the sums are joined and dx is written: 64 images of 256 positions of 4096 bf16 values in
// 32 groups take 89 us, 4.5 TB/s.
template <int XD, int YD, int V, int I, bool FOLD>
__global__ void __launch_bounds__(RESIDENT_BACK) group_bwd_resident_kernel(GroupCall C)
{
    // [2][rows][slab] sums of lanes, [2][slab] of columns, [2][slab] over images, [2][whole]
    extern __shared__ __attribute__((aligned(16))) float lds[];
    const GroupPlan& P = C.P;
    typedef Packed<XD, V> X;
    typedef Packed<YD, V> Y;
    constexpr int YB = Y::SIZE;
    const int cells = P.rows * P.slab;
    float *column = lds + 2 * cells, *over = column + 2 * P.slab, *total = over + 2 * P.slab;
    const int q = threadIdx.x / P.vecs, c = threadIdx.x - q * P.vecs;
    const float m = 1.0f / ((float)C.G.positions * (float)C.columns);
    const long long b = by_xcd(blockIdx.x, gridDim.x);
    const int slab = (int)(b % P.slabs), lane = threadIdx.x & 63, waves = P.threads >> 6;
    const long long col = (long long)slab * P.slab + c * V;
    const int positions = (int)C.G.positions;
    const int mine = q < P.rows && q < positions ? (positions - q + P.rows - 1) / P.rows : 0;
    float w[V], bias[V];
    load_columns<V>(w, mine ? C.weight : nullptr, col, 1.0f);
    load_columns<V>(bias, mine ? C.bias : nullptr, col, 0.0f);
    const long long x_step = P.rows * C.x_stride * X::SIZE, dy_step = P.rows * C.dy_stride * YB;
    const long long out_step = P.rows * C.out_stride * YB;
    for (int t = threadIdx.x; t < 2 * P.slab; t += P.threads) over[t] = 0.0f;
    X v[I], ahead[I];
    Y d[I];
    auto fetch = [&](long long n) {
        const char* x = C.x + ((n * positions + q) * C.x_stride + col) * X::SIZE;
        const char* dy = C.dy + ((n * positions + q) * C.dy_stride + col) * YB;
#pragma unroll
        for (int i = 0; i < I; ++i)
            if (i < mine) {
                ahead[i].load(x + i * x_step);
                d[i].load(dy + i * dy_step);
            }
    };
#pragma unroll
    for (int i = 0; i < I; ++i) ahead[i].clear(), d[i].clear();
    fetch(b / P.slabs);
    for (long long n = b / P.slabs; n < C.G.images; n += P.shares) {
#pragma unroll
        for (int i = 0; i < I; ++i) v[i] = ahead[i];
        const long long stat = n * C.G.groups + (long long)slab * P.whole;
        const OfGroups<V, FOLD> mean(C.mean + stat, c, C.columns), rstd(C.rstd + stat, c, C.columns);
        // a = (x - mean) wr + bias; the sums are of da (x - mean), rstd comes to them at the end
        float da[I][V], wr[V];
#pragma unroll
        for (int k = 0; k < V; ++k) wr[k] = w[k] * rstd[k];
        {
            float s1[V], s2[V];
#pragma unroll
            for (int k = 0; k < V; ++k) s1[k] = s2[k] = 0.0f;
#pragma unroll
            for (int i = 0; i < I; ++i)
                if (i < mine)  // (past the last position mean * rstd alone, which may be out of range, would make a NaN)
#pragma unroll
                    for (int k = 0; k < V; ++k) {
                        const float off = v[i].value(k) - mean[k];
                        da[i][k] = d[i].value(k) * act_slope(C.G.act, __builtin_fmaf(off, wr[k], bias[k]));
                        s1[k] = __builtin_fmaf(da[i][k], off, s1[k]);
                        s2[k] += da[i][k];
                    }
#pragma unroll
            for (int k = 0; k < V; ++k) s1[k] *= rstd[k];
            if (q < P.rows) {
                put_columns<V>(lds + q * P.slab + c * V, s1);
                put_columns<V>(lds + cells + q * P.slab + c * V, s2);
            }
        }
        if (n + P.shares < C.G.images) fetch(n + P.shares);
        __syncthreads();
        for (int t = threadIdx.x; t < 2 * P.slab; t += P.threads) {
            const float* of = lds + (t < P.slab ? t : cells + t - P.slab);
            float s = 0.0f;
#pragma unroll 8
            for (int r = 0; r < P.rows; ++r) s += of[r * P.slab];
            column[t] = s;
            over[t] += s;
        }
        __syncthreads();
        for (int g = threadIdx.x >> 6; g < 2 * P.whole; g += waves) {
            const int which = g >= P.whole, first = (which ? g - P.whole : g) * C.columns;
            float s = 0.0f;
            for (int t = lane; t < C.columns; t += 64) {
                const float wt = C.weight != nullptr ? C.weight[(long long)slab * P.slab + first + t] : 1.0f;
                s = __builtin_fmaf(wt, column[which * P.slab + first + t], s);
            }
            s = lanes_sum(s, 64);
            if (lane == 0) total[g] = s * m;
        }
        __syncthreads();
        const OfGroups<V, FOLD> m1(total, c, C.columns), m2(total + P.whole, c, C.columns);
        float c1[FOLD ? 1 : V], c2[FOLD ? 1 : V];
#pragma unroll
        for (int k = 0; k < (FOLD ? 1 : V); ++k) c1[k] = -(rstd[k] * rstd[k]) * m1[k], c2[k] = -rstd[k] * m2[k];
        char* dx = C.out + ((n * positions + q) * C.out_stride + col) * YB;
#pragma unroll
        for (int i = 0; i < I; ++i) {
            v[i].hold();
            if (i < mine) {
                float f[V];
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    const float rest = __builtin_fmaf(v[i].value(k) - mean[k], c1[FOLD ? 0 : k], c2[FOLD ? 0 : k]);
                    f[k] = __builtin_fmaf(da[i][k], wr[k], rest);
                }
                store_values<YD, V>(dx + i * out_step, f);
            }
        }
    }
    if (C.partial == nullptr) return;
    __syncthreads();
    float* to = C.partial + b / P.slabs * 2 * C.G.width + (long long)slab * P.slab;
    for (int t = threadIdx.x; t < 2 * P.slab; t += P.threads)
        to[t < P.slab ? t : (long long)C.G.width + t - P.slab] = over[t];
}

// ---------------------------------------------------------------------------------------- two passes
// Which work a workgroup does: an image's share of positions of a slab
struct Share2 {
    long long n, first, end;
    int slab, width, share;  // (the slab's columns, its last one's may be fewer)
    long long col;           // the slab's first column
};
__device__ __forceinline__ Share2 share_of(const GroupCall& C, long long b)
{
    const GroupPlan& P = C.P;
    Share2 s;
    s.slab = (int)(b % P.slabs);
    const long long rest = b / P.slabs;
    s.share = (int)(rest % P.shares);
    s.n = rest / P.shares;
    s.first = s.share * P.per;
    s.end = s.first + P.per < C.G.positions ? s.first + P.per : C.G.positions;
    if (P.whole > 0) {
        s.col = (long long)s.slab * P.slab;
        s.width = P.slab;
    } else {
        const int part = s.slab % P.parts;
        s.col = (long long)(s.slab / P.parts) * C.columns + (long long)part * P.slab;
        s.width = part + 1 < P.parts ? P.slab : C.columns - part * P.slab;
    }
    return s;
}

// partial[image][group][share][part][2]: mean and sum of squared distances from it
// (64 images of 1024 positions of 864 fp32 values, 226 MB: 35 us here, some of it from the cache behind HBM, 75 us to apply them)
template <int XD, int V>
__global__ void __launch_bounds__(SHARED) group_stats_kernel(GroupCall C)
{
    extern __shared__ float lds[];  // [2][rows][slab], [2][slab]
    const GroupPlan& P = C.P;
    typedef Packed<XD, V> X;
    const int q = threadIdx.x / P.vecs, c = threadIdx.x - q * P.vecs, cells = P.rows * P.slab;
    float* column = lds + 2 * cells;
    const int lane = threadIdx.x & 63, waves = P.threads >> 6;
    for (long long b = blockIdx.x; b < P.blocks; b += gridDim.x) {
        const Share2 S = share_of(C, by_xcd(b, P.blocks));
        const bool works = q < P.rows && c * V < S.width;
        const char* x = C.x + ((S.n * C.G.positions + S.first) * C.x_stride + S.col + c * V) * X::SIZE;
        const int count = (int)(S.end - S.first);
        float shift[V], s1[V], s2[V];
#pragma unroll
        for (int k = 0; k < V; ++k) shift[k] = s1[k] = s2[k] = 0.0f;
        if (works && q < count) {
            X v;
            v.load(x + q * C.x_stride * X::SIZE);
#pragma unroll
            for (int k = 0; k < V; ++k) shift[k] = v.value(k);
            // The mean so far takes the first value's place after 8, 64, 512, ... values: where the first is far from the others, the squares
            // of those distances, one for each value, would cost the sum its digits (rstd of 2048 images of 4096 positions of 64 fp32
            // values, the first positions' 1000 away: 434 fp32 roundings off without this, 3 with it, in the same time).
            const int values = (count - q + P.rows - 1) / P.rows;
            for (int first = 0, end = 8; first < values; first = end, end = end < (1 << 26) ? end * 8 : values) {
                const int upto = end < values ? end : values;
#pragma unroll 4
                for (int j = first; j < upto; ++j) {
                    v.load(x + (q + (long long)j * P.rows) * C.x_stride * X::SIZE);
#pragma unroll
                    for (int k = 0; k < V; ++k) {
                        const float d = v.value(k) - shift[k];
                        s1[k] += d;
                        s2[k] = __builtin_fmaf(d, d, s2[k]);
                    }
                }
                const float inv = 1.0f / (float)upto;
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    const float off = s1[k] * inv, to = shift[k] + off;
                    s2[k] = __builtin_fmaxf(__builtin_fmaf(-s1[k], off, s2[k]), 0.0f);
                    s1[k] = (off - (to - shift[k])) * (float)upto;  // (what rounding the place left of it)
                    shift[k] = to;
                }
            }
#pragma unroll
            for (int k = 0; k < V; ++k) {
                lds[q * P.slab + c * V + k] = shift[k];
                lds[cells + q * P.slab + c * V + k] = s2[k];
            }
        }
        __syncthreads();
        // columns: the lanes' means and squares joined
        const int held = count < P.rows ? count : P.rows;
        for (int t = threadIdx.x; t < S.width; t += P.threads) {
            const float about = lds[t];
            float a = 0.0f, d = 0.0f;
            for (int r = 1; r < held; ++r)
                a = __builtin_fmaf((float)((count - r + P.rows - 1) / P.rows), lds[r * P.slab + t] - about, a);
            const float mean = about + a / (float)count;
            for (int r = 0; r < held; ++r) {
                const float off = lds[r * P.slab + t] - mean;
                d += __builtin_fmaf((float)((count - r + P.rows - 1) / P.rows) * off, off, lds[cells + r * P.slab + t]);
            }
            column[t] = mean;
            column[P.slab + t] = d;
        }
        __syncthreads();
        const int groups = P.whole > 0 ? P.whole : 1, columns = P.whole > 0 ? C.columns : S.width;
        for (int g = threadIdx.x >> 6; g < groups; g += waves) {
            float s = 0.0f;
            // (about the first column's mean, for the same reason)
            const float about = column[g * columns];
            for (int t = lane; t < columns; t += 64) s += column[g * columns + t] - about;
            const float mean = about + lanes_sum(s, 64) / (float)columns;
            s = 0.0f;
            for (int t = lane; t < columns; t += 64) {
                const float d = column[g * columns + t] - mean;
                s += __builtin_fmaf((float)count * d, d, column[P.slab + g * columns + t]);
            }
            s = lanes_sum(s, 64);
            const long long group = P.whole > 0 ? (long long)S.slab * P.whole + g : S.slab / P.parts;
            const int part = P.whole > 0 ? 0 : S.slab % P.parts;
            float* to = C.partial + (((S.n * C.G.groups + group) * P.shares + S.share) * P.parts + part) * 2;
            if (lane == 0) to[0] = mean, to[1] = s;
        }
        __syncthreads();
    }
}

// joins the shares of a group: a wave for each
__global__ void __launch_bounds__(256) group_join_kernel(GroupCall C, float* mean_to, float* rstd_to)
{
    const GroupPlan& P = C.P;
    const int lane = threadIdx.x & 63;
    const long long many = C.G.images * C.G.groups;
    for (long long g = blockIdx.x * 4ll + (threadIdx.x >> 6); g < many; g += gridDim.x * 4ll) {
        const float* from = C.partial + g * P.shares * P.parts * 2;
        const int entries = (int)(P.shares * P.parts);
        auto count = [&](int e) {
            const long long share = e / P.parts, part = e % P.parts;
            const long long left = C.G.positions - share * P.per;
            const int cols = P.whole > 0 || part + 1 < P.parts ? (P.whole > 0 ? C.columns : P.slab)
                                                               : C.columns - (int)part * P.slab;
            return (float)(left < P.per ? left : P.per) * (float)cols;
        };
        const float m = 1.0f / ((float)C.G.positions * (float)C.columns), about = from[0];
        float s = 0.0f;
        for (int e = lane; e < entries; e += 64) s += count(e) * (from[2 * e] - about);
        const float mean = about + lanes_sum(s, 64) * m;
        s = 0.0f;
        for (int e = lane; e < entries; e += 64) {
            const float d = from[2 * e] - mean;
            s += __builtin_fmaf(count(e) * d, d, from[2 * e + 1]);
        }
        s = lanes_sum(s, 64) * m;
        if (lane == 0) {
            mean_to[g] = mean;
            rstd_to[g] = 1.0f / __builtin_sqrtf(s + C.G.eps);
        }
    }
}

template <int XD, int YD, int V>
__global__ void __launch_bounds__(SHARED) group_apply_kernel(GroupCall C)
{
    const GroupPlan& P = C.P;
    typedef Packed<XD, V> X;
    constexpr int YB = YD == CAPSCAPS_FP32 ? 4 : 2;
    const int q = threadIdx.x / P.vecs, c = threadIdx.x - q * P.vecs;
    for (long long b = blockIdx.x; b < P.blocks; b += gridDim.x) {
        // (last work first: what the pass before read last is still near)
        const Share2 S = share_of(C, by_xcd(P.blocks - 1 - b, P.blocks));
        if (q >= P.rows || c * V >= S.width) continue;
        const long long at = (S.n * C.G.positions + S.first), col = S.col + c * V;
        const char* x = C.x + (at * C.x_stride + col) * X::SIZE;
        char* y = C.out + (at * C.out_stride + col) * YB;
        const int count = (int)(S.end - S.first);
        float mean[V], scale[V], bias[V];
        load_columns<V>(scale, C.weight, col, 1.0f);
        load_columns<V>(bias, C.bias, col, 0.0f);
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const long long g = S.n * C.G.groups + (col + k) / C.columns;
            mean[k] = C.mean[g];
            scale[k] *= C.rstd[g];
        }
#pragma unroll 4
        for (int p = q; p < count; p += P.rows) {
            X v;
            v.load(x + p * C.x_stride * X::SIZE);
            float f[V];
#pragma unroll
            for (int k = 0; k < V; ++k)
                f[k] = act_value(C.G.act, __builtin_fmaf(v.value(k) - mean[k], scale[k], bias[k]));
            store_values<YD, V>(y + p * C.out_stride * YB, f);
        }
    }
}

// partial[image][share][2][width]: sums of da * xn and of da over the share's positions
// (16 images of 1024 positions of 16384 fp16 values: 194 us for 1.07 GB here, 305 for 1.6 GB in group_bwd_apply_kernel, 5.3 to 5.5 TB/s)
template <int XD, int YD, int V>
__global__ void __launch_bounds__(SHARED) group_sums_kernel(GroupCall C)
{
    extern __shared__ float lds[];  // [2][rows][slab]
    const GroupPlan& P = C.P;
    typedef Packed<XD, V> X;
    typedef Packed<YD, V> Y;
    const int q = threadIdx.x / P.vecs, c = threadIdx.x - q * P.vecs, cells = P.rows * P.slab;
    for (long long b = blockIdx.x; b < P.blocks; b += gridDim.x) {
        const Share2 S = share_of(C, by_xcd(b, P.blocks));
        if (q < P.rows && c * V < S.width) {
            const long long at = (S.n * C.G.positions + S.first), col = S.col + c * V;
            const char* x = C.x + (at * C.x_stride + col) * X::SIZE;
            const char* dy = C.dy + (at * C.dy_stride + col) * Y::SIZE;
            const int count = (int)(S.end - S.first);
            float mean[V], rstd[V], w[V], bias[V], s1[V], s2[V];
            load_columns<V>(w, C.weight, col, 1.0f);
            load_columns<V>(bias, C.bias, col, 0.0f);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const long long g = S.n * C.G.groups + (col + k) / C.columns;
                mean[k] = C.mean[g], rstd[k] = C.rstd[g], s1[k] = s2[k] = 0.0f;
            }
#pragma unroll 4
            for (int p = q; p < count; p += P.rows) {
                X v;
                Y d;
                v.load(x + p * C.x_stride * X::SIZE);
                d.load(dy + p * C.dy_stride * Y::SIZE);
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    const GroupBack g = group_back(C.G.act, v.value(k), d.value(k), mean[k], rstd[k], w[k], bias[k]);
                    s1[k] = __builtin_fmaf(g.da, g.xn, s1[k]);
                    s2[k] += g.da;
                }
            }
#pragma unroll
            for (int k = 0; k < V; ++k) {
                lds[q * P.slab + c * V + k] = s1[k];
                lds[cells + q * P.slab + c * V + k] = s2[k];
            }
        }
        __syncthreads();
        float* to = C.partial + (S.n * P.shares + S.share) * 2 * C.G.width + S.col;
        for (int t = threadIdx.x; t < 2 * S.width; t += P.threads) {
            const int which = t >= S.width, k = which ? t - S.width : t;
            float s = 0.0f;
            for (int r = 0; r < P.rows; ++r) s += lds[which * cells + r * P.slab + k];
            to[which * (long long)C.G.width + k] = s;
        }
        __syncthreads();
    }
}

// means over a group of da * weight * xn and of da * weight: means[group of an image][2]
__global__ void __launch_bounds__(SHARED) group_means_kernel(GroupCall C, float* means)
{
    __shared__ float lds[2][SHARED / 64];
    const GroupPlan& P = C.P;
    const long long many = C.G.images * C.G.groups;
    const float m = 1.0f / ((float)C.G.positions * (float)C.columns);
    for (long long ng = blockIdx.x; ng < many; ng += gridDim.x) {
        const long long n = ng / C.G.groups, first = ng % C.G.groups * C.columns;
        float s[2] = {0.0f, 0.0f};
        for (long long share = 0; share < P.shares; ++share) {
            const float* from = C.partial + (n * P.shares + share) * 2 * C.G.width + first;
            for (int t = threadIdx.x; t < C.columns; t += SHARED) {
                const float w = C.weight != nullptr ? C.weight[first + t] : 1.0f;
                s[0] = __builtin_fmaf(w, from[t], s[0]);
                s[1] = __builtin_fmaf(w, from[(long long)C.G.width + t], s[1]);
            }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            s[k] = lanes_sum(s[k], 64);
            if ((threadIdx.x & 63) == 0) lds[k][threadIdx.x >> 6] = s[k];
        }
        __syncthreads();
        if (threadIdx.x < 2) {
            float t = 0.0f;
            for (int k = 0; k < SHARED / 64; ++k) t += lds[threadIdx.x][k];
            means[ng * 2 + threadIdx.x] = t * m;
        }
        __syncthreads();
    }
}

template <int XD, int YD, int V>
__global__ void __launch_bounds__(SHARED) group_bwd_apply_kernel(GroupCall C, const float* means)
{
    const GroupPlan& P = C.P;
    typedef Packed<XD, V> X;
    typedef Packed<YD, V> Y;
    const int q = threadIdx.x / P.vecs, c = threadIdx.x - q * P.vecs;
    for (long long b = blockIdx.x; b < P.blocks; b += gridDim.x) {
        const Share2 S = share_of(C, by_xcd(P.blocks - 1 - b, P.blocks));
        if (q >= P.rows || c * V >= S.width) continue;
        const long long at = (S.n * C.G.positions + S.first), col = S.col + c * V;
        const char* x = C.x + (at * C.x_stride + col) * X::SIZE;
        const char* dy = C.dy + (at * C.dy_stride + col) * Y::SIZE;
        char* dx = C.out + (at * C.out_stride + col) * Y::SIZE;
        const int count = (int)(S.end - S.first);
        float mean[V], rstd[V], w[V], bias[V], s1[V], s2[V];
        load_columns<V>(w, C.weight, col, 1.0f);
        load_columns<V>(bias, C.bias, col, 0.0f);
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const long long g = S.n * C.G.groups + (col + k) / C.columns;
            mean[k] = C.mean[g], rstd[k] = C.rstd[g], s1[k] = means[g * 2], s2[k] = means[g * 2 + 1];
        }
#pragma unroll 4
        for (int p = q; p < count; p += P.rows) {
            X v;
            Y d;
            v.load(x + p * C.x_stride * X::SIZE);
            d.load(dy + p * C.dy_stride * Y::SIZE);
            float f[V];
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const GroupBack g = group_back(C.G.act, v.value(k), d.value(k), mean[k], rstd[k], w[k], bias[k]);
                f[k] = rstd[k] * (__builtin_fmaf(g.da, w[k], -s2[k]) - g.xn * s1[k]);
            }
            store_values<YD, V>(dx + p * C.out_stride * Y::SIZE, f);
        }
    }
}

// dweight, dbias: sums over the partial sums' rows, in their order; 64 columns a workgroup
__global__ void __launch_bounds__(1024) group_column_sums_kernel(const float* partial, long long rows, long long width,
                                                                 float* dweight, float* dbias)
{
    __shared__ float lds[16][64];
    float* to = blockIdx.y == 0 ? dweight : dbias;
    if (to == nullptr) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (long long first = blockIdx.x * 64ll; first < width; first += gridDim.x * 64ll) {
        const long long c = first + lane;
        float s = 0.0f;
        if (c < width)
            for (long long r = wave; r < rows; r += 16) s += partial[(r * 2 + blockIdx.y) * width + c];
        lds[wave][lane] = s;
        __syncthreads();
        if (wave == 0 && c < width) {
#pragma unroll
            for (int k = 1; k < 16; ++k) s += lds[k][lane];
            to[c] = s;
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------------------- host
int check_group(const capscaps_group_norm* g)
{
    if (g == nullptr || g->images < 1 || g->positions < 1 || g->width < 1 || g->groups < 1) return CAPSCAPS_EINVAL;
    if (g->width > (1 << 30) || g->width % g->groups != 0 || g->positions > (1ll << 30)) return CAPSCAPS_EINVAL;
    if (!known_dtype(g->dtype) || (g->x_dtype != CAPSCAPS_FP32 && g->x_dtype != g->dtype)) return CAPSCAPS_EINVAL;
    if (g->act < CAPSCAPS_ACT_LINEAR || g->act > CAPSCAPS_ACT_SILU) return CAPSCAPS_EINVAL;
    if (!(g->eps >= 1.17549435e-38f && g->eps <= 3.4e38f)) return CAPSCAPS_EINVAL;
    // (values, and shares of them, are counted in 64 bits)
    if (g->images > (1ll << 62) / g->width / g->positions) return CAPSCAPS_EINVAL;
    return CAPSCAPS_OK;
}

bool misaligned(const void* p, int dtype)
{
    return (reinterpret_cast<uintptr_t>(p) & (element_bytes(dtype) - 1)) != 0;
}
bool bad_positions(const capscaps_group_norm& G, const void* p, long long stride, int dtype, bool output)
{
    if (p == nullptr || misaligned(p, dtype)) return true;
    if (stride < 0 || stride > (1ll << 40)) return true;
    return output && G.images * G.positions > 1 && stride < G.width;
}

int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }

// Vectors of a lane that the resident kernels are built for
template <bool FORWARD>
int resident_items(int v, int widest, long long need)
{
    for (const int i : {2, 4, 8, 16}) {
        const bool built = v == widest ? i <= (FORWARD ? 16 : 8) : i == 8;
        if (built && need <= i) return i;
    }
    return 0;
}

template <bool FORWARD>
GroupPlan group_plan(const capscaps_group_norm& G)
{
    GroupPlan P{};
    const int columns = G.width / G.groups, widest = G.x_dtype == CAPSCAPS_FP32 ? 4 : 8;
    const int size = G.x_dtype == CAPSCAPS_FP32 ? 4 : 2;
    auto vector = [&](long long cols) { return cols % widest == 0 ? widest : cols % 2 == 0 ? 2 : 1; };
    // Resident: the fewest whole groups whose vectors are whole and whose rows fill a line of memory; more of them
    // where an image's positions leave lanes without work.
    int k = 1;
    for (; k < G.groups; ++k) {
        if (G.groups % k != 0) continue;
        const long long slab = (long long)k * columns;
        if (vector(slab) == widest && slab * size >= 128 && slab / widest * G.positions >= 256) break;
    }
    const long long wide = (long long)k * columns;
    const long long most = FORWARD ? RESIDENT : RESIDENT_BACK / 4;  // vectors (backward: sums of 1024 columns in LDS)
    if (wide / vector(wide) <= most) {
        const int v = vector(wide);
        const long long vecs = wide / v;
        // As few lanes, in whole waves, as hold the slab: more workgroups of a CU then read and write at a time while others
        // compute.  Where there are few workgroups, as many lanes as there are vectors.
        int threads = FORWARD ? RESIDENT : RESIDENT_BACK;
        const bool few = G.images * (G.groups / k) < 2 * CUS;
        const int aim = few ? 2 : v == widest ? (FORWARD ? 16 : 8) : 8;
        while (threads > 64 && threads / 2 >= vecs && ceil_div(G.positions, threads / 2 / vecs) <= aim) threads /= 2;
        const int rows = threads / (int)vecs;
        const int items = resident_items<FORWARD>(v, widest, ceil_div(G.positions, rows));
        // Where vectors straddle groups, a slab that takes a CU's registers for itself waits for its sums by columns alone: 64
        // images of 1024 positions of 32 groups of 30 columns take 144 us in fp32 and 92 in bf16, in two passes 120 and 73;
        // with half the positions, two slabs a CU, 71 and 42, in two passes 65 and 46.
        const bool alone = FORWARD && !few && columns % v != 0 && threads * items > RESIDENT * 8;
        const long long room = ((1ll << 32) - 1) / threads;  // workgroups: a launch has less than 2^32 threads
        if (items > 0 && !alone && G.groups / k <= room) {
            P.v = v, P.items = items, P.threads = threads, P.rows = rows, P.vecs = (int)vecs, P.slab = (int)wide;
            P.whole = k, P.parts = 1, P.slabs = G.groups / k, P.fold = columns % v == 0 ? v : 1;
            // (backward: a workgroup takes one image after the other, and as many lanes as the registers of a CU hold are at work)
            const long long blocks = FORWARD ? std::min<long long>(MOST_BLOCKS, room) : CUS * (RESIDENT_BACK / threads) * (items == 8 ? 1 : 2);
            P.shares = std::max<long long>(1, std::min<long long>(G.images, blocks / P.slabs));
            P.blocks = P.shares * P.slabs;
            return P;
        }
    }
    // Two passes
    P.threads = SHARED;
    P.v = vector(columns);
    const long long vecs = columns / P.v;
    if (vecs > SHARED) {
        P.whole = 0, P.vecs = SHARED, P.slab = SHARED * P.v, P.parts = ceil_div(columns, P.slab);
        P.slabs = G.groups * P.parts;
    } else {
        int k = 1;
        for (int j = 1; j <= G.groups && (long long)j * columns / vector((long long)j * columns) <= SHARED; ++j) {
            if (G.groups % j != 0) continue;
            k = j;
            if (vector((long long)j * columns) == widest && (long long)j * columns * size >= 512) break;
        }
        P.v = vector((long long)k * columns);
        P.whole = k, P.parts = 1, P.slab = k * columns, P.vecs = P.slab / P.v, P.slabs = G.groups / k;
    }
    P.fold = columns % P.v == 0 ? P.v : 1;
    P.rows = SHARED / P.vecs;
    const long long lanes = (long long)P.slabs * G.images;
    const long long wanted = std::max<long long>(1, (8 * CUS + lanes - 1) / lanes);
    P.per = std::max<long long>((G.positions + wanted - 1) / wanted, std::min<long long>(G.positions, 8ll * P.rows));
    P.shares = (G.positions + P.per - 1) / P.per;
    P.blocks = P.shares * P.slabs * G.images;
    return P;
}

template <bool FORWARD>
size_t group_lds(const GroupPlan& P)
{
    if (P.items > 0) {
        if (FORWARD) return ((size_t)P.rows * P.vecs * (P.fold == P.v ? 1 : P.v) + P.whole) * 4;
        return ((size_t)2 * P.rows * P.slab + 4 * P.slab + 2 * P.whole) * 4;
    }
    return ((size_t)2 * P.rows * P.slab + 2 * P.slab) * 4;
}

template <bool FORWARD>
size_t group_workspace(const capscaps_group_norm& G, const GroupPlan& P)
{
    const size_t stats = ((size_t)G.images * G.groups * 8 + 255) / 256 * 256;
    if (FORWARD) return P.items > 0 ? 0 : stats + (size_t)G.images * G.groups * P.shares * P.parts * 8;
    if (P.items > 0) return (size_t)P.shares * 2 * G.width * 4;
    return stats + (size_t)G.images * P.shares * 2 * G.width * 4;
}

unsigned grid_of(long long blocks) { return (unsigned)std::min<long long>(blocks, MOST_BLOCKS); }

template <int N>
using Int = std::integral_constant<int, N>;

// calls f with x's type, the layers' type and a vector's columns as compile-time numbers
template <typename F>
void with_types(const capscaps_group_norm& G, const GroupPlan& P, F f)
{
    auto by_vector = [&](auto xd, auto yd) {
        constexpr int widest = xd.value == CAPSCAPS_FP32 ? 4 : 8;
        if (P.v == widest)
            f(xd, yd, Int<widest>());
        else if (P.v == 2)
            f(xd, yd, Int<2>());
        else
            f(xd, yd, Int<1>());
    };
    auto by_x = [&](auto yd) {
        if (G.x_dtype == CAPSCAPS_FP32)
            by_vector(Int<CAPSCAPS_FP32>(), yd);
        else
            by_vector(yd, yd);
    };
    if (G.dtype == CAPSCAPS_FP32)
        by_x(Int<CAPSCAPS_FP32>());
    else if (G.dtype == CAPSCAPS_BF16)
        by_x(Int<CAPSCAPS_BF16>());
    else
        by_x(Int<CAPSCAPS_FP16>());
}

template <typename K>
hipError_t launch_resident(K kernel, const GroupCall& C, size_t lds, hipStream_t st)
{
    kernel<<<dim3((unsigned)C.P.blocks), dim3(C.P.threads), lds, st>>>(C);
    return hipGetLastError();
}

template <bool FORWARD>
hipError_t run_resident(const GroupCall& C, hipStream_t st)
{
    hipError_t err = hipErrorInvalidValue;
    const size_t lds = group_lds<FORWARD>(C.P);
    with_types(C.G, C.P, [&](auto xd, auto yd, auto v) {
        constexpr int X = xd.value, Y = yd.value, V = v.value;
        auto folded = [&](auto i, auto fold) {
            if constexpr (FORWARD)
                err = launch_resident(group_fwd_resident_kernel<X, Y, V, i.value, fold.value>, C, lds, st);
            else
                err = launch_resident(group_bwd_resident_kernel<X, Y, V, i.value, fold.value>, C, lds, st);
        };
        auto with = [&](auto i) {
            if constexpr (V == 1)
                folded(i, std::true_type());
            else
                C.P.fold == V ? folded(i, std::true_type()) : folded(i, std::false_type());
        };
        if constexpr (V > 2) {
            if (C.P.items == 2) with(Int<2>());
            if (C.P.items == 4) with(Int<4>());
            if (C.P.items == 8) with(Int<8>());
            if constexpr (FORWARD)
                if (C.P.items == 16) with(Int<16>());
        } else {
            with(Int<8>());
        }
    });
    return err;
}

}  // namespace
}  // namespace capscaps

using namespace capscaps;

extern "C" {

// (for tests) the plan of one direction: workgroups and threads of the launch that takes most of them, and 1 where values stay in
// registers, 0 where they are read twice; 0: an invalid norm
int capscaps_testing_group_norm_launch(const capscaps_group_norm* norm, int forward, long long* blocks_threads_resident)
{
    if (check_group(norm) != CAPSCAPS_OK) return 0;
    const GroupPlan P = forward ? group_plan<true>(*norm) : group_plan<false>(*norm);
    blocks_threads_resident[0] = P.items > 0 ? P.blocks : grid_of(P.blocks);
    blocks_threads_resident[1] = P.threads;
    blocks_threads_resident[2] = P.items > 0;
    return 1;
}

size_t capscaps_group_norm_fwd_workspace_bytes(const capscaps_group_norm* norm)
{
    if (check_group(norm) != CAPSCAPS_OK) return 0;
    return group_workspace<true>(*norm, group_plan<true>(*norm));
}

size_t capscaps_group_norm_bwd_workspace_bytes(const capscaps_group_norm* norm)
{
    if (check_group(norm) != CAPSCAPS_OK) return 0;
    return group_workspace<false>(*norm, group_plan<false>(*norm));
}

int capscaps_group_norm_fwd(const capscaps_group_norm* norm, const capscaps_group_fwd_args* args, void* workspace,
                            size_t workspace_bytes, void* stream)
{
    const int rc = check_group(norm);
    if (rc != CAPSCAPS_OK) return rc;
    if (args == nullptr) return CAPSCAPS_EINVAL;
    const capscaps_group_norm& G = *norm;
    const capscaps_group_fwd_args& A = *args;
    if (bad_positions(G, A.x, A.x_stride, G.x_dtype, false) || bad_positions(G, A.y, A.y_stride, G.dtype, true))
        return CAPSCAPS_EINVAL;
    if (A.y == A.x && (A.y_stride != A.x_stride || G.x_dtype != G.dtype)) return CAPSCAPS_EINVAL;
    for (const float* p : {A.weight, A.bias, (const float*)A.mean, (const float*)A.rstd})
        if (misaligned(p, CAPSCAPS_FP32)) return CAPSCAPS_EINVAL;
    const GroupPlan P = group_plan<true>(G);
    const size_t need = group_workspace<true>(G, P);
    if (need > 0 && (workspace == nullptr || workspace_bytes < need)) return CAPSCAPS_EWORKSPACE;
    if (need > 0 && (reinterpret_cast<uintptr_t>(workspace) & 15u) != 0) return CAPSCAPS_EINVAL;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    GroupCall C{G, P, G.width / G.groups, static_cast<const char*>(A.x), nullptr, static_cast<char*>(A.y), A.weight,
                A.bias, A.mean, A.rstd, A.x_stride, 0, A.y_stride, nullptr};
    if (P.items > 0) return status_from_hip(run_resident<true>(C, st));
    const long long many = G.images * G.groups;
    float* stats = static_cast<float*>(workspace);
    C.partial = stats + (many * 8 + 255) / 256 * 64;
    if (C.mean == nullptr) C.mean = stats;
    if (C.rstd == nullptr) C.rstd = stats + many;
    const unsigned grid = grid_of(P.blocks);
    with_types(G, P, [&](auto xd, auto, auto v) {
        group_stats_kernel<xd.value, v.value><<<dim3(grid), dim3(SHARED), group_lds<true>(P), st>>>(C);
    });
    hipError_t err = hipGetLastError();
    if (err != hipSuccess) return status_from_hip(err);
    group_join_kernel<<<dim3(grid_of((many + 3) / 4)), dim3(256), 0, st>>>(C, C.mean, C.rstd);
    err = hipGetLastError();
    if (err != hipSuccess) return status_from_hip(err);
    with_types(G, P, [&](auto xd, auto yd, auto v) {
        group_apply_kernel<xd.value, yd.value, v.value><<<dim3(grid), dim3(SHARED), 0, st>>>(C);
    });
    return status_from_hip(hipGetLastError());
}

int capscaps_group_norm_bwd(const capscaps_group_norm* norm, const capscaps_group_bwd_args* args, void* workspace,
                            size_t workspace_bytes, void* stream)
{
    const int rc = check_group(norm);
    if (rc != CAPSCAPS_OK) return rc;
    if (args == nullptr) return CAPSCAPS_EINVAL;
    const capscaps_group_norm& G = *norm;
    const capscaps_group_bwd_args& A = *args;
    if (bad_positions(G, A.x, A.x_stride, G.x_dtype, false) || bad_positions(G, A.dy, A.dy_stride, G.dtype, false) ||
        bad_positions(G, A.dx, A.dx_stride, G.dtype, true))
        return CAPSCAPS_EINVAL;
    if (A.dx == A.x) return CAPSCAPS_EINVAL;
    if (A.dx == A.dy && A.dx_stride != A.dy_stride) return CAPSCAPS_EINVAL;
    if (A.mean == nullptr || A.rstd == nullptr) return CAPSCAPS_EINVAL;
    for (const float* p : {A.weight, A.bias, A.mean, A.rstd, (const float*)A.dweight, (const float*)A.dbias})
        if (misaligned(p, CAPSCAPS_FP32)) return CAPSCAPS_EINVAL;
    const GroupPlan P = group_plan<false>(G);
    const bool sums = A.dweight != nullptr || A.dbias != nullptr;
    const size_t need = sums || P.items == 0 ? group_workspace<false>(G, P) : 0;
    if (need > 0 && (workspace == nullptr || workspace_bytes < need)) return CAPSCAPS_EWORKSPACE;
    if (need > 0 && (reinterpret_cast<uintptr_t>(workspace) & 15u) != 0) return CAPSCAPS_EINVAL;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    GroupCall C{G, P, G.width / G.groups, static_cast<const char*>(A.x), static_cast<const char*>(A.dy),
                static_cast<char*>(A.dx), A.weight, A.bias, const_cast<float*>(A.mean), const_cast<float*>(A.rstd),
                A.x_stride, A.dy_stride, A.dx_stride, nullptr};
    long long rows = P.shares;
    hipError_t err;
    if (P.items > 0) {
        C.partial = sums ? static_cast<float*>(workspace) : nullptr;
        err = run_resident<false>(C, st);
        if (err != hipSuccess) return status_from_hip(err);
    } else {
        const long long many = G.images * G.groups;
        float* means = static_cast<float*>(workspace);
        C.partial = means + (many * 8 + 255) / 256 * 64;
        rows = G.images * P.shares;
        const unsigned grid = grid_of(P.blocks);
        with_types(G, P, [&](auto xd, auto yd, auto v) {
            group_sums_kernel<xd.value, yd.value, v.value>
                <<<dim3(grid), dim3(SHARED), group_lds<false>(P), st>>>(C);
        });
        err = hipGetLastError();
        if (err != hipSuccess) return status_from_hip(err);
        group_means_kernel<<<dim3(grid_of(many)), dim3(SHARED), 0, st>>>(C, means);
        err = hipGetLastError();
        if (err != hipSuccess) return status_from_hip(err);
        with_types(G, P, [&](auto xd, auto yd, auto v) {
            group_bwd_apply_kernel<xd.value, yd.value, v.value><<<dim3(grid), dim3(SHARED), 0, st>>>(C, means);
        });
        err = hipGetLastError();
        if (err != hipSuccess) return status_from_hip(err);
    }
    if (!sums) return CAPSCAPS_OK;
    group_column_sums_kernel<<<dim3(std::min((G.width + 63) / 64, 1 << 20), 2), dim3(1024), 0, st>>>(C.partial, rows, G.width, A.dweight,
                                                                                 A.dbias);
    return status_from_hip(hipGetLastError());
}

}  // extern "C"
