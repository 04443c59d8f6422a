// The norms around a block of layers with its gate and residual stream, forward and backward.
// Formulas and contracts: include/capscaps.h.
//
// All of it is bounded by memory: some ten to thirty operations for every value moved.  So each value is read
// once and each result written once, with the row in registers between: a group of lanes holds a row in vectors
// (row_vectors.h), and the means are sums over the group.  Groups of up to 64 lanes share a wave and need no
// barrier; wider rows take a workgroup.  Rows that no group holds (over 16384 values) take the kernels at the
// end.
//
// Measured (us; the bytes that must be moved at 6.2 TB/s in parentheses): forward, 65536 rows of 864 fp32 values
// 155 (146), 6.4M rows of 64 bf16 values with a gate for each 667 (671), 65536 x 4096 bf16 376 (346); backward,
// 16384 x 4096 fp32 and bf16 230 (217), 16384 x 16384 fp16 591 (520), 2.1M x 27 fp32 with a gate 386 (295).
#include <hip/hip_runtime.h>
#include <float.h>
#include <math.h>
#include <stdint.h>

#include <initializer_list>
#include <type_traits>

#include "../../include/capscaps.h"
#include "conv_shape.h"
#include "element.h"
#include "row_vectors.h"

namespace capscaps {
namespace {

constexpr int THREADS = 256;
constexpr int CUS = 256;

// act(g) and its derivative (v_rcp_f32 is off by one unit in the last place)
struct Gate {
    float value, slope;
};
__device__ __forceinline__ Gate gate_both(int act, float g)
{
    if (act == CAPSCAPS_ACT_LINEAR) return {g, 1.0f};
    const float q = __builtin_amdgcn_rcpf(1.0f + __expf(-g));
    if (act == CAPSCAPS_ACT_SIGMOID) return {q, q * (1.0f - q)};
    return {g * q, q * (1.0f + g * (1.0f - q))};
}
__device__ __forceinline__ float gate_value(int act, float g) { return gate_both(act, g).value; }
__device__ __forceinline__ float gate_slope(int act, float g) { return gate_both(act, g).slope; }

// sum over the workgroup, in every thread
__device__ __forceinline__ float block_sum(float v, float* lds)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0f;
    for (int w = 0; w < THREADS / 64; ++w) v += lds[w];
    __syncthreads();
    return v;
}

// ------------------------------------------------------------------------------------ rows in registers
// How rows lie on lanes: `group` lanes (a power of two up to 64, or so many waves) hold a row, lane l the vectors l, l + group, ... of `vectors`
// a lane; `per_block` rows at a time in a workgroup of `threads`.
struct RowPlan {
    int n;  // values of a vector
    int group, vectors, threads, per_block;
    unsigned blocks;
    int full, tail;  // whole vectors in a row, and the values after them
    int part;        // the vector that those are in (-1: none)
    bool turns;      // more than one round of rows for a workgroup
};

constexpr int WIDEST = 16384;
// vectors of a lane: 1, 2 in workgroups of up to 1024; 4, 8 in such of 512, whose waves have twice the registers
constexpr int widest_workgroup(int vectors) { return vectors > 2 ? 512 : 1024; }
// (lanes of several vectors are those of a whole workgroup: known to the compiler, which then needs no register
// for every distance between them)
template <int I>
__device__ __forceinline__ int group_of(const RowPlan& P)
{
    return I > 1 ? widest_workgroup(I) : P.group;
}
// Sum over a row's lanes.  Rows of more than one wave go through LDS: two buffers in turn, so that one barrier
// is enough (a wave writes a buffer again only after the barrier of the other one, which every wave reaches
// after it has read).
struct RowSum {
    float* lds;  // [2][16]
    int group, slot, turn;
    __device__ __forceinline__ float operator()(float v)
    {
        if (group <= 64) return lanes_sum(v, group);
        v = lanes_sum(v, 64);
        float* buffer = lds + 16 * turn;
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) buffer[threadIdx.x >> 6] = v;
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
        // the waves of this row; every 16 lanes add up the same sums
        const int waves = group >> 6, wave = threadIdx.x & 15;
        v = wave < waves ? buffer[slot * waves + wave] : 0.0f;
        return lanes_sum(v, 16);
    }
};

// A tensor's rows as the lanes of a workgroup see them: where its rows of this round begin (the same for all
// lanes, so it stays in scalar registers), and a lane's place from there
template <int N>
struct Rows {
    const char* base;
    long long round;  // bytes of a workgroup's rows of one round
    unsigned at;
    // what follows a row, up to a vector, is the next row's or lies before it (it is masked: it may be written meanwhile)
    bool over;
    template <typename T>
    __device__ __forceinline__ Rows(T* p, long long stride, int bytes, const RowPlan& P, int slot, int lane)
    {
        base = (const char*)p;
        round = P.per_block * stride * bytes;
        over = stride >= N;
        at = (unsigned)(slot * stride * bytes) + (unsigned)(lane * N * bytes);
    }
    __device__ __forceinline__ const char* get(long long n, int vectors, int bytes) const
    {
        return base + n * round + (long long)(vectors * N * bytes) + at;
    }
    __device__ __forceinline__ char* put(long long n, int vectors, int bytes) const
    {
        return const_cast<char*>(get(n, vectors, bytes));
    }
};

// A vector of what a column's values are multiplied by, from pre-norm weight, post-norm weight and a shared gate
template <int N>
struct Factors {
    float to_b[N], to_h[N];
};
template <int N, bool TAIL>
__device__ __forceinline__ Factors<N> column_factors(const capscaps_block& B, const float* pre_weight,
                                                     const float* post_weight, const void* gate, const RowPlan& P, int v)
{
    Factors<N> f;
    const bool shared = B.gate == CAPSCAPS_GATE_SHARED;
    const Share has{v < P.full, TAIL && v == P.part, P.tail};
    load_column<N, TAIL>(f.to_b, post_weight, v, has, 1.0f);
    load_column<N, TAIL>(f.to_h, pre_weight, v, has, 1.0f);
    float g[N];
    load_column<N, TAIL>(g, shared ? static_cast<const float*>(gate) : nullptr, v, has, 1.0f);
#pragma unroll
    for (int k = 0; k < N; ++k) f.to_b[k] *= B.branch_scale * (shared ? gate_value(B.gate_act, g[k]) : 1.0f);
    return f;
}
// They are kept in registers where a lane has one vector.  Where it has more, registers are short (the sums over rows
// alone take 32), and they lie in LDS: a lane's own place, so nothing waits for another lane
template <int N, int I>
struct Columns {
    Factors<N> own;
    float* lds;
    int lane;
    __device__ __forceinline__ void put(int i, const Factors<N>& f)
    {
        if constexpr (I == 1) {
            own = f;
        } else {
#pragma unroll
            for (int k = 0; k < N; k += 4) {
                quad(0, i, k) = float4v_t{f.to_b[k], f.to_b[k + 1], f.to_b[k + 2], f.to_b[k + 3]};
                quad(1, i, k) = float4v_t{f.to_h[k], f.to_h[k + 1], f.to_h[k + 2], f.to_h[k + 3]};
            }
        }
    }
    __device__ __forceinline__ void to_b(int i, float* f) const { get(0, i, f, own.to_b); }
    __device__ __forceinline__ void to_h(int i, float* f) const { get(1, i, f, own.to_h); }

private:
    typedef float float4v_t __attribute__((ext_vector_type(4)));
    __device__ __forceinline__ float4v_t& quad(int which, int i, int k) const
    {
        return reinterpret_cast<float4v_t*>(lds)[((which * I + i) * (N / 4) + k / 4) * widest_workgroup(I) + lane];
    }
    __device__ __forceinline__ void get(int which, int i, float* f, const float* kept) const
    {
#pragma unroll
        for (int k = 0; k < N; k += 4) {
            if constexpr (I == 1) {
                for (int j = 0; j < 4; ++j) f[k + j] = kept[k + j];
            } else {
                const float4v_t q = quad(which, i, k);
                for (int j = 0; j < 4; ++j) f[k + j] = q[j];
            }
        }
    }
};

// GATE: a gate for every value.  TURNS: a workgroup takes one round of rows after another (else one round)
template <int DT, bool S16, bool B16, bool GATE, int N, int I, bool TAIL, bool TURNS>
__global__ void __launch_bounds__(widest_workgroup(I))
    block_fwd_kernel(capscaps_block B, capscaps_block_fwd_args A, RowPlan P)
{
    constexpr int SD = S16 ? DT : CAPSCAPS_FP32, BD = B16 ? DT : CAPSCAPS_FP32;
    constexpr int SB = S16 ? 2 : 4, BB = B16 ? 2 : 4, LB = DT == CAPSCAPS_FP32 ? 4 : 2;
    __shared__ float lds[32];
    const int group = group_of<I>(P);
    const int slot = threadIdx.x / group, lane = threadIdx.x - slot * group;
    RowSum sum{lds, group, slot, 0};
    const bool branch = A.branch != nullptr, post = branch && B.post_norm, pre = A.h != nullptr;
    const float inv_width = 1.0f / (float)B.width;
    Factors<N> col[I];
#pragma unroll
    for (int i = 0; i < I; ++i)
        col[i] = column_factors<N, TAIL>(B, A.pre_weight, post ? A.post_weight : nullptr, A.gate, P, lane + i * group);
    Rows<N> rx(A.x, A.x_stride, SB, P, slot, lane), rb(A.branch, A.branch_stride, BB, P, slot, lane);
    Rows<N> rg(A.gate, A.gate_stride, LB, P, slot, lane);
    Rows<N> ry(A.y, A.y_stride, SB, P, slot, lane), rh(A.h, A.h_stride, LB, P, slot, lane);
    const long long rounds = (B.rows + P.per_block - 1) / P.per_block;
    long long n = blockIdx.x;
    do {
        const long long r = n * P.per_block + slot;
        const bool in = r < B.rows, last = r + 1 >= B.rows;
        Raw<SD, N> x[I];
        Raw<BD, N> b[I];
        Raw<DT, N> g[I];
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int v = lane + i * group;
            const Share has{in && v < P.full, TAIL && in && v == P.part, P.tail};
            clear(x[i]);
            clear(b[i]);
            if (branch) load<BD, N, TAIL>(b[i], rb.get(n, i * group, BB), has, rb.over && !last);
            load<SD, N, TAIL>(x[i], rx.get(n, i * group, SB), has, rx.over && !last);
            if constexpr (GATE) {
                clear(g[i]);
                load<DT, N, TAIL>(g[i], rg.get(n, i * group, LB), has, rg.over && !last);
            }
        }
        float rpost = 1.0f;
        if (post) {
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < I; ++i)
#pragma unroll
                for (int k = 0; k < N; ++k) s += value<BD, N>(b[i], k) * value<BD, N>(b[i], k);
            rpost = __builtin_amdgcn_rsqf(sum(s) * inv_width + B.eps);
            if (A.rstd_post != nullptr && lane == 0 && in) A.rstd_post[r] = rpost;
        }
        float y[I][N];
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int v = lane + i * group;
            const Share has{in && v < P.full, TAIL && in && v == P.part, P.tail};
#pragma unroll
            for (int k = 0; k < N; ++k) {
                y[i][k] = value<SD, N>(x[i], k);
                if (branch) {
                    float u = value<BD, N>(b[i], k) * rpost * col[i].to_b[k];
                    if constexpr (GATE) u *= gate_value(B.gate_act, value<DT, N>(g[i], k));
                    y[i][k] = B.residual_scale * y[i][k] + u;
                }
                s += y[i][k] * y[i][k];
            }
            if (A.y != nullptr) store<SD, N, TAIL>(ry.put(n, i * group, SB), y[i], has);
        }
        if (pre) {
            const float rpre = __builtin_amdgcn_rsqf(sum(s) * inv_width + B.eps);
            if (A.rstd_pre != nullptr && lane == 0 && in) A.rstd_pre[r] = rpre;
#pragma unroll
            for (int i = 0; i < I; ++i) {
                const int v = lane + i * group;
                const Share has{in && v < P.full, TAIL && in && v == P.part, P.tail};
                float h[N];
#pragma unroll
                for (int k = 0; k < N; ++k) h[k] = y[i][k] * rpre * col[i].to_h[k];
                store<DT, N, TAIL>(rh.put(n, i * group, LB), h, has);
            }
        }
        n += gridDim.x;
    } while (TURNS && n < rounds);
}

// The way back.  Of the two sums over a row, the first (of dh * pre_weight * yn) needs y and dh, the second dy
// and b: each pair is fetched while the other is worked on.  Sums over rows stay in registers, two for each
// column: of dh * yn, and of d * act * bn, from which both dpost_weight and a shared gate's gradient follow,
// since all their other factors are the column's.  A workgroup's sums go to `partial` [block][2][columns],
// columns in the order of lanes' places.
template <int DT, bool S16, bool B16, bool GATE, int N, int I, bool TAIL>
__global__ void __launch_bounds__(widest_workgroup(I))
    block_bwd_kernel(capscaps_block B, capscaps_block_bwd_args A, RowPlan P, float* partial)
{
    constexpr int SD = S16 ? DT : CAPSCAPS_FP32, BD = B16 ? DT : CAPSCAPS_FP32;
    constexpr int SB = S16 ? 2 : 4, BB = B16 ? 2 : 4, LB = DT == CAPSCAPS_FP32 ? 4 : 2;
    __shared__ float lds[32];
    const int group = group_of<I>(P);
    const int slot = threadIdx.x / group, lane = threadIdx.x - slot * group;
    RowSum sum{lds, group, slot, 0};
    const bool branch = A.branch != nullptr, has_h = A.dh != nullptr;
    const bool post = branch && B.post_norm && A.rstd_post != nullptr;
    const float inv_width = 1.0f / (float)B.width;
    const float to_x = branch ? B.residual_scale : 1.0f;
    extern __shared__ float columns_lds[];
    Columns<N, I> col;
    col.lds = columns_lds;
    col.lane = lane;
#pragma unroll
    for (int i = 0; i < I; ++i)
        col.put(i, column_factors<N, TAIL>(B, A.pre_weight, post ? A.post_weight : nullptr, A.gate, P, lane + i * group));
    float sum_h[I][N], sum_b[I][N];
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int k = 0; k < N; ++k) sum_h[i][k] = sum_b[i][k] = 0.0f;
    Rows<N> ry(A.y, A.y_stride, SB, P, slot, lane), rdh(A.dh, A.dh_stride, LB, P, slot, lane);
    Rows<N> rdy(A.dy, A.dy_stride, SB, P, slot, lane), rb(A.branch, A.branch_stride, BB, P, slot, lane);
    Rows<N> rg(A.gate, A.gate_stride, LB, P, slot, lane), rdg(A.dgate, A.dgate_stride, LB, P, slot, lane);
    Rows<N> rdx(A.dx, A.dx_stride, SB, P, slot, lane), rdb(A.dbranch, A.dbranch_stride, LB, P, slot, lane);
    Raw<SD, N> y[I], dy[I];
    Raw<DT, N> dh[I], g[I];
    Raw<BD, N> b[I];
    float rpre = 1.0f, rpost = 1.0f;
    auto fetch_h = [&](long long n) {
        const long long r = n * P.per_block + slot;
        const bool in = r < B.rows, last = r + 1 >= B.rows;
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int v = lane + i * group;
            const Share has{in && v < P.full, TAIL && in && v == P.part, P.tail};
            clear(y[i]);
            clear(dh[i]);
            if (has_h) {
                load<SD, N, TAIL>(y[i], ry.get(n, i * group, SB), has, ry.over && !last);
                load<DT, N, TAIL>(dh[i], rdh.get(n, i * group, LB), has, rdh.over && !last);
            }
        }
        if (has_h && in) rpre = A.rstd_pre[r];
    };
    auto fetch_b = [&](long long n) {
        const long long r = n * P.per_block + slot;
        const bool in = r < B.rows, last = r + 1 >= B.rows;
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int v = lane + i * group;
            const Share has{in && v < P.full, TAIL && in && v == P.part, P.tail};
            clear(dy[i]);
            clear(b[i]);
            if (A.dy != nullptr) load<SD, N, TAIL>(dy[i], rdy.get(n, i * group, SB), has, rdy.over && !last);
            if (branch) load<BD, N, TAIL>(b[i], rb.get(n, i * group, BB), has, rb.over && !last);
            if constexpr (GATE) {
                clear(g[i]);
                load<DT, N, TAIL>(g[i], rg.get(n, i * group, LB), has, rg.over && !last);
            }
        }
        if (post && in) rpost = A.rstd_post[r];
    };
    const long long rounds = (B.rows + P.per_block - 1) / P.per_block;
    long long n = blockIdx.x;
    constexpr bool AHEAD = I < 8;  // (fp32 rows on 512 threads: no registers for it)
    if constexpr (AHEAD) fetch_h(n);
    for (; n < rounds; n += gridDim.x) {
        const bool in = n * P.per_block + slot < B.rows;
        // waves that hold rows by themselves stay together (wider rows' sums keep them so): their accesses are
        // then one piece of memory after another (6.4M rows of 64 bf16 values: 285 us, without 325; rows of
        // 1024, eight to a workgroup: 139, one: 163)
        if (group <= 64) __builtin_amdgcn_s_barrier();
        if constexpr (!AHEAD) fetch_h(n);
        fetch_b(n);
        float s = 0.0f, mean = 0.0f;
        if (has_h) {
#pragma unroll
            for (int i = 0; i < I; ++i) {
                float wh[N];
                col.to_h(i, wh);
#pragma unroll
                for (int k = 0; k < N; ++k) s += value<DT, N>(dh[i], k) * wh[k] * (value<SD, N>(y[i], k) * rpre);
            }
            mean = sum(s) * inv_width;
        }
        float e[I][N];
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int v = lane + i * group;
            const Share has{in && v < P.full, TAIL && in && v == P.part, P.tail};
            float dx[N], dg[N], cb[N], wh[N];
            col.to_b(i, cb);
            col.to_h(i, wh);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const float yn = value<SD, N>(y[i], k) * rpre, h = value<DT, N>(dh[i], k);
                sum_h[i][k] += h * yn;
                float d = value<SD, N>(dy[i], k);
                if (has_h) d += rpre * (h * wh[k] - yn * mean);
                dx[k] = to_x * d;
                const float bn = value<BD, N>(b[i], k) * rpost;
                if constexpr (GATE) {
                    const Gate q = gate_both(B.gate_act, value<DT, N>(g[i], k));
                    dg[k] = d * cb[k] * bn * q.slope;
                    d *= q.value;
                }
                sum_b[i][k] += d * bn;
                e[i][k] = d * cb[k];
                // (here, not where they are used: the compiler would keep the factors of all these products
                // until then)
                asm volatile("" : "+v"(sum_h[i][k]), "+v"(sum_b[i][k]), "+v"(e[i][k]));
                s += e[i][k] * bn;
            }
            if (A.dx != nullptr) store<SD, N, TAIL>(rdx.put(n, i * group, SB), dx, has);
            if constexpr (GATE) {
                if (A.dgate != nullptr) store<DT, N, TAIL>(rdg.put(n, i * group, LB), dg, has);
            }
        }
        if (AHEAD && n + gridDim.x < rounds) fetch_h(n + gridDim.x);
        if (A.dbranch != nullptr) {
            mean = post ? sum(s) * inv_width : 0.0f;
#pragma unroll
            for (int i = 0; i < I; ++i) {
                const int v = lane + i * group;
                const Share has{in && v < P.full, TAIL && in && v == P.part, P.tail};
                float db[N];
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    // (without the norm the gradient does not depend on b, which may be infinite)
                    db[k] = post ? rpost * (e[i][k] - value<BD, N>(b[i], k) * rpost * mean) : e[i][k];
                }
                store<DT, N, TAIL>(rdb.put(n, i * group, LB), db, has);
            }
        }
    }
    if (partial == nullptr) return;
    const int columns = P.vectors * group * N;
    float* out = partial + (long long)blockIdx.x * 2 * columns;
    if (P.per_block == 1) {
#pragma unroll
        for (int i = 0; i < I; ++i)
#pragma unroll
            for (int k = 0; k < N; ++k) {
                out[(lane + i * group) * N + k] = sum_h[i][k];
                out[columns + (lane + i * group) * N + k] = sum_b[i][k];
            }
        return;
    }
    if (group < 64) {
        // rows of one wave, in halves: lanes that hold the same columns
#pragma unroll
        for (int i = 0; i < I; ++i)
#pragma unroll
            for (int k = 0; k < N; ++k)
                for (int o = 32; o >= group; o >>= 1) {
                    sum_h[i][k] += __shfl_xor(sum_h[i][k], o);
                    sum_b[i][k] += __shfl_xor(sum_b[i][k], o);
                }
    }
    // the rows of the workgroup's waves: `slots` of them hold the same columns (a lane has one vector, or the
    // row a workgroup)
    if constexpr (I == 1) {
        __shared__ float of_slot[1024 * N];
        const int wide = group < 64 ? 64 : group, slots = P.threads / wide, in_row = group * N;
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            __syncthreads();
            if (group >= 64 || (int)(threadIdx.x & 63) < group) {
#pragma unroll
                for (int k = 0; k < N; ++k)
                    of_slot[threadIdx.x / wide * in_row + lane * N + k] = which == 0 ? sum_h[0][k] : sum_b[0][k];
            }
            __syncthreads();
            for (int c = threadIdx.x; c < in_row; c += P.threads) {
                float s = of_slot[c];
                for (int j = 1; j < slots; ++j) s += of_slot[j * in_row + c];
                out[which * columns + c] = s;
            }
        }
    }
}

// Sums the workgroups' sums, 64 columns a workgroup, each by 16 threads that take every 16th in turn
__global__ void __launch_bounds__(1024)
    block_bwd_sums_kernel(capscaps_block B, capscaps_block_bwd_args A, RowPlan P, const float* partial)
{
    __shared__ float lds[16][64];
    const int c = blockIdx.x * 64 + (threadIdx.x & 63), share = threadIdx.x >> 6;
    const int columns = P.vectors * P.group * P.n;
    float s = 0.0f;
    if (c < B.width) {
        const float* p = partial + (long long)blockIdx.y * columns + c;
#pragma unroll 8
        for (int k = share; k < (int)P.blocks; k += 16) s += p[(long long)k * 2 * columns];
    }
    lds[share][threadIdx.x & 63] = s;
    __syncthreads();
    if (share != 0 || c >= B.width) return;
    for (int k = 1; k < 16; ++k) s += lds[k][threadIdx.x];
    if (blockIdx.y == 0) {
        if (A.dpre_weight != nullptr) A.dpre_weight[c] = s;
        return;
    }
    s *= B.branch_scale;
    const bool shared = B.gate == CAPSCAPS_GATE_SHARED;
    const float g = shared ? static_cast<const float*>(A.gate)[c] : 1.0f;
    if (A.dpost_weight != nullptr) A.dpost_weight[c] = shared ? s * gate_value(B.gate_act, g) : s;
    if (shared && A.dgate != nullptr)
        static_cast<float*>(A.dgate)[c] = s * (B.post_norm && A.post_weight != nullptr ? A.post_weight[c] : 1.0f) *
                                          gate_slope(B.gate_act, g);
}

// ------------------------------------------------------------------------------------ rows of any width
__device__ __forceinline__ float gate_at(const capscaps_block& B, const void* gate, long long row, long long stride,
                                         int c)
{
    return B.gate == CAPSCAPS_GATE_SHARED ? static_cast<const float*>(gate)[c]
                                          : load_element(gate, row * stride + c, B.dtype);
}

__global__ void __launch_bounds__(THREADS) block_fwd_any_kernel(capscaps_block B, capscaps_block_fwd_args A)
{
    __shared__ float lds[THREADS / 64];
    for (long long r = blockIdx.x; r < B.rows; r += gridDim.x) {
        float rpost = 1.0f;
        if (A.branch != nullptr && B.post_norm) {
            float s = 0.0f;
            for (int c = threadIdx.x; c < B.width; c += THREADS) {
                const float b = load_element(A.branch, r * A.branch_stride + c, B.branch_dtype);
                s += b * b;
            }
            rpost = 1.0f / sqrtf(block_sum(s, lds) / (float)B.width + B.eps);
            if (A.rstd_post != nullptr && threadIdx.x == 0) A.rstd_post[r] = rpost;
        }
        auto value = [&](int c) {
            const float x = load_element(A.x, r * A.x_stride + c, B.stream_dtype);
            if (A.branch == nullptr) return x;
            float u = load_element(A.branch, r * A.branch_stride + c, B.branch_dtype) * rpost;
            if (B.post_norm && A.post_weight != nullptr) u *= A.post_weight[c];
            if (B.gate != CAPSCAPS_GATE_NONE) u *= gate_value(B.gate_act, gate_at(B, A.gate, r, A.gate_stride, c));
            return B.residual_scale * x + B.branch_scale * u;
        };
        float rpre = 1.0f;
        if (A.h != nullptr) {
            float s = 0.0f;
            for (int c = threadIdx.x; c < B.width; c += THREADS) {
                const float y = value(c);
                s += y * y;
            }
            rpre = 1.0f / sqrtf(block_sum(s, lds) / (float)B.width + B.eps);
            if (A.rstd_pre != nullptr && threadIdx.x == 0) A.rstd_pre[r] = rpre;
        }
        for (int c = threadIdx.x; c < B.width; c += THREADS) {
            const float y = value(c);
            if (A.y != nullptr) store_element(A.y, r * A.y_stride + c, y, B.stream_dtype);
            if (A.h != nullptr)
                store_element(A.h, r * A.h_stride + c, y * rpre * (A.pre_weight != nullptr ? A.pre_weight[c] : 1.0f),
                              B.dtype);
        }
    }
}

// One element of the way back, given the row's mean of dh * pre_weight * yn
struct Back {
    float yn, dh, d;        // d: the gradient that reaches y
    float t, bn, u, a, g;   // of the branch
};
__device__ __forceinline__ Back back_at(const capscaps_block& B, const capscaps_block_bwd_args& A, long long r, int c,
                                        float mean_pre, float rpre, float rpost)
{
    Back k{};
    k.d = A.dy != nullptr ? load_element(A.dy, r * A.dy_stride + c, B.stream_dtype) : 0.0f;
    if (A.dh != nullptr) {
        k.yn = load_element(A.y, r * A.y_stride + c, B.stream_dtype) * rpre;
        k.dh = load_element(A.dh, r * A.dh_stride + c, B.dtype);
        k.d += rpre * (k.dh * (A.pre_weight != nullptr ? A.pre_weight[c] : 1.0f) - k.yn * mean_pre);
    }
    if (A.branch != nullptr) {
        k.t = B.branch_scale * k.d;
        k.bn = load_element(A.branch, r * A.branch_stride + c, B.branch_dtype) * rpost;
        k.u = B.post_norm && A.post_weight != nullptr ? k.bn * A.post_weight[c] : k.bn;
        k.a = 1.0f;
        if (B.gate != CAPSCAPS_GATE_NONE) {
            k.g = gate_at(B, A.gate, r, A.gate_stride, c);
            k.a = gate_value(B.gate_act, k.g);
        }
    }
    return k;
}

// dx, dbranch, a full gate's gradient; the rows' means of dh * pre_weight * yn go to `mean`
__global__ void __launch_bounds__(THREADS)
    block_bwd_rows_kernel(capscaps_block B, capscaps_block_bwd_args A, float* mean)
{
    __shared__ float lds[THREADS / 64];
    for (long long r = blockIdx.x; r < B.rows; r += gridDim.x) {
        const float rpre = A.dh != nullptr ? A.rstd_pre[r] : 1.0f;
        const float rpost = A.branch != nullptr && B.post_norm && A.rstd_post != nullptr ? A.rstd_post[r] : 1.0f;
        float mean_pre = 0.0f;
        if (A.dh != nullptr) {
            float s = 0.0f;
            for (int c = threadIdx.x; c < B.width; c += THREADS) {
                float n = load_element(A.dh, r * A.dh_stride + c, B.dtype);
                if (A.pre_weight != nullptr) n *= A.pre_weight[c];
                s += n * (load_element(A.y, r * A.y_stride + c, B.stream_dtype) * rpre);
            }
            mean_pre = block_sum(s, lds) / (float)B.width;
            if (mean != nullptr && threadIdx.x == 0) mean[r] = mean_pre;
        }
        auto e_of = [&](const Back& k, int c) {
            return k.t * k.a * (B.post_norm && A.post_weight != nullptr ? A.post_weight[c] : 1.0f);
        };
        float mean_post = 0.0f;
        if (A.dbranch != nullptr && B.post_norm) {
            float s = 0.0f;
            for (int c = threadIdx.x; c < B.width; c += THREADS) {
                const Back k = back_at(B, A, r, c, mean_pre, rpre, rpost);
                s += e_of(k, c) * k.bn;
            }
            mean_post = block_sum(s, lds) / (float)B.width;
        }
        for (int c = threadIdx.x; c < B.width; c += THREADS) {
            const Back k = back_at(B, A, r, c, mean_pre, rpre, rpost);
            if (A.dx != nullptr)
                store_element(A.dx, r * A.dx_stride + c, A.branch != nullptr ? B.residual_scale * k.d : k.d,
                              B.stream_dtype);
            if (A.dgate != nullptr && B.gate == CAPSCAPS_GATE_FULL)
                store_element(A.dgate, r * A.dgate_stride + c, k.t * k.u * gate_slope(B.gate_act, k.g), B.dtype);
            if (A.dbranch != nullptr)
                store_element(A.dbranch, r * A.dbranch_stride + c,
                              B.post_norm ? rpost * (e_of(k, c) - k.bn * mean_post) : e_of(k, c), B.dtype);
        }
    }
}

// Sums over a share of the rows, a thread per column: partial[share][3][width] = dpre_weight, dpost_weight, dgate
__global__ void __launch_bounds__(THREADS)
    block_bwd_columns_kernel(capscaps_block B, capscaps_block_bwd_args A, const float* mean, float* partial,
                             long long rows_per_share)
{
    const int c = blockIdx.x * THREADS + threadIdx.x;
    if (c >= B.width) return;
    const long long r0 = blockIdx.y * rows_per_share;
    const long long r1 = r0 + rows_per_share < B.rows ? r0 + rows_per_share : B.rows;
    float pre = 0.0f, post = 0.0f, gate = 0.0f;
    for (long long r = r0; r < r1; ++r) {
        const float rpre = A.dh != nullptr ? A.rstd_pre[r] : 1.0f;
        const float rpost = A.branch != nullptr && B.post_norm && A.rstd_post != nullptr ? A.rstd_post[r] : 1.0f;
        const Back k = back_at(B, A, r, c, A.dh != nullptr ? mean[r] : 0.0f, rpre, rpost);
        pre += k.dh * k.yn;
        post += k.t * k.a * k.bn;
        if (B.gate == CAPSCAPS_GATE_SHARED) gate += k.t * k.u * gate_slope(B.gate_act, k.g);
    }
    float* p = partial + (long long)blockIdx.y * 3 * B.width + c;
    p[0] = pre;
    p[B.width] = post;
    p[2LL * B.width] = gate;
}

__global__ void __launch_bounds__(THREADS)
    block_bwd_sum_kernel(const float* partial, int shares, int width, float* pre, float* post, float* gate)
{
    const int c = blockIdx.x * THREADS + threadIdx.x;
    float* out = blockIdx.y == 0 ? pre : blockIdx.y == 1 ? post : gate;
    if (c >= width || out == nullptr) return;
    float s = 0.0f;
    for (int k = 0; k < shares; ++k) s += partial[((long long)k * 3 + blockIdx.y) * width + c];
    out[c] = s;
}

int row_shares(long long rows) { return rows < 256 ? (int)rows : 256; }

bool misaligned(const void* p, int dtype)
{
    return (reinterpret_cast<uintptr_t>(p) & (element_bytes(dtype) - 1)) != 0;
}

// a tensor that the call reads or writes: aligned to its elements, rows within reach of 62 bits
bool bad_rows(const capscaps_block& B, const void* p, long long stride, int dtype, bool output)
{
    if (p == nullptr) return false;
    if (misaligned(p, dtype) || stride < 0) return true;
    if (output && B.rows > 1 && stride < B.width) return true;
    return (long double)B.rows * (long double)stride > 1e17L;
}

int check_block(const capscaps_block* B)
{
    if (B == nullptr || B->rows <= 0 || B->width <= 0 || !known_dtype(B->dtype)) return CAPSCAPS_EINVAL;
    if (B->stream_dtype != CAPSCAPS_FP32 && B->stream_dtype != B->dtype) return CAPSCAPS_EINVAL;
    if (B->branch_dtype != CAPSCAPS_FP32 && B->branch_dtype != B->dtype) return CAPSCAPS_EINVAL;
    if ((unsigned)B->post_norm > 1 || (unsigned)B->gate > 2 || (unsigned)B->gate_act > 2) return CAPSCAPS_EINVAL;
    if (!isfinite(B->residual_scale) || !isfinite(B->branch_scale)) return CAPSCAPS_EINVAL;
    if (!(B->eps >= FLT_MIN) || !isfinite(B->eps)) return CAPSCAPS_EINVAL;  // (a normal number, for v_rsq_f32)
    if (B->width > (1 << 30) || (long double)B->rows * B->width > 1e17L) return CAPSCAPS_EINVAL;
    return CAPSCAPS_OK;
}

// The lanes of a row: as few as hold it with one vector each, up to a workgroup of 1024; then two vectors of
// four values, or 32 values in a workgroup of 512.  `apart`: rows so far apart that those of one workgroup are
// not within reach of 32-bit offsets, one at a time in a workgroup.
//
// Workgroups of 1024 that go through many rows in step read memory in large pieces, and need the columns'
// factors once; rows of few lanes do better as they come, four waves a workgroup (us, forward, 134M bf16 values
// a tensor, 173 at 6.2 TB/s: rows of 512 183 as they come, 202 in turns; of 1024 192 and 183, of 4096 239 and
// 182; 67M fp32 values: rows of 1024 178 and 188, of 4096 192 and 180).  The way back keeps sums over rows in
// registers, so it always goes in turns.
RowPlan row_plan(const capscaps_block& B, int n, bool forward, bool apart)
{
    RowPlan P;
    P.n = n;
    const int vectors = (B.width + n - 1) / n;
    P.vectors = 1;
    if (vectors <= 64) {
        P.group = apart ? 64 : 1;
        while (P.group < vectors) P.group *= 2;
    } else if (vectors <= 1024) {
        P.group = (vectors + 63) / 64 * 64;
    } else {
        P.vectors = n == 4 && vectors <= 2048 ? 2 : 32 / n;
        P.group = widest_workgroup(P.vectors);
    }
    const bool in_step = !forward || (vectors > 64 && (n == 8 || B.width > 2048));
    // Backward, rows within a wave that no vector divides: their accesses cross lines, and their waves wait
    // longer than others, so more of them, in smaller workgroups (2.1M rows of 27 fp32 values with a gate: 387
    // us, as the others 420; bf16 and fp32 mixed 300, 365; of 27 bf16 values, whose lanes take more registers,
    // two workgroups 170, one 176, three 216)
    const bool crossing = !forward && B.width % n != 0 && vectors <= 64;
    const int step = crossing ? 512 : 1024;
    // (several rows in such a workgroup where there are rows for every unit)
    const int threads = in_step && B.rows * P.group >= (long long)step * CUS ? step : THREADS;
    P.per_block = apart || P.group >= threads || P.vectors > 1 ? 1 : threads / P.group;
    P.threads = P.per_block * P.group;
    const long long blocks = (B.rows + P.per_block - 1) / P.per_block;
    // (a launch has less than 2^32 threads, and rows of 1793 .. 2048 values in fours are workgroups of 512)
    const long long as_they_come = (1LL << 23) - 1;
    const int per_unit = forward ? 2048 : crossing && n == 4 ? 1536 : 1024;  // threads
    const long long most = apart ? CUS : !in_step ? as_they_come : CUS * (per_unit / P.threads);
    P.blocks = (unsigned)(blocks < most ? blocks : most);
    P.turns = P.blocks < blocks;
    P.full = B.width / n;
    P.tail = B.width % n;
    P.part = P.tail != 0 ? P.full : -1;
    return P;
}
bool rows_apart(std::initializer_list<long long> strides)
{
    for (long long s : strides)
        if (s > (1 << 18)) return true;  // 1024 rows of fp32 within 2^30 bytes
    return false;
}
// Values of a vector.  An fp32 branch between 16-bit tensors is taken in eights too in the forward pass, whose waves
// are many and short: half as many of them (us: 192544 rows of 400 values 140, in fours 186; 1.6M of 64 164 and 196;
// 91557 of 2112, in turns, 352 and 335).  On the way back up to 8192 values, where it fits one vector a lane (733139 rows
// of 280 507 and 754, 40685 of 4096 525 and 559, 1.6M of 64 246 and 236; 16384 of 10000 596 and 487)
int vector_values(const capscaps_block& B, bool branch, bool forward)
{
    const bool s16 = B.dtype != CAPSCAPS_FP32 && B.stream_dtype == B.dtype;
    return s16 && (forward || !branch || B.branch_dtype == B.dtype || B.width <= 8192) ? 8 : 4;
}

template <int V>
using Int = std::integral_constant<int, V>;

// calls `launch` with the kernel's compile-time properties: stream and branch of 16 bits, a gate for every
// value, values of a vector, vectors of a lane, a partial vector
template <int DT, bool FORWARD, typename F>
void with_properties(const capscaps_block& B, bool branch, const RowPlan& P, F launch)
{
    const std::true_type yes;
    const std::false_type no;
    auto by_tail = [&](auto s, auto b, auto g, auto n, auto i) {
        P.tail ? launch(s, b, g, n, i, yes) : launch(s, b, g, n, i, no);
    };
    auto by_vectors = [&](auto s, auto b, auto g) {
        if constexpr (s.value && (b.value || FORWARD)) {
            P.vectors == 1 ? by_tail(s, b, g, Int<8>(), Int<1>()) : by_tail(s, b, g, Int<8>(), Int<4>());
        } else if constexpr (s.value) {
            P.n == 8 ? by_tail(s, b, g, Int<8>(), Int<1>()) : by_tail(s, b, g, Int<4>(), Int<8>());
        } else {
            if (P.vectors == 1) by_tail(s, b, g, Int<4>(), Int<1>());
            if (P.vectors == 2) by_tail(s, b, g, Int<4>(), Int<2>());
            if (P.vectors == 8) by_tail(s, b, g, Int<4>(), Int<8>());
        }
    };
    auto by_gate = [&](auto s, auto b) {
        B.gate == CAPSCAPS_GATE_FULL ? by_vectors(s, b, yes) : by_vectors(s, b, no);
    };
    if constexpr (DT == CAPSCAPS_FP32) {
        by_gate(no, no);
    } else {
        const bool s16 = B.stream_dtype == DT, b16 = B.branch_dtype == DT || !branch;
        if (s16)
            b16 ? by_gate(yes, yes) : by_gate(yes, no);
        else
            b16 ? by_gate(no, yes) : by_gate(no, no);
    }
}

template <int DT>
void launch_fwd(const capscaps_block& B, const capscaps_block_fwd_args& A, const RowPlan& P, hipStream_t st)
{
    with_properties<DT, true>(B, A.branch != nullptr, P, [&](auto s, auto b, auto g, auto n, auto i, auto tail) {
        if constexpr (i.value == 1) {
            if (!P.turns) {
                block_fwd_kernel<DT, s.value, b.value, g.value, n.value, i.value, tail.value, false>
                    <<<dim3(P.blocks), dim3(P.threads), 0, st>>>(B, A, P);
                return;
            }
        }
        block_fwd_kernel<DT, s.value, b.value, g.value, n.value, i.value, tail.value, true>
            <<<dim3(P.blocks), dim3(P.threads), 0, st>>>(B, A, P);
    });
}
template <int DT>
hipError_t launch_bwd(const capscaps_block& B, const capscaps_block_bwd_args& A, const RowPlan& P, float* partial,
                      hipStream_t st)
{
    hipError_t err = hipSuccess;
    with_properties<DT, false>(B, A.branch != nullptr, P, [&](auto s, auto b, auto g, auto n, auto i, auto tail) {
        const auto kernel = block_bwd_kernel<DT, s.value, b.value, g.value, n.value, i.value, tail.value>;
        const int lds = i.value == 1 ? 0 : P.group * i.value * n.value * 2 * 4;
        if (i.value > 1) {
            static std::atomic<unsigned long long> done{0};
            err = set_dynamic_lds_once(reinterpret_cast<const void*>(kernel), WIDEST * 2 * 4, done);
            if (err != hipSuccess) return;
        }
        kernel<<<dim3(P.blocks), dim3(P.threads), lds, st>>>(B, A, P, partial);
        err = hipGetLastError();
    });
    return err;
}

unsigned row_blocks(const capscaps_block& B) { return (unsigned)(B.rows < (1 << 20) ? B.rows : (1 << 20)); }

}  // namespace
}  // namespace capscaps

using namespace capscaps;

extern "C" {

int capscaps_block_norm_fwd(const capscaps_block* block, const capscaps_block_fwd_args* args, void* stream)
{
    const int rc = check_block(block);
    if (rc != CAPSCAPS_OK) return rc;
    if (args == nullptr) return CAPSCAPS_EINVAL;
    const capscaps_block& B = *block;
    const capscaps_block_fwd_args& A = *args;
    if (A.x == nullptr || (A.y == nullptr && A.h == nullptr)) return CAPSCAPS_EINVAL;
    if (A.branch == nullptr && (A.y != nullptr || B.gate != CAPSCAPS_GATE_NONE)) return CAPSCAPS_EINVAL;
    if ((A.gate != nullptr) != (B.gate != CAPSCAPS_GATE_NONE)) return CAPSCAPS_EINVAL;
    const bool full = B.gate == CAPSCAPS_GATE_FULL;
    if (bad_rows(B, A.x, A.x_stride, B.stream_dtype, false) ||
        bad_rows(B, A.branch, A.branch_stride, B.branch_dtype, false) ||
        bad_rows(B, A.gate, full ? A.gate_stride : 0, full ? B.dtype : CAPSCAPS_FP32, false) ||
        bad_rows(B, A.y, A.y_stride, B.stream_dtype, true) || bad_rows(B, A.h, A.h_stride, B.dtype, true))
        return CAPSCAPS_EINVAL;
    for (const float* p : {A.pre_weight, A.post_weight, (const float*)A.rstd_pre, (const float*)A.rstd_post})
        if (misaligned(p, CAPSCAPS_FP32)) return CAPSCAPS_EINVAL;
    if (A.y == A.x && A.y_stride != A.x_stride) return CAPSCAPS_EINVAL;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const bool apart = rows_apart({A.x_stride, A.branch_stride, A.gate_stride, A.y_stride, A.h_stride});
    if (B.width > WIDEST) {
        block_fwd_any_kernel<<<dim3(row_blocks(B)), dim3(THREADS), 0, st>>>(B, A);
        return status_from_hip(hipGetLastError());
    }
    const RowPlan P = row_plan(B, vector_values(B, A.branch != nullptr, true), true, apart);
    if (B.dtype == CAPSCAPS_FP32)
        launch_fwd<CAPSCAPS_FP32>(B, A, P, st);
    else if (B.dtype == CAPSCAPS_BF16)
        launch_fwd<CAPSCAPS_BF16>(B, A, P, st);
    else
        launch_fwd<CAPSCAPS_FP16>(B, A, P, st);
    return status_from_hip(hipGetLastError());
}

// (for tests) workgroups and threads of the launch for rows of up to 16384 values; 0: an invalid block, or wider rows
int capscaps_testing_block_norm_launch(const capscaps_block* block, int branch, int forward, int apart,
                                       long long* workgroups_threads)
{
    if (check_block(block) != CAPSCAPS_OK || block->width > WIDEST) return 0;
    const RowPlan P = row_plan(*block, vector_values(*block, branch != 0, forward != 0), forward != 0, apart != 0);
    workgroups_threads[0] = P.blocks;
    workgroups_threads[1] = P.threads;
    return 1;
}

size_t capscaps_block_norm_bwd_workspace_bytes(const capscaps_block* block)
{
    if (check_block(block) != CAPSCAPS_OK) return 0;
    if (block->width <= WIDEST) {
        size_t most = 0;
        for (const bool apart : {false, true})
            for (const bool branch : {false, true}) {
                const RowPlan P = row_plan(*block, vector_values(*block, branch, false), false, apart);
                const size_t bytes = (size_t)P.blocks * 2 * P.vectors * P.group * P.n * 4;
                most = bytes > most ? bytes : most;
            }
        return most;
    }
    const size_t means = (size_t)block->rows * 4, sums = (size_t)row_shares(block->rows) * 3 * block->width * 4;
    return (means + 255) / 256 * 256 + sums;
}

int capscaps_block_norm_bwd(const capscaps_block* block, const capscaps_block_bwd_args* args, void* workspace,
                            size_t workspace_bytes, void* stream)
{
    const int rc = check_block(block);
    if (rc != CAPSCAPS_OK) return rc;
    if (args == nullptr) return CAPSCAPS_EINVAL;
    const capscaps_block& B = *block;
    const capscaps_block_bwd_args& A = *args;
    const bool full = B.gate == CAPSCAPS_GATE_FULL;
    if (A.dh == nullptr && A.dy == nullptr) return CAPSCAPS_EINVAL;
    if (A.dh != nullptr && (A.y == nullptr || A.rstd_pre == nullptr)) return CAPSCAPS_EINVAL;
    if (!A.dx && !A.dbranch && !A.dgate && !A.dpre_weight && !A.dpost_weight) return CAPSCAPS_EINVAL;
    if ((A.gate != nullptr) != (B.gate != CAPSCAPS_GATE_NONE)) return CAPSCAPS_EINVAL;
    const bool branch_wanted = A.dbranch || A.dgate || A.dpost_weight;
    if (A.branch == nullptr && (branch_wanted || B.gate != CAPSCAPS_GATE_NONE)) return CAPSCAPS_EINVAL;
    if (branch_wanted && B.post_norm && A.rstd_post == nullptr) return CAPSCAPS_EINVAL;
    if (A.dgate != nullptr && B.gate == CAPSCAPS_GATE_NONE) return CAPSCAPS_EINVAL;
    if (A.dpre_weight != nullptr && A.dh == nullptr) return CAPSCAPS_EINVAL;
    if (A.dpost_weight != nullptr && !B.post_norm) return CAPSCAPS_EINVAL;
    if (bad_rows(B, A.y, A.y_stride, B.stream_dtype, false) ||
        bad_rows(B, A.branch, A.branch_stride, B.branch_dtype, false) ||
        bad_rows(B, A.gate, full ? A.gate_stride : 0, full ? B.dtype : CAPSCAPS_FP32, false) ||
        bad_rows(B, A.dh, A.dh_stride, B.dtype, false) || bad_rows(B, A.dy, A.dy_stride, B.stream_dtype, false) ||
        bad_rows(B, A.dx, A.dx_stride, B.stream_dtype, true) ||
        bad_rows(B, A.dbranch, A.dbranch_stride, B.dtype, true) ||
        bad_rows(B, A.dgate, full ? A.dgate_stride : B.width, full ? B.dtype : CAPSCAPS_FP32, full))
        return CAPSCAPS_EINVAL;
    for (const float* p : {A.pre_weight, A.post_weight, A.rstd_pre, A.rstd_post, (const float*)A.dpre_weight,
                           (const float*)A.dpost_weight})
        if (misaligned(p, CAPSCAPS_FP32)) return CAPSCAPS_EINVAL;
    float* dgate_sum = B.gate == CAPSCAPS_GATE_SHARED ? static_cast<float*>(A.dgate) : nullptr;
    const bool sums = A.dpre_weight || A.dpost_weight || dgate_sum;
    if (sums) {
        if (workspace == nullptr || workspace_bytes < capscaps_block_norm_bwd_workspace_bytes(block))
            return CAPSCAPS_EWORKSPACE;
        if ((reinterpret_cast<uintptr_t>(workspace) & 15u) != 0) return CAPSCAPS_EINVAL;
    }
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (B.width <= WIDEST) {
        const bool apart = rows_apart({A.y_stride, A.branch_stride, A.gate_stride, A.dh_stride, A.dy_stride, A.dx_stride,
                                       A.dbranch_stride, A.dgate_stride});
        const RowPlan P = row_plan(B, vector_values(B, A.branch != nullptr, false), false, apart);
        float* partial = sums ? static_cast<float*>(workspace) : nullptr;
        const hipError_t err = B.dtype == CAPSCAPS_FP32   ? launch_bwd<CAPSCAPS_FP32>(B, A, P, partial, st)
                               : B.dtype == CAPSCAPS_BF16 ? launch_bwd<CAPSCAPS_BF16>(B, A, P, partial, st)
                                                          : launch_bwd<CAPSCAPS_FP16>(B, A, P, partial, st);
        if (err != hipSuccess || !sums) return status_from_hip(err);
        block_bwd_sums_kernel<<<dim3((B.width + 63) / 64, 2), dim3(1024), 0, st>>>(B, A, P, partial);
        return status_from_hip(hipGetLastError());
    }
    float* mean = sums ? static_cast<float*>(workspace) : nullptr;
    block_bwd_rows_kernel<<<dim3(row_blocks(B)), dim3(THREADS), 0, st>>>(B, A, mean);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess || !sums) return status_from_hip(err);
    float* partial = mean + ((size_t)B.rows + 63) / 64 * 64;
    const int shares = row_shares(B.rows);
    const long long per = (B.rows + shares - 1) / shares;
    const unsigned columns = (unsigned)((B.width + THREADS - 1) / THREADS);
    block_bwd_columns_kernel<<<dim3(columns, shares), dim3(THREADS), 0, st>>>(B, A, mean, partial, per);
    err = hipGetLastError();
    if (err != hipSuccess) return status_from_hip(err);
    block_bwd_sum_kernel<<<dim3(columns, 3), dim3(THREADS), 0, st>>>(partial, shares, B.width, A.dpre_weight,
                                                                     A.dpost_weight, dgate_sum);
    return status_from_hip(hipGetLastError());
}

}  // extern "C"
