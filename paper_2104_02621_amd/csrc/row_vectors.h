// Internal: rows of values of the three element types, eight values a lane, at any address.
//
// A row's values are cut into vectors of eight: 16 bytes of a 16-bit type, two times 16 of fp32, loaded and stored
// whole at any alignment (the hardware takes 16-byte accesses at element addresses).  What a row's length leaves over (1 .. 7 values) is
// one lane's last vector, moved in pieces of 4, 2 and 1 values that have fixed places in the registers: 0 .. 3, 4 .. 5
// and 6.  All tensors of a call and the per-column vectors use the same places, so the kernels need not know.
#pragma once
#include <hip/hip_runtime.h>

#include "element.h"

namespace capscaps {

typedef unsigned uint4v __attribute__((ext_vector_type(4)));
typedef uint4v uint4_a2 __attribute__((aligned(2)));
typedef uint4v uint4_a4 __attribute__((aligned(4)));
typedef unsigned uint2v __attribute__((ext_vector_type(2)));
typedef uint2v uint2_a2 __attribute__((aligned(2)));
typedef uint2v uint2_a4 __attribute__((aligned(4)));
typedef unsigned uint_a2 __attribute__((aligned(2)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));

constexpr int VEC = 8;

template <int DT>
struct Raw {
    static constexpr int QUADS = DT == CAPSCAPS_FP32 ? 2 : 1;
    uint4v q[QUADS];
};

template <int DT>
__device__ __forceinline__ void clear(Raw<DT>& r)
{
#pragma unroll
    for (int k = 0; k < Raw<DT>::QUADS; ++k) r.q[k] = uint4v{0, 0, 0, 0};
}

template <int DT>
__device__ __forceinline__ void load_full(Raw<DT>& r, const char* p)
{
    if constexpr (DT == CAPSCAPS_FP32) {
        r.q[0] = reinterpret_cast<const uint4_a4*>(p)[0];
        r.q[1] = reinterpret_cast<const uint4_a4*>(p)[1];
    } else {
        r.q[0] = *reinterpret_cast<const uint4_a2*>(p);
    }
}
template <int DT>
__device__ __forceinline__ void load_tail(Raw<DT>& r, const char* p, int tail)
{
    if constexpr (DT == CAPSCAPS_FP32) {
        if (tail & 4) r.q[0] = *reinterpret_cast<const uint4_a4*>(p);
        if (tail & 2) {
            const uint2v w = *reinterpret_cast<const uint2_a4*>(p + (tail & 4) * 4);
            r.q[1].x = w.x;
            r.q[1].y = w.y;
        }
        if (tail & 1) r.q[1].z = *reinterpret_cast<const unsigned*>(p + (tail & 6) * 4);
    } else {
        if (tail & 4) {
            const uint2v w = *reinterpret_cast<const uint2_a2*>(p);
            r.q[0].x = w.x;
            r.q[0].y = w.y;
        }
        if (tail & 2) r.q[0].z = *reinterpret_cast<const uint_a2*>(p + (tail & 4) * 2);
        if (tail & 1) r.q[0].w = *reinterpret_cast<const unsigned short*>(p + (tail & 6) * 2);
    }
}
// a lane's vector: whole, the row's remainder, or nothing (zeros)
template <int DT, bool TAIL>
__device__ __forceinline__ void load(Raw<DT>& r, const char* p, bool full, bool part, int tail)
{
    if (full) load_full<DT>(r, p);
    if constexpr (TAIL) {
        if (part) load_tail<DT>(r, p, tail);
    }
}

template <int DT>
__device__ __forceinline__ float value(const Raw<DT>& r, int k)  // (k is a constant after unrolling)
{
    if constexpr (DT == CAPSCAPS_FP32) {
        return __builtin_bit_cast(float, (unsigned)r.q[k / 4][k % 4]);
    } else {
        const unsigned w = r.q[0][k / 2];
        if constexpr (DT == CAPSCAPS_BF16)
            return __builtin_bit_cast(float, (k & 1) ? (w & 0xffff0000u) : (w << 16));
        else
            return Element<DT>::get((unsigned short)((k & 1) ? (w >> 16) : (w & 0xffffu)));
    }
}

template <int DT>
__device__ __forceinline__ Raw<DT> pack(const float* f)
{
    Raw<DT> r;
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
        if constexpr (DT == CAPSCAPS_FP32) {
            r.q[k / 4][k % 4] = __builtin_bit_cast(unsigned, f[k]);
        } else if ((k & 1) == 0) {
            const float2v pair = {f[k], f[k + 1]};
            if constexpr (DT == CAPSCAPS_BF16)
                r.q[0][k / 2] = __builtin_bit_cast(unsigned, __builtin_convertvector(pair, bf16x2v));
            else
                r.q[0][k / 2] = __builtin_bit_cast(unsigned, __builtin_convertvector(pair, half2v));
        }
    }
    return r;
}
template <int DT, bool TAIL>
__device__ __forceinline__ void store(char* p, const float* f, bool full, bool part, int tail)
{
    if (!full && !(TAIL && part)) return;
    const Raw<DT> r = pack<DT>(f);
    if constexpr (DT == CAPSCAPS_FP32) {
        if (full) {
            reinterpret_cast<uint4_a4*>(p)[0] = r.q[0];
            reinterpret_cast<uint4_a4*>(p)[1] = r.q[1];
        } else if constexpr (TAIL) {
            if (tail & 4) *reinterpret_cast<uint4_a4*>(p) = r.q[0];
            if (tail & 2) *reinterpret_cast<uint2_a4*>(p + (tail & 4) * 4) = uint2v{r.q[1].x, r.q[1].y};
            if (tail & 1) *reinterpret_cast<unsigned*>(p + (tail & 6) * 4) = r.q[1].z;
        }
    } else {
        if (full) {
            *reinterpret_cast<uint4_a2*>(p) = r.q[0];
        } else if constexpr (TAIL) {
            if (tail & 4) *reinterpret_cast<uint2_a2*>(p) = uint2v{r.q[0].x, r.q[0].y};
            if (tail & 2) *reinterpret_cast<uint_a2*>(p + (tail & 4) * 2) = r.q[0].z;
            if (tail & 1) *reinterpret_cast<unsigned short*>(p + (tail & 6) * 2) = (unsigned short)r.q[0].w;
        }
    }
}

// a vector of a per-column fp32 tensor (ones where there is none)
template <bool TAIL>
__device__ __forceinline__ void load_column(float* f, const float* p, int vector, bool full, bool part, int tail,
                                            float none)
{
    Raw<CAPSCAPS_FP32> r;
    clear(r);
    if (p != nullptr) load<CAPSCAPS_FP32, TAIL>(r, reinterpret_cast<const char*>(p + (size_t)vector * VEC), full, part, tail);
#pragma unroll
    for (int k = 0; k < VEC; ++k) f[k] = p != nullptr ? value<CAPSCAPS_FP32>(r, k) : none;
}

template <int CTRL>
__device__ __forceinline__ float dpp_add(float v)
{
    return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
// sum over groups of `lanes` (a power of two up to 64) neighbouring lanes, in each of them.  Within 16 lanes by
// data-parallel moves (exchange with the neighbour, the other pair, and mirrored: what is mirrored is equal by then)
__device__ __forceinline__ float lanes_sum(float v, int lanes)
{
    if (lanes > 1) v = dpp_add<0xB1>(v);   // quad_perm 1 0 3 2
    if (lanes > 2) v = dpp_add<0x4E>(v);   // quad_perm 2 3 0 1
    if (lanes > 4) v = dpp_add<0x141>(v);  // row_half_mirror
    if (lanes > 8) v = dpp_add<0x140>(v);  // row_mirror
    if (lanes == 32) {
        v += __builtin_bit_cast(float, __builtin_amdgcn_ds_swizzle(__builtin_bit_cast(int, v), 0x401f));  // lane ^ 16
    } else if (lanes == 64) {
        const int w = __builtin_bit_cast(int, v);
        v = (__builtin_bit_cast(float, __builtin_amdgcn_readlane(w, 0)) +
             __builtin_bit_cast(float, __builtin_amdgcn_readlane(w, 16))) +
            (__builtin_bit_cast(float, __builtin_amdgcn_readlane(w, 32)) +
             __builtin_bit_cast(float, __builtin_amdgcn_readlane(w, 48)));
    }
    return v;
}

}  // namespace capscaps
