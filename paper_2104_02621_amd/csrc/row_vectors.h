// Internal: rows of values of the three element types, some values a lane, at any address.
//
// A row's values are cut into vectors of N values, one of 16 bytes where all tensors of a call have 16-bit elements (N = 8),
// else N = 4: 16 bytes of fp32, 8 of a 16-bit type, so that a wave's access is one contiguous piece in every type.
// They are loaded and stored whole at any alignment (the hardware takes such accesses at element addresses).
// What a row's length leaves over (1 .. N - 1 values) is one lane's last vector, moved in pieces of 4, 2 and 1 values that have fixed
// places in the registers: N = 8: 0 .. 3, 4 .. 5 and 6; N = 4: 0 .. 1 and 2.  All tensors of a call and the per-column vectors
// use the same places, so the kernels need not know.
#pragma once
#include <hip/hip_runtime.h>

#include "element.h"

namespace capscaps {

typedef float float2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
// 16, 8, 4 and 2 bytes at addresses of elements
template <int WORDS, int ALIGN>
struct Words {
    typedef unsigned type __attribute__((ext_vector_type(WORDS)));
    typedef type at __attribute__((aligned(ALIGN)));
};

// N values as they lie in memory
template <int DT, int N>
struct Raw {
    static constexpr int SIZE = DT == CAPSCAPS_FP32 ? 4 : 2, WORDS = N * SIZE / 4;
    typedef typename Words<WORDS, SIZE>::at Whole;
    typename Words<WORDS, SIZE>::type w;
};

template <int DT, int N>
__device__ __forceinline__ void clear(Raw<DT, N>& r)
{
#pragma unroll
    for (int k = 0; k < Raw<DT, N>::WORDS; ++k) r.w[k] = 0;
}

// The piece of 4, 2 or 1 values of a row's last vector: where it lies in the vector's registers, and after how many values in memory
template <int N>
__device__ __forceinline__ constexpr int piece_place(int values)
{
    return N == 8 ? (values == 4 ? 0 : values == 2 ? 4 : 6) : (values == 2 ? 0 : 2);
}
__device__ __forceinline__ int piece_offset(int values, int tail)
{
    return values == 4 ? 0 : values == 2 ? tail & 4 : tail & 6;
}
// place of value j of the last vector
template <int N>
__device__ __forceinline__ int tail_place(int j, int tail)
{
    for (int values = 4; values > 0; values /= 2) {
        const int k = j - piece_offset(values, tail);
        if ((tail & values) && k >= 0 && k < values) return piece_place<N>(values) + k;
    }
    return 0;
}

template <int DT, int N, int VALUES>
__device__ __forceinline__ void load_piece(Raw<DT, N>& r, const char* p, int tail)
{
    if constexpr (VALUES < N) {
        if (!(tail & VALUES)) return;
        typedef Raw<DT, N> R;
        constexpr int words = VALUES * R::SIZE / 4, at = piece_place<N>(VALUES) * R::SIZE / 4;
        p += piece_offset(VALUES, tail) * R::SIZE;
        if constexpr (words == 0) {
            r.w[at] = *reinterpret_cast<const unsigned short*>(p);
        } else {
            const typename Words<words, R::SIZE>::type v = *reinterpret_cast<const typename Words<words, R::SIZE>::at*>(p);
#pragma unroll
            for (int k = 0; k < words; ++k) r.w[at + k] = v[k];
        }
    }
}
template <int DT, int N, int VALUES>
__device__ __forceinline__ void store_piece(char* p, const Raw<DT, N>& r, int tail)
{
    if constexpr (VALUES < N) {
        if (!(tail & VALUES)) return;
        typedef Raw<DT, N> R;
        constexpr int words = VALUES * R::SIZE / 4, at = piece_place<N>(VALUES) * R::SIZE / 4;
        p += piece_offset(VALUES, tail) * R::SIZE;
        if constexpr (words == 0) {
            *reinterpret_cast<unsigned short*>(p) = (unsigned short)r.w[at];
        } else {
            typename Words<words, R::SIZE>::type v;
#pragma unroll
            for (int k = 0; k < words; ++k) v[k] = r.w[at + k];
            *reinterpret_cast<typename Words<words, R::SIZE>::at*>(p) = v;
        }
    }
}

// a lane's vector: whole, the row's remainder, or nothing (the registers stay as they are)
template <int DT, int N, bool TAIL>
__device__ __forceinline__ void load(Raw<DT, N>& r, const char* p, bool full, bool part, int tail)
{
    // (rows without a remainder: lines that no other access of the wave touches, and that nothing reads again)
    if constexpr (TAIL) {
        if (full) r.w = *reinterpret_cast<const typename Raw<DT, N>::Whole*>(p);
        if (part) {
            load_piece<DT, N, 4>(r, p, tail);
            load_piece<DT, N, 2>(r, p, tail);
            load_piece<DT, N, 1>(r, p, tail);
        }
    } else if (full) {
        r.w = __builtin_nontemporal_load(reinterpret_cast<const typename Raw<DT, N>::Whole*>(p));
    }
}

template <int DT, int N>
__device__ __forceinline__ float value(const Raw<DT, N>& r, int k)  // (k is a constant after unrolling)
{
    if constexpr (DT == CAPSCAPS_FP32) {
        return __builtin_bit_cast(float, (unsigned)r.w[k]);
    } else {
        const unsigned w = r.w[k / 2];
        if constexpr (DT == CAPSCAPS_BF16)
            return __builtin_bit_cast(float, (k & 1) ? (w & 0xffff0000u) : (w << 16));
        else
            return Element<DT>::get((unsigned short)((k & 1) ? (w >> 16) : (w & 0xffffu)));
    }
}

template <int DT, int N>
__device__ __forceinline__ Raw<DT, N> pack(const float* f)
{
    Raw<DT, N> r;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        if constexpr (DT == CAPSCAPS_FP32) {
            r.w[k] = __builtin_bit_cast(unsigned, f[k]);
        } else if ((k & 1) == 0) {
            const float2v pair = {f[k], f[k + 1]};
            if constexpr (DT == CAPSCAPS_BF16)
                r.w[k / 2] = __builtin_bit_cast(unsigned, __builtin_convertvector(pair, bf16x2v));
            else
                r.w[k / 2] = __builtin_bit_cast(unsigned, __builtin_convertvector(pair, half2v));
        }
    }
    return r;
}
template <int DT, int N, bool TAIL>
__device__ __forceinline__ void store(char* p, const float* f, bool full, bool part, int tail)
{
    const Raw<DT, N> r = pack<DT, N>(f);
    if constexpr (TAIL) {
        if (full) *reinterpret_cast<typename Raw<DT, N>::Whole*>(p) = r.w;
        if (part) {
            store_piece<DT, N, 4>(p, r, tail);
            store_piece<DT, N, 2>(p, r, tail);
            store_piece<DT, N, 1>(p, r, tail);
        }
    } else if (full) {
        __builtin_nontemporal_store(r.w, reinterpret_cast<typename Raw<DT, N>::Whole*>(p));
    }
}
// a vector of a per-column fp32 tensor (`none` where there is no tensor)
template <int N, bool TAIL>
__device__ __forceinline__ void load_column(float* f, const float* p, int vector, bool full, bool part, int tail,
                                            float none)
{
#pragma unroll
    for (int h = 0; h < N / 4; ++h) {  // (quads: 16 bytes)
        Raw<CAPSCAPS_FP32, 4> r;
        clear(r);
        if (p != nullptr) {
            const float* q = p + (size_t)vector * N + 4 * h;
            if (full) r.w = *reinterpret_cast<const typename Raw<CAPSCAPS_FP32, 4>::Whole*>(q);
            if constexpr (TAIL) {
                if (part) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        // the value whose place is 4 h + k
                        const int place = 4 * h + k, values = N == 8 ? (place < 4 ? 4 : place < 6 ? 2 : 1) : (place < 2 ? 2 : 1);
                        const int j = piece_offset(values, tail) + place - piece_place<N>(values);
                        if ((tail & values) && place - piece_place<N>(values) < values)
                            r.w[k] = __builtin_bit_cast(unsigned, p[(size_t)vector * N + j]);
                    }
                }
            }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) f[4 * h + k] = p != nullptr ? value<CAPSCAPS_FP32, 4>(r, k) : none;
    }
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
