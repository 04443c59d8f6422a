// Internal: rows of values of the three element types, some values a lane, at any address.
//
// A row's values are cut into vectors of N values: 16 bytes where (nearly) all tensors of a call have 16-bit
// elements (N = 8), else N = 4: 16 bytes of fp32, 8 of a 16-bit type, so that a wave's access is one contiguous
// piece in every type. They are loaded and stored whole at any alignment (the hardware takes such accesses at
// element addresses). What a row's length leaves over (1 .. N - 1 values) is one lane's last vector.  It is
// loaded whole too, with the beginning of what follows in memory, which is masked (a load for 1, 2 and 4 values
// each would be three, and as many waits for the same lines); in a tensor's last row, and where rows are not
// apart, in pieces.  It is stored in pieces.
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

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

// The first `tail` (1 .. N - 1) values of a vector in memory, as pieces of 4, 2 and 1 values (tail is the same
// for all lanes)
template <int DT, int N, int FIRST, int VALUES>
__device__ __forceinline__ void load_piece(Raw<DT, N>& r, const char* p)
{
    typedef Raw<DT, N> R;
    constexpr int words = VALUES * R::SIZE / 4, at = FIRST * R::SIZE / 4;
    p += FIRST * R::SIZE;
    if constexpr (words == 0) {
        r.w[at] = *reinterpret_cast<const unsigned short*>(p);
    } else {
        const typename Words<words, R::SIZE>::type v = *reinterpret_cast<const typename Words<words, R::SIZE>::at*>(p);
#pragma unroll
        for (int k = 0; k < words; ++k) r.w[at + k] = v[k];
    }
}
template <int DT, int N, int FIRST, int VALUES>
__device__ __forceinline__ void store_piece(char* p, const Raw<DT, N>& r)
{
    typedef Raw<DT, N> R;
    constexpr int words = VALUES * R::SIZE / 4, at = FIRST * R::SIZE / 4;
    p += FIRST * R::SIZE;
    if constexpr (words == 0) {
        *reinterpret_cast<unsigned short*>(p) = (unsigned short)r.w[at];
    } else {
        typename Words<words, R::SIZE>::type v;
#pragma unroll
        for (int k = 0; k < words; ++k) v[k] = r.w[at + k];
        *reinterpret_cast<typename Words<words, R::SIZE>::at*>(p) = v;
    }
}
// calls f with the (first value, values) of each piece as compile-time numbers
template <int N, typename F>
__device__ __forceinline__ void pieces(int tail, F f)
{
    auto of = [&](auto first) {  // what is left after `first` values: 0 .. 3
        if (tail & 2) {
            f(first, std::integral_constant<int, 2>());
            if (tail & 1) f(std::integral_constant<int, first.value + 2>(), std::integral_constant<int, 1>());
        } else if (tail & 1) {
            f(first, std::integral_constant<int, 1>());
        }
    };
    if constexpr (N == 8) {
        if (tail & 4) {
            f(std::integral_constant<int, 0>(), std::integral_constant<int, 4>());
            of(std::integral_constant<int, 4>());
            return;
        }
    }
    of(std::integral_constant<int, 0>());
}

// What of a lane's vector is the row's: whole, `tail` values, or nothing
struct Share {
    bool full, part;
    int tail;
};

// (nothing: the registers stay as they are).  `over`: what follows the row in memory may be read
template <int DT, int N, bool TAIL>
__device__ __forceinline__ void load(Raw<DT, N>& r, const char* p, const Share& has, bool over)
{
    typedef Raw<DT, N> R;
    if constexpr (!TAIL && R::WORDS <= 4) {
        // (lines that no other access of the wave touches, and that nothing reads again)
        if (has.full) r.w = __builtin_nontemporal_load(reinterpret_cast<const typename R::Whole*>(p));
    } else if constexpr (!TAIL) {
        // (eight fp32 values are two accesses that share lines)
        if (has.full) r.w = *reinterpret_cast<const typename R::Whole*>(p);
    } else {
        if (has.full || (has.part && over)) r.w = *reinterpret_cast<const typename R::Whole*>(p);
        if (has.part && !over)
            pieces<N>(has.tail, [&](auto first, auto values) { load_piece<DT, N, first.value, values.value>(r, p); });
#pragma unroll
        for (int k = 0; k < R::WORDS; ++k) {
            const int values = has.tail - k * (4 / R::SIZE);  // of this word
            const unsigned keep = values <= 0 ? 0u : R::SIZE == 2 && values == 1 ? 0xffffu : ~0u;
            r.w[k] &= has.part ? keep : ~0u;
        }
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
__device__ __forceinline__ void store(char* p, const float* f, const Share& has)
{
    typedef Raw<DT, N> R;
    const R r = pack<DT, N>(f);
    if constexpr (TAIL) {
        if (has.full) *reinterpret_cast<typename R::Whole*>(p) = r.w;
        if (has.part)
            pieces<N>(has.tail, [&](auto first, auto values) { store_piece<DT, N, first.value, values.value>(p, r); });
    } else if (has.full) {
        __builtin_nontemporal_store(r.w, reinterpret_cast<typename R::Whole*>(p));
    }
}

// a vector of a per-column fp32 tensor (`none` where there is no tensor)
template <int N, bool TAIL>
__device__ __forceinline__ void load_column(float* f, const float* p, int vector, const Share& has, float none)
{
#pragma unroll
    for (int h = 0; h < N; h += 4) {  // (16 bytes)
        Raw<CAPSCAPS_FP32, 4> r;
        clear(r);
        if (p != nullptr) {
            const float* q = p + (size_t)vector * N + h;
            if (has.full) r.w = *reinterpret_cast<const typename Raw<CAPSCAPS_FP32, 4>::Whole*>(q);
            if constexpr (TAIL) {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (has.part && h + k < has.tail) r.w[k] = __builtin_bit_cast(unsigned, q[k]);
            }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) f[h + k] = p != nullptr ? value<CAPSCAPS_FP32, 4>(r, k) : none;
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
