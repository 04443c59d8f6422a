// Internal: values of the three element types as fp32, one at a time, for the kernels that are not convolutions.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/capscaps.h"

namespace capscaps {

inline bool known_dtype(int dtype)
{
    return dtype == CAPSCAPS_FP32 || dtype == CAPSCAPS_BF16 || dtype == CAPSCAPS_FP16;
}
inline size_t element_bytes(int dtype) { return dtype == CAPSCAPS_FP32 ? 4 : 2; }

template <int DT>
struct Element;  // of the 16-bit types
template <>
struct Element<CAPSCAPS_BF16> {
    static __device__ __forceinline__ float get(unsigned short v)
    {
        return __builtin_bit_cast(float, (unsigned)v << 16);
    }
    // (to nearest even; one instruction for two values)
    static __device__ __forceinline__ unsigned short put(float v)
    {
        return __builtin_bit_cast(unsigned short, (__bf16)v);
    }
};
template <>
struct Element<CAPSCAPS_FP16> {
    static __device__ __forceinline__ float get(unsigned short v)
    {
        return (float)__builtin_bit_cast(_Float16, v);
    }
    static __device__ __forceinline__ unsigned short put(float v)
    {
        return __builtin_bit_cast(unsigned short, (_Float16)v);
    }
};

// ... of a type known at run time
__device__ __forceinline__ float load_element(const void* p, long long i, int dtype)
{
    if (dtype == CAPSCAPS_FP32) return static_cast<const float*>(p)[i];
    const unsigned short v = static_cast<const unsigned short*>(p)[i];
    return dtype == CAPSCAPS_BF16 ? Element<CAPSCAPS_BF16>::get(v) : Element<CAPSCAPS_FP16>::get(v);
}
__device__ __forceinline__ void store_element(void* p, long long i, float v, int dtype)
{
    if (dtype == CAPSCAPS_FP32)
        static_cast<float*>(p)[i] = v;
    else
        static_cast<unsigned short*>(p)[i] =
            dtype == CAPSCAPS_BF16 ? Element<CAPSCAPS_BF16>::put(v) : Element<CAPSCAPS_FP16>::put(v);
}

}  // namespace capscaps
