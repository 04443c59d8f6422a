// Gradient norm and AdamW over many tensors.  Formulas, state formats and contracts: include/capscaps.h.
//
// Lists of tensors travel in the kernel arguments (nothing is copied to the device before a launch, so calls can be
// captured and the lists may change from call to call): a launch takes as many tensors as 4 KB of arguments hold,
// and a workgroup finds its tensor and its share of it from the running number of shares (one load and a vote).
//
// Everything here is bounded by memory.  A lane has four neighbouring values of a tensor, so that every access
// of a wave is one contiguous piece (1 KB of fp32), at any address, and a workgroup takes its share in one
// pass.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/capscaps.h"
#include "conv_shape.h"
#include "element.h"

// every product and sum below is rounded by itself: the 8-bit states then do not depend on what is fused where
#pragma clang fp contract(off)

namespace capscaps {
namespace {

constexpr int THREADS = 256;
constexpr int STATE_BLOCK = 256;  // values that share an exponent byte

typedef unsigned uint4v __attribute__((ext_vector_type(4)));
typedef unsigned uint2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef uint4v uint4_a4 __attribute__((aligned(4)));
typedef uint2v uint2_a2 __attribute__((aligned(2)));
typedef uint4v uint4_a2 __attribute__((aligned(2)));
typedef unsigned uint_a1 __attribute__((aligned(1)));
typedef uint2v uint2_a1 __attribute__((aligned(1)));

// The tensor whose shares hold number `share`: the last one that begins at or before it (`first` rises, empty tensors
// begin where the next one does)
__device__ __forceinline__ int tensor_of(const int* first, int count, int share)
{
    int k = -1;
    for (int at = 0; at < count; at += 64) {
        const int i = at + (threadIdx.x & 63);
        k += __popcll(__ballot(i < count && first[i] <= share));
    }
    return __builtin_amdgcn_readfirstlane(k);
}

// Four neighbouring values from element i on, of which `n` (1 .. 4) are the tensor's; the others are zeros
__device__ __forceinline__ float4v load4(const void* p, long long i, int n, int dtype)
{
    if (n == 4) {
        if (dtype == CAPSCAPS_FP32) {
            const uint4v w =
                __builtin_nontemporal_load(reinterpret_cast<const uint4_a4*>(static_cast<const float*>(p) + i));
            return __builtin_bit_cast(float4v, w);
        }
        const uint2v w =
            __builtin_nontemporal_load(reinterpret_cast<const uint2_a2*>(static_cast<const unsigned short*>(p) + i));
        if (dtype == CAPSCAPS_BF16)
            return float4v{__builtin_bit_cast(float, w.x << 16), __builtin_bit_cast(float, w.x & 0xffff0000u),
                           __builtin_bit_cast(float, w.y << 16), __builtin_bit_cast(float, w.y & 0xffff0000u)};
        typedef _Float16 half4v __attribute__((ext_vector_type(4)));
        return __builtin_convertvector(__builtin_bit_cast(half4v, w), float4v);
    }
    float4v v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < 3; ++k)
        if (k < n) v[k] = load_element(p, i + k, dtype);
    return v;
}
__device__ __forceinline__ void store4(void* p, long long i, const float4v& v, int n, int dtype)
{
    if (n == 4) {
        if (dtype == CAPSCAPS_FP32) {
            __builtin_nontemporal_store(__builtin_bit_cast(uint4v, v),
                                        reinterpret_cast<uint4_a4*>(static_cast<float*>(p) + i));
            return;
        }
        typedef _Float16 half4v __attribute__((ext_vector_type(4)));
        typedef __bf16 bf16x4v __attribute__((ext_vector_type(4)));
        const uint2v w = dtype == CAPSCAPS_BF16 ? __builtin_bit_cast(uint2v, __builtin_convertvector(v, bf16x4v))
                                                : __builtin_bit_cast(uint2v, __builtin_convertvector(v, half4v));
        __builtin_nontemporal_store(w, reinterpret_cast<uint2_a2*>(static_cast<unsigned short*>(p) + i));
        return;
    }
#pragma unroll
    for (int k = 0; k < 3; ++k)
        if (k < n) store_element(p, i + k, v[k], dtype);
}

bool misaligned(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }

// ------------------------------------------------------------------------------------ gradient norm
constexpr int NORM_TENSORS = 128;
// Values that a workgroup sums at a time: as many as keep four loads of each lane under way for four turns, or for one where
// that would leave units without work (7M values: 14 us, with the shorter shares 9)
constexpr int NORM_SHARE = 16384, SHORT_SHARE = 4096;
constexpr int NORM_SLOTS = CAPSCAPS_GRAD_NORM_WORKSPACE_BYTES / sizeof(double);

struct NormList {
    const void* grad[NORM_TENSORS];
    long long n[NORM_TENSORS];
    int first[NORM_TENSORS + 1];  // shares before the tensor
    unsigned char dtype[NORM_TENSORS];
    int count, share;
};

__device__ __forceinline__ double block_sum(double v, double* lds)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
    for (unsigned w = 0; w < blockDim.x / 64; ++w) v += lds[w];
    __syncthreads();
    return v;
}

// A workgroup sums a share, four loads of 16 bytes of each lane under way at a time, in fp64 (a conversion and a product-sum
// a value: half of what memory leaves time for).  113M values: 76 us at 6.0 TB/s; 4 us more for the launch that
// sums the workgroups' sums.
__global__ void __launch_bounds__(THREADS) grad_norm_kernel(NormList L, double* partial)
{
    __shared__ double lds[THREADS / 64];
    double s = 0.0;
    const int shares = L.first[L.count];
    for (int share = blockIdx.x; share < shares; share += gridDim.x) {
        const int t = tensor_of(L.first, L.count, share);
        const void* grad = L.grad[t];
        const int dtype = L.dtype[t];
        const long long base = (long long)(share - L.first[t]) * L.share, left = L.n[t] - base;
        constexpr int STEP = 4 * THREADS, UNROLL = 4;
        for (int i = 4 * threadIdx.x; i < L.share && i < left; i += UNROLL * STEP) {
            float4v g[UNROLL];
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                const long long rest = left - (i + u * STEP);
                g[u] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
                if (rest > 0) g[u] = load4(grad, base + i + u * STEP, rest < 4 ? (int)rest : 4, dtype);
            }
#pragma unroll
            for (int u = 0; u < UNROLL; ++u)
#pragma unroll
                for (int k = 0; k < 4; ++k) s += (double)g[u][k] * (double)g[u][k];
        }
    }
    s = block_sum(s, lds);
    if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

__global__ void __launch_bounds__(1024)
    grad_control_kernel(const double* partial, int count, float grad_scale, float max_norm,
                        capscaps_grad_control* control)
{
    __shared__ double lds[16];
    double s = 0.0;
    for (int k = threadIdx.x; k < count; k += 1024) s += partial[k];
    s = block_sum(s, lds);
    if (threadIdx.x != 0) return;
    const double norm = fabs((double)grad_scale) * sqrt(s);
    const bool fine = isfinite((float)norm);
    float scale = grad_scale;
    if (max_norm > 0.0f && norm > (double)max_norm) scale = (float)((double)grad_scale * ((double)max_norm / norm));
    control->norm = (float)norm;
    control->scale = fine ? scale : 0.0f;
    control->skip = fine ? 0 : 1;
    if (fine) control->step += 1;
}

// ------------------------------------------------------------------------------------ AdamW
constexpr int ADAM_TENSORS = 44;
// Fours of values that a lane updates, and a workgroup's share.  113M values with fp16 copies, us: 32-bit
// moments 648, 614 and 592 with one, two and four of them; 8-bit ones, read back after the step, 447 with two and 465
// with four, 7M values 38.0 and 39.4
constexpr int units_of(int bits) { return bits == 8 ? 2 : 4; }
constexpr int share_of(int bits) { return units_of(bits) * 4 * THREADS; }
constexpr int VALUES_SHARE = 16 * THREADS;  // values that a workgroup decodes

struct AdamTensor {
    float* param;
    const void* grad;
    void *m, *v;
    unsigned char *m_exp, *v_exp;
    void* copy;
    long long n;
    float weight_decay;
    unsigned short grad_dtype, copy_dtype;
};
struct AdamList {
    AdamTensor t[ADAM_TENSORS];
    int first[ADAM_TENSORS + 1];  // shares before the tensor
    int count;
    int index0;  // of t[0] in the caller's list
};
struct AdamHyper {
    float lr, beta1, beta2, one_minus_beta1, one_minus_beta2, eps;
    float log_beta1, log_beta2;  // for a step that is counted on the device
    float bias1, inv_sqrt_bias2;  // for one that the host counts
    int step;                     // 0: the device's
    unsigned seed;
    const capscaps_grad_control* control;
};
// What a step needs of the host's or the device's counters
struct AdamStep {
    int skip;
    float scale, step_size, inv_sqrt_bias2;
    int t;
};
__device__ __forceinline__ AdamStep adam_step(const AdamHyper& H)
{
    AdamStep s{0, 1.0f, 0.0f, H.inv_sqrt_bias2, H.step};
    float bias1 = H.bias1;
    if (H.control != nullptr) {
        s.skip = H.control->skip != 0;
        s.scale = H.control->scale;
        if (H.step == 0) {
            s.t = H.control->step;
            s.skip |= s.t < 1;  // none has been counted
            bias1 = -expm1f((float)s.t * H.log_beta1);
            s.inv_sqrt_bias2 = 1.0f / sqrtf(-expm1f((float)s.t * H.log_beta2));
        }
    }
    s.step_size = H.lr / bias1;
    return s;
}

// 32 bits from 32: every bit of the argument reaches every bit of the result.  The factors are the fractional parts
// of the square roots of 2 and 3, which have no pattern.
__host__ __device__ __forceinline__ unsigned mix(unsigned x)
{
    x ^= x >> 16;
    x *= 0x6A09E667u;
    x ^= x >> 15;
    x *= 0xBB67AE85u;
    return x ^ (x >> 16);
}

// 8-bit codes (capscaps.h): `below` is the number of octaves below the shared exponent.  A block's exponent is
// the same for a wave, so what depends on it alone is in scalar registers.
__device__ __forceinline__ float decode_magnitude(unsigned c, int exponent, int below)
{
    const unsigned bits = c == 0 ? 0u : (c << 20) + ((unsigned)(exponent - below) << 23);
    return __builtin_bit_cast(float, exponent == 255 ? 0x7fc00000u : bits);
}
// (the code is the lowest byte of `c`)
__device__ __forceinline__ float decode_m(unsigned c, int exponent)
{
    const float v = decode_magnitude(c & 127u, exponent, 15);
    return __builtin_bit_cast(float, __builtin_bit_cast(unsigned, v) | ((c << 24) & 0x80000000u));
}
// The exponent that a block with the largest magnitude `top` (as bits) shares: one more where three bits of mantissa
// cannot reach it, at least what keeps all codes normal numbers
__device__ __forceinline__ int shared_exponent(unsigned top, int below)
{
    if (top >= 0x7f800000u) return 255;
    const int e = (int)((top + 0xfffffu) >> 23);
    return e < below + 1 ? below + 1 : e > 254 ? 254 : e;
}
// `random`: 20 bits, of which the upper 16 count; a carry out of the 20 bits of mantissa that are cut off rounds up
__device__ __forceinline__ int encode_magnitude(unsigned bits, unsigned random, int exponent, int below)
{
    return (int)((bits + random) >> 20) - 8 * (exponent - below);
}
__device__ __forceinline__ int between(int c, int least, int most) { return c < least ? least : c > most ? most : c; }
__device__ __forceinline__ unsigned encode_m(float v, unsigned random, int exponent)
{
    const unsigned bits = __builtin_bit_cast(unsigned, v);
    const int c = encode_magnitude(bits & 0x7fffffffu, random, exponent, 15);
    return (unsigned)between(c, 0, 127) | ((bits >> 24) & 128u);
}
__device__ __forceinline__ unsigned encode_v(float v, unsigned random, int exponent)
{
    const unsigned bits = __builtin_bit_cast(unsigned, v);  // (never negative)
    return (unsigned)between(encode_magnitude(bits, random, exponent, 31), bits != 0 ? 1 : 0, 255);
}

struct Moments {
    float p, m, v;
};
// FAST: v_sqrt_f32 and v_rcp_f32, which are off by one unit in the last place, of a step that is added to p.  They take
// subnormal numbers for 0, so this is for an eps against which the root of such a v is nothing (fast_quotient).
template <bool FAST>
__device__ __forceinline__ Moments adam_value(const AdamHyper& H, const AdamStep& S, float keep, float p, float g,
                                              float m, float v)
{
    g = g * S.scale;
    m = m * H.beta1 + g * H.one_minus_beta1;
    v = v * H.beta2 + (g * g) * H.one_minus_beta2;
    const float root = FAST ? __builtin_amdgcn_sqrtf(v) : sqrtf(v), under = root * S.inv_sqrt_bias2 + H.eps;
    p = p * keep - S.step_size * (FAST ? m * __builtin_amdgcn_rcpf(under) : m / under);
    return {p, m, v};
}
// v below 2^-126 has a root below 2^-63, which the bias correction makes at most 1 / sqrt(1 - beta2) times as large:
// less than half a unit in the last place of eps if eps * sqrt(1 - beta2) is at least 2^-39 (beta2 = 0.999: eps from
// 5.8e-11 on; 113M values with 8-bit moments: 329 us, with the exact root and quotient 336).  Past 2^100 the quotient's
// divisor could have a subnormal reciprocal.
bool fast_quotient(double eps, double beta2) { return eps * sqrt(1.0 - beta2) >= 0x1p-39 && eps <= 0x1p100; }

template <int CTRL>
__device__ __forceinline__ unsigned dpp_max(unsigned v)
{
    const unsigned w = (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
    return v > w ? v : w;
}
// largest over the wave, in a scalar register
__device__ __forceinline__ unsigned wave_max(unsigned v)
{
    v = dpp_max<0xB1>(v);   // quad_perm 1 0 3 2
    v = dpp_max<0x4E>(v);   // quad_perm 2 3 0 1
    v = dpp_max<0x141>(v);  // row_half_mirror
    v = dpp_max<0x140>(v);  // row_mirror: the largest of 16 lanes in each of them
    auto row = [&](int lane) { return (unsigned)__builtin_amdgcn_readlane((int)v, lane); };
    const unsigned a = row(0), b = row(16), c = row(32), d = row(48);
    const unsigned ab = a > b ? a : b, cd = c > d ? c : d;
    return ab > cd ? ab : cd;
}

// Four codes, a byte each; `n` of them are the tensor's
__device__ __forceinline__ unsigned load_codes(const unsigned char* p, long long i, int n)
{
    if (n == 4) return __builtin_nontemporal_load(reinterpret_cast<const uint_a1*>(p + i));
    unsigned c = 0;
#pragma unroll
    for (int k = 0; k < 3; ++k)
        if (k < n) c |= (unsigned)p[i + k] << (8 * k);
    return c;
}
__device__ __forceinline__ void store_codes(unsigned char* p, long long i, unsigned c, int n)
{
    if (n == 4) {
        __builtin_nontemporal_store(c, reinterpret_cast<uint_a1*>(p + i));
        return;
    }
#pragma unroll
    for (int k = 0; k < 3; ++k)
        if (k < n) p[i + k] = (unsigned char)(c >> (8 * k));
}

// A share of a tensor: each wave 256 neighbouring values at a time, which in 8 bits are a block of the state,
// so that the largest magnitudes are the wave's and nothing waits for other waves.  WHOLE: the share lies
// within the tensor.
//
// Bounded by memory, with 8-bit moments only just: decoding, two correctly rounded moments and encoding with
// random bits are some eighty vector instructions a value (113M values: 332 us at 6.1 TB/s; 380 with a quotient
// and a square root rounded to the last bit, 64-bit addresses and a product for each value's random bits).  So
// the bits come from sums, the square root and the quotient from the fast instructions, and exponents,
// addresses and the step's factors are scalars.
template <int BITS, bool FAST, bool WHOLE>
__device__ __forceinline__ void adamw_share(const AdamTensor& T, const AdamHyper& H, unsigned key, long long base,
                                            AdamStep* shared_step)
{
    static_assert(STATE_BLOCK == 4 * 64, "a wave's values share an exponent");
    constexpr int UNITS = units_of(BITS);
    // this wave's values: from here, and each 4 * THREADS on
    const long long i0 = base + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * STATE_BLOCK;
    const int lane4 = 4 * (threadIdx.x & 63);
    float4v p[UNITS], g[UNITS], m[UNITS], v[UNITS];
    unsigned cm[UNITS], cv[UNITS];
    int em[UNITS], ev[UNITS];
    auto count = [&](int u) {  // of a lane's four values, the tensor's
        if (WHOLE) return 4;
        const long long rest = T.n - (i0 + u * 4 * THREADS + lane4);
        return rest >= 4 ? 4 : rest > 0 ? (int)rest : 0;
    };
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        const long long first = i0 + u * 4 * THREADS;
        const int n = count(u);
        p[u] = g[u] = m[u] = v[u] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
        cm[u] = cv[u] = em[u] = ev[u] = 0;
        if (!WHOLE && first >= T.n) break;
        if constexpr (BITS == 8) {
            em[u] = __builtin_amdgcn_readfirstlane(T.m_exp[first / STATE_BLOCK]);
            ev[u] = __builtin_amdgcn_readfirstlane(T.v_exp[first / STATE_BLOCK]);
        }
        if (n == 0) continue;
        p[u] = load4(T.param + first, lane4, n, CAPSCAPS_FP32);
        g[u] = load4(static_cast<const char*>(T.grad) + first * (T.grad_dtype == CAPSCAPS_FP32 ? 4 : 2), lane4, n,
                     T.grad_dtype);
        if constexpr (BITS == 8) {
            cm[u] = load_codes(static_cast<const unsigned char*>(T.m) + first, lane4, n);
            cv[u] = load_codes(static_cast<const unsigned char*>(T.v) + first, lane4, n);
        } else {
            m[u] = load4(static_cast<const float*>(T.m) + first, lane4, n, CAPSCAPS_FP32);
            v[u] = load4(static_cast<const float*>(T.v) + first, lane4, n, CAPSCAPS_FP32);
        }
    }
    // (the loads above are under way while one wave computes the step's factors)
    if (threadIdx.x < 64) {
        const AdamStep s = adam_step(H);
        if (threadIdx.x == 0) *shared_step = s;
    }
    __syncthreads();
    AdamStep S = *shared_step;
    S.skip = __builtin_amdgcn_readfirstlane(S.skip);
    S.t = __builtin_amdgcn_readfirstlane(S.t);
    if (S.skip) return;
    const float keep = 1.0f - H.lr * T.weight_decay;
    key = mix(key + 0x6A09E667u * mix((unsigned)S.t));
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        const long long first = i0 + u * 4 * THREADS;
        const int n = count(u);
        if (!WHOLE && first >= T.n) break;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (BITS == 8) {
                m[u][j] = decode_m(cm[u] >> (8 * j), em[u]);
                v[u][j] = decode_magnitude((cv[u] >> (8 * j)) & 255u, ev[u], 31);
            }
            const Moments r = adam_value<FAST>(H, S, keep, p[u][j], g[u][j], m[u][j], v[u][j]);
            p[u][j] = r.p;
            m[u][j] = r.m;
            v[u][j] = r.v;
        }
        if (n > 0) {
            store4(T.param + first, lane4, p[u], n, CAPSCAPS_FP32);
            if (T.copy != nullptr) store4(static_cast<unsigned short*>(T.copy) + first, lane4, p[u], n, T.copy_dtype);
        }
        if constexpr (BITS == 8) {
            unsigned top_m = 0, top_v = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float mj = m[u][j], vj = v[u][j];  // (a bit cast of a vector's element takes the first one)
                // (values past the tensor's end count for nothing)
                const unsigned am = WHOLE || j < n ? __builtin_bit_cast(unsigned, mj) & 0x7fffffffu : 0u;
                const unsigned av = WHOLE || j < n ? __builtin_bit_cast(unsigned, vj) : 0u;
                top_m = top_m > am ? top_m : am;
                top_v = top_v > av ? top_v : av;
            }
            const int new_em = shared_exponent(wave_max(top_m), 15), new_ev = shared_exponent(wave_max(top_v), 31);
            // (a third factor for the high half of an index that passes 32 bits; 256 values never cross that line)
            const unsigned at = (unsigned)first * 0x9E3779B1u + (unsigned)(first >> 32) * 0xBB67AE85u + key;
            const unsigned x0 = (unsigned)lane4 * 0x9E3779B1u + at;
            unsigned new_m = 0, new_v = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const unsigned x = mix(x0 + (unsigned)j * 0x9E3779B1u);
                new_m |= encode_m(m[u][j], (x & 0xffffu) << 4, new_em) << (8 * j);
                new_v |= encode_v(v[u][j], (x >> 16) << 4, new_ev) << (8 * j);
            }
            if (n > 0) {
                store_codes(static_cast<unsigned char*>(T.m) + first, lane4, new_m, n);
                store_codes(static_cast<unsigned char*>(T.v) + first, lane4, new_v, n);
            }
            if (lane4 == 0) {
                T.m_exp[first / STATE_BLOCK] = (unsigned char)new_em;
                T.v_exp[first / STATE_BLOCK] = (unsigned char)new_ev;
            }
        } else if (n > 0) {
            store4(static_cast<float*>(T.m) + first, lane4, m[u], n, CAPSCAPS_FP32);
            store4(static_cast<float*>(T.v) + first, lane4, v[u], n, CAPSCAPS_FP32);
        }
    }
}

template <int BITS, bool FAST>
__global__ void __launch_bounds__(THREADS) adamw_kernel(AdamList L, AdamHyper H)
{
    __shared__ AdamStep step;
    const int k = tensor_of(L.first, L.count, blockIdx.x);
    const AdamTensor& T = L.t[k];
    const unsigned key = H.seed + 0x9E3779B1u * (unsigned)(L.index0 + k);
    const long long base = (long long)((int)blockIdx.x - L.first[k]) * share_of(BITS);
    if (base + share_of(BITS) <= T.n)
        adamw_share<BITS, FAST, true>(T, H, key, base, &step);
    else
        adamw_share<BITS, FAST, false>(T, H, key, base, &step);
}

struct ValuesList {
    const unsigned char *m[ADAM_TENSORS], *v[ADAM_TENSORS], *m_exp[ADAM_TENSORS], *v_exp[ADAM_TENSORS];
    unsigned short *m_out[ADAM_TENSORS], *v_out[ADAM_TENSORS];
    long long n[ADAM_TENSORS];
    int first[ADAM_TENSORS + 1];
    int count;
};

// Eight codes to 16 bytes of bfloat16 (the lower 16 bits of every value are zero)
template <bool M>
__device__ __forceinline__ void decode8(uint2v codes, unsigned exponent, unsigned short* out)
{
    auto bits = [&](unsigned c) {
        const float v = M ? decode_m(c, exponent) : decode_magnitude(c, exponent, 31);
        return __builtin_bit_cast(unsigned, v) >> 16;
    };
    uint4v w;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const unsigned pair = codes[k / 2] >> (16 * (k & 1));
        w[k] = bits(pair & 255u) | bits((pair >> 8) & 255u) << 16;
    }
    __builtin_nontemporal_store(w, reinterpret_cast<uint4_a2*>(out));
}

// (113M values of each moment: 114 us at 6.0 TB/s; 147 with the loads of a share one after another)
__global__ void __launch_bounds__(THREADS) state_values_kernel(ValuesList L)
{
    const int k = tensor_of(L.first, L.count, blockIdx.x);
    const long long base = (long long)((int)blockIdx.x - L.first[k]) * VALUES_SHARE;
    constexpr int UNITS = VALUES_SHARE / (8 * THREADS);
    const long long n = L.n[k];
    const unsigned char *m = L.m[k], *v = L.v[k], *m_exp = L.m_exp[k], *v_exp = L.v_exp[k];
    unsigned short *m_out = L.m_out[k], *v_out = L.v_out[k];
    uint2v cm[UNITS], cv[UNITS];
    unsigned em[UNITS], ev[UNITS];
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        const long long i = base + 8 * (u * THREADS + threadIdx.x);
        if (i + 8 > n) continue;
        cm[u] = __builtin_nontemporal_load(reinterpret_cast<const uint2_a1*>(m + i));
        cv[u] = __builtin_nontemporal_load(reinterpret_cast<const uint2_a1*>(v + i));
        em[u] = m_exp[i / STATE_BLOCK];
        ev[u] = v_exp[i / STATE_BLOCK];
    }
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        const long long i = base + 8 * (u * THREADS + threadIdx.x);
        if (i + 8 <= n) {
            decode8<true>(cm[u], em[u], m_out + i);
            decode8<false>(cv[u], ev[u], v_out + i);
        } else {
            for (long long j = i; j < n; ++j) {
                store_element(m_out, j, decode_m(m[j], m_exp[j / STATE_BLOCK]), CAPSCAPS_BF16);
                store_element(v_out, j, decode_magnitude(v[j], v_exp[j / STATE_BLOCK], 31), CAPSCAPS_BF16);
            }
        }
    }
}

// Adds the shares of a tensor of n values; false: more workgroups of 256 than a launch takes (less than 2^32 threads)
constexpr long long MOST_SHARES = (1LL << 24) - 1;
bool add_shares(int* first, int count, long long n, int share)
{
    const long long total = first[count] + (n + share - 1) / share;
    if (total > MOST_SHARES) return false;
    first[count + 1] = (int)total;
    return true;
}

}  // namespace
}  // namespace capscaps

using namespace capscaps;

extern "C" {

int capscaps_grad_norm(const capscaps_grad_tensor* grads, int count, float grad_scale, float max_norm,
                       capscaps_grad_control* control, void* workspace, size_t workspace_bytes, void* stream)
{
    if (count < 0 || (count > 0 && grads == nullptr) || control == nullptr || misaligned(control, 16))
        return CAPSCAPS_EINVAL;
    if (!isfinite(grad_scale) || isnan(max_norm)) return CAPSCAPS_EINVAL;
    long long used = 0, shares = 0, values = 0;
    for (int k = 0; k < count; ++k) {
        const capscaps_grad_tensor& g = grads[k];
        if (g.n < 0 || !known_dtype(g.dtype)) return CAPSCAPS_EINVAL;
        if (g.n > 0 && (g.grad == nullptr || misaligned(g.grad, element_bytes(g.dtype)))) return CAPSCAPS_EINVAL;
        shares += g.n / NORM_SHARE + 1;
        if (shares > MOST_SHARES) return CAPSCAPS_EUNSUPPORTED;  // (so that every launch's can be counted)
        used += g.n > 0;
        values += g.n;
    }
    if (workspace == nullptr || workspace_bytes < CAPSCAPS_GRAD_NORM_WORKSPACE_BYTES) return CAPSCAPS_EWORKSPACE;
    if (misaligned(workspace, 16)) return CAPSCAPS_EINVAL;
    const long long launches = (used + NORM_TENSORS - 1) / NORM_TENSORS;
    if (launches > NORM_SLOTS) return CAPSCAPS_EUNSUPPORTED;
    const int most = launches > 0 ? (int)(NORM_SLOTS / launches) : 0;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    double* partial = static_cast<double*>(workspace);
    int slots = 0;
    for (int k = 0; k < count;) {
        NormList L;
        L.share = values < 2048LL * NORM_SHARE ? SHORT_SHARE : NORM_SHARE;
        L.count = 0;
        L.first[0] = 0;
        for (; k < count && L.count < NORM_TENSORS; ++k) {
            if (grads[k].n == 0) continue;
            add_shares(L.first, L.count, grads[k].n, L.share);
            L.grad[L.count] = grads[k].grad;
            L.n[L.count] = grads[k].n;
            L.dtype[L.count] = (unsigned char)grads[k].dtype;
            ++L.count;
        }
        if (L.count == 0) break;
        const int blocks = L.first[L.count] < most ? L.first[L.count] : most;
        grad_norm_kernel<<<dim3(blocks), dim3(THREADS), 0, st>>>(L, partial + slots);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return status_from_hip(err);
        slots += blocks;
    }
    grad_control_kernel<<<dim3(1), dim3(1024), 0, st>>>(partial, slots, grad_scale, max_norm, control);
    return status_from_hip(hipGetLastError());
}

int capscaps_adamw_step(const capscaps_adamw_tensor* tensors, int count, int state_bits, double lr, double beta1,
                        double beta2, double eps, long long step, unsigned seed, const capscaps_grad_control* control,
                        void* stream)
{
    if (count < 0 || (count > 0 && tensors == nullptr) || (state_bits != 32 && state_bits != 8))
        return CAPSCAPS_EINVAL;
    if (!isfinite(lr) || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps > 0.0) ||
        !isfinite(eps) || !((float)eps > 0.0f))
        return CAPSCAPS_EINVAL;
    if (step < 0 || step > 0x7fffffffLL || (step == 0 && control == nullptr) || misaligned(control, 16))
        return CAPSCAPS_EINVAL;
    for (int k = 0; k < count; ++k) {
        const capscaps_adamw_tensor& t = tensors[k];
        if (t.n < 0 || !isfinite(t.weight_decay) || !known_dtype(t.grad_dtype)) return CAPSCAPS_EINVAL;
        if (t.copy != nullptr && t.copy_dtype != CAPSCAPS_BF16 && t.copy_dtype != CAPSCAPS_FP16)
            return CAPSCAPS_EINVAL;
        if (t.n == 0) continue;
        if (!t.param || !t.grad || !t.m || !t.v || misaligned(t.param, 4) ||
            misaligned(t.grad, element_bytes(t.grad_dtype)) || misaligned(t.copy, 2))
            return CAPSCAPS_EINVAL;
        if (state_bits == 8 ? !t.m_exp || !t.v_exp : misaligned(t.m, 4) || misaligned(t.v, 4)) return CAPSCAPS_EINVAL;
        if (t.n > MOST_SHARES * share_of(state_bits)) return CAPSCAPS_EUNSUPPORTED;
    }
    AdamHyper H;
    H.lr = (float)lr;
    H.beta1 = (float)beta1;
    H.beta2 = (float)beta2;
    H.one_minus_beta1 = (float)(1.0 - beta1);
    H.one_minus_beta2 = (float)(1.0 - beta2);
    H.eps = (float)eps;
    H.log_beta1 = (float)log(beta1);  // (beta = 0: minus infinity, and 1 - beta^t is 1)
    H.log_beta2 = (float)log(beta2);
    H.bias1 = (float)(1.0 - pow(beta1, (double)step));
    H.inv_sqrt_bias2 = (float)(1.0 / sqrt(1.0 - pow(beta2, (double)step)));
    H.step = (int)step;
    H.seed = seed;
    H.control = control;
    const bool fast = fast_quotient(eps, beta2);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    for (int k = 0; k < count;) {
        AdamList L;
        L.count = 0;
        L.index0 = k;
        L.first[0] = 0;
        // (empty tensors take a place, so that t[j] is the caller's tensor index0 + j)
        for (; k < count && L.count < ADAM_TENSORS; ++k) {
            const capscaps_adamw_tensor& t = tensors[k];
            if (!add_shares(L.first, L.count, t.n, share_of(state_bits))) break;  // (the next launch's)
            L.t[L.count] = {t.param, t.grad, t.m, t.v, t.m_exp, t.v_exp, t.copy, t.n, t.weight_decay,
                            (unsigned short)t.grad_dtype, (unsigned short)t.copy_dtype};
            ++L.count;
        }
        if (L.first[L.count] == 0) continue;
        const dim3 grid(L.first[L.count]);
        const auto kernel = state_bits == 8 ? fast ? adamw_kernel<8, true> : adamw_kernel<8, false>
                            : fast          ? adamw_kernel<32, true>
                                            : adamw_kernel<32, false>;
        kernel<<<grid, dim3(THREADS), 0, st>>>(L, H);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return status_from_hip(err);
    }
    return CAPSCAPS_OK;
}

int capscaps_adamw_state_values(const capscaps_adamw_tensor* tensors, int count, void* const* m_out,
                                void* const* v_out, void* stream)
{
    if (count < 0 || (count > 0 && (tensors == nullptr || m_out == nullptr || v_out == nullptr)))
        return CAPSCAPS_EINVAL;
    for (int k = 0; k < count; ++k) {
        const capscaps_adamw_tensor& t = tensors[k];
        if (t.n < 0) return CAPSCAPS_EINVAL;
        if (t.n == 0) continue;
        if (!t.m || !t.v || !t.m_exp || !t.v_exp || !m_out[k] || !v_out[k] || misaligned(m_out[k], 2) ||
            misaligned(v_out[k], 2))
            return CAPSCAPS_EINVAL;
        if (t.n > MOST_SHARES * VALUES_SHARE) return CAPSCAPS_EUNSUPPORTED;
    }
    const hipStream_t st = static_cast<hipStream_t>(stream);
    for (int k = 0; k < count;) {
        ValuesList L;
        L.count = 0;
        L.first[0] = 0;
        for (; k < count && L.count < ADAM_TENSORS; ++k) {
            const capscaps_adamw_tensor& t = tensors[k];
            if (t.n == 0) continue;
            const int j = L.count;
            if (!add_shares(L.first, j, t.n, VALUES_SHARE)) break;  // (the next launch's)
            ++L.count;
            L.m[j] = static_cast<const unsigned char*>(t.m);
            L.v[j] = static_cast<const unsigned char*>(t.v);
            L.m_exp[j] = t.m_exp;
            L.v_exp[j] = t.v_exp;
            L.m_out[j] = static_cast<unsigned short*>(m_out[k]);
            L.v_out[j] = static_cast<unsigned short*>(v_out[k]);
            L.n[j] = t.n;
        }
        if (L.count == 0) break;
        state_values_kernel<<<dim3(L.first[L.count]), dim3(THREADS), 0, st>>>(L);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return status_from_hip(err);
    }
    return CAPSCAPS_OK;
}

}  // extern "C"
