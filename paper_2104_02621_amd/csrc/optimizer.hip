// Gradient norm and AdamW over many tensors.  Formulas, state formats and contracts: include/capscaps.h.
//
// Lists of tensors travel in the kernel arguments (nothing is copied to the device before a launch, so calls can be
// captured and the lists may change from call to call): a launch takes as many tensors as 4 KB of arguments hold,
// and a workgroup finds its tensor and its share of it from the running number of shares.
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

bool misaligned(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }

// ------------------------------------------------------------------------------------ gradient norm
constexpr int NORM_TENSORS = 128;
constexpr int NORM_SHARE = 16384;  // values that a workgroup sums at a time
constexpr int NORM_SLOTS = CAPSCAPS_GRAD_NORM_WORKSPACE_BYTES / sizeof(double);

struct NormList {
    const void* grad[NORM_TENSORS];
    long long n[NORM_TENSORS];
    int first[NORM_TENSORS + 1];  // shares before the tensor
    unsigned char dtype[NORM_TENSORS];
    int count;
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

__global__ void __launch_bounds__(THREADS) grad_norm_kernel(NormList L, double* partial)
{
    __shared__ double lds[THREADS / 64];
    double s = 0.0;
    for (int k = blockIdx.x; k < L.first[L.count]; k += gridDim.x) {
        int t = 0;
        while (L.first[t + 1] <= k) ++t;
        const long long i0 = (long long)(k - L.first[t]) * NORM_SHARE;
        const long long i1 = i0 + NORM_SHARE < L.n[t] ? i0 + NORM_SHARE : L.n[t];
        for (long long i = i0 + threadIdx.x; i < i1; i += THREADS) {
            const double g = load_element(L.grad[t], i, L.dtype[t]);
            s += g * g;
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
constexpr int ADAM_SHARE = 2048;  // values that a workgroup updates

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
    bool skip;
    float scale, step_size, inv_sqrt_bias2;
    int t;
};
__device__ __forceinline__ AdamStep adam_step(const AdamHyper& H)
{
    AdamStep s{false, 1.0f, 0.0f, H.inv_sqrt_bias2, H.step};
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

// 8-bit codes (capscaps.h): `below` is the number of octaves below the shared exponent
__device__ __forceinline__ float decode_magnitude(unsigned c, int exponent, int below)
{
    if (exponent == 255) return __builtin_nanf("");
    return c == 0 ? 0.0f : __builtin_bit_cast(float, (c + 8u * (unsigned)(exponent - below)) << 20);
}
__device__ __forceinline__ float decode_m(unsigned c, int exponent)
{
    const float v = decode_magnitude(c & 127u, exponent, 15);
    return (c & 128u) != 0 ? -v : v;
}
// The exponent that a block with the largest magnitude `top` (as bits) shares: one more where three bits of mantissa
// cannot reach it, at least what keeps all codes normal numbers
__device__ __forceinline__ int shared_exponent(unsigned top, int below)
{
    if (top >= 0x7f800000u) return 255;
    const int e = (int)((top + 0xfffffu) >> 23);
    return e < below + 1 ? below + 1 : e > 254 ? 254 : e;
}
// `random`: 16 bits; a carry out of the 20 bits of mantissa that are cut off rounds up
__device__ __forceinline__ int encode_magnitude(unsigned bits, unsigned random, int exponent, int below)
{
    return (int)((bits + (random << 4)) >> 20) - 8 * (exponent - below);
}
__device__ __forceinline__ unsigned encode_m(float v, unsigned random, int exponent)
{
    const unsigned bits = __builtin_bit_cast(unsigned, v);
    const int c = encode_magnitude(bits & 0x7fffffffu, random, exponent, 15);
    return (unsigned)(c < 0 ? 0 : c > 127 ? 127 : c) | (v < 0.0f ? 128u : 0u);
}
__device__ __forceinline__ unsigned encode_v(float v, unsigned random, int exponent)
{
    const unsigned bits = __builtin_bit_cast(unsigned, v) & 0x7fffffffu;
    const int c = encode_magnitude(bits, random, exponent, 31), least = bits != 0 ? 1 : 0;
    return (unsigned)(c < least ? least : c > 255 ? 255 : c);
}

struct Moments {
    float p, m, v;
};
__device__ __forceinline__ Moments adam_value(const AdamHyper& H, const AdamStep& S, float keep, float p, float g,
                                              float m, float v)
{
    g = g * S.scale;
    m = m * H.beta1 + g * H.one_minus_beta1;
    v = v * H.beta2 + (g * g) * H.one_minus_beta2;
    p = p * keep - S.step_size * (m / (sqrtf(v) * S.inv_sqrt_bias2 + H.eps));
    return {p, m, v};
}

__device__ __forceinline__ unsigned block_max(unsigned v, unsigned* lds)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const unsigned w = (unsigned)__shfl_xor((int)v, o);
        v = v > w ? v : w;
    }
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
    for (int w = 1; w < THREADS / 64; ++w) v = v > lds[w] ? v : lds[w];
    __syncthreads();
    return v;
}

template <int BITS>
__global__ void __launch_bounds__(THREADS) adamw_kernel(AdamList L, AdamHyper H)
{
    __shared__ unsigned lds[THREADS / 64];
    int k = 0;
    while (L.first[k + 1] <= (int)blockIdx.x) ++k;
    const AdamTensor& T = L.t[k];
    const AdamStep S = adam_step(H);
    if (S.skip) return;
    const float keep = 1.0f - H.lr * T.weight_decay;
    const unsigned key = mix(H.seed + 0x9E3779B1u * (unsigned)(L.index0 + k) + 0x6A09E667u * mix((unsigned)S.t));
    const long long base = (long long)((int)blockIdx.x - L.first[k]) * ADAM_SHARE;
    for (int j = 0; j < ADAM_SHARE / THREADS; ++j) {
        const long long i = base + j * THREADS + threadIdx.x, block = i / STATE_BLOCK;
        if (base + j * THREADS >= T.n) break;
        const bool in = i < T.n;
        Moments r{0.0f, 0.0f, 0.0f};
        if (in) {
            const float p = T.param[i], g = load_element(T.grad, i, T.grad_dtype);
            float m, v;
            if constexpr (BITS == 8) {
                m = decode_m(static_cast<const unsigned char*>(T.m)[i], T.m_exp[block]);
                v = decode_magnitude(static_cast<const unsigned char*>(T.v)[i], T.v_exp[block], 31);
            } else {
                m = static_cast<const float*>(T.m)[i];
                v = static_cast<const float*>(T.v)[i];
            }
            r = adam_value(H, S, keep, p, g, m, v);
            T.param[i] = r.p;
            if (T.copy != nullptr) store_element(T.copy, i, r.p, T.copy_dtype);
        }
        if constexpr (BITS == 8) {
            static_assert(THREADS == STATE_BLOCK, "a value per thread");
            const unsigned top_m = block_max(__builtin_bit_cast(unsigned, r.m) & 0x7fffffffu, lds);
            const unsigned top_v = block_max(__builtin_bit_cast(unsigned, r.v) & 0x7fffffffu, lds);
            const int em = shared_exponent(top_m, 15), ev = shared_exponent(top_v, 31);
            // (a third factor for the high half of an index that passes 32 bits)
            const unsigned x = mix((unsigned)i * 0x9E3779B1u + (unsigned)(i >> 32) * 0xBB67AE85u + key);
            if (in) {
                static_cast<unsigned char*>(T.m)[i] = (unsigned char)encode_m(r.m, x & 0xffffu, em);
                static_cast<unsigned char*>(T.v)[i] = (unsigned char)encode_v(r.v, x >> 16, ev);
            }
            if (threadIdx.x == 0) {
                T.m_exp[block] = (unsigned char)em;
                T.v_exp[block] = (unsigned char)ev;
            }
        } else if (in) {
            static_cast<float*>(T.m)[i] = r.m;
            static_cast<float*>(T.v)[i] = r.v;
        }
    }
}

struct ValuesList {
    const unsigned char *m[ADAM_TENSORS], *v[ADAM_TENSORS], *m_exp[ADAM_TENSORS], *v_exp[ADAM_TENSORS];
    unsigned short *m_out[ADAM_TENSORS], *v_out[ADAM_TENSORS];
    long long n[ADAM_TENSORS];
    int first[ADAM_TENSORS + 1];
    int count;
};

__global__ void __launch_bounds__(THREADS) state_values_kernel(ValuesList L)
{
    int k = 0;
    while (L.first[k + 1] <= (int)blockIdx.x) ++k;
    const long long base = (long long)((int)blockIdx.x - L.first[k]) * ADAM_SHARE;
    for (int j = 0; j < ADAM_SHARE / THREADS; ++j) {
        const long long i = base + j * THREADS + threadIdx.x, block = i / STATE_BLOCK;
        if (i >= L.n[k]) break;
        store_element(L.m_out[k], i, decode_m(L.m[k][i], L.m_exp[k][block]), CAPSCAPS_BF16);
        store_element(L.v_out[k], i, decode_magnitude(L.v[k][i], L.v_exp[k][block], 31), CAPSCAPS_BF16);
    }
}

// adds the shares of a tensor of n values; false: more than a launch can count
bool add_shares(int* first, int count, long long n, int share)
{
    const long long total = first[count] + (n + share - 1) / share;
    if (total > 0x7fffffffLL) return false;
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
    long long used = 0;
    for (int k = 0; k < count; ++k) {
        const capscaps_grad_tensor& g = grads[k];
        if (g.n < 0 || !known_dtype(g.dtype)) return CAPSCAPS_EINVAL;
        if (g.n > 0 && (g.grad == nullptr || misaligned(g.grad, element_bytes(g.dtype)))) return CAPSCAPS_EINVAL;
        if (g.n > (0x7fffffffLL / NORM_TENSORS - 1) * NORM_SHARE) return CAPSCAPS_EUNSUPPORTED;
        used += g.n > 0;
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
        L.count = 0;
        L.first[0] = 0;
        for (; k < count && L.count < NORM_TENSORS; ++k) {
            if (grads[k].n == 0) continue;
            L.grad[L.count] = grads[k].grad;
            L.n[L.count] = grads[k].n;
            L.dtype[L.count] = (unsigned char)grads[k].dtype;
            add_shares(L.first, L.count, grads[k].n, NORM_SHARE);
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
        if (t.n > (0x7fffffffLL / ADAM_TENSORS - 1) * ADAM_SHARE) return CAPSCAPS_EUNSUPPORTED;
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
    const hipStream_t st = static_cast<hipStream_t>(stream);
    for (int k = 0; k < count;) {
        AdamList L;
        L.count = 0;
        L.index0 = k;
        L.first[0] = 0;
        // (empty tensors take a place, so that t[j] is the caller's tensor index0 + j)
        for (; k < count && L.count < ADAM_TENSORS; ++k) {
            const capscaps_adamw_tensor& t = tensors[k];
            L.t[L.count] = {t.param, t.grad, t.m, t.v, t.m_exp, t.v_exp, t.copy, t.n, t.weight_decay,
                            (unsigned short)t.grad_dtype, (unsigned short)t.copy_dtype};
            add_shares(L.first, L.count, t.n, ADAM_SHARE);
            ++L.count;
        }
        if (L.first[L.count] == 0) continue;
        const dim3 grid(L.first[L.count]);
        if (state_bits == 8)
            adamw_kernel<8><<<grid, dim3(THREADS), 0, st>>>(L, H);
        else
            adamw_kernel<32><<<grid, dim3(THREADS), 0, st>>>(L, H);
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
        if (t.n > (0x7fffffffLL / ADAM_TENSORS - 1) * ADAM_SHARE) return CAPSCAPS_EUNSUPPORTED;
    }
    const hipStream_t st = static_cast<hipStream_t>(stream);
    for (int k = 0; k < count;) {
        ValuesList L;
        L.count = 0;
        L.first[0] = 0;
        for (; k < count && L.count < ADAM_TENSORS; ++k) {
            const capscaps_adamw_tensor& t = tensors[k];
            if (t.n == 0) continue;
            const int j = L.count++;
            L.m[j] = static_cast<const unsigned char*>(t.m);
            L.v[j] = static_cast<const unsigned char*>(t.v);
            L.m_exp[j] = t.m_exp;
            L.v_exp[j] = t.v_exp;
            L.m_out[j] = static_cast<unsigned short*>(m_out[k]);
            L.v_out[j] = static_cast<unsigned short*>(v_out[k]);
            L.n[j] = t.n;
            add_shares(L.first, j, t.n, ADAM_SHARE);
        }
        if (L.count == 0) break;
        state_values_kernel<<<dim3(L.first[L.count]), dim3(THREADS), 0, st>>>(L);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return status_from_hip(err);
    }
    return CAPSCAPS_OK;
}

}  // extern "C"
