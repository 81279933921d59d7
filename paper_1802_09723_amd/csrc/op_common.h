// Shared by the operators between and behind the linear layers: element types, activations, launch declarations.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rrm.h"

namespace rrm {

rrm_status record_failure(rrm_status st, const char* msg) noexcept;  // keeps the text for rrm_last_error

constexpr int OP_WAVE = 64;
constexpr int OP_CUS = 256;  // compute units of the MI355X

inline size_t round256(size_t b) { return (b + 255) & ~size_t(255); }

#ifdef __HIPCC__

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float bf16_lo(unsigned int w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(unsigned int w) { return __uint_as_float(w & 0xffff0000u); }
// two values rounded to nearest even (one conversion instruction)
__device__ __forceinline__ unsigned int bf16_pair(float lo, float hi) {
    bf16x2 v;
    v[0] = (__bf16)lo;
    v[1] = (__bf16)hi;
    return __builtin_bit_cast(unsigned int, v);
}

__device__ __forceinline__ float load_elem(const float* p) { return *p; }
__device__ __forceinline__ float load_elem(const __bf16* p) { return (float)*p; }
__device__ __forceinline__ void store_elem(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_elem(__bf16* p, float v) { *p = (__bf16)v; }

// VEC neighbouring elements as float; p lies at a multiple of their size (see the callers' choice of VEC)
template <int VEC>
__device__ __forceinline__ void load_vec(const float* p, float (&v)[VEC]) {
    if constexpr (VEC == 1) {
        v[0] = *p;
    } else if constexpr (VEC == 2) {
        const float2 a = *reinterpret_cast<const float2*>(p);
        v[0] = a.x, v[1] = a.y;
    } else {
#pragma unroll
        for (int i = 0; i < VEC; i += 4) {
            const float4 a = *reinterpret_cast<const float4*>(p + i);
            v[i] = a.x, v[i + 1] = a.y, v[i + 2] = a.z, v[i + 3] = a.w;
        }
    }
}
template <int VEC>
__device__ __forceinline__ void load_vec(const __bf16* p, float (&v)[VEC]) {
    if constexpr (VEC == 1) {
        v[0] = (float)*p;
    } else if constexpr (VEC == 2) {
        const unsigned int a = *reinterpret_cast<const unsigned int*>(p);
        v[0] = bf16_lo(a), v[1] = bf16_hi(a);
    } else if constexpr (VEC == 4) {
        const u32x2 a = *reinterpret_cast<const u32x2*>(p);
        v[0] = bf16_lo(a.x), v[1] = bf16_hi(a.x), v[2] = bf16_lo(a.y), v[3] = bf16_hi(a.y);
    } else {
#pragma unroll
        for (int i = 0; i < VEC; i += 8) {
            const u32x4 a = *reinterpret_cast<const u32x4*>(p + i);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[i + 2 * k] = bf16_lo(a[k]), v[i + 2 * k + 1] = bf16_hi(a[k]);
        }
    }
}
template <int VEC>
__device__ __forceinline__ void store_vec(float* p, const float (&v)[VEC]) {
    if constexpr (VEC == 1) {
        *p = v[0];
    } else if constexpr (VEC == 2) {
        *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]);
    } else {
#pragma unroll
        for (int i = 0; i < VEC; i += 4) *reinterpret_cast<float4*>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
    }
}
template <int VEC>
__device__ __forceinline__ void store_vec(__bf16* p, const float (&v)[VEC]) {
    if constexpr (VEC == 1) {
        *p = (__bf16)v[0];
    } else if constexpr (VEC == 2) {
        *reinterpret_cast<unsigned int*>(p) = bf16_pair(v[0], v[1]);
    } else if constexpr (VEC == 4) {
        u32x2 a;
        a.x = bf16_pair(v[0], v[1]), a.y = bf16_pair(v[2], v[3]);
        *reinterpret_cast<u32x2*>(p) = a;
    } else {
#pragma unroll
        for (int i = 0; i < VEC; i += 8) {
            u32x4 a;
#pragma unroll
            for (int k = 0; k < 4; ++k) a[k] = bf16_pair(v[i + 2 * k], v[i + 2 * k + 1]);
            *reinterpret_cast<u32x4*>(p + i) = a;
        }
    }
}

// exp2 and 1/x of one instruction each (1 ulp): the gates' and activations' exponentials.  Arguments below -126 give 0.
__device__ __forceinline__ float fast_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896f); }
__device__ __forceinline__ float fast_rcp(float x) { return __builtin_amdgcn_rcpf(x); }

__device__ __forceinline__ float sigmoid(float z) { return fast_rcp(1.0f + fast_exp(-z)); }

// sigmoid(f) and 1 - sigmoid(f), each to its own relative accuracy (1 - a would lose the digits of a gate near 1);
// with e = exp(-|f|) <= 1 nothing overflows, infinite f included
__device__ __forceinline__ void gate_pair(float f, float& a, float& one_minus_a) {
    const float e = fast_exp(-fabsf(f));
    const float r = fast_rcp(1.0f + e), p = e * r;
    a = f >= 0.0f ? r : p;
    one_minus_a = f >= 0.0f ? p : r;
    if (f != f) a = one_minus_a = f;
}

// Phi(z) and its density: erfc(x) = (c1 t + .. + c5 t^5) exp(-x^2) with t = 1 / (1 + p x), x = |z| / sqrt(2)
// (Abramowitz and Stegun 7.1.26, absolute error below 1.5e-7): one exponential serves both, and a negative z needs no
// difference of nearly equal numbers
__device__ __forceinline__ void normal_cdf_pdf(float z, float& cdf, float& pdf) {
    const float e = fast_exp(-0.5f * z * z);
    const float t = fast_rcp(1.0f + 0.3275911f * 0.70710678118655f * fabsf(z));
    const float half = 0.5f * e * t * (0.254829592f + t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f))));
    cdf = z < 0.0f ? half : 1.0f - half;
    pdf = 0.39894228040143f * e;
}

template <int ACT>
__device__ __forceinline__ float act_value(float z) {
    if constexpr (ACT == RRM_ACT_RELU) return z < 0.0f ? 0.0f : z;  // (a not-a-number stays one)
    if constexpr (ACT == RRM_ACT_SILU) return z * sigmoid(z);
    if constexpr (ACT == RRM_ACT_GELU) {
        float cdf, pdf;
        normal_cdf_pdf(z, cdf, pdf);
        return z * cdf;
    }
    return z;
}
// act(z) and act'(z)
template <int ACT>
__device__ __forceinline__ void act_pair(float z, float& value, float& slope) {
    if constexpr (ACT == RRM_ACT_RELU) {
        value = z < 0.0f ? 0.0f : z;
        slope = z > 0.0f ? 1.0f : 0.0f;
    } else if constexpr (ACT == RRM_ACT_SILU) {
        const float p = sigmoid(z);
        value = z * p;
        slope = p + value * (1.0f - p);
    } else if constexpr (ACT == RRM_ACT_GELU) {
        float cdf, pdf;
        normal_cdf_pdf(z, cdf, pdf);
        value = z * cdf;
        slope = cdf + z * pdf;
    } else {
        value = z;
        slope = 1.0f;
    }
}

#endif  // __HIPCC__

// Launchers; descriptors have been checked, and something is to be done.  The *_scratch functions say how many bytes of
// workspace the same descriptor takes.
size_t norm_scratch(const rrm_norm_desc& d, bool backward);
hipError_t launch_group_norm(const rrm_norm_desc& d, const void* x, const float* gamma, const float* beta, void* y, float* stats,
                             void* ws, hipStream_t s);
hipError_t launch_group_norm_backward(const rrm_norm_desc& d, const void* x, const float* stats, const float* gamma,
                                      const float* beta, const void* dy, void* dx, float* dgamma, float* dbeta, void* ws,
                                      hipStream_t s);
size_t scan_scratch(const rrm_scan_desc& d, bool backward);
hipError_t launch_gated_scan(const rrm_scan_desc& d, const void* x, const void* f, const float* h0, const int32_t* lengths,
                             void* y, float* h_last, float* marks, void* ws, hipStream_t s);
hipError_t launch_gated_scan_backward(const rrm_scan_desc& d, const void* x, const void* f, const float* marks,
                                      const int32_t* lengths, const void* dy, const float* dh_last, void* dx, void* df,
                                      float* dh0, void* ws, hipStream_t s);
size_t ff_scratch(const rrm_ff_desc& d, bool backward);
hipError_t launch_gated_ff(const rrm_ff_desc& d, const void* x, const void* wg, const void* wu, void* h, void* g, void* u, void* ws,
                           hipStream_t s);
hipError_t launch_gated_ff_backward(const rrm_ff_desc& d, const void* x, const void* wg, const void* wu, const void* g,
                                    const void* u, const void* dh, void* dx, void* dwg, void* dwu, void* ws, hipStream_t s);

}  // namespace rrm
