// Shared by the operators between and behind the linear layers: element types, activations, launch declarations.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

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

// Words from and to memory at the alignment of an element: one instruction, whatever the address (the hardware takes any).
template <int WORDS>
struct __attribute__((packed, aligned(2))) LooseWords {
    typedef unsigned int vec __attribute__((ext_vector_type(WORDS)));
    vec v;
};
template <int WORDS>
__device__ __forceinline__ void load_words(const void* p, unsigned int (&w)[WORDS]) {
    if constexpr (WORDS == 1) {
        struct __attribute__((packed, aligned(2))) One {
            unsigned int v;
        };
        w[0] = reinterpret_cast<const One*>(p)->v;
    } else if constexpr (WORDS <= 4) {
        const auto v = reinterpret_cast<const LooseWords<WORDS>*>(p)->v;
#pragma unroll
        for (int i = 0; i < WORDS; ++i) w[i] = v[i];
    } else {
#pragma unroll
        for (int k = 0; k < WORDS; k += 4) {
            const auto v = reinterpret_cast<const LooseWords<4>*>(static_cast<const unsigned int*>(p) + k)->v;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[k + i] = v[i];
        }
    }
}
template <int WORDS>
__device__ __forceinline__ void store_words(void* p, const unsigned int (&w)[WORDS]) {
    static_assert(WORDS == 2 || WORDS == 4 || WORDS == 8);
    constexpr int RUN = WORDS < 4 ? WORDS : 4;
#pragma unroll
    for (int k = 0; k < WORDS; k += RUN) {
        typename LooseWords<RUN>::vec v;
#pragma unroll
        for (int i = 0; i < RUN; ++i) v[i] = w[k + i];
        reinterpret_cast<LooseWords<RUN>*>(static_cast<unsigned int*>(p) + k)->v = v;
    }
}
// VEC neighbouring elements as float, and back
template <int VEC, typename T>
__device__ __forceinline__ void load_vec(const T* p, float (&v)[VEC]) {
    if constexpr (VEC == 1) {
        v[0] = load_elem(p);
    } else {
        unsigned int w[VEC * sizeof(T) / 4];
        load_words(p, w);
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            v[i] = sizeof(T) == 4 ? __uint_as_float(w[sizeof(T) == 4 ? i : 0]) : i & 1 ? bf16_hi(w[i >> 1]) : bf16_lo(w[i >> 1]);
    }
}
template <int VEC, typename T>
__device__ __forceinline__ void store_vec(T* p, const float (&v)[VEC]) {
    if constexpr (VEC == 1) {
        store_elem(p, v[0]);
    } else {
        unsigned int w[VEC * sizeof(T) / 4];
#pragma unroll
        for (int i = 0; i < (int)(VEC * sizeof(T) / 4); ++i) w[i] = sizeof(T) == 4 ? __float_as_uint(v[i]) : bf16_pair(v[(2 * i) % VEC], v[(2 * i + 1) % VEC]);
        store_words(p, w);
    }
}
// those from `first` on
template <int VEC, typename T>
__device__ __forceinline__ void store_some(T* p, const float (&v)[VEC], int first) {
    if (first == 0) {
        store_vec<VEC>(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (i >= first) store_elem(p + i, v[i]);
    }
}

template <typename T, int VEC>
struct Held {  // VEC elements as they lie in memory, at the alignment of one
    static constexpr int WORDS = (VEC * (int)sizeof(T) + 3) / 4;
    unsigned int w[WORDS];
    __device__ __forceinline__ void load(const T* p) {
        if constexpr (VEC * sizeof(T) == 2) w[0] = *reinterpret_cast<const unsigned short*>(p);
        else load_words<WORDS>(p, w);
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        return i & 1 ? bf16_hi(w[i >> 1]) : bf16_lo(w[i >> 1]);
    }
};

// A thread's vector of channels: from `at` on.  The last vector of a workgroup whose channels are no whole vectors begins early (never before the
// row: a workgroup has VEC channels at least, or others before it): what it has before `first` is another thread's and not to be
// summed.  It is to be stored from `keep` on: both threads make the same bits of a channel of their workgroup, and one whole store is
// cheaper than its elements; not so where the vector reaches into the workgroup before.  A thread without channels has first = keep = VEC.
template <int VEC>
struct Span {
    int at, first, keep;
    __device__ __forceinline__ Span(int slot, int c0, int cb) {
        const int c = c0 + slot * VEC, end = c0 + cb - VEC;
        const bool none = slot * VEC >= cb;
        at = none || c > end ? (end > 0 ? end : 0) : c;
        first = none ? VEC : c - at;
        keep = none ? VEC : at >= c0 ? 0 : first;
    }
};

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

// calls f(std::integral_constant<int, act>)
template <typename F>
__host__ __device__ __forceinline__ void with_act(int act, F&& f) {
    switch (act) {
        case RRM_ACT_RELU: f(std::integral_constant<int, RRM_ACT_RELU>{}); break;
        case RRM_ACT_SILU: f(std::integral_constant<int, RRM_ACT_SILU>{}); break;
        case RRM_ACT_GELU: f(std::integral_constant<int, RRM_ACT_GELU>{}); break;
        default: f(std::integral_constant<int, RRM_ACT_NONE>{}); break;
    }
}

// A launch takes fewer than 2^32 threads along an axis: f(first workgroup, workgroups) for each part of `total` of them.  Parts begin at whole eights, so
// workgroups stay on their XCD.
template <typename F>
void in_parts(int64_t total, F&& f) {
    constexpr int64_t MOST = 1 << 21;  // of up to 1024 threads
    for (int64_t first = 0; first < total; first += MOST) f((unsigned)first, (unsigned)(total - first < MOST ? total - first : MOST));
}

#endif  // __HIPCC__

// Launchers; descriptors have been checked, and something is to be done.  The *_scratch functions say how many bytes of
// workspace the same descriptor takes, the *_layout functions which kernels (rrm_aux_*_layout).
void norm_layout(const rrm_norm_desc& d, bool backward, int* layout);
void scan_layout(const rrm_scan_desc& d, bool backward, int* layout);
void ff_layout(const rrm_ff_desc& d, int asked, int* layout);
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
