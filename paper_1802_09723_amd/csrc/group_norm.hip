// Group norm with an activation, channels last, and its backward pass.
#include "op_common.h"

namespace rrm {

namespace {

constexpr int GN_THREADS = 256;

// sum over the workgroup, to every thread
__device__ float wg_sum(float v, float* lds) {
#pragma unroll
    for (int m = 1; m < OP_WAVE; m <<= 1) v += __shfl_xor(v, m);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = 0.0f;
    for (int i = 0; i < GN_THREADS / OP_WAVE; ++i) s += lds[i];
    return s;
}

// One workgroup per (sample, group): mean, variance and result in three passes over the group.
template <typename TX, typename TY, int ACT>
__global__ __launch_bounds__(GN_THREADS) void norm_kernel(rrm_norm_desc d, const TX* __restrict__ x, const float* __restrict__ gamma,
                                                          const float* __restrict__ beta, TY* __restrict__ y, float* __restrict__ stats) {
    __shared__ float lds[GN_THREADS / OP_WAVE];
    const int cg = d.c / d.groups, i = (int)blockIdx.x / d.groups, g = (int)blockIdx.x % d.groups;
    const TX* xs = x + i * d.x_sample + g * cg;
    TY* ys = y + i * d.y_sample + g * cg;
    const long long m = (long long)d.positions * cg;
    float s = 0.0f;
    for (long long k = threadIdx.x; k < m; k += GN_THREADS) s += load_elem(xs + (k / cg) * d.x_position + k % cg);
    const float mean = wg_sum(s, lds) / (float)m;
    s = 0.0f;
    for (long long k = threadIdx.x; k < m; k += GN_THREADS) {
        const float v = load_elem(xs + (k / cg) * d.x_position + k % cg) - mean;
        s += v * v;
    }
    const float r = 1.0f / sqrtf(wg_sum(s, lds) / (float)m + d.eps);
    if (stats && threadIdx.x == 0) stats[2 * blockIdx.x] = mean, stats[2 * blockIdx.x + 1] = r;
    for (long long k = threadIdx.x; k < m; k += GN_THREADS) {
        const int c = (int)(k % cg);
        const float xh = (load_elem(xs + (k / cg) * d.x_position + c) - mean) * r;
        const float z = (gamma ? gamma[g * cg + c] : 1.0f) * xh + (beta ? beta[g * cg + c] : 0.0f);
        store_elem(ys + (k / cg) * d.y_position + c, act_value<ACT>(z));
    }
}

// One workgroup per (sample, group): the sums of dz and dz * xh of each channel, left in part[2][n][c], then dx.
template <typename TX, typename TY, int ACT>
__global__ __launch_bounds__(GN_THREADS) void norm_back_kernel(rrm_norm_desc d, const TX* __restrict__ x, const float* __restrict__ stats,
                                                               const float* __restrict__ gamma, const float* __restrict__ beta,
                                                               const TY* __restrict__ dy, TX* __restrict__ dx, float* __restrict__ part) {
    __shared__ float lds[GN_THREADS / OP_WAVE];
    const int cg = d.c / d.groups, i = (int)blockIdx.x / d.groups, g = (int)blockIdx.x % d.groups;
    const TX* xs = x + i * d.x_sample + g * cg;
    const TY* dys = dy + i * d.y_sample + g * cg;
    const float mean = stats[2 * blockIdx.x], r = stats[2 * blockIdx.x + 1];
    float p = 0.0f, q = 0.0f;
    for (int c = 0; c < cg; ++c) {
        const float ga = gamma ? gamma[g * cg + c] : 1.0f, be = beta ? beta[g * cg + c] : 0.0f;
        float s1 = 0.0f, s2 = 0.0f;
        for (int k = threadIdx.x; k < d.positions; k += GN_THREADS) {
            const float xh = (load_elem(xs + k * d.x_position + c) - mean) * r;
            float v, slope;
            act_pair<ACT>(ga * xh + be, v, slope);
            const float dz = load_elem(dys + k * d.y_position + c) * slope;
            s1 += dz;
            s2 += dz * xh;
        }
        s1 = wg_sum(s1, lds);
        s2 = wg_sum(s2, lds);
        if (threadIdx.x == 0) {
            part[(size_t)i * d.c + g * cg + c] = s1;
            part[(size_t)d.n * d.c + (size_t)i * d.c + g * cg + c] = s2;
        }
        p += ga * s1;
        q += ga * s2;
    }
    if (!dx) return;
    TX* dxs = dx + i * d.dx_sample + g * cg;
    const long long m = (long long)d.positions * cg;
    p /= (float)m;
    q /= (float)m;
    for (long long k = threadIdx.x; k < m; k += GN_THREADS) {
        const int c = (int)(k % cg);
        const float ga = gamma ? gamma[g * cg + c] : 1.0f, be = beta ? beta[g * cg + c] : 0.0f;
        const float xh = (load_elem(xs + (k / cg) * d.x_position + c) - mean) * r;
        float v, slope;
        act_pair<ACT>(ga * xh + be, v, slope);
        const float dz = load_elem(dys + (k / cg) * d.y_position + c) * slope;
        store_elem(dxs + (k / cg) * d.dx_position + c, r * (ga * dz - p - xh * q));
    }
}

// dbeta and dgamma: the samples' sums in their order (no samples: zeros)
__global__ void norm_params_kernel(const float* __restrict__ part, int n, int c, float* __restrict__ dgamma, float* __restrict__ dbeta) {
    const int ch = (int)(blockIdx.x * blockDim.x + threadIdx.x);
    if (ch >= c) return;
    float s1 = 0.0f, s2 = 0.0f;
    for (int i = 0; i < n; ++i) {
        s1 += part[(size_t)i * c + ch];
        s2 += part[(size_t)(n + i) * c + ch];
    }
    if (dbeta) dbeta[ch] = s1;
    if (dgamma) dgamma[ch] = s2;
}

// calls f(TX, TY, act) with the descriptor's types
template <typename F>
void with_types(const rrm_norm_desc& d, F&& f) {
    auto act = [&](auto tx, auto ty) {
        switch (d.act) {
            case RRM_ACT_RELU: f(tx, ty, std::integral_constant<int, RRM_ACT_RELU>{}); break;
            case RRM_ACT_SILU: f(tx, ty, std::integral_constant<int, RRM_ACT_SILU>{}); break;
            case RRM_ACT_GELU: f(tx, ty, std::integral_constant<int, RRM_ACT_GELU>{}); break;
            default: f(tx, ty, std::integral_constant<int, RRM_ACT_NONE>{}); break;
        }
    };
    auto out = [&](auto tx) { d.y_elem == RRM_F32 ? act(tx, float{}) : act(tx, __bf16{}); };
    d.x_elem == RRM_F32 ? out(float{}) : out(__bf16{});
}

}  // namespace

size_t norm_scratch(const rrm_norm_desc& d, bool backward) {
    return backward ? round256((size_t)2 * d.n * d.c * 4) : 0;
}

hipError_t launch_group_norm(const rrm_norm_desc& d, const void* x, const float* gamma, const float* beta, void* y, float* stats,
                             void*, hipStream_t s) {
    with_types(d, [&](auto tx, auto ty, auto act) {
        using TX = decltype(tx);
        using TY = decltype(ty);
        hipLaunchKernelGGL((norm_kernel<TX, TY, decltype(act)::value>), dim3((unsigned)(d.n * d.groups)), dim3(GN_THREADS), 0, s, d,
                           (const TX*)x, gamma, beta, (TY*)y, stats);
    });
    return hipGetLastError();
}

hipError_t launch_group_norm_backward(const rrm_norm_desc& d, const void* x, const float* stats, const float* gamma,
                                      const float* beta, const void* dy, void* dx, float* dgamma, float* dbeta, void* ws,
                                      hipStream_t s) {
    const bool some = d.n > 0 && d.positions > 0;
    if (some) {
        with_types(d, [&](auto tx, auto ty, auto act) {
            using TX = decltype(tx);
            using TY = decltype(ty);
            hipLaunchKernelGGL((norm_back_kernel<TX, TY, decltype(act)::value>), dim3((unsigned)(d.n * d.groups)), dim3(GN_THREADS), 0, s,
                               d, (const TX*)x, stats, gamma, beta, (const TY*)dy, (TX*)dx, (float*)ws);
        });
        if (hipError_t e = hipGetLastError()) return e;
    }
    if (dgamma || dbeta)
        hipLaunchKernelGGL(norm_params_kernel, dim3((unsigned)((d.c + 255) / 256)), dim3(256), 0, s, (const float*)ws, some ? d.n : 0,
                           d.c, dgamma, dbeta);
    return hipGetLastError();
}

}  // namespace rrm
