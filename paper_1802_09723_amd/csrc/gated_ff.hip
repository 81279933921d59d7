// Gated feed-forward block and its backward pass.
#include "op_common.h"

namespace rrm {

namespace {

constexpr int FF_TILE = 32;  // a workgroup of 16 x 16 threads makes 32 x 32 results, four a thread

typedef const __bf16* src_t;

// tile[r][k] = p[(row0 + r) * row + (k0 + k) * col], zero outside rows x ks
__device__ __forceinline__ void fetch(float (*tile)[FF_TILE + 1], src_t p, int row0, int rows, int64_t row, int k0, int ks, int64_t col) {
    for (int e = threadIdx.x; e < FF_TILE * FF_TILE; e += 256) {
        const int r = col == 1 ? e / FF_TILE : e % FF_TILE, k = col == 1 ? e % FF_TILE : e / FF_TILE;
        tile[r][k] = row0 + r < rows && k0 + k < ks ? (float)p[(row0 + r) * row + (k0 + k) * col] : 0.0f;
    }
}
__device__ __forceinline__ void multiply(const float (*a)[FF_TILE + 1], const float (*b)[FF_TILE + 1], float (&acc)[2][2]) {
    const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
    for (int k = 0; k < FF_TILE; ++k)
        for (int i = 0; i < 2; ++i)
            for (int j = 0; j < 2; ++j) acc[i][j] += a[ty + 16 * i][k] * b[tx + 16 * j][k];
}

template <int ACT>
__global__ __launch_bounds__(256) void ff_kernel(rrm_ff_desc d, src_t x, src_t wg, src_t wu, __bf16* h, __bf16* g, __bf16* u) {
    __shared__ float a[FF_TILE][FF_TILE + 1], b[FF_TILE][FF_TILE + 1], c[FF_TILE][FF_TILE + 1];
    const int r0 = (int)blockIdx.y * FF_TILE, f0 = (int)blockIdx.x * FF_TILE;
    float sg[2][2] = {}, su[2][2] = {};
    for (int k0 = 0; k0 < d.k; k0 += FF_TILE) {
        __syncthreads();
        fetch(a, x, r0, d.m, d.x_row, k0, d.k, 1);
        fetch(b, wg, f0, d.f, d.wg_row, k0, d.k, 1);
        fetch(c, wu, f0, d.f, d.wu_row, k0, d.k, 1);
        __syncthreads();
        multiply(a, b, sg);
        multiply(a, c, su);
    }
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2; ++j) {
            const int r = r0 + (threadIdx.x >> 4) + 16 * i, f = f0 + (threadIdx.x & 15) + 16 * j;
            if (r >= d.m || f >= d.f) continue;
            h[r * d.h_row + f] = (__bf16)(act_value<ACT>(sg[i][j]) * su[i][j]);
            if (g) {
                g[r * d.gu_row + f] = (__bf16)sg[i][j];
                u[r * d.gu_row + f] = (__bf16)su[i][j];
            }
        }
}

// dG and dU, [m][f] each
template <int ACT>
__global__ __launch_bounds__(256) void ff_slopes_kernel(rrm_ff_desc d, src_t g, src_t u, src_t dh, __bf16* dg, __bf16* du) {
    const int f = (int)(blockIdx.x * 256 + threadIdx.x);
    if (f >= d.f) return;
    for (int r = blockIdx.y; r < d.m; r += gridDim.y) {
        float v, slope;
        act_pair<ACT>((float)g[r * d.gu_row + f], v, slope);
        const float dv = (float)dh[r * d.h_row + f];
        dg[(size_t)r * d.f + f] = (__bf16)(dv * (float)u[r * d.gu_row + f] * slope);
        du[(size_t)r * d.f + f] = (__bf16)(dv * v);
    }
}

// out[i][j] = sum over k of a[i][k] b[j][k], for one pair of operands or the sum over two; element [i][k] of a lies at
// i * a_row + k * a_col
struct Operands {
    src_t a, b;
    int64_t b_row, b_col;
};
__global__ __launch_bounds__(256) void product_kernel(Operands p, Operands q, int64_t a_row, int64_t a_col, int rows, int cols, int ks,
                                                      __bf16* out, int64_t out_row) {
    __shared__ float a[FF_TILE][FF_TILE + 1], b[FF_TILE][FF_TILE + 1];
    const int r0 = (int)blockIdx.y * FF_TILE, c0 = (int)blockIdx.x * FF_TILE;
    float acc[2][2] = {};
    for (int half = 0; half < (q.a ? 2 : 1); ++half) {
        const Operands& o = half ? q : p;
        for (int k0 = 0; k0 < ks; k0 += FF_TILE) {
            __syncthreads();
            fetch(a, o.a, r0, rows, a_row, k0, ks, a_col);
            fetch(b, o.b, c0, cols, o.b_row, k0, ks, o.b_col);
            __syncthreads();
            multiply(a, b, acc);
        }
    }
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2; ++j) {
            const int r = r0 + (threadIdx.x >> 4) + 16 * i, c = c0 + (threadIdx.x & 15) + 16 * j;
            if (r < rows && c < cols) out[r * out_row + c] = (__bf16)acc[i][j];
        }
}

template <typename F>
void with_act(int act, F&& f) {
    switch (act) {
        case RRM_ACT_RELU: f(std::integral_constant<int, RRM_ACT_RELU>{}); break;
        case RRM_ACT_SILU: f(std::integral_constant<int, RRM_ACT_SILU>{}); break;
        case RRM_ACT_GELU: f(std::integral_constant<int, RRM_ACT_GELU>{}); break;
        default: f(std::integral_constant<int, RRM_ACT_NONE>{}); break;
    }
}

unsigned tiles(int n) { return (unsigned)((n + FF_TILE - 1) / FF_TILE); }

}  // namespace

size_t ff_scratch(const rrm_ff_desc& d, bool backward) { return backward ? 2 * round256((size_t)d.m * d.f * 2) : 0; }

hipError_t launch_gated_ff(const rrm_ff_desc& d, const void* x, const void* wg, const void* wu, void* h, void* g, void* u, void*,
                           hipStream_t s) {
    with_act(d.act, [&](auto act) {
        hipLaunchKernelGGL((ff_kernel<decltype(act)::value>), dim3(tiles(d.f), tiles(d.m)), dim3(256), 0, s, d, (src_t)x, (src_t)wg,
                           (src_t)wu, (__bf16*)h, (__bf16*)g, (__bf16*)u);
    });
    return hipGetLastError();
}

hipError_t launch_gated_ff_backward(const rrm_ff_desc& d, const void* x, const void* wg, const void* wu, const void* g,
                                    const void* u, const void* dh, void* dx, void* dwg, void* dwu, void* ws, hipStream_t s) {
    __bf16* dg = (__bf16*)ws;
    __bf16* du = (__bf16*)((char*)ws + round256((size_t)d.m * d.f * 2));
    if (d.m > 0) {
        with_act(d.act, [&](auto act) {
            hipLaunchKernelGGL((ff_slopes_kernel<decltype(act)::value>), dim3((unsigned)((d.f + 255) / 256), (unsigned)(d.m < 65535 ? d.m : 65535)),
                               dim3(256), 0, s, d, (src_t)g, (src_t)u, (src_t)dh, dg, du);
        });
        if (hipError_t e = hipGetLastError()) return e;
        if (dx) {
            const Operands p{dg, (src_t)wg, 1, d.wg_row}, q{du, (src_t)wu, 1, d.wu_row};
            hipLaunchKernelGGL(product_kernel, dim3(tiles(d.k), tiles(d.m)), dim3(256), 0, s, p, q, (int64_t)d.f, (int64_t)1, d.m, d.k, d.f,
                               (__bf16*)dx, d.dx_row);
            if (hipError_t e = hipGetLastError()) return e;
        }
    }
    if (dwg) {
        const Operands none{nullptr, nullptr, 0, 0};
        for (int half = 0; half < 2; ++half) {
            const Operands p{half ? du : dg, (src_t)x, 1, d.x_row};
            hipLaunchKernelGGL(product_kernel, dim3(tiles(d.k), tiles(d.f)), dim3(256), 0, s, p, none, (int64_t)1, (int64_t)d.f, d.f, d.k,
                               d.m, (__bf16*)(half ? dwu : dwg), half ? d.dwu_row : d.dwg_row);
            if (hipError_t e = hipGetLastError()) return e;
        }
    }
    return hipSuccess;
}

}  // namespace rrm
