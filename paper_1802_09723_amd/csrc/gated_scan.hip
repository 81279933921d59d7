// Gated linear recurrence over the frames of videos, and its backward pass.
#include "op_common.h"

namespace rrm {

namespace {

constexpr int GS_THREADS = 64;

__device__ __forceinline__ int video_frames(const int32_t* lengths, int i, int t) {
    if (!lengths) return t;
    const int e = lengths[i];
    return e < 0 ? 0 : e > t ? t : e;
}

// One thread per (video, feature), frame by frame.
template <typename T>
__global__ __launch_bounds__(GS_THREADS) void scan_kernel(rrm_scan_desc d, const T* __restrict__ x, const T* __restrict__ f,
                                                          const float* h0, const int32_t* __restrict__ lengths, T* __restrict__ y,
                                                          float* h_last, float* __restrict__ marks) {
    const int c = (int)(blockIdx.x * GS_THREADS + threadIdx.x), i = (int)blockIdx.y;
    if (c >= d.c) return;
    const int end = video_frames(lengths, i, d.t);
    const int nm = (d.t + RRM_SCAN_MARK_FRAMES - 1) / RRM_SCAN_MARK_FRAMES;
    const size_t at = (size_t)i * d.c + c;
    float h = h0 ? h0[at] : 0.0f;
    for (int k = 0; k < d.t; ++k) {
        if (marks && k % RRM_SCAN_MARK_FRAMES == 0) marks[((size_t)i * nm + k / RRM_SCAN_MARK_FRAMES) * d.c + c] = h;
        float out = 0.0f;
        if (k < end) {
            float a, b;
            gate_pair(load_elem(f + i * d.f_video + k * d.f_frame + c), a, b);
            h = a * h + b * load_elem(x + i * d.x_video + k * d.x_frame + c);
            out = h;
        }
        store_elem(y + i * d.y_video + k * d.y_frame + c, out);
    }
    if (h_last) h_last[at] = h;
}

// One thread per (video, feature): from the last stretch between two marks to the first, h again from the mark, then back.
template <typename T>
__global__ __launch_bounds__(GS_THREADS) void scan_back_kernel(rrm_scan_desc d, const T* __restrict__ x, const T* __restrict__ f,
                                                               const float* __restrict__ marks, const int32_t* __restrict__ lengths,
                                                               const T* __restrict__ dy, const float* dh_last, T* __restrict__ dx,
                                                               T* __restrict__ df, float* dh0) {
    __shared__ float hs[RRM_SCAN_MARK_FRAMES][GS_THREADS];
    const int c = (int)(blockIdx.x * GS_THREADS + threadIdx.x), i = (int)blockIdx.y;
    if (c >= d.c) return;
    const int end = video_frames(lengths, i, d.t);
    const int nm = (d.t + RRM_SCAN_MARK_FRAMES - 1) / RRM_SCAN_MARK_FRAMES;
    const size_t at = (size_t)i * d.c + c;
    for (int k = end; k < d.t; ++k) {
        store_elem(dx + i * d.dx_video + k * d.dx_frame + c, 0.0f);
        store_elem(df + i * d.df_video + k * d.df_frame + c, 0.0f);
    }
    float g = dh_last ? dh_last[at] : 0.0f;  // the gradient of the state after the frame at hand
    for (int m = (end + RRM_SCAN_MARK_FRAMES - 1) / RRM_SCAN_MARK_FRAMES - 1; m >= 0; --m) {
        const int k0 = m * RRM_SCAN_MARK_FRAMES, k1 = k0 + RRM_SCAN_MARK_FRAMES < end ? k0 + RRM_SCAN_MARK_FRAMES : end;
        float h = marks[((size_t)i * nm + m) * d.c + c];
        for (int k = k0; k < k1; ++k) {
            float a, b;
            gate_pair(load_elem(f + i * d.f_video + k * d.f_frame + c), a, b);
            hs[k - k0][threadIdx.x] = h;
            h = a * h + b * load_elem(x + i * d.x_video + k * d.x_frame + c);
        }
        for (int k = k1 - 1; k >= k0; --k) {
            float a, b;
            gate_pair(load_elem(f + i * d.f_video + k * d.f_frame + c), a, b);
            g += load_elem(dy + i * d.y_video + k * d.y_frame + c);
            store_elem(dx + i * d.dx_video + k * d.dx_frame + c, b * g);
            store_elem(df + i * d.df_video + k * d.df_frame + c,
                       g * (hs[k - k0][threadIdx.x] - load_elem(x + i * d.x_video + k * d.x_frame + c)) * (a * b));
            g *= a;
        }
    }
    if (dh0) dh0[at] = g;
}

}  // namespace

size_t scan_scratch(const rrm_scan_desc&, bool) { return 0; }

hipError_t launch_gated_scan(const rrm_scan_desc& d, const void* x, const void* f, const float* h0, const int32_t* lengths,
                             void* y, float* h_last, float* marks, void*, hipStream_t s) {
    const dim3 grid((unsigned)((d.c + GS_THREADS - 1) / GS_THREADS), (unsigned)d.n);
    if (d.elem == RRM_F32)
        hipLaunchKernelGGL((scan_kernel<float>), grid, dim3(GS_THREADS), 0, s, d, (const float*)x, (const float*)f, h0, lengths,
                           (float*)y, h_last, marks);
    else
        hipLaunchKernelGGL((scan_kernel<__bf16>), grid, dim3(GS_THREADS), 0, s, d, (const __bf16*)x, (const __bf16*)f, h0, lengths,
                           (__bf16*)y, h_last, marks);
    return hipGetLastError();
}

hipError_t launch_gated_scan_backward(const rrm_scan_desc& d, const void* x, const void* f, const float* marks,
                                      const int32_t* lengths, const void* dy, const float* dh_last, void* dx, void* df,
                                      float* dh0, void*, hipStream_t s) {
    const dim3 grid((unsigned)((d.c + GS_THREADS - 1) / GS_THREADS), (unsigned)d.n);
    if (d.elem == RRM_F32)
        hipLaunchKernelGGL((scan_back_kernel<float>), grid, dim3(GS_THREADS), 0, s, d, (const float*)x, (const float*)f, marks,
                           lengths, (const float*)dy, dh_last, (float*)dx, (float*)df, dh0);
    else
        hipLaunchKernelGGL((scan_back_kernel<__bf16>), grid, dim3(GS_THREADS), 0, s, d, (const __bf16*)x, (const __bf16*)f, marks,
                           lengths, (const __bf16*)dy, dh_last, (__bf16*)dx, (__bf16*)df, dh0);
    return hipGetLastError();
}

}  // namespace rrm
