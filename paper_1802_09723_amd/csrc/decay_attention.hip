// Linear attention over a video's frames with a decay for each head, and its backward pass.
//
//      S_t = lambda S_{t-1} + k_t^T v_t        o_t = scale q_t S_t
//      D_t = lambda D_{t+1} + scale q_t^T do_t        dq_t = scale S_t do_t        dk_t = D_t v_t        dv_t = k_t D_t        ds0 = lambda D_1
//
// Every one of these is the same walk over the frames: a state W [k][v] that decays and takes up k_j^T v_j, and is read by q_i,
//      result_i = sum over j up to i of lambda^(i-j) (q_i . k_j) v_j + lambda^(i..) q_i W_0:
//      o   from (q, k, v);      dq  from (do, v, k) on S turned;      dk  from (v, do, q) on D turned, last frame first;      dv  from (k, q, do) on D, likewise.
#include "op_common.h"

namespace rrm {

namespace {

struct Operand {
    const void* p;
    int64_t video, frame, head;  // strides
};
// A walk over the frames of n videos and h heads.
struct Walk {
    Operand q, k, v, o;  // o: written
    int n, t, h, dk, dv;
    const float *s_in, *s_out;  // states [n][h][dk][dv] (turned: [dv][dk]); NULL: zeros; not kept.  s_out is written
    bool turned;
    bool back;      // last frame first, and the state decays behind a frame, not before it: what it holds is the gradient of the state before
    float taken, given;  // factors of k^T v as the state takes it up, and of the result
    const float* log_decay;
    const int32_t* lengths;
};

__device__ __forceinline__ int frames_of(const Walk& w, int video) {
    if (!w.lengths) return w.t;
    const int e = w.lengths[video];
    return e < 0 ? 0 : e < w.t ? e : w.t;
}

// The recurrence as it stands, a state in registers: one frame of live videos (and the walk for any).  A workgroup has 64 columns of a head's state; thread
// (g, quad) holds rows g, g + 16, .. of four columns.
template <typename T, int ROWS>
__global__ __launch_bounds__(256) void step_kernel(Walk w, unsigned first) {
    __shared__ float4 sums[2][4][16];
    const int slices = (w.dv + 63) >> 6;
    const unsigned id = first + blockIdx.x;
    const int slice = (int)(id % slices);
    const int64_t pair = id / slices;
    const int video = (int)(pair / w.h), head = (int)(pair % w.h);
    const int tid = threadIdx.x, quad = tid & 15, g = tid >> 4, wave = tid >> 6;
    const int c = slice * 64 + quad * 4, have = w.dv - c;  // columns of this thread: min(have, 4)
    const int frames = frames_of(w, video);
    const T* q = (const T*)w.q.p + video * w.q.video + head * w.q.head;
    const T* k = (const T*)w.k.p + video * w.k.video + head * w.k.head;
    const T* v = (const T*)w.v.p + video * w.v.video + head * w.v.head;
    T* o = (T*)const_cast<void*>(w.o.p) + video * w.o.video + head * w.o.head;
    const int64_t plane = pair * w.dk * w.dv;
    const float decay = w.t > 0 ? expf(w.log_decay[head]) : 1.0f;
    auto four = [&](float4& s, int r, auto each) {  // the places of a row's four values in a state
        float* e = reinterpret_cast<float*>(&s);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < have) each(e[i], plane + (w.turned ? (int64_t)(c + i) * w.dk + r : (int64_t)r * w.dv + c + i));
    };
    float4 s[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int r = g + 16 * i;
        s[i] = make_float4(0, 0, 0, 0);
        if (!w.s_in || r >= w.dk) continue;
        const float* at = w.s_in + plane + (int64_t)r * w.dv + c;
        if (!w.turned && have >= 4 && (w.dv & 3) == 0 && ((uintptr_t)w.s_in & 15) == 0) s[i] = *reinterpret_cast<const float4*>(at);
        else four(s[i], r, [&](float& e, int64_t p) { e = w.s_in[p]; });
    }
    int turn = 0;
    for (int f = 0; f < frames; ++f) {
        const int at = w.back ? frames - 1 - f : f;
        float vv[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) vv[i] = i < have ? w.taken * load_elem(v + at * w.v.frame + c + i) : 0.0f;
        float4 sum = make_float4(0, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const int r = g + 16 * i;
            if (r >= w.dk) continue;
            const float kv = load_elem(k + at * w.k.frame + r), qv = load_elem(q + at * w.q.frame + r);
            const float before = w.back ? 1.0f : decay;
            s[i].x = before * s[i].x + kv * vv[0], s[i].y = before * s[i].y + kv * vv[1];
            s[i].z = before * s[i].z + kv * vv[2], s[i].w = before * s[i].w + kv * vv[3];
            sum.x += qv * s[i].x, sum.y += qv * s[i].y, sum.z += qv * s[i].z, sum.w += qv * s[i].w;
            if (w.back) s[i].x *= decay, s[i].y *= decay, s[i].z *= decay, s[i].w *= decay;
        }
#pragma unroll
        for (int m = 16; m < 64; m <<= 1) {
            sum.x += __shfl_xor(sum.x, m), sum.y += __shfl_xor(sum.y, m);
            sum.z += __shfl_xor(sum.z, m), sum.w += __shfl_xor(sum.w, m);
        }
        if ((tid & 63) < 16) sums[turn][wave][quad] = sum;
        __syncthreads();
        if (tid < 64) {
            const float* part = reinterpret_cast<const float*>(&sums[turn][0][0]);
            const float r = (part[tid] + part[64 + tid]) + (part[128 + tid] + part[192 + tid]);
            if (w.o.p && slice * 64 + tid < w.dv) store_elem(o + at * w.o.frame + slice * 64 + tid, w.given * r);
        }
        turn ^= 1;  // (the other half may still be read)
    }
    if (w.s_out) {
        float* out = const_cast<float*>(w.s_out);
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const int r = g + 16 * i;
            if (r >= w.dk) continue;
            float* at = out + plane + (int64_t)r * w.dv + c;
            if (!w.turned && have >= 4 && (w.dv & 3) == 0 && ((uintptr_t)out & 15) == 0) *reinterpret_cast<float4*>(at) = s[i];
            else four(s[i], r, [&](float& e, int64_t p) { out[p] = e; });
        }
    }
    // behind a video's end
    if (w.o.p) {
        const int cols = w.dv - slice * 64 < 64 ? w.dv - slice * 64 : 64;
        for (int64_t i = (int64_t)frames * 64 + tid; i < (int64_t)w.t * 64; i += 256) {
            const int col = (int)(i & 63);
            if (col < cols) store_elem(o + (i >> 6) * w.o.frame + slice * 64 + col, 0.0f);
        }
    }
}

template <typename T>
hipError_t launch_steps(const Walk& w, hipStream_t s) {
    const int64_t groups = (int64_t)w.n * w.h * ((w.dv + 63) / 64);
    in_parts(groups, [&](unsigned first, unsigned count) {
        if (w.dk <= 64) hipLaunchKernelGGL((step_kernel<T, 4>), dim3(count), dim3(256), 0, s, w, first);
        else if (w.dk <= 128) hipLaunchKernelGGL((step_kernel<T, 8>), dim3(count), dim3(256), 0, s, w, first);
        else hipLaunchKernelGGL((step_kernel<T, 16>), dim3(count), dim3(256), 0, s, w, first);
    });
    return hipGetLastError();
}
hipError_t launch_walk(const Walk& w, int elem, hipStream_t s) {
    return elem == RRM_F32 ? launch_steps<float>(w, s) : launch_steps<__bf16>(w, s);
}

}  // namespace

size_t decay_scratch(const rrm_decay_desc&, bool) { return 0; }

hipError_t launch_decay_attention(const rrm_decay_desc& d, const void* q, const void* k, const void* v, const float* log_decay, const float* s0,
                                  const int32_t* lengths, void* o, float* s_last, void*, hipStream_t s) {
    Walk w{};
    w.q = {q, d.q_video, d.q_frame, d.q_head}, w.k = {k, d.k_video, d.k_frame, d.k_head};
    w.v = {v, d.v_video, d.v_frame, d.v_head}, w.o = {o, d.o_video, d.o_frame, d.o_head};
    w.n = d.n, w.t = d.t, w.h = d.h, w.dk = d.dk, w.dv = d.dv;
    w.s_in = s0, w.s_out = s_last;
    w.taken = 1.0f, w.given = d.scale;
    w.log_decay = log_decay, w.lengths = lengths;
    return launch_walk(w, d.elem, s);
}

hipError_t launch_decay_attention_backward(const rrm_decay_desc& d, const void* q, const void* k, const void* v, const float* log_decay,
                                           const float* s0, const int32_t* lengths, const void* d_o, const float* ds_last, void* dq,
                                           void* dk, void* dv, float* ds0, void*, hipStream_t s) {
    const Operand oq{q, d.q_video, d.q_frame, d.q_head}, ok{k, d.k_video, d.k_frame, d.k_head}, ov{v, d.v_video, d.v_frame, d.v_head};
    const Operand odo{d_o, d.o_video, d.o_frame, d.o_head};
    Walk w{};
    w.n = d.n, w.t = d.t, w.h = d.h, w.log_decay = log_decay, w.lengths = lengths;
    hipError_t e = hipSuccess;
    if (dq && d.t > 0) {
        w.q = odo, w.k = ov, w.v = ok, w.o = {dq, d.dq_video, d.dq_frame, d.dq_head};
        w.dk = d.dv, w.dv = d.dk, w.s_in = s0, w.s_out = nullptr, w.turned = true, w.back = false;
        w.taken = 1.0f, w.given = d.scale;
        if ((e = launch_walk(w, d.elem, s)) != hipSuccess) return e;
    }
    w.back = true, w.taken = d.scale, w.given = 1.0f, w.s_in = ds_last;
    if (dk && d.t > 0) {
        w.q = ov, w.k = odo, w.v = oq, w.o = {dk, d.dk_video, d.dk_frame, d.dk_head};
        w.dk = d.dv, w.dv = d.dk, w.s_out = nullptr, w.turned = true;
        if ((e = launch_walk(w, d.elem, s)) != hipSuccess) return e;
    }
    if ((dv && d.t > 0) || ds0) {
        w.q = ok, w.k = oq, w.v = odo, w.o = {dv, d.dv_video, d.dv_frame, d.dv_head};
        w.dk = d.dk, w.dv = d.dv, w.s_out = ds0, w.turned = false;
        e = launch_walk(w, d.elem, s);
    }
    return e;
}

}  // namespace rrm
