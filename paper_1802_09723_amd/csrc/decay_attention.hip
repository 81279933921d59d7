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


// ---- the walk in chunks, on the matrix cores ----------------------------------------------------------------------------
//
// Of C frames at once, i and j counted from a chunk's first, W the state before it:
//      result_i = sum over j up to i of lambda^(i-j) (q_i . k_j) v_j + lambda^(i+1) q_i W        W' = lambda^C W + sum of lambda^(C-1-j) k_j^T v_j
// (where the state decays behind a frame: lambda^i and lambda^(C-j)).  Only non-negative powers occur, so no decay overflows.
//
// A workgroup has a tile of DV columns of a head's state, in registers in 32 bits, and walks a stretch of frames; a wavefront makes 32 x 32 results and holds
// 32 columns of the state.  q, k, v of the next chunk are fetched into registers while this one is multiplied.  Products are v_mfma_f32_32x32x16_bf16 (fp32
// tensors: v_mfma_f32_32x32x2_f32).  In bfloat16 two operands are rounded: the scores with their decays, and the copy of the state that queries read;
// lambda^(C-1-j) v_j goes into the state as three bfloat16 parts, which hold all 24 bits of it, as the state's rounding errors would stay for as long as it remembers.
typedef float v16f __attribute__((ext_vector_type(16)));
typedef float v8f __attribute__((ext_vector_type(8)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4s* lds4_t;

// Eight elements along the summed axis of one row of an operand, of the 16 that a step takes
template <typename T>
struct FragmentOf;
template <>
struct FragmentOf<__bf16> {
    typedef v8bf type;
};
template <>
struct FragmentOf<float> {
    typedef v8f type;
};
template <typename T>
using Fragment = typename FragmentOf<T>::type;

__device__ __forceinline__ v16f multiply(v8bf a, v8bf b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ v16f multiply(v8f a, v8f b, v16f c) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
    return c;
}
// Rows that lie along the summed axis: lane l has row l % 32, and the eight from (l / 32) * 8 on
__device__ __forceinline__ v8bf along(const unsigned char* row, int step, int half, const __bf16*) {
    return *reinterpret_cast<const v8bf*>(row + step * 32 + half * 16);
}
__device__ __forceinline__ v8f along(const unsigned char* row, int step, int half, const float*) {
    return *reinterpret_cast<const v8f*>(row + step * 64 + half * 32);
}
// Rows that lie across it, turned on the way from LDS: lane l has column c0 + l % 32, and frames 4 (l / 32) + {0 .. 3, 8 .. 11} of the step's
// 16: the order in which the registers of a product hold its rows, so that scores need no turning
template <int PITCH>
__device__ __forceinline__ v8bf across(const unsigned char* tile, int c0, int step, int lane, const __bf16*) {
    const unsigned char* at = tile + (step * 16 + (lane >> 5) * 4 + ((lane >> 2) & 3)) * PITCH + c0 * 2 + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
    struct {
        v4s lo, hi;
    } v;
    v.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4_t)(at));
    v.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4_t)(at + 8 * PITCH));
    return __builtin_bit_cast(v8bf, v);
}
template <int PITCH>
__device__ __forceinline__ v8f across(const unsigned char* tile, int c0, int step, int lane, const float*) {
    v8f v;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        v[e] = *reinterpret_cast<const float*>(tile + (step * 16 + (lane >> 5) * 4 + (e & 3) + (e >> 2) * 8) * PITCH + (c0 + (lane & 31)) * 4);
    return v;
}
__device__ __forceinline__ float power(int e, float log2_decay) { return __builtin_amdgcn_exp2f((float)e * log2_decay); }
// (a decay of 0: its zeroth power is 1)
__device__ __forceinline__ float log2_of(float log_decay) { return fmaxf(log_decay * 1.44269504088896f, -16384.0f); }

// Stretches of the time axis, of `frames` frames each (whole chunks), a workgroup each: states[s] is the state before stretch s + 1, [pair][k][v]
// as the forward pass lays them, or what stretch s alone adds to it.
struct Stretches {
    int count, frames;
    float* states;
};

template <typename T, int DK, int DV, int C>
struct Chunk {
    static constexpr int IB = C / 32, DB = DV / 32, WAVES = IB * DB, THREADS = 64 * WAVES, SB = DK / 32 / IB;
    static constexpr int E = (int)sizeof(T), EPC = 16 / E;  // bytes of an element, elements of 16 bytes
    static constexpr int PK = DK * E + 32, PV = DV * E + 64;  // bytes between rows in LDS: reads of a wavefront meet different banks
    static constexpr int QK_BYTES = C * PK, V_BYTES = C * PV, S_BYTES = DV * PK;
    static constexpr int LDS = 2 * QK_BYTES + V_BYTES + S_BYTES, LDS_STATES = QK_BYTES + V_BYTES;
    static constexpr int NK = C * DK / EPC / THREADS, NV = C * DV / EPC / THREADS;  // 16-byte chunks a thread stages
    static_assert(NK * THREADS * EPC == C * DK && NV * THREADS * EPC == C * DV, "whole chunks a thread");
};

// STATES: what a stretch alone adds to the state (q and the results are not touched)
template <typename T, int DK, int DV, int C, bool STATES>
__global__ __launch_bounds__((Chunk<T, DK, DV, C>::THREADS)) void walk_kernel(Walk w, Stretches st, unsigned units, unsigned first) {
    using K = Chunk<T, DK, DV, C>;
    constexpr int IB = K::IB, SB = K::SB, EPC = K::EPC, STEPS = C / 16;
    __shared__ __attribute__((aligned(256))) unsigned char lds[STATES ? K::LDS_STATES : K::LDS];
    unsigned char* const ks = lds;
    unsigned char* const vs = ks + K::QK_BYTES;
    unsigned char* const qs = vs + K::V_BYTES;
    unsigned char* const ss = qs + K::QK_BYTES;
    const T* const tag = nullptr;

    // tiles of one head's state read the same q and k: beside one another on one XCD (workgroups go to the eight in turn)
    const int slices = (w.dv + DV - 1) / DV;
    const unsigned id = first + blockIdx.x, turn = id >> 3;
    const unsigned unit = (turn / slices) * 8 + (id & 7);
    if (unit >= units) return;
    const int slice = (int)(turn % slices);
    const int stretch = (int)(unit % st.count);
    const int pair = (int)(unit / st.count), video = pair / w.h, head = pair - video * w.h;
    const int end = frames_of(w, video), last = end > 0 ? (end - 1) / st.frames : 0;
    const int f0 = stretch * st.frames;                                     // (counted from the end where the walk goes back)
    const int have = end - f0 < st.frames ? end - f0 : st.frames;           // frames of this stretch, none or fewer behind the end
    if (STATES && stretch >= last) return;

    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, half = lane >> 5, lr = lane & 31;
    const int ib = wave % IB, db = wave / IB;
    const int c0 = slice * DV;  // first column
    const T* q = (const T*)w.q.p + video * w.q.video + head * w.q.head;
    const T* k = (const T*)w.k.p + video * w.k.video + head * w.k.head;
    const T* v = (const T*)w.v.p + video * w.v.video + head * w.v.head + c0;
    T* o = (T*)const_cast<void*>(w.o.p) + video * w.o.video + head * w.o.head + c0;
    const int vcols = w.dv - c0;
    const int64_t area = (int64_t)w.dk * w.dv;
    const int col = c0 + db * 32 + lr;  // of the state, this lane's

    // the state: block i, register 4 q + e: row (ib + i IB) 32 + 8 q + 4 half + e
    v16f state[SB];
    auto state_at = [&](int i, int r) { return (ib + i * IB) * 32 + 8 * (r >> 2) + 4 * half + (r & 3); };
    auto place = [&](int row) { return w.turned ? (int64_t)col * w.dk + row : (int64_t)row * w.dv + col; };
    const float* from = nullptr;
    if (!STATES) from = stretch == 0 ? (w.s_in ? w.s_in + pair * area : nullptr) : st.states + ((int64_t)(stretch - 1) * w.n * w.h + pair) * area;
#pragma unroll
    for (int i = 0; i < SB; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int row = state_at(i, r);
            state[i][r] = from && have >= 0 && row < w.dk && col < w.dv ? from[place(row)] : 0.0f;
        }

    const float decay = log2_of(w.t > 0 ? w.log_decay[head] : 0.0f);
    const int late = w.back ? 0 : 1;

    u32x4 hq[STATES ? 1 : K::NK], hk[K::NK], hv[K::NV];
    auto fetch_one = [&](const T* p, int64_t frame, int row, int c, int cols, int n) -> u32x4 {  // row of a chunk of n frames
        if (row >= n || c >= cols) return u32x4{0, 0, 0, 0};
        const T* at = p + (w.back ? -row : row) * frame + c;
        if (c + EPC <= cols) {
            unsigned int x[4];
            load_words<4>(at, x);
            return u32x4{x[0], x[1], x[2], x[3]};
        }
        u32x4 x = {0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < EPC - 1; ++e)
            if (c + e < cols) {
                if constexpr (sizeof(T) == 4) x[e] = __float_as_uint((float)at[e]);
                else x[e >> 1] |= (unsigned int)__builtin_bit_cast(unsigned short, at[e]) << (16 * (e & 1));
            }
        return x;
    };
    auto fetch = [&](int f) __attribute__((always_inline)) {  // the chunk from frame f0 + f on
        const int n = have - f;
        const int64_t at = w.back ? end - 1 - f0 - f : f0 + f;
        if (!STATES)
#pragma unroll
            for (int i = 0; i < K::NK; ++i) {
                const int x = i * K::THREADS + tid;
                hq[STATES ? 0 : i] = fetch_one(q + at * w.q.frame, w.q.frame, x / (DK / EPC), x % (DK / EPC) * EPC, w.dk, n);
            }
#pragma unroll
        for (int i = 0; i < K::NK; ++i) {
            const int x = i * K::THREADS + tid;
            hk[i] = fetch_one(k + at * w.k.frame, w.k.frame, x / (DK / EPC), x % (DK / EPC) * EPC, w.dk, n);
        }
#pragma unroll
        for (int i = 0; i < K::NV; ++i) {
            const int x = i * K::THREADS + tid;
            hv[i] = fetch_one(v + at * w.v.frame, w.v.frame, x / (DV / EPC), x % (DV / EPC) * EPC, vcols, n);
        }
    };
    auto put = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < K::NK; ++i) {
            const int x = i * K::THREADS + tid, at = x / (DK / EPC) * K::PK + x % (DK / EPC) * 16;
            if (!STATES) *reinterpret_cast<u32x4*>(qs + at) = hq[STATES ? 0 : i];
            *reinterpret_cast<u32x4*>(ks + at) = hk[i];
        }
#pragma unroll
        for (int i = 0; i < K::NV; ++i) {
            const int x = i * K::THREADS + tid;
            *reinterpret_cast<u32x4*>(vs + x / (DV / EPC) * K::PV + x % (DV / EPC) * 16) = hv[i];
        }
    };
    auto put_state = [&]() __attribute__((always_inline)) {  // [column][row]
#pragma unroll
        for (int i = 0; i < SB; ++i)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                unsigned char* at = ss + (db * 32 + lr) * K::PK + state_at(i, r) * K::E;
                if constexpr (sizeof(T) == 4) {
                    *reinterpret_cast<float4*>(at) = make_float4(state[i][r], state[i][r + 1], state[i][r + 2], state[i][r + 3]);
                } else {
                    u32x2 x;
                    x.x = bf16_pair(state[i][r], state[i][r + 1]), x.y = bf16_pair(state[i][r + 2], state[i][r + 3]);
                    *reinterpret_cast<u32x2*>(at) = x;
                }
            }
    };

    // lambda^(i-j) of a block of scores on the diagonal and of one below it (lane: i = l % 32; register 4 q + e: j = 8 q + 4 half + e)
    float on[16], below[IB > 1 ? 16 : 1];
    if (!STATES)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int d = lr - (8 * (r >> 2) + 4 * half + (r & 3));
            on[r] = d >= 0 ? w.given * w.taken * power(d, decay) : 0.0f;
            if (IB > 1) below[IB > 1 ? r : 0] = w.given * w.taken * power(d + 32, decay);
        }
    const float read = w.given * power(ib * 32 + lr + late, decay);
    float enter[STEPS][8], carry;  // lambda^(n-1-j) of the frames as `across` has them, lambda^n
    auto weights = [&](int n) __attribute__((always_inline)) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int d = n - late - (s * 16 + half * 4 + (e & 3) + (e >> 2) * 8);
                enter[s][e] = w.taken * power(d > 0 ? d : 0, decay);  // (behind the last frame: of zeros)
            }
        carry = power(n, decay);
    };
    weights(C);

    if (have > 0) fetch(0);
    for (int f = 0; f < have; f += C) {
        const int n = have - f;
        if (f > 0) __syncthreads();
        put();
        if (!STATES) put_state();
        if (f + C < have) fetch(f + C);
        __syncthreads();
        if (n < C) weights(n);
        v16f out;
        Fragment<T> score[STATES ? 1 : STEPS];
        if constexpr (!STATES) {
            const unsigned char* const mine = qs + (ib * 32 + lr) * K::PK;
#pragma unroll
            for (int r = 0; r < 16; ++r) out[r] = 0.0f;
#pragma unroll
            for (int s = 0; s < DK / 16; ++s)
                out = multiply(along(ss + (db * 32 + lr) * K::PK, s, half, tag), along(mine, s, half, tag), out);
#pragma unroll
            for (int r = 0; r < 16; ++r) out[r] *= read;
#pragma unroll
            for (int jb = 0; jb < IB; ++jb)
                if (jb <= ib) {
                    v16f p;
#pragma unroll
                    for (int r = 0; r < 16; ++r) p[r] = 0.0f;
#pragma unroll
                    for (int s = 0; s < DK / 16; ++s) p = multiply(along(ks + (jb * 32 + lr) * K::PK, s, half, tag), along(mine, s, half, tag), p);
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const float x = p[r] * (jb == ib ? on[r] : below[IB > 1 ? r : 0]);
                        if constexpr (sizeof(T) == 4) score[STATES ? 0 : jb * 2 + (r >> 3)][r & 7] = x;
                        else score[STATES ? 0 : jb * 2 + (r >> 3)][r & 7] = (__bf16)x;
                    }
                }
        }
#pragma unroll
        for (int i = 0; i < SB; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) state[i][r] *= carry;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const Fragment<T> fv = across<K::PV>(vs, db * 32, s, lane, tag);
            if constexpr (!STATES)
                if (s / 2 <= ib) out = multiply(fv, score[STATES ? 0 : s], out);
            Fragment<T> fk[SB];
#pragma unroll
            for (int i = 0; i < SB; ++i) fk[i] = across<K::PK>(ks, (ib + i * IB) * 32, s, lane, tag);
            if constexpr (sizeof(T) == 4) {
                Fragment<T> x;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = fv[e] * enter[s][e];
#pragma unroll
                for (int i = 0; i < SB; ++i) state[i] = multiply(fk[i], x, state[i]);
            } else {
                Fragment<T> hi, mid, lo;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float x = (float)fv[e] * enter[s][e];
                    hi[e] = (__bf16)x;
                    const float rest = x - (float)hi[e];
                    mid[e] = (__bf16)rest;
                    lo[e] = (__bf16)(rest - (float)mid[e]);
                }
#pragma unroll
                for (int i = 0; i < SB; ++i) {
                    state[i] = multiply(fk[i], hi, state[i]);
                    state[i] = multiply(fk[i], mid, state[i]);
                    state[i] = multiply(fk[i], lo, state[i]);
                }
            }
        }
        if constexpr (!STATES) {
            // lane: frame ib 32 + l % 32; registers 4 q + e: columns db 32 + 8 q + 4 half + e
            const int row = ib * 32 + lr;
            if (w.o.p && row < n) {
                T* to = o + (w.back ? end - 1 - f0 - f - row : (int64_t)f0 + f + row) * w.o.frame + db * 32;
                const int cols = vcols - db * 32;
                if constexpr (sizeof(T) == 4) {
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const int c = 8 * g + 4 * half;
                        if (c + 4 <= cols) {
                            const unsigned int x[4] = {__float_as_uint(out[4 * g]), __float_as_uint(out[4 * g + 1]), __float_as_uint(out[4 * g + 2]),
                                                       __float_as_uint(out[4 * g + 3])};
                            store_words<4>(to + c, x);
                        } else {
#pragma unroll
                            for (int e = 0; e < 3; ++e)
                                if (c + e < cols) to[c + e] = out[4 * g + e];
                        }
                    }
                } else {
#pragma unroll
                    for (int g = 0; g < 4; g += 2) {
                        // a lane gets the eight columns 8 (g + half) on: its own four of them and those of the lane 32 from it
                        const auto lo = __builtin_amdgcn_permlane32_swap(bf16_pair(out[4 * g], out[4 * g + 1]), bf16_pair(out[4 * g + 4], out[4 * g + 5]), false, false);
                        const auto hi = __builtin_amdgcn_permlane32_swap(bf16_pair(out[4 * g + 2], out[4 * g + 3]), bf16_pair(out[4 * g + 6], out[4 * g + 7]), false, false);
                        const unsigned int x[4] = {lo[0], hi[0], lo[1], hi[1]};
                        const int c = 8 * (g + half);
                        if (c + 8 <= cols) {
                            store_words<4>(to + c, x);
                        } else {
#pragma unroll
                            for (int e = 0; e < 7; ++e)
                                if (c + e < cols) to[c + e] = __builtin_bit_cast(__bf16, (unsigned short)(x[e >> 1] >> (16 * (e & 1))));
                        }
                    }
                }
            }
        }
    }

    float* keep = nullptr;
    if (STATES) keep = st.states + ((int64_t)stretch * w.n * w.h + pair) * area;
    else if (w.s_out && stretch == last) keep = const_cast<float*>(w.s_out) + pair * area;
    if (keep && col < w.dv) {
#pragma unroll
        for (int i = 0; i < SB; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int row = state_at(i, r);
                if (row < w.dk) keep[place(row)] = state[i][r];
            }
    }
    if (!STATES && w.o.p) {  // behind a video's end
        const int cols = vcols < DV ? vcols : DV, z0 = end > f0 ? end : f0;
        const int z1 = w.t - f0 < st.frames ? w.t : f0 + st.frames;
        for (int64_t i = (int64_t)z0 * DV + tid; i < (int64_t)z1 * DV; i += K::THREADS) {
            const int c = (int)(i % DV);
            if (c < cols) store_elem(o + i / DV * w.o.frame + c, 0.0f);
        }
    }
}

// From what the stretches add to the states before them: state s + 1 = lambda^frames state s + what stretch s adds
__global__ __launch_bounds__(256) void stretches_kernel(Walk w, Stretches st, int64_t area) {
    const int64_t pairs = (int64_t)w.n * w.h, total = pairs * area;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int pair = (int)(i / area), video = pair / w.h, head = pair - video * w.h;
        const int end = frames_of(w, video), last = end > 0 ? (end - 1) / st.frames : 0;
        const float carry = power(st.frames, log2_of(w.log_decay[head]));
        float s = w.s_in ? w.s_in[i] : 0.0f;
#pragma unroll 8
        for (int j = 0; j < last; ++j) {
            float* at = st.states + j * total + i;
            s = carry * s + *at;
            *at = s;
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

// Padded sizes of a walk's kernel: keys of 64, 128 or 256 features; tiles of 64 columns of the state, or of 128 where those leave none empty
// (fp32: 64, as LDS holds no more); chunks of 64 frames, for fp32 keys of more than 128 features 32, for the same reason.
template <typename T, typename F>
void with_chunk(const Walk& w, F&& f) {
    constexpr bool WIDE = sizeof(T) == 4;
    const bool two = !WIDE && ((w.dv + 63) / 64) % 2 == 0;
    if (w.dk <= 64) {
        if (two) f(Chunk<T, 64, WIDE ? 64 : 128, 64>{}, std::integral_constant<int, 64>{}, std::integral_constant<int, WIDE ? 64 : 128>{}, std::integral_constant<int, 64>{});
        else f(Chunk<T, 64, 64, 64>{}, std::integral_constant<int, 64>{}, std::integral_constant<int, 64>{}, std::integral_constant<int, 64>{});
    } else if (w.dk <= 128) {
        if (two) f(Chunk<T, 128, WIDE ? 64 : 128, 64>{}, std::integral_constant<int, 128>{}, std::integral_constant<int, WIDE ? 64 : 128>{}, std::integral_constant<int, 64>{});
        else f(Chunk<T, 128, 64, 64>{}, std::integral_constant<int, 128>{}, std::integral_constant<int, 64>{}, std::integral_constant<int, 64>{});
    } else {
        if (two) f(Chunk<T, 256, WIDE ? 64 : 128, WIDE ? 32 : 64>{}, std::integral_constant<int, 256>{}, std::integral_constant<int, WIDE ? 64 : 128>{}, std::integral_constant<int, WIDE ? 32 : 64>{});
        else f(Chunk<T, 256, 64, WIDE ? 32 : 64>{}, std::integral_constant<int, 256>{}, std::integral_constant<int, 64>{}, std::integral_constant<int, WIDE ? 32 : 64>{});
    }
}

// A frame or two of live videos: the state is the traffic, and each of its values is used once
bool few_frames(int t) { return t <= 2; }

// How the time axis is cut where n * h states alone would leave compute units without work.  A stretch costs what some four chunks do: its own state is written,
// joined and read, so it has eight at least.
Stretches stretches_of(const rrm_decay_desc& d, float* states) {
    Stretches st{1, 0x7fffff00, states};
    if (few_frames(d.t)) return st;
    const int64_t groups = (int64_t)d.n * d.h;
    const int chunks = (d.t + 63) / 64, most = chunks / 8;
    int64_t count = OP_CUS / groups;
    if (count > most) count = most;
    if (count < 2) return st;
    const int per = (int)((chunks + count - 1) / count);
    st.frames = per * 64;
    st.count = (chunks + per - 1) / per;
    return st;
}

template <typename T, bool STATES>
hipError_t launch_chunks(const Walk& w, const Stretches& st, hipStream_t s) {
    with_chunk<T>(w, [&](auto chunk, auto dk, auto dv, auto c) {
        using K = decltype(chunk);
        const unsigned units = (unsigned)((int64_t)w.n * w.h * st.count);
        const int64_t slices = (w.dv + decltype(dv)::value - 1) / decltype(dv)::value;
        in_parts(((int64_t)units + 7) / 8 * 8 * slices, [&](unsigned first, unsigned count) {
            hipLaunchKernelGGL((walk_kernel<T, decltype(dk)::value, decltype(dv)::value, decltype(c)::value, STATES>), dim3(count), dim3(K::THREADS), 0, s, w, st,
                               units, first);
        });
    });
    return hipGetLastError();
}
// What the stretches of a walk begin with
hipError_t launch_states(const Walk& w, const Stretches& st, int elem, hipStream_t s) {
    if (st.count < 2) return hipSuccess;
    hipError_t e = elem == RRM_F32 ? launch_chunks<float, true>(w, st, s) : launch_chunks<__bf16, true>(w, st, s);
    if (e != hipSuccess) return e;
    const int64_t area = (int64_t)w.dk * w.dv, groups = ((int64_t)w.n * w.h * area + 255) / 256;
    hipLaunchKernelGGL(stretches_kernel, dim3((unsigned)(groups < 8192 ? groups : 8192)), dim3(256), 0, s, w, st, area);
    return hipGetLastError();
}
hipError_t launch_walk(const Walk& w, const Stretches& st, int elem, hipStream_t s) {
    if (few_frames(w.t)) return elem == RRM_F32 ? launch_steps<float>(w, s) : launch_steps<__bf16>(w, s);
    return elem == RRM_F32 ? launch_chunks<float, false>(w, st, s) : launch_chunks<__bf16, false>(w, st, s);
}
size_t states_bytes(const rrm_decay_desc& d) {
    const Stretches st = stretches_of(d, nullptr);
    return st.count < 2 ? 0 : round256((size_t)(st.count - 1) * d.n * d.h * d.dk * d.dv * 4);
}

}  // namespace

// forward: [states of the stretches]; backward: those of S, those of D
size_t decay_scratch(const rrm_decay_desc& d, bool backward) { return states_bytes(d) * (backward ? 2 : 1); }

hipError_t launch_decay_attention(const rrm_decay_desc& d, const void* q, const void* k, const void* v, const float* log_decay, const float* s0,
                                  const int32_t* lengths, void* o, float* s_last, void* ws, hipStream_t s) {
    Walk w{};
    w.q = {q, d.q_video, d.q_frame, d.q_head}, w.k = {k, d.k_video, d.k_frame, d.k_head};
    w.v = {v, d.v_video, d.v_frame, d.v_head}, w.o = {o, d.o_video, d.o_frame, d.o_head};
    w.n = d.n, w.t = d.t, w.h = d.h, w.dk = d.dk, w.dv = d.dv;
    w.s_in = s0, w.s_out = s_last;
    w.taken = 1.0f, w.given = d.scale;
    w.log_decay = log_decay, w.lengths = lengths;
    const Stretches st = stretches_of(d, (float*)ws);
    const hipError_t e = launch_states(w, st, d.elem, s);
    return e == hipSuccess ? launch_walk(w, st, d.elem, s) : e;
}

hipError_t launch_decay_attention_backward(const rrm_decay_desc& d, const void* q, const void* k, const void* v, const float* log_decay,
                                           const float* s0, const int32_t* lengths, const void* d_o, const float* ds_last, void* dq,
                                           void* dk, void* dv, float* ds0, void* ws, hipStream_t s) {
    const Operand oq{q, d.q_video, d.q_frame, d.q_head}, ok{k, d.k_video, d.k_frame, d.k_head}, ov{v, d.v_video, d.v_frame, d.v_head};
    const Operand odo{d_o, d.o_video, d.o_frame, d.o_head};
    Walk w{};
    w.n = d.n, w.t = d.t, w.h = d.h, w.log_decay = log_decay, w.lengths = lengths;
    hipError_t e = hipSuccess;
    if (dq && d.t > 0) {
        const Stretches st = stretches_of(d, (float*)ws);
        w.k = ok, w.v = ov, w.dk = d.dk, w.dv = d.dv, w.s_in = s0, w.s_out = nullptr, w.taken = 1.0f, w.given = d.scale;
        if ((e = launch_states(w, st, d.elem, s)) != hipSuccess) return e;
        w.q = odo, w.k = ov, w.v = ok, w.o = {dq, d.dq_video, d.dq_frame, d.dq_head};
        w.dk = d.dv, w.dv = d.dk, w.turned = true;
        if ((e = launch_walk(w, st, d.elem, s)) != hipSuccess) return e;
    }
    const Stretches st = stretches_of(d, (float*)((unsigned char*)ws + states_bytes(d)));
    w.back = true, w.taken = d.scale, w.given = 1.0f, w.s_in = ds_last, w.s_out = nullptr;
    w.k = oq, w.v = odo, w.dk = d.dk, w.dv = d.dv, w.turned = false;
    if (d.t > 0 && (e = launch_states(w, st, d.elem, s)) != hipSuccess) return e;
    if (dk && d.t > 0) {
        w.q = ov, w.k = odo, w.v = oq, w.o = {dk, d.dk_video, d.dk_frame, d.dk_head};
        w.dk = d.dv, w.dv = d.dk, w.turned = true;
        if ((e = launch_walk(w, st, d.elem, s)) != hipSuccess) return e;
    }
    if ((dv && d.t > 0) || ds0) {
        w.q = ok, w.k = oq, w.v = odo, w.o = {dv, d.dv_video, d.dv_frame, d.dv_head};
        w.dk = d.dk, w.dv = d.dv, w.s_out = ds0, w.turned = false;
        e = launch_walk(w, st, d.elem, s);
    }
    return e;
}

}  // namespace rrm
