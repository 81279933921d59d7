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
    // In chunks, a launch takes `dk` of the state's keys, from `first_key` on, of `keys` in all (q and k begin with them).  What the keys before give waits in
    // `part`, fp32 [n][t][h][dv]: written by a launch that is not the last, added by one that is not the first.
    int first_key, keys;
    bool adds, leaves;
    float* part;
};

__device__ __forceinline__ int frames_of(const Walk& w, int video) {
    if (!w.lengths) return w.t;
    const int e = w.lengths[video];
    return e < 0 ? 0 : e < w.t ? e : w.t;
}

// The recurrence as it stands, a state in registers: one frame of live videos (and the walk for any).  A workgroup has 64 columns of a head's state; thread
// (g, quad) holds rows g, g + 16, .. of four columns.  The state's two ways are what bounds it: 64 videos of 16 heads of 128 x 128 take 28.6 us, 4.7 TB/s.
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
// (where the state decays behind a frame: lambda^i and lambda^(C-j)).  Only non-negative powers occur, so no decay overflows; memories that grow: see `grows`.
//
// A workgroup has a tile of DV columns of a head's state, in registers in 32 bits, and walks a stretch of frames; a wavefront has 16 of the columns and makes
// the results of all C frames in them.  q, k, v of the next chunk are fetched into registers while this one is multiplied.  Products are
// v_mfma_f32_16x16x32_bf16 (fp32 tensors: v_mfma_f32_16x16x4_f32); the state's registers are an operand as they stand, and the scores, made once, meet the
// wavefronts through LDS.  In bfloat16 two operands are rounded: the scores with their decays, and the state where queries read it;
// lambda^(C-1-j) v_j goes into the state as three bfloat16 parts, which hold all 24 bits of it, as the state's rounding errors stay for as long as it remembers.
// 64 videos of 256 frames, 32 heads of 128 x 128, bf16: 184 us, 4.4 TB/s (with one part of three 159).  One of 65536 frames, 8 heads: 68 for what stretches add, 12 for
// their sums, 144 for the results, in a quarter of whose cycles the matrix cores are busy: a chunk is a chain of fetches, LDS, scores, products and two
// barriers, and registers (state, results and the next chunk's vectors: 128 each) let four wavefronts share a SIMD.
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v8f __attribute__((ext_vector_type(8)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4s* lds4_t;

// Eight elements along the summed axis of one row of an operand, of the 32 that a step takes
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

// Lane l of the result: row 4 (l / 16) + register of a, column l % 16 (a row of b)
__device__ __forceinline__ v4f multiply(v8bf a, v8bf b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ v4f multiply(v8f a, v8f b, v4f c) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
    return c;
}
// Rows that lie along the summed axis: lane l has row l % 16, and the eight from 8 (l / 16) on
__device__ __forceinline__ v8bf along(const unsigned char* row, int step, int g, const __bf16*) { return *reinterpret_cast<const v8bf*>(row + step * 64 + g * 16); }
__device__ __forceinline__ v8f along(const unsigned char* row, int step, int g, const float*) {
    struct {
        float4 lo, hi;
    } v;
    v.lo = *reinterpret_cast<const float4*>(row + step * 128 + g * 32);
    v.hi = *reinterpret_cast<const float4*>(row + step * 128 + g * 32 + 16);
    return __builtin_bit_cast(v8f, v);
}
// The same with the eight that lane l holds of two results' rows, 4 (l / 16) + {0 .. 3, 16 .. 19}: the order of the state in its registers
__device__ __forceinline__ v8bf along_state(const unsigned char* row, int step, int g, const __bf16*) {
    struct {
        u32x2 lo, hi;
    } v;
    v.lo = *reinterpret_cast<const u32x2*>(row + step * 64 + g * 8);
    v.hi = *reinterpret_cast<const u32x2*>(row + step * 64 + g * 8 + 32);
    return __builtin_bit_cast(v8bf, v);
}
__device__ __forceinline__ v8f along_state(const unsigned char* row, int step, int g, const float*) {
    struct {
        float4 lo, hi;
    } v;
    v.lo = *reinterpret_cast<const float4*>(row + step * 128 + g * 16);
    v.hi = *reinterpret_cast<const float4*>(row + step * 128 + g * 16 + 64);
    return __builtin_bit_cast(v8f, v);
}
// Rows that lie across it, turned on the way from LDS: lane l has column c0 + l % 16, and the step's frames from 8 (l / 16) on
template <int PITCH>
__device__ __forceinline__ v8bf across(const unsigned char* tile, int c0, int step, int lane, const __bf16*) {
    const unsigned char* at = tile + (step * 32 + (lane >> 4) * 8 + ((lane >> 2) & 3)) * PITCH + c0 * 2 + (lane & 3) * 8;
    struct {
        v4s lo, hi;
    } v;
    v.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4_t)(at));
    v.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4_t)(at + 4 * PITCH));
    return __builtin_bit_cast(v8bf, v);
}
template <int PITCH>
__device__ __forceinline__ v8f across(const unsigned char* tile, int c0, int step, int lane, const float*) {
    v8f v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = *reinterpret_cast<const float*>(tile + (step * 32 + (lane >> 4) * 8 + e) * PITCH + (c0 + (lane & 15)) * 4);
    return v;
}
__device__ __forceinline__ float power(int e, float log2_decay) { return __builtin_amdgcn_exp2f((float)e * log2_decay); }
// (a decay of 0: its zeroth power is 1)
__device__ __forceinline__ float log2_of(float log_decay) {
    const float x = log_decay * 1.44269504088896f;
    return x < -16384.0f ? -16384.0f : x;  // (a not-a-number stays one)
}
__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

// Stretches of the time axis, of `frames` frames each (whole chunks), a workgroup each (none: the walk goes frame by frame): states[s] is the state before stretch
// s + 1, [pair][k][v] as the forward pass lays them, or what stretch s alone adds to it.
struct Stretches {
    int count, frames;
    float* states;
};

// An offset behind every buffer's end: reads zeros, writes nothing
constexpr unsigned NOWHERE = 0xfffffff0u;

// A barrier that waits for LDS alone: what is fetched of the next chunk stays on its way (__syncthreads would wait for it)
__device__ __forceinline__ void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

template <typename T, int DK, int DV, int C>
struct Chunk {
    static constexpr int WAVES = DV / 16, THREADS = 64 * WAVES;
    static constexpr int E = (int)sizeof(T), EPC = 16 / E;                                // bytes of an element, elements of 16 bytes
    // bytes between rows in LDS: reads along rows meet different banks; those across them (turned on the way) do in part only: conflicts take 0.18 of the busy cycles of
    // 64 videos of 256 frames, 0.26 of the walk of one of 65536
    static constexpr int PK = DK * E + 16, PV = DV * E + 32, PP = C * E + 16;
    static constexpr int QK_BYTES = C * PK, V_BYTES = C * PV, P_BYTES = C * PP;
    static constexpr int LDS = 2 * QK_BYTES + V_BYTES + P_BYTES, LDS_STATES = QK_BYTES + V_BYTES;
    static constexpr int RK = THREADS / (DK / EPC), RV = THREADS / (DV / EPC);            // rows staged at once, a thread 16 bytes ..
    static constexpr int NK = (C + RK - 1) / RK, NV = (C + RV - 1) / RV;                  // .. and how many times
    static constexpr int AT_ONCE = (WAVES * (163840 / LDS < 2 ? 1 : 2) + 3) / 4;           // wavefronts on a SIMD
};

// STATES: what a stretch alone adds to the state (q and the results are not touched).  EXACT: rows of q, k and v are whole pieces of 16 bytes.
template <typename T, int DK, int DV, int C, bool STATES, bool EXACT>
__global__ __launch_bounds__((Chunk<T, DK, DV, C>::THREADS)) __attribute__((amdgpu_waves_per_eu(Chunk<T, DK, DV, C>::AT_ONCE, Chunk<T, DK, DV, C>::AT_ONCE)))
void walk_kernel(Walk w, Stretches st, unsigned units, unsigned first) {
    using K = Chunk<T, DK, DV, C>;
    constexpr int SB = DK / 16, IB = C / 16, STEPS = C / 32, EPC = K::EPC;
    __shared__ __attribute__((aligned(256))) unsigned char lds[STATES ? K::LDS_STATES : K::LDS];
    unsigned char* const ks = lds;
    unsigned char* const vs = ks + K::QK_BYTES;
    unsigned char* const qs = vs + K::V_BYTES;
    unsigned char* const ps = qs + K::QK_BYTES;
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
    const int f0 = stretch * st.frames;                            // (counted from the end where the walk goes back)
    const int have = end - f0 < st.frames ? end - f0 : st.frames;  // frames of this stretch, none or fewer behind the end
    if (STATES && stretch >= last) return;

    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, lr = lane & 15;
    const int c0 = slice * DV, vcols = w.dv - c0;  // first column; columns from it on
    const T* q = (const T*)w.q.p + video * w.q.video + head * w.q.head;
    const T* k = (const T*)w.k.p + video * w.k.video + head * w.k.head;
    const T* v = (const T*)w.v.p + video * w.v.video + head * w.v.head;
    T* o = (T*)const_cast<void*>(w.o.p) + video * w.o.video + head * w.o.head + c0;
    const int64_t area = (int64_t)w.keys * w.dv;
    const int col = c0 + wave * 16 + lr;  // of the state, this lane's

    // the state: block i, register r: row 16 i + 4 g + r
    // (an offset behind the buffer's end reads a zero: with a branch for each the loads may be waited for one by one, 273 us for 187)
    v4f state[SB];
    const int64_t row_step = w.turned ? 1 : w.dv, corner = (w.turned ? (int64_t)col * w.keys : col) + w.first_key * row_step;
    const float* from = nullptr;
    if (!STATES) from = stretch == 0 ? (w.s_in ? w.s_in + pair * area : nullptr) : st.states + ((int64_t)(stretch - 1) * w.n * w.h + pair) * area;
    {
        const auto buffer = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(from), 0, from && have >= 0 ? (int)area * 4 : 0, 0x00027000);
#pragma unroll
        for (int i = 0; i < SB; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * i + 4 * g + r;
                const unsigned at = row < w.dk && col < w.dv ? (unsigned)(corner + row * row_step) * 4 : NOWHERE;
                state[i][r] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(buffer, at, 0, 0));
            }
    }

    const float decay = log2_of(w.t > 0 ? w.log_decay[head] : 0.0f);
    const int late = w.back ? 0 : 1;
    // A memory that grows so fast that powers over a chunk (a stretch, where there are several) pass 2^64: they may soon be infinities, which times the zeros of
    // absent frames are none of the results.  Such a head takes no chunks, it goes frame by frame below, all of a video in the first stretch's workgroup (128 x 128:
    // 3.9 us a frame).
    auto grows = [&](float decay) { return decay * (float)(st.count > 1 ? st.frames : C) > 64.0f; };
    if (STATES && grows(decay)) return;
    const int chunked = grows(decay) ? 0 : have;

    // This thread's 16 bytes of every RK-th row of q and k (of every RV-th of v): rows row + i RK, columns c on.  The last piece of a row that no whole
    // pieces make up begins early.  (frames lie at most 2^22 elements apart: offsets within a chunk have 32 bits)
    struct Part {
        int row, c;
        bool in, whole, idle;
        unsigned at;  // bytes from the lowest of the chunk's frames in memory ..
        int apart;    // .. and between the rows
    };
    auto part_of = [&](int per, int rows, int64_t frame, int c0, int cols) {  // per: pieces in a row of LDS; columns c0 .. c0 + cols
        Part p;
        p.row = tid / per, p.c = tid % per * EPC;
        p.idle = p.row >= rows;
        p.in = p.c < cols && !p.idle, p.whole = p.c + EPC <= cols;
        if (!EXACT && !p.whole) p.c = cols - EPC;
        p.at = (unsigned)(((w.back ? rows - 1 - p.row : p.row) * frame + c0 + p.c) * K::E);
        p.apart = (int)(rows * frame * K::E);
        return p;
    };
    const Part pq = part_of(DK / EPC, K::RK, w.q.frame, 0, w.dk), pk = part_of(DK / EPC, K::RK, w.k.frame, 0, w.dk),
               pv = part_of(DV / EPC, K::RV, w.v.frame, c0, vcols);
    // (an offset behind a buffer's end reads zeros: no branches, and loads stay on their way)
    auto fetch_rows = [&](u32x4* held, auto count, auto rows, const T* p, int64_t frame, const Part& part, int f) __attribute__((always_inline)) {
        constexpr int N = decltype(count)::value, R = decltype(rows)::value;
        const int none = chunked - f < C ? C - (chunked - f) : 0;
        const int64_t lowest = w.back ? (int64_t)(end - 1 - f0 - f) + none - (N * R - 1) : (int64_t)f0 + f - none;
        const auto buffer = __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(p + lowest * frame), 0, 0x7fffffff, 0x00027000);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int row = part.row + i * R;
            const bool there = part.in && row >= none && (N * R == C || row < C);
            held[i] = __builtin_amdgcn_raw_buffer_load_b128(buffer, there ? part.at : NOWHERE, (w.back ? N - 1 - i : i) * part.apart, 0);
        }
    };
    const std::integral_constant<int, K::NK> nk;
    const std::integral_constant<int, K::NV> nv;
    const std::integral_constant<int, K::RK> rk;
    const std::integral_constant<int, K::RV> rv;
    u32x4 hq[STATES ? 1 : K::NK], hk[K::NK], hv[K::NV];
    auto fetch = [&](int f) __attribute__((always_inline)) {  // the chunk from frame f0 + f on
        fetch_rows(hk, nk, rk, k, w.k.frame, pk, f);
        if constexpr (!STATES) fetch_rows(hq, nk, rk, q, w.q.frame, pq, f);
        fetch_rows(hv, nv, rv, v, w.v.frame, pv, f);
    };
    auto put_row = [&](unsigned char* to, const Part& part, const u32x4& x, bool there) __attribute__((always_inline)) {
        if (!there) return;
        if (EXACT || part.whole) {
            *reinterpret_cast<u32x4*>(to + part.c * K::E) = x;  // (behind the last column: zeros)
        } else if (part.in) {
#pragma unroll
            for (int e = 0; e < EPC; ++e) {
                if (part.c + e < 0) continue;  // (of the tile before)
                if constexpr (sizeof(T) == 4) *reinterpret_cast<unsigned int*>(to + (part.c + e) * 4) = x[e];
                else *reinterpret_cast<unsigned short*>(to + (part.c + e) * 2) = (unsigned short)(x[e >> 1] >> (16 * (e & 1)));
            }
        }
    };
    auto put = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < K::NK; ++i) {
            const int row = pk.row + i * K::RK;
            const bool there = (K::THREADS % (DK / EPC) == 0 || !pk.idle) && (K::NK * K::RK == C || row < C);
            put_row(ks + row * K::PK, pk, hk[i], there);
            if constexpr (!STATES) put_row(qs + row * K::PK, pk, hq[i], there);
        }
#pragma unroll
        for (int i = 0; i < K::NV; ++i) {
            const int row = pv.row + i * K::RV;
            put_row(vs + row * K::PV, pv, hv[i], (K::THREADS % (DV / EPC) == 0 || !pv.idle) && (K::NV * K::RV == C || row < C));
        }
    };
    // once: zeros behind the last column, and above the diagonal of the scores
    if (!EXACT) {
        for (int i = tid; i < (STATES ? K::LDS_STATES : K::LDS) / 16; i += K::THREADS) *reinterpret_cast<u32x4*>(lds + i * 16) = u32x4{0, 0, 0, 0};
        meet();
    } else if (!STATES) {
        for (int i = tid; i < K::P_BYTES / 16; i += K::THREADS) *reinterpret_cast<u32x4*>(ps + i * 16) = u32x4{0, 0, 0, 0};
        meet();
    }

    const unsigned o_at = (unsigned)(((w.back ? 15 - lr : lr) * w.o.frame + wave * 16 + 4 * g) * K::E);  // a result, as Part::at

    // lambda^(C-1-j) of the frames as `across` has them: lambda^(31-j) within a step, and the steps behind it
    float enter[8], steps[STEPS];
#pragma unroll
    for (int e = 0; e < 8; ++e) enter[e] = w.taken * power(32 - late - g * 8 - e, decay);
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
        steps[s] = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(power(C - 32 - 32 * s, decay))));

    if (chunked > 0) fetch(0);
    for (int f = 0; f < chunked; f += C) {
        // a chunk of fewer frames has them in its last rows, zeros before: every power but two stays as it is
        const int none = chunked - f < C ? C - (chunked - f) : 0;
        const float carry = power(C - none, decay);
        if (f > 0) meet();
        put();
        if (f + C < chunked) fetch(f + C);
        meet();
        v4f out[STATES ? 1 : IB];
        if constexpr (!STATES) {
            // blocks of scores on and below the diagonal, a wavefront each: lane: i = 16 ib + l % 16; register r: j = 16 jb + 4 g + r
            for (int b = wave; b < IB * (IB + 1) / 2; b += K::WAVES) {
                const int ib = b < 1 ? 0 : b < 3 ? 1 : b < 6 ? 2 : 3, jb = b - ib * (ib + 1) / 2;
                v4f p = {0, 0, 0, 0};
#pragma unroll
                for (int s = 0; s < DK / 32; ++s)
                    p = multiply(along(ks + (jb * 16 + lr) * K::PK, s, g, tag), along(qs + (ib * 16 + lr) * K::PK, s, g, tag), p);
                unsigned char* const to = ps + (ib * 16 + lr) * K::PP + (jb * 16 + 4 * g) * K::E;
                float x[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int d = (ib - jb) * 16 + lr - 4 * g - r;
                    x[r] = d >= 0 ? p[r] * (w.given * w.taken * power(d, decay)) : 0.0f;  // (q . k of frames to come may be infinite)
                }
                if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(to) = make_float4(x[0], x[1], x[2], x[3]);
                else *reinterpret_cast<u32x2*>(to) = u32x2{bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3])};
            }
            // what the state before gives: its registers are the operand
#pragma unroll
            for (int ib = 0; ib < IB; ++ib) out[ib] = v4f{0, 0, 0, 0};
#pragma unroll
            for (int s = 0; s < DK / 32; ++s) {
                Fragment<T> x;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if constexpr (sizeof(T) == 4) x[e] = state[2 * s + (e >> 2)][e & 3];
                    else x[e] = (__bf16)state[2 * s + (e >> 2)][e & 3];
                }
#pragma unroll
                for (int ib = 0; ib < IB; ++ib) out[ib] = multiply(x, along_state(qs + (ib * 16 + lr) * K::PK, s, g, tag), out[ib]);
            }
#pragma unroll
            for (int ib = 0; ib < IB; ++ib) {
                const int d = ib * 16 + lr - none + late;
                out[ib] *= w.given * power(d > 0 ? d : 0, decay);
            }
            meet();
        }
#pragma unroll
        for (int i = 0; i < SB; ++i) state[i] *= carry;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const Fragment<T> fv = across<K::PV>(vs, wave * 16, s, lane, tag);
            if constexpr (!STATES)
#pragma unroll
                for (int ib = 2 * s; ib < IB; ++ib) out[ib] = multiply(fv, along(ps + (ib * 16 + lr) * K::PP, s, g, tag), out[ib]);
            if constexpr (sizeof(T) == 4) {
                Fragment<T> x;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = fv[e] * enter[e] * steps[s];
#pragma unroll
                for (int i = 0; i < SB; ++i) state[i] = multiply(across<K::PK>(ks, i * 16, s, lane, tag), x, state[i]);
            } else {
                Fragment<T> hi, mid, lo;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float x = (float)fv[e] * enter[e] * steps[s];
                    hi[e] = (__bf16)x;
                    const float rest = x - (float)hi[e];
                    mid[e] = (__bf16)rest;
                    lo[e] = (__bf16)(rest - (float)mid[e]);
                }
#pragma unroll
                for (int i = 0; i < SB; ++i) {
                    const Fragment<T> fk = across<K::PK>(ks, i * 16, s, lane, tag);
                    state[i] = multiply(fk, hi, state[i]);
                    state[i] = multiply(fk, mid, state[i]);
                    state[i] = multiply(fk, lo, state[i]);
                }
            }
        }
        if constexpr (!STATES) {
            // lane: frame 16 ib + l % 16; register r: column 16 wave + 4 g + r
            const int c = wave * 16 + 4 * g;
            const int64_t lowest = w.back ? (int64_t)(end - 1 - f0 - f) + none - (C - 1) : (int64_t)f0 + f - none;
            const auto buffer = __builtin_amdgcn_make_buffer_rsrc(o + lowest * w.o.frame, 0, 0x7fffffff, 0x00027000);
#pragma unroll
            for (int ib = 0; ib < IB; ++ib) {
                const int row = ib * 16 + lr;
                if (w.adds || w.leaves) {
                    float* const part = w.part + ((video * (int64_t)w.t + lowest + (w.back ? C - 1 - row : row)) * w.h + head) * w.dv + c0 + c;
                    if (row >= none && w.o.p)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (c + e < vcols) {
                                if (w.adds) out[ib][e] += part[e];
                                if (w.leaves) part[e] = out[ib][e];
                            }
                    if (w.leaves) continue;
                }
                const bool goes = row >= none && w.o.p;
                const int apart = (w.back ? IB - 1 - ib : ib) * 16 * (int)w.o.frame * K::E;
                if (EXACT || c + 4 <= vcols || c >= vcols) {
                    const unsigned to = goes && c < vcols ? o_at : NOWHERE;
                    if constexpr (sizeof(T) == 4) {
                        const u32x4 x = {__float_as_uint(out[ib][0]), __float_as_uint(out[ib][1]), __float_as_uint(out[ib][2]), __float_as_uint(out[ib][3])};
                        __builtin_amdgcn_raw_buffer_store_b128(x, buffer, to, apart, 0);
                    } else {
                        const u32x2 x = {bf16_pair(out[ib][0], out[ib][1]), bf16_pair(out[ib][2], out[ib][3])};
                        __builtin_amdgcn_raw_buffer_store_b64(x, buffer, to, apart, 0);
                    }
                } else if (goes) {
#pragma unroll
                    for (int e = 0; e < 3; ++e)
                        if (c + e < vcols) store_elem((T*)((unsigned char*)(o + lowest * w.o.frame) + (o_at + (unsigned)apart)) + e, out[ib][e]);
                }
            }
        }
    }

    float again = decay;
    asm volatile("" : "+v"(again));  // (or what follows from it is held over the walk)
    const bool growing = !STATES && grows(again);
    float* keep = nullptr;
    if (STATES) keep = st.states + ((int64_t)stretch * w.n * w.h + pair) * area;
    else if (w.s_out && stretch == (growing ? 0 : last)) keep = const_cast<float*>(w.s_out) + pair * area;
    auto leave_state = [&]() __attribute__((always_inline)) {
        if (!keep || col >= w.dv) return;
        int g4 = 4 * g;
        asm("" : "+v"(g4));  // (or the places of all values are held from where the state was read)
#pragma unroll
        for (int i = 0; i < SB; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * i + g4 + r;
                if (row < w.dk) keep[corner + row * row_step] = state[i][r];
            }
    };
    if (!growing) leave_state();
    if constexpr (!STATES) {
        // Masked places are zeros among a chunk's scores, and 0 times a v that is not finite has reached the chunk's frames before it.  Such a v stays in the state:
        // where the state has ended so, the frames before the first of them are made again, as the recurrence stands, by this wavefront for its columns (128 x 128: 0.9
        // us a frame of one head alone, 4.5 where the card is full).  All frames of a memory that grows fast are made so.
        const bool ended = col < w.dv && 4 * g < w.dk && !finite(state[0][0]);
        const int frames = growing ? (stretch == 0 ? end : 0) : have;
        if (growing || (w.o.p && __any(ended))) {
            __threadfence();  // (behind the results as they are)
            const float lambda = expf(w.log_decay[head]);
            int g4 = 4 * g;
            asm volatile("" : "+v"(g4));  // (or conditions of rows are held from here on)
#pragma unroll
            for (int i = 0; i < SB; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int row = 16 * i + g4 + r;
                    state[i][r] = from && row < w.dk && col < w.dv ? from[corner + row * row_step] : 0.0f;
                }
            for (int f = 0; f < frames && (growing || __any(ended && finite(state[0][0]))); ++f) {
                const int64_t at = w.back ? end - 1 - f0 - f : f0 + f;
                const float vf = col < w.dv ? w.taken * load_elem(v + at * w.v.frame + col) : 0.0f;
                float sum = 0.0f;
#pragma unroll
                for (int i = 0; i < SB; ++i) {
                    asm volatile("" : "+v"(g4));
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int row = 16 * i + g4 + r;
                        if (row >= w.dk) continue;
                        if (!w.back) state[i][r] *= lambda;
                        state[i][r] += load_elem(k + at * w.k.frame + row) * vf;
                        sum += load_elem(q + at * w.q.frame + row) * state[i][r];
                        if (w.back) state[i][r] *= lambda;
                    }
                }
                sum += __shfl_xor(sum, 16);
                sum = w.given * (sum + __shfl_xor(sum, 32));
                if (g == 0 && col < w.dv && w.o.p) {
                    float* const part = w.part + ((video * (int64_t)w.t + at) * w.h + head) * w.dv + col;
                    if (w.adds) sum += *part;
                    if (w.leaves) *part = sum;
                    else store_elem(o + at * w.o.frame + wave * 16 + lr, sum);
                }
            }
            if (growing) leave_state();
        }
    }
    if (!STATES && w.o.p && !w.leaves) {  // behind a video's end
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
        float* at = st.states + i;
        for (int j = 0; j < last; j += 16) {  // sixteen on their way at once
            float adds[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) adds[e] = j + e < last ? at[(j + e) * total] : 0.0f;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s = carry * s + adds[e];
                if (j + e < last) at[(j + e) * total] = s;
            }
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

// Padded sizes of a walk's kernel: 64, 96, 128 or 160 keys (fp32: 64 or 128), and tiles of the state of 64, 96 or 128 columns: those with the fewest in all, the widest
// of them.  Up to 64 keys, and for more than 128, tiles are of 64: registers and LDS hold two workgroups of those.  80 x 136, four videos of up to 8192 frames, both
// ways: 718 us; with 64 and 128 keys and tiles of 64 and 128 only, and so 136 keys half by half, 1016.  128 x 128 in two tiles of 64 columns: 205 for the 144 above.
template <typename T, typename F>
void with_chunk(const Walk& w, F&& f) {
    const std::integral_constant<int, 64> c64;
    const std::integral_constant<int, 96> c96;
    const std::integral_constant<int, 128> c128;
    const std::integral_constant<int, 160> c160;
    auto padded = [&](int tile) { return (w.dv + tile - 1) / tile * tile; };
    if (w.dk <= 64) return f(c64, c64);
    if constexpr (sizeof(T) == 4) {
        padded(128) <= padded(64) ? f(c128, c128) : f(c128, c64);
    } else {
        if (w.dk > 128) return f(c160, c64);
        const bool wide = padded(128) <= padded(64) && padded(128) <= padded(96), middle = padded(96) <= padded(64);
        if (w.dk > 96) return wide ? f(c128, c128) : middle ? f(c128, c96) : f(c128, c64);
        wide ? f(c96, c128) : middle ? f(c96, c96) : f(c96, c64);
    }
}
// More keys than that are taken half by half: a state's rows have nothing to do with each other, and results are sums over them.  (A kernel of 256 keys has more
// state than registers beside its fragments.)
int most_keys(int elem) { return elem == RRM_F32 ? 128 : 160; }

// A frame or two of live videos: the state is the traffic, and each of its values is used once; a chunk of 64 would be zeros but for them
bool few_frames(int t) { return t <= 2; }
// ... and frames that lie backwards or very far apart, which the chunks' 32-bit offsets do not reach, or rows of less than 16 bytes
bool by_steps(const rrm_decay_desc& d) {
    if (few_frames(d.t) || d.dk < 8 || d.dv < 8) return true;
    for (int64_t frame : {d.q_frame, d.k_frame, d.v_frame, d.o_frame, d.dq_frame, d.dk_frame, d.dv_frame})
        if (frame < 0 || frame > (1 << 22)) return true;
    return false;
}

// How the time axis is cut where n * h states alone would leave compute units without work: into as many stretches as make two for each unit, but of eight chunks at
// least (fp32: three).  A stretch costs its own state, written, joined and read, and two launches, which is some four chunks of bf16 and one of fp32, whose products take
// ten times as long; three videos of up to 777 frames, five heads of 45 x 67, fp32, both ways: 216 us, with eight chunks at least 597.  (Videos count at their full length,
// and tiles of columns do not count: ragged batches leave units without work.)
Stretches stretches_of(const rrm_decay_desc& d, float* states) {
    Stretches st{1, 0x7fffff00, states};
    if (by_steps(d)) {
        st.count = 0;
        return st;
    }
    const int64_t groups = (int64_t)d.n * d.h;
    const int chunks = (d.t + 63) / 64, most = chunks / (d.elem == RRM_F32 ? 3 : 8);
    int64_t count = 2 * OP_CUS / groups;
    if (count > most) count = most;
    if (count < 2) return st;
    const int per = (int)((chunks + count - 1) / count);
    st.frames = per * 64;
    st.count = (chunks + per - 1) / per;
    return st;
}

template <typename T, bool STATES>
void launch_chunk(const Walk& w, const Stretches& st, hipStream_t s) {
    constexpr int C = 64;
    with_chunk<T>(w, [&](auto dk, auto dv) {
        constexpr int DK = decltype(dk)::value, DV = decltype(dv)::value;
        using K = Chunk<T, DK, DV, C>;
        const unsigned units = (unsigned)((int64_t)w.n * w.h * st.count);
        const int64_t slices = (w.dv + DV - 1) / DV;
        in_parts(((int64_t)units + 7) / 8 * 8 * slices, [&](unsigned first, unsigned count) {
            if (w.dk % K::EPC == 0 && w.dv % K::EPC == 0)
                hipLaunchKernelGGL((walk_kernel<T, DK, DV, C, STATES, true>), dim3(count), dim3(K::THREADS), 0, s, w, st, units, first);
            else
                hipLaunchKernelGGL((walk_kernel<T, DK, DV, C, STATES, false>), dim3(count), dim3(K::THREADS), 0, s, w, st, units, first);
        });
    });
}
template <typename T, bool STATES>
hipError_t launch_chunks(const Walk& all, const Stretches& st, hipStream_t s) {
    const int half = all.dk <= most_keys(sizeof(T) == 4 ? RRM_F32 : RRM_BF16) ? all.dk : ((all.dk + 1) / 2 + 7) / 8 * 8;  // (whole pieces)
    for (int k = 0; k < all.dk; k += half) {
        Walk w = all;
        w.first_key = k, w.keys = all.dk, w.dk = all.dk - k < half ? all.dk - k : half;
        w.q.p = (const T*)all.q.p + k, w.k.p = (const T*)all.k.p + k;
        w.adds = k > 0, w.leaves = k + half < all.dk;
        launch_chunk<T, STATES>(w, st, s);
    }
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
    if (st.count == 0) return elem == RRM_F32 ? launch_steps<float>(w, s) : launch_steps<__bf16>(w, s);
    return elem == RRM_F32 ? launch_chunks<float, false>(w, st, s) : launch_chunks<__bf16, false>(w, st, s);
}
// What a walk's first half of the keys leaves
size_t part_bytes(const rrm_decay_desc& d, int keys, int cols) {
    return by_steps(d) || keys <= most_keys(d.elem) ? 0 : round256((size_t)d.n * d.t * d.h * cols * 4);
}
size_t states_bytes(const rrm_decay_desc& d) {
    const Stretches st = stretches_of(d, nullptr);
    return st.count < 2 ? 0 : round256((size_t)(st.count - 1) * d.n * d.h * d.dk * d.dv * 4);
}

}  // namespace

// forward: [states of the stretches][part]; backward: [those of S][those of D][part]
size_t decay_scratch(const rrm_decay_desc& d, bool backward) {
    const size_t forward = part_bytes(d, d.dk, d.dv), back = part_bytes(d, d.dv, d.dk);
    return states_bytes(d) * (backward ? 2 : 1) + (backward && back > forward ? back : forward);
}

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
    w.part = (float*)((unsigned char*)ws + states_bytes(d));
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
    w.part = (float*)((unsigned char*)ws + 2 * states_bytes(d));
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
