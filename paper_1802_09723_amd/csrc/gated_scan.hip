// Gated linear recurrence over the frames of videos, and its backward pass.
//
//      a = sigmoid(f)      h_t = a_t h_{t-1} + (1 - a_t) x_t      g_t = dy_t + a_{t+1} g_{t+1}
//
// A frame is an affine map of the state, h -> A h + B, and maps of neighbouring frames join to one: (A2 A1, A2 B1 + B2).  A workgroup has a
// tile of features of one video and goes through its frames in blocks: a thread holds SPAN frames of its features in registers and joins them, the
// rows' maps meet in LDS, where one thread a feature carries the state through them, and each thread makes its frames from the state that it is
// handed.  So x and f are read once.  The gradient runs the other way by the same maps (its A is the same product), and h is made again from
// the state kept every RRM_SCAN_MARK_FRAMES frames, which is less to write and read than h.
//
// States, maps and gradients of states are held in 32 bits; only results are rounded.  What bounds it is memory: x, f and y (backward x, f,
// dy, dx and df) once, with a handful of operations an element.  Measured: 64 x 256 x 4096 bf16, a workgroup a chain, 88 us, 4.6 TB/s;
// 1 x 65536 x 512 fp32, many workgroups a chain, 93 us, 4.3 TB/s (a copy: 5.1); backward, 4 x 4096 x 4096 bf16, 170 us, 4.0 TB/s.
#include <algorithm>

#include "op_common.h"

namespace rrm {

namespace {

constexpr int GS_THREADS = 256;
constexpr int GS_BLOCK = 128;  // frames of a block
constexpr int LONG_BLOCK = 256;  // of long fp32 videos: see forward_block
constexpr int MARK = RRM_SCAN_MARK_FRAMES;
static_assert(GS_BLOCK % MARK == 0, "blocks begin at marks");

__device__ __forceinline__ int video_frames(const int32_t* lengths, int i, int t) {
    if (!lengths) return t;
    const int e = lengths[i];
    return e < 0 ? 0 : e > t ? t : e;
}
// LDS accesses done, then the barrier; loads from memory stay on their way
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Shape of a tile: VEC features a thread, eight threads of a frame (runs of 128 bytes), 32 rows of FRAMES / 32 frames
template <int VEC, int FRAMES = GS_BLOCK>
struct Tile {
    static constexpr int LANES = 8, ROWS = GS_THREADS / LANES, SPAN = FRAMES / ROWS, WIDTH = LANES * VEC;
};

// The gates of a block are made twice, from what memory holds, rather than kept over the wait: their values would take twice to four
// times the registers.  (Says to the compiler that the words may have changed, else it keeps them.)
template <typename T, int VEC>
__device__ __forceinline__ void made_again(Held<T, VEC>& v) {
#pragma unroll
    for (int i = 0; i < Held<T, VEC>::WORDS; ++i) asm volatile("" : "+v"(v.w[i]));
}

// (These values are wanted here: not later, from all that they are made of.)
template <int VEC>
__device__ __forceinline__ void made_now(float (&v)[VEC]) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) asm volatile("" : "+v"(v[i]));
}

// A chain is a tile of features of one video, its blocks one after the other.  Where there are chains enough a workgroup has one and loops over its
// blocks; else a chain's blocks go to many workgroups, x and f are still read once, and the state is handed on in memory:
//
//   - a workgroup takes the chain's next block (a counter, so in the order of time: who holds a block knows that all blocks before it are done, or
//     held by workgroups that run and wait for still earlier ones only; every wait below ends),
//   - writes the block's map (A, B) to the block's slot, one 64-bit word a feature whose top bit says that it is there (A, a product of gates, has
//     no use for its sign; the words are zeros before),
//   - reads the maps of the blocks before it in its group of GROUP and joins them, waits for the state before the group, and has its own state,
//   - and, the last of its group, writes the state before the next one.
//
// Everything is joined in one order, whoever comes first.  A word needs no fence: it is all that is handed over.  A wait is bounded all the same (some
// seconds): it would end in not-a-numbers.  No block is taken ahead, while its predecessor waits: its map would be missed by the others
// (1 x 65536 x 512 fp32 816 us).  Groups of 8, 16 and 64 blocks: 1 x 27594 x 80 fp32 forward and backward 74, 55 and 43 us, 45 with 32;
// 4 x 8192 x 1000 bf16 of unequal lengths 172, 172 and 192, 174 with 32.
constexpr int GROUP = 32;
constexpr int POLLS = 1 << 22;
typedef unsigned long long word_t;
constexpr word_t NEVER = 0xffc000007fc00000ull;  // a map and a state of not-a-numbers
struct Chain {
    int tiles, blocks, groups;  // of features; of frames; of blocks
    int per;                    // workgroups of a chain
    word_t *maps, *states;      // [chain][blocks][WIDTH], [chain][groups][WIDTH]
    unsigned int* counters;     // [chain][16], a cache line each
};

__device__ __forceinline__ word_t word_at(const word_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void put_word(word_t* p, unsigned int high, float low) {
    __hip_atomic_store(p, (word_t)(high | 0x80000000u) << 32 | __float_as_uint(low), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ bool written(word_t w) { return (int64_t)w < 0; }
__device__ __forceinline__ float low_of(word_t w) { return __uint_as_float((unsigned int)w); }
__device__ __forceinline__ float high_of(word_t w) { return __uint_as_float((unsigned int)(w >> 32) & 0x7fffffffu); }

// The state before block k of a chain, in threads j < WIDTH, from the maps of the blocks and the states of the groups before it; all threads
// of the workgroup call.  sa, sb: LDS of a word a thread.
template <int WIDTH>
__device__ __forceinline__ float state_before(const word_t* maps, const word_t* states, int k, float start, float* sa, float* sb) {
    constexpr int SEGS = GS_THREADS / WIDTH, EACH = (GROUP + SEGS - 1) / SEGS;
    const int j = (int)threadIdx.x % WIDTH, seg = (int)threadIdx.x / WIDTH, first = k / GROUP * GROUP, count = k - first;
    if (count > 0) {
        float A = 1.0f, B = 0.0f;
        if (seg * EACH < count) {
            word_t w[EACH];
#pragma unroll 1
            for (int polls = 0;; ++polls) {
                bool all = true;
#pragma unroll
                for (int i = 0; i < EACH; ++i) w[i] = word_at(maps + (int64_t)min(first + seg * EACH + i, k - 1) * WIDTH + j);
#pragma unroll
                for (int i = 0; i < EACH; ++i) all = all && written(w[i]);
                if (all) break;
                if (polls == POLLS) {
                    w[0] = NEVER;
                    break;
                }
                __builtin_amdgcn_s_sleep(1);
            }
#pragma unroll
            for (int i = 0; i < EACH; ++i)
                if (seg * EACH + i < count) {
                    A *= high_of(w[i]);
                    B = high_of(w[i]) * B + low_of(w[i]);
                }
        }
        sa[threadIdx.x] = A;
        sb[threadIdx.x] = B;
    }
    lds_barrier();
    float state = start;
    if (seg == 0) {
        float A = 1.0f, B = 0.0f;
        if (count > 0) {
#pragma unroll
            for (int q = 0; q < SEGS; ++q) {
                A *= sa[q * WIDTH + j];
                B = sa[q * WIDTH + j] * B + sb[q * WIDTH + j];
            }
        }
        if (first > 0) {
            word_t w;
#pragma unroll 1
            for (int polls = 0; !written(w = word_at(states + (int64_t)(first / GROUP - 1) * WIDTH + j)); ++polls) {
                if (polls == POLLS) {
                    w = NEVER;
                    break;
                }
                __builtin_amdgcn_s_sleep(1);
            }
            state = low_of(w);
        }
        state = A * state + B;
    }
    return state;
}

// the next block of a chain, the same for all threads of the workgroup
__device__ __forceinline__ int next_block(unsigned int* counter, int* shared) {
    lds_barrier();  // (the workgroup is done with what it has in LDS)
    if (threadIdx.x == 0) *shared = (int)atomicAdd(counter, 1u);
    lds_barrier();
    return *shared;
}

// A thread's features among those of an LDS row, from `at` on (those before `first` are another thread's); whole vectors in 16-byte pieces
template <int VEC>
__device__ __forceinline__ void put(float* row, int at, int first, const float (&v)[VEC]) {
    if (VEC >= 4 && first == 0) {
#pragma unroll
        for (int i = 0; i < VEC; i += 4) *reinterpret_cast<float4*>(row + at + i) = make_float4(v[i], v[(i + 1) % VEC], v[(i + 2) % VEC], v[(i + 3) % VEC]);
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (i >= first) row[at + i] = v[i];
    }
}
template <int VEC>
__device__ __forceinline__ void take(const float* row, int at, int first, float (&v)[VEC]) {
    if (VEC >= 4 && first == 0) {
#pragma unroll
        for (int i = 0; i < VEC; i += 4) {
            const float4 q = *reinterpret_cast<const float4*>(row + at + i);
            v[i] = q.x, v[(i + 1) % VEC] = q.y, v[(i + 2) % VEC] = q.z, v[(i + 3) % VEC] = q.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = row[at + i < 0 ? 0 : at + i];  // (before the tile: whatever stands there, never stored)
    }
}

// A workgroup a chain.
template <typename T, int VEC>
__global__ __launch_bounds__(GS_THREADS) void scan_kernel(rrm_scan_desc d, int tiles, unsigned from, const T* __restrict__ x, const T* __restrict__ f, const float* h0,
                                                          const int32_t* __restrict__ lengths, T* __restrict__ y,
                                                          float* h_last, float* __restrict__ marks) {
    using Z = Tile<VEC>;
    constexpr int S = Z::SPAN;
    __shared__ __attribute__((aligned(16))) float sa[2][Z::ROWS * Z::WIDTH];
    __shared__ __attribute__((aligned(16))) float sb[2][Z::ROWS * Z::WIDTH];
    const unsigned id = from + blockIdx.x;
    const int video = (int)(id / (unsigned)tiles);
    const int c0 = (int)(id % (unsigned)tiles) * Z::WIDTH, width = min(d.c - c0, Z::WIDTH), row = (int)threadIdx.x / Z::LANES, j = (int)threadIdx.x;
    const Span<VEC> me((int)threadIdx.x % Z::LANES, c0, width);
    const int end = video_frames(lengths, video, d.t);
    const T* xp = x + video * d.x_video + me.at;
    const T* fp = f + video * d.f_video + me.at;
    T* yp = y + video * d.y_video + me.at;
    const int nm = (d.t + MARK - 1) / MARK;
    Held<T, VEC> rx[S], rf[S];
    auto fetch = [&](int tb) __attribute__((always_inline)) {  // (frames behind the end: the last one again, not under a condition)
#pragma unroll
        for (int k = 0; k < S; ++k) {
            const int t = min(tb + row * S + k, end - 1);
            rx[k].load(xp + t * d.x_frame);
            rf[k].load(fp + t * d.f_frame);
        }
    };
    if (end > 0) fetch(0);
    float carry = 0.0f;  // thread j: the state of feature c0 + j before the block
    if (j < width && h0) carry = h0[(int64_t)video * d.c + c0 + j];
    int buf = 0;
    int tb = 0;
    for (; tb < end; tb += GS_BLOCK, buf ^= 1) {
        float a[S][VEC], b[S][VEC], A[VEC], B[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) A[i] = 1.0f, B[i] = 0.0f;
#pragma unroll
        for (int k = 0; k < S; ++k) {
            const bool in = tb + row * S + k < end;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                float o;
                gate_pair(rf[k].get(i), a[k][i], o);
                b[k][i] = in ? o * rx[k].get(i) : 0.0f;
                a[k][i] = in ? a[k][i] : 1.0f;
                A[i] *= a[k][i];
                B[i] = a[k][i] * B[i] + b[k][i];
            }
        }
        if (tb + GS_BLOCK < end) fetch(tb + GS_BLOCK);
        float *ra = sa[buf] + row * Z::WIDTH, *rb = sb[buf] + row * Z::WIDTH;
        put<VEC>(ra, me.at - c0, me.first, A);
        put<VEC>(rb, me.at - c0, me.first, B);
        lds_barrier();
        if (j < width) {
#pragma unroll 8
            for (int r = 0; r < Z::ROWS; ++r) {
                const float ma = sa[buf][r * Z::WIDTH + j], mb = sb[buf][r * Z::WIDTH + j];
                sa[buf][r * Z::WIDTH + j] = carry;  // the state that row r is handed
                carry = ma * carry + mb;
            }
        }
        lds_barrier();
        float h[VEC];
        take<VEC>(ra, me.at - c0, me.first, h);
        if (me.first == VEC) continue;
        if (marks && (row * S) % MARK == 0 && tb + row * S < d.t)
            store_some<VEC>(marks + ((int64_t)video * nm + (tb + row * S) / MARK) * d.c + me.at, h, me.keep);
#pragma unroll
        for (int k = 0; k < S; ++k) {
            const int t = tb + row * S + k;
            float o[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                h[i] = a[k][i] * h[i] + b[k][i];
                o[i] = t < end ? h[i] : 0.0f;
            }
            if (t < d.t) store_some<VEC>(yp + t * d.y_frame, o, me.keep);
        }
    }
    // behind the video's end: zeros, and the last state for the marks
    if (tb < d.t && me.first < VEC) {
        float zero[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) zero[i] = 0.0f;
        for (int t = tb + row; t < d.t; t += Z::ROWS) store_some<VEC>(yp + t * d.y_frame, zero, me.keep);
    }
    if (j < width) {
        if (marks)
            for (int t = tb; t < d.t; t += MARK) marks[((int64_t)video * nm + t / MARK) * d.c + c0 + j] = carry;
        if (h_last) h_last[(int64_t)video * d.c + c0 + j] = carry;
    }
}

// Many workgroups a chain: four a compute unit hide each other's waits (128 registers; two with long blocks).
template <typename T, int VEC, int FRAMES>
__global__ __launch_bounds__(GS_THREADS, FRAMES == GS_BLOCK ? 4 : 2) void chained_scan_kernel(rrm_scan_desc d, Chain ch, const T* __restrict__ x, const T* __restrict__ f,
                                                                     const float* h0, const int32_t* __restrict__ lengths, T* __restrict__ y,
                                                                     float* h_last, float* __restrict__ marks) {
    using Z = Tile<VEC, FRAMES>;
    constexpr int S = Z::SPAN, W = Z::WIDTH;
    __shared__ __attribute__((aligned(16))) float sa[Z::ROWS * W];
    __shared__ __attribute__((aligned(16))) float sb[Z::ROWS * W];
    const int chain = (int)(blockIdx.x % (unsigned)(d.n * ch.tiles)), video = chain / ch.tiles;
    const int c0 = chain % ch.tiles * W, width = min(d.c - c0, W), j = (int)threadIdx.x;
    int row = (int)threadIdx.x / Z::LANES;
    const Span<VEC> me((int)threadIdx.x % Z::LANES, c0, width);
    const int end = video_frames(lengths, video, d.t);
    const T* xp = x + video * d.x_video + me.at;
    const T* fp = f + video * d.f_video + me.at;
    T* yp = y + video * d.y_video + me.at;
    const int nm = (d.t - 1) / MARK + 1;
    float* mp = marks ? marks + (int64_t)video * nm * d.c : nullptr;
    Held<T, VEC> rx[S], rf[S];
    auto fetch = [&](int tb) __attribute__((always_inline)) {  // (frames behind the end: the last one again, not under a condition)
#pragma unroll
        for (int k = 0; k < S; ++k) {
            const int t = max(min(tb + row * S + k, end - 1), 0);
            rx[k].load(xp + t * d.x_frame);
            rf[k].load(fp + t * d.f_frame);
        }
    };
    Held<T, VEC> cx[S], cf[S];  // of the block in hand
    float A[VEC], B[VEC];
    auto rows = [&](int tb) __attribute__((always_inline)) {  // the frames' maps, and the row's
#pragma unroll
        for (int i = 0; i < VEC; ++i) A[i] = 1.0f, B[i] = 0.0f;
#pragma unroll
        for (int k = 0; k < S; ++k) {
            const bool in = tb + row * S + k < end;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                float a, o;
                gate_pair(rf[k].get(i), a, o);
                A[i] = in ? A[i] * a : A[i];
                B[i] = in ? a * B[i] + o * rx[k].get(i) : B[i];
            }
            cx[k] = rx[k], cf[k] = rf[k];
            made_now(A);
            made_now(B);
        }
    };
    auto rows_to_lds = [&]() __attribute__((always_inline)) {
        put<VEC>(sa + row * W, me.at - c0, me.first, A);
        put<VEC>(sb + row * W, me.at - c0, me.first, B);
    };
    auto frames = [&](int tb, float (&h)[VEC]) __attribute__((always_inline)) {  // h: the state before the row
        if (me.first == VEC) return;
        if (mp && (row * S) % MARK == 0 && tb + row * S < d.t) store_some<VEC>(mp + (int64_t)((tb + row * S) / MARK) * d.c + me.at, h, me.keep);
#pragma unroll
        for (int k = 0; k < S; ++k) {
            const int t = tb + row * S + k;
            float o[VEC];
            made_again(cx[k]);
            made_again(cf[k]);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                float a, p;
                gate_pair(cf[k].get(i), a, p);
                h[i] = a * h[i] + p * cx[k].get(i);
                o[i] = t < end ? h[i] : 0.0f;
            }
            if (t < d.t) store_some<VEC>(yp + t * d.y_frame, o, me.keep);
        }
    };
    auto zeros = [&](int tb, int te) __attribute__((always_inline)) {
        if (me.first == VEC) return;
        float zero[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) zero[i] = 0.0f;
        for (int t = tb + row; t < te; t += Z::ROWS) store_some<VEC>(yp + t * d.y_frame, zero, me.keep);
    };
    auto leave = [&](int tb, float state) __attribute__((always_inline)) {  // the state behind the video's last frame; tb: the block behind it
        if (j >= width) return;
        if (mp)
            for (int t = tb; t < d.t; t += MARK) mp[(int64_t)(t / MARK) * d.c + c0 + j] = state;
        if (h_last) h_last[(int64_t)video * d.c + c0 + j] = state;
    };
    const float start = j < width && h0 ? h0[(int64_t)video * d.c + c0 + j] : 0.0f;
    __shared__ float sg[2][GS_THREADS];
    __shared__ __attribute__((aligned(16))) float sh[W];
    __shared__ int sk;
    word_t* maps = ch.maps + (int64_t)chain * ch.blocks * W;
    word_t* states = ch.states + (int64_t)chain * ch.groups * W;
    const int last = end > 0 ? (end - 1) / FRAMES : 0;
    for (int k; (k = next_block(ch.counters + chain * 16, &sk)) < ch.blocks;) {
        asm volatile("" : "+v"(row));  // (what hangs on it is made in each block, not kept in registers over all)
        const int tb = k * FRAMES;
        if (k > last) {
            zeros(tb, min(tb + FRAMES, d.t));
            continue;
        }
        fetch(tb);
        rows(tb);
        rows_to_lds();
        lds_barrier();
        float am = 1.0f, bm = 0.0f;
        if (j < width) {  // the rows' maps become those of what is before them
#pragma unroll 8
            for (int r = 0; r < Z::ROWS; ++r) {
                const float ma = sa[r * W + j], mb = sb[r * W + j];
                sa[r * W + j] = am;
                sb[r * W + j] = bm;
                am *= ma;
                bm = ma * bm + mb;
            }
        }
        if (j < W && k < last) put_word(maps + (int64_t)k * W + j, __float_as_uint(am), bm);
        const float state = state_before<W>(maps, states, k, start, sg[0], sg[1]);
        if (j < W) {
            const float after = am * state + bm;
            if (k < last && k % GROUP == GROUP - 1) put_word(states + (int64_t)(k / GROUP) * W + j, 0u, after);
            sh[j] = state;
            if (k == last) leave(tb + FRAMES, after);
        }
        lds_barrier();
        float h[VEC], pa[VEC], pb[VEC];
        take<VEC>(sa + row * W, me.at - c0, me.first, pa);
        take<VEC>(sb + row * W, me.at - c0, me.first, pb);
        take<VEC>(sh, me.at - c0, me.first, h);
#pragma unroll
        for (int i = 0; i < VEC; ++i) h[i] = pa[i] * h[i] + pb[i];
        frames(tb, h);
    }
}

constexpr int BACK_BLOCK = 64;  // frames of a block where a workgroup has a chain: it holds four values a frame

template <typename T, int VEC>
__global__ __launch_bounds__(GS_THREADS, 3) void scan_back_kernel(rrm_scan_desc d, int tiles, unsigned from, const T* __restrict__ x, const T* __restrict__ f,
                                                               const float* __restrict__ marks, const int32_t* __restrict__ lengths,
                                                               const T* __restrict__ dy, const float* dh_last,
                                                               T* __restrict__ dx, T* __restrict__ df, float* dh0) {
    using Z = Tile<VEC, BACK_BLOCK>;
    constexpr int S = Z::SPAN, MARKS = BACK_BLOCK / MARK, MROWS = Z::ROWS / MARKS;
    __shared__ __attribute__((aligned(16))) float sa[Z::ROWS * Z::WIDTH];
    __shared__ __attribute__((aligned(16))) float sb[Z::ROWS * Z::WIDTH];
    __shared__ __attribute__((aligned(16))) float sg[Z::ROWS * Z::WIDTH];
    const unsigned id = from + blockIdx.x;
    const int video = (int)(id / (unsigned)tiles);
    const int c0 = (int)(id % (unsigned)tiles) * Z::WIDTH, width = min(d.c - c0, Z::WIDTH), row = (int)threadIdx.x / Z::LANES, j = (int)threadIdx.x;
    const Span<VEC> me((int)threadIdx.x % Z::LANES, c0, width);
    const int end = video_frames(lengths, video, d.t);
    const T* xp = x + video * d.x_video + me.at;
    const T* fp = f + video * d.f_video + me.at;
    const T* yp = dy + video * d.y_video + me.at;
    T* dxp = dx + video * d.dx_video + me.at;
    T* dfp = df + video * d.df_video + me.at;
    const int nm = (d.t + MARK - 1) / MARK;
    const int blocks = (end + BACK_BLOCK - 1) / BACK_BLOCK;
    if (me.first < VEC) {  // behind the video's end
        float zero[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) zero[i] = 0.0f;
        for (int t = blocks * BACK_BLOCK + row; t < d.t; t += Z::ROWS) {
            store_some<VEC>(dxp + t * d.dx_frame, zero, me.keep);
            store_some<VEC>(dfp + t * d.df_frame, zero, me.keep);
        }
    }
    Held<T, VEC> rx[S], rf[S], ry[S];
    auto fetch = [&](int tb) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < S; ++k) {
            const int t = min(tb + row * S + k, end - 1);
            rx[k].load(xp + t * d.x_frame);
            rf[k].load(fp + t * d.f_frame);
            ry[k].load(yp + t * d.y_frame);
        }
    };
    if (blocks) fetch((blocks - 1) * BACK_BLOCK);
    float carry = 0.0f;  // thread j: the gradient of the state behind the block, of feature c0 + j
    if (j < width && dh_last) carry = dh_last[(int64_t)video * d.c + c0 + j];
    for (int blk = blocks - 1; blk >= 0; --blk) {
        const int tb = blk * BACK_BLOCK;
        float a[S][VEC], o[S][VEC], v[S][VEC], g[S][VEC], A[VEC], B[VEC], G[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) A[i] = 1.0f, B[i] = 0.0f, G[i] = 0.0f;
#pragma unroll
        for (int k = 0; k < S; ++k) {
            const bool in = tb + row * S + k < end;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                gate_pair(rf[k].get(i), a[k][i], o[k][i]);
                a[k][i] = in ? a[k][i] : 1.0f;
                o[k][i] = in ? o[k][i] : 0.0f;
                v[k][i] = in ? rx[k].get(i) : 0.0f;
                g[k][i] = in ? ry[k].get(i) : 0.0f;
                A[i] *= a[k][i];
                G[i] += g[k][i] * A[i];   // (dy of a frame reaches the state before the row through the gates up to its own)
                B[i] = a[k][i] * B[i] + o[k][i] * v[k][i];
            }
        }
        if (blk > 0) fetch(tb - BACK_BLOCK);
        lds_barrier();  // (the rows have been handed their states of the block before)
        put<VEC>(sa + row * Z::WIDTH, me.at - c0, me.first, A);
        put<VEC>(sb + row * Z::WIDTH, me.at - c0, me.first, B);
        put<VEC>(sg + row * Z::WIDTH, me.at - c0, me.first, G);
        lds_barrier();
        // gradients by the first threads, states by those behind them, each from its mark
        if (j < width) {
#pragma unroll 8
            for (int r = Z::ROWS - 1; r >= 0; --r) {
                const float ma = sa[r * Z::WIDTH + j], mg = sg[r * Z::WIDTH + j];
                sg[r * Z::WIDTH + j] = carry;
                carry = ma * carry + mg;
            }
        }
        for (int k = j - Z::WIDTH; k >= 0 && k < MARKS * Z::WIDTH; k += GS_THREADS - Z::WIDTH) {
            const int m = k / Z::WIDTH, c = k % Z::WIDTH;
            if (c < width && tb + m * MARK < end) {
                float h = marks[((int64_t)video * nm + tb / MARK + m) * d.c + c0 + c];
#pragma unroll 8
                for (int r = m * MROWS; r < (m + 1) * MROWS; ++r) {
                    const float ma = sa[r * Z::WIDTH + c], mb = sb[r * Z::WIDTH + c];
                    sb[r * Z::WIDTH + c] = h;
                    h = ma * h + mb;
                }
            }
        }
        lds_barrier();
        if (me.first == VEC) continue;
        float h[VEC], gr[VEC];
        take<VEC>(sb + row * Z::WIDTH, me.at - c0, me.first, h);
        take<VEC>(sg + row * Z::WIDTH, me.at - c0, me.first, gr);
        // g to the end of the row first, then states from its start
#pragma unroll
        for (int k = S - 1; k >= 0; --k)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                g[k][i] += gr[i];
                gr[i] = a[k][i] * g[k][i];
            }
#pragma unroll
        for (int k = 0; k < S; ++k) {
            const int t = tb + row * S + k;
            float ox[VEC], of[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                ox[i] = t < end ? o[k][i] * g[k][i] : 0.0f;
                of[i] = t < end ? g[k][i] * (h[i] - v[k][i]) * (a[k][i] * o[k][i]) : 0.0f;
                h[i] = a[k][i] * h[i] + o[k][i] * v[k][i];
            }
            if (t < d.t) {
                store_some<VEC>(dxp + t * d.dx_frame, ox, me.keep);
                store_some<VEC>(dfp + t * d.df_frame, of, me.keep);
            }
        }
    }
    if (dh0 && j < width) dh0[(int64_t)video * d.c + c0 + j] = carry;
}

template <typename T, int VEC>
__global__ __launch_bounds__(GS_THREADS, 3) void chained_scan_back_kernel(rrm_scan_desc d, Chain ch, const T* __restrict__ x, const T* __restrict__ f,
                                                                          const float* __restrict__ marks, const int32_t* __restrict__ lengths,
                                                                          const T* __restrict__ dy, const float* dh_last, T* __restrict__ dx,
                                                                          T* __restrict__ df, float* dh0) {
    using Z = Tile<VEC, GS_BLOCK>;
    constexpr int S = Z::SPAN, W = Z::WIDTH;
    static_assert(GS_BLOCK % MARK == 0 && (GS_BLOCK / MARK + 1) * 8 * VEC <= GS_THREADS, "a thread for each state kept in a block");
    __shared__ __attribute__((aligned(16))) float sa[Z::ROWS * W];
    __shared__ __attribute__((aligned(16))) float sb[Z::ROWS * W];
    __shared__ __attribute__((aligned(16))) float sg[Z::ROWS * W];
    const int chain = (int)(blockIdx.x % (unsigned)(d.n * ch.tiles)), video = chain / ch.tiles;
    const int c0 = chain % ch.tiles * W, width = min(d.c - c0, W), j = (int)threadIdx.x;
    int row = (int)threadIdx.x / Z::LANES;
    const Span<VEC> me((int)threadIdx.x % Z::LANES, c0, width);
    const int end = video_frames(lengths, video, d.t);
    const T* xp = x + video * d.x_video + me.at;
    const T* fp = f + video * d.f_video + me.at;
    const T* yp = dy + video * d.y_video + me.at;
    T* dxp = dx + video * d.dx_video + me.at;
    T* dfp = df + video * d.df_video + me.at;
    const float* mp = marks + (int64_t)video * ((d.t - 1) / MARK + 1) * d.c;
    auto zeros = [&](int tb, int te) __attribute__((always_inline)) {
        if (me.first == VEC) return;
        float zero[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) zero[i] = 0.0f;
        for (int t = tb + row; t < te; t += Z::ROWS) {
            store_some<VEC>(dxp + t * d.dx_frame, zero, me.keep);
            store_some<VEC>(dfp + t * d.df_frame, zero, me.keep);
        }
    };
    Held<T, VEC> rx[S], rf[S], ry[S];
    auto fetch = [&](int tb) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < S; ++k) {
            const int t = max(min(tb + row * S + k, end - 1), 0);
            rx[k].load(xp + t * d.x_frame);
            rf[k].load(fp + t * d.f_frame);
            ry[k].load(yp + t * d.y_frame);
        }
    };
    Held<T, VEC> cx[S], cf[S], cy[S];  // of the block in hand
    float A[VEC], B[VEC], G[VEC];
    auto rows = [&](int tb) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) A[i] = 1.0f, B[i] = 0.0f, G[i] = 0.0f;
#pragma unroll
        for (int k = 0; k < S; ++k) {
            const bool in = tb + row * S + k < end;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                float a, o;
                gate_pair(rf[k].get(i), a, o);
                A[i] = in ? A[i] * a : A[i];
                G[i] = in ? G[i] + ry[k].get(i) * A[i] : G[i];  // (dy of a frame reaches the state before the row through the gates up to its own)
                B[i] = in ? a * B[i] + o * rx[k].get(i) : B[i];
            }
            cx[k] = rx[k], cf[k] = rf[k], cy[k] = ry[k];
            made_now(A);
            made_now(B);
            made_now(G);
        }
    };
    auto rows_to_lds = [&]() __attribute__((always_inline)) {
        put<VEC>(sa + row * W, me.at - c0, me.first, A);
        put<VEC>(sb + row * W, me.at - c0, me.first, B);
        put<VEC>(sg + row * W, me.at - c0, me.first, G);
    };
    // a block's states from its marks, by the threads behind the first W
    auto states_of_rows = [&](int tb) __attribute__((always_inline)) {
        constexpr int EACH = Z::ROWS * MARK / GS_BLOCK;  // rows of a mark
        const int m = j / W - 1, c = j % W;
        if (m >= 0 && m < GS_BLOCK / MARK && c < width && tb + m * MARK < end) {
            float h = mp[(int64_t)(tb / MARK + m) * d.c + c0 + c];
#pragma unroll 8
            for (int r = m * EACH; r < (m + 1) * EACH; ++r) {
                const float ma = sa[r * W + c], mb = sb[r * W + c];
                sb[r * W + c] = h;
                h = ma * h + mb;
            }
        }
    };
    auto frames = [&](int tb, float (&h)[VEC], float (&gr)[VEC]) __attribute__((always_inline)) {  // states before, gradients behind the row
        if (me.first == VEC) return;
        // g to the end of the row first, then states from its start
        float g[S][VEC];
#pragma unroll
        for (int k = S - 1; k >= 0; --k) {
            const bool in = tb + row * S + k < end;
            made_again(cx[k]);
            made_again(cf[k]);
            made_again(cy[k]);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                float a, o;
                gate_pair(cf[k].get(i), a, o);
                g[k][i] = in ? cy[k].get(i) + gr[i] : 0.0f;
                gr[i] = in ? a * g[k][i] : gr[i];
            }
            made_now(gr);
            made_now(g[k]);
        }
#pragma unroll
        for (int k = 0; k < S; ++k) {
            const int t = tb + row * S + k;
            float ox[VEC], of[VEC];
            made_again(cf[k]);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float v = cx[k].get(i);
                float a, o;
                gate_pair(cf[k].get(i), a, o);
                ox[i] = t < end ? o * g[k][i] : 0.0f;
                of[i] = t < end ? g[k][i] * (h[i] - v) * (a * o) : 0.0f;
                h[i] = a * h[i] + o * v;
            }
            made_now(h);
            if (t < d.t) {
                store_some<VEC>(dxp + t * d.dx_frame, ox, me.keep);
                store_some<VEC>(dfp + t * d.df_frame, of, me.keep);
            }
        }
    };
    const float start = j < width && dh_last ? dh_last[(int64_t)video * d.c + c0 + j] : 0.0f;
    float h[VEC], gr[VEC];
    __shared__ float ss[2][GS_THREADS];
    __shared__ __attribute__((aligned(16))) float sp[Z::ROWS * W];
    __shared__ __attribute__((aligned(16))) float sc[W];
    __shared__ int sk;
    word_t* maps = ch.maps + (int64_t)chain * ch.blocks * W;
    word_t* states = ch.states + (int64_t)chain * ch.groups * W;
    const int last = end > 0 ? (end - 1) / GS_BLOCK : 0;
    for (int k; (k = next_block(ch.counters + chain * 16, &sk)) < ch.blocks;) {
        asm volatile("" : "+v"(row));  // (what hangs on it is made in each block, not kept in registers over all)
        if (k > last) {  // blocks behind the end come after those with frames: nobody waits for them
            const int tb = k * GS_BLOCK;
            zeros(tb, min(tb + GS_BLOCK, d.t));
            continue;
        }
        const int tb = (last - k) * GS_BLOCK;  // (the chain's k-th block is the k-th from the end)
        fetch(tb);
        rows(tb);
        rows_to_lds();
        lds_barrier();
        float am = 1.0f, gm = 0.0f;
        if (j < width) {
#pragma unroll 8
            for (int r = Z::ROWS - 1; r >= 0; --r) {
                const float ma = sa[r * W + j], mg = sg[r * W + j];
                sg[r * W + j] = gm;
                sp[r * W + j] = am;
                gm = ma * gm + mg;
                am *= ma;
            }
        }
        if (j < W && k < last) put_word(maps + (int64_t)k * W + j, __float_as_uint(am), gm);
        states_of_rows(tb);
        const float carry = state_before<W>(maps, states, k, start, ss[0], ss[1]);
        if (j < W) {
            const float after = am * carry + gm;
            if (k < last && k % GROUP == GROUP - 1) put_word(states + (int64_t)(k / GROUP) * W + j, 0u, after);
            sc[j] = carry;
            if (dh0 && k == last && j < width) dh0[(int64_t)video * d.c + c0 + j] = after;
        }
        lds_barrier();
        float qa[VEC], qg[VEC];
        take<VEC>(sb + row * W, me.at - c0, me.first, h);
        take<VEC>(sp + row * W, me.at - c0, me.first, qa);
        take<VEC>(sg + row * W, me.at - c0, me.first, qg);
        take<VEC>(sc, me.at - c0, me.first, gr);
#pragma unroll
        for (int i = 0; i < VEC; ++i) gr[i] = qa[i] * gr[i] + qg[i];
        frames(tb, h, gr);
    }
}

// Few frames: a thread a vector of features, frame by frame.  A frame of 4096 features takes 3.5 us, most of it the launch.
template <typename T, int VEC>
__global__ __launch_bounds__(64) void short_scan_kernel(rrm_scan_desc d, unsigned from, const T* __restrict__ x, const T* __restrict__ f, const float* h0,
                                                        const int32_t* __restrict__ lengths, T* __restrict__ y, float* h_last,
                                                        float* __restrict__ marks) {
    const unsigned id = from + blockIdx.x, per = ((unsigned)d.c + 64 * VEC - 1) / (64 * VEC);
    const int video = (int)(id / per), c0 = (int)(id % per) * 64 * VEC;
    const Span<VEC> me((int)threadIdx.x, c0, min(d.c - c0, 64 * VEC));
    if (me.first == VEC) return;
    const int end = video_frames(lengths, video, d.t);
    const int64_t at = (int64_t)video * d.c + me.at;
    float h[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) h[i] = h0 ? h0[at + i] : 0.0f;
    const int nm = (d.t + MARK - 1) / MARK;
#pragma unroll 4
    for (int t = 0; t < d.t; ++t) {
        if (marks && t % MARK == 0) store_some<VEC>(marks + ((int64_t)video * nm + t / MARK) * d.c + me.at, h, me.first);
        float v[VEC], g[VEC];
        const int k = t < end ? t : end > 0 ? end - 1 : 0;
        load_vec<VEC>(x + video * d.x_video + k * d.x_frame + me.at, v);
        load_vec<VEC>(f + video * d.f_video + k * d.f_frame + me.at, g);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            float a, o;
            gate_pair(g[i], a, o);
            h[i] = t < end ? a * h[i] + o * v[i] : h[i];
            v[i] = t < end ? h[i] : 0.0f;
        }
        store_some<VEC>(y + video * d.y_video + t * d.y_frame + me.at, v, me.first);
    }
    if (h_last) store_some<VEC>(h_last + at, h, me.first);
}

__global__ __launch_bounds__(256) void copy_state_kernel(float* to, const float* from, int n) {
    const int i = (int)(blockIdx.x * 256 + threadIdx.x);
    if (i < n) to[i] = from ? from[i] : 0.0f;
}

__global__ __launch_bounds__(256) void zero_words_kernel(word_t* p, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i] = 0;
}

int vec_of(const rrm_scan_desc& d) { return d.elem == RRM_F32 ? (d.c >= 4 ? 4 : 1) : (d.c >= 8 ? 8 : 1); }
bool few_frames(const rrm_scan_desc& d) { return d.t <= 16; }

// Frames of a block of the forward pass.  Long fp32 videos go in long blocks, half as many hands (us, blocks of 128 and 256 frames: fp32 1 x 65536 x
// 512 105 and 96, x 256 46 and 42, x 32 24 and 17, 1 x 40000 x 1024 117 and 110; 1 x 8000 x 512 15.2 and 15.2, 8 x 4096 x 1024 98 and 100; bf16 1 x 65536
// x 512 59 and 63, 1 x 40000 x 2048 134 and 139).
int forward_block(const rrm_scan_desc& d) { return d.elem == RRM_F32 && d.t >= 16384 ? LONG_BLOCK : GS_BLOCK; }

// A call's chains, and where their words lie in the workspace.  A chain has one workgroup where it has few frames (us, one workgroup and many: forward
// 2 x t x 512 bf16, t = 384 12 and 15, 768 21 and 15; backward 1 x t x 512 bf16, t = 200 16 and 16, 260 19 and 15, 520 30 and 15; the words have to be
// cleared first) or where chains fill the card by themselves (n x 4096 x 4096 bf16, 64 chains each: forward n = 4 127 and 100, 6 151 and 148, 7 161 and
// 169; backward n = 4 224 and 170, 6 279 and 248, 7 284 and 286).
struct Plan {
    Chain ch;
    int64_t chains, words;  // of the workspace, the counters at its head included
    bool chained;
    Plan(const rrm_scan_desc& d, bool backward, void* ws) {
        const int v = vec_of(d), width = v * Tile<1>::LANES;
        ch.tiles = (int)(((int64_t)d.c + width - 1) / width);
        ch.blocks = (d.t - 1) / (backward ? GS_BLOCK : forward_block(d)) + 1;
        ch.groups = (ch.blocks - 1) / GROUP + 1;
        chains = (int64_t)d.n * ch.tiles;
        chained = chains <= 3 * OP_CUS / 2 && d.t > (backward ? 2 : 5) * GS_BLOCK;
        ch.per = 1;
        if (chained) {
            const int64_t want = (8 * OP_CUS + chains - 1) / chains;
            ch.per = (int)(want < ch.blocks ? want : ch.blocks);
        }
        const int64_t maps = chains * 8, states = maps + chains * ch.blocks * width;
        ch.counters = static_cast<unsigned int*>(ws);
        ch.maps = ws ? static_cast<word_t*>(ws) + maps : nullptr;
        ch.states = ws ? static_cast<word_t*>(ws) + states : nullptr;
        words = chained ? chains * (8 + (int64_t)(ch.blocks + ch.groups) * width) : 0;
    }
    dim3 grid() const { return dim3((unsigned)(chains * ch.per)); }
    void clear(hipStream_t s) const {
        if (chained) hipLaunchKernelGGL(zero_words_kernel, dim3((unsigned)std::min<int64_t>((words + 511) / 512, 8 * OP_CUS)), dim3(256), 0, s, (word_t*)ch.counters, words);
    }
};

// f(element, VEC)
template <typename F>
void with_shape(const rrm_scan_desc& d, F&& f) {
    if (d.elem == RRM_F32)
        vec_of(d) == 4 ? f(float{}, std::integral_constant<int, 4>{}) : f(float{}, std::integral_constant<int, 1>{});
    else
        vec_of(d) == 8 ? f(__bf16{}, std::integral_constant<int, 8>{}) : f(__bf16{}, std::integral_constant<int, 1>{});
}

}  // namespace

size_t scan_scratch(const rrm_scan_desc& d, bool backward) {
    if (d.n == 0 || d.t == 0 || d.c == 0 || (!backward && few_frames(d))) return 0;
    return round256((size_t)Plan(d, backward, nullptr).words * sizeof(word_t));
}

void scan_layout(const rrm_scan_desc& d, bool backward, int* layout) {
    layout[0] = layout[1] = 0;
    if (d.t == 0 || (!backward && few_frames(d))) return;
    const bool chained = Plan(d, backward, nullptr).chained;
    layout[0] = chained ? 2 : 1;
    layout[1] = backward ? (chained ? GS_BLOCK : BACK_BLOCK) : chained ? forward_block(d) : GS_BLOCK;
}

hipError_t launch_gated_scan(const rrm_scan_desc& d, const void* x, const void* f, const float* h0, const int32_t* lengths,
                             void* y, float* h_last, float* marks, void* ws, hipStream_t s) {
    if (d.t == 0) {
        if (h_last)
            hipLaunchKernelGGL(copy_state_kernel, dim3((unsigned)(((int64_t)d.n * d.c + 255) / 256)), dim3(256), 0, s, h_last, h0, d.n * d.c);
        return hipGetLastError();
    }
    with_shape(d, [&](auto t, auto vec) {
        using T = decltype(t);
        constexpr int VEC = decltype(vec)::value;
        if (few_frames(d)) {
            in_parts(d.n * (((int64_t)d.c + 64 * VEC - 1) / (64 * VEC)), [&](unsigned from, unsigned count) {
                hipLaunchKernelGGL((short_scan_kernel<T, VEC>), dim3(count), dim3(64), 0, s, d, from, (const T*)x, (const T*)f, h0, lengths, (T*)y,
                                   h_last, marks);
            });
            return;
        }
        const Plan p(d, false, ws);
        p.clear(s);
        auto chained = [&](auto block) {
            hipLaunchKernelGGL((chained_scan_kernel<T, VEC, decltype(block)::value>), p.grid(), dim3(GS_THREADS), 0, s, d, p.ch, (const T*)x, (const T*)f, h0,
                               lengths, (T*)y, h_last, marks);
        };
        if (p.chained) {
            if constexpr (sizeof(T) == 4) {
                if (forward_block(d) == LONG_BLOCK) return chained(std::integral_constant<int, LONG_BLOCK>{});
            }
            chained(std::integral_constant<int, GS_BLOCK>{});
        } else
            in_parts(p.chains, [&](unsigned from, unsigned count) {
                hipLaunchKernelGGL((scan_kernel<T, VEC>), dim3(count), dim3(GS_THREADS), 0, s, d, p.ch.tiles, from, (const T*)x, (const T*)f, h0, lengths,
                                   (T*)y, h_last, marks);
            });
    });
    return hipGetLastError();
}

hipError_t launch_gated_scan_backward(const rrm_scan_desc& d, const void* x, const void* f, const float* marks,
                                      const int32_t* lengths, const void* dy, const float* dh_last, void* dx, void* df,
                                      float* dh0, void* ws, hipStream_t s) {
    if (d.t == 0) {
        if (dh0)
            hipLaunchKernelGGL(copy_state_kernel, dim3((unsigned)(((int64_t)d.n * d.c + 255) / 256)), dim3(256), 0, s, dh0, dh_last, d.n * d.c);
        return hipGetLastError();
    }
    with_shape(d, [&](auto t, auto vec) {
        using T = decltype(t);
        constexpr int VEC = decltype(vec)::value;
        const Plan p(d, true, ws);
        p.clear(s);
        if (p.chained)
            hipLaunchKernelGGL((chained_scan_back_kernel<T, VEC>), p.grid(), dim3(GS_THREADS), 0, s, d, p.ch, (const T*)x, (const T*)f, marks, lengths, (const T*)dy, dh_last, (T*)dx, (T*)df, dh0);
        else
            in_parts(p.chains, [&](unsigned from, unsigned count) {
                hipLaunchKernelGGL((scan_back_kernel<T, VEC>), dim3(count), dim3(GS_THREADS), 0, s, d, p.ch.tiles, from, (const T*)x, (const T*)f, marks,
                                   lengths, (const T*)dy, dh_last, (T*)dx, (T*)df, dh0);
            });
    });
    return hipGetLastError();
}

}  // namespace rrm
