// Gated linear recurrence over the frames of videos, and its backward pass.
//
//      a = sigmoid(f)      h_t = a_t h_{t-1} + (1 - a_t) x_t      g_t = dy_t + a_{t+1} g_{t+1}
//
// A frame is an affine map of the state, h -> A h + B, and maps of neighbouring frames join to one: (A2 A1, A2 B1 + B2).  A workgroup has a
// tile of features of one video and goes through its frames in blocks: a thread holds SPAN frames of its features in registers and joins them, the
// rows' maps meet in LDS, where one thread a feature carries the state through them, and each thread makes its frames from the state that it is
// handed.  So x and f are read once.  The gradient runs the other way by the same maps (its A is the same product), and h is made again from
// the state kept every RRM_SCAN_MARK_FRAMES frames.
#include "op_common.h"

namespace rrm {

namespace {

constexpr int GS_THREADS = 256;
constexpr int GS_BLOCK = 128;  // frames of a block; the chunks of the time axis are whole blocks
constexpr int MARK = RRM_SCAN_MARK_FRAMES;
static_assert(GS_BLOCK % MARK == 0, "chunks begin at marks");

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

// where the time axis is cut: workgroups of a video's tile, each a number of blocks
struct Cut {
    int tiles, chunks, frames;  // tiles of features; chunks of the frames; frames of a chunk (whole blocks)
};
struct Place {
    int video, tile, chunk;
    __device__ __forceinline__ Place(const Cut& c, int chunks) {
        const unsigned id = blockIdx.x, per = (unsigned)(c.tiles * chunks);
        video = (int)(id / per);
        const unsigned k = id - (unsigned)video * per;
        chunk = (int)(k / (unsigned)c.tiles);
        tile = (int)(k % (unsigned)c.tiles);
    }
};

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

// The map of a chunk, [n][chunks][2][c] (A, B): forward h -> A h + B, backward g -> A g + B from a chunk's end to its start.  Rows have runs of frames of
// their own, so that the maps meet once.
template <typename T, int VEC, bool BACK>
__global__ __launch_bounds__(GS_THREADS) void chunk_maps_kernel(rrm_scan_desc d, Cut cut, const T* __restrict__ in, const T* __restrict__ f,
                                                                const int32_t* __restrict__ lengths, float* __restrict__ maps) {
    using Z = Tile<VEC>;
    __shared__ __attribute__((aligned(16))) float sa[Z::ROWS * Z::WIDTH];
    __shared__ __attribute__((aligned(16))) float sb[Z::ROWS * Z::WIDTH];
    Place w(cut, cut.chunks - 1);  // (forward nobody asks for the last chunk's map, backward for the first's)
    if (BACK) ++w.chunk;
    const int c0 = w.tile * Z::WIDTH, width = min(d.c - c0, Z::WIDTH), row = (int)threadIdx.x / Z::LANES;
    const Span<VEC> me((int)threadIdx.x % Z::LANES, c0, width);
    const int end = video_frames(lengths, w.video, d.t);
    const int t0 = w.chunk * cut.frames, per = cut.frames / Z::ROWS;
    const int b = t0 + row * per, e = min(b + per, end);
    const int64_t in_frame = BACK ? d.y_frame : d.x_frame;
    const T* ip = in + w.video * (BACK ? d.y_video : d.x_video) + me.at;
    const T* fp = f + w.video * d.f_video + me.at;
    float A[VEC], B[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) A[i] = 1.0f, B[i] = 0.0f;
#pragma unroll 4
    for (int t = b; t < e; ++t) {
        float v[VEC], g[VEC];
        load_vec<VEC>(ip + t * in_frame, v);
        load_vec<VEC>(fp + t * d.f_frame, g);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            float a, o;
            gate_pair(g[i], a, o);
            A[i] *= a;
            B[i] = BACK ? B[i] + A[i] * v[i]  // (dy of a frame reaches the state before the chunk through the gates up to its own)
                        : a * B[i] + o * v[i];
        }
    }
    put<VEC>(sa + row * Z::WIDTH, me.at - c0, me.first, A);
    put<VEC>(sb + row * Z::WIDTH, me.at - c0, me.first, B);
    __syncthreads();
    const int j = (int)threadIdx.x;
    if (j >= width) return;
    float a = 1.0f, s = 0.0f;
    for (int r = 0; r < Z::ROWS; ++r) {
        const float ra = sa[r * Z::WIDTH + j], rb = sb[r * Z::WIDTH + j];
        if (BACK) s += a * rb;
        else s = ra * s + rb;
        a *= ra;
    }
    float* to = maps + ((int64_t)w.video * cut.chunks + w.chunk) * 2 * d.c + c0 + j;
    to[0] = a;
    to[d.c] = s;
}

// Thread j < width: `start` through the maps of `count` chunks, the first at `first`, the next `step` on (in floats).  The threads take a stretch of
// chunks of a feature each, and the stretches' maps meet in LDS: some hundred maps one after the other would be as many trips to memory
// (1 x 27594 x 80 fp32, forward and backward: 94 us so, 43 with stretches).
template <int WIDTH>
__device__ __forceinline__ float carried(const float* __restrict__ first, int64_t step, int count, int c, int width, float start, float* sa, float* sb) {
    if (count == 0) return start;
    constexpr int SEGS = GS_THREADS / WIDTH;
    const int j = (int)threadIdx.x % WIDTH, seg = (int)threadIdx.x / WIDTH;
    const int k0 = count * seg / SEGS, k1 = count * (seg + 1) / SEGS;
    float A = 1.0f, B = 0.0f;
    if (j < width) {
#pragma unroll 8
        for (int k = k0; k < k1; ++k) {
            const float ma = first[k * step + j], mb = first[k * step + c + j];
            A *= ma;
            B = ma * B + mb;
        }
    }
    sa[threadIdx.x] = A;
    sb[threadIdx.x] = B;
    lds_barrier();
    if (seg == 0) {
#pragma unroll
        for (int k = 0; k < SEGS; ++k) start = sa[k * WIDTH + j] * start + sb[k * WIDTH + j];
    }
    lds_barrier();
    return start;
}

template <typename T, int VEC>
__global__ __launch_bounds__(GS_THREADS) void scan_kernel(rrm_scan_desc d, Cut cut, const T* __restrict__ x, const T* __restrict__ f, const float* h0,
                                                          const int32_t* __restrict__ lengths, const float* __restrict__ maps, T* __restrict__ y,
                                                          float* h_last, float* __restrict__ marks) {
    using Z = Tile<VEC>;
    constexpr int S = Z::SPAN;
    __shared__ __attribute__((aligned(16))) float sa[2][Z::ROWS * Z::WIDTH];
    __shared__ __attribute__((aligned(16))) float sb[2][Z::ROWS * Z::WIDTH];
    const Place w(cut, cut.chunks);
    const int c0 = w.tile * Z::WIDTH, width = min(d.c - c0, Z::WIDTH), row = (int)threadIdx.x / Z::LANES, j = (int)threadIdx.x;
    const Span<VEC> me((int)threadIdx.x % Z::LANES, c0, width);
    const int end = video_frames(lengths, w.video, d.t);
    const int t0 = w.chunk * cut.frames, t1 = min(t0 + cut.frames, d.t);
    const T* xp = x + w.video * d.x_video + me.at;
    const T* fp = f + w.video * d.f_video + me.at;
    T* yp = y + w.video * d.y_video + me.at;
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
    const int live = min(t1, end);  // frames from here on are zeros
    if (t0 < live) fetch(t0);
    float carry = 0.0f;  // thread j: the state of feature c0 + j before the block
    if (j < width && h0) carry = h0[(int64_t)w.video * d.c + c0 + j];
    carry = carried<Z::WIDTH>(maps + (int64_t)w.video * cut.chunks * 2 * d.c + c0, 2 * (int64_t)d.c, w.chunk, d.c, width, carry, sa[0], sb[0]);
    int buf = 0;
    int tb = t0;
    for (; tb < live; tb += GS_BLOCK, buf ^= 1) {
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
        if (tb + GS_BLOCK < live) fetch(tb + GS_BLOCK);
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
            store_some<VEC>(marks + ((int64_t)w.video * nm + (tb + row * S) / MARK) * d.c + me.at, h, me.keep);
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
    if (tb < t1 && me.first < VEC) {
        float zero[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) zero[i] = 0.0f;
        for (int t = tb + row; t < t1; t += Z::ROWS) store_some<VEC>(yp + t * d.y_frame, zero, me.keep);
    }
    if (j < width) {
        if (marks)
            for (int t = tb; t < t1; t += MARK) marks[((int64_t)w.video * nm + t / MARK) * d.c + c0 + j] = carry;
        if (h_last && w.chunk == cut.chunks - 1) h_last[(int64_t)w.video * d.c + c0 + j] = carry;
    }
}

constexpr int BACK_BLOCK = 64;  // frames of a block of the backward pass: it holds four values a frame

template <typename T, int VEC>
__global__ __launch_bounds__(GS_THREADS, 3) void scan_back_kernel(rrm_scan_desc d, Cut cut, const T* __restrict__ x, const T* __restrict__ f,
                                                               const float* __restrict__ marks, const int32_t* __restrict__ lengths,
                                                               const T* __restrict__ dy, const float* dh_last, const float* __restrict__ maps,
                                                               T* __restrict__ dx, T* __restrict__ df, float* dh0) {
    using Z = Tile<VEC, BACK_BLOCK>;
    constexpr int S = Z::SPAN, MARKS = BACK_BLOCK / MARK, MROWS = Z::ROWS / MARKS;
    __shared__ __attribute__((aligned(16))) float sa[Z::ROWS * Z::WIDTH];
    __shared__ __attribute__((aligned(16))) float sb[Z::ROWS * Z::WIDTH];
    __shared__ __attribute__((aligned(16))) float sg[Z::ROWS * Z::WIDTH];
    const Place w(cut, cut.chunks);
    const int c0 = w.tile * Z::WIDTH, width = min(d.c - c0, Z::WIDTH), row = (int)threadIdx.x / Z::LANES, j = (int)threadIdx.x;
    const Span<VEC> me((int)threadIdx.x % Z::LANES, c0, width);
    const int end = video_frames(lengths, w.video, d.t);
    const int t0 = w.chunk * cut.frames, t1 = min(t0 + cut.frames, d.t), live = min(t1, end);
    const T* xp = x + w.video * d.x_video + me.at;
    const T* fp = f + w.video * d.f_video + me.at;
    const T* yp = dy + w.video * d.y_video + me.at;
    T* dxp = dx + w.video * d.dx_video + me.at;
    T* dfp = df + w.video * d.df_video + me.at;
    const int nm = (d.t + MARK - 1) / MARK;
    const int blocks = live > t0 ? (live - t0 + BACK_BLOCK - 1) / BACK_BLOCK : 0;
    if (me.first < VEC) {  // behind the video's end
        float zero[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) zero[i] = 0.0f;
        for (int t = t0 + blocks * BACK_BLOCK + row; t < t1; t += Z::ROWS) {
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
    if (blocks) fetch(t0 + (blocks - 1) * BACK_BLOCK);
    float carry = 0.0f;  // thread j: the gradient of the state behind the block, of feature c0 + j
    if (j < width && dh_last) carry = dh_last[(int64_t)w.video * d.c + c0 + j];
    carry = carried<Z::WIDTH>(maps + ((int64_t)(w.video + 1) * cut.chunks - 1) * 2 * d.c + c0, -2 * (int64_t)d.c, cut.chunks - 1 - w.chunk, d.c, width,
                              carry, sa, sb);
    for (int blk = blocks - 1; blk >= 0; --blk) {
        const int tb = t0 + blk * BACK_BLOCK;
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
                float h = marks[((int64_t)w.video * nm + tb / MARK + m) * d.c + c0 + c];
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
    if (dh0 && w.chunk == 0 && j < width) dh0[(int64_t)w.video * d.c + c0 + j] = carry;
}

// Few frames: a thread a vector of features, frame by frame.
template <typename T, int VEC>
__global__ __launch_bounds__(64) void short_scan_kernel(rrm_scan_desc d, const T* __restrict__ x, const T* __restrict__ f, const float* h0,
                                                        const int32_t* __restrict__ lengths, T* __restrict__ y, float* h_last,
                                                        float* __restrict__ marks) {
    const int per = (d.c + 64 * VEC - 1) / (64 * VEC), video = (int)(blockIdx.x / (unsigned)per), c0 = (int)(blockIdx.x % (unsigned)per) * 64 * VEC;
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

int vec_of(const rrm_scan_desc& d) { return d.elem == RRM_F32 ? (d.c >= 4 ? 4 : 1) : (d.c >= 8 ? 8 : 1); }
bool few_frames(const rrm_scan_desc& d) { return d.t <= 16; }
Cut cut_of(const rrm_scan_desc& d) {
    const int v = vec_of(d), width = v == 8 ? Tile<8>::WIDTH : v == 4 ? Tile<4>::WIDTH : Tile<1>::WIDTH;
    const int blocks = (d.t + GS_BLOCK - 1) / GS_BLOCK;
    Cut c{(d.c + width - 1) / width, 1, blocks * GS_BLOCK};
    const int64_t tiles = (int64_t)c.tiles * d.n;
    if (tiles >= 2 * OP_CUS || blocks < 2) return c;
    int64_t want = (4 * OP_CUS + tiles - 1) / tiles;
    if (want > blocks) want = blocks;
    const int per = (int)((blocks + want - 1) / want);
    c.frames = per * GS_BLOCK;
    c.chunks = (blocks + per - 1) / per;
    return c;
}

// f(element, VEC)
template <typename F>
void with_shape(const rrm_scan_desc& d, F&& f) {
    if (d.elem == RRM_F32)
        vec_of(d) == 4 ? f(float{}, std::integral_constant<int, 4>{}) : f(float{}, std::integral_constant<int, 1>{});
    else
        vec_of(d) == 8 ? f(__bf16{}, std::integral_constant<int, 8>{}) : f(__bf16{}, std::integral_constant<int, 1>{});
}

}  // namespace

// the chunks' maps
size_t scan_scratch(const rrm_scan_desc& d, bool backward) {
    if (!backward && few_frames(d)) return 0;
    const Cut c = cut_of(d);
    return c.chunks > 1 ? round256((size_t)d.n * c.chunks * 2 * d.c * 4) : 0;
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
            hipLaunchKernelGGL((short_scan_kernel<T, VEC>), dim3((unsigned)((int64_t)d.n * ((d.c + 64 * VEC - 1) / (64 * VEC)))), dim3(64), 0, s, d,
                               (const T*)x, (const T*)f, h0, lengths, (T*)y, h_last, marks);
            return;
        }
        const Cut c = cut_of(d);
        const dim3 grid((unsigned)((int64_t)d.n * c.tiles * c.chunks));
        if (c.chunks > 1)
            hipLaunchKernelGGL((chunk_maps_kernel<T, VEC, false>), dim3((unsigned)((int64_t)d.n * c.tiles * (c.chunks - 1))), dim3(GS_THREADS), 0, s, d, c, (const T*)x, (const T*)f, lengths, (float*)ws);
        hipLaunchKernelGGL((scan_kernel<T, VEC>), grid, dim3(GS_THREADS), 0, s, d, c, (const T*)x, (const T*)f, h0, lengths, (const float*)ws,
                           (T*)y, h_last, marks);
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
        const Cut c = cut_of(d);
        const dim3 grid((unsigned)((int64_t)d.n * c.tiles * c.chunks));
        if (c.chunks > 1)
            hipLaunchKernelGGL((chunk_maps_kernel<T, VEC, true>), dim3((unsigned)((int64_t)d.n * c.tiles * (c.chunks - 1))), dim3(GS_THREADS), 0, s, d, c, (const T*)dy, (const T*)f, lengths, (float*)ws);
        hipLaunchKernelGGL((scan_back_kernel<T, VEC>), grid, dim3(GS_THREADS), 0, s, d, c, (const T*)x, (const T*)f, marks, lengths,
                           (const T*)dy, dh_last, (const float*)ws, (T*)dx, (T*)df, dh0);
    });
    return hipGetLastError();
}

}  // namespace rrm
