// Gated feed-forward block and its backward pass.
//
//      G = X Wg^T     U = X Wu^T     H = act(G) * U
//      dG = dH * U * act'(G)     dU = dH * act(G)     dX = dG Wg + dU Wu     dWg = dG^T X     dWu = dU^T X
//
// Both projections are one product: a wavefront's blocks of 32 columns belong to the one and the other in turn, so act(G) * U is made of two
// registers of one lane, and G and U meet memory only where the backward pass is to have them.  Backward, dG and dU are made once, dX sums both
// products in one accumulator, and both dW are tiles of one launch.  No operand is transposed in memory: what lies across the summed axis is
// turned on its way from LDS to the registers.  All sums are held in 32 bits.
//
// Two roundings to bfloat16 stand between them.  G and U are kept for the backward pass in it: 32 bits would be four more bytes a hidden value and row to
// write, to hold and to read.  dG and dU are made in it, as the matrix cores take them; each goes into k products of each gradient, and two bfloat16 parts of each
// would double those.  Relative error of a gradient (1024 x 512 -> 1024, silu): 0.0030; rounding the result alone leaves 0.0017, with G and U in 32 bits
// 0.0023, with dG and dU 0.0025.
#include "tile_product.h"

namespace rrm {

namespace {

template <int KIND, int ACT, bool PT, bool QT, int MT, int NT, int WM, int WN, int STAGES>
__global__ __launch_bounds__(WM* WN * 64, 2) void tile_kernel(Product a) {
    __shared__ __attribute__((aligned(1024))) unsigned char lds[TILE_LDS<MT, NT, WM, WN, STAGES>];
    tile_product<KIND, ACT, PT, QT, MT, NT, WM, WN, STAGES>(a, lds, (int)blockIdx.x, (int)blockIdx.y);
}
// dX and both dW in one launch, so that the one's last workgroups run beside the other's: first `dx`, its splits one behind the other, `whole_x`
// workgroups each (its tiles, to whole eights: ids go to the XCDs in turn), then `dw` likewise
template <int MT, int NT, int WM, int WN, int STAGES>
__global__ __launch_bounds__(WM* WN * 64, 2) void gradients_kernel(Product dx, Product dw, int whole_x, int whole_w) {
    __shared__ __attribute__((aligned(1024))) unsigned char lds[TILE_LDS<MT, NT, WM, WN, STAGES>];
    const int first = whole_x * dx.splits, id = (int)blockIdx.x;
    if (id < first) {
        const int split = id / whole_x, k = id - split * whole_x;
        if (k < dx.tiles_m * dx.tiles_n) tile_product<PLAIN, RRM_ACT_NONE, false, true, MT, NT, WM, WN, STAGES>(dx, lds, k, split);
    } else {
        const int split = (id - first) / whole_w, k = id - first - split * whole_w;
        if (k < dw.tiles_m * dw.tiles_n) tile_product<HALVES, RRM_ACT_NONE, true, true, MT, NT, WM, WN, STAGES>(dw, lds, k, split);
    }
}

// Few rows (up to 16): the weights are the traffic, and each is read once, from memory straight into the fragments of the
// matrix cores.  A workgroup makes 16 hidden features; its eight wavefronts take eight parts of the summed axis and meet in LDS.
// One row, 4096 -> 4096: 14.1 us, 4.8 TB/s, with weights out of the 256 MB cache, 16.7 with weights out of memory.
constexpr int FEW_WAVES = 8, FEW_F = 16, FEW_ROWS = 16;
typedef float v4f __attribute__((ext_vector_type(4)));

template <int ACT>
__global__ __launch_bounds__(FEW_WAVES * 64, 4) void few_rows_kernel(rrm_ff_desc d, src_t x, src_t wg, src_t wu, __bf16* h, __bf16* g, __bf16* u) {
    __shared__ float sums[FEW_WAVES][2][FEW_F][FEW_ROWS + 1];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int f0 = (int)blockIdx.x * FEW_F;
    // lane l: row l % 16 of the weights (and of x), eight of the summed axis from (l / 16) * 8 on in a step of 32
    const int lr = lane & 15, lk = (lane >> 4) * 8;
    const int fr = f0 + lr < d.f ? f0 + lr : d.f - 1;
    const int steps = (d.k + 31) / 32, s0 = steps * wave / FEW_WAVES, s1 = steps * (wave + 1) / FEW_WAVES;
    const int whole = s1 * 32 <= d.k ? s1 : s1 - 1;  // steps without a ragged end
    const src_t pg = wg + fr * d.wg_row, pu = wu + fr * d.wu_row, px = x + (lr < d.m ? lr : d.m - 1) * d.x_row;
    v4f ag = {0, 0, 0, 0}, au = {0, 0, 0, 0};
    auto some = [&](int s, auto count) __attribute__((always_inline)) {
        constexpr int N = decltype(count)::value;
        v8bf bg[N], bu[N], bx[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int k = (s + j) * 32 + lk;
            bg[j] = __builtin_bit_cast(v8bf, loose_chunk(pg + k));
            bu[j] = __builtin_bit_cast(v8bf, loose_chunk(pu + k));
        }
#pragma unroll
        for (int j = 0; j < N; ++j) bx[j] = __builtin_bit_cast(v8bf, loose_chunk(px + (s + j) * 32 + lk));
        __builtin_amdgcn_sched_barrier(0);  // all of them are on their way before the first is waited for
#pragma unroll
        for (int j = 0; j < N; ++j) {
            ag = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bg[j], bx[j], ag, 0, 0, 0);
            au = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bu[j], bx[j], au, 0, 0, 0);
        }
    };
    int s = s0;
    for (; s + 8 <= whole; s += 8) some(s, std::integral_constant<int, 8>{});
    for (; s < whole; ++s) some(s, std::integral_constant<int, 1>{});
    if (s < s1) {
        auto chunk = [&](src_t row) { return __builtin_bit_cast(v8bf, ragged_chunk(row, s * 32 + lk, d.k)); };
        const v8bf bg = chunk(pg), bu = chunk(pu);
        const v8bf bx = chunk(px);
        ag = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bg, bx, ag, 0, 0, 0);
        au = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bu, bx, au, 0, 0, 0);
    }
    // register e of lane l: feature 4 (l / 16) + e, row l % 16
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        sums[wave][0][(lane >> 4) * 4 + e][lr] = ag[e];
        sums[wave][1][(lane >> 4) * 4 + e][lr] = au[e];
    }
    __syncthreads();
    if (threadIdx.x < FEW_F * FEW_ROWS) {
        const int f = threadIdx.x % FEW_F, r = threadIdx.x / FEW_F;
        if (r >= d.m || f0 + f >= d.f) return;
        float sg = 0.0f, su = 0.0f;
#pragma unroll
        for (int w = 0; w < FEW_WAVES; ++w) sg += sums[w][0][f][r], su += sums[w][1][f][r];
        h[r * d.h_row + f0 + f] = (__bf16)(act_value<ACT>(sg) * su);
        if (g) {
            g[r * d.gu_row + f0 + f] = (__bf16)sg;
            u[r * d.gu_row + f0 + f] = (__bf16)su;
        }
    }
}

// Four neighbours of the splits' sums, in their order
__device__ __forceinline__ float4 joined(const float* __restrict__ part, int64_t at, int64_t plane, int splits) {
    float4 s = *reinterpret_cast<const float4*>(part + at);
    for (int k = 1; k < splits; ++k) {
        const float4 v = *reinterpret_cast<const float4*>(part + k * plane + at);
        s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
    }
    return s;
}
__device__ __forceinline__ void leave_four(__bf16* to, const float (&v)[4], int n) {
    struct __attribute__((packed, aligned(2))) Four {
        u32x2 v;
    };
    if (n >= 4) {
        u32x2 w;
        w.x = bf16_pair(v[0], v[1]), w.y = bf16_pair(v[2], v[3]);
        reinterpret_cast<Four*>(to)->v = w;
    } else {
        to[0] = (__bf16)v[0];
        if (n > 1) to[1] = (__bf16)v[1];
        if (n > 2) to[2] = (__bf16)v[2];
    }
}
// Up to three results (blockIdx.y) of split sums
struct Join {
    const float* part;
    int64_t plane;  // from a split's sums to the next one's
    __bf16* out;
    int64_t row;
    int splits, rows, cols;
};
struct Joins {
    Join j[3];
};
__global__ __launch_bounds__(256) void join_kernel(Joins all) {
    const Join& j = all.j[blockIdx.y];
    const int fours = (j.cols + 3) >> 2;
    const int64_t total = (int64_t)j.rows * fours;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / fours;
        const int c = (int)(i - r * fours) * 4;
        const float4 s = joined(j.part, 4 * i, j.plane, j.splits);
        const float v[4] = {s.x, s.y, s.z, s.w};
        leave_four(j.out + r * j.row + c, v, j.cols - c);
    }
}
// H, G and U of the splits' sums
template <int ACT>
__global__ __launch_bounds__(256) void join_gated_kernel(const float* __restrict__ part, int splits, int rows, int cols, __bf16* __restrict__ h,
                                                         int64_t h_row, __bf16* __restrict__ g, __bf16* __restrict__ u, int64_t gu_row) {
    const int fours = (cols + 3) >> 2;
    const int64_t total = (int64_t)rows * fours;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / fours;
        const int c = (int)(i - r * fours) * 4;
        const float4 sg = joined(part, 4 * i, 8 * total, splits), su = joined(part + 4 * total, 4 * i, 8 * total, splits);
        const float vg[4] = {sg.x, sg.y, sg.z, sg.w}, vu[4] = {su.x, su.y, su.z, su.w};
        float vh[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) vh[e] = act_value<ACT>(vg[e]) * vu[e];
        leave_four(h + r * h_row + c, vh, cols - c);
        if (g) {
            leave_four(g + r * gu_row + c, vg, cols - c);
            leave_four(u + r * gu_row + c, vu, cols - c);
        }
    }
}

// Copies of up to three operands of rows of `len`, padded with zeros to whole chunks; chunk i of all of them
struct PadJob {
    Source from[3];
    __bf16* to[3];
    int64_t first[4];  // chunk that each begins with; the end
    int n, len;
};
__device__ __forceinline__ void pad_chunk(const PadJob& j, int64_t i) {
    const int per = (j.len + 7) / 8;
    const int w = i < j.first[1] || j.n == 1 ? 0 : i < j.first[2] || j.n == 2 ? 1 : 2;
    const Source from = w == 0 ? j.from[0] : w == 1 ? j.from[1] : j.from[2];
    __bf16* to = w == 0 ? j.to[0] : w == 1 ? j.to[1] : j.to[2];
    const int64_t at = i - (w == 0 ? 0 : w == 1 ? j.first[1] : j.first[2]), r = at / per;
    *reinterpret_cast<u32x4*>(to + at * 8) = ragged_chunk(from.p + r * from.row, (int)(at - r * per) * 8, j.len);
}
__global__ __launch_bounds__(256) void pad_kernel(PadJob j) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < j.first[j.n]; i += (int64_t)gridDim.x * 256) pad_chunk(j, i);
}

// dG and dU from dH, G and U (16384 x 4096: 136 us, 4.9 TB/s); rows of `pitch` elements, a multiple of eight, zeros behind column f (they are
// summed over), eight columns a thread; then the padded copies that the products need.
template <int ACT>
__global__ __launch_bounds__(256) void slopes_kernel(rrm_ff_desc d, src_t g, src_t u, src_t dh, int pitch, __bf16* __restrict__ dg, __bf16* __restrict__ du,
                                                     PadJob job) {
    const int64_t chunks = pitch / 8, total = chunks * d.m, all = total + (job.n ? job.first[job.n] : 0);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        if (i >= total) {
            pad_chunk(job, i - total);
            continue;
        }
        const int64_t r = i / chunks;
        const int f = (int)(i - r * chunks) * 8;
        float gv[8], uv[8], dv[8], og[8], ou[8];
        if (f + 8 <= d.f) {
            load_vec<8>(g + r * d.gu_row + f, gv);
            load_vec<8>(u + r * d.gu_row + f, uv);
            load_vec<8>(dh + r * d.h_row + f, dv);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const bool in = f + e < d.f;
                gv[e] = in ? (float)g[r * d.gu_row + f + e] : 0.0f;
                uv[e] = in ? (float)u[r * d.gu_row + f + e] : 0.0f;
                dv[e] = in ? (float)dh[r * d.h_row + f + e] : 0.0f;
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float v, slope;
            act_pair<ACT>(gv[e], v, slope);
            og[e] = dv[e] * uv[e] * slope;
            ou[e] = dv[e] * v;
        }
        store_vec<8>(dg + r * pitch + f, og);
        store_vec<8>(du + r * pitch + f, ou);
    }
}

template <int KIND, int ACT, bool PT, bool QT, int MT, int NT, int WM, int WN, int STAGES>
hipError_t launch_tiles(Product& a, hipStream_t s) {
    constexpr int BM = MT * 32 * WM, BN = NT * 32 * WN / (KIND == GATED ? 2 : 1);
    a.tiles_m = tiles(a.rows, BM) * (KIND == HALVES ? 2 : 1);
    a.tiles_n = tiles(a.cols, BN);
    hipLaunchKernelGGL((tile_kernel<KIND, ACT, PT, QT, MT, NT, WM, WN, STAGES>), dim3((unsigned)(a.tiles_m * a.tiles_n), (unsigned)a.splits),
                       dim3(WM * WN * 64), 0, s, a);
    return hipGetLastError();
}
template <int KIND, int ACT, bool PT, bool QT>
hipError_t launch_product(Product& a, int shape, hipStream_t s) {
    switch (shape) {
        case BIG: return launch_tiles<KIND, ACT, PT, QT, 4, 2, 2, 4, 2>(a, s);
        case WIDE: return launch_tiles<KIND, ACT, PT, QT, 2, 2, 2, 2, 4>(a, s);
        case WIDE_PAIR: return launch_tiles<KIND, ACT, PT, QT, 2, 2, 2, 2, 2>(a, s);
        default: return launch_tiles<KIND, ACT, PT, QT, 1, 2, 2, 2, 3>(a, s);
    }
}
template <int MT, int NT, int WM, int WN, int STAGES>
hipError_t launch_both(Product& x, Product& w, hipStream_t s) {
    constexpr int BM = MT * 32 * WM, BN = NT * 32 * WN;
    x.tiles_m = tiles(x.rows, BM), x.tiles_n = tiles(x.cols, BN);
    w.tiles_m = 2 * tiles(w.rows, BM), w.tiles_n = tiles(w.cols, BN);
    const int whole_x = round8(x.tiles_m * x.tiles_n), whole_w = round8(w.tiles_m * w.tiles_n);
    hipLaunchKernelGGL((gradients_kernel<MT, NT, WM, WN, STAGES>), dim3((unsigned)(whole_x * x.splits + whole_w * w.splits)), dim3(WM * WN * 64), 0, s,
                       x, w, whole_x, whole_w);
    return hipGetLastError();
}
hipError_t launch_gradients(Product& x, Product& w, int shape, hipStream_t s) {
    switch (shape) {
        case BIG: return launch_both<4, 2, 2, 4, 2>(x, w, s);
        case WIDE: return launch_both<2, 2, 2, 2, 4>(x, w, s);
        case WIDE_PAIR: return launch_both<2, 2, 2, 2, 2>(x, w, s);
        default: return launch_both<1, 2, 2, 2, 3>(x, w, s);
    }
}
Plan forward_plan(const rrm_ff_desc& d) {
    return plan_products({d.m, 2 * d.f, tiles(d.k, STEP), 1}, {0, 0, 0, 0}, 2.0f * d.k * ((float)d.m + 2.0f * d.f));
}
// dX and dW, one launch of one shape or each by itself (512 x 4096 x 4096: dX wants few large parts, dW 256 x 256 tiles of eight steps; 106 us
// together, 92 apart; 512 x 1024 x 2048: 27 and 34)
struct GradientsPlan {
    int x_shape, w_shape, x_splits, w_splits;
    bool together;
};
GradientsPlan gradients_plan(const rrm_ff_desc& d, bool dx, bool dw) {
    const Work x{d.m, d.k, 2 * tiles(d.f, STEP), 1}, w{d.f, d.k, tiles(d.m, STEP), 2}, none{0, 0, 0, 0};
    const float of_x = 2.0f * ((float)d.m + d.k) * 2 * d.f, of_w = 2.0f * ((float)d.m * d.k + 2.0f * d.f * d.k);
    const Plan px = plan_products(x, none, of_x), pw = plan_products(w, none, of_w);
    if (dx && dw) {
        const Plan both = plan_products(x, w, of_x + of_w);
        if (both.us < px.us + pw.us) return {both.shape, both.shape, both.splits, both.splits2, true};
    }
    return {px.shape, pw.shape, px.splits, pw.splits, false};
}

// Up to so many rows the weights go from memory into the fragments (few_rows_kernel).  us so and by tiles, weights out of memory, 1 / 8 / 16 rows: 4096 ->
// 4096 16.7 / 17.3 / 18.5 and 20.3 / 20.9 / 22.0; 4096 -> 9216 38.2 / 41.1 / 45.4 and 41.6 / 41.5 / 42.4; 1001 -> 2050 7.7 / 8.8 / 9.4 and
// 17.2 / 17.3 / 17.7.  The rule is by rows alone, and loses where weights are wide and rows many (16 rows, 9216 features: 7%) or the weights, some 150 MB, stay in
// the 256 MB cache (4096 -> 9216 31.2 / 34.3 / 37.7 and 23.9 / 24.0 / 24.4; 4096 -> 4096 14.1 / 15.2 / 16.1 and 17.6 / 17.7 / 18.0).  Beyond 16 rows each
// set of 16 reads the weights again: 4096 -> 4096 32 rows 28 us and 19.
bool few_rows(const rrm_ff_desc& d) { return d.m <= FEW_ROWS; }

// The tile kernel copies whole, aligned 16-byte chunks: rows that are not made of them are copied to the workspace first, padded with zeros.
bool loose_rows(const rrm_ff_desc& d, int64_t row) { return d.unaligned || d.k % 8 != 0 || row % 8 != 0; }
struct Padded {
    size_t x, wg, wu, all;  // places in the workspace, and the bytes of all
};
Padded padded_places(const rrm_ff_desc& d, bool x, bool w) {
    Padded p{};
    const size_t row = (size_t)round8(d.k) * 2;
    auto take = [&](int rows, int64_t stride, bool used) {
        const size_t at = p.all;
        if (used && loose_rows(d, stride)) p.all += round256(row * rows);
        return at;
    };
    p.x = take(d.m, d.x_row, x);
    p.wg = take(d.f, d.wg_row, w);
    p.wu = take(d.f, d.wu_row, w);
    return p;
}
// Sources for the products of up to three operands of rows of k: themselves, or padded copies, which `job` is to make
PadJob sources(const rrm_ff_desc& d, const void* x, const void* wg, const void* wu, unsigned char* ws, Source& sx, Source& sg, Source& su) {
    const Padded at = padded_places(d, x != nullptr, wg != nullptr);
    PadJob job{};
    job.len = d.k;
    auto one = [&](const void* p, int64_t row, int rows, size_t place) {
        if (!p || !loose_rows(d, row)) return Source{(src_t)p, row};
        __bf16* to = (__bf16*)(ws + place);
        job.from[job.n] = Source{(src_t)p, row};
        job.to[job.n] = to;
        job.first[job.n + 1] = job.first[job.n] + (int64_t)rows * (round8(d.k) / 8);
        ++job.n;
        return Source{to, round8(d.k)};
    };
    sx = one(x, d.x_row, d.m, at.x);
    sg = one(wg, d.wg_row, d.f, at.wg);
    su = one(wu, d.wu_row, d.f, at.wu);
    return job;
}
unsigned some_groups(int64_t chunks) {
    const int64_t groups = (chunks + 255) / 256;
    return (unsigned)(groups < OP_CUS * 32 ? groups : OP_CUS * 32);
}

size_t grads_bytes(const rrm_ff_desc& d) { return round256((size_t)d.m * round8(d.f) * 2); }
size_t sums_bytes(int splits, int rows, int cols, int ways) { return splits > 1 ? round256((size_t)splits * rows * tiles(cols, 4) * 16 * ways) : 0; }
size_t split_bytes(const rrm_ff_desc& d, bool backward) {
    if (!backward) return sums_bytes(forward_plan(d).splits, d.m, d.f, 2);
    size_t most = 0;
    for (int asked = 1; asked < 4; ++asked) {  // whichever gradients a call asks for
        const GradientsPlan p = gradients_plan(d, asked & 1, asked & 2);
        const size_t b = sums_bytes(p.x_splits, d.m, d.k, 1) + sums_bytes(p.w_splits, d.f, d.k, 2);
        most = b > most ? b : most;
    }
    return most;
}

}  // namespace

// forward: [padded operands][splits' sums]; backward: [dG][dU][padded operands][splits' sums]
size_t ff_scratch(const rrm_ff_desc& d, bool backward) {
    if (d.m == 0 || (!backward && few_rows(d))) return 0;
    return (backward ? 2 * grads_bytes(d) : 0) + padded_places(d, true, true).all + split_bytes(d, backward);
}

void ff_layout(const rrm_ff_desc& d, int asked, int* layout) {
    layout[0] = layout[2] = -2;
    layout[1] = layout[3] = layout[4] = 0;
    if (asked == 0) {
        const Plan p = forward_plan(d);
        layout[0] = few_rows(d) ? -1 : p.shape;
        layout[1] = few_rows(d) ? 1 : p.splits;
        return;
    }
    const GradientsPlan p = gradients_plan(d, asked & 1, asked & 2);
    if (asked & 1) layout[0] = p.x_shape, layout[1] = p.x_splits;
    if (asked & 2) layout[2] = p.w_shape, layout[3] = p.w_splits;
    layout[4] = p.together;
}

hipError_t launch_gated_ff(const rrm_ff_desc& d, const void* x, const void* wg, const void* wu, void* h, void* g, void* u, void* ws,
                           hipStream_t s) {
    hipError_t e = hipSuccess;
    if (few_rows(d)) {
        with_act(d.act, [&](auto act) {
            hipLaunchKernelGGL((few_rows_kernel<decltype(act)::value>), dim3((unsigned)tiles(d.f, FEW_F)), dim3(FEW_WAVES * 64), 0, s, d,
                               (src_t)x, (src_t)wg, (src_t)wu, (__bf16*)h, (__bf16*)g, (__bf16*)u);
        });
        return hipGetLastError();
    }
    Product a{};
    const PadJob job = sources(d, x, wg, wu, (unsigned char*)ws, a.p[0], a.q[0], a.q[1]);
    if (job.n) {
        hipLaunchKernelGGL(pad_kernel, dim3(some_groups(job.first[job.n])), dim3(256), 0, s, job);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    const Plan plan = forward_plan(d);
    a.pairs = 1, a.splits = plan.splits;
    a.part = (float*)((unsigned char*)ws + padded_places(d, true, true).all);
    a.rows = d.m, a.cols = d.f, a.len = d.k;
    a.out = (__bf16*)h, a.out2 = (__bf16*)g, a.out3 = (__bf16*)u;
    a.out_row = d.h_row, a.out2_row = d.gu_row;
    with_act(d.act, [&](auto act) {
        e = launch_product<GATED, decltype(act)::value, false, false>(a, plan.shape, s);
        if (e != hipSuccess || a.splits == 1) return;
        const int64_t n = ((int64_t)d.m * tiles(d.f, 4) + 255) / 256;
        hipLaunchKernelGGL((join_gated_kernel<decltype(act)::value>), dim3((unsigned)(n < OP_CUS * 16 ? n : OP_CUS * 16)), dim3(256), 0, s, a.part,
                           a.splits, d.m, d.f, (__bf16*)h, d.h_row, (__bf16*)g, (__bf16*)u, d.gu_row);
        e = hipGetLastError();
    });
    return e;
}

hipError_t launch_gated_ff_backward(const rrm_ff_desc& d, const void* x, const void* wg, const void* wu, const void* g,
                                    const void* u, const void* dh, void* dx, void* dwg, void* dwu, void* ws, hipStream_t s) {
    unsigned char* at = (unsigned char*)ws;
    const int pitch = round8(d.f);
    const Source dg{(src_t)at, pitch}, du{(src_t)(at + grads_bytes(d)), pitch};
    Source sx{}, sg{}, su{};
    hipError_t e = hipSuccess;
    if (d.m > 0) {
        at += 2 * grads_bytes(d);
        const PadJob job = sources(d, dwg ? x : nullptr, dx ? wg : nullptr, dx ? wu : nullptr, at, sx, sg, su);
        at += padded_places(d, true, true).all;
        const int64_t chunks = (int64_t)d.m * (pitch / 8) + (job.n ? job.first[job.n] : 0);
        with_act(d.act, [&](auto act) {
            hipLaunchKernelGGL((slopes_kernel<decltype(act)::value>), dim3(some_groups(chunks)), dim3(256), 0, s, d, (src_t)g, (src_t)u, (src_t)dh,
                               pitch, (__bf16*)dg.p, (__bf16*)du.p, job);
        });
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    Product px{}, pw{};
    px.p[0] = dg, px.p[1] = du, px.q[0] = sg, px.q[1] = su;
    px.pairs = 2, px.splits = 1;
    px.part = (float*)at;
    px.rows = d.m, px.cols = d.k, px.len = d.f;
    px.out = (__bf16*)dx, px.out_row = d.dx_row;
    pw.p[0] = dg, pw.p[1] = du, pw.q[0] = sx;  // (no rows: sums of nothing, zeros)
    pw.pairs = 1, pw.splits = 1;
    pw.rows = d.f, pw.cols = d.k, pw.len = d.m;
    pw.out = (__bf16*)dwg, pw.out_row = d.dwg_row, pw.out2 = (__bf16*)dwu, pw.out2_row = d.dwu_row;
    const bool want_x = d.m > 0 && dx;
    if (d.m == 0) return dwg ? launch_product<HALVES, RRM_ACT_NONE, true, true>(pw, SMALL, s) : hipSuccess;
    const GradientsPlan plan = gradients_plan(d, want_x, dwg != nullptr);
    px.splits = plan.x_splits, pw.splits = plan.w_splits;
    pw.part = (float*)((unsigned char*)px.part + (want_x ? sums_bytes(px.splits, d.m, d.k, 1) : 0));
    if (plan.together) {
        e = launch_gradients(px, pw, plan.x_shape, s);
    } else {
        if (want_x) e = launch_product<PLAIN, RRM_ACT_NONE, false, true>(px, plan.x_shape, s);
        if (dwg && e == hipSuccess) e = launch_product<HALVES, RRM_ACT_NONE, true, true>(pw, plan.w_shape, s);
    }
    if (e != hipSuccess) return e;
    Joins joins{};
    int n = 0;
    int64_t fours = 0;
    auto join = [&](const Product& p, int ways, int way, __bf16* out, int64_t row) {
        const int64_t plane = (int64_t)p.rows * tiles(p.cols, 4) * 4;
        joins.j[n++] = Join{p.part + way * plane, ways * plane, out, row, p.splits, p.rows, p.cols};
        fours = plane / 4 > fours ? plane / 4 : fours;
    };
    if (want_x && px.splits > 1) join(px, 1, 0, px.out, px.out_row);
    if (dwg && pw.splits > 1) join(pw, 2, 0, pw.out, pw.out_row), join(pw, 2, 1, pw.out2, pw.out2_row);
    if (n == 0) return hipSuccess;
    const int64_t groups = (fours + 255) / 256;
    hipLaunchKernelGGL(join_kernel, dim3((unsigned)(groups < OP_CUS * 8 ? groups : OP_CUS * 8), (unsigned)n), dim3(256), 0, s, joins);
    return hipGetLastError();
}

}  // namespace rrm
