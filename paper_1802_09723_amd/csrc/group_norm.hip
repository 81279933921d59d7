// Group norm with an activation, channels last, and its backward pass.
//
//      xh = (x - mean) / sqrt(var + eps)      y = act(z),  z = gamma xh + beta      mean, var: over a group's channels and all positions of a sample
//      dz = dy act'(z)      dx = rstd (gamma dz - <gamma dz> - xh <gamma dz xh>)      dgamma = sum of dz xh, dbeta = sum of dz, over all samples
//
// (<..>: the mean over the group.)  Memory bounds it: x and y once (backward x, dy and dx), so a sample that fits is held in registers between its
// statistics and its result.  Sums are held in 32 bits, the variance is summed about a mean.  All sums run in one order: no atomics.
#include "op_common.h"

namespace rrm {

namespace {

constexpr int HELD_GROUPS = 64;  // groups of a workgroup at most
// A few workgroups (fewer than half the compute units) of more values than this take longer than slices on all compute units: us forward and backward,
// 2 x 126 positions x 139 channels fp32 13.5 and 15.4, 14.3 and 18.3 in slices; 5 x 1050 x 28 bf16 15.8 and 25.3, 15.4 and 18.6; 8 x 196 x 512
// bf16 33 and 21, 16 and 20.
constexpr int64_t HELD_FEW = 20000;

// ---- samples that registers hold ---------------------------------------------------------------------------------------
//
// A workgroup has the `cb` channels of whole groups of one sample, all positions; a thread keeps up to P vectors of VEC neighbouring
// channels (always the same channels) of positions R apart in registers.  So x (backward: and dy) is read once, the variance is summed about the
// mean, and the result leaves without another look at memory.
// Measured: 64 x 56 x 56 x 64, fp32 in and bf16 out, 21.0 us, 3.7 TB/s; 64 x 28 x 28 x 128 bf16, one round of workgroups, 12.4 us forward and
// 14.2 backward: their start, the reads, the sums and the writes one after the other, nothing beside them.
struct HeldGeom {
    int cb, blocks;  // channels of a workgroup; workgroups of a sample
    int lanes;       // threads of a position, a power of two
    float r_cg;      // 1 / channels of a group
};

// A workgroup's place: id -> sample, block; a sample's blocks, whose runs share cache lines, are on one XCD (ids go to the eight in turn)
__device__ __forceinline__ bool held_place(unsigned id, int n, int blocks, int& sample, int& block) {
    const int k = (int)(id >> 3);
    block = k % blocks;
    sample = (k / blocks) * 8 + (int)(id & 7);
    return sample < n;
}

// Sums between lanes without a trip through LDS.  A lane's value plus that of another lane of its sixteen:
template <int CTRL>
__device__ __forceinline__ float plus_lane(float v) {
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
// .. plus that of the lane 16 or 32 on (one register's odd rows change places with the other's even ones)
__device__ __forceinline__ float plus_16(float v) {
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}
__device__ __forceinline__ float plus_32(float v) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}
// over the lanes that are `lanes` apart, for each of v; rotations within sixteen
template <int N>
__device__ __forceinline__ void sum_over_rows(float (&v)[N], int lanes) {
    auto all = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = f(v[i]);
    };
    if (lanes <= 1) all([](float x) { return plus_lane<0x121>(x); });
    if (lanes <= 2) all([](float x) { return plus_lane<0x122>(x); });
    if (lanes <= 4) all([](float x) { return plus_lane<0x124>(x); });
    if (lanes <= 8) all([](float x) { return plus_lane<0x128>(x); });
    if (lanes <= 16) all(plus_16);
    if (lanes <= 32) all(plus_32);
}
// over `lanes` neighbouring lanes, aligned; neighbours within four, then mirrored halves of eight and of sixteen
__device__ __forceinline__ float sum_of_neighbours(float v, int lanes) {
    if (lanes > 1) v = plus_lane<0xb1>(v);
    if (lanes > 2) v = plus_lane<0x4e>(v);
    if (lanes > 4) v = plus_lane<0x141>(v);
    if (lanes > 8) v = plus_lane<0x140>(v);
    if (lanes > 16) v = plus_16(v);
    if (lanes > 32) v = plus_32(v);
    return v;
}

// part[row of the workgroup][channel] -> sums over the rows of a wavefront's threads of equal channels are in `v` of its first lanes; here they
// go to LDS, one row a wavefront (or a set of wavefronts that span the channels)
template <int VEC, int NS>
__device__ __forceinline__ void rows_to_lds(float (&v)[NS][VEC], int lanes, int cb, float* part, int stride, int at, int first) {
#pragma unroll
    for (int k = 0; k < NS; ++k) sum_over_rows<VEC>(v[k], lanes);
    const int row = (int)threadIdx.x / (lanes > OP_WAVE ? lanes : OP_WAVE);
    if (((int)threadIdx.x & (OP_WAVE - 1)) < lanes)
#pragma unroll
        for (int k = 0; k < NS; ++k)
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (i >= first) part[k * stride + row * cb + at + i] = v[k][i];
}

// sums over the rows of part and a group's channels, by as many lanes a group as it has channels (up to 64): f(group, sum) once for each
template <int THREADS, typename F>
__device__ __forceinline__ void groups_of_rows(const float* part, int rows, int cb, int cg, F&& f) {
    int per = 1;
    while (per < cg && per < OP_WAVE) per <<= 1;
    const int ng = cb / cg, at = (int)threadIdx.x & (per - 1);
    for (int g = (int)threadIdx.x / per; g < ng; g += THREADS / per) {
        float s = 0.0f;
        for (int r = 0; r < rows; ++r)
            for (int c = at; c < cg; c += per) s += part[r * cb + g * cg + c];
        s = sum_of_neighbours(s, per);  // (lanes without a group come in whole sets of `per`)
        if (at == 0) f(g, s);
    }
}

template <typename TX, typename TY, int VEC, int P, int THREADS>
__global__ __launch_bounds__(THREADS) void held_kernel(rrm_norm_desc d, HeldGeom h, unsigned from, const TX* __restrict__ x, const float* __restrict__ gamma,
                                                       const float* __restrict__ beta, TY* __restrict__ y, float* __restrict__ stats) {
    __shared__ float part[THREADS * VEC];
    __shared__ float gs[2][HELD_GROUPS];
    int sample, block;
    if (!held_place(from + blockIdx.x, d.n, h.blocks, sample, block)) return;
    const int cg = d.c / d.groups, c0 = block * h.cb, cb = d.c - c0 < h.cb ? d.c - c0 : h.cb;
    const int slot = (int)threadIdx.x & (h.lanes - 1), row = (int)threadIdx.x / h.lanes, R = THREADS / h.lanes;
    const int rows = THREADS / (h.lanes > OP_WAVE ? h.lanes : OP_WAVE);  // of part
    const Span<VEC> me(slot, c0, cb);
    const int c = me.at;
    const TX* xs = x + sample * d.x_sample + c;
    Held<TX, VEC> v[P];
#pragma unroll
    for (int j = 0; j < P; ++j) {
        const int pos = row + j * R < d.positions ? row + j * R : d.positions - 1;  // (not under a condition: all loads are on their way at once)
        v[j].load(xs + pos * d.x_position);
    }
    float ga[VEC], be[VEC], mean[VEC], s[1][VEC];
    int gi[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        ga[i] = gamma ? gamma[c + i] : 1.0f;
        be[i] = beta ? beta[c + i] : 0.0f;
        gi[i] = i < me.keep ? 0 : (int)(((float)(c - c0 + i) + 0.5f) * h.r_cg);
        s[0][i] = 0.0f;
    }
#pragma unroll
    for (int j = 0; j < P; ++j)
        if (row + j * R < d.positions)
#pragma unroll
            for (int i = 0; i < VEC; ++i) s[0][i] += v[j].get(i);
    rows_to_lds<VEC, 1>(s, h.lanes, cb, part, 0, c - c0, me.first);
    __syncthreads();
    const float inv = 1.0f / ((float)d.positions * (float)cg);
    float* st = stats ? stats + 2 * ((int64_t)sample * d.groups + c0 / cg) : nullptr;
    groups_of_rows<THREADS>(part, rows, cb, cg, [&](int g, float sum) {
        gs[0][g] = sum * inv;
        if (st) st[2 * g] = sum * inv;
    });
    __syncthreads();
#pragma unroll
    for (int i = 0; i < VEC; ++i) mean[i] = gs[0][gi[i]], s[0][i] = 0.0f;
#pragma unroll
    for (int j = 0; j < P; ++j) {
        if (row + j * R < d.positions)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float t = v[j].get(i) - mean[i];
                s[0][i] += t * t;
            }
    }
    rows_to_lds<VEC, 1>(s, h.lanes, cb, part, 0, c - c0, me.first);
    __syncthreads();
    groups_of_rows<THREADS>(part, rows, cb, cg, [&](int g, float sum) {
        const float r = 1.0f / sqrtf(sum * inv + d.eps);
        gs[1][g] = r;
        if (st) st[2 * g + 1] = r;
    });
    __syncthreads();
    if (me.first == VEC) return;
#pragma unroll
    for (int i = 0; i < VEC; ++i) ga[i] *= gs[1][gi[i]];
    TY* ys = y + sample * d.y_sample + c;
    with_act(d.act, [&](auto act) {
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const int pos = row + j * R;
            if (pos >= d.positions) continue;
            float o[VEC];
#pragma unroll  // (the mean comes off first: a constant gives beta, whatever eps)
            for (int i = 0; i < VEC; ++i) o[i] = act_value<decltype(act)::value>((v[j].get(i) - mean[i]) * ga[i] + be[i]);
            store_some<VEC>(ys + pos * d.y_position, o, me.keep);
        }
    });
}

// sum1, sum2: [n][c], the samples' sums of dz and of dz * xh.  KEEP: dz stays in registers as well, else its slope is made twice
template <typename TX, typename TY, int VEC, int P, int THREADS, bool KEEP>
__global__ __launch_bounds__(THREADS) void held_back_kernel(rrm_norm_desc d, HeldGeom h, unsigned from, const TX* __restrict__ x, const float* __restrict__ stats,
                                                            const float* __restrict__ gamma, const float* __restrict__ beta,
                                                            const TY* __restrict__ dy, TX* __restrict__ dx, float* __restrict__ sum1,
                                                            float* __restrict__ sum2) {
    __shared__ float part[2 * THREADS * VEC];
    __shared__ float gs[2][HELD_GROUPS];
    int sample, block;
    if (!held_place(from + blockIdx.x, d.n, h.blocks, sample, block)) return;
    const int cg = d.c / d.groups, c0 = block * h.cb, cb = d.c - c0 < h.cb ? d.c - c0 : h.cb;
    const int slot = (int)threadIdx.x & (h.lanes - 1), row = (int)threadIdx.x / h.lanes, R = THREADS / h.lanes;
    const int rows = THREADS / (h.lanes > OP_WAVE ? h.lanes : OP_WAVE);
    const Span<VEC> me(slot, c0, cb);
    const int c = me.at;
    const TX* xs = x + sample * d.x_sample + c;
    const TY* dys = dy + sample * d.y_sample + c;
    Held<TX, VEC> v[P];
    Held<TY, VEC> w[P];
#pragma unroll
    for (int j = 0; j < P; ++j) {
        const int pos = row + j * R < d.positions ? row + j * R : d.positions - 1;
        v[j].load(xs + pos * d.x_position);
        w[j].load(dys + pos * d.y_position);
    }
    const float* st = stats + 2 * ((int64_t)sample * d.groups + c0 / cg);
    float ga[VEC], be[VEC], mean[VEC], r[VEC], s[2][VEC];
    int gi[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        ga[i] = gamma ? gamma[c + i] : 1.0f;
        be[i] = beta ? beta[c + i] : 0.0f;
        gi[i] = i < me.keep ? 0 : (int)(((float)(c - c0 + i) + 0.5f) * h.r_cg);
        mean[i] = st[2 * gi[i]];
        r[i] = st[2 * gi[i] + 1];
        s[0][i] = s[1][i] = 0.0f;
    }
    float kept[KEEP ? P : 1][VEC];
    with_act(d.act, [&](auto act) {
#pragma unroll
        for (int j = 0; j < P; ++j) {
            if (row + j * R >= d.positions) continue;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float xh = (v[j].get(i) - mean[i]) * r[i];
                float value, slope;
                act_pair<decltype(act)::value>(ga[i] * xh + be[i], value, slope);
                const float dz = w[j].get(i) * slope;
                if (KEEP) kept[KEEP ? j : 0][i] = dz;
                s[0][i] += dz;
                s[1][i] += dz * xh;
            }
        }
    });
    constexpr int STRIDE = THREADS * VEC;
    rows_to_lds<VEC, 2>(s, h.lanes, cb, part, STRIDE, c - c0, me.first);
    __syncthreads();
    // the channels' sums leave for dgamma and dbeta, and, times gamma, become the first row
    for (int ch = threadIdx.x; ch < cb; ch += THREADS) {
        float s1 = 0.0f, s2 = 0.0f;
        for (int k = 0; k < rows; ++k) s1 += part[k * cb + ch], s2 += part[STRIDE + k * cb + ch];
        sum1[(int64_t)sample * d.c + c0 + ch] = s1;
        sum2[(int64_t)sample * d.c + c0 + ch] = s2;
        const float g = gamma ? gamma[c0 + ch] : 1.0f;
        part[ch] = g * s1;
        part[STRIDE + ch] = g * s2;
    }
    if (!dx) return;
    __syncthreads();
    const float inv = 1.0f / ((float)d.positions * (float)cg);
    groups_of_rows<THREADS>(part, 1, cb, cg, [&](int g, float sum) { gs[0][g] = sum * inv; });
    groups_of_rows<THREADS>(part + STRIDE, 1, cb, cg, [&](int g, float sum) { gs[1][g] = sum * inv; });
    __syncthreads();
    if (me.first == VEC) return;
    TX* dxs = dx + sample * d.dx_sample + c;
    float gp[VEC], gq[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) gp[i] = gs[0][gi[i]], gq[i] = gs[1][gi[i]];
    auto leave = [&](int j, auto dz_of) __attribute__((always_inline)) {
        const int pos = row + j * R;
        if (pos >= d.positions) return;
        float o[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const float xh = (v[j].get(i) - mean[i]) * r[i];
            o[i] = r[i] * (ga[i] * dz_of(i, xh) - gp[i] - xh * gq[i]);
        }
        store_some<VEC>(dxs + pos * d.dx_position, o, me.keep);
    };
    if constexpr (KEEP) {
#pragma unroll
        for (int j = 0; j < P; ++j) leave(j, [&](int i, float) { return kept[KEEP ? j : 0][i]; });
    } else {
        with_act(d.act, [&](auto act) {
#pragma unroll
            for (int j = 0; j < P; ++j)
                leave(j, [&](int i, float xh) {
                    float value, slope;
                    act_pair<decltype(act)::value>(ga[i] * xh + be[i], value, slope);
                    return w[j].get(i) * slope;
                });
        });
    }
}

// ---- samples that registers do not hold ----------------------------------------------------------------------------------
//
// Slices of a sample's positions: their channels' means and squares (backward: sums of dz and dz * xh), a joining of slices and channels for
// each group, and a second pass over x (and dy).
struct SliceGeom {
    int slices, span;   // of a sample; positions of a slice
    int blocks, lanes;  // sets of channels; threads of a position, a power of two
};
constexpr int SLICE_THREADS = 256;

// what a thread of a slice's workgroup has: its channels and rows
template <int VEC>
struct Slice {
    int sample, slice, row, step, p0, p1;
    Span<VEC> me;
    __device__ __forceinline__ Slice(const rrm_norm_desc& d, const SliceGeom& g)
        : sample((int)(blockIdx.x / (unsigned)(g.slices * g.blocks))),
          slice((int)(blockIdx.x / (unsigned)g.blocks) % g.slices),
          row((int)threadIdx.x / g.lanes),
          step(SLICE_THREADS / g.lanes),
          p0(slice * g.span),
          p1(d.positions - p0 > g.span ? p0 + g.span : d.positions),
          me((int)threadIdx.x & (g.lanes - 1), (int)(blockIdx.x % (unsigned)g.blocks) * g.lanes * VEC,
             min(d.c - (int)(blockIdx.x % (unsigned)g.blocks) * g.lanes * VEC, g.lanes * VEC)) {}
};

// The groups of VEC neighbouring channels from c on, by integers: beyond some millions of channels a quotient in 32-bit floats is a group off.
template <int VEC>
__device__ __forceinline__ void groups_from(int c, int cg, int (&gi)[VEC]) {
    int g = c / cg, left = (g + 1) * cg - c;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        gi[i] = g;
        if (--left == 0) ++g, left = cg;
    }
}

// sums over the workgroup's rows, to the first row's threads (lanes <= 256, any number of rows)
template <int VEC, int NS>
__device__ __forceinline__ void sum_rows(float (&v)[NS][VEC], int lanes, float* lds) {
    for (int half = SLICE_THREADS / 2; half >= lanes; half >>= 1) {
        __syncthreads();
        if ((int)threadIdx.x >= half && (int)threadIdx.x < 2 * half)
#pragma unroll
            for (int k = 0; k < NS; ++k)
#pragma unroll
                for (int i = 0; i < VEC; ++i) lds[(k * VEC + i) * SLICE_THREADS / 2 + (int)threadIdx.x - half] = v[k][i];
        __syncthreads();
        if ((int)threadIdx.x < half)
#pragma unroll
            for (int k = 0; k < NS; ++k)
#pragma unroll
                for (int i = 0; i < VEC; ++i) v[k][i] += lds[(k * VEC + i) * SLICE_THREADS / 2 + (int)threadIdx.x];
    }
}

// part: [n][slices][2][c], mean and sum of squares about it of each channel of a slice.  Values are taken less the slice's first: the sums lose
// nothing to a mean far from zero.
template <typename TX, int VEC>
__global__ __launch_bounds__(SLICE_THREADS) void slice_stats_kernel(rrm_norm_desc d, SliceGeom g, const TX* __restrict__ x, float* __restrict__ part) {
    __shared__ float lds[VEC * SLICE_THREADS / 2];
    __shared__ float first_mean[SLICE_THREADS * VEC];
    const Slice<VEC> t(d, g);
    const TX* xs = x + t.sample * d.x_sample + t.me.at;
    const int lane = (int)threadIdx.x & (g.lanes - 1);
    float s[1][VEC], v[VEC], base[VEC];
    load_vec<VEC>(xs + t.p0 * d.x_position, base);
#pragma unroll
    for (int i = 0; i < VEC; ++i) s[0][i] = 0.0f;
#pragma unroll 4
    for (int p = t.p0 + t.row; p < t.p1; p += t.step) {
        load_vec<VEC>(xs + p * d.x_position, v);
#pragma unroll
        for (int i = 0; i < VEC; ++i) s[0][i] += v[i] - base[i];
    }
    sum_rows<VEC, 1>(s, g.lanes, lds);
    const float inv = 1.0f / (float)(t.p1 - t.p0);
    if (t.row == 0)
#pragma unroll
        for (int i = 0; i < VEC; ++i) first_mean[lane * VEC + i] = base[i] + s[0][i] * inv;
    __syncthreads();
    float mean[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) mean[i] = first_mean[lane * VEC + i], s[0][i] = 0.0f;
    // (the slice again: out of the caches where it is some tens of kilobytes; there are some 1025 slices at the most, so those of a sample beyond the 256 MB of
    // the last cache come from memory twice)
#pragma unroll 4
    for (int p = t.p0 + t.row; p < t.p1; p += t.step) {
        load_vec<VEC>(xs + p * d.x_position, v);
#pragma unroll
        for (int i = 0; i < VEC; ++i) s[0][i] += (v[i] - mean[i]) * (v[i] - mean[i]);
    }
    sum_rows<VEC, 1>(s, g.lanes, lds);
    if (t.row != 0) return;
    float* to = part + ((int64_t)t.sample * g.slices + t.slice) * 2 * d.c + t.me.at;
#pragma unroll
    for (int i = 0; i < VEC; ++i)
        if (i >= t.me.first) to[i] = mean[i], to[d.c + i] = s[0][i];
}

constexpr int JOIN_THREADS = 512;
__device__ __forceinline__ float sum_all(float v, float* lds) {
    v = sum_of_neighbours(v, OP_WAVE);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < JOIN_THREADS / OP_WAVE; ++i) s += lds[i];
    return s;
}
// a group's channels over a workgroup's threads: `lanes` of them (a power of two), rows of slices behind
struct JoinShape {
    int lane, row, lanes, rows;
    __device__ __forceinline__ explicit JoinShape(int cg) {
        lanes = 1;
        while (lanes < cg && lanes < JOIN_THREADS) lanes <<= 1;
        rows = JOIN_THREADS / lanes;
        lane = (int)threadIdx.x & (lanes - 1);
        row = (int)threadIdx.x / lanes;
    }
};

// One workgroup a group of a sample: the slices' and channels' means and squares become the group's
__global__ __launch_bounds__(JOIN_THREADS) void join_stats_kernel(rrm_norm_desc d, SliceGeom g, unsigned first, const float* __restrict__ part, float* __restrict__ stats) {
    __shared__ float lds[JOIN_THREADS / OP_WAVE];
    const int cg = d.c / d.groups, id = (int)(first + blockIdx.x), sample = id / d.groups, group = id % d.groups;
    const float* from = part + (int64_t)sample * g.slices * 2 * d.c + group * cg;
    const JoinShape j(cg);
    const float per = 1.0f / ((float)d.positions * (float)cg);
    const float whole = (float)g.span, last = (float)(d.positions - (g.slices - 1) * g.span);
    float m = 0.0f;
    for (int c = j.lane; c < cg; c += j.lanes)
#pragma unroll 4
        for (int k = j.row; k < g.slices; k += j.rows) m += from[(int64_t)k * 2 * d.c + c] * (k + 1 < g.slices ? whole : last);
    const float mean = sum_all(m, lds) * per;
    float q = 0.0f;
    for (int c = j.lane; c < cg; c += j.lanes)
#pragma unroll 4
        for (int k = j.row; k < g.slices; k += j.rows) {
            const float* e = from + (int64_t)k * 2 * d.c + c;
            const float off = e[0] - mean;
            q += e[d.c] + off * off * (k + 1 < g.slices ? whole : last);
        }
    const float r = 1.0f / sqrtf(sum_all(q, lds) * per + d.eps);
    if (threadIdx.x == 0) stats[2 * (int64_t)id] = mean, stats[2 * (int64_t)id + 1] = r;
}

template <typename TX, typename TY, int VEC>
__global__ __launch_bounds__(SLICE_THREADS) void slice_apply_kernel(rrm_norm_desc d, SliceGeom g, const TX* __restrict__ x, const float* __restrict__ gamma,
                                                                    const float* __restrict__ beta, const float* __restrict__ stats, TY* __restrict__ y) {
    const Slice<VEC> t(d, g);
    if (t.me.first == VEC) return;
    const TX* xs = x + t.sample * d.x_sample + t.me.at;
    TY* ys = y + t.sample * d.y_sample + t.me.at;
    const float* st = stats + 2 * (int64_t)t.sample * d.groups;
    float ga[VEC], be[VEC], mean[VEC];
    int gi[VEC];
    groups_from<VEC>(t.me.at, d.c / d.groups, gi);
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const int c = t.me.at + i;
        mean[i] = st[2 * gi[i]];
        ga[i] = (gamma ? gamma[c] : 1.0f) * st[2 * gi[i] + 1];
        be[i] = beta ? beta[c] : 0.0f;
    }
    with_act(d.act, [&](auto act) {
#pragma unroll 4
        for (int p = t.p0 + t.row; p < t.p1; p += t.step) {
            float v[VEC];
            load_vec<VEC>(xs + p * d.x_position, v);
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] = act_value<decltype(act)::value>((v[i] - mean[i]) * ga[i] + be[i]);
            store_vec<VEC>(ys + p * d.y_position, v);  // (channels of the workgroup before too: the same bits)
        }
    });
}

// part: [2][n * slices][c], the slices' sums of dz and dz * xh
template <typename TX, typename TY, int VEC>
__global__ __launch_bounds__(SLICE_THREADS) void slice_sums_kernel(rrm_norm_desc d, SliceGeom g, const TX* __restrict__ x, const float* __restrict__ stats,
                                                                   const float* __restrict__ gamma, const float* __restrict__ beta,
                                                                   const TY* __restrict__ dy, float* __restrict__ part) {
    __shared__ float lds[2 * VEC * SLICE_THREADS / 2];
    const Slice<VEC> t(d, g);
    const TX* xs = x + t.sample * d.x_sample + t.me.at;
    const TY* dys = dy + t.sample * d.y_sample + t.me.at;
    const float* st = stats + 2 * (int64_t)t.sample * d.groups;
    float ga[VEC], be[VEC], mean[VEC], r[VEC], s[2][VEC];
    int gi[VEC];
    groups_from<VEC>(t.me.at, d.c / d.groups, gi);
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const int c = t.me.at + i;
        mean[i] = st[2 * gi[i]];
        r[i] = st[2 * gi[i] + 1];
        ga[i] = gamma ? gamma[c] : 1.0f;
        be[i] = beta ? beta[c] : 0.0f;
        s[0][i] = s[1][i] = 0.0f;
    }
    with_act(d.act, [&](auto act) {
#pragma unroll 2
        for (int p = t.p0 + t.row; p < t.p1; p += t.step) {
            float v[VEC], w[VEC];
            load_vec<VEC>(xs + p * d.x_position, v);
            load_vec<VEC>(dys + p * d.y_position, w);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float xh = (v[i] - mean[i]) * r[i];
                float value, slope;
                act_pair<decltype(act)::value>(ga[i] * xh + be[i], value, slope);
                s[0][i] += w[i] * slope;
                s[1][i] += w[i] * slope * xh;
            }
        }
    });
    sum_rows<VEC, 2>(s, g.lanes, lds);
    if (t.row != 0) return;
    const int64_t k = (int64_t)t.sample * g.slices + t.slice, rows = (int64_t)d.n * g.slices;
#pragma unroll
    for (int i = 0; i < VEC; ++i)
        if (i >= t.me.first) part[k * d.c + t.me.at + i] = s[0][i], part[(rows + k) * d.c + t.me.at + i] = s[1][i];
}

// One workgroup a group of a sample: the slices' sums of each channel, sum1 and sum2 [n][c], and the group's means of gamma dz and of gamma dz xh, [n][groups][2]
__global__ __launch_bounds__(JOIN_THREADS) void join_sums_kernel(rrm_norm_desc d, SliceGeom g, unsigned first, const float* __restrict__ part, const float* __restrict__ gamma,
                                                                 float* __restrict__ sum1, float* __restrict__ sum2, float* __restrict__ means) {
    __shared__ float lds[JOIN_THREADS / OP_WAVE], rows[2][JOIN_THREADS];
    const int cg = d.c / d.groups, id = (int)(first + blockIdx.x), sample = id / d.groups, group = id % d.groups;
    const JoinShape j(cg);
    const int64_t all = (int64_t)d.n * g.slices;
    float p = 0.0f, q = 0.0f;
    for (int c0 = 0; c0 < cg; c0 += j.lanes) {
        const int c = group * cg + c0 + j.lane;
        const bool in = c0 + j.lane < cg;
        float s1 = 0.0f, s2 = 0.0f;
        if (in)
#pragma unroll 4
            for (int k = j.row; k < g.slices; k += j.rows) {
                const int64_t row = (int64_t)sample * g.slices + k;
                s1 += part[row * d.c + c];
                s2 += part[(all + row) * d.c + c];
            }
        __syncthreads();
        rows[0][threadIdx.x] = s1;
        rows[1][threadIdx.x] = s2;
        __syncthreads();
        if (j.row == 0 && in) {
            s1 = s2 = 0.0f;
            for (int k = 0; k < j.rows; ++k) s1 += rows[0][k * j.lanes + j.lane], s2 += rows[1][k * j.lanes + j.lane];
            sum1[(int64_t)sample * d.c + c] = s1;
            sum2[(int64_t)sample * d.c + c] = s2;
            const float ga = gamma ? gamma[c] : 1.0f;
            p += ga * s1;
            q += ga * s2;
        }
    }
    const float per = 1.0f / ((float)d.positions * (float)cg);
    p = sum_all(p, lds) * per;
    q = sum_all(q, lds) * per;
    if (threadIdx.x == 0) means[2 * (int64_t)id] = p, means[2 * (int64_t)id + 1] = q;
}

template <typename TX, typename TY, int VEC>
__global__ __launch_bounds__(SLICE_THREADS) void slice_dx_kernel(rrm_norm_desc d, SliceGeom g, const TX* __restrict__ x, const float* __restrict__ stats,
                                                                 const float* __restrict__ gamma, const float* __restrict__ beta,
                                                                 const TY* __restrict__ dy, const float* __restrict__ means, TX* __restrict__ dx) {
    const Slice<VEC> t(d, g);
    if (t.me.first == VEC) return;
    const TX* xs = x + t.sample * d.x_sample + t.me.at;
    const TY* dys = dy + t.sample * d.y_sample + t.me.at;
    TX* dxs = dx + t.sample * d.dx_sample + t.me.at;
    const float *st = stats + 2 * (int64_t)t.sample * d.groups, *me = means + 2 * (int64_t)t.sample * d.groups;
    float ga[VEC], be[VEC], mean[VEC], r[VEC], gp[VEC], gq[VEC];
    int gi[VEC];
    groups_from<VEC>(t.me.at, d.c / d.groups, gi);
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const int c = t.me.at + i;
        mean[i] = st[2 * gi[i]];
        r[i] = st[2 * gi[i] + 1];
        gp[i] = me[2 * gi[i]];
        gq[i] = me[2 * gi[i] + 1];
        ga[i] = gamma ? gamma[c] : 1.0f;
        be[i] = beta ? beta[c] : 0.0f;
    }
    with_act(d.act, [&](auto act) {
#pragma unroll 2
        for (int p = t.p0 + t.row; p < t.p1; p += t.step) {
            float v[VEC], w[VEC];
            load_vec<VEC>(xs + p * d.x_position, v);
            load_vec<VEC>(dys + p * d.y_position, w);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float xh = (v[i] - mean[i]) * r[i];
                float value, slope;
                act_pair<decltype(act)::value>(ga[i] * xh + be[i], value, slope);
                v[i] = r[i] * (ga[i] * (w[i] * slope) - gp[i] - xh * gq[i]);
            }
            store_vec<VEC>(dxs + p * d.dx_position, v);
        }
    });
}

// dbeta and dgamma: the samples' sums (no samples: zeros).  32 channels a workgroup, 32 threads a channel, joined in their order.
__global__ __launch_bounds__(1024) void norm_params_kernel(const float* __restrict__ sum1, const float* __restrict__ sum2, int n, int c,
                                                           unsigned first, float* __restrict__ dgamma, float* __restrict__ dbeta) {
    __shared__ float lds[2][32][32];
    const int ch = (int)(first + blockIdx.x) * 32 + ((int)threadIdx.x & 31), k = (int)threadIdx.x >> 5;
    float s1 = 0.0f, s2 = 0.0f;
    if (ch < c)
#pragma unroll 4
        for (int i = k; i < n; i += 32) {
            s1 += sum1[(int64_t)i * c + ch];
            s2 += sum2[(int64_t)i * c + ch];
        }
    lds[0][k][threadIdx.x & 31] = s1;
    lds[1][k][threadIdx.x & 31] = s2;
    __syncthreads();
    if (k > 1 || ch >= c) return;
    float s = 0.0f;
#pragma unroll 8
    for (int i = 0; i < 32; ++i) s += lds[k][i][threadIdx.x & 31];
    if (k == 0 && dbeta) dbeta[ch] = s;
    if (k == 1 && dgamma) dgamma[ch] = s;
}

// calls f(TX, TY) with the descriptor's types
template <typename F>
void with_types(const rrm_norm_desc& d, F&& f) {
    auto out = [&](auto tx) { d.y_elem == RRM_F32 ? f(tx, float{}) : f(tx, __bf16{}); };
    d.x_elem == RRM_F32 ? out(float{}) : out(__bf16{});
}

int parts(int64_t n, int64_t of) { return (int)((n + of - 1) / of); }

struct HeldPlan {
    HeldGeom g;
    int vec, which;  // which of the shapes; -1: registers do not hold it
};
struct HeldShape {
    int threads, p;
};
// (64 x 28 x 28 x 128 bf16 in 1024 threads of four and two vectors instead of 512 of eight: 15.2 and 23 us, 13.7 and 18 so)
constexpr int HELD_SHAPES = 4;
constexpr HeldShape FORWARD[] = {{256, 1}, {256, 4}, {512, 8}, {1024, 16}};
constexpr HeldShape BACKWARD[] = {{256, 1}, {256, 4}, {512, 8}, {1024, 8}};

// The held form's shape: the smallest that holds the sample's positions.  Runs of a position are 64 bytes at least (what memory hands out)
// where that fits, and more where there are workgroups enough.  It goes by sizes alone: strides and alignment do not change a result's bits.
HeldPlan plan_held(const rrm_norm_desc& d, int wide, const HeldShape (&shapes)[HELD_SHAPES]) {
    const int cg = d.c / d.groups, esize = d.x_elem == RRM_F32 ? 4 : 2;
    HeldPlan p{{}, d.c >= wide ? wide : 1, -1};
    if (cg > shapes[HELD_SHAPES - 1].threads * p.vec) return p;  // (what is below counts in multiples of cg)
    auto fits = [&](int channels) {
        p.which = -1;
        int lanes = 1;
        while (lanes * p.vec < channels) lanes <<= 1;
        if (channels / cg > HELD_GROUPS) return false;
        for (int w = 0; w < HELD_SHAPES; ++w) {
            if (lanes > shapes[w].threads || (int64_t)shapes[w].threads / lanes * shapes[w].p < d.positions) continue;
            p.which = w;
            p.g = HeldGeom{channels, parts(d.c, channels), lanes, 1.0f / (float)cg};
            return true;
        }
        return false;
    };
    int cb = cg;
    while (cb < d.c && (cb * esize < 64 || cb % p.vec) && cb < HELD_GROUPS * cg) cb += cg;
    // (few samples: narrower runs on more compute units, by whole vectors as far as that goes, then down to single groups; a vector at
    // least: see Span)
    int whole = cg;
    while (whole % p.vec) whole += cg;
    for (int next = cb; next >= p.vec && next > 0; next = cb - (cb - whole >= whole ? whole : cg)) {
        cb = next;
        if (fits(cb) && (int64_t)d.n * p.g.blocks >= OP_CUS) break;
    }
    if (!fits(cb)) return p;
    if ((int64_t)d.n * p.g.blocks < OP_CUS / 2 && (int64_t)cb * d.positions > HELD_FEW) {
        p.which = -1;
        return p;
    }
    while (cb < d.c && (int64_t)d.n * parts(d.c, 2 * cb) >= 4 * OP_CUS) {
        const HeldPlan before = p;
        if (!fits(2 * cb) || p.which > before.which) return before;
        cb *= 2;
    }
    return p;
}
SliceGeom plan_slices(const rrm_norm_desc& d, int vec) {
    SliceGeom g{};
    g.lanes = 1;
    while (g.lanes < SLICE_THREADS && g.lanes * vec < d.c) g.lanes <<= 1;
    g.blocks = parts(d.c, g.lanes * vec);
    const int rows = SLICE_THREADS / g.lanes;
    // some four workgroups a compute unit, of four rows of positions at least
    int64_t want = 4 * OP_CUS / ((int64_t)d.n * g.blocks) + 1, most = parts(d.positions, 4 * rows);
    if (want > most) want = most;
    g.span = parts(d.positions, want);
    g.slices = parts(d.positions, g.span);
    return g;
}
int wide_of(const rrm_norm_desc& d) { return d.x_elem == RRM_F32 ? 4 : 8; }
int slice_vec(const rrm_norm_desc& d) { return d.c >= wide_of(d) ? wide_of(d) : 1; }
HeldPlan plan_held(const rrm_norm_desc& d, bool backward) { return plan_held(d, wide_of(d), backward ? BACKWARD : FORWARD); }
size_t group_bytes(const rrm_norm_desc& d) { return round256((size_t)d.n * d.groups * 8); }

int64_t held_grid(const rrm_norm_desc& d, const HeldPlan& p) { return (int64_t)parts(d.n, 8) * 8 * p.g.blocks; }

}  // namespace

// backward, held: the samples' sums [2][n][c]; else the slices' sums, (backward) the samples' and the groups' two values
size_t norm_scratch(const rrm_norm_desc& d, bool backward) {
    if (plan_held(d, backward).which >= 0) return backward ? round256((size_t)2 * d.n * d.c * 4) : 0;
    return round256((size_t)2 * d.n * plan_slices(d, slice_vec(d)).slices * d.c * 4) + (backward ? round256((size_t)2 * d.n * d.c * 4) : 0) + group_bytes(d);
}

void norm_layout(const rrm_norm_desc& d, bool backward, int* layout) {
    const HeldPlan p = plan_held(d, backward);
    layout[0] = p.which;
    layout[1] = p.which >= 0 ? p.g.cb : plan_slices(d, slice_vec(d)).slices;
}

hipError_t launch_group_norm(const rrm_norm_desc& d, const void* x, const float* gamma, const float* beta, void* y, float* stats,
                             void* ws, hipStream_t s) {
    with_types(d, [&](auto tx, auto ty) {
        using TX = decltype(tx);
        using TY = decltype(ty);
        constexpr int WIDE = 16 / sizeof(TX);
        const HeldPlan p = plan_held(d, WIDE, FORWARD);
        auto go = [&](auto vec, auto which) {
            constexpr HeldShape h = FORWARD[decltype(which)::value];
            in_parts(held_grid(d, p), [&](unsigned from, unsigned count) {
                hipLaunchKernelGGL((held_kernel<TX, TY, decltype(vec)::value, h.p, h.threads>), dim3(count), dim3(h.threads), 0, s, d, p.g, from,
                                   (const TX*)x, gamma, beta, (TY*)y, stats);
            });
        };
        auto by_vec = [&](auto vec) {
            constexpr int VEC = decltype(vec)::value;
            switch (p.which) {
                case 0: go(vec, std::integral_constant<int, 0>{}); break;
                case 1: go(vec, std::integral_constant<int, 1>{}); break;
                case 2: go(vec, std::integral_constant<int, 2>{}); break;
                case 3: go(vec, std::integral_constant<int, 3>{}); break;
                default: {
                    const SliceGeom g = plan_slices(d, VEC);
                    const dim3 grid((unsigned)((int64_t)d.n * g.slices * g.blocks));
                    float* st = stats ? stats : (float*)((char*)ws + round256((size_t)2 * d.n * g.slices * d.c * 4));
                    hipLaunchKernelGGL((slice_stats_kernel<TX, VEC>), grid, dim3(SLICE_THREADS), 0, s, d, g, (const TX*)x, (float*)ws);
                    in_parts((int64_t)d.n * d.groups, [&](unsigned from, unsigned count) {
                        hipLaunchKernelGGL(join_stats_kernel, dim3(count), dim3(JOIN_THREADS), 0, s, d, g, from, (const float*)ws, st);
                    });
                    hipLaunchKernelGGL((slice_apply_kernel<TX, TY, VEC>), grid, dim3(SLICE_THREADS), 0, s, d, g, (const TX*)x, gamma, beta, st, (TY*)y);
                }
            }
        };
        p.vec == 1 ? by_vec(std::integral_constant<int, 1>{}) : by_vec(std::integral_constant<int, WIDE>{});
    });
    return hipGetLastError();
}

hipError_t launch_group_norm_backward(const rrm_norm_desc& d, const void* x, const float* stats, const float* gamma,
                                      const float* beta, const void* dy, void* dx, float* dgamma, float* dbeta, void* ws,
                                      hipStream_t s) {
    const bool some = d.n > 0 && d.positions > 0;
    // [n][c] each; of one sample they are the parameters' gradients
    const bool one = some && d.n == 1;
    float *sum1 = (float*)ws, *sum2 = nullptr;
    auto place_sums = [&](float* at) {
        sum1 = one && dbeta ? dbeta : at;
        sum2 = one && dgamma ? dgamma : at + (size_t)d.n * d.c;
    };
    if (some)
        with_types(d, [&](auto tx, auto ty) {
            using TX = decltype(tx);
            using TY = decltype(ty);
            constexpr int WIDE = 16 / sizeof(TX);
            const HeldPlan p = plan_held(d, WIDE, BACKWARD);
            auto go = [&](auto vec, auto which) {
                constexpr HeldShape h = BACKWARD[decltype(which)::value];
                // (bfloat16, the largest: there are no registers for dz in 32 bits)
                constexpr bool KEEP = sizeof(TX) == 4 || h.threads < 1024;
                place_sums((float*)ws);
                in_parts(held_grid(d, p), [&](unsigned from, unsigned count) {
                    hipLaunchKernelGGL((held_back_kernel<TX, TY, decltype(vec)::value, h.p, h.threads, KEEP>), dim3(count), dim3(h.threads),
                                       0, s, d, p.g, from, (const TX*)x, stats, gamma, beta, (const TY*)dy, (TX*)dx, sum1, sum2);
                });
            };
            auto by_vec = [&](auto vec) {
                constexpr int VEC = decltype(vec)::value;
                switch (p.which) {
                    case 0: go(vec, std::integral_constant<int, 0>{}); break;
                    case 1: go(vec, std::integral_constant<int, 1>{}); break;
                    case 2: go(vec, std::integral_constant<int, 2>{}); break;
                    case 3: go(vec, std::integral_constant<int, 3>{}); break;
                    default: {
                        const SliceGeom g = plan_slices(d, VEC);
                        const dim3 grid((unsigned)((int64_t)d.n * g.slices * g.blocks));
                        float* to = (float*)((char*)ws + round256((size_t)2 * d.n * g.slices * d.c * 4));
                        float* means = (float*)((char*)to + round256((size_t)2 * d.n * d.c * 4));
                        place_sums(to);
                        hipLaunchKernelGGL((slice_sums_kernel<TX, TY, VEC>), grid, dim3(SLICE_THREADS), 0, s, d, g, (const TX*)x, stats, gamma, beta,
                                           (const TY*)dy, (float*)ws);
                        in_parts((int64_t)d.n * d.groups, [&](unsigned from, unsigned count) {
                            hipLaunchKernelGGL(join_sums_kernel, dim3(count), dim3(JOIN_THREADS), 0, s, d, g, from, (const float*)ws, gamma, sum1, sum2, means);
                        });
                        if (!dx) break;
                        hipLaunchKernelGGL((slice_dx_kernel<TX, TY, VEC>), grid, dim3(SLICE_THREADS), 0, s, d, g, (const TX*)x, stats, gamma, beta,
                                           (const TY*)dy, means, (TX*)dx);
                    }
                }
            };
            p.vec == 1 ? by_vec(std::integral_constant<int, 1>{}) : by_vec(std::integral_constant<int, WIDE>{});
        });
    if (hipError_t e = hipGetLastError()) return e;
    if ((dgamma || dbeta) && !one)
        in_parts(parts(d.c, 32), [&](unsigned from, unsigned count) {
            hipLaunchKernelGGL(norm_params_kernel, dim3(count), dim3(1024), 0, s, sum1, sum2, some ? d.n : 0, d.c, from, dgamma, dbeta);
        });
    return hipGetLastError();
}

}  // namespace rrm
