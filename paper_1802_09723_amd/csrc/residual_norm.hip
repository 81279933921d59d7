// What stands between two blocks of a residual network: the norm behind the one, its gate, the residual scale and sum, the norm before the next; and
// the backward pass.  Over a row of c features:
//
//      p = b rb post, rb = 1 / sqrt(mean(b^2) + eps)        r = x + scale sigmoid(gate) p        u = r rr pre, rr = 1 / sqrt(mean(r^2) + eps)
//
//      rh = r rr, bh = b rb, w = du pre:   dx = dr + rr (w - rh mean(w rh))      dgate = dx scale p sg (1 - sg)
//      dp = dx scale sg:                   db = rb (dp post - bh mean(dp post bh))
//      dpre = sum du rh        dscale = sum dx sg p        dpost = sum dp bh        (sums over the rows)
//
// Memory is what bounds both: a row is read once into registers and everything is made of it there.  The backward pass makes r again from x and b, which
// is as many bytes as reading a stored r, and r in 32 bits.
#include "op_common.h"

namespace rrm {

namespace {

constexpr int VEC = 8;  // neighbouring features of a thread

// up to VEC elements, zeros behind the row's end
template <typename T>
__device__ __forceinline__ void load_part(const T* p, int have, float (&v)[VEC]) {
    if (have >= VEC) {
        load_vec<VEC>(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = i < have ? load_elem(p + i) : 0.0f;
    }
}
template <typename T>
__device__ __forceinline__ void store_part(T* p, int have, const float (&v)[VEC]) {
    if (have >= VEC) {
        store_vec<VEC>(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (i < have) store_elem(p + i, v[i]);
    }
}

// Sums over the TPR threads of a row, N at once, in one order; `place`: LDS for [2][N][waves], `turn` flips between calls
template <int TPR, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* place, int& turn) {
#pragma unroll
    for (int m = 1; m < (TPR < 64 ? TPR : 64); m <<= 1)
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += __shfl_xor(v[k], m);
    if constexpr (TPR > 64) {
        constexpr int WAVES = TPR / 64;
        float* mine = place + turn * N * WAVES;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) mine[k * WAVES + (threadIdx.x >> 6)] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < WAVES; ++i) s += mine[k * WAVES + i];
            v[k] = s;
        }
        turn ^= 1;  // (the other half may still be read)
    }
}

// TPR threads hold a row, ITER vectors each; THREADS / TPR rows a workgroup at a time.
template <typename X, typename B, int TPR, int ITER, int THREADS>
__global__ __launch_bounds__(THREADS) void residual_kernel(rrm_residual_desc d, const X* x, const B* b, const B* gate, const float* scale, const float* post,
                                                           const float* pre, X* r, B* u, float* stats) {
    __shared__ float place[2 * 16];
    constexpr int RPW = THREADS / TPR;
    const int t = (int)threadIdx.x % TPR;
    const float inv = 1.0f / d.c;
    int turn = 0;
    for (int64_t row0 = (int64_t)blockIdx.x * RPW; row0 < d.m; row0 += (int64_t)gridDim.x * RPW) {
        const int64_t row = row0 + (int)threadIdx.x / TPR;
        const bool live = row < d.m;
        float rv[ITER][VEC], bv[ITER][VEC], gv[ITER][VEC];
        float sums[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const int c = (i * TPR + t) * VEC, have = live ? d.c - c : 0;
            load_part(x + row * d.x_row + c, have, rv[i]);
            if (b) load_part(b + row * d.b_row + c, have, bv[i]);
            if (gate) load_part(gate + row * d.gate_row + c, have, gv[i]);
        }
        float rb = 1.0f;
        if (b) {
            if (d.post_norm) {
#pragma unroll
                for (int i = 0; i < ITER; ++i)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) sums[0] += bv[i][e] * bv[i][e];
                row_sums<TPR, 1>(sums, place, turn);
                rb = 1.0f / sqrtf(sums[0] * inv + d.eps);
            }
#pragma unroll
            for (int i = 0; i < ITER; ++i) {
                const int c = (i * TPR + t) * VEC, have = live ? d.c - c : 0;
                float sv[VEC], pv[VEC];
                if (scale) load_part(scale + c, have, sv);
                if (post) load_part(post + c, have, pv);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    float p = bv[i][e] * rb;
                    if (post) p *= pv[e];
                    if (gate) p *= sigmoid(gv[i][e]);
                    if (scale) p *= sv[e];
                    if (e < have) rv[i][e] += p;
                }
                if (r) store_part(r + row * d.r_row + c, have, rv[i]);
            }
        }
        float rr = 1.0f;
        if (u) {
            sums[0] = 0.0f;
#pragma unroll
            for (int i = 0; i < ITER; ++i)
#pragma unroll
                for (int e = 0; e < VEC; ++e) sums[0] += rv[i][e] * rv[i][e];
            row_sums<TPR, 1>(sums, place, turn);
            rr = 1.0f / sqrtf(sums[0] * inv + d.eps);
#pragma unroll
            for (int i = 0; i < ITER; ++i) {
                const int c = (i * TPR + t) * VEC, have = live ? d.c - c : 0;
                float wv[VEC];
                if (pre) load_part(pre + c, have, wv);
#pragma unroll
                for (int e = 0; e < VEC; ++e) wv[e] = pre ? rv[i][e] * rr * wv[e] : rv[i][e] * rr;
                store_part(u + row * d.u_row + c, have, wv);
            }
        }
        if (stats && live && t == 0) stats[2 * row] = rb, stats[2 * row + 1] = rr;
    }
}

// Sums over rows of three kinds, a workgroup's each: part [workgroup][3][c]
template <typename X, typename B, int TPR, int ITER, int THREADS>
__global__ __launch_bounds__(THREADS) void residual_back_kernel(rrm_residual_desc d, const X* dr, const B* du, const X* x, const B* b, const float* stats,
                                                                const B* gate, const float* scale, const float* post, const float* pre, X* dx, B* db,
                                                                B* dgate, float* part) {
    constexpr int RPW = THREADS / TPR;
    __shared__ float place[2 * 3 * 16];
    __shared__ float columns[RPW > 1 ? THREADS * VEC * ITER : 1];
    const int t = (int)threadIdx.x % TPR, sub = (int)threadIdx.x / TPR;
    const float inv = 1.0f / d.c;
    int turn = 0;
    float cs[3][ITER][VEC];  // dscale, dpost, dpre
#pragma unroll
    for (int k = 0; k < 3; ++k)
#pragma unroll
        for (int i = 0; i < ITER; ++i)
#pragma unroll
            for (int e = 0; e < VEC; ++e) cs[k][i][e] = 0.0f;
    for (int64_t row0 = (int64_t)blockIdx.x * RPW; row0 < d.m; row0 += (int64_t)gridDim.x * RPW) {
        const int64_t row = row0 + sub;
        const bool live = row < d.m;
        float rb = 0.0f, rr = 0.0f;
        if (live) rb = stats[2 * row], rr = stats[2 * row + 1];
        float xv[ITER][VEC], bv[ITER][VEC], gv[ITER][VEC], rv[ITER][VEC], uv[ITER][VEC];
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const int c = (i * TPR + t) * VEC, have = live ? d.c - c : 0;
            load_part(x + row * d.x_row + c, have, xv[i]);
            if (b) load_part(b + row * d.b_row + c, have, bv[i]);
            if (gate) load_part(gate + row * d.gate_row + c, have, gv[i]);
            if (dr) load_part(dr + row * d.r_row + c, have, rv[i]);
            if (du) load_part(du + row * d.u_row + c, have, uv[i]);
        }
        // sums of w rh, of (dr + rr w) times what db weighs it with, and of rr rh so weighed: dx is linear in the first's mean
        float sums[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const int c = (i * TPR + t) * VEC, have = live ? d.c - c : 0;
            float sv[VEC], pv[VEC], wv[VEC];
            if (scale) load_part(scale + c, have, sv);
            if (post) load_part(post + c, have, pv);
            if (pre) load_part(pre + c, have, wv);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float bh = b ? bv[i][e] * rb : 0.0f;
                const float p = post ? bh * pv[e] : bh;
                const float sg = gate ? sigmoid(gv[i][e]) : 1.0f;
                const float q = scale ? sv[e] * sg : sg;
                const float rh = b ? (xv[i][e] + q * p) * rr : xv[i][e] * rr;
                const float w = !du ? 0.0f : pre ? uv[i][e] * wv[e] : uv[i][e];
                const float first = (dr ? rv[i][e] : 0.0f) + rr * w;
                xv[i][e] = rh;
                rv[i][e] = first;
                sums[0] += w * rh;
                sums[1] += first * q * p;
                sums[2] += rr * rh * q * p;
                if (du) cs[2][i][e] += uv[i][e] * rh;
            }
        }
        row_sums<TPR, 3>(sums, place, turn);
        const float m1 = sums[0] * inv, m2 = (sums[1] - m1 * sums[2]) * inv;
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const int c = (i * TPR + t) * VEC, have = live ? d.c - c : 0;
            float sv[VEC], pv[VEC];
            if (scale) load_part(scale + c, have, sv);
            if (post) load_part(post + c, have, pv);
            float out[VEC], og[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float dxe = rv[i][e] - rr * xv[i][e] * m1;
                rv[i][e] = dxe;
                if (!b) continue;
                const float bh = bv[i][e] * rb;
                const float p = post ? bh * pv[e] : bh;
                float sg = 1.0f, rest = 0.0f;
                if (gate) gate_pair(gv[i][e], sg, rest);
                const float q = scale ? sv[e] * sg : sg;
                const float dp = dxe * q;
                cs[0][i][e] += dxe * sg * p;
                cs[1][i][e] += dp * bh;
                og[e] = dp * p * rest;
                const float weighed = post ? dp * pv[e] : dp;
                out[e] = d.post_norm ? rb * (weighed - bh * m2) : weighed;
            }
            if (dx) store_part(dx + row * d.dx_row + c, have, rv[i]);
            if (db) store_part(db + row * d.db_row + c, have, out);
            if (dgate) store_part(dgate + row * d.dgate_row + c, have, og);
        }
    }
    if (!part) return;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        if constexpr (RPW > 1) {  // the workgroup's rows, in their order
            __syncthreads();
#pragma unroll
            for (int i = 0; i < ITER; ++i)
#pragma unroll
                for (int e = 0; e < VEC; ++e) columns[(sub * ITER * TPR + i * TPR + t) * VEC + e] = cs[k][i][e];
            __syncthreads();
            for (int c = threadIdx.x; c < TPR * ITER * VEC; c += THREADS) {
                float s = 0.0f;
                for (int j = 0; j < RPW; ++j) s += columns[j * TPR * ITER * VEC + c];
                if (c < d.c) part[((int64_t)blockIdx.x * 3 + k) * d.c + c] = s;
            }
        } else {
#pragma unroll
            for (int i = 0; i < ITER; ++i) {
                const int c = (i * TPR + t) * VEC;
                store_part(part + ((int64_t)blockIdx.x * 3 + k) * d.c + c, d.c - c, cs[k][i]);
            }
        }
    }
}

// The workgroups' sums, in one order: 64 columns a workgroup, 16 parts of the list side by side
__global__ __launch_bounds__(1024) void residual_columns_kernel(const float* part, int groups, int c, float* dscale, float* dpost, float* dpre) {
    __shared__ float sums[16][64];
    const int lane = threadIdx.x & 63, slot = threadIdx.x >> 6, kind = blockIdx.y;
    float* out = kind == 0 ? dscale : kind == 1 ? dpost : dpre;
    if (!out) return;
    const int col = (int)blockIdx.x * 64 + lane;
    float s = 0.0f;
    if (col < c)
        for (int g = slot; g < groups; g += 16) s += part[((int64_t)g * 3 + kind) * c + col];
    sums[slot][lane] = s;
    __syncthreads();
    if (slot == 0 && col < c) {
        float all = 0.0f;
        for (int i = 0; i < 16; ++i) all += sums[i][lane];
        out[col] = all;
    }
}

template <int T, int I, int TH>
struct Form {
    static constexpr int TPR = T, ITER = I, THREADS = TH;
};
// The fewest threads that hold a row in two vectors each at the most, by whole wavefronts where a row has more than 16 vectors
template <typename F>
void with_form(int c, F&& f) {
    if (c <= 128) f(Form<16, 1, 256>{});
    else if (c <= 512) f(Form<64, 1, 256>{});
    else if (c <= 1024) f(Form<64, 2, 256>{});
    else if (c <= 2048) f(Form<256, 1, 256>{});
    else if (c <= 4096) f(Form<256, 2, 256>{});
    else if (c <= 8192) f(Form<1024, 1, 1024>{});
    else f(Form<1024, 2, 1024>{});
}
template <typename F>
void with_types(const rrm_residual_desc& d, F&& f) {
    if (d.x_elem == RRM_F32 && d.b_elem == RRM_F32) f(0.0f, 0.0f);
    else if (d.x_elem == RRM_F32) f(0.0f, (__bf16)0.0f);
    else if (d.b_elem == RRM_F32) f((__bf16)0.0f, 0.0f);
    else f((__bf16)0.0f, (__bf16)0.0f);
}

constexpr int FORWARD_GROUPS = 2048, BACK_GROUPS = 512;
int groups_of(const rrm_residual_desc& d, int most) {
    int groups = 0;
    with_form(d.c, [&](auto form) {
        constexpr int RPW = decltype(form)::THREADS / decltype(form)::TPR;
        const int all = (int)(((int64_t)d.m + RPW - 1) / RPW);
        groups = all < most ? all : most;
    });
    return groups;
}

}  // namespace

size_t residual_scratch(const rrm_residual_desc& d) { return round256((size_t)groups_of(d, BACK_GROUPS) * 3 * d.c * sizeof(float)); }

hipError_t launch_residual_norm(const rrm_residual_desc& d, const void* x, const void* b, const void* gate, const float* scale, const float* post,
                                const float* pre, void* r, void* u, float* stats, hipStream_t s) {
    with_types(d, [&](auto xt, auto bt) {
        using X = decltype(xt);
        using B = decltype(bt);
        with_form(d.c, [&](auto form) {
            using F = decltype(form);
            hipLaunchKernelGGL((residual_kernel<X, B, F::TPR, F::ITER, F::THREADS>), dim3((unsigned)groups_of(d, FORWARD_GROUPS)), dim3(F::THREADS), 0, s, d,
                               (const X*)x, (const B*)b, (const B*)gate, scale, post, pre, (X*)r, (B*)u, stats);
        });
    });
    return hipGetLastError();
}

hipError_t launch_residual_norm_backward(const rrm_residual_desc& d, const void* dr, const void* du, const void* x, const void* b,
                                         const float* stats, const void* gate, const float* scale, const float* post, const float* pre,
                                         void* dx, void* db, void* dgate, float* dscale, float* dpost, float* dpre, void* ws, hipStream_t s) {
    const bool sums = dscale || dpost || dpre;
    float* part = sums && d.m > 0 ? (float*)ws : nullptr;
    const int groups = d.m > 0 ? groups_of(d, BACK_GROUPS) : 0;
    hipError_t e = hipSuccess;
    if (d.m > 0) {
        with_types(d, [&](auto xt, auto bt) {
            using X = decltype(xt);
            using B = decltype(bt);
            with_form(d.c, [&](auto form) {
                using F = decltype(form);
                hipLaunchKernelGGL((residual_back_kernel<X, B, F::TPR, F::ITER, F::THREADS>), dim3((unsigned)groups), dim3(F::THREADS), 0, s, d,
                                   (const X*)dr, (const B*)du, (const X*)x, (const B*)b, stats, (const B*)gate, scale, post, pre, (X*)dx, (B*)db, (B*)dgate,
                                   part);
            });
        });
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (sums) {
        hipLaunchKernelGGL(residual_columns_kernel, dim3((unsigned)((d.c + 63) / 64), 3), dim3(1024), 0, s, part, groups, d.c, dscale, dpost, dpre);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace rrm
