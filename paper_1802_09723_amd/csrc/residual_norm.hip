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
// is as many bytes as reading a stored r, and r in 32 bits.  16384 rows of 4096 features with a gate, x fp32 and b bf16: 181 us forward (4.8 TB/s), 328 backward
// (4.7 TB/s) and 5 for the weights' gradients; bf16 throughout 133 forward (5.0 TB/s, a large copy's rate).
#include "op_common.h"

namespace rrm {

namespace {

constexpr int VEC = 8;  // neighbouring features of a thread

// What weights that are NULL read: the sums below then have no branch (a branch for each cost the backward pass the registers of two wavefronts)
constexpr int MOST_COLUMNS = 16384;
struct Ones {
    float v[MOST_COLUMNS];
    constexpr Ones() : v() {
        for (float& e : v) e = 1.0f;
    }
};
__device__ const Ones g_ones{};

// How a thread's vector lies in its row.  WHOLE: rows are whole vectors.  EARLY: the last vector of a row begins early; what it has before `first` is another
// thread's, and counts as zeros.  SHORT: rows of fewer than VEC features, element by element.
enum Lie : int { WHOLE = 0, EARLY = 1, SHORT = 2 };
template <int LIE>
struct Place {
    int at, first;  // the vector's first feature; this thread's first one of it (VEC: none)
    __device__ __forceinline__ Place(int c, int cols) : at(c), first(c < cols ? 0 : VEC) {
        if (LIE == EARLY && c < cols && c + VEC > cols) at = cols - VEC, first = c - at;
        if (LIE == SHORT && c < cols) first = cols;  // (the one thread's: features 0 .. cols)
    }
};
// VEC elements as they lie in memory: not converted until they are used, so that loads stay on their way; zeros where this thread has none
template <typename T, int LIE>
struct Raw {
    static constexpr int WORDS = VEC * (int)sizeof(T) / 4;
    unsigned int w[WORDS];
    __device__ __forceinline__ void load(const T* row, const Place<LIE>& p, bool live) {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) w[i] = 0;
        if (LIE == SHORT) {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (live && p.first < VEC && e < p.first) {
                    if constexpr (sizeof(T) == 4) w[e] = __float_as_uint((float)row[e]);
                    else w[e >> 1] |= (unsigned int)__builtin_bit_cast(unsigned short, row[e]) << (16 * (e & 1));
                }
        } else if (live && p.first < VEC) {
            load_words<WORDS>(row + p.at, w);
        }
    }
    __device__ __forceinline__ float get(int e, const Place<LIE>& p) const {
        float v;
        if constexpr (sizeof(T) == 4) v = __uint_as_float(w[e]);
        else v = e & 1 ? bf16_hi(w[e >> 1]) : bf16_lo(w[e >> 1]);
        return LIE == EARLY && e < p.first ? 0.0f : v;
    }
};
template <typename T, int LIE>
__device__ __forceinline__ void put(T* row, const Place<LIE>& p, bool live, const float (&v)[VEC]) {
    if (!live || p.first >= VEC) return;
    if (LIE == WHOLE) {
        store_vec<VEC>(row + p.at, v);
    } else if (LIE == EARLY) {
        store_some<VEC>(row + p.at, v, p.first);
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            if (e < p.first) store_elem(row + e, v[e]);
    }
}

// Sums over the TPR threads of a row, N at once, in one order; `place`: LDS for [2][rows][N][wavefronts of a row], `turn` flips between calls
template <int TPR, int N, int THREADS>
__device__ __forceinline__ void row_sums(float (&v)[N], float* place, int& turn) {
#pragma unroll
    for (int m = 1; m < (TPR < 64 ? TPR : 64); m <<= 1)
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += __shfl_xor(v[k], m);
    if constexpr (TPR > 64) {
        constexpr int WAVES = TPR / 64;
        float* mine = place + turn * N * (THREADS / 64) + (int)threadIdx.x / TPR * N * WAVES;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) mine[k * WAVES + ((int)threadIdx.x % TPR >> 6)] = v[k];
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
template <typename X, typename B, int TPR, int ITER, int THREADS, int LIE, bool GATE>
__global__ __launch_bounds__(THREADS) void residual_kernel(rrm_residual_desc d, const X* x, const B* b, const B* gate, const float* scale, const float* post,
                                                           const float* pre, X* r, B* u, float* stats) {
    __shared__ float place[2 * 16];
    constexpr int RPW = THREADS / TPR;
    const int t = (int)threadIdx.x % TPR;
    const float inv = 1.0f / d.c;
    int turn = 0;
    if (!scale) scale = g_ones.v;
    if (!post) post = g_ones.v;
    if (!pre) pre = g_ones.v;
    for (int64_t row0 = (int64_t)blockIdx.x * RPW; row0 < d.m; row0 += (int64_t)gridDim.x * RPW) {
        const int64_t row = row0 + (int)threadIdx.x / TPR;
        const bool live = row < d.m;
        Raw<X, LIE> xw[ITER];
        Raw<B, LIE> bw[ITER], gw[ITER];
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const Place<LIE> p((i * TPR + t) * VEC, d.c);
            xw[i].load(x + row * d.x_row, p, live);
            bw[i].load(b + row * d.b_row, p, live && b);
            if (GATE) gw[i].load(gate + row * d.gate_row, p, live);
        }
        float rv[ITER][VEC];
        float sums[1] = {0.0f};
        float rb = 1.0f;
        if (d.post_norm) {
#pragma unroll
            for (int i = 0; i < ITER; ++i) {
                const Place<LIE> p((i * TPR + t) * VEC, d.c);
#pragma unroll
                for (int e = 0; e < VEC; ++e) sums[0] += bw[i].get(e, p) * bw[i].get(e, p);
            }
            row_sums<TPR, 1, THREADS>(sums, place, turn);
            rb = 1.0f / sqrtf(sums[0] * inv + d.eps);
        }
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const Place<LIE> p((i * TPR + t) * VEC, d.c);
            Raw<float, LIE> sw, pw;
            sw.load(scale, p, true);
            pw.load(post, p, true);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                float add = bw[i].get(e, p) * rb * pw.get(e, p) * sw.get(e, p);
                if (GATE) add *= sigmoid(gw[i].get(e, p));
                rv[i][e] = xw[i].get(e, p) + add;
            }
            if (r) put(r + row * d.r_row, p, live, rv[i]);
        }
        float rr = 1.0f;
        if (u) {
            sums[0] = 0.0f;
#pragma unroll
            for (int i = 0; i < ITER; ++i)
#pragma unroll
                for (int e = 0; e < VEC; ++e) sums[0] += rv[i][e] * rv[i][e];
            row_sums<TPR, 1, THREADS>(sums, place, turn);
            rr = 1.0f / sqrtf(sums[0] * inv + d.eps);
#pragma unroll
            for (int i = 0; i < ITER; ++i) {
                const Place<LIE> p((i * TPR + t) * VEC, d.c);
                Raw<float, LIE> ww;
                ww.load(pre, p, true);
                float out[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) out[e] = rv[i][e] * rr * ww.get(e, p);
                put(u + row * d.u_row, p, live, out);
            }
        }
        if (stats && live && t == 0) stats[2 * row] = rb, stats[2 * row + 1] = rr;
    }
}

// The backward pass, and sums over rows of three kinds, a workgroup's each: part [workgroup][3][c].  One reduction a row: dx is linear in mean(w rh), so
// what db needs of dx is put together of two sums that do not wait for it.
template <typename X, typename B, int TPR, int ITER, int THREADS, int LIE, bool GATE>
__global__ __launch_bounds__(THREADS) void residual_back_kernel(rrm_residual_desc d, const X* dr, const B* du, const X* x, const B* b, const float* stats,
                                                                const B* gate, const float* scale_, const float* post_, const float* pre_, X* dx, B* db,
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
        // (weights are read again for each row, out of the nearest cache: held over the loop they would cost the registers of a wavefront more)
        const float *scale = scale_ ? scale_ : g_ones.v, *post = post_ ? post_ : g_ones.v, *pre = pre_ ? pre_ : g_ones.v;
        asm volatile("" : "+s"(scale), "+s"(post), "+s"(pre));
        Raw<X, LIE> xw[ITER], rw[ITER];
        Raw<B, LIE> bw[ITER], gw[ITER], uw[ITER];
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const Place<LIE> p((i * TPR + t) * VEC, d.c);
            xw[i].load(x + row * d.x_row, p, live);
            bw[i].load(b + row * d.b_row, p, live && b);
            if (GATE) gw[i].load(gate + row * d.gate_row, p, live);
            rw[i].load(dr + row * d.r_row, p, live && dr);
            uw[i].load(du + row * d.u_row, p, live && du);
        }
        float rb = 0.0f, rr = 0.0f;
        if (live) rb = stats[2 * row], rr = stats[2 * row + 1];
        // sums of w rh, of (dr + rr w) times what db weighs it with, and of rr rh so weighed
        float sums[3] = {0.0f, 0.0f, 0.0f};
        float rh[ITER][VEC], first[ITER][VEC];
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const Place<LIE> p((i * TPR + t) * VEC, d.c);
            Raw<float, LIE> sw, pw, ww;
            sw.load(scale, p, true);
            pw.load(post, p, true);
            ww.load(pre, p, true);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                float weighed = bw[i].get(e, p) * rb * pw.get(e, p) * sw.get(e, p);  // q p
                if (GATE) weighed *= sigmoid(gw[i].get(e, p));
                rh[i][e] = (xw[i].get(e, p) + weighed) * rr;
                const float ue = uw[i].get(e, p), w = ue * ww.get(e, p);
                first[i][e] = rw[i].get(e, p) + rr * w;
                sums[0] += w * rh[i][e];
                sums[1] += first[i][e] * weighed;
                sums[2] += rh[i][e] * weighed;
                cs[2][i][e] += ue * rh[i][e];
            }
        }
        row_sums<TPR, 3, THREADS>(sums, place, turn);
        const float m1 = sums[0] * inv * rr, m2 = d.post_norm ? (sums[1] - m1 * sums[2]) * inv : 0.0f;
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const Place<LIE> p((i * TPR + t) * VEC, d.c);
            Raw<float, LIE> sw, pw;
            sw.load(scale, p, true);
            pw.load(post, p, true);
            float out[VEC], og[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float dxe = first[i][e] - rh[i][e] * m1;
                first[i][e] = dxe;
                const float bh = bw[i].get(e, p) * rb, pv = pw.get(e, p);
                float sg = 1.0f, rest = 0.0f;
                if (GATE) gate_pair(gw[i].get(e, p), sg, rest);
                const float gated = dxe * sg, dp = gated * sw.get(e, p);
                cs[0][i][e] += gated * (bh * pv);
                cs[1][i][e] += dp * bh;
                if (GATE) og[e] = dp * (bh * pv) * rest;
                out[e] = rb * (dp * pv - bh * m2);
            }
            if (dx) put(dx + row * d.dx_row, p, live, first[i]);
            if (db) put(db + row * d.db_row, p, live, out);
            if (GATE && dgate) put(dgate + row * d.dgate_row, p, live, og);
        }
    }
    if (!part) return;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        float* to = part + ((int64_t)blockIdx.x * 3 + k) * d.c;
        if constexpr (RPW > 1) {  // the workgroup's rows, in their order
            __syncthreads();
#pragma unroll
            for (int i = 0; i < ITER; ++i)
#pragma unroll
                for (int e = 0; e < VEC; ++e) columns[(sub * ITER * TPR + i * TPR + t) * VEC + e] = cs[k][i][e];
            __syncthreads();
            for (int v = threadIdx.x; v < TPR * ITER * VEC; v += THREADS) {
                const Place<LIE> p(v / VEC * VEC, d.c);
                float s = 0.0f;
                for (int j = 0; j < RPW; ++j) s += columns[j * TPR * ITER * VEC + v];
                const int e = v % VEC;
                if (LIE == SHORT ? p.first < VEC && e < p.first : e >= p.first) to[p.at + e] = s;
            }
        } else {
#pragma unroll
            for (int i = 0; i < ITER; ++i) put(to, Place<LIE>((i * TPR + t) * VEC, d.c), true, cs[k][i]);
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
        for (int g = slot; g < groups; g += 128) {  // eight on their way at once
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = g + 16 * i < groups ? part[((int64_t)(g + 16 * i) * 3 + kind) * c + col] : 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[i];
        }
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
// The fewest threads that hold a row, a vector each (two beyond 8192 features)
template <typename F>
void with_form(int c, F&& f) {
    if (c <= 128) f(Form<16, 1, 256>{});
    else if (c <= 512) f(Form<64, 1, 256>{});
    else if (c <= 1024) f(Form<128, 1, 256>{});
    else if (c <= 2048) f(Form<256, 1, 256>{});
    else if (c <= 4096) f(Form<512, 1, 512>{});
    else if (c <= 8192) f(Form<1024, 1, 1024>{});
    else f(Form<1024, 2, 1024>{});
}
template <typename F, typename G>
void with_lie(int c, F, G&& g) {
    if (c % VEC == 0) g(std::integral_constant<int, WHOLE>{});
    else if (c > VEC) g(std::integral_constant<int, EARLY>{});
    else if constexpr (F::TPR == 16) g(std::integral_constant<int, SHORT>{});
}
template <typename F>
void with_types(const rrm_residual_desc& d, F&& f) {
    if (d.x_elem == RRM_F32 && d.b_elem == RRM_F32) f(0.0f, 0.0f);
    else if (d.x_elem == RRM_F32) f(0.0f, (__bf16)0.0f);
    else if (d.b_elem == RRM_F32) f((__bf16)0.0f, 0.0f);
    else f((__bf16)0.0f, (__bf16)0.0f);
}

// Workgroups of a pass: as many as run at once, of the backward pass, each of which leaves sums to be joined (1024 instead of 256 for 4096 features: the join
// takes 26 us instead of 5, the pass itself as long)
int groups_of(const rrm_residual_desc& d, bool backward) {
    int groups = 0;
    with_form(d.c, [&](auto form) {
        constexpr int RPW = decltype(form)::THREADS / decltype(form)::TPR;
        const int most = !backward ? 2048 : decltype(form)::THREADS > 256 ? OP_CUS : 3 * OP_CUS;
        const int all = (int)(((int64_t)d.m + RPW - 1) / RPW);
        groups = all < most ? all : most;
    });
    return groups;
}

}  // namespace

size_t residual_scratch(const rrm_residual_desc& d) { return round256((size_t)groups_of(d, true) * 3 * d.c * sizeof(float)); }

hipError_t launch_residual_norm(const rrm_residual_desc& d, const void* x, const void* b, const void* gate, const float* scale, const float* post,
                                const float* pre, void* r, void* u, float* stats, hipStream_t s) {
    with_types(d, [&](auto xt, auto bt) {
        using X = decltype(xt);
        using B = decltype(bt);
        with_form(d.c, [&](auto form) {
            using F = decltype(form);
            with_lie(d.c, form, [&](auto lie) {
                auto launch = [&](auto gated) {
                    hipLaunchKernelGGL((residual_kernel<X, B, F::TPR, F::ITER, F::THREADS, decltype(lie)::value, decltype(gated)::value>),
                                       dim3((unsigned)groups_of(d, false)), dim3(F::THREADS), 0, s, d, (const X*)x, (const B*)b, (const B*)gate, scale,
                                       post, pre, (X*)r, (B*)u, stats);
                };
                gate ? launch(std::true_type{}) : launch(std::false_type{});
            });
        });
    });
    return hipGetLastError();
}

hipError_t launch_residual_norm_backward(const rrm_residual_desc& d, const void* dr, const void* du, const void* x, const void* b,
                                         const float* stats, const void* gate, const float* scale, const float* post, const float* pre,
                                         void* dx, void* db, void* dgate, float* dscale, float* dpost, float* dpre, void* ws, hipStream_t s) {
    const bool sums = dscale || dpost || dpre;
    float* part = sums && d.m > 0 ? (float*)ws : nullptr;
    const int groups = d.m > 0 ? groups_of(d, true) : 0;
    hipError_t e = hipSuccess;
    if (d.m > 0) {
        with_types(d, [&](auto xt, auto bt) {
            using X = decltype(xt);
            using B = decltype(bt);
            with_form(d.c, [&](auto form) {
                using F = decltype(form);
                with_lie(d.c, form, [&](auto lie) {
                    auto launch = [&](auto gated) {
                        hipLaunchKernelGGL((residual_back_kernel<X, B, F::TPR, F::ITER, F::THREADS, decltype(lie)::value, decltype(gated)::value>),
                                           dim3((unsigned)groups), dim3(F::THREADS), 0, s, d, (const X*)dr, (const B*)du, (const X*)x, (const B*)b, stats,
                                           (const B*)gate, scale, post, pre, (X*)dx, (B*)db, (B*)dgate, part);
                    };
                    gate ? launch(std::true_type{}) : launch(std::false_type{});
                });
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
