// Gated feed-forward block and its backward pass.
#include "op_common.h"

namespace rrm {

namespace {

typedef const __bf16* src_t;
typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef const __attribute__((address_space(1))) unsigned int* gptr_t;
typedef __attribute__((address_space(3))) unsigned int* lptr_t;
typedef __attribute__((address_space(3))) v4s* lds4_t;

constexpr int STEP = 64;  // of the summed axis, staged at once

// What chunks of the summed axis behind its end are read from.
__device__ const u32x4 g_zeros = {0, 0, 0, 0};

// An operand: [rows][summed axis], element (r, k) at p + r * row + k; or, "turned", at p + k * row + r.
struct Source {
    src_t p;
    int64_t row;
};

// out[i][j] = sum over k of P[i][k] Q[j][k], summed over two pairs of operands where there are two.
struct Product {
    Source p[2], q[2];
    int pairs;              // gated: 1, and q[1] is the second projection's weights
    int rows, cols, len;    // of P, of Q (gated: of each projection), of the summed axis (of each pair)
    int tiles_m, tiles_n;   // tiles_m counts those of both products where there are two (see halves)
    int splits;             // parts of the summed axis, one workgroup each; more than one: sums to `part`
    __bf16 *out, *out2, *out3;  // gated: H, G, U (G and U may be nullptr); halves: out2 belongs to p[1]
    int64_t out_row, out2_row;
    float* part;            // [splits][rows][cols]
    int vec_out;            // results may be stored 16 bytes at a time
};

enum Kind : int { GATED = 0, PLAIN = 1, HALVES = 2 };

// 32-byte-window spreading of a turned tile's LDS rows: see the kernel
template <int WINDOWS>
__device__ __forceinline__ int window_turn(int k) {
    return WINDOWS >= 8 ? (k & 3) | ((k >> 1) & 4) : WINDOWS == 4 ? (k & 3) : WINDOWS == 2 ? ((k >> 1) & 1) : 0;
}

// eight elements of a row of `len`, from element k on, at any alignment; zeros behind the end
__device__ __forceinline__ u32x4 ragged_chunk(src_t row, int k, int len) {
    struct __attribute__((packed, aligned(2))) loose {
        u32x4 v;
    };
    u32x4 w = {0, 0, 0, 0};
    if (k + 8 <= len) {
        w = reinterpret_cast<const loose*>(row + k)->v;
    } else if (k < len) {
        unsigned short e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = k + i < len ? __builtin_bit_cast(unsigned short, row[k + i]) : (unsigned short)0;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = (unsigned int)e[2 * i] | ((unsigned int)e[2 * i + 1] << 16);
    }
    return w;
}

// Tile product on the matrix cores.  (comment to come)
template <int KIND, int ACT, bool PT, bool QT, int MT, int NT, int WM, int WN, bool RAGGED>
__global__ __launch_bounds__(WM* WN * 64, WM* WN == 8 ? 2 : 2) void tile_kernel(Product a) {
    constexpr int THREADS = WM * WN * 64, BM = MT * 32 * WM, BN = NT * 32 * WN;
    constexpr int PB = BM * STEP * 2, QB = BN * STEP * 2;                       // bytes of a staged tile
    constexpr int NP = PB / (THREADS * 16), NQ = QB / (THREADS * 16);          // 16-byte chunks a thread stages
    constexpr int OUT_COLS = KIND == GATED ? BN / 2 : BN;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * (PB + QB)];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int wm = wave % WM, wn = wave / WM;

    // tiles XCD by XCD (workgroups go to the eight in turn), and there in blocks of eight rows of tiles
    int tm, tn;
    {
        const int total = a.tiles_m * a.tiles_n, id = (int)blockIdx.x, xcd = id & 7, q = total >> 3, r = total & 7;
        const int t = xcd * q + (xcd < r ? xcd : r) + (id >> 3);
        const int group = 8 * a.tiles_n, g = t / group, first = g * 8, n = a.tiles_m - first < 8 ? a.tiles_m - first : 8;
        tm = first + (t - g * group) % n;
        tn = (t - g * group) / n;
    }
    int half = 0;
    if (KIND == HALVES) {
        const int per = a.tiles_m >> 1;
        half = tm >= per;
        tm -= half * per;
    }
    const int m0 = tm * BM, n0 = tn * OUT_COLS;
    const int steps_of = (a.len + STEP - 1) / STEP;  // of one pair
    const int steps_all = steps_of * (KIND == PLAIN ? a.pairs : 1);
    const int split = (int)blockIdx.y;
    const int s0 = (int)((int64_t)steps_all * split / a.splits), s1 = (int)((int64_t)steps_all * (split + 1) / a.splits);

    // Sources of this thread's chunks.  LDS holds [row][64 of the summed axis] with the eight chunks of a row turned by the row's
    // number (XOR), or, for turned operands, [64][rows] with the 64-byte windows of a row turned likewise, so that the fragment reads of a wavefront
    // meet different banks; the copies write LDS in lane order, so the turning is done on the source's side.
    src_t pp[NP], qp[NQ];
    int pk[NP], qk[NQ];  // place on the summed axis within a step
    int pr[NP], qr[NQ];  // row
    auto row_of_q = [&](int r) -> int {  // tile row -> row of the weights (gated: 32 of the one, 32 of the other)
        return KIND == GATED ? n0 + (r >> 6) * 32 + (r & 31) : n0 + r;
    };
    constexpr int PW = BM * 2 / 64, QW = BN * 2 / 64;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int at = (i * THREADS + tid) * 16;
        if (PT) {
            const int k = at / (BM * 2), c = (at % (BM * 2)) / 16;
            pk[i] = k;
            pr[i] = m0 + (((c >> 2) ^ window_turn<PW>(k)) * 4 + (c & 3)) * 8;
        } else {
            const int r = at / 128;
            pk[i] = (((at % 128) / 16) ^ (r & 7)) * 8;
            pr[i] = m0 + r;
        }
    }
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        const int at = (i * THREADS + tid) * 16;
        if (QT) {
            const int k = at / (BN * 2), c = (at % (BN * 2)) / 16;
            qk[i] = k;
            qr[i] = n0 + (((c >> 2) ^ window_turn<QW>(k)) * 4 + (c & 3)) * 8;
        } else {
            const int r = at / 128;
            qk[i] = (((at % 128) / 16) ^ (r & 7)) * 8;
            qr[i] = row_of_q(r);
        }
    }
    // rows behind the last are read as the last (their results are dropped); turned: as the last chunk of the row
    const int p_last = PT ? (a.rows - 1) & ~7 : a.rows - 1, q_last = QT ? (a.cols - 1) & ~7 : a.cols - 1;
    int64_t p_step = 0, q_step = 0;
    auto point = [&](int s) {  // the chunks' places in step s
        const int pair = KIND == PLAIN && s >= steps_of ? 1 : 0;
        const Source& sp = a.p[KIND == HALVES ? half : pair];
        const int64_t k0 = (int64_t)(s - pair * steps_of) * STEP;
        p_step = PT ? sp.row * STEP : STEP;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int r = pr[i] < p_last ? pr[i] : p_last;
            pp[i] = sp.p + (PT ? (k0 + pk[i]) * sp.row + r : r * sp.row + k0 + pk[i]);
        }
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            const int at = (i * THREADS + tid) * 16;
            const Source& sq = a.q[KIND == GATED ? ((at / 128) >> 5) & 1 : pair];
            if (i == 0) q_step = QT ? sq.row * STEP : STEP;
            const int r = qr[i] < q_last ? qr[i] : q_last;
            qp[i] = sq.p + (QT ? (k0 + qk[i]) * sq.row + r : r * sq.row + k0 + qk[i]);
        }
    };
    const src_t zeros = reinterpret_cast<src_t>(&g_zeros);
    u32x4 pv[RAGGED ? NP : 1], qv[RAGGED ? NQ : 1];
    auto stage = [&](int s, int buf) {  // starts the copies of step s
        const int pair = KIND == PLAIN && s >= steps_of ? 1 : 0;
        const int rem = a.len - (s - pair * steps_of) * STEP;
        unsigned char* dp = lds + buf * (PB + QB);
        unsigned char* dq = dp + PB;
        if (RAGGED) {
#pragma unroll
            for (int i = 0; i < NP; ++i)
                pv[i] = PT ? (pk[i] < rem ? ragged_chunk(pp[i], 0, a.rows - (pr[i] < p_last ? pr[i] : p_last)) : u32x4{0, 0, 0, 0})
                           : ragged_chunk(pp[i] - pk[i], pk[i], rem);
#pragma unroll
            for (int i = 0; i < NQ; ++i)
                qv[i] = QT ? (qk[i] < rem ? ragged_chunk(qp[i], 0, a.cols - (qr[i] < q_last ? qr[i] : q_last)) : u32x4{0, 0, 0, 0})
                           : ragged_chunk(qp[i] - qk[i], qk[i], rem);
        } else {
#pragma unroll
            for (int i = 0; i < NP; ++i)
                __builtin_amdgcn_global_load_lds((gptr_t)(rem >= STEP || pk[i] < rem ? pp[i] : zeros),
                                                 (lptr_t)(dp + (i * THREADS + wave * 64) * 16), 16, 0, 0);
#pragma unroll
            for (int i = 0; i < NQ; ++i)
                __builtin_amdgcn_global_load_lds((gptr_t)(rem >= STEP || qk[i] < rem ? qp[i] : zeros),
                                                 (lptr_t)(dq + (i * THREADS + wave * 64) * 16), 16, 0, 0);
        }
        if (KIND == PLAIN && s + 1 == steps_of && s + 1 < s1) {
            point(s + 1);
        } else {
#pragma unroll
            for (int i = 0; i < NP; ++i) pp[i] += p_step;
#pragma unroll
            for (int i = 0; i < NQ; ++i) qp[i] += q_step;
        }
    };
    auto land = [&](int buf) {  // ragged: what stage() has fetched goes to LDS
        if (RAGGED) {
            unsigned char* dp = lds + buf * (PB + QB);
#pragma unroll
            for (int i = 0; i < NP; ++i) *reinterpret_cast<u32x4*>(dp + (i * THREADS + tid) * 16) = pv[i];
#pragma unroll
            for (int i = 0; i < NQ; ++i) *reinterpret_cast<u32x4*>(dp + PB + (i * THREADS + tid) * 16) = qv[i];
        }
    };

    v16f acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;

    // Fragment reads: lane l holds row l % 32 and eight of the summed axis, (l / 32) * 8 on in a step of 16
    const int flat = (lane & 31) * 128 + (((lane >> 5) ^ (lane & 7)) << 4);
    const int turn = ((lane >> 2) & 3) | ((lane >> 5) << 2), tk = (lane >> 5) * 8 + ((lane >> 2) & 3), tin = ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
    auto frag = [&](const unsigned char* tile, int r0, int ks, auto turned, auto rows) -> v8bf {
        constexpr int ROWS = decltype(rows)::value;
        if constexpr (decltype(turned)::value) {
            constexpr int W = ROWS * 2 / 64;
            const int t = W >= 8 ? turn : W == 4 ? (turn & 3) : W == 2 ? ((turn >> 1) & 1) : 0;
            const unsigned char* at = tile + (ks * 16 + tk) * (ROWS * 2) + (((r0 >> 5) ^ t) << 6) + tin;
            struct {
                v4s lo, hi;
            } v;
            v.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4_t)(at));
            // (four on along the summed axis: the two low bits of k, and so the turn, are the same; W == 2 turns by bit 1 alone)
            v.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4_t)(at + 4 * ROWS * 2));
            return __builtin_bit_cast(v8bf, v);
        } else {
            return *reinterpret_cast<const v8bf*>(tile + r0 * 128 + (flat ^ (ks << 5)));
        }
    };
    const auto p_turned = std::integral_constant<bool, PT>{};
    const auto q_turned = std::integral_constant<bool, QT>{};
    const auto p_rows = std::integral_constant<int, BM>{};
    const auto q_rows = std::integral_constant<int, BN>{};

    if (s0 < s1) {
        point(s0);
        stage(s0, 0);
        land(0);
    }
    for (int s = s0; s < s1; ++s) {
        const int buf = (s - s0) & 1;
        __builtin_amdgcn_s_waitcnt(0);  // this wavefront's copies have landed
        __syncthreads();                // everybody's have; and everybody is done with the other buffer
        if (s + 1 < s1) stage(s + 1, buf ^ 1);
        const unsigned char* tp = lds + buf * (PB + QB);
        const unsigned char* tq = tp + PB;
#pragma unroll
        for (int ks = 0; ks < STEP / 16; ++ks) {
            v8bf fp[MT], fq[NT];
#pragma unroll
            for (int j = 0; j < NT; ++j) fq[j] = frag(tq, (wn * NT + j) * 32, ks, q_turned, q_rows);
#pragma unroll
            for (int i = 0; i < MT; ++i) fp[i] = frag(tp, (wm * MT + i) * 32, ks, p_turned, p_rows);
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fq[j], fp[i], acc[i][j], 0, 0, 0);
        }
        if (s + 1 < s1) land(buf ^ 1);
    }

    // acc[i][j][4 q + e] of lane l: row (wm MT + i) 32 + l % 32, column (wn NT + j) 32 + 8 q + 4 (l / 32) + e
    const int lr = lane & 31, lc = (lane >> 5) * 4;
    if (KIND == PLAIN && a.splits > 1) {
        float* part = a.part + (int64_t)split * a.rows * a.cols;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int r = m0 + (wm * MT + i) * 32 + lr;
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int c = n0 + (wn * NT + j) * 32 + 8 * q + lc;
                    if (r >= a.rows) continue;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (c + e < a.cols) part[(int64_t)r * a.cols + c + e] = acc[i][j][4 * q + e];
                }
        }
        return;
    }
    // Results go through LDS, 32 rows of a wavefront at a time, so that they leave 16 bytes a lane in whole runs.
    __syncthreads();
    constexpr int RUN = KIND == GATED ? 32 : NT * 32, PITCH = RUN * 2 + 16;  // columns of a row; bytes between rows
    static_assert(WM * WN * 32 * PITCH <= 2 * (PB + QB), "the results' staging fits the tiles' place");
    unsigned char* mine = lds + wave * 32 * PITCH;
    const int c0 = n0 + wn * RUN;
    auto leave = [&](int i, __bf16* out, int64_t row, auto value) {  // value(j, e): result e of block j
#pragma unroll
        for (int j = 0; j < RUN / 32; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                u32x2 w;
                w.x = bf16_pair(value(j, 4 * q), value(j, 4 * q + 1));
                w.y = bf16_pair(value(j, 4 * q + 2), value(j, 4 * q + 3));
                *reinterpret_cast<u32x2*>(mine + lr * PITCH + (j * 32 + 8 * q + lc) * 2) = w;
            }
        __builtin_amdgcn_wave_barrier();
        constexpr int LANES = RUN / 8;  // a row's
#pragma unroll
        for (int t = 0; t < 32 * LANES / 64; ++t) {
            const int r = t * (64 / LANES) + lane / LANES, c = (lane % LANES) * 8;
            const u32x4 w = *reinterpret_cast<const u32x4*>(mine + r * PITCH + c * 2);
            const int gr = m0 + (wm * MT + i) * 32 + r, gc = c0 + c;
            if (gr >= a.rows) continue;
            __bf16* to = out + gr * row + gc;
            if (a.vec_out && gc + 8 <= a.cols) {
                *reinterpret_cast<u32x4*>(to) = w;
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (gc + e < a.cols) to[e] = __builtin_bit_cast(__bf16, (unsigned short)(w[e >> 1] >> (16 * (e & 1))));
            }
        }
        __builtin_amdgcn_wave_barrier();
    };
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        if constexpr (KIND == GATED) {
            static_assert(KIND != GATED || NT == 2, "a wavefront holds both projections of its columns");
            leave(i, a.out, a.out_row, [&](int, int e) { return act_value<ACT>(acc[i][0][e]) * acc[i][NT - 1][e]; });
            if (a.out2) {
                leave(i, a.out2, a.out2_row, [&](int, int e) { return acc[i][0][e]; });
                leave(i, a.out3, a.out2_row, [&](int, int e) { return acc[i][NT - 1][e]; });
            }
        } else {
            leave(i, half ? a.out2 : a.out, half ? a.out2_row : a.out_row, [&](int j, int e) { return acc[i][j][e]; });
        }
    }
}

// out = the splits' sums, in their order
__global__ __launch_bounds__(256) void join_kernel(const float* __restrict__ part, int splits, int rows, int cols, __bf16* __restrict__ out,
                                                   int64_t row) {
    const int64_t total = (int64_t)rows * cols;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        float s = 0.0f;
        for (int k = 0; k < splits; ++k) s += part[k * total + i];
        out[i / cols * row + i % cols] = (__bf16)s;
    }
}

// dG and dU from dH, G and U; rows of `pitch` elements, a multiple of eight, zeros behind column f (they are summed over).
// Eight columns a thread.
template <int ACT>
__global__ __launch_bounds__(256) void slopes_kernel(rrm_ff_desc d, src_t g, src_t u, src_t dh, int vec, int pitch, __bf16* __restrict__ dg,
                                                     __bf16* __restrict__ du) {
    const int64_t chunks = pitch / 8, total = chunks * d.m;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / chunks;
        const int f = (int)(i - r * chunks) * 8;
        float gv[8], uv[8], dv[8], og[8], ou[8];
        if (vec && f + 8 <= d.f) {
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

template <typename F>
void with_act(int act, F&& f) {
    switch (act) {
        case RRM_ACT_RELU: f(std::integral_constant<int, RRM_ACT_RELU>{}); break;
        case RRM_ACT_SILU: f(std::integral_constant<int, RRM_ACT_SILU>{}); break;
        case RRM_ACT_GELU: f(std::integral_constant<int, RRM_ACT_GELU>{}); break;
        default: f(std::integral_constant<int, RRM_ACT_NONE>{}); break;
    }
}

int tiles(int n, int of) { return (n + of - 1) / of; }

bool chunked(const void* p, int64_t row, int len) {  // rows of whole, aligned 16-byte chunks
    return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && row % 8 == 0 && len % 8 == 0;
}

template <int KIND, int ACT, bool PT, bool QT, int MT, int NT, int WM, int WN, bool RAGGED>
hipError_t launch_tiles(Product& a, hipStream_t s) {
    constexpr int BM = MT * 32 * WM, BN = NT * 32 * WN / (KIND == GATED ? 2 : 1);
    a.tiles_m = tiles(a.rows, BM) * (KIND == HALVES ? 2 : 1);
    a.tiles_n = tiles(a.cols, BN);
    hipLaunchKernelGGL((tile_kernel<KIND, ACT, PT, QT, MT, NT, WM, WN, RAGGED>), dim3((unsigned)(a.tiles_m * a.tiles_n), (unsigned)a.splits),
                       dim3(WM * WN * 64), 0, s, a);
    return hipGetLastError();
}
template <int KIND, int ACT, bool PT, bool QT>
hipError_t launch_product(Product& a, bool ragged, hipStream_t s) {
    if (ragged) return launch_tiles<KIND, ACT, PT, QT, 2, 2, 2, 2, true>(a, s);
    const int64_t big = (int64_t)tiles(a.rows, 256) * tiles(a.cols, KIND == GATED ? 128 : 256) * (KIND == HALVES ? 2 : 1);
    if (big >= OP_CUS) return launch_tiles<KIND, ACT, PT, QT, 4, 2, 2, 4, false>(a, s);
    return launch_tiles<KIND, ACT, PT, QT, 2, 2, 2, 2, false>(a, s);
}

size_t grads_bytes(const rrm_ff_desc& d) { return round256((size_t)d.m * ((d.f + 7) / 8 * 8) * 2); }

}  // namespace

size_t ff_scratch(const rrm_ff_desc& d, bool backward) { return backward ? 2 * grads_bytes(d) : 0; }

hipError_t launch_gated_ff(const rrm_ff_desc& d, const void* x, const void* wg, const void* wu, void* h, void* g, void* u, void*,
                           hipStream_t s) {
    Product a{};
    a.p[0] = {(src_t)x, d.x_row};
    a.q[0] = {(src_t)wg, d.wg_row};
    a.q[1] = {(src_t)wu, d.wu_row};
    a.pairs = 1, a.splits = 1;
    a.rows = d.m, a.cols = d.f, a.len = d.k;
    a.out = (__bf16*)h, a.out2 = (__bf16*)g, a.out3 = (__bf16*)u;
    a.out_row = d.h_row, a.out2_row = d.gu_row;
    a.vec_out = chunked(h, d.h_row, 8) && (!g || (chunked(g, d.gu_row, 8) && chunked(u, d.gu_row, 8)));
    const bool ragged = !chunked(x, d.x_row, d.k) || !chunked(wg, d.wg_row, d.k) || !chunked(wu, d.wu_row, d.k);
    hipError_t e = hipSuccess;
    with_act(d.act, [&](auto act) { e = launch_product<GATED, decltype(act)::value, false, false>(a, ragged, s); });
    return e;
}

hipError_t launch_gated_ff_backward(const rrm_ff_desc& d, const void* x, const void* wg, const void* wu, const void* g,
                                    const void* u, const void* dh, void* dx, void* dwg, void* dwu, void* ws, hipStream_t s) {
    __bf16* dg = (__bf16*)ws;
    __bf16* du = (__bf16*)((char*)ws + grads_bytes(d));
    const int pitch = (d.f + 7) / 8 * 8;
    if (d.m > 0) {
        const int64_t chunks = (int64_t)d.m * (pitch / 8), groups = (chunks + 255) / 256;
        const int vec = chunked(g, d.gu_row, 8) && chunked(u, d.gu_row, 8) && chunked(dh, d.h_row, 8);
        with_act(d.act, [&](auto act) {
            hipLaunchKernelGGL((slopes_kernel<decltype(act)::value>), dim3((unsigned)(groups < OP_CUS * 32 ? groups : OP_CUS * 32)), dim3(256),
                               0, s, d, (src_t)g, (src_t)u, (src_t)dh, vec, pitch, dg, du);
        });
        if (hipError_t e = hipGetLastError()) return e;
        if (dx) {
            Product a{};
            a.p[0] = {dg, pitch}, a.p[1] = {du, pitch};
            a.q[0] = {(src_t)wg, d.wg_row}, a.q[1] = {(src_t)wu, d.wu_row};
            a.pairs = 2, a.splits = 1;
            a.rows = d.m, a.cols = d.k, a.len = d.f;
            a.out = (__bf16*)dx, a.out_row = d.dx_row;
            a.vec_out = chunked(dx, d.dx_row, 8);
            const bool ragged = !chunked(wg, d.wg_row, d.k) || !chunked(wu, d.wu_row, d.k);
            if (hipError_t e = launch_product<PLAIN, RRM_ACT_NONE, false, true>(a, ragged, s)) return e;
        }
    }
    if (dwg) {
        Product a{};
        a.p[0] = {dg, pitch}, a.p[1] = {du, pitch};
        a.q[0] = {(src_t)x, d.x_row};
        a.pairs = 1, a.splits = 1;
        a.rows = d.f, a.cols = d.k, a.len = d.m;
        a.out = (__bf16*)dwg, a.out_row = d.dwg_row, a.out2 = (__bf16*)dwu, a.out2_row = d.dwu_row;
        a.vec_out = chunked(dwg, d.dwg_row, 8) && chunked(dwu, d.dwu_row, 8);
        const bool ragged = !chunked(x, d.x_row, d.k);
        if (hipError_t e = launch_product<HALVES, RRM_ACT_NONE, true, true>(a, ragged, s)) return e;
    }
    return hipSuccess;
}

}  // namespace rrm
