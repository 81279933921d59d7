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
    float* part;            // [splits][rows][cols, to whole fours] (gated, halves: [splits][2][rows][..])
};

enum Kind : int { GATED = 0, PLAIN = 1, HALVES = 2 };

// The turn of the 64-byte windows of row k of a turned tile in LDS: see tile_product
template <int WINDOWS>
__device__ __forceinline__ int window_turn(int k) {
    return WINDOWS >= 8 ? (k & 3) | ((k >> 1) & 4) : WINDOWS == 4 ? (k & 3) : WINDOWS == 2 ? ((k >> 1) & 1) : 0;
}

// Until at most N of this wavefront's copies to LDS are on their way (they end in the order of their start), and its LDS accesses are done
template <int N>
__device__ __forceinline__ void wait_copies() {
    static_assert(N < 64);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
}
// no waits of its own: those are the callers'
__device__ __forceinline__ void barrier() { asm volatile("s_barrier" ::: "memory"); }

// Eight elements at the alignment of one.
struct __attribute__((packed, aligned(2))) Loose {
    u32x4 v;
};
__device__ __forceinline__ u32x4 loose_chunk(src_t p) { return reinterpret_cast<const Loose*>(p)->v; }
// eight elements of a row of `len`, from element k on; zeros behind the end
__device__ __forceinline__ u32x4 ragged_chunk(src_t row, int k, int len) {
    if (k + 8 <= len) return loose_chunk(row + k);
    unsigned short e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = k + i < len ? __builtin_bit_cast(unsigned short, row[k + i]) : (unsigned short)0;
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (unsigned int)e[2 * i] | ((unsigned int)e[2 * i + 1] << 16);
    return w;
}

// A tile of a product on the matrix cores, v_mfma_f32_32x32x16_bf16.
//
// A workgroup of WM x WN wavefronts makes (32 MT WM) x (32 NT WN) results.  Operands go from memory to LDS directly, 64 of the summed axis at
// a time, STAGES steps ahead; a wavefront reads a fragment for each of its MT + NT rows of blocks and multiplies MT x NT pairs of them.  With 256 x 256
// results (4 x 2 blocks of 2 x 4 wavefronts) that is a byte copied for 64 multiplications, and 3/4 of a fragment read from LDS for each product.
// What feeds the matrix cores without a pause: fragments of the next 16 are read between the products of these; copies are started in
// parts between products; one barrier a step, before its last quarter, so that the next step's first fragments are there when it ends; LDS
// turned so that reads meet different banks (conflicts 6% of its busy cycles; half without).
//
// Measured, 16384 x 4096 rows x 4096 features of each projection: 955 us forward with G and U kept, 1.15 PFLOP/s; dX 910 us, 1.21; both dW 890
// us, 1.24.  A library's plain products of these shapes, nothing fused, reach 1.40, 1.23 and 1.10 PFLOP/s.  The matrix cores
// are busy 69% of the cycles, at the 1.67 GHz that the card's power allows: on rows of equal values the same program runs at 2.0 GHz and takes 732 us,
// and 4% fewer cycles, all operands being in the nearest caches.  Four wavefronts of 128 x 128 results took 932 us where eight took 900; a raised
// wave priority, non-temporal results and copies spread one by one between the products changed nothing.
template <int MT, int NT, int WM, int WN, int STAGES>
constexpr int TILE_LDS = STAGES * (MT * 32 * WM + NT * 32 * WN) * STEP * 2;

template <int KIND, int ACT, bool PT, bool QT, int MT, int NT, int WM, int WN, int STAGES>
__device__ __forceinline__ void tile_product(const Product& a, unsigned char* lds, int id, int split) {
    constexpr int THREADS = WM * WN * 64, BM = MT * 32 * WM, BN = NT * 32 * WN;
    constexpr int PB = BM * STEP * 2, QB = BN * STEP * 2;                       // bytes of a staged tile
    constexpr int NP = PB / (THREADS * 16), NQ = QB / (THREADS * 16);          // 16-byte chunks a thread stages
    constexpr int OUT_COLS = KIND == GATED ? BN / 2 : BN;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int wm = wave % WM, wn = wave / WM;

    // tiles XCD by XCD (workgroups go to the eight in turn), and there in blocks of eight rows of tiles
    int tm, tn;
    {
        const int total = a.tiles_m * a.tiles_n, xcd = id & 7, q = total >> 3, r = total & 7;
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
            pk[i] = (((at % 128) / 16) ^ ((r >> 1) & 7)) * 8;
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
            qk[i] = (((at % 128) / 16) ^ ((r >> 1) & 7)) * 8;
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
    // The copies of a step are started in three parts, between products, so that these do not queue behind all of them
    auto begin = [&](int s) __attribute__((always_inline)) {  // step s is next
        const int pair = KIND == PLAIN && s >= steps_of ? 1 : 0;
        if (KIND == PLAIN && s == steps_of) point(s);
        const int rem = a.len - (s - pair * steps_of) * STEP;
        if (rem < STEP) {  // the summed axis ends in it
#pragma unroll
            for (int i = 0; i < NP; ++i) pp[i] = pk[i] < rem ? pp[i] : zeros;
#pragma unroll
            for (int i = 0; i < NQ; ++i) qp[i] = qk[i] < rem ? qp[i] : zeros;
        }
    };
    auto part = [&](auto which, unsigned char* dp) __attribute__((always_inline)) {
        constexpr int W = decltype(which)::value, PARTS = STAGES == 2 ? 2 : 3;
        constexpr int FROM = (NP + NQ) * (W < PARTS ? W : PARTS) / PARTS, TO = (NP + NQ) * (W + 1 < PARTS ? W + 1 : PARTS) / PARTS;
#pragma unroll
        for (int i = FROM; i < TO; ++i)
            if (i < NP)
                __builtin_amdgcn_global_load_lds((gptr_t)pp[i < NP ? i : 0], (lptr_t)(dp + (i * THREADS + wave * 64) * 16), 16, 0, 0);
            else
                __builtin_amdgcn_global_load_lds((gptr_t)qp[i < NP ? 0 : i - NP], (lptr_t)(dp + PB + ((i - NP) * THREADS + wave * 64) * 16), 16, 0, 0);
    };
    auto end = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NP; ++i) pp[i] += p_step;
#pragma unroll
        for (int i = 0; i < NQ; ++i) qp[i] += q_step;
    };
    const std::integral_constant<int, 0> one;
    const std::integral_constant<int, 1> two;
    const std::integral_constant<int, 2> three;

    v16f acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;

    // Fragment reads: lane l holds row l % 32 and eight of the summed axis, (l / 32) * 8 on in a step of 16
    const int flat = (lane & 31) * 128 + (((lane >> 5) ^ ((lane >> 1) & 7)) << 4);
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

    // Fragments of 16 of the summed axis are read while those before are multiplied, across steps as well: the barrier that publishes
    // the next step stands before the last products of this one.
    v8bf fp[2][MT], fq[2][NT];
    auto place = [&](int i) { return lds + i * (PB + QB); };
    auto fragments = [&](int set, const unsigned char* tp, int ks) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < NT; ++j) fq[set][j] = frag(tp + PB, (wn * NT + j) * 32, ks, q_turned, q_rows);
#pragma unroll
        for (int i = 0; i < MT; ++i) fp[set][i] = frag(tp, (wm * MT + i) * 32, ks, p_turned, p_rows);
    };
    auto products = [&](int set) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fq[set][j], fp[set][i], acc[i][j], 0, 0, 0);
        // one product, one read, ..
        constexpr int READS = MT * (PT ? 2 : 1) + NT * (QT ? 2 : 1), ALL = MT * NT, EACH = (2 * READS + ALL - 1) / ALL;
#pragma unroll
        for (int i = 0; i < ALL; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, EACH, 0);
        }
        __builtin_amdgcn_sched_barrier(0);  // (reads of the next group would be waited for with those of this one)
    };
    if (s0 < s1) {
        point(s0);
#pragma unroll
        for (int i = 0; i < STAGES; ++i)
            if (s0 + i < s1) {
                begin(s0 + i);
                part(one, place(i));
                part(two, place(i));
                part(three, place(i));
                end();
            }
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        fragments(0, lds, 0);
        fragments(1, lds, 1);
        products(0);
        fragments(0, lds, 2);
        products(1);
        fragments(1, lds, 3);
        products(0);
        // From here on a turn takes the last quarter of step s and three of the next one.  `from` and `to` never overlap, which the compiler
        // has to know: it would wait for the copies to `to` before each transposing read of `from`.
        auto turn = [&](const unsigned char* __restrict from, unsigned char* __restrict to) __attribute__((always_inline)) {
            part(one, to);
            fragments(0, from, 0);
            products(1);
            part(two, to);
            fragments(1, from, 1);
            products(0);
            part(three, to);
            fragments(0, from, 2);
            products(1);
            fragments(1, from, 3);
            products(0);
        };
        int s = s0, buf = 0;  // place of step s
        for (; s + STAGES < s1; ++s) {
            const int after = buf + 1 == STAGES ? 0 : buf + 1;
            // this wavefront's copies of the next step have landed (those of later steps may still be on their way), and its reads
            // of this one are done ..
            wait_copies<(STAGES - 2) * (NP + NQ)>();
            barrier();  // .. and so are everybody's
            begin(s + STAGES);
            turn(place(after), place(buf));
            end();
            buf = after;
        }
        for (; s + 1 < s1; ++s) {  // nothing left to be copied
            const int after = buf + 1 == STAGES ? 0 : buf + 1;
            wait_copies<0>();
            barrier();
            fragments(0, place(after), 0);
            products(1);
            fragments(1, place(after), 1);
            products(0);
            fragments(0, place(after), 2);
            products(1);
            fragments(1, place(after), 3);
            products(0);
            buf = after;
        }
        products(1);
    }

    // acc[i][j][4 q + e] of lane l: row (wm MT + i) 32 + l % 32, column (wn NT + j) 32 + 8 q + 4 (l / 32) + e
    const int lr = lane & 31, lc = (lane >> 5) * 4;
    if (a.splits > 1) {
        constexpr int WAYS = KIND == GATED ? 2 : 1;  // results interleaved in a wavefront's blocks of 32 columns
        const int pitch = (a.cols + 3) & ~3;
        const int64_t plane = (int64_t)a.rows * pitch;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int r = m0 + (wm * MT + i) * 32 + lr;
            if (r >= a.rows) continue;
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                float* to = a.part + (int64_t)(KIND == HALVES ? 2 * split + half : split * WAYS + j % WAYS) * plane + r * (int64_t)pitch;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int c = n0 + (wn * NT + j) / WAYS * 32 + 8 * q + lc;
                    if (c < pitch)
                        *reinterpret_cast<float4*>(to + c) = make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
                }
            }
        }
        return;
    }
    // Results go through LDS, 32 rows of a wavefront at a time, so that they leave 16 bytes a lane in whole runs.
    __syncthreads();
    constexpr int RUN = (KIND == GATED ? NT / 2 : NT) * 32, PITCH = RUN * 2 + 16;  // columns of a row; bytes between rows
    static_assert(WM * WN * 32 * PITCH <= STAGES * (PB + QB), "the results' staging fits the tiles' place");
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
            if (gc + 8 <= a.cols) {
                reinterpret_cast<Loose*>(to)->v = w;
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
            static_assert(KIND != GATED || NT % 2 == 0, "a wavefront holds both projections of its columns");
            leave(i, a.out, a.out_row, [&](int j, int e) { return act_value<ACT>(acc[i][2 * j][e]) * acc[i][2 * j + 1][e]; });
            if (a.out2) {
                leave(i, a.out2, a.out2_row, [&](int j, int e) { return acc[i][2 * j][e]; });
                leave(i, a.out3, a.out2_row, [&](int j, int e) { return acc[i][2 * j + 1][e]; });
            }
        } else {
            leave(i, half ? a.out2 : a.out, half ? a.out2_row : a.out_row, [&](int j, int e) { return acc[i][j][e]; });
        }
    }
}

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

int tiles(int n, int of) { return (n + of - 1) / of; }
int round8(int n) { return (n + 7) & ~7; }

template <int KIND, int ACT, bool PT, bool QT, int MT, int NT, int WM, int WN, int STAGES>
hipError_t launch_tiles(Product& a, hipStream_t s) {
    constexpr int BM = MT * 32 * WM, BN = NT * 32 * WN / (KIND == GATED ? 2 : 1);
    a.tiles_m = tiles(a.rows, BM) * (KIND == HALVES ? 2 : 1);
    a.tiles_n = tiles(a.cols, BN);
    hipLaunchKernelGGL((tile_kernel<KIND, ACT, PT, QT, MT, NT, WM, WN, STAGES>), dim3((unsigned)(a.tiles_m * a.tiles_n), (unsigned)a.splits),
                       dim3(WM * WN * 64), 0, s, a);
    return hipGetLastError();
}
// Tile shapes (gated: the columns are both projections').  A step of 64 of the summed axis takes, with `count` workgroups,
// about first * rounds + second * count / 256 us, a round being as many workgroups as run at once (measured: 4096 -> 4096 and 4096 -> 9216
// features, 64 to 16384 rows); the shape and the number of parts of the summed axis with the least of it are taken.
struct Shape {
    int bm, bn, at_once;
    float first, second;
};
enum Which : int { BIG = 0, WIDE = 1, WIDE_PAIR = 2, SMALL = 3 };
constexpr Shape SHAPES[] = {
    {256, 256, 256, 1.4f, 0.6f}, {128, 128, 256, 0.6f, 0.1f}, {128, 128, 512, 0.85f, 0.2f}, {64, 128, 512, 0.45f, 0.2f},
};
struct Plan {
    int shape, splits, splits2;  // parts of the summed axis (of the second product)
    float us;
};
constexpr float LAUNCH_US = 6.0f;  // what a launch of tiles takes beside its steps: its start, its first copies, its results
struct Work {  // a product of rows x cols, `ways` of them, over `steps` steps each
    int rows, cols, steps, ways;
};
// The least estimate for a product, or two in one launch (b.steps > 0); `bytes`: what comes from memory at the least, at some 4 TB/s.
Plan plan_products(const Work& a, const Work& b, float bytes) {
    Plan best{SMALL, 1, 1, 1e30f};
    for (int w = BIG; w <= SMALL; ++w) {
        const Shape& h = SHAPES[w];
        const int64_t ta = (int64_t)tiles(a.rows, h.bm) * tiles(a.cols, h.bn) * a.ways;
        const int64_t tb = b.steps ? (int64_t)tiles(b.rows, h.bm) * tiles(b.cols, h.bn) * b.ways : 0;
        for (int sa = 1; sa <= 16 && (sa == 1 || a.steps / sa >= 4); sa *= 2)
            for (int sb = 1; sb <= 16 && (sb == 1 || b.steps / sb >= 4); sb *= 2) {
                const int ea = tiles(a.steps, sa), eb = tiles(b.steps, sb), longest = ea > eb ? ea : eb;
                const int64_t groups = ta * sa + tb * sb, all = ta * sa * ea + tb * sb * eb;
                // rounds of the longest workgroups' steps; two products share them by their steps
                const int64_t rounds = (groups + h.at_once - 1) / h.at_once;
                float steps = (float)rounds * longest;
                if (b.steps && rounds > 1) steps = (float)all / h.at_once + 0.5f * longest;
                float us = steps * h.first + (float)all / OP_CUS * h.second;
                if (us < bytes / 4e6f) us = bytes / 4e6f;
                // the sums' way through memory and the launch that joins them
                if (sa > 1 || sb > 1) us += 5.0f;
                if (sa > 1) us += (float)sa * a.ways * a.rows * (float)a.cols * 8.0f / 6e6f;
                if (sb > 1) us += (float)sb * b.ways * b.rows * (float)b.cols * 8.0f / 6e6f;
                us += LAUNCH_US;
                if (us < best.us) best = Plan{w, sa, sb, us};
            }
    }
    return best;
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
