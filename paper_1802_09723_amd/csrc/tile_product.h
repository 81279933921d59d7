// Tiles of products on the matrix cores, for the operators whose work is one: operands of 16-bit elements from memory through LDS, sums in 32 bits.
#pragma once
#include "op_common.h"

namespace rrm {

namespace {

typedef const __bf16* src_t;
typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
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

// BLEND: out = alpha * the product + beta * blend, of half-precision operands.  `blend` lies [rows][cols] in rows of whole eights, what its rounding left
// off beside it where with_rest is not NULL; out's lies by out's row at out_rest.
struct Blend {
    const _Float16 *with, *with_rest;  // (not read where beta is 0)
    int64_t row;
    float alpha, beta;
    bool to_bf16;  // out is bfloat16, else half precision like the operands
    _Float16* out_rest;
};

enum Kind : int { GATED = 0, PLAIN = 1, HALVES = 2, BLEND = 3 };

__device__ __forceinline__ unsigned int half_pair(float lo, float hi) {
    f16x2 v;
    v[0] = (_Float16)lo;
    v[1] = (_Float16)hi;
    return __builtin_bit_cast(unsigned int, v);
}

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
__device__ __forceinline__ void tile_product(const Product& a, unsigned char* lds, int id, int split, const Blend& blend = Blend{}) {
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
            for (int j = 0; j < NT; ++j)
                if constexpr (KIND == BLEND)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8h, fq[set][j]), __builtin_bit_cast(v8h, fp[set][i]), acc[i][j], 0, 0, 0);
                else
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fq[set][j], fp[set][i], acc[i][j], 0, 0, 0);
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
                if (KIND == BLEND && !blend.to_bf16) {
                    w.x = half_pair(value(j, 4 * q), value(j, 4 * q + 1));
                    w.y = half_pair(value(j, 4 * q + 2), value(j, 4 * q + 3));
                } else {
                    w.x = bf16_pair(value(j, 4 * q), value(j, 4 * q + 1));
                    w.y = bf16_pair(value(j, 4 * q + 2), value(j, 4 * q + 3));
                }
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
        } else if constexpr (KIND == BLEND) {
            const int r = m0 + (wm * MT + i) * 32 + lr;
            auto blended = [&](const _Float16* with) __attribute__((always_inline)) {
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int c = c0 + j * 32 + 8 * q + lc;
                        const u32x2 d = r < a.rows && c < a.cols ? *reinterpret_cast<const u32x2*>(with + r * blend.row + c) : u32x2{0, 0};
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const unsigned int pair = e & 2 ? d.y : d.x;
                            acc[i][j][4 * q + e] += blend.beta * (float)__builtin_bit_cast(_Float16, (unsigned short)(pair >> (16 * (e & 1))));
                        }
                    }
            };
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] *= blend.alpha;
            if (blend.beta != 0.0f) {
                if (blend.with_rest) blended(blend.with_rest);
                blended(blend.with);
            }
            leave(i, a.out, a.out_row, [&](int j, int e) { return acc[i][j][e]; });
            if (blend.out_rest) leave(i, (__bf16*)blend.out_rest, a.out_row, [&](int j, int e) { return acc[i][j][e] - (float)(_Float16)acc[i][j][e]; });
        } else {
            leave(i, half ? a.out2 : a.out, half ? a.out2_row : a.out_row, [&](int j, int e) { return acc[i][j][e]; });
        }
    }
}

int tiles(int n, int of) { return (n + of - 1) / of; }
int round8(int n) { return (n + 7) & ~7; }

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

}  // namespace

}  // namespace rrm
