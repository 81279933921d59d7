// A weight's update made orthogonal by Newton-Schulz products:
//
//      X = G / (|G| + eps);        `steps` times:  A = X X^T        X <- a X + (b A + c A^2) X
//
// (rows > cols: A = X^T X, X <- a X + X (b A + c A^2)).  Singular value by singular value this is s <- a s + b s^3 + c s^5, and singular vectors stay.
// Three products a step on the matrix cores.  X, A and b A + c A^2 meet memory in half precision, whose eleven bits are eight times as fine as
// bfloat16's at the same rate: a product's rounding errors are taken up by the ones behind it, and with bfloat16 the result would be off by some 1.5%.
// a X, which carries a step's X into the next, is made of X in two parts, the second what the first's rounding left off: the errors of X do not stay (relative error
// of the result beside its own rounding, 256 x 256 and 128 x 512 with a few directions far above the others: 0.0010 and 0.0013, with the first part alone 0.0027 and
// 0.0020; where all directions are alike 0.0016 and 0.0017 instead of 0.0014).
// Half precision ends at 6e-8: X is held at 256 times its size, so that singular values that a few steps still raise to 1 are above its rounding
// (those of A do not need it: what it lacks is small against a).
#include "tile_product.h"

namespace rrm {

namespace {

constexpr float HELD = 256.0f;
constexpr int SUM_PARTS = 256;  // workgroups that sum a matrix's squares

__device__ __forceinline__ double block_sum(double v, double* place) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m);
    if ((threadIdx.x & 63) == 0) place[threadIdx.x >> 6] = v;
    __syncthreads();
    return (place[0] + place[1]) + (place[2] + place[3]);
}

// Squares are summed in 64 bits: no scale of G overflows or vanishes.
template <typename T>
__global__ __launch_bounds__(256) void squares_kernel(rrm_orth_desc d, const T* g, double* part) {
    __shared__ double place[4];
    g += blockIdx.y * d.g_matrix;
    const int chunks = (d.cols + 7) / 8;
    const int64_t total = (int64_t)chunks * d.rows;
    double sum = 0.0;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / chunks;
        const int c = (int)(i - r * chunks) * 8;
        const T* at = g + r * d.g_row + c;
        float v[8];
        if (c + 8 <= d.cols) load_vec<8>(at, v);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = c + e < d.cols ? load_elem(at + e) : 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += (double)v[e] * v[e];
    }
    sum = block_sum(sum, place);
    if (threadIdx.x == 0) part[blockIdx.y * SUM_PARTS + blockIdx.x] = sum;
}

// X = 256 G / (|G| + eps) in rows of `pitch`, zeros behind the last column
template <typename T>
__global__ __launch_bounds__(256) void scaled_kernel(rrm_orth_desc d, const T* g, const double* part, _Float16* x, _Float16* rest, _Float16* next, int pitch, int64_t plane) {
    __shared__ double place[4];
    double sum = threadIdx.x < SUM_PARTS ? part[blockIdx.y * SUM_PARTS + threadIdx.x] : 0.0;
    sum = block_sum(sum, place);
    const double factor = HELD / (sqrt(sum) + d.eps);
    g += blockIdx.y * d.g_matrix;
    x += blockIdx.y * plane;
    rest += blockIdx.y * plane;
    next += blockIdx.y * plane;
    const int chunks = pitch / 8;
    const int64_t total = (int64_t)chunks * d.rows;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / chunks;
        const int c = (int)(i - r * chunks) * 8;
        const T* at = g + r * d.g_row + c;
        float v[8];
        if (c + 8 <= d.cols) load_vec<8>(at, v);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = c + e < d.cols ? load_elem(at + e) : 0.0f;
        u32x4 w, left;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            // (a matrix of zeros with eps = 0 stays one)
            const float lo = v[2 * e] == 0.0f ? 0.0f : (float)(v[2 * e] * factor), hi = v[2 * e + 1] == 0.0f ? 0.0f : (float)(v[2 * e + 1] * factor);
            w[e] = half_pair(lo, hi);
            left[e] = half_pair(lo - (float)(_Float16)lo, hi - (float)(_Float16)hi);
        }
        *reinterpret_cast<u32x4*>(x + r * pitch + c) = w;
        *reinterpret_cast<u32x4*>(rest + r * pitch + c) = left;
        if (c + 8 > d.cols) *reinterpret_cast<u32x4*>(next + r * pitch + c) = u32x4{0, 0, 0, 0};  // (the step after leaves these zeros)
    }
}

// Zeros behind the last column of rows of `pitch`, which products sum over
__global__ __launch_bounds__(256) void edge_kernel(_Float16* p, int64_t rows, int cols, int pitch) {
    for (int64_t r = (int64_t)blockIdx.x * 256 + threadIdx.x; r < rows; r += (int64_t)gridDim.x * 256)
        for (int c = cols; c < pitch; ++c) p[r * pitch + c] = (_Float16)0.0f;
}

// A of split sums, in their order: sums [split][matrix][few][pitch]
__global__ __launch_bounds__(256) void gram_kernel(const float* part, int splits, int64_t all, int few, int pitch, int few_pitch, float alpha, _Float16* a) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all / 4; i += (int64_t)gridDim.x * 256) {
        float4 s = *reinterpret_cast<const float4*>(part + 4 * i);
        for (int k = 1; k < splits; ++k) {
            const float4 v = *reinterpret_cast<const float4*>(part + k * all + 4 * i);
            s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
        }
        const int64_t r = 4 * i / pitch;
        const int c = (int)(4 * i - r * pitch);
        const float v[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < few) a[r * few_pitch + c + e] = (_Float16)(alpha * v[e]);
    }
}

// Up to 128 rows: A of its split sums and b A + c A^2 at once, a workgroup a matrix.  A is in LDS only; rows of 128 there, zeros behind the last.
constexpr int POLY = 128;
__global__ __launch_bounds__(1024) void poly_kernel(const float* part, int splits, int64_t all, int few, int pitch, int few_pitch, float alpha, float b, float c,
                                                   _Float16* out) {
    constexpr int ROW = POLY * 2 + 16;  // bytes
    __shared__ __attribute__((aligned(16))) unsigned char lds[POLY * ROW];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, half = lane >> 5, lr = lane & 31;
    part += (int64_t)blockIdx.x * few * pitch;
    out += (int64_t)blockIdx.x * few * few_pitch;
    constexpr int OWN = POLY * POLY / 4 / 1024;  // fours of a thread
    const int blocks = (few + 31) / 32;
    float4 sum[OWN];
#pragma unroll
    for (int i = 0; i < OWN; ++i) sum[i] = make_float4(0, 0, 0, 0);
#pragma unroll 4
    for (int j = 0; j < splits; ++j)
#pragma unroll
        for (int i = 0; i < OWN; ++i) {
            const int r = (tid + i * 1024) / (POLY / 4), k = tid % (POLY / 4) * 4;
            if (r >= few || k >= few) continue;  // (pitch: whole fours)
            const float4 v = *reinterpret_cast<const float4*>(part + j * all + r * pitch + k);
            sum[i].x += v.x, sum[i].y += v.y, sum[i].z += v.z, sum[i].w += v.w;
        }
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
        const int r = (tid + i * 1024) / (POLY / 4), k = tid % (POLY / 4) * 4;
        const float4 s = sum[i];
        *reinterpret_cast<u32x2*>(lds + r * ROW + k * 2) =
            u32x2{half_pair(k < few ? s.x * alpha : 0.0f, k + 1 < few ? s.y * alpha : 0.0f), half_pair(k + 2 < few ? s.z * alpha : 0.0f, k + 3 < few ? s.w * alpha : 0.0f)};
    }
    __syncthreads();
    const int i = wave >> 2, j = wave & 3;  // a block of 32 x 32 a wavefront
    if (i >= blocks || j >= blocks) return;
    {
        v16f acc;
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[e] = 0.0f;
#pragma unroll
        for (int s = 0; s < POLY / 16; ++s) {
            const v8h q = *reinterpret_cast<const v8h*>(lds + (j * 32 + lr) * ROW + s * 32 + half * 16), p = *reinterpret_cast<const v8h*>(lds + (i * 32 + lr) * ROW + s * 32 + half * 16);
            acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(q, p, acc, 0, 0, 0);
        }
        // register 4 q + e: row 32 i + l % 32, column 32 j + 8 q + 4 (l / 32) + e
        const int r = i * 32 + lr;
        if (r >= few) return;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int k = j * 32 + 8 * q + 4 * half;
            if (k >= few_pitch) continue;
            const u32x2 w = *reinterpret_cast<const u32x2*>(lds + r * ROW + k * 2);
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned int pair = e & 2 ? w.y : w.x;
                v[e] = b * (float)__builtin_bit_cast(_Float16, (unsigned short)(pair >> (16 * (e & 1)))) + c * acc[4 * q + e];
            }
            *reinterpret_cast<u32x2*>(out + r * few_pitch + k) = u32x2{half_pair(v[0], v[1]), half_pair(v[2], v[3])};  // (zeros behind the last column)
        }
    }
}

// Matrices of up to 128 x 512 (or 512 x 128): all steps in one launch, a workgroup a matrix.  X is in registers in 32 bits, 32 columns a wavefront, and in
// LDS in half precision, as are A and then b A + c A^2: 160 KB for the largest.  The sixteen bytes of a row that reads ask for together are turned by
// the row's number (XOR), so that rows meet different banks.  128 x 512: 54 us, most of it
// a step's chain of LDS reads, products and barriers on one compute unit (some 9 us a step); by launches of products 90, each a start and a trip to memory.
constexpr int SMALL_FEW = 128, SMALL_MANY = 512;
typedef __attribute__((address_space(3))) v4s* turned_t;
template <typename T>
__global__ __launch_bounds__(1024) void small_kernel(rrm_orth_desc d, const T* g, __bf16* out) {
    __shared__ __attribute__((aligned(256))) unsigned char lds[SMALL_FEW * SMALL_MANY * 2 + SMALL_FEW * SMALL_FEW * 2];
    unsigned char *const xs = lds, *const as = lds + SMALL_FEW * SMALL_MANY * 2;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, half = lane >> 5, lr = lane & 31;
    const bool tall = d.rows > d.cols;
    const int few = tall ? d.cols : d.rows, many = tall ? d.rows : d.cols, nb = (few + 31) / 32, cb = (many + 31) / 32;
    g += blockIdx.x * d.g_matrix;
    out += blockIdx.x * d.x_matrix;
    auto x_at = [&](int row, int chunk) { return xs + row * (SMALL_MANY * 2) + ((chunk ^ (row & 7)) << 4); };
    auto a_at = [&](int row, int chunk) { return as + row * (SMALL_FEW * 2) + ((chunk ^ (row & 7)) << 4); };
    // element r of block ib: row 32 ib + l % 32, column 32 wave + 8 (r / 4) + 4 half + r % 4
    const int col0 = wave * 32 + half * 4;
    v16f x[4];
    double sum = 0.0;
    if (tall) {  // neighbouring lanes have neighbouring values of G
#pragma unroll
        for (int ib = 0; ib < 4; ++ib)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int row = ib * 32 + lr, col = col0 + (r >> 2) * 8 + (r & 3);
                x[ib][r] = row < few && col < many ? load_elem(g + col * d.g_row + row) : 0.0f;
            }
    } else {  // 32 whole rows at a time through LDS: read as they lie in rows apart they would take 27 us
        constexpr int ROW = SMALL_MANY * 4 + 16, QUADS = SMALL_MANY / 4;
#pragma unroll
        for (int ib = 0; ib < 4; ++ib) {
            if (ib > 0) __syncthreads();
            if (ib < nb)
#pragma unroll
                for (int k = 0; k < 32 * QUADS / 1024; ++k) {
                    const int at = k * 1024 + tid, row = at / QUADS, col = at % QUADS * 4;
                    const T* from = g + (ib * 32 + row) * d.g_row + col;
                    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                    if (ib * 32 + row < few && col < many) {
                        if (col + 4 <= many) load_vec<4>(from, v);
                        else
#pragma unroll
                            for (int e = 0; e < 3; ++e)
                                if (col + e < many) v[e] = load_elem(from + e);
                    }
                    *reinterpret_cast<float4*>(lds + row * ROW + col * 4) = make_float4(v[0], v[1], v[2], v[3]);
                }
            __syncthreads();
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float4 v = ib < nb ? *reinterpret_cast<const float4*>(lds + lr * ROW + (col0 + 8 * q) * 4) : make_float4(0, 0, 0, 0);
                x[ib][4 * q] = v.x, x[ib][4 * q + 1] = v.y, x[ib][4 * q + 2] = v.z, x[ib][4 * q + 3] = v.w;
            }
        }
        __syncthreads();
    }
#pragma unroll
    for (int ib = 0; ib < 4; ++ib)
#pragma unroll
        for (int r = 0; r < 16; ++r) sum += (double)x[ib][r] * x[ib][r];
    double* const place = reinterpret_cast<double*>(as);
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) sum += __shfl_xor(sum, m);
    if (lane == 0) place[wave] = sum;
    __syncthreads();
    sum = 0.0;
    for (int i = 0; i < 16; ++i) sum += place[i];
    const double factor = HELD / (sqrt(sum) + d.eps);
#pragma unroll
    for (int ib = 0; ib < 4; ++ib)
#pragma unroll
        for (int r = 0; r < 16; ++r) x[ib][r] = x[ib][r] == 0.0f ? 0.0f : (float)(x[ib][r] * factor);  // (zeros with eps = 0 stay zeros)
    auto put = [&]() __attribute__((always_inline)) {
        if (wave < cb)
#pragma unroll
            for (int ib = 0; ib < 4; ++ib)
                if (ib < nb)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        *reinterpret_cast<u32x2*>(x_at(ib * 32 + lr, wave * 4 + q) + half * 8) =
                            u32x2{half_pair(x[ib][4 * q], x[ib][4 * q + 1]), half_pair(x[ib][4 * q + 2], x[ib][4 * q + 3])};
    };
    put();
    __syncthreads();
    const int i = wave >> 2, j = wave & 3;  // this wavefront's block of A
    for (int step = 0; step < d.steps; ++step) {
        if (i <= j && j < nb) {
            v16f acc;
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[e] = 0.0f;
#pragma unroll 4
            for (int s = 0; s < 2 * cb; ++s)
                acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const v8h*>(x_at(j * 32 + lr, 2 * s + half)),
                                                             *reinterpret_cast<const v8h*>(x_at(i * 32 + lr, 2 * s + half)), acc, 0, 0, 0);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const u32x2 w = {half_pair(acc[4 * q] * (1.0f / (HELD * HELD)), acc[4 * q + 1] * (1.0f / (HELD * HELD))),
                                 half_pair(acc[4 * q + 2] * (1.0f / (HELD * HELD)), acc[4 * q + 3] * (1.0f / (HELD * HELD)))};
                *reinterpret_cast<u32x2*>(a_at(i * 32 + lr, j * 4 + q) + half * 8) = w;
                if (i < j)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        *reinterpret_cast<unsigned short*>(a_at(j * 32 + 8 * q + 4 * half + e, i * 4 + (lr >> 3)) + (lr & 7) * 2) =
                            (unsigned short)((e & 2 ? w.y : w.x) >> (16 * (e & 1)));
            }
        }
        __syncthreads();
        u32x2 b[4];
        if (i < nb && j < nb) {
            v16f acc;
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[e] = 0.0f;
#pragma unroll 2
            for (int s = 0; s < 2 * nb; ++s)
                acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const v8h*>(a_at(j * 32 + lr, 2 * s + half)),
                                                             *reinterpret_cast<const v8h*>(a_at(i * 32 + lr, 2 * s + half)), acc, 0, 0, 0);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const u32x2 w = *reinterpret_cast<const u32x2*>(a_at(i * 32 + lr, j * 4 + q) + half * 8);
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[e] = d.b * (float)__builtin_bit_cast(_Float16, (unsigned short)((e & 2 ? w.y : w.x) >> (16 * (e & 1)))) + d.c * acc[4 * q + e];
                b[q] = u32x2{half_pair(v[0], v[1]), half_pair(v[2], v[3])};
            }
        }
        __syncthreads();
        if (i < nb && j < nb)
#pragma unroll
            for (int q = 0; q < 4; ++q) *reinterpret_cast<u32x2*>(a_at(i * 32 + lr, j * 4 + q) + half * 8) = b[q];
        __syncthreads();
        if (wave < cb) {
#pragma unroll
            for (int ib = 0; ib < 4; ++ib)
#pragma unroll
                for (int r = 0; r < 16; ++r) x[ib][r] *= d.a;
            for (int s = 0; s < 2 * nb; ++s) {
                const int row = s * 16 + half * 8 + ((lane >> 2) & 3), col = wave * 32 + ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
                struct {
                    v4s lo, hi;
                } v;
                v.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((turned_t)(x_at(row, col >> 3) + (col & 7) * 2));
                v.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((turned_t)(x_at(row + 4, col >> 3) + (col & 7) * 2));
                const v8h xt = __builtin_bit_cast(v8h, v);
#pragma unroll
                for (int ib = 0; ib < 4; ++ib)
                    if (ib < nb) x[ib] = __builtin_amdgcn_mfma_f32_32x32x16_f16(xt, *reinterpret_cast<const v8h*>(a_at(ib * 32 + lr, 2 * s + half)), x[ib], 0, 0, 0);
            }
        }
        if (step + 1 == d.steps) break;
        __syncthreads();
        put();
        __syncthreads();
    }
    if (tall) {
        int lane_row = lr, lane_col = col0;
        asm("" : "+v"(lane_row), "+v"(lane_col));  // (or the places of all values are held from where G was read)
#pragma unroll
        for (int ib = 0; ib < 4; ++ib)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int row = ib * 32 + lane_row, col = lane_col + (r >> 2) * 8 + (r & 3);
                if (row < few && col < many) out[col * d.x_row + row] = (__bf16)(x[ib][r] * (1.0f / HELD));
            }
        return;
    }
    __syncthreads();
    if (wave < cb)
#pragma unroll
        for (int ib = 0; ib < 4; ++ib)
            if (ib < nb)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *reinterpret_cast<u32x2*>(x_at(ib * 32 + lr, wave * 4 + q) + half * 8) =
                        u32x2{bf16_pair(x[ib][4 * q] * (1.0f / HELD), x[ib][4 * q + 1] * (1.0f / HELD)),
                              bf16_pair(x[ib][4 * q + 2] * (1.0f / HELD), x[ib][4 * q + 3] * (1.0f / HELD))};
    __syncthreads();
    for (int at = tid; at < few * (SMALL_MANY / 8); at += 1024) {
        const int row = at / (SMALL_MANY / 8), chunk = at % (SMALL_MANY / 8), col = chunk * 8;
        if (col >= many) continue;
        const u32x4 w = *reinterpret_cast<const u32x4*>(x_at(row, chunk));
        __bf16* to = out + row * d.x_row + col;
        if (col + 8 <= many) {
            reinterpret_cast<Loose*>(to)->v = w;
        } else {
#pragma unroll
            for (int e = 0; e < 7; ++e)
                if (col + e < many) to[e] = __builtin_bit_cast(__bf16, (unsigned short)(w[e >> 1] >> (16 * (e & 1))));
        }
    }
}
bool in_one(const rrm_orth_desc& d) {
    const int few = d.rows < d.cols ? d.rows : d.cols, many = d.rows < d.cols ? d.cols : d.rows;
    return few <= SMALL_FEW && many <= SMALL_MANY;
}

struct Planes {
    int64_t p, q, out, with;  // from a matrix to the next one's
    int64_t part;             // where sums are split
};
template <bool PT, bool QT, int MT, int NT, int WM, int WN, int STAGES>
__global__ __launch_bounds__(WM* WN * 64, 2) void blend_kernel(Product a, Blend b, Planes planes) {
    __shared__ __attribute__((aligned(1024))) unsigned char lds[TILE_LDS<MT, NT, WM, WN, STAGES>];
    const int64_t z = blockIdx.z;
    a.p[0].p += z * planes.p;
    a.q[0].p += z * planes.q;
    a.out += z * planes.out;
    b.with += z * planes.with;
    if (b.with_rest) b.with_rest += z * planes.with;
    if (b.out_rest) b.out_rest += z * planes.out;
    // split sums: [split][matrix][rows][..]: a split's are as far apart as gridDim.z matrices
    if (a.splits > 1) a.part += z * planes.part + (int64_t)blockIdx.y * ((int64_t)gridDim.z - 1) * planes.part;
    tile_product<BLEND, RRM_ACT_NONE, PT, QT, MT, NT, WM, WN, STAGES>(a, lds, (int)blockIdx.x, (int)blockIdx.y, b);
}
template <bool PT, bool QT, int MT, int NT, int WM, int WN, int STAGES>
void launch_blend(Product a, const Blend& b, const Planes& planes, int n, hipStream_t s) {
    a.tiles_m = tiles(a.rows, MT * 32 * WM);
    a.tiles_n = tiles(a.cols, NT * 32 * WN);
    hipLaunchKernelGGL((blend_kernel<PT, QT, MT, NT, WM, WN, STAGES>), dim3((unsigned)(a.tiles_m * a.tiles_n), (unsigned)a.splits, (unsigned)n), dim3(WM * WN * 64), 0, s, a, b,
                       planes);
}
// The shape with the least of the estimate that SHAPES explains
int shape_of(const Product& a, int n) {
    int best = SMALL;
    float least = 1e30f;
    for (int w = BIG; w <= SMALL; ++w) {
        const Shape& h = SHAPES[w];
        const int64_t groups = (int64_t)tiles(a.rows, h.bm) * tiles(a.cols, h.bn) * n;
        const float us = tiles(a.len, STEP) * (h.first * ((groups + h.at_once - 1) / h.at_once) + h.second * groups / OP_CUS);
        if (us < least) least = us, best = w;
    }
    return best;
}
template <bool PT, bool QT>
hipError_t blend(const Product& a, const Blend& b, const Planes& planes, int n, int shape, hipStream_t s) {
    switch (shape) {
        case BIG: launch_blend<PT, QT, 4, 2, 2, 4, 2>(a, b, planes, n, s); break;
        case WIDE: launch_blend<PT, QT, 2, 2, 2, 2, 4>(a, b, planes, n, s); break;
        case WIDE_PAIR: launch_blend<PT, QT, 2, 2, 2, 2, 2>(a, b, planes, n, s); break;
        default: launch_blend<PT, QT, 1, 2, 2, 2, 3>(a, b, planes, n, s);
    }
    return hipGetLastError();
}

// A's sums are over the longer side, and its tiles few: cut into parts as the estimate says (64 x 4096: 16 parts of four steps, 30 us a step less than whole).
// Up to 128 rows such sums are joined where b A + c A^2 is made.
Plan gram_plan(const rrm_orth_desc& d, int few) {
    const int many = d.rows < d.cols ? d.cols : d.rows;
    return plan_products({few, few, tiles(many, STEP), d.n}, {0, 0, 0, 0}, 2.0f * d.n * (float)few * many);
}

struct Places {
    size_t x[2], rest[2], a, b, part, sums, all;
    int few, pitch, few_pitch;
};
Places places_of(const rrm_orth_desc& d) {
    Places p{};
    p.few = d.rows < d.cols ? d.rows : d.cols;
    p.pitch = round8(d.cols), p.few_pitch = round8(p.few);
    auto take = [&](size_t bytes) {
        const size_t at = p.all;
        p.all += round256(bytes);
        return at;
    };
    p.part = take((size_t)d.n * SUM_PARTS * 8);
    for (size_t& x : p.x) x = take((size_t)d.n * d.rows * p.pitch * 2);
    for (size_t& x : p.rest) x = take((size_t)d.n * d.rows * p.pitch * 2);
    p.a = take((size_t)d.n * p.few * p.few_pitch * 2);
    p.b = take((size_t)d.n * p.few * p.few_pitch * 2);
    const Plan gram = gram_plan(d, p.few);
    p.sums = take(gram.splits > 1 ? (size_t)gram.splits * d.n * p.few * (tiles(p.few, 4) * 4) * 4 : 0);
    return p;
}

template <typename T>
void begin(const rrm_orth_desc& d, const void* g, double* part, _Float16* x, _Float16* rest, _Float16* next, int pitch, hipStream_t s) {
    hipLaunchKernelGGL((squares_kernel<T>), dim3(SUM_PARTS, (unsigned)d.n), dim3(256), 0, s, d, (const T*)g, part);
    const int64_t groups = ((int64_t)d.rows * (pitch / 8) + 255) / 256;
    hipLaunchKernelGGL((scaled_kernel<T>), dim3((unsigned)(groups < 2048 ? groups : 2048), (unsigned)d.n), dim3(256), 0, s, d, (const T*)g, part, x, rest, next, pitch,
                       (int64_t)d.rows * pitch);
}

}  // namespace

size_t orth_scratch(const rrm_orth_desc& d) { return in_one(d) ? 0 : places_of(d).all; }

hipError_t launch_orthogonalize(const rrm_orth_desc& d, const void* g, void* out, void* ws, hipStream_t s) {
    if (in_one(d)) {
        if (d.elem == RRM_F32) hipLaunchKernelGGL((small_kernel<float>), dim3((unsigned)d.n), dim3(1024), 0, s, d, (const float*)g, (__bf16*)out);
        else hipLaunchKernelGGL((small_kernel<__bf16>), dim3((unsigned)d.n), dim3(1024), 0, s, d, (const __bf16*)g, (__bf16*)out);
        return hipGetLastError();
    }
    const Places at = places_of(d);
    unsigned char* base = (unsigned char*)ws;
    _Float16* x[2] = {(_Float16*)(base + at.x[0]), (_Float16*)(base + at.x[1])};
    _Float16* rest[2] = {(_Float16*)(base + at.rest[0]), (_Float16*)(base + at.rest[1])};
    _Float16 *a = (_Float16*)(base + at.a), *b = (_Float16*)(base + at.b);
    double* part = (double*)(base + at.part);
    float* sums = (float*)(base + at.sums);
    const Plan gram = gram_plan(d, at.few);
    const bool joined = at.few <= POLY && gram.splits > 1;
    const int sum_pitch = tiles(at.few, 4) * 4;
    const int64_t sum_plane = (int64_t)at.few * sum_pitch;
    const bool tall = d.rows > d.cols;
    const int64_t x_plane = (int64_t)d.rows * at.pitch, a_plane = (int64_t)at.few * at.few_pitch;
    if (d.elem == RRM_F32) begin<float>(d, g, part, x[0], rest[0], x[1], at.pitch, s);
    else begin<__bf16>(d, g, part, x[0], rest[0], x[1], at.pitch, s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    auto edge = [&](_Float16* p, int64_t rows, int cols, int pitch) {
        if (cols == pitch || e != hipSuccess) return;
        const int64_t groups = (rows + 255) / 256;
        hipLaunchKernelGGL(edge_kernel, dim3((unsigned)(groups < 2048 ? groups : 2048)), dim3(256), 0, s, p, rows, cols, pitch);
        e = hipGetLastError();
    };
    if (!joined) edge(a, (int64_t)d.n * at.few, at.few, at.few_pitch);
    if (!joined) edge(b, (int64_t)d.n * at.few, at.few, at.few_pitch);
    for (int i = 0; i < d.steps && e == hipSuccess; ++i) {
        const Source sx{(src_t)x[i & 1], at.pitch}, sa{(src_t)a, at.few_pitch}, sb{(src_t)b, at.few_pitch};
        const bool last = i + 1 == d.steps;
        Product p{};
        p.pairs = p.splits = 1;
        // A = X X^T
        p.rows = p.cols = at.few, p.len = tall ? d.rows : d.cols;
        p.p[0] = p.q[0] = sx;
        p.out = (__bf16*)a, p.out_row = at.few_pitch;
        p.splits = gram.splits;
        p.part = sums;
        Blend bl{nullptr, nullptr, 0, 1.0f / (HELD * HELD), 0.0f, false, nullptr};
        const Planes gp{x_plane, x_plane, a_plane, 0, sum_plane};
        e = tall ? blend<true, true>(p, bl, gp, d.n, gram.shape, s) : blend<false, false>(p, bl, gp, d.n, gram.shape, s);
        if (e != hipSuccess) break;
        // b A + c A^2
        const int64_t all = d.n * sum_plane;
        if (joined) {
            hipLaunchKernelGGL(poly_kernel, dim3((unsigned)d.n), dim3(1024), 0, s, sums, p.splits, all, at.few, sum_pitch, at.few_pitch, bl.alpha, d.b, d.c, b);
            e = hipGetLastError();
        } else {
            if (p.splits > 1) {
                const int64_t groups = (all / 4 + 255) / 256;
                hipLaunchKernelGGL(gram_kernel, dim3((unsigned)(groups < 4096 ? groups : 4096)), dim3(256), 0, s, sums, p.splits, all, at.few, sum_pitch,
                                   at.few_pitch, bl.alpha, a);
                if ((e = hipGetLastError()) != hipSuccess) break;
            }
            p.splits = 1, p.len = at.few, p.p[0] = p.q[0] = sa;
            p.out = (__bf16*)b;
            bl = Blend{a, nullptr, at.few_pitch, d.c, d.b, false, nullptr};
            e = blend<false, false>(p, bl, {a_plane, a_plane, a_plane, a_plane, 0}, d.n, shape_of(p, d.n), s);
        }
        if (e != hipSuccess) break;
        p.splits = 1, p.len = at.few;
        // a X + (b A + c A^2) X
        p.rows = d.rows, p.cols = d.cols;
        p.out = last ? (__bf16*)out : (__bf16*)x[(i + 1) & 1], p.out_row = last ? d.x_row : at.pitch;
        const float size = last ? 1.0f / HELD : 1.0f;
        bl = Blend{x[i & 1], rest[i & 1], at.pitch, size, size * d.a, last, last ? nullptr : rest[(i + 1) & 1]};
        const int64_t out_plane = last ? d.x_matrix : x_plane;
        if (tall) {
            p.p[0] = sx, p.q[0] = sb;
            e = blend<false, false>(p, bl, {x_plane, a_plane, out_plane, x_plane, 0}, d.n, shape_of(p, d.n), s);
        } else {
            p.p[0] = sb, p.q[0] = sx;
            e = blend<false, true>(p, bl, {a_plane, x_plane, out_plane, x_plane, 0}, d.n, shape_of(p, d.n), s);
        }
    }
    return e;
}

}  // namespace rrm
