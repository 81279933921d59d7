// A weight's update made orthogonal by Newton-Schulz products:
//
//      X = G / (|G| + eps);        `steps` times:  A = X X^T        X <- a X + (b A + c A^2) X
//
// (rows > cols: A = X^T X, X <- a X + X (b A + c A^2)).  Singular value by singular value this is s <- a s + b s^3 + c s^5, and singular vectors stay.
// Three products a step on the matrix cores.  X, A and b A + c A^2 meet memory in half precision, whose eleven bits are eight times as fine as
// bfloat16's at the same rate: a product's rounding errors are taken up by the ones behind it, and with bfloat16 the result would be off by some 1.5%.
// a X, which carries a step's X into the next, is made of X in two parts, the second what the first's rounding left off: the errors of X do not stay (relative error
// of the result beside its own rounding, 256 x 256 and 128 x 512: 0.0010 and 0.0013, with the first part alone 0.0027 and 0.0020).
// Half precision ends at 6e-8: X is held at 256 times its size, so that singular values that a few steps still raise to 1 are above its rounding
// (those of A do not need it: what it lacks is small against a).
#include "tile_product.h"

namespace rrm {

namespace {

constexpr float HELD = 256.0f;
constexpr int SUM_PARTS = 64;  // workgroups that sum a matrix's squares

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
__global__ __launch_bounds__(256) void scaled_kernel(rrm_orth_desc d, const T* g, const double* part, _Float16* x, _Float16* rest, int pitch, int64_t plane) {
    __shared__ double place[4];
    double sum = threadIdx.x < SUM_PARTS ? part[blockIdx.y * SUM_PARTS + threadIdx.x] : 0.0;
    sum = block_sum(sum, place);
    const double factor = HELD / (sqrt(sum) + d.eps);
    g += blockIdx.y * d.g_matrix;
    x += blockIdx.y * plane;
    rest += blockIdx.y * plane;
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
    }
}

// Zeros behind the last column of rows of `pitch`, which products sum over
__global__ __launch_bounds__(256) void edge_kernel(_Float16* p, int64_t rows, int cols, int pitch) {
    for (int64_t r = (int64_t)blockIdx.x * 256 + threadIdx.x; r < rows; r += (int64_t)gridDim.x * 256)
        for (int c = cols; c < pitch; ++c) p[r * pitch + c] = (_Float16)0.0f;
}

struct Planes {
    int64_t p, q, out, with;  // from a matrix to the next one's
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
    tile_product<BLEND, RRM_ACT_NONE, PT, QT, MT, NT, WM, WN, STAGES>(a, lds, (int)blockIdx.x, 0, b);
}
template <bool PT, bool QT, int MT, int NT, int WM, int WN, int STAGES>
void launch_blend(Product a, const Blend& b, const Planes& planes, int n, hipStream_t s) {
    a.tiles_m = tiles(a.rows, MT * 32 * WM);
    a.tiles_n = tiles(a.cols, NT * 32 * WN);
    hipLaunchKernelGGL((blend_kernel<PT, QT, MT, NT, WM, WN, STAGES>), dim3((unsigned)(a.tiles_m * a.tiles_n), 1, (unsigned)n), dim3(WM * WN * 64), 0, s, a, b,
                       planes);
}
template <bool PT, bool QT>
hipError_t blend(const Product& a, const Blend& b, const Planes& planes, int n, hipStream_t s) {
    // the shape with the least of the estimate that SHAPES explains
    int best = SMALL;
    float least = 1e30f;
    for (int w = BIG; w <= SMALL; ++w) {
        const Shape& h = SHAPES[w];
        const int64_t groups = (int64_t)tiles(a.rows, h.bm) * tiles(a.cols, h.bn) * n;
        const float us = tiles(a.len, STEP) * (h.first * ((groups + h.at_once - 1) / h.at_once) + h.second * groups / OP_CUS);
        if (us < least) least = us, best = w;
    }
    switch (best) {
        case BIG: launch_blend<PT, QT, 4, 2, 2, 4, 2>(a, b, planes, n, s); break;
        case WIDE: launch_blend<PT, QT, 2, 2, 2, 2, 4>(a, b, planes, n, s); break;
        case WIDE_PAIR: launch_blend<PT, QT, 2, 2, 2, 2, 2>(a, b, planes, n, s); break;
        default: launch_blend<PT, QT, 1, 2, 2, 2, 3>(a, b, planes, n, s);
    }
    return hipGetLastError();
}

struct Places {
    size_t x[2], rest[2], a, b, part, all;
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
    return p;
}

template <typename T>
void begin(const rrm_orth_desc& d, const void* g, double* part, _Float16* x, _Float16* rest, int pitch, hipStream_t s) {
    hipLaunchKernelGGL((squares_kernel<T>), dim3(SUM_PARTS, (unsigned)d.n), dim3(256), 0, s, d, (const T*)g, part);
    const int64_t groups = ((int64_t)d.rows * (pitch / 8) + 255) / 256;
    hipLaunchKernelGGL((scaled_kernel<T>), dim3((unsigned)(groups < 2048 ? groups : 2048), (unsigned)d.n), dim3(256), 0, s, d, (const T*)g, part, x, rest, pitch,
                       (int64_t)d.rows * pitch);
}

}  // namespace

size_t orth_scratch(const rrm_orth_desc& d) { return places_of(d).all; }

hipError_t launch_orthogonalize(const rrm_orth_desc& d, const void* g, void* out, void* ws, hipStream_t s) {
    const Places at = places_of(d);
    unsigned char* base = (unsigned char*)ws;
    _Float16* x[2] = {(_Float16*)(base + at.x[0]), (_Float16*)(base + at.x[1])};
    _Float16* rest[2] = {(_Float16*)(base + at.rest[0]), (_Float16*)(base + at.rest[1])};
    _Float16 *a = (_Float16*)(base + at.a), *b = (_Float16*)(base + at.b);
    double* part = (double*)(base + at.part);
    const bool tall = d.rows > d.cols;
    const int64_t x_plane = (int64_t)d.rows * at.pitch, a_plane = (int64_t)at.few * at.few_pitch;
    if (d.elem == RRM_F32) begin<float>(d, g, part, x[0], rest[0], at.pitch, s);
    else begin<__bf16>(d, g, part, x[0], rest[0], at.pitch, s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    auto edge = [&](_Float16* p, int64_t rows, int cols, int pitch) {
        if (cols == pitch || e != hipSuccess) return;
        const int64_t groups = (rows + 255) / 256;
        hipLaunchKernelGGL(edge_kernel, dim3((unsigned)(groups < 2048 ? groups : 2048)), dim3(256), 0, s, p, rows, cols, pitch);
        e = hipGetLastError();
    };
    if (d.steps > 1) edge(x[1], (int64_t)d.n * d.rows, d.cols, at.pitch);
    edge(a, (int64_t)d.n * at.few, at.few, at.few_pitch);
    edge(b, (int64_t)d.n * at.few, at.few, at.few_pitch);
    for (int i = 0; i < d.steps && e == hipSuccess; ++i) {
        const Source sx{(src_t)x[i & 1], at.pitch}, sa{(src_t)a, at.few_pitch}, sb{(src_t)b, at.few_pitch};
        const bool last = i + 1 == d.steps;
        Product p{};
        p.pairs = p.splits = 1;
        // A = X X^T
        p.rows = p.cols = at.few, p.len = tall ? d.rows : d.cols;
        p.p[0] = p.q[0] = sx;
        p.out = (__bf16*)a, p.out_row = at.few_pitch;
        Blend bl{nullptr, nullptr, 0, 1.0f / (HELD * HELD), 0.0f, false, nullptr};
        e = tall ? blend<true, true>(p, bl, {x_plane, x_plane, a_plane, 0}, d.n, s) : blend<false, false>(p, bl, {x_plane, x_plane, a_plane, 0}, d.n, s);
        if (e != hipSuccess) break;
        // b A + c A^2
        p.len = at.few, p.p[0] = p.q[0] = sa;
        p.out = (__bf16*)b;
        bl = Blend{a, nullptr, at.few_pitch, d.c, d.b, false, nullptr};
        e = blend<false, false>(p, bl, {a_plane, a_plane, a_plane, a_plane}, d.n, s);
        if (e != hipSuccess) break;
        // a X + (b A + c A^2) X
        p.rows = d.rows, p.cols = d.cols;
        p.out = last ? (__bf16*)out : (__bf16*)x[(i + 1) & 1], p.out_row = last ? d.x_row : at.pitch;
        const float size = last ? 1.0f / HELD : 1.0f;
        bl = Blend{x[i & 1], rest[i & 1], at.pitch, size, size * d.a, last, last ? nullptr : rest[(i + 1) & 1]};
        const int64_t out_plane = last ? d.x_matrix : x_plane;
        if (tall) {
            p.p[0] = sx, p.q[0] = sb;
            e = blend<false, false>(p, bl, {x_plane, a_plane, out_plane, x_plane}, d.n, s);
        } else {
            p.p[0] = sb, p.q[0] = sx;
            e = blend<false, true>(p, bl, {a_plane, x_plane, out_plane, x_plane}, d.n, s);
        }
    }
    return e;
}

}  // namespace rrm
