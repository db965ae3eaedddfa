// Newton-Schulz steps: X <- a X + b A X + c A^2 X with A = X X^T, from X / (|X|_F + eps) on; odd polynomials of X, which leave its singular
// vectors as they are and move its singular values.  A is taken on the shorter side: Y is X, or X^T where X has more rows than columns.
//
// Terms.  Every matrix is kept as two fp16 terms, hi = fp16(x s) and lo = fp16(x s - hi), 22 significant bits, and products are formed as
// lo hi + hi lo + hi hi in fp32: half the work of three bfloat16 terms.  That needs scales s that keep fp16's range, known before a matrix is written.  With S a bound of Y's
// singular values A is at most S^2, the factor a I + b A + c A^2 the largest |a + b t + c t^2| on [0, S^2], and the next Y the largest |a v + b v^3 + c v^5| on [0, S]; no
// element is larger than its matrix's norm.  S is the smaller of two: what the coefficients make of 1 from step to step, and ||Y||_F, which is summed while Y is written (||X||_F to
// begin with).  Two terms hold 22 bits of what is within 2^18 of the scale, and the first alone would drift away from matrices that shrink.  Scales are powers of two.
// Where a step's bounds say little (one that may take singular values past 16, or small
// ones down faster than by half: ortho_bounded) matrices stay in fp32 and are multiplied as three bfloat16 terms.  One term would leave 2^-12, and after the growth of small singular values up to
// 2.4e-3 of the result, more than a result in bfloat16 is rounded by; two leave 2e-6 (2048 x 1024 of noise, five steps; the same in fp32 3.3e-6).
#pragma once
#include "direct.hpp"

namespace ivf {

typedef _Float16 halfx2 __attribute__((ext_vector_type(2)));
typedef _Float16 halfx4 __attribute__((ext_vector_type(4)));

constexpr int ORTHO_TERMS = 2;

// Multipliers of a step, the scales included (sy: of Y, sa: of A, sf: of the factor F, sn: of the next Y)
struct OrthoScales {
    float gram;                // Y Y^T -> A sa
    float square, linear, unit;         // the product of A sa by itself, A sa, the diagonal -> F sf
    float direct_linear, direct_unit;   // Y Y^T, the diagonal -> F sf: where c is 0
    float apply, last;         // F Y -> the next Y, scaled, or its value
    double next;               // sn
};

// The power of two that takes values of up to `bound` to 2^15 at most.
__host__ __device__ __forceinline__ double ortho_scale(double bound)
{
    if (!(bound > 0.0)) return 1.0;
    const int e = bound < HUGE_VAL ? 14 - ilogb(bound) : 0;
    return ldexp(1.0, e < -400 ? -400 : e > 400 ? 400 : e);
}

// The bounds of a step from S, that of the singular values before it: of the factor, and of the values after it.
struct OrthoBounds {
    double factor, next;
};

__host__ __device__ inline OrthoBounds ortho_bounds(double a, double b, double c, double S)
{
    const double T = S * S;
    auto odd = [&](double t) { return fabs(sqrt(t) * (a + b * t + c * t * t)); };               // of a singular value whose square is t
    auto even = [&](double t) { return fabs(a + b * t + c * t * t); };
    OrthoBounds r{fmax(fabs(a), even(T)), odd(T)};
    auto look = [&](double t) { if (t > 0.0 && t < T) r.next = fmax(r.next, odd(t)); };
    if (c != 0.0) {
        const double d = 9.0 * b * b - 20.0 * a * c;           // a + 3 b t + 5 c t^2 = 0
        if (d >= 0.0) look((-3.0 * b + sqrt(d)) / (10.0 * c)), look((-3.0 * b - sqrt(d)) / (10.0 * c));
        const double t = -b / (2.0 * c);
        if (t > 0.0 && t < T) r.factor = fmax(r.factor, even(t));
    } else if (b != 0.0) {
        look(-a / (3.0 * b));
    }
    return r;
}

// Y is kept in both orientations because the products sum along rows of either.
struct OrthoMatrix {
    uint16_t *p;               // [batch][rows][ld / 32][ORTHO_TERMS][32]
    int rows, cols, ld;        // ld: cols rounded up to 32, zeros there
    // the first term of an element; the next is 32 further
    __device__ __forceinline__ uint16_t *at(int64_t matrix, int row, int col) const
    {
        return p + (matrix * rows + row) * (ORTHO_TERMS * (int64_t)ld) + col / 32 * (32 * ORTHO_TERMS) + col % 32;
    }
};

// Sums of squares in 64 bits, NORM_CHUNK elements of a matrix each workgroup (a matrix has its own sums[matrix * parts ..]); 32 bytes a lane and
// step keep enough of memory on its way: 16.8 MB of bfloat16 in 6 us.
constexpr int NORM_CHUNK = 16384;
template <Type T>
__global__ __launch_bounds__(256) void ortho_norm_kernel(uint32_t first, const void *__restrict__ x, int64_t size, int parts, double *__restrict__ sums)
{
    __shared__ double wave_sums[4];
    const uint32_t place = first + blockIdx.x;
    const int64_t matrix = place / parts, a = (int64_t)(place % parts) * NORM_CHUNK, b = a + NORM_CHUNK < size ? a + NORM_CHUNK : size;
    double s = 0.0;
#pragma unroll 4
    for (int64_t i = a + 8 * (int)threadIdx.x; i < b; i += 8 * 256) {
        float v[8];
        if (i + 8 <= b) {
            eight<T>(x, matrix * size + i, v);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = i + j < b ? element<T>(x, matrix * size + i + j) : 0.f;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) s += (double)v[j] * v[j];
    }
#pragma unroll
    for (int o = WAVE / 2; o > 0; o >>= 1) s += __shfl_xor(s, o, WAVE);
    if ((threadIdx.x & 63) == 0) wave_sums[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) sums[place] = wave_sums[0] + wave_sums[1] + wave_sums[2] + wave_sums[3];
}

// 1 / (norm + eps); 0 for a matrix of zeros, which stays one whatever eps is; NaN for one with an infinity or a NaN
__device__ __forceinline__ double ortho_inverse(double squares, double eps)
{
    return squares == 0.0 ? 0.0 : squares < HUGE_VAL ? 1.0 / (sqrt(squares) + eps) : __builtin_nan("");
}

// The sum of `parts` numbers, for every lane of a wavefront.
__device__ __forceinline__ double ortho_sum(const double *sums, int parts)
{
    double s = 0.0;
    for (int i = threadIdx.x; i < parts; i += 64) s += sums[i];
#pragma unroll
    for (int o = WAVE / 2; o > 0; o >>= 1) s += __shfl_xor(s, o, WAVE);
    return s;
}

// 1 / (norm + eps) of every matrix and its norm after that, a wavefront each.
__global__ __launch_bounds__(64) void ortho_inverse_kernel(uint32_t first, const double *__restrict__ sums, int parts, double eps, double *__restrict__ inverse, double *__restrict__ norms)
{
    const int64_t matrix = first + blockIdx.x;
    const double s = ortho_sum(sums + matrix * parts, parts), by = ortho_inverse(s, eps);
    if (threadIdx.x == 0) {
        inverse[matrix] = by;
        norms[matrix] = sqrt(s) * by;
    }
}

// The multipliers of every matrix's next step, a wavefront each: of the first one (sums NULL) from norms, of others from the squares of the scaled Y that the last
// step's workgroups have summed.  most: a bound of its singular values that follows from the coefficients.
__global__ __launch_bounds__(64) void ortho_scales_kernel(uint32_t first, const double *__restrict__ sums, int parts, const double *__restrict__ norms, double a, double b, double c,
                                                          double most, OrthoScales *__restrict__ scales)
{
    const int64_t matrix = first + blockIdx.x;
    OrthoScales &s = scales[matrix];
    const double sy = sums ? s.next : ortho_scale(norms[matrix]);
    const double S = fmin(most, sums ? sqrt(ortho_sum(sums + matrix * parts, parts)) / sy : norms[matrix]);
    if (threadIdx.x != 0) return;
    const OrthoBounds bound = ortho_bounds(a, b, c, S);
    const double sa = ortho_scale(S * S), sf = ortho_scale(bound.factor), sn = ortho_scale(bound.next);
    s.gram = (float)(sa / sy / sy);
    s.square = (float)(c * sf / sa / sa);
    s.linear = (float)(b * sf / sa);
    s.unit = (float)(a * sf);
    s.direct_linear = (float)(b * sf / sy / sy);
    s.direct_unit = (float)(a * sf);
    s.apply = (float)(sn / sf / sy);
    s.last = (float)(1.0 / sf / sy);
    s.next = sn;
}

// Terms of N values (N even), two a word.
template <int N>
__device__ __forceinline__ void ortho_cut(const float (&v)[N], uint32_t (&out)[ORTHO_TERMS][N / 2])
{
#pragma unroll
    for (int j = 0; j < N / 2; ++j) {
        // (the value itself, rounded to 32 bits: were the product it comes from fused with one of its two uses and not with the other, the terms
        // would not belong together)
        float x = v[2 * j], y = v[2 * j + 1];
        asm("" : "+v"(x), "+v"(y));
        const _Float16 a = (_Float16)x, b = (_Float16)y;
        out[0][j] = __builtin_bit_cast(uint32_t, halfx2{a, b});
        out[1][j] = __builtin_bit_cast(uint32_t, halfx2{(_Float16)(x - (float)a), (_Float16)(y - (float)b)});
    }
}

// x over its norm, scaled, as terms, in x's orientation (same) and transposed: 32 x 32 elements a workgroup.
template <Type T>
__global__ __launch_bounds__(256) void ortho_first_kernel(uint32_t first, const void *__restrict__ x, int rows, int cols, const double *__restrict__ inverse,
                                                          const double *__restrict__ norms, OrthoMatrix same, OrthoMatrix turned)
{
    __shared__ float tile[32][33];
    const int across = (cols + 31) / 32, down = (rows + 31) / 32;
    const uint32_t place = first + blockIdx.x;
    const int64_t matrix = place / (across * down);
    const int c0 = (int)(place % across) * 32, r0 = (int)(place / across % down) * 32;
    const double by = ortho_scale(norms[matrix]) * inverse[matrix];
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
#pragma unroll
    for (int i = 0; i < 32; i += 8) {
        const int r = r0 + ty + i, c = c0 + tx;
        tile[ty + i][tx] = r < rows && c < cols ? (float)(element<T>(x, (matrix * rows + r) * cols + c) * by) : 0.f;
    }
    __syncthreads();
    const int r = threadIdx.x >> 3, c = 4 * (threadIdx.x & 7);
    auto write = [&](const OrthoMatrix &m, int row, int col, const float (&v)[4]) {
        if (row >= m.rows) return;                             // (columns up to ld are written)
        uint32_t t[ORTHO_TERMS][2];
        ortho_cut<4>(v, t);
#pragma unroll
        for (int q = 0; q < ORTHO_TERMS; ++q)
            *reinterpret_cast<wordx2 *>(m.at(matrix, row, col) + 32 * q) = wordx2{t[q][0], t[q][1]};
    };
    const float v[4] = {tile[r][c], tile[r][c + 1], tile[r][c + 2], tile[r][c + 3]};
    const float u[4] = {tile[c][r], tile[c + 1][r], tile[c + 2][r], tile[c + 3][r]};
    write(same, r0 + r, c0 + c, v);
    write(turned, c0 + r, r0 + c, u);
}

// Four scaled values in a run of a row, in both orientations where those are asked for (p not NULL).  Past the matrix's rows and columns the
// tile holds products of others: zeros are written there, up to ld.
__device__ __forceinline__ void put_terms(const OrthoMatrix &same, const OrthoMatrix &turned, int64_t matrix, int row, int col, floatx4 v)
{
    const int rows = same.p ? same.rows : turned.cols, cols = same.p ? same.cols : turned.rows;
    float f[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = row < rows && col + j < cols ? v[j] : 0.f;
    uint32_t t[ORTHO_TERMS][2];
    ortho_cut<4>(f, t);
    if (same.p && row < same.rows && col < same.ld)
#pragma unroll
        for (int q = 0; q < ORTHO_TERMS; ++q)
            *reinterpret_cast<wordx2 *>(same.at(matrix, row, col) + 32 * q) = wordx2{t[q][0], t[q][1]};
    if (turned.p && row < turned.ld)
#pragma unroll
        for (int q = 0; q < ORTHO_TERMS; ++q)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (col + j < turned.rows)
                    turned.at(matrix, col + j, row)[32 * q] = (uint16_t)(t[q][j / 2] >> (16 * (j & 1)));
}

__device__ __forceinline__ DirectSource ortho_source(const OrthoMatrix &m, int64_t matrix, int row0)
{
    return DirectSource{m.at(matrix, row0, 0), (int64_t)ORTHO_TERMS * m.ld, m.rows - row0};
}

template <int B, int W>
using OrthoTile = DirectTile<false, ORTHO_TERMS, B, W, false, ORTHO_TERMS, B, W, 32, 2, true>;

// 2048 x 4096: A 82 us, A^2 46, the product with Y 102 (630, 560 and 1010 TFLOP/s of terms' products; the matrix units are busy for 36, 31 and 56 % of the units' time).
// Symmetric results, the tiles on and below the diagonal, each written to both sides.
//   GRAM: to = Y Y^T, or a I + b Y Y^T (direct)      else: to = a I + b F + c F F, F symmetric
template <int B, int W, bool GRAM>
__global__ __launch_bounds__(WAVE *W *W) void ortho_symmetric_kernel(uint32_t first, OrthoMatrix from, OrthoMatrix to, const OrthoScales *__restrict__ scales, int direct)
{
    using P = OrthoTile<B, W>;
    __shared__ __attribute__((aligned(16))) uint16_t lds[P::LDS_HALVES];
    const int side = (from.rows + B - 1) / B, count = side * (side + 1) / 2;
    const uint32_t place = first + place_of_block(blockIdx.x, gridDim.x);
    const int64_t matrix = place / count;
    int i, j;
    triangle_of_place((int)(place % count), side, i, j);
    const int i0 = i * B, j0 = j * B;
    P t;
    t.clear();
    t.product(ortho_source(from, matrix, i0), ortho_source(from, matrix, j0), from.ld, lds);
    const OrthoMatrix none{nullptr, 0, 0, 0};
    const OrthoScales s = scales[matrix];
    t.each([&](int ri, int rj, floatx4 v) {
        const int row = j0 + rj, col = i0 + ri;
        if constexpr (GRAM) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                v[q] = direct ? s.direct_linear * v[q] + (row == col + q && row < from.rows ? s.direct_unit : 0.f) : s.gram * v[q];
        } else {
            if (row < from.rows && col < from.ld) {
                const uint16_t *f = from.at(matrix, row, col);
                const halfx4 hi = *reinterpret_cast<const halfx4 *>(f), lo = *reinterpret_cast<const halfx4 *>(f + 32);
#pragma unroll
                for (int q = 0; q < 4; ++q) v[q] = s.square * v[q] + s.linear * ((float)hi[q] + (float)lo[q]) + (row == col + q ? s.unit : 0.f);
            }
        }
        put_terms(to, i0 == j0 ? none : to, matrix, row, col, v);
    });
}

// Y <- F Y from Y transposed: both orientations and the sum of the squares of its scaled elements, or the result itself in x's (last).
template <int B, int W>
__global__ __launch_bounds__(WAVE *W *W) void ortho_apply_kernel(uint32_t first, OrthoMatrix yt, OrthoMatrix f, OrthoMatrix to, OrthoMatrix to_t, const OrthoScales *__restrict__ scales,
                                                                 double *__restrict__ sums, void *out, Type type, int turned)
{
    using P = OrthoTile<B, W>;
    __shared__ __attribute__((aligned(16))) uint16_t lds[P::LDS_HALVES];
    const int across = (yt.rows + B - 1) / B, down = (f.rows + B - 1) / B;
    const uint32_t place = first + place_of_block(blockIdx.x, gridDim.x);
    const int64_t matrix = place / (across * down);
    int i, j;
    tile_of_place(place % (across * down), down, across, i, j);
    const int j0 = j * B, i0 = i * B;
    P t;
    t.clear();
    t.product(ortho_source(yt, matrix, j0), ortho_source(f, matrix, i0), f.ld, lds);
    const int m = f.rows, n = yt.rows;
    const float by = out ? scales[matrix].last : scales[matrix].apply;
    float squares = 0.f;
    t.each([&](int rj, int ri, floatx4 v) {
        const int row = i0 + ri, col = j0 + rj;                // of Y
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            v[q] *= by;
            squares = row < m && col + q < n ? fmaf(v[q], v[q], squares) : squares;
        }
        if (!out) {
            put_terms(to, to_t, matrix, row, col, v);
        } else if (row < m && col < n) {
            if (!turned) put4(out, (matrix * m + row) * n + col, v, n - col, type);
            else
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (col + q < n) put4(out, (matrix * n + col + q) * m + row, floatx4{v[q], 0.f, 0.f, 0.f}, 1, type);
        }
    });
    if (out) return;
    double *wave_sums = reinterpret_cast<double *>(lds);      // (nobody reads it any more)
    const double s = wave_sum((double)squares);
    if (threadIdx.x % WAVE == 0) wave_sums[threadIdx.x / WAVE] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        double all = 0.0;
#pragma unroll
        for (int w = 0; w < W * W; ++w) all += wave_sums[w];
        sums[matrix * (across * down) + i * across + j] = all;
    }
}

// Coefficients without useful bounds: matrices in fp32, without padding.
template <Type T>
__global__ __launch_bounds__(256) void ortho_first_general_kernel(const void *__restrict__ x, int64_t batch, int rows, int cols, const double *__restrict__ inverse,
                                                                  float *__restrict__ same, float *__restrict__ turned)
{
    const int64_t size = (int64_t)rows * cols;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < batch * size; i += (int64_t)gridDim.x * 256) {
        const int64_t matrix = i / size, at = i - matrix * size, r = at / cols, c = at - r * cols;
        const float v = (float)(element<T>(x, i) * inverse[matrix]);
        same[i] = v;
        turned[matrix * size + c * rows + r] = v;
    }
}

// to [rows_q][rows_p] = by p q^T transposed + plus `from` + unit I, for p [rows_p][K] and q [rows_q][K]; also to to_t, or (out) as the result in x's
// shape and type.
struct OrthoGeneral {
    const float *p, *q;
    int rows_p, rows_q, K;
    float by, plus, unit;
    const float *from;
    float *to, *to_t;
    void *out;
    Type type;
    int turned;
};

__global__ __launch_bounds__(256) void ortho_general_kernel(uint32_t first, OrthoGeneral g)
{
    using P = Tile<Form::F_ROWS, 3, 64, 2, Form::F_ROWS, 3, 64, 2, 32, 1, false, true>;
    __shared__ __attribute__((aligned(16))) uint16_t lds[P::LDS_HALVES];
    const int across = (g.rows_p + 63) / 64, down = (g.rows_q + 63) / 64;
    const uint32_t place = first + blockIdx.x;
    const int64_t matrix = place / (across * down), size = (int64_t)g.rows_p * g.rows_q;
    const int i0 = (int)(place % across) * 64, j0 = (int)(place / across % down) * 64;
    auto source = [&](const float *p, int rows, int row) {
        return Source{reinterpret_cast<const uint8_t *>(p + (matrix * rows + row) * g.K), nullptr, g.K, rows - row < 64 ? rows - row : 64};
    };
    P t;
    t.clear();
    t.product(source(g.p, g.rows_p, i0), source(g.q, g.rows_q, j0), 0, g.K, lds);
    t.each([&](int ri, int rj, floatx4 v) {
        const int row = j0 + rj, col = i0 + ri;
        if (row >= g.rows_q) return;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (col + e >= g.rows_p) break;
            const int64_t at = matrix * size + (int64_t)row * g.rows_p + col + e, at_t = matrix * size + (int64_t)(col + e) * g.rows_q + row;
            float w = g.by * v[e];
            if (g.from) w += g.plus * g.from[at];
            if (row == col + e) w += g.unit;
            if (g.out) {
                put4(g.out, g.turned ? at_t : at, floatx4{w, 0.f, 0.f, 0.f}, 1, g.type);
            } else {
                g.to[at] = w;
                if (g.to_t) g.to_t[at_t] = w;
            }
        }
    });
}

}  // namespace ivf
