// Newton-Schulz steps on matrices of up to 128 x 128 (the rotations of regions): all steps in one launch, a workgroup a matrix, nothing but the
// matrix itself read and written.
//
// A wavefront owns 32 rows of Y (MB wavefronts, Y of up to 32 MB x 32 NB).  Every product is formed with the shared operand's rows as the
// first operand, from LDS, and the wavefront's own rows as the second, from registers, so that a lane's accumulators run along its own row:
// exchanged between the halves of the wavefront they are fragments again (own_fragments).  LDS holds one matrix at a time, Y or A as
// terms, which for 96 x 96 is 37 KB.  Y stands in LDS once for both of its uses: along its rows for A = Y Y^T, and by transposing reads for F Y.
//
// Scales are powers of two that bring a matrix's largest element, as it is, to 2^13 .. 2^15: of A the largest on its diagonal, of F that of a wavefront's own
// rows (nobody else has them), of Y that of all of it.  So nothing has to be known of the coefficients: what bounds of the singular values would allow drifts away from what
// they are when a matrix shrinks for many steps, and two fp16 terms hold 22 bits only of what is within 2^18 of their scale.
//
// 4096 x 96 x 96 fp32, ten steps: 805 - 820 us in long runs (900 from cold clocks), the matrix units busy for 37 % of it, LDS for 35; the rest cuts values into terms and waits at
// barriers.  Three wavefronts a SIMD, for which 25 registers are spilled.  1.2e-7 of the result against 64 bits, the same steps in fp32 1.1e-7.
#pragma once
#include "direct.hpp"
#include "ortho.hpp"

namespace ivf {

constexpr int ORTHO_SMALL_SIDE = 128;
constexpr int ORTHO_SMALL_STEPS = 256;                        // whose coefficients are arguments of the launch
constexpr int ORTHO_TOP = 14;                                 // exponent of a scaled matrix's largest element
constexpr int NOTHING = -(1 << 20);                           // in the place of an exponent: all zeros

struct OrthoSmallArgs {
    const void *x;
    void *out;
    int rows, cols, steps, turned;                            // turned: Y is X transposed
    Type type;
    double eps;
    uint32_t first;                                           // matrix that this launch begins with
    const float *more;                                        // more steps: where their coefficients are
    float coefs[3 * ORTHO_SMALL_STEPS];
};

// Coefficients into memory: the arguments of a launch hold no more than these.
struct OrthoCoefs {
    float *to;
    int count;
    float coefs[3 * ORTHO_SMALL_STEPS];
};

__global__ __launch_bounds__(256) void ortho_coefs_kernel(OrthoCoefs c)
{
    for (int i = threadIdx.x; i < c.count; i += 256) c.to[i] = c.coefs[i];
}

// What takes a value of those magnitude bits to 2^ORTHO_TOP: the power of two's exponent.
__device__ __forceinline__ int ortho_shift(uint32_t top)
{
    const int e = ORTHO_TOP + 127 - (int)(top >> 23);
    return top == 0 ? 0 : e > 126 ? 126 : e;
}

__device__ __forceinline__ float ortho_power(int e) { return ldexpf(1.f, e); }
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// A fragment: 16 elements along a row, 8 of them in a lane.
struct Terms {
    wordx4 t[ORTHO_TERMS];
};

// The accumulators, times `by`, of 32 columns (lane: row lane % 32, columns 8 q + 4 (lane / 32) + 0..3) as terms of two fragments of 16 columns.
__device__ __forceinline__ void own_fragments(const floatx16 &v, float by, Terms (&to)[2])
{
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        uint32_t t[2][ORTHO_TERMS][2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const float f[4] = {v[8 * s + 4 * u] * by, v[8 * s + 4 * u + 1] * by, v[8 * s + 4 * u + 2] * by, v[8 * s + 4 * u + 3] * by};
            ortho_cut<4>(f, t[u]);
        }
#pragma unroll
        for (int q = 0; q < ORTHO_TERMS; ++q) {
            const wordx2 x = __builtin_bit_cast(wordx2, __builtin_amdgcn_permlane32_swap(t[0][q][0], t[1][q][0], false, false));
            const wordx2 y = __builtin_bit_cast(wordx2, __builtin_amdgcn_permlane32_swap(t[0][q][1], t[1][q][1], false, false));
            to[s].t[q] = wordx4{x[0], y[0], x[1], y[1]};
        }
    }
}

template <int MB, int NB>
struct OrthoSmall {
    static constexpr int TERMS = ORTHO_TERMS;
    static constexpr int M = 32 * MB, N = 32 * NB, NT = WAVE * MB;
    static constexpr int LDS_HALVES = TERMS * M * N;

    wordx4 y[TERMS][2 * NB];                                  // own rows of Y

    static __device__ __forceinline__ floatx16 zero()
    {
        floatx16 z;
#pragma unroll
        for (int e = 0; e < 16; ++e) z[e] = 0.f;
        return z;
    }

    // acc += a b; the products with a low term, a thousandth of the others, go into a sum of their own, so that acc is rounded once where it would be three times
    static __device__ __forceinline__ void multiply(const Terms &a, const wordx4 (&b)[TERMS], floatx16 &acc, floatx16 &low)
    {
        low = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(halfx8, a.t[0]), __builtin_bit_cast(halfx8, b[1]), low, 0, 0, 0);
        low = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(halfx8, a.t[1]), __builtin_bit_cast(halfx8, b[0]), low, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(halfx8, a.t[0]), __builtin_bit_cast(halfx8, b[0]), acc, 0, 0, 0);
    }

    static __device__ __forceinline__ void add(floatx16 &acc, const floatx16 &low)
    {
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[e] += low[e];
        __builtin_amdgcn_sched_barrier(0);                    // (one block's fragments at a time)
    }

    // own rows into LDS
    template <int W>
    static __device__ __forceinline__ void put(uint16_t *lds, int term, int piece, wordx4 v)
    {
        const int lane = threadIdx.x & 63, row = (int)(threadIdx.x / WAVE) * 32 + (lane & 31);
        *reinterpret_cast<wordx4 *>(lds + term * (M * W) + line_at<W>(row, 2 * piece + lane / 32)) = v;
    }

    // 16 elements of the 32 rows from `row` on
    template <int W>
    static __device__ __forceinline__ Terms row_fragment(const uint16_t *lds, int row, int p)
    {
        const int lane = threadIdx.x & 63;
        Terms v;
#pragma unroll
        for (int t = 0; t < TERMS; ++t) v.t[t] = *reinterpret_cast<const wordx4 *>(lds + t * (M * W) + line_at<W>(row + (lane & 31), 2 * p + lane / 32));
        return v;
    }

    __device__ __forceinline__ void put_y(uint16_t *lds) const
    {
#pragma unroll
        for (int t = 0; t < TERMS; ++t)
#pragma unroll
            for (int p = 0; p < 2 * NB; ++p) put<N>(lds, t, p, y[t][p]);
    }

    template <Type T>
    static __device__ __forceinline__ double squares(const void *x, int64_t at, int size, uint32_t &top)
    {
        double s = 0.0;
        for (int i = threadIdx.x; i < size; i += NT) {
            const float f = element<T>(x, at + i);
            const double v = f;
            s += v * v;
            top = magnitude(f) > top ? magnitude(f) : top;
        }
        return s;
    }

    // Y into LDS by pieces of 8 columns: neighbouring threads along a row of X, so along a column of Y where that is X transposed
    template <Type T>
    static __device__ __forceinline__ void bring(const OrthoSmallArgs &g, int64_t at, int m, int n, double by, uint16_t *lds)
    {
        for (int id = threadIdx.x; id < M * N / 8; id += NT) {
            const int row = g.turned ? id % M : id / (N / 8), piece = g.turned ? id / M : id % (N / 8);
            const int first = g.turned ? 8 * piece * m + row : row * n + 8 * piece, apart = g.turned ? m : 1;
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = row < m && 8 * piece + j < n ? (float)(element<T>(g.x, at + first + j * apart) * by) : 0.f;
            uint32_t t[TERMS][4];
            ortho_cut<8>(v, t);
#pragma unroll
            for (int q = 0; q < TERMS; ++q)
                *reinterpret_cast<wordx4 *>(lds + q * (M * N) + line_at<N>(row, piece)) = wordx4{t[q][0], t[q][1], t[q][2], t[q][3]};
        }
    }

    // Where an element of the result stands in LDS: in 32 bits, which is as much as its two terms, runs of four exchanged by the row's number.
    static __device__ __forceinline__ int place(int row, int col) { return row * N + (((col / 4) ^ (row & 7)) * 4) + col % 4; }

    // the result from LDS to X's shape, in runs of four along X's rows
    static __device__ __forceinline__ void give(const OrthoSmallArgs &g, int64_t at, int m, int n, const float *lds)
    {
        const int rows = g.turned ? n : m, cols = g.turned ? m : n, runs = (cols + 3) / 4;
        for (int id = threadIdx.x; id < rows * runs; id += NT) {
            const int r = id / runs, c = id % runs * 4;
            floatx4 v;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = lds[g.turned ? place(c + j, r) : place(r, c + j)];   // (up to three past the end, inside the padding)
            put4(g.out, at + (int64_t)r * cols + c, v, cols - c, g.type);
        }
    }

    __device__ __forceinline__ void run(const OrthoSmallArgs &g, uint16_t *lds, double *sums, int *tops)
    {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / WAVE));
        const int64_t matrix = g.first + blockIdx.x, size = (int64_t)g.rows * g.cols;
        const int m = g.turned ? g.cols : g.rows, n = g.turned ? g.rows : g.cols;
        // the largest of what the wavefronts have put into tops
        auto largest = [&]() {
            int v = tops[0];
#pragma unroll
            for (int w = 1; w < MB; ++w) v = tops[w] > v ? tops[w] : v;
            return __builtin_amdgcn_readfirstlane(v);
        };
        double s = 0.0;
        uint32_t top = 0;
        if (g.type == Type::F32) s = squares<Type::F32>(g.x, matrix * size, (int)size, top);
        else if (g.type == Type::F16) s = squares<Type::F16>(g.x, matrix * size, (int)size, top);
        else s = squares<Type::BF16>(g.x, matrix * size, (int)size, top);
#pragma unroll
        for (int o = WAVE / 2; o > 0; o >>= 1) s += __shfl_xor(s, o, WAVE);
        top = wave_extreme<true>(top);
        if (lane == 0) sums[wave] = s, tops[wave] = (int)top;
        __syncthreads();
        s = 0.0;
#pragma unroll
        for (int w = 0; w < MB; ++w) s += sums[w];
        const double inverse = ortho_inverse(s, g.eps);
        // Y's elements are y 2^-ey of the scaled ones
        int ey = (int)(ORTHO_TOP + 1023 - (__double_as_longlong((double)__uint_as_float((uint32_t)largest()) * inverse) >> 52 & 2047));
        const double by = ldexp(inverse, ey);
        if (g.type == Type::F32) bring<Type::F32>(g, matrix * size, m, n, by, lds);
        else if (g.type == Type::F16) bring<Type::F16>(g, matrix * size, m, n, by, lds);
        else bring<Type::BF16>(g, matrix * size, m, n, by, lds);
        __syncthreads();
#pragma unroll
        for (int t = 0; t < TERMS; ++t)
#pragma unroll
            for (int p = 0; p < 2 * NB; ++p)
                y[t][p] = *reinterpret_cast<const wordx4 *>(lds + t * (M * N) + line_at<N>(32 * wave + (lane & 31), 2 * p + lane / 32));

        floatx16 next[NB];                                    // the next Y: 2^fe of these
        int fe;
        uint32_t high;
        for (int step = 0;; ++step) {
            const float ca = g.more ? g.more[3 * step] : g.coefs[3 * step], cb = g.more ? g.more[3 * step + 1] : g.coefs[3 * step + 1],
                        cc = g.more ? g.more[3 * step + 2] : g.coefs[3 * step + 2];
            floatx16 a[MB];
            // A = Y Y^T: columns of own rows
#pragma unroll
            for (int i = 0; i < MB; ++i) {
                floatx16 low = zero();
                a[i] = zero();
#pragma unroll
                for (int p = 0; p < 2 * NB; ++p) {
                    wordx4 v[TERMS];
#pragma unroll
                    for (int t = 0; t < TERMS; ++t) v[t] = y[t][p];
                    multiply(row_fragment<N>(lds, 32 * i, p), v, a[i], low);
                }
                add(a[i], low);
            }
            high = 0;
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (i == wave && 8 * (e / 4) + 4 * (lane / 32) + e % 4 == (lane & 31)) high = magnitude(a[i][e]);
            high = wave_extreme<true>(high);
            if (lane == 0) tops[wave] = (int)high;
            __syncthreads();                                  // Y has been read
            high = (uint32_t)largest();
            const int to_a = ortho_shift(high), ea = 2 * ey + to_a;
            // F = factor 2^fe (sums): those start from what is left of b A + a I.  Over c, so that c A A is their products of A's terms, unless it is below
            // what 32 bits keep of the rest (which the sums could not hold over c either).
            const double T = fmin(ldexp((double)__uint_as_float(high), -2 * ey), 1e300), rest = fabs((double)ca) + fabs((double)cb) * T;
            const bool square = fabs((double)cc) * T * T >= 0x1p-60 * rest && cc != 0.f;
            const int unit = (int)(1022 - (__double_as_longlong(rest) >> 52 & 2047));
            const double over = square ? 1.0 / (double)cc : 1.0;
            const float start_unit = (float)ldexp(ca * over, square ? 2 * ea : unit), start_linear = (float)ldexp(cb * over, square ? 2 * to_a + 2 * ey : unit - 2 * ey);
            const float factor = square ? cc : 1.f;
            fe = square ? -2 * ea : -unit;
            const float scale_a = ortho_power(to_a);
#pragma unroll
            for (int i = 0; i < MB; ++i) {
                Terms t2[2];
                own_fragments(a[i], scale_a, t2);
#pragma unroll
                for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
                    for (int t = 0; t < TERMS; ++t) put<M>(lds, t, 2 * i + s2, t2[s2].t[t]);
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    a[i][e] = start_linear * a[i][e] + (i == wave && 8 * (e / 4) + 4 * (lane / 32) + e % 4 == (lane & 31) ? start_unit : 0.f);
            }
            __syncthreads();
            if (square)
#pragma unroll
                for (int i = 0; i < MB; ++i) {
                    floatx16 low = zero();
#pragma unroll
                    for (int p = 0; p < 2 * MB; ++p) multiply(row_fragment<M>(lds, 32 * i, p), row_fragment<M>(lds, 32 * wave, p).t, a[i], low);
                    add(a[i], low);
                }
            high = 0;
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) high = magnitude(a[i][e]) > high ? magnitude(a[i][e]) : high;
            // (times c here, not later: near its fixed point the factor is close to the identity, which one term holds as it is)
            high = wave_extreme<true>(high);
            const int to_f = high ? ORTHO_TOP + 253 - (int)(high >> 23) - (int)(magnitude(factor) >> 23) : 0;
            const float scale_f = ldexpf(factor, to_f);
            fe -= to_f;
            __syncthreads();                                  // A has been read
            put_y(lds);
            __builtin_amdgcn_sched_barrier(0);                // (Y's registers are free for F)
            wordx4 f[TERMS][2 * MB];                          // own rows of F
#pragma unroll
            for (int i = 0; i < MB; ++i) {
                Terms t2[2];
                own_fragments(a[i], scale_f, t2);
#pragma unroll
                for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
                    for (int t = 0; t < TERMS; ++t) f[t][2 * i + s2] = t2[s2].t[t];
            }
            __syncthreads();
            // own rows of F Y: column block by column block, Y's columns as the first operand
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                floatx16 low = zero();
                next[j] = zero();
#pragma unroll
                for (int p = 0; p < 2 * MB; ++p) {
                    Terms u;
                    wordx4 v[TERMS];
#pragma unroll
                    for (int t = 0; t < TERMS; ++t) {
                        // sixteen lanes read 4 rows x 16 columns and get 4 rows of a column each
                        const int row = 16 * p + 8 * (lane / 32) + (lane & 15) / 4, col = 32 * j + (lane & 16) + 4 * (lane & 3);
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint16_t *from = lds + t * (M * N) + line_at<N>(row + 4 * h, col / 8) + (col & 7);
                            const wordx2 w = __builtin_bit_cast(wordx2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((direct_trptr_t)from));
                            u.t[t][2 * h] = w[0];
                            u.t[t][2 * h + 1] = w[1];
                        }
                        v[t] = f[t][p];
                    }
                    multiply(u, v, next[j], low);
                }
                add(next[j], low);
            }
            high = 0;
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) high = magnitude(next[j][e]) > high ? magnitude(next[j][e]) : high;
            high = wave_extreme<true>(high);
            fe -= ey;
            if (lane == 0) tops[wave] = high == 0 ? NOTHING : (int)(high >> 23) - 127 + fe;
            __syncthreads();                                  // the old Y has been read
            if (step + 1 == g.steps) break;
            const int e = largest();
            ey = e == NOTHING ? 0 : ORTHO_TOP - e;
            const float scale_y = high ? ortho_power(fe + ey) : 0.f;
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                Terms t2[2];
                own_fragments(next[j], scale_y, t2);
#pragma unroll
                for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
                    for (int t = 0; t < TERMS; ++t) y[t][2 * j + s2] = t2[s2].t[t];
            }
            put_y(lds);
            __syncthreads();
        }
        const float half = high ? ortho_power(fe / 2) : 0.f, other = high ? ortho_power(fe - fe / 2) : 0.f;   // (no infinity times zero)
        float *result = reinterpret_cast<float *>(lds);
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                floatx4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = next[j][4 * q + e] * half * other;
                *reinterpret_cast<floatx4 *>(result + place(32 * wave + (lane & 31), 32 * j + 8 * q + 4 * (lane / 32))) = v;
            }
        __syncthreads();
        give(g, matrix * size, m, n, result);
    }
};

template <int MB, int NB>
__global__ __launch_bounds__(WAVE *MB) __attribute__((amdgpu_waves_per_eu(NB <= 3 ? 3 : 2))) void ortho_small_kernel(OrthoSmallArgs g)
{
    __shared__ __attribute__((aligned(16))) uint16_t lds[OrthoSmall<MB, NB>::LDS_HALVES];
    __shared__ double sums[MB];
    __shared__ int tops[MB];
    OrthoSmall<MB, NB> s;
    s.run(g, lds, sums, tops);
}

}  // namespace ivf
