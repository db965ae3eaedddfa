// A workgroup's tile of a matrix product a b^T on the matrix cores, shared by the grouped products, the orthogonalising steps and the
// products with 4-bit rows: operands of several element types and orientations go through registers into LDS as 16-bit terms, from there as
// fragments into v_mfma_f32_32x32x16 with fp32 accumulators.
//
// Terms.  16-bit operands of one type are multiplied as they are.  Otherwise an operand is a sum of bfloat16 terms: a 32-bit value is cut
// into three (8 significant bits each, x = t0 + t1 + t2 exactly while t2 is no subnormal), an fp16 value into two, a 4-bit value with its scale is one.  Of the products of
// terms those with i + j < max(terms of a, terms of b) are formed: for two 32-bit operands six of nine, what is left out is below
// 2^-21 |a_k b_k| each and about 2^-24 on average, an fp32 rounding.  bfloat16 has fp32's range of exponents, so no scale has to be found
// first (a pass over the rows, and over the columns for a gradient); an fp32 MFMA reaches a sixteenth of the 16-bit rate, six products a
// sixth.  The instructions round their sum, which makes six roundings of it for 16 products where fp32 by itself would have 16: sums of a few hundred products and more are
// less accurate than plain fp32 by that (1024 products 4.9e-7 of the result, plain 2.9e-7), which all nine products would not change (4.9e-7).  So the five products with a
// later term, a 128th of the first's size, go into sums of their own (APART), added at the end: 1.9e-7.  Infinite 32-bit operands need care: infinity less infinity is NaN, and infinity times a later
// term that is zero.  By single terms (4-bit values) they are the first term and nothing else; results of two 32-bit operands that come out as NaN are formed again in fp32 (mend).
#pragma once
#include <type_traits>

#include "util.hpp"

namespace ivf {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t wordx2 __attribute__((ext_vector_type(2)));
typedef uint32_t wordx4 __attribute__((ext_vector_type(4)));

// How an operand's element (r, k), k the index that is summed over, lies in memory:
//   *_ROWS  at r * ld + k;  *_COLS  at k * ld + r;  X4_*: rows of 4-bit values with scale bytes, ld bytes of codes and ld / 16 scales a row
enum class Form { H_ROWS, H_COLS, F_ROWS, F_COLS, HALF_ROWS, X4_ROWS, X4_COLS };

// Words at any address of global memory (the hardware takes them unaligned).
template <class W>
__device__ __forceinline__ W words_at(const void *p)
{
    W w;
    __builtin_memcpy(&w, p, sizeof w);
    return w;
}

template <class W>
__device__ __forceinline__ void put_words(void *p, W w) { __builtin_memcpy(p, &w, sizeof w); }

struct Source {
    const uint8_t *p;          // element (0, 0) of the tile's first row
    const uint8_t *scale;      // X4: its scale byte
    int64_t ld;
    int rows;                  // rows that exist, from the first on: others count as zeros
};

// LDS image of an operand: [term][row][BK], pieces of 8 elements (16 bytes) exchanged inside a row so that 16 rows in a
// run have the same piece in 16 different 16-byte places of the 256 bytes that one access covers.
template <int BK>
__device__ __forceinline__ int piece_at(int row, int piece)
{
    constexpr int CH = BK / 8, RUN = 16 / CH;
    return row * BK + ((piece ^ ((row / RUN) & (CH - 1))) * 8);
}

// The same for lines of W = 32, 64, 96 or 128 elements that transposing reads take columns of as well.  Pieces are exchanged inside a line so that the same piece of 16
// lines, and the four neighbouring pieces of four lines that a transposing read takes, lie in different 16-byte places of 256.
template <int W>
__device__ __forceinline__ int line_at(int line, int piece)
{
    const int low = (line >> 2) & 3;
    const int by = W == 128 ? ((line & 3) << 2) | low : W == 64 ? ((line & 2) << 1) | low : low;
    return line * W + ((piece ^ by) * 8);
}

__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// Terms of N 32-bit values (N even), two a word: the high 16 bits, then those of what is left; the last term rounded to nearest, which for
// three terms is exact and for two leaves 2^-17.  INFINITE: of an infinity nothing is left (else infinity less infinity, NaN), so that its products with
// single terms are what they are in fp32.
template <int TERMS, int N, bool INFINITE>
__device__ __forceinline__ void cut(const float (&v)[N], uint32_t (&out)[TERMS][N / 2])
{
    float x[N];
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = v[j];
#pragma unroll
    for (int t = 0; t < TERMS; ++t) {
#pragma unroll
        for (int j = 0; j < N / 2; ++j) {
            if (t + 1 < TERMS) out[t][j] = high_halves(__float_as_uint(x[2 * j]), __float_as_uint(x[2 * j + 1]));
            else out[t][j] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x[2 * j], (__bf16)x[2 * j + 1]});
        }
        if (t + 1 < TERMS)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float high = __uint_as_float(__float_as_uint(x[j]) & 0xFFFF0000u);
                x[j] = INFINITE && t == 0 && x[j] == high ? 0.f : x[j] - high;
            }
    }
}

// Eight 4-bit values (the low one first) times 2^(scale - 127) as bfloat16; scale 255 makes all of them NaN.
__device__ __forceinline__ wordx4 expand8(uint32_t codes, float scale)
{
    wordx4 o;
    o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
    o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
    o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
    o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
    return o;
}

// 2^(byte - 127); 2^-127 as the subnormal that it is, 255 as NaN
__device__ __forceinline__ float scale_of(uint32_t byte)
{
    return __uint_as_float(byte == 0 ? 0x00400000u : byte == 255 ? 0x7FC00000u : byte << 23);
}

// Brings ROWS x BK elements of an operand into LDS by NT threads: load() requests them into registers, store() writes them.  INFINITE: as cut().
template <Form FORM, int ROWS, int BK, int NT, int TERMS, bool INFINITE>
struct Loader {
    static constexpr int CH = BK / 8;
    static constexpr bool HALVES = FORM == Form::H_ROWS || FORM == Form::HALF_ROWS;
    static constexpr bool COLS = FORM == Form::H_COLS || FORM == Form::F_COLS;   // an item: 8 k of two neighbouring rows
    static constexpr int ITEM_COUNT = COLS ? ROWS / 2 * CH : FORM == Form::X4_ROWS ? ROWS * CH / 4
                                      : FORM == Form::X4_COLS ? ROWS / 8 * CH : ROWS * CH;
    static constexpr int ITEMS = (ITEM_COUNT + NT - 1) / NT;
    static constexpr int WORDS = HALVES ? 4 : FORM == Form::X4_ROWS ? 5 : FORM == Form::X4_COLS || FORM == Form::F_COLS ? 16 : 8;
    static constexpr int LDS_HALVES = TERMS * ROWS * BK;
    uint32_t w[ITEMS][WORDS];

    __device__ __forceinline__ void load(const Source &s, int64_t k0, int64_t K)
    {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int id = (int)threadIdx.x + i * NT;
            uint32_t(&v)[WORDS] = w[i];
#pragma unroll
            for (int j = 0; j < WORDS; ++j) v[j] = 0;
            if (ITEM_COUNT % NT != 0 && id >= ITEM_COUNT) continue;
            if constexpr (HALVES) {
                const int row = id / CH;
                const int64_t k = k0 + (id % CH) * 8;
                if (row >= s.rows || k >= K) continue;
                const uint16_t *p = reinterpret_cast<const uint16_t *>(s.p) + row * s.ld + k;
                if (k + 8 <= K) {
                    const wordx4 q = words_at<wordx4>(p);
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = q[j];
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (k + j < K) v[j / 2] |= (uint32_t)p[j] << (16 * (j & 1));
                }
            } else if constexpr (FORM == Form::F_ROWS) {
                const int row = id / CH;
                const int64_t k = k0 + (id % CH) * 8;
                if (row >= s.rows || k >= K) continue;
                const uint32_t *p = reinterpret_cast<const uint32_t *>(s.p) + row * s.ld + k;
                if (k + 8 <= K) {
                    const wordx4 q0 = words_at<wordx4>(p), q1 = words_at<wordx4>(p + 4);
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = q0[j], v[j + 4] = q1[j];
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (k + j < K) v[j] = p[j];
                }
            } else if constexpr (COLS) {
                // a wavefront that has one piece of k only reads at addresses that lanes add one offset to
                const int r = 2 * (id % (ROWS / 2)), c = id / (ROWS / 2);
                const int64_t k = k0 + 8 * (ROWS / 2 % WAVE == 0 ? __builtin_amdgcn_readfirstlane(c) : c);
                if (r >= s.rows) continue;
                const bool two = r + 1 < s.rows;
                constexpr int E = FORM == Form::F_COLS ? 4 : 2;
                const uint8_t *line = s.p + k * s.ld * E;
                const uint32_t off = (uint32_t)r * E;
#pragma unroll
                for (int j = 0; j < 8; ++j, line += s.ld * E) {
                    if (k + j >= K) continue;
                    if constexpr (FORM == Form::F_COLS) {
                        if (two) {
                            const wordx2 q = words_at<wordx2>(line + off);
                            v[2 * j] = q[0], v[2 * j + 1] = q[1];
                        } else {
                            v[2 * j] = *reinterpret_cast<const uint32_t *>(line + off);
                        }
                    } else {
                        v[j] = two ? words_at<uint32_t>(line + off) : *reinterpret_cast<const uint16_t *>(line + off);
                    }
                }
            } else if constexpr (FORM == Form::X4_ROWS) {
                const int row = id / (CH / 4);
                const int64_t block = k0 / 32 + id % (CH / 4);
                if (row >= s.rows || block * 32 >= K) continue;
                const wordx4 q = *reinterpret_cast<const wordx4 *>(s.p + row * s.ld + block * 16);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = q[j];
                v[4] = s.scale[row * (s.ld / 16) + block];
            } else {
                const int r = 8 * (id % (ROWS / 8));
                const int64_t k = k0 + (id / (ROWS / 8)) * 8;
                if (r >= s.rows) continue;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (k + j < K) {
                        v[j] = *reinterpret_cast<const uint32_t *>(s.p + (k + j) * s.ld + r / 2);
                        v[8 + j] = s.scale[(k + j) * (s.ld / 16) + r / 32];
                    }
            }
        }
    }

    __device__ __forceinline__ void store(uint16_t *lds) const
    {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int id = (int)threadIdx.x + i * NT;
            const uint32_t(&v)[WORDS] = w[i];
            if (ITEM_COUNT % NT != 0 && id >= ITEM_COUNT) continue;
            auto put = [&](int term, int row, int piece, wordx4 q) {
                *reinterpret_cast<wordx4 *>(lds + term * (ROWS * BK) + piece_at<BK>(row, piece)) = q;
            };
            if constexpr (FORM == Form::H_ROWS) {
                put(0, id / CH, id % CH, wordx4{v[0], v[1], v[2], v[3]});
            } else if constexpr (FORM == Form::H_COLS) {
                const int r = 2 * (id % (ROWS / 2)), c = id / (ROWS / 2);
                put(0, r, c, wordx4{low_halves(v[0], v[1]), low_halves(v[2], v[3]), low_halves(v[4], v[5]), low_halves(v[6], v[7])});
                put(0, r + 1, c, wordx4{high_halves(v[0], v[1]), high_halves(v[2], v[3]), high_halves(v[4], v[5]), high_halves(v[6], v[7])});
            } else if constexpr (FORM == Form::X4_ROWS) {
                const int row = id / (CH / 4), c = 4 * (id % (CH / 4));
                const float sc = scale_of(v[4]);
#pragma unroll
                for (int j = 0; j < 4; ++j) put(0, row, c + j, expand8(v[j], sc));
            } else if constexpr (FORM == Form::X4_COLS) {
                const int r = 8 * (id % (ROWS / 8)), c = id / (ROWS / 8);
                wordx4 e[8];                                   // [k] eight components
#pragma unroll
                for (int j = 0; j < 8; ++j) e[j] = expand8(v[j], scale_of(v[8 + j]));
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    put(0, r + 2 * h, c, wordx4{low_halves(e[0][h], e[1][h]), low_halves(e[2][h], e[3][h]), low_halves(e[4][h], e[5][h]), low_halves(e[6][h], e[7][h])});
                    put(0, r + 2 * h + 1, c, wordx4{high_halves(e[0][h], e[1][h]), high_halves(e[2][h], e[3][h]), high_halves(e[4][h], e[5][h]), high_halves(e[6][h], e[7][h])});
                }
            } else if constexpr (FORM == Form::F_COLS) {
                const int r = 2 * (id % (ROWS / 2)), c = id / (ROWS / 2);
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    float x[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(v[2 * j + u]);
                    uint32_t t[TERMS][4];
                    cut<TERMS, 8, INFINITE>(x, t);
#pragma unroll
                    for (int q = 0; q < TERMS; ++q) put(q, r + u, c, wordx4{t[q][0], t[q][1], t[q][2], t[q][3]});
                }
            } else {
                float x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if constexpr (FORM == Form::HALF_ROWS) x[j] = (float)__builtin_bit_cast(_Float16, (uint16_t)(v[j / 2] >> (16 * (j & 1))));
                    else x[j] = __uint_as_float(v[j]);
                }
                uint32_t t[TERMS][4];
                cut<TERMS, 8, INFINITE>(x, t);
#pragma unroll
                for (int q = 0; q < TERMS; ++q) put(q, id / CH, id % CH, wordx4{t[q][0], t[q][1], t[q][2], t[q][3]});
            }
        }
    }
};

// Element types of the C ABI, and results rounded once to them.
enum class Type { F32, F16, BF16 };

template <Type T>
__device__ __forceinline__ float element(const void *p, int64_t at)
{
    if constexpr (T == Type::F32) return static_cast<const float *>(p)[at];
    else if constexpr (T == Type::F16) return (float)static_cast<const _Float16 *>(p)[at];
    else return (float)static_cast<const __bf16 *>(p)[at];
}

// Eight elements in a run.
template <Type T>
__device__ __forceinline__ void eight(const void *p, int64_t at, float (&v)[8])
{
    if constexpr (T == Type::F32) {
        const floatx4 q[2] = {words_at<floatx4>(static_cast<const float *>(p) + at), words_at<floatx4>(static_cast<const float *>(p) + at + 4)};
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = q[j / 4][j % 4];
    } else {
        const wordx4 q = words_at<wordx4>(static_cast<const uint16_t *>(p) + at);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint16_t h = (uint16_t)(q[j / 2] >> (16 * (j & 1)));
            v[j] = T == Type::F16 ? (float)__builtin_bit_cast(_Float16, h) : __uint_as_float((uint32_t)h << 16);
        }
    }
}

// Eight elements in a run, `count` of them there, zeros for the others.
template <Type T>
__device__ __forceinline__ void eight_of(const void *p, int64_t at, int count, float (&v)[8])
{
    if (count >= 8) {
        eight<T>(p, at, v);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < count ? element<T>(p, at + j) : 0.f;
    }
}

__device__ __forceinline__ uint32_t two_halves(float a, float b, bool bf16)
{
    if (bf16) return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
    typedef _Float16 halfx2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, halfx2{(_Float16)a, (_Float16)b});
}

// Up to four values in a run to row-major memory.
__device__ __forceinline__ void put4(void *out, int64_t at, floatx4 v, int count, Type type)
{
    if (type == Type::F32) {
        float *p = static_cast<float *>(out) + at;
        if (count >= 4) {
            put_words(p, v);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j < count) p[j] = v[j];
        }
    } else {
        uint16_t *p = static_cast<uint16_t *>(out) + at;
        const wordx2 h = {two_halves(v[0], v[1], type == Type::BF16), two_halves(v[2], v[3], type == Type::BF16)};
        if (count >= 4) {
            put_words(p, h);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j < count) p[j] = (uint16_t)(h[j / 2] >> (16 * (j & 1)));
        }
    }
}

// A tile of a row-major result: rows of b are its rows, rows of a its columns, `rows` by `cols` of them there.  A lane's accumulators are runs of four columns of one row: written as they are, an instruction would touch
// 32 rows by 32 bytes.  Each wavefront turns its 32 rows through LDS (its own part of `lds`, which nobody reads any more), 16-byte pieces of a
// row exchanged by the row's number against bank conflicts, and writes rows in whole.
// F: accumulators side by side that are turned at a time (a wavefront's room is 4 KB for each).
template <int F, class P>
__device__ __forceinline__ void store_tile(const P &t, void *out, int64_t ld, int rows, int cols, Type type, uint16_t *lds)
{
    constexpr int W = 32 * F, CH = W / 4;                      // columns at a time, pieces of four of them
    const int lane = threadIdx.x & (WAVE - 1);
    float *own = reinterpret_cast<float *>(lds) + (int)(threadIdx.x / WAVE) * (32 * W);
#pragma unroll
    for (int at = 0; at < P::FA * P::FB / F; ++at) {
        const int j = at / (P::FA / F), first = at % (P::FA / F) * F, c0 = P::row_a(first);
        const int r0 = P::row_b(j), row = lane & 31;
        if (r0 >= rows || c0 >= cols) continue;
        wave_sync();
#pragma unroll
        for (int i = 0; i < F; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<floatx4 *>(own + row * W + (((8 * i + 2 * q + lane / 32) ^ (row & (CH - 1))) * 4)) =
                    floatx4{t.acc[first + i][j][4 * q], t.acc[first + i][j][4 * q + 1], t.acc[first + i][j][4 * q + 2], t.acc[first + i][j][4 * q + 3]};
        wave_sync();
        if (type == Type::F32) {
#pragma unroll
            for (int k = 0; k < CH * 32 / WAVE; ++k) {
                const int r = (k * WAVE + lane) / CH, c = (k * WAVE + lane) % CH;
                const floatx4 v = *reinterpret_cast<const floatx4 *>(own + r * W + ((c ^ (r & (CH - 1))) * 4));
                const int col = c0 + 4 * c;
                if (r0 + r < rows && col < cols) put4(out, (r0 + r) * ld + col, v, cols - col, Type::F32);
            }
        } else {
#pragma unroll
            for (int k = 0; k < CH * 16 / WAVE; ++k) {
                const int r = (k * WAVE + lane) / (CH / 2), c = (k * WAVE + lane) % (CH / 2) * 2;
                const floatx4 u = *reinterpret_cast<const floatx4 *>(own + r * W + ((c ^ (r & (CH - 1))) * 4));
                const floatx4 v = *reinterpret_cast<const floatx4 *>(own + r * W + (((c + 1) ^ (r & (CH - 1))) * 4));
                const int col = c0 + 4 * c;
                if (r0 + r >= rows || col >= cols) continue;
                uint16_t *p = static_cast<uint16_t *>(out) + (r0 + r) * ld + col;
                if (col + 8 <= cols) {
                    wordx4 h;
                    if (type == Type::BF16) h = wordx4{two_halves(u[0], u[1], true), two_halves(u[2], u[3], true), two_halves(v[0], v[1], true), two_halves(v[2], v[3], true)};
                    else h = wordx4{two_halves(u[0], u[1], false), two_halves(u[2], u[3], false), two_halves(v[0], v[1], false), two_halves(v[2], v[3], false)};
                    put_words(p, h);
                } else {
                    put4(p, 0, u, cols - col, type);
                    if (col + 4 < cols) put4(p, 4, v, cols - col - 4, type);
                }
            }
        }
    }
}

// Whether any element of the workgroup's tile is NaN, for all of its threads.
template <class P>
__device__ __forceinline__ bool any_nan(const P &t)
{
    bool bad = false;
#pragma unroll
    for (int i = 0; i < P::FA; ++i)
#pragma unroll
        for (int j = 0; j < P::FB; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) bad |= t.acc[i][j][e] != t.acc[i][j][e];
    return __syncthreads_or(bad);
}

// Elements of a stored tile [rows][cols] that are NaN anew, as the sum of a(row, k) b(col, k) over k < K one after the other in fp32: for tiles with infinities, or with NaN, whose
// sums end at the first.
template <class A, class B>
__device__ void mend(float *out, int64_t ld, int rows, int cols, int64_t K, A a, B b)
{
    __syncthreads();                                          // the tile is stored
    for (int i = threadIdx.x; i < rows * cols; i += blockDim.x) {
        const int row = i / cols, col = i % cols;
        float *p = out + row * ld + col;
        if (*p == *p) continue;
        float s = 0.f;
        for (int64_t k = 0; k < K && s == s; ++k) s = fmaf(a(row, k), b(col, k), s);
        *p = s;
    }
}

// Workgroups are dealt to the eight XCDs in turn: the place in a list of which every XCD takes one run, so that
// neighbours in the list share that XCD's L2.
__device__ __forceinline__ uint32_t place_of_block(uint32_t block, uint32_t blocks)
{
    const uint32_t xcd = block % 8, each = blocks / 8, more = blocks % 8;
    return xcd * each + (xcd < more ? xcd : more) + block / 8;
}

// What a tile is made of: BA rows of a by BB rows of b, wavefronts as WA x WB of them, BK elements a step, one or two steps' room in LDS (two
// spare a barrier, one leaves room for more workgroups).  APART: the products of later terms have sums of their own.
template <Form FORM_A, int TERMS_A, int BA, int WA, Form FORM_B, int TERMS_B, int BB, int WB, int BK, int BUFS, bool HALF, bool APART = false>
struct Tile {
    static constexpr int NT = WAVE * WA * WB;
    static constexpr int FA = BA / WA / 32, FB = BB / WB / 32;       // accumulators of a wavefront
    static constexpr int MOST = TERMS_A > TERMS_B ? TERMS_A : TERMS_B;
    using LA = Loader<FORM_A, BA, BK, NT, TERMS_A, TERMS_B == 1>;
    using LB = Loader<FORM_B, BB, BK, NT, TERMS_B, TERMS_A == 1>;
    static constexpr int STEP = LA::LDS_HALVES + LB::LDS_HALVES;     // 16-bit words of LDS a step
    static constexpr int OUT_HALVES = NT / WAVE * 32 * (32 * FA) * 2;   // what store() needs
    static constexpr int LDS_HALVES = BUFS * STEP > OUT_HALVES ? BUFS * STEP : OUT_HALVES;

    floatx16 acc[FA][FB], later[APART ? FA : 1][APART ? FB : 1];

    static __device__ __forceinline__ int row_a(int f) { return (int)(threadIdx.x / WAVE) / WB * (FA * 32) + f * 32; }
    static __device__ __forceinline__ int row_b(int f) { return (int)(threadIdx.x / WAVE) % WB * (FB * 32) + f * 32; }

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < FA; ++i)
#pragma unroll
            for (int j = 0; j < FB; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    acc[i][j][e] = 0.f;
                    if constexpr (APART) later[i][j][e] = 0.f;
                }
    }

    // rows_a, rows_b: rows that exist; fragments of others are not multiplied
    __device__ __forceinline__ void step(const uint16_t *la, const uint16_t *lb, int rows_a, int rows_b)
    {
        const int lane = threadIdx.x & (WAVE - 1);
        const int there_a = __builtin_amdgcn_readfirstlane(rows_a - row_a(0)), there_b = __builtin_amdgcn_readfirstlane(rows_b - row_b(0));
#pragma unroll
        for (int ks = 0; ks < BK / 16; ++ks) {
            wordx4 a[TERMS_A][FA], b[TERMS_B][FB];
            const int piece = 2 * ks + lane / 32;
#pragma unroll
            for (int t = 0; t < TERMS_A; ++t)
#pragma unroll
                for (int i = 0; i < FA; ++i)
                    a[t][i] = *reinterpret_cast<const wordx4 *>(la + t * (BA * BK) + piece_at<BK>(row_a(i) + (lane & 31), piece));
#pragma unroll
            for (int t = 0; t < TERMS_B; ++t)
#pragma unroll
                for (int j = 0; j < FB; ++j)
                    b[t][j] = *reinterpret_cast<const wordx4 *>(lb + t * (BB * BK) + piece_at<BK>(row_b(j) + (lane & 31), piece));
            // the small products first
#pragma unroll
            for (int order = MOST - 1; order >= 0; --order)
#pragma unroll
                for (int t = 0; t < TERMS_A; ++t) {
                    if (order - t < 0 || order - t >= TERMS_B) continue;
#pragma unroll
                    for (int i = 0; i < FA; ++i)
#pragma unroll
                        for (int j = 0; j < FB; ++j) {
                            if (FA * FB > 1 && (there_a <= 32 * i || there_b <= 32 * j)) continue;
                            const wordx4 u = a[t][i], v = b[order - t][j];
                            floatx16 *sum = &acc[i][j];
                            if constexpr (APART) sum = order > 0 ? &later[i][j] : sum;
                            if constexpr (HALF)
                                *sum = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(halfx8, u), __builtin_bit_cast(halfx8, v), *sum, 0, 0, 0);
                            else
                                *sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, u), __builtin_bit_cast(bf16x8, v), *sum, 0, 0, 0);
                        }
                }
        }
    }

    // acc += a b^T over k in [from, K); lds: LDS_HALVES words
    __device__ __forceinline__ void product(const Source &sa, const Source &sb, int64_t from, int64_t K, uint16_t *lds)
    {
        LA la;
        LB lb;
        la.load(sa, from, K);
        lb.load(sb, from, K);
        int at = 0;
        for (int64_t k = from; k < K; k += BK, at ^= BUFS - 1) {
            uint16_t *buf = lds + at * STEP;
            if (BUFS == 1 && k > from) __syncthreads();
            la.store(buf);
            lb.store(buf + LA::LDS_HALVES);
            __syncthreads();
            if (k + BK < K) {
                la.load(sa, k + BK, K);
                lb.load(sb, k + BK, K);
            }
            step(buf, buf + LA::LDS_HALVES, sa.rows, sb.rows);
        }
        if constexpr (APART)
#pragma unroll
            for (int i = 0; i < FA; ++i)
#pragma unroll
                for (int j = 0; j < FB; ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        acc[i][j][e] += later[i][j][e];
                        later[i][j][e] = 0.f;
                    }
        __syncthreads();
    }

    __device__ __forceinline__ void store(void *out, int64_t ld, int rows, int cols, Type type, uint16_t *lds) const { store_tile<FA>(*this, out, ld, rows, cols, type, lds); }

    // f(row of a, row of b, four values of rows of a in a run): every element of the tile, four at a time
    template <class F>
    __device__ __forceinline__ void each(F f) const
    {
        const int lane = threadIdx.x & (WAVE - 1);
#pragma unroll
        for (int i = 0; i < FA; ++i)
#pragma unroll
            for (int j = 0; j < FB; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const floatx4 v = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                    f(row_a(i) + 8 * q + 4 * (lane / 32), row_b(j) + (lane & 31), v);
                }
    }
};

}  // namespace ivf
