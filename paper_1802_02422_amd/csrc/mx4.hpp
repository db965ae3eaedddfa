// Rows in microscaled 4-bit floating point (OCP MX: E2M1 elements, one E8M0 scale for 32): a row of D components is ceil(D / 32) blocks of 16
// bytes, two elements a byte, the first in the low half, and as many scale bytes s for 2^(s - 127).  Elements stand for 0, 0.5, 1, 1.5, 2, 3, 4, 6 (bit 3:
// the sign).  A block's scale is 2^(floor(log2 largest magnitude) - 2), not below 2^-127; elements are rounded to nearest, ties to even,
// and held to 6.  A block with an infinity or a NaN gets the scale byte 255, which makes all of it NaN; elements past D are zeros.
#pragma once
#include "ortho.hpp"

namespace ivf {

// Bound by memory: a lane takes eight components (one or two 16-byte words), four lanes a block, whose largest magnitude they share by DPP; codes
// are written as a 4-byte word a lane, next to each other.
// 10^6 x 96 fp32: 99 us, 4.4 TB/s.
template <Type T>
__global__ __launch_bounds__(256) void mx4_quantise_kernel(const void *__restrict__ x, int64_t ldx, int64_t n, int D, uint32_t *__restrict__ codes,
                                                           uint8_t *__restrict__ scales)
{
    const int blocks = (D + 31) / 32;
    const uint32_t id = blockIdx.x * 256 + threadIdx.x, row = id / (uint32_t)(4 * blocks);
    if (row >= n) return;                                      // (four lanes of a block together)
    const int c0 = (int)(id - row * (uint32_t)(4 * blocks)) * 8;
    const int64_t at = (int64_t)row * ldx + c0;
    float v[8];
    if (c0 + 8 <= D) {
        eight<T>(x, at, v);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = c0 + j < D ? element<T>(x, at + j) : 0.f;
    }
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t u = __float_as_uint(v[j]) & 0x7FFFFFFFu;
        top = u > top ? u : top;
    }
    uint32_t other = dpp_word_or_self<0xB1, 0xf>(top);         // quad_perm: lane ^ 1
    top = other > top ? other : top;
    other = dpp_word_or_self<0x4E, 0xf>(top);                  // lane ^ 2
    top = other > top ? other : top;
    // the scale's byte is the exponent's less two (a subnormal largest magnitude: 0, as below 2^-125)
    const uint32_t e = top >> 23;
    const uint32_t byte = e == 255 ? 255u : e < 2 ? 0u : e - 2;
    const float by = __uint_as_float((254u - (byte == 255 ? 127u : byte)) << 23);   // 2^(127 - byte), at most 2^127
    // scaled by a power of two the conversion's own scale is 1: it rounds to nearest, ties to even, and saturates
    uint32_t word = 0;
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[0] * by, v[1] * by, 1.f, 0);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[2] * by, v[3] * by, 1.f, 1);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[4] * by, v[5] * by, 1.f, 2);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[6] * by, v[7] * by, 1.f, 3);
    codes[id] = byte == 255 ? 0u : word;
    if ((c0 & 31) == 0) scales[id / 4] = (uint8_t)byte;
}

// A lane writes 16 bytes: four values in 32 bits, eight in 16.  10^6 x 96 to fp32: 85 us, 5.1 TB/s.
template <bool FLOAT>
__global__ __launch_bounds__(256) void mx4_expand_kernel(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales, int64_t n, int blocks, int D,
                                                         void *__restrict__ out, int64_t ldo, Type type)
{
    constexpr int PER = FLOAT ? 4 : 8;
    const int per = (D + PER - 1) / PER;
    const uint32_t id = blockIdx.x * 256 + threadIdx.x, row = id / (uint32_t)per;
    if (row >= n) return;
    const int c0 = (int)(id - row * (uint32_t)per) * PER;
    const uint8_t *p = codes + (int64_t)row * (blocks * 16) + c0 / 2;
    const float by = scale_of(scales[(int64_t)row * blocks + c0 / 32]);
    const uint32_t word = FLOAT ? *reinterpret_cast<const uint16_t *>(p) : *reinterpret_cast<const uint32_t *>(p);
    const wordx4 e = expand8(word, by);                        // (bfloat16: exact but for what 32 bits hold as infinity)
    if constexpr (FLOAT) {
        put4(out, row * ldo + c0, floatx4{__uint_as_float(e[0] << 16), __uint_as_float(e[0] & 0xFFFF0000u), __uint_as_float(e[1] << 16), __uint_as_float(e[1] & 0xFFFF0000u)},
             D - c0, Type::F32);
    } else {
        wordx4 h = e;
        if (type == Type::F16)
#pragma unroll
            for (int j = 0; j < 4; ++j) h[j] = two_halves(__uint_as_float(e[j] << 16), __uint_as_float(e[j] & 0xFFFF0000u), false);
        uint16_t *o = static_cast<uint16_t *>(out) + row * ldo + c0;
        if (c0 + 8 <= D) {
            put_words(o, h);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c0 + j < D) o[j] = (uint16_t)(h[j / 2] >> (16 * (j & 1)));
        }
    }
}

// out = a b^T, both in 4 bits, on v_mfma_scale_f32_32x32x64_f8f6f4: a lane gives 32 elements of a row, which is a block, and their scale byte.
// The codes go through LDS as pieces of 16 bytes like those of 16-bit operands (a block in a piece's place).
struct Mx4Args {
    const uint8_t *a, *sa;
    int64_t m;
    const uint8_t *b, *sb;
    int64_t n;
    int blocks;
    void *out;
    int64_t ldo;
    Type type;
    uint32_t first;            // workgroup of the list that this launch begins with
};

typedef int intx8 __attribute__((ext_vector_type(8)));

// Codes are copied into LDS as 16-bit operands are (direct.hpp), a block in the place of a piece.  Scale bytes go there too, a thread a row and 16 of
// them for every second step: rows lie a line or so apart, and lanes that fetched their own rows' eight bytes asked for four times as many
// lines as the codes have (335 us for 8192 x 8192 x 4096).  Two workgroups of 128 x 128 a compute unit (210 us, 2.62 PFLOP/s) do better than one of
// 256 x 256 (282 us), whose start and end nothing overlaps.
template <int BA, int WA, int BB, int WB>
struct Mx4Tile : DirectTile<false, 1, BA, WA, false, 1, BB, WB, 64, 2, false> {
    using P = DirectTile<false, 1, BA, WA, false, 1, BB, WB, 64, 2, false>;
    static constexpr int SUBS = 4, BLOCKS = 8;                 // of 64 elements, and blocks: a step

    static constexpr int ROWS = BA + BB;                      // scale bytes of a's rows, then of b's
    static_assert(P::NT == ROWS, "a thread a row");

    // Eight scale bytes of rows `row` + 32 f + lane % 32; the upper half of the wavefront takes odd blocks.
    template <int F>
    struct Scales {
        uint32_t w[F][2];
        template <class ROW>
        __device__ __forceinline__ void fetch(const wordx4 *scales, int odd, ROW row)
        {
            const int lane = threadIdx.x & 63;
#pragma unroll
            for (int f = 0; f < F; ++f) {
                const wordx2 v = reinterpret_cast<const wordx2 *>(scales + row(f) + (lane & 31))[odd];
                w[f][0] = v[0] >> lane / 32 * 8;
                w[f][1] = v[1] >> lane / 32 * 8;
            }
        }
    };

    // Sixteen scale bytes of a row from block k on, 127 (one) past the last.
    static __device__ __forceinline__ wordx4 scales_of_row(const uint8_t *p, int k, int blocks)
    {
        if (k + 16 <= blocks) return words_at<wordx4>(p + k);
        wordx4 v;
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            v[h] = 0x7F7F7F7Fu;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (k + 4 * h + j < blocks) v[h] = (v[h] & ~(255u << 8 * j)) | (uint32_t)p[k + 4 * h + j] << 8 * j;
        }
        return v;
    }

    template <int KS>
    __device__ __forceinline__ void multiply4(const typename P::Fragments &f, const Scales<P::FA> &sa, const Scales<P::FB> &sb)
    {
        constexpr int SEL = 2 * (KS & 1);
#pragma unroll
        for (int i = 0; i < P::FA; ++i)
#pragma unroll
            for (int j = 0; j < P::FB; ++j) {
                const wordx4 u = f.a[0][i], v = f.b[0][j];
                this->acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(intx8{(int)u[0], (int)u[1], (int)u[2], (int)u[3], 0, 0, 0, 0},
                                                                                 intx8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0}, this->acc[i][j], 4, 4,
                                                                                 SEL, (int)sa.w[i][KS / 2], SEL, (int)sb.w[j][KS / 2]);
            }
    }

    // as DirectTile::product, over `blocks` blocks
    __device__ __forceinline__ void product4(const DirectSource &sa, const uint8_t *ea, const DirectSource &sb, const uint8_t *eb, int blocks, uint16_t *lds,
                                             wordx4 (&scales)[2][ROWS])
    {
        constexpr int BK = 64;
        const int64_t K = (int64_t)blocks * 8;
        typename P::LA la;
        typename P::LB lb;
        la.init(sa);
        lb.init(sb);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            la.copy(sa, s * BK, K, lds + s * P::STEP);
            lb.copy(sb, s * BK, K, lds + s * P::STEP + P::LA::LDS_HALVES);
        }
        const bool of_a = threadIdx.x < BA;
        const int row = of_a ? (int)threadIdx.x : (int)threadIdx.x - BA, rows = of_a ? sa.rows : sb.rows;
        const uint8_t *own = (of_a ? ea : eb) + (int64_t)(row < rows ? row : 0) * blocks;
        scales[0][threadIdx.x] = scales_of_row(own, 0, blocks);
        wordx4 held;
        Scales<P::FA> xa;
        Scales<P::FB> xb;
        __builtin_amdgcn_s_waitcnt(direct_vmcnt(0));
        __syncthreads();
        typename P::Fragments f[2];
        P::fetch(f[0], lds, lds + P::LA::LDS_HALVES, 0);
        xa.fetch(scales[0], 0, P::row_a);
        xb.fetch(scales[0] + BA, 0, P::row_b);
        int at = 0;
        for (int k = 0; k < blocks; k += BLOCKS, at ^= 1) {
            uint16_t *buf = lds + at * P::STEP;
            const int pair = k / (2 * BLOCKS), odd = k / BLOCKS & 1;
            if (!odd) held = scales_of_row(own, k + 2 * BLOCKS, blocks);
            P::fetch(f[1], buf, buf + P::LA::LDS_HALVES, 1);
            multiply4<0>(f[0], xa, xb);
            P::template mix<0>();
            P::fetch(f[0], buf, buf + P::LA::LDS_HALVES, 2);
            multiply4<1>(f[1], xa, xb);
            P::template mix<0>();
            P::fetch(f[1], buf, buf + P::LA::LDS_HALVES, 3);
            multiply4<2>(f[0], xa, xb);
            P::template mix<0>();
            if (odd) scales[(pair + 1) & 1][threadIdx.x] = held;
            __builtin_amdgcn_s_waitcnt(direct_vmcnt(0));
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            const uint16_t *next = lds + (at ^ 1) * P::STEP;
            const Scales<P::FA> ya = xa;
            const Scales<P::FB> yb = xb;
            P::fetch(f[0], next, next + P::LA::LDS_HALVES, 0);
            xa.fetch(scales[(pair + odd) & 1], odd ^ 1, P::row_a);
            xb.fetch(scales[(pair + odd) & 1] + BA, odd ^ 1, P::row_b);
#pragma unroll
            for (int i = 0; i < P::LA::ITEMS; ++i) la.copy_one(sa, i, (int64_t)k * 8 + 2 * BK, K, buf);
#pragma unroll
            for (int i = 0; i < P::LB::ITEMS; ++i) lb.copy_one(sb, i, (int64_t)k * 8 + 2 * BK, K, buf + P::LA::LDS_HALVES);
            multiply4<3>(f[1], ya, yb);
            P::template mix<P::COPIES, P::FA + P::FB>();
        }
        __builtin_amdgcn_s_waitcnt(direct_vmcnt(0));
        __syncthreads();
    }
};

template <int BA, int WA, int BB, int WB>
__global__ __launch_bounds__(WAVE *WA *WB) void mx4_product_kernel(Mx4Args g)
{
    using P = Mx4Tile<BB, WB, BA, WA>;                         // b is the first operand: a lane gets neighbouring columns
    __shared__ __attribute__((aligned(16))) uint16_t lds[P::LDS_HALVES];
    __shared__ wordx4 scales[2][BA + BB];
    const int across = (int)((g.n + BB - 1) / BB), down = (int)((g.m + BA - 1) / BA);
    int i, j;
    tile_of_place(g.first + place_of_block(blockIdx.x, gridDim.x), down, across, i, j);
    const int64_t i0 = (int64_t)i * BA, j0 = (int64_t)j * BB;
    P t;
    t.clear();
    const DirectSource sa{reinterpret_cast<const uint16_t *>(g.a + i0 * g.blocks * 16), g.blocks * 8, (int)(g.m - i0 < BA ? g.m - i0 : BA)};
    const DirectSource sb{reinterpret_cast<const uint16_t *>(g.b + j0 * g.blocks * 16), g.blocks * 8, (int)(g.n - j0 < BB ? g.n - j0 : BB)};
    t.product4(sb, g.sb + j0 * g.blocks, sa, g.sa + i0 * g.blocks, g.blocks, lds, scales);
    t.store(static_cast<uint8_t *>(g.out) + (i0 * g.ldo + j0) * (g.type == Type::F32 ? 4 : 2), g.ldo, sa.rows, sb.rows, g.type, lds);
}

// A row's terms are cut anew for each tile; 256 fp32 rows by 65 536 rows of 96 components 22 us, 4096 rows 278 (where runs of tiles take 223).
// out = a b^T (a in 16 or 32 bits, b in 4 bits), or out = a b (TRANSPOSED: the sum goes over the rows of b, in parts where it is long and the
// result small, added afterwards in their order).
struct Mx4RowsArgs {
    const uint8_t *a;
    int64_t lda, m;
    const uint8_t *codes, *scales;
    int64_t n;
    int D;
    void *out;
    int64_t ldo;
    Type type;
    int parts;                 // TRANSPOSED: more than one: their sums go to part_sums
    int64_t part_rows;
    float *part_sums;          // [parts][m][D]
    uint32_t first;            // as in Mx4Args
};

template <Type T>
struct RowsElem {
    static constexpr Form form = T == Type::F32 ? Form::F_ROWS : T == Type::F16 ? Form::HALF_ROWS : Form::H_ROWS;
    static constexpr int terms = T == Type::F32 ? 3 : T == Type::F16 ? 2 : 1;
    static constexpr int bytes = T == Type::F32 ? 4 : 2;
    static constexpr int step = T == Type::BF16 ? 64 : 32;
    static constexpr int bufs = T == Type::F32 ? 1 : 2;
};

// Where b's values stand expanded as bfloat16 ([n][ld], ld: D rounded up to 8, zeros there).
struct Mx4Values {
    const uint16_t *p;
    int64_t ld;
};

// EXPANDED (TRANSPOSED only): b from its values.  Each tile of rows of a takes all of b, and to expand columns from their codes costs a piece of
// eight rows by eight columns some hundred instructions; from 256 rows of a on it is done once.
template <Type T, bool TRANSPOSED, bool EXPANDED, int BM, int BN>
__global__ __launch_bounds__(256) void mx4_rows_product_kernel(Mx4RowsArgs g, Mx4Values values)
{
    using E = RowsElem<T>;
    constexpr int WB = BM >= 64 ? 2 : 1;
    using P = Tile<EXPANDED ? Form::H_COLS : TRANSPOSED ? Form::X4_COLS : Form::X4_ROWS, 1, BN, 4 / WB, E::form, E::terms, BM, WB, E::step, E::bufs, false>;
    __shared__ __attribute__((aligned(16))) uint16_t lds[P::LDS_HALVES];
    const int blocks = (g.D + 31) / 32;
    const int64_t cols = TRANSPOSED ? g.D : g.n, across = (cols + BN - 1) / BN, down = (g.m + BM - 1) / BM;
    const uint32_t place = g.first + blockIdx.x;
    const int64_t j0 = (place % across) * BN, i0 = (place / across % down) * BM;
    const int part = (int)(place / (across * down));
    P t;
    t.clear();
    Source sb = EXPANDED ? Source{reinterpret_cast<const uint8_t *>(values.p + j0), nullptr, values.ld, (int)(cols - j0 < BN ? cols - j0 : BN)} : Source{TRANSPOSED ? g.codes + j0 / 2 : g.codes + j0 * blocks * 16, TRANSPOSED ? g.scales + j0 / 32 : g.scales + j0 * blocks, (int64_t)blocks * 16,
              (int)(cols - j0 < BN ? cols - j0 : BN)};
    Source sa{g.a + i0 * g.lda * E::bytes, nullptr, g.lda, (int)(g.m - i0 < BM ? g.m - i0 : BM)};
    const int64_t from = TRANSPOSED ? part * g.part_rows : 0;
    const int64_t to = TRANSPOSED ? (from + g.part_rows < g.n ? from + g.part_rows : g.n) : g.D;
    t.product(sb, sa, from, to, lds);
    if (!TRANSPOSED || g.parts == 1)
        t.store(static_cast<uint8_t *>(g.out) + (i0 * g.ldo + j0) * (g.type == Type::F32 ? 4 : 2), g.ldo, sa.rows, sb.rows, g.type, lds);
    else t.store(g.part_sums + (part * g.m + i0) * g.D + j0, g.D, sa.rows, sb.rows, Type::F32, lds);
}

// out = a b^T for rows of up to 128 components and many of them on both sides (queries against the rows of an index): a workgroup keeps 128 rows of a as
// fragments in registers, 32 a wavefront, cut into terms once, and goes over rows of b, 64 at a time.  Their codes are requested two tiles ahead and
// expanded into one of two buffers while the other is multiplied; the result's rows leave through LDS.  One barrier a tile.  4096 fp32 rows by
// 65 536 rows of 96 components: 223 us, bound by the 1.07 GB of scores (4.8 TB/s); 128 components 285 (198 registers, two wavefronts a SIMD).
struct SweepTile {
    static constexpr int FA = 2, FB = 1, NT = 256;
    floatx16 acc[FA][FB];
    static __device__ __forceinline__ int row_a(int f) { return 32 * f; }
    static __device__ __forceinline__ int row_b(int) { return (int)(threadIdx.x / WAVE) * 32; }
};

constexpr int SWEEP_ROWS = 128, SWEEP_COLS = 64;

template <Type T, int BLOCKS>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void mx4_sweep_kernel(Mx4RowsArgs g, int run)
{
    using E = RowsElem<T>;
    constexpr int TERMS = E::terms, W = 32 * BLOCKS, KS = 2 * BLOCKS;
    __shared__ __attribute__((aligned(16))) uint16_t values[2][SWEEP_COLS * W];
    __shared__ __attribute__((aligned(16))) float turned[4][32 * 32];
    const int lane = threadIdx.x & 63;
    const uint32_t down = (uint32_t)((g.m + SWEEP_ROWS - 1) / SWEEP_ROWS), place = g.first + place_of_block(blockIdx.x, gridDim.x);
    const int64_t i0 = (int64_t)(place % down) * SWEEP_ROWS, tiles = (g.n + SWEEP_COLS - 1) / SWEEP_COLS;
    const int64_t first = (int64_t)(place / down) * run, end = first + run < tiles ? first + run : tiles;
    const int rows = (int)(g.m - i0 < SWEEP_ROWS ? g.m - i0 : SWEEP_ROWS), own = __builtin_amdgcn_readfirstlane(SweepTile::row_b(0));
    wordx4 a[KS][TERMS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        const int k = 16 * ks + 8 * (lane / 32), row = own + (lane & 31);
        float v[8];
        eight_of<T>(g.a, (i0 + (row < rows ? row : 0)) * g.lda + k, row < rows ? g.D - k : 0, v);
        uint32_t t[TERMS][4];
        cut<TERMS, 8, true>(v, t);
#pragma unroll
        for (int q = 0; q < TERMS; ++q) a[ks][q] = wordx4{t[q][0], t[q][1], t[q][2], t[q][3]};
    }
    // a thread a block of a row of b
    const int line = threadIdx.x / BLOCKS, block = threadIdx.x % BLOCKS;
    wordx4 codes;
    uint32_t scale;
    auto bring = [&](int64_t tile) {
        const int64_t row = tile * SWEEP_COLS + line;
        codes = wordx4{0, 0, 0, 0};
        scale = 127;
        if (line < SWEEP_COLS && tile < end && row < g.n) {
            codes = *reinterpret_cast<const wordx4 *>(g.codes + (row * BLOCKS + block) * 16);
            scale = g.scales[row * BLOCKS + block];
        }
    };
    auto put = [&](uint16_t *to) {
        if (line >= SWEEP_COLS) return;
        const float by = scale_of(scale);
#pragma unroll
        for (int j = 0; j < 4; ++j) *reinterpret_cast<wordx4 *>(to + line_at<W>(line, 4 * block + j)) = expand8(codes[j], by);
    };
    bring(first);
    put(values[0]);
    bring(first + 1);
    SweepTile t;
    int at = 0;
    for (int64_t tile = first; tile < end; ++tile, at ^= 1) {
        __syncthreads();                                      // this tile's values are there, and the other buffer has been read
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
            for (int e = 0; e < 16; ++e) t.acc[f][0][e] = 0.f;
        if (own < rows)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                wordx4 b[2];
#pragma unroll
                for (int f = 0; f < 2; ++f) b[f] = *reinterpret_cast<const wordx4 *>(values[at] + line_at<W>(32 * f + (lane & 31), 2 * ks + lane / 32));
#pragma unroll
                for (int q = TERMS - 1; q >= 0; --q)          // the small terms first
#pragma unroll
                    for (int f = 0; f < 2; ++f)
                        t.acc[f][0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, b[f]), __builtin_bit_cast(bf16x8, a[ks][q]), t.acc[f][0], 0, 0, 0);
            }
        put(values[at ^ 1]);
        bring(tile + 2);
        const int64_t j0 = tile * SWEEP_COLS;
        store_tile<1>(t, static_cast<uint8_t *>(g.out) + (i0 * g.ldo + j0) * (g.type == Type::F32 ? 4 : 2), g.ldo, rows,
                      (int)(g.n - j0 < SWEEP_COLS ? g.n - j0 : SWEEP_COLS), g.type, reinterpret_cast<uint16_t *>(turned));
    }
}

// The same for a in bfloat16 with lines of whole 16-byte words and b's values: both straight into LDS.  4096 x 8192 by 8192 x 1024: 73 us,
// 940 TFLOP/s, where codes expanded for every tile took 236.
template <bool TRANSPOSED, int BM, int BN, int WM, int WN, int BK, int BUFS>
__global__ __launch_bounds__(WAVE *WM *WN) void mx4_direct_kernel(Mx4RowsArgs g, Mx4Values values)
{
    using P = DirectTile<TRANSPOSED, 1, BN, WN, false, 1, BM, WM, BK, BUFS, false>;
    __shared__ __attribute__((aligned(16))) uint16_t lds[P::LDS_HALVES];
    const int64_t cols = TRANSPOSED ? g.D : g.n;
    const int across = (int)((cols + BN - 1) / BN), down = (int)((g.m + BM - 1) / BM);
    const uint32_t place = g.first + place_of_block(blockIdx.x, gridDim.x), part = place / ((uint32_t)across * down);
    int i, j;
    tile_of_place(place % ((uint32_t)across * down), down, across, i, j);
    const int64_t i0 = (int64_t)i * BM, j0 = (int64_t)j * BN;
    const int64_t from = TRANSPOSED ? part * g.part_rows : 0, left = TRANSPOSED ? g.n - from : g.D, K = TRANSPOSED && left > g.part_rows ? g.part_rows : left;
    const DirectSource sb{values.p + (TRANSPOSED ? from * values.ld + j0 : j0 * values.ld), values.ld, (int)(cols - j0 < BN ? cols - j0 : BN)};
    const DirectSource sa{reinterpret_cast<const uint16_t *>(g.a) + i0 * g.lda + from, g.lda, (int)(g.m - i0 < BM ? g.m - i0 : BM)};
    P t;
    t.clear();
    t.product(sb, sa, K, lds);
    if (!TRANSPOSED || g.parts == 1)
        t.store(static_cast<uint8_t *>(g.out) + (i0 * g.ldo + j0) * (g.type == Type::F32 ? 4 : 2), g.ldo, sa.rows, sb.rows, g.type, lds);
    else t.store(g.part_sums + (part * g.m + i0) * g.D + j0, g.D, sa.rows, sb.rows, Type::F32, lds);
}

__global__ __launch_bounds__(256) void mx4_join_kernel(Mx4RowsArgs g)
{
    const int64_t size = g.m * g.D;
    const int per = (g.D + 3) / 4;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < g.m * per; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / per;
        const int c = (int)(i - row * per) * 4, count = g.D - c;
        floatx4 s = {0.f, 0.f, 0.f, 0.f};
        for (int q = 0; q < g.parts; ++q) {
            const float *p = g.part_sums + q * size + row * g.D + c;
            if (count >= 4) {
                s += words_at<floatx4>(p);
            } else {
#pragma unroll
                for (int j = 0; j < 3; ++j)
                    if (j < count) s[j] += p[j];
            }
        }
        put4(g.out, row * g.ldo + c, s, count, g.type);
    }
}

// out = a b^T for up to four rows of a (one query, one token): b is read once and is the traffic.  A lane takes a block of 32 components and keeps
// a's in registers (ONE: a row of b has no more blocks than LANES, the lanes that share it) or reads them from LDS, where blocks lie 36 words
// apart so that 16 lanes' words are in different banks.  1 x 10^6 x 128: 17 us, 4.1 TB/s.
constexpr int MX4_FEW = 4, MX4_PITCH = 36;

__device__ __forceinline__ void any_eight(const void *p, int64_t at, int count, Type type, float (&v)[8])
{
    if (type == Type::F32) eight_of<Type::F32>(p, at, count, v);
    else if (type == Type::F16) eight_of<Type::F16>(p, at, count, v);
    else eight_of<Type::BF16>(p, at, count, v);
}

// Sum over LANES lanes in a run, for each of them.
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v)
{
    if constexpr (LANES == 64) return wave_total(v);
    if constexpr (LANES == 16) return sum_of_16(v);
    v += dpp_or_self<0xB1, 0xf>(v);                            // quad_perm: lane ^ 1
    return v + dpp_or_self<0x4E, 0xf>(v);                      // lane ^ 2
}

// acc[i] += the products of a block's 32 values with a[i]
template <int M>
__device__ __forceinline__ void mx4_block(wordx4 codes, float scale, const float (&a)[M][32], float (&acc)[M])
{
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        typedef float floatx2 __attribute__((ext_vector_type(2)));
        const floatx2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[w], scale, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[w], scale, 1),
                              __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[w], scale, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[w], scale, 3)};
#pragma unroll
        for (int i = 0; i < M; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[i] = fmaf(v[j / 2][j % 2], a[i][8 * w + j], acc[i]);
    }
}

template <int M, int LANES, bool ONE>
__global__ __launch_bounds__(256) void mx4_few_kernel(Mx4RowsArgs g, Type type_a)
{
    extern __shared__ __attribute__((aligned(16))) float held[];               // !ONE: [M][blocks][MX4_PITCH]
    constexpr int PER = WAVE / LANES, RUN = M > 2 ? 2 : 4;                     // rows of b of a wavefront: side by side, and on their way
    const int blocks = (g.D + 31) / 32, lane = threadIdx.x & 63, sub = lane % LANES;
    float a[M][32];
    if constexpr (ONE) {
#pragma unroll
        for (int i = 0; i < M; ++i)
#pragma unroll
            for (int j = 0; j < 32; j += 8) {
                float v[8];
                any_eight(g.a, i * g.lda + 32 * sub + j, i < g.m ? g.D - 32 * sub - j : 0, type_a, v);
#pragma unroll
                for (int k = 0; k < 8; ++k) a[i][j + k] = v[k];
            }
    } else {
        for (int k = threadIdx.x; k < M * blocks * 4; k += 256) {
            const int i = k / (blocks * 4), c = k % (blocks * 4) * 8;
            float v[8];
            any_eight(g.a, i * g.lda + c, i < g.m ? g.D - c : 0, type_a, v);
            floatx4 *to = reinterpret_cast<floatx4 *>(held + (i * blocks + c / 32) * MX4_PITCH + c % 32);
            to[0] = floatx4{v[0], v[1], v[2], v[3]};
            to[1] = floatx4{v[4], v[5], v[6], v[7]};
        }
        __syncthreads();
    }
    const int64_t wave = (int64_t)blockIdx.x * 4 + threadIdx.x / WAVE, stride = (int64_t)gridDim.x * (4 * PER * RUN);
    struct Blocks {
        wordx4 codes[RUN];
        uint32_t scale[RUN];
    };
    auto bring = [&](int64_t first, int b) {
        Blocks v;
#pragma unroll
        for (int u = 0; u < RUN; ++u) {
            const int64_t row = first + u * PER + lane / LANES;
            const bool there = row < g.n && b < blocks;
            v.codes[u] = there ? *reinterpret_cast<const wordx4 *>(g.codes + (row * blocks + b) * 16) : wordx4{0, 0, 0, 0};
            v.scale[u] = there ? g.scales[row * blocks + b] : 127;
        }
        return v;
    };
    // the next blocks are on their way while these are multiplied
    Blocks next = bring(wave * (PER * RUN), sub);
    for (int64_t first = wave * (PER * RUN); first < g.n; first += stride) {
        float acc[RUN][M];
#pragma unroll
        for (int u = 0; u < RUN; ++u)
#pragma unroll
            for (int i = 0; i < M; ++i) acc[u][i] = 0.f;
        for (int b = sub; b - sub < blocks; b += LANES) {      // (all lanes go round together; ONE: once)
            const Blocks now = next;
            const bool again = !ONE && b - sub + LANES < blocks;
            next = bring(again ? first : first + stride, again ? b + LANES : sub);
            if constexpr (!ONE)
#pragma unroll
                for (int i = 0; i < M; ++i)
#pragma unroll
                    for (int j = 0; j < 32; j += 4) {
                        const floatx4 v = b < blocks ? *reinterpret_cast<const floatx4 *>(held + (i * blocks + b) * MX4_PITCH + j) : floatx4{0.f, 0.f, 0.f, 0.f};
                        a[i][j] = v[0], a[i][j + 1] = v[1], a[i][j + 2] = v[2], a[i][j + 3] = v[3];
                    }
#pragma unroll
            for (int u = 0; u < RUN; ++u) mx4_block<M>(now.codes[u], scale_of(now.scale[u]), a, acc[u]);
        }
#pragma unroll
        for (int u = 0; u < RUN; ++u) {
            const int64_t row = first + u * PER + lane / LANES;
#pragma unroll
            for (int i = 0; i < M; ++i) {
                const float v = lanes_sum<LANES>(acc[u][i]);
                if (sub == 0 && row < g.n && i < g.m) put4(g.out, i * g.ldo + row, floatx4{v, 0.f, 0.f, 0.f}, 1, g.type);
            }
        }
    }
}

}  // namespace ivf
