// The tile product of tile.hpp for 16-bit operands that need no change on their way (16-bit elements, or terms made earlier) and whose rows
// are whole 16-byte words: they are copied from memory straight into LDS, a step ahead of the products, without registers.
#pragma once
#include "tile.hpp"

namespace ivf {

typedef const __attribute__((address_space(1))) uint32_t *direct_gptr_t;
typedef __attribute__((address_space(3))) uint32_t *direct_lptr_t;
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) shortx4 *direct_trptr_t;

// where copies of what does not exist come from
__device__ __attribute__((aligned(16))) const uint32_t direct_zeros[4] = {0, 0, 0, 0};

// s_waitcnt immediate: at most n vector-memory operations of the wavefront are on their way
constexpr int direct_vmcnt(int n) { return (n & 15) | ((n >> 4) << 14) | 0x0F70; }

// An operand's element (r, k): at r * ld + k, or (COLS) k * ld + r.  ld, and rows (COLS) or K, are multiples of 8.  Several terms stand next to each
// other for every BK of k, so that a step's terms of a row are one run of memory (a 128-byte line for two terms of 32 elements: with a matrix for
// each term the halves of lines that a step needs cost as many requests as lines): term t of (r, k) at r * ld + (k / BK TERMS + t) BK + k % BK.
struct DirectSource {
    const uint16_t *p;
    int64_t ld;
    int rows;
};

// LDS image of a step: rows of BK TERMS elements as in tile.hpp (piece_at); COLS: [BK][ROWS], the 32-byte pairs of pieces of row k exchanged by k mod 4, so that
// the four rows of k that a transposing read takes in one access lie in different banks.
template <bool COLS, int ROWS, int BK, int NT, int TERMS>
struct DirectLoader {
    static_assert(!COLS || TERMS == 1, "columns are read as one term");
    static constexpr int LINE = COLS ? ROWS : BK * TERMS;
    static constexpr int CH = LINE / 8;                        // pieces of a line
    static constexpr int PIECES = TERMS * ROWS * BK / 8;
    static constexpr int ITEMS = PIECES / NT;
    static_assert(PIECES % NT == 0, "whole copies");
    static constexpr int LDS_HALVES = PIECES * 8;

    uint32_t at[ITEMS];                                        // bytes from the source's first element
    int wave;

    __device__ __forceinline__ void init(const DirectSource &s)
    {
        wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / WAVE));
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int id = i * NT + (int)threadIdx.x, line = id / CH, place = id % CH;
            if constexpr (COLS) {
                const int r = (place ^ ((line & 3) << 2)) * 8;
                at[i] = (uint32_t)(line * s.ld + (r < s.rows ? r : 0)) * 2u;   // (columns that do not exist are never stored)
            } else {
                const int piece = place ^ ((line / (16 / CH)) & (CH - 1));
                at[i] = (uint32_t)((line < s.rows ? line : 0) * s.ld + piece * 8) * 2u;
            }
        }
    }

    __device__ __forceinline__ void copy(const DirectSource &s, int64_t k0, int64_t K, uint16_t *lds) const
    {
        const uint8_t *base = reinterpret_cast<const uint8_t *>(s.p + (COLS ? k0 * s.ld : k0 * TERMS));
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const uint8_t *from = base + at[i];
            if (k0 + BK > K) {                                 // the last step may be short
                const int id = i * NT + (int)threadIdx.x, line = id / CH, place = id % CH;
                const int64_t k = COLS ? line : (place ^ ((line / (16 / CH)) & (CH - 1))) * 8 % BK;
                if (k0 + k >= K) from = reinterpret_cast<const uint8_t *>(direct_zeros);
            }
            __builtin_amdgcn_global_load_lds((direct_gptr_t)from, (direct_lptr_t)(lds + (i * NT + wave * WAVE) * 8), 16, 0, 0);
        }
    }

    // copy number i of a step, by itself and without a branch
    __device__ __forceinline__ void copy_one(const DirectSource &s, int i, int64_t k0, int64_t K, uint16_t *lds) const
    {
        const int id = i * NT + (int)threadIdx.x, line = id / CH, place = id % CH;
        const int k = COLS ? line : (place ^ ((line / (16 / CH)) & (CH - 1))) * 8 % BK;
        const uint8_t *from = reinterpret_cast<const uint8_t *>(s.p + (COLS ? k0 * s.ld : k0 * TERMS)) + at[i];
        from = k < K - k0 ? from : reinterpret_cast<const uint8_t *>(direct_zeros);
        __builtin_amdgcn_global_load_lds((direct_gptr_t)from, (direct_lptr_t)(lds + (i * NT + wave * WAVE) * 8), 16, 0, 0);
    }

    // the fragment of 32 rows from `row` on and the 16 elements of sub-step ks: 8 of lane % 32's row
    static __device__ __forceinline__ wordx4 fragment(const uint16_t *lds, int term, int row, int ks)
    {
        const int lane = threadIdx.x & (WAVE - 1);
        if constexpr (COLS) {
            // sixteen lanes read 4 k x 16 rows and get 4 k of a row each
            const int k = 16 * ks + 8 * (lane / 32) + (lane & 15) / 4, r = row + (lane & 16) + 4 * (lane & 3);
            wordx4 v;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int kk = k + 4 * h;                      // (kk & 3 == k & 3)
                const uint16_t *p = lds + kk * ROWS + (((r / 8) ^ ((kk & 3) << 2)) * 8) + (r & 7);
                const wordx2 t = __builtin_bit_cast(wordx2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((direct_trptr_t)p));
                v[2 * h] = t[0];
                v[2 * h + 1] = t[1];
            }
            return v;
        } else {
            return *reinterpret_cast<const wordx4 *>(lds + piece_at<LINE>(row + (lane & 31), term * (BK / 8) + 2 * ks + lane / 32));
        }
    }
};

template <bool COLS_A, int TERMS_A, int BA, int WA, bool COLS_B, int TERMS_B, int BB, int WB, int BK, int BUFS, bool HALF>
struct DirectTile {
    static constexpr int NT = WAVE * WA * WB;
    static constexpr int FA = BA / WA / 32, FB = BB / WB / 32;
    static constexpr int MOST = TERMS_A > TERMS_B ? TERMS_A : TERMS_B;
    static_assert(BK % 32 == 0, "the fragments change places an even number of times a step");
    using LA = DirectLoader<COLS_A, BA, BK, NT, TERMS_A>;
    using LB = DirectLoader<COLS_B, BB, BK, NT, TERMS_B>;
    static constexpr int STEP = LA::LDS_HALVES + LB::LDS_HALVES;
    static constexpr int OUT_HALVES = NT / WAVE * 32 * (32 * FA) * 2;   // what store() needs
    static constexpr int LDS_HALVES = BUFS * STEP > OUT_HALVES ? BUFS * STEP : OUT_HALVES;
    static constexpr int COPIES = LA::ITEMS + LB::ITEMS;       // of a wavefront and step

    floatx16 acc[FA][FB];

    static __device__ __forceinline__ int row_a(int f) { return (int)(threadIdx.x / WAVE) / WB * (FA * 32) + f * 32; }
    static __device__ __forceinline__ int row_b(int f) { return (int)(threadIdx.x / WAVE) % WB * (FB * 32) + f * 32; }

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < FA; ++i)
#pragma unroll
            for (int j = 0; j < FB; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    }

    struct Fragments {
        wordx4 a[TERMS_A][FA], b[TERMS_B][FB];
    };

    static __device__ __forceinline__ void fetch(Fragments &f, const uint16_t *la, const uint16_t *lb, int ks)
    {
#pragma unroll
        for (int t = 0; t < TERMS_B; ++t)
#pragma unroll
            for (int j = 0; j < FB; ++j) f.b[t][j] = LB::fragment(lb, t, row_b(j), ks);
#pragma unroll
        for (int t = 0; t < TERMS_A; ++t)
#pragma unroll
            for (int i = 0; i < FA; ++i) f.a[t][i] = LA::fragment(la, t, row_a(i), ks);
    }

    __device__ __forceinline__ void multiply(const Fragments &f)
    {
#pragma unroll
        for (int order = MOST - 1; order >= 0; --order)       // the small products first
#pragma unroll
            for (int t = 0; t < TERMS_A; ++t) {
                if (order - t < 0 || order - t >= TERMS_B) continue;
#pragma unroll
                for (int i = 0; i < FA; ++i)
#pragma unroll
                    for (int j = 0; j < FB; ++j) {
                        const wordx4 u = f.a[t][i], v = f.b[order - t][j];
                        if constexpr (HALF)
                            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(halfx8, u), __builtin_bit_cast(halfx8, v), acc[i][j], 0, 0, 0);
                        else
                            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, u), __builtin_bit_cast(bf16x8, v), acc[i][j], 0, 0, 0);
                    }
            }
    }

    // Interleaves the products of the present fragments with the reads of the next ones and, behind those, VMEM copies.  A product first: what it waits for was
    // read a sub-step ago, what is read behind it need not be waited for.  (Priorities set around the products end the compiler's regions, and all reads come
    // before all products again: transposed products of 16 384 rows 442 us, so 405.)
    template <int VMEM, int MORE = 0>
    static __device__ __forceinline__ void mix()
    {
        constexpr int READS = (COLS_A ? 2 : 1) * TERMS_A * FA + (COLS_B ? 2 : 1) * TERMS_B * FB + MORE;
        constexpr int PRODUCTS = FA * FB * (MOST == 3 ? TERMS_A == TERMS_B ? 6 : 3 : MOST == 2 ? TERMS_A == TERMS_B ? 3 : 2 : 1);
        constexpr int OTHERS = READS + VMEM, EACH = (OTHERS + PRODUCTS - 1) / PRODUCTS;
#pragma unroll
        for (int r = 0; r < PRODUCTS; ++r) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
#pragma unroll
            for (int e = 0; e < EACH; ++e) {
                const int o = r * EACH + e;
                if (o < READS) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                else if (o < OTHERS) __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    }

    // acc += a b^T over k in [0, K): a ring of BUFS buffers, BUFS - 1 steps' copies on their way (past K zeros, so that their number is always
    // the same).  One barrier a step, before the products of its last sub-step: everyone has the fragments for those by then, so that the
    // step's buffer is free for the next copies, and everyone's copies of the next step have landed, whose first fragments come while they run.
    // (Columns: the compiler waits for all copies before a step's first transposing read, as if that depended on them, so they are drained one to three products after they were issued.)
    __device__ __forceinline__ void product(const DirectSource &sa, const DirectSource &sb, int64_t K, uint16_t *lds)
    {
        if (K <= 0) return;
        constexpr int SUBS = BK / 16;
        LA la;
        LB lb;
        la.init(sa);
        lb.init(sb);
#pragma unroll
        for (int s = 0; s < BUFS; ++s) {
            la.copy(sa, s * BK, K, lds + s * STEP);
            lb.copy(sb, s * BK, K, lds + s * STEP + LA::LDS_HALVES);
        }
        __builtin_amdgcn_s_waitcnt(direct_vmcnt((BUFS - 1) * COPIES));
        asm volatile("s_barrier" ::: "memory");
        Fragments f[2];
        fetch(f[0], lds, lds + LA::LDS_HALVES, 0);
        int at = 0;
        for (int64_t k = 0; k < K; k += BK) {
            uint16_t *buf = lds + at * STEP;
#pragma unroll
            for (int ks = 0; ks + 1 < SUBS; ++ks) {
                fetch(f[(ks + 1) & 1], buf, buf + LA::LDS_HALVES, ks + 1);
                multiply(f[ks & 1]);
                mix<0>();
            }
            __builtin_amdgcn_s_waitcnt(direct_vmcnt((BUFS - 2) * COPIES));
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            at = at + 1 == BUFS ? 0 : at + 1;
            const uint16_t *next = lds + at * STEP;
            fetch(f[SUBS & 1], next, next + LA::LDS_HALVES, 0);                     // (behind the last step: not used)
#pragma unroll
            for (int i = 0; i < LA::ITEMS; ++i) la.copy_one(sa, i, k + BUFS * BK, K, buf);
#pragma unroll
            for (int i = 0; i < LB::ITEMS; ++i) lb.copy_one(sb, i, k + BUFS * BK, K, buf + LA::LDS_HALVES);
            multiply(f[(SUBS - 1) & 1]);
            mix<COPIES>();
        }
        __builtin_amdgcn_s_waitcnt(direct_vmcnt(0));          // no copy into LDS may outlive the workgroup, or come behind what is written there next
        __syncthreads();
    }

    __device__ __forceinline__ void store(void *out, int64_t ld, int rows, int cols, Type type, uint16_t *lds) const { store_tile<FA>(*this, out, ld, rows, cols, type, lds); }

    // f(row of a, row of b, four values of rows of a in a run), as Tile::each
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

// The tile for large products of rows: 256 x 256 by four wavefronts of 128 x 128, whose fragments are read from LDS half as often for a product as those of 64 x 64,
// and steps of 64 of k, so that copies are of whole 128-byte lines.  LDS is five slots, each an operand's 256 rows of a step: both of the present step, both of
// the next, and a's of the one after.  a's copies come between the products of a step's first half, b's behind the barrier of its last sub-step, where the present
// slots become free, so that copies have three sub-steps at least and the matrix units wait for neither reads nor copies.
template <bool HALF>
struct WideTile : DirectTile<false, 1, 256, 2, false, 1, 256, 2, 64, 2, HALF> {
    using Base = DirectTile<false, 1, 256, 2, false, 1, 256, 2, 64, 2, HALF>;
    using LA = typename Base::LA;
    using LB = typename Base::LB;
    using Fragments = typename Base::Fragments;
    static constexpr int SLOT = LA::LDS_HALVES, SLOTS = 5, BK = 64, SUBS = 4, ITEMS = LA::ITEMS;
    static_assert(LA::LDS_HALVES == LB::LDS_HALVES && LA::ITEMS == LB::ITEMS, "slots are alike");
    static constexpr int LDS_HALVES = SLOTS * SLOT;
    static_assert(LDS_HALVES >= Base::OUT_HALVES, "store() has room");

    // as DirectTile::product
    __device__ __forceinline__ void product(const DirectSource &sa, const DirectSource &sb, int64_t K, uint16_t *lds)
    {
        if (K <= 0) return;
        LA la;
        LB lb;
        la.init(sa);
        lb.init(sb);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) la.copy_one(sa, i, 0, K, lds);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) lb.copy_one(sb, i, 0, K, lds + SLOT);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) la.copy_one(sa, i, BK, K, lds + 2 * SLOT);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) lb.copy_one(sb, i, BK, K, lds + 3 * SLOT);
        __builtin_amdgcn_s_waitcnt(direct_vmcnt(2 * ITEMS));
        asm volatile("s_barrier" ::: "memory");
        Fragments f[2];
        Base::fetch(f[0], lds, lds + SLOT, 0);
        int a = 0;                                             // the slot of a; b's follows
        for (int64_t k = 0; k < K; k += BK) {
            const int b = a + 1 == SLOTS ? 0 : a + 1, na = b + 1 == SLOTS ? 0 : b + 1, nb = na + 1 == SLOTS ? 0 : na + 1, slot = nb + 1 == SLOTS ? 0 : nb + 1;
            const uint16_t *pa = lds + a * SLOT, *pb = lds + b * SLOT;
#pragma unroll
            for (int ks = 0; ks + 1 < SUBS; ++ks) {
                Base::fetch(f[(ks + 1) & 1], pa, pb, ks + 1);
                if (ks < 2) {
#pragma unroll
                    for (int i = ks * ITEMS / 2; i < (ks + 1) * ITEMS / 2; ++i) la.copy_one(sa, i, k + 2 * BK, K, lds + slot * SLOT);
                }
                Base::multiply(f[ks & 1]);
                if (ks < 2) Base::template mix<ITEMS / 2>();
                else Base::template mix<0>();
            }
            // this step's fragments are all read; the next step's operands have landed (a's of the one behind may be under way)
            __builtin_amdgcn_s_waitcnt(direct_vmcnt(ITEMS));
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            Base::fetch(f[SUBS & 1], lds + na * SLOT, lds + nb * SLOT, 0);
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) lb.copy_one(sb, i, k + 2 * BK, K, lds + a * SLOT);
            Base::multiply(f[(SUBS - 1) & 1]);
            Base::template mix<ITEMS>();
            a = na;
        }
        __builtin_amdgcn_s_waitcnt(direct_vmcnt(0));
        __syncthreads();
    }
};

// Tile `place` of a grid of down x across, in bands of BAND rows and column by column in a band, so that a run of places is a block of tiles.
constexpr int BAND = 8;
__device__ __forceinline__ void tile_of_place(uint32_t place, int down, int across, int &i, int &j)
{
    const uint32_t size = BAND * (uint32_t)across;
    const int band = (int)(place / size), left = (int)(place % size);
    const int height = down - band * BAND < BAND ? down - band * BAND : BAND;
    i = band * BAND + left % height;
    j = left / height;
}

// The same for the tiles on and below the diagonal of side x side.
__device__ __forceinline__ void triangle_of_place(int place, int side, int &i, int &j)
{
    int first = 0;                                             // row of the band
    while (first + BAND < side && place >= (first + BAND) * (first + BAND + 1) / 2) first += BAND;
    int left = place - first * (first + 1) / 2;
    const int height = side - first < BAND ? side - first : BAND;
    if (left < first * height) {
        i = first + left % height;
        j = left / height;
    } else {
        left -= first * height;
        i = 0;
        while (left > i) left -= ++i;                          // row i of the triangle has i + 1 tiles
        i += first;
        j = first + left;
    }
}

}  // namespace ivf
