// Products of rows with a matrix of their group (a region's rotation, an expert's weights), and the gradient of those matrices.
// Rows stand group by group; how many each group has is known on the device only.
#pragma once
#include "direct.hpp"

namespace ivf {

// Rows offsets[g] .. offsets[g + 1] are group g's, in pieces of T rows.  Piece numbers are handed out without a prefix sum over the
// groups: group g's begin at offsets[g] / T + g, which leaves room for all of them because (b - a) rows have at most
// floor(b / T) - floor(a / T) + 1 pieces.  So n / T + G + 1 numbers are enough (the last group, number G, holds the rows behind offsets[G]), any one of
// them is found from the offsets alone, and at most one number a group has no rows.  Offsets are read as if offsets[0] were 0, and are cut to n.
struct Piece {
    int group;                 // G: rows that belong to no group
    int row;                   // first row
    int rows;                  // 0: nothing to do
    int index;                 // of the group's pieces
    int begin, group_rows;
};

__device__ __forceinline__ uint32_t group_begin(const uint32_t *offsets, int G, uint32_t n, int g)
{
    if (g == 0) return 0;
    if (g > G) return n;
    const uint32_t o = offsets[g];
    return o < n ? o : n;
}

// The piece of that number, of 2^shift rows, by all lanes of a wavefront: 64 groups are looked at in a step.
__device__ __forceinline__ Piece find_piece(const uint32_t *offsets, int G, uint32_t n, int shift, uint32_t number)
{
    const int lane = threadIdx.x & (WAVE - 1);
    int lo = 0, hi = G + 1;                                   // the group lies in [lo, hi)
    uint32_t a, b;
    while (true) {
        const int step = (hi - lo + WAVE - 1) / WAVE, g = lo + lane * step;
        const uint32_t begin = group_begin(offsets, G, n, g < hi ? g : hi);
        const bool before = g < hi && (g == lo || (begin >> shift) + g <= number);
        const int count = __popcll(__ballot(before));         // a run from lane 0 on, which always counts
        lo += (count - 1) * step;
        if (step == 1) {                                      // the lanes hold where the groups begin
            a = __builtin_amdgcn_readlane(begin, count - 1);
            b = count < WAVE ? __builtin_amdgcn_readlane(begin, count & (WAVE - 1)) : group_begin(offsets, G, n, lo + 1);
            break;
        }
        hi = lo + step < hi ? lo + step : hi;
    }
    Piece p;
    p.group = __builtin_amdgcn_readfirstlane(lo);
    p.begin = __builtin_amdgcn_readfirstlane((int)a);
    p.group_rows = __builtin_amdgcn_readfirstlane((int)(b - a));   // (below 0 where offsets do not ascend)
    p.index = (int)(number - ((uint32_t)p.begin >> shift) - (uint32_t)p.group);
    const int64_t row = p.begin + ((int64_t)p.index << shift), left = p.index < 0 ? 0 : (int64_t)p.begin + p.group_rows - row;
    p.row = (int)row;
    p.rows = left <= 0 ? 0 : left < 1 << shift ? (int)left : 1 << shift;
    return p;
}

constexpr int log2_of(int v) { return v <= 1 ? 0 : 1 + log2_of(v / 2); }

template <Type T>
struct Elem;
template <>
struct Elem<Type::F32> {
    static constexpr Form rows = Form::F_ROWS, cols = Form::F_COLS;
    static constexpr int terms = 3, bytes = 4, step = 32, bufs = 1;
    static constexpr bool half = false;
};
template <>
struct Elem<Type::F16> {
    static constexpr Form rows = Form::H_ROWS, cols = Form::H_COLS;
    static constexpr int terms = 1, bytes = 2, step = 64, bufs = 2;
    static constexpr bool half = true;
};
template <>
struct Elem<Type::BF16> {
    static constexpr Form rows = Form::H_ROWS, cols = Form::H_COLS;
    static constexpr int terms = 1, bytes = 2, step = 64, bufs = 2;
    static constexpr bool half = false;
};

struct GroupedArgs {
    const uint8_t *x;
    int64_t ldx;
    const uint8_t *w;
    int n, G, R, C;
    const uint32_t *offsets;
    void *y;
    int64_t ldy;
    Type out;
    uint32_t first;            // workgroup of the list that this launch begins with
};

// Bound by latency where groups are short (a piece's rows and matrix are a few loads): several workgroups a compute unit.  500 000 rows of 96
// fp32 components in 4096 groups: 143 us, 3.7 TB/s.
// One workgroup: BX rows of a group by BW columns of the result, W's rows (or columns) as the first operand so that a lane holds four
// neighbouring columns of a row.
template <Type T, bool TRANSPOSED, int BX, int BW, bool APART>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(APART && BX == 128 ? 2 : 3))) void grouped_product_kernel(GroupedArgs g)
{
    using E = Elem<T>;
    constexpr int WB = BX >= 64 ? 2 : 1;
    using P = Tile<TRANSPOSED ? E::cols : E::rows, E::terms, BW, 4 / WB, E::rows, E::terms, BX, WB, E::step, E::bufs, E::half, APART>;
    __shared__ __attribute__((aligned(16))) uint16_t lds[P::LDS_HALVES];
    const int cols = TRANSPOSED ? g.C : g.R, K = TRANSPOSED ? g.R : g.C;
    const int tiles = (cols + BW - 1) / BW;
    const uint32_t place = g.first + place_of_block(blockIdx.x, gridDim.x);
    const Piece p = find_piece(g.offsets, g.G, g.n, log2_of(BX), place / tiles);
    if (p.rows == 0) return;
    const int c0 = (int)(place % tiles) * BW;
    P t;
    t.clear();
    if (p.group < g.G) {
        Source sw{g.w + ((int64_t)p.group * g.R * g.C + (TRANSPOSED ? (int64_t)c0 : (int64_t)c0 * g.C)) * E::bytes, nullptr, g.C, cols - c0 < BW ? cols - c0 : BW};
        Source sx{g.x + p.row * g.ldx * E::bytes, nullptr, g.ldx, p.rows};
        t.product(sw, sx, 0, K, lds);
    }
    const bool bad = T == Type::F32 && any_nan(t);
    t.store(static_cast<uint8_t *>(g.y) + (p.row * g.ldy + c0) * (g.out == Type::F32 ? 4 : 2), g.ldy, p.rows, cols - c0, g.out, lds);
    if (bad && p.group < g.G) {
        const float *x = reinterpret_cast<const float *>(g.x) + p.row * g.ldx, *w = reinterpret_cast<const float *>(g.w) + (int64_t)p.group * g.R * g.C;
        mend(static_cast<float *>(g.y) + p.row * g.ldy + c0, g.ldy, p.rows, cols - c0 < BW ? cols - c0 : BW, K, [&](int row, int64_t k) { return x[row * g.ldx + k]; },
             [&](int col, int64_t k) { return TRANSPOSED ? w[k * g.C + c0 + col] : w[(int64_t)(c0 + col) * g.C + k]; });
    }
}

// The same for 16-bit rows and matrices whose lines are whole 16-byte words: 8192 rows, 32 matrices of 2048 x 2048 in bfloat16 128 us, 540 TFLOP/s with groups of
// unequal size.  Transposed (8192 rows, 16 of 2048 x 1024: 62 us) the units are busy for 62 % of the time and the matrix units for 39 % of that: the step's copies are waited for before the
// first columns are read.  The workgroups that an XCD runs at a time share rows of x and of W
// (tile_of_place).
template <bool HALF, bool TRANSPOSED, int BX, int BW, int WX, int WW, int BK, int BUFS>
__global__ __launch_bounds__(WAVE *WX *WW) void grouped_product_direct_kernel(GroupedArgs g, int pieces)
{
    using P = DirectTile<TRANSPOSED, 1, BW, WW, false, 1, BX, WX, BK, BUFS, HALF>;
    __shared__ __attribute__((aligned(16))) uint16_t lds[P::LDS_HALVES];
    const int cols = TRANSPOSED ? g.C : g.R, K = TRANSPOSED ? g.R : g.C;
    const int tiles = (cols + BW - 1) / BW;
    const uint32_t place = g.first + place_of_block(blockIdx.x, gridDim.x);
    int piece, tile;
    tile_of_place(place, pieces, tiles, piece, tile);
    const Piece p = find_piece(g.offsets, g.G, g.n, log2_of(BX), piece);
    if (p.rows == 0) return;
    const int c0 = tile * BW;
    P t;
    t.clear();
    if (p.group < g.G) {
        const uint16_t *w = reinterpret_cast<const uint16_t *>(g.w) + (int64_t)p.group * g.R * g.C + (TRANSPOSED ? (int64_t)c0 : (int64_t)c0 * g.C);
        t.product(DirectSource{w, g.C, cols - c0}, DirectSource{reinterpret_cast<const uint16_t *>(g.x) + p.row * g.ldx, g.ldx, p.rows}, K, lds);
    }
    t.store(static_cast<uint8_t *>(g.y) + (p.row * g.ldy + c0) * (g.out == Type::F32 ? 4 : 2), g.ldy, p.rows, cols - c0, g.out, lds);
}

// The same for large groups by tiles of 256 x 256, not transposed: 16 384 rows, 8 matrices of 4096 x 2048 in bfloat16 285 us, 963 TFLOP/s (338 by tiles of
// 128 x 256), 32 matrices 365 - 380 us.  Bound by a workgroup's first loads and its stores, during which its compute unit has nothing else, and by a last round of tiles for
// part of the units: those are busy for 63 % of the time, the matrix units for 61 % of that.
template <bool HALF>
__global__ __launch_bounds__(256) void grouped_product_wide_kernel(GroupedArgs g, int pieces)
{
    using P = WideTile<HALF>;
    constexpr int BX = 256, BW = 256;
    __shared__ __attribute__((aligned(16))) uint16_t lds[P::LDS_HALVES];
    const int tiles = (g.R + BW - 1) / BW;
    const uint32_t place = g.first + place_of_block(blockIdx.x, gridDim.x);
    int piece, tile;
    tile_of_place(place, pieces, tiles, piece, tile);
    const Piece p = find_piece(g.offsets, g.G, g.n, log2_of(BX), piece);
    if (p.rows == 0) return;
    const int c0 = tile * BW;
    P t;
    t.clear();
    if (p.group < g.G) {
        const uint16_t *w = reinterpret_cast<const uint16_t *>(g.w) + (int64_t)p.group * g.R * g.C + (int64_t)c0 * g.C;
        t.product(DirectSource{w, g.C, g.R - c0}, DirectSource{reinterpret_cast<const uint16_t *>(g.x) + p.row * g.ldx, g.ldx, p.rows}, g.C, lds);
    }
    t.store(static_cast<uint8_t *>(g.y) + (p.row * g.ldy + c0) * (g.out == Type::F32 ? 4 : 2), g.ldy, p.rows, g.R - c0, g.out, lds);
}

// Groups of a few rows (serving: a token or two for an expert): the matrices are read once and are the traffic, so each wavefront reads lines of
// them whole, keeps many on their way and multiplies in fp32 by up to FEW_ROWS rows; no matrix instruction would be a quarter full.  16 rows, 16 matrices of 2048 x 1024 in bfloat16: 16 us, 2.6 TB/s of the matrices with rows;
// with tiles of 32 rows 34 us.
constexpr int FEW_ROWS = 4;
constexpr int FEW_LINES = 4;                                  // lines of W of a wavefront
template <Type T>
__global__ __launch_bounds__(256) void grouped_few_kernel(GroupedArgs g)
{
    const int lane = threadIdx.x & 63, tiles = (g.R + 4 * FEW_LINES - 1) / (4 * FEW_LINES);
    const uint32_t place = g.first + place_of_block(blockIdx.x, gridDim.x);
    const Piece p = find_piece(g.offsets, g.G, g.n, log2_of(FEW_ROWS), place / tiles);
    const int r0 = (int)(place % tiles) * (4 * FEW_LINES) + __builtin_amdgcn_readfirstlane((int)(threadIdx.x / WAVE)) * FEW_LINES;
    if (p.rows == 0 || r0 >= g.R) return;
    const int lines = g.R - r0 < FEW_LINES ? g.R - r0 : FEW_LINES;
    float acc[FEW_LINES][FEW_ROWS];
#pragma unroll
    for (int w = 0; w < FEW_LINES; ++w)
#pragma unroll
        for (int i = 0; i < FEW_ROWS; ++i) acc[w][i] = 0.f;
    if (p.group < g.G) {
        const int64_t first = ((int64_t)p.group * g.R + r0) * g.C;
#pragma unroll 2
        for (int c = 8 * lane; c < g.C; c += 8 * WAVE) {
            float w[FEW_LINES][8], x[FEW_ROWS][8];
            auto bring = [&](const uint8_t *from, int64_t at, float (&v)[8]) {
                if (c + 8 <= g.C) {
                    eight<T>(from, at + c, v);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = c + j < g.C ? element<T>(from, at + c + j) : 0.f;
                }
            };
#pragma unroll
            for (int l = 0; l < FEW_LINES; ++l) bring(g.w, first + (int64_t)(l < lines ? l : 0) * g.C, w[l]);
#pragma unroll
            for (int i = 0; i < FEW_ROWS; ++i)
                if (i < p.rows) bring(g.x, (p.row + i) * g.ldx, x[i]);
#pragma unroll
            for (int i = 0; i < FEW_ROWS; ++i)
                if (i < p.rows)
#pragma unroll
                    for (int l = 0; l < FEW_LINES; ++l)
#pragma unroll
                        for (int j = 0; j < 8; ++j) acc[l][i] = fmaf(w[l][j], x[i][j], acc[l][i]);
        }
    }
#pragma unroll
    for (int i = 0; i < FEW_ROWS; ++i) {
        if (i >= p.rows) break;
        float v = 0.f;                                        // lane l: line l's
#pragma unroll
        for (int l = 0; l < FEW_LINES; ++l) {
            const float sum = wave_total(acc[l][i]);
            v = lane == l ? sum : v;
        }
        if (lane < lines) put4(g.y, (p.row + i) * g.ldy + r0 + lane, floatx4{v, 0.f, 0.f, 0.f}, 1, g.out);
    }
}

// The same for W^T: 64 columns a workgroup, eight of them a lane; eight lines of W a wavefront and step, whose sums are added at the end.
template <Type T>
__global__ __launch_bounds__(256) void grouped_few_transposed_kernel(GroupedArgs g)
{
    __shared__ float sums[4][FEW_ROWS][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x / WAVE, tiles = (g.C + 63) / 64;
    const uint32_t place = g.first + place_of_block(blockIdx.x, gridDim.x);
    const Piece p = find_piece(g.offsets, g.G, g.n, log2_of(FEW_ROWS), place / tiles);
    if (p.rows == 0) return;
    const int c0 = (int)(place % tiles) * 64, c = c0 + 8 * (lane & 7);
    float acc[FEW_ROWS][8];
#pragma unroll
    for (int i = 0; i < FEW_ROWS; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[i][j] = 0.f;
    if (p.group < g.G && c < g.C) {
        const int64_t first = (int64_t)p.group * g.R * g.C + c;
#pragma unroll 4
        for (int r = wave * 8 + lane / 8; r < g.R; r += 32) {
            float w[8];
            const int64_t at = first + (int64_t)r * g.C;
            if (c + 8 <= g.C) {
                eight<T>(g.w, at, w);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j] = c + j < g.C ? element<T>(g.w, at + j) : 0.f;
            }
#pragma unroll
            for (int i = 0; i < FEW_ROWS; ++i)
                if (i < p.rows) {
                    const float x = element<T>(g.x, (p.row + i) * g.ldx + r);
#pragma unroll
                    for (int j = 0; j < 8; ++j) acc[i][j] = fmaf(w[j], x, acc[i][j]);
                }
        }
    }
#pragma unroll
    for (int i = 0; i < FEW_ROWS; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
#pragma unroll
            for (int o = 8; o < WAVE; o <<= 1) acc[i][j] += __shfl_xor(acc[i][j], o, WAVE);
            if (lane < 8) sums[wave][i][8 * lane + j] = acc[i][j];
        }
    __syncthreads();
    const int i = threadIdx.x / 64, col = threadIdx.x & 63;
    static_assert(FEW_ROWS == 4, "a thread an element");
    if (i < p.rows && c0 + col < g.C)
        put4(g.y, (p.row + i) * g.ldy + c0 + col, floatx4{(sums[0][i][col] + sums[1][i][col]) + (sums[2][i][col] + sums[3][i][col]), 0.f, 0.f, 0.f}, 1, g.out);
}

struct GradientArgs {
    const uint8_t *dy;
    int64_t lddy;
    const uint8_t *x;
    int64_t ldx;
    int n, G, R, C;
    const uint32_t *offsets;
    void *dw;
    Type out;
    int shift;                 // rows of a piece are 2^shift: the sum of a longer group is taken in pieces
    float *parts;              // their sums
    uint32_t first;            // as in GroupedArgs
};

// Where the sums of a group's pieces are kept: groups with more than one piece have more than T rows, and from
// 2 floor(a / T) on there is room for all of them before the next such group's.
__device__ __forceinline__ int64_t part_of(int begin, int shift) { return 2 * (int64_t)(begin >> shift); }

// Piece and tile of a workgroup.  Pieces differ in rows, so every XCD takes an eighth of each piece's tiles where there are eight (16 experts of
// 8192 rows together: 114 us where it took an eighth of the pieces, 77 so); single tiles go by pieces.
__host__ __device__ __forceinline__ uint32_t gradient_tiles(uint32_t tiles) { return tiles < 8 ? tiles : (tiles + 7) / 8 * 8; }

__device__ __forceinline__ void gradient_place(uint32_t first, uint32_t tiles, uint32_t &piece, uint32_t &tile)
{
    if (tiles < 8) {
        const uint32_t place = first + place_of_block(blockIdx.x, gridDim.x);
        piece = place / tiles;
        tile = place % tiles;
    } else {
        const uint32_t slice = (tiles + 7) / 8, local = (first + blockIdx.x) / 8;   // (first: a multiple of 8)
        piece = local / slice;
        tile = blockIdx.x % 8 * slice + local % slice;         // (past the last: nothing to do)
    }
}

__device__ __forceinline__ float *gradient_part(const GradientArgs &g, const Piece &p) { return g.parts + (part_of(p.begin, g.shift) + p.index) * ((int64_t)g.R * g.C); }

template <class P>
__device__ __forceinline__ void store_gradient(const P &t, const GradientArgs &g, const Piece &p, int r0, int c0, uint16_t *lds)
{
    const int64_t at = (int64_t)r0 * g.C + c0, size = (int64_t)g.R * g.C;
    if (p.group_rows <= 1 << g.shift)
        t.store(static_cast<uint8_t *>(g.dw) + (p.group * size + at) * (g.out == Type::F32 ? 4 : 2), g.C, g.R - r0, g.C - c0, g.out, lds);
    else
        t.store(gradient_part(g, p) + at, g.C, g.R - r0, g.C - c0, Type::F32, lds);
}

// Both operands by columns.  500 000 rows of 96 fp32 components in 4096 groups: 205 us in long runs (245 from cold clocks), bound by the latency of a short group's steps: the
// matrix units are busy for 16 % of the units' time.  Sums apart cost a third wavefront a SIMD (170 us with one sum for all products; 200 to 215 with a sum for each 16 rows that is added by
// itself, 455 by eight wavefronts of half the tile).
template <Type T, int BR, int BC>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void grouped_gradient_kernel(GradientArgs g)
{
    using E = Elem<T>;
    using P = Tile<E::cols, E::terms, BC, 2, E::cols, E::terms, BR, 2, E::step, E::bufs, E::half, T == Type::F32>;
    __shared__ __attribute__((aligned(16))) uint16_t lds[P::LDS_HALVES];
    const int across = (g.C + BC - 1) / BC, down = (g.R + BR - 1) / BR;
    uint32_t piece, tile;
    gradient_place(g.first, (uint32_t)across * down, piece, tile);
    if (tile >= (uint32_t)across * down) return;
    const Piece p = find_piece(g.offsets, g.G, g.n, g.shift, piece);
    // (a group without rows still has its zeros written, by the number that it leaves unused)
    if (p.group >= g.G || p.index < 0 || (p.rows == 0 && p.index > 0)) return;
    int i, j;
    tile_of_place(tile, down, across, i, j);
    const int c0 = j * BC, r0 = i * BR;
    P t;
    t.clear();
    Source sx{g.x + (p.row * g.ldx + c0) * E::bytes, nullptr, g.ldx, g.C - c0 < BC ? g.C - c0 : BC};
    Source sd{g.dy + (p.row * g.lddy + r0) * E::bytes, nullptr, g.lddy, g.R - r0 < BR ? g.R - r0 : BR};
    t.product(sx, sd, 0, p.rows, lds);
    const bool bad = T == Type::F32 && any_nan(t);
    store_gradient(t, g, p, r0, c0, lds);
    if (bad) {
        const float *dy = reinterpret_cast<const float *>(g.dy) + p.row * g.lddy + r0, *x = reinterpret_cast<const float *>(g.x) + p.row * g.ldx + c0;
        float *out = p.group_rows <= 1 << g.shift ? static_cast<float *>(g.dw) + p.group * ((int64_t)g.R * g.C) : gradient_part(g, p);
        mend(out + (int64_t)r0 * g.C + c0, g.C, g.R - r0 < BR ? g.R - r0 : BR, g.C - c0 < BC ? g.C - c0 : BC, p.rows,
             [&](int row, int64_t k) { return dy[k * g.lddy + row]; }, [&](int col, int64_t k) { return x[k * g.ldx + col]; });
    }
}

template <bool HALF, int BR, int BC, int WR, int WC>
__global__ __launch_bounds__(WAVE *WR *WC) void grouped_gradient_direct_kernel(GradientArgs g)
{
    using P = DirectTile<true, 1, BC, WC, true, 1, BR, WR, 64, 2, HALF>;
    __shared__ __attribute__((aligned(16))) uint16_t lds[P::LDS_HALVES];
    const int across = (g.C + BC - 1) / BC, down = (g.R + BR - 1) / BR;
    uint32_t piece, tile;
    gradient_place(g.first, (uint32_t)across * down, piece, tile);
    if (tile >= (uint32_t)across * down) return;
    const Piece p = find_piece(g.offsets, g.G, g.n, g.shift, piece);
    // (a group without rows still has its zeros written, by the number that it leaves unused)
    if (p.group >= g.G || p.index < 0 || (p.rows == 0 && p.index > 0)) return;
    int i, j;
    tile_of_place(tile, down, across, i, j);
    const int c0 = j * BC, r0 = i * BR;
    P t;
    t.clear();
    t.product(DirectSource{reinterpret_cast<const uint16_t *>(g.x) + p.row * g.ldx + c0, g.ldx, g.C - c0},
              DirectSource{reinterpret_cast<const uint16_t *>(g.dy) + p.row * g.lddy + r0, g.lddy, g.R - r0}, p.rows, lds);
    store_gradient(t, g, p, r0, c0, lds);
}

// Adds the pieces of the groups that have several, in their order.
__global__ __launch_bounds__(256) void gradient_join_kernel(GradientArgs g)
{
    const int64_t size = (int64_t)g.R * g.C;
    for (int64_t group = blockIdx.y; group < g.G; group += gridDim.y) {
        const int a = (int)group_begin(g.offsets, g.G, g.n, (int)group), rows = (int)group_begin(g.offsets, g.G, g.n, (int)group + 1) - a;
        if (rows <= 1 << g.shift) continue;
        const int pieces = (rows - 1 >> g.shift) + 1;
        const float *part = g.parts + part_of(a, g.shift) * size;
        for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < size; i += (int64_t)gridDim.x * 256) {
            float s = 0.f;
            for (int q = 0; q < pieces; ++q) s += part[q * size + i];
            if (g.out == Type::F32) static_cast<float *>(g.dw)[group * size + i] = s;
            else static_cast<uint16_t *>(g.dw)[group * size + i] = (uint16_t)two_halves(s, s, g.out == Type::BF16);
        }
    }
}

}  // namespace ivf
