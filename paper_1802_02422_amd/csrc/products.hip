// C ABI of the matrix operators (see include/ivf_gp.h): argument checks and launches.  They are asynchronous on the caller's stream and allocate
// nothing: where scratch is needed the caller gives it.  gfx950 only.
#include "../../include/ivf_gp.h"

#include <algorithm>
#include <cmath>
#include <utility>

#include "error.hpp"
#include "grouped.hpp"
#include "mx4.hpp"
#include "ortho.hpp"
#include "ortho_small.hpp"

using namespace ivf;

namespace {

bool type_known(int t) { return t == IVF_F32 || t == IVF_F16 || t == IVF_BF16; }
Type type_of(int t) { return t == IVF_F32 ? Type::F32 : t == IVF_F16 ? Type::F16 : Type::BF16; }
int bytes_of(int t) { return t == IVF_F32 ? 4 : 2; }
bool aligned(const void *p, int64_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

int check_types(int type, int out_type)
{
    if (!type_known(type)) return fail(IVF_EINVAL, "type=%d is none of IVF_F32, IVF_F16, IVF_BF16", type);
    if (out_type != type && out_type != IVF_F32) return fail(IVF_EINVAL, "out_type=%d must be the operands' type or IVF_F32", out_type);
    return IVF_OK;
}

// A launch has less than 2^32 threads.  launch(first, count) for as many of them as `blocks` workgroups take; they number their work from `first` on, a multiple of 8
// (the XCDs).
template <class F>
int in_launches(int64_t blocks, int threads, F launch)
{
    if (blocks >= 1ll << 32) return fail(IVF_EINVAL, "too large (%lld workgroups)", (long long)blocks);
    const int64_t most = ((1ll << 32) - 1) / threads / 8 * 8;
    for (int64_t first = 0; first < blocks; first += most)
        if (int rc = launch((uint32_t)first, dim3((unsigned)std::min(most, blocks - first)))) return rc;
    return IVF_OK;
}

int check_groups(int64_t n, int64_t G, int R, int C)
{
    if (n < 0 || n >= (1ll << 31)) return fail(IVF_EINVAL, "n=%lld out of range", (long long)n);
    if (G < 1 || G >= (1ll << 30)) return fail(IVF_EINVAL, "G=%lld out of range", (long long)G);
    if (R < 1 || C < 1 || R > IVF_MAX_SIDE || C > IVF_MAX_SIDE) return fail(IVF_EINVAL, "R=%d and C=%d must be in [1, %d]", R, C, IVF_MAX_SIDE);
    return IVF_OK;
}

// Lines of whole 16-byte words, near enough to each other that a tile's fit 32 bits of offset: they can be copied straight into LDS
// (x [n][cols] with rows ld apart).
bool direct_rows(const void *p, int64_t ld, int64_t cols, int type) { return type != IVF_F32 && aligned(p, 16) && ld % 8 == 0 && cols % 8 == 0 && ld < (1 << 22); }

// fn<Type>() for the ABI's type
template <class F>
int by_type(int type, F fn)
{
    if (type == IVF_F32) return fn(std::integral_constant<Type, Type::F32>{});
    if (type == IVF_F16) return fn(std::integral_constant<Type, Type::F16>{});
    return fn(std::integral_constant<Type, Type::BF16>{});
}

// Rows of a group whose sum of products is one workgroup's (ivf_grouped_gradient), 2 to the power of the result: so many that about a thousand workgroups have work, which
// leaves long groups in pieces and bounds the pieces' sums to about 128 MiB.  Where the groups alone make a thousand, only those of more than
// eight times the average are cut.
int gradient_shift(int64_t n, int64_t G, int R, int C)
{
    const int64_t tiles = ceil_div(R, 128) * ceil_div(C, 128);
    int64_t T = ceil_div(n * tiles, 1024);
    if (G * tiles >= 1024) T = std::max(T, ceil_div(8 * n, G));
    int shift = 8;
    while ((1ll << shift) < T && shift < 24) ++shift;
    return shift;
}

}  // namespace

extern "C" int ivf_grouped_product(const void *x, int64_t ldx, int64_t n, const void *w, int64_t G, int R, int C, const uint32_t *offsets,
                                   int transposed, int type, void *y, int64_t ldy, int out_type, void *hip_stream)
{
    if (!offsets || !w || (n > 0 && (!x || !y))) return fail(IVF_EINVAL, "NULL argument");
    int rc = check_types(type, out_type);
    if (!rc) rc = check_groups(n, G, R, C);
    if (rc) return rc;
    const int in = transposed ? R : C, cols = transposed ? C : R;
    if (ldx < in || ldy < cols) return fail(IVF_EINVAL, "ldx=%lld or ldy=%lld is less than a row", (long long)ldx, (long long)ldy);
    if (!aligned(x, bytes_of(type)) || !aligned(w, bytes_of(type)) || !aligned(y, bytes_of(out_type))) return fail(IVF_EINVAL, "an array is not aligned to its elements");
    if (n == 0) return IVF_OK;
    GroupedArgs a{static_cast<const uint8_t *>(x), ldx, static_cast<const uint8_t *>(w), (int)n, (int)G, R, C, offsets, y, ldy, type_of(out_type), 0};
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    return by_type(type, [&](auto t) -> int {
        constexpr Type T = decltype(t)::value;
        auto launch = [&](auto kernel, int BX, int BW) -> int {
            return in_launches((n / BX + G + 1) * ceil_div(cols, BW), 256, [&](uint32_t first, dim3 grid) -> int {
                a.first = first;
                kernel<<<grid, dim3(256), 0, st>>>(a);
                LAUNCHCHK("grouped_product_kernel");
                return IVF_OK;
            });
        };
        if constexpr (T != Type::F32) {
            constexpr bool HALF = T == Type::F16;
            if (n / G >= 64 && direct_rows(x, ldx, in, type) && direct_rows(w, C, C, type)) {
                auto direct = [&](auto kernel, int BX, int BW, int threads) -> int {
                    const int64_t pieces = n / BX + G + 1;
                    return in_launches(pieces * ceil_div(cols, BW), threads, [&](uint32_t first, dim3 grid) -> int {
                        a.first = first;
                        kernel<<<grid, dim3((unsigned)threads), 0, st>>>(a, (int)pieces);
                        LAUNCHCHK("grouped_product_direct_kernel");
                        return IVF_OK;
                    });
                };
                // Tiles of 256 x 256 fill the units with half as many and leave more of the last ones empty, and their first loads and stores are hidden by nothing,
                // so: long sums, large groups, half the units at least.  Against the others: 2048 rows, 4 matrices of 4096 x 2048 56 us to 63, 16 384 rows and 32 of
                // them 372 to 406, 8192 rows, 8 of 1024 x 4096 85 to 114; but 8192 rows, 16 of 2048 x 1024 62 to 53, 32 of 2048 x 2048 146 to 130, 4096 rows, 4
                // of 1024 x 2048 48 to 34.  In between (256 to 768 rows a group, 1024 to 2048 terms) they are within 10 % of each other but where one of them needs one round of the units more:
                // 6144 rows, 16 of 1024 x 4096 80 to 109, 12 288 of them 169 to 124.
                // Transposed products read W by columns, with twice the reads: 470 us by such tiles, 404 by the others, for 16 384 rows and 16 of 4096 x 2048.
                if (!transposed && C >= 2048 && n / G >= 512 && n / 256 * ceil_div(cols, 256) >= 128)
                    return direct(grouped_product_wide_kernel<HALF>, 256, 256, 256);
                return transposed ? direct(grouped_product_direct_kernel<HALF, true, 128, 256, 2, 4, 32, 3>, 128, 256, 512)
                                  : direct(grouped_product_direct_kernel<HALF, false, 128, 256, 2, 4, 32, 3>, 128, 256, 512);
            }
        }
        if (ceil_div(n, G) <= FEW_ROWS) return transposed ? launch(grouped_few_transposed_kernel<T>, FEW_ROWS, 64) : launch(grouped_few_kernel<T>, FEW_ROWS, 4 * FEW_LINES);
        // Rows of a tile by the average group: a last piece is half empty on average, and the smaller tile leaves room for a fourth workgroup on a
        // compute unit (500 000 x 96 fp32 in 4096 groups: 173 us with 64 rows, 318 with 128).  Sums of up to 128 products in fp32 need no sums apart (96 products: 1.5e-7 of
        // the result in 143 us, plain fp32 1.8e-7; 0.8e-7 in 160 us with them).
        auto by_rows = [&](auto apart) -> int {
            constexpr bool APART = decltype(apart)::value;
            if (n / G < 256 && n / G >= 32) return transposed ? launch(grouped_product_kernel<T, true, 64, 128, APART>, 64, 128) : launch(grouped_product_kernel<T, false, 64, 128, APART>, 64, 128);
            if (n / G >= 256) return transposed ? launch(grouped_product_kernel<T, true, 128, 128, APART>, 128, 128) : launch(grouped_product_kernel<T, false, 128, 128, APART>, 128, 128);
            return transposed ? launch(grouped_product_kernel<T, true, 32, 128, APART>, 32, 128) : launch(grouped_product_kernel<T, false, 32, 128, APART>, 32, 128);
        };
        if constexpr (T == Type::F32)
            if (in > 128) return by_rows(std::true_type{});
        return by_rows(std::false_type{});
    });
}

extern "C" int64_t ivf_grouped_gradient_workspace(int64_t n, int64_t G, int R, int C)
{
    if (check_groups(n, G, R, C)) return IVF_EINVAL;
    const int64_t T = 1ll << gradient_shift(n, G, R, C);
    return n <= T ? 0 : (2 * (n / T) + 2) * R * C * (int64_t)sizeof(float);
}

extern "C" int ivf_grouped_gradient(const void *dy, int64_t lddy, const void *x, int64_t ldx, int64_t n, int64_t G, int R, int C,
                                    const uint32_t *offsets, int type, void *dw, int out_type, void *workspace, int64_t workspace_bytes,
                                    void *hip_stream)
{
    if (!offsets || !dw || (n > 0 && (!x || !dy))) return fail(IVF_EINVAL, "NULL argument");
    int rc = check_types(type, out_type);
    if (!rc) rc = check_groups(n, G, R, C);
    if (rc) return rc;
    if (ldx < C || lddy < R) return fail(IVF_EINVAL, "ldx=%lld or lddy=%lld is less than a row", (long long)ldx, (long long)lddy);
    if (!aligned(x, bytes_of(type)) || !aligned(dy, bytes_of(type)) || !aligned(dw, bytes_of(out_type))) return fail(IVF_EINVAL, "an array is not aligned to its elements");
    const int64_t need = ivf_grouped_gradient_workspace(n, G, R, C);
    if (workspace_bytes < need || (need > 0 && !workspace)) return fail(IVF_EINVAL, "workspace of %lld bytes, %lld needed", (long long)workspace_bytes, (long long)need);
    if (need > 0 && !aligned(workspace, 16)) return fail(IVF_EINVAL, "workspace must be 16-byte aligned");
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const int shift = gradient_shift(n, G, R, C);
    GradientArgs a{static_cast<const uint8_t *>(dy), lddy, static_cast<const uint8_t *>(x), ldx, (int)n, (int)G, R, C, offsets, dw, type_of(out_type),
                   shift, static_cast<float *>(workspace), 0};
    const int64_t pieces = (n >> shift) + G + 1, blocks = pieces * gradient_tiles((uint32_t)(ceil_div(R, 128) * ceil_div(C, 128)));
    rc = by_type(type, [&](auto t) -> int {
        constexpr Type E = decltype(t)::value;
        auto launch = [&](auto kernel) -> int {
            return in_launches(blocks, 256, [&](uint32_t first, dim3 grid) -> int {
                a.first = first;
                kernel<<<grid, dim3(256), 0, st>>>(a);
                LAUNCHCHK("grouped_gradient_kernel");
                return IVF_OK;
            });
        };
        if constexpr (E != Type::F32)
            if (direct_rows(x, ldx, C, type) && direct_rows(dy, lddy, R, type)) return launch(grouped_gradient_direct_kernel<E == Type::F16, 128, 128, 2, 2>);
        return launch(grouped_gradient_kernel<E, 128, 128>);
    });
    if (rc || need == 0) return rc;
    // (few groups have several pieces: workgroups look at many)
    const int64_t down = std::min<int64_t>(G, 1024), across = std::max<int64_t>(1, std::min(ceil_div((int64_t)R * C, 1024), 4096 / down));
    gradient_join_kernel<<<dim3((unsigned)across, (unsigned)down), dim3(256), 0, st>>>(a);
    LAUNCHCHK("gradient_join_kernel");
    return IVF_OK;
}

namespace {

constexpr int ORTHO_MOST_STEPS = 1000;

struct OrthoPlan {
    int m, n, ldm, ldn, chunks, parts;
    int64_t y, yt, f, sums, total;                            // bytes
    bool small;
};

int ortho_plan(int64_t batch, int rows, int cols, int type, OrthoPlan &p)
{
    if (!type_known(type)) return fail(IVF_EINVAL, "type=%d is none of IVF_F32, IVF_F16, IVF_BF16", type);
    if (rows < 1 || cols < 1 || rows > IVF_MAX_SIDE || cols > IVF_MAX_SIDE) return fail(IVF_EINVAL, "rows=%d and cols=%d must be in [1, %d]", rows, cols, IVF_MAX_SIDE);
    if (batch < 0 || batch * rows >= (1ll << 31) || batch * cols >= (1ll << 31)) return fail(IVF_EINVAL, "batch=%lld out of range", (long long)batch);
    p.m = rows < cols ? rows : cols;
    p.n = rows < cols ? cols : rows;
    p.ldm = (int)ceil_div(p.m, 32) * 32;
    p.ldn = (int)ceil_div(p.n, 32) * 32;
    const int64_t size = (int64_t)rows * cols;
    p.chunks = (int)ceil_div(size, NORM_CHUNK);
    auto whole = [](int64_t b) { return ceil_div(b, 256) * 256; };
    p.y = whole(batch * ORTHO_TERMS * p.m * p.ldn * 2);
    p.yt = whole(batch * ORTHO_TERMS * p.n * p.ldm * 2);
    p.f = whole(batch * ORTHO_TERMS * p.m * p.ldm * 2);
    // sums of squares by chunks of X or by tiles of Y, of 64 x 64 at least; of each matrix an inverse norm, a norm and the multipliers
    p.parts = (int)std::max<int64_t>(p.chunks, ceil_div(p.m, 64) * ceil_div(p.n, 64));
    p.sums = whole(batch * (p.parts * 8 + 16 + (int64_t)sizeof(OrthoScales)));
    // (matrices that one launch takes through all steps: no more than the coefficients of a long run)
    p.small = rows <= ORTHO_SMALL_SIDE && cols <= ORTHO_SMALL_SIDE;
    p.total = p.small ? whole(3 * ORTHO_MOST_STEPS * sizeof(float)) : p.y + 2 * p.yt + 2 * p.f + p.sums;
    return IVF_OK;
}

// Whether every step's bounds are near enough to what it makes for scales that they give.
bool ortho_bounded(int steps, const float *coefs)
{
    double S = 1.0;
    for (int i = 0; i < steps; ++i) {
        if (std::fabs(coefs[3 * i]) < 0.5) return false;
        S = ortho_bounds(coefs[3 * i], coefs[3 * i + 1], coefs[3 * i + 2], S).next;
        if (!(S <= 16.0)) return false;
    }
    return true;
}

// What stands behind the matrices in the workspace.
struct OrthoSums {
    double *parts, *inverse, *norms;
    OrthoScales *scales;
    OrthoSums(uint8_t *ws, int64_t batch, const OrthoPlan &p)
        : parts(reinterpret_cast<double *>(ws + p.y + 2 * p.yt + 2 * p.f)), inverse(parts + batch * p.parts), norms(inverse + batch),
          scales(reinterpret_cast<OrthoScales *>(norms + batch)) {}
};

// the inverse norms of x's matrices, and their norms after that
template <Type T>
int ortho_norms(const void *x, int64_t batch, int64_t size, int chunks, float eps, const OrthoSums &sums, hipStream_t st)
{
    int rc = in_launches(batch * chunks, 256, [&](uint32_t first, dim3 grid) -> int {
        ortho_norm_kernel<T><<<grid, dim3(256), 0, st>>>(first, x, size, chunks, sums.parts);
        LAUNCHCHK("ortho_norm_kernel");
        return IVF_OK;
    });
    if (rc) return rc;
    return in_launches(batch, 64, [&](uint32_t first, dim3 grid) -> int {
        ortho_inverse_kernel<<<grid, dim3(64), 0, st>>>(first, sums.parts, chunks, eps, sums.inverse, sums.norms);
        LAUNCHCHK("ortho_inverse_kernel");
        return IVF_OK;
    });
}

template <Type T>
int ortho_general(const void *x, int64_t batch, int rows, int cols, int steps, const float *coefs, float eps, void *out, const OrthoPlan &p, uint8_t *ws,
                  hipStream_t st)
{
    const bool turned = rows > cols;
    // (as many bytes an element as two terms have)
    float *y = reinterpret_cast<float *>(ws), *yt = reinterpret_cast<float *>(ws + p.y), *yt2 = reinterpret_cast<float *>(ws + p.y + p.yt);
    float *a = reinterpret_cast<float *>(ws + p.y + 2 * p.yt), *f = reinterpret_cast<float *>(ws + p.y + 2 * p.yt + p.f);
    const OrthoSums sums(ws, batch, p);
    if (int rc = ortho_norms<T>(x, batch, (int64_t)rows * cols, p.chunks, eps, sums, st)) return rc;
    ortho_first_general_kernel<T><<<dim3(4096), dim3(256), 0, st>>>(x, batch, rows, cols, sums.inverse, turned ? yt : y, turned ? y : yt);
    LAUNCHCHK("ortho_first_general_kernel");
    auto product = [&](const OrthoGeneral &g) -> int {
        return in_launches(batch * ceil_div(g.rows_p, 64) * ceil_div(g.rows_q, 64), 256, [&](uint32_t first, dim3 grid) -> int {
            ortho_general_kernel<<<grid, dim3(256), 0, st>>>(first, g);
            LAUNCHCHK("ortho_general_kernel");
            return IVF_OK;
        });
    };
    for (int s = 0; s < steps; ++s) {
        const float *c = coefs + 3 * s;
        // (without a last coefficient A^2, which may leave fp32's range, is not formed)
        if (c[2] == 0.f) {
            if (int rc = product({y, y, p.m, p.m, p.n, c[1], 0.f, c[0], nullptr, f, nullptr, nullptr, T, 0})) return rc;
        } else {
            if (int rc = product({y, y, p.m, p.m, p.n, 1.f, 0.f, 0.f, nullptr, a, nullptr, nullptr, T, 0})) return rc;
            if (int rc = product({a, a, p.m, p.m, p.m, c[2], c[1], c[0], a, f, nullptr, nullptr, T, 0})) return rc;
        }
        if (int rc = product({yt, f, p.n, p.m, p.m, 1.f, 0.f, 0.f, nullptr, y, yt2, s + 1 == steps ? out : nullptr, T, turned})) return rc;
        std::swap(yt, yt2);
    }
    return IVF_OK;
}

template <Type T, int B, int BS>
int ortho_steps(const void *x, int64_t batch, int rows, int cols, int steps, const float *coefs, float eps, void *out, const OrthoPlan &p, uint8_t *ws,
                hipStream_t st)
{
    const bool turned = rows > cols;                          // Y is X transposed
    OrthoMatrix y{reinterpret_cast<uint16_t *>(ws), p.m, p.n, p.ldn};
    OrthoMatrix yt{reinterpret_cast<uint16_t *>(ws + p.y), p.n, p.m, p.ldm};
    OrthoMatrix yt2{reinterpret_cast<uint16_t *>(ws + p.y + p.yt), p.n, p.m, p.ldm};
    OrthoMatrix a{reinterpret_cast<uint16_t *>(ws + p.y + 2 * p.yt), p.m, p.m, p.ldm};
    OrthoMatrix f{reinterpret_cast<uint16_t *>(ws + p.y + 2 * p.yt + p.f), p.m, p.m, p.ldm};
    const OrthoSums sums(ws, batch, p);
    const int64_t side = ceil_div(p.m, BS), sym = batch * side * (side + 1) / 2, tiles = ceil_div(p.m, B) * ceil_div(p.n, B), all = batch * tiles;
    constexpr int NT = 256;
    if (int rc = ortho_norms<T>(x, batch, (int64_t)rows * cols, p.chunks, eps, sums, st)) return rc;
    int rc = in_launches(batch * ceil_div(rows, 32) * ceil_div(cols, 32), NT, [&](uint32_t first, dim3 grid) -> int {
        ortho_first_kernel<T><<<grid, dim3(NT), 0, st>>>(first, x, rows, cols, sums.inverse, sums.norms, turned ? yt : y, turned ? y : yt);
        LAUNCHCHK("ortho_first_kernel");
        return IVF_OK;
    });
    double most = 1.0;
    for (int s = 0; s < steps && !rc; ++s) {
        const float *c = coefs + 3 * s;
        const int direct = c[2] == 0.f;
        rc = in_launches(batch, 64, [&](uint32_t first, dim3 grid) -> int {
            ortho_scales_kernel<<<grid, dim3(64), 0, st>>>(first, s ? sums.parts : nullptr, (int)tiles, sums.norms, c[0], c[1], c[2], most, sums.scales);
            LAUNCHCHK("ortho_scales_kernel");
            return IVF_OK;
        });
        most = ortho_bounds(c[0], c[1], c[2], most).next;
        if (!rc)
            rc = in_launches(sym, NT, [&](uint32_t first, dim3 grid) -> int {
                ortho_symmetric_kernel<BS, 2, true><<<grid, dim3(NT), 0, st>>>(first, y, direct ? f : a, sums.scales, direct);
                LAUNCHCHK("ortho_symmetric_kernel");
                return IVF_OK;
            });
        if (!rc && !direct)
            rc = in_launches(sym, NT, [&](uint32_t first, dim3 grid) -> int {
                ortho_symmetric_kernel<BS, 2, false><<<grid, dim3(NT), 0, st>>>(first, a, f, sums.scales, 0);
                LAUNCHCHK("ortho_symmetric_kernel");
                return IVF_OK;
            });
        if (!rc)
            rc = in_launches(all, NT, [&](uint32_t first, dim3 grid) -> int {
                ortho_apply_kernel<B, 2><<<grid, dim3(NT), 0, st>>>(first, yt, f, y, yt2, sums.scales, sums.parts, s + 1 == steps ? out : nullptr, T, turned);
                LAUNCHCHK("ortho_apply_kernel");
                return IVF_OK;
            });
        std::swap(yt, yt2);
    }
    return rc;
}

template <int MB, int NB>
int ortho_small(OrthoSmallArgs &a, int64_t batch, hipStream_t st)
{
    return in_launches(batch, WAVE * MB, [&](uint32_t first, dim3 grid) -> int {
        a.first = first;
        ortho_small_kernel<MB, NB><<<grid, dim3(WAVE * MB), 0, st>>>(a);
        LAUNCHCHK("ortho_small_kernel");
        return IVF_OK;
    });
}

int ortho_small(OrthoSmallArgs &a, int64_t batch, hipStream_t st)
{
    const int m = a.turned ? a.cols : a.rows, n = a.turned ? a.rows : a.cols;
    switch ((m + 31) / 32 * 10 + (n + 31) / 32) {
    case 11: return ortho_small<1, 1>(a, batch, st);
    case 12: return ortho_small<1, 2>(a, batch, st);
    case 13: return ortho_small<1, 3>(a, batch, st);
    case 14: return ortho_small<1, 4>(a, batch, st);
    case 22: return ortho_small<2, 2>(a, batch, st);
    case 23: return ortho_small<2, 3>(a, batch, st);
    case 24: return ortho_small<2, 4>(a, batch, st);
    case 33: return ortho_small<3, 3>(a, batch, st);
    case 34: return ortho_small<3, 4>(a, batch, st);
    default: return ortho_small<4, 4>(a, batch, st);
    }
}

}  // namespace

extern "C" int64_t ivf_orthogonalise_workspace(int64_t batch, int rows, int cols, int type)
{
    OrthoPlan p;
    const int rc = ortho_plan(batch, rows, cols, type, p);
    return rc ? rc : p.total;
}

extern "C" int ivf_orthogonalise(const void *x, int64_t batch, int rows, int cols, int type, int steps, const float *coefs, float eps, void *out,
                                 void *workspace, int64_t workspace_bytes, void *hip_stream)
{
    OrthoPlan p;
    if (int rc = ortho_plan(batch, rows, cols, type, p)) return rc;
    if (!coefs || (batch > 0 && (!x || !out))) return fail(IVF_EINVAL, "NULL argument");
    if (steps < 1 || steps > ORTHO_MOST_STEPS) return fail(IVF_EINVAL, "steps=%d out of range", steps);
    if (!(eps >= 0.f) || eps > 1e30f) return fail(IVF_EINVAL, "eps must be finite and not negative");
    for (int i = 0; i < 3 * steps; ++i)
        if (!std::isfinite(coefs[i])) return fail(IVF_EINVAL, "a coefficient is not finite");
    if (!aligned(x, bytes_of(type)) || !aligned(out, bytes_of(type))) return fail(IVF_EINVAL, "an array is not aligned to its elements");
    if (batch == 0) return IVF_OK;
    if (workspace_bytes < p.total || (p.total > 0 && !workspace)) return fail(IVF_EINVAL, "workspace of %lld bytes, %lld needed", (long long)workspace_bytes, (long long)p.total);
    if (!aligned(workspace, 16)) return fail(IVF_EINVAL, "workspace must be 16-byte aligned");
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    if (p.small) {
        OrthoSmallArgs a{x, out, rows, cols, steps, rows > cols, type_of(type), eps, 0, nullptr, {}};
        if (steps <= ORTHO_SMALL_STEPS) {
            std::copy(coefs, coefs + 3 * steps, a.coefs);
        } else {
            a.more = static_cast<const float *>(workspace);
            for (int i = 0; i < steps; i += ORTHO_SMALL_STEPS) {
                OrthoCoefs c{static_cast<float *>(workspace) + 3 * i, 3 * std::min(ORTHO_SMALL_STEPS, steps - i), {}};
                std::copy(coefs + 3 * i, coefs + 3 * i + c.count, c.coefs);
                ortho_coefs_kernel<<<dim3(1), dim3(256), 0, st>>>(c);
                LAUNCHCHK("ortho_coefs_kernel");
            }
        }
        return ortho_small(a, batch, st);
    }
    const bool bounded = ortho_bounded(steps, coefs);
    return by_type(type, [&](auto t) -> int {
        constexpr Type T = decltype(t)::value;
        if (!bounded) return ortho_general<T>(x, batch, rows, cols, steps, coefs, eps, out, p, ws, st);
        // Tiles of 128 where they are enough for the compute units: of the symmetric products only about half are formed, 136 for 2048 x 2048, one on
        // half of the units; of 64 there are 528.
        const int64_t side = ceil_div(p.m, 128), all = batch * side * ceil_div(p.n, 128), sym = batch * side * (side + 1) / 2;
        auto go = [&](auto b, auto bs) { return ortho_steps<T, decltype(b)::value, decltype(bs)::value>(x, batch, rows, cols, steps, coefs, eps, out, p, ws, st); };
        using B64 = std::integral_constant<int, 64>;
        using B128 = std::integral_constant<int, 128>;
        if (all < 256) return go(B64{}, B64{});
        if (sym < 512) return go(B128{}, B64{});
        return go(B128{}, B128{});
    });
}

namespace {

int check_mx4(const void *codes, const void *scales, int64_t n, int D)
{
    if (n < 0 || n >= (1ll << 40) || D < 1 || D > IVF_MAX_SIDE) return fail(IVF_EINVAL, "n=%lld or D=%d out of range", (long long)n, D);
    if (n > 0 && (!codes || !scales)) return fail(IVF_EINVAL, "NULL argument");
    if (!aligned(codes, 16)) return fail(IVF_EINVAL, "codes must be 16-byte aligned");
    return IVF_OK;
}

// launch(first row, rows, grid) for as many launches as rows of `lanes` lanes take, which are numbered in 32 bits
template <class F>
int rows_in_launches(int64_t n, int64_t lanes, F launch)
{
    const int64_t most = ((1ll << 32) - 256) / lanes;
    for (int64_t first = 0; first < n; first += most) {
        const int64_t rows = std::min(most, n - first);
        if (int rc = launch(first, rows, dim3((unsigned)ceil_div(rows * lanes, 256)))) return rc;
    }
    return IVF_OK;
}

// the values of rows of D components, `width` (0: D) of each row of out written
int mx4_expand(const uint8_t *codes, const uint8_t *scales, int64_t n, int D, void *out, int64_t ldo, int out_type, hipStream_t st, int width = 0)
{
    const int64_t blocks = ceil_div(D, 32);
    if (width) D = width;                                     // (no more than the blocks hold)
    const bool f32 = out_type == IVF_F32;
    return rows_in_launches(n, ceil_div(D, f32 ? 4 : 8), [&](int64_t first, int64_t rows, dim3 grid) -> int {
        const uint8_t *c = codes + first * blocks * 16, *s = scales + first * blocks;
        void *o = static_cast<uint8_t *>(out) + first * ldo * bytes_of(out_type);
        if (f32) mx4_expand_kernel<true><<<grid, dim3(256), 0, st>>>(c, s, rows, (int)blocks, D, o, ldo, type_of(out_type));
        else mx4_expand_kernel<false><<<grid, dim3(256), 0, st>>>(c, s, rows, (int)blocks, D, o, ldo, type_of(out_type));
        LAUNCHCHK("mx4_expand_kernel");
        return IVF_OK;
    });
}

}  // namespace

extern "C" int ivf_mx4_quantise(const void *x, int64_t ldx, int64_t n, int D, int type, uint8_t *codes, uint8_t *scales, void *hip_stream)
{
    if (!type_known(type)) return fail(IVF_EINVAL, "type=%d is none of IVF_F32, IVF_F16, IVF_BF16", type);
    if (int rc = check_mx4(codes, scales, n, D)) return rc;
    if (n > 0 && !x) return fail(IVF_EINVAL, "NULL argument");
    if (ldx < D) return fail(IVF_EINVAL, "ldx=%lld is less than a row", (long long)ldx);
    if (!aligned(x, bytes_of(type))) return fail(IVF_EINVAL, "x is not aligned to its elements");
    if (n == 0) return IVF_OK;
    const int64_t blocks = ceil_div(D, 32);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    return by_type(type, [&](auto t) -> int {
        return rows_in_launches(n, 4 * blocks, [&](int64_t first, int64_t rows, dim3 grid) -> int {
            mx4_quantise_kernel<decltype(t)::value><<<grid, dim3(256), 0, st>>>(static_cast<const uint8_t *>(x) + first * ldx * bytes_of(type), ldx, rows, D,
                                                                               reinterpret_cast<uint32_t *>(codes + first * blocks * 16), scales + first * blocks);
            LAUNCHCHK("mx4_quantise_kernel");
            return IVF_OK;
        });
    });
}

extern "C" int ivf_mx4_expand(const uint8_t *codes, const uint8_t *scales, int64_t n, int D, void *out, int64_t ldo, int out_type, void *hip_stream)
{
    if (!type_known(out_type)) return fail(IVF_EINVAL, "out_type=%d is none of IVF_F32, IVF_F16, IVF_BF16", out_type);
    if (int rc = check_mx4(codes, scales, n, D)) return rc;
    if (n > 0 && !out) return fail(IVF_EINVAL, "NULL argument");
    if (ldo < D) return fail(IVF_EINVAL, "ldo=%lld is less than a row", (long long)ldo);
    if (!aligned(out, bytes_of(out_type))) return fail(IVF_EINVAL, "out is not aligned to its elements");
    if (n == 0) return IVF_OK;
    return mx4_expand(codes, scales, n, D, out, ldo, out_type, static_cast<hipStream_t>(hip_stream));
}

extern "C" int ivf_mx4_product(const uint8_t *a_codes, const uint8_t *a_scales, int64_t m, const uint8_t *b_codes, const uint8_t *b_scales, int64_t n,
                               int D, void *out, int64_t ldo, int out_type, void *hip_stream)
{
    if (!type_known(out_type)) return fail(IVF_EINVAL, "out_type=%d is none of IVF_F32, IVF_F16, IVF_BF16", out_type);
    int rc = check_mx4(a_codes, a_scales, m, D);
    if (!rc) rc = check_mx4(b_codes, b_scales, n, D);
    if (rc) return rc;
    if (m > 0 && n > 0 && !out) return fail(IVF_EINVAL, "NULL argument");
    if (ldo < n) return fail(IVF_EINVAL, "ldo=%lld is less than a row", (long long)ldo);
    if (!aligned(out, bytes_of(out_type))) return fail(IVF_EINVAL, "out is not aligned to its elements");
    if (m == 0 || n == 0) return IVF_OK;
    Mx4Args g{a_codes, a_scales, m, b_codes, b_scales, n, (int)ceil_div(D, 32), out, ldo, type_of(out_type), 0};
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    return in_launches(ceil_div(m, 128) * ceil_div(n, 128), 256, [&](uint32_t first, dim3 grid) -> int {
        g.first = first;
        mx4_product_kernel<128, 2, 128, 2><<<grid, dim3(256), 0, st>>>(g);
        LAUNCHCHK("mx4_product_kernel");
        return IVF_OK;
    });
}

namespace {

// How a product of rows with 4-bit rows goes: through b's values (bfloat16, in the workspace) where enough rows of a share them, up to 1 GiB (not transposed only for rows
// of a that are copied straight into LDS, `words`: others multiply expanded codes faster, 4096 x 8192 x 1024 in 170 us against 250); and
// in how many parts of how many rows of b the sum over those is taken (TRANSPOSED): as many as make `wanted` workgroups, of no less than 256 rows.
struct RowsPlan {
    int64_t ld, values, parts, part_rows, sums;               // bytes of the values and of the parts' sums
};

RowsPlan rows_plan(int64_t m, int64_t n, int D, int transposed, int type, bool words)
{
    RowsPlan p{};
    p.ld = ceil_div(D, 8) * 8;
    if (m >= 256 && n > 0 && (transposed || (words && type == IVF_BF16 && D >= 512)) && n * p.ld * 2 <= 1ll << 30) p.values = ceil_div(n * p.ld * 2, 256) * 256;
    p.parts = 1;
    p.part_rows = n;
    if (!transposed || m == 0 || n == 0) return p;
    const int64_t wanted = p.values ? 512 : 1024, tiles = ceil_div(m, m > 32 ? 128 : 32) * ceil_div(D, 128);
    p.parts = std::max<int64_t>(1, std::min(ceil_div(wanted, tiles), n / 256));
    p.part_rows = ceil_div(ceil_div(n, p.parts), 64) * 64;
    p.parts = ceil_div(n, p.part_rows);
    p.sums = p.parts == 1 ? 0 : p.parts * m * D * (int64_t)sizeof(float);
    return p;
}

int check_rows_product(int64_t m, int64_t n, int D)
{
    if (m < 0 || m >= (1ll << 40) || n < 0 || n >= (1ll << 40) || D < 1 || D > IVF_MAX_SIDE)
        return fail(IVF_EINVAL, "m=%lld, n=%lld or D=%d out of range", (long long)m, (long long)n, D);
    return IVF_OK;
}

}  // namespace

namespace {

// up to MX4_FEW rows of a against rows of b whose blocks have room in LDS, where a wavefront's lanes have one each or more
bool mx4_few_fits(int64_t m, int D) { return m <= MX4_FEW && (m <= 2 ? 2 : 4) * ceil_div(D, 32) * MX4_PITCH * 4 <= 64 << 10; }

int mx4_few(const Mx4RowsArgs &g, Type type, hipStream_t st)
{
    const int64_t blocks = ceil_div(g.D, 32);
    const int lanes = blocks <= 4 ? 4 : blocks <= 16 ? 16 : 64, M = g.m == 1 ? 1 : g.m == 2 ? 2 : 4;
    const int64_t rows = 4 * (WAVE / lanes) * (M > 2 ? 2 : 4), groups = std::min<int64_t>(ceil_div(g.n, rows), 1024);
    auto go = [&](auto kernel, size_t lds) {
        kernel<<<dim3((unsigned)groups), dim3(256), lds, st>>>(g, type);
        LAUNCHCHK("mx4_few_kernel");
        return (int)IVF_OK;
    };
    auto by_rows = [&](auto m) -> int {
        constexpr int R = decltype(m)::value;
        if (blocks > 64) return go(mx4_few_kernel<R, 64, false>, (size_t)(R * blocks * MX4_PITCH * 4));
        return lanes == 4 ? go(mx4_few_kernel<R, 4, true>, 0) : lanes == 16 ? go(mx4_few_kernel<R, 16, true>, 0) : go(mx4_few_kernel<R, 64, true>, 0);
    };
    return M == 1 ? by_rows(std::integral_constant<int, 1>{}) : M == 2 ? by_rows(std::integral_constant<int, 2>{}) : by_rows(std::integral_constant<int, 4>{});
}

}  // namespace

namespace {

int mx4_sweep(Mx4RowsArgs &g, int type, hipStream_t st)
{
    const int64_t down = ceil_div(g.m, SWEEP_ROWS), tiles = ceil_div(g.n, SWEEP_COLS);
    // runs of tiles: three workgroups a compute unit, or more where runs would be long
    const int64_t wanted = std::max<int64_t>(1, 3 * 256 / down), run = std::max<int64_t>(8, std::min<int64_t>(ceil_div(tiles, wanted), 256));
    return by_type(type, [&](auto t) -> int {
        constexpr Type T = decltype(t)::value;
        auto go = [&](auto kernel) -> int {
            return in_launches(down * ceil_div(tiles, run), 256, [&](uint32_t first, dim3 grid) -> int {
                g.first = first;
                kernel<<<grid, dim3(256), 0, st>>>(g, (int)run);
                LAUNCHCHK("mx4_sweep_kernel");
                return IVF_OK;
            });
        };
        switch ((g.D + 31) / 32) {
        case 2: return go(mx4_sweep_kernel<T, 2>);
        case 3: return go(mx4_sweep_kernel<T, 3>);
        default: return go(mx4_sweep_kernel<T, 4>);
        }
    });
}

}  // namespace

extern "C" int64_t ivf_mx4_rows_product_workspace(int64_t m, int64_t n, int D, int transposed, int type)
{
    if (!type_known(type)) return fail(IVF_EINVAL, "type=%d is none of IVF_F32, IVF_F16, IVF_BF16", type);
    if (check_rows_product(m, n, D)) return IVF_EINVAL;
    const RowsPlan p = rows_plan(m, n, D, transposed, type, D % 8 == 0);
    return p.values + p.sums;
}

extern "C" int ivf_mx4_rows_product(const void *a, int64_t lda, int64_t m, int type, const uint8_t *codes, const uint8_t *scales, int64_t n, int D,
                                    int transposed, void *out, int64_t ldo, int out_type, void *workspace, int64_t workspace_bytes,
                                    void *hip_stream)
{
    int rc = check_types(type, out_type);
    if (!rc) rc = check_rows_product(m, n, D);
    if (!rc) rc = check_mx4(codes, scales, n, D);
    if (rc) return rc;
    const int64_t in = transposed ? n : D, cols = transposed ? D : n;
    if (lda < in || ldo < cols) return fail(IVF_EINVAL, "lda=%lld or ldo=%lld is less than a row", (long long)lda, (long long)ldo);
    if (m > 0 && cols > 0 && (!out || (in > 0 && !a))) return fail(IVF_EINVAL, "NULL argument");
    if (!aligned(a, bytes_of(type)) || !aligned(out, bytes_of(out_type))) return fail(IVF_EINVAL, "an array is not aligned to its elements");
    const bool direct = type == IVF_BF16 && direct_rows(a, lda, in, type);
    const RowsPlan p = rows_plan(m, n, D, transposed, type, direct);
    const int64_t need = p.values + p.sums;
    if (workspace_bytes < need || (need > 0 && !workspace)) return fail(IVF_EINVAL, "workspace of %lld bytes, %lld needed", (long long)workspace_bytes, (long long)need);
    if (need > 0 && !aligned(workspace, 16)) return fail(IVF_EINVAL, "workspace must be 16-byte aligned");
    if (m == 0 || cols == 0) return IVF_OK;
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    Mx4RowsArgs g{static_cast<const uint8_t *>(a), lda, m, codes, scales, n, D, out, ldo, type_of(out_type), (int)p.parts, p.part_rows,
                  reinterpret_cast<float *>(ws + p.values), 0};
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (!transposed && mx4_few_fits(m, D)) return mx4_few(g, type_of(type), st);
    // Runs of tiles need work for every compute unit: a run is a chain of eight tiles at least.  Of 96 components in fp32 against single tiles 128 x 65 536 20
    // us to 14, 256 x 65 536 21 to 22, 512 x 65 536 29 to 35, 4096 x 65 536 223 to 278; of one block of components never faster (218 to 193).
    if (!transposed && D > 32 && D <= 128 && m >= 64 && n >= 16 * SWEEP_COLS && m >= (int64_t{1} << 24) / n) return mx4_sweep(g, type, st);
    const Mx4Values v{reinterpret_cast<const uint16_t *>(ws), p.ld};
    auto launch = [&](auto kernel, int BM, int BN, unsigned threads) -> int {
        return in_launches(ceil_div(m, BM) * ceil_div(cols, BN) * p.parts, (int)threads, [&](uint32_t first, dim3 grid) -> int {
            g.first = first;
            kernel<<<grid, dim3(threads), 0, st>>>(g, v);
            LAUNCHCHK("mx4_rows_product_kernel");
            return IVF_OK;
        });
    };
    if (p.values) {
        // (columns up to ld: zeros, as the codes past D are)
        if ((rc = mx4_expand(codes, scales, n, D, ws, p.ld, IVF_BF16, st, (int)p.ld))) return rc;
        if (direct) rc = transposed ? launch(mx4_direct_kernel<true, 128, 128, 2, 2, 64, 2>, 128, 128, 256) : launch(mx4_direct_kernel<false, 128, 256, 2, 4, 32, 3>, 128, 256, 512);
        else if (type == IVF_F32) rc = launch(mx4_rows_product_kernel<Type::F32, true, true, 128, 128>, 128, 128, 256);
        else if (type == IVF_F16) rc = launch(mx4_rows_product_kernel<Type::F16, true, true, 128, 128>, 128, 128, 256);
        else rc = launch(mx4_rows_product_kernel<Type::BF16, true, true, 128, 128>, 128, 128, 256);
    } else {
        rc = by_type(type, [&](auto t) -> int {
            constexpr Type T = decltype(t)::value;
            if (m > 32) return transposed ? launch(mx4_rows_product_kernel<T, true, false, 128, 128>, 128, 128, 256) : launch(mx4_rows_product_kernel<T, false, false, 128, 128>, 128, 128, 256);
            return transposed ? launch(mx4_rows_product_kernel<T, true, false, 32, 128>, 32, 128, 256) : launch(mx4_rows_product_kernel<T, false, false, 32, 128>, 32, 128, 256);
        });
    }
    if (rc || p.parts == 1) return rc;
    const int64_t blocks = ceil_div(m * ceil_div(D, 4), 256);
    mx4_join_kernel<<<dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, st>>>(g);
    LAUNCHCHK("mx4_join_kernel");
    return IVF_OK;
}
