// Gated layer: H = act(X Wg) o (X Wu), and its backward pass.
#include <algorithm>

#include "cbm_aligned.h"
#include "cbm_few_rows.h"
#include "cbm_internal.h"
#include "cbm_products.h"
#include "cbm_small.h"

namespace {

template <class T, int ACT>
__device__ __forceinline__ float activated(float g) {
    if constexpr (ACT == CBM_RELU) return g <= 0.0f ? 0.0f : g;  // (NaN stays)
    if constexpr (ACT == CBM_SILU) return g / (1.0f + cbm_exp<T>(-g));
    return 0.5f * g * erfcf(g * -0.70710678f);
}
// the activation and its slope
template <class T, int ACT>
__device__ __forceinline__ void activated(float g, float& value, float& slope) {
    if constexpr (ACT == CBM_RELU) {
        value = activated<T, ACT>(g);
        slope = g > 0.0f ? 1.0f : 0.0f;
    } else if constexpr (ACT == CBM_SILU) {
        const float s = 1.0f / (1.0f + cbm_exp<T>(-g));
        value = g * s;
        slope = s * fmaf(g, 1.0f - s, 1.0f);
    } else {
        const float below = 0.5f * erfcf(g * -0.70710678f);
        value = g * below;
        slope = fmaf(g, 0.39894228f * cbm_exp<T>(-0.5f * g * g), below);
    }
}
template <class F>
void with_activation(int32_t act, F&& f) {
    using std::integral_constant;
    if (act == CBM_SILU) f(integral_constant<int, CBM_SILU>{});
    else if (act == CBM_GELU) f(integral_constant<int, CBM_GELU>{});
    else f(integral_constant<int, CBM_RELU>{});
}

// Both projections in one product: a wave's tiles of 32 columns come from Wg and Wu in turn, so a lane has both sums of a value of H.
template <class Tiles, class T, int ACT>
__global__ __launch_bounds__(256, Tiles::GROUPS) void cbm_gated_kernel(CbmOperand<T> a, CbmOperand<T> b, int64_t m, int64_t chunks, T* __restrict__ H, int64_t ldh, T* __restrict__ G, int64_t ldg,
                                                                    T* __restrict__ U, int64_t ldu, bool far) {
    __shared__ uintx4 lds[Tiles::UNITS];
    const CbmTilePlace at = cbm_tile_place((a.count + Tiles::ROWS - 1) / Tiles::ROWS, (m + Tiles::COLUMNS / 2 - 1) / (Tiles::COLUMNS / 2), 1);
    if (!at.any) return;
    Tiles t;
    t.run(lds, a, b, at.m, at.n, 0, (int)chunks);
    constexpr int W = cbm_wide<T>;
    t.template pairs<W>(lds, at.m, at.n, [&](int64_t r, int64_t c, float (&g)[W], float (&u)[W]) {
        if (r >= a.count) return;
        float h[W];
#pragma unroll
        for (int v = 0; v < W; ++v) h[v] = activated<T, ACT>(g[v]) * u[v];
        cbm_put(H + r * ldh, c, m, h, far);
        if (G) cbm_put(G + r * ldg, c, m, g, far);
        if (U) cbm_put(U + r * ldu, c, m, u, far);
    });
}

// A small product: 32 x 32 values of G and of U a workgroup, its waves sharing K (64 x 256 with 2 x 256 in fp32 21 -> 6 us).
template <class T, int ACT>
__global__ __launch_bounds__(512) void cbm_gated_small_kernel(int64_t n, int64_t k, int64_t m, const T* __restrict__ X, int64_t ldx, const T* __restrict__ Wg, int64_t ldwg, const T* __restrict__ Wu,
                                                            int64_t ldwu, T* __restrict__ H, int64_t ldh, T* __restrict__ G, int64_t ldg, T* __restrict__ U, int64_t ldu) {
    typedef CbmSmallTile<T, T, ALONG_K, ACROSS_K, 2> Tile;
    __shared__ typename Tile::Room room;
    const int64_t r0 = (int64_t)blockIdx.y * Tile::SIDE, c0 = (int64_t)blockIdx.x * Tile::SIDE, r = r0 + Tile::row(), c = c0 + Tile::column();
    Tile t;
    t.add(X, ldx, n, r0, {Wg, Wu}, {ldwg, ldwu}, m, c0, k);
    t.share(room);
    if (r >= n) return;
    float g[2], u[2], h[2];
    Tile::total(room, 0, g);
    Tile::total(room, 1, u);
#pragma unroll
    for (int j = 0; j < 2; ++j) h[j] = activated<T, ACT>(g[j]) * u[j];
    cbm_put(H + r * ldh, c, m, h);
    if (G) cbm_put(G + r * ldg, c, m, g);
    if (U) cbm_put(U + r * ldu, c, m, u);
}

// A few rows: the weights are read once, in pieces of 64 bytes of a row, a workgroup for each 64 bytes of columns.
constexpr int few_waves(int rows) { return rows >= 8 ? 8 : 16; }
template <class T, int NR, int ACT>
__global__ __launch_bounds__(64 * few_waves(NR)) void cbm_gated_few_kernel(int64_t n, int64_t k, int64_t m, const T* __restrict__ X, int64_t ldx, const T* __restrict__ Wg, int64_t ldwg,
                                                                    const T* __restrict__ Wu, int64_t ldwu, T* __restrict__ H, int64_t ldh, T* __restrict__ G, int64_t ldg, T* __restrict__ U,
                                                                    int64_t ldu) {
    typedef CbmFewRows<T, NR, 2, 4, few_waves(NR)> Rows;
    __shared__ typename Rows::Room room;
    const int64_t first = cbm_few_piece() * Rows::COLS, above = (int64_t)blockIdx.y * NR;
    if (first >= m) return;
    Rows::run(room, X + above * ldx, ldx, n - above, k, {Wg, Wu}, {ldwg, ldwu}, m, first);
    const int in = threadIdx.x / Rows::COLS, j = threadIdx.x % Rows::COLS;
    const int64_t c = first + j, r = above + in;
    if (r >= n || in >= NR || c >= m) return;
    const float g = Rows::total(room, 0, in, j), u = Rows::total(room, 1, in, j);
    H[r * ldh + c] = (T)(activated<T, ACT>(g) * u);
    if (G) G[r * ldg + c] = (T)g;
    if (U) U[r * ldu + c] = (T)u;
}

// dG and dU side by side in `out`, from column 0 and column `at` on, zeros between: in fp32 for small products, else rounded to the type (half a step each, as much as the gradients that are made of them are
// rounded by, so that those are off by 1.4 times as much as they would be; a second part would take the products twice as long).
// Rounded to fp16 they are kept at a power of two, or products of what fp16 holds would not fit it (65504^2) or vanish (2^-48) where the gradients do not.  It goes by the largest finite one, which the launch that
// makes them finds out: at 2^10 first, and once more, by a launch that otherwise ends at once, where that puts the largest outside 2^3 to 65504, at the power that puts it below 2^15.  What is made of them is
// multiplied by scale[0].  (16384 x 4096: 124 and 5 us, or 124 and 130 where they are made twice; in bf16 one launch takes 111.)
constexpr int SLOPE_GROUPS = 2048;  // parts of the largest (all of them are read by every group of the second launch: of 8192 parts that takes 25 us instead of 5)
constexpr float SLOPES_AT = 0x1p10f, LEAST_SLOPE = 0x1p3f, MOST_SLOPE = 65504.0f;
template <class T, class S>
constexpr bool cbm_scaled_slopes = sizeof(S) == 2 && !std::is_same<T, __bf16>::value;

__device__ __forceinline__ float largest_of_group(float most, float (&room)[4]) {
    most = lanes_all<64>(most, [](float a, float b) { return fmaxf(a, b); });
    if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = most;
    __syncthreads();
    return fmaxf(fmaxf(room[0], room[1]), fmaxf(room[2], room[3]));
}

// again: of `most` as the first launch left it
template <class T, class S, int ACT>
__global__ __launch_bounds__(256) void cbm_gated_slopes_kernel(int64_t n, int m, const T* __restrict__ dH, int64_t lddh, const T* __restrict__ G, int64_t ldg, const T* __restrict__ U,
                                                            int64_t ldu, S* __restrict__ out, int64_t at, float* __restrict__ scale, float* __restrict__ most, bool again) {
    constexpr int V = 16 / (int)sizeof(T);
    constexpr bool SCALED = cbm_scaled_slopes<T, S>;
    const int64_t pieces = at / V;
    float up = 1.0f, largest = 0.0f;
    __shared__ float room[SCALED ? 4 : 1];
    if constexpr (SCALED) {
        up = SLOPES_AT;
        if (again) {
            for (uint32_t i = threadIdx.x; i < gridDim.x; i += 256) largest = fmaxf(largest, most[i]);
            largest = largest_of_group(largest, room);
            const bool fits = largest == 0.0f || (largest * SLOPES_AT >= LEAST_SLOPE && largest * SLOPES_AT <= MOST_SLOPE);
            if (!fits) up = ldexpf(1.0f, min(14 - ilogbf(largest), 100));
            if (blockIdx.x == 0 && threadIdx.x == 0) scale[0] = 1.0f / up;
            if (fits) return;
        }
    }
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n * pieces; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / pieces;
        const int c = (int)(i % pieces) * V;
        float dh[V] = {}, g[V] = {}, u[V] = {}, dg[V], du[V];
        if (c + V <= m) {
            load_piece<V>(dh, dH + r * lddh + c);
            load_piece<V>(g, G + r * ldg + c);
            load_piece<V>(u, U + r * ldu + c);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (c + j < m) {
                    dh[j] = (float)dH[r * lddh + c + j];
                    g[j] = (float)G[r * ldg + c + j];
                    u[j] = (float)U[r * ldu + c + j];
                }
        }
#pragma unroll
        for (int j = 0; j < V; ++j) {
            float value, slope;
            activated<T, ACT>(g[j], value, slope);
            du[j] = c + j < m ? dh[j] * value : 0.0f;
            dg[j] = c + j < m ? dh[j] * u[j] * slope : 0.0f;
            if constexpr (SCALED) {
                const float a = fabsf(du[j]), b = fabsf(dg[j]);
                largest = fmaxf(largest, fmaxf(a < INFINITY ? a : 0.0f, b < INFINITY ? b : 0.0f));
                du[j] *= up;
                dg[j] *= up;
            }
        }
        store_piece<V>(out + r * 2 * at + c, dg);
        store_piece<V>(out + r * 2 * at + at + c, du);
    }
    if constexpr (SCALED) {
        if (again) return;
        largest = largest_of_group(largest, room);
        if (threadIdx.x == 0) most[blockIdx.x] = largest;
    }
}

}  // namespace

namespace {

// Copies of X (n x k, rows of whole units) and of the weights turned, blocks of 32 columns of Wg and Wu in turn (rows of the result's columns).
struct Copies {
    int64_t ld, weights, bytes;  // where the weights begin; X is first
};
Copies copies_of(int64_t n, int32_t k, int32_t m, int32_t type) {
    if (!cbm_may_pack(n, k, 2 * (int64_t)m, type)) return {};
    const int64_t ld = cbm_whole(k, 8);
    const int64_t x = 2 * cbm_whole(n, 8) * ld;
    return {ld, x, x + 4 * cbm_whole(m, 32) * ld};
}

}  // namespace

int64_t cbm_gated_workspace(int64_t n, int32_t k, int32_t m, int32_t type) { return cbm_too_many_tiles(n, 2 * (int64_t)m) ? 0 : copies_of(n, k, m, type).bytes; }

cbm_status cbm_launch_gated(int64_t n, int32_t k, int32_t m, int32_t type, int32_t act, const void* X, int64_t ldx, const void* Wg, int64_t ldwg, const void* Wu, int64_t ldwu, void* H,
                            int64_t ldh, void* G, int64_t ldg, void* U, int64_t ldu, void* workspace, void* stream) {
    if (n == 0) return CBM_OK;
    if (cbm_too_many_tiles(n, 2 * (int64_t)m)) return CBM_ERR_UNSUPPORTED;
    const Copies copies = copies_of(n, k, m, type);
    cbm_with_type(type, [&](auto t) {
        using T = decltype(t);
        constexpr int V = 16 / (int)sizeof(T);
        if (n <= cbm_most_few_rows<T> && m >= V) {
            cbm_with_few_rows(n, [&](auto rows) {
                with_activation(act, [&](auto which) {
                    cbm_gated_few_kernel<T, decltype(rows)::value, decltype(which)::value><<<dim3((unsigned)(((int64_t)m + 32 * V - 1) / (32 * V) * 8), (unsigned)((n + CBM_FEW_ROWS - 1) / CBM_FEW_ROWS)), 64 * few_waves(decltype(rows)::value), 0, (hipStream_t)stream>>>(
                        n, k, m, (const T*)X, ldx, (const T*)Wg, ldwg, (const T*)Wu, ldwu, (T*)H, ldh, (T*)G, ldg, (T*)U, ldu);
                });
            });
            return;
        }
        if (cbm_small_forward(n, k, 2 * (int64_t)m, cbm_small_groups(n, m), type)) {
            with_activation(act, [&](auto which) {
                cbm_gated_small_kernel<T, decltype(which)::value><<<dim3((unsigned)((m + 31) / 32), (unsigned)((n + 31) / 32)), 512, 0, (hipStream_t)stream>>>(
                    n, k, m, (const T*)X, ldx, (const T*)Wg, ldwg, (const T*)Wu, ldwu, (T*)H, ldh, (T*)G, ldg, (T*)U, ldu);
            });
            return;
        }
        auto run = [&](auto* tiles_type, const CbmOperand<T>& a, const CbmOperand<T>& b) {
            typedef std::remove_pointer_t<decltype(tiles_type)> Tiles;
            const int64_t tiles = (n + Tiles::ROWS - 1) / Tiles::ROWS * (((int64_t)m + Tiles::COLUMNS / 2 - 1) / (Tiles::COLUMNS / 2));
            with_activation(act, [&](auto which) {
                cbm_gated_kernel<Tiles, T, decltype(which)::value><<<(unsigned)((tiles + CBM_XCD - 1) / CBM_XCD * CBM_XCD), 256, 0, (hipStream_t)stream>>>(
                    a, b, m, (k + Tiles::BK - 1) / Tiles::BK, (T*)H, ldh, (T*)G, ldg, (T*)U, ldu, n * m * (int64_t)sizeof(T) >= CBM_FAR_BYTES);
            });
        };
        CbmOperand<T> a{{(const T*)X, nullptr}, {ldx, 0}, n, k, 0}, b{{(const T*)Wg, (const T*)Wu}, {ldwg, ldwu}, m, k, 0};
        if constexpr (sizeof(T) == 2) {
            const bool large = cbm_product_tile(n, 2 * (int64_t)m, k, type) == 256;
            bool units = cbm_units(a.p[0], ldx, k);
            const bool whole = cbm_units(b.p[0], ldwg, m) && cbm_units(b.p[1], ldwu, m) && ldwg == ldwu;
            if (!units && copies.bytes) {
                cbm_launch_pack(X, ldx, n, k, false, workspace, copies.ld, 0, 0, stream);
                a = {{(const T*)workspace, nullptr}, {copies.ld, 0}, n, copies.ld, 0};
                units = true;
            }
            if (units && copies.bytes && (!whole || n >= CBM_TURN_ROWS)) {
                T* turned = (T*)((char*)workspace + copies.weights);
                cbm_launch_pack(Wg, ldwg, m, k, true, turned, copies.ld, 64, 0, stream);
                cbm_launch_pack(Wu, ldwu, m, k, true, turned, copies.ld, 64, 32, stream);
                b = {{turned, nullptr}, {copies.ld, 0}, 2 * cbm_whole(m, 32), copies.ld, 0};
                if (large) run((CbmAlignedTiles<T, 256, 256, ALONG_K, ALONG_K, SINGLE>*)nullptr, a, b);
                else run((CbmAlignedTiles<T, 128, 128, ALONG_K, ALONG_K, SINGLE>*)nullptr, a, b);
                return;
            }
            if (units && whole) {
                if (large) run((CbmAlignedTiles<T, 256, 256, ALONG_K, ACROSS_K, PAIR_ROWS>*)nullptr, a, b);
                else run((CbmAlignedTiles<T, 128, 128, ALONG_K, ACROSS_K, PAIR_ROWS>*)nullptr, a, b);
                return;
            }
        }
        if constexpr (sizeof(T) == 4)
            if (cbm_is_narrow(2 * (int64_t)m, type)) return run((CbmTiles<T, 256, 64, 4, 1, ALONG_K, ACROSS_K, PAIR_ROWS>*)nullptr, a, b);
        run((CbmTiles<T, 128, 128, 2, 2, ALONG_K, ACROSS_K, PAIR_ROWS>*)nullptr, a, b);
    });
    return cbm_launched("gated layer launch");
}

namespace {

// dG and dU side by side, their power of two and largest ones, copies of X and of the weights (rows of whole units), shares of K.
struct BackRoom {
    int64_t at, scale, x, weights, parts, bytes;  // column of dU; where they begin
    bool copies, small;
};
BackRoom back_room(int64_t n, int32_t k, int32_t m, int32_t type) {
    BackRoom r{};
    const int64_t bytes = type == CBM_F32 ? 4 : 2, wide = cbm_whole(k, 8);
    r.at = cbm_whole(m, type == CBM_F32 ? 32 : 64);  // (chunks of the products)
    r.small = cbm_small_backward(n, k, 2 * (int64_t)m, 0, cbm_small_groups(n, k) + 2 * cbm_small_groups(k, m), type);
    if (r.small) {
        r.bytes = n * 2 * r.at * 4;
        return r;
    }
    r.copies = cbm_may_pack(n, k, 2 * (int64_t)m, type);
    r.scale = cbm_whole(n * 2 * r.at * bytes, 16);
    r.x = r.scale + (type == CBM_F16 ? 16 + 4 * SLOPE_GROUPS : 0);
    r.weights = r.x + (r.copies ? 2 * cbm_whole(n, 8) * wide : 0);
    r.parts = r.weights + (r.copies ? 4 * wide * r.at : 0);
    int64_t parts = 0;
    const int64_t dx = cbm_product_parts(n, k, 2 * r.at, type), dw = cbm_product_parts(wide, 2 * r.at, n, type);
    if (dx > 1) parts = dx * n * k;
    if (dw > 1) parts = std::max(parts, dw * wide * 2 * r.at);
    r.bytes = r.parts + 4 * parts;
    return r;
}

}  // namespace

namespace {

bool back_too_large(int64_t n, int32_t k, int32_t m) { return cbm_too_many_tiles(n, k) || cbm_too_many_tiles(cbm_whole(k, 8), 2 * cbm_whole(m, 64)); }

}  // namespace

int64_t cbm_gated_back_workspace(int64_t n, int32_t k, int32_t m, int32_t type) { return back_too_large(n, k, m) ? 0 : back_room(n, k, m, type).bytes; }

cbm_status cbm_launch_gated_backward(int64_t n, int32_t k, int32_t m, int32_t type, int32_t act, const void* dH, int64_t lddh, const void* X, int64_t ldx, const void* Wg, int64_t ldwg,
                                     const void* Wu, int64_t ldwu, const void* G, int64_t ldg, const void* U, int64_t ldu, void* dX, int64_t lddx, void* dWg, int64_t lddwg, void* dWu,
                                     int64_t lddwu, void* workspace, void* stream) {
    if (back_too_large(n, k, m)) return CBM_ERR_UNSUPPORTED;
    const BackRoom room = back_room(n, k, m, type);
    const int64_t at = room.at;
    char* base = (char*)workspace;
    float *parts = (float*)(base + room.parts), *scale = type == CBM_F16 && !room.small && n > 0 ? (float*)(base + room.scale) : nullptr;
    if (n > 0)
        cbm_with_type(type, [&](auto t) {
            using T = decltype(t);
            const int64_t blocks = (n * (at * (int64_t)sizeof(T) / 16) + 255) / 256;
            with_activation(act, [&](auto which) {
                auto slopes = [&](auto* out) {
                    using S = std::remove_pointer_t<decltype(out)>;
                    const unsigned grid = (unsigned)std::min<int64_t>(blocks, cbm_scaled_slopes<T, S> ? SLOPE_GROUPS : 1 << 22);
                    for (int again = 0; again < (cbm_scaled_slopes<T, S> ? 2 : 1); ++again)
                        cbm_gated_slopes_kernel<T, S, decltype(which)::value><<<grid, 256, 0, (hipStream_t)stream>>>(n, m, (const T*)dH, lddh, (const T*)G, ldg, (const T*)U, ldu, out, at, scale,
                                                                                                                    scale ? scale + 4 : nullptr, again != 0);
                };
                if (room.small) slopes((float*)workspace);
                else slopes((T*)workspace);
            });
        });
    if (room.small) {
        const float* slopes = (const float*)workspace;
        if (dX && n > 0) cbm_launch_small_along(type, n, k, m, slopes, slopes + at, 2 * at, Wg, ldwg, Wu, ldwu, dX, lddx, stream);
        if (dWg || dWu) cbm_launch_small_across(type, k, m, n, X, ldx, slopes, slopes + at, 2 * at, dWg, lddwg, dWu, lddwu, stream);
        return cbm_launched("gated layer backward launch");
    }
    CbmProduct p{};
    p.type = type;
    p.A = workspace;
    p.lda = 2 * at;
    p.out.factor = scale;
    auto in_units = [&](const void* q, int64_t ld, int64_t along) { return cbm_units((const _Float16*)q, ld, along); };
    if (dX && n > 0) {
        p.M = n;
        p.N = k;
        p.K = m;
        p.at = at;
        p.B[0] = Wg;
        p.B[1] = Wu;
        p.ldb[0] = ldwg;
        p.ldb[1] = ldwu;
        if (room.copies && !(in_units(Wg, ldwg, m) && in_units(Wu, ldwu, m) && ldwg == ldwu)) {
            for (int i = 0; i < 2; ++i) {
                void* to = base + room.weights + i * 2 * cbm_whole(k, 8) * at;
                cbm_launch_pack(p.B[i], p.ldb[i], k, m, false, to, at, 0, 0, stream);
                p.B[i] = to;
                p.ldb[i] = at;
            }
            p.K = at;  // (zeros beyond m)
        }
        p.out.C[0] = dX;
        p.out.ldc[0] = lddx;
        p.out.columns = k;
        p.parts = cbm_product_parts(n, k, 2 * at, type) > 1 ? parts : nullptr;
        cbm_launch_tiles(p, stream);
    }
    if (dWg || dWu) {
        p.M = k;
        p.N = 2 * at;
        p.K = n;
        p.at = 0;
        p.A = X;
        p.lda = ldx;
        p.a_across = p.b_across = true;
        if (room.copies && n > 0 && !in_units(X, ldx, k)) {
            p.lda = p.M = cbm_whole(k, 8);
            p.out.rows = k;
            p.A = base + room.x;
            cbm_launch_pack(X, ldx, n, k, false, base + room.x, p.lda, 0, 0, stream);
        }
        p.B[0] = workspace;
        p.B[1] = nullptr;
        p.ldb[0] = 2 * at;
        p.out.C[0] = dWg;
        p.out.C[1] = dWu;
        p.out.ldc[0] = lddwg;
        p.out.ldc[1] = lddwu;
        p.out.columns = m;
        p.out.at = (int32_t)at;
        p.parts = cbm_product_parts(cbm_whole(k, 8), 2 * at, n, type) > 1 ? parts : nullptr;
        cbm_launch_tiles(p, stream);
    }
    return cbm_launched("gated layer backward launch");
}
