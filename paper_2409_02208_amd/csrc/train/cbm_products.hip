// Products in tiles with a plain end: sums scaled, added to and rounded.  The gradients of the operators that are made of products, and the steps of the orthogonal update.
#include <algorithm>
#include <type_traits>

#include "cbm_aligned.h"
#include "cbm_internal.h"
#include "cbm_products.h"

namespace {

template <class TO, int W>
__device__ __forceinline__ void finish(const CbmProductOut& o, int64_t M, int64_t N, int64_t r, int64_t c, float (&v)[W]) {
    if (r >= M || c >= N) return;
    if (o.sums) {
        float* s = o.sums + r * N + c;
        if (!o.first)
#pragma unroll
            for (int j = 0; j < W; ++j)
                if (c + j < N) v[j] += s[j];
        if (!o.last) return cbm_put<W>(o.sums + r * N, c, N, v);
    }
    float up = o.alpha;
    if (o.factor) up *= *o.factor;
#pragma unroll
    for (int j = 0; j < W; ++j) v[j] *= up;
    if (o.more)
#pragma unroll
        for (int j = 0; j < W; ++j)
            if (c + j < N) v[j] = fmaf(o.beta, o.more[r * o.ldm + c + j], v[j]);
    const bool second = o.at && c >= o.at;
    if (second) c -= o.at;
    TO* C = (TO*)o.C[second];
    const int64_t ld = o.ldc[second];
    if (!C) return;
    if (o.transposed) {
#pragma unroll
        for (int j = 0; j < W; ++j)
            if (c + j < o.columns) C[(c + j) * ld + r] = (TO)v[j];
    } else {
        cbm_put<W>(C + r * ld, c, o.columns, v);
    }
}

template <class Tiles, class T, class TO>
__global__ __launch_bounds__(256, Tiles::GROUPS) void cbm_product_kernel(CbmOperand<T> a, CbmOperand<T> b, int64_t chunks, int64_t splits, CbmProductOut o, float* __restrict__ parts) {
    __shared__ uintx4 lds[Tiles::UNITS];
    const CbmTilePlace at = cbm_tile_place((a.count + Tiles::ROWS - 1) / Tiles::ROWS, (b.count + Tiles::COLUMNS - 1) / Tiles::COLUMNS, splits);
    if (!at.any) return;
    Tiles t;
    t.run(lds, a, b, at.m, at.n, (int)(chunks * at.split / splits), (int)(chunks * (at.split + 1) / splits));
    constexpr int W = cbm_wide<TO>;
    t.template pieces<W>(lds, at.m, at.n, [&](int64_t r, int64_t c, float (&v)[W]) {
        if (splits > 1) {
            if (r < a.count) cbm_put<W>(parts + (at.split * a.count + r) * b.count, c, b.count, v);
        } else {
            finish<TO>(o, a.count, b.count, r, c, v);
        }
    });
}

// The shares of K of a product, added in order: four values a thread, SLICES threads for the shares of a value where values are few (100 x 512, 64 shares: 34 us with one thread, 6 with eight).
template <class TO, int SLICES>
__global__ __launch_bounds__(256) void cbm_product_join_kernel(int64_t M, int64_t N, int64_t splits, const float* __restrict__ parts, CbmProductOut o) {
    constexpr int PIECES = 256 / SLICES;
    __shared__ floatx4 room[SLICES > 1 ? SLICES : 1][PIECES];
    const int slice = threadIdx.x / PIECES, mine = threadIdx.x % PIECES;
    const uint32_t pieces = (uint32_t)((N + 3) / 4), count = (uint32_t)M * pieces;  // (few tiles: below 2^27)
    for (uint32_t i0 = blockIdx.x * PIECES; i0 < count; i0 += gridDim.x * PIECES) {
        const uint32_t i = i0 + mine;
        const int64_t r = i / pieces, c = i % pieces * 4;
        float v[4] = {};
        if (i < count && c + 4 <= N) {
            const float* p = parts + r * N + c;
#pragma unroll 4
            for (int s = slice; s < (int)splits; s += SLICES) {
                float x[4];
                load_piece<4>(x, p + s * M * N);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] += x[j];
            }
        } else if (i < count) {
            for (int s = slice; s < (int)splits; s += SLICES)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (c + j < N) v[j] += parts[(s * M + r) * N + c + j];
        }
        if constexpr (SLICES > 1) {
            room[slice][mine] = (floatx4){v[0], v[1], v[2], v[3]};
            __syncthreads();
            if (slice == 0)
#pragma unroll
                for (int s = 1; s < SLICES; ++s) {
                    const floatx4 x = room[s][mine];
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] += x[j];
                }
        }
        if (slice == 0 && i < count) finish<TO>(o, M, N, r, c, v);
        if constexpr (SLICES > 1) __syncthreads();
    }
}

// Which tiles, and how many shares of K.
struct Plan {
    int tile;  // 256 and 128: units straight to LDS; 0: 128 x 128 of any matrices
    int64_t splits;
    double us;
};
// Microseconds as measured: a workgroup's rate, by how many of a tile run at once; what a workgroup takes beside its products (the first loads, the result); shares of K are written, read and joined in a launch
// of its own.  Shares of at least 256 k.
Plan plan(int64_t M, int64_t N, int64_t K, int32_t type, int tile) {
    const int64_t side = tile ? tile : 128, tiles = std::max<int64_t>(1, (M + side - 1) / side * ((N + side - 1) / side)), at_once = tile == 256 ? 256 : 512;
    const double tflops = tile == 256 ? 1150.0 : tile == 128 ? 900.0 : type == CBM_F32 ? 140.0 : 550.0, beside = tile == 256 ? 9.0 : 5.0;
    const double each = 2.0 * (double)(side * side * K) / (tflops * 1e6 / (double)at_once);
    Plan best{tile, 1, 1e30};
    for (int64_t s = 1; s <= 128 && (s == 1 || (s * 256 <= K && tiles <= 1024)); ++s) {
        const double rounds = (double)((tiles * s + at_once - 1) / at_once);
        const double us = rounds * (each / (double)s + beside) + (s > 1 ? 4.0 + 8.0 * (double)(s * M * N) / 4e6 : 0.0);
        if (us < 0.97 * best.us) best = {tile, s, us};
    }
    return best;
}
Plan plan(int64_t M, int64_t N, int64_t K, int32_t type, bool units) {
    if (!units) return plan(M, N, K, type, 0);
    const Plan large = plan(M, N, K, type, 256), small = plan(M, N, K, type, 128);
    return large.us < small.us ? large : small;
}

template <class T, class TO, CbmTileOrder OA, CbmTileOrder OB, CbmTilePair PAIR>
void launch(const CbmProduct& p, hipStream_t stream) {
    const int64_t K = p.at ? p.at + p.K : p.K;
    const CbmOperand<T> a{{(const T*)p.A, nullptr}, {p.lda, 0}, p.M, K, 0};
    const CbmOperand<T> b{{(const T*)p.B[0], (const T*)p.B[1]}, {p.ldb[0], p.ldb[1]}, p.N, p.K, p.at};
    bool units = false;
    if constexpr (sizeof(T) == 2)
        units = cbm_units(a.p[0], a.ld[0], OA == ALONG_K ? K : p.M) && cbm_units(b.p[0], b.ld[0], OB == ALONG_K ? p.K : p.N) && (PAIR == SINGLE || (cbm_units(b.p[1], b.ld[1], p.K) && b.ld[1] == b.ld[0]));
    const Plan how = plan(p.M, p.N, K, p.type, units);
    const int64_t splits = p.parts ? how.splits : 1;
    auto run = [&](auto* tiles_type) {
        typedef std::remove_pointer_t<decltype(tiles_type)> Tiles;
        const int64_t tiles = (p.M + Tiles::ROWS - 1) / Tiles::ROWS * ((p.N + Tiles::COLUMNS - 1) / Tiles::COLUMNS), chunks = (K + Tiles::BK - 1) / Tiles::BK;
        cbm_product_kernel<Tiles, T, TO><<<(unsigned)((tiles * splits + CBM_XCD - 1) / CBM_XCD * CBM_XCD), 256, 0, stream>>>(a, b, chunks, splits, p.out, p.parts);
    };
    if (how.tile == 0) run((CbmTiles<T, 128, 128, 2, 2, OA, OB, PAIR>*)nullptr);
    if constexpr (sizeof(T) == 2) {
        if (how.tile == 128) run((CbmAlignedTiles<T, 128, 128, OA, OB, PAIR>*)nullptr);
        if (how.tile == 256) run((CbmAlignedTiles<T, 256, 256, OA, OB, PAIR>*)nullptr);
    }
    if (splits > 1) {
        const int64_t pieces = p.M * ((p.N + 3) / 4);
        auto join = [&](auto slices) {
            constexpr int SLICES = decltype(slices)::value, EACH = 256 / SLICES;
            cbm_product_join_kernel<TO, SLICES><<<(unsigned)std::min<int64_t>((pieces + EACH - 1) / EACH, 1 << 20), 256, 0, stream>>>(p.M, p.N, splits, p.parts, p.out);
        };
        if (splits >= 8 && pieces < 1 << 16) join(std::integral_constant<int, 8>{});
        else join(std::integral_constant<int, 1>{});
    }
}
template <class T, class TO>
void launch(const CbmProduct& p, hipStream_t stream) {
    if (p.at) launch<T, TO, ALONG_K, ALONG_K, PAIR_K>(p, stream);
    else if (p.a_across) launch<T, TO, ACROSS_K, ACROSS_K, SINGLE>(p, stream);
    else if (p.b_across) launch<T, TO, ALONG_K, ACROSS_K, SINGLE>(p, stream);
    else launch<T, TO, ALONG_K, ALONG_K, SINGLE>(p, stream);
}

}  // namespace

// The most that a product of the size is cut into, however its matrices lie.
int64_t cbm_product_parts(int64_t M, int64_t N, int64_t K, int32_t type) {
    const int64_t any = plan(M, N, K, type, false).splits;
    return type == CBM_F32 ? any : std::max(any, plan(M, N, K, type, true).splits);
}

int cbm_product_tile(int64_t M, int64_t N, int64_t K, int32_t type) {
    const Plan large = plan(M, N, K, type, 256), small = plan(M, N, K, type, 128);
    return large.us < small.us ? 256 : 128;
}

void cbm_launch_tiles(const CbmProduct& p, void* stream) {
    cbm_with_type(p.type, [&](auto t) {
        using T = decltype(t);
        if constexpr (std::is_same<T, float>::value) cbm_with_type(p.out.type, [&](auto to) { launch<float, decltype(to)>(p, (hipStream_t)stream); });
        else launch<T, T>(p, (hipStream_t)stream);
    });
}

cbm_status cbm_launched(const char* what) {
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return CBM_OK;
    cbm_set_error_detail(what, hipGetErrorString(e));
    return CBM_ERR_HIP;
}
