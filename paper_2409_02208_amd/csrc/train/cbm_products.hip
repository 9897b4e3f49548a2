// Products in tiles with a plain end: sums added to, scaled and rounded.  The gradients of the operators that are made of products.
#include <algorithm>
#include <type_traits>

#include "cbm_aligned.h"
#include "cbm_internal.h"
#include "cbm_products.h"
#include "cbm_small.h"

namespace {

template <class T, int W>
__device__ __forceinline__ void finish(const CbmProductOut& o, int64_t N, int64_t r, int64_t c, float (&v)[W]) {
    if (r >= o.rows || c >= N) return;
    if (o.sums) {
        float* s = o.sums + r * N + c;
        if (!o.first)
#pragma unroll
            for (int j = 0; j < W; ++j)
                if (c + j < N) v[j] += s[j];
        if (!o.last) return cbm_put<W>(o.sums + r * N, c, N, v);
    }
    if (o.factor) {
        const float up = *o.factor;
#pragma unroll
        for (int j = 0; j < W; ++j) v[j] *= up;
    }
    const bool second = o.at && c >= o.at;
    if (second) c -= o.at;
    if (o.C[second]) cbm_put((T*)o.C[second] + r * o.ldc[second], c, o.columns, v);
}

template <class Tiles, class T>
__global__ __launch_bounds__(256, Tiles::GROUPS) void cbm_product_kernel(CbmOperand<T> a, CbmOperand<T> b, int64_t chunks, int64_t splits, CbmProductOut o, float* __restrict__ parts) {
    __shared__ uintx4 lds[Tiles::UNITS];
    const CbmTilePlace at = cbm_tile_place((a.count + Tiles::ROWS - 1) / Tiles::ROWS, (b.count + Tiles::COLUMNS - 1) / Tiles::COLUMNS, splits);
    if (!at.any) return;
    Tiles t;
    t.run(lds, a, b, at.m, at.n, (int)(chunks * at.split / splits), (int)(chunks * (at.split + 1) / splits));
    constexpr int W = cbm_wide<T>;
    t.template pieces<W>(lds, at.m, at.n, [&](int64_t r, int64_t c, float (&v)[W]) {
        if (splits > 1) {
            if (r < a.count) cbm_put<W>(parts + (at.split * a.count + r) * b.count, c, b.count, v);
        } else {
            finish<T>(o, b.count, r, c, v);
        }
    });
}

// The shares of K of a product, added in order: four values a thread, SLICES threads for the shares of a value where values are few (100 x 512, 64 shares: 34 us with one thread, 6 with eight).
template <class T, int SLICES>
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
        if (slice == 0 && i < count) finish<T>(o, N, r, c, v);
        if constexpr (SLICES > 1) __syncthreads();
    }
}

template <class T>
__global__ __launch_bounds__(512) void cbm_small_along_kernel(int64_t M, int64_t N, int64_t K, const float* __restrict__ S0, const float* __restrict__ S1, int64_t lds, const T* __restrict__ B0, int64_t ldb0,
                                                            const T* __restrict__ B1, int64_t ldb1, T* __restrict__ C, int64_t ldc) {
    typedef CbmSmallTile<float, T, ALONG_K, ALONG_K, 1> Tile;
    __shared__ typename Tile::Room room;
    const int64_t r0 = (int64_t)blockIdx.y * Tile::SIDE, c0 = (int64_t)blockIdx.x * Tile::SIDE, r = r0 + Tile::row();
    Tile t;
    t.add(S0, lds, M, r0, {B0}, {ldb0}, N, c0, K);
    if (S1) t.add(S1, lds, M, r0, {B1}, {ldb1}, N, c0, K);
    t.share(room);
    float v[2];
    Tile::total(room, 0, v);
    if (r < M) cbm_put(C + r * ldc, c0 + Tile::column(), N, v);
}
template <class T>
__global__ __launch_bounds__(512) void cbm_small_across_kernel(int64_t M, int64_t N, int64_t K, const T* __restrict__ A, int64_t lda, const float* __restrict__ S0, const float* __restrict__ S1, int64_t lds,
                                                             T* __restrict__ C0, int64_t ldc0, T* __restrict__ C1, int64_t ldc1) {
    typedef CbmSmallTile<T, float, ACROSS_K, ACROSS_K, 1> Tile;
    __shared__ typename Tile::Room room;
    const bool second = !C0 || blockIdx.z;
    const int64_t r0 = (int64_t)blockIdx.y * Tile::SIDE, c0 = (int64_t)blockIdx.x * Tile::SIDE, r = r0 + Tile::row();
    Tile t;
    t.add(A, lda, M, r0, {second ? S1 : S0}, {lds}, N, c0, K);
    t.share(room);
    float v[2];
    Tile::total(room, 0, v);
    if (r < M) cbm_put(second ? C1 + r * ldc1 : C0 + r * ldc0, c0 + Tile::column(), N, v);
}

// 64 x 64 values a workgroup, through LDS.
__global__ __launch_bounds__(256) void cbm_pack_kernel(const uint16_t* __restrict__ from, int64_t ld, int64_t rows, int64_t columns, bool turned, uint16_t* __restrict__ to, int64_t ldt, int64_t blocks,
                                                     int64_t at) {
    __shared__ uint16_t room[64][66];  // [row][column]
    typedef uint16_t Four __attribute__((ext_vector_type(4), aligned(2)));
    const int64_t r0 = (int64_t)blockIdx.y * 64, c0 = (int64_t)blockIdx.x * 64;
    const int64_t high = turned ? columns : rows, wide = turned ? rows : columns, h0 = turned ? c0 : r0, w0 = turned ? r0 : c0;  // as `from` lies
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int h = threadIdx.x / 16 + 16 * i, w = threadIdx.x % 16 * 4;
        uint16_t v[4] = {};
        if (h0 + h < high) {
            const uint16_t* p = from + (h0 + h) * ld + w0 + w;
            if (w0 + w + 4 <= wide) {
                const Four x = *reinterpret_cast<const Four*>(p);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = x[j];
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (w0 + w + j < wide) v[j] = p[j];
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) (turned ? room[w + j][h] : room[h][w + j]) = v[j];
    }
    __syncthreads();
    typedef uint16_t Eight __attribute__((ext_vector_type(8)));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int r = threadIdx.x / 8 + 32 * i, c = threadIdx.x % 8 * 8;
        if (r0 + r >= (rows + 7) / 8 * 8 || c0 + c >= ldt) continue;
        Eight v;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = room[r][c + j];
        const int64_t row = r0 + r, out = blocks ? row / 32 * blocks + row % 32 + at : row;
        *reinterpret_cast<Eight*>(to + out * ldt + c0 + c) = v;
    }
}

template <class T, CbmTileOrder OA, CbmTileOrder OB, CbmTilePair PAIR>
void launch(const CbmProduct& p, hipStream_t stream) {
    const int64_t K = p.at ? p.at + p.K : p.K;
    const CbmOperand<T> a{{(const T*)p.A, nullptr}, {p.lda, 0}, p.M, K, 0};
    const CbmOperand<T> b{{(const T*)p.B[0], (const T*)p.B[1]}, {p.ldb[0], p.ldb[1]}, p.N, p.K, p.at};
    bool units = false;
    if constexpr (sizeof(T) == 2)
        units = cbm_units(a.p[0], a.ld[0], OA == ALONG_K ? K : p.M) && cbm_units(b.p[0], b.ld[0], OB == ALONG_K ? p.K : p.N) && (PAIR == SINGLE || (cbm_units(b.p[1], b.ld[1], p.K) && b.ld[1] == b.ld[0]));
    const CbmPlan how = cbm_plan(p.M, p.N, p.at ? 2 * p.at : K, p.type, units);
    const int64_t splits = p.parts ? how.splits : 1;
    CbmProductOut out = p.out;
    if (!out.rows) out.rows = p.M;
    auto run = [&](auto* tiles_type) {
        typedef std::remove_pointer_t<decltype(tiles_type)> Tiles;
        const int64_t tiles = (p.M + Tiles::ROWS - 1) / Tiles::ROWS * ((p.N + Tiles::COLUMNS - 1) / Tiles::COLUMNS), chunks = (K + Tiles::BK - 1) / Tiles::BK;
        cbm_product_kernel<Tiles, T><<<(unsigned)((tiles * splits + CBM_XCD - 1) / CBM_XCD * CBM_XCD), 256, 0, stream>>>(a, b, chunks, splits, out, p.parts);
    };
    if constexpr (sizeof(T) == 4)
        if (cbm_is_narrow(p.N, p.type)) run((CbmTiles<T, OA == ALONG_K ? 256 : 128, 64, OA == ALONG_K ? 4 : 2, OA == ALONG_K ? 1 : 2, OA, OB, PAIR>*)nullptr);  // (registers)
    if (how.tile == 0 && !cbm_is_narrow(p.N, p.type)) run((CbmTiles<T, 128, 128, 2, 2, OA, OB, PAIR>*)nullptr);
    if constexpr (sizeof(T) == 2) {
        if (how.tile == 128) run((CbmAlignedTiles<T, 128, 128, OA, OB, PAIR>*)nullptr);
        if (how.tile == 256) run((CbmAlignedTiles<T, 256, 256, OA, OB, PAIR>*)nullptr);
    }
    if (splits > 1) {
        const int64_t pieces = p.M * ((p.N + 3) / 4);
        auto join = [&](auto slices) {
            constexpr int SLICES = decltype(slices)::value, EACH = 256 / SLICES;
            cbm_product_join_kernel<T, SLICES><<<(unsigned)std::min<int64_t>((pieces + EACH - 1) / EACH, 1 << 20), 256, 0, stream>>>(p.M, p.N, splits, p.parts, out);
        };
        if (splits >= 8 && pieces < 1 << 16) join(std::integral_constant<int, 8>{});
        else join(std::integral_constant<int, 1>{});
    }
}
template <class T>
void launch(const CbmProduct& p, hipStream_t stream) {
    if (p.at) launch<T, ALONG_K, ALONG_K, PAIR_K>(p, stream);
    else if (p.a_across) launch<T, ACROSS_K, ACROSS_K, SINGLE>(p, stream);
    else if (p.b_across) launch<T, ALONG_K, ACROSS_K, SINGLE>(p, stream);
    else launch<T, ALONG_K, ALONG_K, SINGLE>(p, stream);
}

}  // namespace

void cbm_launch_pack(const void* from, int64_t ld, int64_t rows, int64_t columns, bool turned, void* to, int64_t ldt, int64_t blocks, int64_t at, void* stream) {
    // (a grid is 65,535 high at most)
    for (int64_t r = 0; r < rows; r += 4194240) {  // (a multiple of 64)
        const int64_t some = std::min<int64_t>(rows - r, 4194240);
        cbm_pack_kernel<<<dim3((unsigned)((ldt + 63) / 64), (unsigned)((some + 63) / 64)), 256, 0, (hipStream_t)stream>>>((const uint16_t*)from + (turned ? r : r * ld), ld, some, columns, turned,
                                                                                                                (uint16_t*)to + (blocks ? r / 32 * blocks : r) * ldt, ldt, blocks, at);
    }
}

void cbm_launch_tiles(const CbmProduct& p, void* stream) {
    cbm_with_type(p.type, [&](auto t) { launch<decltype(t)>(p, (hipStream_t)stream); });
}

void cbm_launch_small_along(int32_t type, int64_t M, int64_t N, int64_t K, const float* S0, const float* S1, int64_t lds, const void* B0, int64_t ldb0, const void* B1, int64_t ldb1, void* C, int64_t ldc,
                            void* stream) {
    cbm_with_type(type, [&](auto t) {
        using T = decltype(t);
        cbm_small_along_kernel<T><<<dim3((unsigned)((N + 31) / 32), (unsigned)((M + 31) / 32)), 512, 0, (hipStream_t)stream>>>(M, N, K, S0, S1, lds, (const T*)B0, ldb0, (const T*)B1, ldb1, (T*)C, ldc);
    });
}

void cbm_launch_small_across(int32_t type, int64_t M, int64_t N, int64_t K, const void* A, int64_t lda, const float* S0, const float* S1, int64_t lds, void* C0, int64_t ldc0, void* C1, int64_t ldc1,
                             void* stream) {
    cbm_with_type(type, [&](auto t) {
        using T = decltype(t);
        cbm_small_across_kernel<T><<<dim3((unsigned)((N + 31) / 32), (unsigned)((M + 31) / 32), C0 && C1 ? 2 : 1), 512, 0, (hipStream_t)stream>>>(M, N, K, (const T*)A, lda, S0, S1, lds, (T*)C0, ldc0,
                                                                                                                                       (T*)C1, ldc1);
    });
}

cbm_status cbm_launched(const char* what) {
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return CBM_OK;
    cbm_set_error_detail(what, hipGetErrorString(e));
    return CBM_ERR_HIP;
}
