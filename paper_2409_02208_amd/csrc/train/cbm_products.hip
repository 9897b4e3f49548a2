// Products in tiles with a plain end: sums scaled, added to and rounded.  The gradients of the operators that are made of products, and the steps of the orthogonal update.
#include <algorithm>

#include "cbm_internal.h"
#include "cbm_products.h"
#include "cbm_tiles.h"

namespace {

constexpr int BM = 128, BN = 128;

template <class TO>
__device__ __forceinline__ void finish(const CbmProductOut& o, int64_t M, int64_t N, int64_t r, int64_t c, float (&v)[4]) {
    if (r >= M || c >= N) return;
    if (o.sums) {
        float* s = o.sums + r * N + c;
        if (!o.first)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c + j < N) v[j] += s[j];
        if (!o.last) return cbm_put4<float>(o.sums + r * N, c, N, v);
    }
    float up = o.alpha;
    if (o.factor) up *= *o.factor;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] *= up;
    if (o.more)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (c + j < N) v[j] = fmaf(o.beta, o.more[r * o.ldm + c + j], v[j]);
    const bool second = o.at && c >= o.at;
    if (second) c -= o.at;
    TO* C = (TO*)o.C[second];
    const int64_t ld = o.ldc[second];
    if (!C) return;
    if (o.transposed) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (c + j < o.columns) C[(c + j) * ld + r] = (TO)v[j];
    } else {
        cbm_put4<TO>(C + r * ld, c, o.columns, v);
    }
}

template <class T, class TO, CbmTileOrder OA, CbmTileOrder OB, CbmTilePair PAIR>
__global__ __launch_bounds__(256, 2) void cbm_product_kernel(CbmOperand<T> a, CbmOperand<T> b, int64_t chunks, int64_t splits, CbmProductOut o, float* __restrict__ parts) {
    typedef CbmTiles<T, BM, BN, 2, 2, OA, OB, PAIR> Tiles;
    __shared__ uintx4 lds[Tiles::UNITS];
    const CbmTilePlace at = cbm_tile_place((a.count + BM - 1) / BM, (b.count + BN - 1) / BN, splits);
    if (!at.any) return;
    Tiles t;
    t.run(lds, a, b, at.m, at.n, chunks * at.split / splits, chunks * (at.split + 1) / splits);
    t.pieces(at.m, at.n, [&](int64_t r, int64_t c, const float (&s)[4]) {
        float v[4] = {s[0], s[1], s[2], s[3]};
        if (splits > 1) {
            if (r < a.count) cbm_put4<float>(parts + (at.split * a.count + r) * b.count, c, b.count, v);
        } else {
            finish<TO>(o, a.count, b.count, r, c, v);
        }
    });
}

// The shares of K of a product, added in order.
template <class TO>
__global__ __launch_bounds__(256) void cbm_product_join_kernel(int64_t M, int64_t N, int64_t splits, const float* __restrict__ parts, CbmProductOut o) {
    const int64_t pieces = (N + 3) / 4;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < M * pieces; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / pieces, c = i % pieces * 4;
        float v[4] = {};
        for (int64_t s = 0; s < splits; ++s) {
            const float* p = parts + (s * M + r) * N + c;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c + j < N) v[j] += p[j];
        }
        finish<TO>(o, M, N, r, c, v);
    }
}

int64_t chunk(int32_t type) { return type == CBM_F32 ? 32 : 64; }

template <class T, class TO>
void launch(const CbmProduct& p, hipStream_t stream) {
    const int64_t chunks = p.at ? (p.at + p.K + chunk(p.type) - 1) / chunk(p.type) : (p.K + chunk(p.type) - 1) / chunk(p.type);
    const int64_t tiles = (p.M + BM - 1) / BM * ((p.N + BN - 1) / BN), splits = p.parts ? cbm_product_parts(p.M, p.N, p.at ? p.at + p.K : p.K, p.type) : 1;
    const CbmOperand<T> a{{(const T*)p.A, nullptr}, {p.lda, 0}, p.M, p.at ? p.at + p.K : p.K, 0};
    const CbmOperand<T> b{{(const T*)p.B[0], (const T*)p.B[1]}, {p.ldb[0], p.ldb[1]}, p.N, p.K, p.at};
    const unsigned grid = (unsigned)((tiles * splits + CBM_XCD - 1) / CBM_XCD * CBM_XCD);
    if (p.at) cbm_product_kernel<T, TO, ALONG_K, ALONG_K, PAIR_K><<<grid, 256, 0, stream>>>(a, b, chunks, splits, p.out, p.parts);
    else if (p.a_across) cbm_product_kernel<T, TO, ACROSS_K, ACROSS_K, SINGLE><<<grid, 256, 0, stream>>>(a, b, chunks, splits, p.out, p.parts);
    else if (p.b_across) cbm_product_kernel<T, TO, ALONG_K, ACROSS_K, SINGLE><<<grid, 256, 0, stream>>>(a, b, chunks, splits, p.out, p.parts);
    else cbm_product_kernel<T, TO, ALONG_K, ALONG_K, SINGLE><<<grid, 256, 0, stream>>>(a, b, chunks, splits, p.out, p.parts);
    if (splits > 1) {
        const int64_t blocks = (p.M * ((p.N + 3) / 4) + 255) / 256;
        cbm_product_join_kernel<TO><<<(unsigned)std::min<int64_t>(blocks, 1 << 20), 256, 0, stream>>>(p.M, p.N, splits, p.parts, p.out);
    }
}

}  // namespace

// Few tiles share K so that the compute units have work, each share at least 512 k.
int64_t cbm_product_parts(int64_t M, int64_t N, int64_t K, int32_t type) {
    const int64_t tiles = std::max<int64_t>(1, (M + BM - 1) / BM * ((N + BN - 1) / BN)), most = K / 512;
    return std::max<int64_t>(1, std::min(most, 512 / tiles));
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
