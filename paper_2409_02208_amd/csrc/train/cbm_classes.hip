// Log probabilities of labels straight from a layer's outputs and the classes' weights, Z = X W, without keeping Z, and the gradients of both.
#include <algorithm>

#include "cbm_internal.h"
#include "cbm_products.h"
#include "cbm_tiles.h"

namespace {

constexpr int BM = 128, BN = 128, WN = 2;  // WN: waves along a tile's columns, each with a partial result of its own
constexpr float LOG2E = 1.44269504f;

// m and sum exp(z - m) of two sets of scores as one
struct Sums {
    float m, s;
};
__device__ __forceinline__ Sums joined(Sums a, Sums b) {
    const float m = fmaxf(a.m, b.m), away = m == -INFINITY ? 0.0f : m;  // (NaN is in s)
    return {m, a.s * exp2f((a.m - away) * LOG2E) + b.s * exp2f((b.m - away) * LOG2E)};
}

__device__ __forceinline__ int64_t label_of(const void* labels, int bits, int64_t r) { return bits == 64 ? ((const int64_t*)labels)[r] : ((const int32_t*)labels)[r]; }

// A wave's part of each of its rows: the largest score and the sum, and the label's score where it is among them.
template <class T>
__global__ __launch_bounds__(256, 2) void cbm_classes_kernel(CbmOperand<T> a, CbmOperand<T> b, int64_t chunks, const void* __restrict__ labels, int label_bits, Sums* __restrict__ parts,
                                                          float* __restrict__ chosen) {
    typedef CbmTiles<T, BM, BN, 2, WN, ALONG_K, ACROSS_K, SINGLE> Tiles;
    __shared__ uintx4 lds[Tiles::UNITS];
    const int64_t tiles_n = (b.count + BN - 1) / BN;
    const CbmTilePlace at = cbm_tile_place((a.count + BM - 1) / BM, tiles_n, 1);
    if (!at.any) return;
    Tiles t;
    t.run(lds, a, b, at.m, at.n, 0, chunks);
    const int l32 = threadIdx.x & 31, half = threadIdx.x >> 5 & 1;
    const int64_t c0 = at.n * BN + t.first_column() + 4 * half;  // the lane's first column
#pragma unroll
    for (int i = 0; i < Tiles::TM; ++i) {
        const int64_t r = at.m * BM + t.first_row() + 32 * i + l32;
        int64_t given = labels && r < a.count ? label_of(labels, label_bits, r) : -1;
        if (given >= b.count) given = -1;
        const int label = (int)max(min(given - c0, (int64_t)4096), (int64_t)-1);
        Sums all{-INFINITY, 0.0f};
        float z = 0.0f;
        if ((at.n + 1) * BN > b.count)
#pragma unroll
            for (int j = 0; j < Tiles::TN; ++j)
#pragma unroll
                for (int v = 0; v < 16; ++v) t.acc[i][j][v] = c0 + 32 * j + 8 * (v / 4) + v % 4 < b.count ? t.acc[i][j][v] : -INFINITY;
#pragma unroll
        for (int j = 0; j < Tiles::TN; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                all.m = fmaxf(all.m, t.acc[i][j][v]);
                z = label == 32 * j + 8 * (v / 4) + v % 4 ? t.acc[i][j][v] : z;
            }
        const float away = all.m == -INFINITY ? 0.0f : all.m;
#pragma unroll
        for (int j = 0; j < Tiles::TN; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) all.s += exp2f((t.acc[i][j][v] - away) * LOG2E);
        Sums low, high;  // the halves' sums, in the same order in both
        lane_pair<32>(all.m, [&](float x, float y) { low.m = x, high.m = y; return x; });
        lane_pair<32>(all.s, [&](float x, float y) { low.s = x, high.s = y; return x; });
        all = joined(low, high);
        if (r >= a.count) continue;
        if (half == 0) parts[r * (tiles_n * WN) + at.n * WN + t.wave() / 2] = all;
        if (label >= 0 && label < 32 * Tiles::TN && !(label & 4)) chosen[r] = z;
    }
}

// A wave a row: its parts in order, a lane's 64 apart, then over the lanes.
__global__ __launch_bounds__(256) void cbm_classes_join_kernel(int64_t n, int64_t c, int64_t count, const void* __restrict__ labels, int label_bits, const Sums* __restrict__ parts,
                                                             const float* __restrict__ chosen, float* __restrict__ logp, float* __restrict__ stats) {
    const int lane = threadIdx.x & 63;
    const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (r >= n) return;
    Sums all{-INFINITY, 0.0f};
    for (int64_t i = lane; i < count; i += 64) all = joined(all, parts[r * count + i]);
    const float m = lanes_all<64>(all.m, [](float a, float b) { return fmaxf(a, b); }), away = m == -INFINITY ? 0.0f : m;
    const float s = lanes_sum<64>(all.s * exp2f((all.m - away) * LOG2E));
    if (lane) return;
    const bool bad = !(s < INFINITY);
    const float largest = bad ? NAN : m, l = bad ? NAN : logf(s);
    if (stats) {
        stats[2 * r] = largest;
        stats[2 * r + 1] = l;
    }
    if (logp) {
        const int64_t label = label_of(labels, label_bits, r);
        logp[r] = label < 0 || label >= c ? 0.0f : bad ? NAN : m == -INFINITY ? m : (chosen[r] - m) - l;
    }
}

// fp16: the gradients of a batch's scores are small beside 2^-14.  They are kept at 2^15 over the largest |dlogp| of their size, where 1 - p fits and a p down to 2^-29 keeps all its bits; what is
// made of them is multiplied by the factor, scale[0], and they by scale[1] dlogp.
__global__ __launch_bounds__(1024) void cbm_classes_scale_kernel(int64_t n, const float* __restrict__ dlogp, float* __restrict__ scale) {
    __shared__ float room[16];
    float most = 0.0f;
    for (int64_t i = threadIdx.x; i < n; i += 1024) most = fmaxf(most, fabsf(dlogp[i]));
    most = lanes_all<64>(most, [](float a, float b) { return fmaxf(a, b); });
    if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = most;
    __syncthreads();
    if (threadIdx.x) return;
    for (int i = 1; i < 16; ++i) most = fmaxf(most, room[i]);
    scale[0] = most * 0x1p-15f;
    scale[1] = most > 0.0f ? 0x1p15f / most : 0.0f;
}

// dZ of columns first .. first + b.count - 1, rounded to the type (half a step, as much as the gradients that are made of it are rounded by).
template <class T>
__global__ __launch_bounds__(256, 2) void cbm_classes_slopes_kernel(CbmOperand<T> a, CbmOperand<T> b, int64_t chunks, int64_t first, int64_t c, const void* __restrict__ labels, int label_bits,
                                                                 const float* __restrict__ stats, const float* __restrict__ dlogp, const float* __restrict__ scale, T* __restrict__ dZ,
                                                                 int64_t lddz) {
    typedef CbmTiles<T, BM, BN, 2, WN, ALONG_K, ACROSS_K, SINGLE> Tiles;
    __shared__ uintx4 lds[Tiles::UNITS];
    const CbmTilePlace at = cbm_tile_place((a.count + BM - 1) / BM, (b.count + BN - 1) / BN, 1);
    if (!at.any) return;
    Tiles t;
    t.run(lds, a, b, at.m, at.n, 0, chunks);
    const int l32 = threadIdx.x & 31, half = threadIdx.x >> 5 & 1;
#pragma unroll
    for (int i = 0; i < Tiles::TM; ++i) {
        const int64_t r = at.m * BM + t.first_row() + 32 * i + l32;
        if (r >= a.count) continue;
        int64_t label = label_of(labels, label_bits, r);
        const float m = stats[2 * r], l = stats[2 * r + 1];
        const bool none = label < 0 || label >= c || m == -INFINITY;
        float up = dlogp[r];
        if (scale) up *= scale[1];
        label -= first;
#pragma unroll
        for (int j = 0; j < Tiles::TN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int64_t col = at.n * BN + t.first_column() + 32 * j + 8 * q + 4 * half;
                float v[4];
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const float p = exp2f(((t.acc[i][j][4 * q + w] - m) - l) * LOG2E);
                    v[w] = none ? 0.0f : up * ((col + w == label ? 1.0f : 0.0f) - p);
                }
                cbm_put4<T>(dZ + r * lddz, col, b.count, v);
            }
    }
}

int64_t rounded16(int64_t bytes) { return (bytes + 15) / 16 * 16; }
int64_t bytes_of(int32_t type) { return type == CBM_F32 ? 4 : 2; }

// Columns of a piece of the classes whose dZ is kept at a time: 512 MiB, at least 1,024 columns.
int64_t piece_of(int64_t n, int32_t c, int32_t type) {
    const int64_t fit = ((int64_t)512 << 20) / (std::max<int64_t>(n, 1) * bytes_of(type)) / 128 * 128;
    return std::min<int64_t>(((int64_t)c + 7) / 8 * 8, std::max<int64_t>(fit, 1024));
}

struct Room {
    int64_t scale, sums, parts, bytes;  // where they begin; dZ is first
};
Room back_room(int64_t n, int32_t d, int32_t c, int32_t type) {
    const int64_t piece = piece_of(n, c, type), last = c % piece ? c % piece : piece;
    int64_t parts = 0;
    for (int64_t w : {piece, last}) {
        const int64_t dx = cbm_product_parts(n, d, w, type), dw = cbm_product_parts(d, w, n, type);
        if (dx > 1) parts = std::max(parts, dx * n * d);
        if (dw > 1) parts = std::max(parts, dw * d * w);
    }
    Room r;
    r.scale = rounded16(n * piece * bytes_of(type));
    r.sums = r.scale + 16;
    r.parts = r.sums + (piece < c ? rounded16(4 * n * d) : 0);
    r.bytes = r.parts + 4 * parts;
    return r;
}

template <class T>
int64_t chunks_of(int64_t k) {
    const int64_t chunk = 8 * CbmTileType<T>::KG;
    return (k + chunk - 1) / chunk;
}
unsigned grid_of(int64_t n, int64_t c) {
    const int64_t tiles = (n + BM - 1) / BM * ((c + BN - 1) / BN);
    return (unsigned)((tiles + CBM_XCD - 1) / CBM_XCD * CBM_XCD);
}

}  // namespace

int64_t cbm_classes_workspace(int64_t n, int32_t, int32_t c, int32_t) { return rounded16(n * (((int64_t)c + BN - 1) / BN) * WN * (int64_t)sizeof(Sums)) + 4 * n; }

cbm_status cbm_launch_classes(int64_t n, int32_t d, int32_t c, int32_t type, const void* X, int64_t ldx, const void* W, int64_t ldw, const void* labels, int label_bits, float* logp, float* stats,
                              void* workspace, void* stream_) {
    hipStream_t stream = (hipStream_t)stream_;
    if (n == 0) return CBM_OK;
    const int64_t count = ((int64_t)c + BN - 1) / BN * WN;
    Sums* parts = (Sums*)workspace;
    float* chosen = (float*)((char*)workspace + rounded16(n * count * (int64_t)sizeof(Sums)));
    cbm_with_type(type, [&](auto t) {
        using T = decltype(t);
        const CbmOperand<T> a{{(const T*)X, nullptr}, {ldx, 0}, n, d, 0}, b{{(const T*)W, nullptr}, {ldw, 0}, c, d, 0};
        cbm_classes_kernel<T><<<grid_of(n, c), 256, 0, stream>>>(a, b, chunks_of<T>(d), logp ? labels : nullptr, label_bits, parts, chosen);
    });
    cbm_classes_join_kernel<<<(unsigned)((n + 3) / 4), 256, 0, stream>>>(n, c, count, labels, label_bits, parts, chosen, logp, stats);
    return cbm_launched("linear log probabilities launch");
}

int64_t cbm_classes_back_workspace(int64_t n, int32_t d, int32_t c, int32_t type) { return back_room(n, d, c, type).bytes; }

cbm_status cbm_launch_classes_backward(int64_t n, int32_t d, int32_t c, int32_t type, const void* X, int64_t ldx, const void* W, int64_t ldw, const void* labels, int label_bits,
                                       const float* stats, const float* dlogp, void* dX, int64_t lddx, void* dW, int64_t lddw, void* workspace, void* stream_) {
    hipStream_t stream = (hipStream_t)stream_;
    const Room room = back_room(n, d, c, type);
    const int64_t piece = piece_of(n, c, type), bytes = bytes_of(type);
    float *scale = (float*)((char*)workspace + room.scale), *sums = (float*)((char*)workspace + room.sums), *parts = (float*)((char*)workspace + room.parts);
    if (type != CBM_F16) scale = nullptr;
    if (scale && n > 0) cbm_classes_scale_kernel<<<1, 1024, 0, stream>>>(n, dlogp, scale);
    for (int64_t first = 0; first < c; first += piece) {
        const int64_t width = std::min<int64_t>(piece, c - first);
        const void* Wp = (const char*)W + first * bytes;
        if (n > 0)
            cbm_with_type(type, [&](auto t) {
                using T = decltype(t);
                const CbmOperand<T> a{{(const T*)X, nullptr}, {ldx, 0}, n, d, 0}, b{{(const T*)Wp, nullptr}, {ldw, 0}, width, d, 0};
                cbm_classes_slopes_kernel<T><<<grid_of(n, width), 256, 0, stream>>>(a, b, chunks_of<T>(d), first, c, labels, label_bits, stats, dlogp, scale, (T*)workspace, piece);
            });
        CbmProduct p{};
        p.type = p.out.type = type;
        p.out.alpha = 1.0f;
        p.out.factor = n > 0 ? scale : nullptr;
        p.A = workspace;
        p.lda = piece;
        if (dX && n > 0) {
            p.M = n;
            p.N = d;
            p.K = width;
            p.B[0] = Wp;
            p.ldb[0] = ldw;
            p.out.C[0] = dX;
            p.out.ldc[0] = lddx;
            p.out.columns = d;
            p.out.sums = piece < c ? sums : nullptr;
            p.out.first = first == 0;
            p.out.last = first + piece >= c;
            p.parts = cbm_product_parts(n, d, width, type) > 1 ? parts : nullptr;
            cbm_launch_tiles(p, stream);
        }
        if (dW) {
            p.M = d;
            p.N = width;
            p.K = n;
            p.A = X;
            p.lda = ldx;
            p.a_across = p.b_across = true;
            p.B[0] = workspace;
            p.ldb[0] = piece;
            p.out.C[0] = (char*)dW + first * bytes;
            p.out.ldc[0] = lddw;
            p.out.columns = width;
            p.out.sums = nullptr;
            p.parts = cbm_product_parts(d, width, n, type) > 1 ? parts : nullptr;
            cbm_launch_tiles(p, stream);
        }
    }
    return cbm_launched("linear log probabilities backward launch");
}
