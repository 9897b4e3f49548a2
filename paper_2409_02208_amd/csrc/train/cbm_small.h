// Small products: a workgroup makes 32 x 32 values of the result, and its eight waves share K, so that few rows and columns with a long K fill the device too.  The operands come straight from the caches
// into registers, in whatever order and at whatever alignment their matrices lie; 16-bit values are multiplied as they are, everything else in fp32 by fp32 matrix instructions, which keep slopes that are
// only made to be multiplied once more in 32 bits.  (128 x 512 with 512 x 512 classes, gradients, bf16: 29 us in tiles of 128, 14 here; bound by the latency of its loads and by three launches.)
#pragma once

#include "cbm_products.h"
#include "cbm_tiles.h"

template <class TA, class TB, CbmTileOrder ORDER_A, CbmTileOrder ORDER_B, int MATS>
struct CbmSmallTile {
    static constexpr bool SHORT = sizeof(TA) == 2 && sizeof(TB) == 2;
    static constexpr int WAVES = 8, THREADS = 64 * WAVES, SIDE = 32, STRIDE = SIDE + 4, AHEAD = SHORT ? 4 : 2;
    typedef float Room[WAVES][MATS][SIDE * STRIDE];  // of each wave, in LDS
    template <class S>
    struct Eight {
        typename Piece<S, 8>::type v;
    };
    // eight k of a row, from k on; zeros beyond K
    template <CbmTileOrder ORDER, class S>
    static __device__ __forceinline__ Eight<S> eight(const S* p, int64_t ld, int64_t r, int64_t k, int64_t K) {
        Eight<S> e;
        if (ORDER == ALONG_K && k + 8 <= K) {
            e.v = raw_piece<8>(p + r * ld + k);
        } else if (k + 8 <= K) {
            const S* q = p + k * ld + r;
#pragma unroll
            for (int i = 0; i < 8; ++i) e.v[i] = q[i * ld];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int64_t at = min(k + i, K - 1);
                const S x = ORDER == ALONG_K ? p[r * ld + at] : p[at * ld + r];
                e.v[i] = k + i < K ? x : (S)0.0f;
            }
        }
        return e;
    }
    floatx16 acc[MATS];

    __device__ __forceinline__ CbmSmallTile() {
#pragma unroll
        for (int m = 0; m < MATS; ++m)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[m][v] = 0.0f;
    }
    // adds A . B[m], rows r0 and columns c0 on; of the rows and columns that there are
    __device__ __forceinline__ void add(const TA* A, int64_t lda, int64_t rows, int64_t r0, const TB* const (&B)[MATS], const int64_t (&ldb)[MATS], int64_t columns, int64_t c0, int64_t K) {
        const int lane = threadIdx.x & 63, half = lane >> 5;
        const int64_t r = min(r0 + (lane & 31), rows - 1), c = min(c0 + (lane & 31), columns - 1);
        int64_t k = 16 * (int64_t)(threadIdx.x >> 6);
        auto some = [&](auto count) {
            constexpr int COUNT = decltype(count)::value;
            Eight<TA> x[COUNT];
            Eight<TB> y[COUNT][MATS];
#pragma unroll
            for (int i = 0; i < COUNT; ++i) {
                const int64_t at = k + 16 * WAVES * i + 8 * half;
                x[i] = eight<ORDER_A>(A, lda, r, at, K);
#pragma unroll
                for (int m = 0; m < MATS; ++m) y[i][m] = eight<ORDER_B>(B[m], ldb[m], c, at, K);
            }
#pragma unroll
            for (int i = 0; i < COUNT; ++i)
#pragma unroll
                for (int m = 0; m < MATS; ++m)
                    if constexpr (SHORT) {
                        acc[m] = cbm_multiply<TA>(__builtin_bit_cast(uintx4, y[i][m].v), __builtin_bit_cast(uintx4, x[i].v), acc[m]);
                    } else {
#pragma unroll
                        for (int j = 0; j < 8; ++j) acc[m] = __builtin_amdgcn_mfma_f32_32x32x2f32((float)y[i][m].v[j], (float)x[i].v[j], acc[m], 0, 0, 0);
                    }
            k += 16 * WAVES * COUNT;
        };
        while (k + 16 * WAVES * (AHEAD - 1) < K) some(std::integral_constant<int, AHEAD>{});
        while (k < K) some(std::integral_constant<int, 1>{});
    }
    // a thread has two neighbouring values of the sums of each matrix: row() and column() on
    static __device__ __forceinline__ int row() { return threadIdx.x / 16; }
    static __device__ __forceinline__ int column() { return threadIdx.x % 16 * 2; }
    __device__ __forceinline__ void share(Room& room) const {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
        for (int m = 0; m < MATS; ++m)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *(floatx4*)&room[wave][m][(lane & 31) * STRIDE + 8 * q + 4 * (lane >> 5)] = (floatx4){acc[m][4 * q], acc[m][4 * q + 1], acc[m][4 * q + 2], acc[m][4 * q + 3]};
        __syncthreads();
    }
    static __device__ __forceinline__ void total(const Room& room, int m, float (&v)[2]) {
        v[0] = v[1] = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w)
#pragma unroll
            for (int j = 0; j < 2; ++j) v[j] += room[w][m][row() * STRIDE + column() + j];
    }
};
