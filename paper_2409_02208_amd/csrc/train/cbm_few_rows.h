// Products of a few rows with large matrices, which are bound by reading those once: every lane has 16 bytes of a row of W at a time and its sums in fp32, no matrix cores.  (1 x 1024 with 1024 x 32000 in bf16: tiles
// of 128 x 128 23.8 us with the joining launch, this 17.8; 1 x 1024 with two of 1024 x 4096 18.4, 7.7.)
#pragma once

#include "cbm_elems.h"

// NR rows of X, MATS matrices, a workgroup of WAVES waves for CL pieces of 16 bytes of W's columns; a wave has 64 / CL rows of W at a time.
template <class T, int NR, int MATS, int CL, int WAVES>
struct CbmFewRows {
    static constexpr int V = 16 / (int)sizeof(T), COLS = CL * V, RL = 64 / CL, STEP = RL * WAVES, AHEAD = NR * MATS >= 8 ? 2 : NR * MATS == 1 ? 8 : 4;
    typedef float Room[WAVES][MATS][NR][COLS];  // of each wave, in LDS
    static_assert(CL == 4 || CL == 8, "");

    // The sums of columns `first` .. first + COLS - 1 (of those there are), each wave's share of K; W has at least V columns.
    static __device__ __forceinline__ void run(Room& room, const T* __restrict__ X, int64_t ldx, int64_t n, int64_t K, const T* const (&W)[MATS], const int64_t (&ldw)[MATS], int64_t columns, int64_t first) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const int64_t c = first + lane % CL * V, at = min(c, columns - V);  // (the last piece starts early, and keeps what is its own)
        float sum[MATS][NR][V];
#pragma unroll
        for (int m = 0; m < MATS; ++m)
#pragma unroll
            for (int r = 0; r < NR; ++r)
#pragma unroll
                for (int j = 0; j < V; ++j) sum[m][r][j] = 0.0f;
        const T* x[NR];
#pragma unroll
        for (int r = 0; r < NR; ++r) x[r] = X + min((int64_t)r, n - 1) * ldx;
        int64_t k = wave * RL + lane / CL;
        auto some = [&](auto count) {
            constexpr int COUNT = decltype(count)::value;
            typename Piece<T, V>::type w[COUNT][MATS];
            float v[COUNT][NR];
#pragma unroll
            for (int i = 0; i < COUNT; ++i) {
#pragma unroll
                for (int m = 0; m < MATS; ++m) w[i][m] = raw_piece<V>(W[m] + (k + i * STEP) * ldw[m] + at);
#pragma unroll
                for (int r = 0; r < NR; ++r) v[i][r] = (float)x[r][k + i * STEP];
            }
#pragma unroll
            for (int i = 0; i < COUNT; ++i)
#pragma unroll
                for (int m = 0; m < MATS; ++m)
#pragma unroll
                    for (int j = 0; j < V; ++j)
#pragma unroll
                        for (int r = 0; r < NR; ++r) sum[m][r][j] = fmaf((float)w[i][m][j], v[i][r], sum[m][r][j]);
            k += COUNT * STEP;
        };
        while (k + (AHEAD - 1) * STEP < K) some(std::integral_constant<int, AHEAD>{});
        while (k < K) some(std::integral_constant<int, 1>{});
#pragma unroll
        for (int m = 0; m < MATS; ++m)
#pragma unroll
            for (int r = 0; r < NR; ++r)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    auto add = [](float a, float b) { return a + b; };
                    float s = sum[m][r][j];  // over the wave's rows of W: rotations of 8 and 4 lanes in sixteen, then across
                    s += __uint_as_float(lane_moved<0x128>(__float_as_uint(s)));
                    if constexpr (CL == 4) s += __uint_as_float(lane_moved<0x124>(__float_as_uint(s)));
                    s = lane_pair<32>(lane_pair<16>(s, add), add);
                    if (lane < CL && at + j >= c) room[wave][m][r][at + j - first] = s;
                }
        __syncthreads();
    }
    static __device__ __forceinline__ float total(const Room& room, int m, int r, int column) {
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) s += room[w][m][r][column];
        return s;
    }
};
constexpr int64_t CBM_FEW_ROWS = 8;  // at a time
// Up to so many rows altogether: in fp32, where tiles are slower, 32 (with 1024 x 4096 twice, 16 rows: tiles 62 us, 8 rows here 10).
template <class T>
constexpr int64_t cbm_most_few_rows = sizeof(T) == 4 ? 4 * CBM_FEW_ROWS : CBM_FEW_ROWS;

// The piece of columns of workgroup b of a grid of a multiple of 8: neighbours on one XCD (b mod 8), which halves of a line of 128 bytes then reach once (1 x 4096 with two of 4096 x 8192 40 -> 25 us).
__device__ __forceinline__ int64_t cbm_few_piece() { return (int64_t)(blockIdx.x % 8) * (gridDim.x / 8) + blockIdx.x / 8; }

// f(2, 4 or 8 rows at most, or one)
template <class F>
inline void cbm_with_few_rows(int64_t n, F&& f) {
    using std::integral_constant;
    if (n == 1) f(integral_constant<int, 1>{});
    else if (n == 2) f(integral_constant<int, 2>{});
    else if (n <= 4) f(integral_constant<int, 4>{});
    else f(integral_constant<int, 8>{});
}
