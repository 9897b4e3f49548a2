// Which kernel a product is made by, and in how many shares: rules on sizes and types (host code, no GPU needed).
#pragma once

#include <algorithm>
#include <cstdint>

#include "cbm.h"

// A launch has fewer than 2^32 threads, 256 for each tile of 128 x 128 values or larger, in a grid of a multiple of eight.
inline bool cbm_too_many_tiles(int64_t rows, int64_t columns) { return ((rows + 127) / 128 * ((columns + 127) / 128) + 7) / 8 * 8 >= (int64_t)1 << 24; }
// Large products of 16-bit values: matrices that do not lie in whole units of 16 bytes are copied so that they do, and a matrix whose rows of k many rows of the other meet is turned to lie along k; their
// workspace has room for it.  (us as they lie / copied, forward and backward, odd strides: 100000 x 1001 with 2 x 1001 columns 777 / 675 and 1447 / 1326; 16384 x 333 with 2 x 500 38 / 47, 105 / 108;
// 1024 x 1000 with 2 x 4000 37 / 48, 105 / 104.  Turned: 65536 x 1024 with 2 x 4096 1342 / 1218.)  A copy's row is shorter than 2^22 values, as that of any matrix whose units go straight to LDS (cbm_units).
inline bool cbm_may_pack(int64_t rows, int64_t K, int64_t columns, int32_t type) { return type != CBM_F32 && rows >= 1024 && K >= 256 && K <= (1 << 22) - 8 && 2e-11 * (double)rows * (double)K * (double)columns >= 1.0; }
constexpr int64_t CBM_TURN_ROWS = 4096;  // from so many rows on turning pays
inline int64_t cbm_whole(int64_t v, int64_t of) { return (v + of - 1) / of * of; }
// fp32 with so few columns: tiles of 256 x 64, which waste half as much as those of 128 x 128.
inline bool cbm_is_narrow(int64_t columns, int32_t type) { return type == CBM_F32 && columns <= 64; }
// Which tiles, and how many shares of K.
struct CbmPlan {
    int tile;  // 256 and 128: units straight to LDS; 0: 128 x 128 of any matrices
    int64_t splits;
    double us;
};
// Microseconds as measured: a workgroup's rate, by how many of a tile run at once; what a workgroup takes beside its products (the first loads, the result); shares of K are written, read and joined in a launch
// of its own.  Shares of at least 256 k.
inline CbmPlan cbm_plan(int64_t M, int64_t N, int64_t K, int32_t type, int tile) {
    M = cbm_whole(M, 8), N = cbm_whole(N, 8), K = cbm_whole(K, 64);  // (a copy in whole units has the same plan)
    const bool narrow = !tile && cbm_is_narrow(N, type);
    const int64_t side = tile ? tile : 128, tiles = std::max<int64_t>(1, narrow ? (M + 255) / 256 : (M + side - 1) / side * ((N + side - 1) / side)), at_once = tile == 256 ? 256 : 512;
    const double tflops = tile == 256 ? 1150.0 : tile == 128 ? 900.0 : type == CBM_F32 ? 140.0 : 550.0, beside = tile == 256 ? 9.0 : 5.0;
    const double each = 2.0 * (double)(side * side * K) / (tflops * 1e6 / (double)at_once);
    CbmPlan best{tile, 1, 1e30};
    for (int64_t s = 1; s <= 128 && (s == 1 || (s * 256 <= K && tiles <= 1024)); ++s) {
        const double rounds = (double)((tiles * s + at_once - 1) / at_once);
        const double us = rounds * (each / (double)s + beside) + (s > 1 ? 4.0 + 8.0 * (double)(s * M * N) / 4e6 : 0.0);
        if (us < 0.97 * best.us) best = {tile, s, us};
    }
    return best;
}
inline CbmPlan cbm_plan(int64_t M, int64_t N, int64_t K, int32_t type, bool units) {
    if (!units) return cbm_plan(M, N, K, type, 0);
    const CbmPlan large = cbm_plan(M, N, K, type, 256), small = cbm_plan(M, N, K, type, 128);
    return large.us < small.us ? large : small;
}

// The most that a product of the size is cut into, however its matrices lie.
inline int64_t cbm_product_parts(int64_t M, int64_t N, int64_t K, int32_t type) {
    const int64_t any = cbm_plan(M, N, K, type, false).splits;
    return type == CBM_F32 ? any : std::max(any, cbm_plan(M, N, K, type, true).splits);
}

// 256 or 128: the tiles that a product whose units go straight to LDS is made in
inline int cbm_product_tile(int64_t M, int64_t N, int64_t K, int32_t type) {
    const CbmPlan large = cbm_plan(M, N, K, type, 256), small = cbm_plan(M, N, K, type, 128);
    return large.us < small.us ? 256 : 128;
}

// Products that are made 32 x 32 values at a time (cbm_small.h), where that takes less: microseconds as measured, of tiles that go through LDS a start, what a k takes and what a million operations take; of
// small products what a workgroup takes, too.  A gradient's call: three products or (given G and U) two, of altogether `again` + n + columns steps of k.  (Tiles / small, us: 2000 x 2000 with 2 x 40 in fp32 126 / 31,
// 512 x 512 with 2 x 512 in bf16 10.5 / 6.7, 1024 x 1024 with 2 x 1024 17 / 35; gradients of 128 x 512 with 512 x 512 classes 71 / 16 and 29 / 14, of 4000 x 512 with 512 x 512 98 / 102 and 44 / 97.)
inline bool cbm_small_forward(int64_t rows, int64_t K, int64_t columns, int64_t groups, int32_t type) {
    const bool f32 = type == CBM_F32;
    const double work = 2e-6 * (double)rows * (double)K * (double)columns;
    return rows <= 1 << 20 && 3.0 + 0.0065 * (double)K + (f32 ? 0.009 : 0.0053) * work + 0.0075 * (double)groups < 6.0 + (f32 ? 0.058 : 0.0125) * (double)K + 0.0007 * work;
}
inline bool cbm_small_backward(int64_t n, int64_t k, int64_t columns, int64_t again, int64_t groups, int32_t type) {
    const bool f32 = type == CBM_F32;
    const double work = (again ? 6e-6 : 4e-6) * (double)n * (double)k * (double)columns;
    const double small = 6.3 + 0.007 * (double)(n + columns + again) + 0.009 * work + 0.005 * (double)groups;
    return n <= 1 << 20 && k <= 1 << 20 && small < (f32 ? 33.5 : 20.0) + (f32 ? 0.064 : 0.014) * (double)again + (f32 ? 0.006 : 0.004) * work + 0.0008 * (double)n;
}
inline int64_t cbm_small_groups(int64_t rows, int64_t columns) { return (rows + 31) / 32 * ((columns + 31) / 32); }
// The side of the tiles that a product of the orthogonal update takes least with (half: only those on and below the diagonal): rounds of workgroups, each its products at what a compute unit's share reaches and what it
// takes beside them.  (4096 x 4096's Gram matrix is 136 tiles of 256 on and below the diagonal, which take as long as 256 of them, and 253 of 192: 231 and 191 us.)
inline int cbm_orthogonal_side(int64_t M, int64_t N, int64_t K, bool half) {
    double best = 1e30;
    int side = 256;
    for (int b : {256, 192, 128, 64, 32}) {
        const int64_t m = (M + b - 1) / b, tiles = half ? m * (m + 1) / 2 : m * ((N + b - 1) / b), at_once = b == 128 ? 512 : 256;
        const double each = 6.0 * b * b * (double)K / ((b == 256 ? 1250.0 : b == 192 ? 1150.0 : b == 128 ? 1050.0 : b == 64 ? 800.0 : 450.0) * 1e6 / (double)at_once) * (b == 128 && tiles <= 256 ? 0.6 : 1.0);
        const double us = (double)((tiles + at_once - 1) / at_once) * (each + (b == 256 ? 12.0 : b == 192 ? 9.0 : b == 128 ? 5.0 : b == 64 ? 7.0 : 4.0));
        if (us < best) best = us, side = b;
    }
    return side;
}
