// Products that the operators of a training step are made of (cbm_products.hip): which matrices, and what becomes of the sums.
#pragma once

#include <cstdint>

#include "cbm.h"

// value (r, c) of the result from its sum s: s += sums[r, c] unless `first`; kept there if not `last`; else s (times *factor), rounded to the operands' type.
struct CbmProductOut {
    void* C[2];          // columns from `at` on belong to the second one's first (0: there is one)
    int64_t ldc[2];
    int64_t rows;        // of the result that are written; 0: all
    int32_t columns;     // of each
    int32_t at;
    const float* factor; // on the device; may be NULL
    float* sums;         // M x N, packed; may be NULL
    bool first, last;
};
// A . B with A M x K and B K x N.  across: A lies as K x M, B as K x N (otherwise N x K).  B[1]: its k follow those of B[0] from `at` on, each has K.
struct CbmProduct {
    int32_t type;
    int64_t M, N, K;
    const void* A;
    int64_t lda;
    bool a_across;
    const void* B[2];
    int64_t ldb[2];
    bool b_across;
    int64_t at;
    CbmProductOut out;
    float* parts;  // cbm_product_parts() M x N values, packed, where that is more than one
};
// A launch has fewer than 2^32 threads, 256 for each tile of 128 x 128 values or larger, in a grid of a multiple of eight.
inline bool cbm_too_many_tiles(int64_t rows, int64_t columns) { return ((rows + 127) / 128 * ((columns + 127) / 128) + 7) / 8 * 8 >= (int64_t)1 << 24; }
int64_t cbm_product_parts(int64_t M, int64_t N, int64_t K, int32_t type);
// Large products of 16-bit values: matrices that do not lie in whole units of 16 bytes are copied so that they do, and a matrix whose rows of k many rows of the other meet is turned to lie along k; their
// workspace has room for it.  (us as they lie / copied, forward and backward, odd strides: 100000 x 1001 with 2 x 1001 columns 777 / 675 and 1447 / 1326; 16384 x 333 with 2 x 500 38 / 47, 105 / 108;
// 1024 x 1000 with 2 x 4000 37 / 48, 105 / 104.  Turned: 65536 x 1024 with 2 x 4096 1342 / 1218.)
inline bool cbm_may_pack(int64_t rows, int64_t K, int64_t columns, int32_t type) { return type != CBM_F32 && rows >= 1024 && K >= 256 && 2e-11 * (double)rows * (double)K * (double)columns >= 1.0; }
constexpr int64_t CBM_TURN_ROWS = 4096;  // from so many rows on turning pays
inline int64_t cbm_whole(int64_t v, int64_t of) { return (v + of - 1) / of * of; }
// Rows of `columns` values and zeros up to ldt, a multiple of 8, and rows of zeros up to a multiple of 8, which a copy's place has room for: row r at row `blocks` (r / 32) + r % 32 + `at` where blocks are asked for, else r.  turned: value
// (r, c) is from[c ld + r].
void cbm_launch_pack(const void* from, int64_t ld, int64_t rows, int64_t columns, bool turned, void* to, int64_t ldt, int64_t blocks, int64_t at, void* stream);
// 256 or 128: the tiles that a product whose units go straight to LDS is made in
int cbm_product_tile(int64_t M, int64_t N, int64_t K, int32_t type);
void cbm_launch_tiles(const CbmProduct& p, void* stream);
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
// C = S0 B0^T + S1 B1^T (M x N, K each; S1 may be NULL) and C0 = A^T S0, C1 = A^T S1 (M x N; each may be NULL) with slopes S in fp32, the other matrices of `type`.
void cbm_launch_small_along(int32_t type, int64_t M, int64_t N, int64_t K, const float* S0, const float* S1, int64_t lds, const void* B0, int64_t ldb0, const void* B1, int64_t ldb1, void* C, int64_t ldc,
                            void* stream);
void cbm_launch_small_across(int32_t type, int64_t M, int64_t N, int64_t K, const void* A, int64_t lda, const float* S0, const float* S1, int64_t lds, void* C0, int64_t ldc0, void* C1, int64_t ldc1,
                             void* stream);
// fp32 with so few columns: tiles of 256 x 64, which waste half as much as those of 128 x 128.
inline bool cbm_is_narrow(int64_t columns, int32_t type) { return type == CBM_F32 && columns <= 64; }
cbm_status cbm_launched(const char* what);  // the status of the launches since the last look
