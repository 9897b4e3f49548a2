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
int64_t cbm_product_parts(int64_t M, int64_t N, int64_t K, int32_t type);
// Large products of 16-bit values: matrices that do not lie in whole units of 16 bytes are copied so that they do, and a matrix whose rows of k many rows of the other meet is turned to lie along k; their
// workspace has room for it.  (us as they lie / copied, forward and backward, odd strides: 100000 x 1001 with 2 x 1001 columns 777 / 675 and 1447 / 1326; 16384 x 333 with 2 x 500 38 / 47, 105 / 108;
// 1024 x 1000 with 2 x 4000 37 / 48, 105 / 104.  Turned: 65536 x 1024 with 2 x 4096 1342 / 1218.)
inline bool cbm_may_pack(int64_t rows, int64_t K, int64_t columns, int32_t type) { return type != CBM_F32 && rows >= 1024 && K >= 256 && 2e-11 * (double)rows * (double)K * (double)columns >= 1.0; }
constexpr int64_t CBM_TURN_ROWS = 4096;  // from so many rows on turning pays
inline int64_t cbm_whole(int64_t v, int64_t of) { return (v + of - 1) / of * of; }
// Rows of `columns` values and zeros up to ldt, a multiple of 8, and rows of zeros up to a multiple of 8: row r at row `blocks` (r / 32) + r % 32 + `at` where blocks are asked for, else r.  turned: value
// (r, c) is from[c ld + r].
void cbm_launch_pack(const void* from, int64_t ld, int64_t rows, int64_t columns, bool turned, void* to, int64_t ldt, int64_t blocks, int64_t at, void* stream);
// 256 or 128: the tiles that a product whose units go straight to LDS is made in
int cbm_product_tile(int64_t M, int64_t N, int64_t K, int32_t type);
void cbm_launch_tiles(const CbmProduct& p, void* stream);
cbm_status cbm_launched(const char* what);  // the status of the launches since the last look
