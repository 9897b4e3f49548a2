// Products that the operators of a training step are made of (cbm_products.hip): which matrices, and what becomes of the sums.
#pragma once

#include <cstdint>

#include "cbm.h"
#include "cbm_product_rules.h"

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
// Rows of `columns` values and zeros up to ldt, a multiple of 8, and rows of zeros up to a multiple of 8, which a copy's place has room for: row r at row `blocks` (r / 32) + r % 32 + `at` where blocks are asked for, else r.  turned: value
// (r, c) is from[c ld + r].
void cbm_launch_pack(const void* from, int64_t ld, int64_t rows, int64_t columns, bool turned, void* to, int64_t ldt, int64_t blocks, int64_t at, void* stream);
void cbm_launch_tiles(const CbmProduct& p, void* stream);
// C = S0 B0^T + S1 B1^T (M x N, K each; S1 may be NULL) and C0 = A^T S0, C1 = A^T S1 (M x N; each may be NULL) with slopes S in fp32, the other matrices of `type`.
void cbm_launch_small_along(int32_t type, int64_t M, int64_t N, int64_t K, const float* S0, const float* S1, int64_t lds, const void* B0, int64_t ldb0, const void* B1, int64_t ldb1, void* C, int64_t ldc,
                            void* stream);
void cbm_launch_small_across(int32_t type, int64_t M, int64_t N, int64_t K, const void* A, int64_t lda, const float* S0, const float* S1, int64_t lds, void* C0, int64_t ldc0, void* C1, int64_t ldc1,
                             void* stream);
cbm_status cbm_launched(const char* what);  // the status of the launches since the last look
