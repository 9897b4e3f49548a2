// Products that the operators of a training step are made of (cbm_products.hip): which matrices, and what becomes of the sums.
#pragma once

#include <cstdint>

#include "cbm.h"

// value (r, c) of the result from its sum s: s += sums[r, c] unless `first`; kept there if not `last`; else alpha s (times *factor) + beta more[r, c], rounded to `type`.
struct CbmProductOut {
    int32_t type;        // cbm_dtype of what is written
    void* C[2];          // columns from `at` on belong to the second one's first (0: there is one)
    int64_t ldc[2];
    int32_t columns;     // of each
    int32_t at;
    bool transposed;     // value (r, c) goes to C[c, r]
    float alpha, beta;
    const float* factor; // on the device; may be NULL
    const float* more;   // may be NULL
    int64_t ldm;
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
// 256 or 128: the tiles that a product whose units go straight to LDS is made in
int cbm_product_tile(int64_t M, int64_t N, int64_t K, int32_t type);
void cbm_launch_tiles(const CbmProduct& p, void* stream);
cbm_status cbm_launched(const char* what);  // the status of the launches since the last look
