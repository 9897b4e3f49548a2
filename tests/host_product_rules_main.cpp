// Which kernels the sizes of the GPU tests are made by: a change of the rules that leaves a kernel without a test fails here.
#include <cstdio>
#include <cstdlib>

#include "train/cbm_product_rules.h"

static int bad = 0;
static void expect(const char* what, long got, long want) {
    if (got == want) return;
    std::printf("%s: %ld, not %ld\n", what, got, want);
    ++bad;
}

// The update of s x l: tiles of Z Z^T, of the polynomial and of a step (test_gpu_orthogonalise_tiles.py).
static void update(long s, long l, int gram, int poly, int step) {
    char name[96];
    std::snprintf(name, sizeof name, "update %ld x %ld", s, l);
    expect(name, cbm_orthogonal_side(s, s, l, true), gram);
    expect(name, cbm_orthogonal_side(s, s, s, true), poly);
    expect(name, cbm_orthogonal_side(s, l, s, false), step);
}

// The gated layer, n x k with 2 x m (test_gpu_product_paths.py): whether the products are small, copied, in tiles of 256, 128 or (any matrices) 0, shares of K of dX's and of the weights' gradients' products.
static void gated(long n, long k, long m, int type, bool copied, int tile, bool units, bool shares_dx, bool shares_dw) {
    char name[96];
    std::snprintf(name, sizeof name, "gated %ld x %ld, 2 x %ld, type %d", n, k, m, type);
    const long at = cbm_whole(m, type == CBM_F32 ? 32 : 64), wide = cbm_whole(k, 8);
    expect(name, cbm_small_forward(n, k, 2 * m, cbm_small_groups(n, m), type), 0);
    expect(name, cbm_small_backward(n, k, 2 * m, 0, cbm_small_groups(n, k) + 2 * cbm_small_groups(k, m), type), 0);
    expect(name, cbm_may_pack(n, k, 2 * m, type), copied);
    if (units) expect(name, cbm_product_tile(n, 2 * m, k, type), tile);
    expect(name, cbm_plan(n, k, 2 * at, type, units).splits > 1, shares_dx);
    expect(name, cbm_plan(units ? wide : k, 2 * at, n, type, units).splits > 1, shares_dw);
}

// Log probabilities of n x d with d x c (the same file): small or not, copied, tiles.
static void classes(long n, long d, long c, int type, bool copied, int tile, bool units) {
    char name[96];
    std::snprintf(name, sizeof name, "classes %ld x %ld, %ld, type %d", n, d, c, type);
    expect(name, cbm_small_forward(n, d, c, cbm_small_groups(n, c), type), 0);
    expect(name, cbm_small_backward(n, d, c, d, cbm_small_groups(n, c) + cbm_small_groups(n, d) + cbm_small_groups(d, c), type), 0);
    expect(name, cbm_may_pack(n, d, c, type), copied);
    if (units) expect(name, cbm_product_tile(n, c, d, type), tile);
}

int main() {
    update(513, 1537, 32, 32, 64);
    update(1025, 1031, 64, 64, 64);
    update(2049, 2051, 128, 128, 128);
    update(3001, 3003, 128, 128, 192);
    update(3073, 4001, 64, 128, 256);
    update(4097, 4099, 192, 192, 192);
    update(4353, 4361, 256, 256, 128);
    for (int type : {CBM_F32, CBM_BF16, CBM_F16}) {
        const bool wide = type != CBM_F32;
        gated(9001, 17, 300, type, false, 0, false, true, true);
        gated(4100, 136, 1024, type, false, 256, wide, true, true);
        gated(12001, 515, 4099, type, wide, 256, wide, false, true);
        gated(4097, 512, 12288, type, wide, 256, wide, true, !wide);
        classes(9001, 17, 300, type, false, 0, false);
        classes(2304, 320, 4096, type, false, 256, wide);
        classes(12001, 515, 8199, type, wide, 256, wide);
        classes(4097, 512, 24576, type, wide, 256, wide);
        classes(20003, 65, 47, type, false, 0, false);
        classes(70001, 9, 20, type, false, 0, false);
    }
    // (in fp32 the products of 128 x 128 and narrower are what there is)
    gated(20003, 65, 47, CBM_F16, false, 0, false, false, true);
    gated(5000, 64, 264, CBM_F16, false, 128, true, true, true);
    if (!bad) std::printf("product rules ok\n");
    return bad != 0;
}
