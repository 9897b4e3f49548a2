// The orthogonal update: a matrix's singular values driven towards one by products alone.
//
// Z (s x l, the shorter side first) is held as two fp16 parts that add up to 22 bits of each value, at a power of two times its size that fits the largest it can have: Z's singular values are at most one at first, and
// each step's largest follows from the coefficients, so the host knows a bound of every entry.  Three products of parts (hh, hl, lh) then stand for one in 32 bits: what is left out is 2^-22 of a term, and
// sums are fp32.  (500 x 1333 in fp32: error 1.4e-6; with three bf16 parts and six products 1.1e-6, and twice as long.)  Nothing below 2^-25 of 2^-14 of the largest bound is lost.
//
// All operands lie along k: Z and its transpose are both kept (Z Z^T reads rows of the one, P Z rows of P and of the other), A and P = a I + b A + c A^2 are symmetric: their tiles on one side of the diagonal are
// made, and written to both.  A row in memory is blocks of 32 values: their high parts, then their low parts, 128 bytes together, so that a chunk of 64 halves is 32 k of both parts.
#include <algorithm>
#include <cmath>

#include "cbm_aligned.h"
#include "cbm_internal.h"
#include "cbm_products.h"

namespace {

constexpr int PARTS = 256;  // workgroups that share the sum of squares

// Squares in 64 bits: no value of fp32 overflows or vanishes there.  Four pieces of 16 bytes a thread under way (4096 x 4096 in bf16 one value at a time 105 us).
template <class T>
__global__ __launch_bounds__(256) void cbm_orthogonal_norm_kernel(int64_t m, int64_t n, const T* __restrict__ X, int64_t ldx, double* __restrict__ parts) {
    constexpr int V = 16 / (int)sizeof(T), AHEAD = 4;
    __shared__ double room[4];
    double s = 0.0;
    const uint32_t wide = (uint32_t)((n + 256 * V - 1) / (256 * V)), count = (uint32_t)m * wide;  // pieces of a row, of V values a thread
    for (uint32_t i = blockIdx.x; i < count; i += AHEAD * gridDim.x) {
        float x[AHEAD][V];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const uint32_t at = min(i + k * gridDim.x, count - 1), r = at / wide;
            const T* row = X + (int64_t)r * ldx;
            const int64_t c = ((int64_t)(at - r * wide) * 256 + threadIdx.x) * V;
            const bool any = i + k * gridDim.x < count;
            if (any && c + V <= n) {
                load_piece<V>(x[k], row + c);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) x[k][j] = any && c + j < n ? (float)row[c + j] : 0.0f;
            }
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) s += (double)x[k][j] * (double)x[k][j];
    }
#pragma unroll
    for (int step = 1; step < 64; step *= 2) s += __shfl_xor(s, step);
    if (threadIdx.x % 64 == 0) room[threadIdx.x / 64] = s;
    __syncthreads();
    if (threadIdx.x == 0) parts[blockIdx.x] = (room[0] + room[1]) + (room[2] + room[3]);
}

// A matrix in parts: rows of blocks of 32 columns.
struct Halves {
    _Float16* p;
    int64_t rows, columns;
    __host__ __device__ int64_t ld() const { return (columns + 31) / 32 * 64; }
    __host__ __device__ int64_t bytes() const { return rows * ld() * 2; }
};
__device__ __forceinline__ void cut(float v, _Float16& h, _Float16& l) {
    h = (_Float16)v;
    l = (_Float16)(v - (float)h);
}
// Four values of row r from column c on, columns a multiple of four, zeros beyond the last (up to a whole block: products read those).
__device__ __forceinline__ void put_halves(const Halves& x, int64_t r, int64_t c, const float (&v)[4]) {
    if (r >= x.rows || c >= x.ld() / 2) return;
    typedef _Float16 Four __attribute__((ext_vector_type(4)));
    Four h, l;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        _Float16 a, b;
        cut(c + j < x.columns ? v[j] : 0.0f, a, b);
        h[j] = a;
        l[j] = b;
    }
    _Float16* to = x.p + r * x.ld() + c / 32 * 64 + c % 32;
    *reinterpret_cast<Four*>(to) = h;
    *reinterpret_cast<Four*>(to + 32) = l;
}

// Z at 2^up times its size and its transpose, from X or its transpose over its norm + eps, a block of 32 x 32 a workgroup.
template <class T>
__global__ __launch_bounds__(256) void cbm_orthogonal_begin_kernel(const T* __restrict__ X, int64_t ldx, bool transposed, float eps, float up, const double* __restrict__ parts, Halves z, Halves zt) {
    __shared__ float room[32][33];
    __shared__ double squares[4];
    double s = parts[threadIdx.x];
#pragma unroll
    for (int step = 1; step < 64; step *= 2) s += __shfl_xor(s, step);
    if (threadIdx.x % 64 == 0) squares[threadIdx.x / 64] = s;
    __syncthreads();
    const double by = (double)up / (sqrt((squares[0] + squares[1]) + (squares[2] + squares[3])) + (double)eps);
    const int64_t r0 = (int64_t)blockIdx.y * 32, c0 = (int64_t)blockIdx.x * 32;
#pragma unroll
    for (int i = 0; i < 4; ++i) {  // along X's rows
        const int slow = threadIdx.x / 32 + 8 * i, fast = threadIdx.x % 32;
        const int64_t r = r0 + (transposed ? fast : slow), c = c0 + (transposed ? slow : fast);
        float v = 0.0f;
        if (r < z.rows && c < z.columns) v = (float)((double)(float)(transposed ? X[c * ldx + r] : X[r * ldx + c]) * by);
        room[r - r0][c - c0] = v;
    }
    __syncthreads();
    const int row = threadIdx.x / 8, four = threadIdx.x % 8 * 4;
    const float along[4] = {room[row][four], room[row][four + 1], room[row][four + 2], room[row][four + 3]}, across[4] = {room[four][row], room[four + 1][row], room[four + 2][row], room[four + 3][row]};
    put_halves(z, r0 + row, c0 + four, along);
    put_halves(zt, c0 + row, r0 + four, across);
}

template <class T>
__global__ __launch_bounds__(256) void cbm_orthogonal_scaled_kernel(int64_t m, int64_t n, const T* __restrict__ X, int64_t ldx, float eps, float scale, const double* __restrict__ parts, T* __restrict__ Y,
                                                                 int64_t ldy) {
    double s = 0.0;
    for (int i = 0; i < PARTS; ++i) s += parts[i];
    const double size = sqrt(s) + (double)eps;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < m * n; i += (int64_t)gridDim.x * 256) Y[i / n * ldy + i % n] = (T)(scale * (float)((double)(float)X[i / n * ldx + i % n] / size));
}

// The sums of a tile of B x B of a product of matrices in parts, as CbmAlignedTiles makes them: a step of 16 k is three products, and its units are read as the first of them and the one before go on.
template <int B>
struct HalvesTiles : CbmTileSums<B, B, 2, 2> {
    typedef CbmTileSums<B, B, 2, 2> Sums;
    typedef CbmAlignedSide<_Float16, B, ALONG_K, SINGLE> Side;
    static constexpr int TM = Sums::TM, TN = Sums::TN, BK = 64, SLOT = Side::UNITS, UNITS = 5 * SLOT, GROUPS = B > 128 ? 1 : 2, LOADS = Side::LOADS, HALF = LOADS / 2;
    static_assert(UNITS >= Sums::OUT_UNITS, "");
    using Sums::acc;

    __device__ __forceinline__ void run(uintx4* lds, const CbmOperand<_Float16>& a, const CbmOperand<_Float16>& b, int tile_m, int tile_n, int last) {
        this->clear();
        const int wave = Sums::wave(), wm = Sums::first_row(), wn = Sums::first_column();
        Side sa, sb;
        sa.begin(a, tile_m, wave);
        sb.begin(b, tile_n, wave);
        auto load = [&](auto whole, Side& s, const CbmOperand<_Float16>& o, int c, uintx4* to, int i) { s.template load<decltype(whole)::value>(o, c, o.K, to, wave, i); };
        uintx4 *a0 = lds, *b0 = lds + SLOT, *a1 = lds + 2 * SLOT, *b1 = lds + 3 * SLOT, *a2 = lds + 4 * SLOT;
        constexpr std::false_type some;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) load(some, sa, a, 0, a0, i);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) load(some, sb, b, 0, b0, i);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) load(some, sa, a, 1, a1, i);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) load(some, sb, b, 1, b1, i);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) load(some, sa, a, 2, a2, i);
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(3 * LOADS) : "memory");
        uintx4 xh[2][TM], yh[2][TN], xl[TM], yl[TN];
        auto read = [&](const uintx4* la, const uintx4* lb, int s, uintx4 (&x)[TM], uintx4 (&y)[TN]) {
#pragma unroll
            for (int i = 0; i < TM; ++i) x[i] = Side::unit(la, wm + 32 * i, s);
#pragma unroll
            for (int j = 0; j < TN; ++j) y[j] = Side::unit(lb, wn + 32 * j, s);
        };
        auto multiply = [&](const uintx4 (&x)[TM], const uintx4 (&y)[TN]) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = cbm_multiply<_Float16>(y[j], x[i], acc[i][j]);
        };
        // a read, or a load, between two products
        auto order = [&](auto products_) {
            constexpr int PRODUCTS = decltype(products_)::value, READS = TM + TN, AT_ONCE = PRODUCTS / 2 >= READS ? 1 : READS, GROUPS_OF_READS = (READS + AT_ONCE - 1) / AT_ONCE;
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
#pragma unroll
            for (int i = 0; i < GROUPS_OF_READS; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x100, AT_ONCE, 0);
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            }
#pragma unroll
            for (int i = 0; i < HALF; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            }
            constexpr int LEFT = PRODUCTS - 1 - GROUPS_OF_READS - HALF;
            if constexpr (LEFT > 0) __builtin_amdgcn_sched_group_barrier(0x008, LEFT, 0);
            __builtin_amdgcn_sched_barrier(0);
        };
        using std::integral_constant;
        read(a0, b0, 0, xh[0], yh[0]);
        auto chunk = [&](auto whole, int c) {
            read(a0, b0, 2, xl, yl);
#pragma unroll
            for (int i = HALF; i < LOADS; ++i) load(whole, sb, b, c + 1, b1, i);
            multiply(xh[0], yh[0]);
            order(integral_constant<int, TM * TN>{});
            read(a0, b0, 1, xh[1], yh[1]);
#pragma unroll
            for (int i = 0; i < HALF; ++i) load(whole, sa, a, c + 2, a2, i);
            multiply(xh[0], yl);
            multiply(xl, yh[0]);
            order(integral_constant<int, 2 * TM * TN>{});
            read(a0, b0, 3, xl, yl);
#pragma unroll
            for (int i = HALF; i < LOADS; ++i) load(whole, sa, a, c + 2, a2, i);
            multiply(xh[1], yh[1]);
            order(integral_constant<int, TM * TN>{});
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LOADS) : "memory");
            __builtin_amdgcn_sched_barrier(0);
            read(a1, b1, 0, xh[0], yh[0]);
#pragma unroll
            for (int i = 0; i < HALF; ++i) load(whole, sb, b, c + 2, a0, i);
            multiply(xh[1], yl);
            multiply(xl, yh[1]);
            order(integral_constant<int, 2 * TM * TN>{});
            uintx4 *fa = a0, *fb = b0;
            a0 = a1, b0 = b1, a1 = a2, b1 = fa, a2 = fb;
        };
        int c = 0;
        for (; c + 2 < last; ++c) chunk(std::true_type{}, c);
        for (; c < last; ++c) chunk(std::false_type{}, c);
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }
    // f(row, column of the first, four sums) and g(column, row of the first, four sums): along the rows and along the columns of the result
    template <class F, class G>
    __device__ __forceinline__ void both(uintx4* lds, int tile_m, int tile_n, F&& f, bool down, G&& g) const {
        const int lane = threadIdx.x & 63;
        uintx4* mine = lds + Sums::wave() * 32 * Sums::OUT_STRIDE;
        const int64_t row = (int64_t)tile_m * B + Sums::first_row(), column = (int64_t)tile_n * B + Sums::first_column();
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            this->band_to_lds(mine, i);
#pragma unroll 1
            for (int t = 0; t < Sums::COLS / 8; ++t) {
                const int at = 64 * t + lane, r = at / (Sums::COLS / 4), c = at % (Sums::COLS / 4);
                float v[4];
                Sums::from_lds(v, mine + r * Sums::OUT_STRIDE + c);
                f(row + 32 * i + r, column + 4 * c, v);
                if (down) mine[r * Sums::OUT_STRIDE + c] = __builtin_bit_cast(uintx4, (floatx4){v[0], v[1], v[2], v[3]});  // (as f left them)
            }
            if (down) {
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
                const float* of = (const float*)mine;
#pragma unroll 1
                for (int t = 0; t < Sums::COLS / 8; ++t) {
                    const int r = lane % 8 * 4, c = t * 8 + lane / 8;
                    float v[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = of[(r + j) * (4 * Sums::OUT_STRIDE) + c];
                    g(column + c, row + 32 * i + r, v);
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
    }
};

// The same for few tiles, of 64 x 64 or of 32 x 32: each wave has all of the tile for its share of K, with units of its own in LDS, so that no wave waits for another until they add up.  (500 x 1333's Gram
// matrix: 36 tiles of 64 x 64 whose four waves have a quarter of the tile 21 us, of K 12.9; 136 of 32 x 32 whose eight waves share K 8.0.  Its steps, 168 or 672 tiles: 10.0 and 15.)
template <int B, int WAVES>
struct HalvesShares {
    typedef CbmAlignedSide<_Float16, 4 * B, ALONG_K, SINGLE> Side;  // (a wave's loads are B rows)
    static constexpr int ROWS = B, THREADS = 64 * WAVES, GROUPS = 1, LOADS = Side::LOADS, SLOT = B * 8, TM = B / 32, OUT_STRIDE = B / 4 + 1, UNITS = WAVES * 4 * SLOT;
    static_assert(LOADS == B / 8 && UNITS >= WAVES * B * OUT_STRIDE && WAVES >= 4, "");

    __device__ __forceinline__ void run(uintx4* lds, const CbmOperand<_Float16>& a, const CbmOperand<_Float16>& b, int tile_m, int tile_n, int last) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
        floatx16 acc[TM][TM] = {};
        Side sa, sb;
        sa.begin(a, tile_m, 0, B);
        sb.begin(b, tile_n, 0, B);
        uintx4 *here = lds + wave * 4 * SLOT, *next = here + 2 * SLOT;
        auto load = [&](int c, uintx4* to) {  // (zeros beyond the last chunk: as many loads are under way to the end)
#pragma unroll
            for (int i = 0; i < LOADS; ++i) sa.template load<false>(a, c, a.K, to, 0, i);
#pragma unroll
            for (int i = 0; i < LOADS; ++i) sb.template load<false>(b, c, b.K, to + SLOT, 0, i);
        };
        load(wave, here);
        load(wave + WAVES, next);
        for (int c = wave; c < last; c += WAVES) {
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * LOADS) : "memory");
            uintx4 x[TM][4], y[TM][4];
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    x[i][s] = Side::unit(here, 32 * i, s);
                    y[i][s] = Side::unit(here + SLOT, 32 * i, s);
                }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
            load(c + 2 * WAVES, here);
#pragma unroll
            for (int p = 0; p < 6; ++p)  // high by high, high by low, low by high, of either half of the chunk
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TM; ++j) acc[i][j] = cbm_multiply<_Float16>(y[j][p % 2 + (p / 2 == 1 ? 2 : 0)], x[i][p % 2 + (p / 2 == 2 ? 2 : 0)], acc[i][j]);
            uintx4* t = here;
            here = next;
            next = t;
        }
        asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
        uintx4* mine = lds + wave * B * OUT_STRIDE;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TM; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    mine[(32 * i + (lane & 31)) * OUT_STRIDE + 8 * j + 2 * q + (lane >> 5)] =
                        __builtin_bit_cast(uintx4, (floatx4){acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]});
        __syncthreads();
    }
    // four waves, a quarter of the rows each
    template <class F, class G>
    __device__ __forceinline__ void both(uintx4* lds, int tile_m, int tile_n, F&& f, bool down, G&& g) const {
        constexpr int R = B / 4, QUADS = R / 4;
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), first = R * wave;
        if (wave >= 4) return;
        const int64_t row = (int64_t)tile_m * B + first, column = (int64_t)tile_n * B;
#pragma unroll 1
        for (int t = 0; t < R * B / 256; ++t) {
            const int r = (256 / B) * t + lane / (B / 4), c = lane % (B / 4);
            uintx4* at = lds + (first + r) * OUT_STRIDE + c;
            floatx4 sum = __builtin_bit_cast(floatx4, at[0]);
#pragma unroll
            for (int w = 1; w < WAVES; ++w) sum += __builtin_bit_cast(floatx4, at[w * B * OUT_STRIDE]);
            float v[4] = {sum[0], sum[1], sum[2], sum[3]};
            f(row + r, column + 4 * c, v);
            at[0] = __builtin_bit_cast(uintx4, (floatx4){v[0], v[1], v[2], v[3]});
        }
        if (!down) return;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        const float* of = (const float*)(lds + first * OUT_STRIDE);
#pragma unroll 1
        for (int t = 0; t < B * QUADS / 64; ++t) {
            const int r = lane % QUADS * 4, c = t * (64 / QUADS) + lane / QUADS;
            float v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = of[(r + j) * (4 * OUT_STRIDE) + c];
            g(column + c, row + r, v);
        }
    }
};

enum { GRAM, POLYNOMIAL, STEP, LAST };
struct ProductArgs {
    Halves a, b;     // rows of both, along k
    Halves out, outt;  // GRAM, POLYNOMIAL: out; STEP: both
    Halves gram;     // POLYNOMIAL
    float up;        // of the sums, to the size that is written
    float of_gram, of_one;  // POLYNOMIAL: times the Gram matrix as it is kept, and on the diagonal
    void* Y;         // LAST
    int64_t ldy;
    bool transposed;
};

// Tile `at` of those on and below the diagonal.
__device__ __forceinline__ void below(int at, int& m, int& n) {
    m = (int)((sqrtf(8.0f * (float)at + 1.0f) - 1.0f) * 0.5f);
    while ((int64_t)(m + 1) * (m + 2) / 2 <= at) ++m;
    while ((int64_t)m * (m + 1) / 2 > at) --m;
    n = at - (int)((int64_t)m * (m + 1) / 2);
}

template <class Tiles, int MODE, class T>
__global__ __launch_bounds__(Tiles::THREADS, Tiles::GROUPS) void cbm_orthogonal_product_kernel(ProductArgs p) {
    constexpr int B = Tiles::ROWS;
    __shared__ uintx4 lds[Tiles::UNITS];
    int m, n;
    const int tiles_m = (int)((p.a.rows + B - 1) / B), tiles_n = (int)((p.b.rows + B - 1) / B);
    if constexpr (MODE == GRAM || MODE == POLYNOMIAL) {
        const int at = blockIdx.x % 8 * (gridDim.x / 8) + blockIdx.x / 8;
        if (at >= tiles_m * (tiles_m + 1) / 2) return;
        below(at, m, n);
        m = __builtin_amdgcn_readfirstlane(m);
        n = __builtin_amdgcn_readfirstlane(n);
    } else {
        const CbmTilePlace at = cbm_tile_place(tiles_m, tiles_n, 1);
        if (!at.any) return;
        m = at.m, n = at.n;
    }
    Tiles t;
    t.run(lds, {{p.a.p, nullptr}, {p.a.ld(), 0}, p.a.rows, p.a.ld(), 0}, {{p.b.p, nullptr}, {p.b.ld(), 0}, p.b.rows, p.b.ld(), 0}, m, n, (int)(p.a.ld() / 64));
    if constexpr (MODE == LAST) {
        T* Y = (T*)p.Y;
        t.both(
            lds, m, n,
            [&](int64_t r, int64_t c, float (&v)[4]) {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] *= p.up;
                if (!p.transposed && r < p.a.rows) cbm_put(Y + r * p.ldy, c, p.b.rows, v);
            },
            p.transposed, [&](int64_t c, int64_t r, float (&v)[4]) { if (c < p.b.rows) cbm_put(Y + c * p.ldy, r, p.a.rows, v); });
    } else {
        t.both(
            lds, m, n,
            [&](int64_t r, int64_t c, float (&v)[4]) {
                float g[4] = {};
                if constexpr (MODE == POLYNOMIAL)
                    if (r < p.gram.rows && c < p.gram.rows) {
                        typedef _Float16 Four __attribute__((ext_vector_type(4)));
                        const _Float16* from = p.gram.p + r * p.gram.ld() + c / 32 * 64 + c % 32;
                        const Four h = *reinterpret_cast<const Four*>(from), l = *reinterpret_cast<const Four*>(from + 32);
#pragma unroll
                        for (int j = 0; j < 4; ++j) g[j] = (float)h[j] + (float)l[j];
                    }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    v[j] *= p.up;
                    if constexpr (MODE == POLYNOMIAL) v[j] = fmaf(p.of_gram, g[j], v[j]) + (r == c + j ? p.of_one : 0.0f);
                    if (r >= p.a.rows) v[j] = 0.0f;  // (rows beyond the last are the last one's again; down a column they are zeros)
                }
                put_halves(p.out, r, c, v);
            },
            MODE == STEP || m != n, [&](int64_t c, int64_t r, float (&v)[4]) { put_halves(MODE == STEP ? p.outt : p.out, c, r, v); });
    }
}

// Small matrices: everything in one workgroup's LDS, Z and A (which P takes the place of), rows of blocks as in memory and one unit more, so that sixteen neighbouring rows' units fall on different banks.
// A wave has a tile of 32 x 32.  Z's columns, which P Z wants, are turned as they are read.  What bounds it is one compute unit's LDS and the five barriers of a step (five steps of 64 x 64
// 18 us, of 128 x 128 45, of 16 x 300 26 and of 64 x 250 35; the launches of the general way take 75 at 64 x 500 or 129 x 130).
constexpr int SMALL_STEPS = 16;
struct SmallArgs {
    int rows, columns, steps;  // of Z
    bool transposed;
    float eps, first, last;              // powers: of Z at first, and back to its size (and Y's scale) at last
    float gram[SMALL_STEPS], square[SMALL_STEPS], of_gram[SMALL_STEPS], of_one[SMALL_STEPS], next[SMALL_STEPS];
};
constexpr int small_pitch(int k) { return k * 4 + 16; }  // bytes of a row of k (a multiple of 32) values in parts

__device__ __forceinline__ uintx4 small_unit(const char* at) { return *reinterpret_cast<const uintx4*>(at); }
// eight k of column lane % 32 from k 8 (lane / 32) on: `at` is the first row's first column
template <int PITCH>
__device__ __forceinline__ uintx4 small_turned(const char* at) {
    typedef short Four __attribute__((ext_vector_type(4)));
    const int lane = threadIdx.x & 63;
    const char* p = at + (8 * (lane >> 5) + (lane >> 2 & 3)) * PITCH + (lane >> 4 & 1) * 32 + (lane & 3) * 8;
    struct {
        Four low, high;
    } v;
    v.low = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) Four*)p);
    v.high = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) Four*)(p + 4 * PITCH));
    return __builtin_bit_cast(uintx4, v);
}
// Rows m .. m + 31 of x times rows n .. n + 31 of y (TURNED: times columns n .. n + 31), over K.  Lane l has row l % 32 and columns 8 q + 4 (l / 32) on.
template <bool TURNED, int K, int PX, int PY>
__device__ __forceinline__ floatx16 small_product(const char* x, int m, const char* y, int n) {
    const int lane = threadIdx.x & 63, of = (lane >> 5) * 16;
    const char *ax = x + (m + (lane & 31)) * PX + of, *ay = TURNED ? y + n * 4 : y + (n + (lane & 31)) * PY + of;
    floatx16 high{}, hl{}, lh{};  // (three chains: a product waits for the one before in its own)
#pragma unroll
    for (int s = 0; s < K / 16; ++s) {
        const int at = s / 2 * 128 + s % 2 * 32;
        const uintx4 xh = small_unit(ax + at), xl = small_unit(ax + at + 64), yh = TURNED ? small_turned<PY>(ay + 16 * s * PY) : small_unit(ay + at),
                     yl = TURNED ? small_turned<PY>(ay + 16 * s * PY + 64) : small_unit(ay + at + 64);
        high = cbm_multiply<_Float16>(yh, xh, high);
        hl = cbm_multiply<_Float16>(yl, xh, hl);
        lh = cbm_multiply<_Float16>(yh, xl, lh);
    }
    return high + (hl + lh);
}
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
// f(q, columns 8 q + 4 (lane / 32) on of the lane's row in x) of a tile
template <class F>
__device__ __forceinline__ void small_places(char* x, int pitch, int m, int n, F&& f) {
    const int lane = threadIdx.x & 63;
    char* row = x + (m + (lane & 31)) * pitch + n * 4 + (lane >> 5) * 8;
#pragma unroll
    for (int q = 0; q < 4; ++q) f(q, row + 16 * q);
}
__device__ __forceinline__ void small_put(char* x, int pitch, int m, int n, const floatx16& v, float up) {
    small_places(x, pitch, m, n, [&](int q, char* at) {
        f16x4 h, l;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            _Float16 a, b;
            cut(v[4 * q + j] * up, a, b);
            h[j] = a;
            l[j] = b;
        }
        *reinterpret_cast<f16x4*>(at) = h;
        *reinterpret_cast<f16x4*>(at + 64) = l;
    });
}

// S x L: Z's rows and columns with zeros beyond them.
template <class T, int S, int L>
__global__ __launch_bounds__(S * L / 16) void cbm_orthogonal_small_kernel(SmallArgs p, const T* X, int64_t ldx, T* Y, int64_t ldy) {
    constexpr int PZ = small_pitch(L), PG = small_pitch(S), WAVES = S / 32 * (L / 32), THREADS = 64 * WAVES, EACH = S * L / THREADS;
    static_assert(S <= L, "");
    __shared__ uintx4 all[S * (PZ + PG) / 16];
    __shared__ double squares[WAVES];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    char *z = (char*)all, *g = z + S * PZ;
    // X's values, neighbouring threads along its rows; zeros beyond it
    const uint32_t height = p.transposed ? p.columns : p.rows, width = p.transposed ? p.rows : p.columns, down = THREADS / width, along = THREADS % width, r0 = threadIdx.x / width, c0 = threadIdx.x - r0 * width;
    auto next = [&](uint32_t& r, uint32_t& c) {
        c += along;
        r += down + (c >= width ? 1 : 0);
        c -= c >= width ? width : 0;
    };
    float x[EACH];
    double sum = 0.0;
    uint32_t xr = r0, xc = c0;
#pragma unroll
    for (int i = 0; i < EACH; ++i, next(xr, xc)) x[i] = xr < height ? (float)X[xr * ldx + xc] : 0.0f;
    for (int i = threadIdx.x; i < S * PZ / 16; i += THREADS) all[i] = (uintx4){0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < EACH; ++i) sum += (double)x[i] * (double)x[i];
#pragma unroll
    for (int step = 1; step < 64; step *= 2) sum += __shfl_xor(sum, step);
    if (lane == 0) squares[wave] = sum;
    __syncthreads();
    sum = 0.0;
    for (int i = 0; i < WAVES; ++i) sum += squares[i];
    const double up = (double)p.first / (sqrt(sum) + (double)p.eps);
    xr = r0, xc = c0;
#pragma unroll
    for (int i = 0; i < EACH; ++i, next(xr, xc)) {
        if (xr >= height) continue;
        const uint32_t zr = p.transposed ? xc : xr, zc = p.transposed ? xr : xc;
        _Float16 h, low;
        cut((float)((double)x[i] * up), h, low);
        _Float16* to = (_Float16*)(z + zr * PZ + zc / 32 * 128 + zc % 32 * 2);
        to[0] = h;
        to[32] = low;
    }
    // a step's factors: a lane each
    const int mine = lane % SMALL_STEPS, m = wave / (L / 32) * 32, n = wave % (L / 32) * 32;
    const float gram = p.gram[mine], square = p.square[mine], by_gram = p.of_gram[mine], by_one = p.of_one[mine], by_next = p.next[mine];
    __syncthreads();
    floatx16 acc{};
    for (int step = 0;; ++step) {
        auto of_step = [&](float v) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), step)); };
        if (n < S) small_put(g, PG, m, n, small_product<false, L, PZ, PZ>(z, m, z, n), of_step(gram));
        __syncthreads();
        if (n < S) {
            acc = small_product<false, S, PG, PG>(g, m, g, n);
            const float up_square = of_step(square), of_gram = of_step(by_gram), of_one = of_step(by_one);
            const int r = m + (lane & 31), c = n + 4 * (lane >> 5);
            small_places(g, PG, m, n, [&](int q, const char* at) {
                const f16x4 h = *reinterpret_cast<const f16x4*>(at), low = *reinterpret_cast<const f16x4*>(at + 64);
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[4 * q + j] = fmaf(of_gram, (float)h[j] + (float)low[j], acc[4 * q + j] * up_square) + (r == c + 8 * q + j ? of_one : 0.0f);
            });
        }
        __syncthreads();
        if (n < S) small_put(g, PG, m, n, acc, 1.0f);
        __syncthreads();
        acc = small_product<true, S, PG, PZ>(g, m, z, n);
        if (step + 1 >= p.steps) break;
        __syncthreads();
        small_put(z, PZ, m, n, acc, of_step(by_next));
        __syncthreads();
    }
    const int r = m + (lane & 31);
    if (r >= p.rows) return;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int c = n + 8 * q + 4 * (lane >> 5);
        const float out[4] = {acc[4 * q] * p.last, acc[4 * q + 1] * p.last, acc[4 * q + 2] * p.last, acc[4 * q + 3] * p.last};
        if (!p.transposed) cbm_put(Y + r * ldy, c, p.columns, out);
        else
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c + j < p.columns) Y[(c + j) * ldy + r] = (T)out[j];
    }
}

int64_t rounded(int64_t bytes) { return (bytes + 255) / 256 * 256; }

// Largest |f| on [0, top] of an odd polynomial a x + b x^3 + c x^5, and of a + b x^2 + c x^4: at an end or where the slope is zero.
double largest(const float* abc, double top, bool odd) {
    const double a = abc[0], b = abc[1], c = abc[2];
    auto f = [&](double x) { return std::fabs((a + b * x * x + c * x * x * x * x) * (odd ? x : 1.0)); };
    double most = std::max(f(0.0), f(top));
    // odd: a + 3 b y + 5 c y^2 = 0 in y = x^2; even: x = 0 or b + 2 c y = 0
    double roots[2] = {-1.0, -1.0};
    if (odd) {
        const double q = 9 * b * b - 20 * a * c;
        if (c == 0.0) roots[0] = b == 0.0 ? -1.0 : -a / (3 * b);
        else if (q >= 0.0) {
            roots[0] = (-3 * b + std::sqrt(q)) / (10 * c);
            roots[1] = (-3 * b - std::sqrt(q)) / (10 * c);
        }
    } else if (c != 0.0) {
        roots[0] = -b / (2 * c);
    }
    for (double y : roots)
        if (y > 0.0 && y < top * top) most = std::max(most, f(std::sqrt(y)));
    return most;
}
// The power of two at which values up to `most` are kept: at most 2^14 there.
int power(double most) {
    if (!(most > 0.0)) return 0;
    return (int)std::max(-100.0, std::min(100.0, 14.0 - std::ceil(std::log2(most))));
}

// What a step multiplies its sums by: to the size that A is kept at, to P's, A as it is kept and one to P's, to the size that the next Z is kept at; and the power of two back to Z's own size.
// `top` and `up`, a bound of Z's singular values and the power that it is kept at, become the next Z's.
struct Powers {
    float gram, square, of_gram, of_one, next;
    int back;
    Powers(const float* abc, double& top, int& up) {
        const int up_gram = power(top * top), up_poly = power(largest(abc, top, false));
        top = largest(abc, top, true) * (1.0 + 0x1p-10);
        const int up_next = power(top);
        gram = (float)std::ldexp(1.0, up_gram - 2 * up);
        square = (float)std::ldexp((double)abc[2], up_poly - 2 * up_gram);
        of_gram = (float)std::ldexp((double)abc[1], up_poly - up_gram);
        of_one = (float)std::ldexp((double)abc[0], up_poly);
        next = (float)std::ldexp(1.0, up_next - up - up_poly);
        back = -up - up_poly;
        up = up_next;
    }
};

// Whether the bounds stay where the powers of two reach, 2^24 for Z and 2^100 for P, and near what they bound: singular values near zero, most of a matrix's, have |a| in P, and the lower parts of its values
// there would go below fp16's smallest if the bound were far above that (a, b, c = 2, -3, 50: 0.4 % off after two steps of 150 x 200).
bool stays(const float* abc, int steps) {
    double top = 1.0 + 0x1p-10;
    for (int i = 0; i < steps; ++i) {
        const double most = largest(abc, top, false);
        if (!(top <= 0x1p24) || !(most <= 0x1p100) || !(most <= 16.0 * std::fabs((double)abc[0]))) return false;
        top = largest(abc, top, true) * (1.0 + 0x1p-10);
    }
    return true;
}

struct Room {
    int64_t squares, z[2], zt[2], gram, poly, bytes;
};
Room room_of(int64_t s, int64_t l) {
    Room r;
    const int64_t z = rounded(Halves{nullptr, s, l}.bytes()), zt = rounded(Halves{nullptr, l, s}.bytes()), sq = rounded(Halves{nullptr, s, s}.bytes());
    r.squares = 0;
    r.z[0] = rounded(PARTS * 8);
    r.z[1] = r.z[0] + z;
    r.zt[0] = r.z[1] + z;
    r.zt[1] = r.zt[0] + zt;
    r.gram = r.zt[1] + zt;
    r.poly = r.gram + sq;
    r.bytes = r.poly + sq;
    return r;
}

// f(the tiles that take least)
template <class F>
void with_tiles(int64_t M, int64_t N, int64_t K, bool half, F&& f) {
    const int side = cbm_orthogonal_side(M, N, K, half);
    if (side == 256) f((HalvesTiles<256>*)nullptr);
    else if (side == 192) f((HalvesTiles<192>*)nullptr);
    else if (side == 128) f((HalvesTiles<128>*)nullptr);
    else if (side == 64) f((HalvesShares<64, 4>*)nullptr);
    else f((HalvesShares<32, 8>*)nullptr);
}

template <int MODE, class T>
void product(const ProductArgs& p, hipStream_t stream) {
    const bool half = MODE == GRAM || MODE == POLYNOMIAL;
    with_tiles(p.a.rows, p.b.rows, p.a.columns, half, [&](auto* tiles_type) {
        typedef std::remove_pointer_t<decltype(tiles_type)> Tiles;
        const int64_t m = (p.a.rows + Tiles::ROWS - 1) / Tiles::ROWS, tiles = half ? m * (m + 1) / 2 : m * ((p.b.rows + Tiles::ROWS - 1) / Tiles::ROWS);
        cbm_orthogonal_product_kernel<Tiles, MODE, T><<<(unsigned)((tiles + CBM_XCD - 1) / CBM_XCD * CBM_XCD), Tiles::THREADS, 0, stream>>>(p);
    });
}

}  // namespace

int64_t cbm_orthogonal_workspace(int32_t m, int32_t n, int32_t) { return room_of(std::min(m, n), std::max(m, n)).bytes; }

cbm_status cbm_launch_orthogonal(int32_t m, int32_t n, int32_t type, const void* X, int64_t ldx, int32_t steps, const float* abc, float eps, float scale, void* Y, int64_t ldy, void* workspace,
                                 void* stream_) {
    hipStream_t stream = (hipStream_t)stream_;
    if (!stays(abc, steps)) return CBM_ERR_UNSUPPORTED;
    const bool tall = m > n;
    const int64_t s = std::min(m, n), l = std::max(m, n);
    const Room room = room_of(s, l);
    char* base = (char*)workspace;
    double* squares = (double*)(base + room.squares);
    double top = 1.0 + 0x1p-10;  // a bound of Z's singular values
    int up = power(top);
    if (l <= (s <= 32 ? 512 : s <= 64 ? 256 : 128) && steps > 0 && steps <= SMALL_STEPS) {
        SmallArgs p{};
        p.rows = (int)s;
        p.columns = (int)l;
        p.steps = steps;
        p.transposed = tall;
        p.eps = eps;
        p.first = (float)std::ldexp(1.0, up);
        for (int i = 0; i < steps; ++i) {
            const Powers w(abc, top, up);
            p.gram[i] = w.gram;
            p.square[i] = w.square;
            p.of_gram[i] = w.of_gram;
            p.of_one[i] = w.of_one;
            p.next[i] = w.next;
            p.last = (float)std::ldexp((double)scale, w.back);
        }
        cbm_with_type(type, [&](auto t) {
            using T = decltype(t);
            auto go = [&](auto rows, auto columns) {
                constexpr int S = decltype(rows)::value, L = decltype(columns)::value;
                cbm_orthogonal_small_kernel<T, S, L><<<1, S * L / 16, 0, stream>>>(p, (const T*)X, ldx, (T*)Y, ldy);
            };
            using std::integral_constant;
            if (l <= 32) go(integral_constant<int, 32>{}, integral_constant<int, 32>{});
            else if (l <= 64) go(integral_constant<int, 64>{}, integral_constant<int, 64>{});
            else if (s <= 64 && l <= 128) go(integral_constant<int, 64>{}, integral_constant<int, 128>{});
            else if (l <= 128) go(integral_constant<int, 128>{}, integral_constant<int, 128>{});
            else if (s <= 32 && l <= 256) go(integral_constant<int, 32>{}, integral_constant<int, 256>{});
            else if (s <= 32) go(integral_constant<int, 32>{}, integral_constant<int, 512>{});
            else go(integral_constant<int, 64>{}, integral_constant<int, 256>{});
        });
        return cbm_launched("orthogonal update launch");
    }
    Halves z{(_Float16*)(base + room.z[0]), s, l}, zt{(_Float16*)(base + room.zt[0]), l, s};
    const Halves gram{(_Float16*)(base + room.gram), s, s}, poly{(_Float16*)(base + room.poly), s, s};
    cbm_with_type(type, [&](auto t) {
        using T = decltype(t);
        cbm_orthogonal_norm_kernel<T><<<PARTS, 256, 0, stream>>>(m, n, (const T*)X, ldx, squares);
        if (steps == 0) {
            cbm_orthogonal_scaled_kernel<T><<<(unsigned)std::min<int64_t>((s * l + 255) / 256, 1 << 20), 256, 0, stream>>>(m, n, (const T*)X, ldx, eps, scale, squares, (T*)Y, ldy);
            return;
        }
        cbm_orthogonal_begin_kernel<T><<<dim3((unsigned)((l + 31) / 32), (unsigned)((s + 31) / 32)), 256, 0, stream>>>((const T*)X, ldx, tall, eps, (float)std::ldexp(1.0, up), squares, z, zt);
        for (int i = 0; i < steps; ++i) {
            const Powers w(abc, top, up);
            ProductArgs p{};
            p.a = p.b = z;
            p.out = gram;
            p.up = w.gram;
            product<GRAM, float>(p, stream);
            p.a = p.b = p.gram = gram;
            p.out = poly;
            p.up = w.square;
            p.of_gram = w.of_gram;
            p.of_one = w.of_one;
            product<POLYNOMIAL, float>(p, stream);
            p.a = poly;
            p.b = zt;
            if (i + 1 < steps) {
                p.out = {(_Float16*)(base + room.z[(i + 1) % 2]), s, l};
                p.outt = {(_Float16*)(base + room.zt[(i + 1) % 2]), l, s};
                p.up = w.next;
                product<STEP, float>(p, stream);
                z = p.out;
                zt = p.outt;
            } else {
                p.Y = Y;
                p.ldy = ldy;
                p.transposed = tall;
                p.up = (float)std::ldexp((double)scale, w.back);
                product<LAST, T>(p, stream);
            }
        }
    });
    return cbm_launched("orthogonal update launch");
}
