// Layer norm over the rows of a matrix, forward and backward.
//   y = (x - m) r g + b,  m = mean(x),  r = (mean((x - m)^2) + eps)^-1/2 along a row of k columns;
//   with h = (x - m) r and u = dy g:  dx = r (u - mean(u) - h mean(u h)),  dg = sum over rows of dy h,  db = sum over rows of dy.
// All of it is bound by memory: 8 (forward) and 14 (backward) operations a value against 8 and 12 bytes in fp32.  A row is read once and stays in the registers of
// a group of lanes (a workgroup for wide rows), so the second pass of the variance, which keeps it exact where |m| is large beside the deviations, costs no
// traffic.  A sum of k values in fp32 leaves m off by some units of its last place: nothing beside deviations of |m| / 32, but more than those of a row of equal values.  Rows with smaller ones
// than that (`near_mean`) have m corrected by the mean of the deviations, and the squares added up anew (30000 x 4099 fp32 397 us for 260 where all of them do, 132534 x 100 22.5 for 19).
// Statistics and sums are fp32; y and dx are rounded once, to their type.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "cbm_elems.h"
#include "cbm_internal.h"

namespace {

typedef float floatx2 __attribute__((ext_vector_type(2)));
constexpr int NORM_THREADS = 256;
// Backward: rows that are read twice rather than joined by a second launch.  Microseconds a call, one launch or two: 300 x 4096 fp32 6.9 or 11.0, 300 x 8000 14.4 or 15.1, 600 x 8000 24.1
// or 18.0, 1024 x 512 6.4 or 8.2, 1024 x 1000 8.0 or 9.4, 1000 x 4096 17.7 or 14.5, 208 x 12064 bf16 14.4 or 17.0, 512 x 12064 25.0 or 21.4, 1024 x 2500 10.5 or 12.6; more rows are a longer
// walk for a lane: 2048 x 256 fp32 6.8 or 7.8, 2048 x 512 12.3 or 8.0, 4096 x 64 10 or 10.
bool few_rows(int64_t n, int k) { return (n <= 1024 && n * k <= 5 << 19) || (n <= 2048 && k <= 256); }
constexpr int BACK_THREADS = 512, BACK_GROUPS = 512;  // backward: workgroups at most, each with partial sums of dg and db of its own

// Sums of two values over a workgroup, in every thread.  `room` has a pair for every wave, twice: calls take turns (`turn`), so one barrier each is enough (who writes a
// room again has passed the barrier of the call between, and with it everybody's reads).
template <int THREADS>
__device__ __forceinline__ void block_sum2(float& a, float& b, floatx2* room, int& turn) {
    constexpr int WAVES = THREADS / 64;
    a = lanes_sum<64>(a);
    b = lanes_sum<64>(b);
    floatx2* mine = room + turn * WAVES;
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) mine[threadIdx.x / 64] = floatx2{a, b};
    __syncthreads();
    a = b = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        a += mine[w][0];
        b += mine[w][1];
    }
}
// over the LANES lanes of a row: part of a wave, or the whole workgroup
template <int LANES>
__device__ __forceinline__ void row_sum2(float& a, float& b, floatx2* room, int& turn) {
    if constexpr (LANES <= 64) {
        a = lanes_sum<LANES>(a);
        b = lanes_sum<LANES>(b);
    } else {
        block_sum2<LANES>(a, b, room, turn);
    }
}

// Whether there are deviations from m (v: their mean square), but so small ones that the rounding of m shows.  False for what is not finite: an infinity stays the mean.
__device__ __forceinline__ bool near_mean(float v, float m) { return v > 0.0f && v * 1024.0f < m * m; }

// V values of gamma or beta from `at` on; `other` where there are none.
template <int V>
__device__ __forceinline__ void load_columns(float (&x)[V], const float* p, int at, float other) {
    if (p) {
        constexpr int W = V < 4 ? V : 4;
#pragma unroll
        for (int w = 0; w < V; w += W) {
            float four[W];
            load_piece<W>(four, p + at + w);
#pragma unroll
            for (int j = 0; j < W; ++j) x[w + j] = four[j];
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = other;
    }
}

// The sums of a piece's columns, those that count.
template <int V, bool WHOLE>
__device__ __forceinline__ void store_columns(float* out, const float (&x)[V], const Place<V, WHOLE>& p) {
    if (p.seen <= 0) {
        constexpr int W = V < 4 ? V : 4;
#pragma unroll
        for (int w = 0; w < V; w += W) {
            float four[W];
#pragma unroll
            for (int j = 0; j < W; ++j) four[j] = x[w + j];
            store_piece<W>(out + p.at + w, four);
        }
    } else if (p.any()) {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (p.counts(j)) out[p.at + j] = x[j];
    }
}

// Forward.  LANES lanes have a row, each R pieces of V columns: as few lanes as hold a row in up to two pieces, so that a wave's reductions serve several rows, and a workgroup
// once a wave would need more than two.  The grid is what the compute units hold at once, and workgroups walk on over the rows, so gamma and beta are loaded once a workgroup
// (a workgroup for every few rows: 2097152 x 128 fp32 570 us for 454), in pieces of 16 bytes (value by value 16384 x 4096 bf16 took 68 us, so 54).  A row of one piece or two has as many
// lanes (1218193 x 8 bf16 9.1 us, with eight lanes a row 19).  Bound by memory: 2097152 x 128 fp32 440 us, 4.9 TB/s of 2.15 GB, waves waiting for 60 % of their cycles (a copy
// alone 386); rows of a workgroup of 1,024 by its barriers too: 30000 x 4099 259 us, a copy 171.  1024 x 64 2.7 us, a launch.
// Waves of a SIMD: two pieces of fp32 a lane fit eight, if only just (30000 x 1200 51 us, with seven 59).
template <int V, int LANES, int R>
constexpr int NORM_WAVES = V == 4 && LANES == 256 && R == 2 ? 8 : 1;
template <class T, int V, int LANES, int R, bool WHOLE>
__global__ __launch_bounds__(LANES > NORM_THREADS ? LANES : NORM_THREADS, (NORM_WAVES<V, LANES, R>)) void cbm_norm_kernel(int64_t n, int k, const T* __restrict__ X, int64_t ldx, const float* __restrict__ gamma,
                                                                                              const float* __restrict__ beta, float eps, T* __restrict__ Y, int64_t ldy,
                                                                                              float* __restrict__ mean, float* __restrict__ rstd, bool far) {
    constexpr int THREADS = LANES > NORM_THREADS ? LANES : NORM_THREADS, ROWS = THREADS / LANES;
    __shared__ floatx2 room[LANES > 64 ? 2 * (LANES / 64) : 1];
    const int lane = threadIdx.x % LANES;
    int turn = 0;
    float g[R][V], b[R][V];
#pragma unroll
    for (int c = 0; c < R; ++c) {
        const Place<V, WHOLE> p(c * LANES + lane, k);
        load_columns<V>(g[c], gamma, p.at, 1.0f);
        load_columns<V>(b[c], beta, p.at, 0.0f);
    }
    typename Piece<T, V>::type next[R];  // AHEAD: of the workgroup's next row, whose loads pass the barriers of this one
    constexpr bool AHEAD = LANES > 64;
    auto load = [&](int64_t row) {
        const T* x_row = X + (row < n ? row : n - 1) * ldx;
#pragma unroll
        for (int c = 0; c < R; ++c) next[c] = raw_piece<V>(x_row + Place<V, WHOLE>(c * LANES + lane, k).at);
    };
    if (AHEAD) load(blockIdx.x);
    for (int64_t row0 = (int64_t)blockIdx.x * ROWS; row0 < n; row0 += (int64_t)gridDim.x * ROWS) {
        const int64_t row = row0 + threadIdx.x / LANES;
        float x[R][V], sum = 0.0f, squares = 0.0f, none = 0.0f;
        if (!AHEAD) load(row);
#pragma unroll
        for (int c = 0; c < R; ++c) widen<V, T>(x[c], next[c]);
        if (AHEAD) load(row + gridDim.x);
#pragma unroll
        for (int c = 0; c < R; ++c) {
            const Place<V, WHOLE> p(c * LANES + lane, k);
#pragma unroll
            for (int j = 0; j < V; ++j) sum += p.counts(j) ? x[c][j] : 0.0f;
        }
        row_sum2<LANES>(sum, none, room, turn);
        float m = sum / (float)k;
#pragma unroll
        for (int c = 0; c < R; ++c) {
            const Place<V, WHOLE> p(c * LANES + lane, k);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                x[c][j] -= m;
                squares += p.counts(j) ? x[c][j] * x[c][j] : 0.0f;
            }
        }
        row_sum2<LANES>(squares, none, room, turn);
        const bool near = near_mean(squares / (float)k, m);
        if (LANES > 64 ? near : __any(near)) {  // (a wave's other rows take off 0, and keep their squares)
            float off = 0.0f, again = 0.0f;
#pragma unroll
            for (int c = 0; c < R; ++c) {
                const Place<V, WHOLE> p(c * LANES + lane, k);
#pragma unroll
                for (int j = 0; j < V; ++j) off += p.counts(j) ? x[c][j] : 0.0f;
            }
            row_sum2<LANES>(off, none, room, turn);
            off = near ? off / (float)k : 0.0f;
            m += off;
#pragma unroll
            for (int c = 0; c < R; ++c) {
                const Place<V, WHOLE> p(c * LANES + lane, k);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    x[c][j] -= off;
                    again += p.counts(j) ? x[c][j] * x[c][j] : 0.0f;
                }
            }
            row_sum2<LANES>(again, none, room, turn);
            squares = near ? again : squares;
        }
        const float r = 1.0f / sqrtf(squares / (float)k + eps);
        if (row >= n) continue;  // (only where a row is part of a wave: with a workgroup a row, row0 is the row)
        T* y_row = Y + row * ldy;
#pragma unroll
        for (int c = 0; c < R; ++c) {
            const Place<V, WHOLE> p(c * LANES + lane, k);
            float y[V];
#pragma unroll
            for (int j = 0; j < V; ++j) y[j] = x[c][j] * r * g[c][j] + b[c][j];
            if (p.any()) store_piece<V>(y_row + p.at, y, far);
        }
        if (lane == 0) {
            if (mean) mean[row] = m;
            if (rstd) rstd[row] = r;
        }
    }
}

// Rows of over 16,384 columns, too wide for registers: a workgroup reads its row three times (all but the first time out of L2), which the caches' rate bounds; five times if near its mean.
template <class T, int V, bool WHOLE>
__global__ __launch_bounds__(1024) void cbm_norm_wide_kernel(int64_t n, int k, const T* __restrict__ X, int64_t ldx, const float* __restrict__ gamma, const float* __restrict__ beta,
                                                             float eps, T* __restrict__ Y, int64_t ldy, float* __restrict__ mean, float* __restrict__ rstd, bool far) {
    __shared__ floatx2 room[32];
    int turn = 0;
    const int pieces = (k + V - 1) / V;
    for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
        const T* x_row = X + row * ldx;
        float x[V];
        auto mean_of = [&](auto&& f) {  // of f(value)
            float sum = 0.0f, none = 0.0f;
            for (int c = threadIdx.x; c < pieces; c += 1024) {
                const Place<V, WHOLE> p(c, k);
                load_piece<V>(x, x_row + p.at);
#pragma unroll
                for (int j = 0; j < V; ++j) sum += p.counts(j) ? f(x[j]) : 0.0f;
            }
            block_sum2<1024>(sum, none, room, turn);
            return sum / (float)k;
        };
        const float first = mean_of([](float v) { return v; });
        float m = first, off = 0.0f, variance = mean_of([=](float v) { return (v - first) * (v - first); });
        if (near_mean(variance, first)) {
            off = mean_of([=](float v) { return v - first; });
            m += off;
            variance = mean_of([=](float v) { return (v - first - off) * (v - first - off); });
        }
        const float r = 1.0f / sqrtf(variance + eps);
        for (int c = threadIdx.x; c < pieces; c += 1024) {
            const Place<V, WHOLE> p(c, k);
            load_piece<V>(x, x_row + p.at);
            float g[V], b[V];
            load_columns<V>(g, gamma, p.at, 1.0f);
            load_columns<V>(b, beta, p.at, 0.0f);
#pragma unroll
            for (int j = 0; j < V; ++j) x[j] = (x[j] - first - off) * r * g[j] + b[j];
            store_piece<V>(Y + row * ldy + p.at, x, far);
        }
        if (threadIdx.x == 0) {
            if (mean) mean[row] = m;
            if (rstd) rstd[row] = r;
        }
    }
}

// dg and db of 16 columns over all rows, by a workgroup whose every 16 lanes have a share of the rows.
template <class T, int THREADS>
__device__ __forceinline__ void columns_alone(int64_t n, int k, int first, const T* __restrict__ dY, int64_t lddy, const T* __restrict__ X, int64_t ldx, const float* __restrict__ mean,
                                              const float* __restrict__ rstd, float* __restrict__ dgamma, float* __restrict__ dbeta, floatx2* room) {
    constexpr int SHARES = THREADS / 16;
    const int column = first + (threadIdx.x & 15), share = threadIdx.x / 16;
    float dg = 0.0f, db = 0.0f;
    if (column < k)
#pragma unroll 8
        for (int64_t row = share; row < n; row += SHARES) {
            const float dy = (float)dY[row * lddy + column];
            dg += dy * (((float)X[row * ldx + column] - mean[row]) * rstd[row]);
            db += dy;
        }
    room[threadIdx.x] = floatx2{dg, db};
    __syncthreads();
    if (threadIdx.x >= 16 || column >= k) return;
    dg = db = 0.0f;
#pragma unroll 8
    for (int i = 0; i < SHARES; ++i) {
        dg += room[i * 16 + threadIdx.x][0];
        db += room[i * 16 + threadIdx.x][1];
    }
    if (dgamma) dgamma[column] = dg;
    if (dbeta) dbeta[column] = db;
}

// Backward in the same shape.  A lane has the same columns in all rows that it meets, so dg and db of these columns add up in its registers; a workgroup adds its
// lanes' sums in LDS, in a fixed order, and writes one partial row of each to `parts` (workgroup, dg then db, column).  With few rows a second launch would take longer than
// everything else: workgroups beyond the first `row_groups` then have dg and db of 16 columns each, and read all rows once more.
// Bound by memory: 132534 x 100 fp32 34.5 us for 159 MB (4.6 TB/s, waves waiting for 80 % of their cycles) and 4 to 5 for the join; 16384 x 4096 bf16 78 us with the join for
// 403 MB (5.2 TB/s).  Reading and writing as much, and nothing else: 29 and 72.
template <class T, int V, int LANES, int R, int THREADS, bool WHOLE>
__global__ __launch_bounds__(THREADS) void cbm_norm_back_kernel(int64_t n, int k, const T* __restrict__ dY, int64_t lddy, const T* __restrict__ X, int64_t ldx,
                                                                const float* __restrict__ gamma, const float* __restrict__ mean, const float* __restrict__ rstd,
                                                                T* __restrict__ dX, int64_t lddx, float* __restrict__ parts, int row_groups, float* __restrict__ dgamma,
                                                                float* __restrict__ dbeta, bool far) {
    constexpr int ROWS = THREADS / LANES;
    constexpr int COLUMNS = LANES * R * V;
    constexpr int ROOM = LANES > 64 ? 2 * (LANES / 64) : (THREADS / 64) * COLUMNS;
    __shared__ floatx2 room[ROOM > THREADS ? ROOM : THREADS];
    if ((int)blockIdx.x >= row_groups) {
        columns_alone<T, THREADS>(n, k, 16 * (blockIdx.x - row_groups), dY, lddy, X, ldx, mean, rstd, dgamma, dbeta, room);
        return;
    }
    const int lane = threadIdx.x % LANES;
    int turn = 0;
    float g[R][V], dg[R][V], db[R][V];
#pragma unroll
    for (int c = 0; c < R; ++c) {
        const Place<V, WHOLE> p(c * LANES + lane, k);
        load_columns<V>(g[c], gamma, p.at, 1.0f);
#pragma unroll
        for (int j = 0; j < V; ++j) dg[c][j] = db[c][j] = 0.0f;
    }
    typename Piece<T, V>::type next_x[R], next_dy[R];
    float next_m, next_r;
    constexpr bool AHEAD = LANES > 64 && (R * V <= 8 || (WHOLE && LANES < 1024));  // (as far as registers go)
    auto load = [&](int64_t row) {
        const int64_t at = row < n ? row : n - 1;
        const T *x_row = X + at * ldx, *dy_row = dY + at * lddy;
#pragma unroll
        for (int c = 0; c < R; ++c) {
            const Place<V, WHOLE> p(c * LANES + lane, k);
            next_x[c] = raw_piece<V>(x_row + p.at);
            next_dy[c] = raw_piece<V>(dy_row + p.at);
        }
        next_m = mean[at];
        next_r = rstd[at];
    };
    if (AHEAD) load(blockIdx.x);
    for (int64_t row0 = (int64_t)blockIdx.x * ROWS; row0 < n; row0 += (int64_t)row_groups * ROWS) {
        const int64_t row = row0 + threadIdx.x / LANES;
        float h[R][V], u[R][V], sum = 0.0f, along = 0.0f;
        if (!AHEAD) load(row);
#pragma unroll
        for (int c = 0; c < R; ++c) {
            widen<V, T>(h[c], next_x[c]);
            widen<V, T>(u[c], next_dy[c]);
        }
        const float m = next_m, r = next_r;
        int lane_now = lane;
        if constexpr (!WHOLE && R * V >= 16) asm volatile("" : "+v"(lane_now));  // (every row's comparisons anew: kept from row to row they need more scalar registers than there are)
        if (AHEAD) load(row + row_groups);
#pragma unroll
        for (int c = 0; c < R; ++c) {
            const Place<V, WHOLE> p(c * LANES + lane_now, k);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                h[c][j] = (h[c][j] - m) * r;
                const bool counts = p.counts(j) && row < n;
                const float dy = u[c][j];
                dg[c][j] += counts ? dy * h[c][j] : 0.0f;
                db[c][j] += counts ? dy : 0.0f;
                u[c][j] = dy * g[c][j];
                sum += counts ? u[c][j] : 0.0f;
                along += counts ? u[c][j] * h[c][j] : 0.0f;
            }
        }
        if (!dX) continue;
        row_sum2<LANES>(sum, along, room, turn);
        sum /= (float)k;
        along /= (float)k;
        if (row >= n) continue;
#pragma unroll
        for (int c = 0; c < R; ++c) {
            const Place<V, WHOLE> p(c * LANES + lane_now, k);
            float dx[V];
#pragma unroll
            for (int j = 0; j < V; ++j) dx[j] = r * (u[c][j] - sum - h[c][j] * along);
            if (p.any()) store_piece<V>(dX + row * lddx + p.at, dx, (WHOLE || R * V < 16) && far);  // (as far as registers go)
        }
    }
    if (!parts) return;
    float* out = parts + (int64_t)blockIdx.x * 2 * k;
    if constexpr (LANES > 64) {
#pragma unroll
        for (int c = 0; c < R; ++c) {
            const Place<V, WHOLE> p(c * LANES + lane, k);
            store_columns<V, WHOLE>(out, dg[c], p);
            store_columns<V, WHOLE>(out + k, db[c], p);
        }
    } else {
        const int wave = threadIdx.x / 64;
        __syncthreads();
#pragma unroll
        for (int c = 0; c < R; ++c)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float a = dg[c][j], b = db[c][j];
#pragma unroll
                for (int step = LANES; step < 64; step *= 2) {  // the rows of a wave
                    a += __shfl_xor(a, step);
                    b += __shfl_xor(b, step);
                }
                if ((threadIdx.x & 63) < LANES) {
                    const int slot = (c * LANES + lane) * V + j;
                    room[wave * COLUMNS + slot] = floatx2{a, b};
                }
            }
        __syncthreads();
        for (int slot = threadIdx.x; slot < COLUMNS; slot += THREADS) {
            const Place<V, WHOLE> p(slot / V, k);
            if (!p.counts(slot % V)) continue;
            float a = 0.0f, b = 0.0f;
#pragma unroll
            for (int w = 0; w < THREADS / 64; ++w) {
                a += room[w * COLUMNS + slot][0];
                b += room[w * COLUMNS + slot][1];
            }
            out[p.at + slot % V] = a;
            out[k + p.at + slot % V] = b;
        }
    }
}

// Rows too wide for registers: dx by a workgroup a row, which reads x and dy twice; dg and db by workgroups of 256 pieces and a share of the rows.
template <class T, int V, bool WHOLE>
__global__ __launch_bounds__(1024) void cbm_norm_back_wide_kernel(int64_t n, int k, const T* __restrict__ dY, int64_t lddy, const T* __restrict__ X, int64_t ldx,
                                                                  const float* __restrict__ gamma, const float* __restrict__ mean, const float* __restrict__ rstd,
                                                                  T* __restrict__ dX, int64_t lddx, bool far) {
    __shared__ floatx2 room[32];
    int turn = 0;
    const int pieces = (k + V - 1) / V;
    for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
        const float m = mean[row], r = rstd[row];
        float sum = 0.0f, along = 0.0f, x[V], dy[V];
        for (int c = threadIdx.x; c < pieces; c += 1024) {
            const Place<V, WHOLE> p(c, k);
            load_piece<V>(x, X + row * ldx + p.at);
            load_piece<V>(dy, dY + row * lddy + p.at);
            float g[V];
            load_columns<V>(g, gamma, p.at, 1.0f);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float u = dy[j] * g[j];
                sum += p.counts(j) ? u : 0.0f;
                along += p.counts(j) ? u * ((x[j] - m) * r) : 0.0f;
            }
        }
        block_sum2<1024>(sum, along, room, turn);
        sum /= (float)k;
        along /= (float)k;
        for (int c = threadIdx.x; c < pieces; c += 1024) {
            const Place<V, WHOLE> p(c, k);
            load_piece<V>(x, X + row * ldx + p.at);
            load_piece<V>(dy, dY + row * lddy + p.at);
            float g[V];
            load_columns<V>(g, gamma, p.at, 1.0f);
#pragma unroll
            for (int j = 0; j < V; ++j) x[j] = r * (dy[j] * g[j] - sum - (x[j] - m) * r * along);
            store_piece<V>(dX + row * lddx + p.at, x, far);
        }
    }
}
template <class T, int V, bool WHOLE>
__global__ __launch_bounds__(256) void cbm_norm_back_columns_kernel(int64_t n, int k, const T* __restrict__ dY, int64_t lddy, const T* __restrict__ X, int64_t ldx,
                                                                    const float* __restrict__ mean, const float* __restrict__ rstd, float* __restrict__ parts) {
    const Place<V, WHOLE> p(blockIdx.x * 256 + threadIdx.x, k);
    if (!p.any()) return;
    float dg[V] = {}, db[V] = {};
#pragma unroll 4
    for (int64_t row = blockIdx.y; row < n; row += gridDim.y) {
        float x[V], dy[V];
        load_piece<V>(x, X + row * ldx + p.at);
        load_piece<V>(dy, dY + row * lddy + p.at);
        const float m = mean[row], r = rstd[row];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            dg[j] += dy[j] * ((x[j] - m) * r);
            db[j] += dy[j];
        }
    }
    float* out = parts + (int64_t)blockIdx.y * 2 * k;
    store_columns<V, WHOLE>(out, dg, p);
    store_columns<V, WHOLE>(out + k, db, p);
}

// dg and db from `count` partial rows of each, in a fixed order: 32 columns a workgroup, the partial rows shared by its 32 groups of lanes, each with 16 loads under way.  Bound by
// the latency of a launch and of these loads: 512 x 100 4 to 5 us.
__global__ __launch_bounds__(1024) void cbm_norm_join_kernel(int count, int k, const float* __restrict__ parts, float* __restrict__ dgamma, float* __restrict__ dbeta) {
    __shared__ float room[32][33];
    const int which = blockIdx.y, column = blockIdx.x * 32 + (threadIdx.x & 31), slice = threadIdx.x / 32;
    float* out = which ? dbeta : dgamma;
    if (!out) return;  // (the whole workgroup)
    float s = 0.0f;
    if (column < k)
#pragma unroll 16
        for (int i = slice; i < count; i += 32) s += parts[((int64_t)i * 2 + which) * k + column];
    room[slice][threadIdx.x & 31] = s;
    __syncthreads();
    if (slice == 0 && column < k) {
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < 32; ++i) s += room[i][threadIdx.x];
        out[column] = s;
    }
}

cbm_status launched(const char* what) {
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return CBM_OK;
    cbm_set_error_detail(what, hipGetErrorString(e));
    return CBM_ERR_HIP;
}

int64_t at_most(int64_t rows, int rows_each, int64_t most) { return std::min<int64_t>((rows + rows_each - 1) / rows_each, most); }

// Backward: pieces of a row that stays in registers, and workgroups with partial rows of their own for a row of `pieces`.  Half as many (of twice the waves) where partial rows are long: 16384 x 4096 bf16
// 89.7 us with 512 workgroups, 85.2 with 256; 100000 x 1200 254 and 371.  Rows too wide for registers: eight a compute unit, each for 256 pieces and a share of the rows.
constexpr int64_t back_held(int v) { return (v == 4 ? 3 : 2) * 1024; }
int64_t back_groups(int v, int64_t pieces) {
    return pieces <= 384 ? BACK_GROUPS : pieces <= back_held(v) ? BACK_GROUPS / 2 : std::max<int64_t>(1, 2048 / ((pieces + 255) / 256));
}

// f(a value of the type, whether its 16-byte pieces divide a row of k)
template <class F>
void with_shape(int32_t type, int32_t k, F&& f) {
    cbm_with_type(type, [&](auto t) {
        if (k % (16 / (int)sizeof(t)) == 0) f(t, std::true_type{});
        else f(t, std::false_type{});
    });
}

}  // namespace

// Partial rows of the backward pass at most, whatever the type and with it the shape.
int64_t cbm_norm_parts(int64_t n, int32_t k) {
    return std::min(n, std::max(back_groups(4, ((int64_t)k + 3) / 4), back_groups(8, ((int64_t)k + 7) / 8)));
}

cbm_status cbm_launch_norm(int64_t n, int32_t k, int32_t type, const void* X_, int64_t ldx, const float* gamma, const float* beta, float eps, void* Y_, int64_t ldy,
                           float* mean, float* rstd, void* stream_) {
    if (n == 0) return CBM_OK;
    hipStream_t stream = (hipStream_t)stream_;
    with_shape(type, k, [&](auto t, auto whole) {
        using T = decltype(t);
        constexpr bool WHOLE = decltype(whole)::value;
        const T* X = (const T*)X_;
        T* Y = (T*)Y_;
        constexpr int V = 16 / (int)sizeof(T);
        const int64_t pieces = ((int64_t)k + V - 1) / V;
        const bool far = n * k * (int64_t)sizeof(T) >= CBM_FAR_BYTES;
#define CBM_NORM(V_, LANES, R)                                                                                                                                                        \
    cbm_norm_kernel<T, V_, LANES, R, WHOLE><<<(unsigned)at_most(n, (LANES > NORM_THREADS ? LANES : NORM_THREADS) / LANES, 256 * (LANES == 1024 ? 1 : LANES > NORM_THREADS ? 2 : 8)), \
                                              LANES > NORM_THREADS ? LANES : NORM_THREADS, 0, stream>>>(n, k, X, ldx, gamma, beta, eps, Y, ldy, mean, rstd, far)
        if (k <= V) {
            if constexpr (WHOLE) CBM_NORM(V, 1, 1);
            else cbm_narrow_row<V>(k, [&](auto v, auto lanes) { CBM_NORM(v(), lanes(), 1); });
        } else if (pieces <= 2) CBM_NORM(V, 2, 1);
        else if (pieces <= 4) CBM_NORM(V, 4, 1);
        else if (pieces <= 8) CBM_NORM(V, 8, 1);
        else if (pieces <= 16) CBM_NORM(V, 16, 1);
        else if (pieces <= 32) CBM_NORM(V, 32, 1);
        else if (pieces <= 64) CBM_NORM(V, 64, 1);
        else if (pieces <= 128) CBM_NORM(V, 64, 2);
        else if (pieces <= 256) CBM_NORM(V, 256, 1);
        else if (pieces <= 512) CBM_NORM(V, 256, 2);
        else if (pieces <= 1024) CBM_NORM(V, 512, 2);
        else if (V == 4 && pieces <= 2048) CBM_NORM(V, 1024, 2);
        else if (k <= 16384) CBM_NORM(V, 1024, 16 / V);
        else hipLaunchKernelGGL((cbm_norm_wide_kernel<T, V, WHOLE>), dim3((unsigned)std::min<int64_t>(n, 512)), dim3(1024), 0, stream, n, k, X, ldx, gamma, beta, eps, Y, ldy, mean, rstd, far);
#undef CBM_NORM
    });
    return launched("layer norm launch");
}

cbm_status cbm_launch_norm_backward(int64_t n, int32_t k, int32_t type, const void* dY_, int64_t lddy, const void* X_, int64_t ldx, const float* gamma, const float* mean,
                                    const float* rstd, void* dX_, int64_t lddx, float* dgamma, float* dbeta, float* parts, void* stream_) {
    hipStream_t stream = (hipStream_t)stream_;
    int64_t count = 0;  // partial rows written
    const bool sums = dgamma || dbeta;
    bool joined = !sums;
    if (!sums) parts = nullptr;
    if (n > 0)
        with_shape(type, k, [&](auto t, auto whole) {
            using T = decltype(t);
            constexpr bool WHOLE = decltype(whole)::value;
            const T *dY = (const T*)dY_, *X = (const T*)X_;
            T* dX = (T*)dX_;
            constexpr int V = 16 / (int)sizeof(T);
            const int64_t pieces = ((int64_t)k + V - 1) / V, groups = back_groups(V, pieces);
            const bool far = n * k * (int64_t)sizeof(T) >= CBM_FAR_BYTES;
            const bool once = sums && few_rows(n, k) && pieces <= back_held(V);  // (dg and db in the same launch)
            const unsigned alone = once ? (unsigned)(((int64_t)k + 15) / 16) : 0;
            if (once) parts = nullptr;
#define CBM_BACK(V_, LANES, R, THREADS)                                                                                                                                                   \
    (count = at_most(n, THREADS / LANES, groups),                                                                                                                                   \
     cbm_norm_back_kernel<T, V_, LANES, R, THREADS, WHOLE><<<(unsigned)(dX || !once ? count : 0) + alone, THREADS, 0, stream>>>(n, k, dY, lddy, X, ldx, gamma, mean, rstd, dX, lddx, parts, \
                                                                                                                               dX || !once ? (int)count : 0, dgamma, dbeta, far),      \
     joined = once)
            if (k <= V) {
                if constexpr (WHOLE) CBM_BACK(V, 1, 1, BACK_THREADS);
                else cbm_narrow_row<V>(k, [&](auto v, auto lanes) { CBM_BACK(v(), lanes(), 1, BACK_THREADS); });
            } else if (pieces <= 2) CBM_BACK(V, 2, 1, BACK_THREADS);
            else if (pieces <= 4) CBM_BACK(V, 4, 1, BACK_THREADS);
            else if (pieces <= 8) CBM_BACK(V, 8, 1, BACK_THREADS);
            else if (pieces <= 16) CBM_BACK(V, 16, 1, BACK_THREADS);
            else if (pieces <= 32) CBM_BACK(V, 32, 1, BACK_THREADS);
            else if (pieces <= 64) CBM_BACK(V, 64, 1, BACK_THREADS);
            else if (pieces <= 128) CBM_BACK(V, 64, 2, 256);
            else if (pieces <= 256) CBM_BACK(V, 256, 1, 256);
            else if (pieces <= 384) CBM_BACK(V, 256, 2, 256);
            else if (pieces <= 512) CBM_BACK(V, 512, 1, 512);
            else if (pieces <= 1024) CBM_BACK(V, 512, 2, 512);
            else if (V == 4 && pieces <= 2048) CBM_BACK(V, 1024, 2, 1024);
            else if (pieces <= back_held(V)) CBM_BACK(V, 1024, V == 4 ? 3 : 2, 1024);
            else {
                if (dX) hipLaunchKernelGGL((cbm_norm_back_wide_kernel<T, V, WHOLE>), dim3((unsigned)std::min<int64_t>(n, 512)), dim3(1024), 0, stream, n, k, dY, lddy, X, ldx, gamma, mean, rstd, dX, lddx, far);
                count = std::min(n, groups);
                if (parts)
                    cbm_norm_back_columns_kernel<T, V, WHOLE><<<dim3((unsigned)((pieces + 255) / 256), (unsigned)count), 256, 0, stream>>>(n, k, dY, lddy, X, ldx, mean, rstd, parts);
            }
#undef CBM_BACK
        });
    if (!joined) hipLaunchKernelGGL(cbm_norm_join_kernel, dim3((unsigned)(((int64_t)k + 31) / 32), 2), dim3(1024), 0, stream, (int)count, k, parts, dgamma, dbeta);
    return launched("layer norm backward launch");
}
