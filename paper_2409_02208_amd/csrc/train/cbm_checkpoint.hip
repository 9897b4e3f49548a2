// Activations kept in 8 bits until the backward pass.  32 columns of a row share a step 2^e, e six below the exponent of the largest of them:
//   q = sign(x) min(127, max(1, round(|x| 2^-e))), 0 for 0;  x~ = q 2^e.
// A step that is a power of two costs half a bit against largest / 127, and gives: quotients and x~ that are exact, a byte a step, and x~ that is a bf16 value, so that
// the weights' gradient takes one operand of the matrix cores as it is.  Values other than zero keep a step at least, so the sign, and with it a ReLU's mask, is kept.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "cbm_elems.h"
#include "cbm_internal.h"
#include "cbm_split.h"

namespace {

constexpr int BLOCK = 32;      // columns that share a step
constexpr int NOT_FINITE = 255;  // the code of a block that holds a value that is not finite: all of it comes back NaN

__device__ __forceinline__ float step_of(uint32_t code) { return __uint_as_float(code << 23); }  // 2^(code - 127); of NOT_FINITE: infinity
__device__ __forceinline__ float value_of(int q, uint32_t code) { return code == NOT_FINITE ? NAN : (float)q * step_of(code); }

// What a lane has of a row: V columns from `at` on, the first `seen` of them another lane's; fewer than V columns where the row has no more (k < V).
template <int V, class T>
__device__ __forceinline__ void load_row_piece(float (&x)[V], const T* row, const Place<V, false>& p, int k) {
    if (k >= V) {
        load_piece<V>(x, row + p.at);
    } else {  // (at < 0: column at + j from 0 on)
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = p.at + j >= 0 ? (float)row[p.at + j] : 0.0f;
    }
}
// How many values of a piece may be another lane's as well for the lane to write all of it: in a row's last piece they get the same bits from both lanes where they share the step (and a gradient in
// place, gated twice, is gated once).
template <int V>
__device__ __forceinline__ int most_seen(int k) {
    return k >= V && (k - V) / BLOCK == (k - 1) / BLOCK ? V - 1 : 0;
}
template <int V>
__device__ __forceinline__ void load_row_bytes(int (&q)[V], const int8_t* row, const Place<V, false>& p, int k) {
    if (k >= V) {
        const typename Piece<int8_t, V>::type v = *reinterpret_cast<const typename Piece<int8_t, V>::type*>(row + p.at);
#pragma unroll
        for (int j = 0; j < V; ++j) q[j] = v[j];
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) q[j] = p.at + j >= 0 ? row[p.at + j] : 0;
    }
}

// Save.  LANES lanes a row (and a share of its columns: blockIdx.y), V columns a lane, of R rows; of R places along the row where a wave has it (R = 2).  A block of 32 columns is 32 / V lanes, which find its largest value by DPP; nothing
// else is shared.  Bound by the latency of a lane's few loads: 19717 x 500 fp32 11 to 13 us for 49.6 MB (4 TB/s; waves waiting for 64 % of their cycles; reading and writing as much, and nothing else, 8).
template <class T, int LANES, int R>
__global__ __launch_bounds__(256) void cbm_checkpoint_save_kernel(int64_t n, int k, const T* __restrict__ X, int64_t ldx, int8_t* __restrict__ Q, int64_t ldq,
                                                                  uint8_t* __restrict__ E, int64_t lde) {
    constexpr int V = 16 / (int)sizeof(T), PER_BLOCK = BLOCK / V;
    constexpr int ROWS = 256 / LANES, ACROSS = LANES == 64 ? R : 1, DOWN = LANES == 64 ? 1 : R;
    const int lane = threadIdx.x % LANES, first = blockIdx.y * ACROSS * LANES + lane, blocks = (k + BLOCK - 1) / BLOCK, most = most_seen<V>(k);
    for (int64_t row0 = (int64_t)blockIdx.x * (DOWN * ROWS) + threadIdx.x / LANES; row0 < n; row0 += (int64_t)gridDim.x * (DOWN * ROWS)) {
        float x[R][V];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int64_t row = min(row0 + i % DOWN * ROWS, n - 1);
            load_row_piece<V>(x[i], X + row * ldx, Place<V, false>(first + i % ACROSS * LANES, k), k);
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int64_t row = row0 + i % DOWN * ROWS;
            if (DOWN > 1 && row >= n) break;
            int c = first + i % ACROSS * LANES;
            asm volatile("" : "+v"(c));  // (every row's comparisons anew: kept from row to row they are more than the scalar registers hold)
            const Place<V, false> p(c, k);
            // the largest size by its bits, which order sizes, infinity and NaN as they should
            uint32_t largest = 0;
#pragma unroll
            for (int j = 0; j < V; ++j) largest = max(largest, p.counts(j) ? __float_as_uint(x[i][j]) & 0x7fffffffu : 0u);
            if constexpr (LANES >= 2) largest = max(largest, lane_other<1>(largest));
            if constexpr (LANES >= 4) largest = max(largest, lane_other<2>(largest));
            if constexpr (LANES >= 8 && PER_BLOCK == 8) largest = max(largest, lane_other<4>(largest));
            const bool finite = largest < 0x7f800000u;
            const uint32_t code = finite ? (uint32_t)max((int)(largest >> 23) - 6, 1) : NOT_FINITE;
            const float up = __uint_as_float((254u - (finite ? code : 127u)) << 23);
            uint32_t packed[V / 4];
#pragma unroll
            for (int w = 0; w < V / 4; ++w) {
                packed[w] = 0;
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const float v = x[i][4 * w + b], size = fminf(fmaxf(rintf(fabsf(v) * up), 1.0f), 127.0f);
                    const int q = v == 0.0f || !finite ? 0 : (int)copysignf(size, v);
                    packed[w] |= ((uint32_t)q & 255u) << (8 * b);
                }
            }
            int8_t* out = Q + row * ldq + p.at;
            if (p.seen <= most) {
                typedef uint32_t Words __attribute__((ext_vector_type(V / 4), aligned(1)));
                Words words;
#pragma unroll
                for (int w = 0; w < V / 4; ++w) words[w] = packed[w];
                *reinterpret_cast<Words*>(out) = words;
            } else if (p.any()) {
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (p.counts(j)) out[j] = (int8_t)(packed[j / 4] >> (8 * (j % 4)));
            }
            if (c % PER_BLOCK == 0 && c / PER_BLOCK < blocks) E[row * lde + c / PER_BLOCK] = (uint8_t)code;
        }
    }
}

// Restore, and the backward pass of a ReLU (GATED: dx = q > 0 ? dy : 0), in the shape of saving.  Bound by memory: 19717 x 500 restored to fp32 8.6 to 10 us for 49.6 MB (5 TB/s);
// gated, 235868 x 128 bf16 32 us for 152 MB (4.7 TB/s; waves waiting for 82 % of their cycles: a piece of each stream a lane).  Reading and writing as much, and nothing else: 8 and 21, some of it out of the
// memory-side cache.
template <class T, int LANES, int R, bool GATED>
__global__ __launch_bounds__(256) void cbm_checkpoint_load_kernel(int64_t n, int k, const int8_t* __restrict__ Q, int64_t ldq, const uint8_t* __restrict__ E, int64_t lde, const T* dY,
                                                                  int64_t lddy, T* out, int64_t ldo, bool far) {
    constexpr int V = 16 / (int)sizeof(T);
    constexpr int ROWS = 256 / LANES, ACROSS = LANES == 64 ? R : 1, DOWN = LANES == 64 ? 1 : R;
    const int lane = threadIdx.x % LANES, first = blockIdx.y * ACROSS * LANES + lane, blocks = (k + BLOCK - 1) / BLOCK, most = most_seen<V>(k);
    for (int64_t row0 = (int64_t)blockIdx.x * (DOWN * ROWS) + threadIdx.x / LANES; row0 < n; row0 += (int64_t)gridDim.x * (DOWN * ROWS)) {
        int q[R][V];
        float x[R][V];
        uint32_t code[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int64_t row = min(row0 + i % DOWN * ROWS, n - 1);
            const Place<V, false> p(first + i % ACROSS * LANES, k);
            load_row_bytes<V>(q[i], Q + row * ldq, p, k);
            if constexpr (GATED) load_row_piece<V>(x[i], dY + row * lddy, p, k);
            code[i] = E[row * lde + min((first + i % ACROSS * LANES) * V / BLOCK, blocks - 1)];
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int64_t row = row0 + i % DOWN * ROWS;
            if (DOWN > 1 && row >= n) break;
            int c = first + i % ACROSS * LANES;
            asm volatile("" : "+v"(c));  // (as above)
            const Place<V, false> p(c, k);
#pragma unroll
            for (int j = 0; j < V; ++j) x[i][j] = !GATED ? value_of(q[i][j], code[i]) : code[i] == NOT_FINITE ? NAN : q[i][j] > 0 ? x[i][j] : 0.0f;
            T* to = out + row * ldo + p.at;
            if (p.seen <= most) {
                store_piece<V>(to, x[i], far);
            } else if (p.any()) {
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (p.counts(j)) to[j] = (T)x[i][j];
            }
        }
    }
}

// dW = X~^T dY, a sum over the rows.  Both operands lie along their columns in memory and the matrix cores want eight rows of a column in a lane, so a lane loads, for
// eight rows, MT (4) neighbouring columns of Q and NT (2) of dY: 32 MT columns of Q and 32 NT of dY by 16 rows a wave, with neither LDS nor transposes, only with columns of dW
// in an order of their own (tile t has columns MT i + t of Q, and NT i + t of dY).  x~ is a bf16 value; dY is split into one (bf16), two (fp16) or three (fp32) bf16 values that add
// up to it, so the products are exact and the sums fp32.  The waves of a workgroup and the workgroups of a tile share the rows; a workgroup adds its waves' sums in LDS, in order.
// Narrow matrices take narrow tiles, of which a compute unit holds two workgroups (524288 x 32, 32 columns of bf16 45 us with wide tiles, 20 with narrow ones).
// The next step's loads are under way while a step is multiplied; two steps ahead cost registers and gained nothing (279 us, 292).  2097152 x 128, 128 columns of fp32: 275 us for
// 1.35 GB (4.9 TB/s; reading alone takes 209) and 206 GFLOP of parts (750 TFLOP/s, the matrix cores busy for 40 % of the cycles): waves wait for a quarter of their cycles only, so it is bound by the vector
// instructions that split dY and widen Q between the matrix instructions.  Several tiles do both again for each: 300000 x 300, 100 columns 112 us, reading alone 33.  132534 x 100, 47 columns: 16 us, of which 5.5 are there whatever the rows (the launch, first loads, sums in LDS).
constexpr int GRAD_WAVES = 8, GRAD_ROWS = 16;
int grad_mt(int32_t k) { return k <= 32 ? 1 : k <= 64 ? 2 : 4; }
int grad_nt(int32_t c) { return c <= 32 ? 1 : 2; }
constexpr int grad_groups(int mt, int nt) { return mt <= 2 && nt == 1 ? 2 : 1; }  // workgroups in a compute unit

template <int MT>
struct GradWord {
    typedef uint32_t type __attribute__((aligned(1)));
};
template <>
struct GradWord<2> {
    typedef uint16_t type __attribute__((aligned(1)));
};
template <>
struct GradWord<1> {
    typedef uint8_t type;
};
template <class T, int MT, int NT>
struct GradStep {  // what a lane has loaded: eight rows
    typename GradWord<MT>::type q[8];
    T y[8][NT];
    uint8_t e;  // of row lane / 4 of the sixteen, and block lane % 4 of the tile's columns
};
template <class T>
struct GradArgs {
    int64_t n;
    int k, c;
    const int8_t* Q;
    int64_t ldq;
    const uint8_t* E;
    int64_t lde;
    const T* dY;
    int64_t lddy;
};
template <int NT, class T>
__device__ __forceinline__ void grad_values(T (&to)[NT], const T* y) {
    const auto v = raw_piece<NT>(y);
#pragma unroll
    for (int u = 0; u < NT; ++u) to[u] = v[u];
}
// Rows row0 + 8 half .. + 7 (of the last row where there are none), MT columns of Q from at_q on and NT of dY from at_y.
template <class T, int MT, int NT>
__device__ __forceinline__ void grad_load(GradStep<T, MT, NT>& s, const GradArgs<T>& a, int64_t row0, int at_q, int at_y, int half, int block) {
    s.e = a.E[min(row0 + (int)(threadIdx.x & 63) / 4, a.n - 1) * a.lde + block];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int64_t at = min(row0 + 8 * half + j, a.n - 1);
        s.q[j] = *reinterpret_cast<const typename GradWord<MT>::type*>(a.Q + at * a.ldq + at_q);
        grad_values<NT>(s.y[j], a.dY + at * a.lddy + at_y);
        __builtin_amdgcn_sched_barrier(0);  // (a row's addresses at a time: registers)
    }
}
// The same for rows that are all there, with what all lanes share of an address in scalar registers and a lane's own 32 bits beside it (64-bit products of a row and
// a stride for each load of each lane took more time than everything else).
template <class T, int MT, int NT>
__device__ __forceinline__ void grad_load_whole(GradStep<T, MT, NT>& s, const GradArgs<T>& a, int64_t row0, uint32_t of_q, uint32_t of_e, uint32_t of_y) {
    const char *q = (const char*)a.Q + row0 * a.ldq, *e = (const char*)a.E + row0 * a.lde, *y = (const char*)(a.dY + row0 * a.lddy);
    s.e = *reinterpret_cast<const uint8_t*>(e + of_e);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        s.q[j] = *reinterpret_cast<const typename GradWord<MT>::type*>(q + j * (uint32_t)a.ldq + of_q);
        grad_values<NT>(s.y[j], reinterpret_cast<const T*>(y + j * (uint32_t)(a.lddy * sizeof(T)) + of_y));
    }
}

// near: eight rows are within 32 bits of an address.  SHIFT: MT does not divide k, or NT not c (2097152 x 128, 128 columns of bf16 160 us without shifts, 173 with them).
template <class T, int MT, int NT, bool SHIFT>
__global__ __launch_bounds__(64 * GRAD_WAVES, 2 * grad_groups(MT, NT)) void cbm_checkpoint_grad_kernel(GradArgs<T> a, int tiles_c, int tiles, int splits, float* __restrict__ parts, int64_t ldp,
                                                                                                    int64_t part, bool near) {
    constexpr int PARTS = std::is_same<T, float>::value ? 3 : std::is_same<T, _Float16>::value ? 2 : 1;  // 24, 11 and 8 bits, eight a part
    __shared__ floatx2 room[GRAD_WAVES * NT * 8 * 64];
    // workgroup b runs on XCD b mod 8: what an XCD has is neighbouring shares of the rows, all tiles of each as far as that goes
    const int per = gridDim.x / CBM_XCD, at = blockIdx.x % CBM_XCD * per + blockIdx.x / CBM_XCD, split = at / tiles, tile = at % tiles;
    if (split >= splits) return;
    const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int k0 = tile / tiles_c * (32 * MT) + MT * (lane & 31), c0 = tile % tiles_c * (32 * NT) + NT * (lane & 31);
    const int at_q = min(k0, a.k - MT), at_y = min(c0, a.c - NT);  // (the last load of a row starts earlier, and is shifted)
    const int late_q = 8 * min(k0 - at_q, MT - 1);                 // bits before the lane's first column in what it loads
    const bool late_y = NT == 2 && c0 > at_y;
    const int64_t steps = (a.n + GRAD_ROWS - 1) / GRAD_ROWS;
    const int64_t first = steps * split / splits, last = steps * (split + 1) / splits;
    floatx16 acc[MT][NT];
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int u = 0; u < NT; ++u)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[t][u][v] = 0.0f;
    uint32_t minus_low = 0xbf80u;
    asm("" : "+s"(minus_low));
    const int block = min(tile / tiles_c * MT + min(lane & 3, MT - 1), (a.k + BLOCK - 1) / BLOCK - 1), from = (32 * half + (lane & 31) / (32 / MT)) * 4;
    const uint32_t of_q = (uint32_t)(8 * half * a.ldq + at_q), of_e = (uint32_t)(lane / 4 * a.lde + block), of_y = (uint32_t)((8 * half * a.lddy + at_y) * (int64_t)sizeof(T));
    GradStep<T, MT, NT> next;
    auto load = [&](int64_t step) {
        if (!near || (step + 1) * GRAD_ROWS > a.n) grad_load<T, MT, NT>(next, a, step * GRAD_ROWS, at_q, at_y, half, block);
        else grad_load_whole<T, MT, NT>(next, a, step * GRAD_ROWS, of_q, of_e, of_y);
    };
    if (first + wave < last) load(first + wave);
    for (int64_t i = first + wave; i < last; i += GRAD_WAVES) {
        struct {
            uint32_t q[8];
            float step[8], y[NT][8];
        } s;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            s.q[j] = SHIFT ? (uint32_t)next.q[j] >> late_q : (uint32_t)next.q[j];
            s.step[j] = step_of(__builtin_amdgcn_ds_bpermute(from + 16 * j, (int)next.e));
            s.y[NT - 1][j] = (float)next.y[j][NT - 1];
            if constexpr (NT == 2) s.y[0][j] = (float)(SHIFT && late_y ? next.y[j][1] : next.y[j][0]);
        }
        if ((i + 1) * GRAD_ROWS > a.n) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (i * GRAD_ROWS + 8 * half + j >= a.n) {
                    s.q[j] = 0;
                    s.step[j] = 1.0f;
#pragma unroll
                    for (int u = 0; u < NT; ++u) s.y[u][j] = 0.0f;
                }
        }
        if (i + GRAD_WAVES < last) load(i + GRAD_WAVES);
        uintx4 y[NT][PARTS];
        if constexpr (PARTS == 1) {
#pragma unroll
            for (int u = 0; u < NT; ++u)
#pragma unroll
                for (int j = 0; j < 4; ++j) y[u][0][j] = high_halves(s.y[u][2 * j], s.y[u][2 * j + 1]);
        } else {
            float odd = 0.0f;  // NaN where a value of dY has no parts
#pragma unroll
            for (int u = 0; u < NT; ++u)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t part[3];
                    split_pair_nearest(s.y[u][2 * j], s.y[u][2 * j + 1], minus_low, part[0], part[1], part[2]);
                    odd = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, part[1]), __builtin_bit_cast(bf16x2, 0u), odd, false);
#pragma unroll
                    for (int p = 0; p < PARTS; ++p) y[u][p][j] = part[p];
                }
            if (__any(odd != odd)) {  // values that are not finite, which are their own high part, or that round up to infinity: parts by truncation
#pragma unroll
                for (int u = 0; u < NT; ++u)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float v0 = s.y[u][2 * j], v1 = s.y[u][2 * j + 1];
                        const bool fine0 = fabsf(v0) < INFINITY, fine1 = fabsf(v1) < INFINITY;
                        uint32_t part[3];  // (with zeros: the remainder of one value reads the parts of both)
                        split_pair(fine0 ? v0 : 0.0f, fine1 ? v1 : 0.0f, minus_low, part[0], part[1], part[2]);
                        y[u][0][j] = part[0] | (fine0 ? 0u : (__float_as_uint(v0) >> 16) | (v0 != v0 ? 0x40u : 0u)) |
                                     (fine1 ? 0u : (__float_as_uint(v1) & 0xffff0000u) | (v1 != v1 ? 0x400000u : 0u));
#pragma unroll
                        for (int p = 1; p < PARTS; ++p) y[u][p][j] = part[p];
                    }
            }
        }
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            uintx4 x;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float v[2];
#pragma unroll
                for (int w = 0; w < 2; ++w) v[w] = (float)(int8_t)(s.q[2 * j + w] >> (8 * t)) * s.step[2 * j + w];  // (NOT_FINITE: 0 times infinity)
                x[j] = high_halves(v[0], v[1]);
            }
#pragma unroll
            for (int p = PARTS - 1; p >= 0; --p)
#pragma unroll
                for (int u = 0; u < NT; ++u)
                    acc[t][u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y[u][p]), acc[t][u], 0, 0, 0);
        }
    }
    // The waves' sums, a tile of Q's columns at a time: every wave writes its own, then every thread adds two rows of NT neighbouring columns.
    float* out = parts + split * part;
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        __syncthreads();
#pragma unroll
        for (int u = 0; u < NT; ++u)
#pragma unroll
            for (int v = 0; v < 8; ++v) room[((wave * NT + u) * 8 + v) * 64 + lane] = floatx2{acc[t][u][2 * v], acc[t][u][2 * v + 1]};
        __syncthreads();
        floatx2 sum[NT] = {};
#pragma unroll
        for (int w = 0; w < GRAD_WAVES; ++w)
#pragma unroll
            for (int u = 0; u < NT; ++u) {
                const floatx2 x = room[((w * NT + u) * 8 + wave) * 64 + lane];
                sum[u][0] += x[0];
                sum[u][1] += x[1];
            }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int v = 2 * wave + i, row = tile / tiles_c * (32 * MT) + MT * (8 * (v / 4) + 4 * half + v % 4) + t;
            float* to = out + (int64_t)row * ldp + c0;
            if (row < a.k && c0 + NT <= a.c) {
                float all[NT];
#pragma unroll
                for (int u = 0; u < NT; ++u) all[u] = sum[u][i];
                store_piece<NT>(to, all);
            } else if (row < a.k && c0 < a.c) {
                *to = sum[0][i];
            }
        }
    }
}

// dW from `count` partial sums, in order: 1024 / SLICES values a workgroup, the partial sums shared by its SLICES groups of lanes.  Bound by the latency of a launch and of the loads of
// a lane, so few partial sums have few slices and a lane up to 16 loads: 256 of 100 x 47 (32 slices) 4 to 5 us, 24 of 572 x 94 (4) 4.7 (8.3 with 32), 4 of 1024 x 512 (1) 5.
template <int SLICES>
__global__ __launch_bounds__(1024) void cbm_checkpoint_join_kernel(int count, int64_t size, int c, const float* __restrict__ parts, float* __restrict__ dW, int64_t lddw) {
    constexpr int VALUES = 1024 / SLICES;
    __shared__ float room[SLICES > 1 ? SLICES : 1][VALUES + 1];
    const int slice = threadIdx.x / VALUES, mine = threadIdx.x % VALUES;
    for (int64_t i0 = (int64_t)blockIdx.x * VALUES; i0 < size; i0 += (int64_t)gridDim.x * VALUES) {
        const int64_t i = i0 + mine;
        float s = 0.0f;
        if (i < size)
#pragma unroll 16
            for (int p = slice; p < count; p += SLICES) s += parts[p * size + i];
        if constexpr (SLICES > 1) {
            room[slice][mine] = s;
            __syncthreads();
            s = 0.0f;
            if (slice == 0)
#pragma unroll
                for (int p = 0; p < SLICES; ++p) s += room[p][mine];
        }
        if (slice == 0 && i < size) dW[i / c * lddw + i % c] = s;
        if constexpr (SLICES > 1) __syncthreads();
    }
}

cbm_status launched(const char* what) {
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return CBM_OK;
    cbm_set_error_detail(what, hipGetErrorString(e));
    return CBM_ERR_HIP;
}

// f(lanes a row, pieces a lane, workgroups) for rows of `pieces` pieces.  Four rows a lane, so that its loads are under way together, in fp32 where a row has enough
// lanes: 2097152 x 64 saved and restored 245 us for 275 with one, 300000 x 100 61 for 69; not in 16 bits, whose pieces are twice the work (235868 x 128 44 for 40), nor where rows are
// narrow (1000000 x 16 gated 28.2 for 26.6), nor for few workgroups.
template <class T, class F>
void along_rows(int64_t n, int64_t pieces, F&& f) {
    auto go = [&](auto lanes, auto each) {
        constexpr int LANES = decltype(lanes)::value, R = decltype(each)::value, ROWS = 256 / LANES * (LANES == 64 ? 1 : R), AT_ONCE = LANES * (LANES == 64 ? R : 1);
        f(lanes, each, dim3((unsigned)std::min<int64_t>((n + ROWS - 1) / ROWS, 1 << 23), (unsigned)((pieces + AT_ONCE - 1) / AT_ONCE)));
    };
    using std::integral_constant;
    constexpr integral_constant<int, 1> one;
    auto some = [&](auto lanes) {
        if constexpr (sizeof(T) == 4)
            if (n * pieces >= 1 << 20) return go(lanes, integral_constant<int, 4>{});
        go(lanes, one);
    };
    if (pieces <= 1) go(one, one);
    else if (pieces <= 2) go(integral_constant<int, 2>{}, one);
    else if (pieces <= 4) go(integral_constant<int, 4>{}, one);
    else if (pieces <= 8) go(integral_constant<int, 8>{}, one);
    else if (pieces <= 16) some(integral_constant<int, 16>{});
    else if (pieces <= 32) some(integral_constant<int, 32>{});
    else if (pieces <= 64) go(integral_constant<int, 64>{}, one);
    else go(integral_constant<int, 64>{}, integral_constant<int, 2>{});
}

}  // namespace

// A compute unit holds one workgroup of the gradient at a time (two with narrow tiles), so s shares take ceil(s tiles / units) rounds, each 1 / s of what one workgroup takes for all
// rows, and more shares cost more partial sums: the most shares for a number of rounds, from few rounds to many, the first that another does not beat by a tenth.  A share has 64 rows at
// least.  (300000 x 300, 100 columns, six tiles: 200 us with 42 shares of which two XCDs had 36 workgroups for their 32 units, 120 with 40, 116 with 42 and 32
// workgroups an XCD; 13613 x 323, 359 columns, 18 tiles: 41 us with 40 shares in three rounds, 26 with 14 in one.)
int64_t cbm_grad_splits(int64_t n, int32_t k, int32_t c) {
    const int mt = grad_mt(k), nt = grad_nt(c);
    const int64_t units = 32 * CBM_XCD * grad_groups(mt, nt), tiles = ((int64_t)k + 32 * mt - 1) / (32 * mt) * (((int64_t)c + 32 * nt - 1) / (32 * nt));
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>(4 * units / tiles, (n + 4 * GRAD_ROWS - 1) / (4 * GRAD_ROWS)));
    int64_t rounds = (tiles + units - 1) / units, best = std::min(most, rounds * units / tiles);
    for (int64_t r = rounds + 1; r <= 4; ++r) {
        const int64_t s = std::min(most, r * units / tiles);
        if ((double)r * (double)best * 1.1 < (double)rounds * (double)s) rounds = r, best = s;
    }
    return best;
}

cbm_status cbm_launch_checkpoint_save(int64_t n, int32_t k, int32_t type, const void* X, int64_t ldx, int8_t* Q, int64_t ldq, uint8_t* E, int64_t lde, void* stream) {
    if (n == 0) return CBM_OK;
    cbm_with_type(type, [&](auto t) {
        using T = decltype(t);
        constexpr int V = 16 / (int)sizeof(T);
        along_rows<T>(n, ((int64_t)k + V - 1) / V, [&](auto lanes, auto each, dim3 grid) {
            cbm_checkpoint_save_kernel<T, decltype(lanes)::value, decltype(each)::value><<<grid, 256, 0, (hipStream_t)stream>>>(n, k, (const T*)X, ldx, Q, ldq, E, lde);
        });
    });
    return launched("checkpoint save launch");
}

cbm_status cbm_launch_checkpoint_load(int64_t n, int32_t k, const int8_t* Q, int64_t ldq, const uint8_t* E, int64_t lde, int32_t type, const void* dY, int64_t lddy, void* out,
                                      int64_t ldo, void* stream) {
    if (n == 0) return CBM_OK;
    cbm_with_type(type, [&](auto t) {
        using T = decltype(t);
        constexpr int V = 16 / (int)sizeof(T);
        along_rows<T>(n, ((int64_t)k + V - 1) / V, [&](auto lanes, auto each, dim3 grid) {
            constexpr int LANES = decltype(lanes)::value, R = decltype(each)::value;
            const bool far = n * k * (int64_t)sizeof(T) >= CBM_FAR_BYTES;
            if (dY) cbm_checkpoint_load_kernel<T, LANES, R, true><<<grid, 256, 0, (hipStream_t)stream>>>(n, k, Q, ldq, E, lde, (const T*)dY, lddy, (T*)out, ldo, far);
            else cbm_checkpoint_load_kernel<T, LANES, R, false><<<grid, 256, 0, (hipStream_t)stream>>>(n, k, Q, ldq, E, lde, nullptr, 0, (T*)out, ldo, far);
        });
    });
    return launched("checkpoint load launch");
}

cbm_status cbm_launch_checkpoint_grad(int64_t n, int32_t k, int32_t c, const int8_t* Q, int64_t ldq, const uint8_t* E, int64_t lde, int32_t type, const void* dY, int64_t lddy,
                                      float* dW, int64_t lddw, float* parts, void* stream_) {
    hipStream_t stream = (hipStream_t)stream_;
    const int64_t size = (int64_t)k * c;
    const int splits = n == 0 ? 0 : (int)cbm_grad_splits(n, k, c);
    if (splits)
        cbm_with_type(type, [&](auto t) {
            using T = decltype(t);
            const int mt = grad_mt(k), nt = grad_nt(c), tiles_c = (int)(((int64_t)c + 32 * nt - 1) / (32 * nt)), tiles = (int)(((int64_t)k + 32 * mt - 1) / (32 * mt)) * tiles_c;
            const unsigned grid = (unsigned)(((int64_t)splits * tiles + CBM_XCD - 1) / CBM_XCD * CBM_XCD);
            const GradArgs<T> a{n, k, c, Q, ldq, E, lde, (const T*)dY, lddy};
            float* to = splits == 1 ? dW : parts;
            const int64_t ldp = splits == 1 ? lddw : c;
            const bool near = std::max(std::max(ldq, lde), lddy * (int64_t)sizeof(T)) < 1 << 27;
            auto go = [&](auto m, auto o) {
                constexpr int MT = decltype(m)::value, NT = decltype(o)::value;
                if (MT == 4 && NT == 2 && k % MT == 0 && c % NT == 0) cbm_checkpoint_grad_kernel<T, 4, 2, false><<<grid, 64 * GRAD_WAVES, 0, stream>>>(a, tiles_c, tiles, splits, to, ldp, size, near);
                else cbm_checkpoint_grad_kernel<T, MT, NT, true><<<grid, 64 * GRAD_WAVES, 0, stream>>>(a, tiles_c, tiles, splits, to, ldp, size, near);
            };
            using std::integral_constant;
            auto narrow = [&](auto m) { nt == 1 ? go(m, integral_constant<int, 1>{}) : go(m, integral_constant<int, 2>{}); };
            mt == 1 ? narrow(integral_constant<int, 1>{}) : mt == 2 ? narrow(integral_constant<int, 2>{}) : narrow(integral_constant<int, 4>{});
        });
#define CBM_JOIN(SLICES) \
    cbm_checkpoint_join_kernel<SLICES><<<(unsigned)std::min<int64_t>((size + 1024 / SLICES - 1) / (1024 / SLICES), 1 << 20), 1024, 0, stream>>>(splits, size, c, parts, dW, lddw)
    if (splits == 1) {
    } else if (splits <= 16) CBM_JOIN(1);
    else if (splits <= 96) CBM_JOIN(4);
    else CBM_JOIN(32);
#undef CBM_JOIN
    return launched("checkpoint gradient launch");
}
