// Log probabilities of given labels, with entropy and the top alternatives, and their gradient.  Along a row z of C scores
//   m = max z,  l = log sum exp(z - m),  log p = z - m - l,  H = -sum p log p = l - sum (z - m) exp(z - m) / sum exp(z - m);
//   dz = a (1[label] - p) - h p (log p + H),  a and h the gradients of log p[label] and of H.
// Bound by memory: z is read once, forward and backward.  Short rows stay in the registers of a group of lanes; long ones pass through a workgroup with a
// running maximum and sums in every lane, few and long ones through several, which a second launch joins.  Statistics are fp32; exp is the hardware's 2^x.
// Scores of -infinity are ruled out; a row with nothing else has no distribution (m = l = -infinity, H = 0).  NaN or +infinity makes the sums NaN, and with them all of the row.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cbm_elems.h"
#include "cbm_internal.h"

namespace {

constexpr float LOG2E = 1.44269504088896341f;
constexpr int MOST_TOP = CBM_MOST_TOP;
constexpr int MOST_SPLITS = 64;    // workgroups that share a row: a lane each when they are joined
constexpr int LONG_THREADS = 256;
constexpr float FAR = -200.0f;     // exp of less is 0 in fp32: stands for -infinity where it is multiplied by that 0

__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * LOG2E); }
// values in an order of whole numbers: 0 for what is no alternative (-infinity), -0 as 0
__device__ __forceinline__ uint32_t ordered(float v) {
    const uint32_t b = __float_as_uint(v + 0.0f);
    return v > -INFINITY ? b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u) : 0u;
}
__device__ __forceinline__ float in_order(uint32_t o) { return __uint_as_float(o ^ ((uint32_t)((int32_t)~o >> 31) | 0x80000000u)); }
// the larger value first, of equal ones the lower column; 0: none
__device__ __forceinline__ uint64_t key_of(uint32_t o, int column) { return o ? (uint64_t)o << 32 | (uint32_t)~column : 0; }

struct Scores {
    int64_t n;
    int c;
    const void* z;
    int64_t ldz;
    const void* labels;
    int wide_labels;  // 64 bits
    float *logp, *entropy, *stats;
    int top;
    float* values;
    int32_t* columns;
};
__device__ __forceinline__ int64_t label_of(const void* labels, int wide, int64_t row) { return wide ? ((const int64_t*)labels)[row] : (int64_t)((const int32_t*)labels)[row]; }

// What one lane writes of a row, from its statistics and its score at the label (`given`: it has one).
__device__ __forceinline__ void write_row(const Scores& a, int64_t row, float m, float l, float entropy, float at_label, bool given) {
    if (a.stats) {
        a.stats[2 * row] = m;
        a.stats[2 * row + 1] = l;
    }
    if (a.entropy) a.entropy[row] = entropy;
    if (a.logp) a.logp[row] = !given ? 0.0f : m == -INFINITY ? m : at_label - m - l;
}
// statistics from the maximum and the sums of e = exp(z - m) and of (z - m) e
__device__ __forceinline__ void finish(float& m, float s, float t, float& l, float& entropy) {
    if (m == -INFINITY && s == 0.0f) {
        l = m;
        entropy = 0.0f;
    } else {
        l = logf(s);
        entropy = l - t / s;
        if (s != s) m = s;
    }
}

template <int LANES>
__device__ __forceinline__ float lanes_max(float v) {
    return lanes_all<LANES>(v, [](float a, float b) { return fmaxf(a, b); });
}
template <int LANES>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v) {
    return lanes_all<LANES>(v, [](uint32_t a, uint32_t b) { return max(a, b); });
}

// The largest whole number that at least `top` lanes of the wave have or exceed, bit by bit; the smallest that is an alternative where fewer lanes have one.  All the bits that a T has: scores of
// N(0, 3) + 1000 differ in the last ones of fp32 only (65536 x 1000, top 8, 69 us, with 16 bits 245; without the offset 65.5 either way).
template <class T>
__device__ __forceinline__ uint32_t bound_of_heads(uint32_t head, int top) {
    uint32_t bound = 0;
    for (int bit = 31; bit >= 32 - 8 * (int)sizeof(T); --bit) {
        const int have = __popcll(__ballot(head >= (bound | 1u << bit)));
        if (have >= top) bound |= 1u << bit;
        if (have == top) break;  // (they all exceed what the bits below could add, or the bound is a little low, which costs nothing)
    }
    return max(bound, 0x00800000u);  // (of the lowest finite value; what is below it is no value's)
}
__device__ __forceinline__ uint64_t lane_value(uint64_t v, int lane) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}

// More than one alternative of a row in registers.  own: the largest of the lane's scores.
template <class T, int V, int LANES, int R>
__device__ __forceinline__ void write_alternatives(const Scores& a, int64_t row, int lane, const float (&x)[R][V], float own, float m, float l) {
    const bool none = m != m;  // of the row's scores is an alternative
    float* values = a.values + (row < a.n ? row : a.n - 1) * a.top;
    int32_t* columns = a.columns + (row < a.n ? row : a.n - 1) * a.top;
    constexpr int MOST = LANES * V < MOST_TOP ? LANES * V : MOST_TOP;  // alternatives of a row of one piece a lane
    constexpr int FOUND = 64 * R * V < 256 ? 64 * R * V : 256;           // room of a wave for candidates
    __shared__ uint64_t room[LANES < 64 ? 256 / LANES * MOST : 4 * FOUND];  // what a row (a wave) has found
    if constexpr (LANES < 64 && sizeof(T) == 2) {
        uint64_t* kept = room + threadIdx.x / LANES * MOST;
        // A value's 16 bits in order, then its column from behind, make one whole number; every lane's in descending order, then `top` times the largest head.
        uint32_t key[V];
        const int at0 = Place<V, false>(lane, a.c).at;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const uint32_t u = __builtin_bit_cast(uint16_t, (T)(x[0][j] + 0.0f));
            key[j] = !none && x[0][j] > -INFINITY ? (u ^ (u & 0x8000u ? 0xffffu : 0x8000u)) << 16 | (0xffffu - (uint32_t)(at0 + j)) : 0u;
        }
#pragma unroll
        for (int round = 0; round < V; ++round)
#pragma unroll
            for (int j = round % 2; j + 1 < V; j += 2) {
                const uint32_t first = max(key[j], key[j + 1]), second = min(key[j], key[j + 1]);
                key[j] = first, key[j + 1] = second;
            }
        for (int r = 0; r < min(a.top, MOST); ++r) {
            const uint32_t best = lanes_max<LANES>(key[0]);
            const bool mine = key[0] == best;
            if (mine) kept[r] = best;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const uint32_t stays = key[j], comes = j + 1 < V ? +key[j + 1] : 0u;  // (values: a choice of places would become an index)
                key[j] = mine ? comes : stays;
            }
        }
        __builtin_amdgcn_wave_barrier();
        for (int r = lane; r < a.top; r += LANES) {
            const uint32_t best = r < MOST ? (uint32_t)kept[r] : 0u, o = best >> 16, u = o ^ (o & 0x8000u ? 0x8000u : 0xffffu);
            if (row >= a.n) break;
            values[r] = none ? NAN : best ? (float)__builtin_bit_cast(T, (uint16_t)u) - m - l : -INFINITY;
            columns[r] = best ? (int32_t)(0xffffu - (best & 0xffffu)) : -1;
        }
        __builtin_amdgcn_wave_barrier();  // (kept is the next row's)
    } else if constexpr (LANES < 64) {
        // Every lane's values in descending order (neighbours change places only where the later one is larger, so the lower column stays first), then `top` times the
        // largest head: of equal ones the first lane's, whose columns are lower.
        uint64_t* kept = room + threadIdx.x / LANES * MOST;
        uint32_t o[V], which[V];
        const int at0 = Place<V, false>(lane, a.c).at;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            o[j] = none ? 0u : ordered(x[0][j]);
            which[j] = j;
        }
#pragma unroll
        for (int round = 0; round < V; ++round)
#pragma unroll
            for (int j = round % 2; j + 1 < V; j += 2) {
                const bool change = o[j] < o[j + 1];
                const uint32_t first = max(o[j], o[j + 1]), second = min(o[j], o[j + 1]);
                const uint32_t here = which[j], next = which[j + 1];  // (values: a choice of places would become an index)
                o[j] = first, o[j + 1] = second;
                which[j] = change ? next : here, which[j + 1] = change ? here : next;
            }
        const uint64_t group = ((1ull << LANES) - 1) << (threadIdx.x & 63 & ~(LANES - 1));
        for (int r = 0; r < min(a.top, MOST); ++r) {
            const uint32_t best = lanes_max<LANES>(o[0]);
            const uint64_t have = __ballot(o[0] == best) & group;
            const bool mine = o[0] == best && __builtin_amdgcn_mbcnt_hi((uint32_t)(have >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)have, 0)) == 0;
            if (mine) kept[r] = (uint64_t)best << 32 | (uint32_t)(at0 + (int)which[0]);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const uint32_t stays = o[j], comes = j + 1 < V ? +o[j + 1] : 0u, w1 = which[j], w2 = which[j + 1 < V ? j + 1 : j];
                o[j] = mine ? comes : stays;
                which[j] = mine ? w2 : w1;
            }
        }
        __builtin_amdgcn_wave_barrier();
        for (int r = lane; r < a.top; r += LANES) {
            const uint32_t best = r < MOST ? (uint32_t)(kept[r] >> 32) : 0u;
            if (row >= a.n) break;
            values[r] = none ? NAN : best ? in_order(best) - m - l : -INFINITY;
            columns[r] = best ? (int32_t)kept[r] : -1;
        }
        __builtin_amdgcn_wave_barrier();  // (kept is the next row's)
    } else {
        // As for a long row: the top-th largest of the lanes' largest bounds the answer from below; what is as large is collected and ranked by counting.  Where that is more than there
        // is room for (many equal scores), the largest score below the last one, `top` times.
        uint64_t* found = room + threadIdx.x / 64 * FOUND;
        float* values = a.values + (row < a.n ? row : a.n - 1) * a.top;
        int32_t* columns = a.columns + (row < a.n ? row : a.n - 1) * a.top;
        const uint32_t bound = none ? ~0u : bound_of_heads<T>(ordered(own), a.top);
        const float least = in_order(bound);
        int count = 0;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int at = Place<V, false>(i * LANES + lane, a.c).at;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const uint64_t takes = none ? 0 : __ballot(x[i][j] >= least);
                if (!takes) continue;
                const int to = count + __builtin_amdgcn_mbcnt_hi((uint32_t)(takes >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)takes, 0));
                if (x[i][j] >= least && to < FOUND) found[to] = (uint64_t)__float_as_uint(x[i][j]) << 32 | (uint32_t)(at + j);
                count += __popcll(takes);
            }
            if constexpr (R * V > 16) __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_wave_barrier();
        if (count <= FOUND) {
            auto key_at = [&](int i) {
                const uint64_t both = found[min(i, FOUND - 1)];
                return i < count ? key_of(ordered(__uint_as_float((uint32_t)(both >> 32))), (int)(uint32_t)both) : 0;
            };
            for (int i0 = 0; i0 < count; i0 += 64) {
                const uint64_t mine = key_at(i0 + lane);
                int rank = 0;
                for (int j0 = 0; j0 < count; j0 += 64) {
                    const uint64_t other = j0 == i0 ? mine : key_at(j0 + lane);
                    const int some = min(64, count - j0);
                    for (int j = 0; j < some; ++j) rank += lane_value(other, j) > mine;
                }
                if (mine && rank < a.top && row < a.n) {
                    values[rank] = in_order((uint32_t)(mine >> 32)) - m - l;
                    columns[rank] = (int32_t)~(uint32_t)mine;
                }
            }
        } else {
            uint64_t last = ~0ull;
            for (int r = 0; r < a.top; ++r) {  // (there are more than `top` of them)
                uint64_t best = 0;
#pragma unroll
                for (int i = 0; i < R; ++i) {
                    int piece = i * LANES + lane;
                    asm volatile("" : "+v"(piece));  // (as above, for places and values)
                    const int at = Place<V, false>(piece, a.c).at;
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        float z = x[i][j];
                        asm volatile("" : "+v"(z));
                        const uint64_t key = key_of(ordered(z), at + j);
                        best = key < last && key > best ? key : best;
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                const uint32_t high = lanes_max<64>((uint32_t)(best >> 32)), low = lanes_max<64>((uint32_t)(best >> 32) == high ? (uint32_t)best : 0u);
                last = (uint64_t)high << 32 | low;
                if (lane == r && row < a.n) {
                    values[r] = in_order(high) - m - l;
                    columns[r] = (int32_t)~low;
                }
            }
        }
        if (lane >= count && lane < a.top && row < a.n) {
            values[lane] = none ? NAN : -INFINITY;
            columns[lane] = -1;
        }
        __builtin_amdgcn_wave_barrier();  // (found is the next row's)
    }
}

// Short rows.  LANES lanes a row, each R pieces of V columns.  SELECT: more alternatives than the best one.  Without it four pieces of fp32 (two of 16 bits) a lane, so that many rows share a
// wave's reductions (235868 x 112 33 us with one piece a lane, 20 with four); with it one piece as long as that is enough, since alternatives come out of sorted lanes.
// Bound by memory in fp32: 235868 x 112 23 us for 108 MB (4.7 TB/s), 8192 x 4000 23 us for 131 MB; by vector instructions in 16 bits (21 a value, and a row's
// reductions: 30310 x 567 bf16 15 us for 35 MB, reading alone 6.4) and with alternatives (65536 x 1000 fp32, top 8, 71 us for 262 MB, reading alone 41; 110318 x 133 fp16, top 20, 58 us, 20 times the largest
// head, reading alone 6).  19717 x 3 2.8 us, a launch.
template <class T, int V, int LANES, int R, bool SELECT>
__global__ __launch_bounds__(256) void cbm_scores_kernel(Scores a) {
    const int lane = threadIdx.x % LANES;
    for (int64_t row0 = (int64_t)blockIdx.x * (256 / LANES); row0 < a.n; row0 += (int64_t)gridDim.x * (256 / LANES)) {
        const int64_t row = row0 + threadIdx.x / LANES, at = row < a.n ? row : a.n - 1;
        const T* z_row = (const T*)a.z + at * a.ldz;
        float x[R][V], m = -INFINITY;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const Place<V, false> p(i * LANES + lane, a.c);
            load_piece<V>(x[i], z_row + p.at);
        }
        bool given = false;
        float at_label = 0.0f;
        if (a.logp && lane == 0) {
            const int64_t label = label_of(a.labels, a.wide_labels, at);
            given = label >= 0 && label < a.c;
            if (given) at_label = (float)z_row[label];
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            int piece = i * LANES + lane;
            if constexpr (R * V > 16 || (SELECT && R > 1)) asm volatile("" : "+v"(piece));  // (every row's comparisons anew, a piece's at a time: kept they are more than the scalar registers hold)
            const Place<V, false> p(piece, a.c);
            if (R == 1 || __any(p.seen > 0)) {  // (the last piece of a row, and what lies behind it)
#pragma unroll
                for (int j = 0; j < V; ++j) x[i][j] = p.counts(j) ? x[i][j] : -INFINITY;
            }
#pragma unroll
            for (int j = 0; j < V; ++j) m = fmaxf(m, x[i][j]);
            if constexpr (R * V > 16 || (SELECT && R > 1)) __builtin_amdgcn_sched_barrier(0);
        }
        const float own = m;  // of the lane's columns
        m = lanes_max<LANES>(m);
        const float base = m == -INFINITY ? 0.0f : m;
        float s = 0.0f, t = 0.0f, l, entropy;
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = x[i][j] - base, e = exp_of(d);
                s += e;
                t += e * fmaxf(d, FAR);
            }
        s = lanes_sum<LANES>(s);
        t = lanes_sum<LANES>(t);
        finish(m, s, t, l, entropy);
        if (lane == 0 && row < a.n) write_row(a, row, m, l, entropy, at_label, given);
        if (!SELECT && !a.top) continue;
        if constexpr (!SELECT) {  // one: the largest is known, it is the lowest column that has it
            uint32_t column = 0;  // (its complement)
#pragma unroll
            for (int i = R - 1; i >= 0; --i) {
                const Place<V, false> p(i * LANES + lane, a.c);
                if constexpr (R * V > 16) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int j = V - 1; j >= 0; --j) column = x[i][j] == m ? ~(uint32_t)(p.at + j) : column;
            }
            column = lanes_max<LANES>(column);
            if (lane == 0 && row < a.n) {
                const bool is = m > -INFINITY;
                a.values[row] = is ? -l : m;  // (m - m - l)
                a.columns[row] = is ? (int32_t)~column : -1;
            }
        } else {
            write_alternatives<T, V, LANES, R>(a, row, lane, x, own, m, l);
        }
    }
}

// What a workgroup finds its alternatives with.
template <int CAP>
struct Select {
    uint64_t head[64], list[MOST_TOP], found[CAP];
    uint64_t bound;
    int count, lanes;
    uint16_t lane[LONG_THREADS];
};
// The `top` largest of found[0 .. count) to the list, by counting what is larger (keys differ, so do ranks).
template <int THREADS, int CAP>
__device__ __forceinline__ void rank_found(Select<CAP>& s, int top, int count) {
    for (int i = threadIdx.x; i < count; i += THREADS) {
        const uint64_t mine = s.found[i];
        int rank = 0;
#pragma unroll 8
        for (int j = 0; j < count; ++j) rank += s.found[j] > mine;
        if (rank < top) s.list[rank] = mine;
    }
    __syncthreads();
}
// The `top` largest of the list's keys and of those that each(take) takes.  `head`: the largest of each of 64 parts of these, so that the top-th largest head bounds the answer
// from below; the parts are so small that there is room for what is as large.
template <int THREADS, int CAP, class F>
__device__ __forceinline__ void select_keys(Select<CAP>& s, int top, F&& each) {
    __syncthreads();
    if (threadIdx.x < 64) {
        const uint64_t mine = s.head[threadIdx.x];
        const int there = __popcll(__ballot(mine != 0));
        int rank = 0;
#pragma unroll 2
        for (int i = 0; i < 64; ++i) rank += lane_value(mine, i) > mine;
        if (there < top ? threadIdx.x == 0 : mine && rank == top - 1) s.bound = there < top ? 1 : mine;
        if (threadIdx.x == 0) s.count = 0;
    }
    __syncthreads();
    const uint64_t bound = s.bound;
    auto take = [&](uint64_t key) {
        if (key >= bound) s.found[atomicAdd(&s.count, 1)] = key;
    };
    each(take);
    if ((int)threadIdx.x < top) take(s.list[threadIdx.x]);
    __syncthreads();
    const int count = s.count;
    if ((int)threadIdx.x < top) s.list[threadIdx.x] = 0;
    __syncthreads();
    rank_found<THREADS>(s, top, count);
}

__device__ __forceinline__ void write_top(const Scores& a, int64_t row, const uint64_t* list, float m, float l) {
    if ((int)threadIdx.x >= a.top) return;
    const uint64_t key = m == m ? list[threadIdx.x] : 0;
    a.values[row * a.top + threadIdx.x] = m != m ? m : key ? in_order((uint32_t)(key >> 32)) - m - l : -INFINITY;
    a.columns[row * a.top + threadIdx.x] = key ? (int32_t)~(uint32_t)key : -1;
}

struct Part {  // of a row that several workgroups share; `top` keys follow
    float m, s, t, unused;
};
__device__ __forceinline__ char* part_at(char* parts, int64_t i, int top) { return parts + i * (int64_t)(sizeof(Part) + top * sizeof(uint64_t)); }

// Sums over the lanes of a wave, each with a maximum of its own.
__device__ __forceinline__ void join_wave(float& m, float& s, float& t) {
    const float all = lanes_max<64>(m), base = all == -INFINITY ? 0.0f : all;
    const float d = m - base, f = exp_of(d);
    t = lanes_sum<64>(f * (t + fmaxf(d, FAR) * s));
    s = lanes_sum<64>(f * s);
    m = all;
}

// Long rows.  A workgroup (of four waves or one) a row, or a share of `columns` of its columns (a multiple of V); R pieces of V columns a lane and turn.  The alternatives come last: of what each four lanes (one of a single wave)
// have met, the maximum is known by then; the top-th largest of these 64 bounds the answer from below, the columns of the few lanes that hold as much are looked through
// once more (out of L2, most likely), and what is found is ranked.  Where that is more than there is room for (equal scores, or orders that leave the largest
// to a few lanes), all columns are gone through again in turns of one piece a lane, each of which adds to the list what exceeds it.
// Bound by memory while rows are many: 4096 x 32000 bf16 with top 8 55 us for 262 MB (4.8 TB/s, waves waiting for 52 % of their cycles: a turn's loads are not under way while the turn before
// it is added up; reading alone 41; 145 with a list kept sorted on the way).
// One row of 128,000 fp32 in 63 shares: 5.3 us, and 5.4 more for the join, each a launch and three dependent loads.
template <class T, int V, int R, bool TOP, int THREADS>
__global__ __launch_bounds__(THREADS) void cbm_scores_long_kernel(Scores a, int splits, int columns, char* __restrict__ parts) {
    constexpr int TURN = THREADS * R * V, WAVES = THREADS / 64, CAP = TOP ? MOST_TOP * WAVES * V + MOST_TOP : 1;
    static_assert(WAVES == 1 || WAVES == 4, "");
    __shared__ Select<CAP> sel;
    __shared__ float room[3][WAVES];
    const int wave = threadIdx.x / 64;
    for (int64_t item = blockIdx.x; item < a.n * splits; item += gridDim.x) {
        const int64_t row = item / splits;
        const int split = (int)(item % splits);
        const T* z_row = (const T*)a.z + row * a.ldz;
        const int begin = split * columns, end = min(begin + columns, a.c);
        float m = -INFINITY, s = 0.0f, t = 0.0f;
        auto rise = [&](float most) {  // the maximum so far, and the sums as seen from it
            const float now = fmaxf(m, most), base = now == -INFINITY ? 0.0f : now, d = m - base, f = exp_of(d);
            t = f * (t + fmaxf(d, FAR) * s);
            s *= f;
            m = now;
            return base;
        };
        auto add = [&](float z, float base) {
            const float d = z - base, e = exp_of(d);
            s += e;
            t += e * fmaxf(d, FAR);
        };
        for (int turn = begin; turn < end; turn += TURN) {
            float x[R][V], most = -INFINITY;
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const Place<V, false> p(turn / V + i * THREADS + threadIdx.x, a.c);
                load_piece<V>(x[i], z_row + p.at);
            }
            if (turn + TURN <= end) {
#pragma unroll
                for (int i = 0; i < R; ++i)
#pragma unroll
                    for (int j = 0; j < V; ++j) most = fmaxf(most, x[i][j]);
                const float base = rise(most);
#pragma unroll
                for (int i = 0; i < R; ++i)
#pragma unroll
                    for (int j = 0; j < V; ++j) add(x[i][j], base);
            } else {  // the last turn: a piece at a time, as far as there are any
#pragma unroll
                for (int i = 0; i < R; ++i) {
                    if (turn + i * THREADS * V >= end) break;
                    const int piece = turn / V + i * THREADS + threadIdx.x, seen = piece * V < end ? Place<V, false>(piece, a.c).seen : V;
                    most = -INFINITY;
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        x[i][j] = j >= seen ? x[i][j] : -INFINITY;
                        most = fmaxf(most, x[i][j]);
                    }
                    const float base = rise(most);
#pragma unroll
                    for (int j = 0; j < V; ++j) add(x[i][j], base);
                }
            }
        }
        const float best = m;  // of this lane's columns
        join_wave(m, s, t);
        __syncthreads();
        if (WAVES > 1 && (threadIdx.x & 63) == 0) {
            room[0][wave] = m;
            room[1][wave] = s;
            room[2][wave] = t;
        }
        if constexpr (TOP) {  // a key for each four lanes (each lane of a wave alone), of which only the value matters
            float some = best;
            if constexpr (WAVES == 4) {
                some = fmaxf(some, lane_other<1>(some));
                some = fmaxf(some, lane_other<2>(some));
            }
            if (threadIdx.x % WAVES == 0) sel.head[threadIdx.x / WAVES] = key_of(ordered(some), 0);
            if ((int)threadIdx.x < MOST_TOP) sel.list[threadIdx.x] = 0;
            if (threadIdx.x == 0) sel.count = sel.lanes = 0;
        }
        __syncthreads();
        if constexpr (WAVES > 1) {
            const int w = min((int)threadIdx.x & 63, WAVES - 1);
            const bool first = (threadIdx.x & 63) < WAVES;
            m = first ? room[0][w] : -INFINITY;
            s = first ? room[1][w] : 0.0f;
            t = first ? room[2][w] : 0.0f;
            join_wave(m, s, t);
        }
        if constexpr (TOP) {
            // f(value, column) for the lane's columns that count, of the piece `piece`
            auto scan = [&](int piece, auto&& f) {
                if (piece * V >= end) return;
                const Place<V, false> p(piece, a.c);
                float x[V];
                load_piece<V>(x, z_row + p.at);
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (p.counts(j)) f(x[j], p.at + j);
            };
            // what is as large as the bound: the row's maximum where one alternative is asked for
            const uint32_t bound = a.top == 1 ? max(ordered(m), 1u) : bound_of_heads<T>((uint32_t)(sel.head[threadIdx.x & 63] >> 32), a.top);
            auto take = [&](float v, int column) {
                if (ordered(v) < bound) return;
                const int at = atomicAdd(&sel.count, 1);
                if (at < CAP) sel.found[at] = key_of(ordered(v), column);
            };
            if (ordered(best) >= bound) sel.lane[atomicAdd(&sel.lanes, 1)] = (uint16_t)threadIdx.x;
            __syncthreads();
            const int lanes = sel.lanes, turns = (end - begin + THREADS * V - 1) / (THREADS * V);
            for (int i = threadIdx.x; i < lanes * turns; i += THREADS)  // (the lanes' pieces are shared out, so that they are loaded at once)
                scan(begin / V + i / lanes * THREADS + sel.lane[i % lanes], take);
            __syncthreads();
            const int count = sel.count;
            const bool done = count <= CAP;
            if (done) rank_found<THREADS>(sel, a.top, count);
            if (!done) {
                float least = -INFINITY;  // the last of the alternatives so far; a later column has to exceed it
                for (int turn = begin / V; turn * V < end; turn += THREADS) {
                    uint64_t mine = 0;
                    scan(turn + threadIdx.x, [&](float v, int column) {
                        const uint64_t key = v > least ? key_of(ordered(v), column) : 0;
                        mine = key > mine ? key : mine;
                    });
                    if (!__syncthreads_or(mine != 0)) continue;
                    uint64_t some = mine;
#pragma unroll
                    for (int step = 1; step < WAVES; step *= 2) {
                        const uint64_t other = (uint64_t)__shfl_xor((unsigned long long)some, step);
                        some = other > some ? other : some;
                    }
                    if (threadIdx.x % WAVES == 0) sel.head[threadIdx.x / WAVES] = some;
                    select_keys<THREADS>(sel, a.top, [&](auto&& take) {
                        if (mine >= sel.bound) scan(turn + threadIdx.x, [&](float v, int column) { take(v > least ? key_of(ordered(v), column) : 0); });  // (0 < 1 <= bound)
                    });
                    const uint64_t last = sel.list[a.top - 1];
                    least = last ? in_order((uint32_t)(last >> 32)) : -INFINITY;
                }
            }
        }
        if (splits > 1) {
            char* part = part_at(parts, item, a.top);
            if (threadIdx.x == 0) *(Part*)part = Part{m, s, t, 0.0f};
            if constexpr (TOP)
                if ((int)threadIdx.x < a.top) ((uint64_t*)(part + sizeof(Part)))[threadIdx.x] = sel.list[threadIdx.x];
        } else {
            float l, entropy;
            finish(m, s, t, l, entropy);
            if (threadIdx.x == 0) {
                const int64_t label = a.logp ? label_of(a.labels, a.wide_labels, row) : -1;
                const bool given = label >= 0 && label < a.c;
                write_row(a, row, m, l, entropy, given ? (float)z_row[label] : 0.0f, given);
            }
            if constexpr (TOP) write_top(a, row, sel.list, m, l);
        }
    }
}

// Rows that several workgroups have shared: a workgroup each.
template <class T>
__global__ __launch_bounds__(LONG_THREADS) void cbm_scores_join_kernel(Scores a, int splits, char* __restrict__ parts) {
    __shared__ Select<MOST_TOP * MOST_TOP> sel;  // (of at most `top` parts, `top` keys each)
    constexpr int WAVES = LONG_THREADS / 64, EACH = MOST_TOP / WAVES;
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        Part mine{-INFINITY, 0.0f, 0.0f, 0.0f};
        uint64_t keys[EACH] = {};  // every fourth of a share's, from its first (wave 0), second ... on
        if (lane < splits) {
            const char* part = part_at(parts, row * splits + lane, a.top);
            mine = *(const Part*)part;
#pragma unroll
            for (int i = 0; i < EACH; ++i)
                if (i * WAVES + wave < a.top) keys[i] = ((const uint64_t*)(part + sizeof(Part)))[i * WAVES + wave];
        }
        float m = mine.m, s = mine.s, t = mine.t, l, entropy;
        join_wave(m, s, t);
        finish(m, s, t, l, entropy);
        if (threadIdx.x == 0) {
            const int64_t label = a.logp ? label_of(a.labels, a.wide_labels, row) : -1;
            const bool given = label >= 0 && label < a.c;
            write_row(a, row, m, l, entropy, given ? (float)((const T*)a.z)[row * a.ldz + label] : 0.0f, given);
        }
        if (!a.top) continue;
        __syncthreads();
        if ((int)threadIdx.x < 64) sel.head[lane] = keys[0];
        if ((int)threadIdx.x < MOST_TOP) sel.list[threadIdx.x] = 0;
        select_keys<LONG_THREADS>(sel, a.top, [&](auto&& take) {
#pragma unroll
            for (int i = 0; i < EACH; ++i)
                if (keys[i]) take(keys[i]);
        });
        write_top(a, row, sel.list, m, l);
    }
}

struct Slopes {
    int64_t n;
    int c;
    const void* z;
    int64_t ldz;
    const void* labels;
    int wide_labels;
    const float *stats, *entropy, *dlogp, *dentropy;
    void* dz;
    int64_t lddz;
};
// Backward.  LANES lanes a row and a share of its columns (blockIdx.y), V columns a lane and turn; no lane needs another's, since the forward pass kept m and l.  Bound by memory:
// 132534 x 47 fp32 11 us for 51.4 MB (4.7 TB/s, waves waiting for 66 % of their cycles; a copy alone, some of it out of the memory-side cache, 7.5), bf16 8.1 (10.4 with a row's last piece written value by value).
template <class T, int V, int LANES>
__global__ __launch_bounds__(256) void cbm_scores_back_kernel(Slopes a, int turns, bool far) {
    const int lane = threadIdx.x % LANES, pieces = (a.c + V - 1) / V;
    const int most = a.dz == a.z ? 0 : V - 1;  // of a piece's values that are another lane's as well: they get the same bits twice, but where dz is z that lane may not have read them yet
    for (int64_t row = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES; row < a.n; row += (int64_t)gridDim.x * (256 / LANES)) {
        const float m = a.stats[2 * row], l = a.stats[2 * row + 1];
        const int64_t label = a.dlogp ? label_of(a.labels, a.wide_labels, row) : -1;
        const bool given = label >= 0 && label < a.c, empty = m == -INFINITY;
        const float slope = given ? a.dlogp[row] : 0.0f, of_entropy = a.dentropy ? a.dentropy[row] : 0.0f, entropy = a.dentropy ? a.entropy[row] : 0.0f;
        const T* z_row = (const T*)a.z + row * a.ldz;
        T* out = (T*)a.dz + row * a.lddz;
        for (int turn = 0; turn < turns; ++turn) {
            const int piece = (blockIdx.y * turns + turn) * LANES + lane;
            if (piece >= pieces) break;
            const Place<V, false> p(piece, a.c);
            float x[V];
            load_piece<V>(x, z_row + p.at);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float log_p = x[j] - m - l, pr = exp_of(log_p);
                const float own = p.at + j == label ? slope : 0.0f;
                const float v = own - pr * (slope + of_entropy * (fmaxf(log_p, FAR) + entropy));
                x[j] = empty ? 0.0f : v;
            }
            if (p.seen <= most) {
                store_piece<V>(out + p.at, x, far);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (p.counts(j)) out[p.at + j] = (T)x[j];
            }
        }
    }
}

cbm_status launched(const char* what) {
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return CBM_OK;
    cbm_set_error_detail(what, hipGetErrorString(e));
    return CBM_ERR_HIP;
}
// Columns that a wave keeps in its registers in 16 values a lane; a wave has rows of twice as many, four times where no alternatives but the best are asked for (17261 x 2015 fp32 with the best
// 24.5 us, by a workgroup a row 51, top 8 40 and 54, bf16 30 and 56; 8192 x 4000 with the best 23 and 34, bf16 18 and 35, but top 8 70 and 37; with 8,192 columns a wave 8192 x 5000 bf16
// took 52, a workgroup a row 35).
constexpr int SHORT_ROW = 1024;
// Columns up to which a workgroup has a row alone whatever the number of rows, since a second launch takes longer than its turns.  Microseconds alone and shared, top 8, captured
// (calls one after the other): one row of 16,384 columns 5.9 and 9.7 (7.5 and 10.8), 49,152 9.1 and 9.7 (8.8 and 10.9), 65,536 10.4 and 9.7 (10.1 and 10.9); 100 rows of 49,152 11.5 and 13.9.
constexpr int ALONE = 49152;
// Rows that a wave passes through alone, and bytes of each: four waves share a row's values, but each does its reductions.  Microseconds, a wave and four: 52207 x 2273 fp16, top 8, 76 and 195,
// 17261 x 5000 bf16 36 and 49, top 8 46 and 70, 1024 x 2195 fp32 6.1 and 6.7, 1024 x 5000 bf16 8.0 and 8.0; longer rows leave too few loads under way: 17261 x 5000 fp32, top 20, 99 and 80,
// 8192 x 16000 bf16, top 8, 77 and 61.
constexpr int MANY_ROWS = 1024, WAVE_ROW = 16384;

}  // namespace

// Workgroups that share a row of over ALONE columns: two for every compute unit over all rows, 64 a row at most, of about 2,048 columns or more.  Few shorter rows are asked for a workspace as if
// they were shared, although each has one workgroup and nothing reads it.
int cbm_scores_splits(int64_t n, int32_t c) {
    if (c <= SHORT_ROW || n == 0) return 1;
    return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(MOST_SPLITS, 512 / n), ((int64_t)c + 2047) / 2048));
}
size_t cbm_scores_part_bytes(int32_t top) { return sizeof(Part) + (size_t)top * sizeof(uint64_t); }

cbm_status cbm_launch_scores(int64_t n, int32_t c, int32_t type, const void* z, int64_t ldz, const void* labels, int label_bits, float* logp, float* entropy, float* stats, int32_t top,
                             float* values, int32_t* columns, void* parts, void* stream_) {
    if (n == 0) return CBM_OK;
    hipStream_t stream = (hipStream_t)stream_;
    const Scores a{n, c, z, ldz, labels, label_bits == 64, logp, entropy, stats, top, values, columns};
    cbm_with_type(type, [&](auto t) {
        using T = decltype(t);
        constexpr int V = 16 / (int)sizeof(T);
        const int pieces = (c + V - 1) / V;
#define CBM_SCORES(V_, LANES, R, SELECT) \
    cbm_scores_kernel<T, V_, LANES, R, SELECT><<<(unsigned)std::min<int64_t>((n + 256 / LANES - 1) / (256 / LANES), 1 << 23), 256, 0, stream>>>(a)
        constexpr int R = 16 / V;
        if (c < V) cbm_narrow_row<V>(c, [&](auto v, auto lanes) { top > 1 ? CBM_SCORES(v(), lanes(), 1, true) : CBM_SCORES(v(), lanes(), 1, false); });
        else if (top > 1 && pieces <= 64) {
            if (pieces <= 1) CBM_SCORES(V, 1, 1, true);
            else if (pieces <= 2) CBM_SCORES(V, 2, 1, true);
            else if (pieces <= 4) CBM_SCORES(V, 4, 1, true);
            else if (pieces <= 8) CBM_SCORES(V, 8, 1, true);
            else if (pieces <= 16) CBM_SCORES(V, 16, 1, true);
            else if (pieces <= 32) CBM_SCORES(V, 32, 1, true);
            else CBM_SCORES(V, 64, 1, true);
        } else if (top > 1 && c <= SHORT_ROW) CBM_SCORES(V, 64, R, true);
        else if (top > 1 && c <= 2 * SHORT_ROW) CBM_SCORES(V, 64, 2 * R, true);
        else if (pieces <= 1) CBM_SCORES(V, 1, 1, false);
        else if (pieces <= 2) CBM_SCORES(V, 2, 1, false);
        else if (pieces <= 4) CBM_SCORES(V, 4, 1, false);
        else if (pieces <= 4 * R) CBM_SCORES(V, 4, R, false);
        else if (pieces <= 8 * R) CBM_SCORES(V, 8, R, false);
        else if (pieces <= 16 * R) CBM_SCORES(V, 16, R, false);
        else if (pieces <= 32 * R) CBM_SCORES(V, 32, R, false);
        else if (c <= SHORT_ROW) CBM_SCORES(V, 64, R, false);
        else if (c <= 2 * SHORT_ROW) CBM_SCORES(V, 64, 2 * R, false);
        else if (top <= 1 && c <= 4 * SHORT_ROW) CBM_SCORES(V, 64, 4 * R, false);
#undef CBM_SCORES
        else {
            const int splits = c <= ALONE ? 1 : cbm_scores_splits(n, c);
            int share = ((c + splits - 1) / splits + V - 1) / V * V;
            const unsigned grid = (unsigned)std::min<int64_t>(n * splits, 1 << 20);
#define CBM_LONG(R, TOP, THREADS) cbm_scores_long_kernel<T, V, R, TOP, THREADS><<<grid, THREADS, 0, stream>>>(a, splits, share, (char*)parts)
            if (n >= MANY_ROWS && c * (int)sizeof(T) <= WAVE_ROW)  // (splits is 1)
                top ? CBM_LONG(32 / V, true, 64) : CBM_LONG(32 / V, false, 64);
            else if (share <= 2048) top ? CBM_LONG(8 / V, true, LONG_THREADS) : CBM_LONG(8 / V, false, LONG_THREADS);
            else top ? CBM_LONG(32 / V, true, LONG_THREADS) : CBM_LONG(32 / V, false, LONG_THREADS);
#undef CBM_LONG
            if (splits > 1) cbm_scores_join_kernel<T><<<(unsigned)std::min<int64_t>(n, 1 << 20), LONG_THREADS, 0, stream>>>(a, splits, (char*)parts);
        }
    });
    return launched("log probabilities launch");
}

cbm_status cbm_launch_scores_backward(int64_t n, int32_t c, int32_t type, const void* z, int64_t ldz, const void* labels, int label_bits, const float* stats, const float* entropy,
                                      const float* dlogp, const float* dentropy, void* dz, int64_t lddz, void* stream_) {
    if (n == 0) return CBM_OK;
    hipStream_t stream = (hipStream_t)stream_;
    const Slopes a{n, c, z, ldz, labels, label_bits == 64, stats, entropy, dlogp, dentropy, dz, lddz};
    cbm_with_type(type, [&](auto t) {
        using T = decltype(t);
        constexpr int V = 16 / (int)sizeof(T);
        const int64_t pieces = (c + V - 1) / V;
        const bool far = n * c * (int64_t)sizeof(T) >= CBM_FAR_BYTES;
#define CBM_BACK(V_, LANES)                                                                                                                                                  \
    {                                                                                                                                                                        \
        const int turns = pieces <= LANES ? 1 : 4;                                                                                                                           \
        cbm_scores_back_kernel<T, V_, LANES><<<dim3((unsigned)std::min<int64_t>((n + 256 / LANES - 1) / (256 / LANES), 1 << 23),                                             \
                                                    (unsigned)((pieces + LANES * turns - 1) / (LANES * turns))), 256, 0, stream>>>(a, turns, far);                              \
    }
        if (c < V) cbm_narrow_row<V>(c, [&](auto v, auto lanes) {
                const int64_t pieces = lanes();
                CBM_BACK(v(), lanes())
            });
        else if (pieces <= 1) CBM_BACK(V, 1)
        else if (pieces <= 2) CBM_BACK(V, 2)
        else if (pieces <= 4) CBM_BACK(V, 4)
        else if (pieces <= 8) CBM_BACK(V, 8)
        else if (pieces <= 16) CBM_BACK(V, 16)
        else if (pieces <= 32) CBM_BACK(V, 32)
        else CBM_BACK(V, 64)
#undef CBM_BACK
    });
    return launched("log probabilities backward launch");
}
