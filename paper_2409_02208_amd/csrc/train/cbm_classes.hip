// Log probabilities of labels straight from a layer's outputs and the classes' weights, Z = X W, without keeping Z, and the gradients of both.
#include <algorithm>

#include "cbm_aligned.h"
#include "cbm_few_rows.h"
#include "cbm_internal.h"
#include "cbm_products.h"
#include "cbm_small.h"

namespace {

constexpr float LOG2E = 1.44269504f;

// m and sum exp(z - m) of two sets of scores as one
struct Sums {
    float m, s;
};
__device__ __forceinline__ Sums joined(Sums a, Sums b) {
    const float m = fmaxf(a.m, b.m), away = m == -INFINITY ? 0.0f : m;  // (NaN is in s)
    return {m, a.s * __builtin_amdgcn_exp2f((a.m - away) * LOG2E) + b.s * __builtin_amdgcn_exp2f((b.m - away) * LOG2E)};
}

__device__ __forceinline__ int64_t label_of(const void* labels, int bits, int64_t r) { return bits == 64 ? ((const int64_t*)labels)[r] : ((const int32_t*)labels)[r]; }

// A wave's part of each of its rows: the largest score and the sum, and the label's score where it is among them.
template <class Tiles, class T>
__global__ __launch_bounds__(256, Tiles::GROUPS) void cbm_classes_kernel(CbmOperand<T> a, CbmOperand<T> b, int64_t chunks, const void* __restrict__ labels, int label_bits, Sums* __restrict__ parts,
                                                          float* __restrict__ chosen) {
    constexpr int BM = Tiles::ROWS, BN = Tiles::COLUMNS, WN = Tiles::ACROSS;
    __shared__ uintx4 lds[Tiles::UNITS];
    const int64_t tiles_n = (b.count + BN - 1) / BN;
    const CbmTilePlace at = cbm_tile_place((a.count + BM - 1) / BM, tiles_n, 1);
    if (!at.any) return;
    Tiles t;
    t.run(lds, a, b, at.m, at.n, 0, (int)chunks);
    // 32 rows at a time through LDS: two lanes a row, each half of the wave's columns
    constexpr int EACH = Tiles::COLS / 8;  // pieces of four
    const int lane = threadIdx.x & 63, half = lane & 1;
    const int64_t c0 = (int64_t)at.n * BN + t.first_column();                   // the wave's first column
    const int left = (int)min(b.count - c0, (int64_t)4096) - 4 * EACH * half;   // columns from the lane's first on
    uintx4* band = lds + t.wave() * 32 * Tiles::OUT_STRIDE;
#pragma unroll
    for (int i = 0; i < Tiles::TM; ++i) {
        __builtin_amdgcn_sched_barrier(0);
        t.band_to_lds(band, i);
        const int64_t r = (int64_t)at.m * BM + t.first_row() + 32 * i + lane / 2;
        const uintx4* row = band + lane / 2 * Tiles::OUT_STRIDE;
        if (labels && half == 0 && r < a.count) {
            const int64_t label = label_of(labels, label_bits, r), place = label - c0;
            if (label < b.count && place >= 0 && place < Tiles::COLS) chosen[r] = ((const float*)row)[place];
        }
        float z[EACH][4];
#pragma unroll
        for (int k = 0; k < EACH; ++k) t.from_lds(z[k], row + EACH * half + k);
        if (c0 + Tiles::COLS > b.count) {
            int here = left;
            asm("" : "+v"(here));  // (or a mask for each column stays in scalar registers from band to band)
#pragma unroll
            for (int k = 0; k < EACH; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) z[k][j] = 4 * k + j < here ? z[k][j] : -INFINITY;
        }
        Sums all{-INFINITY, 0.0f};
#pragma unroll
        for (int k = 0; k < EACH; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j) all.m = fmaxf(all.m, z[k][j]);
        const float away = all.m == -INFINITY ? 0.0f : all.m;
#pragma unroll
        for (int k = 0; k < EACH; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j) all.s += __builtin_amdgcn_exp2f((z[k][j] - away) * LOG2E);
        const Sums other{lane_other<1>(all.m), lane_other<1>(all.s)};
        all = half ? joined(other, all) : joined(all, other);
        if (r < a.count && half == 0) parts[r * (tiles_n * WN) + at.n * WN + t.across()] = all;
        __builtin_amdgcn_wave_barrier();
    }
}

// A few rows: W is read once, a workgroup for each 128 bytes of columns, whose scores of a row are a part.
constexpr int FEW_WAVES = 8;
template <class T, int NR>
__global__ __launch_bounds__(64 * FEW_WAVES) void cbm_classes_few_kernel(int64_t n, int64_t d, int64_t c, const T* __restrict__ X, int64_t ldx, const T* __restrict__ W, int64_t ldw,
                                                                      const void* __restrict__ labels, int label_bits, Sums* __restrict__ parts, float* __restrict__ chosen) {
    typedef CbmFewRows<T, NR, 1, 8, FEW_WAVES> Rows;
    __shared__ typename Rows::Room room;
    const int64_t piece = cbm_few_piece(), first = piece * Rows::COLS, above = (int64_t)blockIdx.y * NR;
    if (first >= c) return;
    Rows::run(room, X + above * ldx, ldx, n - above, d, {W}, {ldw}, c, first);
    const int in = threadIdx.x >> 6, lane = threadIdx.x & 63;  // a wave a row
    const int64_t r = above + in;
    if (r >= n || in >= NR) return;
    const bool some = lane < Rows::COLS && first + lane < c;
    const float z = some ? Rows::total(room, 0, in, lane < Rows::COLS ? lane : 0) : -INFINITY;
    const float m = lanes_all<64>(z, [](float a, float b) { return fmaxf(a, b); }), away = m == -INFINITY ? 0.0f : m;
    const float s = lanes_sum<64>(__builtin_amdgcn_exp2f((z - away) * LOG2E));
    if (lane == 0) parts[r * ((c + Rows::COLS - 1) / Rows::COLS) + piece] = {m, s};
    if (labels && some && label_of(labels, label_bits, r) == first + lane) chosen[r] = z;
}

// A small product: a workgroup's 32 columns are a part of its rows (256 x 1024 with 1024 x 256 in fp32 67 -> 12 us).
template <class T>
__global__ __launch_bounds__(512) void cbm_classes_small_kernel(int64_t n, int64_t d, int64_t c, const T* __restrict__ X, int64_t ldx, const T* __restrict__ W, int64_t ldw, const void* __restrict__ labels,
                                                              int label_bits, Sums* __restrict__ parts, float* __restrict__ chosen) {
    typedef CbmSmallTile<T, T, ALONG_K, ACROSS_K, 1> Tile;
    __shared__ typename Tile::Room room;
    const int64_t r0 = (int64_t)blockIdx.y * Tile::SIDE, c0 = (int64_t)blockIdx.x * Tile::SIDE, r = r0 + Tile::row(), column = c0 + Tile::column();
    Tile t;
    t.add(X, ldx, n, r0, {W}, {ldw}, c, c0, d);
    t.share(room);
    float z[2];
    Tile::total(room, 0, z);
#pragma unroll
    for (int j = 0; j < 2; ++j)
        if (column + j >= c) z[j] = -INFINITY;
    const float m = lanes_all<16>(fmaxf(z[0], z[1]), [](float a, float b) { return fmaxf(a, b); }), away = m == -INFINITY ? 0.0f : m;
    const float s = lanes_sum<16>(cbm_exp<T>(z[0] - away) + cbm_exp<T>(z[1] - away));
    if (r >= n) return;
    if (Tile::column() == 0) parts[r * gridDim.x + blockIdx.x] = {m, s};
    if (!labels) return;
    const int64_t place = label_of(labels, label_bits, r) - column;
    if (place >= 0 && place < 2 && column + place < c) chosen[r] = place ? z[1] : z[0];
}

// A small product's dZ, in fp32.
template <class T>
__global__ __launch_bounds__(512) void cbm_classes_small_slopes_kernel(int64_t n, int64_t d, int64_t c, const T* __restrict__ X, int64_t ldx, const T* __restrict__ W, int64_t ldw,
                                                                     const void* __restrict__ labels, int label_bits, const float* __restrict__ stats, const float* __restrict__ dlogp,
                                                                     float* __restrict__ dZ, int64_t lddz) {
    typedef CbmSmallTile<T, T, ALONG_K, ACROSS_K, 1> Tile;
    __shared__ typename Tile::Room room;
    const int64_t r0 = (int64_t)blockIdx.y * Tile::SIDE, c0 = (int64_t)blockIdx.x * Tile::SIDE, r = r0 + Tile::row(), column = c0 + Tile::column();
    Tile t;
    t.add(X, ldx, n, r0, {W}, {ldw}, c, c0, d);
    t.share(room);
    if (r >= n) return;
    float z[2], v[2];
    Tile::total(room, 0, z);
    const int64_t label = label_of(labels, label_bits, r);
    const float m = stats[2 * r], l = stats[2 * r + 1], slope = dlogp[r];
    const bool none = label < 0 || label >= c || m == -INFINITY;
#pragma unroll
    for (int j = 0; j < 2; ++j) v[j] = none ? 0.0f : (column + j == label ? slope : 0.0f) - slope * cbm_exp<float>((z[j] - m) - l);
    cbm_put(dZ + r * lddz, column, c, v);
}

// A row's parts in order, those of LANES lanes LANES apart, then over the lanes: a wave a row, or a lane a row where many have few parts.
template <int LANES>
__global__ __launch_bounds__(256) void cbm_classes_join_kernel(int64_t n, int64_t c, int64_t count, const void* __restrict__ labels, int label_bits, const Sums* __restrict__ parts,
                                                             const float* __restrict__ chosen, float* __restrict__ logp, float* __restrict__ stats) {
    const int lane = threadIdx.x % LANES;
    for (int64_t r = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES; r < n; r += (int64_t)gridDim.x * (256 / LANES)) {
        Sums all{-INFINITY, 0.0f};
        constexpr int AHEAD = LANES == 1 ? 2 : 8;  // (one row of 32,000 columns has 500 parts: their loads under way together, and one maximum for eight: 19.5 -> 17.9 us)
        for (int64_t i = lane; i < count; i += LANES * AHEAD) {
            Sums some[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) some[k] = i + LANES * k < count ? parts[r * count + i + LANES * k] : Sums{-INFINITY, 0.0f};
            float m = all.m;
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) m = fmaxf(m, some[k].m);
            const float away = m == -INFINITY ? 0.0f : m;
            float s = all.s * __builtin_amdgcn_exp2f((all.m - away) * LOG2E);
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) s += some[k].s * __builtin_amdgcn_exp2f((some[k].m - away) * LOG2E);
            all = {m, s};
        }
        const float m = lanes_all<LANES>(all.m, [](float a, float b) { return fmaxf(a, b); }), away = m == -INFINITY ? 0.0f : m;
        const float s = lanes_sum<LANES>(all.s * __builtin_amdgcn_exp2f((all.m - away) * LOG2E));
        if (lane) continue;
        const bool bad = !(s < INFINITY);
        const float largest = bad ? NAN : m, l = bad ? NAN : logf(s);
        if (stats) {
            stats[2 * r] = largest;
            stats[2 * r + 1] = l;
        }
        if (logp) {
            const int64_t label = label_of(labels, label_bits, r);
            logp[r] = label < 0 || label >= c ? 0.0f : bad ? NAN : m == -INFINITY ? m : (chosen[r] - m) - l;
        }
    }
}

// Types of 16 bits: dZ is kept at 2^15 over the largest finite |dlogp| of its size, of the rows that have a label and a distribution (nothing comes of the others, whatever dlogp has there); what is made of it is multiplied by the factor, scale[0], and dlogp by scale[1].  In fp16 the gradients of a batch's
// scores would be small beside 2^-14: here 1 - p fits and a p down to 2^-29 keeps all its bits.  In both types the rows of a mean, which all have the same dlogp, have their labels' own 1 - p just below a
// power of two, where half a step is 2^-9 (bf16) of it at most and p itself where that is less; at 1 / n it would be up to 2^-8, the same for every row, and nothing evens it out.
constexpr int SCALE_GROUPS = 256;
__global__ __launch_bounds__(1024) void cbm_classes_scale_kernel(int64_t n, const float* __restrict__ from, const void* __restrict__ labels, int label_bits, int64_t c, const float* __restrict__ stats,
                                                               float* __restrict__ scale, float* __restrict__ parts) {  // labels: NULL where `from` has parts
    __shared__ float room[16];
    constexpr int AHEAD = 8;
    float most = 0x1p-100f;  // (neither factor overflows)
    for (int64_t i = (int64_t)blockIdx.x * 1024 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 1024 * AHEAD) {
        float v[AHEAD];
        auto row = [&](int k) { return min(i + (int64_t)gridDim.x * 1024 * k, n - 1); };
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) v[k] = fabsf(from[row(k)]);
        if (labels) {
            int64_t label[AHEAD];
            float m[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) m[k] = stats[2 * row(k)];
            if (label_bits == 64)
#pragma unroll
                for (int k = 0; k < AHEAD; ++k) label[k] = ((const int64_t*)labels)[row(k)];
            else
#pragma unroll
                for (int k = 0; k < AHEAD; ++k) label[k] = ((const int32_t*)labels)[row(k)];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
                if (label[k] < 0 || label[k] >= c || m[k] == -INFINITY) v[k] = 0.0f;
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) most = v[k] < INFINITY ? fmaxf(most, v[k]) : most;
    }
    most = lanes_all<64>(most, [](float a, float b) { return fmaxf(a, b); });
    if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = most;
    __syncthreads();
    if (threadIdx.x) return;
    for (int i = 1; i < 16; ++i) most = fmaxf(most, room[i]);
    if (parts) {
        parts[blockIdx.x] = most;
        return;
    }
    scale[0] = most * 0x1p-15f;
    scale[1] = 0x1p15f / most;
}

// dZ of columns first .. first + width - 1, rounded to the type (half a step, as much as the gradients that are made of it are rounded by, so that those are off by 1.4 times as much as they would be; a second
// part would take their products twice as long).
template <class Tiles, class T>
__global__ __launch_bounds__(256, Tiles::GROUPS) void cbm_classes_slopes_kernel(CbmOperand<T> a, CbmOperand<T> b, int64_t width, int64_t chunks, int64_t first, int64_t c, const void* __restrict__ labels, int label_bits,
                                                                 const float* __restrict__ stats, const float* __restrict__ dlogp, const float* __restrict__ scale, T* __restrict__ dZ,
                                                                 int64_t lddz) {
    constexpr int BM = Tiles::ROWS, BN = Tiles::COLUMNS;
    __shared__ uintx4 lds[Tiles::UNITS];
    const CbmTilePlace at = cbm_tile_place((a.count + BM - 1) / BM, (b.count + BN - 1) / BN, 1);
    if (!at.any) return;
    Tiles t;
    t.run(lds, a, b, at.m, at.n, 0, (int)chunks);
    const int l32 = threadIdx.x & 31, half = threadIdx.x >> 5 & 1;
    int hot[Tiles::TM];
    float up[Tiles::TM];
#pragma unroll
    for (int i = 0; i < Tiles::TM; ++i) {
        __builtin_amdgcn_sched_barrier(0);  // (32 rows at a time: registers)
        const int64_t r = (int64_t)at.m * BM + t.first_row() + 32 * i + l32;
        const int64_t at_r = min(r, a.count - 1), label = label_of(labels, label_bits, at_r);
        const float m = stats[2 * at_r], l = stats[2 * at_r + 1];
        const bool none = label < 0 || label >= c || m == -INFINITY;
        const float slope = none ? 0.0f : scale ? dlogp[at_r] * scale[1] : dlogp[at_r], from = none ? 0.0f : m, down = none ? -INFINITY : -l * (sizeof(T) == 4 ? 1.0f : LOG2E);
        const int64_t place = label - first - ((int64_t)at.n * BN + t.first_column());
        hot[i] = none || place < 0 || place >= 32 * Tiles::TN ? -1 : (int)place;  // the label's place among the wave's columns
        up[i] = slope;
#pragma unroll
        for (int j = 0; j < Tiles::TN; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const float under = t.acc[i][j][v] - from;
                t.acc[i][j][v] = -slope * (sizeof(T) == 4 ? cbm_exp<T>(under + down) : __builtin_amdgcn_exp2f(fmaf(under, LOG2E, down)));
            }
    }
    constexpr int W = cbm_wide<T>;
    t.template pieces<W>(
        lds, at.m, at.n, [&](int64_t r, int64_t col, float (&v)[W]) {
            if (r >= a.count) return;
            if (col + W > width)
#pragma unroll
                for (int j = 0; j < W; ++j)
                    if (col + j >= width) v[j] = 0.0f;  // (products of 16 bits read whole units)
            cbm_put(dZ + r * lddz, col, (width + 7) / 8 * 8, v, true);
        },
        [&](int i, float* row) {  // a lane's row in LDS: the label's own
            if (half == 0 && hot[i] >= 0) row[hot[i]] += up[i];
        });
}

// parts of a row's scores: of 32 columns at least where rows are few or the product is small, of 64 else
bool is_small(int64_t n, int32_t d, int32_t c, int32_t type) { return cbm_small_forward(n, d, c, cbm_small_groups(n, c), type); }
int64_t most_parts(int64_t n, int32_t d, int32_t c, int32_t type) { return std::max(n <= cbm_most_few_rows<float> || is_small(n, d, c, type) ? ((int64_t)c + 31) / 32 : 0, ((int64_t)c + 127) / 128 * 2); }
int64_t rounded16(int64_t bytes) { return (bytes + 15) / 16 * 16; }
// Rows whose parts are kept at a time: 512 MiB of them, at least 256 rows.  (Also what keeps a launch below 2^32 threads: 2^18 tiles of 128 x 128 at most.)
int64_t band_of(int64_t n, int32_t d, int32_t c, int32_t type) {
    const int64_t fit = ((int64_t)512 << 20) / (most_parts(n, d, c, type) * (int64_t)sizeof(Sums)) / 256 * 256;
    return std::min(n, std::max<int64_t>(fit, 256));
}
int64_t bytes_of(int32_t type) { return type == CBM_F32 ? 4 : 2; }

// Columns of a piece of the classes whose dZ is kept at a time: 512 MiB, at least 1,024 columns.
int64_t piece_of(int64_t n, int32_t c, int32_t type) {
    const int64_t fit = ((int64_t)512 << 20) / (std::max<int64_t>(n, 1) * bytes_of(type)) / 128 * 128;
    return std::min<int64_t>(((int64_t)c + 7) / 8 * 8, std::max<int64_t>(fit, 1024));
}

// Copies of X, rows of whole units, and of W turned.
struct Copies {
    int64_t ld, weights, bytes;  // where the weights begin; X is first
};
Copies copies_of(int64_t n, int32_t d, int32_t c, int32_t type) {
    if (!cbm_may_pack(n, d, c, type)) return {};
    const int64_t ld = cbm_whole(d, 8);
    const int64_t x = 2 * cbm_whole(n, 8) * ld;
    return {ld, x, x + 2 * cbm_whole(c, 8) * ld};
}

struct Room {
    int64_t scale, sums, copies, parts, bytes;  // where they begin; dZ is first
    bool small;
};
Room back_room(int64_t n, int32_t d, int32_t c, int32_t type) {
    Room r{};
    r.small = cbm_small_backward(n, d, c, d, cbm_small_groups(n, c) + cbm_small_groups(n, d) + cbm_small_groups(d, c), type);
    if (r.small) {
        r.bytes = n * cbm_whole(c, 4) * 4;
        return r;
    }
    const int64_t piece = piece_of(n, c, type), last = c % piece ? c % piece : piece, wide = cbm_whole(d, 8);
    int64_t parts = 0;
    for (int64_t w : {piece, last}) {
        const int64_t dx = cbm_product_parts(n, d, w, type), dw = cbm_product_parts(d, w, n, type);
        if (dx > 1) parts = std::max(parts, dx * n * wide);
        if (dw > 1) parts = std::max(parts, dw * wide * cbm_whole(w, 8));
    }
    r.scale = rounded16(n * piece * bytes_of(type));
    r.sums = r.scale + 16 + 4 * SCALE_GROUPS;
    r.copies = r.sums + (piece < c ? rounded16(4 * n * wide) : 0);
    r.parts = r.copies + copies_of(n, d, c, type).bytes;
    r.bytes = r.parts + 4 * parts;
    return r;
}

// X and W as the scores' products read them: as they lie, or copies.
template <class T>
struct Operands {
    CbmOperand<T> a, b;
    bool units, turned;
    Operands(int64_t n, int32_t d, int32_t c, int32_t type, const void* X, int64_t ldx, const void* W, int64_t ldw, char* room, hipStream_t stream)
        : a{{(const T*)X, nullptr}, {ldx, 0}, n, d, 0}, b{{(const T*)W, nullptr}, {ldw, 0}, c, d, 0}, units(false), turned(false) {
        if constexpr (sizeof(T) == 2) {
            const Copies copies = copies_of(n, d, c, type);
            const bool whole = cbm_units(b.p[0], ldw, c);
            units = cbm_units(a.p[0], ldx, d);
            if (!units && copies.bytes) {
                cbm_launch_pack(X, ldx, n, d, false, room, copies.ld, 0, 0, stream);
                a = {{(const T*)room, nullptr}, {copies.ld, 0}, n, copies.ld, 0};
                units = true;
            }
            turned = units && copies.bytes && (!whole || n >= CBM_TURN_ROWS);
            if (turned) {
                cbm_launch_pack(W, ldw, c, d, true, room + copies.weights, copies.ld, 0, 0, stream);
                b = {{(const T*)(room + copies.weights), nullptr}, {copies.ld, 0}, c, copies.ld, 0};
            }
            units = units && (turned || whole);
        }
    }
    // rows `first` .. first + height - 1 of X
    CbmOperand<T> rows(int64_t first, int64_t height) const {
        CbmOperand<T> o = a;
        o.p[0] += first * a.ld[0];
        o.count = height;
        return o;
    }
    // columns `first` .. first + width - 1
    CbmOperand<T> some(int64_t first, int64_t width) const {
        CbmOperand<T> o = b;
        o.p[0] += turned ? first * b.ld[0] : first;
        o.count = width;
        return o;
    }
};

// f(tiles, grid, chunks) for a product n x d . d x c of scores
template <class T, class F>
void with_tiles(int64_t n, int64_t d, int64_t c, const Operands<T>& o, int32_t type, F&& f) {
    auto run = [&](auto* tiles_type) {
        typedef std::remove_pointer_t<decltype(tiles_type)> Tiles;
        const int64_t tiles = (n + Tiles::ROWS - 1) / Tiles::ROWS * ((c + Tiles::COLUMNS - 1) / Tiles::COLUMNS);
        f(tiles_type, (unsigned)((tiles + CBM_XCD - 1) / CBM_XCD * CBM_XCD), (d + Tiles::BK - 1) / Tiles::BK);
    };
    if constexpr (sizeof(T) == 2)
        if (o.units) {
            const bool large = cbm_product_tile(n, c, d, type) == 256;
            if (o.turned && large) run((CbmAlignedTiles<T, 256, 256, ALONG_K, ALONG_K, SINGLE>*)nullptr);
            else if (o.turned) run((CbmAlignedTiles<T, 128, 128, ALONG_K, ALONG_K, SINGLE>*)nullptr);
            else if (large) run((CbmAlignedTiles<T, 256, 256, ALONG_K, ACROSS_K, SINGLE>*)nullptr);
            else run((CbmAlignedTiles<T, 128, 128, ALONG_K, ACROSS_K, SINGLE>*)nullptr);
            return;
        }
    if constexpr (sizeof(T) == 4)
        if (cbm_is_narrow(c, type)) return run((CbmTiles<T, 256, 64, 4, 1, ALONG_K, ACROSS_K, SINGLE>*)nullptr);
    run((CbmTiles<T, 128, 128, 2, 2, ALONG_K, ACROSS_K, SINGLE>*)nullptr);
}

}  // namespace

int64_t cbm_classes_workspace(int64_t n, int32_t d, int32_t c, int32_t type) {
    const int64_t band = band_of(n, d, c, type);
    return rounded16(band * most_parts(n, d, c, type) * (int64_t)sizeof(Sums)) + rounded16(4 * band) + copies_of(n, d, c, type).bytes;
}

cbm_status cbm_launch_classes(int64_t n, int32_t d, int32_t c, int32_t type, const void* X, int64_t ldx, const void* W, int64_t ldw, const void* labels, int label_bits, float* logp, float* stats,
                              void* workspace, void* stream_) {
    hipStream_t stream = (hipStream_t)stream_;
    if (n == 0) return CBM_OK;
    const int64_t band = band_of(n, d, c, type);
    Sums* parts = (Sums*)workspace;
    float* chosen = (float*)((char*)workspace + rounded16(band * most_parts(n, d, c, type) * (int64_t)sizeof(Sums)));
    // rows r0 .. r0 + rows - 1 from their `count` parts each, of the waves along a tile's columns
    auto join = [&](int64_t r0, int64_t rows, int64_t count) {
        auto go = [&](auto lanes) {
            constexpr int LANES = decltype(lanes)::value, ROWS = 256 / LANES;
            cbm_classes_join_kernel<LANES><<<(unsigned)std::min<int64_t>((rows + ROWS - 1) / ROWS, 1 << 20), 256, 0, stream>>>(
                rows, c, count, (const char*)labels + r0 * (label_bits / 8), label_bits, parts, chosen, logp ? logp + r0 : nullptr, stats ? stats + 2 * r0 : nullptr);
        };
        // (us with 64 lanes a row / these: 2097152 x 128 with 128 x 40 857 / 325; 65536 x 64 with 64 x 1000 93 / 80)
        if (count <= 8 && rows >= 4096) go(std::integral_constant<int, 1>{});
        else if (count <= 64 && rows >= 4096) go(std::integral_constant<int, 8>{});
        else go(std::integral_constant<int, 64>{});
    };
    cbm_with_type(type, [&](auto t) {
        using T = decltype(t);
        constexpr int V = 16 / (int)sizeof(T);
        if (n <= cbm_most_few_rows<T> && c >= V) {
            const int64_t count = ((int64_t)c + 8 * V - 1) / (8 * V);
            cbm_with_few_rows(n, [&](auto rows) {
                cbm_classes_few_kernel<T, decltype(rows)::value><<<dim3((unsigned)((count + 7) / 8 * 8), (unsigned)((n + CBM_FEW_ROWS - 1) / CBM_FEW_ROWS)), 64 * FEW_WAVES, 0, stream>>>(n, d, c, (const T*)X, ldx, (const T*)W, ldw, logp ? labels : nullptr, label_bits, parts, chosen);
            });
            return join(0, n, count);
        }
        if (is_small(n, d, c, type)) {
            const int64_t count = ((int64_t)c + 31) / 32;
            cbm_classes_small_kernel<T><<<dim3((unsigned)count, (unsigned)((n + 31) / 32)), 512, 0, stream>>>(n, d, c, (const T*)X, ldx, (const T*)W, ldw, logp ? labels : nullptr, label_bits, parts, chosen);
            return join(0, n, count);
        }
        const Operands<T> o(n, d, c, type, X, ldx, W, ldw, (char*)chosen + rounded16(4 * band), stream);
        for (int64_t r0 = 0; r0 < n; r0 += band) {
            const int64_t rows = std::min(band, n - r0);
            with_tiles<T>(rows, d, c, o, type, [&](auto* tiles_type, unsigned grid, int64_t chunks) {
                typedef std::remove_pointer_t<decltype(tiles_type)> Tiles;
                cbm_classes_kernel<Tiles, T><<<grid, 256, 0, stream>>>(o.rows(r0, rows), o.b, chunks, logp ? (const char*)labels + r0 * (label_bits / 8) : nullptr, label_bits, parts, chosen);
                join(r0, rows, ((int64_t)c + Tiles::COLUMNS - 1) / Tiles::COLUMNS * Tiles::ACROSS);
            });
        }
    });
    return cbm_launched("linear log probabilities launch");
}

namespace {

bool back_too_large(int64_t n, int32_t d, int32_t c, int32_t type) {
    const int64_t piece = piece_of(n, c, type);
    return cbm_too_many_tiles(n, piece) || cbm_too_many_tiles(n, cbm_whole(d, 8)) || cbm_too_many_tiles(cbm_whole(d, 8), piece);
}

}  // namespace

int64_t cbm_classes_back_workspace(int64_t n, int32_t d, int32_t c, int32_t type) { return back_too_large(n, d, c, type) ? 0 : back_room(n, d, c, type).bytes; }

cbm_status cbm_launch_classes_backward(int64_t n, int32_t d, int32_t c, int32_t type, const void* X, int64_t ldx, const void* W, int64_t ldw, const void* labels, int label_bits,
                                       const float* stats, const float* dlogp, void* dX, int64_t lddx, void* dW, int64_t lddw, void* workspace, void* stream_) {
    hipStream_t stream = (hipStream_t)stream_;
    if (back_too_large(n, d, c, type)) return CBM_ERR_UNSUPPORTED;
    const Room room = back_room(n, d, c, type);
    if (room.small) {
        float* dZ = (float*)workspace;
        const int64_t ld = cbm_whole(c, 4);
        if (n > 0)
            cbm_with_type(type, [&](auto t) {
                using T = decltype(t);
                cbm_classes_small_slopes_kernel<T><<<dim3((unsigned)((c + 31) / 32), (unsigned)((n + 31) / 32)), 512, 0, stream>>>(n, d, c, (const T*)X, ldx, (const T*)W, ldw, labels, label_bits, stats,
                                                                                                                        dlogp, dZ, ld);
            });
        if (dX && n > 0) cbm_launch_small_along(type, n, d, c, dZ, nullptr, ld, W, ldw, nullptr, 0, dX, lddx, stream);
        if (dW) cbm_launch_small_across(type, d, c, n, X, ldx, dZ, nullptr, ld, dW, lddw, nullptr, 0, stream);
        return cbm_launched("linear log probabilities backward launch");
    }
    const int64_t piece = piece_of(n, c, type);
    float *scale = (float*)((char*)workspace + room.scale), *sums = (float*)((char*)workspace + room.sums), *parts = (float*)((char*)workspace + room.parts);
    if (type == CBM_F32) scale = nullptr;
    if (scale && n > 0) {
        float* most = scale + 4;
        const bool many = n > 1 << 16;  // (of a million rows one workgroup takes 80 us)
        if (many) cbm_classes_scale_kernel<<<SCALE_GROUPS, 1024, 0, stream>>>(n, dlogp, labels, label_bits, c, stats, nullptr, most);
        cbm_classes_scale_kernel<<<1, 1024, 0, stream>>>(many ? SCALE_GROUPS : n, many ? most : dlogp, many ? nullptr : labels, label_bits, c, stats, scale, nullptr);
    }
    cbm_with_type(type, [&](auto t) {
        using T = decltype(t);
        const Operands<T> o(n, d, c, type, X, ldx, W, ldw, (char*)workspace + room.copies, n > 0 ? stream : nullptr);
        for (int64_t first = 0; first < c; first += piece) {
            const int64_t width = std::min<int64_t>(piece, c - first);
            const CbmOperand<T> b = o.some(first, width);
            if (n > 0)
                with_tiles<T>(n, d, width, o, type, [&](auto* tiles_type, unsigned grid, int64_t chunks) {
                    cbm_classes_slopes_kernel<std::remove_pointer_t<decltype(tiles_type)>, T><<<grid, 256, 0, stream>>>(o.a, b, width, chunks, first, c, labels, label_bits, stats, dlogp, scale,
                                                                                                              (T*)workspace, piece);
                });
            CbmProduct p{};
            p.type = type;
            p.out.factor = n > 0 ? scale : nullptr;
            p.A = workspace;
            p.lda = piece;
            if (dX && n > 0) {
                p.M = n;
                p.N = d;
                p.K = width;
                p.B[0] = (const T*)W + first;
                p.ldb[0] = ldw;
                if (o.turned && !cbm_units((const T*)W, ldw, c)) {  // (dZ has whole units, and zeros beyond the last class; so has the copy)
                    p.B[0] = b.p[0];
                    p.ldb[0] = p.N = b.ld[0];
                    p.K = cbm_whole(width, 8);
                    p.b_across = true;
                }
                p.out.C[0] = dX;
                p.out.ldc[0] = lddx;
                p.out.columns = d;
                p.out.sums = piece < c ? sums : nullptr;
                p.out.first = first == 0;
                p.out.last = first + piece >= c;
                p.parts = cbm_product_parts(n, d, width, type) > 1 ? parts : nullptr;
                cbm_launch_tiles(p, stream);
            }
            if (dW) {
                p.M = d;
                p.N = width;
                p.K = n;
                p.A = X;
                p.lda = ldx;
                if (o.a.p[0] != (const T*)X) {
                    p.A = o.a.p[0];
                    p.lda = p.M = o.a.ld[0];
                    p.out.rows = d;
                }
                if (sizeof(T) == 2) p.N = cbm_whole(width, 8);
                p.a_across = p.b_across = true;
                p.B[0] = workspace;
                p.ldb[0] = piece;
                p.out.C[0] = (T*)dW + first;
                p.out.ldc[0] = lddw;
                p.out.columns = (int32_t)width;
                p.out.sums = nullptr;
                p.parts = cbm_product_parts(d, width, n, type) > 1 ? parts : nullptr;
                cbm_launch_tiles(p, stream);
            }
        }
    });
    return cbm_launched("linear log probabilities backward launch");
}
