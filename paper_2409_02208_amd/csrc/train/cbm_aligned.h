// Products in tiles as in cbm_tiles.h, for large matrices of 16-bit values whose rows start on 16-byte boundaries and are whole numbers of units of eight values: units go from memory into LDS
// without passing through registers, while the matrix cores work on others.
//
// Five places of an operand's 64 k each go round: both operands of a chunk, both of the next and the first of the one after.  A wave has 128 x 128 (or 64 x 64) sums and issues, between two products, at most
// one read of LDS (the next step's units) or one load: loads issued together wait for the queue to take them, and the products behind them too.  8192 x 4096 . 4096 x 8192 in bf16 (a card whose library product
// takes 405 us): two places of both operands, loads together 554 us; five places of 32 k, loads between products 500 (half of each 128-byte line a request); this 440.
// Both operands across k ask for twice as many reads, of half the size: eight at a time, or the last come too late (weights' gradients of 16384 x 1024 with 2 x 4096, slopes and all, two at a time 416 us, four 397,
// eight 394, all sixteen 396; with both along k, the gradient of X, one at a time 288, two 293, four 303).
#pragma once

#include "cbm_tiles.h"

// 16 bytes of memory to LDS for each lane: the wave's 64 units follow one another from `to` on.
__device__ __forceinline__ void cbm_unit_to_lds(const void* from, uintx4* to) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}
// What stands in for k beyond the last.
static __device__ const uintx4 cbm_no_unit = {0, 0, 0, 0};

// One operand: a tile of B rows by 64 k is 8 B units in LDS.  ALONG_K: a row's eight units follow one another, unit s of row r holding k 8 (s ^ (r / 2 & 7)) on, so that sixteen neighbouring rows' units of
// the same k fall on different banks.  ACROSS_K: the B / 8 units of a k follow one another, pairs of units (16 rows) of k changed places by 2 (k & 3), so that the four k that two times sixteen lanes turn together
// (ds_read_tr) do.
template <class T, int B, CbmTileOrder ORDER, CbmTilePair PAIR>
struct CbmAlignedSide {
    static_assert(sizeof(T) == 2, "");
    static constexpr int BK = 64, LOADS = B / 32, UNITS = 8 * B, PER = B / 8, READS = ORDER == ALONG_K ? 1 : 2;  // loads of a wave; units of a k (ACROSS_K); reads of a unit
    uint32_t offset[LOADS];                              // bytes from the tile's first value in the chunk
    const char* from[PAIR == PAIR_ROWS ? LOADS : 1];     // the unit in the first chunk, in either matrix (rows of which are as long)
    const char* base[PAIR == PAIR_K ? 2 : 1];            // of the tile's rows, k = 0
    int64_t step;                                        // bytes from a chunk to the next

    // a load's unit: row of the tile and k
    static __device__ __forceinline__ void place(int i, int wave, int lane, int& row, int& k) {
        if constexpr (ORDER == ALONG_K) {
            row = (wave * LOADS + i) * 8 + (lane >> 3);
            k = 8 * ((lane & 7) ^ (row >> 1 & 7));
        } else {
            const int slot = lane % PER;
            k = ((wave * LOADS + i) * 64 + lane) / PER;
            row = 8 * (((slot >> 1) ^ 2 * (k & 3)) << 1 | (slot & 1));
        }
    }
    __device__ __forceinline__ void begin(const CbmOperand<T>& o, int64_t tile, int wave, int rows = B) {  // tiles of `rows` rows
        const int lane = threadIdx.x & 63;
        const int64_t first = tile * rows;
        step = (ORDER == ALONG_K ? BK : BK * o.ld[0]) * 2;
        if constexpr (PAIR != PAIR_ROWS)
#pragma unroll
            for (int m = 0; m < (PAIR == PAIR_K ? 2 : 1); ++m) base[m] = (const char*)(o.p[m] + (ORDER == ALONG_K ? first * o.ld[m] : first));
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            int row, k;
            place(i, wave, lane, row, k);
            if constexpr (PAIR == PAIR_ROWS) from[i] = (const char*)(o.p[row >> 5 & 1] + k * o.ld[0] + min(tile * (B / 2) + (row >> 6) * 32 + (row & 31), o.count - 8));
            else if constexpr (ORDER == ALONG_K) offset[i] = (uint32_t)(min((int64_t)row, o.count - 1 - first) * o.ld[0] + k) * 2;
            else offset[i] = (uint32_t)(k * o.ld[0] + min((int64_t)row, o.count - 8 - first)) * 2;
        }
    }
    // WHOLE: all k of the chunk are there
    template <bool WHOLE>
    __device__ __forceinline__ void load(const CbmOperand<T>& o, int64_t chunk, int64_t end, uintx4* lds, int wave, int i) {
        const bool other = PAIR == PAIR_K && chunk * BK >= o.at;
        if (other) {
            chunk -= o.at / BK;
            end -= o.at;
        }
        const char* p;
        if constexpr (PAIR == PAIR_ROWS) p = from[i] + chunk * step;
        else p = base[PAIR == PAIR_K && other ? 1 : 0] + chunk * step + offset[i];
        if constexpr (!WHOLE) {
            int row, k;
            place(i, wave, threadIdx.x & 63, row, k);
            p = chunk * BK + k < min(end, o.K) ? p : (const char*)&cbm_no_unit;
        }
        cbm_unit_to_lds(p, lds + (wave * LOADS + i) * 64);
    }
    // the operand of rows row .. row + 31, k 16 s + 8 (lane / 32) on of the chunk
    static __device__ __forceinline__ uintx4 unit(const uintx4* lds, int row, int s) {
        const int lane = threadIdx.x & 63;
        if constexpr (ORDER == ALONG_K) {
            const int r = row + (lane & 31);
            return lds[r * 8 + ((2 * s + (lane >> 5)) ^ (r >> 1 & 7))];
        } else {
            typedef short Four __attribute__((ext_vector_type(4)));
            const int k = 16 * s + 8 * (lane >> 5) + (lane >> 2 & 3), block = ((row >> 4) + (lane >> 4 & 1)) ^ 2 * (lane >> 2 & 3);
            const char* p = (const char*)lds + k * (2 * B) + block * 32 + (lane & 3) * 8;
            struct {
                Four low, high;
            } v;
            v.low = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) Four*)p);
            v.high = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) Four*)(p + 4 * (2 * B)));
            return __builtin_bit_cast(uintx4, v);
        }
    }
};

// As CbmTiles, of 256 threads.
template <class T, int BM, int BN, CbmTileOrder ORDER_A, CbmTileOrder ORDER_B, CbmTilePair PAIR_B>
struct CbmAlignedTiles : CbmTileSums<BM, BN, 2, 2> {
    typedef CbmTileSums<BM, BN, 2, 2> Sums;
    static constexpr int TM = Sums::TM, TN = Sums::TN, BK = 64;
    typedef CbmAlignedSide<T, BM, ORDER_A, SINGLE> A;
    typedef CbmAlignedSide<T, BN, ORDER_B, PAIR_B> B;
    static constexpr int SLOT = A::UNITS > B::UNITS ? A::UNITS : B::UNITS, UNITS = 5 * SLOT, GROUPS = BM * BN > 128 * 128 ? 1 : 2;  // GROUPS: workgroups a compute unit
    static_assert(UNITS >= Sums::OUT_UNITS, "");
    using Sums::acc;

    __device__ __forceinline__ void run(uintx4* lds, const CbmOperand<T>& a, const CbmOperand<T>& b, int tile_m, int tile_n, int first, int last) {
        this->clear();
        const int wave = Sums::wave(), wm = Sums::first_row(), wn = Sums::first_column();
        A sa;
        B sb;
        sa.begin(a, tile_m, wave);
        sb.begin(b, tile_n, wave);
        const int64_t end = (int64_t)last * BK;
        auto load_a = [&](auto whole, int64_t c, uintx4* to, int i) { sa.template load<decltype(whole)::value>(a, c, end, to, wave, i); };
        auto load_b = [&](auto whole, int64_t c, uintx4* to, int i) { sb.template load<decltype(whole)::value>(b, c, end, to, wave, i); };
        if (first >= last) return;
        uintx4 *a0 = lds, *b0 = lds + SLOT, *a1 = lds + 2 * SLOT, *b1 = lds + 3 * SLOT, *a2 = lds + 4 * SLOT;
        constexpr std::false_type some;
#pragma unroll
        for (int i = 0; i < A::LOADS; ++i) load_a(some, first, a0, i);
#pragma unroll
        for (int i = 0; i < B::LOADS; ++i) load_b(some, first, b0, i);
#pragma unroll
        for (int i = 0; i < A::LOADS; ++i) load_a(some, first + 1, a1, i);
#pragma unroll
        for (int i = 0; i < B::LOADS; ++i) load_b(some, first + 1, b1, i);
#pragma unroll
        for (int i = 0; i < A::LOADS; ++i) load_a(some, first + 2, a2, i);
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(2 * A::LOADS + B::LOADS) : "memory");
        uintx4 x[2][TM], y[2][TN];
        auto read = [&](const uintx4* la, const uintx4* lb, int s) {
#pragma unroll
            for (int i = 0; i < TM; ++i) x[s & 1][i] = A::unit(la, wm + 32 * i, s);
#pragma unroll
            for (int j = 0; j < TN; ++j) y[s & 1][j] = B::unit(lb, wn + 32 * j, s);
        };
        auto multiply = [&](auto step, auto loads_) {
            constexpr int S = decltype(step)::value, LOADS_HERE = decltype(loads_)::value;
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = cbm_multiply<T>(y[S & 1][j], x[S & 1][i], acc[i][j]);
            constexpr int READS = TM * A::READS + TN * B::READS, AT_ONCE = READS > 12 ? 8 : (2 * READS + TM * TN - 1) / (TM * TN);
            __builtin_amdgcn_sched_group_barrier(0x008, 1, S);
#pragma unroll
            for (int i = 0; i < READS; i += AT_ONCE) {
                __builtin_amdgcn_sched_group_barrier(0x100, AT_ONCE, S);
                __builtin_amdgcn_sched_group_barrier(0x008, 1, S);
            }
#pragma unroll
            for (int i = 0; i < LOADS_HERE; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x020, 1, S);
                __builtin_amdgcn_sched_group_barrier(0x008, 1, S);
            }
            constexpr int LEFT = TM * TN - 1 - (READS + AT_ONCE - 1) / AT_ONCE - LOADS_HERE;
            if constexpr (LEFT > 0) __builtin_amdgcn_sched_group_barrier(0x008, LEFT, S);
            __builtin_amdgcn_sched_barrier(0);
        };
        using std::integral_constant;
        constexpr int HALF_A = A::LOADS / 2, HALF_B = B::LOADS / 2;
        read(a0, b0, 0);
        // on entry A and B of chunk c are there, A and half of B of the next under way (in the first chunk everything; what is there is loaded again, the same values)
        auto chunk = [&](auto whole, int c) {
            read(a0, b0, 1);
#pragma unroll
            for (int i = HALF_B; i < B::LOADS; ++i) load_b(whole, c + 1, b1, i);
            multiply(integral_constant<int, 0>{}, integral_constant<int, HALF_B>{});
            read(a0, b0, 2);
#pragma unroll
            for (int i = 0; i < HALF_A; ++i) load_a(whole, c + 2, a2, i);
            multiply(integral_constant<int, 1>{}, integral_constant<int, HALF_A>{});
            read(a0, b0, 3);
#pragma unroll
            for (int i = HALF_A; i < A::LOADS; ++i) load_a(whole, c + 2, a2, i);
            multiply(integral_constant<int, 2>{}, integral_constant<int, HALF_A>{});
            // A and B of the next chunk are there, in every wave, and this one's places are free: its last units are in registers
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(A::LOADS) : "memory");
            __builtin_amdgcn_sched_barrier(0);
            read(a1, b1, 0);
#pragma unroll
            for (int i = 0; i < HALF_B; ++i) load_b(whole, c + 2, a0, i);
            multiply(integral_constant<int, 3>{}, integral_constant<int, HALF_B>{});
            uintx4 *fa = a0, *fb = b0;
            a0 = a1, b0 = b1, a1 = a2, b1 = fa, a2 = fb;
        };
        const int64_t rest = PAIR_B != PAIR_K ? min(a.K, b.K) : b.at == b.K ? a.K : 0, whole = min(rest, end) / BK;  // (chunks that have all k)
        int c = first;
        for (; c + 2 < whole; ++c) chunk(std::true_type{}, c);
        for (; c < last; ++c) chunk(std::false_type{}, c);
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");  // (the places are free for what comes next)
    }
};

// Whether a matrix can be read in whole units from 16-byte boundaries (o: along the units), a tile's within 32 bits of its first.
template <class T>
inline bool cbm_units(const T* p, int64_t ld, int64_t along) {
    return ((uintptr_t)p & 15) == 0 && ld % 8 == 0 && along % 8 == 0 && ld < (int64_t)1 << 22;
}
