// Products of matrices of fp32, bf16 or fp16 values in tiles, with the sums left in registers for whatever a kernel makes of them (device code of the
// operators that are made of products: gated layer, log probabilities of a layer's classes, orthogonal update).
//
// The operands of a matrix instruction are units of eight consecutive k of one row (of the result's rows, or of its columns).  A workgroup keeps a chunk of both operands in LDS as such
// units, in whatever order the matrices lie in memory: along k a unit is read as it is, across k a thread reads the same few columns of eight k and turns them in registers.
// fp32 values are split into three bf16 parts that add up to them as they are stored (cbm_split.h), and six products of parts are made, as in cbm_gemm_split.hip: what is left out is
// at most 2^-24 of a term.  Parts below 2^-126 are taken for zero, and a value that is not finite makes NaN of the sums that it reaches.
#pragma once

#include "cbm_elems.h"
#include "cbm_split.h"

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

template <class T>
struct CbmTileType {  // 16 bits
    static constexpr int PARTS = 1, KG = 8;  // parts of a value, units of eight k in a chunk
};
template <>
struct CbmTileType<float> {
    static constexpr int PARTS = 3, KG = 4;
};

// e^x from 2^x.  fp32: with what x log2(e) loses when it is rounded, which at an x of -20 is twenty steps of the result.
template <class T>
__device__ __forceinline__ float cbm_exp(float x) {
    const float t = x * 1.44269504f;
    if constexpr (sizeof(T) == 2) return __builtin_amdgcn_exp2f(t);
    const float lost = fmaxf(fmaf(x, 1.44269504f, -t) + x * 1.92596299e-8f, -1.0f);  // (NaN where x is infinite)
    return __builtin_amdgcn_exp2f(t) * fmaf(lost, 0.693147181f, 1.0f);
}

enum CbmTileOrder { ALONG_K, ACROSS_K };

// One operand of a product: `count` rows of `K` values.  ALONG_K: value (r, k) is p[r ld + k]; ACROSS_K: p[k ld + r].  Two matrices may share the operand: PAIR_K, the second one's k follow
// those of the first from `at` on (a multiple of the chunk; both have K of their own); PAIR_ROWS, blocks of 32 rows of the tile come from the one and the other in turn.
enum CbmTilePair { SINGLE, PAIR_K, PAIR_ROWS };
template <class T>
struct CbmOperand {
    const T* p[2];
    int64_t ld[2];
    int64_t count;
    int64_t K;   // of one of the matrices
    int64_t at;  // PAIR_K
};

template <class T, int B, int THREADS, CbmTileOrder ORDER, CbmTilePair PAIR>
struct CbmTileSide {
    static constexpr int PARTS = CbmTileType<T>::PARTS, KG = CbmTileType<T>::KG, BK = 8 * KG;
    static constexpr int EACH = B * KG / THREADS;  // units a thread stages
    // Places of units in LDS: sixteen neighbouring rows, sixteen groups of four rows (or of two) and four rows of four k each fall on different banks.
    static constexpr int STRIDE = B + 17, PLANE = KG * STRIDE, UNITS = PARTS * PLANE;
    static __device__ __forceinline__ int place(int kg, int row) { return kg * STRIDE + (row & 3) * (B / 4 + 4) + (row >> 2); }
    static_assert(B * KG % THREADS == 0 && THREADS % KG == 0, "");
    typedef typename Piece<T, EACH>::type Across;
    typedef typename Piece<T, 16 / (int)sizeof(T)>::type Quad;  // 16 bytes
    static constexpr int QUADS = 8 * sizeof(T) / 16;

    const T* base[EACH];  // ALONG_K: the unit's first value of k = 0; ACROSS_K: [0], the thread's first column of k = 0
    const T* second[PAIR == PAIR_K ? EACH : 1];
    int64_t ld;
    int shift;     // ACROSS_K: columns that the thread loads and another one has: its own come after them
    bool element = false;  // ACROSS_K: fewer columns than a thread has
    int most;      // the last column, as seen from the thread's first (element)
    int kg0, row0;
    union {
        Quad along[EACH][QUADS];
        Across across[8];
    } raw;

    __device__ __forceinline__ void begin(const CbmOperand<T>& o, int64_t tile) {
        const int t = threadIdx.x;
        if constexpr (ORDER == ALONG_K) {
            kg0 = t % KG;
            row0 = t / KG;
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                const int64_t r = min(tile * B + row0 + i * (THREADS / KG), o.count - 1);
                base[i] = o.p[0] + r * o.ld[0] + 8 * kg0;
                if constexpr (PAIR == PAIR_K) second[i] = o.p[1] + r * o.ld[1] + 8 * kg0;
            }
        } else {
            row0 = t % (B / EACH) * EACH;
            kg0 = t / (B / EACH);
            const int which = PAIR == PAIR_ROWS ? row0 >> 5 & 1 : 0;
            const int64_t c = PAIR == PAIR_ROWS ? tile * (B / 2) + (row0 >> 6) * 32 + (row0 & 31) : tile * B + row0;
            element = o.count < EACH;
            const int64_t from = element ? 0 : min(c, o.count - EACH);
            shift = element ? 0 : (int)min(c - from, (int64_t)EACH);
            most = (int)o.count - 1;
            ld = o.ld[which];
            base[0] = o.p[which] + from + 8 * kg0 * ld;
        }
    }
    // the thread's units of the chunk at k0
    __device__ __forceinline__ void load(const CbmOperand<T>& o, int64_t k0) {
        const int64_t K = o.K;
        if constexpr (ORDER == ALONG_K) {
            const bool other = PAIR == PAIR_K && k0 >= o.at;
            if (other) k0 -= o.at;
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                const T* p = (PAIR == PAIR_K && other ? second[PAIR == PAIR_K ? i : 0] : base[i]) + k0;
                if (k0 + BK <= K || k0 + 8 * kg0 + 8 <= K) {
#pragma unroll
                    for (int q = 0; q < QUADS; ++q) raw.along[i][q] = *reinterpret_cast<const Quad*>(p + q * (16 / (int)sizeof(T)));
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) raw.along[i][j * (int)sizeof(T) / 16][j % (16 / (int)sizeof(T))] = k0 + 8 * kg0 + j < K ? p[j] : (T)0.0f;
                }
            }
        } else {
            const T* p = base[0] + k0 * ld;
            if (k0 + BK <= K && !element) {
#pragma unroll
                for (int j = 0; j < 8; ++j) raw.across[j] = *reinterpret_cast<const Across*>(p + j * ld);
            } else {
                const int left = (int)min(K - k0 - 8 * kg0, (int64_t)8);  // of the thread's eight k
                if (left <= 0) p = base[0] - 8 * kg0 * ld;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const T* q = p + max(min(j, left - 1), 0) * ld;
                    if (element) {
#pragma unroll
                        for (int i = 0; i < EACH; ++i) raw.across[j][i] = q[min(i, most)];
                    } else {
                        raw.across[j] = *reinterpret_cast<const Across*>(q);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint32_t keep = j < left ? ~0u : 0u;
                    typedef uint32_t Words __attribute__((ext_vector_type(EACH * (int)sizeof(T) / 4)));
                    raw.across[j] = __builtin_bit_cast(Across, __builtin_bit_cast(Words, raw.across[j]) & keep);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
    }
    static __device__ __forceinline__ void put(uintx4* lds, int at, const float (&x)[8], uint32_t minus_low) {
        uintx4 q[3];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t h, m, l;
            split_pair_nearest(x[2 * i], x[2 * i + 1], minus_low, h, m, l);
            q[0][i] = h;
            q[1][i] = m;
            q[2][i] = l;
        }
#pragma unroll
        for (int i = 0; i < 3; ++i) lds[i * PLANE + at] = q[i];
    }
    // unit i to LDS
    __device__ __forceinline__ void store(uintx4* lds, uint32_t minus_low, int i) {
        const int at = ORDER == ALONG_K ? place(kg0, row0 + i * (THREADS / KG))
                       : i < shift      ? kg0 * STRIDE + B + 16  // (columns that another thread has go to a place that nobody reads)
                                        : place(kg0, row0 + i - shift);
        if constexpr (PARTS == 1) {
            if constexpr (ORDER == ALONG_K) {
                lds[at] = __builtin_bit_cast(uintx4, raw.along[i][0]);
            } else {
                typedef uint32_t Words __attribute__((ext_vector_type(EACH / 2)));
                uintx4 q;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    q[j] = __builtin_amdgcn_perm(__builtin_bit_cast(Words, raw.across[2 * j + 1])[i / 2], __builtin_bit_cast(Words, raw.across[2 * j])[i / 2],
                                                 i % 2 ? 0x07060302u : 0x05040100u);
                lds[at] = q;
            }
        } else {
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = ORDER == ALONG_K ? (float)raw.along[i][j / 4][j % 4] : (float)raw.across[j][i];
            put(lds, at, x, minus_low);
        }
    }
};

template <class T>
__device__ __forceinline__ floatx16 cbm_multiply(uintx4 a, uintx4 b, floatx16 sum) {
    if constexpr (std::is_same<T, _Float16>::value) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), sum, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), sum, 0, 0, 0);
}

// The sums of a workgroup's tile, BM rows by BN columns of the result.  A wave has TM x TN tiles of 32 x 32; lane l's row in a tile is l % 32, its
// columns are 8 q + 4 (l / 32) + 0 .. 3 for q = 0 .. 3 (the operands change places in the instruction, so that a lane's values lie along the result's rows).
template <int BM, int BN, int WM, int WN>
struct CbmTileSums {
    static constexpr int ROWS = BM, COLUMNS = BN, WAVES = WM * WN, THREADS = 64 * WAVES, TM = BM / WM / 32, TN = BN / WN / 32, ACROSS = WN;
    floatx16 acc[TM][TN];

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;
    }
    static __device__ __forceinline__ int wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }
    // the wave's first row and column in the tile, and its place among the waves along the columns
    static __device__ __forceinline__ int first_row() { return wave() % WM * (32 * TM); }
    static __device__ __forceinline__ int first_column() { return wave() / WM * (32 * TN); }
    static __device__ __forceinline__ int across() { return wave() / WM; }
    // f(row, column of the first, four sums) for the wave's part of the result, rows of lanes along its rows: through LDS, 32 rows at a time, a place for each wave (65536 x 1024 with 2 x 4096
    // in bf16: pieces of 8 bytes 1596 us, of 16, and past the caches where the result does not fit them, 1342).  The operands' places in LDS have to be free.
    static constexpr int COLS = 32 * TN, OUT_STRIDE = COLS / 4 + 1, OUT_UNITS = WAVES * 32 * OUT_STRIDE;
    __device__ __forceinline__ void band_to_lds(uintx4* to, int i) const {
        const int l32 = threadIdx.x & 31, half = threadIdx.x >> 5 & 1;
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                to[l32 * OUT_STRIDE + 8 * j + 2 * q + half] = __builtin_bit_cast(uintx4, (floatx4){acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]});
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    template <int W>
    static __device__ __forceinline__ void from_lds(float (&v)[W], const uintx4* p) {
#pragma unroll
        for (int k = 0; k < W / 4; ++k) {
            const floatx4 x = __builtin_bit_cast(floatx4, p[k]);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[4 * k + j] = x[j];
        }
    }
    struct Nothing {
        __device__ __forceinline__ void operator()(int, float*) const {}
    };
    // W sums a lane at a time.  change(i, row): of lanes 0 .. 31, band i's sums of the lane's row before f sees them
    template <int W, class F, class G = Nothing>
    __device__ __forceinline__ void pieces(uintx4* lds, int64_t tile_m, int64_t tile_n, F&& f, G&& change = G()) const {
        const int lane = threadIdx.x & 63;
        uintx4* mine = lds + wave() * 32 * OUT_STRIDE;
        const int64_t row = tile_m * BM + first_row(), column = tile_n * BN + first_column();
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            band_to_lds(mine, i);
            if constexpr (!std::is_same<std::remove_reference_t<G>, Nothing>::value) {
                change(i, (float*)(mine + (lane & 31) * OUT_STRIDE));
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
            }
#pragma unroll 1
            for (int t = 0; t < COLS / 2 / W; ++t) {
                const int at = 64 * t + lane, r = at / (COLS / W), c = at % (COLS / W);
                float v[W];
                from_lds(v, mine + r * OUT_STRIDE + W / 4 * c);
                f(row + 32 * i + r, column + W * c, v);
            }
            __builtin_amdgcn_wave_barrier();
        }
    }
    // PAIR_ROWS: f(row, column, W sums of the first matrix's columns, of the second's)
    template <int W, class F>
    __device__ __forceinline__ void pairs(uintx4* lds, int64_t tile_m, int64_t tile_n, F&& f) const {
        const int lane = threadIdx.x & 63;
        uintx4* mine = lds + wave() * 32 * OUT_STRIDE;
        const int64_t row = tile_m * BM + first_row(), column = tile_n * (BN / 2) + first_column() / 2;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            band_to_lds(mine, i);
#pragma unroll 1
            for (int t = 0; t < COLS / 4 / W; ++t) {
                const int at = 64 * t + lane, r = at / (COLS / 2 / W), c = at % (COLS / 2 / W) * (W / 4), p = r * OUT_STRIDE + c / 8 * 16 + c % 8;
                float x[W], y[W];
                from_lds(x, mine + p);
                from_lds(y, mine + p + 8);
                f(row + 32 * i + r, column + 4 * c, x, y);
            }
            __builtin_amdgcn_wave_barrier();
        }
    }
};

// Over chunks first .. last - 1 of K.
template <class T, int BM, int BN, int WM, int WN, CbmTileOrder ORDER_A, CbmTileOrder ORDER_B, CbmTilePair PAIR_B>
struct CbmTiles : CbmTileSums<BM, BN, WM, WN> {
    typedef CbmTileSums<BM, BN, WM, WN> Sums;
    static constexpr int THREADS = Sums::THREADS, TM = Sums::TM, TN = Sums::TN;
    typedef CbmTileSide<T, BM, THREADS, ORDER_A, SINGLE> A;
    typedef CbmTileSide<T, BN, THREADS, ORDER_B, PAIR_B> B;
    static constexpr int PARTS = A::PARTS, BK = A::BK, OPERANDS = A::UNITS + B::UNITS, UNITS = OPERANDS > Sums::OUT_UNITS ? OPERANDS : Sums::OUT_UNITS, GROUPS = 2;  // GROUPS: workgroups a compute unit
    using Sums::acc;

    __device__ __forceinline__ void run(uintx4* lds, const CbmOperand<T>& a, const CbmOperand<T>& b, int tile_m, int tile_n, int first, int last) {
        constexpr int P2 = PARTS == 1 ? 0 : 1;
        floatx16 small[P2 ? TM : 1][P2 ? TN : 1];
        this->clear();
        if constexpr (P2)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) small[i][j] = acc[i][j];
        uint32_t minus_low = 0xbf80u;
        asm("" : "+s"(minus_low));
        const int l32 = threadIdx.x & 31, half = threadIdx.x >> 5 & 1, wm = Sums::first_row(), wn = Sums::first_column();
        uintx4 *la = lds, *lb = lds + A::UNITS;
        A sa;
        B sb;
        sa.begin(a, tile_m);
        sb.begin(b, tile_n);
        if (first < last) {
            sa.load(a, (int64_t)first * BK);
            sb.load(b, (int64_t)first * BK);
        }
        for (int c = first; c < last; ++c) {
#pragma unroll
            for (int i = 0; i < A::EACH; ++i) sa.store(la, minus_low, i);
#pragma unroll
            for (int i = 0; i < B::EACH; ++i) sb.store(lb, minus_low, i);
            __syncthreads();
            if (c + 1 < last) {
                sa.load(a, (int64_t)(c + 1) * BK);
                sb.load(b, (int64_t)(c + 1) * BK);
            }
            const int left = P2 && PAIR_B != PAIR_K ? (int)min(b.K - (int64_t)c * BK, (int64_t)BK) : BK;  // (K = 100: seven steps of 16 instead of eight)
#pragma unroll
            for (int s = 0; s < BK / 16; ++s) {
                if (s > 0 && 16 * s >= left) break;
                uintx4 x[TM][PARTS], y[TN][PARTS];
#pragma unroll
                for (int p = 0; p < PARTS; ++p) {
#pragma unroll
                    for (int i = 0; i < TM; ++i) x[i][p] = la[p * A::PLANE + A::place(2 * s + half, wm + 32 * i + l32)];
#pragma unroll
                    for (int j = 0; j < TN; ++j) y[j][p] = lb[p * B::PLANE + B::place(2 * s + half, wn + 32 * j + l32)];
                }
                if constexpr (P2) {
                    constexpr int PA[6] = {2, 0, 1, 1, 0, 0}, PB[6] = {0, 2, 1, 0, 1, 0};  // the product of the large parts last, into sums of its own
#pragma unroll
                    for (int q = 0; q < 6; ++q)
#pragma unroll
                        for (int i = 0; i < TM; ++i)
#pragma unroll
                            for (int j = 0; j < TN; ++j) {
                                floatx16& sum = q < 5 ? small[i][j] : acc[i][j];
                                sum = cbm_multiply<T>(y[j][PB[q]], x[i][PA[q]], sum);
                            }
                } else {
#pragma unroll
                    for (int i = 0; i < TM; ++i)
#pragma unroll
                        for (int j = 0; j < TN; ++j) acc[i][j] = cbm_multiply<T>(y[j][0], x[i][0], acc[i][j]);
                }
            }
            __syncthreads();
        }
        if constexpr (P2)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int v = 0; v < 16; ++v) acc[i][j][v] += small[i][j][v];
    }
};

// Tiles of the result for workgroup b of a grid of a multiple of 8: an XCD (b mod 8) has neighbouring ones, in blocks of 8 tiles of rows, so that what its workgroups read
// at a time fits its L2.
struct CbmTilePlace {
    int m, n, split;
    bool any;
};
__device__ __forceinline__ CbmTilePlace cbm_tile_place(int64_t tiles_m, int64_t tiles_n, int64_t splits) {
    const uint32_t high_all = (uint32_t)tiles_m, wide = (uint32_t)tiles_n, per = gridDim.x / 8, at = blockIdx.x % 8 * per + blockIdx.x / 8, tiles = high_all * wide, split = at / tiles, tile = at % tiles;
    const uint32_t group = tile / (8 * wide), high = min(8u, high_all - 8 * group), in = tile - group * 8 * wide;
    auto whole = [](uint32_t v) { return __builtin_amdgcn_readfirstlane((int)v); };  // (divisions are made in vector registers, and would stay there)
    return {whole(8 * group + in % high), whole(in / high), whole(split), split < (uint32_t)splits};
}

// W values of a row of `columns` from `c` on (none beyond them); far: past the caches.
template <int W, class T>
__device__ __forceinline__ void cbm_put(T* row, int64_t c, int64_t columns, const float (&v)[W], bool far = false) {
    if (c + W <= columns) {
        store_piece<W>(row + c, v, far);
    } else {
#pragma unroll
        for (int j = 0; j < W; ++j)
            if (c + j < columns) row[c + j] = (T)v[j];
    }
}
// values of 16 bytes
template <class T>
constexpr int cbm_wide = 16 / (int)sizeof(T);
