// Matrices of fp32, bf16 or fp16 values seen as fp32, rows cut into pieces for lanes, and sums over lanes (device code of the operators that go
// along rows: layer norm, 8-bit checkpoints, log probabilities).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "cbm.h"

// V values of a row as fp32.  The loads ask for the alignment of one element: on gfx950 a 128-bit load may start at any of them.
template <class T, int V>
struct Piece {
    typedef T type __attribute__((ext_vector_type(V), aligned(sizeof(T))));
};
template <int V, class T>
__device__ __forceinline__ typename Piece<T, V>::type raw_piece(const T* p) {
    return *reinterpret_cast<const typename Piece<T, V>::type*>(p);
}
template <int V, class T>
__device__ __forceinline__ void widen(float (&x)[V], const typename Piece<T, V>::type& v) {
#pragma unroll
    for (int j = 0; j < V; ++j) x[j] = (float)v[j];
}
template <int V, class T>
__device__ __forceinline__ void load_piece(float (&x)[V], const T* p) {
    widen<V, T>(x, raw_piece<V>(p));
}
// far: past the caches.  Outputs that do not fit the memory-side cache of 256 MiB only push out what does (2097152 x 128 layer norm 454 -> 441 us, 2097152 x 64 restored
// from 8 bits 178 -> 106); smaller ones are left where the next call finds them.
constexpr int64_t CBM_FAR_BYTES = 256 << 20;
template <int V, class T>
__device__ __forceinline__ void store_piece(T* p, const float (&x)[V], bool far = false) {
    if constexpr (V == 1) {
        *p = (T)x[0];
    } else {
        typename Piece<T, V>::type v, *to = reinterpret_cast<typename Piece<T, V>::type*>(p);
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = (T)x[j];
        if (far) {
            asm volatile("");  // (or the two stores become one, of the usual kind)
            __builtin_nontemporal_store(v, to);
            asm volatile("");
        } else {
            *to = v;
        }
    }
}

// Piece c of a row of k >= V values: it starts at column c V, the last one at k - V where V does not divide k (WHOLE: it does).  The first `seen` of its values
// then belong to the piece before it: they are read (and written with the same bits) twice, and counted once.  A piece beyond the row has seen >= V.
template <int V, bool WHOLE>
struct Place {
    int at, seen;
    __device__ __forceinline__ Place(int c, int k) {
        at = min(c * V, k - V);
        seen = c * V - at;
    }
    __device__ __forceinline__ bool any() const { return seen < V; }
    __device__ __forceinline__ bool counts(int j) const { return WHOLE ? seen <= 0 : j >= seen; }
};

// f(the largest power of two up to k, how many lanes have such a piece each) for a row of k < V values.
template <int V, class F>
inline void cbm_narrow_row(int k, F&& f) {
    if constexpr (V > 1) {
        using std::integral_constant;
        constexpr int HALF = V / 2;
        if (k < HALF) cbm_narrow_row<HALF>(k, f);
        else if (k == HALF) f(integral_constant<int, HALF>{}, integral_constant<int, 1>{});
        else if constexpr (HALF > 1) f(integral_constant<int, HALF>{}, integral_constant<int, 2>{});
    }
}

// Sums and maxima over groups of LANES consecutive lanes, the same bits in all of them: inside a row of 16 lanes by DPP, across rows by swaps.
template <int CTRL>
__device__ __forceinline__ uint32_t lane_moved(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xf, 0xf, true);
}
template <int STEP>  // the value of the lane at distance STEP of a butterfly whose smaller steps are done
__device__ __forceinline__ uint32_t lane_other(uint32_t v) {
    static_assert(STEP == 1 || STEP == 2 || STEP == 4 || STEP == 8, "");
    if constexpr (STEP == 1) return lane_moved<0xb1>(v);        // quad_perm 1 0 3 2
    else if constexpr (STEP == 2) return lane_moved<0x4e>(v);   // quad_perm 2 3 0 1
    else if constexpr (STEP == 4) return lane_moved<0x141>(v);  // row_half_mirror: all four lanes of a quad are alike by now
    else return lane_moved<0x140>(v);                           // row_mirror
}
template <int STEP>
__device__ __forceinline__ float lane_other(float v) {
    return __uint_as_float(lane_other<STEP>(__float_as_uint(v)));
}
// f(v of the lane's even row, or half, v of its odd one): both lanes of a pair have the same two values, in the same order
template <int STEP, class U, class F>
__device__ __forceinline__ U lane_pair(U v, F&& f) {
    static_assert(STEP == 16 || STEP == 32, "");
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    if constexpr (STEP == 16) {
        const auto both = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        return f(__builtin_bit_cast(U, (uint32_t)both[0]), __builtin_bit_cast(U, (uint32_t)both[1]));
    } else {
        const auto both = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        return f(__builtin_bit_cast(U, (uint32_t)both[0]), __builtin_bit_cast(U, (uint32_t)both[1]));
    }
}
template <int LANES, class U, class F>
__device__ __forceinline__ U lanes_all(U v, F&& f) {
    if constexpr (LANES >= 2) v = f(v, lane_other<1>(v));
    if constexpr (LANES >= 4) v = f(v, lane_other<2>(v));
    if constexpr (LANES >= 8) v = f(v, lane_other<4>(v));
    if constexpr (LANES >= 16) v = f(v, lane_other<8>(v));
    if constexpr (LANES >= 32) v = lane_pair<16>(v, f);
    if constexpr (LANES >= 64) v = lane_pair<32>(v, f);
    return v;
}
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v) {
    return lanes_all<LANES>(v, [](float a, float b) { return a + b; });
}

// f(one of float, __bf16, _Float16), by a cbm_dtype; false: there is no such type
template <class F>
inline bool cbm_with_type(int32_t type, F&& f) {
    switch (type) {
        case CBM_F32: f(float{}); return true;
        case CBM_BF16: f(__bf16{}); return true;
        case CBM_F16: f(_Float16{}); return true;
    }
    return false;
}
