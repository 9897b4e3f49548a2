// The orthogonal update: a matrix's singular values driven towards one by products alone.
#include <algorithm>

#include "cbm_internal.h"
#include "cbm_products.h"
#include "cbm_tiles.h"

namespace {

constexpr int PARTS = 256;  // workgroups that share the sum of squares

// Squares in 64 bits: no value of fp32 overflows or vanishes there.
template <class T>
__global__ __launch_bounds__(256) void cbm_orthogonal_norm_kernel(int64_t m, int64_t n, const T* __restrict__ X, int64_t ldx, double* __restrict__ parts) {
    __shared__ double room[256];
    double s = 0.0;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < m * n; i += (int64_t)gridDim.x * 256) {
        const double x = (double)(float)X[i / n * ldx + i % n];
        s += x * x;
    }
    room[threadIdx.x] = s;
    __syncthreads();
    for (int step = 128; step; step /= 2) {
        if ((int)threadIdx.x < step) room[threadIdx.x] += room[threadIdx.x + step];
        __syncthreads();
    }
    if (threadIdx.x == 0) parts[blockIdx.x] = room[0];
}

// The matrix, or its transpose, over its norm + eps, in 32 bits.
template <class T>
__global__ __launch_bounds__(256) void cbm_orthogonal_begin_kernel(int64_t m, int64_t n, const T* __restrict__ X, int64_t ldx, bool transposed, float eps, const double* __restrict__ parts,
                                                                float* __restrict__ out) {
    double s = 0.0;
    for (int i = 0; i < PARTS; ++i) s += parts[i];
    const double size = sqrt(s) + (double)eps;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < m * n; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / n, c = i % n;  // of `out`
        const double x = (double)(float)(transposed ? X[c * ldx + r] : X[r * ldx + c]);
        out[i] = (float)(x / size);
    }
}

template <class T>
__global__ __launch_bounds__(256) void cbm_orthogonal_end_kernel(int64_t m, int64_t n, const float* __restrict__ x, bool transposed, float scale, T* __restrict__ Y, int64_t ldy) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < m * n; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / n, c = i % n;  // of Y
        Y[r * ldy + c] = (T)(scale * x[transposed ? c * m + r : i]);
    }
}

int64_t padded(int64_t v) { return (v + 3) / 4 * 4; }
unsigned blocks_of(int64_t values) { return (unsigned)std::min<int64_t>((values + 255) / 256, 1 << 20); }

}  // namespace

int64_t cbm_orthogonal_workspace(int32_t m, int32_t n, int32_t) {
    const int64_t s = std::min(m, n), l = std::max(m, n);
    const int64_t parts = std::max(cbm_product_parts(s, s, l, CBM_F32) * s * s, cbm_product_parts(s, l, s, CBM_F32) * s * l);
    return PARTS * 8 + 4 * (2 * padded(s * l) + 2 * padded(s * s) + parts);
}

cbm_status cbm_launch_orthogonal(int32_t m, int32_t n, int32_t type, const void* X, int64_t ldx, int32_t steps, const float* abc, float eps, float scale, void* Y, int64_t ldy, void* workspace,
                                 void* stream_) {
    hipStream_t stream = (hipStream_t)stream_;
    const bool tall = m > n;
    const int64_t s = std::min(m, n), l = std::max(m, n);
    double* squares = (double*)workspace;
    float *x = (float*)(squares + PARTS), *other = x + padded(s * l), *gram = other + padded(s * l), *poly = gram + padded(s * s), *parts = poly + padded(s * s);
    cbm_with_type(type, [&](auto t) {
        using T = decltype(t);
        cbm_orthogonal_norm_kernel<T><<<PARTS, 256, 0, stream>>>(m, n, (const T*)X, ldx, squares);
        cbm_orthogonal_begin_kernel<T><<<blocks_of(s * l), 256, 0, stream>>>(s, l, (const T*)X, ldx, tall, eps, squares, x);
    });
    for (int i = 0; i < steps; ++i) {
        CbmProduct p{};
        p.type = p.out.type = CBM_F32;
        p.out.first = p.out.last = true;
        auto run = [&](int64_t M, int64_t N, int64_t K, const float* a, const float* b, bool across, float* c, float alpha, const float* more, float beta) {
            p.M = M;
            p.N = N;
            p.K = K;
            p.A = a;
            p.lda = K;
            p.B[0] = b;
            p.ldb[0] = across ? N : K;
            p.b_across = across;
            p.out.C[0] = c;
            p.out.ldc[0] = p.out.ldm = N;
            p.out.columns = (int32_t)N;
            p.out.alpha = alpha;
            p.out.more = more;
            p.out.beta = beta;
            p.parts = parts;
            cbm_launch_tiles(p, stream);
        };
        run(s, s, l, x, x, false, gram, 1.0f, nullptr, 0.0f);
        run(s, s, s, gram, gram, false, poly, abc[2], gram, abc[1]);  // (the Gram matrix is symmetric)
        run(s, l, s, poly, x, true, other, 1.0f, x, abc[0]);
        std::swap(x, other);
    }
    cbm_with_type(type, [&](auto t) {
        using T = decltype(t);
        cbm_orthogonal_end_kernel<T><<<blocks_of(s * l), 256, 0, stream>>>(m, n, x, tall, scale, (T*)Y, ldy);
    });
    return cbm_launched("orthogonal update launch");
}
