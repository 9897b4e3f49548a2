// extern "C" boundary of the operators between the products: layer norm, 8-bit checkpoints, log probabilities.  Argument checks and dispatch.
#include <cmath>
#include <cstdint>

#include "cbm_internal.h"

namespace {

constexpr int32_t MOST_COLUMNS = 1 << 24;

int64_t element_bytes(int32_t type) { return type == CBM_F32 ? 4 : type == CBM_BF16 || type == CBM_F16 ? 2 : 0; }

int64_t steps(int32_t k) { return ((int64_t)k + 31) / 32; }  // blocks of columns in a row of the 8-bit form

// The memory that an operand spans, from its first element to its last.
struct Span {
    const void* p;
    uintptr_t b, e;
};
// A matrix of n rows of k elements.  *st: what is wrong with it, if anything is.
Span matrix(const void* p, int64_t n, int64_t k, int64_t ld, int64_t bytes, cbm_status* st) {
    Span s{p, (uintptr_t)p, (uintptr_t)p};
    if (ld < k || (n > 0 && k > 0 && !p) || (uintptr_t)p % (uintptr_t)bytes) {
        *st = CBM_ERR_INVALID_ARG;
    } else if (n > 0 && k > 0) {
        if (ld > (INT64_MAX / 16) / n) *st = *st == CBM_OK ? CBM_ERR_UNSUPPORTED : *st;
        else s.e = s.b + (uintptr_t)(((n - 1) * ld + k) * bytes);
    }
    return s;
}
Span maybe(const void* p, int64_t count, int64_t bytes, cbm_status* st) { return p ? matrix(p, 1, count, count, bytes, st) : Span{nullptr, 0, 0}; }
// Whether one of the outputs overlaps an input or another output.
template <int I, int O>
bool overlap(const Span (&in)[I], const Span (&out)[O]) {
    auto meet = [](const Span& a, const Span& b) { return a.b < b.e && b.b < a.e; };
    for (int o = 0; o < O; ++o) {
        for (const Span& s : in)
            if (meet(s, out[o])) return true;
        for (int q = 0; q < o; ++q)
            if (meet(out[q], out[o])) return true;
    }
    return false;
}

}  // namespace

extern "C" {

cbm_status cbm_layer_norm(int64_t n, int32_t k, int32_t type, const void* X, int64_t ldx, const float* gamma, const float* beta, float eps, void* Y, int64_t ldy,
                          float* mean, float* rstd, void* hip_stream) {
    const int64_t bytes = element_bytes(type);
    if (n < 0 || k <= 0 || !bytes || !(eps >= 0.0f) || !std::isfinite(eps)) return CBM_ERR_INVALID_ARG;
    if (k > MOST_COLUMNS) return CBM_ERR_UNSUPPORTED;
    cbm_status st = CBM_OK;
    const Span in[3] = {matrix(X, n, k, ldx, bytes, &st), maybe(gamma, k, 4, &st), maybe(beta, k, 4, &st)};
    const Span out[3] = {matrix(Y, n, k, ldy, bytes, &st), maybe(mean, n, 4, &st), maybe(rstd, n, 4, &st)};
    if (st != CBM_OK) return st;
    if (overlap(in, out)) return CBM_ERR_INVALID_ARG;
    return cbm_launch_norm(n, k, type, X, ldx, gamma, beta, eps, Y, ldy, mean, rstd, hip_stream);
}

size_t cbm_layer_norm_workspace_bytes(int64_t n, int32_t k) {
    return n < 0 || k <= 0 || k > MOST_COLUMNS ? 0 : (size_t)cbm_norm_parts(n, k) * 2 * (size_t)k * sizeof(float);
}

cbm_status cbm_layer_norm_backward(int64_t n, int32_t k, int32_t type, const void* dY, int64_t lddy, const void* X, int64_t ldx, const float* gamma, const float* mean,
                                   const float* rstd, void* dX, int64_t lddx, float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const int64_t bytes = element_bytes(type);
    if (n < 0 || k <= 0 || !bytes || (!dX && !dgamma && !dbeta)) return CBM_ERR_INVALID_ARG;
    if (k > MOST_COLUMNS) return CBM_ERR_UNSUPPORTED;
    cbm_status st = CBM_OK;
    const bool sums = dgamma || dbeta;
    const size_t need = sums ? cbm_layer_norm_workspace_bytes(n, k) : 0;
    if (need && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 15))) return CBM_ERR_INVALID_ARG;
    const Span in[5] = {matrix(dY, n, k, lddy, bytes, &st), matrix(X, n, k, ldx, bytes, &st), maybe(gamma, k, 4, &st), matrix(mean, 1, n, n, 4, &st), matrix(rstd, 1, n, n, 4, &st)};
    const Span out[4] = {dX ? matrix(dX, n, k, lddx, bytes, &st) : Span{nullptr, 0, 0}, maybe(dgamma, k, 4, &st), maybe(dbeta, k, 4, &st),
                         Span{workspace, (uintptr_t)workspace, (uintptr_t)workspace + need}};
    if (st != CBM_OK) return st;
    if (overlap(in, out)) return CBM_ERR_INVALID_ARG;
    return cbm_launch_norm_backward(n, k, type, dY, lddy, X, ldx, gamma, mean, rstd, dX, lddx, dgamma, dbeta, (float*)workspace, hip_stream);
}

cbm_status cbm_checkpoint_save(int64_t n, int32_t k, int32_t type, const void* X, int64_t ldx, int8_t* Q, int64_t ldq, uint8_t* E, int64_t lde, void* hip_stream) {
    const int64_t bytes = element_bytes(type);
    if (n < 0 || k <= 0 || !bytes) return CBM_ERR_INVALID_ARG;
    if (k > MOST_COLUMNS) return CBM_ERR_UNSUPPORTED;
    cbm_status st = CBM_OK;
    const Span in[1] = {matrix(X, n, k, ldx, bytes, &st)};
    const Span out[2] = {matrix(Q, n, k, ldq, 1, &st), matrix(E, n, steps(k), lde, 1, &st)};
    if (st != CBM_OK) return st;
    if (overlap(in, out)) return CBM_ERR_INVALID_ARG;
    return cbm_launch_checkpoint_save(n, k, type, X, ldx, Q, ldq, E, lde, hip_stream);
}

cbm_status cbm_checkpoint_restore(int64_t n, int32_t k, const int8_t* Q, int64_t ldq, const uint8_t* E, int64_t lde, int32_t type, void* X, int64_t ldx, void* hip_stream) {
    const int64_t bytes = element_bytes(type);
    if (n < 0 || k <= 0 || !bytes) return CBM_ERR_INVALID_ARG;
    if (k > MOST_COLUMNS) return CBM_ERR_UNSUPPORTED;
    cbm_status st = CBM_OK;
    const Span in[2] = {matrix(Q, n, k, ldq, 1, &st), matrix(E, n, steps(k), lde, 1, &st)};
    const Span out[1] = {matrix(X, n, k, ldx, bytes, &st)};
    if (st != CBM_OK) return st;
    if (overlap(in, out)) return CBM_ERR_INVALID_ARG;
    return cbm_launch_checkpoint_load(n, k, Q, ldq, E, lde, type, nullptr, 0, X, ldx, hip_stream);
}

cbm_status cbm_checkpoint_relu_backward(int64_t n, int32_t k, const int8_t* Q, int64_t ldq, const uint8_t* E, int64_t lde, int32_t type, const void* dY, int64_t lddy, void* dX,
                                        int64_t lddx, void* hip_stream) {
    const int64_t bytes = element_bytes(type);
    if (n < 0 || k <= 0 || !bytes) return CBM_ERR_INVALID_ARG;
    if (k > MOST_COLUMNS) return CBM_ERR_UNSUPPORTED;
    cbm_status st = CBM_OK;
    const Span dy = matrix(dY, n, k, lddy, bytes, &st);
    const bool in_place = dX == dY && lddx == lddy;  // (what two lanes read and write, of a row's last piece, is the same gated once or twice)
    const Span in[3] = {matrix(Q, n, k, ldq, 1, &st), matrix(E, n, steps(k), lde, 1, &st), in_place ? Span{nullptr, 0, 0} : dy};
    const Span out[1] = {matrix(dX, n, k, lddx, bytes, &st)};
    if (st != CBM_OK) return st;
    if (overlap(in, out)) return CBM_ERR_INVALID_ARG;
    return cbm_launch_checkpoint_load(n, k, Q, ldq, E, lde, type, dY, lddy, dX, lddx, hip_stream);
}

size_t cbm_checkpoint_workspace_bytes(int64_t n, int32_t k, int32_t c) {
    if (n <= 0 || k <= 0 || c <= 0 || k > MOST_COLUMNS || c > MOST_COLUMNS) return 0;
    const int64_t splits = cbm_grad_splits(n, k, c);
    return splits == 1 ? 0 : (size_t)splits * (size_t)k * (size_t)c * sizeof(float);
}

cbm_status cbm_checkpoint_weight_grad(int64_t n, int32_t k, int32_t c, const int8_t* Q, int64_t ldq, const uint8_t* E, int64_t lde, int32_t type, const void* dY, int64_t lddy,
                                      float* dW, int64_t lddw, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const int64_t bytes = element_bytes(type);
    if (n < 0 || k <= 0 || c <= 0 || !bytes) return CBM_ERR_INVALID_ARG;
    if (k > MOST_COLUMNS || c > MOST_COLUMNS || (int64_t)k * c > (int64_t)1 << 32) return CBM_ERR_UNSUPPORTED;
    const size_t need = cbm_checkpoint_workspace_bytes(n, k, c);
    if (need && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 15))) return CBM_ERR_INVALID_ARG;
    cbm_status st = CBM_OK;
    const Span in[3] = {matrix(Q, n, k, ldq, 1, &st), matrix(E, n, steps(k), lde, 1, &st), matrix(dY, n, c, lddy, bytes, &st)};
    const Span out[2] = {matrix(dW, k, c, lddw, 4, &st), Span{workspace, (uintptr_t)workspace, (uintptr_t)workspace + need}};
    if (st != CBM_OK) return st;
    if (overlap(in, out)) return CBM_ERR_INVALID_ARG;
    return cbm_launch_checkpoint_grad(n, k, c, Q, ldq, E, lde, type, dY, lddy, dW, lddw, (float*)workspace, hip_stream);
}

size_t cbm_log_probs_workspace_bytes(int64_t n, int32_t c, int32_t top) {
    if (n <= 0 || c <= 0 || c > MOST_COLUMNS || top < 0 || top > CBM_MOST_TOP) return 0;
    const int splits = cbm_scores_splits(n, c);
    return splits == 1 ? 0 : (size_t)n * (size_t)splits * cbm_scores_part_bytes(top);
}

cbm_status cbm_log_probs(int64_t n, int32_t c, int32_t type, const void* Z, int64_t ldz, const void* labels, int32_t label_bits, float* logp, float* entropy, float* stats, int32_t top,
                         float* top_values, int32_t* top_columns, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const int64_t bytes = element_bytes(type);
    if (n < 0 || c <= 0 || !bytes || top < 0 || top > CBM_MOST_TOP || (label_bits != 32 && label_bits != 64)) return CBM_ERR_INVALID_ARG;
    if (c > MOST_COLUMNS) return CBM_ERR_UNSUPPORTED;
    const size_t need = cbm_log_probs_workspace_bytes(n, c, top);
    if (need && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 15))) return CBM_ERR_INVALID_ARG;
    cbm_status st = CBM_OK;
    const Span none{nullptr, 0, 0};
    const Span in[2] = {matrix(Z, n, c, ldz, bytes, &st), logp ? matrix(labels, 1, n, n, label_bits / 8, &st) : none};
    const Span out[6] = {maybe(logp, n, 4, &st), maybe(entropy, n, 4, &st), maybe(stats, 2 * n, 4, &st), top ? matrix(top_values, n, top, top, 4, &st) : none,
                         top ? matrix(top_columns, n, top, top, 4, &st) : none, Span{workspace, (uintptr_t)workspace, (uintptr_t)workspace + need}};
    if (st != CBM_OK) return st;
    if (overlap(in, out)) return CBM_ERR_INVALID_ARG;
    return cbm_launch_scores(n, c, type, Z, ldz, labels, label_bits, logp, entropy, stats, top, top_values, top_columns, workspace, hip_stream);
}

cbm_status cbm_log_probs_backward(int64_t n, int32_t c, int32_t type, const void* Z, int64_t ldz, const void* labels, int32_t label_bits, const float* stats, const float* entropy,
                                  const float* dlogp, const float* dentropy, void* dZ, int64_t lddz, void* hip_stream) {
    const int64_t bytes = element_bytes(type);
    if (n < 0 || c <= 0 || !bytes || (label_bits != 32 && label_bits != 64) || (n > 0 && !dlogp && !dentropy)) return CBM_ERR_INVALID_ARG;
    if (c > MOST_COLUMNS) return CBM_ERR_UNSUPPORTED;
    cbm_status st = CBM_OK;
    const Span none{nullptr, 0, 0}, z = matrix(Z, n, c, ldz, bytes, &st);
    const bool in_place = dZ == Z && lddz == ldz;  // (a value is read for good before it is written, by one lane)
    const Span in[6] = {in_place ? none : z, dlogp ? matrix(labels, 1, n, n, label_bits / 8, &st) : none, matrix(stats, 1, 2 * n, 2 * n, 4, &st),
                        dentropy ? matrix(entropy, 1, n, n, 4, &st) : none, maybe(dlogp, n, 4, &st), maybe(dentropy, n, 4, &st)};
    const Span out[1] = {matrix(dZ, n, c, lddz, bytes, &st)};
    if (st != CBM_OK) return st;
    if (overlap(in, out)) return CBM_ERR_INVALID_ARG;
    return cbm_launch_scores_backward(n, c, type, Z, ldz, labels, label_bits, stats, entropy, dlogp, dentropy, dZ, lddz, hip_stream);
}

}  // extern "C"
