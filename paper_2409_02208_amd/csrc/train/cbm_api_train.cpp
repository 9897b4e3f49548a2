// extern "C" boundary of the operators of a training step: layer norm, 8-bit checkpoints, log probabilities, gated layer, log probabilities of a layer's classes, orthogonal update.
// Argument checks and dispatch.
#include <cmath>
#include <cstdint>

#include "cbm_internal.h"

namespace {

constexpr int32_t MOST_COLUMNS = 1 << 24;
constexpr int64_t MOST_ROWS = (int64_t)1 << 31;  // of a product
constexpr int32_t MOST_SIDE = 1 << 16;           // of a matrix whose powers are made
constexpr int32_t MOST_STEPS = 100;

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
Span perhaps(const void* p, int64_t n, int64_t k, int64_t ld, int64_t bytes, cbm_status* st) { return p ? matrix(p, n, k, ld, bytes, st) : Span{nullptr, 0, 0}; }
Span room(const void* p, size_t bytes) { return Span{p, (uintptr_t)p, (uintptr_t)p + bytes}; }
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

size_t cbm_gated_linear_workspace_bytes(int64_t n, int32_t k, int32_t m, int32_t type) {
    return n <= 0 || k <= 0 || m <= 0 || n > MOST_ROWS || k > MOST_COLUMNS || m > MOST_COLUMNS || !element_bytes(type) ? 0 : (size_t)cbm_gated_workspace(n, k, m, type);
}

cbm_status cbm_gated_linear(int64_t n, int32_t k, int32_t m, int32_t type, int32_t activation, const void* X, int64_t ldx, const void* Wg, int64_t ldwg, const void* Wu, int64_t ldwu, void* H,
                            int64_t ldh, void* G, int64_t ldg, void* U, int64_t ldu, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const int64_t bytes = element_bytes(type);
    if (n < 0 || k <= 0 || m <= 0 || !bytes || activation < CBM_SILU || activation > CBM_RELU) return CBM_ERR_INVALID_ARG;
    if (k > MOST_COLUMNS || m > MOST_COLUMNS || n > MOST_ROWS) return CBM_ERR_UNSUPPORTED;
    const size_t need = cbm_gated_linear_workspace_bytes(n, k, m, type);
    if (need && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 15))) return CBM_ERR_INVALID_ARG;
    cbm_status st = CBM_OK;
    const Span in[3] = {matrix(X, n, k, ldx, bytes, &st), matrix(Wg, k, m, ldwg, bytes, &st), matrix(Wu, k, m, ldwu, bytes, &st)};
    const Span out[4] = {matrix(H, n, m, ldh, bytes, &st), perhaps(G, n, m, ldg, bytes, &st), perhaps(U, n, m, ldu, bytes, &st), room(workspace, need)};
    if (st != CBM_OK) return st;
    if (overlap(in, out)) return CBM_ERR_INVALID_ARG;
    return cbm_launch_gated(n, k, m, type, activation, X, ldx, Wg, ldwg, Wu, ldwu, H, ldh, G, ldg, U, ldu, workspace, hip_stream);
}

size_t cbm_gated_linear_backward_workspace_bytes(int64_t n, int32_t k, int32_t m, int32_t type) {
    return n < 0 || k <= 0 || m <= 0 || n > MOST_ROWS || k > MOST_COLUMNS || m > MOST_COLUMNS || !element_bytes(type) ? 0 : (size_t)cbm_gated_back_workspace(n, k, m, type);
}

cbm_status cbm_gated_linear_backward(int64_t n, int32_t k, int32_t m, int32_t type, int32_t activation, const void* dH, int64_t lddh, const void* X, int64_t ldx, const void* Wg, int64_t ldwg,
                                     const void* Wu, int64_t ldwu, const void* G, int64_t ldg, const void* U, int64_t ldu, void* dX, int64_t lddx, void* dWg, int64_t lddwg, void* dWu,
                                     int64_t lddwu, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const int64_t bytes = element_bytes(type);
    if (n < 0 || k <= 0 || m <= 0 || !bytes || activation < CBM_SILU || activation > CBM_RELU || (!dX && !dWg && !dWu)) return CBM_ERR_INVALID_ARG;
    if (k > MOST_COLUMNS || m > MOST_COLUMNS || n > MOST_ROWS) return CBM_ERR_UNSUPPORTED;
    const size_t need = cbm_gated_linear_backward_workspace_bytes(n, k, m, type);
    if (need && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 15))) return CBM_ERR_INVALID_ARG;
    cbm_status st = CBM_OK;
    const Span in[6] = {matrix(dH, n, m, lddh, bytes, &st), matrix(X, n, k, ldx, bytes, &st), matrix(Wg, k, m, ldwg, bytes, &st), matrix(Wu, k, m, ldwu, bytes, &st),
                        matrix(G, n, m, ldg, bytes, &st), matrix(U, n, m, ldu, bytes, &st)};
    const Span out[4] = {perhaps(dX, n, k, lddx, bytes, &st), perhaps(dWg, k, m, lddwg, bytes, &st), perhaps(dWu, k, m, lddwu, bytes, &st), room(workspace, need)};
    if (st != CBM_OK) return st;
    if (overlap(in, out)) return CBM_ERR_INVALID_ARG;
    return cbm_launch_gated_backward(n, k, m, type, activation, dH, lddh, X, ldx, Wg, ldwg, Wu, ldwu, G, ldg, U, ldu, dX, lddx, dWg, lddwg, dWu, lddwu, workspace, hip_stream);
}

size_t cbm_linear_log_probs_workspace_bytes(int64_t n, int32_t d, int32_t c, int32_t type) {
    return n <= 0 || d <= 0 || c <= 0 || n > MOST_ROWS || d > MOST_COLUMNS || c > MOST_COLUMNS || !element_bytes(type) ? 0 : (size_t)cbm_classes_workspace(n, d, c, type);
}

cbm_status cbm_linear_log_probs(int64_t n, int32_t d, int32_t c, int32_t type, const void* X, int64_t ldx, const void* W, int64_t ldw, const void* labels, int32_t label_bits, float* logp,
                                float* stats, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const int64_t bytes = element_bytes(type);
    if (n < 0 || d <= 0 || c <= 0 || !bytes || (label_bits != 32 && label_bits != 64)) return CBM_ERR_INVALID_ARG;
    if (d > MOST_COLUMNS || c > MOST_COLUMNS || n > MOST_ROWS) return CBM_ERR_UNSUPPORTED;
    const size_t need = cbm_linear_log_probs_workspace_bytes(n, d, c, type);
    if (need && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 15))) return CBM_ERR_INVALID_ARG;
    cbm_status st = CBM_OK;
    const Span none{nullptr, 0, 0};
    const Span in[3] = {matrix(X, n, d, ldx, bytes, &st), matrix(W, d, c, ldw, bytes, &st), logp ? matrix(labels, 1, n, n, label_bits / 8, &st) : none};
    const Span out[3] = {maybe(logp, n, 4, &st), maybe(stats, 2 * n, 4, &st), room(workspace, need)};
    if (st != CBM_OK) return st;
    if (overlap(in, out)) return CBM_ERR_INVALID_ARG;
    return cbm_launch_classes(n, d, c, type, X, ldx, W, ldw, labels, label_bits, logp, stats, workspace, hip_stream);
}

size_t cbm_linear_log_probs_backward_workspace_bytes(int64_t n, int32_t d, int32_t c, int32_t type) {
    return n < 0 || d <= 0 || c <= 0 || n > MOST_ROWS || d > MOST_COLUMNS || c > MOST_COLUMNS || !element_bytes(type) ? 0 : (size_t)cbm_classes_back_workspace(n, d, c, type);
}

cbm_status cbm_linear_log_probs_backward(int64_t n, int32_t d, int32_t c, int32_t type, const void* X, int64_t ldx, const void* W, int64_t ldw, const void* labels, int32_t label_bits,
                                         const float* stats, const float* dlogp, void* dX, int64_t lddx, void* dW, int64_t lddw, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const int64_t bytes = element_bytes(type);
    if (n < 0 || d <= 0 || c <= 0 || !bytes || (label_bits != 32 && label_bits != 64) || (!dX && !dW)) return CBM_ERR_INVALID_ARG;
    if (d > MOST_COLUMNS || c > MOST_COLUMNS || n > MOST_ROWS) return CBM_ERR_UNSUPPORTED;
    const size_t need = cbm_linear_log_probs_backward_workspace_bytes(n, d, c, type);
    if (need && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 15))) return CBM_ERR_INVALID_ARG;
    cbm_status st = CBM_OK;
    const Span in[5] = {matrix(X, n, d, ldx, bytes, &st), matrix(W, d, c, ldw, bytes, &st), matrix(labels, 1, n, n, label_bits / 8, &st), matrix(stats, 1, 2 * n, 2 * n, 4, &st),
                        matrix(dlogp, 1, n, n, 4, &st)};
    const Span out[3] = {perhaps(dX, n, d, lddx, bytes, &st), perhaps(dW, d, c, lddw, bytes, &st), room(workspace, need)};
    if (st != CBM_OK) return st;
    if (overlap(in, out)) return CBM_ERR_INVALID_ARG;
    return cbm_launch_classes_backward(n, d, c, type, X, ldx, W, ldw, labels, label_bits, stats, dlogp, dX, lddx, dW, lddw, workspace, hip_stream);
}

size_t cbm_orthogonalise_workspace_bytes(int32_t m, int32_t n, int32_t type) {
    return m <= 0 || n <= 0 || m > MOST_SIDE || n > MOST_SIDE || !element_bytes(type) ? 0 : (size_t)cbm_orthogonal_workspace(m, n, type);
}

cbm_status cbm_orthogonalise(int32_t m, int32_t n, int32_t type, const void* X, int64_t ldx, int32_t steps, const float* coefficients, float eps, float scale, void* Y, int64_t ldy,
                             void* workspace, size_t workspace_bytes, void* hip_stream) {
    static const float usual[3] = {3.4445f, -4.7750f, 2.0315f};
    const float* abc = coefficients ? coefficients : usual;
    const int64_t bytes = element_bytes(type);
    if (m <= 0 || n <= 0 || !bytes || steps < 0 || steps > MOST_STEPS || !(eps >= 0.0f) || !std::isfinite(eps) || !std::isfinite(scale)) return CBM_ERR_INVALID_ARG;
    for (int i = 0; i < 3; ++i)
        if (!std::isfinite(abc[i])) return CBM_ERR_INVALID_ARG;
    if (m > MOST_SIDE || n > MOST_SIDE) return CBM_ERR_UNSUPPORTED;
    const size_t need = cbm_orthogonalise_workspace_bytes(m, n, type);
    if (need && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 15))) return CBM_ERR_INVALID_ARG;
    cbm_status st = CBM_OK;
    const Span x = matrix(X, m, n, ldx, bytes, &st);
    const bool in_place = Y == X && ldy == ldx;  // (X is read before the first product)
    const Span in[1] = {in_place ? Span{nullptr, 0, 0} : x};
    const Span out[2] = {matrix(Y, m, n, ldy, bytes, &st), room(workspace, need)};
    if (st != CBM_OK) return st;
    if (overlap(in, out)) return CBM_ERR_INVALID_ARG;
    return cbm_launch_orthogonal(m, n, type, X, ldx, steps, abc, eps, scale, Y, ldy, workspace, hip_stream);
}

}  // extern "C"
