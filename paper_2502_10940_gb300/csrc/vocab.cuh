// vocab.cuh -- kernels over rows of vocabulary logits: log probabilities of
// given tokens with the row's entropy and most likely tokens, the distillation
// loss against a teacher's most likely tokens, and the gradients of both.
//
// Mathematics (row x of V logits, temperature T, c = 1 / T):
//   m = max x,  s = sum exp(c (x - m)),  logp_j = c (x_j - m) - log s,  p = exp(logp)
//   H = log s - c sum p_j (x_j - m)                     (both terms >= 0: nothing cancels)
//   d(g logp_y + h H)/dx_j = c (g [j = y] - p_j (g + h (logp_j + H)))
// Distillation: with q over the teacher's list, R the tokens outside it and
// (m_R, s_R) their own maximum and sum,
//   p_R = exp(c (m_R - m)) s_R / s                      (not 1 - sum p: no cancellation)
//   dx_j = w T rate exp(c (x_j - m_R)) / s_R  for j in R,   w T (Q p_k - q_k) on the list,
//   rate = sum q - sum p (rest counted) or Q p_R, Q = 1 or sum q.
#pragma once
#include <cuda_runtime.h>

namespace cola {

constexpr int VOCAB_MAX = 1 << 20;      // tokens of a vocabulary
constexpr long long VOCAB_MAX_ROWS = 1ll << 28;   // rows stay below it: a CTA of the grid each
constexpr int VOCAB_MAX_K = 256;        // alternatives, entries of a teacher's list
enum { VOCAB_FWD = 0, VOCAB_STEP = 1, VOCAB_BWD = 2 };

struct VocabParams {
    const void* logits;
    void* dlogits;
    long long n, ld, ld_d;
    int vocab, k, rest;
    int ahead;                // rows from one CTA to the next in its place
    int each;                 // 16-byte vectors of a row per CTA (the grid's y: CTAs of a row)
    float temperature;
    float c;                  // 1 / temperature
    float c2;                 // log2(e) / temperature
    float* stats;             // n x 4, written by the forward, read by the backward
    // token log probabilities
    const long long* targets;
    float* logp;
    float* entropy;
    long long* top_ids;
    float* top_logp;
    int top_each, top_before; // of each warp's largest maxima, the one it gives; how many of those lie before the bound
    const float* dlogp;
    const float* dentropy;
    // distillation
    const long long* t_ids;
    const float* t_vals;
    const float* t_lse;
    float t_c;                // 1 / the teacher's temperature
    const float* dloss;
    float* loss;
};

cudaError_t launch_token_logprob(const VocabParams& p, int dtype, int pass, int sms, cudaStream_t stream);
// the forward with p.k > 0 alternatives
cudaError_t launch_token_logprob_top(const VocabParams& p, int dtype, int sms, cudaStream_t stream);
cudaError_t launch_topk_distill(const VocabParams& p, int dtype, int pass, int sms, cudaStream_t stream);

}  // namespace cola
