// constrain.cuh -- what a server imposes on rows of logits before a token is
// taken from them: penalties for tokens that occurred, biases, masks; and the
// gradient through them.
//
// Mathematics (logit x of a token that occurs c times in its row's history
// after the prompt; r, f, p the row's penalties):
//   x := x > 0 ? x / r : x r     where the whole history has the token
//   x := x - f c - p [c > 0],    x := x + the sum of its entries among the biases
//   x := -inf                    where the row's mask has a 0 bit for it
//   dx = dy (1 / r or r as above, else 1), 0 where masked
#pragma once
#include <cuda_runtime.h>

namespace cola {

constexpr int BIAS_MAX = 1024;                          // entries of a row
constexpr long long HISTORY_MAX = (1ll << 28) - 1;      // ids of a row

struct ConstrainParams {
    const void* logits;
    const void* src;          // what is copied: the logits, or the upstream gradient
    void* dst;
    long long n, ld, ld_src, ld_dst;
    int vocab;
    int each;                 // 16-byte vectors of a row per CTA (the grid's y)
    int words, counts;        // of a CTA's tokens: words of a bit each, words of counts
    int list;                 // tokens that a CTA may list
    int over;                 // the gradient lies over the logits
    const long long* history;
    long long history_width, ld_history;
    const long long* history_len;
    const long long* prompt_len;
    const float* repetition;
    const float* frequency;
    const float* presence;
    const long long* bias_ids;
    const float* bias;
    int n_bias;
    const unsigned int* masks;
    long long n_masks, ld_masks;
    const long long* mask_of;
};

cudaError_t launch_constrain(const ConstrainParams& p, int dtype, bool backward, int sms, cudaStream_t stream);

}  // namespace cola
