// Launchers of the token log probabilities with top alternatives (vocab_top.cuh).
#include "vocab_plan.cuh"
#include "vocab_top.cuh"

namespace cola {
namespace {

template <class T, bool ENT>
cudaError_t logprob_top(VocabParams& p, int sms, cudaStream_t stream)
{
    constexpr int E = Elem<T>::E;
    const Plan s = plan(p, E, VOCAB_FWD, false, p.k, 0, sms);
    // a cluster's bound: of each warp, a little more of its largest than k over the warps
    // (one CTA, with more than k warps too: the k-th largest of the warps' maxima)
    const int warps = s.threads / 32 * s.parts;
    p.top_each = p.k <= warps || s.parts == 1 ? 1 : (3 * p.k + 2 * warps - 1) / (2 * warps);
    p.top_before = (p.k + p.top_each - 1) / p.top_each - 1;
    switch (s.threads) {
    case 32: return launch_rows(token_logprob_top_warp_kernel<T, ENT>, p, E, s, false, 0, sms, stream);
    case 128:
        // (more than 64 only of rows that 128 threads hold)
        return p.k > 64 ? launch_rows(token_logprob_top_kernel<T, 128, ENT, true>, p, E, s, false, 0, sms, stream)
                        : launch_rows(token_logprob_top_kernel<T, 128, ENT, false>, p, E, s, false, 0, sms, stream);
    case 256: return launch_rows(token_logprob_top_kernel<T, 256, ENT, false>, p, E, s, true, 0, sms, stream);
    default: return launch_rows(token_logprob_top_kernel<T, 512, ENT, false>, p, E, s, true, 0, sms, stream);
    }
}

template <class T>
cudaError_t logprob_top_dtype(VocabParams p, int sms, cudaStream_t stream)
{
    return p.entropy || p.stats ? logprob_top<T, true>(p, sms, stream) : logprob_top<T, false>(p, sms, stream);
}

}  // namespace

cudaError_t launch_token_logprob_top(const VocabParams& p, int dtype, int sms, cudaStream_t stream)
{
    return dtype == 0 ? logprob_top_dtype<__nv_bfloat16>(p, sms, stream) : logprob_top_dtype<float>(p, sms, stream);
}

}  // namespace cola
