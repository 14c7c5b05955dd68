// Launchers of the token log probabilities (vocab_logprob.cuh).
#include "vocab_logprob.cuh"
#include "vocab_plan.cuh"

namespace cola {
namespace {

template <class T, int PASS, bool ENT, bool APART>
cudaError_t logprob_rows(VocabParams& p, const Plan& s, int sms, cudaStream_t stream)
{
    constexpr int E = Elem<T>::E;
    const bool cluster = PASS != VOCAB_BWD;   // the backward's CTAs have nothing to exchange
    switch (s.threads) {
    case 32: return launch_rows(token_logprob_kernel<T, PASS, 32, ENT, false>, p, E, s, cluster, 0, sms, stream);
    case 128: return launch_rows(token_logprob_kernel<T, PASS, 128, ENT, APART>, p, E, s, cluster, 0, sms, stream);
    default:
        if constexpr (PASS == VOCAB_STEP)
            if (s.threads == 512)
                return launch_rows(token_logprob_kernel<T, PASS, 512, ENT, APART>, p, E, s, cluster, 0, sms, stream);
        return launch_rows(token_logprob_kernel<T, PASS, 256, ENT, APART>, p, E, s, cluster, 0, sms, stream);
    }
}

template <class T, int PASS, bool ENT>
cudaError_t logprob(VocabParams& p, int sms, cudaStream_t stream)
{
    const Plan s = plan(p, Elem<T>::E, PASS, PASS == VOCAB_BWD, 0, 0, sms);
    if constexpr (PASS != VOCAB_FWD)
        if (lies_apart(p, Elem<T>::E)) return logprob_rows<T, PASS, ENT, true>(p, s, sms, stream);
    return logprob_rows<T, PASS, ENT, false>(p, s, sms, stream);
}

template <class T>
cudaError_t logprob_pass(VocabParams p, int pass, int sms, cudaStream_t stream)
{
    if (pass == VOCAB_FWD)
        return p.entropy || p.stats ? logprob<T, VOCAB_FWD, true>(p, sms, stream) : logprob<T, VOCAB_FWD, false>(p, sms, stream);
    if (pass == VOCAB_STEP)
        return p.entropy || p.dentropy ? logprob<T, VOCAB_STEP, true>(p, sms, stream)
                                       : logprob<T, VOCAB_STEP, false>(p, sms, stream);
    return p.dentropy ? logprob<T, VOCAB_BWD, true>(p, sms, stream) : logprob<T, VOCAB_BWD, false>(p, sms, stream);
}

}  // namespace

cudaError_t launch_token_logprob(const VocabParams& p, int dtype, int pass, int sms, cudaStream_t stream)
{
    if (pass == VOCAB_FWD && p.k > 0) return launch_token_logprob_top(p, dtype, sms, stream);
    return dtype == 0 ? logprob_pass<__nv_bfloat16>(p, pass, sms, stream) : logprob_pass<float>(p, pass, sms, stream);
}

}  // namespace cola
