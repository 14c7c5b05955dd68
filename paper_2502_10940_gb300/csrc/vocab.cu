// Launchers of the vocabulary kernels (vocab.cuh).
#define COLA_DEFINE_VOCAB
#include "vocab.cuh"

#include <algorithm>

namespace cola {
namespace {

template <class K>
cudaError_t launch_rows(K kern, const VocabParams& p, int threads, int rows, bool cluster, cudaStream_t stream)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned int>((p.n + rows - 1) / rows * p.parts));
    cfg.blockDim = dim3(threads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    if (cluster && p.parts > 1) {
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = p.parts;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
    }
    return cudaLaunchKernelEx(&cfg, kern, p);
}

// Threads per row: a warp where its registers hold the row (NV vectors a
// thread), four warps likewise, else sixteen, by themselves or as one of
// `parts` CTAs: as many as hold the row in registers, up to a portable
// cluster's eight; more where there are fewer rows than CTAs the device runs at
// once (two per SM), down to a vector per thread.
int plan(VocabParams* p, int e, int least, int sms)
{
    const int nvec = (p->vocab + 2 * e - 2) / e;
    p->parts = 1;
    if (least <= 32 && nvec <= 32 * NV) return 32;
    if (least <= 128 && nvec <= 128 * NV) return 128;
    const int hold = (nvec + 512 * NV - 1) / (512 * NV);
    const int fill = static_cast<int>(std::min<long long>(2ll * sms / p->n, nvec / 512));
    p->parts = std::min(CLUSTER_MAX, std::max({1, hold, fill}));
    return 512;
}

template <class T, int PASS>
cudaError_t logprob(VocabParams p, int sms, cudaStream_t stream)
{
    const bool cluster = PASS != VOCAB_BWD;   // the backward's CTAs have nothing to exchange
    if (PASS == VOCAB_FWD && p.k > 0) {
        if (plan(&p, Elem<T>::E, p.k <= 64 ? 128 : 512, sms) == 128)
            return launch_rows(token_logprob_top_kernel<T, 128>, p, 128, 1, cluster, stream);
        return launch_rows(token_logprob_top_kernel<T, 512>, p, 512, 1, cluster, stream);
    }
    switch (plan(&p, Elem<T>::E, 32, sms)) {
    case 32: return launch_rows(token_logprob_kernel<T, PASS, 32>, p, 128, 4, cluster, stream);
    case 128: return launch_rows(token_logprob_kernel<T, PASS, 128>, p, 128, 1, cluster, stream);
    default: return launch_rows(token_logprob_kernel<T, PASS, 512>, p, 512, 1, cluster, stream);
    }
}

template <class T, int PASS>
cudaError_t distill(VocabParams p, int sms, cudaStream_t stream)
{
    switch (plan(&p, Elem<T>::E, 32, sms)) {
    case 32: return launch_rows(topk_distill_kernel<T, PASS, 32>, p, 128, 4, true, stream);
    case 128: return launch_rows(topk_distill_kernel<T, PASS, 128>, p, 128, 1, true, stream);
    default: return launch_rows(topk_distill_kernel<T, PASS, 512>, p, 512, 1, true, stream);
    }
}

template <class T>
cudaError_t logprob_pass(const VocabParams& p, int pass, int sms, cudaStream_t stream)
{
    return pass == VOCAB_FWD    ? logprob<T, VOCAB_FWD>(p, sms, stream)
           : pass == VOCAB_STEP ? logprob<T, VOCAB_STEP>(p, sms, stream)
                                : logprob<T, VOCAB_BWD>(p, sms, stream);
}

template <class T>
cudaError_t distill_pass(const VocabParams& p, int pass, int sms, cudaStream_t stream)
{
    return pass == VOCAB_FWD    ? distill<T, VOCAB_FWD>(p, sms, stream)
           : pass == VOCAB_STEP ? distill<T, VOCAB_STEP>(p, sms, stream)
                                : distill<T, VOCAB_BWD>(p, sms, stream);
}

}  // namespace

cudaError_t launch_token_logprob(const VocabParams& p, int dtype, int pass, int sms, cudaStream_t stream)
{
    return dtype == 0 ? logprob_pass<__nv_bfloat16>(p, pass, sms, stream) : logprob_pass<float>(p, pass, sms, stream);
}

cudaError_t launch_topk_distill(const VocabParams& p, int dtype, int pass, int sms, cudaStream_t stream)
{
    return dtype == 0 ? distill_pass<__nv_bfloat16>(p, pass, sms, stream) : distill_pass<float>(p, pass, sms, stream);
}

}  // namespace cola
