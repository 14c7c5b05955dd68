// Launchers of the vocabulary kernels (vocab.cuh): one CTA per row.
#define COLA_DEFINE_VOCAB
#include "vocab.cuh"

#include <atomic>

namespace cola {
namespace {

template <class K>
cudaError_t launch_rows(K kern, const VocabParams& p, size_t smem, std::atomic<unsigned long long>& configured,
                        cudaStream_t stream)
{
    if (smem > 32 * 1024) {
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        if (dev >= 64 || !((configured.load(std::memory_order_acquire) >> dev) & 1ull)) {
            e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, VOCAB_MAX / 8 + 1024);
            if (e != cudaSuccess) return e;
            if (dev < 64) configured.fetch_or(1ull << dev, std::memory_order_acq_rel);
        }
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned int>(p.n));
    cfg.blockDim = dim3(VT);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    return cudaLaunchKernelEx(&cfg, kern, p);
}

template <class T, int PASS>
cudaError_t logprob(const VocabParams& p, cudaStream_t stream)
{
    static std::atomic<unsigned long long> configured{0};
    return launch_rows(token_logprob_kernel<T, PASS>, p, 0, configured, stream);
}

template <class T, int PASS>
cudaError_t distill(const VocabParams& p, cudaStream_t stream)
{
    static std::atomic<unsigned long long> configured{0};
    return launch_rows(topk_distill_kernel<T, PASS>, p, (static_cast<size_t>(p.vocab) + 8 + 31) / 32 * 4, configured,
                       stream);
}

}  // namespace

cudaError_t launch_token_logprob(const VocabParams& p, int dtype, int pass, cudaStream_t stream)
{
    if (dtype == 0)
        return pass == VOCAB_FWD ? logprob<__nv_bfloat16, VOCAB_FWD>(p, stream)
               : pass == VOCAB_STEP ? logprob<__nv_bfloat16, VOCAB_STEP>(p, stream)
                                    : logprob<__nv_bfloat16, VOCAB_BWD>(p, stream);
    return pass == VOCAB_FWD ? logprob<float, VOCAB_FWD>(p, stream)
           : pass == VOCAB_STEP ? logprob<float, VOCAB_STEP>(p, stream)
                                : logprob<float, VOCAB_BWD>(p, stream);
}

cudaError_t launch_topk_distill(const VocabParams& p, int dtype, int pass, cudaStream_t stream)
{
    if (dtype == 0)
        return pass == VOCAB_FWD ? distill<__nv_bfloat16, VOCAB_FWD>(p, stream)
               : pass == VOCAB_STEP ? distill<__nv_bfloat16, VOCAB_STEP>(p, stream)
                                    : distill<__nv_bfloat16, VOCAB_BWD>(p, stream);
    return pass == VOCAB_FWD ? distill<float, VOCAB_FWD>(p, stream)
           : pass == VOCAB_STEP ? distill<float, VOCAB_STEP>(p, stream)
                                : distill<float, VOCAB_BWD>(p, stream);
}

}  // namespace cola
