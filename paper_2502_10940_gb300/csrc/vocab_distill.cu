// Launchers of the distillation (vocab_distill.cuh).
#include "vocab_distill.cuh"

#include <atomic>

#include "vocab_plan.cuh"

namespace cola {
namespace {

template <class T, int PASS, int GT, bool APART>
cudaError_t distill_rows(VocabParams& p, const Plan& s, int sms, cudaStream_t stream)
{
    constexpr int E = Elem<T>::E;
    auto kern = topk_distill_kernel<T, PASS, GT, APART>;
    size_t smem = 0;
    if (PASS != VOCAB_BWD) {   // a word of bits per thread and tile
        const int each = (p.vocab / E + s.parts - 1) / s.parts;
        const int tiles = (each + GT * NV - 1) / (GT * NV);
        smem = static_cast<size_t>(std::max(tiles, 1)) * Group<GT>::THREADS * sizeof(Bits<T>);
        // beyond what a launch may have without asking for more (the static arrays take up to 6 KB)
        if (smem > 40 * 1024) {
            static std::atomic<unsigned long long> configured{0};   // bit d: set on device d
            int dev = 0;
            cudaError_t e = cudaGetDevice(&dev);
            if (e != cudaSuccess) return e;
            if (dev >= 64 || !((configured.load(std::memory_order_acquire) >> dev) & 1ull)) {
                e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, VOCAB_MAX / 8 + 8192);
                if (e != cudaSuccess) return e;
                if (dev < 64) configured.fetch_or(1ull << dev, std::memory_order_acq_rel);
            }
        }
    }
    return launch_rows(kern, p, E, s, true, smem, sms, stream);
}

template <class T, int PASS, bool APART>
cudaError_t distill_plan(VocabParams& p, const Plan& s, int sms, cudaStream_t stream)
{
    switch (s.threads) {
    case 32: return distill_rows<T, PASS, 32, false>(p, s, sms, stream);
    case 128: return distill_rows<T, PASS, 128, APART>(p, s, sms, stream);
    default:
        if constexpr (PASS == VOCAB_STEP)
            if (s.threads == 512) return distill_rows<T, PASS, 512, APART>(p, s, sms, stream);
        return distill_rows<T, PASS, 256, APART>(p, s, sms, stream);
    }
}

template <class T, int PASS>
cudaError_t distill(VocabParams p, int sms, cudaStream_t stream)
{
    const Plan s = plan(p, Elem<T>::E, PASS, false, 0, p.k, sms);
    if constexpr (PASS != VOCAB_FWD)
        if (lies_apart(p, Elem<T>::E)) return distill_plan<T, PASS, true>(p, s, sms, stream);
    return distill_plan<T, PASS, false>(p, s, sms, stream);
}

template <class T>
cudaError_t distill_pass(const VocabParams& p, int pass, int sms, cudaStream_t stream)
{
    return pass == VOCAB_FWD    ? distill<T, VOCAB_FWD>(p, sms, stream)
           : pass == VOCAB_STEP ? distill<T, VOCAB_STEP>(p, sms, stream)
                                : distill<T, VOCAB_BWD>(p, sms, stream);
}

}  // namespace

cudaError_t launch_topk_distill(const VocabParams& p, int dtype, int pass, int sms, cudaStream_t stream)
{
    return dtype == 0 ? distill_pass<__nv_bfloat16>(p, pass, sms, stream) : distill_pass<float>(p, pass, sms, stream);
}

}  // namespace cola
