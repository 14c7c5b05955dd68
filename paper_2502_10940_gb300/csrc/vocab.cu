// Launchers of the vocabulary kernels (vocab.cuh).
#define COLA_DEFINE_VOCAB
#include "vocab.cuh"

#include <algorithm>
#include <atomic>

namespace cola {
namespace {

// How a row is shared: `threads` of a CTA (32: a warp, four rows a CTA) and `parts` CTAs.
struct Plan {
    int threads, parts;
};

#ifndef VOCAB_FWD_GT
#define VOCAB_FWD_GT 256
#endif
#ifndef VOCAB_STEP_GT
#define VOCAB_STEP_GT 256
#endif
#ifndef VOCAB_HOLD_KB
#define VOCAB_HOLD_KB 256
#endif

// A warp or four warps where their registers hold the row (NV vectors a
// thread).  Longer rows: a forward reads tile after tile with eight warps, so
// that the ends of several rows overlap on an SM; a step, which writes what it
// has read, takes sixteen warps and as many CTAs as hold the row in
// registers, up to a portable cluster's eight; a backward a CTA per tile.  All
// take more CTAs where there are fewer rows than the device runs CTAs at once,
// down to a vector per thread.
Plan plan(const VocabParams& p, int e, int pass, bool split, int least, int sms)
{
    const int nvec = (p.vocab + e - 1) / e;
    if (least <= 32 && nvec <= 32 * NV) return {32, 1};
    if (least <= 128 && nvec <= 128 * NV) return {128, 1};
    const int threads = least > 256 ? 512 : pass == VOCAB_FWD ? VOCAB_FWD_GT : pass == VOCAB_STEP ? VOCAB_STEP_GT : 512;
    const int hold = pass == VOCAB_STEP ? (nvec * 16 <= VOCAB_HOLD_KB * 1024 ? 1 : (nvec + 512 * NV - 1) / (512 * NV))
                     : split            ? (nvec + 512 * NV - 1) / (512 * NV)
                                        : 1;
    const int fill = static_cast<int>(std::min<long long>(1024ll / threads * sms / p.n, nvec / threads));
    return {threads, std::min(CLUSTER_MAX, std::max({1, hold, fill}))};
}

template <class K>
cudaError_t launch_rows(K kern, VocabParams& p, int e, const Plan& s, bool cluster, size_t smem, cudaStream_t stream)
{
    const int rows = s.threads == 32 ? 4 : 1;
    p.each = (p.vocab / e + s.parts - 1) / s.parts;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned int>((p.n + rows - 1) / rows), s.parts);
    cfg.blockDim = dim3(s.threads * rows);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    if (cluster && s.parts > 1) {
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.y = s.parts;
        attr[0].val.clusterDim.x = attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
    }
    return cudaLaunchKernelEx(&cfg, kern, p);
}

template <class T, bool ENT>
cudaError_t logprob_top(VocabParams& p, int sms, cudaStream_t stream)
{
    constexpr int E = Elem<T>::E;
    const Plan s = plan(p, E, VOCAB_FWD, false, p.k <= 64 ? 128 : 512, sms);
    switch (s.threads) {
    case 128: return launch_rows(token_logprob_top_kernel<T, 128, ENT>, p, E, s, true, 0, stream);
    case 256: return launch_rows(token_logprob_top_kernel<T, 256, ENT>, p, E, s, true, 0, stream);
    default: return launch_rows(token_logprob_top_kernel<T, 512, ENT>, p, E, s, true, 0, stream);
    }
}

template <class T, int PASS, bool ENT>
cudaError_t logprob(VocabParams& p, int sms, cudaStream_t stream)
{
    constexpr int E = Elem<T>::E;
    const bool cluster = PASS != VOCAB_BWD;   // the backward's CTAs have nothing to exchange
    constexpr int GT = PASS == VOCAB_FWD ? VOCAB_FWD_GT : PASS == VOCAB_STEP ? VOCAB_STEP_GT : 512;
    const Plan s = plan(p, E, PASS, !cluster, 32, sms);
    switch (s.threads) {
    case 32: return launch_rows(token_logprob_kernel<T, PASS, 32, ENT>, p, E, s, cluster, 0, stream);
    case 128: return launch_rows(token_logprob_kernel<T, PASS, 128, ENT>, p, E, s, cluster, 0, stream);
    default: return launch_rows(token_logprob_kernel<T, PASS, GT, ENT>, p, E, s, cluster, 0, stream);
    }
}

template <class T>
cudaError_t logprob_pass(VocabParams p, int pass, int sms, cudaStream_t stream)
{
    if (pass == VOCAB_FWD) {
        const bool ent = p.entropy || p.stats;
        if (p.k > 0) return ent ? logprob_top<T, true>(p, sms, stream) : logprob_top<T, false>(p, sms, stream);
        return ent ? logprob<T, VOCAB_FWD, true>(p, sms, stream) : logprob<T, VOCAB_FWD, false>(p, sms, stream);
    }
    if (pass == VOCAB_STEP)
        return p.entropy || p.dentropy ? logprob<T, VOCAB_STEP, true>(p, sms, stream)
                                       : logprob<T, VOCAB_STEP, false>(p, sms, stream);
    return p.dentropy ? logprob<T, VOCAB_BWD, true>(p, sms, stream) : logprob<T, VOCAB_BWD, false>(p, sms, stream);
}

template <class T, int PASS, int GT>
cudaError_t distill_rows(VocabParams& p, const Plan& s, cudaStream_t stream)
{
    constexpr int E = Elem<T>::E;
    auto kern = topk_distill_kernel<T, PASS, GT>;
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
    return launch_rows(kern, p, E, s, true, smem, stream);
}

template <class T, int PASS>
cudaError_t distill(VocabParams p, int sms, cudaStream_t stream)
{
    constexpr int GT = PASS == VOCAB_FWD ? VOCAB_FWD_GT : PASS == VOCAB_STEP ? VOCAB_STEP_GT : 512;
    const Plan s = plan(p, Elem<T>::E, PASS, false, 32, sms);
    switch (s.threads) {
    case 32: return distill_rows<T, PASS, 32>(p, s, stream);
    case 128: return distill_rows<T, PASS, 128>(p, s, stream);
    default: return distill_rows<T, PASS, GT>(p, s, stream);
    }
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
