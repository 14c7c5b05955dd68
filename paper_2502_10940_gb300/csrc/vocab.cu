// Launchers of the vocabulary kernels (vocab.cuh).
#define COLA_DEFINE_VOCAB
#include "vocab.cuh"

#include <algorithm>
#include <atomic>
#include <cmath>

namespace cola {
namespace {

// How a row is shared: `threads` of a CTA (32: a warp, four rows a CTA) and `parts` CTAs.
struct Plan {
    int threads, parts;
};

// Bytes of the rows that the device works on at once that L2 still holds when a
// step reads them again, its stores beside them: at 39 and 61 MB a step over rows
// of 64 and 100 KB runs at 1.00 and 0.93 of the copy bandwidth, at 122 MB (rows of
// 200 KB on one CTA each) at 0.84, on two at 0.93.
constexpr double STEP_L2_BYTES = 62e6;

// A warp or four warps where their registers hold the row (NV vectors a
// thread).  Longer rows take eight warps, so that the phases of four rows overlap
// on an SM, tile after tile; sixteen where eight have too few threads for the
// bound of the top k (`least`).  A step reads its row twice, the second time from L2:
// as many CTAs share a row as keep the rows in flight within it, sixteen warps
// where that would take more than a portable cluster's eight CTAs.  The
// backward without a list (`split`) exchanges nothing: a CTA per tile.  All take more CTAs
// where there are fewer rows than the device runs CTAs at once, down to a vector
// per thread.  CTAs that form a cluster are a power of two: threes and sixes
// leave SMs empty (390 us against 332 us for a step of 2048 x 262144 on six and four).
Plan plan(const VocabParams& p, int e, int pass, bool split, int least, int sms)
{
    const int nvec = (p.vocab + e - 1) / e;
    if (least <= 32 && nvec <= 32 * NV) return {32, 1};
    if (least <= 128 && nvec <= 128 * NV) return {128, 1};
    int threads = least <= 256 ? 256 : 512, hold = 1;
    if (pass == VOCAB_STEP) {
        hold = static_cast<int>(std::ceil(4.0 * sms * 16.0 * nvec / STEP_L2_BYTES));
        if (hold > CLUSTER_MAX) threads = 512, hold = (hold + 1) / 2;
    } else if (pass == VOCAB_BWD) {
        threads = 512;
        if (split) hold = (nvec + 512 * NV - 1) / (512 * NV);
    }
    const int fill = static_cast<int>(std::min<long long>(1024ll / threads * sms / p.n, nvec / threads));
    if (split) return {threads, std::min(CLUSTER_MAX, std::max(hold, fill))};
    int parts = 1;
    while (parts < CLUSTER_MAX && (parts < hold || 2 * parts <= fill)) parts *= 2;
    return {threads, parts};
}

template <class K>
cudaError_t launch_rows(K kern, VocabParams& p, int e, const Plan& s, bool cluster, size_t smem, int sms, cudaStream_t stream)
{
    const int rows = s.threads == 32 ? 4 : 1;
    p.each = (p.vocab / e + s.parts - 1) / s.parts;
    p.ahead = static_cast<int>(sms * 1024ll / (s.threads * rows) / s.parts * rows);
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
    const Plan s = plan(p, E, VOCAB_FWD, false, p.k <= 64 ? 128 : p.k <= 128 ? 256 : 512, sms);
    // one CTA: the k-th largest of its warps' maxima, or (counted by the CTA) of its threads';
    // a cluster: of each warp a little more of the largest than k over the warps
    const int warps = s.threads / 32 * s.parts;
    p.top_each = p.k <= warps ? 1 : s.parts == 1 ? (p.k <= s.threads ? 1 : 0) : (3 * p.k + 2 * warps - 1) / (2 * warps);
    if (p.top_each > 24) p.top_each = 0;
    p.top_before = p.top_each ? (p.k + p.top_each - 1) / p.top_each - 1 : 0;
    switch (s.threads) {
    case 128: return launch_rows(token_logprob_top_kernel<T, 128, ENT>, p, E, s, true, 0, sms, stream);
    case 256: return launch_rows(token_logprob_top_kernel<T, 256, ENT>, p, E, s, true, 0, sms, stream);
    default: return launch_rows(token_logprob_top_kernel<T, 512, ENT>, p, E, s, true, 0, sms, stream);
    }
}

template <class T, int PASS, bool ENT>
cudaError_t logprob(VocabParams& p, int sms, cudaStream_t stream)
{
    constexpr int E = Elem<T>::E;
    const bool cluster = PASS != VOCAB_BWD;   // the backward's CTAs have nothing to exchange
    const Plan s = plan(p, E, PASS, !cluster, 32, sms);
    switch (s.threads) {
    case 32: return launch_rows(token_logprob_kernel<T, PASS, 32, ENT>, p, E, s, cluster, 0, sms, stream);
    case 128: return launch_rows(token_logprob_kernel<T, PASS, 128, ENT>, p, E, s, cluster, 0, sms, stream);
    case 256: return launch_rows(token_logprob_kernel<T, PASS, 256, ENT>, p, E, s, cluster, 0, sms, stream);
    default: return launch_rows(token_logprob_kernel<T, PASS, 512, ENT>, p, E, s, cluster, 0, sms, stream);
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
cudaError_t distill_rows(VocabParams& p, const Plan& s, int sms, cudaStream_t stream)
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
    return launch_rows(kern, p, E, s, true, smem, sms, stream);
}

template <class T, int PASS>
cudaError_t distill(VocabParams p, int sms, cudaStream_t stream)
{
    const Plan s = plan(p, Elem<T>::E, PASS, false, 32, sms);
    switch (s.threads) {
    case 32: return distill_rows<T, PASS, 32>(p, s, sms, stream);
    case 128: return distill_rows<T, PASS, 128>(p, s, sms, stream);
    case 256: return distill_rows<T, PASS, 256>(p, s, sms, stream);
    default: return distill_rows<T, PASS, 512>(p, s, sms, stream);
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
