// vocab_plan.cuh -- how the rows of a vocabulary call are shared by threads
// and CTAs, and their launch.
#pragma once
#include <algorithm>
#include <cmath>

#include "vocab_rows.cuh"

namespace cola {

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
// thread); four too for a teacher's `list` beyond a warp's lanes, where the device
// runs all rows at once (7.2 us against 11.3 us for 86 rows of 552 and lists of 220,
// but 162 us against 86 us for 24727 of 672 and 138), and of many rows up to 4096
// vectors (2560 in a step, whose rows in flight L2 holds), tile after tile, so that the
// phases of eight rows overlap on an SM: 193 us against 229 us for a step of 32768 x
// 10000 bf16, 97 us against 122 us for a forward of 16384 x 20000; but 506 us against 463 us
// for a step of 32768 x 25000.  Longer rows, and few, take eight warps.
//   - A forward with the `top` k (0: without) takes sixteen where eight have too
//     few threads for its bound, and four where many rows of up to 4096 vectors
//     have enough of 128: much of its work is the same for every warp (116 us
//     against 129 us for the top 64 of 8192 x 32000, but 130 us against 105 us for
//     2048 x 128000).  A cluster's bound is looser than one CTA's, and long lists
//     ranked by one of its CTAs: up to 4096 vectors one CTA takes the top 65 and
//     more (8 to 12 us against 9 to 22 us for 44 x 13613, 18 against 14 for 1 x 128000).
//   - A step reads its row twice, the second time from L2: as many CTAs share a row
//     as keep the rows in flight within it, of sixteen warps where that would
//     take more than a portable cluster's eight CTAs.
//   - A backward without a list (`split`: its CTAs exchange nothing) takes a CTA per
//     tile.  (Sixteen warps leave short rows' threads idle, 211 us against 121 us for
//     16384 x 10000 bf16 with a list, and long ones gain nothing: 313 against 308 us
//     for 8192 x 65536.)
//   - All take more CTAs a row where there are few rows, to two CTAs of eight warps
//     per SM (one per SM, or as many as it can hold, took 0.3 to 1.5 us more),
//     down to a vector per thread.
// CTAs that form a cluster are a power of two: threes and sixes leave SMs empty
// (390 us on six, 332 us on four for a step of 2048 x 262144).
inline Plan plan(const VocabParams& p, int e, int pass, bool split, int top, int list, int sms)
{
    const int nvec = (p.vocab + e - 1) / e;
    if (nvec <= 32 * NV && (list <= 32 || p.n > 8ll * sms)) return {32, 1};
    if (nvec <= 128 * NV) return {128, 1};
    if (top == 0 && p.n >= 4ll * sms && nvec <= (pass == VOCAB_STEP ? 2560 : 4096)) return {128, 1};
    int threads = 256, hold = 1;
    if (pass == VOCAB_FWD) {
        if (top > 0 && top <= 64 && nvec <= 4096 && p.n >= 4ll * sms) return {128, 1};
        if (top > 128) threads = 512;
        if (top > 64 && nvec <= 4096) return {threads, 1};
    } else if (pass == VOCAB_STEP) {
        hold = static_cast<int>(std::ceil(4.0 * sms * 16.0 * nvec / STEP_L2_BYTES));
        if (hold > CLUSTER_MAX) threads = 512, hold = (hold + 1) / 2;
    } else if (split) {
        hold = (nvec + 256 * NV - 1) / (256 * NV);
    }
    const int fill = static_cast<int>(std::min<long long>(512ll * sms / threads / p.n, nvec / threads));
    if (split) return {threads, std::min(CLUSTER_MAX, std::max(hold, fill))};
    int parts = 1;
    while (parts < CLUSTER_MAX && (parts < hold || 2 * parts <= fill)) parts *= 2;
    return {threads, parts};
}

// Whether any row of the gradient lies otherwise on 16-byte boundaries than its logits.
inline bool lies_apart(const VocabParams& p, int e)
{
    return p.dlogits && (((reinterpret_cast<uintptr_t>(p.logits) - reinterpret_cast<uintptr_t>(p.dlogits)) & 15u) != 0 ||
                         (p.n > 1 && (p.ld - p.ld_d) % e != 0));
}

template <class K>
inline cudaError_t launch_rows(K kern, VocabParams& p, int e, const Plan& s, bool cluster, size_t smem, int sms,
                               cudaStream_t stream)
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

}  // namespace cola
