// Kernels of the constraints on logits (constrain.cuh) and their launcher.
#include "constrain.cuh"

#include <algorithm>
#include <atomic>

#include "vocab_rows.cuh"

namespace cola {
namespace {

constexpr int SMEM_MOST = 200 * 1024;

// A row's mask, the words of the CTA's tokens in shared memory.
struct Mask {
    const unsigned int* words;   // nullptr: everything is allowed
    int first;                   // the token of the first word's first bit
    __device__ __forceinline__ bool allows(int token) const { return !words || (words[(token - first) >> 5] >> ((token - first) & 31) & 1); }
    // of the E tokens from `token` on
    template <int E>
    __device__ __forceinline__ unsigned int banned(int token) const
    {
        const int w = (token - first) >> 5;
        return ~__funnelshift_r(words[w], words[w + 1], (token - first) & 31) & ((1u << E) - 1);
    }
};

template <class T, bool BWD>
__device__ __forceinline__ void ban(uint4& v, unsigned int banned)
{
    if constexpr (!BWD) {
        Elem<T>::ban(v, banned);
    } else if constexpr (sizeof(T) == 4) {
        if (banned & 1) v.x = 0;
        if (banned & 2) v.y = 0;
        if (banned & 4) v.z = 0;
        if (banned & 8) v.w = 0;
    } else {
        const auto keep = [](uint32_t bits) { return ~(((bits | bits << 15) & 0x00010001u) * 0xffffu); };
        v.x &= keep(banned), v.y &= keep(banned >> 2), v.z &= keep(banned >> 4), v.w &= keep(banned >> 6);
    }
}

// A CTA has a share of a row's tokens.  In one loop it copies them, masked logits replaced,
// and goes through the row's history: a bit of shared memory tells of each token whether the
// history names it, and those behind the prompt are counted (COUNTS: in 16 or 32 bits, where
// anything depends on it; 0: not).  Who sets a bit lists the token; or, LATE, those with a bit
// are listed after the loop, and on fewer than 1024 threads counted by their place there.  Then the listed and the biased tokens' results are stored over the copies:
// every token once, so that lanes are full and a result may lie over its input.  Counts do
// not depend on the order of the atomics, and a token's place in the list does not matter.
//
// The copy is bound by HBM, alone 79 us for 4096 x 32000 bf16 (524 MB); the rest by latency,
// a chain of the row's scalars, ids, atomics in shared memory and scattered logits.  With
// both, us: the gradient of 4096 x 32000 bf16 with histories of 1024 101 (0.92 of the copy
// rate of what it moves: a logit read for its sign costs 64 bytes), 256 x 128000 bf16 with
// histories of 4096 35, 32 x 50021 fp32 with 32768 16.0, 1 x 128000 with 2048 4.8.  Named
// tokens in hashed slots took 127, 51, 26 and 5.0 there, bits ranked by counting and
// passed between the CTAs of a cluster 121, 73, 32 and 6.4.  Four vectors a thread at once
// in a gradient, three in a forward: 101 against 107, 36.1 against 36.8.
template <class T, bool BWD, int COUNTS, int THREADS, bool LATE>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) constrain_kernel(const ConstrainParams P)
{
    constexpr int E = Elem<T>::E, U = BWD ? 4 : 3, IDS = 4, NAMES = 4, LOOKS = 4;
    constexpr bool RANKED = COUNTS && LATE && THREADS < 1024;
    // bits of the share's tokens (P.words each): named by the history, masked, biased or (a
    // gradient over the logits) of a positive logit, biased more than once; counts; biases;
    // the list
    extern __shared__ __align__(16) unsigned int seen[];
    __shared__ int listed, warp_sum[LATE ? THREADS / 32 : 1];
    const int n_bias = BWD ? 0 : P.n_bias;
    unsigned int *words = seen + P.words, *extra = words + P.words, *again = extra + P.words;
    unsigned int* counts = again + (n_bias ? P.words : 0);
    int* bias_ids = reinterpret_cast<int*>(counts + P.counts);
    float* bias = reinterpret_cast<float*>(bias_ids + n_bias);
    unsigned short* list = reinterpret_cast<unsigned short*>(bias + n_bias);
    unsigned short* base = list + P.list;
    const long long i = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const T* logits = static_cast<const T*>(P.logits) + i * P.ld;
    const T* in = static_cast<const T*>(P.src) + i * P.ld_src;
    T* out = static_cast<T*>(P.dst) + i * P.ld_dst;
    const Row<T> row(in, P.vocab);
    const int v0 = min(static_cast<int>(blockIdx.y) * P.each, row.full), v1 = min(v0 + P.each, row.full);
    const bool last = blockIdx.y == gridDim.y - 1;
    const int begin = blockIdx.y == 0 ? 0 : row.head + v0 * E, end = last ? P.vocab : row.head + v1 * E;
    const bool in_place = static_cast<const void*>(in) == static_cast<void*>(out);
    const bool same = ((reinterpret_cast<uintptr_t>(in) ^ reinterpret_cast<uintptr_t>(out)) & 15u) == 0;
    // the first ids on their way with what tells how many count
    const long long* h = P.history + i * P.ld_history;
    const int width = P.history ? static_cast<int>(P.history_width) : 0;
    long long id[IDS];
    const auto get_ids = [&](int k, int stop) {
#pragma unroll
        for (int j = 0; j < IDS; ++j) id[j] = k + j * THREADS < stop ? h[k + j * THREADS] : -1;
    };
    get_ids(tid, width);
    const long long length = !P.history ? 0 : P.history_len ? P.history_len[i] : P.history_width;
    const long long prompt = COUNTS && P.prompt_len ? P.prompt_len[i] : 0;
    const long long which = !P.masks ? -1 : P.mask_of ? P.mask_of[i] : i;
    const float r = P.repetition ? P.repetition[i] : 1.f;
    const float f = COUNTS && P.frequency ? P.frequency[i] : 0.f, p = COUNTS && P.presence ? P.presence[i] : 0.f;
    for (int k = tid; k < P.words; k += THREADS) {
        seen[k] = extra[k] = 0;
        if (n_bias) again[k] = 0;
    }
    if (COUNTS)
        for (int k = tid * 4; k < P.counts; k += THREADS * 4) *reinterpret_cast<uint4*>(counts + k) = make_uint4(0, 0, 0, 0);
    if (tid == 0) listed = 0;
    const int n = static_cast<int>(min(max(length, 0ll), static_cast<long long>(width)));
    const bool masked = which >= 0 && which < P.n_masks;
    if (masked) {
        const unsigned int* m = P.masks + which * P.ld_masks;
        for (int w = begin / 32 + tid; w < (end + 31) / 32; w += THREADS) words[w - begin / 32] = m[w];
    }
    const Mask mask{masked ? words : nullptr, begin / 32 * 32};
    __syncthreads();
    // an id's number in the share, -1 where it is not of the share
    const auto number = [&](long long t) {
        return static_cast<unsigned long long>(t - begin) < static_cast<unsigned long long>(end - begin) ? static_cast<int>(t - begin) : -1;
    };
    const auto get_bit = [](const unsigned int* bits, int t) { return bits[t >> 5] >> (t & 31) & 1; };
    const auto set_bit = [](unsigned int* bits, int t) { return atomicOr(bits + (t >> 5), 1u << (t & 31)) >> (t & 31) & 1; };
    const auto append = [&](int t) {   // (one atomic for all that get here together)
        const unsigned int together = __activemask(), first = __ffs(together) - 1;
        int at = 0;
        if (lane == static_cast<int>(first)) at = atomicAdd(&listed, __popc(together));
        at = __shfl_sync(together, at, first) + __popc(together & ((1u << lane) - 1));
        list[at] = static_cast<unsigned short>(t);
    };
    if constexpr (!BWD)
        for (int k = tid; k < n_bias; k += THREADS) {
            const int t = number(P.bias_ids[i * n_bias + k]);
            bias_ids[k] = t;
            bias[k] = P.bias[i * n_bias + k];
            if (t >= 0 && set_bit(extra, t)) set_bit(again, t);
        }
    const auto place = [&](int t) { return base[t >> 5] + __popc(seen[t >> 5] & ((1u << (t & 31)) - 1)); };   // (RANKED)
    const uint4* src = row.vec();
    T* dst = out + row.head;
    // (a gradient over the logits: first the names, then their logits' signs, then the copy)
    const bool over = BWD && P.over;
    for (int step = over ? 0 : 1; step < 2; ++step) {
        const int stop = step && (!in_place || masked) ? v1 : v0, ids = step && over ? 0 : n;
        int v = v0 + tid - lane;
        uint4 d[U];
        unsigned int banned[U];
        const auto load = [&] {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int at = v + u * THREADS + lane;
                banned[u] = 0;
                d[u] = make_uint4(0, 0, 0, 0);
                if (at >= stop) continue;
                if (masked) banned[u] = mask.template banned<E>(row.head + at * E);
                if (banned[u] != (1u << E) - 1 && (!in_place || banned[u])) d[u] = src[at];
            }
        };
        const auto store = [&] {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int at = v + u * THREADS + lane;
                if (v + u * THREADS >= stop) break;
                if (banned[u]) ban<T, BWD>(d[u], banned[u]);
                if (!same) store_apart(dst + at * E, d[u], at < stop);
                else if (at < stop && (!in_place || banned[u])) reinterpret_cast<uint4*>(dst)[at] = d[u];
            }
        };
        for (int k = tid; k - lane < ids; k += IDS * THREADS) {
            int here[IDS];
#pragma unroll
            for (int j = 0; j < IDS; ++j) here[j] = k + j * THREADS < n ? number(id[j]) : -1;
            get_ids(k + IDS * THREADS, n);
            if (v < stop) load();
#pragma unroll
            for (int j = 0; j < IDS; ++j) {
                const int t = here[j];
                if (t < 0) continue;
                if (COUNTS && !RANKED && k + j * THREADS >= prompt) {
                    if (COUNTS == 16) atomicAdd(counts + (t >> 1), 1u << (t & 1) * 16);
                    else atomicAdd(counts + t, 1u);
                }
                if (!get_bit(seen, t) && !set_bit(seen, t) && !LATE) append(t);
            }
            __syncwarp();
            if (v < stop) store();
            v += U * THREADS;
        }
        for (; v < stop; v += U * THREADS) {
            load();
            store();
        }
        if (step == 1) break;
        __syncthreads();
        for (int k = tid; k < end - begin; k += THREADS)
            if (get_bit(seen, k) && Elem<T>::get(logits + begin + k) > 0.f) set_bit(extra, k);
        __syncthreads();
    }
    for (int k = tid; k < row.edges(); k += THREADS) {
        const int t = row.edge(k);
        if (t < row.head ? blockIdx.y != 0 : !last) continue;
        if (!mask.allows(t)) Elem<T>::put(out + t, BWD ? 0.f : NEG_INF);
        else if (!in_place) out[t] = in[t];
    }
    __syncthreads();
    if constexpr (LATE) {
        // every thread has every THREADS-th word of bits: frequent tokens' ids lie together
        const int used = (end - begin + 31) / 32;
        int sum = 0;
        for (int w = tid; w < used; w += THREADS) sum += __popc(seen[w]);
        int up = sum;
#pragma unroll
        for (int k = 1; k < 32; k <<= 1) {
            const int v = __shfl_up_sync(~0u, up, k);
            if (lane >= k) up += v;
        }
        if (lane == 31) warp_sum[warp] = up;
        __syncthreads();
        const int sums = lane < THREADS / 32 ? warp_sum[lane] : 0, all = __reduce_add_sync(~0u, sums);
        int at = __reduce_add_sync(~0u, lane < warp ? sums : 0) + up - sum;
        for (int w = tid; w < used; w += THREADS) {
            if (RANKED) base[w] = static_cast<unsigned short>(at);
            for (unsigned int bits = seen[w]; bits; bits &= bits - 1) list[at++] = static_cast<unsigned short>(w * 32 + __ffs(bits) - 1);
        }
        if (tid == 0) listed = all;
        __syncthreads();
        if constexpr (RANKED) {
            constexpr int MORE = 8;
            for (int k = tid; k < n; k += MORE * THREADS) {
                long long more[MORE];
#pragma unroll
                for (int j = 0; j < MORE; ++j) more[j] = k + j * THREADS < n && k + j * THREADS >= prompt ? h[k + j * THREADS] : -1;
#pragma unroll
                for (int j = 0; j < MORE; ++j) {
                    const int t = number(more[j]);
                    if (t < 0) continue;
                    const int at = place(t);
                    atomicAdd(counts + (at >> 1), 1u << (at & 1) * 16);
                }
            }
            __syncthreads();
        }
    }
    // x of a named token with the penalties; at: where its count is
    const auto penalized = [&](float x, int at) {
        float y = x > 0.f ? x / r : x * r;
        if (COUNTS) {
            const unsigned int times = COUNTS == 16 ? counts[at >> 1] >> (at & 1) * 16 & 0xffffu : counts[at];
            if (times) y = y - f * static_cast<float>(times) - p;
        }
        return y;
    };
    const int names = listed;
    // (a thread's first biased token, its logit on its way with the listed ones; few of each
    // are on different warps)
    const int k0 = THREADS - 32 - warp * 32;
    const auto biased = [&](int k) { return k < n_bias && bias_ids[k] >= 0 && mask.allows(begin + bias_ids[k]) ? bias_ids[k] : -1; };
    const int t0 = biased(k0 + lane);
    const float x0 = t0 >= 0 ? Elem<T>::get(logits + begin + t0) : 0.f;
    for (int k = tid; k < names; k += NAMES * THREADS) {
        int token[NAMES];
        float x[NAMES], g[NAMES];
#pragma unroll
        for (int j = 0; j < NAMES; ++j) {
            const int t = k + j * THREADS < names ? list[k + j * THREADS] : -1;
            token[j] = t >= 0 && mask.allows(begin + t) && !(n_bias && get_bit(extra, t)) ? t : -1;
            if (token[j] < 0) continue;
            if (!over) x[j] = Elem<T>::get(logits + begin + t);
            if (BWD) g[j] = Elem<T>::get(in + begin + t);
        }
#pragma unroll
        for (int j = 0; j < NAMES; ++j) {
            const int t = token[j];
            if (t < 0) continue;
            float y;
            if constexpr (BWD) y = (over ? get_bit(extra, t) != 0 : x[j] > 0.f) ? g[j] / r : g[j] * r;
            else y = penalized(x[j], RANKED ? k + j * THREADS : t);
            Elem<T>::put(out + begin + t, y);
        }
    }
    if constexpr (BWD) return;
    // The biased tokens, each by the first of its entries; for each of few that have several a
    // warp looks through all, of many (small vocabularies) every thread for its own.  20 of one
    // row 4.8 us, 300 of 256 x 128000 with histories of 4096 39 (57 where every listed token
    // looked for its bias), 1000 of 64 rows 17 (every thread for its own: 36), 300 of 25 x 386
    // 13 (by warps: 40).
    for (int k = k0; k < n_bias; k += THREADS) {
        const int t = biased(k + lane);
        float x = x0, sum = 0.f;
        if (t >= 0) {
            if (k != k0) x = Elem<T>::get(logits + begin + t);
            sum = bias[k + lane];
        }
        bool stored = t < 0;   // or will be by another
        unsigned int several = __ballot_sync(~0u, t >= 0 && get_bit(again, t));
        if (__popc(several) > 6) {
            if (several >> lane & 1) {
                int found = k + lane;
                sum = 0.f;
#pragma unroll 4
                for (int e = 0; e < n_bias; ++e)
                    if (bias_ids[e] == t) sum += bias[e], found = min(found, e);
                stored = found < k + lane;
            }
            several = 0;
        }
        for (; several; several &= several - 1) {
            const int of = __ffs(several) - 1, token = __shfl_sync(~0u, t, of);
            float all = 0.f;
            bool first = true;
            for (int e = lane; e - lane < n_bias && first; e += 32 * LOOKS) {
                unsigned int entries[LOOKS];
                float b[LOOKS];
#pragma unroll
                for (int u = 0; u < LOOKS; ++u) {
                    const bool same = e + u * 32 < n_bias && bias_ids[e + u * 32] == token;
                    b[u] = same ? bias[e + u * 32] : 0.f;
                    entries[u] = __ballot_sync(~0u, same);
                }
#pragma unroll
                for (int u = 0; u < LOOKS; ++u) {
                    if (entries[u]) first = first && e - lane + u * 32 + __ffs(entries[u]) - 1 >= k + of;
                    for (unsigned int left = entries[u]; left; left &= left - 1) all += __shfl_sync(~0u, b[u], __ffs(left) - 1);
                }
            }
            if (lane == of) sum = all, stored = !first;
        }
        if (stored) continue;
        const float y = get_bit(seen, t) ? penalized(x, RANKED ? place(t) : t) : x;
        Elem<T>::put(out + begin + t, y + sum);
    }
}

template <class T, bool BWD, int COUNTS, int THREADS, bool LATE>
cudaError_t constrain(const ConstrainParams& p, int parts, size_t smem, cudaStream_t stream)
{
    auto kern = constrain_kernel<T, BWD, COUNTS, THREADS, LATE>;
    static std::atomic<unsigned long long> configured{0};   // bit d: set on device d
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !((configured.load(std::memory_order_acquire) >> dev) & 1ull)) {
        e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_MOST);
        if (e != cudaSuccess) return e;
        if (dev < 64) configured.fetch_or(1ull << dev, std::memory_order_acq_rel);
    }
    kern<<<dim3(static_cast<unsigned int>(p.n), parts), THREADS, smem, stream>>>(p);
    return cudaGetLastError();
}

// CTAs of a row.  Every CTA of a row reads all of its history, and its bits, list and counts
// limit what one holds.
//   - Many rows: CTAs of 256 threads, as many as run at once, four an SM (with counts, bf16,
//     histories of 4096: 64 x 128000 13.9 us, twice as many 19.6, 256 x 50021 fp32 26.4 and
//     29.4), of 32768 tokens at most: 256 x 128000 takes four a row, which is 1.7 waves, 36.4
//     us; two a row of 64000 tokens 39.3 (512 rows 71 and 68).  Without counts, where rows
//     leave no more than one each, two times as many: the gradient of 509 x 50021 fp32 51 us
//     against 53; of 256 x 128000 bf16 30 against 34.
//   - Many rows of longer histories, with counts up to 16384: 512 threads, two an SM, of up
//     to 65024 tokens (histories of 8192: 256 x 128000 bf16 41 us against 55 on 1024 threads,
//     its gradient 38 against 54; 64 rows 15.4 against 15.9, 32 rows 13.4 against 10.6; 16384:
//     256 rows 58 against 65; 32768: 51 against 49 for 128 rows, but gradients of 512 x 32000
//     59 against 63).  256 and 512 threads are even at 2000 to 2600 ids (fp32, gradients
//     of 1024 rows and more), at 5000 to 6000 (64, 1024 and 4096 rows of bf16).  At 4096, us: 64 x
//     128000 13.2 and 14.1, 1024 x 32000 47 and 47, but their gradients 12.1 and 12.4, 50 and 39.
//   - Few rows, and other histories beyond 4096 ids: 1024 threads, an SM each, and a vector
//     for every sixteenth id at least (1 x 128000: 4.8 us against 6.0 on 256 threads).  Of
//     long histories the list is made after the loop: 15 us against 22 for 32 x 50021 and 32768
//     ids, but 5.4 against 4.8 for 1 x 128000 and 2048, 114 against 101 for the gradient of
//     4096 x 32000 and 1024.
// Counts on fewer than 1024 threads are one per listed token, on 1024 one per token: the
// list's places are known after the loop alone, and finding them reads the history again
// (32768 ids too many for few CTAs), but 16 bits a token leave room for three CTAs an SM: 64
// x 128000 18 us against 14, 256 x 128000 39.6 against 36, 512 x 128000 87 against 71.
template <class T, bool BWD, int COUNTS>
cudaError_t constrain_plan(ConstrainParams p, int sms, cudaStream_t stream)
{
    constexpr int E = Elem<T>::E;
    const int full = p.vocab / E;
    const long long width = p.history ? p.history_width : 0;
    const bool many = 2 * p.n > sms && (!COUNTS || width <= 16384);
    const int threads = 8 * p.n <= sms ? 1024 : width <= 4096 ? 256 : many ? 512 : 1024;
    const int most = COUNTS == 32 ? 16384 : threads == 512 ? 65024 : 32768;   // tokens of a CTA (their numbers have 16 bits)
    const long long once = 1024 / threads * static_cast<long long>(sms) / p.n;   // CTAs of a row, of those that run at once
    const long long fill = threads > 256 || COUNTS || once > 1 ? once : (8ll * sms + p.n - 1) / p.n;
    const long long wanted = std::min<long long>(fill, full / std::max<long long>(threads == 1024 ? 64 : 256, width / 16));
    const int parts = static_cast<int>(std::max({wanted, static_cast<long long>((p.vocab + most - 1) / most), 1ll}));
    p.each = (full + parts - 1) / parts;
    const int tokens = p.each * E + 2 * E;
    p.words = (tokens / 32 + 3 + 3) / 4 * 4;   // (one more than a mask's, which is read in pairs)
    p.list = static_cast<int>(std::min<long long>(tokens, width));
    const bool ranked = COUNTS && threads < 1024;
    p.counts = COUNTS ? ((ranked ? p.list : tokens) / (32 / COUNTS) + 4) / 4 * 4 : 0;
    p.over = BWD && p.logits == p.dst && p.logits != p.src;
    const size_t smem = 4 * static_cast<size_t>((p.n_bias ? 4 : 3) * p.words + p.counts + 2 * p.n_bias) +
                        2 * static_cast<size_t>(p.list + (ranked ? p.words : 0));
    if constexpr (COUNTS == 32) {   // (histories of 65536 ids and more)
        return constrain<T, BWD, COUNTS, 1024, true>(p, parts, smem, stream);
    } else {
        if (threads == 512) return constrain<T, BWD, COUNTS, 512, true>(p, parts, smem, stream);
        if (threads == 256) return constrain<T, BWD, COUNTS, 256, COUNTS != 0>(p, parts, smem, stream);
        return width > 4096 ? constrain<T, BWD, COUNTS, 1024, true>(p, parts, smem, stream)
                            : constrain<T, BWD, COUNTS, 1024, false>(p, parts, smem, stream);
    }
}

template <class T>
cudaError_t constrain_counts(const ConstrainParams& p, bool backward, int sms, cudaStream_t stream)
{
    if (backward) return constrain_plan<T, true, 0>(p, sms, stream);
    if (!p.history || !(p.frequency || p.presence)) return constrain_plan<T, false, 0>(p, sms, stream);
    return p.history_width < 65536 ? constrain_plan<T, false, 16>(p, sms, stream) : constrain_plan<T, false, 32>(p, sms, stream);
}

}  // namespace

cudaError_t launch_constrain(const ConstrainParams& p, int dtype, bool backward, int sms, cudaStream_t stream)
{
    return dtype == 0 ? constrain_counts<__nv_bfloat16>(p, backward, sms, stream) : constrain_counts<float>(p, backward, sms, stream);
}

}  // namespace cola
