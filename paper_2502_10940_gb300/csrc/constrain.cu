// Kernels of the constraints on logits (constrain.cuh) and their launcher.
#include "constrain.cuh"

#include <algorithm>
#include <atomic>

#include "vocab_rows.cuh"

namespace cola {
namespace {

// of a token that the history or the biases name: flags above its count
constexpr unsigned int SEEN = 1u << 31, BIASED = 1u << 30, COUNT = BIASED - 1;
constexpr int MOST_TOKENS = 24576;            // of a CTA
constexpr int SMEM_MOST = 200 * 1024;

struct Mask {
    const unsigned int* words;   // nullptr: everything is allowed
    __device__ __forceinline__ bool allows(int token) const { return !words || (words[token >> 5] >> (token & 31) & 1); }
    // of the E tokens from `token` on, which all lie in the row
    template <int E>
    __device__ __forceinline__ unsigned int banned(int token) const
    {
        const int w = token >> 5, s = token & 31;
        const unsigned int lo = words[w], hi = s + E > 32 ? words[w + 1] : 0;
        return ~__funnelshift_r(lo, hi, s) & ((1u << E) - 1);
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

// A CTA has a share of a row's tokens.  In one loop
//   - it counts those of them that the row's history and biases name, each in a slot of its
//     own in shared memory: one per token of the share, or, where the history may name few
//     of the share, slots found by a hash of the id.  Whoever finds a slot empty lists it.
//   - it copies the share, masked logits replaced: neither waits for the other.
// Then the listed tokens' results are stored over the copies.  The counts do not depend on
// the order of the atomics, and a listed token's place in the list does not matter.
template <class T, bool BWD, int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) constrain_kernel(const ConstrainParams P)
{
    constexpr int E = Elem<T>::E, U = 4, IDS = 4;
    extern __shared__ __align__(16) unsigned int count[];   // P.slots of them, P.room of the list, P.slots of keys (hashed)
    __shared__ int bias_ids[BWD ? 1 : BIAS_MAX];
    __shared__ float bias[BWD ? 1 : BIAS_MAX];
    __shared__ unsigned int listed;
    unsigned int *list = count + P.slots, *keys = list + P.room;
    const long long i = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 31;
    const long long* h = P.history + i * P.ld_history;
    const long long length = !P.history ? 0 : P.history_len ? P.history_len[i] : P.history_width;
    const long long prompt = P.prompt_len ? P.prompt_len[i] : 0;
    const long long which = !P.masks ? -1 : P.mask_of ? P.mask_of[i] : i;
    const T* logits = static_cast<const T*>(P.logits) + i * P.ld;
    const T* in = static_cast<const T*>(P.src) + i * P.ld_src;
    T* out = static_cast<T*>(P.dst) + i * P.ld_dst;
    const Row<T> row(in, P.vocab);
    const int v0 = min(static_cast<int>(blockIdx.y) * P.each, row.full), v1 = min(v0 + P.each, row.full);
    const bool last = blockIdx.y == gridDim.y - 1;
    const int begin = blockIdx.y == 0 ? 0 : row.head + v0 * E, end = last ? P.vocab : row.head + v1 * E;
    const bool in_place = static_cast<const void*>(in) == static_cast<void*>(out);
    const bool same = ((reinterpret_cast<uintptr_t>(in) ^ reinterpret_cast<uintptr_t>(out)) & 15u) == 0;
    const uint4* src = row.vec();
    T* dst = out + row.head;
    for (int k = tid; k < P.slots; k += THREADS) count[k] = 0;
    if (P.hashed)
        for (int k = tid; k < P.slots; k += THREADS) keys[k] = 0;
    if (tid == 0) listed = 0;
    const int n = static_cast<int>(min(max(length, 0ll), P.history_width));
    const Mask mask{which >= 0 && which < P.n_masks ? P.masks + which * P.ld_masks : nullptr};
    __syncthreads();
    const auto name = [&](long long id, unsigned int flag) {   // flag 0: counted
        if (id < begin || id >= end) return;
        unsigned int slot = static_cast<unsigned int>(id - begin);
        if (P.hashed) {
            const unsigned int key = slot + 1;
            slot = __umulhi(key * 2654435769u, P.slots);
            for (unsigned int old; (old = atomicCAS(keys + slot, 0u, key)) != 0 && old != key;)
                if (++slot == static_cast<unsigned int>(P.slots)) slot = 0;   // (more slots than names: there is one)
        }
        if ((flag ? atomicOr(count + slot, flag) : atomicAdd(count + slot, 1u)) == 0) list[atomicAdd(&listed, 1u)] = slot;
    };
    if constexpr (!BWD)
        for (int k = tid; k < P.n_bias; k += THREADS) {
            const long long id = P.bias_ids[i * P.n_bias + k];
            bias_ids[k] = id >= begin && id < end ? static_cast<int>(id) : -1;
            bias[k] = P.bias[i * P.n_bias + k];
            name(id, BIASED);
        }
    // (a gradient over the logits: their signs are read before they are gone)
    const bool over = BWD && !in_place && static_cast<const void*>(logits) == static_cast<void*>(out);
    const int stop = (!in_place || mask.words) && !over ? v1 : v0;
    const auto copy = [&](int from, int to, bool ids) {
        for (int v = from + tid - lane, k = tid; v < to || (ids && k - lane < n); v += U * THREADS, k += IDS * THREADS) {
            long long id[IDS];
            uint4 d[U];
            unsigned int banned[U];
#pragma unroll
            for (int j = 0; j < IDS; ++j) id[j] = ids && k + j * THREADS < n ? h[k + j * THREADS] : -1;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int at = v + u * THREADS + lane;
                banned[u] = 0;
                d[u] = make_uint4(0, 0, 0, 0);
                if (at >= to) continue;
                if (mask.words) banned[u] = mask.template banned<E>(row.head + at * E);
                if (banned[u] != (1u << E) - 1 && (!in_place || banned[u])) d[u] = src[at];
            }
#pragma unroll
            for (int j = 0; j < IDS; ++j) name(id[j], BWD || k + j * THREADS < prompt ? SEEN : 0);
            __syncwarp();
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int at = v + u * THREADS + lane;
                if (v + u * THREADS >= to) break;
                if (banned[u]) ban<T, BWD>(d[u], banned[u]);
                if (!same) store_apart(dst + at * E, d[u], at < to);
                else if (at < to && (!in_place || banned[u])) reinterpret_cast<uint4*>(dst)[at] = d[u];
            }
        }
    };
    const auto copy_edges = [&] {
        for (int k = tid; k < row.edges(); k += THREADS) {
            const int id = row.edge(k);
            if (id < row.head ? blockIdx.y != 0 : !last) continue;
            if (!mask.allows(id)) Elem<T>::put(out + id, BWD ? 0.f : NEG_INF);
            else if (!in_place) out[id] = in[id];
        }
    };
    copy(v0, stop, true);
    if (!over) copy_edges();
    __syncthreads();
    const int names = listed;
    const float r = P.repetition ? P.repetition[i] : 1.f;
    const float f = !BWD && P.frequency ? P.frequency[i] : 0.f, p = !BWD && P.presence ? P.presence[i] : 0.f;
    const auto token_of = [&](unsigned int slot) { return begin + static_cast<int>(P.hashed ? keys[slot] - 1 : slot); };
    const auto result = [&](unsigned int slot, int token) -> float {
        const unsigned int c = count[slot], times = c & COUNT;
        float x = Elem<T>::get(logits + token);
        if constexpr (BWD) {
            const float g = Elem<T>::get(in + token);
            return x > 0.f ? g / r : g * r;
        }
        if (c & ~BIASED) x = x > 0.f ? x / r : x * r;
        if (times) x = x - f * static_cast<float>(times) - p;
        if (c & BIASED) {
            float sum = 0.f;
            for (int e = 0; e < P.n_bias; ++e)
                if (bias_ids[e] == token) sum += bias[e];
            x += sum;
        }
        return x;
    };
    if (over) {
        for (int k = tid; k < names; k += THREADS) count[list[k]] = __float_as_uint(result(list[k], token_of(list[k])));
        __syncthreads();
        copy(v0, v1, false);
        copy_edges();
        __syncthreads();
    }
#pragma unroll 2
    for (int k = tid; k < names; k += THREADS) {
        const unsigned int slot = list[k];
        const int token = token_of(slot);
        if (!mask.allows(token)) continue;
        Elem<T>::put(out + token, over ? __uint_as_float(count[slot]) : result(slot, token));
    }
}

template <class T, bool BWD, int THREADS>
cudaError_t constrain(ConstrainParams& p, int parts, cudaStream_t stream)
{
    constexpr int E = Elem<T>::E;
    const int full = p.vocab / E;
    p.each = (full + parts - 1) / parts;
    const long long tokens = p.each * E + 2 * E, names = (p.history ? p.history_width : 0) + p.n_bias;
    p.room = static_cast<int>(std::min(tokens, names));
    p.hashed = names + names / 2 < tokens;
    p.slots = static_cast<int>(p.hashed ? names + names / 2 + 1 : p.room ? tokens : 0);
    const size_t smem = sizeof(unsigned int) * ((p.hashed ? 2 : 1) * p.slots + p.room);
    auto kern = constrain_kernel<T, BWD, THREADS>;
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

// Many rows: CTAs of 256 threads and up to 32768 tokens, eight an SM if there are as many.
// Few: more CTAs a row, to a vector per thread; but every CTA of a row reads all of its
// history, so that a CTA has a sixteenth as many vectors as the history has ids at least.
template <class T, bool BWD>
cudaError_t constrain_plan(ConstrainParams p, int sms, cudaStream_t stream)
{
    constexpr int E = Elem<T>::E;
    const int full = p.vocab / E;
    const long long width = p.history ? p.history_width : 0;
    const long long wanted = std::min<long long>((8ll * sms + p.n - 1) / p.n, full / std::max(256ll, width / 16));
    // (shared memory: 12 bytes for each token at most, or 16 for each name)
    const long long least = (full * static_cast<long long>(E) + MOST_TOKENS - 1) / MOST_TOKENS;
    const int parts = static_cast<int>(std::max({wanted, least, 1ll}));
    if (width > 16 * 256 && p.n * parts <= 2ll * sms) return constrain<T, BWD, 1024>(p, parts, stream);
    return constrain<T, BWD, 256>(p, parts, stream);
}

}  // namespace

cudaError_t launch_constrain(const ConstrainParams& p, int dtype, bool backward, int sms, cudaStream_t stream)
{
    using bf16 = __nv_bfloat16;
    if (dtype == 0) return backward ? constrain_plan<bf16, true>(p, sms, stream) : constrain_plan<bf16, false>(p, sms, stream);
    return backward ? constrain_plan<float, true>(p, sms, stream) : constrain_plan<float, false>(p, sms, stream);
}

}  // namespace cola
