// Kernels of the constraints on logits (constrain.cuh) and their launcher.
#include "constrain.cuh"

#include <algorithm>
#include <atomic>

#include "vocab_rows.cuh"

namespace cola {
namespace {

constexpr int THREADS = 256;
constexpr unsigned int SEEN = 1u << 31, BIASED = 1u << 30, POSITIVE = 1u << 29, COUNT = POSITIVE - 1;

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
__device__ __forceinline__ uint4 blend(const uint4& v, unsigned int banned)
{
    uint4 r = v;
    if constexpr (!BWD) {
        Elem<T>::ban(r, banned);
    } else {
        float x[Elem<T>::E];
        Elem<T>::unpack(v, x);
#pragma unroll
        for (int e = 0; e < Elem<T>::E; ++e)
            if (banned >> e & 1) x[e] = 0.f;
        r = Elem<T>::pack(x);
    }
    return r;
}

// A CTA has a share of a row's tokens: it counts those of the history that lie in
// it, copies the share with the masked logits replaced, then puts the logits of the
// tokens that were counted or biased over it.
template <class T, bool BWD>
__global__ void __launch_bounds__(THREADS) constrain_kernel(const ConstrainParams P)
{
    constexpr int E = Elem<T>::E;
    extern __shared__ __align__(16) unsigned int count[];   // of this CTA's tokens
    __shared__ int bias_at[BWD ? 1 : BIAS_MAX];
    __shared__ float bias[BWD ? 1 : BIAS_MAX];
    const long long i = blockIdx.x;
    const int tid = threadIdx.x;
    const T* logits = static_cast<const T*>(P.logits) + i * P.ld;
    const T* in = static_cast<const T*>(P.src) + i * P.ld_src;
    T* out = static_cast<T*>(P.dst) + i * P.ld_dst;
    const Row<T> row(in, P.vocab);
    const int v0 = min(static_cast<int>(blockIdx.y) * P.each, row.full), v1 = min(v0 + P.each, row.full);
    const bool last = blockIdx.y == gridDim.y - 1;
    const int begin = blockIdx.y == 0 ? 0 : row.head + v0 * E, end = last ? P.vocab : row.head + v1 * E;
    const int words = (end - begin + 3) / 4 * 4;
    for (int k = tid * 4; k < words; k += THREADS * 4) *reinterpret_cast<uint4*>(count + k) = make_uint4(0, 0, 0, 0);
    Mask mask{nullptr};
    if (P.masks) {
        const long long m = P.mask_of ? P.mask_of[i] : i;
        if (m >= 0 && m < P.n_masks) mask.words = P.masks + m * P.ld_masks;
    }
    __syncthreads();
    if (P.history) {
        const long long* h = P.history + i * P.ld_history;
        const long long n = min(max(P.history_len ? P.history_len[i] : P.history_width, 0ll), P.history_width);
        const long long prompt = P.prompt_len ? P.prompt_len[i] : 0;
        for (long long k = tid; k < n; k += THREADS) {
            const long long id = h[k];
            if (id < begin || id >= end) continue;
            unsigned int* c = count + (id - begin);
            if (BWD) {
                if (atomicOr(c, SEEN) == 0 && Elem<T>::get(logits + id) > 0.f) atomicOr(c, POSITIVE);
            } else if (k < prompt) {
                atomicOr(c, SEEN);
            } else {
                atomicAdd(c, 1u);
            }
        }
    }
    if constexpr (!BWD)
        for (int k = tid; k < P.n_bias; k += THREADS) {
            const long long id = P.bias_ids[i * P.n_bias + k];
            const bool here = id >= begin && id < end;
            bias_at[k] = here ? static_cast<int>(id) : -1;
            bias[k] = P.bias[i * P.n_bias + k];
            if (here) atomicOr(count + (id - begin), BIASED);
        }
    if (BWD) __syncthreads();   // (the result may lie over the logits, whose signs were read)
    // the copy
    const bool in_place = static_cast<const void*>(in) == static_cast<void*>(out);
    if (!in_place || mask.words) {
        const uint4* src = row.vec();
        T* dst = out + row.head;
        const bool same = ((reinterpret_cast<uintptr_t>(in) ^ reinterpret_cast<uintptr_t>(out)) & 15u) == 0;
        for (int v = v0 + (tid & ~31); v < v1; v += THREADS) {
            const int mine = v + (tid & 31);
            const bool there = mine < v1;
            unsigned int banned = 0;
            uint4 d = make_uint4(0, 0, 0, 0);
            if (there) {
                if (mask.words) banned = mask.template banned<E>(row.head + mine * E);
                if (banned != (1u << E) - 1) d = src[mine];
                if (banned) d = blend<T, BWD>(d, banned);
            }
            if (!same) store_apart(dst + mine * E, d, there);
            else if (there) reinterpret_cast<uint4*>(dst)[mine] = d;
        }
        for (int k = tid; k < row.edges(); k += THREADS) {
            const int id = row.edge(k);
            if (id < row.head ? blockIdx.y == 0 : last) out[id] = mask.allows(id) ? in[id] : T(BWD ? 0.f : NEG_INF);
        }
    }
    __syncthreads();
    // the tokens counted or biased
    const float r = P.repetition ? P.repetition[i] : 1.f;
    const float f = !BWD && P.frequency ? P.frequency[i] : 0.f, p = !BWD && P.presence ? P.presence[i] : 0.f;
    for (int k = tid; k < end - begin; k += THREADS) {
        const unsigned int c = count[k];
        const int id = begin + k;
        if (c == 0 || !mask.allows(id)) continue;
        if constexpr (BWD) {
            const float g = Elem<T>::get(in + id);
            Elem<T>::put(out + id, c & POSITIVE ? g / r : g * r);
        } else {
            float x = Elem<T>::get(logits + id);
            const unsigned int times = c & COUNT;
            if (c & ~BIASED) x = x > 0.f ? x / r : x * r;
            if (times) x = x - f * static_cast<float>(times) - p;
            if (c & BIASED) {
                float sum = 0.f;
                for (int e = 0; e < P.n_bias; ++e)
                    if (bias_at[e] == id) sum += bias[e];
                x += sum;
            }
            Elem<T>::put(out + id, x);
        }
    }
}

template <class T, bool BWD>
cudaError_t constrain(ConstrainParams p, int sms, cudaStream_t stream)
{
    constexpr int E = Elem<T>::E, MOST = 8192 / E;   // vectors of a CTA
    const int full = p.vocab / E;
    const long long wanted = std::min<long long>((4ll * sms + p.n - 1) / p.n, full / THREADS);
    const int parts = static_cast<int>(std::max<long long>(std::max<long long>(wanted, 1), (full + MOST - 1) / MOST));
    p.each = (full + parts - 1) / parts;
    const size_t smem = sizeof(unsigned int) * static_cast<size_t>(p.each * E + 2 * E + 4);
    auto kern = constrain_kernel<T, BWD>;
    kern<<<dim3(static_cast<unsigned int>(p.n), parts), THREADS, smem, stream>>>(p);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_constrain(const ConstrainParams& p, int dtype, bool backward, int sms, cudaStream_t stream)
{
    if (dtype == 0)
        return backward ? constrain<__nv_bfloat16, true>(p, sms, stream) : constrain<__nv_bfloat16, false>(p, sms, stream);
    return backward ? constrain<float, true>(p, sms, stream) : constrain<float, false>(p, sms, stream);
}

}  // namespace cola
