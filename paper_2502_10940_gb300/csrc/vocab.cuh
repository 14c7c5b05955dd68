// vocab.cuh -- kernels over rows of vocabulary logits: log probabilities of
// given tokens with the row's entropy and most likely tokens, the distillation
// loss against a teacher's most likely tokens, and the gradients of both.
//
// Mathematics (row x of V logits, temperature T, c = 1 / T):
//   m = max x,  s = sum exp(c (x - m)),  logp_j = c (x_j - m) - log s,  p = exp(logp)
//   H = log s - c sum p_j (x_j - m)                     (both terms >= 0: nothing cancels)
//   d(g logp_y + h H)/dx_j = c (g [j = y] - p_j (g + h (logp_j + H)))
// Distillation: with q over the teacher's list, R the tokens outside it and
// (m_R, s_R) their own maximum and sum,
//   p_R = exp(c (m_R - m)) s_R / s                      (not 1 - sum p: no cancellation)
//   dx_j = w T rate exp(c (x_j - m_R)) / s_R  for j in R,   w T (Q p_k - q_k) on the list,
//   rate = sum q - sum p (rest counted) or Q p_R, Q = 1 or sum q.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

namespace cola {

constexpr int VOCAB_MAX = 1 << 20;      // tokens of a vocabulary
constexpr int VOCAB_MAX_K = 256;        // alternatives, entries of a teacher's list
enum { VOCAB_FWD = 0, VOCAB_STEP = 1, VOCAB_BWD = 2 };

struct VocabParams {
    const void* logits;
    void* dlogits;
    long long n, ld, ld_d;
    int vocab, k, rest;
    float temperature;
    float c;                  // 1 / temperature
    float c2;                 // log2(e) / temperature
    float* stats;             // n x 4, written by the forward, read by the backward
    // token log probabilities
    const long long* targets;
    float* logp;
    float* entropy;
    long long* top_ids;
    float* top_logp;
    const float* dlogp;
    const float* dentropy;
    // distillation
    const long long* t_ids;
    const float* t_vals;
    const float* t_lse;
    float t_c;                // 1 / the teacher's temperature
    const float* dloss;
    float* loss;
};

cudaError_t launch_token_logprob(const VocabParams& p, int dtype, int pass, cudaStream_t stream);
cudaError_t launch_topk_distill(const VocabParams& p, int dtype, int pass, cudaStream_t stream);

#ifdef COLA_DEFINE_VOCAB
constexpr int VT = 512;                 // threads of a CTA
constexpr int VW = VT / 32;
constexpr int CAND_MAX = 1024;          // candidates for the top k kept on chip
constexpr float NEG_INF = -__builtin_huge_valf();
constexpr float LOG2E = 1.4426950408889634f;
constexpr float FLOOR = -1e20f;         // below any difference of finite logits that exp does not flush to 0

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Maximum that a NaN wins.
__device__ __forceinline__ float max_nan(float a, float b)
{
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}

// ------------------------------------------------------------- rows in memory
// A row of `vocab` elements as 16-byte vectors at 16-byte boundaries: vector v
// holds elements v E - off .. v E - off + E - 1; those outside the row read as
// -inf and are never stored.  Pitch and base need the element's alignment only.
template <class T>
struct Row {
    static constexpr int E = 16 / sizeof(T);
    T* p;
    int off, nvec, vocab;

    __device__ Row(T* row, int v) : p(row), vocab(v)
    {
        off = static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T));
        nvec = (off + vocab + E - 1) / E;
    }
    __device__ __forceinline__ int first(int v) const { return v * E - off; }
    __device__ __forceinline__ void load(int v, float (&x)[E]) const;
    __device__ __forceinline__ void store(int v, const float (&x)[E]) const;
};

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_float(float* p, float x) { *p = x; }
__device__ __forceinline__ void from_float(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

__device__ __forceinline__ void unpack(const uint4& u, float (&x)[4])
{
    x[0] = __uint_as_float(u.x), x[1] = __uint_as_float(u.y), x[2] = __uint_as_float(u.z), x[3] = __uint_as_float(u.w);
}
__device__ __forceinline__ void unpack(const uint4& u, float (&x)[8])
{
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint4 pack(const float (&x)[4])
{
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}
__device__ __forceinline__ uint4 pack(const float (&x)[8])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <class T>
__device__ __forceinline__ void Row<T>::load(int v, float (&x)[E]) const
{
    const int j = first(v);
    if (j >= 0 && j + E <= vocab) {
        unpack(*reinterpret_cast<const uint4*>(p + j), x);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = j + e >= 0 && j + e < vocab ? to_float(p[j + e]) : NEG_INF;
    }
}

// The elements of vector v of a row whose off is that of the row x was loaded
// from, or any other: then element by element.
template <class T>
__device__ __forceinline__ void store_row(const Row<T>& in, T* out, bool same, int v, const float (&x)[Row<T>::E])
{
    constexpr int E = Row<T>::E;
    const int j = in.first(v);
    if (same && j >= 0 && j + E <= in.vocab) {
        *reinterpret_cast<uint4*>(out + j) = pack(x);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (j + e >= 0 && j + e < in.vocab) from_float(out + j + e, x[e]);
    }
}

// -------------------------------------------------------- softmax statistics
// m = max x, s = sum 2^(c2 (x - m)), t = sum 2^(c2 (x - m)) (x - m), in fp32.
// Nothing seen: m = -inf, s = t = 0.  A NaN, or +inf, makes s NaN.
struct Acc {
    float m, s, t;
};

__device__ __forceinline__ Acc acc_none() { return Acc{NEG_INF, 0.f, 0.f}; }

__device__ __forceinline__ Acc acc_merge(const Acc& a, const Acc& b, float c2)
{
    Acc r;
    r.m = max_nan(a.m, b.m);
    // differences are clamped: a sum times the distance from a mask of the
    // type's lowest value would overflow where its weight is 0
    const float da = a.s == 0.f ? 0.f : fmaxf(a.m - r.m, FLOOR), fa = ex2(da * c2);
    const float db = b.s == 0.f ? 0.f : fmaxf(b.m - r.m, FLOOR), fb = ex2(db * c2);
    r.s = a.s * fa + b.s * fb;
    r.t = fa * (a.t + a.s * da) + fb * (b.t + b.s * db);
    return r;
}

template <int N>
__device__ __forceinline__ void acc_add(Acc& a, const float (&x)[N], float c2)
{
    float m = a.m;
#pragma unroll
    for (int e = 0; e < N; ++e) m = max_nan(m, x[e]);
    if (m == NEG_INF) return;
    Acc b{m, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const float d = x[e] - m, w = ex2(d * c2);
        b.s += w;
        b.t += w * fmaxf(d, FLOOR);
    }
    a = acc_merge(a, b, c2);
}

__device__ __forceinline__ Acc acc_shfl(const Acc& a, int mask)
{
    return Acc{__shfl_xor_sync(~0u, a.m, mask), __shfl_xor_sync(~0u, a.s, mask), __shfl_xor_sync(~0u, a.t, mask)};
}

__device__ __forceinline__ Acc acc_warp(Acc a, float c2)
{
#pragma unroll
    for (int i = 16; i; i >>= 1) {
        const Acc b = acc_shfl(a, i);
        a = threadIdx.x & i ? acc_merge(b, a, c2) : acc_merge(a, b, c2);   // the same order in both lanes
    }
    return a;
}

// Every thread gets the whole CTA's; `buf` may be used again after the next barrier.
__device__ __forceinline__ Acc acc_block(Acc a, float c2, Acc* buf)
{
    a = acc_warp(a, c2);
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = a;
    __syncthreads();
    Acc r = buf[0];
    for (int w = 1; w < VW; ++w) r = acc_merge(r, buf[w], c2);
    return r;
}

__device__ __forceinline__ float sum_block(float v, float* buf)
{
#pragma unroll
    for (int i = 16; i; i >>= 1) v += __shfl_xor_sync(~0u, v, i);
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    float r = 0.f;
    for (int w = 0; w < VW; ++w) r += buf[w];
    return r;
}

__device__ __forceinline__ float max_block(float v, float* buf)
{
#pragma unroll
    for (int i = 16; i; i >>= 1) v = max_nan(v, __shfl_xor_sync(~0u, v, i));
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    float r = NEG_INF;
    for (int w = 0; w < VW; ++w) r = max_nan(r, buf[w]);
    return r;
}

// --------------------------------------------------------------- top k of a row
// Order of tokens as a whole number: the logit first (NaN above +inf, -0 equal
// to 0), then the lower id.  All keys of a row differ.
__device__ __forceinline__ uint32_t value_key(float x)
{
    if (x != x) return 0xffffffffu;
    const uint32_t b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k)
{
    return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);   // 0xffffffff: a NaN
}
__device__ __forceinline__ unsigned long long token_key(float x, int j)
{
    return static_cast<unsigned long long>(value_key(x)) << 32 | (0xffffffffu - static_cast<uint32_t>(j));
}

struct TopShared {
    unsigned long long key[CAND_MAX];
    unsigned int hist[256];
    unsigned int count, digit, above;
};

// Gathers at least k and at most CAND_MAX keys, the k largest among them, by a
// radix search from the top digit that stops as soon as few enough are left.
template <class T>
__device__ void top_gather(const Row<const T>& row, int k, TopShared& sh)
{
    constexpr int E = Row<const T>::E;
    unsigned long long bound = 0;
    unsigned int taken = 0;              // keys above the digits found so far
    for (int shift = 56; shift >= 0; shift -= 8) {
        if (threadIdx.x < 256) sh.hist[threadIdx.x] = 0;
        __syncthreads();
        for (int v = threadIdx.x; v < row.nvec; v += VT) {
            float x[E];
            row.load(v, x);
            for (int e = 0; e < E; ++e) {
                const int j = row.first(v) + e;
                if (j < 0 || j >= row.vocab) continue;
                const unsigned long long key = token_key(x[e], j);
                if (shift == 56 || key >> (shift + 8) == bound >> (shift + 8))
                    atomicAdd(&sh.hist[key >> shift & 255u], 1u);
            }
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            unsigned int above = taken;
            int d = 255;
            while (d > 0 && above + sh.hist[d] < static_cast<unsigned int>(k)) above += sh.hist[d--];
            sh.digit = d;
            sh.above = above;
            sh.count = 0;
        }
        __syncthreads();
        taken = sh.above;
        bound |= static_cast<unsigned long long>(sh.digit) << shift;
        if (taken + sh.hist[sh.digit] <= CAND_MAX) break;
        __syncthreads();
    }
    for (int v = threadIdx.x; v < row.nvec; v += VT) {
        float x[E];
        row.load(v, x);
        for (int e = 0; e < E; ++e) {
            const int j = row.first(v) + e;
            if (j < 0 || j >= row.vocab) continue;
            const unsigned long long key = token_key(x[e], j);
            if (key >= bound) sh.key[atomicAdd(&sh.count, 1u)] = key;
        }
    }
    __syncthreads();
}

// ------------------------------------------------- token log probabilities
template <class T, int PASS>
__global__ void __launch_bounds__(VT) token_logprob_kernel(const VocabParams P)
{
    constexpr int E = Row<const T>::E;
    __shared__ Acc accs[VW];
    __shared__ TopShared top;
    const long long i = blockIdx.x;
    const Row<const T> row(static_cast<const T*>(P.logits) + i * P.ld, P.vocab);
    float m, logs, H;
    if (PASS == VOCAB_BWD) {
        const float4 st = reinterpret_cast<const float4*>(P.stats)[i];
        m = st.x, logs = st.y, H = st.z;
    } else {
        Acc a = acc_none();
        for (int v = threadIdx.x; v < row.nvec; v += VT) {
            float x[E];
            row.load(v, x);
            acc_add(a, x, P.c2);
        }
        a = acc_block(a, P.c2, accs);
        m = a.m;
        logs = m == NEG_INF ? 0.f : logf(a.s);
        H = m == NEG_INF ? 0.f : logs - P.c * (a.t / a.s);
    }
    const float m0 = m == NEG_INF ? 0.f : m;
    const long long y = P.targets ? P.targets[i] : -1;
    const bool there = y >= 0 && y < P.vocab;
    if (PASS != VOCAB_BWD && threadIdx.x == 0) {
        if (P.logp) P.logp[i] = there ? (to_float(row.p[y]) - m0) * P.c - logs : 0.f;
        if (P.entropy) P.entropy[i] = H;
        if (PASS == VOCAB_FWD && P.stats) reinterpret_cast<float4*>(P.stats)[i] = make_float4(m, logs, H, 0.f);
    }
    if (PASS == VOCAB_FWD && P.k > 0) {
        top_gather(row, P.k, top);
        for (unsigned int a = threadIdx.x; a < top.count; a += VT) {
            const unsigned long long key = top.key[a];
            int rank = 0;
            for (unsigned int b = 0; b < top.count; ++b) rank += top.key[b] > key;
            if (rank < P.k) {
                P.top_ids[i * P.k + rank] = 0xffffffffu - static_cast<uint32_t>(key);
                P.top_logp[i * P.k + rank] = (key_value(static_cast<uint32_t>(key >> 32)) - m0) * P.c - logs;
            }
        }
    }
    if (PASS != VOCAB_FWD) {
        T* out = static_cast<T*>(P.dlogits) + i * P.ld_d;
        const bool same = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(row.p)) & 15u) == 0;
        const float g = there && P.dlogp ? P.dlogp[i] : 0.f, h = P.dentropy ? P.dentropy[i] : 0.f;
        const bool live = (g != 0.f || h != 0.f) && m != NEG_INF;
        if (PASS == VOCAB_STEP) __syncthreads();   // in place: logp_y is read before the row is written over
        for (int v = threadIdx.x; v < row.nvec; v += VT) {
            float x[E] = {};
            if (live) {
                row.load(v, x);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float l = (x[e] - m0) * P.c - logs, p = ex2(l * LOG2E);
                    x[e] = -P.c * p * (g + h * (fmaxf(l, FLOOR) + H));
                    if (row.first(v) + e == y) x[e] += P.c * g;
                }
            }
            store_row(Row<T>(const_cast<T*>(row.p), P.vocab), out, same, v, x);
        }
    }
}

// ------------------------------------------------------------- distillation
// r + exp(-r) - 1 >= 0.  Where q and p both sum to 1, KL(q || p) is the sum of
// q excess(log q / p): a sum of nonnegative terms, exact to a few ulp where
// that of q log(q / p) cancels.
__device__ __forceinline__ float excess(float r)
{
    if (fabsf(r) < 0.3f)
        return r * r * (0.5f - r * (1.f / 6 - r * (1.f / 24 - r * (1.f / 120 - r * (1.f / 720 - r / 5040)))));
    return r + expm1f(-r);
}

template <class T, int PASS>
__global__ void __launch_bounds__(VT) topk_distill_kernel(const VocabParams P)
{
    constexpr int E = Row<const T>::E;
    extern __shared__ uint32_t listed[];   // one bit per element: on the teacher's list
    __shared__ Acc accs[2 * VW];
    __shared__ float sums[4 * VW];
    const long long i = blockIdx.x;
    const Row<const T> row(static_cast<const T*>(P.logits) + i * P.ld, P.vocab);
    for (int w = threadIdx.x; w < (row.nvec * E + 31) / 32; w += VT) listed[w] = 0;
    __syncthreads();
    // one thread per entry of the list: the teacher's probability, the student's logit
    int id = -1;
    float u = NEG_INF, xk = NEG_INF;
    if (threadIdx.x < P.k) {
        const long long t = P.t_ids[i * P.k + threadIdx.x];
        if (t >= 0 && t < P.vocab) {
            id = static_cast<int>(t);
            atomicOr(&listed[(id + row.off) >> 5], 1u << ((id + row.off) & 31));
            xk = to_float(row.p[id]);
            u = P.t_vals[i * P.k + threadIdx.x] * P.t_c - (P.rest && P.t_lse ? P.t_lse[i] : 0.f);
        }
    }
    float logq = u;
    if (!P.rest) {
        const float um = max_block(u, sums);
        const float um0 = um == NEG_INF ? 0.f : um;
        const float us = sum_block(expf(u - um0), sums + VW);
        logq = (u - um0) - (um == NEG_INF ? 0.f : logf(us));
    }
    const float q = id >= 0 ? expf(logq) : 0.f;
    const float Qs = sum_block(q, sums + 2 * VW);   // also the barrier after the list's bits
    float m, logs, mr, logr;
    if (PASS == VOCAB_BWD) {
        const float4 st = reinterpret_cast<const float4*>(P.stats)[i];
        m = st.x, logs = st.y, mr = st.z, logr = st.w;
    } else {
        Acc a = acc_none();
        for (int v = threadIdx.x; v < row.nvec; v += VT) {
            float x[E];
            row.load(v, x);
            const uint32_t bits = listed[v * E >> 5] >> (v * E & 31);
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (bits >> e & 1u) x[e] = NEG_INF;
            acc_add(a, x, P.c2);
        }
        const Acc r = acc_block(a, P.c2, accs);
        a = acc_none();
        if (id >= 0) {
            const float x1[1] = {xk};
            acc_add(a, x1, P.c2);
        }
        a = acc_merge(acc_block(a, P.c2, accs + VW), r, P.c2);
        m = a.m, mr = r.m;
        logs = m == NEG_INF ? 0.f : logf(a.s);
        logr = mr == NEG_INF ? 0.f : logf(r.s);
    }
    const float m0 = m == NEG_INF ? 0.f : m, mr0 = mr == NEG_INF ? 0.f : mr;
    const float logp = (xk - m0) * P.c - logs, p = id >= 0 ? expf(logp) : 0.f;
    const float logpr = (mr - m0) * P.c + logr - logs;
    const float qr = P.rest && mr != NEG_INF ? fmaxf(1.f - Qs, 0.f) : 0.f;
    const bool entry = qr > 0.f;
    if (PASS != VOCAB_BWD) {
        float term = 0.f;
        if (id >= 0) {
            if (entry) term = q > 0.f ? q * excess(logq - logp) : p;
            else term = q > 0.f ? q * (logq - logp) : 0.f * q;
        }
        float kl = sum_block(term, sums);
        if (entry) kl += qr * excess(log1pf(-Qs) - logpr);
        if (threadIdx.x == 0) {
            P.loss[i] = P.temperature * P.temperature * kl;
            if (PASS == VOCAB_FWD && P.stats) reinterpret_cast<float4*>(P.stats)[i] = make_float4(m, logs, mr, logr);
        }
    }
    if (PASS != VOCAB_FWD) {
        T* out = static_cast<T*>(P.dlogits) + i * P.ld_d;
        const bool same = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(row.p)) & 15u) == 0;
        const float w = P.dloss[i] * P.temperature;
        const bool live = P.dloss[i] != 0.f && m != NEG_INF;
        const float drop = sum_block(q - p, sums + VW);
        const float coef = w * (entry ? drop : Qs * expf(logpr));
        for (int v = threadIdx.x; v < row.nvec; v += VT) {
            float x[E] = {};
            if (live) {
                row.load(v, x);
#pragma unroll
                for (int e = 0; e < E; ++e) x[e] = mr == NEG_INF ? 0.f : coef * ex2(((x[e] - mr0) * P.c - logr) * LOG2E);
            }
            store_row(Row<T>(const_cast<T*>(row.p), P.vocab), out, same, v, x);
        }
        __syncthreads();
        if (live && id >= 0) from_float(out + id, w * ((entry ? 1.f : Qs) * p - q));
    }
}
#endif

}  // namespace cola
