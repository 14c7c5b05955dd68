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

#include "ptx.cuh"

namespace cola {

constexpr int VOCAB_MAX = 1 << 20;      // tokens of a vocabulary
constexpr int VOCAB_MAX_K = 256;        // alternatives, entries of a teacher's list
enum { VOCAB_FWD = 0, VOCAB_STEP = 1, VOCAB_BWD = 2 };

struct VocabParams {
    const void* logits;
    void* dlogits;
    long long n, ld, ld_d;
    int vocab, k, rest;
    int parts;                // CTAs of a row
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

cudaError_t launch_token_logprob(const VocabParams& p, int dtype, int pass, int sms, cudaStream_t stream);
cudaError_t launch_topk_distill(const VocabParams& p, int dtype, int pass, int sms, cudaStream_t stream);

#ifdef COLA_DEFINE_VOCAB
constexpr int NV = 8;                   // 16-byte vectors a thread holds at once
constexpr int CLUSTER_MAX = 8;
constexpr int CAND_MAX = 1024;          // candidates for the top k kept on chip
constexpr float NEG_INF = -__builtin_huge_valf();
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
constexpr float FLOOR = -1e4f;          // an exponent of 2 whose power is 0
constexpr float NEAR = 1e6f;            // maxima, in powers of 2, whose rounding stays far below 1

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Maximum that a NaN wins; over a warp.
__device__ __forceinline__ float max_nan(float a, float b)
{
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}
__device__ __forceinline__ float max_nan_warp(float a)
{
    float y;
    asm volatile("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(a));
    return y;
}
__device__ __forceinline__ float sum_warp(float v)
{
#pragma unroll
    for (int i = 16; i; i >>= 1) v += __shfl_xor_sync(~0u, v, i);
    return v;
}

// Pairs of fp32 in one 64-bit register, for the two-lane arithmetic.
using Pair = unsigned long long;
__device__ __forceinline__ Pair pair(float lo, float hi)
{
    Pair r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void split(Pair p, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(p)); }
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c)
{
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ Pair add2(Pair a, Pair b)
{
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b)
{
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// ------------------------------------------------------------- element types
template <class T>
struct Elem;

template <>
struct Elem<float> {
    static constexpr int E = 4;
    static constexpr uint32_t FILL = 0xff800000u;   // -inf
    __device__ static float get(const float* p) { return *p; }
    __device__ static void put(float* p, float x) { *p = x; }
    __device__ __forceinline__ static void unpack(const uint4& u, float (&x)[4])
    {
        x[0] = __uint_as_float(u.x), x[1] = __uint_as_float(u.y), x[2] = __uint_as_float(u.z), x[3] = __uint_as_float(u.w);
    }
    __device__ __forceinline__ static uint4 pack(const float (&x)[4])
    {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
    __device__ __forceinline__ static float max_of(const uint4 (&d)[NV])
    {
        float m = NEG_INF;
#pragma unroll
        for (int j = 0; j < NV; ++j)
            m = max_nan(m, max_nan(max_nan(__uint_as_float(d[j].x), __uint_as_float(d[j].y)),
                                   max_nan(__uint_as_float(d[j].z), __uint_as_float(d[j].w))));
        return m;
    }
    // the elements whose bits are set := -inf
    __device__ __forceinline__ static void ban(uint4& u, uint32_t bits)
    {
        if (bits & 1) u.x = FILL;
        if (bits & 2) u.y = FILL;
        if (bits & 4) u.z = FILL;
        if (bits & 8) u.w = FILL;
    }
};

template <>
struct Elem<__nv_bfloat16> {
    static constexpr int E = 8;
    static constexpr uint32_t FILL = 0xff80ff80u;
    __device__ static float get(const __nv_bfloat16* p) { return __bfloat162float(*p); }
    __device__ static void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }
    __device__ __forceinline__ static void unpack(const uint4& u, float (&x)[8])
    {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    __device__ __forceinline__ static uint4 pack(const float (&x)[8])
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ __forceinline__ static uint32_t max_pair(uint32_t a, uint32_t b)
    {
        const __nv_bfloat162 r = __hmax2_nan(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
        return *reinterpret_cast<const uint32_t*>(&r);
    }
    __device__ __forceinline__ static float max_of(const uint4 (&d)[NV])
    {
        uint32_t m = FILL;
#pragma unroll
        for (int j = 0; j < NV; ++j) m = max_pair(m, max_pair(max_pair(d[j].x, d[j].y), max_pair(d[j].z, d[j].w)));
        return max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
    }
    __device__ __forceinline__ static void ban(uint4& u, uint32_t bits)
    {
        u.x = ban_pair(u.x, bits), u.y = ban_pair(u.y, bits >> 2), u.z = ban_pair(u.z, bits >> 4), u.w = ban_pair(u.w, bits >> 6);
    }
    __device__ __forceinline__ static uint32_t ban_pair(uint32_t w, uint32_t bits)
    {
        const uint32_t m = (bits & 1 ? 0x0000ffffu : 0u) | (bits & 2 ? 0xffff0000u : 0u);
        return (w & ~m) | (FILL & m);
    }
};

// ------------------------------------------------------------- rows in memory
// A row of `vocab` elements as 16-byte vectors at 16-byte boundaries: vector v
// holds elements v E - off .. v E - off + E - 1; those outside the row read as
// -inf and are never stored.  Pitch and base need the element's alignment only.
template <class T>
struct Row {
    static constexpr int E = Elem<T>::E;
    const T* p;
    int off, nvec, vocab;

    __device__ Row(const T* row, int v) : p(row), vocab(v)
    {
        off = static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T));
        nvec = (off + vocab + E - 1) / E;
    }
    __device__ __forceinline__ int first(int v) const { return v * E - off; }
    __device__ __forceinline__ uint4 load(int v) const
    {
        const int j = first(v);
        if (j >= 0 && j + E <= vocab) return *reinterpret_cast<const uint4*>(p + j);
        float x[E];
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = j + e >= 0 && j + e < vocab ? Elem<T>::get(p + j + e) : NEG_INF;
        return Elem<T>::pack(x);
    }
    // x into the same elements of `out`; `same`: out has this row's offset from a 16-byte boundary
    __device__ __forceinline__ void store(T* out, bool same, int v, const float (&x)[E]) const
    {
        const int j = first(v);
        if (same && j >= 0 && j + E <= vocab) {
            *reinterpret_cast<uint4*>(out + j) = Elem<T>::pack(x);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (j + e >= 0 && j + e < vocab) Elem<T>::put(out + j + e, x[e]);
        }
    }
};

// The GT threads that work on one row in one CTA: a warp (four rows a CTA) or
// the whole CTA, of `parts` that share the row as a cluster.
template <int GT>
struct Group {
    static constexpr int ROWS = GT == 32 ? 4 : 1, THREADS = GT * ROWS, W = GT / 32, TILE = GT * NV;
    static constexpr int CTAS = GT == 32 ? 6 : 1024 / THREADS;   // an SM's, for the registers a thread may have
    long long row;
    int rank, tid, lane, warp, slot;

    __device__ explicit Group(int parts)
    {
        tid = GT == 32 ? threadIdx.x & 31 : threadIdx.x;
        lane = threadIdx.x & 31;
        warp = tid >> 5;
        slot = GT == 32 ? threadIdx.x >> 5 : 0;
        row = GT == 32 ? blockIdx.x * 4ll + slot : blockIdx.x / static_cast<unsigned int>(parts);
        rank = GT == 32 ? 0 : blockIdx.x % static_cast<unsigned int>(parts);
    }
    __device__ __forceinline__ static void sync()
    {
        if (GT == 32) __syncwarp();
        else __syncthreads();
    }
};

// The vectors of one CTA of a row, in tiles of GT x NV.
template <class T, int GT>
struct Part {
    int begin, end, tiles;

    __device__ Part(const Row<T>& row, const Group<GT>& g, int parts)
    {
        const int each = (row.nvec + parts - 1) / parts;
        begin = min(g.rank * each, row.nvec);
        end = min(begin + each, row.nvec);
        tiles = (end - begin + Group<GT>::TILE - 1) / Group<GT>::TILE;
    }
    __device__ __forceinline__ int at(const Group<GT>& g, int tile, int j) const
    {
        return begin + tile * Group<GT>::TILE + j * GT + g.tid;
    }
    __device__ __forceinline__ void load(const Row<T>& row, const Group<GT>& g, int tile, uint4 (&d)[NV]) const
    {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int v = at(g, tile, j);
            d[j] = make_uint4(Elem<T>::FILL, Elem<T>::FILL, Elem<T>::FILL, Elem<T>::FILL);
            if (v < end) d[j] = row.load(v);
        }
    }
};

// ------------------------------------------------------------ thread clusters
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void st_cluster_f4(uint32_t addr, float4 v)
{
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
__device__ __forceinline__ void st_cluster_u64(uint32_t addr, unsigned long long v)
{
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(addr), "l"(v) : "memory");
}
__device__ __forceinline__ uint32_t add_cluster_u32(uint32_t addr, uint32_t v)
{
    uint32_t r;
    asm volatile("atom.shared::cluster.add.u32 %0, [%1], %2;" : "=r"(r) : "r"(addr), "r"(v) : "memory");
    return r;
}

// -------------------------------------------------------- softmax statistics
// m = max x, s = sum 2^y, t = sum 2^y y with y = c2 (x - m), in fp32.
// Nothing seen: m = -inf, s = t = 0.  A NaN, or +inf, makes s NaN.
struct Acc {
    float m, s, t;
};

__device__ __forceinline__ Acc acc_none() { return Acc{NEG_INF, 0.f, 0.f}; }

// Moves a's sums to a maximum m that is not below a's.  Differences are held
// above FLOOR: a sum times the distance from a mask of the type's lowest value
// would overflow where its weight is 0.
__device__ __forceinline__ Acc acc_to(const Acc& a, float m, float c2)
{
    const float d = a.s == 0.f ? 0.f : fmaxf((a.m - m) * c2, FLOOR), f = ex2(d);
    return Acc{m, a.s * f, f * (a.t + a.s * d)};
}

__device__ __forceinline__ Acc acc_merge(const Acc& a, const Acc& b, float c2)
{
    const float m = max_nan(a.m, b.m);
    const Acc x = acc_to(a, m, c2), y = acc_to(b, m, c2);
    return Acc{m, x.s + y.s, x.t + y.t};
}

__device__ __forceinline__ Acc acc_warp(const Acc& a, float c2)
{
    const float m = max_nan_warp(a.m);
    const Acc x = acc_to(a, m, c2);
    return Acc{m, sum_warp(x.s), sum_warp(x.t)};
}

// y = c2 x - b with b = c2 m rounded takes one fused operation per element and
// is exact but for its own rounding; that y is off from c2 (x - m) by the
// same delta = c2 m - b for all elements.
struct Base {
    float b, delta;
    __device__ __forceinline__ Base(float m, float c2) : b(m * c2), delta(fmaf(m, c2, -(m * c2))) {}
};

// The statistics of the elements of one tile that a thread holds; ENT: with t.
template <class T, bool ENT>
__device__ __forceinline__ Acc acc_tile(const uint4 (&d)[NV], float m, float c2)
{
    constexpr int E = Elem<T>::E;
    Acc a{m, 0.f, 0.f};
    if (m == NEG_INF) return a;
    if (fabsf(m * c2) < NEAR) {
        const Base base(m, c2);
        const Pair cc = pair(c2, c2), nb = pair(-base.b, -base.b);
        Pair s2[2] = {0, 0}, t2[2] = {0, 0};
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float x[E];
            Elem<T>::unpack(d[j], x);
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                float y0, y1;
                split(fma2(pair(x[e], x[e + 1]), cc, nb), y0, y1);
                const Pair w = pair(ex2(y0), ex2(y1));
                s2[e >> 1 & 1] = add2(s2[e >> 1 & 1], w);
                if (ENT) t2[e >> 1 & 1] = fma2(w, pair(fmaxf(y0, FLOOR), fmaxf(y1, FLOOR)), t2[e >> 1 & 1]);
            }
        }
        float lo, hi;
        split(add2(s2[0], s2[1]), lo, hi);
        const float s = lo + hi, f = ex2(-base.delta);
        a.s = s * f;
        if (ENT) {
            split(add2(t2[0], t2[1]), lo, hi);
            a.t = f * (lo + hi - base.delta * s);
        }
    } else {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float x[E];
            Elem<T>::unpack(d[j], x);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float y = (x[e] - m) * c2, w = ex2(y);
                a.s += w;
                a.t += w * fmaxf(y, FLOOR);
            }
        }
    }
    return a;
}

// The row's statistics in every thread, from those of each thread; slots: one
// per warp of each CTA of the row.
template <int GT>
__device__ __forceinline__ Acc acc_row(Acc a, float c2, const Group<GT>& g, int parts, float4* slots)
{
    a = acc_warp(a, c2);
    if (GT == 32) return a;
    const float4 mine = make_float4(a.m, a.s, a.t, 0.f);
    if (parts == 1) {
        if (g.lane == 0) slots[g.warp] = mine;
        __syncthreads();
    } else {
        cluster_wait();   // every CTA of the row runs
        if (g.lane < parts) st_cluster_f4(mapa_shared(smem_u32(slots + g.rank * Group<GT>::W + g.warp), g.lane), mine);
        cluster_sync();
    }
    a = acc_none();
    for (int i = g.lane; i < Group<GT>::W * parts; i += 32) {
        const float4 o = slots[i];
        a = acc_merge(a, Acc{o.x, o.y, o.z}, c2);
    }
    return acc_warp(a, c2);
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

constexpr int TOP_MAX_VALUES = VOCAB_MAX_K + CLUSTER_MAX * 16;

struct TopShared {
    unsigned long long key[CAND_MAX];
    uint32_t value[TOP_MAX_VALUES];     // the largest thread maxima of each warp
    unsigned int hist[256];
    unsigned int count, digit, above, bound;
};

// Gathers at least k and at most CAND_MAX keys of a row in memory, the k
// largest among them, by a radix search from the top digit that stops as soon
// as few enough are left: for rows whose largest tokens are not spread over the threads.
template <class T, int GT>
__device__ void top_radix(const Row<T>& row, int k, const Group<GT>& g, TopShared& sh)
{
    constexpr int E = Elem<T>::E;
    unsigned long long bound = 0;
    unsigned int taken = 0;              // keys above the digits found so far
    for (int shift = 56; shift >= 0; shift -= 8) {
        g.sync();
        for (int i = g.tid; i < 256; i += GT) sh.hist[i] = 0;
        g.sync();
        for (int v = g.tid; v < row.nvec; v += GT) {
            float x[E];
            Elem<T>::unpack(row.load(v), x);
            for (int e = 0; e < E; ++e) {
                const int j = row.first(v) + e;
                if (j < 0 || j >= row.vocab) continue;
                const unsigned long long key = token_key(x[e], j);
                if (shift == 56 || key >> (shift + 8) == bound >> (shift + 8))
                    atomicAdd(&sh.hist[key >> shift & 255u], 1u);
            }
        }
        g.sync();
        if (g.tid == 0) {
            unsigned int above = taken;
            int d = 255;
            while (d > 0 && above + sh.hist[d] < static_cast<unsigned int>(k)) above += sh.hist[d--];
            sh.digit = d;
            sh.above = above;
            sh.count = 0;
        }
        g.sync();
        taken = sh.above;
        bound |= static_cast<unsigned long long>(sh.digit) << shift;
        if (taken + sh.hist[sh.digit] <= CAND_MAX) break;
    }
    for (int v = g.tid; v < row.nvec; v += GT) {
        float x[E];
        Elem<T>::unpack(row.load(v), x);
        for (int e = 0; e < E; ++e) {
            const int j = row.first(v) + e;
            if (j < 0 || j >= row.vocab) continue;
            const unsigned long long key = token_key(x[e], j);
            if (key >= bound) sh.key[atomicAdd(&sh.count, 1u)] = key;
        }
    }
    g.sync();
}

// ------------------------------------------------- token log probabilities
template <class T, int PASS, int GT>
__global__ void __launch_bounds__(Group<GT>::THREADS, Group<GT>::CTAS) token_logprob_kernel(const VocabParams P)
{
    constexpr int E = Elem<T>::E;
    using G = Group<GT>;
    __shared__ float4 slots[PASS == VOCAB_BWD || GT == 32 ? 1 : CLUSTER_MAX * G::W];
    const G g(P.parts);
    if (GT == 32 && g.row >= P.n) return;
    const int parts = GT == 32 ? 1 : P.parts;
    const bool cluster = PASS != VOCAB_BWD && GT != 32 && parts > 1;
    if (cluster) cluster_arrive();
    const Row<T> row(static_cast<const T*>(P.logits) + g.row * P.ld, P.vocab);
    const Part<T, GT> part(row, g, parts);
    uint4 d[NV];
    part.load(row, g, 0, d);
    const long long y = P.targets ? P.targets[g.row] : -1;
    const bool there = y >= 0 && y < P.vocab;
    float up_g = 0.f, up_h = 0.f, xy = 0.f;
    if (PASS != VOCAB_FWD) {
        up_g = there && P.dlogp ? P.dlogp[g.row] : 0.f;
        up_h = P.dentropy ? P.dentropy[g.row] : 0.f;
    }
    float m, logs, H;
    if (PASS == VOCAB_BWD) {
        const float4 st = reinterpret_cast<const float4*>(P.stats)[g.row];
        m = st.x, logs = st.y, H = st.z;
    } else {
        if (P.logp && there && g.rank == 0 && g.tid == 0) xy = Elem<T>::get(row.p + y);
        const bool ent = P.entropy || P.stats || (PASS == VOCAB_STEP && P.dentropy);
        Acc a = acc_none();
        for (int t = 0; t < part.tiles; ++t) {
            if (t > 0) part.load(row, g, t, d);
            const float mt = Elem<T>::max_of(d);
            const Acc b = ent ? acc_tile<T, true>(d, mt, P.c2) : acc_tile<T, false>(d, mt, P.c2);
            a = t > 0 ? acc_merge(a, b, P.c2) : b;
        }
        a = acc_row(a, P.c2, g, parts, slots);
        m = a.m;
        logs = m == NEG_INF ? 0.f : logf(a.s);
        H = m == NEG_INF ? 0.f : logs - LN2 * (a.t / a.s);
    }
    const float m0 = m == NEG_INF ? 0.f : m;
    if (PASS != VOCAB_BWD && g.rank == 0 && g.tid == 0) {
        if (P.logp) P.logp[g.row] = there ? (xy - m0) * P.c - logs : 0.f;
        if (P.entropy) P.entropy[g.row] = H;
        if (PASS == VOCAB_FWD && P.stats) reinterpret_cast<float4*>(P.stats)[g.row] = make_float4(m, logs, H, 0.f);
    }
    if constexpr (PASS != VOCAB_FWD) {
        T* out = static_cast<T*>(P.dlogits) + g.row * P.ld_d;
        const bool same = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(row.p)) & 15u) == 0;
        const bool live = (up_g != 0.f || up_h != 0.f) && m != NEG_INF;
        const bool near = fabsf(m * P.c2) < NEAR;
        const Base base(m0, P.c2);
        const float scale = -P.c * ex2(-base.delta - logs * LOG2E);   // - c / s, to the base's power
        const float A = scale * (up_g + up_h * (H - logs - LN2 * base.delta)), B = scale * up_h * LN2;
        const Pair cc = pair(P.c2, P.c2), nb = pair(-base.b, -base.b), A2 = pair(A, A), B2 = pair(B, B);
        const int vy = there ? (static_cast<int>(y) + row.off) / E : -1, ey = (static_cast<int>(y) + row.off) % E;
        for (int t = part.tiles - 1; t >= 0; --t) {
            if (t < part.tiles - 1 || (PASS == VOCAB_BWD && t > 0)) part.load(row, g, t, d);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int v = part.at(g, t, j);
                if (v >= part.end) break;
                float x[E];
                Elem<T>::unpack(d[j], x);
                if (!live) {
#pragma unroll
                    for (int e = 0; e < E; ++e) x[e] = 0.f;
                } else if (near) {
#pragma unroll
                    for (int e = 0; e < E; e += 2) {
                        float y0, y1;
                        split(fma2(pair(x[e], x[e + 1]), cc, nb), y0, y1);
                        const Pair w = pair(ex2(y0), ex2(y1));
                        const Pair r = up_h == 0.f ? mul2(w, A2) : mul2(w, fma2(pair(fmaxf(y0, FLOOR), fmaxf(y1, FLOOR)), B2, A2));
                        split(r, x[e], x[e + 1]);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const float l = (x[e] - m0) * P.c - logs, p = ex2(l * LOG2E);
                        x[e] = -P.c * p * (up_g + up_h * (fmaxf(l, FLOOR) + H));
                    }
                }
                if (live && v == vy) {
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (e == ey) x[e] += P.c * up_g;
                }
                row.store(out, same, v, x);
            }
        }
    }
}

// The forward with the k most likely tokens.  A bound that at least k tokens
// reach is the k-th largest of thread maxima, of which each warp gives its
// `each` largest (each x warps >= k): one barrier more than the statistics.
// Tokens of this value and above (few more than k, when the largest are spread
// over the threads) are gathered from the registers, and ranked.
template <class T, int GT>
__global__ void __launch_bounds__(Group<GT>::THREADS, Group<GT>::CTAS) token_logprob_top_kernel(const VocabParams P)
{
    constexpr int E = Elem<T>::E;
    using G = Group<GT>;
    static_assert(GT > 32, "a warp's rows have no candidates list of their own");
    __shared__ float4 slots[CLUSTER_MAX * G::W];
    __shared__ TopShared top;
    const G g(P.parts);
    const bool cluster = P.parts > 1;
    if (g.tid == 0) top.count = 0;
    __syncwarp();
    if (cluster) cluster_arrive();   // this CTA runs, its count is set
    const Row<T> row(static_cast<const T*>(P.logits) + g.row * P.ld, P.vocab);
    const Part<T, GT> part(row, g, P.parts);
    uint4 d[NV];
    part.load(row, g, 0, d);
    const long long y = P.targets ? P.targets[g.row] : -1;
    const bool there = y >= 0 && y < P.vocab;
    float xy = 0.f;
    if (there && g.rank == 0 && g.tid == 0) xy = Elem<T>::get(row.p + y);
    const bool ent = P.entropy || P.stats;
    Acc a = acc_none();
    for (int t = 0; t < part.tiles; ++t) {
        if (t > 0) part.load(row, g, t, d);
        const float mt = Elem<T>::max_of(d);
        const Acc b = ent ? acc_tile<T, true>(d, mt, P.c2) : acc_tile<T, false>(d, mt, P.c2);
        a = t > 0 ? acc_merge(a, b, P.c2) : b;
    }
    const uint32_t mine = value_key(a.m);   // of this thread
    if (cluster) cluster_wait();
    // each warp's largest thread maxima, to every CTA of the row
    const int full = (row.nvec + P.parts - 1) / P.parts;
    const int warps = min(G::W, (full + 31) / 32) * P.parts;   // warps of the row that hold tokens
    const int each = (P.k + warps - 1) / warps;
    const int values = each * G::W * P.parts;
    const bool bounded = each <= 32 && values <= TOP_MAX_VALUES;
    if (bounded) {
        uint32_t left = mine;
        for (int i = 0; i < each; ++i) {
            const uint32_t best = __reduce_max_sync(~0u, left);
            const uint32_t at = (g.rank * G::W + g.warp) * each + i;
            if (!cluster) {
                if (g.lane == 0) top.value[at] = best;
            } else if (g.lane < P.parts) {
                st_shared_cluster_u32(mapa_shared(smem_u32(top.value + at), g.lane), best);
            }
            if (g.lane == __ffs(__ballot_sync(~0u, left == best)) - 1) left = 0;
        }
    }
    {
        a = acc_warp(a, P.c2);
        const float4 o = make_float4(a.m, a.s, a.t, 0.f);
        if (!cluster) {
            if (g.lane == 0) slots[g.warp] = o;
            __syncthreads();
        } else {
            if (g.lane < P.parts) st_cluster_f4(mapa_shared(smem_u32(slots + g.rank * G::W + g.warp), g.lane), o);
            cluster_sync();
        }
        a = acc_none();
        for (int i = g.lane; i < G::W * P.parts; i += 32) {
            const float4 s = slots[i];
            a = acc_merge(a, Acc{s.x, s.y, s.z}, P.c2);
        }
        a = acc_warp(a, P.c2);
    }
    const float m = a.m, m0 = m == NEG_INF ? 0.f : m;
    const float logs = m == NEG_INF ? 0.f : logf(a.s);
    const float H = m == NEG_INF ? 0.f : logs - LN2 * (a.t / a.s);
    if (g.rank == 0 && g.tid == 0) {
        if (P.logp) P.logp[g.row] = there ? (xy - m0) * P.c - logs : 0.f;
        if (P.entropy) P.entropy[g.row] = H;
        if (P.stats) reinterpret_cast<float4*>(P.stats)[g.row] = make_float4(m, logs, H, 0.f);
    }
    if (bounded) {
        // the k-th largest value: the one with k - 1 before it
        for (int i = g.warp; i < values; i += G::W) {
            const uint32_t v = top.value[i];
            unsigned int before = 0;
            for (int q = g.lane; q < values; q += 32) before += top.value[q] > v || (top.value[q] == v && q < i);
            if (__reduce_add_sync(~0u, before) == P.k - 1u && g.lane == 0) top.bound = v;
        }
        __syncthreads();
        const uint32_t bound = top.bound;
        const uint32_t count_at = cluster ? mapa_shared(smem_u32(&top.count), 0) : smem_u32(&top.count);
        const uint32_t key_at = cluster ? mapa_shared(smem_u32(top.key), 0) : smem_u32(top.key);
        if (mine >= bound) {
            const float limit = key_value(bound);
            for (int t = part.tiles - 1; t >= 0; --t) {
                if (t < part.tiles - 1) part.load(row, g, t, d);
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    float x[E];
                    Elem<T>::unpack(d[j], x);
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const int id = row.first(part.at(g, t, j)) + e;
                        // not below: a NaN is a candidate too
                        if (!(x[e] < limit) && part.at(g, t, j) < part.end && id >= 0 && id < row.vocab) {
                            const uint32_t at = cluster ? add_cluster_u32(count_at, 1) : atomicAdd(&top.count, 1u);
                            if (at < CAND_MAX) {
                                if (cluster) st_cluster_u64(key_at + 8 * at, token_key(x[e], id));
                                else top.key[at] = token_key(x[e], id);
                            }
                        }
                    }
                }
            }
        }
        if (cluster) cluster_sync();
        else __syncthreads();
    }
    if (g.rank != 0) return;
    if (!bounded || top.count > CAND_MAX) top_radix(row, P.k, g, top);
    const unsigned int count = top.count;
    for (unsigned int i = g.warp; i < count; i += G::W) {
        const unsigned long long key = top.key[i];
        unsigned int before = 0;
        for (unsigned int q = g.lane; q < count; q += 32) before += top.key[q] > key;
        before = __reduce_add_sync(~0u, before);
        if (before < P.k && g.lane == 0) {
            P.top_ids[g.row * P.k + before] = 0xffffffffu - static_cast<uint32_t>(key);
            P.top_logp[g.row * P.k + before] = (key_value(static_cast<uint32_t>(key >> 32)) - m0) * P.c - logs;
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

// A teacher's list, taken in by one warp of each CTA of the row.
struct ListShared {
    int id[VOCAB_MAX_K];
    float logq[VOCAB_MAX_K], q[VOCAB_MAX_K], x[VOCAB_MAX_K];   // x: the student's logit
    float m, s, Q;                                             // the student's statistics on the list, sum of q
};

// Bans the elements of a tile that are on the list: one word of bits per
// thread, a bit per element it holds, set by the warp that has the list.
template <class T, int GT>
__device__ __forceinline__ void ban_listed(const Row<T>& row, const Part<T, GT>& part, const Group<GT>& g, int tile, int k,
                                           const ListShared& list, unsigned long long* bits, uint4 (&d)[NV])
{
    constexpr int E = Elem<T>::E;
    bits[g.tid] = 0;
    g.sync();
    if (g.warp == 0) {
        for (int i = g.lane; i < k; i += 32) {
            const int at = list.id[i] + row.off, v = at / E - part.begin - tile * Group<GT>::TILE;
            if (list.id[i] >= 0 && v >= 0 && v < Group<GT>::TILE && at / E < part.end)
                atomicOr(bits + v % GT, 1ull << (v / GT * E + at % E));
        }
    }
    g.sync();
    const unsigned long long mine = bits[g.tid];
    if (mine) {
#pragma unroll
        for (int j = 0; j < NV; ++j) Elem<T>::ban(d[j], static_cast<uint32_t>(mine >> (j * E)));
    }
}

template <class T, int PASS, int GT>
__global__ void __launch_bounds__(Group<GT>::THREADS, Group<GT>::CTAS) topk_distill_kernel(const VocabParams P)
{
    constexpr int E = Elem<T>::E;
    using G = Group<GT>;
    __shared__ float4 slots[GT == 32 ? 1 : CLUSTER_MAX * G::W];
    __shared__ unsigned long long bits[G::THREADS];
    __shared__ ListShared lists[G::ROWS];
    const G g(P.parts);
    if (GT == 32 && g.row >= P.n) return;
    const int parts = GT == 32 ? 1 : P.parts;
    const bool cluster = GT != 32 && parts > 1;
    if (cluster) cluster_arrive();
    const Row<T> row(static_cast<const T*>(P.logits) + g.row * P.ld, P.vocab);
    const Part<T, GT> part(row, g, parts);
    ListShared& list = lists[g.slot];
    uint4 d[NV];
    part.load(row, g, 0, d);
    float m = 0.f, logs = 0.f, mr = 0.f, logr = 0.f;
    if (PASS == VOCAB_BWD) {
        const float4 st = reinterpret_cast<const float4*>(P.stats)[g.row];
        m = st.x, logs = st.y, mr = st.z, logr = st.w;
    }
    const float w = PASS != VOCAB_FWD ? P.dloss[g.row] : 0.f;
    if (g.warp == 0) {
        const float shift = P.rest && P.t_lse ? P.t_lse[g.row] : 0.f;
        float um = NEG_INF, xm = NEG_INF;
        for (int i = g.lane; i < P.k; i += 32) {
            const long long t = P.t_ids[g.row * P.k + i];
            const bool there = t >= 0 && t < P.vocab;
            const float u = there ? P.t_vals[g.row * P.k + i] * P.t_c - shift : NEG_INF;
            const float x = there ? Elem<T>::get(row.p + t) : NEG_INF;
            list.id[i] = there ? static_cast<int>(t) : -1;
            list.logq[i] = u;
            list.x[i] = x;
            um = max_nan(um, u);
            xm = max_nan(xm, x);
        }
        um = max_nan_warp(um);
        xm = max_nan_warp(xm);
        float logu = 0.f;
        if (!P.rest && um != NEG_INF) {
            float us = 0.f;
            for (int i = g.lane; i < P.k; i += 32) us += expf(list.logq[i] - um);
            logu = logf(sum_warp(us));
        }
        float Q = 0.f, xs = 0.f;
        for (int i = g.lane; i < P.k; i += 32) {
            const float lq = P.rest ? list.logq[i] : (list.logq[i] - (um == NEG_INF ? 0.f : um)) - logu;
            const float q = list.id[i] >= 0 ? expf(lq) : 0.f;
            list.logq[i] = lq;
            list.q[i] = q;
            Q += q;
            if (xm != NEG_INF) xs += ex2((list.x[i] - xm) * P.c2);
        }
        Q = sum_warp(Q);
        xs = sum_warp(xs);
        if (g.lane == 0) {
            list.m = xm;
            list.s = xs;
            list.Q = Q;
        }
    }
    float pl;   // the student's probability of the list
    if (PASS == VOCAB_BWD) {
        // in place: the list's logits are read before any CTA of the row stores
        if (cluster) {
            cluster_wait();
            cluster_sync();
        } else {
            g.sync();
        }
        pl = list.m == NEG_INF ? 0.f : list.s * ex2(((list.m - m) * P.c - logs) * LOG2E);
    } else {
        Acc a = acc_none();
        for (int t = 0; t < part.tiles; ++t) {
            if (t > 0) part.load(row, g, t, d);
            ban_listed(row, part, g, t, P.k, list, bits + g.slot * GT, d);
            const float mt = Elem<T>::max_of(d);
            const Acc b = acc_tile<T, false>(d, mt, P.c2);
            a = t > 0 ? acc_merge(a, b, P.c2) : b;
        }
        const Acc r = acc_row(a, P.c2, g, parts, slots);
        const Acc l{list.m, list.s, 0.f};
        a = acc_merge(l, r, P.c2);
        m = a.m, mr = r.m;
        logs = m == NEG_INF ? 0.f : logf(a.s);
        logr = mr == NEG_INF ? 0.f : logf(r.s);
        pl = acc_to(l, m, P.c2).s / a.s;
    }
    const float m0 = m == NEG_INF ? 0.f : m, mr0 = mr == NEG_INF ? 0.f : mr;
    const float logpr = (mr - m0) * P.c + logr - logs;
    const float Q = list.Q, qr = P.rest && mr != NEG_INF ? fmaxf(1.f - Q, 0.f) : 0.f;
    const bool entry = qr > 0.f;
    const float whole = entry ? 1.f : Q;
    if (PASS != VOCAB_BWD && g.rank == 0 && g.warp == 0) {
        float kl = 0.f;
        for (int i = g.lane; i < P.k; i += 32) {
            if (list.id[i] < 0) continue;
            const float q = list.q[i], logp = (list.x[i] - m0) * P.c - logs, r = list.logq[i] - logp;
            if (entry) kl += q > 0.f ? q * excess(r) : expf(logp);
            else kl += q > 0.f ? q * r : 0.f * q;
        }
        kl = sum_warp(kl);
        if (entry) kl += qr * excess(log1pf(-Q) - logpr);
        if (g.lane == 0) {
            P.loss[g.row] = P.temperature * P.temperature * kl;
            if (PASS == VOCAB_FWD && P.stats) reinterpret_cast<float4*>(P.stats)[g.row] = make_float4(m, logs, mr, logr);
        }
    }
    if constexpr (PASS != VOCAB_FWD) {
        T* out = static_cast<T*>(P.dlogits) + g.row * P.ld_d;
        const bool same = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(row.p)) & 15u) == 0;
        const float wt = w * P.temperature;
        const bool live = w != 0.f && m != NEG_INF;
        const bool near = fabsf(mr * P.c2) < NEAR;
        const Base base(mr0, P.c2);
        const float rate = wt * (entry ? Q - pl : Q * expf(logpr));
        const float A = mr == NEG_INF ? 0.f : rate * ex2(-base.delta - logr * LOG2E);
        const Pair cc = pair(P.c2, P.c2), nb = pair(-base.b, -base.b), A2 = pair(A, A);
        for (int t = part.tiles - 1; t >= 0; --t) {
            if (t < part.tiles - 1 || (PASS == VOCAB_BWD && t > 0)) part.load(row, g, t, d);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int v = part.at(g, t, j);
                if (v >= part.end) break;
                float x[E];
                Elem<T>::unpack(d[j], x);
                if (!live) {
#pragma unroll
                    for (int e = 0; e < E; ++e) x[e] = 0.f;
                } else if (near) {
#pragma unroll
                    for (int e = 0; e < E; e += 2) {
                        float y0, y1;
                        split(fma2(pair(x[e], x[e + 1]), cc, nb), y0, y1);
                        split(mul2(pair(ex2(y0), ex2(y1)), A2), x[e], x[e + 1]);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e) x[e] = mr == NEG_INF ? 0.f : rate * ex2(((x[e] - mr0) * P.c - logr) * LOG2E);
                }
                row.store(out, same, v, x);
            }
        }
        g.sync();
        if (g.warp == 0 && live) {
            for (int i = g.lane; i < P.k; i += 32) {
                const int id = list.id[i], v = (id + row.off) / E;
                if (id < 0 || v < part.begin || v >= part.end) continue;
                const float p = expf((list.x[i] - m0) * P.c - logs);
                Elem<T>::put(out + id, wt * (whole * p - list.q[i]));
            }
        }
    }
}
#endif

}  // namespace cola
