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
    int ahead;                // rows from one CTA to the next in its place
    int each;                 // 16-byte vectors of a row per CTA (the grid's y: CTAs of a row)
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
    int top_each, top_before; // of each warp's largest, the one it gives; how many of those lie before the bound (each 0: no bound)
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

__device__ __forceinline__ float rcp(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
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
    using Bits = unsigned int;                       // one per element of NV vectors
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
    // a bit for each element that reaches `limit` (or is NaN), and the place of a bit's element in its tile
    static constexpr float LOWEST = -3.402823466e38f;
    __device__ __forceinline__ static unsigned long long reach(const uint4 (&d)[NV], float limit)
    {
        unsigned int bits = 0;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float x[4];
            unpack(d[j], x);
#pragma unroll
            for (int e = 0; e < 4; ++e) bits |= x[e] < limit ? 0u : 1u << (j * 4 + e);
        }
        return bits;
    }
    __device__ __forceinline__ static int place(int bit) { return bit; }
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
    using Bits = unsigned long long;
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
    // as above; a word's two elements compared at once, the bits of words 0..15 and 16..31 in
    // halves: low elements, then high ones
    static constexpr float LOWEST = -3.38953139e38f;
    __device__ __forceinline__ static unsigned long long reach(const uint4 (&d)[NV], float limit)
    {
        const __nv_bfloat162 l = __float2bfloat162_rn(limit);   // exact: an element's value
        uint32_t bits[2] = {0, 0};
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const uint32_t w[4] = {d[j].x, d[j].y, d[j].z, d[j].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t below = __hlt2_mask(*reinterpret_cast<const __nv_bfloat162*>(&w[i]), l);
                bits[j / 4] |= ~below & (0x00010001u << (j % 4 * 4 + i));
            }
        }
        return static_cast<unsigned long long>(bits[1]) << 32 | bits[0];
    }
    __device__ __forceinline__ static int place(int bit) { return (bit >> 5) * 32 + (bit & 15) * 2 + (bit >> 4 & 1); }
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
        const uint32_t m = ((bits | bits << 15) & 0x00010001u) * 0xffffu;
        return (w & ~m) | (FILL & m);
    }
};

__device__ __forceinline__ void prefetch_l2_bulk(const void* p, int bytes)
{
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p), "r"(bytes) : "memory");
}

// ------------------------------------------------------------- rows in memory
// A row of `vocab` elements: the 16-byte vectors at 16-byte boundaries, and up
// to E - 1 single elements before and after them (its edges).  Pitch and base
// need the element's alignment only.
template <class T>
struct Row {
    static constexpr int E = Elem<T>::E;
    const T* p;
    int vocab, head, full, tail;   // elements before the vectors, vectors, elements after them

    __device__ Row(const T* row, int v) : p(row), vocab(v)
    {
        const int over = static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T));
        head = min((E - over) % E, v);
        full = (v - head) / E;
        tail = v - head - full * E;
    }
    __device__ __forceinline__ int edges() const { return head + tail; }
    __device__ __forceinline__ int edge(int i) const { return i < head ? i : vocab - tail + i - head; }
    __device__ __forceinline__ const uint4* vec() const { return reinterpret_cast<const uint4*>(p + head); }
};

// The GT threads that work on one row in one CTA: a warp (four rows a CTA) or
// the whole CTA; the row's CTAs lie along the grid's y, and form a cluster
// where they exchange anything.
template <int GT>
struct Group {
    static constexpr int ROWS = GT == 32 ? 4 : 1, THREADS = GT * ROWS, W = GT / 32, TILE = GT * NV;
    static constexpr int CTAS = GT == 32 ? 6 : 1024 / THREADS;   // an SM's, for the registers a thread may have
    long long row;
    int rank, parts, tid, lane, warp, slot;

    __device__ Group()
    {
        tid = GT == 32 ? threadIdx.x & 31 : threadIdx.x;
        lane = threadIdx.x & 31;
        warp = tid >> 5;
        slot = GT == 32 ? threadIdx.x >> 5 : 0;
        row = GT == 32 ? blockIdx.x * 4ll + slot : blockIdx.x;
        rank = GT == 32 ? 0 : blockIdx.y;
        parts = GT == 32 ? 1 : gridDim.y;
    }
    __device__ __forceinline__ static void sync()
    {
        if (GT == 32) __syncwarp();
        else __syncthreads();
    }
    // the one warp that has the row's edges, an element per lane
    __device__ __forceinline__ bool has_edges() const { return rank == 0 && warp == W - 1; }
};

// The vectors of one CTA of a row, in tiles of GT x NV.
template <class T, int GT>
struct Part {
    int begin, end, tiles;

    __device__ Part(const Row<T>& row, const Group<GT>& g, int each)
    {
        begin = min(g.rank * each, row.full);
        end = min(begin + each, row.full);
        tiles = (end - begin + Group<GT>::TILE - 1) / Group<GT>::TILE;
    }
    // this thread's first vector of a tile; vector j lies GT j after it and is there where left > GT j
    __device__ __forceinline__ int at(const Group<GT>& g, int tile) const { return begin + tile * Group<GT>::TILE + g.tid; }
    __device__ __forceinline__ int left(const Group<GT>& g, int tile) const { return end - at(g, tile); }
    // vectors of a tile that any thread holds
    __device__ __forceinline__ int used(int tile) const { return (end - begin - tile * Group<GT>::TILE + GT - 1) / GT; }
    // LAST: for the last time (streaming stores and these leave L2 to rows still to be read again)
    template <bool LAST = false>
    __device__ __forceinline__ void load(const Row<T>& row, const Group<GT>& g, int tile, uint4 (&d)[NV]) const
    {
        const uint4* q = row.vec() + at(g, tile);
        const int n = left(g, tile);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            d[j] = make_uint4(Elem<T>::FILL, Elem<T>::FILL, Elem<T>::FILL, Elem<T>::FILL);
            if (n > j * GT) d[j] = LAST ? __ldcs(q + j * GT) : q[j * GT];
        }
    }
    // the tiles after the first on their way to L2, ahead of the loads
    __device__ __forceinline__ void prefetch(const Row<T>& row, const Group<GT>& g) const
    {
        const int from = begin + Group<GT>::TILE;
        if (g.tid == 0 && from < end) prefetch_l2_bulk(row.vec() + from, (end - from) * 16);
    }
    // a tile again into a thread's registers; what lies past its vectors stays what it was
    __device__ __forceinline__ void reload(const Row<T>& row, const Group<GT>& g, int tile, uint4 (&d)[NV]) const
    {
        const uint4* q = row.vec() + at(g, tile);
        const int n = left(g, tile);
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (n > j * GT) d[j] = q[j * GT];
    }
    // the thread that holds vector v
    __device__ __forceinline__ bool owns(const Group<GT>& g, int v) const
    {
        return v >= begin && v < end && (v - begin) % GT == g.tid;
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
// m = max x, s = sum 2^y, t = sum 2^y y with y = c2 (x - m), in fp32 (t where ENT).
// Nothing seen: m = -inf, s = t = 0.  A NaN, or +inf, makes s NaN.
struct Acc {
    float m, s, t;
};

__device__ __forceinline__ Acc acc_none() { return Acc{NEG_INF, 0.f, 0.f}; }

// Moves a's sums to a maximum m that is not below a's.  Differences are held
// above FLOOR: a sum times the distance from a mask of the type's lowest value
// would overflow where its weight is 0.
template <bool ENT>
__device__ __forceinline__ Acc acc_to(const Acc& a, float m, float c2)
{
    const float d = a.s == 0.f ? 0.f : fmaxf((a.m - m) * c2, FLOOR), f = ex2(d);
    return Acc{m, a.s * f, ENT ? f * (a.t + a.s * d) : 0.f};
}

template <bool ENT>
__device__ __forceinline__ Acc acc_merge(const Acc& a, const Acc& b, float c2)
{
    const float m = max_nan(a.m, b.m);
    const Acc x = acc_to<ENT>(a, m, c2), y = acc_to<ENT>(b, m, c2);
    return Acc{m, x.s + y.s, x.t + y.t};
}

template <bool ENT>
__device__ __forceinline__ Acc acc_warp(const Acc& a, float c2)
{
    const float m = max_nan_warp(a.m);
    const Acc x = acc_to<ENT>(a, m, c2);
    return Acc{m, sum_warp(x.s), ENT ? sum_warp(x.t) : 0.f};
}

// One element of maximum x.
__device__ __forceinline__ Acc acc_one(float x)
{
    return Acc{x, x == NEG_INF ? 0.f : x - x == 0.f ? 1.f : __int_as_float(0x7fffffff), 0.f};
}

// y = c2 x - b with b = c2 m rounded takes one fused operation per element and
// is exact but for its own rounding; that y is off from c2 (x - m) by the
// same delta = c2 m - b for all elements.
struct Base {
    float b, delta;
    __device__ __forceinline__ Base(float m, float c2) : b(m * c2), delta(fmaf(m, c2, -(m * c2))) {}
};

// The statistics of the elements of one tile that a thread holds.  FAR: for
// maxima whose exponent rounds coarsely (masks of the lowest value, +inf, NaN),
// the difference from the maximum first, as an operation of its own.
template <class T, bool ENT, bool FAR>
__device__ __forceinline__ Acc acc_tile_from(const uint4 (&d)[NV], int used, float m, float c2)
{
    constexpr int E = Elem<T>::E;
    const Base base(FAR ? 0.f : m, c2);
    const Pair cc = pair(c2, c2), nb = pair(-base.b, -base.b), nm = pair(-m, -m);
    Pair s2[2] = {0, 0}, t2[2] = {0, 0};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (j % 2 == 0 && j >= used) break;
        float x[E];
        Elem<T>::unpack(d[j], x);
#pragma unroll
        for (int e = 0; e < E; e += 2) {
            const Pair v = pair(x[e], x[e + 1]);
            float y0, y1;
            split(FAR ? mul2(add2(v, nm), cc) : fma2(v, cc, nb), y0, y1);
            const Pair w = pair(ex2(y0), ex2(y1));
            s2[e >> 1 & 1] = add2(s2[e >> 1 & 1], w);
            if (ENT) t2[e >> 1 & 1] = fma2(w, pair(fmaxf(y0, FLOOR), fmaxf(y1, FLOOR)), t2[e >> 1 & 1]);
        }
    }
    float lo, hi;
    split(add2(s2[0], s2[1]), lo, hi);
    const float s = lo + hi, f = FAR ? 1.f : ex2(-base.delta);
    Acc a{m, s * f, 0.f};
    if (ENT) {
        split(add2(t2[0], t2[1]), lo, hi);
        a.t = f * (lo + hi - base.delta * s);
    }
    return a;
}

template <class T, bool ENT>
__device__ __forceinline__ Acc acc_tile(const uint4 (&d)[NV], int used, float m, float c2)
{
    if (m == NEG_INF) return acc_none();
    if (fabsf(m * c2) < NEAR) return acc_tile_from<T, ENT, false>(d, used, m, c2);
    return acc_tile_from<T, ENT, true>(d, used, m, c2);
}

// Every warp's statistics to every CTA of the row; the barrier of the exchange.
template <int GT>
__device__ __forceinline__ void exchange(const Acc& a, float extra, const Group<GT>& g, float4* slots)
{
    const float4 mine = make_float4(a.m, a.s, a.t, extra);
    if (g.parts == 1) {
        if (g.lane == 0) slots[g.warp] = mine;
        __syncthreads();
    } else {
        cluster_wait();   // every CTA of the row runs
        if (g.lane < g.parts) st_cluster_f4(mapa_shared(smem_u32(slots + g.rank * Group<GT>::W + g.warp), g.lane), mine);
        cluster_sync();
    }
}

template <int GT, bool ENT>
__device__ __forceinline__ Acc acc_slots(const float4* slots, int count, const Group<GT>& g, float c2)
{
    Acc a = acc_none();
    if (g.lane < count) {
        const float4 o = slots[g.lane];
        a = Acc{o.x, o.y, o.z};
    }
    for (int i = g.lane + 32; i < count; i += 32) {
        const float4 o = slots[i];
        a = acc_merge<ENT>(a, Acc{o.x, o.y, o.z}, c2);
    }
    return acc_warp<ENT>(a, c2);
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

// The candidates of a row's top k, in the first of its CTAs.
struct TopShared {
    unsigned long long key[CAND_MAX];
    int found[CAND_MAX];                  // ids; a share for each CTA of the row
    unsigned int hist[256];
    unsigned int counts[CLUSTER_MAX];
    unsigned int count, digit, above, bound, local;
};

// Gathers at least k and at most CAND_MAX keys of a row in memory, the k
// largest among them, by a radix search from the top digit that stops as soon
// as few enough are left: for rows whose largest tokens are not spread over the
// threads, or tie in great number.
template <class T, int GT>
__device__ __noinline__ void top_radix(const T* p, int vocab, unsigned int k, TopShared& sh)
{
    unsigned long long bound = 0;
    unsigned int taken = 0;              // keys above the digits found so far
    for (int shift = 56; shift >= 0; shift -= 8) {
        __syncthreads();
        for (int i = threadIdx.x; i < 256; i += GT) sh.hist[i] = 0;
        __syncthreads();
        for (int j = threadIdx.x; j < vocab; j += GT) {
            const unsigned long long key = token_key(Elem<T>::get(p + j), j);
            if (shift == 56 || key >> (shift + 8) == bound >> (shift + 8)) atomicAdd(&sh.hist[key >> shift & 255u], 1u);
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            unsigned int above = taken;
            int d = 255;
            while (d > 0 && above + sh.hist[d] < k) above += sh.hist[d--];
            sh.digit = d;
            sh.above = above;
            sh.count = 0;
        }
        __syncthreads();
        taken = sh.above;
        bound |= static_cast<unsigned long long>(sh.digit) << shift;
        if (taken + sh.hist[sh.digit] <= min(CAND_MAX, 2u * k + 64u)) break;
    }
    for (int j = threadIdx.x; j < vocab; j += GT) {
        const unsigned long long key = token_key(Elem<T>::get(p + j), j);
        if (key >= bound) sh.key[atomicAdd(&sh.count, 1u)] = key;
    }
    __syncthreads();
}

// Sorts key[0 .. n), n a power of two, falling, by the whole CTA.
template <int GT>
__device__ __noinline__ void sort_block(unsigned long long* key, int n)
{
    for (int size = 2; size <= n; size *= 2) {
        for (int step = size / 2; step; step /= 2) {
            __syncthreads();
            for (int i = threadIdx.x; i < n / 2; i += GT) {
                const int a = i / step * 2 * step + i % step, b = a + step;
                const unsigned long long x = key[a], y = key[b];
                if ((a & size) == 0 ? x < y : x > y) key[a] = y, key[b] = x;
            }
        }
    }
    __syncthreads();
}

// ------------------------------------------------- token log probabilities
// The gradient of one CTA's share of a row.  H: with the entropy's term,
//   c p (-g - h (logp + H)) = 2^y (A + B y),   y = c2 x - base.b.
template <class T, int PASS, int GT, bool ENT>
__device__ __forceinline__ void emit_logprob(const VocabParams& P, const Row<T>& row, const Part<T, GT>& part, const Group<GT>& g,
                                             float m, float inv_s, float logs, float H, float up_g, float up_h, int y, float xe,
                                             uint4 (&d)[NV])
{
    constexpr int E = Elem<T>::E;
    T* out = static_cast<T*>(P.dlogits) + g.row * P.ld_d;
    uint4* vout = reinterpret_cast<uint4*>(out + row.head);
    const bool same = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(row.p)) & 15u) == 0;
    const bool live = (up_g != 0.f || up_h != 0.f) && m != NEG_INF, near = fabsf(m * P.c2) < NEAR;
    const Base base(m, P.c2);
    const float scale = -P.c * inv_s * ex2(-base.delta);
    const float A = scale * (up_g + (ENT ? up_h * (H - logs - LN2 * base.delta) : 0.f)), B = ENT ? scale * up_h * LN2 : 0.f;
    const auto one = [&](float x) -> float {   // without the target's own term
        if (!live) return 0.f;
        const float l = (x - m) * P.c2, p = inv_s * ex2(l);
        return -P.c * p * (up_g + (ENT ? up_h * (LN2 * fmaxf(l, FLOOR) - logs + H) : 0.f));
    };
    for (int t = part.tiles - 1; t >= 0; --t) {
        const int first = part.at(g, t), left = part.left(g, t);
        if (live && near && same) {
            if (t < part.tiles - 1 || (PASS == VOCAB_BWD && t > 0)) part.template load<true>(row, g, t, d);
            const Pair cc = pair(P.c2, P.c2), nb = pair(-base.b, -base.b), A2 = pair(A, A), B2 = pair(B, B);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                if (j % 2 == 0 && j >= part.used(t)) break;
                float x[E];
                Elem<T>::unpack(d[j], x);
#pragma unroll
                for (int e = 0; e < E; e += 2) {
                    float y0, y1;
                    split(fma2(pair(x[e], x[e + 1]), cc, nb), y0, y1);
                    const Pair w = pair(ex2(y0), ex2(y1));
                    split(mul2(w, ENT ? fma2(pair(fmaxf(y0, FLOOR), fmaxf(y1, FLOOR)), B2, A2) : A2), x[e], x[e + 1]);
                }
                if (left > j * GT) __stcs(vout + first + j * GT, Elem<T>::pack(x));
            }
        } else {
#pragma unroll 1
            for (int j = 0; j * GT < left && j < NV; ++j) {
                float x[E] = {};
                if (live) Elem<T>::unpack(row.vec()[first + j * GT], x);
#pragma unroll
                for (int e = 0; e < E; ++e) x[e] = one(x[e]);
                if (same) {
                    vout[first + j * GT] = Elem<T>::pack(x);
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e) Elem<T>::put(out + row.head + (first + j * GT) * E + e, x[e]);
                }
            }
        }
    }
    if (g.has_edges() && g.lane < row.edges()) {
        const int id = row.edge(g.lane);
        Elem<T>::put(out + id, one(xe) + (live && id == y ? P.c * up_g : 0.f));
    }
}

template <class T, int PASS, int GT, bool ENT>
__global__ void __launch_bounds__(Group<GT>::THREADS, Group<GT>::CTAS) token_logprob_kernel(const VocabParams P)
{
    constexpr int E = Elem<T>::E;
    using G = Group<GT>;
    __shared__ float4 slots[PASS == VOCAB_BWD || GT == 32 ? 1 : CLUSTER_MAX * G::W];
    const G g;
    if (GT == 32 && g.row >= P.n) return;
    if (PASS != VOCAB_BWD && g.parts > 1) cluster_arrive();
    const Row<T> row(static_cast<const T*>(P.logits) + g.row * P.ld, P.vocab);
    const Part<T, GT> part(row, g, P.each);
    uint4 d[NV];
    part.load(row, g, 0, d);
    if (PASS == VOCAB_STEP) part.prefetch(row, g);
    const long long target = P.targets ? P.targets[g.row] : -1;
    const bool there = target >= 0 && target < P.vocab;
    const int y = there ? static_cast<int>(target) : -1;
    // the target's logit: for its log probability, and its own gradient (the
    // thread that holds its vector)
    const int vy = y >= row.head && y < row.head + row.full * E ? (y - row.head) / E : -1;
    const bool owner = PASS != VOCAB_FWD && part.owns(g, vy);
    float xy = 0.f, xe = NEG_INF, up_g = 0.f, up_h = 0.f;
    if (there && (owner || (PASS != VOCAB_BWD && g.rank == 0 && g.tid == 0))) xy = Elem<T>::get(row.p + y);
    if (g.has_edges() && g.lane < row.edges()) xe = Elem<T>::get(row.p + row.edge(g.lane));
    if (PASS != VOCAB_FWD) {
        up_g = there && P.dlogp ? P.dlogp[g.row] : 0.f;
        up_h = ENT && P.dentropy ? P.dentropy[g.row] : 0.f;
    }
    float m, s, logs = 0.f, H = 0.f;
    if (PASS == VOCAB_BWD) {
        const float4 st = reinterpret_cast<const float4*>(P.stats)[g.row];
        m = st.x, logs = st.y, H = st.z, s = expf(logs);
    } else {
        Acc a = acc_none();
        for (int t = 0; t < part.tiles; ++t) {
            if (t > 0) part.load(row, g, t, d);
            const Acc b = acc_tile<T, ENT>(d, part.used(t), Elem<T>::max_of(d), P.c2);
            a = t > 0 ? acc_merge<ENT>(a, b, P.c2) : b;
        }
        if (g.has_edges() && row.edges() > 0) a = acc_merge<ENT>(a, acc_one(xe), P.c2);
        a = acc_warp<ENT>(a, P.c2);
        if (GT != 32) {
            exchange(a, 0.f, g, slots);
            if (PASS == VOCAB_FWD && (g.rank != 0 || g.warp != 0)) return;
            a = acc_slots<GT, ENT>(slots, G::W * g.parts, g, P.c2);
        }
        m = a.m, s = a.s;
        if (ENT || (g.rank == 0 && g.warp == 0)) {
            logs = m == NEG_INF ? 0.f : logf(s);
            H = ENT && m != NEG_INF ? logs - LN2 * (a.t / s) : 0.f;
        }
    }
    if (PASS != VOCAB_BWD && g.rank == 0 && g.tid == 0) {
        if (P.logp) P.logp[g.row] = there ? (xy - (m == NEG_INF ? 0.f : m)) * P.c - logs : 0.f;
        if (ENT && P.entropy) P.entropy[g.row] = H;
        if (PASS == VOCAB_FWD && P.stats) reinterpret_cast<float4*>(P.stats)[g.row] = make_float4(m, logs, H, 0.f);
    }
    if constexpr (PASS != VOCAB_FWD) {
        const float inv_s = rcp(s);
        if (!ENT || up_h == 0.f) emit_logprob<T, PASS, GT, false>(P, row, part, g, m, inv_s, logs, H, up_g, 0.f, y, xe, d);
        else emit_logprob<T, PASS, GT, true>(P, row, part, g, m, inv_s, logs, H, up_g, up_h, y, xe, d);
        if (owner && m != NEG_INF && (up_g != 0.f || up_h != 0.f)) {   // over its own store of that vector
            const float l = (xy - m) * P.c2, p = inv_s * ex2(l);
            const float r = P.c * (up_g - p * (up_g + up_h * (LN2 * fmaxf(l, FLOOR) - logs + H)));
            Elem<T>::put(static_cast<T*>(P.dlogits) + g.row * P.ld_d + y, r);
        }
    }
}

// The forward with the k most likely tokens.  At least k tokens reach the k-th
// largest of the threads' maxima, and few more than k do where the largest are
// spread over the threads (74 at k = 64 of 32000 in random order, 256 threads).
// In a cluster, whose threads are too many and too far apart for that, each warp
// gives with its statistics the `each`-th largest of its threads' maxima, and at
// least k tokens reach the ceil(k / each)-th largest of those.  The tokens that
// reach the bound are gathered, by their bits, from the registers (or, of a tile
// before the last, read again), and each takes as its place the number of
// candidates before it.
template <class T, int GT, bool ENT>
__global__ void __launch_bounds__(Group<GT>::THREADS, Group<GT>::CTAS) token_logprob_top_kernel(const VocabParams P)
{
    constexpr int E = Elem<T>::E;
    using G = Group<GT>;
    static_assert(GT > 32, "one list of candidates per CTA");
    __shared__ float4 slots[CLUSTER_MAX * G::W];
    __shared__ TopShared top;
    const G g;
    const bool cluster = g.parts > 1;
    if (cluster) cluster_arrive();
    const Row<T> row(static_cast<const T*>(P.logits) + g.row * P.ld, P.vocab);
    const Part<T, GT> part(row, g, P.each);
    uint4 d[NV];
    part.load(row, g, 0, d);
    if (g.tid == 0) top.local = 0;
    const long long y = P.targets ? P.targets[g.row] : -1;
    const bool there = y >= 0 && y < P.vocab;
    float xy = 0.f, xe = NEG_INF;
    if (there && g.rank == 0 && g.tid == 0) xy = Elem<T>::get(row.p + y);
    const bool edge = g.has_edges() && g.lane < row.edges();
    if (edge) xe = Elem<T>::get(row.p + row.edge(g.lane));
    Acc a = acc_none();
    uint32_t mine = 0, second = 0;   // this thread's largest, the largest of its other tiles
    int tile = 0;                    // and the tile that has it
    for (int t = 0; t < part.tiles; ++t) {
        if (t > 0) part.load(row, g, t, d);
        const float mt = Elem<T>::max_of(d);
        const uint32_t key = value_key(mt);
        second = max(second, min(mine, key));
        if (key > mine) mine = key, tile = t;
        const Acc b = acc_tile<T, ENT>(d, part.used(t), mt, P.c2);
        a = t > 0 ? acc_merge<ENT>(a, b, P.c2) : b;
    }
    if (g.has_edges() && row.edges() > 0) a = acc_merge<ENT>(a, acc_one(xe), P.c2);
    a = acc_warp<ENT>(a, P.c2);
    const int warps = G::W * g.parts;
    const bool bounded = P.top_each > 0;
    uint32_t best = 0;
    if (bounded && (cluster || P.k <= G::W)) {
        uint32_t left = mine;
        for (int i = 0; i < P.top_each; ++i) {
            best = __reduce_max_sync(~0u, left);
            if (g.lane == __ffs(__ballot_sync(~0u, left == best)) - 1) left = 0;
        }
    }
    exchange(a, __uint_as_float(best), g, slots);
    a = acc_slots<GT, ENT>(slots, warps, g, P.c2);
    const float m = a.m, m0 = m == NEG_INF ? 0.f : m, logs = m == NEG_INF ? 0.f : logf(a.s);
    if (g.rank == 0 && g.tid == 0) {
        const float H = ENT && m != NEG_INF ? logs - LN2 * (a.t / a.s) : 0.f;
        if (P.logp) P.logp[g.row] = there ? (xy - m0) * P.c - logs : 0.f;
        if (ENT && P.entropy) P.entropy[g.row] = H;
        if (P.stats) reinterpret_cast<float4*>(P.stats)[g.row] = make_float4(m, logs, H, 0.f);
    }
    unsigned int count = CAND_MAX + 1;
    if (bounded) {
        uint32_t bound = 0;
        if (!cluster && P.k > G::W) {
            // the k-th largest of the threads' maxima, from above to its upper 16 bits
            const uint32_t most = value_key(m);
            // (its upper bits, where few more than k reach them)
            for (uint32_t bit = 0x80000000u; bit > 0x8000u; bit >>= 1) {
                if ((bound | bit) > most) continue;
                const int n = __syncthreads_count(mine >= (bound | bit));
                if (n >= P.k) bound |= bit;
                if (n >= P.k && n <= P.k + (P.k >> 3) + 2) break;
            }
        } else {
            // the warps' value with top_before before it: each warp counts for one of each CTA
            uint32_t all[CLUSTER_MAX * G::W / 32];
#pragma unroll
            for (int q = 0; q < CLUSTER_MAX * G::W / 32; ++q)
                all[q] = g.lane + 32 * q < warps ? __float_as_uint(slots[g.lane + 32 * q].w) : 0u;
#pragma unroll
            for (int r = 0; r < CLUSTER_MAX; ++r) {
                if (r < g.parts) {
                    const int i = r * G::W + g.warp;
                    const uint32_t v = __float_as_uint(slots[i].w);
                    unsigned int n = 0;
#pragma unroll
                    for (int q = 0; q < CLUSTER_MAX * G::W / 32; ++q) n += all[q] > v || (all[q] == v && g.lane + 32 * q < i);
                    if (__reduce_add_sync(~0u, n) == static_cast<unsigned int>(P.top_before) && g.lane == 0) top.bound = v;
                }
            }
            __syncthreads();
            bound = top.bound;
        }
        // a bound of -inf: what lies above it here; the first of the -inf tokens follow below
        const float limit = bound <= value_key(NEG_INF) ? Elem<T>::LOWEST : key_value(bound);
        const unsigned int share = CAND_MAX >> (31 - __clz(g.parts));   // clusters are powers of two
        const uint32_t list = cluster ? mapa_shared(smem_u32(top.found + g.rank * share), 0) : 0;
        const auto take = [&](int id) {
            const unsigned int at = atomicAdd(&top.local, 1u);
            if (at < share) {
                if (cluster) st_shared_cluster_u32(list + 4 * at, id);
                else top.found[at] = id;
            }
        };
        const auto take_tile = [&](int t) {
            unsigned long long bits = Elem<T>::reach(d, limit);
            while (bits) {
                const int b = Elem<T>::place(__ffsll(bits) - 1);
                bits &= bits - 1;
                if (b / E * GT < part.left(g, t)) take(row.head + (part.at(g, t) + b / E * GT) * E + b % E);
            }
        };
        if (mine >= bound) {   // each thread the tile of its largest, then the rest if its second reaches too
            if (part.tiles > 1) part.reload(row, g, tile, d);
            take_tile(tile);
            for (int t = 0; second >= bound && t < part.tiles; ++t) {
                if (t == tile) continue;
                part.reload(row, g, t, d);
                take_tile(t);
            }
        }
        if (edge && !(xe < limit)) take(row.edge(g.lane));
        __syncthreads();
        if (cluster) {
            if (g.tid == 0) st_shared_cluster_u32(mapa_shared(smem_u32(top.counts + g.rank), 0), top.local);
            cluster_sync();
            if (g.rank != 0) return;
            count = 0;
            for (int r = 0; r < g.parts; ++r) count = top.counts[r] > share ? 2 * CAND_MAX : count + top.counts[r];
        } else {
            count = top.local;
        }
        if (count <= CAND_MAX) {
            for (unsigned int c = g.tid; c < count; c += GT) {
                unsigned int at = c;
                for (int r = 0; cluster && r < g.parts - 1 && at >= r * share + top.counts[r]; ++r) at += share - top.counts[r];
                const int id = top.found[at];
                top.key[c] = token_key(Elem<T>::get(row.p + id), id);
            }
        }
        if (count < static_cast<unsigned int>(P.k) && g.warp == 0) {
            // fewer than k tokens above -inf: the lowest ids of the others follow,
            // all of them among the first k + count ids
            unsigned int n = count;
            for (int id = g.lane; n < static_cast<unsigned int>(P.k); id += 32) {
                const bool none = id < P.vocab && Elem<T>::get(row.p + id) == NEG_INF;
                const unsigned int set = __ballot_sync(~0u, none);
                const unsigned int at = n + __popc(set & ((1u << g.lane) - 1));
                if (none && at < CAND_MAX) top.key[at] = token_key(NEG_INF, id);
                n += __popc(set);
            }
            if (g.lane == 0) top.count = min(n, static_cast<unsigned int>(CAND_MAX));
        }
        __syncthreads();
        if (count < static_cast<unsigned int>(P.k)) count = top.count;
    } else if (g.rank != 0) {
        return;
    }
    if (count > CAND_MAX) {
        top_radix<T, GT>(row.p, P.vocab, P.k, top);
        count = top.count;
    }
    const auto give = [&](unsigned long long key, unsigned int place) {
        P.top_ids[g.row * P.k + place] = 0xffffffffu - static_cast<uint32_t>(key);
        P.top_logp[g.row * P.k + place] = (key_value(static_cast<uint32_t>(key >> 32)) - m0) * P.c - logs;
    };
    const int n = count <= 2 ? static_cast<int>(count) : 1 << (32 - __clz(count - 1));
    // counting takes count^2 / 32 steps of all warps together, sorting 30 to 55 barriers
    if (n <= min(GT, 256)) {
        // `share` neighbouring threads count for one candidate
        const int log_share = min(5, __clz(n) - __clz(GT));
        const unsigned int share = 1u << log_share, c = g.tid >> log_share;
        const unsigned long long key = c < count ? top.key[c] : 0;
        unsigned int before = 0;
        if (g.warp * 32u >> log_share < count) {   // the warp has candidates
#pragma unroll 4
            for (unsigned int i = g.tid & (share - 1); i < count; i += share) before += top.key[i] > key;
            for (unsigned int i = share / 2; i; i /= 2) before += __shfl_xor_sync(~0u, before, i);
            if (c < count && (g.tid & (share - 1)) == 0 && before < static_cast<unsigned int>(P.k)) give(key, before);
        }
    } else {
        for (int i = count + g.tid; i < n; i += GT) top.key[i] = 0;
        sort_block<GT>(top.key, n);
        for (int i = g.tid; i < P.k; i += GT) give(top.key[i], i);
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

// A teacher's list, taken in by every CTA of the row: entry i by thread i mod GT.
template <int GT>
struct ListShared {
    int id[VOCAB_MAX_K];                    // -1: no token
    float u[VOCAB_MAX_K], x[VOCAB_MAX_K];   // the teacher's exponent, the student's logit
    float2 student[Group<GT>::W], teacher[Group<GT>::W];   // maximum and sum, per warp
    float sum[Group<GT>::W];
    unsigned int edges;                     // bits of the row's edge elements that are on the list
};

template <class T>
using Bits = typename Elem<T>::Bits;        // a bit per element of a tile that a thread holds

// PASS: the forward, forward and backward, or the backward from saved statistics.
template <class T, int PASS, int GT>
__global__ void __launch_bounds__(Group<GT>::THREADS, Group<GT>::CTAS) topk_distill_kernel(const VocabParams P)
{
    constexpr int E = Elem<T>::E;
    using G = Group<GT>;
    extern __shared__ unsigned long long listed_raw[];   // forward: a word of bits per thread and tile
    __shared__ float4 slots[GT == 32 || PASS == VOCAB_BWD ? 1 : CLUSTER_MAX * G::W];
    __shared__ ListShared<GT> lists[G::ROWS];
    const G g;
    if (GT == 32 && g.row >= P.n) return;
    const bool cluster = g.parts > 1;
    if (cluster) cluster_arrive();
    const Row<T> row(static_cast<const T*>(P.logits) + g.row * P.ld, P.vocab);
    const Part<T, GT> part(row, g, P.each);
    ListShared<GT>& list = lists[g.slot];
    // the list's loads are under way before the row's
    const float shift = P.rest && P.t_lse ? P.t_lse[g.row] : 0.f;
    const long long t0 = g.tid < P.k ? P.t_ids[g.row * P.k + g.tid] : -1;
    const float u0 = g.tid < P.k ? P.t_vals[g.row * P.k + g.tid] : 0.f;
    uint4 d[NV];
    part.load(row, g, 0, d);
    if (PASS == VOCAB_STEP) part.prefetch(row, g);
    if (g.warp == 0 && g.row + P.ahead < P.n) {   // a later row's list
        const long long at = (g.row + P.ahead) * P.k;
        if (g.lane * 16 < P.k) prefetch_l2(P.t_ids + at + g.lane * 16);
        if (g.lane * 32 < P.k) prefetch_l2(P.t_vals + at + g.lane * 32);
    }
    const bool edge = g.has_edges() && g.lane < row.edges();
    const int edge_id = edge ? row.edge(g.lane) : -1;
    float xe = edge ? Elem<T>::get(row.p + edge_id) : NEG_INF;
    const float w = PASS != VOCAB_FWD ? P.dloss[g.row] : 0.f;
    float m = 0.f, logs = 0.f, mr = 0.f, logr = 0.f, s, sr;
    if (PASS == VOCAB_BWD) {
        const float4 st = reinterpret_cast<const float4*>(P.stats)[g.row];
        m = st.x, logs = st.y, mr = st.z, logr = st.w;
        s = expf(logs), sr = expf(logr);
    }
    Bits<T>* listed = reinterpret_cast<Bits<T>*>(listed_raw) + g.slot * GT;
    if (PASS != VOCAB_BWD) {
        for (int t = 0; t < part.tiles; ++t) listed[t * GT + g.tid] = 0;
        if (g.tid == 0) list.edges = 0;
        G::sync();
    }
    const bool lister = g.warp * 32 < P.k;   // the warp has entries
    float x0 = NEG_INF;                      // the thread's first entry's, under way until after the barrier
    if (lister) {
        float um = NEG_INF, us = 0.f;
        for (int i = g.tid; i < P.k; i += GT) {
            const long long t = i == g.tid ? t0 : P.t_ids[g.row * P.k + i];
            const bool there = t >= 0 && t < P.vocab;
            const int id = there ? static_cast<int>(t) : -1;
            if (there) {
                if (i == g.tid) x0 = Elem<T>::get(row.p + id);
                if (PASS != VOCAB_BWD) {
                    const int at = id - row.head, v = at / E - part.begin, tile = v / G::TILE;
                    if (at < 0 || at >= row.full * E)
                        atomicOr(&list.edges, 1u << (at < 0 ? id : row.head + at - row.full * E));
                    else if (v >= 0 && part.begin + v < part.end)
                        atomicOr(listed + tile * GT + v % GT, static_cast<Bits<T>>(1) << (v % G::TILE / GT * E + at % E));
                }
            }
            const float u = there ? (i == g.tid ? u0 : P.t_vals[g.row * P.k + i]) * P.t_c - shift : NEG_INF;
            list.id[i] = id;
            list.u[i] = u;
            um = max_nan(um, u);
        }
        um = P.rest ? 0.f : max_nan_warp(um);
        for (int i = g.tid; i < P.k; i += GT)
            if (list.id[i] >= 0 && um != NEG_INF) us += expf(list.u[i] - um);
        us = sum_warp(us);
        if (g.lane == 0) list.teacher[g.warp] = make_float2(um, us);
    }
    if (PASS != VOCAB_BWD) {
        G::sync();
        if (edge && list.edges >> g.lane & 1) xe = NEG_INF;
    }
    // the student's statistics on the list, a share per warp (the gathers were issued before the barrier)
    const auto gather = [&]() {
        if (!lister) return;
        float xm = NEG_INF, xs = 0.f;
        for (int i = g.tid; i < P.k; i += GT) {
            const int id = list.id[i];
            const float x = i == g.tid ? x0 : id >= 0 ? Elem<T>::get(row.p + id) : NEG_INF;
            list.x[i] = x;
            xm = max_nan(xm, x);
        }
        xm = max_nan_warp(xm);
        for (int i = g.tid; i < P.k; i += GT)
            if (list.id[i] >= 0 && xm != NEG_INF) xs += ex2((list.x[i] - xm) * P.c2);
        xs = sum_warp(xs);
        if (g.lane == 0) list.student[g.warp] = make_float2(xm, xs);
    };
    Acc r = acc_none();
    if (PASS == VOCAB_BWD) {
        gather();
        // in place: the list's logits are read before any CTA of the row stores
        if (cluster) {
            cluster_wait();
            cluster_sync();
        } else {
            G::sync();
        }
    } else {
        Acc a = acc_none();
        for (int t = 0; t < part.tiles; ++t) {
            if (t > 0) part.load(row, g, t, d);
            const Bits<T> mine = listed[t * GT + g.tid];
            if (mine) {
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    const uint32_t b = static_cast<uint32_t>(mine >> (j * E)) & ((1u << E) - 1);
                    if (b) Elem<T>::ban(d[j], b);
                }
            }
            const Acc b = acc_tile<T, false>(d, part.used(t), Elem<T>::max_of(d), P.c2);
            a = t > 0 ? acc_merge<false>(a, b, P.c2) : b;
        }
        if (g.has_edges() && row.edges() > 0) a = acc_merge<false>(a, acc_one(xe), P.c2);
        gather();
        r = acc_warp<false>(a, P.c2);
        if (GT == 32) {
            G::sync();
        } else {
            exchange(r, 0.f, g, slots);
            if (PASS == VOCAB_FWD && (g.rank != 0 || !lister)) {
                if (g.rank == 0) __syncthreads();
                return;
            }
            r = acc_slots<GT, false>(slots, G::W * g.parts, g, P.c2);
        }
        mr = r.m, sr = r.s;
    }
    // the list's statistics over its warps: the student's, the teacher's
    Acc l = acc_none();
    float um = NEG_INF, us = 0.f;
    if (g.lane < G::W && g.lane * 32 < P.k) {
        const float2 o = list.student[g.lane], q = list.teacher[g.lane];
        l = Acc{o.x, o.y, 0.f};
        um = q.x, us = q.y;
    }
    l = acc_warp<false>(l, P.c2);
    if (P.rest) {
        us = sum_warp(us);
    } else {
        const float uml = max_nan_warp(um);
        us = sum_warp(us == 0.f ? 0.f : us * expf(um - uml));
        um = uml;
    }
    if (PASS != VOCAB_BWD) {
        m = max_nan(l.m, r.m);
        s = acc_to<false>(l, m, P.c2).s + acc_to<false>(r, m, P.c2).s;
    }
    const float m0 = m == NEG_INF ? 0.f : m;
    // teacher: q_k = exp(u_k - um) / us or exp(u_k); Q = sum q; rest: an entry of its own where q_R > 0
    const float Q = P.rest ? us : us == 0.f ? 0.f : us - us + 1.f;
    const float qr = P.rest && mr != NEG_INF ? fmaxf(1.f - Q, 0.f) : 0.f;
    const bool entry = qr > 0.f;
    const float wt = w * P.temperature;
    const bool live = w != 0.f && m != NEG_INF;
    float logpr = 0.f;
    // loss, and the list's gradients (stored over the row's below)
    float kl = 0.f;
    if (lister) {
        if (PASS != VOCAB_BWD) {
            logs = m == NEG_INF ? 0.f : logf(s);
            logr = mr == NEG_INF ? 0.f : logf(sr);
        }
        logpr = (mr - m0) * P.c + logr - logs;
        const float u_log = P.rest ? 0.f : us == 0.f ? 0.f : um + logf(us);
        for (int i = g.tid; i < P.k; i += GT) {
            if (list.id[i] < 0) continue;
            const float logq = list.u[i] - u_log, q = us == 0.f ? 0.f : P.rest ? expf(logq) : expf(list.u[i] - um) / us;
            const float logp = (list.x[i] - m0) * P.c - logs, p = expf(logp);
            if (PASS != VOCAB_BWD) {
                if (entry) kl += q > 0.f ? q * excess(logq - logp) : p;
                else kl += q > 0.f ? q * (logq - logp) : 0.f * q;
            }
            if (PASS != VOCAB_FWD) list.u[i] = wt * ((entry ? 1.f : Q) * p - q);
        }
        if (PASS != VOCAB_BWD) {
            kl = sum_warp(kl);
            if (g.lane == 0) list.sum[g.warp] = kl;
        }
    }
    if constexpr (PASS != VOCAB_FWD) {
        T* out = static_cast<T*>(P.dlogits) + g.row * P.ld_d;
        uint4* vout = reinterpret_cast<uint4*>(out + row.head);
        const bool same = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(row.p)) & 15u) == 0;
        const bool near = fabsf(mr * P.c2) < NEAR;
        const Base base(mr, P.c2);
        // rate of exp(c (x - mr)): with the rest (Q - sum p) / sr, else Q p_R / sr
        const float rate = mr == NEG_INF ? 0.f
                           : entry       ? wt * (Q - acc_to<false>(l, m, P.c2).s * rcp(s)) * rcp(sr)
                                         : wt * Q * ex2((mr - m) * P.c2) * rcp(s);
        const float A = rate * ex2(-base.delta);
        const auto one = [&](float x) -> float {
            if (!live || mr == NEG_INF) return 0.f;
            return rate * ex2((x - mr) * P.c2);
        };
        for (int t = part.tiles - 1; t >= 0; --t) {
            const int first = part.at(g, t), left = part.left(g, t);
            if (live && near && same) {
                if (t < part.tiles - 1 || (PASS == VOCAB_BWD && t > 0)) part.template load<true>(row, g, t, d);
                const Pair cc = pair(P.c2, P.c2), nb = pair(-base.b, -base.b), A2 = pair(A, A);
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    if (j % 2 == 0 && j >= part.used(t)) break;
                    float x[E];
                    Elem<T>::unpack(d[j], x);
#pragma unroll
                    for (int e = 0; e < E; e += 2) {
                        float y0, y1;
                        split(fma2(pair(x[e], x[e + 1]), cc, nb), y0, y1);
                        split(mul2(pair(ex2(y0), ex2(y1)), A2), x[e], x[e + 1]);
                    }
                    if (left > j * GT) __stcs(vout + first + j * GT, Elem<T>::pack(x));
                }
            } else {
#pragma unroll 1
                for (int j = 0; j * GT < left && j < NV; ++j) {
                    float x[E] = {};
                    if (live) Elem<T>::unpack(row.vec()[first + j * GT], x);
#pragma unroll
                    for (int e = 0; e < E; ++e) x[e] = one(x[e]);
                    if (same) {
                        vout[first + j * GT] = Elem<T>::pack(x);
                    } else {
#pragma unroll
                        for (int e = 0; e < E; ++e) Elem<T>::put(out + row.head + (first + j * GT) * E + e, x[e]);
                    }
                }
            }
        }
        if (edge) Elem<T>::put(out + edge_id, one(xe));
        G::sync();
        for (int i = g.tid; live && i < P.k; i += GT) {
            const int id = list.id[i];
            if (id < 0) continue;
            const int at = id - row.head, v = at / E;
            const bool vector = at >= 0 && v < row.full;
            if (vector ? v >= part.begin && v < part.end : g.rank == 0) Elem<T>::put(out + id, list.u[i]);
        }
    } else {
        G::sync();
    }
    if (PASS != VOCAB_BWD && g.rank == 0 && g.tid == 0) {
        kl = 0.f;
        for (int i = 0; i < G::W && i * 32 < P.k; ++i) kl += list.sum[i];
        if (entry) kl += qr * excess(log1pf(-Q) - logpr);
        P.loss[g.row] = P.temperature * P.temperature * kl;
        if (PASS == VOCAB_FWD && P.stats) reinterpret_cast<float4*>(P.stats)[g.row] = make_float4(m, logs, mr, logr);
    }
}
#endif

}  // namespace cola
