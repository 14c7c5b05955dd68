// vocab_rows.cuh -- rows of vocabulary logits: element types, loads and stores, softmax
// statistics and their exchange between the warps and CTAs of a row.
#pragma once
#include <cuda_bf16.h>

#include <cstdint>

#include "ptx.cuh"
#include "vocab.cuh"

namespace cola {

constexpr int NV = 8;                   // 16-byte vectors a thread holds at once
constexpr int CLUSTER_MAX = 8;
constexpr int CAND_MAX = 1024;          // candidates for the top k kept on chip
constexpr float NEG_INF = -__builtin_huge_valf();
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
    __device__ __forceinline__ static float largest(const uint4& u)
    {
        return max_nan(max_nan(__uint_as_float(u.x), __uint_as_float(u.y)), max_nan(__uint_as_float(u.z), __uint_as_float(u.w)));
    }
    // bits whose upper half alone tells x apart from 0 where it is below
    __device__ __forceinline__ static uint32_t above_half(float x)
    {
        const uint32_t b = __float_as_uint(x);
        return b > 0x80000000u && b < 0x80010000u ? 0x80010000u : b;
    }
    // upper halves of the maxima of two parts of two vectors (here: of each vector)
    __device__ __forceinline__ static uint32_t halves(const uint4& a, const uint4& b)
    {
        return __byte_perm(above_half(largest(a)), above_half(largest(b)), 0x7632);
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
    // a bit for each element of the first `used` vectors that is not below `limit` (a NaN is not),
    // NANS: that is a NaN; and the place of a bit's element in its tile
    template <bool NANS = false>
    __device__ __forceinline__ static unsigned long long reach(const uint4 (&d)[NV], int used, float limit)
    {
        unsigned int bits = 0;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (j % 2 == 0 && j >= used) break;
            float x[4];
            unpack(d[j], x);
#pragma unroll
            for (int e = 0; e < 4; ++e) bits |= (NANS ? x[e] != x[e] : !(x[e] < limit)) ? 1u << (j * 4 + e) : 0u;
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
    // as above; the limit's upper half (a key between two values of this type stands for the one above),
    // a word's two elements compared at once, the bits of words 0..15 and 16..31 in halves:
    // low elements, then high ones
    template <bool NANS = false>
    __device__ __forceinline__ static unsigned long long reach(const uint4 (&d)[NV], int used, float limit)
    {
        const uint32_t half = __float_as_uint(limit) >> 16, both = half << 16 | half;
        const __nv_bfloat162 l = *reinterpret_cast<const __nv_bfloat162*>(&both);
        uint32_t bits[2] = {0, 0};
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (j % 2 == 0 && j >= used) break;
            const uint32_t w[4] = {d[j].x, d[j].y, d[j].z, d[j].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const __nv_bfloat162 x = *reinterpret_cast<const __nv_bfloat162*>(&w[i]);
                const uint32_t there = NANS ? __hneu2_mask(x, x) : ~__hlt2_mask(x, l);
                bits[j / 4] |= there & (0x00010001u << (j % 4 * 4 + i));
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
    __device__ __forceinline__ static float largest(const uint4& u)
    {
        const uint32_t m = max_pair(max_pair(u.x, u.y), max_pair(u.z, u.w));
        return max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
    }
    __device__ __forceinline__ static uint32_t halves(const uint4& a, const uint4& b)   // (of their even and odd elements)
    {
        return max_pair(max_pair(max_pair(a.x, a.y), max_pair(a.z, a.w)), max_pair(max_pair(b.x, b.y), max_pair(b.z, b.w)));
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

// Stores a warp's consecutive vectors (those that are `mine`, from lane 0 on) where
// they do not begin on a 16-byte boundary: each lane the 16-byte block that begins
// within its vector and ends in the next lane's; the ends element by element.
template <class T>
__device__ __forceinline__ void store_apart(T* dst, const uint4& p, bool mine)
{
    constexpr int E = Elem<T>::E;
    const int lane = threadIdx.x & 31;
    const unsigned int cut = 16 - static_cast<unsigned int>(reinterpret_cast<uintptr_t>(dst) & 15u);   // bytes before the block
    const uint32_t c[8] = {p.x, p.y, p.z, p.w, __shfl_down_sync(~0u, p.x, 1), __shfl_down_sync(~0u, p.y, 1),
                           __shfl_down_sync(~0u, p.z, 1), __shfl_down_sync(~0u, p.w, 1)};
    const bool next = __shfl_down_sync(~0u, mine, 1) && lane < 31;
    uint32_t a[7], b[5];
#pragma unroll
    for (int i = 0; i < 7; ++i) a[i] = cut & 8 ? c[i + 2 < 8 ? i + 2 : 7] : c[i];
#pragma unroll
    for (int i = 0; i < 5; ++i) b[i] = cut & 4 ? a[i + 1] : a[i];
    const unsigned int bits = (cut & 3) * 8;
    if (cut == 16) {   // (some rows may lie alike)
        if (mine) __stcs(reinterpret_cast<uint4*>(dst), p);
        return;
    }
    if (mine && next)
        __stcs(reinterpret_cast<uint4*>(reinterpret_cast<char*>(dst) + cut),
               make_uint4(__funnelshift_r(b[0], b[1], bits), __funnelshift_r(b[1], b[2], bits), __funnelshift_r(b[2], b[3], bits),
                          __funnelshift_r(b[3], b[4], bits)));
    if (mine && (lane == 0 || !next)) {
        const int first = static_cast<int>(cut / sizeof(T));
        float x[E];
        Elem<T>::unpack(p, x);
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (e < first ? lane == 0 : !next) Elem<T>::put(dst + e, x[e]);
    }
}

// The GT threads that work on one row in one CTA: a warp (four rows a CTA) or
// the whole CTA; the row's CTAs lie along the grid's y, and form a cluster
// where they exchange anything.  A warp's rows gain from eight CTAs an SM although
// some of their forms then spill a few registers (65536 rows: bf16 entropy backward of
// 1000 logits 53 us against 58 us on six, fp32 entropy step of 504 54 against 57 us; of
// 1000 it loses, 84 against 81 us).
template <int GT>
struct Group {
    static constexpr int ROWS = GT == 32 ? 4 : 1, THREADS = GT * ROWS, W = GT / 32, TILE = GT * NV;
    static constexpr int CTAS = 1024 / THREADS;   // an SM's, for the registers a thread may have
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

// A tile's gradient 2^y (A + B y), y = c2 (x - m), read from memory again (zeros
// where not `live`): for rows without gradient and maxima far from 0, and, APART,
// for results that lie otherwise on 16-byte boundaries than the logits.
template <class T, int GT, bool APART>
__device__ __forceinline__ void emit_again(const uint4* src, T* dst, int left, int used, float m, float c2, float A, float B,
                                           bool live)
{
    constexpr int E = Elem<T>::E;
    const bool same = (reinterpret_cast<uintptr_t>(dst) & 15u) == 0;
#pragma unroll(APART ? 4 : 1)
    for (int j = 0; j < used; ++j) {
        const bool mine = left > j * GT;
        float x[E] = {};
        if (live && mine) Elem<T>::unpack(src[j * GT], x);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float y = (x[e] - m) * c2;
            x[e] = live ? ex2(y) * fmaf(fmaxf(y, FLOOR), B, A) : 0.f;
        }
        if constexpr (APART) {
            store_apart(dst + j * GT * E, Elem<T>::pack(x), mine);
        } else if (mine) {
            if (same) {
                __stcs(reinterpret_cast<uint4*>(dst) + j * GT, Elem<T>::pack(x));
            } else {   // (a warp's rows alone)
#pragma unroll
                for (int e = 0; e < E; ++e) Elem<T>::put(dst + j * GT * E + e, x[e]);
            }
        }
    }
}

}  // namespace cola
