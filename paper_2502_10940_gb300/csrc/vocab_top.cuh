// vocab_top.cuh -- log probabilities with the row's most likely tokens.
#pragma once
#include "vocab_rows.cuh"

namespace cola {

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

// The same in 32 bits, for bf16 logits (their value keys differ in the upper
// half alone) and ids of 16 bits.
__device__ __forceinline__ uint32_t narrow_key(float x, int j)
{
    return (value_key(x) & 0xffff0000u) | (0xffffu - static_cast<uint32_t>(j));
}

__device__ __forceinline__ int key_id(unsigned long long key)
{
    return static_cast<int>(0xffffffffu - static_cast<uint32_t>(key));
}
__device__ __forceinline__ int key_id(uint32_t key) { return static_cast<int>(0xffffu - (key & 0xffffu)); }
__device__ __forceinline__ float key_logit(unsigned long long key) { return key_value(static_cast<uint32_t>(key >> 32)); }
__device__ __forceinline__ float key_logit(uint32_t key)
{
    return key_value(key & 0x80000000u ? key & 0xffff0000u : key | 0xffffu);
}

constexpr uint32_t KEY_NEG_INF = 0x007fffffu, KEY_POS_INF = 0xff800000u;   // of the infinities; above the latter, NaNs

// The lowest value key above `key` that a value of type T may have; the bits of a key that tell values apart.
template <class T>
__device__ __forceinline__ uint32_t next_key(uint32_t key) { return sizeof(T) == 2 ? (key & 0xffff0000u) + 0x10000u : key + 1; }
template <class T>
__device__ __forceinline__ bool same_key(uint32_t a, uint32_t b) { return sizeof(T) == 2 ? a >> 16 == b >> 16 : a == b; }

// Bits of the elements of a tile whose value key is at least `from`.
template <class T>
__device__ __forceinline__ unsigned long long reach(const uint4 (&d)[NV], int used, uint32_t from)
{
    if (from > KEY_POS_INF) return Elem<T>::template reach<true>(d, used, 0.f);
    return Elem<T>::template reach<false>(d, used, from <= KEY_NEG_INF ? NEG_INF : key_value(from));
}

// How many of `count` keys (zeros after them, to a multiple of 16 bytes) are
// above `key`, the 16-byte words first, first + step, ... counted.
__device__ __forceinline__ unsigned int count_above(const unsigned long long* keys, unsigned int count, unsigned long long key,
                                                    unsigned int first, unsigned int step)
{
    unsigned int n = 0;
#pragma unroll 4
    for (unsigned int i = first; 2 * i < count; i += step) {
        const ulonglong2 o = reinterpret_cast<const ulonglong2*>(keys)[i];
        n += (o.x > key) + (o.y > key);
    }
    return n;
}
__device__ __forceinline__ unsigned int count_above(const uint32_t* keys, unsigned int count, uint32_t key, unsigned int first,
                                                    unsigned int step)
{
    unsigned int n = 0;
#pragma unroll 4
    for (unsigned int i = first; 4 * i < count; i += step) {
        const uint4 o = reinterpret_cast<const uint4*>(keys)[i];
        n += (o.x > key) + (o.y > key) + (o.z > key) + (o.w > key);
    }
    return n;
}

// The candidates of a row's top k, in the first of its CTAs.
struct TopShared {
    alignas(16) unsigned long long key[CAND_MAX];
    int found[CAND_MAX];                  // ids; a share for each CTA of the row
    unsigned int hist[256];
    unsigned int counts[CLUSTER_MAX];
    unsigned int count, digit, above, bound, local;
    unsigned int part[2][16];           // counts of the warps, in turn
};

constexpr unsigned int RANK_MAX = 512;   // candidates that are counted, not sorted

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
    if (threadIdx.x == 0 && sh.count < CAND_MAX) sh.key[sh.count] = 0;
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

// The forward with the k most likely tokens.  FEW: k is more than half of the
// threads, whose registers hold the row; the tokens themselves are counted, by
// their bits, for the bound.  Else at least k tokens reach the k-th
// largest of the threads' maxima, and few more than k do where the largest are
// spread over the threads (74 at k = 64 of 32000 in random order, 256 threads).
// In a cluster, whose threads are too many and too far apart for that, each warp
// gives with its statistics the `each`-th largest of its threads' maxima, and at
// least k tokens reach the ceil(k / each)-th largest of those.  The tokens that
// reach the bound are gathered, by their bits, from the registers (or, of a tile
// before the last, read again), and each takes as its place the number of
// candidates before it.
// One pass of HBM, which the bound, the gather and the ranking follow in each row:
// what overlaps them is the next rows of the SM.  4096 x 32000 fp32, k = 1: 84 us,
// 6.2 TB/s; 8192 x 32000 bf16, k = 64: 120 us, 4.4 TB/s, where each row's 12,500
// instructions fill 66 % of the issue slots and the barriers between the bound's
// steps most of the others.
template <class T, int GT, bool ENT, bool FEW>
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
    // the maxima of this thread's two tiles with the largest, their numbers, and the maximum of its others
    uint32_t mine = 0, second = 0, third = 0;
    int tile = 0, tile2 = 0;
    for (int t = 0; t < part.tiles; ++t) {
        if (t > 0) part.load(row, g, t, d);
        const float mt = Elem<T>::max_of(d);
        const uint32_t key = value_key(mt);
        third = max(third, min(second, key));
        if (key > mine) second = mine, tile2 = tile, mine = key, tile = t;
        else if (key > second) second = key, tile2 = t;
        const Acc b = acc_tile<T, ENT>(d, part.used(t), mt, P.c2);
        a = t > 0 ? acc_merge<ENT>(a, b, P.c2) : b;
    }
    if (g.has_edges() && row.edges() > 0) a = acc_merge<ENT>(a, acc_one(xe), P.c2);
    a = acc_warp<ENT>(a, P.c2);
    const int warps = G::W * g.parts;
    uint32_t best = 0;
    if (cluster || P.k <= G::W) {
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
    unsigned int count = 0;
    bool narrow = false;
    uint32_t* key32 = reinterpret_cast<uint32_t*>(top.key);
    uint32_t bound = 0;
    const uint32_t most = value_key(m);
    int turn = 0;
    const auto reached = [&](uint32_t from) -> int {
        if constexpr (!FEW) return __syncthreads_count(mine >= from);
        const int n = __reduce_add_sync(~0u, __popcll(reach<T>(d, part.used(0), from)) + (edge && value_key(xe) >= from));
        if (g.lane == 0) top.part[turn][g.warp] = n;
        __syncthreads();
        int all = 0;
#pragma unroll
        for (int w = 0; w < G::W; ++w) all += top.part[turn][w];
        turn ^= 1;
        return all;
    };
    if (!cluster && P.k > G::W) {
        // the k-th largest of the threads' maxima, or of the tokens: its upper 16
        // bits from above, as far as more than a few above k reach them
        for (uint32_t bit = 0x80000000u; bit > 0x8000u; bit >>= 1) {
            if ((bound | bit) > most) continue;
            const int n = reached(bound | bit);
            if (n >= P.k) bound |= bit;
            if (n >= P.k && n <= P.k + (P.k >> 3) + 2) break;
        }
    } else {
        // the warps' value with top_before before it: each warp counts for one of each CTA
        uint32_t all[(CLUSTER_MAX * G::W + 31) / 32];
#pragma unroll
        for (int q = 0; q < (CLUSTER_MAX * G::W + 31) / 32; ++q)
            all[q] = g.lane + 32 * q < warps ? __float_as_uint(slots[g.lane + 32 * q].w) : 0u;
#pragma unroll
        for (int r = 0; r < CLUSTER_MAX; ++r) {
            if (r < g.parts) {
                const int i = r * G::W + g.warp;
                const uint32_t v = __float_as_uint(slots[i].w);
                unsigned int n = 0;
#pragma unroll
                for (int q = 0; q < (CLUSTER_MAX * G::W + 31) / 32; ++q) n += all[q] > v || (all[q] == v && g.lane + 32 * q < i);
                if (__reduce_add_sync(~0u, n) == static_cast<unsigned int>(P.top_before) && g.lane == 0) top.bound = v;
            }
        }
        __syncthreads();
        bound = top.bound;
    }
    const unsigned int share = CAND_MAX >> (31 - __clz(g.parts));   // clusters are powers of two
    const uint32_t list = cluster ? mapa_shared(smem_u32(top.found + g.rank * share), 0) : 0;
    const auto take = [&](int id) {
        const unsigned int at = atomicAdd(&top.local, 1u);
        if (at < share) {
            if (cluster) st_shared_cluster_u32(list + 4 * at, id);
            else top.found[at] = id;
        }
    };
    // a bound of -inf: what lies above it, then the first of the -inf tokens
    bool above = bound <= KEY_NEG_INF;
    bound = max(bound, KEY_NEG_INF);
    for (;;) {
        const uint32_t from = above ? next_key<T>(bound) : bound;
        if (mine >= from && from >= KEY_NEG_INF) {   // (0: nothing lies above a NaN)
            // each thread the tile of its largest, that of its second, rarely all others
            int next = 0;
            for (int i = 0, t = tile;; ++i) {
                if (part.tiles > 1) part.reload(row, g, t, d);
                unsigned long long bits = reach<T>(d, NV, from);
                while (bits) {
                    const int b = Elem<T>::place(__ffsll(bits) - 1);
                    bits &= bits - 1;
                    if (b / E * GT < part.left(g, t)) take(row.head + (part.at(g, t) + b / E * GT) * E + b % E);
                }
                if (i == 0) {
                    if (second < from) break;
                    t = tile2;
                } else {
                    if (third < from) break;
                    while (next == tile || next == tile2) ++next;
                    if (next >= part.tiles) break;
                    t = next++;
                }
            }
        }
        if (edge && value_key(xe) >= from && from >= KEY_NEG_INF) take(row.edge(g.lane));
        __syncthreads();
        if (cluster || above || top.local <= CAND_MAX) break;
        // many tie: the whole bound, what lies above it, and the lowest ids at it
        for (uint32_t bit = 0x80000000u; bit; bit >>= 1)
            if (!(bound & bit) && (bound | bit) <= most && reached(bound | bit) >= P.k) bound |= bit;
        __syncthreads();
        if (g.tid == 0) top.local = 0;
        __syncthreads();
        above = true;
    }
    if (cluster) {
        if (g.tid == 0) st_shared_cluster_u32(mapa_shared(smem_u32(top.counts + g.rank), 0), top.local);
        cluster_sync();
        if (g.rank != 0) return;
        count = 0;
        for (int r = 0; r < g.parts; ++r) count = top.counts[r] > share ? 2 * CAND_MAX : count + top.counts[r];
    } else {
        count = top.local;
    }
    const auto put = [&](unsigned int at, float x, int id) {
        if (narrow) key32[at] = narrow_key(x, id);
        else top.key[at] = token_key(x, id);
    };
    narrow = sizeof(T) == 2 && P.vocab <= 65536 && max(count, static_cast<unsigned int>(P.k)) <= RANK_MAX;
    if (count <= CAND_MAX) {
        for (unsigned int c = g.tid; c < count; c += GT) {
            unsigned int at = c;
            for (int r = 0; cluster && r < g.parts - 1 && at >= r * share + top.counts[r]; ++r) at += share - top.counts[r];
            const int id = top.found[at];
            put(c, Elem<T>::get(row.p + id), id);
        }
    }
    if (count < static_cast<unsigned int>(P.k) && g.warp == 0) {
        // fewer than k tokens lie above the bound: the lowest ids of those at it follow
        unsigned int n = count;
        for (int id = g.lane; n < static_cast<unsigned int>(P.k) && id - g.lane < P.vocab; id += 32) {
            const float x = id < P.vocab ? Elem<T>::get(row.p + id) : 0.f;
            const bool at_bound = id < P.vocab && same_key<T>(value_key(x), bound);
            const unsigned int set = __ballot_sync(~0u, at_bound);
            const unsigned int at = n + __popc(set & ((1u << g.lane) - 1));
            if (at_bound && at < static_cast<unsigned int>(P.k)) put(at, x, id);
            n += __popc(set);
        }
    }
    count = max(count, static_cast<unsigned int>(P.k));
    // zeros after the last key
    if (count <= CAND_MAX - 4 && g.tid < 4) {
        if (narrow) key32[count + g.tid] = 0;
        else top.key[count + g.tid] = 0;
    }
    __syncthreads();
    if (count > CAND_MAX) {
        top_radix<T, GT>(row.p, P.vocab, P.k, top);
        count = top.count;
    }
    const auto give = [&](auto key, unsigned int place) {
        P.top_ids[g.row * P.k + place] = key_id(key);
        P.top_logp[g.row * P.k + place] = (key_logit(key) - m0) * P.c - logs;
    };
    const int n = count <= 2 ? static_cast<int>(count) : 1 << (32 - __clz(count - 1));
    // counting takes count^2 / 32 steps of all warps together, sorting 45 to 55 barriers
    if (count <= RANK_MAX) {
        // `share` neighbouring threads count for one candidate
        const int log_share = n <= GT ? min(5, __clz(n) - __clz(GT)) : 0;
        const unsigned int share = 1u << log_share, first = g.tid & (share - 1);
        const auto rank = [&](const auto* keys) {
            for (unsigned int c0 = g.warp * 32u >> log_share; c0 < count; c0 += GT) {   // the warp has candidates
                const unsigned int c = c0 + (g.lane >> log_share);
                const auto key = keys[min(c, count - 1)];
                unsigned int before = count_above(keys, count, key, first, share);
                for (unsigned int i = share / 2; i; i /= 2) before += __shfl_xor_sync(~0u, before, i);
                if (c < count && first == 0 && before < static_cast<unsigned int>(P.k)) give(key, before);
            }
        };
        if (narrow) rank(key32);
        else rank(top.key);
    } else {
        for (int i = count + g.tid; i < n; i += GT) top.key[i] = 0;
        sort_block<GT>(top.key, n);
        for (int i = g.tid; i < P.k; i += GT) give(top.key[i], i);
    }
}

// Sorts 32 R keys falling in one warp: key r 32 + lane in register r.
template <class K, int R>
__device__ __forceinline__ void sort_warp(K (&key)[R], int lane)
{
#pragma unroll
    for (int size = 2; size <= 32 * R; size *= 2) {
#pragma unroll
        for (int step = size / 2; step; step /= 2) {
            if (step >= 32) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const int o = r ^ step / 32;
                    if (o > r) {
                        const bool falling = (r * 32 & size) == 0;
                        const K a = key[r], b = key[o];
                        key[r] = falling ? max(a, b) : min(a, b);
                        key[o] = falling ? min(a, b) : max(a, b);
                    }
                }
            } else {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const K o = __shfl_xor_sync(~0u, key[r], step);
                    const int i = r * 32 + lane;
                    const bool larger = ((i & size) == 0) == ((i & step) == 0);   // this lane keeps the larger
                    key[r] = larger ? max(key[r], o) : min(key[r], o);
                }
            }
        }
    }
}

template <class T>
struct WarpKey {
    using K = unsigned long long;
    __device__ static K make(float x, int j) { return token_key(x, j); }
};
template <>
struct WarpKey<__nv_bfloat16> {
    using K = uint32_t;   // rows of a warp have fewer than 2^16 tokens
    __device__ static K make(float x, int j) { return narrow_key(x, j); }
};

// The same for rows that one warp holds: the bound is the k-th largest of the
// lanes' maxima where these are enough (k <= 16), else of the tokens themselves,
// counted by their bits; candidates are gathered and sorted within the warp.
template <class T, bool ENT>
__global__ void __launch_bounds__(128, 6) token_logprob_top_warp_kernel(const VocabParams P)
{
    constexpr int E = Elem<T>::E, CAND = VOCAB_MAX_K;
    using G = Group<32>;
    using K = typename WarpKey<T>::K;
    __shared__ K keys[G::ROWS][CAND];
    __shared__ int ids[G::ROWS][CAND];
    const G g;
    if (g.row >= P.n) return;
    const int lane = g.lane;
    const Row<T> row(static_cast<const T*>(P.logits) + g.row * P.ld, P.vocab);
    const Part<T, 32> part(row, g, P.each);
    uint4 d[NV];
    part.load(row, g, 0, d);
    const bool edge = lane < row.edges();
    const float xe = edge ? Elem<T>::get(row.p + row.edge(lane)) : NEG_INF;
    const long long y = P.targets ? P.targets[g.row] : -1;
    const bool there = y >= 0 && y < P.vocab;
    const float xy = there ? Elem<T>::get(row.p + y) : 0.f;
    const int used = part.used(0);
    const float mt = Elem<T>::max_of(d);
    Acc a = acc_tile<T, ENT>(d, used, mt, P.c2);
    if (row.edges() > 0) a = acc_merge<ENT>(a, acc_one(xe), P.c2);
    a = acc_warp<ENT>(a, P.c2);
    const float m = a.m, m0 = m == NEG_INF ? 0.f : m, logs = m == NEG_INF ? 0.f : logf(a.s);
    if (lane == 0) {
        const float H = ENT && m != NEG_INF ? logs - LN2 * (a.t / a.s) : 0.f;
        if (P.logp) P.logp[g.row] = there ? (xy - m0) * P.c - logs : 0.f;
        if (ENT && P.entropy) P.entropy[g.row] = H;
        if (P.stats) reinterpret_cast<float4*>(P.stats)[g.row] = make_float4(m, logs, H, 0.f);
    }
    const uint32_t most = value_key(m);
    const auto reached = [&](uint32_t from) -> int {
        return __reduce_add_sync(~0u, __popcll(reach<T>(d, used, from)) + (edge && value_key(xe) >= from));
    };
    const auto gather = [&](uint32_t from) -> int {
        unsigned long long bits = reach<T>(d, used, from);
        bool also = edge && value_key(xe) >= from;
        int count = 0;
        while (__any_sync(~0u, bits != 0 || also)) {
            int id = -1;
            if (bits) {
                const int b = Elem<T>::place(__ffsll(bits) - 1);
                bits &= bits - 1;
                if (b / E * 32 < part.left(g, 0)) id = row.head + (part.at(g, 0) + b / E * 32) * E + b % E;
            } else if (also) {
                also = false;
                id = row.edge(lane);
            }
            const unsigned int set = __ballot_sync(~0u, id >= 0);
            const int at = count + __popc(set & ((1u << lane) - 1));
            if (id >= 0 && at < CAND) ids[g.slot][at] = id;
            count += __popc(set);
        }
        return count;
    };
    uint32_t bound = 0;
    if (P.k <= 16) {
        uint32_t best[1] = {max(value_key(mt), value_key(xe))};
        sort_warp(best, lane);
        bound = __shfl_sync(~0u, best[0], P.k - 1);
    } else {
        for (uint32_t bit = 0x80000000u; bit > 0x8000u; bit >>= 1) {
            if ((bound | bit) > most) continue;
            const int n = reached(bound | bit);
            if (n >= P.k) bound |= bit;
            if (n >= P.k && n <= min(P.k + (P.k >> 3) + 2, CAND)) break;
        }
    }
    // a bound of -inf: what lies above it, then the first of the -inf tokens
    int count = gather(bound <= KEY_NEG_INF ? next_key<T>(KEY_NEG_INF) : bound);
    bound = max(bound, KEY_NEG_INF);
    if (count > CAND) {
        // many tie: the k-th largest itself, fewer than k above it, and the lowest ids at it
        bound = 0;
        for (uint32_t bit = 0x80000000u; bit; bit >>= 1)
            if ((bound | bit) <= most && reached(bound | bit) >= P.k) bound |= bit;
        count = bound == 0xffffffffu ? 0 : gather(next_key<T>(bound));   // (nothing lies above a NaN)
    }
    __syncwarp();
    for (int i = lane; i < count; i += 32)
        keys[g.slot][i] = WarpKey<T>::make(Elem<T>::get(row.p + ids[g.slot][i]), ids[g.slot][i]);
    for (int j0 = 0; count < P.k && j0 < P.vocab; j0 += 32) {
        const int j = j0 + lane;
        const float x = j < P.vocab ? Elem<T>::get(row.p + j) : 0.f;
        const bool at_bound = j < P.vocab && same_key<T>(value_key(x), bound);
        const unsigned int set = __ballot_sync(~0u, at_bound);
        const int at = count + __popc(set & ((1u << lane) - 1));
        if (at_bound && at < P.k) keys[g.slot][at] = WarpKey<T>::make(x, j);
        count = min(count + __popc(set), P.k);
    }
    __syncwarp();
    const auto sorted = [&](auto& key) {
        constexpr int R = sizeof(key) / sizeof(key[0]);
#pragma unroll
        for (int i = 0; i < R; ++i) key[i] = i * 32 + lane < count ? keys[g.slot][i * 32 + lane] : K(0);
        sort_warp(key, lane);
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int place = i * 32 + lane;
            if (place < P.k) {
                P.top_ids[g.row * P.k + place] = key_id(key[i]);
                P.top_logp[g.row * P.k + place] = (key_logit(key[i]) - m0) * P.c - logs;
            }
        }
    };
    if (count <= 32) {
        K key[1];
        sorted(key);
    } else if (count <= 128) {
        K key[4];
        sorted(key);
    } else {
        K key[8];
        sorted(key);
    }
}

}  // namespace cola
