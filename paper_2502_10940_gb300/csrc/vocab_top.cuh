// vocab_top.cuh -- log probabilities with the row's most likely tokens.
#pragma once
#include <type_traits>

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

// By one warp: the key of the k-th largest of 1024 maxima, of which each word holds
// the upper halves of two, cut where no more than a few above k reach it; at most that
// of +inf, and that of -inf where fewer than k are above it.
__device__ __forceinline__ uint32_t search_bound(const uint4* halves, int k, int lane)
{
    uint32_t least = ~0u, most = 0;
    int n = 0;
    const auto each = [&](auto f) {
        asm volatile("" ::: "memory");   // (read again each time: the caller's registers are full)
#pragma unroll 2
        for (int i = 0; i < 4; ++i) {
            const uint4 h = halves[lane + i * 32];
            f(h.x), f(h.y), f(h.z), f(h.w);
        }
    };
    each([&](uint32_t w) {
        for (uint32_t half : {w << 16, w & 0xffff0000u}) {
            const uint32_t key = min(value_key(__uint_as_float(half)), KEY_POS_INF) & 0xffff0000u;
            most = max(most, key);
            if (key > KEY_NEG_INF) least = min(least, key), ++n;
        }
    });
    if (__reduce_add_sync(~0u, n) < k) return KEY_NEG_INF;
    least = __reduce_min_sync(~0u, least), most = __reduce_max_sync(~0u, most);
    // they agree in the bits above the first that differs
    const int agree = __clz(least ^ most);
    uint32_t bound = agree >= 16 ? least : least & ~(0xffffffffu >> agree);
    for (uint32_t bit = agree >= 16 ? 0 : 0x80000000u >> agree; bit > 0x8000u; bit >>= 1) {
        if ((bound | bit) > most) continue;   // (beyond +inf lie NaNs' patterns, which every maximum would reach)
        const uint32_t from = __float_as_uint(key_value(bound | bit)) >> 16, both = from << 16 | from;
        __nv_bfloat162 reach = __floats2bfloat162_rn(0.f, 0.f);   // (counts to 16: exact)
        each([&](uint32_t w) {
            reach = __hadd2(reach, __hgeu2(*reinterpret_cast<const __nv_bfloat162*>(&w),
                                           *reinterpret_cast<const __nv_bfloat162*>(&both)));
        });
        n = __reduce_add_sync(~0u, static_cast<int>(__low2float(reach) + __high2float(reach)));
        if (n >= k) bound |= bit;
        if (n >= k && n <= k + (k >> 3) + 2) break;
    }
    return bound;
}

// The candidates of a row's top k, in the first of its CTAs.
struct TopShared {
    alignas(16) unsigned long long key[CAND_MAX];
    int found[CAND_MAX];                  // ids; a share for each CTA of the row
    unsigned int hist[256];
    unsigned int counts[CLUSTER_MAX];
    unsigned int count, digit, above, bound, local;
    unsigned int part[2][16];           // counts of the warps, in turn
    float max, log_sum;
};

constexpr unsigned int RANK_MAX = 512;   // candidates that are sorted in runs of a warp's lanes

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

// How many of 32 keys, falling, are above `key`.
template <class K>
__device__ __forceinline__ unsigned int above_in(const K* keys, K key)
{
    unsigned int n = 0;
#pragma unroll
    for (unsigned int step = 16; step; step /= 2) n += keys[n + step - 1] > key ? step : 0;
    return n + (keys[n] > key);
}

// The forward with the k most likely tokens.  At least k tokens reach the k-th
// largest of the threads' maxima, and few more than k do where the largest are
// spread over the threads (74 at k = 64 of 32000 in random order, 256 threads).
// FEW: k is more than half of the threads, whose registers hold the row; the bound
// is that of eight maxima of each thread, which one warp searches, or, where the row
// has fewer than 1.5 k vectors, of the tokens themselves, counted by their bits.
// In a cluster, whose threads are too many and too far apart for that, each warp
// gives with its statistics the `each`-th largest of its threads' maxima, and at
// least k tokens reach the ceil(k / each)-th largest of those.  The tokens that
// reach the bound are gathered, by their bits, from the registers (of rows of more
// than a tile, read again).  Warps sort them in runs of 32, and a token's place is that in
// its run and the number before it in each of the others.
// One pass of HBM, which the bound, the gather and the ranking follow in each row:
// what overlaps them is the other rows of the SM.  4096 x 32000 fp32, k = 1: 84 us,
// 6.2 TB/s; 8192 x 32000 bf16, k = 64: 116 us, 4.6 TB/s, where each row takes 11,600
// instructions; 32768 x 5000 bf16: 150 us at k = 20, 234 us at k = 100.
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
    if (FEW)
        reinterpret_cast<uint4*>(top.key)[g.tid] = make_uint4(Elem<T>::halves(d[0], d[1]), Elem<T>::halves(d[2], d[3]),
                                                              Elem<T>::halves(d[4], d[5]), Elem<T>::halves(d[6], d[7]));
    exchange(a, __uint_as_float(best), g, slots);
    float m = 0.f, logs = 0.f;
    uint32_t bound = 0;
    // whether k is too near the vectors' number for their maxima to tell a bound
    const bool tokens = FEW && 3 * P.k > 2 * row.full;
    if (!FEW || g.warp == 0) {
        a = acc_slots<GT, ENT>(slots, warps, g, P.c2);
        m = a.m, logs = m == NEG_INF ? 0.f : logf(a.s);
        if (g.rank == 0 && g.tid == 0) {
            const float H = ENT && m != NEG_INF ? logs - LN2 * (a.t / a.s) : 0.f;
            if (P.logp) P.logp[g.row] = there ? (xy - (m == NEG_INF ? 0.f : m)) * P.c - logs : 0.f;
            if (ENT && P.entropy) P.entropy[g.row] = H;
            if (P.stats) reinterpret_cast<float4*>(P.stats)[g.row] = make_float4(m, logs, H, 0.f);
        }
    }
    if (FEW) {
        if (g.warp == 0) {
            if (!tokens) bound = search_bound(reinterpret_cast<const uint4*>(top.key), P.k, g.lane);
            if (g.lane == 0) top.bound = bound, top.max = m, top.log_sum = logs;
        }
        __syncthreads();
        bound = top.bound, m = top.max, logs = top.log_sum;
    }
    const float m0 = m == NEG_INF ? 0.f : m;
    unsigned int count = 0;
    bool narrow = false;
    uint32_t* key32 = reinterpret_cast<uint32_t*>(top.key);
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
    if (FEW ? tokens : !cluster && P.k > G::W) {
        // the k-th largest of the threads' maxima, or of the tokens: its upper 16
        // bits from above, as far as more than a few above k reach them
        for (uint32_t bit = 0x80000000u; bit > 0x8000u; bit >>= 1) {
            if ((bound | bit) > most) continue;
            const int n = reached(bound | bit);
            if (n >= P.k) bound |= bit;
            if (n >= P.k && n <= P.k + (P.k >> 3) + 2) break;
        }
    } else if (!FEW) {
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
    // (clusters are powers of two; a row of which one CTA has more than its share goes to the radix search
    // of one CTA: 1 x 128000, k = 20, of rising logits or with ids 0..999 alone allowed, 230 us against 6.3)
    const unsigned int share = CAND_MAX >> (31 - __clz(g.parts));
    const uint32_t list = cluster ? mapa_shared(smem_u32(top.found + g.rank * share), 0) : 0;
    const auto place = [&](unsigned int at, int id) {
        if (at < share) {
            if (cluster) st_shared_cluster_u32(list + 4 * at, id);
            else top.found[at] = id;
        }
    };
    const auto take = [&](int id) { place(atomicAdd(&top.local, 1u), id); };
    // a bound of -inf: what lies above it, then the first of the -inf tokens
    bool above = bound <= KEY_NEG_INF;
    bound = max(bound, KEY_NEG_INF);
    for (;;) {
        const uint32_t from = above ? next_key<T>(bound) : bound;
        if (mine >= from && from >= KEY_NEG_INF) {   // (0: nothing lies above a NaN)
            if (FEW || part.tiles == 1) {
                unsigned long long bits = reach<T>(d, part.used(0), from);
                unsigned int at = atomicAdd(&top.local, static_cast<unsigned int>(__popcll(bits)));
                const int id = row.head + part.at(g, 0) * E;
                while (bits) {
                    const int b = Elem<T>::place(__ffsll(bits) - 1);
                    bits &= bits - 1;
                    place(at++, id + b / E * (GT * E) + b % E);
                }
            } else {
                // each thread the tile of its largest, that of its second, rarely all others
                int next = 0;
                for (int i = 0, t = tile;; ++i) {
                    part.reload(row, g, t, d);
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
        }
        if (edge && value_key(xe) >= from && from >= KEY_NEG_INF) take(row.edge(g.lane));
        __syncthreads();
        if (cluster || above || top.local <= CAND_MAX) break;
        // many tie: the whole bound, what lies above it, and the lowest ids at it
        bound = 0;
        for (uint32_t bit = 0x80000000u; bit; bit >>= 1)
            if ((bound | bit) <= most && reached(bound | bit) >= P.k) bound |= bit;
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
    __syncthreads();
    if (count > CAND_MAX) {
        top_radix<T, GT>(row.p, P.vocab, P.k, top);
        count = top.count;
    }
    const auto give = [&](auto key, unsigned int place) {
        P.top_ids[g.row * P.k + place] = key_id(key);
        P.top_logp[g.row * P.k + place] = (key_logit(key) - m0) * P.c - logs;
    };
    if (count <= RANK_MAX) {
        // each run of 32 sorted by a warp; a key's place is that in its run and the number above it in each other
        const auto rank = [&](auto* keys) {
            using K = typename std::remove_reference<decltype(*keys)>::type;
            if (count <= 32) {
                if (g.warp != 0) return;
                const K key = g.lane < count ? keys[g.lane] : K(0);
                unsigned int before = 0;
#pragma unroll 4
                for (unsigned int i = 0; i < count; ++i) before += __shfl_sync(~0u, key, i) > key;
                if (g.lane < count && before < static_cast<unsigned int>(P.k)) give(key, before);
                return;
            }
            for (unsigned int c = g.tid; c < (count + 31) / 32 * 32; c += GT) {
                K key[1] = {c < count ? keys[c] : K(0)};
                sort_warp(key, g.lane);
                keys[c] = key[0];
            }
            __syncthreads();
            for (unsigned int c = g.tid; c < count; c += GT) {
                const K key = keys[c];
                unsigned int before = c & 31;
#pragma unroll 4
                for (unsigned int r = 0; r < count; r += 32)
                    if (r != (c & ~31u)) before += above_in(keys + r, key);
                if (before < static_cast<unsigned int>(P.k)) give(key, before);
            }
        };
        if (narrow) rank(key32);
        else rank(top.key);
    } else {
        const int n = 1 << (32 - __clz(count - 1));
        for (int i = count + g.tid; i < n; i += GT) top.key[i] = 0;
        sort_block<GT>(top.key, n);
        for (int i = g.tid; i < P.k; i += GT) give(top.key[i], i);
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
// lanes' maxima where these are enough (k <= 16), of the vectors' where there are
// half as many again as k, else of the tokens themselves, counted by their bits;
// candidates are gathered and sorted within the warp.  Chains of shuffles and votes
// bound it, so as many warps as 64 registers allow (65 us against 76 us for the top 5
// of 65536 x 2000 bf16; the top 40: 104 us).
template <class T, bool ENT>
__global__ void __launch_bounds__(Group<32>::THREADS, Group<32>::CTAS) token_logprob_top_warp_kernel(const VocabParams P)
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
    } else if (3 * P.k <= 2 * row.full) {
        uint32_t v[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) v[j] = value_key(Elem<T>::largest(d[j]));
        const uint32_t ve = edge ? value_key(xe) : 0;
        for (uint32_t bit = 0x80000000u; bit > 0x8000u; bit >>= 1) {
            const uint32_t from = bound | bit;
            if (from > most) continue;
            int n = ve >= from;
#pragma unroll
            for (int j = 0; j < NV; ++j) n += v[j] >= from;
            n = __reduce_add_sync(~0u, n);
            if (n >= P.k) bound = from;
            if (n >= P.k && n <= P.k + (P.k >> 3) + 2) break;
        }
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
    } else if (count <= 64) {
        K key[2];
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
