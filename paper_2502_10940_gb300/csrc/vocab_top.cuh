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
__device__ __forceinline__ uint32_t narrow_key(float x, int j) { return (value_key(x) & 0xffff0000u) | (0xffffu - static_cast<uint32_t>(j)); }

__device__ __forceinline__ int key_id(unsigned long long key) { return static_cast<int>(0xffffffffu - static_cast<uint32_t>(key)); }
__device__ __forceinline__ int key_id(uint32_t key) { return static_cast<int>(0xffffu - (key & 0xffffu)); }
__device__ __forceinline__ float key_logit(unsigned long long key) { return key_value(static_cast<uint32_t>(key >> 32)); }
__device__ __forceinline__ float key_logit(uint32_t key) { return key_value(key & 0x80000000u ? key & 0xffff0000u : key | 0xffffu); }

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
    bool narrow = false;
    uint32_t* key32 = reinterpret_cast<uint32_t*>(top.key);
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
        if (mine >= bound) {   // each thread the tile of its largest, that of its second, rarely all others
            if (part.tiles > 1) part.reload(row, g, tile, d);
            take_tile(tile);
            if (second >= bound) {
                part.reload(row, g, tile2, d);
                take_tile(tile2);
                for (int t = 0; third >= bound && t < part.tiles; ++t) {
                    if (t == tile || t == tile2) continue;
                    part.reload(row, g, t, d);
                    take_tile(t);
                }
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
        const auto put = [&](unsigned int at, float x, int id) {
            if (narrow) key32[at] = narrow_key(x, id);
            else top.key[at] = token_key(x, id);
        };
        narrow = sizeof(T) == 2 && P.vocab <= 65536 && count <= 128;
        if (count <= CAND_MAX) {
            for (unsigned int c = g.tid; c < count; c += GT) {
                unsigned int at = c;
                for (int r = 0; cluster && r < g.parts - 1 && at >= r * share + top.counts[r]; ++r) at += share - top.counts[r];
                const int id = top.found[at];
                put(c, Elem<T>::get(row.p + id), id);
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
                if (none && at < static_cast<unsigned int>(P.k)) put(at, NEG_INF, id);
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
    } else if (g.rank != 0) {
        return;
    }
    if (count > CAND_MAX) {
        top_radix<T, GT>(row.p, P.vocab, P.k, top);
        count = top.count;
    }
    const auto give = [&](auto key, unsigned int place) {
        P.top_ids[g.row * P.k + place] = key_id(key);
        P.top_logp[g.row * P.k + place] = (key_logit(key) - m0) * P.c - logs;
    };
    const int n = count <= 2 ? static_cast<int>(count) : 1 << (32 - __clz(count - 1));
    // counting takes count^2 / 32 steps of all warps together, sorting 30 to 55 barriers
    if (n <= min(GT, 256)) {
        // `share` neighbouring threads count for one candidate
        const int log_share = min(5, __clz(n) - __clz(GT));
        const unsigned int share = 1u << log_share, c = g.tid >> log_share, first = g.tid & (share - 1);
        if (g.warp * 32u >> log_share < count) {   // the warp has candidates
            const auto rank = [&](const auto* keys) {
                const auto key = keys[min(c, count - 1)];
                unsigned int before = count_above(keys, count, key, first, share);
                for (unsigned int i = share / 2; i; i /= 2) before += __shfl_xor_sync(~0u, before, i);
                if (c < count && first == 0 && before < static_cast<unsigned int>(P.k)) give(key, before);
            };
            if (narrow) rank(key32);
            else rank(top.key);
        }
    } else {
        for (int i = count + g.tid; i < n; i += GT) top.key[i] = 0;
        sort_block<GT>(top.key, n);
        for (int i = g.tid; i < P.k; i += GT) give(top.key[i], i);
    }
}

}  // namespace cola
