// Kernels of the token embedding (embed.cuh) and their launchers.
#include "embed.cuh"

#include <algorithm>
#include <atomic>

#include "vocab_rows.cuh"

namespace cola {
namespace {

// ------------------------------------------------- eight columns of a row
// Pitches are multiples of 8 elements, so that every eight columns begin on a
// 16-byte boundary; the last of a row may be fewer.
template <class T>
struct Eight;

template <>
struct Eight<__nv_bfloat16> {
    uint4 u;
    __device__ __forceinline__ void load(const __nv_bfloat16* p, int left)
    {
        if (left >= 8) {
            u = *reinterpret_cast<const uint4*>(p);
        } else {
            float x[8] = {};
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (i < left) x[i] = __bfloat162float(p[i]);
            u = Elem<__nv_bfloat16>::pack(x);
        }
    }
    __device__ __forceinline__ void values(float (&x)[8]) const { Elem<__nv_bfloat16>::unpack(u, x); }
    __device__ __forceinline__ static void store(__nv_bfloat16* p, const float (&x)[8], int left)
    {
        if (left >= 8) {
            *reinterpret_cast<uint4*>(p) = Elem<__nv_bfloat16>::pack(x);
        } else {
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (i < left) p[i] = __float2bfloat16_rn(x[i]);
        }
    }
};

template <>
struct Eight<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float* p, int left)
    {
        if (left >= 8) {
            a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
        } else {
            float x[8] = {};
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (i < left) x[i] = p[i];
            a = make_float4(x[0], x[1], x[2], x[3]), b = make_float4(x[4], x[5], x[6], x[7]);
        }
    }
    __device__ __forceinline__ void values(float (&x)[8]) const
    {
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    }
    __device__ __forceinline__ static void store(float* p, const float (&x)[8], int left)
    {
        if (left >= 8) {
            reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
            reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
        } else {
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (i < left) p[i] = x[i];
        }
    }
};

// ------------------------------------------------------------------ lookup
// UNITS pieces of eight columns a thread, 256 apart in the rows laid end to end:
// their ids and then their rows are loaded together.
template <class TE, class TX, int UNITS>
__global__ void __launch_bounds__(256) embed_rows_kernel(const EmbedParams P)
{
    const unsigned int units = (P.d + 7) / 8;
    const long long first = blockIdx.x * (256ll * UNITS), t0 = first / units;
    const unsigned int c0 = static_cast<unsigned int>(first - t0 * units) + threadIdx.x;
    long long id[UNITS];
    Eight<TE> e[UNITS];
    const auto row = [&](int u) { return t0 + (c0 + u * 256) / units; };
    const auto col = [&](int u) { return static_cast<int>((c0 + u * 256) % units) * 8; };
#pragma unroll
    for (int u = 0; u < UNITS; ++u) id[u] = row(u) < P.n ? P.ids[row(u)] : -1;
#pragma unroll
    for (int u = 0; u < UNITS; ++u)
        if (id[u] >= 0 && id[u] < P.vocab) e[u].load(static_cast<const TE*>(P.src) + id[u] * P.ld_src + col(u), P.d - col(u));
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        if (row(u) >= P.n) break;
        float x[8] = {};
        if (id[u] >= 0 && id[u] < P.vocab) {
            e[u].values(x);
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] *= P.scale;
        }
        Eight<TX>::store(static_cast<TX*>(P.dst) + row(u) * P.ld_dst + col(u), x, P.d - col(u));
    }
}

// ------------------------------------------------------------- rows of no token
// Rows [first, last) of the gradient := 0 but for those that `named` tells, by the
// warps of `ctas` CTAs of which this is number `cta`.
template <class TD, class F>
__device__ __forceinline__ void fill_rows(const EmbedParams& P, int first, int last, int cta, int ctas, const F& named)
{
    const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    const float zero[8] = {};
    for (int v = first + cta * warps + (threadIdx.x >> 5); v < last; v += ctas * warps)
        if (!named(v))
            for (int c = lane * 8; c < P.d; c += 256) Eight<TD>::store(static_cast<TD*>(P.dst) + v * P.ld_dst + c, zero, P.d - c);
}

// ------------------------------------------------------- few tokens by counting
constexpr unsigned int NO_KEY = ~0u;

__device__ __forceinline__ unsigned int key_of(long long id, int vocab)
{
    return id >= 0 && id < vocab ? static_cast<unsigned int>(id) : NO_KEY;
}

// A token's place is the number of tokens before it: of lower ids, or of its own id
// and earlier.  Every CTA reads all ids; its eight warps count for 32 tokens, each
// over an eighth of the ids.  Every CTA also has a share of the table's rows, and
// sets those to 0 that no id names (TD, where `filled`).
template <class TD>
__global__ void __launch_bounds__(256) embed_order_kernel(const EmbedParams P, int order_ctas, int rows_each)
{
    extern __shared__ __align__(16) unsigned int keys[];   // n of them up to a multiple of 256, then a bit for each of this CTA's rows
    __shared__ unsigned int count[8][32];
    __shared__ unsigned int valid;
    const int n = static_cast<int>(P.n), tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, all = (n + 255) / 256 * 256;
    unsigned int* named = keys + all;
    const int first = min(P.vocab, static_cast<int>(blockIdx.x) * rows_each), last = min(P.vocab, first + rows_each);
    for (int i = tid; i < (rows_each + 31) / 32; i += 256) named[i] = 0;
    if (tid == 0) valid = 0;
    __syncthreads();
    unsigned int mine = 0;
#pragma unroll 8
    for (int i = tid; i < all; i += 256) {
        const unsigned int key = i < n ? key_of(P.ids[i], P.vocab) : NO_KEY;
        keys[i] = key;
        mine += key != NO_KEY;
        if (key != NO_KEY && key >= first && key < last) atomicOr(named + ((key - first) >> 5), 1u << ((key - first) & 31));
    }
    if (blockIdx.x == 0) atomicAdd(&valid, mine);
    __syncthreads();
    if (blockIdx.x == 0 && tid == 0) *P.count = valid, *P.long_count = 0;
    if (static_cast<int>(blockIdx.x) < order_ctas) {
        const int i0 = blockIdx.x * 32, eighth = all / 8, from = warp * eighth, to = from + eighth;
        const unsigned int key = i0 + lane < n ? keys[i0 + lane] : NO_KEY;
        unsigned int sum = 0;
        const auto below = [&](int lo, int hi, unsigned int bound) {
#pragma unroll 4
            for (int j = lo; j < hi; j += 4) {
                const uint4 k = *reinterpret_cast<const uint4*>(keys + j);
                sum += (k.x < bound) + (k.y < bound) + (k.z < bound) + (k.w < bound);
            }
        };
        below(from, min(to, i0), key + 1);
        below(max(from, i0 + 32), to, key);
        if (i0 >= from && i0 < to)
            for (int j = 0; j < 32; ++j) sum += keys[i0 + j] < key + (j < lane);
        count[warp][lane] = sum;
        __syncthreads();
        if (warp == 0 && key != NO_KEY) {
            for (int w = 1; w < 8; ++w) sum += count[w][lane];
            P.sorted[sum] = make_uint2(key, i0 + lane);
        }
    }
    if (rows_each) fill_rows<TD>(P, first, last, 0, 1, [&](int v) { return named[(v - first) >> 5] >> ((v - first) & 31) & 1; });
}

// --------------------------------------------------------- many tokens by digits
// One or two passes of a stable counting sort by up to ten bits, each in two
// launches.  Every CTA has consecutive tokens; the first counts its digits, the
// second ranks them: every warp has consecutive ones of the CTA's, 32 a round, and
// ranks each round's among those of their digit; counts become first places, over
// the digits, the CTAs and the warps.
constexpr int SORT_THREADS = 1024, SORT_WARPS = 32;
constexpr int ROUNDS = 8;                   // whose tokens a warp holds at once
constexpr int KEY_BITS = 20;                // a held token: its rank in its warp above its key

struct SortPass {
    const uint2* from;        // nullptr: the ids (those that name no token are left out)
    uint2* to;
    unsigned int* hist;       // [CTA][digit]
    int shift, bits, ctas;
    unsigned int each;        // tokens of a warp, a multiple of 32
    int fill_first, fill_last, fill_ctas;   // rows that CTAs behind the others set to 0 where no token names them
};

// A batch of a warp's tokens: NO_KEY where there is none.
template <bool FIRST>
__device__ __forceinline__ void sort_load(const EmbedParams& P, const SortPass& S, unsigned int i, unsigned int end,
                                          unsigned int (&key)[ROUNDS], unsigned int (&token)[ROUNDS])
{
#pragma unroll
    for (int j = 0; j < ROUNDS; ++j) {
        key[j] = NO_KEY, token[j] = i + j * 32;
        if (i + j * 32 >= end) continue;
        if (FIRST) {
            key[j] = key_of(P.ids[i + j * 32], P.vocab);
        } else {
            const uint2 item = S.from[i + j * 32];
            key[j] = item.x, token[j] = item.y;
        }
    }
}

template <class TD, bool FIRST>
__global__ void __launch_bounds__(SORT_THREADS) embed_count_kernel(const EmbedParams P, const SortPass S)
{
    __shared__ unsigned int total[1024];
    const int cta = blockIdx.x, digits = 1 << S.bits, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (!FIRST && cta >= S.ctas) {
        fill_rows<TD>(P, S.fill_first, S.fill_last, cta - S.ctas, S.fill_ctas, [&](int v) { return P.present[v >> 5] >> (v & 31) & 1; });
        return;
    }
    if (FIRST) {
        for (int i = cta * SORT_THREADS + threadIdx.x; i < (P.vocab + 31) / 32; i += S.ctas * SORT_THREADS) P.present[i] = 0;
        if (cta == 0 && threadIdx.x == 0) *P.long_count = 0;
    }
    if (threadIdx.x < digits) total[threadIdx.x] = 0;
    __syncthreads();
    const unsigned int n = FIRST ? static_cast<unsigned int>(P.n) : *P.count;
    const unsigned int begin = min(n, (cta * SORT_WARPS + warp) * S.each), end = min(n, begin + S.each);
    for (unsigned int b = begin; b < end; b += ROUNDS * 32) {
        unsigned int key[ROUNDS], token[ROUNDS];
        sort_load<FIRST>(P, S, b + lane, end, key, token);
#pragma unroll
        for (int j = 0; j < ROUNDS; ++j)
            if (key[j] != NO_KEY) atomicAdd(total + (key[j] >> S.shift & (digits - 1)), 1u);
    }
    __syncthreads();
    if (threadIdx.x < digits) S.hist[(cta << S.bits) + threadIdx.x] = total[threadIdx.x];
}

// rank: what mine[digit] held, and the lanes of the digit before this one; mine counts on.
__device__ __forceinline__ unsigned int sort_rank(unsigned int key, int shift, int bits, unsigned int* mine)
{
    const unsigned int digit = key >> shift & ((1u << bits) - 1), lane = threadIdx.x & 31;
    unsigned int peers = __ballot_sync(~0u, key != NO_KEY);
#pragma unroll
    for (int k = 0; k < 10; ++k) {
        if (k >= bits) break;
        const unsigned int set = __ballot_sync(~0u, digit >> k & 1);
        peers &= digit >> k & 1 ? set : ~set;
    }
    const unsigned int below = peers & ((1u << lane) - 1);
    unsigned int rank = 0;
    if (key != NO_KEY) rank = mine[digit] + __popc(below);
    __syncwarp();
    if (key != NO_KEY && below == 0) mine[digit] += __popc(peers);
    __syncwarp();
    return rank;
}

template <class TD, bool FIRST>
__global__ void __launch_bounds__(SORT_THREADS) embed_place_kernel(const EmbedParams P, const SortPass S)
{
    extern __shared__ unsigned int place[];   // [warp][digit]
    __shared__ unsigned int before[1024], all[1024], warp_sum[SORT_WARPS];
    const int cta = blockIdx.x, digits = 1 << S.bits, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, tid = threadIdx.x;
    if (!FIRST && cta >= S.ctas) {
        fill_rows<TD>(P, S.fill_first, S.fill_last, cta - S.ctas, S.fill_ctas, [&](int v) { return P.present[v >> 5] >> (v & 31) & 1; });
        return;
    }
    const unsigned int n = FIRST ? static_cast<unsigned int>(P.n) : *P.count;
    const unsigned int begin = min(n, (cta * SORT_WARPS + warp) * S.each), end = min(n, begin + S.each);
    const bool once = S.each <= ROUNDS * 32;
    unsigned int* mine = place + (warp << S.bits);
    unsigned int key[ROUNDS], token[ROUNDS];
    sort_load<FIRST>(P, S, begin + lane, end, key, token);
    for (int i = lane; i < digits; i += 32) mine[i] = 0;
    if (tid < digits) before[tid] = all[tid] = 0;
    __syncwarp();
    for (unsigned int b = begin;;) {
#pragma unroll
        for (int j = 0; j < ROUNDS; ++j) {
            if (b + j * 32 >= end) break;
            const unsigned int r = sort_rank(key[j], S.shift, S.bits, mine);
            if (once && key[j] != NO_KEY) key[j] |= r << KEY_BITS;
        }
        b += ROUNDS * 32;
        if (b >= end) break;
        sort_load<FIRST>(P, S, b + lane, end, key, token);
    }
    __syncthreads();
    // each digit's tokens of all CTAs and of those before this one, by 1024 / digits threads
    {
        const int d = tid & (digits - 1);
        unsigned int a = 0, f = 0;
#pragma unroll 8
        for (int c = tid >> S.bits; c < S.ctas; c += SORT_THREADS >> S.bits) {
            const unsigned int x = S.hist[(c << S.bits) + d];
            a += x;
            if (c < cta) f += x;
        }
        atomicAdd(all + d, a);
        atomicAdd(before + d, f);
    }
    if (tid < digits) {
        unsigned int sum = 0;
#pragma unroll 8
        for (int w = 0; w < SORT_WARPS; ++w) {
            const unsigned int x = place[(w << S.bits) + tid];
            place[(w << S.bits) + tid] = sum;
            sum += x;
        }
    }
    __syncthreads();
    // first place of each digit: a scan over the threads
    const unsigned int a = tid < digits ? all[tid] : 0;
    unsigned int up = a;
#pragma unroll
    for (int k = 1; k < 32; k <<= 1) {
        const unsigned int v = __shfl_up_sync(~0u, up, k);
        if (lane >= k) up += v;
    }
    if (lane == 31) warp_sum[warp] = up;
    __syncthreads();
    const unsigned int base = up - a + __reduce_add_sync(~0u, lane < warp ? warp_sum[lane] : 0u);
    if (tid < digits) before[tid] += base;
    if (FIRST && cta == 0 && tid == SORT_THREADS - 1) *P.count = base + a;
    __syncthreads();
    const auto put = [&](unsigned int at, unsigned int k, unsigned int t) { S.to[at] = make_uint2(k, t); };
    if (once) {
#pragma unroll
        for (int j = 0; j < ROUNDS; ++j) {
            if (begin + j * 32 >= end) break;
            if (key[j] == NO_KEY) continue;
            const unsigned int k = key[j] & ((1u << KEY_BITS) - 1), digit = k >> S.shift & (digits - 1);
            put(before[digit] + mine[digit] + (key[j] >> KEY_BITS), k, token[j]);
        }
    } else {
        for (unsigned int b = begin; b < end; b += ROUNDS * 32) {
            sort_load<FIRST>(P, S, b + lane, end, key, token);
#pragma unroll
            for (int j = 0; j < ROUNDS; ++j) {
                if (b + j * 32 >= end) break;
                const unsigned int r = sort_rank(key[j], S.shift, S.bits, mine);
                if (key[j] != NO_KEY) put(before[key[j] >> S.shift & (digits - 1)] + r, key[j], token[j]);
            }
        }
    }
    if (!FIRST || P.accumulate) return;
    // the rows that the CTA's tokens name, in shared memory first: a few frequent tokens'
    // bits set one by one in L2 would take 20 us of 131072 tokens
    __syncthreads();
    const int words = (P.vocab + 31) / 32;
    for (int i = tid; i < words; i += SORT_THREADS) place[i] = 0;
    __syncthreads();
    for (unsigned int b = begin; b < end; b += ROUNDS * 32) {
        if (!once) sort_load<FIRST>(P, S, b + lane, end, key, token);
#pragma unroll
        for (int j = 0; j < ROUNDS; ++j) {
            const unsigned int k = key[j] & ((1u << KEY_BITS) - 1);
            if (key[j] != NO_KEY) atomicOr(place + (k >> 5), 1u << (k & 31));
        }
    }
    __syncthreads();
    for (int i = tid; i < words; i += SORT_THREADS)
        if (place[i]) atomicOr(P.present + i, place[i]);
}

// ---------------------------------------------------------------------- sums
// Eight columns' sum, in pairs.
struct Sum {
    Pair p[4];
    __device__ __forceinline__ void clear() { p[0] = p[1] = p[2] = p[3] = 0; }
    template <class T>
    __device__ __forceinline__ void add(const Eight<T>& row)
    {
        float x[8];
        row.values(x);
#pragma unroll
        for (int k = 0; k < 4; ++k) p[k] = add2(p[k], pair(x[2 * k], x[2 * k + 1]));
    }
    __device__ __forceinline__ void values(float (&x)[8]) const
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) split(p[k], x[2 * k], x[2 * k + 1]);
    }
};

template <class TD>
__device__ __forceinline__ void store_sum(const EmbedParams& P, unsigned int id, int c, const Sum& sum)
{
    TD* p = static_cast<TD*>(P.dst) + id * P.ld_dst + c;
    float x[8] = {}, s[8];
    if (P.accumulate) {
        Eight<TD> old;
        old.load(p, P.d - c);
        old.values(x);
    }
    sum.values(s);
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = fmaf(P.scale, s[k], x[k]);
    Eight<TD>::store(p, x, P.d - c);
}

__device__ __forceinline__ float* partial_at(const EmbedParams& P, int chunk, int after, int c)
{
    return P.partials + (chunk * 2ll + after) * ((P.d + 7) / 8 * 8) + c;
}

// The first place from `i` on, below `end`, whose id is not `id`; by a whole warp.
__device__ __forceinline__ unsigned int run_end(const uint2* items, unsigned int i, unsigned int end, unsigned int id)
{
    const unsigned int lane = threadIdx.x & 31;
    for (; i < end; i += 32) {
        const unsigned int other = __ballot_sync(~0u, i + lane >= end || items[i + lane].x != id);
        if (other) return min(end, i + __ffs(other) - 1);
    }
    return end;
}

// `group` threads share a chunk of the sorted tokens, eight columns each; wider
// rows are shared by `tiles` such groups.  A chunk's group takes the sums that begin
// in it, up to a chunk's length beyond its end.  Longer sums are split at the
// chunks' bounds into parts that embed_join_kernel adds.
template <class TX, class TD>
__global__ void __launch_bounds__(256) embed_sum_kernel(const EmbedParams P, int group, int tiles, int sum_ctas, int fill_first)
{
    constexpr int U = sizeof(TX) == 2 ? 8 : 4;   // rows whose columns a thread has on their way: 128 bytes of them
    if (static_cast<int>(blockIdx.x) >= sum_ctas) {
        fill_rows<TD>(P, fill_first, P.vocab, blockIdx.x - sum_ctas, gridDim.x - sum_ctas, [&](int v) { return P.present[v >> 5] >> (v & 31) & 1; });
        return;
    }
    const int at = blockIdx.x * (256 / group) + threadIdx.x / group, chunk = at / tiles, tile = at - chunk * tiles;
    const int c = (tile * group + threadIdx.x % group) * 8;
    const unsigned int valid = *P.count, length = P.chunk, begin = static_cast<unsigned int>(chunk) * length;
    if (chunk >= P.chunks || begin >= valid) return;
    const uint2* items = P.sorted;
    const unsigned int end = min(valid, begin + length);
    const unsigned int head = items[begin].x, tail = items[end - 1].x;
    bool open = begin > 0 && items[begin - 1].x == head;
    bool goes_on = end < valid && items[end].x == tail;
    unsigned int i = begin, stop = end;
    if (open && (begin == length || items[begin - length - 1].x != head) && !(goes_on && head == tail)) {
        i = run_end(items, begin, end, head);   // the chunk before has it all
        open = false;
    }
    if (goes_on && !(open && head == tail)) {
        if (end + length >= valid || items[end + length].x != tail) {
            stop = run_end(items, end, min(valid, end + length), tail);
            goes_on = false;
        } else if (tile == 0 && threadIdx.x % group == 0) {
            P.long_sums[atomicAdd(P.long_count, 1u)] = chunk;
        }
    }
    if (i >= stop) return;
    const bool mine = c < P.d;
    const TX* src = static_cast<const TX*>(P.src) + c;
    const int lane = threadIdx.x & 31;
    unsigned int cur = items[i].x;
    Sum sum;
    sum.clear();
    const auto flush = [&](bool part, int after) {
        if (!mine) return;
        if (part) {
            float x[8];
            sum.values(x);
            Eight<float>::store(partial_at(P, chunk, after, c), x, 8);
        } else {
            store_sum<TD>(P, cur, c, sum);
        }
    };
    for (; i < stop; i += 32) {   // a lane holds an item of the next 32
        const uint2 item = i + lane < stop ? items[i + lane] : make_uint2(NO_KEY, 0);
        unsigned int before = __shfl_up_sync(~0u, item.x, 1);
        if (lane == 0) before = cur;
        const unsigned int begins = __ballot_sync(~0u, item.x != before);
        const int count = min(32u, stop - i);
        for (int j = 0; j < count; j += U) {
            Eight<TX> row[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const unsigned int t = __shfl_sync(~0u, item.y, j + u);
                if (mine && j + u < count) row[u].load(src + t * P.ld_src, P.d - c);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (j + u >= count) break;
                if (begins >> (j + u) & 1) {
                    flush(open, 0);
                    cur = __shfl_sync(~0u, item.x, j + u), open = false;
                    sum.clear();
                }
                sum.add(row[u]);
            }
        }
    }
    flush(open || goes_on, open ? 0 : 1);
}

// The long sums, 128 columns of one at a time: eight warps add their shares of its
// parts, then one warp the shares.
template <class TD>
__global__ void __launch_bounds__(256) embed_join_kernel(const EmbedParams P)
{
    __shared__ float4 share[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const unsigned int slices = (P.d + 127) / 128, valid = *P.count, work = *P.long_count * slices;
    const int filled = (valid + P.chunk - 1) / P.chunk;   // chunks that hold tokens
    for (unsigned int w = blockIdx.x; w < work; w += gridDim.x) {
        const int first = P.long_sums[w / slices], c = (w % slices) * 128 + lane * 4;
        const unsigned int id = P.sorted[(first + 1ll) * P.chunk].x;
        // the chunks behind the first that begin with the id: 32 are looked at together, then
        // every 32nd part of what is left
        int last = first, above = filled;
        for (int step = 1; above - last > 1;) {
            const long long chunk = last + (lane + 1ll) * step;
            const unsigned int yes = __ballot_sync(~0u, chunk < above && P.sorted[chunk * P.chunk].x == id);
            const int count = __popc(yes);
            last += count * step;
            if (count < 32) above = static_cast<int>(min(static_cast<long long>(above), last + static_cast<long long>(step)));
            step = max(1, (above - last + 31) / 33);
        }
        // part i: of chunk first + i
        const int parts = last - first + 1, each = (parts + 7) / 8, from = warp * each, to = min(parts, from + each);
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        if (c < P.d) {
#pragma unroll 8
            for (int i = from; i < to; ++i) {
                const float4 x = *reinterpret_cast<const float4*>(partial_at(P, first + i, i == 0 ? 1 : 0, c));
                sum.x += x.x, sum.y += x.y, sum.z += x.z, sum.w += x.w;
            }
        }
        share[warp][lane] = sum;
        __syncthreads();
        if (warp == 0) {
            for (int k = 1; k < 8; ++k) {
                const float4 x = share[k][lane];
                sum.x += x.x, sum.y += x.y, sum.z += x.z, sum.w += x.w;
            }
            const float s[4] = {sum.x, sum.y, sum.z, sum.w};
            TD* p = static_cast<TD*>(P.dst) + id * P.ld_dst + c;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (c + k < P.d) Elem<TD>::put(p + k, fmaf(P.scale, s[k], P.accumulate ? Elem<TD>::get(p + k) : 0.f));
        }
        __syncthreads();
    }
}

struct Groups {
    int group, tiles;
};
Groups groups(int d)
{
    const int units = (d + 7) / 8;
    int group = 32;
    while (group < 256 && group < units) group *= 2;
    return {group, (units + group - 1) / group};
}

template <class TS, class TD>
cudaError_t rows(const EmbedParams& p, int sms, cudaStream_t stream)
{
    const long long units = (p.d + 7) / 8 * p.n;
    if (units < 2048ll * sms) embed_rows_kernel<TS, TD, 1><<<static_cast<unsigned int>((units + 255) / 256), 256, 0, stream>>>(p);
    else embed_rows_kernel<TS, TD, 4><<<static_cast<unsigned int>((units + 1023) / 1024), 256, 0, stream>>>(p);
    return cudaGetLastError();
}

template <class TS, class TD>
cudaError_t sums(const EmbedParams& p, int sms, cudaStream_t stream)
{
    const Groups g = groups(p.d);
    const int per = 256 / g.group;
    const int ctas = static_cast<int>((static_cast<long long>(p.chunks) * g.tiles + per - 1) / per);
    const int fill = p.filled < p.vocab ? std::min(4 * sms, (p.vocab - p.filled + 7) / 8) : 0;
    embed_sum_kernel<TS, TD><<<ctas + fill, 256, 0, stream>>>(p, g.group, g.tiles, ctas, p.filled);
    return cudaGetLastError();
}

template <class K>
cudaError_t allow_smem(K kern, size_t bytes, std::atomic<unsigned long long>& configured)   // bit d: set on device d
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !((configured.load(std::memory_order_acquire) >> dev) & 1ull)) {
        e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes));
        if (e != cudaSuccess) return e;
        if (dev < 64) configured.fetch_or(1ull << dev, std::memory_order_acq_rel);
    }
    return cudaSuccess;
}

template <class TD>
cudaError_t order(const EmbedParams& p, int sms, cudaStream_t stream)
{
    const int n = static_cast<int>(p.n), order_ctas = (n + 31) / 32;
    const int ctas = p.accumulate ? order_ctas : std::max(order_ctas, std::min(2 * sms, (p.vocab + 7) / 8));
    const int rows_each = p.accumulate ? 0 : (p.vocab + ctas - 1) / ctas;
    const size_t smem = sizeof(unsigned int) * ((n + 255) / 256 * 256 + (rows_each + 31) / 32);
    if (smem > 40 * 1024) {   // beyond what a launch may have without asking for more
        static std::atomic<unsigned long long> configured{0};
        const cudaError_t e = allow_smem(embed_order_kernel<TD>, sizeof(unsigned int) * (EMBED_FEW + EMBED_VOCAB_MAX / 32 + 1), configured);
        if (e != cudaSuccess) return e;
    }
    embed_order_kernel<TD><<<ctas, 256, smem, stream>>>(p, order_ctas, rows_each);
    return cudaGetLastError();
}

template <class TD, bool FIRST>
cudaError_t count(const EmbedParams& p, const SortPass& s, cudaStream_t stream)
{
    embed_count_kernel<TD, FIRST><<<s.ctas + s.fill_ctas, SORT_THREADS, 0, stream>>>(p, s);
    return cudaGetLastError();
}

template <class TD, bool FIRST>
cudaError_t place(const EmbedParams& p, const SortPass& s, cudaStream_t stream)
{
    static std::atomic<unsigned long long> configured{0};
    const cudaError_t e = allow_smem(embed_place_kernel<TD, FIRST>, sizeof(unsigned int) * SORT_WARPS << 10, configured);
    if (e != cudaSuccess) return e;
    embed_place_kernel<TD, FIRST><<<s.ctas + s.fill_ctas, SORT_THREADS, sizeof(unsigned int) * SORT_WARPS << s.bits, stream>>>(p, s);
    return cudaGetLastError();
}

// Rows of the table that the CTAs beside one of the sort's launches set to 0: what HBM
// takes in the time that the launch takes anyway.
constexpr double FILL_BYTES = 16e6;

SortPass sort_pass(const EmbedParams& p, int step)   // 0: by the lower digit, 1: by the upper
{
    SortPass s = {};
    s.from = step ? p.between : nullptr;
    s.to = step || !p.high ? p.sorted : p.between;
    s.hist = p.hist[step];
    s.shift = step ? p.low : 0;
    s.bits = step ? p.high : p.low;
    s.ctas = p.sort_ctas;
    s.each = p.sort_each;
    return s;
}

template <class TD>
cudaError_t sort_launch(EmbedParams& p, int launch, int sms, cudaStream_t stream)
{
    SortPass s = sort_pass(p, launch / 2);
    if (launch < 2) return launch == 0 ? count<TD, true>(p, s, stream) : place<TD, true>(p, s, stream);
    if (!p.accumulate) {   // (the first pass found out which rows the tokens name)
        const double row = static_cast<double>(p.d) * sizeof(TD);
        s.fill_first = p.filled;
        s.fill_last = p.filled = static_cast<int>(std::min<double>(p.vocab, p.filled + FILL_BYTES / row));
        s.fill_ctas = s.fill_last > s.fill_first && sms > s.ctas ? sms - s.ctas : 0;
        if (!s.fill_ctas) p.filled = s.fill_first;
    }
    return launch == 2 ? count<TD, false>(p, s, stream) : place<TD, false>(p, s, stream);
}

template <class TD>
cudaError_t join(const EmbedParams& p, int sms, cudaStream_t stream)
{
    embed_join_kernel<TD><<<8 * sms, 256, 0, stream>>>(p);
    return cudaGetLastError();
}

}  // namespace

EmbedLayout embed_layout(long long n, int vocab, int d, int sms, size_t at)
{
    EmbedLayout l = {};
    const auto take = [&](size_t bytes) {
        const size_t a = at;
        at = (at + bytes + 255) / 256 * 256;
        return a;
    };
    const Groups g = groups(d);
    // eight CTAs' worth of groups for every SM, of eight tokens at least
    const double per = static_cast<double>(n) * g.tiles * g.group / (8.0 * sms * 256);
    l.chunk = std::max(8, static_cast<int>(std::min(per / 8 + 1, 1e6)) * 8);
    l.chunks = static_cast<int>((n + l.chunk - 1) / l.chunk);
    l.sorted = take(n * sizeof(uint2));
    l.counts = take(2 * sizeof(unsigned int));
    l.long_sums = take(l.chunks * sizeof(unsigned int));
    l.partials = take(sizeof(float) * 2 * l.chunks * static_cast<size_t>((d + 7) / 8 * 8));
    if (n > EMBED_FEW) {
        int bits = 1;
        while ((1 << bits) < vocab) ++bits;
        l.low = bits > 10 ? (bits + 1) / 2 : bits, l.high = bits - l.low;
        // up to 64 CTAs of few rounds, then up to 256 of many
        const long long rounds = std::max((n + 64 * SORT_THREADS - 1) / (64 * SORT_THREADS), 1ll);
        const long long most = (n + 256 * SORT_THREADS - 1) / (256 * SORT_THREADS);
        l.sort_each = static_cast<unsigned int>(std::max(std::min<long long>(rounds, ROUNDS), most) * 32);
        l.sort_ctas = static_cast<int>((n + l.sort_each * SORT_WARPS - 1) / (l.sort_each * SORT_WARPS));
        l.between = take(n * sizeof(uint2));
        l.present = take((vocab + 31) / 32 * sizeof(unsigned int));
        l.hist[0] = take(sizeof(unsigned int) * l.sort_ctas << l.low);
        l.hist[1] = take(sizeof(unsigned int) * l.sort_ctas << l.high);
    }
    l.total = at;
    return l;
}

cudaError_t launch_embed_rows(const EmbedParams& p, int dtype_src, int dtype_dst, int sms, cudaStream_t stream)
{
    using bf16 = __nv_bfloat16;
    if (dtype_src == 0) return dtype_dst == 0 ? rows<bf16, bf16>(p, sms, stream) : rows<bf16, float>(p, sms, stream);
    return dtype_dst == 0 ? rows<float, bf16>(p, sms, stream) : rows<float, float>(p, sms, stream);
}

cudaError_t launch_embed_order(EmbedParams& p, int dtype_dst, int sms, cudaStream_t stream)
{
    const cudaError_t e = dtype_dst == 0 ? order<__nv_bfloat16>(p, sms, stream) : order<float>(p, sms, stream);
    p.filled = p.vocab;
    return e;
}

cudaError_t launch_embed_sort(EmbedParams& p, int launch, int dtype_dst, int sms, cudaStream_t stream)
{
    return dtype_dst == 0 ? sort_launch<__nv_bfloat16>(p, launch, sms, stream) : sort_launch<float>(p, launch, sms, stream);
}

cudaError_t launch_embed_sums(const EmbedParams& p, int dtype_src, int dtype_dst, int sms, cudaStream_t stream)
{
    using bf16 = __nv_bfloat16;
    if (dtype_src == 0) return dtype_dst == 0 ? sums<bf16, bf16>(p, sms, stream) : sums<bf16, float>(p, sms, stream);
    return dtype_dst == 0 ? sums<float, bf16>(p, sms, stream) : sums<float, float>(p, sms, stream);
}

cudaError_t launch_embed_join(const EmbedParams& p, int dtype_dst, int sms, cudaStream_t stream)
{
    return dtype_dst == 0 ? join<__nv_bfloat16>(p, sms, stream) : join<float>(p, sms, stream);
}

}  // namespace cola
