// Kernels of the token embedding (embed.cuh) and their launchers.
#include "embed.cuh"

#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

#include "vocab_rows.cuh"

namespace cola {
namespace {

// ------------------------------------------------- eight columns of a row
// Pitches are multiples of 8 elements, so that every eight columns begin on a
// 16-byte boundary.  WHOLE: the width is one too; else the last of a row may be
// fewer, `left` of them.
template <class T>
struct Eight;

template <>
struct Eight<__nv_bfloat16> {
    uint4 u;
    template <bool WHOLE>
    __device__ __forceinline__ void load(const __nv_bfloat16* p, int left)
    {
        if (WHOLE || left >= 8) {
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
    template <bool WHOLE, bool LAST = false>   // LAST: nobody reads it soon
    __device__ __forceinline__ static void store(__nv_bfloat16* p, const float (&x)[8], int left)
    {
        if (WHOLE || left >= 8) {
            if (LAST) __stcs(reinterpret_cast<uint4*>(p), Elem<__nv_bfloat16>::pack(x));
            else *reinterpret_cast<uint4*>(p) = Elem<__nv_bfloat16>::pack(x);
        } else {
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (i < left) p[i] = __float2bfloat16_rn(x[i]);
        }
    }
};

template <>
struct Eight<float> {
    float x[8];
    // in one piece where it lies on a 32-byte boundary: two pieces would touch every
    // sector twice
    template <bool WHOLE>
    __device__ __forceinline__ void load(const float* p, int left)
    {
        if (WHOLE || left >= 8) {
            if ((reinterpret_cast<uintptr_t>(p) & 16) == 0) {
                asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                             : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7])
                             : "l"(p));
            } else {
                const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
                x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = i < left ? p[i] : 0.f;
        }
    }
    __device__ __forceinline__ void values(float (&y)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = x[i];
    }
    template <bool WHOLE, bool LAST = false>
    __device__ __forceinline__ static void store(float* p, const float (&x)[8], int left)
    {
        if (WHOLE || left >= 8) {
            if ((reinterpret_cast<uintptr_t>(p) & 16) == 0) {
                if (LAST)
                    asm volatile("st.global.cs.v8.f32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"f"(x[0]), "f"(x[1]), "f"(x[2]),
                                 "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]), "l"(p)
                                 : "memory");
                else
                    asm volatile("st.global.v8.f32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"f"(x[0]), "f"(x[1]), "f"(x[2]),
                                 "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]), "l"(p)
                                 : "memory");
            } else {
                reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
                reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (i < left) p[i] = x[i];
        }
    }
};

// `1 << shift` threads of a CTA of 256 share a row, eight columns each; wider rows are
// shared by `tiles` such groups.
struct Groups {
    int shift, tiles;
};

// ------------------------------------------------------------------ lookup
// ROWS rows a thread, whose ids and then whose columns are loaded together; no division
// finds them.  Bound by HBM: 32768 x 2048 bf16 26.5 us, 0.94 of the copy rate of X and the
// rows that are named, each read once (one row a thread, found by dividing, took 40 us).
template <class TE, class TX, bool WHOLE, int ROWS>
__global__ void __launch_bounds__(256) embed_rows_kernel(const EmbedParams P, const Groups g)
{
    const int c = (blockIdx.y << g.shift | (threadIdx.x & ((1 << g.shift) - 1))) * 8, step = 256 >> g.shift;
    if (c >= P.d) return;
    const long long t0 = static_cast<long long>(blockIdx.x) * (ROWS * step) + (threadIdx.x >> g.shift);
    const TE* src = static_cast<const TE*>(P.src) + c;
    TX* dst = static_cast<TX*>(P.dst) + c;
    long long id[ROWS];
    Eight<TE> e[ROWS];
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
        id[u] = t0 + u * step < P.n ? P.ids[t0 + u * step] : -1;
        if (id[u] >= P.vocab) id[u] = -1;
    }
#pragma unroll
    for (int u = 0; u < ROWS; ++u)
        if (id[u] >= 0) e[u].template load<WHOLE>(src + id[u] * P.ld_src, P.d - c);
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
        if (t0 + u * step >= P.n) break;
        float x[8] = {};
        if (id[u] >= 0) {
            e[u].values(x);
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] *= P.scale;
        }
        TX* at = dst + (t0 + u * step) * P.ld_dst;
        if (P.stream) Eight<TX>::template store<WHOLE, true>(at, x, P.d - c);
        else Eight<TX>::template store<WHOLE>(at, x, P.d - c);
    }
}

// ------------------------------------------------------------- rows of no token
// Rows [first, last) of the gradient := 0, by the warps of `ctas` CTAs of which this is
// number `cta`, in pieces of up to 2048 columns, alike in width (whole rows on a warp, 8083 of
// 8099 columns in fp32 took 52 us instead of 47); NAMED: but for those that tokens name.
template <class TD, bool WHOLE, bool NAMED>
__device__ __forceinline__ void fill_rows(const EmbedParams& P, int first, int last, int cta, int ctas)
{
    const int lane = threadIdx.x & 31, warps = blockDim.x >> 5, pieces = (P.d + 2047) / 2048;
    const int width = ((P.d + pieces - 1) / pieces + 255) / 256 * 256;
    const unsigned int step = ctas * warps, end = static_cast<unsigned int>(last - first) * pieces;
    const float zero[8] = {};
    const auto named = [&](unsigned int u) {
        const int v = first + u / pieces;
        return NAMED && u < end ? P.present[v >> 5] >> (v & 31) & 1 : 0u;
    };
    unsigned int u = cta * warps + (threadIdx.x >> 5);
    for (unsigned int skip = named(u), next; u < end; u += step, skip = next) {
        next = named(u + step);   // (on its way while this piece is stored)
        if (skip) continue;
        const unsigned int v = first + u / pieces, from = u % pieces * width, to = min(P.d, static_cast<int>(from) + width);
        TD* row = static_cast<TD*>(P.dst) + v * P.ld_dst;
        for (int c = from + lane * 8; c < static_cast<int>(to); c += 256) Eight<TD>::template store<WHOLE>(row + c, zero, P.d - c);
    }
}

// While tokens are sorted, CTAs of the same launches set rows [first, last) to 0, the
// last rows of the table first, whether or not a token names them: the sums are stored
// later, HBM has nothing else to do, and where ids go by frequency few of those are named.
struct Fill {
    int first, last, ctas;
};

// -------------------------------------------------------------- few tokens at once
constexpr unsigned int NO_KEY = ~0u;

__device__ __forceinline__ unsigned int key_of(long long id, int vocab)
{
    return id >= 0 && id < vocab ? static_cast<unsigned int>(id) : NO_KEY;
}

// Up to EMBED_FEW tokens in one launch, in which no CTA waits for another: each sorts all
// of them into bins by the lower ten bits of their ids, in shared memory and in any order,
// and finds the places of its own tokens, by the number of tokens of lower bins and of
// those in its bin that come before it (their order is by the ids' lower bits first).
// Bound by latency: 2048 tokens 4 us, 8191 8 us (counting every token against all others
// took 20 us there, the sort by digits 16).
// They also set the bits of the rows that are named (`words_each` words each).
constexpr int ORDER_THREADS = 512, ORDER_TOKENS = 64, ORDER_EACH = EMBED_FEW / ORDER_THREADS, BIN_BITS = 10, INDEX_BITS = 13;
static_assert(EMBED_FEW <= 1 << INDEX_BITS && EMBED_VOCAB_MAX <= 1 << (BIN_BITS + 32 - INDEX_BITS), "a token's word");

template <class TD, bool WHOLE>
__global__ void __launch_bounds__(ORDER_THREADS) embed_order_kernel(const EmbedParams P, const Fill fill, int order_ctas, int words_each)
{
    extern __shared__ unsigned int bits[];   // of rows
    __shared__ unsigned int first[1 << BIN_BITS], next[1 << BIN_BITS], warp_sum[ORDER_THREADS / 32];
    __shared__ unsigned int binned[EMBED_FEW];
    const int n = static_cast<int>(P.n), tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    grid_launch_dependents();
    if (static_cast<int>(blockIdx.x) >= order_ctas) {
        fill_rows<TD, WHOLE, false>(P, fill.first, fill.last, blockIdx.x - order_ctas, fill.ctas);
        return;
    }
    unsigned int key[ORDER_EACH];
#pragma unroll
    for (int j = 0; j < ORDER_EACH; ++j) {
        const int i = j * ORDER_THREADS + tid;
        key[j] = i < n ? key_of(P.ids[i], P.vocab) : NO_KEY;
    }
    const unsigned int r0 = blockIdx.x * words_each * 32u, r1 = min(static_cast<unsigned int>(P.unfilled), r0 + words_each * 32u);
    const int words = r1 > r0 ? (r1 - r0 + 31) / 32 : 0;
    for (int i = tid; i < words; i += ORDER_THREADS) bits[i] = 0;
    next[tid] = next[tid + 512] = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < ORDER_EACH; ++j) {
        if (key[j] >= r0 && key[j] < r1) atomicOr(bits + ((key[j] - r0) >> 5), 1u << ((key[j] - r0) & 31));
        if (key[j] != NO_KEY) atomicAdd(next + (key[j] & 1023), 1u);
    }
    __syncthreads();
    for (int i = tid; i < words; i += ORDER_THREADS) P.present[r0 / 32 + i] = bits[i];
    // first places of the bins, two a thread
    const unsigned int c0 = next[2 * tid], c1 = next[2 * tid + 1];
    unsigned int up = c0 + c1;
#pragma unroll
    for (int k = 1; k < 32; k <<= 1) {
        const unsigned int v = __shfl_up_sync(~0u, up, k);
        if (lane >= k) up += v;
    }
    if (lane == 31) warp_sum[warp] = up;
    __syncthreads();
    const unsigned int base = up - c0 - c1 + __reduce_add_sync(~0u, lane < warp ? warp_sum[lane] : 0u);
    first[2 * tid] = next[2 * tid] = base, first[2 * tid + 1] = next[2 * tid + 1] = base + c0;
    if (blockIdx.x == 0 && tid == ORDER_THREADS - 1) *P.count = base + c0 + c1, *P.long_count = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < ORDER_EACH; ++j)
        if (key[j] != NO_KEY) binned[atomicAdd(next + (key[j] & 1023), 1u)] = key[j] >> BIN_BITS << INDEX_BITS | (j * ORDER_THREADS + tid);
    __syncthreads();
    // a warp a token (behind its last token, `next` is where a bin ends)
    for (int i = blockIdx.x * ORDER_TOKENS + warp; i < min(n, static_cast<int>(blockIdx.x + 1) * ORDER_TOKENS); i += ORDER_THREADS / 32) {
        const unsigned int k = key_of(P.ids[i], P.vocab);
        if (k == NO_KEY) continue;
        const unsigned int word = k >> BIN_BITS << INDEX_BITS | i, begin = first[k & 1023], end = next[k & 1023];
        unsigned int before = 0;
        for (unsigned int m = begin + lane; m < end; m += 32) before += binned[m] < word;
        before = __reduce_add_sync(~0u, before);
        if (lane == 0) P.sorted[begin + before] = make_uint2(k, i);
    }
}

// --------------------------------------------------------- many tokens by digits
// One or two passes of a stable counting sort by up to ten bits, each in two
// launches.  Every CTA has consecutive tokens; the first counts its digits, the
// second ranks them: every warp has consecutive ones of the CTA's, 32 a round, and
// ranks each round's among those of their digit, by ballots over the digit's bits; counts
// become first places, over the digits, the CTAs and the warps.  Bound by latency, of four
// launches that overlap: 16 us for 32768 tokens, 20 us for 131072 (one cluster of 8 or 16
// CTAs took 28 and 78 us: a round of a CTA takes 0.65 us, with __match_any_sync 0.9 us
// where digits differ, and an SM scatters a pair per cycle).
constexpr int SORT_THREADS = 1024, SORT_WARPS = 32;
constexpr int ROUNDS = 8;                   // whose tokens a warp holds at once
constexpr int KEY_BITS = 20;                // a held token: its rank in its warp above its key

struct SortPass {
    const uint2* from;        // nullptr: the ids (those that name no token are left out)
    uint2* to;
    unsigned int* hist;       // [CTA][digit]
    int shift, bits, ctas;
    unsigned int each;        // tokens of a warp, a multiple of 32
    Fill fill;                // by the CTAs behind the others
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

template <bool FIRST>
__global__ void __launch_bounds__(SORT_THREADS) embed_count_kernel(const EmbedParams P, const SortPass S)
{
    __shared__ unsigned int total[1024];
    const int cta = blockIdx.x, digits = 1 << S.bits, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (!FIRST) grid_dependency_wait();
    grid_launch_dependents();
    if (FIRST) {
        for (int i = cta * SORT_THREADS + threadIdx.x; i < (P.unfilled + 31) / 32; i += S.ctas * SORT_THREADS) P.present[i] = 0;
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

template <class TD, bool WHOLE, bool FIRST>
__global__ void __launch_bounds__(SORT_THREADS) embed_place_kernel(const EmbedParams P, const SortPass S)
{
    extern __shared__ unsigned int place[];   // [warp][digit]
    __shared__ unsigned int before[1024], all[1024], warp_sum[SORT_WARPS];
    const int cta = blockIdx.x, digits = 1 << S.bits, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, tid = threadIdx.x;
    // the launch before this one counts; what this one ranks was there before that launch
    grid_launch_dependents();
    if (cta >= S.ctas) {
        fill_rows<TD, WHOLE, false>(P, S.fill.first, S.fill.last, cta - S.ctas, S.fill.ctas);
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
    grid_dependency_wait();
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
    if (!FIRST || P.unfilled == 0) return;
    // the rows that the CTA's tokens name, in shared memory first: a few frequent tokens'
    // bits set one by one in L2 would take 20 us of 131072 tokens
    __syncthreads();
    const int words = (P.unfilled + 31) / 32;
    for (int i = tid; i < words; i += SORT_THREADS) place[i] = 0;
    __syncthreads();
    for (unsigned int b = begin; b < end; b += ROUNDS * 32) {
        if (!once) sort_load<FIRST>(P, S, b + lane, end, key, token);
#pragma unroll
        for (int j = 0; j < ROUNDS; ++j) {
            const unsigned int k = key[j] & ((1u << KEY_BITS) - 1);
            if (key[j] != NO_KEY && k < P.unfilled) atomicOr(place + (k >> 5), 1u << (k & 31));
        }
    }
    __syncthreads();
    for (int i = tid; i < words; i += SORT_THREADS)
        if (place[i]) atomicOr(P.present + i, place[i]);
}

// ---------------------------------------------------------------------- sums
// A thread has 16 bytes of columns of each row of dX: four of fp32, eight of bf16.
template <class TX>
constexpr int COLS = 16 / sizeof(TX);

template <int N>
struct Sum {
    Pair p[N / 2];
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int k = 0; k < N / 2; ++k) p[k] = 0;
    }
    template <class TX>
    __device__ __forceinline__ void add(const uint4& row)
    {
        float x[N];
        Elem<TX>::unpack(row, x);
#pragma unroll
        for (int k = 0; k < N / 2; ++k) p[k] = add2(p[k], pair(x[2 * k], x[2 * k + 1]));
    }
    __device__ __forceinline__ void values(float (&x)[N]) const
    {
#pragma unroll
        for (int k = 0; k < N / 2; ++k) split(p[k], x[2 * k], x[2 * k + 1]);
    }
};

// N columns at a multiple of N, `left` of them there.
template <int N>
__device__ __forceinline__ void store_columns(float* p, const float (&x)[N], int left)
{
    if (left >= N) {
#pragma unroll
        for (int k = 0; k < N; k += 4) *reinterpret_cast<float4*>(p + k) = make_float4(x[k], x[k + 1], x[k + 2], x[k + 3]);
    } else {
#pragma unroll
        for (int k = 0; k < N - 1; ++k)
            if (k < left) p[k] = x[k];
    }
}
template <int N>
__device__ __forceinline__ void store_columns(__nv_bfloat16* p, const float (&x)[N], int left)
{
    if (left >= N) {
        uint2 u[N / 4];
#pragma unroll
        for (int k = 0; k < N; k += 4) {
            const __nv_bfloat162 lo = __floats2bfloat162_rn(x[k], x[k + 1]), hi = __floats2bfloat162_rn(x[k + 2], x[k + 3]);
            u[k / 4] = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
        }
        if constexpr (N == 8) *reinterpret_cast<uint4*>(p) = make_uint4(u[0].x, u[0].y, u[1].x, u[1].y);
        else *reinterpret_cast<uint2*>(p) = u[0];
    } else {
#pragma unroll
        for (int k = 0; k < N - 1; ++k)
            if (k < left) p[k] = __float2bfloat16_rn(x[k]);
    }
}

// Four columns of fp32 are added to, without waiting for what they were.  (Nobody else
// adds to them in this call: the order of the addition is no matter.  Values below the
// smallest normal number count as 0 there.)
__device__ __forceinline__ void add_four(float* p, float a, float b, float c, float d)
{
    asm volatile("red.relaxed.gpu.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(p), "f"(a), "f"(b), "f"(c), "f"(d) : "memory");
}

template <class TD, int N>
__device__ __forceinline__ void store_sum(const EmbedParams& P, unsigned int id, int c, const Sum<N>& sum)
{
    TD* p = static_cast<TD*>(P.dst) + id * P.ld_dst + c;
    float x[N];
    sum.values(x);
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] *= P.scale;
    if constexpr (sizeof(TD) == 4) {
        if (P.accumulate) {
            if (P.d - c >= N) {
#pragma unroll
                for (int k = 0; k < N; k += 4) add_four(p + k, x[k], x[k + 1], x[k + 2], x[k + 3]);
            } else {
#pragma unroll
                for (int k = 0; k < N - 1; ++k)
                    if (k < P.d - c) p[k] += x[k];
            }
            return;
        }
    }
    store_columns(p, x, P.d - c);
}

__device__ __forceinline__ float* partial_at(const EmbedParams& P, int chunk, int after, int c)
{
    return P.partials + (chunk * 2ll + after) * ((P.d + 7) / 8 * 8) + c;
}

__device__ __forceinline__ void copy_async(uint32_t to, const void* from, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// ------------------------------------------------------- few tokens in one launch
// A small gradient in one launch, without the workspace: row v of the table belongs to CTA
// v % (CTAs), so that frequent tokens, whose ids lie together, are spread.  Every CTA reads
// all ids and keeps those of its rows, sorts them (few by counting the smaller ones, more by
// a bitonic network, which takes 2,048 of one row from 110 us a call to 52 us), adds their
// rows of dX, and sets its other rows to 0.  Its warps share the sorted tokens in ranges and
// the columns in tiles; a sum that crosses ranges is added from parts in shared memory.
// Bound by latency, and by one SM where one token has most rows, whence the limits.  bf16,
// table of 32,000: 2,048 tokens of 512 columns 10.6 us, 16.5 us in three launches; if all of
// them are one token 44 us and 22 us.  Twice the bytes (1,024 columns) would have 14.3 and
// 76 us here against 20.0 and 28 us: it is left to the three launches.  Four micro-batches of
// 2,048 x 512 in fp32, one overwriting and three adding: 37 us, 57 us in three launches each.
// The limit in bytes bounds what one repeated token costs: of ids spread over the table one
// launch is ahead of three at all of 300 to 2,048 tokens of 128 to 2,048 columns (bf16 into fp32,
// 0.54 to 0.93 of their time overwritten, 0.42 to 0.69 added), of one token it takes 2.4 times
// theirs for 2,048 x 512 (60 us against 25 overwritten) and 3.2 times for 2,048 x 2,048.  fp32 dX
// of 2,048 x 512 goes to three launches: 19.5 us (one: 16.6; one token 27 and 87).
// Two CTAs an SM, in 64 registers with six rows on their way per warp: one alone, of the same
// or twice as many threads, has 12 us with up to 16 rows on their way.
constexpr int ONE_THREADS = 512, ONE_WARPS = 16, ONE_INDEX = 11, ONE_RANKED = 256;
static_assert(EMBED_ONE == 1 << ONE_INDEX && EMBED_VOCAB_MAX <= 1 << (32 - ONE_INDEX), "a token's word");
static_assert(ONE_RANKED <= ONE_THREADS && ONE_WARPS * 32 == ONE_THREADS, "one word a thread");

template <class TX, class TD, bool WHOLE>
__global__ void __launch_bounds__(ONE_THREADS, 2) embed_one_kernel(const EmbedParams P, int rows_each)
{
    constexpr int N = COLS<TX>, U = 6;
    extern __shared__ __align__(16) unsigned int one_smem[];
    __shared__ int kept;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = static_cast<int>(P.n), ctas = gridDim.x, cta = blockIdx.x;
    unsigned int *list = one_smem, *sorted = list + EMBED_ONE, *bits = sorted + EMBED_ONE;   // (row << ONE_INDEX | token)
    float* parts = reinterpret_cast<float*>(bits + (rows_each + 127) / 128 * 4);               // [range][open or not][column]
    for (int i = tid; i < (rows_each + 31) / 32; i += ONE_THREADS) bits[i] = 0;
    if (tid == 0) kept = 0;
    unsigned int key[EMBED_ONE / ONE_THREADS];
#pragma unroll
    for (int j = 0; j < EMBED_ONE / ONE_THREADS; ++j) {
        const int i = j * ONE_THREADS + tid;
        key[j] = i < n ? key_of(P.ids[i], P.vocab) : NO_KEY;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < EMBED_ONE / ONE_THREADS; ++j) {
        const unsigned int row = key[j] / ctas;
        const bool keep = key[j] != NO_KEY && key[j] - row * ctas == static_cast<unsigned int>(cta);
        const unsigned int mask = __ballot_sync(~0u, keep);
        if (mask == 0) continue;
        int base = lane == 0 ? atomicAdd(&kept, __popc(mask)) : 0;
        base = __shfl_sync(~0u, base, 0);
        if (!keep) continue;
        list[base + __popc(mask & ((1u << lane) - 1))] = row << ONE_INDEX | (j * ONE_THREADS + tid);
    }
    __syncthreads();
    const int m = kept;
    if (m <= ONE_RANKED) {
        if (tid < 4 && m + tid < (m + 3) / 4 * 4) list[m + tid] = NO_KEY;
        __syncthreads();
        if (tid < m) {
            const unsigned int word = list[tid];
            int before = 0;
            for (int q = 0; q < m; q += 4) {
                const uint4 w = *reinterpret_cast<const uint4*>(list + q);
                before += (w.x < word) + (w.y < word) + (w.z < word) + (w.w < word);
            }
            sorted[before] = word;
        }
        __syncthreads();
    } else {
        const int length = 1 << (32 - __clz(m - 1));
        for (int i = m + tid; i < length; i += ONE_THREADS) list[i] = NO_KEY;
        __syncthreads();
        for (int run = 2; run <= length; run *= 2)
            for (int apart = run / 2; apart > 0; apart /= 2) {
                for (int k = tid; k < length / 2; k += ONE_THREADS) {
                    const int i = 2 * k - (k & (apart - 1)), other = i + apart;
                    const unsigned int a = list[i], b = list[other];
                    if ((a > b) == ((i & run) == 0)) list[i] = b, list[other] = a;
                }
                __syncthreads();
            }
        sorted = list;
    }
    if (!P.accumulate)
        for (int k = tid; k < m; k += ONE_THREADS) {
            const unsigned int row = sorted[k] >> ONE_INDEX;
            if (k == 0 || sorted[k - 1] >> ONE_INDEX != row) atomicOr(bits + (row >> 5), 1u << (row & 31));
        }
    if (m > 0) {
        const int tiles = (P.d + 32 * N - 1) / (32 * N), stride = tiles * 32 * N;
        const int each = (m + max(1, ONE_WARPS / tiles) - 1) / max(1, ONE_WARPS / tiles), ranges = (m + each - 1) / each;
        const auto row_at = [&](int i) { return sorted[i] >> ONE_INDEX; };
        for (int u = warp; u < ranges * tiles; u += ONE_WARPS) {
            const int range = u / tiles, c = ((u - range * tiles) * 32 + lane) * N, left = P.d - c;
            const int begin = range * each, end = min(m, begin + each);
            const TX* src = static_cast<const TX*>(P.src) + c;
            unsigned int cur = row_at(begin);
            bool open = begin > 0 && row_at(begin - 1) == cur;
            const bool goes_on = end < m && row_at(end) == row_at(end - 1);
            Sum<N> sum;
            sum.clear();
            const auto flush = [&](bool part, int after) {
                if (left <= 0) return;
                if (part) {
                    float x[N];
                    sum.values(x);
                    store_columns(parts + (range * 2 + after) * stride + c, x, N);
                } else {
                    store_sum<TD>(P, cur * ctas + cta, c, sum);
                }
            };
            for (int i = begin; i < end; i += U) {
                uint4 row[U];
#pragma unroll
                for (int k = 0; k < U; ++k)
                    if (i + k < end && left > 0) {
                        const TX* at = src + (sorted[i + k] & (EMBED_ONE - 1)) * P.ld_src;
                        if (WHOLE || left >= N) {
                            row[k] = *reinterpret_cast<const uint4*>(at);
                        } else {
                            float x[N];
#pragma unroll
                            for (int e = 0; e < N; ++e) x[e] = e < left ? Elem<TX>::get(at + e) : 0.f;
                            row[k] = Elem<TX>::pack(x);
                        }
                    }
                if (i + U <= end && row_at(i + U - 1) == cur) {   // (sorted: all of them)
#pragma unroll
                    for (int k = 0; k < U; ++k) sum.template add<TX>(row[k]);
                    continue;
                }
#pragma unroll
                for (int k = 0; k < U; ++k) {
                    if (i + k >= end) break;
                    if (row_at(i + k) != cur) {
                        flush(open, 0);
                        cur = row_at(i + k), open = false;
                        sum.clear();
                    }
                    sum.template add<TX>(row[k]);
                }
            }
            flush(open || goes_on, open ? 0 : 1);
        }
        __syncthreads();
        // the sums that cross ranges, by the range that they begin in
        for (int u = tid; u < (ranges - 1) * P.d; u += ONE_THREADS) {
            const int range = u / P.d, c = u - range * P.d, begin = range * each, end = begin + each;
            const unsigned int row = row_at(end);
            if (row_at(end - 1) != row || (begin > 0 && row_at(begin - 1) == row)) continue;
            float sum = parts[(range * 2 + 1) * stride + c];
            for (int k = range + 1; k < ranges && row_at(k * each) == row; ++k) sum += parts[k * 2 * stride + c];
            TD* p = static_cast<TD*>(P.dst) + (static_cast<long long>(row) * ctas + cta) * P.ld_dst + c;
            Elem<TD>::put(p, fmaf(P.scale, sum, P.accumulate ? Elem<TD>::get(p) : 0.f));
        }
    }
    if (P.accumulate) return;
    __syncthreads();   // (the bits)
    const int pieces = (P.d + 2047) / 2048, width = ((P.d + pieces - 1) / pieces + 255) / 256 * 256;
    const float zero[8] = {};
    for (int u = warp; u < rows_each * pieces; u += ONE_WARPS) {
        const int row = u / pieces, from = (u - row * pieces) * width, to = min(P.d, from + width);
        const long long v = static_cast<long long>(row) * ctas + cta;
        if (v >= P.vocab || (bits[row >> 5] >> (row & 31) & 1)) continue;
        for (int c = from + lane * 8; c < to; c += 256)
            Eight<TD>::template store<WHOLE>(static_cast<TD*>(P.dst) + v * P.ld_dst + c, zero, P.d - c);
    }
}

// ------------------------------------------------------------- sums of many tokens
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

// The last chunk that begins with the id, of those from `first` + 1 on (which does) below
// `above`; by a whole warp: 32 chunks together, then every 33rd part of what is left.
__device__ __forceinline__ int last_chunk(const EmbedParams& P, int first, int above, unsigned int id)
{
    int last = first + 1;
    for (int step = 1; above - last > 1; step = max(1, (above - last + 31) / 33)) {
        const long long chunk = last + ((threadIdx.x & 31) + 1ll) * step;
        const int yes = __popc(__ballot_sync(~0u, chunk < above && P.sorted[chunk * P.chunk].x == id));
        last += yes * step;
        if (yes < 32) above = min(above, last + step);
    }
    return last;
}

// A group has a chunk of the sorted tokens.  It takes the sums that begin
// in it, up to a chunk's length beyond its end.  Longer sums are split at the
// chunks' bounds into parts that embed_join_kernel adds: a frequent token's rows are
// shared by as many groups as they fill, and the order of its sum is the chunks'.
//
// A thread copies its columns of every row into shared memory of its own, BATCHES
// batches of BATCH rows ahead of the one that it adds: no thread waits for another, and
// an SM has 192 KB of rows on their way (as many in registers, eight rows together: 253
// us against 217 us for 131072 x 4096 bf16).  Bound by HBM, 206 us and 6.2 TB/s there; of
// 32768 x 2048, 41 us and 5.3 TB/s, by the start of its CTAs too: each reads where its
// sums begin, then its first rows.
constexpr int BATCH = 4, BATCHES = 4;

template <class TX, class TD, bool WHOLE>
__global__ void __launch_bounds__(256, 3) embed_sum_kernel(const EmbedParams P, const Groups g, int fill_first)
{
    constexpr int N = COLS<TX>;
    extern __shared__ uint4 ring[];   // [row of the batches][thread]
    grid_dependency_wait();
    if (P.chunks > 1) grid_launch_dependents();   // (embed_join_kernel, which waits)
    const int at = blockIdx.x << (8 - g.shift) | threadIdx.x >> g.shift, chunk = at / g.tiles, tile = at - chunk * g.tiles;
    const int member = threadIdx.x & ((1 << g.shift) - 1), c = (tile << g.shift | member) * N;
    const int lane = threadIdx.x & 31;
    const unsigned int n = static_cast<unsigned int>(P.n), length = P.chunk, begin = static_cast<unsigned int>(chunk) * length;
    const uint2* items = P.sorted;
    // what tells where the chunk's sums begin and end, and its first items, all loaded
    // together (what lies behind the last token is not used)
    const unsigned int valid = *P.count;
    const auto id_at = [&](unsigned int k) { return items[min(k, n - 1)].x; };
    const unsigned int before_chunk = id_at(max(begin, 1u) - 1), head = id_at(begin), two_before = id_at(max(begin, length + 1) - length - 1);
    const unsigned int full_tail = id_at(begin + length - 1), behind = id_at(begin + length), far_behind = id_at(begin + 2 * length);
    uint2 item = items[min(begin + lane, n - 1)];   // a lane holds an item of 32
    unsigned int i = begin, stop = begin;
    bool open = false, goes_on = false;
    if (chunk < P.chunks && begin < valid) {
        const unsigned int end = min(valid, begin + length), tail = end == begin + length ? full_tail : items[end - 1].x;
        open = begin > 0 && before_chunk == head;
        goes_on = end < valid && behind == tail;
        stop = end;
        if (open && (begin == length || two_before != head) && !(goes_on && head == tail)) {
            i = run_end(items, begin, end, head);   // the chunk before has it all
            open = false;
        }
        if (goes_on && !(open && head == tail)) {
            if (end + length >= valid || far_behind != tail) {
                stop = run_end(items, end, min(valid, end + length), tail);
                goes_on = false;
            } else if (tile == 0 && member < 32) {
                const int last = last_chunk(P, chunk, (valid + length - 1) / length, tail);
                if (lane == 0) P.long_sums[atomicAdd(P.long_count, 1u)] = make_uint4(chunk, last, tail, 0);
            }
        }
    }
    const bool mine = c < P.d;
    const int bytes = max(0, min(P.d - c, N)) * static_cast<int>(sizeof(TX));
    const TX* src = static_cast<const TX*>(P.src) + c;
    const unsigned int ld = static_cast<unsigned int>(P.ld_src);
    const uint32_t slot = smem_u32(ring + threadIdx.x);
    const auto get = [&](unsigned int k) { return k + lane < stop ? items[k + lane] : make_uint2(NO_KEY, 0); };
    if (i != begin || i + 32 > stop) item = get(i);
    // the rows of batch b of those 32 items, the first of them number `first`
    const auto fetch = [&](unsigned int first, const uint2& from, int b) {
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            const unsigned int t = __shfl_sync(~0u, from.y, b * BATCH + u);
            if (mine && first + b * BATCH + u < stop)
                copy_async(slot + (b % BATCHES * BATCH + u) * 4096, src + static_cast<unsigned long long>(t) * ld, bytes);
        }
        copy_commit();
    };
    if (i < stop) {
#pragma unroll
        for (int b = 0; b < BATCHES; ++b) fetch(i, item, b);
    }
    // rows that no token names, while the first rows come
    const int fill = static_cast<int>(blockIdx.x) - fill_first;
    if (fill >= 0) fill_rows<TD, WHOLE, true>(P, 0, P.unfilled, fill, gridDim.x - fill_first);
    if (i >= stop) return;
    unsigned int cur = __shfl_sync(~0u, item.x, 0);
    Sum<N> sum;
    sum.clear();
    const auto flush = [&](bool part, int after) {
        if (!mine) return;
        if (part) {
            float x[N];
            sum.values(x);
            store_columns(partial_at(P, chunk, after, c), x, N);
        } else {
            store_sum<TD>(P, cur, c, sum);
        }
    };
    for (; i < stop; i += 32) {
        const uint2 next = get(i + 32);
        unsigned int before = __shfl_up_sync(~0u, item.x, 1);
        if (lane == 0) before = cur;
        const unsigned int begins = __ballot_sync(~0u, item.x != before);
        const int count = min(32u, stop - i);
#pragma unroll 1
        for (int b = 0; b < 32 / BATCH; ++b) {
            copy_wait<BATCHES - 1>();
#pragma unroll
            for (int u = 0; u < BATCH; ++u) {
                const int j = b * BATCH + u;
                if (j >= count) break;
                if (begins >> j & 1) {
                    flush(open, 0);
                    cur = __shfl_sync(~0u, item.x, j), open = false;
                    sum.clear();
                }
                sum.template add<TX>(ring[(b % BATCHES * BATCH + u) * 256 + threadIdx.x]);
            }
            if (b + BATCHES < 32 / BATCH) fetch(i, item, b + BATCHES);
            else fetch(i + 32, next, b + BATCHES - 32 / BATCH);
        }
        item = next;
    }
    copy_wait<0>();
    flush(open || goes_on, open ? 0 : 1);
}

// The long sums, 128 columns of one at a time: eight warps add their shares of its
// parts, then one warp the shares.  Bound by latency, 3 to 6 us (one group for all parts
// of a sum took 30 us for 92 of them).
template <class TD>
__global__ void __launch_bounds__(256) embed_join_kernel(const EmbedParams P)
{
    __shared__ float4 share[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int slices = (P.d + 127) / 128;
    grid_dependency_wait();
    const int work = static_cast<int>(*P.long_count) * slices;   // (at most chunks x slices)
    for (int w = blockIdx.x; w < P.chunks * slices; w += gridDim.x) {
        const uint4 item = P.long_sums[w / slices];   // with the count, on its way together with it
        if (w >= work) return;
        const int first = item.x, last = item.y, c = (w % slices) * 128 + lane * 4;
        const unsigned int id = item.z;
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

// The widest groups that leave few threads without columns.
Groups groups(int d, int columns)
{
    const int units = (d + columns - 1) / columns;
    Groups best = {5, (units + 31) / 32};
    for (int shift = 6; shift <= 8; ++shift) {
        const int tiles = (units + (1 << shift) - 1) >> shift;
        if (tiles << shift <= best.tiles << best.shift || (tiles << shift) * 16 <= units * 17) best = {shift, tiles};
    }
    return best;
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

// A launch that may begin while the one before it in the stream still runs, and waits for
// it on the device.
template <class K, class... A>
cudaError_t launch_behind(K kern, int ctas, int threads, size_t smem, cudaStream_t stream, const A&... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kern, args...);
}

template <class TE, class TX, bool WHOLE, int ROWS>
cudaError_t rows(const EmbedParams& p, const Groups& g, cudaStream_t stream)
{
    const int each = ROWS * (256 >> g.shift);
    embed_rows_kernel<TE, TX, WHOLE, ROWS><<<dim3(static_cast<unsigned int>((p.n + each - 1) / each), g.tiles), 256, 0, stream>>>(p, g);
    return cudaGetLastError();
}

// An X that L2 would not hold for its reader is stored past the table's rows there: 26 us
// against 29 us for 32768 x 2048 (134 MB).
constexpr double STREAM_BYTES = 64e6;

template <class TE, class TX, bool WHOLE>
cudaError_t rows(EmbedParams p, int sms, cudaStream_t stream)
{
    const Groups g = groups(p.d, 8);
    p.stream = static_cast<double>(p.n) * p.d * sizeof(TX) > STREAM_BYTES;
    return (p.n * g.tiles << g.shift) < 2048ll * sms ? rows<TE, TX, WHOLE, 1>(p, g, stream) : rows<TE, TX, WHOLE, 4>(p, g, stream);
}

template <class TX, class TD, bool WHOLE>
cudaError_t sums(const EmbedParams& p, int sms, cudaStream_t stream)
{
    static std::atomic<unsigned long long> configured{0};
    constexpr size_t smem = BATCH * BATCHES * 256 * sizeof(uint4);
    const cudaError_t e = allow_smem(embed_sum_kernel<TX, TD, WHOLE>, smem, configured);
    if (e != cudaSuccess) return e;
    const Groups g = groups(p.d, COLS<TX>);
    const int per = 256 >> g.shift;
    const int ctas = static_cast<int>((static_cast<long long>(p.chunks) * g.tiles + per - 1) / per);
    // rows of no token: by the CTAs of the sums, or, of fewer than run at once, by others beside them
    const int fill = ctas < 3 * sms ? std::min(3 * sms, (p.unfilled + 7) / 8) : 0;
    return launch_behind(embed_sum_kernel<TX, TD, WHOLE>, ctas + fill, 256, smem, stream, p, g, fill ? ctas : 0);
}

template <class TX, class TD, bool WHOLE>
cudaError_t one(const EmbedParams& p, int sms, cudaStream_t stream)
{
    const int ctas = std::min(2 * sms, p.vocab), rows_each = (p.vocab + ctas - 1) / ctas;
    constexpr int tile = 32 * COLS<TX>;
    const int tiles = (p.d + tile - 1) / tile, ranges = std::max(1, ONE_WARPS / tiles);
    const size_t smem = sizeof(unsigned int) * (2 * EMBED_ONE + (rows_each + 127) / 128 * 4) +
                        (ranges > 1 ? sizeof(float) * ranges * 2 * tiles * tile : 0);
    static std::atomic<unsigned long long> configured{0};
    const cudaError_t e = allow_smem(embed_one_kernel<TX, TD, WHOLE>, sizeof(unsigned int) * (2 * EMBED_ONE + EMBED_VOCAB_MAX / 32 + 4) +
                                         sizeof(float) * ONE_WARPS * 2 * tile, configured);
    if (e != cudaSuccess) return e;
    embed_one_kernel<TX, TD, WHOLE><<<ctas, ONE_THREADS, smem, stream>>>(p, rows_each);
    return cudaGetLastError();
}

// What a launch that places tokens sets to 0 beside that: what HBM takes in the 6 us that it
// runs anyway (a launch that counts is too short to gain from it).
constexpr double FILL_BYTES = 24e6;

Fill take_fill(EmbedParams& p, size_t element, int ctas)
{
    Fill f = {p.unfilled, p.unfilled, 0};
    if (ctas <= 0) return f;   // (the sort itself has a CTA for every SM)
    f.first = static_cast<int>(std::max(0.0, p.unfilled - FILL_BYTES / (static_cast<double>(p.d) * element)));
    f.ctas = std::min(ctas, f.last - f.first);
    p.unfilled = f.first;
    return f;
}

template <class TD, bool WHOLE>
cudaError_t order(EmbedParams& p, int sms, cudaStream_t stream)
{
    const int n = static_cast<int>(p.n), order_ctas = (n + ORDER_TOKENS - 1) / ORDER_TOKENS;
    const Fill fill = take_fill(p, sizeof(TD), sms);
    const int words_each = ((p.unfilled + 31) / 32 + order_ctas - 1) / order_ctas;
    static std::atomic<unsigned long long> configured{0};
    const cudaError_t e = allow_smem(embed_order_kernel<TD, WHOLE>, EMBED_VOCAB_MAX / 8, configured);
    if (e != cudaSuccess) return e;
    embed_order_kernel<TD, WHOLE><<<order_ctas + fill.ctas, ORDER_THREADS, sizeof(unsigned int) * words_each, stream>>>(p, fill, order_ctas, words_each);
    return cudaGetLastError();
}

template <bool FIRST>
cudaError_t count(const EmbedParams& p, const SortPass& s, cudaStream_t stream)
{
    if (!FIRST) return launch_behind(embed_count_kernel<FIRST>, s.ctas, SORT_THREADS, 0, stream, p, s);
    embed_count_kernel<FIRST><<<s.ctas, SORT_THREADS, 0, stream>>>(p, s);
    return cudaGetLastError();
}

template <class TD, bool WHOLE, bool FIRST>
cudaError_t place(const EmbedParams& p, const SortPass& s, cudaStream_t stream)
{
    static std::atomic<unsigned long long> configured{0};
    const cudaError_t e = allow_smem(embed_place_kernel<TD, WHOLE, FIRST>, sizeof(unsigned int) * SORT_WARPS << 10, configured);
    if (e != cudaSuccess) return e;
    return launch_behind(embed_place_kernel<TD, WHOLE, FIRST>, s.ctas + s.fill.ctas, SORT_THREADS,
                         sizeof(unsigned int) * SORT_WARPS << s.bits, stream, p, s);
}

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

template <class TD, bool WHOLE>
cudaError_t sort_launch(EmbedParams& p, int launch, int sms, cudaStream_t stream)
{
    SortPass s = sort_pass(p, launch / 2);
    s.fill = take_fill(p, sizeof(TD), launch % 2 ? sms - s.ctas : 0);
    switch (launch) {
    case 0: return count<true>(p, s, stream);
    case 1: return place<TD, WHOLE, true>(p, s, stream);
    case 2: return count<false>(p, s, stream);
    default: return place<TD, WHOLE, false>(p, s, stream);
    }
}

template <class TD>
cudaError_t join(const EmbedParams& p, int sms, cudaStream_t stream)
{
    return launch_behind(embed_join_kernel<TD>, 8 * sms, 256, 0, stream, p);
}

}  // namespace

// Sorted tokens of the longest chunk, eight at a time (a place behind it still has 32 bits).
constexpr double CHUNK_MOST = 1e6;

EmbedLayout embed_layout(long long n, int vocab, int d, int dtype_x, int sms, size_t at)
{
    EmbedLayout l = {};
    const auto take = [&](size_t bytes) {
        const size_t a = at;
        at = (at + bytes + 255) / 256 * 256;
        return a;
    };
    const Groups g = groups(d, dtype_x == 0 ? COLS<__nv_bfloat16> : COLS<float>);
    // twelve CTAs' worth of groups for every SM, of eight tokens at least (131072 x 4096 bf16:
    // 209 us, with eight 217, five 233, three 262)
    const double threads = 12.0 * sms * 256, per = static_cast<double>(n) * (g.tiles << g.shift) / threads;
    l.chunk = std::max(8, static_cast<int>(std::min(per / 8 + 1, CHUNK_MOST)) * 8);
    l.chunks = static_cast<int>((n + l.chunk - 1) / l.chunk);
    // Room for the chunks of n or of any fewer tokens, so that a batch's workspace serves shorter
    // ones: lengths go in steps, and fewer tokens may have more chunks.  A length is 8 or more,
    // and more than `per` unless it is the longest.
    const long long most_chunks = std::min((n + 7) / 8, std::max(static_cast<long long>(std::ceil(threads / (g.tiles << g.shift))),
                                                                 static_cast<long long>(n / (8 * CHUNK_MOST)) + 1));
    l.sorted = take(n * sizeof(uint2));
    l.counts = take(2 * sizeof(unsigned int));
    l.long_sums = take(most_chunks * sizeof(uint4));
    l.partials = take(sizeof(float) * 2 * most_chunks * static_cast<size_t>((d + 7) / 8 * 8));
    l.present = take((vocab + 31) / 32 * sizeof(unsigned int));
    if (n > EMBED_FEW) {
        int bits = 1;
        while ((1 << bits) < vocab) ++bits;
        l.low = bits > 10 ? (bits + 1) / 2 : bits, l.high = bits - l.low;
        // up to 64 CTAs of few rounds, then up to 256 of many
        const auto ctas = [&](long long tokens) { return (n + tokens - 1) / tokens; };   // of so many each
        const long long rounds = std::max(ctas(64 * SORT_THREADS), 1ll), most = ctas(256 * SORT_THREADS);
        l.sort_each = static_cast<unsigned int>(std::max(std::min<long long>(rounds, ROUNDS), most) * 32);
        l.sort_ctas = static_cast<int>(ctas(l.sort_each * SORT_WARPS));
        // (room as above: fewer tokens have up to 64 CTAs, or up to 256 of ROUNDS)
        const size_t most_ctas = std::min(ctas(SORT_THREADS), std::max(64ll, std::min(256ll, ctas(ROUNDS * SORT_THREADS))));
        l.between = take(n * sizeof(uint2));
        l.hist[0] = take(sizeof(unsigned int) * most_ctas << l.low);
        l.hist[1] = take(sizeof(unsigned int) * most_ctas << l.high);
    }
    l.total = at;
    return l;
}

namespace {

// f with the types and the width's rest of a call
template <class F>
cudaError_t by_type(int dtype, int d, const F& f)
{
    if (dtype == 0) return d % 8 ? f(__nv_bfloat16(), std::false_type()) : f(__nv_bfloat16(), std::true_type());
    return d % 8 ? f(float(), std::false_type()) : f(float(), std::true_type());
}

}  // namespace

cudaError_t launch_embed_rows(const EmbedParams& p, int dtype_src, int dtype_dst, int sms, cudaStream_t stream)
{
    return by_type(dtype_dst, p.d, [&](auto x, auto whole) {
        using TX = decltype(x);
        constexpr bool WHOLE = decltype(whole)::value;
        return dtype_src == 0 ? rows<__nv_bfloat16, TX, WHOLE>(p, sms, stream) : rows<float, TX, WHOLE>(p, sms, stream);
    });
}

cudaError_t launch_embed_one(const EmbedParams& p, int dtype_src, int dtype_dst, int sms, cudaStream_t stream)
{
    return by_type(dtype_dst, p.d, [&](auto x, auto whole) {
        using TD = decltype(x);
        constexpr bool WHOLE = decltype(whole)::value;
        return dtype_src == 0 ? one<__nv_bfloat16, TD, WHOLE>(p, sms, stream) : one<float, TD, WHOLE>(p, sms, stream);
    });
}

cudaError_t launch_embed_order(EmbedParams& p, int dtype_dst, int sms, cudaStream_t stream)
{
    return by_type(dtype_dst, p.d, [&](auto x, auto whole) { return order<decltype(x), decltype(whole)::value>(p, sms, stream); });
}

cudaError_t launch_embed_sort(EmbedParams& p, int launch, int dtype_dst, int sms, cudaStream_t stream)
{
    return by_type(dtype_dst, p.d, [&](auto x, auto whole) {
        return sort_launch<decltype(x), decltype(whole)::value>(p, launch, sms, stream);
    });
}

cudaError_t launch_embed_sums(const EmbedParams& p, int dtype_src, int dtype_dst, int sms, cudaStream_t stream)
{
    return by_type(dtype_dst, p.d, [&](auto x, auto whole) {
        using TD = decltype(x);
        constexpr bool WHOLE = decltype(whole)::value;
        return dtype_src == 0 ? sums<__nv_bfloat16, TD, WHOLE>(p, sms, stream) : sums<float, TD, WHOLE>(p, sms, stream);
    });
}

cudaError_t launch_embed_join(const EmbedParams& p, int dtype_dst, int sms, cudaStream_t stream)
{
    return dtype_dst == 0 ? join<__nv_bfloat16>(p, sms, stream) : join<float>(p, sms, stream);
}

}  // namespace cola
