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
template <class TE, class TX>
__global__ void __launch_bounds__(256) embed_rows_kernel(const EmbedParams P)
{
    const int units = (P.d + 7) / 8;
    const long long i = blockIdx.x * 256ll + threadIdx.x, t = i / units;
    if (t >= P.n) return;
    const int c = static_cast<int>(i - t * units) * 8, left = P.d - c;
    const long long id = P.ids[t];
    float x[8] = {};
    if (id >= 0 && id < P.vocab) {
        Eight<TE> e;
        e.load(static_cast<const TE*>(P.src) + id * P.ld_src + c, left);
        e.values(x);
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] *= P.scale;
    }
    Eight<TX>::store(static_cast<TX*>(P.dst) + t * P.ld_dst + c, x, left);
}

// ------------------------------------------------------------------- sorting
// Tokens sorted by id: one or two passes of a stable counting sort by up to ten
// bits, in one cluster of CTAs.  Every warp has consecutive tokens; it counts
// its digits, the counts become first places (over the warps of a CTA, the CTAs
// and the digits), and the warp hands the places out again in order.
constexpr int SORT_THREADS = 1024, SORT_WARPS = 32;

struct SortShared {
    unsigned int total[1024];          // of each digit in this CTA; read by the others
    unsigned int warp_sum[SORT_WARPS];
    unsigned int valid;
    unsigned int place[1];             // [warp][digit]
};

__device__ __forceinline__ unsigned int ld_cluster_u32(uint32_t addr)
{
    unsigned int v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}

// FIRST: from the ids (those that name no token are left out), else from pairs.
template <bool FIRST>
__device__ __forceinline__ void sort_pass(const EmbedParams& P, SortShared& S, const uint2* from, uint2* to, unsigned int n,
                                          int shift, int bits, bool last, int rank, int ctas)
{
    const int digits = 1 << bits, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    unsigned int* mine = S.place + (warp << bits);
    for (int i = lane; i < digits; i += 32) mine[i] = 0;
    __syncwarp();
    const unsigned int each = (n + ctas * SORT_THREADS - 1) / (ctas * SORT_THREADS) * 32;   // tokens of a warp
    const unsigned int begin = min(n, (rank * SORT_WARPS + warp) * each), end = min(n, begin + each);
    const auto get = [&](unsigned int i, uint2& item) -> bool {
        if (i >= end) return false;
        if (!FIRST) {
            item = from[i];
            return true;
        }
        const long long id = P.ids[i];
        item = make_uint2(static_cast<unsigned int>(id), i);
        return id >= 0 && id < P.vocab;
    };
    uint2 item;
    for (unsigned int i = begin + lane; i - lane < end; i += 32)
        if (get(i, item)) atomicAdd(mine + (item.x >> shift & (digits - 1)), 1u);
    __syncthreads();
    const int b = threadIdx.x;
    unsigned int sum = 0;
    if (b < digits) {
        for (int w = 0; w < SORT_WARPS; ++w) {
            const unsigned int c = S.place[(w << bits) + b];
            S.place[(w << bits) + b] = sum;
            sum += c;
        }
        S.total[b] = sum;
    }
    cluster_sync();
    unsigned int before = 0, all = 0;
    if (b < digits)
        for (int r = 0; r < ctas; ++r) {
            const unsigned int c = ld_cluster_u32(mapa_shared(smem_u32(S.total + b), r));
            if (r < rank) before += c;
            all += c;
        }
    // first place of each digit: a scan over the threads
    unsigned int up = all;
#pragma unroll
    for (int k = 1; k < 32; k <<= 1) {
        const unsigned int v = __shfl_up_sync(~0u, up, k);
        if (lane >= k) up += v;
    }
    if (lane == 31) S.warp_sum[warp] = up;
    __syncthreads();
    unsigned int base = up - all + before;
    for (int w = 0; w < warp; ++w) base += S.warp_sum[w];
    if (b < digits)
        for (int w = 0; w < SORT_WARPS; ++w) S.place[(w << bits) + b] += base;
    if (b == SORT_THREADS - 1) S.valid = base - before + all;
    __syncthreads();
    for (unsigned int i = begin + lane; i - lane < end; i += 32) {
        const bool there = get(i, item);
        const unsigned int digit = there ? item.x >> shift & (digits - 1) : ~0u;
        const unsigned int peers = __match_any_sync(~0u, digit), below = peers & ((1u << lane) - 1);
        unsigned int at = 0;
        if (there) at = mine[digit] + __popc(below);
        __syncwarp();
        if (there) {
            if (below == 0) mine[digit] += __popc(peers);
            to[at] = item;
            if (last) atomicOr(P.present + (item.x >> 5), 1u << (item.x & 31));
        }
        __syncwarp();
    }
    cluster_sync();
}

__global__ void __launch_bounds__(SORT_THREADS) embed_sort_kernel(const EmbedParams P, int low, int high)
{
    extern __shared__ __align__(16) unsigned char smem[];
    SortShared& S = *reinterpret_cast<SortShared*>(smem);
    const int rank = cluster_ctarank(), ctas = gridDim.x;
    for (int i = rank * SORT_THREADS + threadIdx.x; i < (P.vocab + 31) / 32; i += ctas * SORT_THREADS) P.present[i] = 0;
    const unsigned int n = static_cast<unsigned int>(P.n);
    sort_pass<true>(P, S, nullptr, P.pairs[high ? 0 : 1], n, 0, low, high == 0, rank, ctas);
    const unsigned int valid = S.valid;
    __syncthreads();
    if (rank == 0 && threadIdx.x == 0) *P.count = valid;
    if (high) sort_pass<false>(P, S, P.pairs[0], P.pairs[1], valid, low, high, true, rank, ctas);
}

// ---------------------------------------------------------------------- sums
constexpr unsigned int NO_KEY = ~0u;

template <class TD>
__device__ __forceinline__ void store_sum(const EmbedParams& P, unsigned int id, int c, const float (&sum)[8])
{
    TD* p = static_cast<TD*>(P.dst) + id * P.ld_dst + c;
    float x[8] = {};
    if (P.accumulate) {
        Eight<TD> old;
        old.load(p, P.d - c);
        old.values(x);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = fmaf(P.scale, sum[k], x[k]);
    Eight<TD>::store(p, x, P.d - c);
}

__device__ __forceinline__ float* partial_at(const EmbedParams& P, int chunk, int after, int c)
{
    return P.partials + (chunk * 2ll + after) * ((P.d + 7) / 8 * 8) + c;
}

// `group` threads share a chunk of the sorted tokens, eight columns each; wider
// rows are shared by `tiles` such groups.  A sum that lies within the chunk is
// stored; of one that began before or goes on behind it the chunk's part is kept.
template <class TX, class TD>
__global__ void __launch_bounds__(256) embed_sum_kernel(const EmbedParams P, int group, int tiles, int sum_ctas)
{
    constexpr int U = 8;
    if (static_cast<int>(blockIdx.x) >= sum_ctas) {   // rows that no token names
        const int lane = threadIdx.x & 31;
        const float zero[8] = {};
        for (int v = (blockIdx.x - sum_ctas) * 8 + (threadIdx.x >> 5); v < P.vocab; v += (gridDim.x - sum_ctas) * 8)
            if (!(P.present[v >> 5] >> (v & 31) & 1))
                for (int c = lane * 8; c < P.d; c += 256) Eight<TD>::store(static_cast<TD*>(P.dst) + v * P.ld_dst + c, zero, P.d - c);
        return;
    }
    const int at = blockIdx.x * (256 / group) + threadIdx.x / group, chunk = at / tiles;
    const int c = ((at - chunk * tiles) * group + threadIdx.x % group) * 8;
    const unsigned int valid = *P.count, begin = static_cast<unsigned int>(chunk) * P.chunk;
    if (chunk >= P.chunks || begin >= valid || c >= P.d) return;
    const unsigned int end = min(valid, begin + P.chunk);
    const uint2* items = P.pairs[1];
    const TX* src = static_cast<const TX*>(P.src) + c;
    unsigned int cur = items[begin].x;
    bool open = begin > 0 && items[begin - 1].x == cur;
    const bool goes_on = end < valid && items[end].x == items[end - 1].x;
    float sum[8] = {};
    for (unsigned int i = begin; i < end; i += U) {
        uint2 item[U];
        Eight<TX> row[U];
#pragma unroll
        for (int u = 0; u < U; ++u) item[u] = i + u < end ? items[i + u] : make_uint2(NO_KEY, 0);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i + u < end) row[u].load(src + item[u].y * P.ld_src, P.d - c);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i + u >= end) break;
            if (item[u].x != cur) {
                if (open) Eight<float>::store(partial_at(P, chunk, 0, c), sum, 8);
                else store_sum<TD>(P, cur, c, sum);
                cur = item[u].x, open = false;
#pragma unroll
                for (int k = 0; k < 8; ++k) sum[k] = 0.f;
            }
            float x[8];
            row[u].values(x);
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] += x[k];
        }
    }
    if (open || goes_on) Eight<float>::store(partial_at(P, chunk, open ? 0 : 1, c), sum, 8);
    else store_sum<TD>(P, cur, c, sum);
}

// The sums that cross chunks, by the chunk that they begin in.
template <class TD>
__global__ void __launch_bounds__(256) embed_join_kernel(const EmbedParams P, int group, int tiles)
{
    const int at = blockIdx.x * (256 / group) + threadIdx.x / group, chunk = at / tiles;
    const int c = ((at - chunk * tiles) * group + threadIdx.x % group) * 8;
    const unsigned int valid = *P.count, begin = static_cast<unsigned int>(chunk) * P.chunk, end = begin + P.chunk;
    if (chunk >= P.chunks || end >= valid || c >= P.d) return;
    const uint2* items = P.pairs[1];
    const unsigned int id = items[end].x;
    if (items[end - 1].x != id || (begin > 0 && items[begin - 1].x == id)) return;
    unsigned int lo = end, hi = valid;   // the first place behind the id's tokens
    while (lo < hi) {
        const unsigned int mid = lo + (hi - lo) / 2;
        if (items[mid].x > id) hi = mid;
        else lo = mid + 1;
    }
    const int last = (lo - 1) / P.chunk;
    float sum[8], x[8];
    Eight<float> part;
    part.load(partial_at(P, chunk, 1, c), 8);
    part.values(sum);
    for (int i = chunk + 1; i <= last; ++i) {
        part.load(partial_at(P, i, 0, c), 8);
        part.values(x);
#pragma unroll
        for (int k = 0; k < 8; ++k) sum[k] += x[k];
    }
    store_sum<TD>(P, id, c, sum);
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
cudaError_t rows(const EmbedParams& p, cudaStream_t stream)
{
    const long long units = (p.d + 7) / 8 * p.n;
    embed_rows_kernel<TS, TD><<<static_cast<unsigned int>((units + 255) / 256), 256, 0, stream>>>(p);
    return cudaGetLastError();
}

template <class TS, class TD>
cudaError_t sums(const EmbedParams& p, int sms, cudaStream_t stream)
{
    const Groups g = groups(p.d);
    const int per = 256 / g.group;
    const int ctas = static_cast<int>((static_cast<long long>(p.chunks) * g.tiles + per - 1) / per);
    const int zero = p.accumulate ? 0 : std::min(4 * sms, (p.vocab + 7) / 8);
    embed_sum_kernel<TS, TD><<<ctas + zero, 256, 0, stream>>>(p, g.group, g.tiles, ctas);
    return cudaGetLastError();
}

template <class TD>
cudaError_t join(const EmbedParams& p, cudaStream_t stream)
{
    const Groups g = groups(p.d);
    const int per = 256 / g.group;
    const int ctas = static_cast<int>((static_cast<long long>(p.chunks) * g.tiles + per - 1) / per);
    embed_join_kernel<TD><<<ctas, 256, 0, stream>>>(p, g.group, g.tiles);
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
    l.pairs[0] = take(n * sizeof(uint2));
    l.pairs[1] = take(n * sizeof(uint2));
    l.count = take(sizeof(unsigned int));
    l.present = take((vocab + 31) / 32 * sizeof(unsigned int));
    l.partials = take(sizeof(float) * 2 * l.chunks * static_cast<size_t>((d + 7) / 8 * 8));
    l.total = at;
    return l;
}

cudaError_t launch_embed_rows(const EmbedParams& p, int dtype_src, int dtype_dst, cudaStream_t stream)
{
    using bf16 = __nv_bfloat16;
    if (dtype_src == 0) return dtype_dst == 0 ? rows<bf16, bf16>(p, stream) : rows<bf16, float>(p, stream);
    return dtype_dst == 0 ? rows<float, bf16>(p, stream) : rows<float, float>(p, stream);
}

cudaError_t launch_embed_sort(const EmbedParams& p, cudaStream_t stream)
{
    int bits = 1;
    while ((1 << bits) < p.vocab) ++bits;
    const int low = bits > 10 ? (bits + 1) / 2 : bits, high = bits - low;
    const size_t smem = sizeof(SortShared) + (sizeof(unsigned int) * SORT_WARPS << low);
    static std::atomic<unsigned long long> configured{0};   // bit d: set on device d
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !((configured.load(std::memory_order_acquire) >> dev) & 1ull)) {
        e = cudaFuncSetAttribute(embed_sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 static_cast<int>(sizeof(SortShared) + (sizeof(unsigned int) * SORT_WARPS << 10)));
        if (e != cudaSuccess) return e;
        if (dev < 64) configured.fetch_or(1ull << dev, std::memory_order_acq_rel);
    }
    int ctas = 1;
    while (ctas < 8 && ctas * 4096ll < p.n) ctas *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(SORT_THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, embed_sort_kernel, p, low, high);
}

cudaError_t launch_embed_sums(const EmbedParams& p, int dtype_src, int dtype_dst, int sms, cudaStream_t stream)
{
    using bf16 = __nv_bfloat16;
    if (dtype_src == 0) return dtype_dst == 0 ? sums<bf16, bf16>(p, sms, stream) : sums<bf16, float>(p, sms, stream);
    return dtype_dst == 0 ? sums<float, bf16>(p, sms, stream) : sums<float, float>(p, sms, stream);
}

cudaError_t launch_embed_join(const EmbedParams& p, int dtype_dst, cudaStream_t stream)
{
    return dtype_dst == 0 ? join<__nv_bfloat16>(p, stream) : join<float>(p, stream);
}

}  // namespace cola
