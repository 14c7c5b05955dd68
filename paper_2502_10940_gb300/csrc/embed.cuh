// embed.cuh -- token embedding: rows of the table for token ids, and the
// table's gradient.
//
// Mathematics (table E [vocab x d], scale s, tokens t < n):
//   X_t = s E[id_t]   (0 where id_t names no token)
//   dE_v = s sum_{t: id_t = v} dX_t
// The sum's rows are found by sorting (id, t) by id, stably.  A token's rows are added
// in fp32 in the order of the tokens, or, where a sum crosses bounds between warps or
// chunks, in parts, which are added then.  The parts depend on the ids, n, vocab, d, the
// type of dX and the device alone, no two of them meet in an atomic: the same bits from
// every call.  A finished sum is scaled in fp32, then rounded to dE's type or added to dE
// (most columns by a reduction in memory, where no other sum goes).
#pragma once
#include <cuda_runtime.h>

#include <cstddef>

namespace cola {

constexpr int EMBED_VOCAB_MAX = 1 << 20;           // rows of a table: two digits of up to ten bits
constexpr long long EMBED_MAX_ROWS = 1ll << 28;    // tokens of a call stay below it
constexpr int EMBED_MAX_WIDTH = 1 << 20;
constexpr int EMBED_FEW = 8192;                    // tokens that are ordered in one launch
constexpr int EMBED_ONE = 2048;                    // tokens whose gradient is, of at most so many bytes of dX
constexpr long long EMBED_ONE_BYTES = 2 << 20;

struct EmbedParams {
    const long long* ids;
    const void* src;          // E, or dX
    void* dst;                // X, or dE
    long long n, ld_src, ld_dst;
    int vocab, d;
    float scale;
    int accumulate;           // the gradient is added into
    int stream;               // X is stored past L2
    // the gradient's workspace
    uint2* sorted;            // (id, token)
    unsigned int* count;      // tokens that name a row
    unsigned int* long_count; // sums that are split over chunks
    uint4* long_sums;         // of each the chunks that it begins and ends in, and its id
    float* partials;          // 2 per chunk, d rounded up to 8: of a sum that began before the chunk, and of one that goes on behind it
    int chunk, chunks;        // sorted tokens of a chunk; chunks of n
    unsigned int* present;    // a bit for each row below `unfilled` that a token names
    int unfilled;             // the rows of no token that are still to be set to 0 lie below this one
    // more than EMBED_FEW tokens
    uint2* between;           // after the first pass of the sort
    unsigned int* hist[2];
    int low, high;            // bits of the two digits (high 0: one pass)
    int sort_ctas;
    unsigned int sort_each;
};

// Byte offsets in the gradient's workspace, from `at` on, and the shares of the work.
struct EmbedLayout {
    size_t sorted, counts, long_sums, partials, between, present, hist[2], total;
    int chunk, chunks, low, high, sort_ctas;
    unsigned int sort_each;
};
EmbedLayout embed_layout(long long n, int vocab, int d, int dtype_x, int sms, size_t at);

// dtypes: cola_dtype_t of src and dst
cudaError_t launch_embed_rows(const EmbedParams& p, int dtype_src, int dtype_dst, int sms, cudaStream_t stream);
// The gradient of up to EMBED_ONE tokens of EMBED_ONE_BYTES.
cudaError_t launch_embed_one(const EmbedParams& p, int dtype_src, int dtype_dst, int sms, cudaStream_t stream);
// The order of up to EMBED_FEW tokens; that of more, in launches 0 .. 3 (0 and 1 where high
// is 0).  They also set rows to 0, and lower p.unfilled.
cudaError_t launch_embed_order(EmbedParams& p, int dtype_dst, int sms, cudaStream_t stream);
cudaError_t launch_embed_sort(EmbedParams& p, int launch, int dtype_dst, int sms, cudaStream_t stream);
cudaError_t launch_embed_sums(const EmbedParams& p, int dtype_src, int dtype_dst, int sms, cudaStream_t stream);
cudaError_t launch_embed_join(const EmbedParams& p, int dtype_dst, int sms, cudaStream_t stream);   // where chunks > 1

}  // namespace cola
