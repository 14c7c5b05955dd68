// embed.cuh -- token embedding: rows of the table for token ids, and the
// table's gradient.
//
// Mathematics (table E [vocab x d], scale s, tokens t < n):
//   X_t = s E[id_t]   (0 where id_t names no token)
//   dE_v = s sum_{t: id_t = v} dX_t
// The sum's rows are found by sorting (id, t) by id, stably, so that every
// token's rows are added in the order of the tokens: no atomics on values,
// and the same bits from every call.
#pragma once
#include <cuda_runtime.h>

#include <cstddef>

namespace cola {

constexpr int EMBED_VOCAB_MAX = 1 << 20;           // rows of a table: two digits of up to ten bits
constexpr long long EMBED_MAX_ROWS = 1ll << 28;    // tokens of a call stay below it
constexpr int EMBED_MAX_WIDTH = 1 << 20;

struct EmbedParams {
    const long long* ids;
    const void* src;          // E, or dX
    void* dst;                // X, or dE
    long long n, ld_src, ld_dst;
    int vocab, d;
    float scale;
    int accumulate;
    // the gradient's workspace
    uint2* pairs[2];          // n each: (id, token); the sorted ones in [1]
    unsigned int* count;      // tokens that name a row
    unsigned int* present;    // a bit per row of the table
    float* partials;          // 2 per chunk, d rounded up to 8: of a sum that began before the chunk, and of one that goes on behind it
    int chunk, chunks;        // sorted tokens of a chunk; chunks of n
};

// Byte offsets in the gradient's workspace, from `at` on.
struct EmbedLayout {
    size_t pairs[2], count, present, partials, total;
    int chunk, chunks;
};
EmbedLayout embed_layout(long long n, int vocab, int d, int sms, size_t at);

// dtypes: cola_dtype_t of src and dst
cudaError_t launch_embed_rows(const EmbedParams& p, int dtype_src, int dtype_dst, cudaStream_t stream);
cudaError_t launch_embed_sort(const EmbedParams& p, cudaStream_t stream);
cudaError_t launch_embed_sums(const EmbedParams& p, int dtype_src, int dtype_dst, int sms, cudaStream_t stream);
cudaError_t launch_embed_join(const EmbedParams& p, int dtype_dst, cudaStream_t stream);   // where chunks > 1

}  // namespace cola
