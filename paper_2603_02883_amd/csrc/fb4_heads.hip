// C ABI of the FB4 quantizer library, the attention path itself: norms and rotation of queries and keys, the choice of key
// blocks, attention over them.  Declarations and contracts are in include/fb4.h.
#include <algorithm>
#include <cmath>

#include "fb4_block_attention.hpp"
#include "fb4_common.hpp"
#include "fb4_rope.hpp"

using namespace fb4;

namespace {

constexpr int64_t kMaxTokens = 0x7FFFFFFF;
constexpr int64_t kMaxThreads = 0xFFFFFFFFll;       // of a launch
constexpr int64_t kMaxWorkgroups = (1 << 24) - 1;   // ... of 256 threads each

// (batch, head, token) strides in elements to units of 8: what the kernels count in.
template <typename T>
int strides_of(const int64_t* strides, T* out)
{
    for (int i = 0; i < 3; ++i) {
        if (strides[i] < 0) return FB4_ERR_INVALID_ARG;
        if (strides[i] % 8 || strides[i] / 8 > 0xFFFFFFFFll) return FB4_ERR_UNSUPPORTED;
    }
    *out = T{(uint32_t)(strides[0] / 8), (uint32_t)(strides[1] / 8), (uint32_t)(strides[2] / 8)};
    return FB4_OK;
}

// What the choice of blocks and the attention have in common.
int check_blocks(int64_t batch, int heads, int heads_k, int64_t tokens_q, int64_t tokens_k, int64_t dim, int block_q, int block_k, BlockShape* s)
{
    if (batch < 0 || heads < 1 || heads_k < 1 || tokens_q < 0 || tokens_k < 0 || dim < 1 || heads % heads_k) return FB4_ERR_INVALID_ARG;
    if ((block_q != 64 && block_q != 128) || (block_k != 64 && block_k != 128)) return FB4_ERR_UNSUPPORTED;
    if (heads > 65535 || dim % 8 || dim > 128 || tokens_q > kMaxTokens || tokens_k > kMaxTokens || batch > kMaxTokens) return FB4_ERR_UNSUPPORTED;
    *s = BlockShape{(uint32_t)tokens_q, (uint32_t)tokens_k, (uint16_t)heads, (uint16_t)heads_k, (uint16_t)block_q, (uint16_t)block_k,
                    (uint32_t)((tokens_q + block_q - 1) / block_q), (uint32_t)((tokens_k + block_k - 1) / block_k)};
    // (2^41 blocks are more than any memory holds; below that no product of sizes passes 64 bits)
    if ((double)batch * heads * s->blocks_q > 0x1p40 || (double)batch * heads_k * s->blocks_k > 0x1p40) return FB4_ERR_UNSUPPORTED;
    return FB4_OK;
}

// Parts of a block of queries' list, each with a workgroup of its own: the number with the least cost, in times of one tile of 64
// keys (about 1 us).  A compute unit with two pairs of wavefronts takes 0.7 of its rounds one after the other, three 2.1, four 2.8; a
// workgroup's start and end cost about a tile, the join two and 2 ps per row, part and channel.  At most four pairs of wavefronts
// for each of 256 compute units.  Over 98 calls of 8 to 400 blocks and 2 to 256 tiles the choice is 1.8 % slower than the best of 1 to
// 64 parts in the mean, over 72 of other shapes 3.6 % (512 / n parts wherever n <= 256: 6.6 % over the first).  8 single queries of 128
// channels, 256 tiles: 64 parts 18.8 us, one 350; 200 blocks of 64 queries of 72 channels: 64 tiles three parts 56.0 us, one 75.6; 8 tiles
// one part 13.5 us, two 17.3.
int64_t attention_parts(int64_t n, int64_t rows, int64_t dim, int64_t top, const BlockShape& s)
{
    const int64_t entries = top == FB4_ALL_BLOCKS ? s.blocks_k : top, tiles = s.block_k / 64, pairs = s.block_q / 64;
    if (n < 1 || entries < 2) return 1;
    const int64_t most = std::min<int64_t>(entries, 1024 / pairs / n);
    int64_t best = 1;
    double least = 0.0;
    for (int64_t p = 1; p <= most; p += 1 + p / 8) {
        const double rounds = std::max(1.0, 0.7 * (double)((n * p * pairs + 255) / 256));
        const double cost = rounds * (double)((entries + p - 1) / p * tiles + 1) + (p > 1 ? 2.0 + 2e-6 * (double)(rows * p * dim) : 0.0);
        if (p == 1 || cost < least) {
            best = p;
            least = cost;
        }
    }
    return best;
}

}  // namespace

extern "C" {

int fb4_qk_norm_rope(const void* q, const int64_t* q_strides, const void* k, const int64_t* k_strides, int64_t batch, int64_t tokens, int heads_q,
                     int heads_k, int64_t dim, int norm, const float* gamma_q, const float* gamma_k, float eps, const int32_t* positions,
                     int positions_shared, const double* freqs, const int32_t* axis_pairs, int n_axes, int pairing, void* q_out, void* k_out,
                     void* stream)
{
    if (batch < 0 || tokens < 0 || heads_q < 1 || heads_k < 0 || dim < 1 || (norm != 0 && norm != 1) ||
        (positions_shared != 0 && positions_shared != 1) || n_axes < 0 || (pairing != FB4_ROPE_ADJACENT && pairing != FB4_ROPE_HALVES))
        return FB4_ERR_INVALID_ARG;
    if (norm && !(eps >= 0.0f)) return FB4_ERR_INVALID_ARG;
    if (n_axes > 4) return FB4_ERR_UNSUPPORTED;
    if (n_axes > 0 && !axis_pairs) return FB4_ERR_INVALID_ARG;
    int64_t pairs = 0;
    uint8_t ends[4] = {0, 0, 0, 0};
    for (int a = 0; a < 4; ++a) {
        if (a < n_axes) {
            if (axis_pairs[a] < 1 || axis_pairs[a] > dim) return FB4_ERR_INVALID_ARG;
            pairs += axis_pairs[a];
        }
        if (2 * pairs > dim) return FB4_ERR_INVALID_ARG;
        ends[a] = (uint8_t)std::min<int64_t>(pairs, 255);
    }
    if (dim % 8 || dim > 256 || heads_q > 65535 || heads_k > 65535 || (pairing == FB4_ROPE_HALVES && pairs % 4)) return FB4_ERR_UNSUPPORTED;
    if (batch == 0 || tokens == 0) return FB4_OK;
    if (!q || !q_strides || !q_out || (heads_k > 0 && (!k || !k_strides || !k_out)) || (pairs > 0 && (!positions || !freqs))) return FB4_ERR_INVALID_ARG;
    RopeStrides sq = {0, 0, 0}, sk = {0, 0, 0};
    if (int rc = strides_of(q_strides, &sq)) return rc;
    if (heads_k > 0) {
        if (int rc = strides_of(k_strides, &sk)) return rc;
    }
    if (!aligned(q, 16) || !aligned(q_out, 16) || (heads_k > 0 && (!aligned(k, 16) || !aligned(k_out, 16))) || !aligned(gamma_q, 4) ||
        !aligned(gamma_k, 4) || !aligned(positions, 4) || !aligned(freqs, 8))
        return FB4_ERR_UNSUPPORTED;
    if (batch > (1 << 25) || tokens > (1 << 25) || batch * tokens > (1 << 25)) return FB4_ERR_UNSUPPORTED;   // (2^26 wavefronts to a launch)
    // Outputs on memory that another workgroup may still read.  In place a row is read and written by the same lanes, in that order.
    const int64_t row = dim * 2, size_q = batch * heads_q * tokens * row, size_k = batch * heads_k * tokens * row;
    const uintptr_t at_q = (uintptr_t)q_out, at_k = (uintptr_t)k_out;
    const RowSet rows_q(q_strides, batch, heads_q, tokens, row);
    if (!(rows_q.dense && q == q_out) && meets(rows_q, (uintptr_t)q, at_q, at_q + (uintptr_t)size_q)) return FB4_ERR_INVALID_ARG;
    if (heads_k > 0) {
        const RowSet rows_k(k_strides, batch, heads_k, tokens, row);
        if ((!(rows_k.dense && k == k_out) && meets(rows_k, (uintptr_t)k, at_k, at_k + (uintptr_t)size_k)) || meets(rows_q, (uintptr_t)q, at_k, at_k + (uintptr_t)size_k) ||
            meets(rows_k, (uintptr_t)k, at_q, at_q + (uintptr_t)size_q) || (at_q < at_k + (uintptr_t)size_k && at_k < at_q + (uintptr_t)size_q))
            return FB4_ERR_INVALID_ARG;
    }
    const int pieces = (int)(dim / 8);
    // A wavefront per run of tokens; several, each with some of the heads, while there are few tokens: up to 8192 wavefronts (16384: the
    // permuted input of fb4_rope.hpp 58.5 us and not 61, the packed one 87 and not 83; 4096: 66 and 82).
    const int64_t n = batch * tokens, rows = 64 / pieces, runs = (n + rows - 1) / rows;
    const int64_t heads = heads_q + heads_k, most = std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(heads, 255), 8192 / runs));
    const int64_t each = (heads + most - 1) / most, chunks = (heads + each - 1) / each;
    const RopeShape s = {(uint32_t)tokens, (uint32_t)n, (uint16_t)heads_q, (uint16_t)heads_k, eps, (uint8_t)pieces, {ends[0], ends[1], ends[2]},
                         (uint8_t)n_axes, (uint8_t)pairs, (uint8_t)((norm ? kRopeNorm : 0) | (positions_shared ? kRopeShared : 0)), (uint8_t)chunks};
    const dim3 grid((unsigned)((runs + kRopeThreads / 64 - 1) / (kRopeThreads / 64) * chunks));
#define FB4_ROPE_LAUNCH(pairing_) launch(qk_norm_rope_kernel<pairing_>, grid, dim3(kRopeThreads), 0, static_cast<hipStream_t>(stream), static_cast<const uint16_t*>(q), static_cast<const uint16_t*>(k), static_cast<uint16_t*>(q_out), static_cast<uint16_t*>(k_out), gamma_q, gamma_k, freqs, positions, sq, sk, s)
    if (pairing == FB4_ROPE_ADJACENT) FB4_ROPE_LAUNCH(kRopeAdjacent);
    else FB4_ROPE_LAUNCH(kRopeHalves);
#undef FB4_ROPE_LAUNCH
    return hipGetLastError() == hipSuccess ? FB4_OK : FB4_ERR_HIP;
}

size_t fb4_select_key_blocks_workspace(int64_t batch, int heads, int heads_k, int64_t tokens_q, int64_t tokens_k, int64_t dim, int block_q, int block_k)
{
    BlockShape s;
    if (check_blocks(batch, heads, heads_k, tokens_q, tokens_k, dim, block_q, block_k, &s) != FB4_OK) return 0;
    return (size_t)batch * ((size_t)heads * s.blocks_q + (size_t)heads_k * s.blocks_k) * (size_t)dim * sizeof(double);
}

int fb4_select_key_blocks(const void* q, const void* k, int64_t batch, int heads, int heads_k, int64_t tokens_q, int64_t tokens_k, int64_t dim,
                          const int32_t* lens, int block_q, int block_k, int64_t top, int32_t* blocks, float* scores, void* workspace,
                          size_t workspace_bytes, void* stream)
{
    BlockShape s;
    if (int rc = check_blocks(batch, heads, heads_k, tokens_q, tokens_k, dim, block_q, block_k, &s)) return rc;
    if (top < 0) return FB4_ERR_INVALID_ARG;
    if (batch == 0 || tokens_q == 0 || top == 0) return FB4_OK;
    if (!q || (tokens_k > 0 && !k) || !blocks || !workspace) return FB4_ERR_INVALID_ARG;
    if (workspace_bytes < fb4_select_key_blocks_workspace(batch, heads, heads_k, tokens_q, tokens_k, dim, block_q, block_k)) return FB4_ERR_INVALID_ARG;
    const int64_t n_q = batch * heads * s.blocks_q, n_k = batch * heads_k * s.blocks_k;
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(lens, 4) || !aligned(blocks, 4) || !aligned(scores, 4) || !aligned(workspace, 16)) return FB4_ERR_UNSUPPORTED;
    const int values = s.blocks_k <= 128 ? 2 : s.blocks_k <= 512 ? 8 : s.blocks_k <= 1024 ? 16 : 32;
    const uint32_t rows = 16 * select_sets(values), row_tiles = (s.blocks_q + rows - 1) / rows;
    if (s.blocks_k > kSelectMaxBlocks || n_q + n_k > kMaxWorkgroups || batch * heads * row_tiles * select_threads(values) > kMaxThreads || top > kMaxTokens)
        return FB4_ERR_UNSUPPORTED;
    hipStream_t st = static_cast<hipStream_t>(stream);
    double* means = static_cast<double*>(workspace);
    const uint32_t pieces = (uint32_t)(dim / 8);
    const dim3 grid((unsigned)(n_q + n_k));
#define FB4_MEANS(l) launch(block_means_kernel<l>, grid, dim3(kMeanThreads), 0, st, static_cast<const uint16_t*>(q), static_cast<const uint16_t*>(k), lens, means, (uint32_t)n_q, pieces, s)
    if (pieces > 8) FB4_MEANS(16);
    else if (pieces > 4) FB4_MEANS(8);
    else FB4_MEANS(4);
#undef FB4_MEANS
    const dim3 sgrid((unsigned)(batch * heads * row_tiles));
#define FB4_SELECT_LAUNCH(d, v) launch(select_blocks_kernel<d, v>, sgrid, dim3(select_threads(v)), 0, st, means, lens, blocks, scores, (uint32_t)top, (uint32_t)n_q, (uint32_t)dim, row_tiles, sgrid.x, s)
#define FB4_SELECT_CASE(d)                                       \
    case d:                                                      \
        if (values == 2) FB4_SELECT_LAUNCH(d, 2);                \
        else if (values == 8) FB4_SELECT_LAUNCH(d, 8);           \
        else if (values == 16) FB4_SELECT_LAUNCH(d, 16);         \
        else FB4_SELECT_LAUNCH(d, 32);                           \
        break;
    switch ((dim + 15) / 16) {
        FB4_SELECT_CASE(1) FB4_SELECT_CASE(2) FB4_SELECT_CASE(3) FB4_SELECT_CASE(4)
        FB4_SELECT_CASE(5) FB4_SELECT_CASE(6) FB4_SELECT_CASE(7) FB4_SELECT_CASE(8)
    }
#undef FB4_SELECT_CASE
#undef FB4_SELECT_LAUNCH
    return hipGetLastError() == hipSuccess ? FB4_OK : FB4_ERR_HIP;
}

size_t fb4_block_attention_workspace(int64_t batch, int heads, int heads_k, int64_t tokens_q, int64_t tokens_k, int64_t dim, int64_t top, int block_q,
                                     int block_k)
{
    BlockShape s;
    if (check_blocks(batch, heads, heads_k, tokens_q, tokens_k, dim, block_q, block_k, &s) != FB4_OK || top < FB4_ALL_BLOCKS) return 0;
    const int64_t parts = attention_parts(batch * heads * s.blocks_q, batch * heads * tokens_q, dim, top, s);
    return parts > 1 ? (size_t)(parts * batch * heads * tokens_q * (dim + 2)) * sizeof(float) : 0;
}

int fb4_block_attention(const void* q, const void* k, const void* v, const int64_t* v_strides, int64_t batch, int heads, int heads_k, int64_t tokens_q,
                        int64_t tokens_k, int64_t dim, const int32_t* lens, const int32_t* blocks, int64_t top, int block_q, int block_k, float scale,
                        void* out, const int64_t* out_strides, float* lse, void* workspace, size_t workspace_bytes, void* stream)
{
    BlockShape s;
    if (int rc = check_blocks(batch, heads, heads_k, tokens_q, tokens_k, dim, block_q, block_k, &s)) return rc;
    if (top < FB4_ALL_BLOCKS || !(scale > 0.0f) || !std::isfinite(scale)) return FB4_ERR_INVALID_ARG;
    if (scale > 0x1p127f) return FB4_ERR_UNSUPPORTED;   // (times log2 e: no number)
    if (top == FB4_ALL_BLOCKS ? blocks != nullptr : top > 0 && !blocks) return FB4_ERR_INVALID_ARG;
    if (batch == 0 || tokens_q == 0) return FB4_OK;
    if (!q || !out || !out_strides || (tokens_k > 0 && (!k || !v || !v_strides))) return FB4_ERR_INVALID_ARG;
    const size_t needed = fb4_block_attention_workspace(batch, heads, heads_k, tokens_q, tokens_k, dim, top, block_q, block_k);
    if (workspace_bytes < needed || (needed > 0 && !workspace)) return FB4_ERR_INVALID_ARG;
    TensorStrides sv = {0, 0, 0}, so;
    if (tokens_k > 0) {
        if (int rc = strides_of(v_strides, &sv)) return rc;
        if (v_strides[2] >= 1 << 25) return FB4_ERR_UNSUPPORTED;   // (a tile's rows by 32-bit offsets)
    }
    if (int rc = strides_of(out_strides, &so)) return rc;
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16) || !aligned(lens, 4) || !aligned(blocks, 4) || !aligned(lse, 4) ||
        !aligned(workspace, 16))
        return FB4_ERR_UNSUPPORTED;
    const int64_t n = batch * heads * s.blocks_q;
    if (n > kMaxWorkgroups || top > kMaxTokens) return FB4_ERR_UNSUPPORTED;
    const int64_t parts = attention_parts(n, batch * heads * tokens_q, dim, top, s);
    const AttentionShape a = {s.tokens_q, s.tokens_k, (uint32_t)top, s.heads, s.heads_k, (uint8_t)(block_q / 64), (uint8_t)(block_k / 64),
                              (uint16_t)parts, s.blocks_q, (uint32_t)(n * parts), scale};
    hipStream_t st = static_cast<hipStream_t>(stream);
    const dim3 grid((unsigned)(n * parts));
#define FB4_ATTENTION_LAUNCH(p, w, split) launch(block_attention_kernel<p, w, split>, grid, dim3(64 * w), 0, st, static_cast<const uint16_t*>(q), static_cast<const uint16_t*>(k), static_cast<const uint16_t*>(v), static_cast<uint16_t*>(split ? workspace : out), lse, blocks, lens, sv, so, a)
#define FB4_ATTENTION_CASE(p)                                              \
    case p:                                                                \
        if (block_q == 64 && parts > 1) FB4_ATTENTION_LAUNCH(p, 2, true);  \
        else if (block_q == 64) FB4_ATTENTION_LAUNCH(p, 2, false);         \
        else if (parts > 1) FB4_ATTENTION_LAUNCH(p, 4, true);              \
        else FB4_ATTENTION_LAUNCH(p, 4, false);                            \
        break;
    switch (dim / 8) {
        FB4_ATTENTION_CASE(1) FB4_ATTENTION_CASE(2) FB4_ATTENTION_CASE(3) FB4_ATTENTION_CASE(4) FB4_ATTENTION_CASE(5) FB4_ATTENTION_CASE(6)
        FB4_ATTENTION_CASE(7) FB4_ATTENTION_CASE(8) FB4_ATTENTION_CASE(9) FB4_ATTENTION_CASE(10) FB4_ATTENTION_CASE(11) FB4_ATTENTION_CASE(12)
        FB4_ATTENTION_CASE(13) FB4_ATTENTION_CASE(14) FB4_ATTENTION_CASE(15) FB4_ATTENTION_CASE(16)
    }
#undef FB4_ATTENTION_CASE
#undef FB4_ATTENTION_LAUNCH
    if (parts > 1) {
        const int64_t rows = batch * heads * tokens_q;   // (at most 512 blocks; of more than eight parts 113)
        const bool many = parts > 8;
        launch(many ? join_parts_kernel<true> : join_parts_kernel<false>, dim3((unsigned)(many ? rows : (rows + 7) / 8)), dim3(256), 0, st,
               static_cast<const float*>(workspace), lens, static_cast<uint16_t*>(out), lse, so, (uint32_t)parts, (uint32_t)rows, s.tokens_q, (uint32_t)heads,
               (uint32_t)dim, scale);
    }
    return hipGetLastError() == hipSuccess ? FB4_OK : FB4_ERR_HIP;
}

}  // extern "C"
