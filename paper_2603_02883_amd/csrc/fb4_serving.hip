// C ABI of the FB4 quantizer library, serving a few tokens at a time: few rows times FB4 weights, and the 8-bit cache of keys and values --
// its pages' plan, the store and the attention that reads it.  Declarations and contracts are in include/fb4.h.
#include <algorithm>
#include <cmath>

#include "fb4_cache_attention.hpp"
#include "fb4_cache_plan.hpp"
#include "fb4_cache_store.hpp"
#include "fb4_common.hpp"
#include "fb4_matvec.hpp"

using namespace fb4;

namespace {

constexpr int64_t kMaxInt = 0x7FFFFFFF;

// log2 of a page's tokens, -1 for a size that is not served.
int page_bits_of(int page) { return page == 16 ? 4 : page == 32 ? 5 : page == 64 ? 6 : page == 128 ? 7 : -1; }

// (head, token) strides in elements to units of 8.
template <typename T>
int strides_of(const int64_t* strides, T* out)
{
    for (int i = 0; i < 2; ++i) {
        if (strides[i] < 0) return FB4_ERR_INVALID_ARG;
        if (strides[i] % 8 || strides[i] / 8 > 0xFFFFFFFFll) return FB4_ERR_UNSUPPORTED;
    }
    *out = T{(uint32_t)(strides[0] / 8), (uint32_t)(strides[1] / 8)};
    return FB4_OK;
}

struct CachePlan {
    uint32_t tile_rows;
    bool split;
    int64_t positions;
};
// Tiles of few rows from which on a workgroup takes all keys of one, and keys up to which it does.  (A token each of sequences of up to 8192
// keys, 24 heads over 8, us, whole and in parts: 40 sequences 112, 105; 48 121, 124; 64 149, 160.  One sequence: 1024 keys 12.0, 14.9; 1536 16.5, 14.9.)
constexpr int kCacheFew = 384, kCacheShort = 1024;

// Sizes that are served, the tiles' size, and whether the keys are shared among workgroups.
int plan_attention(int64_t tokens, int heads, int heads_k, int64_t dim, int page, int64_t max_pages, int64_t batch, CachePlan* p)
{
    if (tokens < 0 || heads < 1 || heads_k < 1 || dim < 1 || max_pages < 0 || batch < 0 || heads % heads_k) return FB4_ERR_INVALID_ARG;
    const int bits = page_bits_of(page);
    if (bits < 0 || heads > 65535 || dim % 8 || dim > 128 || tokens > kMaxInt || max_pages > kMaxInt >> bits || batch > kCacheMaxBatch) return FB4_ERR_UNSUPPORTED;
    const int64_t rows = tokens * (heads / heads_k);
    if (rows > kMaxInt) return FB4_ERR_UNSUPPORTED;
    // 16 rows to a workgroup, or 128: by the rows of a sequence on average, as both cost alike from 40 to 64 on -- 64 sequences of up to 4096 keys, 24
    // heads over 8, us: 24 rows 121, 149; 39 145, 170; 48 173, 172; 66 209, 179; 192 458, 329; 8 sequences, 16 heads of 72 channels: 32 45, 52; 40 45, 46; 64
    // 52, 48 -- and where the rows beyond a token each are a long prompt's, which 16 at a time take twice as long, among many sequences of few or none.
    const bool many = rows > 40 * batch || rows >= 16384 + batch * (heads / heads_k);
    p->tile_rows = many ? kTileRows : 16;
    // (at least so many tiles have rows)
    const int64_t tiles = std::max((rows + p->tile_rows - 1) / p->tile_rows, batch) * heads_k, keys = max_pages << bits;
    p->split = many ? tiles <= (int64_t)kTilesTarget && tile_parts((uint32_t)tiles, (uint32_t)((keys + kCacheStep - 1) / kCacheStep * 16)) > 1 : tiles < kCacheFew && keys > kCacheShort;
    // (a sequence of S steps has at most S / share + 1 parts to a tile, which over all tiles is the target's number and one more each)
    p->positions = (rows / p->tile_rows + batch) * heads_k + (p->split ? many ? kTilesTarget : kCacheTarget : 0);
    if (p->positions > (1 << 24) - 1) return FB4_ERR_UNSUPPORTED;
    return FB4_OK;
}

}  // namespace

extern "C" {

int fb4_matvec(const fb4_luts* luts, const void* x, int64_t rows, int64_t x_row_stride, const uint8_t* codes, const uint16_t* meta, int64_t n, int64_t cols,
               int block, const float* bias, void* out, int out_dtype, int64_t out_row_stride, void* stream)
{
    if (!luts || rows < 0 || n < 0 || cols < 0 || x_row_stride < cols || out_row_stride < n || (block != 32 && block != 16) ||
        (out_dtype != FB4_DTYPE_BF16 && out_dtype != FB4_DTYPE_F32))
        return FB4_ERR_INVALID_ARG;
    if (rows > kMatvecMaxRows || cols % 32 || n > (1 << 28) - 32 || cols >= 1 << 25)   // (at most 16 threads to one of so many rows; 2^32 are no launch)
        return FB4_ERR_UNSUPPORTED;
    if (rows == 0 || n == 0) return FB4_OK;
    if (!out || (cols > 0 && (!x || !codes || !meta))) return FB4_ERR_INVALID_ARG;
    if (!aligned(x, 16) || (rows > 1 && cols > 0 && x_row_stride % 8) || (cols > 0 && x_row_stride / 8 > 0xFFFFFFFFll) || !aligned(codes, 16) || !aligned(meta, block == 16 ? 4 : 2) ||
        !aligned(bias, 4) || !aligned(out, out_dtype == FB4_DTYPE_F32 ? 4 : 2) || (rows > 1 && out_row_stride > 1ll << 40))
        return FB4_ERR_UNSUPPORTED;
    // Results on memory that other workgroups may still read (beside it, between its rows too, is none).
    const int64_t halves = out_dtype == FB4_DTYPE_F32 ? 2 : 1, results_strides[3] = {0, 0, out_row_stride * halves};
    const RowSet results(results_strides, 1, 1, rows, n * halves * 2);
    if (touches(results, out, codes, (uint64_t)n * cols / 2) || touches(results, out, meta, (uint64_t)n * (cols / block) * 2) ||
        touches(results, out, bias, (uint64_t)n * 4))
        return FB4_ERR_INVALID_ARG;
    if (touches(results, out, x, (uint64_t)(cols ? (rows > 1 ? (rows - 1) * x_row_stride : 0) + cols : 0) * 2)) {
        for (int64_t r = 0; r < rows; ++r) {
            if (touches(results, out, static_cast<const uint16_t*>(x) + r * x_row_stride, (uint64_t)cols * 2)) return FB4_ERR_INVALID_ARG;
        }
    }
    if (int rc = check_device(luts)) return rc;
    const int sets = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    const int64_t chunks = cols / 32;
    // Rows of the weights to a workgroup, 16 to a tile: each reads all of x, so the more rows x has the fewer workgroups, down to one or two per
    // compute unit.  (4096 channels, one, two and four tiles, us.  One row: 8192 rows of weights 6.9, 7.6, 11.5; 16384: 12.0, 11.0, 12.2; 49152 x
    // 8192: 53.6, 47.3, 43.4.  Four: 12288: 10.4, 11.2, 12.0.  Eight: 5120: 8.7, 7.5, 11.3; 24576: 22.2, 17.7, 19.6.  Sixteen: 8192: 11.6, 9.6,
    // 13.2; 12288: 16.1, 14.5, 13.4; 16384: 21.2, 15.0, 14.2.  Thirty-two: 12288: 27.0, 25.3, 18.3.  Sixty-four, one and two: 4096: 19.0, 21.6; 4610: 35.1, 21.8)
    const int tiles = sets < 4 && n > (rows > 8 ? 8192 : 32768) ? 4 : n > (rows > 4 ? 4096 : 12288) ? 2 : 1;
    const int64_t steps = (chunks + 3) / 4;
    const int waves = (int)std::max<int64_t>(1, std::min<int64_t>(steps, 8));
    const bool direct = tiles == 1 && steps <= 2 * waves;
    const MatvecShape s = {(uint32_t)n, (uint32_t)chunks, (uint32_t)(x_row_stride / 8), (uint32_t)waves, out_row_stride, (uint16_t)rows,
                           (uint16_t)(out_dtype == FB4_DTYPE_F32)};
    const dim3 grid((unsigned)((n + 16 * tiles - 1) / (16 * tiles)));
    const size_t words = direct ? 0 : (size_t)16 * tiles * (std::min<size_t>(chunks, matvec_chunks(tiles, block == 16)) * (block == 16 ? 4 : 2) + 16);
    const size_t lds = 256 + std::max(words, (size_t)waves * 16 * sets * 16 * tiles * sizeof(float));
#define FB4_MATVEC_LAUNCH(t, u, h, d) launch(matvec_kernel<t, u, h, d>, grid, dim3(64 * waves), lds, static_cast<hipStream_t>(stream), codes, meta, static_cast<const uint16_t*>(x), luts->dev_blob, bias, out, s)
#define FB4_MATVEC_CASE(t, u, d)                             \
    if (tiles == t && sets == u && direct == d) {            \
        if (block == 16) FB4_MATVEC_LAUNCH(t, u, true, d);   \
        else FB4_MATVEC_LAUNCH(t, u, false, d);              \
    }
    FB4_MATVEC_CASE(1, 1, true) FB4_MATVEC_CASE(1, 2, true) FB4_MATVEC_CASE(1, 4, true) FB4_MATVEC_CASE(1, 1, false) FB4_MATVEC_CASE(1, 2, false)
    FB4_MATVEC_CASE(1, 4, false) FB4_MATVEC_CASE(2, 1, false) FB4_MATVEC_CASE(2, 2, false) FB4_MATVEC_CASE(2, 4, false) FB4_MATVEC_CASE(4, 1, false)
    FB4_MATVEC_CASE(4, 2, false)
#undef FB4_MATVEC_CASE
#undef FB4_MATVEC_LAUNCH
    return hipGetLastError() == hipSuccess ? FB4_OK : FB4_ERR_HIP;
}

int fb4_cache_plan(const int32_t* lens, const int32_t* adds, int64_t batch, int page, int32_t* tables, int64_t max_pages, int32_t* free_pages, int64_t n_free,
                   const int32_t* free_count, int32_t* lens_out, int32_t* free_count_out, int32_t* starts, int32_t* slots, int32_t* positions, int64_t tokens,
                   void* stream)
{
    if (batch < 0 || max_pages < 0 || n_free < 0 || tokens < 0) return FB4_ERR_INVALID_ARG;
    const int bits = page_bits_of(page);
    if (bits < 0 || batch > (int64_t)kPlanMaxBatch || max_pages > kMaxInt >> bits || batch * max_pages > kMaxInt || n_free > kMaxInt || tokens > kMaxInt)
        return FB4_ERR_UNSUPPORTED;
    if (!free_count || !free_count_out || !starts || (batch > 0 && (!lens || !adds || !lens_out)) || (batch * max_pages > 0 && !tables) ||
        (n_free > 0 && !free_pages) || (tokens > 0 && !slots))
        return FB4_ERR_INVALID_ARG;
    for (const void* p : {static_cast<const void*>(lens), static_cast<const void*>(adds), static_cast<const void*>(tables), static_cast<const void*>(free_pages),
                          static_cast<const void*>(free_count), static_cast<const void*>(lens_out), static_cast<const void*>(free_count_out),
                          static_cast<const void*>(starts), static_cast<const void*>(slots), static_cast<const void*>(positions)}) {
        if (!aligned(p, 4)) return FB4_ERR_UNSUPPORTED;
    }
    // (few sequences and tokens: few wavefronts to wait for each other; 256 sequences of a token 4.8 us and 5.0, 8 of 2048 at most 20 and 8.0)
    const int64_t most = std::max(batch, std::min<int64_t>(tokens / 4, kPlanMost));
    const uint32_t threads = most <= 256 ? 256 : kPlanMost;
    const PlanShape s = {(uint32_t)batch, (uint32_t)max_pages, (uint32_t)n_free, (uint32_t)tokens, (uint32_t)bits, threads};
    hipStream_t st = static_cast<hipStream_t>(stream);
    launch(batch > (int64_t)kPlanMost ? cache_plan_kernel<4> : cache_plan_kernel<1>, dim3(1), dim3(threads), 0, st, lens, adds, free_count, tables, free_pages, lens_out,
           free_count_out, starts, slots, positions, s);
    if (tokens > (int64_t)kPlanOwnTokens)
        launch(cache_slots_kernel, dim3((unsigned)((tokens + 1023) / 1024)), dim3(256), 0, st, starts, lens_out, tables, slots, positions, s);
    return hipGetLastError() == hipSuccess ? FB4_OK : FB4_ERR_HIP;
}

int fb4_cache_store(const void* k, const int64_t* k_strides, const void* v, const int64_t* v_strides, int64_t tokens, int heads_k, int64_t dim,
                    const int32_t* slots, uint8_t* cache, uint8_t* scales, int64_t pages, int page, void* stream)
{
    if (tokens < 0 || heads_k < 1 || dim < 1 || pages < 0) return FB4_ERR_INVALID_ARG;
    const int bits = page_bits_of(page);
    if (bits < 0 || heads_k > 65535 || dim % 8 || dim > 128 || tokens > kMaxInt || pages > kMaxInt >> bits) return FB4_ERR_UNSUPPORTED;
    if (tokens == 0 || pages == 0) return FB4_OK;
    if (!k || !k_strides || !v || !v_strides || !slots || !cache || !scales) return FB4_ERR_INVALID_ARG;
    StoreStrides sk, sv;
    if (int rc = strides_of(k_strides, &sk)) return rc;
    if (int rc = strides_of(v_strides, &sv)) return rc;
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(slots, 4) || !aligned(cache, 16)) return FB4_ERR_UNSUPPORTED;
    // Tokens whose runs a workgroup takes, one run after the other: what the tokens are is on the device.  Sequences of a token each want few (1024: one
    // 70.0 us, four 62.8, sixteen 73.2; 64: one 9.2, four 14.2), prompts a page's (16 of up to 1024 tokens: one 141, four 59, 64 22.7; of up to 4096: 579, 87).
    const int64_t span = std::max<int64_t>(1, std::min<int64_t>(page, tokens / 256));
    const int64_t groups = (tokens + span - 1) / span * heads_k * 2;
    if (groups > (1 << 24) - 1) return FB4_ERR_UNSUPPORTED;
    // What other workgroups read, on memory that one writes.
    const int64_t rows_k[3] = {0, k_strides[0], k_strides[1]}, rows_v[3] = {0, v_strides[0], v_strides[1]}, none[3] = {0, 0, 0};
    const RowSet inputs[3] = {RowSet(rows_k, 1, heads_k, tokens, dim * 2), RowSet(rows_v, 1, heads_k, tokens, dim * 2), RowSet(none, 1, 1, 1, tokens * 4)};
    const void* const at[3] = {k, v, slots};
    const uint64_t held = (uint64_t)2 * pages * heads_k * page * dim, sizes = (uint64_t)2 * pages * heads_k;
    for (int i = 0; i < 3; ++i) {
        if (touches(inputs[i], at[i], cache, held) || touches(inputs[i], at[i], scales, sizes)) return FB4_ERR_INVALID_ARG;
    }
    if (touches(RowSet(none, 1, 1, 1, (int64_t)sizes), scales, cache, held)) return FB4_ERR_INVALID_ARG;
    const StoreShape s = {(uint32_t)tokens, (uint32_t)pages, (uint32_t)span, (uint16_t)heads_k, (uint8_t)bits, (uint8_t)(dim / 8)};
    launch(dim / 8 * page / 4 > kStoreThreads ? cache_store_kernel<2> : cache_store_kernel<1>, dim3((unsigned)groups), dim3(kStoreThreads), 0, static_cast<hipStream_t>(stream), static_cast<const uint16_t*>(k),
           static_cast<const uint16_t*>(v), slots, cache, scales, sk, sv, s);
    return hipGetLastError() == hipSuccess ? FB4_OK : FB4_ERR_HIP;
}

size_t fb4_cache_attention_workspace(int64_t tokens, int heads, int heads_k, int64_t dim, int page, int64_t max_pages, int64_t batch)
{
    CachePlan p;
    if (plan_attention(tokens, heads, heads_k, dim, page, max_pages, batch, &p) != FB4_OK || !p.split || tokens == 0 || batch == 0) return 0;
    return (size_t)p.positions * p.tile_rows * (size_t)(dim + 2) * sizeof(float);
}

int fb4_cache_attention(const void* q, const int64_t* q_strides, int64_t tokens, int heads, int heads_k, int64_t dim, const uint8_t* cache, const uint8_t* scales,
                        int64_t pages, int page, const int32_t* tables, int64_t max_pages, const int32_t* lens, const int32_t* starts, int64_t batch, int causal,
                        float scale, void* out, const int64_t* out_strides, float* lse, void* workspace, size_t workspace_bytes, void* stream)
{
    CachePlan p;
    if (int rc = plan_attention(tokens, heads, heads_k, dim, page, max_pages, batch, &p)) return rc;
    if (pages < 0 || (causal != 0 && causal != 1) || !(scale > 0.0f) || !std::isfinite(scale)) return FB4_ERR_INVALID_ARG;
    if (scale > 0x1p127f || pages > kMaxInt >> page_bits_of(page)) return FB4_ERR_UNSUPPORTED;
    if (tokens == 0 || batch == 0) return FB4_OK;
    if (!q || !q_strides || !lens || !starts || !out || !out_strides || (pages > 0 && max_pages > 0 && (!cache || !scales || !tables))) return FB4_ERR_INVALID_ARG;
    const size_t needed = fb4_cache_attention_workspace(tokens, heads, heads_k, dim, page, max_pages, batch);
    if (workspace_bytes < needed || (needed > 0 && !workspace)) return FB4_ERR_INVALID_ARG;
    CacheStrides sq, so;
    if (int rc = strides_of(q_strides, &sq)) return rc;
    if (int rc = strides_of(out_strides, &so)) return rc;
    if (!aligned(q, 16) || !aligned(cache, 16) || !aligned(tables, 4) || !aligned(lens, 4) || !aligned(starts, 4) || !aligned(out, 16) || !aligned(lse, 4) ||
        !aligned(workspace, 16))
        return FB4_ERR_UNSUPPORTED;
    // (no pages: no sequence has a key)
    const CacheShape s = {(uint32_t)tokens, pages ? (uint32_t)max_pages : 0u, (uint32_t)pages, (uint16_t)batch, (uint16_t)heads, (uint16_t)heads_k,
                          (uint8_t)page_bits_of(page), (uint8_t)(dim / 8 + 128 * causal), scale};
    hipStream_t st = static_cast<hipStream_t>(stream);
    float* parts = static_cast<float*>(workspace);
    const dim3 grid((unsigned)p.positions);
#define FB4_CACHE_KERNEL(kernel) launch(kernel, grid, dim3(64 * kCacheWaves), 0, st, static_cast<const uint16_t*>(q), cache, scales, tables, lens, starts, static_cast<uint16_t*>(out), lse, parts, sq, so, s)
#define FB4_CACHE_LAUNCH(d, w, split) FB4_CACHE_KERNEL((cache_attention_kernel<d, w, split>))
#define FB4_CACHE_TILES(d, w, split) FB4_CACHE_KERNEL((cache_tiles_kernel<d, w, split>))
#define FB4_CACHE_SETS(d, w, split)                             \
    if (p.tile_rows == kTileRows) FB4_CACHE_TILES(d, w, split); \
    else FB4_CACHE_LAUNCH(d, w, split)
#define FB4_CACHE_CASE(d)                               \
    case d:                                             \
        if (dim == 32 * d) {                            \
            if (p.split) { FB4_CACHE_SETS(d, true, true); } \
            else { FB4_CACHE_SETS(d, true, false); }    \
        } else {                                        \
            if (p.split) { FB4_CACHE_SETS(d, false, true); } \
            else { FB4_CACHE_SETS(d, false, false); }   \
        }                                               \
        break;
    switch ((dim + 31) / 32) {
        FB4_CACHE_CASE(1) FB4_CACHE_CASE(2) FB4_CACHE_CASE(3) FB4_CACHE_CASE(4)
    }
#undef FB4_CACHE_CASE
#undef FB4_CACHE_SETS
#undef FB4_CACHE_TILES
#undef FB4_CACHE_LAUNCH
#undef FB4_CACHE_KERNEL
    if (p.split) {
        const int64_t rows = tokens * heads;   // (below the rows of kTilesTarget tiles)
        const bool few = rows <= kJoinFew;
        launch(few ? cache_join_kernel<kJoinWaves> : cache_join_kernel<1>, dim3((unsigned)(few ? rows : (rows + 4 * kJoinRows - 1) / (4 * kJoinRows))),
               dim3(256), 0, st, parts, lens, starts, static_cast<uint16_t*>(out), lse, (uint32_t)p.positions, p.tile_rows, so, s);
    }
    return hipGetLastError() == hipSuccess ? FB4_OK : FB4_ERR_HIP;
}

}  // extern "C"
