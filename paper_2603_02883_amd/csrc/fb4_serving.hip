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
    int rows16;             // rows of a tile / 16: 8 for the kernel of many queries
    bool split;
    int64_t tiles, positions;
    int target;             // workgroups that parts make, about
};
constexpr int kCacheFew = 768, kCacheTarget = 768, kTilesTarget = 1536;

// Sizes that are served, the tiles' size, and whether the keys are shared among workgroups.
int plan_attention(int64_t tokens, int heads, int heads_k, int64_t dim, int page, int64_t max_pages, int64_t batch, CachePlan* p)
{
    if (tokens < 0 || heads < 1 || heads_k < 1 || dim < 1 || max_pages < 0 || batch < 0 || heads % heads_k) return FB4_ERR_INVALID_ARG;
    const int bits = page_bits_of(page);
    if (bits < 0 || heads > 65535 || dim % 8 || dim > 128 || tokens > kMaxInt || max_pages > kMaxInt >> bits || batch > kCacheMaxBatch) return FB4_ERR_UNSUPPORTED;
    const int64_t rows = tokens * (heads / heads_k);
    if (rows > kMaxInt) return FB4_ERR_UNSUPPORTED;
    const int64_t each = batch ? rows / batch : 0;
    p->rows16 = each > 40 || (tokens - batch) * (heads / heads_k) >= 1024 ? 8 : each > 16 ? 2 : 1;
    p->tiles = rows / (16 * p->rows16) + batch;
    p->target = p->rows16 == 8 ? kTilesTarget : kCacheTarget;
    p->split = p->tiles * heads_k < kCacheFew && (max_pages << bits) > (int64_t)kCacheLeastShare * kCacheStep;
    p->positions = p->tiles * heads_k + (p->split ? p->target : 0);
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
    if (rows > kMatvecMaxRows || cols % 32 || n >= 1 << 28 || cols >= 1 << 25) return FB4_ERR_UNSUPPORTED;
    if (rows == 0 || n == 0) return FB4_OK;
    if (!out || (cols > 0 && (!x || !codes || !meta))) return FB4_ERR_INVALID_ARG;
    if (!aligned(x, 16) || (rows > 1 && x_row_stride % 8) || x_row_stride / 8 > 0xFFFFFFFFll || !aligned(codes, 16) || !aligned(meta, block == 16 ? 4 : 2) ||
        !aligned(bias, 4) || !aligned(out, out_dtype == FB4_DTYPE_F32 ? 4 : 2))
        return FB4_ERR_UNSUPPORTED;
    if (int rc = check_device(luts)) return rc;
    const int sets = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    const int64_t chunks = cols / 32;
    // Rows of the weights to a workgroup, 16 to a tile: as many as leave every compute unit a workgroup, since each reads all of x (16 rows,
    // 16384 x 4096: 14.5 us with four tiles, 15.1 with two, 21 with one; 37 rows, 4610 x 1184: two 8.2, one 8.8; one row, 6912 x 1152: one 4.35, two 4.40)
    const int tiles = sets == 4 ? (n >= 4096 ? 2 : 1) : n >= 16384 ? 4 : n >= 8192 ? 2 : 1;
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
    // (few sequences and tokens: few wavefronts to wait for each other)
    const int64_t most = std::max(batch, std::min<int64_t>(tokens / 4, kPlanMost));
    const uint32_t threads = most <= 64 ? 64 : most <= 256 ? 256 : kPlanMost;
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
    // Runs begin at any token; a workgroup per token while there are few, one per page's tokens where whole pages come.
    const int64_t span = std::max<int64_t>(1, std::min<int64_t>(page, tokens / 256));
    const int64_t groups = (tokens + span - 1) / span * heads_k * 2;
    if (groups > (1 << 24) - 1) return FB4_ERR_UNSUPPORTED;
    const StoreShape s = {(uint32_t)tokens, (uint32_t)pages, (uint32_t)span, (uint16_t)heads_k, (uint8_t)bits, (uint8_t)(dim / 8)};
    launch(dim / 8 * page / 4 > kStoreThreads ? cache_store_kernel<2> : cache_store_kernel<1>, dim3((unsigned)groups), dim3(kStoreThreads), 0, static_cast<hipStream_t>(stream), static_cast<const uint16_t*>(k),
           static_cast<const uint16_t*>(v), slots, cache, scales, sk, sv, s);
    return hipGetLastError() == hipSuccess ? FB4_OK : FB4_ERR_HIP;
}

size_t fb4_cache_attention_workspace(int64_t tokens, int heads, int heads_k, int64_t dim, int page, int64_t max_pages, int64_t batch)
{
    CachePlan p;
    if (plan_attention(tokens, heads, heads_k, dim, page, max_pages, batch, &p) != FB4_OK || !p.split || tokens == 0 || batch == 0) return 0;
    return (size_t)p.positions * (size_t)(16 * p.rows16) * (size_t)(dim + 2) * sizeof(float);
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
                          (uint16_t)p.target, (uint8_t)page_bits_of(page), (uint8_t)(dim / 8), (uint8_t)causal, (uint8_t)p.rows16, scale};
    hipStream_t st = static_cast<hipStream_t>(stream);
    float* parts = static_cast<float*>(workspace);
    float* states = p.split ? parts + (size_t)p.positions * (16 * p.rows16) * dim : nullptr;
    const dim3 grid((unsigned)p.positions);
#define FB4_CACHE_KERNEL(kernel, split) launch(kernel, grid, dim3(64 * kCacheWaves), 0, st, static_cast<const uint16_t*>(q), cache, scales, tables, lens, starts, static_cast<uint16_t*>(split ? workspace : out), split ? states : lse, sq, so, s)
#define FB4_CACHE_LAUNCH(d, u, w, split) FB4_CACHE_KERNEL((cache_attention_kernel<d, u, w, split>), split)
#define FB4_CACHE_TILES(d, w, split) FB4_CACHE_KERNEL((cache_tiles_kernel<d, w, split>), split)
#define FB4_CACHE_SETS(d, w, split)                     \
    if (p.rows16 == 8) FB4_CACHE_TILES(d, w, split);     \
    else if (p.rows16 == 2) FB4_CACHE_LAUNCH(d, 2, w, split); \
    else FB4_CACHE_LAUNCH(d, 1, w, split)
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
        const int64_t rows = tokens * heads;   // (below the target's tiles of 64 rows and the batch's)
        const bool few = rows <= 4096;
        launch(few ? cache_join_kernel<4> : cache_join_kernel<1>, dim3((unsigned)(few ? rows : (rows + 4 * kJoinRows - 1) / (4 * kJoinRows))), dim3(256), 0, st, parts,
               reinterpret_cast<const float2*>(states), lens, starts, static_cast<uint16_t*>(out), lse, (uint32_t)p.positions, so, s);
    }
    return hipGetLastError() == hipSuccess ? FB4_OK : FB4_ERR_HIP;
}

}  // extern "C"
