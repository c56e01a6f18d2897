// cpes_eval_api.hip -- host runtime of the operators that evaluate a member
// (include/cpes.h): argument validation and dispatch.  As in cpes_api.hip, every
// check runs before anything is enqueued, and no HIP call is made before
// validation passes.
#include "cpes.h"

#include <algorithm>
#include <cfloat>
#include <cmath>

#include "cpes_eval.hpp"
#include "cpes_host.hpp"

namespace {

using cpes::aligned16;
using cpes::fail;
using cpes::hip_status;

// No buffer has more; what is below adds up to byte offsets of 64 bits.
constexpr double kMaxElements = 1152921504606846976.0 / 16;     // 2^60 / 16

int check_cache(const cpes_cache* c, const char* fn)
{
    if (!c) return fail(CPES_ERR_INVALID_ARGUMENT, "%s: cache is null", fn);
    if (!c->k_dev || !c->v_dev) return fail(CPES_ERR_INVALID_ARGUMENT, "%s: cache keys or values are null", fn);
    if (c->dtype != CPES_BF16 && c->dtype != CPES_F32)
        return fail(CPES_ERR_INVALID_ARGUMENT, "%s: unknown cache dtype %d", fn, c->dtype);
    if (c->layers < 1 || c->pages < 1 || c->heads < 1 || c->page_size < 1)
        return fail(CPES_ERR_INVALID_ARGUMENT, "%s: cache of %d layers, %d pages, %d heads, %d tokens a page", fn,
                    c->layers, c->pages, c->heads, c->page_size);
    if (c->head_dim < 8 || c->head_dim > CPES_MAX_HEAD_DIM || c->head_dim % 8 != 0)
        return fail(CPES_ERR_INVALID_ARGUMENT, "%s: head_dim %d is not a multiple of 8 in [8, %d]", fn, c->head_dim,
                    CPES_MAX_HEAD_DIM);
    const struct {
        int64_t stride;
        int32_t count;
    } dims[] = {{c->layer_stride, c->layers}, {c->page_stride, c->pages}, {c->head_stride, c->heads}, {c->token_stride, c->page_size}};
    for (const auto& d : dims)
        if (d.stride < 0 || (double)d.stride * d.count > kMaxElements)
            return fail(CPES_ERR_INVALID_ARGUMENT, "%s: cache stride %lld negative or beyond any memory", fn, (long long)d.stride);
    if (c->heads > CPES_MAX_HEADS) return fail(CPES_ERR_UNSUPPORTED, "%s: %d heads above CPES_MAX_HEADS", fn, c->heads);
    return CPES_OK;
}

int check_pool(const cpes_pool* p, bool refs, const char* fn)
{
    if (!p) return fail(CPES_ERR_INVALID_ARGUMENT, "%s: pool is null", fn);
    if (!p->table_dev || !p->lengths_dev) return fail(CPES_ERR_INVALID_ARGUMENT, "%s: page table or lengths are null", fn);
    if (p->sequences < 1 || p->width < 1 || p->page_size < 1 || p->table_stride < p->width)
        return fail(CPES_ERR_INVALID_ARGUMENT, "%s: pool of %d sequences, %d pages each (stride %lld), %d tokens a page", fn,
                    p->sequences, p->width, (long long)p->table_stride, p->page_size);
    if (refs && (!p->refs_dev || p->pages < 1))
        return fail(CPES_ERR_INVALID_ARGUMENT, "%s: the pool's reference counts are missing", fn);
    return CPES_OK;
}

int check_fit(const cpes_cache* c, const cpes_pool* p, const char* fn)
{
    if (c->page_size != p->page_size)
        return fail(CPES_ERR_INVALID_ARGUMENT, "%s: pages of %d tokens in the cache, %d in the pool", fn, c->page_size,
                    p->page_size);
    if (p->refs_dev && c->pages != p->pages)
        return fail(CPES_ERR_INVALID_ARGUMENT, "%s: %d pages in the cache, %d in the pool", fn, c->pages, p->pages);
    return CPES_OK;
}

int check_list(int32_t n, bool present, const char* fn)
{
    if (n < 0) return fail(CPES_ERR_INVALID_ARGUMENT, "%s: n %d is negative", fn, n);
    if (n > 0 && !present) return fail(CPES_ERR_INVALID_ARGUMENT, "%s: a list is null", fn);
    if (n > CPES_MAX_SEQUENCES) return fail(CPES_ERR_UNSUPPORTED, "%s: n %d above CPES_MAX_SEQUENCES", fn, n);
    return CPES_OK;
}

int check_workspace(const void* ws, size_t given, size_t needed, const char* fn)
{
    if (needed == 0) return CPES_OK;
    if (!ws || given < needed)
        return fail(CPES_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, needed, ws ? given : (size_t)0);
    if (!aligned16(ws)) return fail(CPES_ERR_WORKSPACE, "%s: workspace must be 16-byte aligned", fn);
    return CPES_OK;
}

int check_layer(const cpes_cache* c, int32_t layer, const char* fn)
{
    if (layer < 0 || layer >= c->layers)
        return fail(CPES_ERR_INVALID_ARGUMENT, "%s: layer %d outside [0, %d)", fn, layer, c->layers);
    return CPES_OK;
}

int check_longest(int32_t longest, const char* fn)
{
    if (longest < 1) return fail(CPES_ERR_INVALID_ARGUMENT, "%s: longest %d is not positive", fn, longest);
    if (longest > CPES_MAX_TREE)
        return fail(CPES_ERR_UNSUPPORTED, "%s: longest %d above CPES_MAX_TREE", fn, longest);
    return CPES_OK;
}

cpes::PoolArgs pool_args(const cpes_pool* p)
{
    cpes::PoolArgs a;
    a.table = p->table_dev;
    a.lengths = p->lengths_dev;
    a.refs = p->refs_dev;
    a.table_stride = p->table_stride;
    a.sequences = p->sequences;
    a.width = p->width;
    a.pages = p->pages;
    a.page_size = p->page_size;
    return a;
}

int64_t elem_size(int dtype)
{
    return dtype == CPES_BF16 ? 2 : 4;
}

char* at_layer(const cpes_cache* c, void* base, int32_t layer)
{
    return static_cast<char*>(base) + layer * c->layer_stride * elem_size(c->dtype);
}

// A page as runs of consecutive elements: heads and tokens joined where they
// follow each other in memory.
int page_args(const cpes_cache* c, cpes::PageArgs* a, const char* fn)
{
    const int64_t e = elem_size(c->dtype), H = c->heads, P = c->page_size, D = c->head_dim;
    if (2.0 * c->layers * H * P * D * e / 16 >= 2147483648.0)
        return fail(CPES_ERR_UNSUPPORTED, "%s: a page of more than 32 GB", fn);
    int64_t run = D, outers = H, outer = c->head_stride, inners = P, inner = c->token_stride;
    if (P == 1 || inner == D) {
        run = P * D;
        inners = 1;
        if (H == 1 || outer == run) {
            run *= H;
            outers = 1;
        }
    } else if (H == 1 || outer == D) {
        run = H * D;
        outers = P;
        outer = inner;
        inners = 1;
        if (outer == run) {
            run *= P;
            outers = 1;
        }
    }
    const int64_t units = 2 * c->layers * outers * inners * (run * e / 16);
    a->k = static_cast<char*>(c->k_dev);
    a->v = static_cast<char*>(c->v_dev);
    a->page_bytes = c->page_stride * e;
    a->layer_bytes = c->layer_stride * e;
    a->outer_bytes = outer * e;
    a->inner_bytes = inner * e;
    a->outers = cpes::Divisor((uint32_t)outers);
    a->inners = cpes::Divisor((uint32_t)inners);
    a->run = cpes::Divisor((uint32_t)(run * e / 16));
    a->units = (uint32_t)units;
    return CPES_OK;
}

constexpr size_t round16(size_t x)
{
    return (x + 15) / 16 * 16;
}

// Workgroups of an attention launch on the 256 CUs of an MI355X: two per CU of four
// waves, one where a head's tiles fill the registers of a whole SIMD.
int attend_groups(int32_t head_dim)
{
    return head_dim > 128 ? 256 : 512;
}

int32_t head_blocks(int32_t group)
{
    return (group + cpes::kAttendHeads - 1) / cpes::kAttendHeads;
}

// log2 of a page's tokens, -1 if that is no whole number.
int32_t page_shift(int32_t page_size)
{
    for (int b = 0; b < 31; ++b)
        if (page_size == (int32_t)1 << b) return b;
    return -1;
}

bool check_heads(int32_t q_heads, int32_t kv_heads, int32_t head_dim)
{
    return kv_heads >= 1 && q_heads >= 1 && q_heads <= CPES_MAX_HEADS && q_heads % kv_heads == 0 && head_dim >= 8 &&
           head_dim <= CPES_MAX_HEAD_DIM && head_dim % 8 == 0;
}

// What attention over one layer of the cache needs, whatever its rows are.
int check_attend(const cpes_cache* cache, int32_t layer, const cpes_pool* pool, int32_t q_heads, float scale, int32_t window,
                 int32_t sinks, int64_t q_stride, int64_t q_head_stride, int64_t out_stride, int64_t out_head_stride,
                 const char* fn)
{
    int rc = check_cache(cache, fn);
    if (!rc) rc = check_pool(pool, false, fn);
    if (!rc) rc = check_fit(cache, pool, fn);
    if (!rc) rc = check_layer(cache, layer, fn);
    if (!rc && (q_heads < 1 || q_heads % cache->heads != 0))
        rc = fail(CPES_ERR_INVALID_ARGUMENT, "%s: %d query heads for %d key-value heads", fn, q_heads, cache->heads);
    if (!rc && q_heads > CPES_MAX_HEADS) rc = fail(CPES_ERR_UNSUPPORTED, "%s: %d query heads above CPES_MAX_HEADS", fn, q_heads);
    if (!rc && !std::isfinite(scale)) rc = fail(CPES_ERR_INVALID_ARGUMENT, "%s: scale %g is not finite", fn, (double)scale);
    if (!rc && (window < 0 || sinks < 0))
        rc = fail(CPES_ERR_INVALID_ARGUMENT, "%s: window %d or sinks %d negative", fn, window, sinks);
    if (!rc && (q_stride < 0 || q_head_stride < 0 || out_stride < 0 || out_head_stride < 0))
        rc = fail(CPES_ERR_INVALID_ARGUMENT, "%s: negative stride", fn);
    return rc;
}

// Workgroups of the shares of trees: two per CU, one of eight waves or where a wave's state fills its SIMD's registers.
int tree_groups(const cpes::TreeShape& t, int32_t head_dim)
{
    return t.beside <= 4 && (t.wide || (head_dim <= 128 && t.sets == 1)) ? 512 : 256;
}

size_t tree_parts_bytes(const cpes::TreeShape& t, int32_t head_dim)
{
    const size_t waves = std::max<size_t>(cpes::kAttendWaves, t.beside);
    return 2 * (size_t)tree_groups(t, head_dim) * waves * cpes::tree_part_floats(t.sets, head_dim) * sizeof(float);
}

// Two partial results a wave, then the shares of every job.
size_t tree_bytes(int32_t rows, const cpes::TreeShape& t, int32_t kv_heads, int32_t head_dim)
{
    return round16(tree_parts_bytes(t, head_dim) + (size_t)rows * t.pieces * kv_heads * t.blocks * sizeof(int2));
}

// Two partial results a share, then the shares of every row and head block.
size_t attend_parts_bytes(int32_t head_dim)
{
    return 2 * (size_t)attend_groups(head_dim) * cpes::kAttendWaves * cpes::attend_part_floats(head_dim) * sizeof(float);
}

size_t attend_bytes(int32_t rows, int32_t q_heads, int32_t kv_heads, int32_t head_dim)
{
    return round16(attend_parts_bytes(head_dim) + (size_t)rows * kv_heads * head_blocks(q_heads / kv_heads) * sizeof(int2));
}

size_t sample_bytes(int32_t rows, int32_t vocab, int dtype)
{
    rows = std::min(rows, cpes::kSampleAtOnce);
    const cpes::SampleSplit x = cpes::sample_split(rows, vocab, dtype);
    if (x.slices == 0) return 0;
    return rows * round16((size_t)x.strips() * (x.note_slots * 2 * cpes::kSampleLanes * sizeof(uint16_t) +
                                                x.slots * (sizeof(double) + sizeof(float)) + sizeof(float)));
}

size_t logprob_bytes(int32_t rows, int32_t slices, int32_t top)
{
    return slices > 1 ? (size_t)rows * slices * (sizeof(float4) + (size_t)top * sizeof(unsigned long long)) : 0;
}

int check_logits(const void* x, int dtype, int32_t rows, int32_t vocab, int64_t stride, float scale, const char* fn)
{
    if (dtype != CPES_BF16 && dtype != CPES_F32) return fail(CPES_ERR_INVALID_ARGUMENT, "%s: unknown dtype %d", fn, dtype);
    if (rows < 0 || vocab < 1) return fail(CPES_ERR_INVALID_ARGUMENT, "%s: %d rows of %d logits", fn, rows, vocab);
    if (!x && rows > 0) return fail(CPES_ERR_INVALID_ARGUMENT, "%s: logits are null", fn);
    if (rows > 1 && stride < vocab)
        return fail(CPES_ERR_INVALID_ARGUMENT, "%s: row stride %lld below the %d logits of a row", fn, (long long)stride, vocab);
    if (!(scale > 0.f) || !(scale <= FLT_MAX / 2))
        return fail(CPES_ERR_INVALID_ARGUMENT, "%s: scale %g is not positive or above FLT_MAX / 2", fn, (double)scale);
    return CPES_OK;
}

}  // namespace

extern "C" {

size_t cpes_pages_workspace_bytes(int32_t pages)
{
    if (pages < 1) return 0;
    return round16((cpes::kPagesHeader + 2 * (size_t)pages) * sizeof(int32_t));
}

int cpes_pages_reserve(const cpes_pool* pool, int32_t n, const int32_t* seqs_dev, const int32_t* new_lengths_dev,
                       void* workspace_dev, size_t workspace_bytes, int32_t* status_dev, void* stream)
{
    cpes::clear_error();
    const char* fn = "cpes_pages_reserve";
    int rc = check_pool(pool, true, fn);
    if (!rc) rc = check_list(n, seqs_dev && new_lengths_dev, fn);
    if (!rc && n > pool->sequences)
        rc = fail(CPES_ERR_INVALID_ARGUMENT, "%s: %d of %d sequences listed", fn, n, pool->sequences);
    if (!rc) rc = check_workspace(workspace_dev, workspace_bytes, cpes_pages_workspace_bytes(pool->pages), fn);
    if (rc) return rc;
    return hip_status(cpes::launch_pages_reserve(pool_args(pool), n, seqs_dev, new_lengths_dev,
                                                 static_cast<int32_t*>(workspace_dev), status_dev, (hipStream_t)stream),
                      fn);
}

int cpes_pages_fork(const cpes_cache* cache, const cpes_pool* pool, int32_t n, const int32_t* parents_dev,
                    const int32_t* children_dev, void* workspace_dev, size_t workspace_bytes, int32_t* status_dev,
                    void* stream)
{
    cpes::clear_error();
    const char* fn = "cpes_pages_fork";
    cpes::PageArgs page;
    int rc = check_cache(cache, fn);
    if (!rc) rc = check_pool(pool, true, fn);
    if (!rc) rc = check_fit(cache, pool, fn);
    if (!rc) rc = check_list(n, parents_dev && children_dev, fn);
    if (!rc && n > pool->sequences)
        rc = fail(CPES_ERR_INVALID_ARGUMENT, "%s: %d of %d sequences listed", fn, n, pool->sequences);
    if (!rc) rc = check_workspace(workspace_dev, workspace_bytes, cpes_pages_workspace_bytes(pool->pages), fn);
    if (!rc) rc = page_args(cache, &page, fn);
    if (rc) return rc;
    return hip_status(cpes::launch_pages_fork(page, pool_args(pool), n, parents_dev, children_dev,
                                              static_cast<int32_t*>(workspace_dev), status_dev, (hipStream_t)stream),
                      fn);
}

int cpes_pages_free(const cpes_pool* pool, int32_t n, const int32_t* seqs_dev, int32_t* status_dev, void* stream)
{
    cpes::clear_error();
    const char* fn = "cpes_pages_free";
    int rc = check_pool(pool, true, fn);
    if (!rc) rc = check_list(n, seqs_dev, fn);
    if (rc) return rc;
    return hip_status(cpes::launch_pages_free(pool_args(pool), n, seqs_dev, status_dev, (hipStream_t)stream), fn);
}

int cpes_pages_copy(const cpes_cache* cache, int32_t n, const int32_t* src_dev, const int32_t* dst_dev, void* stream)
{
    cpes::clear_error();
    const char* fn = "cpes_pages_copy";
    cpes::PageArgs page;
    int rc = check_cache(cache, fn);
    if (!rc && n < 0) rc = fail(CPES_ERR_INVALID_ARGUMENT, "%s: n %d is negative", fn, n);
    if (!rc && n > 0 && (!src_dev || !dst_dev)) rc = fail(CPES_ERR_INVALID_ARGUMENT, "%s: a list is null", fn);
    if (!rc) rc = page_args(cache, &page, fn);
    if (rc || n == 0) return rc;
    return hip_status(cpes::launch_pages_copy(page, cache->pages, n, src_dev, dst_dev, (hipStream_t)stream), fn);
}

int cpes_pages_compact(const cpes_cache* cache, const cpes_pool* pool, const cpes_pool* packed, void* workspace_dev,
                       size_t workspace_bytes, int32_t* moved_dev, void* stream)
{
    cpes::clear_error();
    const char* fn = "cpes_pages_compact";
    cpes::PageArgs page;
    int rc = check_cache(cache, fn);
    if (!rc) rc = check_pool(pool, true, fn);
    if (!rc) rc = check_pool(packed, true, fn);
    if (!rc) rc = check_fit(cache, pool, fn);
    if (!rc && (packed->sequences != pool->sequences || packed->width != pool->width || packed->pages != pool->pages ||
                packed->page_size != pool->page_size))
        rc = fail(CPES_ERR_INVALID_ARGUMENT, "%s: the packed pool has another shape", fn);
    if (!rc && packed->table_dev == pool->table_dev && packed->table_stride != pool->table_stride)
        rc = fail(CPES_ERR_INVALID_ARGUMENT, "%s: one table with two strides", fn);
    if (!rc) rc = check_workspace(workspace_dev, workspace_bytes, cpes_pages_workspace_bytes(pool->pages), fn);
    if (!rc) rc = page_args(cache, &page, fn);
    if (rc) return rc;
    return hip_status(cpes::launch_pages_compact(page, pool_args(pool), pool_args(packed),
                                                 static_cast<int32_t*>(workspace_dev), moved_dev, (hipStream_t)stream),
                      fn);
}

int cpes_cache_append(const cpes_cache* cache, int32_t layer, const cpes_pool* pool, int32_t n, const int32_t* seqs_dev,
                      const int32_t* positions_dev, const void* k_new_dev, const void* v_new_dev, int64_t new_stride,
                      int64_t new_head_stride, void* stream)
{
    cpes::clear_error();
    const char* fn = "cpes_cache_append";
    int rc = check_cache(cache, fn);
    if (!rc) rc = check_pool(pool, false, fn);
    if (!rc) rc = check_fit(cache, pool, fn);
    if (!rc) rc = check_layer(cache, layer, fn);
    if (!rc && n < 0) rc = fail(CPES_ERR_INVALID_ARGUMENT, "%s: n %d is negative", fn, n);
    if (!rc && n > 0 && (!positions_dev || !k_new_dev || !v_new_dev))
        rc = fail(CPES_ERR_INVALID_ARGUMENT, "%s: positions, keys or values are null", fn);
    if (!rc && (new_stride < 0 || new_head_stride < 0)) rc = fail(CPES_ERR_INVALID_ARGUMENT, "%s: negative stride", fn);
    if (rc || n == 0) return rc;
    const int64_t e = elem_size(cache->dtype);
    cpes::AppendArgs a;
    a.pool = pool_args(pool);
    a.pool.pages = cache->pages;
    a.k = at_layer(cache, cache->k_dev, layer);
    a.v = at_layer(cache, cache->v_dev, layer);
    a.k_new = static_cast<const char*>(k_new_dev);
    a.v_new = static_cast<const char*>(v_new_dev);
    a.seqs = seqs_dev;
    a.positions = positions_dev;
    a.page_bytes = cache->page_stride * e;
    a.head_bytes = cache->head_stride * e;
    a.token_bytes = cache->token_stride * e;
    a.new_bytes = new_stride * e;
    a.new_head_bytes = new_head_stride * e;
    a.n = n;
    a.heads = cache->heads;
    const int64_t run = cache->head_dim * e / 16, token = run * cache->heads;      // below 2^22
    a.run = cpes::Divisor((uint32_t)run);
    a.token = cpes::Divisor((uint32_t)token);
    return hip_status(cpes::launch_append(a, (hipStream_t)stream), fn);
}

size_t cpes_attend_workspace_bytes(int32_t rows, int32_t q_heads, int32_t kv_heads, int32_t head_dim)
{
    if (rows < 0 || rows > CPES_MAX_SEQUENCES || !check_heads(q_heads, kv_heads, head_dim)) return 0;
    return attend_bytes(rows, q_heads, kv_heads, head_dim);
}

int cpes_attend(const cpes_cache* cache, int32_t layer, const cpes_pool* pool, int32_t rows, const int32_t* seqs_dev,
                const void* q_dev, int64_t q_stride, int64_t q_head_stride, int32_t q_heads, float scale, int32_t window,
                int32_t sinks, void* out_dev, int64_t out_stride, int64_t out_head_stride, float* lse_dev,
                void* workspace_dev, size_t workspace_bytes, void* stream)
{
    cpes::clear_error();
    const char* fn = "cpes_attend";
    int rc = check_attend(cache, layer, pool, q_heads, scale, window, sinks, q_stride, q_head_stride, out_stride,
                          out_head_stride, fn);
    if (!rc) rc = check_list(rows, q_dev && out_dev, fn);
    if (!rc) rc = check_workspace(workspace_dev, workspace_bytes, attend_bytes(rows, q_heads, cache->heads, cache->head_dim), fn);
    if (rc || rows == 0) return rc;
    cpes::AttendArgs a;
    a.k = at_layer(cache, cache->k_dev, layer);
    a.v = at_layer(cache, cache->v_dev, layer);
    a.q = q_dev;
    a.out = out_dev;
    a.lse = lse_dev;
    a.seqs = seqs_dev;
    a.table = pool->table_dev;
    a.lengths = pool->lengths_dev;
    a.groups = attend_groups(cache->head_dim);
    a.parts = static_cast<float*>(workspace_dev);
    a.joins = reinterpret_cast<int2*>(static_cast<char*>(workspace_dev) + attend_parts_bytes(cache->head_dim));
    a.page_stride = cache->page_stride;
    a.head_stride = cache->head_stride;
    a.token_stride = cache->token_stride;
    a.table_stride = pool->table_stride;
    a.q_stride = q_stride;
    a.q_head_stride = q_head_stride;
    a.out_stride = out_stride;
    a.out_head_stride = out_head_stride;
    a.rows = rows;
    a.heads = cache->heads;
    a.group = q_heads / cache->heads;
    a.blocks = head_blocks(a.group);
    a.dim = cache->head_dim;
    a.page_size = cache->page_size;
    a.page_shift = page_shift(cache->page_size);
    a.pages = cache->pages;
    a.width = pool->width;
    a.sequences = pool->sequences;
    a.window = window;
    a.sinks = sinks;
    a.scale = scale;
    return hip_status(cpes::launch_attend(cache->dtype, a, (hipStream_t)stream), fn);
}

size_t cpes_logprobs_workspace_bytes(int32_t rows, int32_t vocab, int32_t top)
{
    if (rows < 0 || vocab < 1 || top < 0 || top > CPES_MAX_ALTERNATIVES) return 0;
    // the most that any number of rows up to this takes: fewer rows are cut into more slices
    size_t most = 0;
    for (int32_t r = 1; r <= std::min<int32_t>(rows, cpes::kMaxSlicedRows); ++r)
        for (int dtype : {CPES_BF16, CPES_F32}) {
            int32_t per;
            most = std::max(most, logprob_bytes(r, cpes::logprob_slices(r, vocab, dtype, &per), top));
        }
    return most;
}

int cpes_logprobs(const void* x_dev, int dtype, int32_t rows, int32_t vocab, int64_t stride, float scale,
                  const int64_t* targets_dev, float* logp_dev, float* entropy_dev, float* lse_dev, float* stats_dev,
                  int32_t top, float* top_logp_dev, int64_t* top_ids_dev, void* workspace_dev, size_t workspace_bytes,
                  void* stream)
{
    cpes::clear_error();
    const char* fn = "cpes_logprobs";
    int rc = check_logits(x_dev, dtype, rows, vocab, stride, scale, fn);
    if (!rc && logp_dev && !targets_dev && rows > 0)
        rc = fail(CPES_ERR_INVALID_ARGUMENT, "%s: log probabilities without targets", fn);
    if (!rc && (top < 0 || top > CPES_MAX_ALTERNATIVES))
        rc = fail(CPES_ERR_INVALID_ARGUMENT, "%s: top %d outside [0, %d]", fn, top, CPES_MAX_ALTERNATIVES);
    if (!rc && top > 0 && rows > 0 && (!top_logp_dev || !top_ids_dev))
        rc = fail(CPES_ERR_INVALID_ARGUMENT, "%s: alternatives without both outputs", fn);
    if (rc) return rc;
    cpes::LogprobArgs a;
    a.slices = cpes::logprob_slices(rows, vocab, dtype, &a.per_slice);
    rc = check_workspace(workspace_dev, workspace_bytes, logprob_bytes(rows, a.slices, top), fn);
    if (rc || rows == 0) return rc;
    a.x = x_dev;
    a.targets = targets_dev;
    a.logp = logp_dev;
    a.entropy = entropy_dev;
    a.lse = lse_dev;
    a.stats = stats_dev;
    a.top_logp = top_logp_dev;
    a.top_ids = top_ids_dev;
    a.parts = static_cast<float4*>(workspace_dev);
    a.keys = a.slices > 1 ? reinterpret_cast<unsigned long long*>(a.parts + (int64_t)rows * a.slices) : nullptr;
    a.stride = stride;
    a.rows = rows;
    a.vocab = vocab;
    a.top = top;
    a.scale = scale;
    const double c = (double)scale * M_LOG2E;
    a.c = (float)c;
    a.excess = (float)(((double)a.c / c - 1.0) * M_LN2);
    return hip_status(cpes::launch_logprobs(dtype, a, (hipStream_t)stream), fn);
}

int cpes_logprobs_backward(const void* x_dev, int dtype, int32_t rows, int32_t vocab, int64_t stride, float scale,
                           const int64_t* targets_dev, const float* stats_dev, const float* entropy_dev,
                           const float* d_logp_dev, const float* d_entropy_dev, void* dx_dev, int64_t dx_stride,
                           void* stream)
{
    cpes::clear_error();
    const char* fn = "cpes_logprobs_backward";
    int rc = check_logits(x_dev, dtype, rows, vocab, stride, scale, fn);
    if (!rc && rows > 0 && (!stats_dev || !dx_dev)) rc = fail(CPES_ERR_INVALID_ARGUMENT, "%s: stats or dx are null", fn);
    if (!rc && rows > 0 && ((d_logp_dev && !targets_dev) || (d_entropy_dev && !entropy_dev)))
        rc = fail(CPES_ERR_INVALID_ARGUMENT, "%s: d_logp needs targets, d_entropy the entropies", fn);
    if (!rc && rows > 1 && dx_stride < vocab)
        rc = fail(CPES_ERR_INVALID_ARGUMENT, "%s: row stride %lld below the %d gradients of a row", fn, (long long)dx_stride,
                  vocab);
    if (!rc && dx_dev == x_dev && rows > 1 && dx_stride != stride)
        rc = fail(CPES_ERR_INVALID_ARGUMENT, "%s: in place with two strides", fn);
    if (rc || rows == 0) return rc;
    cpes::LogprobGradArgs a;
    a.x = x_dev;
    a.dx = dx_dev;
    a.targets = targets_dev;
    a.stats = stats_dev;
    a.entropy = entropy_dev;
    a.d_logp = d_logp_dev;
    a.d_entropy = d_entropy_dev;
    a.stride = stride;
    a.dx_stride = dx_stride;
    a.rows = rows;
    a.vocab = vocab;
    a.scale = scale;
    return hip_status(cpes::launch_logprobs_backward(dtype, a, (hipStream_t)stream), fn);
}

size_t cpes_pages_keep_workspace_bytes(int32_t n, int32_t longest)
{
    if (n < 0 || longest < 1 || longest > CPES_MAX_TREE) return 0;
    return round16((size_t)cpes::keep_words(n, longest + 1) * sizeof(int32_t));
}

int cpes_pages_keep(const cpes_cache* cache, const cpes_pool* pool, int32_t n, const int32_t* seqs_dev,
                    const int32_t* starts_dev, int32_t longest, const int32_t* kept_dev, const int32_t* path_dev,
                    void* workspace_dev, size_t workspace_bytes, int32_t* status_dev, void* stream)
{
    cpes::clear_error();
    const char* fn = "cpes_pages_keep";
    cpes::PageArgs page;                  // checked for its size
    int rc = check_cache(cache, fn);
    if (!rc) rc = check_pool(pool, true, fn);
    if (!rc) rc = check_fit(cache, pool, fn);
    if (!rc) rc = check_list(n, starts_dev && kept_dev && path_dev, fn);
    if (!rc && n > pool->sequences)
        rc = fail(CPES_ERR_INVALID_ARGUMENT, "%s: %d of %d sequences listed", fn, n, pool->sequences);
    if (!rc) rc = check_longest(longest, fn);
    if (!rc) rc = check_workspace(workspace_dev, workspace_bytes, cpes_pages_keep_workspace_bytes(n, longest), fn);
    if (!rc) rc = page_args(cache, &page, fn);
    if (rc) return rc;
    const int64_t e = elem_size(cache->dtype), run = cache->head_dim * e / 16;
    cpes::KeepArgs a;
    a.pool = pool_args(pool);
    a.k = page.k;
    a.v = page.v;
    a.seqs = seqs_dev;
    a.starts = starts_dev;
    a.kept = kept_dev;
    a.path = path_dev;
    a.ws = static_cast<int32_t*>(workspace_dev);
    a.page_bytes = page.page_bytes;
    a.layer_bytes = page.layer_bytes;
    a.head_bytes = cache->head_stride * e;
    a.token_bytes = cache->token_stride * e;
    a.n = n;
    a.longest = longest;
    // `longest` tokens that begin at the end of a page, and end at the beginning of one
    a.span = (int32_t)std::min<int64_t>(longest + 1, ((int64_t)longest - 1 + pool->page_size - 1) / pool->page_size + 1);
    a.run = cpes::Divisor((uint32_t)run);
    a.heads = cpes::Divisor((uint32_t)cache->heads);
    a.units = (uint32_t)(2 * (int64_t)cache->layers * cache->heads * run);      // below a page's
    return hip_status(cpes::launch_pages_keep(a, status_dev, (hipStream_t)stream), fn);
}

size_t cpes_attend_tree_workspace_bytes(int32_t rows, int32_t tokens, int32_t longest, int32_t q_heads, int32_t kv_heads,
                                        int32_t head_dim)
{
    if (rows < 0 || rows > CPES_MAX_SEQUENCES || tokens < 0 || (tokens > 0 && (longest < 1 || longest > tokens)) ||
        !check_heads(q_heads, kv_heads, head_dim))
        return 0;
    size_t most = 0;             // either type's, through shared memory or not
    for (int way = 0; way < 3; ++way)
        most = std::max(most, tree_bytes(rows, cpes::tree_shape(way > 0, way > 1, std::max(1, longest), q_heads / kv_heads, head_dim), kv_heads, head_dim));
    return most;
}

int cpes_attend_tree(const cpes_cache* cache, int32_t layer, const cpes_pool* pool, int32_t rows, const int32_t* seqs_dev,
                     const int32_t* starts_dev, int32_t tokens, int32_t longest, const int32_t* parents_dev,
                     const void* q_dev, int64_t q_stride, int64_t q_head_stride, int32_t q_heads, float scale,
                     int32_t window, int32_t sinks, void* out_dev, int64_t out_stride, int64_t out_head_stride,
                     float* lse_dev, void* workspace_dev, size_t workspace_bytes, void* stream)
{
    cpes::clear_error();
    const char* fn = "cpes_attend_tree";
    int rc = check_attend(cache, layer, pool, q_heads, scale, window, sinks, q_stride, q_head_stride, out_stride,
                          out_head_stride, fn);
    if (!rc) rc = check_list(rows, starts_dev, fn);
    if (!rc && tokens < 0) rc = fail(CPES_ERR_INVALID_ARGUMENT, "%s: %d tokens", fn, tokens);
    if (!rc && tokens > 0 && (!q_dev || !out_dev)) rc = fail(CPES_ERR_INVALID_ARGUMENT, "%s: q or out are null", fn);
    if (!rc && tokens > 0 && (longest < 1 || longest > tokens))
        rc = fail(CPES_ERR_INVALID_ARGUMENT, "%s: longest %d outside [1, %d]", fn, longest, tokens);
    if (!rc && tokens > 0 && parents_dev && longest > CPES_MAX_TREE)
        rc = fail(CPES_ERR_UNSUPPORTED, "%s: longest %d above CPES_MAX_TREE", fn, longest);
    if (rc) return rc;
    const char* const k = at_layer(cache, cache->k_dev, layer);
    const char* const v = at_layer(cache, cache->v_dev, layer);
    // straight into shared memory go 16 bytes that lie at a multiple of 16
    const bool aligned = ((uintptr_t)k | (uintptr_t)v | (uintptr_t)((cache->page_stride | cache->head_stride | cache->token_stride) * 2)) % 16 == 0;
    // that form takes scores times scale log2 e, which has to be a number with all its bits; the other takes them times scale first
    const bool ordinary = std::fabs(scale) >= 1e-30f && std::fabs(scale) <= 1e30f;
    const cpes::TreeShape shape = cpes::tree_shape(cache->dtype == CPES_BF16, aligned && ordinary, std::max(1, longest),
                                                   q_heads / cache->heads, cache->head_dim);
    rc = check_workspace(workspace_dev, workspace_bytes, tree_bytes(rows, shape, cache->heads, cache->head_dim), fn);
    if (rc || rows == 0 || tokens == 0) return rc;
    cpes::TreeArgs a;
    a.k = k;
    a.v = v;
    a.q = q_dev;
    a.out = out_dev;
    a.lse = lse_dev;
    a.seqs = seqs_dev;
    a.starts = starts_dev;
    a.parents = parents_dev;
    a.table = pool->table_dev;
    a.lengths = pool->lengths_dev;
    a.groups = tree_groups(shape, cache->head_dim);
    a.parts = static_cast<float*>(workspace_dev);
    a.joins = reinterpret_cast<int2*>(static_cast<char*>(workspace_dev) + tree_parts_bytes(shape, cache->head_dim));
    a.page_stride = cache->page_stride;
    a.head_stride = cache->head_stride;
    a.token_stride = cache->token_stride;
    a.table_stride = pool->table_stride;
    a.q_stride = q_stride;
    a.q_head_stride = q_head_stride;
    a.out_stride = out_stride;
    a.out_head_stride = out_head_stride;
    a.rows = rows;
    a.tokens = tokens;
    a.longest = longest;
    a.heads = cache->heads;
    a.group = q_heads / cache->heads;
    a.columns = shape.columns;
    a.wide = shape.wide;
    a.sets = shape.sets;
    a.beside = shape.beside;
    a.job_heads = shape.job_heads;
    a.blocks = shape.blocks;
    a.job_tokens = shape.job_tokens;
    a.pieces = shape.pieces;
    a.dim = cache->head_dim;
    a.page_size = cache->page_size;
    a.page_shift = page_shift(cache->page_size);
    a.pages = cache->pages;
    a.width = pool->width;
    a.sequences = pool->sequences;
    a.window = window;
    a.sinks = sinks;
    a.scale = scale;
    return hip_status(cpes::launch_attend_tree(cache->dtype, a, (hipStream_t)stream), fn);
}

int cpes_tree_accept(int32_t rows, const int32_t* starts_dev, int32_t tokens, int32_t longest, const int32_t* parents_dev,
                     const int64_t* drafted_dev, const int64_t* sampled_dev, int32_t* kept_dev, int32_t* path_dev,
                     int64_t* next_dev, void* stream)
{
    cpes::clear_error();
    const char* fn = "cpes_tree_accept";
    int rc = check_list(rows, starts_dev && kept_dev && path_dev && next_dev, fn);
    if (!rc && tokens < 0) rc = fail(CPES_ERR_INVALID_ARGUMENT, "%s: %d tokens", fn, tokens);
    if (!rc && tokens > 0 && (!drafted_dev || !sampled_dev))
        rc = fail(CPES_ERR_INVALID_ARGUMENT, "%s: drafted or sampled tokens are null", fn);
    if (!rc) rc = check_longest(longest, fn);
    if (rc || rows == 0) return rc;
    cpes::AcceptArgs a;
    a.starts = starts_dev;
    a.parents = parents_dev;
    a.drafted = drafted_dev;
    a.sampled = sampled_dev;
    a.kept = kept_dev;
    a.path = path_dev;
    a.next = next_dev;
    a.rows = rows;
    a.tokens = tokens;
    a.longest = longest;
    return hip_status(cpes::launch_tree_accept(a, (hipStream_t)stream), fn);
}

size_t cpes_sample_workspace_bytes(int32_t rows, int32_t vocab)
{
    if (rows < 0 || vocab < 1) return 0;
    // the most that any number of rows up to this takes: fewer rows are cut into more slices
    size_t most = 0;
    for (int dtype : {CPES_BF16, CPES_F32}) {
        for (int32_t r = 1; r <= std::min<int32_t>(rows, cpes::kSampleRows); ++r) most = std::max(most, sample_bytes(r, vocab, dtype));
        most = std::max(most, sample_bytes(rows, vocab, dtype));
    }
    return most;
}

int cpes_sample(const void* x_dev, int dtype, int32_t rows, int32_t vocab, int64_t stride, float scale, int32_t top_k,
                float top_p, float min_p, const float* uniforms_dev, int64_t* tokens_dev, float* logp_dev,
                void* workspace_dev, size_t workspace_bytes, void* stream)
{
    cpes::clear_error();
    const char* fn = "cpes_sample";
    int rc = check_logits(x_dev, dtype, rows, vocab, stride, scale, fn);
    if (!rc && rows > 0 && (!uniforms_dev || !tokens_dev))
        rc = fail(CPES_ERR_INVALID_ARGUMENT, "%s: uniforms or tokens are null", fn);
    if (!rc && top_k < 0) rc = fail(CPES_ERR_INVALID_ARGUMENT, "%s: top_k %d is negative", fn, top_k);
    if (!rc && !(top_p > 0.f && top_p <= 1.f))
        rc = fail(CPES_ERR_INVALID_ARGUMENT, "%s: top_p %g outside (0, 1]", fn, (double)top_p);
    if (!rc && !(min_p >= 0.f && min_p <= 1.f))
        rc = fail(CPES_ERR_INVALID_ARGUMENT, "%s: min_p %g outside [0, 1]", fn, (double)min_p);
    if (rc) return rc;
    rc = check_workspace(workspace_dev, workspace_bytes, sample_bytes(rows, vocab, dtype), fn);
    if (rc || rows == 0) return rc;
    cpes::SampleArgs a;
    int32_t at_once = std::min(rows, cpes::kSampleAtOnce);
    const cpes::SampleSplit split = cpes::sample_split(at_once, vocab, dtype);
    if (split.slices == 0) at_once = rows;                       // nothing in the workspace
    a.slices = split.slices;
    a.strip_steps = split.strip_steps;
    a.shift = split.shift;
    a.slots = split.slots;
    a.note_shift = split.note_shift;
    a.note_slots = split.note_slots;
    a.group = split.group;
    const size_t strips = (size_t)at_once * split.strips(), notes = strips * split.note_slots * cpes::kSampleLanes;
    a.notes = static_cast<uint16_t*>(workspace_dev);            // 16 bytes at a time
    a.samples = a.notes + notes;
    a.sums = reinterpret_cast<double*>(a.samples + notes);
    a.refs = reinterpret_cast<float*>(a.sums + strips * split.slots);
    a.most = a.refs + strips * split.slots;
    a.stride = stride;
    a.vocab = vocab;
    a.top_k = top_k >= vocab ? 0 : top_k;
    a.top_p = top_p;
    a.least = min_p > 0.f ? std::log((double)min_p) : -INFINITY;
    a.scale = scale;
    a.c = (double)scale * M_LOG2E;
    for (int32_t r = 0; r < rows && !rc; r += at_once) {
        a.rows = std::min(at_once, rows - r);
        a.x = static_cast<const char*>(x_dev) + (int64_t)r * stride * elem_size(dtype);
        a.uniforms = uniforms_dev + r;
        a.tokens = tokens_dev + r;
        a.logp = logp_dev ? logp_dev + r : nullptr;
        rc = hip_status(cpes::launch_sample(dtype, a, (hipStream_t)stream), fn);
        if (rows - r <= at_once) break;                          // r may not pass 2^31
    }
    return rc;
}

}  // extern "C"
