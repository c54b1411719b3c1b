// C ABI of the paged K/V cache: argument validation and launch set-up.
#include "../../include/bsfa.h"
#include "bsfa_internal.h"

#include <algorithm>
#include <cmath>
#include <cstring>

namespace {

using bsfa::fail_with;
#define FAIL(status, ...) return static_cast<bsfa_status>(fail_with(status, __VA_ARGS__))

bool misaligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

constexpr int64_t kMaxPlaces = 1 << 30;                 // of one block table
constexpr int64_t kMaxTokens = 1 << 25, kMaxRows = 1 << 26, kMaxUnits = 1 << 23;      // (grids of less than 2^32 threads)
constexpr int64_t kMaxTokenStride = 1 << 25;            // a copy addresses 16 tokens of a page with 32-bit offsets

// strides of a tensor's dimensions that have more than one element (those of the others are never used).  Of a tensor that is
// written no two elements may be the same: a dimension's step lies behind all that the dimensions of smaller steps hold.
bsfa_status check_strides(const char *name, const int64_t *stride, const int64_t *size, int n, int64_t row, bool written = false)
{
    int order[3], dims = 0;                              // by step, the smallest first
    for (int x = 0; x < n; ++x) {
        if (size[x] < 2) continue;
        if (stride[x] < 0 || stride[x] % 8) FAIL(BSFA_ERR_SHAPE, "%s: stride #%d = %lld must be a non-negative multiple of 8 elements", name, x, (long long)stride[x]);
        if ((x > 0 || written) && stride[x] < row) FAIL(BSFA_ERR_SHAPE, "%s: stride #%d = %lld is smaller than head_dim", name, x, (long long)stride[x]);
        int y = dims++;
        for (; y > 0 && stride[order[y - 1]] > stride[x]; --y) order[y] = order[y - 1];
        order[y] = x;
    }
    int64_t held = row;
    for (int y = 0; written && y < dims; ++y) {
        const int64_t step = stride[order[y]];
        if (step < held) FAIL(BSFA_ERR_SHAPE, "%s: stride #%d = %lld: two elements would be written to one place", name, order[y], (long long)step);
        if (step > INT64_MAX / size[order[y]]) FAIL(BSFA_ERR_SHAPE, "%s: stride #%d = %lld exceeds the address space", name, order[y], (long long)step);
        held += (size[order[y]] - 1) * step;
    }
    return BSFA_OK;
}

bsfa_status check_cache(const bsfa_cache *c, bool written = false)
{
    if (!c) FAIL(BSFA_ERR_NULL, "cache descriptor is NULL");
    if (c->dtype != BSFA_BF16 && c->dtype != BSFA_FP16) FAIL(BSFA_ERR_DTYPE, "dtype %d not supported (bf16 and fp16 only)", c->dtype);
    if (c->n_pages < 1 || c->n_kv_heads < 1) FAIL(BSFA_ERR_SHAPE, "n_pages and n_kv_heads must be positive");
    if (c->page_size < 16 || c->page_size > (1 << 20) || (c->page_size & (c->page_size - 1)))
        FAIL(BSFA_ERR_SHAPE, "page_size %d is not a power of two between 16 and 2^20", c->page_size);
    if (c->head_dim != 64 && c->head_dim != 128) FAIL(BSFA_ERR_UNSUPPORTED, "head_dim %d is not built (64 and 128 are)", c->head_dim);
    const int64_t size[3] = {c->n_pages, c->page_size, c->n_kv_heads};
    const int64_t k[3] = {c->k_stride_page, c->k_stride_n, c->k_stride_h}, v[3] = {c->v_stride_page, c->v_stride_n, c->v_stride_h};
    bsfa_status s = check_strides("k cache", k, size, 3, c->head_dim, written);
    if (s == BSFA_OK) s = check_strides("v cache", v, size, 3, c->head_dim, written);
    if (s != BSFA_OK) return s;
    if (k[1] > kMaxTokenStride || v[1] > kMaxTokenStride) FAIL(BSFA_ERR_SHAPE, "token strides of the cache must not exceed 2^25 elements");
    return BSFA_OK;
}

bsfa_status check_table(const bsfa_cache *c, const char *name, const int32_t *table, int64_t pages, int64_t stride_b, int batch)
{
    if (pages < 1) FAIL(BSFA_ERR_SHAPE, "%s: table_pages must be positive", name);
    if (pages * c->page_size > kMaxPlaces) FAIL(BSFA_ERR_SHAPE, "%s: %lld pages of %d tokens exceed 2^30 places", name, (long long)pages, c->page_size);
    if (batch > 1 && stride_b < 0) FAIL(BSFA_ERR_SHAPE, "%s: table_stride_b must not be negative", name);
    if (misaligned(table, 4)) FAIL(BSFA_ERR_SHAPE, "%s must be 4-byte aligned", name);
    return BSFA_OK;
}

bsfa_status check_batch(const bsfa_cache *c, int batch, int hq, int seqlen)
{
    if (batch < 1 || hq < 1 || seqlen < 1) FAIL(BSFA_ERR_SHAPE, "batch, n_q_heads and seqlen must be positive");
    if (hq % c->n_kv_heads) FAIL(BSFA_ERR_SHAPE, "n_q_heads (%d) is not a multiple of n_kv_heads (%d)", hq, c->n_kv_heads);
    if ((int64_t)batch * seqlen > kMaxTokens) FAIL(BSFA_ERR_SHAPE, "batch * seqlen exceeds 2^25 tokens");
    if ((int64_t)batch * seqlen * hq > kMaxRows) FAIL(BSFA_ERR_SHAPE, "batch * seqlen * n_q_heads exceeds 2^26 rows");
    if ((int64_t)batch * c->n_kv_heads > kMaxUnits) FAIL(BSFA_ERR_SHAPE, "batch * n_kv_heads exceeds 2^23");
    return BSFA_OK;
}

void fill_pages(bsfa::PageLayout &y, const bsfa_cache *c)
{
    y = {c->k_stride_page, c->k_stride_n, c->k_stride_h, c->v_stride_page, c->v_stride_n, c->v_stride_h, 0, c->n_pages};
    while ((1 << y.page_log2) < c->page_size) ++y.page_log2;
}

// Everything about a bsfa_paged but the data pointers.
bsfa_status check_paged(const bsfa_cache *c, const bsfa_paged *p, bool prefix)
{
    bsfa_status s = check_cache(c);
    if (s != BSFA_OK) return s;
    if (!p) FAIL(BSFA_ERR_NULL, "problem descriptor is NULL");
    s = check_batch(c, p->batch, p->n_q_heads, p->seqlen);
    if (s == BSFA_OK) s = check_table(c, "block_table", p->block_table, p->table_pages, p->table_stride_b, p->batch);
    if (s == BSFA_OK && prefix) s = check_table(c, "prefix_table", p->prefix_table, p->prefix_pages, 0, 1);
    const int64_t size[3] = {p->batch, p->seqlen, p->n_q_heads};
    const int64_t q[3] = {p->q_stride_b, p->q_stride_n, p->q_stride_h}, o[3] = {p->o_stride_b, p->o_stride_n, p->o_stride_h};
    if (s == BSFA_OK) s = check_strides("q", q, size, 3, c->head_dim);
    if (s == BSFA_OK) s = check_strides("out", o, size, 3, c->head_dim, true);
    if (s != BSFA_OK) return s;
    if (prefix && (p->prefix_len < 1 || p->prefix_len > (int64_t)p->prefix_pages * c->page_size))
        FAIL(BSFA_ERR_SHAPE, "prefix_len %d must be positive and fit %d pages of %d tokens", p->prefix_len, p->prefix_pages, c->page_size);
    if ((int64_t)p->batch * p->table_pages * (c->page_size / 16) > kMaxPlaces) FAIL(BSFA_ERR_SHAPE, "the block tables of the batch hold more than 2^34 places");
    if (p->max_cache_len < 0) FAIL(BSFA_ERR_SHAPE, "max_cache_len must not be negative");
    if (misaligned(p->q_lens, 4) || misaligned(p->cache_lens, 4)) FAIL(BSFA_ERR_SHAPE, "q_lens and cache_lens must be 4-byte aligned");
    if (p->workspace_bytes < 0) FAIL(BSFA_ERR_WORKSPACE, "workspace_bytes must not be negative");
    return BSFA_OK;
}

void fill_paged(bsfa::PagedParams &y, const bsfa_cache *c, const bsfa_paged *p, bool prefix)
{
    memset(&y, 0, sizeof(y));
    fill_pages(y.pages, c);
    y.k_cache = static_cast<const uint16_t *>(c->k);
    y.v_cache = static_cast<const uint16_t *>(c->v);
    y.cache_lens = p->cache_lens;
    y.q_lens = p->q_lens;
    y.table = p->block_table;
    y.tsb = p->table_stride_b;
    y.qsb = p->q_stride_b; y.qsn = p->q_stride_n; y.qsh = p->q_stride_h;
    y.osb = p->o_stride_b; y.osn = p->o_stride_n; y.osh = p->o_stride_h;
    y.batch = p->batch; y.seqlen = p->seqlen; y.hq = p->n_q_heads; y.hkv = c->n_kv_heads;
    y.group = p->n_q_heads / c->n_kv_heads;
    y.max_len = p->table_pages * c->page_size;
    if (p->max_cache_len) y.max_len = std::min(y.max_len, p->max_cache_len);
    if (prefix) {
        y.prefix_table = p->prefix_table;
        y.prefix = p->prefix_len;
    }
    y.scale_log2 = (float)(1.4426950408889634 / sqrt((double)c->head_dim));
}

bsfa_status attend(const bsfa_cache *c, const bsfa_paged *p, const void *q, int causal, void *out, float *lse, bool prefix, void *hip_stream)
{
    bsfa_status s = check_paged(c, p, prefix);
    if (s != BSFA_OK) return s;
    if (!c->k || !c->v || !q || !out || !p->cache_lens || !p->block_table || (prefix && !p->prefix_table))
        FAIL(BSFA_ERR_NULL, "the cache, q, out, cache_lens and the page tables must be non-NULL");
    if (misaligned(c->k, 16) || misaligned(c->v, 16) || misaligned(q, 16) || misaligned(out, 16) || misaligned(lse, 4))
        FAIL(BSFA_ERR_SHAPE, "the cache, q and out must be 16-byte aligned, lse 4-byte");
    bsfa::PagedParams y;
    fill_paged(y, c, p, prefix);
    y.q = static_cast<const uint16_t *>(q);
    y.out = static_cast<uint16_t *>(out);
    y.lse = lse;
    y.causal = causal ? 1 : 0;
    const size_t need = bsfa::paged_workspace_bytes(y, c->head_dim);
    if (need) {
        if (!p->workspace || (size_t)p->workspace_bytes < need)
            FAIL(BSFA_ERR_WORKSPACE, "workspace of %zu bytes needed, %lld given", need, p->workspace ? (long long)p->workspace_bytes : 0ll);
        if (misaligned(p->workspace, 256)) FAIL(BSFA_ERR_WORKSPACE, "the workspace must be 256-byte aligned");
        y.workspace = static_cast<unsigned char *>(p->workspace);
    }
    const hipError_t e = bsfa::launch_paged(y, c->head_dim, c->dtype == BSFA_FP16, static_cast<hipStream_t>(hip_stream));
    if (e != hipSuccess) FAIL(BSFA_ERR_HIP, "attention launch failed: %s", hipGetErrorString(e));
    return BSFA_OK;
}

}  // namespace

extern "C" {

bsfa_status bsfa_cache_append(const bsfa_cache *c, const bsfa_append *p, const void *q, const void *k, const void *v,
                              void *q_out, void *k_out, void *hip_stream)
{
    bsfa_status s = check_cache(c, true);
    if (s != BSFA_OK) return s;
    if (!p) FAIL(BSFA_ERR_NULL, "problem descriptor is NULL");
    s = check_batch(c, p->batch, p->n_q_heads, p->seqlen);
    if (s == BSFA_OK) s = check_table(c, "block_table", p->block_table, p->table_pages, p->table_stride_b, p->batch);
    if (s != BSFA_OK) return s;
    if (!c->k || !c->v || !k || !v || !p->start || !p->block_table) FAIL(BSFA_ERR_NULL, "the cache, k, v, start and block_table must be non-NULL");
    if (q && !q_out) FAIL(BSFA_ERR_NULL, "q_out must be non-NULL where q is given");
    if (q && !p->cos_sin) FAIL(BSFA_ERR_NULL, "q without cos_sin: nothing would be done to it");
    const int64_t size[3] = {p->batch, p->seqlen, c->n_kv_heads}, size_q[3] = {p->batch, p->seqlen, p->n_q_heads};
    const struct { const char *name; const void *at; const int64_t *size, stride[3]; } t[5] = {
        {"q", q, size_q, {p->q_stride_b, p->q_stride_n, p->q_stride_h}}, {"q_out", q ? q_out : nullptr, size_q, {p->qo_stride_b, p->qo_stride_n, p->qo_stride_h}},
        {"k", k, size, {p->k_stride_b, p->k_stride_n, p->k_stride_h}}, {"v", v, size, {p->v_stride_b, p->v_stride_n, p->v_stride_h}},
        {"k_out", k_out, size, {p->ko_stride_b, p->ko_stride_n, p->ko_stride_h}}};
    for (const auto &x : t) {
        if (!x.at) continue;
        s = check_strides(x.name, x.stride, x.size, 3, c->head_dim, x.at == q_out || x.at == k_out);
        if (s != BSFA_OK) return s;
        if (misaligned(x.at, 16)) FAIL(BSFA_ERR_SHAPE, "%s must be 16-byte aligned", x.name);
    }
    const int in_place[2][2] = {{0, 1}, {2, 4}};         // q and q_out, k and k_out
    for (const auto &pair : in_place) {
        const auto &in = t[pair[0]], &out = t[pair[1]];
        for (int y = 0; in.at && in.at == out.at && y < 3; ++y)
            if (in.size[y] > 1 && in.stride[y] != out.stride[y])
                FAIL(BSFA_ERR_SHAPE, "%s at the place of %s must have its strides (#%d: %lld, %lld)", out.name, in.name, y, (long long)out.stride[y], (long long)in.stride[y]);
    }
    if (misaligned(c->k, 16) || misaligned(c->v, 16)) FAIL(BSFA_ERR_SHAPE, "the cache must be 16-byte aligned");
    if (misaligned(p->seqlens, 4) || misaligned(p->start, 4)) FAIL(BSFA_ERR_SHAPE, "seqlens and start must be 4-byte aligned");
    if (p->interleaved != 0 && p->interleaved != 1) FAIL(BSFA_ERR_SHAPE, "interleaved must be 0 or 1");
    if (p->cos_sin) {
        if (p->rot_dim < 16 || p->rot_dim % 16 || p->rot_dim > c->head_dim) FAIL(BSFA_ERR_SHAPE, "rot_dim %d must be a multiple of 16 up to head_dim", p->rot_dim);
        if (p->n_positions < (int64_t)p->table_pages * c->page_size)
            FAIL(BSFA_ERR_SHAPE, "cos_sin has %d positions, the block table holds %lld", p->n_positions, (long long)p->table_pages * c->page_size);
        if (misaligned(p->cos_sin, 16)) FAIL(BSFA_ERR_SHAPE, "cos_sin must be 16-byte aligned");
    }
    bsfa::AppendParams y;
    memset(&y, 0, sizeof(y));
    fill_pages(y.pages, c);
    y.q = static_cast<const uint16_t *>(q);
    y.k = static_cast<const uint16_t *>(k);
    y.v = static_cast<const uint16_t *>(v);
    y.q_out = static_cast<uint16_t *>(q_out);
    y.k_out = static_cast<uint16_t *>(k_out);
    y.k_cache = static_cast<uint16_t *>(c->k);
    y.v_cache = static_cast<uint16_t *>(c->v);
    y.seqlens = p->seqlens; y.start = p->start; y.table = p->block_table; y.cos_sin = p->cos_sin;
    y.qsb = p->q_stride_b; y.qsn = p->q_stride_n; y.qsh = p->q_stride_h;
    y.ksb = p->k_stride_b; y.ksn = p->k_stride_n; y.ksh = p->k_stride_h;
    y.vsb = p->v_stride_b; y.vsn = p->v_stride_n; y.vsh = p->v_stride_h;
    y.qosb = p->qo_stride_b; y.qosn = p->qo_stride_n; y.qosh = p->qo_stride_h;
    y.kosb = p->ko_stride_b; y.kosn = p->ko_stride_n; y.kosh = p->ko_stride_h;
    y.tsb = p->table_stride_b;
    y.batch = p->batch; y.seqlen = p->seqlen; y.hq = p->n_q_heads; y.hkv = c->n_kv_heads;
    y.table_pages = p->table_pages;
    y.rot = p->cos_sin ? p->rot_dim : 0;
    y.interleaved = p->interleaved;
    const hipError_t e = bsfa::launch_append(y, c->head_dim, c->dtype == BSFA_FP16, static_cast<hipStream_t>(hip_stream));
    if (e != hipSuccess) FAIL(BSFA_ERR_HIP, "append launch failed: %s", hipGetErrorString(e));
    return BSFA_OK;
}

bsfa_status bsfa_paged_attention(const bsfa_cache *c, const bsfa_paged *p, const void *q, int causal, void *out, float *lse, void *hip_stream)
{
    return attend(c, p, q, causal, out, lse, false, hip_stream);
}

bsfa_status bsfa_prefix_attention(const bsfa_cache *c, const bsfa_paged *p, const void *q, int causal, void *out, float *lse, void *hip_stream)
{
    return attend(c, p, q, causal, out, lse, true, hip_stream);
}

size_t bsfa_paged_workspace_bytes(const bsfa_cache *c, const bsfa_paged *p)
{
    const bool prefix = p && p->prefix_table;
    if (check_paged(c, p, prefix) != BSFA_OK) return 0;
    bsfa::PagedParams y;
    fill_paged(y, c, p, prefix);
    return bsfa::paged_workspace_bytes(y, c->head_dim);
}

}  // extern "C"
