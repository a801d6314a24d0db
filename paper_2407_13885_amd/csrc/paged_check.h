// Argument validation that the entry points of the paged caches share.
#pragma once

#include "attnw.h"
#include "paged_common.h"

#include <cmath>

namespace {

using attnw::CacheView;
using attnw::DType;
using attnw::RuleView;

inline bool mul_overflows(int64_t a, int64_t b, int64_t* out) { return __builtin_mul_overflow(a, b, out); }
inline bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
inline bool known(int dtype) { return dtype == ATTNW_F32 || dtype == ATTNW_BF16; }
inline int64_t size_of(int dtype) { return dtype == ATTNW_F32 ? 4 : 2; }

// half-open byte ranges [a, a + na) and [b, b + nb)
inline bool overlaps(const void* a, int64_t na, const void* b, int64_t nb)
{
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
    return a0 < b0 + (uintptr_t)nb && b0 < a0 + (uintptr_t)na;
}

constexpr int64_t kMostSlots = (int64_t)1 << 30;

// Bytes from a tensor's start to the end of its last row: rows of `wide` elements, `stride` apart.
inline int64_t extent(int64_t rows, int64_t stride, int64_t wide, int64_t size) { return ((rows - 1) * stride + wide) * size; }

// Everything about a cache that the host can see.  (size: bytes of an element of K and V; the type of what meets them, but for caches in 8 bits)
inline int check_sizes(const attnw_cache* c, int64_t size)
{
    if (!known(c->dtype)) return ATTNW_ERR_DTYPE;
    if (c->batch < 0 || c->pages < 0 || c->max_pages < 0 || c->page_size < 0 || c->kv_heads < 0 || c->d < 0) return ATTNW_ERR_SHAPE;
    int64_t rows, bytes, slots;
    if (mul_overflows(c->pages, c->page_size, &rows) || mul_overflows(rows, c->kv_heads, &rows) || mul_overflows(rows, c->d, &bytes) ||
        mul_overflows(bytes, size, &bytes) || mul_overflows(c->max_pages, c->page_size, &slots))
        return ATTNW_ERR_SHAPE;
    return ATTNW_OK;
}

inline int check_support(const attnw_cache* c, int64_t size)
{
    const int64_t step = size == 4 ? 4 : 16;
    if (c->d < step || c->d > 256 || c->d % step != 0) return ATTNW_ERR_UNSUPPORTED;
    if (c->pages < 1 || c->max_pages < 1 || c->page_size < 1 || c->kv_heads < 1) return ATTNW_ERR_UNSUPPORTED;
    const int64_t most = (int64_t)1 << 30;
    int64_t heads;
    if (c->pages > most || c->batch > most || c->kv_heads > (1 << 16) || c->max_pages * c->page_size > kMostSlots ||
        mul_overflows(c->batch, c->kv_heads, &heads) || heads > (1 << 23) ||
        c->kv_heads * c->page_size * c->d * size >= (int64_t)1 << 32)   // (a page: offsets in it have 32 bits)
        return ATTNW_ERR_UNSUPPORTED;
    return ATTNW_OK;
}

inline int check_pointers(const attnw_cache* c)
{
    return c->K && c->V && c->table && c->lengths ? ATTNW_OK : ATTNW_ERR_NULL;
}

inline bool cache_aligned(const attnw_cache* c)
{
    return aligned(c->K, 16) && aligned(c->V, 16) && aligned(c->table, 4) && aligned(c->lengths, 4);
}

inline int64_t cache_bytes(const attnw_cache* c, int64_t size) { return c->pages * c->page_size * c->kv_heads * c->d * size; }

inline CacheView view(const attnw_cache* c, int64_t size)
{
    CacheView v;
    v.K = static_cast<const char*>(c->K);
    v.V = static_cast<const char*>(c->V);
    v.table = c->table;
    v.lengths = c->lengths;
    v.row_bytes = (int32_t)(c->d * size);
    v.head_bytes = (uint32_t)(c->page_size * v.row_bytes);
    v.page_bytes = (uint32_t)(c->kv_heads * v.head_bytes);
    v.batch = (int32_t)c->batch;
    v.pages = (int32_t)c->pages;
    v.max_pages = (int32_t)c->max_pages;
    v.kv_heads = (int32_t)c->kv_heads;
    v.slots = (int32_t)(c->max_pages * c->page_size);
    v.page = attnw::fast_div((uint32_t)c->page_size);
    return v;
}

// Shared by attention and sums: sizes of the call, and the rule of the scores.
inline int check_call(const attnw_cache* c, const attnw_rule* r, int64_t tokens, int64_t heads, int64_t q_stride)
{
    if (tokens < 0 || heads < 0 || q_stride < 0 || r->window < 0 || !(r->cap >= 0.0f)) return ATTNW_ERR_SHAPE;
    int64_t n;
    if (mul_overflows(tokens, heads, &n) || mul_overflows(n, c->d * size_of(c->dtype), &n) || mul_overflows(tokens, q_stride, &n) ||
        mul_overflows(n, size_of(c->dtype), &n))
        return ATTNW_ERR_SHAPE;
    return ATTNW_OK;
}

inline int check_call_support(const attnw_cache* c, int64_t size, const attnw_rule* r, int64_t tokens, int64_t heads, int64_t q_stride)
{
    const int e = check_support(c, size);
    if (e != ATTNW_OK) return e;
    if (heads % c->kv_heads != 0 || heads > (1 << 16) || tokens > ((int64_t)1 << 30) || tokens * heads > ((int64_t)1 << 30)) return ATTNW_ERR_UNSUPPORTED;
    if (q_stride < heads * c->d || q_stride * size_of(c->dtype) % 16 != 0) return ATTNW_ERR_UNSUPPORTED;
    if (!std::isfinite(r->scale) || !std::isfinite(r->cap)) return ATTNW_ERR_UNSUPPORTED;
    return ATTNW_OK;
}

inline RuleView view(const attnw_rule* r)
{
    return {r->scale, r->cap, r->slopes, r->prefix, (int32_t)(r->window == 0 || r->window > attnw::kNoWindow ? attnw::kNoWindow : r->window)};
}

// (caches of their dtype)
inline int check_sizes(const attnw_cache* c) { return check_sizes(c, size_of(c->dtype)); }
inline int check_support(const attnw_cache* c) { return check_support(c, size_of(c->dtype)); }
inline int check_call_support(const attnw_cache* c, const attnw_rule* r, int64_t tokens, int64_t heads, int64_t q_stride)
{
    return check_call_support(c, size_of(c->dtype), r, tokens, heads, q_stride);
}
inline int64_t cache_bytes(const attnw_cache* c) { return cache_bytes(c, size_of(c->dtype)); }
inline CacheView view(const attnw_cache* c) { return view(c, size_of(c->dtype)); }

inline int status(hipError_t e) { return e == hipSuccess ? ATTNW_OK : ATTNW_ERR_LAUNCH; }

}  // namespace
