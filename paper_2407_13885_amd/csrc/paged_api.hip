// C ABI of the paged cache and of rotary positions (declared in include/attnw.h): argument validation on the host, then launches on the caller's stream.
#include "paged_check.h"

extern "C" {

int attnw_rotary_table(float* table, int64_t positions, int64_t rot, double base, double factor, double low, double high, double original, double gain,
                       void* stream)
{
    if (positions < 0 || rot < 0) return ATTNW_ERR_SHAPE;
    if (positions == 0 || rot == 0) return ATTNW_OK;
    if (!table) return ATTNW_ERR_NULL;
    int64_t bytes;
    if (mul_overflows(positions, rot, &bytes) || mul_overflows(bytes, 4, &bytes)) return ATTNW_ERR_SHAPE;
    if (rot % 2 != 0 || rot > 256 || positions > ((int64_t)1 << 30)) return ATTNW_ERR_UNSUPPORTED;
    if (!(base > 0.0) || !(factor > 0.0) || !std::isfinite(base) || !std::isfinite(factor) || !std::isfinite(gain) || !(low >= 0.0) || !(high >= low) ||
        !std::isfinite(original) || !(original >= 0.0))
        return ATTNW_ERR_UNSUPPORTED;
    if (!aligned(table, 16)) return ATTNW_ERR_ALIGN;
    return status(attnw::launch_rotary_table(table, positions, rot, base, factor, low, high, original, gain, static_cast<hipStream_t>(stream)));
}

int attnw_rotary(const void* X, void* Y, const float* table, const int32_t* positions, int64_t tokens, int64_t heads, int64_t d, int64_t rot, int64_t rows,
                 int64_t x_stride, int64_t y_stride, int layout, int inverse, int dtype, void* stream)
{
    if (!known(dtype)) return ATTNW_ERR_DTYPE;
    if (tokens < 0 || heads < 0 || d < 0 || rot < 0 || rows < 0 || x_stride < 0 || y_stride < 0) return ATTNW_ERR_SHAPE;
    if (tokens == 0 || heads == 0 || d == 0) return ATTNW_OK;
    if (!X || !Y || !table || !positions) return ATTNW_ERR_NULL;
    int64_t wide, n;
    const int64_t size = size_of(dtype);
    if (mul_overflows(heads, d, &wide) || mul_overflows(tokens, x_stride, &n) || mul_overflows(n, size, &n) || mul_overflows(tokens, y_stride, &n) ||
        mul_overflows(n, size, &n) || mul_overflows(rows, rot, &n) || mul_overflows(n, 4, &n))
        return ATTNW_ERR_SHAPE;
    if (rot < 2 || rot % 2 != 0 || rot > d || d > 256 || rows < 1 || (layout != ATTNW_HALVES && layout != ATTNW_PAIRS) || tokens > ((int64_t)1 << 30) ||
        heads > (1 << 16) || x_stride < wide || y_stride < wide)
        return ATTNW_ERR_UNSUPPORTED;
    if (!aligned(X, 16) || !aligned(Y, 16) || !aligned(table, 16) || !aligned(positions, 4)) return ATTNW_ERR_ALIGN;
    const int64_t x_bytes = extent(tokens, x_stride, wide, size), y_bytes = extent(tokens, y_stride, wide, size);
    if (!(X == Y && x_stride == y_stride) && overlaps(X, x_bytes, Y, y_bytes)) return ATTNW_ERR_ALIAS;
    if (overlaps(Y, y_bytes, table, rows * rot * 4) || overlaps(Y, y_bytes, positions, tokens * 4)) return ATTNW_ERR_ALIAS;
    attnw::RotaryArgs a{};
    a.dt = static_cast<DType>(dtype);
    a.Q = X;
    a.R = Y;
    a.angles = table;
    a.positions = positions;
    a.tokens = tokens;
    a.heads = heads;
    a.d = d;
    a.rot = rot;
    a.rows = rows;
    a.q_stride = x_stride;
    a.r_stride = y_stride;
    a.interleaved = layout == ATTNW_PAIRS;
    a.inverse = inverse != 0;
    return status(attnw::launch_rotary(a, static_cast<hipStream_t>(stream)));
}

int attnw_cache_append(const attnw_cache* cache, const void* Q, const void* K, const void* V, void* R, const float* table, const int32_t* positions,
                       const int32_t* starts, int64_t tokens, int64_t heads, int64_t rot, int64_t rows, int64_t q_stride, int64_t kv_stride, int layout,
                       void* stream)
{
    if (!cache) return ATTNW_ERR_NULL;
    int e = check_sizes(cache);
    if (e != ATTNW_OK) return e;
    if (tokens < 0 || heads < 0 || rot < 0 || rows < 0 || q_stride < 0 || kv_stride < 0) return ATTNW_ERR_SHAPE;
    if (cache->batch == 0 || tokens == 0) return ATTNW_OK;
    if ((e = check_pointers(cache)) != ATTNW_OK) return e;
    if (!K || !V || !starts || (heads > 0 && (!Q || !R)) || (rot > 0 && !table)) return ATTNW_ERR_NULL;
    const int64_t size = size_of(cache->dtype);
    int64_t n, wide;
    if (mul_overflows(heads, cache->d, &wide) || mul_overflows(tokens, q_stride, &n) || mul_overflows(n, size, &n) || mul_overflows(tokens, kv_stride, &n) ||
        mul_overflows(n, size, &n) || mul_overflows(tokens, wide, &n) || mul_overflows(n, size, &n) || mul_overflows(rows, rot, &n) ||
        mul_overflows(n, 4, &n))
        return ATTNW_ERR_SHAPE;
    if ((e = check_support(cache)) != ATTNW_OK) return e;
    const int64_t kv_wide = cache->kv_heads * cache->d;
    if (rot % 2 != 0 || rot > cache->d || (rot > 0 && rows < 1) || (layout != ATTNW_HALVES && layout != ATTNW_PAIRS) || tokens > ((int64_t)1 << 30) ||
        heads > (1 << 16) || q_stride < wide || kv_stride < kv_wide)
        return ATTNW_ERR_UNSUPPORTED;
    if (!cache_aligned(cache) || !aligned(Q, 16) || !aligned(K, 16) || !aligned(V, 16) || !aligned(R, 16) || !aligned(table, 16) ||
        !aligned(positions, 4) || !aligned(starts, 4))
        return ATTNW_ERR_ALIGN;
    const int64_t kv_bytes = extent(tokens, kv_stride, kv_wide, size), all = cache_bytes(cache);
    struct Range { const void* at; int64_t bytes; };
    const Range read[] = {{K, kv_bytes}, {V, kv_bytes}, {table, rows * rot * 4}, {positions, tokens * 4}, {starts, (cache->batch + 1) * 4},
                          {cache->table, cache->batch * cache->max_pages * 4}, {cache->lengths, cache->batch * 4}};
    for (const Range& r : read)
        if (r.at && (overlaps(cache->K, all, r.at, r.bytes) || overlaps(cache->V, all, r.at, r.bytes))) return ATTNW_ERR_ALIAS;
    if (overlaps(cache->K, all, cache->V, all)) return ATTNW_ERR_ALIAS;
    if (heads > 0) {
        const int64_t q_bytes = extent(tokens, q_stride, wide, size), r_bytes = tokens * wide * size;
        if (!(Q == R && q_stride == wide) && overlaps(Q, q_bytes, R, r_bytes)) return ATTNW_ERR_ALIAS;
        if (overlaps(cache->K, all, Q, q_bytes) || overlaps(cache->V, all, Q, q_bytes) || overlaps(cache->K, all, R, r_bytes) ||
            overlaps(cache->V, all, R, r_bytes))
            return ATTNW_ERR_ALIAS;
        for (const Range& r : read)
            if (r.at && overlaps(R, r_bytes, r.at, r.bytes)) return ATTNW_ERR_ALIAS;
    }
    attnw::RotaryArgs a{};
    a.dt = static_cast<DType>(cache->dtype);
    a.Q = Q;
    a.K = K;
    a.V = V;
    a.R = R;
    a.Kc = cache->K;
    a.Vc = cache->V;
    a.angles = table;
    a.positions = positions;
    a.starts = starts;
    a.tokens = tokens;
    a.heads = heads;
    a.d = cache->d;
    a.rot = rot;
    a.rows = rows;
    a.q_stride = q_stride;
    a.kv_stride = kv_stride;
    a.r_stride = wide;
    a.interleaved = layout == ATTNW_PAIRS;
    a.cache = view(cache);
    return status(attnw::launch_rotary(a, static_cast<hipStream_t>(stream)));
}

int64_t attnw_paged_workspace(const attnw_cache* cache, int64_t tokens, int64_t heads)
{
    if (!cache) return ATTNW_ERR_NULL;
    int e = check_sizes(cache);
    if (e != ATTNW_OK) return e;
    const attnw_rule rule = {1.0f, 0.0f, nullptr, nullptr, 0};
    int64_t wide;
    if (mul_overflows(heads, cache->d, &wide)) return ATTNW_ERR_SHAPE;
    if ((e = check_call(cache, &rule, tokens, heads, wide)) != ATTNW_OK) return e;
    if (cache->batch == 0 || tokens == 0 || heads == 0) return 0;
    if ((e = check_call_support(cache, &rule, tokens, heads, wide)) != ATTNW_OK) return e;
    attnw::PagedArgs a{};
    a.dt = static_cast<DType>(cache->dtype);
    a.cache = view(cache);
    a.tokens = tokens;
    a.heads = heads;
    return attnw::paged_workspace(a);
}

int attnw_paged_attention(const attnw_cache* cache, const attnw_rule* rule, const void* Q, void* O, float* lse, const int32_t* starts, int64_t tokens,
                          int64_t heads, int64_t q_stride, void* workspace, int64_t workspace_bytes, void* stream)
{
    if (!cache || !rule) return ATTNW_ERR_NULL;
    int e = check_sizes(cache);
    if (e != ATTNW_OK) return e;
    if ((e = check_call(cache, rule, tokens, heads, q_stride)) != ATTNW_OK) return e;
    if (workspace_bytes < 0) return ATTNW_ERR_SHAPE;
    if (cache->batch == 0 || tokens == 0 || heads == 0) return ATTNW_OK;
    if ((e = check_pointers(cache)) != ATTNW_OK) return e;
    if (!Q || !O || !starts) return ATTNW_ERR_NULL;
    if ((e = check_call_support(cache, rule, tokens, heads, q_stride)) != ATTNW_OK) return e;
    attnw::PagedArgs a{};
    a.dt = static_cast<DType>(cache->dtype);
    a.cache = view(cache);
    a.rule = view(rule);
    a.Q = Q;
    a.O = O;
    a.lse = lse;
    a.workspace = static_cast<float*>(workspace);
    a.starts = starts;
    a.tokens = tokens;
    a.heads = heads;
    a.q_stride = q_stride;
    const int64_t need = attnw::paged_workspace(a);
    if (need > 0 && !workspace) return ATTNW_ERR_NULL;
    if (workspace_bytes < need) return ATTNW_ERR_WORKSPACE;
    if (!cache_aligned(cache) || !aligned(Q, 16) || !aligned(O, 16) || !aligned(lse, 4) || !aligned(starts, 4) || !aligned(workspace, 16) ||
        !aligned(rule->slopes, 4) || !aligned(rule->prefix, 4))
        return ATTNW_ERR_ALIGN;
    const int64_t size = size_of(cache->dtype), out = tokens * heads * cache->d * size, all = cache_bytes(cache);
    struct Range { const void* at; int64_t bytes; };
    const Range written[] = {{O, out}, {lse, tokens * heads * 4}, {workspace, need}};
    const Range read[] = {{Q, extent(tokens, q_stride, heads * cache->d, size)}, {cache->K, all}, {cache->V, all}, {cache->table, cache->batch * cache->max_pages * 4},
                          {cache->lengths, cache->batch * 4}, {starts, (cache->batch + 1) * 4}, {rule->slopes, heads * 4}, {rule->prefix, cache->batch * 4}};
    for (const Range& w : written) {
        if (!w.at || !w.bytes) continue;
        for (const Range& r : read)
            if (r.at && overlaps(w.at, w.bytes, r.at, r.bytes)) return ATTNW_ERR_ALIAS;
        for (const Range& o : written)
            if (&o != &w && o.at && o.bytes && overlaps(w.at, w.bytes, o.at, o.bytes)) return ATTNW_ERR_ALIAS;
    }
    return status(attnw::launch_paged_attention(a, static_cast<hipStream_t>(stream)));
}

int attnw_paged_sums(const attnw_cache* cache, const attnw_rule* rule, const void* Q, const float* lse, const float* before, float* sums,
                     const int32_t* starts, int64_t tokens, int64_t heads, int64_t q_stride, void* stream)
{
    if (!cache || !rule) return ATTNW_ERR_NULL;
    int e = check_sizes(cache);
    if (e != ATTNW_OK) return e;
    if ((e = check_call(cache, rule, tokens, heads, q_stride)) != ATTNW_OK) return e;
    int64_t elems;
    if (mul_overflows(cache->batch, cache->kv_heads, &elems) || mul_overflows(elems, cache->max_pages * cache->page_size, &elems) ||
        mul_overflows(elems, 4, &elems))
        return ATTNW_ERR_SHAPE;
    if (cache->batch == 0) return ATTNW_OK;
    if (!cache->K || !cache->table || !cache->lengths) return ATTNW_ERR_NULL;
    // (no tokens: the sums from before, still)
    if (!sums || !starts || (tokens > 0 && heads > 0 && (!Q || !lse))) return ATTNW_ERR_NULL;
    if ((e = check_call_support(cache, rule, tokens, heads, q_stride)) != ATTNW_OK) return e;
    if (heads == 0 || elems > (int64_t)1 << 36) return ATTNW_ERR_UNSUPPORTED;   // (blocks of 16 slots or more: fewer than 2^31)
    if (!aligned(cache->K, 16) || !aligned(cache->table, 4) || !aligned(cache->lengths, 4) || !aligned(Q, 16) || !aligned(lse, 4) || !aligned(before, 4) ||
        !aligned(sums, 4) || !aligned(starts, 4) || !aligned(rule->slopes, 4) || !aligned(rule->prefix, 4))
        return ATTNW_ERR_ALIGN;
    struct Range { const void* at; int64_t bytes; };
    const Range read[] = {{tokens > 0 ? Q : nullptr, extent(tokens, q_stride, heads * cache->d, size_of(cache->dtype))}, {cache->K, cache_bytes(cache)},
                          {cache->V, cache_bytes(cache)},          // (not read here, but the cache's)
                          {cache->table, cache->batch * cache->max_pages * 4}, {cache->lengths, cache->batch * 4}, {starts, (cache->batch + 1) * 4},
                          {rule->slopes, heads * 4}, {rule->prefix, cache->batch * 4}, {tokens > 0 ? lse : nullptr, tokens * heads * 4},
                          {before == sums ? nullptr : before, elems}};
    for (const Range& r : read)
        if (r.at && overlaps(sums, elems, r.at, r.bytes)) return ATTNW_ERR_ALIAS;
    attnw::SumsArgs a{};
    a.dt = static_cast<DType>(cache->dtype);
    a.cache = view(cache);
    a.rule = view(rule);
    a.Q = Q;
    a.lse = lse;
    a.before = before;
    a.sums = sums;
    a.starts = starts;
    a.tokens = tokens;
    a.heads = heads;
    a.q_stride = q_stride;
    return status(attnw::launch_paged_sums(a, static_cast<hipStream_t>(stream)));
}

int attnw_cache_evict(const attnw_cache* cache, const attnw_cache* into, const float* sums, float* into_sums, int32_t* kept, int64_t keep, int64_t recent,
                      void* stream)
{
    if (!cache || !into) return ATTNW_ERR_NULL;
    int e = check_sizes(cache);
    if (e == ATTNW_OK) e = check_sizes(into);
    if (e != ATTNW_OK) return e;
    if (keep < 0 || recent < 0 || recent > keep) return ATTNW_ERR_SHAPE;
    if (into->dtype != cache->dtype) return ATTNW_ERR_DTYPE;
    if (into->batch != cache->batch || into->kv_heads != cache->kv_heads || into->d != cache->d) return ATTNW_ERR_SHAPE;
    int64_t heads, from_elems, into_elems, kept_elems;
    if (mul_overflows(cache->batch, cache->kv_heads, &heads) || mul_overflows(heads, cache->max_pages * cache->page_size, &from_elems) ||
        mul_overflows(heads, into->max_pages * into->page_size, &into_elems) || mul_overflows(heads, keep, &kept_elems) ||
        mul_overflows(from_elems, 4, &from_elems) || mul_overflows(into_elems, 4, &into_elems) || mul_overflows(kept_elems, 4, &kept_elems))
        return ATTNW_ERR_SHAPE;
    if (cache->batch == 0) return ATTNW_OK;
    if ((e = check_pointers(cache)) != ATTNW_OK || (e = check_pointers(into)) != ATTNW_OK) return e;
    if (!sums || !into_sums || !kept) return ATTNW_ERR_NULL;
    if ((e = check_support(cache)) != ATTNW_OK || (e = check_support(into)) != ATTNW_OK) return e;
    // (a sequence keeps at least one slot: what is left of it is a sequence still)
    if (keep < 1 || keep > into->max_pages * into->page_size || keep * (cache->d * size_of(cache->dtype) / 16) > ((int64_t)1 << 30)) return ATTNW_ERR_UNSUPPORTED;
    if (!cache_aligned(cache) || !cache_aligned(into) || !aligned(sums, 4) || !aligned(into_sums, 4) || !aligned(kept, 4)) return ATTNW_ERR_ALIGN;
    struct Range { const void* at; int64_t bytes; };
    const int64_t from_bytes = cache_bytes(cache), into_bytes = cache_bytes(into);
    const Range written[] = {{into->K, into_bytes}, {into->V, into_bytes}, {into_sums, into_elems}, {kept, kept_elems}, {into->lengths, into->batch * 4}};
    const Range read[] = {{cache->K, from_bytes}, {cache->V, from_bytes}, {sums, from_elems}, {cache->table, cache->batch * cache->max_pages * 4},
                          {into->table, into->batch * into->max_pages * 4}, {cache->lengths, cache->batch * 4}};
    for (const Range& w : written) {
        for (const Range& r : read) {
            // the pages may be of one pool, and the lengths may take the place of the old ones
            const bool same_pool = (w.at == into->K && r.at == cache->K) || (w.at == into->V && r.at == cache->V);
            if ((same_pool || (w.at == into->lengths && r.at == cache->lengths)) && w.at == r.at && w.bytes == r.bytes) continue;
            if (overlaps(w.at, w.bytes, r.at, r.bytes)) return ATTNW_ERR_ALIAS;
        }
        for (const Range& o : written)
            if (&o != &w && overlaps(w.at, w.bytes, o.at, o.bytes)) return ATTNW_ERR_ALIAS;
    }
    return status(attnw::launch_evict(view(cache), view(into), into->lengths, sums, into_sums, kept, keep, recent, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
