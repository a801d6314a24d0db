// C ABI of the paged cache in 8 bits and of rotary positions with several axes (declared in include/attnw.h): argument validation on the host, then launches on the
// caller's stream.
#include "paged_check.h"

namespace {

using attnw::AxesMap;
using attnw::ScalesView;

// Sizes of the axes of a rotation, and which pair of columns is whose.
int check_axes(const attnw_axes* a)
{
    if (a->count < 0) return ATTNW_ERR_SHAPE;
    for (int i = 0; i < a->count && i < 4; ++i)
        if (a->pairs[i] < 0) return ATTNW_ERR_SHAPE;
    return ATTNW_OK;
}
int map_axes(const attnw_axes* a, int64_t rot, AxesMap* m)
{
    if (a->count < 1 || a->count > 4 || (a->order != ATTNW_SECTIONS && a->order != ATTNW_TURNS)) return ATTNW_ERR_UNSUPPORTED;
    int64_t all = 0;
    for (int i = 0; i < a->count; ++i) {
        if (a->pairs[i] < 1) return ATTNW_ERR_UNSUPPORTED;
        all += a->pairs[i];
    }
    if (all * 2 != rot || rot > 256) return ATTNW_ERR_UNSUPPORTED;
    *m = AxesMap{};
    m->count = a->count;
    m->fresh = a->fresh != 0;
    int given[4] = {};
    for (int i = 0; i < a->count; ++i) m->pairs[i] = a->pairs[i];
    for (int j = 0, axis = 0; j < all; ++j) {
        while (given[axis] == m->pairs[axis]) axis = (axis + 1) % m->count;   // (one has some left)
        m->axis[j] = (uint8_t)axis;
        m->index[j] = (uint8_t)given[axis]++;
        if (a->order == ATTNW_TURNS) axis = (axis + 1) % m->count;
    }
    return ATTNW_OK;
}

// Everything about a cache in 8 bits that the host can see: an element of K and V is a byte.
int check_sizes(const attnw_byte_cache* c)
{
    const int e = check_sizes(&c->cache, 1);
    return e != ATTNW_OK ? e : c->block < 0 ? ATTNW_ERR_SHAPE : ATTNW_OK;
}
int check_pointers(const attnw_byte_cache* c)
{
    const int e = check_pointers(&c->cache);
    return e != ATTNW_OK ? e : c->K_scales && c->V_scales ? ATTNW_OK : ATTNW_ERR_NULL;
}
int check_block(const attnw_byte_cache* c)   // (of a cache whose sizes are supported otherwise)
{
    if (c->block < 1 || c->block > c->cache.page_size || c->cache.page_size % c->block != 0) return ATTNW_ERR_UNSUPPORTED;
    return cache_bytes(&c->cache, 1) < (int64_t)1 << 47 ? ATTNW_OK : ATTNW_ERR_UNSUPPORTED;   // (kernels keep scales beside 48 bits of a place)
}
constexpr int64_t kMostBlock = (int64_t)1 << 30;    // elements of a block and head: appending counts its units, a column each at the least, in 32 bits
int64_t scale_bytes(const attnw_byte_cache* c) { return c->cache.pages * c->cache.kv_heads * (c->cache.page_size / c->block); }
ScalesView scales(const attnw_byte_cache* c)
{
    return {c->K_scales, c->V_scales, attnw::fast_div((uint32_t)c->block), (int32_t)(c->cache.page_size / c->block)};
}

struct Range {
    const void* at;
    int64_t bytes;
};
// Whether something that is written overlaps something else that is written or read.
template <int W, int R> bool any_overlap(const Range (&written)[W], const Range (&read)[R])
{
    for (const Range& w : written) {
        if (!w.at || !w.bytes) continue;
        for (const Range& r : read)
            if (r.at && r.bytes && overlaps(w.at, w.bytes, r.at, r.bytes)) return true;
        for (const Range& o : written)
            if (&o != &w && o.at && o.bytes && overlaps(w.at, w.bytes, o.at, o.bytes)) return true;
    }
    return false;
}

}  // namespace

extern "C" {

int attnw_rotary_axes_table(float* table, const attnw_axes* axes, int64_t positions, int64_t rot, double base, double factor, double low, double high, double original,
                            double gain, void* stream)
{
    if (!axes) return ATTNW_ERR_NULL;
    if (positions < 0 || rot < 0) return ATTNW_ERR_SHAPE;
    int e = check_axes(axes);
    if (e != ATTNW_OK) return e;
    if (positions == 0 || rot == 0) return ATTNW_OK;
    if (!table) return ATTNW_ERR_NULL;
    int64_t bytes;
    if (mul_overflows(positions, rot, &bytes) || mul_overflows(bytes, 4, &bytes)) return ATTNW_ERR_SHAPE;
    if (rot % 2 != 0 || rot > 256 || positions > ((int64_t)1 << 30)) return ATTNW_ERR_UNSUPPORTED;
    if (!(base > 0.0) || !(factor > 0.0) || !std::isfinite(base) || !std::isfinite(factor) || !std::isfinite(gain) || !(low >= 0.0) || !(high >= low) ||
        !std::isfinite(original) || !(original >= 0.0))
        return ATTNW_ERR_UNSUPPORTED;
    AxesMap map;
    if ((e = map_axes(axes, rot, &map)) != ATTNW_OK) return e;
    if (!aligned(table, 16)) return ATTNW_ERR_ALIGN;
    return status(attnw::launch_rotary_axes_table(table, map, positions, rot, base, factor, low, high, original, gain, static_cast<hipStream_t>(stream)));
}

int attnw_rotary_axes(const void* X, void* Y, const float* table, const int32_t* positions, const attnw_axes* axes, int64_t tokens, int64_t heads, int64_t d, int64_t rot,
                      int64_t rows, int64_t x_stride, int64_t y_stride, int layout, int inverse, int dtype, void* stream)
{
    if (!axes) return ATTNW_ERR_NULL;
    if (!known(dtype)) return ATTNW_ERR_DTYPE;
    if (tokens < 0 || heads < 0 || d < 0 || rot < 0 || rows < 0 || x_stride < 0 || y_stride < 0) return ATTNW_ERR_SHAPE;
    int e = check_axes(axes);
    if (e != ATTNW_OK) return e;
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
    AxesMap map;
    if ((e = map_axes(axes, rot, &map)) != ATTNW_OK) return e;
    if (!aligned(X, 16) || !aligned(Y, 16) || !aligned(table, 16) || !aligned(positions, 4)) return ATTNW_ERR_ALIGN;
    const int64_t x_bytes = extent(tokens, x_stride, wide, size), y_bytes = extent(tokens, y_stride, wide, size);
    if (!(X == Y && x_stride == y_stride) && overlaps(X, x_bytes, Y, y_bytes)) return ATTNW_ERR_ALIAS;
    if (overlaps(Y, y_bytes, table, rows * rot * 4) || overlaps(Y, y_bytes, positions, map.count * tokens * 4)) return ATTNW_ERR_ALIAS;
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
    return status(attnw::launch_rotary_axes(a, map, static_cast<hipStream_t>(stream)));
}

int attnw_byte_cache_append(const attnw_byte_cache* cache, const void* Q, const void* K, const void* V, void* R, const float* table, const int32_t* positions,
                        const attnw_axes* axes, const int32_t* starts, int64_t tokens, int64_t heads, int64_t rot, int64_t rows, int64_t q_stride, int64_t kv_stride,
                        int layout, void* stream)
{
    if (!cache) return ATTNW_ERR_NULL;
    int e = check_sizes(cache);
    if (e != ATTNW_OK) return e;
    if (tokens < 0 || heads < 0 || rot < 0 || rows < 0 || q_stride < 0 || kv_stride < 0) return ATTNW_ERR_SHAPE;
    if (axes && (e = check_axes(axes)) != ATTNW_OK) return e;
    const attnw_cache& c = cache->cache;
    if (c.batch == 0 || tokens == 0) return ATTNW_OK;
    if ((e = check_pointers(cache)) != ATTNW_OK) return e;
    if (!K || !V || !starts || (heads > 0 && (!Q || !R)) || (rot > 0 && !table) || (axes && !positions)) return ATTNW_ERR_NULL;
    const int64_t size = size_of(c.dtype);
    int64_t n, wide;
    if (mul_overflows(heads, c.d, &wide) || mul_overflows(tokens, q_stride, &n) || mul_overflows(n, size, &n) || mul_overflows(tokens, kv_stride, &n) ||
        mul_overflows(n, size, &n) || mul_overflows(tokens, wide, &n) || mul_overflows(n, size, &n) || mul_overflows(rows, rot, &n) || mul_overflows(n, 4, &n))
        return ATTNW_ERR_SHAPE;
    if ((e = check_support(&c, 1)) != ATTNW_OK || (e = check_block(cache)) != ATTNW_OK) return e;
    if (cache->block * c.d > kMostBlock) return ATTNW_ERR_UNSUPPORTED;
    const int64_t kv_wide = c.kv_heads * c.d;
    if (rot % 2 != 0 || rot > c.d || (rot > 0 && rows < 1) || (layout != ATTNW_HALVES && layout != ATTNW_PAIRS) || tokens > ((int64_t)1 << 30) ||
        heads > (1 << 16) || q_stride < wide || kv_stride < kv_wide)
        return ATTNW_ERR_UNSUPPORTED;
    AxesMap map;
    if (axes && (e = map_axes(axes, rot, &map)) != ATTNW_OK) return e;
    if (!cache_aligned(&c) || !aligned(Q, 16) || !aligned(K, 16) || !aligned(V, 16) || !aligned(R, 16) || !aligned(table, 16) || !aligned(positions, 4) ||
        !aligned(starts, 4))
        return ATTNW_ERR_ALIGN;
    const int64_t kv_bytes = extent(tokens, kv_stride, kv_wide, size), all = cache_bytes(&c, 1), of_scales = scale_bytes(cache);
    const int64_t q_bytes = heads > 0 ? extent(tokens, q_stride, wide, size) : 0, r_bytes = tokens * wide * size;
    const bool in_place = Q == R && q_stride == wide;
    const Range written[] = {{c.K, all}, {c.V, all}, {cache->K_scales, of_scales}, {cache->V_scales, of_scales}, {heads > 0 ? R : nullptr, r_bytes}};
    const Range read[] = {{in_place ? nullptr : Q, q_bytes}, {K, kv_bytes}, {V, kv_bytes}, {table, rows * rot * 4}, {positions, (axes ? map.count : 1) * tokens * 4},
                          {starts, (c.batch + 1) * 4}, {c.table, c.batch * c.max_pages * 4}, {c.lengths, c.batch * 4}};
    if (any_overlap(written, read)) return ATTNW_ERR_ALIAS;
    attnw::RotaryArgs a{};
    a.dt = static_cast<DType>(c.dtype);
    a.Q = Q;
    a.K = K;
    a.V = V;
    a.R = R;
    a.Kc = c.K;
    a.Vc = c.V;
    a.angles = table;
    a.positions = positions;
    a.starts = starts;
    a.tokens = tokens;
    a.heads = heads;
    a.d = c.d;
    a.rot = rot;
    a.rows = rows;
    a.q_stride = q_stride;
    a.kv_stride = kv_stride;
    a.r_stride = wide;
    a.interleaved = layout == ATTNW_PAIRS;
    a.cache = view(&c, 1);
    return status(attnw::launch_byte_append(a, scales(cache), axes ? &map : nullptr, static_cast<hipStream_t>(stream)));
}

int64_t attnw_byte_paged_workspace(const attnw_byte_cache* cache, int64_t tokens, int64_t heads)
{
    if (!cache) return ATTNW_ERR_NULL;
    int e = check_sizes(cache);
    if (e != ATTNW_OK) return e;
    const attnw_cache& c = cache->cache;
    const attnw_rule rule = {1.0f, 0.0f, nullptr, nullptr, 0};
    int64_t wide;
    if (mul_overflows(heads, c.d, &wide)) return ATTNW_ERR_SHAPE;
    if ((e = check_call(&c, &rule, tokens, heads, wide)) != ATTNW_OK) return e;
    if (c.batch == 0 || tokens == 0 || heads == 0) return 0;
    if ((e = check_call_support(&c, 1, &rule, tokens, heads, wide)) != ATTNW_OK || (e = check_block(cache)) != ATTNW_OK) return e;
    attnw::PagedArgs a{};
    a.dt = static_cast<DType>(c.dtype);
    a.cache = view(&c, 1);
    a.tokens = tokens;
    a.heads = heads;
    return attnw::byte_workspace(a);
}

int attnw_byte_paged_attention(const attnw_byte_cache* cache, const attnw_rule* rule, const void* Q, void* O, float* lse, const int32_t* starts, int64_t tokens,
                           int64_t heads, int64_t q_stride, void* workspace, int64_t workspace_bytes, void* stream)
{
    if (!cache || !rule) return ATTNW_ERR_NULL;
    int e = check_sizes(cache);
    if (e != ATTNW_OK) return e;
    const attnw_cache& c = cache->cache;
    if ((e = check_call(&c, rule, tokens, heads, q_stride)) != ATTNW_OK) return e;
    if (workspace_bytes < 0) return ATTNW_ERR_SHAPE;
    if (c.batch == 0 || tokens == 0 || heads == 0) return ATTNW_OK;
    if ((e = check_pointers(cache)) != ATTNW_OK) return e;
    if (!Q || !O || !starts) return ATTNW_ERR_NULL;
    if ((e = check_call_support(&c, 1, rule, tokens, heads, q_stride)) != ATTNW_OK || (e = check_block(cache)) != ATTNW_OK) return e;
    attnw::PagedArgs a{};
    a.dt = static_cast<DType>(c.dtype);
    a.cache = view(&c, 1);
    a.rule = view(rule);
    a.Q = Q;
    a.O = O;
    a.lse = lse;
    a.workspace = static_cast<float*>(workspace);
    a.starts = starts;
    a.tokens = tokens;
    a.heads = heads;
    a.q_stride = q_stride;
    const ScalesView s = scales(cache);
    const int64_t need = attnw::byte_workspace(a);
    if (need > 0 && !workspace) return ATTNW_ERR_NULL;
    if (workspace_bytes < need) return ATTNW_ERR_WORKSPACE;
    if (!cache_aligned(&c) || !aligned(Q, 16) || !aligned(O, 16) || !aligned(lse, 4) || !aligned(starts, 4) || !aligned(workspace, 16) || !aligned(rule->slopes, 4) ||
        !aligned(rule->prefix, 4))
        return ATTNW_ERR_ALIGN;
    const int64_t size = size_of(c.dtype), all = cache_bytes(&c, 1), of_scales = scale_bytes(cache);
    const Range written[] = {{O, tokens * heads * c.d * size}, {lse, tokens * heads * 4}, {workspace, need}};
    const Range read[] = {{Q, extent(tokens, q_stride, heads * c.d, size)}, {c.K, all}, {c.V, all}, {cache->K_scales, of_scales}, {cache->V_scales, of_scales},
                          {c.table, c.batch * c.max_pages * 4}, {c.lengths, c.batch * 4}, {starts, (c.batch + 1) * 4}, {rule->slopes, heads * 4},
                          {rule->prefix, c.batch * 4}};
    if (any_overlap(written, read)) return ATTNW_ERR_ALIAS;
    return status(attnw::launch_byte_attention(a, s, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
