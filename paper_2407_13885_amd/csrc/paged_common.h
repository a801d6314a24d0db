// Shared by the kernels of the paged cache: how a slot is found, what a row of queries sees, how the work of a ragged batch is dealt out.
//
// What comes from device memory (lengths, starts, page ids) cannot be checked before the launch; the kernels bring it into range where they
// read it, so that nothing outside the caller's arrays is touched whatever it holds.
#pragma once

#include "qk_common.h"
#include "launchers.h"

namespace attnw {

// n / d for 0 <= n < 2^31, d >= 1.  With 2^l >= d > 2^(l - 1), m = ceil(2^(31 + l) / d) is at most 2^32 - 1 for d > 1 and m d - 2^(31 + l) < d <= 2^l, so
// that floor(n m / 2^(31 + l)) is exact; d = 1 has m = 0 and n itself added.
struct FastDiv {
    uint32_t d, m, shift, self;
};
inline FastDiv fast_div(uint32_t d)
{
    if (d == 1) return {1, 0, 0, ~0u};
    uint32_t l = 1;
    while (((uint64_t)1 << l) < d) ++l;
    const uint64_t one = (uint64_t)1 << (31 + l);
    return {d, (uint32_t)((one + d - 1) / d), l - 1, 0};
}
__host__ __device__ __forceinline__ uint32_t quotient(uint32_t n, const FastDiv& f)
{
    return ((uint32_t)(((uint64_t)n * f.m) >> 32) >> f.shift) + (n & f.self);
}

// The cache as kernels take it.
struct CacheView {
    const char *K, *V;
    const int32_t *table, *lengths;
    uint32_t page_bytes, head_bytes;              // of a page, of one head's rows in it
    int32_t batch, pages, max_pages, kv_heads, slots, row_bytes;   // slots: a sequence can have
    FastDiv page;
};

// Slots of sequence b in use, new tokens of it and its first row of the call.
struct Sequence {
    int32_t length, tokens, first;
};
__device__ __forceinline__ Sequence sequence_at(const CacheView& c, const int32_t* starts, int32_t all, int b)
{
    Sequence s;
    s.length = max(0, min(c.lengths[b], c.slots));
    s.first = max(0, min(starts[b], all));
    s.tokens = max(0, max(0, min(starts[b + 1], all)) - s.first);   // (the least int would wrap)
    return s;
}

// Bytes from the start of K or V to slot j (in range) of a sequence's head.
__device__ __forceinline__ int64_t slot_offset(const CacheView& c, const int32_t* pages_of, int kv_head, int j)
{
    const uint32_t p = quotient((uint32_t)j, c.page);
    const int32_t id = max(0, min(pages_of[p], c.pages - 1));
    return (int64_t)((uint64_t)(uint32_t)id * c.page_bytes) + (uint32_t)kv_head * c.head_bytes + (uint32_t)(j - (int)(p * c.page.d)) * (uint32_t)c.row_bytes;
}

// Kernels keep on chip where keys are, 8 bytes for 2^grain of them (16 at most, so many that they lie in one page), for so many of these at a time.
constexpr int kPlaces = 1024;
inline int key_grain(const CacheView& c)
{
    const uint32_t page = c.page.d;
    return page % 16 == 0 ? 4 : page % 8 == 0 ? 3 : page % 4 == 0 ? 2 : page % 2 == 0 ? 1 : 0;
}

// What the scores are made of beside the products.
struct RuleView {
    float scale, cap;
    const float* slopes;
    const int32_t* prefix;
    int32_t window;                               // kNoWindow: none
};
constexpr int32_t kNoWindow = 1 << 30;            // (as many slots as a sequence can have)

// What a rule has beside the scale: kernels are built for each.
enum : int { kPlain = 0, kCap = 1, kBias = 2 };
inline int rule_mode(const RuleView& r) { return (r.cap > 0.0f ? kCap : kPlain) | (r.slopes ? kBias : kPlain); }

// Scores as exponents of 2, of some dot products at once: scale (or cap) and log2(e) in them.
// The cap: c tanh(t), t = scale dot / cap, in fp32 (EXACT) by tanhf, else c - 2 c / (2^(2 log2(e) t) + 1), off by 2^-22 c: two transcendental instructions and three
// others.  That is 2^-15 of an exponent at most up to a cap of 128; where caps are larger, t below a quarter goes by its series (the next term is 2^-27 of the first),
// and the error is 2^-20 of the score.  (Not for all: a chunk of 2048 tokens over 14336 slots 640 us, with the series 1122.)  In fp32 the series is for caps where
// scale / cap might no longer be a normal number.
template <bool CAPPED, bool EXACT> struct ScoreMap {
    float c, inner, plain, ratio;                 // plain: scale; ratio: dot -> t; inner: as large() takes it
    bool series;
    __device__ __forceinline__ explicit ScoreMap(const RuleView& r)
    {
        const auto finite = [](float x) __attribute__((always_inline)) { return fmaxf(-3.4e38f, fminf(x, 3.4e38f)); };
        plain = r.scale * kLog2e;
        c = CAPPED ? finite(r.cap * kLog2e) : plain;
        ratio = CAPPED ? finite(r.scale / r.cap) : 0.0f;
        inner = EXACT ? ratio : finite(ratio * (2.0f * kLog2e));
        series = r.cap > (EXACT ? 0x1p100f : 128.0f);
    }
    __device__ __forceinline__ float large(float dot) const
    {
        if constexpr (!CAPPED) return dot * c;
        else if constexpr (EXACT) return c * tanhf(dot * inner);
        else return __builtin_fmaf(-2.0f * c, __builtin_amdgcn_rcpf(fast_exp2(dot * inner) + 1.0f), c);
    }
    __device__ __forceinline__ float any(float dot) const
    {
        const float t = dot * ratio, u = t * t;
        const float p = __builtin_fmaf(u, __builtin_fmaf(u, __builtin_fmaf(u, 62.0f / 2835.0f, -17.0f / 315.0f), 2.0f / 15.0f), -1.0f / 3.0f);
        const float x = dot * plain;
        return fabsf(t) < 0.25f ? __builtin_fmaf(x * u, p, x) : large(dot);
    }
    template <int N> __device__ __forceinline__ void operator()(float (&x)[N]) const
    {
        if constexpr (CAPPED) {
            if (apart_uniform(series) != 0) {     // (where it stands: not two of every loop around it)
#pragma unroll
                for (int i = 0; i < N; ++i) x[i] = any(x[i]);
                return;
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = large(x[i]);
    }
};

// Of 16 bytes of elements T: whether one is infinite or NaN; those of a kind as 1 and the others as 0; all of them as 0.  (An exponent of ones carries into
// the sign's place when one is added at its end.)
template <typename T> __device__ __forceinline__ uint32_t lost_signs(uint32_t w)
{
    if constexpr (sizeof(T) == 4) return ((w & 0x7f800000u) + 0x00800000u) & 0x80000000u;
    else return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
}
template <typename T> __device__ __forceinline__ uint32_t any_lost(const u32x4& v)
{
    return lost_signs<T>(v[0]) | lost_signs<T>(v[1]) | lost_signs<T>(v[2]) | lost_signs<T>(v[3]);
}
enum { kAny, kUp, kDown };                        // of those that are lost: all; +infinity and NaN; -infinity and NaN
template <typename T, int KIND> __device__ __forceinline__ u32x4 lost_as_one(const u32x4& v)
{
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = v[i], nan = sizeof(T) == 4 ? (w & 0x7fffffffu) + 0x007fffffu : (w & 0x7fff7fffu) + 0x007f007fu;   // (in the signs' places)
        const uint32_t t = lost_signs<T>(w) & (KIND == kAny ? ~0u : KIND == kUp ? ~w | nan : w | nan);
        r[i] = (t >> 1) - (t >> 8);               // 0x40.. - 0x00800..
    }
    return r;
}
template <typename T> __device__ __forceinline__ u32x4 without_lost(const u32x4& v)
{
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t t = lost_signs<T>(v[i]);
        r[i] = v[i] & ~(sizeof(T) == 4 ? (uint32_t)((int32_t)t >> 31) : (t << 1) - (t >> 15));
    }
    return r;
}

// Rows that are shorter than their place on chip.  Zeros of Q behind their end would make NaN of a product with infinity, so that nothing is multiplied by 0: a key
// has its first chunks of 16 bytes there once more (d = 4 in fp32: its only one, three times), and the query shares their columns out between the two places (the
// four), which adds up to the same.
// Where the chunk at byte `at` of a place comes from, rows being rb bytes, which are half a place at least but for that one:
__device__ __forceinline__ int chunk_in_row(int at, int rb) { return at < rb ? at : min(at - rb, rb - 16); }
// Numbers times 2^-halvings: exact, as those below 2^-118, where it might not be, are whole in their first place and 0 in the others (an infinite key makes NaN
// of those).  Infinities and NaN as they are.
template <typename T> __device__ __forceinline__ uint32_t shared_out(uint32_t w, int halvings, bool first)
{
    // (flags in the signs' places: an exponent field of 9 or more)
    const uint32_t can = sizeof(T) == 4 ? ((w & 0x7f800000u) + 0x7b800000u) & 0x80000000u : ((w & 0x7f807f80u) + 0x7b807b80u) & 0x80008000u;
    const uint32_t less = w - ((can & ~lost_signs<T>(w)) >> 8) * halvings;
    return first ? less : less & (sizeof(T) == 4 ? (uint32_t)((int32_t)can >> 31) : (can << 1) - (can >> 15));
}
// The chunk of a query that meets chunk `ch` of a key's place of `all` chunks.
template <typename T> __device__ __forceinline__ u32x4 query_chunk(const char* q, int ch, int all, int rb)
{
    const int from = chunk_in_row(ch * 16, rb);
    const int halvings = rb == 16 ? all / 2 : from + rb < all * 16 ? 1 : 0;   // (rb = 16: all = 4)
    u32x4 v = *reinterpret_cast<const u32x4*>(q + from);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = shared_out<T>(v[i], halvings, ch * 16 < rb);
    return v;
}

// Below 0 where a token at slot `query` does not see slot j, `past` the first that nobody sees: in numbers, as conditions the compiler makes a branch of each.
struct Sight {
    int32_t low, high, prefix;
    __device__ __forceinline__ Sight(int32_t query, const RuleView& r, int32_t prefix_, int32_t past)
        : low(query - r.window + 1), high(min(query, past - 1)), prefix(min(prefix_, past))
    {
    }
    __device__ __forceinline__ int32_t hidden(int32_t j) const { return ((j - low) | (high - j)) & ~(j - prefix); }
};

// A value that all lanes of a wave have, as one that the compiler knows they have.
__device__ __forceinline__ int32_t uniform(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }

// Numbers of places are counted up to 2^31 - 1 and no further: more there are only where starts are in no order, and then what comes out is any of the rows, but of
// the caller's arrays.
__device__ __forceinline__ int32_t plus(int32_t x, int32_t y) { return __builtin_elementwise_add_sat(x, y); }

// (of the first n lanes)
__device__ __forceinline__ int32_t wave_inclusive_sum(int32_t v, int lane, int n = 64)
{
    for (int off = 1; off < n; off <<= 1) {
        const int32_t o = __shfl_up(v, off, 64);
        if (lane >= off) v = plus(v, o);
    }
    return v;
}

// All places of a batch (a wave's lanes count the sequences), `count(b)` being those of sequence b.
template <typename Count> __device__ __forceinline__ int32_t plan_total(int batch, int lane, Count&& count)
{
    int32_t sum = 0;
    for (int b = lane; b < batch; b += 64) sum = plus(sum, count(b));
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) sum = plus(sum, __shfl_xor(sum, off, 64));
    return uniform(sum);
}
// The sequence that holds place `at` of the total, and the places before it.
template <typename Count> __device__ __forceinline__ void plan_find(int batch, int lane, int32_t at, Count&& count, int32_t& found, int32_t& before)
{
    int32_t base = 0;
    for (int b0 = 0; b0 < batch; b0 += 64) {
        const int32_t end = plus(base, wave_inclusive_sum(b0 + lane < batch ? count(b0 + lane) : 0, lane));
        const uint64_t past = __builtin_amdgcn_ballot_w64(end > at);
        if (past) {
            const int first = __builtin_ctzll(past);
            found = b0 + first;
            before = first > 0 ? __builtin_amdgcn_readlane(end, first - 1) : base;
            return;
        }
        base = __builtin_amdgcn_readlane(end, 63);
    }
    found = batch;
    before = base;
}

// A list of places dealt out: workgroup w has first(w) .. first(w + 1) - 1, `each` of them or one more; all workgroups have some.
struct Deal {
    int32_t each, more, workgroups;               // the first `more` have one more
    __device__ __forceinline__ int32_t first(int32_t w) const { return w * each + min(w, more); }
    __device__ __forceinline__ int32_t owner(int32_t x) const   // whose place x is
    {
        const int32_t those = more * (each + 1);
        return x < those ? (int32_t)((uint32_t)x / (uint32_t)(each + 1)) : more + (int32_t)((uint32_t)(x - those) / (uint32_t)each);
    }
};
__device__ __forceinline__ Deal deal_out(int32_t total, int32_t most)
{
    Deal d;
    d.workgroups = min(total, most);
    d.each = total < most ? 1 : uniform((int32_t)((uint32_t)total / (uint32_t)most));
    d.more = total < most ? 0 : total - d.each * most;
    return d;
}
// Which workgroup a block of the launch is (from d.workgroups on: none): neighbours on one XCD, also where there are fewer than were launched.
__device__ __forceinline__ int32_t dealt_workgroup(const Deal& d)
{
    const uint32_t padded = (d.workgroups + 7) & ~7u;
    return (int32_t)(blockIdx.x >= padded ? blockIdx.x : xcd_contiguous_block_id(blockIdx.x, padded));
}

// Keys that the rows at positions first .. last of a sequence see, as units of 2^log keys: [0, head) and [tail, end).
struct Span {
    int32_t head, tail, end;
    __device__ __forceinline__ int32_t count() const { return head + end - tail; }
    __device__ __forceinline__ int32_t unit(int32_t i) const { return i < head ? i : tail + (i - head); }
};
__device__ __forceinline__ Span visible_span(int32_t log, int32_t first, int32_t last, int32_t length, int32_t prefix, int32_t window)
{
    Span s;
    s.head = (int32_t)((uint32_t)(min(prefix, length) + (1 << log) - 1) >> log);
    s.tail = max(s.head, max(0, first - window + 1) >> log);
    s.end = max(s.tail, (int32_t)((uint32_t)(max(0, last + 1) + (1 << log) - 1) >> log));
    return s;
}

// Launchers (arguments validated).
hipError_t launch_rotary_table(float* table, int64_t positions, int64_t rot, double base, double factor, double low, double high, double original,
                               double gain, hipStream_t stream);
struct RotaryArgs {
    DType dt;
    const void *Q, *K, *V;                        // K, V: null where only Q is turned
    void *R, *Kc, *Vc;
    const float* angles;
    const int32_t *positions, *starts;
    int64_t tokens, heads, d, rot, rows, q_stride, kv_stride, r_stride;
    bool interleaved, inverse;
    CacheView cache;                              // (where K, V are given)
};
hipError_t launch_rotary(const RotaryArgs& a, hipStream_t stream);

struct PagedArgs {
    DType dt;
    CacheView cache;
    RuleView rule;
    const void* Q;
    void* O;
    float *lse, *workspace;
    const int32_t* starts;
    int64_t tokens, heads, q_stride;
};
int64_t paged_workspace(const PagedArgs& a);       // (of a, sizes alone)
hipError_t launch_paged_attention(const PagedArgs& a, hipStream_t stream);
// Blocks of 16 rows, each wave with keys of its own: any call.
int64_t paged_rows_workspace_f32(const PagedArgs& a);
hipError_t launch_paged_rows_f32(const PagedArgs& a, hipStream_t stream);
// Blocks of 128 rows (fp32: 64), which share the keys: any call, for chunks.
bool prefers_paged_tiles(const PagedArgs& a);
int64_t paged_tiles_workspace(const PagedArgs& a);
hipError_t launch_paged_tiles(const PagedArgs& a, hipStream_t stream);
int64_t paged_tiles_workspace_f32(const PagedArgs& a);
hipError_t launch_paged_tiles_f32(const PagedArgs& a, hipStream_t stream);
hipError_t launch_paged_tiles_cap(const PagedArgs& a, hipStream_t stream);
hipError_t launch_paged_tiles_bias(const PagedArgs& a, hipStream_t stream);
hipError_t launch_paged_tiles_both(const PagedArgs& a, hipStream_t stream);

struct SumsArgs {
    DType dt;
    CacheView cache;
    RuleView rule;
    const void* Q;
    const float *lse, *before;
    float* sums;
    const int32_t* starts;
    int64_t tokens, heads, q_stride;
};
hipError_t launch_paged_sums(const SumsArgs& a, hipStream_t stream);

hipError_t launch_evict(const CacheView& from, const CacheView& into, int32_t* into_lengths, const float* sums, float* into_sums, int32_t* kept,
                        int64_t keep, int64_t recent, hipStream_t stream);

}  // namespace attnw
