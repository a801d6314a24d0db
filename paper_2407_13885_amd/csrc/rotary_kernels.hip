// Rotary positions, and queries, keys and values of new tokens on their way to attention over a paged cache.
//
// The first `rot` columns of a head are pairs (a, b) -- columns (j, j + rot / 2), or (2 j, 2 j + 1) -- that turn by an angle of their token:
//     a' = a cos - b sin,   b' = b cos + a sin
// (the gradient is the same map transposed: the angle's sign changes).  cos and sin come from a table that is made once, in 64 bits: a position
// of 10^5 times a frequency of 1 has lost its last 7 bits as an fp32 product.
//
// What bounds it: memory, 2 bytes moved for every byte of the rows; a row of the table serves all heads of a token from the caches.  One launch
// turns the queries, turns the keys and lays keys and values into their pages.
#include "paged_common.h"

namespace attnw {
namespace {

template <typename T, int V> struct alignas(sizeof(T) * V) Chunk { T x[V]; };

template <typename T> __device__ __forceinline__ float wide(T x);
template <> __device__ __forceinline__ float wide<float>(float x) { return x; }
template <> __device__ __forceinline__ float wide<uint16_t>(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
template <typename T> __device__ __forceinline__ T narrow(float x);
template <> __device__ __forceinline__ float narrow<float>(float x) { return x; }
template <> __device__ __forceinline__ uint16_t narrow<uint16_t>(float x) { return (uint16_t)pack_bf16x2(x, 0.0f); }

struct Units {
    int32_t per_head, pairs;                      // units of a head; those of them that turn
    int32_t per_token, heads, kv_heads;
    int32_t block_tokens;
    FastDiv by_token, by_head, by_value_head;
};

// A unit: V columns and their V partners (halves), V neighbouring columns (interleaved), or V columns behind the turned ones, which are copied.
// CACHE: with keys and values; heads 0 .. heads - 1 are queries, then kv_heads of keys, then kv_heads of values (which have the units of a
// head that does not turn).
// With caches a thread loads all it needs for some units before it stores any (chunks of 9923 tokens, 48 heads of 128 80 -> 64 us).
template <typename T, int V, bool INTERLEAVED, bool CACHE>
__global__ __launch_bounds__(256)
void rotary_kernel(const T* Q, const T* K, const T* Vn, T* R, T* Kc, T* Vc, const float* __restrict__ angles, const int32_t* __restrict__ positions,
                   const int32_t* __restrict__ starts, int32_t tokens, int32_t d, int32_t rot, int64_t rows, int64_t q_stride, int64_t kv_stride,
                   int64_t r_stride, float sign, CacheView cache, Units u)
{
    typedef Chunk<T, V> C;
    constexpr bool TWO = !INTERLEAVED || V == 1;               // a unit's partners lie elsewhere
    constexpr int P = TWO ? V : V / 2;                         // pairs of a unit
    constexpr int AT_ONCE = !CACHE ? 1 : TWO && V > 1 ? 2 : 3;
    const int lane = threadIdx.x & 63;
    const int32_t turned_heads = u.heads + (CACHE ? u.kv_heads : 0);
    for (int64_t t0 = (int64_t)blockIdx.x * u.block_tokens; t0 < tokens; t0 += (int64_t)gridDim.x * u.block_tokens) {
        int b0 = 0;
        if constexpr (CACHE) {                    // the sequence of token t0: so many of the ends are not past it
            for (int i = 0; i < cache.batch; i += 64) {
                const bool ended = i + lane < cache.batch && starts[i + lane + 1] <= t0;
                b0 += __builtin_popcountll(__builtin_amdgcn_ballot_w64(ended));
            }
        }
        struct Token {
            int64_t position, place;              // place: of its rows in K and V, in elements (-1: none)
        };
        const auto token_at = [&](int64_t t) __attribute__((always_inline)) {
            Token k{positions ? positions[t] : -1, -1};
            if constexpr (CACHE) {
                int b = b0;
                while (b < cache.batch && starts[b + 1] <= t) ++b;
                if (b < cache.batch) {
                    const Sequence s = sequence_at(cache, starts, tokens, b);
                    const int32_t slot = (int32_t)(s.length - s.tokens + (t - s.first));
                    if (slot >= 0 && t >= s.first) {
                        const uint32_t p = quotient((uint32_t)slot, cache.page);
                        const int32_t id = cache.table[(int64_t)b * cache.max_pages + p];
                        if ((uint32_t)id < (uint32_t)cache.pages)
                            k.place = ((int64_t)id * cache.kv_heads * cache.page.d + (slot - (int32_t)(p * cache.page.d))) * d;
                        if (!positions) k.position = slot;
                    }
                }
            }
            return k;
        };
        const Token only = token_at(t0);          // (of one that a workgroup has alone)
        const int32_t mine = (int32_t)min((int64_t)u.block_tokens, tokens - t0) * u.per_token;
        for (int32_t i0 = threadIdx.x + blockIdx.y * 256; i0 < mine; i0 += AT_ONCE * 256 * gridDim.y) {
            T* dst[AT_ONCE];
            int ia[AT_ONCE], ib[AT_ONCE];         // ib < 0: copied; ia < 0: nothing to do
            float lost[AT_ONCE];
            C va[AT_ONCE], vb[AT_ONCE];
            Chunk<float, P> co[AT_ONCE], si[AT_ONCE];
#pragma unroll
            for (int n = 0; n < AT_ONCE; ++n) {
                const int32_t i = i0 + n * 256 * gridDim.y;
                ia[n] = -1;
                if (i >= mine) continue;
                const int32_t in_block = u.block_tokens == 1 ? 0 : (int32_t)quotient(i, u.by_token), unit = i - in_block * u.per_token;
                const int64_t t = t0 + in_block;
                const Token tok = in_block == 0 ? only : token_at(t);
                const bool value = CACHE && unit >= turned_heads * u.per_head;
                const int32_t k = value ? unit - turned_heads * u.per_head : unit;
                const int32_t head = value ? (int32_t)quotient(k, u.by_value_head) : (int32_t)quotient(k, u.by_head);
                const int32_t x = k - head * (value ? (int32_t)u.by_value_head.d : u.per_head);
                const T* src;
                if (!CACHE || (!value && head < u.heads)) {
                    src = Q + t * q_stride + (int64_t)head * d;
                    dst[n] = R + t * r_stride + (int64_t)head * d;
                } else {
                    if (tok.place < 0) continue;  // no such slot: nothing is cached
                    const int32_t h = value ? head : head - u.heads;
                    src = (value ? Vn : K) + t * kv_stride + (int64_t)h * d;
                    dst[n] = (value ? Vc : Kc) + tok.place + (int64_t)h * cache.page.d * d;
                }
                const bool turns = !value && x < u.pairs;
                ia[n] = value ? x * V : !turns ? rot + (x - u.pairs) * V : INTERLEAVED && V == 1 ? 2 * x : x * V;
                ib[n] = !turns ? -1 : !TWO ? ia[n] : INTERLEAVED ? 2 * x + 1 : x * V + rot / 2;
                va[n] = *reinterpret_cast<const C*>(src + ia[n]);
                if (turns) {
                    if constexpr (TWO) vb[n] = *reinterpret_cast<const C*>(src + ib[n]);
                    const bool known = tok.position >= 0 && tok.position < rows;
                    const float* row = angles + (known ? tok.position : 0) * (int64_t)rot + x * P;
                    co[n] = *reinterpret_cast<const Chunk<float, P>*>(row);
                    si[n] = *reinterpret_cast<const Chunk<float, P>*>(row + rot / 2);
                    lost[n] = known ? 0.0f : __builtin_nanf("");
                }
            }
#pragma unroll
            for (int n = 0; n < AT_ONCE; ++n) {
                if (ia[n] < 0) continue;
                if (ib[n] >= 0) {
#pragma unroll
                    for (int e = 0; e < P; ++e) {
                        T& x = TWO ? va[n].x[e] : va[n].x[2 * e % V];
                        T& y = TWO ? vb[n].x[e] : va[n].x[(2 * e + 1) % V];
                        const float a = wide(x), b = wide(y), c = co[n].x[e] + lost[n], s = sign * si[n].x[e];
                        x = narrow<T>(a * c - b * s);
                        y = narrow<T>(b * c + a * s);
                    }
                    if constexpr (TWO) *reinterpret_cast<C*>(dst[n] + ib[n]) = vb[n];
                }
                *reinterpret_cast<C*>(dst[n] + ia[n]) = va[n];
            }
        }
    }
}

template <typename T, int V, bool INTERLEAVED>
hipError_t launch(const RotaryArgs& a, hipStream_t stream)
{
    const bool with_cache = a.K != nullptr;
    Units u;
    u.heads = (int32_t)a.heads;
    u.kv_heads = with_cache ? a.cache.kv_heads : 0;
    u.pairs = (int32_t)(INTERLEAVED && V > 1 ? a.rot / V : a.rot / 2 / V);
    u.per_head = u.pairs + (int32_t)((a.d - a.rot) / V);
    u.per_token = (u.heads + u.kv_heads) * u.per_head + u.kv_heads * (int32_t)(a.d / V);
    u.block_tokens = u.per_token >= 256 ? 1 : 256 / u.per_token;
    u.by_token = fast_div(u.per_token);
    u.by_head = fast_div(u.per_head);
    u.by_value_head = fast_div((uint32_t)(a.d / V));
    const int64_t all = (a.tokens + u.block_tokens - 1) / u.block_tokens;
    const uint32_t blocks = (uint32_t)(all < 1 << 20 ? all : 1 << 20);   // (a launch has less than 2^32 threads)
    // few tokens: the units of one over several workgroups
    uint32_t across = 1;
    while (blocks * across < 512 && across * 256 < (uint32_t)u.per_token) ++across;
    const float sign = a.inverse ? -1.0f : 1.0f;
    auto go = [&](auto kernel) {
        kernel<<<dim3(blocks, across), 256, 0, stream>>>(static_cast<const T*>(a.Q), static_cast<const T*>(a.K), static_cast<const T*>(a.V), static_cast<T*>(a.R),
                                                       static_cast<T*>(a.Kc), static_cast<T*>(a.Vc), a.angles, a.positions, a.starts, (int32_t)a.tokens,
                                                       (int32_t)a.d, (int32_t)a.rot, a.rows, a.q_stride, a.kv_stride, a.r_stride, sign, a.cache, u);
        return hipGetLastError();
    };
    if (with_cache) return go(rotary_kernel<T, V, INTERLEAVED, true>);
    return go(rotary_kernel<T, V, INTERLEAVED, false>);
}

template <typename T, int V>
hipError_t launch_typed(const RotaryArgs& a, hipStream_t stream)
{
    // 16 bytes at a time where rows, halves and the rest are whole chunks of them, else element by element
    const bool chunks = a.d % V == 0 && a.q_stride % V == 0 && a.r_stride % V == 0 && (!a.K || a.kv_stride % V == 0) &&
                        (a.interleaved ? a.rot % V == 0 : a.rot % (2 * V) == 0);
    if (a.interleaved) return chunks ? launch<T, V, true>(a, stream) : launch<T, 1, true>(a, stream);
    return chunks ? launch<T, V, false>(a, stream) : launch<T, 1, false>(a, stream);
}

// table[p][j], table[p][rot / 2 + j] = gain cos, gain sin of p f_j.  f_j = base^(-2 j / rot), slowed down for contexts beyond `original` tokens: a
// column that turns up to `low` times in them by `factor`, from `high` times on not at all, in between by the mean of the two that lies as
// far along.  The angle is reduced in 64 bits, in half turns.
__global__ __launch_bounds__(256)
void rotary_table_kernel(float* table, int64_t positions, int32_t half, double step, double factor, double low, double high, double original, double gain)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < positions * half; i += (int64_t)gridDim.x * 256) {
        const int64_t p = i / half;
        const int32_t j = (int32_t)(i - p * half);
        const double f = exp2(-step * j);         // radians a token
        const double turns = original * f * 0.15915494309189535;
        const double keep = turns >= high ? 1.0 : turns <= low ? 0.0 : (turns - low) / (high - low);
        const double half_turns = (double)p * (f * (keep + (1.0 - keep) / factor)) * 0.3183098861837907;
        double s, c;
        sincospi(half_turns, &s, &c);
        table[p * 2 * half + j] = (float)(gain * c);
        table[p * 2 * half + half + j] = (float)(gain * s);
    }
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, hipStream_t stream)
{
    return a.dt == DType::F32 ? launch_typed<float, 4>(a, stream) : launch_typed<uint16_t, 8>(a, stream);
}

hipError_t launch_rotary_table(float* table, int64_t positions, int64_t rot, double base, double factor, double low, double high, double original,
                               double gain, hipStream_t stream)
{
    const int64_t count = positions * (rot / 2);
    const int64_t blocks = (count + 255) / 256;
    rotary_table_kernel<<<dim3((uint32_t)(blocks < 1 << 16 ? blocks : 1 << 16)), 256, 0, stream>>>(table, positions, (int32_t)(rot / 2), log2(base) * 2.0 / (double)rot,
                                                                                   factor, low, high, original, gain);
    return hipGetLastError();
}

}  // namespace attnw
