// Shared by the kernels that turn columns by positions: elements, angles of a table, and positions on several axes.
#pragma once

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

// The angle of position p in half turns, in 64 bits: p radians times 2^-exponent, slowed down by `factor` for contexts beyond `original` tokens (a column that turns up to
// `low` times in them wholly, from `high` times on not at all, in between by the mean of the two that lies as far along).
__device__ __forceinline__ double rotary_half_turns(int64_t p, double exponent, double factor, double low, double high, double original)
{
    const double f = exp2(-exponent);             // radians a token
    const double turns = original * f * 0.15915494309189535;
    const double keep = turns >= high ? 1.0 : turns <= low ? 0.0 : (turns - low) / (high - low);
    return (double)p * (f * (keep + (1.0 - keep) / factor)) * 0.3183098861837907;
}

// Which axis each pair of columns turns by (2 bits a pair, 16 pairs a word), and where a token stands on them: positions [axes][tokens].
struct AxesView {
    const int32_t* positions;
    int64_t tokens;
    int32_t count;
    uint32_t of[8];
};
inline AxesView axes_view(const AxesMap& map, const int32_t* positions, int64_t tokens)
{
    AxesView v{positions, tokens, map.count, {}};
    for (int j = 0; j < 128; ++j) v.of[j / 16] |= (uint32_t)map.axis[j] << 2 * (j % 16);
    return v;
}

// cos and sin of the P pairs from pair j0 on (P divides 16 and j0), of a token that stands at position(axis): NaN where the table has no such row.  One axis for all of
// them is the rule where axes have whole ranges of pairs; where they are mixed every axis that occurs is read and its pairs taken.
template <int P, typename Position>
__device__ __forceinline__ void load_angles(const float* __restrict__ angles, int32_t rot, int64_t rows, int32_t j0, int32_t axes, const uint32_t* of, Position&& position,
                                            Chunk<float, P>& co, Chunk<float, P>& si)
{
    const auto row_of = [&](int axis, Chunk<float, P>& c, Chunk<float, P>& s) __attribute__((always_inline)) {
        const int64_t p = position(axis);
        const bool known = p >= 0 && p < rows;
        const float* row = angles + (known ? p : 0) * (int64_t)rot + j0;
        c = *reinterpret_cast<const Chunk<float, P>*>(row);
        s = *reinterpret_cast<const Chunk<float, P>*>(row + rot / 2);
        if (!known)
#pragma unroll
            for (int e = 0; e < P; ++e) c.x[e] = s.x[e] = __builtin_nanf("");
    };
    if (axes == 1) return row_of(0, co, si);
    constexpr uint32_t ALL = P == 16 ? ~0u : (1u << 2 * P) - 1;
    const uint32_t bits = of[j0 >> 4] >> 2 * (j0 & 15) & ALL, first = bits & 3;
    row_of((int)first, co, si);
    if (bits == (first * 0x55555555u & ALL)) return;
    for (int axis = 0; axis < axes; ++axis) {
        const uint32_t other = bits ^ ((uint32_t)axis * 0x55555555u & ALL);    // (0 where a pair is this axis')
        if (axis == (int)first || ((other | other >> 1) & 0x55555555u & ALL) == (0x55555555u & ALL)) continue;
        Chunk<float, P> c, s;
        row_of(axis, c, s);
#pragma unroll
        for (int e = 0; e < P; ++e) {
            const bool mine = (other >> 2 * e & 3) == 0;
            co.x[e] = mine ? c.x[e] : co.x[e];
            si.x[e] = mine ? s.x[e] : si.x[e];
        }
    }
}

// cos and sin of pair j of a token that stands at position(axis).
template <typename Position>
__device__ __forceinline__ f32x2 angle_of(const float* __restrict__ angles, int32_t rot, int64_t rows, int32_t axes, const uint32_t* of, int32_t j, Position&& position)
{
    const int64_t p = position(axes == 1 ? 0 : (int)(of[j >> 4] >> 2 * (j & 15) & 3));
    const bool known = p >= 0 && p < rows;
    const float* const row = angles + (known ? p : 0) * (int64_t)rot + j;
    const float c = row[0], s = row[rot / 2];
    return known ? f32x2{c, s} : f32x2{__builtin_nanf(""), __builtin_nanf("")};
}

// The angles of whole tokens, side by side in LDS: cos and sin of the pairs as their axes have them.  (All heads of a token use them; where axes take pairs in turns,
// every unit would read a row for each.)
template <typename Position>
__device__ __forceinline__ void stage_angles(float* staged, const float* __restrict__ angles, int32_t rot, const FastDiv& by_half, int64_t rows, int32_t axes, const uint32_t* of,
                                             int32_t tokens, int64_t t0, Position&& position, int32_t thread, int32_t threads)
{
    const int32_t half = rot / 2;
    for (int32_t i = thread; i < tokens * half; i += threads) {
        const int32_t t = (int32_t)quotient(i, by_half), j = i - t * half;
        const f32x2 cs = angle_of(angles, rot, rows, axes, of, j, [&](int axis) __attribute__((always_inline)) { return position(t0 + t, axis); });
        staged[t * rot + j] = cs[0];
        staged[t * rot + half + j] = cs[1];
    }
}

// How the rows of a token fall into units: V columns and their V partners (halves), V neighbouring columns (pairs), or V columns behind the turned ones.
struct TurnUnits {
    int32_t per_head, pairs;                      // units of a head; those of them that turn
    int32_t per_token, block_tokens;
    FastDiv by_token, by_head, by_half;           // by_half: pairs of a token's angles
};
// (a block of threads takes `at_once` units a thread at a time, of tokens with at most so many angles)
template <int V, bool INTERLEAVED> inline TurnUnits turn_units(int64_t heads, int64_t d, int64_t rot, int at_once, int angles)
{
    TurnUnits u;
    u.pairs = (int32_t)(INTERLEAVED && V > 1 ? rot / V : rot / 2 / V);
    u.per_head = u.pairs + (int32_t)((d - rot) / V);
    u.per_token = (int32_t)heads * u.per_head;
    u.block_tokens = u.per_token >= 256 * at_once ? 1 : 256 * at_once / u.per_token;
    if (u.block_tokens * rot > angles) u.block_tokens = (int32_t)(angles / rot);
    u.by_half = fast_div((uint32_t)(rot > 0 ? rot / 2 : 1));
    u.by_token = fast_div(u.per_token);
    u.by_head = fast_div(u.per_head);
    return u;
}
// Blocks of 256 threads over the tokens, and across the units of one where there are few tokens.
inline dim3 turn_grid(const TurnUnits& u, int64_t tokens)
{
    const int64_t all = (tokens + u.block_tokens - 1) / u.block_tokens;
    const uint32_t blocks = (uint32_t)(all < 1 << 20 ? all : 1 << 20);   // (a launch has less than 2^32 threads)
    uint32_t across = 1;
    while (blocks * across < 512 && across * 256 < (uint32_t)u.per_token) ++across;
    return dim3(blocks, across);
}
// Whether units of V elements will do: rows, strides, halves and the rest are whole ones of them.  (Callers begin at 16 bytes and halve V until they are.)
inline bool turns_by_chunks(int V, int64_t d, int64_t rot, int64_t x_stride, int64_t y_stride, bool interleaved)
{
    return d % V == 0 && x_stride % V == 0 && y_stride % V == 0 && (interleaved ? rot % V == 0 : rot % (2 * V) == 0);
}

// Where the columns of unit x of a head lie: `a`, and `b` those of the partners (`a` again where they are among the same columns); -1: copied.
struct UnitColumns { int32_t a, b; };
template <int V, bool INTERLEAVED> __device__ __forceinline__ UnitColumns unit_columns(const TurnUnits& u, int32_t x, int32_t rot)
{
    constexpr bool TWO = !INTERLEAVED || V == 1;
    if (x >= u.pairs) return {rot + (x - u.pairs) * V, -1};
    const int32_t a = INTERLEAVED && V == 1 ? 2 * x : x * V;
    return {a, !TWO ? a : INTERLEAVED ? 2 * x + 1 : x * V + rot / 2};
}

// A unit turned.
template <bool TWO, typename T, int V, int P>
__device__ __forceinline__ void turn_unit(Chunk<T, V>& va, Chunk<T, V>& vb, const Chunk<float, P>& co, const Chunk<float, P>& si, float sign)
{
#pragma unroll
    for (int e = 0; e < P; ++e) {
        T& p = TWO ? va.x[e] : va.x[2 * e % V];
        T& q = TWO ? vb.x[e] : va.x[(2 * e + 1) % V];
        const float a = wide(p), b = wide(q), c = co.x[e], s = sign * si.x[e];
        p = narrow<T>(a * c - b * s);
        q = narrow<T>(b * c + a * s);
    }
}

// Tokens from block `block` of `blocks` on: rows of X turned (sign -1: back) into rows of Y.  position(t, axis).
template <typename T, int V, bool INTERLEAVED, typename Position>
__device__ __forceinline__ void turn_rows(const T* X, T* Y, const float* __restrict__ angles, int32_t axes, const uint32_t* of, Position&& position, int32_t tokens, int32_t d,
                                          int32_t rot, int64_t rows, int64_t x_stride, int64_t y_stride, float sign, const TurnUnits& u, uint32_t block, uint32_t blocks,
                                          uint32_t part, uint32_t parts)
{
    typedef Chunk<T, V> C;
    constexpr bool TWO = !INTERLEAVED || V == 1;
    constexpr int P = TWO ? V : V / 2;                         // pairs of a unit
    for (int64_t t0 = (int64_t)block * u.block_tokens; t0 < tokens; t0 += (int64_t)blocks * u.block_tokens) {
        const int32_t mine = (int32_t)min((int64_t)u.block_tokens, tokens - t0) * u.per_token;
        for (int32_t i = threadIdx.x + part * 256; i < mine; i += 256 * parts) {
            const int32_t in_block = u.block_tokens == 1 ? 0 : (int32_t)quotient(i, u.by_token), unit = i - in_block * u.per_token;
            const int32_t head = (int32_t)quotient(unit, u.by_head), x = unit - head * u.per_head;
            const int64_t t = t0 + in_block;
            const T* const src = X + t * x_stride + (int64_t)head * d;
            T* const dst = Y + t * y_stride + (int64_t)head * d;
            const UnitColumns at = unit_columns<V, INTERLEAVED>(u, x, rot);
            C va = *reinterpret_cast<const C*>(src + at.a), vb = va;
            if (at.b >= 0) {
                if constexpr (TWO) vb = *reinterpret_cast<const C*>(src + at.b);
                Chunk<float, P> co, si;
                load_angles<P>(angles, rot, rows, x * P, axes, of, [&](int axis) __attribute__((always_inline)) { return position(t, axis); }, co, si);
                turn_unit<TWO>(va, vb, co, si, sign);
                if constexpr (TWO) *reinterpret_cast<C*>(dst + at.b) = vb;
            }
            *reinterpret_cast<C*>(dst + at.a) = va;
        }
    }
}

// The same with the angles of the tokens in LDS (u made for so many).  AT_ONCE: units that a thread loads before it stores any.
template <typename T, int V, bool INTERLEAVED, int AT_ONCE, typename Position>
__device__ __forceinline__ void turn_rows_staged(const T* X, T* Y, const float* __restrict__ angles, int32_t axes, const uint32_t* of, float* staged, Position&& position,
                                          int32_t tokens, int32_t d, int32_t rot, int64_t rows, int64_t x_stride, int64_t y_stride, float sign, const TurnUnits& u,
                                          uint32_t block, uint32_t blocks, uint32_t part, uint32_t parts)
{
    typedef Chunk<T, V> C;
    constexpr bool TWO = !INTERLEAVED || V == 1;
    constexpr int P = TWO ? V : V / 2;                         // pairs of a unit
    for (int64_t t0 = (int64_t)block * u.block_tokens; t0 < tokens; t0 += (int64_t)blocks * u.block_tokens) {
        const int32_t here = (int32_t)min((int64_t)u.block_tokens, tokens - t0), mine = here * u.per_token;
        C va[AT_ONCE], vb[AT_ONCE];
        UnitColumns at[AT_ONCE];
        T* dst[AT_ONCE];
        const float* turns[AT_ONCE];
        const auto load = [&](int32_t i0) __attribute__((always_inline)) {
#pragma unroll
            for (int n = 0; n < AT_ONCE; ++n) {
                const int32_t i = i0 + n * 256 * (int32_t)parts;
                if (i >= mine) break;
                const int32_t in_block = u.block_tokens == 1 ? 0 : (int32_t)quotient(i, u.by_token), unit = i - in_block * u.per_token;
                const int32_t head = (int32_t)quotient(unit, u.by_head), x = unit - head * u.per_head;
                const int64_t t = t0 + in_block;
                const T* const src = X + t * x_stride + (int64_t)head * d;
                dst[n] = Y + t * y_stride + (int64_t)head * d;
                at[n] = unit_columns<V, INTERLEAVED>(u, x, rot);
                turns[n] = staged + in_block * rot + x * P;
                va[n] = *reinterpret_cast<const C*>(src + at[n].a);
                if constexpr (TWO)
                    if (at[n].b >= 0) vb[n] = *reinterpret_cast<const C*>(src + at[n].b);
            }
        };
        const int32_t first = threadIdx.x + part * 256;
        load(first);
        stage_angles(staged, angles, rot, u.by_half, rows, axes, of, here, t0, position, threadIdx.x, 256);
        __syncthreads();
        for (int32_t i0 = first; i0 < mine; i0 += 256 * parts * AT_ONCE) {
            if (i0 != first) load(i0);
#pragma unroll
            for (int n = 0; n < AT_ONCE; ++n) {
                if (i0 + n * 256 * (int32_t)parts >= mine) break;
                if (at[n].b >= 0) {
                    turn_unit<TWO>(va[n], vb[n], *reinterpret_cast<const Chunk<float, P>*>(turns[n]), *reinterpret_cast<const Chunk<float, P>*>(turns[n] + rot / 2), sign);
                    if constexpr (TWO) *reinterpret_cast<C*>(dst[n] + at[n].b) = vb[n];
                }
                *reinterpret_cast<C*>(dst[n] + at[n].a) = va[n];
            }
        }
        __syncthreads();      // (the angles have been read)
    }
}

}  // namespace
}  // namespace attnw
