// New tokens on their way into a paged cache that holds a byte an element: queries turned, keys turned and rounded, values rounded.
//
// The slots of a block share a scale 2^e, e the least with max |x| <= 448 2^e over the block's rows; a block that had rows before keeps at least the e that it had, and
// where that grows its old rows are rounded again.  So a block's rows, old and new, are the work of one group of lanes: they turn the new rows and keep them in registers, find
// the largest element, and store.  No atomics, and nothing that depends on which block comes first.
//
// What bounds it: memory.  Rows of queries are turned as without a cache (rotary_common.h), by other workgroups of the same launch.  Measured: 9045 tokens, 32 heads on 8 of
// 128, bf16, pairs of 64 columns by three axes, 206 MB 55 us = 3.75 TB/s (waves wait 73 % of their life, the vector unit works 42 % of the cycles; halves of all columns 48), fp32
// by halves 62 to 88; eight tokens 6.2 us, a chain of the plan, the page, the rows and the largest.  Keys and values alone take 26, queries alone 38.6.
// A block is the work of one group however long it is: the same tokens on 32 heads, halves, blocks of 16 slots 44.5 us, 128 47.6, 512 60, 1024 98, 4096 350.  A block of
// 128 whose scale grows, a token each of 64 sequences, 9.4 instead of 7.1.
// Workgroups of both in turns took 72, keys' angles by way of LDS 68, a block's older rows on their way early 77 (registers).
#include "rotary_common.h"
#include "byte_cache.h"

namespace attnw {
namespace {

struct AppendArgs {
    const void *Q, *K, *V;
    void* R;
    uint8_t *Kc, *Vc;
    const float* angles;
    const int32_t* starts;
    AxesView axes;
    CacheView cache;
    ScalesView scales;
    TurnUnits queries;
    FastDiv key_units, value_units;               // units of a row of keys, of values
    FastDiv per_block;                            // groups of heads, of keys and of values
    int32_t blocks;                               // that the launch takes at a time
    int64_t rows, q_stride, kv_stride;
    int32_t tokens, heads, d, rot, most_blocks;   // most_blocks: of all sequences, at most
    uint32_t kv_workgroups, q_blocks, q_parts;
};

// (each product rounded: the scale that a block gets is the one that the definition in fp32 gives it)
__device__ __forceinline__ void turn_apart(float& x, float& y, float c, float s)
{
#pragma clang fp contract(off)
    const float a = x * c - y * s, b = y * c + x * s;
    x = a;
    y = b;
}

// Of a row of keys or values a unit is V neighbouring columns (pairs, V > 1: INTERLEAVED) or twice V: those that turn together, or neighbours; in single columns (V = 1) a
// pair of columns, or one that does not turn.
// LANES: so many share a block of a head; HOLD: units of it that a lane keeps (32 elements, 16 of single columns; the others are read again).
template <int V, bool INTERLEAVED> constexpr int kHold = V == 1 ? 8 : (INTERLEAVED ? 32 : 16) / V;
constexpr int kStaged = 4096;                     // angles in LDS, of the tokens whose queries a workgroup turns
constexpr int kQueriesAtOnce = 4;                 // (the kernel has the registers of few waves: each has more on its way)

// (Neighbouring columns: held to the registers of four waves of a SIMD, 9045 tokens of 48 heads of 128 58.8 -> 54.6 us; halves, which hold more at once, 48 us, so held 59.)
template <typename T, int V, bool INTERLEAVED, int LANES, int WAVES = (INTERLEAVED && V > 1 ? 4 : 1)>
__global__ __launch_bounds__(256, WAVES)
void byte_append_kernel(AppendArgs a)
{
    typedef Chunk<T, V> C;
    constexpr bool TWO = !INTERLEAVED || V == 1;
    constexpr int P = TWO ? V : V / 2, HOLD = kHold<V, INTERLEAVED>, HEADS = LANES < 64 ? 64 / LANES : 1;   // HEADS: that a wave works on at once
    __shared__ uint32_t of[8];
    __shared__ float tops[4];
    __shared__ __align__(32) float staged[kStaged];
    if (threadIdx.x < 8) of[threadIdx.x] = a.axes.of[threadIdx.x];
    __syncthreads();
    const CacheView& cache = a.cache;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);

    if (blockIdx.x >= a.kv_workgroups) {          // ---- queries ----------------------------------------------------------------------------
        const auto position = [&](int64_t t, int axis) __attribute__((always_inline)) {
            if (a.axes.positions) return (int64_t)a.axes.positions[axis * a.axes.tokens + t];
            int low = 0, high = cache.batch;      // the first sequence that ends behind t
            while (low < high) {
                const int mid = (low + high) >> 1;
                if (a.starts[mid + 1] > t) high = mid;
                else low = mid + 1;
            }
            if (low >= cache.batch) return (int64_t)-1;
            const Sequence s = sequence_at(cache, a.starts, a.tokens, low);
            const int64_t slot = s.length - s.tokens + (t - s.first);
            return t >= s.first ? slot : (int64_t)-1;
        };
        const uint32_t w = blockIdx.x - a.kv_workgroups, block = w % a.q_blocks;
        turn_rows_staged<T, V, INTERLEAVED, kQueriesAtOnce>(static_cast<const T*>(a.Q), static_cast<T*>(a.R), a.angles, a.axes.count, of, staged, position, a.tokens, a.d, a.rot, a.rows, a.q_stride,
                                     (int64_t)a.heads * a.d, 1.0f, a.queries, block, a.q_blocks, w / a.q_blocks, a.q_parts);
        return;
    }

    // ---- keys and values -------------------------------------------------------------------------------------------------------------------
    const int32_t size = (int32_t)a.scales.block.d;
    const auto blocks_in = [&](const Sequence& s) __attribute__((always_inline)) {   // that its new tokens lie in
        if (s.tokens == 0 || s.length == 0) return 0;
        return (int32_t)(quotient(s.length - 1, a.scales.block) - quotient(max(0, s.length - s.tokens), a.scales.block)) + 1;
    };
    const auto blocks_of = [&](int b) __attribute__((always_inline)) { return blocks_in(sequence_at(cache, a.starts, a.tokens, b)); };
    // (of up to 64 sequences each lane holds one, read once)
    const bool one_look = cache.batch <= 64;
    Sequence own{0, 0, 0};
    int32_t upto = 0, total;
    if (one_look) {
        if (lane < cache.batch) own = sequence_at(cache, a.starts, a.tokens, lane);
        upto = wave_inclusive_sum(lane < cache.batch ? blocks_in(own) : 0, lane, cache.batch);
        total = __builtin_amdgcn_readlane(upto, cache.batch - 1);
    } else {
        total = plan_total(cache.batch, lane, blocks_of);
    }
    constexpr int AT_ONCE = LANES == 256 ? 1 : 4;              // items of a workgroup
    const int l = LANES == 256 ? (int)threadIdx.x : lane % LANES;
    const uint32_t item = blockIdx.x * AT_ONCE + (AT_ONCE > 1 ? wave : 0), begin = quotient(item, a.per_block);
    const int32_t of_block = (int32_t)(item - begin * a.per_block.d), groups = (int32_t)(a.per_block.d / 2);
    const bool value = of_block >= groups;
    const int32_t head = (value ? of_block - groups : of_block) * HEADS + (HEADS > 1 ? lane / LANES : 0);
    if ((int32_t)begin >= a.blocks) return;
    for (int32_t block = (int32_t)begin; block < total; block = plus(block, a.blocks)) {
        int32_t b, before;
        Sequence s;
        if (one_look) {
            const uint64_t past = __builtin_amdgcn_ballot_w64(lane < cache.batch && upto > block);
            if (past == 0) break;                 // (starts in no order)
            b = __builtin_ctzll(past);
            before = b > 0 ? __builtin_amdgcn_readlane(upto, b - 1) : 0;
            s = Sequence{__builtin_amdgcn_readlane(own.length, b), __builtin_amdgcn_readlane(own.tokens, b), __builtin_amdgcn_readlane(own.first, b)};
        } else {
            plan_find(cache.batch, lane, block, blocks_of, b, before);
            if (b >= cache.batch) break;
            s = sequence_at(cache, a.starts, a.tokens, b);
        }
        const int32_t base = max(0, s.length - s.tokens);
        const int32_t slot0 = (int32_t)(quotient(base, a.scales.block) + (block - before)) * size;   // the block's first
        const int32_t first = max(slot0, base), count = min(slot0 + size, s.length) - first;          // its new ones
        const uint32_t page = quotient(slot0, cache.page);
        const int32_t id = cache.table[(int64_t)b * cache.max_pages + page];
        const int32_t row0 = slot0 - (int32_t)(page * cache.page.d);
        const bool active = head < cache.kv_heads;
        const T* const src = static_cast<const T*>(value ? a.V : a.K) + (int64_t)(active ? head : 0) * a.d;
        const int64_t t0 = (int64_t)s.first + s.tokens - (s.length - first);                           // the token of slot `first`
        const FastDiv by_row = value ? a.value_units : a.key_units;
        const int32_t units = active ? count * (int32_t)by_row.d : 0;

        const auto position = [&](int64_t t, int axis) __attribute__((always_inline)) {
            return a.axes.positions ? (int64_t)a.axes.positions[axis * a.axes.tokens + t] : first + (t - t0);
        };
        struct Unit { C a, b; };
        float x[HOLD][TWO ? 2 : 1][V];
        const int32_t turning = value ? 0 : (TWO ? a.rot / 2 : a.rot) / V;   // units of a row
        struct Columns { int32_t a, b; bool turned; };         // b < 0: none
        const auto columns = [&](int32_t row, int32_t u) __attribute__((always_inline)) {
            const int32_t k = u - row * (int32_t)by_row.d, rest = (value ? 0 : a.rot) + (k - turning) * (TWO && V > 1 ? 2 * V : V);
            Columns c;
            c.turned = k < turning;
            c.a = !c.turned ? rest : INTERLEAVED && V == 1 ? 2 * k : k * V;
            c.b = !TWO ? -1 : c.turned ? (INTERLEAVED ? c.a + 1 : c.a + a.rot / 2) : V > 1 ? rest + V : -1;
            return c;
        };
        const auto load = [&](int32_t u) __attribute__((always_inline)) {
            const int32_t row = (int32_t)quotient(u, by_row);
            const Columns c = columns(row, u);
            const T* const p = src + (t0 + row) * a.kv_stride;
            Unit r;
            r.a = *reinterpret_cast<const C*>(p + c.a);
            r.b = r.a;
            if constexpr (TWO)
                if (c.b >= 0) r.b = *reinterpret_cast<const C*>(p + c.b);
            return r;
        };
        const auto turn = [&](int32_t u, const Unit& r, float (&y)[TWO ? 2 : 1][V]) __attribute__((always_inline)) {
            const int32_t row = (int32_t)quotient(u, by_row);
            const Columns c = columns(row, u);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                y[0][e] = wide(r.a.x[e]);
                if constexpr (TWO) y[TWO ? 1 : 0][e] = c.b < 0 ? 0.0f : wide(r.b.x[e]);
            }
            if (!c.turned) {                      // (quiet, as products are: the largest of a signalling NaN and a number is NaN, and of that and the next the next)
#pragma unroll
                for (int n = 0; n < (TWO ? 2 : 1); ++n)
#pragma unroll
                    for (int e = 0; e < V; ++e) y[n][e] = __builtin_canonicalizef(y[n][e]);
                return;
            }
            const int32_t pair = (u - row * (int32_t)by_row.d) * P;
            Chunk<float, P> co, si;
            load_angles<P>(a.angles, a.rot, a.rows, pair, a.axes.count, of, [&](int axis) __attribute__((always_inline)) { return position(t0 + row, axis); }, co, si);
#pragma unroll
            for (int e = 0; e < P; ++e) turn_apart(TWO ? y[0][e] : y[0][2 * e % V], TWO ? y[TWO ? 1 : 0][e] : y[0][(2 * e + 1) % V], co.x[e], si.x[e]);
        };
        // (fmaxf leaves NaN aside)
        const auto largest = [](float top, const float (&y)[TWO ? 2 : 1][V]) __attribute__((always_inline)) {
#pragma unroll
            for (int n = 0; n < (TWO ? 2 : 1); ++n)
#pragma unroll
                for (int e = 0; e < V; e += 2) top = V == 1 ? fmaxf(top, fabsf(y[n][0])) : max3(top, fabsf(y[n][e]), fabsf(y[n][(e + 1) % V]));
            return top;
        };
        const auto largest_finite = [](float top, const float (&y)[TWO ? 2 : 1][V]) __attribute__((always_inline)) {
#pragma unroll
            for (int n = 0; n < (TWO ? 2 : 1); ++n)
#pragma unroll
                for (int e = 0; e < V; ++e) top = fabsf(y[n][e]) < __builtin_inff() ? fmaxf(top, fabsf(y[n][e])) : top;
            return top;
        };
        const auto store = [&](uint8_t* at, int32_t u, const float (&y)[TWO ? 2 : 1][V], float scale_up) __attribute__((always_inline)) {
            const int32_t row = (int32_t)quotient(u, by_row);
            const Columns c = columns(row, u);
            uint8_t* const to = at + (int64_t)(first - slot0 + row) * a.d;
#pragma unroll
            for (int n = 0; n < (TWO ? 2 : 1); ++n) {
                if (n == 1 && c.b < 0) break;
                uint8_t* const p = to + (n == 0 ? c.a : c.b);
                if constexpr (V == 1) {
                    *p = (uint8_t)pack_e4m3<false>(y[n][0], 0.0f, 0, scale_up);
                } else if constexpr (V == 2) {
                    *reinterpret_cast<uint16_t*>(p) = (uint16_t)pack_e4m3<false>(y[n][0], y[n][1], 0, scale_up);
                } else {
                    uint32_t w[V / 4 > 0 ? V / 4 : 1];
#pragma unroll
                    for (int q = 0; q < V / 4; ++q) w[q] = pack_e4m3(y[n][4 * q], y[n][(4 * q + 1) % V], y[n][(4 * q + 2) % V], y[n][(4 * q + 3) % V], scale_up);
                    if constexpr (V == 8) *reinterpret_cast<u32x2*>(p) = u32x2{w[0], w[V / 4 > 1 ? 1 : 0]};
                    else *reinterpret_cast<uint32_t*>(p) = w[0];
                }
            }
        };

        float top = 0.0f;
        Unit raw[HOLD];                           // (on their way before it is known where they go)
#pragma unroll
        for (int n = 0; n < HOLD; ++n)
            if (l + n * LANES < units) raw[n] = load(l + n * LANES);
        if ((uint32_t)id >= (uint32_t)cache.pages) continue;  // no such page: nothing is cached
        const int64_t place = (int64_t)id * cache.kv_heads + (active ? head : 0);
        uint8_t* const at = (value ? a.Vc : a.Kc) + (place * cache.page.d + row0) * a.d;              // of slot0
        uint8_t* const scale = (value ? a.scales.V : a.scales.K) + place * a.scales.per_page + quotient(row0, a.scales.block);
        const int32_t held = first > slot0 ? (int32_t)*scale : 0;   // (the block had rows before)
        {
#pragma unroll
            for (int n = 0; n < HOLD; ++n)
                if (l + n * LANES < units) {
                    turn(l + n * LANES, raw[n], x[n]);
                    top = largest(top, x[n]);
                }
        }
        for (int32_t u = l + HOLD * LANES; u < units; u += LANES) {
            float y[TWO ? 2 : 1][V];
            turn(u, load(u), y);
            top = largest(top, y);
        }
        const auto of_all = [&](float x) __attribute__((always_inline)) {   // the lanes of the block
#pragma unroll
            for (int off = (LANES < 64 ? LANES : 64) / 2; off > 0; off >>= 1) x = fmaxf(x, __shfl_xor(x, off, 64));
            if constexpr (LANES == 256) {
                if (lane == 0) tops[wave] = x;
                __syncthreads();
                x = fmaxf(max3(tops[0], tops[1], tops[2]), tops[3]);
                __syncthreads();
            }
            return x;
        };
        top = of_all(top);
        // (infinities and NaN come to be NaN and leave the others their scale: where there is one they are looked through once more)
        if (__builtin_amdgcn_ballot_w64(top == __builtin_inff()) != 0) {
            float rest = 0.0f;
            for (int32_t u = l; u < units; u += LANES) {
                float y[TWO ? 2 : 1][V];
                turn(u, load(u), y);
                rest = largest_finite(rest, y);
            }
            rest = of_all(rest);
            top = top == __builtin_inff() ? rest : top;
        }
        if (!active) continue;
        int e = exponent_for(__float_as_uint(top));
        if (first > slot0) {
            const int old = max(1, min(held, 127 + kMostScale)) - 127;   // (below kLeastScale where something else wrote it: scale_of)
            if (e > old) {                        // in units of the new scale
                const float down = scale_of(127 + e - old);
                const auto again = [&](u32x4 w) __attribute__((always_inline)) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(w[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w[i], true);
                        w[i] = pack_e4m3(lo[0], lo[1], hi[0], hi[1], down);
                    }
                    return w;
                };
                u32x4* const older = reinterpret_cast<u32x4*>(at);
#pragma unroll 2
                for (int32_t i = l; i < (first - slot0) * (a.d / 16); i += LANES) older[i] = again(older[i]);
            } else {
                e = old;
            }
        }
        if (l == 0) *scale = (uint8_t)(e + 127);
        const float up = scale_of(e + 127);       // what the elements are in units of
        // (beyond 448 of the greatest scale)
        const auto clamp = [&](float (&y)[TWO ? 2 : 1][V]) __attribute__((always_inline)) {
            if (e < kMostScale) return;
            const float most = 448.0f * up;
#pragma unroll
            for (int n = 0; n < (TWO ? 2 : 1); ++n)
#pragma unroll
                for (int i = 0; i < V; ++i) y[n][i] = fabsf(y[n][i]) < __builtin_inff() ? __builtin_amdgcn_fmed3f(y[n][i], -most, most) : y[n][i];
        };
#pragma unroll
        for (int n = 0; n < HOLD; ++n)
            if (l + n * LANES < units) {
                clamp(x[n]);
                store(at, l + n * LANES, x[n], up);
            }
        for (int32_t u = l + HOLD * LANES; u < units; u += LANES) {
            float y[TWO ? 2 : 1][V];
            turn(u, load(u), y);
            clamp(y);
            store(at, u, y, up);
        }
    }
}

template <typename T, int V, bool INTERLEAVED> hipError_t launch(AppendArgs a, hipStream_t stream)
{
    a.queries = turn_units<V, INTERLEAVED>(a.heads > 0 ? a.heads : 1, a.d, a.rot, kQueriesAtOnce, kStaged);
    const int64_t of_values = a.d / (INTERLEAVED || V == 1 ? V : 2 * V), of_keys = V > 1 ? of_values : a.rot / 2 + (a.d - a.rot);
    a.key_units = fast_div((uint32_t)of_keys);
    a.value_units = fast_div((uint32_t)of_values);
    const dim3 q = turn_grid(a.queries, a.tokens);
    a.q_blocks = q.x;
    a.q_parts = q.y;
    const int64_t units = (int64_t)a.scales.block.d * of_values;   // of a block, at most
    auto go = [&](auto kernel, int lanes) {
        const int64_t groups = lanes < 64 ? (a.cache.kv_heads + 64 / lanes - 1) / (64 / lanes) : a.cache.kv_heads;
        const int64_t at_once = ((int64_t)1 << 20) / (2 * groups);
        a.per_block = fast_div((uint32_t)(2 * groups));
        a.blocks = (int32_t)(a.most_blocks < at_once ? a.most_blocks : at_once);
        const uint32_t items = (uint32_t)(a.blocks * 2 * groups);
        a.kv_workgroups = lanes == 256 ? items : (items + 3) / 4;
        kernel<<<a.kv_workgroups + (a.heads > 0 ? a.q_blocks * a.q_parts : 0), 256, 0, stream>>>(a);
        return hipGetLastError();
    };
    if (units <= 16 * kHold<V, INTERLEAVED>) return go(byte_append_kernel<T, V, INTERLEAVED, 16>, 16);
    if (units <= 64 * kHold<V, INTERLEAVED>) return go(byte_append_kernel<T, V, INTERLEAVED, 64>, 64);
    return go(byte_append_kernel<T, V, INTERLEAVED, 256>, 256);
}

// The widest units that rows, halves and the rest are whole ones of.  (9000 tokens, 32 heads on 8 of 128, bf16, us: pairs, 100 columns turned, four at a time 65, one 158; 98, two at
// a time 88, one 159; halves, 120 columns, four 77, one 143; 98 by one 158.)
template <typename T, int V> hipError_t launch_typed(const RotaryArgs& r, const AppendArgs& a, hipStream_t stream)
{
    if constexpr (V > 1)
        if (!turns_by_chunks(V, a.d, a.rot, a.heads > 0 ? a.q_stride : V, a.kv_stride, r.interleaved)) return launch_typed<T, V / 2>(r, a, stream);
    return r.interleaved ? launch<T, V, true>(a, stream) : launch<T, V, false>(a, stream);
}

}  // namespace

hipError_t launch_byte_append(const RotaryArgs& r, const ScalesView& scales, const AxesMap* map, hipStream_t stream)
{
    AppendArgs a{};
    a.Q = r.Q;
    a.K = r.K;
    a.V = r.V;
    a.R = r.R;
    a.Kc = static_cast<uint8_t*>(r.Kc);
    a.Vc = static_cast<uint8_t*>(r.Vc);
    a.angles = r.angles;
    a.starts = r.starts;
    if (map) a.axes = axes_view(*map, r.positions, r.tokens);
    else a.axes = AxesView{r.positions, r.tokens, 1, {}};
    a.cache = r.cache;
    a.scales = scales;
    a.rows = r.rows;
    a.q_stride = r.q_stride;
    a.kv_stride = r.kv_stride;
    a.tokens = (int32_t)r.tokens;
    a.heads = (int32_t)r.heads;
    a.d = (int32_t)r.d;
    a.rot = (int32_t)r.rot;
    const int64_t blocks = r.tokens / scales.block.d + 2 * (int64_t)r.cache.batch;
    a.most_blocks = (int32_t)(blocks < r.tokens ? blocks : r.tokens);
    return r.dt == DType::F32 ? launch_typed<float, 4>(r, a, stream) : launch_typed<uint16_t, 8>(r, a, stream);
}

}  // namespace attnw
