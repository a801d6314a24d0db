// Attention of new tokens over a paged cache in 8 bits, blocks of 16 rows: single tokens and short chunks.
//
//     O = softmax(s) V,  s = scale q . k  -> cap tanh(s / cap) -> s - slope |i - j|,  over the slots j that the token at slot i sees
//
// As paged_rows.h: a row is one query head of one token, the heads of a kv head and their tokens share a block, each wave has keys of its own, tiles of 32, that go
// from their pages into its part of LDS as they lie in memory, one tile under way while it computes another.  An element becomes bf16 (which holds it exactly) on its way
// to the matrix instruction, two to an instruction: keys with their scale, values without, whose scale goes into the weights.  A lane's 16 bytes
// of a key are 16 columns, the operands of two instructions; of values the transposing read of bytes gives a lane a column of the 8 keys that its weights are for.
// fp32 queries and weights are three bf16 parts, three products where the fp32 instruction would take eight times as long.  In bf16 a weight is rounded once, to bf16, as
// over a cache in bf16: a second part would be a second product of everything, and the roundings, up to 2^-8 of a weight, differ from key to key and mostly cancel (off the
// definition in 64 bits by 0.0016 to 0.0017 of the 2-norm, 0.0020 for 2048 tokens over 14336 slots; with weights in fp32 by 0.0016 to 0.0017, which is the output's own rounding).
//
// What bounds it: the read of K and V.  Measured, 32 heads on 8 of 128: a token each of 64 sequences of up to 16384 slots (1.22 GB) 230 us = 5.3 TB/s, of 16384 all 377 us =
// 5.7 TB/s (a cache in bf16 723); fp32, 64 of 8192 slots, 200 us (a cache in fp32 720).  One sequence of 4096 slots: 7.5 us, a chain of set-up, one tile and the waves' join.
// Four waves a workgroup: with eight the batch takes 229, drafts of 5 tokens over up to 8192 slots, 16 sequences, 29 instead of 21.
#pragma once

#include "paged_attention.h"
#include "byte_cache.h"

namespace attnw {
namespace {

// UB: 64-byte groups of a row on chip.  NX: blocks of 16 rows that share the keys.
template <int UB, int NX> struct ByteRowsCfg {
    static constexpr int ROWS = 16 * NX;
    static constexpr int KT = 32;                 // keys of a tile
    static constexpr int DB = UB * 64, CPR = UB * 4, TILE = KT * DB, XFERS = TILE / 1024;
    static constexpr int COLS = DB, CB = COLS / 16;
    static constexpr int NW = 4;
    static constexpr int UNIT = KT * NW;          // keys of a place
    static constexpr int PITCH = COLS + 4;        // floats of a row of partial results
    static constexpr int STAGES = NW * 4 * TILE, PLACES = kPlaces;
    static constexpr int LDS = STAGES + PLACES * 8 + NW * ROWS * 8;
    static constexpr int PER_CU = LDS > 80 * 1024 ? 1 : 2;
    static_assert(4 * TILE >= 16 * PITCH * 4, "partial results of 16 rows of a wave in its stages");
    static_assert(STAGES <= kDirectLds);
};

// Transposing LDS read of bytes (ds_read_b64_tr_b8): each group of 16 lanes reads eight runs of 16 bytes, lanes 2j and 2j + 1 run j, and lane i of the group gets
// byte i of the eight runs.
__device__ __forceinline__ u32x2 lds_read_tr8(const char* p)
{
#if defined(__HIP_DEVICE_COMPILE__)
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    typedef i32x2 __attribute__((address_space(3)))* tr_ptr;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((tr_ptr)(p)));
#else
    (void)p;
    return u32x2{0u, 0u};
#endif
}
// EXACT: rows fill their place on chip.  UNIFORM: 16 keys lie in one page and share their scales, so that where they are and what they count are numbers of the wave
// (together with K of the tile after the next on its way earlier: 32 tokens over 16384 slots, d = 128 35.1 -> 32.8 us, 128 tokens, d = 256 308 -> 291).
template <typename T, int UB, int NX, int MODE, bool EXACT, bool UNIFORM, int THREADS = 64 * ByteRowsCfg<UB, NX>::NW, int BLOCKS = ByteRowsCfg<UB, NX>::PER_CU>
__global__ __launch_bounds__(THREADS, BLOCKS)
void byte_rows_kernel(AttendArgs a, ScalesView scales, int grain)
{
    using C = ByteRowsCfg<UB, NX>;
    using L = RowLayout<UB>;
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
    constexpr bool F32 = PARTS == 3;
    constexpr int NW = C::NW, KT = C::KT, DB = C::DB, CPR = C::CPR, TILE = C::TILE, XFERS = C::XFERS, CB = C::CB, NK = KT / 16, PITCH = C::PITCH;
    __shared__ __align__(1024) char lds[C::LDS];
    int64_t* const places = reinterpret_cast<int64_t*>(lds + C::STAGES);
    float* const stats = reinterpret_cast<float*>(lds + C::STAGES + C::PLACES * 8);   // [wave][row]{maximum, sum}

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, l16 = lane & 15, quarter = lane >> 4;
    char* const stage = lds + wave * 4 * TILE;    // K, V of one tile, K, V of the next
    const uint32_t stage_at = lds_offset_of(stage);
    const int rb = EXACT ? DB : a.cache.row_bytes;

    Walk<C::ROWS> walk(a, lane);
    if (walk.at >= walk.end) return;

    const ScoreMap<(MODE & kCap) != 0, F32> map(a.rule);
    // Chunks of 16 bytes of V trade places so that eight rows of the transposing read (keys 4 q .. + 3 and 16 more) lie in different eighths of 128 bytes.
    const auto v_chunk = [](int key) __attribute__((always_inline)) {
        return UB % 2 == 0 ? (key & 3) | (key >> 2 & 4) : (key >> 1 & 1) | (key >> 3 & 2);
    };
    int k_from[UB], v_from[XFERS];                // UNIFORM: where a lane's 16 bytes lie in the 16 keys
    if constexpr (UNIFORM) {
#pragma unroll
        for (int j = 0; j < XFERS; ++j) {
            const int x = j * 64 + lane, key = x / CPR, c = x - key * CPR;
            const auto at = [&](int ch) __attribute__((always_inline)) { return (key & 15) * rb + (EXACT ? ch * 16 : chunk_in_row(ch * 16, rb)); };
            if (j < UB) k_from[j] = at(c ^ L::k_chunk(key));
            v_from[j] = at(c ^ v_chunk(key));
        }
    }
    Segment seg;
    while (walk.next(seg)) {
        const Sequence& seq = seg.seq;
        const int prefix = seg.prefix, kv_head = seg.kv_head, row0 = seg.row0, rows = seg.rows;
        // ---- the rows of the block ------------------------------------------------------------------------------------------------
        const int group = a.group.d, base = seq.length - seq.tokens;              // slot of the first new token
        const int first = base + (int)quotient(row0, a.group), last = base + (int)quotient(row0 + rows - 1, a.group);
        int query[NX];                            // sees the slots query - window + 1 .. query
        float slope[NX];
        Parts<PARTS> qf[NX][2 * UB];              // columns 64 g + 16 quarter .. + 7, and the 8 behind them (zeros behind the row's end)
#pragma unroll
        for (int n = 0; n < NX; ++n) {
            const int row = row0 + min(16 * n + l16, rows - 1);
            const int token = (int)quotient(row, a.group), head = kv_head * group + row - token * group;
            query[n] = base + token;
            slope[n] = MODE & kBias ? a.rule.slopes[head] * kLog2e : 0.0f;
            const char* q = a.Q + (int64_t)(seq.first + token) * a.q_stride + (int64_t)head * rb * (int)sizeof(T);
#pragma unroll
            for (int g = 0; g < UB; ++g) {
                const int at = (4 * g + quarter) * 16;
                const bool inside = EXACT || at < rb;
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const char* const p = q + (inside ? at + 8 * half : 0) * (int)sizeof(T);
                    if constexpr (F32) {
                        const f32x4 lo = *reinterpret_cast<const f32x4*>(p), hi = *reinterpret_cast<const f32x4*>(p + 16);
                        float y[8];
#pragma unroll
                        for (int i = 0; i < 4; ++i) y[i] = inside ? lo[i] : 0.0f, y[4 + i] = inside ? hi[i] : 0.0f;
                        qf[n][2 * g + half] = parts_of<PARTS>(y);
                    } else {
                        qf[n][2 * g + half].of[0] = inside ? *reinterpret_cast<const u32x4*>(p) : u32x4{0, 0, 0, 0};
                    }
                }
            }
        }
        f32x4 oacc[CB][NX];
#pragma unroll
        for (int c = 0; c < CB; ++c)
#pragma unroll
            for (int n = 0; n < NX; ++n) oacc[c][n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        float m_run[NX], l_run[NX];
#pragma unroll
        for (int n = 0; n < NX; ++n) m_run[n] = -__builtin_inff(), l_run[n] = 0.0f;

        // ---- the keys of places v0 .. v1 - 1 -----------------------------------------------------------------------------------------
        const Span span = visible_span(a.unit_log, first, last, seq.length, prefix, a.rule.window);
        const int units = last < 0 && span.head == 0 ? 0 : span.count();
        const int u0 = walk.share(seg, seg.v0, units), u1 = walk.share(seg, seg.v1, units);
        const int seen = min(seq.length, max(prefix, last + 1));
        const int32_t* const pages_of = a.cache.table + (int64_t)seg.b * a.cache.max_pages;

        auto sweep = [&](int from, int to) __attribute__((always_inline)) {   // keys
            const int most = C::PLACES << grain;    // (a whole number of units: the waves' tiles stay where they are)
            for (int k0 = from; k0 < to;) {
                const int k1 = min(to, k0 + most);
                __syncthreads();
                for (int i = threadIdx.x; i < (k1 - k0 + (1 << grain) - 1) >> grain; i += 64 * NW)
                    places[i] = slot_place(a.cache, scales, pages_of, kv_head, k0 + (i << grain));
                wait_vmem();
                __syncthreads();

                // K (v = 0) or V of a tile into stage s.  Past the end: the last slot, or, of 16 keys some of which are there, those behind them, which nobody sees.
                // (Behind a row's end on chip: its first chunks, which meet zeros of Q and make columns of V that nobody stores.)
                auto issue = [&](int v, int key0, int s) __attribute__((always_inline)) {
                    const char* const from = v ? a.cache.V : a.cache.K;
                    if constexpr (UNIFORM) {
                        const char* half[2];
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const int64_t place = places[(min(key0 + 16 * k, k1 - 1) - k0) >> 4];
                            half[k] = from + ((int64_t)(uint32_t)uniform((int)place) | (int64_t)(uniform((int)(place >> 32)) & 0xffff) << 32);
                        }
#pragma unroll
                        for (int j = 0; j < XFERS; ++j)
                            dma16_untracked(half[j / UB], (uint32_t)(v ? v_from[j] : k_from[j % UB]), stage_at + (2 * s + v) * TILE + j * 1024);
                    } else {
#pragma unroll
                        for (int j = 0; j < XFERS; ++j) {
                            const int x = j * 64 + lane, key = x / CPR, c = x - key * CPR, slot = min(key0 + key, k1 - 1) - k0;
                            const int ch = v == 0 ? c ^ L::k_chunk(key) : c ^ v_chunk(key);
                            dma16_untracked(from + place_offset(places[slot >> grain]) + (slot & ((1 << grain) - 1)) * rb + (EXACT ? ch * 16 : chunk_in_row(ch * 16, rb)),
                                            stage_at + (2 * s + v) * TILE + j * 1024);
                        }
                    }
                };
                const auto high_of = [&](int key) __attribute__((always_inline)) {   // of a key's place the half with the scales
                    return reinterpret_cast<const uint32_t*>(places)[2 * ((min(key, k1 - 1) - k0) >> (UNIFORM ? 4 : grain)) + 1];
                };
                auto compute = [&](int key0, int s, bool more, bool yet_more) __attribute__((always_inline)) {
                    const char* const kt = stage + 2 * s * TILE;
                    const char* const vt = kt + TILE;
                    if (more) arrived<3 * XFERS>();
                    else arrived<XFERS>();
                    float x[NX][NK * 4];
#pragma unroll
                    for (int k = 0; k < NK; ++k) {
                        const float ks = key_scale(high_of(key0 + 16 * k + (UNIFORM ? 0 : l16)));
                        f32x4 acc[NX];
#pragma unroll
                        for (int n = 0; n < NX; ++n) acc[n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                        for (int g = 0; g < UB; ++g) {
                            const u32x4 w = *reinterpret_cast<const u32x4*>(kt + (16 * k + l16) * DB + ((4 * g + quarter) ^ L::k_chunk(l16)) * 16);
                            const u32x4 lo = bf16_of(w[0], w[1], ks), hi = bf16_of(w[2], w[3], ks);
#pragma unroll
                            for (int n = 0; n < NX; ++n) {
                                multiply_parts(acc[n], lo, qf[n][2 * g]);
                                multiply_parts(acc[n], hi, qf[n][2 * g + 1]);
                            }
                        }
#pragma unroll
                        for (int n = 0; n < NX; ++n)
#pragma unroll
                            for (int r = 0; r < 4; ++r) x[n][4 * k + r] = acc[n][r];
                    }
                    if (yet_more) {                            // (K has been read: its place is the tile's after the next)
                        wait_lds();
                        issue(0, key0 + 2 * C::UNIT, s);
                    }
                    const int key = key0 + 4 * quarter;        // + 16 k + r
                    const bool whole = key0 + KT <= k1 && ((key0 + KT - 1 <= first && key0 > last - a.rule.window) || key0 + KT <= prefix);
                    // the values' scales, which go into the weights (powers of 2: no rounding)
                    float vs[NK * 4];
#pragma unroll
                    for (int k = 0; k < NK; ++k) {
                        if (UNIFORM || grain >= 2) {
                            const float same = value_scale(high_of((UNIFORM ? key0 : key) + 16 * k));
#pragma unroll
                            for (int r = 0; r < 4; ++r) vs[4 * k + r] = same;
                        } else {
#pragma unroll
                            for (int r = 0; r < 4; ++r) vs[4 * k + r] = value_scale(high_of(key + 16 * k + r));
                        }
                    }
                    Parts<PARTS> pw[NX];
#pragma unroll
                    for (int n = 0; n < NX; ++n) {
                        float (&y)[NK * 4] = x[n];
                        map(y);
                        if constexpr ((MODE & kBias) != 0) {
#pragma unroll
                            for (int i = 0; i < NK * 4; ++i) y[i] -= slope[n] * (float)abs(query[n] - (key + 16 * (i / 4) + i % 4));
                        }
                        if (!whole) {
                            const Sight sight(query[n], a.rule, prefix, k1);
#pragma unroll
                            for (int i = 0; i < NK * 4; ++i) y[i] = sight.hidden(key + 16 * (i / 4) + i % 4) < 0 ? -__builtin_inff() : y[i];
                        }
                        float top = y[0];
#pragma unroll
                        for (int i = 1; i < NK * 4; ++i) top = fmaxf(top, y[i]);
                        top = quarter_wave_max(top);
                        if (__builtin_amdgcn_ballot_w64(top > m_run[n]) != 0) {
                            const float m = fmaxf(m_run[n], top), alpha = m == -__builtin_inff() ? 1.0f : fast_exp2(m_run[n] - m);
                            l_run[n] *= alpha;
#pragma unroll
                            for (int c = 0; c < CB; ++c) oacc[c][n] *= alpha;
                            m_run[n] = m;
                        }
                        const float ref = m_run[n] == -__builtin_inff() ? 0.0f : m_run[n];   // (nothing seen yet: all weights 0)
#pragma unroll
                        for (int i = 0; i < NK * 4; ++i) {
                            y[i] = fast_exp2(y[i] - ref);
                            l_run[n] += y[i];
                            y[i] *= vs[i];
                        }
                        pw[n] = parts_of<PARTS>(y);
                    }
                    if (yet_more) arrived<3 * XFERS>();
                    else if (more) arrived<2 * XFERS>();
                    else arrived<0>();
                    // fragments of V: 16 columns x the keys of this lane's weights
                    const int vkey = 4 * quarter + (l16 >> 1 & 3) + (l16 >> 3) * 16;
                    const auto v_frag = [&](int c) __attribute__((always_inline)) {
                        const u32x2 w = lds_read_tr8(vt + vkey * DB + (c ^ v_chunk(vkey)) * 16 + (lane & 1) * 8);
                        return bf16_of(w[0], w[1], 1.0f);
                    };
                    if (!whole) {
                        uint32_t bad = 0;
#pragma unroll
                        for (int c = 0; c < CB; ++c) bad |= any_lost<uint16_t>(v_frag(c));
                        if (__builtin_amdgcn_ballot_w64(bad != 0) != 0) {
                            // NaN among the values, which must not reach rows that do not see them by way of a weight of 0: 0 in the product, and NaN for those that do
                            u32x4 so[NX];
#pragma unroll
                            for (int n = 0; n < NX; ++n) {
                                const Sight sight(query[n], a.rule, prefix, k1);
                                float some[NK * 4];
#pragma unroll
                                for (int i = 0; i < NK * 4; ++i) some[i] = sight.hidden(key + 16 * (i / 4) + i % 4) < 0 ? 0.0f : 1.0f;
                                so[n] = parts_of<1>(some).of[0];
                            }
#pragma unroll
                            for (int c = 0; c < CB; ++c) {
                                const u32x4 v = v_frag(c);
#pragma unroll
                                for (int n = 0; n < NX; ++n) {
                                    f32x4 lost = {0.0f, 0.0f, 0.0f, 0.0f};
                                    mma16(lost, lost_as_one<uint16_t, kAny>(v), so[n]);
                                    multiply_parts(oacc[c][n], without_lost<uint16_t>(v), pw[n]);
#pragma unroll
                                    for (int r = 0; r < 4; ++r) oacc[c][n][r] = lost[r] > 0.0f ? __builtin_nanf("") : oacc[c][n][r];
                                }
                            }
                            return;
                        }
                    }
#pragma unroll
                    for (int c = 0; c < CB; ++c) {
                        const u32x4 v = v_frag(c);
#pragma unroll
                        for (int n = 0; n < NX; ++n) multiply_parts(oacc[c][n], v, pw[n]);
                    }
                };
                int key = k0 + wave * KT, s = 0;
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int v = 0; v < 2; ++v)
                        if (key + n * C::UNIT < k1) issue(v, key + n * C::UNIT, n);
                for (; key < k1; key += C::UNIT, s ^= 1) {
                    const bool more = key + C::UNIT < k1, yet_more = key + 2 * C::UNIT < k1;
                    compute(key, s, more, yet_more);
                    if (yet_more) {
                        wait_lds();               // (the fragments have left the place that is filled next)
                        issue(1, key + 2 * C::UNIT, s);
                    }
                }
                k0 = k1;
            }
        };
#pragma clang loop unroll(disable)
        for (int part = 0; part < 2; ++part) {    // of the prefix, of what is near
            const int f = part == 0 ? u0 : max(u0, span.head), t = part == 0 ? min(u1, span.head) : u1;
            if (f < t) sweep(span.unit(f) << a.unit_log, (int)min((int64_t)seen, (int64_t)(span.unit(t - 1) + 1) << a.unit_log));
        }
        // ---- the waves' results into one, 16 rows at a time -----------------------------------------------------------------------------
        const bool complete = seg.slot < 0;
        float* const out = a.partial + max(seg.slot, 0) * (int64_t)(C::ROWS * (C::COLS + 2));
        constexpr int QUADS = C::COLS / 4;
#pragma unroll
        for (int n = 0; n < NX; ++n) {
            const float l_all = quarter_wave_sum(l_run[n]);
            __syncthreads();
            if (quarter == 0) {
                stats[(wave * 16 + l16) * 2] = m_run[n];
                stats[(wave * 16 + l16) * 2 + 1] = l_all;
            }
            float* const mine = reinterpret_cast<float*>(stage);
#pragma unroll
            for (int c = 0; c < CB; ++c) *reinterpret_cast<f32x4*>(mine + l16 * PITCH + 16 * c + 4 * quarter) = oacc[c][n];
            __syncthreads();
            for (int i = threadIdx.x; i < min(16, rows - 16 * n) * QUADS; i += 64 * NW) {
                const int r = i / QUADS, c = (i - r * QUADS) * 4;
                float top = -__builtin_inff();
#pragma unroll
                for (int w = 0; w < NW; ++w) top = fmaxf(top, stats[(w * 16 + r) * 2]);
                const float ref = top == -__builtin_inff() ? 0.0f : top;
                f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
                float l = 0.0f;
#pragma unroll
                for (int w = 0; w < NW; ++w) {
                    const float f = fast_exp2(stats[(w * 16 + r) * 2] - ref);
                    l += f * stats[(w * 16 + r) * 2 + 1];
                    sum += *reinterpret_cast<const f32x4*>(lds + w * 4 * TILE + (r * PITCH + c) * 4) * f;
                }
                const int row = 16 * n + r;
                if (complete) {
                    const int tk = (int)quotient(row0 + row, a.group), h = kv_head * group + row0 + row - tk * group;
                    const int64_t o = (int64_t)(seq.first + tk) * a.heads + h;
                    store_output<T>(a.O, o, rb * (int)sizeof(T), c, sum, l);
                    if (c == 0 && a.lse) a.lse[o] = log_sum(top, l);
                } else {
                    *reinterpret_cast<f32x4*>(out + row * C::COLS + c) = sum;
                    if (c == 0) {
                        out[C::ROWS * C::COLS + 2 * row] = top;
                        out[C::ROWS * C::COLS + 2 * row + 1] = l;
                    }
                }
            }
        }
    }
}

// Blocks of 32 rows where a sequence has more than 16: 256 rows over 16384 slots, d = 128, a kv head, 202 -> 139 us (up to d = 128, fp32 64: beyond, the registers do not
// hold them, d = 256 588 -> 692).
template <typename T, int UB> constexpr int kMostBlocks = UB == 1 || (UB == 2 && sizeof(T) == 2) ? 2 : 1;
inline int blocks_of(const PagedArgs& p, int most) { return most > 1 && p.tokens * (p.heads / p.cache.kv_heads) > 16 * (int64_t)p.cache.batch ? 2 : 1; }

template <int UB, int NX> int byte_workgroups() { return (compute_units() * ByteRowsCfg<UB, NX>::PER_CU + 7) & ~7; }

template <typename T, int UB, int NX, int MODE> hipError_t launch(const PagedArgs& p, const ScalesView& scales, hipStream_t stream)
{
    using C = ByteRowsCfg<UB, NX>;
    AttendArgs a = attend_args(p, byte_workgroups<UB, NX>(), C::ROWS, C::UNIT, sizeof(T));
    const int grain = key_grain(a.cache, scales);
    // (rows that fill their place: kernels of their own for the usual sizes)
    constexpr bool OWN = UB != 3;
    if (grain < 4) byte_rows_kernel<T, UB, NX, MODE, false, false><<<a.workgroups, 64 * C::NW, 0, stream>>>(a, scales, grain);
    else if (OWN && a.cache.row_bytes == C::DB) byte_rows_kernel<T, UB, NX, MODE, OWN, true><<<a.workgroups, 64 * C::NW, 0, stream>>>(a, scales, grain);
    else byte_rows_kernel<T, UB, NX, MODE, false, true><<<a.workgroups, 64 * C::NW, 0, stream>>>(a, scales, grain);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    a.cache.row_bytes *= (int)sizeof(T);          // (of the output)
    return launch_join<T>(a, C::ROWS, C::COLS, stream);
}

template <typename F> auto by_row(int row_bytes, F&& f)
{
    const int ub = (row_bytes + 63) / 64;
    if (ub <= 1) return f(IC<1>{});
    if (ub <= 2) return f(IC<2>{});
    if (ub <= 3) return f(IC<3>{});
    return f(IC<4>{});
}

template <typename T> int64_t rows_workspace(const PagedArgs& p)
{
    return by_row(p.cache.row_bytes, [&](auto ubc) {
        constexpr int UB = decltype(ubc)::value, MOST = kMostBlocks<T, UB>;
        const auto of = [](auto nx) {
            using C = ByteRowsCfg<UB, decltype(nx)::value>;
            return partial_bytes(byte_workgroups<UB, decltype(nx)::value>(), C::ROWS, C::COLS);
        };
        return blocks_of(p, MOST) == 2 ? of(IC<MOST>{}) : of(IC<1>{});
    });
}

template <typename T> hipError_t launch_rows(const PagedArgs& p, const ScalesView& scales, hipStream_t stream)
{
    return by_row(p.cache.row_bytes, [&](auto ubc) {
        constexpr int UB = decltype(ubc)::value, MOST = kMostBlocks<T, UB>;
        const auto by_rule = [&](auto nx) {
            constexpr int NX = decltype(nx)::value;
            switch (rule_mode(p.rule)) {
            case kPlain: return launch<T, UB, NX, kPlain>(p, scales, stream);
            case kCap: return launch<T, UB, NX, kCap>(p, scales, stream);
            case kBias: return launch<T, UB, NX, kBias>(p, scales, stream);
            default: return launch<T, UB, NX, kCap | kBias>(p, scales, stream);
            }
        };
        return blocks_of(p, MOST) == 2 ? by_rule(IC<MOST>{}) : by_rule(IC<1>{});
    });
}

}  // namespace
}  // namespace attnw
