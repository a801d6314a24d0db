// Attention of new tokens over a paged cache, blocks of 16 rows: single tokens and short chunks.
//
//     O = softmax(s) V,  s = scale q . k  -> cap tanh(s / cap) -> s - slope |i - j|,  over the slots j that the token at slot i sees
//
// A row is one query head of one token; the heads of a kv head and their tokens share a block, so that K and V are read once for all of them.
// The running maximum and sum of the softmax make one sweep over the keys enough.
//
// What bounds it: the read of K and V.  Nothing is used by two waves, so each wave brings its own tiles into LDS, 16 bytes a lane straight
// from memory, one tile under way while it computes another, and no barrier ties the waves together; they meet once a segment, when their
// partial results are joined.  The places of a ragged batch are dealt out evenly (Walk): a sequence of 16384 slots beside 63 short ones is
// shared by as many workgroups as its length is worth.  Measured: a token each of 64 sequences of 16384 slots, 8 kv heads of 128 691 us, 6.2 TB/s; one sequence of 4097 slots
// 7.7 us and 4 more for the join, most of it the chain of instructions before the first load.
#pragma once

#include "paged_attention.h"

namespace attnw {
namespace {

constexpr int kRows = 16;                         // of a block

// UB: 64-byte groups of a row on chip.
template <typename T, int UB> struct RowsCfg {
    static constexpr bool F32 = sizeof(T) == 4;
    static constexpr int KT = F32 ? 16 : 32;      // keys of a tile
    static constexpr int DB = UB * 64, CPR = UB * 4, TILE = KT * DB, XFERS = TILE / 1024;
    static constexpr int COLS = DB / (int)sizeof(T), CB = COLS / 16;
    static constexpr int FIT = 128 * 1024 / (4 * TILE);
    static constexpr int NW = FIT >= 8 ? 8 : FIT >= 4 ? 4 : 2;
    static constexpr int UNIT = KT * NW;          // keys of a place
    static constexpr int PITCH = COLS + 4;        // floats of a row of partial results
    static constexpr int STAGES = NW * 4 * TILE;
    static constexpr int LDS = STAGES + kPlaces * 8 + NW * kRows * 8;
    static constexpr int PER_CU = LDS > 80 * 1024 ? 1 : 2;
    static_assert(4 * TILE >= kRows * PITCH * 4, "partial results of a wave in its stages");
    static_assert(STAGES <= kDirectLds && FIT >= 2);
};

// EXACT: rows fill their place on chip.
template <typename T, int UB, int MODE, bool EXACT, int THREADS = 64 * RowsCfg<T, UB>::NW, int WAVES = UB <= (sizeof(T) == 4 ? 8 : 5) ? 2 : 1>
__global__ __launch_bounds__(THREADS, WAVES)
void paged_rows_kernel(AttendArgs a, int grain)
{
    using C = RowsCfg<T, UB>;
    using L = RowLayout<UB>;
    constexpr bool F32 = C::F32;
    constexpr int NW = C::NW, KT = C::KT, DB = C::DB, CPR = C::CPR, TILE = C::TILE, XFERS = C::XFERS, CB = C::CB, NK = KT / 16, PITCH = C::PITCH;
    __shared__ __align__(1024) char lds[C::LDS];
    int64_t* const places = reinterpret_cast<int64_t*>(lds + C::STAGES);
    float* const stats = reinterpret_cast<float*>(lds + C::STAGES + kPlaces * 8);   // [wave][row]{maximum, sum}

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, l16 = lane & 15, quarter = lane >> 4;
    char* const stage = lds + wave * 4 * TILE;    // K, V of one tile, K, V of the next
    const uint32_t stage_at = lds_offset_of(stage);
    const int rb = EXACT ? DB : a.cache.row_bytes;

    Walk<kRows> walk(a, lane);
    if (walk.at >= walk.end) return;

    const ScoreMap<(MODE & kCap) != 0, F32> map(a.rule);
    Segment seg;
    while (walk.next(seg)) {
        const Sequence& seq = seg.seq;
        const int prefix = seg.prefix, kv_head = seg.kv_head, row0 = seg.row0, rows = seg.rows;
        // ---- the rows of the block ------------------------------------------------------------------------------------------------
        const int group = a.group.d, base = seq.length - seq.tokens;              // slot of the first new token
        const int first = base + (int)quotient(row0, a.group), last = base + (int)quotient(row0 + rows - 1, a.group);
        const int row = row0 + min(l16, rows - 1);
        const int token = (int)quotient(row, a.group), head = kv_head * group + row - token * group;
        const int query = base + token;   // sees the slots query - window + 1 .. query
        const float slope = MODE & kBias ? a.rule.slopes[head] * kLog2e : 0.0f;

        u32x4 qf[UB];
        {
            const char* q = a.Q + (int64_t)(seq.first + token) * a.q_stride + (int64_t)head * rb;
#pragma unroll
            for (int g = 0; g < UB; ++g) {
                const int ch = 4 * g + quarter;
                qf[g] = EXACT ? *reinterpret_cast<const u32x4*>(q + ch * 16) : query_chunk<T>(q, ch, CPR, rb);
            }
        }
        f32x4 oacc[CB];
#pragma unroll
        for (int c = 0; c < CB; ++c) oacc[c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        float m_run = -__builtin_inff(), l_run = 0.0f;

        // ---- the keys of places v0 .. v1 - 1 -----------------------------------------------------------------------------------------
        const Span span = visible_span(a.unit_log, first, last, seq.length, prefix, a.rule.window);
        const int units = last < 0 && span.head == 0 ? 0 : span.count();
        const int u0 = walk.share(seg, seg.v0, units), u1 = walk.share(seg, seg.v1, units);
        const int seen = min(seq.length, max(prefix, last + 1));
        const int32_t* const pages_of = a.cache.table + (int64_t)seg.b * a.cache.max_pages;

        auto sweep = [&](int from, int to) __attribute__((always_inline)) {   // keys
            const int most = kPlaces << grain;    // (a whole number of units: the waves' tiles stay where they are)
            for (int k0 = from; k0 < to;) {
                const int k1 = min(to, k0 + most);
                __syncthreads();
                for (int i = threadIdx.x; i < (k1 - k0 + (1 << grain) - 1) >> grain; i += 64 * NW)
                    places[i] = slot_offset(a.cache, pages_of, kv_head, k0 + (i << grain));
                wait_vmem();
                __syncthreads();

                auto issue = [&](int key0, int s) __attribute__((always_inline)) {
                    int64_t row[XFERS];
#pragma unroll
                    for (int j = 0; j < XFERS; ++j) {          // (past the end the last slot)
                        const int slot = min(key0 + (j * 64 + lane) / CPR, k1 - 1) - k0;
                        row[j] = places[slot >> grain] + (slot & ((1 << grain) - 1)) * rb;
                    }
#pragma unroll
                    for (int v = 0; v < 2; ++v)
#pragma unroll
                        for (int j = 0; j < XFERS; ++j) {
                            const int x = j * 64 + lane, key = x / CPR, c = x - key * CPR;
                            const int ch = v == 0 ? c ^ L::k_chunk(key)
                                         : F32 ? c ^ ((UB % 4 == 0 ? (key >> 2) & 3 : UB % 4 == 2 ? (key >> 2) & 1 : 0) * 4)
                                               : c ^ (L::v16_block(key) * 2);
                            // (behind a row's end on chip: its first chunks, which query_chunk expects and which make columns of V that nobody stores)
                            dma16_untracked((v ? a.cache.V : a.cache.K) + row[j] + (EXACT ? ch * 16 : chunk_in_row(ch * 16, rb)), stage_at + (2 * s + v) * TILE + j * 1024);
                        }
                };
                auto compute = [&](int key0, int s, bool more) __attribute__((always_inline)) {
                    const char* const kt = stage + 2 * s * TILE;
                    const char* const vt = kt + TILE;
                    if (more) arrived<3 * XFERS>();
                    else arrived<XFERS>();
                    float x[NK * 4];
#pragma unroll
                    for (int k = 0; k < NK; ++k) {
                        f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                        for (int g = 0; g < UB; ++g) {
                            const u32x4 kf = *reinterpret_cast<const u32x4*>(kt + (16 * k + l16) * DB + ((4 * g + quarter) ^ L::k_chunk(l16)) * 16);
                            if constexpr (F32) {
#pragma unroll
                                for (int i = 0; i < 4; ++i)
                                    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[i]), __uint_as_float(qf[g][i]), acc, 0, 0, 0);
                            } else {
                                mma16(acc, kf, qf[g]);
                            }
                        }
#pragma unroll
                        for (int r = 0; r < 4; ++r) x[4 * k + r] = acc[r];
                    }
                    map(x);
                    const int key = key0 + 4 * quarter;        // + 16 k + r
                    if constexpr ((MODE & kBias) != 0) {
#pragma unroll
                        for (int i = 0; i < NK * 4; ++i) x[i] -= slope * (float)abs(query - (key + 16 * (i / 4) + i % 4));
                    }
                    const bool whole = key0 + KT <= k1 && ((key0 + KT - 1 <= first && key0 > last - a.rule.window) || key0 + KT <= prefix);
                    if (!whole) {
                        const Sight sight(query, a.rule, prefix, k1);
#pragma unroll
                        for (int i = 0; i < NK * 4; ++i) x[i] = sight.hidden(key + 16 * (i / 4) + i % 4) < 0 ? -__builtin_inff() : x[i];
                    }
                    float top = x[0];
#pragma unroll
                    for (int i = 1; i < NK * 4; ++i) top = fmaxf(top, x[i]);
                    top = quarter_wave_max(top);
                    if (__builtin_amdgcn_ballot_w64(top > m_run) != 0) {
                        const float m = fmaxf(m_run, top), alpha = m == -__builtin_inff() ? 1.0f : fast_exp2(m_run - m);
                        l_run *= alpha;
#pragma unroll
                        for (int c = 0; c < CB; ++c) oacc[c] *= alpha;
                        m_run = m;
                    }
                    const float ref = m_run == -__builtin_inff() ? 0.0f : m_run;   // (nothing seen yet: all weights 0)
                    float p[NK * 4];
#pragma unroll
                    for (int i = 0; i < NK * 4; ++i) {
                        p[i] = fast_exp2(x[i] - ref);
                        l_run += p[i];
                    }
                    if (more) arrived<2 * XFERS>();
                    else arrived<0>();
                    // fragments of V: 16 columns x the keys of this lane's weights
                    const int vkey = 4 * quarter + (l16 >> 2);
                    const auto v_frag = [&](int c) __attribute__((always_inline)) {
                        if constexpr (F32) {
                            const int turn = UB % 4 == 0 ? quarter & 3 : UB % 4 == 2 ? quarter & 1 : 0;
                            u32x4 v;
#pragma unroll
                            for (int r = 0; r < 4; ++r) v[r] = *reinterpret_cast<const uint32_t*>(vt + (4 * quarter + r) * DB + (c ^ turn) * 64 + l16 * 4);
                            return v;
                        } else {
                            const char* const v = vt + vkey * DB + (lane & 3) * 8 + (c ^ L::v16_block(vkey)) * 32;
                            return u32x4_of(lds_read_tr16(v), lds_read_tr16(v + 16 * DB));
                        }
                    };
                    const auto multiply = [&](f32x4& acc, const u32x4& v, const u32x4& w) __attribute__((always_inline)) {
                        if constexpr (F32) {
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[r]), __uint_as_float(w[r]), acc, 0, 0, 0);
                        } else {
                            mma16(acc, v, w);
                        }
                    };
                    const auto operand = [&](const float (&y)[NK * 4]) __attribute__((always_inline)) {
                        if constexpr (F32) return u32x4{__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]), __float_as_uint(y[3])};
                        else return u32x4{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7])};
                    };
                    const u32x4 pw = operand(p);
                    if (!whole) {
                        uint32_t bad = 0;
#pragma unroll
                        for (int c = 0; c < CB; ++c) bad |= any_lost<T>(v_frag(c));
                        if (__builtin_amdgcn_ballot_w64(bad != 0) != 0) {                      // (lost_part)
                            const Sight sight(query, a.rule, prefix, k1);
                            float some[NK * 4], none[NK * 4];
#pragma unroll
                            for (int i = 0; i < NK * 4; ++i) {
                                const bool hidden = sight.hidden(key + 16 * (i / 4) + i % 4) < 0;
                                const uint32_t weight = F32 ? pw[i % 4] : i % 2 ? pw[i / 2 % 4] >> 16 : pw[i / 2 % 4] & 0xffffu;   // (as it is multiplied)
                                some[i] = hidden || weight == 0 ? 0.0f : 1.0f;
                                none[i] = hidden || weight != 0 ? 0.0f : 1.0f;
                            }
                            const u32x4 so = operand(some), no = operand(none);
#pragma unroll
                            for (int c = 0; c < CB; ++c) {
                                const u32x4 v = v_frag(c);
                                multiply(oacc[c], without_lost<T>(v), pw);
                                oacc[c] += lost_part<T>(v, so, no, multiply);
                            }
                            return;
                        }
                    }
#pragma unroll
                    for (int c = 0; c < CB; ++c) multiply(oacc[c], v_frag(c), pw);
                };
                int key = k0 + wave * KT, s = 0;
                if (key < k1) issue(key, 0);
                for (; key < k1; key += C::UNIT, s ^= 1) {
                    const bool more = key + C::UNIT < k1;
                    if (more) issue(key + C::UNIT, s ^ 1);
                    compute(key, s, more);
                    wait_lds();                   // (the fragments have left the stage that is filled next)
                }
                k0 = k1;
            }
        };
#pragma clang loop unroll(disable)
        for (int part = 0; part < 2; ++part) {    // of the prefix, of what is near
            const int f = part == 0 ? u0 : max(u0, span.head), t = part == 0 ? min(u1, span.head) : u1;
            if (f < t) sweep(span.unit(f) << a.unit_log, (int)min((int64_t)seen, (int64_t)(span.unit(t - 1) + 1) << a.unit_log));
        }
        l_run = quarter_wave_sum(l_run);

        // ---- the waves' results into one -----------------------------------------------------------------------------------------------
        __syncthreads();
        if (quarter == 0) {
            stats[(wave * kRows + l16) * 2] = m_run;
            stats[(wave * kRows + l16) * 2 + 1] = l_run;
        }
        float* const mine = reinterpret_cast<float*>(stage);
#pragma unroll
        for (int c = 0; c < CB; ++c) *reinterpret_cast<f32x4*>(mine + l16 * PITCH + 16 * c + 4 * quarter) = oacc[c];
        __syncthreads();
        const bool complete = seg.slot < 0;
        float* const out = a.partial + max(seg.slot, 0) * (int64_t)(kRows * (C::COLS + 2));
        constexpr int QUADS = C::COLS / 4;
        for (int i = threadIdx.x; i < rows * QUADS; i += 64 * NW) {
            const int r = i / QUADS, c = (i - r * QUADS) * 4;
            float top = -__builtin_inff();
#pragma unroll
            for (int n = 0; n < NW; ++n) top = fmaxf(top, stats[(n * kRows + r) * 2]);
            const float ref = top == -__builtin_inff() ? 0.0f : top;
            f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
            float l = 0.0f;
#pragma unroll
            for (int n = 0; n < NW; ++n) {
                const float f = fast_exp2(stats[(n * kRows + r) * 2] - ref);
                l += f * stats[(n * kRows + r) * 2 + 1];
                sum += *reinterpret_cast<const f32x4*>(lds + n * 4 * TILE + (r * PITCH + c) * 4) * f;
            }
            if (complete) {
                const int tk = (int)quotient(row0 + r, a.group), h = kv_head * group + row0 + r - tk * group;
                const int64_t o = (int64_t)(seq.first + tk) * a.heads + h;
                store_output<T>(a.O, o, rb, c, sum, l);
                if (c == 0 && a.lse) a.lse[o] = log_sum(top, l);
            } else {
                *reinterpret_cast<f32x4*>(out + r * C::COLS + c) = sum;
                if (c == 0) {
                    out[kRows * C::COLS + 2 * r] = top;
                    out[kRows * C::COLS + 2 * r + 1] = l;
                }
            }
        }
    }
}

template <typename T, int UB> int workgroups() { return (compute_units() * RowsCfg<T, UB>::PER_CU + 7) & ~7; }

template <typename T, int UB, int MODE> hipError_t launch(const PagedArgs& p, hipStream_t stream)
{
    using C = RowsCfg<T, UB>;
    const AttendArgs a = attend_args(p, workgroups<T, UB>(), kRows, C::UNIT, sizeof(T));
    const int grain = key_grain(a.cache);
    // (rows that fill their place: kernels of their own for the usual sizes)
    constexpr bool OWN = UB == 2 || UB == 4 || UB == 8;
    if (OWN && a.cache.row_bytes == C::DB) paged_rows_kernel<T, UB, MODE, OWN><<<a.workgroups, 64 * C::NW, 0, stream>>>(a, grain);
    else paged_rows_kernel<T, UB, MODE, false><<<a.workgroups, 64 * C::NW, 0, stream>>>(a, grain);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : launch_join<T>(a, kRows, C::COLS, stream);
}

template <typename T, int UB> int64_t workspace() { return partial_bytes(workgroups<T, UB>(), kRows, RowsCfg<T, UB>::COLS); }

template <typename T, typename F> auto by_row(int row_bytes, F&& f)
{
    const int ub = (row_bytes + 63) / 64;
    if (ub <= 1) return f(IC<1>{});
    if (ub <= 2) return f(IC<2>{});
    if constexpr (sizeof(T) == 2) if (ub <= 3) return f(IC<3>{});
    if (ub <= 4) return f(IC<4>{});
    if constexpr (sizeof(T) == 2) if (ub <= 5) return f(IC<5>{});
    if (ub <= 6) return f(IC<6>{});
    if constexpr (sizeof(T) == 2) {
        if (ub <= 7) return f(IC<7>{});
        return f(IC<8>{});
    } else {
        if (ub <= 8) return f(IC<8>{});
        if (ub <= 12) return f(IC<12>{});
        return f(IC<16>{});
    }
}

template <typename T> int64_t rows_workspace(const PagedArgs& p)
{
    return by_row<T>(p.cache.row_bytes, [&](auto ub) { return workspace<T, decltype(ub)::value>(); });
}

template <typename T> hipError_t launch_rows(const PagedArgs& p, hipStream_t stream)
{
    return by_row<T>(p.cache.row_bytes, [&](auto ubc) {
        constexpr int UB = decltype(ubc)::value;
        switch (rule_mode(p.rule)) {
        case kPlain: return launch<T, UB, kPlain>(p, stream);
        case kCap: return launch<T, UB, kCap>(p, stream);
        case kBias: return launch<T, UB, kBias>(p, stream);
        default: return launch<T, UB, kCap | kBias>(p, stream);
        }
    });
}

}  // namespace
}  // namespace attnw
