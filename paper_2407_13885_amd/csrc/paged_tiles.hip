// Attention of new tokens over a paged cache, bf16, blocks of 128 or 256 rows: chunks of prompts.
//
//     O = softmax(s) V over the slots that a token sees (paged_rows.hip), one sweep with a running exponent and sum
//
// A row is one query head of one token; the heads of a kv head share a block with their tokens, so that a block of 128 rows spans few tokens and few of its
// tiles are seen in part.  A wave has 32 rows and all keys pass by, tiles of 32 of them, in LDS for all waves of the workgroup, 16 bytes a lane straight from
// their pages.
//
// What bounds it: the matrix unit, beside a vector unit that makes an exponential for every 4 d operations.
#include "paged_attention.h"

#include <cstdlib>
#include <cstring>

namespace attnw {
namespace {

constexpr int kIds = 1024;                        // page ids kept on chip at a time

template <int UB> struct TilesCfg {
    static constexpr int NX = UB <= 5 ? 2 : 1;    // blocks of 16 rows of a wave
    static constexpr int NW = UB <= 5 ? 4 : 8;    // waves
    static constexpr int ROWS = 16 * NX * NW, UNIT = 128;
    static constexpr int DB = UB * 64, CPR = UB * 4, TILE = 32 * DB, XFERS = TILE / 1024, XW = (XFERS + NW - 1) / NW;
    static constexpr int COLS = DB / 2, CB = COLS / 16;
    static constexpr int RING = 4;                // tiles of K, and of V, on chip
    static constexpr int LDS = 2 * RING * TILE + kIds * 4;
    static constexpr int PER_CU = NW == 4 && LDS <= 80 * 1024 ? 2 : 1;
    static_assert(2 * RING * TILE <= kDirectLds, "reach of direct transfers");
};

template <int UB, bool GENERAL, int THREADS = 64 * TilesCfg<UB>::NW, int BLOCKS = TilesCfg<UB>::NW == 4 ? 2 : 1>
__global__ __launch_bounds__(THREADS, BLOCKS)
void paged_tiles_kernel(AttendArgs a)
{
    using C = TilesCfg<UB>;
    using L = RowLayout<UB>;
    constexpr int NW = C::NW, DB = C::DB, CPR = C::CPR, TILE = C::TILE, XFERS = C::XFERS, XW = C::XW, CB = C::CB, RING = C::RING, G = UB, NX = C::NX;
    __shared__ __align__(1024) char lds[C::LDS];
    char* const k_lds = lds;
    char* const v_lds = lds + RING * TILE;
    int32_t* const ids = reinterpret_cast<int32_t*>(lds + 2 * RING * TILE);

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, l16 = lane & 15, quarter = lane >> 4;
    const uint32_t k_at = lds_offset_of(k_lds), v_at = lds_offset_of(v_lds);
    const int rb = a.cache.row_bytes;

    const Counted count{a};
    const int64_t total = plan_total(a.cache.batch, lane, count);
    const int64_t per = places_each(a.plan, total);
    const int64_t w = xcd_contiguous_block_id(blockIdx.x, gridDim.x);
    int64_t at = w * per;
    const int64_t end = at + per < total ? at + per : total;
    if (at >= end) return;
    int32_t b;
    int64_t before;
    plan_find(a.cache.batch, lane, at, count, b, before);

    if (rb < DB) {                                // (columns that no transfer touches)
        for (int i = threadIdx.x; i < 2 * RING * TILE / 16; i += 64 * NW) *reinterpret_cast<u32x4*>(lds + i * 16) = u32x4{0u, 0u, 0u, 0u};
    }
    // A score as exponent of 2: c times the product (a negative scale negates Q), or by the map.
    const float c = GENERAL ? 1.0f : fabsf(a.rule.scale) * kLog2e;
    const uint32_t sign_flip = !GENERAL && a.rule.scale < 0.0f ? Mma<uint16_t>::kSignMask : 0u;
    const ScoreMap<false, false> plain(a.rule);
    const ScoreMap<true, false> capped(a.rule);

    // ---- per-lane places of the operand fragments ------------------------------------------------------------------------
    const char* const krow = k_lds + l16 * DB;
    constexpr int KPERIOD = UB % 4 == 0 ? 4 : UB % 4 == 2 ? 2 : 1, VPERIOD = L::V16PERIOD;
    int koff[KPERIOD];
#pragma unroll
    for (int g = 0; g < KPERIOD; ++g) koff[g] = ((4 * g + quarter) ^ L::k_chunk(l16)) * 16;
    // keys 16 (f % 2) .. + 15 x columns 32 (f / 2) .. + 31 (8 a lane)
    auto k_frag = [&](int buf, int f) __attribute__((always_inline)) {
        const int g = f / 2;
        return *reinterpret_cast<const u32x4*>(krow + buf * TILE + (f % 2) * 16 * DB + (g / KPERIOD) * KPERIOD * 64 + koff[g % KPERIOD]);
    };
    const int vkey = 4 * quarter + (l16 >> 2);    // a lane's row of the 16 keys that it reads
    const char* const vrow = v_lds + vkey * DB + (lane & 3) * 8;
    int voff[VPERIOD];
#pragma unroll
    for (int x = 0; x < VPERIOD; ++x) voff[x] = (x ^ L::v16_block(vkey)) * 32;
    // 16 columns x 32 keys: of a lane keys 4 quarter .. + 3 and 16 more than these, as its weights
    auto v_frag = [&](int buf, int x) __attribute__((always_inline)) {
        const char* p = vrow + buf * TILE + (x / VPERIOD) * VPERIOD * 32 + voff[x % VPERIOD];
        return u32x4_of(lds_read_tr16(p), lds_read_tr16(p + 16 * DB));
    };

    bool first_segment = true;
    for (; at < end && b < a.cache.batch; first_segment = false) {
        const Sequence seq = sequence_at(a.cache, a.starts, a.tokens, b);
        const int32_t prefix = a.rule.prefix ? max(0, min(a.rule.prefix[b], seq.length)) : 0;
        const SequencePlan plan = sequence_plan(a.plan, seq, prefix, a.rule.window);
        const int64_t in_head = (int64_t)plan.blocks * plan.units, here = at - before;
        if (here >= in_head * a.cache.kv_heads) {
            before += in_head * a.cache.kv_heads;
            ++b;
            continue;
        }
        const int kv_head = (int)(here / in_head);
        const int64_t rest = here - kv_head * in_head;
        const int block = (int)(rest / plan.units);
        const int v0 = (int)(rest - (int64_t)block * plan.units);
        const int v1 = (int)min((int64_t)plan.units, v0 + (end - at));
        at += v1 - v0;

        // ---- the rows of the block ------------------------------------------------------------------------------------------------
        const int64_t row0 = (int64_t)block * C::ROWS;
        const int rows = (int)min((int64_t)C::ROWS, (int64_t)seq.tokens * a.group - row0);
        const int base = seq.length - seq.tokens;              // slot of the first new token
        const int first = base + (int)(row0 / a.group), last = base + (int)((row0 + rows - 1) / a.group);
        const bool active = wave * 16 * NX < rows;
        int query[NX];
        float slope[NX];
        u32x4 qf[NX][G];
#pragma unroll
        for (int x = 0; x < NX; ++x) {
            const int64_t row = row0 + min(wave * 16 * NX + 16 * x + l16, rows - 1);
            const int token = (int)(row / a.group), head = kv_head * a.group + (int)(row - (int64_t)token * a.group);
            query[x] = base + token;
            slope[x] = GENERAL && a.rule.slopes ? a.rule.slopes[head] * kLog2e : 0.0f;
            const char* q = a.Q + (int64_t)(seq.first + token) * a.q_stride + (int64_t)head * rb;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const int ch = 4 * g + quarter;
                qf[x][g] = ch * 16 < rb ? *reinterpret_cast<const u32x4*>(q + ch * 16) ^ sign_flip : u32x4{0u, 0u, 0u, 0u};
            }
        }
        f32x4 oacc[CB][NX];                        // columns 16 i + 4 quarter .. + 3 of rows l16, 16 + l16
#pragma unroll
        for (int i = 0; i < CB; ++i)
#pragma unroll
            for (int x = 0; x < NX; ++x) oacc[i][x] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        // the exponent that weights are taken against, the sum of a lane's weights.  (Finite before any score: masked ones are -infinity.)
        float m_run[NX], l_run[NX];
#pragma unroll
        for (int x = 0; x < NX; ++x) m_run[x] = kNegBig, l_run[x] = 0.0f;

        const Span span = visible_span(C::UNIT, first, last, seq.length, prefix, a.rule.window);
        const int units = last < 0 && span.head == 0 ? 0 : span.count();
        const int u0 = (int)((int64_t)v0 * units / plan.units), u1 = (int)((int64_t)v1 * units / plan.units);
        const int seen = min(seq.length, max(prefix, last + 1));
        const int32_t* const pages_of = a.cache.table + (int64_t)b * a.cache.max_pages;

        // a tile out of buffer `buf`, one step after the other
        auto tile_alone = [&](int buf, int key0, int past) __attribute__((always_inline)) {
            float y[NX][8];
            {
                f32x4 s[2][NX];                   // keys 16 k + 4 quarter .. + 3, rows 16 x + l16
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int x = 0; x < NX; ++x) s[k][x] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int f = 0; f < 2 * G; ++f) {
                    const u32x4 kf = k_frag(buf, f);
#pragma unroll
                    for (int x = 0; x < NX; ++x) mma16(s[f % 2][x], kf, qf[x][f / 2]);
                }
#pragma unroll
                for (int x = 0; x < NX; ++x)
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[x][i] = s[i / 4][x][i % 4];
            }
            const int key = key0 + 4 * quarter;
#pragma unroll
            for (int x = 0; x < NX; ++x)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if constexpr (GENERAL) {
                        y[x][i] = a.rule.cap > 0.0f ? capped(y[x][i]) : plain(y[x][i]);
                        y[x][i] -= slope[x] * (float)abs(query[x] - (key + 16 * (i / 4) + i % 4));
                    } else {
                        y[x][i] *= c;
                    }
                }
            const bool whole = key0 + 32 <= past && ((key0 + 31 <= first && key0 > last - a.rule.window) || key0 + 32 <= prefix);
            if (!whole) {
#pragma unroll
                for (int x = 0; x < NX; ++x)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int j = key + 16 * (i / 4) + i % 4;
                        if (j >= past || ((uint32_t)(query[x] - j) >= (uint32_t)a.rule.window && j >= prefix)) y[x][i] = -__builtin_inff();
                    }
            }
            float p[NX][8];
            u32x4 pw[NX];
#pragma unroll
            for (int x = 0; x < NX; ++x) {
                const float top = fmaxf(max3(max3(y[x][0], y[x][1], y[x][2]), max3(y[x][3], y[x][4], y[x][5]), y[x][6]), y[x][7]);
                if (__builtin_amdgcn_ballot_w64(top > m_run[x]) != 0) {
                    const float m = fmaxf(m_run[x], quarter_wave_max(top)), alpha = fast_exp2(m_run[x] - m);
                    l_run[x] *= alpha;
#pragma unroll
                    for (int i = 0; i < CB; ++i) oacc[i][x] *= alpha;
                    m_run[x] = m;
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    p[x][i] = fast_exp2(y[x][i] - m_run[x]);
                    l_run[x] += p[x][i];
                }
                pw[x] = u32x4{pack_bf16x2(p[x][0], p[x][1]), pack_bf16x2(p[x][2], p[x][3]), pack_bf16x2(p[x][4], p[x][5]), pack_bf16x2(p[x][6], p[x][7])};
            }
            if (!whole) {
                // (a value that is no number must not reach the rows that do not see it: paged_rows.hip)
                uint32_t bad = 0;
#pragma unroll
                for (int i = 0; i < CB; ++i) bad |= any_lost<uint16_t>(v_frag(buf, i));
                if (__builtin_amdgcn_ballot_w64(bad != 0) != 0) {
                    u32x4 sw[NX];
#pragma unroll
                    for (int x = 0; x < NX; ++x) {
                        float saw[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) saw[i] = y[x][i] == -__builtin_inff() ? 0.0f : 1.0f;
                        sw[x] = u32x4{pack_bf16x2(saw[0], saw[1]), pack_bf16x2(saw[2], saw[3]), pack_bf16x2(saw[4], saw[5]), pack_bf16x2(saw[6], saw[7])};
                    }
#pragma unroll
                    for (int i = 0; i < CB; ++i) {
                        const u32x4 v = v_frag(buf, i), lost = lost_as_one<uint16_t>(v), rest_of = without_lost<uint16_t>(v);
#pragma unroll
                        for (int x = 0; x < NX; ++x) {
                            f32x4 hits = {0.0f, 0.0f, 0.0f, 0.0f};
                            mma16(hits, lost, sw[x]);
                            mma16(oacc[i][x], rest_of, pw[x]);
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                if (hits[r] > 0.0f) oacc[i][x][r] = __builtin_nanf("");
                        }
                    }
                    return;
                }
            }
#pragma unroll
            for (int i = 0; i < CB; ++i) {
                const u32x4 v = v_frag(buf, i);
#pragma unroll
                for (int x = 0; x < NX; ++x) mma16(oacc[i][x], v, pw[x]);
            }
        };

        // keys from .. to - 1, which begin a place
        auto sweep = [&](int from, int to) __attribute__((always_inline)) {
            const int64_t most = max((int64_t)C::UNIT, min((int64_t)(kIds - 1) * a.cache.page.d, (int64_t)1 << 30) / C::UNIT * C::UNIT);
            for (int k0 = from; k0 < to;) {
                const int k1 = (int)min((int64_t)to, k0 + most);
                const int p0 = quotient(k0, a.cache.page), p1 = quotient(k1 - 1, a.cache.page);
                __syncthreads();                  // (the ids, and the tiles, of what was before have been read)
                for (int p = p0 + threadIdx.x; p <= p1; p += 64 * NW) ids[p - p0] = max(0, min(pages_of[p], a.cache.pages - 1));
                wait_vmem();
                __syncthreads();
                const int t0 = k0 / 32, t1 = (k1 + 31) / 32;
                auto issue = [&](int t) __attribute__((always_inline)) {
                    const int buf = t & (RING - 1);
#pragma unroll
                    for (int j = 0; j < XW; ++j) {
                        if (XFERS % NW != 0 && wave + NW * j >= XFERS) break;
                        const int x = (wave + NW * j) * 64 + lane, key = x / CPR, ch = x - key * CPR;
                        const int slot = min(t * 32 + key, k1 - 1);   // (past the end the last)
                        const uint32_t p = quotient(slot, a.cache.page);
                        const int64_t off = (int64_t)((uint64_t)(uint32_t)ids[p - p0] * a.cache.page_bytes) +
                                            (uint32_t)(slot - (int)(p * a.cache.page.d)) * (uint32_t)rb + (uint32_t)kv_head * a.cache.head_bytes;
                        const int kc = (ch ^ L::k_chunk(key)) * 16, vc = (ch ^ (L::v16_block(key) * 2)) * 16;
                        if (kc < rb) dma16_untracked(a.cache.K + off + kc, k_at + buf * TILE + (wave + NW * j) * 1024);
                        if (vc < rb) dma16_untracked(a.cache.V + off + vc, v_at + buf * TILE + (wave + NW * j) * 1024);
                    }
                };
                issue(t0);
                if (t0 + 1 < t1) issue(t0 + 1);
#pragma clang loop unroll(disable)
                for (int t = t0; t < t1; ++t) {
                    if (t % 2 == 0) {             // (t0 is even)
                        wait_vmem();
                        __syncthreads();          // two tiles are there, and nobody reads the two before them any more
                        if (t + 2 < t1) issue(t + 2);
                        if (t + 3 < t1) issue(t + 3);
                    }
                    if (active) tile_alone(t & (RING - 1), t * 32, k1);
                }
                k0 = k1;
            }
        };
#pragma clang loop unroll(disable)
        for (int part = 0; part < 2; ++part) {    // of the prefix, of what is near
            const int f = part == 0 ? u0 : max(u0, span.head), t = part == 0 ? min(u1, span.head) : u1;
            if (f < t) sweep(span.unit(f) * C::UNIT, min(seen, (span.unit(t - 1) + 1) * C::UNIT));
        }

        // ---- normalise, round once, store; or leave sums and exponents to the join --------------------------------------------------------
        const bool complete = v0 == 0 && v1 == plan.units;
        float* const out = a.partial + (2 * w + (first_segment ? 0 : 1)) * (int64_t)(C::ROWS * (C::COLS + 2));
        if (active) {
#pragma unroll
            for (int x = 0; x < NX; ++x) {
                const float l = quarter_wave_sum(l_run[x]);
                const int r = wave * 16 * NX + 16 * x + l16;
                if (r >= rows) continue;
                if (complete) {
                    const int64_t row = row0 + r;
                    const int token = (int)(row / a.group), head = kv_head * a.group + (int)(row - (int64_t)token * a.group);
                    const int64_t o = (int64_t)(seq.first + token) * a.heads + head;
#pragma unroll
                    for (int i = 0; i < CB; ++i) store_output<uint16_t>(a.O, o, rb, 16 * i + 4 * quarter, oacc[i][x], l);
                    if (quarter == 0 && a.lse) a.lse[o] = log_sum(m_run[x], l);
                } else {
#pragma unroll
                    for (int i = 0; i < CB; ++i) *reinterpret_cast<f32x4*>(out + r * C::COLS + 16 * i + 4 * quarter) = oacc[i][x];
                    if (quarter == 0) {
                        out[C::ROWS * C::COLS + 2 * r] = m_run[x];
                        out[C::ROWS * C::COLS + 2 * r + 1] = l;
                    }
                }
            }
        }
    }
}

template <int UB> PlanShape plan_of(const PagedArgs& p)
{
    using C = TilesCfg<UB>;
    return {C::ROWS, C::UNIT, (int32_t)(p.heads / p.cache.kv_heads), (compute_units() * C::PER_CU + 7) & ~7, 1};
}

template <int UB> hipError_t launch(const PagedArgs& p, hipStream_t stream)
{
    using C = TilesCfg<UB>;
    const AttendArgs a = attend_args(p, plan_of<UB>(p), 2);
    if (p.rule.cap > 0.0f || p.rule.slopes) paged_tiles_kernel<UB, true><<<a.plan.workgroups, 64 * C::NW, 0, stream>>>(a);
    else paged_tiles_kernel<UB, false><<<a.plan.workgroups, 64 * C::NW, 0, stream>>>(a);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : launch_join<uint16_t>(a, C::COLS, stream);
}

template <typename F> auto by_row(int row_bytes, F&& f)
{
    switch ((row_bytes + 63) / 64) {
    case 1: return f(IC<1>{});
    case 2: return f(IC<2>{});
    case 3: return f(IC<3>{});
    case 4: return f(IC<4>{});
    case 5: return f(IC<5>{});
    case 6: return f(IC<6>{});
    default: return f(IC<8>{});
    }
}

}  // namespace

bool prefers_paged_tiles(const PagedArgs& p)
{
    if (p.dt != DType::BF16) return false;
    // (ATTNW_PAGED_KERNEL=rows / =tiles: tests and measurements compare the two)
    const char* force = getenv("ATTNW_PAGED_KERNEL");
    if (force && strcmp(force, "rows") == 0) return false;
    if (force && strcmp(force, "tiles") == 0) return true;
    const int64_t rows = p.tokens * (p.heads / p.cache.kv_heads);
    return rows > 48 * (int64_t)p.cache.batch;
}

int64_t paged_tiles_workspace(const PagedArgs& p)
{
    return by_row(p.cache.row_bytes, [&](auto ub) { return partial_bytes(plan_of<decltype(ub)::value>(p), TilesCfg<decltype(ub)::value>::COLS); });
}

hipError_t launch_paged_tiles(const PagedArgs& p, hipStream_t stream)
{
    return by_row(p.cache.row_bytes, [&](auto ub) { return launch<decltype(ub)::value>(p, stream); });
}

}  // namespace attnw
