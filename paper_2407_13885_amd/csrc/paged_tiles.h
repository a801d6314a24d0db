// Attention of new tokens over a paged cache, blocks of 128 rows (fp32: 64): chunks of prompts.
//
//     O = softmax(s) V over the slots that a token sees (paged_rows.h), one sweep with a running exponent and sum
//
// A row is one query head of one token; the heads of a kv head share a block with their tokens, so that a block of 128 rows spans few tokens and few of its
// tiles are seen in part.  A wave has 32 rows (fp32, and beyond d = 160: 16) and all keys pass by, tiles of 32 of them, in LDS for all waves of the workgroup, 16 bytes a lane straight from
// their pages.
//
// What bounds it: the matrix unit, beside a vector unit that makes an exponential for every 4 d operations.  Measured: 2048 tokens over 14336 slots, 32
// heads on 8 of 128, causal, 482 to 514 us (1.07 to 1.0 PFLOP/s); fp32 ragged chunks of d = 80 with bias, window and prefix 48 us.
//
// BYTES: a cache in 8 bits (byte_cache.h).  Two tiles of keys, then two of values, come as they lie in memory; the wave that brought 16 bytes a lane makes bf16 of them, scales
// included, where the other kernels have the rows themselves.  From there on everything is the same; fp32 queries and weights are three bf16 parts each.  The read is
// half, the work of every workgroup a quarter of the vector unit more: the chunk above 505 to 540 us by the card and its clock, beside 486 to 510 over a cache in bf16.  In the
// loop of tiles that all rows see whole the pieces are asked for, read and laid among the steps of the products (in a row: 691 us); places, where keys
// lie, are half as many as elsewhere, for room on chip.  (Up to d = 160.  The pieces are among the steps where blocks of slots are multiples of 16, d = 48, 64, 112, 128, or
// else of 32: the chunk above, one set of inputs, in blocks of 32 / of 16: d = 96 394 / 523 us, 160 839 / 1158.)
#pragma once

#include "paged_attention.h"
#include "byte_cache.h"

namespace attnw {
namespace {

template <typename T, int UB, bool BYTES = false> struct TilesCfg {
    static constexpr bool F32 = sizeof(T) == 4 && !BYTES;      // on chip
    static constexpr int PARTS = sizeof(T) == 4 && BYTES ? 3 : 1;
    static constexpr int NX = !F32 && PARTS == 1 && UB <= 5 ? 2 : 1;         // blocks of 16 rows of a wave
    static constexpr int NW = F32 || (UB <= 5 && PARTS == 1) ? 4 : 8;        // waves (PARTS = 3, with four: 512 tokens over 3584 slots, d = 160 316 instead of 158 us)
    static constexpr int ROWS = 16 * NX * NW, UNIT = F32 ? 64 : 128, KT = F32 ? 16 : 32;   // keys of a tile
    static constexpr int DB = UB * 64, CPR = UB * 4, TILE = KT * DB, XFERS = TILE / 1024, XW = (XFERS + NW - 1) / NW;
    static constexpr int COLS = DB / (F32 ? 4 : 2), CB = COLS / 16;
    static constexpr bool PIPE = NX == 2;         // registers for the scores of two tiles
    static constexpr int RING = 4;                // tiles of K, and of V, on chip
    static constexpr int RAW = BYTES ? TILE : 0, XR = (2 * UB + NW - 1) / NW;   // two tiles in bytes, and their transfers for a wave
    static constexpr int PLACES = BYTES ? kPlaces / 2 : kPlaces;
    static constexpr int LDS = RAW + 2 * RING * TILE + PLACES * 8 + RING * 32;
    static constexpr int PER_CU = NW == 4 && LDS <= 80 * 1024 ? 2 : 1;
    static_assert((BYTES ? RAW : 2 * RING * TILE) <= kDirectLds, "reach of direct transfers");
};

struct ByteAttendArgs : AttendArgs {
    ScalesView scales;
};
template <bool BYTES> struct TilesArgs { using type = AttendArgs; };
template <> struct TilesArgs<true> { using type = ByteAttendArgs; };

// SHORT: by how many bytes a row in memory (of bytes: as bf16) is shorter than on chip (up to d = 160: 0 or 32; beyond, -1: known at run time).
template <typename T, int UB, int SHORT, int MODE, bool UNIFORM, bool BYTES = false, int THREADS = 64 * TilesCfg<T, UB, BYTES>::NW,
          int BLOCKS = TilesCfg<T, UB, BYTES>::NW == 8 || (UB > (TilesCfg<T, UB, BYTES>::F32 ? 8 : 5)) ? 1 : 2>
__global__ __launch_bounds__(THREADS, BLOCKS)
void paged_tiles_kernel(typename TilesArgs<BYTES>::type a, int grain)
{
    using C = TilesCfg<T, UB, BYTES>;
    using L = RowLayout<UB>;
    constexpr int NW = C::NW, DB = C::DB, CPR = C::CPR, TILE = C::TILE, XFERS = C::XFERS, XW = C::XW, CB = C::CB, RING = C::RING, G = UB, NX = C::NX, KT = C::KT, NK = KT / 16;
    constexpr int PARTS = C::PARTS;
    constexpr bool F32 = C::F32;
    typedef std::conditional_t<BYTES, uint16_t, T> E;          // an element on chip
    __shared__ __align__(1024) char lds[C::LDS];
    char* const k_lds = lds + C::RAW;
    char* const v_lds = k_lds + RING * TILE;
    int64_t* const places = reinterpret_cast<int64_t*>(k_lds + 2 * RING * TILE);
    uint32_t* const lost_in = reinterpret_cast<uint32_t*>(k_lds + 2 * RING * TILE + C::PLACES * 8);   // [tile of V][wave]: what is no number there
    if constexpr (UNIFORM) grain = 4;

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, l16 = lane & 15, quarter = lane >> 4;
    const uint32_t k_at = lds_offset_of(k_lds);
    const int rb = SHORT >= 0 ? DB - SHORT : a.cache.row_bytes * (BYTES ? 2 : 1);
    const int qb = PARTS == 3 ? 2 * rb : rb;      // of a row of Q and O

    Walk<C::ROWS> walk(a, lane);
    if (walk.at >= walk.end) return;

    // A score as exponent of 2: c times the product (a negative scale negates Q), or by the map.
    const float c = MODE != kPlain ? 1.0f : fabsf(a.rule.scale) * kLog2e;
    const uint32_t sign_flip = MODE == kPlain && a.rule.scale < 0.0f ? Mma<E>::kSignMask : 0u;
    const ScoreMap<(MODE & kCap) != 0, sizeof(T) == 4> map(a.rule);

    // ---- per-lane places of the operand fragments ------------------------------------------------------------------------
    const char* const krow = k_lds + l16 * DB;
    constexpr int KPERIOD = UB % 4 == 0 ? 4 : UB % 4 == 2 ? 2 : 1, VPERIOD = L::V16PERIOD;
    int koff[KPERIOD];
#pragma unroll
    for (int g = 0; g < KPERIOD; ++g) koff[g] = ((4 * g + quarter) ^ L::k_chunk(l16)) * 16;
    // keys 16 (f % NK) .. + 15 x 64 bytes of their rows (16 a lane)
    auto k_frag = [&](int buf, int f) __attribute__((always_inline)) {
        const int g = f / NK;
        return *reinterpret_cast<const u32x4*>(krow + buf * TILE + (f % NK) * 16 * DB + (g / KPERIOD) * KPERIOD * 64 + koff[g % KPERIOD]);
    };
    const int vkey = 4 * quarter + (l16 >> 2);    // a lane's row of the 16 keys that it reads
    const char* const vrow = v_lds + vkey * DB + (lane & 3) * 8;
    int voff[VPERIOD];
#pragma unroll
    for (int x = 0; x < VPERIOD; ++x) voff[x] = (x ^ L::v16_block(vkey)) * 32;
    // 16 columns x 32 keys: of a lane keys 4 quarter .. + 3 and 16 more than these, as its weights
    // (fp32: 16 columns, of a lane its column of keys 4 quarter .. + 3)
    auto v_frag = [&](int buf, int x) __attribute__((always_inline)) {
        if constexpr (F32) {
            const int turn = UB % 4 == 0 ? quarter & 3 : UB % 4 == 2 ? quarter & 1 : 0;
            const char* p = v_lds + buf * TILE + 4 * quarter * DB + (x ^ turn) * 64 + l16 * 4;
            return u32x4{*reinterpret_cast<const uint32_t*>(p), *reinterpret_cast<const uint32_t*>(p + DB), *reinterpret_cast<const uint32_t*>(p + 2 * DB),
                         *reinterpret_cast<const uint32_t*>(p + 3 * DB)};
        } else {
            const char* p = vrow + buf * TILE + (x / VPERIOD) * VPERIOD * 32 + voff[x % VPERIOD];
            return u32x4_of(lds_read_tr16(p), lds_read_tr16(p + 16 * DB));
        }
    };
    typedef std::conditional_t<PARTS == 1, u32x4, Parts<PARTS>> Operand;
    auto multiply = [&](f32x4& acc, const u32x4& x, const Operand& y) __attribute__((always_inline)) {
        if constexpr (PARTS != 1) {
            multiply_parts(acc, x, y);
        } else if constexpr (F32) {
#pragma unroll
            for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x[i]), __uint_as_float(y[i]), acc, 0, 0, 0);
        } else {
            mma16(acc, x, y);
        }
    };
    // where chunk c of key's row lies in its place of V on chip
    auto v_chunk = [&](int key, int c) __attribute__((always_inline)) {
        return F32 ? c ^ ((UB % 4 == 0 ? (key >> 2) & 3 : UB % 4 == 2 ? (key >> 2) & 1 : 0) * 4) : c ^ (L::v16_block(key) * 2);
    };

    Segment seg;
    while (walk.next(seg)) {
        const Sequence& seq = seg.seq;
        const int prefix = seg.prefix, kv_head = seg.kv_head, row0 = seg.row0, rows = seg.rows;
        // ---- the rows of the block ------------------------------------------------------------------------------------------------
        const int group = a.group.d, base = seq.length - seq.tokens;              // slot of the first new token
        const int first = base + (int)quotient(row0, a.group), last = base + (int)quotient(row0 + rows - 1, a.group);
        const bool active = wave * 16 * NX < rows;
        const int lane_of_rows = apart(lane), row_of_lane = lane_of_rows & 15, chunk_of_lane = lane_of_rows >> 4 & 3;
        int query[NX];
        float slope[NX];
        Operand qf[NX][G];
#pragma unroll
        for (int x = 0; x < NX; ++x) {
            const int row = row0 + min(wave * 16 * NX + 16 * x + row_of_lane, rows - 1);
            const int token = (int)quotient(row, a.group), head = kv_head * group + row - token * group;
            query[x] = base + token;
            slope[x] = MODE & kBias ? a.rule.slopes[head] * kLog2e : 0.0f;
            const char* q = a.Q + (int64_t)(seq.first + token) * a.q_stride + (int64_t)head * qb;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const int ch = 4 * g + chunk_of_lane;
                if constexpr (PARTS != 1) {       // (zeros behind a row's end: the key has its first chunks there once more, nothing infinite, and NaN where it is NaN anyway)
                    const bool inside = ch * 16 < rb;
                    const f32x4 lo = *reinterpret_cast<const f32x4*>(q + (inside ? ch * 32 : 0)), hi = *reinterpret_cast<const f32x4*>(q + (inside ? ch * 32 + 16 : 0));
                    float y[8];
#pragma unroll
                    for (int i = 0; i < 4; ++i) y[i] = inside ? lo[i] : 0.0f, y[4 + i] = inside ? hi[i] : 0.0f;
                    qf[x][g] = parts_of<PARTS>(y);
#pragma unroll
                    for (int n = 0; n < PARTS; ++n) qf[x][g].of[n] ^= sign_flip;
                } else
                qf[x][g] = (SHORT == 0 ? *reinterpret_cast<const u32x4*>(q + ch * 16) : query_chunk<T>(q, ch, CPR, rb)) ^ sign_flip;
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

        const Span span = visible_span(a.unit_log, first, last, seq.length, prefix, a.rule.window);
        const int units = last < 0 && span.head == 0 ? 0 : span.count();
        const int u0 = walk.share(seg, seg.v0, units), u1 = walk.share(seg, seg.v1, units);
        const int seen = min(seq.length, max(prefix, last + 1));
        const int32_t* const pages_of = a.cache.table + (int64_t)seg.b * a.cache.max_pages;

        // weights as the operand of the second product
        auto operand = [&](const float (&y)[4 * NK]) __attribute__((always_inline)) {
            if constexpr (PARTS != 1) return parts_of<PARTS>(y);
            else if constexpr (F32) return u32x4{__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]), __float_as_uint(y[3])};
            else return u32x4{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7])};
        };
        // a tile out of buffer `buf`, one step after the other
        auto tile_alone = [&](int buf, int key0, int past) __attribute__((always_inline)) {
            float y[NX][4 * NK];
            {
                f32x4 s[NK][NX];                  // keys 16 k + 4 quarter .. + 3, rows 16 x + l16
#pragma unroll
                for (int k = 0; k < NK; ++k)
#pragma unroll
                    for (int x = 0; x < NX; ++x) s[k][x] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int f = 0; f < NK * G; ++f) {
                    const u32x4 kf = k_frag(buf, f);
#pragma unroll
                    for (int x = 0; x < NX; ++x) multiply(s[f % NK][x], kf, qf[x][f / NK]);
                }
#pragma unroll
                for (int x = 0; x < NX; ++x)
#pragma unroll
                    for (int i = 0; i < 4 * NK; ++i) y[x][i] = s[i / 4][x][i % 4];
            }
            const int key = key0 + 4 * quarter;
#pragma unroll
            for (int x = 0; x < NX; ++x) {
                if constexpr (MODE != kPlain) map(y[x]);
#pragma unroll
                for (int i = 0; i < 4 * NK; ++i) {
                    if constexpr (MODE == kPlain) y[x][i] *= c;
                    if constexpr ((MODE & kBias) != 0) y[x][i] -= slope[x] * (float)abs(query[x] - (key + 16 * (i / 4) + i % 4));
                }
            }
            const bool whole = key0 + KT <= past && ((key0 + KT - 1 <= first && key0 > last - a.rule.window) || key0 + KT <= prefix);
            if (!whole) {
#pragma unroll
                for (int x = 0; x < NX; ++x) {
                    const Sight sight(query[x], a.rule, prefix, past);
#pragma unroll
                    for (int i = 0; i < 4 * NK; ++i) y[x][i] = sight.hidden(key + 16 * (i / 4) + i % 4) < 0 ? -__builtin_inff() : y[x][i];
                }
            }
            float p[NX][4 * NK];
            Operand pw[NX];
#pragma unroll
            for (int x = 0; x < NX; ++x) {
                float top = max3(y[x][0], y[x][1], fmaxf(y[x][2], y[x][3]));
                if constexpr (NK == 2) top = max3(top, max3(y[x][4], y[x][5], y[x][6]), y[x][7]);
                if (__builtin_amdgcn_ballot_w64(top > m_run[x]) != 0) {
                    const float m = fmaxf(m_run[x], quarter_wave_max(top)), alpha = fast_exp2(m_run[x] - m);
                    l_run[x] *= alpha;
#pragma unroll
                    for (int i = 0; i < CB; ++i) oacc[i][x] *= alpha;
                    m_run[x] = m;
                }
#pragma unroll
                for (int i = 0; i < 4 * NK; ++i) {
                    p[x][i] = fast_exp2(y[x][i] - m_run[x]);
                    l_run[x] += p[x][i];
                }
                pw[x] = operand(p[x]);
            }
            if (!whole) {
                u32x4 bad = *reinterpret_cast<const u32x4*>(lost_in + buf * 8);
                if constexpr (NW == 8) bad |= *reinterpret_cast<const u32x4*>(lost_in + buf * 8 + 4);
                if (__builtin_amdgcn_readfirstlane(bad[0] | bad[1] | bad[2] | bad[3]) != 0) {   // (lost_part)
                    if constexpr (BYTES) {        // (NaN, whatever the weight)
                        u32x4 so[NX];
#pragma unroll
                        for (int x = 0; x < NX; ++x) {
                            const Sight sight(query[x], a.rule, prefix, past);
                            float some[4 * NK];
#pragma unroll
                            for (int i = 0; i < 4 * NK; ++i) some[i] = sight.hidden(key + 16 * (i / 4) + i % 4) < 0 ? 0.0f : 1.0f;
                            so[x] = parts_of<1>(some).of[0];
                        }
#pragma unroll
                        for (int i = 0; i < CB; ++i) {
                            const u32x4 v = v_frag(buf, i), rest_of = without_lost<E>(v), lost_of = lost_as_one<E, kAny>(v);
#pragma unroll
                            for (int x = 0; x < NX; ++x) {
                                f32x4 lost = {0.0f, 0.0f, 0.0f, 0.0f};
                                mma16(lost, lost_of, so[x]);
                                multiply(oacc[i][x], rest_of, pw[x]);
#pragma unroll
                                for (int r = 0; r < 4; ++r) oacc[i][x][r] = lost[r] > 0.0f ? __builtin_nanf("") : oacc[i][x][r];
                            }
                        }
                        return;
                    } else {
                    u32x4 so[NX], no[NX];
#pragma unroll
                    for (int x = 0; x < NX; ++x) {
                        const Sight sight(query[x], a.rule, prefix, past);
                        float some[4 * NK], none[4 * NK];
#pragma unroll
                        for (int i = 0; i < 4 * NK; ++i) {
                            const bool hidden = sight.hidden(key + 16 * (i / 4) + i % 4) < 0;
                            const uint32_t weight = F32 ? pw[x][i % 4] : i % 2 ? pw[x][i / 2 % 4] >> 16 : pw[x][i / 2 % 4] & 0xffffu;   // (as it is multiplied)
                            some[i] = hidden || weight == 0 ? 0.0f : 1.0f;
                            none[i] = hidden || weight != 0 ? 0.0f : 1.0f;
                        }
                        so[x] = operand(some);
                        no[x] = operand(none);
                    }
#pragma unroll
                    for (int i = 0; i < CB; ++i) {
                        const u32x4 v = v_frag(buf, i), rest_of = without_lost<T>(v);
#pragma unroll
                        for (int x = 0; x < NX; ++x) {
                            multiply(oacc[i][x], rest_of, pw[x]);
                            oacc[i][x] += lost_part<T>(v, so[x], no[x], multiply);
                        }
                    }
                    return;
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < CB; ++i) {
                const u32x4 v = v_frag(buf, i);
#pragma unroll
                for (int x = 0; x < NX; ++x) multiply(oacc[i][x], v, pw[x]);
            }
        };

        // ---- a cache in 8 bits: two tiles of K or V on their way.  A wave brings pieces of 1 KiB, as many as its lanes, and makes bf16 of what it brought itself --------
        // tiles tile, tile + 1 (of 32 keys from key 0 on; past `last` that one), slots from k0 on in `places`, past k1 the last
        auto bring = [&](bool v, int tile, int last_tile, int k0, int k1) __attribute__((always_inline)) {
            if constexpr (BYTES) {
                const int lane_here = apart(lane), wave_here = apart_uniform(wave);
                const char* const from = v ? a.cache.V : a.cache.K;
#pragma unroll
                for (int j = 0; j < C::XR; ++j) {
                    const int y = wave_here + NW * j;
                    if (2 * UB % NW != 0 && y >= 2 * UB) continue;
                    const int x = (y >= UB ? y - UB : y) * 64 + lane_here, key = x / (2 * UB), at = (x - key * (2 * UB)) * 16;
                    const int slot = min(min(tile + (y >= UB ? 1 : 0), last_tile) * KT + key, k1 - 1) - k0;
                    dma16_untracked(from + place_offset(places[slot >> grain]) + (slot & ((1 << grain) - 1)) * (rb / 2) + (SHORT == 0 || at < rb / 2 ? at : at - rb / 2),
                                    (uint32_t)uniform((int)(k_at - C::RAW + y * 1024)));
                }
            }
        };
        // the same two, which have arrived, into the ring; of V also whether something is no number
        auto settle = [&](bool v, int tile, int last_tile, int k0, int k1, int ring0, auto lookc) __attribute__((always_inline)) {
            constexpr bool LOOK = decltype(lookc)::value != 0;
            if constexpr (BYTES) {
                const int lane_here = apart(lane), wave_here = apart_uniform(wave);
                uint32_t bad[2] = {0, 0};
#pragma unroll
                for (int j = 0; j < C::XR; ++j) {
                    const int y = wave_here + NW * j;
                    if (2 * UB % NW != 0 && y >= 2 * UB) continue;
                    const int second = y >= UB ? 1 : 0, x = (y - second * UB) * 64 + lane_here, key = x / (2 * UB), c = (x - key * (2 * UB)) * 2;
                    const int slot = min(min(tile + second, last_tile) * KT + key, k1 - 1) - k0;
                    const uint32_t high = reinterpret_cast<const uint32_t*>(places)[2 * (slot >> grain) + 1];
                    const u32x4 w = *reinterpret_cast<const u32x4*>(lds + y * 1024 + lane_here * 16);
                    const float scale = v ? value_scale(high) : key_scale(high);
                    const u32x4 lo = bf16_of(w[0], w[1], scale), hi = bf16_of(w[2], w[3], scale);
                    char* const row = (v ? v_lds : k_lds) + ((ring0 + second) & (RING - 1)) * TILE + key * DB;
                    *reinterpret_cast<u32x4*>(row + (v ? v_chunk(key, c) : c ^ L::k_chunk(key)) * 16) = lo;
                    *reinterpret_cast<u32x4*>(row + (v ? v_chunk(key, c + 1) : (c + 1) ^ L::k_chunk(key)) * 16) = hi;
                    if constexpr (LOOK)
                        if (v) bad[second] |= any_nan(w[0]) | any_nan(w[1]) | any_nan(w[2]) | any_nan(w[3]);
                }
                if (LOOK && v) {
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const uint32_t some = __builtin_amdgcn_ballot_w64(bad[k] != 0) != 0 ? 1u : 0u;
                        if (lane_here == 0) lost_in[((ring0 + k) & (RING - 1)) * 8 + wave_here] = some;
                    }
                }
                wait_lds();                       // (what has been read may be brought over)
            }
        };

        // Tiles wa .. wb - 1 (six at least), all rows seeing all of them: in the time of tile t the vector unit makes its weights while the matrix unit makes
        // the output of tile t - 1 and the scores of tile t + 1 (attention_pipe.hip says why).  One barrier for two tiles.
        auto run_piped = [&](int wa, int wb, int k0) __attribute__((always_inline)) {
            if constexpr (C::PIPE) {
            const int n_tiles = wb - wa, wave_here = apart_uniform(wave), k_here = apart_uniform((int)k_at), v_here = k_here + RING * TILE;
            // ---- transfers.  UNIFORM: the keys of one lie in one page, its place a number of the wave -----------------------------------------
            // (The places of 32 tiles wait in a lane each.  One transfer's keys are among 16 of a tile; where rows are no power of two they are all in one page.)
            constexpr bool HALVES = 64 % CPR == 0;
            constexpr int OFFS = UB == 4 ? 1 : XW;             // (the keys of transfers j and j + 1 of d = 128 are 16 apart)
            int64_t place = 0;
            int place_base = 0;
            int lane_off[2][OFFS];
            const int lane_here = apart(lane);
            if constexpr (UNIFORM) {
#pragma unroll
                for (int v = 0; v < 2; ++v)
#pragma unroll
                    for (int j = 0; j < OFFS; ++j) {
                        const int x = (wave_here + NW * j) * 64 + lane_here, key = x / CPR;
                        const int ch = (v ? v_chunk(key, x - key * CPR) : (x - key * CPR) ^ L::k_chunk(key)) * 16;
                        lane_off[v][j] = (HALVES ? key & 15 : key) * rb + (SHORT == 0 ? ch : chunk_in_row(ch, rb));
                    }
            }
            auto look_up = [&](int t) __attribute__((always_inline)) {   // for the requests from tile t on, 15 tiles at least
                if constexpr (UNIFORM) {
                    place_base = 2 * t;
                    place = places[((wa * 32 - k0) >> 4) + min(2 * t + lane_here, 2 * n_tiles - 1)];
                }
            };
            auto transfer = [&](int t, int j, int i) __attribute__((always_inline)) {   // i: which of the four tiles of a pair's requests
                if (XFERS % NW != 0 && wave_here + NW * j >= XFERS) return;
                const bool v = i >= 2;
                const int ahead = t + (i < 2 ? 4 + i : i - 1), tile = min(ahead, n_tiles - 1);
                const uint32_t to = uniform((int)((v ? v_here : k_here) + (ahead & (RING - 1)) * TILE + (wave_here + NW * j) * 1024));
                const char* const where = v ? a.cache.V : a.cache.K;
                if constexpr (UNIFORM) {
                    const int half = HALVES ? ((wave_here + NW * j) * 64 / CPR) >> 4 : 0, from = 2 * tile + half - place_base;
                    const int64_t off = (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)place, from) |
                                        (int64_t)__builtin_amdgcn_readlane((int)(place >> 32), from) << 32;
                    dma16_untracked(where + off, (uint32_t)lane_off[v][j % OFFS], to);
                } else {
                    const int x = (wave_here + NW * j) * 64 + lane_here, key = x / CPR;
                    const int ch = (v ? v_chunk(key, x - key * CPR) : (x - key * CPR) ^ L::k_chunk(key)) * 16;
                    const int slot = (wa + tile) * 32 + key - k0;
                    const char* src = where + places[slot >> grain] + (slot & ((1 << grain) - 1)) * rb + (SHORT == 0 ? ch : chunk_in_row(ch, rb));   // (behind a row's end: paged_rows.h)
                    dma16_untracked(src, to);
                }
            };
            auto request = [&](int t, int i) __attribute__((always_inline)) {
#pragma unroll
                for (int j = 0; j < XW; ++j) transfer(t, j, i);
            };
            auto end_of_pair = [&]() __attribute__((always_inline)) {
                wait_vmem();
                __syncthreads();                  // (and the wave's fragments have left the buffers)
            };
            // (bytes: K of tiles t + 4 and t + 5 come while tile t is made, t even, V of t + 1 and t + 2 while t + 1 is)
            auto bring_pair = [&](bool v, int t) __attribute__((always_inline)) { bring(v, wa + t, wb - 1, k0, wb * 32); };
            auto settle_pair = [&](bool v, int t) __attribute__((always_inline)) {
                arrived<0>();
                settle(v, wa + t, wb - 1, k0, wb * 32, t & (RING - 1), IC<0>{});   // (all rows see all of it: what is no number goes its way)
            };
            // UNIFORM: where a piece comes from and what its scale is are numbers of the wave, and a lane's places within it do not change
            constexpr bool BY16 = UB == 2 || UB == 4;          // (a piece's keys are among 16; else they are any of a tile's)
            constexpr int BYTE_OFFS = BYTES ? (UB == 4 ? 1 : C::XR) : 1;
            int byte_off[BYTE_OFFS], k_to[BYTE_OFFS], v_to[BYTE_OFFS];
            float byte_scale[C::XR];
            u32x4 piece[C::XR];
            if constexpr (BYTES && UNIFORM) {
#pragma unroll
                for (int j = 0; j < BYTE_OFFS; ++j) {
                    const int y = wave_here + NW * j, x = (y >= UB ? y - UB : y) % UB * 64 + lane_here, key = x / (2 * UB), c = (x - key * (2 * UB)) * 2;
                    byte_off[j] = (BY16 ? key & 15 : key) * (rb / 2) + (SHORT == 0 || c * 8 < rb / 2 ? c * 8 : c * 8 - rb / 2);
                    k_to[j] = key * DB + (c ^ L::k_chunk(key)) * 16;
                    v_to[j] = key * DB + v_chunk(key, c) * 16;
                }
            }
            auto bring_piece = [&](bool v, int t, int j) __attribute__((always_inline)) {
                const int y = wave_here + NW * j, second = y >= UB ? 1 : 0;
                if (2 * UB % NW != 0 && y >= 2 * UB) return;
                const int half = BY16 ? ((y - second * UB) * 64 / (2 * UB)) >> 4 : 0, from = 2 * min(t + second, n_tiles - 1) + half - place_base;
                const uint32_t high = (uint32_t)__builtin_amdgcn_readlane((int)(place >> 32), from);
                const int64_t off = (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)place, from) | (int64_t)(high & 0xffffu) << 32;
                byte_scale[j] = v ? value_scale(high) : key_scale(high);
                dma16_untracked((v ? a.cache.V : a.cache.K) + off, (uint32_t)byte_off[j % BYTE_OFFS], (uint32_t)uniform((int)(k_here - C::RAW + y * 1024)));
            };
            auto read_piece = [&](int j) __attribute__((always_inline)) {
                const int y = wave_here + NW * j;
                if (2 * UB % NW != 0 && y >= 2 * UB) return;
                piece[j] = *reinterpret_cast<const u32x4*>(lds + y * 1024 + lane_here * 16);
            };
            auto lay_piece = [&](bool v, int ring0, int j) __attribute__((always_inline)) {
                const int y = wave_here + NW * j, second = y >= UB ? 1 : 0;
                if (2 * UB % NW != 0 && y >= 2 * UB) return;
                const u32x4 lo = bf16_of(piece[j][0], piece[j][1], byte_scale[j]), hi = bf16_of(piece[j][2], piece[j][3], byte_scale[j]);
                char* const to = (v ? v_lds : k_lds) + ((ring0 + second) & (RING - 1)) * TILE;
                const int at = v ? v_to[j % BYTE_OFFS] : k_to[j % BYTE_OFFS];
                *reinterpret_cast<u32x4*>(to + at) = lo;
                *reinterpret_cast<u32x4*>(to + (v ? at + 16 : at ^ 16)) = hi;   // (chunks of V trade places by twos)
            };
            __syncthreads();                      // (what the ring held has been read)
            if constexpr (BYTES) {
                look_up(0);
#pragma unroll
                for (int i = 0; i < 3; ++i) {     // K of tiles 0 to 3, V of 0 and 1
                    bring_pair(i == 2, i == 1 ? 2 : 0);
                    settle_pair(i == 2, i == 1 ? 2 : 0);
                }
            } else {
            look_up(0);
            request(-4, 0);                       // K of tiles 0, 1
            request(-4, 1);
            request(-2, 0);                       // 2, 3
            request(-2, 1);
            request(-1, 2);                       // V of tile 0
            }
            end_of_pair();
            if (!active) {                        // (a wave without rows only moves tiles)
                __syncthreads();
                if constexpr (BYTES) {
                    for (int t = 0; t < n_tiles - 1; ++t) {
                        if (t % 2 == 0) {
                            bring_pair(false, t + 4);
                            settle_pair(false, t + 4);
                        } else {
                            bring_pair(true, t);
                            settle_pair(true, t);
                            end_of_pair();
                        }
                    }
                    if (n_tiles % 2 == 0) {
                        bring_pair(true, n_tiles - 1);
                        settle_pair(true, n_tiles - 1);
                    }
                    end_of_pair();
                    return;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) request(0, i);
                for (int t = 1; t < n_tiles - 1; ++t) {
                    if (t % 16 == 0) look_up(t);
                    if (t % 2 == 0) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) request(t, i);
                    } else {
                        end_of_pair();
                    }
                }
                end_of_pair();
                return;
            }
            struct Scores { f32x4 s[2][2]; };     // keys 16 k + 4 quarter .. + 3, rows 16 x + l16
            struct Weights { u32x4 w[2]; };
            constexpr int KF = 2 * G, RV = G == 1 ? 2 : 4;   // fragments of K of a tile; those of V held at a time
            float p[2][8];                        // the weights of the tile before the one whose scores are s
            // scores of tile t as they count: by the rule, as exponents
            auto ruled = [&](Scores& r, int t) __attribute__((always_inline)) {
                if constexpr (MODE != kPlain) {
                    const int key = (wa + t) * 32 + 4 * quarter;
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            float y = map.large(r.s[i / 4][x][i % 4]);
                            if constexpr ((MODE & kBias) != 0) y -= slope[x] * (float)abs(query[x] - (key + 16 * (i / 4) + i % 4));
                            r.s[i / 4][x][i % 4] = y;
                        }
                }
            };
            auto scores = [&](int buf, int t) __attribute__((always_inline)) {
                Scores r;
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int x = 0; x < 2; ++x) r.s[k][x] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int f = 0; f < KF; ++f) {
                    const u32x4 kf = k_frag(buf, f);
                    const int k = f % 2;
                    mma16(r.s[k][k], kf, qf[k][f / 2]);
                    mma16(r.s[k][1 - k], kf, qf[1 - k][f / 2]);
                }
                ruled(r, t);
                return r;
            };
            auto output = [&](int buf, const Weights& pw) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < CB; ++i) {
                    const u32x4 v = v_frag(buf, i);
                    mma16(oacc[i][i & 1], v, pw.w[i & 1]);
                    mma16(oacc[i][1 - (i & 1)], v, pw.w[1 - (i & 1)]);
                }
            };
            auto pack = [&]() __attribute__((always_inline)) {
                Weights pw;
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int i = 0; i < 4; ++i) pw.w[x][i] = pack_bf16x2(p[x][2 * i], p[x][2 * i + 1]);
                return pw;
            };
            auto largest = [&](const Scores& r, int x) __attribute__((always_inline)) {
                return fmaxf(max3(max3(max3(r.s[0][x][0], r.s[0][x][1], r.s[0][x][2]), r.s[0][x][3], r.s[1][x][0]), r.s[1][x][1], r.s[1][x][2]), r.s[1][x][3]);
            };
            // The exponents move where the largest score of some row is far above (or above at all: ahead > far), and with them the weights p and all before them.
            constexpr float kLazy = 6.0f;         // binades that the maximum may run ahead of the exponent
            auto follow = [&](const float (&top)[2], float far, bool weights) __attribute__((always_inline)) {
                const float ahead[2] = {__builtin_fmaf(top[0], c, -m_run[0]), __builtin_fmaf(top[1], c, -m_run[1])};
                if (__builtin_amdgcn_ballot_w64(fmaxf(ahead[0], ahead[1]) > far) == 0) return;
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    if (__builtin_amdgcn_ballot_w64(ahead[x] > far) == 0) continue;
                    const float m = fmaxf(m_run[x], reference_exponent(quarter_wave_max(top[x]), c));
                    const float alpha = fast_exp2(m_run[x] - m);     // exactly 1 for lanes whose exponent stands
                    l_run[x] *= alpha;
#pragma unroll
                    for (int i = 0; i < CB; ++i) oacc[i][x] *= alpha;
                    if (weights) {
#pragma unroll
                        for (int r = 0; r < 8; ++r) p[x][r] *= alpha;
                    }
                    m_run[x] = m;
                }
            };
            Scores s = scores(0, 0), sn = scores(1, 1);
            __syncthreads();
            if constexpr (BYTES) {
                bring_pair(false, 4);
            } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) request(0, i);
            }
            {
                const float top[2] = {fmaxf(largest(s, 0), largest(sn, 0)), fmaxf(largest(s, 1), largest(sn, 1))};
                follow(top, 0.0f, false);
            }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    p[x][r] = fast_exp2(__builtin_fmaf(s.s[r / 4][x][r % 4], c, -m_run[x]));
                    l_run[x] += p[x][r];
                }
            }
            s = sn;
            if constexpr (BYTES) {
                settle_pair(false, 4);
                if constexpr (!UNIFORM) bring_pair(true, 1);
            }
            u32x4 kf[KF], vf[RV];
#pragma unroll
            for (int f = 0; f < KF; ++f) kf[f] = k_frag(2, f);

            // ---- Tile t: its weights, the output of tile t - 1, the scores of tile t + 1 ------------------------------------------------------
            auto tile = [&](int t, auto bufc) __attribute__((always_inline)) {
                constexpr int BUF = decltype(bufc)::value;         // t mod 4
                constexpr int STEPS = 2 * (KF + CB), OPS = 8 + 32 + 16 + (MODE != kPlain ? 0 : 8);
                Weights pw;
                float pn[2][8], sum[2], top[2];
                if constexpr (BYTES && !UNIFORM && BUF % 2 == 0) bring_pair(false, t + 4);
                auto vector_op = [&](auto oc) __attribute__((always_inline)) {
                    constexpr int I = decltype(oc)::value;
                    if constexpr (I < 8) {
                        constexpr int X = I / 4, J = I % 4;
                        pw.w[X][J] = pack_bf16x2(p[X][2 * J], p[X][2 * J + 1]);
                    } else if constexpr (I < 40) {
                        // (f0 f1 e0 f2 e1 .. f15 e14 e15: an exponential does not wait for the product right before it)
                        constexpr int J = I - 8;
                        constexpr bool EXP = J == 31 || (J >= 2 && J % 2 == 0);
                        constexpr int E = J == 31 ? 15 : EXP ? J / 2 - 1 : (J + 1) / 2;
                        constexpr int X = E / 8, R = E % 8;
                        if constexpr (EXP) pn[X][R] = fast_exp2(pn[X][R]);
                        else pn[X][R] = __builtin_fmaf(s.s[R / 4][X][R % 4], c, -m_run[X]);
                    } else if constexpr (I < 56) {
                        constexpr int X = (I - 40) % 2, R = (I - 40) / 2;
                        if constexpr (R == 0) sum[X] = pn[X][0];
                        else sum[X] += pn[X][R];
                        if constexpr (R == 7) l_run[X] += sum[X];
                    } else {
                        constexpr int X = (I - 56) % 2, J = (I - 56) / 2;
                        if constexpr (J == 0) top[X] = max3(sn.s[0][X][0], sn.s[0][X][1], sn.s[0][X][2]);
                        if constexpr (J == 1) top[X] = max3(top[X], sn.s[0][X][3], sn.s[1][X][0]);
                        if constexpr (J == 2) top[X] = max3(top[X], sn.s[1][X][1], sn.s[1][X][2]);
                        if constexpr (J == 3) top[X] = fmaxf(top[X], sn.s[1][X][3]);
                    }
                };
                static_for<STEPS>([&](auto ic) __attribute__((always_inline)) {
                    constexpr int I = decltype(ic)::value, F = I / 2, SECOND = I % 2;
                    if constexpr (F < KF) {
                        constexpr int GR = F / 2, KB = F % 2, X = SECOND ? 1 - KB : KB;
                        if constexpr (GR == 0) sn.s[KB][X] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                        mma16(sn.s[KB][X], kf[F], qf[X][GR]);
                        if constexpr (SECOND && F >= KF - RV) vf[F - (KF - RV)] = v_frag((BUF + 3) % 4, F - (KF - RV));
                    } else {
                        constexpr int B = F - KF, X = SECOND ? 1 - B % 2 : B % 2, NEXT = I - 2 * KF;
                        mma16(oacc[B][X], vf[B % RV], pw.w[X]);
                        if constexpr (SECOND && B + RV < CB) vf[B % RV] = v_frag((BUF + 3) % 4, B + RV);
                        if constexpr (NEXT < KF) kf[NEXT] = k_frag((BUF + 2) % 4, NEXT);      // (in the first of these steps: arrived by the end of the tile)
                    }
                    static_for<(I + 1) * OPS / STEPS - I * OPS / STEPS>([&](auto jc) __attribute__((always_inline)) {
                        vector_op(IC<I * OPS / STEPS + decltype(jc)::value>{});
                    });
                    if constexpr (BYTES && UNIFORM) {          // of K tiles t + 4 and t + 5, or, t odd, of V t and t + 1
                        constexpr bool V = BUF % 2 == 1;
                        constexpr int READ = STEPS * 11 / 16;  // (when they have arrived; at 1/2 530 us, 5/8 525, 11/16 515, later 522 to 526)
                        static_assert(READ + 2 * C::XR < STEPS);
                        if constexpr (I < C::XR) bring_piece(V, V ? t : t + 4, I);
                        if constexpr (I == READ) {
                            arrived<0>();
#pragma unroll
                            for (int j = 0; j < C::XR; ++j) read_piece(j);
                        }
                        if constexpr (I > READ + 1 && (I - READ) % 2 == 0 && I <= READ + 2 * C::XR) lay_piece(V, BUF, (I - READ) / 2 - 1);
                    }
                    // (transfers between the steps: a wave that issues them in a row waits 50 cycles for each)
                    if constexpr (!BYTES && BUF % 2 == 0 && I % 2 == 0 && I / 2 < 4 * XW) transfer(t, I / 2 % XW, I / 2 / XW);
                    __builtin_amdgcn_sched_barrier(0);
                });
                static_assert(2 * CB >= KF && 8 * XW <= STEPS);
                if constexpr (MODE != kPlain) {
                    ruled(sn, t + 1);
                    top[0] = largest(sn, 0);
                    top[1] = largest(sn, 1);
                }
                s = sn;
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int r = 0; r < 8; ++r) p[x][r] = pn[x][r];
                follow(top, kLazy, true);
                if constexpr (BYTES && !UNIFORM) {
                    if constexpr (BUF % 2 == 0) {
                        settle_pair(false, t + 4);
                        bring_pair(true, t + 1);
                    } else {
                        settle_pair(true, t);
                    }
                }
                if constexpr (BUF % 2 == 1) end_of_pair();
            };
            for (int t = 1;;) {
                if (t >= n_tiles - 1) break;
                tile(t++, IC<1>{});
                if (t >= n_tiles - 1) break;
                tile(t++, IC<2>{});
                if (t >= n_tiles - 1) break;
                tile(t++, IC<3>{});
                if (t >= n_tiles - 1) break;
                if (t % 16 == 0) look_up(t);
                tile(t++, IC<0>{});
            }
            if constexpr (BYTES)
                if (n_tiles % 2 == 0) {
                    if constexpr (UNIFORM) bring_pair(true, n_tiles - 1);
                    settle_pair(true, n_tiles - 1);
                }
            end_of_pair();
            // ---- the last two tiles ---------------------------------------------------------------------------------------------------------
            output((n_tiles - 2) & 3, pack());
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    p[x][r] = fast_exp2(__builtin_fmaf(s.s[r / 4][x][r % 4], c, -m_run[x]));
                    l_run[x] += p[x][r];
                }
            output((n_tiles - 1) & 3, pack());
            }
        };

        // keys from .. to - 1, which begin a place
        auto sweep = [&](int from, int to, bool near) __attribute__((always_inline)) {
            const int most = C::PLACES << grain;  // (a whole number of places of the plan)
            for (int k0 = from; k0 < to;) {
                const int k1 = min(to, k0 + most);
                __syncthreads();                  // (the places, and the tiles, of what was before have been read)
                for (int i = threadIdx.x; i < (k1 - k0 + (1 << grain) - 1) >> grain; i += 64 * NW)
                    if constexpr (BYTES) places[i] = slot_place(a.cache, a.scales, pages_of, kv_head, k0 + (i << grain));
                    else places[i] = slot_offset(a.cache, pages_of, kv_head, k0 + (i << grain));
                wait_vmem();
                __syncthreads();
                // a transfer of tile t, by lanes: any pages; slots past the end are read as the last
                auto transfer = [&](const char* from_where, uint32_t to, int t, int j, bool v, int lane_here, int wave_here) __attribute__((always_inline)) {
                    if (XFERS % NW != 0 && wave_here + NW * j >= XFERS) return;
                    const int x = (wave_here + NW * j) * 64 + lane_here, key = x / CPR;
                    const int ch = (v ? v_chunk(key, x - key * CPR) : (x - key * CPR) ^ L::k_chunk(key)) * 16;
                    const int slot = min(t * KT + key, k1 - 1) - k0;
                    const char* src = from_where + places[slot >> grain] + (slot & ((1 << grain) - 1)) * rb + (SHORT == 0 ? ch : chunk_in_row(ch, rb));   // (behind a row's end: paged_rows.h)
                    dma16_untracked(src, to + (wave_here + NW * j) * 1024);
                };
                // tiles ta .. tb - 1 one after the other
                auto run_alone = [&](int ta, int tb) __attribute__((always_inline)) {
                    if constexpr (BYTES) {
                        const int n = tb - ta;
                        auto bring_pair = [&](bool v, int i) __attribute__((always_inline)) { bring(v, ta + i, tb - 1, k0, k1); };
                        auto settle_pair = [&](bool v, int i) __attribute__((always_inline)) {
                            arrived<0>();
                            settle(v, ta + i, tb - 1, k0, k1, i & (RING - 1), IC<1>{});
                        };
                        __syncthreads();
#pragma unroll
                        for (int v = 0; v < 2; ++v) {
                            bring_pair(v, 0);
                            settle_pair(v, 0);
                        }
#pragma clang loop unroll(disable)
                        for (int i = 0; i < n; ++i) {
                            const bool even = i % 2 == 0, more = even ? i + 2 < n : i + 1 < n;
                            if (even) {
                                __syncthreads();  // two tiles are there, and nobody reads the two before them any more
                                if (more) bring_pair(false, i + 2);
                            }
                            if (active) tile_alone(i & (RING - 1), (ta + i) * KT, k1);
                            if (!more) continue;
                            if (even) {
                                settle_pair(false, i + 2);
                                bring_pair(true, i + 2);
                            } else {
                                settle_pair(true, i + 1);
                            }
                        }
                        return;
                    }
                    const int lane_here = apart(lane), wave_here = apart_uniform(wave), k_here = apart_uniform((int)k_at), v_here = k_here + RING * TILE;
                    auto issue = [&](int i) __attribute__((always_inline)) {
#pragma unroll
                        for (int j = 0; j < XW; ++j) {
                            transfer(a.cache.K, uniform((int)(k_here + (i & (RING - 1)) * TILE)), ta + i, j, false, lane_here, wave_here);
                            transfer(a.cache.V, uniform((int)(v_here + (i & (RING - 1)) * TILE)), ta + i, j, true, lane_here, wave_here);
                        }
                    };
                    const int n = tb - ta;
                    __syncthreads();
                    issue(0);
                    if (1 < n) issue(1);
#pragma clang loop unroll(disable)
                    for (int i = 0; i < n; ++i) {
                        if (i % 2 == 0) {
                            arrived<0>();
                            // (what a wave brought of V it looks over itself)
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                const int buf = (i + k) & (RING - 1);
                                uint32_t bad = 0;
#pragma unroll
                                for (int j = 0; j < XW; ++j)
                                    if (XFERS % NW == 0 || wave_here + NW * j < XFERS)
                                        bad |= any_lost<T>(*reinterpret_cast<const u32x4*>(v_lds + buf * TILE + (wave_here + NW * j) * 1024 + lane_here * 16));
                                const uint32_t some = __builtin_amdgcn_ballot_w64(bad != 0) != 0 ? 1u : 0u;
                                if (lane_here == 0) lost_in[buf * 8 + wave_here] = some;
                            }
                            __syncthreads();      // two tiles are there, and nobody reads the two before them any more
                            if (i + 2 < n) issue(i + 2);
                            if (i + 3 < n) issue(i + 3);
                        }
                        if (active) tile_alone(i & (RING - 1), (ta + i) * KT, k1);
                    }
                };
                // Tiles that all rows of the block see whole go through run_piped, those before and behind them, with masks, one by one.  (So do all of a call whose cap is so
                // large that scores go by a series: it would take the registers that run_piped has none of to spare.)
                int f0 = k0 / KT, f1 = (k1 + KT - 1) / KT, w0 = f1, w1 = f1;
                if constexpr (C::PIPE) {
                    if (near) w0 = max(f0, (max(0, last - a.rule.window + 1) + 31) / 32), w1 = min(k1, max(0, first + 1)) / 32;
                    else w0 = f0, w1 = min(k1, prefix) / 32;
                    if (w1 - w0 < 6 || map.series) w0 = w1 = f1;
                }
#pragma clang loop unroll(disable)
                for (int side = 0; side < 2; ++side) {
                    const int ta = side == 0 ? f0 : w1, tb = side == 0 ? w0 : f1;
                    if constexpr (C::PIPE) {
                        if (side == 1 && w0 < w1) run_piped(w0, w1, k0);
                    }
                    if (ta < tb) run_alone(ta, tb);
                }
                k0 = k1;
            }
        };
#pragma clang loop unroll(disable)
        for (int part = 0; part < 2; ++part) {    // of the prefix, of what is near
            const int f = part == 0 ? u0 : max(u0, span.head), t = part == 0 ? min(u1, span.head) : u1;
            if (f < t) sweep(span.unit(f) << a.unit_log, (int)min((int64_t)seen, (int64_t)(span.unit(t - 1) + 1) << a.unit_log), part == 1);
        }

        // ---- normalise, round once, store; or leave sums and exponents to the join --------------------------------------------------------
        const bool complete = seg.slot < 0;
        float* const out = a.partial + max(seg.slot, 0) * (int64_t)(C::ROWS * (C::COLS + 2));
        if (active) {
            const int lane_here = apart(lane), row_of_lane = lane_here & 15, quarter_of_lane = lane_here >> 4 & 3;
#pragma unroll
            for (int x = 0; x < NX; ++x) {
                const float l = quarter_wave_sum(l_run[x]);
                const int r = wave * 16 * NX + 16 * x + row_of_lane;
                if (r >= rows) continue;
                if (complete) {
                    const int row = row0 + r, token = (int)quotient(row, a.group), head = kv_head * group + row - token * group;
                    const int64_t o = (int64_t)(seq.first + token) * a.heads + head;
#pragma unroll
                    for (int i = 0; i < CB; ++i) store_output<T>(a.O, o, qb, 16 * i + 4 * quarter_of_lane, oacc[i][x], l);
                    if (quarter_of_lane == 0 && a.lse) a.lse[o] = log_sum(m_run[x], l);
                } else {
#pragma unroll
                    for (int i = 0; i < CB; ++i) *reinterpret_cast<f32x4*>(out + r * C::COLS + 16 * i + 4 * quarter_of_lane) = oacc[i][x];
                    if (quarter_of_lane == 0) {
                        out[C::ROWS * C::COLS + 2 * r] = m_run[x];
                        out[C::ROWS * C::COLS + 2 * r + 1] = l;
                    }
                }
            }
        }
    }
}

template <typename T, int UB> int byte_workgroups() { return (compute_units() * TilesCfg<T, UB, true>::PER_CU + 7) & ~7; }
template <typename T, int UB> int workgroups() { return (compute_units() * TilesCfg<T, UB>::PER_CU + 7) & ~7; }

template <typename T, int UB, int SHORT, int MODE> hipError_t launch(const PagedArgs& p, hipStream_t stream)
{
    using C = TilesCfg<T, UB>;
    const AttendArgs a = attend_args(p, workgroups<T, UB>(), C::ROWS, C::UNIT, sizeof(T));
    const int page = (int)a.cache.page.d, grain = key_grain(a.cache);
    constexpr bool CAN = C::PIPE;
    if (CAN && page % (64 % C::CPR == 0 ? 16 : 32) == 0) paged_tiles_kernel<T, UB, SHORT, MODE, CAN><<<a.workgroups, 64 * C::NW, 0, stream>>>(a, grain);
    else paged_tiles_kernel<T, UB, SHORT, MODE, false><<<a.workgroups, 64 * C::NW, 0, stream>>>(a, grain);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : launch_join<T>(a, C::ROWS, C::COLS, stream);
}

// The same over a cache in 8 bits: rows of 2 d bytes on chip.
template <typename T, int UB, int SHORT, int MODE> hipError_t launch_bytes(const PagedArgs& p, const ScalesView& scales, hipStream_t stream)
{
    using C = TilesCfg<T, UB, true>;
    ByteAttendArgs a;
    static_cast<AttendArgs&>(a) = attend_args(p, byte_workgroups<T, UB>(), C::ROWS, C::UNIT, sizeof(T));
    a.scales = scales;
    // (16 keys that share a page and scales, or a tile's)
    constexpr bool CAN = C::PIPE;
    if (CAN && scales.block.d % (UB == 2 || UB == 4 ? 16 : 32) == 0) paged_tiles_kernel<T, UB, SHORT, MODE, CAN, true><<<a.workgroups, 64 * C::NW, 0, stream>>>(a, 4);
    else paged_tiles_kernel<T, UB, SHORT, MODE, false, true><<<a.workgroups, 64 * C::NW, 0, stream>>>(a, key_grain(a.cache, scales));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    a.cache.row_bytes *= (int)sizeof(T);          // (of the output)
    return launch_join<T>(a, C::ROWS, C::COLS, stream);
}

template <typename T, typename F> auto by_row(int row_bytes, F&& f)
{
    const int ub = (row_bytes + 63) / 64;
    if (ub <= 1) return f(IC<1>{});
    if (ub <= 2) return f(IC<2>{});
    if (ub <= 3) return f(IC<3>{});
    if (ub <= 4) return f(IC<4>{});
    if (ub <= 5) return f(IC<5>{});
    if (ub <= 6) return f(IC<6>{});
    if constexpr (sizeof(T) == 2) {
        return f(IC<8>{});
    } else {
        if (ub <= 8) return f(IC<8>{});
        if (ub <= 12) return f(IC<12>{});
        return f(IC<16>{});
    }
}

template <typename T, int MODE> hipError_t launch_tiles(const PagedArgs& p, hipStream_t stream)
{
    return by_row<T>(p.cache.row_bytes, [&](auto ubc) {
        constexpr int UB = decltype(ubc)::value;
        if constexpr (sizeof(T) == 4 || UB > 5) return launch<T, UB, -1, MODE>(p, stream);
        else return p.cache.row_bytes == UB * 64 ? launch<T, UB, 0, MODE>(p, stream) : launch<T, UB, 32, MODE>(p, stream);
    });
}

// (fp32: d = 80 and 96, and beyond 128, prefers_byte_tiles says why)
template <typename T, typename F> auto by_byte_row(int row_bytes, F&& f)
{
    if constexpr (sizeof(T) == 4) {
        const int ub = (2 * row_bytes + 63) / 64;
        return ub <= 3 ? f(IC<3>{}) : ub <= 5 ? f(IC<5>{}) : ub <= 6 ? f(IC<6>{}) : f(IC<8>{});
    } else {
        return by_row<T>(2 * row_bytes, f);
    }
}

template <typename T, int MODE> hipError_t launch_byte_tiles(const PagedArgs& p, const ScalesView& scales, hipStream_t stream)
{
    return by_byte_row<T>(p.cache.row_bytes, [&](auto ubc) {
        constexpr int UB = decltype(ubc)::value;
        if constexpr (sizeof(T) == 4 || UB > 5) return launch_bytes<T, UB, -1, MODE>(p, scales, stream);
        else return 2 * p.cache.row_bytes == UB * 64 ? launch_bytes<T, UB, 0, MODE>(p, scales, stream) : launch_bytes<T, UB, 32, MODE>(p, scales, stream);
    });
}

template <typename T> int64_t byte_tiles_workspace(const PagedArgs& p)
{
    return by_byte_row<T>(p.cache.row_bytes, [&](auto ubc) {
        constexpr int UB = decltype(ubc)::value;
        return partial_bytes(byte_workgroups<T, UB>(), TilesCfg<T, UB, true>::ROWS, TilesCfg<T, UB, true>::COLS);
    });
}

template <typename T> int64_t tiles_workspace(const PagedArgs& p)
{
    return by_row<T>(p.cache.row_bytes, [&](auto ubc) {
        constexpr int UB = decltype(ubc)::value;
        return partial_bytes(workgroups<T, UB>(), TilesCfg<T, UB>::ROWS, TilesCfg<T, UB>::COLS);
    });
}

}  // namespace
}  // namespace attnw
