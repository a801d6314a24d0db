// What the slots of a paged cache are worth to new tokens:
//
//     sums[b][kv_head][j] = before[b][kv_head][j] + sum over the new tokens i and the heads of the kv head of exp(s_ij - lse_i),
//
// the weights that attention gave the slot (s and what a token sees as there, lse from there).
//
// A workgroup owns the slots that it sums over: no atomics, K read once, sums in an order that the sizes alone decide.  Chunks: the waves of a workgroup keep
// the same keys in registers and take the rows in turn, 16 at a time, straight from the caches, the next ones on their way; their sums are joined in the end (what
// bounds it are the exponentials, as many as scores: three transcendental instructions each with a cap; two chunks of 1024 tokens over 9216 slots at most, 16 heads of 64 with a
// cap and a window 91 us).  Single tokens and short chunks: the waves hold the rows and have keys of their own, some tiles of which are always on their way into LDS
// (what bounds it is the read of K; one token each over 64 sequences of 16384 slots, 8 kv heads of 128 422 us, 5.1 TB/s).
#include "qk_common.h"
#include "attention_common.h"
#include "paged_common.h"

namespace attnw {
namespace {

struct SumsKernelArgs {
    const char* Q;
    const float *lse, *before;
    float* sums;
    const int32_t* starts;
    int64_t q_stride;                             // bytes
    int32_t tokens, heads;
    FastDiv group;
    CacheView cache;
    RuleView rule;
};

// NK: blocks of 16 keys of a wave.
template <typename T, int UB> struct SumsCfg {
    static constexpr int NW = 4, NK = UB <= 2 ? 4 : UB <= 4 ? (sizeof(T) == 2 ? 4 : 2) : UB <= 8 ? 2 : 1, KEYS = 16 * NK;
    static constexpr int FULL = UB / 2;           // of the groups of 64 bytes, those that rows fill (launch_paged_sums)
};
// Single tokens: KT keys of a wave's tile, RING tiles on chip.
template <typename T, int UB> struct StepCfg {
    static constexpr int KT = sizeof(T) == 4 ? 16 : 32, DB = UB * 64, TILE = KT * DB, XFERS = TILE / 1024, PLACE = TILE + 256;
    static constexpr int NW = TILE > 8192 ? 2 : 4, KEYS = KT * NW;
    static constexpr int FIT = kDirectLds / (NW * PLACE), RING = FIT >= 4 ? 4 : FIT;
    static constexpr int TILES = NW * RING * PLACE, LDS = TILES + kPlaces * 8;
    static constexpr int PER_CU = LDS <= 40 * 1024 ? 4 : LDS <= 80 * 1024 ? 2 : 1;
    static_assert(RING >= 2 && TILES <= kDirectLds && LDS <= 160 * 1024);
};

// The sum over the 16 lanes of a row, in each of them.
__device__ __forceinline__ float sum_of_16(float x)
{
#if defined(__HIP_DEVICE_COMPILE__)
    const auto turned = [&](auto n) __attribute__((always_inline)) {   // of the lane n places on (row_ror)
        return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x120 + decltype(n)::value, 0xf, 0xf, true));
    };
    x += turned(IC<8>{});
    x += turned(IC<4>{});
    x += turned(IC<2>{});
    x += turned(IC<1>{});
#endif
    return x;
}

// 16 rows, of a lane one: rows r .. r + 15 of those of a kv head of a sequence, up to `last`.
template <int UB> struct Rows {
    u32x4 q[UB];
    float lse, slope;
    int query;
};
// TWICE: against keys that have their first chunks once more behind their end (chunk_in_row); else zeros there.
template <typename T, int UB, int MODE, bool TWICE>
__device__ __forceinline__ Rows<UB> fetch_rows(const SumsKernelArgs& a, const Sequence& seq, int kv_head, int rb, int r, int last, int lane)
{
    Rows<UB> x;
    const int group = a.group.d, row = min(r + (lane & 15), last), token = (int)quotient(row, a.group), head = kv_head * group + row - token * group;
    const int64_t at_row = seq.first + token;
    const char* q = a.Q + at_row * a.q_stride + (int64_t)head * rb;
#pragma unroll
    for (int g = 0; g < UB; ++g) {
        const int ch = 4 * g + (lane >> 4);
        if constexpr (TWICE) {
            x.q[g] = query_chunk<T>(q, ch, 4 * UB, rb);
        } else {
            x.q[g] = *reinterpret_cast<const u32x4*>(q + (ch * 16 < rb ? ch * 16 : 0));
            if (ch * 16 >= rb) x.q[g] = u32x4{0u, 0u, 0u, 0u};
        }
    }
    x.lse = a.lse[at_row * a.heads + head];
    x.slope = MODE & kBias ? a.rule.slopes[head] * kLog2e : 0.0f;
    x.query = seq.length - seq.tokens + token;
    return x;
}

// What 16 rows (those from r on that are below r1) give NK blocks of 16 keys, from slot `mine` on: of a lane keys 4 quarter .. + 3 of a block and row l16.
template <typename T, int UB, int MODE, int NK, typename KeyFragment, typename Map>
__device__ __forceinline__ void add_weights(f32x4 (&sum)[NK], const SumsKernelArgs& a, const Sequence& seq, int prefix, int mine, int r, int r1, const Rows<UB>& x,
                                            int lane, KeyFragment&& keys, const Map& map)
{
    const int l16 = lane & 15, quarter = lane >> 4;
    f32x4 acc[NK];
#pragma unroll
    for (int k = 0; k < NK; ++k) acc[k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int g = 0; g < UB; ++g)
#pragma unroll
        for (int k = 0; k < NK; ++k) {
            const u32x4 kf = keys(k, g);
            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    acc[k] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[e]), __uint_as_float(x.q[g][e]), acc[k], 0, 0, 0);
            } else {
                mma16(acc[k], kf, x.q[g]);
            }
        }
    // a row that saw nothing, or that is not there, adds nothing
    const float lse = x.lse == -__builtin_inff() || r + l16 >= r1 ? __builtin_inff() : x.lse * kLog2e;
    // (tokens of the rows: first .. last)
    const int first = __builtin_amdgcn_readlane(x.query, 0), last = __builtin_amdgcn_readlane(x.query, 15);
    const bool whole = mine + 16 * NK <= seq.length && ((mine + 16 * NK - 1 <= first && mine > last - a.rule.window) || mine + 16 * NK <= prefix);
    float y[4 * NK];
#pragma unroll
    for (int i = 0; i < 4 * NK; ++i) y[i] = acc[i / 4][i % 4];
    map(y);
#pragma unroll
    for (int i = 0; i < 4 * NK; ++i) {
        if constexpr ((MODE & kBias) != 0) y[i] -= x.slope * (float)abs(x.query - (mine + 16 * (i / 4) + 4 * quarter + i % 4));
        acc[i / 4][i % 4] = fast_exp2(y[i] - lse);
    }
    if (!whole) {
        const Sight sight(x.query, a.rule, prefix, seq.length);
#pragma unroll
        for (int k = 0; k < NK; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[k][e] = sight.hidden(mine + 16 * k + 4 * quarter + e) < 0 ? 0.0f : acc[k][e];
    }
    const bool nothing = x.lse == -__builtin_inff();
    if (__builtin_amdgcn_ballot_w64(nothing) != 0) {           // (whatever its scores are: NaN is not 0 by now)
#pragma unroll
        for (int k = 0; k < NK; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[k][e] = nothing ? 0.0f : acc[k][e];
    }
#pragma unroll
    for (int k = 0; k < NK; ++k) sum[k] += acc[k];
}

// A workgroup's way through its blocks of KEYS keys: runs of them of one kv head of a sequence, at most as long as there is room on chip for where they are.
template <int KEYS> struct SumsWalk {
    const SumsKernelArgs& a;
    int grain;
    int32_t b, at, end, before;
    struct Run {
        Sequence seq;
        int kv_head, prefix, base, k0, k1, blocks;             // keys k0 .. k1 - 1; base: slot of the first new token
        int64_t row;                                           // of its sums
    };
    __device__ __forceinline__ SumsWalk(const SumsKernelArgs& args, int grain_, int lane) : a(args), grain(grain_)
    {
        const auto count = [&](int i) __attribute__((always_inline)) {
            return (max(0, min(a.cache.lengths[i], a.cache.slots)) + KEYS - 1) / KEYS * a.cache.kv_heads;
        };
        const Deal deal = deal_out(plan_total(a.cache.batch, lane, count), (int32_t)gridDim.x);
        const int w = dealt_workgroup(deal);
        at = end = 0;
        if (w >= deal.workgroups) return;
        at = deal.first(w);
        end = deal.first(w + 1);
        plan_find(a.cache.batch, lane, at, count, b, before);
    }
    // The next run, where its keys are put on chip (all waves of the workgroup take part).
    __device__ __forceinline__ bool next(Run& r, int64_t* places)
    {
        for (;; ++b) {
            if (at >= end || b >= a.cache.batch) return false;
            r.seq = sequence_at(a.cache, a.starts, a.tokens, b);
            const int blocks = (r.seq.length + KEYS - 1) / KEYS, here = at - before;
            if (here >= blocks * a.cache.kv_heads) {
                before += blocks * a.cache.kv_heads;
                continue;
            }
            r.kv_head = uniform((int32_t)((uint32_t)here / (uint32_t)blocks));
            const int block0 = here - r.kv_head * blocks;
            r.blocks = min(min(blocks - block0, end - at), (kPlaces << grain) / KEYS);
            at += r.blocks;
            r.prefix = a.rule.prefix ? max(0, min(a.rule.prefix[b], r.seq.length)) : 0;
            r.base = r.seq.length - r.seq.tokens;
            r.k0 = block0 * KEYS;
            r.k1 = min(r.seq.length, r.k0 + r.blocks * KEYS);
            r.row = ((int64_t)b * a.cache.kv_heads + r.kv_head) * a.cache.slots;
            const int32_t* const pages_of = a.cache.table + (int64_t)b * a.cache.max_pages;
            __syncthreads();
            for (int i = threadIdx.x; i < (r.k1 - r.k0 + (1 << grain) - 1) >> grain; i += blockDim.x)
                places[i] = slot_offset(a.cache, pages_of, r.kv_head, r.k0 + (i << grain));
            __syncthreads();
            return true;
        }
    }
    // the tokens that see some of keys mine .. mine + n - 1: t0 .. t1 - 1
    __device__ __forceinline__ void viewers(const Run& r, int mine, int n, int& t0, int& t1) const
    {
        t0 = 0;
        t1 = r.seq.tokens;
        if (mine >= r.prefix) {
            t0 = max(0, mine - r.base);
            t1 = (int)max((int64_t)t0, min((int64_t)t1, (int64_t)mine + n - 1 + a.rule.window - r.base));
        }
        if (mine >= r.seq.length) t1 = t0;
    }
};

// Sums of keys `mine` + 16 k + 4 quarter .. + 3 in a lane -> lanes l16 < 4: the one of key 4 quarter + l16.
__device__ __forceinline__ float own_sum(const f32x4& s, int l16) { return l16 == 0 ? s[0] : l16 == 1 ? s[1] : l16 == 2 ? s[2] : s[3]; }

template <typename T, int UB, int MODE>
__global__ __launch_bounds__(256)
void paged_sums_kernel(SumsKernelArgs a, int grain)
{
    using C = SumsCfg<T, UB>;
    constexpr int NK = C::NK, NW = C::NW, KEYS = C::KEYS;
    __shared__ int64_t places[kPlaces];
    __shared__ f32x4 joined[NW][NK][4];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, l16 = lane & 15, quarter = lane >> 4;
    const int rb = a.cache.row_bytes, group = a.group.d;
    const ScoreMap<(MODE & kCap) != 0, sizeof(T) == 4> map(a.rule);
    SumsWalk<KEYS> walk(a, grain, lane);
    typename SumsWalk<KEYS>::Run run;
    while (walk.next(run, places)) {
        for (int mine = run.k0; mine < run.k1; mine += KEYS) {
            u32x4 kf[NK][UB];
#pragma unroll
            for (int k = 0; k < NK; ++k) {
                const int slot = min(mine + 16 * k + l16, run.k1 - 1) - run.k0;
                const char* src = a.cache.K + places[slot >> grain] + (slot & ((1 << grain) - 1)) * rb;
#pragma unroll
                for (int g = 0; g < UB; ++g) {
                    const int ch = 4 * g + quarter;    // (behind a row's end: zeros, as the rows have them)
                    kf[k][g] = *reinterpret_cast<const u32x4*>(src + (ch * 16 < rb ? ch * 16 : 0));
                    if (g >= C::FULL && ch * 16 >= rb) kf[k][g] = u32x4{0u, 0u, 0u, 0u};
                }
            }
            int t0, t1;
            walk.viewers(run, mine, KEYS, t0, t1);
            const int r1 = t1 * group;
            f32x4 sum[NK];
#pragma unroll
            for (int k = 0; k < NK; ++k) sum[k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            const auto work = [&](int r, const Rows<UB>& x) __attribute__((always_inline)) {
                add_weights<T, UB, MODE>(sum, a, run.seq, run.prefix, mine, r, r1, x, lane, [&](int k, int g) __attribute__((always_inline)) { return kf[k][g]; }, map);
            };
            int r = t0 * group + wave * 16;
            if (r < r1) {
                Rows<UB> x = fetch_rows<T, UB, MODE, false>(a, run.seq, run.kv_head, rb, r, r1 - 1, lane);
                for (; r + 16 * NW < r1; r += 16 * NW) {
                    const Rows<UB> y = fetch_rows<T, UB, MODE, false>(a, run.seq, run.kv_head, rb, r + 16 * NW, r1 - 1, lane);
                    work(r, x);
                    x = y;
                }
                work(r, x);
            }
#pragma unroll
            for (int k = 0; k < NK; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[k][e] = sum_of_16(sum[k][e]);
            __syncthreads();                      // (what is there of the keys before has been read)
            if (l16 == 0)
#pragma unroll
                for (int k = 0; k < NK; ++k) joined[wave][k][quarter] = sum[k];
            __syncthreads();
            if (wave != 0) continue;
#pragma unroll
            for (int k = 0; k < NK; ++k) {
#pragma unroll
                for (int n = 1; n < NW; ++n) sum[k] += joined[n][k][quarter];
                const int j = mine + 16 * k + 4 * quarter + l16;
                // (slots of the new tokens have no weight from before)
                if (l16 < 4 && j < run.k1) a.sums[run.row + j] = (a.before && j < run.base ? a.before[run.row + j] : 0.0f) + own_sum(sum[k], l16);
            }
        }
    }
}

// EXACT: rows fill their place on chip.
template <typename T, int UB, int MODE, bool EXACT, int THREADS = 64 * StepCfg<T, UB>::NW>
__global__ __launch_bounds__(THREADS, 2)
void paged_sums_step_kernel(SumsKernelArgs a, int grain)
{
    using C = StepCfg<T, UB>;
    using L = RowLayout<UB>;
    constexpr int NW = C::NW, KT = C::KT, NK = KT / 16, DB = C::DB, CPR = UB * 4, TILE = C::TILE, XFERS = C::XFERS, RING = C::RING, KEYS = C::KEYS;
    constexpr int PLACE = C::PLACE;
    __shared__ __align__(1024) char lds[C::LDS];
    int64_t* const places = reinterpret_cast<int64_t*>(lds + C::TILES);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, l16 = lane & 15, quarter = lane >> 4;
    const int rb = EXACT ? DB : a.cache.row_bytes, group = a.group.d;
    char* const tiles = lds + wave * RING * PLACE;      // K of a tile, what its slots had
    const uint32_t tiles_at = lds_offset_of(tiles);
    const ScoreMap<(MODE & kCap) != 0, sizeof(T) == 4> map(a.rule);
    SumsWalk<KEYS> walk(a, grain, lane);
    typename SumsWalk<KEYS>::Run run;
    while (walk.next(run, places)) {
        const int all = run.seq.tokens * group;
        Rows<UB> held;
        if (all > 0) held = fetch_rows<T, UB, MODE, !EXACT>(a, run.seq, run.kv_head, rb, 0, all - 1, lane);
        wait_vmem();
        const float* const had = (a.before ? a.before : a.sums) + run.row;
        // Tile i of the wave (behind the last it is transferred again, unused: as many transfers are under way at any time.)
        const auto issue = [&](int i, int buf) __attribute__((always_inline)) {
            const int first = run.k0 + min(i, run.blocks - 1) * KEYS + wave * KT;
            const uint32_t to = tiles_at + buf * PLACE;
#pragma unroll
            for (int j = 0; j < XFERS; ++j) {
                const int x = j * 64 + lane, key = x / CPR, ch = ((x - key * CPR) ^ L::k_chunk(key)) * 16, slot = min(first + key, run.k1 - 1) - run.k0;
                dma16_untracked(a.cache.K + places[slot >> grain] + (slot & ((1 << grain) - 1)) * rb + (EXACT ? ch : chunk_in_row(ch, rb)), to + j * 1024);
            }
            dma4_untracked(reinterpret_cast<const char*>(had + min(first + lane, run.k1 - 1)), to + TILE);
        };
        for (int n = 0; n < RING; ++n) issue(n, n);
        for (int i = 0, buf = 0; i < run.blocks; ++i, buf = buf + 1 == RING ? 0 : buf + 1) {
            const int mine = run.k0 + i * KEYS + wave * KT;
            const char* const kt = tiles + buf * PLACE;
            wait_vmem_le<(RING - 1) * (XFERS + 1)>();
#if defined(__HIP_DEVICE_COMPILE__)
            asm volatile("" ::: "memory");
#endif
            f32x4 sum[NK];
#pragma unroll
            for (int k = 0; k < NK; ++k) sum[k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            const auto work = [&](int r, int r1, const Rows<UB>& x, bool twice) __attribute__((always_inline)) {
                add_weights<T, UB, MODE>(sum, a, run.seq, run.prefix, mine, r, r1, x, lane, [&](int k, int g) __attribute__((always_inline)) {
                    const u32x4 kf = *reinterpret_cast<const u32x4*>(kt + (16 * k + l16) * DB + ((4 * g + quarter) ^ L::k_chunk(l16)) * 16);
                    const uint32_t keep = EXACT || twice || g < SumsCfg<T, UB>::FULL || (4 * g + quarter) * 16 < rb ? ~0u : 0u;
                    return u32x4{kf[0] & keep, kf[1] & keep, kf[2] & keep, kf[3] & keep};
                }, map);
            };
            if (all > 16) {                       // (a sequence of more tokens than a step's: rows as they are, zeros of keys)
                int t0, t1;
                walk.viewers(run, mine, KT, t0, t1);
                for (int r = t0 * group; r < t1 * group; r += 16) work(r, t1 * group, fetch_rows<T, UB, MODE, false>(a, run.seq, run.kv_head, rb, r, t1 * group - 1, lane), false);
            } else if (all > 0 && mine < run.k1) {
                work(0, all, held, true);
            }
            float before[NK];
#pragma unroll
            for (int k = 0; k < NK; ++k) before[k] = *reinterpret_cast<const float*>(kt + TILE + (16 * k + 4 * quarter + (l16 & 3)) * 4);
#pragma unroll
            for (int k = 0; k < NK; ++k) {
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[k][e] = sum_of_16(sum[k][e]);
                const int j = mine + 16 * k + 4 * quarter + l16;
                if (l16 < 4 && j < run.k1) a.sums[run.row + j] = (a.before && j < run.base ? before[k] : 0.0f) + own_sum(sum[k], l16);
            }
            wait_lds();                           // (the tile has left its place)
            issue(i + RING, buf);
        }
        wait_vmem();
    }
}

template <typename T, int UB, int MODE> hipError_t launch(const SumsArgs& p, hipStream_t stream)
{
    SumsKernelArgs a;
    a.Q = static_cast<const char*>(p.Q);
    a.lse = p.lse;
    a.before = p.before;
    a.sums = p.sums;
    a.starts = p.starts;
    a.q_stride = p.q_stride * (int64_t)sizeof(T);
    a.tokens = (int32_t)p.tokens;
    a.heads = (int32_t)p.heads;
    a.group = fast_div((uint32_t)(p.heads / p.cache.kv_heads));
    a.cache = p.cache;
    a.rule = p.rule;
    // (workgroups of unequal work in several rounds: those that end early make room)
    // Rows of a sequence, on average.  Held / in turns, us: bf16, 8 sequences of 4096 slots, 4 kv heads of 128: 128 rows 30 / 40, 256 47 / 44, 384 63 / 51, 1024
    // 151 / 88; 64 of them 183 / 238, 333 / 294, 530 / 350, 1433 / 630; d = 64 256 rows 22 / 26, 384 29 / 30.  fp32, 4 of them: 96 rows 38 / 51, 128 47 / 52, 256 84 / 70; d = 64, a
    // cap: 128 rows 25 / 30, 192 33 / 34; d = 100 128 rows 44 / 43.
    const bool turns = p.tokens * (int64_t)a.group.d > (sizeof(T) == 2 ? 256 : 128) * (int64_t)p.cache.batch;
    const uint32_t grid = (uint32_t)((compute_units() * (turns ? 16 : StepCfg<T, UB>::PER_CU) + 7) & ~7);
    const int grain = key_grain(a.cache);
    constexpr bool OWN = UB > 1;                  // rows that fill their place: kernels of their own
    if (turns) paged_sums_kernel<T, UB, MODE><<<grid, 256, 0, stream>>>(a, grain);
    else if (OWN && p.cache.row_bytes == UB * 64) paged_sums_step_kernel<T, UB, MODE, OWN><<<grid, 64 * StepCfg<T, UB>::NW, 0, stream>>>(a, grain);
    else paged_sums_step_kernel<T, UB, MODE, false><<<grid, 64 * StepCfg<T, UB>::NW, 0, stream>>>(a, grain);
    return hipGetLastError();
}

template <typename T, int UB> hipError_t launch_mode(const SumsArgs& p, hipStream_t stream)
{
    switch (rule_mode(p.rule)) {
    case kPlain: return launch<T, UB, kPlain>(p, stream);
    case kCap: return launch<T, UB, kCap>(p, stream);
    case kBias: return launch<T, UB, kBias>(p, stream);
    default: return launch<T, UB, kCap | kBias>(p, stream);
    }
}

}  // namespace

hipError_t launch_paged_sums(const SumsArgs& a, hipStream_t stream)
{
    const int ub = (a.cache.row_bytes + 63) / 64;
    if (a.dt == DType::F32) {
        if (ub <= 1) return launch_mode<float, 1>(a, stream);
        if (ub <= 2) return launch_mode<float, 2>(a, stream);
        if (ub <= 4) return launch_mode<float, 4>(a, stream);
        if (ub <= 8) return launch_mode<float, 8>(a, stream);
        return launch_mode<float, 16>(a, stream);
    }
    if (ub <= 1) return launch_mode<uint16_t, 1>(a, stream);
    if (ub <= 2) return launch_mode<uint16_t, 2>(a, stream);
    if (ub <= 4) return launch_mode<uint16_t, 4>(a, stream);
    return launch_mode<uint16_t, 8>(a, stream);
}

}  // namespace attnw
