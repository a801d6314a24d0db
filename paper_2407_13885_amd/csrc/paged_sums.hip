// What the slots of a paged cache are worth to new tokens:
//
//     sums[b][kv_head][j] = before[b][kv_head][j] + sum over the new tokens i and the heads of the kv head of exp(s_ij - lse_i),
//
// the weights that attention gave the slot (s and what a token sees as there, lse from there).
//
// A workgroup owns the slots that it sums over, and its waves keep the keys of theirs in registers while rows pass by, straight from the caches, 16
// at a time, the next ones on their way: no atomics, K read once, sums in an order that the sizes alone decide.  Single tokens: the waves have keys of
// their own (what bounds it is the read of K).  Chunks: all waves have the same keys and take the rows in turn, their sums joined in the end (what
// bounds it are the exponentials, as many as scores: three transcendental instructions each with a cap).
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
    static constexpr int NW = 4, NK = UB <= 2 ? 4 : UB <= 4 ? (sizeof(T) == 2 ? 4 : 2) : UB <= 8 ? 2 : 1;
};

// TURNS: all waves of a workgroup have the same keys.
template <typename T, int UB, int MODE, bool TURNS>
__global__ __launch_bounds__(256)
void paged_sums_kernel(SumsKernelArgs a)
{
    using C = SumsCfg<T, UB>;
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int NK = C::NK, NW = C::NW, KEYS = 16 * NK * (TURNS ? 1 : NW);
    __shared__ f32x4 joined[TURNS ? NW : 1][NK][4];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, l16 = lane & 15, quarter = lane >> 4;
    const int rb = a.cache.row_bytes, group = a.group.d;
    const auto count = [&](int b) __attribute__((always_inline)) {
        const int32_t n = max(0, min(a.cache.lengths[b], a.cache.slots));
        return ((n + KEYS - 1) / KEYS) * a.cache.kv_heads;
    };
    const int32_t total = plan_total(a.cache.batch, lane, count);
    const Deal deal = deal_out(total, (int32_t)gridDim.x);
    const int w = dealt_workgroup(deal);
    if (w >= deal.workgroups) return;
    int32_t at = deal.first(w);
    const int32_t end = deal.first(w + 1);
    int32_t b, before;
    plan_find(a.cache.batch, lane, at, count, b, before);
    const ScoreMap<(MODE & kCap) != 0, F32> map(a.rule);

    while (at < end && b < a.cache.batch) {
        const Sequence seq = sequence_at(a.cache, a.starts, a.tokens, b);
        const int blocks = (seq.length + KEYS - 1) / KEYS;
        const int32_t here = at - before;
        if (here >= blocks * a.cache.kv_heads) {
            before += blocks * a.cache.kv_heads;
            ++b;
            continue;
        }
        ++at;
        const int kv_head = uniform((int32_t)((uint32_t)here / (uint32_t)blocks)), key0 = (here - kv_head * blocks) * KEYS;
        const int prefix = a.rule.prefix ? max(0, min(a.rule.prefix[b], seq.length)) : 0;
        const int base = seq.length - seq.tokens;
        const int mine = key0 + (TURNS ? 0 : wave * 16 * NK);  // the first of the wave's keys
        const int32_t* const pages_of = a.cache.table + (int64_t)b * a.cache.max_pages;
        u32x4 kf[NK][UB];
#pragma unroll
        for (int k = 0; k < NK; ++k) {
            const char* src = a.cache.K + slot_offset(a.cache, pages_of, kv_head, min(mine + 16 * k + l16, seq.length - 1));
#pragma unroll
            for (int g = 0; g < UB; ++g) {
                const int ch = 4 * g + quarter;
                kf[k][g] = ch * 16 < rb ? *reinterpret_cast<const u32x4*>(src + ch * 16) : u32x4{0u, 0u, 0u, 0u};
            }
        }
        // the tokens that see some of the wave's keys
        int t0 = 0, t1 = seq.tokens;
        if (mine >= prefix) {
            t0 = max(0, mine - base);
            t1 = (int)max((int64_t)t0, min((int64_t)t1, (int64_t)mine + 16 * NK - 1 + a.rule.window - base));
        }
        if (mine >= seq.length) t1 = t0;
        const int64_t r0 = (int64_t)t0 * group, r1 = (int64_t)t1 * group;
        f32x4 sum[NK];
#pragma unroll
        for (int k = 0; k < NK; ++k) sum[k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

        struct Rows {                             // 16 of them, of a lane one
            u32x4 q[UB];
            float lse, slope;
            int query;
        };
        const auto fetch = [&](int64_t r) __attribute__((always_inline)) {
            Rows x;
            // (row r0 + i: its token and head, r0 itself being the first head of a token)
            const uint32_t i = (uint32_t)min(r - r0 + l16, r1 - 1 - r0), t = quotient(i, a.group);
            const int token = t0 + (int)t, head = kv_head * group + (int)(i - t * group);
            const int64_t at_row = seq.first + token;
            const char* q = a.Q + at_row * a.q_stride + (int64_t)head * rb;
#pragma unroll
            for (int g = 0; g < UB; ++g) {
                const int ch = 4 * g + quarter;
                x.q[g] = ch * 16 < rb ? *reinterpret_cast<const u32x4*>(q + ch * 16) : u32x4{0u, 0u, 0u, 0u};
            }
            x.lse = a.lse[at_row * a.heads + head];
            x.slope = MODE & kBias ? a.rule.slopes[head] * kLog2e : 0.0f;
            x.query = base + token;
            return x;
        };
        const auto work = [&](int64_t r, const Rows& x) __attribute__((always_inline)) {
            f32x4 acc[NK];
#pragma unroll
            for (int k = 0; k < NK; ++k) acc[k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int g = 0; g < UB; ++g)
#pragma unroll
                for (int k = 0; k < NK; ++k) {
                    if constexpr (F32) {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            acc[k] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[k][g][i]), __uint_as_float(x.q[g][i]), acc[k], 0, 0, 0);
                    } else {
                        mma16(acc[k], kf[k][g], x.q[g]);
                    }
                }
            // a row that saw nothing, or that is not there, adds nothing
            const float lse = x.lse == -__builtin_inff() || r + l16 >= r1 ? __builtin_inff() : x.lse * kLog2e;
            // (tokens of the rows: first .. last)
            const int first = __builtin_amdgcn_readlane(x.query, 0), last = __builtin_amdgcn_readlane(x.query, 15);
            const bool whole = mine + 16 * NK <= seq.length && ((mine + 16 * NK - 1 <= first && mine > last - a.rule.window) || mine + 16 * NK <= prefix);
#pragma unroll
            for (int k = 0; k < NK; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float y = map(acc[k][i]);
                    if constexpr ((MODE & kBias) != 0) y -= x.slope * (float)abs(x.query - (mine + 16 * k + 4 * quarter + i));
                    acc[k][i] = fast_exp2(y - lse);
                }
            if (!whole) {
#pragma unroll
                for (int k = 0; k < NK; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int j = mine + 16 * k + 4 * quarter + i;
                        if (j >= seq.length || ((uint32_t)(x.query - j) >= (uint32_t)a.rule.window && j >= prefix)) acc[k][i] = 0.0f;
                    }
            }
#pragma unroll
            for (int k = 0; k < NK; ++k) sum[k] += acc[k];
        };
        constexpr int STEP = 16 * (TURNS ? NW : 1);
        int64_t r = r0 + (TURNS ? wave * 16 : 0);
        if (r < r1) {
            Rows x = fetch(r);
            for (; r + STEP < r1; r += STEP) {
                const Rows y = fetch(r + STEP);
                work(r, x);
                x = y;
            }
            work(r, x);
        }
#pragma unroll
        for (int off = 1; off < 16; off <<= 1)
#pragma unroll
            for (int k = 0; k < NK; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[k][i] += __shfl_xor(sum[k][i], off, 64);
        if constexpr (TURNS) {
            __syncthreads();                      // (what is there of the keys before has been read)
            if (l16 == 0)
#pragma unroll
                for (int k = 0; k < NK; ++k) joined[wave][k][quarter] = sum[k];
            __syncthreads();
            if (wave != 0) continue;
#pragma unroll
            for (int k = 0; k < NK; ++k)
#pragma unroll
                for (int n = 1; n < NW; ++n) sum[k] += joined[n][k][quarter];
        }
        const int64_t row = ((int64_t)b * a.cache.kv_heads + kv_head) * a.cache.slots;
#pragma unroll
        for (int k = 0; k < NK; ++k) {
            const int j = mine + 16 * k + 4 * quarter + l16;
            const float v = l16 == 0 ? sum[k][0] : l16 == 1 ? sum[k][1] : l16 == 2 ? sum[k][2] : sum[k][3];
            // (slots of the new tokens have no weight from before)
            if (l16 < 4 && j < seq.length) a.sums[row + j] = (a.before && j < base ? a.before[row + j] : 0.0f) + v;
        }
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
    const bool turns = p.tokens * (int64_t)a.group.d > 32 * (int64_t)p.cache.batch;
    const uint32_t grid = (uint32_t)((compute_units() * (turns ? 16 : 8) + 7) & ~7);
    if (turns) paged_sums_kernel<T, UB, MODE, true><<<grid, 256, 0, stream>>>(a);
    else paged_sums_kernel<T, UB, MODE, false><<<grid, 256, 0, stream>>>(a);
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
