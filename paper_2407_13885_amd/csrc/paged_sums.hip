// What the slots of a paged cache are worth to new tokens:
//
//     sums[b][kv_head][j] = before[b][kv_head][j] + sum over the new tokens i and the heads of the kv head of exp(s_ij - lse_i),
//
// the weights that attention gave the slot (s and what a token sees as there, lse from there).
//
// A workgroup owns the slots that it sums over, and its waves keep the keys of theirs in registers while all rows pass by: no atomics, one order of
// summation whatever the launch, K read once.  What bounds it: for single tokens the read of K; for chunks the products, of which the exponentials are as
// many as the scores.
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
    int32_t tokens, heads, group;
    CacheView cache;
    RuleView rule;
};

template <typename T, int UB> struct SumsCfg {
    static constexpr bool F32 = sizeof(T) == 4;
    static constexpr int NK = UB <= 4 ? 2 : 1;    // blocks of 16 keys of a wave
    static constexpr int NW = 4, KEYS = 16 * NK * NW;
};

template <typename T, int UB, bool GENERAL>
__global__ __launch_bounds__(256)
void paged_sums_kernel(SumsKernelArgs a)
{
    using C = SumsCfg<T, UB>;
    constexpr bool F32 = C::F32;
    constexpr int NK = C::NK, KEYS = C::KEYS;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, l16 = lane & 15, quarter = lane >> 4;
    const int rb = a.cache.row_bytes;
    const auto count = [&](int b) __attribute__((always_inline)) {
        const int32_t n = max(0, min(a.cache.lengths[b], a.cache.slots));
        return (int64_t)((n + KEYS - 1) / KEYS) * a.cache.kv_heads;
    };
    const int64_t total = plan_total(a.cache.batch, lane, count);
    const int64_t per = (total + gridDim.x - 1) / gridDim.x;
    int64_t at = xcd_contiguous_block_id(blockIdx.x, gridDim.x) * per;
    const int64_t end = min(total, at + per);
    if (at >= end) return;
    int32_t b;
    int64_t before;
    plan_find(a.cache.batch, lane, at, count, b, before);
    const ScoreMap<false, F32> plain(a.rule);

    while (at < end && b < a.cache.batch) {
        const Sequence seq = sequence_at(a.cache, a.starts, a.tokens, b);
        const int blocks = (seq.length + KEYS - 1) / KEYS;
        const int64_t here = at - before;
        if (here >= (int64_t)blocks * a.cache.kv_heads) {
            before += (int64_t)blocks * a.cache.kv_heads;
            ++b;
            continue;
        }
        ++at;
        const int kv_head = (int)(here / blocks), key0 = (int)(here - (int64_t)kv_head * blocks) * KEYS;
        const int prefix = a.rule.prefix ? max(0, min(a.rule.prefix[b], seq.length)) : 0;
        const int base = seq.length - seq.tokens;
        const int mine = key0 + wave * 16 * NK;    // the first of the wave's keys
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
        const int64_t r1 = (int64_t)t1 * a.group;
        f32x4 sum[NK];
#pragma unroll
        for (int k = 0; k < NK; ++k) sum[k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        for (int64_t r0 = (int64_t)t0 * a.group; r0 < r1; r0 += 16) {
            const int64_t row = min(r0 + l16, r1 - 1);
            const int token = (int)(row / a.group), head = kv_head * a.group + (int)(row - (int64_t)token * a.group);
            const int query = base + token, low = query - a.rule.window;
            const float slope = GENERAL && a.rule.slopes ? a.rule.slopes[head] * kLog2e : 0.0f;
            const char* q = a.Q + (int64_t)(seq.first + token) * a.q_stride + (int64_t)head * rb;
            float lse = a.lse[(int64_t)(seq.first + token) * a.heads + head] * kLog2e;
            if (lse == -__builtin_inff()) lse = __builtin_inff();   // a row that saw nothing adds nothing
            f32x4 acc[NK];
#pragma unroll
            for (int k = 0; k < NK; ++k) acc[k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int g = 0; g < UB; ++g) {
                const int ch = 4 * g + quarter;
                const u32x4 qf = ch * 16 < rb ? *reinterpret_cast<const u32x4*>(q + ch * 16) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
                for (int k = 0; k < NK; ++k) {
                    if constexpr (F32) {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            acc[k] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[k][g][i]), __uint_as_float(qf[i]), acc[k], 0, 0, 0);
                    } else {
                        mma16(acc[k], kf[k][g], qf);
                    }
                }
            }
#pragma unroll
            for (int k = 0; k < NK; ++k)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int j = mine + 16 * k + 4 * quarter + r;
                    float x;
                    if (GENERAL && a.rule.cap > 0.0f) x = ScoreMap<true, F32>(a.rule)(acc[k][r]);
                    else x = plain(acc[k][r]);
                    if constexpr (GENERAL) x -= slope * (float)abs(query - j);
                    const bool sees = r0 + l16 < r1 && j < seq.length && ((j <= query && j > low) || j < prefix);
                    sum[k][r] += sees ? fast_exp2(x - lse) : 0.0f;
                }
        }
#pragma unroll
        for (int off = 1; off < 16; off <<= 1)
#pragma unroll
            for (int k = 0; k < NK; ++k)
#pragma unroll
                for (int r = 0; r < 4; ++r) sum[k][r] += __shfl_xor(sum[k][r], off, 64);
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

template <typename T, int UB> hipError_t launch(const SumsArgs& p, hipStream_t stream)
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
    a.group = (int32_t)(p.heads / p.cache.kv_heads);
    a.cache = p.cache;
    a.rule = p.rule;
    const uint32_t grid = (uint32_t)((compute_units() * 4 + 7) & ~7);
    if (p.rule.cap > 0.0f || p.rule.slopes) paged_sums_kernel<T, UB, true><<<grid, 256, 0, stream>>>(a);
    else paged_sums_kernel<T, UB, false><<<grid, 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_sums(const SumsArgs& a, hipStream_t stream)
{
    const int ub = (a.cache.row_bytes + 63) / 64;
    if (a.dt == DType::F32) {
        if (ub <= 1) return launch<float, 1>(a, stream);
        if (ub <= 2) return launch<float, 2>(a, stream);
        if (ub <= 4) return launch<float, 4>(a, stream);
        if (ub <= 8) return launch<float, 8>(a, stream);
        return launch<float, 16>(a, stream);
    }
    if (ub <= 1) return launch<uint16_t, 1>(a, stream);
    if (ub <= 2) return launch<uint16_t, 2>(a, stream);
    if (ub <= 4) return launch<uint16_t, 4>(a, stream);
    return launch<uint16_t, 8>(a, stream);
}

}  // namespace attnw
