// Shared by the kernels of attention over a paged cache: what they are given, and the join of partial results.
#pragma once

#include "qk_common.h"
#include "attention_common.h"
#include "paged_common.h"

namespace attnw {
namespace {

// At most N transfers under way, and no read from LDS before that.
template <int N> __device__ __forceinline__ void arrived()
{
    wait_vmem_le<N>();
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("" ::: "memory");
#endif
}

struct AttendArgs {
    const char* Q;
    char* O;
    float *lse, *partial;
    const int32_t* starts;
    int64_t q_stride;                             // bytes of a token's row of Q
    int32_t tokens, heads, group;
    CacheView cache;
    RuleView rule;
    PlanShape plan;
};

struct Counted {
    const AttendArgs& a;
    __device__ __forceinline__ int64_t operator()(int b) const
    {
        const Sequence s = sequence_at(a.cache, a.starts, a.tokens, b);
        const SequencePlan p = sequence_plan(a.plan, s, a.rule.prefix ? a.rule.prefix[b] : 0, a.rule.window);
        return (int64_t)p.blocks * p.units * a.cache.kv_heads;
    }
};

// A row of partial results, or a whole one: 4 columns of the output of token, head (numbered o), l the sum of its weights.
template <typename T> __device__ __forceinline__ void store_output(char* O, int64_t o, int rb, int c, f32x4 y, float l)
{
    y *= l == 0.0f ? 0.0f : 1.0f / l;
    if (c * (int)sizeof(T) >= rb) return;
    if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4*>(O + o * rb + c * 4) = y;
    else *reinterpret_cast<u32x2*>(O + o * rb + c * 2) = u32x2{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
}
// log of a sum l of weights 2^(x - top)
__device__ __forceinline__ float log_sum(float top, float l) { return l == 0.0f ? -__builtin_inff() : (top + fast_log2(l)) * (1.0f / kLog2e); }

// The partial results of blocks that several workgroups worked on.  A workgroup per (block, kv head).
template <typename T>
__global__ __launch_bounds__(256)
void paged_join_kernel(AttendArgs a, int32_t cols)
{
    const int lane = threadIdx.x & 63;
    const Counted count{a};
    const int64_t total = plan_total(a.cache.batch, lane, count);
    const Deal deal = deal_out(total, a.plan.workgroups, a.plan.least);
    const auto blocks = [&](int i) __attribute__((always_inline)) {
        const Sequence s = sequence_at(a.cache, a.starts, a.tokens, i);
        return (((int64_t)s.tokens * a.group + a.plan.rows - 1) / a.plan.rows) * a.cache.kv_heads;
    };
    for (int64_t x = blockIdx.x;; x += gridDim.x) {
        int32_t b;
        int64_t before;
        plan_find(a.cache.batch, lane, x, blocks, b, before);
            if (b < 0) return;
        const Sequence seq = sequence_at(a.cache, a.starts, a.tokens, b);
        const SequencePlan plan = sequence_plan(a.plan, seq, a.rule.prefix ? a.rule.prefix[b] : 0, a.rule.window);
        const int64_t mine = x - before;
        const int kv_head = (int)(mine / plan.blocks), block = (int)(mine - (int64_t)kv_head * plan.blocks);
        int64_t x0 = 0;
        for (int i = lane; i < b; i += 64) x0 += count(i);
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) x0 += __shfl_xor(x0, off, 64);
        x0 = uniform(x0) + mine * plan.units;
        const int64_t w0 = deal.owner(x0), w1 = deal.owner(x0 + plan.units - 1);
        if (w0 == w1) continue;
        const int64_t row0 = (int64_t)block * a.plan.rows;
        const int rows = (int)min((int64_t)a.plan.rows, (int64_t)seq.tokens * a.group - row0);
        const int64_t slot = (int64_t)a.plan.rows * (cols + 2);
        const bool later = deal.first(w0) != x0;   // (the first of them began with another block)
        const auto part = [&](int64_t w) __attribute__((always_inline)) { return a.partial + (2 * w + (w == w0 && later ? 1 : 0)) * slot; };
        const int quads = cols / 4, rb = a.cache.row_bytes;
        for (int i = threadIdx.x; i < rows * quads; i += 256) {
            const int r = i / quads, c = (i - r * quads) * 4;
            float top = -__builtin_inff();
            for (int64_t w = w0; w <= w1; ++w) top = fmaxf(top, part(w)[a.plan.rows * cols + 2 * r]);
            const float ref = top == -__builtin_inff() ? 0.0f : top;
            f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
            float l = 0.0f;
#pragma unroll 4
            for (int64_t w = w0; w <= w1; ++w) {
                const float* p = part(w);
                const float f = fast_exp2(p[a.plan.rows * cols + 2 * r] - ref);
                l += f * p[a.plan.rows * cols + 2 * r + 1];
                sum += *reinterpret_cast<const f32x4*>(p + r * cols + c) * f;
            }
            const int64_t rr = row0 + r;
            const int tk = (int)(rr / a.group), h = kv_head * a.group + (int)(rr - (int64_t)tk * a.group);
            const int64_t o = (int64_t)(seq.first + tk) * a.heads + h;
            store_output<T>(a.O, o, rb, c, sum, l);
            if (c == 0 && a.lse) a.lse[o] = log_sum(top, l);
        }
    }
}

inline AttendArgs attend_args(const PagedArgs& p, const PlanShape& plan, int64_t size)
{
    AttendArgs a;
    a.Q = static_cast<const char*>(p.Q);
    a.O = static_cast<char*>(p.O);
    a.lse = p.lse;
    a.partial = p.workspace;
    a.starts = p.starts;
    a.q_stride = p.q_stride * size;
    a.tokens = (int32_t)p.tokens;
    a.heads = (int32_t)p.heads;
    a.group = plan.group;
    a.cache = p.cache;
    a.rule = p.rule;
    a.plan = plan;
    return a;
}

// Two places for every workgroup: of the block that its stretch begins in, and of the one that it ends in.
inline int64_t partial_bytes(const PlanShape& plan, int cols) { return (int64_t)plan.workgroups * 2 * plan.rows * (cols + 2) * 4; }

template <typename T> hipError_t launch_join(const AttendArgs& a, int cols, hipStream_t stream)
{
    // (every sequence may have one block that is not full)
    const int64_t blocks = ((int64_t)a.tokens * a.group / a.plan.rows + a.cache.batch) * a.cache.kv_heads;
    paged_join_kernel<T><<<(uint32_t)(blocks < 1 << 20 ? blocks : 1 << 20), 256, 0, stream>>>(a, cols);
    return hipGetLastError();
}

}  // namespace
}  // namespace attnw
