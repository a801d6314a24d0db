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

// (also: how many workgroups the work is dealt to)
struct AttendArgs {
    const char* Q;
    char* O;
    float *lse, *partial;
    struct Joint* joints;                         // one for each workgroup
    const int32_t* starts;
    int64_t q_stride;                             // bytes of a token's row of Q
    int32_t tokens, heads;
    FastDiv group;
    CacheView cache;
    RuleView rule;
    int32_t workgroups, unit_log;
};

// A piece of a block that several workgroups work on ends in a workgroup that did not begin it: what the join, a workgroup for each, has to know.
struct Joint {
    int32_t first;                                // the workgroup that the block begins in, -1: nothing to join
    int32_t later;                                // which of its two places: 1 if it had another block before
    int32_t rows, kv_head, row0, token0;
};

// The work of a ragged batch as one list: a block (ROWS rows of one kv head of one sequence) is `units` places of it, one for each 2^unit_log keys that its last rows
// see.  A workgroup takes as many consecutive places as any other, so that long and short sequences load all of them alike; a block whose
// places fall to several of them leaves partial results, which a second launch joins.  Every block of a sequence has the same number of places: a
// block whose rows see fewer keys has them spread over its places.
struct Segment {                                  // the places of one block that are a workgroup's
    Sequence seq;
    int32_t b, prefix, kv_head, row0, rows;       // (row0: the block's first, of the kv head's rows of the sequence)
    int32_t v0, v1, units;                        // places v0 .. v1 - 1 of its `units`
    int32_t slot;                                 // where partial results go, -1: the block is all here
};

// A workgroup's way through its places.  (Sequences: of up to 64 each lane of a wave holds one, read once.  What a kernel for single tokens does before its first
// load counts: 32 bits throughout, the host makes places of more keys where there would be 2^31.)
template <int ROWS> struct Walk {
    const AttendArgs& a;
    bool held, begun;
    Sequence own;
    int32_t own_prefix;
    Deal deal;
    int32_t w, b;                                 // workgroup, sequence
    int32_t at, end, before;                      // places: next, behind the last, of the sequences before b

    struct Plan { int32_t blocks, units; };       // of a kv head
    __device__ __forceinline__ int32_t units_of(uint32_t keys) const { return (int32_t)((keys + (1u << a.unit_log) - 1) >> a.unit_log); }
    __device__ __forceinline__ Plan plan(const Sequence& s, int32_t prefix) const
    {
        Plan p;
        p.blocks = (int32_t)((uint32_t)(s.tokens * (int32_t)a.group.d + ROWS - 1) / ROWS);
        p.units = max(1, units_of(s.length));
        if (a.rule.window < kNoWindow) {
            // a block's rows belong to so many tokens at most, which together see a window and so many keys more
            const uint32_t span = min((int32_t)quotient(ROWS - 2 + a.group.d, a.group) + 1, s.tokens);
            p.units = min(p.units, units_of(prefix) + units_of(a.rule.window + span) + 2);
        }
        return p;
    }
    __device__ __forceinline__ int32_t prefix_at(int i, const Sequence& s) const { return a.rule.prefix ? max(0, min(a.rule.prefix[i], s.length)) : 0; }
    __device__ __forceinline__ int32_t places(const Plan& p) const { return p.blocks * p.units * a.cache.kv_heads; }
    __device__ __forceinline__ Walk(const AttendArgs& args, int lane) : a(args), held(args.cache.batch <= 64), begun(false)
    {
        const auto of = [&](int i) __attribute__((always_inline)) {
            const Sequence s = sequence_at(a.cache, a.starts, a.tokens, i);
            return places(plan(s, prefix_at(i, s)));
        };
        own = Sequence{0, 0, 0};
        own_prefix = 0;
        int32_t upto = 0;
        if (held) {
            int32_t mine = 0;
            if (lane < a.cache.batch) {
                own = sequence_at(a.cache, a.starts, a.tokens, lane);
                own_prefix = prefix_at(lane, own);
                mine = places(plan(own, own_prefix));
            }
            upto = wave_inclusive_sum(mine, lane, a.cache.batch);
            deal = deal_out(__builtin_amdgcn_readlane(upto, a.cache.batch - 1), a.workgroups);
        } else {
            deal = deal_out(plan_total(a.cache.batch, lane, of), a.workgroups);
        }
        w = dealt_workgroup(deal);
        if (threadIdx.x == 0) a.joints[w].first = -1;          // (unless a block ends here)
        at = end = 0;
        if (w >= deal.workgroups) return;
        at = deal.first(w);
        end = deal.first(w + 1);
        if (held) {
            const uint64_t past = __builtin_amdgcn_ballot_w64(lane < a.cache.batch && upto > at);
            b = past ? __builtin_ctzll(past) : a.cache.batch;
            before = past && b > 0 ? __builtin_amdgcn_readlane(upto, b - 1) : 0;
        } else {
            plan_find(a.cache.batch, lane, at, of, b, before);
        }
    }
    // The next segment, if there is one.
    __device__ __forceinline__ bool next(Segment& g)
    {
        for (;; ++b) {
            if (at >= end || b >= a.cache.batch) return false;
            g.seq = held ? Sequence{__builtin_amdgcn_readlane(own.length, b), __builtin_amdgcn_readlane(own.tokens, b), __builtin_amdgcn_readlane(own.first, b)}
                         : sequence_at(a.cache, a.starts, a.tokens, b);
            g.prefix = held ? __builtin_amdgcn_readlane(own_prefix, b) : prefix_at(b, g.seq);
            const Plan p = plan(g.seq, g.prefix);
            const int32_t here = at - before;
            if (here >= places(p)) {
                before += places(p);
                continue;
            }
            const int32_t block = p.units == 1 ? here : uniform((int32_t)((uint32_t)here / (uint32_t)p.units));
            g.kv_head = p.blocks == 1 ? block : uniform((int32_t)((uint32_t)block / (uint32_t)p.blocks));
            g.row0 = (block - g.kv_head * p.blocks) * ROWS;
            g.b = b;
            g.units = p.units;
            g.rows = min(ROWS, g.seq.tokens * (int32_t)a.group.d - g.row0);
            g.v0 = here - block * p.units;
            g.v1 = min(g.units, g.v0 + (end - at));
            g.slot = g.v0 == 0 && g.v1 == g.units ? -1 : 2 * w + (begun ? 1 : 0);
            if (!begun && g.v0 > 0 && g.v1 == g.units && threadIdx.x == 0) {
                Joint j;
                j.first = deal.owner(at - g.v0);
                j.later = deal.first(j.first) != at - g.v0 ? 1 : 0;
                j.rows = g.rows;
                j.kv_head = g.kv_head;
                j.row0 = g.row0;
                j.token0 = g.seq.first;
                a.joints[w] = j;
            }
            at += g.v1 - g.v0;
            begun = true;
            return true;
        }
    }
    // Of n units of keys (which may be fewer than the segment's block has places) the first that are a segment's, or behind its last.
    __device__ __forceinline__ int32_t share(const Segment& g, int32_t v, int32_t n) const
    {
        return n == g.units ? v : uniform((int32_t)((uint64_t)v * n / (uint32_t)g.units));
    }
};

// Values that are not finite must not reach the rows that do not see them, by way of a weight of 0: where some are, they count as 0 in the product, and this is
// what they add to the rows that do see them.  v: a fragment of V; some, none: the weights that are seen, as 1 where they are not 0, and where they are (0
// times infinity is NaN); multiply(sum, v, weights).
template <typename T, typename Multiply> __device__ __forceinline__ f32x4 lost_part(const u32x4& v, const u32x4& some, const u32x4& none, Multiply&& multiply)
{
    f32x4 up = {0.0f, 0.0f, 0.0f, 0.0f}, down = up, r;
    multiply(up, lost_as_one<T, kUp>(v), some);
    multiply(down, lost_as_one<T, kDown>(v), some);
    multiply(up, lost_as_one<T, kAny>(v), none);
    multiply(down, lost_as_one<T, kAny>(v), none);
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = (up[i] > 0.0f ? __builtin_inff() : 0.0f) - (down[i] > 0.0f ? __builtin_inff() : 0.0f);
    return r;
}

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

// A slice of ROWS rows of one block's partial results, which end in workgroup w's stretch and did not begin there.  Two loads one after the other bound
// it: the threads of a workgroup read the parts' exponents at once, then share the columns and the parts.
template <typename T, int ROWS>
__device__ __forceinline__ void join_rows(const AttendArgs& a, const Joint& j, int w, int first, int32_t block_rows, int32_t cols, float (&tops)[256], float (&sums)[256][5])
{
    const int rows = min(ROWS, j.rows - first), parts = w - j.first + 1, tid = threadIdx.x;
    if (rows <= 0) return;
    const int64_t slot = (int64_t)block_rows * (cols + 2);
    const float* const p0 = a.partial + (2 * (int64_t)j.first + j.later) * slot;         // the first part; the others are 2 places apart
    const float* const p1 = a.partial + 2 * (int64_t)j.first * slot;
    const auto part = [&](int k) __attribute__((always_inline)) { return k == 0 ? p0 : p1 + 2 * (int64_t)k * slot; };
    const int stats = block_rows * cols + 2 * first;
    {
        const int r = tid % ROWS;
        float top = -__builtin_inff();
        if (r < rows)
#pragma unroll 8
            for (int k = tid / ROWS; k < parts; k += 256 / ROWS) top = fmaxf(top, part(k)[stats + 2 * r]);
        tops[tid] = top;
    }
    __syncthreads();
    const int quads = cols / 4, items = rows * quads, rb = a.cache.row_bytes;
    int share = 1;                                // threads that share an item
    while (share < 16 && share * 2 * items <= 256) share *= 2;
    const int step = 256 / share, mine = tid / step;
    for (int i0 = 0; i0 < items; i0 += step) {
        const int i = i0 + tid % step, r = min(i / quads, rows - 1), c = (i - i / quads * quads) * 4;
        float top = tops[r];
#pragma unroll
        for (int k = 1; k < 256 / ROWS; ++k) top = fmaxf(top, tops[r + k * ROWS]);
        const float ref = top == -__builtin_inff() ? 0.0f : top;
        f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
        float l = 0.0f;
#pragma unroll 8
        for (int k = mine; k < parts; k += share) {
            const float* p = part(k);
            const float f = fast_exp2(p[stats + 2 * r] - ref);
            l += f * p[stats + 2 * r + 1];
            sum += *reinterpret_cast<const f32x4*>(p + (first + r) * cols + c) * f;
        }
        if (share > 1) {                          // (then one round is enough: no barrier in front)
            float* const s = sums[tid];
            s[0] = sum[0], s[1] = sum[1], s[2] = sum[2], s[3] = sum[3], s[4] = l;
            __syncthreads();
            if (mine != 0) return;
            for (int k = 1; k < share; ++k) {
                const float* const o = sums[tid + k * step];
                sum += f32x4{o[0], o[1], o[2], o[3]};
                l += o[4];
            }
        }
        if (i >= items) continue;
        const int row = j.row0 + first + r;
        const uint32_t tk = quotient(row, a.group);
        const int64_t o = (int64_t)(j.token0 + (int)tk) * a.heads + j.kv_head * (int)a.group.d + (int)(row - tk * a.group.d);
        store_output<T>(a.O, o, rb, c, sum, l);
        if (c == 0 && a.lse) a.lse[o] = log_sum(top, l);
    }
}

// One workgroup for each note and slice that there might be.
template <typename T, int ROWS>
__global__ __launch_bounds__(256)
void paged_join_kernel(AttendArgs a, int32_t block_rows, int32_t cols)
{
    __shared__ float tops[256];
    __shared__ float sums[256][5];
    const Joint j = a.joints[blockIdx.x];
    if (j.first < 0) return;
    join_rows<T, ROWS>(a, j, blockIdx.x, blockIdx.y * ROWS, block_rows, cols, tops, sums);
}

// The same where that would be many more than there are (blocks of 128 rows, of which few are in pieces: 128 rows of 8 heads over 4096 slots 36 us of 54 for workgroups without
// work, listed 8): every workgroup lists the notes that say something, and takes what is its own of them.  (Up to 2048 workgroups 5 us, listed 7.)
constexpr int kMostJoints = 1024;
template <typename T, int ROWS>
__global__ __launch_bounds__(256)
void paged_join_listed_kernel(AttendArgs a, int32_t block_rows, int32_t cols)
{
    __shared__ float tops[256];
    __shared__ float sums[256][5];
    __shared__ uint16_t list[kMostJoints];
    __shared__ int counts[kMostJoints / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    uint64_t some[kMostJoints / 256];
#pragma unroll
    for (int n = 0; n < kMostJoints / 256; ++n) {
        const int w = 256 * n + tid;
        some[n] = __builtin_amdgcn_ballot_w64(w < a.workgroups && a.joints[min(w, a.workgroups - 1)].first >= 0);
        if (lane == 0) counts[4 * n + wave] = __builtin_popcountll(some[n]);
    }
    __syncthreads();
    int count = 0;
#pragma unroll
    for (int n = 0; n < kMostJoints / 256; ++n)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (k == wave && (some[n] >> lane & 1) != 0) list[count + __builtin_popcountll(some[n] & (((uint64_t)1 << lane) - 1))] = (uint16_t)(256 * n + tid);
            count += counts[4 * n + k];
        }
    __syncthreads();
    const int slices = block_rows / ROWS;
    for (int item = blockIdx.x; item < count * slices; item += gridDim.x) {
        const int w = list[item / slices];
        const Joint j = a.joints[w];
        __syncthreads();                          // (the sums of the piece before have been read)
        join_rows<T, ROWS>(a, j, w, item % slices * ROWS, block_rows, cols, tops, sums);
    }
}

inline AttendArgs attend_args(const PagedArgs& p, int workgroups, int rows, int unit, int64_t size)
{
    AttendArgs a;
    a.Q = static_cast<const char*>(p.Q);
    a.O = static_cast<char*>(p.O);
    a.lse = p.lse;
    a.joints = reinterpret_cast<Joint*>(p.workspace);
    a.partial = p.workspace + workgroups * sizeof(Joint) / 4;
    a.starts = p.starts;
    a.q_stride = p.q_stride * size;
    a.tokens = (int32_t)p.tokens;
    a.heads = (int32_t)p.heads;
    a.group = fast_div((uint32_t)(p.heads / p.cache.kv_heads));
    a.cache = p.cache;
    a.rule = p.rule;
    a.workgroups = workgroups;
    a.unit_log = 31 - __builtin_clz(unit);
    const int64_t blocks = (p.tokens * a.group.d / rows + p.cache.batch) * p.cache.kv_heads;
    while (blocks * ((p.cache.slots >> a.unit_log) + 1) >= (int64_t)1 << 31) ++a.unit_log;
    return a;
}

// Two places for every workgroup: of the block that its stretch begins in, and of the one that it ends in.
inline int64_t partial_bytes(int workgroups, int rows, int cols) { return (int64_t)workgroups * (2 * rows * (cols + 2) * 4 + (int64_t)sizeof(Joint)); }

template <typename T> hipError_t launch_join(const AttendArgs& a, int rows, int cols, hipStream_t stream)
{
    // Few blocks are in many parts each: then more workgroups to a block.  4 rows a workgroup / 16, us of attention and join: a token over 16384 slots, one
    // kv head of 128 18.6 / 21.3, 8 kv heads and 4097 slots 12.6 / 12.5; 512 tokens over 14336 slots, 8 kv heads (blocks of 128 rows, before their pieces were listed) 159 / 146.
    const int64_t blocks = ((int64_t)a.tokens * a.group.d / rows + a.cache.batch) * a.cache.kv_heads;
    const int few = blocks * 8 <= a.workgroups ? 4 : 16;
    if (rows > 16 && a.workgroups * (rows / few) > 2048 && a.workgroups <= kMostJoints) {
        // so many pieces there are at most, where starts are in order
        const int64_t pieces = (blocks < a.workgroups ? blocks : a.workgroups) * (rows / few);
        const uint32_t grid = (uint32_t)(pieces < 2048 ? pieces : 2048);
        if (few == 4) paged_join_listed_kernel<T, 4><<<grid, 256, 0, stream>>>(a, rows, cols);
        else paged_join_listed_kernel<T, 16><<<grid, 256, 0, stream>>>(a, rows, cols);
        return hipGetLastError();
    }
    if (few == 4) paged_join_kernel<T, 4><<<dim3(a.workgroups, rows / 4), 256, 0, stream>>>(a, rows, cols);
    else paged_join_kernel<T, 16><<<dim3(a.workgroups, rows / 16), 256, 0, stream>>>(a, rows, cols);
    return hipGetLastError();
}

}  // namespace
}  // namespace attnw
