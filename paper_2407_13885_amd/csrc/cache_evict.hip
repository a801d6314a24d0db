// Eviction from a paged cache: of every sequence and kv head the last `recent` slots stay, and of the others those that collected the most weight, as
// many as `keep` has room for (equal ones: the lower slot; NaN counts as less than anything), in their order, in other pages.
//
// First launch, a workgroup per (sequence, kv head): the smallest sum that stays is found digit by digit (8 bits of the sums, mapped to whole numbers
// of the same order, in 256 counters on chip, four times), and the slots that stay are written in order.  Second launch: their rows of K and V, and their sums, are moved.
// What bounds them: the chain of the four counts; the bytes moved.
#include "paged_common.h"

namespace attnw {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;

__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t u = __float_as_uint(x == 0.0f ? 0.0f : x);   // (-0 is 0)
    if (x != x) return 0;
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__global__ __launch_bounds__(kThreads)
void evict_select_kernel(CacheView from, const float* __restrict__ sums, int32_t* __restrict__ kept, int32_t keep, int32_t recent)
{
    __shared__ uint32_t bins[256];
    __shared__ uint32_t above[kWaves], equal[kWaves];
    __shared__ uint32_t digit, left;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int b = blockIdx.x / from.kv_heads;
    const int n = max(0, min(from.lengths[b], from.slots));
    const float* const x = sums + (int64_t)blockIdx.x * from.slots;
    int32_t* const out = kept + (int64_t)blockIdx.x * keep;
    if (n <= keep) {
        for (int i = tid; i < keep; i += kThreads) out[i] = i < n ? i : -1;
        return;
    }
    const int old = n - recent;                   // slots that may go
    uint32_t want = keep - recent;                // of them stay
    for (int i = tid; i < recent; i += kThreads) out[want + i] = old + i;
    if (want == 0) return;

    uint32_t prefix = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) bins[tid] = 0;
        __syncthreads();
        for (int i = tid; i < old; i += kThreads) {
            const uint32_t u = ordered(x[i]);
            if (shift == 24 || (u >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&bins[(u >> shift) & 255], 1u);
        }
        __syncthreads();
        if (wave == 0) {                          // four bins a lane, from the highest
            uint32_t c[4], sum = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) sum += c[k] = bins[255 - 4 * lane - k];
            uint32_t upto = sum;
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) {
                const uint32_t o = __shfl_up(upto, off, 64);
                if (lane >= off) upto += o;
            }
            uint32_t seen = upto - sum;
            if (seen < want && upto >= want) {    // (one lane)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (seen < want && seen + c[k] >= want) {
                        digit = 255 - 4 * lane - k;
                        left = want - seen;
                    }
                    seen += c[k];
                }
            }
        }
        __syncthreads();
        prefix |= digit << shift;
        want = left;                              // of those with these digits
    }
    // The waves have consecutive ranges, of whole 64s.  Counted first, then written.
    const int share = ((old + kWaves - 1) / kWaves + 63) & ~63;
    const int i0 = min(old, wave * share), i1 = min(old, i0 + share);
    uint32_t more = 0, same = 0;
    for (int i = i0; i < i1; i += 64) {
        const uint32_t u = i + lane < i1 ? ordered(x[i + lane]) : 0u;
        const bool in = i + lane < i1;
        more += __builtin_popcountll(__builtin_amdgcn_ballot_w64(in && u > prefix));
        same += __builtin_popcountll(__builtin_amdgcn_ballot_w64(in && u == prefix));
    }
    if (lane == 0) {
        above[wave] = more;
        equal[wave] = same;
    }
    __syncthreads();
    uint32_t to = 0, ties = 0;                    // before the wave's range: written, equal to the smallest that stays
    for (int k = 0; k < wave; ++k) {
        to += above[k];
        ties += equal[k];
    }
    to += min(ties, want);
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    for (int i = i0; i < i1; i += 64) {
        const bool in = i + lane < i1;
        const uint32_t u = in ? ordered(x[i + lane]) : 0u;
        const uint64_t eq = __builtin_amdgcn_ballot_w64(in && u == prefix);
        const bool stays = in && (u > prefix || (u == prefix && ties + __builtin_popcountll(eq & below) < want));
        const uint64_t st = __builtin_amdgcn_ballot_w64(stays);
        if (stays) out[to + __builtin_popcountll(st & below)] = i + lane;
        to += __builtin_popcountll(st);
        ties += __builtin_popcountll(eq);
    }
}

// A thread moves 16 bytes of K and of V.
__global__ __launch_bounds__(256)
void evict_move_kernel(CacheView from, CacheView into, int32_t* into_lengths, const float* __restrict__ sums, float* __restrict__ into_sums,
                       const int32_t* __restrict__ kept, int32_t keep, int32_t chunks, FastDiv by_chunk, uint32_t per_head)
{
    const uint32_t bh = blockIdx.x / per_head;
    const uint32_t first = (blockIdx.x - bh * per_head) * 256 + threadIdx.x;
    const int b = bh / from.kv_heads, h = bh - b * from.kv_heads;
    if (h == 0 && first == 0) into_lengths[b] = min(keep, max(0, min(from.lengths[b], from.slots)));
    for (uint32_t i = first;; i += per_head * 256) {
        const uint32_t row = quotient(i, by_chunk), c = i - row * chunks;
        if (row >= (uint32_t)keep) return;
        const int32_t slot = kept[(int64_t)bh * keep + row];
        if (slot < 0) return;                     // (and none behind it)
        if (c == 0) into_sums[(int64_t)bh * into.slots + row] = sums[(int64_t)bh * from.slots + slot];
        const uint32_t p = quotient(row, into.page);
        const int32_t id = into.table[(int64_t)b * into.max_pages + p];
        if ((uint32_t)id >= (uint32_t)into.pages) continue;    // no such page: nothing is moved
        const int64_t to = (int64_t)((uint64_t)(uint32_t)id * into.page_bytes) + (uint32_t)h * into.head_bytes + (row - p * into.page.d) * (uint32_t)into.row_bytes + c * 16;
        const int64_t at = slot_offset(from, from.table + (int64_t)b * from.max_pages, h, slot) + c * 16;
        const uint4 k = *reinterpret_cast<const uint4*>(from.K + at), v = *reinterpret_cast<const uint4*>(from.V + at);
        *reinterpret_cast<uint4*>(const_cast<char*>(into.K) + to) = k;
        *reinterpret_cast<uint4*>(const_cast<char*>(into.V) + to) = v;
    }
}

}  // namespace

hipError_t launch_evict(const CacheView& from, const CacheView& into, int32_t* into_lengths, const float* sums, float* into_sums, int32_t* kept,
                        int64_t keep, int64_t recent, hipStream_t stream)
{
    const uint32_t heads = (uint32_t)((int64_t)from.batch * from.kv_heads);
    evict_select_kernel<<<heads, kThreads, 0, stream>>>(from, sums, kept, (int32_t)keep, (int32_t)recent);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int32_t chunks = from.row_bytes / 16;
    // (a launch has less than 2^32 threads)
    const int64_t per_head64 = (keep * chunks + 255) / 256, most = ((int64_t)1 << 23) / heads;
    const uint32_t per_head = (uint32_t)(per_head64 < most ? per_head64 : most > 0 ? most : 1);
    evict_move_kernel<<<heads * per_head, 256, 0, stream>>>(from, into, into_lengths, sums, into_sums, kept, (int32_t)keep, chunks, fast_div(chunks), per_head);
    return hipGetLastError();
}

}  // namespace attnw
