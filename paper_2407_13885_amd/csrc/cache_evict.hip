// Eviction from a paged cache: of every sequence and kv head the last `recent` slots stay, and of the others those that collected the most weight, as
// many as `keep` has room for (equal ones: the lower slot; NaN counts as less than anything), in their order, in other pages.
//
// First launch, a workgroup per (sequence, kv head): the smallest sum that stays is found digit by digit (11, 11 and 10 bits of the sums, mapped to whole
// numbers of the same order, counted on chip: the first digit holds the exponent and two bits more, so that sums of all sizes do not meet in a few counters), and the slots
// that stay are written in order.  Sums of up to 32768 slots wait in registers meanwhile.  Second launch: their rows of K and V, and their sums, are moved.
// What bounds them: the chain of three counts; the bytes moved.
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

// The sum of what the waves before this one counted.
__device__ __forceinline__ uint32_t of_waves_before(const uint32_t (&counts)[kWaves], int wave)
{
    uint32_t sum = 0;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) sum += k < wave ? counts[k] : 0u;
    return sum;
}

// HELD: elements of a thread that wait in registers, 0: all are read again in each pass.
template <int HELD>
__global__ __launch_bounds__(kThreads)
void evict_select_kernel(CacheView from, const float* __restrict__ sums, int32_t* __restrict__ kept, int32_t keep, int32_t recent)
{
    constexpr int BINS = 2048;
    __shared__ uint32_t bins[BINS];
    __shared__ __align__(16) uint32_t above[kWaves], equal[kWaves];
    __shared__ uint32_t found[2];                 // the digit, and how many of those that have it stay
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
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

    // The waves have consecutive ranges, of whole 64s.
    const int share = ((old + kWaves - 1) / kWaves + 63) & ~63;
    const int i0 = min(old, wave * share), i1 = min(old, i0 + share);
    uint32_t held[HELD > 0 ? HELD : 1];
    if constexpr (HELD > 0) {
#pragma unroll
        for (int k = 0; k < HELD; ++k) held[k] = i0 + k * 64 + lane < i1 ? ordered(x[i0 + k * 64 + lane]) : 0u;
    }
    // f(number, whether there is one, its slot) for all that a lane has, 64 consecutive slots at a time
    const auto each = [&](auto&& f) __attribute__((always_inline)) {
        if constexpr (HELD > 0) {
#pragma unroll
            for (int k = 0; k < HELD; ++k)
                if (i0 + k * 64 < i1) f(held[k], i0 + k * 64 + lane < i1, i0 + k * 64 + lane);
        } else {
            for (int i = i0; i < i1; i += 64) f(i + lane < i1 ? ordered(x[i + lane]) : 0u, i + lane < i1, i + lane);
        }
    };

    uint32_t prefix = 0;
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, before = pass == 0 ? 32 : pass == 1 ? 21 : 10;
        for (int i = tid; i < BINS; i += kThreads) bins[i] = 0;
        __syncthreads();
        each([&](uint32_t u, bool in, int) __attribute__((always_inline)) {
            if (in && (pass == 0 || u >> before == prefix >> before)) atomicAdd(&bins[(u >> shift) & (BINS - 1)], 1u);
        });
        __syncthreads();
        // two bins a thread, from the highest: which one the last that stays is in
        const uint32_t hi = bins[BINS - 1 - 2 * tid], lo = bins[BINS - 2 - 2 * tid];
        uint32_t upto = hi + lo;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const uint32_t o = __shfl_up(upto, off, 64);
            if (lane >= off) upto += o;
        }
        if (lane == 63) above[wave] = upto;
        __syncthreads();
        uint32_t seen = upto - hi - lo + of_waves_before(above, wave);
        if (seen < want && seen + hi + lo >= want) {           // (one thread)
            const bool first = seen + hi >= want;
            found[0] = BINS - 1 - 2 * tid - (first ? 0 : 1);
            found[1] = want - seen - (first ? 0 : hi);
        }
        __syncthreads();
        prefix |= found[0] << shift;
        want = found[1];
    }
    // Counted first, then written.
    uint32_t more = 0, same = 0;
    each([&](uint32_t u, bool in, int) __attribute__((always_inline)) {
        more += __builtin_popcountll(__builtin_amdgcn_ballot_w64(in && u > prefix));
        same += __builtin_popcountll(__builtin_amdgcn_ballot_w64(in && u == prefix));
    });
    if (lane == 0) {
        above[wave] = more;
        equal[wave] = same;
    }
    __syncthreads();
    // before the wave's range: equal to the smallest that stays, staying
    uint32_t ties = of_waves_before(equal, wave), to = of_waves_before(above, wave) + min(ties, want);
    const auto below = [](uint64_t m) __attribute__((always_inline)) {
        return (uint32_t)__builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
    };
    each([&](uint32_t u, bool in, int slot) __attribute__((always_inline)) {
        const uint64_t eq = __builtin_amdgcn_ballot_w64(in && u == prefix);
        const bool stays = in && (u > prefix || (u == prefix && ties + below(eq) < want));
        const uint64_t st = __builtin_amdgcn_ballot_w64(stays);
        if (stays) out[to + below(st)] = slot;
        to += __builtin_popcountll(st);
        ties += __builtin_popcountll(eq);
    });
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
    // By the slots that a sequence can have.  In registers / read in each pass, us with the moves: 32 sequences, 8 kv heads, 4096 slots 15 / 17, 16384
    // 27 / 35, 32768 44 / 56.  More registers than needed cost: 4096 slots by 16 a thread 18, 16384 by 32 32.
    if (from.slots <= 4 * kThreads) evict_select_kernel<4><<<heads, kThreads, 0, stream>>>(from, sums, kept, (int32_t)keep, (int32_t)recent);
    else if (from.slots <= 16 * kThreads) evict_select_kernel<16><<<heads, kThreads, 0, stream>>>(from, sums, kept, (int32_t)keep, (int32_t)recent);
    else if (from.slots <= 32 * kThreads) evict_select_kernel<32><<<heads, kThreads, 0, stream>>>(from, sums, kept, (int32_t)keep, (int32_t)recent);
    else evict_select_kernel<0><<<heads, kThreads, 0, stream>>>(from, sums, kept, (int32_t)keep, (int32_t)recent);
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
