// Rotary positions with several axes: tokens of images and video stand at a height, a width and a time, and every pair of columns turns by one of them.
//
//     (x, y) -> (x cos - y sin, y cos + x sin),   cos, sin: column j of row p of the table, p the token's position on the axis of pair j
//
// (the gradient is the transposed map: the angle's sign changes.)  The table is made once, in 64 bits, and its columns have the frequencies: one run of them over all pairs,
// or one that begins again with each axis.
//
// What bounds it: memory, 2 bytes moved for every byte of the rows; the tables' rows come from the caches.  Measured: 16384 tokens of 16 heads of 128, bf16, 29.7 us = 4.8 TB/s,
// where a copy of 1 GiB reaches 5.1; 1731 tokens of 12 heads of 64, fp32, 4.1 us.
#include "rotary_common.h"

namespace attnw {
namespace {

constexpr int kStaged = 4096;                     // angles in LDS
// MIXED: the pairs of a unit belong to several axes.
template <typename T, int V, bool INTERLEAVED, bool MIXED>
__global__ __launch_bounds__(256)
void rotary_axes_kernel(const T* X, T* Y, const float* __restrict__ angles, AxesView axes, int32_t tokens, int32_t d, int32_t rot, int64_t rows, int64_t x_stride,
                        int64_t y_stride, float sign, TurnUnits u)
{
    __shared__ uint32_t of[8];
    if (threadIdx.x < 8) of[threadIdx.x] = axes.of[threadIdx.x];
    __syncthreads();
    const auto position = [&](int64_t t, int axis) __attribute__((always_inline)) { return (int64_t)axes.positions[axis * axes.tokens + t]; };
    if constexpr (MIXED) {
        __shared__ __align__(32) float staged[kStaged];
        turn_rows_staged<T, V, INTERLEAVED, 1>(X, Y, angles, axes.count, of, staged, position, tokens, d, rot, rows, x_stride, y_stride, sign, u, blockIdx.x, gridDim.x,
                                               blockIdx.y, gridDim.y);
    } else {
        turn_rows<T, V, INTERLEAVED>(X, Y, angles, axes.count, of, position, tokens, d, rot, rows, x_stride, y_stride, sign, u, blockIdx.x, gridDim.x, blockIdx.y, gridDim.y);
    }
}

template <typename T, int V, bool INTERLEAVED> hipError_t launch(const RotaryArgs& a, const AxesView& axes, hipStream_t stream)
{
    const TurnUnits u = turn_units<V, INTERLEAVED>(a.heads, a.d, a.rot, 1, kStaged);
    constexpr int P = V == 1 ? 1 : INTERLEAVED ? V / 2 : V;    // pairs of a unit
    bool mixed = false;
    for (int j = 0; j < a.rot / 2; ++j) mixed |= (axes.of[j / 16] >> 2 * (j % 16) & 3) != (axes.of[j / P * P / 16] >> 2 * (j / P * P % 16) & 3);
    auto go = [&](auto kernel) {
        kernel<<<turn_grid(u, a.tokens), 256, 0, stream>>>(static_cast<const T*>(a.Q), static_cast<T*>(a.R), a.angles, axes, (int32_t)a.tokens, (int32_t)a.d, (int32_t)a.rot, a.rows,
                                                          a.q_stride, a.r_stride, a.inverse ? -1.0f : 1.0f, u);
    };
    // (16384 tokens of 16 heads of 128, sections of 16 and 24 pairs 28.4 us, staged 30.4; 4099 tokens of 20 heads of 80, the axes in turns 12.0, staged 8.2)
    if (V > 1 && mixed) go(rotary_axes_kernel<T, V, INTERLEAVED, (V > 1)>);
    else go(rotary_axes_kernel<T, V, INTERLEAVED, false>);
    return hipGetLastError();
}

// The widest units that rows, halves and the rest are whole ones of.  (8974 tokens of 16 heads of 72, bf16, 18 columns by pairs: two
// at a time 16.1 us, one 26.2; 36 columns by halves, two 17.2, one 24.1.)
template <typename T, int V> hipError_t launch_typed(const RotaryArgs& a, const AxesView& axes, hipStream_t stream)
{
    if constexpr (V > 1)
        if (!turns_by_chunks(V, a.d, a.rot, a.q_stride, a.r_stride, a.interleaved)) return launch_typed<T, V / 2>(a, axes, stream);
    return a.interleaved ? launch<T, V, true>(a, axes, stream) : launch<T, V, false>(a, axes, stream);
}

// step[j]: the exponent of 2 that column j's frequency is the inverse of
struct Steps { double of[128]; };

__global__ __launch_bounds__(256)
void rotary_axes_table_kernel(float* table, int64_t positions, int32_t half, Steps step, double factor, double low, double high, double original, double gain)
{
    __shared__ double of[128];
    if (threadIdx.x < 128) of[threadIdx.x] = step.of[threadIdx.x];
    __syncthreads();
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < positions * half; i += (int64_t)gridDim.x * 256) {
        const int64_t p = i / half;
        const int32_t j = (int32_t)(i - p * half);
        double s, c;
        sincospi(rotary_half_turns(p, of[j], factor, low, high, original), &s, &c);
        table[p * 2 * half + j] = (float)(gain * c);
        table[p * 2 * half + half + j] = (float)(gain * s);
    }
}

}  // namespace

hipError_t launch_rotary_axes(const RotaryArgs& a, const AxesMap& map, hipStream_t stream)
{
    const AxesView axes = axes_view(map, a.positions, a.tokens);
    return a.dt == DType::F32 ? launch_typed<float, 4>(a, axes, stream) : launch_typed<uint16_t, 8>(a, axes, stream);
}

hipError_t launch_rotary_axes_table(float* table, const AxesMap& map, int64_t positions, int64_t rot, double base, double factor, double low, double high, double original,
                                    double gain, hipStream_t stream)
{
    const int32_t half = (int32_t)(rot / 2);
    Steps step{};
    for (int j = 0; j < half; ++j) step.of[j] = log2(base) * (map.fresh ? (double)map.index[j] / map.pairs[map.axis[j]] : (double)j / half);
    const int64_t blocks = (positions * half + 255) / 256;
    rotary_axes_table_kernel<<<dim3((uint32_t)(blocks < 1 << 16 ? blocks : 1 << 16)), 256, 0, stream>>>(table, positions, half, step, factor, low, high, original, gain);
    return hipGetLastError();
}

}  // namespace attnw
