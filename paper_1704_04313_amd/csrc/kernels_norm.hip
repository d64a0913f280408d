// Norm behind a block, its gate and residual scale, and the norm in front of the next block, in one pass: the row is read
// once and stays on the chip until both outputs are written.
#include "tokens.h"

namespace cbk {
namespace {

__device__ __forceinline__ float wave_sum(float v)
{
    for (int off = 32; off; off >>= 1) v += __shfl_xor(v, off);
    return v;
}

// Sum over the workgroup of 256; every thread gets it.
__device__ __forceinline__ float block_sum(float v, float *scratch)
{
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
    __syncthreads();
    return (scratch[0] + scratch[1]) + (scratch[2] + scratch[3]);
}

__device__ __forceinline__ float gate_of(float g, int kind)
{
    const float open = 1.0f / (1.0f + __expf(-g));
    return kind == CBINFER_GATE_SIGMOID ? open : g * open;
}

// Any size, group, stride and alignment: the row lies in LDS as float32.
template <int DT, int DS>
__global__ __launch_bounds__(256) void norm_row_kernel(const cbinfer_gated_norm_args a)
{
    typedef typename Elem<DT>::type T;
    typedef typename Elem<DS>::type R;
    extern __shared__ float row[]; // size values, then a factor for each group, then four sums
    const int d = (int)a.size, group = a.group ? a.group : d, groups = d / group, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    float *factor = row + d, *scratch = factor + groups;
    const int64_t r = blockIdx.x;
    const T *x = static_cast<const T *>(a.x) + r * a.x_stride;
    const T *gate = static_cast<const T *>(a.gate) + r * a.gate_stride;
    const R *residual = static_cast<const R *>(a.residual) + r * a.residual_stride;
    R *h = static_cast<R *>(a.h) + r * a.h_stride;
    T *y = static_cast<T *>(a.y) + r * a.y_stride;
    for (int i = threadIdx.x; i < d; i += 256) row[i] = Elem<DT>::get(x[i]);
    __syncthreads();
    if (a.weight) {
        for (int g = wave; g < groups; g += 4) {
            float s = 0.0f;
            for (int i = lane; i < group; i += 64) s = __builtin_fmaf(row[g * group + i], row[g * group + i], s);
            s = wave_sum(s);
            if (lane == 0) factor[g] = 1.0f / sqrtf(s / group + a.eps);
        }
        __syncthreads();
    }
    float sum = 0.0f;
    for (int i = threadIdx.x; i < d; i += 256) {
        float u = row[i];
        if (a.weight) u *= factor[i / group] * a.weight[i];
        if (a.gate) u *= gate_of(Elem<DT>::get(gate[i]), a.gate_kind);
        u *= a.scale;
        if (a.channel_scale) u *= a.channel_scale[i];
        if (a.residual) u += Elem<DS>::get(residual[i]);
        if (a.h) h[i] = Elem<DS>::put(u);
        row[i] = u;
        sum = __builtin_fmaf(u, u, sum);
    }
    if (!a.y) return;
    sum = block_sum(sum, scratch);
    const float f = 1.0f / sqrtf(sum / d + a.eps);
    for (int i = threadIdx.x; i < d; i += 256) y[i] = Elem<DT>::put(row[i] * f * a.next_weight[i]);
}

} // namespace

hipError_t gated_norm(hipStream_t st, const cbinfer_gated_norm_args &a)
{
    const int groups = a.group ? (int)(a.size / a.group) : 1;
    const size_t lds = (size_t)(a.size + groups + 4) * sizeof(float);
    const dim3 grid((unsigned)a.rows);
    auto kernel = a.dtype == kF32 ? norm_row_kernel<kF32, kF32> : a.sum_dtype == kF32 ? norm_row_kernel<kBF16, kF32> : norm_row_kernel<kBF16, kBF16>;
    if (lds > 65536)
        if (hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds)) return e;
    kernel<<<grid, 256, lds, st>>>(a);
    return hipGetLastError();
}

} // namespace cbk
