// Norm behind a block, its gate and residual scale, and the norm in front of the next block, in one pass: the row is read
// once and stays on the chip until both outputs are written.
#include "tokens.h"

#include <algorithm>

namespace cbk {
namespace {

__device__ __forceinline__ float wave_sum(float v)
{
    for (int off = 32; off; off >>= 1) v += __shfl_xor(v, off);
    return v;
}

// Sum over a workgroup of 256; every thread gets it.
__device__ __forceinline__ float block_sum(float v, float *scratch)
{
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
    __syncthreads();
    return (scratch[0] + scratch[1]) + (scratch[2] + scratch[3]);
}

// exp(-|g|), which never overflows, so that gates far below zero keep their bits down to the smallest number.  As the square of
// 2^(-|g| log2(e) / 2), which is a normal number wherever the square is any; log2(e) / 2 in two parts, the first of which times a bfloat16
// is exact, and what its product with a float32 is rounded by, make up for an exponent that would be off by up to 2^-18.  A gate is off
// by 2^-21 of itself at most.
template <int DT>
__device__ __forceinline__ float exp_down(float g)
{
    constexpr double kHalf = 0.72134752044448170368, kLn4 = 1.38629436111989061883;
    constexpr float kFirst = DT == kBF16 ? 47274.0f / 65536.0f : (float)kHalf, kRest = (float)((kHalf - kFirst) * kLn4);
    static_assert(DT != kBF16 || kRest > 0.0f, "a factor below 1");
    const float a = -fabsf(g), t = a * kFirst, e = __builtin_amdgcn_exp2f(t);
    float f = __builtin_fmaf(a, kRest, 1.0f);
    if (DT == kF32) f = __builtin_fmaf(__builtin_fmaf(a, kFirst, -t), (float)kLn4, f);
    f = DT == kF32 ? __builtin_amdgcn_fmed3f(f, 0.5f, 2.0f) : __builtin_amdgcn_fmed3f(f, 0.0f, 1.0f); // infinite or NaN where g is infinite, and e is 0
    return e * e * f;
}

template <int DT>
__device__ __forceinline__ float gate_of(float g, int kind)
{
    const float e = exp_down<DT>(g), most = __builtin_amdgcn_rcpf(1.0f + e), open = g < 0.0f ? e * most : most;
    return kind == CBINFER_GATE_SIGMOID ? open : g * open;
}

// Groups of any size: the row lies in LDS as float32.  One value a thread and load: 8192 rows of 4095 bfloat16 with a gate and groups of
// 45 155 us, where rows of 4096 in groups of 64 take 43 in the kernel below.
template <int DT, int DS>
__global__ __launch_bounds__(256) void norm_row_kernel(const cbinfer_gated_norm_args a, int64_t first)
{
    typedef typename Elem<DT>::type T;
    typedef typename Elem<DS>::type R;
    extern __shared__ float row[]; // size values, then a factor for each group, then four sums
    const int d = (int)a.size, group = a.group ? a.group : d, groups = d / group, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    float *factor = row + d, *scratch = factor + groups;
    const int64_t r = first + blockIdx.x;
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
        if (a.gate) u *= gate_of<DT>(Elem<DT>::get(gate[i]), a.gate_kind);
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

// Eight values as they lie in memory, 16 bytes at a time, at any address.
template <int DT>
struct Eight {
    typedef typename Elem<DT>::type T;
    typedef unsigned Words __attribute__((ext_vector_type(4), aligned(2)));
    uint4 u[DT == kF32 ? 2 : 1];
    __device__ __forceinline__ void load(const T *p)
    {
#pragma unroll
        for (int i = 0; i < (DT == kF32 ? 2 : 1); ++i) {
            const Words w = *reinterpret_cast<const Words *>(p + 4 * i);
            u[i] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    __device__ __forceinline__ void load(const T *p, int n) // of them n, then zeros
    {
        union { T e[8]; uint4 u[DT == kF32 ? 2 : 1]; } v;
#pragma unroll
        for (int e = 0; e < 8; ++e) v.e[e] = e < n ? p[e] : T(0);
#pragma unroll
        for (int i = 0; i < (DT == kF32 ? 2 : 1); ++i) u[i] = v.u[i];
    }
    __device__ __forceinline__ float get(int e) const { return Unit<DT>::get(u[DT == kF32 ? e / 4 : 0], DT == kF32 ? e % 4 : e); }
    static __device__ __forceinline__ void store(T *p, const float (&v)[8])
    {
        if constexpr (DT == kF32) {
#pragma unroll
            for (int i = 0; i < 8; i += 4)
                *reinterpret_cast<Words *>(p + i) = Words{__float_as_uint(v[i]), __float_as_uint(v[i + 1]), __float_as_uint(v[i + 2]), __float_as_uint(v[i + 3])};
        } else {
            *reinterpret_cast<Words *>(p) = Words{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
        }
    }
    static __device__ __forceinline__ void store(T *p, const float (&v)[8], int n)
    {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) p[e] = Elem<DT>::put(v[e]);
    }
};

// Groups of whole eights, or the row as one: a wave a row (MOST 64, four rows a workgroup) or a workgroup of up to MOST threads, as
// many waves as the row needs; NV times eight values a thread, in registers from the first load to the last store.  A workgroup goes on to further rows with the weights it has.  Bound by memory: 8192 rows of 4096
// with a float32 residual and both norms, 470 MB, 96 us.  TAIL: the last eight of a row is not whole.
template <int DT, int DS, int MOST, int NV, bool TAIL>
__global__ __launch_bounds__(MOST < 256 ? 256 : MOST) void norm_kernel(const cbinfer_gated_norm_args a)
{
    typedef typename Elem<DT>::type T;
    typedef typename Elem<DS>::type R;
    constexpr int ROWS = MOST < 256 ? 256 / MOST : 1, WAVES = MOST / 64;
    __shared__ float scratch[2][WAVES];
    const int threads = ROWS > 1 ? MOST : blockDim.x; // of a row
    extern __shared__ float squares[]; // sums of eight squares, where a group is not a power of two lanes
    const int d = (int)a.size, thread = ROWS > 1 ? threadIdx.x % MOST : threadIdx.x, lane = threadIdx.x & 63, wave = thread >> 6, eights = (d + 7) / 8;
    const int share = a.group && a.group != d ? a.group / 8 : eights; // eights of a group
    const bool by_lanes = share <= 64 && (share & (share - 1)) == 0, by_row = share == eights;
    int at[NV];
    bool there[NV];
    float w[NV][8], scale[NV][8], next[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        at[i] = (i * threads + thread) * 8;
        there[i] = at[i] < d;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bool is = TAIL ? at[i] + e < d : there[i];
            w[i][e] = is && a.weight ? a.weight[at[i] + e] : 1.0f;
            scale[i][e] = is && a.channel_scale ? a.scale * a.channel_scale[at[i] + e] : a.scale;
            next[i][e] = is && a.y ? a.next_weight[at[i] + e] : 0.0f;
        }
    }
    auto row_sum = [&](float v, int which) {
        v = wave_sum(v);
        if (WAVES > 1) {
            if (lane == 0) scratch[which][wave] = v;
            __syncthreads();
            v = 0.0f;
#pragma unroll
            for (int i = 0; i < WAVES; ++i) v += i * 64 < threads ? scratch[which][i] : 0.0f;
        }
        return v;
    };
    for (int64_t r = (int64_t)blockIdx.x * ROWS + (ROWS > 1 ? threadIdx.x / MOST : 0); r < a.rows; r += (int64_t)gridDim.x * ROWS) {
        const T *x = static_cast<const T *>(a.x) + r * a.x_stride, *gate = static_cast<const T *>(a.gate) + r * a.gate_stride;
        const R *residual = static_cast<const R *>(a.residual) + r * a.residual_stride;
        Eight<DT> xs[NV], gs[NV];
        Eight<DS> rs[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (TAIL && at[i] + 8 > d) {
                xs[i].load(x + at[i], d - at[i]);
                if (a.gate) gs[i].load(gate + at[i], d - at[i]);
                if (a.residual) rs[i].load(residual + at[i], d - at[i]);
            } else if (there[i]) {
                xs[i].load(x + at[i]);
                if (a.gate) gs[i].load(gate + at[i]);
                if (a.residual) rs[i].load(residual + at[i]);
            }
        float u[NV][8], f[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            f[i] = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                u[i][e] = there[i] ? xs[i].get(e) : 0.0f;
                f[i] = __builtin_fmaf(u[i][e], u[i][e], f[i]);
            }
        }
        if (a.weight) {
            if (by_row) {
                float s = 0.0f;
#pragma unroll
                for (int i = 0; i < NV; ++i) s += f[i];
                s = row_sum(s, 0);
#pragma unroll
                for (int i = 0; i < NV; ++i) f[i] = s;
            } else if (by_lanes) {
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    for (int off = share / 2; off; off >>= 1) f[i] += __shfl_xor(f[i], off);
            } else {
                float *mine = squares + (ROWS > 1 ? threadIdx.x / MOST : 0) * eights;
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if (there[i]) mine[at[i] / 8] = f[i];
                if (WAVES > 1) __syncthreads(); else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if (there[i]) {
                        const int from = at[i] / 8 / share * share;
                        f[i] = 0.0f;
                        for (int j = 0; j < share; ++j) f[i] += mine[from + j];
                    }
                if (WAVES > 1) __syncthreads(); else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            }
            const float each = by_row ? d : 8 * share;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                f[i] = 1.0f / sqrtf(f[i] / each + a.eps);
#pragma unroll
                for (int e = 0; e < 8; ++e) u[i][e] *= f[i] * w[i][e];
            }
        }
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (there[i]) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (a.gate) u[i][e] *= gate_of<DT>(gs[i].get(e), a.gate_kind);
                    u[i][e] = a.residual ? __builtin_fmaf(u[i][e], scale[i][e], rs[i].get(e)) : u[i][e] * scale[i][e];
                    sum = __builtin_fmaf(u[i][e], u[i][e], sum);
                }
                R *h = static_cast<R *>(a.h) + r * a.h_stride + at[i];
                if (TAIL && at[i] + 8 > d) {
                    if (a.h) Eight<DS>::store(h, u[i], d - at[i]);
                } else if (a.h) {
                    Eight<DS>::store(h, u[i]);
                }
            }
        if (a.y) {
            sum = row_sum(sum, 1);
            const float g = 1.0f / sqrtf(sum / d + a.eps);
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (there[i]) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) u[i][e] *= g * next[i][e];
                    T *y = static_cast<T *>(a.y) + r * a.y_stride + at[i];
                    if (TAIL && at[i] + 8 > d)
                        Eight<DT>::store(y, u[i], d - at[i]);
                    else
                        Eight<DT>::store(y, u[i]);
                }
        }
        if (WAVES > 1) __syncthreads(); // the sums are read before the next row's come
    }
}

template <int DT, int DS, bool TAIL>
hipError_t by_eights(hipStream_t st, const cbinfer_gated_norm_args &a)
{
    const int eights = (int)((a.size + 7) / 8);
    const size_t lds = a.weight && a.group && a.group != a.size ? (size_t)eights * sizeof(float) : 0;
    // A workgroup reads the weights once for all its rows: few of them pay, if they still cover the memory's latency.  us with 1024, 2048, 4096
    // and 8192 waves.  Gate, float32 residual and both norms: 8192 rows of 4096 bfloat16 126, 97, 111, 117, float32 147, 132, 141, 152; 8192 of 768
    // 36, 23, 24, 29; 3000 of 8192 86, 87, 88, 102.  A gate alone: 8192 of 4096 in groups of 64 81, 53, 43, 44; 8192 of 2048 in groups of 128 44, 27,
    // 23, 25, float32 58, 36, 37, 40; 3000 of 8192 40, 40, 34, 37.
    const int waves = a.y ? 2048 : 4096;
    // 8192 rows of 768 bfloat16, a residual and both norms: two waves a row 23 us, four 34
    const int threads = eights <= 64 ? 256 : ((eights <= 256 ? eights : (eights + 1) / 2) + 63) / 64 * 64, rows = eights <= 64 ? 4 : 1;
    const int each = std::max(1, (waves * 64 + 128 * threads) / (256 * threads)); // of a compute unit, all the same
    const unsigned blocks = (unsigned)std::min<int64_t>((a.rows + rows - 1) / rows, 256 * each);
    if (eights <= 64)
        norm_kernel<DT, DS, 64, 1, TAIL><<<blocks, threads, 4 * lds, st>>>(a);
    else if (eights <= 256)
        norm_kernel<DT, DS, 256, 1, TAIL><<<blocks, threads, lds, st>>>(a);
    else if (eights <= 512)
        norm_kernel<DT, DS, 256, 2, TAIL><<<blocks, threads, lds, st>>>(a);
    else if (eights <= 1024)
        norm_kernel<DT, DS, 512, 2, TAIL><<<blocks, threads, lds, st>>>(a);
    else
        norm_kernel<DT, DS, 1024, 2, TAIL><<<blocks, threads, lds, st>>>(a);
    return hipGetLastError();
}

template <bool TAIL>
hipError_t by_eights(hipStream_t st, const cbinfer_gated_norm_args &a)
{
    return a.dtype == kF32 ? by_eights<kF32, kF32, TAIL>(st, a) : a.sum_dtype == kF32 ? by_eights<kBF16, kF32, TAIL>(st, a) : by_eights<kBF16, kBF16, TAIL>(st, a);
}

constexpr int64_t kMostBlocks = 1 << 22; // of a launch: threads are counted in 32 bits

} // namespace

hipError_t gated_norm(hipStream_t st, const cbinfer_gated_norm_args &a)
{
    if (a.group == 0 || a.group == a.size || a.group % 8 == 0) return a.size % 8 == 0 ? by_eights<false>(st, a) : by_eights<true>(st, a);
    const int groups = a.group ? (int)(a.size / a.group) : 1;
    const size_t lds = (size_t)(a.size + groups + 4) * sizeof(float);
    auto kernel = a.dtype == kF32 ? norm_row_kernel<kF32, kF32> : a.sum_dtype == kF32 ? norm_row_kernel<kBF16, kF32> : norm_row_kernel<kBF16, kBF16>;
    if (lds > 65536)
        if (hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds)) return e;
    for (int64_t first = 0; first < a.rows; first += kMostBlocks) {
        kernel<<<(unsigned)std::min(kMostBlocks, a.rows - first), 256, lds, st>>>(a, first);
        if (hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

} // namespace cbk
