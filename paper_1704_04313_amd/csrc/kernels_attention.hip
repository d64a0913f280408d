// Linear attention with a decay for each head.
//
// S_t = g S_(t-1) + k_t (x) v_t, o_t = scale q_t S_t: every column of S (an index of v) is a recurrence of its own.
#include "tokens.h"

namespace cbk {
namespace {

// Token after token, the state in registers.  A workgroup holds `columns` columns of one stream's head: DVL lanes side by
// side, VEC columns each, and 256 / DVL groups of lanes that share the rows (RPT each).  Bound by the state's way through memory
// where tokens are few: it is read and written once, whole rows of 16 VEC bytes a group.
template <int DT, int VEC, int DVL, int RPT>
__global__ __launch_bounds__(256) void recurrent_kernel(const cbinfer_linear_attention_args a, int slices)
{
    typedef typename Elem<DT>::type T;
    constexpr int RG = 256 / DVL, C = DVL * VEC;
    __shared__ float qs[256], ks[256], part[4][C];
    const int slice = blockIdx.x % slices, h = (blockIdx.x / slices) % a.heads, b = blockIdx.x / slices / a.heads;
    const int lane = threadIdx.x % DVL, group = threadIdx.x / DVL, c0 = slice * C + lane * VEC;
    const int dk = a.key_size, dv = a.value_size, hk = h / (a.heads / a.kv_heads);
    const int n = a.lengths ? min(max(a.lengths[b], 0), a.tokens) : a.tokens;
    const T *q = static_cast<const T *>(a.q) + b * a.q_stride[0] + h * a.q_stride[2];
    const T *k = static_cast<const T *>(a.k) + b * a.k_stride[0] + hk * a.k_stride[2];
    const T *v = static_cast<const T *>(a.v) + b * a.v_stride[0] + hk * a.v_stride[2];
    T *o = static_cast<T *>(a.o) + b * a.o_stride[0] + h * a.o_stride[2];
    float *state = a.state + ((int64_t)b * a.heads + h) * dk * dv;
    const float g = a.decay[h];

    float S[RPT][VEC];
    if (n > 0) {
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
            const int r = group + i * RG;
            if (VEC == 4) {
                float4 x = make_float4(0, 0, 0, 0);
                if (r < dk && c0 < dv) x = *reinterpret_cast<const float4 *>(state + (int64_t)r * dv + c0);
                S[i][0] = x.x; S[i][1 % VEC] = x.y; S[i][2 % VEC] = x.z; S[i][3 % VEC] = x.w;
            } else {
                S[i][0] = r < dk && c0 < dv ? state[(int64_t)r * dv + c0] : 0.0f;
            }
        }
    }
    for (int t = 0; t < n; ++t) {
        if (threadIdx.x < dk) {
            qs[threadIdx.x] = Elem<DT>::get(q[t * a.q_stride[1] + threadIdx.x]);
            ks[threadIdx.x] = Elem<DT>::get(k[t * a.k_stride[1] + threadIdx.x]);
        }
        float x[VEC], out[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            x[j] = c0 + j < dv ? Elem<DT>::get(v[t * a.v_stride[1] + c0 + j]) : 0.0f;
            out[j] = 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
            const int r = group + i * RG;
            if (r < dk) {
                const float kr = ks[r], qr = qs[r];
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    S[i][j] = __builtin_fmaf(g, S[i][j], kr * x[j]);
                    out[j] = __builtin_fmaf(qr, S[i][j], out[j]);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < VEC; ++j)
            for (int off = DVL; off < 64; off *= 2) out[j] += __shfl_xor(out[j], off);
        if ((threadIdx.x & 63) < DVL)
#pragma unroll
            for (int j = 0; j < VEC; ++j) part[threadIdx.x >> 6][lane * VEC + j] = out[j];
        __syncthreads();
        if (threadIdx.x < C && slice * C + (int)threadIdx.x < dv) {
            const int c = threadIdx.x;
            o[t * a.o_stride[1] + slice * C + c] = Elem<DT>::put(a.scale * ((part[0][c] + part[1][c]) + (part[2][c] + part[3][c])));
        }
    }
    for (int t = n; t < a.tokens; ++t)
        if (threadIdx.x < C && slice * C + (int)threadIdx.x < dv) o[t * a.o_stride[1] + slice * C + threadIdx.x] = Elem<DT>::put(0.0f);
    if (n > 0) {
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
            const int r = group + i * RG;
            if (r < dk && c0 < dv) {
                if (VEC == 4)
                    *reinterpret_cast<float4 *>(state + (int64_t)r * dv + c0) = make_float4(S[i][0], S[i][1 % VEC], S[i][2 % VEC], S[i][3 % VEC]);
                else
                    state[(int64_t)r * dv + c0] = S[i][0];
            }
        }
    }
}

template <int DT, int VEC, int DVL>
hipError_t recurrent(hipStream_t st, const cbinfer_linear_attention_args &a)
{
    constexpr int RG = 256 / DVL, C = DVL * VEC;
    const int slices = (a.value_size + C - 1) / C, rows = (a.key_size + RG - 1) / RG;
    const dim3 grid((unsigned)a.streams * a.heads * slices);
    if (rows <= 64 / RG)
        recurrent_kernel<DT, VEC, DVL, 64 / RG><<<grid, 256, 0, st>>>(a, slices);
    else if (rows <= 128 / RG)
        recurrent_kernel<DT, VEC, DVL, 128 / RG><<<grid, 256, 0, st>>>(a, slices);
    else
        recurrent_kernel<DT, VEC, DVL, 256 / RG><<<grid, 256, 0, st>>>(a, slices);
    return hipGetLastError();
}

template <int DT>
hipError_t recurrent_any(hipStream_t st, const cbinfer_linear_attention_args &a)
{
    const bool whole = a.value_size % 4 == 0 && reinterpret_cast<uintptr_t>(a.state) % 16 == 0;
    if (!whole) return recurrent<DT, 1, 32>(st, a);
    return recurrent<DT, 4, 8>(st, a);
}

} // namespace

size_t linear_attention_workspace(const cbinfer_linear_attention_args &) { return 0; }

hipError_t linear_attention(hipStream_t st, const cbinfer_linear_attention_args &a)
{
    return a.dtype == kF32 ? recurrent_any<kF32>(st, a) : recurrent_any<kBF16>(st, a);
}

} // namespace cbk
