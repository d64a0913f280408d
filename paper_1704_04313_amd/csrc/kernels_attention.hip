// Linear attention with a decay for each head.
//
// S_t = g S_(t-1) + k_t (x) v_t, o_t = scale q_t S_t: every column of S (an index of v) is a recurrence of its own.
#include "tokens.h"

#include <algorithm>
#include <cstdlib>

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


// ---- prompts: 64 tokens at a time ----------------------------------------------------------------
// With i and j counting the m tokens of a chunk and S the state in front of it,
//   O = diag(g^(i+1)) (Q S) + (Q K^T o g^(i-j), i >= j) V        S' = g^m S + K^T diag(g^(m-1-j)) V
// are matrix products.  A workgroup takes a stream's head and 32 columns of v a wave; each wave keeps its columns of S in the
// accumulators of the matrix instruction from chunk to chunk, and uses them as an operand as they lie there: the order in
// which a sum over rows of S runs is free, so Q is read in the order that the accumulators have.  Q, K, V and the
// scores lie in LDS, the next chunk's are on their way in registers.
//
// bfloat16: what is computed on the way enters a product as a sum of bfloat16 -- scores and states two (16 bits are kept;
// the output keeps 8), the faded values, from which the state is added up, three (24 bits, exact).  float32: the float32
// instruction.
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kChunk = 64;

__device__ __forceinline__ f32x16 multiply(const u32x4 &a, const u32x4 &b, const f32x16 &c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 multiply(float a, float b, const f32x16 &c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }

// The upper halves of two words: the first in the lower half.
__device__ __forceinline__ unsigned upper_halves(float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u); }
__device__ __forceinline__ float cut(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }

// Eight floats as a sum of PARTS bfloat16: cut off, the last one rounded.
template <int PARTS>
__device__ __forceinline__ void split(const float (&x)[8], u32x4 (&p)[PARTS])
{
    float r[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = x[e];
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
#pragma unroll
        for (int w = 0; w < 4; ++w) p[i][w] = i + 1 < PARTS ? upper_halves(r[2 * w], r[2 * w + 1]) : bf16_pair(r[2 * w], r[2 * w + 1]);
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] -= cut(r[e]);
    }
}

// g^n, n >= 0: products in 64 bits, as powers of powers are used all along a sequence.
__device__ __forceinline__ float power(float g, int n)
{
    double p = 1.0, b = g;
    for (; n; n >>= 1, b *= b)
        if (n & 1) p *= b;
    return (float)p;
}

template <int DT, int KT, int NW>
struct alignas(16) ChunkLds {
    typedef typename Elem<DT>::type T;
    static constexpr int K = 32 * KT, V = 32 * NW, PAD = 16 / (int)sizeof(T); // rows 16 bytes longer: 16 lanes reach all banks
    T q[kChunk][K + PAD], k[kChunk][K + PAD], v[kChunk][V + PAD];
    T p[DT == kBF16 ? 2 : 1][kChunk][kChunk + PAD]; // scores, by query; bfloat16: in two parts
    float fade[kChunk + 1];      // g^0 ... g^64
    float fade_back[2 * kChunk]; // g^63 ... g^0, then ones
};

// OUT: outputs of the tokens of a part (`per` chunks) of the sequence, from the state in front of it.  Otherwise what those
// tokens leave in a state of zero, where further tokens follow.  `states`: [stream][head][part][key_size][value_size].
template <int DT, int KT, int NW, bool OUT>
__global__ __launch_bounds__(NW * 64) void chunk_kernel(const cbinfer_linear_attention_args a, int slices, int per, int parts, float *states, int whole)
{
    typedef typename Elem<DT>::type T;
    typedef ChunkLds<DT, KT, NW> Lds;
    constexpr int E = 16 / (int)sizeof(T), NT = NW * 64; // E: values in 16 bytes
    constexpr int QP = kChunk * Lds::K / E / NT, VP = kChunk * Lds::V / E / NT; // pieces of 16 bytes a thread
    __shared__ Lds lds;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, side = lane & 31, half = lane >> 5;
    const int slice = blockIdx.x % slices, bh = blockIdx.x / slices, b = bh / a.heads, h = bh - b * a.heads, hk = h / (a.heads / a.kv_heads);
    const int part = blockIdx.y, dk = a.key_size, dv = a.value_size, column = slice * Lds::V + wave * 32 + side;
    const int n = a.lengths ? min(max(a.lengths[b], 0), a.tokens) : a.tokens;
    const int t0 = part * per * kChunk, t1 = min(n, t0 + per * kChunk);
    T *o = static_cast<T *>(a.o) + b * a.o_stride[0] + h * a.o_stride[2];
    if (OUT) {
        const int end = min(a.tokens, t0 + per * kChunk);
        for (int64_t t = max(n, t0) + half; t < end; t += 2)
            if (column < dv) o[t * a.o_stride[1] + column] = Elem<DT>::put(0.0f);
        if (t0 >= n) return;
    } else if (t0 + per * kChunk >= n) {
        return;
    }
    const T *q = static_cast<const T *>(a.q) + b * a.q_stride[0] + h * a.q_stride[2];
    const T *k = static_cast<const T *>(a.k) + b * a.k_stride[0] + hk * a.k_stride[2];
    const T *v = static_cast<const T *>(a.v) + b * a.v_stride[0] + hk * a.v_stride[2] + slice * Lds::V;

    // 16 bytes of a row, zeros beyond the tokens and the row
    auto piece = [&](const T *x, int64_t stride, int t, int at, int size) {
        u32x4 r = {0, 0, 0, 0};
        if (t < t1 && at < size) {
            const T *from = x + t * stride + at;
            if (whole && at + E <= size) {
                r = *reinterpret_cast<const u32x4 *>(from);
            } else {
                union { T e[E]; u32x4 v; } u;
                u.v = r;
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (at + e < size) u.e[e] = from[e];
                r = u.v;
            }
        }
        return r;
    };
    u32x4 qr[OUT ? QP : 1], kr[QP], vr[VP];
    auto load = [&](int t) {
#pragma unroll
        for (int i = 0; i < QP; ++i) {
            const int at = i * NT + threadIdx.x, row = at / (Lds::K / E), col = at % (Lds::K / E) * E;
            if (OUT) qr[OUT ? i : 0] = piece(q, a.q_stride[1], t + row, col, dk);
            kr[i] = piece(k, a.k_stride[1], t + row, col, dk);
        }
#pragma unroll
        for (int i = 0; i < VP; ++i) {
            const int at = i * NT + threadIdx.x, row = at / (Lds::V / E), col = at % (Lds::V / E) * E;
            vr[i] = piece(v, a.v_stride[1], t + row, col, dv - slice * Lds::V);
        }
    };
    load(t0);

    const float g = a.decay[h];
    for (int i = threadIdx.x; i <= kChunk; i += NT) {
        const float f = power(g, i);
        lds.fade[i] = f;
        if (i < kChunk) lds.fade_back[kChunk - 1 - i] = f;
        if (i < kChunk) lds.fade_back[kChunk + i] = 1.0f;
    }

    // rows of S: 32 kt + 8 (r / 4) + 4 half + r % 4 for register r; the lane's column
    f32x16 S[KT];
    float *state = a.state + (int64_t)bh * dk * dv;
    {
        const float *from = parts > 1 ? states + ((int64_t)bh * parts + part) * dk * dv : state;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int row = 32 * kt + 8 * (r / 4) + 4 * half + r % 4;
                S[kt][r] = OUT && row < dk && column < dv ? from[(int64_t)row * dv + column] : 0.0f;
            }
    }

    for (int t = t0; t < t1; t += kChunk) {
        const int m = min(kChunk, t1 - t);
        __syncthreads(); // the chunk before is done with LDS
#pragma unroll
        for (int i = 0; i < QP; ++i) {
            const int at = i * NT + threadIdx.x, row = at / (Lds::K / E), col = at % (Lds::K / E) * E;
            *reinterpret_cast<u32x4 *>(&lds.k[row][col]) = kr[i];
            if (OUT) {
                if (DT == kBF16) { // of 16 values, groups of four in the order 0 2 1 3: as the accumulators have S
                    u32x4 &x = qr[OUT ? i : 0];
                    const int to = (col & ~15) + (col & 8 ? 4 : 0);
                    *reinterpret_cast<uint2 *>(&lds.q[row][to]) = make_uint2(x[0], x[1]);
                    *reinterpret_cast<uint2 *>(&lds.q[row][to + 8]) = make_uint2(x[2], x[3]);
                } else {
                    *reinterpret_cast<u32x4 *>(&lds.q[row][col]) = qr[OUT ? i : 0];
                }
            }
        }
#pragma unroll
        for (int i = 0; i < VP; ++i) {
            const int at = i * NT + threadIdx.x, row = at / (Lds::V / E), col = at % (Lds::V / E) * E;
            *reinterpret_cast<u32x4 *>(&lds.v[row][col]) = vr[i];
        }
        __syncthreads();
        if (t + kChunk < t1) load(t + kChunk);

        f32x16 acc[2];
        if (OUT) {
            // scores of 32 queries and 32 keys each: keys are the rows, so that a lane has four next to one another
            for (int tile = wave; tile < 3; tile += NW) {
                const int j0 = tile == 2 ? 32 : 0, i0 = tile == 0 ? 0 : 32;
                f32x16 p = {};
                if constexpr (DT == kBF16) {
#pragma unroll
                    for (int s = 0; s < 2 * KT; ++s) {
                        const uint2 x = *reinterpret_cast<const uint2 *>(&lds.k[j0 + side][16 * s + 4 * half]), y = *reinterpret_cast<const uint2 *>(&lds.k[j0 + side][16 * s + 8 + 4 * half]);
                        p = multiply(u32x4{x.x, x.y, y.x, y.y}, *reinterpret_cast<const u32x4 *>(&lds.q[i0 + side][16 * s + 8 * half]), p);
                    }
                } else {
#pragma unroll
                    for (int s = 0; s < 4 * KT; ++s) {
                        const float4 x = *reinterpret_cast<const float4 *>(&lds.k[j0 + side][8 * s + 4 * half]), y = *reinterpret_cast<const float4 *>(&lds.q[i0 + side][8 * s + 4 * half]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) p = multiply((&x.x)[e], (&y.x)[e], p);
                    }
                }
                const int i = i0 + side;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int j = j0 + 8 * c + 4 * half;
                    float x[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = i >= j + e ? p[4 * c + e] * lds.fade[max(i - j - e, 0)] : 0.0f;
                    if constexpr (DT == kBF16) {
                        *reinterpret_cast<uint2 *>(&lds.p[0][i][j]) = make_uint2(upper_halves(x[0], x[1]), upper_halves(x[2], x[3]));
                        *reinterpret_cast<uint2 *>(&lds.p[DT == kBF16][i][j]) = make_uint2(bf16_pair(x[0] - cut(x[0]), x[1] - cut(x[1])), bf16_pair(x[2] - cut(x[2]), x[3] - cut(x[3])));
                    } else {
                        *reinterpret_cast<float4 *>(&lds.p[0][i][j]) = make_float4(x[0], x[1], x[2], x[3]);
                    }
                }
            }
            // Q S
            acc[0] = f32x16{};
            acc[1] = f32x16{};
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
                if constexpr (DT == kBF16) {
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        float x[8];
                        u32x4 y[2];
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[e] = S[kt][8 * s + e];
                        split(x, y);
#pragma unroll
                        for (int it = 0; it < 2; ++it) {
                            const u32x4 z = *reinterpret_cast<const u32x4 *>(&lds.q[32 * it + side][32 * kt + 16 * s + 8 * half]);
                            acc[it] = multiply(z, y[0], acc[it]);
                            acc[it] = multiply(z, y[1], acc[it]);
                        }
                    }
                } else {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int it = 0; it < 2; ++it) {
                            const float4 z = *reinterpret_cast<const float4 *>(&lds.q[32 * it + side][32 * kt + 8 * c + 4 * half]);
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[it] = multiply((&z.x)[e], S[kt][4 * c + e], acc[it]);
                        }
                }
            }
        }

        // the wave's columns of V as the second operand: of 32 tokens by the lane half, 16 values in all
        u32x4 vb[DT == kBF16 ? 4 : 1];
        float vf[DT == kBF16 ? 1 : 32], poison = 0.0f;
        if constexpr (DT == kBF16) {
            const int in = lane & 15;
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const T *from = &lds.v[16 * s + 8 * half + in / 4][wave * 32 + (lane & 16) + 4 * (in & 3)];
                const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)from);
                const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(from + 4 * (Lds::V + Lds::PAD)));
                const uint2 xu = __builtin_bit_cast(uint2, x), yu = __builtin_bit_cast(uint2, y);
                vb[s] = u32x4{xu.x, xu.y, yu.x, yu.y};
            }
        } else {
#pragma unroll
            for (int c = 0; c < 8; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) vf[4 * c + e] = lds.v[8 * c + 4 * half + e][wave * 32 + side];
        }
        auto value = [&](int s, int e) { return __uint_as_float(e & 1 ? vb[s][e / 2] & 0xffff0000u : vb[s][e / 2] << 16); };

        if (OUT) {
            if constexpr (DT == kBF16) {
#pragma unroll
                for (int s = 0; s < 4; ++s)
#pragma unroll
                    for (int e = 0; e < 8; ++e) poison = __builtin_fmaf(value(s, e), 0.0f, poison);
            } else {
#pragma unroll
                for (int e = 0; e < 32; ++e) poison = __builtin_fmaf(vf[e], 0.0f, poison);
            }
            __syncthreads(); // scores are there
#pragma unroll
            for (int it = 0; it < 2; ++it)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[it][r] *= lds.fade[32 * it + 8 * (r / 4) + 4 * half + r % 4 + 1];
            if (!__any(poison != 0.0f)) {
                if constexpr (DT == kBF16) {
#pragma unroll
                    for (int it = 0; it < 2; ++it)
#pragma unroll
                        for (int s = 0; s < 2 + 2 * it; ++s)
#pragma unroll
                            for (int i = 0; i < 2; ++i) acc[it] = multiply(*reinterpret_cast<const u32x4 *>(&lds.p[DT == kBF16 ? i : 0][32 * it + side][16 * s + 8 * half]), vb[s], acc[it]);
                } else {
#pragma unroll
                    for (int it = 0; it < 2; ++it)
#pragma unroll
                        for (int c = 0; c < 4 + 4 * it; ++c) {
                            const float4 z = *reinterpret_cast<const float4 *>(&lds.p[0][32 * it + side][8 * c + 4 * half]);
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[it] = multiply((&z.x)[e], vf[4 * c + e], acc[it]);
                        }
                }
            } else { // a value that is not finite: its product with the score 0 of an earlier token must not be added
                for (int j = 0; j < m; ++j) {
                    const float x = Elem<DT>::get(lds.v[j][wave * 32 + side]);
#pragma unroll
                    for (int it = 0; it < 2; ++it)
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const int i = 32 * it + 8 * (r / 4) + 4 * half + r % 4;
                            if (i >= j) {
                                float p = Elem<DT>::get(lds.p[0][i][j]);
                                if (DT == kBF16) p += Elem<DT>::get(lds.p[DT == kBF16][i][j]);
                                acc[it][r] = __builtin_fmaf(p, x, acc[it][r]);
                            }
                        }
                }
            }
#pragma unroll
            for (int it = 0; it < 2; ++it)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int i = 32 * it + 8 * (r / 4) + 4 * half + r % 4;
                    if (i < m && column < dv) o[(int64_t)(t + i) * a.o_stride[1] + column] = Elem<DT>::put(a.scale * acc[it][r]);
                }
        }

        // the state behind the chunk
        const float all = lds.fade[m], *fade = lds.fade_back + kChunk - m; // of token j: g^(m-1-j), and 1 beyond, where values are 0
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) S[kt][r] *= all;
        if constexpr (DT == kBF16) {
            const int in = lane & 15;
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                float x[8];
                u32x4 y[3];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = value(s, e) * fade[16 * s + 8 * half + e];
                split(x, y);
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) {
                    const T *from = &lds.k[16 * s + 8 * half + in / 4][32 * kt + (lane & 16) + 4 * (in & 3)];
                    const uint2 p = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)from));
                    const uint2 u = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(from + 4 * (Lds::K + Lds::PAD))));
#pragma unroll
                    for (int i = 0; i < 3; ++i) S[kt] = multiply(u32x4{p.x, p.y, u.x, u.y}, y[i], S[kt]);
                }
            }
        } else {
#pragma unroll
            for (int c = 0; c < 8; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int j = 8 * c + 4 * half + e;
                    const float x = vf[4 * c + e] * fade[j];
#pragma unroll
                    for (int kt = 0; kt < KT; ++kt) S[kt] = multiply(lds.k[j][32 * kt + side], x, S[kt]);
                }
        }
    }

    float *to = OUT ? state : states + ((int64_t)bh * parts + part + 1) * dk * dv;
    if (!OUT || t1 == n) // the part with the last token
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int row = 32 * kt + 8 * (r / 4) + 4 * half + r % 4;
                if (row < dk && column < dv) to[(int64_t)row * dv + column] = S[kt][r];
            }
}

// What the parts of a sequence leave by themselves (places 1, 2, ...) becomes the states in front of the parts.
__global__ __launch_bounds__(256) void join_parts_kernel(const cbinfer_linear_attention_args a, int per, int parts, float *states)
{
    const int bh = blockIdx.y, size = a.key_size * a.value_size, at = blockIdx.x * 256 + threadIdx.x, b = bh / a.heads;
    if (at >= size) return;
    const int n = a.lengths ? min(max(a.lengths[b], 0), a.tokens) : a.tokens;
    const float g = power(a.decay[bh - b * a.heads], per * kChunk);
    float *s = states + (int64_t)bh * parts * size + at, x = a.state[(int64_t)bh * size + at];
    s[0] = x;
    for (int p = 1; p < parts && (int64_t)p * per * kChunk < n; ++p) {
        x = __builtin_fmaf(g, x, s[(int64_t)p * size]);
        s[(int64_t)p * size] = x;
    }
}

struct Plan {
    bool chunks;
    int slices, per, parts, tiles; // tiles: of 32 columns a workgroup
};

Plan plan(const cbinfer_linear_attention_args &a)
{
    Plan p = {false, 1, 1, 1, 4};
    if (a.tokens < 16 || (a.dtype == kF32 && a.key_size > 128)) return p; // float32 rows of 256 keys do not fit LDS
    p.chunks = true;
    const int tiles = (a.value_size + 31) / 32;
    p.tiles = tiles <= 2 && a.key_size <= 128 ? 2 : 4;
    p.slices = (tiles + p.tiles - 1) / p.tiles;
    const int64_t groups = (int64_t)a.streams * a.heads * p.slices, chunks = (a.tokens + kChunk - 1) / kChunk;
    static const int TG = getenv("CBG") ? atoi(getenv("CBG")) : 512;
    p.parts = (int)std::max<int64_t>(1, std::min<int64_t>(chunks / 2, TG / std::max<int64_t>(groups, 1)));
    p.per = (int)((chunks + p.parts - 1) / p.parts);
    p.parts = (int)((chunks + p.per - 1) / p.per);
    return p;
}

template <int DT, int KT, int NW>
hipError_t chunked(hipStream_t st, const cbinfer_linear_attention_args &a, const Plan &p)
{
    const size_t e = DT == kF32 ? 4 : 2;
    auto fits = [&](const void *x, const int64_t *stride) {
        for (int i = 0; i < 3; ++i)
            if (stride[i] * e % 16) return 0;
        return reinterpret_cast<uintptr_t>(x) % 16 == 0 ? 1 : 0;
    };
    const int whole = fits(a.q, a.q_stride) & fits(a.k, a.k_stride) & fits(a.v, a.v_stride);
    float *states = static_cast<float *>(a.workspace);
    const unsigned groups = (unsigned)(a.streams * a.heads * p.slices);
    if (p.parts > 1) {
        chunk_kernel<DT, KT, NW, false><<<dim3(groups, p.parts - 1), NW * 64, 0, st>>>(a, p.slices, p.per, p.parts, states, whole);
        if (hipError_t err = hipGetLastError()) return err;
        join_parts_kernel<<<dim3((a.key_size * a.value_size + 255) / 256, a.streams * a.heads), 256, 0, st>>>(a, p.per, p.parts, states);
        if (hipError_t err = hipGetLastError()) return err;
    }
    chunk_kernel<DT, KT, NW, true><<<dim3(groups, p.parts), NW * 64, 0, st>>>(a, p.slices, p.per, p.parts, states, whole);
    return hipGetLastError();
}

template <int DT>
hipError_t chunked_any(hipStream_t st, const cbinfer_linear_attention_args &a, const Plan &p)
{
    if (a.key_size <= 64) return p.tiles == 2 ? chunked<DT, 2, 2>(st, a, p) : chunked<DT, 2, 4>(st, a, p);
    if (a.key_size <= 128) return p.tiles == 2 ? chunked<DT, 4, 2>(st, a, p) : chunked<DT, 4, 4>(st, a, p);
    if constexpr (DT == kBF16) return chunked<DT, 8, 4>(st, a, p);
    return hipErrorInvalidValue;
}

} // namespace

size_t linear_attention_workspace(const cbinfer_linear_attention_args &a)
{
    const Plan p = plan(a);
    return p.parts > 1 ? (size_t)a.streams * a.heads * p.parts * a.key_size * a.value_size * sizeof(float) : 0;
}

hipError_t linear_attention(hipStream_t st, const cbinfer_linear_attention_args &a)
{
    const Plan p = plan(a);
    if (p.chunks) return a.dtype == kF32 ? chunked_any<kF32>(st, a, p) : chunked_any<kBF16>(st, a, p);
    return a.dtype == kF32 ? recurrent_any<kF32>(st, a) : recurrent_any<kBF16>(st, a);
}

} // namespace cbk
