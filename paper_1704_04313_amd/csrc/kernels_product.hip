// Few tokens times a matrix of 4-bit weights: y[m][n] = bias[n] + sum over groups of scale[n][group] * (sum of x[m][k] value(code[n][k])).
//
// Packed weights.  A block is 16 rows x 128 columns: 1 KiB of codes, 16 bytes a lane, as the matrix instruction 16x16x32 takes
// them -- lane l holds row l % 16, and its word j the columns 32 j + 8 (l / 16) + 0 .. 7 of the block, the first in the lowest
// four bits.  Blocks of a row tile follow one another, row tiles too.  Behind the codes the scales, [row tile][block][16
// rows][128 / group] bfloat16.  What lies beyond the matrix has code 0 and scale 0.
#include "tokens.h"

namespace cbk {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

inline int64_t blocks_of(int64_t cols) { return (cols + 127) / 128; }
inline int64_t tiles_of(int64_t rows) { return (rows + 15) / 16; }
inline size_t code_bytes(int64_t rows, int64_t cols) { return (size_t)(tiles_of(rows) * blocks_of(cols)) * 1024; }

// The eight values of a word of codes: the conversion is exact, the scale argument is 1.
__device__ __forceinline__ bf16x8 values_of(unsigned w)
{
    union { bf16x2 h[4]; bf16x8 v; } u;
    u.h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 0);
    u.h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 1);
    u.h[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 2);
    u.h[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 3);
    return u.v;
}

// ---- laying out ----------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void pack_codes_kernel(const uint8_t *codes, int64_t rows, int64_t cols, int64_t blocks, int64_t units, uint4 *to)
{
    const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; // 16 bytes: a lane's part of a block
    if (u >= units) return;
    const int lane = u & 63;
    const int64_t tile = (u >> 6) / blocks, block = (u >> 6) - tile * blocks;
    const int64_t n = tile * 16 + (lane & 15), k0 = block * 128 + (lane >> 4) * 8;
    unsigned w[4];
    for (int j = 0; j < 4; ++j) {
        w[j] = 0;
        for (int e = 0; e < 8; ++e) {
            const int64_t k = k0 + j * 32 + e;
            if (n < rows && k < cols) w[j] |= (unsigned)(codes[n * cols + k] & 15) << (4 * e);
        }
    }
    to[u] = make_uint4(w[0], w[1], w[2], w[3]);
}

__global__ __launch_bounds__(256) void pack_scales_kernel(const uint16_t *scales, int64_t rows, int64_t groups, int64_t blocks, int per_block, int64_t total, uint16_t *to)
{
    const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (u >= total) return;
    const int g = (int)(u % per_block);
    const int64_t r = u / per_block, tile = (r >> 4) / blocks, block = (r >> 4) - tile * blocks;
    const int64_t n = tile * 16 + (r & 15), k = block * per_block + g;
    to[u] = n < rows && k < groups ? scales[n * groups + k] : (uint16_t)0;
}

// 32 lanes a group.
template <int DT>
__global__ __launch_bounds__(256) void quantise_kernel(const typename Elem<DT>::type *w, int64_t rows, int64_t cols, int64_t stride, int group, int64_t groups, uint8_t *codes, uint16_t *scales)
{
    const int64_t at = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (at >= rows * groups) return;
    const int64_t n = at / groups, k0 = (at - n * groups) * group;
    const int lane = threadIdx.x & 31;
    float x[4], most = 0.0f;
    for (int i = 0; i < 4; ++i) {
        const int64_t k = k0 + i * 32 + lane;
        x[i] = i * 32 < group && k < cols ? Elem<DT>::get(w[n * stride + k]) : 0.0f;
        most = fmaxf(most, fabsf(x[i]));
    }
    for (int off = 16; off; off >>= 1) most = fmaxf(most, __shfl_xor(most, off));
    const uint16_t bits = Elem<kBF16>::put(most / 6.0f);
    const float scale = Elem<kBF16>::get(bits);
    if (lane == 0) scales[at] = bits;
    for (int i = 0; i < 4; ++i) {
        const int64_t k = k0 + i * 32 + lane;
        if (i * 32 >= group || k >= cols) continue;
        const float v = scale > 0.0f ? fabsf(x[i]) / scale : 0.0f;
        const int c = (v > 0.25f) + (v >= 0.75f) + (v > 1.25f) + (v >= 1.75f) + (v > 2.5f) + (v >= 3.5f) + (v > 5.0f);
        codes[n * cols + k] = (uint8_t)(c && x[i] < 0.0f ? c | 8 : c);
    }
}

// ---- the product ---------------------------------------------------------------------------------
// Eight values of a token from column k on, zeros beyond the row.
template <int DT>
__device__ __forceinline__ void load_eight(const typename Elem<DT>::type *x, int64_t k, int64_t cols, bool there, float (&v)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = there && k + e < cols ? Elem<DT>::get(x[k + e]) : 0.0f;
}

// A float as the sum of three bfloat16, exactly: eight bits are cut off each time.  Infinities stay in the first.
template <int PARTS>
__device__ __forceinline__ void split(const float (&v)[8], bf16x8 (&p)[PARTS])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float r = v[e];
#pragma unroll
        for (int i = 0; i < PARTS; ++i) {
            const float top = __uint_as_float(__float_as_uint(r) & 0xffff0000u);
            p[i][e] = (__bf16)top;
            r = __builtin_isinf(top) ? 0.0f : r - top;
        }
    }
}

// A workgroup multiplies one tile of 16 rows with 16 tokens; its four waves take the blocks of columns in turn.
template <int DT>
__global__ __launch_bounds__(256) void product_kernel(const cbinfer_quantised_product_args a, const uint16_t *scales, int blocks)
{
    typedef typename Elem<DT>::type T;
    constexpr int PARTS = DT == kF32 ? 3 : 1;
    __shared__ float sums[4][256];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, per_block = 128 / a.group;
    const int64_t tile = blockIdx.x, token = (int64_t)blockIdx.y * 16 + (lane & 15);
    const uint4 *codes = static_cast<const uint4 *>(a.packed) + tile * blocks * 64 + lane;
    const uint16_t *sc = scales + (tile * blocks * 16 + (lane & 15)) * per_block;
    const T *x = static_cast<const T *>(a.x) + token * a.x_stride;
    const bool there = token < a.tokens;
    f32x4 acc = {0, 0, 0, 0};
    for (int b = wave; b < blocks; b += 4) {
        const uint4 w = codes[(int64_t)b * 64];
        f32x4 part = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float v[8];
            bf16x8 p[PARTS];
            load_eight<DT>(x, (int64_t)b * 128 + j * 32 + (lane >> 4) * 8, a.cols, there, v);
            split<PARTS>(v, p);
            const bf16x8 q = values_of((&w.x)[j]);
#pragma unroll
            for (int i = 0; i < PARTS; ++i) part = __builtin_amdgcn_mfma_f32_16x16x32_bf16(p[i], q, part, 0, 0, 0);
            if ((j + 1) * 32 % a.group == 0) { // the group ends here
                const float s = Elem<kBF16>::get(sc[(int64_t)b * 16 * per_block + j * 32 / a.group]);
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[r] = __builtin_fmaf(s, part[r], acc[r]);
                part = {0, 0, 0, 0};
            }
        }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) sums[wave][r * 64 + lane] = acc[r];
    __syncthreads();
    const int i = threadIdx.x, n16 = i & 15, t16 = ((i & 63) >> 4) * 4 + (i >> 6);
    const int64_t n = tile * 16 + n16, t = (int64_t)blockIdx.y * 16 + t16;
    if (n < a.rows && t < a.tokens)
        static_cast<T *>(a.y)[t * a.y_stride + n] = Elem<DT>::put((sums[0][i] + sums[1][i]) + (sums[2][i] + sums[3][i]) + (a.bias ? a.bias[n] : 0.0f));
}

} // namespace

hipError_t quantise_weights(hipStream_t st, const void *weights, int dtype, int64_t rows, int64_t cols, int64_t row_stride,
                            int group, uint8_t *codes, uint16_t *scales)
{
    const int64_t groups = (cols + group - 1) / group;
    const unsigned grid = (unsigned)((rows * groups + 7) / 8);
    if (dtype == kF32)
        quantise_kernel<kF32><<<grid, 256, 0, st>>>(static_cast<const float *>(weights), rows, cols, row_stride, group, groups, codes, scales);
    else
        quantise_kernel<kBF16><<<grid, 256, 0, st>>>(static_cast<const uint16_t *>(weights), rows, cols, row_stride, group, groups, codes, scales);
    return hipGetLastError();
}

size_t packed_weights_bytes(int64_t rows, int64_t cols, int group)
{
    return code_bytes(rows, cols) + (size_t)(tiles_of(rows) * blocks_of(cols)) * 16 * (128 / group) * 2;
}

hipError_t pack_weights(hipStream_t st, const uint8_t *codes, const uint16_t *scales, int64_t rows, int64_t cols, int group,
                        void *packed)
{
    const int64_t blocks = blocks_of(cols), units = tiles_of(rows) * blocks * 64, per_block = 128 / group, total = units / 4 * per_block;
    pack_codes_kernel<<<(unsigned)((units + 255) / 256), 256, 0, st>>>(codes, rows, cols, blocks, units, static_cast<uint4 *>(packed));
    if (hipError_t e = hipGetLastError()) return e;
    pack_scales_kernel<<<(unsigned)((total + 255) / 256), 256, 0, st>>>(scales, rows, (cols + group - 1) / group, blocks, (int)per_block, total,
        reinterpret_cast<uint16_t *>(static_cast<char *>(packed) + code_bytes(rows, cols)));
    return hipGetLastError();
}

size_t quantised_product_workspace(const cbinfer_quantised_product_args &) { return 0; }

hipError_t quantised_product(hipStream_t st, const cbinfer_quantised_product_args &a)
{
    const dim3 grid((unsigned)tiles_of(a.rows), (unsigned)((a.tokens + 15) / 16));
    const uint16_t *scales = reinterpret_cast<const uint16_t *>(static_cast<const char *>(a.packed) + code_bytes(a.rows, a.cols));
    if (a.dtype == kF32)
        product_kernel<kF32><<<grid, 256, 0, st>>>(a, scales, (int)blocks_of(a.cols));
    else
        product_kernel<kBF16><<<grid, 256, 0, st>>>(a, scales, (int)blocks_of(a.cols));
    return hipGetLastError();
}

} // namespace cbk
