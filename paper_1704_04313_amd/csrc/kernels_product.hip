// Few tokens times a matrix of 4-bit weights: y[m][n] = bias[n] + sum over groups of scale[n][group] * (sum of x[m][k] value(code[n][k])).
//
// Packed weights.  A block is 16 rows x 128 columns: 1 KiB of codes, 16 bytes a lane, as the matrix instruction 16x16x32 takes
// them -- lane l holds row l % 16, and its word j the columns 32 j + 8 (l / 16) + 0 .. 7 of the block, the first in the lowest
// four bits.  Blocks of a row tile follow one another, row tiles too.  Behind the codes the scales, [row tile][block][16
// rows][128 / group] bfloat16.  What lies beyond the matrix has code 0 and scale 0.
#include "tokens.h"

#include <algorithm>
#include <cstdlib>

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
// Eight values of a token from column k on as they lie in memory, zeros beyond the row.
template <int DT>
struct Eight {
    uint4 u[DT == kF32 ? 2 : 1];
    template <bool WHOLE> // rows at 16-byte addresses
    __device__ __forceinline__ void load(const typename Elem<DT>::type *x, int64_t k, int64_t cols, bool there)
    {
        typedef typename Elem<DT>::type T;
        constexpr int N = DT == kF32 ? 2 : 1;
#pragma unroll
        for (int i = 0; i < N; ++i) u[i] = make_uint4(0, 0, 0, 0);
        if (!there || k >= cols) return;
        if (WHOLE && k + 8 <= cols) {
#pragma unroll
            for (int i = 0; i < N; ++i) u[i] = reinterpret_cast<const uint4 *>(x + k)[i];
            return;
        }
        union { T e[8]; uint4 u[N]; } v;
#pragma unroll
        for (int e = 0; e < 8; ++e) v.e[e] = k + e < cols ? x[k + e] : T(0);
#pragma unroll
        for (int i = 0; i < N; ++i) u[i] = v.u[i];
    }
    __device__ __forceinline__ float get(int e) const { return Unit<DT>::get(u[DT == kF32 ? e / 4 : 0], DT == kF32 ? e % 4 : e); }
};

// A float as the sum of three bfloat16, exactly: eight bits are cut off each time.  Infinities stay in the first.
__device__ __forceinline__ void parts_of(const Eight<kBF16> &v, bf16x8 (&p)[1]) { p[0] = __builtin_bit_cast(bf16x8, v.u[0]); }
__device__ __forceinline__ void parts_of(const Eight<kF32> &v, bf16x8 (&p)[3])
{
    constexpr int PARTS = 3;
    float r[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = v.get(e);
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
        uint4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) (&w.x)[j] = __builtin_amdgcn_perm(__float_as_uint(r[2 * j + 1]), __float_as_uint(r[2 * j]), 0x07060302u);
        p[i] = __builtin_bit_cast(bf16x8, w);
        if (i + 1 < PARTS)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float top = __uint_as_float(__float_as_uint(r[e]) & 0xffff0000u);
                r[e] = __builtin_isinf(top) ? 0.0f : r[e] - top;
            }
    }
}

// A wave multiplies R tiles of 16 rows with MT tiles of 16 tokens over its share of the blocks of columns: the waves of a
// workgroup take them in turn and add up through LDS.  blockIdx.y: a part of the blocks (their sums then go to `partial`, part by part),
// blockIdx.z: the tokens.  Tokens are the matrix instruction's rows, weights its columns: a lane has one row's scale at a time.
template <int DT, int MT, int R, bool WHOLE>
__global__ __launch_bounds__(512) void product_kernel(const cbinfer_quantised_product_args a, const uint16_t *scales, int blocks, int tiles, int per, float *partial)
{
    typedef typename Elem<DT>::type T;
    constexpr int PARTS = DT == kF32 ? 3 : 1;
    extern __shared__ f32x4 sums[]; // [wave][R][MT][lane]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, per_block = 128 / a.group, step = a.group / 32;
    const int64_t token0 = (int64_t)blockIdx.z * (16 * MT), tile0 = (int64_t)blockIdx.x * R;
    const T *x[MT];
    bool there[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int64_t t = token0 + 16 * i + (lane & 15);
        there[i] = t < a.tokens;
        x[i] = static_cast<const T *>(a.x) + (there[i] ? t : 0) * a.x_stride;
    }
    const uint4 *codes[R];
    const uint16_t *sc[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int64_t tile = tile0 + r < tiles ? tile0 + r : tiles - 1; // beyond the last: computed again, not written
        codes[r] = static_cast<const uint4 *>(a.packed) + tile * blocks * 64 + lane;
        sc[r] = scales + (tile * blocks * 16 + (lane & 15)) * per_block;
    }
    f32x4 acc[R][MT];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[r][i] = f32x4{0, 0, 0, 0};
    const int end = min(blocks, ((int)blockIdx.y + 1) * per);
    // of a block: the codes, the scales of a row, and with one tile of tokens their values;
    // the next block's are on their way while one is worked on
    struct Block {
        uint4 w[R];
        uint2 s[R];
        Eight<DT> x[4];
    };
    auto values = [&](int b, int j, int i) {
        Eight<DT> v;
        v.template load<WHOLE>(x[i], (int64_t)b * 128 + j * 32 + (lane >> 4) * 8, a.cols, there[i]);
        return v;
    };
    auto load = [&](Block &k, int b) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            k.w[r] = codes[r][(int64_t)b * 64];
            const uint16_t *p = sc[r] + (int64_t)b * 16 * per_block;
            if (step == 1)
                k.s[r] = *reinterpret_cast<const uint2 *>(p);
            else if (step == 2)
                k.s[r].x = *reinterpret_cast<const unsigned *>(p);
            else
                k.s[r].x = *p;
        }
        if (MT == 1)
#pragma unroll
            for (int j = 0; j < 4; ++j) k.x[j] = values(b, j, 0);
    };
    Block next;
    int b = blockIdx.y * per + wave;
    if (b < end) load(next, b);
    for (; b < end; b += waves) {
        const Block now = next;
        if (b + waves < end) load(next, b + waves);
        f32x4 part[R][MT];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (j % step == 0)
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int i = 0; i < MT; ++i) part[r][i] = f32x4{0, 0, 0, 0};
            bf16x8 p[MT][PARTS];
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                parts_of(MT == 1 ? now.x[j] : values(b, j, i), p[i]);
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const bf16x8 q = values_of((&now.w[r].x)[j]);
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int k = 0; k < PARTS; ++k) part[r][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(p[i][k], q, part[r][i], 0, 0, 0);
            }
            if ((j + 1) % step == 0) // the group ends here
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const int g = step == 1 ? j : step == 2 ? j / 2 : 0; // of the block's groups
                    const unsigned u = g < 2 ? now.s[r].x : now.s[r].y;
                    const float s = __uint_as_float(g & 1 ? u & 0xffff0000u : u << 16);
#pragma unroll
                    for (int i = 0; i < MT; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[r][i][e] = __builtin_fmaf(s, part[r][i][e], acc[r][i][e]);
                }
        }
    }
    if (waves > 1) {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < MT; ++i) sums[(wave * R * MT + r * MT + i) * 64 + lane] = acc[r][i];
        __syncthreads();
    }
    // a wave writes tiles of its own
    for (int at = wave; at < R * MT; at += waves) {
        const int r = at / MT, i = at - r * MT;
        f32x4 y = {0, 0, 0, 0};
        if (waves > 1) {
            for (int k = 0; k < waves; ++k) y += sums[(k * R * MT + at) * 64 + lane];
        } else {
#pragma unroll
            for (int k = 0; k < R * MT; ++k)
                if (k == at) y = acc[k / MT][k % MT];
        }
        const int64_t n = (tile0 + r) * 16 + (lane & 15), t = token0 + 16 * i + (lane >> 4) * 4;
        if (tile0 + r >= tiles || n >= a.rows) continue;
        const float bias = a.bias && !partial ? a.bias[n] : 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (t + e < a.tokens) {
                if (partial)
                    partial[((int64_t)blockIdx.y * a.tokens + t + e) * a.rows + n] = y[e];
                else
                    static_cast<T *>(a.y)[(t + e) * a.y_stride + n] = Elem<DT>::put(y[e] + bias);
            }
    }
}

// The parts' sums, in order.
template <int DT>
__global__ __launch_bounds__(256) void join_parts_kernel(const cbinfer_quantised_product_args a, int parts, const float *partial)
{
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, all = a.tokens * a.rows;
    if (at >= all) return;
    const int64_t t = at / a.rows, n = at - t * a.rows;
    float y = a.bias ? a.bias[n] : 0.0f;
    for (int p = 0; p < parts; ++p) y += partial[p * all + at];
    static_cast<typename Elem<DT>::type *>(a.y)[t * a.y_stride + n] = Elem<DT>::put(y);
}

struct Plan {
    int mt, r, waves, parts, per;
};

Plan plan(const cbinfer_quantised_product_args &a)
{
    Plan p;
    const int64_t tiles = tiles_of(a.rows), blocks = blocks_of(a.cols);
    p.mt = a.tokens <= 16 ? 1 : a.tokens <= 32 ? 2 : 4;
    static const int R_ = getenv("CBR") ? atoi(getenv("CBR")) : 0, W_ = getenv("CBW") ? atoi(getenv("CBW")) : 0, P_ = getenv("CBP") ? atoi(getenv("CBP")) : 0;
    p.r = R_ ? R_ : tiles >= 2048 ? 4 : tiles >= 512 ? 2 : 1;
    p.waves = W_ ? W_ : 8;
    while (p.waves * p.r * p.mt > 64) p.waves /= 2; // their sums in 64 KiB of LDS
    p.parts = P_ ? P_ : 1;
    p.per = (int)((blocks + p.parts - 1) / p.parts);
    p.parts = (int)((blocks + p.per - 1) / p.per);
    return p;
}

template <int DT, int MT, int R>
hipError_t launch(hipStream_t st, const cbinfer_quantised_product_args &a, const Plan &p)
{
    const int64_t tiles = tiles_of(a.rows), blocks = blocks_of(a.cols);
    const uint16_t *scales = reinterpret_cast<const uint16_t *>(static_cast<const char *>(a.packed) + code_bytes(a.rows, a.cols));
    const bool whole = reinterpret_cast<uintptr_t>(a.x) % 16 == 0 && a.x_stride * (DT == kF32 ? 4 : 2) % 16 == 0;
    float *partial = p.parts > 1 ? static_cast<float *>(a.workspace) : nullptr;
    const dim3 grid((unsigned)((tiles + R - 1) / R), p.parts, (unsigned)((a.tokens + 16 * MT - 1) / (16 * MT)));
    const size_t lds = p.waves > 1 ? (size_t)p.waves * R * MT * 64 * sizeof(f32x4) : 0;
    if (whole)
        product_kernel<DT, MT, R, true><<<grid, p.waves * 64, lds, st>>>(a, scales, (int)blocks, (int)tiles, p.per, partial);
    else
        product_kernel<DT, MT, R, false><<<grid, p.waves * 64, lds, st>>>(a, scales, (int)blocks, (int)tiles, p.per, partial);
    if (hipError_t e = hipGetLastError()) return e;
    if (partial) {
        join_parts_kernel<DT><<<(unsigned)((a.tokens * a.rows + 255) / 256), 256, 0, st>>>(a, p.parts, partial);
        return hipGetLastError();
    }
    return hipSuccess;
}

template <int DT, int MT>
hipError_t launch_rows(hipStream_t st, const cbinfer_quantised_product_args &a, const Plan &p)
{
    return p.r == 4 ? launch<DT, MT, 4>(st, a, p) : p.r == 2 ? launch<DT, MT, 2>(st, a, p) : launch<DT, MT, 1>(st, a, p);
}

template <int DT>
hipError_t launch_any(hipStream_t st, const cbinfer_quantised_product_args &a, const Plan &p)
{
    return p.mt == 1 ? launch_rows<DT, 1>(st, a, p) : p.mt == 2 ? launch_rows<DT, 2>(st, a, p) : launch_rows<DT, 4>(st, a, p);
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

size_t quantised_product_workspace(const cbinfer_quantised_product_args &a)
{
    const Plan p = plan(a);
    return p.parts > 1 ? (size_t)p.parts * a.tokens * a.rows * sizeof(float) : 0;
}

hipError_t quantised_product(hipStream_t st, const cbinfer_quantised_product_args &a)
{
    const Plan p = plan(a);
    return a.dtype == kF32 ? launch_any<kF32>(st, a, p) : launch_any<kBF16>(st, a, p);
}

} // namespace cbk
