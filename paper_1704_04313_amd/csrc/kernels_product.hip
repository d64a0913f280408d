// Few tokens times a matrix of 4-bit weights: y[m][n] = bias[n] + sum over groups of scale[n][group] * (sum of x[m][k] value(code[n][k])).
//
// Packed weights.  A block is 16 rows x 128 columns: 1 KiB of codes, 16 bytes a lane, as the matrix instruction 16x16x32 takes
// them -- lane l holds row l % 16, and its word j the columns 32 j + 8 (l / 16) + 0 .. 7 of the block, the first in the lowest
// four bits.  Blocks of a row tile follow one another, row tiles too.  Behind the codes the scales, [row tile][block][16
// rows][128 / group] bfloat16.  What lies beyond the matrix has code 0 and scale 0.
#include "tokens.h"

#include <algorithm>

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
__device__ __forceinline__ unsigned four_codes(unsigned x) // of four bytes, in the lower half
{
    x &= 0x0f0f0f0fu;
    x = (x | x >> 4) & 0x00ff00ffu;
    return (x | x >> 8) & 0xffffu;
}

// Once a layer.  WHOLE: eight codes at 8-byte addresses at a time, 100003 x 2048 76 us (308 MB); one by one 100003 x 2047 314.
template <bool WHOLE>
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
        const int64_t k = k0 + j * 32;
        if (n >= rows) continue;
        if (WHOLE) {
            if (k >= cols) continue;
            const uint2 x = *reinterpret_cast<const uint2 *>(codes + n * cols + k);
            w[j] = four_codes(x.x) | four_codes(x.y) << 16;
        } else {
            for (int e = 0; e < 8; ++e)
                if (k + e < cols) w[j] |= (unsigned)(codes[n * cols + k + e] & 15) << (4 * e);
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

// 32 lanes a group; 100003 x 2048 float32 447 us, not bound by memory (bfloat16, half the bytes: 484).
template <int DT>
__global__ __launch_bounds__(256) void quantise_kernel(const typename Elem<DT>::type *w, int64_t rows, int64_t cols, int64_t stride, int group, int64_t groups, int64_t first, uint8_t *codes, uint16_t *scales)
{
    const int64_t at = first + (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
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
    typedef unsigned u32x4 __attribute__((ext_vector_type(4), aligned(2))); // one load at any alignment
    static constexpr int N = DT == kF32 ? 2 : 1;
    uint4 u[N];
    // at any address; it is valid also where the token is not there
    __device__ __forceinline__ void load(const typename Elem<DT>::type *x, bool there)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const u32x4 y = *reinterpret_cast<const u32x4 *>(x + i * 4);
            u[i] = there ? make_uint4(y[0], y[1], y[2], y[3]) : make_uint4(0, 0, 0, 0);
        }
    }
    __device__ __forceinline__ void load_singly(const typename Elem<DT>::type *x, int64_t k, int64_t cols, bool there)
    {
        typedef typename Elem<DT>::type T;
        union { T e[8]; uint4 u[N]; } v;
#pragma unroll
        for (int e = 0; e < 8; ++e) v.e[e] = there && k + e < cols ? x[k + e] : T(0);
#pragma unroll
        for (int i = 0; i < N; ++i) u[i] = v.u[i];
    }
    __device__ __forceinline__ float get(int e) const { return Unit<DT>::get(u[DT == kF32 ? e / 4 : 0], DT == kF32 ? e % 4 : e); }
};

// A float as the sum of three bfloat16, exactly: eight bits are cut off each time.  Infinities stay in the first; a NaN, of
// which that may leave an infinity, is in the others.
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
                r[e] = __builtin_isinf(r[e]) ? 0.0f : r[e] - top;
            }
    }
}

// A workgroup keeps its part of the columns of MT tiles of 16 tokens in registers, each of its waves BP blocks of them, and
// streams weights past them: R tiles of 16 rows at a time, the next on their way while these are multiplied.  The waves add up
// through LDS.  blockIdx.y: the part of the columns (of several, each leaves its sums in `partial`), blockIdx.z: the tokens.
// Tokens are the matrix instruction's rows, weights its columns, so that a lane needs one row's scales.
template <int DT, int MT, int BP, int R, int WAVES, int PER_CU>
__global__ __launch_bounds__(WAVES * 64, WAVES * PER_CU / 4) void product_kernel(const cbinfer_quantised_product_args a, const uint16_t *scales, int blocks, int tiles, float *partial)
{
    typedef typename Elem<DT>::type T;
    constexpr int PARTS = DT == kF32 ? 3 : 1;
    __shared__ f32x4 sums[2][WAVES][R * MT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, per_block = 128 / a.group, step = a.group / 32;
    const int64_t token0 = (int64_t)blockIdx.z * (16 * MT);
    const int block0 = blockIdx.y * (WAVES * BP) + wave; // then every WAVES-th

    struct Weights {
        uint4 w[R][BP];
        uint2 s[R][BP];
    };
    const uint4 *codes = static_cast<const uint4 *>(a.packed) + lane;
    const uint16_t *sc = scales + (lane & 15) * per_block;
    Weights k; // each of its blocks is read again, for the next turn, as soon as it has been multiplied
    auto load = [&](int group, int r, int i) {
        const int64_t tile = min(group * R + r, tiles - 1); // beyond the last: multiplied again, not written
        const int64_t at = tile * blocks + min(block0 + i * WAVES, blocks - 1); // beyond the last: times zeros
        k.w[r][i] = codes[at * 64];
        const uint16_t *p = sc + at * 16 * per_block;
        if (step == 1)
            k.s[r][i] = *reinterpret_cast<const uint2 *>(p);
        else if (step == 2)
            k.s[r][i].x = *reinterpret_cast<const unsigned *>(p);
        else
            k.s[r][i].x = *p;
    };
    const int groups = (tiles + R - 1) / R;
#pragma unroll
    for (int i = 0; i < BP; ++i)
#pragma unroll
        for (int r = 0; r < R; ++r) load(blockIdx.x, r, i);

    bf16x8 x[MT][BP][4][PARTS];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int64_t t = token0 + 16 * m + (lane & 15);
        const T *row = static_cast<const T *>(a.x) + (t < a.tokens ? t : 0) * a.x_stride;
#pragma unroll
        for (int i = 0; i < BP; ++i) {
            const int64_t k0 = (int64_t)(block0 + i * WAVES) * 128;
            Eight<DT> v[4];
            if (k0 + 128 <= a.cols) {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j].load(row + k0 + j * 32 + (lane >> 4) * 8, t < a.tokens);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int64_t k = k0 + j * 32 + (lane >> 4) * 8;
                    if (k + 8 <= a.cols)
                        v[j].load(row + k, t < a.tokens);
                    else
                        v[j].load_singly(row, k, a.cols, t < a.tokens);
                    asm volatile("" ::: "memory"); // one after the other: together they would take most of the registers
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) parts_of(v[j], x[m][i][j]);
        }
    }

    int turn = 0;
    for (int group = blockIdx.x; group < groups; group += gridDim.x, turn ^= 1) {
        const int then = min(group + (int)gridDim.x, groups - 1);
        f32x4 acc[R][MT];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int m = 0; m < MT; ++m) acc[r][m] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < BP; ++i)
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const uint4 w = k.w[r][i];
                // beyond the last block: infinite scales would make NaN of the zeros
                const uint2 s2 = block0 + i * WAVES < blocks ? k.s[r][i] : make_uint2(0, 0);
                f32x4 part[MT];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (j % step == 0)
#pragma unroll
                        for (int m = 0; m < MT; ++m) part[m] = f32x4{0, 0, 0, 0};
                    const bf16x8 q = values_of((&w.x)[j]);
#pragma unroll
                    for (int m = 0; m < MT; ++m)
#pragma unroll
                        for (int p = 0; p < PARTS; ++p) part[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[m][i][j][p], q, part[m], 0, 0, 0);
                    if ((j + 1) % step == 0) { // the group ends here
                        const int g = step == 1 ? j : step == 2 ? j / 2 : 0; // of the block's groups
                        const unsigned u = g < 2 ? s2.x : s2.y;
                        const float s = __uint_as_float(g & 1 ? u & 0xffff0000u : u << 16);
#pragma unroll
                        for (int m = 0; m < MT; ++m)
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[r][m][e] = __builtin_fmaf(s, part[m][e], acc[r][m][e]);
                    }
                }
                load(then, r, i);
            }
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int m = 0; m < MT; ++m) sums[turn][wave][r * MT + m][lane] = acc[r][m];
        __syncthreads(); // the other turn's sums were read before this
        // every wave its share, V values a lane: a few waves alone would hold the others up (24 tokens, 100003 x 2048: 47 us, so 32)
        constexpr int V = R * MT % WAVES == 0 ? 4 : 2 * R * MT % WAVES == 0 ? 2 : 1, AHEAD = V == 4 ? 4 : 8; // more would cost registers that hold x
        typedef float Values __attribute__((ext_vector_type(V)));
        for (int at = threadIdx.x; at < R * MT * 256 / V; at += WAVES * 64) {
            const int tile = at / (256 / V), r = tile / MT, m = tile - r * MT, l = at / (4 / V) & 63;
            const int64_t n = ((int64_t)group * R + r) * 16 + (l & 15), t = token0 + 16 * m + (l >> 4) * 4 + at % (4 / V) * V;
            if (n >= a.rows || t >= a.tokens) continue;
            const Values *z = reinterpret_cast<const Values *>(&sums[turn][0][0][0]) + at;
            Values y = z[0];
#pragma unroll AHEAD
            for (int w = 1; w < WAVES; ++w) y += z[w * (R * MT * 256 / V)];
            const float bias = a.bias && !partial ? a.bias[n] : 0.0f;
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (t + e < a.tokens) {
                    const float v = y[e];
                    if (partial)
                        partial[((int64_t)blockIdx.y * a.tokens + t + e) * a.rows + n] = v;
                    else
                        static_cast<T *>(a.y)[(t + e) * a.y_stride + n] = Elem<DT>::put(v + bias);
                }
        }
    }
}

// The parts' sums, in order; blockIdx.y: the token.
template <int DT>
__global__ __launch_bounds__(256) void join_parts_kernel(const cbinfer_quantised_product_args a, int parts, const float *partial)
{
    const int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x, step = a.tokens * a.rows;
    if (n >= a.rows) return;
    for (int64_t t = blockIdx.y; t < a.tokens; t += gridDim.y) {
        const float *p = partial + t * a.rows + n;
        float y = a.bias ? a.bias[n] : 0.0f;
        int i = 0;
        for (; i + 8 <= parts; i += 8) {
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = p[(i + k) * step];
#pragma unroll
            for (int k = 0; k < 8; ++k) y += v[k];
        }
        for (; i < parts; ++i) y += p[i * step];
        static_cast<typename Elem<DT>::type *>(a.y)[t * a.y_stride + n] = Elem<DT>::put(y);
    }
}

// PER_CU: workgroups that run on a compute unit at a time.
template <int DT, int MT, int BP, int R, int WAVES, int PER_CU>
struct Shape {
    static int parts(const cbinfer_quantised_product_args &a) { return (int)((blocks_of(a.cols) + WAVES * BP - 1) / (WAVES * BP)); }
    static hipError_t run(hipStream_t st, const cbinfer_quantised_product_args &a)
    {
        const int64_t tiles = tiles_of(a.rows), blocks = blocks_of(a.cols), groups = (tiles + R - 1) / R;
        const uint16_t *scales = reinterpret_cast<const uint16_t *>(static_cast<const char *>(a.packed) + code_bytes(a.rows, a.cols));
        const int n = parts(a);
        float *partial = n > 1 ? static_cast<float *>(a.workspace) : nullptr;
        const unsigned z = (unsigned)((a.tokens + 16 * MT - 1) / (16 * MT));
        // as many workgroups as run at a time, each with the same number of turns or one less
        const int64_t room = std::max<int64_t>(1, 256 * PER_CU / (n * z)), turns = (groups + room - 1) / room;
        const dim3 grid((unsigned)((groups + turns - 1) / turns), n, z);
        product_kernel<DT, MT, BP, R, WAVES, PER_CU><<<grid, WAVES * 64, 0, st>>>(a, scales, (int)blocks, (int)tiles, partial);
        if (hipError_t e = hipGetLastError()) return e;
        if (partial) {
            join_parts_kernel<DT><<<dim3((unsigned)((a.rows + 255) / 256), (unsigned)std::min<int64_t>(a.tokens, 1024)), 256, 0, st>>>(a, n, partial);
            return hipGetLastError();
        }
        return hipSuccess;
    }
};

// A wave a block, and as many more workgroups: 54 tokens, 42672 x 168: two waves 12.8 us, eight 19.9; 1 token, 100003 x 512: four 9.0, eight 13.6.
template <int DT, int MT, int R, typename F>
auto short_rows(int64_t blocks, F f)
{
    if (blocks <= 2) return f(Shape<DT, MT, 1, R, 2, 8>());
    if (blocks <= 4) return f(Shape<DT, MT, 1, R, 4, 4>());
    return f(Shape<DT, MT, 1, R, 8, 2>());
}

// Calls f with the shape for these sizes.  A workgroup's waves times their blocks should be the blocks of a row, or a part of
// them without much left over: waves without a block wait for the others.
template <int DT, typename F>
auto with_shape(const cbinfer_quantised_product_args &a, F f)
{
    const int64_t tiles = tiles_of(a.rows), blocks = blocks_of(a.cols);
    if constexpr (DT == kBF16) {
        if (a.tokens <= 16) {
            if (blocks <= 8) return short_rows<DT, 1, 4>(blocks, f);
            if (blocks > 16 && blocks <= 32) {
                // 1 token, 4096 x 4096: a row's tiles one by one 7.3, in two parts of 8 waves 14; 20000 x 4096: 11.1, two at a time 11.7
                if (tiles <= 512) return f(Shape<DT, 1, 2, 1, 16, 1>());
                // 16 tokens, 100003 x 4096: 46.7, tiles one by one 57.7
                return f(Shape<DT, 1, 2, 2, 16, 1>());
            }
            // 16 tokens, 100003 x 2048 (115 MB): 29.8, four tiles at a time 31.5, two 48, of 8 waves with two blocks each 32.6; 4 tokens,
            // 4729 x 20806: 19.7, parts of 32 blocks 23.7
            return f(Shape<DT, 1, 1, 3, 16, 1>());
        }
        // 17 tokens, 40000 x 1000: 14.1, of 16 waves, half of them without a block, 18.2
        if (blocks <= 8) return short_rows<DT, 2, 2>(blocks, f);
        if (a.tokens > 32 && tiles >= 1024) {
            // three tiles of tokens at a time, 48 tokens, 100003 x 2048: 47, four 58; 37 tokens, 56488 x 1310: 29, 35
            if (a.tokens <= 48) return f(Shape<DT, 3, 2, 2, 8, 1>());
            // 64 tokens, 100003 x 2048 in groups of 128: 16 waves 56, eight with two blocks each 72; 20000 x 1500: 17.2, 20.7
            if (blocks <= 16) return f(Shape<DT, 4, 1, 1, 16, 1>());
            // 256 tokens, 20000 x 4096: 97, 16 waves 105, two tiles of tokens 115
            return f(Shape<DT, 4, 2, 2, 8, 1>());
        }
        // 64 tokens, 4096 x 4096: 16 waves and a tile at a time, which take rows whole, 10.2, two tiles in two parts 13.7, of 8 waves 14.5
        // (24 tokens, 50000 x 4096: 53, as the weights pass twice, and two tiles 43)
        if (blocks > 16 && blocks <= 32 && tiles < 1024) return f(Shape<DT, 1, 2, 2, 16, 1>());
        if (blocks > 16 && blocks <= 32) return f(Shape<DT, 2, 2, 2, 8, 1>());
        // 64 tokens, 8192 x 2048: 9.4, one tile at a time 16.7, 8 waves 10.9; 256 x 38400: 14.1, 16.1, 16.9
        return f(Shape<DT, 2, 1, 2, 16, 1>());
    } else {
        // three parts of x take three times the registers
        if (a.tokens <= 16 && blocks <= 8) return short_rows<DT, 1, 4>(blocks, f);
        // 17 tokens, 40000 x 1000: 16, of 16 waves 25
        if (blocks <= 8) return short_rows<DT, 1, 2>(blocks, f);
        // 16 tokens, 100003 x 2048: 30.7, of 8 waves 40.6; 36122 x 5669: 44.6, 46.1.  64 tokens, 256 x 38400: 17.7, 8 waves and two tiles of
        // tokens at a time 21.2, four tiles of rows 20.4
        if (a.tokens <= 16 || tiles < 64) return f(Shape<DT, 1, 1, 2, 16, 1>());
        // 64 tokens, 8192 x 2048: 12.7, three tiles at a time 14.3; 100003 x 2048: 113, 103
        if (tiles < 1024) return f(Shape<DT, 1, 1, 4, 16, 1>());
        return f(Shape<DT, 1, 1, 3, 16, 1>());
    }
}

} // namespace

hipError_t quantise_weights(hipStream_t st, const void *weights, int dtype, int64_t rows, int64_t cols, int64_t row_stride,
                            int group, uint8_t *codes, uint16_t *scales)
{
    const int64_t groups = (cols + group - 1) / group;
    constexpr int64_t kMostBlocks = 1 << 22; // of a launch: threads are counted in 32 bits
    for (int64_t first = 0; first < rows * groups; first += 8 * kMostBlocks) {
        const unsigned grid = (unsigned)std::min(kMostBlocks, (rows * groups - first + 7) / 8);
        if (dtype == kF32)
            quantise_kernel<kF32><<<grid, 256, 0, st>>>(static_cast<const float *>(weights), rows, cols, row_stride, group, groups, first, codes, scales);
        else
            quantise_kernel<kBF16><<<grid, 256, 0, st>>>(static_cast<const uint16_t *>(weights), rows, cols, row_stride, group, groups, first, codes, scales);
        if (hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

size_t packed_weights_bytes(int64_t rows, int64_t cols, int group)
{
    return code_bytes(rows, cols) + (size_t)(tiles_of(rows) * blocks_of(cols)) * 16 * (128 / group) * 2;
}

hipError_t pack_weights(hipStream_t st, const uint8_t *codes, const uint16_t *scales, int64_t rows, int64_t cols, int group,
                        void *packed)
{
    const int64_t blocks = blocks_of(cols), units = tiles_of(rows) * blocks * 64, per_block = 128 / group, total = units / 4 * per_block;
    const auto pack = cols % 8 == 0 && reinterpret_cast<uintptr_t>(codes) % 8 == 0 ? pack_codes_kernel<true> : pack_codes_kernel<false>;
    pack<<<(unsigned)((units + 255) / 256), 256, 0, st>>>(codes, rows, cols, blocks, units, static_cast<uint4 *>(packed));
    if (hipError_t e = hipGetLastError()) return e;
    pack_scales_kernel<<<(unsigned)((total + 255) / 256), 256, 0, st>>>(scales, rows, (cols + group - 1) / group, blocks, (int)per_block, total,
        reinterpret_cast<uint16_t *>(static_cast<char *>(packed) + code_bytes(rows, cols)));
    return hipGetLastError();
}

size_t quantised_product_workspace(const cbinfer_quantised_product_args &a)
{
    const auto parts = [&](auto shape) { return shape.parts(a); };
    const int n = a.dtype == kF32 ? with_shape<kF32>(a, parts) : with_shape<kBF16>(a, parts);
    return n > 1 ? (size_t)n * a.tokens * a.rows * sizeof(float) : 0;
}

hipError_t quantised_product(hipStream_t st, const cbinfer_quantised_product_args &a)
{
    const auto run = [&](auto shape) { return shape.run(st, a); };
    return a.dtype == kF32 ? with_shape<kF32>(a, run) : with_shape<kBF16>(a, run);
}

} // namespace cbk
