// Linear attention with a decay for each head.
//
// S_t = g S_(t-1) + k_t (x) v_t, o_t = scale q_t S_t: every column of S (an index of v) is a recurrence of its own.
#include "tokens.h"

#include <algorithm>

namespace cbk {
namespace {

// Token after token, the state in registers.  A workgroup holds `columns` columns of one stream's head: DVL lanes side by
// side, VEC columns each, and 256 / DVL groups of lanes that share the rows (RPT each).  Bound by the state's way through memory
// where tokens are few (see plan()): it is read and written once, 128 bytes of a row by 8 lanes.  64 streams of 16 heads of 128 x 128, one token:
// 25 us for 135 MB, 5.4 TB/s; where rows of the state are not whole pieces of 16 bytes (128 x 127), a column a lane, 40.
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
// are matrix products.  A workgroup takes a stream's head and NC times 32 columns of v, two waves for each: one keeps the upper
// half of the rows of S in the accumulators of the matrix instruction from chunk to chunk, one the lower, and uses them as an
// operand as they lie there: the order in which a sum over rows of S runs is free, so Q is read in the order that the accumulators
// have.  The two exchange half of their parts of Q S through LDS and then have 32 queries each.  Q, K, V and
// the scores lie in LDS, the next chunk's are on their way in registers.
//
// A workgroup of eight waves takes 6.4 us for 64 tokens and a state of 128 x 128 in bfloat16: 1.7 us of matrix instructions, 2.5 of other
// vector instructions (splitting values most of all), three barriers, and the two waves of a SIMD hardly overlap the two kinds.
// 8192 tokens of 16 such heads: outputs 57 us for 134 MB, the joining of 16 parts among them (without it 51), before that what the parts
// leave 22.
//
// bfloat16: what is computed on the way (scores, states, faded values) enters a product as a sum of three bfloat16, 24 bits: exactly.
// float32: the float32 instruction.
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kChunk = 64;

// Memory with its size: what is read beyond it is zero, what is written there is dropped, so that ragged edges take no branches
// (code that runs once is fetched from far away, and costs more than it executes).  Offsets in bytes; kBeyond is beyond any.
typedef __amdgpu_buffer_rsrc_t Buffer;
constexpr unsigned kBeyond = 0x80000000u;
__device__ __forceinline__ Buffer buffer(const void *p, unsigned bytes) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, bytes, 0x00027000); }

// 32 x 32 and 16 x 16
__device__ __forceinline__ f32x16 multiply(const u32x4 &a, const u32x4 &b, const f32x16 &c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 multiply(float a, float b, const f32x16 &c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 multiply(const u32x4 &a, const u32x4 &b, const f32x4 &c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 multiply(float a, float b, const f32x4 &c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// Four bfloat16 of a column: 16 lanes give the addresses of four rows' four times four.
__device__ __forceinline__ uint2 across_rows(const unsigned short *from)
{
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)from));
}

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

template <int DT, int KT, int NC, bool OUT>
struct alignas(16) ChunkLds {
    typedef typename Elem<DT>::type T;
    // Rows are 16 bytes longer so that lanes which read as much of a row each reach different banks; bfloat16 K and V are read across
    // their rows too, see swizzle().
    static constexpr int K = 32 * KT, V = 32 * NC, PAD = 16 / (int)sizeof(T), ACROSS = DT == kBF16 ? 0 : PAD;
    T k[kChunk][K + ACROSS], v[kChunk][V + ACROSS], q[OUT ? kChunk : 1][K + PAD];
    // Scores, by query; bfloat16: in three parts, and the first 32 queries have rows of 32 keys, so that two workgroups of two tiles and keys
    // of 128 find room in a compute unit.
    static constexpr int LONG = kChunk + PAD, SHORT = DT == kBF16 ? kChunk / 2 + PAD : LONG, PARTS = DT == kBF16 ? 3 : 1;
    static __device__ __forceinline__ int query(int i) { return SHORT == LONG || i < kChunk / 2 ? i * SHORT : kChunk / 2 * SHORT + (i - kChunk / 2) * LONG; }
    T p[PARTS][OUT ? kChunk / 2 * (SHORT + LONG) : 1];
    f32x4 other[OUT ? 2 * NC : 1][4][64]; // a wave's part of Q S for the queries of the wave beside it
    float fade_v[kChunk];        // g^(m-1) ... g^0 of the chunk at hand, then ones
    float fade_q[kChunk];        // scale g^1 ... scale g^64
    float fade_back[2 * kChunk]; // scale g^63 ... scale g^0, then zeros
    float fade[kChunk + 1];      // g^0 ... g^64
    int odd[2];                  // whether the chunk, and the next, hold a value that is not finite
};

// bfloat16 K is read along its rows for the scores (16 rows, 16 bytes of each) and across them for the state (four rows, 64
// bytes of each): its pieces of 16 bytes change places within 256 bytes so that either takes 256 bytes from all the banks.  What
// to exclusive-or a piece's number with.
template <int KT>
__device__ __forceinline__ int swizzle(int row)
{
    return KT == 2 ? (row & 2) << 1 | (row >> 2 & 3) : (row & 3) << 2 | (row >> 2 & 3);
}

// V is read across its rows alone: what to exclusive-or a column with.
template <int NC>
__device__ __forceinline__ int swizzle_across(int row)
{
    return NC == 2 ? (row & 2) << 4 : (row & 3) << 5;
}

// Outputs and states are sums over the keys' values: float32 keys of more than 128, of which a chunk does not fit LDS, are taken in
// pieces, each with its rows of the states, and every piece after the first adds to the outputs.
struct Keys {
    int64_t state; // from a head's state to the next
    bool add;
    bool fold; // the outputs' kernel joins the parts itself
};

// OUT: outputs of the tokens of a part (`per` chunks) of the sequence, from the state in front of it.  Otherwise what those
// tokens leave in a state of zero, the first part's in the state that is there, where further tokens follow.  `states`:
// [stream][head][part][key_size][value_size], first the state that was there, then what part 0, 1, ... leaves.
// WHOLE: rows are pieces of 16 bytes at 16-byte addresses.
template <int DT, int KT, int NC, bool OUT, bool WHOLE>
__global__ __launch_bounds__(NC * 128, NC == 4 || DT == kBF16 ? 2 : 1) void chunk_kernel(const cbinfer_linear_attention_args a, int slices, int per, int parts, float *states, Keys keys)
{
    typedef typename Elem<DT>::type T;
    typedef ChunkLds<DT, KT, NC, OUT> Lds;
    constexpr int E = 16 / (int)sizeof(T), NT = NC * 128, KH = KT / 2; // E: values in 16 bytes
    constexpr int KW = Lds::K / E, VW = Lds::V / E, KR = NT / KW, VR = NT / VW; // pieces of 16 bytes in a row, rows at a time
    constexpr int KP = kChunk / KR, VP = kChunk / VR;
    static_assert(KR * KW == NT && VR * VW == NT && KP >= 1 && VP >= 1, "whole rows at a time");
    __shared__ Lds lds;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), side = lane & 31, half = lane >> 5, low = (wave ^ wave >> 2) & 1, tile = wave >> 1;
    const int slice = blockIdx.x % slices, bh = blockIdx.x / slices, b = bh / a.heads, h = bh - b * a.heads, hk = h / (a.heads / a.kv_heads);
    const int part = blockIdx.y, dk = a.key_size, dv = a.value_size, column = slice * Lds::V + tile * 32 + side;
    const int n = a.lengths ? min(max(a.lengths[b], 0), a.tokens) : a.tokens;
    const int t0 = part * per * kChunk, t1 = min(n, t0 + per * kChunk);
    T *o = static_cast<T *>(a.o) + b * a.o_stride[0] + h * a.o_stride[2];
    if (OUT) {
        const int end = min(a.tokens, t0 + per * kChunk);
        for (int64_t t = max(n, t0) + 2 * low + half; t < end; t += 4)
            if (column < dv) o[t * a.o_stride[1] + column] = Elem<DT>::put(0.0f);
        if (t0 >= n) return;
    } else if (t0 + per * kChunk >= n) {
        return;
    }

    // what this thread brings of a chunk: pieces at one place of the row, KR (VR) rows apart
    const int krow = threadIdx.x / KW, kcol = threadIdx.x % KW * E, vrow = threadIdx.x / VW, vcol = threadIdx.x % VW * E;
    const int vsize = dv - slice * Lds::V;
    const T *q = static_cast<const T *>(a.q) + b * a.q_stride[0] + h * a.q_stride[2] + t0 * a.q_stride[1];
    const T *k = static_cast<const T *>(a.k) + b * a.k_stride[0] + hk * a.k_stride[2] + t0 * a.k_stride[1];
    const T *v = static_cast<const T *>(a.v) + b * a.v_stride[0] + hk * a.v_stride[2] + t0 * a.v_stride[1] + slice * Lds::V;
    auto rows = [&](auto &r, const T *from, int64_t stride, int tokens, int row, int col, int step, int size) {
        constexpr int N = sizeof(r) / sizeof(r[0]);
        if constexpr (WHOLE) {
            const unsigned each = (unsigned)stride * sizeof(T);
            const Buffer x = buffer(from, (min(tokens, kChunk) - 1) * each + size * sizeof(T));
            unsigned at = col < size ? row * each + col * (unsigned)sizeof(T) : kBeyond;
#pragma unroll
            for (int i = 0; i < N; ++i, at += step * each) r[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(x, at, 0, 0));
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                union { T e[E]; u32x4 v; } u;
                u.v = u32x4{0, 0, 0, 0};
                const T *p = from + (row + i * step) * stride + col;
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (row + i * step < tokens && col + e < size) u.e[e] = p[e];
                r[i] = u.v;
            }
        }
    };
    u32x4 qr[OUT ? KP : 1], kr[KP], vr[VP];
    auto load = [&](int tokens) { // those left
        if constexpr (OUT) rows(qr, q, a.q_stride[1], tokens, krow, kcol, KR, dk);
        rows(kr, k, a.k_stride[1], tokens, krow, kcol, KR, dk);
        rows(vr, v, a.v_stride[1], tokens, vrow, vcol, VR, vsize);
        q += kChunk * a.q_stride[1];
        k += kChunk * a.k_stride[1];
        v += kChunk * a.v_stride[1];
    };
    load(t1 - t0);

    const float g = a.decay[h];
    if (threadIdx.x < kChunk) {
        const int i = threadIdx.x;
        const float f = power(g, i);
        lds.fade_v[kChunk - 1 - i] = f;
        lds.fade_back[kChunk - 1 - i] = a.scale * f;
        lds.fade_back[kChunk + i] = 0.0f;
        const float next = power(g, i + 1);
        lds.fade_q[i] = a.scale * next;
        lds.fade[i + 1] = next;
        if (i == 0) lds.fade[0] = 1.0f;
    }
    if (threadIdx.x < 2) lds.odd[threadIdx.x] = 0;
    if (OUT) // scores of later keys in the tiles that are multiplied all the same
        for (int i = threadIdx.x; i < 2 * 16 * 16; i += NT) {
            const int at = i >> 8, row = 32 * at + (i >> 4 & 15), col = 32 * at + 16 + (i & 15);
#pragma unroll
            for (int part = 0; part < Lds::PARTS; ++part) lds.p[part][Lds::query(row) + col] = 0;
        }

    // rows of S: row0 + 32 kt + 8 (r / 4) + r % 4 for register r; the lane's column
    const int row0 = 32 * KH * low + 4 * half;
    const unsigned state_bytes = (unsigned)(dk * dv) * 4, state_at = column < dv ? (unsigned)(row0 * dv + column) * 4 : kBeyond;
    auto place = [&](int kt, int r) { return state_at + (unsigned)((32 * kt + 8 * (r / 4) + r % 4) * dv) * 4; };
    f32x16 S[KH] = {};
    float *state = a.state + bh * keys.state;
    const int64_t size = (int64_t)dk * dv;
    states += bh * parts * size;
    if (OUT || part == 0) {
        const bool whole = !OUT || n <= per * kChunk; // nobody else writes the state, or only later
        const Buffer from = buffer(whole ? state : states + (keys.fold ? min(part, 1) : part) * size, state_bytes), first = buffer(states, state_bytes);
#pragma unroll
        for (int kt = 0; kt < KH; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) S[kt][r] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(from, place(kt, r), 0, 0));
        if (!OUT) {
#pragma unroll
            for (int kt = 0; kt < KH; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(S[kt][r]), first, place(kt, r), 0, 0);
        }
    }
    if (OUT && keys.fold) {
        const float through = power(g, per * kChunk);
        for (int p = 2; p <= part; ++p) {
            const Buffer from = buffer(states + p * size, state_bytes);
#pragma unroll
            for (int kt = 0; kt < KH; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    S[kt][r] = __builtin_fmaf(through, S[kt][r], __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(from, place(kt, r), 0, 0)));
        }
    }

    int turn = 0;
    for (int t = t0; t < t1; t += kChunk, turn ^= 1) {
        const int m = min(kChunk, t1 - t);
        __syncthreads(); // the chunk before is done with LDS
#pragma unroll
        for (int i = 0; i < KP; ++i) {
            const int kat = DT == kBF16 ? 8 * (kcol / 8 ^ swizzle<KT>(krow + i * KR)) : kcol;
            *reinterpret_cast<u32x4 *>(&lds.k[krow + i * KR][kat]) = kr[i];
            if (OUT) {
                const u32x4 &x = qr[OUT ? i : 0];
                if (DT == kBF16) { // of 16 values, groups of four in the order 0 2 1 3: as the accumulators have S
                    T *to = &lds.q[krow + i * KR][(kcol & ~15) + (kcol & 8 ? 4 : 0)];
                    *reinterpret_cast<uint2 *>(to) = make_uint2(x[0], x[1]);
                    *reinterpret_cast<uint2 *>(to + 8) = make_uint2(x[2], x[3]);
                } else {
                    *reinterpret_cast<u32x4 *>(&lds.q[krow + i * KR][kcol]) = x;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < VP; ++i) *reinterpret_cast<u32x4 *>(&lds.v[vrow + i * VR][DT == kBF16 ? vcol ^ swizzle_across<NC>(vrow + i * VR) : vcol]) = vr[i];
        if (OUT) {
            bool odd = false;
            if (DT == kBF16) {
                u16x2 most = {0, 0};
#pragma unroll
                for (int i = 0; i < VP; ++i)
#pragma unroll
                    for (int w = 0; w < 4; ++w) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, vr[i][w] & 0x7fff7fffu));
                odd = most[0] >= 0x7f80 || most[1] >= 0x7f80;
            } else {
                unsigned most = 0;
#pragma unroll
                for (int i = 0; i < VP; ++i)
#pragma unroll
                    for (int w = 0; w < 4; ++w) most = max(most, vr[i][w] & 0x7fffffffu);
                odd = most >= 0x7f800000u;
            }
            if (odd) lds.odd[turn] = 1;
        }
        if (m < kChunk && threadIdx.x < kChunk) lds.fade_v[threadIdx.x] = lds.fade[max(m - 1 - (int)threadIdx.x, 0)];
        __syncthreads();
        if (t + kChunk < t1) load(t1 - t - kChunk);

        // The wave's columns of V as the second operand of a product: bfloat16 of 16 tokens from 16 s on, 8 for either half of the lanes;
        // float32 of 8 from 8 c on, 4 for either.
        u32x4 vs[DT == kBF16 ? 4 : 8];
        if constexpr (DT == kBF16) {
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int row = 8 * half + (lane & 15) / 4;
                const T *from = &lds.v[16 * s + row][(tile * 32 + (lane & 16) + 4 * (lane & 3)) ^ swizzle_across<NC>(row)];
                const uint2 x = across_rows(from), y = across_rows(from + 4 * Lds::V);
                vs[s] = u32x4{x.x, x.y, y.x, y.y};
            }
        } else {
#pragma unroll
            for (int c = 0; c < 8; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) vs[c][e] = __float_as_uint(Elem<DT>::get(lds.v[8 * c + 4 * half + e][tile * 32 + side]));
        }

        f32x16 acc;
        if (OUT) {
            if (threadIdx.x == 0) lds.odd[turn ^ 1] = 0;
            // scores of 16 queries and 16 keys at a time, not of later keys: keys are the rows, so that a lane has four next to one another
            for (int at = wave; at < 10; at += 2 * NC) {
                const int it = at < 1 ? 0 : at < 3 ? 1 : at < 6 ? 2 : 3, j0 = 16 * (at - it * (it + 1) / 2), col = lane & 15, quarter = lane >> 4;
                f32x4 p = {0, 0, 0, 0};
                if constexpr (DT == kBF16) {
                    const T *kp = &lds.k[j0 + col][4 * (quarter & 1)], *qp = &lds.q[16 * it + col][8 * quarter];
                    const int piece = 2 * (quarter >> 1) ^ swizzle<KT>(col);
#pragma unroll 4
                    for (int s = 0; s < KT; ++s) {
                        const uint2 x = *reinterpret_cast<const uint2 *>(kp + 8 * (4 * s ^ piece)), y = *reinterpret_cast<const uint2 *>(kp + 8 * (4 * s + 1 ^ piece));
                        p = multiply(u32x4{x.x, x.y, y.x, y.y}, *reinterpret_cast<const u32x4 *>(qp + 32 * s), p);
                    }
                } else {
                    const T *kp = &lds.k[j0 + col][4 * quarter], *qp = &lds.q[16 * it + col][4 * quarter];
#pragma unroll 4
                    for (int s = 0; s < 2 * KT; ++s) {
                        const f32x4 x = *reinterpret_cast<const f32x4 *>(kp + 16 * s), y = *reinterpret_cast<const f32x4 *>(qp + 16 * s);
#pragma unroll
                        for (int e = 0; e < 4; ++e) p = multiply(x[e], y[e], p);
                    }
                }
                const int i = 16 * it + col, j = j0 + 4 * quarter;
                const float *fade = lds.fade_back + (kChunk - 1 - i + j);
                float x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = i >= j + e ? p[e] * fade[e] : 0.0f;
                const int to = Lds::query(i) + j;
                if constexpr (DT == kBF16) {
#pragma unroll
                    for (int part = 0; part < Lds::PARTS; ++part) {
                        *reinterpret_cast<uint2 *>(&lds.p[part][to]) = make_uint2(upper_halves(x[0], x[1]), upper_halves(x[2], x[3]));
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[e] -= cut(x[e]);
                    }
                } else {
                    *reinterpret_cast<f32x4 *>(&lds.p[0][to]) = f32x4{x[0], x[1], x[2], x[3]};
                }
            }
            // this wave's rows of S in Q S
            f32x16 qs[2] = {}; // for the queries that are its own, and for the other wave's
            const int across = 32 * (low ? -1 : 1) * (Lds::K + Lds::PAD);
#pragma unroll
            for (int kt = 0; kt < KH; ++kt) {
                if constexpr (DT == kBF16) {
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        float x[8];
                        u32x4 y[3];
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[e] = S[kt][8 * s + e];
                        split(x, y);
                        const T *qp = &lds.q[32 * low + side][32 * (KH * low + kt) + 16 * s + 8 * half];
                        const u32x4 z0 = *reinterpret_cast<const u32x4 *>(qp), z1 = *reinterpret_cast<const u32x4 *>(qp + across);
#pragma unroll
                        for (int i = 0; i < 3; ++i) {
                            qs[0] = multiply(z0, y[i], qs[0]);
                            qs[1] = multiply(z1, y[i], qs[1]);
                        }
                    }
                } else {
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const T *qp = &lds.q[32 * low + side][32 * (KH * low + kt) + 8 * c + 4 * half];
                        const f32x4 z0 = *reinterpret_cast<const f32x4 *>(qp), z1 = *reinterpret_cast<const f32x4 *>(qp + across);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            qs[0] = multiply(z0[e], S[kt][4 * c + e], qs[0]);
                            qs[1] = multiply(z1[e], S[kt][4 * c + e], qs[1]);
                        }
                    }
                }
            }
            acc = qs[0];
#pragma unroll
            for (int c = 0; c < 4; ++c) lds.other[wave ^ 1][c][lane] = f32x4{qs[1][4 * c], qs[1][4 * c + 1], qs[1][4 * c + 2], qs[1][4 * c + 3]};
        }

        // the state behind the chunk
        const float all = lds.fade[m];
#pragma unroll
        for (int kt = 0; kt < KH; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) S[kt][r] *= all;
        if constexpr (DT == kBF16) {
            const int in = lane & 15;
#pragma unroll 4
            for (int s = 0; s < 4; ++s) {
                const f32x4 f0 = *reinterpret_cast<const f32x4 *>(&lds.fade_v[16 * s + 8 * half]), f1 = *reinterpret_cast<const f32x4 *>(&lds.fade_v[16 * s + 8 * half + 4]);
                float x[8];
                u32x4 y[3];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(e & 1 ? vs[s][e / 2] & 0xffff0000u : vs[s][e / 2] << 16) * (e < 4 ? f0[e % 4] : f1[e % 4]);
                split(x, y);
#pragma unroll
                for (int kt = 0; kt < KH; ++kt) {
                    const int row = 8 * half + in / 4, piece = 4 * (KH * low + kt) + (lane >> 3 & 2) + (in >> 1 & 1);
                    const T *from = &lds.k[16 * s + row][8 * (piece ^ swizzle<KT>(row)) + 4 * (in & 1)];
                    const T *next = &lds.k[16 * s + row + 4][8 * (piece ^ swizzle<KT>(row + 4)) + 4 * (in & 1)];
                    const uint2 p = across_rows(from), u = across_rows(next);
#pragma unroll
                    for (int i = 0; i < 3; ++i) S[kt] = multiply(u32x4{p.x, p.y, u.x, u.y}, y[i], S[kt]);
                }
            }
        } else {
#pragma unroll 4
            for (int c = 0; c < 8; ++c) {
                const f32x4 f = *reinterpret_cast<const f32x4 *>(&lds.fade_v[8 * c + 4 * half]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = __uint_as_float(vs[DT == kBF16 ? 0 : c][e]) * f[e];
#pragma unroll
                    for (int kt = 0; kt < KH; ++kt) S[kt] = multiply(lds.k[8 * c + 4 * half + e][32 * (KH * low + kt) + side], x, S[kt]);
                }
            }
        }
        if (OUT) {
            __syncthreads(); // the scores are there, and the other wave's part
            const int i0 = 32 * low + 4 * half; // of register r: query i0 + 8 (r / 4) + r % 4
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const f32x4 x = lds.other[wave][c][lane], f = *reinterpret_cast<const f32x4 *>(&lds.fade_q[i0 + 8 * c]);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[4 * c + e] = (acc[4 * c + e] + x[e]) * f[e];
            }
            const T *scores = &lds.p[0][Lds::query(32 * low + side)];
            if (!lds.odd[turn]) {
                if constexpr (DT == kBF16) {
#pragma unroll
                    for (int s = 0; s < 4; ++s)
                        if (s < 2 + 2 * low)
#pragma unroll
                            for (int i = 0; i < 3; ++i) acc = multiply(*reinterpret_cast<const u32x4 *>(scores + i * (sizeof(lds.p[0]) / sizeof(T)) + 16 * s + 8 * half), vs[s], acc);
                } else {
#pragma unroll
                    for (int c = 0; c < 8; ++c)
                        if (c < 4 + 4 * low) {
                            const f32x4 z = *reinterpret_cast<const f32x4 *>(scores + 8 * c + 4 * half);
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc = multiply(z[e], __uint_as_float(vs[c % (DT == kBF16 ? 4 : 8)][e]), acc);
                        }
                }
            } else { // a value that is not finite: its product with the score 0 of an earlier token must not be added
                for (int j = 0; j < m; ++j) {
                    const float x = Elem<DT>::get(lds.v[j][DT == kBF16 ? (tile * 32 + side) ^ swizzle_across<NC>(j) : tile * 32 + side]);
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int i = i0 + 8 * (r / 4) + r % 4;
                        if (i >= j) {
                            float p = 0.0f;
#pragma unroll
                            for (int part = Lds::PARTS - 1; part >= 0; --part) p += Elem<DT>::get(lds.p[part][Lds::query(i) + j]);
                            acc[r] = __builtin_fmaf(p, x, acc[r]);
                        }
                    }
                }
            }
            if constexpr (WHOLE) {
                const unsigned each = (unsigned)a.o_stride[1] * sizeof(T), from = column < dv ? i0 * each + column * (unsigned)sizeof(T) : kBeyond;
                const Buffer to = buffer(o + t * a.o_stride[1], (m - 1) * each + dv * sizeof(T));
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const unsigned at = from + (8 * (r / 4) + r % 4) * each;
                    if (DT == kF32 && keys.add) acc[r] += __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(to, at, 0, 0));
                    if constexpr (DT == kBF16)
                        __builtin_amdgcn_raw_buffer_store_b16(Elem<DT>::put(acc[r]), to, at, 0, 0);
                    else
                        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(acc[r]), to, at, 0, 0);
                }
            } else {
                T *to = o + (int64_t)(t + i0) * a.o_stride[1] + column;
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (i0 + 8 * (r / 4) + r % 4 < m && column < dv) {
                        T &x = to[(8 * (r / 4) + r % 4) * a.o_stride[1]];
                        x = Elem<DT>::put(DT == kF32 && keys.add ? acc[r] + Elem<DT>::get(x) : acc[r]);
                    }
            }
        }
    }

    if (!OUT || t1 == n) { // the part with the last token
        const Buffer to = buffer(OUT ? state : states + (part + 1) * size, state_bytes);
#pragma unroll
        for (int kt = 0; kt < KH; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(S[kt][r]), to, place(kt, r), 0, 0);
    }
}

// What the parts of a sequence leave (places 1, 2, ...) becomes the states in front of the parts.  Bound by memory: 16 heads of
// 128 x 128 in 16 parts, 33 MB, 8 us.
__global__ __launch_bounds__(256) void join_parts_kernel(const cbinfer_linear_attention_args a, int per, int parts, float *states)
{
    const int bh = blockIdx.y, size = a.key_size * a.value_size, at = blockIdx.x * 256 + threadIdx.x, b = bh / a.heads;
    if (at >= size) return;
    const int n = a.lengths ? min(max(a.lengths[b], 0), a.tokens) : a.tokens;
    const int last = (int)min((int64_t)parts, ((int64_t)n + per * kChunk - 1) / (per * kChunk)); // parts with tokens
    if (last <= 2) return;
    const float g = power(a.decay[bh - b * a.heads], per * kChunk);
    float *s = states + (int64_t)bh * parts * size + at, x = s[size];
    for (int p0 = 2; p0 < last; p0 += 8) { // eight loads on their way at a time
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = p0 + i < last ? s[(int64_t)(p0 + i) * size] : 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x = __builtin_fmaf(g, x, v[i]);
            if (p0 + i < last) s[(int64_t)(p0 + i) * size] = x;
        }
    }
}

struct Plan {
    bool chunks;
    int slices, per, parts, tiles; // tiles: of 32 columns a workgroup
};

Plan plan(const cbinfer_linear_attention_args &a)
{
    Plan p = {false, 1, 1, 1, 4};
    // us for 64 streams, 16 heads of 128 x 128, token after token and in chunks: bfloat16 4 tokens 36.5, 40.2, 5 tokens 40.1, 39.5, 8 tokens 51, 39; float32
    // 12 tokens 57, 75; 16 streams, 8 heads, bfloat16 4 tokens 8.7, 9.4, 5 tokens 9.7, 9.4, float32 15 tokens: 19, 17.
    if (a.tokens < (a.dtype == kF32 ? 16 : 5)) return p;
    p.chunks = true;
    const int tiles = (a.value_size + 31) / 32;
    const int64_t heads = (int64_t)a.streams * a.heads, chunks = (a.tokens + kChunk - 1) / kChunk;
    // Two tiles where all chunks together do not fill the chip twice: their scores are computed twice, but four waves are through sooner
    // than eight.  us for 82 tokens, 4 heads of 96 x 128 float32: 24, four tiles 28; 8192 tokens, 16 heads: 86, 77.
    p.tiles = (a.dtype == kF32 || a.key_size <= 128) && (tiles <= 2 || heads * ((tiles + 1) / 2) * chunks <= 512) ? 2 : 4;
    p.slices = (tiles + p.tiles - 1) / p.tiles;
    const int64_t groups = heads * p.slices;
    // Parts until every compute unit has a workgroup; their keys and values are read twice.  us for 8192 tokens, 16 heads of 128: 8 parts 107,
    // 16 78, 20 107.  Streams of different lengths leave compute units idle: half as many again (12 streams of up to 1023 tokens, 6 heads,
    // float32: 3 parts 83, 6 62, 7 70, 8 64).  Of two tiles in bfloat16 a compute unit takes two workgroups (6 streams of 1749 tokens, 12 heads
    // of 96 x 64: 51, with one 64).
    const int64_t room = (a.lengths ? 400 : 256) * (p.tiles == 2 && a.dtype == kBF16 ? 2 : 1);
    // From 256 on they do not pay (16 streams of up to 500 tokens, 16 heads of 64 x 64: 32, in three parts 35); below, already with three chunks
    // (2 streams of 190 tokens, 16 heads of 128 x 128: 16.6, in three parts 14.1; two chunks, 2 streams of 100, 4 heads of 64 x 64: 10.3, 11.9), in
    // float32 with two (4 streams of 100 tokens, 4 heads of 64 x 128: 18.6, 17.0).
    const bool pays = groups < 256 && chunks > (a.dtype == kF32 ? 1 : 2);
    p.parts = pays ? (int)std::max<int64_t>(1, std::min(chunks, room / std::max<int64_t>(groups, 1))) : 1;
    p.per = (int)((chunks + p.parts - 1) / p.parts);
    p.parts = (int)((chunks + p.per - 1) / p.per);
    return p;
}

template <int DT, int KT, int NC, bool WHOLE>
hipError_t chunked(hipStream_t st, const cbinfer_linear_attention_args &a, const Plan &p, const Keys &keys)
{
    float *states = static_cast<float *>(a.workspace);
    const unsigned groups = (unsigned)(a.streams * a.heads * p.slices);
    if (p.parts > 1) {
        chunk_kernel<DT, KT, NC, false, WHOLE><<<dim3(groups, p.parts - 1), NC * 128, 0, st>>>(a, p.slices, p.per, p.parts, states, keys);
        if (hipError_t err = hipGetLastError()) return err;
        if (!keys.fold) {
            join_parts_kernel<<<dim3((a.key_size * a.value_size + 255) / 256, a.streams * a.heads), 256, 0, st>>>(a, p.per, p.parts, states);
            if (hipError_t err = hipGetLastError()) return err;
        }
    }
    chunk_kernel<DT, KT, NC, true, WHOLE><<<dim3(groups, p.parts), NC * 128, 0, st>>>(a, p.slices, p.per, p.parts, states, keys);
    return hipGetLastError();
}

constexpr int kKeys = 128; // at a time, float32
constexpr int kFold = 16; // parts up to which the outputs' kernel joins them: 4 streams of 1000 tokens, 16 heads of 128 x 128, 4 parts: 43 us, joined before 51; one of 8192, 16 parts: 75, 74

template <int DT, bool WHOLE>
hipError_t chunked_any(hipStream_t st, const cbinfer_linear_attention_args &a, const Plan &p)
{
    if constexpr (DT == kBF16)
        if (a.key_size > 128) return chunked<DT, 8, 4, WHOLE>(st, a, p, {(int64_t)a.key_size * a.value_size, false, p.parts <= kFold});
    for (int k0 = 0; k0 < a.key_size; k0 += kKeys) { // once but for float32 keys of more than 128
        cbinfer_linear_attention_args b = a;
        b.key_size = std::min(a.key_size - k0, kKeys);
        b.q = static_cast<const typename Elem<DT>::type *>(a.q) + k0;
        b.k = static_cast<const typename Elem<DT>::type *>(a.k) + k0;
        b.state = a.state + (int64_t)k0 * a.value_size;
        const Keys keys = {(int64_t)a.key_size * a.value_size, k0 > 0, p.parts <= kFold};
        const hipError_t err = b.key_size <= 64 ? p.tiles == 2 ? chunked<DT, 2, 2, WHOLE>(st, b, p, keys) : chunked<DT, 2, 4, WHOLE>(st, b, p, keys)
                                                : p.tiles == 2 ? chunked<DT, 4, 2, WHOLE>(st, b, p, keys) : chunked<DT, 4, 4, WHOLE>(st, b, p, keys);
        if (err) return err;
    }
    return hipSuccess;
}

template <int DT>
hipError_t chunked_any(hipStream_t st, const cbinfer_linear_attention_args &a, const Plan &p)
{
    const size_t e = DT == kF32 ? 4 : 2;
    // rows at 16-byte addresses, those of a chunk in order and within the 31 bits of a buffer's offsets
    auto fits = [&](const void *x, const int64_t *stride, int size) {
        for (int i = 0; i < 3; ++i)
            if (stride[i] * e % 16) return false;
        return reinterpret_cast<uintptr_t>(x) % 16 == 0 && size * e % 16 == 0 && stride[1] >= size && stride[1] < (1 << 30) / (int64_t)(kChunk * e);
    };
    const bool whole = fits(a.q, a.q_stride, a.key_size) && fits(a.k, a.k_stride, a.key_size) && fits(a.v, a.v_stride, a.value_size) &&
                       fits(a.o, a.o_stride, a.value_size);
    return whole ? chunked_any<DT, true>(st, a, p) : chunked_any<DT, false>(st, a, p);
}

} // namespace

size_t linear_attention_workspace(const cbinfer_linear_attention_args &a)
{
    const Plan p = plan(a);
    const int keys = a.dtype == kF32 ? std::min(a.key_size, kKeys) : a.key_size;
    return p.parts > 1 ? (size_t)a.streams * a.heads * p.parts * keys * a.value_size * sizeof(float) : 0;
}

hipError_t linear_attention(hipStream_t st, const cbinfer_linear_attention_args &a)
{
    const Plan p = plan(a);
    if (p.chunks) return a.dtype == kF32 ? chunked_any<kF32>(st, a, p) : chunked_any<kBF16>(st, a, p);
    return a.dtype == kF32 ? recurrent_any<kF32>(st, a) : recurrent_any<kBF16>(st, a);
}

} // namespace cbk
