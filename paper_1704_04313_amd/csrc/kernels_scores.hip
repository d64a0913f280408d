// Log probabilities, entropy and alternatives of class scores, in one pass over the scores.
//
// A lane keeps the running maximum m, s = sum exp(x - m) and t = sum exp(x - m) (x - m) of the scores it
// has seen; a larger maximum m' multiplies both by exp(m - m') after t has taken (m - m') s.  Two such triples
// join the same way, and log s - t / s is the entropy: two terms of one sign, nothing cancels.
#include "tokens.h"

namespace cbk {
namespace {

constexpr float kLowest = -3.402823466e38f; // a maximum over nothing: finite, so that differences from it are no NaN

struct Sums {
    float m, s, t;
};

__device__ __forceinline__ void raise_to(Sums &a, float m)
{
    const float d = fmaxf(a.m - m, -1e4f); // exp is 0 far before; an infinite difference would make 0 * inf
    const float c = __expf(d);
    a.t = (a.t + a.s * d) * c;
    a.s *= c;
    a.m = m;
}

__device__ __forceinline__ void add(Sums &a, float x)
{
    const float d = x - a.m, e = __expf(d);
    a.s += e;
    a.t += e * fmaxf(d, -200.0f); // scores of -inf: e is 0
}

__device__ __forceinline__ void join(Sums &a, Sums b)
{
    const float m = fmaxf(a.m, b.m);
    raise_to(a, m);
    raise_to(b, m);
    a.s += b.s;
    a.t += b.t;
}

// The largest `k` of what a wave has seen, best first: lane j holds the one of rank j.  Among equal values the
// lower index comes first.  Places not taken yet hold -inf and an index behind all others.
struct Best {
    float v;
    int i;
    float least; // of rank k - 1, the same in every lane
    int n;       // places taken, the same in every lane
};
constexpr int kNone = 0x7fffffff;

__device__ __forceinline__ Best best_none() { return {-__builtin_inff(), kNone, -__builtin_inff(), 0}; }

__device__ __forceinline__ void insert(Best &b, int k, float x, int i)
{
    const int lane = threadIdx.x & 63;
    const bool before = lane < k && (b.v > x || (b.v == x && b.i < i));
    const int at = __popcll(__ballot(before));
    const float pv = __shfl_up(b.v, 1);
    const int pi = __shfl_up(b.i, 1);
    if (lane > at) { b.v = pv; b.i = pi; }
    if (lane == at) { b.v = x; b.i = i; }
    b.least = __shfl(b.v, k - 1);
    b.n = min(b.n + 1, k);
}

// What lanes hold is to be taken in lane order, which is the order of their indices: every lane whose x is larger than
// the least of the list (a full list keeps the earlier of equals).
__device__ __forceinline__ void offer(Best &b, int k, float x, int i, bool there)
{
    int from = 0;
    for (;;) {
        const unsigned long long m = __ballot(there && (b.n < k || x > b.least)) >> from << from;
        if (!m) return;
        const int l = __ffsll((long long)m) - 1;
        insert(b, k, __shfl(x, l), __shfl(i, l));
        if (l == 63) return;
        from = l + 1;
    }
}

// Order of scores with NaN in front of every number.
__device__ __forceinline__ int rank_key(float x)
{
    if (x != x) return kNone;
    const int b = __float_as_int(x + 0.0f);
    return b < 0 ? b ^ 0x7fffffff : b;
}

template <int DT>
__device__ __forceinline__ float score(const cbinfer_log_probs_args &a, int64_t at)
{
    return Elem<DT>::get(static_cast<const typename Elem<DT>::type *>(a.scores)[at]);
}

// Rows that hold a NaN or +inf: a wave finds the alternatives one after the other, each in a pass over the row.
template <int DT>
__device__ void careful_top(const cbinfer_log_probs_args &a, int64_t base, int64_t to)
{
    const int lane = threadIdx.x & 63;
    int key = kNone, index = -1; // the one found last; first: as if in front of every other
    for (int j = 0; j < a.top; ++j) {
        int bk = -kNone - 1, bi = kNone;
        for (int c = lane; c < (int)a.classes; c += 64) {
            const int k = rank_key(score<DT>(a, base + c * a.class_stride));
            const bool behind = j == 0 || k < key || (k == key && c > index);
            if (behind && (k > bk || (k == bk && c < bi))) { bk = k; bi = c; }
        }
        for (int off = 32; off; off >>= 1) {
            const int ok = __shfl_xor(bk, off), oi = __shfl_xor(bi, off);
            if (ok > bk || (ok == bk && oi < bi)) { bk = ok; bi = oi; }
        }
        key = bk;
        index = bi;
        if (lane == 0) {
            a.top_values[to + j * a.inner] = __builtin_nanf("");
            a.top_index[to + j * a.inner] = bi;
        }
    }
}

__device__ __forceinline__ float log_prob(float x, const Sums &t, float log_s)
{
    return t.s != t.s ? __builtin_nanf("") : t.s == 0.0f ? -__builtin_inff() : (x - t.m) - log_s;
}

// Label and entropy of a position from its sums: lane-wise work, `scores` at its base.
template <int DT>
__device__ __forceinline__ void write_position(const cbinfer_log_probs_args &a, int64_t pos, int64_t base, const Sums &t, float log_s)
{
    if (a.entropy) a.entropy[pos] = t.s != t.s ? __builtin_nanf("") : t.s == 0.0f ? 0.0f : log_s - t.t / t.s;
    if (a.label) {
        const int64_t l = a.label_bytes == 8 ? static_cast<const int64_t *>(a.labels)[pos] : static_cast<const int32_t *>(a.labels)[pos];
        float v = 0.0f;
        if (l >= a.classes)
            v = __builtin_nanf("");
        else if (l >= 0)
            v = log_prob(score<DT>(a, base + l * a.class_stride), t, log_s);
        a.label[pos] = v;
    }
}

// One wave a position, any strides.
template <int DT>
__global__ __launch_bounds__(256) void wave_kernel(const cbinfer_log_probs_args a)
{
    const int lane = threadIdx.x & 63;
    const int64_t pos = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (pos >= a.outer * a.inner) return;
    const int64_t o = pos / a.inner, i = pos - o * a.inner;
    const int64_t base = o * a.outer_stride + i * a.inner_stride, to = o * a.top * a.inner + i;
    Sums t = {kLowest, 0.0f, 0.0f};
    Best b = best_none();
    for (int64_t c0 = 0; c0 < a.classes; c0 += 64) {
        const int64_t c = c0 + lane;
        const bool there = c < a.classes;
        const float x = there ? score<DT>(a, base + c * a.class_stride) : -__builtin_inff();
        if (x > t.m) raise_to(t, x);
        add(t, x);
        if (a.top) offer(b, a.top, x, (int)c, there);
    }
    for (int off = 32; off; off >>= 1) join(t, {__shfl_xor(t.m, off), __shfl_xor(t.s, off), __shfl_xor(t.t, off)});
    const float log_s = logf(t.s);
    if (lane == 0) write_position<DT>(a, pos, base, t, log_s);
    if (!a.top) return;
    if (t.s != t.s) {
        careful_top<DT>(a, base, to);
    } else if (lane < a.top) {
        a.top_values[to + lane * a.inner] = log_prob(b.v, t, log_s);
        a.top_index[to + lane * a.inner] = b.i;
    }
}

} // namespace

size_t log_probs_workspace(const cbinfer_log_probs_args &) { return 0; }

hipError_t log_probs(hipStream_t st, const cbinfer_log_probs_args &a)
{
    const unsigned blocks = (unsigned)((a.outer * a.inner + 3) / 4);
    if (a.dtype == kF32)
        wave_kernel<kF32><<<blocks, 256, 0, st>>>(a);
    else
        wave_kernel<kBF16><<<blocks, 256, 0, st>>>(a);
    return hipGetLastError();
}

} // namespace cbk
