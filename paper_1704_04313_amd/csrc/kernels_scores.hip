// Log probabilities, entropy and alternatives of class scores, in one pass over the scores.
//
// A lane keeps the running maximum m, s = sum exp(x - m) and t = sum exp(x - m) (x - m) of the scores it
// has seen; a larger maximum m' multiplies both by exp(m - m') after t has taken (m - m') s.  Two such triples
// join the same way, and log s - t / s is the entropy: two terms of one sign, nothing cancels.
#include "tokens.h"
#include <algorithm>

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
    a.t = __builtin_fmaf(e, fmaxf(d, -200.0f), a.t); // scores of -inf: e is 0
}

__device__ __forceinline__ void join(Sums &a, Sums b)
{
    const float m = fmaxf(a.m, b.m);
    raise_to(a, m);
    raise_to(b, m);
    a.s += b.s;
    a.t += b.t;
}

constexpr int kNone = 0x7fffffff; // an index behind all others

// Order of scores with NaN in front of every number.
__device__ __forceinline__ int rank_key(float x)
{
    if (x != x) return kNone;
    const int b = __float_as_int(x + 0.0f);
    return b < 0 ? b ^ 0x7fffffff : b;
}
__device__ __forceinline__ float of_key(int key) { return __int_as_float(key < 0 ? key ^ 0x7fffffff : key); }

__device__ __forceinline__ float lane_value(float v, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); }
// The value of the lane before; lane 0 keeps its own.
__device__ __forceinline__ int from_lane_before(int v) { return __builtin_amdgcn_update_dpp(v, v, 0x138 /* wave_shr:1 */, 0xf, 0xf, false); }
__device__ __forceinline__ int lanes_below(unsigned long long m) { return __builtin_amdgcn_mbcnt_hi((unsigned)(m >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)m, 0)); }
__device__ __forceinline__ void wave_fence() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

struct Entry {
    float v;
    int i;
};
__device__ __forceinline__ bool better(const Entry &a, const Entry &b) { return a.v > b.v || (a.v == b.v && a.i < b.i); }

// The k best scores of what a wave has seen: the largest, the lower index first among equals.  While it looks, a wave only
// gathers candidates, in a buffer of 64 in LDS, against a bound that it raises now and then: keeping a list sorted score by
// score costs more than the sums.  A buffer that runs full is worked into a list, of which lane j holds rank j.
struct Best {
    Entry *buffer;
    int k, n;    // n: candidates in the buffer
    bool listed; // whether there is a list
    Entry mine;  // of the list
    // the same in every lane: a score has to exceed `least`, or equal it at a lower index than `last` -- those of rank k - 1 of the
    // list, or of a value that k of the scores at least reach, with the index behind all others
    float least;
    int last;

    __device__ __forceinline__ void begin(Entry *b, int k_)
    {
        buffer = b;
        k = k_;
        n = 0;
        listed = false;
        mine = {-__builtin_inff(), kNone};
        least = -__builtin_inff();
        last = kNone;
    }
    __device__ __forceinline__ bool wanted(const Entry &e) const { return e.v > least || (e.v == least && e.i < last); }
    // Whether any of several scores may be, `most` the largest, of higher indices than those in the list.
    __device__ __forceinline__ bool any_wanted(float most) const { return most > least || (last == kNone && most == least); }
    __device__ __forceinline__ void raise(float to, int at)
    {
        if (to > least || (to == least && at < last)) {
            least = to;
            last = at;
        }
    }
    // A value that k of the scores at least reach, from one score a lane: close to the k-th largest of these.  What is below
    // cannot be among the k largest.
    __device__ __forceinline__ void bound(float most)
    {
        const unsigned key = (unsigned)rank_key(most) ^ 0x80000000u; // ascending as unsigned numbers
        unsigned at = 0;
#pragma nounroll
        for (unsigned bit = 1u << 31; bit >= 1u << 16; bit >>= 1) // the upper half: somewhat below is a bound as well
            if (__popcll(__ballot(key >= (at | bit))) >= k) at |= bit;
        const float f = of_key((int)(at ^ 0x80000000u));
        if (f == f) raise(f, kNone);
    }
    __device__ void flush()
    {
        const int lane = threadIdx.x & 63;
        wave_fence();
        const Entry e = lane < n ? buffer[lane] : Entry{-__builtin_inff(), kNone};
        wave_fence();
        if (n >= k) bound(e.v);
        unsigned long long m = __ballot(lane < n && wanted(e));
        while (m) {
            const int l = __ffsll((long long)m) - 1;
            const Entry x = {lane_value(e.v, l), __builtin_amdgcn_readlane(e.i, l)};
            m &= m - 1;
            if (!wanted(x)) continue;
            const int at = __popcll(__ballot(lane < k && better(mine, x)));
            const Entry before = {__int_as_float(from_lane_before(__float_as_int(mine.v))), from_lane_before(mine.i)};
            mine = lane > at ? before : lane == at ? x : mine;
            raise(lane_value(mine.v, k - 1), __builtin_amdgcn_readlane(mine.i, k - 1));
        }
        n = 0;
        listed = true;
    }
    // One score a lane, in any order.
    __device__ __forceinline__ void offer(const Entry &e, bool there)
    {
        unsigned long long m = __ballot(there && wanted(e));
        if (!m) return;
        if (n + __popcll(m) > 64) {
            flush();
            m = __ballot(there && wanted(e));
        }
        if (m >> (threadIdx.x & 63) & 1) buffer[n + lanes_below(m)] = e;
        n += __popcll(m);
    }
    // Nothing more comes: at most 64 candidates in the buffer, those of the list included.
    __device__ __forceinline__ void settle()
    {
        if (listed) {
            flush();
            const unsigned long long m = __ballot((threadIdx.x & 63) < (unsigned)k && mine.i != kNone);
            if (m >> (threadIdx.x & 63) & 1) buffer[threadIdx.x & 63] = mine;
            n = __popcll(m);
        }
        wave_fence();
    }
    // Behind settle(): every candidate's rank among them; k and more, or the lane holds none: not among the best.
    __device__ __forceinline__ int ranked(Entry &e) const
    {
        const int lane = threadIdx.x & 63;
        e = lane < n ? buffer[lane] : Entry{-__builtin_inff(), kNone};
        int rank = lane < n ? 0 : 64;
#pragma nounroll
        for (int l = 0; l < n; ++l) {
            const Entry o = {lane_value(e.v, l), __builtin_amdgcn_readlane(e.i, l)};
            rank += better(o, e);
        }
        return rank;
    }
};

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
        for (int64_t c = lane; c < a.classes; c += 64) { // 64 beyond the last may pass 31 bits
            const int k = rank_key(score<DT>(a, base + c * a.class_stride));
            const bool behind = j == 0 || k < key || (k == key && c > index);
            if (behind && (k > bk || (k == bk && c < bi))) { bk = k; bi = (int)c; }
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

// What a position's label asks for, read before the scores are: two dependent loads, whose time would otherwise come on top.
struct Label {
    int64_t l;
    float x;
};
template <int DT>
__device__ __forceinline__ Label read_label(const cbinfer_log_probs_args &a, int64_t pos, int64_t base)
{
    Label r = {-1, 0.0f};
    if (!a.label) return r;
    r.l = a.label_bytes == 8 ? static_cast<const int64_t *>(a.labels)[pos] : static_cast<const int32_t *>(a.labels)[pos];
    if (r.l >= 0 && r.l < a.classes) r.x = score<DT>(a, base + r.l * a.class_stride);
    return r;
}

// Label and entropy of a position from its sums.
__device__ __forceinline__ void write_position(const cbinfer_log_probs_args &a, int64_t pos, const Label &label, const Sums &t, float log_s)
{
    if (a.entropy) a.entropy[pos] = t.s != t.s ? __builtin_nanf("") : t.s == 0.0f ? 0.0f : log_s - t.t / t.s;
    if (a.label)
        a.label[pos] = label.l < 0 ? 0.0f : label.l >= a.classes ? __builtin_nanf("") : log_prob(label.x, t, log_s);
}

// Sums of a wave, in every lane.
__device__ __forceinline__ void join_lanes(Sums &t)
{
    for (int off = 32; off; off >>= 1) join(t, {__shfl_xor(t.m, off), __shfl_xor(t.s, off), __shfl_xor(t.t, off)});
}

// Everything of a position from the sums and the list of the whole row, by one wave.
template <int DT>
__device__ void finish(const cbinfer_log_probs_args &a, int64_t pos, int64_t base, int64_t to, const Label &label, const Sums &t, Best &b)
{
    const int lane = threadIdx.x & 63;
    const float log_s = logf(t.s);
    if (lane == 0) write_position(a, pos, label, t, log_s);
    if (!a.top) return;
    if (t.s != t.s) {
        careful_top<DT>(a, base, to);
        return;
    }
    Entry e;
    const int rank = b.ranked(e);
    if (rank < a.top) {
        a.top_values[to + rank * a.inner] = log_prob(e.v, t, log_s);
        a.top_index[to + rank * a.inner] = e.i;
    }
}

// One wave a position, any strides, one class a lane at a time, one load of a wave under way: bound by their latency.  2048 rows of 4000
// bfloat16 classes, two apart (33 MB of lines): 7.6 us for the sums, 12.6 with 5 alternatives.
template <int DT>
__global__ __launch_bounds__(256) void wave_kernel(const cbinfer_log_probs_args a, int64_t first, FastDiv inner)
{
    const int lane = threadIdx.x & 63;
    const int64_t pos = first + (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (pos >= a.outer * a.inner) return;
    const int64_t o = fast_div((int)pos, inner), i = pos - o * a.inner;
    const int64_t base = o * a.outer_stride + i * a.inner_stride, to = o * a.top * a.inner + i;
    __shared__ Entry buffers[4][64];
    const Label label = read_label<DT>(a, pos, base);
    Sums t = {kLowest, 0.0f, 0.0f};
    Best b;
    b.begin(buffers[threadIdx.x >> 6], a.top);
    for (int64_t c0 = 0; c0 < a.classes; c0 += 64) {
        const int64_t c = c0 + lane;
        const bool there = c < a.classes;
        const float x = there ? score<DT>(a, base + c * a.class_stride) : -__builtin_inff();
        if (x > t.m) raise_to(t, x);
        add(t, x);
        if (a.top) b.offer({x, (int)c}, there);
    }
    if (a.top) b.settle();
    join_lanes(t);
    finish<DT>(a, pos, base, to, label, t, b);
}

// ---- classes behind one another ----------------------------------------------------------------
template <int DT>
struct Row {
    static constexpr int V = DT == kF32 ? 4 : 8; // scores in 16 bytes
    static __device__ __forceinline__ void unpack(const uint4 &u, float (&x)[V])
    {
#pragma unroll
        for (int e = 0; e < V; ++e) x[e] = Unit<DT>::get(u, e);
    }
};

// What a workgroup that shares a row leaves of it: the sums, then `top` entries, best first.
inline __host__ __device__ int segment_floats(int top) { return 3 + 2 * top; }

// `WAVES` waves of a workgroup take a row, or with several segments a row their part of it.  A wave loads 16 bytes a lane, U
// times over before it uses them; rows may begin at any address: the scores in front of the first 16-byte boundary and
// behind the last one are taken one by one.
// bfloat16 is bound by its instructions too: two loads ahead and eight waves a SIMD, 127 us for 2047 rows of 131071 and 8
// alternatives (537 MB), against 134 with four loads and five waves.  float32 takes four loads.
template <int DT, int WAVES, int U>
__global__ __launch_bounds__(WAVES < 4 ? 256 : WAVES * 64, DT == kBF16 ? 8 : 1) void rows_kernel(const cbinfer_log_probs_args a, int64_t first_row, FastDiv inner, int segments, float *found)
{
    typedef typename Elem<DT>::type T;
    constexpr int V = Row<DT>::V, ROWS = WAVES < 4 ? 4 / WAVES : 1, NT = WAVES * 64;
    __shared__ float shared[WAVES > 1 ? NT : 1];
    __shared__ Entry buffers[WAVES < 4 ? 4 : WAVES][64];
    __shared__ int counts[WAVES];
    const int lane = threadIdx.x & 63, wave = (threadIdx.x >> 6) % WAVES, thread = threadIdx.x % NT;
    const int64_t row = first_row + (int64_t)blockIdx.x * ROWS + (WAVES < 4 ? threadIdx.x / NT : 0);
    if (ROWS > 1 && row >= a.outer * a.inner) return; // a whole wave, and WAVES is 1 then
    const int segment = blockIdx.y;
    const int64_t o = fast_div((int)row, inner), in = row - o * a.inner, base = o * a.outer_stride + in * a.inner_stride;
    const T *x = static_cast<const T *>(a.scores) + base;
    const int n = (int)a.classes, k = a.top;
    const int head = min(n, (int)(-(reinterpret_cast<uintptr_t>(x) / sizeof(T)) & (V - 1))), units = (n - head) / V, tail = head + units * V;
    const int per = (units + segments - 1) / segments, end = min(units, (segment + 1) * per);
    const uint4 *body = reinterpret_cast<const uint4 *>(x + head);
    const Label label = segments == 1 ? read_label<DT>(a, row, base) : Label{-1, 0.0f};

    Sums t = {kLowest, 0.0f, 0.0f};
    Best b;
    b.begin(buffers[threadIdx.x >> 6], k);
    auto few = [&](int from, int to) { // fewer than 64, by the first wave
        if (from >= to || wave != 0) return;
        const bool there = lane < to - from; // their sum may pass 31 bits
        const float v = there ? Elem<DT>::get(x[from + lane]) : -__builtin_inff();
        if (v > t.m) raise_to(t, v);
        add(t, v);
        if (k) b.offer({v, from + lane}, there);
    };
    if (segment == 0) few(0, head);
    uint4 next[U];
    auto load = [&](int u0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int at = u0 + u * NT + thread;
            const unsigned none = DT == kF32 ? 0xff800000u : 0xff80ff80u; // -inf
            next[u] = make_uint4(none, none, none, none);
            if (at < end) next[u] = body[at];
        }
    };
    load(segment * per);
    int again = 0, round = 0;
#pragma nounroll
    for (int u0 = segment * per; u0 < end; u0 += U * NT, ++round) {
        uint4 raw[U];
        float largest[U], most;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            raw[u] = next[u];
            float v[V];
            Row<DT>::unpack(raw[u], v);
            largest[u] = v[0];
#pragma unroll
            for (int e = 1; e < V; ++e) largest[u] = fmaxf(largest[u], v[e]);
            most = u ? fmaxf(most, largest[u]) : largest[u];
        }
        load(u0 + U * NT);
        raise_to(t, fmaxf(t.m, most));
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[V];
            Row<DT>::unpack(raw[u], v);
#pragma unroll
            for (int e = 0; e < V; ++e) add(t, v[e]);
        }
        if (!k) continue;
        if (round == again) { // rounds 0, 1, 3, 7, ...: what a round wants in the mean falls with the scores that the bound has seen
            again = 2 * again + 1;
            float top = t.m == kLowest ? most : t.m; // the largest so far; of scores of -inf t.m says nothing
            if (WAVES > 1) {
                shared[threadIdx.x] = top;
                __syncthreads();
#pragma unroll
                for (int w = 0; w < WAVES; ++w) top = fmaxf(top, shared[w * 64 + lane]);
                __syncthreads();
            }
            b.bound(top);
        }
        const unsigned long long hit = __ballot(b.any_wanted(most));
        if (!hit) continue;
        if (__popcll(hit) > 32) b.bound(most); // scores that rise
        unsigned long long units[U], left = 0; // lanes whose unit may hold one
#pragma unroll
        for (int u = 0; u < U; ++u) {
            units[u] = __ballot(b.any_wanted(largest[u]) && u0 + u * NT + thread < end);
            left |= units[u];
        }
        while (left) { // a lane's unit, a score a lane; one place in the code for all of them
            unsigned long long m = units[U - 1];
            uint4 unit = raw[U - 1];
            int u = U - 1;
#pragma unroll
            for (int j = U - 2; j >= 0; --j)
                if (units[j]) {
                    m = units[j];
                    unit = raw[j];
                    u = j;
                }
            const int l = __ffsll((long long)m) - 1;
            m &= m - 1;
            left = 0;
#pragma unroll
            for (int j = 0; j < U; ++j) {
                if (j == u) units[j] = m;
                left |= units[j];
            }
            unit.x = __builtin_amdgcn_readlane(unit.x, l);
            unit.y = __builtin_amdgcn_readlane(unit.y, l);
            unit.z = __builtin_amdgcn_readlane(unit.z, l);
            unit.w = __builtin_amdgcn_readlane(unit.w, l);
            const int word = lane / (V / 4);
            const unsigned w = word == 0 ? unit.x : word == 1 ? unit.y : word == 2 ? unit.z : unit.w;
            const float x = __uint_as_float(DT == kF32 ? w : lane & 1 ? w & 0xffff0000u : w << 16);
            b.offer({x, head + (u0 + u * NT + thread - lane + l) * V + lane}, lane < V);
        }
    }
    if (segment == segments - 1) few(tail, n);
    if (k) b.settle();
    join_lanes(t);
    if (WAVES > 1) {
        if (lane == 0) {
            shared[wave * 3] = t.m; shared[wave * 3 + 1] = t.s; shared[wave * 3 + 2] = t.t;
            counts[wave] = b.n;
        }
        __syncthreads();
        if (wave != 0) return;
        t = {kLowest, 0.0f, 0.0f};
        if (lane < WAVES) t = {shared[lane * 3], shared[lane * 3 + 1], shared[lane * 3 + 2]};
        join_lanes(t);
        if (k) { // the first wave's buffer is read before it is used again
            Entry e[WAVES];
            float most = -__builtin_inff();
            int all = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                e[w] = lane < counts[w] ? buffers[w][lane] : Entry{-__builtin_inff(), kNone};
                most = fmaxf(most, e[w].v);
                all += counts[w];
            }
            wave_fence();
            const float least = b.least;
            b.begin(buffers[0], k);
            b.raise(least, kNone);
            if (all > 2 * k) b.bound(most);
#pragma nounroll
            for (int w = 0; w < WAVES; ++w) {
                b.offer(e[0], lane < counts[w]);
#pragma unroll
                for (int j = 0; j + 1 < WAVES; ++j) e[j] = e[j + 1];
            }
            b.settle();
        }
    }
    if (segments == 1) {
        finish<DT>(a, row, base, o * a.top * a.inner + in, label, t, b);
    } else {
        float *mine = found + (row * segments + segment) * segment_floats(k);
        if (lane == 0) { mine[0] = t.m; mine[1] = t.s; mine[2] = t.t; }
        if (k) {
            Entry e;
            const int rank = b.ranked(e);
            if (rank < k) { mine[3 + rank] = e.v; mine[3 + k + rank] = __int_as_float(e.i); }
            if (lane >= b.n && lane < k) { mine[3 + lane] = -__builtin_inff(); mine[3 + k + lane] = __int_as_float(kNone); }
        }
    }
}

// The segments of a row, a wave a row: a chain of dependent steps on a few kilobytes, 5 us for 64 rows in 13 segments.
template <int DT>
__global__ __launch_bounds__(256) void join_kernel(const cbinfer_log_probs_args a, int64_t first, FastDiv inner, int segments, const float *found)
{
    __shared__ Entry buffers[4][64];
    const int lane = threadIdx.x & 63, k = a.top, each = segment_floats(k);
    const int64_t row = first + (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= a.outer * a.inner) return;
    const int64_t o = fast_div((int)row, inner), in = row - o * a.inner;
    found += row * segments * each;
    const int64_t base = o * a.outer_stride + in * a.inner_stride;
    const Label label = read_label<DT>(a, row, base);
    Sums t = {kLowest, 0.0f, 0.0f};
    float best = -__builtin_inff(), least = best; // of a segment: below the least of k a score has k better ones, ...
    if (lane < segments) {
        t = {found[lane * each], found[lane * each + 1], found[lane * each + 2]};
        if (k) {
            best = found[lane * each + 3];
            least = found[lane * each + 3 + k - 1];
        }
    }
    join_lanes(t);
    Best b;
    b.begin(buffers[threadIdx.x >> 6], k);
    if (k) {
        for (int off = 32; off; off >>= 1) least = fmaxf(least, __shfl_xor(least, off));
        b.raise(least, kNone);
        if (segments >= k) b.bound(best); // ... and below the k-th largest of the segments' best too
        for (int at = lane; at - lane < segments * k; at += 64) {
            const bool there = at < segments * k;
            const int list = there ? at / k : 0, j = there ? at - list * k : 0;
            b.offer({found[list * each + 3 + j], __float_as_int(found[list * each + 3 + k + j])}, there);
        }
        b.settle();
    }
    finish<DT>(a, row, base, o * a.top * a.inner + in, label, t, b);
}

// ---- positions behind one another: maps ------------------------------------------------------------
// A lane takes a position and keeps its K best in registers, best first.  A score and its class are one key, so that the
// larger and the smaller of two are one instruction each: CH classes are put in order by a network of such pairs, and joined with
// the K so far by another.  Lanes differ in which scores are wanted, so nothing would be gained by asking.
// bfloat16: 32 bits, 16 of the score and 16 of the class.  float32: 64 bits, 32 of the score and 31 of the class, as a
// positive double: whatever a number's bits are, its exponent is not that of infinity, NaN or a denormal.
template <int DT>
struct Key;
template <>
struct Key<kBF16> {
    unsigned k;
    static __device__ __forceinline__ Key none() { return {0u}; }
    static __device__ __forceinline__ Key of(float x, int c)
    {
        const unsigned b = __float_as_uint(x + 0.0f); // -0 is 0
        return {((b ^ ((unsigned)((int)b >> 31) | 0x80000000u)) & 0xffff0000u) | (0xffffu - (unsigned)c)};
    }
    __device__ __forceinline__ int index() const { return (int)(0xffffu - (k & 0xffffu)); }
    __device__ __forceinline__ float value() const { return __uint_as_float((k & 0x80000000u ? k ^ 0x80000000u : ~k) & 0xffff0000u); }
    static __device__ __forceinline__ Key larger(Key a, Key b) { return {max(a.k, b.k)}; }
    static __device__ __forceinline__ Key smaller(Key a, Key b) { return {min(a.k, b.k)}; }
    static constexpr int kClasses = 1 << 16;
};
template <>
struct Key<kF32> {
    double k;
    static __device__ __forceinline__ Key none() { return {0.0}; }
    static __device__ __forceinline__ Key of(float x, int c)
    {
        const unsigned b = __float_as_uint(x + 0.0f), u = b ^ ((unsigned)((int)b >> 31) | 0x80000000u);
        return {__hiloint2double((int)(u >> 1), (int)(u << 31 | (0x7fffffffu - (unsigned)c)))};
    }
    __device__ __forceinline__ int index() const { return (int)(0x7fffffffu - ((unsigned)__double2loint(k) & 0x7fffffffu)); }
    __device__ __forceinline__ float value() const
    {
        const unsigned u = (unsigned)__double2hiint(k) << 1 | (unsigned)__double2loint(k) >> 31;
        return of_key((int)(u ^ 0x80000000u));
    }
    // fmax and fmin would first make quiet NaNs of signalling ones; there are none
    static __device__ __forceinline__ Key larger(Key a, Key b)
    {
        double r;
        asm("v_max_f64 %0, %1, %2" : "=v"(r) : "v"(a.k), "v"(b.k));
        return {r};
    }
    static __device__ __forceinline__ Key smaller(Key a, Key b)
    {
        double r;
        asm("v_min_f64 %0, %1, %2" : "=v"(r) : "v"(a.k), "v"(b.k));
        return {r};
    }
};

template <typename T>
__device__ __forceinline__ void order(T &a, T &b)
{
    const T x = T::larger(a, b);
    b = T::smaller(a, b);
    a = x;
}

// Largest first.  A sequence that rises and falls (or the other way) is put in order by log2 N rounds of pairs.
template <int N, typename T>
__device__ __forceinline__ void order_bitonic(T (&x)[N])
{
#pragma unroll
    for (int d = N / 2; d; d /= 2)
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (!(i & d)) order(x[i], x[i + d]);
}
template <int N, typename T>
__device__ __forceinline__ void order_all(T (&x)[N])
{
#pragma unroll
    for (int n = 2; n <= N; n *= 2) {
#pragma unroll
        for (int i = 0; i < N; i += n) // two ordered halves: the first against the second turned round
#pragma unroll
            for (int j = 0; j < n / 2; ++j) order(x[i + j], x[i + n - 1 - j]);
#pragma unroll
        for (int d = n / 4; d; d /= 2)
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (!(i & d)) order(x[i], x[i + d]);
    }
}
// The N largest of both, in order.
template <int N, typename T>
__device__ __forceinline__ void order_join(T (&x)[N], const T (&y)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = T::larger(x[i], y[N - 1 - i]);
    order_bitonic(x);
}

// careful_top for a lane by itself.
template <int DT>
__device__ void careful_top_lane(const cbinfer_log_probs_args &a, int64_t base, int64_t to)
{
    int key = kNone, index = -1;
    for (int j = 0; j < a.top; ++j) {
        int bk = -kNone - 1, bi = kNone;
        for (int c = 0; c < (int)a.classes; ++c) {
            const int k = rank_key(score<DT>(a, base + c * a.class_stride));
            const bool behind = j == 0 || k < key || (k == key && c > index);
            if (behind && k > bk) { bk = k; bi = c; }
        }
        key = bk;
        index = bi;
        a.top_values[to + j * a.inner] = __builtin_nanf("");
        a.top_index[to + j * a.inner] = bi;
    }
}

// PARTS > 1: the waves of a workgroup share the classes of 256 / PARTS positions, for maps that would not fill the chip
// otherwise.  CH classes are loaded while those before are worked on.  Bound by memory without alternatives or with few (64 x 8 x 180 x
// 320 float32, 3 alternatives: 221 MB in 40 us), by the network's instructions with more (10 x 256 x 180 x 320, 590 MB of float32: 110 us
// without, 127 with 8; bfloat16 64 and 100).  Where a class lies is the same for every lane, where a position lies does not change: an
// address costs no vector instruction (with 64 bits a lane and a bounds check for each: 119, 143, 80 and 132).
template <int DT, int K, int PARTS>
__global__ __launch_bounds__(256) void map_kernel(const cbinfer_log_probs_args a, FastDiv inner)
{
    typedef typename Elem<DT>::type T;
    typedef Key<DT> Ranked;
    constexpr int KK = K ? K : 1, CH = K > 8 ? K : 8, NP = 256 / PARTS;
    __shared__ float sums[PARTS > 1 ? PARTS - 1 : 1][3][PARTS > 1 ? NP : 1];
    __shared__ Ranked lists[PARTS > 1 ? PARTS - 1 : 1][KK][PARTS > 1 ? NP : 1];
    const int part = threadIdx.x / NP, place = threadIdx.x % NP;
    const int64_t pos = (int64_t)blockIdx.x * NP + place;
    const bool there = pos < a.outer * a.inner;
    const int64_t mine = there ? pos : a.outer * a.inner - 1; // the others read what the last position reads
    const int o = fast_div((int)mine, inner);
    const int64_t i = mine - (int64_t)o * a.inner, base = o * a.outer_stride + i * a.inner_stride;
    const Label label = there && part == 0 ? read_label<DT>(a, pos, base) : Label{-1, 0.0f};
    // Whole rounds of CH: what a round has beyond `end` is a score of -inf at the next classes' numbers, which must not be those of another part
    const int n = (int)a.classes, each = PARTS == 1 ? n : ((n + PARTS - 1) / PARTS + CH - 1) / CH * CH, end = min(n, (part + 1) * each);
    const int64_t first = (int64_t)blockIdx.x * NP;
    const int o0 = fast_div((int)first, inner);
    const int64_t base0 = o0 * a.outer_stride + (first - (int64_t)o0 * a.inner) * a.inner_stride; // of the workgroup's first position
    const unsigned offset = (unsigned)(base - base0) * (unsigned)sizeof(T); // positions ascend, see run()
    const int start = __builtin_amdgcn_readfirstlane(part * each);
    const T *x = static_cast<const T *>(a.scores) + base0 + (int64_t)start * a.class_stride;
    Sums t = {kLowest, 0.0f, 0.0f};
    Ranked best[KK];
#pragma unroll
    for (int j = 0; j < KK; ++j) best[j] = Ranked::none();
    const int last_class = __builtin_amdgcn_readfirstlane(end);
    T next[CH];
    const T none = Elem<DT>::put(-__builtin_inff());
    auto load = [&](int c0) {
#pragma unroll
        for (int e = 0; e < CH; ++e) {
            // beyond the last class the last again, also where a part has none
            const T *y = x + min(e, last_class - 1 - c0) * a.class_stride;
            next[e] = *reinterpret_cast<const T *>(reinterpret_cast<const char *>(y) + offset);
        }
        x += CH * a.class_stride;
        if (c0 + CH > last_class)
#pragma unroll
            for (int e = 0; e < CH; ++e)
                if (c0 + e >= last_class) next[e] = none;
    };
    load(start);
    for (int c0 = start; c0 < last_class; c0 += CH) {
        float v[CH], most = kLowest;
#pragma unroll
        for (int e = 0; e < CH; ++e) {
            v[e] = Elem<DT>::get(next[e]);
            most = fmaxf(most, v[e]);
        }
        if (c0 + CH < last_class) load(c0 + CH);
        raise_to(t, fmaxf(t.m, most));
#pragma unroll
        for (int e = 0; e < CH; ++e) add(t, v[e]);
        if constexpr (K == 1) {
#pragma unroll
            for (int e = 0; e < CH; ++e) best[0] = Ranked::larger(best[0], Ranked::of(v[e], c0 + e));
        } else if constexpr (K > 1) {
#pragma unroll
            for (int g = 0; g < CH; g += KK) {
                Ranked y[KK];
#pragma unroll
                for (int j = 0; j < KK; ++j) y[j] = Ranked::of(v[g + j], c0 + g + j);
                order_all(y);
                order_join(best, y);
            }
        }
    }
    if (PARTS > 1) {
        if (part) {
            sums[part - 1][0][place] = t.m; sums[part - 1][1][place] = t.s; sums[part - 1][2][place] = t.t;
#pragma unroll
            for (int j = 0; j < K; ++j) lists[part - 1][j][place] = best[j];
        }
        __syncthreads();
        if (part) return;
        for (int p = 0; p + 1 < PARTS; ++p) {
            join(t, {sums[p][0][place], sums[p][1][place], sums[p][2][place]});
            if constexpr (K > 0) {
                Ranked y[KK];
#pragma unroll
                for (int j = 0; j < KK; ++j) y[j] = lists[p][j][place];
                order_join(best, y);
            }
        }
    }
    if (!there) return;
    const float log_s = logf(t.s);
    write_position(a, pos, label, t, log_s);
    if (!K) return;
    const int64_t to = (int64_t)o * a.top * a.inner + i;
    if (t.s != t.s) {
        careful_top_lane<DT>(a, base, to);
        return;
    }
#pragma unroll
    for (int j = 0; j < K; ++j)
        if (j < a.top) {
            a.top_values[to + j * a.inner] = log_prob(best[j].value(), t, log_s);
            a.top_index[to + j * a.inner] = best[j].index();
        }
}

template <int DT, int PARTS>
hipError_t map_any(hipStream_t st, const cbinfer_log_probs_args &a)
{
    const unsigned grid = (unsigned)((a.outer * a.inner + 256 / PARTS - 1) / (256 / PARTS));
    const FastDiv inner = make_fastdiv((int)a.inner);
    auto kernel = a.top == 0 ? map_kernel<DT, 0, PARTS> : a.top == 1 ? map_kernel<DT, 1, PARTS> : a.top <= 4 ? map_kernel<DT, 4, PARTS> :
                  a.top <= 8 ? map_kernel<DT, 8, PARTS> : map_kernel<DT, 16, PARTS>;
    kernel<<<grid, 256, 0, st>>>(a, inner);
    return hipGetLastError();
}

} // namespace
namespace {
enum { kAnyStride, kRows, kMaps };
struct Plan {
    int kind, waves, segments;
};

Plan plan(const cbinfer_log_probs_args &a)
{
    Plan p = {kAnyStride, 1, 1};
    const int64_t positions = a.outer * a.inner;
    if (a.class_stride == 1) {
        p.kind = kRows;
        // us a call with 5 alternatives, a wave each and four waves each.  4096 rows bfloat16: 1000 classes 12.6, 20.7, 2048 17.1, 20.1, 4000 24.6,
        // 19.9; float32 11.7, 22.6, 18.2, 22.4, 26.7, 22.9.  512 rows of 2048 bfloat16 11.1, 10.8, of 4000 16.4, 11.4.
        if (a.classes <= 2048) return p;
        p.waves = 4;
        // Few long rows are cut into segments of one or two rounds of loads, up to 1024 workgroups, and joined by a second launch.
        // 64 rows of 100003 bfloat16: 29 us whole, 18 in segments, join included; one of 131071: 28 and 14.
        const int64_t round = 4 * 64 * 4 * (a.dtype == kF32 ? 4 : 8), segments = std::min<int64_t>({(a.classes + round - 1) / round, 64, 1024 / std::max<int64_t>(positions, 1)});
        if (segments >= 4) p.segments = (int)segments;
    } else if (a.classes <= 1 << 30 && a.inner_stride == 1 && a.inner >= 16 && (a.outer == 1 || a.outer_stride >= a.inner) && a.top <= 16 && (a.classes <= 1024 || positions >= 16384) &&
               (a.dtype == kF32 || a.classes <= Key<kBF16>::kClasses)) {
        // A lane a position or a wave each, us with 3 alternatives: 2000 maps of 64 classes and 16 positions 10.8, 46, of 8 (taken by waves) 10.6, 26;
        // float32 the same.  Many classes need as many positions: 4 x 2000 classes x 256 positions bfloat16 38, 25, 4 x 2000 x 1024 39, 39, 16 x 2000 x
        // 1024 39, 130; 4 x 1024 x 256 20, 16, 4 x 1024 x 1024 21, 23.
        p.kind = kMaps; // counts classes in whole rounds and parts, in 32 bits
        // 5 x 191 x 148 x 269 bfloat16, 3 alternatives: a wave each 34 us, four waves 29; float32 without: 29.5, 34
        p.waves = positions < (a.top ? 262144 : 65536) && a.classes >= 32 ? 4 : 1;
    }
    return p;
}

constexpr int64_t kMostBlocks = 1 << 20; // of a launch: threads are counted in 32 bits

template <int DT>
hipError_t run(hipStream_t st, const cbinfer_log_probs_args &a)
{
    const Plan p = plan(a);
    const int64_t positions = a.outer * a.inner;
    if (p.kind == kMaps) {
        const auto maps = [&](const cbinfer_log_probs_args &b) { return p.waves == 4 ? map_any<DT, 4>(st, b) : map_any<DT, 1>(st, b); };
        // offsets from a workgroup's first position have 32 bits
        const int64_t e = sizeof(typename Elem<DT>::type);
        if (a.outer == 1 || a.outer_stride < (((int64_t)1 << 32) / e - 256) / (255 / a.inner + 2)) return maps(a);
        for (int64_t o = 0; o < a.outer; ++o) { // maps of gigabytes, one at a time
            cbinfer_log_probs_args b = a;
            b.outer = 1;
            b.scores = static_cast<const typename Elem<DT>::type *>(a.scores) + o * a.outer_stride;
            if (a.labels) b.labels = static_cast<const char *>(a.labels) + o * a.inner * a.label_bytes;
            if (a.label) b.label = a.label + o * a.inner;
            if (a.entropy) b.entropy = a.entropy + o * a.inner;
            if (a.top_values) b.top_values = a.top_values + o * a.top * a.inner;
            if (a.top_index) b.top_index = a.top_index + o * a.top * a.inner;
            if (hipError_t err = maps(b)) return err;
        }
        return hipSuccess;
    }
    constexpr int U = DT == kF32 ? 4 : 2;
    float *found = static_cast<float *>(a.workspace);
    const FastDiv inner = make_fastdiv((int)a.inner);
    const int per_block = p.kind == kRows && p.waves > 1 ? 1 : 4;
    for (int64_t first = 0; first < positions; first += kMostBlocks * per_block) {
        const unsigned blocks = (unsigned)std::min(kMostBlocks, (positions - first + per_block - 1) / per_block);
        const dim3 grid(blocks, p.segments);
        if (p.kind != kRows)
            wave_kernel<DT><<<blocks, 256, 0, st>>>(a, first, inner);
        else if (p.waves == 1)
            rows_kernel<DT, 1, U><<<grid, 256, 0, st>>>(a, first, inner, p.segments, found);
        else
            rows_kernel<DT, 4, U><<<grid, 256, 0, st>>>(a, first, inner, p.segments, found);
        if (hipError_t e = hipGetLastError()) return e;
    }
    if (p.segments > 1) {
        join_kernel<DT><<<(unsigned)((positions + 3) / 4), 256, 0, st>>>(a, 0, inner, p.segments, found);
        return hipGetLastError();
    }
    return hipSuccess;
}
} // namespace

size_t log_probs_workspace(const cbinfer_log_probs_args &a)
{
    const Plan p = plan(a);
    return p.segments > 1 ? (size_t)(a.outer * a.inner) * p.segments * segment_floats(a.top) * sizeof(float) : 0;
}

hipError_t log_probs(hipStream_t st, const cbinfer_log_probs_args &a) { return a.dtype == kF32 ? run<kF32>(st, a) : run<kBF16>(st, a); }

} // namespace cbk
