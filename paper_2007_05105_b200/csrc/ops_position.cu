// Attention weights with a learned bias by relative position, and their gradient.
//
//   p = softmax over the live keys of  scale s + table[bucket(j - pos_i), h]
//   g = p (dp - sum p dp),   ds = scale g,   dtable[k, h] = sum of g over bucket k
//
// One pass over the data: a group of threads (8 lanes, a warp, or a block, by the length of a row) holds a row in registers
// between the maximum, the sum and the result.  Bound by memory.  Keys that are not live are not read, but for those that share 16
// bytes with the last live one.
//
// The bias is never in memory: a block works on one head and keeps that head's bias by distance in shared memory, up to
// max_distance, where it stops changing; beyond, a register has it.  A thread's 4 or 8 adjacent keys want as many adjacent
// entries, which begin anywhere: four copies, each shifted by one entry, let 16-byte reads fetch them (single reads: four lanes a
// bank).  Above kCopiesMax the copies would not fit, and the bucket of each distance is looked up.
//
// The gradient of the table is summed without atomics: every lane has a column of its own in shared memory (bank = lane), one
// entry a bucket; keys further than max_distance, most of them, are summed in two registers.  A thread's adjacent keys are in one
// bucket if the first and the last of them are, since buckets are monotone on either side.  Blocks leave their sums, a
// second kernel adds them up in order.
//
// Measured on a B200: weights of 32 x 8 x 512 x 512 float32, ragged, 88 us (5.3 TB/s of the bytes that it cannot do without), of
// 8 x 16 x 1024 x 1024 bf16, causal, 92 us, its gradient 104 (5.1 TB/s); each writes 268 MB, which alone take 70 us at the rate of a plain
// write.
//
// While a row is worked on, the group's next one is on its way into shared memory, each thread's part to a place of its own.
//
// Rows may start anywhere (then without that): accesses are cut at 16-byte boundaries of memory; what one brings of the next row is not used,
// and the ragged ends of a row are stored in pieces.  Short ones have kernels of their own.
#include "ops_common.cuh"

#include <algorithm>
#include <utility>

namespace {

constexpr int kBordersMax = ADASCALE_POSITION_MAX_BUCKETS / 2;
constexpr long long kMaxLen = 1LL << 29, kMaxStart = 1LL << 30;  // distances stay 32-bit numbers
constexpr int kBlocksMax = 2048;   // of all heads, roughly; the gradient's partial sums are that many times the buckets
constexpr int kCopiesMax = 1024;   // max_distance up to which the bias is kept by distance (33 KB)
constexpr float kLog2e = 1.4426950408889634f;

// Buckets of a side: n < exact by itself, then one more for every border that is not above n.
struct Buckets {
    int n, m, exact, max_distance, both;
    int n_borders;
    short border[kBordersMax];
};

struct Strides {
    long long b, h, q;
};

struct PositionArgs {
    const void *s, *dp;  // scores; or the weights and what arrives at them
    void *out;           // weights; or the scores' gradient
    const float *table;
    float *partials;
    const void *lengths, *starts;
    Strides s_at, dp_at, out_at;
    long long s_span, dp_span;  // elements from the first one to behind the last
    long long rows;      // batch * n_queries
    long long ld_table;
    int n_queries, n_keys, chunks;
    int wide_lengths, wide_starts, causal;
    float scale;
    Buckets buckets;
};

__device__ __forceinline__ int bucket_of(const Buckets &b, int d)
{
    int n = d < 0 ? -d : (b.both ? d : 0);
    int k = n;
    if (n >= b.exact) {
        int lo = 0, hi = b.n_borders;  // the number of borders that are not above n
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (b.border[mid] <= n) lo = mid + 1;
            else hi = mid;
        }
        k = b.exact + lo;
    }
    return k + (b.both && d > 0 ? b.m : 0);
}

// ---- rows ----------------------------------------------------------------------------------

// A row's batch and query; the position of its query, and how many keys are live.
struct Row {
    int b, i, pos, live;
    int n;         // keys of the row: 0 behind the last
    long long at;  // where it begins in the first matrix
};
__device__ __forceinline__ void look_up(const PositionArgs &a, Row &w)
{
    w.pos = w.i;
    if (a.starts) {
        const long long start = load_id(a.starts, a.wide_starts, w.b);
        w.pos += (int)(start < -kMaxStart ? -kMaxStart : start > kMaxStart ? kMaxStart : start);
    }
    w.live = a.n_keys;
    if (a.lengths) {
        const long long n = load_id(a.lengths, a.wide_lengths, w.b);
        w.live = n < 0 ? 0 : n < w.live ? (int)n : w.live;
    }
    if (a.causal) w.live = min(w.live, max(w.pos + 1, 0));
}
__device__ __forceinline__ long long offset_of(const Strides &at, const Row &w, int head) { return w.b * at.b + head * at.h + w.i * at.q; }

// Walks over every chunks * kGroups-th row of all: neighbours, which have as many live keys, go to different blocks.
template <int kGroups> struct Walk {
    unsigned r, step;
    int step_b, step_i;
    long long step_at, wrap_at;  // of the offset in the first matrix
    Row w;
    __device__ __forceinline__ Walk(const PositionArgs &a, int head, int chunk, int group)
    {
        const unsigned n = (unsigned)a.n_queries;
        step = (unsigned)(a.chunks * kGroups);
        r = (unsigned)(chunk * kGroups + group);
        step_b = (int)(step / n);
        step_i = (int)(step % n);
        w.b = (int)(r / n);
        w.i = (int)(r % n);
        w.at = offset_of(a.s_at, w, head);
        step_at = step_b * a.s_at.b + step_i * a.s_at.q;
        wrap_at = a.s_at.b - n * a.s_at.q;
    }
    // The row where it stands.
    __device__ __forceinline__ Row here(const PositionArgs &a) const
    {
        Row x = w;
        x.n = x.pos = x.live = 0;
        if (r < (unsigned)a.rows) {
            x.n = a.n_keys;
            look_up(a, x);
        }
        return x;
    }
    __device__ __forceinline__ void next(const PositionArgs &a)
    {
        r += step;  // below 2^31 + 2^17
        w.b += step_b;
        w.i += step_i;
        w.at += step_at;
        if (w.i >= a.n_queries) {
            w.i -= a.n_queries;
            ++w.b;
            w.at += wrap_at;
        }
    }
};

// Whether the next row is requested while one is worked on: bf16 rows have twice the arithmetic a byte, and the warps that fit do not cover
// the wait for memory (gradient of 8 x 16 x 1024 x 1024, causal: 126 us without, 114 with; float32 of 32 x 8 x 512 x 512: 127 and 150).
template <typename T, bool LONG, bool EVEN> constexpr bool kRowsAhead = sizeof(T) == 2 && EVEN && !LONG;

// Elements by which an address lies behind a 16-byte boundary.
template <typename T> __device__ __forceinline__ int off16(const T *p) { return (int)((uintptr_t)p % 16 / sizeof(T)); }

// How 16 bytes of a row are read that reach over its ends: whole where they are on a boundary and, `inside`, the matrix goes on around the
// row (what they bring of it is not used; one by one, the ends' elements are a wait for memory of their own: bf16 rows of 500, gradient, 135 us, 105);
// element by element where it does not.
struct Reach {
    bool aligned, inside;
};
template <typename T> __device__ __forceinline__ Reach reach_of(const T *row, int off, long long at, int n, long long span)
{
    constexpr int V = 16 / sizeof(T);
    return {off16(row) == off, at >= V && at + n + V <= span};
}
// 16 bytes: elements c .. c + V - 1 of a row of n, of which one at least is the row's; what lies outside is 0 or anything.  EVEN: rows begin
// on and end at 16-byte boundaries, and all matrices have the same strides.
template <bool EVEN, typename T> __device__ __forceinline__ uint4 load_raw(const T *row, int c, int n, Reach reach)
{
    constexpr int V = 16 / sizeof(T);
    if (EVEN || (reach.aligned && (reach.inside || (c >= 0 && c + V <= n)))) return *reinterpret_cast<const uint4 *>(row + c);
    union {
        uint4 raw;
        T x[V];
    } u;
    u.raw = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int e = 0; e < V; ++e)
        if (c + e >= 0 && c + e < n) u.x[e] = row[c + e];
    return u.raw;
}
// Zeros for the elements outside [0, live).
template <bool EVEN, typename T> __device__ __forceinline__ void keep_live(uint4 &raw, int c, int live)
{
    constexpr int V = 16 / sizeof(T);
    if ((EVEN || c >= 0) && c + V <= live) return;
    unsigned *x = reinterpret_cast<unsigned *>(&raw);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            if (c + i < 0 || c + i >= live) x[i] = 0u;
        } else {
            if (c + 2 * i < 0 || c + 2 * i >= live) x[i] &= 0xffff0000u;
            if (c + 2 * i + 1 < 0 || c + 2 * i + 1 >= live) x[i] &= 0xffffu;
        }
    }
}
// Its elements, two and two.
__device__ __forceinline__ void spread(const uint4 &r, f2 (&x)[2], float)
{
    x[0] = pack2(__uint_as_float(r.x), __uint_as_float(r.y));
    x[1] = pack2(__uint_as_float(r.z), __uint_as_float(r.w));
}
__device__ __forceinline__ void spread(const uint4 &r, f2 (&x)[4], bf16)
{
    x[0] = pack2(bf_lo(r.x), bf_hi(r.x));
    x[1] = pack2(bf_lo(r.y), bf_hi(r.y));
    x[2] = pack2(bf_lo(r.z), bf_hi(r.z));
    x[3] = pack2(bf_lo(r.w), bf_hi(r.w));
}
template <int P> __device__ __forceinline__ void flat(const f2 (&x)[P], float (&y)[2 * P])
{
#pragma unroll
    for (int i = 0; i < P; ++i) unpack2(x[i], y[2 * i], y[2 * i + 1]);
}
// Elements outside [0, live) become `other`.
template <bool EVEN, int P> __device__ __forceinline__ void keep_live(f2 (&x)[P], int c, int live, float other)
{
    if ((EVEN || c >= 0) && c + 2 * P <= live) return;
#pragma unroll
    for (int i = 0; i < P; ++i) {
        float lo, hi;
        unpack2(x[i], lo, hi);
        lo = (EVEN || c + 2 * i >= 0) && c + 2 * i < live ? lo : other;
        hi = (EVEN || c + 2 * i + 1 >= 0) && c + 2 * i + 1 < live ? hi : other;
        x[i] = pack2(lo, hi);
    }
}
// Elements lo .. hi - 1 of 16 bytes on a boundary, where lo is 0 or hi is V.
__device__ __forceinline__ void store_end(float *p, int lo, int hi, const float (&x)[4])
{
    if (lo == 0) {
        if (hi & 2) *reinterpret_cast<float2 *>(p) = make_float2(x[0], x[1]);
        if (hi & 1) p[hi - 1] = hi & 2 ? x[2] : x[0];
    } else {
        const int k = 4 - lo;
        if (k & 2) *reinterpret_cast<float2 *>(p + 2) = make_float2(x[2], x[3]);
        if (k & 1) p[lo] = k & 2 ? x[1] : x[3];
    }
}
__device__ __forceinline__ void store_end(bf16 *p, int lo, int hi, const float (&x)[8])
{
    unsigned *q = reinterpret_cast<unsigned *>(p);
    const unsigned a = bf_pack(x[0], x[1]), b = bf_pack(x[2], x[3]), c = bf_pack(x[4], x[5]), d = bf_pack(x[6], x[7]);
    unsigned short *h = reinterpret_cast<unsigned short *>(p);
    if (lo == 0) {
        if (hi & 4) *reinterpret_cast<uint2 *>(q) = make_uint2(a, b);
        if (hi & 2) q[hi & 4 ? 2 : 0] = hi & 4 ? c : a;
        if (hi & 1) h[hi - 1] = (unsigned short)(hi & 4 ? (hi & 2 ? d : c) : (hi & 2 ? b : a));
    } else {
        const int k = 8 - lo;
        if (k & 4) *reinterpret_cast<uint2 *>(q + 2) = make_uint2(c, d);
        if (k & 2) q[k & 4 ? 1 : 3] = k & 4 ? b : d;
        if (k & 1) h[lo] = (unsigned short)((k & 4 ? (k & 2 ? a : b) : (k & 2 ? c : d)) >> 16);
    }
}
template <bool EVEN, typename T, int P> __device__ __forceinline__ void store_cols(T *row, int c, int n, bool aligned, const f2 (&x)[P])
{
    float y[2 * P];
    flat(x, y);
    if (EVEN || (aligned && c >= 0 && c + 2 * P <= n)) {
        store_vec_streaming<2 * P>(row + c, y);
    } else if (aligned && (c >= 0 || c + 2 * P <= n)) {  // one end: elements from `lo` on or up to `hi`, in pieces of powers of two
        store_end(row + c, c < 0 ? -c : 0, c < 0 ? 2 * P : n - c, y);
    } else {
#pragma unroll
        for (int e = 0; e < 2 * P; ++e)
            if (c + e >= 0 && c + e < n) put(row + c + e, y[e]);
    }
}

// Sum or maximum over the GS threads of a group, the same in each of them.  `scratch` is another one for each of two joins that
// follow each other, so that one barrier a join is enough.
template <int GS, bool MAX> __device__ __forceinline__ float group_join(float v, float (*scratch)[32])
{
    constexpr int kLanes = GS < 32 ? GS : 32;
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1) {
        const float w = __shfl_xor_sync(0xffffffffu, v, o);
        v = MAX ? fmaxf(v, w) : v + w;
    }
    if constexpr (GS > 32) {
        constexpr int kWarps = GS / 32;
        float *mine = *scratch + threadIdx.x / GS * kWarps;
        if (threadIdx.x % 32 == 0) mine[threadIdx.x % GS / 32] = v;
        asm volatile("bar.sync %0, %1;" ::"r"((int)threadIdx.x / GS + 1), "n"(GS) : "memory");
        v = mine[threadIdx.x % kWarps];
#pragma unroll
        for (int o = kWarps / 2; o > 0; o >>= 1) {
            const float w = __shfl_xor_sync(0xffffffffu, v, o);
            v = MAX ? fmaxf(v, w) : v + w;
        }
    }
    return v;
}

// ---- weights -------------------------------------------------------------------------------

// The head's bias.  By distance: entry d of copy k at [k][d + reach + k], reach being max_distance and the 8 keys of an access more,
// in rows of `pitch`.  Otherwise: the buckets of all distances, and the bias of each bucket behind them.
struct Bias {
    const float *by_distance;
    const unsigned char *bucket;
    int max_distance, reach, pitch;
    float behind, ahead;  // of distances beyond it
};
__host__ __device__ inline int bias_reach(int max_distance) { return max_distance + 8; }
__host__ __device__ inline int bias_pitch(int max_distance) { return (2 * bias_reach(max_distance) + 1 + 8 + 3) / 4 * 4; }
__host__ __device__ inline int bucket_bytes(int max_distance) { return (2 * max_distance + 1 + 15) / 16 * 16; }
__host__ __device__ inline size_t bias_bytes(int max_distance, int n_buckets)
{
    return max_distance <= kCopiesMax ? 16 * (size_t)bias_pitch(max_distance) : bucket_bytes(max_distance) + 16 * (size_t)((n_buckets + 3) / 4);
}

__device__ __forceinline__ Bias make_bias(const PositionArgs &a, int head, unsigned char *room)
{
    Bias t;
    const int m = a.buckets.max_distance;
    t.max_distance = m;
    t.reach = bias_reach(m);
    t.pitch = bias_pitch(m);
    const auto value = [&](int d) {
        d = d < -m ? -m : d > m ? m : d;
        return a.table[bucket_of(a.buckets, d) * a.ld_table + head];
    };
    t.behind = value(-m);
    t.ahead = value(m);
    float *f = reinterpret_cast<float *>(room);
    if (m <= kCopiesMax) {
        for (int i = threadIdx.x; i < t.pitch; i += blockDim.x) {
            const float v = value(i - t.reach);
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (i + k < t.pitch) f[k * t.pitch + i + k] = v;
        }
        t.by_distance = f;
        t.bucket = nullptr;
    } else {
        for (int i = threadIdx.x; i <= 2 * m; i += blockDim.x) room[i] = (unsigned char)bucket_of(a.buckets, i - m);
        f = reinterpret_cast<float *>(room + bucket_bytes(m));
        for (int i = threadIdx.x; i < a.buckets.n; i += blockDim.x) f[i] = a.table[i * a.ld_table + head];
        t.by_distance = f;
        t.bucket = room;
    }
    return t;
}
// Of V adjacent keys, the first at distance d.
template <int P> __device__ __forceinline__ void bias_of(const Bias &t, int d, f2 (&bias)[P])
{
    const int m = t.max_distance;
    if (d >= m || d + 2 * P - 1 <= -m) {
        const float v = d >= m ? t.ahead : t.behind;
#pragma unroll
        for (int i = 0; i < P; ++i) bias[i] = pack2(v, v);
    } else if (!t.bucket) {
        const int at = d + t.reach, k = -at & 3;  // of the copy in which this entry begins 16 bytes
        const ulonglong2 *p = reinterpret_cast<const ulonglong2 *>(t.by_distance + k * t.pitch + at + k);
#pragma unroll
        for (int i = 0; i < P / 2; ++i) {
            const ulonglong2 q = p[i];
            bias[2 * i] = q.x;
            bias[2 * i + 1] = q.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            float v[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int e = d + 2 * i + k, near = e < -m ? -m : e > m ? m : e;
                v[k] = t.by_distance[t.bucket[near + m]];
            }
            bias[i] = pack2(v[0], v[1]);
        }
    }
}

__device__ __forceinline__ float exp2_of(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// 2^((x - top) log2 e).  The factor is not in the logits: the type's lowest value would be infinite with it, and a row of
// nothing else has weights all the same.  It is rounded once, by 2^-24 of the exponent: float32 weights are 1.15e-7 off where those of the plain
// form are 1.08e-7.
__device__ __forceinline__ float exp_of(float x, float top) { return exp2_of((x - top) * kLog2e); }
template <int P> __device__ __forceinline__ void exp_of(f2 (&x)[P], float top)
{
    const f2 less = pack2(-top, -top), log2e = pack2(kLog2e, kLog2e);
#pragma unroll
    for (int i = 0; i < P; ++i) {
        float lo, hi;
        unpack2(mul2(add2(x[i], less), log2e), lo, hi);
        x[i] = pack2(exp2_of(lo), exp2_of(hi));
    }
}
// off by one unit in the last place at most
__device__ __forceinline__ float reciprocal(float x)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
template <int P> __device__ __forceinline__ float sum_of(const f2 (&x)[P])
{
    f2 s = x[0];
#pragma unroll
    for (int i = 1; i < P; ++i) s = add2(s, x[i]);
    float lo, hi;
    unpack2(s, lo, hi);
    return lo + hi;
}
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
template <int P> __device__ __forceinline__ float max_of(const f2 (&x)[P], float m)
{
#pragma unroll
    for (int i = 0; i < P; ++i) {
        float lo, hi;
        unpack2(x[i], lo, hi);
        m = max3(m, lo, hi);
    }
    return m;
}

// Logits of V adjacent keys; -inf where not live.
// INNER: all of them are.
template <bool EVEN, bool INNER, typename T, int P>
__device__ __forceinline__ void logits(const Bias &t, const Row &w, const uint4 &raw, int c, float scale, f2 (&x)[P])
{
    f2 bias[P];
    spread(raw, x, T());
    bias_of(t, c - w.pos, bias);
#pragma unroll
    for (int i = 0; i < P; ++i) x[i] = fma2(pack2(scale, scale), x[i], bias[i]);
    if constexpr (!INNER) keep_live<EVEN>(x, c, w.live, -INFINITY);
}

// Blocks of an SM: registers for E elements a thread decide.  16 kernels spill a little: bf16 of 32 elements, on 16-byte boundaries, 64 bytes,
// float32 of 32 in groups of 256 60, of 24 48, the others 8 to 20.
template <typename T, int GS, int E, bool EVEN>
constexpr int kSoftmaxBlocks = GS > 256                   ? 1
                               : E <= 8                   ? 4
                               : E <= 16                  ? (EVEN || sizeof(T) == 2 ? 4 : 3)
                               : E <= 24                  ? (EVEN || sizeof(T) == 2 ? 3 : 2)
                               : EVEN && sizeof(T) == 2   ? 3
                                                          : 2;

// GS threads a row, E elements a thread; LONG: rows of any length, read twice.
template <typename T, int GS, int E, bool LONG, bool EVEN>
__global__ void __launch_bounds__(GS > 256 ? GS : 256, kSoftmaxBlocks<T, GS, E, EVEN>) k_softmax(const __grid_constant__ PositionArgs a)
{
    constexpr int V = 16 / sizeof(T), P = V / 2, NV = E / V, kThreads = GS > 256 ? GS : 256, kGroups = kThreads / GS;
    extern __shared__ __align__(16) unsigned char room[];
    __shared__ float scratch[2][32];
    griddep_wait();
    griddep_launch();
    const int head = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
    const Bias t = make_bias(a, head, room);
    __syncthreads();
    const int lane = threadIdx.x % GS;
    constexpr bool kAhead = kRowsAhead<T, LONG, EVEN>;
    uint4 *mine = reinterpret_cast<uint4 *>(room + bias_bytes(a.buckets.max_distance, a.buckets.n)) + threadIdx.x;
    const auto request = [&](const Row &w) {
#pragma unroll
        for (int v = 0; v < NV; ++v)
            if ((v * GS + lane) * V < w.live) copy_async(mine + v * kThreads, static_cast<const T *>(a.s) + w.at + (v * GS + lane) * V);
        copy_commit();
    };
    // where the thread's v-th access begins, in a row on a 16-byte boundary
    const auto at = [&](int v) { return (v * GS + lane) * V; };
    Walk<kGroups> walk(a, head, chunk, threadIdx.x / GS);
    Row w = walk.here(a), next;
    if constexpr (kAhead) request(w);
    // the groups of a block take as many rounds
    for (unsigned r = chunk * kGroups; r < (unsigned)a.rows; r += walk.step, w = next) {
        walk.next(a);
        next = walk.here(a);
        const int n = w.n;
        const T *s = static_cast<const T *>(a.s) + w.at;
        T *p = static_cast<T *>(a.out) + (EVEN ? w.at : offset_of(a.out_at, w, head));
        const int off = EVEN ? 0 : off16(s);
        const bool aligned = off16(p) == off;
        const Reach reach = reach_of(s, off, w.at, n, a.s_span);
        if constexpr (!LONG) {
            f2 x[NV][P];
            uint4 raw[NV];
            float top = -INFINITY, sum = 0.f;
            if constexpr (kAhead) copy_wait<0>();
#pragma unroll
            for (int v = 0; v < NV; ++v)
                if (at(v) - off < w.live) raw[v] = kAhead ? mine[v * kThreads] : load_raw<EVEN>(s, at(v) - off, n, reach);
            // the group's accesses that end before `plain` are live and far behind: most of them, with nothing to look up
            const int plain = EVEN ? min(w.live, w.pos - t.max_distance + 1) : 0;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c = at(v) - off;
                if ((v + 1) * GS * V <= plain) {
                    const f2 factor = pack2(a.scale, a.scale), bias = pack2(t.behind, t.behind);
                    spread(raw[v], x[v], T());
#pragma unroll
                    for (int i = 0; i < P; ++i) x[v][i] = fma2(factor, x[v][i], bias);
                    top = max_of(x[v], top);
                } else if (EVEN && (v + 1) * GS * V <= w.live) {
                    logits<EVEN, true, T, P>(t, w, raw[v], c, a.scale, x[v]);
                    top = max_of(x[v], top);
                } else if (c < w.live) {
                    logits<EVEN, false, T, P>(t, w, raw[v], c, a.scale, x[v]);
                    top = max_of(x[v], top);
                } else if (v * GS * V - off < w.live) {
#pragma unroll
                    for (int i = 0; i < P; ++i) x[v][i] = pack2(-INFINITY, -INFINITY);
                }
            }
            top = group_join<GS, true>(top, scratch);
            if constexpr (kAhead) request(next);  // its place has been read
            if (top == -INFINITY) top = 0.f;  // nothing is live, all is -inf, or the rest is NaN
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                if (v * GS * V - off < w.live) {
                    exp_of(x[v], top);
                    sum += sum_of(x[v]);
                }
            }
            sum = group_join<GS, false>(sum, scratch + 1);
            const float inv = sum == 0.f ? 0.f : reciprocal(sum);
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c = at(v) - off;
                if (v * GS * V - off < w.live) {
#pragma unroll
                    for (int i = 0; i < P; ++i) x[v][i] = mul2(x[v][i], pack2(inv, inv));
                    if (inv != inv) keep_live<EVEN>(x[v], c, w.live, 0.f);  // NaN, but not where nothing is live
                } else {
#pragma unroll
                    for (int i = 0; i < P; ++i) x[v][i] = 0ull;
                }
                if (c < n) store_cols<EVEN, T, P>(p, c, n, aligned, x[v]);
            }
        } else {
            float top = -INFINITY, sum = 0.f;
            for (int c = lane * V - off; c < w.live; c += GS * V) {
                f2 x[P];
                logits<EVEN, false, T, P>(t, w, load_raw<EVEN>(s, c, n, reach), c, a.scale, x);
                const float best = max_of(x, top), base = best == -INFINITY ? 0.f : best;
                exp_of(x, base);
                sum = sum * exp_of(top == -INFINITY ? base : top, base) + sum_of(x);
                top = best;
            }
            float all = group_join<GS, true>(top, scratch);
            if (all == -INFINITY) all = 0.f;
            sum = group_join<GS, false>(sum * exp_of(top == -INFINITY ? all : top, all), scratch + 1);
            const float inv = sum == 0.f ? 0.f : reciprocal(sum);
            for (int c = lane * V - off; c < n; c += GS * V) {
                f2 x[P] = {};
                if (c < w.live) {
                    logits<EVEN, false, T, P>(t, w, load_raw<EVEN>(s, c, n, reach), c, a.scale, x);
                    exp_of(x, all);
#pragma unroll
                    for (int i = 0; i < P; ++i) x[i] = mul2(x[i], pack2(inv, inv));
                    if (inv != inv) keep_live<EVEN>(x, c, w.live, 0.f);
                }
                store_cols<EVEN, T, P>(p, c, n, aligned, x);
            }
        }
    }
}

// ---- gradient ------------------------------------------------------------------------------

// Near the diagonal adjacent keys are in different buckets: those are summed by distance, in registers.  A warp puts its values at the
// keys from 128 before the query to 136 behind it, in whole accesses, into shared memory, and lane l takes the distances
// l - 136, l - 104, ... from there.  (One by one into the sums by bucket: 9 instructions a key, for 8 keys wherever one lane's keys are
// in different buckets.)
constexpr int kNear = 128, kNearKeys = 2 * kNear + 16, kNearTakes = 9, kNearRoom = 32 * kNearTakes;
struct Near {
    float *room;  // [kNearRoom] of this warp
    float sum[kNearTakes];
    __device__ __forceinline__ static int distance(int k) { return (int)threadIdx.x % 32 - kNear - 8 + 32 * k; }
    // The first key: as many elements behind a boundary of 8 as the rows begin before one.
    __device__ __forceinline__ static int first(const Row &w, int off) { return ((w.pos - kNear + off) & ~7) - off; }
};

// Shared memory before the rows that are on their way: the buckets by distance, the sums.
__host__ __device__ inline size_t grad_bytes(int max_distance, int n_buckets)
{
    return bucket_bytes(max_distance) + (n_buckets ? 8 * (128 * (size_t)n_buckets + 4 * kNearRoom) : 0);
}

// Adds V adjacent values, the first at distance d, to the lane's sums by bucket.
template <int P>
__device__ __forceinline__ void add_buckets(const unsigned char *bucket, int m, float *lane_sums, int d, const f2 (&g)[P], float &behind, float &ahead)
{
    if (d + 2 * P - 1 <= -m) {
        behind += sum_of(g);
    } else if (d >= m) {
        ahead += sum_of(g);
    } else {
        const auto at = [&](int e) {
            e = e < -m ? -m : e > m ? m : e;
            return (int)bucket[e + m];
        };
        const int first = at(d), last = at(d + 2 * P - 1);
        if (first == last) {
            lane_sums[first * 32] += sum_of(g);
        } else {
            float y[2 * P];
            flat(g, y);
#pragma unroll
            for (int e = 0; e < 2 * P; ++e) lane_sums[at(d + e) * 32] += y[e];
        }
    }
}

// Blocks of an SM, as registers for two rows of E elements a thread allow (bf16, 1024 keys: 118 us with two blocks or three, 127 with three and
// 80 bytes spilled; two kernels off 16-byte boundaries spill 16 and 24 bytes).
template <typename T, int E> constexpr int kGradBlocks = sizeof(T) == 2 ? (E <= 8 ? 4 : E <= 24 ? 3 : 2) : (E <= 8 ? 4 : E <= 16 ? 3 : 2);

// The sums by bucket of a block, in shared memory behind the buckets of all distances, and of a thread.
struct Sums {
    float *lane_sums, *all;  // of this lane, one every 32; [warp][bucket][lane]
    float behind, ahead;
    Near near;
    __device__ __forceinline__ Sums(const PositionArgs &a, unsigned char *room)
    {
        const int m = a.buckets.max_distance, n = a.buckets.n;
        all = reinterpret_cast<float *>(room + bucket_bytes(m));
        if (a.partials) {
            for (int i = threadIdx.x; i <= 2 * m; i += 256) room[i] = (unsigned char)bucket_of(a.buckets, i - m);
            for (int i = threadIdx.x; i < 8 * n * 8; i += 256) reinterpret_cast<float4 *>(all)[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
        __syncthreads();
        lane_sums = all + (threadIdx.x / 32) * n * 32 + threadIdx.x % 32;
        behind = ahead = 0.f;
        near.room = all + 8 * n * 32 + threadIdx.x / 32 * kNearRoom;
#pragma unroll
        for (int k = 0; k < kNearTakes; ++k) near.sum[k] = 0.f;
    }
    // What the warp has put into its room from key `first` on; the group's threads have V adjacent keys each,
    // `off` elements in front of the row the first.
    template <int GS, int V> __device__ __forceinline__ void take(const PositionArgs &a, const Row &w, int first, int off)
    {
        constexpr unsigned kWarps = GS < 32 ? 1 : GS / 32;
        __syncwarp();
#pragma unroll
        for (int k = 0; k < kNearTakes; ++k) {
            if (a.causal && k > 4) break;  // distances from 24 on
            const int j = w.pos + Near::distance(k);
            // live, and one of this warp's
            if (j >= 0 && j < w.live && (kWarps == 1 || (unsigned)(j + off) / (32 * V) % kWarps == threadIdx.x % GS / 32) &&
                (V == 1 || (unsigned)(j - first) < (unsigned)kNearKeys))
                near.sum[k] += near.room[j - first];
        }
        __syncwarp();
    }
    __device__ __forceinline__ void leave(const PositionArgs &a, const unsigned char *room, int head, int chunk)
    {
        const int m = a.buckets.max_distance, n = a.buckets.n;
        if (!a.partials) return;
#pragma unroll
        for (int k = 0; k < kNearTakes; ++k) {
            int d = Near::distance(k);
            d = d < -m ? -m : d > m ? m : d;
            lane_sums[room[d + m] * 32] += near.sum[k];
        }
        lane_sums[room[0] * 32] += behind;
        lane_sums[room[2 * m] * 32] += ahead;
        __syncthreads();
        // a warp adds up a bucket: lane by lane over the warps, then over the lanes
#pragma unroll 4
        for (int k = threadIdx.x / 32; k < n; k += 8) {
            float v = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) v += all[(i * n + k) * 32 + threadIdx.x % 32];
            v = warp_sum(v);
            if (threadIdx.x % 32 == 0) a.partials[((long long)head * n + k) * a.chunks + chunk] = v;
        }
    }
};

template <typename T, int GS, int E, bool LONG, bool EVEN>
__global__ void __launch_bounds__(256, kGradBlocks<T, E>) k_softmax_grad(const __grid_constant__ PositionArgs a)
{
    constexpr int V = 16 / sizeof(T), P = V / 2, NV = E / V, kGroups = 256 / GS;
    extern __shared__ __align__(16) unsigned char room[];
    __shared__ float scratch[2][32];
    int turn = 0;
    griddep_wait();
    if (a.partials) griddep_launch();  // the successor is another kernel of this call
    const int head = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks, m = a.buckets.max_distance;
    Sums sums(a, room);
    f2 behind2 = 0ull;
    const int far_from = m > kNear + 8 ? m : kNear + 8;  // keys so far behind are in the last bucket and none of those by distance
    constexpr bool kByDistance = GS >= 32;
    const int lane = threadIdx.x % GS;
    const f2 scale = pack2(a.scale, a.scale);
    const auto at = [&](int v) { return (v * GS + lane) * V; };
    constexpr bool kAhead = kRowsAhead<T, LONG, EVEN>;
    uint4 *mine = reinterpret_cast<uint4 *>(room + grad_bytes(m, a.partials ? a.buckets.n : 0)) + threadIdx.x;
    const auto request = [&](const Row &w) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * GS + lane) * V;
            if (c < w.live) {
                copy_async(mine + 2 * v * 256, static_cast<const T *>(a.s) + w.at + c);
                copy_async(mine + (2 * v + 1) * 256, static_cast<const T *>(a.dp) + w.at + c);
            }
        }
        copy_commit();
    };
    Walk<kGroups> walk(a, head, chunk, threadIdx.x / GS);
    Row w = walk.here(a), next;
    if constexpr (kAhead) request(w);
    for (unsigned r = chunk * kGroups; r < (unsigned)a.rows; r += walk.step, w = next) {
        walk.next(a);
        next = walk.here(a);
        const int n = w.n;
        const long long dp_from = EVEN ? w.at : offset_of(a.dp_at, w, head);
        const T *p = static_cast<const T *>(a.s) + w.at, *dp = static_cast<const T *>(a.dp) + dp_from;
        T *ds = static_cast<T *>(a.out) + (EVEN ? w.at : offset_of(a.out_at, w, head));
        const int off = EVEN ? 0 : off16(p);
        const bool out_aligned = off16(ds) == off;
        const Reach reach = reach_of(p, off, w.at, n, a.s_span), dp_reach = reach_of(dp, off, dp_from, n, a.dp_span);
        const int near_first = Near::first(w, off);
        // of V adjacent keys, with zeros where nothing is live: g, its sums, ds
        const auto finish = [&](const uint4 &p_raw, const uint4 &dp_raw, int c, float dot) {
            f2 g[P], y[P];
            if (c < w.live) {
                const f2 less = pack2(-dot, -dot);
                spread(p_raw, g, T());
                spread(dp_raw, y, T());
#pragma unroll
                for (int i = 0; i < P; ++i) g[i] = mul2(g[i], add2(y[i], less));
                if (!isfinite(dot)) keep_live<EVEN>(g, c, w.live, 0.f);
                if (a.partials) {
                    if (kByDistance && (unsigned)(c - near_first) < (unsigned)kNearKeys) {
                        float x[V];
                        flat(g, x);
                        store_vec<V>(sums.near.room + (c - near_first), x);
                    } else {
                        add_buckets<P>(room, m, sums.lane_sums, c - w.pos, g, sums.behind, sums.ahead);
                    }
                }
#pragma unroll
                for (int i = 0; i < P; ++i) y[i] = mul2(g[i], scale);
            } else {
#pragma unroll
                for (int i = 0; i < P; ++i) y[i] = 0ull;
            }
            if (a.out) store_cols<EVEN, T, P>(ds, c, n, out_aligned, y);
        };
        const auto products = [&](const uint4 &p_raw, const uint4 &dp_raw, f2 sum) {
            f2 x[P], y[P];
            spread(p_raw, x, T());
            spread(dp_raw, y, T());
#pragma unroll
            for (int i = 0; i < P; ++i) sum = fma2(x[i], y[i], sum);
            return sum;
        };
        // zeros where nothing is live
        const auto fetch = [&](int c, uint4 &p_raw, uint4 &dp_raw) {
            p_raw = load_raw<EVEN>(p, c, n, reach);
            dp_raw = load_raw<EVEN>(dp, c, n, dp_reach);
            keep_live<EVEN, T>(p_raw, c, w.live);
            keep_live<EVEN, T>(dp_raw, c, w.live);
        };
        f2 sum = 0ull;
        float dot, odd;
        if constexpr (!LONG) {
            uint4 x[NV], y[NV];
            if constexpr (kAhead) copy_wait<0>();
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c = at(v) - off;
                if (c < w.live) {
                    x[v] = kAhead ? mine[2 * v * 256] : load_raw<EVEN>(p, c, n, reach);
                    y[v] = kAhead ? mine[(2 * v + 1) * 256] : load_raw<EVEN>(dp, c, n, dp_reach);
                }
            }
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c = at(v) - off;
                if (c < w.live) {
                    if (!EVEN || (v + 1) * GS * V > w.live) {
                        keep_live<EVEN, T>(x[v], c, w.live);
                        keep_live<EVEN, T>(y[v], c, w.live);
                    }
                    sum = products(x[v], y[v], sum);
                }
            }
            unpack2(sum, dot, odd);
            dot = group_join<GS, false>(dot + odd, scratch + (turn ^= 1));
            if constexpr (kAhead) request(next);  // its place has been read
            // the group's accesses that end before `plain` are live and in the last bucket
            const int plain = EVEN && isfinite(dot) ? min(w.live, w.pos - far_from) : 0;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                if ((v + 1) * GS * V <= plain) {
                    f2 g[P], d[P];
                    const f2 less = pack2(-dot, -dot);
                    spread(x[v], g, T());
                    spread(y[v], d, T());
#pragma unroll
                    for (int i = 0; i < P; ++i) {
                        g[i] = mul2(g[i], add2(d[i], less));
                        behind2 = add2(behind2, g[i]);
                        d[i] = mul2(g[i], scale);
                    }
                    if (a.out) store_cols<EVEN, T, P>(ds, at(v), n, true, d);
                } else if (v * GS * V - off >= w.live) {
                    const f2 zero[P] = {};
                    if (a.out && at(v) - off < n) store_cols<EVEN, T, P>(ds, at(v) - off, n, out_aligned, zero);
                } else if (at(v) - off < n) {
                    finish(x[v], y[v], at(v) - off, dot);
                }
            }
        } else {
            uint4 x, y;
            for (int c = lane * V - off; c < w.live; c += GS * V) {
                fetch(c, x, y);
                sum = products(x, y, sum);
            }
            unpack2(sum, dot, odd);
            dot = group_join<GS, false>(dot + odd, scratch + (turn ^= 1));
            for (int c = lane * V - off; c < n; c += GS * V) {
                if (c < w.live) fetch(c, x, y);
                finish(x, y, c, dot);
            }
        }
        if (kByDistance && a.partials) sums.template take<GS, V>(a, w, near_first, off);
    }
    float lo, hi;
    unpack2(behind2, lo, hi);
    sums.behind += lo + hi;
    sums.leave(a, room, head, chunk);
}

// ---- short rows anywhere --------------------------------------------------------------------
// Rows of up to kAnyMax elements that do not begin on and end at 16-byte boundaries, or whose matrices have different strides: the threads of
// a group take adjacent elements, one each.  16-byte accesses spend more on the ragged ends (120 MB of bf16 rows of 130: 232 us, 195; of 250
// 144 and 129; gradient 336 and 220, 195 and 167), longer rows do not (float32 of 250: 63 and 67, gradient 81 and 92).
template <typename T> constexpr int kAnyMax = sizeof(T) == 4 ? 192 : 256;

__device__ __forceinline__ float bias_at(const Bias &t, int d)
{
    const int m = t.max_distance;
    d = d < -m ? -m : d > m ? m : d;
    return t.bucket ? t.by_distance[t.bucket[d + m]] : t.by_distance[d + t.reach];
}

template <typename T, int GS, int E>
__global__ void __launch_bounds__(GS > 256 ? GS : 256, kSoftmaxBlocks<T, GS, E, false>) k_softmax_any(const __grid_constant__ PositionArgs a)
{
    constexpr int kThreads = GS > 256 ? GS : 256, kGroups = kThreads / GS;
    extern __shared__ __align__(16) unsigned char room[];
    __shared__ float scratch[2][32];
    griddep_wait();
    griddep_launch();
    const int head = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
    const Bias t = make_bias(a, head, room);
    __syncthreads();
    const int lane = threadIdx.x % GS;
    Walk<kGroups> walk(a, head, chunk, threadIdx.x / GS);
    // the groups of a block take as many rounds
    for (unsigned r = chunk * kGroups; r < (unsigned)a.rows; r += walk.step, walk.next(a)) {
        const Row w = walk.here(a);
        const T *s = static_cast<const T *>(a.s) + w.at;
        T *p = static_cast<T *>(a.out) + offset_of(a.out_at, w, head);
        const int far = w.pos - t.max_distance + 1;  // keys before it are far behind
        float x[E], top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int k = 0; k < E; ++k)
            if (k * GS + lane < w.live) x[k] = to_f32(s[k * GS + lane]);
#pragma unroll
        for (int k = 0; k < E; ++k) {
            const int c = k * GS + lane;
            if (k * GS >= w.live) break;
            if ((k + 1) * GS <= min(far, w.live)) x[k] = fmaf(a.scale, x[k], t.behind);
            else x[k] = c < w.live ? fmaf(a.scale, x[k], bias_at(t, c - w.pos)) : -INFINITY;
            top = fmaxf(top, x[k]);
        }
        top = group_join<GS, true>(top, scratch);
        if (top == -INFINITY) top = 0.f;  // nothing is live, all is -inf, or the rest is NaN
#pragma unroll
        for (int k = 0; k < E; ++k) {
            if (k * GS >= w.live) break;
            sum += x[k] = exp_of(x[k], top);
        }
        sum = group_join<GS, false>(sum, scratch + 1);
        const float inv = sum == 0.f ? 0.f : reciprocal(sum);
#pragma unroll
        for (int k = 0; k < E; ++k) {
            const int c = k * GS + lane;
            if (c < w.n) put(p + c, c < w.live ? x[k] * inv : 0.f);
        }
    }
}

template <typename T, int E> constexpr int kGradAnyBlocks = E <= 8 ? 4 : E <= 16 ? 3 : 2;

template <typename T, int GS, int E>
__global__ void __launch_bounds__(256, kGradAnyBlocks<T, E>) k_softmax_grad_any(const __grid_constant__ PositionArgs a)
{
    constexpr int kGroups = 256 / GS;
    extern __shared__ __align__(16) unsigned char room[];
    __shared__ float scratch[2][32];
    int turn = 0;
    griddep_wait();
    if (a.partials) griddep_launch();  // the successor is another kernel of this call
    const int head = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks, m = a.buckets.max_distance;
    Sums sums(a, room);
    constexpr bool kByDistance = GS >= 32;
    const int far_from = m > kNear + 8 ? m : kNear + 8;  // keys so far behind are in the last bucket and none of those by distance
    const int lane = threadIdx.x % GS;
    Walk<kGroups> walk(a, head, chunk, threadIdx.x / GS);
    for (unsigned r = chunk * kGroups; r < (unsigned)a.rows; r += walk.step, walk.next(a)) {
        const Row w = walk.here(a);
        const T *p = static_cast<const T *>(a.s) + w.at, *dp = static_cast<const T *>(a.dp) + offset_of(a.dp_at, w, head);
        T *ds = static_cast<T *>(a.out) + offset_of(a.out_at, w, head);
        const int near_first = w.pos - kNear - 8;
        // g of a live key
        const auto add = [&](float g, int c) {
            if (kByDistance && (unsigned)(c - near_first) < (unsigned)kNearRoom) {
                sums.near.room[c - near_first] = g;
            } else {
                const int d = c - w.pos;
                if (d <= -m) sums.behind += g;
                else if (d >= m) sums.ahead += g;
                else sums.lane_sums[room[d + m] * 32] += g;
            }
        };
        float dot = 0.f;
        float x[E], y[E];
#pragma unroll
        for (int k = 0; k < E; ++k) {
            if (k * GS + lane < w.live) {
                x[k] = to_f32(p[k * GS + lane]);
                y[k] = to_f32(dp[k * GS + lane]);
            }
        }
#pragma unroll
        for (int k = 0; k < E; ++k)
            if (k * GS + lane < w.live) dot = fmaf(x[k], y[k], dot);
        dot = group_join<GS, false>(dot, scratch + (turn ^= 1));
#pragma unroll
        for (int k = 0; k < E; ++k) {
            const int c = k * GS + lane;
            if (k * GS >= w.n) break;
            float g = 0.f;
            if (c < w.live) {
                g = x[k] * (y[k] - dot);
                if ((k + 1) * GS <= w.pos - far_from) sums.behind += g;
                else if (a.partials) add(g, c);
            }
            if (a.out && c < w.n) put(ds + c, a.scale * g);
        }
        if (kByDistance && a.partials) sums.template take<GS, 1>(a, w, near_first, 0);
    }
    sums.leave(a, room, head, chunk);
}

struct JoinArgs {
    const float *partials;  // [heads, buckets, chunks]
    void *dtable;
    long long ld;
    int heads, n_buckets, chunks, accumulate;
};
template <typename T> __global__ void __launch_bounds__(256) k_join_buckets(const JoinArgs a)
{
    griddep_wait();
    const int at = blockIdx.x * 8 + threadIdx.x / 32, lane = threadIdx.x % 32;
    if (at >= a.heads * a.n_buckets) return;
    const float *p = a.partials + (long long)at * a.chunks;
    double v = 0.0;
    for (int i = lane; i < a.chunks; i += 32) v += p[i];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (lane == 0) {
        T *out = static_cast<T *>(a.dtable) + (at % a.n_buckets) * a.ld + at / a.n_buckets;
        put(out, (float)(a.accumulate ? v + to_f32(*out) : v));
    }
}

// ---- host side -----------------------------------------------------------------------------

// n^far against exact^(far - k) * max_distance^k, in whole numbers where logarithms do not tell.
struct Big {
    uint32_t limb[32] = {1};  // 1024 bits: 64 factors of at most 2^14 need 896
    void times(uint32_t f)
    {
        uint64_t carry = 0;
        for (uint32_t &l : limb) {
            carry += (uint64_t)l * f;
            l = (uint32_t)carry;
            carry >>= 32;
        }
    }
    bool operator>=(const Big &o) const
    {
        for (int i = 31; i >= 0; --i)
            if (limb[i] != o.limb[i]) return limb[i] > o.limb[i];
        return true;
    }
};
bool reaches(int n, int far, int k, int exact, int max_distance)
{
    const double diff = far * std::log2((double)n) - ((far - k) * std::log2((double)exact) + k * std::log2((double)max_distance));
    if (std::fabs(diff) > 1e-9) return diff > 0;
    Big left, right;
    for (int i = 0; i < far; ++i) {
        left.times((uint32_t)n);
        right.times((uint32_t)(i < k ? max_distance : exact));
    }
    return left >= right;
}
Buckets make_buckets(int n_buckets, int max_distance, int both)
{
    Buckets b;
    b.n = n_buckets;
    b.both = both;
    b.m = both ? n_buckets / 2 : n_buckets;
    b.exact = b.m / 2;
    b.max_distance = max_distance;
    const int far = b.m - b.exact;
    b.n_borders = far - 1;
    const double lo = std::log2((double)b.exact), step = (std::log2((double)max_distance) - lo) / far;
    for (int k = 1; k < far; ++k) {
        int n = std::max(b.exact, (int)std::exp2(lo + k * step) - 1);
        while (!reaches(n, far, k, b.exact, max_distance)) ++n;  // ends: max_distance reaches
        b.border[k - 1] = (short)n;
    }
    return b;
}
adascale_status check_buckets(long long n_buckets, long long max_distance, int both)
{
    if (n_buckets < (both ? 4 : 2) || (both && n_buckets % 2)) return ADASCALE_ERR_INVALID_ARG;
    if (n_buckets > ADASCALE_POSITION_MAX_BUCKETS || max_distance > ADASCALE_POSITION_MAX_DISTANCE) return ADASCALE_ERR_TOO_LARGE;
    return max_distance > (both ? n_buckets / 2 : n_buckets) / 2 ? ADASCALE_OK : ADASCALE_ERR_INVALID_ARG;
}
// What the forward and the gradient call share.
template <typename A> adascale_status check_common(const A &a)
{
    if (a.batch < 0 || a.heads < 0 || a.n_queries < 0 || a.n_keys < 0 || !is_dtype(a.dtype) || !std::isfinite(a.scale)) return ADASCALE_ERR_INVALID_ARG;
    if ((a.lengths && !is_itype(a.length_type)) || (a.starts && !is_itype(a.start_type))) return ADASCALE_ERR_INVALID_ARG;
    const adascale_status bad = check_buckets(a.n_buckets, a.max_distance, a.bidirectional);
    if (bad != ADASCALE_OK) return bad;
    if (a.n_queries > kMaxLen || a.n_keys > kMaxLen || a.heads > 65535 || a.batch > kMaxRows ||
        (a.batch && a.n_queries > kMaxRows / a.batch))
        return ADASCALE_ERR_TOO_LARGE;
    return ADASCALE_OK;
}
// Inputs may be broadcast (stride 0); no two rows of an output share an element.
bool readable(long long b, long long h, long long q) { return b >= 0 && h >= 0 && q >= 0; }
template <typename A> bool writable(const A &a, long long b, long long h, long long q)
{
    std::pair<long long, long long> dims[3] = {{b, a.batch}, {h, a.heads}, {q, a.n_queries}};
    std::sort(dims, dims + 3);
    long long extent = a.n_keys;
    for (const auto &d : dims) {
        if (d.second <= 1) continue;
        if (d.first < extent) return false;
        if (d.first > (1LL << 60) / d.second) return false;
        extent += d.first * (d.second - 1);
    }
    return true;
}

// Blocks of a head: as many as the device holds at once, fewer where there are few rows.
int chunks_of(long long rows, long long heads, int groups, int sms, int blocks, size_t smem)
{
    const long long held = std::max<long long>(1, std::min<long long>(blocks, (227 << 10) / (long long)(smem + 2048)));  // beside static and reserved memory
    const long long want = std::max<long long>(1, sms * held / heads), most = std::max<long long>(1, kBlocksMax / heads);
    return (int)std::max<long long>(1, std::min(std::min(want, most), ceil_div(rows, groups)));
}

// How rows are read: 16 bytes a thread, on boundaries or with ragged ends, or one element a thread.
enum Rows { kEven, kRagged, kAny };

template <typename T, int GS, int E, bool LONG, Rows R> cudaError_t run_softmax(PositionArgs &a, int heads, int sms, cudaStream_t s)
{
    static OncePerDevice known;
    constexpr int kThreads = GS > 256 ? GS : 256;
    void (*kernel)(PositionArgs);
    if constexpr (R == kAny) kernel = k_softmax_any<T, GS, E>;
    else kernel = k_softmax<T, GS, E, LONG, R == kEven>;
    cudaError_t e = allow_smem(reinterpret_cast<const void *>(kernel), known);
    if (e != cudaSuccess) return e;
    const size_t smem = bias_bytes(a.buckets.max_distance, a.buckets.n) + (R != kAny && kRowsAhead<T, LONG, R == kEven> ? kThreads * E * sizeof(T) : 0);
    a.chunks = chunks_of(a.rows, heads, kThreads / GS, sms, kSoftmaxBlocks<T, GS, E, R == kEven>, smem);
    return launch(kernel, (long long)heads * a.chunks, kThreads, smem, s, a);
}
// Whether all rows of a matrix begin on 16-byte boundaries.
template <typename T> bool on16(const void *p, const Strides &at)
{
    constexpr long long V = 16 / (long long)sizeof(T);
    return !p || (on(p, 16) && at.b % V == 0 && at.h % V == 0 && at.q % V == 0);
}
// The elements that a row's group has to hold: with rows off 16-byte boundaries up to V - 1 before it too.
template <typename T> long long held(const PositionArgs &a)
{
    return a.n_keys + (on16<T>(a.s, a.s_at) ? 0 : 16 / (long long)sizeof(T) - 1);
}
template <typename T> bool all_even(const PositionArgs &a)
{
    const auto same = [&](const void *p, const Strides &at) { return !p || (on(p, 16) && at.b == a.s_at.b && at.h == a.s_at.h && at.q == a.s_at.q); };
    return a.n_keys % (16 / (int)sizeof(T)) == 0 && on16<T>(a.s, a.s_at) && same(a.dp, a.dp_at) && same(a.out, a.out_at);
}
// The narrowest group whose registers hold a row.
template <typename T, Rows R> cudaError_t pick_softmax(PositionArgs &a, int heads, int sms, cudaStream_t s)
{
    const long long n = R == kRagged ? held<T>(a) : a.n_keys;
    if constexpr (R != kRagged) {
        if (n <= 8 * 8) return run_softmax<T, 8, 8, false, R>(a, heads, sms, s);
        if (n <= 8 * 16) return run_softmax<T, 8, 16, false, R>(a, heads, sms, s);
    }
    if (R == kAny || n <= 32 * 8) return run_softmax<T, 32, 8, false, R>(a, heads, sms, s);
    if constexpr (R != kAny) {
        if (n <= 32 * 16) return run_softmax<T, 32, 16, false, R>(a, heads, sms, s);
        if (n <= 32 * 24) return run_softmax<T, 32, 24, false, R>(a, heads, sms, s);
        if (n <= 32 * 32) return run_softmax<T, 32, 32, false, R>(a, heads, sms, s);
        if (n <= 64 * 32) return run_softmax<T, 64, 32, false, R>(a, heads, sms, s);
        if (n <= 128 * 32) return run_softmax<T, 128, 32, false, R>(a, heads, sms, s);
        if (n <= 256 * 32) return run_softmax<T, 256, 32, false, R>(a, heads, sms, s);
        if (n <= 1024 * 16) return run_softmax<T, 1024, 16, false, R>(a, heads, sms, s);
        return run_softmax<T, 1024, 8, true, R>(a, heads, sms, s);
    }
}
template <typename T> cudaError_t pick_softmax(PositionArgs &a, int heads, int sms, cudaStream_t s)
{
    if (all_even<T>(a)) return pick_softmax<T, kEven>(a, heads, sms, s);
    return a.n_keys <= kAnyMax<T> ? pick_softmax<T, kAny>(a, heads, sms, s) : pick_softmax<T, kRagged>(a, heads, sms, s);
}

template <typename T, int GS, int E, bool LONG, Rows R> cudaError_t run_grad(PositionArgs &a, int heads, int sms, cudaStream_t s)
{
    static OncePerDevice known;
    void (*kernel)(PositionArgs);
    if constexpr (R == kAny) kernel = k_softmax_grad_any<T, GS, E>;
    else kernel = k_softmax_grad<T, GS, E, LONG, R == kEven>;
    cudaError_t e = allow_smem(reinterpret_cast<const void *>(kernel), known);
    if (e != cudaSuccess) return e;
    const size_t smem = grad_bytes(a.buckets.max_distance, a.partials ? a.buckets.n : 0) +
                        (R != kAny && kRowsAhead<T, LONG, R == kEven> ? 256 * 2 * E * sizeof(T) : 0);
    a.chunks = chunks_of(a.rows, heads, 256 / GS, sms, R == kAny ? kGradAnyBlocks<T, E> : kGradBlocks<T, E>, smem);
    return launch(kernel, (long long)heads * a.chunks, 256, smem, s, a);
}
template <typename T, Rows R> cudaError_t pick_grad(PositionArgs &a, int heads, int sms, cudaStream_t s)
{
    const long long n = R == kRagged ? held<T>(a) : a.n_keys;
    if constexpr (R != kRagged) {
        if (n <= 8 * 8) return run_grad<T, 8, 8, false, R>(a, heads, sms, s);
        if (n <= 8 * 16) return run_grad<T, 8, 16, false, R>(a, heads, sms, s);
    }
    if (R == kAny || n <= 32 * 8) return run_grad<T, 32, 8, false, R>(a, heads, sms, s);
    if constexpr (R != kAny) {
        if (n <= 32 * 16) return run_grad<T, 32, 16, false, R>(a, heads, sms, s);
        if (n <= 32 * 24) return run_grad<T, 32, 24, false, R>(a, heads, sms, s);
        if (n <= 32 * 32) return run_grad<T, 32, 32, false, R>(a, heads, sms, s);
        if (n <= 64 * 32) return run_grad<T, 64, 32, false, R>(a, heads, sms, s);
        if (n <= 128 * 32) return run_grad<T, 128, 32, false, R>(a, heads, sms, s);
        if (n <= 256 * 32) return run_grad<T, 256, 32, false, R>(a, heads, sms, s);
        return run_grad<T, 256, 8, true, R>(a, heads, sms, s);
    }
}
template <typename T> cudaError_t pick_grad(PositionArgs &a, int heads, int sms, cudaStream_t s)
{
    if (all_even<T>(a)) return pick_grad<T, kEven>(a, heads, sms, s);
    return a.n_keys <= kAnyMax<T> ? pick_grad<T, kAny>(a, heads, sms, s) : pick_grad<T, kRagged>(a, heads, sms, s);
}

// Strides, 0 where there is only one; and how many elements a matrix reaches over.
template <typename A> Strides used(const A &a, long long b, long long h, long long q)
{
    return {a.batch > 1 ? b : 0, a.heads > 1 ? h : 0, a.n_queries > 1 ? q : 0};
}
template <typename A> long long span_of(const A &a, const Strides &at)
{
    return (a.batch - 1) * at.b + (a.heads - 1) * at.h + (a.n_queries - 1) * at.q + a.n_keys;
}
template <typename A> void fill_common(PositionArgs &p, const A &a)
{
    p.lengths = a.lengths;
    p.starts = a.starts;
    p.wide_lengths = a.length_type == ADASCALE_I64;
    p.wide_starts = a.start_type == ADASCALE_I64;
    p.causal = a.causal != 0;
    p.rows = a.batch * a.n_queries;
    p.n_queries = (int)a.n_queries;
    p.n_keys = (int)a.n_keys;
    p.scale = a.scale;
    p.buckets = make_buckets(a.n_buckets, a.max_distance, a.bidirectional != 0);
}

}  // namespace

extern "C" adascale_status adascale_position_softmax(const adascale_position_softmax_args *args, void *cuda_stream)
{
    if (!args) return ADASCALE_ERR_INVALID_ARG;
    const adascale_position_softmax_args &a = *args;
    const adascale_status bad = check_common(a);
    if (bad != ADASCALE_OK) return bad;
    if (a.ld_table < a.heads || !readable(a.scores_stride_b, a.scores_stride_h, a.scores_stride_q) ||
        !writable(a, a.probs_stride_b, a.probs_stride_h, a.probs_stride_q))
        return ADASCALE_ERR_INVALID_ARG;
    if (a.batch == 0 || a.heads == 0 || a.n_queries == 0 || a.n_keys == 0) return ADASCALE_OK;
    if (!a.scores || !a.probs || !a.table) return ADASCALE_ERR_INVALID_ARG;
    if (a.probs == a.scores && (a.probs_stride_b != a.scores_stride_b || a.probs_stride_h != a.scores_stride_h || a.probs_stride_q != a.scores_stride_q))
        return ADASCALE_ERR_INVALID_ARG;
    const int b = elem_bytes(a.dtype);
    if (!on(a.scores, b) || !on(a.probs, b) || !on(a.table, 4) || (a.lengths && !on(a.lengths, id_bytes(a.length_type))) ||
        (a.starts && !on(a.starts, id_bytes(a.start_type))))
        return ADASCALE_ERR_ALIGNMENT;
    const int sms = sm_count();
    if (sms <= 0) return ADASCALE_ERR_CUDA;
    PositionArgs p = {};
    fill_common(p, a);
    p.s = a.scores;
    p.out = a.probs;
    p.table = a.table;
    p.ld_table = a.ld_table;
    p.s_at = used(a, a.scores_stride_b, a.scores_stride_h, a.scores_stride_q);
    p.out_at = used(a, a.probs_stride_b, a.probs_stride_h, a.probs_stride_q);
    p.s_span = span_of(a, p.s_at);
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    if (a.dtype == ADASCALE_BF16) OPS_CU(pick_softmax<bf16>(p, (int)a.heads, sms, s));
    else OPS_CU(pick_softmax<float>(p, (int)a.heads, sms, s));
    return ADASCALE_OK;
}

extern "C" int64_t adascale_position_softmax_grad_workspace(int64_t heads, int64_t n_buckets)
{
    if (heads < 0 || heads > 65535 || n_buckets < 2 || n_buckets > ADASCALE_POSITION_MAX_BUCKETS) return 0;
    // the sums of every block
    return 4 * n_buckets * std::max<long long>(1, heads * std::max<long long>(1, kBlocksMax / std::max<int64_t>(heads, 1)));
}

extern "C" adascale_status adascale_position_softmax_grad(const adascale_position_softmax_grad_args *args, void *cuda_stream)
{
    if (!args) return ADASCALE_ERR_INVALID_ARG;
    const adascale_position_softmax_grad_args &a = *args;
    const adascale_status bad = check_common(a);
    if (bad != ADASCALE_OK) return bad;
    if ((!a.dscores && !a.dtable) || (a.dtable && (!is_dtype(a.wgrad_dtype) || a.ld_dtable < a.heads || !a.workspace ||
                                                   a.workspace_bytes < adascale_position_softmax_grad_workspace(a.heads, a.n_buckets))) ||
        !readable(a.probs_stride_b, a.probs_stride_h, a.probs_stride_q) || !readable(a.dprobs_stride_b, a.dprobs_stride_h, a.dprobs_stride_q) ||
        (a.dscores && !writable(a, a.dscores_stride_b, a.dscores_stride_h, a.dscores_stride_q)))
        return ADASCALE_ERR_INVALID_ARG;
    const bool nothing = a.batch == 0 || a.n_queries == 0 || a.n_keys == 0;
    if (a.heads == 0 || (nothing && (!a.dtable || a.accumulate))) return ADASCALE_OK;
    if (!nothing && (!a.probs || !a.dprobs)) return ADASCALE_ERR_INVALID_ARG;
    const auto other = [&](long long sb, long long sh, long long sq) {
        return sb != a.dscores_stride_b || sh != a.dscores_stride_h || sq != a.dscores_stride_q;
    };
    if (a.dscores && ((a.dscores == a.probs && other(a.probs_stride_b, a.probs_stride_h, a.probs_stride_q)) ||
                      (a.dscores == a.dprobs && other(a.dprobs_stride_b, a.dprobs_stride_h, a.dprobs_stride_q))))
        return ADASCALE_ERR_INVALID_ARG;
    const int b = elem_bytes(a.dtype);
    if (!on(a.probs, b) || !on(a.dprobs, b) || !on(a.dscores, b) || (a.dtable && (!on(a.dtable, elem_bytes(a.wgrad_dtype)) || !on(a.workspace, 16))) ||
        (a.lengths && !on(a.lengths, id_bytes(a.length_type))) || (a.starts && !on(a.starts, id_bytes(a.start_type))))
        return ADASCALE_ERR_ALIGNMENT;
    const int sms = sm_count();
    if (sms <= 0) return ADASCALE_ERR_CUDA;
    PositionArgs p = {};
    fill_common(p, a);
    p.s = a.probs;
    p.dp = a.dprobs;
    p.out = a.dscores;
    p.partials = a.dtable ? static_cast<float *>(a.workspace) : nullptr;
    p.s_at = used(a, a.probs_stride_b, a.probs_stride_h, a.probs_stride_q);
    p.dp_at = used(a, a.dprobs_stride_b, a.dprobs_stride_h, a.dprobs_stride_q);
    p.out_at = used(a, a.dscores_stride_b, a.dscores_stride_h, a.dscores_stride_q);
    p.s_span = span_of(a, p.s_at);
    p.dp_span = span_of(a, p.dp_at);
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    if (!nothing) {
        if (a.dtype == ADASCALE_BF16) OPS_CU(pick_grad<bf16>(p, (int)a.heads, sms, s));
        else OPS_CU(pick_grad<float>(p, (int)a.heads, sms, s));
    }
    if (!a.dtable) return ADASCALE_OK;
    JoinArgs j = {p.partials, a.dtable, a.ld_dtable, (int)a.heads, a.n_buckets, nothing ? 0 : p.chunks, a.accumulate != 0};
    const long long blocks = ceil_div(a.heads * a.n_buckets, 8);
    if (a.wgrad_dtype == ADASCALE_BF16) OPS_CU(launch(k_join_buckets<bf16>, blocks, 256, 0, s, j));
    else OPS_CU(launch(k_join_buckets<float>, blocks, 256, 0, s, j));
    return ADASCALE_OK;
}
