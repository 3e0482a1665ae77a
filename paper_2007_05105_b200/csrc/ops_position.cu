// Attention weights with a learned bias by relative position, and their gradient.
//
//   p = softmax over the live keys of  scale s + table[bucket(j - pos_i), h]
//   g = p (dp - sum p dp),   ds = scale g,   dtable[k, h] = sum of g over bucket k
//
// One pass over the data: a group of threads (8 lanes, a warp, or a block, by the length of a row) holds a row in registers
// between the maximum, the sum and the result.  Bound by memory.  The bias is never in memory: a block works on one head, keeps
// that head's table column and the bucket of every distance up to max_distance in shared memory, and asks for the buckets of the
// first and the last of the 4 or 8 adjacent keys that a thread holds; where they are equal - everywhere but near the
// diagonal - all of them are, since buckets are monotone on either side.  Keys that are not live are not read.
//
// The gradient of the table is summed without atomics: every lane has a column of its own in shared memory (bank = lane), one
// entry a bucket; keys further than max_distance, most of them, are summed in two registers.  Blocks leave their sums, a
// second kernel adds them up in order.
//
// Rows may start anywhere: accesses are cut at 16-byte boundaries of memory, the ragged ends of a row go element by element.
#include "ops_common.cuh"

#include <algorithm>
#include <utility>

namespace {

constexpr int kBordersMax = ADASCALE_POSITION_MAX_BUCKETS / 2;
constexpr long long kMaxLen = 1LL << 29, kMaxStart = 1LL << 30;  // distances stay 32-bit numbers
constexpr int kBlocksMax = 2048;   // of all heads, roughly; the gradient's partial sums are that many times the buckets
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
        k = b.exact;
        for (int i = 0; i < b.n_borders; ++i) k += b.border[i] <= n;
    }
    return k + (b.both && d > 0 ? b.m : 0);
}

// Shared memory: the head's table column, the buckets by distance, the lanes' sums.
struct Tables {
    float *bias;
    unsigned char *bucket;  // of distance d at d + max_distance
    int max_distance;
    __device__ __forceinline__ int at(int d) const
    {
        d = d < -max_distance ? -max_distance : d > max_distance ? max_distance : d;
        return bucket[d + max_distance];
    }
};
__host__ __device__ inline int bucket_bytes(int max_distance) { return (2 * max_distance + 1 + 15) / 16 * 16; }

__device__ __forceinline__ Tables make_tables(const PositionArgs &a, int head, unsigned char *room, bool bias)
{
    Tables t;
    t.max_distance = a.buckets.max_distance;
    t.bucket = room;
    t.bias = reinterpret_cast<float *>(room + bucket_bytes(t.max_distance));
    for (int i = threadIdx.x; i <= 2 * t.max_distance; i += blockDim.x) t.bucket[i] = (unsigned char)bucket_of(a.buckets, i - t.max_distance);
    if (bias)
        for (int i = threadIdx.x; i < a.buckets.n; i += blockDim.x) t.bias[i] = a.table[i * a.ld_table + head];
    return t;
}

// A row: its address in each matrix, the position of its query, and how many keys are live.
struct Row {
    long long b;
    int i, pos, live;
};
__device__ __forceinline__ Row row_of(const PositionArgs &a, long long r, long long end)
{
    Row w = {0, 0, 0, 0};
    if (r >= end) return w;
    w.b = (unsigned)r / (unsigned)a.n_queries;
    w.i = (int)(r - w.b * a.n_queries);
    long long start = a.starts ? load_id(a.starts, a.wide_starts, w.b) : 0;
    start = start < -kMaxStart ? -kMaxStart : start > kMaxStart ? kMaxStart : start;
    w.pos = (int)start + w.i;
    long long live = a.n_keys;
    if (a.lengths) {
        const long long n = load_id(a.lengths, a.wide_lengths, w.b);
        live = n < 0 ? 0 : n < live ? n : live;
    }
    if (a.causal && w.pos < live) live = w.pos < 0 ? 0 : (long long)w.pos + 1 < live ? w.pos + 1 : live;
    w.live = (int)live;
    return w;
}
template <typename T> __device__ __forceinline__ T *row_at(const void *base, const Strides &at, const Row &w, int head)
{
    return static_cast<T *>(const_cast<void *>(base)) + w.b * at.b + head * at.h + w.i * at.q;
}
// Elements by which an address lies behind a 16-byte boundary.
template <typename T> __device__ __forceinline__ int off16(const T *p) { return (int)((uintptr_t)p % 16 / sizeof(T)); }

// Elements c .. c + V - 1 of a row of which [0, end) may be read; others are 0.
template <typename T, int V> __device__ __forceinline__ void load_cols(const T *row, int c, int end, bool aligned, float (&x)[V])
{
    if (aligned && c >= 0 && c + V <= end) {
        load_vec<V>(row + c, x);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) x[e] = c + e >= 0 && c + e < end ? to_f32(row[c + e]) : 0.f;
    }
}
template <typename T, int V> __device__ __forceinline__ void store_cols(T *row, int c, int end, bool aligned, const float (&x)[V])
{
    if (aligned && c >= 0 && c + V <= end) {
        store_vec<V>(row + c, x);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (c + e >= 0 && c + e < end) put(row + c + e, x[e]);
    }
}

// Sum or maximum over the GS threads of a group, the same in each of them.
template <int GS, bool MAX> __device__ __forceinline__ float group_join(float v, float *scratch)
{
    constexpr int kLanes = GS < 32 ? GS : 32;
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1) {
        const float w = __shfl_xor_sync(0xffffffffu, v, o);
        v = MAX ? fmaxf(v, w) : v + w;
    }
    if constexpr (GS > 32) {  // the group is the block; scratch is used in turn, so that one barrier a join is enough
        if (threadIdx.x % 32 == 0) scratch[threadIdx.x / 32] = v;
        __syncthreads();
        v = scratch[threadIdx.x % 32 < GS / 32 ? threadIdx.x % 32 : 0];
        if (!MAX && threadIdx.x % 32 >= GS / 32) v = 0.f;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const float w = __shfl_xor_sync(0xffffffffu, v, o);
            v = MAX ? fmaxf(v, w) : v + w;
        }
    }
    return v;
}

// scale s + bias of V adjacent keys; -inf where not live
template <int V> __device__ __forceinline__ void logits(const Tables &t, const Row &w, int c, float scale, float (&x)[V])
{
    const int d = c - w.pos, first = t.at(d), last = t.at(d + V - 1);
    if (first == last) {
        const float bias = t.bias[first];
#pragma unroll
        for (int e = 0; e < V; ++e) x[e] = fmaf(scale, x[e], bias);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) x[e] = fmaf(scale, x[e], t.bias[t.at(d + e)]);
    }
    if (c < 0 || c + V > w.live) {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (c + e < 0 || c + e >= w.live) x[e] = -INFINITY;
    }
}

// 2^((x - top) log2 e): the difference is taken first, so that large logits lose nothing
__device__ __forceinline__ float exp_of(float x, float top)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"((x - top) * kLog2e));
    return r;
}

// GS threads a row, E elements a thread; LONG: rows of any length, read twice.
template <typename T, int GS, int E, bool LONG>
__global__ void __launch_bounds__(GS > 256 ? GS : 256) k_softmax(const PositionArgs a)
{
    constexpr int V = 16 / sizeof(T), NV = E / V, kThreads = GS > 256 ? GS : 256, kGroups = kThreads / GS;
    extern __shared__ __align__(16) unsigned char room[];
    __shared__ float scratch[3][32];
    griddep_wait();
    griddep_launch();
    const int head = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
    const Tables t = make_tables(a, head, room, true);
    __syncthreads();
    const long long begin = a.rows * chunk / a.chunks, end = a.rows * (chunk + 1) / a.chunks;
    const int group = threadIdx.x / GS, lane = threadIdx.x % GS;
    for (long long r = begin; r < end; r += kGroups) {
        const Row w = row_of(a, r + group, end);
        const int n = r + group < end ? a.n_keys : 0;
        const T *s = row_at<T>(a.s, a.s_at, w, head);
        T *p = row_at<T>(a.out, a.out_at, w, head);
        const int off = off16(s);
        const bool aligned = off16(p) == off;
        if constexpr (!LONG) {
            float x[NV][V], top = -INFINITY, sum = 0.f;
#pragma unroll
            for (int v = 0; v < NV; ++v) load_cols<T, V>(s, (v * GS + lane) * V - off, w.live, true, x[v]);
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                logits<V>(t, w, (v * GS + lane) * V - off, a.scale, x[v]);
#pragma unroll
                for (int e = 0; e < V; ++e) top = fmaxf(top, x[v][e]);
            }
            top = group_join<GS, true>(top, scratch[0]);
            if (top == -INFINITY) top = 0.f;  // nothing is live, all is -inf, or the rest is NaN
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int e = 0; e < V; ++e) sum += x[v][e] = exp_of(x[v][e], top);
            sum = group_join<GS, false>(sum, scratch[1]);
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c = (v * GS + lane) * V - off;
                if (c >= n) break;
#pragma unroll
                for (int e = 0; e < V; ++e) x[v][e] = c + e < w.live ? x[v][e] * inv : 0.f;  // not NaN where not live
                store_cols<T, V>(p, c, n, aligned, x[v]);
            }
            if constexpr (GS > 32) __syncthreads();  // scratch is free for the next row
        } else {
            float top = -INFINITY, sum = 0.f;
            for (int c = lane * V - off; c < w.live; c += GS * V) {
                float x[V], best = top;
                load_cols<T, V>(s, c, w.live, true, x);
                logits<V>(t, w, c, a.scale, x);
#pragma unroll
                for (int e = 0; e < V; ++e) best = fmaxf(best, x[e]);
                const float base = best == -INFINITY ? 0.f : best;
                sum *= exp_of(top == -INFINITY ? base : top, base);
#pragma unroll
                for (int e = 0; e < V; ++e) sum += exp_of(x[e], base);
                top = best;
            }
            float all = group_join<GS, true>(top, scratch[0]);
            if (all == -INFINITY) all = 0.f;
            sum = group_join<GS, false>(sum * exp_of(top == -INFINITY ? all : top, all), scratch[1]);
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            for (int c = lane * V - off; c < n; c += GS * V) {
                float x[V];
                load_cols<T, V>(s, c, w.live, true, x);
                logits<V>(t, w, c, a.scale, x);
#pragma unroll
                for (int e = 0; e < V; ++e) x[e] = c + e < w.live ? exp_of(x[e], all) * inv : 0.f;
                store_cols<T, V>(p, c, n, aligned, x);
            }
            __syncthreads();
        }
    }
}

// ---- gradient ------------------------------------------------------------------------------

// Adds V adjacent values to the lane's sums by bucket.
template <int V> __device__ __forceinline__ void add_buckets(const Tables &t, float *lane_sums, int d, const float (&g)[V], float &behind, float &ahead)
{
    if (d + V - 1 <= -t.max_distance || d >= t.max_distance) {
        float all = 0.f;
#pragma unroll
        for (int e = 0; e < V; ++e) all += g[e];
        if (d < 0) behind += all;
        else ahead += all;
        return;
    }
    const int first = t.at(d), last = t.at(d + V - 1);
    if (first == last) {
        float all = 0.f;
#pragma unroll
        for (int e = 0; e < V; ++e) all += g[e];
        lane_sums[first * 32] += all;
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) lane_sums[t.at(d + e) * 32] += g[e];
    }
}

template <typename T, int GS, int E, bool LONG> __global__ void __launch_bounds__(256) k_softmax_grad(const PositionArgs a)
{
    constexpr int V = 16 / sizeof(T), NV = E / V, kGroups = 256 / GS;
    extern __shared__ __align__(16) unsigned char room[];
    __shared__ float scratch[32];
    griddep_wait();
    if (a.partials) griddep_launch();  // the successor is another kernel of this call
    const int head = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
    const Tables t = make_tables(a, head, room, false);
    float *sums = t.bias;  // [warp][bucket][lane]
    const int n_buckets = a.buckets.n;
    if (a.partials)
        for (int i = threadIdx.x; i < 8 * n_buckets * 32; i += 256) sums[i] = 0.f;
    __syncthreads();
    float *lane_sums = sums + (threadIdx.x / 32) * n_buckets * 32 + threadIdx.x % 32;
    float behind = 0.f, ahead = 0.f;
    const long long begin = a.rows * chunk / a.chunks, end = a.rows * (chunk + 1) / a.chunks;
    const int group = threadIdx.x / GS, lane = threadIdx.x % GS;
    for (long long r = begin; r < end; r += kGroups) {
        const Row w = row_of(a, r + group, end);
        const int n = r + group < end ? a.n_keys : 0;
        const T *p = row_at<T>(a.s, a.s_at, w, head), *dp = row_at<T>(a.dp, a.dp_at, w, head);
        T *ds = row_at<T>(a.out, a.out_at, w, head);
        const int off = off16(p);
        const bool aligned = off16(dp) == off, out_aligned = off16(ds) == off;
        if constexpr (!LONG) {
            float x[NV][V], y[NV][V], dot = 0.f;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                load_cols<T, V>(p, (v * GS + lane) * V - off, w.live, true, x[v]);
                load_cols<T, V>(dp, (v * GS + lane) * V - off, w.live, aligned, y[v]);
            }
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int e = 0; e < V; ++e) dot = fmaf(x[v][e], y[v][e], dot);
            dot = group_join<GS, false>(dot, scratch);
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c = (v * GS + lane) * V - off;
                if (c >= n) break;
#pragma unroll
                for (int e = 0; e < V; ++e) x[v][e] = c + e >= 0 && c + e < w.live ? x[v][e] * (y[v][e] - dot) : 0.f;
                if (a.partials && c < w.live) add_buckets<V>(t, lane_sums, c - w.pos, x[v], behind, ahead);
                if (a.out) {
#pragma unroll
                    for (int e = 0; e < V; ++e) x[v][e] *= a.scale;
                    store_cols<T, V>(ds, c, n, out_aligned, x[v]);
                }
            }
        } else {
            float dot = 0.f;
            for (int c = lane * V - off; c < w.live; c += GS * V) {
                float x[V], y[V];
                load_cols<T, V>(p, c, w.live, true, x);
                load_cols<T, V>(dp, c, w.live, aligned, y);
#pragma unroll
                for (int e = 0; e < V; ++e) dot = fmaf(x[e], y[e], dot);
            }
            dot = group_join<GS, false>(dot, scratch);
            for (int c = lane * V - off; c < n; c += GS * V) {
                float x[V], y[V];
                load_cols<T, V>(p, c, w.live, true, x);
                load_cols<T, V>(dp, c, w.live, aligned, y);
#pragma unroll
                for (int e = 0; e < V; ++e) x[e] = c + e >= 0 && c + e < w.live ? x[e] * (y[e] - dot) : 0.f;
                if (a.partials && c < w.live) add_buckets<V>(t, lane_sums, c - w.pos, x, behind, ahead);
                if (a.out) {
#pragma unroll
                    for (int e = 0; e < V; ++e) x[e] *= a.scale;
                    store_cols<T, V>(ds, c, n, out_aligned, x);
                }
            }
        }
        if constexpr (GS > 32) __syncthreads();  // scratch is free for the next row
    }
    if (!a.partials) return;
    lane_sums[t.at(-t.max_distance) * 32] += behind;
    lane_sums[t.at(t.max_distance) * 32] += ahead;
    __syncthreads();
    // a warp adds up a bucket: lane by lane over the warps, then over the lanes
    for (int k = threadIdx.x / 32; k < n_buckets; k += 8) {
        float v = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) v += sums[(i * n_buckets + k) * 32 + threadIdx.x % 32];
        v = warp_sum(v);
        if (threadIdx.x % 32 == 0) a.partials[((long long)head * n_buckets + k) * a.chunks + chunk] = v;
    }
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

// Head by head, in chunks of rows: enough blocks to fill the device several times over, fewer where there are few rows.
int chunks_of(long long rows, long long heads, int groups, int sms, int blocks_per_sm)
{
    const long long want = ceil_div((long long)sms * blocks_per_sm, heads), most = std::max<long long>(1, kBlocksMax / heads);
    return (int)std::max<long long>(1, std::min(std::min(want, most), ceil_div(rows, groups)));
}

template <typename T, int GS, int E, bool LONG> cudaError_t run_softmax(PositionArgs &a, int heads, int sms, cudaStream_t s)
{
    static OncePerDevice known;
    constexpr int kThreads = GS > 256 ? GS : 256;
    cudaError_t e = allow_smem(reinterpret_cast<const void *>(&k_softmax<T, GS, E, LONG>), known);
    if (e != cudaSuccess) return e;
    a.chunks = chunks_of(a.rows, heads, kThreads / GS, sms, 2048 / kThreads);
    const size_t smem = bucket_bytes(a.buckets.max_distance) + 4 * (size_t)a.buckets.n;
    return launch(k_softmax<T, GS, E, LONG>, (long long)heads * a.chunks, kThreads, smem, s, a);
}
// The elements that a row's group has to hold: with rows off 16-byte boundaries up to V - 1 before it too.
template <typename T> long long held(const PositionArgs &a)
{
    constexpr long long V = 16 / (long long)sizeof(T);
    const bool aligned = on(a.s, 16) && a.s_at.b % V == 0 && a.s_at.h % V == 0 && a.s_at.q % V == 0;
    return a.n_keys + (aligned ? 0 : V - 1);
}
// The narrowest group whose registers hold a row.
template <typename T> cudaError_t pick_softmax(PositionArgs &a, int heads, int sms, cudaStream_t s)
{
    const long long n = held<T>(a);
    if (n <= 8 * 8) return run_softmax<T, 8, 8, false>(a, heads, sms, s);
    if (n <= 8 * 16) return run_softmax<T, 8, 16, false>(a, heads, sms, s);
    if (n <= 32 * 8) return run_softmax<T, 32, 8, false>(a, heads, sms, s);
    if (n <= 32 * 16) return run_softmax<T, 32, 16, false>(a, heads, sms, s);
    if (n <= 32 * 32) return run_softmax<T, 32, 32, false>(a, heads, sms, s);
    if (n <= 256 * 8) return run_softmax<T, 256, 8, false>(a, heads, sms, s);
    if (n <= 256 * 16) return run_softmax<T, 256, 16, false>(a, heads, sms, s);
    if (n <= 256 * 32) return run_softmax<T, 256, 32, false>(a, heads, sms, s);
    if (n <= 1024 * 32) return run_softmax<T, 1024, 32, false>(a, heads, sms, s);
    return run_softmax<T, 1024, 8, true>(a, heads, sms, s);
}

template <typename T, int GS, int E, bool LONG> cudaError_t run_grad(PositionArgs &a, int heads, int sms, cudaStream_t s)
{
    static OncePerDevice known;
    cudaError_t e = allow_smem(reinterpret_cast<const void *>(&k_softmax_grad<T, GS, E, LONG>), known);
    if (e != cudaSuccess) return e;
    a.chunks = chunks_of(a.rows, heads, 256 / GS, sms, 8);
    const size_t smem = bucket_bytes(a.buckets.max_distance) + (a.partials ? 8 * 128 * (size_t)a.buckets.n : 0);
    return launch(k_softmax_grad<T, GS, E, LONG>, (long long)heads * a.chunks, 256, smem, s, a);
}
template <typename T> cudaError_t pick_grad(PositionArgs &a, int heads, int sms, cudaStream_t s)
{
    const long long n = held<T>(a);
    if (n <= 8 * 8) return run_grad<T, 8, 8, false>(a, heads, sms, s);
    if (n <= 8 * 16) return run_grad<T, 8, 16, false>(a, heads, sms, s);
    if (n <= 32 * 8) return run_grad<T, 32, 8, false>(a, heads, sms, s);
    if (n <= 32 * 16) return run_grad<T, 32, 16, false>(a, heads, sms, s);
    if (n <= 32 * 32) return run_grad<T, 32, 32, false>(a, heads, sms, s);
    if (n <= 256 * 8) return run_grad<T, 256, 8, false>(a, heads, sms, s);
    if (n <= 256 * 16) return run_grad<T, 256, 16, false>(a, heads, sms, s);
    if (n <= 256 * 32) return run_grad<T, 256, 32, false>(a, heads, sms, s);
    return run_grad<T, 256, 8, true>(a, heads, sms, s);
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
    p.s_at = {a.scores_stride_b, a.scores_stride_h, a.scores_stride_q};
    p.out_at = {a.probs_stride_b, a.probs_stride_h, a.probs_stride_q};
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
    p.s_at = {a.probs_stride_b, a.probs_stride_h, a.probs_stride_q};
    p.dp_at = {a.dprobs_stride_b, a.dprobs_stride_h, a.dprobs_stride_q};
    p.out_at = {a.dscores_stride_b, a.dscores_stride_h, a.dscores_stride_q};
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
