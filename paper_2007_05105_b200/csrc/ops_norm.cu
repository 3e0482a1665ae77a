// Block boundary: norm of a block's output, gate, residual scale, norm of the stream for the next
// block, and its gradient (adascale_residual_norm, adascale_residual_norm_grad).
//
// With n = (v - mean) r, r = 1 / sqrt(var + eps) (RMS: mean = 0) and dn = dout * w, the gradient of a norm is
//   dv = r [ dn - n mean(dn n) - mean(dn) ]          (RMS: without the last term)
// so both directions of a row need its elements and a handful of sums over them.
//
// Both kernels are bound by memory: every array is read or written once, and a row's elements
// stay in registers between the sums.  A row belongs to a group of threads: a warp with up to 40 (gradient: 16)
// elements a lane, which needs no barrier, or a block of as many warps as the row fills; persistent groups walk over
// the rows.  In the gradient, and forward where it pays, the next row of every array
// arrives in shared memory by one bulk copy each while the group works on the current one.  What had
// to be brought down is the number of instructions: with 8 elements a thread, plain loads and the
// kinds of matrix and row told apart at run time, a row of 1024 cost 2400 warp instructions forward and 3500 backward
// (the SM issues at most 2100 and 3100 in the time that the row's bytes take).  Hence work on packed pairs, many
// elements a thread, kernels compiled for the types and for how far rows fill their groups.
#include "ops_common.cuh"

namespace {

constexpr int kSums = 5;            // dw_pre, db_pre, dw_post, db_post, dgate
enum { kDwPre, kDbPre, kDwPost, kDbPost, kDgate };
constexpr int kStages = 2;
constexpr size_t kStageMost = 224 * 1024;  // bytes of stages in a block, at most

struct Rows {
    char *p;
    long long pitch;  // bytes between rows
    int is_bf16;
    __device__ __forceinline__ char *row(long long r) const { return p + r * pitch; }
};

// Types of the stream and of the block's side that a kernel is compiled for; kAny: told apart at run time.
enum { kF32 = 0, kBf16 = 1, kAny = 2 };
template <int T> __device__ __forceinline__ bool is_bf16(const Rows &m)
{
    if constexpr (T == kAny) return m.is_bf16;
    return T == kBf16;
}

__host__ __device__ constexpr int sure_of(int e) { return e - (e > 16 ? 8 : 4); }

// A thread's elements are E / V sets of V adjacent ones: set j starts at column (j * stride + t) * V.  V = 4 where
// rows start on 16-byte boundaries (16 or 8 bytes an access, adjacent over the lanes), 1 otherwise.  How far the group's
// places are filled: kFull, the row has exactly as many columns; kMostly, only the last 4 (E > 16: 8) elements of a
// thread can lie beyond the row, and the others are not asked (with all of them asked a gradient of 16800000 elements took
// 102 us at 768 columns, 70 so); kAsk, any may.  The sets of a thread are as far apart as its group has threads; with kAsk
// each warp has adjacent columns, so that the distance is a constant.  Elements are kept as pairs.
enum { kAsk, kMostly, kFull };
template <int E, int V, int FILL> struct Place {
    static constexpr int kSure = FILL == kFull ? E : FILL == kMostly ? sure_of(E) : 0;
    int stride, t, dim;
    __device__ __forceinline__ int column(int j) const { return (j * stride + t) * V; }
    __device__ __forceinline__ bool has(int j) const { return (j + 1) * V <= kSure || column(j) < dim; }
};

// Groups: a warp (any number of them in a block, each for itself), a block of a number of threads that is
// known at compile time, or kBlock, a block of any number of warps.
constexpr int kBlock = 0;
template <int E, int V, int FILL, int GROUP> __device__ __forceinline__ Place<E, V, FILL> place_of(int dim)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if constexpr (GROUP == 32) return {32, lane, dim};
    else if constexpr (FILL == kAsk) return {32, warp * (32 * E / V) + lane, dim};
    else return {GROUP == kBlock ? (int)blockDim.x : GROUP, (int)threadIdx.x, dim};
}

// The thread's elements of the row at p; those that it does not have become `none`.
template <int E, int V, int FILL> __device__ __forceinline__ void read(const Place<E, V, FILL> &at, const char *p, bool bf, f2 (&x)[E / 2], float none = 0.f)
{
    if constexpr (V == 4) {
#pragma unroll
        for (int j = 0; j < E / 4; ++j) {
            if (!at.has(j)) {
                x[2 * j] = x[2 * j + 1] = pack2(none, none);
            } else if (bf) {
                const uint2 q = *reinterpret_cast<const uint2 *>(p + (unsigned)at.column(j) * 2);
                x[2 * j] = pack2(bf_lo(q.x), bf_hi(q.x));
                x[2 * j + 1] = pack2(bf_lo(q.y), bf_hi(q.y));
            } else {
                const float4 q = *reinterpret_cast<const float4 *>(p + (unsigned)at.column(j) * 4);
                x[2 * j] = pack2(q.x, q.y);
                x[2 * j + 1] = pack2(q.z, q.w);
            }
        }
    } else {
        float v[E];
#pragma unroll
        for (int j = 0; j < E; ++j) {
            v[j] = none;
            if (at.has(j)) v[j] = bf ? to_f32(reinterpret_cast<const bf16 *>(p)[at.column(j)]) : reinterpret_cast<const float *>(p)[at.column(j)];
        }
#pragma unroll
        for (int i = 0; i < E / 2; ++i) x[i] = pack2(v[2 * i], v[2 * i + 1]);
    }
}
// The thread's columns of a float32 vector.
template <int E, int V, int FILL> __device__ __forceinline__ void read(const Place<E, V, FILL> &at, const float *p, f2 (&x)[E / 2])
{
    read<E, V, FILL>(at, reinterpret_cast<const char *>(p), false, x);
}

template <int E, int V, int FILL> __device__ __forceinline__ void write(const Place<E, V, FILL> &at, char *p, bool bf, const f2 (&x)[E / 2])
{
    float v[E];
#pragma unroll
    for (int i = 0; i < E / 2; ++i) unpack2(x[i], v[2 * i], v[2 * i + 1]);
#pragma unroll
    for (int j = 0; j < E / V; ++j) {
        if (!at.has(j)) continue;
        if constexpr (V == 4) {
            const float *s = v + 4 * j;
            if (bf) *reinterpret_cast<uint2 *>(p + (size_t)at.column(j) * 2) = make_uint2(bf_pack(s[0], s[1]), bf_pack(s[2], s[3]));
            else *reinterpret_cast<float4 *>(p + (size_t)at.column(j) * 4) = make_float4(s[0], s[1], s[2], s[3]);
        } else {
            if (bf) put(reinterpret_cast<bf16 *>(p) + at.column(j), v[j]);
            else put(reinterpret_cast<float *>(p) + at.column(j), v[j]);
        }
    }
}

template <int E> __device__ __forceinline__ void fill(f2 (&x)[E / 2], float v)
{
#pragma unroll
    for (int i = 0; i < E / 2; ++i) x[i] = pack2(v, v);
}

// Sums of two values over the lanes of a warp: the first exchange halves the work by sending each half of
// the warp one of the two.  Lanes 0-15 end up with the first sum, lanes 16-31 with the second.
__device__ __forceinline__ float warp_sum_pair(float a, float b, int lane)
{
    const bool upper = lane & 16;
    float mine = upper ? b : a;
    mine += __shfl_xor_sync(0xffffffffu, upper ? a : b, 16);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
    return mine;
}

__host__ __device__ constexpr int scratch_warps(int group, int most) { return group == kBlock ? (most / 32 + 3) / 4 * 4 : group / 32; }

// Sums over a row's group; in a block with one barrier (consecutive calls use alternate halves of the scratch,
// which has zeros where the block has no warp).
template <int GROUP, int WARPS> struct GroupSum {
    float (*scratch)[WARPS][2];  // [2]
    int turn;

    __device__ __forceinline__ void operator()(float &a, float &b)
    {
        const int lane = threadIdx.x & 31;
        const float mine = warp_sum_pair(a, b, lane);
        if constexpr (GROUP == 32) {
            a = __shfl_sync(0xffffffffu, mine, 0);
            b = __shfl_sync(0xffffffffu, mine, 16);
        } else {
            if ((lane & 15) == 0) scratch[turn][threadIdx.x >> 5][lane >> 4] = mine;
            __syncthreads();
            if constexpr (GROUP != kBlock) {
                const float2 v = *reinterpret_cast<const float2 *>(scratch[turn][lane & (WARPS - 1)]);
                a = v.x;
                b = v.y;
#pragma unroll
                for (int o = WARPS / 2; o > 0; o >>= 1) {
                    a += __shfl_xor_sync(0xffffffffu, a, o);
                    b += __shfl_xor_sync(0xffffffffu, b, o);
                }
            } else if (blockDim.x <= 128) {
                const float4 *two = reinterpret_cast<const float4 *>(scratch[turn]);
                const float4 p = two[0], q = two[1];
                a = p.x + p.z + (q.x + q.z);
                b = p.y + p.w + (q.y + q.w);
            } else {
                const float2 v = lane < WARPS ? *reinterpret_cast<const float2 *>(scratch[turn][lane]) : make_float2(0.f, 0.f);
                const float sum = warp_sum_pair(v.x, v.y, lane);
                a = __shfl_sync(0xffffffffu, sum, 0);
                b = __shfl_sync(0xffffffffu, sum, 16);
            }
            turn ^= 1;
        }
    }
    __device__ __forceinline__ void operator()(float &a)
    {
        if constexpr (GROUP == 32) {
            a = warp_sum(a);
        } else {
            float none = 0.f;
            (*this)(a, none);
        }
    }
};

template <int E> __device__ __forceinline__ float total(const f2 (&v)[E / 2])
{
    f2 s = v[0];
#pragma unroll
    for (int i = 1; i < E / 2; ++i) s = add2(s, v[i]);
    float a, b;
    unpack2(s, a, b);
    return a + b;
}
template <int E> __device__ __forceinline__ float products(const f2 (&v)[E / 2], const f2 (&w)[E / 2])
{
    f2 s = mul2(v[0], w[0]);
#pragma unroll
    for (int i = 1; i < E / 2; ++i) s = fma2(v[i], w[i], s);
    float a, b;
    unpack2(s, a, b);
    return a + b;
}
// v - mean; elements that the thread does not have stay 0.
template <int E, int V, int FILL> __device__ __forceinline__ void centre(const Place<E, V, FILL> &at, f2 (&v)[E / 2], float mean)
{
    const f2 m = pack2(-mean, -mean);
#pragma unroll
    for (int i = 0; i < E / 2; ++i) v[i] = add2(v[i], m);
    if constexpr (FILL != kFull) {
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
            float a, b;
            unpack2(v[i], a, b);
            v[i] = pack2(at.has(2 * i / V) ? a : 0.f, at.has((2 * i + 1) / V) ? b : 0.f);
        }
    }
}
template <int E> __device__ __forceinline__ void scale(f2 (&v)[E / 2], float s)
{
    const f2 q = pack2(s, s);
#pragma unroll
    for (int i = 0; i < E / 2; ++i) v[i] = mul2(v[i], q);
}
template <int E> __device__ __forceinline__ void times(f2 (&v)[E / 2], const f2 (&w)[E / 2])
{
#pragma unroll
    for (int i = 0; i < E / 2; ++i) v[i] = mul2(v[i], w[i]);
}
template <int E> __device__ __forceinline__ void plus(f2 (&v)[E / 2], const f2 (&w)[E / 2])
{
#pragma unroll
    for (int i = 0; i < E / 2; ++i) v[i] = add2(v[i], w[i]);
}
template <int E> __device__ __forceinline__ void sigmoids(f2 (&v)[E / 2])
{
#pragma unroll
    for (int i = 0; i < E / 2; ++i) {
        float a, b;
        unpack2(v[i], a, b);
        v[i] = pack2(1.f / (1.f + __expf(-a)), 1.f / (1.f + __expf(-b)));
    }
}

// The rows of a group in shared memory, kStages at a time: the arrays of a row one after another.  One thread
// of the group asks for them; a stage is asked for again after a barrier of the group behind its last read.
// A copy that does not arrive within the wait's bound is given up: the group stops, and its results from that row on
// become NaN.
struct Stages {
    char *base;       // the group's
    u64 *full;        // [kStages]
    unsigned bytes;   // of a row, all arrays
    template <int N> __device__ __forceinline__ void request(const Rows *const (&arrays)[N], long long row, int dim, int stage) const
    {
        mbar_expect_tx(full + stage, bytes);
        char *to = base + stage * bytes;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            if (!arrays[k]->p) continue;
            const unsigned part = (unsigned)dim * (arrays[k]->is_bf16 ? 2 : 4);
            bulk_load(to, arrays[k]->row(row), part, full + stage);
            to += part;
        }
    }
};

// In the gradient: the row at which each group of a block gave up; kNone as a rule.  What follows a group's rows asks for it, so
// that nothing of it is alive in the walk over them.  (With NaN written in the walk, kernels of 512 threads spilled 700 bytes for 424.)
template <int GROUPS> struct Lost {
    static constexpr u64 kNone = ~0ull;
    u64 row[GROUPS];
    __device__ __forceinline__ void from(int group, long long r) { atomicMin(row + group, (u64)r); }
    __device__ __forceinline__ bool any() const
    {
        bool some = false;
        for (int q = 0; q < GROUPS; ++q) some |= row[q] != kNone;
        return some;
    }
};
__device__ __noinline__ void poison(const Rows &m, u64 row, long long n, long long step, int dim, int t, int threads)
{
    for (long long r = (long long)row; m.p && r < n; r += step)
        for (int c = t; c < dim; c += threads) {
            if (m.is_bf16) put(reinterpret_cast<bf16 *>(m.row(r)) + c, __int_as_float(0x7fffffff));
            else put(reinterpret_cast<float *>(m.row(r)) + c, __int_as_float(0x7fffffff));
        }
}

template <int GROUP> __device__ __forceinline__ void group_barrier()
{
    if constexpr (GROUP == 32) __syncwarp();
    else __syncthreads();
}

struct NormArgs {
    Rows x, y, x_new, h, gate;  // y.p null: the norm alone
    const float *gate_channel, *w_post, *b_post, *w_pre, *b_pre;
    long long n;
    int dim;
    int post, pre, gate_kind;
    unsigned stage_bytes;
    unsigned weight_bytes;  // of the vectors' copies in shared memory; 0: read where they are
    float inv_dim, res_scale, eps;
};

// Threads that an SM holds: as many as leave one the registers that it needs for its elements.  Gradient, 16384 x 1024
// (f32 stream, bf16 block, layer norms, channel gate), E = 16: 384 threads (168 registers) 61 us, 512 (128) 81.  Forward,
// E = 24: rows of 640 columns by warps, 640 threads 41 us, 512 46; of 1280 by blocks, 640 threads 54 us, 512 51.
__host__ __device__ constexpr int forward_threads(int e, int group) { return e > 32 ? 384 : e > 24 ? 512 : e > 16 ? group == 32 ? 640 : 512 : e > 8 ? 768 : 1024; }
__host__ __device__ constexpr int gradient_threads(int e) { return e > 12 ? 384 : e > 8 ? 512 : e > 4 ? 640 : 896; }
constexpr int kGradientBlock = 128;  // of a block whose warps are groups of their own

// Rows by bulk copies ahead of the work where both types are bf16 and a row is a warp's (16384 x 1024: 28 us against
// 32); otherwise each row is loaded when its turn comes (f32 stream: 39 us against 42; 16384 x 2048: 74 against 83).
template <int XT, int YT, int V, int GROUP> __host__ __device__ constexpr bool forward_staged()
{
    return V == 4 && GROUP == 32 && XT == kBf16 && YT == kBf16;
}

template <int XT, int YT, int V, int FILL, int GROUP, int E>
__global__ void __launch_bounds__(forward_threads(E, GROUP), 1) k_boundary(const __grid_constant__ NormArgs a)
{
    constexpr int kMostWarps = forward_threads(E, GROUP) / 32, kScratch = scratch_warps(GROUP, forward_threads(E, GROUP));
    constexpr bool kWarp = GROUP == 32, kStaged = forward_staged<XT, YT, V, GROUP>();
    extern __shared__ __align__(128) char room[];
    __shared__ __align__(16) float scratch[2][kScratch][2];
    __shared__ u64 full[kStaged ? kMostWarps : 1][kStages];
    const int mine = kWarp ? threadIdx.x / 32 : 0, groups = kWarp ? blockDim.x / 32 : 1;
    const Place<E, V, FILL> at = place_of<E, V, FILL, GROUP>(a.dim);
    const long long all = (long long)gridDim.x * groups;
    const Stages stages = {room + a.weight_bytes + mine * kStages * a.stage_bytes, full[kStaged ? mine : 0], a.stage_bytes};
    GroupSum<GROUP, kScratch> sum = {scratch, 0};
    for (int i = threadIdx.x; GROUP == kBlock && i < 4 * kScratch; i += blockDim.x) (&scratch[0][0][0])[i] = 0.f;
    long long row = (long long)blockIdx.x * groups + mine;
    if (kStaged && at.t == 0) {
        for (int s = 0; s < kStages; ++s) mbar_init(stages.full + s, 1);
        mbar_publish();
    }
    group_barrier<GROUP>();
    griddep_wait();
    griddep_launch();
    const float *w_post = a.w_post, *b_post = a.b_post, *channel = a.gate_channel, *w_pre = a.w_pre, *b_pre = a.b_pre;
    if (a.weight_bytes) {  // many rows: the vectors over the columns in shared memory
        float *at_room = reinterpret_cast<float *>(room);
        const float **all_of_them[5] = {&w_post, &b_post, &channel, &w_pre, &b_pre};
#pragma unroll
        for (int k = 0; k < 5; ++k) {
            const float *&w = *all_of_them[k];
            if (!w) continue;
            for (int c = threadIdx.x; c < a.dim; c += blockDim.x) at_room[c] = w[c];
            w = at_room;
            at_room += (a.dim + 3) / 4 * 4;
        }
        __syncthreads();
    }
    const Rows *const arrays[3] = {&a.x, &a.y, &a.gate};
    if (kStaged && at.t == 0)
        for (int s = 0; s < kStages; ++s)
            if (row + s * all < a.n) stages.request(arrays, row + s * all, a.dim, s);
    int stage = 0;
    unsigned parity = 0;
    for (; row < a.n; row += all) {
        const char *px = a.x.row(row), *py = a.y.row(row), *pg = a.gate.row(row);
        if constexpr (kStaged) {
            if (!mbar_wait(stages.full + stage, parity)) {
                mbar_wait(stages.full + (stage ^ 1), parity ^ (stage == 1));  // the other copy in flight
                f2 lost[E / 2];
                fill<E>(lost, __int_as_float(0x7fffffff));
                for (; row < a.n; row += all) {
                    if (a.y.p) write<E, V, FILL>(at, a.x_new.row(row), is_bf16<XT>(a.x_new), lost);
                    write<E, V, FILL>(at, a.h.row(row), is_bf16<YT>(a.h), lost);
                }
                break;
            }
            px = stages.base + stage * stages.bytes;
            py = px + a.dim * (is_bf16<XT>(a.x) ? 2 : 4);
            pg = py + a.dim * (is_bf16<YT>(a.y) ? 2 : 4);
        }
        f2 x[E / 2], y[E / 2], w[E / 2];
        float s;
        read<E, V, FILL>(at, px, is_bf16<XT>(a.x), x);
        if (a.y.p) {
            read<E, V, FILL>(at, py, is_bf16<YT>(a.y), y);
            if (a.post != ADASCALE_NORM_NONE) {
                if (a.post == ADASCALE_NORM_LAYER) {
                    s = total<E>(y);
                    sum(s);
                    centre<E, V, FILL>(at, y, s * a.inv_dim);
                }
                s = products<E>(y, y);
                sum(s);
                scale<E>(y, rsqrtf(fmaf(s, a.inv_dim, a.eps)));
                read<E, V, FILL>(at, w_post, w);
                times<E>(y, w);
                if (b_post) {
                    read<E, V, FILL>(at, b_post, w);
                    plus<E>(y, w);
                }
            }
            if (a.gate_kind != ADASCALE_GATE_NONE) {
                if (a.gate_kind == ADASCALE_GATE_CHANNEL) {
                    read<E, V, FILL>(at, channel, w);
                } else {
                    read<E, V, FILL>(at, pg, is_bf16<YT>(a.gate), w);
                    sigmoids<E>(w);
                }
                times<E>(y, w);
            }
            const f2 rs = pack2(a.res_scale, a.res_scale);
#pragma unroll
            for (int i = 0; i < E / 2; ++i) x[i] = fma2(rs, y[i], x[i]);
            write<E, V, FILL>(at, a.x_new.row(row), is_bf16<XT>(a.x_new), x);
        }
        if constexpr (kStaged) {  // everything of the stage has been read
            group_barrier<GROUP>();
            if (at.t == 0 && row + kStages * all < a.n) stages.request(arrays, row + kStages * all, a.dim, stage);
            stage ^= 1;
            parity ^= stage == 0;
        }
        if (a.pre == ADASCALE_NORM_LAYER) {
            s = total<E>(x);
            sum(s);
            centre<E, V, FILL>(at, x, s * a.inv_dim);
        }
        s = products<E>(x, x);
        sum(s);
        scale<E>(x, rsqrtf(fmaf(s, a.inv_dim, a.eps)));
        read<E, V, FILL>(at, w_pre, w);
        times<E>(x, w);
        if (b_pre) {
            read<E, V, FILL>(at, b_pre, w);
            plus<E>(x, w);
        }
        write<E, V, FILL>(at, a.h.row(row), is_bf16<YT>(a.h), x);
    }
}

struct GradArgs {
    Rows x, y, dx_new, dh, gate, dx, dy, dgate;  // absent ones have a null pointer
    const float *gate_channel, *w_post, *b_post, *w_pre;
    float *partial;  // [blocks][kSums][ld_partial]
    long long n;
    int dim, ld_partial;
    int post, pre, gate_kind;
    int followed;  // by k_columns
    unsigned stage_bytes;
    float inv_dim, res_scale, eps;
};

// NaN as the rows' results of the groups that gave up, and as the block's column sums.
template <int GROUPS> __device__ __noinline__ void poison(const GradArgs &a, const Lost<GROUPS> &lost)
{
    for (int q = 0; q < GROUPS; ++q) {
        if (lost.row[q] == lost.kNone) continue;
        const long long step = (long long)gridDim.x * GROUPS;
        poison(a.dx, lost.row[q], a.n, step, a.dim, threadIdx.x, blockDim.x);
        poison(a.dy, lost.row[q], a.n, step, a.dim, threadIdx.x, blockDim.x);
        poison(a.dgate, lost.row[q], a.n, step, a.dim, threadIdx.x, blockDim.x);
    }
    const Rows sums = {reinterpret_cast<char *>(a.partial + (long long)blockIdx.x * kSums * a.ld_partial), a.ld_partial * 4LL, 0};
    poison(sums, 0, kSums, 1, a.dim, threadIdx.x, blockDim.x);
}

// Every thread keeps the column sums of its columns in registers over all its rows; at the end the
// warps of a block are added in order, where they are groups, and the block leaves one row of partial
// sums.  The sums over a row come in pairs (x and y, twice; the two of each norm's gradient): four
// barriers a row, none where a row is one warp's.
template <int XT, int YT, int V, int FILL, int GROUP, int E, int MOST>
__global__ void __launch_bounds__(MOST, 1) k_boundary_grad(const __grid_constant__ GradArgs a)
{
    constexpr int kGroups = GROUP == 32 ? kGradientBlock / 32 : 1, kScratch = scratch_warps(GROUP, MOST);
    constexpr bool kWarp = GROUP == 32, kStaged = V == 4 && XT != kAny;
    extern __shared__ __align__(128) char room[];
    __shared__ __align__(16) float scratch[2][kScratch][2];
    __shared__ u64 full[kGroups][kStages];
    __shared__ Lost<kGroups> lost;
    const int mine = kWarp ? threadIdx.x / 32 : 0;
    const Place<E, V, FILL> at = place_of<E, V, FILL, GROUP>(a.dim);
    const long long all = (long long)gridDim.x * kGroups;
    const Stages stages = {room + mine * kStages * a.stage_bytes, full[mine], a.stage_bytes};
    GroupSum<GROUP, kScratch> sum = {scratch, 0};
    for (int i = threadIdx.x; GROUP == kBlock && i < 4 * kScratch; i += blockDim.x) (&scratch[0][0][0])[i] = 0.f;
    long long row = (long long)blockIdx.x * kGroups + mine;
    if (kStaged && at.t == 0) {
        for (int s = 0; s < kStages; ++s) mbar_init(stages.full + s, 1);
        mbar_publish();
        lost.row[mine] = lost.kNone;
    }
    group_barrier<GROUP>();
    griddep_wait();
    if (a.followed) griddep_launch();
    const Rows *const arrays[5] = {&a.x, &a.dh, &a.dx_new, &a.y, &a.gate};
    if (kStaged && at.t == 0)
        for (int s = 0; s < kStages; ++s)
            if (row + s * all < a.n) stages.request(arrays, row + s * all, a.dim, s);
    const bool has_y = a.y.p != nullptr, arrives = a.dx_new.p != nullptr, post = a.post != ADASCALE_NORM_NONE;
    const bool centre_x = a.pre == ADASCALE_NORM_LAYER, centre_y = has_y && a.post == ADASCALE_NORM_LAYER;
    f2 acc[kSums][E / 2];
#pragma unroll
    for (int k = 0; k < kSums; ++k) fill<E>(acc[k], 0.f);
    int stage = 0;
    unsigned parity = 0;
    for (; row < a.n; row += all) {
        const char *px = a.x.row(row), *ph = a.dh.row(row), *pd = a.dx_new.row(row), *py = a.y.row(row), *pg = a.gate.row(row);
        if constexpr (kStaged) {
            if (!mbar_wait(stages.full + stage, parity)) {
                lost.from(mine, row);
                mbar_wait(stages.full + (stage ^ 1), parity ^ (stage == 1));  // the other copy in flight
                break;
            }
            px = stages.base + stage * stages.bytes;
            ph = px + a.dim * (is_bf16<XT>(a.x) ? 2 : 4);
            pd = ph + a.dim * (is_bf16<YT>(a.dh) ? 2 : 4);
            py = arrives ? pd + a.dim * (is_bf16<XT>(a.dx_new) ? 2 : 4) : pd;
            pg = py + a.dim * (is_bf16<YT>(a.y) ? 2 : 4);
        }
        f2 x[E / 2], y[E / 2], dx[E / 2], dh[E / 2], w[E / 2];
        float s0, s1;
        read<E, V, FILL>(at, px, is_bf16<XT>(a.x), x);
        read<E, V, FILL>(at, ph, is_bf16<YT>(a.dh), dh);
        if (has_y) read<E, V, FILL>(at, py, is_bf16<YT>(a.y), y);
        else fill<E>(y, 0.f);
        if (centre_x || centre_y) {
            s0 = total<E>(x);
            s1 = total<E>(y);
            sum(s0, s1);
            if (centre_x) centre<E, V, FILL>(at, x, s0 * a.inv_dim);
            if (centre_y) centre<E, V, FILL>(at, y, s1 * a.inv_dim);
        }
        s0 = products<E>(x, x);
        s1 = products<E>(y, y);
        sum(s0, s1);
        const float rx = rsqrtf(fmaf(s0, a.inv_dim, a.eps)), ry = post ? rsqrtf(fmaf(s1, a.inv_dim, a.eps)) : 1.f;

        // dx = dx' + pre^T(dh)
        scale<E>(x, rx);
        read<E, V, FILL>(at, a.w_pre, w);
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
            acc[kDwPre][i] = fma2(dh[i], x[i], acc[kDwPre][i]);
            acc[kDbPre][i] = add2(acc[kDbPre][i], dh[i]);
            dh[i] = mul2(dh[i], w[i]);
        }
        s0 = products<E>(dh, x);
        s1 = total<E>(dh);
        sum(s0, s1);
        if (arrives) read<E, V, FILL>(at, pd, is_bf16<XT>(a.dx_new), dx);
        else fill<E>(dx, 0.f);
        {
            const float mean = centre_x ? s1 * a.inv_dim : 0.f;
            const f2 minus = pack2(-mean, -mean), share = pack2(-s0 * a.inv_dim, -s0 * a.inv_dim), r = pack2(rx, rx);
#pragma unroll
            for (int i = 0; i < E / 2; ++i) dx[i] = fma2(r, fma2(x[i], share, add2(dh[i], minus)), dx[i]);
        }
        write<E, V, FILL>(at, a.dx.row(row), is_bf16<XT>(a.dx), dx);

        if (has_y) {  // gate and post; x, dh are free
            if (post) scale<E>(y, ry);
            scale<E>(dx, a.res_scale);
            if (a.gate_kind != ADASCALE_GATE_NONE) {
                f2 (&u)[E / 2] = x;
#pragma unroll
                for (int i = 0; i < E / 2; ++i) u[i] = y[i];
                if (post) {
                    read<E, V, FILL>(at, a.w_post, w);
                    times<E>(u, w);
                    if (a.b_post) {
                        read<E, V, FILL>(at, a.b_post, w);
                        plus<E>(u, w);
                    }
                }
                times<E>(u, dx);  // gradient of the gate
                if (a.gate_kind == ADASCALE_GATE_SIGMOID) {
                    read<E, V, FILL>(at, pg, is_bf16<YT>(a.gate), w);
                    sigmoids<E>(w);
                    if (a.dgate.p) {
                        const f2 one = pack2(1.f, 1.f), minus_one = pack2(-1.f, -1.f);
#pragma unroll
                        for (int i = 0; i < E / 2; ++i) u[i] = mul2(mul2(u[i], w[i]), fma2(w[i], minus_one, one));
                        write<E, V, FILL>(at, a.dgate.row(row), is_bf16<YT>(a.dgate), u);
                    }
                } else {
                    read<E, V, FILL>(at, a.gate_channel, w);
                    plus<E>(acc[kDgate], u);
                }
                times<E>(dx, w);
            }
            if (post) {
                read<E, V, FILL>(at, a.w_post, w);
#pragma unroll
                for (int i = 0; i < E / 2; ++i) {
                    acc[kDwPost][i] = fma2(dx[i], y[i], acc[kDwPost][i]);
                    acc[kDbPost][i] = add2(acc[kDbPost][i], dx[i]);
                    dx[i] = mul2(dx[i], w[i]);
                }
                s0 = products<E>(dx, y);
                s1 = total<E>(dx);
                sum(s0, s1);
                const float mean = centre_y ? s1 * a.inv_dim : 0.f;
                const f2 minus = pack2(-mean, -mean), share = pack2(-s0 * a.inv_dim, -s0 * a.inv_dim), r = pack2(ry, ry);
#pragma unroll
                for (int i = 0; i < E / 2; ++i) dx[i] = mul2(r, fma2(y[i], share, add2(dx[i], minus)));
            }
            if (a.dy.p) write<E, V, FILL>(at, a.dy.row(row), is_bf16<YT>(a.dy), dx);
        }
        if constexpr (kStaged) {
            group_barrier<GROUP>();
            if (at.t == 0 && row + kStages * all < a.n) stages.request(arrays, row + kStages * all, a.dim, stage);
            stage ^= 1;
            parity ^= stage == 0;
        }
    }

    // one set of sums at a time: the block's group, or its warps in order
    char *to = reinterpret_cast<char *>(a.partial + (long long)blockIdx.x * kSums * a.ld_partial);
    float *gather = reinterpret_cast<float *>(room);  // [kGroups][ld_partial]
#pragma unroll
    for (int k = 0; k < kSums; ++k) {
        if constexpr (kGroups == 1) {
            write<E, V, FILL>(at, to + (size_t)k * a.ld_partial * 4, false, acc[k]);
        } else {
            __syncthreads();
            write<E, V, FILL>(at, reinterpret_cast<char *>(gather + mine * a.ld_partial), false, acc[k]);
            __syncthreads();
            for (int c = threadIdx.x; c < a.dim; c += kGradientBlock) {
                float s = gather[c];
                for (int q = 1; q < kGroups; ++q) s += gather[q * a.ld_partial + c];
                reinterpret_cast<float *>(to)[k * a.ld_partial + c] = s;
            }
        }
    }
    if constexpr (kStaged) {
        __syncthreads();
        if (lost.any()) poison(a, lost);
    }
}

struct ColumnArgs {
    const float *partial;
    void *out[kSums];
    int dim, ld_partial, n_partials, bf16_out;
};

// Column sums of the blocks' partial sums, in a fixed order: 32 columns per block, warp q adds rows q, q + 32, ...
constexpr int kColumnWarps = 32;
__global__ void __launch_bounds__(kColumnWarps * 32) k_columns(const __grid_constant__ ColumnArgs a)
{
    __shared__ float part[kColumnWarps][33];
    griddep_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int chunks = (a.dim + 31) / 32, which = blockIdx.x / chunks, c0 = (blockIdx.x % chunks) * 32, c = c0 + lane;
    if (!a.out[which]) return;
    float s = 0.f;
    if (c < a.dim) {
        constexpr int U = 10;
        const float *p = a.partial + (long long)which * a.ld_partial + c;
        const long long pitch = (long long)kSums * a.ld_partial;
        for (int q = warp; q < a.n_partials; q += U * kColumnWarps) {
            float x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) x[u] = q + u * kColumnWarps < a.n_partials ? __ldcg(p + (q + u * kColumnWarps) * pitch) : 0.f;
#pragma unroll
            for (int u = 0; u < U; ++u) s += x[u];
        }
    }
    part[warp][lane] = s;
    __syncthreads();
    s = warp_sum(part[lane][warp]);  // column c0 + warp
    if (lane || c0 + warp >= a.dim) return;
    if (a.bf16_out)
        put(static_cast<bf16 *>(a.out[which]) + c0 + warp, s);
    else
        put(static_cast<float *>(a.out[which]) + c0 + warp, s);
}

// ---- host side -----------------------------------------------------------------------------

constexpr int kMaxPartials = 148 * 16;  // blocks of a gradient launch, at most

// Elements a thread and threads of a row's group.  A warp has a row as long as its elements fit (1280 columns forward,
// bf16: 31 us, by a block 45; with 48 elements a lane 1536 columns of f32 took 49 us, by a block 46); beyond that a
// block of warps, from a list of E and most threads, that leaves the fewest places empty, of equals the
// one with more elements a thread.
struct Split {
    int e, group;
};
template <int N, int M> Split split_of(long long dim, const int (&by_warp)[N], const Split (&by_block)[M])
{
    for (int e : by_warp)
        if (32LL * e >= dim) return {e, 32};
    Split best = {0, 0};
    for (const Split b : by_block) {
        const int g = (int)ceil_div(dim, 32 * b.e) * 32;
        if ((long long)sure_of(b.e) * g <= dim && g <= b.group && (!best.e || b.e * g <= best.e * best.group)) best = {b.e, g};
    }
    return best;
}
Split forward_split(long long dim) { return split_of(dim, {4, 8, 12, 16, 24, 32, 40}, {{24, 512}, {32, 512}}); }
bool power_of_two(long long v) { return v > 0 && !(v & (v - 1)); }

bool norm_kind(int k, bool none_too) { return k == ADASCALE_NORM_RMS || k == ADASCALE_NORM_LAYER || (none_too && k == ADASCALE_NORM_NONE); }

Rows rows(const void *p, long long ld, int dtype)
{
    return {static_cast<char *>(const_cast<void *>(p)), ld * elem_bytes(dtype), dtype == ADASCALE_BF16};
}
unsigned row_bytes(const Rows &m, int dim) { return !m.p ? 0 : (unsigned)dim * (m.is_bf16 ? 2 : 4); }

// Blocks of a persistent launch: `most` an SM, fewer where their stages do not fit.
long long resident(int sms, int most, size_t smem)
{
    const long long fit = (long long)(227 * 1024 / (smem + 1280));
    return (long long)sms * (fit < most ? (fit < 1 ? 1 : fit) : most);
}

// Where a row is a warp's: few rows, blocks of four warps that read the vectors where they are; many rows, blocks that
// fill an SM with a copy of the vectors in shared memory (in L1 they are evicted between rows: 42 us for 39).
template <int XT, int YT, int V, int FILL, int GROUP, int E> cudaError_t launch_boundary(NormArgs a, int group, int sms, cudaStream_t s)
{
    constexpr bool kWarp = GROUP == 32;
    const int vectors = (a.w_post != nullptr) + (a.b_post != nullptr) + (a.gate_channel != nullptr) + 1 + (a.b_pre != nullptr);
    const unsigned copies = (unsigned)(vectors * ((a.dim + 3) / 4 * 4) * sizeof(float));
    const size_t stages = forward_staged<XT, YT, V, GROUP>() ? (size_t)kStages * a.stage_bytes : 0;  // of a group
    int groups = kWarp ? 4 : 1;
    if (kWarp && a.n >= forward_threads(E, GROUP) / 8LL * sms) {
        groups = forward_threads(E, GROUP) / 32;
        a.weight_bytes = copies;
    }
    const size_t smem = groups * stages + a.weight_bytes;
    const long long need = ceil_div(a.n, groups), most = resident(sms, forward_threads(E, GROUP) / (groups * group), smem);
    static OncePerDevice known;
    const cudaError_t e = allow_smem(reinterpret_cast<const void *>(&k_boundary<XT, YT, V, FILL, GROUP, E>), known);
    return e != cudaSuccess ? e : launch(k_boundary<XT, YT, V, FILL, GROUP, E>, need < most ? need : most, groups * group, smem, s, a);
}
template <int XT, int YT, int V, int FILL> cudaError_t launch_by_warp(const NormArgs &a, int e, int sms, cudaStream_t s)
{
    switch (e) {
    case 4: return launch_boundary<XT, YT, V, FILL, 32, 4>(a, 32, sms, s);
    case 8: return launch_boundary<XT, YT, V, FILL, 32, 8>(a, 32, sms, s);
    case 12: return launch_boundary<XT, YT, V, FILL, 32, 12>(a, 32, sms, s);
    case 16: return launch_boundary<XT, YT, V, FILL, 32, 16>(a, 32, sms, s);
    case 24: return launch_boundary<XT, YT, V, FILL, 32, 24>(a, 32, sms, s);
    case 40: return launch_boundary<XT, YT, V, FILL, 32, 40>(a, 32, sms, s);
    }
    return launch_boundary<XT, YT, V, FILL, 32, 32>(a, 32, sms, s);
}
// Rows that fill a power of two: the group's size is a constant (2048 columns 41 us, with kBlock 48).
template <int XT, int YT> cudaError_t launch_by_power(const NormArgs &a, int group, int sms, cudaStream_t s)
{
    switch (group) {
    case 64: return launch_boundary<XT, YT, 4, kFull, 64, 32>(a, group, sms, s);
    case 128: return launch_boundary<XT, YT, 4, kFull, 128, 32>(a, group, sms, s);
    case 256: return launch_boundary<XT, YT, 4, kFull, 256, 32>(a, group, sms, s);
    }
    return launch_boundary<XT, YT, 4, kFull, 512, 32>(a, group, sms, s);
}
template <int XT, int YT, int FILL> cudaError_t launch_by_block(const NormArgs &a, Split p, int sms, cudaStream_t s)
{
    return p.e == 24 ? launch_boundary<XT, YT, 4, FILL, kBlock, 24>(a, p.group, sms, s) : launch_boundary<XT, YT, 4, FILL, kBlock, 32>(a, p.group, sms, s);
}
template <int XT, int YT> cudaError_t launch_boundary(const NormArgs &a, bool vec, int sms, cudaStream_t s)
{
    const Split p = forward_split(a.dim);
    const bool full = p.group * p.e == a.dim;
    if (p.group == 32) {
        if (!vec) return launch_by_warp<XT, YT, 1, kMostly>(a, p.e, sms, s);
        return full ? launch_by_warp<XT, YT, 4, kFull>(a, p.e, sms, s) : launch_by_warp<XT, YT, 4, kMostly>(a, p.e, sms, s);
    }
    // without alignment: 16 elements a thread as long as two blocks fit an SM (f32 stream, 5321 columns: 65 us against
    // 83 with 32; 8191: 83 against 69)
    if (!vec && a.dim <= 16 * forward_threads(16, kBlock) / 2)
        return launch_boundary<XT, YT, 1, kAsk, kBlock, 16>(a, (int)ceil_div(a.dim, 512) * 32, sms, s);
    if (!vec) return launch_boundary<XT, YT, 1, kAsk, kBlock, 32>(a, (int)ceil_div(a.dim, 1024) * 32, sms, s);
    if (power_of_two(a.dim)) return launch_by_power<XT, YT>(a, a.dim / 32, sms, s);
    return full ? launch_by_block<XT, YT, kFull>(a, p, sms, s) : launch_by_block<XT, YT, kMostly>(a, p, sms, s);
}

template <int XT, int YT, int V, int FILL, int GROUP, int E, int MOST>
cudaError_t launch_grad(const GradArgs &a, int group, int sms, cudaStream_t s, int &partials)
{
    constexpr int kGroups = GROUP == 32 ? kGradientBlock / 32 : 1;
    constexpr bool kStaged = V == 4 && XT != kAny;
    const int threads = kGroups * group;
    const long long need = ceil_div(a.n, kGroups);
    size_t smem = kStaged ? (size_t)kGroups * kStages * a.stage_bytes : 0;
    const size_t gather = (size_t)kGroups * a.ld_partial * sizeof(float);
    if (kGroups > 1 && smem < gather) smem = gather;
    long long blocks = resident(sms, MOST / threads, smem);
    if (blocks > kMaxPartials) blocks = kMaxPartials;
    if (blocks > need) blocks = need;
    partials = (int)blocks;
    static OncePerDevice known;
    const cudaError_t e = allow_smem(reinterpret_cast<const void *>(&k_boundary_grad<XT, YT, V, FILL, GROUP, E, MOST>), known);
    return e != cudaSuccess ? e : launch(k_boundary_grad<XT, YT, V, FILL, GROUP, E, MOST>, blocks, threads, smem, s, a);
}
template <int XT, int YT, int V, int FILL> cudaError_t launch_by_warp(const GradArgs &a, int e, int sms, cudaStream_t s, int &partials)
{
    switch (e) {
    case 4: return launch_grad<XT, YT, V, FILL, 32, 4, gradient_threads(4)>(a, 32, sms, s, partials);
    case 8: return launch_grad<XT, YT, V, FILL, 32, 8, gradient_threads(8)>(a, 32, sms, s, partials);
    case 12: return launch_grad<XT, YT, V, FILL, 32, 12, gradient_threads(12)>(a, 32, sms, s, partials);
    }
    return launch_grad<XT, YT, V, FILL, 32, 16, 384>(a, 32, sms, s, partials);
}
template <int XT, int YT> cudaError_t launch_by_power(const GradArgs &a, int group, int sms, cudaStream_t s, int &partials)
{
    switch (group) {
    case 64: return launch_grad<XT, YT, 4, kFull, 64, 16, 384>(a, group, sms, s, partials);
    case 128: return launch_grad<XT, YT, 4, kFull, 128, 16, 384>(a, group, sms, s, partials);
    case 256: return launch_grad<XT, YT, 4, kFull, 256, 16, 256>(a, group, sms, s, partials);
    }
    return launch_grad<XT, YT, 4, kFull, 512, 16, 512>(a, group, sms, s, partials);
}
// Rows that are too wide for stages: one kernel for all types.
template <int V> cudaError_t launch_wide(const GradArgs &a, int group, int sms, cudaStream_t s, int &partials)
{
    if constexpr (V == 4)
        if (group <= 512) return launch_grad<kAny, kAny, V, kAsk, kBlock, 16, 512>(a, group, sms, s, partials);
    return launch_grad<kAny, kAny, V, kAsk, kBlock, 16, 1024>(a, group, sms, s, partials);
}
template <int XT, int YT, int FILL> cudaError_t launch_by_block(const GradArgs &a, Split p, int sms, cudaStream_t s, int &partials)
{
    if (p.e == 12) return launch_grad<XT, YT, 4, FILL, kBlock, 12, 384>(a, p.group, sms, s, partials);
    return p.group <= 384 ? launch_grad<XT, YT, 4, FILL, kBlock, 16, 384>(a, p.group, sms, s, partials)
                          : launch_grad<XT, YT, 4, FILL, kBlock, 16, 512>(a, p.group, sms, s, partials);
}
template <int XT, int YT> cudaError_t launch_grad(const GradArgs &a, bool vec, int sms, cudaStream_t s, int &partials)
{
    const Split p = split_of(a.dim, {4, 8, 12, 16}, {{12, 384}, {16, 512}});
    const bool full = p.group * p.e == a.dim;
    if (p.group == 32) {
        if (!vec) return launch_by_warp<XT, YT, 1, kMostly>(a, p.e, sms, s, partials);
        return full ? launch_by_warp<XT, YT, 4, kFull>(a, p.e, sms, s, partials) : launch_by_warp<XT, YT, 4, kMostly>(a, p.e, sms, s, partials);
    }
    const int group = (int)ceil_div(a.dim, 512) * 32;
    if (!vec) {
        if (group <= 384) return launch_grad<XT, YT, 1, kAsk, kBlock, 16, 384>(a, group, sms, s, partials);
        if (group <= 512) return launch_grad<XT, YT, 1, kAsk, kBlock, 16, 512>(a, group, sms, s, partials);
        return launch_wide<1>(a, group, sms, s, partials);
    }
    if (!p.group || kStages * (size_t)a.stage_bytes > kStageMost) return launch_wide<4>(a, group, sms, s, partials);
    if (power_of_two(a.dim)) return launch_by_power<XT, YT>(a, a.dim / 16, sms, s, partials);
    return full ? launch_by_block<XT, YT, kFull>(a, p, sms, s, partials) : launch_by_block<XT, YT, kMostly>(a, p, sms, s, partials);
}

}  // namespace

extern "C" {

adascale_status adascale_residual_norm(const adascale_residual_norm_args *g, void *cuda_stream)
{
    if (!g || g->n_rows < 0 || g->dim < 1 || !is_dtype(g->x_dtype) || !is_dtype(g->y_dtype) || !norm_kind(g->pre, false) ||
        !norm_kind(g->post, true) || g->gate_kind < ADASCALE_GATE_NONE || g->gate_kind > ADASCALE_GATE_SIGMOID ||
        !std::isfinite(g->res_scale) || !(g->eps >= 0.f) || !std::isfinite(g->eps))
        return ADASCALE_ERR_INVALID_ARG;
    if (g->n_rows > kMaxRows || g->dim > ADASCALE_NORM_MAX_DIM) return ADASCALE_ERR_TOO_LARGE;
    if (g->n_rows == 0) return ADASCALE_OK;
    const bool gated = g->y && g->gate_kind != ADASCALE_GATE_NONE, matrix = gated && g->gate_kind == ADASCALE_GATE_SIGMOID;
    const bool post = g->y && g->post != ADASCALE_NORM_NONE;
    if (!g->x || !g->h || !g->w_pre || (g->y && !g->x_new) || (post && !g->w_post) || (gated && !g->gate) || g->ld_x < g->dim ||
        g->ld_h < g->dim || (g->y && (g->ld_y < g->dim || g->ld_x_new < g->dim)) || (matrix && g->ld_gate < g->dim))
        return ADASCALE_ERR_INVALID_ARG;
    if ((g->x_new == g->x && g->y && g->ld_x_new != g->ld_x) || (g->h == g->y && g->ld_h != g->ld_y)) return ADASCALE_ERR_INVALID_ARG;
    const int ex = elem_bytes(g->x_dtype), ey = elem_bytes(g->y_dtype);
    if (!on(g->x, ex) || !on(g->x_new, ex) || !on(g->y, ey) || !on(g->h, ey) || (gated && !on(g->gate, matrix ? ey : 4)) ||
        !on(g->w_post, 4) || !on(g->b_post, 4) || !on(g->w_pre, 4) || !on(g->b_pre, 4))
        return ADASCALE_ERR_ALIGNMENT;
    const int sms = sm_count();
    if (!sms) return ADASCALE_ERR_CUDA;
    NormArgs a = {};
    a.x = rows(g->x, g->ld_x, g->x_dtype);
    a.y = rows(g->y, g->ld_y, g->y_dtype);
    a.x_new = rows(g->x_new, g->ld_x_new, g->x_dtype);
    a.h = rows(g->h, g->ld_h, g->y_dtype);
    a.gate = rows(matrix ? g->gate : nullptr, g->ld_gate, g->y_dtype);
    a.gate_channel = gated && !matrix ? static_cast<const float *>(g->gate) : nullptr;
    a.w_post = post ? g->w_post : nullptr;
    a.b_post = g->post == ADASCALE_NORM_LAYER ? g->b_post : nullptr;
    a.w_pre = g->w_pre;
    a.b_pre = g->pre == ADASCALE_NORM_LAYER ? g->b_pre : nullptr;
    a.n = g->n_rows;
    a.dim = (int)g->dim;
    a.post = g->post;
    a.pre = g->pre;
    a.gate_kind = gated ? g->gate_kind : ADASCALE_GATE_NONE;
    a.inv_dim = 1.f / (float)g->dim;
    a.res_scale = g->res_scale;
    a.eps = g->eps;
    const long long n = g->n_rows;
    // four elements an access; bulk copies want 16 bytes: forward_staged() for the types and the group that the width gets
    const bool bulk = ex == 2 && ey == 2 && forward_split(g->dim).group == 32;
    const int bx = bulk ? 16 : 4 * ex, by = bulk ? 16 : 4 * ey;
    const bool vec = g->dim % (bulk ? 8 : 4) == 0 && rows_on(g->x, g->ld_x, n, ex, bx) && rows_on(g->h, g->ld_h, n, ey, by) && on(a.w_pre, 16) &&
                     on(a.b_pre, 16) && (!g->y || (rows_on(g->y, g->ld_y, n, ey, by) && rows_on(g->x_new, g->ld_x_new, n, ex, bx))) &&
                     on(a.w_post, 16) && on(a.b_post, 16) && on(a.gate_channel, 16) && rows_on(a.gate.p, g->ld_gate, n, ey, by);
    cudaStream_t s = (cudaStream_t)cuda_stream;
    a.stage_bytes = row_bytes(a.x, a.dim) + row_bytes(a.y, a.dim) + row_bytes(a.gate, a.dim);
    if (g->x_dtype == ADASCALE_F32)
        OPS_CU(g->y_dtype == ADASCALE_F32 ? launch_boundary<kF32, kF32>(a, vec, sms, s) : launch_boundary<kF32, kBf16>(a, vec, sms, s));
    else
        OPS_CU(g->y_dtype == ADASCALE_F32 ? launch_boundary<kBf16, kF32>(a, vec, sms, s) : launch_boundary<kBf16, kBf16>(a, vec, sms, s));
    return ADASCALE_OK;
}

// One row of partial sums of each kind per block.
int64_t adascale_residual_norm_grad_workspace(int64_t n_rows, int64_t dim)
{
    if (n_rows < 0 || n_rows > kMaxRows || dim < 1 || dim > ADASCALE_NORM_MAX_DIM) return 0;
    const long long rows = n_rows < kMaxPartials ? n_rows : kMaxPartials;
    return rows * kSums * ceil_div(dim, 8) * 8 * (long long)sizeof(float);
}

adascale_status adascale_residual_norm_grad(const adascale_residual_norm_grad_args *g, void *cuda_stream)
{
    if (!g || g->n_rows < 0 || g->dim < 1 || !is_dtype(g->x_dtype) || !is_dtype(g->y_dtype) || !is_dtype(g->wgrad_dtype) ||
        !norm_kind(g->pre, false) || !norm_kind(g->post, true) || g->gate_kind < ADASCALE_GATE_NONE ||
        g->gate_kind > ADASCALE_GATE_SIGMOID || !std::isfinite(g->res_scale) || !(g->eps >= 0.f) || !std::isfinite(g->eps))
        return ADASCALE_ERR_INVALID_ARG;
    if (g->n_rows > kMaxRows || g->dim > ADASCALE_NORM_MAX_DIM) return ADASCALE_ERR_TOO_LARGE;
    const bool gated = g->y && g->gate_kind != ADASCALE_GATE_NONE, matrix = gated && g->gate_kind == ADASCALE_GATE_SIGMOID;
    const bool post = g->y && g->post != ADASCALE_NORM_NONE;
    const int ex = elem_bytes(g->x_dtype), ey = elem_bytes(g->y_dtype), ew = elem_bytes(g->wgrad_dtype);
    if (g->n_rows > 0) {
        if (!g->x_new || !g->dh || !g->dx || !g->w_pre || (post && !g->w_post) || (gated && !g->gate) || !g->workspace ||
            g->workspace_bytes < adascale_residual_norm_grad_workspace(g->n_rows, g->dim))
            return ADASCALE_ERR_INVALID_ARG;
        if (g->ld_x_new < g->dim || g->ld_dh < g->dim || g->ld_dx < g->dim || (g->dx_new && g->ld_dx_new < g->dim) ||
            (g->y && (g->ld_y < g->dim || (g->dy && g->ld_dy < g->dim))) ||
            (matrix && (g->ld_gate < g->dim || (g->dgate && g->ld_dgate < g->dim))))
            return ADASCALE_ERR_INVALID_ARG;
        if ((g->dx == g->dx_new && g->ld_dx != g->ld_dx_new) || (g->dy && g->dy == g->dh && g->ld_dy != g->ld_dh))
            return ADASCALE_ERR_INVALID_ARG;
        if (!on(g->x_new, ex) || !on(g->y, ey) || !on(g->dx_new, ex) || !on(g->dh, ey) || !on(g->dx, ex) || !on(g->dy, ey) ||
            (gated && (!on(g->gate, matrix ? ey : 4) || !on(g->dgate, matrix ? ey : ew))) || !on(g->w_post, 4) || !on(g->b_post, 4) ||
            !on(g->w_pre, 4) || !on(g->dw_post, ew) || !on(g->db_post, ew) || !on(g->dw_pre, ew) || !on(g->db_pre, ew) ||
            !on(g->workspace, 16))
            return ADASCALE_ERR_ALIGNMENT;
    }
    const int sms = sm_count();
    if (!sms) return ADASCALE_ERR_CUDA;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    ColumnArgs b = {};
    b.partial = static_cast<const float *>(g->workspace);
    b.out[kDwPre] = g->dw_pre;
    b.out[kDbPre] = g->pre == ADASCALE_NORM_LAYER ? g->db_pre : nullptr;
    b.out[kDwPost] = post ? g->dw_post : nullptr;
    b.out[kDbPost] = post && g->post == ADASCALE_NORM_LAYER ? g->db_post : nullptr;
    b.out[kDgate] = gated && !matrix ? g->dgate : nullptr;
    const bool columns = b.out[0] || b.out[1] || b.out[2] || b.out[3] || b.out[4];
    int partials = 0;
    const int ld_partial = (int)(ceil_div(g->dim, 8) * 8);
    if (g->n_rows > 0) {
        GradArgs a = {};
        a.x = rows(g->x_new, g->ld_x_new, g->x_dtype);
        a.y = rows(g->y, g->ld_y, g->y_dtype);
        a.dx_new = rows(g->dx_new, g->ld_dx_new, g->x_dtype);
        a.dh = rows(g->dh, g->ld_dh, g->y_dtype);
        a.gate = rows(matrix ? g->gate : nullptr, g->ld_gate, g->y_dtype);
        a.dx = rows(g->dx, g->ld_dx, g->x_dtype);
        a.dy = rows(g->y ? g->dy : nullptr, g->ld_dy, g->y_dtype);
        a.dgate = rows(matrix ? g->dgate : nullptr, g->ld_dgate, g->y_dtype);
        a.gate_channel = gated && !matrix ? static_cast<const float *>(g->gate) : nullptr;
        a.w_post = post ? g->w_post : nullptr;
        a.b_post = g->post == ADASCALE_NORM_LAYER ? g->b_post : nullptr;
        a.w_pre = g->w_pre;
        a.partial = static_cast<float *>(g->workspace);
        a.n = g->n_rows;
        a.dim = (int)g->dim;
        a.ld_partial = ld_partial;
        a.followed = columns;
        a.post = g->post;
        a.pre = g->pre;
        a.gate_kind = gated ? g->gate_kind : ADASCALE_GATE_NONE;
        a.inv_dim = 1.f / (float)g->dim;
        a.res_scale = g->res_scale;
        a.eps = g->eps;
        const long long n = g->n_rows;
        const bool vec = g->dim % 8 == 0 && rows_on(g->x_new, g->ld_x_new, n, ex, 16) && rows_on(g->dh, g->ld_dh, n, ey, 16) &&
                         rows_on(g->dx, g->ld_dx, n, ex, 16) && rows_on(g->dx_new, g->ld_dx_new, n, ex, 16) && on(a.w_pre, 16) &&
                         (!g->y || (rows_on(g->y, g->ld_y, n, ey, 16) && rows_on(g->dy, g->ld_dy, n, ey, 16))) && on(a.w_post, 16) &&
                         on(a.b_post, 16) && on(a.gate_channel, 16) && rows_on(a.gate.p, g->ld_gate, n, ey, 16) &&
                         rows_on(a.dgate.p, g->ld_dgate, n, ey, 16);
        a.stage_bytes = row_bytes(a.x, a.dim) + row_bytes(a.dh, a.dim) + row_bytes(a.dx_new, a.dim) + row_bytes(a.y, a.dim) + row_bytes(a.gate, a.dim);
        if (g->x_dtype == ADASCALE_F32)
            OPS_CU(g->y_dtype == ADASCALE_F32 ? launch_grad<kF32, kF32>(a, vec, sms, s, partials) : launch_grad<kF32, kBf16>(a, vec, sms, s, partials));
        else
            OPS_CU(g->y_dtype == ADASCALE_F32 ? launch_grad<kBf16, kF32>(a, vec, sms, s, partials) : launch_grad<kBf16, kBf16>(a, vec, sms, s, partials));
    }
    b.dim = (int)g->dim;
    b.ld_partial = ld_partial;
    b.n_partials = partials;
    b.bf16_out = g->wgrad_dtype == ADASCALE_BF16;
    if (columns)
        OPS_CU(launch(k_columns, kSums * ceil_div(g->dim, 32), kColumnWarps * 32, 0, s, b));
    return ADASCALE_OK;
}

}  // extern "C"
