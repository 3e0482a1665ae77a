// Block boundary: norm of a block's output, gate, residual scale, norm of the stream for the next
// block, and its gradient (adascale_residual_norm, adascale_residual_norm_grad).
//
// With n = (v - mean) r, r = 1 / sqrt(var + eps) (RMS: mean = 0) and dn = dout * w, the gradient of a norm is
//   dv = r [ dn - n mean(dn n) - mean(dn) ]          (RMS: without the last term)
// so both directions of a row need its elements and a handful of sums over them.
#include "ops_common.cuh"

namespace {

constexpr int kMinThreads = 128;   // of a block
constexpr int kMaxThreads = 1024;
constexpr int kElems = 8;          // of a row per thread and vector set
constexpr int kSets = 5;           // column sums of the gradient: dw_pre, db_pre, dw_post, db_post, dgate
enum { kDwPre, kDbPre, kDwPost, kDbPost, kDgate };

// A row belongs to a group of `group` threads (a power of two, 32 .. 1024); thread t has NV sets of eight
// elements: with V = 8 vector i is (i * group + t), with V = 1 the elements i * group + t.
template <int NV, int V> __device__ __forceinline__ int column(int j, int group, int t)
{
    return (j * group + t) * V;
}

// Sums of K values over each group of threads, for all groups of the block at once; one
// barrier: consecutive calls use alternate halves of the scratch.
template <int K> struct GroupSum {
    float (*scratch)[kMaxThreads / 32][K];  // [2][warps][K]
    int group, turn;

    __device__ __forceinline__ void operator()(float (&v)[K])
    {
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = warp_sum(v[k]);
        if (group == 32) return;
        const int warp = threadIdx.x >> 5, per = group >> 5, first = warp & ~(per - 1);
        if ((threadIdx.x & 31) == 0) {
#pragma unroll
            for (int k = 0; k < K; ++k) scratch[turn][warp][k] = v[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float s = 0.f;
            for (int w = 0; w < per; ++w) s += scratch[turn][first + w][k];
            v[k] = s;
        }
        turn ^= 1;
    }
};

struct NormArgs {
    const void *x, *y, *gate;
    void *x_new, *h;
    const float *w_post, *b_post, *w_pre, *b_pre;
    long long n, ld_x, ld_y, ld_x_new, ld_h, ld_gate;
    int dim, group;
    int post, pre, gate_kind;
    float inv_dim, res_scale, eps;
};

__device__ __forceinline__ float sigmoid(float a) { return 1.f / (1.f + __expf(-a)); }

// R rows per group of threads at once: their loads are in flight together, a weight is read
// once for R rows, and a barrier serves R sums.
template <typename XT, typename YT, int V, int NV, int R>
__global__ void __launch_bounds__(kMaxThreads) k_boundary(const __grid_constant__ NormArgs a)
{
    constexpr int J = NV * kElems / V;  // accesses per thread and row
    __shared__ float scratch[2][kMaxThreads / 32][R];
    griddep_wait();
    const int t = threadIdx.x & (a.group - 1), groups = blockDim.x / a.group;
    const long long row0 = ((long long)blockIdx.x * groups + threadIdx.x / a.group) * R;
    GroupSum<R> sum = {scratch, a.group, 0};
    float x[R][J][V], y[R][J][V];

#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int c = column<NV, V>(j, a.group, t);
            const bool in = c < a.dim && row0 + r < a.n;
#pragma unroll
            for (int e = 0; e < V; ++e) x[r][j][e] = y[r][j][e] = 0.f;
            if (in) load_vec<V>(static_cast<const XT *>(a.x) + (row0 + r) * a.ld_x + c, x[r][j]);
            if (in && a.y) load_vec<V>(static_cast<const YT *>(a.y) + (row0 + r) * a.ld_y + c, y[r][j]);
        }
    }
    float s[R];
    // mean and 1 / deviation of every row of v; v is centred
    auto stats = [&](float (&v)[R][J][V], int kind) {
        if (kind == ADASCALE_NORM_LAYER) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                s[r] = 0.f;
#pragma unroll
                for (int j = 0; j < J; ++j)
#pragma unroll
                    for (int e = 0; e < V; ++e) s[r] += v[r][j][e];
            }
            sum(s);
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    const bool in = column<NV, V>(j, a.group, t) < a.dim;
#pragma unroll
                    for (int e = 0; e < V; ++e) v[r][j][e] = in ? v[r][j][e] - s[r] * a.inv_dim : 0.f;
                }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            s[r] = 0.f;
#pragma unroll
            for (int j = 0; j < J; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) s[r] = fmaf(v[r][j][e], v[r][j][e], s[r]);
        }
        sum(s);
#pragma unroll
        for (int r = 0; r < R; ++r) s[r] = rsqrtf(fmaf(s[r], a.inv_dim, a.eps));
    };

    if (a.y) {
        if (a.post != ADASCALE_NORM_NONE) stats(y, a.post);
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int c = column<NV, V>(j, a.group, t);
            if (c >= a.dim) continue;
            float w[V], b[V], g[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                w[e] = g[e] = 1.f;
                b[e] = 0.f;
            }
            if (a.post != ADASCALE_NORM_NONE) load_vec<V>(a.w_post + c, w);
            if (a.b_post) load_vec<V>(a.b_post + c, b);
            if (a.gate_kind == ADASCALE_GATE_CHANNEL) load_vec<V>(static_cast<const float *>(a.gate) + c, g);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (row0 + r >= a.n) break;
                if (a.gate_kind == ADASCALE_GATE_SIGMOID) {
                    load_vec<V>(static_cast<const YT *>(a.gate) + (row0 + r) * a.ld_gate + c, g);
#pragma unroll
                    for (int e = 0; e < V; ++e) g[e] = sigmoid(g[e]);
                }
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float u = a.post != ADASCALE_NORM_NONE ? fmaf(y[r][j][e] * s[r], w[e], b[e]) : y[r][j][e];
                    x[r][j][e] = fmaf(a.res_scale * g[e], u, x[r][j][e]);
                }
                store_vec<V>(static_cast<XT *>(a.x_new) + (row0 + r) * a.ld_x_new + c, x[r][j]);
            }
        }
    }
    stats(x, a.pre);
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int c = column<NV, V>(j, a.group, t);
        if (c >= a.dim) continue;
        float w[V], b[V];
        load_vec<V>(a.w_pre + c, w);
#pragma unroll
        for (int e = 0; e < V; ++e) b[e] = 0.f;
        if (a.b_pre) load_vec<V>(a.b_pre + c, b);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (row0 + r >= a.n) break;
#pragma unroll
            for (int e = 0; e < V; ++e) x[r][j][e] = fmaf(x[r][j][e] * s[r], w[e], b[e]);
            store_vec<V>(static_cast<YT *>(a.h) + (row0 + r) * a.ld_h + c, x[r][j]);
        }
    }
}

struct GradArgs {
    const void *x, *y, *dx_new, *dh, *gate;
    const float *w_post, *b_post, *w_pre;
    void *dx, *dy, *dgate;
    float *partial;  // [groups of the launch][kSets][ld_partial]
    long long n, ld_x, ld_y, ld_dx_new, ld_dh, ld_gate, ld_dx, ld_dy, ld_dgate;
    int dim, group, ld_partial;
    int post, pre, gate_kind;
    float inv_dim, res_scale, eps;
};

// A group of threads walks over rows group, group + groups, ...; every thread keeps the column sums
// of its columns in registers and leaves them at the end, one row of partial sums per group.
template <typename XT, typename YT, int V, int NV, int THREADS>
__global__ void __launch_bounds__(THREADS) k_boundary_grad(const __grid_constant__ GradArgs a)
{
    constexpr int J = NV * kElems / V;
    __shared__ float scratch1[2][kMaxThreads / 32][1], scratch2[2][kMaxThreads / 32][2];
    griddep_wait();
    griddep_launch();
    const int t = threadIdx.x & (a.group - 1), groups = blockDim.x / a.group;
    const long long me = (long long)blockIdx.x * groups + threadIdx.x / a.group, all = (long long)gridDim.x * groups;
    GroupSum<1> sum1 = {scratch1, a.group, 0};
    GroupSum<2> sum2 = {scratch2, a.group, 0};
    float acc[kSets][J][V];
#pragma unroll
    for (int k = 0; k < kSets; ++k)
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) acc[k][j][e] = 0.f;

    auto stats = [&](float (&v)[J][V], int kind) -> float {  // centres v, returns 1 / deviation
        float s[1] = {0.f};
        if (kind == ADASCALE_NORM_LAYER) {
#pragma unroll
            for (int j = 0; j < J; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) s[0] += v[j][e];
            sum1(s);
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const bool in = column<NV, V>(j, a.group, t) < a.dim;
#pragma unroll
                for (int e = 0; e < V; ++e) v[j][e] = in ? v[j][e] - s[0] * a.inv_dim : 0.f;
            }
        }
        s[0] = 0.f;
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) s[0] = fmaf(v[j][e], v[j][e], s[0]);
        sum1(s);
        return rsqrtf(fmaf(s[0], a.inv_dim, a.eps));
    };

    for (long long base = 0; base < a.n; base += all) {  // the same number of rounds for every group of a block
        const long long row = base + me;
        const bool live = row < a.n;
        float x[J][V], y[J][V], dx[J][V], dh[J][V];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int c = column<NV, V>(j, a.group, t);
            const bool in = live && c < a.dim;
#pragma unroll
            for (int e = 0; e < V; ++e) x[j][e] = y[j][e] = dx[j][e] = dh[j][e] = 0.f;
            if (in) {
                load_vec<V>(static_cast<const XT *>(a.x) + row * a.ld_x + c, x[j]);
                load_vec<V>(static_cast<const YT *>(a.dh) + row * a.ld_dh + c, dh[j]);
                if (a.dx_new) load_vec<V>(static_cast<const XT *>(a.dx_new) + row * a.ld_dx_new + c, dx[j]);
                if (a.y) load_vec<V>(static_cast<const YT *>(a.y) + row * a.ld_y + c, y[j]);
            }
        }
        // dx = dx' + pre^T(dh)
        float r = stats(x, a.pre);
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int c = column<NV, V>(j, a.group, t);
            if (c >= a.dim) continue;
            float w[V];
            load_vec<V>(a.w_pre + c, w);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                x[j][e] *= r;
                acc[kDwPre][j][e] = fmaf(dh[j][e], x[j][e], acc[kDwPre][j][e]);
                acc[kDbPre][j][e] += dh[j][e];
                dh[j][e] *= w[e];
                s[0] = fmaf(dh[j][e], x[j][e], s[0]);
                s[1] += dh[j][e];
            }
        }
        sum2(s);
        if (a.pre != ADASCALE_NORM_LAYER) s[1] = 0.f;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int c = column<NV, V>(j, a.group, t);
#pragma unroll
            for (int e = 0; e < V; ++e)
                dx[j][e] = fmaf(r, fmaf(-x[j][e], s[0] * a.inv_dim, dh[j][e] - s[1] * a.inv_dim), dx[j][e]);
            if (live && c < a.dim) store_vec<V>(static_cast<XT *>(a.dx) + row * a.ld_dx + c, dx[j]);
        }
        if (!a.y) continue;
        // gate and post
        r = a.post != ADASCALE_NORM_NONE ? stats(y, a.post) : 1.f;
        s[0] = s[1] = 0.f;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int c = column<NV, V>(j, a.group, t);
            if (c >= a.dim || !live) continue;
            float w[V], b[V], g[V], da[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                w[e] = g[e] = 1.f;
                b[e] = 0.f;
            }
            if (a.post != ADASCALE_NORM_NONE) load_vec<V>(a.w_post + c, w);
            if (a.b_post) load_vec<V>(a.b_post + c, b);
            if (a.gate_kind == ADASCALE_GATE_CHANNEL) load_vec<V>(static_cast<const float *>(a.gate) + c, g);
            if (a.gate_kind == ADASCALE_GATE_SIGMOID) {
                load_vec<V>(static_cast<const YT *>(a.gate) + row * a.ld_gate + c, g);
#pragma unroll
                for (int e = 0; e < V; ++e) g[e] = sigmoid(g[e]);
            }
#pragma unroll
            for (int e = 0; e < V; ++e) {
                y[j][e] *= r;
                const float ds = a.res_scale * dx[j][e], dg = ds * fmaf(y[j][e], w[e], b[e]);
                da[e] = dg * g[e] * (1.f - g[e]);
                acc[kDgate][j][e] += dg;
                const float du = ds * g[e];
                acc[kDwPost][j][e] = fmaf(du, y[j][e], acc[kDwPost][j][e]);
                acc[kDbPost][j][e] += du;
                dx[j][e] = du * w[e];
                s[0] = fmaf(dx[j][e], y[j][e], s[0]);
                s[1] += dx[j][e];
            }
            if (a.gate_kind == ADASCALE_GATE_SIGMOID && a.dgate)
                store_vec<V>(static_cast<YT *>(a.dgate) + row * a.ld_dgate + c, da);
        }
        if (a.post != ADASCALE_NORM_NONE) {
            sum2(s);
            if (a.post != ADASCALE_NORM_LAYER) s[1] = 0.f;
        } else {
            s[0] = s[1] = 0.f;
        }
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int c = column<NV, V>(j, a.group, t);
            if (!live || c >= a.dim || !a.dy) continue;
#pragma unroll
            for (int e = 0; e < V; ++e) dx[j][e] = r * fmaf(-y[j][e], s[0] * a.inv_dim, dx[j][e] - s[1] * a.inv_dim);
            store_vec<V>(static_cast<YT *>(a.dy) + row * a.ld_dy + c, dx[j]);
        }
    }
    if (me >= a.n) return;  // no row, and no partial sums are read
#pragma unroll
    for (int k = 0; k < kSets; ++k)
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int c = column<NV, V>(j, a.group, t);
            if (c < a.dim) store_vec<V>(a.partial + (me * kSets + k) * a.ld_partial + c, acc[k][j]);
        }
}

struct ColumnArgs {
    const float *partial;
    void *out[kSets];
    int dim, ld_partial, n_partials, bf16_out;
};

// Column sums of the partial sums, in a fixed order: 32 columns per block, warp q adds rows q, q + 16, ...
constexpr int kColumnWarps = 16;
__global__ void __launch_bounds__(kColumnWarps * 32) k_columns(const __grid_constant__ ColumnArgs a)
{
    __shared__ float part[kColumnWarps][32];
    griddep_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int chunks = (a.dim + 31) / 32, set = blockIdx.x / chunks, c = (blockIdx.x % chunks) * 32 + lane;
    if (!a.out[set]) return;
    float s = 0.f;
    if (c < a.dim) {
#pragma unroll 4
        for (int p = warp; p < a.n_partials; p += kColumnWarps) s += a.partial[((long long)p * kSets + set) * a.ld_partial + c];
    }
    part[warp][lane] = s;
    __syncthreads();
    if (warp || c >= a.dim) return;
#pragma unroll
    for (int q = 1; q < kColumnWarps; ++q) s += part[q][lane];
    if (a.bf16_out)
        put(static_cast<bf16 *>(a.out[set]) + c, s);
    else
        put(static_cast<float *>(a.out[set]) + c, s);
}

// ---- host side -----------------------------------------------------------------------------

constexpr int kMaxPartials = 148 * 16;  // groups of a gradient launch, at most

// Threads per row for `per` elements each.
int group_of(long long dim, int per)
{
    int g = 32;
    while ((long long)g * per < dim) g *= 2;
    return g;
}

bool norm_kind(int k, bool none_too) { return k == ADASCALE_NORM_RMS || k == ADASCALE_NORM_LAYER || (none_too && k == ADASCALE_NORM_NONE); }

template <typename XT, typename YT, int V>
cudaError_t launch_boundary(NormArgs a, int sms, cudaStream_t s)
{
    const bool wide = a.dim > kMaxThreads * kElems;
    a.group = group_of(a.dim, wide ? 2 * kElems : kElems);
    const int threads = a.group < kMinThreads ? kMinThreads : a.group, groups = threads / a.group;
    if (wide) return launch(k_boundary<XT, YT, V, 2, 1>, ceil_div(a.n, groups), threads, 0, s, a);
    if (a.n >= 4LL * sms * (2048 / a.group)) return launch(k_boundary<XT, YT, V, 1, 2>, ceil_div(a.n, 2 * groups), threads, 0, s, a);
    return launch(k_boundary<XT, YT, V, 1, 1>, ceil_div(a.n, groups), threads, 0, s, a);
}

template <typename XT, typename YT> cudaError_t launch_boundary(const NormArgs &a, bool vec, int sms, cudaStream_t s)
{
    return vec ? launch_boundary<XT, YT, 8>(a, sms, s) : launch_boundary<XT, YT, 1>(a, sms, s);
}

// Blocks of a gradient launch.
long long grad_blocks(long long n, int group, int sms)
{
    const int threads = group < kMinThreads ? kMinThreads : group, groups = threads / group;
    long long blocks = (long long)sms * (512 / threads < 1 ? 1 : 512 / threads);
    if (blocks * groups > kMaxPartials) blocks = kMaxPartials / groups;
    const long long need = ceil_div(n, groups);
    return blocks < need ? blocks : need;
}

template <typename XT, typename YT, int V>
cudaError_t launch_grad(GradArgs a, int sms, cudaStream_t s, long long &partials)
{
    const bool wide = a.dim > 512 * kElems;
    a.group = group_of(a.dim, wide ? 2 * kElems : kElems);
    const int threads = a.group < kMinThreads ? kMinThreads : a.group, groups = threads / a.group;
    const long long blocks = grad_blocks(a.n, a.group, sms);
    partials = blocks * groups < a.n ? blocks * groups : a.n;
    if (threads <= 256) return launch(k_boundary_grad<XT, YT, V, 1, 256>, blocks, threads, 0, s, a);
    if (threads <= 512) return wide ? launch(k_boundary_grad<XT, YT, V, 2, 512>, blocks, threads, 0, s, a)
                                    : launch(k_boundary_grad<XT, YT, V, 1, 512>, blocks, threads, 0, s, a);
    return launch(k_boundary_grad<XT, YT, V, 2, 1024>, blocks, threads, 0, s, a);
}

template <typename XT, typename YT>
cudaError_t launch_grad(const GradArgs &a, bool vec, int sms, cudaStream_t s, long long &partials)
{
    return vec ? launch_grad<XT, YT, 8>(a, sms, s, partials) : launch_grad<XT, YT, 1>(a, sms, s, partials);
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
    a.x = g->x;
    a.y = g->y;
    a.x_new = g->x_new;
    a.h = g->h;
    a.gate = g->gate;
    a.w_post = g->w_post;
    a.b_post = g->post == ADASCALE_NORM_LAYER ? g->b_post : nullptr;
    a.w_pre = g->w_pre;
    a.b_pre = g->pre == ADASCALE_NORM_LAYER ? g->b_pre : nullptr;
    a.n = g->n_rows;
    a.ld_x = g->ld_x;
    a.ld_y = g->ld_y;
    a.ld_x_new = g->ld_x_new;
    a.ld_h = g->ld_h;
    a.ld_gate = g->ld_gate;
    a.dim = (int)g->dim;
    a.post = g->post;
    a.pre = g->pre;
    a.gate_kind = gated ? g->gate_kind : ADASCALE_GATE_NONE;
    a.inv_dim = 1.f / (float)g->dim;
    a.res_scale = g->res_scale;
    a.eps = g->eps;
    const long long n = g->n_rows;
    const bool vec = g->dim % 8 == 0 && rows_on(a.x, a.ld_x, n, ex, 16) && rows_on(a.h, a.ld_h, n, ey, 16) && on(a.w_pre, 16) &&
                     on(a.b_pre, 16) && (!a.y || (rows_on(a.y, a.ld_y, n, ey, 16) && rows_on(a.x_new, a.ld_x_new, n, ex, 16) &&
                     on(a.w_post, 16) && on(a.b_post, 16))) && (!gated || (matrix ? rows_on(a.gate, a.ld_gate, n, ey, 16) : on(a.gate, 16)));
    cudaStream_t s = (cudaStream_t)cuda_stream;
    if (g->x_dtype == ADASCALE_F32)
        OPS_CU(g->y_dtype == ADASCALE_F32 ? launch_boundary<float, float>(a, vec, sms, s) : launch_boundary<float, bf16>(a, vec, sms, s));
    else
        OPS_CU(g->y_dtype == ADASCALE_F32 ? launch_boundary<bf16, float>(a, vec, sms, s) : launch_boundary<bf16, bf16>(a, vec, sms, s));
    return ADASCALE_OK;
}

// One row of partial sums of each kind per group of threads.
int64_t adascale_residual_norm_grad_workspace(int64_t n_rows, int64_t dim)
{
    if (n_rows < 0 || n_rows > kMaxRows || dim < 1 || dim > ADASCALE_NORM_MAX_DIM) return 0;
    const long long rows = n_rows < kMaxPartials ? n_rows : kMaxPartials;
    return rows * kSets * ceil_div(dim, 8) * 8 * (long long)sizeof(float);
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
    long long partials = 0;
    const int ld_partial = (int)(ceil_div(g->dim, 8) * 8);
    if (g->n_rows > 0) {
        GradArgs a = {};
        a.x = g->x_new;
        a.y = g->y;
        a.dx_new = g->dx_new;
        a.dh = g->dh;
        a.gate = g->gate;
        a.w_post = g->w_post;
        a.b_post = g->post == ADASCALE_NORM_LAYER ? g->b_post : nullptr;
        a.w_pre = g->w_pre;
        a.dx = g->dx;
        a.dy = g->dy;
        a.dgate = g->dgate;
        a.partial = static_cast<float *>(g->workspace);
        a.n = g->n_rows;
        a.ld_x = g->ld_x_new;
        a.ld_y = g->ld_y;
        a.ld_dx_new = g->ld_dx_new;
        a.ld_dh = g->ld_dh;
        a.ld_gate = g->ld_gate;
        a.ld_dx = g->ld_dx;
        a.ld_dy = g->ld_dy;
        a.ld_dgate = g->ld_dgate;
        a.dim = (int)g->dim;
        a.ld_partial = ld_partial;
        a.post = g->post;
        a.pre = g->pre;
        a.gate_kind = gated ? g->gate_kind : ADASCALE_GATE_NONE;
        a.inv_dim = 1.f / (float)g->dim;
        a.res_scale = g->res_scale;
        a.eps = g->eps;
        const long long n = g->n_rows;
        const bool vec = g->dim % 8 == 0 && rows_on(a.x, a.ld_x, n, ex, 16) && rows_on(a.dh, a.ld_dh, n, ey, 16) &&
                         rows_on(a.dx, a.ld_dx, n, ex, 16) && rows_on(a.dx_new, a.ld_dx_new, n, ex, 16) && on(a.w_pre, 16) &&
                         (!a.y || (rows_on(a.y, a.ld_y, n, ey, 16) && rows_on(a.dy, a.ld_dy, n, ey, 16) && on(a.w_post, 16) && on(a.b_post, 16))) &&
                         (!gated || (matrix ? rows_on(a.gate, a.ld_gate, n, ey, 16) && rows_on(a.dgate, a.ld_dgate, n, ey, 16) : on(a.gate, 16)));
        if (g->x_dtype == ADASCALE_F32)
            OPS_CU(g->y_dtype == ADASCALE_F32 ? launch_grad<float, float>(a, vec, sms, s, partials)
                                              : launch_grad<float, bf16>(a, vec, sms, s, partials));
        else
            OPS_CU(g->y_dtype == ADASCALE_F32 ? launch_grad<bf16, float>(a, vec, sms, s, partials)
                                              : launch_grad<bf16, bf16>(a, vec, sms, s, partials));
    }
    ColumnArgs b = {};
    b.partial = static_cast<const float *>(g->workspace);
    b.out[kDwPre] = g->dw_pre;
    b.out[kDbPre] = g->pre == ADASCALE_NORM_LAYER ? g->db_pre : nullptr;
    b.out[kDwPost] = post ? g->dw_post : nullptr;
    b.out[kDbPost] = post && g->post == ADASCALE_NORM_LAYER ? g->db_post : nullptr;
    b.out[kDgate] = gated && !matrix ? g->dgate : nullptr;
    b.dim = (int)g->dim;
    b.ld_partial = ld_partial;
    b.n_partials = (int)partials;
    b.bf16_out = g->wgrad_dtype == ADASCALE_BF16;
    if (b.out[0] || b.out[1] || b.out[2] || b.out[3] || b.out[4])
        OPS_CU(launch(k_columns, kSets * ceil_div(g->dim, 32), kColumnWarps * 32, 0, s, b));
    return ADASCALE_OK;
}

}  // extern "C"
