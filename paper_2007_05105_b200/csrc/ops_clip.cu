// Global 2-norm of many gradients, and clipping by it on the way into the slots of a gradient row.
//
//   norm = sqrt(sum g^2),   out = c g,   c = min(1, max_norm / (norm + eps))
//
// Two kernels: k_squares leaves one 64-bit sum a block, k_scale adds those up - every block all of them, in the same order, so
// that no block waits for another - and writes c g.  Bound by memory: the gradients are read twice, because c is not known
// before the last one was read; what the L2 cache still holds of them comes from there, since k_scale walks backwards (lists of 32 MB: all
// at twice the copy rate; of 96 MB and more hardly any).  Measured on a B200: 61M float32 elements, norm 40.7 us (6.0 TB/s), clipped into a
// bf16 row 98 us, 354M bf16 elements 353 us: 6.2 and 6.0 TB/s of three passes.
// The tensors' addresses travel as a kernel argument (29 bytes each, 1024 a launch), so that nothing is copied to
// the device or kept there and a captured call holds its own list.
#include "ops_common.cuh"

#include <algorithm>
#include <vector>

namespace {

constexpr int kThreads = 256;
constexpr int kBlocksPerSm = 4;
constexpr long long kUnit = 4096;        // elements; blocks get equal numbers of units
constexpr int kTableMax = 1024;          // tensors of one launch: the argument stays below the 32764 bytes that one may have
constexpr long long kPartialsMax = 2048; // blocks of one launch
constexpr int kVec = 8;                  // elements of one access: 16 bytes of bf16, two times 16 of f32
constexpr int kUnroll = 4;

// grad type, out type, as bits 0 and 1 of `types`
template <int T> struct ClipArgs {
    const void *g[T];
    void *o[T];
    long long numel[T];
    int first[T + 1];  // units before each tensor; first[n] is the number of them all
    unsigned char types[T];
    int n;
    double *partials;       // this launch's
    const double *all;      // those of every launch
    int n_all;
    float *norm;
    float max_norm, eps;
    int write;              // 0: the norm alone
};

// The part [lo, hi) of tensor t that belongs to a block, tensor by tensor.
struct Range {
    long long unit, end;
};
template <int T> __device__ __forceinline__ Range units_of_block(const ClipArgs<T> &a)
{
    const long long all = a.first[a.n];
    return {all * blockIdx.x / gridDim.x, all * (blockIdx.x + 1) / gridDim.x};
}
// The tensor that unit u is of.
template <int T> __device__ __forceinline__ int tensor_of(const ClipArgs<T> &a, long long u)
{
    int lo = 0, hi = a.n;  // first[lo] <= u < first[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (a.first[mid] <= u) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Squares of M elements, of which the 32-bit sum is taken where it can be trusted: not where squares may have overflowed, nor
// where they are so small that their last bits are below the smallest number.
template <int M> __device__ __forceinline__ double squares(const float (&x)[M])
{
    float s = 0.f;
    unsigned any = 0;
#pragma unroll
    for (int i = 0; i < M; ++i) {
        s = fmaf(x[i], x[i], s);
        any |= __float_as_uint(x[i]);
    }
    if (s < 1e38f && (s > 1e-30f || (any & 0x7fffffffu) == 0)) return s;
    double d = 0.0;
#pragma unroll
    for (int i = 0; i < M; ++i) d = fma((double)x[i], (double)x[i], d);
    return d;
}

template <typename G> __device__ __forceinline__ double sum_of(const G *p, long long n)
{
    double sum = 0.0;
    long long head = (16 - (uintptr_t)p % 16) % 16 / sizeof(G);
    head = head < n ? head : n;
    if (threadIdx.x < head) {
        const float x[1] = {to_f32(p[threadIdx.x])};
        sum += squares<1>(x);
    }
    p += head;
    n -= head;
    constexpr long long kStep = (long long)kThreads * kVec;
    long long i = (long long)threadIdx.x * kVec;
    for (; i + (kUnroll - 1) * kStep + kVec <= n; i += kUnroll * kStep) {
        float x[kUnroll * kVec];
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) load_vec<kVec>(p + i + k * kStep, *reinterpret_cast<float(*)[kVec]>(x + k * kVec));
        sum += squares<kUnroll * kVec>(x);
    }
    for (; i + kVec <= n; i += kStep) {
        float x[kVec];
        load_vec<kVec>(p + i, x);
        sum += squares<kVec>(x);
    }
    for (; i < n; ++i) {  // the one thread whose elements end inside its access
        const float x[1] = {to_f32(p[i])};
        sum += squares<1>(x);
    }
    return sum;
}

__device__ __forceinline__ double block_sum(double v)
{
    __shared__ double part[kThreads / 32];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = v;
    __syncthreads();
    double all = 0.0;
#pragma unroll
    for (int i = 0; i < kThreads / 32; ++i) all += part[i];
    return all;
}

template <int T> __global__ void __launch_bounds__(kThreads, kBlocksPerSm) k_squares(const __grid_constant__ ClipArgs<T> a)
{
    griddep_wait();
    griddep_launch();  // the successor is another kernel of this call
    Range r = units_of_block(a);
    double sum = 0.0;
    for (int t = tensor_of(a, r.unit); r.unit < r.end; ++t) {
        const long long end = r.end < a.first[t + 1] ? r.end : a.first[t + 1];
        const long long lo = (r.unit - a.first[t]) * kUnit, hi = (end - a.first[t]) * kUnit;
        const long long n = (hi < a.numel[t] ? hi : a.numel[t]) - lo;
        if (a.types[t] & 1) sum += sum_of(static_cast<const bf16 *>(a.g[t]) + lo, n);
        else sum += sum_of(static_cast<const float *>(a.g[t]) + lo, n);
        r.unit = end;
    }
    sum = block_sum(sum);
    if (threadIdx.x == 0) a.partials[blockIdx.x] = sum;
}

template <typename G, typename O> __device__ __forceinline__ void scale_part(const G *g, O *o, long long n, float c)
{
    long long head = (16 - (uintptr_t)g % 16) % 16 / sizeof(G);
    if (n < kVec || (uintptr_t)(o + head) % 16 != 0) head = n;  // no common boundary: element by element
    head = head < n ? head : n;
    for (long long i = threadIdx.x; i < head; i += kThreads) put(o + i, c * to_f32(g[i]));
    g += head;
    o += head;
    n -= head;
    // backwards, as the blocks walk over their parts
    constexpr long long kStep = (long long)kThreads * kVec;
    const long long whole = n / (kUnroll * kStep) * (kUnroll * kStep);
    for (long long i = whole + (long long)threadIdx.x * kVec; i < n; i += kStep) {
        if (i + kVec <= n) {
            float x[kVec];
            load_vec<kVec>(g + i, x);
#pragma unroll
            for (int k = 0; k < kVec; ++k) x[k] *= c;
            store_vec_streaming<kVec>(o + i, x);
        } else {
            for (long long k = i; k < n; ++k) put(o + k, c * to_f32(g[k]));
        }
    }
    for (long long i = whole - kUnroll * kStep + (long long)threadIdx.x * kVec; i >= 0; i -= kUnroll * kStep) {
        float x[kUnroll][kVec];
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) load_vec<kVec>(g + i + k * kStep, x[k]);
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) {
#pragma unroll
            for (int j = 0; j < kVec; ++j) x[k][j] *= c;
            store_vec_streaming<kVec>(o + i + k * kStep, x[k]);
        }
    }
}

template <int T> __global__ void __launch_bounds__(kThreads, kBlocksPerSm) k_scale(const __grid_constant__ ClipArgs<T> a)
{
    griddep_wait();
    double sum = 0.0;
    for (int i = threadIdx.x; i < a.n_all; i += kThreads) sum += a.all[i];
    const double norm = sqrt(block_sum(sum));
    if (a.norm && blockIdx.x == 0 && threadIdx.x == 0) *a.norm = (float)norm;
    if (!a.write) return;
    double ratio = (double)a.max_norm / (norm + (double)a.eps);
    if (norm + (double)a.eps == 0.0) ratio = 1.0;  // nothing to scale
    const float c = ratio > 1.0 ? 1.f : (float)ratio;
    Range r = units_of_block(a);
    if (r.unit == r.end) return;
    for (int t = tensor_of(a, r.end - 1); r.unit < r.end; --t) {
        const long long begin = r.unit > a.first[t] ? r.unit : a.first[t];
        const long long lo = (begin - a.first[t]) * kUnit, hi = (r.end - a.first[t]) * kUnit;
        const long long n = (hi < a.numel[t] ? hi : a.numel[t]) - lo;
        r.end = begin;
        if (a.o[t] == a.g[t] && c == 1.f) continue;
        switch (a.types[t]) {
        case 0: scale_part(static_cast<const float *>(a.g[t]) + lo, static_cast<float *>(a.o[t]) + lo, n, c); break;
        case 1: scale_part(static_cast<const bf16 *>(a.g[t]) + lo, static_cast<float *>(a.o[t]) + lo, n, c); break;
        case 2: scale_part(static_cast<const float *>(a.g[t]) + lo, static_cast<bf16 *>(a.o[t]) + lo, n, c); break;
        default: scale_part(static_cast<const bf16 *>(a.g[t]) + lo, static_cast<bf16 *>(a.o[t]) + lo, n, c); break;
        }
    }
}

// ---- host side -----------------------------------------------------------------------------

bool same(const adascale_clip_grads_args &a, long long k) { return a.out && a.out[k] == a.grads[k]; }

// Whether an output overlaps another or a gradient that is not its own.  Slots of a row ascend, and gradients mostly lie outside all of it:
// that takes one look at each (a sort of the addresses of 300 tensors takes 20 us).
bool overlapping(const adascale_clip_grads_args &a)
{
    struct Span {
        uintptr_t lo, hi;
        bool out;
    };
    const auto grad_end = [&](long long k) { return (uintptr_t)a.grads[k] + (uintptr_t)a.numels[k] * elem_bytes(a.grad_dtypes[k]); };
    const auto out_end = [&](long long k) { return (uintptr_t)a.out[k] + (uintptr_t)a.numels[k] * elem_bytes(a.out_dtypes[k]); };
    uintptr_t lowest = UINTPTR_MAX, reach = 0;
    bool ascending = true;
    for (long long k = 0; k < a.n_tensors; ++k) {
        if (!a.numels[k]) continue;
        ascending &= (uintptr_t)a.out[k] >= reach;
        lowest = std::min(lowest, (uintptr_t)a.out[k]);
        reach = std::max(reach, out_end(k));
    }
    bool apart = ascending;
    for (long long k = 0; k < a.n_tensors && apart; ++k)
        apart = !a.numels[k] || same(a, k) || grad_end(k) <= lowest || (uintptr_t)a.grads[k] >= reach;
    if (apart) return false;
    std::vector<Span> spans;
    spans.reserve(2 * (size_t)a.n_tensors);
    for (long long k = 0; k < a.n_tensors; ++k) {
        if (!a.numels[k]) continue;
        if (!same(a, k)) spans.push_back({(uintptr_t)a.grads[k], grad_end(k), false});
        spans.push_back({(uintptr_t)a.out[k], out_end(k), true});
    }
    std::sort(spans.begin(), spans.end(), [](const Span &x, const Span &y) { return x.lo < y.lo; });
    uintptr_t any_end = 0, outs_end = 0;  // how far the spans seen, and the outputs among them, reach
    for (const Span &s : spans) {
        if (s.lo < (s.out ? any_end : outs_end)) return true;
        any_end = std::max(any_end, s.hi);
        if (s.out) outs_end = std::max(outs_end, s.hi);
    }
    return false;
}

adascale_status check_clip(const adascale_clip_grads_args &a)
{
    if (a.n_tensors > ADASCALE_CLIP_MAX_TENSORS) return ADASCALE_ERR_TOO_LARGE;  // for which there is no workspace either
    if (a.n_tensors < 0 || !a.norm || !a.workspace) return ADASCALE_ERR_INVALID_ARG;
    if (a.n_tensors && (!a.grads || !a.numels || !a.grad_dtypes || (a.out && !a.out_dtypes))) return ADASCALE_ERR_INVALID_ARG;
    if (a.out && !(std::isfinite(a.max_norm) && a.max_norm >= 0.f && std::isfinite(a.eps) && a.eps >= 0.f)) return ADASCALE_ERR_INVALID_ARG;
    if (a.workspace_bytes < adascale_clip_grads_workspace(a.n_tensors)) return ADASCALE_ERR_INVALID_ARG;
    bool aligned = on(a.norm, 4) && on(a.workspace, 16), large = false;  // told apart after all else
    long long all = 0;  // elements
    for (long long k = 0; k < a.n_tensors; ++k) {
        const long long n = a.numels[k];
        if (n < 0 || !is_dtype(a.grad_dtypes[k]) || (a.out && !is_dtype(a.out_dtypes[k]))) return ADASCALE_ERR_INVALID_ARG;
        if (!n) continue;
        if (!a.grads[k] || (a.out && !a.out[k])) return ADASCALE_ERR_INVALID_ARG;
        if (same(a, k) && a.out_dtypes[k] != a.grad_dtypes[k]) return ADASCALE_ERR_INVALID_ARG;
        aligned &= on(a.grads[k], elem_bytes(a.grad_dtypes[k])) && (!a.out || on(a.out[k], elem_bytes(a.out_dtypes[k])));
        large |= n > 1LL << 40 || (all += n) > 1LL << 42;
    }
    if (!aligned) return ADASCALE_ERR_ALIGNMENT;
    if (large) return ADASCALE_ERR_TOO_LARGE;
    return a.out && overlapping(a) ? ADASCALE_ERR_INVALID_ARG : ADASCALE_OK;
}

// One launch of each kernel for every T tensors.
template <int T> adascale_status run_clip(const adascale_clip_grads_args &a, long long live, cudaStream_t s)
{
    const int sms = sm_count();
    if (sms <= 0) return ADASCALE_ERR_CUDA;
    double *partials = static_cast<double *>(a.workspace);
    const long long most = std::min<long long>((long long)sms * kBlocksPerSm, kPartialsMax);
    std::vector<ClipArgs<T>> tables((size_t)std::max<long long>(1, ceil_div(live, T)));
    long long n_partials = 0;
    std::vector<long long> blocks;
    long long k = 0;
    for (ClipArgs<T> &c : tables) {
        c.n = 0;
        c.first[0] = 0;
        for (; k < a.n_tensors && c.n < T; ++k) {
            if (!a.numels[k]) continue;
            const int i = c.n++;
            c.g[i] = a.grads[k];
            c.o[i] = a.out ? a.out[k] : nullptr;
            c.numel[i] = a.numels[k];
            c.types[i] = (unsigned char)(a.grad_dtypes[k] | (a.out ? 2 * a.out_dtypes[k] : 0));
            c.first[i + 1] = c.first[i] + (int)ceil_div(a.numels[k], kUnit);
        }
        c.partials = partials + n_partials;
        // few units: half of the SM is left to k_scale's blocks, which then wait there (3.2M elements 12.4 us, 11.1)
        blocks.push_back(std::min<long long>(c.first[c.n], c.first[c.n] < 2LL * kBlocksPerSm * sms ? most / 2 : most));
        n_partials += blocks.back();
    }
    for (size_t i = 0; i < tables.size(); ++i)
        if (blocks[i]) OPS_CU(launch(k_squares<T>, blocks[i], kThreads, 0, s, tables[i]));
    for (size_t i = 0; i < tables.size(); ++i) {
        ClipArgs<T> &c = tables[i];
        c.all = partials;
        c.n_all = (int)n_partials;
        c.norm = i ? nullptr : a.norm;
        c.max_norm = a.max_norm;
        c.eps = a.eps;
        c.write = a.out != nullptr;
        if (i == 0 || c.write) OPS_CU(launch(k_scale<T>, c.write ? std::max<long long>(blocks[i], 1) : 1, kThreads, 0, s, c));
    }
    return ADASCALE_OK;
}

}  // namespace

extern "C" int64_t adascale_clip_grads_workspace(int64_t n_tensors)
{
    if (n_tensors < 0 || n_tensors > ADASCALE_CLIP_MAX_TENSORS) return 0;
    // a launch of every size of table has at most kPartialsMax blocks
    return (int64_t)sizeof(double) * kPartialsMax * std::max<long long>(1, ceil_div(n_tensors, kTableMax));
}

extern "C" adascale_status adascale_clip_grads(const adascale_clip_grads_args *args, void *cuda_stream)
{
    if (!args) return ADASCALE_ERR_INVALID_ARG;
    try {
        const adascale_clip_grads_args &a = *args;
        const adascale_status bad = check_clip(a);
        if (bad != ADASCALE_OK) return bad;
        long long live = 0;
        for (long long k = 0; k < a.n_tensors; ++k) live += a.numels[k] != 0;
        cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
        // the smallest table that holds the list: an argument of 30 KB costs host time
        if (live <= 64) return run_clip<64>(a, live, s);
        if (live <= 384) return run_clip<384>(a, live, s);
        return run_clip<kTableMax>(a, live, s);
    } catch (...) {  // no memory on the host
        return ADASCALE_ERR_CUDA;
    }
}
