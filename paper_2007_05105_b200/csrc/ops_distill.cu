// Distillation from a teacher's top logits, with its gradient (adascale_distill).
//
// For one row, with z the student's logits, everything the loss and its gradient need of the
// vocabulary is the maximum m and one or two sums:
//
//   s_T = sum_v exp((z_v - m) / T),  s_1 = sum_v exp(z_v - m)
//   alpha part: T^2 [ sum_k q_k (log q_k - (z_{i_k} - m) / T) + log s_T ]      beta part: log s_1 - (z_y - m)
//   dz_v = weight [ alpha T exp((z_v - m) / T) / s_T + beta exp(z_v - m) / s_1 ]  for every v, and
//   in addition  - weight alpha T q_k  at i_k,  - weight beta  at y
//
// z - m is formed before the multiplication by log2(e) / T: for logits at the type's lowest value
// the product of each alone would overflow, and the difference of near values is exact.
#include "ops_common.cuh"

#include <cfloat>
#include <cooperative_groups.h>

namespace {

namespace cg = cooperative_groups;

// Four blocks of 256 threads per SM and four 16-byte pieces in flight per thread: 361 us on 8192 rows of 50257
// bf16 logits (T = 2) against 372 (512 threads, three blocks), 370 (256, six) and 437 (512, two).
constexpr int kThreads = 256;
constexpr int kBlocks = 4;
constexpr int kUnroll = 4;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxK = ADASCALE_DISTILL_MAX_K;
constexpr int kMaxCluster = 8;

struct RowArgs {
    const void *z;
    void *dz;
    const void *t, *ids, *labels;
    const float *weight;
    float *row_loss;
    long long n, vocab, ld_z, ld_dz, ld_t, ld_ids;
    int k, t_bf16, wide_ids, wide_labels;
    float T, invT, alpha, beta;
    float cT, c1;     // log2(e) / T and log2(e); cT alone where one sum serves both parts
    int one_sum;      // T = 1, or only one of the parts is asked for
    int aligned_out;  // dz's rows start at the same place within 16 bytes as z's
};

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// The walks over a row work on packed pairs: they are bound by instruction issue before anything else
// (26.8 instructions per entry without pairs, 62 % of the issue slots taken at half the memory's rate).
__device__ __forceinline__ f2 ex2_2(f2 v)
{
    float a, b;
    unpack2(v, a, b);
    return pack2(ex2(a), ex2(b));
}

// Sixteen bytes of a row: four pairs (bf16) or two (f32), and their largest value.
template <typename ZT> struct Piece;
template <> struct Piece<bf16> {
    static constexpr int kPairs = 4;
    uint4 w;
    __device__ __forceinline__ unsigned word(int i) const { return i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w; }
    __device__ __forceinline__ f2 pair(int i) const { return pack2(bf_lo(word(i)), bf_hi(word(i))); }
    __device__ __forceinline__ float top() const
    {
        const __nv_bfloat162 a = *reinterpret_cast<const __nv_bfloat162 *>(&w.x), b = *reinterpret_cast<const __nv_bfloat162 *>(&w.y),
                             c = *reinterpret_cast<const __nv_bfloat162 *>(&w.z), d = *reinterpret_cast<const __nv_bfloat162 *>(&w.w);
        const __nv_bfloat162 m = __hmax2(__hmax2(a, b), __hmax2(c, d));
        return fmaxf(__low2float(m), __high2float(m));
    }
    __device__ __forceinline__ void set(int i, f2 v)
    {
        float lo, hi;
        unpack2(v, lo, hi);
        const unsigned p = bf_pack(lo, hi);
        if (i == 0) w.x = p; else if (i == 1) w.y = p; else if (i == 2) w.z = p; else w.w = p;
    }
    __device__ __forceinline__ void store_each(bf16 *p) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            reinterpret_cast<unsigned short *>(p)[2 * i] = (unsigned short)word(i);
            reinterpret_cast<unsigned short *>(p)[2 * i + 1] = (unsigned short)(word(i) >> 16);
        }
    }
};
template <> struct Piece<float> {
    static constexpr int kPairs = 2;
    uint4 w;
    __device__ __forceinline__ f2 pair(int i) const
    {
        return i == 0 ? pack2(__uint_as_float(w.x), __uint_as_float(w.y)) : pack2(__uint_as_float(w.z), __uint_as_float(w.w));
    }
    __device__ __forceinline__ float top() const
    {
        return fmaxf(fmaxf(__uint_as_float(w.x), __uint_as_float(w.y)), fmaxf(__uint_as_float(w.z), __uint_as_float(w.w)));
    }
    __device__ __forceinline__ void set(int i, f2 v)
    {
        float lo, hi;
        unpack2(v, lo, hi);
        if (i == 0) {
            w.x = __float_as_uint(lo);
            w.y = __float_as_uint(hi);
        } else {
            w.z = __float_as_uint(lo);
            w.w = __float_as_uint(hi);
        }
    }
    __device__ __forceinline__ void store_each(float *p) const
    {
        reinterpret_cast<unsigned *>(p)[0] = w.x;
        reinterpret_cast<unsigned *>(p)[1] = w.y;
        reinterpret_cast<unsigned *>(p)[2] = w.z;
        reinterpret_cast<unsigned *>(p)[3] = w.w;
    }
};

// How the second sum's exponential comes from the first's:  0 not needed;  1, 2 T = 2, 4: its
// square, its fourth power;  3 a second evaluation.
template <int SECOND> __device__ __forceinline__ float second(float eT, float d, float c1)
{
    if constexpr (SECOND == 1) return eT * eT;
    if constexpr (SECOND == 2) return (eT * eT) * (eT * eT);
    if constexpr (SECOND == 3) return ex2(d * c1);
    return 0.f;
}

// Maximum and sums of a part of the row, relative to that maximum.
struct Sums {
    float m, sT, s1;
};

template <int SECOND> __device__ __forceinline__ Sums join(const Sums &a, const Sums &b, float cT, float c1)
{
    Sums r;
    r.m = fmaxf(a.m, b.m);
    const float da = a.m - r.m, db = b.m - r.m;
    const float fa = ex2(da * cT), fb = ex2(db * cT);
    r.sT = fmaf(a.sT, fa, b.sT * fb);
    r.s1 = SECOND ? fmaf(a.s1, second<SECOND>(fa, da, c1), b.s1 * second<SECOND>(fb, db, c1)) : 0.f;
    return r;
}

// A thread's running maximum and sums, the sums in pairs.
template <int SECOND> struct Running {
    float m = -FLT_MAX;
    f2 sT = 0, s1 = 0;  // two zeros

    __device__ __forceinline__ void raise(float top, float cT, float c1)
    {
        if (top > m) {
            const float d = m - top, f = ex2(d * cT);
            sT = mul2(sT, pack2(f, f));
            if (SECOND) {
                const float g = second<SECOND>(f, d, c1);
                s1 = mul2(s1, pack2(g, g));
            }
            m = top;
        }
    }
    // x - m of a pair of entries under the current maximum
    __device__ __forceinline__ void add(f2 x, f2 minus_m, f2 cT, f2 c1)
    {
        const f2 d = add2(x, minus_m), e = ex2_2(mul2(d, cT));
        sT = add2(sT, e);
        if constexpr (SECOND == 1) s1 = fma2(e, e, s1);
        if constexpr (SECOND == 2) {
            const f2 q = mul2(e, e);
            s1 = fma2(q, q, s1);
        }
        if constexpr (SECOND == 3) s1 = add2(s1, ex2_2(mul2(d, c1)));
    }
    template <int N, typename ZT> __device__ __forceinline__ void absorb(const Piece<ZT> (&p)[N], float cT, float c1)
    {
        float top = p[0].top();
#pragma unroll
        for (int u = 1; u < N; ++u) top = fmaxf(top, p[u].top());
        raise(top, cT, c1);
        const f2 minus_m = pack2(-m, -m), cT2 = pack2(cT, cT), c12 = pack2(c1, c1);
#pragma unroll
        for (int u = 0; u < N; ++u)
#pragma unroll
            for (int i = 0; i < Piece<ZT>::kPairs; ++i) add(p[u].pair(i), minus_m, cT2, c12);
    }
    __device__ __forceinline__ Sums sums() const
    {
        float a, b, c, d;
        unpack2(sT, a, b);
        unpack2(s1, c, d);
        return {m, a + b, c + d};
    }
};

// One row per cluster of 1, 2, 4 or 8 blocks; each block has a contiguous part of the vocabulary.
// First walk: maximum and sums, rescaled as the maximum grows, while the last warp turns the
// teacher's list into q.  Second walk (with a gradient): the part is read again - it is still in
// L2 - and the gradient of every entry written as if no list existed; then the few entries
// that the list or the label names are written again with their whole value.
template <typename ZT, int SECOND, bool GRAD>
__global__ void __launch_bounds__(kThreads, kBlocks) k_distill_rows(const __grid_constant__ RowArgs a)
{
    constexpr int V = 16 / sizeof(ZT);
    __shared__ float q[kMaxK], zk[kMaxK];
    __shared__ int id[kMaxK];
    __shared__ Sums warp_sums[kWarps];
    __shared__ Sums block_sums[kMaxCluster];  // of every block of the cluster
    __shared__ float list_total;              // sum of exp((t - max) / T); 0 for an empty list
    griddep_wait();
    cg::cluster_group cluster = cg::this_cluster();
    const int parts = (int)cluster.num_blocks(), part = (int)cluster.block_rank();
    const long long row = blockIdx.x / parts;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const ZT *z = static_cast<const ZT *>(a.z) + row * a.ld_z;
    ZT *dz = GRAD ? static_cast<ZT *>(a.dz) + row * a.ld_dz : nullptr;

    // this block's part: 16-byte pieces [v0, v1) of the row's aligned middle; block 0 also has the
    // few entries before and after it
    const long long mis = (long long)((uintptr_t)z & 15) / (long long)sizeof(ZT);
    long long head = mis ? V - mis : 0;
    if (head > a.vocab) head = a.vocab;
    const int nv = (int)((a.vocab - head) / V);
    const int tail = (int)(a.vocab - head - (long long)nv * V);
    const int v0 = (int)((long long)nv * part / parts), v1 = (int)((long long)nv * (part + 1) / parts);
    const int loose = part == 0 ? (int)head + tail : 0;  // fewer than 16
    const long long loose_at = tid < head ? tid : head + (long long)nv * V + (tid - head);

    const float weight = a.weight ? a.weight[row] : 1.f;
    long long label = -1;
    if (a.beta != 0.f && a.labels) {
        label = load_id(a.labels, a.wide_labels, row);
        if (label < 0 || label >= a.vocab) label = -1;
    }
    const bool live = weight != 0.f && (label >= 0 || (a.alpha != 0.f && a.k > 0));
    float kT = 0.f, k1 = 0.f, aT = 0.f, b1 = 0.f, m = 0.f;

    if (live) {
        if (warp == kWarps - 1) {  // the teacher's list
            float top = -FLT_MAX;
            bool any = false;
            for (int k = lane; k < a.k; k += 32) {
                const long long i = load_id(a.ids, a.wide_ids, row * a.ld_ids + k);
                const long long at = row * a.ld_t + k;
                const float t = a.t_bf16 ? to_f32(static_cast<const bf16 *>(a.t)[at]) : static_cast<const float *>(a.t)[at];
                const bool valid = a.alpha != 0.f && i >= 0 && i < a.vocab && t != -INFINITY;
                id[k] = valid ? (int)i : -1;
                q[k] = t;
                zk[k] = valid ? to_f32(z[i]) : 0.f;
                any |= valid;
                if (valid) top = fmaxf(top, t);
            }
            any = __any_sync(0xffffffffu, any);
            top = warp_max(top);
            float sum = 0.f;
            for (int k = lane; k < a.k; k += 32) {
                const float e = id[k] >= 0 ? expf((q[k] - top) * a.invT) : 0.f;
                q[k] = e;
                sum += e;
            }
            sum = warp_sum(sum);
            if (lane == 0) list_total = any ? sum : 0.f;
        }
        Running<SECOND> run;
        const uint4 *mid = reinterpret_cast<const uint4 *>(z + head);
        int v = v0 + tid;
        for (; v + (kUnroll - 1) * kThreads < v1; v += kUnroll * kThreads) {
            Piece<ZT> p[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) p[u].w = mid[v + u * kThreads];
            run.absorb(p, a.cT, a.c1);
        }
        for (; v < v1; v += kThreads) {
            Piece<ZT> p[1];
            p[0].w = mid[v];
            run.absorb(p, a.cT, a.c1);
        }
        Sums s = run.sums();
        if (tid < loose) s = join<SECOND>(s, {to_f32(z[loose_at]), 1.f, 1.f}, a.cT, a.c1);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const Sums b = {__shfl_xor_sync(0xffffffffu, s.m, o), __shfl_xor_sync(0xffffffffu, s.sT, o),
                            __shfl_xor_sync(0xffffffffu, s.s1, o)};
            s = join<SECOND>(s, b, a.cT, a.c1);
        }
        if (lane == 0) warp_sums[warp] = s;
        __syncthreads();
        s = warp_sums[lane % kWarps];
#pragma unroll
        for (int o = kWarps / 2; o > 0; o >>= 1) {
            const Sums b = {__shfl_xor_sync(0xffffffffu, s.m, o), __shfl_xor_sync(0xffffffffu, s.sT, o),
                            __shfl_xor_sync(0xffffffffu, s.s1, o)};
            s = join<SECOND>(s, b, a.cT, a.c1);
        }
        if (parts > 1) {
            if (tid < parts) *cluster.map_shared_rank(&block_sums[part], tid) = s;
            cluster.sync();
            s = block_sums[0];
            for (int r = 1; r < parts; ++r) s = join<SECOND>(s, block_sums[r], a.cT, a.c1);
        }
        m = s.m;
        const float s1 = a.one_sum ? s.sT : s.s1;
        const bool has_list = list_total != 0.f;  // NaN counts
        const bool has_logits = s.sT != 0.f;      // NaN counts; 0 when all are -inf
        aT = has_list && has_logits ? weight * a.alpha * a.T : 0.f;
        b1 = label >= 0 && has_logits ? weight * a.beta : 0.f;
        const float inv_list = 1.f / list_total;
        if (part == 0 && warp == 0) {
            float loss = 0.f;
            if (aT != 0.f) {
                for (int k = lane; k < a.k; k += 32) {
                    const float p = q[k] * inv_list;
                    if (id[k] >= 0 && p != 0.f) loss += p * (logf(p) - (zk[k] - m) * a.invT);
                }
                loss = (warp_sum(loss) + logf(s.sT)) * a.T * aT;
            }
            if (b1 != 0.f) loss += b1 * (logf(s1) - (to_f32(z[label]) - m));
            if (lane == 0) a.row_loss[row] = loss;
        }
        kT = aT != 0.f ? aT / s.sT : 0.f;
        k1 = b1 != 0.f ? b1 / s1 : 0.f;
        if (a.one_sum) {
            kT += k1;
            k1 = 0.f;
        }
    } else if (part == 0 && tid == 0) {
        a.row_loss[row] = 0.f;
    }
    if constexpr (!GRAD) return;

    float z_label = 0.f;
    if (live && GRAD) {
        z_label = label >= 0 ? to_f32(z[label]) : 0.f;
        // all reads of named entries are done before any block writes (dz may be z)
        if (parts > 1) cluster.sync(); else __syncthreads();
    }
    const bool nothing = kT == 0.f && k1 == 0.f;  // zeros, whatever the logits hold
    auto slope = [&](float x) {
        const float d = x - m, e = ex2(d * a.cT);
        return SECOND ? fmaf(kT, e, k1 * second<SECOND>(e, d, a.c1)) : kT * e;
    };
    const uint4 *mid = reinterpret_cast<const uint4 *>(z + head);
    ZT *out = dz + head;
    const f2 minus_m = pack2(-m, -m), cT2 = pack2(a.cT, a.cT), c12 = pack2(a.c1, a.c1), kT2 = pack2(kT, kT), k12 = pack2(k1, k1);
    auto write = [&](int v, const Piece<ZT> &p) {
        if (a.aligned_out)
            __stcs(reinterpret_cast<uint4 *>(out) + v, p.w);
        else
            p.store_each(out + (long long)v * V);
    };
    if (nothing) {
        Piece<ZT> p;
        p.w = make_uint4(0, 0, 0, 0);
        for (int v = v0 + tid; v < v1; v += kThreads) write(v, p);
        if (tid < loose) put(dz + loose_at, 0.f);
        return;
    }
    auto slopes = [&](Piece<ZT> &p) {
#pragma unroll
        for (int i = 0; i < Piece<ZT>::kPairs; ++i) {
            const f2 d = add2(p.pair(i), minus_m), e = ex2_2(mul2(d, cT2));
            f2 g;
            if constexpr (SECOND == 0) g = mul2(kT2, e);
            if constexpr (SECOND == 1) g = mul2(e, fma2(k12, e, kT2));
            if constexpr (SECOND == 2) g = mul2(e, fma2(k12, mul2(e, mul2(e, e)), kT2));
            if constexpr (SECOND == 3) g = fma2(kT2, e, mul2(k12, ex2_2(mul2(d, c12))));
            p.set(i, g);
        }
    };
    int v = v0 + tid;
    for (; v + (kUnroll - 1) * kThreads < v1; v += kUnroll * kThreads) {
        Piece<ZT> p[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) p[u].w = __ldcs(mid + v + u * kThreads);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            slopes(p[u]);
            write(v + u * kThreads, p[u]);
        }
    }
    for (; v < v1; v += kThreads) {
        Piece<ZT> p;
        p.w = __ldcs(mid + v);
        slopes(p);
        write(v, p);
    }
    if (tid < loose) put(dz + loose_at, slope(to_f32(z[loose_at])));
    __syncthreads();
    // the named entries of this block's part: the first entry of the list that has an id adds up all that have it
    const float list_scale = aT != 0.f ? aT / list_total : 0.f;
    const long long c0 = head + (long long)v0 * V, c1 = head + (long long)v1 * V;
    for (int k = tid; k <= a.k; k += kThreads) {
        const bool is_label = k == a.k;
        const long long i = is_label ? label : aT != 0.f ? id[k] : -1;
        if (i < 0) continue;
        const bool middle = i >= head && i < head + (long long)nv * V;
        if (middle ? (i < c0 || i >= c1) : part != 0) continue;
        bool first = true;
        float mass = 0.f;
        if (aT != 0.f) {
            for (int j = 0; j < a.k; ++j) {
                if (id[j] == i) {
                    if (j < k) first = false;
                    mass += q[j];
                }
            }
        }
        if (!first) continue;
        float g = slope(is_label ? z_label : zk[k]) - list_scale * mass;
        if (i == label) g -= b1;
        put(dz + i, g);
    }
}

struct TotalArgs {
    const float *row_loss;
    float *loss;
    long long n;
};

// The rows' sum, in 64 bits and a fixed order, by one block.
__global__ void __launch_bounds__(1024) k_total(const __grid_constant__ TotalArgs a)
{
    __shared__ double part[32];
    griddep_wait();
    double s = 0.0;
    for (long long i = threadIdx.x; i < a.n; i += 1024) s += (double)__ldcg(a.row_loss + i);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x < 32) {
        s = part[threadIdx.x];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (threadIdx.x == 0) *a.loss = (float)s;
    }
}

// ---- host side -----------------------------------------------------------------------------

template <typename ZT, int SECOND> cudaError_t launch_rows(const RowArgs &a, int parts, cudaStream_t s)
{
    return a.dz ? launch(k_distill_rows<ZT, SECOND, true>, a.n * parts, kThreads, 0, s, a, parts)
                : launch(k_distill_rows<ZT, SECOND, false>, a.n * parts, kThreads, 0, s, a, parts);
}

template <typename ZT> cudaError_t launch_rows(const RowArgs &a, int second, int parts, cudaStream_t s)
{
    switch (second) {
    case 0: return launch_rows<ZT, 0>(a, parts, s);
    case 1: return launch_rows<ZT, 1>(a, parts, s);
    case 2: return launch_rows<ZT, 2>(a, parts, s);
    }
    return launch_rows<ZT, 3>(a, parts, s);
}

}  // namespace

extern "C" {

adascale_status adascale_distill(const adascale_distill_args *g, void *cuda_stream)
{
    if (!g || g->n_rows < 0 || g->vocab < 1 || g->n_top < 0 || !is_dtype(g->dtype) || !is_dtype(g->teacher_dtype) ||
        !is_itype(g->id_type) || !is_itype(g->label_type) || !g->loss)
        return ADASCALE_ERR_INVALID_ARG;
    if (!(g->temperature >= 1e-3f && g->temperature <= 1e3f) || !(g->alpha >= 0.f) || !(g->beta >= 0.f) ||
        !std::isfinite(g->alpha) || !std::isfinite(g->beta))
        return ADASCALE_ERR_INVALID_ARG;
    if (g->n_rows > kMaxRows / kMaxCluster || g->vocab > kMaxRows || g->n_top > kMaxK) return ADASCALE_ERR_TOO_LARGE;
    if (!on(g->loss, 4)) return ADASCALE_ERR_ALIGNMENT;
    const int ez = elem_bytes(g->dtype);
    if (g->n_rows > 0) {
        if (!g->logits || !g->row_loss || g->ld_logits < g->vocab || (g->dlogits && g->ld_dlogits < g->vocab))
            return ADASCALE_ERR_INVALID_ARG;
        if (g->n_top > 0 && (!g->teacher_logits || !g->teacher_ids || g->ld_teacher < g->n_top || g->ld_ids < g->n_top))
            return ADASCALE_ERR_INVALID_ARG;
        if (g->dlogits == g->logits && g->ld_dlogits != g->ld_logits) return ADASCALE_ERR_INVALID_ARG;
        if (!on(g->logits, ez) || !on(g->dlogits, ez) || !on(g->row_loss, 4) || !on(g->weight, 4) ||
            !on(g->teacher_logits, elem_bytes(g->teacher_dtype)) || !on(g->teacher_ids, id_bytes(g->id_type)) ||
            !on(g->labels, id_bytes(g->label_type)))
            return ADASCALE_ERR_ALIGNMENT;
    }
    const int sms = sm_count();
    if (!sms) return ADASCALE_ERR_CUDA;
    cudaStream_t s = (cudaStream_t)cuda_stream;

    if (g->n_rows > 0) {
        RowArgs a = {};
        a.z = g->logits;
        a.dz = g->dlogits;
        a.t = g->teacher_logits;
        a.ids = g->teacher_ids;
        a.labels = g->labels;
        a.weight = g->weight;
        a.row_loss = g->row_loss;
        a.n = g->n_rows;
        a.vocab = g->vocab;
        a.ld_z = g->ld_logits;
        a.ld_dz = g->ld_dlogits;
        a.ld_t = g->ld_teacher;
        a.ld_ids = g->ld_ids;
        a.k = (int)g->n_top;
        a.t_bf16 = g->teacher_dtype == ADASCALE_BF16;
        a.wide_ids = g->id_type == ADASCALE_I64;
        a.wide_labels = g->label_type == ADASCALE_I64;
        a.T = g->temperature;
        a.invT = 1.f / g->temperature;
        a.alpha = g->n_top > 0 ? g->alpha : 0.f;
        a.beta = g->labels ? g->beta : 0.f;
        const double log2e = 1.4426950408889634;
        a.c1 = (float)log2e;
        const bool only_beta = a.alpha == 0.f;
        a.cT = only_beta ? a.c1 : (float)(log2e / (double)g->temperature);
        a.one_sum = only_beta || a.beta == 0.f || g->temperature == 1.f;
        a.aligned_out = g->dlogits && ((uintptr_t)g->dlogits - (uintptr_t)g->logits) % 16 == 0 &&
                        (g->n_rows <= 1 || (g->ld_dlogits - g->ld_logits) * ez % 16 == 0);
        const int second = a.one_sum ? 0 : g->temperature == 2.f ? 1 : g->temperature == 4.f ? 2 : 3;
        int parts = 1;  // few rows: several blocks share one
        while (parts < kMaxCluster && g->n_rows * parts * 2 <= sms && g->vocab >= 4096 * parts) parts *= 2;
        OPS_CU(g->dtype == ADASCALE_F32 ? launch_rows<float>(a, second, parts, s) : launch_rows<bf16>(a, second, parts, s));
    }
    TotalArgs t = {g->row_loss, g->loss, g->n_rows};
    OPS_CU(launch(k_total, 1, 1024, 0, s, t));
    return ADASCALE_OK;
}

}  // extern "C"
