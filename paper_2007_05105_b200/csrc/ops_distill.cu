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
    float c0, c1;     // what exps() takes
    float headroom;   // kHeadroom powers of two, in logits
    int log_parts;    // blocks that share a row, a power of two (a 64-bit division here took as long as a tenth of a row)
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
    // x - m of pair i: sm_100 subtracts a float from a bf16 with one instruction, which widens it exactly
    __device__ __forceinline__ f2 less(int i, float m) const
    {
        float lo, hi;
        const unsigned w = word(i);
        asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tsub.rn.f32.bf16 %0, l, %3;\n\tsub.rn.f32.bf16 %1, h, %3;\n\t}" : "=f"(lo), "=f"(hi) : "r"(w), "f"(m));
        return pack2(lo, hi);
    }
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
    __device__ __forceinline__ f2 less(int i, float m) const
    {
        const f2 x = i == 0 ? pack2(__uint_as_float(w.x), __uint_as_float(w.y)) : pack2(__uint_as_float(w.z), __uint_as_float(w.w));
        return add2(x, pack2(-m, -m));
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

// Both exponentials of an entry from one evaluation where T is a ratio of small numbers: with u = exp(d / p) and
// T = p / q, exp(d / T) = u^q and exp(d) = u^p.  FORM: one sum serves both parts (u itself); T = 2, 3, 4,
// 3/2; any other T, by two evaluations (8192 x 50257 bf16: T = 1.5 335 us, T = 1.3 442: there the evaluations are the limit).
enum { kOneSum = 0, kTwo, kThree, kFour, kThreeHalves, kAnyT };
struct Exps {
    float eT, e1;
};
// d: z - m;  c0: log2(e) / T (kThreeHalves: log2(e) / 3);  c1: log2(e)
template <int FORM> __device__ __forceinline__ Exps exps(float d, float c0, float c1)
{
    const float u = ex2(d * c0);
    if constexpr (FORM == kTwo) return {u, u * u};
    if constexpr (FORM == kThree) return {u, u * u * u};
    if constexpr (FORM == kFour) return {u, (u * u) * (u * u)};
    if constexpr (FORM == kThreeHalves) return {u * u, u * u * u};
    if constexpr (FORM == kAnyT) return {u, ex2(d * c1)};
    return {u, 0.f};
}

// Maximum and sums of a part of the row, relative to that maximum.
struct Sums {
    float m, sT, s1;
};

template <int FORM> __device__ __forceinline__ Sums join(const Sums &a, const Sums &b, float c0, float c1)
{
    Sums r;
    r.m = fmaxf(a.m, b.m);
    const Exps fa = exps<FORM>(a.m - r.m, c0, c1), fb = exps<FORM>(b.m - r.m, c0, c1);
    r.sT = fmaf(a.sT, fa.eT, b.sT * fb.eT);
    r.s1 = FORM ? fmaf(a.s1, fa.e1, b.s1 * fb.e1) : 0.f;
    return r;
}

// The sums of LANES neighbouring lanes; sums relative to the same reference, as they mostly are, are added.
template <int FORM, int LANES> __device__ __forceinline__ Sums join_lanes(Sums s, float c0, float c1)
{
    if (__all_sync(0xffffffffu, s.m == __shfl_sync(0xffffffffu, s.m, 0))) {
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) {
            s.sT += __shfl_xor_sync(0xffffffffu, s.sT, o);
            if (FORM) s.s1 += __shfl_xor_sync(0xffffffffu, s.s1, o);
        }
        return s;
    }
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) {
        const Sums b = {__shfl_xor_sync(0xffffffffu, s.m, o), __shfl_xor_sync(0xffffffffu, s.sT, o), __shfl_xor_sync(0xffffffffu, s.s1, o)};
        s = join<FORM>(s, b, c0, c1);
    }
    return s;
}

// A thread's running reference and sums, the sums in pairs.
template <int FORM> struct Running {
    float m = -FLT_MAX;
    f2 sT = 0, s1 = 0;  // two zeros

    // Keeps entries within `headroom` above the reference m: 0 makes m the maximum so far.
    __device__ __forceinline__ void raise(float top, float c0, float c1, float headroom)
    {
        if (top - m > headroom) {
            const Exps f = exps<FORM>(m - top, c0, c1);
            sT = mul2(sT, pack2(f.eT, f.eT));
            if (FORM) s1 = mul2(s1, pack2(f.e1, f.e1));
            m = top;
        }
    }
    // d: a pair of entries less the reference
    __device__ __forceinline__ void add(f2 d, f2 c0, f2 c1)
    {
        const f2 u = ex2_2(mul2(d, c0));
        if constexpr (FORM == kThreeHalves) {
            const f2 q = mul2(u, u);
            sT = add2(sT, q);
            s1 = fma2(q, u, s1);
        } else {
            sT = add2(sT, u);
        }
        if constexpr (FORM == kTwo) s1 = fma2(u, u, s1);
        if constexpr (FORM == kThree) s1 = fma2(mul2(u, u), u, s1);
        if constexpr (FORM == kFour) {
            const f2 q = mul2(u, u);
            s1 = fma2(q, q, s1);
        }
        if constexpr (FORM == kAnyT) s1 = add2(s1, ex2_2(mul2(d, c1)));
    }
    template <int N, typename ZT> __device__ __forceinline__ void absorb(const Piece<ZT> (&p)[N], float c0, float c1, float headroom)
    {
        float top = p[0].top();
#pragma unroll
        for (int u = 1; u < N; ++u) top = fmaxf(top, p[u].top());
        raise(top, c0, c1, headroom);
        const f2 c02 = pack2(c0, c0), c12 = pack2(c1, c1);
#pragma unroll
        for (int u = 0; u < N; ++u)
#pragma unroll
            for (int i = 0; i < Piece<ZT>::kPairs; ++i) add(p[u].less(i, m), c02, c12);
    }
    __device__ __forceinline__ Sums sums() const
    {
        float a, b, c, d;
        unpack2(sT, a, b);
        unpack2(s1, c, d);
        return {m, a + b, c + d};
    }
};

// A piece's logits become its gradient as if no list and no label named them:  kT e_T + k1 e_1.
template <int FORM, typename ZT> __device__ __forceinline__ void slopes(Piece<ZT> &p, float m, f2 c0, f2 c1, f2 kT, f2 k1)
{
#pragma unroll
    for (int i = 0; i < Piece<ZT>::kPairs; ++i) {
        const f2 d = p.less(i, m), u = ex2_2(mul2(d, c0));
        f2 g;
        if constexpr (FORM == kOneSum) g = mul2(kT, u);
        if constexpr (FORM == kTwo) g = mul2(u, fma2(k1, u, kT));
        if constexpr (FORM == kThree) g = mul2(u, fma2(k1, mul2(u, u), kT));
        if constexpr (FORM == kFour) g = mul2(u, fma2(k1, mul2(u, mul2(u, u)), kT));
        if constexpr (FORM == kThreeHalves) g = mul2(mul2(u, u), fma2(k1, u, kT));
        if constexpr (FORM == kAnyT) g = fma2(kT, u, mul2(k1, ex2_2(mul2(d, c1))));
        p.set(i, g);
    }
}
// The same of one entry.
template <int FORM> __device__ __forceinline__ float slope_of(float x, float m, float c0, float c1, float kT, float k1)
{
    const Exps e = exps<FORM>(x - m, c0, c1);
    return FORM ? fmaf(kT, e.eT, k1 * e.e1) : kT * e.eT;
}

// One row per cluster of 1, 2, 4 or 8 blocks; each block has a contiguous part of the vocabulary.
// First walk: maximum and sums, rescaled as the maximum grows, while the last warp turns the
// teacher's list into q.  Second walk (with a gradient): the part is read again - it is still in
// L2 - and the gradient of every entry written as if no list existed; then the few entries
// that the list or the label names are written again with their whole value.
template <typename ZT, int FORM, bool GRAD>
__global__ void __launch_bounds__(kThreads, GRAD ? kBlocks : 2 * kBlocks) k_distill_rows(const __grid_constant__ RowArgs a)
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
    const long long row = blockIdx.x >> a.log_parts;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const ZT *z = static_cast<const ZT *>(a.z) + row * a.ld_z;
    ZT *dz = GRAD ? static_cast<ZT *>(a.dz) + row * a.ld_dz : nullptr;

    // this block's part: 16-byte pieces [v0, v1) of the row's aligned middle; block 0 also has the
    // few entries before and after it
    const long long mis = (long long)((uintptr_t)z & 15) / (long long)sizeof(ZT);
    long long head = mis ? V - mis : 0;
    if (head > a.vocab) head = a.vocab;
    const int nv = (int)((unsigned long long)(a.vocab - head) / V);
    const int tail = (int)(a.vocab - head - (long long)nv * V);
    const int v0 = (int)((long long)nv * part >> a.log_parts), v1 = (int)((long long)nv * (part + 1) >> a.log_parts);
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
        Running<FORM> run;
        const uint4 *mid = reinterpret_cast<const uint4 *>(z + head);
        int v = v0 + tid;
        for (; v + (kUnroll - 1) * kThreads < v1; v += kUnroll * kThreads) {
            Piece<ZT> p[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) p[u].w = mid[v + u * kThreads];
            run.absorb(p, a.c0, a.c1, 0.f);
        }
        for (; v < v1; v += kThreads) {
            Piece<ZT> p[1];
            p[0].w = mid[v];
            run.absorb(p, a.c0, a.c1, 0.f);
        }
        Sums s = run.sums();
        if (tid < loose) s = join<FORM>(s, {to_f32(z[loose_at]), 1.f, 1.f}, a.c0, a.c1);
        s = join_lanes<FORM, 32>(s, a.c0, a.c1);
        if (lane == 0) warp_sums[warp] = s;
        __syncthreads();
        s = join_lanes<FORM, kWarps>(warp_sums[lane % kWarps], a.c0, a.c1);
        if (parts > 1) {
            if (tid < parts) *cluster.map_shared_rank(&block_sums[part], tid) = s;
            cluster.sync();
            s = block_sums[0];
            for (int r = 1; r < parts; ++r) s = join<FORM>(s, block_sums[r], a.c0, a.c1);
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
        if (a.dz == a.z) {  // all reads of named entries are done before any block writes
            if (parts > 1) cluster.sync();
            else __syncthreads();
        }
    }
    const bool nothing = kT == 0.f && k1 == 0.f;  // zeros, whatever the logits hold
    auto slope = [&](float x) {
        return slope_of<FORM>(x, m, a.c0, a.c1, kT, k1);
    };
    const uint4 *mid = reinterpret_cast<const uint4 *>(z + head);
    ZT *out = dz + head;
    const f2 c02 = pack2(a.c0, a.c0), c12 = pack2(a.c1, a.c1), kT2 = pack2(kT, kT), k12 = pack2(k1, k1);
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
    int v = v0 + tid;
    for (; v + (kUnroll - 1) * kThreads < v1; v += kUnroll * kThreads) {
        Piece<ZT> p[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) p[u].w = __ldcs(mid + v + u * kThreads);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            slopes<FORM>(p[u], m, c02, c12, kT2, k12);
            write(v + u * kThreads, p[u]);
        }
    }
    for (; v < v1; v += kThreads) {
        Piece<ZT> p;
        p.w = __ldcs(mid + v);
        slopes<FORM>(p, m, c02, c12, kT2, k12);
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
        bool first = true, in_list = false;
        float mass = 0.f;
        if (aT != 0.f) {
            for (int j = 0; j < a.k; ++j) {
                if (id[j] == i) {
                    if (j < k) first = false;
                    in_list = true;
                    mass += q[j];
                }
            }
        }
        if (!first) continue;
        float g = slope(is_label ? z_label : zk[k]);
        if (in_list) g -= list_scale * mass;  // NaN where the teacher's logits make q NaN
        if (i == label) g -= b1;
        put(dz + i, g);
    }
}

// ---------------------------------------------------------------------------------------------
// Rows kept in shared memory
// ---------------------------------------------------------------------------------------------
// The kernel above reads a row twice, the second time from L2, and a block does nothing else while a
// row's first pieces or its sums are on their way.  Here a row is read once: a block (or a cluster of
// them for rows that do not fit one) keeps it in a ring of shared-memory slots.  Five jobs run
// side by side and hand over through mbarriers:
//   loader    one thread: bulk copies of the next row's pieces into slots as they become free
//   lists     two or four warps, rows ahead, each its own: weight, label, the teacher's list turned into q
//   workers   four, eight or sixteen warps: maximum and sums as the pieces arrive; then the gradient of every entry, over the row in its slots
//   storer    one warp: the named entries' whole values into the slots, bulk copies out, slots back to the loader; the row's loss
// Every wait is bounded; a job that gives up leaves NaN as the row's loss and ends, and the others follow when their waits run
// out.  The storer, which no row passes by, then leaves NaN as the loss and in the block's part of the gradient of all rows to come.
constexpr int kStagedMaxK = 128;  // list entries: a lists' warp has a few rows' time for them
constexpr int kPiecesEach = 2;    // 16-byte pieces of a slot per worker thread

// Three shapes.  Four worker warps and four blocks per SM for short rows, whose time is the jobs' latency: more rows are
// on their way, and the jobs may be eight rows apart (8192 x 4000 bf16, K = 16: 55 us; eight warps 99; four rows apart 59,
// two 66; three blocks of fifteen slots 72).  Eight worker warps and two blocks per SM, where the ring takes a whole row: while
// one block joins its sums or waits for its row the other computes (323 us on 8192 x 50257 bf16, T = 2; one block of sixteen
// 360 before the forms of exps(), two blocks that share rows with another SM 420).  Sixteen and one block for longer rows, whose
// parts fill two thirds of the ring and leave the rest to the next row (2048 x 32768 f32: 93 us).
template <int WORKERS> struct Shape {
    static constexpr int kBlocks = 16 / WORKERS;                    // per SM
    static constexpr int kListWarps = WORKERS == 16 ? 4 : 2;
    static constexpr int kInfos = WORKERS == 8 ? 2 : 8;             // rows that the jobs may be apart: a power of two, a multiple of kListWarps
    static constexpr int kWorkerThreads = WORKERS * 32;
    static constexpr int kThreads = kWorkerThreads + (kListWarps + 2) * 32;
    static constexpr int kSlotPieces = kWorkerThreads * kPiecesEach;
    static constexpr int kSlotBytes = kSlotPieces * 16;
    static constexpr int kSlots = WORKERS == 4 ? 9 : WORKERS == 8 ? 13 : 12;
    static constexpr int kPartPieces = (WORKERS == 16 ? 8 : kSlots) * kSlotPieces;  // of a row that one block takes, at most
};
constexpr float kHeadroom = 40.f;                       // powers of two that an entry may exceed the reference by

struct RowInfo {
    float weight, z_label;
    float ref;                // largest of the named logits: near the row's maximum as a rule
    int label, live, has_list;
    // left by the workers
    float m, s1, sT, aT, b1, kT, k1;
    __align__(16) int id[kStagedMaxK];  // -1: not valid
    float q[kStagedMaxK];     // 0: not valid
    float mass[kStagedMaxK];  // q of all entries with this id, at the first of them; < 0 at the others
    float zk[kStagedMaxK];
    float loose[16];          // logits before and after the aligned pieces
};

template <int WORKERS> struct StagedShared {
    static constexpr int kSlots = Shape<WORKERS>::kSlots, kInfos = Shape<WORKERS>::kInfos;
    u64 full[kSlots], done[kSlots], empty[kSlots];
    u64 info_full[kInfos], info_empty[kInfos], stats_full[kInfos], sums_ready[2], exchange[2];
    Sums warp_sums[2][WORKERS];
    Sums block_sums[2][kMaxCluster];
    RowInfo info[kInfos];
};

template <typename ZT, int FORM, int kWorkers>
__global__ void __launch_bounds__(Shape<kWorkers>::kThreads, Shape<kWorkers>::kBlocks) k_distill_staged(const __grid_constant__ RowArgs a)
{
    typedef Shape<kWorkers> S;
    constexpr int V = 16 / sizeof(ZT), kWorkerThreads = S::kWorkerThreads, kListWarps = S::kListWarps, kInfos = S::kInfos, kSlots = S::kSlots,
                  kSlotPieces = S::kSlotPieces, kSlotBytes = S::kSlotBytes;
    extern __shared__ __align__(128) char ring[];
    __shared__ StagedShared<kWorkers> sh;
    cg::cluster_group cluster = cg::this_cluster();
    const int parts = (int)cluster.num_blocks(), part = (int)cluster.block_rank();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const long long first = blockIdx.x >> a.log_parts, step = gridDim.x >> a.log_parts;
    if (tid == 0) {
        for (int i = 0; i < kSlots; ++i) {
            mbar_init(sh.full + i, 1);
            mbar_init(sh.done + i, kWorkers);
            mbar_init(sh.empty + i, 1);
        }
        for (int b = 0; b < kInfos; ++b) {
            mbar_init(sh.info_full + b, 1);
            mbar_init(sh.info_empty + b, kWorkers + 2);
            mbar_init(sh.stats_full + b, 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(sh.sums_ready + b, kWorkers);
            mbar_init(sh.exchange + b, (unsigned)parts);
        }
        mbar_publish();
    }
    cluster.sync();
    griddep_wait();
    griddep_launch();

    // where a row's part lies
    struct Part {
        const ZT *z;
        long long head;  // entries before the aligned middle
        int nv, v0, v1;  // pieces of the middle; this block's
        int pieces;      // slots that they take
    };
    auto part_of = [&](long long row) {
        Part p;
        p.z = static_cast<const ZT *>(a.z) + row * a.ld_z;
        const int mis = (int)((uintptr_t)p.z & 15) / (int)sizeof(ZT);
        p.head = mis ? V - mis : 0;
        p.nv = (int)((unsigned long long)(a.vocab - p.head) / V);
        p.v0 = (int)((long long)p.nv * part >> a.log_parts);
        p.v1 = (int)((long long)p.nv * (part + 1) >> a.log_parts);
        p.pieces = (p.v1 - p.v0 + kSlotPieces - 1) / kSlotPieces;
        return p;
    };
    auto loose_of = [&](const Part &p) { return part == 0 ? (int)(a.vocab - (long long)p.nv * V) : 0; };  // fewer than 16
    auto loose_at = [&](const Part &p, int i) { return i < p.head ? (long long)i : (long long)p.nv * V + i; };
    auto lost = [&](long long row) { a.row_loss[row] = __int_as_float(0x7fffffff); };
    unsigned slot = 0, turn = 0;  // of the next piece, and the parity of the ring's round; every job counts for itself
    auto advance = [&]() {
        if (++slot == kSlots) {
            slot = 0;
            turn ^= 1;
        }
    };

    long long i = 0;  // rows of this cluster so far; row i uses info[i % kInfos]
    if (warp == kWorkers) {  // ---- loader
        long long asked = 0;
        bool ok = true;
        for (long long row = first; row < a.n && ok && lane == 0; row += step, ++i) {
            const int b = (int)i & (kInfos - 1);
            ok = mbar_wait(sh.info_full + b, (unsigned)i / kInfos & 1);
            if (ok && sh.info[b].live) {
                const Part p = part_of(row);
                for (int c = 0; c < p.pieces && ok; ++c, ++asked, advance()) {
                    if (asked >= kSlots) ok = mbar_wait(sh.empty + slot, turn ^ 1);
                    if (!ok) break;
                    const int at = p.v0 + c * kSlotPieces;
                    const unsigned bytes = 16u * (unsigned)min(kSlotPieces, p.v1 - at);
                    mbar_expect_tx(sh.full + slot, bytes);
                    bulk_load(ring + slot * kSlotBytes, p.z + p.head + (long long)at * V, bytes, sh.full + slot);
                }
            }
            if (!ok) lost(row);
            mbar_arrive(sh.info_empty + b);
        }
        if (!ok && lane == 0) {  // copies that may still be on their way
            for (int k = 0; k < kSlots && k < asked; ++k) {
                slot = slot ? slot - 1 : kSlots - 1;
                turn ^= slot == kSlots - 1;
                mbar_wait(sh.full + slot, turn);
            }
        }
    } else if (warp > kWorkers + 1) {  // ---- lists: warp l of them has rows l, l + kListWarps, ...
        constexpr int kMine = kStagedMaxK / 32;
        struct Raw {  // a row's inputs, asked for a row before they are needed
            float weight, t[kMine];
            long long label, id[kMine];
        };
        auto ask = [&](long long row, Raw &r) {
            if (row >= a.n) return;
            r.weight = a.weight ? a.weight[row] : 1.f;
            r.label = a.beta != 0.f && a.labels ? load_id(a.labels, a.wide_labels, row) : -1;
#pragma unroll
            for (int u = 0; u < kMine; ++u) {
                const int k = lane + 32 * u;
                r.id[u] = -1;
                r.t[u] = 0.f;
                if (k >= a.k || a.alpha == 0.f) continue;
                const long long at = row * a.ld_t + k;
                r.id[u] = load_id(a.ids, a.wide_ids, row * a.ld_ids + k);
                r.t[u] = a.t_bf16 ? to_f32(static_cast<const bf16 *>(a.t)[at]) : static_cast<const float *>(a.t)[at];
            }
        };
        Raw next;
        i = warp - (kWorkers + 2);
        ask(first + i * step, next);
        for (long long row = first + i * step; row < a.n; row += kListWarps * step, i += kListWarps) {
            const int b = (int)i & (kInfos - 1);
            RowInfo &f = sh.info[b];
            const ZT *z = static_cast<const ZT *>(a.z) + row * a.ld_z;
            const Raw r = next;
            ask(row + kListWarps * step, next);
            const int label = r.label >= 0 && r.label < a.vocab ? (int)r.label : -1;
            int id[kMine];
            float z_k[kMine], q[kMine], top = -FLT_MAX;
            bool any = false;
#pragma unroll
            for (int u = 0; u < kMine; ++u) {
                id[u] = r.weight != 0.f && r.id[u] >= 0 && r.id[u] < a.vocab && r.t[u] != -INFINITY ? (int)r.id[u] : -1;
                z_k[u] = id[u] >= 0 ? to_f32(z[id[u]]) : 0.f;
                any |= id[u] >= 0;
                if (id[u] >= 0) top = fmaxf(top, r.t[u]);
            }
            const float z_label = r.weight != 0.f && label >= 0 ? to_f32(z[label]) : 0.f;
            const Part p = part_of(row);
            const float z_loose = r.weight != 0.f && lane < loose_of(p) ? to_f32(z[loose_at(p, lane)]) : 0.f;
            any = __any_sync(0xffffffffu, any);
            top = warp_max(top);
            float sum = 0.f;
#pragma unroll
            for (int u = 0; u < kMine; ++u) {
                q[u] = id[u] >= 0 ? expf((r.t[u] - top) * a.invT) : 0.f;
                sum += q[u];
            }
            const float inv = 1.f / warp_sum(sum);
            if (i >= kInfos && !mbar_wait(sh.info_empty + b, ((unsigned)i / kInfos - 1) & 1)) {
                if (lane == 0) lost(row);
                break;
            }
#pragma unroll
            for (int u = 0; u < kMine; ++u) {
                q[u] = id[u] >= 0 ? q[u] * inv : 0.f;
                f.id[lane + 32 * u] = id[u];
                f.q[lane + 32 * u] = q[u];
                f.zk[lane + 32 * u] = z_k[u];
            }
            __syncwarp();
            // the first entry that has an id stands for all that have it; repetitions are rare
            bool again = false;
            const int4 *ids = reinterpret_cast<const int4 *>(f.id);
#pragma unroll 4
            for (int j = 0; j < (a.k + 3) / 4; ++j) {
                const int4 w = ids[j];
#pragma unroll
                for (int u = 0; u < kMine; ++u) {
                    const int k = lane + 32 * u, c = 4 * j;
                    again |= id[u] >= 0 && ((w.x == id[u] && c < k) | (w.y == id[u] && c + 1 < k) | (w.z == id[u] && c + 2 < k) | (w.w == id[u] && c + 3 < k));
                }
            }
            float mass[kMine];
#pragma unroll
            for (int u = 0; u < kMine; ++u) mass[u] = id[u] >= 0 ? q[u] : -1.f;
            if (__any_sync(0xffffffffu, again)) {
#pragma unroll
                for (int u = 0; u < kMine; ++u) {
                    const int k = lane + 32 * u;
                    if (id[u] < 0) continue;
                    mass[u] = 0.f;
                    for (int j = 0; j < a.k; ++j) {
                        if (f.id[j] != id[u]) continue;
                        if (j < k) mass[u] = -1.f;
                        if (mass[u] < 0.f) break;
                        mass[u] += f.q[j];
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < kMine; ++u) f.mass[lane + 32 * u] = mass[u];
            if (lane < 16) f.loose[lane] = z_loose;
            float ref = label >= 0 ? z_label : -FLT_MAX;
#pragma unroll
            for (int u = 0; u < kMine; ++u)
                if (id[u] >= 0) ref = fmaxf(ref, z_k[u]);
            ref = fmaxf(warp_max(ref), -FLT_MAX);
            if (lane == 0) {
                f.weight = r.weight;
                f.ref = ref;
                f.label = label;
                f.has_list = any;
                f.live = r.weight != 0.f && (label >= 0 || any);
                f.z_label = z_label;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(sh.info_full + b);
        }
    } else if (warp == kWorkers + 1) {  // ---- storer
        int unread = -1;  // slot whose copy out may still be reading
        for (long long row = first; row < a.n; row += step, ++i) {
            const int b = (int)i & (kInfos - 1);
            RowInfo &f = sh.info[b];
            bool ok = mbar_wait(sh.info_full + b, (unsigned)i / kInfos & 1);
            if (ok && !f.live) {
                if (lane == 0 && part == 0) a.row_loss[row] = 0.f;
            } else if (ok) {
                const Part p = part_of(row);
                ZT *dz = static_cast<ZT *>(a.dz) + row * a.ld_dz;
                const int loose = loose_of(p);
                const float z_loose = lane < loose ? f.loose[lane] : 0.f;
                ok = mbar_wait(sh.stats_full + b, (unsigned)i / kInfos & 1);
                const float m = f.m, kT = f.kT, k1 = f.k1, aT = f.aT, b1 = f.b1;
                auto slope = [&](float x) {
                    return slope_of<FORM>(x, m, a.c0, a.c1, kT, k1);
                };
                const bool nothing = kT == 0.f && k1 == 0.f;
                if (lane < loose) put(dz + loose_at(p, lane), nothing ? 0.f : slope(z_loose));
                __syncwarp();
                // whole values of the named entries: where in this part they lie (-1: not in its slots), and what
                constexpr int kMine = kStagedMaxK / 32 + 1;
                int where[kMine];
                float value[kMine];
#pragma unroll
                for (int u = 0; u < kMine; ++u) {
                    const bool is_label = u == kMine - 1;
                    const int k = lane + 32 * u;
                    where[u] = -1;
                    value[u] = 0.f;
                    long long at = -1;
                    float mass = 0.f, x = 0.f;
                    if (is_label) {
                        if (lane == 0) at = f.label;
                        x = f.z_label;
                    } else if (k < a.k && aT != 0.f && !(f.mass[k] < 0.f)) {  // NaN counts
                        at = f.id[k];
                        mass = f.mass[k];
                        x = f.zk[k];
                    }
                    bool in_list = false;  // the label's entry is the list's business if the list names it
                    if (is_label && aT != 0.f) {
                        bool mine = false;
                        for (int j = lane; j < a.k; j += 32) mine |= f.id[j] == f.label;
                        in_list = __any_sync(0xffffffffu, mine);
                    }
                    if (at < 0 || in_list || nothing) continue;
                    value[u] = slope(x) - aT * mass;
                    if (at == f.label) value[u] -= b1;
                    const long long middle = at - p.head;
                    if (middle < 0 || middle >= (long long)p.nv * V) {
                        if (part == 0) put(dz + at, value[u]);
                    } else if (middle >= (long long)p.v0 * V && middle < (long long)p.v1 * V) {
                        where[u] = (int)(middle - (long long)p.v0 * V);
                    }
                }
                constexpr int slot_entries = kSlotPieces * V;
                for (int c = 0; c < p.pieces && ok; ++c, advance()) {
                    ok = mbar_wait(sh.done + slot, turn);
                    if (!ok) break;
                    ZT *data = reinterpret_cast<ZT *>(ring + slot * kSlotBytes);
#pragma unroll
                    for (int u = 0; u < kMine; ++u) {
                        const int at = where[u] - c * slot_entries;
                        if (where[u] >= 0 && at >= 0 && at < slot_entries) put(data + at, value[u]);
                    }
                    copy_fence();
                    __syncwarp();
                    if (lane == 0) {
                        const int at = p.v0 + c * kSlotPieces;
                        bulk_store(dz + p.head + (long long)at * V, data, 16u * (unsigned)min(kSlotPieces, p.v1 - at));
                        bulk_commit();
                        if (unread >= 0) {
                            bulk_wait_read<1>();
                            mbar_arrive(sh.empty + unread);
                        }
                        unread = (int)slot;
                    }
                }
                if (part == 0) {
                    float loss = 0.f;
                    if (aT != 0.f) {
                        for (int k = lane; k < a.k; k += 32) {
                            const float q = f.q[k];
                            if (q != 0.f) loss += q * (logf(q) - (f.zk[k] - m) * a.invT);
                        }
                        loss = (warp_sum(loss) + logf(f.sT)) * a.T * aT;
                    }
                    if (b1 != 0.f) loss += b1 * (logf(f.s1) - (f.z_label - m));
                    if (lane == 0) a.row_loss[row] = loss;
                }
                if (lane == 0 && unread >= 0) {  // the row's last
                    bulk_wait_read<0>();
                    mbar_arrive(sh.empty + unread);
                    unread = -1;
                }
            }
            if (!ok) {
                if (lane == 0) bulk_wait_all();
                __syncwarp();
                for (; row < a.n; row += step) {
                    const Part p = part_of(row);
                    ZT *dz = static_cast<ZT *>(a.dz) + row * a.ld_dz;
                    for (long long v = (long long)p.v0 * V + lane; v < (long long)p.v1 * V; v += 32) put(dz + p.head + v, __int_as_float(0x7fffffff));
                    if (lane < loose_of(p)) put(dz + loose_at(p, lane), __int_as_float(0x7fffffff));
                    if (lane == 0) lost(row);
                }
                break;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(sh.info_empty + b);
        }
        if (lane == 0) bulk_wait_all();
    } else {  // ---- workers
        long long live_rows = 0;  // sums and exchanges alternate over these
        for (long long row = first; row < a.n; row += step, ++i) {
            const int b = (int)i & (kInfos - 1);
            RowInfo &f = sh.info[b];
            if (!mbar_wait(sh.info_full + b, (unsigned)i / kInfos & 1)) break;
            const Part p = part_of(row);
            if (!f.live) {  // zeros, and nothing is read
                ZT *dz = static_cast<ZT *>(a.dz) + row * a.ld_dz;
                for (int v = p.v0 + tid; v < p.v1; v += kWorkerThreads) __stcs(reinterpret_cast<uint4 *>(dz + p.head) + v, make_uint4(0, 0, 0, 0));
                if (tid < loose_of(p)) put(dz + loose_at(p, tid), 0.f);
                if (tid == 0) mbar_arrive(sh.stats_full + b);  // its phases go by rows
                __syncwarp();
                if (lane == 0) mbar_arrive(sh.info_empty + b);
                continue;
            }
            const int e = (int)(live_rows & 1);
            const unsigned e_parity = (unsigned)(live_rows >> 1) & 1;
            ++live_rows;
            const unsigned slot0 = slot;
            Running<FORM> run;
            const float ref = f.ref;
            run.m = ref;
            const bool loose = tid < loose_of(p);
            const float z_loose = loose ? f.loose[tid] : 0.f;
            const int mine = p.v1 - p.v0;  // pieces
            bool ok = true;
            for (int c = 0; c < p.pieces; ++c, advance()) {
                ok &= mbar_wait(sh.full + slot, turn);
                const uint4 *data = reinterpret_cast<const uint4 *>(ring + slot * kSlotBytes) + tid;
                const int have = mine - c * kSlotPieces;
                if (have >= kSlotPieces) {
                    Piece<ZT> q[kPiecesEach];
#pragma unroll
                    for (int u = 0; u < kPiecesEach; ++u) q[u].w = data[u * kWorkerThreads];
                    run.absorb(q, a.c0, a.c1, a.headroom);
                } else {
#pragma unroll
                    for (int u = 0; u < kPiecesEach; ++u) {
                        if (tid + u * kWorkerThreads >= have) break;
                        Piece<ZT> q[1];
                        q[0].w = data[u * kWorkerThreads];
                        run.absorb(q, a.c0, a.c1, a.headroom);
                    }
                }
            }
            // As a rule no entry exceeded the reference by the headroom and all sums are relative to it: they only have to be added.
            Sums s = run.sums();
            if (loose) s = join<FORM>(s, {z_loose, 1.f, 1.f}, a.c0, a.c1);
            s = join_lanes<FORM, 32>(s, a.c0, a.c1);
            if (lane == 0) {
                sh.warp_sums[e][warp] = s;
                mbar_arrive(sh.sums_ready + e);
            }
            ok &= mbar_wait(sh.sums_ready + e, e_parity);
            s = join_lanes<FORM, kWorkers>(sh.warp_sums[e][lane % kWorkers], a.c0, a.c1);
            if (parts > 1) {  // every block tells every block of the cluster, itself included
                if (tid < parts) {
                    *cluster.map_shared_rank(&sh.block_sums[e][part], tid) = s;
                    asm volatile("{\n\t.reg .b32 r;\n\tmapa.shared::cluster.u32 r, %0, %1;\n\tmbarrier.arrive.release.cluster.shared::cluster.b64 _, [r];\n\t}" ::"r"(
                                     smem_u32(sh.exchange + e)),
                                 "r"(tid)
                                 : "memory");
                }
                ok &= mbar_wait<true>(sh.exchange + e, e_parity);
                s = sh.block_sums[e][0];
                for (int r = 1; r < parts; ++r) s = join<FORM>(s, sh.block_sums[e][r], a.c0, a.c1);
            }
            if (!ok) break;
            const bool has_logits = s.sT != 0.f;  // NaN counts; 0 when all are -inf
            const float s1 = a.one_sum ? s.sT : s.s1, m = s.m;
            const float aT = f.has_list && has_logits ? f.weight * a.alpha * a.T : 0.f, b1 = f.label >= 0 && has_logits ? f.weight * a.beta : 0.f;
            float kT = aT != 0.f ? aT / s.sT : 0.f, k1 = b1 != 0.f ? b1 / s1 : 0.f;
            if (a.one_sum) {
                kT += k1;
                k1 = 0.f;
            }
            if (tid == 0) {
                f.m = m;
                f.sT = s.sT;
                f.s1 = s1;
                f.aT = aT;
                f.b1 = b1;
                f.kT = kT;
                f.k1 = k1;
                mbar_arrive(sh.stats_full + b);
            }
            const bool nothing = kT == 0.f && k1 == 0.f;
            const f2 c02 = pack2(a.c0, a.c0), c12 = pack2(a.c1, a.c1), kT2 = pack2(kT, kT), k12 = pack2(k1, k1);
            unsigned out = slot0;
            for (int c = 0; c < p.pieces; ++c, out = out + 1 == kSlots ? 0 : out + 1) {
                uint4 *data = reinterpret_cast<uint4 *>(ring + out * kSlotBytes) + tid;
                const int have = mine - c * kSlotPieces;
                if (nothing) {
#pragma unroll
                    for (int u = 0; u < kPiecesEach; ++u)
                        if (tid + u * kWorkerThreads < have) data[u * kWorkerThreads] = make_uint4(0, 0, 0, 0);
                } else if (have >= kSlotPieces) {
                    Piece<ZT> q[kPiecesEach];
#pragma unroll
                    for (int u = 0; u < kPiecesEach; ++u) q[u].w = data[u * kWorkerThreads];
#pragma unroll
                    for (int u = 0; u < kPiecesEach; ++u) {
                        slopes<FORM>(q[u], m, c02, c12, kT2, k12);
                        data[u * kWorkerThreads] = q[u].w;
                    }
                } else {
#pragma unroll
                    for (int u = 0; u < kPiecesEach; ++u) {
                        if (tid + u * kWorkerThreads >= have) break;
                        Piece<ZT> q;
                        q.w = data[u * kWorkerThreads];
                        slopes<FORM>(q, m, c02, c12, kT2, k12);
                        data[u * kWorkerThreads] = q.w;
                    }
                }
                copy_fence();
                __syncwarp();
                if (lane == 0) mbar_arrive(sh.done + out);
            }
            if (lane == 0) mbar_arrive(sh.info_empty + b);
        }
    }
    __syncwarp();
    cluster.sync();  // no block leaves while another may still write to its shared memory
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

template <typename ZT, int FORM> cudaError_t launch_rows(const RowArgs &a, int parts, cudaStream_t s)
{
    return a.dz ? launch(k_distill_rows<ZT, FORM, true>, a.n * parts, kThreads, 0, s, a, parts)
                : launch(k_distill_rows<ZT, FORM, false>, a.n * parts, kThreads, 0, s, a, parts);
}

template <typename ZT, int FORM, int WORKERS> cudaError_t launch_staged(const RowArgs &a, int parts, int sms, cudaStream_t s)
{
    typedef Shape<WORKERS> S;
    constexpr size_t smem = (size_t)S::kSlots * S::kSlotBytes;
    static OncePerDevice known;
    const cudaError_t e = allow_smem(reinterpret_cast<const void *>(&k_distill_staged<ZT, FORM, WORKERS>), known);
    if (e != cudaSuccess) return e;
    const int most = sms * S::kBlocks / parts;
    return launch(k_distill_staged<ZT, FORM, WORKERS>, (a.n < most ? a.n : most) * parts, S::kThreads, smem, s, a, parts);
}
template <typename ZT, int WORKERS> cudaError_t launch_staged(const RowArgs &a, int form, int parts, int sms, cudaStream_t s)
{
    switch (form) {
    case kOneSum: return launch_staged<ZT, kOneSum, WORKERS>(a, parts, sms, s);
    case kTwo: return launch_staged<ZT, kTwo, WORKERS>(a, parts, sms, s);
    case kThree: return launch_staged<ZT, kThree, WORKERS>(a, parts, sms, s);
    case kFour: return launch_staged<ZT, kFour, WORKERS>(a, parts, sms, s);
    case kThreeHalves: return launch_staged<ZT, kThreeHalves, WORKERS>(a, parts, sms, s);
    }
    return launch_staged<ZT, kAnyT, WORKERS>(a, parts, sms, s);
}

// Rows in shared memory where a gradient is asked for, its rows lie as the logits' do and the lists are
// not long; and where it measured faster than reading them twice (us; staged, twice):
//   rows, 50257 bf16: 900: 50, 51; 1200: 61, 68; 450: 33, 27.  32768 f32: 900: 50, 57; 450: 31, 28.  1000 bf16: 1200: 12, 14; 600: 10, 10; 300: 9, 6
//   length, 8192 rows bf16: 8000: 80, 161; 520: 42, 57; 200: 42, 56
//   blocks that share a row: two: 177, 191 (2048 x 50257 f32); four: 620, 464 (2048 x 120000 f32)
//   two evaluations an entry (T = 1.3): bf16 472, 441; f32 98, 117
constexpr int kStagedRows = 6;     // per SM
constexpr int kStagedLeast = 16;   // pieces of a row
constexpr int kStagedParts = 2;
template <typename ZT> bool staged(RowArgs a, int form, int sms, cudaStream_t s, cudaError_t &e)
{
    const long long pieces = a.vocab / (16 / (long long)sizeof(ZT));
    if (!a.dz || !a.aligned_out || a.k > kStagedMaxK || a.n < (long long)sms * kStagedRows || pieces < kStagedLeast ||
        pieces > (long long)kStagedParts * Shape<16>::kPartPieces || (form == kAnyT && sizeof(ZT) == 2))
        return false;
    if (pieces <= Shape<4>::kPartPieces) {
        e = launch_staged<ZT, 4>(a, form, 1, sms, s);
        return true;
    }
    if (pieces <= Shape<8>::kPartPieces) {
        e = launch_staged<ZT, 8>(a, form, 1, sms, s);
        return true;
    }
    int parts = 1;
    while (ceil_div(pieces, parts) > Shape<16>::kPartPieces) {
        parts *= 2;
        ++a.log_parts;
    }
    e = launch_staged<ZT, 16>(a, form, parts, sms, s);
    return true;
}

template <typename ZT> cudaError_t launch_rows(const RowArgs &a, int form, int parts, cudaStream_t s)
{
    switch (form) {
    case kOneSum: return launch_rows<ZT, kOneSum>(a, parts, s);
    case kTwo: return launch_rows<ZT, kTwo>(a, parts, s);
    case kThree: return launch_rows<ZT, kThree>(a, parts, s);
    case kFour: return launch_rows<ZT, kFour>(a, parts, s);
    case kThreeHalves: return launch_rows<ZT, kThreeHalves>(a, parts, s);
    }
    return launch_rows<ZT, kAnyT>(a, parts, s);
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
        a.one_sum = only_beta || a.beta == 0.f || g->temperature == 1.f;
        const float T = g->temperature;
        const int form = a.one_sum ? kOneSum : T == 2.f ? kTwo : T == 3.f ? kThree : T == 4.f ? kFour : T == 1.5f ? kThreeHalves : kAnyT;
        const double cT = only_beta ? log2e : log2e / (double)T;
        a.c0 = (float)(form == kThreeHalves ? log2e / 3.0 : cT);
        a.headroom = (float)(kHeadroom / (cT > log2e ? cT : log2e));
        a.aligned_out = g->dlogits && ((uintptr_t)g->dlogits - (uintptr_t)g->logits) % 16 == 0 &&
                        (g->n_rows <= 1 || (g->ld_dlogits - g->ld_logits) * ez % 16 == 0);
        cudaError_t e = cudaSuccess;
        if (g->dtype == ADASCALE_F32 ? staged<float>(a, form, sms, s, e) : staged<bf16>(a, form, sms, s, e)) {
            OPS_CU(e);
            OPS_CU(launch(k_total, 1, 1024, 0, s, TotalArgs{g->row_loss, g->loss, g->n_rows}));
            return ADASCALE_OK;
        }
        int parts = 1;  // few rows: several blocks share one
        while (parts < kMaxCluster && g->n_rows * parts * 2 <= sms && g->vocab >= 4096 * parts) {
            parts *= 2;
            ++a.log_parts;
        }
        OPS_CU(g->dtype == ADASCALE_F32 ? launch_rows<float>(a, form, parts, s) : launch_rows<bf16>(a, form, parts, s));
    }
    TotalArgs t = {g->row_loss, g->loss, g->n_rows};
    OPS_CU(launch(k_total, 1, 1024, 0, s, t));
    return ADASCALE_OK;
}

}  // extern "C"
