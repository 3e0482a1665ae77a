// Token table: scaled lookup, and its gradient by sorted tokens (adascale_embed, adascale_embed_grad).
#include "ops_common.cuh"

#include <cooperative_groups.h>

namespace {

namespace cg = cooperative_groups;

// ---------------------------------------------------------------------------------------------
// lookup
// ---------------------------------------------------------------------------------------------

struct LookupArgs {
    const void *tokens, *table;
    void *out;
    long long n, vocab, ld_table, ld_out;
    int wide, nv;  // 64-bit ids; vectors of a row
    float scale;
};

constexpr int kLookupThreads = 256;

// One warp per row: V elements per lane and access, every access of the row requested before the
// first is used (up to four), so the two dependent round trips to memory (id, then row) are paid
// once per warp and covered by the other 63 warps of the SM.
template <typename TT, typename OT, int V>
__global__ void __launch_bounds__(kLookupThreads) k_lookup(const __grid_constant__ LookupArgs a)
{
    griddep_wait();
    const long long row = (long long)blockIdx.x * (kLookupThreads / 32) + (threadIdx.x >> 5);
    if (row >= a.n) return;
    const int lane = threadIdx.x & 31;
    const long long id = load_id(a.tokens, a.wide, row);
    const bool known = id >= 0 && id < a.vocab;
    const TT *src = static_cast<const TT *>(a.table) + (known ? id : 0) * a.ld_table;
    OT *dst = static_cast<OT *>(a.out) + row * a.ld_out;
    for (int j0 = lane; j0 < a.nv; j0 += 128) {
        float x[4][V];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int j = j0 + 32 * u;
            if (known && j < a.nv) {
                load_vec<V>(src + (long long)j * V, x[u]);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) x[u][i] = 0.f;
            }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int j = j0 + 32 * u;
            if (j >= a.nv) break;
            if (known) {
#pragma unroll
                for (int i = 0; i < V; ++i) x[u][i] *= a.scale;
            }
            store_vec<V>(dst + (long long)j * V, x[u]);
        }
    }
}

// ---------------------------------------------------------------------------------------------
// gradient
// ---------------------------------------------------------------------------------------------
// Three launches: sort the tokens (one cluster) while all other clusters write the rows of absent
// tokens; sum the rows of dout window by window of the sorted order; join the pieces of
// the tokens that fill whole windows.

struct Pair {
    int key;  // token; the vocabulary's size stands for "no part in the gradient"
    int pos;  // where in the batch
};

constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortCluster = 8;      // portable cluster size
constexpr int kSortBits = 8;         // digit of one pass
constexpr int kSortBins = 1 << kSortBits;
constexpr int kZeroRun = 16;         // adjacent vocabulary rows that belong to one block of the zero-fill
constexpr int kZeroBits = 32 * 1024; // rows that a block keeps presence bits of at a time
constexpr int kWindow = 64;          // sorted entries of one window
constexpr int kSumThreads = 128;

struct SortArgs {
    const void *tokens;
    Pair *buf[2];       // ping-pong; the result is in buf[passes & 1]
    void *grad;
    long long n, vocab, ld_grad, padding;
    long long row_bytes;  // of the gradient; its rows are zeroed where no token points
    int wide, passes;
    int zero_blocks;    // blocks after the sorting cluster; 0 when accumulating
    int grad_bytes;     // bytes of a gradient element
    int vec;            // gradient rows can be written in 16-byte pieces
};

__device__ __forceinline__ int key_of(const SortArgs &a, long long i)
{
    const long long id = load_id(a.tokens, a.wide, i);
    return id >= 0 && id < a.vocab && id != a.padding ? (int)id : (int)a.vocab;
}

// Zeros for the rows that no token names.  Block z of Z has the vocabulary rows whose run number
// (row / kZeroRun) is z modulo Z, so that a batch that uses only frequent, adjacent ids still
// spreads evenly.  It marks the present ones in a bit field while it reads the whole list of
// tokens (from L2: the list is small beside what is written), then writes the others.
__device__ void zero_absent(const SortArgs &a, unsigned *bits, int z)
{
    const int Z = a.zero_blocks;
    const long long runs = ceil_div(a.vocab, kZeroRun);
    const long long mine = z < runs ? (runs - 1 - z) / Z + 1 : 0;  // runs of this block
    constexpr int kRuns = kZeroBits / kZeroRun;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (long long r0 = 0; r0 < mine; r0 += kRuns) {
        const int here = (int)(mine - r0 < kRuns ? mine - r0 : kRuns);
        __syncthreads();
        for (int i = threadIdx.x; i < (here * kZeroRun + 31) / 32; i += kSortThreads) bits[i] = 0u;
        __syncthreads();
        for (long long i = threadIdx.x; i < a.n; i += kSortThreads) {
            const unsigned key = (unsigned)key_of(a, i), run = key / kZeroRun;
            if (run % (unsigned)Z != (unsigned)z) continue;
            const long long local = (long long)(run / (unsigned)Z) - r0;
            if (local < 0 || local >= here) continue;
            const int b = (int)local * kZeroRun + (int)(key % kZeroRun);
            atomicOr(&bits[b >> 5], 1u << (b & 31));
        }
        __syncthreads();
        for (int b = warp; b < here * kZeroRun; b += kSortWarps) {
            if (bits[b >> 5] >> (b & 31) & 1u) continue;
            const long long row = ((r0 + b / kZeroRun) * Z + z) * kZeroRun + b % kZeroRun;
            if (row >= a.vocab) continue;
            char *p = static_cast<char *>(a.grad) + row * a.ld_grad * a.grad_bytes;
            if (a.vec) {
                for (long long j = lane; j < a.row_bytes / 16; j += 32) reinterpret_cast<uint4 *>(p)[j] = make_uint4(0, 0, 0, 0);
            } else if (a.grad_bytes == 4) {
                for (long long j = lane; j < a.row_bytes / 4; j += 32) reinterpret_cast<unsigned *>(p)[j] = 0u;
            } else {
                for (long long j = lane; j < a.row_bytes / 2; j += 32) reinterpret_cast<unsigned short *>(p)[j] = 0;
            }
        }
    }
}

// Stable radix sort of (token, position) by token, least significant digit first, by the eight
// blocks of one cluster.  Every warp owns a contiguous stretch of the current order.  Per pass: it
// counts its stretch's digits in shared memory (match_any groups equal digits of 32 entries, one
// lane adds the group's size: no atomics, and the order within a group is the lane order), the
// counts are turned into first destinations (over digits, blocks and warps in that order; block
// totals travel through distributed shared memory), and a second walk over the stretch writes
// each entry to its place.  The list stays in L2; what a pass costs is two cluster barriers
// and one scattered 8-byte store per entry.
__global__ void __launch_bounds__(kSortThreads, 1) k_sort_tokens(const __grid_constant__ SortArgs a)
{
    __shared__ unsigned count[kSortWarps][kSortBins];  // also the bit field of the zero-fill
    __shared__ unsigned total[kSortBins];              // of this block, read by the whole cluster
    __shared__ unsigned scan[kSortBins / 32];
    static_assert(sizeof(count) * 8 >= kZeroBits, "the zero-fill's bits fit");
    griddep_wait();
    griddep_launch();
    if (blockIdx.x >= kSortCluster) {
        zero_absent(a, &count[0][0], blockIdx.x - kSortCluster);
        return;
    }
    cg::cluster_group cluster = cg::this_cluster();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, rank = (int)blockIdx.x;
    const unsigned below = (1u << lane) - 1u;
    const long long stretch = ceil_div(ceil_div(a.n, kSortCluster * kSortWarps), 32) * 32;
    const long long first = ((long long)rank * kSortWarps + warp) * stretch;
    const long long last = first + stretch < a.n ? first + stretch : a.n;

    for (int pass = 0; pass < a.passes; ++pass) {
        const Pair *src = a.buf[pass & 1];
        Pair *dst = a.buf[(pass + 1) & 1];
        const int shift = pass * kSortBits;
        for (int i = lane; i < kSortBins; i += 32) count[warp][i] = 0u;
        __syncwarp();
        for (long long i0 = first; i0 < last; i0 += 32) {
            const long long i = i0 + lane;
            const bool has = i < last;
            const int key = !has ? 0 : pass ? __ldcg(&src[i].key) : key_of(a, i);
            const unsigned digit = has ? (unsigned)key >> shift & (kSortBins - 1) : kSortBins;
            const unsigned same = __match_any_sync(0xffffffffu, digit);
            if (has && !(same & below)) count[warp][digit] += __popc(same);
            __syncwarp();
        }
        __syncthreads();
        unsigned sum = 0;
        if (tid < kSortBins) {  // exclusive prefix over the block's warps; the block's total
            for (int w = 0; w < kSortWarps; ++w) {
                const unsigned c = count[w][tid];
                count[w][tid] = sum;
                sum += c;
            }
            total[tid] = sum;
        }
        cluster.sync();
        unsigned before = 0, all = 0;  // entries with this digit in earlier blocks, in the cluster
        if (tid < kSortBins) {
#pragma unroll
            for (int r = 0; r < kSortCluster; ++r) {
                const unsigned c = *cluster.map_shared_rank(&total[tid], r);
                before += r < rank ? c : 0u;
                all += c;
            }
            unsigned run = all;  // inclusive prefix over the digits: within the warp, then over the 8 warps
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const unsigned up = __shfl_up_sync(0xffffffffu, run, o);
                if (lane >= o) run += up;
            }
            if (lane == 31) scan[warp] = run;
            before += run - all;
        }
        __syncthreads();
        if (tid < kSortBins) {
            for (int w = 0; w < warp; ++w) before += scan[w];
            for (int w = 0; w < kSortWarps; ++w) count[w][tid] += before;
        }
        __syncthreads();
        for (long long i0 = first; i0 < last; i0 += 32) {
            const long long i = i0 + lane;
            const bool has = i < last;
            Pair p;
            if (has && pass) {
                const int2 q = __ldcg(reinterpret_cast<const int2 *>(src) + i);
                p.key = q.x;
                p.pos = q.y;
            } else {
                p.key = has ? key_of(a, i) : 0;
                p.pos = (int)i;
            }
            const unsigned digit = has ? (unsigned)p.key >> shift & (kSortBins - 1) : kSortBins;
            const unsigned same = __match_any_sync(0xffffffffu, digit);
            const unsigned at = has ? count[warp][digit] + __popc(same & below) : 0u;
            __syncwarp();
            if (has && !(same & below)) count[warp][digit] += __popc(same);
            if (has) reinterpret_cast<int2 *>(dst)[at] = make_int2(p.key, p.pos);
            __syncwarp();
        }
        // the next pass reads what all blocks wrote (and their totals are free again)
        __threadfence();
        cluster.sync();
    }
}

struct SumArgs {
    const Pair *sorted;
    const void *dout;
    void *grad;
    float *pieces;      // [windows][2][ld_piece]: a window's part of a long run: 0 one that began earlier, 1 one that begins here
    long long n, vocab, ld_dout, ld_grad, ld_piece;
    int nv;             // vectors of a row
    int accumulate;
    float scale;
};

template <typename GT, int V>
__device__ __forceinline__ void write_row(const SumArgs &a, int key, int c, float (&acc)[V])
{
    GT *p = static_cast<GT *>(a.grad) + (long long)key * a.ld_grad + (long long)c * V;
    float out[V];
    if (a.accumulate) {
        load_vec<V>(p, out);
#pragma unroll
        for (int i = 0; i < V; ++i) out[i] = fmaf(a.scale, acc[i], out[i]);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) out[i] = a.scale * acc[i];
    }
    store_vec<V>(p, out);
}

// A run of equal tokens that crosses at most one window boundary is short: the window in which it
// begins sums it to its end and writes its row.  One that crosses two or more is long: every window
// that it touches leaves the sum of its part, and k_join adds those up in order.  So no window
// sums more than two windows' entries, however the tokens are distributed, and both sides of a
// boundary decide from a few keys, without knowing where the run begins or ends:
//   at the front of window [a, b):  long  <=>  it fills the window too (key[b] is the same), or key[a-kWindow-1] is the same
//   at its back:                    long  <=>  key[a-1] is the same, or key[b+kWindow] is the same
__device__ __forceinline__ bool same_key(const Pair *s, long long n, long long i, int key)
{
    return i >= 0 && i < n && s[i].key == key;
}

// One thread per window and vector of 16 bytes of dout.
template <typename DT, typename GT, int V>
__global__ void __launch_bounds__(kSumThreads) k_sum_windows(const __grid_constant__ SumArgs a)
{
    griddep_wait();
    const long long t = (long long)blockIdx.x * kSumThreads + threadIdx.x;
    const long long w = t / a.nv;
    const int c = (int)(t % a.nv);
    const long long lo = w * kWindow, hi = lo + kWindow < a.n ? lo + kWindow : a.n;
    if (lo >= a.n) return;
    const Pair *s = a.sorted;
    long long i = lo;
    int key = s[lo].key;
    bool head = same_key(s, a.n, lo - 1, key);  // the run at the front began earlier
    const bool head_long = head && (same_key(s, a.n, hi, key) || same_key(s, a.n, lo - kWindow - 1, key));
    if (key >= a.vocab) return;
    if (head && !head_long) {  // another window's: on to the run after it
        long long past = hi;
        while (i < past) {
            const long long mid = (i + past) / 2;
            if (s[mid].key == key)
                i = mid + 1;
            else
                past = mid;
        }
        if (i == hi) return;
        key = s[i].key;
        if (key >= a.vocab) return;
        head = false;
    }
    const int back = s[hi - 1].key;
    const bool crosses = same_key(s, a.n, hi, back);
    const bool back_long = crosses && (same_key(s, a.n, lo - 1, back) || same_key(s, a.n, hi + kWindow, back));
    const long long end = crosses && !back_long ? (hi + kWindow < a.n ? hi + kWindow : a.n) : hi;

    float acc[V];
#pragma unroll
    for (int e = 0; e < V; ++e) acc[e] = 0.f;
    const DT *dout = static_cast<const DT *>(a.dout) + (long long)c * V;
    bool done = false;
    constexpr int U = 4;  // rows requested together
    for (; i < end && !done; i += U) {
        int2 p[U];
        float x[U][V];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            p[u] = i + u < end ? reinterpret_cast<const int2 *>(s)[i + u] : make_int2(-1, 0);
            if (i + u >= hi && p[u].x != back) p[u].x = -1;  // past the window only its last run may go on
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p[u].x >= 0 && p[u].x < a.vocab) load_vec<V>(dout + (long long)p[u].y * a.ld_dout, x[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (done || i + u >= end) continue;
            if (p[u].x != key) {  // the run ends here
                if (key < a.vocab) {
                    if (head)
                        store_vec<V>(a.pieces + 2 * w * a.ld_piece + (long long)c * V, acc);
                    else
                        write_row<GT, V>(a, key, c, acc);
                }
                head = false;
                key = p[u].x;
                done = key < 0 || key >= a.vocab;
#pragma unroll
                for (int e = 0; e < V; ++e) acc[e] = 0.f;
            }
            if (!done) {
#pragma unroll
                for (int e = 0; e < V; ++e) acc[e] += x[u][e];
            }
        }
    }
    if (done) return;
    if (head || back_long)
        store_vec<V>(a.pieces + (2 * w + (head ? 0 : 1)) * a.ld_piece + (long long)c * V, acc);
    else
        write_row<GT, V>(a, key, c, acc);
}

// The rows of long runs: block (w, slab) has the run that begins in window w, if one does.
template <typename GT, int V>
__global__ void __launch_bounds__(kSumThreads) k_join(const __grid_constant__ SumArgs a)
{
    griddep_wait();
    const long long slabs = (a.nv + 31) / 32;
    const long long w = blockIdx.x / slabs;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    constexpr int kWarps = kSumThreads / 32;
    const int c = (int)(blockIdx.x % slabs) * 32 + lane;
    const long long lo = w * kWindow, hi = lo + kWindow;
    const Pair *s = a.sorted;
    if (hi >= a.n) return;
    const int key = s[hi - 1].key;
    if (key >= a.vocab || same_key(s, a.n, lo - 1, key) || !same_key(s, a.n, hi, key) || !same_key(s, a.n, hi + kWindow, key)) return;
    // windows that the run touches: w .. last
    long long last = w + 2;
    for (;;) {  // 32 windows at a time
        const long long v = last + 1 + lane;
        const unsigned goes_on = __ballot_sync(0xffffffffu, same_key(s, a.n, v * kWindow, key));
        const int more = goes_on == 0xffffffffu ? 32 : __ffs(~goes_on) - 1;
        last += more;
        if (more < 32) break;
    }
    __shared__ float part[kWarps][32][V];
    float acc[V];
#pragma unroll
    for (int e = 0; e < V; ++e) acc[e] = 0.f;
    if (c < a.nv) {
        // warp q adds windows w + q, w + q + 4, ... ; then the four sums are added in order
        for (long long v = w + warp; v <= last; v += 4 * kWarps) {
            float x[4][V];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const long long at = v + u * kWarps;
                if (at <= last) load_vec<V>(a.pieces + (2 * at + (at == w ? 1 : 0)) * a.ld_piece + (long long)c * V, x[u]);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (v + u * kWarps > last) break;
#pragma unroll
                for (int e = 0; e < V; ++e) acc[e] += x[u][e];
            }
        }
    }
#pragma unroll
    for (int e = 0; e < V; ++e) part[warp][lane][e] = acc[e];
    __syncthreads();
    if (warp || c >= a.nv) return;
#pragma unroll
    for (int q = 1; q < kWarps; ++q) {
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] += part[q][lane][e];
    }
    write_row<GT, V>(a, key, c, acc);
}

// ---- host side -----------------------------------------------------------------------------

template <typename TT, typename OT>
cudaError_t launch_lookup(const adascale_embed_args &g, LookupArgs a, bool vec, cudaStream_t s)
{
    constexpr int V = 8;
    a.nv = (int)(vec ? g.dim / V : g.dim);
    const long long blocks = ceil_div(g.n_tokens, kLookupThreads / 32);
    return vec ? launch(k_lookup<TT, OT, V>, blocks, kLookupThreads, 0, s, a)
               : launch(k_lookup<TT, OT, 1>, blocks, kLookupThreads, 0, s, a);
}

template <typename DT, typename GT, int V>
cudaError_t launch_sums(SumArgs a, long long dim, cudaStream_t s)
{
    a.nv = (int)(dim / V);
    const long long windows = ceil_div(a.n, kWindow);
    cudaError_t e = launch(k_sum_windows<DT, GT, V>, ceil_div(windows * a.nv, kSumThreads), kSumThreads, 0, s, a);
    // a long run touches three windows at least
    if (e == cudaSuccess && windows > 2) e = launch(k_join<GT, V>, (windows - 2) * ceil_div(a.nv, 32), kSumThreads, 0, s, a);
    return e;
}

template <typename DT, typename GT>
cudaError_t launch_sums(const SumArgs &a, long long dim, bool vec, cudaStream_t s)
{
    constexpr int V = 16 / sizeof(DT);
    return vec ? launch_sums<DT, GT, V>(a, dim, s) : launch_sums<DT, GT, 1>(a, dim, s);
}

long long piece_stride(long long dim) { return ceil_div(dim, 8) * 8; }

}  // namespace

extern "C" {

adascale_status adascale_embed(const adascale_embed_args *g, void *cuda_stream)
{
    if (!g || g->n_tokens < 0 || g->vocab < 1 || g->dim < 1 || !is_dtype(g->table_dtype) || !is_dtype(g->out_dtype) ||
        !is_itype(g->token_type) || !std::isfinite(g->scale))
        return ADASCALE_ERR_INVALID_ARG;
    if (g->n_tokens > kMaxRows || g->vocab > kMaxRows || g->dim > kMaxRows) return ADASCALE_ERR_TOO_LARGE;
    if (g->n_tokens == 0) return ADASCALE_OK;
    if (!g->tokens || !g->table || !g->out || g->ld_table < g->dim || g->ld_out < g->dim) return ADASCALE_ERR_INVALID_ARG;
    const int et = elem_bytes(g->table_dtype), eo = elem_bytes(g->out_dtype);
    if (!on(g->tokens, id_bytes(g->token_type)) || !on(g->table, et) || !on(g->out, eo)) return ADASCALE_ERR_ALIGNMENT;
    const bool vec = g->dim % 8 == 0 && rows_on(g->table, g->ld_table, g->vocab, et, 16) &&
                     rows_on(g->out, g->ld_out, g->n_tokens, eo, 16);
    LookupArgs a = {g->tokens, g->table, g->out, g->n_tokens, g->vocab, g->ld_table, g->ld_out, g->token_type == ADASCALE_I64, 0,
                    g->scale};
    cudaStream_t s = (cudaStream_t)cuda_stream;
    if (g->table_dtype == ADASCALE_F32)
        OPS_CU(g->out_dtype == ADASCALE_F32 ? launch_lookup<float, float>(*g, a, vec, s) : launch_lookup<float, bf16>(*g, a, vec, s));
    else
        OPS_CU(g->out_dtype == ADASCALE_F32 ? launch_lookup<bf16, float>(*g, a, vec, s) : launch_lookup<bf16, bf16>(*g, a, vec, s));
    return ADASCALE_OK;
}

// Two lists of pairs and two rows of 32-bit sums per window.
int64_t adascale_embed_grad_workspace(int64_t n_tokens, int64_t dim)
{
    if (n_tokens < 0 || n_tokens > kMaxRows || dim < 1 || dim > kMaxRows) return 0;
    const long long pairs = ceil_div(n_tokens, 2) * 2;
    return 2 * pairs * (long long)sizeof(Pair) + ceil_div(n_tokens, kWindow) * 2 * piece_stride(dim) * (long long)sizeof(float);
}

adascale_status adascale_embed_grad(const adascale_embed_grad_args *g, void *cuda_stream)
{
    if (!g || g->n_tokens < 0 || g->vocab < 1 || g->dim < 1 || !is_dtype(g->dout_dtype) || !is_dtype(g->grad_dtype) ||
        !is_itype(g->token_type) || !std::isfinite(g->scale) || !g->grad || g->ld_grad < g->dim)
        return ADASCALE_ERR_INVALID_ARG;
    if (g->n_tokens > kMaxRows || g->vocab > kMaxRows || g->dim > kMaxRows) return ADASCALE_ERR_TOO_LARGE;
    const int ed = elem_bytes(g->dout_dtype), eg = elem_bytes(g->grad_dtype);
    if (!on(g->grad, eg)) return ADASCALE_ERR_ALIGNMENT;
    if (g->n_tokens == 0 && g->accumulate) return ADASCALE_OK;
    if (g->n_tokens > 0) {
        if (!g->tokens || !g->dout || !g->workspace || g->ld_dout < g->dim ||
            g->workspace_bytes < adascale_embed_grad_workspace(g->n_tokens, g->dim))
            return ADASCALE_ERR_INVALID_ARG;
        if (!on(g->tokens, id_bytes(g->token_type)) || !on(g->dout, ed) || !on(g->workspace, 16)) return ADASCALE_ERR_ALIGNMENT;
    }
    const int sms = sm_count();
    if (!sms) return ADASCALE_ERR_CUDA;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    const long long pairs = ceil_div(g->n_tokens, 2) * 2;

    SortArgs a = {};
    a.tokens = g->tokens;
    a.buf[0] = static_cast<Pair *>(g->workspace);
    a.buf[1] = a.buf[0] + pairs;
    a.grad = g->grad;
    a.n = g->n_tokens;
    a.vocab = g->vocab;
    a.ld_grad = g->ld_grad;
    a.padding = g->padding_idx;
    a.row_bytes = g->dim * eg;
    a.wide = g->token_type == ADASCALE_I64;
    while ((g->vocab >> (kSortBits * a.passes)) > 0) ++a.passes;  // the largest key is vocab itself
    a.grad_bytes = eg;
    a.vec = rows_on(g->grad, g->ld_grad, g->vocab, eg, 16) && a.row_bytes % 16 == 0;
    if (!g->accumulate) {  // one block per SM, in whole clusters; fewer for a small vocabulary
        long long blocks = sms / kSortCluster * kSortCluster - kSortCluster;
        const long long runs = ceil_div(g->vocab, kZeroRun);
        if (blocks > runs) blocks = ceil_div(runs, kSortCluster) * kSortCluster;
        a.zero_blocks = (int)(blocks < kSortCluster ? kSortCluster : blocks);
    }
    OPS_CU(launch(k_sort_tokens, kSortCluster + a.zero_blocks, kSortThreads, 0, s, a, kSortCluster));
    if (g->n_tokens == 0) return ADASCALE_OK;

    SumArgs b = {};
    b.sorted = a.buf[a.passes & 1];
    b.dout = g->dout;
    b.grad = g->grad;
    b.pieces = reinterpret_cast<float *>(a.buf[1] + pairs);
    b.n = g->n_tokens;
    b.vocab = g->vocab;
    b.ld_dout = g->ld_dout;
    b.ld_grad = g->ld_grad;
    b.ld_piece = piece_stride(g->dim);
    b.accumulate = g->accumulate != 0;
    b.scale = g->scale;
    const bool vec = g->dim % 8 == 0 && rows_on(g->dout, g->ld_dout, g->n_tokens, ed, 16) &&
                     rows_on(g->grad, g->ld_grad, g->vocab, eg, 16);
    if (g->dout_dtype == ADASCALE_F32)
        OPS_CU(g->grad_dtype == ADASCALE_F32 ? launch_sums<float, float>(b, g->dim, vec, s) : launch_sums<float, bf16>(b, g->dim, vec, s));
    else
        OPS_CU(g->grad_dtype == ADASCALE_F32 ? launch_sums<bf16, float>(b, g->dim, vec, s) : launch_sums<bf16, bf16>(b, g->dim, vec, s));
    return ADASCALE_OK;
}

}  // extern "C"
