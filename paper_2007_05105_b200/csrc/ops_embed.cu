// Token table: scaled lookup, and its gradient by sorted tokens (adascale_embed, adascale_embed_grad).
#include "ops_common.cuh"

#include <cooperative_groups.h>

namespace {

namespace cg = cooperative_groups;

// Columns are counted in 32 bits, some beyond a row's last one: by steps of 128 (lookup), rounded up to 32 (join).
constexpr long long kMaxDim = ADASCALE_EMBED_MAX_DIM;
static_assert(kMaxDim + 1024 < 2147483648LL, "columns beyond a row's last one stay positive");

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

// One warp per row: V elements per lane and access, up to four accesses requested before the first is
// used, so the two dependent round trips to memory (id, then row) are paid once per warp and covered
// by the SM's other warps.  V is 16 bytes of the wider type: with 8 floats a lane, as two accesses 32
// bytes apart from lane to lane, 65536 rows of 512 floats took 33 us instead of 27 (94 % of the measured
// copy rate).  The result leaves L2 first, so that the table's frequent rows stay.
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
            store_vec_streaming<V>(dst + (long long)j * V, x[u]);
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
// Blocks that sort together: sixteen (beyond the portable cluster size) for long lists, eight for short ones, whose barriers
// cost less.  32768 tokens accumulating 56 us, with eight 60; 65536: 84, 94; 8000: 25, 24.
constexpr int kSortCluster = 8, kSortWide = 16, kSortWideFrom = 16384;
// Tokens up to which places are counted instead of sorted by digits.  Accumulating: one wave of blocks (4099 tokens: 6.7 us
// against 10.4; 5000: 12.5 against 10.6).  Beside the zero-fill, which takes longer than either and starts
// sooner beside the sort's few blocks: 4000 tokens into 50257 rows of 1024 bf16 33.7 us in all, sorted 30.9.
constexpr int kRankMost = 148 * 32, kRankBesideZeros = 1024;
constexpr int kSortBits = 8;         // digit of one pass
constexpr int kSortBins = 1 << kSortBits;
// Blocks that write zeros beside the sort: with it, the clusters that are resident at once (15 of eight, 7 of
// sixteen; with two of eight more the last ones started when the first were done, 32 us for 22).
constexpr int kZeroBlocks = 112, kZeroWide = 96;
constexpr int kZeroRun = 16;         // adjacent vocabulary rows that belong to one of them
constexpr int kZeroBits = 32 * 1024; // rows that a block keeps presence bits of at a time
constexpr int kBatch = 8;            // tokens that a thread requests together
constexpr int kSumThreads = 128;
constexpr int kDepth = 16;             // rows on their way per thread of the window sums
constexpr int kSumBlocks = 5;       // their blocks per SM
constexpr int kMostPairs = 1024;     // sorted entries that a block of them holds
constexpr int kLeastWindow = 8;
constexpr int kColumns = 4;          // elements of a row per thread where rows are not aligned (see k_sum_windows)
constexpr int kSpill = 8;            // entries that a window takes from the next one to finish its last run

struct SortArgs {
    const void *tokens;
    Pair *buf[2];       // ping-pong; the result is in buf[passes & 1]
    void *grad;
    long long n, vocab, ld_grad, padding;
    long long row_bytes;  // of the gradient; its rows are zeroed where no token points
    int wide, passes;
    int zero_blocks;    // 0 when accumulating
    int grad_bytes;     // bytes of a gradient element
    int followed;       // by another kernel of the call
};

__device__ __forceinline__ int key_of(const SortArgs &a, long long i)
{
    const long long id = load_id(a.tokens, a.wide, i);
    return id >= 0 && id < a.vocab && id != a.padding ? (int)id : (int)a.vocab;
}

// One warp: 16 bytes a lane, the few before and after the aligned middle two at a time.
__device__ __forceinline__ void zero_row(char *p, long long bytes, int lane)
{
    long long front = (long long)(-(uintptr_t)p & 15);
    if (front > bytes) front = bytes;
    const long long middle = (bytes - front) / 16, back = bytes - front - middle * 16;
    if (lane < front / 2) reinterpret_cast<unsigned short *>(p)[lane] = 0;
    for (long long j = lane; j < middle; j += 32) reinterpret_cast<uint4 *>(p + front)[j] = make_uint4(0, 0, 0, 0);
    if (lane < back / 2) reinterpret_cast<unsigned short *>(p + front + middle * 16)[lane] = 0;
}

// Zeros for the rows that no token names, while other blocks sort.  Block z has the
// vocabulary rows whose run number (row / kZeroRun) is z modulo their number, so that a batch that uses
// only frequent, adjacent ids still spreads evenly.  The blocks of a cluster share the reading
// of the token list: each reads its part and sets presence bits in the shared memory of
// the block that has the row; then every block writes its absent rows.
__device__ void zero_absent(const SortArgs &a, unsigned *bits, const cg::cluster_group &cluster, int z)
{
    const int blocks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const long long runs = ceil_div(a.vocab, kZeroRun);
    const int Z = a.zero_blocks;
    const long long most = ceil_div(runs, Z);  // runs of a block
    constexpr int kRuns = kZeroBits / kZeroRun;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long part = ceil_div(a.n, blocks), from = part * rank, to = from + part < a.n ? from + part : a.n;
    for (long long r0 = 0; r0 < most; r0 += kRuns) {
        const int here = (int)(most - r0 < kRuns ? most - r0 : kRuns);
        for (int i = threadIdx.x; i < here * kZeroRun / 32 + 1; i += kSortThreads) bits[i] = 0u;
        cluster.sync();
        for (long long i0 = from + threadIdx.x; i0 < to; i0 += kBatch * kSortThreads) {
            unsigned key[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const long long i = i0 + u * kSortThreads;
                key[u] = i < to ? (unsigned)key_of(a, i) : (unsigned)a.vocab;
            }
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const unsigned run = key[u] / kZeroRun, owner = run % (unsigned)Z;
                const long long local = (long long)(run / (unsigned)Z) - r0;
                if (owner / blocks != (unsigned)(z / blocks) || local < 0 || local >= here || key[u] == (unsigned)a.vocab) continue;
                const int b = (int)local * kZeroRun + (int)(key[u] % kZeroRun);
                atomicOr(cluster.map_shared_rank(&bits[b >> 5], owner % blocks), 1u << (b & 31));
            }
        }
        cluster.sync();
        for (int b = warp; b < here * kZeroRun; b += kSortWarps) {
            if (bits[b >> 5] >> (b & 31) & 1u) continue;
            const long long row = ((r0 + b / kZeroRun) * Z + z) * kZeroRun + b % kZeroRun;
            if (row >= a.vocab) continue;
            zero_row(static_cast<char *>(a.grad) + row * a.ld_grad * a.grad_bytes, a.row_bytes, lane);
        }
        __syncthreads();  // the bits are read before the next range clears them
    }
}

// Lanes of the warp with this lane's digit, among those in `has`.  Eight votes: __match_any_sync
// took about 800 cycles a call here with 32 warps at it.
__device__ __forceinline__ unsigned same_digit(unsigned digit, unsigned has)
{
    unsigned same = has;
#pragma unroll
    for (int b = 0; b < kSortBits; ++b) {
        const bool set = digit >> b & 1u;
        const unsigned vote = __ballot_sync(0xffffffffu, set);
        same &= set ? vote : ~vote;
    }
    return same;
}

// Stable radix sort of (token, position) by token, least significant digit first, by the blocks
// of one cluster.  Every warp owns a contiguous stretch of the current order.  Per pass: it
// counts its stretch's digits in shared memory (votes group equal digits of 32 entries, one
// lane adds the group's size: no atomics, and the order within a group is the lane order), the
// counts are turned into first destinations (over digits, blocks and warps in that order; block
// totals travel through distributed shared memory), and a second walk over the stretch writes
// each entry to its place.  The list stays in L2; what a pass costs is two cluster barriers
// and one scattered 8-byte store per entry.
__global__ void __launch_bounds__(kSortThreads, 1) k_sort_tokens(const __grid_constant__ SortArgs a)
{
    __shared__ unsigned count[kSortWarps][kSortBins];  // also the bit field of the zero-fill
    __shared__ unsigned total[kSortBins];              // of this block, read by the whole cluster
    __shared__ unsigned scan[kSortBins / 32], start[kSortBins];
    static_assert(sizeof(count) * 8 >= kZeroBits, "the zero-fill's bits fit");
    griddep_wait();
    if (a.followed) griddep_launch();
    const cg::cluster_group cluster = cg::this_cluster();
    const int blocks = (int)cluster.num_blocks();
    if ((int)blockIdx.x >= blocks) {
        zero_absent(a, &count[0][0], cluster, (int)blockIdx.x - blocks);
        return;
    }
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, rank = (int)blockIdx.x;
    const unsigned below = (1u << lane) - 1u;
    const long long stretch = ceil_div(ceil_div(a.n, blocks * kSortWarps), 32) * 32;
    const long long first = ((long long)rank * kSortWarps + warp) * stretch;
    const long long last = first + stretch < a.n ? first + stretch : a.n;

    for (int pass = 0; pass < a.passes; ++pass) {
        const Pair *src = a.buf[pass & 1];
        Pair *dst = a.buf[(pass + 1) & 1];
        const int shift = pass * kSortBits;
        Pair p[kBatch];  // of the batch read last: a stretch of one batch is read once per pass
        auto read = [&](long long i0) {
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const long long i = i0 + 32 * u + lane;
                p[u].key = p[u].pos = 0;
                if (i >= last) continue;
                if (pass) {
                    const int2 q = __ldcg(reinterpret_cast<const int2 *>(src) + i);
                    p[u].key = q.x;
                    p[u].pos = q.y;
                } else {
                    p[u].key = key_of(a, i);
                    p[u].pos = (int)i;
                }
            }
        };
        for (int i = lane; i < kSortBins; i += 32) count[warp][i] = 0u;
        __syncwarp();
        for (long long i0 = first; i0 < last; i0 += 32 * kBatch) {
            read(i0);
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                if (i0 + 32 * u >= last) break;
                const bool has = i0 + 32 * u + lane < last;
                const unsigned digit = (unsigned)p[u].key >> shift & (kSortBins - 1);
                const unsigned same = same_digit(digit, __ballot_sync(0xffffffffu, has));
                if (has && !(same & below)) count[warp][digit] += __popc(same);
                __syncwarp();
            }
        }
        __syncthreads();
        unsigned sum = 0;
        if (tid < kSortBins) {  // exclusive prefix over the block's warps; the block's total
#pragma unroll 8
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
#pragma unroll 8
            for (int r = 0; r < blocks; ++r) {
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
            start[tid] = before;
        }
        __syncthreads();
        for (long long i0 = first; i0 < last; i0 += 32 * kBatch) {
            if (stretch > 32 * kBatch) read(i0);
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                if (i0 + 32 * u >= last) break;
                const bool has = i0 + 32 * u + lane < last;
                const unsigned digit = (unsigned)p[u].key >> shift & (kSortBins - 1);
                const unsigned same = same_digit(digit, __ballot_sync(0xffffffffu, has));
                const unsigned at = has ? start[digit] + count[warp][digit] + __popc(same & below) : 0u;
                __syncwarp();
                if (has && !(same & below)) count[warp][digit] += __popc(same);
                if (has) reinterpret_cast<int2 *>(dst)[at] = make_int2(p[u].key, p[u].pos);
                __syncwarp();
            }
        }
        // the next pass reads what all blocks wrote (the barrier orders it), and their totals are free again
        cluster.sync();
    }
}

// Short lists: an entry's place is the number of entries before it in the order, counted by comparing
// it with all others.  That many comparisons (17 million for 4099 tokens) cost less than the digit passes'
// barriers and scattered stores.  A block has 32 entries, one per lane; its warps share
// the list.
__global__ void __launch_bounds__(kSortThreads, 2) k_rank_tokens(const __grid_constant__ SortArgs a)
{
    __shared__ __align__(16) int keys[kRankMost];  // also the bit field of the zero-fill
    __shared__ int part[kSortWarps][32];
    static_assert(sizeof(keys) * 8 >= kZeroBits, "the zero-fill's bits fit");
    griddep_wait();
    if (a.followed) griddep_launch();
    const int n = (int)a.n;
    if ((int)blockIdx.x < a.zero_blocks) {  // first, as they take longest
        zero_absent(a, reinterpret_cast<unsigned *>(keys), cg::this_cluster(), (int)blockIdx.x);
        return;
    }
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    for (int i0 = tid; i0 < (n + 3) / 4 * 4; i0 += kBatch * kSortThreads) {
        int key[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) key[u] = i0 + u * kSortThreads < n ? key_of(a, i0 + u * kSortThreads) : 0x7fffffff;
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
            if (i0 + u * kSortThreads < kRankMost) keys[i0 + u * kSortThreads] = key[u];
    }
    __syncthreads();
    const int mine = ((int)blockIdx.x - a.zero_blocks) * 32 + lane, key = mine < n ? keys[mine] : 0;
    const int quads = (n + 3) / 4, per = (quads + kSortWarps - 1) / kSortWarps;
    const int first = warp * per, last = first + per < quads ? first + per : quads;
    int before = 0;
#pragma unroll 4
    for (int q = first; q < last; ++q) {
        const int4 k = reinterpret_cast<const int4 *>(keys)[q];
        const int j = 4 * q;
        before += (k.x < key) | ((k.x == key) & (j < mine));
        before += (k.y < key) | ((k.y == key) & (j + 1 < mine));
        before += (k.z < key) | ((k.z == key) & (j + 2 < mine));
        before += (k.w < key) | ((k.w == key) & (j + 3 < mine));
    }
    part[warp][lane] = before;
    __syncthreads();
    if (warp || mine >= n) return;
    int at = 0;
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) at += part[w][lane];
    reinterpret_cast<int2 *>(a.buf[0])[at] = make_int2(key, mine);
}

struct SumArgs {
    const Pair *sorted;
    const void *dout;
    void *grad;
    float *pieces;      // [windows][2][ld_piece]: a window's part of a run that 0 began earlier, 1 begins here and goes on
    long long n, vocab, ld_dout, ld_grad, ld_piece;
    int window;         // sorted entries of one window
    int nv;             // vectors of a row
    int threads;        // of a window: one per vector, or per kColumns elements
    int accumulate;
    int followed;       // by k_join
    float scale;
};

// A row's sums (V columns at c) to the gradient.  Accumulating into 32 bits is left to the L2
// cache, which adds without making the walk wait for the old value (one addition per element and call, so
// the order is fixed; subnormal numbers count as zeros there); bf16 needs the one rounding of old + new and is read, added and written here.
template <typename GT, int V>
__device__ __forceinline__ void write_row(const SumArgs &a, int key, int c, float (&acc)[V])
{
    GT *p = static_cast<GT *>(a.grad) + (long long)key * a.ld_grad + (long long)c * V;
    float out[V];
    if (a.accumulate) {
        if constexpr (sizeof(GT) == 4) {
            if constexpr (V == 1) {
                asm volatile("red.global.add.f32 [%0], %1;" ::"l"(p), "f"(a.scale * acc[0]) : "memory");
            } else {
#pragma unroll
                for (int i = 0; i < V; i += 4)
                    asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(p + i), "f"(a.scale * acc[i]),
                                 "f"(a.scale * acc[i + 1]), "f"(a.scale * acc[i + 2]), "f"(a.scale * acc[i + 3])
                                 : "memory");
            }
            return;
        }
        load_vec<V>(p, out);
#pragma unroll
        for (int i = 0; i < V; ++i) out[i] = fmaf(a.scale, acc[i], out[i]);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) out[i] = a.scale * acc[i];
    }
    store_vec<V>(p, out);
}

// Adds V elements of dout as they lie in 16 bytes.
template <typename DT, int V> __device__ __forceinline__ void add_to(float (&acc)[V], const uint4 &w)
{
    const unsigned q[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (V == 8) {
            acc[2 * i] += bf_lo(q[i]);
            acc[2 * i + 1] += bf_hi(q[i]);
        } else {
            acc[i] += __uint_as_float(q[i]);
        }
    }
}

__device__ __forceinline__ bool same_key(const Pair *s, long long n, long long i, int key)
{
    return i >= 0 && i < n && s[i].key == key;
}

// The sorted list is cut into windows of equal length; one thread walks over a window for one
// vector (16 bytes of dout; one element where rows are not aligned) and adds rows until the token
// changes.  A run that crosses into the next window by at most kSpill entries is finished by the window
// it comes from; where it goes further, each window leaves the sum of its part as a piece, and
// k_join adds the pieces in order.  So no window has more than kSpill entries more than another, however
// the tokens are distributed, and both sides of a boundary decide from one key: that of entry
// kSpill after it.  The pairs come through shared memory, the rows through a
// ring of kDepth asynchronous 16-byte copies per thread that only this thread reads: no barrier,
// no registers held, and a row's trip to memory is covered by the ones before it.  (With rows
// requested four at a time into registers the walk took about 10 us per window of 16, latency after latency:
// 22 us for 32768 x 1024 bf16, against 11 us for the bytes.)
template <typename DT, typename GT, int V>
__global__ void __launch_bounds__(kSumThreads, kSumBlocks) k_sum_windows(const __grid_constant__ SumArgs a)
{
    __shared__ uint4 ring[V == 1 ? 1 : kDepth][V == 1 ? 1 : kSumThreads];
    __shared__ int2 pairs[kMostPairs + kSpill + 2];
    griddep_wait();
    if (a.followed) griddep_launch();
    const long long t0 = (long long)blockIdx.x * kSumThreads, t1 = t0 + kSumThreads - 1;
    const long long base = t0 / a.threads * a.window - 1;  // entry of pairs[0]
    const int here = (int)(t1 / a.threads - t0 / a.threads + 1) * a.window + kSpill + 2;
    for (int i = threadIdx.x; i < here; i += kSumThreads) {
        const long long at = base + i;
        pairs[i] = at >= 0 && at < a.n ? __ldcg(reinterpret_cast<const int2 *>(a.sorted) + at) : make_int2(-1, 0);
    }
    __syncthreads();
    const long long t = t0 + threadIdx.x, w = t / a.threads;
    const int c = (int)(t - w * a.threads);
    if (w * a.window >= a.n) return;
    int lo = (int)(w * a.window - base);  // places in pairs; entries beyond the list have key -1
    int hi = lo + (int)(a.n - w * a.window < a.window ? a.n - w * a.window : a.window);
    const int absent = (int)a.vocab;
    bool head = pairs[lo - 1].x == pairs[lo].x;  // the run at the front began earlier
    if (head && pairs[lo + kSpill].x != pairs[lo].x) {  // and is finished there
        const int old = pairs[lo].x;
        while (lo < hi && pairs[lo].x == old) ++lo;
        head = false;
    }
    if (lo == hi) return;
    int key = pairs[lo].x;
    if (key == absent) return;  // entries without a part come last in the list
    const int back = pairs[hi - 1].x;
    const bool tail = back != absent && pairs[hi].x == back && pairs[hi + kSpill].x == back;
    if (back == absent) {  // of those there may be any number, and none is added
        while (pairs[hi - 1].x == absent) --hi;
    } else if (!tail) {  // the run ends within kSpill entries
        while (pairs[hi].x == back) ++hi;
    }

    float acc[V];
#pragma unroll
    for (int e = 0; e < V; ++e) acc[e] = 0.f;
    const DT *dout = static_cast<const DT *>(a.dout) + (long long)c * V;
    auto row = [&](int i) { return dout + (long long)pairs[i].y * a.ld_dout; };
    if constexpr (V == 1) {  // columns c, c + threads, c + 2 threads, ... of the window
        float sums[kColumns];
#pragma unroll
        for (int q = 0; q < kColumns; ++q) sums[q] = 0.f;
        auto finish = [&](bool piece, int which) {
#pragma unroll
            for (int q = 0; q < kColumns; ++q) {
                if (c + q * a.threads >= a.nv) break;
                float one[1] = {sums[q]};
                if (piece) a.pieces[(2 * w + which) * a.ld_piece + c + q * a.threads] = sums[q];
                else write_row<GT, 1>(a, key, c + q * a.threads, one);
                sums[q] = 0.f;
            }
        };
        constexpr int U = 4;  // rows requested together
        for (int i = lo; i < hi; i += U) {
            DT x[U][kColumns];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const DT *p = row(i + u < hi ? i + u : hi - 1);
#pragma unroll
                for (int q = 0; q < kColumns; ++q)
                    if (c + q * a.threads < a.nv) x[u][q] = p[q * a.threads];
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (i + u >= hi) break;
                const int k = pairs[i + u].x;
                if (k != key) {
                    finish(head, 0);
                    head = false;
                    key = k;
                }
#pragma unroll
                for (int q = 0; q < kColumns; ++q) sums[q] += to_f32(x[u][q]);
            }
        }
        finish(head || tail, head ? 0 : 1);
        return;
    } else {
        auto next_run = [&](int i) {  // before entry i is added
            const int k = pairs[i].x;
            if (k == key) return;
            if (head)
                store_vec<V>(a.pieces + 2 * w * a.ld_piece + (long long)c * V, acc);
            else
                write_row<GT, V>(a, key, c, acc);
            head = false;
            key = k;
#pragma unroll
            for (int e = 0; e < V; ++e) acc[e] = 0.f;
        };
        // bf16 rows that are added to: the old row of a run that ends kDepth entries on is asked for into L2 (32768 x 1024
        // accumulating: 54 us for 57)
        auto early = [&](int i) {
            if constexpr (sizeof(GT) == 2) {
                if (!a.accumulate || pairs[i].x == pairs[i + 1].x) return;
                asm volatile("prefetch.global.L2 [%0];" ::"l"(static_cast<GT *>(a.grad) + (long long)pairs[i].x * a.ld_grad + (long long)c * V));
            }
        };
        uint4 *mine = &ring[0][threadIdx.x];
        for (int u = 0; u < kDepth; ++u) {
            if (lo + u < hi) {
                copy_async(mine + u * kSumThreads, row(lo + u));
                early(lo + u);
            }
            copy_commit();
        }
        for (int i = lo, slot = 0; i < hi; ++i, slot = slot + 1 == kDepth ? 0 : slot + 1) {
            copy_wait<kDepth - 1>();
            const uint4 x = mine[slot * kSumThreads];
            next_run(i);
            add_to<DT, V>(acc, x);
            if (i + kDepth < hi) {
                copy_async(mine + slot * kSumThreads, row(i + kDepth));
                early(i + kDepth);
            }
            copy_commit();
        }
    }
    if (head || tail)
        store_vec<V>(a.pieces + (2 * w + (head ? 0 : 1)) * a.ld_piece + (long long)c * V, acc);
    else
        write_row<GT, V>(a, key, c, acc);
}

// The rows of runs that windows left in pieces: warp (w, slab) has the run that begins in window w,
// if it was.  Nearly all warps find none and leave after one round trip.
template <typename GT, int V>
__global__ void __launch_bounds__(kSumThreads) k_join(const __grid_constant__ SumArgs a)
{
    griddep_wait();
    const int slabs = (a.nv + 31) / 32;
    const long long item = (long long)blockIdx.x * (kSumThreads / 32) + (threadIdx.x >> 5), w = item / slabs;
    const int lane = threadIdx.x & 31, c = (int)(item % slabs) * 32 + lane;
    const long long lo = w * a.window, hi = lo + a.window;
    const Pair *s = a.sorted;
    if (hi >= a.n) return;
    // windows w + 1 + lane that have a piece of the run, if it begins in w; every key is asked for at once
    const int key = s[hi - 1].key, front = s[lo].key, before = lo ? s[lo - 1].key : -1;
    const long long ask = hi + (long long)lane * a.window + kSpill;
    const int there = ask < a.n ? s[ask].key : -1;
    unsigned reached = __ballot_sync(0xffffffffu, there == key);
    if (key >= a.vocab || !(reached & 1u) || (front == key && before == key)) return;
    long long last = w;
    for (;;) {  // 32 windows at a time
        const int more = reached == 0xffffffffu ? 32 : __ffs(~reached) - 1;
        last += more;
        if (more < 32) break;
        reached = __ballot_sync(0xffffffffu, same_key(s, a.n, (last + 1 + lane) * a.window + kSpill, key));
    }
    if (c >= a.nv) return;
    float acc[V];
    const float *piece = a.pieces + (long long)c * V;
    load_vec<V>(piece + (2 * w + 1) * a.ld_piece, acc);
    constexpr int U = 16;
    for (long long v = w + 1; v <= last; v += U) {
        float x[U][V];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (v + u <= last) load_vec<V>(piece + 2 * (v + u) * a.ld_piece, x[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (v + u > last) break;
#pragma unroll
            for (int e = 0; e < V; ++e) acc[e] += x[u][e];
        }
    }
    write_row<GT, V>(a, key, c, acc);
}

// ---- host side -----------------------------------------------------------------------------

template <typename TT, typename OT>
cudaError_t launch_lookup(const adascale_embed_args &g, LookupArgs a, bool vec, cudaStream_t s)
{
    constexpr int V = sizeof(TT) + sizeof(OT) > 4 ? 4 : 8;
    a.nv = (int)(vec ? g.dim / V : g.dim);
    const long long blocks = ceil_div(g.n_tokens, kLookupThreads / 32);
    return vec ? launch(k_lookup<TT, OT, V>, blocks, kLookupThreads, 0, s, a)
               : launch(k_lookup<TT, OT, 1>, blocks, kLookupThreads, 0, s, a);
}

// Entries of a window: one wave of blocks, but no more than a block's pairs have room for.
int window_of(long long n, int of_window, int sms)
{
    const long long threads = (long long)sms * kSumBlocks * kSumThreads;
    long long w = ceil_div(n * of_window, threads);
    const long long most = kMostPairs / (kSumThreads / of_window + 2);  // windows of a block, at most
    if (w > most) w = most;
    return (int)(w < kLeastWindow ? kLeastWindow : w);
}

template <typename DT, typename GT, int V>
cudaError_t launch_sums(SumArgs a, long long dim, int sms, cudaStream_t s)
{
    a.nv = (int)(dim / V);
    a.threads = V == 1 ? (int)ceil_div(dim, kColumns) : a.nv;
    a.window = window_of(a.n, a.threads, sms);
    const long long windows = ceil_div(a.n, a.window);
    a.followed = windows > 1;
    cudaError_t e = launch(k_sum_windows<DT, GT, V>, ceil_div(windows * a.threads, kSumThreads), kSumThreads, 0, s, a);
    if (e != cudaSuccess || !a.followed) return e;
    constexpr int JV = V == 1 ? 1 : 4;
    a.nv = (int)(dim / JV);
    return launch(k_join<GT, JV>, ceil_div((windows - 1) * ceil_div(a.nv, 32), kSumThreads / 32), kSumThreads, 0, s, a);
}

template <typename DT, typename GT>
cudaError_t launch_sums(const SumArgs &a, long long dim, bool vec, int sms, cudaStream_t s)
{
    constexpr int V = 16 / sizeof(DT);
    return vec ? launch_sums<DT, GT, V>(a, dim, sms, s) : launch_sums<DT, GT, 1>(a, dim, sms, s);
}

long long piece_stride(long long dim) { return ceil_div(dim, 8) * 8; }

}  // namespace

extern "C" {

adascale_status adascale_embed(const adascale_embed_args *g, void *cuda_stream)
{
    if (!g || g->n_tokens < 0 || g->vocab < 1 || g->dim < 1 || !is_dtype(g->table_dtype) || !is_dtype(g->out_dtype) ||
        !is_itype(g->token_type) || !std::isfinite(g->scale))
        return ADASCALE_ERR_INVALID_ARG;
    if (g->n_tokens > kMaxRows || g->vocab > kMaxRows || g->dim > kMaxDim) return ADASCALE_ERR_TOO_LARGE;
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
    if (n_tokens < 0 || n_tokens > kMaxRows || dim < 1 || dim > kMaxDim) return 0;
    const long long pairs = ceil_div(n_tokens, 2) * 2;
    return 2 * pairs * (long long)sizeof(Pair) + ceil_div(n_tokens, kLeastWindow) * 2 * piece_stride(dim) * (long long)sizeof(float);
}

adascale_status adascale_embed_grad(const adascale_embed_grad_args *g, void *cuda_stream)
{
    if (!g || g->n_tokens < 0 || g->vocab < 1 || g->dim < 1 || !is_dtype(g->dout_dtype) || !is_dtype(g->grad_dtype) ||
        !is_itype(g->token_type) || !std::isfinite(g->scale) || !g->grad || g->ld_grad < g->dim)
        return ADASCALE_ERR_INVALID_ARG;
    if (g->n_tokens > kMaxRows || g->vocab > kMaxRows || g->dim > kMaxDim) return ADASCALE_ERR_TOO_LARGE;
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
    a.followed = g->n_tokens > 0;
    const bool counted = g->n_tokens <= (g->accumulate ? kRankMost : kRankBesideZeros), wide = g->n_tokens >= kSortWideFrom;
    a.zero_blocks = g->accumulate ? 0 : wide ? kZeroWide : kZeroBlocks;
    if (counted) {
        OPS_CU(launch(k_rank_tokens, ceil_div(g->n_tokens, 32) + a.zero_blocks, kSortThreads, 0, s, a));
    } else {
        static OncePerDevice allowed;
        int dev = 0;
        OPS_CU(cudaGetDevice(&dev));
        if (wide && !allowed.has(dev)) {
            OPS_CU(cudaFuncSetAttribute(k_sort_tokens, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
            allowed.set(dev);
        }
        const int cluster = wide ? kSortWide : kSortCluster;
        OPS_CU(launch(k_sort_tokens, cluster + a.zero_blocks, kSortThreads, 0, s, a, cluster));
    }
    if (g->n_tokens == 0) return ADASCALE_OK;

    SumArgs b = {};
    b.sorted = counted ? a.buf[0] : a.buf[a.passes & 1];
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
        OPS_CU(g->grad_dtype == ADASCALE_F32 ? launch_sums<float, float>(b, g->dim, vec, sms, s) : launch_sums<float, bf16>(b, g->dim, vec, sms, s));
    else
        OPS_CU(g->grad_dtype == ADASCALE_F32 ? launch_sums<bf16, float>(b, g->dim, vec, sms, s) : launch_sums<bf16, bf16>(b, g->dim, vec, sms, s));
    return ADASCALE_OK;
}

}  // extern "C"
