// Products with experts' weights over ragged groups of rows, and their gradients, on the fifth-generation tensor cores.
//
//   y_r = W_e x_r       dx_r = W_e^T dy_r       dW_e (+)= sum over e's rows of dy_r x_r^T
//
// One kernel of three forms.  Each computes tiles D[lanes x columns] = A[lanes x k] B[columns x k]^T with A's rows on the
// lanes of tensor memory:
//
//            lanes (A)        columns (B)      summed over
//   Y        W_e's rows       e's rows of x    in_dim
//   DX       W_e's columns    e's rows of dy   out_dim
//   DW       dy's columns     x's columns      e's rows
//
// The ragged side is the one of the columns: a tile of tokens is as wide as it has to be (the instruction's n), an expert's rows
// are cut into tiles of equal width, and few tokens cost few columns.  Where a tile's last columns reach into the next
// expert's rows, their products are not stored.  In the weights' gradient the rows are summed over: what the last
// 64 of them bring of the next expert is set to zero in shared memory.
//
// A block a SM, or a pair of them, walks over the tiles: one warp issues the copies (tensor maps, 128-byte swizzle) into a ring of
// stages of 64 summands, one the matrix instructions, eight bring finished tiles from tensor memory, where two take turns,
// through shared memory to whole lines of memory.  In a pair both have 128 lanes and half of the columns' operand each, and the
// first one's instructions work on both: 256 x 256 results for 32 KB a stage and SM where a block alone takes 48 KB for half as
// many, and 48 KB are what the L2 cache does not deliver in the time that they are worked on.
// Every block works out the tiles from the offsets by itself: no host, no kernel before.
//
// Measured on a B200: 16384 rows over 16 experts of 1024 -> 4096 in 113 us (1220 TFLOP/s; 133 to 136 us under the power cap of a long run,
// where equal groups take 129 and the library's batched product of them 127), dx of 8192 rows over 8 experts 59 us, dw 62; 16 rows over 8
// experts, 59 MB of weights, 13 to 16 us.  Bound by the tensor cores' power, by what brings operands in, and by results (16 us of
// the first, whose stores do not all hide) where rows are many, by the weights' bytes where they are few.
//
// The tensor cores cut, not round, when they add to the 32-bit sums: of sums of one sign 6e-7 to 1.3e-6 is lost over 768 summands, 8e-6 to
// 1.4e-5 over 4096, 6.5e-5 to 8.2e-5 over 16384, 6e-9 m over m beyond (two units in the last place an instruction; measured).  So
// no sum is longer than kPart for float32 results, kLongPart for bf16 ones, whose own rounding is 2e-3 to 4e-3: the parts are added up,
// rounded, by the warps that read them, in tensor memory.  (bf16 dw of 131072 rows of one expert, 1024 x 1024: 578 us without parts,
// 583 with parts of 32768, 590 of 16384, 603 of 8192.)
#include "ops_common.cuh"

#include <cuda.h>

#include <algorithm>

namespace {

constexpr int kMaxExperts = ADASCALE_EXPERT_MAX_EXPERTS;
constexpr int kLanes = 128;      // of a block
constexpr int kK = 64;           // summands of a stage: 128 bytes, the swizzle's width
constexpr int kPart = 12 * kK;       // summands of one sum in tensor memory, for float32 results
constexpr int kLongPart = 256 * kK;  // and for bf16 results
constexpr int kResultWarps = 8;
constexpr int kThreads = 128 + 32 * kResultWarps;  // warps: copies, matrix instructions, ends of groups, one idle; results
constexpr int kDynamicMax = 216 * 1024;

enum Form { Y, DX, DW };

struct ExpertArgs {
    CUtensorMap a, b, c;  // operands; results
    const void *offsets;
    void *out;
    long long n_rows;
    long long ld_out, stride_out;  // DW: rows and experts of dw
    int n_experts, wide_offsets;
    int lanes, columns, summed;    // extents; the one that is e's rows is 0
    int accumulate, out_aligned;
    int part;                      // summands at which sums are cut
    // Two kernels of one call that do not need each other: the first (leads) lets the second (follows) start as soon as all of its blocks
    // have passed their wait for what was before it - which is then done for the second too - so that the second's blocks take the SMs
    // that the first one's leave.  The second waits for the first before it ends, so that who waits for it has waited for both.
    int leads, follows;
};

// ---- tensor memory and matrix instructions: of a block, or of a pair -----------------------

template <bool PAIR> __device__ __forceinline__ void tmem_alloc(unsigned *where, unsigned columns)
{
    if constexpr (PAIR) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(where)), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(where)), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
}
template <bool PAIR> __device__ __forceinline__ void tmem_free(unsigned base, unsigned columns)
{
    if constexpr (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns));
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns));
}
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// All matrix instructions that this thread has issued arrive at the barrier (in a pair: of both blocks) when they are done.
template <bool PAIR> __device__ __forceinline__ void mma_commit(u64 *bar)
{
    if constexpr (PAIR)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)),
                     "h"((unsigned short)3)
                     : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
template <bool PAIR> __device__ __forceinline__ void mma(unsigned d, u64 a, u64 b, unsigned what, bool add)
{
    if constexpr (PAIR)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a),
                     "l"(b), "r"(what), "r"((unsigned)add)
                     : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a),
                     "l"(b), "r"(what), "r"((unsigned)add)
                     : "memory");
}
// One thread of the warp.  What it alone does stands inside one branch on this, waits and all: with a branch on the thread's
// number a matrix instruction goes out every 128 cycles at best, be it of 64 columns or 256.
__device__ __forceinline__ bool elected()
{
    unsigned is;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(is));
    return is;
}
// 32 columns of this warp's 32 lanes; they are there after tmem_loaded, which all uses of x come behind.
__device__ __forceinline__ void tmem_load(unsigned at, unsigned (&r)[32])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
                   "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
                   "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(at));
}
__device__ __forceinline__ void tmem_loaded(unsigned (&r)[32])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) asm volatile("" : "+r"(r[i]));  // not read before
}
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_store(unsigned at, const unsigned (&x)[32])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
                 "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
                 "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(at),
                 "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7]), "r"(x[8]), "r"(x[9]), "r"(x[10]),
                 "r"(x[11]), "r"(x[12]), "r"(x[13]), "r"(x[14]), "r"(x[15]), "r"(x[16]), "r"(x[17]), "r"(x[18]), "r"(x[19]), "r"(x[20]),
                 "r"(x[21]), "r"(x[22]), "r"(x[23]), "r"(x[24]), "r"(x[25]), "r"(x[26]), "r"(x[27]), "r"(x[28]), "r"(x[29]), "r"(x[30]),
                 "r"(x[31])
                 : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap *map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
// A copy by a tensor map into this block's shared memory; the innermost coordinate is a multiple of 8 elements (16 bytes).  In a pair
// the barrier may be the other block's.
template <bool PAIR> __device__ __forceinline__ void tensor_load(void *dst, const CUtensorMap *map, int x, int y, int z, unsigned bar)
{
    if constexpr (PAIR)
        asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(
                         smem_u32(dst)),
                     "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z)
                     : "memory");
    else
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(smem_u32(dst)),
                     "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z)
                     : "memory");
}

// Shared memory operand, rows of 128 swizzled bytes, eight of them a group of 1024.
//   Summands along the rows: groups follow each other every 1024 bytes (`next` is not used: 16); 16 summands further are 32
//   bytes further.
//   Summands across the rows (each row has 64 lanes or columns): eight summands a group, the next 64 lanes or columns
//   `next` bytes further; 16 summands further are two groups further.
__device__ __forceinline__ u64 operand(unsigned addr, unsigned next)
{
    return (u64)((addr & 0x3ffff) >> 4) | (u64)((next & 0x3ffff) >> 4) << 16 | (u64)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}

// ---- pairs of blocks -----------------------------------------------------------------------

__device__ __forceinline__ unsigned pair_rank()
{
    unsigned r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void pair_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The first block's barrier of the same place.
__device__ __forceinline__ unsigned at_first(u64 *bar)
{
    unsigned there;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(there) : "r"(smem_u32(bar)));
    return there;
}
__device__ __forceinline__ void arrive_at_first(u64 *bar)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(at_first(bar)) : "memory");
}

// ---- tiles ---------------------------------------------------------------------------------

// What other kernels may have written is read past the L1 cache: the second gradient's kernel does not begin with a wait.
__device__ __forceinline__ float load_new(const float *p) { return __ldcg(p); }
__device__ __forceinline__ float load_new(const bf16 *p) { return __uint_as_float((unsigned)__ldcg(reinterpret_cast<const unsigned short *>(p)) << 16); }
__device__ __forceinline__ void load_new(const float *p, float (&x)[32])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float4 q = __ldcg(reinterpret_cast<const float4 *>(p) + i);
        x[4 * i] = q.x, x[4 * i + 1] = q.y, x[4 * i + 2] = q.z, x[4 * i + 3] = q.w;
    }
}
__device__ __forceinline__ void load_new(const bf16 *p, float (&x)[32])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint4 q = __ldcg(reinterpret_cast<const uint4 *>(p) + i);
        x[8 * i] = bf_lo(q.x), x[8 * i + 1] = bf_hi(q.x), x[8 * i + 2] = bf_lo(q.y), x[8 * i + 3] = bf_hi(q.y);
        x[8 * i + 4] = bf_lo(q.z), x[8 * i + 5] = bf_hi(q.z), x[8 * i + 6] = bf_lo(q.w), x[8 * i + 7] = bf_hi(q.w);
    }
}

// Of each expert: its rows, and the number of tiles before it.
struct Experts {
    int *begin;  // [n + 1]: begin[e + 1] is where e ends
    int *tiles;  // [n + 1]
    int *most;   // rows of the largest
};

// By one warp: offsets, ascending and within the rows, and running sums of the tiles.
template <Form F, int NT, int LANES> __device__ __forceinline__ void find_tiles(const ExpertArgs &a, const Experts &x)
{
    const int lane = threadIdx.x % 32, lane_tiles = (a.lanes + LANES - 1) / LANES;
    int floor = 0;
    for (int i = lane; i - lane <= a.n_experts; i += 32) {
        long long o = 0;
        if (i <= a.n_experts) o = a.wide_offsets ? __ldcg(static_cast<const long long *>(a.offsets) + i) : (long long)__ldcg(static_cast<const int *>(a.offsets) + i);
        int v = (int)(o < 0 ? 0 : o > a.n_rows ? a.n_rows : o);
        v = v > floor ? v : floor;
#pragma unroll
        for (int k = 1; k < 32; k *= 2) {
            const int before = __shfl_up_sync(0xffffffffu, v, k);
            if (lane >= k && before > v) v = before;
        }
        if (i <= a.n_experts) x.begin[i] = v;
        floor = __shfl_sync(0xffffffffu, v, 31);
    }
    __syncwarp();
    int sum = 0, most = 0;
    for (int i = lane; i - lane < a.n_experts; i += 32) {
        int v = 0;
        if (i < a.n_experts) {
            const int rows = x.begin[i + 1] - x.begin[i];
            most = max(most, rows);
            v = rows || (F == DW && !a.accumulate) ? lane_tiles * (((F == DW ? a.columns : rows) + NT - 1) / NT) : 0;
        }
#pragma unroll
        for (int k = 1; k < 32; k *= 2) {
            const int before = __shfl_up_sync(0xffffffffu, v, k);
            if (lane >= k) v += before;
        }
        v += sum;
        if (i < a.n_experts) x.tiles[i + 1] = v;
        sum = __shfl_sync(0xffffffffu, v, 31);
    }
    most = __reduce_max_sync(0xffffffffu, most);
    if (lane == 0) {
        x.tiles[0] = 0;
        *x.most = most;
    }
}

struct Tile {
    int expert;
    int lane;           // this block's first lane
    int column, width;  // first column (Y, DX: a row of the tokens), how many
    int row, summands;  // DW: first row; how many summands there are
};
// Tiles ascend from call to call.
template <Form F, int NT, int LANES> __device__ __forceinline__ void find_tile(const ExpertArgs &a, const Experts &x, int tile, int rank, Tile &t)
{
    constexpr int kStep = LANES > kLanes ? 32 : 16;  // of n, the width that an instruction can have
    while (tile >= x.tiles[t.expert + 1]) ++t.expert;
    const int begin = x.begin[t.expert], rows = x.begin[t.expert + 1] - begin, k = tile - x.tiles[t.expert];
    const int across = ((F == DW ? a.columns : rows) + NT - 1) / NT, col = k % across;
    t.lane = k / across * LANES + rank * kLanes;
    if (F == DW) {
        t.column = col * NT;
        t.width = min(NT, a.columns - t.column);
        t.row = begin;
        t.summands = rows;
    } else {  // of equal width
        const int each = ((rows + across - 1) / across + kStep - 1) / kStep * kStep;
        t.column = begin + col * each;
        t.width = min(each, rows - col * each);  // not less than 1: across - 1 of them are fewer than the rows
        t.row = 0;
        t.summands = a.summed;
    }
}

// Waits of this kernel have a limit like all others (kWaitNs, or kPolls, in which the block gets no further), and one that runs out sets a flag that ends the block's others.
// Who gave up does nothing further that others go by: no instruction is issued and no barrier arrived at for what has not come, so
// that in a pair the other block's waits run out too, rather than that it stores half a sum.  What a block has not computed is NaN.
// The thread that issues copies does not look at the flag: in a pair both then stop at the same stage, and their copies are seen
// through (see the end of its branch), as are the matrix instructions, before shared and tensor memory are given up.
#ifndef ADASCALE_EXPERT_POLLS  // a test makes the waits run out at once
#define ADASCALE_EXPERT_POLLS (1u << 22)
#endif
constexpr unsigned kPolls = ADASCALE_EXPERT_POLLS;
// What a block's waits go by.
struct Waits {
    volatile int gave_up;
    volatile unsigned issued;  // stages, by the thread that issues copies
};
template <bool CLUSTER> __device__ __noinline__ bool wait_long(u64 *bar, unsigned parity, Waits &waits)
{
    // A sum may last (2^31 rows of 8 columns, one block's, 13 s), and who waits for its end or for the end of a group behind it is not late: the
    // limit holds for a time in which nothing was issued either.
    u64 t0 = 0;
    unsigned seen = 0;
    for (unsigned spin = 0; spin < kPolls; ++spin) {
        if (mbar_poll<CLUSTER>(smem_u32(bar), parity)) return true;
        if (waits.gave_up) return false;
        if ((spin & 63u) == 63u) {
            const unsigned issued = waits.issued;
            u64 now;
            asm volatile("mov.u64 %0, %globaltimer;" : "=l"(now));
            if (t0 == 0 || issued != seen) t0 = now, seen = issued, spin = 63;
            else if (now - t0 > kWaitNs) break;
        }
    }
    waits.gave_up = 1;
    return false;
}
// False if it gave up.
template <bool CLUSTER = false> __device__ __forceinline__ bool wait_for(u64 *bar, unsigned parity, Waits &waits)
{
    return mbar_poll<CLUSTER>(smem_u32(bar), parity) || wait_long<CLUSTER>(bar, parity, waits);
}

// ---- results -------------------------------------------------------------------------------
// Two warps share 32 lanes and take every other 32 columns of them, each by way of its room of 32 x 32 results in shared memory and a
// copy by tensor map, which leaves out what lies outside the matrix - in units of 16 bytes: of a row that ends inside 16 it would write
// zeros behind the end.  So the map ends before, and the rows' last elements are stored by the warp.

// Until the last copy out of the warp's room has read it; lane 0 has the copies.
__device__ __forceinline__ void room_wait()
{
    if (threadIdx.x % 32 == 0) bulk_wait_read<0>();
    __syncwarp();
}
// What was put into it by all lanes goes out.
template <typename Issue> __device__ __forceinline__ void copy_out(Issue issue)
{
    copy_fence();
    __syncwarp();
    if (threadIdx.x % 32 == 0) {
        issue();
        bulk_commit();
    }
}
__device__ __forceinline__ void tensor_store(const CUtensorMap *map, int x, int y, int z, const void *src)
{
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map), "r"(smem_u32(src)), "r"(x), "r"(y), "r"(z)
                 : "memory");
}
__device__ __forceinline__ void tensor_add(const CUtensorMap *map, int x, int y, int z, const void *src)
{
    asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map), "r"(smem_u32(src)), "r"(x), "r"(y),
                 "r"(z)
                 : "memory");
}

// Y, DX: of n columns (tokens) the lanes from lane0 on, adjacent elements of a token's row.  A row of `room` is a token's.
template <typename O> __device__ __forceinline__ void store_tokens(const ExpertArgs &a, const float (&v)[32], O *room, int lane0, int token, int n)
{
    constexpr int V = 16 / sizeof(O), kPieces = 32 / V, kAtOnce = 32 / kPieces;
    const int me = threadIdx.x % 32;
    if (lane0 >= a.lanes) return;
    O *out = static_cast<O *>(a.out) + (long long)token * a.ld_out + lane0;
    if (!a.out_aligned) {
        if (lane0 + me < a.lanes)
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (i < n) put(out + i * a.ld_out + me, v[i]);
        return;
    }
    room_wait();
#pragma unroll
    for (int i = 0; i < 32; ++i) put(room + i * 32 + me, v[i]);
    if (n == 32) {
        const int all = a.lanes - lane0, copied = all / V * V;  // of this token's row; lane0 is a multiple of V
        copy_out([&] {
            if (copied > 0) tensor_store(&a.c, lane0, token, 0, room);
        });
        if (all < 32)
            for (int e = copied; e < all; ++e) out[me * a.ld_out + e] = room[me * 32 + e];
        return;
    }
    __syncwarp();  // the last tokens of a group: what follows them is not ours
    const int piece = me % kPieces, left = a.lanes - lane0 - piece * V;
    for (int k = me / kPieces; k < n; k += kAtOnce) {
        const O *q = room + k * 32 + piece * V;
        O *p = out + k * a.ld_out + piece * V;
        if (left >= V) {
            *reinterpret_cast<uint4 *>(p) = *reinterpret_cast<const uint4 *>(q);
        } else {
            for (int e = 0; e < left; ++e) p[e] = q[e];
        }
    }
    __syncwarp();
}

// DW: n columns of the warp's lanes, each lane a row of dw.  Rows of `room` are 128 bytes (float32) or 64, with their 16-byte pieces in
// the order of the tensor map's swizzle, which keeps banks apart.
template <typename O> __device__ __forceinline__ void store_rows(const ExpertArgs &a, float (&v)[32], O *room, int expert, int lane0, int column, int n)
{
    constexpr int V = 16 / sizeof(O), kPieces = 32 / V;
    const int me = threadIdx.x % 32;
    if (lane0 >= a.lanes) return;
    O *p = static_cast<O *>(a.out) + expert * a.stride_out + (lane0 + me) * a.ld_out + column;
    if (!a.out_aligned || (column + 32 > a.columns && a.columns % V != 0)) {  // nothing of these 32 x 32 is copied
        if (lane0 + me < a.lanes)
#pragma unroll
            for (int j = 0; j < kPieces; ++j) {
                float x[V];
#pragma unroll
                for (int e = 0; e < V; ++e) x[e] = v[j * V + e] + (a.accumulate && j * V + e < n ? load_new(p + j * V + e) : 0.f);
                if (a.out_aligned && (j + 1) * V <= n) {
                    store_vec<V>(p + j * V, x);
                } else {
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        if (j * V + e < n) put(p + j * V + e, x[e]);
                }
            }
        return;
    }
    // a float32 gradient is added to on the way; others are read, added to in 32 bits and rounded once
    if (sizeof(O) == 2 && a.accumulate && lane0 + me < a.lanes) {
        if (n == 32) {
            float old[32];
            load_new(p, old);
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] += old[i];
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (i < n) v[i] += load_new(p + i);
        }
    }
    room_wait();
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
        float x[V];
#pragma unroll
        for (int e = 0; e < V; ++e) x[e] = v[j * V + e];
        store_vec<V>(room + me * 32 + (j ^ (kPieces == 8 ? me & 7 : me >> 1 & 3)) * V, x);
    }
    copy_out([&] {
        if (sizeof(O) == 4 && a.accumulate) tensor_add(&a.c, column, lane0, expert, room);
        else tensor_store(&a.c, column, lane0, expert, room);
    });
}

// ---- the kernel ----------------------------------------------------------------------------

template <int NT, bool PAIR> constexpr int kStageBytes = (kLanes + (PAIR ? NT / 2 : NT)) * kK * 2;
template <typename O> constexpr int kStaging = kResultWarps * 32 * 32 * (int)sizeof(O);
template <int NT, bool PAIR, typename O> constexpr int kStages = (kDynamicMax - kStaging<O>) / kStageBytes<NT, PAIR>;
// staging and ring, which start on a boundary of 1024
template <int NT, bool PAIR, typename O> constexpr int kSmemBytes = 1024 + kStaging<O> + kStages<NT, PAIR, O> * kStageBytes<NT, PAIR>;
template <int NT> constexpr int kTokenBox = NT < 64 ? NT : 64;  // rows of one copy of tokens

template <Form F, int NT, bool PAIR, typename O> __global__ void __launch_bounds__(kThreads) k_expert(const __grid_constant__ ExpertArgs a)
{
    constexpr int S = kStages<NT, PAIR, O>, LANES = PAIR ? 2 * kLanes : kLanes, kA = kLanes * kK * 2, kBox = kTokenBox<NT>;
    constexpr unsigned kColumns = 2 * NT;
    extern __shared__ unsigned char raw[];
    __shared__ u64 full[S], there[S], empty[S], done[2], taken[2], arrived, ended;
    __shared__ unsigned tmem_base;
    __shared__ Waits waits;
    __shared__ int begins[kMaxExperts + 1], tile_sums[kMaxExperts + 1], most_rows;
    unsigned char *staging = raw + (1024 - smem_u32(raw) % 1024) % 1024, *ring = staging + kStaging<O>;
    const Experts x = {begins, tile_sums, &most_rows};
    const int warp = threadIdx.x / 32, rank = PAIR ? (int)pair_rank() : 0;

    if (threadIdx.x == 0) {
        for (int i = 0; i < S; ++i) {
            // the copies of a stage are there: of both blocks, at the first one's barrier; but the last 64 rows of a group of DW, which
            // have to be ended first, arrive at each block's own, and are worked on when `there` says that the second block has ended its
            mbar_init(&full[i], 1);
            mbar_init(&there[i], 1);
            mbar_init(&empty[i], 1);
        }
        waits.gave_up = 0;
        waits.issued = 0;
        mbar_init(&arrived, 1);
        mbar_init(&ended, 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&done[i], 1);
            mbar_init(&taken[i], PAIR ? 2 * kResultWarps : kResultWarps);
        }
        mbar_publish();
    }
    if (warp == 1) tmem_alloc<PAIR>(&tmem_base, kColumns);
    if (warp == 3 && elected()) {
        if (a.n_rows > 0) {  // without rows there are no operands' maps
            prefetch_map(&a.a);
            prefetch_map(&a.b);
        }
        if (a.out_aligned) prefetch_map(&a.c);
    }
    if (!a.follows) griddep_wait();
    if (a.leads) griddep_launch();
    if (warp == 0) find_tiles<F, NT, LANES>(a, x);
    tmem_fence_before();
    __syncthreads();
    if constexpr (PAIR) pair_sync();
    tmem_fence_after();
    const unsigned tmem = tmem_base;
    const int n_tiles = x.tiles[a.n_experts], first_tile = PAIR ? blockIdx.x / 2 : blockIdx.x, step = PAIR ? gridDim.x / 2 : gridDim.x;
    // Sums in parts have one buffer of tensor memory, the other holds what has been added up: only where a sum is that long.  (By the rows of
    // all experts instead, us: 1024 x 4096, f32 dw of 8192 rows over 11 experts 96, 88 so; over 16 97 and 92; 1024 x 1024 over 64 61.1 and 62.5.)
    const bool in_parts = (F == DW ? most_rows : a.summed) > a.part;
    const int part = in_parts ? a.part : 0x7fffffc0;  // more than there are rows
    // operands whose summands lie across the rows in memory
    constexpr bool kAcrossA = F != Y, kAcrossB = F == DW;

    if (warp == 0) {
        if (elected()) {
            Tile t = {};
            int stage = 0, issued = 0;
            bool in_time = true;
            unsigned phase = 1;  // the first pass over the ring waits for nobody
            for (int tile = first_tile; in_time && tile < n_tiles; tile += step) {
                find_tile<F, NT, LANES>(a, x, tile, rank, t);
                // this block's columns: all of them, or its half
                const int half = PAIR ? (t.width + 31) / 32 * 16 : t.width, column = t.column + rank * half;
                const int boxes = F == DW ? (half + 63) / 64 : (half + kBox - 1) / kBox;
                for (int k = 0; k < t.summands; k += kK) {
                    in_time = mbar_wait(&empty[stage], phase);
                    if (!in_time) {
                        waits.gave_up = 1;
                        break;
                    }
                    unsigned char *as = ring + stage * kStageBytes<NT, PAIR>, *bs = as + kA;
                    const int bytes = kA + boxes * (F == DW ? 64 : kBox) * kK * 2;
                    // in a pair the first block's barrier takes both blocks' bytes; the ends of groups go to each one's own
                    const bool own = !PAIR || (F == DW && t.summands - k < kK);
                    const unsigned bar = own ? smem_u32(&full[stage]) : at_first(&full[stage]);
                    if (own || rank == 0) mbar_expect_tx(&full[stage], own ? bytes : 2 * bytes);
                    if constexpr (F == DW) {
                        for (int i = 0; i < 2; ++i) tensor_load<PAIR>(as + i * 8192, &a.a, t.lane + 64 * i, t.row + k, 0, bar);
                        for (int i = 0; i < boxes; ++i) tensor_load<PAIR>(bs + i * 8192, &a.b, column + 64 * i, t.row + k, 0, bar);
                    } else {
                        if constexpr (F == Y) {
                            tensor_load<PAIR>(as, &a.a, k, t.lane, t.expert, bar);
                        } else {
                            for (int i = 0; i < 2; ++i) tensor_load<PAIR>(as + i * 8192, &a.a, t.lane + 64 * i, k, t.expert, bar);
                        }
                        for (int i = 0; i < boxes; ++i) tensor_load<PAIR>(bs + i * kBox * kK * 2, &a.b, k, column + i * kBox, 0, bar);
                    }
                    waits.issued = ++issued;
                    if (++stage == S) stage = 0, phase ^= 1;
                }
            }
            // Copies in flight end before the block does.  The first block's barriers know of both blocks' (which leave together); the second
            // one sees its last stage worked on, or has waited for it as long as a wait can last.
            for (int i = 0; i < min(issued, S) && rank == 0; ++i) {
                const int n = issued - 1 - i;
                if (!mbar_wait(&full[n % S], (n / S) & 1)) break;
            }
            if (rank == 1 && issued > 0) (void)mbar_wait(&empty[(issued - 1) % S], ((issued - 1) / S) & 1);
        }
    } else if (warp == 1 && rank == 0) {
        if (elected()) {
            Tile t = {};
            int stage = 0, turn = 0;
            bool in_time = true;
            unsigned phase = 0, free_phase = 1, end_phase = 0, there_phase = 0;
            for (int tile = first_tile; in_time && tile < n_tiles; tile += step) {
                find_tile<F, NT, LANES>(a, x, tile, rank, t);
                const unsigned n = PAIR ? (t.width + 31) / 32 * 32 : (t.width + 15) / 16 * 16;
                const unsigned what =
                    1u << 4 | 1u << 7 | 1u << 10 | (kAcrossA ? 1u << 15 : 0u) | (kAcrossB ? 1u << 16 : 0u) | n / 8 << 17 | (unsigned)(LANES / 16) << 24;
                for (int left = t.summands; left > 0; left -= part) {
                    in_time = wait_for<PAIR>(&taken[turn], free_phase, waits);
                    if (!in_time) break;
                    tmem_fence_after();
                    const unsigned d = tmem + turn * NT;
                    const int now = min(left, part);
                    for (int k = 0; k < now; k += kK) {
                        in_time = wait_for(&full[stage], phase, waits);
                        if (F == DW && in_time && left - k < kK) {  // it is there: warp 2 may end it
                            mbar_arrive(&arrived);
                            in_time = wait_for(&ended, end_phase, waits);
                            end_phase ^= 1;
                            if constexpr (PAIR) {
                                in_time = in_time && wait_for<true>(&there[stage], there_phase >> stage & 1, waits);
                                there_phase ^= 1u << stage;
                            }
                        }
                        if (!in_time) break;
                        tmem_fence_after();
                        const unsigned as = smem_u32(ring + stage * kStageBytes<NT, PAIR>);
                        const u64 da = operand(as, kAcrossA ? 8192 : 16), db = operand(as + kA, kAcrossB ? 8192 : 16);
#pragma unroll
                        for (int i = 0; i < kK / 16; ++i)  // summands behind the last are zeros
                            mma<PAIR>(d, da + (u64)(i * (kAcrossA ? 2048 : 32) >> 4), db + (u64)(i * (kAcrossB ? 2048 : 32) >> 4), what, k + i > 0);
                        mma_commit<PAIR>(&empty[stage]);
                        if (++stage == S) stage = 0, phase ^= 1;
                    }
                    if (!in_time) break;
                    mma_commit<PAIR>(&done[turn]);
                    if (in_parts) {
                        free_phase ^= 1;
                    } else {
                        free_phase ^= turn;
                        turn ^= 1;
                    }
                }
            }
            // those in flight end before the block does: the last one's stage
            if (stage == 0) phase ^= 1;
            (void)mbar_wait(&empty[stage == 0 ? S - 1 : stage - 1], phase);
        }
    } else if (F == DW && warp == 2) {  // rows of the next expert, or of nobody, behind the last of e's: zeros
        Tile t = {};
        int blocks = 0;
        unsigned phase = 0;  // rank 1: of every stage
        for (int tile = first_tile; tile < n_tiles; tile += step) {
            find_tile<F, NT, LANES>(a, x, tile, rank, t);
            blocks += (t.summands + kK - 1) / kK;
            const int left = t.summands % kK;
            if (left == 0) continue;
            const int stage = (blocks - 1) % S;
            bool in_time;
            if (rank == 0) {
                in_time = wait_for(&arrived, phase, waits);
                phase ^= 1;
            } else {
                in_time = wait_for(&full[stage], phase >> stage & 1, waits);
                phase ^= 1u << stage;
            }
            if (!__all_sync(0xffffffffu, in_time)) break;
            unsigned char *as = ring + stage * kStageBytes<NT, PAIR>;
            const int half = PAIR ? (t.width + 31) / 32 * 16 : t.width, boxes = 2 + (half + 63) / 64;
            for (int box = 0; box < boxes; ++box)
                for (int i = threadIdx.x % 32; i < (kK - left) * 8; i += 32)
                    reinterpret_cast<uint4 *>(as + box * 8192 + left * 128)[i] = make_uint4(0, 0, 0, 0);
            copy_fence();
            __syncwarp();
            if (threadIdx.x % 32 == 0) {
                if (rank == 0) mbar_arrive(&ended);
                else arrive_at_first(&there[stage]);
            }
        }
    } else if (warp >= 4) {
        const int quarter = warp % 4;  // a warp reads the quarter of the lanes that its number names
        O *room = reinterpret_cast<O *>(staging) + (warp - 4) * 32 * 32;
        const unsigned mine = (unsigned)(quarter * 32) << 16;
        constexpr int kEvery = kResultWarps / 4 * 32;
        const int first = (warp - 4) / 4 * 32;
        Tile t = {};
        int turn = 0;
        unsigned phase = 0;
        bool lost = false;  // a wait ran out, in this tile or one before: NaN from here on
        for (int tile = first_tile; tile < n_tiles; tile += step) {
            find_tile<F, NT, LANES>(a, x, tile, rank, t);
            for (int left = t.summands; left > 0 || left == t.summands; left -= part) {
                const bool any = t.summands > 0, first_part = left == t.summands, last = left <= part;
                if (any && !lost) {
                    lost = !__all_sync(0xffffffffu, wait_for(&done[turn], phase, waits));
                    tmem_fence_after();
                }
                const unsigned from = tmem + turn * NT + mine, sums = tmem + NT + mine;
                const auto taken_now = [&] {
                    tmem_fence_before();
                    __syncwarp();
                    if (threadIdx.x % 32 == 0) {
                        if constexpr (PAIR) arrive_at_first(&taken[turn]);
                        else mbar_arrive(&taken[turn]);
                    }
                };
                if (in_parts && any && !lost) {  // to the running sum at once, so that the next part may begin before results are stored
                    for (int c = first; c < t.width; c += kEvery) {
                        unsigned now[32], before[32];
                        tmem_load(from + c, now);
                        if (!first_part) tmem_load(sums + c, before);
                        tmem_loaded(now);
                        if (!first_part) {
                            tmem_loaded(before);
#pragma unroll
                            for (int i = 0; i < 32; i += 2) {
                                float lo, hi;
                                unpack2(add2(pack2(__uint_as_float(now[i]), __uint_as_float(now[i + 1])),
                                             pack2(__uint_as_float(before[i]), __uint_as_float(before[i + 1]))),
                                        lo, hi);
                                now[i] = __float_as_uint(lo), now[i + 1] = __float_as_uint(hi);
                            }
                        }
                        tmem_store(sums + c, now);
                    }
                    tmem_stored();
                    taken_now();
                }
                if (last) {
                    for (int c = first; c < t.width; c += kEvery) {
                        unsigned now[32];
                        float v[32];
                        if (any && !lost) {
                            tmem_load(in_parts ? sums + c : from + c, now);
                            tmem_loaded(now);
#pragma unroll
                            for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(now[i]);
                        } else {
#pragma unroll
                            for (int i = 0; i < 32; ++i) v[i] = any ? NAN : 0.f;
                        }
                        const int n = min(32, t.width - c);
                        if constexpr (F == DW) store_rows<O>(a, v, room, t.expert, t.lane + quarter * 32, t.column + c, n);
                        else store_tokens<O>(a, v, room, t.lane + quarter * 32, t.column + c, n);
                    }
                }
                if (!any || lost) continue;
                if (!in_parts) taken_now();
                if (in_parts) {
                    phase ^= 1;
                } else {
                    phase ^= turn;
                    turn ^= 1;
                }
            }
        }
        if (threadIdx.x % 32 == 0) bulk_wait_all();
    }
    tmem_fence_before();
    __syncthreads();
    if constexpr (PAIR) pair_sync();  // neither ends while the other may arrive at its barriers
    tmem_fence_after();
    if (warp == 1) tmem_free<PAIR>(tmem, kColumns);
    if (a.follows) griddep_wait();
}

// ---- host side -----------------------------------------------------------------------------

typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled()
{
    static std::atomic<EncodeTiled> known{nullptr};  // every thread finds the same one
    EncodeTiled f = known.load(std::memory_order_relaxed);
    if (f) return f;
    void *p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) {
        (void)cudaGetLastError();
        return nullptr;
    }
    f = reinterpret_cast<EncodeTiled>(p);
    known.store(f, std::memory_order_relaxed);
    return f;
}
// [n, rows, cols] with `ld` and `stride` elements between rows and matrices.
struct Extents {
    long long n, rows, cols, stride, ld;
};
bool make_map(CUtensorMap *map, const void *p, Extents x, int dtype, int box_cols, int box_rows, CUtensorMapSwizzle swizzle)
{
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    // strides that are never used still have to be some
    if (x.rows <= 1) x.ld = (x.cols + 7) / 8 * 8;
    if (x.n <= 1) x.stride = x.ld * x.rows;
    const cuuint64_t b = (cuuint64_t)elem_bytes(dtype), dims[3] = {(cuuint64_t)x.cols, (cuuint64_t)x.rows, (cuuint64_t)x.n};
    const cuuint64_t strides[2] = {(cuuint64_t)x.ld * b, (cuuint64_t)x.stride * b};
    const cuuint32_t boxes[3] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, 1}, steps[3] = {1, 1, 1};
    return encode(map, dtype == ADASCALE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, const_cast<void *>(p), dims, strides,
                  boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// An operand: 64 columns and `box` rows a copy.
bool operand_map(CUtensorMap *map, const void *p, const Extents &x, int box)
{
    return make_map(map, p, x, ADASCALE_BF16, 64, box, CU_TENSOR_MAP_SWIZZLE_128B);
}
// Results, 32 x 32 a copy, where their rows allow it: as far as they go in whole 16 bytes.
bool result_map(ExpertArgs &e, Extents x, int dtype, CUtensorMapSwizzle swizzle)
{
    const int b = elem_bytes(dtype);
    x.cols = x.cols * b / 16 * 16 / b;
    e.out_aligned = x.cols > 0 && on(e.out, 16) && (x.rows <= 1 || x.ld * b % 16 == 0) && (x.n <= 1 || x.stride * b % 16 == 0);
    return !e.out_aligned || make_map(&e.c, e.out, x, dtype, 32, 32, swizzle);
}

template <Form F, int NT, bool PAIR, typename O> cudaError_t run_tiles(const ExpertArgs &a, long long tiles, cudaStream_t s)
{
    static OncePerDevice known;
    cudaError_t e = allow_smem(reinterpret_cast<const void *>(&k_expert<F, NT, PAIR, O>), known);
    if (e != cudaSuccess) return e;
    const int sms = sm_count();
    if (sms < 2) return cudaErrorUnknown;
    const long long blocks = PAIR ? 2 * std::min<long long>(tiles, sms / 2) : std::min<long long>(tiles, sms);
    return launch(k_expert<F, NT, PAIR, O>, blocks, kThreads, kSmemBytes<NT, PAIR, O>, s, a, PAIR ? 2 : 1);
}
template <Form F, int NT, bool PAIR = false> cudaError_t run_type(ExpertArgs &a, int dtype, cudaStream_t s)
{
    const long long lane_tiles = ceil_div(a.lanes, PAIR ? 2 * kLanes : kLanes);
    a.part = dtype == ADASCALE_F32 ? kPart : kLongPart;
    // at most this many tiles: each expert may have one that is not full
    const long long tiles = F == DW ? a.n_experts * lane_tiles * ceil_div(a.columns, NT)
                                    : lane_tiles * (a.n_rows / NT + std::min<long long>(a.n_experts, a.n_rows));
    return dtype == ADASCALE_BF16 ? run_tiles<F, NT, PAIR, bf16>(a, tiles, s) : run_tiles<F, NT, PAIR, float>(a, tiles, s);
}
// Pairs of blocks where there are lanes for both and the summands (of an expert on average) are many: with few of them the time goes into
// bringing results out, and half as many, twice as large tiles leave more SMs without one.  Pair against blocks alone, us:
// 1024 x 4096 over 8 experts, weights' gradient of 256 rows each 33.4 and 28.2, of 512 rows 41.8 and 42.8, product of 256 rows
// each (1024 summands) 26.4 and 29.1; 512 x 512 over 64 experts, 256 rows each (512 summands) 24.5 and 21.8.
template <Form F> cudaError_t run_wide(ExpertArgs &a, int dtype, cudaStream_t s)
{
    const long long summands = F == DW ? a.n_rows / a.n_experts : a.summed;
    return a.lanes > kLanes && summands > 512 ? run_type<F, 256, true>(a, dtype, s) : run_type<F, 256>(a, dtype, s);
}
// Tiles of tokens are as wide as the rows of an expert on average, as far as the host knows: rows before the first offset and behind the last
// count.  With room for 16384 more behind 16 to 2048 rows of 8 or 16 experts a product takes 0.8 to 1.4 us longer (11.3 and 12.1, 8.7 and 10.1),
// a weights' gradient, which then takes pairs, 3 to 5 (14.3 and 17.4, 22.2 and 27.3): a caller who knows the rows gives a slice.
template <Form F> cudaError_t run_tokens(ExpertArgs &a, int dtype, cudaStream_t s, int n)
{
    if (n == 32) return run_type<F, 32>(a, dtype, s);
    if (n == 128) return run_type<F, 128>(a, dtype, s);
    return run_wide<F>(a, dtype, s);
}
int token_tile(long long n_rows, long long n_experts)
{
    // groups of 32 rows on average have larger ones among them, whose weights would be fetched twice (32 experts of 1024 x 1024, mean 20:
    // 16.9 us with 32 columns, 17.5 with 128; mean 32: 20.4 and 17.5)
    const long long mean = ceil_div(n_rows, n_experts);
    return mean <= 24 ? 32 : mean <= 128 ? 128 : 256;
}

bool rows16(const void *p, long long ld, long long rows, long long stride, long long n)
{
    return on(p, 16) && (rows <= 1 || ld % 8 == 0) && (n <= 1 || stride % 8 == 0);
}
// Extents that both calls share.
template <typename A> adascale_status check_sizes(const A &a)
{
    if (a.n_rows < 0 || a.n_experts < 1 || a.in_dim < 1 || a.out_dim < 1 || !is_itype(a.offset_type) || !a.offsets) return ADASCALE_ERR_INVALID_ARG;
    if (a.n_rows > kMaxRows - 512 || a.n_experts > kMaxExperts || a.in_dim > ADASCALE_EXPERT_MAX_DIM || a.out_dim > ADASCALE_EXPERT_MAX_DIM) return ADASCALE_ERR_TOO_LARGE;
    // tiles are counted in 32 bits
    const long long in = ceil_div(a.in_dim, kLanes), out = ceil_div(a.out_dim, kLanes);
    if ((a.n_rows / 32 + a.n_experts) > (1LL << 30) / std::max(in, out) || in * out > (1LL << 30) / a.n_experts) return ADASCALE_ERR_TOO_LARGE;
    return ADASCALE_OK;
}
template <typename A> bool weights_overlap(const A &a, long long ld, long long stride)
{
    return (a.out_dim > 1 && ld < a.in_dim) || (a.n_experts > 1 && stride < (a.out_dim - 1) * ld + a.in_dim);
}
template <typename A> ExpertArgs make_args(const A &a)
{
    ExpertArgs e = {};
    e.offsets = a.offsets;
    e.wide_offsets = a.offset_type == ADASCALE_I64;
    e.n_rows = a.n_rows;
    e.n_experts = (int)a.n_experts;
    return e;
}

}  // namespace

extern "C" adascale_status adascale_expert_matmul(const adascale_expert_matmul_args *args, void *cuda_stream)
{
    if (!args) return ADASCALE_ERR_INVALID_ARG;
    const adascale_expert_matmul_args &a = *args;
    const adascale_status bad = check_sizes(a);
    if (bad != ADASCALE_OK) return bad;
    if (!is_dtype(a.y_dtype) || !a.w || (a.n_rows > 0 && (!a.x || !a.y)) || (a.n_rows > 1 && (a.ld_x < a.in_dim || a.ld_y < a.out_dim)) ||
        weights_overlap(a, a.ld_w, a.stride_w))
        return ADASCALE_ERR_INVALID_ARG;
    if (!on(a.offsets, id_bytes(a.offset_type)) || !on(a.y, elem_bytes(a.y_dtype)) || !rows16(a.x, a.ld_x, a.n_rows, 0, 1) ||
        !rows16(a.w, a.ld_w, a.out_dim, a.stride_w, a.n_experts))
        return ADASCALE_ERR_ALIGNMENT;
    if (a.n_rows == 0) return ADASCALE_OK;
    ExpertArgs e = make_args(a);
    e.out = a.y;
    e.ld_out = a.ld_y;
    e.lanes = (int)a.out_dim;
    e.summed = (int)a.in_dim;
    e.leads = 1;  // this is no gradient: whatever comes next may start
    const int n = token_tile(a.n_rows, a.n_experts);
    if (!operand_map(&e.a, a.w, {a.n_experts, a.out_dim, a.in_dim, a.stride_w, a.ld_w}, kLanes) ||
        !operand_map(&e.b, a.x, {1, a.n_rows, a.in_dim, 0, a.ld_x}, std::min(n, 64)) ||
        !result_map(e, {1, a.n_rows, a.out_dim, 0, a.ld_y}, a.y_dtype, CU_TENSOR_MAP_SWIZZLE_NONE))
        return ADASCALE_ERR_CUDA;
    OPS_CU(run_tokens<Y>(e, a.y_dtype, static_cast<cudaStream_t>(cuda_stream), n));
    return ADASCALE_OK;
}

extern "C" adascale_status adascale_expert_matmul_grad(const adascale_expert_matmul_grad_args *args, void *cuda_stream)
{
    if (!args) return ADASCALE_ERR_INVALID_ARG;
    const adascale_expert_matmul_grad_args &a = *args;
    const adascale_status bad = check_sizes(a);
    if (bad != ADASCALE_OK) return bad;
    const bool rows = a.n_rows > 0;
    // without rows there is nothing to differentiate, but dw may have to be zero
    const bool want_dx = a.w && rows, want_dw = a.dw && (rows ? a.x != nullptr : !a.accumulate);
    if ((!a.w && !a.x && !a.dw) || (rows && !a.dy) || (want_dx && !a.dx) || (rows && a.x && !a.dw) || (want_dx && !is_dtype(a.dx_dtype)) ||
        (want_dw && !is_dtype(a.dw_dtype)) || (a.n_rows > 1 && (a.ld_dy < a.out_dim || (want_dx && a.ld_dx < a.in_dim) || (a.x && a.ld_x < a.in_dim))) ||
        (a.w && weights_overlap(a, a.ld_w, a.stride_w)) || (want_dw && weights_overlap(a, a.ld_dw, a.stride_dw)))
        return ADASCALE_ERR_INVALID_ARG;
    if (!on(a.offsets, id_bytes(a.offset_type)) || (want_dx && !on(a.dx, elem_bytes(a.dx_dtype))) || (want_dw && !on(a.dw, elem_bytes(a.dw_dtype))) ||
        (rows && (!rows16(a.dy, a.ld_dy, a.n_rows, 0, 1) || !rows16(a.x, a.ld_x, a.n_rows, 0, 1))) ||
        (a.w && !rows16(a.w, a.ld_w, a.out_dim, a.stride_w, a.n_experts)))
        return ADASCALE_ERR_ALIGNMENT;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    if (want_dx) {
        ExpertArgs e = make_args(a);
        e.out = a.dx;
        e.ld_out = a.ld_dx;
        e.lanes = (int)a.in_dim;
        e.summed = (int)a.out_dim;
        e.leads = want_dw;
        const int n = token_tile(a.n_rows, a.n_experts);
        if (!operand_map(&e.a, a.w, {a.n_experts, a.out_dim, a.in_dim, a.stride_w, a.ld_w}, kK) ||
            !operand_map(&e.b, a.dy, {1, a.n_rows, a.out_dim, 0, a.ld_dy}, std::min(n, 64)) ||
            !result_map(e, {1, a.n_rows, a.in_dim, 0, a.ld_dx}, a.dx_dtype, CU_TENSOR_MAP_SWIZZLE_NONE))
            return ADASCALE_ERR_CUDA;
        OPS_CU(run_tokens<DX>(e, a.dx_dtype, s, n));
    }
    if (want_dw) {
        ExpertArgs e = make_args(a);
        e.out = a.dw;
        e.ld_out = a.ld_dw;
        e.stride_out = a.stride_dw;
        e.lanes = (int)a.out_dim;
        e.columns = (int)a.in_dim;
        e.accumulate = a.accumulate != 0;
        e.follows = want_dx;
        // without rows no operand is copied
        if ((rows && (!operand_map(&e.a, a.dy, {1, a.n_rows, a.out_dim, 0, a.ld_dy}, kK) || !operand_map(&e.b, a.x, {1, a.n_rows, a.in_dim, 0, a.ld_x}, kK))) ||
            !result_map(e, {a.n_experts, a.out_dim, a.in_dim, a.stride_dw, a.ld_dw}, a.dw_dtype,
                        a.dw_dtype == ADASCALE_F32 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B))
            return ADASCALE_ERR_CUDA;
        OPS_CU(run_wide<DW>(e, a.dw_dtype, s));
    }
    return ADASCALE_OK;
}
