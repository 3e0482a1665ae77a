// Products with experts' weights over ragged groups of rows, and their gradients, on the fifth-generation tensor cores.
//
//   y_r = W_e x_r       dx_r = W_e^T dy_r       dW_e (+)= sum over e's rows of dy_r x_r^T
//
// One kernel of three forms.  Each computes tiles D[128 x n] = A[128 x k] B[n x k]^T with A's rows on the 128 lanes of tensor
// memory and n, a multiple of 16 up to NT, its columns:
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
// A block a SM walks over the tiles: one warp issues the copies (tensor maps, 128-byte swizzle) into a ring of stages of 64
// summands, one the matrix instructions, four bring finished tiles from tensor memory, where two take turns, to memory.
// Every block works out the tiles from the offsets by itself: no host, no kernel before.
#include "ops_common.cuh"

#include <cuda.h>

#include <algorithm>

namespace {

constexpr int kMaxExperts = ADASCALE_EXPERT_MAX_EXPERTS;
constexpr int kM = 128;          // lanes of a tile
constexpr int kK = 64;           // summands of a stage: 128 bytes, the swizzle's width
constexpr int kTokenBox = 32;    // rows of one copy of tokens
constexpr int kThreads = 192;    // copies, matrix instructions, four warps for results
constexpr int kRingMax = 200 * 1024;

enum Form { Y, DX, DW };

struct ExpertArgs {
    CUtensorMap a, b;
    const void *offsets;
    void *out;
    long long n_rows;
    long long ld_out, stride_out;  // DW: rows and experts of dw
    int n_experts, wide_offsets;
    int lanes, columns, summed;    // extents; the one that is e's rows is 0
    int accumulate, out_aligned;
};

// ---- tensor memory and matrix instructions -------------------------------------------------

__device__ __forceinline__ void tmem_alloc(unsigned *where, unsigned columns)
{
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(where)), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(unsigned base, unsigned columns)
{
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns));
}
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// All matrix instructions that this thread has issued arrive at the barrier when they are done.
__device__ __forceinline__ void mma_commit(u64 *bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void mma(unsigned d, u64 a, u64 b, unsigned what, bool add)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b),
                 "r"(what), "r"((unsigned)add)
                 : "memory");
}
// 32 columns of this warp's 32 lanes
__device__ __forceinline__ void tmem_load(unsigned at, float (&x)[32])
{
    unsigned r[32];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
                   "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
                   "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(at));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) x[i] = __uint_as_float(r[i]);
}
// A copy by a tensor map; the innermost coordinate is a multiple of 8 elements (16 bytes).
__device__ __forceinline__ void tensor_load(void *dst, const CUtensorMap *map, int x, int y, int z, u64 *bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(smem_u32(dst)),
                 "l"(map), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z)
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

// ---- tiles ---------------------------------------------------------------------------------

// Of each expert: its rows, and the number of tiles before it.
struct Experts {
    int *begin;  // [n + 1]: begin[e + 1] is where e ends
    int *tiles;  // [n + 1]
};

// Tiles of one expert: across the lanes, and across the columns.
template <Form F, int NT> __device__ __forceinline__ int column_tiles(const ExpertArgs &a, int rows)
{
    return F == DW ? (a.columns + NT - 1) / NT : (rows + NT - 1) / NT;
}

// By one warp: offsets, ascending and within the rows, and running sums of the tiles.
template <Form F, int NT> __device__ __forceinline__ void find_tiles(const ExpertArgs &a, const Experts &x)
{
    const int lane = threadIdx.x % 32, lane_tiles = (a.lanes + kM - 1) / kM;
    int floor = 0;
    for (int i = lane; i - lane <= a.n_experts; i += 32) {
        long long o = i <= a.n_experts ? load_id(a.offsets, a.wide_offsets, i) : 0;
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
    int sum = 0;
    for (int i = lane; i - lane < a.n_experts; i += 32) {
        int v = 0;
        if (i < a.n_experts) {
            const int rows = x.begin[i + 1] - x.begin[i];
            v = rows || (F == DW && !a.accumulate) ? lane_tiles * column_tiles<F, NT>(a, rows) : 0;
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
    if (lane == 0) x.tiles[0] = 0;
}

struct Tile {
    int expert;
    int lane;           // first lane
    int column, width;  // first column (Y, DX: a row of the tokens), how many
    int row, summands;  // DW: first row; how many summands there are
};
// The tile that comes after `t.expert`'s first tiles; tiles ascend from call to call.
template <Form F, int NT> __device__ __forceinline__ void find_tile(const ExpertArgs &a, const Experts &x, int tile, Tile &t)
{
    while (tile >= x.tiles[t.expert + 1]) ++t.expert;
    const int begin = x.begin[t.expert], rows = x.begin[t.expert + 1] - begin, k = tile - x.tiles[t.expert];
    const int across = column_tiles<F, NT>(a, rows), col = k % across;
    t.lane = k / across * kM;
    if (F == DW) {
        t.column = col * NT;
        t.width = min(NT, a.columns - t.column);
        t.row = begin;
        t.summands = rows;
    } else {  // of equal width, in steps of 16
        const int each = ((rows + across - 1) / across + 15) / 16 * 16;
        t.column = begin + col * each;
        t.width = min(each, rows - col * each);
        t.row = 0;
        t.summands = a.summed;
    }
}

// A wait of a whole warp, with one answer for all of it.
__device__ __forceinline__ bool wait_all(u64 *bar, unsigned parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity)); }

// ---- the kernel ----------------------------------------------------------------------------

template <int NT> constexpr int kStageBytes = (kM + NT) * kK * 2;
template <int NT> constexpr int kStages = kRingMax / kStageBytes<NT>;
template <int NT> constexpr int kSmemBytes = 1024 + kStages<NT> * kStageBytes<NT>;  // the ring starts on a boundary of 1024

template <Form F, int NT, typename O> __global__ void __launch_bounds__(kThreads) k_expert(const __grid_constant__ ExpertArgs a)
{
    constexpr int S = kStages<NT>;
    constexpr unsigned kColumns = NT <= 16 ? 32 : 2 * NT;
    extern __shared__ unsigned char raw[];
    __shared__ u64 full[S], empty[S], done[2], taken[2];
    __shared__ unsigned tmem_base;
    __shared__ int begins[kMaxExperts + 1], tile_sums[kMaxExperts + 1];
    unsigned char *ring = raw + (1024 - smem_u32(raw) % 1024) % 1024;
    const Experts x = {begins, tile_sums};
    const int warp = threadIdx.x / 32;

    if (threadIdx.x == 0) {
        for (int i = 0; i < S; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&done[i], 1);
            mbar_init(&taken[i], 128);
        }
        mbar_publish();
    }
    if (warp == 1) tmem_alloc(&tmem_base, kColumns);
    griddep_wait();
    if (warp == 0) find_tiles<F, NT>(a, x);
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const unsigned tmem = tmem_base;
    const int n_tiles = x.tiles[a.n_experts];
    // operands whose summands lie across the rows in memory
    constexpr bool kAcrossA = F != Y, kAcrossB = F == DW;

    if (warp == 0) {
        if (threadIdx.x == 0) {
            Tile t = {};
            int stage = 0, issued = 0;
            unsigned phase = 1;  // the first pass over the ring waits for nobody
            bool ok = true;
            for (int tile = blockIdx.x; tile < n_tiles && ok; tile += gridDim.x) {
                find_tile<F, NT>(a, x, tile, t);
                for (int k = 0; k < t.summands; k += kK) {
                    if (!mbar_wait(&empty[stage], phase)) {
                        ok = false;
                        break;
                    }
                    unsigned char *as = ring + stage * kStageBytes<NT>, *bs = as + kM * kK * 2;
                    u64 *bar = &full[stage];
                    if constexpr (F == DW) {
                        const int boxes = (t.width + 63) / 64;
                        mbar_expect_tx(bar, (2 + boxes) * 8192);
                        for (int i = 0; i < 2; ++i) tensor_load(as + i * 8192, &a.a, t.lane + 64 * i, t.row + k, 0, bar);
                        for (int i = 0; i < boxes; ++i) tensor_load(bs + i * 8192, &a.b, t.column + 64 * i, t.row + k, 0, bar);
                    } else {
                        const int boxes = (t.width + kTokenBox - 1) / kTokenBox;
                        mbar_expect_tx(bar, kM * kK * 2 + boxes * kTokenBox * kK * 2);
                        if constexpr (F == Y) {
                            tensor_load(as, &a.a, k, t.lane, t.expert, bar);
                        } else {
                            for (int i = 0; i < 2; ++i) tensor_load(as + i * 8192, &a.a, t.lane + 64 * i, k, t.expert, bar);
                        }
                        for (int i = 0; i < boxes; ++i) tensor_load(bs + i * kTokenBox * kK * 2, &a.b, k, t.column + i * kTokenBox, 0, bar);
                    }
                    ++issued;
                    if (++stage == S) stage = 0, phase ^= 1;
                }
            }
            // copies in flight end before the block does
            for (int i = 0; i < min(issued, S); ++i) {
                const int n = issued - 1 - i;
                mbar_wait(&full[n % S], (n / S) & 1);
            }
        }
    } else if (warp == 1) {
        Tile t = {};
        int stage = 0, turn = 0;
        unsigned phase = 0, free_phase[2] = {1, 1};
        bool ok = true;
        for (int tile = blockIdx.x; tile < n_tiles && ok; tile += gridDim.x) {
            find_tile<F, NT>(a, x, tile, t);
            if (t.summands == 0) continue;
            ok = wait_all(&taken[turn], free_phase[turn]);
            free_phase[turn] ^= 1;
            tmem_fence_after();
            const unsigned d = tmem + turn * NT;
            const unsigned what = 1u << 4 | 1u << 7 | 1u << 10 | (kAcrossA ? 1u << 15 : 0u) | (kAcrossB ? 1u << 16 : 0u) |
                                  (unsigned)((t.width + 15) / 16 * 2) << 17 | (unsigned)(kM / 16) << 24;
            for (int k = 0; k < t.summands && ok; k += kK) {
                ok = wait_all(&full[stage], phase);
                if (!ok) break;
                tmem_fence_after();
                unsigned char *as = ring + stage * kStageBytes<NT>, *bs = as + kM * kK * 2;
                const int left = t.summands - k;
                if (F == DW && left < kK) {  // rows of the next expert, or of nobody
                    const int boxes = 2 + (t.width + 63) / 64, step_end = (left + 15) / 16 * 16;
                    for (int box = 0; box < boxes; ++box)
                        for (int i = threadIdx.x % 32; i < (step_end - left) * 8; i += 32)
                            reinterpret_cast<uint4 *>(as + box * 8192 + left * 128)[i] = make_uint4(0, 0, 0, 0);
                    copy_fence();
                    __syncwarp();
                }
                if (threadIdx.x % 32 == 0) {
                    const u64 da = operand(smem_u32(as), kAcrossA ? 8192 : 16), db = operand(smem_u32(bs), kAcrossB ? 8192 : 16);
#pragma unroll
                    for (int i = 0; i < kK / 16; ++i) {
                        if (16 * i >= left) break;
                        mma(d, da + (u64)(i * (kAcrossA ? 2048 : 32) >> 4), db + (u64)(i * (kAcrossB ? 2048 : 32) >> 4), what, k + i > 0);
                    }
                    mma_commit(&empty[stage]);
                }
                __syncwarp();
                if (++stage == S) stage = 0, phase ^= 1;
            }
            if (ok && threadIdx.x % 32 == 0) mma_commit(&done[turn]);
            __syncwarp();
            turn ^= 1;
        }
    } else {
        const int lane = threadIdx.x % 32, quarter = warp % 4;  // a warp reads the quarter of the lanes that its number names
        Tile t = {};
        int turn = 0;
        unsigned phase[2] = {0, 0};
        bool ok = true;
        O *out = static_cast<O *>(a.out);
        for (int tile = blockIdx.x; tile < n_tiles; tile += gridDim.x) {
            find_tile<F, NT>(a, x, tile, t);
            const bool any = t.summands > 0;
            if (any && ok) {
                ok = wait_all(&done[turn], phase[turn]);
                tmem_fence_after();
            }
            if (any) phase[turn] ^= 1;
            const int row = t.lane + quarter * 32 + lane;
            const unsigned at = tmem + turn * NT + ((unsigned)(quarter * 32) << 16);
            for (int c = 0; c < t.width; c += 32) {
                float v[32];
                __syncwarp();
                if (any && ok) {
                    tmem_load(at + c, v);
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = any ? NAN : 0.f;  // NaN: a wait was given up
                }
                const int n = row < a.lanes ? min(32, t.width - c) : 0;
                if constexpr (F == DW) {
                    O *p = out + t.expert * a.stride_out + row * a.ld_out + t.column + c;
                    if (a.out_aligned && n == 32) {
                        constexpr int V = 16 / sizeof(O);
#pragma unroll
                        for (int i = 0; i < 32; i += V) {
                            float part[V];
#pragma unroll
                            for (int k = 0; k < V; ++k) part[k] = v[i + k];
                            if (a.accumulate) {
                                float old[V];
                                load_vec<V>(p + i, old);
#pragma unroll
                                for (int k = 0; k < V; ++k) part[k] += old[k];
                            }
                            store_vec<V>(p + i, part);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (i < n) put(p + i, a.accumulate ? v[i] + to_f32(p[i]) : v[i]);
                    }
                } else {
                    O *p = out + (t.column + c) * a.ld_out + row;
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (i < n) put(p + i * a.ld_out, v[i]);
                }
            }
            if (any) {
                tmem_fence_before();
                mbar_arrive(&taken[turn]);
                turn ^= 1;
            }
        }
    }
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    if (warp == 1) tmem_free(tmem, kColumns);
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
// [n, rows, cols] of bf16 with `ld` and `stride` elements between rows and matrices; boxes of 64 columns and `box` rows.
bool make_map(CUtensorMap *map, const void *p, long long n, long long rows, long long cols, long long stride, long long ld, int box)
{
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    const long long wide = (cols + 7) / 8 * 8;  // a stride that is never used still has to be one
    if (rows <= 1) ld = std::max(ld, wide) / 8 * 8;
    if (n <= 1) stride = ld * rows;
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)n}, strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)stride * 2};
    const cuuint32_t boxes[3] = {64, (cuuint32_t)box, 1}, steps[3] = {1, 1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(p), dims, strides, boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <Form F, int NT, typename O> cudaError_t run_tiles(const ExpertArgs &a, long long tiles, cudaStream_t s)
{
    static OncePerDevice known;
    cudaError_t e = allow_smem(reinterpret_cast<const void *>(&k_expert<F, NT, O>), known);
    if (e != cudaSuccess) return e;
    const int sms = sm_count();
    if (sms <= 0) return cudaErrorUnknown;
    return launch(k_expert<F, NT, O>, std::min<long long>(tiles, sms), kThreads, kSmemBytes<NT>, s, a);
}
template <Form F, int NT> cudaError_t run_type(const ExpertArgs &a, int dtype, cudaStream_t s)
{
    const long long lane_tiles = ceil_div(a.lanes, kM);
    // at most this many tiles: each expert may have one that is not full
    const long long tiles = F == DW ? a.n_experts * lane_tiles * ceil_div(a.columns, NT)
                                    : lane_tiles * (a.n_rows / NT + std::min<long long>(a.n_experts, a.n_rows));
    return dtype == ADASCALE_BF16 ? run_tiles<F, NT, bf16>(a, tiles, s) : run_tiles<F, NT, float>(a, tiles, s);
}
// Tiles of tokens are as wide as the rows of an expert on average, as far as the host knows.
template <Form F> cudaError_t run_tokens(const ExpertArgs &a, int dtype, cudaStream_t s)
{
    const long long mean = ceil_div(a.n_rows, a.n_experts);
    if (mean <= 32) return run_type<F, 32>(a, dtype, s);
    if (mean <= 128) return run_type<F, 128>(a, dtype, s);
    return run_type<F, 256>(a, dtype, s);
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
    const long long in = ceil_div(a.in_dim, kM), out = ceil_div(a.out_dim, kM);
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
    if (!make_map(&e.a, a.w, a.n_experts, a.out_dim, a.in_dim, a.stride_w, a.ld_w, kM) ||
        !make_map(&e.b, a.x, 1, a.n_rows, a.in_dim, 0, a.ld_x, kTokenBox))
        return ADASCALE_ERR_CUDA;
    OPS_CU(run_tokens<Y>(e, a.y_dtype, static_cast<cudaStream_t>(cuda_stream)));
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
        if (!make_map(&e.a, a.w, a.n_experts, a.out_dim, a.in_dim, a.stride_w, a.ld_w, kK) ||
            !make_map(&e.b, a.dy, 1, a.n_rows, a.out_dim, 0, a.ld_dy, kTokenBox))
            return ADASCALE_ERR_CUDA;
        OPS_CU(run_tokens<DX>(e, a.dx_dtype, s));
    }
    if (want_dw) {
        ExpertArgs e = make_args(a);
        e.out = a.dw;
        e.ld_out = a.ld_dw;
        e.stride_out = a.stride_dw;
        e.lanes = (int)a.out_dim;
        e.columns = (int)a.in_dim;
        e.accumulate = a.accumulate != 0;
        const int v = 16 / elem_bytes(a.dw_dtype);
        e.out_aligned = on(a.dw, 16) && a.ld_dw % v == 0 && a.stride_dw % v == 0;
        // without rows no copy is made
        if (rows && (!make_map(&e.a, a.dy, 1, a.n_rows, a.out_dim, 0, a.ld_dy, kK) || !make_map(&e.b, a.x, 1, a.n_rows, a.in_dim, 0, a.ld_x, kK)))
            return ADASCALE_ERR_CUDA;
        OPS_CU(run_type<DW, 256>(e, a.dw_dtype, s));
    }
    return ADASCALE_OK;
}
