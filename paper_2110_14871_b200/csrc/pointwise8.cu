// The pointwise product on rows in 8 bits: y[r,d] = (sum_c x[r,c] w[d,c]) * ws[d] * xs[r] + bias[d].
#include <math.h>

#include <atomic>

#include "rows.cuh"

namespace gdws {
namespace {

__device__ int g_rows_status;        // status word of the calls on rows, one per device

// fp32 in the order that the interface names.  floor: 0 with ReLU, else -infinity; NaN stays NaN.
__device__ __forceinline__ float finish8(int sum, float ws, float xs, float bias, float floor)
{
    float v = fmaf((float)sum * ws, xs, bias);
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(v) : "f"(floor));
    return v;
}
__device__ __forceinline__ void store8(float *y, float v) { *y = v; }
__device__ __forceinline__ void store8(__nv_bfloat16 *y, float v) { *y = __float2bfloat16_rn(v); }

struct P8Params {
    const int8_t *x, *w;
    const float *xs, *ws, *bias;
    void *y;
    int64_t ldx, ldw, ldy;
    float floor;
    int rows, K, D;
    bool out_f32;
};

// ------------------------------------------------------------------------------------------
// Any alignment: 64 rows x 64 output channels a block, 64 bytes of the rows at a time through shared memory, products of four
// bytes on the ALUs.
// ------------------------------------------------------------------------------------------
__device__ __forceinline__ int load4(const int8_t *row, int k, int K, bool words)
{
    if (words && k + 4 <= K) return *reinterpret_cast<const int *>(row + k);
    int v = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (k + e < K) v |= (int)(uint8_t)row[k + e] << (8 * e);
    return v;
}

template <typename Y>
__global__ void __launch_bounds__(256) p8_alu_kernel(const __grid_constant__ P8Params P, int tiles_d)
{
    grid_launch_dependents();
    grid_dependency_wait();
    __shared__ int xt[64][17], wt[64][17];
    const int tile_r = (int)blockIdx.x / tiles_d, r0 = tile_r * 64, d0 = ((int)blockIdx.x - tile_r * tiles_d) * 64;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const bool xw = !(((uintptr_t)P.x | (uintptr_t)P.ldx) & 3), ww = !(((uintptr_t)P.w | (uintptr_t)P.ldw) & 3);
    int acc[4][4] = {};
    for (int k0 = 0; k0 < P.K; k0 += 64) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = ty + 16 * i;
            xt[row][tx] = r0 + row < P.rows ? load4(P.x + (int64_t)(r0 + row) * P.ldx, k0 + 4 * tx, P.K, xw) : 0;
            wt[row][tx] = d0 + row < P.D ? load4(P.w + (int64_t)(d0 + row) * P.ldw, k0 + 4 * tx, P.K, ww) : 0;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            int a[4], b[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) { a[i] = xt[ty + 16 * i][k]; b[i] = wt[tx + 16 * i][k]; }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = __dp4a(a[i], b[j], acc[i][j]);
        }
        __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int d = d0 + tx + 16 * j;
        if (d >= P.D) continue;
        const float ws = P.ws[d], bias = P.bias ? P.bias[d] : 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = r0 + ty + 16 * i;
            if (r < P.rows) store8((Y *)P.y + (int64_t)r * P.ldy + d, finish8(acc[i][j], ws, P.xs[r], bias, P.floor));
        }
    }
}

gdws_status_t p8_alu(const P8Params &P, cudaStream_t st)
{
    const int64_t tiles_d = ((int64_t)P.D + 63) / 64, tiles = ((int64_t)P.rows + 63) / 64 * tiles_d;
    if (tiles > 0x7fffffff) return fail(GDWS_ERR_UNSUPPORTED, "gdws_pointwise8: %d x %d outputs are more than one launch covers", P.rows, P.D);
    const cudaError_t e = launch_overlapped(P.out_f32 ? p8_alu_kernel<float> : p8_alu_kernel<__nv_bfloat16>, dim3((unsigned)tiles), 256u, 0, st, P, (int)tiles_d);
    return launched(e, "p8_alu_kernel launch");
}

// ------------------------------------------------------------------------------------------
// Tensor cores: kind::i8 products, 32-bit integer sums in tensor memory.
//
// Output channels are the products' rows (lanes of tensor memory), rows of x their columns: a warp that reads a column holds 32
// consecutive channels of one row of y, which it stores as they are -- any alignment and distance of y's rows, no staging --
// and a lane keeps its channel's scale and bias in registers.
//
// Operands: 128-byte pieces of 128 (weights) and nt (x) rows by TMA with the 128-byte swizzle; four products of 32 bytes each.
// TMA clips to the matrices and fills with zeros, which is what the sums need behind the last column.
// ------------------------------------------------------------------------------------------
constexpr int kP8Stages = 12;        // at most
constexpr int kPiece = 128;          // bytes of a row in a stage

struct alignas(64) P8TcParams {
    CUtensorMap tw, tx;
    const float *xs, *ws, *bias;
    void *y;
    int64_t ldy;
    float floor;
    int rows, D;
    int pieces;                      // of 128 columns
    int nt, tiles_r, split, ns, stage_bytes;      // slices
    int tiles_d, nitems, band;                    // pairs
};

__device__ __forceinline__ void umma8(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void umma8_pair(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
// Instruction descriptor of kind::i8: 32-bit integer sums, signed 8-bit operands, m x n.
__host__ __device__ constexpr uint32_t idesc8(int m, int n)
{
    return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t (&r)[8])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void st_cluster(uint32_t addr, int v)
{
    asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}

// Few outputs: a cluster of `split` blocks shares a tile of 128 channels x nt rows, each block sums a slice of the columns.  The
// partial sums are integers, so that adding them up in any order gives the same bits: each block sends its sums of column c of
// the tile to block c / (nt / split), which adds them and stores.
template <typename Y>
__global__ void __launch_bounds__(256, 1) p8_slices_kernel(const __grid_constant__ P8TcParams P)
{
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[2 * kP8Stages + 1];      // full, empty, done
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;
    __shared__ float xs_s[128];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    uint8_t *base = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const uint32_t s_s = smem_u32(base), recv_s = s_s + (uint32_t)(P.ns * P.stage_bytes);
    const uint32_t bar_full = smem_u32(&bars[0]), bar_empty = bar_full + 8 * kP8Stages, bar_done = bar_empty + 8 * kP8Stages;
    volatile int *const vabort = &abort_flag;
    const int rank = P.split > 1 ? (int)cluster_rank() : 0, tile = (int)blockIdx.x / P.split;
    const int tile_d = tile / P.tiles_r, d0 = tile_d * 128, r0 = (tile - tile_d * P.tiles_r) * P.nt;
    const int p0 = P.pieces * rank / P.split, n = P.pieces * (rank + 1) / P.split - p0;
    const uint32_t cols = (uint32_t)max(P.nt, 32);

    if (tid == 0) {
        abort_flag = 0;
        for (int i = 0; i < 2 * kP8Stages + 1; ++i) mbar_init(bar_full + 8 * i, 1);
        fence_mbar_init();
    }
    __syncwarp();
    grid_launch_dependents();
    if (warp == 0 && lane == 0) { prefetch_tensor_map(&P.tw); prefetch_tensor_map(&P.tx); }
    if (warp == 2) tmem_alloc(smem_u32(&tmem_slot), cols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (P.split > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");      // this block runs: its memory may be written
    grid_dependency_wait();
    const uint32_t tmem = tmem_slot;
    const int d = d0 + (tid & 127);
    const float ws = d < P.D ? P.ws[d] : 0.f, bias = d < P.D && P.bias ? P.bias[d] : 0.f;

    if (warp == 0) {
        if (lane == 0) {
            uint32_t s = 0, par = 1;
            int i = 0;
            for (; i < n; ++i) {
                if (i >= P.ns) mbar_wait_call(bar_empty + 8 * s, par, &abort_flag, &g_rows_status, kStatusWaitStage);
                if (*vabort) break;
                const uint32_t dst = s_s + s * (uint32_t)P.stage_bytes;
                mbar_expect_tx(bar_full + 8 * s, (uint32_t)P.stage_bytes);
                tma_load_2d(dst, &P.tw, (p0 + i) * kPiece, d0, bar_full + 8 * s);
                tma_load_2d(dst + 16384u, &P.tx, (p0 + i) * kPiece, r0, bar_full + 8 * s);
                if (++s == (uint32_t)P.ns) { s = 0; par ^= 1; }
            }
            // no copy into this block's memory may be in flight when it ends
            for (int j = 0; j < P.ns && j < i; ++j) mbar_wait_drain(bar_full + 8 * j, (uint32_t)((i - 1 - j) / P.ns) & 1u);
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0) {
            const uint32_t idesc = idesc8(128, P.nt);
            uint32_t s = 0, par = 0;
            for (int i = 0; i < n; ++i) {
                mbar_wait_call(bar_full + 8 * s, par, &abort_flag, &g_rows_status, kStatusWaitOperand);
                tc_fence_after();
                const uint32_t a = s_s + s * (uint32_t)P.stage_bytes;
#pragma unroll
                for (int k = 0; k < 4; ++k) umma8(tmem, make_sdesc(a + 32 * k, 16, 1024), make_sdesc(a + 16384u + 32 * k, 16, 1024), idesc, (uint32_t)(i | k));
                umma_commit(bar_empty + 8 * s);
                if (++s == (uint32_t)P.ns) { s = 0; par ^= 1; }
            }
            umma_commit(bar_done);
        }
        __syncwarp();
    } else if (warp >= 4 && tid - 128 < P.nt) {
        xs_s[tid - 128] = r0 + tid - 128 < P.rows ? P.xs[r0 + tid - 128] : 0.f;
    }
    __syncthreads();
    if (lane == 0) mbar_wait_call(bar_done, 0, &abort_flag, &g_rows_status, kStatusWaitMma);
    __syncwarp();
    tc_fence_after();

    const uint32_t t_base = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    Y *const y = (Y *)P.y + (int64_t)r0 * P.ldy + d;
    const int live = d < P.D ? P.rows - r0 : 0;      // columns of the tile that this lane stores
    if (P.split == 1) {
        for (int c = (warp >> 2) * 8; c < P.nt; c += 16) {
            uint32_t acc[8];
            tmem_ld8(t_base + (uint32_t)c, acc);
            tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (c + e < live) store8(y + (c + e) * P.ldy, finish8((int)acc[e], ws, xs_s[c + e], bias, P.floor));
        }
    } else {
        const int per = P.nt / P.split;             // columns that a block stores
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        for (int c = (warp >> 2) * 8; c < P.nt; c += 16) {
            uint32_t acc[8];
            tmem_ld8(t_base + (uint32_t)c, acc);
            tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int owner = (c + e) / per, at = rank * per + (c + e) - owner * per;
                st_cluster(map_shared(recv_s + (uint32_t)(at * 128 + (tid & 127)) * 4u, (uint32_t)owner), (int)acc[e]);
            }
        }
        cluster_sync();
        const int *recv = reinterpret_cast<const int *>(base + P.ns * P.stage_bytes);
        for (int c = tid >> 7; c < per; c += 2) {
            int sum = 0;
            for (int o = 0; o < P.split; ++o) sum += recv[(o * per + c) * 128 + (tid & 127)];
            const int at = rank * per + c;
            if (at < live) store8(y + at * P.ldy, finish8(sum, ws, xs_s[at], bias, P.floor));
        }
    }
    tc_fence_before();
    __syncthreads();
    __syncwarp();
    if (warp == 2) tmem_dealloc(tmem, cols);
}

// Many outputs: pairs of blocks (cta_group::2) compute 256 channels x 256 rows, each block's tensor memory holding its 128
// channels; persistent, two accumulators, so that a tile's epilogue passes under the next one's products.  A pair fetches 64 KB
// for 256 x 256 x 128 products, each block half of either operand.
constexpr int kPairStages = 6;
constexpr int kPairStage = 32768;
constexpr int kPairSmem = 1024 + kPairStages * kPairStage;
constexpr int kPairThreads = 12 * 32;       // loader, products, tensor memory, -, eight epilogue warps
struct P8Tile { int d0, r0; };
__device__ __forceinline__ P8Tile pair_tile(const P8TcParams &P, int item)
{
    // bands of rows' tiles, channels outermost within a band: what runs at a time reads about as many rows of x as of w
    const int per_band = P.band * P.tiles_d, b = item / per_band, in = item - b * per_band;
    const int h = min(P.band, P.tiles_r - b * P.band), d = in / h;
    return {d * 256, (b * P.band + in - d * h) * 256};
}

template <typename Y>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1) p8_pairs_kernel(const __grid_constant__ P8TcParams P)
{
    extern __shared__ uint8_t smem_raw[];
    constexpr int kBars = 2 * kPairStages + 5;
    __shared__ __align__(8) uint64_t bars[kBars];      // full, empty, accfull[2], accfree[2], drain
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;
    __shared__ float xs_s[2][256];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = cluster_rank();
    volatile int *const vabort = &abort_flag;
    uint8_t *base = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const uint32_t s_s = smem_u32(base);
    const uint32_t bar_full = smem_u32(&bars[0]), bar_empty = bar_full + 8 * kPairStages, bar_accfull = bar_empty + 8 * kPairStages, bar_accfree = bar_accfull + 16, bar_drain = bar_accfree + 16;

    if (tid == 0) {
        abort_flag = 0;
        for (int i = 0; i < kBars; ++i) mbar_init(bar_full + 8 * i, i >= 2 * kPairStages + 2 && i < 2 * kPairStages + 4 ? 16u : 1u);
        fence_mbar_init();
    }
    __syncwarp();
    grid_launch_dependents();
    if (warp == 0 && lane == 0) { prefetch_tensor_map(&P.tw); prefetch_tensor_map(&P.tx); }
    if (warp == 2) tmem_alloc_pair(smem_u32(&tmem_slot), 512);
    tc_fence_before();
    __syncthreads();
    cluster_sync();              // both blocks' barriers are initialised before either signals the other's
    tc_fence_after();
    grid_dependency_wait();
    const uint32_t tmem = tmem_slot;
    const int pair = (int)blockIdx.x >> 1, npairs = (int)gridDim.x >> 1;
    const int my_items = (P.nitems - pair + npairs - 1) / npairs;

    if (warp == 0) {
        if (lane == 0) {
            uint32_t s = 0, par = 1;
            int i = 0;
            bool stop = false;
            const uint32_t full0 = map_shared(bar_full, 0);
#pragma unroll 1
            for (int it = 0; it < my_items && !stop; ++it) {
                const P8Tile t = pair_tile(P, pair + it * npairs);
#pragma unroll 1
                for (int p = 0; p < P.pieces; ++p, ++i) {
                    if (i >= kPairStages) mbar_wait_call(bar_empty + 8 * s, par, &abort_flag, &g_rows_status, kStatusWaitStage);
                    if (*vabort) { stop = true; break; }
                    const uint32_t dst = s_s + s * (uint32_t)kPairStage;
                    if (rank == 0) mbar_expect_tx(bar_full + 8 * s, 2u * kPairStage);
                    tma_load_2d_pair(dst, &P.tw, p * kPiece, t.d0 + (int)rank * 128, full0 + 8 * s);
                    tma_load_2d_pair(dst + 16384u, &P.tx, p * kPiece, t.r0 + (int)rank * 128, full0 + 8 * s);
                    if (++s == (uint32_t)kPairStages) { s = 0; par ^= 1; }
                }
            }
            // the last phase armed on each stage completes when both blocks' copies have landed
            if (rank == 0)
                for (int j = 0; j < kPairStages && j < i; ++j) mbar_wait_drain(bar_full + 8 * j, (uint32_t)((i - 1 - j) / kPairStages) & 1u);
        }
        __syncwarp();
    } else if (warp == 1) {
        if (rank == 0 && lane == 0) {
            const uint32_t idesc = idesc8(256, 256);
            uint32_t s = 0, par = 0;
#pragma unroll 1
            for (int it = 0; it < my_items; ++it) {
                const int buf = it & 1;
                if (it >= 2) mbar_wait_cluster(bar_accfree + 8 * buf, (uint32_t)((it >> 1) - 1) & 1u, &abort_flag, &g_rows_status, kStatusWaitStage);
                tc_fence_after();
                const uint32_t acc = tmem + (uint32_t)(buf * 256);
#pragma unroll 1
                for (int p = 0; p < P.pieces; ++p) {
                    mbar_wait_call(bar_full + 8 * s, par, &abort_flag, &g_rows_status, kStatusWaitOperand);
                    tc_fence_after();
                    const uint32_t a = s_s + s * (uint32_t)kPairStage;
#pragma unroll
                    for (int k = 0; k < 4; ++k) umma8_pair(acc, make_sdesc(a + 32 * k, 16, 1024), make_sdesc(a + 16384u + 32 * k, 16, 1024), idesc, (uint32_t)(p | k));
                    umma_commit_pair(bar_empty + 8 * s);
                    if (++s == (uint32_t)kPairStages) { s = 0; par ^= 1; }
                }
                umma_commit_pair(bar_accfull + 8 * buf);
            }
            umma_commit_pair(bar_drain);
        }
        __syncwarp();
    } else if (warp >= 4) {
        const int et = tid - 128, half = et >> 7;      // this warp's half of the tile's rows
        const uint32_t free0 = map_shared(bar_accfree, 0);
#pragma unroll 1
        for (int it = 0; it < my_items; ++it) {
            const P8Tile t = pair_tile(P, pair + it * npairs);
            const int buf = it & 1, d = t.d0 + (int)rank * 128 + (et & 127);
            xs_s[buf][et] = t.r0 + et < P.rows ? P.xs[t.r0 + et] : 0.f;
            const float ws = d < P.D ? P.ws[d] : 0.f, bias = d < P.D && P.bias ? P.bias[d] : 0.f;
            named_bar_sync(1, 256);
            if (lane == 0) mbar_wait_relaxed_call<4096>(bar_accfull + 8 * buf, (uint32_t)(it >> 1) & 1u, &abort_flag, &g_rows_status, kStatusWaitMma);
            __syncwarp();
            tc_fence_after();
            const uint32_t t_base = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)(buf * 256 + half * 128);
            const int live = min(128, P.rows - t.r0 - half * 128);
#pragma unroll 1
            for (int c = 0; c < live; c += 32) {
                uint32_t acc[32];
                tmem_ld32(t_base + (uint32_t)c, acc);
                tmem_ld_wait();
                const float *xs = &xs_s[buf][half * 128 + c];
                Y *y = (Y *)P.y + (int64_t)(t.r0 + half * 128 + c) * P.ldy + d;
                if (d < P.D) {
                    // no condition between the columns of a whole block: 32 independent chains
                    if (c + 32 <= live) {
#pragma unroll
                        for (int e = 0; e < 32; ++e, y += P.ldy) store8(y, finish8((int)acc[e], ws, xs[e], bias, P.floor));
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; ++e, y += P.ldy)
                            if (c + e < live) store8(y, finish8((int)acc[e], ws, xs[e], bias, P.floor));
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(free0 + 8 * buf);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (tid == 0) mbar_wait_drain(bar_drain, 0);      // bounded, ignores the abort flag
    __syncwarp();
    cluster_sync();              // nothing of this pair is in flight any more: either block may end
    __syncwarp();
    if (warp == 2) tmem_dealloc_pair(tmem, 512);
}

gdws_status_t rows_map(CUtensorMap *map, const int8_t *q, int64_t rows, int cols, int64_t ld, int box_rows, int device)
{
    tensor_map_encode_fn encode = encode_fn();
    if (!encode) return fail(GDWS_ERR_CUDA, "cuTensorMapEncodeTiled is not available from this driver");
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)ld};
    const cuuint32_t box[2] = {(cuuint32_t)kPiece, (cuuint32_t)box_rows};
    const cuuint32_t estr[2] = {1, 1};
    auto make = [&] {
        return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<int8_t *>(q), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                      CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    };
    CUresult r = make();
    // a host thread whose first CUDA call this is has a current device, but no context bound to it yet
    if (r == CUDA_ERROR_INVALID_CONTEXT && cudaSetDevice(device) == cudaSuccess) r = make();
    return r == CUDA_SUCCESS ? GDWS_OK : fail(GDWS_ERR_CUDA, "cuTensorMapEncodeTiled failed with code %d", (int)r);
}

struct P8Choice {
    int kernel = GDWS_KERNEL8_ALU;
    int nt = 0, split = 1;
};

// Whether TMA can read these rows.
bool whole16(const int8_t *q, int64_t rows, int64_t ld) { return !((uintptr_t)q & 15) && (rows == 1 || ld % 16 == 0); }

P8Choice p8_choose(const P8Params &P, int sms)
{
    P8Choice c;
    if (!whole16(P.x, P.rows, P.ldx) || !whole16(P.w, P.D, P.ldw)) return c;
    const int pieces = (P.K + kPiece - 1) / kPiece;
    const int64_t pair_tiles = ((int64_t)P.D + 255) / 256 * (((int64_t)P.rows + 255) / 256);
    if (pair_tiles >= sms / 4) {
        c.kernel = GDWS_KERNEL8_PAIRS;
        return c;
    }
    c.kernel = GDWS_KERNEL8_SLICES;
    c.nt = 16;
    while (c.nt < 128 && c.nt < P.rows) c.nt *= 2;
    const int64_t tiles = ((int64_t)P.D + 127) / 128 * (((int64_t)P.rows + c.nt - 1) / c.nt);
    while (c.split < 8 && tiles * c.split * 2 <= sms && c.split * 2 <= pieces) c.split *= 2;
    return c;
}

gdws_status_t p8_tc(const P8Params &A, const P8Choice &c, int device, int sms, cudaStream_t st)
{
    P8TcParams P;
    const bool pairs = c.kernel == GDWS_KERNEL8_PAIRS;
    const int64_t ldx = (A.ldx + 15) / 16 * 16, ldw = (A.ldw + 15) / 16 * 16;      // of a single row any will do
    gdws_status_t rc = rows_map(&P.tw, A.w, A.D, A.K, ldw, 128, device);
    if (rc == GDWS_OK) rc = rows_map(&P.tx, A.x, A.rows, A.K, ldx, pairs ? 128 : c.nt, device);
    if (rc != GDWS_OK) return rc;
    P.xs = A.xs; P.ws = A.ws; P.bias = A.bias; P.y = A.y; P.ldy = A.ldy; P.rows = A.rows; P.D = A.D; P.floor = A.floor;
    P.pieces = (A.K + kPiece - 1) / kPiece;
    static std::atomic<bool> allowed[64];
    if (!allowed[device].load(std::memory_order_acquire)) {      // once per device: the full dynamic shared memory
        const cudaFuncAttribute most = cudaFuncAttributeMaxDynamicSharedMemorySize;
        cudaError_t e = cudaFuncSetAttribute(p8_slices_kernel<float>, most, kMaxSmem);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(p8_slices_kernel<__nv_bfloat16>, most, kMaxSmem);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(p8_pairs_kernel<float>, most, kPairSmem);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(p8_pairs_kernel<__nv_bfloat16>, most, kPairSmem);
        if (e != cudaSuccess) return launched(e, "cudaFuncSetAttribute(pointwise8)");
        allowed[device].store(true, std::memory_order_release);
    }
    cudaError_t e;
    if (pairs) {
        P.tiles_d = (A.D + 255) / 256; P.tiles_r = (int)(((int64_t)A.rows + 255) / 256);
        const int64_t items = (int64_t)P.tiles_d * P.tiles_r;
        if (items > 0x3fffffff) return fail(GDWS_ERR_UNSUPPORTED, "gdws_pointwise8: %d x %d outputs are more than one launch covers", A.rows, A.D);
        P.nitems = (int)items; P.band = 8;
        const unsigned grid = 2u * (unsigned)std::min<int64_t>(items, sms / 2);
        e = launch_overlapped(A.out_f32 ? p8_pairs_kernel<float> : p8_pairs_kernel<__nv_bfloat16>, dim3(grid), (unsigned)kPairThreads, kPairSmem, st, P);
    } else {
        P.nt = c.nt; P.split = c.split; P.tiles_r = (int)(((int64_t)A.rows + c.nt - 1) / c.nt);
        const int64_t blocks = ((int64_t)A.D + 127) / 128 * P.tiles_r * c.split;
        if (blocks > 0x7fffffff) return fail(GDWS_ERR_UNSUPPORTED, "gdws_pointwise8: %d x %d outputs are more than one launch covers", A.rows, A.D);
        P.stage_bytes = 16384 + c.nt * kPiece;
        const size_t recv = c.split > 1 ? (size_t)c.nt * 512 : 0;
        P.ns = std::min({(P.pieces + c.split - 1) / c.split, kP8Stages, (int)((kMaxSmem - 1024 - recv) / P.stage_bytes)});
        // Blocks of a cluster that wait for each other hold tensor memory meanwhile.  Two such kernels on one SM could each hold what
        // a block of the other's clusters waits for, so they take more than half of the shared memory: one block per SM.
        const size_t need = 1024 + (size_t)P.ns * P.stage_bytes + recv;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)blocks); cfg.blockDim = dim3(256); cfg.stream = st;
        cfg.dynamicSmemBytes = c.split > 1 ? std::max(need, (size_t)kMaxSmem / 2 + 2048) : smem_for_tmem(need, std::max(c.nt, 32));
        cudaLaunchAttribute attr[2];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = (unsigned)c.split; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
        cfg.attrs = attr; cfg.numAttrs = c.split > 1 ? 2 : 1;
        e = A.out_f32 ? cudaLaunchKernelEx(&cfg, p8_slices_kernel<float>, P) : cudaLaunchKernelEx(&cfg, p8_slices_kernel<__nv_bfloat16>, P);
    }
    return launched(e, pairs ? "p8_pairs_kernel launch" : "p8_slices_kernel launch");
}

// The call's arguments as the kernels take them; a single row has no distance to a next one.
P8Params p8_params(const gdws_rows8_t *x, const gdws_rows8_t *w, const float *bias, int relu, const gdws_rows_t *y)
{
    P8Params P;
    P.x = x->q; P.w = w->q; P.xs = x->scale; P.ws = w->scale; P.bias = bias; P.y = y->ptr;
    P.ldx = x->rows > 1 ? x->ld : x->cols; P.ldw = w->rows > 1 ? w->ld : w->cols; P.ldy = y->rows > 1 ? y->ld : y->cols;
    P.rows = (int)x->rows; P.K = x->cols; P.D = (int)w->rows; P.floor = relu ? 0.f : -INFINITY; P.out_f32 = y->dtype == GDWS_F32;
    return P;
}

}  // namespace
}  // namespace gdws

using namespace gdws;

extern "C" {

gdws_status_t gdws_pointwise8(const gdws_rows8_t *x, const gdws_rows8_t *w, const float *bias, int relu, const gdws_rows_t *y, void *stream)
{
    gdws_status_t st = check_pointwise8(x, w, bias, y);
    if (st != GDWS_OK || !x->rows) return st;
    int device, sms;
    st = rows_device(&device, &sms);
    if (st != GDWS_OK) return st;
    const P8Params P = p8_params(x, w, bias, relu, y);
    const P8Choice c = p8_choose(P, sms);
    return c.kernel == GDWS_KERNEL8_ALU ? p8_alu(P, (cudaStream_t)stream) : p8_tc(P, c, device, sms, (cudaStream_t)stream);
}

gdws_status_t gdws_pointwise8_kernel(const gdws_rows8_t *x, const gdws_rows8_t *w, const gdws_rows_t *y, int *kernel)
{
    const gdws_status_t st = check_pointwise8(x, w, nullptr, y);
    if (st != GDWS_OK) return st;
    if (!kernel) return fail(GDWS_ERR_INVALID_ARG, "gdws_pointwise8_kernel: kernel is NULL");
    int device, sms = kB200Sms;
    if (cudaGetDevice(&device) != cudaSuccess || rows_device(&device, &sms) != GDWS_OK) { cudaGetLastError(); sms = kB200Sms; }
    *kernel = x->rows ? p8_choose(p8_params(x, w, nullptr, 0, y), sms).kernel : GDWS_KERNEL8_NONE;
    return GDWS_OK;
}

gdws_status_t gdws_rows_status(void)
{
    int device, sms;
    const gdws_status_t st = rows_device(&device, &sms);
    if (st != GDWS_OK) return st;
    int word = 0;
    const int zero = 0;
    cudaError_t e = cudaDeviceSynchronize();
    if (e == cudaSuccess) e = cudaMemcpyFromSymbol(&word, g_rows_status, sizeof(int));
    if (e == cudaSuccess && word) e = cudaMemcpyToSymbol(g_rows_status, &zero, sizeof(int));
    if (e != cudaSuccess) return cuda_fail(e, "status read");
    if (word) return fail(GDWS_ERR_DEVICE_TIMEOUT, "a bounded wait inside a kernel expired (status word 0x%x)", word);
    return GDWS_OK;
}

}  // extern "C"
