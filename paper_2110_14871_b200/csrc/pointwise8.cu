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
    const float v = fmaf((float)sum * ws, xs, bias);
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(v), "f"(floor));
    return r;
}
__device__ __forceinline__ void store8(float *y, float v) { *y = v; }
__device__ __forceinline__ void store8(__nv_bfloat16 *y, float v) { *y = __float2bfloat16_rn(v); }

// The same for two outputs at a time, on packed pairs.
__device__ __forceinline__ uint64_t pair_of(float lo, float hi)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void finish8x2(uint32_t a, uint32_t b, uint64_t ws, uint64_t xs, uint64_t bias, float &lo, float &hi)
{
    uint64_t v = pair_of((float)(int)a, (float)(int)b);
    asm("mul.rn.f32x2 %0, %0, %1;" : "+l"(v) : "l"(ws));
    asm("fma.rn.f32x2 %0, %0, %1, %2;" : "+l"(v) : "l"(xs), "l"(bias));
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
// Rounding is monotonic: the larger of the rounded value and the floor is the rounded larger one.
__device__ __forceinline__ uint32_t round_bf16x2(float lo, float hi, uint32_t floor2)
{
    uint32_t v = pack_bf16x2(lo, hi);
    asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(v) : "r"(floor2));
    return v;
}
__device__ __forceinline__ float max_nan(float v, float floor)
{
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(v) : "f"(floor));
    return v;
}

// Whether rows start at multiples of 16 bytes, as TMA and 16-byte loads need it.
bool whole16(const int8_t *q, int64_t rows, int64_t ld) { return !((uintptr_t)q & 15) && (rows == 1 || ld % 16 == 0); }

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
// Any alignment: 64 rows x 64 output channels a block, 64 columns of the rows at a time through registers into shared memory, from
// there by warp-wide products of 16 x 8 x 32 (four-byte dot products run at some 30 a clock and SM here: 4000 x 2001 -> 2000 510 us).
// ------------------------------------------------------------------------------------------
__device__ __forceinline__ int dot16(const int4 &a, const int4 &b, int acc) { return __dp4a(a.w, b.w, __dp4a(a.z, b.z, __dp4a(a.y, b.y, __dp4a(a.x, b.x, acc)))); }
// A row that starts anywhere, read by aligned words that hold at least one of its bytes.
struct Bytes {
    const uint32_t *first;
    int last;                    // the last such word
    uint32_t shift;
    __device__ __forceinline__ Bytes() {}
    __device__ __forceinline__ Bytes(const int8_t *row, int K)
    {
        const int off = (int)((uintptr_t)row & 3);
        first = reinterpret_cast<const uint32_t *>(row - off);
        last = (off + K - 1) / 4;
        shift = 8u * (uint32_t)off;
    }
    // the two words around columns k to k + 3 (k a multiple of 4), put together when they are needed, so that many are on their way
    // at once; what lies behind the last column is anything
    __device__ __forceinline__ uint2 load(int k) const { return make_uint2(first[min(k / 4, last)], first[min(k / 4 + 1, last)]); }
    __device__ __forceinline__ int join(uint2 v) const { return (int)__funnelshift_r(v.x, v.y, shift); }
};
// The first n of four bytes, zeros for the others (it suffices that one factor has them).
__device__ __forceinline__ int first4(int v, int n) { return n >= 4 ? v : (n <= 0 ? 0 : v & ((1 << (8 * n)) - 1)); }

template <typename Y>
__global__ void __launch_bounds__(256) p8_any_kernel(const __grid_constant__ P8Params P, int tiles_d)
{
    grid_launch_dependents();
    grid_dependency_wait();
    __shared__ int xt[64][20], wt[64][20];           // 16 words a row; pitch 20: eight rows' four words lie in 32 banks
    const int tile_r = (int)blockIdx.x / tiles_d, r0 = tile_r * 64, d0 = ((int)blockIdx.x - tile_r * tiles_d) * 64;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // rows and channels behind the last repeat it: what comes of them is not stored
    Bytes xr[4], wr[4];
    uint2 xn[4], wn[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        xr[i] = Bytes(P.x + (int64_t)min(r0 + ty + 16 * i, P.rows - 1) * P.ldx, P.K);
        wr[i] = Bytes(P.w + (int64_t)min(d0 + ty + 16 * i, P.D - 1) * P.ldw, P.K);
    }
    auto fetch = [&](int k0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            xn[i] = xr[i].load(k0 + 4 * tx);
            wn[i] = wr[i].load(k0 + 4 * tx);
        }
    };
    // a warp: 16 rows, 32 channels as four products of 8; lane l has the sums of rows l / 4 and l / 4 + 8, channels 2 (l % 4) and the next
    const int m0 = (warp & 3) * 16 + lane / 4, n0 = (warp >> 2) * 32, kw = lane % 4;
    int acc[4][4] = {};
    fetch(0);
    for (int k0 = 0; k0 < P.K; k0 += 64) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) { xt[ty + 16 * i][tx] = first4(xr[i].join(xn[i]), P.K - k0 - 4 * tx); wt[ty + 16 * i][tx] = wr[i].join(wn[i]); }
        __syncthreads();
        if (k0 + 64 < P.K) fetch(k0 + 64);               // under this piece's products
#pragma unroll
        for (int k = 0; k < 16; k += 8) {
            const int a0 = xt[m0][k + kw], a1 = xt[m0 + 8][k + kw], a2 = xt[m0][k + 4 + kw], a3 = xt[m0 + 8][k + 4 + kw];
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const int b0 = wt[n0 + 8 * n + lane / 4][k + kw], b1 = wt[n0 + 8 * n + lane / 4][k + 4 + kw];
                asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                    : "+r"(acc[n][0]), "+r"(acc[n][1]), "+r"(acc[n][2]), "+r"(acc[n][3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
            }
        }
    }
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int r = r0 + m0 + (e >> 1) * 8, d = d0 + n0 + 8 * n + 2 * kw + (e & 1);
            if (r < P.rows && d < P.D) store8((Y *)P.y + (int64_t)r * P.ldy + d, finish8(acc[n][e], P.ws[d], P.xs[r], P.bias ? P.bias[d] : 0.f, P.floor));
        }
}

gdws_status_t p8_any(const P8Params &P, cudaStream_t st)
{
    const int64_t tiles_d = ((int64_t)P.D + 63) / 64, tiles = ((int64_t)P.rows + 63) / 64 * tiles_d;
    if (tiles > 0x7fffffff) return fail(GDWS_ERR_UNSUPPORTED, "gdws_pointwise8: %d x %d outputs are more than one launch covers", P.rows, P.D);
    const cudaError_t e = launch_overlapped(P.out_f32 ? p8_any_kernel<float> : p8_any_kernel<__nv_bfloat16>, dim3((unsigned)tiles), 256u, 0, st, P, (int)tiles_d);
    return launched(e, "p8_any_kernel launch");
}

// ------------------------------------------------------------------------------------------
// A few rows (single tokens): the time is that of reading w.  A warp takes kFewD output channels; its lanes read 16 bytes each of
// 512 consecutive ones of every channel's row, straight into registers, and multiply them with the same piece of the R rows of x
// (which stay in L1) by four-byte dot products.  `share` warps of a block share the columns of a group of channels.  (The tensor
// cores take some 115 cycles for a 128 x 32 byte piece of w whatever the rows of x are, 36 bytes a clock: a tile of 128 channels is
// slower there unless a cluster shares its sum, which costs a microsecond: 1 x 4096 -> 4096 6.8 us, here 3.9.)
// ------------------------------------------------------------------------------------------
constexpr int kFewD = 4, kFewRows = 8;
// (Not through the read-only path: this kernel may have started before the one that writes w ended.)
__device__ __forceinline__ int4 load_weights(const int8_t *p)
{
    int4 v;
    asm volatile("ld.global.L1::no_allocate.L2::256B.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

// WHOLE: rows start at multiples of 16 bytes; otherwise the lanes take four columns each.
template <typename Y, int R, bool WHOLE>
__global__ void __launch_bounds__(256) p8_few_kernel(const __grid_constant__ P8Params P, int share)
{
    grid_launch_dependents();
    grid_dependency_wait();
    constexpr int kSums = kFewD * R;
    static_assert(kSums <= 32, "a lane per sum");
    __shared__ int part[8][kSums];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int me = warp % share;                                            // which part of the columns
    const int64_t group = (int64_t)blockIdx.x * (8 / share) + warp / share;
    const int d0 = (int)min(group * kFewD, (int64_t)P.D - 1);                // a group behind the last one repeats a channel and stores nothing
    const int8_t *w[kFewD], *x[R];
#pragma unroll
    for (int c = 0; c < kFewD; ++c) w[c] = P.w + (int64_t)min(d0 + c, P.D - 1) * P.ldw;
#pragma unroll
    for (int r = 0; r < R; ++r) x[r] = P.x + (int64_t)min(r, P.rows - 1) * P.ldx;
    // the sum this lane finishes
    const int my_d = (int)min(group * kFewD + lane / R, (int64_t)0x7fffffff), my_r = lane % R;
    const bool mine = me == 0 && lane < kSums && my_d < P.D && my_r < P.rows;
    const float ws = mine ? P.ws[my_d] : 0.f, xs = mine ? P.xs[my_r] : 0.f, bias = mine && P.bias ? P.bias[my_d] : 0.f;
    int acc[kFewD][R] = {};
    if constexpr (WHOLE) {
        const int whole = P.K & ~15;
        constexpr int kAhead = R <= 2 ? 4 : 2;                                   // pieces in flight
        for (int k = (me * 32 + lane) * 16; k < whole; k += kAhead * share * 512) {
            int4 a[kAhead][kFewD];
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
#pragma unroll
                for (int c = 0; c < kFewD; ++c) a[i][c] = k + i * share * 512 < whole ? load_weights(w[c] + k + i * share * 512) : make_int4(0, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const int4 b = k + i * share * 512 < whole ? *reinterpret_cast<const int4 *>(x[r] + k + i * share * 512) : make_int4(0, 0, 0, 0);
#pragma unroll
                    for (int c = 0; c < kFewD; ++c) acc[c][r] = dot16(a[i][c], b, acc[c][r]);
                }
        }
        if (me == 0 && lane < P.K - whole) {                                     // the last columns, one by one
#pragma unroll
            for (int c = 0; c < kFewD; ++c)
#pragma unroll
                for (int r = 0; r < R; ++r) acc[c][r] += (int)w[c][whole + lane] * (int)x[r][whole + lane];
        }
    } else {
        constexpr int kAhead = R <= 2 ? 8 : 4;
        Bytes wb[kFewD], xb[R];
#pragma unroll
        for (int c = 0; c < kFewD; ++c) wb[c] = Bytes(w[c], P.K);
#pragma unroll
        for (int r = 0; r < R; ++r) xb[r] = Bytes(x[r], P.K);
        for (int k0 = (me * 32 + lane) * 4; k0 < P.K; k0 += kAhead * share * 128) {
            uint2 a[kAhead][kFewD];
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
#pragma unroll
                for (int c = 0; c < kFewD; ++c) a[i][c] = wb[c].load(k0 + i * share * 128);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int k = k0 + i * share * 128;
                int v[kFewD];
#pragma unroll
                for (int c = 0; c < kFewD; ++c) v[c] = wb[c].join(a[i][c]);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const int u = first4(xb[r].join(xb[r].load(k)), P.K - k);
#pragma unroll
                    for (int c = 0; c < kFewD; ++c) acc[c][r] = __dp4a(v[c], u, acc[c][r]);
                }
            }
        }
    }
    int sum = 0;
#pragma unroll
    for (int c = 0; c < kFewD; ++c)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int v = __reduce_add_sync(0xffffffffu, acc[c][r]);
            if (lane == c * R + r) sum = v;
        }
    if (share > 1) {
        if (lane < kSums) part[warp][lane] = sum;
        __syncthreads();
        if (mine)
            for (int o = 1; o < share; ++o) sum += part[warp + o][lane];
    }
    if (mine) store8((Y *)P.y + (int64_t)my_r * P.ldy + my_d, finish8(sum, ws, xs, bias, P.floor));
}

template <typename Y, bool WHOLE>
cudaError_t launch_few(const P8Params &P, unsigned blocks, int share, cudaStream_t st)
{
    auto kernel = P.rows == 1 ? p8_few_kernel<Y, 1, WHOLE> : P.rows == 2 ? p8_few_kernel<Y, 2, WHOLE> : P.rows <= 4 ? p8_few_kernel<Y, 4, WHOLE> : p8_few_kernel<Y, 8, WHOLE>;
    return launch_overlapped(kernel, dim3(blocks), 256u, 0, st, P, share);
}
gdws_status_t p8_few(const P8Params &P, int share, cudaStream_t st)
{
    const int64_t groups = ((int64_t)P.D + kFewD - 1) / kFewD;
    const unsigned blocks = (unsigned)((groups * share + 7) / 8);
    const bool whole = whole16(P.x, P.rows, P.ldx) && whole16(P.w, P.D, P.ldw);
    const cudaError_t e = P.out_f32 ? (whole ? launch_few<float, true>(P, blocks, share, st) : launch_few<float, false>(P, blocks, share, st))
                                    : (whole ? launch_few<__nv_bfloat16, true>(P, blocks, share, st) : launch_few<__nv_bfloat16, false>(P, blocks, share, st));
    return launched(e, "p8_few_kernel launch");
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
constexpr int kP8Stages = 32;        // at most
constexpr int kP8Loaders = 4;
constexpr int kPiece = 128;          // bytes of a row in a stage

struct alignas(64) P8TcParams {
    CUtensorMap tw, tx;
    const float *xs, *ws, *bias;
    void *y;
    int64_t ldy;
    float floor;
    int rows, D;
    int pieces;                      // of 128 columns
    int nt, tiles_r, split, ns, stage_bytes, recv, per_shift;      // slices
    int tiles_d, nitems, band, pitch;             // pairs; pitch: bytes between rows of y
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
template <int V> struct IntVec;
template <> struct IntVec<2> { typedef int2 type; };
template <> struct IntVec<4> { typedef int4 type; };

// Adds up a cluster's sums of a tile and stores them.  A block's share are 2^per_shift columns; what it receives lies there as
// [block of the cluster][channel][column], a channel's columns padded by 16 bytes so that 32 channels' vectors meet no bank twice.
template <int V, typename Y>
__device__ __forceinline__ void sum_slices(const P8TcParams &P, const uint8_t *base, uint32_t s_s, uint32_t t_base, int rank, int row, Y *y, int live, float ws, float bias, const float *xs)
{
    const int per = 1 << P.per_shift, pitch = per + 4, half = threadIdx.x >> 7;
    for (int c = half * 8; c < P.nt; c += 16) {
        uint32_t acc[8];
        tmem_ld8(t_base + (uint32_t)c, acc);
        tmem_ld_wait();
#pragma unroll
        for (int e = 0; e < 8; e += V) {
            const int owner = (c + e) >> P.per_shift, col = (c + e) & (per - 1);
            const uint32_t to = map_shared(s_s + (uint32_t)(P.recv + ((rank * 128 + row) * pitch + col) * 4), (uint32_t)owner);
            if constexpr (V == 4) asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(acc[e]), "r"(acc[e + 1]), "r"(acc[e + 2]), "r"(acc[e + 3]) : "memory");
            else asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(to), "r"(acc[e]), "r"(acc[e + 1]) : "memory");
        }
    }
    cluster_sync();
    const int *recv = reinterpret_cast<const int *>(base + P.recv) + row * pitch;
    for (int c = half * V; live > 0 && c < per; c += 2 * V) {
        int sum[V] = {};
#pragma unroll 4
        for (int o = 0; o < P.split; ++o) {
            union { typename IntVec<V>::type v; int e[V]; } got;
            got.v = *reinterpret_cast<const typename IntVec<V>::type *>(recv + o * 128 * pitch + c);
#pragma unroll
            for (int e = 0; e < V; ++e) sum[e] += got.e[e];
        }
        const int at = rank * per + c;
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (at + e < live) store8(y + (at + e) * P.ldy, finish8(sum[e], ws, xs[at + e], bias, P.floor));
    }
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
    const uint32_t s_s = smem_u32(base);
    const uint32_t bar_full = smem_u32(&bars[0]), bar_empty = bar_full + 8 * kP8Stages, bar_done = bar_empty + 8 * kP8Stages;
    volatile int *const vabort = &abort_flag;
    const int rank = P.split > 1 ? (int)cluster_rank() : 0, tile = (int)blockIdx.x / P.split;
    const int tile_d = tile / P.tiles_r, d0 = tile_d * 128, r0 = (tile - tile_d * P.tiles_r) * P.nt;
    const int p0 = P.pieces * rank / P.split, n = P.pieces * (rank + 1) / P.split - p0;
    const uint32_t cols = (uint32_t)max(P.nt, 32);

    if (tid == 0) abort_flag = 0;
    if (tid < 2 * kP8Stages + 1) {
        mbar_init(bar_full + 8 * tid, 1);
        fence_mbar_init();
    }
    __syncwarp();
    if (warp == 0 && lane == 0) { prefetch_tensor_map(&P.tw); prefetch_tensor_map(&P.tx); }
    if (warp == 2) {
        tmem_alloc(smem_u32(&tmem_slot), cols);
        grid_launch_dependents();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (P.split > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");      // this block runs: its memory may be written
    grid_dependency_wait();
    const uint32_t tmem = tmem_slot;
    const int row = tid & 127, d = d0 + row;      // this lane's channel
    const float ws = d < P.D ? P.ws[d] : 0.f, bias = d < P.D && P.bias ? P.bias[d] : 0.f;

    if (warp >= 4) {
        // Four threads ask for every fourth piece each (a copy costs its thread some 200 cycles).  ns is a multiple of four
        // where stages are used again, so that a stage is always the same thread's.
        if (lane == 0) {
            int i = warp - 4;
            for (uint32_t s = (uint32_t)i, par = 1; i < n; i += kP8Loaders) {
                if (i >= P.ns) mbar_wait_call(bar_empty + 8 * s, par, &abort_flag, &g_rows_status, kStatusWaitStage);
                if (*vabort) break;
                const uint32_t dst = s_s + s * (uint32_t)P.stage_bytes;
                mbar_expect_tx(bar_full + 8 * s, (uint32_t)P.stage_bytes);
                tma_load_2d(dst, &P.tw, (p0 + i) * kPiece, d0, bar_full + 8 * s);
                tma_load_2d(dst + 16384u, &P.tx, (p0 + i) * kPiece, r0, bar_full + 8 * s);
                s += kP8Loaders;
                if (s >= (uint32_t)P.ns) { s -= (uint32_t)P.ns; par ^= 1; }
            }
            // no copy into this block's memory may be in flight when it ends: the last one into each of this thread's stages
            for (int j = i - kP8Loaders; j >= 0 && j >= i - kP8Loaders + 1 - P.ns; j -= kP8Loaders) mbar_wait_drain(bar_full + 8 * (j % P.ns), (uint32_t)(j / P.ns) & 1u);
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
    } else if (warp == 0) {
        for (int c = lane; c < P.nt; c += 32) xs_s[c] = r0 + c < P.rows ? P.xs[r0 + c] : 0.f;
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
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (P.per_shift >= 2) sum_slices<4>(P, base, s_s, t_base, rank, row, y, live, ws, bias, xs_s);
        else sum_slices<2>(P, base, s_s, t_base, rank, row, y, live, ws, bias, xs_s);
    }
    tc_fence_before();
    __syncthreads();
    __syncwarp();
    if (warp == 2) tmem_dealloc(tmem, cols);
}

// Many outputs: pairs of blocks (cta_group::2) compute 256 channels x 256 rows, each block's tensor memory holding its 128
// channels; persistent, two accumulators, so that a tile's epilogue passes under the next one's products.  A pair fetches 64 KB
// for 256 x 256 x 128 products, each block half of either operand.  4096 x 4096 -> 4096: 51 us, 2690 Tera-operations/s (71 % of the
// tensor pipe's cycles); 8192 x 4096 -> 8192 180 us in short runs, 216 under sustained load, where the power limit lowers the clocks.
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
    __shared__ __align__(16) float xs_s[2][256];
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
    if (warp == 0 && lane == 0) { prefetch_tensor_map(&P.tw); prefetch_tensor_map(&P.tx); }
    if (warp == 2) {
        tmem_alloc_pair(smem_u32(&tmem_slot), 512);
        grid_launch_dependents();
    }
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
                    const uint32_t a = s_s + s * (uint32_t)kPairStage, b = a + 16384u;
#pragma unroll
                    for (int k = 0; k < 4; ++k) umma8_pair(acc, make_sdesc(a + 32 * k, 16, 1024), make_sdesc(b + 32 * k, 16, 1024), idesc, (uint32_t)(p | k));
                    umma_commit_pair(bar_empty + 8 * s);
                    if (++s == (uint32_t)kPairStages) { s = 0; par ^= 1; }
                }
                umma_commit_pair(bar_accfull + 8 * buf);
            }
            umma_commit_pair(bar_drain);
        }
        __syncwarp();
    } else if (warp >= 4) {
        // A warp has a quarter of the channels and half of the rows of a tile.  The rows' scales lie in shared memory, twice; the next
        // tile's are fetched under this one.
        const int et = tid - 128, ln = et & 127, c0 = (et >> 7) * 128;
        const uint32_t free0 = map_shared(bar_accfree, 0), floor2 = pack_bf16x2(P.floor, P.floor);
        P8Tile t = pair_tile(P, pair);
        float xs = 0.f, ws = 0.f, bias = 0.f;
        auto scales = [&]() {
            const int r = t.r0 + et, d = t.d0 + (int)rank * 128 + ln;
            xs = r < P.rows ? P.xs[r] : 0.f;
            ws = d < P.D ? P.ws[d] : 0.f;
            bias = d < P.D && P.bias ? P.bias[d] : 0.f;
        };
        scales();
#pragma unroll 1
        for (int it = 0; it < my_items; ++it) {
            const int buf = it & 1;
            xs_s[buf][et] = xs;
            const uint64_t ws2 = pair_of(ws, ws), bias2 = pair_of(bias, bias);
            const int r = t.r0 + c0, d = t.d0 + (int)rank * 128 + ln;
            const int columns = min(128, P.rows - r), live = d < P.D ? columns : 0;      // of the tile, and those that this lane stores
            const float my_ws = ws, my_bias = bias;
            char *const y = (char *)P.y + ((int64_t)r * P.ldy + d) * (int64_t)sizeof(Y);
            if (it + 1 < my_items) {
                t = pair_tile(P, pair + (it + 1) * npairs);
                scales();
            }
            named_bar_sync(1, 256);
            if (lane == 0) mbar_wait_relaxed_call<4096>(bar_accfull + 8 * buf, (uint32_t)(it >> 1) & 1u, &abort_flag, &g_rows_status, kStatusWaitMma);
            __syncwarp();
            tc_fence_after();
            const uint32_t t_base = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)(buf * 256 + c0);
#pragma unroll 1
            for (int c = 0; c < columns; c += 32) {
                uint32_t acc[32];
                tmem_ld32(t_base + (uint32_t)c, acc);
                tmem_ld_wait();
                // all before the first store: the compiler cannot know that y is not this memory, and would load one after the other
                float2 x[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) x[e] = reinterpret_cast<const float2 *>(&xs_s[buf][c0 + c])[e];
                char *const at = y + (int64_t)c * P.pitch;
                // no condition between the rows of a whole block: 32 independent chains
                if (c + 32 <= live) {
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        float lo, hi;
                        finish8x2(acc[e], acc[e + 1], ws2, pair_of(x[e / 2].x, x[e / 2].y), bias2, lo, hi);
                        char *const to = at + (int64_t)e * P.pitch, *const to2 = at + (int64_t)(e + 1) * P.pitch;
                        if constexpr (sizeof(Y) == 2) {
                            const uint32_t o = round_bf16x2(lo, hi, floor2);
                            *reinterpret_cast<uint16_t *>(to) = (uint16_t)o;
                            *reinterpret_cast<uint16_t *>(to2) = (uint16_t)(o >> 16);
                        } else {
                            *reinterpret_cast<float *>(to) = max_nan(lo, P.floor);
                            *reinterpret_cast<float *>(to2) = max_nan(hi, P.floor);
                        }
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        if (c + e < live) store8(reinterpret_cast<Y *>(at + (int64_t)e * P.pitch), finish8((int)acc[e], my_ws, e & 1 ? x[e / 2].y : x[e / 2].x, my_bias, P.floor));
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_relaxed(free0 + 8 * buf);
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
    const cuuint64_t strides[1] = {(cuuint64_t)((ld + 15) / 16 * 16)};      // of a single row any multiple will do
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
    int kernel = GDWS_KERNEL8_ANY;
    int nt = 0, split = 1;       // slices: rows of a tile, blocks of a cluster; few rows: warps that share a group's columns (split)
};

// Shared memory of the slices: bytes of a stage, of what a block receives, and the number of stages.
int slices_stage(int nt) { return 16384 + nt * kPiece; }
int slices_recv(const P8Choice &c) { return c.split > 1 ? (c.nt + 4 * c.split) * 512 : 0; }
int slices_stages(const P8Choice &c, int pieces)
{
    const int mine = (pieces + c.split - 1) / c.split, most = std::min(kP8Stages, (kMaxSmem - 1024 - slices_recv(c)) / slices_stage(c.nt));
    return mine <= most ? mine : most / kP8Loaders * kP8Loaders;
}

// Estimated times in us, of calls on data in L2, fitted by hand to timings of 40 sizes with each kernel on a B200 (most within 15 %;
// they decide between kernels, nothing else rests on them).
//
// Few rows: reading w at what the dot products of so many rows leave of it, and the sums across a warp.
double few_us(const P8Params &P)
{
    const double rate = P.rows == 1 ? 8.8e6 : P.rows == 2 ? 6.4e6 : P.rows <= 4 ? 5.2e6 : 4.1e6;
    return 2.0 + std::max((double)P.D * P.K / rate, 1.2e-4 * P.D) + 1.8e-5 * P.D * P.rows;
}
// Slices: per wave of blocks 2 us, the epilogue's columns and the pieces, each bound by reading its 128 rows of w and nt of x from
// shared memory (0.25 us for nt = 16, 0.34 for 128); blocks that share an SM share that.  A cluster's sum costs its exchange.
double slices_us(const P8Choice &c, const P8Params &P, int sms, const int *clusters)
{
    const int pieces = (P.K + kPiece - 1) / kPiece, mine = (pieces + c.split - 1) / c.split;
    const double tiles = (double)(((int64_t)P.D + 127) / 128) * (double)(((int64_t)P.rows + c.nt - 1) / c.nt);
    const double piece = 0.237 + 0.0008 * c.nt;
    double waves, together = 1, sum = 0;
    if (c.split > 1) {
        if (!clusters[c.split]) return 1e9;
        waves = ceil(tiles / clusters[c.split]);
        const int steps = c.split == 2 ? 1 : c.split == 4 ? 2 : 3;
        sum = steps * (0.3 + 0.013 * c.nt);
    } else {
        const int room = std::min(3, kMaxSmem / (1024 + slices_stages(c, pieces) * slices_stage(c.nt)));       // blocks on an SM
        waves = ceil(tiles / ((double)sms * room));
        together = std::min((double)room, ceil(tiles / sms));
    }
    return 1.0 + waves * (2.0 + 0.012 * c.nt + mine * piece * together + sum);
}
// Pairs: per tile 0.33 us a piece.
double pairs_us(const P8Params &P, int sms)
{
    const double tiles = (double)(((int64_t)P.D + 255) / 256) * (double)(((int64_t)P.rows + 255) / 256);
    return 5.0 + ceil(tiles / (sms / 2)) * (((P.K + kPiece - 1) / kPiece) * 0.33 + 0.7);
}

P8Choice p8_choose(const P8Params &P, int sms, const int *clusters)
{
    P8Choice best;
    const bool whole = whole16(P.x, P.rows, P.ldx) && whole16(P.w, P.D, P.ldw);
    const int pieces = (P.K + kPiece - 1) / kPiece;
    double us = 1e9;
    // (the pairs' kernel keeps the distance of y's rows in 32 bits)
    if (whole && P.ldy < 0x1fffffff) { best.kernel = GDWS_KERNEL8_PAIRS; us = pairs_us(P, sms); }
    if (P.rows <= kFewRows && few_us(P) < us) {
        us = few_us(P);
        best.kernel = GDWS_KERNEL8_FEW;
        // As many warps to a group of channels as it takes to fill the chip.  Eight rows' sums leave room for 16 warps on an SM: no more
        // than that, and two to a group (5 x 919 -> 6251 4.3 us with one, 6.3 with two; 7 x 1064 -> 4609 6.0 | 4.3).
        const int64_t groups = ((int64_t)P.D + kFewD - 1) / kFewD;
        if (P.rows <= 4) while (best.split < 8 && groups * best.split < 16 * sms && best.split * 512 < P.K) best.split *= 2;
        else if (groups * 2 <= 16 * sms && P.K > 512) best.split = 2;
    }
    if (!whole) return best;
    for (int nt = 16; nt <= 128; nt *= 2) {
        for (int split = 1; split <= std::min(8, pieces); split *= 2) {
            P8Choice c;
            c.kernel = GDWS_KERNEL8_SLICES; c.nt = nt; c.split = split;
            const double t = slices_us(c, P, sms, clusters);
            if (t < us) { us = t; best = c; }
        }
        if (nt >= P.rows) break;
    }
    return best;
}

gdws_status_t p8_tc(const P8Params &A, const P8Choice &c, int device, int sms, cudaStream_t st)
{
    P8TcParams P;
    const bool pairs = c.kernel == GDWS_KERNEL8_PAIRS;
    gdws_status_t rc = rows_map(&P.tw, A.w, A.D, A.K, A.ldw, 128, device);
    if (rc == GDWS_OK) rc = rows_map(&P.tx, A.x, A.rows, A.K, A.ldx, pairs ? 128 : c.nt, device);
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
        P.nitems = (int)items; P.band = 8; P.pitch = (int)(A.ldy * (A.out_f32 ? 4 : 2));
        const unsigned grid = 2u * (unsigned)std::min<int64_t>(items, sms / 2);
        e = launch_overlapped(A.out_f32 ? p8_pairs_kernel<float> : p8_pairs_kernel<__nv_bfloat16>, dim3(grid), (unsigned)kPairThreads, kPairSmem, st, P);
    } else {
        P.nt = c.nt; P.split = c.split; P.tiles_r = (int)(((int64_t)A.rows + c.nt - 1) / c.nt);
        const int64_t blocks = ((int64_t)A.D + 127) / 128 * P.tiles_r * c.split;
        if (blocks > 0x7fffffff) return fail(GDWS_ERR_UNSUPPORTED, "gdws_pointwise8: %d x %d outputs are more than one launch covers", A.rows, A.D);
        P.stage_bytes = slices_stage(c.nt);
        const int recv = slices_recv(c);
        P.ns = slices_stages(c, P.pieces);
        P.recv = P.ns * P.stage_bytes;
        P.per_shift = 0;
        while (c.split << P.per_shift < c.nt) ++P.per_shift;
        // Blocks of a cluster that wait for each other hold tensor memory meanwhile.  Two such kernels on one SM could each hold what
        // a block of the other's clusters waits for, so they take more than half of the shared memory: one block per SM.  (Blocks that
        // wait for nobody may share an SM with any kernel: see grid_launch_dependents on what the order of allocations has to be.)
        const size_t need = 1024 + (size_t)P.recv + recv;
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

cudaError_t rows_status_word(int **word) { return cudaGetSymbolAddress((void **)word, g_rows_status); }

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
    int clusters[kMostSlices + 1];
    cluster_capacities(device, sms, clusters);
    const P8Choice c = p8_choose(P, sms, clusters);
    if (c.kernel == GDWS_KERNEL8_FEW) return p8_few(P, c.split, (cudaStream_t)stream);
    return c.kernel == GDWS_KERNEL8_ANY ? p8_any(P, (cudaStream_t)stream) : p8_tc(P, c, device, sms, (cudaStream_t)stream);
}

gdws_status_t gdws_pointwise8_kernel(const gdws_rows8_t *x, const gdws_rows8_t *w, const gdws_rows_t *y, int *kernel)
{
    const gdws_status_t st = check_pointwise8(x, w, nullptr, y);
    if (st != GDWS_OK) return st;
    if (!kernel) return fail(GDWS_ERR_INVALID_ARG, "gdws_pointwise8_kernel: kernel is NULL");
    int device, sms, clusters[kMostSlices + 1];
    if (rows_device(&device, &sms) == GDWS_OK) {
        cluster_capacities(device, sms, clusters);
    } else {                     // no such device: as for a B200
        cudaGetLastError();
        sms = kB200Sms;
        std::copy(kB200Clusters, kB200Clusters + kMostSlices + 1, clusters);
    }
    *kernel = x->rows ? p8_choose(p8_params(x, w, nullptr, 0, y), sms, clusters).kernel : GDWS_KERNEL8_NONE;
    return GDWS_OK;
}

gdws_status_t gdws_rows_status(void)
{
    int device, sms;
    const gdws_status_t st = rows_device(&device, &sms);
    if (st != GDWS_OK) return st;
    int word = 0, *at = nullptr;
    cudaError_t e = cudaDeviceSynchronize();
    if (e == cudaSuccess) e = rows_status_word(&at);
    if (e == cudaSuccess) e = cudaMemcpy(&word, at, sizeof(int), cudaMemcpyDeviceToHost);
    if (e == cudaSuccess && word) e = cudaMemset(at, 0, sizeof(int));
    if (e != cudaSuccess) return cuda_fail(e, "status read");
    if (word) return fail(GDWS_ERR_DEVICE_TIMEOUT, "a bounded wait inside a kernel expired (status word 0x%x)", word);
    return GDWS_OK;
}

}  // extern "C"
