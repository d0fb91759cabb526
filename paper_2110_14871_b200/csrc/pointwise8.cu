// The pointwise product on rows in 8 bits: y[r,d] = (sum_c x[r,c] w[d,c]) * ws[d] * xs[r] + bias[d].
#include "rows.cuh"

namespace gdws {
namespace {

__device__ int g_rows_status;        // status word of the calls on rows, one per device

// fp32 in the order that the interface names; NaN stays NaN.
__device__ __forceinline__ float finish8(int sum, float ws, float xs, float bias, int relu)
{
    const float v = fmaf((float)sum * ws, xs, bias);
    return relu && v < 0.f ? 0.f : v;
}
__device__ __forceinline__ void store8(void *y, bool f32, int64_t at, float v)
{
    if (f32) ((float *)y)[at] = v;
    else ((__nv_bfloat16 *)y)[at] = __float2bfloat16_rn(v);
}

struct P8Params {
    const int8_t *x, *w;
    const float *xs, *ws, *bias;
    void *y;
    int64_t ldx, ldw, ldy;
    int rows, K, D, relu;
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
            if (r < P.rows) store8(P.y, P.out_f32, (int64_t)r * P.ldy + d, finish8(acc[i][j], ws, P.xs[r], bias, P.relu));
        }
    }
}

gdws_status_t p8_alu(const P8Params &P, cudaStream_t st)
{
    const int64_t tiles_d = ((int64_t)P.D + 63) / 64, tiles = ((int64_t)P.rows + 63) / 64 * tiles_d;
    if (tiles > 0x7fffffff) return fail(GDWS_ERR_UNSUPPORTED, "gdws_pointwise8: %d x %d outputs are more than one launch covers", P.rows, P.D);
    const cudaError_t e = launch_overlapped(p8_alu_kernel, dim3((unsigned)tiles), 256u, 0, st, P, (int)tiles_d);
    return e == cudaSuccess ? GDWS_OK : cuda_fail(e, "p8_alu_kernel launch");
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
    P8Params P;
    P.x = x->q; P.w = w->q; P.xs = x->scale; P.ws = w->scale; P.bias = bias; P.y = y->ptr;
    P.ldx = x->rows > 1 ? x->ld : x->cols; P.ldw = w->rows > 1 ? w->ld : w->cols; P.ldy = y->rows > 1 ? y->ld : y->cols;
    P.rows = (int)x->rows; P.K = x->cols; P.D = (int)w->rows; P.relu = relu != 0; P.out_f32 = y->dtype == GDWS_F32;
    return p8_alu(P, (cudaStream_t)stream);
}

gdws_status_t gdws_pointwise8_kernel(const gdws_rows8_t *x, const gdws_rows8_t *w, const gdws_rows_t *y, int *kernel)
{
    const gdws_status_t st = check_pointwise8(x, w, nullptr, y);
    if (st != GDWS_OK) return st;
    if (!kernel) return fail(GDWS_ERR_INVALID_ARG, "gdws_pointwise8_kernel: kernel is NULL");
    *kernel = GDWS_KERNEL8_ALU;
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
