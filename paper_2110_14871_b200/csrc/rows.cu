// Rows in 8 bits: residual addition, root-mean-square norm, quantization and back; argument checks of the calls on rows.
#include <cuda_bf16.h>
#include <math.h>

#include <atomic>

#include "rows.cuh"

namespace gdws {

// ------------------------------------------------------------------------------------------
// Argument checks
// ------------------------------------------------------------------------------------------
namespace {

constexpr int kDevices = 64;
std::atomic<int> g_sms[kDevices];

struct Extent {            // bytes of a matrix: rows of `width`, `pitch` apart
    uintptr_t at;
    int64_t rows, width, pitch;
    uintptr_t end() const { return at + (uintptr_t)((rows - 1) * pitch + width); }
};

bool meet(const Extent &a, const Extent &b)
{
    if (a.at >= b.end() || b.at >= a.end()) return false;
    if (a.pitch == b.pitch && a.rows > 1 && b.rows > 1) {           // columns of one buffer
        const int64_t d = (int64_t)((b.at > a.at ? b.at - a.at : a.pitch - (int64_t)((a.at - b.at) % (uintptr_t)a.pitch)) % (uintptr_t)a.pitch);
        return d < a.width || d + b.width > a.pitch;
    }
    return true;
}

Extent extent(const gdws_rows_t *m)
{
    const int64_t e = (int64_t)dtype_size(m->dtype), width = m->cols * e;
    return {(uintptr_t)m->ptr, m->rows, width, m->rows > 1 ? m->ld * e : width};
}
Extent extent(const gdws_rows8_t *m) { return {(uintptr_t)m->q, m->rows, m->cols, m->rows > 1 ? m->ld : m->cols}; }
Extent scales(const gdws_rows8_t *m) { return {(uintptr_t)m->scale, 1, m->rows * 4, m->rows * 4}; }
Extent vector_of(const void *p, int64_t bytes) { return {(uintptr_t)p, 1, bytes, bytes}; }

gdws_status_t check_shape(const char *call, const char *name, int64_t rows, int64_t cols, int64_t ld)
{
    if (rows < 0 || rows > 0x7fffffff) return fail(GDWS_ERR_INVALID_ARG, "%s: %s->rows=%lld is outside 0..2^31-1", call, name, (long long)rows);
    if (cols < 1) return fail(GDWS_ERR_INVALID_ARG, "%s: %s->cols must be >= 1 (got %lld)", call, name, (long long)cols);
    if (rows > 1 && (ld < cols || ld > ((int64_t)1 << 40) / 4)) return fail(GDWS_ERR_INVALID_ARG, "%s: %s->ld=%lld does not fit rows of %lld", call, name, (long long)ld, (long long)cols);
    return GDWS_OK;
}

}  // namespace

gdws_status_t check_rows(const char *call, const char *name, const gdws_rows_t *m)
{
    if (!m) return fail(GDWS_ERR_INVALID_ARG, "%s: %s is NULL", call, name);
    if (m->dtype != GDWS_F32 && m->dtype != GDWS_BF16) return fail(GDWS_ERR_INVALID_ARG, "%s: %s: bad dtype", call, name);
    const gdws_status_t st = check_shape(call, name, m->rows, m->cols, m->ld);
    if (st != GDWS_OK) return st;
    if (m->rows && (!m->ptr || (uintptr_t)m->ptr % dtype_size(m->dtype)))
        return fail(GDWS_ERR_INVALID_ARG, "%s: %s->ptr is NULL or not aligned to its type", call, name);
    return GDWS_OK;
}

gdws_status_t check_rows8(const char *call, const char *name, const gdws_rows8_t *m)
{
    if (!m) return fail(GDWS_ERR_INVALID_ARG, "%s: %s is NULL", call, name);
    const gdws_status_t st = check_shape(call, name, m->rows, m->cols, m->ld);
    if (st != GDWS_OK) return st;
    if (m->rows && (!m->q || !m->scale || (uintptr_t)m->scale & 3))
        return fail(GDWS_ERR_INVALID_ARG, "%s: %s->q or %s->scale is NULL, or the scales are not 4-byte aligned", call, name, name);
    return GDWS_OK;
}

gdws_status_t rows_device(int *device, int *sms)
{
    cudaError_t e = cudaGetDevice(device);
    if (e != cudaSuccess) return cuda_fail(e, "cudaGetDevice");
    if (*device < 0 || *device >= kDevices) return fail(GDWS_ERR_UNSUPPORTED, "device index %d is outside 0..%d", *device, kDevices - 1);
    *sms = g_sms[*device].load(std::memory_order_acquire);
    if (*sms > 0) return GDWS_OK;
    const gdws_status_t st = check_arch();
    if (st != GDWS_OK) return st;
    e = cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, *device);
    if (e != cudaSuccess) return cuda_fail(e, "cudaDeviceGetAttribute(MultiProcessorCount)");
    g_sms[*device].store(*sms, std::memory_order_release);
    return GDWS_OK;
}

gdws_status_t check_pointwise8(const gdws_rows8_t *x, const gdws_rows8_t *w, const float *bias, const gdws_rows_t *y)
{
    const char *call = "gdws_pointwise8";
    gdws_status_t st = check_rows8(call, "x", x);
    if (st == GDWS_OK) st = check_rows8(call, "w", w);
    if (st == GDWS_OK) st = check_rows(call, "y", y);
    if (st != GDWS_OK) return st;
    if (w->rows < 1) return fail(GDWS_ERR_INVALID_ARG, "%s: w has no rows", call);
    if (x->cols != w->cols) return fail(GDWS_ERR_INVALID_ARG, "%s: rows of x have %d columns, those of w %d", call, x->cols, w->cols);
    if (y->rows != x->rows || y->cols != w->rows)
        return fail(GDWS_ERR_INVALID_ARG, "%s: y is %lld x %d but the product is %lld x %lld", call, (long long)y->rows, y->cols, (long long)x->rows, (long long)w->rows);
    if ((uintptr_t)bias & 3) return fail(GDWS_ERR_INVALID_ARG, "%s: bias is not 4-byte aligned", call);
    if (x->cols > kMost8) return fail(GDWS_ERR_UNSUPPORTED, "%s: sums of more than %d products may pass 32 bits", call, kMost8);
    if (!x->rows) return GDWS_OK;
    const Extent o = extent(y);
    if (meet(o, extent(x)) || meet(o, scales(x)) || meet(o, extent(w)) || meet(o, scales(w)) || (bias && meet(o, vector_of(bias, 4 * w->rows))))
        return fail(GDWS_ERR_INVALID_ARG, "%s: y overlaps an input", call);
    return GDWS_OK;
}

namespace {

// ------------------------------------------------------------------------------------------
// Rows to 8 bits
// ------------------------------------------------------------------------------------------
struct RowsParams {
    const void *x, *residual, *weight;
    void *total;
    int8_t *q;
    float *scale;
    int64_t ldx, ldr, ldt, ldq;
    float eps;
    int rows, cols;
    bool weight_f32;
};

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void from_float(float v, float &o) { o = v; }
__device__ __forceinline__ void from_float(float v, __nv_bfloat16 &o) { o = __float2bfloat16_rn(v); }

// VEC consecutive values (VEC > 1: as 16-byte pieces where all of them exist; zeros from `cols` on).
template <int VEC, typename T>
__device__ __forceinline__ void load_vec(const T *row, int c, int cols, float (&v)[VEC])
{
    if constexpr (VEC == 1) {
        v[0] = c < cols ? to_float(row[c]) : 0.f;
    } else {
        if (c + VEC <= cols) {
            union { uint4 w[VEC * sizeof(T) / 16]; T e[VEC]; } b;
#pragma unroll
            for (int i = 0; i < (int)(VEC * sizeof(T) / 16); ++i) b.w[i] = reinterpret_cast<const uint4 *>(row + c)[i];
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[e] = to_float(b.e[e]);
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[e] = c + e < cols ? to_float(row[c + e]) : 0.f;
        }
    }
}
template <int VEC, typename T>
__device__ __forceinline__ void store_vec(T *row, int c, int cols, const float (&v)[VEC])
{
    if constexpr (VEC == 1) {
        if (c < cols) from_float(v[0], row[c]);
    } else {
        if (c + VEC <= cols) {
            union { uint4 w[VEC * sizeof(T) / 16]; T e[VEC]; } b;
#pragma unroll
            for (int e = 0; e < VEC; ++e) from_float(v[e], b.e[e]);
#pragma unroll
            for (int i = 0; i < (int)(VEC * sizeof(T) / 16); ++i) reinterpret_cast<uint4 *>(row + c)[i] = b.w[i];
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (c + e < cols) from_float(v[e], row[c + e]);
        }
    }
}

// What a row's elements are divided by.  m: max |u| (finite).  Magnitudes below 2^-60 are lifted by 2^64, which is exact, so that
// 127 / m stays in range.
struct Steps {
    float lift, m, inv;
    __device__ __forceinline__ explicit Steps(float most)
    {
        lift = most < 0x1p-60f ? 0x1p64f : 1.f;
        m = most * lift;
        inv = m > 0.f ? 127.f / m : 0.f;
    }
};
// 127 u / m rounded to the nearest integer.  u * inv is off by at most 127 * 2^-23 = 1.5e-5 from the quotient: where it lies that
// close to the middle of two integers (one element of 16000 at random), the exact comparison of 254 |u| with (2 j + 1) m decides;
// both are products of a 24-bit and an 8-bit number, exact in fp64.  kMagic brings the integer into the low mantissa bits.
constexpr float kMagic = 12582912.f, kNear = 0.5f - 3e-5f;
template <int VEC>
__device__ __forceinline__ void quantize_vec(const float (&u)[VEC], const Steps &s, int (&q)[VEC])
{
    float t[VEC], far = 0.f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
        t[e] = u[e] * s.lift * s.inv;
        const float r = t[e] + kMagic;
        q[e] = __float_as_int(r);
        far = fmaxf(far, fabsf(t[e] - (r - kMagic)));
    }
    if (far > kNear) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const float r = t[e] + kMagic;
            if (fabsf(t[e] - (r - kMagic)) > kNear) {
                const int j = (int)fabsf(t[e]);
                const double a = 254.0 * (double)fabsf(u[e] * s.lift), b = (double)(2 * j + 1) * (double)s.m;
                const int n = a > b || (a == b && (j & 1)) ? j + 1 : j;
                q[e] = t[e] < 0.f ? -n : n;
            }
        }
    }
}
template <int VEC>
__device__ __forceinline__ void store_steps(int8_t *row, int c, int cols, const int (&q)[VEC])
{
    if constexpr (VEC == 8) {
        if (c + 8 <= cols) {
            uint2 w;
            w.x = __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
            w.y = __byte_perm(__byte_perm(q[4], q[5], 0x0040), __byte_perm(q[6], q[7], 0x0040), 0x5410);
            *reinterpret_cast<uint2 *>(row + c) = w;
            return;
        }
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e)
        if (c + e < cols) row[c + e] = (int8_t)q[e];
}

// Largest magnitude (as bits: infinity and NaN compare above every finite value) and sum of squares over the TPR threads of a row.
template <int TPR, bool NORM>
__device__ __forceinline__ void reduce_row(uint32_t &most, float &squares)
{
    most = __reduce_max_sync(0xffffffffu, most);
    if (NORM) {
#pragma unroll
        for (int o = 16; o; o >>= 1) squares += __shfl_xor_sync(0xffffffffu, squares, o);
    }
    if constexpr (TPR > 32) {
        constexpr int kWarps = TPR / 32;
        __shared__ uint32_t most_of[kWarps];
        __shared__ float squares_of[kWarps];
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        if (lane == 0) { most_of[warp] = most; squares_of[warp] = squares; }
        __syncthreads();
        most = __reduce_max_sync(0xffffffffu, most_of[lane & (kWarps - 1)]);
        if (NORM) {
            squares = squares_of[lane & (kWarps - 1)];
#pragma unroll
            for (int o = kWarps / 2; o; o >>= 1) squares += __shfl_xor_sync(0xffffffffu, squares, o);
        }
    }
}

// A row's scale from its largest |u| and its sum of squares; false: the row is not finite.
template <bool NORM>
__device__ __forceinline__ bool row_scale(uint32_t most, float squares, const RowsParams &P, float *scale)
{
    const bool fine = most < 0x7f800000u && (!NORM || squares < INFINITY);
    *scale = __uint_as_float(most) / 127.f;
    if (NORM) *scale /= sqrtf(squares / (float)P.cols + P.eps);
    if (!fine) *scale = __uint_as_float(0x7fffffffu);
    return fine;
}

template <bool NORM, int VEC, typename T>
__device__ __forceinline__ void load_sum(const RowsParams &P, int64_t r, int c, float (&h)[VEC], float (&u)[VEC])
{
    load_vec<VEC>((const T *)P.x + r * P.ldx, c, P.cols, h);
    if (NORM && P.residual) {
        float a[VEC];
        load_vec<VEC>((const T *)P.residual + r * P.ldr, c, P.cols, a);
#pragma unroll
        for (int e = 0; e < VEC; ++e) h[e] += a[e];
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) u[e] = h[e];
    if (NORM && P.weight) {
        float a[VEC];
        if (P.weight_f32) load_vec<VEC>((const float *)P.weight, c, P.cols, a);
        else load_vec<VEC>((const __nv_bfloat16 *)P.weight, c, P.cols, a);
#pragma unroll
        for (int e = 0; e < VEC; ++e) u[e] *= a[e];
    }
}

// One pass: TPR threads hold a row in registers, N values each, in vectors of VEC.
template <typename T, int VEC, int N, int TPR, bool NORM>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) rows8_kernel(const __grid_constant__ RowsParams P)
{
    grid_launch_dependents();
    grid_dependency_wait();
    const int64_t r = TPR < 256 ? (int64_t)blockIdx.x * (256 / TPR) + threadIdx.x / TPR : blockIdx.x;
    if (r >= P.rows) return;
    const int t = threadIdx.x % TPR;
    float u[N / VEC][VEC];
    uint32_t most = 0;
    float squares = 0.f;
#pragma unroll
    for (int i = 0; i < N / VEC; ++i) {
        const int c = (t + i * TPR) * VEC;
        float h[VEC];
        if (c < P.cols) {
            load_sum<NORM, VEC, T>(P, r, c, h, u[i]);
            if (NORM && P.total) store_vec<VEC>((T *)P.total + r * P.ldt, c, P.cols, h);
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) h[e] = u[i][e] = 0.f;
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            most = max(most, __float_as_uint(u[i][e]) & 0x7fffffffu);
            if (NORM) squares = fmaf(h[e], h[e], squares);
        }
    }
    reduce_row<TPR, NORM>(most, squares);
    float scale;
    const bool fine = row_scale<NORM>(most, squares, P, &scale);
    if (t == 0) P.scale[r] = scale;
    const Steps s(fine ? __uint_as_float(most) : 0.f);
#pragma unroll
    for (int i = 0; i < N / VEC; ++i) {
        const int c = (t + i * TPR) * VEC;
        if (c >= P.cols) break;
        int q[VEC];
        if (!fine) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) u[i][e] = 0.f;
        }
        quantize_vec<VEC>(u[i], s, q);
        store_steps<VEC>(P.q + r * P.ldq, c, P.cols, q);
    }
}

// Rows of any length: a block reads its row twice.  `total` is written in the second pass, by the thread that reads the element,
// so that it may be the residual's or x's own memory.
template <typename T, bool NORM>
__global__ void __launch_bounds__(1024) rows8_long_kernel(const __grid_constant__ RowsParams P)
{
    grid_launch_dependents();
    grid_dependency_wait();
    const int64_t r = blockIdx.x;
    uint32_t most = 0;
    float squares = 0.f;
    for (int c = threadIdx.x; c < P.cols; c += 1024) {
        float h[1], u[1];
        load_sum<NORM, 1, T>(P, r, c, h, u);
        most = max(most, __float_as_uint(u[0]) & 0x7fffffffu);
        if (NORM) squares = fmaf(h[0], h[0], squares);
    }
    reduce_row<1024, NORM>(most, squares);
    float scale;
    const bool fine = row_scale<NORM>(most, squares, P, &scale);
    if (threadIdx.x == 0) P.scale[r] = scale;
    const Steps s(fine ? __uint_as_float(most) : 0.f);
    for (int c = threadIdx.x; c < P.cols; c += 1024) {
        float h[1], u[1];
        int q[1];
        load_sum<NORM, 1, T>(P, r, c, h, u);
        if (NORM && P.total) store_vec<1>((T *)P.total + r * P.ldt, c, P.cols, h);
        if (!fine) u[0] = 0.f;
        quantize_vec<1>(u, s, q);
        store_steps<1>(P.q + r * P.ldq, c, P.cols, q);
    }
}

template <typename T, int VEC, int N, int TPR, bool NORM>
cudaError_t launch_rows(const RowsParams &P, cudaStream_t st)
{
    constexpr int per = TPR < 256 ? 256 / TPR : 1;
    return launch_overlapped(rows8_kernel<T, VEC, N, TPR, NORM>, dim3((unsigned)((P.rows + per - 1) / per)), TPR < 256 ? 256u : (unsigned)TPR, 0, st, P);
}
template <typename T, int VEC, bool NORM>
cudaError_t launch_rows(const RowsParams &P, cudaStream_t st)
{
    if (P.cols <= 256) return launch_rows<T, VEC, 8, 32, NORM>(P, st);
    if (P.cols <= 512) return launch_rows<T, VEC, 16, 32, NORM>(P, st);
    if (P.cols <= 2048) return launch_rows<T, VEC, 8, 256, NORM>(P, st);
    if (P.cols <= 4096) return launch_rows<T, VEC, 16, 256, NORM>(P, st);
    if (P.cols <= 8192) return launch_rows<T, VEC, 8, 1024, NORM>(P, st);
    if (P.cols <= 16384) return launch_rows<T, VEC, 16, 1024, NORM>(P, st);
    if (P.cols <= 32768) return launch_rows<T, VEC, 32, 1024, NORM>(P, st);
    return launch_overlapped(rows8_long_kernel<T, NORM>, dim3((unsigned)P.rows), 1024u, 0, st, P);
}
template <bool NORM>
cudaError_t launch_rows(const RowsParams &P, bool f32, cudaStream_t st)
{
    // 16-byte pieces of the inputs and 8-byte ones of q where every row starts on such a boundary
    const int64_t unit = f32 ? 4 : 8;
    auto whole = [&](const void *p, int64_t ld) { return !((uintptr_t)p & 15) && (P.rows == 1 || ld % unit == 0); };
    const bool vec = whole(P.x, P.ldx) && (!P.residual || whole(P.residual, P.ldr)) && (!P.total || whole(P.total, P.ldt)) && !((uintptr_t)P.weight & 15) &&
                     !((uintptr_t)P.q & 7) && (P.rows == 1 || P.ldq % 8 == 0);
    if (f32) return vec ? launch_rows<float, 8, NORM>(P, st) : launch_rows<float, 1, NORM>(P, st);
    return vec ? launch_rows<__nv_bfloat16, 8, NORM>(P, st) : launch_rows<__nv_bfloat16, 1, NORM>(P, st);
}

// ------------------------------------------------------------------------------------------
// 8 bits back to values
// ------------------------------------------------------------------------------------------
struct ValuesParams {
    const int8_t *q;
    const float *scale;
    void *y;
    int64_t ldq, ldy;
    int rows, cols;
};

// blockDim: x along a row, y rows.
template <typename T, int VEC>
__global__ void __launch_bounds__(256) values_kernel(const __grid_constant__ ValuesParams P)
{
    grid_launch_dependents();
    grid_dependency_wait();
    const int64_t r = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    if (r >= P.rows) return;
    const float s = P.scale[r];
    const int8_t *q = P.q + r * P.ldq;
    T *y = (T *)P.y + r * P.ldy;
    for (int c = threadIdx.x * VEC; c < P.cols; c += blockDim.x * VEC) {
        float v[VEC];
        if (VEC == 8 && c + 8 <= P.cols) {
            union { uint2 w; int8_t e[8]; } b;
            b.w = *reinterpret_cast<const uint2 *>(q + c);
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[e] = (float)b.e[e] * s;
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[e] = c + e < P.cols ? (float)q[c + e] * s : 0.f;
        }
        store_vec<VEC>(y, c, P.cols, v);
    }
}

template <typename T>
cudaError_t launch_values(const ValuesParams &P, cudaStream_t st)
{
    const bool vec = !((uintptr_t)P.q & 7) && !((uintptr_t)P.y & 15) && (P.rows == 1 || (P.ldq % 8 == 0 && P.ldy % (16 / (int64_t)sizeof(T)) == 0));
    const int64_t n = vec ? (P.cols + 7) / 8 : P.cols;
    unsigned tx = 1;
    while (tx < 256 && tx < n) tx *= 2;
    const unsigned ty = 256 / tx;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(((unsigned)P.rows + ty - 1) / ty); cfg.blockDim = dim3(tx, ty); cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = 1;
    return vec ? cudaLaunchKernelEx(&cfg, values_kernel<T, 8>, P) : cudaLaunchKernelEx(&cfg, values_kernel<T, 1>, P);
}

gdws_status_t same_shape(const char *call, const char *name, int64_t rows, int cols, const gdws_rows8_t *q)
{
    if (rows != q->rows || cols != q->cols)
        return fail(GDWS_ERR_INVALID_ARG, "%s: %s is %lld x %d but q is %lld x %d", call, name, (long long)rows, cols, (long long)q->rows, q->cols);
    return GDWS_OK;
}

RowsParams params_of(const gdws_rows_t *x, const gdws_rows8_t *q)
{
    RowsParams P = {};
    P.x = x->ptr; P.ldx = x->ld; P.q = q->q; P.ldq = q->ld; P.scale = q->scale;
    P.rows = (int)x->rows; P.cols = x->cols;
    return P;
}

}  // namespace
}  // namespace gdws

using namespace gdws;

extern "C" {

gdws_status_t gdws_quantize_rows(const gdws_rows_t *x, const gdws_rows8_t *q, void *stream)
{
    const char *call = "gdws_quantize_rows";
    gdws_status_t st = check_rows(call, "x", x);
    if (st == GDWS_OK) st = check_rows8(call, "q", q);
    if (st == GDWS_OK) st = same_shape(call, "x", x->rows, x->cols, q);
    if (st != GDWS_OK) return st;
    if (!x->rows) return GDWS_OK;
    if (meet(extent(q), extent(x)) || meet(scales(q), extent(x)) || meet(scales(q), extent(q))) return fail(GDWS_ERR_INVALID_ARG, "%s: q or its scales overlap x or each other", call);
    int device, sms;
    st = rows_device(&device, &sms);
    if (st != GDWS_OK) return st;
    const cudaError_t e = launch_rows<false>(params_of(x, q), x->dtype == GDWS_F32, (cudaStream_t)stream);
    return launched(e, "rows8_kernel launch");
}

gdws_status_t gdws_norm_quantize_rows(const gdws_rows_t *x, const gdws_rows_t *residual, const gdws_rows_t *total, const void *weight,
                                      gdws_dtype_t weight_dtype, float eps, const gdws_rows8_t *q, void *stream)
{
    const char *call = "gdws_norm_quantize_rows";
    gdws_status_t st = check_rows(call, "x", x);
    if (st == GDWS_OK && residual) st = check_rows(call, "residual", residual);
    if (st == GDWS_OK && total) st = check_rows(call, "total", total);
    if (st == GDWS_OK) st = check_rows8(call, "q", q);
    if (st == GDWS_OK) st = same_shape(call, "x", x->rows, x->cols, q);
    if (st == GDWS_OK && residual) st = same_shape(call, "residual", residual->rows, residual->cols, q);
    if (st == GDWS_OK && total) st = same_shape(call, "total", total->rows, total->cols, q);
    if (st != GDWS_OK) return st;
    if ((residual && residual->dtype != x->dtype) || (total && total->dtype != x->dtype)) return fail(GDWS_ERR_INVALID_ARG, "%s: residual and total have x's type", call);
    if (weight && weight_dtype != GDWS_F32 && weight_dtype != GDWS_BF16) return fail(GDWS_ERR_INVALID_ARG, "%s: weight: bad dtype", call);
    if (weight && (uintptr_t)weight % dtype_size(weight_dtype)) return fail(GDWS_ERR_INVALID_ARG, "%s: weight is not aligned to its type", call);
    if (!(eps >= 0x1p-126f) || !(eps < INFINITY)) return fail(GDWS_ERR_INVALID_ARG, "%s: eps must be finite and at least 2^-126", call);
    if (!x->rows) return GDWS_OK;
    const int64_t wbytes = weight ? x->cols * (int64_t)dtype_size(weight_dtype) : 0;
    const Extent inputs[3] = {extent(x), residual ? extent(residual) : extent(x), weight ? vector_of(weight, wbytes) : extent(x)};
    for (const Extent &in : inputs)
        if (meet(extent(q), in) || meet(scales(q), in)) return fail(GDWS_ERR_INVALID_ARG, "%s: q or its scales overlap an input", call);
    if (meet(scales(q), extent(q))) return fail(GDWS_ERR_INVALID_ARG, "%s: q and its scales overlap", call);
    if (total) {
        const Extent o = extent(total);
        auto same = [&](const Extent &in) { return in.at == o.at && in.pitch == o.pitch; };
        if ((!same(inputs[0]) && meet(o, inputs[0])) || (!same(inputs[1]) && meet(o, inputs[1])) || (weight && meet(o, inputs[2])) || meet(o, extent(q)) || meet(o, scales(q)))
            return fail(GDWS_ERR_INVALID_ARG, "%s: total overlaps q, the weight, or x or the residual without being the same rows", call);
    }
    int device, sms;
    st = rows_device(&device, &sms);
    if (st != GDWS_OK) return st;
    RowsParams P = params_of(x, q);
    P.eps = eps; P.weight = weight; P.weight_f32 = weight_dtype == GDWS_F32;
    if (residual) { P.residual = residual->ptr; P.ldr = residual->ld; }
    if (total) { P.total = total->ptr; P.ldt = total->ld; }
    const cudaError_t e = launch_rows<true>(P, x->dtype == GDWS_F32, (cudaStream_t)stream);
    return launched(e, "rows8_kernel launch");
}

gdws_status_t gdws_dequantize_rows(const gdws_rows8_t *q, const gdws_rows_t *y, void *stream)
{
    const char *call = "gdws_dequantize_rows";
    gdws_status_t st = check_rows8(call, "q", q);
    if (st == GDWS_OK) st = check_rows(call, "y", y);
    if (st == GDWS_OK) st = same_shape(call, "y", y->rows, y->cols, q);
    if (st != GDWS_OK) return st;
    if (!q->rows) return GDWS_OK;
    if (meet(extent(y), extent(q)) || meet(extent(y), scales(q))) return fail(GDWS_ERR_INVALID_ARG, "%s: y overlaps q or its scales", call);
    int device, sms;
    st = rows_device(&device, &sms);
    if (st != GDWS_OK) return st;
    ValuesParams P = {q->q, q->scale, y->ptr, q->ld, y->ld, (int)q->rows, q->cols};
    const cudaError_t e = y->dtype == GDWS_F32 ? launch_values<float>(P, (cudaStream_t)stream) : launch_values<__nv_bfloat16>(P, (cudaStream_t)stream);
    return launched(e, "values_kernel launch");
}

}  // extern "C"
