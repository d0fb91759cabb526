// Rows in 8 bits: residual addition, root-mean-square norm, quantization and back; argument checks of the calls on rows.
#include <cuda_bf16.h>
#include <math.h>

#include <atomic>
#include <type_traits>

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
    if (rows < 0 || rows > kMostRows) return fail(GDWS_ERR_INVALID_ARG, "%s: %s->rows=%lld is outside 0..2^31-1024", call, name, (long long)rows);
    if (cols < 1 || cols > kMostCols) return fail(GDWS_ERR_INVALID_ARG, "%s: %s->cols=%lld is outside 1..2^30", call, name, (long long)cols);
    if (rows > 1 && (ld < cols || ld > ((int64_t)1 << 40) / 4)) return fail(GDWS_ERR_INVALID_ARG, "%s: %s->ld=%lld does not fit rows of %lld", call, name, (long long)ld, (long long)cols);
    // so that the bytes of a matrix fit 64 bits, whatever its type: overlaps are looked for by address
    if (rows > 1 && rows - 1 > ((int64_t)1 << 56) / ld) return fail(GDWS_ERR_INVALID_ARG, "%s: %s spans more than 2^56 elements", call, name);
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
    bool weight_f32, weight_whole;      // weight_whole: on a boundary of 16 bytes
};

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void from_float(float v, float &o) { o = v; }
__device__ __forceinline__ void from_float(float v, __nv_bfloat16 &o) { o = __float2bfloat16_rn(v); }

// Two fp32 operations in one instruction; each rounds as the single one.
__device__ __forceinline__ void mul2(float &a, float &b, float x, float y)
{
    asm("{\n\t.reg .b64 p, q;\n\tmov.b64 p, {%0, %1};\n\tmov.b64 q, {%2, %3};\n\tmul.rn.f32x2 p, p, q;\n\tmov.b64 {%0, %1}, p;\n\t}" : "+f"(a), "+f"(b) : "f"(x), "f"(y));
}
__device__ __forceinline__ void add2(float &a, float &b, float x, float y)
{
    asm("{\n\t.reg .b64 p, q;\n\tmov.b64 p, {%0, %1};\n\tmov.b64 q, {%2, %3};\n\tadd.rn.f32x2 p, p, q;\n\tmov.b64 {%0, %1}, p;\n\t}" : "+f"(a), "+f"(b) : "f"(x), "f"(y));
}
__device__ __forceinline__ void square2(float &a, float &b, float x, float y)      // a += x^2, b += y^2
{
    asm("{\n\t.reg .b64 p, q;\n\tmov.b64 p, {%0, %1};\n\tmov.b64 q, {%2, %3};\n\tfma.rn.f32x2 p, q, q, p;\n\tmov.b64 {%0, %1}, p;\n\t}" : "+f"(a), "+f"(b) : "f"(x), "f"(y));
}
// The larger of a and |b|; a NaN stays.
__device__ __forceinline__ float larger(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(fabsf(b)));
    return r;
}

// VEC consecutive values as they lie in memory (VEC > 1: 16-byte pieces where all of them exist; zeros from `cols` on).
template <int VEC, typename T>
union Raw {
    uint4 w[VEC == 1 ? 1 : VEC * sizeof(T) / 16];
    T e[VEC];
    __device__ __forceinline__ Raw() {}
};
// c may be negative.  whole: all of them exist and lie on a boundary of 16 bytes.  Others are taken one by one, or, where they are
// known to lie on such a boundary (ALIGNED), as every piece that holds a value of the row, and what else it holds is set to zero.
// (1000 x 10001, quantization: 21 us one by one, 13.5 by pieces.  Norms of rows on boundaries, whose only such vector is the last, were
// slower by pieces: 8192 x 4096, in an earlier form, 46 -> 60 us, whatever the order of the conditions.)
template <int VEC, bool ALIGNED, typename T>
__device__ __forceinline__ void load_raw(const T *row, int c, int cols, bool whole, Raw<VEC, T> &b)
{
    if constexpr (VEC == 1) {
        from_float(0.f, b.e[0]);
        if (c < cols) b.e[0] = row[c];
    } else {
        constexpr int kPieces = (int)(VEC * sizeof(T) / 16), kPer = 16 / (int)sizeof(T);
#pragma unroll
        for (int i = 0; i < kPieces; ++i) b.w[i] = make_uint4(0, 0, 0, 0);
        if (whole) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) b.w[i] = reinterpret_cast<const uint4 *>(row + c)[i];
        } else if constexpr (ALIGNED) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
                if (c + kPer * (i + 1) > 0 && c + kPer * i < cols) b.w[i] = reinterpret_cast<const uint4 *>(row + c)[i];
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if ((unsigned)(c + e) >= (unsigned)cols) from_float(0.f, b.e[e]);
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if ((unsigned)(c + e) < (unsigned)cols) b.e[e] = row[c + e];
        }
    }
}
template <int VEC, typename T>
__device__ __forceinline__ void store_vec(T *row, int c, int cols, bool whole, const float (&v)[VEC])
{
    if constexpr (VEC == 1) {
        if (c < cols) from_float(v[0], row[c]);
    } else {
        Raw<VEC, T> b;
#pragma unroll
        for (int e = 0; e < VEC; ++e) from_float(v[e], b.e[e]);
        if (whole) {
#pragma unroll
            for (int i = 0; i < (int)(VEC * sizeof(T) / 16); ++i) reinterpret_cast<uint4 *>(row + c)[i] = b.w[i];
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if ((unsigned)(c + e) < (unsigned)cols) row[c + e] = b.e[e];
        }
    }
}

// 127 u / m rounded to the nearest integer, m = max |u|.  t = u * inv (inv = 127 / m, rounded) is off by at most 127 * 2^-23 = 1.5e-5
// from the quotient; kMagic brings its integer r into the low mantissa bits.  Where t lies that close to the middle between r and
// its neighbour (one fp32 number of 16000 at random; bf16 numbers often lie on it), the sign of 254 u - (2 r +- 1) m decides.  It is
// exact: 254 u is taken in two terms, and what is left of the difference has a few bits.  (All times 2^-8, so that nothing overflows.)
constexpr float kMagic = 12582912.f, kNear = 0.5f - 3e-5f;
// m as the divisions take it, and what u is multiplied with before: magnitudes below 2^-60 are lifted by 2^64, which is exact, so
// that 127 / m stays in range.
__device__ __forceinline__ float lifted(float &m)
{
    const float lift = m < 0x1p-60f ? 0x1p64f : 1.f;
    m *= lift;
    return lift;
}
// The integer in r = t + kMagic or its neighbour towards t; d = t - (r - kMagic), some half.  (q comes from the very r that d comes
// from: the compiler may form u * inv + kMagic in one rounding in one place and in two in another.)
__device__ __forceinline__ int exact_step(float u, float m, float r, float d)
{
    const int q = __float_as_int(r);
    const float s = copysignf(1.f, d), k = fmaf(2.f, r - kMagic, s) * 0x1p-8f;
    const float a = u * (254.f / 256.f), a2 = fmaf(u, 254.f / 256.f, -a);
    const float past = (fmaf(-k, m, a) + a2) * s;          // how far the quotient lies beyond the middle
    return past > 0.f || (past == 0.f && (q & 1)) ? q + (int)s : q;
}
template <int N>
__device__ __forceinline__ void quantize(const float (&u)[N], float m, float inv, int (&q)[N])
{
    float t[N], far = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) t[e] = u[e];
    if constexpr (N % 2 == 0) {
#pragma unroll
        for (int e = 0; e < N; e += 2) {
            mul2(t[e], t[e + 1], inv, inv);
            float r0 = t[e], r1 = t[e + 1], d0 = t[e], d1 = t[e + 1];
            add2(r0, r1, kMagic, kMagic);
            q[e] = __float_as_int(r0);
            q[e + 1] = __float_as_int(r1);
            add2(r0, r1, -kMagic, -kMagic);
            add2(d0, d1, -r0, -r1);
            far = fmaxf(fmaxf(far, fabsf(d0)), fabsf(d1));
        }
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            t[e] *= inv;
            const float r = t[e] + kMagic;
            q[e] = __float_as_int(r);
            far = fmaxf(far, fabsf(t[e] - (r - kMagic)));
        }
    }
    if (far > kNear) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float r = t[e] + kMagic, d = t[e] - (r - kMagic);
            if (fabsf(d) > kNear) q[e] = exact_step(u[e], m, r, d);
        }
    }
}
// The same for bf16 numbers u and m, where a third of the warps would have an element to decide about.  With 8-bit significands the
// quotient lies exactly in the middle or at least 1 / (254 * 255) = 1.5e-5 of itself away from it.  t is off by 1.2e-7 of itself, so
// rounding it to 17 bits (2^-18, by Veltkamp's splitting: c = (2^7 + 1) t, c - (c - t)) moves it onto the middle if it belongs
// there and not across it otherwise; the addition of kMagic then rounds as it should.
__device__ __forceinline__ void quantize_short(const float (&u)[8], float inv, int (&q)[8])
{
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        float t0 = u[e], t1 = u[e + 1];
        mul2(t0, t1, inv, inv);
        float c0 = t0, c1 = t1;
        mul2(c0, c1, 128.f, 128.f);          // exact, so that a fused multiply-add makes no difference
        add2(c0, c1, t0, t1);
        float d0 = c0, d1 = c1;
        add2(d0, d1, -t0, -t1);
        add2(c0, c1, -d0, -d1);
        add2(c0, c1, kMagic, kMagic);
        q[e] = __float_as_int(c0);
        q[e + 1] = __float_as_int(c1);
    }
}
template <int VEC>
__device__ __forceinline__ void store_steps(int8_t *row, int c, int cols, bool whole, const int *q)
{
    if constexpr (VEC == 8) {
        if (whole) {
            uint2 w;
            w.x = __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
            w.y = __byte_perm(__byte_perm(q[4], q[5], 0x0040), __byte_perm(q[6], q[7], 0x0040), 0x5410);
            *reinterpret_cast<uint2 *>(row + c) = w;
            return;
        }
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e)
        if ((unsigned)(c + e) < (unsigned)cols) row[c + e] = (int8_t)q[e];
}

// The same where q's vectors lie `by` bytes before its boundaries of 8 bytes: a lane stores the word that begins inside its
// vector, with the first bytes of the next lane's; what no such word covers goes byte by byte.  All lanes of a warp take part.
template <int TPR>
__device__ __forceinline__ void store_steps_across(int8_t *row, int c, int cols, int by, bool live, bool whole, const int (&q)[8])
{
    uint32_t lo = __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
    uint32_t hi = __byte_perm(__byte_perm(q[4], q[5], 0x0040), __byte_perm(q[6], q[7], 0x0040), 0x5410);
    const uint64_t mine = (uint64_t)hi << 32 | lo;
    const uint64_t next = (uint64_t)__shfl_down_sync(0xffffffffu, hi, 1) << 32 | __shfl_down_sync(0xffffffffu, lo, 1);
    if (!live) return;
    if (!by) return store_steps<8>(row, c, cols, whole, q);
    constexpr int kLanes = TPR < 32 ? TPR : 32;
    const int lane = threadIdx.x & (kLanes - 1);
    const bool word = lane != kLanes - 1 && c + by >= 0 && c + by + 8 <= cols;
    const bool before = lane != 0 && c - 8 + by >= 0 && c + by <= cols;         // the lane before stores this one's first bytes
    if (word) *reinterpret_cast<uint64_t *>(row + c + by) = mine >> (8 * by) | next << (64 - 8 * by);
    if (!word || !before) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if ((e < by ? !before : !word) && (unsigned)(c + e) < (unsigned)cols) row[c + e] = (int8_t)q[e];
    }
}

// Largest magnitude (as bits: infinity and NaN compare above every finite value) and sum of squares over the TPR threads of a row;
// all threads of a warp take part.
template <int TPR, bool NORM>
__device__ __forceinline__ void reduce_row(uint32_t &most, float &squares)
{
    constexpr int kLanes = TPR < 32 ? TPR : 32;
    if constexpr (kLanes == 32) {
        most = __reduce_max_sync(0xffffffffu, most);
    } else {
#pragma unroll
        for (int o = kLanes / 2; o; o >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
    }
    if (NORM) {
#pragma unroll
        for (int o = kLanes / 2; o; o >>= 1) squares += __shfl_xor_sync(0xffffffffu, squares, o);
    }
    if constexpr (TPR > 32) {
        constexpr int kWarps = TPR / 32, kAll = TPR < 128 ? 4 : kWarps;      // of a row, of the block
        __shared__ uint32_t most_of[kAll];
        __shared__ float squares_of[kAll];
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        if (lane == 0) { most_of[warp] = most; squares_of[warp] = squares; }
        __syncthreads();
        const int from = (warp & ~(kWarps - 1)) + (lane & (kWarps - 1));
        most = __reduce_max_sync(0xffffffffu, most_of[from]);
        if (NORM) {
            squares = squares_of[from];
#pragma unroll
            for (int o = kWarps / 2; o; o >>= 1) squares += __shfl_xor_sync(0xffffffffu, squares, o);
        }
    }
}

template <bool NORM>
__device__ __forceinline__ bool finite_row(uint32_t most, float squares) { return most < 0x7f800000u && (!NORM || squares < INFINITY); }
template <bool NORM>
__device__ __forceinline__ float row_scale(uint32_t most, float squares, const RowsParams &P)
{
    float scale = __uint_as_float(most) / 127.f;
    if (NORM) scale /= sqrtf(squares / (float)P.cols + P.eps);
    return finite_row<NORM>(most, squares) ? scale : __uint_as_float(0x7fffffffu);
}

// VEC values of a row: x, what is added to it and what multiplies it, and from them h and u.
template <typename T, int VEC, bool SHIFTED, bool NORM>
struct Piece {
    Raw<VEC, T> x, residual;
    float weight[VEC];
    __device__ __forceinline__ void load(const RowsParams &P, int64_t r, int c, bool whole)
    {
        load_raw<VEC, !NORM || SHIFTED>((const T *)P.x + r * P.ldx, c, P.cols, whole, x);
        if (NORM && P.residual) load_raw<VEC, SHIFTED>((const T *)P.residual + r * P.ldr, c, P.cols, whole, residual);
    }
    // shift: how far before a multiple of VEC the row's vectors begin, the same for all threads of a row
    __device__ __forceinline__ void load_weight(const RowsParams &P, int c, bool whole, int shift)
    {
#pragma unroll
        for (int e = 0; e < VEC; ++e) weight[e] = 1.f;
        if (!NORM || !P.weight) return;
        if constexpr (VEC == 8) {
            // fp32 weights at an odd place: three aligned pieces, moved down by one and by two
            const int off = c & 3;
            if (shift && P.weight_f32 && P.weight_whole) {
                float w[12];
#pragma unroll
                for (int i = 0; i < 3; ++i) {
                    const int at = c - off + 4 * i;          // a piece that holds a weight of the row, or none
                    const float4 v = at + 4 > 0 && at < P.cols ? *reinterpret_cast<const float4 *>((const float *)P.weight + at) : make_float4(0.f, 0.f, 0.f, 0.f);
                    w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
                }
#pragma unroll
                for (int e = 0; e < 11; ++e) w[e] = off & 1 ? w[e + 1] : w[e];
#pragma unroll
                for (int e = 0; e < VEC; ++e) weight[e] = off & 2 ? w[e + 2] : w[e];
                // what the last piece holds behind the weight is not the caller's: zero times it may be NaN
                if (!whole) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e)
                        if ((unsigned)(c + e) >= (unsigned)P.cols) weight[e] = 0.f;
                }
                return;
            }
        }
        whole = whole && shift == 0 && P.weight_whole;
        if (P.weight_f32) {
            Raw<VEC, float> w;
            load_raw<VEC, false>((const float *)P.weight, c, P.cols, whole, w);
#pragma unroll
            for (int e = 0; e < VEC; ++e) weight[e] = w.e[e];
        } else {
            Raw<VEC, __nv_bfloat16> w;
            load_raw<VEC, false>((const __nv_bfloat16 *)P.weight, c, P.cols, whole, w);
#pragma unroll
            for (int e = 0; e < VEC; ++e) weight[e] = to_float(w.e[e]);
        }
    }
    // h and u of these values, h stored as total, the row's largest |u| and sum of squares
    __device__ __forceinline__ void values(const RowsParams &P, int64_t r, int c, bool whole, bool store, float *u, float &most, float (&squares)[2]) const
    {
        float h[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) h[e] = to_float(x.e[e]);
        if (NORM && P.residual) {
            if constexpr (VEC == 1) h[0] += to_float(residual.e[0]);
            else
#pragma unroll
                for (int e = 0; e < VEC; e += 2) add2(h[e], h[e + 1], to_float(residual.e[e]), to_float(residual.e[e + 1]));
        }
        if (NORM && store) store_vec<VEC>((T *)P.total + r * P.ldt, c, P.cols, whole, h);
#pragma unroll
        for (int e = 0; e < VEC; ++e) u[e] = h[e];
        if (NORM) {
            if constexpr (VEC == 1) {
                u[0] *= weight[0];
                squares[0] = fmaf(h[0], h[0], squares[0]);
            } else {
#pragma unroll
                for (int e = 0; e < VEC; e += 2) {
                    mul2(u[e], u[e + 1], weight[e], weight[e + 1]);
                    square2(squares[0], squares[1], h[e], h[e + 1]);
                }
            }
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) most = larger(most, u[e]);
    }
};

// One pass: TPR threads hold a row in registers, N values each, in vectors of VEC.  Everything is asked for before the first store:
// total may be x's or the residual's memory for all that the compiler knows.  SHIFTED: rows start anywhere (contiguous rows of an odd
// length); the vectors are those of the memory, a row's first begins up to VEC - 1 values before it, and x, residual and total
// have to lie alike.
// Bound by reading and writing for long rows (8192 x 4096 bf16: norm 41 us, 5.7 TB/s; quantization 17 us, 5.9 TB/s); short ones by what a
// row costs each of its threads.
template <typename T, int VEC, bool SHIFTED, int N, int TPR, bool NORM>
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR) rows8_kernel(const __grid_constant__ RowsParams P)
{
    constexpr int kPer = TPR < 128 ? 128 / TPR : 1, kPieces = N / VEC;
    grid_launch_dependents();
    grid_dependency_wait();
    int64_t r = (int64_t)blockIdx.x * kPer + threadIdx.x / TPR;
    const bool live = r < P.rows;                    // a group behind the last row goes through that one again and stores nothing
    if (!live) r = P.rows - 1;
    const int t = threadIdx.x % TPR;
    int8_t *const qrow = P.q + r * P.ldq;
    const int shift = SHIFTED ? (int)((uintptr_t)((const T *)P.x + r * P.ldx) % 16 / sizeof(T)) : 0;
    const int by = SHIFTED ? (int)((8 - ((uintptr_t)qrow - (uintptr_t)shift) % 8) % 8) : 0;      // from q's vectors to its next boundary of 8 bytes
    auto column = [&](int i) { return (t + i * TPR) * VEC - shift; };
    auto whole = [&](int c) { return VEC > 1 && (!SHIFTED || c >= 0) && c + VEC <= P.cols; };
    // bf16 values that nothing is added to stay as they are, two to a register: half of the registers, more rows at a time
    constexpr bool kPacked = !NORM && VEC == 8 && sizeof(T) == 2;
    float u[kPacked ? 1 : N], most = 0.f, squares[2] = {};
    Piece<T, VEC, SHIFTED, NORM> p[kPieces];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) p[i].load(P, r, column(i), whole(column(i)));
    if constexpr (kPacked) {
        uint32_t most2 = 0;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const uint32_t w[4] = {p[i].x.w[0].x, p[i].x.w[0].y, p[i].x.w[0].z, p[i].x.w[0].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(most2) : "r"(w[e] & 0x7fff7fffu));
        }
        most = larger(__uint_as_float(most2 << 16), __uint_as_float(most2 & 0xffff0000u));
    } else {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int c = column(i);
            p[i].load_weight(P, c, whole(c), shift);
            p[i].values(P, r, c, whole(c), live && P.total, u + i * VEC, most, squares);
        }
    }
    uint32_t top = __float_as_uint(most);
    squares[0] += squares[1];
    reduce_row<TPR, NORM>(top, squares[0]);
    if (t == 0 && live) P.scale[r] = row_scale<NORM>(top, squares[0], P);
    const bool fine = finite_row<NORM>(top, squares[0]);
    float m = fine ? __uint_as_float(top) : 0.f;
    const float lift = lifted(m), inv = m > 0.f ? 127.f / m : 0.f;
    const bool odd = lift != 1.f || !fine;
#pragma unroll
    for (int g = 0; g < N; g += 8) {
        float v[8];
        int q[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if constexpr (kPacked) v[e] = to_float(p[g / VEC].x.e[e]);
            else v[e] = u[g + e];
        }
        if (odd) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = fine ? v[e] * lift : 0.f;
        }
        if constexpr (kPacked) quantize_short(v, inv, q);
        else quantize<8>(v, m, inv, q);
        if constexpr (SHIFTED) {
            if (__any_sync(0xffffffffu, by != 0)) {          // a warp's rows may lie differently
                const int c = column(g / VEC);
                store_steps_across<TPR>(qrow, c, P.cols, by, live, whole(c), q);
                continue;
            }
        }
#pragma unroll
        for (int e = 0; e < 8; e += VEC) {
            const int c = column((g + e) / VEC);
            if (live) store_steps<VEC>(qrow, c, P.cols, whole(c), q + e);
        }
    }
}

// Rows of any length: a block reads its row twice.  `total` is written in the second pass, by the thread that reads the element,
// so that it may be the residual's or x's own memory.  A thread adds up as many as 2^20 squares, in 64 bits: in 32 equal ones
// come out 7e-5 off after 2^14 additions, 4e-3 after 2^20.
template <typename T, bool NORM>
__global__ void __launch_bounds__(1024) rows8_long_kernel(const __grid_constant__ RowsParams P)
{
    grid_launch_dependents();
    grid_dependency_wait();
    const int64_t r = blockIdx.x;
    float most = 0.f, squares[2];
    double sum = 0.0;
    for (int c = threadIdx.x; c < P.cols; c += 1024) {
        Piece<T, 1, false, NORM> p;
        float u[1];
        p.load(P, r, c, false);
        p.load_weight(P, c, false, 0);
        squares[0] = 0.f;
        p.values(P, r, c, false, false, u, most, squares);
        if (NORM) sum += (double)squares[0];
    }
    squares[0] = (float)sum;
    uint32_t top = __float_as_uint(most);
    reduce_row<1024, NORM>(top, squares[0]);
    if (threadIdx.x == 0) P.scale[r] = row_scale<NORM>(top, squares[0], P);
    const bool fine = finite_row<NORM>(top, squares[0]);
    float m = fine ? __uint_as_float(top) : 0.f;
    const float lift = lifted(m), inv = m > 0.f ? 127.f / m : 0.f;
    for (int c = threadIdx.x; c < P.cols; c += 1024) {
        Piece<T, 1, false, NORM> p;
        float u[1];
        int q[1];
        p.load(P, r, c, false);
        p.load_weight(P, c, false, 0);
        p.values(P, r, c, false, P.total != nullptr, u, most, squares);
        u[0] = fine ? u[0] * lift : 0.f;
        quantize<1>(u, m, inv, q);
        store_steps<1>(P.q + r * P.ldq, c, P.cols, false, q);
    }
}

template <typename T, int VEC, bool SHIFTED, int N, int TPR, bool NORM>
cudaError_t launch_rows(const RowsParams &P, cudaStream_t st)
{
    constexpr int per = TPR < 128 ? 128 / TPR : 1;
    return launch_overlapped(rows8_kernel<T, VEC, SHIFTED, N, TPR, NORM>, dim3((unsigned)(((int64_t)P.rows + per - 1) / per)), TPR < 128 ? 128u : (unsigned)TPR, 0, st, P);
}
// Values and threads for a row.  With many rows few threads with many values each: loads in flight, and what a row costs every
// thread (sums, divisions) spread over them (8192 x 4096 bf16, an earlier form of the norm: 128 threads 45.3 us, 256 47.3, 512 78).  With few rows, where
// the chip is not full anyway, more threads.
template <typename T, bool SHIFTED, bool NORM>
cudaError_t launch_rows(const RowsParams &P, bool few, cudaStream_t st)
{
    const int n = P.cols + (SHIFTED ? 7 : 0);
    if (few && n > 256) {
        if (n > 1024 && n <= 2048) return launch_rows<T, 8, SHIFTED, 8, 256, NORM>(P, st);
        if (n <= 1024) return launch_rows<T, 8, SHIFTED, 8, 128, NORM>(P, st);
        if (n <= 4096) return launch_rows<T, 8, SHIFTED, 8, 512, NORM>(P, st);
    }
    if (n <= 32) return launch_rows<T, 8, SHIFTED, 16, 2, NORM>(P, st);
    if (n <= 64) return launch_rows<T, 8, SHIFTED, 16, 4, NORM>(P, st);
    if (n <= 128) return launch_rows<T, 8, SHIFTED, 16, 8, NORM>(P, st);
    if (n <= 256) return launch_rows<T, 8, SHIFTED, 16, 16, NORM>(P, st);
    if (n <= 512) return launch_rows<T, 8, SHIFTED, 16, 32, NORM>(P, st);
    // (Norms below: contiguous rows, with residual, total and fp32 weight; without the rule -> with it.)
    if constexpr (NORM && SHIFTED) {       // more registers a value: fewer values where that is not half of the threads more (10000 x 801 bf16 36.2 -> 24.7 us, 4000 x 3001 48 -> 37.5)
        if (n > 768 && n <= 1024) return launch_rows<T, 8, SHIFTED, 16, 64, NORM>(P, st);
        if (n > 1536 && n <= 2048) return launch_rows<T, 8, SHIFTED, 16, 128, NORM>(P, st);
        if (n > 2048 && n <= 4096) return launch_rows<T, 8, SHIFTED, 16, 256, NORM>(P, st);
    }
    if (n <= 768) return launch_rows<T, 8, SHIFTED, 24, 32, NORM>(P, st);
    if (n <= 1024) return launch_rows<T, 8, SHIFTED, 32, 32, NORM>(P, st);
    if constexpr (!NORM && !SHIFTED && sizeof(T) == 2) {       // few registers: a warp to a row goes further (16384 x 1152 13.3 -> 11.9 us; with 48 values up to 1536 13.2 -> 13.1)
        if (n <= 1280) return launch_rows<T, 8, SHIFTED, 40, 32, NORM>(P, st);
    }
    if (n <= 1536) return launch_rows<T, 8, SHIFTED, 24, 64, NORM>(P, st);
    if (n <= 2048) return launch_rows<T, 8, SHIFTED, 32, 64, NORM>(P, st);
    if (n <= 4096) return launch_rows<T, 8, SHIFTED, 32, 128, NORM>(P, st);
    if constexpr (NORM && (SHIFTED || sizeof(T) == 4)) {       // more registers a value: fewer values (4000 x 7999 bf16 131 -> 82 us, 2000 x 7000 fp32 42 -> 36)
        if (SHIFTED && n <= 6144) return launch_rows<T, 8, SHIFTED, 24, 256, NORM>(P, st);
        if (n <= 8192) return launch_rows<T, 8, SHIFTED, 16, 512, NORM>(P, st);
    }
    if (n <= 6144) return launch_rows<T, 8, SHIFTED, 24, 256, NORM>(P, st);
    if (n <= 8192) return launch_rows<T, 8, SHIFTED, 32, 256, NORM>(P, st);
    if (n <= 12288) return launch_rows<T, 8, SHIFTED, 24, 512, NORM>(P, st);
    if constexpr (NORM) {        // 32 values and what is added to them leave one block of 512 threads on an SM (2000 x 16000 bf16 63 -> 56 us)
        if (n <= 16384) return launch_rows<T, 8, SHIFTED, 16, 1024, NORM>(P, st);
    }
    if (n <= 16384) return launch_rows<T, 8, SHIFTED, 32, 512, NORM>(P, st);
    if (n <= 32768) return launch_rows<T, 8, SHIFTED, 32, 1024, NORM>(P, st);
    return launch_overlapped(rows8_long_kernel<T, NORM>, dim3((unsigned)P.rows), 1024u, 0, st, P);
}
// Rows that lie neither on boundaries of 16 bytes nor alike, and shifted ones of which the vectors cut off at either end are a large
// part (300000 x 30 bf16: 60 us by vectors): one value at a time.
template <typename T, bool NORM>
cudaError_t launch_single(const RowsParams &P, cudaStream_t st)
{
    if (P.cols <= 32) return launch_rows<T, 1, false, 8, 4, NORM>(P, st);
    if (P.cols <= 64) return launch_rows<T, 1, false, 8, 8, NORM>(P, st);
    if (P.cols <= 256) return launch_rows<T, 1, false, 8, 32, NORM>(P, st);
    if (P.cols <= 1024) return launch_rows<T, 1, false, 8, 128, NORM>(P, st);
    if (P.cols <= 4096) return launch_rows<T, 1, false, 8, 512, NORM>(P, st);
    if (P.cols <= 16384) return launch_rows<T, 1, false, 16, 1024, NORM>(P, st);
    return launch_overlapped(rows8_long_kernel<T, NORM>, dim3((unsigned)P.rows), 1024u, 0, st, P);
}
template <typename T, bool NORM>
cudaError_t launch_typed(const RowsParams &P, int sms, cudaStream_t st)
{
    const int64_t unit = 16 / sizeof(T);
    auto whole = [&](const void *p, int64_t ld) { return !p || (!((uintptr_t)p & 15) && (P.rows == 1 || ld % unit == 0)); };
    auto alike = [&](const void *p, int64_t ld) { return !p || ((uintptr_t)p % 16 == (uintptr_t)P.x % 16 && (P.rows == 1 || (ld - P.ldx) % unit == 0)); };
    const bool few = (int64_t)P.rows * P.cols <= (int64_t)8 * 2048 * sms;        // 8 values a thread do not fill the chip
    if (whole(P.x, P.ldx) && whole(P.residual, P.ldr) && whole(P.total, P.ldt) && !((uintptr_t)P.q & 7) && (P.rows == 1 || P.ldq % 8 == 0))
        return launch_rows<T, false, NORM>(P, few, st);
    return P.cols > 64 && alike(P.residual, P.ldr) && alike(P.total, P.ldt) ? launch_rows<T, true, NORM>(P, few, st) : launch_single<T, NORM>(P, st);
}
template <bool NORM>
cudaError_t launch_rows(const RowsParams &P, bool f32, int sms, cudaStream_t st)
{
    return f32 ? launch_typed<float, NORM>(P, sms, st) : launch_typed<__nv_bfloat16, NORM>(P, sms, st);
}

// ------------------------------------------------------------------------------------------
// 8 bits back to values
// ------------------------------------------------------------------------------------------
struct ValuesParams {
    const int8_t *q;
    const float *scale;
    void *y;
    int64_t ldq, ldy, pieces;        // pieces of VEC values in all
    int cols, per_row;               // pieces of a row
    uint32_t dv_row[2];              // divisions by per_row
};

// VEC 8-bit values (8 or 4) in a word.
template <int VEC>
struct Steps {
    typedef typename std::conditional<VEC == 8, uint64_t, uint32_t>::type word;
};
// Columns c to c + VEC - 1 of a row, zeros for those that it does not have.  ALIGNED: they lie on a boundary of VEC bytes.
template <int VEC, bool ALIGNED>
__device__ __forceinline__ typename Steps<VEC>::word load_steps(const int8_t *row, int c, int cols)
{
    typedef typename Steps<VEC>::word Word;
    const int off = ALIGNED ? 0 : (int)((uintptr_t)(row + c) % VEC);
    if ((ALIGNED || c >= 0) && c + VEC <= cols && off == 0) return *reinterpret_cast<const Word *>(row + c);
    if constexpr (!ALIGNED) {
        if (off && c >= off && c - off + 2 * VEC <= cols) {                   // two aligned words of the row
            const Word *a = reinterpret_cast<const Word *>(row + c - off);
            return a[0] >> (8 * off) | a[1] << (8 * (VEC - off));
        }
    }
    Word w = 0;
#pragma unroll
    for (int e = 0; e < VEC; ++e)
        if ((unsigned)(c + e) < (unsigned)cols) w |= (Word)(uint8_t)row[c + e] << (8 * e);
    return w;
}

// A block takes 256 * kAhead pieces in a row, whatever rows they belong to, and asks for all of them before it stores.  A piece is
// what a 16-byte store of y takes; SHIFTED: rows of y start anywhere, a row's first piece before it (as in rows8_kernel).
template <typename T, bool SHIFTED>
__global__ void __launch_bounds__(256) values_kernel(const __grid_constant__ ValuesParams P)
{
    constexpr int VEC = 16 / sizeof(T), kAhead = 4;
    grid_launch_dependents();
    grid_dependency_wait();
    const int64_t first = (int64_t)blockIdx.x * (256 * kAhead), row0 = first / P.per_row;
    const int in_row = (int)(first - row0 * P.per_row), here = (int)min(P.pieces - first, (int64_t)(256 * kAhead));
    typename Steps<VEC>::word q[kAhead];
    float s[kAhead];
    // the i-th piece of this thread: its row, and its first column; false: there is none
    auto piece = [&](int i, int64_t &row, int &c) {
        const int at = i * 256 + (int)threadIdx.x, dr = div_by(in_row + at, P.dv_row);
        row = row0 + dr;
        c = (in_row + at - dr * P.per_row) * VEC;
        if (SHIFTED) c -= (int)((uintptr_t)((T *)P.y + row * P.ldy) % 16 / sizeof(T));
        return at < here;
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
        int64_t row;
        int c;
        if (!piece(i, row, c)) break;
        s[i] = P.scale[row];
        q[i] = load_steps<VEC, !SHIFTED>(P.q + row * P.ldq, c, P.cols);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
        int64_t row;
        int c;
        if (!piece(i, row, c)) break;
        float v[VEC];
        // q + 128 in the low mantissa bits of 2^23: one byte permutation, and an exact subtraction for two values at a time
#pragma unroll
        for (int e = 0; e < VEC; e += 2) {
            const uint32_t w = (e < 4 ? (uint32_t)q[i] : (uint32_t)(q[i] >> (VEC == 8 ? 32 : 0))) ^ 0x80808080u;
            v[e] = __uint_as_float(__byte_perm(w, 0x4B000000u, 0x7550 + e % 4));
            v[e + 1] = __uint_as_float(__byte_perm(w, 0x4B000000u, 0x7551 + e % 4));
            add2(v[e], v[e + 1], -8388736.f, -8388736.f);
            mul2(v[e], v[e + 1], s[i], s[i]);
        }
        store_vec<VEC>((T *)P.y + row * P.ldy, c, P.cols, (!SHIFTED || c >= 0) && c + VEC <= P.cols, v);
    }
}

template <typename T>
cudaError_t launch_values(ValuesParams P, int64_t rows, cudaStream_t st)
{
    constexpr int kVec = 16 / sizeof(T);
    const bool whole = !((uintptr_t)P.q % kVec) && !((uintptr_t)P.y & 15) && (rows == 1 || (P.ldq % kVec == 0 && P.ldy % kVec == 0));
    P.per_row = (int)(((int64_t)P.cols + kVec - 1 + (whole ? 0 : kVec - 1)) / kVec);
    P.pieces = rows * P.per_row;
    div_magic(P.per_row, P.dv_row);
    const int64_t blocks = (P.pieces + 1023) / 1024;
    if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
    return launch_overlapped(whole ? values_kernel<T, false> : values_kernel<T, true>, dim3((unsigned)blocks), 256u, 0, st, P);
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
    const cudaError_t e = launch_rows<false>(params_of(x, q), x->dtype == GDWS_F32, sms, (cudaStream_t)stream);
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
    P.eps = eps; P.weight = weight; P.weight_f32 = weight_dtype == GDWS_F32; P.weight_whole = !((uintptr_t)weight & 15);
    if (residual) { P.residual = residual->ptr; P.ldr = residual->ld; }
    if (total) { P.total = total->ptr; P.ldt = total->ld; }
    const cudaError_t e = launch_rows<true>(P, x->dtype == GDWS_F32, sms, (cudaStream_t)stream);
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
    ValuesParams P = {};
    P.q = q->q; P.scale = q->scale; P.y = y->ptr; P.ldq = q->ld; P.ldy = y->ld; P.cols = q->cols;
    const cudaError_t e = y->dtype == GDWS_F32 ? launch_values<float>(P, q->rows, (cudaStream_t)stream) : launch_values<__nv_bfloat16>(P, q->rows, (cudaStream_t)stream);
    return launched(e, "values_kernel launch");
}

}  // extern "C"
