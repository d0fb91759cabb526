// Shared by the calls on rows (rows.cu, pointwise8.cu).
#pragma once

#include "sm100.cuh"

namespace gdws {

constexpr int kMostRows = 0x7fffffff - 1023, kMostCols = 1 << 30;      // so that 32-bit indexes may go a tile too far
constexpr int kMost8 = 131071;      // products of two 8-bit integers whose sum fits 32 bits: 131071 * 2^14 < 2^31

gdws_status_t check_rows(const char *call, const char *name, const gdws_rows_t *m);
gdws_status_t check_rows8(const char *call, const char *name, const gdws_rows8_t *m);
gdws_status_t check_pointwise8(const gdws_rows8_t *x, const gdws_rows8_t *w, const float *bias, const gdws_rows_t *y);
gdws_status_t rows_device(int *device, int *sms);       // the current device, checked to be compute capability 10.x, and its SMs

cudaError_t rows_status_word(int **word);               // where the calls on rows of the current device note a wait that ran out

// A launch's result as a status; a refused launch leaves no error behind for the caller's next CUDA call.
inline gdws_status_t launched(cudaError_t e, const char *what)
{
    if (e == cudaSuccess) return GDWS_OK;
    cudaGetLastError();
    return cuda_fail(e, what);
}

// An arrival, at a barrier of either block of a pair, that gives tensor memory back.  It publishes nothing in memory and orders nothing by
// itself: the caller has waited for its loads from tensor memory (tcgen05.wait::ld) and fenced them before the threads' meeting
// (tcgen05.fence::before_thread_sync), so the registers hold what is about to be overwritten.  (A releasing arrival also waits until
// the warp's stores to y have been performed.)
__device__ __forceinline__ void mbar_arrive_relaxed(uint32_t bar)
{
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

// A wait on arrivals from both blocks of a pair: acquire at cluster scope, bounded like the others.
static __device__ __noinline__ void mbar_wait_cluster(uint32_t bar, uint32_t parity, volatile int *abort_flag, int *status, int code)
{
    for (uint32_t it = 0; it < kSpinLimit; ++it) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
        if (ok) return;
        if (it > 4096) __nanosleep(64);
        if ((it & 1023) == 0 && *abort_flag) return;
    }
    *abort_flag = 1;
    atomicOr(status, code);
}

}  // namespace gdws
