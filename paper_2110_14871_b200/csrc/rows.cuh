// Shared by the calls on rows (rows.cu, pointwise8.cu).
#pragma once

#include "sm100.cuh"

namespace gdws {

constexpr int kMost8 = 131071;      // products of two 8-bit integers whose sum fits 32 bits: 131071 * 2^14 < 2^31

gdws_status_t check_rows(const char *call, const char *name, const gdws_rows_t *m);
gdws_status_t check_rows8(const char *call, const char *name, const gdws_rows8_t *m);
gdws_status_t check_pointwise8(const gdws_rows8_t *x, const gdws_rows8_t *w, const float *bias, const gdws_rows_t *y);
gdws_status_t rows_device(int *device, int *sms);       // the current device, checked to be compute capability 10.x, and its SMs

}  // namespace gdws
