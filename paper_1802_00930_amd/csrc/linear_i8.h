// Launchers of the INT8 linear layers (quant_i8.hip, linear_i8.hip).
#pragma once

#include "dfp_internal.h"
#include "mm_plan.h"

namespace dfp {

// Rows of src (times colw of the column, nullable) to q [rows][i8_ld(cols)] and scale [rows].
dfp_status launch_rows_i8(int32_t type, int32_t rounding, uint64_t seed, uint32_t role, const void* src, int64_t rows,
                          int64_t cols, const float* colw, int8_t* q, float* scale, hipStream_t st);
dfp_status launch_transpose_i8(const int8_t* q, int64_t rows, int64_t cols, int8_t* qt, hipStream_t st);

// Columns of src times roww of the row, to qt [cols][i8_ld(rows)] and scale [cols]; sums (nullable): src summed
// over the rows.  ws: plan_cols_i8(...).bytes.
struct ColPlan {
  int64_t slice, parts, bytes;
};
ColPlan plan_cols_i8(int64_t rows, int64_t cols);
dfp_status launch_cols_i8_t(int32_t type, int32_t rounding, uint64_t seed, uint32_t role, const void* src,
                            int64_t rows, int64_t cols, const float* roww, int8_t* qt, float* scale, float* sums,
                            void* ws, hipStream_t st);

// out [m][n] (type) = (sum over k of a b) sa[m] sb[n] + bias[n]; sb, bias nullable.  ws: plan_gemm_i8(...).bytes
// (mm_plan.h).
dfp_status launch_gemm_i8(int32_t m, int32_t n, int32_t k, const int8_t* a, const float* sa, const int8_t* b,
                          const float* sb, const float* bias, int32_t type, void* out, void* ws, hipStream_t st);
// The forward call for a few tokens in one launch, where fits_token_i8.
bool fits_token_i8(int64_t m, int64_t k);
dfp_status launch_token_i8(int32_t m, int32_t n, int32_t k, int32_t type, int32_t rounding, uint64_t seed,
                           const void* x, const int8_t* b, const float* sb, const float* bias, void* out,
                           hipStream_t st);

}  // namespace dfp
