// Checks that the entry points with norms and rotations share, and what they make of them for the kernels.
#pragma once

#include "api_checks.hpp"
#include "rows_params.hpp"

// One of a call's tensors, as the entry points are given it.
struct dbsp_rows_tensor {
  const void* x;
  int64_t batch, head, token;
};

// Norm, rotation and positions of a call with `rows` tokens a sequence; which kernel (norm's kind, halves).
int dbsp_rows_settle(const char* who, const dbsp_head_norm* norm, const dbsp_rotary* rotary, const int32_t* positions, int64_t pos_batch,
                     int64_t pos_token, int32_t B, int32_t N, int32_t d, dbsp_rows_params& p, int& kind, bool& halves);
// A tensor that is read or written.
int dbsp_rows_check(const char* who, const char* name, const dbsp_rows_tensor& t, bool written, int32_t B, int32_t heads, int32_t N, int32_t d);
// Deals the heads of a launch's tensors to workgroups, `most` in all where there is enough to deal.
int dbsp_rows_deal(const char* who, dbsp_rows_params& p, int d, int64_t most);
