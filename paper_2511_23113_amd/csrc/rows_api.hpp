// Checks that the entry points with norms and rotations share, and what they make of them for the kernels.
#pragma once

#include "api_checks.hpp"
#include "rows_params.hpp"

// A call's sizes, norm, rotation and positions; which kernel (norm's kind, halves).
int dbsp_rows_settle(const char* who, const dbsp_qk_rows* rows, const dbsp_head_norm* norm, const dbsp_rotary* rotary, dbsp_rows_params& p, int& kind,
                     bool& halves);
// A tensor that is read or written.
int dbsp_rows_check(const char* who, const char* name, const dbsp_heads& t, bool written, int32_t B, int32_t heads, int32_t N, int32_t d);
// Deals the heads of a launch's tensors to workgroups, `most` in all where there is enough to deal.
int dbsp_rows_deal(const char* who, dbsp_rows_params& p, int d, int64_t most);

namespace {

inline void set_in(dbsp_rows_part& part, const dbsp_heads& t, int32_t B, int32_t heads, int32_t N) {
  part.x = static_cast<const uint16_t*>(t.x);
  part.x_sb = step(B, t.stride[0]);
  part.x_sh = step(heads, t.stride[1]);
  part.x_st = step(N, t.stride[2]);
  part.heads = heads;
}
inline void set_out(dbsp_rows_part& part, const dbsp_heads& t, int32_t B, int32_t heads, int32_t N) {
  part.y = static_cast<uint16_t*>(t.x);
  part.y_sb = step(B, t.stride[0]);
  part.y_sh = step(heads, t.stride[1]);
  part.y_st = step(N, t.stride[2]);
}

}  // namespace
