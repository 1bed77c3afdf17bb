// What the entry points' argument checks share: error returns, alignment, strides.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cstdint>
#include <string>

#include "dbsp.h"
#include "plan.hpp"

namespace {

inline int fail(const char* who, int code, const char* what) { return dbsp_set_error(code, std::string(who) + ": " + what); }

inline int done(const char* who, hipError_t e) {
  if (e == hipSuccess) return DBSP_OK;
  (void)hipGetLastError();
  return dbsp_set_error(DBSP_EHIP, std::string(who) + ": " + hipGetErrorString(e));
}

inline bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// Strides (the token's last) are ones that the kernels can go by; that of a dimension of one says nothing.
inline bool strides_ok(const int64_t* size, const int64_t* s, int n) {
  for (int i = 0; i < n; ++i)
    if (size[i] > 1 && (s[i] < 0 || s[i] % 8 != 0 || s[i] > (int64_t)1 << (i == n - 1 ? 24 : 40))) return false;
  return true;
}
inline int64_t step(int64_t size, int64_t stride) { return size > 1 ? stride : 0; }

// No two elements of a tensor with these sizes and strides (its last dimension dense, d long) share a place: in the order of their
// strides each dimension steps over all that the ones before it reach.
inline bool distinct(const int64_t* size, const int64_t* stride, int64_t d) {
  int order[3] = {0, 1, 2};
  std::sort(order, order + 3, [&](int a, int b) { return stride[a] < stride[b]; });
  __int128 reach = d;
  for (int i : order) {
    if (size[i] <= 1) continue;
    if (stride[i] < reach) return false;
    reach += (__int128)stride[i] * (size[i] - 1);
  }
  return true;
}

inline int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

constexpr int64_t kMost = INT_MAX / 2;
constexpr int64_t kMostThreads = UINT32_MAX;       // of a launch along a dimension: HIP has no more

}  // namespace
