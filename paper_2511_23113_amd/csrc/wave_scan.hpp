// Sums and the like over a wave's lanes, in registers (data-parallel primitives, no trip through the LDS).
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

namespace {

// Sum over the wave's lanes up to and with this one: within rows of 16 lanes, then from the ends of rows on.
__device__ __forceinline__ int scan_wave(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);      // row_shr:1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);      // row_bcast:15, into rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);      // row_bcast:31, into rows 2 and 3
  return x;
}

// f over the 16 lanes of a row, in each of them; all of the row's lanes are active.
template <class X, class F>
__device__ __forceinline__ X over_row(X x, F&& f) {
  auto ror = [](X v, auto by) { return __builtin_bit_cast(X, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x120 + decltype(by)::value, 0xf, 0xf, false)); };
  x = f(x, ror(x, std::integral_constant<int, 8>{}));
  x = f(x, ror(x, std::integral_constant<int, 4>{}));
  x = f(x, ror(x, std::integral_constant<int, 2>{}));
  return f(x, ror(x, std::integral_constant<int, 1>{}));
}

}  // namespace
