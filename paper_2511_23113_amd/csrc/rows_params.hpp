// Kernel argument blocks of the norms and rotations of queries and keys (device pointers and sizes only), and their launches.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

constexpr int kRowThreads = 256;       // of a workgroup: d / 8 lanes a row, each row of them another token
constexpr int kRowGroups = 2048;       // workgroups that a launch is cut into where there is enough to cut: eight a compute unit
constexpr int kGradGroups = 1024;      // those of the backward pass, which leave a partial sum each

// Bytes that a launch reads and writes from which it goes past the caches, which hold 256 MB: what it leaves there does not live until it is
// read.  us, through / past them, and with a reader of the results behind it: 32,760 tokens of 40 + 40 heads of 128 (1342 MB) 265 / 253,
// 483 / 474, 8000 tokens 68 / 63, 115 / 116, but 12,303 tokens of 30 + 10 heads of 64 (126 MB) 30.5 / 33.3, 52.6 / 59.7.
constexpr int64_t kRowStream = (int64_t)512 << 20;
// And if whole lines of 128 bytes are stored at a time, as pieces of lines are joined in the caches only: rotations by halves of 64 pairs, or none.
// Halves of 32 pairs, 32,760 tokens of 80 + 40 heads of 64 215 / 238, gradients 178 / 192; of 64 pairs at d = 128 264 / 249, 224 / 214.
constexpr bool row_lines_whole(bool halves, int turned) { return !halves || turned == 64; }

// One of a launch's tensors: queries, keys, or (appended) values, whose heads are dealt to `groups` workgroups, `per` each.
struct dbsp_rows_part {
  const uint16_t* x;                   // [B, heads, N, d], strides in elements
  const uint16_t* dy;                  // backward only
  uint16_t* y;                         // the result; null: the pool's pages
  int64_t x_sb, x_sh, x_st, dy_sb, dy_sh, dy_st, y_sb, y_sh, y_st;
  const void *gain, *bias;             // [d] or null
  int32_t heads, per, groups;
  int32_t plain;                       // neither norm nor rotation
  int64_t page_s;                      // of the pool (y_sh and y_st are its head's and slot's)
  uint16_t* pool;
};

struct dbsp_rows_params {
  dbsp_rows_part part[3];
  int32_t B, N;
  int32_t tiles;                       // of tokens, those of a workgroup each
  int32_t groups;                      // of heads, over all parts
  int32_t gains_f32;
  int32_t stream;                      // see kRowStream
  float eps;
  const int32_t* positions;            // [B, N, axes], or null: the token's place, or its slot
  int64_t pos_sb, pos_st;
  int32_t turned;                      // R
  int32_t ends[3];                     // first pairs of axes 1, 2, 3
  // paged
  const int32_t *lens, *new_lens, *pages;
  int64_t pages_stride;
  int32_t n_pages, page_size, cap;
  // backward
  float* grads;                        // [4, d] or null
  float* sums;                         // workspace [workgroup][gain, bias][d], those of the first part first
  int32_t walkers;                     // workgroups of a group of heads, which take the tiles in turn
  double turns[64];                    // freqs / (2 pi)
};

hipError_t dbsp_launch_rows(const dbsp_rows_params& p, int d, bool fp16, int kind, bool halves, bool paged, hipStream_t stream);
hipError_t dbsp_launch_rows_grad(const dbsp_rows_params& p, int d, bool fp16, int kind, bool halves, hipStream_t stream);
