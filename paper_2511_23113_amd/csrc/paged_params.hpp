// Kernel argument block of attention over a paged cache (device pointers and sizes only), and what host and kernels have to agree on.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

constexpr int64_t kMostSlots = (int64_t)1 << 30;      // of a sequence, and less
constexpr int kPagedKeys = 64;         // keys of a tile, 16 a wave
// Rows of a row tile, by how many there are.  At d = 128 more than 32 take the registers of one wave a SIMD: 256 (sequence, KV head) pairs of 41 tiles
// and 40 rows 89.6 us, with two row tiles of 32 116; 128 of them with 48 53.7, 64; 64 of 80 and 100 rows 79.4, 92; 40 of 78 and 64 rows 42.4, 43.2.
constexpr int paged_tile_rows(int64_t rows) { return rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 48 ? 48 : 64; }
constexpr int kPagedWhole = 10;        // tiles that a row tile may have at most where each goes to a workgroup of its own, without a merge

// slot / page_size as slot * mul >> shift, for slots below 2^31: with 2^s >= page_size, mul = 2^(31 + s) / page_size rounded up is too large by
// less than 1, so the product by less than slot / 2^(31 + s) < 2^-s <= 1 / page_size of the quotient.
inline void paged_divisor(int page_size, uint32_t& mul, uint32_t& shift) {
  shift = 31;
  while (((int64_t)1 << (shift - 31)) < page_size) ++shift;
  mul = (uint32_t)((((uint64_t)1 << shift) + page_size - 1) / page_size);
}
__host__ __device__ inline int paged_quotient(int slot, uint32_t mul, uint32_t shift) { return (int)(((uint64_t)(uint32_t)slot * mul) >> shift); }

// The list of tiles is cut into runs if row tiles have at least kPagedLong tiles each on average and 512 runs would have eight, else row tiles are
// cut into parts for themselves, kPagedRuns in all, and one more a row tile at most.  us, runs / parts: 256 (sequence, KV head) pairs of 41 tiles 67.4 / 72,
// 8 of 1650 83 / 87, 400 of 13 42.4 / 45; but 512 of 9 37.5 / 35.1, and at d = 64 2048 of 6 52.4 / 45.7, 240 of 12 with 21 rows each 24.3 / 18.
constexpr unsigned kPagedLong = 12, kPagedRuns = 512;
// Runs: two workgroups a compute unit, or one where it draws as much from memory, that is for single tokens at d = 128 over row tiles of
// kPagedEnds tiles and more on average (at a row tile's end nothing else runs on the compute unit).  us, one / two: 256 pairs of 41 tiles
// 67.4 / 68.9, 64 of 258 89.4 / 91.2, 64 of 62 31.1 / 32.1, 1024 of 20 134.5 / 137; but 512 of 14 54.3 / 51.9, 240 of 13 30.4 / 27.6, 400 of 13
// 43.3 / 42.4; at d = 64 256 of 83 69.1 / 67.0, and 240 of 12 with 21 rows each 43.4 / 29.2.
// And 256 where only one fits: more than 32 rows at d = 128 (with 512 for two rounds 95.2 us where 256 take 89.6, and 29.3 where they take 21.7).
constexpr unsigned kPagedEnds = 20;
constexpr unsigned paged_slots(int64_t rows, int d) { return d == 128 && rows > 32 ? kPagedRuns / 2 : kPagedRuns; }
constexpr unsigned paged_runs(int64_t rows, int d) { return d == 128 && rows <= 16 ? kPagedRuns / 2 : paged_slots(rows, d); }

struct dbsp_paged_attn_params {
  const uint16_t* q;
  const unsigned char *k, *v;
  uint16_t* o;
  float* lse;                          // f32 [B,H,Nq] or null
  const int32_t *lens, *q_lens, *pages;
  int64_t q_sb, q_sh, q_st, o_sb, o_sh, o_st;      // strides in elements: batch, head, token
  int64_t k_sh, v_sh;                              // in bytes: head
  uint32_t k_sp, k_ss, v_sp, v_ss;                 // in bytes: page, slot
  int64_t pages_stride;
  int32_t B, H, Hk, G, Nq, n_pages, page_size, max_pages, cap;
  uint32_t page_mul, page_shift;       // see paged_quotient
  int32_t causal, whole;
  int32_t page_16;                     // a page's slots are a multiple of a wave's 16
  uint32_t slots, runs;                // parts, or runs over short row tiles, that the list of tiles is cut into, and runs over long ones
  int32_t row_tiles, own_rows;         // of a (sequence, KV head); rows of a partial result
  float scale_log2;                    // softmax scale * log2(e)
  // workspace
  int32_t* table;                      // [2 + 2 B] tiles of a run or part, and which (1: parts, 2: nothing is cut); of every sequence what is before it, and its tiles
  float *part_o, *part_lse;            // f32 [parts][own_rows][d], [parts][own_rows] (base 2)
  int32_t merge_groups, merge_ways;    // workgroups of the merge, and how many of a row's parts it takes at a time, eight each
};

hipError_t dbsp_launch_paged_attn(const dbsp_paged_attn_params& p, int d, bool fp16, int grid, hipStream_t stream);
