// Kernel argument block of attention over a paged cache (device pointers and sizes only), and what host and kernels have to agree on.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

constexpr int kPagedKeys = 64;         // keys of a tile, 16 a wave
// Rows of a row tile: 16, 32, or at d = 64 64, by how many there are (64 of d = 128 do not fit into the registers of two waves)
constexpr int paged_tile_rows(int64_t rows, int d) { return rows <= 16 ? 16 : rows <= 32 || d == 128 ? 32 : 64; }
constexpr int kPagedTarget = 1024;     // items that a launch is cut into where there is enough to cut
constexpr int kPagedWhole = 10;        // tiles that are not cut
constexpr int kPagedMergeRows = 2048;  // rows up to which a workgroup joins the parts of one

// slot / page_size as slot * mul >> shift, for slots below 2^31: with 2^s >= page_size, mul = 2^(31 + s) / page_size rounded up is too large by
// less than 1, so the product by less than slot / 2^(31 + s) < 2^-s <= 1 / page_size of the quotient.
inline void paged_divisor(int page_size, uint32_t& mul, uint32_t& shift) {
  shift = 31;
  while (((int64_t)1 << (shift - 31)) < page_size) ++shift;
  mul = (uint32_t)((((uint64_t)1 << shift) + page_size - 1) / page_size);
}
__host__ __device__ inline int paged_quotient(int slot, uint32_t mul, uint32_t shift) { return (int)(((uint64_t)(uint32_t)slot * mul) >> shift); }

struct dbsp_paged_attn_params {
  const uint16_t* q;
  const unsigned char *k, *v;
  uint16_t* o;
  float* lse;                          // f32 [B,H,Nq] or null
  const int32_t *lens, *q_lens, *pages;
  int64_t q_sb, q_sh, q_st, o_sb, o_sh, o_st;      // strides in elements: batch, head, token
  int64_t k_sp, k_sh, v_sp, v_sh;                  // in bytes: page, head
  int32_t k_ss, v_ss;                              // in bytes: slot
  int64_t pages_stride;
  int32_t B, H, Hk, G, Nq, n_pages, page_size, max_pages, cap;
  uint32_t page_mul, page_shift;       // see paged_quotient
  int32_t causal, split, target;
  int32_t row_tiles, own_rows;         // of a (sequence, KV head); rows of a partial result
  float scale_log2;                    // softmax scale * log2(e)
  // workspace
  int32_t* table;                      // [2 B] first part and parts of every sequence
  float *part_o, *part_lse;            // f32 [items][own_rows][d], [items][own_rows] (base 2)
  int32_t merge_groups, merge_by_row;
};

hipError_t dbsp_launch_paged_attn(const dbsp_paged_attn_params& p, int d, bool fp16, int grid, hipStream_t stream);
