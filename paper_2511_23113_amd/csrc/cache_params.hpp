// Kernel argument blocks of the key/value cache's operators (device pointers and sizes only), and what host and kernels have to
// agree on: tile sizes and the shape of the workspace.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

constexpr int kCacheKeys = 64;         // keys of a tile
constexpr int kCacheRows = 128;        // rows of a workgroup of the kernel for few queries: four waves of 32
// Of the kernel for many queries: waves of 64 rows (two of them a workgroup: frames of 1560 queries 1.5 % slower, though they
// leave 6 % of the rows of their tiles empty and not 13, causal prompts 1.6 % faster). Which launches
// are its: cache_api.hip, is_many.
constexpr int kLongWaves = 4, kLongRows = 64 * kLongWaves;
constexpr int kLongSlots = 256;        // of its workgroups at a time at d = 128: a compute unit each; at d = 64 twice as many
// Items that a launch is cut into where there is enough to cut: two rounds of the chip at d = 128, one at d = 64.  us with 512 / 1024 /
// 2048 / 4096: 384 (sequence, head) pairs of 1500 own keys behind 4096 shared ones 89 / 85 / 88 / 96, 4 heads' prefix of 131,072 84 /
// 84 / 98 / 123, 256 pairs of 4400 keys 143 / 135 / 130 / 145, 240 pairs of 21 rows 32 / 31 / 35 / 45.
constexpr int kCacheTarget = 1024;
// Tiles that are not cut: a launch less, and the merge.  us with 4 / 8 / 16: 256 pairs of 8 tiles 18.3 / 12.4 / 12.4, 8 pairs of 8 tiles
// 11.4 / 9.7 / 9.7, of 16 tiles 10.5 / 10.5 / 14.0.
constexpr int kCacheWhole = 10;
// Prefix tiles that every sequence reads for itself.  us with 2 / 4 / 8: 256 pairs of 5 tiles behind 6 prefix tiles 46 / 46 / 50, 1024 of
// 24 tiles behind 4 148 / 143 / 143, behind 8 149 / 149 / 151.
constexpr int kPooledFrom = 4;
// Rows of a (sequence, KV head) up to which scores are kept for the weights, at d = 128 (half as many at d = 64): they are written and read,
// 8 bytes a row and key, where forming them anew reads 2 d bytes a key, from memory or a cache.  us, anew / kept: 128 pairs of
// 1500 keys at d = 128 16 rows 60 / 46, 32 rows 69 / 59, 64 rows 74 / 81; at d = 64 16 rows 41 / 30, 32 rows 46 / 40; 512 pairs of
// 6000 keys at d = 64 16 rows 349 / 294, 32 rows 347 / 392.
constexpr int kScoreRows = 48;
constexpr int kWeightKeys = 256;       // own keys of a workgroup that forms their scores anew: 64 a wave
// Rows up to which a workgroup joins the parts of one, else of 8 or 16: so much the better the more parts a row has.  us of a call by one /
// by several: 300 rows 14.4 / 20.9, behind 60,000 keys 45 / 68, 480 at d = 64 14.5 / 23.4, 768 23.0 / 23.8, behind 20,000 37 / 46, 1000 at d = 64
// 19.0 / 19.4, 1536 behind 8000 28.6 / 30.6, behind 40,000 58.8 / 61.8; but 1920 behind 2000 27.3 / 25.0, 2304 of 3000 own keys 70.8 / 66.5, 2560 behind
// 16,384 120.6 / 118, 2400 at d = 64 behind 60,000 70.4 / 70.2, 3200 behind 4096 28.6 / 23.3, 5040 37.0 / 28.4, 12,000 of 1500 own keys 50 / 29.
constexpr int kMergeRows = 2048;
constexpr int kScoreSlots = 1024;      // own keys of a workgroup that sums kept scores, four a thread
constexpr int kEvictWhole = 32768;     // slots that a workgroup chooses among by itself: what its registers hold; and those of a
constexpr int kEvictPart = 8192;       // part where there are more
// Threads that choose among so many slots.  us with 1024 / 512 / 256: 2048 (sequence, head) pairs of 750 slots 87 / - / 65, of 3000 slots
// 179 / 160 / 164, 256 of 2064 15.5 / 15.5 / 19, 16 of 3800 14.3 / 15.1 / 19.6.
constexpr int evict_threads(int slots) { return slots <= 1024 ? 256 : slots <= 4096 ? 512 : 1024; }

// How a launch of the kernel for many queries is cut: its row tiles, `per` for each of `dies` dies (workgroup number mod 8), of which
// the first `whole` are one item each and the `tail` others `k` parts, so that the last round of workgroups ends together.
struct dbsp_cache_long_cut {
  int32_t items, dies, per, whole, tail, k, longest_first;
};

struct dbsp_cache_attn_params {
  const uint16_t *q, *pk, *pv, *k, *v;
  uint16_t* o;
  float* lse;                          // f32 [B,H,Nq] or null
  float* weights;                      // f32 [B,Hk,cap] or null
  const int32_t *lens, *q_lens;        // [B]; null: no own keys; every sequence has Nq new tokens
  int64_t q_sb, q_sh, q_st, o_sb, o_sh, o_st;      // strides in elements: batch, head, token
  int64_t pk_sh, pv_sh, k_sb, k_sh, v_sb, v_sh;
  int32_t pk_st, pv_st, k_st, v_st;                // token strides in bytes
  int32_t B, H, Hk, G, Nq, P, cap;
  int32_t causal;
  int32_t many;                        // the kernel of cache_attn_long.hip
  int32_t pooled;                      // the prefix is read by the rows of all sequences together, own keys apart
  int32_t split;                       // items may be parts of a row tile's keys: partial results, and a merge behind the kernel (kernel for few queries)
  int32_t target;                      // items that the launch is cut into where there is enough to cut
  int32_t pre_longer;                  // times the tiles of an own item that one of the pooled prefix has
  int32_t pre_tiles;                   // tiles of the prefix
  int32_t pre_row_tiles, own_row_tiles;            // row tiles of a KV head: of all sequences together (pooled), of one sequence
  int32_t own_tile_rows;               // rows of an own item: kCacheRows, or kLongRows for the kernel of cache_attn_long.hip
  int32_t own_rows;                    // and of its partial result: not more than Nq * G
  int32_t row_shift;                   // with longest_first: so many rows of the first row tile are none, as it has the fewest keys
  int32_t max_pre_items;
  dbsp_cache_long_cut cut;             // with `many` only
  float scale_log2;                    // softmax scale * log2(e)
  float decay;
  // workspace
  int32_t* table;                      // [2 + 2 B] chunks and items of the prefix, then first own item and chunks of every sequence
  float* row_lse;                      // f32 [B,H,Nq]: log2 of the sum of exp, for the weights
  float* part_o;                       // f32 [items][rows][D], prefix items first
  float* part_lse;                     // f32 [items][rows], base 2
  float* scores;                       // f32 [B,Hk][own_rows][score_pitch] q.k of the own keys (-inf where not seen), or null
  int64_t score_pitch;
  int32_t row_parts;                   // parts into which the rows are cut for the weights of own keys, and f32 [row_parts][B,Hk,cap]
  float* part_w;                       // for their sums where there are more than one
  // workgroups of the finishing launch: those that join parts, a row each with merge_by_row, and those that sum kept scores
  int32_t merge_groups, merge_by_row, sum_groups;
};

struct dbsp_cache_evict_params {
  unsigned char *k, *v;
  float* weights;                      // [B,Hk,cap]
  int32_t* positions;                  // [B,Hk,cap]
  int32_t* lens;                       // [B]
  const int32_t* keep_from;            // [B] or null
  int64_t k_sb, k_sh, k_st, v_sb, v_sh, v_st;      // strides in bytes
  int32_t B, Hk, cap, row_bytes;
  int32_t budget, sinks;
  int32_t max_moves;                   // min(budget, cap - budget)
  int32_t n_parts;                     // parts of kEvictPart slots; 0: a workgroup takes a (sequence, head) whole
  // workspace
  int32_t* n_moves;                    // [B Hk]
  int32_t *holes, *fillers;            // [B Hk][max_moves]
  uint32_t* digits;                    // [B Hk][3][2048] images by digit; only with parts
  uint32_t* chosen;                    // [B Hk][3] the limit, how many of its equals stay, and how many there are
  int32_t* parts;                      // [B Hk][n_parts][4] images above the limit and equal to it, below the budget and from it on
};

hipError_t dbsp_launch_cache_attn(const dbsp_cache_attn_params& p, int d, bool fp16, int grid, hipStream_t stream);
hipError_t dbsp_launch_cache_attn_long(const dbsp_cache_attn_params& p, int d, bool fp16, int grid, hipStream_t stream);
hipError_t dbsp_launch_cache_weights(const dbsp_cache_attn_params& p, int d, bool fp16, hipStream_t stream);
hipError_t dbsp_launch_cache_evict(const dbsp_cache_evict_params& p, hipStream_t stream);
