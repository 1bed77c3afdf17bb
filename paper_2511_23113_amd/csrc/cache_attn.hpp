// What the kernels of attention over a key/value cache share: types, the layout of tiles in the LDS, copies, and which item a workgroup has.
#pragma once

#include <hip/hip_runtime.h>

#include <cfloat>
#include <climits>
#include <cstdint>

#include "attn_common.hpp"
#include "cache_params.hpp"
#include "wave_scan.hpp"

namespace {

// Probabilities are formed against a running max as it stands, and may pass 1 by this (a single one, or a lane's sum of 16) before it
// is raised: f32 sums hold that as they hold 1, and so do fp16's 65504 and its 2^-14 at the other end.  (64: 2 % slower)
constexpr float kRaiseAt = 1024.f;

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

struct Bf16 {
  // 16 x 16 outputs, over 32 or 16 products
  static __device__ __forceinline__ f32x4 mfma32(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x4 mfma16(u32x2 a, u32x2 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, a), __builtin_bit_cast(s16x4, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack(float a, float b) { return pack_bf16x2(a, b); }
  static __device__ __forceinline__ uint32_t pack_o(float a, float b) { return pack(a, b); }
};
struct Fp16 {
  static __device__ __forceinline__ f32x4 mfma32(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x4 mfma16(u32x2 a, u32x2 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x16f16(__builtin_bit_cast(f16x4, a), __builtin_bit_cast(f16x4, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    f32x2 f = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, f16x2));      // round to nearest even
  }
  // Of O: no larger than the largest v, 65504 at most, but the rounded probabilities may sum to 1 + 2^-11, and from 65520 on a number is
  // rounded to infinity.  Those that are finite in f32 stop at 65504 (by their bits: NaNs are not regarded in these files, and stay).
  static __device__ __forceinline__ float within(float x) {
    constexpr uint32_t kTop = 0x477fe000u;       // 65504
    return (__builtin_bit_cast(uint32_t, x) & 0x7fffffffu) - kTop < 0x7f800000u - kTop ? __builtin_copysignf(65504.f, x) : x;
  }
  static __device__ __forceinline__ uint32_t pack_o(float a, float b) { return pack(within(a), within(b)); }
};

// Of a d-wide K or V tile in the LDS: rows unpadded, 16-byte chunks XOR-swizzled inside each row (K by the row, so that the
// operand reads of 16 consecutive keys hit distinct banks; V by (row & 3), for the 4 keys of a transposing read).
template <int D>
struct Lay {
  static constexpr int DT = D / 32, KS = D / 16, NCH = D / 8, RPL = 128 / D, ROWB = 2 * D;
  static constexpr int TILE = kCacheKeys * ROWB;       // bytes of a K (or V) tile
  static constexpr int RPC = 64 / NCH;                 // rows that one copy instruction of a wave moves
  static constexpr int COPIES = 16 / RPC;              // a wave copies 16 rows of K and 16 of V
  static __device__ __forceinline__ int k_swz(int row) { return (row / RPL) % NCH; }
  static __device__ __forceinline__ int v_swz(int row) { return ((row / RPL) % (NCH / 4)) << 2; }
};

// 16 bytes a lane from base + voff to the LDS at dst + 16 * lane.  Its own wait counts: see wait_all.
__device__ __forceinline__ void copy_row16(const unsigned char* base, uint32_t voff, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(voff), "s"(base), "s"(dst) : "memory");
}
__device__ __forceinline__ void wait_all() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); }

__device__ __forceinline__ int len_of(const dbsp_cache_attn_params& p, int b) { return p.lens ? max(0, min(p.lens[b], p.cap)) : 0; }
__device__ __forceinline__ int q_len_of(const dbsp_cache_attn_params& p, int b) { return p.q_lens ? max(0, min(p.q_lens[b], p.Nq)) : p.Nq; }
__device__ __forceinline__ int tiles_of(int keys) { return (int)(((unsigned)keys + kCacheKeys - 1) / kCacheKeys); }
// key tiles of sequence b's row tiles (the last one's, where causality leaves the others fewer)
__device__ __forceinline__ int own_tiles(const dbsp_cache_attn_params& p, int b) {
  return (p.pooled ? 0 : p.pre_tiles) + tiles_of(len_of(p, b));
}

struct Item {
  int b;                 // sequence, -1: an item of the pooled prefix
  int hk, rt;            // KV head, row tile
  int c, n;              // part c of n
  int64_t slot;          // of its partial result
};

// Row tile x of all, sequence by sequence and head by head, the last rows first.
__device__ __forceinline__ void row_tile(const dbsp_cache_attn_params& p, int x, Item& it) {
  it.rt = p.own_row_tiles - 1 - x % p.own_row_tiles;
  it.hk = x / p.own_row_tiles % p.Hk;
  it.b = x / p.own_row_tiles / p.Hk;
}
// Row tile x of a die, of a launch of the kernel for many queries; false: it has no such.  Either a run of the tiles in the order
// above, so that those of the same keys run at the same time, or, where causality makes the tiles of different lengths, the
// longest ones first, the (sequence, head) pairs dealt to the dies in turn.
__device__ __forceinline__ bool long_row_tile(const dbsp_cache_attn_params& p, int die, int x, Item& it) {
  const dbsp_cache_long_cut& cut = p.cut;
  const int n = cut.longest_first ? x * cut.dies + die : die * cut.per + x;
  if (n >= cut.items) return false;
  if (cut.longest_first) {
    const int pairs = p.B * p.Hk;
    it.rt = p.own_row_tiles - 1 - n / pairs;
    it.hk = n % pairs % p.Hk;
    it.b = n % pairs / p.Hk;
  } else {
    row_tile(p, n, it);
  }
  return true;
}

// Which item this workgroup has; false: none.  All of the workgroup's threads call it.
__device__ __forceinline__ bool find_item(const dbsp_cache_attn_params& p, Item& it) {
  constexpr int NT = 256, WAVES = NT / 64;
  const int t = threadIdx.x, w = t >> 6, l = t & 63;
  const int unit = p.Hk * p.own_row_tiles;
  if (!p.split) {        // a row tile an item
    const int n = p.B * unit, per = (n + 7) / 8, x = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per || x >= n) return false;
    row_tile(p, x, it);
    it.c = 0;
    it.n = 1;
    it.slot = -1;
    return true;
  }
  // Parts of every sequence, and where they begin: a sequence (or a run of them) a thread.  Up to 64 of them each wave works it
  // out for itself, without a barrier.
  const bool by_wave = p.B <= 64;
  const int x = by_wave ? l : t, per_thread = by_wave ? 1 : (p.B + NT - 1) / NT, b0 = min(x * per_thread, p.B), b1 = min(b0 + per_thread, p.B);
  __shared__ int64_t tile_sum[WAVES];
  __shared__ int part_sum[WAVES], found[3];
  int64_t own = 0;
  for (int b = b0; b < b1; ++b) own += own_tiles(p, b);
  if (by_wave) {
    own = __builtin_amdgcn_readlane(scan_wave((int)own), 63);
  } else {
    for (int s = 32; s > 0; s >>= 1) own += __shfl_xor(own, s);
    if (l == 0) tile_sum[w] = own;
    __syncthreads();
    own = 0;
    for (int i = 0; i < WAVES; ++i) own += tile_sum[i];
  }
  const int64_t total = own * unit + (p.pooled ? (int64_t)p.Hk * p.pre_row_tiles * p.pre_tiles : 0);
  // (of short key lists up to four tiles an item as long as there are 256 of them, as every part costs the merge: 8 heads over 7600
  // keys 23.3 us with one tile an item, 17.9 with two, 16.3 with four)
  const int chunk = (int)max(max((int64_t)1, min((int64_t)4, total / 256)), min((int64_t)(1 << 30), (total + p.target - 1) / p.target));
  auto parts = [&](int n) { return max(1, (n + chunk - 1) / chunk); };
  int mine = 0;
  for (int b = b0; b < b1; ++b) mine += parts(own_tiles(p, b));
  const int upto = scan_wave(mine);
  int before = 0, all = __builtin_amdgcn_readlane(upto, 63);
  if (!by_wave) {
    if (l == 63) part_sum[w] = upto;
    __syncthreads();
    all = 0;
    for (int i = 0; i < WAVES; ++i) {
      if (i < w) before += part_sum[i];
      all += part_sum[i];
    }
  }
  const int pre_parts = p.pooled ? max(1, (p.pre_tiles + chunk * p.pre_longer - 1) / (chunk * p.pre_longer)) : 0, pre_items = p.Hk * p.pre_row_tiles * pre_parts;
  int first = before + upto - mine;        // parts of the sequences before this thread's
  if (blockIdx.x == 0 && (w == 0 || !by_wave)) {      // for the merge
    if (t == 0) { p.table[0] = pre_parts; p.table[1] = pre_items; }
    int f = first;
    for (int b = b0; b < b1; ++b) {
      const int n = parts(own_tiles(p, b));
      p.table[2 + 2 * b] = f;
      p.table[3 + 2 * b] = n;
      f += n;
    }
  }
  // every die has its share of the prefix's items, then of the own ones: the first are bound by the matrix pipe where their rows are
  // many, the others by memory, and neither is left to a few dies
  const int die = blockIdx.x & 7, i = blockIdx.x >> 3;
  auto share = [](int64_t n, int d) { return (int)(n * d / 8); };
  const int own_items = unit * all, p0 = share(pre_items, die), np = share(pre_items, die + 1) - p0, o0 = share(own_items, die);
  if (i >= np + share(own_items, die + 1) - o0) return false;
  if (i < np) {
    const int z = p0 + i;
    it.b = -1;
    it.rt = z % p.pre_row_tiles;
    it.c = z / p.pre_row_tiles % pre_parts;
    it.hk = z / p.pre_row_tiles / pre_parts;
    it.n = pre_parts;
    it.slot = z;
    return true;
  }
  const int y = o0 + i - np, part = y / unit;      // parts before it, over all sequences
  int n = mine;
  if (by_wave) {
    const int at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(part >= first && part < first + mine));
    it.b = at;
    first = __builtin_amdgcn_readlane(first, at);
    n = __builtin_amdgcn_readlane(mine, at);
  } else {
    if (part >= first && part < first + mine) {
      for (int b = b0; b < b1; ++b) {
        n = parts(own_tiles(p, b));
        if (part < first + n) {
          found[0] = b;
          found[1] = first;
          found[2] = n;
          break;
        }
        first += n;
      }
    }
    __syncthreads();
    it.b = found[0];
    first = found[1];
    n = found[2];
  }
  const int z = y - first * unit;
  it.n = n;
  it.rt = p.own_row_tiles - 1 - z % p.own_row_tiles;
  it.c = z / p.own_row_tiles % it.n;
  it.hk = z / p.own_row_tiles / it.n;
  // partial results lie by sequence, head, part and row tile as the merge counts them; one item alone needs none
  it.slot = (it.n == 1 && !p.pooled) ? -1 : (int64_t)first * unit + (it.hk * it.n + it.c) * p.own_row_tiles + it.rt;
  return true;
}

// The same for the kernel for many queries.  Parts at the same place of their tiles' keys lie next to each other.
__device__ __forceinline__ bool find_long_item(const dbsp_cache_attn_params& p, Item& it) {
  const dbsp_cache_long_cut& cut = p.cut;
  const int die = blockIdx.x % cut.dies, y = blockIdx.x / cut.dies, z = y - cut.whole, x = z < 0 ? y : cut.whole + z % cut.tail;
  if (!long_row_tile(p, die, x, it)) return false;
  it.n = z < 0 ? 1 : cut.k;
  it.c = z < 0 ? 0 : z / cut.tail;
  it.slot = it.n == 1 ? -1 : ((int64_t)die * cut.tail + x - cut.whole) * cut.k + it.c;
  return true;
}

// Where an own (or prefix) item's partial result begins, in rows.
__device__ __forceinline__ int64_t part_row(const dbsp_cache_attn_params& p, bool own, int64_t slot) {
  return own ? (int64_t)p.max_pre_items * kCacheRows + slot * p.own_rows : slot * kCacheRows;
}

// Row r of a row list: token, head of the group, sequence.
struct Row { int b, t, g; };
__device__ __forceinline__ Row row_of(const dbsp_cache_attn_params& p, int b, int r) {
  const int tok = r / p.G, g = r % p.G;
  if (b >= 0) return {b, tok, g};
  return {tok / p.Nq, tok % p.Nq, g};
}

// The result of one row of an item: lanes (r, g) of its wave hold, of tile dt of the head dim, values 8 i + 4 g .. + 3 in o[dt][4 i ..].
// Behind a division by the sum of its probabilities (inv) it goes to O, or, of a part, to the workspace.
template <class T, int D>
__device__ __forceinline__ void store_row(const dbsp_cache_attn_params& p, const Item& it, const f32x16 (&o)[D / 32], const Row& at, int h, int row_in_tile,
                                          int g, float inv, float lse2) {
  if (it.slot >= 0) {
    const int64_t pr = part_row(p, it.b >= 0, it.slot) + row_in_tile;
    float* to = p.part_o + pr * D + 4 * g;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4*>(to + 32 * dt + 8 * i) = f32x4{o[dt][4 * i] * inv, o[dt][4 * i + 1] * inv, o[dt][4 * i + 2] * inv, o[dt][4 * i + 3] * inv};
    if (g == 0) p.part_lse[pr] = lse2;
    return;
  }
  uint16_t* to = p.o + at.b * p.o_sb + h * p.o_sh + at.t * p.o_st + 4 * g;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<u32x2*>(to + 32 * dt + 8 * i) = u32x2{T::pack_o(o[dt][4 * i] * inv, o[dt][4 * i + 1] * inv), T::pack_o(o[dt][4 * i + 2] * inv, o[dt][4 * i + 3] * inv)};
  if (g == 0) {
    const int64_t q_row = ((int64_t)at.b * p.H + h) * p.Nq + at.t;
    if (p.lse) p.lse[q_row] = lse2 * 0.69314718055994531f;
    if (p.weights) p.row_lse[q_row] = lse2;
  }
}

}  // namespace
