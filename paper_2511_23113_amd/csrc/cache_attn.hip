// Attention of new tokens over a key/value cache: a prefix that all sequences of the batch share, and each sequence's own keys.
//
// For query t of sequence b, head h of KV head hk = h / G, over the prefix's keys and the own keys that it sees
// (slot < len_b, causal: slot <= len_b - qlen_b + t):
//   s = scale q.k,  LSE = ln sum exp(s),  O = sum exp(s - LSE) v,
// in one pass with a running max and sum, and O = 0, LSE = -inf without a key.  With weights, a second pass over the own keys:
//   W[b, hk, slot] = decay W + sum over the group's heads and the sequence's queries of exp(s - LSE).
//
// Rows.  The G heads of a group read the same keys, so a row is a (token, head of the group) pair and a workgroup's tile is 128
// rows.  Where one sequence does not fill a tile (p.pooled) the prefix is read by the rows of all sequences together, once,
// and the own keys by each sequence's rows apart; else a row tile goes over the prefix and then over its own keys.
//
// Items.  An item is a row tile and a range of its key tiles.  Lengths are known on the device only, so every workgroup
// works out from them how the launch is cut: about kCacheTarget items of equally many tiles, each sequence into equal parts.
// Parts leave partial results (O, and LSE to base 2, in f32) that a second launch joins: LSE = log sum exp LSE_i,
// O = sum exp(LSE_i - LSE) O_i.  Items of the same keys lie next to each other and on the same die (workgroup number mod 8).
//
// A workgroup is four waves of 32 queries each.  Tiles of 64 keys go to the LDS directly (global_load_lds_dwordx4), two in
// turn, one barrier a tile.  Products are formed transposed, S^T = K Q^T and O^T = V^T P^T, with 32x32x16 MFMAs: lane r holds
// query r; the packed probabilities are the second product's operand as they lie, and V^T comes from transposing LDS reads
// (the layouts are those of attn_fwd.hip).  Probabilities are rounded to the inputs' type for that product, as they
// must be for the matrix pipe: half a step of it relative to each; sums are of the f32 values.
#include <hip/hip_runtime.h>

#include <cfloat>
#include <climits>
#include <cstdint>

#include "attn_common.hpp"
#include "cache_params.hpp"

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

struct Bf16 {
  static __device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack(float a, float b) { return pack_bf16x2(a, b); }
};
struct Fp16 {
  static __device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    f32x2 f = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, f16x2));      // round to nearest even
  }
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

// Which item this workgroup has; false: none.  All of the workgroup's threads call it.
__device__ __forceinline__ bool find_item(const dbsp_cache_attn_params& p, Item& it) {
  const int t = threadIdx.x, w = t >> 6, l = t & 63;
  const int unit = p.Hk * p.own_row_tiles;
  if (!p.split) {        // a row tile an item
    const int n = p.B * unit, per = (n + 7) / 8, x = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per || x >= n) return false;
    it.b = x / unit;
    it.hk = x % unit / p.own_row_tiles;
    it.rt = p.own_row_tiles - 1 - x % p.own_row_tiles;      // the longest first
    it.c = 0;
    it.n = 1;
    it.slot = -1;
    return true;
  }
  __shared__ int64_t tile_sum[4];
  __shared__ int part_sum[4], found[3];
  const int per_thread = (p.B + 255) / 256, b0 = min(t * per_thread, p.B), b1 = min(b0 + per_thread, p.B);
  int64_t tiles = 0;
  for (int b = b0; b < b1; ++b) tiles += own_tiles(p, b);
  for (int s = 32; s > 0; s >>= 1) tiles += __shfl_xor(tiles, s);
  if (l == 0) tile_sum[w] = tiles;
  __syncthreads();
  const int64_t total = (tile_sum[0] + tile_sum[1] + tile_sum[2] + tile_sum[3]) * unit + (p.pooled ? (int64_t)p.Hk * p.pre_row_tiles * p.pre_tiles : 0);
  const int chunk = (int)max((int64_t)1, min((int64_t)(1 << 30), (total + kCacheTarget - 1) / kCacheTarget));
  auto parts = [&](int n) { return max(1, (n + chunk - 1) / chunk); };
  int mine = 0;
  for (int b = b0; b < b1; ++b) mine += parts(own_tiles(p, b));
  int upto = mine;
  for (int s = 1; s < 64; s <<= 1) {
    const int o = __shfl_up(upto, s);
    if (l >= s) upto += o;
  }
  if (l == 63) part_sum[w] = upto;
  __syncthreads();
  int before = 0, all = 0;
  for (int i = 0; i < 4; ++i) {
    if (i < w) before += part_sum[i];
    all += part_sum[i];
  }
  const int pre_parts = p.pooled ? parts(p.pre_tiles) : 0, pre_items = p.Hk * p.pre_row_tiles * pre_parts;
  int first = before + upto - mine;        // parts of the sequences before this thread's
  if (blockIdx.x == 0) {                   // for the merge
    if (t == 0) { p.table[0] = pre_parts; p.table[1] = pre_items; }
    int f = first;
    for (int b = b0; b < b1; ++b) {
      const int n = parts(own_tiles(p, b));
      p.table[2 + 2 * b] = f;
      p.table[3 + 2 * b] = n;
      f += n;
    }
  }
  const int n_items = pre_items + unit * all, per = (n_items + 7) / 8, x = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per || x >= n_items) return false;
  if (x < pre_items) {
    it.b = -1;
    it.rt = x % p.pre_row_tiles;
    it.c = x / p.pre_row_tiles % pre_parts;
    it.hk = x / p.pre_row_tiles / pre_parts;
    it.n = pre_parts;
    it.slot = x;
    return true;
  }
  const int y = x - pre_items, part = y / unit;      // parts before it, over all sequences
  if (part >= first && part < first + mine) {
    for (int b = b0; b < b1; ++b) {
      const int n = parts(own_tiles(p, b));
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
  const int z = y - found[1] * unit;
  it.b = found[0];
  it.n = found[2];
  it.rt = p.own_row_tiles - 1 - z % p.own_row_tiles;
  it.c = z / p.own_row_tiles % it.n;
  it.hk = z / p.own_row_tiles / it.n;
  // partial results lie by sequence, head, part and row tile as the merge counts them; one item alone needs none
  it.slot = (it.n == 1 && !p.pooled) ? -1 : (int64_t)found[1] * unit + (it.hk * it.n + it.c) * p.own_row_tiles + it.rt;
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

template <class T, int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2)))
void dbsp_cache_attn_kernel(const dbsp_cache_attn_params p) {
  using L = Lay<D>;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[4 * L::TILE];      // [buffer][K, V]
  const uint32_t lds_base = (uint32_t)(uintptr_t)(LDS_PTR(unsigned char))lds;
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l = threadIdx.x & 63, r = l & 31, g = l >> 5;
  Item it;
  if (!find_item(p, it)) return;
  const int b = __builtin_amdgcn_readfirstlane(it.b), hk = __builtin_amdgcn_readfirstlane(it.hk), rt = __builtin_amdgcn_readfirstlane(it.rt);
  const bool own = b >= 0;
  const int len = own ? len_of(p, b) : 0, q_len = own ? q_len_of(p, b) : 0;
  const int rows = (own ? p.Nq : p.B * p.Nq) * p.G, row0 = rt * kCacheRows;
  const int base = len - q_len + 1;        // causal: query t sees the first base + t own keys
  // keys of this row tile: the prefix's (where it is not pooled, or the item is one of it), then own ones
  const int pre_tiles = (own && p.pooled) ? 0 : p.pre_tiles;
  int seen = len;
  if (own) {
    if (row0 / p.G >= q_len) return;       // no query here: its rows stay as they are
    if (p.causal) seen = max(0, min(len, base + min(q_len - 1, (row0 + kCacheRows - 1) / p.G)));
  }
  const int n_all = own ? own_tiles(p, b) : p.pre_tiles, per = (n_all + it.n - 1) / it.n;
  const int n_here = pre_tiles + tiles_of(seen);
  const int t0 = __builtin_amdgcn_readfirstlane(min(it.c * per, n_here)), t1 = __builtin_amdgcn_readfirstlane(min((it.c + 1) * per, n_here));

  // this lane's query
  const int row = row0 + 32 * w + r;
  const Row at = row_of(p, b, min(row, rows - 1));
  const bool valid = row < rows && at.t < (own ? q_len : q_len_of(p, at.b));
  const bool active = __builtin_amdgcn_ballot_w64(valid) != 0;
  const int h = hk * p.G + at.g;
  const int limit = p.causal ? max(0, min(len, base + at.t)) : len;       // own keys that it sees
  // a tile whose keys all of the wave's queries see needs no mask
  int all_see = valid ? limit : INT_MAX;
  for (int s = 16; s > 0; s >>= 1) all_see = min(all_see, __shfl_xor(all_see, s));
  all_see = __builtin_amdgcn_readfirstlane(all_see);
  u32x4 q[L::KS];
  {
    const uint16_t* src = p.q + at.b * p.q_sb + h * p.q_sh + at.t * p.q_st;
#pragma unroll
    for (int ks = 0; ks < L::KS; ++ks) q[ks] = *reinterpret_cast<const u32x4*>(src + 16 * ks + 8 * g);
  }

  // copies: this wave moves rows 16 w .. 16 w + 15 of a tile
  const int row_in = l / L::NCH, pch = l % L::NCH;
  auto copy_tile = [&](int t, int buf) __attribute__((always_inline)) {
    const bool pre = t < pre_tiles;
    const int tok = (pre ? t : t - pre_tiles) * kCacheKeys;
    const int there = (pre ? p.P : len) - tok;             // rows of the tile that hold keys; the others repeat the last one
    const uint32_t kst = pre ? p.pk_st : p.k_st, vst = pre ? p.pv_st : p.v_st;
    const unsigned char* kb = reinterpret_cast<const unsigned char*>(pre ? p.pk + hk * p.pk_sh : p.k + b * p.k_sb + hk * p.k_sh) + (int64_t)tok * kst;
    const unsigned char* vb = reinterpret_cast<const unsigned char*>(pre ? p.pv + hk * p.pv_sh : p.v + b * p.v_sb + hk * p.v_sh) + (int64_t)tok * vst;
    const uint32_t dst = lds_base + buf * 2 * L::TILE + 16 * w * L::ROWB;
#pragma unroll
    for (int x = 0; x < L::COPIES; ++x) {
      const int in = x * L::RPC + row_in, from = min(16 * w + in, there - 1);
      copy_row16(kb, from * kst + ((pch ^ L::k_swz(in)) << 4), dst + x * 1024);
      copy_row16(vb, from * vst + ((pch ^ L::v_swz(in)) << 4), dst + L::TILE + x * 1024);
    }
  };
  // operand reads, as in attn_fwd.hip
  uint32_t k_rd[L::KS], v_rd[L::DT];
#pragma unroll
  for (int ks = 0; ks < L::KS; ++ks) k_rd[ks] = lds_base + r * L::ROWB + (((2 * ks + g) ^ L::k_swz(r)) << 4);
  {
    const int hh = (l >> 4) & 1, key = 4 * g + ((l & 15) >> 2), a4 = l & 3;
#pragma unroll
    for (int dt = 0; dt < L::DT; ++dt)
      v_rd[dt] = lds_base + L::TILE + key * L::ROWB + ((((4 * dt) ^ L::v_swz(key)) + 2 * hh + (a4 >> 1)) << 4) + (a4 & 1) * 8;
  }

  f32x16 o[L::DT];
#pragma unroll
  for (int dt = 0; dt < L::DT; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[dt][e] = 0.f;
  // the running max starts at the lowest finite value: scores of -inf then have probability 0 wherever they come
  float mc = -FLT_MAX, sum = 0.f;          // max * scale_log2
  const float c = p.scale_log2;

  auto tile = [&](int t, int buf) __attribute__((always_inline)) {
    const uint32_t off = buf * 2 * L::TILE;
    f32x16 s[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[u][e] = 0.f;
#pragma unroll
      for (int ks = 0; ks < L::KS; ++ks)
        s[u] = T::mfma(*(LDS_PTR(u32x4))(uintptr_t)(k_rd[ks] + off + u * 32 * L::ROWB), q[ks], s[u]);
    }
    const bool pre = t < pre_tiles;
    const int tok = (pre ? t : t - pre_tiles) * kCacheKeys;
    if (tok + kCacheKeys > (pre ? p.P : all_see)) {
      const int left = (pre ? p.P : limit) - tok - 4 * g;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (32 * u + 8 * (e / 4) + e % 4 >= left) s[u][e] = -INFINITY;
    }
    if (p.scores && !pre && valid) {       // few rows: kept for the weights, which then need not read K again
      float* to = p.scores + (((int64_t)b * p.Hk + hk) * p.own_rows + row) * p.score_pitch + tok + 4 * g;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<f32x4*>(to + 32 * u + 8 * i) = f32x4{s[u][4 * i], s[u][4 * i + 1], s[u][4 * i + 2], s[u][4 * i + 3]};
    }
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, s[u][e]);
    top = max_xor32(top) * c;
    // The max is raised where probabilities could pass 2^8 (f32 sums and either type hold that without loss)
    if (__builtin_amdgcn_ballot_w64(top > mc + 8.f) != 0) {
      const float to = top > mc + 8.f ? top : mc, f = __builtin_amdgcn_exp2f(mc - to);
      mc = to;
      sum *= f;
#pragma unroll
      for (int dt = 0; dt < L::DT; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[dt][e] *= f;
    }
    u32x4 pb[4];                           // [16-key step]
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][e], c, -mc)), y = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][e + 1], c, -mc));
        s0 += x;
        s1 += y;
        pb[2 * u + e / 8][e % 8 / 2] = T::pack(x, y);
      }
    sum += s0 + s1;
#pragma unroll
    for (int st = 0; st < 4; ++st)
#pragma unroll
      for (int dt = 0; dt < L::DT; ++dt) {
        u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(uintptr_t)(v_rd[dt] + off + (16 * st) * L::ROWB)));
        u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(uintptr_t)(v_rd[dt] + off + (16 * st + 8) * L::ROWB)));
        o[dt] = T::mfma(u32x4{lo.x, lo.y, hi.x, hi.y}, pb[st], o[dt]);
      }
  };

  if (t0 < t1) copy_tile(t0, 0);
  for (int t = t0; t < t1; ++t) {
    const int buf = (t - t0) & 1;
    wait_all();                            // this wave's share of the tile has landed, and its reads of the other buffer are done
    __builtin_amdgcn_s_barrier();          // everybody's
    asm volatile("" ::: "memory");
    if (t + 1 < t1) copy_tile(t + 1, buf ^ 1);
    if (active) tile(t, buf);
  }

  sum = sum_xor32(sum);
  if (!valid) return;
  const bool none = __builtin_bit_cast(uint32_t, sum) == 0u;      // (by its bits: NaNs are not regarded in this file)
  const float inv = none ? 0.f : 1.f / sum, lse2 = none ? -INFINITY : mc + __builtin_amdgcn_logf(sum);
  if (it.slot >= 0) {
    const int64_t pr = part_row(p, own, it.slot) + 32 * w + r;
    float* to = p.part_o + pr * D + 4 * g;
#pragma unroll
    for (int dt = 0; dt < L::DT; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4*>(to + 32 * dt + 8 * i) = f32x4{o[dt][4 * i] * inv, o[dt][4 * i + 1] * inv, o[dt][4 * i + 2] * inv, o[dt][4 * i + 3] * inv};
    if (g == 0) p.part_lse[pr] = lse2;
    return;
  }
  uint16_t* to = p.o + at.b * p.o_sb + h * p.o_sh + at.t * p.o_st + 4 * g;
#pragma unroll
  for (int dt = 0; dt < L::DT; ++dt)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<u32x2*>(to + 32 * dt + 8 * i) = u32x2{T::pack(o[dt][4 * i] * inv, o[dt][4 * i + 1] * inv), T::pack(o[dt][4 * i + 2] * inv, o[dt][4 * i + 3] * inv)};
  if (g == 0) {
    const int64_t q_row = ((int64_t)at.b * p.H + h) * p.Nq + at.t;
    if (p.lse) p.lse[q_row] = lse2 * 0.69314718055994531f;
    if (p.weights) p.row_lse[q_row] = lse2;
  }
}

// Where the partial results of a query lie: parts of the pooled prefix, then parts of its own items.
struct Parts {
  int pre, own;
  int64_t pre_row, pre_step, own_row, own_step;        // rows of the first part, and from part to part
  __device__ __forceinline__ int64_t row(int i) const { return i < pre ? pre_row + i * pre_step : own_row + (i - pre) * own_step; }
};
__device__ __forceinline__ Parts parts_of(const dbsp_cache_attn_params& p, int b, int hk, int t, int g) {
  const int own = t * p.G + g, pre = (b * p.Nq + t) * p.G + g;
  Parts x;
  x.pre = p.table[0];
  x.own = p.table[3 + 2 * b];
  x.pre_row = part_row(p, false, (int64_t)hk * x.pre * p.pre_row_tiles + pre / kCacheRows) + pre % kCacheRows;
  x.pre_step = (int64_t)p.pre_row_tiles * kCacheRows;
  x.own_row = part_row(p, true, ((int64_t)p.table[2 + 2 * b] * p.Hk + (int64_t)hk * x.own) * p.own_row_tiles + own / kCacheRows) + own % kCacheRows;
  x.own_step = (int64_t)p.own_row_tiles * p.own_rows;
  return x;
}

// Behind the attention kernel.  The first p.merge_groups workgroups join partial results, D / 4 lanes a part of a row, four values
// each: WAYS of them a row, which take its parts in turn (rows are few where parts are many).  The others sum the
// weights from the scores that the attention kernel has kept, 1024 slots of a (sequence, KV head) each.
template <class T, int D, int WAYS>
__device__ __forceinline__ void merge_rows(const dbsp_cache_attn_params& p) {
  constexpr int LANES = D / 4, ROWS = 256 / LANES / WAYS, U = 4;
  const int unit = threadIdx.x / LANES, way = unit % WAYS, x = 4 * (threadIdx.x % LANES);
  const int64_t q_row = (int64_t)blockIdx.x * ROWS + unit / WAYS;      // [b][h][t]
  const bool there = q_row < (int64_t)p.B * p.H * p.Nq;
  const int t = there ? (int)(q_row % p.Nq) : 0, h = there ? (int)(q_row / p.Nq % p.H) : 0, b = there ? (int)(q_row / p.Nq / p.H) : 0;
  const Parts parts = parts_of(p, b, h / p.G, t, h % p.G);
  const int n = parts.pre + parts.own;
  const bool mine = there && t < q_len_of(p, b) && n > 1;      // (a part alone has been written as it is)
  float m = -FLT_MAX, sum = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int i0 = way; mine && i0 < n; i0 += U * WAYS) {
    float ls[U];
    f32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * WAYS;
      const int64_t row = parts.row(min(i, n - 1));
      ls[u] = i < n ? p.part_lse[row] : -INFINITY;
      v[u] = *reinterpret_cast<const f32x4*>(p.part_o + row * D + x);
    }
    float to = m;
#pragma unroll
    for (int u = 0; u < U; ++u) to = fmaxf(to, ls[u]);
    const float f = __builtin_amdgcn_exp2f(m - to);
    m = to;
    sum *= f;
    acc *= f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i0 + u * WAYS >= n) break;
      const float wgt = __builtin_amdgcn_exp2f(ls[u] - m);
      sum += wgt;
      acc += wgt * v[u];                   // (a part without a key has zeros)
    }
  }
  if constexpr (WAYS > 1) {
    static_assert(ROWS == 1, "a row a workgroup");
    __shared__ f32x4 accs[WAYS][LANES];
    __shared__ float ms[WAYS], sums[WAYS];
    accs[way][threadIdx.x % LANES] = acc;
    if (x == 0) {
      ms[way] = m;
      sums[way] = sum;
    }
    __syncthreads();
    if (way != 0) return;
#pragma unroll
    for (int y = 1; y < WAYS; ++y) m = fmaxf(m, ms[y]);
    sum = 0.f;
    acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int y = 0; y < WAYS; ++y) {
      const float f = __builtin_amdgcn_exp2f(ms[y] - m);
      sum += f * sums[y];
      acc += f * accs[y][threadIdx.x % LANES];
    }
  }
  if (!mine) return;
  const bool none = __builtin_bit_cast(uint32_t, sum) == 0u;
  acc *= none ? 0.f : 1.f / sum;
  *reinterpret_cast<u32x2*>(p.o + b * p.o_sb + h * p.o_sh + t * p.o_st + x) = u32x2{T::pack(acc.x, acc.y), T::pack(acc.z, acc.w)};
  if (x == 0) {
    const float lse2 = none ? -INFINITY : m + __builtin_amdgcn_logf(sum);
    if (p.lse) p.lse[q_row] = lse2 * 0.69314718055994531f;
    if (p.weights) p.row_lse[q_row] = lse2;
  }
}

constexpr int kSlots = 1024;       // a workgroup's, four a thread

__device__ __forceinline__ void sum_scores(const dbsp_cache_attn_params& p, int group) {
  __shared__ float row_lse[kScoreRows];
  const int per_pair = (p.cap + kSlots - 1) / kSlots, pair = group / per_pair, slot0 = group % per_pair * kSlots;
  const int b = pair / p.Hk, hk = pair % p.Hk, len = len_of(p, b), tid = threadIdx.x, w = tid >> 6, l = tid & 63;
  if (slot0 >= len) return;
  const int rows = q_len_of(p, b) * p.G, slot = slot0 + 4 * tid;
  float* to = p.weights + (int64_t)pair * p.cap + slot;
  f32x4 old;
#pragma unroll
  for (int i = 0; i < 4; ++i) old[i] = p.decay != 0.f && slot + i < len ? p.decay * to[i] : 0.f;
  // LSE of the group's rows, from their parts: a wave a row
  for (int r = w; r < rows; r += 4) {
    const int t = r / p.G, g = r % p.G;
    float ls = 0.f;
    if (p.split) {
      const Parts parts = parts_of(p, b, hk, t, g);
      const int n = parts.pre + parts.own;
      float m = -FLT_MAX, sum = 0.f;
      for (int i = l; i < n; i += 64) {
        const float x = p.part_lse[parts.row(i)], up = fmaxf(m, x);
        sum = sum * __builtin_amdgcn_exp2f(m - up) + __builtin_amdgcn_exp2f(x - up);
        m = up;
      }
      float top = m;
#pragma unroll
      for (int s = 32; s > 0; s >>= 1) top = fmaxf(top, __shfl_xor(top, s));
      sum *= __builtin_amdgcn_exp2f(m - top);
#pragma unroll
      for (int s = 32; s > 0; s >>= 1) sum += __shfl_xor(sum, s);
      ls = __builtin_bit_cast(uint32_t, sum) == 0u ? -INFINITY : top + __builtin_amdgcn_logf(sum);
      if (n == 1) ls = p.row_lse[((int64_t)b * p.H + hk * p.G + g) * p.Nq + t];
    } else {
      ls = p.row_lse[((int64_t)b * p.H + hk * p.G + g) * p.Nq + t];
    }
    if (__builtin_bit_cast(uint32_t, ls) == 0xff800000u) ls = INFINITY;      // a row without a key: probabilities of 0
    if (l == 0) row_lse[r] = ls;
  }
  __syncthreads();
  if (slot >= len) return;
  const float* s = p.scores + (int64_t)pair * p.own_rows * p.score_pitch + slot;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int r = 0; r < rows; ++r, s += p.score_pitch) {
    const f32x4 x = *reinterpret_cast<const f32x4*>(s);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] += __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], p.scale_log2, -row_lse[r]));
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (slot + i < len) to[i] = old[i] + acc[i];
}

template <class T, int D, int WAYS>
__global__ __launch_bounds__(256) void dbsp_cache_finish_kernel(const dbsp_cache_attn_params p) {
  if ((int)blockIdx.x < p.merge_groups) merge_rows<T, D, WAYS>(p);
  else sum_scores(p, blockIdx.x - p.merge_groups);
}

// The own keys' weights: a workgroup has 128 keys of a (sequence, KV head), 32 a wave with K as an operand in registers, and
// goes over the sequence's rows, 64 at a time by way of the LDS.
template <class T, int D>
__global__ __launch_bounds__(256) void dbsp_cache_weights_kernel(const dbsp_cache_attn_params p) {
  using L = Lay<D>;
  constexpr int RT = 64, PER = RT * L::NCH / 256;      // 16-byte chunks of a row tile that a thread moves
  __shared__ __attribute__((aligned(1024))) unsigned char lds[RT * L::ROWB];
  __shared__ float row_lse[RT];
  __shared__ int row_limit[RT];
  const uint32_t lds_base = (uint32_t)(uintptr_t)(LDS_PTR(unsigned char))lds;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63, r = l & 31, g = l >> 5;
  const int b = blockIdx.x / p.Hk, hk = blockIdx.x % p.Hk;
  const int len = len_of(p, b), q_len = q_len_of(p, b), key0 = blockIdx.y * 128;
  if (key0 >= len) return;
  const int rows = q_len * p.G;
  // causal: the first query that sees key0
  const int base = len - q_len + 1, t_first = p.causal ? max(0, key0 + 1 - base) : 0;
  const int mykey0 = key0 + 32 * w;
  u32x4 k[L::KS];
  {
    const unsigned char* src = reinterpret_cast<const unsigned char*>(p.k + b * p.k_sb + hk * p.k_sh) + (int64_t)min(mykey0 + r, len - 1) * p.k_st;
#pragma unroll
    for (int ks = 0; ks < L::KS; ++ks) k[ks] = *reinterpret_cast<const u32x4*>(src + 32 * ks + 16 * g);
  }
  float acc[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) acc[e] = 0.f;
  const float c = p.scale_log2;
  for (int r0 = t_first * p.G / RT * RT; r0 < rows; r0 += RT) {
    __syncthreads();
#pragma unroll
    for (int y = 0; y < PER; ++y) {
      const int i = (y * 256 + tid) / L::NCH, ch = tid % L::NCH;
      const Row at = row_of(p, b, r0 + i);
      u32x4 v = {0u, 0u, 0u, 0u};          // (rows that are not there: no NaN may come of them)
      if (r0 + i < rows) v = *reinterpret_cast<const u32x4*>(p.q + b * p.q_sb + (hk * p.G + at.g) * p.q_sh + at.t * p.q_st + 8 * ch);
      *(LDS_PTR(u32x4))(uintptr_t)(lds_base + i * L::ROWB + ((ch ^ L::k_swz(i)) << 4)) = v;
    }
    if (tid < RT) {
      const Row at = row_of(p, b, r0 + tid);
      float ls = INFINITY;                 // a row without a key, or none: probabilities of 0
      if (r0 + tid < rows) {
        ls = p.row_lse[((int64_t)b * p.H + hk * p.G + at.g) * p.Nq + at.t];
        if (__builtin_bit_cast(uint32_t, ls) == 0xff800000u) ls = INFINITY;
      }
      row_lse[tid] = ls;
      row_limit[tid] = p.causal ? base + at.t : len;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < RT / 32; ++u) {
      f32x16 s;
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
      for (int ks = 0; ks < L::KS; ++ks)
        s = T::mfma(k[ks], *(LDS_PTR(u32x4))(uintptr_t)(lds_base + (32 * u + r) * L::ROWB + (((2 * ks + g) ^ L::k_swz(r)) << 4)), s);
      const float ls = row_lse[32 * u + r];
      const int left = row_limit[32 * u + r] - mykey0 - 4 * g;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], c, -ls));
        acc[e] += 8 * (e / 4) + e % 4 < left ? x : 0.f;
      }
    }
  }
#pragma unroll
  for (int e = 0; e < 16; ++e)
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) acc[e] += __shfl_xor(acc[e], s);
  float* to = p.weights + (int64_t)blockIdx.x * p.cap;
  // lane e of each half stores its key e
  float mine = 0.f;
#pragma unroll
  for (int e = 0; e < 16; ++e) mine = r == e ? acc[e] : mine;
  const int key = mykey0 + 8 * (r / 4) + 4 * g + r % 4;
  if (r < 16 && key < len) to[key] = (p.decay == 0.f ? 0.f : p.decay * to[key]) + mine;
}

template <class T, int D>
hipError_t launch(dbsp_cache_attn_params p, int grid, hipStream_t stream) {
  dbsp_cache_attn_kernel<T, D><<<grid, 256, 0, stream>>>(p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  constexpr int UNITS = 256 / (D / 4);
  const int64_t rows = (int64_t)p.B * p.H * p.Nq, sums = p.scores ? (int64_t)p.B * p.Hk * ((p.cap + kSlots - 1) / kSlots) : 0;
  const bool all_ways = rows <= kMergeRows;
  p.merge_groups = !p.split ? 0 : (int)(all_ways ? rows : (rows + UNITS - 1) / UNITS);
  if (p.merge_groups + sums > 0) {
    const unsigned groups = (unsigned)(p.merge_groups + sums);
    if (all_ways) dbsp_cache_finish_kernel<T, D, UNITS><<<groups, 256, 0, stream>>>(p);
    else dbsp_cache_finish_kernel<T, D, 1><<<groups, 256, 0, stream>>>(p);
    e = hipGetLastError();
  }
  if (e == hipSuccess && p.weights && !p.scores) {
    dbsp_cache_weights_kernel<T, D><<<dim3(p.B * p.Hk, (p.cap + 127) / 128), 256, 0, stream>>>(p);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

hipError_t dbsp_launch_cache_attn(const dbsp_cache_attn_params& p, int d, bool fp16, int grid, hipStream_t stream) {
  if (d == 64) return fp16 ? launch<Fp16, 64>(p, grid, stream) : launch<Bf16, 64>(p, grid, stream);
  return fp16 ? launch<Fp16, 128>(p, grid, stream) : launch<Bf16, 128>(p, grid, stream);
}
