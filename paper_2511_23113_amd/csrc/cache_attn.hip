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
// works out from them how the launch is cut: about p.target items of equally many tiles, each sequence into equal parts.
// Parts leave partial results (O, and LSE to base 2, in f32) that a second launch joins: LSE = log sum exp LSE_i,
// O = sum exp(LSE_i - LSE) O_i.  Items of the same keys lie next to each other and on the same die (workgroup number mod 8).
//
// A workgroup is four waves.  Tiles of 64 keys go to the LDS directly (global_load_lds_dwordx4), two in turn.  Products are formed
// transposed, S^T = K Q^T and O^T = V^T P^T: a lane holds a query, the packed probabilities are the second product's operand as they
// lie, and V^T comes from transposing LDS reads (the layouts are those of attn_fwd.hip).  Up to 32 rows are given to all waves, which
// share the keys (few_rows); more are dealt to them, 32 each (the kernel).  Probabilities are rounded to the inputs' type for the second
// product, as they must be for the matrix pipe: half a step of it relative to each; LSE's sums are of the f32 values.
//
// Bound by reading K and V once.  32 sequences of 32 heads on 8 KV heads over 4400 own keys each (577 MB): 120 us, 4.8 TB/s, where a large copy
// reaches 5.0; 8 KV heads over 123,000 keys (506 MB) 95 us, 5.3 TB/s; without any of its arithmetic the kernel takes 3 to 8 % less.
// 64 sequences of 40 heads on 8 behind 16,384 shared keys, 605 MB in all: 122 us, 5.0 TB/s; there the prefix's rows fill 3 tiles of 128 a KV
// head, bound by the matrix pipe, and run beside own keys on every die (20 us more with the prefix on the first dies alone).
#include <hip/hip_runtime.h>

#include <type_traits>

#include "cache_attn.hpp"

namespace {

// Where an item's rows and keys are: sequence (-1: the pooled prefix), KV head, first row and rows of the sequence, used slots, new
// tokens, tiles of the prefix in front of the own ones, and the item's tiles.
struct Span { int b, hk, row0, rows, len, q_len, pre_tiles, t0, t1; };

// Row tiles of at most 16 NR rows, the form for single tokens: bound by the stream of K and V (with 32 rows a wave, three of the four
// waves idle, single rows over 4400 keys took 134 us where they take 120).  The keys of a tile are dealt to the
// waves, 16 each, with 16 x 16 MFMAs: lane (n, g) of 16 x 4 has row n and keys 4 g .. 4 g + 3, and the packed probabilities
// are the second product's operand again.  A wave reads what it has copied itself, so no barrier couples the waves; each has
// statistics of its own, against which it forms its probabilities as they stand (the max is raised where one passes kRaiseAt), and
// the four are joined through the LDS at the end.
template <class T, int D, int NR>
__device__ __forceinline__ void few_rows(const dbsp_cache_attn_params& p, const Item& it, const Span& s, unsigned char* lds) {
  using L = Lay<D>;
  constexpr int KS = D / 32, DT = D / 16, CH = D / 4;
  const uint32_t lds_base = (uint32_t)(uintptr_t)(LDS_PTR(unsigned char))lds;
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l = threadIdx.x & 63, n = l & 15, g = l >> 4;
  const bool own = s.b >= 0;
  const int base = s.len - s.q_len + 1;
  int limit[NR], all_see = INT_MAX;
  bool valid[NR];
  u32x4 q[NR][KS];
#pragma unroll
  for (int y = 0; y < NR; ++y) {
    const int row = s.row0 + 16 * y + n;
    const Row at = row_of(p, s.b, min(row, s.rows - 1));
    valid[y] = row < s.rows && at.t < (own ? s.q_len : q_len_of(p, at.b));
    limit[y] = p.causal ? max(0, min(s.len, base + at.t)) : s.len;
    all_see = min(all_see, valid[y] ? limit[y] : INT_MAX);
    const uint16_t* src = p.q + at.b * p.q_sb + (s.hk * p.G + at.g) * p.q_sh + at.t * p.q_st;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) q[y][ks] = *reinterpret_cast<const u32x4*>(src + 32 * ks + 8 * g);
  }
  all_see = over_row(all_see, [](int x, int y) { return min(x, y); });
  all_see = __builtin_amdgcn_readfirstlane(all_see);

  const int row_in = l / L::NCH, pch = l % L::NCH;
  auto copy_tile = [&](int t, int buf) __attribute__((always_inline)) {
    const bool pre = t < s.pre_tiles;
    const int tok = (pre ? t : t - s.pre_tiles) * kCacheKeys, there = (pre ? p.P : s.len) - tok;
    const uint32_t kst = pre ? p.pk_st : p.k_st, vst = pre ? p.pv_st : p.v_st;
    const unsigned char* kb = reinterpret_cast<const unsigned char*>(pre ? p.pk + s.hk * p.pk_sh : p.k + s.b * p.k_sb + s.hk * p.k_sh) + (int64_t)tok * kst;
    const unsigned char* vb = reinterpret_cast<const unsigned char*>(pre ? p.pv + s.hk * p.pv_sh : p.v + s.b * p.v_sb + s.hk * p.v_sh) + (int64_t)tok * vst;
    const uint32_t dst = lds_base + buf * 2 * L::TILE + 16 * w * L::ROWB;
#pragma unroll
    for (int x = 0; x < L::COPIES; ++x) {
      const int in = x * L::RPC + row_in, from = min(16 * w + in, there - 1);
      copy_row16(kb, from * kst + ((pch ^ L::k_swz(in)) << 4), dst + x * 1024);
      copy_row16(vb, from * vst + ((pch ^ L::v_swz(in)) << 4), dst + L::TILE + x * 1024);
    }
  };
  // operand reads: K rows n with 16-byte chunk 4 ks + g; of V^T, lane 4 j + a of 16 has the address of four values of key j
  const uint32_t mine = lds_base + 16 * w * L::ROWB;
  uint32_t k_rd[KS], v_rd[DT];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) k_rd[ks] = mine + n * L::ROWB + (((4 * ks + g) ^ L::k_swz(n)) << 4);
  {
    const int key = 4 * g + (n >> 2), a4 = n & 3;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) v_rd[dt] = mine + L::TILE + key * L::ROWB + (((2 * dt + (a4 >> 1)) ^ L::v_swz(key)) << 4) + (a4 & 1) * 8;
  }
  // rounded[y]: sums of the rounded probabilities, by one more MFMA against ones, all four alike.  O is divided by them, so that the
  // rounding of a key that has most of its row's attention drops out (fp16, 30 rows: 2-norm error 3.2e-4 by the others' sum); LSE is of `sum`.
  f32x4 o[NR][DT], rounded[NR];
  float mc[NR], sum[NR];
#pragma unroll
  for (int y = 0; y < NR; ++y) {
    mc[y] = -FLT_MAX;
    sum[y] = 0.f;
    rounded[y] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[y][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const u32x2 ones = {T::pack(1.f, 1.f), T::pack(1.f, 1.f)};
  const float c = p.scale_log2;
  float* scores = p.scores && own ? p.scores + ((int64_t)s.b * p.Hk + s.hk) * p.own_rows * p.score_pitch : nullptr;

  if (s.t0 < s.t1) copy_tile(s.t0, 0);
  for (int t = s.t0; t < s.t1; ++t) {
    const int buf = (t - s.t0) & 1;
    if (t + 1 < s.t1) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");         // what was read there has arrived
      copy_tile(t + 1, buf ^ 1);
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * L::COPIES) : "memory");      // this tile has landed, the next one is under way
    } else {
      wait_all();
    }
    const uint32_t off = buf * 2 * L::TILE;
    const bool pre = t < s.pre_tiles;
    const int tok = (pre ? t : t - s.pre_tiles) * kCacheKeys, key = tok + 16 * w + 4 * g;
    u32x4 kf[KS];
    u32x2 vf[DT], pb[NR];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) kf[ks] = *(LDS_PTR(u32x4))(uintptr_t)(k_rd[ks] + off);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) vf[dt] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(uintptr_t)(v_rd[dt] + off)));
#pragma unroll
    for (int y = 0; y < NR; ++y) {
      f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) x = T::mfma32(kf[ks], q[y][ks], x);
      if (tok + kCacheKeys > (pre ? p.P : all_see)) {
        const int left = (pre ? p.P : limit[y]) - key;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (i >= left) x[i] = -INFINITY;
      }
      if (scores && !pre && valid[y]) *reinterpret_cast<f32x4*>(scores + (int64_t)(s.row0 + 16 * y + n) * p.score_pitch + key) = x;
      float pr[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) pr[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], c, -mc[y]));
      const float top4 = fmaxf(fmaxf(pr[0], pr[1]), fmaxf(pr[2], pr[3]));
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(top4 > kRaiseAt) != 0, 0)) {
        float top = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float to = fmaxf(mc[y], top * c), f = __builtin_amdgcn_exp2f(mc[y] - to);
        mc[y] = to;
        sum[y] *= f;
        rounded[y] *= f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[y][dt] *= f;
#pragma unroll
        for (int i = 0; i < 4; ++i) pr[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], c, -to));
      }
      sum[y] += (pr[0] + pr[1]) + (pr[2] + pr[3]);
      pb[y] = u32x2{T::pack(pr[0], pr[1]), T::pack(pr[2], pr[3])};
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int y = 0; y < NR; ++y) o[y][dt] = T::mfma16(vf[dt], pb[y], o[y][dt]);
#pragma unroll
    for (int y = 0; y < NR; ++y) rounded[y] = T::mfma16(ones, pb[y], rounded[y]);
  }

  // the waves' results: [wave][row][16-byte chunk of the head dim, by row swizzled]
  __shared__ float mcs[4][16 * NR], sums[4][16 * NR], rounds[4][16 * NR];
  __syncthreads();                         // everybody has read its last tile
  f32x4* const os = reinterpret_cast<f32x4*>(lds);
#pragma unroll
  for (int y = 0; y < NR; ++y) {
    sum[y] += __shfl_xor(sum[y], 16);
    sum[y] += __shfl_xor(sum[y], 32);
    if (g == 0) {
      mcs[w][16 * y + n] = mc[y];
      sums[w][16 * y + n] = sum[y];
      rounds[w][16 * y + n] = rounded[y][0];
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) os[(w * 16 * NR + 16 * y + n) * CH + ((4 * dt + g) ^ n)] = o[y][dt];
  }
  __syncthreads();
#pragma unroll
  for (int z = 0; z < 16 * NR * CH / 256; ++z) {
    const int i = z * 256 + threadIdx.x, in = i / CH, ch = i % CH, row = s.row0 + in;
    if (row >= s.rows) continue;
    const Row at = row_of(p, s.b, row);
    if (at.t >= (own ? s.q_len : q_len_of(p, at.b))) continue;
    float m = mcs[0][in];
#pragma unroll
    for (int x = 1; x < 4; ++x) m = fmaxf(m, mcs[x][in]);
    float all = 0.f, all_rounded = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const float f = __builtin_amdgcn_exp2f(mcs[x][in] - m);
      all += f * sums[x][in];
      all_rounded += f * rounds[x][in];
      acc += f * os[(x * 16 * NR + in) * CH + (ch ^ (in & 15))];
    }
    const bool none = __builtin_bit_cast(uint32_t, all) == 0u;
    acc *= none ? 0.f : 1.f / all_rounded;
    const float lse2 = none ? -INFINITY : m + __builtin_amdgcn_logf(all);
    const int h = s.hk * p.G + at.g;
    if (it.slot >= 0) {
      const int64_t pr = part_row(p, own, it.slot) + in;
      *reinterpret_cast<f32x4*>(p.part_o + pr * D + 4 * ch) = acc;
      if (ch == 0) p.part_lse[pr] = lse2;
    } else {
      *reinterpret_cast<u32x2*>(p.o + at.b * p.o_sb + h * p.o_sh + at.t * p.o_st + 4 * ch) = u32x2{T::pack_o(acc.x, acc.y), T::pack_o(acc.z, acc.w)};
      if (ch == 0) {
        const int64_t q_row = ((int64_t)at.b * p.H + h) * p.Nq + at.t;
        if (p.lse) p.lse[q_row] = lse2 * 0.69314718055994531f;
        if (p.weights) p.row_lse[q_row] = lse2;
      }
    }
  }
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

  const Span span{b, hk, row0, rows, len, q_len, pre_tiles, t0, t1};
  if (min(rows - row0, kCacheRows) <= 16) return few_rows<T, D, 1>(p, it, span, lds);
  if (min(rows - row0, kCacheRows) <= 32) return few_rows<T, D, 2>(p, it, span, lds);

  // this lane's query
  const int row = row0 + 32 * w + r;
  const Row at = row_of(p, b, min(row, rows - 1));
  const bool valid = row < rows && at.t < (own ? q_len : q_len_of(p, at.b));
  const bool active = __builtin_amdgcn_ballot_w64(valid) != 0;
  const int h = hk * p.G + at.g;
  const int limit = p.causal ? max(0, min(len, base + at.t)) : len;       // own keys that it sees
  // a tile whose keys all of the wave's queries see needs no mask
  int all_see = valid ? limit : INT_MAX;
  all_see = over_row(all_see, [](int x, int y) { return min(x, y); });
  all_see = min(all_see, __shfl_xor(all_see, 16));
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
  store_row<T, D>(p, it, o, at, h, 32 * w + r, g, none ? 0.f : 1.f / sum, none ? -INFINITY : mc + __builtin_amdgcn_logf(sum));
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
// weights from the scores that the attention kernel has kept, 1024 slots of a (sequence, KV head) each.  Bound by latencies: 6 us behind
// 384 rows of 9 parts and as many (sequence, head) pairs of 1500 keys, 9 us behind 96 rows of 205 parts.
template <class T, int D, int WAYS>
__device__ __forceinline__ void merge_rows(const dbsp_cache_attn_params& p) {
  constexpr int LANES = D / 4, ROWS = 256 / LANES / WAYS, U = WAYS > 1 ? 8 : 4;
  const int unit = threadIdx.x / LANES, way = unit % WAYS, x = 4 * (threadIdx.x % LANES);
  const int64_t nth = (int64_t)blockIdx.x * ROWS + unit / WAYS;
  Parts parts;
  int b, h, t;
  bool there;
  if (p.many) {      // the rows of the tiles that were cut
    const dbsp_cache_long_cut& cut = p.cut;
    const int z = (int)(nth / p.own_rows), in = (int)(nth % p.own_rows);
    Item it;
    there = z < cut.dies * cut.tail && long_row_tile(p, z / cut.tail, cut.whole + z % cut.tail, it);
    if (!there) it = {0, 0, 0, 0, 0, 0};
    const int row = max(0, it.rt * kLongRows - p.row_shift + in);
    there = there && it.rt * kLongRows + in >= p.row_shift;
    b = it.b;
    t = row / p.G;
    h = it.hk * p.G + row % p.G;
    parts = {0, cut.k, 0, 0, (int64_t)z * cut.k * p.own_rows + in, p.own_rows};
  } else {
    there = nth < (int64_t)p.B * p.H * p.Nq;      // [b][h][t]
    t = there ? (int)(nth % p.Nq) : 0;
    h = there ? (int)(nth / p.Nq % p.H) : 0;
    b = there ? (int)(nth / p.Nq / p.H) : 0;
    parts = parts_of(p, b, h / p.G, t, h % p.G);
  }
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
  *reinterpret_cast<u32x2*>(p.o + b * p.o_sb + h * p.o_sh + t * p.o_st + x) = u32x2{T::pack_o(acc.x, acc.y), T::pack_o(acc.z, acc.w)};
  if (x == 0) {
    const int64_t q_row = ((int64_t)b * p.H + h) * p.Nq + t;
    const float lse2 = none ? -INFINITY : m + __builtin_amdgcn_logf(sum);
    if (p.lse) p.lse[q_row] = lse2 * 0.69314718055994531f;
    if (p.weights) p.row_lse[q_row] = lse2;
  }
}

__device__ __forceinline__ void sum_scores(const dbsp_cache_attn_params& p, int group) {
  __shared__ float row_lse[kScoreRows];
  const int per_pair = (p.cap + kScoreSlots - 1) / kScoreSlots, pair = group / per_pair, slot0 = group % per_pair * kScoreSlots;
  const int b = pair / p.Hk, hk = pair % p.Hk, len = len_of(p, b), tid = threadIdx.x;
  if (slot0 >= len) return;
  const int rows = q_len_of(p, b) * p.G, slot = slot0 + 4 * tid;
  float* to = p.weights + (int64_t)pair * p.cap + slot;
  f32x4 old;
#pragma unroll
  for (int i = 0; i < 4; ++i) old[i] = p.decay != 0.f && slot + i < len ? p.decay * to[i] : 0.f;
  // LSE of the group's rows, from their parts: 16 lanes a row
  const int lane = tid & 15;
  for (int r = tid >> 4; r < rows; r += 16) {
    const int t = r / p.G, g = r % p.G;
    float ls = 0.f;
    Parts parts{0, 1, 0, 0, 0, 0};
    if (p.split) parts = parts_of(p, b, hk, t, g);
    const int n = parts.pre + parts.own;
    if (n > 1) {
      float m = -FLT_MAX, sum = 0.f;
      for (int i = lane; i < n; i += 16) {
        const float x = p.part_lse[parts.row(i)], up = fmaxf(m, x);
        sum = sum * __builtin_amdgcn_exp2f(m - up) + __builtin_amdgcn_exp2f(x - up);
        m = up;
      }
      const float top = over_row(m, [](float x, float y) { return fmaxf(x, y); });
      sum *= __builtin_amdgcn_exp2f(m - top);
      sum = over_row(sum, [](float x, float y) { return x + y; });
      ls = __builtin_bit_cast(uint32_t, sum) == 0u ? -INFINITY : top + __builtin_amdgcn_logf(sum);
    } else {
      ls = p.row_lse[((int64_t)b * p.H + hk * p.G + g) * p.Nq + t];
    }
    if (__builtin_bit_cast(uint32_t, ls) == 0xff800000u) ls = INFINITY;      // a row without a key: probabilities of 0
    if (lane == 0) row_lse[r] = ls;
  }
  __syncthreads();
  if (slot >= len) return;
  const float* s = p.scores + (int64_t)pair * p.own_rows * p.score_pitch + slot;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  constexpr int U = 4;
  for (int r = 0; r < rows; r += U, s += U * p.score_pitch) {
    f32x4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = *reinterpret_cast<const f32x4*>(s + (r + u < rows ? u : 0) * p.score_pitch);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float ls = r + u < rows ? row_lse[r + u] : INFINITY;      // (a row again: probabilities of 0)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] += __builtin_amdgcn_exp2f(__builtin_fmaf(x[u][i], p.scale_log2, -ls));
    }
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

template <class T, int D>
hipError_t launch(const dbsp_cache_attn_params& p, int grid, hipStream_t stream) {
  hipError_t e;
  if (p.many) {
    e = dbsp_launch_cache_attn_long(p, D, std::is_same_v<T, Fp16>, grid, stream);
  } else {
    dbsp_cache_attn_kernel<T, D><<<grid, 256, 0, stream>>>(p);
    e = hipGetLastError();
  }
  if (e != hipSuccess) return e;
  if (const int groups = p.merge_groups + p.sum_groups; groups > 0) {
    if (p.merge_by_row) dbsp_cache_finish_kernel<T, D, 256 / (D / 4)><<<groups, 256, 0, stream>>>(p);
    else dbsp_cache_finish_kernel<T, D, 1><<<groups, 256, 0, stream>>>(p);
    e = hipGetLastError();
  }
  if (e == hipSuccess && p.weights && !p.scores) e = dbsp_launch_cache_weights(p, D, std::is_same_v<T, Fp16>, stream);
  return e;
}

}  // namespace

hipError_t dbsp_launch_cache_attn(const dbsp_cache_attn_params& p, int d, bool fp16, int grid, hipStream_t stream) {
  if (d == 64) return fp16 ? launch<Fp16, 64>(p, grid, stream) : launch<Bf16, 64>(p, grid, stream);
  return fp16 ? launch<Fp16, 128>(p, grid, stream) : launch<Bf16, 128>(p, grid, stream);
}
