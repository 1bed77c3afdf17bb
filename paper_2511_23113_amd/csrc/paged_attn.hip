// Attention of new tokens over a paged key/value cache.
//
// For query t of sequence b, head h of KV head hk = h / G, over the slots j < len_b (causal: j <= len_b - qlen_b + t) whose page is there:
//   s = scale q.k,  LSE = ln sum exp(s),  O = sum exp(s - LSE) v,
// in one pass with a running max and sum, and O = 0, LSE = -inf without a key.
//
// Rows and items.  The G heads of a group read the same keys: a row is a (token, head of the group) pair, and a workgroup has up to 32 of them
// (d = 64: 64), one token's most often.  An item is a row tile and a range of its tiles of 64 keys; lengths are known on the device only, so every
// wave works out from them how the launch is cut, about p.target items of equally many tiles.  Parts leave partial results that a second
// launch joins: LSE = log sum exp LSE_i, O = sum exp(LSE_i - LSE) O_i.
//
// A workgroup is four waves, which share the rows and have 16 keys of a tile each: a wave copies them into the LDS directly and reads nothing that
// another has copied, so no barrier couples the waves; their statistics are joined through the LDS at the end.  The pages of a tile's
// keys are copied there as well, a tile ahead of the keys, so that the table's latency is paid once.  Every lane forms the address of its own
// 16 bytes: a page may end anywhere.  Slots without a key, behind the length or of a page that is not there, are copied from a row of
// zeros, as what lies in their place could be infinite or a NaN.  Products are formed transposed, S^T = K Q^T and O^T = V^T P^T, with 16 x 16
// MFMAs: lane (n, g) of 16 x 4 has row n and keys 4 g .. 4 g + 3, and the packed probabilities are the second product's operand as they lie.
// Probabilities are rounded to the inputs' type for it, half a step of it relative to each; LSE's sums are of the f32 values.
#include <hip/hip_runtime.h>

#include "cache_attn.hpp"
#include "paged_params.hpp"

namespace {

// What slots without a key hold.
__device__ const u32x4 kZeros[16] = {};

// 16 bytes a lane from an address of its own to the LDS at dst + 16 * lane, and 4 bytes to dst + 4 * lane.
__device__ __forceinline__ void copy_lane16(uint64_t from, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(dst) : "memory");
}
__device__ __forceinline__ void copy_lane4(uint64_t from, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(from), "s"(dst) : "memory");
}

__device__ __forceinline__ int paged_len(const dbsp_paged_attn_params& p, int b) { return max(0, min(p.lens[b], p.cap)); }
__device__ __forceinline__ int paged_q_len(const dbsp_paged_attn_params& p, int b) { return p.q_lens ? max(0, min(p.q_lens[b], p.Nq)) : p.Nq; }
__device__ __forceinline__ int page_of(const dbsp_paged_attn_params& p, int slot) { return paged_quotient(slot, p.page_mul, p.page_shift); }

struct PagedItem {
  int b, hk, rt;         // sequence, KV head, row tile
  int c, n;              // part c of n
  int64_t slot;          // of its partial result, -1: none
};

// Which item this workgroup has; false: none.  Every wave works it out for itself, 64 sequences at a time.
__device__ __forceinline__ bool find_paged_item(const dbsp_paged_attn_params& p, PagedItem& it) {
  const int unit = p.Hk * p.row_tiles, die = blockIdx.x & 7, i = blockIdx.x >> 3, l = threadIdx.x & 63;
  if (!p.split) {
    const int n = p.B * unit, per = (n + 7) / 8, x = die * per + i;
    if (i >= per || x >= n) return false;
    it.rt = x % p.row_tiles;
    it.hk = x / p.row_tiles % p.Hk;
    it.b = x / p.row_tiles / p.Hk;
    it.c = 0;
    it.n = 1;
    it.slot = -1;
    return true;
  }
  auto tiles = [&](int b) { return b < p.B ? tiles_of(paged_len(p, b)) : 0; };
  const int first_tiles = tiles(l);
  int64_t total = 0;
  for (int b0 = 0; b0 < p.B; b0 += 64) total += __builtin_amdgcn_readlane(scan_wave(b0 == 0 ? first_tiles : tiles(b0 + l)), 63);
  total *= unit;
  // (of few tiles up to four an item as long as there are 256 of them, as every part costs the merge)
  const int chunk = (int)max(max((int64_t)1, min((int64_t)4, total / 256)), min((int64_t)(1 << 30), (total + p.target - 1) / p.target));
  auto parts = [&](int b, int tiles) { return b < p.B ? max(1, (tiles + chunk - 1) / chunk) : 0; };
  // parts of all sequences, and where those of each begin
  const bool writes = blockIdx.x == 0 && threadIdx.x < 64;
  int all = 0;
  for (int b0 = 0; b0 < p.B; b0 += 64) {
    const int b = b0 + l, n = parts(b, b0 == 0 ? first_tiles : tiles(b)), upto = scan_wave(n);
    if (writes && b < p.B) {
      p.table[2 * b] = all + upto - n;
      p.table[2 * b + 1] = n;
    }
    all += __builtin_amdgcn_readlane(upto, 63);
  }
  // a run of the items for every die
  const int64_t items = (int64_t)unit * all, from = items * die / 8;
  if (from + i >= items * (die + 1) / 8) return false;
  const int64_t y = from + i;
  const int part = (int)(y / unit);
  int before = 0;
  for (int b0 = 0; b0 < p.B; b0 += 64) {
    const int n = parts(b0 + l, b0 == 0 ? first_tiles : tiles(b0 + l)), upto = scan_wave(n), here = __builtin_amdgcn_readlane(upto, 63);
    if (part < before + here) {
      const int at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(part < before + upto));
      it.b = b0 + at;
      it.n = __builtin_amdgcn_readlane(n, at);
      const int first = before + __builtin_amdgcn_readlane(upto, at) - it.n;
      const int z = (int)(y - (int64_t)first * unit);
      it.rt = z % p.row_tiles;
      it.c = z / p.row_tiles % it.n;
      it.hk = z / p.row_tiles / it.n;
      it.slot = it.n == 1 ? -1 : (int64_t)first * unit + ((int64_t)it.hk * it.n + it.c) * p.row_tiles + it.rt;
      return true;
    }
    before += here;
  }
  return false;          // (not reached: part < all)
}

template <class T, int D, int NR>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2)))
void dbsp_paged_attn_kernel(const dbsp_paged_attn_params p) {
  using L = Lay<D>;
  constexpr int KS = D / 32, DT = D / 16, CH = D / 4, ROWS = 16 * NR;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[4 * L::TILE];      // [buffer][K, V]
  __shared__ int page_ids[4][2][64];
  PagedItem it;
  if (!find_paged_item(p, it)) return;
  const int b = __builtin_amdgcn_readfirstlane(it.b), hk = __builtin_amdgcn_readfirstlane(it.hk), rt = __builtin_amdgcn_readfirstlane(it.rt);
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l = threadIdx.x & 63, n = l & 15, g = l >> 4;
  const int len = paged_len(p, b), q_len = paged_q_len(p, b), rows = p.Nq * p.G, row0 = rt * ROWS, base = len - q_len + 1;
  if (row0 / p.G >= q_len) return;         // no query here: its rows stay as they are
  const int tiles = tiles_of(len), per = (tiles + it.n - 1) / it.n;
  const int t0 = __builtin_amdgcn_readfirstlane(min(it.c * per, tiles)), t1 = __builtin_amdgcn_readfirstlane(min((it.c + 1) * per, tiles));

  const uint32_t lds_base = (uint32_t)(uintptr_t)(LDS_PTR(unsigned char))lds;
  const uint32_t ids_base = (uint32_t)(uintptr_t)(LDS_PTR(int))&page_ids[w][0][0];
  const int32_t* const row_pages = p.pages + b * p.pages_stride;
  // lane l asks for the page of the wave's key l % 16 of tile t (past the end of the table: its last entry, which is not looked at)
  auto copy_ids = [&](int t) __attribute__((always_inline)) {
    const int slot = min(t, t1 - 1) * kPagedKeys + 16 * w + n;
    copy_lane4((uint64_t)(uintptr_t)(row_pages + min(page_of(p, slot), p.max_pages - 1)), ids_base + (t & 1) * 256);
  };
  if (t0 < t1) {
    copy_ids(t0);
    copy_ids(t0 + 1);
  }

  int limit[NR], all_see = INT_MAX;
  bool valid[NR];
  u32x4 q[NR][KS];
#pragma unroll
  for (int y = 0; y < NR; ++y) {
    const int row = row0 + 16 * y + n, in = min(row, rows - 1), tok = in / p.G, gh = in % p.G;
    valid[y] = row < rows && tok < q_len;
    limit[y] = p.causal ? max(0, min(len, base + tok)) : len;
    all_see = min(all_see, valid[y] ? limit[y] : INT_MAX);
    const uint16_t* src = p.q + b * p.q_sb + (hk * p.G + gh) * p.q_sh + tok * p.q_st;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) q[y][ks] = *reinterpret_cast<const u32x4*>(src + 32 * ks + 8 * g);
  }
  all_see = over_row(all_see, [](int x, int y) { return min(x, y); });
  all_see = __builtin_amdgcn_readfirstlane(all_see);
  // the queries are waited for here, in front of the copies, which the compiler does not count
#pragma unroll
  for (int y = 0; y < NR; ++y)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(q[y][ks]));

  const int row_in = l / L::NCH, pch = l % L::NCH;
  const uint64_t k_head = (uint64_t)(uintptr_t)(p.k + hk * p.k_sh), v_head = (uint64_t)(uintptr_t)(p.v + hk * p.v_sh);
  const uint64_t zeros = (uint64_t)(uintptr_t)kZeros + (pch << 4);
  // copies this wave's keys of tile t; which of them are there, a bit each
  auto copy_tile = [&](int t, int buf) __attribute__((always_inline)) {
    const uint32_t dst = lds_base + buf * 2 * L::TILE + 16 * w * L::ROWB, ids = ids_base + (t & 1) * 256;
    const int slot0 = t * kPagedKeys + 16 * w;
#pragma unroll
    for (int x = 0; x < L::COPIES; ++x) {
      const int in = x * L::RPC + row_in, slot = slot0 + in;
      const int page = *(LDS_PTR(int))(uintptr_t)(ids + 4 * in), at = slot - page_of(p, slot) * p.page_size;
      const bool there = slot < len && (unsigned)page < (unsigned)p.n_pages;
      const uint64_t k_at = k_head + (int64_t)page * p.k_sp + (int64_t)at * p.k_ss + ((pch ^ L::k_swz(in)) << 4);
      const uint64_t v_at = v_head + (int64_t)page * p.v_sp + (int64_t)at * p.v_ss + ((pch ^ L::v_swz(in)) << 4);
      copy_lane16(there ? k_at : zeros, dst + x * 1024);
      copy_lane16(there ? v_at : zeros, dst + L::TILE + x * 1024);
    }
    const int page = *(LDS_PTR(int))(uintptr_t)(ids + 4 * n);
    return (uint32_t)__builtin_amdgcn_ballot_w64(slot0 + n < len && (unsigned)page < (unsigned)p.n_pages) & 0xffffu;
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
  // rounding of a key that has most of its row's attention drops out; LSE is of `sum`.
  f32x4 o[NR][DT], rounded[NR];
  float mc[NR], sum[NR];                   // the max starts at the lowest finite value: scores of -inf then have probability 0
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

  uint32_t there = 0;
  if (t0 < t1) {
    wait_all();                            // the first two tiles' pages
    there = copy_tile(t0, 0);
  }
  for (int t = t0; t < t1; ++t) {
    const int buf = (t - t0) & 1;
    uint32_t there_next = 0;
    if (t + 1 < t1) {
      // the pages of tile t + 1 have landed (younger are the copies of tile t only), and what was read in its buffer has arrived
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * L::COPIES) : "memory");
      copy_ids(t + 2);
      there_next = copy_tile(t + 1, buf ^ 1);
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * L::COPIES + 1) : "memory");      // this tile has landed, the next one is under way
    } else {
      wait_all();
    }
    const uint32_t off = buf * 2 * L::TILE;
    const int key = t * kPagedKeys + 16 * w + 4 * g;
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
      if (there != 0xffffu || (t + 1) * kPagedKeys > all_see) {
        const int left = limit[y] - key;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (i >= left || !((there >> (4 * g + i)) & 1)) x[i] = -INFINITY;
      }
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
    there = there_next;
  }

  // the waves' results, up to 32 rows at a time: [wave][row][16-byte chunk of the head dim, by row swizzled]
  constexpr int AT = NR < 2 ? NR : 2;
  __shared__ float mcs[4][16 * AT], sums[4][16 * AT], rounds[4][16 * AT];
  f32x4* const os = reinterpret_cast<f32x4*>(lds);
#pragma unroll
  for (int y0 = 0; y0 < NR; y0 += AT) {
    __syncthreads();                       // everybody has read its last tile, or the rows before
#pragma unroll
    for (int z = 0; z < AT; ++z) {
      const int y = y0 + z;
      sum[y] += __shfl_xor(sum[y], 16);
      sum[y] += __shfl_xor(sum[y], 32);
      if (g == 0) {
        mcs[w][16 * z + n] = mc[y];
        sums[w][16 * z + n] = sum[y];
        rounds[w][16 * z + n] = rounded[y][0];
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) os[(w * 16 * AT + 16 * z + n) * CH + ((4 * dt + g) ^ n)] = o[y][dt];
    }
    __syncthreads();
#pragma unroll
    for (int z = 0; z < 16 * AT * CH / 256; ++z) {
      const int i = z * 256 + threadIdx.x, in = i / CH, ch = i % CH, row = row0 + 16 * y0 + in, tok = row / p.G;
      if (row >= rows || tok >= q_len) continue;
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
        acc += f * os[(x * 16 * AT + in) * CH + (ch ^ (in & 15))];
      }
      const bool none = __builtin_bit_cast(uint32_t, all) == 0u;      // (by its bits: NaNs are not regarded in this file)
      acc *= none ? 0.f : 1.f / all_rounded;
      const float lse2 = none ? -INFINITY : m + __builtin_amdgcn_logf(all);
      if (it.slot >= 0) {
        const int64_t pr = it.slot * p.own_rows + 16 * y0 + in;
        *reinterpret_cast<f32x4*>(p.part_o + pr * D + 4 * ch) = acc;
        if (ch == 0) p.part_lse[pr] = lse2;
      } else {
        const int h = hk * p.G + row % p.G;
        *reinterpret_cast<u32x2*>(p.o + b * p.o_sb + h * p.o_sh + tok * p.o_st + 4 * ch) = u32x2{T::pack_o(acc.x, acc.y), T::pack_o(acc.z, acc.w)};
        if (ch == 0 && p.lse) p.lse[((int64_t)b * p.H + h) * p.Nq + tok] = lse2 * 0.69314718055994531f;
      }
    }
  }
}

// Joins partial results, D / 4 lanes a part of a row, four values each: WAYS of them a row, which take its parts in turn.
template <class T, int D, int WAYS>
__global__ __launch_bounds__(256) void dbsp_paged_merge_kernel(const dbsp_paged_attn_params p, int tile_rows) {
  constexpr int LANES = D / 4, ROWS = 256 / LANES / WAYS, U = WAYS > 1 ? 8 : 4;
  const int unit = threadIdx.x / LANES, way = unit % WAYS, x = 4 * (threadIdx.x % LANES);
  const int64_t nth = (int64_t)blockIdx.x * ROWS + unit / WAYS;      // [b][h][t]
  const bool there = nth < (int64_t)p.B * p.H * p.Nq;
  const int t = there ? (int)(nth % p.Nq) : 0, h = there ? (int)(nth / p.Nq % p.H) : 0, b = there ? (int)(nth / p.Nq / p.H) : 0;
  const int first = p.table[2 * b], n = p.table[2 * b + 1], row = t * p.G + h % p.G;
  const bool mine = there && t < paged_q_len(p, b) && n > 1;      // (a part alone has been written as it is)
  const int64_t step = (int64_t)p.row_tiles * p.own_rows;
  const int64_t at = ((int64_t)first * p.Hk * p.row_tiles + (int64_t)(h / p.G) * n * p.row_tiles + row / tile_rows) * p.own_rows + row % tile_rows;
  float m = -FLT_MAX, sum = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int i0 = way; mine && i0 < n; i0 += U * WAYS) {
    float ls[U];
    f32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * WAYS;
      const int64_t pr = at + min(i, n - 1) * step;
      ls[u] = i < n ? p.part_lse[pr] : -INFINITY;
      v[u] = *reinterpret_cast<const f32x4*>(p.part_o + pr * D + x);
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
  if (x == 0 && p.lse) p.lse[((int64_t)b * p.H + h) * p.Nq + t] = (none ? -INFINITY : m + __builtin_amdgcn_logf(sum)) * 0.69314718055994531f;
}

template <class T, int D>
hipError_t launch(const dbsp_paged_attn_params& p, int grid, hipStream_t stream) {
  const int tile_rows = paged_tile_rows((int64_t)p.Nq * p.G, D);
  if (tile_rows == 16) dbsp_paged_attn_kernel<T, D, 1><<<grid, 256, 0, stream>>>(p);
  else if (tile_rows == 32) dbsp_paged_attn_kernel<T, D, 2><<<grid, 256, 0, stream>>>(p);
  else if constexpr (D == 64) dbsp_paged_attn_kernel<T, D, 4><<<grid, 256, 0, stream>>>(p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.merge_groups == 0) return e;
  if (p.merge_by_row) dbsp_paged_merge_kernel<T, D, 256 / (D / 4)><<<p.merge_groups, 256, 0, stream>>>(p, tile_rows);
  else dbsp_paged_merge_kernel<T, D, 1><<<p.merge_groups, 256, 0, stream>>>(p, tile_rows);
  return hipGetLastError();
}

}  // namespace

hipError_t dbsp_launch_paged_attn(const dbsp_paged_attn_params& p, int d, bool fp16, int grid, hipStream_t stream) {
  if (d == 64) return fp16 ? launch<Fp16, 64>(p, grid, stream) : launch<Bf16, 64>(p, grid, stream);
  return fp16 ? launch<Fp16, 128>(p, grid, stream) : launch<Bf16, 128>(p, grid, stream);
}
