// Attention of new tokens over a paged key/value cache.
//
// For query t of sequence b, head h of KV head hk = h / G, over the slots j < len_b (causal: j <= len_b - qlen_b + t) whose page is there:
//   s = scale q.k,  LSE = ln sum exp(s),  O = sum exp(s - LSE) v,
// in one pass with a running max and sum, and O = 0, LSE = -inf without a key.
//
// Rows and runs.  The G heads of a group read the same keys: a row is a (token, head of the group) pair, and a row tile has up to 64 of them,
// one token's most often.  The tiles of 64 keys of all row tiles, one sequence and KV head behind the other, are one list, of which
// every workgroup has a run of equally many: as many workgroups as the chip holds at a time begin and end together, whatever the
// lengths, which are known on the device only.  A row tile that lies in one run is written as it is; the others leave a partial result for
// every run, which a second launch joins: LSE = log sum exp LSE_i, O = sum exp(LSE_i - LSE) O_i.  Where there is little to read, or row tiles are
// short, they are cut into parts for themselves or not at all (see kPagedLong).
//
// A workgroup is four waves, which share the rows and have 16 keys of a tile each: a wave copies them into the LDS directly and reads nothing that
// another has copied, so no barrier couples the waves; their statistics are joined through the LDS at the end.  The pages of a tile's
// keys are copied there as well, a tile ahead of the keys, so that the table's latency is paid once.  Every lane forms the address of its own
// 16 bytes: a page may end anywhere.  Slots without a key, behind the length or of a page that is not there, are copied from a row of
// zeros, as what lies in their place could be infinite or a NaN.  Products are formed transposed, S^T = K Q^T and O^T = V^T P^T, with 16 x 16
// MFMAs: lane (n, g) of 16 x 4 has row n and keys 4 g .. 4 g + 3, and the packed probabilities are the second product's operand as they lie.
// For it each probability is the sum of two numbers of the inputs' type (see Halves), beside one another along the keys against V twice: an MFMA over
// 32 products takes as long as one over 16.  LSE's sums, which O is divided by, are of the f32 values.
//
// Bound by reading K and V once: 32 sequences of 40 heads on 8 KV heads, 880 to 4400 keys each (347 MB on average) 65 us and 4.8 for the merge; two
// sequences of some 111,000 keys and 4 KV heads (456 MB) 79 us, 5.8 TB/s, and 5.0.  Where there are few tiles a workgroup, by latencies: lengths,
// pages, first tile, some 4 us before anything is computed (24 sequences of 10 KV heads and 21 rows over 39 to 750 keys, 50 MB: 15.9 us and 4).
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

// Of a sequence that all lanes ask for, by way of the scalar cache: a vector load would be waited for with the copies that are under way.
__device__ __forceinline__ int scalar_load(const int32_t* from, int i) {
  return *reinterpret_cast<const __attribute__((address_space(4))) int32_t*>(reinterpret_cast<uintptr_t>(from + __builtin_amdgcn_readfirstlane(i)));
}
__device__ __forceinline__ int paged_len(const dbsp_paged_attn_params& p, int b) { return max(0, min(scalar_load(p.lens, b), p.cap)); }
__device__ __forceinline__ int paged_q_len(const dbsp_paged_attn_params& p, int b) { return p.q_lens ? max(0, min(scalar_load(p.q_lens, b), p.Nq)) : p.Nq; }
__device__ __forceinline__ int page_of(const dbsp_paged_attn_params& p, int slot) { return paged_quotient(slot, p.page_mul, p.page_shift); }

// Tiles that sequence b's row tiles have in the list: one where there is nothing to read, in which zeros are written.
__device__ __forceinline__ int listed_tiles(int len, int q_len) { return q_len > 0 ? max(1, tiles_of(len)) : 1; }

// A workgroup's run of the list: where it begins, and its length (0: it has none).
struct Run {
  int b, pair;           // sequence, and of its row tiles (KV head by KV head) which
  int t, left;           // tile of the row tile, tiles of the run
  int n;                 // number of the run
  int len, q_len;        // of the sequence
};

// Every wave works it out for itself: sums over blocks of 64 sequences, a block a lane (of more than 4096 sequences some multiple of 64), and then
// the sequences of the block that has the run, a sequence a lane.
__device__ __forceinline__ Run find_run(const dbsp_paged_attn_params& p) {
  const int l = threadIdx.x & 63, unit = p.Hk * p.row_tiles;
  Run run;
  run.t = run.left = 0;
  // number of the run that this workgroup has of so many: neighbouring ones on one die (workgroup number mod 8); false: it has none
  auto take = [&](unsigned count) {
    const unsigned per = (count + 7) / 8, i = blockIdx.x >> 3;
    run.n = (int)((blockIdx.x & 7) * per + i);
    return i < per && (unsigned)run.n < count;
  };
  auto alone = [&] {       // a row tile a workgroup
    run.b = (int)((unsigned)run.n / (unsigned)unit);
    run.pair = run.n - run.b * unit;
    run.len = paged_len(p, run.b);
    run.q_len = paged_q_len(p, run.b);
    run.left = listed_tiles(run.len, run.q_len);
  };
  if (p.whole) {
    if (take((unsigned)p.B * (unsigned)unit)) alone();
    return run;
  }
  // (lengths and new tokens are asked for at once: lanes without a sequence ask for the last one's, so that no branch stands between)
  const int32_t* const q_lens = p.q_lens ? p.q_lens : p.lens;
  auto get = [&](int b, int& len, int& q_len) __attribute__((always_inline)) {
    const int at = min(b, p.B - 1), as_given = p.lens[at], q_as_given = q_lens[at];
    len = max(0, min(as_given, p.cap));
    q_len = p.q_lens ? max(0, min(q_as_given, p.Nq)) : p.Nq;
    return b < p.B ? listed_tiles(len, q_len) : 0;
  };
  const int chunks = (p.B + 63) / 64, per_block = (chunks + 63) / 64;
  int len, q_len, tiles = get(l, len, q_len);
  // f(first sequence of 64, this lane's tiles), eight loads under way at a time
  auto over_chunks = [&](auto f) __attribute__((always_inline)) {
    f(0, tiles);
    for (int c0 = 1; c0 < chunks; c0 += 8) {
      int x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        int no_len, no_q_len;
        x[u] = get((c0 + u) * 64 + l, no_len, no_q_len);
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) f(c0 + u, x[u]);
    }
  };
  int sum = 0, longest = 0;
  over_chunks([&](int, int tiles) {
    sum += tiles;
    longest = max(longest, tiles);
  });
  const unsigned total = (unsigned)__builtin_amdgcn_readlane(scan_wave(sum), 63) * (unsigned)unit, row_tiles = (unsigned)p.B * (unsigned)unit;
  const bool parts = total < max(8 * p.slots, kPagedLong * row_tiles);
  const unsigned runs = total < kPagedEnds * row_tiles ? p.slots : p.runs;
  // (of few tiles up to four a part as long as there are 256 of them, as every part costs the merge; of many row tiles fewer parts, as each
  // has one that is not full: 128 pairs of 9 to 18 tiles 19.3 / 17.7 us)
  const unsigned full = p.slots - min(row_tiles / 2, p.slots / 2);
  const unsigned chunk = parts ? max(max(1u, min(4u, total / 256)), (total + full - 1) / full) : (total + runs - 1) / runs;
  // no row tile is cut where that leaves a workgroup four tiles more than a part at most, or ten in all: 512 pairs of 4 to 9 tiles 33.4 us cut
  // down to 7, 23.8 uncut
  if (parts && __builtin_amdgcn_ballot_w64(longest > max(kPagedWhole, (int)chunk + 4)) == 0) {
    if (blockIdx.x == 0 && threadIdx.x == 0) p.table[1] = 2;
    if (take(row_tiles)) alone();
    return run;
  }
  // what is counted: parts, or tiles of one KV head
  auto counted = [&](int tiles) { return parts ? (int)((tiles + chunk - 1) / chunk) : tiles; };
  int mine = 0;            // of block l
  over_chunks([&](int c, int tiles) {
    const int sum = __builtin_amdgcn_readlane(scan_wave(counted(tiles)), 63);
    mine += l == c / per_block ? sum : 0;
  });
  int upto = scan_wave(mine);
  if (!take(parts ? (unsigned)__builtin_amdgcn_readlane(upto, 63) * (unsigned)unit : (total + chunk - 1) / chunk)) return run;
  if (blockIdx.x == 0 && threadIdx.x < 64) {      // for the merge
    if (l == 0) {
      p.table[0] = (int)chunk;
      p.table[1] = parts;
    }
    int before = 0;
    for (int c = 0; c < chunks; ++c) {
      int x, y;
      const int b = c * 64 + l, n = c == 0 ? tiles : get(b, x, y), here = counted(n), here_upto = scan_wave(here);
      if (b < p.B) {
        p.table[2 + 2 * b] = before + here_upto - here;
        p.table[3 + 2 * b] = n;
      }
      before += __builtin_amdgcn_readlane(here_upto, 63);
    }
  }
  const unsigned from = parts ? (unsigned)run.n : run.n * chunk, where = from / (unsigned)unit;
  int at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(where < (unsigned)upto));
  unsigned before = (unsigned)(__builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(mine, at));
  const int b0 = at * per_block * 64;
  for (int i0 = 0; i0 < per_block * 64; i0 += 64) {
    if (b0 + i0 > 0) tiles = get(b0 + i0 + l, len, q_len);
    mine = counted(tiles);
    upto = scan_wave(mine);
    const uint64_t behind = __builtin_amdgcn_ballot_w64(where < before + upto);
    if (behind) {
      at = __builtin_ctzll(behind);
      run.b = b0 + i0 + at;
      before += (unsigned)(__builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(mine, at));
      break;
    }
    before += (unsigned)__builtin_amdgcn_readlane(upto, 63);
  }
  const int n = __builtin_amdgcn_readlane(mine, at), of = __builtin_amdgcn_readlane(tiles, at);
  const unsigned in = from - before * unit;
  run.pair = (int)(in / (unsigned)n);
  run.t = (int)(in - run.pair * n);
  run.left = (int)min(chunk, total - from);
  if (parts) {             // part run.t of n, of equally many tiles
    const int per = (int)((unsigned)(of + n - 1) / (unsigned)n);
    run.t = min(run.t * per, of);
    run.left = min(per, of - run.t);
  }
  run.len = __builtin_amdgcn_readlane(len, at);
  run.q_len = __builtin_amdgcn_readlane(q_len, at);
  return run;
}

// A tile of the list: sequence, row tile of it, tile of that; and what goes with the sequence.
struct At {
  int b, pair, t;
  int len, listed;       // used slots, tiles of its row tiles in the list
};
__device__ __forceinline__ void to_next(const dbsp_paged_attn_params& p, int unit, At& x) {
  if (++x.t < x.listed) return;
  x.t = 0;
  if (++x.pair < unit) return;
  x.pair = 0;
  if (++x.b >= p.B) return;                // (past the end: not looked at)
  x.len = paged_len(p, x.b);
  x.listed = listed_tiles(x.len, paged_q_len(p, x.b));
}

// Probabilities p >= 0, times kScale, as sums of two numbers of 16 bits; and what they may be (kRaise) before the running max is raised.  bf16 has
// f32's exponents: the sum is off by 2^-16 p at most, half a step of the second number.  fp16 has steps of 2^-24 and ends at 65504: the sum is off by
// 2^-21 p, and by half such a step where that is more, which is 2^-35 of the largest p.  Without the scale keys 17.4 or more below the largest
// score would be lost, however many they are.
template <class T> struct Halves;
template <> struct Halves<Bf16> {
  static constexpr float kScale = 1.f, kRaise = kRaiseAt;
  static __device__ __forceinline__ void split(float a, float b, uint32_t& x, uint32_t& rest) {
    x = Bf16::pack(a, b);
    rest = Bf16::pack(a - __builtin_bit_cast(float, x << 16), b - __builtin_bit_cast(float, x & 0xffff0000u));
  }
};
template <> struct Halves<Fp16> {
  static constexpr float kScale = 1024.f, kRaise = 32.f;
  static __device__ __forceinline__ void split(float a, float b, uint32_t& x, uint32_t& rest) {
    a *= kScale;
    b *= kScale;
    const f16x2 cut = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_pkrtz(a, b));
    x = __builtin_bit_cast(uint32_t, cut);
    rest = Fp16::pack(a - (float)cut.x, b - (float)cut.y);
  }
};

template <class T, int D, int NR>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(D == 128 && NR > 2 ? 1 : 2)))
void dbsp_paged_attn_kernel(const dbsp_paged_attn_params p) {
  using L = Lay<D>;
  constexpr int KS = D / 32, DT = D / 16, CH = D / 4, ROWS = 16 * NR;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[4 * L::TILE];      // [buffer][K, V]
  __shared__ int page_ids[4][2][64];
  __shared__ float mcs[4][16], sums[4][16];
  const Run run = find_run(p);
  const int left = __builtin_amdgcn_readfirstlane(run.left), run_n = __builtin_amdgcn_readfirstlane(run.n), unit = p.Hk * p.row_tiles;
  if (left == 0) return;
  At at;
  at.b = __builtin_amdgcn_readfirstlane(run.b);
  at.pair = __builtin_amdgcn_readfirstlane(run.pair);
  at.t = __builtin_amdgcn_readfirstlane(run.t);
  at.len = __builtin_amdgcn_readfirstlane(run.len);
  int q_len = __builtin_amdgcn_readfirstlane(run.q_len);
  at.listed = listed_tiles(at.len, q_len);
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l = threadIdx.x & 63, n = l & 15, g = l >> 4;
  const int rows = p.Nq * p.G;
  const uint32_t lds_base = (uint32_t)(uintptr_t)(LDS_PTR(unsigned char))lds;
  const uint32_t ids_base = (uint32_t)(uintptr_t)(LDS_PTR(int))&page_ids[w][0][0];
  // lane l asks for the page of the wave's key l % 16 of a tile (past the end of the table: its last entry, which is not looked at)
  auto copy_ids = [&](const At& x, int parity) __attribute__((always_inline)) {
    const int slot = x.t * kPagedKeys + 16 * w + n;
    copy_lane4((uint64_t)(uintptr_t)(p.pages + x.b * p.pages_stride + min(page_of(p, slot), p.max_pages - 1)), ids_base + parity * 256);
  };
  At next = at, after;
  copy_ids(at, 0);
  if (left > 1) to_next(p, unit, next);
  copy_ids(next, 1);
  after = next;

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
  const float c = p.scale_log2;
  const int row_in = l / L::NCH, pch = l % L::NCH;
  const uint64_t zeros = (uint64_t)(uintptr_t)kZeros + (pch << 4);
  // where a lane's 16 bytes of a row lie, behind the wave's first slot, where all its slots are in one page
  uint32_t k_in[L::COPIES], v_in;
#pragma unroll
  for (int i = 0; i < L::COPIES; ++i) k_in[i] = row_in * p.k_ss + ((pch ^ L::k_swz(i * L::RPC + row_in)) << 4);
  v_in = row_in * p.v_ss + ((pch ^ L::v_swz(row_in)) << 4);
  static_assert(L::RPC % (L::RPL * L::NCH / 4) == 0, "V's chunks lie alike in all of a wave's copies");
  // copies this wave's keys of a tile; which of them are there, a bit each
  auto copy_tile = [&](const At& x, int buf) __attribute__((always_inline)) {
    const uint32_t dst = lds_base + buf * 2 * L::TILE + 16 * w * L::ROWB, ids = ids_base + buf * 256;
    const int slot0 = x.t * kPagedKeys + 16 * w, hk = (int)((unsigned)x.pair / (unsigned)p.row_tiles);
    const uint64_t k_head = (uint64_t)(uintptr_t)(p.k + hk * p.k_sh), v_head = (uint64_t)(uintptr_t)(p.v + hk * p.v_sh);
    const int page_n = *(LDS_PTR(int))(uintptr_t)(ids + 4 * n);
    const uint32_t there = (uint32_t)__builtin_amdgcn_ballot_w64(slot0 + n < x.len && (unsigned)page_n < (unsigned)p.n_pages) & 0xffffu;
    // (next tokens of 32 sequences in pages of 16 slots 68.0 us a lane, 67.3 so, 128 sequences 139 / 135; by copies of 8 or 4 slots in smaller pages no faster)
    if (p.page_16 && there == 0xffffu) {
      const uint64_t page = (unsigned)__builtin_amdgcn_readfirstlane(page_n), place = (unsigned)__builtin_amdgcn_readfirstlane(slot0 - page_of(p, slot0) * p.page_size);
      const unsigned char* k_at = reinterpret_cast<const unsigned char*>(k_head + page * p.k_sp + place * p.k_ss);
      const unsigned char* v_at = reinterpret_cast<const unsigned char*>(v_head + page * p.v_sp + place * p.v_ss);
#pragma unroll
      for (int i = 0; i < L::COPIES; ++i) {
        copy_row16(k_at + (uint64_t)(i * L::RPC) * p.k_ss, k_in[i], dst + i * 1024);
        copy_row16(v_at + (uint64_t)(i * L::RPC) * p.v_ss, v_in, dst + L::TILE + i * 1024);
      }
      return there;
    }
#pragma unroll
    for (int i = 0; i < L::COPIES; ++i) {
      const int in = i * L::RPC + row_in, slot = slot0 + in;
      const uint32_t page = *(LDS_PTR(uint32_t))(uintptr_t)(ids + 4 * in), place = slot - page_of(p, slot) * p.page_size;
      const bool here = slot < x.len && page < (unsigned)p.n_pages;
      uint64_t k_at = k_head + (uint64_t)page * p.k_sp + (uint64_t)place * p.k_ss + ((pch ^ L::k_swz(in)) << 4);
      uint64_t v_at = v_head + (uint64_t)page * p.v_sp + (uint64_t)place * p.v_ss + ((pch ^ L::v_swz(in)) << 4);
      asm("" : "+v"(k_at), "+v"(v_at));      // (formed by all lanes: no branch for the choice)
      copy_lane16(here ? k_at : zeros, dst + i * 1024);
      copy_lane16(here ? v_at : zeros, dst + L::TILE + i * 1024);
    }
    return there;
  };

  int limit[NR], all_see, row0, hk;
  bool valid[NR];
  u32x4 q[NR][KS];
  f32x4 o[NR][DT];
  float mc[NR], sum[NR];                   // the max starts at the lowest finite value: scores of -inf then have probability 0
  // the queries and limits of a row tile, and statistics of nothing yet
  auto begin = [&](const At& x) __attribute__((always_inline)) {
    hk = (int)((unsigned)x.pair / (unsigned)p.row_tiles);
    row0 = (x.pair - hk * p.row_tiles) * ROWS;
    all_see = INT_MAX;
#pragma unroll
    for (int y = 0; y < NR; ++y) {
      const int row = row0 + 16 * y + n, in = min(row, rows - 1), tok = (int)((unsigned)in / (unsigned)p.G), gh = in - tok * p.G;
      valid[y] = row < rows && tok < q_len;
      limit[y] = p.causal ? max(0, min(x.len, x.len - q_len + 1 + tok)) : x.len;
      all_see = min(all_see, valid[y] ? limit[y] : INT_MAX);
      const uint16_t* src = p.q + x.b * p.q_sb + (hk * p.G + gh) * p.q_sh + tok * p.q_st;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) q[y][ks] = *reinterpret_cast<const u32x4*>(src + 32 * ks + 8 * g);
      mc[y] = -FLT_MAX;
      sum[y] = 0.f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[y][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    all_see = over_row(all_see, [](int x, int y) { return min(x, y); });
    all_see = __builtin_amdgcn_readfirstlane(all_see);
    // the queries are waited for here and not between copies, which the compiler does not count
#pragma unroll
    for (int y = 0; y < NR; ++y)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(q[y][ks]));
  };
  begin(at);
  wait_all();                              // the first two tiles' pages
  uint32_t there = copy_tile(at, 0);
  int first = at.t;                        // of the row tile's tiles in this run
  for (int j = 0; j < left; ++j) {
    const int buf = j & 1;
    uint32_t there_next = 0;
    if (j + 1 < left) {
      // the pages of the next tile have landed (younger are the copies of this tile only), and what was read in its buffer has arrived
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * L::COPIES) : "memory");
      if (j + 2 < left) to_next(p, unit, after);
      copy_ids(after, buf);
      there_next = copy_tile(next, buf ^ 1);
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * L::COPIES + 1) : "memory");      // this tile has landed, the next one is under way
    } else {
      wait_all();
    }
    const uint32_t off = buf * 2 * L::TILE;
    const int key = at.t * kPagedKeys + 16 * w + 4 * g;
    u32x4 kf[KS];
    u32x2 vf[DT];
    u32x4 pb[NR];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) kf[ks] = *(LDS_PTR(u32x4))(uintptr_t)(k_rd[ks] + off);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) vf[dt] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(uintptr_t)(v_rd[dt] + off)));
#pragma unroll
    for (int y = 0; y < NR; ++y) {
      f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) x = T::mfma32(kf[ks], q[y][ks], x);
      if (there != 0xffffu || (at.t + 1) * kPagedKeys > all_see) {
        const int see = limit[y] - key;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (i >= see || !((there >> (4 * g + i)) & 1)) x[i] = -INFINITY;
      }
      float pr[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) pr[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], c, -mc[y]));
      const float top4 = fmaxf(fmaxf(pr[0], pr[1]), fmaxf(pr[2], pr[3]));
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(top4 > Halves<T>::kRaise) != 0, 0)) {
        float top = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float to = fmaxf(mc[y], top * c), f = __builtin_amdgcn_exp2f(mc[y] - to);
        mc[y] = to;
        sum[y] *= f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[y][dt] *= f;
#pragma unroll
        for (int i = 0; i < 4; ++i) pr[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], c, -to));
      }
      sum[y] += (pr[0] + pr[1]) + (pr[2] + pr[3]);
      uint32_t x01, x23, rest01, rest23;
      Halves<T>::split(pr[0], pr[1], x01, rest01);
      Halves<T>::split(pr[2], pr[3], x23, rest23);
      pb[y] = u32x4{x01, x23, rest01, rest23};
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int y = 0; y < NR; ++y) o[y][dt] = T::mfma32(u32x4{vf[dt].x, vf[dt].y, vf[dt].x, vf[dt].y}, pb[y], o[y][dt]);
    there = there_next;
    if (j + 1 < left && next.t != 0) {
      at = next;
      next = after;
      continue;
    }

    // The row tile's last tile, here or at all: the waves' results, 16 rows at a time, by way of the buffer that has been read (the next tile
    // is under way to the other one): [wave][row][16-byte chunk of the head dim, by row swizzled].
    const bool part = first != 0 || at.t + 1 != at.listed;
    const int64_t slot = (int64_t)run_n + (int64_t)at.b * unit + at.pair;      // of a partial result: from each to the next one of the two grows
    f32x4* const os = reinterpret_cast<f32x4*>(lds + off);
#pragma unroll
    for (int y = 0; y < NR; ++y) {
      __syncthreads();                     // everybody has read the tile, or the rows before
      sum[y] += __shfl_xor(sum[y], 16);
      sum[y] += __shfl_xor(sum[y], 32);
      if (g == 0) {
        mcs[w][n] = mc[y];
        sums[w][n] = sum[y];
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) os[(w * 16 + n) * CH + ((4 * dt + g) ^ n)] = o[y][dt];
      __syncthreads();
#pragma unroll
      for (int z = 0; z < 16 * CH / 256; ++z) {
        const int i = z * 256 + threadIdx.x, in = i / CH, ch = i % CH, row = row0 + 16 * y + in, tok = (int)((unsigned)row / (unsigned)p.G);
        if (row >= rows || tok >= q_len) continue;
        float m = mcs[0][in];
#pragma unroll
        for (int x = 1; x < 4; ++x) m = fmaxf(m, mcs[x][in]);
        float all = 0.f;
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const float f = __builtin_amdgcn_exp2f(mcs[x][in] - m);
          all += f * sums[x][in];
          acc += f * os[(x * 16 + in) * CH + (ch ^ in)];
        }
        const bool none = __builtin_bit_cast(uint32_t, all) == 0u;      // (by its bits: NaNs are not regarded in this file)
        acc *= none ? 0.f : 1.f / Halves<T>::kScale / all;
        const float lse2 = none ? -INFINITY : m + __builtin_amdgcn_logf(all);
        if (part) {
          const int64_t pr = slot * p.own_rows + 16 * y + in;
          *reinterpret_cast<f32x4*>(p.part_o + pr * D + 4 * ch) = acc;
          if (ch == 0) p.part_lse[pr] = lse2;
        } else {
          const int h = hk * p.G + row - tok * p.G;
          *reinterpret_cast<u32x2*>(p.o + at.b * p.o_sb + h * p.o_sh + tok * p.o_st + 4 * ch) = u32x2{T::pack_o(acc.x, acc.y), T::pack_o(acc.z, acc.w)};
          if (ch == 0 && p.lse) p.lse[((int64_t)at.b * p.H + h) * p.Nq + tok] = lse2 * 0.69314718055994531f;
        }
      }
    }
    if (j + 1 == left) return;
    __syncthreads();                       // the tile behind the next one goes where the results were
    if (next.b != at.b) q_len = paged_q_len(p, next.b);
    at = next;
    next = after;
    first = 0;
    begin(at);
  }
}

// Joins partial results, D / 4 lanes a part of a row, four values each: WAYS of them a row, which take its parts in turn.
template <class T, int D, int WAYS>
__global__ __launch_bounds__(256) void dbsp_paged_merge_kernel(const dbsp_paged_attn_params p, int tile_rows) {
  constexpr int LANES = D / 4, ROWS = 256 / LANES / WAYS, U = 8;
  const int lanes = threadIdx.x / LANES, way = lanes % WAYS, x = 4 * (threadIdx.x % LANES);
  const unsigned nth = blockIdx.x * ROWS + lanes / WAYS, all = (unsigned)p.B * p.H * p.Nq, at_row = min(nth, all - 1);      // [b][h][t]
  const unsigned bh = at_row / (unsigned)p.Nq;
  const int t = (int)(at_row - bh * p.Nq), b = (int)(bh / (unsigned)p.H), h = (int)(bh - b * p.H), hk = (int)((unsigned)h / (unsigned)p.G);
  const int32_t* const q_lens = p.q_lens ? p.q_lens : p.lens;
  const unsigned chunk = (unsigned)p.table[0], parts = (unsigned)p.table[1], before = (unsigned)p.table[2 + 2 * b], tiles = (unsigned)p.table[3 + 2 * b];
  const int q_as_given = q_lens[b];
  if (parts == 2) return;                  // no row tile was cut
  const int row = t * p.G + h - hk * p.G, rt = row / tile_rows;
  // the runs that the row tile lies in, or its parts
  const unsigned unit = (unsigned)(p.Hk * p.row_tiles), pair = (unsigned)(hk * p.row_tiles + rt);
  unsigned run0, n;
  if (parts) {
    n = (tiles + chunk - 1) / chunk;
    run0 = before * unit + pair * n;
    const unsigned per = (tiles + n - 1) / n;
    n = (tiles + per - 1) / per;           // (the last ones may have none left)
  } else {
    const unsigned from = before * unit + pair * tiles;
    run0 = from / chunk;
    n = (from + tiles - 1) / chunk - run0 + 1;
  }
  const bool mine = nth < all && (!p.q_lens || t < q_as_given) && n > 1;      // (a row tile in one run has been written as it is)
  const int64_t step = p.own_rows, at = ((int64_t)run0 + (int64_t)b * unit + pair) * p.own_rows + row - rt * tile_rows;
  float m = -FLT_MAX, sum = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int i0 = way; mine && i0 < (int)n; i0 += U * WAYS) {
    float ls[U];
    f32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * WAYS;
      const int64_t pr = at + min(i, (int)n - 1) * step;
      ls[u] = i < (int)n ? p.part_lse[pr] : -INFINITY;
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
      const float wgt = __builtin_amdgcn_exp2f(ls[u] - m);
      sum += wgt;
      acc += wgt * v[u];                   // (a part without a key has zeros; the last part again, past the end, weighs nothing)
    }
  }
  if constexpr (WAYS > 1) {
    __shared__ f32x4 accs[ROWS][WAYS][LANES];
    __shared__ float ms[ROWS][WAYS], sums[ROWS][WAYS];
    const int r = lanes / WAYS, lane = threadIdx.x % LANES;
    accs[r][way][lane] = acc;
    if (x == 0) {
      ms[r][way] = m;
      sums[r][way] = sum;
    }
    __syncthreads();
    if (way != 0) return;
#pragma unroll
    for (int y = 1; y < WAYS; ++y) m = fmaxf(m, ms[r][y]);
    sum = 0.f;
    acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int y = 0; y < WAYS; ++y) {
      const float f = __builtin_amdgcn_exp2f(ms[r][y] - m);
      sum += f * sums[r][y];
      acc += f * accs[r][y][lane];
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
  const int tile_rows = paged_tile_rows((int64_t)p.Nq * p.G);
  if (tile_rows == 16) dbsp_paged_attn_kernel<T, D, 1><<<grid, 256, 0, stream>>>(p);
  else if (tile_rows == 32) dbsp_paged_attn_kernel<T, D, 2><<<grid, 256, 0, stream>>>(p);
  else if (tile_rows == 48) dbsp_paged_attn_kernel<T, D, 3><<<grid, 256, 0, stream>>>(p);
  else dbsp_paged_attn_kernel<T, D, 4><<<grid, 256, 0, stream>>>(p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.merge_groups == 0) return e;
  if (p.merge_ways == 1) dbsp_paged_merge_kernel<T, D, 1><<<p.merge_groups, 256, 0, stream>>>(p, tile_rows);
  else if (p.merge_ways == 2) dbsp_paged_merge_kernel<T, D, 2><<<p.merge_groups, 256, 0, stream>>>(p, tile_rows);
  else if (p.merge_ways == 4) dbsp_paged_merge_kernel<T, D, 4><<<p.merge_groups, 256, 0, stream>>>(p, tile_rows);
  else dbsp_paged_merge_kernel<T, D, 8><<<p.merge_groups, 256, 0, stream>>>(p, tile_rows);
  return hipGetLastError();
}

}  // namespace

hipError_t dbsp_launch_paged_attn(const dbsp_paged_attn_params& p, int d, bool fp16, int grid, hipStream_t stream) {
  if (d == 64) return fp16 ? launch<Fp16, 64>(p, grid, stream) : launch<Bf16, 64>(p, grid, stream);
  return fp16 ? launch<Fp16, 128>(p, grid, stream) : launch<Bf16, 128>(p, grid, stream);
}
