// Eviction from the own keys of a key/value cache: of every (sequence, KV head) with more than `budget` keys the `budget`
// largest by weight stay (sinks and recent positions above all others; NaN as -inf; of equal ones the lowest slots).
//
// Attention does not ask for the order of the keys before the newest ones, so nothing is shifted: a kept key behind the
// budget moves into the hole that an evicted one leaves in front of it, both in ascending order.  Sources (slots >= budget) and
// destinations (slots < budget) are disjoint, so rows move in place, in parallel, and only those that have to.
//
// Choosing goes by the weights' order-preserving 32-bit images, of which the budget-th largest is the limit: counts by digits of 11, 11
// and 10 bits from the top, the second and third only among images that agree with the limit so far.  Whole numbers are added, so
// their order of arrival does not matter.
//   * Up to 32,768 slots a workgroup has a (sequence, head), its images in registers, read once, and the counts in the LDS; it
//     stops at the digit at which all images that have it stay.  256 heads of 2064 slots: 9 us, of which the exchanges between a
//     workgroup's 8 waves are most; 96 of 11,500 slots: 18 us, by instructions (46 with four digits of 8 bits, read anew for each; two
//     bits a step by ballots took twice as long as digits).  Prefix sums of a wave by DPP: 0.7 us less than by way of the LDS.
//   * Longer ones are cut into workgroups of 8192 slots: three launches count, a fourth counts what each part keeps, a fifth
//     lists holes and fillers, 5 to 8 us each.  8 heads of 131,100 slots: 66 us with the moves, 431 by a workgroup a head.
// A last launch moves the rows, 64 moves of a workgroup in flight at once, bound by memory: 96 heads, 1700 rows of K and V each (167 MB
// read and written) 38 us, 4.4 TB/s.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "cache_params.hpp"
#include "wave_scan.hpp"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kMovesPerGroup = 64;
// Images a thread: as many as the capacity needs, in four steps.  us of a call with 20 / 32: 8 (sequence, head) pairs of 13,000 slots 24.9 / 28.2, 96
// 46.6 / 49.8, 600 154 / 164, 8 of 20,000 31.0 / 34.7, 96 of 10,000 - 20,000 106.7 / 109.0, 600 of 20,000 187 / 198.
constexpr int kNT = evict_threads(kEvictWhole);

// Larger weight, larger image; what must stay comes last.
__device__ __forceinline__ uint32_t image(float w, bool stays) {
  if (stays) return 0xffffffffu;
  uint32_t x = __builtin_bit_cast(uint32_t, w);
  if ((x & 0x7fffffffu) > 0x7f800000u) x = 0xff800000u;      // NaN as -inf
  if (x == 0x80000000u) x = 0u;                              // -0 as 0
  return (x >> 31) ? ~x : x | 0x80000000u;
}

// Images of the slots first + j * NT + t below n, j = 0 .. R - 1; 0, which is nobody's, past them.
template <int NT, int R>
__device__ __forceinline__ void load_images(const dbsp_cache_evict_params& p, int pair, int first, int n, uint32_t (&x)[R]) {
  const float* weights = p.weights + (int64_t)pair * p.cap;
  const int32_t* positions = p.positions + (int64_t)pair * p.cap;
  const bool recent = p.keep_from != nullptr;
  const int keep_from = recent ? p.keep_from[pair / p.Hk] : 0;
  float w[R];
  int at[R];
#pragma unroll
  for (int j = 0; j < R; ++j) {
    w[j] = 0.f;
    at[j] = 0;
    if (first + j * NT >= n) continue;
    const int i = min(first + j * NT + (int)threadIdx.x, n - 1);
    w[j] = weights[i];
    at[j] = positions[i];
  }
#pragma unroll
  for (int j = 0; j < R; ++j)
    x[j] = first + j * NT + (int)threadIdx.x < n ? image(w[j], at[j] < p.sinks || (recent && at[j] >= keep_from)) : 0u;
}

__device__ __forceinline__ int used_of(const dbsp_cache_evict_params& p, int pair) { return max(0, min(p.lens[pair / p.Hk], p.cap)); }

// Exclusive prefix, in slot order, of the counts that every wave has for its j-th run of 64 slots: table[j * WAVES + w].
template <int NT, int R>
__device__ __forceinline__ void scan_table(int (&table)[R * NT / 64 + 1]) {
  constexpr int N = R * NT / 64, PER = (N + 63) / 64;
  __syncthreads();
  if (threadIdx.x < 64) {
    const int l = threadIdx.x;
    int v[PER], mine = 0;
#pragma unroll
    for (int y = 0; y < PER; ++y) {
      const int i = l * PER + y;
      v[y] = i < N ? table[i] : 0;
      mine += v[y];
    }
    const int upto = scan_wave(mine);
    int before = upto - mine;
#pragma unroll
    for (int y = 0; y < PER; ++y) {
      const int i = l * PER + y;
      if (i < N) table[i] = before;
      before += v[y];
    }
    if (l == 63) table[N] = upto;
  }
  __syncthreads();
}

// What stays, of R images a thread: those above the limit, and of its equals the first stay_equal (counted from equal_before of them
// in front of these slots); and the ranks of holes (slots below the budget that go) and fillers (slots from it on that stay).
template <int NT, int R, class F>
__device__ __forceinline__ void list_moves(const uint32_t (&x)[R], int first, int n, int budget, uint32_t limit, int stay_equal, bool some_equals_go,
                                           int equal_before, int (&table)[R * NT / 64 + 1], F&& each, int* n_holes, int* n_fillers) {
  constexpr int WAVES = NT / 64;
  const int w = threadIdx.x >> 6, l = threadIdx.x & 63;
  const uint64_t below = (1ull << l) - 1;
  uint32_t kept = 0;
  if (some_equals_go) {
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const uint64_t m = __builtin_amdgcn_ballot_w64(x[j] == limit);
      if (l == 0) table[j * WAVES + w] = __popcll(m);
    }
    scan_table<NT, R>(table);
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const uint64_t m = __builtin_amdgcn_ballot_w64(x[j] == limit);
      const int e = equal_before + table[j * WAVES + w] + __popcll(m & below);
      kept |= (uint32_t)(x[j] > limit || (x[j] == limit && e < stay_equal)) << j;
    }
    __syncthreads();                       // before the table is used again
  } else {
#pragma unroll
    for (int j = 0; j < R; ++j) kept |= (uint32_t)(x[j] >= limit) << j;
  }
  // holes and fillers counted in one: no wave's run of 64 slots has more than 64 of either
#pragma unroll
  for (int j = 0; j < R; ++j) {
    const int i = first + j * NT + (int)threadIdx.x;
    const bool stays = kept >> j & 1, in = i < n;
    const uint64_t hm = __builtin_amdgcn_ballot_w64(in && i < budget && !stays), fm = __builtin_amdgcn_ballot_w64(in && i >= budget && stays);
    if (l == 0) table[j * WAVES + w] = __popcll(hm) | __popcll(fm) << 16;
    if (first + (j + 1) * NT >= n) {       // none behind
#pragma unroll
      for (int y = j + 1; y < R; ++y)
        if (l == 0) table[y * WAVES + w] = 0;
      break;
    }
  }
  scan_table<NT, R>(table);
#pragma unroll
  for (int j = 0; j < R; ++j) {
    if (first + j * NT >= n) break;
    const int i = first + j * NT + (int)threadIdx.x;
    const bool stays = kept >> j & 1, in = i < n, hole = in && i < budget && !stays, filler = in && i >= budget && stays;
    const uint64_t hm = __builtin_amdgcn_ballot_w64(hole), fm = __builtin_amdgcn_ballot_w64(filler);
    const int before = table[j * WAVES + w];
    each(j, i, hole, filler, in && !stays, hole ? (before & 0xffff) + __popcll(hm & below) : (before >> 16) + __popcll(fm & below));
  }
  *n_holes = table[R * WAVES] & 0xffff;
  *n_fillers = table[R * WAVES] >> 16;
}

// Counts digit PASS of the `here` images that agree with `limit` above it: hist, 2048 zeros before.
constexpr int kDigits = 2048, kShift[3] = {21, 10, 0};
template <int PASS, int NT, int R>
__device__ __forceinline__ void count_digits(const uint32_t (&x)[R], int here, uint32_t limit, uint32_t* hist) {
#pragma unroll
  for (int j = 0; j < R; ++j) {
    if (j * NT >= here) break;
    const bool in = x[j] != 0u && (PASS == 0 || (x[j] ^ limit) >> kShift[PASS ? PASS - 1 : 0] == 0u);
    if (in) atomicAdd(&hist[x[j] >> kShift[PASS] & (PASS == 2 ? 1023 : 2047)], 1u);
  }
}

// A thread's share of a digit's 2048 counts: thread 0 has those of the largest digits, the largest first.
template <int NT>
struct Share { uint32_t c[kDigits / NT]; };
template <int NT>
__device__ __forceinline__ Share<NT> my_digits(const uint32_t* counts) {
  constexpr int PER = kDigits / NT;
  Share<NT> s;
#pragma unroll
  for (int y = 0; y < PER; ++y) s.c[y] = counts[kDigits - 1 - PER * (int)threadIdx.x - y];
  return s;
}

// Of the images whose upper bits are those of `limit`: the digit below them at which `left` of them, from the largest on, are
// reached.  limit and left are brought up to date; returns how many have the chosen digit.  (PASS: its own places in the LDS)
template <int PASS, int NT>
__device__ __forceinline__ uint32_t pick_digit(const Share<NT>& s, uint32_t& limit, uint32_t& left) {
  constexpr int PER = kDigits / NT;
  __shared__ uint32_t wave_sum[NT / 64], got[3];
  const int t = threadIdx.x, w = t >> 6, l = t & 63;
  uint32_t mine = 0;
#pragma unroll
  for (int y = 0; y < PER; ++y) mine += s.c[y];
  const uint32_t upto = scan_wave((int)mine);
  if (l == 63) wave_sum[w] = upto;
  __syncthreads();
  uint32_t before = upto - mine;
#pragma unroll
  for (int y = 0; y < NT / 64; ++y) before += y < w ? wave_sum[y] : 0u;
  if (before < left && left <= before + mine) {
#pragma unroll
    for (int y = 0; y < PER; ++y) {
      if (before < left && left <= before + s.c[y]) {
        got[0] = kDigits - 1 - PER * t - y;
        got[1] = left - before;
        got[2] = s.c[y];
      }
      before += s.c[y];
    }
  }
  __syncthreads();
  limit |= got[0] << kShift[PASS];
  left = got[1];
  return got[2];
}

template <int NT, int R>
__global__ __launch_bounds__(NT) void dbsp_cache_choose_kernel(const dbsp_cache_evict_params p) {
  static_assert(R <= 32 && NT * R <= kEvictWhole, "16 bits a count, a bit a slot");
  __shared__ uint32_t hist[3 * kDigits];
  __shared__ int table[R * NT / 64 + 1];
  const int pair = blockIdx.x, t = threadIdx.x;
  const int n = used_of(p, pair), budget = p.budget;
  for (int i = t; i < 3 * kDigits; i += NT) hist[i] = 0;      // while the length is under way
  if (n <= budget) {
    if (t == 0) p.n_moves[pair] = 0;
    return;
  }
  uint32_t x[R];
  load_images<NT, R>(p, pair, 0, n, x);
  __syncthreads();
  // `left` of the `equal` images that have the limit's digits so far stay, and all above them
  uint32_t limit = 0, left = (uint32_t)budget;
  count_digits<0, NT, R>(x, n, limit, hist);
  __syncthreads();
  uint32_t equal = pick_digit<0>(my_digits<NT>(hist), limit, left);
  if (equal != left) {
    count_digits<1, NT, R>(x, n, limit, hist + kDigits);
    __syncthreads();
    equal = pick_digit<1>(my_digits<NT>(hist + kDigits), limit, left);
  }
  if (equal != left) {
    count_digits<2, NT, R>(x, n, limit, hist + 2 * kDigits);
    __syncthreads();
    equal = pick_digit<2>(my_digits<NT>(hist + 2 * kDigits), limit, left);
  }
  int32_t *holes = p.holes + (int64_t)pair * p.max_moves, *fillers = p.fillers + (int64_t)pair * p.max_moves;
  float* weights = p.weights + (int64_t)pair * p.cap;
  int n_holes, n_fillers;
  list_moves<NT, R>(x, 0, n, budget, limit, (int)left, equal != left, 0, table,
                     [&](int, int i, bool hole, bool filler, bool goes, int rank) {
                       if (hole) holes[rank] = i;
                       if (filler) fillers[rank] = i;
                       if (goes && i >= budget) weights[i] = 0.f;
                     }, &n_holes, &n_fillers);
  if (t == 0) p.n_moves[pair] = n_fillers;
}

// Long caches, a part a workgroup.
constexpr int kR = 8;
static_assert(kNT * kR == kEvictPart, "slots of a part");

__global__ __launch_bounds__(256) void dbsp_cache_clear_kernel(uint32_t* digits, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) digits[i] = 0;
}

// PASS 0, 1, 2: counts the digits of 11, 11 and 10 bits from the top.  PASS 3: counts what each part keeps.  PASS 4: lists.
template <int PASS>
__global__ __launch_bounds__(kNT) void dbsp_cache_part_kernel(const dbsp_cache_evict_params p) {
  __shared__ uint32_t hist[PASS < 3 ? kDigits : 1];
  __shared__ int table[PASS == 4 ? kR * kNT / 64 + 1 : 1];
  __shared__ int sums[PASS >= 3 ? 4 : 1];
  const int pair = blockIdx.x, part = blockIdx.y, t = threadIdx.x, first = part * kEvictPart;
  const int n = used_of(p, pair), budget = p.budget;
  if (n <= budget) {
    if (PASS == 4 && part == 0 && t == 0) p.n_moves[pair] = 0;
    return;
  }
  if (first >= n) return;
  uint32_t x[kR];
  uint32_t* digits = p.digits + (int64_t)pair * 3 * kDigits;
  uint32_t limit = 0, left = (uint32_t)budget, equal = 0;
  uint32_t* chosen = p.chosen + pair * 3;
  Share<kNT> counts[PASS > 0 && PASS < 4 ? PASS : 1];
  if constexpr (PASS == 4) {
    limit = chosen[0];
    left = chosen[1];
    equal = chosen[2];
  }
#pragma unroll
  for (int y = 0; y < PASS && PASS < 4; ++y) counts[y] = my_digits<kNT>(digits + y * kDigits);
  load_images<kNT, kR>(p, pair, first, n, x);
  if constexpr (PASS > 0 && PASS < 4) equal = pick_digit<0>(counts[0], limit, left);
  if constexpr (PASS > 1 && PASS < 4) equal = pick_digit<1>(counts[1], limit, left);
  if constexpr (PASS > 2 && PASS < 4) equal = pick_digit<2>(counts[2], limit, left);
  if (PASS == 3 && part == 0 && t == 0) {
    chosen[0] = limit;
    chosen[1] = left;
    chosen[2] = equal;
  }
  if constexpr (PASS < 3) {
    for (int i = t; i < kDigits; i += kNT) hist[i] = 0;
    __syncthreads();
    count_digits<PASS, kNT, kR>(x, n - first, limit, hist);
    __syncthreads();
    for (int i = t; i < kDigits; i += kNT)
      if (hist[i]) atomicAdd(&digits[PASS * kDigits + i], hist[i]);
  } else {
    // above the limit and equal to it, in slots below the budget and from it on
    int32_t* parts = p.parts + (int64_t)pair * p.n_parts * 4;
    if (t < 4) sums[t] = 0;
    __syncthreads();
    if constexpr (PASS == 3) {
      int c[4] = {0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < kR; ++j) {
        const bool late = first + j * kNT + t >= budget;
        c[0] += __popcll(__builtin_amdgcn_ballot_w64(x[j] > limit && !late));
        c[1] += __popcll(__builtin_amdgcn_ballot_w64(x[j] == limit && !late));
        c[2] += __popcll(__builtin_amdgcn_ballot_w64(x[j] > limit && late));
        c[3] += __popcll(__builtin_amdgcn_ballot_w64(x[j] == limit && late));
      }
#pragma unroll
      for (int y = 0; y < 4; ++y)
        if ((t & 63) == 0) atomicAdd(&sums[y], c[y]);
      __syncthreads();
      if (t < 4) parts[part * 4 + t] = sums[t];
    } else {
      // of the parts in front of this one: equals, holes and fillers.  Equals stay in slot order, so how many of a part's do
      // follows from the equals in front of it.
      int eq = 0;
      for (int y = t; y < part; y += kNT) eq += parts[y * 4 + 1] + parts[y * 4 + 3];
      if (eq) atomicAdd(&sums[0], eq);
      __syncthreads();
      const int equal_before = sums[0];
      // kept slots below the budget in front of this part, and from it on: equals that stay are the first `left`
      int gt_early = 0, eq_early = 0, gt_late = 0;
      for (int y = t; y < part; y += kNT) {
        gt_early += parts[y * 4];
        eq_early += parts[y * 4 + 1];
        gt_late += parts[y * 4 + 2];
      }
      if (gt_early) atomicAdd(&sums[1], gt_early);
      if (eq_early) atomicAdd(&sums[2], eq_early);
      if (gt_late) atomicAdd(&sums[3], gt_late);
      __syncthreads();
      const int early = min(first, budget), stay_early = sums[1] + min((int)left, sums[2]);
      const int holes_before = early - stay_early;
      const int fillers_before = sums[3] + min((int)left, equal_before) - min((int)left, sums[2]);
      int32_t *holes = p.holes + (int64_t)pair * p.max_moves + holes_before, *fillers = p.fillers + (int64_t)pair * p.max_moves + fillers_before;
      float* weights = p.weights + (int64_t)pair * p.cap;
      int n_holes, n_fillers;
      list_moves<kNT, kR>(x, first, n, budget, limit, (int)left, equal != left, equal_before, table,
                          [&](int, int i, bool hole, bool filler, bool goes, int rank) {
                            if (hole) holes[rank] = i;
                            if (filler) fillers[rank] = i;
                            if (goes && i >= budget) weights[i] = 0.f;
                          }, &n_holes, &n_fillers);
      if (t == 0 && first + kEvictPart >= n) p.n_moves[pair] = fillers_before + n_fillers;
    }
  }
}

// LANES 16-byte pieces a row; a workgroup's moves are all in flight at once.
template <int LANES>
__global__ __launch_bounds__(256) void dbsp_cache_move_kernel(const dbsp_cache_evict_params p) {
  constexpr int ROWS = 256 / LANES, U = kMovesPerGroup / ROWS;
  const int pair = blockIdx.x, b = pair / p.Hk, hk = pair % p.Hk, t = threadIdx.x, x = t % LANES * 16;
  const int first = (int)blockIdx.y * kMovesPerGroup + t / LANES, n = p.n_moves[pair];
  const int32_t *fillers = p.fillers + (int64_t)pair * p.max_moves, *holes = p.holes + (int64_t)pair * p.max_moves;
  int from32[U], to32[U];                  // asked for with n, not after it; what lies behind the first n is not used
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = min(first + u * ROWS, p.max_moves - 1);
    from32[u] = fillers[i];
    to32[u] = holes[i];
  }
  if (hk == 0 && blockIdx.y == 0 && t == 0 && p.lens[b] > p.budget) p.lens[b] = p.budget;
  if ((int)blockIdx.y * kMovesPerGroup >= n) return;
  unsigned char *k = p.k + b * p.k_sb + hk * p.k_sh + x, *v = p.v + b * p.v_sb + hk * p.v_sh + x;
  float* weights = p.weights + (int64_t)pair * p.cap;
  int32_t* positions = p.positions + (int64_t)pair * p.cap;
  int64_t from[U], to[U];
  u32x4 kr[U], vr[U];
  float w[U];
  int32_t at[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const bool there = first + u * ROWS < n;           // (else a row that is read and not stored)
    from[u] = there ? from32[u] : 0;
    to[u] = there ? to32[u] : 0;
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    kr[u] = *reinterpret_cast<const u32x4*>(k + from[u] * p.k_st);
    vr[u] = *reinterpret_cast<const u32x4*>(v + from[u] * p.v_st);
    w[u] = weights[from[u]];
    at[u] = positions[from[u]];
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (first + u * ROWS >= n) continue;
    *reinterpret_cast<u32x4*>(k + to[u] * p.k_st) = kr[u];
    *reinterpret_cast<u32x4*>(v + to[u] * p.v_st) = vr[u];
    if (x == 0) {
      weights[to[u]] = w[u];
      positions[to[u]] = at[u];
      weights[from[u]] = 0.f;              // (what a freed slot's next key starts from is nothing; the others' weights are cleared already)
    }
  }
}

}  // namespace

hipError_t dbsp_launch_cache_evict(const dbsp_cache_evict_params& p, hipStream_t stream) {
  const int pairs = p.B * p.Hk;
  if (p.n_parts > 0) {
    const int64_t n = (int64_t)pairs * 3 * kDigits;
    dbsp_cache_clear_kernel<<<(unsigned)((n + 4095) / 4096), 256, 0, stream>>>(p.digits, n);
    const dim3 grid(pairs, p.n_parts);
    dbsp_cache_part_kernel<0><<<grid, kNT, 0, stream>>>(p);
    dbsp_cache_part_kernel<1><<<grid, kNT, 0, stream>>>(p);
    dbsp_cache_part_kernel<2><<<grid, kNT, 0, stream>>>(p);
    dbsp_cache_part_kernel<3><<<grid, kNT, 0, stream>>>(p);
    dbsp_cache_part_kernel<4><<<grid, kNT, 0, stream>>>(p);
  } else if (evict_threads(p.cap) == 256) {
    dbsp_cache_choose_kernel<256, 4><<<pairs, 256, 0, stream>>>(p);
  } else if (evict_threads(p.cap) == 512) {
    dbsp_cache_choose_kernel<512, 8><<<pairs, 512, 0, stream>>>(p);
  } else if (p.cap <= 12 * kNT) {
    dbsp_cache_choose_kernel<kNT, 12><<<pairs, kNT, 0, stream>>>(p);
  } else if (p.cap <= 20 * kNT) {
    dbsp_cache_choose_kernel<kNT, 20><<<pairs, kNT, 0, stream>>>(p);
  } else {
    dbsp_cache_choose_kernel<kNT, 32><<<pairs, kNT, 0, stream>>>(p);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 grid(pairs, (p.max_moves + kMovesPerGroup - 1) / kMovesPerGroup);
  if (p.row_bytes == 256) dbsp_cache_move_kernel<16><<<grid, 256, 0, stream>>>(p);
  else dbsp_cache_move_kernel<8><<<grid, 256, 0, stream>>>(p);
  return hipGetLastError();
}
