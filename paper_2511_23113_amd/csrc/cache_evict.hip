// Eviction from the own keys of a key/value cache: of every (sequence, KV head) with more than `budget` keys the `budget`
// largest by weight stay (sinks and recent positions above all others; NaN as -inf; of equal ones the lowest slots).
//
// Attention does not ask for the order of the keys before the newest ones, so nothing is shifted: a kept key behind the
// budget moves into the hole that an evicted one leaves in front of it, both in ascending order.  Sources (slots >= budget) and
// destinations (slots < budget) are disjoint, so rows move in place, in parallel, and only those that have to.
//
// Choosing: a workgroup a (sequence, head) finds the budget-th largest of the weights' order-preserving 32-bit images, eight
// bits at a time by counting (the counts are whole numbers: their order of arrival does not matter), lists holes and
// fillers by a running count in slot order, and moves weights and positions.  A second launch moves the rows of K and V.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "cache_params.hpp"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int NT = 1024, WAVES = NT / 64;
constexpr int kMovesPerGroup = 64;

// Larger weight, larger image; what must stay comes last.
__device__ __forceinline__ uint32_t image(float w, bool stays) {
  if (stays) return 0xffffffffu;
  uint32_t x = __builtin_bit_cast(uint32_t, w);
  if ((x & 0x7fffffffu) > 0x7f800000u) x = 0xff800000u;      // NaN as -inf
  if (x == 0x80000000u) x = 0u;                              // -0 as 0
  return (x >> 31) ? ~x : x | 0x80000000u;
}

__global__ __launch_bounds__(NT) void dbsp_cache_choose_kernel(const dbsp_cache_evict_params p) {
  __shared__ uint32_t hist[256];
  __shared__ uint32_t chosen, rank_left;
  __shared__ int wave_equal[WAVES], wave_out[WAVES];
  const int pair = blockIdx.x, b = pair / p.Hk, t = threadIdx.x, w = t >> 6, l = t & 63;
  const int n = max(0, min(p.lens[b], p.cap));
  if (n <= p.budget) {
    if (t == 0) p.n_moves[pair] = 0;
    return;
  }
  float* weights = p.weights + (int64_t)pair * p.cap;
  int32_t* positions = p.positions + (int64_t)pair * p.cap;
  const bool recent = p.keep_from != nullptr;
  const int keep_from = recent ? p.keep_from[b] : 0;
  auto image_of = [&](int i) {
    const int at = positions[i];
    return image(weights[i], at < p.sinks || (recent && at >= keep_from));
  };
  // the budget-th largest image: `chosen`, and how many of its equals stay
  uint32_t prefix = 0, left = (uint32_t)p.budget;
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (t < 256) hist[t] = 0;
    __syncthreads();
    for (int i = t; i < n; i += NT) {
      const uint32_t x = image_of(i);
      if (shift == 24 || (x >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(x >> shift) & 255], 1u);
    }
    __syncthreads();
    if (w == 0) {                          // lane l: digits 4 l .. 4 l + 3, counted from the largest
      uint32_t c[4], mine = 0;
      for (int j = 0; j < 4; ++j) mine += c[j] = hist[4 * l + j];
      uint32_t above = mine;               // of this lane and those behind it
      for (int s = 1; s < 64; s <<= 1) {
        const uint32_t o = __shfl_down(above, s);
        if (l + s < 64) above += o;
      }
      above -= mine;
      for (int j = 3; j >= 0; --j) {
        if (above < left && left <= above + c[j]) {
          chosen = prefix | (uint32_t)(4 * l + j) << shift;
          rank_left = left - above;
        }
        above += c[j];
      }
    }
    __syncthreads();
    prefix = chosen;
    left = rank_left;
    __syncthreads();
  }
  // in slot order: equals of the chosen image stay until `left` of them have
  const uint32_t limit = prefix;
  const int stay_equal = (int)left;
  int32_t *holes = p.holes + (int64_t)pair * p.max_moves, *fillers = p.fillers + (int64_t)pair * p.max_moves;
  int equal_before = 0, holes_before = 0, fillers_before = 0;
  for (int i0 = 0; i0 < n; i0 += NT) {
    const int i = i0 + t;
    const uint32_t x = i < n ? image_of(i) : 0u;
    const bool equal = i < n && x == limit;
    const uint64_t em = __builtin_amdgcn_ballot_w64(equal), below = (1ull << l) - 1;
    if (l == 0) wave_equal[w] = __popcll(em);
    __syncthreads();
    int e = equal_before + __popcll(em & below);
    for (int y = 0; y < WAVES; ++y) {
      if (y < w) e += wave_equal[y];
      equal_before += wave_equal[y];
    }
    const bool kept = i < n && (x > limit || (equal && e < stay_equal));
    const bool hole = i < p.budget && !kept, filler = i >= p.budget && kept;
    const uint64_t hm = __builtin_amdgcn_ballot_w64(hole), fm = __builtin_amdgcn_ballot_w64(filler);
    if (l == 0) wave_out[w] = __popcll(hm) | __popcll(fm) << 16;
    __syncthreads();
    int at_h = holes_before + __popcll(hm & below), at_f = fillers_before + __popcll(fm & below);
    for (int y = 0; y < WAVES; ++y) {
      const int h = wave_out[y] & 0xffff, f = wave_out[y] >> 16;
      if (y < w) { at_h += h; at_f += f; }
      holes_before += h;
      fillers_before += f;
    }
    if (hole) holes[at_h] = i;
    if (filler) fillers[at_f] = i;
  }
  __syncthreads();                         // the lists are this workgroup's own
  for (int i = t; i < fillers_before; i += NT) {
    const int from = fillers[i], to = holes[i];
    weights[to] = weights[from];
    positions[to] = positions[from];
  }
  __syncthreads();
  for (int i = p.budget + t; i < n; i += NT) weights[i] = 0.f;      // what is appended there starts from nothing
  if (t == 0) p.n_moves[pair] = fillers_before;
}

__global__ __launch_bounds__(256) void dbsp_cache_move_kernel(const dbsp_cache_evict_params p) {
  const int pair = blockIdx.x, b = pair / p.Hk, hk = pair % p.Hk, t = threadIdx.x;
  if (pair % p.Hk == 0 && blockIdx.y == 0 && t == 0 && p.lens[b] > p.budget) p.lens[b] = p.budget;
  const int lanes = p.row_bytes / 16, x = t % lanes * 16;
  const int n = min(p.n_moves[pair], ((int)blockIdx.y + 1) * kMovesPerGroup);
  for (int i = (int)blockIdx.y * kMovesPerGroup + t / lanes; i < n; i += 256 / lanes) {
    const int64_t from = p.fillers[(int64_t)pair * p.max_moves + i], to = p.holes[(int64_t)pair * p.max_moves + i];
    unsigned char *k = p.k + b * p.k_sb + hk * p.k_sh + x, *v = p.v + b * p.v_sb + hk * p.v_sh + x;
    const u32x4 kr = *reinterpret_cast<const u32x4*>(k + from * p.k_st), vr = *reinterpret_cast<const u32x4*>(v + from * p.v_st);
    *reinterpret_cast<u32x4*>(k + to * p.k_st) = kr;
    *reinterpret_cast<u32x4*>(v + to * p.v_st) = vr;
  }
}

}  // namespace

hipError_t dbsp_launch_cache_evict(const dbsp_cache_evict_params& p, hipStream_t stream) {
  dbsp_cache_choose_kernel<<<p.B * p.Hk, NT, 0, stream>>>(p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  dbsp_cache_move_kernel<<<dim3(p.B * p.Hk, (p.max_moves + kMovesPerGroup - 1) / kMovesPerGroup), 256, 0, stream>>>(p);
  return hipGetLastError();
}
