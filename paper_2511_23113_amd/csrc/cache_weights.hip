// The attention that the own keys of a key/value cache draw, where the queries are too many for their scores to be kept:
//   W[b, hk, slot] = decay W + sum over the rows (token, head of the group) that see the slot of exp2(scale_log2 q.k - LSE2[row]),
// the scores formed anew, LSE2 (to base 2) from the attention kernel or the merge behind it.
//
// 2 d flops and an exponential a (row, key).  Bound by the vector pipe: at d = 128 a step of 32 keys by 32 rows has 8 MFMAs and 51 other vector
// instructions, and 33 more are its share of a tile's copies (addresses from two 64-bit strides), of its rows and of the kernel's ends; a masked step has
// another 33, which the others jump over.  A workgroup has 256 keys of
// a (sequence, KV head), 64 a wave with K as an operand in registers, and goes over the rows in steps of 32, Q by way of the LDS, 64 rows at a
// time in three places (64 keys a wave, as each operand of Q then feeds two MFMAs).  As in cache_attn_long.hip a step is a sequence
// of fenced sub-slots: an MFMA of the next step's S^T = K Q^T, two exponentials of this one's, an operand read.  Lane r has
// row r of a step and sums 32 keys; the lanes are added once, at the end.  Where there are fewer workgroups than the chip
// holds the rows are cut into p.row_parts, whose sums a small launch adds (2 KV heads of 4 query heads each, 4096 causal queries: 387 us
// attention included without, 120 so).
// Measured: 80 (sequence, head) pairs of 4680 keys and 1560 queries (150 GFLOP) 180 - 195 us, 770 - 830 TFLOP/s; with 32 keys a wave and Q by way of
// registers 320.
#include <hip/hip_runtime.h>

#include <type_traits>
#include <utility>

#include "cache_attn.hpp"

namespace {

template <class F, int... I>
__device__ __forceinline__ void for_each_of(F& f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, class F>
__device__ __forceinline__ void for_each(F&& f) { for_each_of(f, std::make_integer_sequence<int, N>{}); }

template <class T, int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2)))
void dbsp_cache_weights_kernel(const dbsp_cache_attn_params p) {
  using L = Lay<D>;
  constexpr int RT = 64, PLACES = 3, TILE = RT * L::ROWB, COPIES = L::COPIES, SUB = L::KS;      // sub-slots of a step
  __shared__ __attribute__((aligned(1024))) unsigned char lds[PLACES * TILE];
  const uint32_t lds_base = (uint32_t)(uintptr_t)(LDS_PTR(unsigned char))lds;
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l = threadIdx.x & 63, r = l & 31, g = l >> 5;
  const int b = blockIdx.x / p.Hk, hk = blockIdx.x % p.Hk, part = blockIdx.z;
  const int len = len_of(p, b), q_len = q_len_of(p, b), key0 = blockIdx.y * kWeightKeys, my_key0 = key0 + 64 * w;
  if (key0 >= len) return;
  // rows of this part; causal ones begin at the first query that sees key0
  const int base = len - q_len + 1;        // query t sees the first base + t own keys
  const int t_first = p.causal ? min(q_len, max(0, key0 + 1 - base)) : 0, t_per = (q_len - t_first + p.row_parts - 1) / p.row_parts;
  const int row0 = min(t_first + part * t_per, q_len) * p.G, row1 = min(t_first + (part + 1) * t_per, q_len) * p.G;
  const int steps = (row1 - row0 + 31) / 32;

  u32x4 k[2][L::KS];
#pragma unroll
  for (int y = 0; y < 2; ++y) {
    const unsigned char* src = reinterpret_cast<const unsigned char*>(p.k + b * p.k_sb + hk * p.k_sh) + (int64_t)min(my_key0 + 32 * y + r, len - 1) * p.k_st;
#pragma unroll
    for (int ks = 0; ks < L::KS; ++ks) k[y][ks] = *reinterpret_cast<const u32x4*>(src + 32 * ks + 16 * g);
  }
  f32x16 zero;
#pragma unroll
  for (int e = 0; e < 16; ++e) zero[e] = 0.f;
  f32x16 acc[2] = {zero, zero};

  // Copies: lane l moves 16 bytes of rows 16 w + x RPC + l / NCH of a tile; token and head of its row go on by 64 rows a tile
  const uint16_t* const q0 = p.q + b * p.q_sb + (int64_t)hk * p.G * p.q_sh;
  const int row_in = l / L::NCH, pch = l % L::NCH, t64 = 64 / p.G, g64 = 64 % p.G;
  int ct[COPIES], cg[COPIES], copied = row0;
#pragma unroll
  for (int x = 0; x < COPIES; ++x) {
    const int row = row0 + 16 * w + x * L::RPC + row_in;
    ct[x] = row / p.G;
    cg[x] = row % p.G;
  }
  const int t_last = (row1 - 1) / p.G;
  auto copy_tile = [&](uint32_t place) __attribute__((always_inline)) {      // rows past the end: some row of the last query
    if (copied >= row1) return;
    copied += RT;
#pragma unroll
    for (int x = 0; x < COPIES; ++x) {
      const int in = x * L::RPC + row_in;
      const uint16_t* src = q0 + min(ct[x], t_last) * p.q_st + cg[x] * p.q_sh + ((pch ^ L::k_swz(in)) << 3);
      asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(src), "s"(lds_base + place * TILE + 16 * w * L::ROWB + x * 1024) : "memory");
      ct[x] += t64;
      cg[x] += g64;
      if (cg[x] >= p.G) {
        cg[x] -= p.G;
        ++ct[x];
      }
    }
  };
  // this lane's row of a step: LSE, and how many own keys it sees
  const int t32 = 32 / p.G, g32 = 32 % p.G;
  int row = row0 + r, rt = row / p.G, rg = row % p.G;
  const float* const lse0 = p.row_lse + ((int64_t)b * p.H + hk * p.G) * p.Nq;
  auto next_row = [&](float& lse, int& limit) __attribute__((always_inline)) {
    lse = row < row1 ? lse0[(int64_t)rg * p.Nq + rt] : INFINITY;      // a row that is not there: probabilities of 0
    limit = p.causal ? base + rt : len;
    row += 32;
    rt += t32;
    rg += g32;
    if (rg >= p.G) {
      rg -= p.G;
      ++rt;
    }
  };
  uint32_t q_rd[L::KS];
#pragma unroll
  for (int ks = 0; ks < L::KS; ++ks) q_rd[ks] = lds_base + r * L::ROWB + (((2 * ks + g) ^ L::k_swz(r)) << 4);
  u32x4 qf[L::KS];
  f32x16 s[2];                             // by key tile
  const float c = p.scale_log2;
  float lse[2];
  int limit[2];
  // Key tile Y of the step of rows PAR: its exponentials; the products of the unit behind it, which for Y == 0 are the last of this
  // step's rows: Q of the next ones (half 1 - PAR of a tile, q_rd at it) is read behind them.
  auto step = [&](auto y_tag, auto par_tag) __attribute__((always_inline)) {
    constexpr int Y = decltype(y_tag)::value, PAR = decltype(par_tag)::value, N = 1 - Y, PER = 16 / SUB;
    // a row without a key has LSE -inf, and no probabilities
    const float ls = __builtin_bit_cast(uint32_t, lse[PAR]) == 0xff800000u ? INFINITY : lse[PAR];
    float xs[16], ps[16];
    for_each<SUB>([&](auto z_tag) __attribute__((always_inline)) {
      constexpr int z = decltype(z_tag)::value;
      s[N] = T::mfma(k[N][z], qf[z], z == 0 ? zero : s[N]);
      if constexpr (Y == 0) qf[z] = *(LDS_PTR(u32x4))(uintptr_t)(q_rd[z] + (1 - PAR) * 32 * L::ROWB);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int at = e / PER;
        if (z == (at > 0 ? at - 1 : 0)) xs[e] = __builtin_fmaf(s[Y][e], c, -ls);
        if (z == at) ps[e] = __builtin_amdgcn_exp2f(xs[e]);
        if (z == (at + 1 < SUB ? at + 1 : at)) {
          acc[Y][e] += ps[e];
          asm volatile("" : "+v"(acc[Y][e]));      // here, not where the sum is needed next
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  auto mask = [&](int y, int par) __attribute__((always_inline)) {
    const int left = limit[par] - my_key0 - 32 * y - 4 * g;
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (8 * (e / 4) + e % 4 >= left) s[y][e] = -INFINITY;
  };
  constexpr std::integral_constant<int, 0> P0{};
  constexpr std::integral_constant<int, 1> P1{};
  // rows from here on see all of the wave's keys (steps in front of it are masked)
  const int free_row = p.causal ? max(0, min(q_len, my_key0 + 64 - base)) * p.G : 0;

  if (steps > 0) {
    copy_tile(0);
    copy_tile(1);
    wait_all();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    next_row(lse[0], limit[0]);
#pragma unroll
    for (int ks = 0; ks < L::KS; ++ks) qf[ks] = *(LDS_PTR(u32x4))(uintptr_t)q_rd[ks];
#pragma unroll
    for (int ks = 0; ks < L::KS; ++ks) s[0] = T::mfma(k[0][ks], qf[ks], ks == 0 ? zero : s[0]);
    if (row0 < free_row) mask(0, 0);
  }
  uint32_t place = 0;
  for (int i = 0; i < steps; i += 2) {     // a tile of 64 rows
    wait_all();                            // the next tile has landed, and this wave has read the one before this
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    const uint32_t next = place == PLACES - 1 ? 0 : place + 1;
    copy_tile(next == PLACES - 1 ? 0 : next + 1);
    next_row(lse[1], limit[1]);
    step(P0, P0);
    if (row0 + 32 * i < free_row) mask(1, 0);
    step(P1, P0);
    if (row0 + 32 * (i + 1) < free_row) mask(0, 1);
#pragma unroll
    for (int ks = 0; ks < L::KS; ++ks) q_rd[ks] += (next - place) * TILE;
    place = next;
    next_row(lse[0], limit[0]);
    step(P0, P1);
    if (row0 + 32 * (i + 1) < free_row) mask(1, 1);
    step(P1, P1);
    if (row0 + 32 * (i + 2) < free_row) mask(0, 0);
  }
  wait_all();
#pragma unroll
  for (int y = 0; y < 2; ++y) {
#pragma unroll
    for (int e = 0; e < 16; ++e)
#pragma unroll
      for (int x = 16; x > 0; x >>= 1) acc[y][e] += __shfl_xor(acc[y][e], x);
    // lane e of each half stores its key e
    float mine = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) mine = r == e ? acc[y][e] : mine;
    const int key = my_key0 + 32 * y + 8 * (r / 4) + 4 * g + r % 4;
    if (r < 16 && key < len) {
      const int64_t at = (int64_t)blockIdx.x * p.cap + key;
      if (p.row_parts > 1) p.part_w[(int64_t)part * p.B * p.Hk * p.cap + at] = mine;
      else p.weights[at] = (p.decay == 0.f ? 0.f : p.decay * p.weights[at]) + mine;
    }
  }
}

__global__ __launch_bounds__(256) void dbsp_cache_add_weights_kernel(const dbsp_cache_attn_params p) {
  const int slot = blockIdx.y * 256 + threadIdx.x;
  if (slot >= len_of(p, blockIdx.x / p.Hk)) return;
  const int64_t at = (int64_t)blockIdx.x * p.cap + slot, step = (int64_t)p.B * p.Hk * p.cap;
  float sum = 0.f;
  for (int y = 0; y < p.row_parts; ++y) sum += p.part_w[y * step + at];
  p.weights[at] = (p.decay == 0.f ? 0.f : p.decay * p.weights[at]) + sum;
}

}  // namespace

hipError_t dbsp_launch_cache_weights(const dbsp_cache_attn_params& p, int d, bool fp16, hipStream_t stream) {
  const dim3 grid(p.B * p.Hk, (p.cap + kWeightKeys - 1) / kWeightKeys, p.row_parts);
  if (d == 64) {
    if (fp16) dbsp_cache_weights_kernel<Fp16, 64><<<grid, 256, 0, stream>>>(p);
    else dbsp_cache_weights_kernel<Bf16, 64><<<grid, 256, 0, stream>>>(p);
  } else {
    if (fp16) dbsp_cache_weights_kernel<Fp16, 128><<<grid, 256, 0, stream>>>(p);
    else dbsp_cache_weights_kernel<Bf16, 128><<<grid, 256, 0, stream>>>(p);
  }
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && p.row_parts > 1) {
    dbsp_cache_add_weights_kernel<<<dim3(p.B * p.Hk, (p.cap + 255) / 256), 256, 0, stream>>>(p);
    e = hipGetLastError();
  }
  return e;
}
