// Attention over a key/value cache where a sequence brings many queries (prompts, frames): the operator, its items and its layouts are
// those of cache_attn.hip; this kernel is for row tiles that are full, where the matrix pipe bounds.
//
// A wave has 64 queries, two tiles of 32, so that each operand of K and V that it reads from the LDS feeds two MFMAs (with 32
// queries a wave the LDS is as busy as the matrix pipe).  The unit of work is 32 keys by 32 queries; the units of 32 keys
// alternate between the query tiles.  A step has three parts that do not depend on each other,
//   K Q^T of the next unit, the probabilities of this one, V^T P^T of the one before,
// as a sequence of fenced sub-slots: one MFMA each (the pipe is busy with it for 32 clocks in which the wave can issue other
// work), a part of the softmax in three stages (difference, exponential, sum and packing), and what there is of operand reads,
// which are a step ahead of their use, and copies.
// The running max is not looked for: probabilities are formed against it as it stands, and only where a lane's sum of a unit's 16
// passes kRaiseAt (some score is far above it) is it raised, O rescaled and the unit's probabilities formed anew.
// Measured: 40 heads of 2 sequences, 1560 queries over 12,870 keys, d = 128 (822 GFLOP) 771 us, 1066 TFLOP/s where a large bf16 product
// reaches 1212 (750 - 810 from card to card once the clock has settled, up to 990 in the first dozen launches of a process); 16 heads on 4, 8192
// causal queries, 249 us, 1100 TFLOP/s.  The first loses 13 % to its last row tiles, which hold 24 rows of
// 256.  A tile of 64 keys takes a wave 3300 clocks, 2048 of them MFMAs; leaving out the operand reads takes 17 % off, the copies
// 8 %, the exponentials 9 %, the barrier 1 % (wrong results, same addresses).  At d = 64 two exponentials for every one at d = 128 and
// MFMA bound it: 48 heads, 4101 causal queries (119 GFLOP) 149 us, 800 TFLOP/s.
// K tiles of 64 keys have three places in the LDS, V tiles two; one barrier a tile publishes the next K tile and this V tile, and
// the copies of the tiles behind them follow it.  Past an item's end the last tile is copied again, to places that nobody
// reads: that costs less than branches among the sub-slots.
#include <type_traits>
#include <utility>

#include "cache_attn.hpp"

namespace {

// f(0), ..., f(N - 1), as constants
template <class F, int... I>
__device__ __forceinline__ void for_each_of(F& f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, class F>
__device__ __forceinline__ void for_each(F&& f) { for_each_of(f, std::make_integer_sequence<int, N>{}); }

template <class T, int D, int NW>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(D == 64 ? 2 : 1, D == 64 ? 2 : 1)))
void dbsp_cache_attn_long_kernel(const dbsp_cache_attn_params p) {
  using L = Lay<D>;
  constexpr int ROWS = 64 * NW, SHARE = 64 / NW, COPIES = SHARE / L::RPC;
  constexpr int SUB = 2 * L::KS;           // sub-slots of a step
  constexpr int KP = 3, VP = 2;            // places
  constexpr int kBias = 3 * 1024;
  static_assert(COPIES <= 4, "a group's copies share a destination");
  __shared__ __attribute__((aligned(1024))) unsigned char lds[(KP + VP) * L::TILE];
  const uint32_t lds_base = (uint32_t)(uintptr_t)(LDS_PTR(unsigned char))lds;
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l = threadIdx.x & 63, r = l & 31, g = l >> 5;
  Item it;
  if (!find_long_item(p, it)) return;
  const int b = __builtin_amdgcn_readfirstlane(it.b), hk = __builtin_amdgcn_readfirstlane(it.hk), rt = __builtin_amdgcn_readfirstlane(it.rt);
  const int len = len_of(p, b), q_len = q_len_of(p, b), row0 = rt * ROWS - p.row_shift;      // (rows below 0 are none)
  if (max(row0, 0) / p.G >= q_len) return; // no query here: its rows stay as they are
  const int base = len - q_len + 1;        // causal: query t sees the first base + t own keys
  const int seen = p.causal ? max(0, min(len, base + min(q_len - 1, (row0 + ROWS - 1) / p.G))) : len;
  const int pre_tiles = p.pre_tiles, n_all = own_tiles(p, b), per = (n_all + it.n - 1) / it.n, n_here = pre_tiles + tiles_of(seen);
  const int t0 = __builtin_amdgcn_readfirstlane(min(it.c * per, n_here)), t1 = __builtin_amdgcn_readfirstlane(min((it.c + 1) * per, n_here));

  // this lane's queries, one of each tile
  const int rows = p.Nq * p.G;
  Row at[2];
  bool valid[2];
  int h[2], limit[2], all_see = INT_MAX, any_sees = 0;
  u32x4 q[2][L::KS];
#pragma unroll
  for (int y = 0; y < 2; ++y) {
    const int row = row0 + 64 * w + 32 * y + r;
    at[y] = row_of(p, b, max(0, min(row, rows - 1)));
    valid[y] = row >= 0 && row < rows && at[y].t < q_len;
    h[y] = hk * p.G + at[y].g;
    limit[y] = p.causal ? max(0, min(len, base + at[y].t)) : len;
    all_see = min(all_see, valid[y] ? limit[y] : INT_MAX);
    any_sees = max(any_sees, valid[y] ? limit[y] : 0);
    const uint16_t* src = p.q + b * p.q_sb + h[y] * p.q_sh + at[y].t * p.q_st;
#pragma unroll
    for (int ks = 0; ks < L::KS; ++ks) q[y][ks] = *reinterpret_cast<const u32x4*>(src + 16 * ks + 8 * g);
  }
  // (d = 128: MFMAs read Q from accumulation registers)
#pragma unroll
  for (int y = 0; y < 2; ++y)
#pragma unroll
    for (int ks = 0; ks < L::KS; ++ks) {
      if constexpr (D == 128) asm volatile("" : "+a"(q[y][ks]));
    }
  for (int s = 16; s > 0; s >>= 1) {
    all_see = min(all_see, __shfl_xor(all_see, s));
    any_sees = max(any_sees, __shfl_xor(any_sees, s));
  }
  all_see = __builtin_amdgcn_readfirstlane(all_see);
  // the tiles that some query of this wave sees
  const bool active = __builtin_amdgcn_ballot_w64(valid[0] || valid[1]) != 0;
  const int mine = active ? __builtin_amdgcn_readfirstlane(min(t1, pre_tiles + tiles_of(any_sees))) : t0;

  // Copies: this wave's share of a tile.  Where a tile lies and how its rows are clamped changes at the ends of prefix and own keys only
  const int row_in = l / L::NCH, pch = l % L::NCH;
  struct Source {
    const unsigned char* at;               // of the tile, less kBias
    int64_t step;                          // from tile to tile
    int until;                             // tiles in front of this one are whole, and of the same list of keys
    int there;                             // rows of the tile that hold keys, as far as the offsets go by it
    uint32_t off[COPIES];
  } ksrc{nullptr, 0, 0, -1, {}}, vsrc{nullptr, 0, 0, -1, {}};
  auto aim = [&](Source& src, int t, auto is_k_tag) __attribute__((always_inline)) {
    constexpr bool IS_K = decltype(is_k_tag)::value;
    t = min(t, t1 - 1);
    const bool pre = t < pre_tiles;
    const int tok = (pre ? t : t - pre_tiles) * kCacheKeys, there = min((pre ? p.P : len) - tok, kCacheKeys) + (pre ? 2 * kCacheKeys : 0);
    const uint32_t st = IS_K ? (pre ? p.pk_st : p.k_st) : (pre ? p.pv_st : p.v_st);
    const uint16_t* from = IS_K ? (pre ? p.pk + hk * p.pk_sh : p.k + b * p.k_sb + hk * p.k_sh) : (pre ? p.pv + hk * p.pv_sh : p.v + b * p.v_sb + hk * p.v_sh);
    src.at = reinterpret_cast<const unsigned char*>(from) + (int64_t)tok * st - kBias;
    src.step = (int64_t)kCacheKeys * st;
    src.until = min(pre ? p.P / kCacheKeys : pre_tiles + len / kCacheKeys, t1);
    if (there != src.there) {
      src.there = there;
      const int last = (pre ? there - 2 * kCacheKeys : there) - 1;
#pragma unroll
      for (int x = 0; x < COPIES; ++x) {
        const int in = x * L::RPC + row_in;
        src.off[x] = min(w * SHARE + in, last) * st + ((pch ^ (IS_K ? L::k_swz(in) : L::v_swz(in))) << 4) + kBias - x * 1024;
      }
    }
  };
  constexpr std::integral_constant<bool, true> K_{};
  constexpr std::integral_constant<bool, false> V_{};
  auto aim_next = [&](Source& src, int t, auto is_k_tag) __attribute__((always_inline)) {      // from tile t - 1
    if (t < src.until) src.at += src.step;
    else aim(src, t, is_k_tag);
  };
  const uint32_t share = lds_base + w * SHARE * L::ROWB;
  // a group's destination, and its copies: the instruction's offset, x KiB, counts on both sides, and kBias keeps the source's other
  // offset from below 0
  auto copy_to = [&](uint32_t place) __attribute__((always_inline)) { set_copy_dst(share + place * L::TILE); };
  auto copy = [&](const Source& src, int x) __attribute__((always_inline)) { copy16_nth(x, src.at, src.off[x]); };
  auto copy_all = [&](const Source& src, uint32_t place) __attribute__((always_inline)) {
    copy_to(place);
#pragma unroll
    for (int x = 0; x < COPIES; ++x) copy(src, x);
  };

  // operand reads, at the place of this tile
  uint32_t k_rd[L::KS], v_rd[L::DT];
#pragma unroll
  for (int ks = 0; ks < L::KS; ++ks) k_rd[ks] = lds_base + r * L::ROWB + (((2 * ks + g) ^ L::k_swz(r)) << 4);
  {
    const int hh = (l >> 4) & 1, key = 4 * g + ((l & 15) >> 2), a4 = l & 3;
#pragma unroll
    for (int dt = 0; dt < L::DT; ++dt)
      v_rd[dt] = lds_base + KP * L::TILE + key * L::ROWB + ((((4 * dt) ^ L::v_swz(key)) + 2 * hh + (a4 >> 1)) << 4) + (a4 & 1) * 8;
  }
  u32x4 kf[L::KS], vf[L::KS];              // operands: of V by 16-key step * DT + d-tile
  auto read_k = [&](int ks, int half) __attribute__((always_inline)) { kf[ks] = *(LDS_PTR(u32x4))(uintptr_t)(k_rd[ks] + half * 32 * L::ROWB); };
  auto read_v = [&](int x, int part, int half) __attribute__((always_inline)) {      // part 0, 1: keys 0 .. 7, 8 .. 15 of its 16
    const uint32_t a = v_rd[x % L::DT] + (32 * half + 16 * (x / L::DT) + 8 * part) * L::ROWB;
    const u32x2 v = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(uintptr_t)(a)));
    vf[x][2 * part] = v.x;
    vf[x][2 * part + 1] = v.y;
  };

  f32x16 o[2][L::DT], s[2];                // by query tile
  u32x4 pr[2][2];                          // probabilities by query tile and 16-key step
  f32x16 zero;
#pragma unroll
  for (int e = 0; e < 16; ++e) zero[e] = 0.f;
#pragma unroll
  for (int y = 0; y < 2; ++y)
#pragma unroll
    for (int dt = 0; dt < L::DT; ++dt) o[y][dt] = zero;
  float mc[2] = {-FLT_MAX, -FLT_MAX}, sum[2] = {0.f, 0.f};      // max * scale_log2
  const float c = p.scale_log2;

  // the key at which query tile y's scores of a unit at `key` end, less the lane group's offset
  auto mask = [&](int y, bool pre, int key) __attribute__((always_inline)) {
    const int left = (pre ? p.P : limit[y]) - key - 4 * g;
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (8 * (e / 4) + e % 4 >= left) s[y][e] = -INFINITY;
  };
  auto needs_mask = [&](int t) { return t < pre_tiles ? (t + 1) * kCacheKeys > p.P : (t - pre_tiles + 1) * kCacheKeys > all_see; };
  auto exp_at = [](int j) constexpr { return 1 + j * (SUB - 4) / 16; };

  // Step of query tile Y in half HALF of a tile: copies from `src` to its place where there are any.
  auto step = [&](auto y_tag, auto half_tag, const Source* src, uint32_t place) __attribute__((always_inline)) {
    constexpr int Y = decltype(y_tag)::value, HALF = decltype(half_tag)::value, N = 1 - Y;
    float xs[16], ps[16], l0 = 0.f, l1 = 0.f;
    bool far = false;
    if constexpr (HALF == 0) copy_to(place);
    for_each<SUB>([&](auto z_tag) __attribute__((always_inline)) {
      constexpr int z = decltype(z_tag)::value, x = z / 2;
      if constexpr (z % 2 == 0) {
        s[N] = T::mfma(kf[x], q[N][x], x == 0 ? zero : s[N]);
      } else {
        o[N][x % L::DT] = T::mfma(vf[x], pr[N][x / L::DT], o[N][x % L::DT]);
      }
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        if (z == exp_at(j) - 1) xs[j] = __builtin_fmaf(s[Y][j], c, -mc[Y]);
        if (z == exp_at(j)) ps[j] = __builtin_amdgcn_exp2f(xs[j]);
        if (z == exp_at(j) + 1) {
          if (j == 0) l0 = ps[0];
          else if (j == 1) l1 = ps[1];
          else if (j & 1) l1 += ps[j];
          else l0 += ps[j];
          if (j & 1) {
            uint32_t both = T::pack(ps[j - 1], ps[j]);
            asm volatile("" : "+v"(both));      // here, not behind the branch at the step's end
            pr[Y][j / 8][j % 8 / 2] = both;
          }
        }
      }
      // operand x is used a last time in sub-slots 2 x and 2 x + 1 of the first step, and next at the same place of the second: its
      // three reads are dealt evenly over both (K of the next 32 keys: k_rd is at the next tile in the second half)
      constexpr int rd = Y * SUB + z - 1, rx = rd / 3;
      if constexpr (rd >= 0 && rx < L::KS) {
        if constexpr (rd % 3 == 0) read_k(rx, 1 - HALF);
        else read_v(rx, rd % 3 - 1, HALF);
      }
      if constexpr (HALF == 0 && z % (SUB / 4) == SUB / 8 && z * 4 / SUB < COPIES) copy(*src, z * 4 / SUB);
      if constexpr (z == SUB - 2) {        // (a sub-slot ahead of the branch)
        l0 += l1;
        far = __builtin_amdgcn_ballot_w64(l0 > kRaiseAt) != 0;
      }
      __builtin_amdgcn_sched_barrier(0);
    });
    if (__builtin_expect(far, 0)) {
      float top = s[Y][0];
#pragma unroll
      for (int e = 1; e < 16; ++e) top = fmaxf(top, s[Y][e]);
      const float to = fmaxf(mc[Y], max_xor32(top) * c), f = __builtin_amdgcn_exp2f(mc[Y] - to);
      mc[Y] = to;
      sum[Y] *= f;
#pragma unroll
      for (int dt = 0; dt < L::DT; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[Y][dt][e] *= f;
      l0 = 0.f;
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        const float a = __builtin_amdgcn_exp2f(__builtin_fmaf(s[Y][e], c, -to)), z = __builtin_amdgcn_exp2f(__builtin_fmaf(s[Y][e + 1], c, -to));
        l0 += a + z;
        pr[Y][e / 8][e % 8 / 2] = T::pack(a, z);
      }
    }
    sum[Y] += l0;
  };
  constexpr std::integral_constant<int, 0> C0{};
  constexpr std::integral_constant<int, 1> C1{};

  // a product of zeros takes the place of the one behind the step before the first
#pragma unroll
  for (int x = 0; x < L::KS; ++x) vf[x] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
  for (int st = 0; st < 2; ++st) pr[1][st] = u32x4{0u, 0u, 0u, 0u};
  if (t0 < t1) {
    aim(ksrc, t0, K_);
    copy_all(ksrc, 0);
    aim(vsrc, t0, V_);
    copy_all(vsrc, KP);
    aim(ksrc, t0 + 1, K_);
    copy_all(ksrc, 1);
    wait_all();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (t0 < mine) {
#pragma unroll
      for (int ks = 0; ks < L::KS; ++ks) read_k(ks, 0);
#pragma unroll
      for (int ks = 0; ks < L::KS; ++ks) s[0] = T::mfma(kf[ks], q[0][ks], ks == 0 ? zero : s[0]);
      if (needs_mask(t0)) mask(0, t0 < pre_tiles, (t0 < pre_tiles ? t0 : t0 - pre_tiles) * kCacheKeys);
    }
  }
  uint32_t kp = 0, vp = 0;                 // places of this tile
  int m_n = t0 < t1 ? needs_mask(t0) : 0;
  for (int t = t0; t < t1; ++t) {
    wait_all();                            // this wave's copies have landed, and its reads of what the next ones overwrite are done
    __builtin_amdgcn_s_barrier();          // everybody's
    asm volatile("" ::: "memory");
    const uint32_t k_next = kp == KP - 1 ? 0 : kp + 1, k_to = k_next == KP - 1 ? 0 : k_next + 1, v_next = vp ^ 1;
    aim_next(vsrc, t + 1, V_);
    aim_next(ksrc, t + 2, K_);
    if (t < mine) {
      const bool pre = t < pre_tiles, pre_n = t + 1 < pre_tiles;
      const int key = (pre ? t : t - pre_tiles) * kCacheKeys, key_n = (pre_n ? t + 1 : t + 1 - pre_tiles) * kCacheKeys;
      const int m = m_n;
      m_n = __builtin_amdgcn_readfirstlane(needs_mask(t + 1));
      step(C0, C0, &vsrc, KP + v_next);
      if (m) mask(1, pre, key);
      step(C1, C0, &ksrc, k_to);
      if (m) mask(0, pre, key + 32);
#pragma unroll
      for (int ks = 0; ks < L::KS; ++ks) k_rd[ks] += (k_next - kp) * L::TILE;
      step(C0, C1, nullptr, 0);
      if (m) mask(1, pre, key + 32);
      step(C1, C1, nullptr, 0);
#pragma unroll
      for (int dt = 0; dt < L::DT; ++dt) v_rd[dt] += (v_next - vp) * L::TILE;
      if (m_n) mask(0, pre_n, key_n);
    } else {
      copy_all(vsrc, KP + v_next);
      copy_all(ksrc, k_to);
    }
    kp = k_next;
    vp = v_next;
  }
  if (t0 < mine) {
#pragma unroll
    for (int x = 0; x < L::KS; ++x) o[1][x % L::DT] = T::mfma(vf[x], pr[1][x / L::DT], o[1][x % L::DT]);
  }
  wait_all();                              // the LDS is somebody else's once this wave has ended

#pragma unroll
  for (int y = 0; y < 2; ++y) {
    const float all = sum_xor32(sum[y]);
    if (!valid[y]) continue;
    const bool none = __builtin_bit_cast(uint32_t, all) == 0u;
    store_row<T, D>(p, it, o[y], at[y], h[y], 64 * w + 32 * y + r, g, none ? 0.f : 1.f / all, none ? -INFINITY : mc[y] + __builtin_amdgcn_logf(all));
  }
}

}  // namespace

template <int NW>
hipError_t launch(const dbsp_cache_attn_params& p, int d, bool fp16, int grid, hipStream_t stream) {
  if (d == 64) {
    if (fp16) dbsp_cache_attn_long_kernel<Fp16, 64, NW><<<grid, 64 * NW, 0, stream>>>(p);
    else dbsp_cache_attn_long_kernel<Bf16, 64, NW><<<grid, 64 * NW, 0, stream>>>(p);
  } else {
    if (fp16) dbsp_cache_attn_long_kernel<Fp16, 128, NW><<<grid, 64 * NW, 0, stream>>>(p);
    else dbsp_cache_attn_long_kernel<Bf16, 128, NW><<<grid, 64 * NW, 0, stream>>>(p);
  }
  return hipGetLastError();
}

hipError_t dbsp_launch_cache_attn_long(const dbsp_cache_attn_params& p, int d, bool fp16, int grid, hipStream_t stream) {
  return launch<kLongWaves>(p, d, fp16, grid, stream);
}
