// Norms and rotations of queries and keys, from a projection's output to the layout that attention takes or to a paged cache, and their
// gradients.
//
//   n = (x - mu) r gain + bias,  r = 1 / sqrt(mean((x - mu)^2) + eps),  (y1, y2) = (n1 cos a - n2 sin a, n1 sin a + n2 cos a),
//   dn = the rotation by -a of dy,  dgain = sum dn xh,  dbias = sum dn,  e = dn gain,  dx = r (e - mean(e xh) xh - [mean(e)]),  xh = (x - mu) r.
//
// A row (one head of one token) has d / 8 lanes, which hold four pairs each, in registers from the load to the store: sums over a
// row are data-parallel primitives inside 16 lanes.  A workgroup takes 16 (d = 64: 32) tokens and goes over its heads, so an
// angle's cosine and sine are formed once for all of them.  Angles are formed in 64 bits, in turns, and only what is left of whole
// turns is rounded to f32.
//
// Bound by reading and writing once: 40 + 40 heads of 128 of 32,760 tokens (1342 MB) 263 us, 5.1 TB/s, where a large copy reaches 5.0; their
// gradients at 17,550 tokens (1078 MB) 209 us and 4.7 for the sums of gains.  Smaller ones by a workgroup's first loads (lengths and
// positions, then rows) and by what comes before its first row, some 200 instructions: 12,303 tokens of 30 + 10 heads of 64 (126 MB) 30 us,
// 4.2 TB/s, where one head a workgroup takes 57.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "attn_common.hpp"
#include "rows_params.hpp"

namespace {

typedef _Float16 f16x2r __attribute__((ext_vector_type(2)));

struct RowBf16 {
  static __device__ __forceinline__ float lo(uint32_t u) { return __builtin_bit_cast(float, u << 16); }
  static __device__ __forceinline__ float hi(uint32_t u) { return __builtin_bit_cast(float, u & 0xffff0000u); }
  static __device__ __forceinline__ uint32_t pack(float a, float b) { return pack_bf16x2(a, b); }
};
struct RowFp16 {
  static __device__ __forceinline__ float lo(uint32_t u) { return (float)__builtin_bit_cast(f16x2r, u).x; }
  static __device__ __forceinline__ float hi(uint32_t u) { return (float)__builtin_bit_cast(f16x2r, u).y; }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    f32x2 f = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, f16x2r));      // round to nearest even
  }
};

// Eight values of a row: those of a lane's four pairs.
struct Pairs { f32x4 a, b; };

// Where a lane's values lie: 16 bytes at `at`, or with HALVES 8 bytes at `at` and 8 at `other`.
struct Place { int at, other; };
template <bool HALVES>
__device__ __forceinline__ Place place_of(int c, int turned) {
  if (HALVES && 4 * c < turned) return {4 * c, turned + 4 * c};
  return {8 * c, 8 * c + 4};
}

// Loads and stores past the caches (STREAM): see kRowStream.
template <bool STREAM, class V>
__device__ __forceinline__ V load(const V* from) {
  if constexpr (STREAM) return __builtin_nontemporal_load(from);
  else return *from;
}
template <bool STREAM, class V>
__device__ __forceinline__ void store(V* to, V v) {
  if constexpr (STREAM) __builtin_nontemporal_store(v, to);
  else *to = v;
}
template <bool HALVES, bool STREAM>
__device__ __forceinline__ u32x4 load_row(const uint16_t* row, Place at) {
  if constexpr (HALVES) {
    const u32x2 x = load<STREAM>(reinterpret_cast<const u32x2*>(row + at.at)), y = load<STREAM>(reinterpret_cast<const u32x2*>(row + at.other));
    return {x.x, x.y, y.x, y.y};
  } else {
    return load<STREAM>(reinterpret_cast<const u32x4*>(row + at.at));
  }
}
template <bool HALVES, bool STREAM>
__device__ __forceinline__ void store_row(uint16_t* row, Place at, u32x4 v) {
  if constexpr (HALVES) {
    store<STREAM>(reinterpret_cast<u32x2*>(row + at.at), u32x2{v.x, v.y});
    store<STREAM>(reinterpret_cast<u32x2*>(row + at.other), u32x2{v.z, v.w});
  } else {
    store<STREAM>(reinterpret_cast<u32x4*>(row + at.at), v);
  }
}

// (halves: the lane's first four values are its pairs' first ones, also where they are not turned and only a norm looks at them)
template <class T, bool HALVES>
__device__ __forceinline__ Pairs unpack(u32x4 v) {
  if constexpr (HALVES) return {{T::lo(v.x), T::hi(v.x), T::lo(v.y), T::hi(v.y)}, {T::lo(v.z), T::hi(v.z), T::lo(v.w), T::hi(v.w)}};
  else return {{T::lo(v.x), T::lo(v.y), T::lo(v.z), T::lo(v.w)}, {T::hi(v.x), T::hi(v.y), T::hi(v.z), T::hi(v.w)}};
}
template <class T, bool HALVES>
__device__ __forceinline__ u32x4 pack(const Pairs& x) {
  if constexpr (HALVES) return {T::pack(x.a[0], x.a[1]), T::pack(x.a[2], x.a[3]), T::pack(x.b[0], x.b[1]), T::pack(x.b[2], x.b[3])};
  else return {T::pack(x.a[0], x.b[0]), T::pack(x.a[1], x.b[1]), T::pack(x.a[2], x.b[2]), T::pack(x.a[3], x.b[3])};
}

// Of gains or biases, the lane's.
template <class T, bool HALVES>
__device__ __forceinline__ Pairs weights_of(const void* w, bool f32, float none, Place at) {
  Pairs x;
  if (!w) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x.a[i] = x.b[i] = none;
    return x;
  }
  if (!f32) return unpack<T, HALVES>(load_row<HALVES, false>(static_cast<const uint16_t*>(w), at));
  const f32x4 u = *reinterpret_cast<const f32x4*>(static_cast<const float*>(w) + at.at), v = *reinterpret_cast<const f32x4*>(static_cast<const float*>(w) + at.other);
  if constexpr (HALVES) return {u, v};
  else return {{u.x, u.z, v.x, v.z}, {u.y, u.w, v.y, v.w}};
}

// Sum over a row's lanes, in each of them.
template <int LANES>
__device__ __forceinline__ float over_lanes(float x) {
  auto from = [](float v, auto ctrl) { return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(ctrl)::value, 0xf, 0xf, false)); };
  x += from(x, std::integral_constant<int, 0xb1>{});       // quad_perm: lane ^ 1, lane ^ 2
  x += from(x, std::integral_constant<int, 0x4e>{});
  x += from(x, std::integral_constant<int, 0x141>{});      // row_half_mirror: the other quad of eight
  if constexpr (LANES == 16) x += from(x, std::integral_constant<int, 0x140>{});      // row_mirror: the other eight
  return x;
}
__device__ __forceinline__ float sum8(const Pairs& x) { return ((x.a[0] + x.a[1]) + (x.a[2] + x.a[3])) + ((x.b[0] + x.b[1]) + (x.b[2] + x.b[3])); }
__device__ __forceinline__ float dot8(const Pairs& x, const Pairs& y) {
  float s = x.a[0] * y.a[0], u = x.b[0] * y.b[0];
#pragma unroll
  for (int i = 1; i < 4; ++i) {
    s = __builtin_fmaf(x.a[i], y.a[i], s);
    u = __builtin_fmaf(x.b[i], y.b[i], u);
  }
  return s + u;
}

// x becomes (x - mu) r; returns r.
template <int D, int KIND>
__device__ __forceinline__ float normalise(Pairs& x, float eps) {
  if constexpr (KIND == 2) {
    const float mu = over_lanes<D / 8>(sum8(x)) * (1.f / D);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x.a[i] -= mu;
      x.b[i] -= mu;
    }
  }
  const float r = __builtin_amdgcn_rsqf(__builtin_fmaf(over_lanes<D / 8>(dot8(x, x)), 1.f / D, eps));      // (to a unit of the last place)
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x.a[i] *= r;
    x.b[i] *= r;
  }
  return r;
}

// Pairs that are not turned are `still`: their cosine is 1 and their sine 0, but 0 times an infinite neighbour would not be nothing.
struct Turn {
  f32x4 c, s;
  bool still[4];
};
template <bool BACK>
__device__ __forceinline__ void rotate(Pairs& x, const Turn& t, bool all_turned) {
  const Pairs was = x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float a = x.a[i], b = x.b[i], s = BACK ? -t.s[i] : t.s[i];
    x.a[i] = __builtin_fmaf(a, t.c[i], -(b * s));
    x.b[i] = __builtin_fmaf(b, t.c[i], a * s);
  }
  if (all_turned) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x.a[i] = t.still[i] ? was.a[i] : x.a[i];
    x.b[i] = t.still[i] ? was.b[i] : x.b[i];
  }
}

// Sine and cosine of 2 pi x, |x| <= 1 / 2: by quarters of a turn down to |y| <= pi / 4, where the Taylor polynomials of degree 9 and 8 are off by
// less than 2^-25.  (12,303 tokens of 30 + 10 heads of 64, layer norm: 33.6 us with the math library's and gains apart from the rotation, 31.4 so)
__device__ __forceinline__ void sine_cosine(float x, float& sine, float& cosine) {
  const float quarters = __builtin_rintf(4.f * x), y = __builtin_fmaf(quarters, -0.25f, x) * 6.2831853071795865f, z = y * y;
  float s = __builtin_fmaf(z, 1.f / 362880.f, -1.f / 5040.f), c = __builtin_fmaf(z, 1.f / 40320.f, -1.f / 720.f);
  s = __builtin_fmaf(z, s, 1.f / 120.f);
  c = __builtin_fmaf(z, c, 1.f / 24.f);
  s = __builtin_fmaf(z, s, -1.f / 6.f);
  c = __builtin_fmaf(z, c, -0.5f);
  s = __builtin_fmaf(z * y, s, y);
  c = __builtin_fmaf(z, c, 1.f);
  const int q = (int)quarters;             // -2 .. 2
  const uint32_t s_bits = __builtin_bit_cast(uint32_t, q & 1 ? c : s) ^ ((uint32_t)(q & 2) << 30);
  const uint32_t c_bits = __builtin_bit_cast(uint32_t, q & 1 ? s : c) ^ ((uint32_t)((q + 1) & 2) << 30);
  sine = __builtin_bit_cast(float, s_bits);
  cosine = __builtin_bit_cast(float, c_bits);
}

// Of a lane's pairs 4 c .. 4 c + 3, at the position of token n of sequence b (`place` where positions are not given).
__device__ __forceinline__ Turn turn_of(const dbsp_rows_params& p, int c, int b, int n, int place) {
  Turn t;
  double turns[4];
  int at[4];
  const int32_t* const here = p.positions + (b * p.pos_sb + n * p.pos_st);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int pair = 4 * c + i, axis = (pair >= p.ends[0]) + (pair >= p.ends[1]) + (pair >= p.ends[2]);
    turns[i] = p.turns[pair];              // (0 from p.turned on)
    t.still[i] = pair >= p.turned;
    at[i] = place;
    if (p.positions) at[i] = here[pair < p.turned ? axis : 0];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    turns[i] *= (double)at[i];
    float sine, cosine;
    sine_cosine((float)(turns[i] - __builtin_rint(turns[i])), sine, cosine);
    t.s[i] = sine;
    t.c[i] = cosine;
  }
  return t;
}

// Which of a launch's tensors a group of heads is of, and its first and last head.
struct Heads { int part, h0, h1; };
__device__ __forceinline__ Heads heads_of(const dbsp_rows_params& p, int group) {
  int part = 0;
  while (part < 2 && group >= p.part[part].groups) group -= p.part[part++].groups;
  const int h0 = group * p.part[part].per;
  return {part, h0, min(h0 + p.part[part].per, p.part[part].heads)};
}

template <class T, int D, int KIND, bool HALVES, bool PAGED, bool STREAM>
__global__ __launch_bounds__(kRowThreads) __attribute__((amdgpu_waves_per_eu(8))) void dbsp_rows_kernel(const dbsp_rows_params p) {
  constexpr int LANES = D / 8, TOKENS = kRowThreads / LANES, U = 3;
  const int c = threadIdx.x % LANES;
  const Heads at = heads_of(p, blockIdx.x % p.groups);
  const dbsp_rows_part& part = p.part[at.part];
  const unsigned i = blockIdx.x / p.groups * TOKENS + threadIdx.x / LANES, all = (unsigned)p.B * p.N, j = min(i, all - 1);
  const int b = (int)(j / p.N), n = (int)(j % p.N);
  const Place lane = place_of<HALVES>(c, p.turned);
  bool there = i < all;
  int place = n;
  uint16_t* to = part.y + b * part.y_sb + n * part.y_st;
  if constexpr (PAGED) {
    const int len = max(0, min(p.lens[b], p.cap)), fresh = p.new_lens ? max(0, min(p.new_lens[b], p.N)) : p.N;
    place = len - fresh + n;
    there = there && n < fresh && place >= 0;
    if (__builtin_amdgcn_ballot_w64(there) == 0) return;      // none of the wave's tokens
    if (!part.y) {
      int page = -1;
      if (there) page = p.pages[b * p.pages_stride + place / p.page_size];
      there = (unsigned)page < (unsigned)p.n_pages;
      to = part.pool + (int64_t)max(page, 0) * part.page_s + (int64_t)(place % p.page_size) * part.y_st;
    }
  }
  const uint16_t* from = part.x + b * part.x_sb + n * part.x_st;
  u32x4 in[U];
#pragma unroll
  for (int u = 0; u < U; ++u) in[u] = load_row<HALVES, STREAM>(from + min(at.h0 + u, at.h1 - 1) * part.x_sh, lane);
  // Gain, bias and rotation in one: y1 = n1 (g1 cos) - n2 (g2 sin) + (b1 cos - b2 sin) and so on, of the normed values n
  Turn t;
  Pairs cosines, sines, bias;
  const bool all_turned = 2 * p.turned == D;
  if (!part.plain) {
    t = turn_of(p, c, b, n, place);
    if constexpr (KIND != 0) {
      const Pairs gain = weights_of<T, HALVES>(part.gain, p.gains_f32, 1.f, lane);
      bias = weights_of<T, HALVES>(part.bias, p.gains_f32, 0.f, lane);
      rotate<false>(bias, t, all_turned);
      cosines = {gain.a * t.c, gain.b * t.c};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        sines.a[e] = t.still[e] ? 0.f : gain.a[e] * t.s[e];
        sines.b[e] = t.still[e] ? 0.f : gain.b[e] * t.s[e];
      }
    }
  }
  for (int h = at.h0; h < at.h1; h += U) {
    u32x4 next[U];
#pragma unroll
    for (int u = 0; u < U; ++u) next[u] = in[u];
    if (h + U < at.h1) {
#pragma unroll
      for (int u = 0; u < U; ++u) next[u] = load_row<HALVES, STREAM>(from + min(h + U + u, at.h1 - 1) * part.x_sh, lane);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (h + u >= at.h1) break;
      u32x4 out = in[u];
      if (!part.plain) {
        Pairs x = unpack<T, HALVES>(in[u]);
        if constexpr (KIND != 0) {
          normalise<D, KIND>(x, p.eps);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float n1 = x.a[e], n2 = x.b[e];
            x.a[e] = __builtin_fmaf(n1, cosines.a[e], __builtin_fmaf(-n2, sines.b[e], bias.a[e]));
            x.b[e] = __builtin_fmaf(n2, cosines.b[e], __builtin_fmaf(n1, sines.a[e], bias.b[e]));
          }
        } else {
          rotate<false>(x, t, all_turned);
        }
        out = pack<T, HALVES>(x);
      }
      if (there) store_row<HALVES, STREAM>(to + (h + u) * part.y_sh, lane, out);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) in[u] = next[u];
  }
}

template <class T, int D, int KIND, bool HALVES, bool STREAM>
__global__ __launch_bounds__(kRowThreads) void dbsp_rows_grad_kernel(const dbsp_rows_params p) {
  constexpr int LANES = D / 8, TOKENS = kRowThreads / LANES, U = 2;
  const int c = threadIdx.x % LANES;
  const int group = blockIdx.x % p.groups, walker = blockIdx.x / p.groups;
  const Heads at = heads_of(p, group);
  const dbsp_rows_part& part = p.part[at.part];
  const unsigned all = (unsigned)p.B * p.N;
  const Place lane = place_of<HALVES>(c, p.turned);
  const bool all_turned = 2 * p.turned == D;
  Pairs gain, d_gain = {}, d_bias = {};
  if constexpr (KIND != 0) gain = weights_of<T, HALVES>(part.gain, p.gains_f32, 1.f, lane);
  for (int tile = walker; tile < p.tiles; tile += p.walkers) {
    const unsigned i = (unsigned)tile * TOKENS + threadIdx.x / LANES, j = min(i, all - 1);
    const int b = (int)(j / p.N), n = (int)(j % p.N);
    const bool there = i < all;
    const uint16_t *x_at = part.x + b * part.x_sb + n * part.x_st, *dy_at = part.dy + b * part.dy_sb + n * part.dy_st;
    uint16_t* to = part.y + b * part.y_sb + n * part.y_st;
    u32x4 x_in[U], dy_in[U];
    auto load = [&](int h) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t head = min(h + u, at.h1 - 1);
        dy_in[u] = load_row<HALVES, STREAM>(dy_at + head * part.dy_sh, lane);
        if constexpr (KIND != 0) x_in[u] = load_row<HALVES, STREAM>(x_at + head * part.x_sh, lane);
      }
    };
    load(at.h0);
    const Turn t = turn_of(p, c, b, n, n);
    for (int h = at.h0; h < at.h1; h += U) {
      u32x4 x_now[U], dy_now[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        x_now[u] = x_in[u];
        dy_now[u] = dy_in[u];
      }
      if (h + U < at.h1) load(h + U);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (h + u >= at.h1) break;
        Pairs dn = unpack<T, HALVES>(dy_now[u]);
        rotate<true>(dn, t, all_turned);
        if constexpr (KIND != 0) {
          Pairs hat = unpack<T, HALVES>(x_now[u]);
          const float r = normalise<D, KIND>(hat, p.eps);
          Pairs e;
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            if (there) {
              d_gain.a[y] = __builtin_fmaf(dn.a[y], hat.a[y], d_gain.a[y]);
              d_gain.b[y] = __builtin_fmaf(dn.b[y], hat.b[y], d_gain.b[y]);
              d_bias.a[y] += dn.a[y];
              d_bias.b[y] += dn.b[y];
            }
            e.a[y] = dn.a[y] * gain.a[y];
            e.b[y] = dn.b[y] * gain.b[y];
          }
          const float along = over_lanes<LANES>(dot8(e, hat)) * (1.f / D);
          float mean = 0.f;
          if constexpr (KIND == 2) mean = over_lanes<LANES>(sum8(e)) * (1.f / D);
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            dn.a[y] = r * (__builtin_fmaf(-along, hat.a[y], e.a[y]) - mean);
            dn.b[y] = r * (__builtin_fmaf(-along, hat.b[y], e.b[y]) - mean);
          }
        }
        if (there) store_row<HALVES, STREAM>(to + (h + u) * part.y_sh, lane, pack<T, HALVES>(dn));
      }
    }
  }
  if constexpr (KIND != 0) {
    if (!p.grads) return;
    // the workgroup's sums: over the rows of a wave in registers, over the waves in the LDS, always in the same order
    constexpr int WAVES = kRowThreads / 64;
    __shared__ float sums[WAVES][2][D];
    float v[16];
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      v[y] = d_gain.a[y];
      v[4 + y] = d_gain.b[y];
      v[8 + y] = d_bias.a[y];
      v[12 + y] = d_bias.b[y];
    }
#pragma unroll
    for (int y = 0; y < 16; ++y)
#pragma unroll
      for (int by = LANES; by < 64; by *= 2) v[y] += __shfl_xor(v[y], by);
    const int wave = threadIdx.x / 64;
    if (threadIdx.x % 64 < LANES) {
#pragma unroll
      for (int y = 0; y < 16; ++y) {
        const int e = y % 4, second = y / 4 % 2;      // pair 4 c + e, its first or second place
        const int where = HALVES ? (second ? lane.other : lane.at) + e : lane.at + 2 * e + second;
        sums[wave][y / 8][where] = v[y];
      }
    }
    __syncthreads();
    // (groups of a part lie behind one another, so that a part's sums are a run of them)
    float* to = p.sums + ((int64_t)group * p.walkers + walker) * 2 * D;
    for (int y = threadIdx.x; y < 2 * D; y += kRowThreads) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) s += sums[w][y / D][y % D];
      to[y] = s;
    }
  }
}

// Gradients of gains and biases from the workgroups' sums: 16 of a gradient's values a workgroup, 64 threads each.
template <int D>
__global__ __launch_bounds__(1024) void dbsp_rows_sum_kernel(const dbsp_rows_params p) {
  constexpr int COLS = 16, WAYS = 1024 / COLS;
  const int row = blockIdx.x / (D / COLS), col = blockIdx.x % (D / COLS) * COLS + threadIdx.x % COLS, way = threadIdx.x / COLS;
  const int part = row % 2, what = row / 2;      // q's gain, k's gain, q's bias, k's bias
  const int64_t n = (int64_t)p.part[part].groups * p.walkers;
  const float* from = p.sums + (part ? (int64_t)p.part[0].groups * p.walkers * 2 * D : 0) + what * D + col;
  float s = 0.f;
#pragma unroll 4
  for (int64_t i = way; i < n; i += WAYS) s += from[i * 2 * D];
  __shared__ float sums[WAYS][COLS + 1];
  sums[way][threadIdx.x % COLS] = s;
  for (int half = WAYS / 2; half > 0; half /= 2) {
    __syncthreads();
    if (way < half) sums[way][threadIdx.x % COLS] += sums[way + half][threadIdx.x % COLS];
  }
  if (way == 0) p.grads[row * D + col] = sums[0][threadIdx.x];
}

template <class T, int D, int KIND, bool HALVES>
hipError_t launch(const dbsp_rows_params& p, bool paged, bool grad, hipStream_t stream) {
  const int grid = p.groups * (grad ? p.walkers : p.tiles);
  if (grad) {
    if (p.stream) dbsp_rows_grad_kernel<T, D, KIND, HALVES, true><<<grid, kRowThreads, 0, stream>>>(p);
    else dbsp_rows_grad_kernel<T, D, KIND, HALVES, false><<<grid, kRowThreads, 0, stream>>>(p);
    const hipError_t e = hipGetLastError();
    if (KIND == 0 || !p.grads || e != hipSuccess) return e;
    dbsp_rows_sum_kernel<D><<<4 * D / 16, 1024, 0, stream>>>(p);
  } else if (paged) {
    dbsp_rows_kernel<T, D, KIND, HALVES, true, false><<<grid, kRowThreads, 0, stream>>>(p);
  } else if (p.stream) {
    dbsp_rows_kernel<T, D, KIND, HALVES, false, true><<<grid, kRowThreads, 0, stream>>>(p);
  } else {
    dbsp_rows_kernel<T, D, KIND, HALVES, false, false><<<grid, kRowThreads, 0, stream>>>(p);
  }
  return hipGetLastError();
}

template <class T, int D>
hipError_t launch_kind(const dbsp_rows_params& p, int kind, bool halves, bool paged, bool grad, hipStream_t stream) {
  if (kind == 0) return halves ? launch<T, D, 0, true>(p, paged, grad, stream) : launch<T, D, 0, false>(p, paged, grad, stream);
  if (kind == 1) return halves ? launch<T, D, 1, true>(p, paged, grad, stream) : launch<T, D, 1, false>(p, paged, grad, stream);
  return halves ? launch<T, D, 2, true>(p, paged, grad, stream) : launch<T, D, 2, false>(p, paged, grad, stream);
}

hipError_t launch_any(const dbsp_rows_params& p, int d, bool fp16, int kind, bool halves, bool paged, bool grad, hipStream_t stream) {
  if (d == 64) return fp16 ? launch_kind<RowFp16, 64>(p, kind, halves, paged, grad, stream) : launch_kind<RowBf16, 64>(p, kind, halves, paged, grad, stream);
  return fp16 ? launch_kind<RowFp16, 128>(p, kind, halves, paged, grad, stream) : launch_kind<RowBf16, 128>(p, kind, halves, paged, grad, stream);
}

}  // namespace

hipError_t dbsp_launch_rows(const dbsp_rows_params& p, int d, bool fp16, int kind, bool halves, bool paged, hipStream_t stream) {
  return launch_any(p, d, fp16, kind, halves, paged, false, stream);
}
hipError_t dbsp_launch_rows_grad(const dbsp_rows_params& p, int d, bool fp16, int kind, bool halves, hipStream_t stream) {
  return launch_any(p, d, fp16, kind, halves, false, true, stream);
}
