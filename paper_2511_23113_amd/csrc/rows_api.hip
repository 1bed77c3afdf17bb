// C ABI of the norms and rotations of queries and keys: argument checks, workspaces, launches.
#include "rows_api.hpp"

#include <cmath>

int dbsp_rows_settle(const char* who, const dbsp_qk_rows* rows, const dbsp_head_norm* norm, const dbsp_rotary* rotary, dbsp_rows_params& p, int& kind,
                     bool& halves) {
  if (!rows) return fail(who, DBSP_EINVAL, "null pointer (rows)");
  const int32_t B = rows->B, N = rows->N, d = rows->d;
  if (rows->dtype != DBSP_BF16 && rows->dtype != DBSP_FP16) return fail(who, DBSP_EINVAL, "dtype must be DBSP_BF16 or DBSP_FP16");
  if (d != 64 && d != 128) return fail(who, DBSP_EINVAL, "head dim must be 64 or 128");
  if (B <= 0 || N <= 0) return fail(who, DBSP_EINVAL, "the numbers of sequences and tokens must be positive");
  if ((int64_t)B * N > kMost) return fail(who, DBSP_ESHAPE, "too many tokens");
  p.B = B;
  p.N = N;
  kind = norm ? norm->kind : DBSP_NORM_NONE;
  if (kind < DBSP_NORM_NONE || kind > DBSP_NORM_LAYER) return fail(who, DBSP_EINVAL, "the norm's kind must be one of DBSP_NORM_*");
  if (kind != DBSP_NORM_NONE) {
    if (!(norm->eps >= 1e-30f && norm->eps <= 1e30f)) return fail(who, DBSP_EINVAL, "eps must lie between 1e-30 and 1e30");
    if (!aligned(norm->q_gain, 16) || !aligned(norm->k_gain, 16) || !aligned(norm->q_bias, 16) || !aligned(norm->k_bias, 16))
      return fail(who, DBSP_EINVAL, "gains and biases must be 16-byte aligned");
    p.gains_f32 = norm->gains_f32 != 0;
    p.eps = norm->eps;
  }
  const int axes = rotary ? rotary->axes : 0;
  if (axes < 0 || axes > 4) return fail(who, DBSP_EINVAL, "a rotation has 0 to 4 axes");
  halves = axes > 0 && rotary->halves != 0;
  p.turned = 0;
  for (int i = 0; i < 3; ++i) p.ends[i] = INT_MAX;
  for (int i = 0; i < axes; ++i) {
    if (rotary->pairs[i] < 1 || rotary->pairs[i] > d / 2 - p.turned) return fail(who, DBSP_EINVAL, "pairs must be positive, and at most d / 2 in all");
    if (i > 0) p.ends[i - 1] = p.turned;
    p.turned += rotary->pairs[i];
  }
  if (halves && p.turned % 4 != 0) return fail(who, DBSP_EINVAL, "the pairs of a rotation by halves must be a multiple of 4 in all");
  if (axes > 0 && !rotary->freqs) return fail(who, DBSP_EINVAL, "null pointer (freqs)");
  for (int i = 0; i < p.turned; ++i) {
    if (!std::isfinite(rotary->freqs[i])) return fail(who, DBSP_EINVAL, "freqs must be finite");
    p.turns[i] = rotary->freqs[i] * 0.15915494309189533577;      // 1 / (2 pi)
  }
  const int32_t* positions = rows->positions;
  if (!positions && axes > 1) return fail(who, DBSP_EINVAL, "a rotation of several axes needs positions");
  if (!aligned(positions, 4)) return fail(who, DBSP_EINVAL, "positions must be 4-byte aligned");
  if (positions && axes > 0) {
    const int64_t size[2] = {B, N};
    for (int i = 0; i < 2; ++i)
      if (size[i] > 1 && (rows->pos_stride[i] < 0 || rows->pos_stride[i] > (int64_t)1 << 40)) return fail(who, DBSP_EINVAL, "the strides of positions must not be negative");
    p.positions = positions;
    p.pos_sb = step(B, rows->pos_stride[0]);
    p.pos_st = step(N, rows->pos_stride[1]);
  }
  return DBSP_OK;
}

int dbsp_rows_check(const char* who, const char* name, const dbsp_heads& t, bool written, int32_t B, int32_t heads, int32_t N, int32_t d) {
  if (!t.x) return dbsp_set_error(DBSP_EINVAL, std::string(who) + ": null pointer (" + name + ")");
  const int64_t size[3] = {B, heads, N};
  if (!strides_ok(size, t.stride, 3) || !aligned(t.x, 16))
    return dbsp_set_error(DBSP_EINVAL, std::string(who) + ": " + name + " must be 16-byte aligned, its strides multiples of 8 and a token's at most 2^24");
  if (written && !distinct(size, t.stride, d)) return dbsp_set_error(DBSP_EINVAL, std::string(who) + ": elements of " + name + " overlap");
  return DBSP_OK;
}

int dbsp_rows_deal(const char* who, dbsp_rows_params& p, int d, int64_t most) {
  const int tokens = kRowThreads / (d / 8);
  const int64_t tiles = ((int64_t)p.B * p.N + tokens - 1) / tokens;
  int64_t heads = 0;
  for (const dbsp_rows_part& x : p.part) heads += x.heads;
  if (heads > kMost) return fail(who, DBSP_ESHAPE, "too many heads");
  // As many heads a workgroup as leave `most` of them, dealt evenly, and six where that leaves two a compute unit: 2000 tokens of 16 + 16
  // heads of 128 with three a workgroup 9.1 us, with six 8.4.
  const int64_t per = std::max({(int64_t)1, heads * tiles / most, std::min<int64_t>(6, heads * tiles / 512)});
  int64_t groups = 0;
  for (dbsp_rows_part& x : p.part) {
    x.groups = x.heads == 0 ? 0 : (int32_t)((x.heads + per - 1) / per);
    x.per = x.heads == 0 ? 0 : (x.heads + x.groups - 1) / x.groups;
    if (x.heads > 0) x.groups = (x.heads + x.per - 1) / x.per;
    groups += x.groups;
  }
  if (groups * tiles > kMostThreads / kRowThreads) return fail(who, DBSP_ESHAPE, "too many tokens and heads");
  p.tiles = (int32_t)tiles;
  p.groups = (int32_t)groups;
  p.walkers = (int32_t)std::min(tiles, std::max<int64_t>(1, most / groups));
  return DBSP_OK;
}

namespace {

int64_t grad_bytes(const dbsp_rows_params& p, int d) { return round_up((int64_t)p.groups * p.walkers * 2 * d * 4, 256); }

// Of queries and keys together.
int64_t tensor_bytes(const dbsp_rows_params& p, int d) { return (int64_t)p.B * p.N * (p.part[0].heads + p.part[1].heads) * d * 2; }

// Heads of the queries (0) or keys (1) of a call; 0: it has no such.
int heads_of(const char* who, const dbsp_qk_rows* rows, int i, int32_t& heads) {
  heads = i == 0 ? rows->H : rows->k.x ? rows->Hk : 0;
  return heads > 0 || (i == 1 && !rows->k.x) ? DBSP_OK : fail(who, DBSP_EINVAL, "the numbers of heads must be positive");
}

}  // namespace

extern "C" {

int dbsp_qk_norm_rope_fwd(const dbsp_qk_rows* rows, const dbsp_head_norm* norm, const dbsp_rotary* rotary, void* stream) {
  const char* who = "dbsp_qk_norm_rope_fwd";
  dbsp_rows_params p = {};
  int kind = 0, rc;
  bool halves = false;
  if ((rc = dbsp_rows_settle(who, rows, norm, rotary, p, kind, halves)) != DBSP_OK) return rc;
  for (int i = 0; i < 2; ++i) {
    int32_t heads;
    if ((rc = heads_of(who, rows, i, heads)) != DBSP_OK) return rc;
    if (heads == 0) continue;
    const dbsp_heads &in = i == 0 ? rows->q : rows->k, &out = i == 0 ? rows->q_out : rows->k_out;
    if ((rc = dbsp_rows_check(who, i == 0 ? "q" : "k", in, false, p.B, heads, p.N, rows->d)) != DBSP_OK) return rc;
    if ((rc = dbsp_rows_check(who, i == 0 ? "q_out" : "k_out", out, true, p.B, heads, p.N, rows->d)) != DBSP_OK) return rc;
    set_in(p.part[i], in, p.B, heads, p.N);
    set_out(p.part[i], out, p.B, heads, p.N);
    p.part[i].plain = kind == DBSP_NORM_NONE && p.turned == 0;
    if (kind != DBSP_NORM_NONE) {
      p.part[i].gain = i == 0 ? norm->q_gain : norm->k_gain;
      p.part[i].bias = i == 0 ? norm->q_bias : norm->k_bias;
    }
  }
  if ((rc = dbsp_rows_deal(who, p, rows->d, kRowGroups)) != DBSP_OK) return rc;
  p.stream = tensor_bytes(p, rows->d) * 2 >= kRowStream && row_lines_whole(halves, p.turned);
  return done(who, dbsp_launch_rows(p, rows->d, rows->dtype == DBSP_FP16, kind, halves, false, static_cast<hipStream_t>(stream)));
}

int dbsp_qk_norm_rope_bwd_workspace(int32_t B, int32_t N, int32_t d, int32_t H, int32_t Hk, int64_t* bytes) {
  const char* who = "dbsp_qk_norm_rope_bwd_workspace";
  if (!bytes) return fail(who, DBSP_EINVAL, "null pointer");
  *bytes = 0;
  if (H <= 0 || Hk < 0) return fail(who, DBSP_EINVAL, "the numbers of heads must be positive");
  dbsp_qk_rows rows = {};
  rows.B = B;
  rows.N = N;
  rows.d = d;
  dbsp_rows_params p = {};
  int kind, rc;
  bool halves;
  if ((rc = dbsp_rows_settle(who, &rows, nullptr, nullptr, p, kind, halves)) != DBSP_OK) return rc;
  p.part[0].heads = H;
  p.part[1].heads = Hk;
  if ((rc = dbsp_rows_deal(who, p, d, kGradGroups)) != DBSP_OK) return rc;
  *bytes = grad_bytes(p, d);
  return DBSP_OK;
}

int dbsp_qk_norm_rope_bwd(const dbsp_qk_rows* rows, const dbsp_heads* dq, const dbsp_heads* dk, const dbsp_head_norm* norm,
                          const dbsp_rotary* rotary, float* grads, void* workspace, int64_t workspace_bytes, void* stream) {
  const char* who = "dbsp_qk_norm_rope_bwd";
  dbsp_rows_params p = {};
  int kind = 0, rc;
  bool halves = false;
  if ((rc = dbsp_rows_settle(who, rows, norm, rotary, p, kind, halves)) != DBSP_OK) return rc;
  for (int i = 0; i < 2; ++i) {
    int32_t heads;
    if ((rc = heads_of(who, rows, i, heads)) != DBSP_OK) return rc;
    if (heads == 0) continue;
    const dbsp_heads &in = i == 0 ? rows->q : rows->k, &dy = i == 0 ? rows->q_out : rows->k_out, *dx = i == 0 ? dq : dk;
    if (!dx) return fail(who, DBSP_EINVAL, i == 0 ? "null pointer (dq)" : "null pointer (dk)");
    if ((rc = dbsp_rows_check(who, i == 0 ? "q" : "k", in, false, p.B, heads, p.N, rows->d)) != DBSP_OK) return rc;
    if ((rc = dbsp_rows_check(who, i == 0 ? "q_out" : "k_out", dy, false, p.B, heads, p.N, rows->d)) != DBSP_OK) return rc;
    if ((rc = dbsp_rows_check(who, i == 0 ? "dq" : "dk", *dx, true, p.B, heads, p.N, rows->d)) != DBSP_OK) return rc;
    dbsp_rows_part& part = p.part[i];
    set_in(part, in, p.B, heads, p.N);
    set_out(part, *dx, p.B, heads, p.N);
    part.dy = static_cast<const uint16_t*>(dy.x);
    part.dy_sb = step(p.B, dy.stride[0]);
    part.dy_sh = step(heads, dy.stride[1]);
    part.dy_st = step(p.N, dy.stride[2]);
    if (kind != DBSP_NORM_NONE) part.gain = i == 0 ? norm->q_gain : norm->k_gain;
  }
  if (grads && kind == DBSP_NORM_NONE) return fail(who, DBSP_EINVAL, "without a norm there are no gains to form gradients of");
  if (!aligned(grads, 16)) return fail(who, DBSP_EINVAL, "grads must be 16-byte aligned");
  if ((rc = dbsp_rows_deal(who, p, rows->d, kGradGroups)) != DBSP_OK) return rc;
  p.stream = tensor_bytes(p, rows->d) * 3 >= kRowStream && row_lines_whole(halves, p.turned);
  if (grads) {
    const int64_t need = grad_bytes(p, rows->d);
    if (!workspace) return fail(who, DBSP_EINVAL, "null pointer (workspace)");
    if (!aligned(workspace, 256)) return fail(who, DBSP_EINVAL, "the workspace must be 256-byte aligned");
    if (workspace_bytes < need)
      return dbsp_set_error(DBSP_EINVAL, std::string(who) + ": the workspace holds " + std::to_string(workspace_bytes) + " bytes, the call needs " + std::to_string(need));
    p.grads = grads;
    p.sums = static_cast<float*>(workspace);
  }
  return done(who, dbsp_launch_rows_grad(p, rows->d, rows->dtype == DBSP_FP16, kind, halves, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
