// C ABI of the norms and rotations of queries and keys: argument checks, workspaces, launches.
#include "rows_api.hpp"

#include <cmath>

int dbsp_rows_settle(const char* who, const dbsp_head_norm* norm, const dbsp_rotary* rotary, const int32_t* positions, int64_t pos_batch,
                     int64_t pos_token, int32_t B, int32_t N, int32_t d, dbsp_rows_params& p, int& kind, bool& halves) {
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
  if (!positions && axes > 1) return fail(who, DBSP_EINVAL, "a rotation of several axes needs positions");
  if (!aligned(positions, 4)) return fail(who, DBSP_EINVAL, "positions must be 4-byte aligned");
  if (positions && axes > 0) {
    if ((B > 1 && (pos_batch < 0 || pos_batch > (int64_t)1 << 40)) || (N > 1 && (pos_token < 0 || pos_token > (int64_t)1 << 40)))
      return fail(who, DBSP_EINVAL, "the strides of positions must not be negative");
    p.positions = positions;
    p.pos_sb = step(B, pos_batch);
    p.pos_st = step(N, pos_token);
  }
  return DBSP_OK;
}

int dbsp_rows_check(const char* who, const char* name, const dbsp_rows_tensor& t, bool written, int32_t B, int32_t heads, int32_t N, int32_t d) {
  if (!t.x) return dbsp_set_error(DBSP_EINVAL, std::string(who) + ": null pointer (" + name + ")");
  const int64_t size[3] = {B, heads, N}, stride[3] = {t.batch, t.head, t.token};
  if (!strides_ok(size, stride, 3) || !aligned(t.x, 16))
    return dbsp_set_error(DBSP_EINVAL, std::string(who) + ": " + name + " must be 16-byte aligned, its strides multiples of 8 and a token's at most 2^24");
  if (written && !distinct(size, stride, d)) return dbsp_set_error(DBSP_EINVAL, std::string(who) + ": elements of " + name + " overlap");
  return DBSP_OK;
}

int dbsp_rows_deal(const char* who, dbsp_rows_params& p, int d, int64_t most) {
  const int tokens = kRowThreads / (d / 8);
  const int64_t tiles = ((int64_t)p.B * p.N + tokens - 1) / tokens;
  int64_t heads = 0;
  for (const dbsp_rows_part& x : p.part) heads += x.heads;
  if (heads > kMost) return fail(who, DBSP_ESHAPE, "too many heads");
  // as many heads a workgroup as leave `most` of them, dealt evenly
  const int64_t per = std::max<int64_t>(1, heads * tiles / most);
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

int check_dtype(const char* who, int32_t dtype) { return dtype == DBSP_BF16 || dtype == DBSP_FP16 ? DBSP_OK : fail(who, DBSP_EINVAL, "dtype must be DBSP_BF16 or DBSP_FP16"); }

void set_in(dbsp_rows_part& part, const dbsp_rows_tensor& t, int32_t B, int32_t heads, int32_t N) {
  part.x = static_cast<const uint16_t*>(t.x);
  part.x_sb = step(B, t.batch);
  part.x_sh = step(heads, t.head);
  part.x_st = step(N, t.token);
  part.heads = heads;
}
void set_out(dbsp_rows_part& part, const dbsp_rows_tensor& t, int32_t B, int32_t heads, int32_t N) {
  part.y = static_cast<uint16_t*>(const_cast<void*>(t.x));
  part.y_sb = step(B, t.batch);
  part.y_sh = step(heads, t.head);
  part.y_st = step(N, t.token);
}

int64_t grad_bytes(const dbsp_rows_params& p, int d) { return round_up((int64_t)p.groups * p.walkers * 2 * d * 4, 256); }

}  // namespace

extern "C" {

int dbsp_qk_norm_rope_fwd(int32_t dtype, int32_t B, int32_t N, int32_t d, const void* q, int64_t q_batch, int64_t q_head, int64_t q_token,
                          void* q_out, int64_t q_out_batch, int64_t q_out_head, int64_t q_out_token, int32_t H, const void* k, int64_t k_batch,
                          int64_t k_head, int64_t k_token, void* k_out, int64_t k_out_batch, int64_t k_out_head, int64_t k_out_token, int32_t Hk,
                          const dbsp_head_norm* norm, const dbsp_rotary* rotary, const int32_t* positions, int64_t pos_batch, int64_t pos_token,
                          void* stream) {
  const char* who = "dbsp_qk_norm_rope_fwd";
  dbsp_rows_params p = {};
  int kind = 0, rc = check_dtype(who, dtype);
  bool halves = false;
  if (rc == DBSP_OK) rc = dbsp_rows_settle(who, norm, rotary, positions, pos_batch, pos_token, B, N, d, p, kind, halves);
  if (rc != DBSP_OK) return rc;
  if (H <= 0 || (k && Hk <= 0)) return fail(who, DBSP_EINVAL, "the numbers of heads must be positive");
  const dbsp_rows_tensor in[2] = {{q, q_batch, q_head, q_token}, {k, k_batch, k_head, k_token}};
  const dbsp_rows_tensor out[2] = {{q_out, q_out_batch, q_out_head, q_out_token}, {k_out, k_out_batch, k_out_head, k_out_token}};
  static const char* const names[2][2] = {{"q", "q_out"}, {"k", "k_out"}};
  for (int i = 0; i < (k ? 2 : 1); ++i) {
    const int32_t heads = i == 0 ? H : Hk;
    if ((rc = dbsp_rows_check(who, names[i][0], in[i], false, B, heads, N, d)) != DBSP_OK) return rc;
    if ((rc = dbsp_rows_check(who, names[i][1], out[i], true, B, heads, N, d)) != DBSP_OK) return rc;
    set_in(p.part[i], in[i], B, heads, N);
    set_out(p.part[i], out[i], B, heads, N);
    if (kind != DBSP_NORM_NONE) {
      p.part[i].gain = i == 0 ? norm->q_gain : norm->k_gain;
      p.part[i].bias = i == 0 ? norm->q_bias : norm->k_bias;
    }
  }
  if ((rc = dbsp_rows_deal(who, p, d, kRowGroups)) != DBSP_OK) return rc;
  return done(who, dbsp_launch_rows(p, d, dtype == DBSP_FP16, kind, halves, false, static_cast<hipStream_t>(stream)));
}

int dbsp_qk_norm_rope_bwd_workspace(int32_t B, int32_t N, int32_t d, int32_t H, int32_t Hk, int64_t* bytes) {
  const char* who = "dbsp_qk_norm_rope_bwd_workspace";
  if (!bytes) return fail(who, DBSP_EINVAL, "null pointer");
  *bytes = 0;
  if (H <= 0 || Hk < 0) return fail(who, DBSP_EINVAL, "the numbers of heads must be positive");
  dbsp_rows_params p = {};
  int kind;
  bool halves;
  int rc = dbsp_rows_settle(who, nullptr, nullptr, nullptr, 0, 0, B, N, d, p, kind, halves);
  if (rc != DBSP_OK) return rc;
  p.part[0].heads = H;
  p.part[1].heads = Hk;
  if ((rc = dbsp_rows_deal(who, p, d, kGradGroups)) != DBSP_OK) return rc;
  *bytes = grad_bytes(p, d);
  return DBSP_OK;
}

int dbsp_qk_norm_rope_bwd(int32_t dtype, int32_t B, int32_t N, int32_t d, const void* q, int64_t q_batch, int64_t q_head, int64_t q_token,
                          const void* dq_out, int64_t dq_out_batch, int64_t dq_out_head, int64_t dq_out_token, void* dq, int64_t dq_batch,
                          int64_t dq_head, int64_t dq_token, int32_t H, const void* k, int64_t k_batch, int64_t k_head, int64_t k_token,
                          const void* dk_out, int64_t dk_out_batch, int64_t dk_out_head, int64_t dk_out_token, void* dk, int64_t dk_batch,
                          int64_t dk_head, int64_t dk_token, int32_t Hk, const dbsp_head_norm* norm, const dbsp_rotary* rotary,
                          const int32_t* positions, int64_t pos_batch, int64_t pos_token, float* grads, void* workspace, int64_t workspace_bytes,
                          void* stream) {
  const char* who = "dbsp_qk_norm_rope_bwd";
  dbsp_rows_params p = {};
  int kind = 0, rc = check_dtype(who, dtype);
  bool halves = false;
  if (rc == DBSP_OK) rc = dbsp_rows_settle(who, norm, rotary, positions, pos_batch, pos_token, B, N, d, p, kind, halves);
  if (rc != DBSP_OK) return rc;
  if (H <= 0 || (k && Hk <= 0)) return fail(who, DBSP_EINVAL, "the numbers of heads must be positive");
  const dbsp_rows_tensor in[2] = {{q, q_batch, q_head, q_token}, {k, k_batch, k_head, k_token}};
  const dbsp_rows_tensor dy[2] = {{dq_out, dq_out_batch, dq_out_head, dq_out_token}, {dk_out, dk_out_batch, dk_out_head, dk_out_token}};
  const dbsp_rows_tensor dx[2] = {{dq, dq_batch, dq_head, dq_token}, {dk, dk_batch, dk_head, dk_token}};
  static const char* const names[2][3] = {{"q", "dq_out", "dq"}, {"k", "dk_out", "dk"}};
  for (int i = 0; i < (k ? 2 : 1); ++i) {
    const int32_t heads = i == 0 ? H : Hk;
    if ((rc = dbsp_rows_check(who, names[i][0], in[i], false, B, heads, N, d)) != DBSP_OK) return rc;
    if ((rc = dbsp_rows_check(who, names[i][1], dy[i], false, B, heads, N, d)) != DBSP_OK) return rc;
    if ((rc = dbsp_rows_check(who, names[i][2], dx[i], true, B, heads, N, d)) != DBSP_OK) return rc;
    dbsp_rows_part& part = p.part[i];
    set_in(part, in[i], B, heads, N);
    set_out(part, dx[i], B, heads, N);
    part.dy = static_cast<const uint16_t*>(dy[i].x);
    part.dy_sb = step(B, dy[i].batch);
    part.dy_sh = step(heads, dy[i].head);
    part.dy_st = step(N, dy[i].token);
    if (kind != DBSP_NORM_NONE) part.gain = i == 0 ? norm->q_gain : norm->k_gain;
  }
  if (grads && kind == DBSP_NORM_NONE) return fail(who, DBSP_EINVAL, "without a norm there are no gains to form gradients of");
  if (!aligned(grads, 16)) return fail(who, DBSP_EINVAL, "grads must be 16-byte aligned");
  if ((rc = dbsp_rows_deal(who, p, d, kGradGroups)) != DBSP_OK) return rc;
  if (grads) {
    const int64_t need = grad_bytes(p, d);
    if (!workspace) return fail(who, DBSP_EINVAL, "null pointer (workspace)");
    if (!aligned(workspace, 256)) return fail(who, DBSP_EINVAL, "the workspace must be 256-byte aligned");
    if (workspace_bytes < need)
      return dbsp_set_error(DBSP_EINVAL, std::string(who) + ": the workspace holds " + std::to_string(workspace_bytes) + " bytes, the call needs " + std::to_string(need));
    p.grads = grads;
    p.sums = static_cast<float*>(workspace);
  }
  return done(who, dbsp_launch_rows_grad(p, d, dtype == DBSP_FP16, kind, halves, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
