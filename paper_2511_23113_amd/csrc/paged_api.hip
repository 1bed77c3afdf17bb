// C ABI of the paged key/value cache's operators: argument checks, workspaces, launches.
#include <cmath>

#include "paged_params.hpp"
#include "rows_api.hpp"

namespace {

int check_paged(const char* who, const dbsp_paged_cache* c) {
  if (!c) return fail(who, DBSP_EINVAL, "null cache");
  if (c->dtype != DBSP_BF16 && c->dtype != DBSP_FP16) return fail(who, DBSP_EINVAL, "dtype must be DBSP_BF16 or DBSP_FP16");
  if (c->d != 64 && c->d != 128) return fail(who, DBSP_EINVAL, "head dim must be 64 or 128");
  if (c->B <= 0 || c->Hk <= 0) return fail(who, DBSP_EINVAL, "B and Hk must be positive");
  if (c->n_pages <= 0 || c->page_size <= 0 || c->max_pages <= 0) return fail(who, DBSP_EINVAL, "n_pages, page_size and max_pages must be positive");
  if ((int64_t)c->max_pages * c->page_size >= kMostSlots || (int64_t)c->B * c->Hk > kMost) return fail(who, DBSP_ESHAPE, "the cache is too large");
  if (!c->k || !c->v || !c->pages || !c->lens) return fail(who, DBSP_EINVAL, "null pointer (k, v, pages or lens)");
  const int64_t size[3] = {c->n_pages, c->Hk, c->page_size};
  if (!strides_ok(size, c->k_stride, 3) || !strides_ok(size, c->v_stride, 3) || !aligned(c->k, 16) || !aligned(c->v, 16))
    return fail(who, DBSP_EINVAL, "k and v must be 16-byte aligned, their strides multiples of 8 and a slot's at most 2^24");
  if (c->n_pages > 1 && (c->k_stride[0] > (int64_t)1 << 30 || c->v_stride[0] > (int64_t)1 << 30)) return fail(who, DBSP_EINVAL, "the pages of k and v must be at most 2^30 elements apart");
  if (c->B > 1 && (c->pages_stride < 0 || c->pages_stride > (int64_t)1 << 40)) return fail(who, DBSP_EINVAL, "pages_stride must not be negative");
  if (!aligned(c->pages, 4) || !aligned(c->lens, 4)) return fail(who, DBSP_EINVAL, "pages and lens must be 4-byte aligned");
  return DBSP_OK;
}

struct Cut {             // how an attention call is laid out
  dbsp_paged_attn_params p;
  int64_t grid, part_o_at, part_lse_at, bytes;
};

int lay_out(const char* who, const dbsp_paged_cache* c, int32_t H, int32_t Nq, Cut& cut) {
  const int rc = check_paged(who, c);
  if (rc != DBSP_OK) return rc;
  if (H <= 0 || Nq <= 0) return fail(who, DBSP_EINVAL, "H and Nq must be positive");
  if (H % c->Hk != 0) return fail(who, DBSP_ESHAPE, "H must be a multiple of the cache's KV heads");
  dbsp_paged_attn_params& p = cut.p;
  p = {};
  p.B = c->B; p.H = H; p.Hk = c->Hk; p.G = H / c->Hk; p.Nq = Nq;
  p.n_pages = c->n_pages; p.page_size = c->page_size; p.max_pages = c->max_pages; p.cap = c->max_pages * c->page_size;
  const int64_t rows = (int64_t)Nq * p.G, q_rows = (int64_t)p.B * H * Nq;
  if (rows > kMost || q_rows > kMost) return fail(who, DBSP_ESHAPE, "too many queries");
  const int tile_rows = paged_tile_rows(rows);
  const int64_t row_tiles = (rows + tile_rows - 1) / tile_rows, all = row_tiles * p.B * p.Hk, tiles = (p.cap + kPagedKeys - 1) / kPagedKeys;
  p.row_tiles = (int32_t)row_tiles;
  p.own_rows = (int32_t)std::min<int64_t>(rows, tile_rows);
  if (all * tiles > kMost) return fail(who, DBSP_ESHAPE, "the cache is too large for so many sequences, heads and queries");
  p.whole = tiles <= kPagedWhole;
  p.slots = paged_slots(rows, c->d);
  p.runs = paged_runs(rows, c->d);
  // runs, or parts: at most 1 / chunk of the tiles and one a row tile, with chunk at least 1 and 1 / kPagedRuns of them
  cut.grid = round_up(p.whole ? all : std::min(all * tiles, (int64_t)kPagedRuns + all), 8);
  // parts of a row on average, if all sequences are as long; a merge workgroup has 1024 / d of them in hand at a time, eight of a row each
  int ways = 1;
  while (ways < 8 && 8 * ways * all < p.runs) ways *= 2;
  const int64_t by = 1024 / c->d / ways, merges = p.whole ? 0 : (q_rows + by - 1) / by;
  if (std::max(cut.grid, merges) > kMostThreads / 256) return fail(who, DBSP_ESHAPE, "too many queries or sequences");
  p.merge_groups = (int32_t)merges;
  p.merge_ways = ways;
  const int64_t part_rows = p.whole ? 0 : (cut.grid + all) * p.own_rows;
  cut.part_o_at = round_up((2 + 2 * (int64_t)p.B) * 4, 256);
  cut.part_lse_at = cut.part_o_at + part_rows * c->d * 4;
  cut.bytes = p.whole ? 0 : round_up(cut.part_lse_at + part_rows * 4, 256);
  return DBSP_OK;
}

}  // namespace

extern "C" {

int dbsp_paged_append(const dbsp_paged_cache* cache, const dbsp_qk_rows* rows, const dbsp_heads* v, const int32_t* new_lens,
                      const dbsp_head_norm* norm, const dbsp_rotary* rotary, void* stream) {
  const char* who = "dbsp_paged_append";
  dbsp_rows_params p = {};
  int kind = 0, rc = check_paged(who, cache);
  bool halves = false;
  if (rc == DBSP_OK) rc = dbsp_rows_settle(who, rows, norm, rotary, p, kind, halves);
  if (rc != DBSP_OK) return rc;
  const int32_t B = cache->B, Hk = cache->Hk, d = cache->d, N = rows->N;
  if (rows->dtype != cache->dtype || rows->B != B || rows->d != d || rows->Hk != Hk) return fail(who, DBSP_ESHAPE, "type, sequences, head dim and KV heads must be the cache's");
  if (rows->q.x && rows->H <= 0) return fail(who, DBSP_EINVAL, "H must be positive");
  const int64_t size[3] = {cache->n_pages, Hk, cache->page_size};
  if (!distinct(size, cache->k_stride, d) || !distinct(size, cache->v_stride, d)) return fail(who, DBSP_EINVAL, "elements of the pool's k or v overlap");
  if (!v) return fail(who, DBSP_EINVAL, "null pointer (v)");
  if (!aligned(new_lens, 4)) return fail(who, DBSP_EINVAL, "new_lens must be 4-byte aligned");
  // queries, keys, values
  for (int i = rows->q.x ? 0 : 1; i < 3; ++i) {
    dbsp_rows_part& part = p.part[i];
    const dbsp_heads& in = i == 0 ? rows->q : i == 1 ? rows->k : *v;
    const int32_t heads = i == 0 ? rows->H : Hk;
    if ((rc = dbsp_rows_check(who, i == 0 ? "q" : i == 1 ? "k" : "v", in, false, B, heads, N, d)) != DBSP_OK) return rc;
    set_in(part, in, B, heads, N);
    part.plain = i == 2 || (kind == DBSP_NORM_NONE && p.turned == 0);
    if (kind != DBSP_NORM_NONE && i < 2) {
      part.gain = i == 0 ? norm->q_gain : norm->k_gain;
      part.bias = i == 0 ? norm->q_bias : norm->k_bias;
    }
    if (i == 0) {
      if ((rc = dbsp_rows_check(who, "q_out", rows->q_out, true, B, heads, N, d)) != DBSP_OK) return rc;
      set_out(part, rows->q_out, B, heads, N);
      continue;
    }
    const int64_t* stride = i == 1 ? cache->k_stride : cache->v_stride;
    part.pool = static_cast<uint16_t*>(i == 1 ? cache->k : cache->v);
    part.page_s = step(size[0], stride[0]);
    part.y_sh = step(size[1], stride[1]);
    part.y_st = step(size[2], stride[2]);
  }
  p.lens = cache->lens;
  p.new_lens = new_lens;
  p.pages = cache->pages;
  p.pages_stride = step(B, cache->pages_stride);
  p.n_pages = cache->n_pages;
  p.page_size = cache->page_size;
  p.cap = cache->max_pages * cache->page_size;
  if ((rc = dbsp_rows_deal(who, p, d, kRowGroups)) != DBSP_OK) return rc;
  return done(who, dbsp_launch_rows(p, d, cache->dtype == DBSP_FP16, kind, halves, true, static_cast<hipStream_t>(stream)));
}

int dbsp_paged_attn_workspace(const dbsp_paged_cache* cache, int32_t H, int32_t Nq, int64_t* bytes) {
  const char* who = "dbsp_paged_attn_workspace";
  if (!bytes) return fail(who, DBSP_EINVAL, "null pointer");
  Cut cut;
  const int rc = lay_out(who, cache, H, Nq, cut);
  *bytes = rc == DBSP_OK ? cut.bytes : 0;
  return rc;
}

int dbsp_paged_attn_fwd(const dbsp_paged_cache* cache, const void* q, int64_t q_batch, int64_t q_head, int64_t q_token, void* o,
                        int64_t o_batch, int64_t o_head, int64_t o_token, float* lse, const int32_t* q_lens, int32_t H, int32_t Nq,
                        int32_t causal, float softmax_scale, void* workspace, int64_t workspace_bytes, void* stream) {
  const char* who = "dbsp_paged_attn_fwd";
  if (!(softmax_scale == softmax_scale) || softmax_scale > 1e30f || (softmax_scale > 0.f && softmax_scale < 1e-30f))
    return fail(who, DBSP_EINVAL, "softmax_scale must be 0 or between 1e-30 and 1e30");
  Cut cut;
  int rc = lay_out(who, cache, H, Nq, cut);
  if (rc != DBSP_OK) return rc;
  if ((rc = dbsp_rows_check(who, "q", {const_cast<void*>(q), {q_batch, q_head, q_token}}, false, cache->B, H, Nq, cache->d)) != DBSP_OK) return rc;
  if ((rc = dbsp_rows_check(who, "o", {o, {o_batch, o_head, o_token}}, true, cache->B, H, Nq, cache->d)) != DBSP_OK) return rc;
  if (!aligned(lse, 4) || !aligned(q_lens, 4)) return fail(who, DBSP_EINVAL, "lse and q_lens must be 4-byte aligned");
  if (!workspace && cut.bytes > 0) return fail(who, DBSP_EINVAL, "null pointer (workspace)");
  if (!aligned(workspace, 256)) return fail(who, DBSP_EINVAL, "the workspace must be 256-byte aligned");
  if (workspace_bytes < cut.bytes)
    return dbsp_set_error(DBSP_EINVAL, std::string(who) + ": the workspace holds " + std::to_string(workspace_bytes) + " bytes, the call needs " + std::to_string(cut.bytes));
  dbsp_paged_attn_params& p = cut.p;
  p.q = static_cast<const uint16_t*>(q);
  p.o = static_cast<uint16_t*>(o);
  p.k = static_cast<const unsigned char*>(cache->k);
  p.v = static_cast<const unsigned char*>(cache->v);
  p.lse = lse;
  p.lens = cache->lens;
  p.q_lens = q_lens;
  p.pages = cache->pages;
  p.pages_stride = step(p.B, cache->pages_stride);
  p.q_sb = step(p.B, q_batch); p.q_sh = step(H, q_head); p.q_st = step(Nq, q_token);
  p.o_sb = step(p.B, o_batch); p.o_sh = step(H, o_head); p.o_st = step(Nq, o_token);
  auto bytes = [](int64_t size, int64_t stride) { return (uint32_t)(step(size, stride) * 2); };
  p.k_sp = bytes(p.n_pages, cache->k_stride[0]); p.k_sh = step(p.Hk, cache->k_stride[1]) * 2; p.k_ss = bytes(p.page_size, cache->k_stride[2]);
  p.v_sp = bytes(p.n_pages, cache->v_stride[0]); p.v_sh = step(p.Hk, cache->v_stride[1]) * 2; p.v_ss = bytes(p.page_size, cache->v_stride[2]);
  p.page_16 = p.page_size % 16 == 0;
  paged_divisor(p.page_size, p.page_mul, p.page_shift);
  p.causal = causal != 0;
  p.scale_log2 = (softmax_scale > 0.f ? softmax_scale : 1.0f / std::sqrt((float)cache->d)) * 1.4426950408889634f;
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  p.table = reinterpret_cast<int32_t*>(ws);
  p.part_o = reinterpret_cast<float*>(ws + cut.part_o_at);
  p.part_lse = reinterpret_cast<float*>(ws + cut.part_lse_at);
  return done(who, dbsp_launch_paged_attn(p, cache->d, cache->dtype == DBSP_FP16, (int)cut.grid, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
