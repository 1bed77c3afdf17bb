// C ABI of the key/value cache's operators: argument checks, workspaces, launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <string>

#include "api_checks.hpp"
#include "cache_params.hpp"
#include "dbsp.h"
#include "dbsp_diag.h"

namespace {

int check_cache(const char* who, const dbsp_cache* c) {
  if (!c) return fail(who, DBSP_EINVAL, "null cache");
  if (c->dtype != DBSP_BF16 && c->dtype != DBSP_FP16) return fail(who, DBSP_EINVAL, "dtype must be DBSP_BF16 or DBSP_FP16");
  if (c->d != 64 && c->d != 128) return fail(who, DBSP_EINVAL, "head dim must be 64 or 128");
  if (c->B <= 0 || c->Hk <= 0) return fail(who, DBSP_EINVAL, "B and Hk must be positive");
  if (c->n_prefix < 0 || c->capacity < 0) return fail(who, DBSP_EINVAL, "n_prefix and capacity must not be negative");
  if (c->n_prefix > kMost || c->capacity > 65535 * 128 || (int64_t)c->B * c->Hk > kMost) return fail(who, DBSP_ESHAPE, "the cache is too large");
  if (c->n_prefix > 0) {
    if (!c->prefix_k || !c->prefix_v) return fail(who, DBSP_EINVAL, "null pointer (prefix)");
    const int64_t size[2] = {c->Hk, c->n_prefix};
    if (!strides_ok(size, c->prefix_k_stride, 2) || !strides_ok(size, c->prefix_v_stride, 2) || !aligned(c->prefix_k, 16) || !aligned(c->prefix_v, 16))
      return fail(who, DBSP_EINVAL, "the prefix must be 16-byte aligned, its strides multiples of 8 and a token's at most 2^24");
  }
  if (c->capacity > 0) {
    if (!c->k || !c->v || !c->lens) return fail(who, DBSP_EINVAL, "null pointer (k, v or lens)");
    const int64_t size[3] = {c->B, c->Hk, c->capacity};
    if (!strides_ok(size, c->k_stride, 3) || !strides_ok(size, c->v_stride, 3) || !aligned(c->k, 16) || !aligned(c->v, 16))
      return fail(who, DBSP_EINVAL, "k and v must be 16-byte aligned, their strides multiples of 8 and a token's at most 2^24");
    if (!aligned(c->lens, 4) || !aligned(c->weights, 4) || !aligned(c->positions, 4))
      return fail(who, DBSP_EINVAL, "lens, weights and positions must be 4-byte aligned");
  }
  return DBSP_OK;
}

struct Cut {             // how an attention call is laid out
  dbsp_cache_attn_params p;
  int64_t grid, row_lse_at, part_o_at, part_lse_at, scores_at, part_w_at, bytes;
};

// Of a launch of n row tiles on a chip that holds `slots` workgroups at a time.  They have `tiles` key tiles each: whole rounds of row
// tiles go as they are, and the last one or two are cut into parts that fill their rounds.  Or causality leaves the first
// ones `span` fewer: then the longest go first, and all are cut if the longest alone would outlast the others' share.
// us, in a run / longest first: 48 heads, 4101 causal queries at d = 64 187 / 168 (160 with the part tile in front, row_shift), 16 heads
// of 8192 339 / 263; 40 heads, 1560 queries behind 12,870 keys 1250 uncut but for 1024 items, 1101 so.
// What an item costs beside its tiles, in tiles: kStart, and kPart more for a part (its result goes to memory and back; 4 and 16
// choose the same cuts but for half a per cent).
constexpr double kStart = 2, kPart = 8;
dbsp_cache_long_cut cut_long(int64_t n, int64_t tiles, int64_t span, int slots) {
  const int dies = n < 64 ? 1 : 8;         // few row tiles: their parts go to all dies
  const int64_t per = (n + dies - 1) / dies, room = slots / dies;
  const bool longest_first = 4 * span > tiles;
  dbsp_cache_long_cut best = {(int32_t)n, dies, (int32_t)per, (int32_t)per, 0, 1, longest_first};
  auto take = [&](double cost, double& least, int64_t whole, int64_t k) {
    if (cost >= least) return;
    least = cost;
    best.whole = (int32_t)(k > 1 ? whole : per);
    best.tail = (int32_t)(k > 1 ? per - whole : 0);
    best.k = (int32_t)k;
  };
  // the parts that fill 1 .. 6 rounds with n row tiles (fewer parts of as many rounds only leave places empty)
  auto fills = [&](int64_t n, int64_t round) { return std::min(round * room / std::max<int64_t>(n, 1), tiles / 2); };
  double least = 1e300;
  if (longest_first) {
    const double work = (double)per * (tiles - 0.5 * span), longest = (double)tiles;
    auto cost = [&](int64_t k) {
      const double more = kStart + (k > 1 ? kPart : 0);
      return std::max((work + per * k * more) / room, longest / k + more) + 0.15 * longest / k;
    };
    take(cost(1), least, 0, 1);
    for (int64_t k = 2; k <= 4 && k <= tiles / 2; ++k) take(cost(k), least, 0, k);
    for (int64_t round = 1; round <= 6; ++round)
      if (const int64_t k = fills(per, round); k > 4) take(cost(k), least, 0, k);
    return best;
  }
  least = (double)((per + room - 1) / room) * (tiles + kStart);
  for (int64_t whole = per / room * room; whole >= 0 && whole + 2 * room > per; whole -= room)
    for (int64_t round = 1; round <= 6 && per > whole; ++round)
      if (const int64_t k = fills(per - whole, round); k > 1)
        take((double)(whole / room) * (tiles + kStart) + (double)round * ((tiles + k - 1) / k + kStart + kPart), least, whole, k);
  return best;
}

// Which launches the kernel for many queries has, of those with more than 128 rows a (sequence, KV head): not those of short key lists,
// as it has one workgroup a compute unit (two at d = 64) and nothing runs beside a workgroup's first loads and last stores, and its
// tiles of 256 rows leave more of them empty; nor those with little to do, 12 or 16 tiles of 128 rows by 64 keys a compute unit, for
// which the other kernel has more workgroups.  us, many / few queries' kernel: 1024 (sequence, head) pairs of 200 rows, 250 keys 80 / 66, at
// d = 64 41 / 34; 512 of 380 rows and keys 77 / 60, 38 / 33, of 512 96.5 / 94.6, 46 / 50; 256 of 620 72 / 63, of 1000 122 / 125, all seen 161 / 173.
// And 128 of 300 22 / 17, 8 of 300 20 / 12, of 1000 30 / 24, of 1500 32 / 29, of 2000 38 / 39, at d = 64 32 / 27, 32 of 800 36.5 / 37.6, 31 / 26;
// 8 of 200 over 2300 27 / 23, over 8000 30 / 28, over 16,000 35 / 38, 28 / 26; 160 of 150 over 1000 36 / 44, 27 / 29, 4 of 4000 47 / 60, 37 / 35.
bool is_many(int64_t rows, int64_t row_tiles, int64_t tiles, int d) {
  if (rows <= kCacheRows) return false;
  return d == 128 ? tiles > 10 && row_tiles * tiles > 3000 : tiles > 6 && row_tiles * tiles > 4096;
}

int lay_out(const char* who, const dbsp_cache* c, int32_t H, int32_t Nq, bool causal, bool with_weights, Cut& cut) {
  const int rc = check_cache(who, c);
  if (rc != DBSP_OK) return rc;
  if (H <= 0 || Nq <= 0) return fail(who, DBSP_EINVAL, "H and Nq must be positive");
  if (H % c->Hk != 0) return fail(who, DBSP_ESHAPE, "H must be a multiple of the cache's KV heads");
  if (with_weights && c->capacity > 0 && !c->weights) return fail(who, DBSP_EINVAL, "the cache has no weights");
  dbsp_cache_attn_params& p = cut.p;
  p = {};
  p.B = c->B; p.H = H; p.Hk = c->Hk; p.G = H / c->Hk; p.Nq = Nq; p.P = c->n_prefix; p.cap = c->capacity;
  const int64_t rows = (int64_t)Nq * p.G, all_rows = rows * p.B, q_rows = (int64_t)p.B * Nq * H;
  if (rows > kMost || all_rows > kMost || q_rows > INT_MAX) return fail(who, DBSP_ESHAPE, "too many queries");
  p.pre_tiles = (p.P + kCacheKeys - 1) / kCacheKeys;
  const int64_t tiles = p.pre_tiles + (int64_t)(p.cap + kCacheKeys - 1) / kCacheKeys;
  p.pooled = tiles > kCacheWhole && p.pre_tiles > kPooledFrom && p.B > 1 && rows < kCacheRows;
  p.pre_row_tiles = p.pooled ? (int32_t)((all_rows + kCacheRows - 1) / kCacheRows) : 0;
  p.many = is_many(rows, (rows + kCacheRows - 1) / kCacheRows * c->B * c->Hk, tiles, c->d);
  p.own_tile_rows = p.many ? kLongRows : kCacheRows;
  p.own_row_tiles = (int32_t)((rows + p.own_tile_rows - 1) / p.own_tile_rows);
  p.own_rows = (int32_t)std::min<int64_t>(rows, p.own_tile_rows);
  const int64_t unit = (int64_t)p.Hk * p.own_row_tiles, pre_unit = (int64_t)p.Hk * p.pre_row_tiles, row_tiles = unit * p.B;
  const int64_t most_tiles = (p.pooled ? 0 : p.pre_tiles) + (p.cap + kCacheKeys - 1) / kCacheKeys;
  if (row_tiles > kMost) return fail(who, DBSP_ESHAPE, "too many queries");
  const bool many = p.many;
  p.split = !many && (p.pooled || (row_tiles < kCacheTarget && most_tiles > kCacheWhole));
  const int64_t span = causal ? std::min(Nq, c->capacity) / kCacheKeys : 0;
  if (many) p.cut = cut_long(row_tiles, most_tiles, span, (c->d == 128 ? 1 : 2) * kLongSlots * 4 / kLongWaves);
  p.row_shift = many && p.cut.longest_first && p.own_row_tiles > 1 ? (int32_t)(p.own_row_tiles * (int64_t)kLongRows - rows) : 0;
  // Rows leave as many partial results: of more than 32 a (sequence, KV head) parts are fewer, 256 items at d = 128 and 512 at d = 64
  // (us with 1024: 8 heads of 128 rows over 57,000 keys 80 / 59, 128 pairs of 100 rows 92 / 76, 256 of 33 rows 87 / 74, 128 of 48
  // rows 56 / 59, at d = 64 16 heads of 64 rows over 57,000 keys 56 / 54), and those of a prefix whose rows fill tiles where the own
  // rows do not have twice the keys of an own one (64 sequences of 5 rows behind 16,384 keys 131 / 122, 40 of 25 rows 67 / 63; four
  // times 171 and 73).
  p.target = rows <= 32 ? kCacheTarget : kCacheTarget * 32 / c->d;
  p.pre_longer = rows <= 32 && all_rows > 32 ? 2 : 1;
  // items are at most 1 / chunk of the tiles and one a row tile, with chunk at least 1 and 1 / target of them
  const int64_t pre_items = std::min(pre_unit * p.pre_tiles, p.target + pre_unit);
  const int64_t own_items = many ? (int64_t)p.cut.dies * p.cut.tail * p.cut.k : p.split ? std::min(row_tiles * std::max<int64_t>(most_tiles, 1), p.target + row_tiles) : row_tiles;
  if (many) cut.grid = (int64_t)p.cut.dies * (p.cut.whole + (int64_t)p.cut.tail * p.cut.k);
  else if (p.split) cut.grid = round_up(std::min(pre_items + own_items, p.target + pre_unit + row_tiles), 8) + 16;      // (dies' shares of two lists, rounded up)
  else cut.grid = round_up(row_tiles, 8);
  if (cut.grid > kMost || pre_items > kMost / kCacheRows) return fail(who, DBSP_ESHAPE, "too many queries");
  p.max_pre_items = p.pooled ? (int32_t)pre_items : 0;
  cut.row_lse_at = round_up((2 + 2 * (int64_t)p.B) * 4, 256);
  cut.part_o_at = cut.row_lse_at + (with_weights ? round_up(q_rows * 4, 256) : 0);
  const int64_t part_rows = p.split || many ? p.max_pre_items * (int64_t)kCacheRows + own_items * p.own_rows : 0;
  cut.part_lse_at = cut.part_o_at + part_rows * c->d * 4;
  cut.scores_at = round_up(cut.part_lse_at + part_rows * 4, 256);
  const bool keep_scores = with_weights && p.cap > 0 && rows * 128 <= kScoreRows * c->d;
  p.score_pitch = keep_scores ? round_up(p.cap, kCacheKeys) : 0;
  cut.part_w_at = round_up(cut.scores_at + (int64_t)p.B * p.Hk * rows * p.score_pitch * 4, 256);
  // Rows are cut: down to 128 a part for two workgroups a compute unit, down to 512 for four.  us with 1 / 2 / 3 / 4 / 6 / 8 / 12 parts: 8 pairs
  // of 1000 rows, 1000 slots (32 workgroups) 53 / 46 / 44 / 42 / 40 / 38 / 42, 64 of 1200, 300 (128) 69 / 55 / 53 / 50.5 / 50 / 55 / 62, 154 of 776,
  // 194 (154) 53 / 49 / 45.5 / 50 / 51.5 / 53 / 62, 24 of 1560, 2000 (192) 116 / 111.5 / 107 / 116 / 114 / 120 / 129; of 4096, 4096 at d = 64 (384) 164 / 148.
  const int64_t groups = (int64_t)p.B * p.Hk * ((p.cap + kWeightKeys - 1) / kWeightKeys);
  const int64_t cuts = std::max(std::min(2 * kLongSlots / std::max<int64_t>(groups, 1), rows / 128), std::min(4 * kLongSlots / std::max<int64_t>(groups, 1), rows / 512));
  p.row_parts = with_weights && p.cap > 0 && !keep_scores ? (int32_t)std::clamp<int64_t>(cuts, 1, 64) : 1;
  cut.bytes = round_up(cut.part_w_at + (p.row_parts > 1 ? (int64_t)p.row_parts * p.B * p.Hk * p.cap * 4 : 0), 256);
  if (!p.split && p.cut.k <= 1 && !with_weights) cut.bytes = 0;      // one launch, and nothing between workgroups
  // the finishing launch: rows that are joined, 1024 / d of them a workgroup or one, and (sequence, KV head) pairs whose scores are summed
  const bool cut_up = many && p.cut.k > 1;
  const int64_t joined = cut_up ? (int64_t)p.cut.dies * p.cut.tail * p.own_rows : p.split ? q_rows : 0, by = joined <= kMergeRows ? 1 : 1024 / c->d;
  const int64_t merges = (joined + by - 1) / by, pairs = (int64_t)p.B * p.Hk, sums = keep_scores ? pairs * ((p.cap + kScoreSlots - 1) / kScoreSlots) : 0;
  if (std::max({cut.grid, merges + sums, with_weights ? pairs : 0}) > kMostThreads / 256) return fail(who, DBSP_ESHAPE, "too many queries or sequences");
  p.merge_groups = (int32_t)merges;
  p.merge_by_row = by == 1;
  p.sum_groups = (int32_t)sums;
  return DBSP_OK;
}

struct Moves {           // an eviction's workspace
  int64_t most, parts, holes_at, fillers_at, digits_at, chosen_at, parts_at, bytes;
};

int lay_out_evict(const char* who, const dbsp_cache* c, int32_t budget, Moves& m) {
  const int rc = check_cache(who, c);
  if (rc != DBSP_OK) return rc;
  if (budget < 1) return fail(who, DBSP_EINVAL, "budget must be positive");
  m.most = std::min<int64_t>(budget, std::max(0, c->capacity - budget));
  m.parts = c->capacity > kEvictWhole ? (c->capacity + kEvictPart - 1) / kEvictPart : 0;
  const int64_t pairs = (int64_t)c->B * c->Hk;
  if (pairs > kMostThreads / evict_threads(c->capacity)) return fail(who, DBSP_ESHAPE, "too many sequences");
  m.holes_at = round_up(pairs * 4, 256);
  m.fillers_at = m.holes_at + round_up(pairs * m.most * 4, 256);
  m.digits_at = m.fillers_at + round_up(pairs * m.most * 4, 256);
  m.chosen_at = m.digits_at + (m.parts > 0 ? pairs * 3 * 2048 * 4 : 0);
  m.parts_at = m.chosen_at + (m.parts > 0 ? round_up(pairs * 3 * 4, 256) : 0);
  m.bytes = round_up(m.parts_at + pairs * m.parts * 16, 256);
  return DBSP_OK;
}

}  // namespace

extern "C" {

int dbsp_cache_attn_workspace(const dbsp_cache* cache, int32_t H, int32_t Nq, int32_t causal, int32_t with_weights, int64_t* bytes) {
  const char* who = "dbsp_cache_attn_workspace";
  if (!bytes) return fail(who, DBSP_EINVAL, "null pointer");
  Cut cut;
  const int rc = lay_out(who, cache, H, Nq, causal != 0, with_weights != 0, cut);
  *bytes = rc == DBSP_OK ? cut.bytes : 0;
  return rc;
}

int dbsp_cache_attn_layout(const dbsp_cache* cache, int32_t H, int32_t Nq, int32_t causal, int32_t with_weights, dbsp_cache_layout* layout) {
  const char* who = "dbsp_cache_attn_layout";
  if (!layout) return fail(who, DBSP_EINVAL, "null pointer");
  Cut cut;
  *layout = {};
  if (const int rc = lay_out(who, cache, H, Nq, causal != 0, with_weights != 0, cut); rc != DBSP_OK) return rc;
  const dbsp_cache_attn_params& p = cut.p;
  layout->many = p.many;
  layout->pooled = p.pooled;
  layout->joined = p.merge_groups > 0;
  layout->join_by_row = p.merge_groups > 0 && p.merge_by_row;
  layout->row_tiles = p.cut.items;
  layout->cut = p.cut.tail;
  layout->parts = p.cut.k;
  layout->longest_first = p.cut.longest_first;
  layout->scores_kept = p.score_pitch > 0;
  layout->weight_parts = with_weights && p.cap > 0 && p.score_pitch == 0 ? p.row_parts : 0;
  return DBSP_OK;
}

int dbsp_cache_attn_fwd(const dbsp_cache* cache, const void* q, int64_t q_batch, int64_t q_head, int64_t q_token, void* o,
                        int64_t o_batch, int64_t o_head, int64_t o_token, float* lse, const int32_t* q_lens, int32_t H, int32_t Nq,
                        int32_t causal, float softmax_scale, float decay, void* workspace, int64_t workspace_bytes, void* stream) {
  const char* who = "dbsp_cache_attn_fwd";
  if (!(decay == decay) || decay > 3.0e38f) return fail(who, DBSP_EINVAL, "decay must be finite");
  if (!(softmax_scale == softmax_scale) || softmax_scale > 1e30f || (softmax_scale > 0.f && softmax_scale < 1e-30f))
    return fail(who, DBSP_EINVAL, "softmax_scale must be 0 or between 1e-30 and 1e30");
  const bool with_weights = decay >= 0.f;
  Cut cut;
  const int rc = lay_out(who, cache, H, Nq, causal != 0, with_weights, cut);
  if (rc != DBSP_OK) return rc;
  if (!q || !o || (!workspace && cut.bytes > 0)) return fail(who, DBSP_EINVAL, "null pointer");
  const int64_t size[3] = {cache->B, H, Nq}, q_stride[3] = {q_batch, q_head, q_token}, o_stride[3] = {o_batch, o_head, o_token};
  if (!strides_ok(size, q_stride, 3) || !strides_ok(size, o_stride, 3) || !aligned(q, 16) || !aligned(o, 16))
    return fail(who, DBSP_EINVAL, "q and o must be 16-byte aligned, their strides multiples of 8 and a token's at most 2^24");
  if (!distinct(size, o_stride, cache->d)) return fail(who, DBSP_EINVAL, "elements of o overlap");
  if (!aligned(lse, 4) || !aligned(q_lens, 4)) return fail(who, DBSP_EINVAL, "lse and q_lens must be 4-byte aligned");
  if (!aligned(workspace, 256)) return fail(who, DBSP_EINVAL, "the workspace must be 256-byte aligned");
  if (workspace_bytes < cut.bytes)
    return dbsp_set_error(DBSP_EINVAL, std::string(who) + ": the workspace holds " + std::to_string(workspace_bytes) + " bytes, the call needs " + std::to_string(cut.bytes));
  dbsp_cache_attn_params& p = cut.p;
  auto u16 = [](const void* x) { return static_cast<const uint16_t*>(x); };
  p.q = u16(q); p.pk = u16(cache->prefix_k); p.pv = u16(cache->prefix_v); p.k = u16(cache->k); p.v = u16(cache->v);
  p.o = static_cast<uint16_t*>(o);
  p.lse = lse;
  p.weights = with_weights && p.cap > 0 ? cache->weights : nullptr;
  p.lens = p.cap > 0 ? cache->lens : nullptr;
  p.q_lens = q_lens;
  p.q_sb = step(p.B, q_batch); p.q_sh = step(H, q_head); p.q_st = step(Nq, q_token);
  p.o_sb = step(p.B, o_batch); p.o_sh = step(H, o_head); p.o_st = step(Nq, o_token);
  p.pk_sh = step(p.Hk, cache->prefix_k_stride[0]); p.pv_sh = step(p.Hk, cache->prefix_v_stride[0]);
  p.k_sb = step(p.B, cache->k_stride[0]); p.k_sh = step(p.Hk, cache->k_stride[1]);
  p.v_sb = step(p.B, cache->v_stride[0]); p.v_sh = step(p.Hk, cache->v_stride[1]);
  p.pk_st = (int32_t)(step(p.P, cache->prefix_k_stride[1]) * 2); p.pv_st = (int32_t)(step(p.P, cache->prefix_v_stride[1]) * 2);
  p.k_st = (int32_t)(step(p.cap, cache->k_stride[2]) * 2); p.v_st = (int32_t)(step(p.cap, cache->v_stride[2]) * 2);
  p.causal = causal != 0;
  p.scale_log2 = (softmax_scale > 0.f ? softmax_scale : 1.0f / std::sqrt((float)cache->d)) * 1.4426950408889634f;
  p.decay = decay;
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  p.table = reinterpret_cast<int32_t*>(ws);
  p.row_lse = reinterpret_cast<float*>(ws + cut.row_lse_at);
  p.part_o = reinterpret_cast<float*>(ws + cut.part_o_at);
  p.part_lse = reinterpret_cast<float*>(ws + cut.part_lse_at);
  p.scores = p.score_pitch > 0 ? reinterpret_cast<float*>(ws + cut.scores_at) : nullptr;
  p.part_w = reinterpret_cast<float*>(ws + cut.part_w_at);
  return done(who, dbsp_launch_cache_attn(p, cache->d, cache->dtype == DBSP_FP16, (int)cut.grid, static_cast<hipStream_t>(stream)));
}

int dbsp_cache_evict_workspace(const dbsp_cache* cache, int32_t budget, int64_t* bytes) {
  const char* who = "dbsp_cache_evict_workspace";
  if (!bytes) return fail(who, DBSP_EINVAL, "null pointer");
  Moves m;
  const int rc = lay_out_evict(who, cache, budget, m);
  *bytes = rc == DBSP_OK ? m.bytes : 0;
  return rc;
}

int dbsp_cache_evict(const dbsp_cache* cache, int32_t budget, int32_t sinks, const int32_t* keep_from, void* workspace,
                     int64_t workspace_bytes, void* stream) {
  const char* who = "dbsp_cache_evict";
  Moves m;
  const int rc = lay_out_evict(who, cache, budget, m);
  if (rc != DBSP_OK) return rc;
  if (sinks < 0) return fail(who, DBSP_EINVAL, "sinks must not be negative");
  if (cache->capacity == 0) return DBSP_OK;
  if (!cache->weights || !cache->positions) return fail(who, DBSP_EINVAL, "the cache has no weights or no positions");
  const int64_t size[3] = {cache->B, cache->Hk, cache->capacity};
  if (!distinct(size, cache->k_stride, cache->d) || !distinct(size, cache->v_stride, cache->d)) return fail(who, DBSP_EINVAL, "elements of k or v overlap");
  if (!aligned(keep_from, 4)) return fail(who, DBSP_EINVAL, "keep_from must be 4-byte aligned");
  if (!workspace) return fail(who, DBSP_EINVAL, "null pointer");
  if (!aligned(workspace, 256)) return fail(who, DBSP_EINVAL, "the workspace must be 256-byte aligned");
  if (workspace_bytes < m.bytes)
    return dbsp_set_error(DBSP_EINVAL, std::string(who) + ": the workspace holds " + std::to_string(workspace_bytes) + " bytes, the call needs " + std::to_string(m.bytes));
  if (m.most == 0) return DBSP_OK;          // budget >= capacity: nothing is over it
  dbsp_cache_evict_params p = {};
  p.k = static_cast<unsigned char*>(cache->k); p.v = static_cast<unsigned char*>(cache->v);
  p.weights = cache->weights; p.positions = cache->positions; p.lens = cache->lens; p.keep_from = keep_from;
  p.k_sb = step(size[0], cache->k_stride[0]) * 2; p.k_sh = step(size[1], cache->k_stride[1]) * 2; p.k_st = step(size[2], cache->k_stride[2]) * 2;
  p.v_sb = step(size[0], cache->v_stride[0]) * 2; p.v_sh = step(size[1], cache->v_stride[1]) * 2; p.v_st = step(size[2], cache->v_stride[2]) * 2;
  p.B = cache->B; p.Hk = cache->Hk; p.cap = cache->capacity; p.row_bytes = cache->d * 2;
  p.budget = budget; p.sinks = sinks; p.max_moves = (int32_t)m.most; p.n_parts = (int32_t)m.parts;
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  p.n_moves = reinterpret_cast<int32_t*>(ws);
  p.holes = reinterpret_cast<int32_t*>(ws + m.holes_at);
  p.fillers = reinterpret_cast<int32_t*>(ws + m.fillers_at);
  p.digits = reinterpret_cast<uint32_t*>(ws + m.digits_at);
  p.chosen = reinterpret_cast<uint32_t*>(ws + m.chosen_at);
  p.parts = reinterpret_cast<int32_t*>(ws + m.parts_at);
  return done(who, dbsp_launch_cache_evict(p, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
