// C entry points of the rotation, of the paged 8-bit cache, of trees over it and of its pool of pages: argument validation, workspace carving, kernel sequencing.
#include <math.h>

#include <algorithm>

#include "ag_q8.h"

namespace {

constexpr int kMostCu = 256;  // CUs of a gfx950, at most: for sizes that are asked for without a device

bool aligned(std::initializer_list<const void *> p) {
  return std::all_of(p.begin(), p.end(), [](const void *x) { return ((uintptr_t)x & 15) == 0; });
}

// Checks `r` for vectors of D values; tokens = B * L.
ag_status check_rope(ag_ctx *ctx, const char *who, const ag_rope *r, int D, int64_t tokens, ag_rope_dev *dev, bool quads = true) {
  *dev = ag_rope_dev{nullptr, nullptr, 0, 1, 0, 0, 1, tokens};
  if (!r) return AG_OK;
  AG_REQUIRE(r->table && r->pos, AG_EINVAL, "%s: rope: null pointer", who);
  AG_REQUIRE(r->n_rows > 0, AG_EINVAL, "%s: rope: n_rows must be positive", who);
  AG_REQUIRE(r->n_axes >= 1 && r->n_axes <= 3, AG_EINVAL, "%s: rope: n_axes = %d outside [1, 3]", who, r->n_axes);
  int64_t sum = 0;
  for (int i = 0; i < r->n_axes; ++i) {
    AG_REQUIRE(r->section[i] >= 0, AG_EINVAL, "%s: rope: a section is negative", who);
    sum += r->section[i];
  }
  AG_REQUIRE(sum == D / 2, AG_EINVAL, "%s: rope: the sections add up to %lld pairs, a vector has %d", who, (long long)sum, D / 2);
  AG_REQUIRE(aligned({r->table}), AG_EINVAL, "%s: rope: the table must be 16-byte aligned", who);
  dev->table = r->table;
  dev->pos = r->pos;
  dev->n_rows = r->n_rows;
  dev->n_axes = r->n_axes;
  dev->end0 = r->section[0];
  dev->end1 = r->n_axes > 1 ? r->section[0] + r->section[1] : D / 2;
  AG_REQUIRE(!quads || (dev->end0 % 4 == 0 && dev->end1 % 4 == 0), AG_EUNSUPPORTED,
             "%s: rope: sections that are not multiples of 4 pairs (turn by ag_rotate first)", who);
  dev->quads = dev->end0 % 4 == 0 && dev->end1 % 4 == 0;
  return AG_OK;
}

ag_status check_q8(ag_ctx *ctx, const char *who, const ag_q8_cache *c, ag_q8_dev *dev) {
  AG_REQUIRE(c, AG_EINVAL, "%s: cache is NULL", who);
  AG_REQUIRE(c->k && c->v && c->k_scale && c->v_scale && c->k_tail && c->v_tail && c->page && c->len, AG_EINVAL, "%s: cache: null pointer", who);
  AG_REQUIRE(c->B > 0 && c->Hkv > 0 && c->D > 0 && c->n_pages > 0 && c->max_blocks > 0, AG_EINVAL, "%s: cache: sizes must be positive", who);
  AG_REQUIRE(c->D == 128 || c->D == 64, AG_EUNSUPPORTED, "%s: cache: D = %d (built for 128 and 64)", who, c->D);
  AG_REQUIRE((int64_t)c->B * c->Hkv <= kDecodeMaxUnits, AG_EUNSUPPORTED, "%s: cache: more than %d units", who, kDecodeMaxUnits);
  AG_REQUIRE(c->max_blocks <= (1 << 24), AG_EUNSUPPORTED, "%s: cache: max_blocks = %d exceeds %d", who, c->max_blocks, 1 << 24);
  AG_REQUIRE(aligned({c->k, c->v, c->k_tail, c->v_tail}), AG_EINVAL, "%s: cache: pages and tails must be 16-byte aligned", who);
  *dev = ag_q8_dev{(uint8_t *)c->k, (uint8_t *)c->v, c->k_scale, c->v_scale, (uint16_t *)c->k_tail, (uint16_t *)c->v_tail, c->page, c->len,
                   c->n_pages, c->max_blocks};
  return AG_OK;
}

bool group_ok(int Hq, int Hkv) {
  if (Hq <= 0 || Hkv <= 0 || Hq % Hkv) return false;
  const int G = Hq / Hkv;
  return G == 1 || G == 2 || G == 4 || G == 8;
}

// What ag_q8_append and ag_q8_prefill_attn share: the flags' masks, if there are flags.
struct scan_ws {
  uint64_t *words;
  int32_t *blk_off;
};
ag_q8_pool_ws take_pool(ws_cursor &ws, int units, int n_pages) {
  ag_q8_pool_ws w;
  const size_t chunks = ag_q8_page_chunks(n_pages);
  w.list = ws.take<int32_t>(chunks * kQ8PageChunk);
  w.count = ws.take<int32_t>(chunks);
  w.need = ws.take<int32_t>(units);
  return w;
}
// The checks that the pool's calls share.
ag_status check_pool(ag_ctx *ctx, const char *who, const ag_q8_cache *c, const int32_t *ref, ag_q8_dev *dev) {
  const ag_status st = check_q8(ctx, who, c, dev);
  if (st != AG_OK) return st;
  AG_REQUIRE(ref, AG_EINVAL, "%s: null pointer", who);
  AG_REQUIRE(c->n_pages <= kQ8MaxPages, AG_EUNSUPPORTED, "%s: cache: n_pages = %d exceeds %d", who, c->n_pages, kQ8MaxPages);
  return AG_OK;
}
int32_t *table_of(const ag_q8_cache *c) { return const_cast<int32_t *>(c->page); }  // (the pool's calls write it)

scan_ws take_scan(ws_cursor &ws, const uint8_t *flags, int units, int L) {
  scan_ws s{nullptr, nullptr};
  if (!flags) return s;
  s.words = ws.take<uint64_t>((size_t)units * ag_nwords(L));
  s.blk_off = ws.take<int32_t>((size_t)units * (ag_nwords(L) + 1));
  return s;
}

}  // namespace

extern "C" {

ag_status ag_rotate(ag_ctx *ctx, void *hip_stream, const void *q, const void *k, ag_dtype dtype, int B, int Hq, int Hkv, int L,
                    int D, const ag_rope *rope, void *q_out, void *k_out) {
  if (!ctx) return AG_EINVAL;
  AG_REQUIRE(q && q_out && rope && (k == nullptr) == (k_out == nullptr), AG_EINVAL, "ag_rotate: null pointer");
  if (!k) Hkv = 0;
  AG_REQUIRE(B > 0 && Hq > 0 && L > 0 && D > 0 && (!k || Hkv > 0), AG_EINVAL, "ag_rotate: sizes must be positive");
  AG_REQUIRE(dtype == AG_F32 || dtype == AG_BF16, AG_EINVAL, "ag_rotate: unknown dtype %d", (int)dtype);
  AG_REQUIRE(D % 16 == 0 && D <= 512, AG_EUNSUPPORTED, "ag_rotate: D = %d (a multiple of 16, at most 512)", D);
  const int pieces = D / 2 / (dtype == AG_BF16 ? 8 : 4);  // (a token's threads; a launch has fewer than 2^32)
  AG_REQUIRE(L <= kMaxL && (int64_t)B * L < (1ll << 31) && (int64_t)B * L * pieces <= (1ll << 32) - 256 && (int64_t)Hq + Hkv <= 65535, AG_EUNSUPPORTED,
             "ag_rotate: problem too large");
  AG_REQUIRE(aligned({q, k, q_out, k_out}), AG_EINVAL, "ag_rotate: tensors must be 16-byte aligned");
  ag_rope_dev r;
  ag_status st = check_rope(ctx, "ag_rotate", rope, D, (int64_t)B * L, &r, false);
  if (st != AG_OK) return st;
  st = ag_need_device(ctx);
  if (st != AG_OK) return st;
  AG_HIP(ag_launch_rotate(ctx, (hipStream_t)hip_stream, q, k, dtype, B, Hq, Hkv, L, D, r, q_out, k_out));
  return AG_OK;
}

size_t ag_q8_workspace_bytes(int B, int L, int Hq, int Hkv, int D, int max_blocks) {
  if (B <= 0 || L <= 0 || (D != 128 && D != 64) || max_blocks <= 0 || !group_ok(Hq, Hkv) || (int64_t)B * Hkv > kDecodeMaxUnits || L > kMaxL) return 0;
  const int units = B * Hkv;
  static const uint8_t some = 0;
  size_t most = 0;
  for (int l = L; l > 0; l = ag_q8_prefill_shorter(Hq, Hkv, l)) {  // (shorter calls are cut into more pieces: the most that any needs)
    ws_cursor ws{nullptr, ~size_t(0) >> 1, 0, true};
    take_scan(ws, &some, units, l);
    ag_q8_prefill_ws w;
    ag_q8_prefill_plan(kMostCu, units, Hq, Hkv, l, D, max_blocks, ws, &w);
    most = std::max(most, ws.off);
  }
  return std::max(most, ag_align256(ag_ws_q8_decode_floats(kMostCu, Hq / Hkv, D) * sizeof(float))) + 4096;
}

ag_status ag_q8_append(ag_ctx *ctx, void *hip_stream, const void *k, const void *v, const uint8_t *flags, int L,
                       const ag_rope *rope, ag_q8_cache *cache) {
  if (!ctx) return AG_EINVAL;
  AG_REQUIRE(k && v, AG_EINVAL, "ag_q8_append: null pointer");
  AG_REQUIRE(L > 0, AG_EINVAL, "ag_q8_append: L must be positive");
  AG_REQUIRE(L <= kMaxL, AG_EUNSUPPORTED, "ag_q8_append: L = %d exceeds %d", L, kMaxL);
  ag_q8_dev c;
  ag_status st = check_q8(ctx, "ag_q8_append", cache, &c);
  if (st != AG_OK) return st;
  AG_REQUIRE(aligned({k, v}), AG_EINVAL, "ag_q8_append: k and v must be 16-byte aligned");
  ag_rope_dev r;
  st = check_rope(ctx, "ag_q8_append", rope, cache->D, (int64_t)cache->B * L, &r);
  if (st != AG_OK) return st;
  const int units = cache->B * cache->Hkv;
  ws_cursor ws{ctx->ws, ctx->ws_bytes, 0, true};
  const scan_ws scan = take_scan(ws, flags, units, L);
  AG_REQUIRE(ws.ok, AG_EWORKSPACE, "ag_q8_append: workspace of %zu bytes is too small (need %zu)", ctx->ws_bytes, ws.off);
  st = ag_need_device(ctx);
  if (st != AG_OK) return st;
  hipStream_t s = (hipStream_t)hip_stream;
  AG_HIP(ag_launch_q8_fill(ctx, s, k, v, flags, cache->B, cache->Hkv, L, cache->D, scan.words, scan.blk_off, r, c, nullptr, nullptr, nullptr));
  return AG_OK;
}

ag_status ag_q8_prefill_attn(ag_ctx *ctx, void *hip_stream, const void *q, const void *k, const void *v, const uint8_t *flags,
                             int L, int Hq, const ag_rope *rope, float scale, ag_q8_cache *cache, void *out) {
  if (!ctx) return AG_EINVAL;
  AG_REQUIRE(q && k && v && out, AG_EINVAL, "ag_q8_prefill_attn: null pointer");
  AG_REQUIRE(L > 0, AG_EINVAL, "ag_q8_prefill_attn: L must be positive");
  AG_REQUIRE(L <= kMaxL, AG_EUNSUPPORTED, "ag_q8_prefill_attn: L = %d exceeds %d", L, kMaxL);
  AG_REQUIRE(scale > 0.f && isfinite(scale), AG_EINVAL, "ag_q8_prefill_attn: scale must be positive and finite");
  ag_q8_dev c;
  ag_status st = check_q8(ctx, "ag_q8_prefill_attn", cache, &c);
  if (st != AG_OK) return st;
  AG_REQUIRE(Hq > 0 && Hq % cache->Hkv == 0, AG_EINVAL, "ag_q8_prefill_attn: Hq must be a positive multiple of Hkv");
  AG_REQUIRE(group_ok(Hq, cache->Hkv), AG_EUNSUPPORTED, "ag_q8_prefill_attn: %d query heads per KV head", Hq / cache->Hkv);
  AG_REQUIRE(aligned({q, k, v, out}), AG_EINVAL, "ag_q8_prefill_attn: tensors must be 16-byte aligned");
  ag_rope_dev r;
  st = check_rope(ctx, "ag_q8_prefill_attn", rope, cache->D, (int64_t)cache->B * L, &r);
  if (st != AG_OK) return st;
  const int units = cache->B * cache->Hkv;
  ws_cursor ws{ctx->ws, ctx->ws_bytes, 0, true};
  const scan_ws scan = take_scan(ws, flags, units, L);
  ag_q8_prefill_ws w;
  ag_q8_prefill_plan(ctx->num_cu, units, Hq, cache->Hkv, L, cache->D, cache->max_blocks, ws, &w);
  AG_REQUIRE((int64_t)units * w.n_qt * w.n_split < (1ll << 28), AG_EUNSUPPORTED, "ag_q8_prefill_attn: problem too large");
  AG_REQUIRE(ws.ok, AG_EWORKSPACE, "ag_q8_prefill_attn: workspace of %zu bytes is too small (need %zu)", ctx->ws_bytes, ws.off);
  st = ag_need_device(ctx);
  if (st != AG_OK) return st;
  hipStream_t s = (hipStream_t)hip_stream;
  AG_HIP(ag_launch_q8_fill(ctx, s, k, v, flags, cache->B, cache->Hkv, L, cache->D, scan.words, scan.blk_off, r, c, w.tiles, w.info, w.meta));
  AG_HIP(ag_launch_q8_prefill(ctx, s, q, k, v, cache->B, Hq, cache->Hkv, L, cache->D, scan.words, scan.blk_off, r, scale, c, w, out));
  return AG_OK;
}

ag_status ag_q8_decode_attn(ag_ctx *ctx, void *hip_stream, const void *q, const void *k_new, const void *v_new,
                            const uint8_t *new_flags, int Hq, const ag_rope *rope, float scale, ag_q8_cache *cache, void *out) {
  if (!ctx) return AG_EINVAL;
  AG_REQUIRE(q && k_new && v_new && out, AG_EINVAL, "ag_q8_decode_attn: null pointer");
  AG_REQUIRE(scale > 0.f && isfinite(scale), AG_EINVAL, "ag_q8_decode_attn: scale must be positive and finite");
  ag_q8_dev c;
  ag_status st = check_q8(ctx, "ag_q8_decode_attn", cache, &c);
  if (st != AG_OK) return st;
  AG_REQUIRE(Hq > 0 && Hq % cache->Hkv == 0, AG_EINVAL, "ag_q8_decode_attn: Hq must be a positive multiple of Hkv");
  AG_REQUIRE(group_ok(Hq, cache->Hkv), AG_EUNSUPPORTED, "ag_q8_decode_attn: %d query heads per KV head", Hq / cache->Hkv);
  AG_REQUIRE(aligned({q, k_new, v_new, out}), AG_EINVAL, "ag_q8_decode_attn: tensors must be 16-byte aligned");
  AG_REQUIRE(ag_q8_decode_cost((int64_t)cache->B * cache->Hkv, cache->max_blocks) < (1ll << 31), AG_EUNSUPPORTED,
             "ag_q8_decode_attn: cache: %d units of max_blocks = %d are too many", cache->B * cache->Hkv, cache->max_blocks);
  ag_rope_dev r;
  st = check_rope(ctx, "ag_q8_decode_attn", rope, cache->D, cache->B, &r);
  if (st != AG_OK) return st;
  ws_cursor ws{ctx->ws, ctx->ws_bytes, 0, true};
  float *rec = ws.take<float>(ag_ws_q8_decode_floats(ctx->num_cu, Hq / cache->Hkv, cache->D));
  AG_REQUIRE(ws.ok, AG_EWORKSPACE, "ag_q8_decode_attn: workspace of %zu bytes is too small (need %zu)", ctx->ws_bytes, ws.off);
  st = ag_need_device(ctx);
  if (st != AG_OK) return st;
  AG_HIP(ag_launch_q8_decode(ctx, (hipStream_t)hip_stream, q, k_new, v_new, new_flags, cache->B, Hq, cache->Hkv, cache->D, r, scale, c, out, rec));
  return AG_OK;
}

ag_status ag_norm_rotate(ag_ctx *ctx, void *hip_stream, const void *q, const void *k, ag_dtype dtype, int B, int Hq, int Hkv, int L,
                         int D, const void *q_weight, const void *k_weight, float eps, const ag_rope *rope, void *q_out, void *k_out) {
  if (!ctx) return AG_EINVAL;
  AG_REQUIRE(q && q_out && q_weight && (k == nullptr) == (k_out == nullptr) && (k == nullptr) == (k_weight == nullptr), AG_EINVAL,
             "ag_norm_rotate: null pointer");
  if (!k) Hkv = 0;
  AG_REQUIRE(B > 0 && Hq > 0 && L > 0 && D > 0 && (!k || Hkv > 0), AG_EINVAL, "ag_norm_rotate: sizes must be positive");
  AG_REQUIRE(dtype == AG_F32 || dtype == AG_BF16, AG_EINVAL, "ag_norm_rotate: unknown dtype %d", (int)dtype);
  AG_REQUIRE(eps >= 0x1p-100f && isfinite(eps), AG_EINVAL, "ag_norm_rotate: eps must be finite and at least 2^-100");
  AG_REQUIRE(D % 16 == 0 && D <= 512, AG_EUNSUPPORTED, "ag_norm_rotate: D = %d (a multiple of 16, at most 512)", D);
  const int piece = dtype == AG_BF16 ? 8 : 4;  // (a token's threads: its pairs' pieces of 16 bytes, rounded up to a power of two; a launch has fewer than 2^32)
  int64_t threads = (int64_t)B * L;
  for (int n = 1; n < D / 2 / piece; n *= 2) threads *= 2;
  AG_REQUIRE(L <= kMaxL && (int64_t)B * L < (1ll << 31) && threads <= (1ll << 32) - 256 && (int64_t)Hq + Hkv <= 65535, AG_EUNSUPPORTED,
             "ag_norm_rotate: problem too large");
  AG_REQUIRE(aligned({q, k, q_weight, k_weight, q_out, k_out}), AG_EINVAL, "ag_norm_rotate: tensors must be 16-byte aligned");
  ag_rope_dev r;
  ag_status st = check_rope(ctx, "ag_norm_rotate", rope, D, (int64_t)B * L, &r, false);
  if (st != AG_OK) return st;
  st = ag_need_device(ctx);
  if (st != AG_OK) return st;
  AG_HIP(ag_launch_norm_rotate(ctx, (hipStream_t)hip_stream, q, k, dtype, B, Hq, Hkv, L, D, q_weight, k_weight, eps, r, q_out, k_out));
  return AG_OK;
}

size_t ag_q8_tree_workspace_bytes(int B, int L, int Hq, int Hkv, int D, int max_blocks) {
  if (B <= 0 || L <= 0 || L > kQ8TreeMost || (D != 128 && D != 64) || max_blocks <= 0 || !group_ok(Hq, Hkv) || (int64_t)B * Hkv > kDecodeMaxUnits) return 0;
  return ag_align256(ag_ws_q8_tree_floats(kMostCu, L * (Hq / Hkv), D) * sizeof(float)) + 4096;
}

ag_status ag_q8_tree_attn(ag_ctx *ctx, void *hip_stream, const void *q, const void *k, const void *v, const uint8_t *flags,
                          const int32_t *parent, int L, int Hq, const ag_rope *rope, float scale, const ag_q8_cache *cache, void *out) {
  if (!ctx) return AG_EINVAL;
  AG_REQUIRE(q && k && v && parent && out, AG_EINVAL, "ag_q8_tree_attn: null pointer");
  AG_REQUIRE(L > 0, AG_EINVAL, "ag_q8_tree_attn: L must be positive");
  AG_REQUIRE(L <= kQ8TreeMost, AG_EUNSUPPORTED, "ag_q8_tree_attn: L = %d exceeds %d", L, kQ8TreeMost);
  AG_REQUIRE(scale > 0.f && isfinite(scale), AG_EINVAL, "ag_q8_tree_attn: scale must be positive and finite");
  ag_q8_dev c;
  ag_status st = check_q8(ctx, "ag_q8_tree_attn", cache, &c);
  if (st != AG_OK) return st;
  AG_REQUIRE(Hq > 0 && Hq % cache->Hkv == 0, AG_EINVAL, "ag_q8_tree_attn: Hq must be a positive multiple of Hkv");
  AG_REQUIRE(group_ok(Hq, cache->Hkv), AG_EUNSUPPORTED, "ag_q8_tree_attn: %d query heads per KV head", Hq / cache->Hkv);
  AG_REQUIRE(aligned({q, k, v, out}), AG_EINVAL, "ag_q8_tree_attn: tensors must be 16-byte aligned");
  const int units = cache->B * cache->Hkv, rows = L * (Hq / cache->Hkv);
  AG_REQUIRE(ag_q8_tree_cost(units, rows, cache->max_blocks) < (1ll << 31), AG_EUNSUPPORTED,
             "ag_q8_tree_attn: cache: %d units of max_blocks = %d are too many", units, cache->max_blocks);
  ag_rope_dev r;
  st = check_rope(ctx, "ag_q8_tree_attn", rope, cache->D, (int64_t)cache->B * L, &r);
  if (st != AG_OK) return st;
  ws_cursor ws{ctx->ws, ctx->ws_bytes, 0, true};
  float *rec = ws.take<float>(ag_ws_q8_tree_floats(ctx->num_cu, rows, cache->D));
  AG_REQUIRE(ws.ok, AG_EWORKSPACE, "ag_q8_tree_attn: workspace of %zu bytes is too small (need %zu)", ctx->ws_bytes, ws.off);
  st = ag_need_device(ctx);
  if (st != AG_OK) return st;
  AG_HIP(ag_launch_q8_tree(ctx, (hipStream_t)hip_stream, q, k, v, flags, parent, cache->B, Hq, cache->Hkv, L, cache->D, r, scale, c, out, rec));
  return AG_OK;
}

ag_status ag_q8_tree_append(ag_ctx *ctx, void *hip_stream, const void *k, const void *v, const uint8_t *flags, const int32_t *parent,
                            const int32_t *last, int L, const ag_rope *rope, ag_q8_cache *cache) {
  if (!ctx) return AG_EINVAL;
  AG_REQUIRE(k && v && parent && last, AG_EINVAL, "ag_q8_tree_append: null pointer");
  AG_REQUIRE(L > 0, AG_EINVAL, "ag_q8_tree_append: L must be positive");
  AG_REQUIRE(L <= kQ8TreeMost, AG_EUNSUPPORTED, "ag_q8_tree_append: L = %d exceeds %d", L, kQ8TreeMost);
  ag_q8_dev c;
  ag_status st = check_q8(ctx, "ag_q8_tree_append", cache, &c);
  if (st != AG_OK) return st;
  AG_REQUIRE(aligned({k, v}), AG_EINVAL, "ag_q8_tree_append: k and v must be 16-byte aligned");
  ag_rope_dev r;
  st = check_rope(ctx, "ag_q8_tree_append", rope, cache->D, (int64_t)cache->B * L, &r);
  if (st != AG_OK) return st;
  st = ag_need_device(ctx);
  if (st != AG_OK) return st;
  AG_HIP(ag_launch_q8_tree_append(ctx, (hipStream_t)hip_stream, k, v, flags, parent, last, cache->B, cache->Hkv, L, cache->D, r, c));
  return AG_OK;
}

size_t ag_q8_pool_workspace_bytes(int B, int Hkv, int n_pages) {
  if (B <= 0 || Hkv <= 0 || (int64_t)B * Hkv > kDecodeMaxUnits || n_pages <= 0 || n_pages > kQ8MaxPages) return 0;
  ws_cursor ws{nullptr, ~size_t(0) >> 1, 0, true};
  take_pool(ws, B * Hkv, n_pages);
  return ws.off + 4096;
}

ag_status ag_q8_reserve(ag_ctx *ctx, void *hip_stream, ag_q8_cache *cache, int32_t *ref, int rows) {
  if (!ctx) return AG_EINVAL;
  ag_q8_dev c;
  ag_status st = check_pool(ctx, "ag_q8_reserve", cache, ref, &c);
  if (st != AG_OK) return st;
  AG_REQUIRE(rows >= 0, AG_EINVAL, "ag_q8_reserve: rows is negative");
  const int units = cache->B * cache->Hkv;
  ws_cursor ws{ctx->ws, ctx->ws_bytes, 0, true};
  const ag_q8_pool_ws w = take_pool(ws, units, cache->n_pages);
  AG_REQUIRE(ws.ok, AG_EWORKSPACE, "ag_q8_reserve: workspace of %zu bytes is too small (need %zu)", ctx->ws_bytes, ws.off);
  st = ag_need_device(ctx);
  if (st != AG_OK) return st;
  AG_HIP(ag_launch_q8_reserve(ctx, (hipStream_t)hip_stream, units, c, table_of(cache), ref, rows, w));
  return AG_OK;
}

ag_status ag_q8_fork(ag_ctx *ctx, void *hip_stream, const ag_q8_cache *src, const int32_t *parent, ag_q8_cache *dst, int32_t *ref) {
  if (!ctx) return AG_EINVAL;
  ag_q8_dev from, to;
  ag_status st = check_pool(ctx, "ag_q8_fork", src, ref, &from);
  if (st == AG_OK) st = check_pool(ctx, "ag_q8_fork", dst, ref, &to);
  if (st != AG_OK) return st;
  AG_REQUIRE(parent, AG_EINVAL, "ag_q8_fork: null pointer");
  AG_REQUIRE(src->k == dst->k && src->v == dst->v && src->k_scale == dst->k_scale && src->v_scale == dst->v_scale && src->n_pages == dst->n_pages,
             AG_EINVAL, "ag_q8_fork: src and dst are not caches over one pool");
  AG_REQUIRE(src->Hkv == dst->Hkv && src->D == dst->D, AG_EINVAL, "ag_q8_fork: src and dst differ in their heads");
  AG_REQUIRE(dst->max_blocks >= src->max_blocks, AG_EINVAL, "ag_q8_fork: dst's table is shorter than src's");
  AG_REQUIRE(src->page != dst->page && src->len != dst->len && src->k_tail != dst->k_tail && src->v_tail != dst->v_tail, AG_EINVAL,
             "ag_q8_fork: src and dst share a table, lengths or tails");
  st = ag_need_device(ctx);
  if (st != AG_OK) return st;
  AG_HIP(ag_launch_q8_fork(ctx, (hipStream_t)hip_stream, from, src->B, parent, to, table_of(dst), dst->B, dst->Hkv, dst->D, ref));
  return AG_OK;
}

ag_status ag_q8_release(ag_ctx *ctx, void *hip_stream, ag_q8_cache *cache, int32_t *ref, const uint8_t *which) {
  if (!ctx) return AG_EINVAL;
  ag_q8_dev c;
  ag_status st = check_pool(ctx, "ag_q8_release", cache, ref, &c);
  if (st != AG_OK) return st;
  st = ag_need_device(ctx);
  if (st != AG_OK) return st;
  AG_HIP(ag_launch_q8_release(ctx, (hipStream_t)hip_stream, cache->B, cache->Hkv, c, table_of(cache), ref, which));
  return AG_OK;
}

ag_status ag_q8_compact_pages(ag_ctx *ctx, void *hip_stream, ag_q8_cache *cache, int32_t *ref, int32_t *moved, int32_t *used) {
  if (!ctx) return AG_EINVAL;
  ag_q8_dev c;
  ag_status st = check_pool(ctx, "ag_q8_compact_pages", cache, ref, &c);
  if (st != AG_OK) return st;
  AG_REQUIRE(moved && used, AG_EINVAL, "ag_q8_compact_pages: null pointer");
  AG_REQUIRE(moved != ref && used != ref && used != moved, AG_EINVAL, "ag_q8_compact_pages: ref, moved and used share an address");
  ws_cursor ws{ctx->ws, ctx->ws_bytes, 0, true};
  const ag_q8_pool_ws w = take_pool(ws, 1, cache->n_pages);
  AG_REQUIRE(ws.ok, AG_EWORKSPACE, "ag_q8_compact_pages: workspace of %zu bytes is too small (need %zu)", ctx->ws_bytes, ws.off);
  st = ag_need_device(ctx);
  if (st != AG_OK) return st;
  AG_HIP(ag_launch_q8_compact_pages(ctx, (hipStream_t)hip_stream, c, cache->D, ref, moved, used, w));
  return AG_OK;
}

ag_status ag_q8_remap(ag_ctx *ctx, void *hip_stream, ag_q8_cache *cache, const int32_t *moved) {
  if (!ctx) return AG_EINVAL;
  ag_q8_dev c;
  ag_status st = check_pool(ctx, "ag_q8_remap", cache, moved, &c);
  if (st != AG_OK) return st;
  st = ag_need_device(ctx);
  if (st != AG_OK) return st;
  AG_HIP(ag_launch_q8_remap(ctx, (hipStream_t)hip_stream, cache->B * cache->Hkv, c, table_of(cache), moved));
  return AG_OK;
}

}  // extern "C"
