// Entry points of the long-context operators: rotary positions, the 8-bit KV
// cache's append and attention, its eviction.  Host-side validation and launches,
// as in api.cpp: no kernel is launched unless every check passes.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>

#include "kernels.hpp"
#include "stage.hpp"

using namespace tri;

tri_status tri::check_kv8_cache(const tri_kv8_cache* c) {
  if (!c) return TRI_ERR_NULL;
  if (!c->k || !c->v || !c->k_scale || !c->v_scale) return TRI_ERR_NULL;
  if (c->n_slots <= 0 || c->max_seq <= 0) return TRI_ERR_SHAPE;
  if (c->max_seq > 1 << 23) return TRI_ERR_RANGE;  // a head's rows within 32-bit offsets
  if (c->format != TRI_KV8_INT8 && c->format != TRI_KV8_E4M3) return TRI_ERR_UNSUPPORTED;
  if (c->scale_rows != 32 && c->scale_rows != 64 && c->scale_rows != 128) return TRI_ERR_UNSUPPORTED;
  if (c->block_table) {
    if (c->block_size <= 0 || c->n_blocks <= 0) return TRI_ERR_SHAPE;
    if (c->block_size % 64 != 0) return TRI_ERR_UNSUPPORTED;
    if (c->block_size % c->scale_rows != 0 || c->max_seq % c->block_size != 0) return TRI_ERR_SHAPE;
  }
  if (!aligned16(c->k) || !aligned16(c->v)) return TRI_ERR_ALIGN;
  for (const void* p : {(const void*)c->k_scale, (const void*)c->v_scale, (const void*)c->mass,
                        (const void*)c->stamp, (const void*)c->block_table})
    if ((uintptr_t)p & 3u) return TRI_ERR_ALIGN;
  return TRI_OK;
}

Kv8Dev tri::kv8_dev(const tri_kv8_cache* c) {
  Kv8Dev d{};
  d.kv = KvDev{c->n_slots, c->max_seq, c->block_table, c->block_table ? c->block_size : 0,
               c->block_table ? c->n_blocks : 0};
  d.k = (uint8_t*)c->k;
  d.v = (uint8_t*)c->v;
  d.k_scale = c->k_scale;
  d.v_scale = c->v_scale;
  d.mass = c->mass;
  d.stamp = c->stamp;
  d.scale_shift = c->scale_rows == 32 ? 5 : (c->scale_rows == 64 ? 6 : 7);
  return d;
}

constexpr int kMaxGrid = 65535;  // y and z extents of a grid

tri_status tri::check_kv8_batch(const tri_kv8_cache* cache, const tri_batch* b) {
  if (b->n_seqs > kMaxGrid) return TRI_ERR_RANGE;
  if (b->max_ctx_len > cache->max_seq || b->max_q_len > cache->max_seq) return TRI_ERR_RANGE;
  if (b->n_tokens > 0 && b->max_ctx_len >= cache->max_seq) return TRI_ERR_RANGE;
  return TRI_OK;
}

tri_status tri::check_kv8_queries(const tri_layer_config* c, const tri_batch* b) {
  if (c->n_q_heads > kMaxGrid) return TRI_ERR_RANGE;
  return (int64_t)b->n_tokens * c->n_q_heads > kMaxPackedRows ? TRI_ERR_RANGE : TRI_OK;
}

namespace {

// The fields of the layer config that these operators read.
tri_status check_heads(const tri_layer_config* c) {
  if (!c) return TRI_ERR_NULL;
  if (c->dtype != TRI_BF16) return TRI_ERR_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128) return TRI_ERR_UNSUPPORTED;
  if (c->n_kv_heads <= 0) return TRI_ERR_SHAPE;
  if (c->n_kv_heads > kMaxGrid) return TRI_ERR_RANGE;
  return TRI_OK;
}

BatchDev batch_dev(const tri_batch* b) {
  return BatchDev{b->cu_q, b->ctx_len, b->slot, b->pos, b->n_seqs, b->n_tokens, b->max_q_len,
                  b->max_ctx_len};
}

// Config, cache and batch of one call; a batch without sequences passes unread.
tri_status check_call(const tri_layer_config* cfg, const tri_kv8_cache* cache, const tri_batch* b) {
  tri_status st = check_heads(cfg);
  if (st != TRI_OK) return st;
  if (!cache) return TRI_ERR_NULL;
  if ((st = check_batch_scalars(b)) != TRI_OK) return st;
  if (b->n_seqs == 0) return TRI_OK;
  if ((st = check_kv8_cache(cache)) != TRI_OK) return st;
  return check_kv8_batch(cache, b);
}

tri_status check_group(const tri_layer_config* c) {
  if (c->n_q_heads <= 0 || c->n_q_heads % c->n_kv_heads != 0) return TRI_ERR_SHAPE;
  if (c->n_q_heads / c->n_kv_heads > 32) return TRI_ERR_UNSUPPORTED;
  return TRI_OK;
}

tri_status check_budget(const tri_kv8_cache* c, int32_t budget) {
  if (budget <= 0 || budget % c->scale_rows != 0) return TRI_ERR_SHAPE;
  return budget > c->max_seq ? TRI_ERR_RANGE : TRI_OK;
}

// Bytes from the first to the last element of T rows of `width`, `stride` apart.
size_t extent(int64_t rows, int64_t width, int64_t stride, int size) {
  return (size_t)((rows - 1) * stride + width) * size;
}

// What a configuration and its table share.
template <typename C>
tri_status check_rope_dims(const C* c) {
  if (c->head_dim < 2 || c->head_dim > 2 * TRI_ROPE_MAX_PAIRS || c->head_dim % 2)
    return TRI_ERR_UNSUPPORTED;
  if (c->rotary_dim < 2 || c->rotary_dim > c->head_dim || c->rotary_dim % 2) return TRI_ERR_SHAPE;
  if (c->layout != TRI_ROPE_HALF && c->layout != TRI_ROPE_INTERLEAVED) return TRI_ERR_UNSUPPORTED;
  return isfinite(c->magnitude) ? TRI_OK : TRI_ERR_RANGE;
}

tri_status check_rope(const tri_rope_config* c) {
  if (!c) return TRI_ERR_NULL;
  const tri_status st = check_rope_dims(c);
  if (st != TRI_OK) return st;
  if (c->scaling < TRI_ROPE_PLAIN || c->scaling > TRI_ROPE_INDEX) return TRI_ERR_UNSUPPORTED;
  if (!(c->base > 0.f) || !isfinite(c->base)) return TRI_ERR_RANGE;
  if (c->scaling != TRI_ROPE_PLAIN && (!(c->factor > 0.f) || !isfinite(c->factor))) return TRI_ERR_RANGE;
  if (c->scaling == TRI_ROPE_TURNS || c->scaling == TRI_ROPE_INDEX) {
    if (c->original_len <= 0 || !(c->low > 0.f) || !(c->high > c->low) || !isfinite(c->high))
      return TRI_ERR_RANGE;
    if (c->scaling == TRI_ROPE_INDEX && !(c->base > 1.f)) return TRI_ERR_RANGE;
  }
  return TRI_OK;
}

// Every pair's turns per position, f / 2 pi (the formulas of tri_rope_config).
void rope_turns(const tri_rope_config* c, double* turns) {
  const double two_pi = 6.283185307179586, n = c->rotary_dim, factor = c->factor;
  double base = c->base;
  if (c->scaling == TRI_ROPE_BASE && c->rotary_dim > 2) base *= pow(factor, n / (n - 2));
  double lo = 0, hi = 0;
  if (c->scaling == TRI_ROPE_INDEX) {
    auto at = [&](double turns) { return n * log(c->original_len / (two_pi * turns)) / (2 * log(base)); };
    lo = std::max(floor(at(c->high)), 0.0);
    hi = std::min(ceil(at(c->low)), n - 1);
  }
  for (int i = 0; i < c->rotary_dim / 2; ++i) {
    const double w = pow(base, -2.0 * i / n);
    double f = w;
    if (c->scaling == TRI_ROPE_LINEAR) f = w / factor;
    if (c->scaling == TRI_ROPE_TURNS) {
      const double t = std::min(1.0, std::max(0.0, (c->original_len * w / two_pi - c->low) /
                                                       ((double)c->high - c->low)));
      f = w * (t + (1 - t) / factor);
    }
    if (c->scaling == TRI_ROPE_INDEX) {
      const double u = std::min(1.0, std::max(0.0, (i - lo) / std::max(hi - lo, 0.001)));
      f = w * (1 - u) + w / factor * u;
    }
    turns[i] = f / two_pi;
  }
}

}  // namespace

extern "C" {

tri_status tri_rope_table_make(const tri_rope_config* cfg, tri_rope_table* table) {
  if (!table) return TRI_ERR_NULL;
  const tri_status st = check_rope(cfg);
  if (st != TRI_OK) return st;
  *table = tri_rope_table{cfg->head_dim, cfg->rotary_dim, cfg->layout, cfg->magnitude, {}};
  rope_turns(cfg, table->turns);
  return TRI_OK;
}

tri_status tri_rope(const tri_rope_table* cfg, const void* x, int64_t x_stride, void* y,
                    int64_t y_stride, const int32_t* pos, int32_t n_tokens, int32_t n_heads,
                    int32_t dtype, void* stream) {
  if (!cfg) return TRI_ERR_NULL;
  tri_status st = check_rope_dims(cfg);
  if (st != TRI_OK) return st;
  if (dtype != TRI_BF16 && dtype != TRI_F32) return TRI_ERR_UNSUPPORTED;
  if (n_tokens < 0 || n_heads < 0) return TRI_ERR_SHAPE;
  const int64_t width = (int64_t)n_heads * cfg->head_dim;
  if (x_stride < width || y_stride < width) return TRI_ERR_SHAPE;
  if (width > 1 << 24) return TRI_ERR_RANGE;  // 32-bit counts within a workgroup
  if (n_tokens == 0 || n_heads == 0) return TRI_OK;
  if (!x || !y || !pos) return TRI_ERR_NULL;
  const int size = dtype == TRI_F32 ? 4 : 2;
  if ((uintptr_t)x % size || (uintptr_t)y % size || (uintptr_t)pos % 4) return TRI_ERR_ALIGN;
  if (!(x == y && x_stride == y_stride) &&
      overlaps(x, extent(n_tokens, width, x_stride, size), y,
               extent(n_tokens, width, y_stride, size)))
    return TRI_ERR_ALIAS;
  TRI_HIP(launch_rope(*cfg, n_heads, x, x_stride, y, y_stride, pos, n_tokens, dtype == TRI_F32,
                      (hipStream_t)stream));
  return TRI_OK;
}

tri_status tri_kv8_append(const tri_layer_config* cfg, const tri_kv8_cache* cache,
                          const tri_batch* b, const void* k_new, const void* v_new, int64_t stride,
                          void* stream) {
  tri_status st = check_call(cfg, cache, b);
  if (st != TRI_OK) return st;
  if (b->n_tokens == 0) return TRI_OK;
  if (!k_new || !v_new || !b->cu_q || !b->ctx_len || !b->slot) return TRI_ERR_NULL;
  if (cache->stamp && !b->pos) return TRI_ERR_NULL;
  if (stride < (int64_t)cfg->n_kv_heads * cfg->head_dim) return TRI_ERR_SHAPE;
  if (stride % 8 || !aligned16(k_new) || !aligned16(v_new)) return TRI_ERR_ALIGN;
  StageTimer t_(ST_APPEND, (hipStream_t)stream);
  TRI_HIP(launch_kv8_append(batch_dev(b), kv8_dev(cache), cache->format == TRI_KV8_E4M3,
                            cfg->n_kv_heads, cfg->head_dim, k_new, v_new, stride,
                            (hipStream_t)stream));
  return TRI_OK;
}

tri_status tri_kv8_attention_workspace_size(const tri_layer_config* cfg,
                                            const tri_kv8_cache* cache, const tri_batch* b,
                                            size_t* bytes) {
  if (!bytes) return TRI_ERR_NULL;
  tri_status st = check_call(cfg, cache, b);
  if (st == TRI_OK) st = check_group(cfg);
  if (st == TRI_OK) st = check_kv8_queries(cfg, b);
  if (st != TRI_OK) return st;
  *bytes = b->n_tokens == 0 ? 0 : attn_kv8_workspace_bytes(batch_dev(b), kv8_dev(cache), cfg->n_q_heads,
                                                           cfg->n_kv_heads, cfg->head_dim);
  return TRI_OK;
}

tri_status tri_kv8_attention(const tri_layer_config* cfg, const tri_kv8_cache* cache,
                             const tri_batch* b, const void* q, int64_t q_stride, void* out,
                             void* ws, size_t ws_bytes, void* stream) {
  size_t need = 0;
  tri_status st = tri_kv8_attention_workspace_size(cfg, cache, b, &need);
  if (st != TRI_OK) return st;
  if (b->n_tokens == 0) return TRI_OK;
  if (!q || !out || !b->cu_q || !b->ctx_len || !b->slot) return TRI_ERR_NULL;
  const int64_t width = (int64_t)cfg->n_q_heads * cfg->head_dim;
  if (q_stride < width) return TRI_ERR_SHAPE;
  if (q_stride > 1 << 22) return TRI_ERR_RANGE;  // 31-bit byte offsets within a tile of rows
  if (q_stride % 8 || !aligned16(q) || !aligned16(out)) return TRI_ERR_ALIGN;
  if (need > 0 && (!ws || ws_bytes < need)) return TRI_ERR_WORKSPACE;
  if (need > 0 && ((uintptr_t)ws & (kAlign - 1)) != 0) return TRI_ERR_ALIGN;
  const size_t q_bytes = extent(b->n_tokens, width, q_stride, 2);
  const size_t out_bytes = (size_t)b->n_tokens * width * 2;
  if (overlaps(q, q_bytes, out, out_bytes)) return TRI_ERR_ALIAS;
  if (need > 0 && (overlaps(ws, need, q, q_bytes) || overlaps(ws, need, out, out_bytes)))
    return TRI_ERR_ALIAS;
  TRI_HIP(launch_attn_kv8(batch_dev(b), kv8_dev(cache), cache->format == TRI_KV8_E4M3,
                          cfg->n_q_heads, cfg->n_kv_heads, cfg->head_dim, q, q_stride, out, ws,
                          (hipStream_t)stream));
  return TRI_OK;
}

tri_status tri_kv8_select_workspace_size(const tri_layer_config* cfg, const tri_kv8_cache* cache,
                                         const tri_batch* b, int32_t budget, size_t* bytes) {
  if (!bytes) return TRI_ERR_NULL;
  tri_status st = check_call(cfg, cache, b);
  if (st != TRI_OK) return st;
  *bytes = 0;
  if (b->n_seqs == 0) return TRI_OK;
  if ((st = check_budget(cache, budget)) != TRI_OK) return st;
  *bytes = kv8_select_workspace_bytes(batch_dev(b), cfg->n_kv_heads, budget);
  return TRI_OK;
}

tri_status tri_kv8_select(const tri_layer_config* cfg, const tri_kv8_cache* cache,
                          const tri_batch* b, int32_t budget, int32_t n_first, int32_t n_recent,
                          int32_t* plan, int32_t* new_len, void* ws, size_t ws_bytes,
                          void* stream) {
  size_t need = 0;
  tri_status st = tri_kv8_select_workspace_size(cfg, cache, b, budget, &need);
  if (st != TRI_OK) return st;
  if (b->n_seqs == 0) return TRI_OK;
  if (!plan || !cache->mass || !b->cu_q || !b->ctx_len || !b->slot) return TRI_ERR_NULL;
  if (n_first < 0 || n_recent < 0 || (int64_t)n_first + n_recent > budget) return TRI_ERR_SHAPE;
  if ((uintptr_t)plan % 4 || (uintptr_t)new_len % 4) return TRI_ERR_ALIGN;
  if (need > 0 && (!ws || ws_bytes < need)) return TRI_ERR_WORKSPACE;
  if (need > 0 && ((uintptr_t)ws & (kAlign - 1)) != 0) return TRI_ERR_ALIGN;
  const size_t plan_bytes = (size_t)b->n_seqs * cfg->n_kv_heads * budget * 4;
  if (need > 0 && overlaps(ws, need, plan, plan_bytes)) return TRI_ERR_ALIAS;
  TRI_HIP(launch_kv8_select(batch_dev(b), kv8_dev(cache), cfg->n_kv_heads, budget, n_first, n_recent,
                            plan, new_len, ws, (hipStream_t)stream));
  return TRI_OK;
}

tri_status tri_kv8_move(const tri_layer_config* cfg, const tri_kv8_cache* cache,
                        const tri_batch* b, const int32_t* plan, int32_t budget, void* stream) {
  tri_status st = check_call(cfg, cache, b);
  if (st != TRI_OK) return st;
  if (b->n_seqs == 0) return TRI_OK;
  if (!plan || !b->slot) return TRI_ERR_NULL;
  if ((st = check_budget(cache, budget)) != TRI_OK) return st;
  if ((uintptr_t)plan % 4) return TRI_ERR_ALIGN;
  TRI_HIP(launch_kv8_move(batch_dev(b), kv8_dev(cache), cache->format == TRI_KV8_E4M3,
                          cfg->n_kv_heads, cfg->head_dim, plan, budget, (hipStream_t)stream));
  return TRI_OK;
}

}  // extern "C"
