// C ABI of the key/value cache operators: host-side validation and launches on the caller's
// stream. Every check runs on the host before any device work is enqueued.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdio>
#include <memory>

#include "rrs.h"
#include "rrs_check.h"
#include "rrs_kv.h"

using rrs::check_device;
using rrs::debug_check_finite_f16;
using rrs::debug_enabled;
using rrs::debug_fetch_new;
using rrs::from_hip;
using rrs::is_aligned;

namespace {

bool any_null(const rrs_kv_cache* c) {
  return !c || !c->k || !c->v || !c->table ||
         (c->format == RRS_KV_INT4 && (!c->k_scale || !c->v_scale));
}

bool valid_shape(const rrs_kv_cache& c) {
  const int P = c.page_size;
  return (c.head_dim == 64 || c.head_dim == 128 || c.head_dim == 256) &&
         (P == 16 || P == 32 || P == 64 || P == 128 || P == 256) && c.pages >= 1 &&
         c.kv_heads >= 1 && c.sequences >= 1 && c.max_pages >= 1 &&
         (int64_t)c.sequences * c.kv_heads < ((int64_t)1 << 23) &&
         (int64_t)c.max_pages * P <= ((int64_t)1 << 30);
}

int capacity(const rrs_kv_cache& c) { return c.max_pages * c.page_size; }

bool valid_heads(const rrs_kv_cache& c, int heads) {
  return heads >= 1 && heads % c.kv_heads == 0 &&
         (int64_t)c.sequences * heads < ((int64_t)1 << 23);
}

bool valid_format(const rrs_kv_cache& c) {
  return c.format == RRS_KV_F16 || c.format == RRS_KV_INT4;
}

bool aligned(const rrs_kv_cache& c) {
  return is_aligned(c.k) && is_aligned(c.v) && is_aligned(c.table) &&
         (c.format != RRS_KV_INT4 || (is_aligned(c.k_scale) && is_aligned(c.v_scale)));
}

rrs::KvView view(const rrs_kv_cache& c) {
  const bool q = c.format == RRS_KV_INT4;
  int log_page = 0;
  while ((1 << log_page) < c.page_size) ++log_page;
  return rrs::KvView{static_cast<uint8_t*>(c.k),
                     static_cast<uint8_t*>(c.v),
                     q ? static_cast<uint16_t*>(c.k_scale) : nullptr,
                     q ? static_cast<uint16_t*>(c.v_scale) : nullptr,
                     c.table,
                     c.pages,
                     c.kv_heads,
                     log_page,
                     c.head_dim,
                     c.sequences,
                     c.max_pages};
}

// ---------------------------------------------------------------------------
// RRS_DEBUG: device indices are what the call needs. As in rrs_api.cpp these copy
// to host memory on the caller's stream and wait.
// ---------------------------------------------------------------------------

// lo <= every entry < hi.
rrs_status debug_check_range(const int32_t* p, size_t count, int64_t lo, int64_t hi,
                             const char* what, void* stream) {
  std::unique_ptr<int32_t[]> h;
  if (rrs_status e = debug_fetch_new(&h, p, count, stream)) return e;
  for (size_t i = 0; i < count; ++i)
    if (h[i] < lo || h[i] >= hi) {
      std::fprintf(stderr, "[rrs] RRS_DEBUG: %s[%zu] = %d is outside [%lld, %lld)\n", what, i,
                   (int)h[i], (long long)lo, (long long)hi);
      return RRS_ERR_PRECONDITION;
    }
  return RRS_OK;
}

// Lengths within max_length, and the pages of every slot below them within the cache.
rrs_status debug_check_lengths(const rrs_kv_cache& c, const int32_t* lengths, int max_length,
                               void* stream) {
  if (rrs_status e = debug_check_range(lengths, (size_t)c.sequences, 0, (int64_t)max_length + 1,
                                       "lengths", stream))
    return e;
  std::unique_ptr<int32_t[]> n, t;
  if (rrs_status e = debug_fetch_new(&n, lengths, (size_t)c.sequences, stream)) return e;
  if (rrs_status e =
          debug_fetch_new(&t, c.table, (size_t)c.sequences * (size_t)c.max_pages, stream))
    return e;
  for (int b = 0; b < c.sequences; ++b)
    for (int i = 0; (int64_t)i * c.page_size < n[(size_t)b]; ++i) {
      const int32_t p = t[(size_t)b * (size_t)c.max_pages + (size_t)i];
      if (p < 0 || p >= c.pages) {
        std::fprintf(stderr, "[rrs] RRS_DEBUG: table[%d][%d] = %d is outside [0, %d)\n", b, i,
                     (int)p, (int)c.pages);
        return RRS_ERR_PRECONDITION;
      }
    }
  return RRS_OK;
}

// The pages that M tokens are written to are pages of the cache.
rrs_status debug_check_places(const rrs_kv_cache& c, const int32_t* seq, const int32_t* slot,
                              int M, void* stream) {
  std::unique_ptr<int32_t[]> b, s, t;
  if (rrs_status e = debug_fetch_new(&b, seq, (size_t)M, stream)) return e;
  if (rrs_status e = debug_fetch_new(&s, slot, (size_t)M, stream)) return e;
  if (rrs_status e =
          debug_fetch_new(&t, c.table, (size_t)c.sequences * (size_t)c.max_pages, stream))
    return e;
  for (int m = 0; m < M; ++m) {
    const int32_t bm = b[(size_t)m], sm = s[(size_t)m];
    if (bm < 0 || bm >= c.sequences || sm < 0 || sm >= capacity(c)) continue;  // not stored
    const int i = sm / c.page_size;
    const int32_t p = t[(size_t)bm * (size_t)c.max_pages + (size_t)i];
    if (p < 0 || p >= c.pages) {
      std::fprintf(stderr, "[rrs] RRS_DEBUG: table[%d][%d] = %d is outside [0, %d)\n", (int)bm, i,
                   (int)p, (int)c.pages);
      return RRS_ERR_PRECONDITION;
    }
  }
  return RRS_OK;
}

void debug_print(const char* call, const rrs_kv_cache* c) {
  if (!c) {
    std::fprintf(stderr, "[rrs] %s cache=NULL\n", call);
    return;
  }
  std::fprintf(stderr,
               "[rrs] %s k=%p v=%p k_scale=%p v_scale=%p table=%p format=%d pages=%d kv_heads=%d "
               "page_size=%d head_dim=%d sequences=%d max_pages=%d\n",
               call, c->k, c->v, c->k_scale, c->v_scale, (const void*)c->table, c->format,
               c->pages, c->kv_heads, c->page_size, c->head_dim, c->sequences, c->max_pages);
}

}  // namespace

extern "C" {

rrs_status rrs_rope_kv_append(const void* qkv, int64_t row_stride, int M, int heads,
                              const int32_t* positions, int axes, const int32_t* sections,
                              const float* rope, int rope_rows, int rotary_dim, int flags,
                              const rrs_kv_cache* cache, const int32_t* seq, const int32_t* slot,
                              void* Q, float* weights, int32_t* slot_pos, void* stream) {
  const bool debug = debug_enabled();
  if (debug) debug_print("rope_kv_append", cache);
  if (!qkv || !positions || !sections || !rope || !seq || !slot || !Q || any_null(cache))
    return RRS_ERR_NULL;
  const rrs_kv_cache& c = *cache;
  if (!valid_shape(c) || heads < 1 || M < 1 || !rrs::append_fits(M) || axes < 1 || axes > 4 || rope_rows < 1 ||
      rotary_dim < 16 || rotary_dim % 16 != 0 || rotary_dim > c.head_dim)
    return RRS_ERR_SHAPE;
  const int64_t width = ((int64_t)heads + 2 * (int64_t)c.kv_heads) * c.head_dim;
  if (width >= ((int64_t)1 << 31) || row_stride < width || row_stride % 8 != 0)
    return RRS_ERR_SHAPE;
  rrs::RopeArgs a{};
  int64_t sum = 0;
  for (int i = 0; i < 4; ++i) {
    if (i < axes) {
      if (sections[i] < 0) return RRS_ERR_SHAPE;
      sum += sections[i];
    }
    a.bound[i] = (int)(sum < rotary_dim ? sum : rotary_dim);
  }
  if (sum != rotary_dim / 2) return RRS_ERR_SHAPE;
  if (!valid_format(c) || (flags & ~RRS_ROPE_INTERLEAVED) != 0) return RRS_ERR_FLAGS;
  if (!aligned(c) || !is_aligned(qkv) || !is_aligned(positions) || !is_aligned(rope) ||
      !is_aligned(seq) || !is_aligned(slot) || !is_aligned(Q) || !is_aligned(weights) ||
      !is_aligned(slot_pos))
    return RRS_ERR_ALIGN;
  if (rrs_status s = check_device()) return s;
  if (debug) {
    for (int m = 0; m < M; ++m)
      if (rrs_status s = debug_check_finite_f16(
              static_cast<const uint16_t*>(qkv) + (size_t)m * (size_t)row_stride, (size_t)width,
              "qkv", stream))
        return s;
    if (rrs_status s = debug_check_range(positions, (size_t)M * (size_t)axes, 0, rope_rows,
                                         "positions", stream))
      return s;
    if (rrs_status s = debug_check_places(c, seq, slot, M, stream)) return s;
  }
  a.qkv = static_cast<const uint16_t*>(qkv);
  a.row_stride = row_stride;
  a.M = M;
  a.heads = heads;
  a.positions = positions;
  a.axes = axes;
  a.rope = rope;
  a.rope_rows = rope_rows;
  a.rotary_dim = rotary_dim;
  a.interleaved = (flags & RRS_ROPE_INTERLEAVED) != 0;
  a.seq = seq;
  a.slot = slot;
  a.Q = static_cast<uint16_t*>(Q);
  a.weights = weights;
  a.slot_pos = slot_pos;
  return from_hip(rrs::launch_rope_kv_append(a, view(c), static_cast<hipStream_t>(stream)));
}

size_t rrs_paged_attention_workspace_bytes(const rrs_kv_cache* cache, int heads, int max_length,
                                           int with_weights) {
  if (!cache || !valid_shape(*cache) || !valid_format(*cache) || !valid_heads(*cache, heads) ||
      max_length < 1 || max_length > capacity(*cache) ||
      !rrs::attention_fits(view(*cache), heads, max_length, with_weights != 0))
    return 0;
  return rrs::attention_workspace_bytes(view(*cache), heads, max_length, with_weights != 0);
}

rrs_status rrs_paged_attention(const void* Q, int heads, const rrs_kv_cache* cache,
                               const int32_t* lengths, int max_length, float scale,
                               const uint8_t* mask, float* weights, void* out, float* lse,
                               void* workspace, size_t workspace_bytes, void* stream) {
  const bool debug = debug_enabled();
  if (debug) debug_print("paged_attention", cache);
  if (!Q || !lengths || !out || any_null(cache)) return RRS_ERR_NULL;
  const rrs_kv_cache& c = *cache;
  if (!valid_shape(c) || !valid_heads(c, heads) || max_length < 1 || max_length > capacity(c) ||
      !rrs::attention_fits(view(c), heads, max_length, weights != nullptr))
    return RRS_ERR_SHAPE;
  if (!valid_format(c) || !std::isfinite(scale)) return RRS_ERR_FLAGS;
  const size_t need =
      rrs::attention_workspace_bytes(view(c), heads, max_length, weights != nullptr);
  if (need > 0 && !workspace) return RRS_ERR_NULL;
  if (!aligned(c) || !is_aligned(Q) || !is_aligned(lengths) || !is_aligned(mask) ||
      !is_aligned(weights) || !is_aligned(out) || !is_aligned(lse) || !is_aligned(workspace))
    return RRS_ERR_ALIGN;
  if (workspace_bytes < need) return RRS_ERR_WORKSPACE;
  if (rrs_status s = check_device()) return s;
  if (debug) {
    if (rrs_status s = debug_check_finite_f16(
            Q, (size_t)c.sequences * (size_t)heads * (size_t)c.head_dim, "Q", stream))
      return s;
    if (rrs_status s = debug_check_lengths(c, lengths, max_length, stream)) return s;
  }
  const rrs::AttentionArgs a{static_cast<const uint16_t*>(Q), heads, lengths, max_length, scale,
                             mask, weights, static_cast<uint16_t*>(out), lse, workspace};
  return from_hip(rrs::launch_paged_attention(a, view(c), static_cast<hipStream_t>(stream)));
}

size_t rrs_kv_evict_workspace_bytes(const rrs_kv_cache* cache, int max_length, int budget) {
  if (!cache || !valid_shape(*cache) || !valid_format(*cache) || max_length < 1 ||
      max_length > capacity(*cache) || budget < 1 || budget > capacity(*cache) ||
      !rrs::evict_fits(view(*cache), max_length, budget))
    return 0;
  return rrs::evict_workspace_bytes(view(*cache), max_length, budget);
}

rrs_status rrs_kv_evict(const rrs_kv_cache* cache, const int32_t* lengths, int max_length,
                        const float* weights, const int32_t* slot_pos, const int32_t* keep_from,
                        int budget, int32_t* kept, int32_t* new_lengths, float* weights_out,
                        int32_t* pos_out, void* workspace, size_t workspace_bytes, void* stream) {
  const bool debug = debug_enabled();
  if (debug) debug_print("kv_evict", cache);
  if (!lengths || !weights || !slot_pos || !keep_from || !kept || !new_lengths || !weights_out ||
      !pos_out || any_null(cache))
    return RRS_ERR_NULL;
  const rrs_kv_cache& c = *cache;
  if (!valid_shape(c) || max_length < 1 || max_length > capacity(c) || budget < 1 ||
      budget > capacity(c) || !rrs::evict_fits(view(c), max_length, budget))
    return RRS_ERR_SHAPE;
  if (!valid_format(c)) return RRS_ERR_FLAGS;
  const size_t need = rrs::evict_workspace_bytes(view(c), max_length, budget);
  if (need > 0 && !workspace) return RRS_ERR_NULL;
  if (!aligned(c) || !is_aligned(workspace) || !is_aligned(lengths) || !is_aligned(weights) || !is_aligned(slot_pos) ||
      !is_aligned(keep_from) || !is_aligned(kept) || !is_aligned(new_lengths) ||
      !is_aligned(weights_out) || !is_aligned(pos_out))
    return RRS_ERR_ALIGN;
  if (workspace_bytes < need) return RRS_ERR_WORKSPACE;
  if (rrs_status s = check_device()) return s;
  if (debug)
    if (rrs_status s = debug_check_lengths(c, lengths, max_length, stream)) return s;
  const rrs::EvictArgs a{lengths, max_length, weights,     slot_pos,    keep_from,
                         budget,  kept,       new_lengths, weights_out, pos_out};
  return from_hip(rrs::launch_kv_evict(a, view(c), workspace, static_cast<hipStream_t>(stream)));
}

rrs_status rrs_kv_read(const rrs_kv_cache* cache, const int32_t* lengths, int max_length, void* K,
                       void* V, void* stream) {
  const bool debug = debug_enabled();
  if (debug) debug_print("kv_read", cache);
  if (!lengths || !K || !V || any_null(cache)) return RRS_ERR_NULL;
  const rrs_kv_cache& c = *cache;
  if (!valid_shape(c) || max_length < 1 || max_length > capacity(c) ||
      !rrs::read_fits(view(c), max_length))
    return RRS_ERR_SHAPE;
  if (!valid_format(c)) return RRS_ERR_FLAGS;
  if (!aligned(c) || !is_aligned(lengths) || !is_aligned(K) || !is_aligned(V))
    return RRS_ERR_ALIGN;
  if (rrs_status s = check_device()) return s;
  if (debug)
    if (rrs_status s = debug_check_lengths(c, lengths, max_length, stream)) return s;
  return from_hip(rrs::launch_kv_read(view(c), lengths, max_length, static_cast<uint16_t*>(K),
                                      static_cast<uint16_t*>(V),
                                      static_cast<hipStream_t>(stream)));
}

}  // extern "C"
