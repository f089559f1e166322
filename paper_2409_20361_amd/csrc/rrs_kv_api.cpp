// C ABI of the key/value cache operators: host-side validation and launches on the caller's
// stream. Every check runs on the host before any device work is enqueued.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <memory>

#include "rrs.h"
#include "rrs_check.h"
#include "rrs_kv.h"

using rrs::check_device;
using rrs::debug_check_finite_f16;
using rrs::debug_enabled;
using rrs::debug_fetch;
using rrs::debug_fetch_new;
using rrs::from_hip;
using rrs::is_aligned;

namespace {

bool has_scales(const rrs_kv_cache& c) {
  return c.format == RRS_KV_INT4 || c.format == RRS_KV_FP8;
}

bool any_null(const rrs_kv_cache* c) {
  return !c || !c->k || !c->v || !c->table ||
         (has_scales(*c) && (!c->k_scale || !c->v_scale));
}

bool valid_page_size(int P) {
  return P == 16 || P == 32 || P == 64 || P == 128 || P == 256;
}

bool valid_shape(const rrs_kv_cache& c) {
  const int P = c.page_size;
  return (c.head_dim == 64 || c.head_dim == 128 || c.head_dim == 256) &&
         valid_page_size(P) && c.pages >= 1 &&
         c.kv_heads >= 1 && c.sequences >= 1 && c.max_pages >= 1 &&
         (int64_t)c.sequences * c.kv_heads < ((int64_t)1 << 23) &&
         (int64_t)c.max_pages * P <= ((int64_t)1 << 30);
}

int log2_of(int P) {
  int l = 0;
  while ((1 << l) < P) ++l;
  return l;
}

bool valid_table(int sequences, int max_pages, int page_size, int pages) {
  return valid_page_size(page_size) && sequences >= 1 && sequences < (1 << 23) && max_pages >= 1 &&
         (int64_t)max_pages * page_size <= ((int64_t)1 << 30) && pages >= 1 &&
         pages <= rrs::most_pages();
}

int capacity(const rrs_kv_cache& c) { return c.max_pages * c.page_size; }

bool valid_heads(const rrs_kv_cache& c, int heads) {
  return heads >= 1 && heads % c.kv_heads == 0 &&
         (int64_t)c.sequences * heads < ((int64_t)1 << 23);
}

bool valid_format(const rrs_kv_cache& c) {
  return c.format == RRS_KV_F16 || has_scales(c);
}

bool aligned(const rrs_kv_cache& c) {
  return is_aligned(c.k) && is_aligned(c.v) && is_aligned(c.table) &&
         (!has_scales(c) || (is_aligned(c.k_scale) && is_aligned(c.v_scale)));
}

rrs::KvView view(const rrs_kv_cache& c) {
  const bool q = has_scales(c);
  return rrs::KvView{static_cast<uint8_t*>(c.k),
                     static_cast<uint8_t*>(c.v),
                     q ? static_cast<uint16_t*>(c.k_scale) : nullptr,
                     q ? static_cast<uint16_t*>(c.v_scale) : nullptr,
                     c.table,
                     c.pages,
                     c.kv_heads,
                     log2_of(c.page_size),
                     c.head_dim,
                     c.sequences,
                     c.max_pages,
                     c.format};
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

rrs_status shared_page(int page, int row, int other) {
  std::fprintf(stderr, "[rrs] RRS_DEBUG: page %d, which the call writes into, is in rows %d and %d\n",
               page, row, other);
  return RRS_ERR_PRECONDITION;
}

// The pages that M tokens are written to are pages of the cache, each of one row: of rows that have a token here, as
// far as their last one's page (entries behind a row's length may hold anything, and the lengths are not known).
rrs_status debug_check_places(const rrs_kv_cache& c, const int32_t* seq, const int32_t* slot,
                              int M, void* stream) {
  std::unique_ptr<int32_t[]> b, s, t;
  if (rrs_status e = debug_fetch_new(&b, seq, (size_t)M, stream)) return e;
  if (rrs_status e = debug_fetch_new(&s, slot, (size_t)M, stream)) return e;
  if (rrs_status e =
          debug_fetch_new(&t, c.table, (size_t)c.sequences * (size_t)c.max_pages, stream))
    return e;
  std::unique_ptr<int64_t[]> written(new (std::nothrow) int64_t[(size_t)M]);  // page, row
  std::unique_ptr<int32_t[]> entries(new (std::nothrow) int32_t[(size_t)c.sequences]());
  if (!written || !entries) return RRS_ERR_HIP;
  size_t count = 0;
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
    written[count++] = (int64_t)p << 32 | bm;
    entries[(size_t)bm] = std::max(entries[(size_t)bm], i + 1);
  }
  int64_t* end = written.get() + count;
  std::sort(written.get(), end);
  for (size_t j = 1; j < count; ++j)
    if (written[j] != written[j - 1] && written[j] >> 32 == written[j - 1] >> 32)
      return shared_page((int)(written[j] >> 32), (int)(written[j - 1] & INT32_MAX),
                         (int)(written[j] & INT32_MAX));
  for (int r = 0; r < c.sequences; ++r)
    for (int i = 0; i < entries[(size_t)r]; ++i) {
      const int32_t p = t[(size_t)r * (size_t)c.max_pages + (size_t)i];
      if (p < 0) continue;
      const int64_t* at = std::lower_bound(written.get(), end, (int64_t)p << 32);
      if (at != end && *at >> 32 == p && (*at & INT32_MAX) != r)
        return shared_page(p, r, (int)(*at & INT32_MAX));
    }
  return RRS_OK;
}

// No page below the lengths is there twice. After debug_check_lengths.
rrs_status debug_check_unshared(const rrs_kv_cache& c, const int32_t* lengths, void* stream) {
  const size_t all = (size_t)c.sequences * (size_t)c.max_pages;
  std::unique_ptr<int32_t[]> n, t;
  if (rrs_status e = debug_fetch_new(&n, lengths, (size_t)c.sequences, stream)) return e;
  if (rrs_status e = debug_fetch_new(&t, c.table, all, stream)) return e;
  std::unique_ptr<int64_t[]> pages(new (std::nothrow) int64_t[all]);  // page, row
  if (!pages) return RRS_ERR_HIP;
  size_t count = 0;
  for (int b = 0; b < c.sequences; ++b)
    for (int i = 0; (int64_t)i * c.page_size < n[(size_t)b]; ++i)
      pages[count++] = (int64_t)t[(size_t)b * (size_t)c.max_pages + (size_t)i] << 32 | b;
  std::sort(pages.get(), pages.get() + count);
  for (size_t j = 1; j < count; ++j)
    if (pages[j] >> 32 == pages[j - 1] >> 32)
      return shared_page((int)(pages[j] >> 32), (int)(pages[j - 1] & INT32_MAX),
                         (int)(pages[j] & INT32_MAX));
  return RRS_OK;
}

// Lengths not negative and within the table, and the pages below them within the pool.
rrs_status debug_check_table(const int32_t* table, int sequences, int max_pages, int page_size,
                             int pages, const int32_t* lengths, void* stream) {
  rrs_kv_cache c{};
  c.table = table;
  c.pages = pages;
  c.page_size = page_size;
  c.sequences = sequences;
  c.max_pages = max_pages;
  return debug_check_lengths(c, lengths, max_pages * page_size, stream);
}

// Pages of the cache; no page is written twice or both read and written.
rrs_status debug_check_pairs(const rrs_kv_cache& c, const int32_t* src, const int32_t* dst, int n,
                             const int32_t* count, void* stream) {
  int32_t pairs = n;
  if (count) {
    if (rrs_status e = debug_fetch(&pairs, count, sizeof(pairs), stream)) return e;
    if (pairs < 0 || pairs > n) {
      std::fprintf(stderr, "[rrs] RRS_DEBUG: count = %d is outside [0, %d]\n", (int)pairs, n);
      return RRS_ERR_PRECONDITION;
    }
  }
  if (pairs == 0) return RRS_OK;
  if (rrs_status e = debug_check_range(src, (size_t)pairs, 0, c.pages, "src", stream)) return e;
  if (rrs_status e = debug_check_range(dst, (size_t)pairs, 0, c.pages, "dst", stream)) return e;
  std::unique_ptr<int32_t[]> s, d;
  if (rrs_status e = debug_fetch_new(&s, src, (size_t)pairs, stream)) return e;
  if (rrs_status e = debug_fetch_new(&d, dst, (size_t)pairs, stream)) return e;
  std::sort(d.get(), d.get() + pairs);
  for (int i = 0; i < pairs; ++i)
    if ((i > 0 && d[(size_t)i] == d[(size_t)i - 1]) ||
        std::binary_search(d.get(), d.get() + pairs, s[(size_t)i])) {
      std::fprintf(stderr, "[rrs] RRS_DEBUG: a page in dst is there twice, or in src\n");
      return RRS_ERR_PRECONDITION;
    }
  return RRS_OK;
}

// Row numbers that do not decrease, within [0, M], of at most max_tokens rows per sequence.
rrs_status debug_check_starts(const int32_t* row_start, int sequences, int M, int max_tokens,
                              void* stream) {
  const size_t count = (size_t)sequences + 1;
  if (rrs_status e = debug_check_range(row_start, count, 0, (int64_t)M + 1, "row_start", stream))
    return e;
  std::unique_ptr<int32_t[]> h;
  if (rrs_status e = debug_fetch_new(&h, row_start, count, stream)) return e;
  for (size_t b = 0; b + 1 < count; ++b)
    if (h[b + 1] < h[b] || h[b + 1] - h[b] > max_tokens) {
      std::fprintf(stderr, "[rrs] RRS_DEBUG: sequence %zu has rows [%d, %d), max_tokens = %d\n", b,
                   (int)h[b], (int)h[b + 1], max_tokens);
      return RRS_ERR_PRECONDITION;
    }
  return RRS_OK;
}

// FP8: no block of 16 slots gets its tokens from two runs of rows.
rrs_status debug_check_runs(const rrs_kv_cache& c, const int32_t* seq, const int32_t* slot, int M,
                            void* stream) {
  std::unique_ptr<int32_t[]> b, s;
  if (rrs_status e = debug_fetch_new(&b, seq, (size_t)M, stream)) return e;
  if (rrs_status e = debug_fetch_new(&s, slot, (size_t)M, stream)) return e;
  std::unique_ptr<int64_t[]> blocks(new (std::nothrow) int64_t[(size_t)M]);
  if (!blocks) return RRS_ERR_HIP;
  size_t count = 0;
  const int per_block = rrs::kSlots8;
  for (size_t m = 0; m < (size_t)M; ++m) {
    if (b[m] < 0 || b[m] >= c.sequences || s[m] < 0 || s[m] >= capacity(c)) continue;
    if (m > 0 && s[m] % per_block != 0 && b[m - 1] == b[m] && s[m - 1] == s[m] - 1) continue;
    blocks[count++] = (int64_t)b[m] << 32 | s[m] / per_block;
  }
  std::sort(blocks.get(), blocks.get() + count);
  for (size_t i = 1; i < count; ++i)
    if (blocks[i] == blocks[i - 1]) {
      std::fprintf(stderr,
                   "[rrs] RRS_DEBUG: tokens of slots %lld.. of sequence %d are not in one run of "
                   "rows\n",
                   (long long)((blocks[i] & 0xFFFFFFFF) * per_block), (int)(blocks[i] >> 32));
      return RRS_ERR_PRECONDITION;
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
  if (!valid_shape(c) || heads < 1 || M < 1 || axes < 1 || axes > 4 || rope_rows < 1 ||
      rotary_dim < 16 || rotary_dim % 16 != 0 || rotary_dim > c.head_dim)
    return RRS_ERR_SHAPE;
  const int64_t width = ((int64_t)heads + 2 * (int64_t)c.kv_heads) * c.head_dim;
  if (width >= ((int64_t)1 << 31) || row_stride < width || row_stride % 8 != 0 ||
      !rrs::append_fits(M, heads, view(c)))
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
    if (c.format == RRS_KV_FP8)
      if (rrs_status s = debug_check_runs(c, seq, slot, M, stream)) return s;
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

size_t rrs_prompt_attention_workspace_bytes(const rrs_kv_cache* cache, int heads, int max_tokens,
                                            int max_length) {
  if (!cache || !valid_shape(*cache) || !valid_format(*cache) || !valid_heads(*cache, heads) ||
      max_tokens < 1 || max_length < 1 || max_length > capacity(*cache) ||
      !rrs::prompt_fits(view(*cache), heads, max_tokens, max_length))
    return 0;
  return rrs::prompt_workspace_bytes(view(*cache), heads, max_tokens, max_length);
}

rrs_status rrs_prompt_attention(const void* Q, int M, int heads, const rrs_kv_cache* cache,
                                const int32_t* row_start, int max_tokens, const int32_t* lengths,
                                int max_length, float scale, const uint8_t* mask, void* out,
                                float* lse, void* workspace, size_t workspace_bytes,
                                void* stream) {
  const bool debug = debug_enabled();
  if (debug) debug_print("prompt_attention", cache);
  if (!Q || !row_start || !lengths || !out || any_null(cache)) return RRS_ERR_NULL;
  const rrs_kv_cache& c = *cache;
  if (!valid_shape(c) || !valid_heads(c, heads) || M < 1 || max_tokens < 1 || max_tokens > M ||
      max_length < 1 || max_length > capacity(c) ||
      !rrs::prompt_fits(view(c), heads, max_tokens, max_length))
    return RRS_ERR_SHAPE;
  if (!valid_format(c) || !std::isfinite(scale)) return RRS_ERR_FLAGS;
  const size_t need = rrs::prompt_workspace_bytes(view(c), heads, max_tokens, max_length);
  if (need > 0 && !workspace) return RRS_ERR_NULL;
  if (!aligned(c) || !is_aligned(Q) || !is_aligned(row_start) || !is_aligned(lengths) ||
      !is_aligned(mask) || !is_aligned(out) || !is_aligned(lse) || !is_aligned(workspace))
    return RRS_ERR_ALIGN;
  if (workspace_bytes < need) return RRS_ERR_WORKSPACE;
  if (rrs_status s = check_device()) return s;
  if (debug) {
    if (rrs_status s = debug_check_starts(row_start, c.sequences, M, max_tokens, stream)) return s;
    int32_t begin = 0, end = 0;  // rows of no sequence may hold anything
    if (rrs_status s = debug_fetch(&begin, row_start, sizeof(begin), stream)) return s;
    if (rrs_status s = debug_fetch(&end, row_start + c.sequences, sizeof(end), stream)) return s;
    const size_t row = (size_t)heads * (size_t)c.head_dim;
    if (rrs_status s =
            debug_check_finite_f16(static_cast<const uint16_t*>(Q) + (size_t)begin * row,
                                   (size_t)(end - begin) * row, "Q", stream))
      return s;
    if (rrs_status s = debug_check_lengths(c, lengths, max_length, stream)) return s;
  }
  const rrs::PromptArgs a{static_cast<const uint16_t*>(Q), M, heads, row_start, max_tokens,
                          lengths, max_length, scale, mask, static_cast<uint16_t*>(out), lse};
  return from_hip(rrs::launch_prompt_attention(a, view(c), workspace,
                                               static_cast<hipStream_t>(stream)));
}

size_t rrs_kv_evict_workspace_bytes(const rrs_kv_cache* cache, int max_length, int budget) {
  if (!cache || !valid_shape(*cache) || !valid_format(*cache) || cache->format == RRS_KV_FP8 ||
      max_length < 1 || max_length > capacity(*cache) || budget < 1 || budget > capacity(*cache) ||
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
  if (!valid_format(c) || c.format == RRS_KV_FP8) return RRS_ERR_FLAGS;
  const size_t need = rrs::evict_workspace_bytes(view(c), max_length, budget);
  if (need > 0 && !workspace) return RRS_ERR_NULL;
  if (!aligned(c) || !is_aligned(workspace) || !is_aligned(lengths) || !is_aligned(weights) || !is_aligned(slot_pos) ||
      !is_aligned(keep_from) || !is_aligned(kept) || !is_aligned(new_lengths) ||
      !is_aligned(weights_out) || !is_aligned(pos_out))
    return RRS_ERR_ALIGN;
  if (workspace_bytes < need) return RRS_ERR_WORKSPACE;
  if (rrs_status s = check_device()) return s;
  if (debug) {
    if (rrs_status s = debug_check_lengths(c, lengths, max_length, stream)) return s;
    if (rrs_status s = debug_check_unshared(c, lengths, stream)) return s;
  }
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

size_t rrs_kv_fork_workspace_bytes(int sequences, int max_pages, int page_size, int pages) {
  return valid_table(sequences, max_pages, page_size, pages)
             ? rrs::fork_workspace_bytes(sequences, pages)
             : 0;
}

rrs_status rrs_kv_fork(const int32_t* table, int sequences, int max_pages, int page_size, int pages,
                       const int32_t* lengths, const int32_t* parent, const int32_t* room,
                       int32_t* table_out, int32_t* lengths_out, int32_t* room_out, int32_t* src,
                       int32_t* dst, int32_t* count, void* workspace, size_t workspace_bytes,
                       void* stream) {
  const bool debug = debug_enabled();
  if (debug)
    std::fprintf(stderr, "[rrs] kv_fork table=%p sequences=%d max_pages=%d page_size=%d pages=%d\n",
                 (const void*)table, sequences, max_pages, page_size, pages);
  if (!table || !lengths || !room || !table_out || !lengths_out || !room_out || !src || !dst ||
      !count || !workspace)
    return RRS_ERR_NULL;
  if (!valid_table(sequences, max_pages, page_size, pages)) return RRS_ERR_SHAPE;
  for (const void* p : {(const void*)table, (const void*)lengths, (const void*)parent,
                        (const void*)room, (const void*)table_out, (const void*)lengths_out,
                        (const void*)room_out, (const void*)src, (const void*)dst,
                        (const void*)count, (const void*)workspace})
    if (!is_aligned(p)) return RRS_ERR_ALIGN;
  if (workspace_bytes < rrs::fork_workspace_bytes(sequences, pages)) return RRS_ERR_WORKSPACE;
  if (rrs_status s = check_device()) return s;
  if (debug)
    if (rrs_status s =
            debug_check_table(table, sequences, max_pages, page_size, pages, lengths, stream))
      return s;
  const rrs::ForkArgs a{table,  sequences, max_pages, log2_of(page_size), pages,
                        lengths, parent,   room,      table_out,          lengths_out,
                        room_out, src,     dst,       count};
  return from_hip(rrs::launch_kv_fork(a, workspace, static_cast<hipStream_t>(stream)));
}

size_t rrs_kv_compact_workspace_bytes(int sequences, int max_pages, int page_size, int pages) {
  return valid_table(sequences, max_pages, page_size, pages) ? rrs::compact_workspace_bytes(pages)
                                                             : 0;
}

rrs_status rrs_kv_compact(const int32_t* table, int sequences, int max_pages, int page_size,
                          int pages, const int32_t* lengths, int32_t* table_out, int32_t* src,
                          int32_t* dst, int32_t* count, void* workspace, size_t workspace_bytes,
                          void* stream) {
  const bool debug = debug_enabled();
  if (debug)
    std::fprintf(stderr,
                 "[rrs] kv_compact table=%p sequences=%d max_pages=%d page_size=%d pages=%d\n",
                 (const void*)table, sequences, max_pages, page_size, pages);
  if (!table || !lengths || !table_out || !src || !dst || !count || !workspace)
    return RRS_ERR_NULL;
  if (!valid_table(sequences, max_pages, page_size, pages)) return RRS_ERR_SHAPE;
  for (const void* p : {(const void*)table, (const void*)lengths, (const void*)table_out,
                        (const void*)src, (const void*)dst, (const void*)count,
                        (const void*)workspace})
    if (!is_aligned(p)) return RRS_ERR_ALIGN;
  if (workspace_bytes < rrs::compact_workspace_bytes(pages)) return RRS_ERR_WORKSPACE;
  if (rrs_status s = check_device()) return s;
  if (debug)
    if (rrs_status s =
            debug_check_table(table, sequences, max_pages, page_size, pages, lengths, stream))
      return s;
  const rrs::CompactArgs a{table,   sequences, max_pages, log2_of(page_size), pages,
                           lengths, table_out, src,       dst,                count};
  return from_hip(rrs::launch_kv_compact(a, workspace, static_cast<hipStream_t>(stream)));
}

rrs_status rrs_kv_copy_pages(const rrs_kv_cache* cache, const int32_t* src, const int32_t* dst,
                             int n, const int32_t* count, void* stream) {
  const bool debug = debug_enabled();
  if (debug) debug_print("kv_copy_pages", cache);
  if (!src || !dst || any_null(cache)) return RRS_ERR_NULL;
  const rrs_kv_cache& c = *cache;
  if (!valid_shape(c) || n < 1) return RRS_ERR_SHAPE;
  if (!valid_format(c)) return RRS_ERR_FLAGS;
  // Bytes of a page are counted in 31 bits.
  if ((int64_t)c.kv_heads * c.page_size * view(c).row_bytes() >= ((int64_t)1 << 31))
    return RRS_ERR_SHAPE;
  if (!aligned(c) || !is_aligned(src) || !is_aligned(dst) || !is_aligned(count))
    return RRS_ERR_ALIGN;
  if (rrs_status s = check_device()) return s;
  if (debug)
    if (rrs_status s = debug_check_pairs(c, src, dst, n, count, stream)) return s;
  return from_hip(rrs::launch_kv_copy_pages(view(c), src, dst, n, count,
                                            static_cast<hipStream_t>(stream)));
}

}  // extern "C"
