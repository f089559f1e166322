// The paged key/value cache as the kernels see it, and the launchers of its operators
// (arguments validated by rrs_kv_api.cpp).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace rrs {

// include/rrs.h, RRS_KV_*.
constexpr int kCacheF16 = 0, kCacheInt4 = 1, kCacheFp8 = 8;
// FP8: slots that share a scale, and its smallest and largest exponent.
constexpr int kSlots8 = 16, kLowest8 = -15, kHighest8 = 8;

// include/rrs.h, rrs_kv_cache. Row r of k or v: row_bytes() bytes at r * row_bytes(); its scale at
// r (FP8: r / 16, of its block). Products of pages, heads and slots pass 32 bits, so rows are 64-bit numbers.
struct KvView {
  uint8_t* k;
  uint8_t* v;
  uint16_t* k_scale;  // nullptr for float16 values
  uint16_t* v_scale;
  const int32_t* table;
  int pages;
  int heads;
  int log_page;
  int dim;
  int sequences;
  int max_pages;
  int format;

  __host__ __device__ bool int4() const { return format == kCacheInt4; }
  __host__ __device__ int row_bytes() const {
    return format == kCacheInt4 ? dim / 2 : format == kCacheFp8 ? dim : 2 * dim;
  }
  __host__ __device__ int capacity() const { return max_pages << log_page; }
  // First row of (page, head).
  __device__ size_t page_row(int page, int head) const {
    return ((size_t)(uint32_t)page * (uint32_t)heads + (uint32_t)head) << log_page;
  }
  // Page of table entry i of sequence b; one that does not exist reads as page 0.
  __device__ int page_of(int b, int i) const {
    const int p = table[(size_t)b * max_pages + i];
    return (uint32_t)p < (uint32_t)pages ? p : 0;
  }
  __device__ size_t row_of(int b, int head, int slot) const {
    return page_row(page_of(b, slot >> log_page), head) + (slot & ((1 << log_page) - 1));
  }
  // For rows that are written: false where the table names no page of the cache.
  __device__ bool find_row(int b, int head, int slot, size_t* row) const {
    const int p = table[(size_t)b * max_pages + (slot >> log_page)];
    *row = page_row(p, head) + (slot & ((1 << log_page) - 1));
    return (uint32_t)p < (uint32_t)pages;
  }
};

// A grid of so many workgroups can be launched (the runtime counts threads in 32 bits).
inline bool fits_grid(long long workgroups, int threads) {
  return workgroups * threads < (1ll << 32);
}

struct RopeArgs {
  const uint16_t* qkv;
  int64_t row_stride;
  int M;
  int heads;
  const int32_t* positions;
  int axes;
  int bound[4];  // end of axis a's frequencies (the last: rotary_dim / 2)
  const float* rope;
  int rope_rows;
  int rotary_dim;
  bool interleaved;
  const int32_t* seq;
  const int32_t* slot;
  uint16_t* Q;
  float* weights;
  int32_t* slot_pos;
};
bool append_fits(int M, int heads, const KvView& c);  // ..._fits: the call's launches are within fits_grid
hipError_t launch_rope_kv_append(const RopeArgs& a, const KvView& c, hipStream_t stream);

bool read_fits(const KvView& c, int max_length);
hipError_t launch_kv_read(const KvView& c, const int32_t* lengths, int max_length, uint16_t* K,
                          uint16_t* V, hipStream_t stream);

struct AttentionArgs {
  const uint16_t* Q;
  int heads;
  const int32_t* lengths;
  int max_length;
  float scale;
  const uint8_t* mask;  // or nullptr
  float* weights;       // or nullptr
  uint16_t* out;
  float* lse;  // or nullptr
  void* workspace;
};
bool attention_fits(const KvView& c, int heads, int max_length, bool with_weights);
size_t attention_workspace_bytes(const KvView& c, int heads, int max_length, bool with_weights);
hipError_t launch_paged_attention(const AttentionArgs& a, const KvView& c, hipStream_t stream);

struct PromptArgs {
  const uint16_t* Q;
  int M;
  int heads;
  const int32_t* row_start;
  int max_tokens;
  const int32_t* lengths;
  int max_length;
  float scale;
  const uint8_t* mask;  // or nullptr
  uint16_t* out;
  float* lse;  // or nullptr
};
bool prompt_fits(const KvView& c, int heads, int max_tokens, int max_length);
size_t prompt_workspace_bytes(const KvView& c, int heads, int max_tokens, int max_length);
hipError_t launch_prompt_attention(const PromptArgs& a, const KvView& c, void* workspace,
                                   hipStream_t stream);

// The same for few tokens, by the attention of single ones.
bool few_tokens(const KvView& c, int heads, int max_tokens, int max_length);
bool few_tokens_fits(const KvView& c, int heads, int max_tokens, int max_length);
size_t few_tokens_workspace_bytes(const KvView& c, int heads, int max_tokens, int max_length);
hipError_t launch_few_tokens(const PromptArgs& a, const KvView& c, void* workspace,
                             hipStream_t stream);

struct EvictArgs {
  const int32_t* lengths;
  int max_length;
  const float* weights;
  const int32_t* slot_pos;
  const int32_t* keep_from;
  int budget;
  int32_t* kept;
  int32_t* new_lengths;
  float* weights_out;
  int32_t* pos_out;
};
bool evict_fits(const KvView& c, int max_length, int budget);
size_t evict_workspace_bytes(const KvView& c, int max_length, int budget);
hipError_t launch_kv_evict(const EvictArgs& a, const KvView& c, void* workspace,
                           hipStream_t stream);

struct ForkArgs {
  const int32_t* table;
  int sequences;
  int max_pages;
  int log_page;
  int pages;
  const int32_t* lengths;
  const int32_t* parent;  // or nullptr
  const int32_t* room;
  int32_t* table_out;
  int32_t* lengths_out;
  int32_t* room_out;
  int32_t* src;
  int32_t* dst;
  int32_t* count;
};
int most_pages();  // of the planners
size_t fork_workspace_bytes(int sequences, int pages);
hipError_t launch_kv_fork(const ForkArgs& a, void* workspace, hipStream_t stream);

struct CompactArgs {
  const int32_t* table;
  int sequences;
  int max_pages;
  int log_page;
  int pages;
  const int32_t* lengths;
  int32_t* table_out;
  int32_t* src;
  int32_t* dst;
  int32_t* count;
};
size_t compact_workspace_bytes(int pages);
hipError_t launch_kv_compact(const CompactArgs& a, void* workspace, hipStream_t stream);

hipError_t launch_kv_copy_pages(const KvView& c, const int32_t* src, const int32_t* dst, int n,
                                const int32_t* count, hipStream_t stream);

// Inclusive prefix sums over the wave; the last lane holds the total.
__device__ __forceinline__ int wave_prefix(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);  // from 1 lane below in the row
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);  // 2
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);  // 4
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);  // 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);  // rows 0, 2 into 1, 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);  // the lower half's total
  return x;
}
__device__ __forceinline__ int wave_total(int x) {
  return __builtin_amdgcn_readlane(wave_prefix(x), 63);
}

// 8 packed codes (low nibble first) as float16 of q s, s a float16 scale.
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
__device__ __forceinline__ v4u dequant8(uint32_t codes, float s) {
  v4u w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const _Float16 lo = (_Float16)((float)((int)(codes << (28 - 8 * i)) >> 28) * s);
    const _Float16 hi = (_Float16)((float)((int)(codes << (24 - 8 * i)) >> 28) * s);
    w[i] = (uint32_t)__builtin_bit_cast(uint16_t, lo) |
           ((uint32_t)__builtin_bit_cast(uint16_t, hi) << 16);
  }
  return w;
}

// An FP8 block's scale: 2 to its exponent, a finite number whatever the float16 is (of a block that was
// never written, all of whose slots take no part).
__device__ __forceinline__ float block_unit(uint32_t half) {
  return __builtin_bit_cast(float, ((half & 0x7C00u) << 13) + ((127u - 15u) << 23));
}

// Two e4m3 codes, bytes 2 kHalf and 2 kHalf + 1 of w, as float16 in units of a power of two (of which the
// instruction takes the exponent). Exact from 2^-15 on: a code's smallest step is 2^-9, float16's 2^-24.
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
template <int kHalf>
__device__ __forceinline__ v2h two_fp8(uint32_t w, float unit) {
  return __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, unit, kHalf != 0);
}
__device__ __forceinline__ v4u dequant8_fp8(uint2 w, float unit) {
  return v4u{__builtin_bit_cast(uint32_t, two_fp8<0>(w.x, unit)),
             __builtin_bit_cast(uint32_t, two_fp8<1>(w.x, unit)),
             __builtin_bit_cast(uint32_t, two_fp8<0>(w.y, unit)),
             __builtin_bit_cast(uint32_t, two_fp8<1>(w.y, unit))};
}

}  // namespace rrs
