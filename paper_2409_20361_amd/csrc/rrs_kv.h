// The paged key/value cache as the kernels see it, and the launchers of its operators
// (arguments validated by rrs_kv_api.cpp).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace rrs {

// include/rrs.h, rrs_kv_cache. Row r of k or v: row_bytes() bytes at r * row_bytes(); its scale at
// r. Products of pages, heads and slots pass 32 bits, so rows are 64-bit numbers.
struct KvView {
  uint8_t* k;
  uint8_t* v;
  uint16_t* k_scale;  // nullptr: float16 values
  uint16_t* v_scale;
  const int32_t* table;
  int pages;
  int heads;
  int log_page;
  int dim;
  int sequences;
  int max_pages;

  __host__ __device__ bool int4() const { return k_scale != nullptr; }
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
bool append_fits(int M);  // ..._fits: the call's launches are within fits_grid
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

}  // namespace rrs
