// Causal attention of every sequence's new tokens over its paged cache. gfx950 only.
//
// For a sequence and a KV head the rows are its new tokens times the query heads that share the
// head: row r is head r % group of token r / group, so all of them read the same keys and values, and a few
// tokens fill a tile as well as many. A workgroup takes 128 or 256 rows, a wave 32, and walks
// along the slots in tiles (64, or 32 at head dim 256) that its waves bring through registers to LDS, as
// float16 whatever the cache holds (INT4 as fp16(q s), FP8 exactly), two tiles in turn. Per block of 32 slots:
//   S^T = K Q^T    mfma 32x32x16, keys from LDS, queries in registers;
//   p = 2^(S - m)  a lane holds one row's p of 16 of 32 slots (lanes l and l + 32 share a row);
//   O^T += V^T P^T values from LDS, transposed (ds_read_b64_tr), in the order of slots that the lane's p
//                  have, so that P goes from one product's result into the other's operand.
// p is rounded to float16 in units that leave a row's largest at 2^12 or more, as in the attention
// of single tokens, and divided by the sum of what it was rounded to, so that the weights of a row add up to 1
// (of slots with equal values the output is that value); sums are float32.
//
// The matrix instructions bound it (4 D flops per row and slot), if the vector instructions (an exponential, a
// product, a sum and a maximum per row and slot, and a part of each tile's way to LDS) run beside them.
// The next block's S^T is computed beside this block's exponentials, and every product's operands are
// read three products ahead, in an issue order that is written out: left to itself the compiler reads an
// operand and waits for it (four prompts of up to 8192 tokens, 32 / 8 heads of 128, FP8: 1147 -> 915 us).
// Addresses of a wave's rows are scalar (its rows lie in one block of 16 slots, one page), and what is rare is
// kept out of the loop, where its constants cost the scalar registers of all (1147 -> 983 us).
// Measured: that batch 905 us (950 TFLOP/s; a float16 product of 8192^3 in the library reaches 1210; without the
// exponentials, or without the way to LDS, 7 and 12 % less), 890 to 960 from card to card; as float16 955 us (900),
// with 32 heads of 64 538 (800), two of up to 8192 with 16 / 8 heads of 256 813 (720: one workgroup per CU, and a
// barrier for every 32 slots); 1024 tokens after 12288 in INT4 with lse 271 us (790). One prompt, 32 / 8 heads of
// 128: 1024 tokens 33 us (260), 2048 64 (540): tiles that see most end long after the others. Small calls are a chain of launch,
// rows, pages and tiles and a second launch: eight of up to 16 tokens after up to 3000, 27 us. A few tokens over a
// long cache leave most of the matrix instructions' columns empty and are bound by HBM:
// they go to the kernel of single tokens (few_tokens).
//
// Where the rows do not fill the card, the slots are cut into pieces, joined by a second kernel in order.
//
// Slots that a row must not see get p = 0. What is there may still not be finite, and 0 times
// it is NaN: slots past the end and under the mask are 0 in LDS; of tiles on the diagonal the
// numbers that are not finite are, too, and are added at the end to the rows that do see them.
#include <algorithm>
#include <type_traits>

#include "rrs_device.h"
#include "rrs_kv.h"

namespace rrs {
namespace {

typedef _Float16 v4h __attribute__((ext_vector_type(4)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4s* lds_v4s;

constexpr int kJoinThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kLift = 12;
constexpr float kRoom = 15.0f;

template <int N>
using Int = std::integral_constant<int, N>;

template <int D, int kFormat, int kWaves>
struct Tile {
  static constexpr int kThreads = 64 * kWaves, kRows = 32 * kWaves;
  static constexpr int kSlots = D == 256 ? 32 : 64;
  static constexpr int kBlocks = kSlots / 32;
  static constexpr int kSteps = D / 16;   // mfma steps of a logit
  static constexpr int kOut = D / 32;     // blocks of output channels
  static constexpr int kBytes = kSlots * D * 2;
  // Loads: kWidth bytes per thread (16, or what gives every wave something), kLanes threads to a row. The
  // rows that a wave loads at a time, at most 16, lie in one block of 16 slots: their page and address are
  // the wave's.
  static constexpr int kRow = kFormat == kCacheInt4 ? D / 2 : kFormat == kCacheFp8 ? D : 2 * D;
  static constexpr int kLanes = kRow / 16 > kThreads / kSlots ? kRow / 16 : kThreads / kSlots;
  static constexpr int kWidth = kRow / kLanes;
  static constexpr int kWaveRows = 64 / kLanes;
  static constexpr int kPasses = kSlots / (kWaves * kWaveRows);
  // 8 float16 numbers each.
  static constexpr int kChunks = kWidth / (kFormat == kCacheInt4 ? 4 : kFormat == kCacheFp8 ? 8 : 16);
  static constexpr int kPerSimd = D == 256 ? 1 : D == 64 ? 3 : 2;

  // Byte of 16-byte chunk c of slot t. Keys are read 16 rows at a time, a chunk of each; values four
  // rows, four neighbouring chunks of each: both then touch all banks.
  static constexpr int kPerLine = 2 * D < 256 ? 256 / (2 * D) : 1;  // rows of a line of banks
  static __device__ __forceinline__ int key_at(int t, int c) {
    const int x = t / kPerLine & (D / 8 < 16 ? D / 8 - 1 : 15);
    return t * (2 * D) + ((c ^ x) << 4);
  }
  static __device__ __forceinline__ int value_at(int t, int c) {
    const int y = t / kPerLine & (D / 8 < 16 ? D / 32 - 1 : 3), x = (y << 2) | (y & 1);
    return t * (2 * D) + ((c ^ x) << 4);
  }
};

struct Plan {
  int group;
  int waves;   // per workgroup
  int rows;    // per workgroup, 32 per wave
  int tiles;   // of rows, per sequence and KV head
  int pieces;  // of the slots, per tile
  int pairs;   // sequences x KV heads
  bool by_xcd;
  float* part;    // pairs x tiles x pieces x rows x D: sums relative to m; nullptr: one piece
  float2* stats;  // the same without D: m (base 2) and the sum of p as float16
  float* sums;    // the sum of p as float32: for lse
};

__device__ __forceinline__ float larger(float a, float b) {
  return __builtin_elementwise_maximum(a, b);
}
// The larger of the two lanes of a row.
__device__ __forceinline__ float row_max(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return larger(__builtin_bit_cast(float, (uint32_t)a[0]),
                __builtin_bit_cast(float, (uint32_t)a[1]));
}

__device__ __forceinline__ float log_sum(float m, float sum) {
  if (sum == 0.0f) return -INFINITY;
  const float e = m + (float)__builtin_amdgcn_frexp_expf(sum);
  return (e + __builtin_amdgcn_logf(__builtin_amdgcn_frexp_mantf(sum))) / kLog2e;
}

// Eight INT4 codes times s, each rounded once: fp16(q s). The largest scale there is, 9360, counts as
// the float16 below it, so that 7 s is finite.
__device__ __forceinline__ v4u eight_int4(uint32_t w, _Float16 s) {
  const v2h s2 = {s, s};
  const v2h off = {(_Float16)1032.0f, (_Float16)1032.0f};
  uint32_t y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {  // codes i and i + 4: exact as 1024 + code + 8
    const uint32_t x = ((w >> (4 * i)) & 0x000F000Fu) ^ 0x64086408u;
    y[i] = __builtin_bit_cast(uint32_t, (__builtin_bit_cast(v2h, x) - off) * s2);
  }
  return v4u{__builtin_amdgcn_perm(y[1], y[0], 0x05040100u),
             __builtin_amdgcn_perm(y[3], y[2], 0x05040100u),
             __builtin_amdgcn_perm(y[1], y[0], 0x07060302u),
             __builtin_amdgcn_perm(y[3], y[2], 0x07060302u)};
}

// Halves of w that are not finite: a bit for each (0 and 16).
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {
  const uint32_t e = w & 0x7C007C00u;
  return ((e + 0x04000400u) >> 15) & 0x00010001u;
}

// The T at byte `at` past an address that is the same for the wave, which stays in scalar registers.
template <typename T>
__device__ __forceinline__ T load_at(const void* base, uint32_t at) {
  typedef const __attribute__((address_space(1))) uint8_t* Global;
  Global p = (Global)base;
  asm("" : "+s"(p), "+v"(at));
  return *(const __attribute__((address_space(1))) T*)(p + at);
}

// Where a tile of rows belongs: new tokens [0, count) of sequence b, the first of which is row `first` of
// Q and sees slots [0, seen).
struct Where {
  int b, hk, tile, piece, count, seen, length;
  size_t first;
};
__device__ __forceinline__ bool find_tile(const PromptArgs& a, const KvView& c, const Plan& plan,
                                          Where* w) {
  // A pair's tiles that see most come first; pairs come in their order, whatever they see. A pair's tiles are on one
  // XCD and share its L2, where that leaves no XCD without work.
  const int per = plan.tiles * plan.pieces;
  int pair, k;
  if (plan.by_xcd) {
    pair = blockIdx.x / (8 * per) * 8 + blockIdx.x % 8;
    if (pair >= plan.pairs) return false;
    k = blockIdx.x / 8 % per;
  } else {
    pair = blockIdx.x % plan.pairs;
    k = blockIdx.x / plan.pairs;
  }
  w->tile = plan.tiles - 1 - k / plan.pieces;
  w->piece = k % plan.pieces;
  w->b = pair / c.heads;
  w->hk = pair % c.heads;
  const int start = min(max(a.row_start[w->b], 0), a.M);
  const int end = min(max(a.row_start[w->b + 1], start), a.M);
  w->first = start;
  w->count = min(end - start, a.max_tokens);
  w->length = min(max(a.lengths[w->b], 0), a.max_length);
  w->seen = w->length - w->count + 1;
  return (long long)w->tile * plan.rows < (long long)w->count * plan.group;
}

// kLse: the logarithm of the sum is asked for, which takes the weights before they are rounded: a second sum (four
// prompts of up to 8192 tokens, 32 / 8 heads of 128, FP8: 905 us without, 939 with it; with the float32 sum alone, by
// which a row of equal values is off by a float16 step, 893).
template <int D, int kFormat, bool kMask, bool kLse, int kWaves>
__global__ void __launch_bounds__((Tile<D, kFormat, kWaves>::kThreads),
                                  (Tile<D, kFormat, kWaves>::kPerSimd))
    prompt_kernel(PromptArgs a, KvView c, Plan plan) {
  using T = Tile<D, kFormat, kWaves>;
  __shared__ __attribute__((aligned(16))) uint8_t keys[2][T::kBytes];
  __shared__ __attribute__((aligned(16))) uint8_t values[2][T::kBytes];
  // Slots with values that are not finite, of the tiles that some rows see in part.
  constexpr int kPartial = T::kRows / T::kSlots + 2;
  __shared__ uint32_t bad_slots[kPartial * T::kBlocks];

  Where at;
  if (!find_tile(a, c, plan, &at)) return;
  const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rows = at.count * plan.group;  // below 2^31: checked by the host
  const int row0 = at.tile * T::kRows;
  const int my_row = min(row0 + 32 * wave + col, rows - 1);
  const int token = my_row / plan.group;
  const int head = at.hk * plan.group + my_row % plan.group;
  const int seen = min(max(at.seen + token, 0), at.length);
  // Slots that all, or any, of the wave's and the workgroup's rows see.
  const auto seen_by = [&](int r) {
    return min(max(at.seen + min(r, rows - 1) / plan.group, 0), at.length);
  };
  const int wave_all = seen_by(row0 + 32 * wave);
  const int all = seen_by(row0), any = seen_by(row0 + T::kRows - 1);
  const bool wave_works = row0 + 32 * wave < rows;

  const int steps = (any + T::kSlots - 1) / T::kSlots;
  const int s0 = (int)((long long)steps * at.piece / plan.pieces);
  const int s1 = (int)((long long)steps * (at.piece + 1) / plan.pieces);

  // Queries: column col, channels 16 i + 8 half ...
  v8h q[T::kSteps];
  const uint16_t* qrow = a.Q + ((at.first + token) * a.heads + head) * D;
#pragma unroll
  for (int i = 0; i < T::kSteps; ++i)
    q[i] = *reinterpret_cast<const v8h*>(qrow + 16 * i + 8 * half);
  // Logits are compared unscaled: a negative scale turns the queries around, and of no scale at
  // all every logit is 0.
  float scale = a.scale * kLog2e;
  if (!(scale > 0.0f)) {
    const _Float16 turn = (_Float16)(scale < 0.0f ? -1.0f : 0.0f);
#pragma unroll
    for (int i = 0; i < T::kSteps; ++i) q[i] *= turn;
    scale = scale < 0.0f ? -scale : 1.0f;
  }

  v16f o[T::kOut] = {};
  float m = -INFINITY;
  float sum = 0.0f;    // of p as it goes into the product with V
  float before = 0.0f;  // of p before it is rounded

  // A wave's part of a tile: in pass p rows kWaveRows (4 p + wave) ... of it, kLanes threads to each.
  const int my_row_of = lane / T::kLanes, my_lane = lane % T::kLanes;
  const uint32_t lane_at = my_row_of * T::kRow + my_lane * T::kWidth;
  typedef uint32_t Piece __attribute__((ext_vector_type(T::kWidth / 4)));
  struct Loaded {
    Piece x[T::kPasses];
    uint16_t scale[T::kPasses];
  };
  Loaded key, val;
  const int last = (at.length - 1) & ~15;
  // ahead: 32 for keys, whose tiles lie a block of 32 slots later.
  const auto group_slot = [&](int step, int p, int ahead) {
    return max(min(step * T::kSlots + ahead + T::kWaveRows * (kWaves * p + wave),
                   last + 16 - T::kWaveRows), 0);
  };
  const int32_t* table = c.table + (size_t)at.b * c.max_pages;
  const int page_slots = 1 << c.log_page;
  const size_t page_rows = (size_t)c.heads << c.log_page, head_rows = (size_t)at.hk << c.log_page;
  const auto load_pages = [&](int step, int ahead, int (&page)[T::kPasses]) {
#pragma unroll
    for (int p = 0; p < T::kPasses; ++p)
      page[p] = load_at<int>(table + (group_slot(step, p, ahead) >> c.log_page), 0);
  };
  const auto load = [&](int step, int ahead, const int (&page)[T::kPasses], const uint8_t* pool,
                        const uint16_t* scales, Loaded& x) {
#pragma unroll
    for (int p = 0; p < T::kPasses; ++p) {
      const int t = group_slot(step, p, ahead) & (page_slots - 1);
      const uint32_t id = __builtin_amdgcn_readfirstlane(page[p]);
      const size_t row = (id < (uint32_t)c.pages ? id : 0) * page_rows + (head_rows + t);
      x.x[p] = load_at<Piece>(pool + row * T::kRow, lane_at);
      if constexpr (kFormat == kCacheFp8) x.scale[p] = load_at<uint16_t>(scales + row / kSlots8, 0);
      if constexpr (kFormat == kCacheInt4)
        x.scale[p] = load_at<uint16_t>(scales + row, 2 * my_row_of);
    }
  };
  // The mask: a lane has its slot of the tile, and of the tile's rows that it brings.
  uint8_t mask[kMask ? T::kPasses : 1], mask_of_tile = 0;
  const uint8_t* mask_row = kMask ? a.mask + (size_t)at.b * c.capacity() : nullptr;
  const auto load_mask = [&](int step) {
    if constexpr (kMask)
#pragma unroll
      for (int p = 0; p < T::kPasses; ++p)
        mask[p] = load_at<uint8_t>(mask_row + group_slot(step, p, 0), my_row_of);
  };
  const auto load_tile_mask = [&](int step) {
    if constexpr (kMask)
      mask_of_tile =
          load_at<uint8_t>(mask_row, min(step * T::kSlots + lane % T::kSlots, at.length - 1));
  };
  // Chunk i (of 8 numbers) of pass p as float16.
  const auto convert = [&](const Loaded& from, int p, int i) -> v4u {
    if constexpr (kFormat == kCacheInt4) {
      _Float16 s = __builtin_bit_cast(_Float16, from.scale[p]);
      s = s == (_Float16)9360.0f ? (_Float16)9352.0f : s;
      return eight_int4(from.x[p][i], s);
    } else if constexpr (kFormat == kCacheFp8) {
      return dequant8_fp8(make_uint2(from.x[p][2 * i], from.x[p][2 * i + 1]),
                          block_unit(from.scale[p]));
    } else {
      return from.x[p];
    }
  };
  constexpr int kParts = T::kPasses * T::kChunks;  // of a thread
  struct Rows {
    v4u x[kParts];
  };
  const auto convert_all = [&](const Loaded& from, Rows& to) {
#pragma unroll
    for (int k = 0; k < kParts; ++k) to.x[k] = convert(from, k / T::kChunks, k % T::kChunks);
  };
  const auto write_keys = [&](int k, v4u x, int buf) {
    const int r = T::kWaveRows * (kWaves * (k / T::kChunks) + wave) + my_row_of;
    *reinterpret_cast<v4u*>(keys[buf] + T::key_at(r, my_lane * T::kChunks + k % T::kChunks)) = x;
  };
  const auto write_values = [&](const Rows& v, int buf) {
#pragma unroll
    for (int k = 0; k < kParts; ++k) {
      const int r = T::kWaveRows * (kWaves * (k / T::kChunks) + wave) + my_row_of;
      *reinterpret_cast<v4u*>(values[buf] +
                              T::value_at(r, my_lane * T::kChunks + k % T::kChunks)) = v.x[k];
    }
  };
  const auto write_all_keys = [&](const Loaded& from, int buf) {
#pragma unroll
    for (int k = 0; k < kParts; ++k)
      write_keys(k, convert(from, k / T::kChunks, k % T::kChunks), buf);
  };
  // Values that not every row of the tile sees: 0 where no row does, and 0 and a mark where a number is not
  // finite, of tiles from first_partial on.
  const int first_partial = all / T::kSlots;
  const auto guarded = [&](int step) { return kMask || step >= first_partial; };
  const auto guard = [&](int step, Rows& v) {
    const bool marks = step >= first_partial;
#pragma unroll
    for (int p = 0; p < T::kPasses; ++p) {
      const int r = T::kWaveRows * (kWaves * p + wave) + my_row_of;
      const bool live = step * T::kSlots + r < at.length && (!kMask || mask[p] != 0);
      uint32_t found = 0;
#pragma unroll
      for (int i = 0; i < T::kChunks; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t w = v.x[p * T::kChunks + i][e];
          const uint32_t bits = marks ? not_finite(w) : 0;
          found |= bits;
          v.x[p * T::kChunks + i][e] = live ? w & ~(bits * 0xFFFFu) : 0u;
        }
      if (live && found)
        atomicOr(&bad_slots[(step - first_partial) * T::kBlocks + r / 32], 1u << (r % 32));
    }
  };
  // Operands: keys of block u of a tile, channels 16 i ...; values of 16 slots 16 w ... of it, channels
  // 32 j ...: lanes 4 r .. 4 r + 3 of 16 name row r, 16 channels of 4 slots; those of half h begin
  // at 4 h and 8 + 4 h.
  const auto key_of = [&](int buf, int u, int i) {
    return *reinterpret_cast<const v8h*>(keys[buf] + T::key_at(32 * u + col, 2 * i + half));
  };
  const int vt = 4 * half + ((lane & 15) >> 2);
  const int vc = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
  const auto value_of = [&](int buf, int u, int w, int j) {
    const uint8_t* lo =
        values[buf] + T::value_at(32 * u + 16 * w + vt, 4 * j + vc) + 8 * (lane & 1);
    const uint8_t* hi =
        values[buf] + T::value_at(32 * u + 16 * w + 8 + vt, 4 * j + vc) + 8 * (lane & 1);
    const v4s x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)lo);
    const v4s y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)hi);
    return __builtin_bit_cast(v8h, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  const auto top_of = [](const v16f& s) {
    float top = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) top = larger(top, s[r]);
    return top;
  };

  // The logits of a block of 32 slots are computed beside the exponentials of the block before it. Step n
  // has its tile of values and the keys 32 slots later in buffer n & 1, step n + 1's in registers.
  if (s0 < s1) {
    int page[T::kPasses];
    Rows v;
    if (threadIdx.x < kPartial * T::kBlocks) bad_slots[threadIdx.x] = 0;
    load_tile_mask(s0);
    load_pages(s0 - 1, 32, page);
    load(s0 - 1, 32, page, c.k, c.k_scale, key);
    load_pages(s0, 0, page);
    load(s0, 0, page, c.v, c.v_scale, val);
    load_mask(s0);
    __syncthreads();
    write_all_keys(key, 1);
    load_pages(s0, 32, page);
    load(s0, 32, page, c.k, c.k_scale, key);
    convert_all(val, v);
    if (guarded(s0)) guard(s0, v);
    write_values(v, 0);
    load_pages(s0 + 1, 0, page);
    load(s0 + 1, 0, page, c.v, c.v_scale, val);
    load_mask(s0 + 1);
    write_all_keys(key, 0);
    load_pages(s0 + 1, 32, page);
    load(s0 + 1, 32, page, c.k, c.k_scale, key);
  }
  __syncthreads();

  float top = -INFINITY;  // of the lane's logits of the block that is next
  // Block u of step `step`: its logits are in l, those of the block after it go to `next`.
  const auto run = [&](int step, auto parity, auto block, v16f& l, v16f& next) {
    constexpr int buf = decltype(parity)::value, u = decltype(block)::value;
    constexpr bool kFirst = u == 0, kLast = u == T::kBlocks - 1;
    const int t0 = step * T::kSlots + 32 * u;
    int key_page[T::kPasses], val_page[T::kPasses];
    if constexpr (kFirst) load_pages(step + 2, 32, key_page);
    if constexpr (kLast) load_pages(step + 2, 0, val_page);
    if (kMask || t0 + 32 > wave_all) {
      uint32_t on = ~0u;
      if constexpr (kMask) on = (uint32_t)(__ballot(mask_of_tile != 0) >> (32 * u));
      const int n = seen - t0;  // slots of the block that the row sees
      on &= n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1;
      on >>= 4 * half;
#pragma unroll
      for (int r = 0; r < 16; ++r) l[r] = on >> (8 * (r / 4) + r % 4) & 1 ? l[r] : -INFINITY;
      top = top_of(l);
    }
    if (__any(top * scale > m + kRoom)) {
      top = row_max(top) * scale;
      const float up = fmaxf(m, top - kLift);
      const float shrink = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - up);
      m = up;
      sum *= shrink;
      if constexpr (kLse) before *= shrink;
#pragma unroll
      for (int j = 0; j < T::kOut; ++j) o[j] *= shrink;
    }
    const float base = m == -INFINITY ? 0.0f : m;
    // The order below is the one that is issued: operands are read kAhead products ahead, and the vector
    // instructions stand between the products, which take 32 cycles each.
    constexpr int kAhead = 3, kProducts = 2 * T::kOut, kEach = 16 / T::kSteps;
    v8h p[2], ks[kAhead], vs[kAhead];
    Rows v;
    float x[16];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) ks[i] = key_of(buf, u, i);
    next = v16f{};
    const auto add = [&](int r) {  // of a pair
      if constexpr (kLse) {
        before += x[r];
        before += x[r + 1];
      }
      const v2h two = {(_Float16)x[r], (_Float16)x[r + 1]};
      p[r / 8][r % 8] = two[0];
      p[r / 8][r % 8 + 1] = two[1];
      sum = __builtin_amdgcn_fdot2(two, v2h{(_Float16)1.0f, (_Float16)1.0f}, sum, false);
    };
#pragma unroll
    for (int i = 0; i < T::kSteps; ++i) {
      next = __builtin_amdgcn_mfma_f32_32x32x16_f16(ks[i % kAhead], q[i], next, 0, 0, 0);
      if (i + kAhead < T::kSteps)
        ks[i % kAhead] = key_of(buf, u, i + kAhead);
      else if (i + kAhead - T::kSteps < kProducts)
        vs[i + kAhead - T::kSteps] = value_of(buf, u, (i + kAhead - T::kSteps) / T::kOut,
                                              (i + kAhead - T::kSteps) % T::kOut);
#pragma unroll
      for (int r = kEach * i; r < kEach * (i + 1); ++r) {
        x[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(l[r], scale, -base));
        if (r % 2 == 1 && r >= 3) add(r - 3);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    add(14);
    top = -INFINITY;
#pragma unroll
    for (int n = 0; n < kProducts; ++n) {
      o[n % T::kOut] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vs[n % kAhead], p[n / T::kOut],
                                                             o[n % T::kOut], 0, 0, 0);
      if (n + kAhead < kProducts)
        vs[n % kAhead] = value_of(buf, u, (n + kAhead) / T::kOut, (n + kAhead) % T::kOut);
      if (n % (kProducts / kParts) == 0) {
        const int k = n / (kProducts / kParts);
        if constexpr (kFirst) write_keys(k, convert(key, k / T::kChunks, k % T::kChunks), buf ^ 1);
        if constexpr (kLast) v.x[k] = convert(val, k / T::kChunks, k % T::kChunks);
      }
      if (n >= kProducts / 2) {  // the new logits are there
#pragma unroll
        for (int r = 32 / kProducts * (n - kProducts / 2);
             r < 32 / kProducts * (n + 1 - kProducts / 2); ++r)
          top = larger(top, next[r]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (kFirst) load(step + 2, 32, key_page, c.k, c.k_scale, key);
    if constexpr (kLast) {
      if (step + 1 < s1 && guarded(step + 1)) guard(step + 1, v);
      write_values(v, buf ^ 1);
      load(step + 2, 0, val_page, c.v, c.v_scale, val);
      load_mask(step + 2);
      load_tile_mask(step + 1);
      __syncthreads();
    }
  };
  if (wave_works) {
    v16f l[2];
    if (s0 < s1) {
      l[0] = v16f{};
#pragma unroll
      for (int i = 0; i < T::kSteps; ++i)
        l[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(key_of(1, T::kBlocks - 1, i), q[i], l[0], 0,
                                                      0, 0);
      top = top_of(l[0]);
    }
    __syncthreads();
    for (int step = s0; step < s1; step += 2) {
      if constexpr (T::kBlocks == 2) {
        run(step, Int<0>(), Int<0>(), l[0], l[1]);
        run(step, Int<0>(), Int<1>(), l[1], l[0]);
        if (step + 1 == s1) break;
        run(step + 1, Int<1>(), Int<0>(), l[0], l[1]);
        run(step + 1, Int<1>(), Int<1>(), l[1], l[0]);
      } else {
        run(step, Int<0>(), Int<0>(), l[0], l[1]);
        if (step + 1 == s1) break;
        run(step + 1, Int<1>(), Int<0>(), l[1], l[0]);
      }
    }
  } else {  // loads for the others
    __syncthreads();
    for (int step = s0; step < s1; ++step) {
      const int buf = (step - s0) & 1;
      int page[T::kPasses];
      Rows x;
      write_all_keys(key, buf ^ 1);
      load_pages(step + 2, 32, page);
      load(step + 2, 32, page, c.k, c.k_scale, key);
      convert_all(val, x);
      if (step + 1 < s1 && guarded(step + 1)) guard(step + 1, x);
      write_values(x, buf ^ 1);
      load_pages(step + 2, 0, page);
      load(step + 2, 0, page, c.v, c.v_scale, val);
      load_mask(step + 2);
      __syncthreads();
    }
  }

  // Values that are not finite, for the rows that see them.
  for (int i = 0; s0 < s1 && i < kPartial * T::kBlocks; ++i)
    for (uint32_t left = bad_slots[i]; left; left &= left - 1) {
      const int t = first_partial * T::kSlots + 32 * i + __builtin_ctz(left);
      if (t >= s1 * T::kSlots) break;
      const size_t row = c.row_of(at.b, at.hk, t);
      float all_of_row = 0.0f;  // INT4: a scale that is not finite
      if constexpr (kFormat == kCacheInt4) all_of_row = half_to_float(c.v_scale[row]) * 0.0f;
#pragma unroll
      for (int j = 0; j < T::kOut; ++j)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          const int d = 32 * j + 2 * r + 4 * half;
          uint2 w = make_uint2(0, 0);
          if constexpr (kFormat == kCacheFp8)
            w.x = *reinterpret_cast<const uint32_t*>(c.v + row * D + d);
          else if constexpr (kFormat == kCacheF16)
            w = *reinterpret_cast<const uint2*>(c.v + (row * D + d) * 2);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float x = all_of_row;
            if constexpr (kFormat == kCacheFp8)
              x = (w.x >> (8 * e) & 127) == 127 ? NAN : 0.0f;
            else if constexpr (kFormat == kCacheF16)
              x = half_to_float((e < 2 ? w.x : w.y) >> (16 * (e & 1)) & 0xFFFFu);
            if (t < seen && !(fabsf(x) < INFINITY)) o[j][r + e] += x;
          }
        }
    }

  const auto both_lanes = [](float x) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto y = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __builtin_bit_cast(float, (uint32_t)y[0]) + __builtin_bit_cast(float, (uint32_t)y[1]);
  };
  sum = both_lanes(sum);
  if constexpr (kLse) before = both_lanes(before);
  if (row0 + 32 * wave + col >= rows) return;
  if (plan.part) {
    const size_t unit =
        (((size_t)(at.b * c.heads + at.hk) * plan.tiles + at.tile) * plan.pieces + at.piece) *
            T::kRows + 32 * wave + col;
    if (half == 0) plan.stats[unit] = make_float2(m, sum);
    if (kLse && half == 0) plan.sums[unit] = before;
    float* out = plan.part + unit * D;
#pragma unroll
    for (int j = 0; j < T::kOut; ++j)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        *reinterpret_cast<v4f*>(out + 32 * j + 2 * r + 4 * half) =
            v4f{o[j][r], o[j][r + 1], o[j][r + 2], o[j][r + 3]};
    return;
  }
  const size_t row = (at.first + token) * a.heads + head;
  const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;  // (NaN where the sum is)
  uint16_t* out = a.out + row * D;
#pragma unroll
  for (int j = 0; j < T::kOut; ++j)
#pragma unroll
    for (int r = 0; r < 16; r += 4)
      *reinterpret_cast<v4h*>(out + 32 * j + 2 * r + 4 * half) =
          v4h{(_Float16)(o[j][r] * inv), (_Float16)(o[j][r + 1] * inv),
              (_Float16)(o[j][r + 2] * inv), (_Float16)(o[j][r + 3] * inv)};
  if (kLse && half == 0) a.lse[row] = log_sum(m, before);
}

// Pieces of a row joined: D / 4 threads to a row, or several groups of so many, which take the row's pieces in
// turn. Grid: pairs x tiles x groups of kRowsAtOnce rows.
template <int D, int kRowsAtOnce>
__global__ void __launch_bounds__(kJoinThreads)
    prompt_join_kernel(PromptArgs a, KvView c, Plan plan) {
  constexpr int kLanes = D / 4, kGroups = kJoinThreads / (kLanes * kRowsAtOnce);
  __shared__ v4f sums[kGroups > 1 ? kJoinThreads : 1];
  __shared__ float2 stats[kGroups > 1 ? kGroups : 1][kRowsAtOnce];
  __shared__ float befores[kGroups > 1 ? kGroups : 1][kRowsAtOnce];
  const int blocks = plan.rows / kRowsAtOnce, unit = blockIdx.x / blocks;
  const int pair = unit / plan.tiles, tile = unit % plan.tiles;
  const int b = pair / c.heads, hk = pair % c.heads;
  const int mine = threadIdx.x / kLanes % kRowsAtOnce, group = threadIdx.x / (kLanes * kRowsAtOnce);
  const int r = blockIdx.x % blocks * kRowsAtOnce + mine;
  const int d = threadIdx.x % kLanes * 4;
  const int start = min(max(a.row_start[b], 0), a.M);
  const int end = min(max(a.row_start[b + 1], start), a.M);
  const long long my_row = (long long)tile * plan.rows + r;
  const bool there = my_row < (long long)min(end - start, a.max_tokens) * plan.group;
  const size_t first = (size_t)unit * plan.pieces * plan.rows + r;
  float top = -INFINITY, total = 0.0f, before = 0.0f;
  v4f acc = {};
  if (there) {
#pragma unroll 4
    for (int i = group; i < plan.pieces; i += kGroups)
      top = fmaxf(top, plan.stats[first + (size_t)i * plan.rows].x);
    const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll 4
    for (int i = group; i < plan.pieces; i += kGroups) {
      const size_t at = first + (size_t)i * plan.rows;
      const float2 st = plan.stats[at];
      const float f = __builtin_amdgcn_exp2f(st.x - base);
      total += st.y * f;
      if (a.lse) before += plan.sums[at] * f;
      acc += *reinterpret_cast<const v4f*>(plan.part + at * D + d) * f;
    }
  }
  if constexpr (kGroups > 1) {
    sums[threadIdx.x] = acc;
    if (d == 0) {
      stats[group][mine] = make_float2(top, total);
      befores[group][mine] = before;
    }
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) top = fmaxf(top, stats[g][mine].x);
    const float base = top == -INFINITY ? 0.0f : top;
    total = before = 0.0f;
    acc = v4f{};
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const float f = __builtin_amdgcn_exp2f(stats[g][mine].x - base);
      total += stats[g][mine].y * f;
      before += befores[g][mine] * f;
      acc += sums[g * kLanes * kRowsAtOnce + threadIdx.x] * f;
    }
  }
  if (!there) return;
  const float inv = total != 0.0f ? 1.0f / total : 0.0f;
  const size_t row = ((size_t)start + my_row / plan.group) * a.heads + hk * plan.group +
                     my_row % plan.group;
  *reinterpret_cast<v4h*>(a.out + row * D + d) =
      v4h{(_Float16)(acc[0] * inv), (_Float16)(acc[1] * inv), (_Float16)(acc[2] * inv),
          (_Float16)(acc[3] * inv)};
  if (d == 0 && a.lse) a.lse[row] = log_sum(top, before);
}

// Rows of a workgroup of the join: up to eight pieces one after the other; more by eight groups of threads (head
// dim 256: four) at once (62 pieces of 5 tokens with 40 heads over 16000 slots: 40 -> 22 us; 5 pieces of 96
// tiles 41 -> 47).
int join_rows(int dim, int pieces) {
  const int all = kJoinThreads / (dim / 4);
  return pieces <= 8 ? all : all > 8 ? all / 8 : 1;
}

// At head dim 128 workgroups of eight waves bring each tile to LDS for twice as many rows, but are half as many.
// They are taken for 1024 rows or more of one sequence behind at least as many cached tokens (32 / 8 heads:
// 1024 after 8000, INT4, 206 -> 187 us, 512 after 8000, FP8, 106 -> 97; 2000 after 2000, 32 / 32 heads, float16,
// 163 -> 144; but 300 after 300, 32 / 32 heads, 26 against 31) and from so many rows of all sequences and KV heads
// times slots on (4096 tokens of one sequence 188 -> 170, up to 8192 of four 937 -> 891); not for less without a past
// (2048 of one 66 against 72, up to 512 of four after up to 4000 120 against 129).
constexpr long long kWide = 5ll << 26;
bool eight_waves(const KvView& c, int heads, int max_tokens, int max_length) {
  if (c.dim != 128) return false;
  const long long rows = (long long)max_tokens * (heads / c.heads);
  if (c.sequences == 1 && rows >= 1024 && max_length / 2 >= max_tokens) return true;
  return rows * c.heads * c.sequences >= kWide / max_length;
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

long long units_of(const Plan& p) { return (long long)p.pairs * p.tiles * p.pieces; }
long long first_grid(const Plan& p) {
  return (p.by_xcd ? ((long long)p.pairs + 7) / 8 * 8 : p.pairs) * p.tiles * p.pieces;
}
long long second_grid(const Plan& p, int dim) {
  return p.pieces > 1 ? (long long)p.pairs * p.tiles * (p.rows / join_rows(dim, p.pieces)) : 0;
}

Plan make_plan(const KvView& c, int heads, int max_tokens, int max_length, void* workspace,
               size_t* bytes) {
  Plan p{};
  p.group = heads / c.heads;
  p.pairs = c.sequences * c.heads;
  // Grids past what a launch may hold do without eight waves, and without the rounding that by_xcd brings.
  for (p.waves = eight_waves(c, heads, max_tokens, max_length) ? 8 : 4;; p.waves = 4) {
    p.rows = 32 * p.waves;
    p.tiles = (int)(((long long)max_tokens * p.group - 1) / p.rows + 1);
    if (p.waves == 4 || fits_grid((long long)p.pairs * p.tiles, 64 * p.waves)) break;
  }
  // Pieces, of four steps at least, where the tiles alone do not fill the card.
  const int slots = c.dim == 256 ? 32 : 64;
  const long long resident = c.dim == 256 || p.waves == 8 ? 256 : c.dim == 64 ? 768 : 512;
  const long long units = (long long)p.pairs * p.tiles;
  const long long most = std::max(1, ((max_length - 1) / slots + 1) / 4);
  p.pieces = (int)std::min(most, std::max(1ll, resident / units));
  // With a workgroup on every CU already, a second one and the join pay from some 20 steps on (32 / 8 heads:
  // 1024 tokens 39 us in two pieces, 34 in one, 32 x up to 30 after up to 700 34 and 28, after up to 2000 51 and 54).
  if (units >= 256 && max_length < 1280) p.pieces = 1;
  p.by_xcd = p.pairs % 8 == 0 || p.pairs >= 64;
  p.by_xcd = p.by_xcd && fits_grid(first_grid(p), 64 * p.waves);
  const size_t rows = p.pieces > 1 ? (size_t)units_of(p) * p.rows : 0;
  const size_t stats = align256(rows * sizeof(float2)), sums = align256(rows * sizeof(float));
  *bytes = stats + sums + rows * c.dim * 4;
  if (workspace && rows) {
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    p.stats = reinterpret_cast<float2*>(ws);
    p.sums = reinterpret_cast<float*>(ws + stats);
    p.part = reinterpret_cast<float*>(ws + stats + sums);
  }
  return p;
}

template <int D>
hipError_t launch(const PromptArgs& a, const KvView& c, const Plan& p, hipStream_t stream) {
  const unsigned grid = (unsigned)first_grid(p);
  const auto run = [&](auto format) {
    constexpr int f = decltype(format)::value;
    const auto go = [&](auto kernel) { kernel<<<grid, 64 * p.waves, 0, stream>>>(a, c, p); };
    const auto by_mask = [&](auto lse, auto waves) {
      constexpr bool kLse = decltype(lse)::value != 0;
      constexpr int kWaves = decltype(waves)::value;
      a.mask ? go(prompt_kernel<D, f, true, kLse, kWaves>)
             : go(prompt_kernel<D, f, false, kLse, kWaves>);
    };
    if constexpr (D == 128)
      if (p.waves == 8) return a.lse ? by_mask(Int<1>(), Int<8>()) : by_mask(Int<0>(), Int<8>());
    a.lse ? by_mask(Int<1>(), Int<4>()) : by_mask(Int<0>(), Int<4>());
  };
  switch (c.format) {
    case kCacheInt4: run(Int<kCacheInt4>()); break;
    case kCacheFp8: run(Int<kCacheFp8>()); break;
    default: run(Int<kCacheF16>());
  }
  if (hipError_t e = hipGetLastError()) return e;
  if (p.pieces > 1) {
    constexpr int kAll = kJoinThreads / (D / 4);
    const unsigned joins = (unsigned)second_grid(p, D);
    if (join_rows(D, p.pieces) == kAll)
      prompt_join_kernel<D, kAll><<<joins, kJoinThreads, 0, stream>>>(a, c, p);
    else
      prompt_join_kernel<D, (kAll > 8 ? kAll / 8 : 1)><<<joins, kJoinThreads, 0, stream>>>(a, c, p);
  }
  return hipGetLastError();
}

}  // namespace

bool prompt_fits(const KvView& c, int heads, int max_tokens, int max_length) {
  // Rows of a sequence and KV head are numbered in 31 bits.
  if ((long long)max_tokens * (heads / c.heads) >= (1ll << 31) - 256) return false;
  if (few_tokens(c, heads, max_tokens, max_length))
    return few_tokens_fits(c, heads, max_tokens, max_length);
  size_t bytes;
  const Plan p = make_plan(c, heads, max_tokens, max_length, nullptr, &bytes);
  return fits_grid(first_grid(p), 64 * p.waves) && fits_grid(second_grid(p, c.dim), kJoinThreads);
}

size_t prompt_workspace_bytes(const KvView& c, int heads, int max_tokens, int max_length) {
  if (few_tokens(c, heads, max_tokens, max_length))
    return few_tokens_workspace_bytes(c, heads, max_tokens, max_length);
  size_t bytes;
  make_plan(c, heads, max_tokens, max_length, nullptr, &bytes);
  return bytes;
}

hipError_t launch_prompt_attention(const PromptArgs& a, const KvView& c, void* workspace,
                                   hipStream_t stream) {
  if (few_tokens(c, a.heads, a.max_tokens, a.max_length))
    return launch_few_tokens(a, c, workspace, stream);
  size_t bytes;
  const Plan p = make_plan(c, a.heads, a.max_tokens, a.max_length, workspace, &bytes);
  switch (c.dim) {
    case 64: return launch<64>(a, c, p, stream);
    case 128: return launch<128>(a, c, p, stream);
    default: return launch<256>(a, c, p, stream);
  }
}

}  // namespace rrs
