// Attention of one new token per sequence over its paged cache. gfx950 only.
//
// For a sequence and a KV head, up to 16 of the query heads that share it are the columns of the
// matrix products. A wave takes tiles of slots (32 float16, 64 INT4), with
// the running maximum m and sum of the softmax of each column kept in its registers:
//   S^T = K Q^T    mfma 16x16x32: a lane reads 16 bytes of its slot's row (lane & 15) as the
//                  operand itself, straight from the cache;
//   p = 2^(S - m)  a lane holds 4 slots (quarter lane >> 4) of each block of 16;
//   O^T += V^T P^T the product sums over slots, so V has to come with the slots of a lane side by
//                  side: its rows go through LDS and are read back transposed
//                  (ds_read_b64_tr). The slots that a quarter of the wave reads are those whose p it holds,
//                  so P goes from the first product's result into the second's operand without leaving the lane.
// All of it is streaming: HBM bounds it (4 D bytes and 4 D flops per slot and query head), so
// loads for the next tile are issued before the current one is computed.
//
// The slots of a sequence are cut into chunks, one workgroup each; its four waves
// take the chunk's tiles in turn and are joined in LDS, chunks of one sequence by a second kernel
// in chunk order (so results repeat bit for bit). That kernel also turns the logits, kept
// in the workspace when they are asked for, into attention weights.
//
// INT4. Codes become float16 exactly (an exponent is or-ed on, an offset taken off). A key's scale
// multiplies its logit; a value's scale multiplies its p before p is rounded to float16.
// So that this product neither overflows nor loses bits to subnormals, m is the maximum
// of S + e, 2^e >= scale: p scale <= 1 and p <= 2^24.
//
// p is rounded to float16 (as the matrix instruction needs it): 2^-11 relative per term, no
// more than the rounding of the output itself. Everything else is float32.
#include "rrs_device.h"
#include "rrs_kv.h"

namespace rrs {
namespace {

typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef int v2i __attribute__((ext_vector_type(2)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4s* lds_v4s;
typedef __attribute__((address_space(3))) v2i* lds_v2i;

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kRows = 16;  // query heads per workgroup: columns of the products
constexpr float kLog2e = 1.4426950408889634f;

// Sizes of a launch, and where its pieces lie in the workspace.
struct Plan {
  int group;       // query heads per KV head
  int row_blocks;  // workgroups per KV head and chunk: ceil(group / kRows)
  int chunk;       // slots per workgroup
  int chunks;      // of the longest sequence
  int ld_logits;   // row stride of the logits: max_length rounded up to whole blocks of 16
  float* part;     // sequences x heads x chunks x dim: sums relative to the chunk's m
  float2* stats;   // sequences x heads x chunks: m (base 2) and the sum of p
  float* logits;   // sequences x heads x ld_logits, base 2; nullptr: not wanted
};

template <int D, bool kInt4>
struct Shape {
  static constexpr int kTile = kInt4 ? 64 : 32;      // slots per wave and step
  static constexpr int kBlocks = kTile / 16;         // of 16 slots
  static constexpr int kRow = kInt4 ? D / 2 : 2 * D; // bytes of a cache row
  static constexpr int kSteps = D / 32;              // mfma steps of a logit
  static constexpr int kOut = D / 16;                // blocks of output channels
  static constexpr int kKey = kRow / 4;              // bytes of a key row per lane
  static constexpr int kLane = kRow / 4;             // bytes of a block of 16 value rows per lane
  static constexpr int kPiece = kLane < 16 ? kLane : 16;
  static constexpr int kPieces = kLane / kPiece;     // loads of them
  static constexpr int kLdO = D + 4;                 // row stride of the waves' sums in LDS
  static constexpr int kValues = kTile * kRow;       // bytes of a wave's value tile
  static constexpr int kSums = kRows * kLdO * 4;
  static constexpr int kLds = kValues > kSums ? kValues : kSums;  // per wave

  // Where 16-byte chunk c of slot t's value row lies in the wave's tile. The chunks of a row are
  // permuted by the slot, so that the rows that one transposed read touches lie in
  // different banks.
  static __device__ __forceinline__ int at(int t, int c) {
    int x;
    if constexpr (kInt4)
      x = D == 64 ? (t >> 2) & 1 : D == 128 ? (t >> 1) & 3 : t & 7;
    else
      x = (D == 64 ? t & 3 : t & 7) << 1;
    return t * kRow + ((c ^ x) << 4);
  }
};

// Two INT4 codes at bits 0-3 and 16-19 (kShift 0) or 4-7 and 20-23 (kShift 4) as float16, exact:
// the code plus 8 (its sign bit flipped) becomes the low mantissa bits of 1024 + it (or
// 1024 + 16 it).
template <int kShift>
__device__ __forceinline__ v2h two_codes(uint32_t w) {
  constexpr uint32_t mask = 0x000F000Fu << kShift;
  constexpr uint32_t flip = (0x00080008u << kShift) | 0x64006400u;
  const v2h h = __builtin_bit_cast(v2h, (w & mask) ^ flip);
  if constexpr (kShift == 0)
    return h - v2h{(_Float16)1032.0f, (_Float16)1032.0f};
  else
    return __builtin_elementwise_fma(h, v2h{(_Float16)0.0625f, (_Float16)0.0625f},
                                     v2h{(_Float16)-72.0f, (_Float16)-72.0f});
}

// Eight packed codes as float16, in the order 0 4 1 5 2 6 3 7.
__device__ __forceinline__ v8h eight_codes(uint32_t w) {
  const v2h a = two_codes<0>(w), b = two_codes<4>(w);
  const v2h c = two_codes<0>(w >> 8), d = two_codes<4>(w >> 8);
  return v8h{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ int code_order(int e) { return (e >> 1) + 4 * (e & 1); }

__device__ __forceinline__ v8h mask_halves(v8h x, const bool (&live)[8]) {
  v4u w = __builtin_bit_cast(v4u, x);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] &= (live[2 * i] ? 0xFFFFu : 0u) | (live[2 * i + 1] ? 0xFFFF0000u : 0u);
  return __builtin_bit_cast(v8h, w);
}

// Grid: units (sequence, KV head) x row blocks x chunks. The row blocks of a unit and chunk read
// the same rows: they are 8 apart, on one XCD, and share its L2.
template <int D, bool kInt4>
__global__ void __launch_bounds__(kThreads)
    attention_kernel(AttentionArgs a, KvView c, Plan plan) {
  using S = Shape<D, kInt4>;
  __shared__ __attribute__((aligned(16))) uint8_t lds[kWaves * S::kLds];
  __shared__ float2 wave_stats[kWaves][kRows];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15;  // a slot of a block of 16, and a query head
  const int quarter = lane >> 4;

  int unit = blockIdx.x, rb = 0;
  if (plan.row_blocks > 1) {
    rb = unit / 8 % plan.row_blocks;
    unit = unit / (8 * plan.row_blocks) * 8 + unit % 8;
  }
  const int chunk = unit % plan.chunks;
  unit /= plan.chunks;
  if (unit >= c.sequences * c.heads) return;  // the last eight may be short
  const int b = unit / c.heads, hk = unit % c.heads;
  const int n = min(a.lengths[b], a.max_length);
  const int begin = chunk * plan.chunk;
  if (begin >= n && chunk > 0) return;
  const int end = min(n, begin + plan.chunk);
  const bool whole = n <= plan.chunk;  // the sequence is this one chunk

  // Queries as the second operand: column col, channels as the keys' lanes hold them.
  const int rows = min(plan.group - rb * kRows, kRows);
  const int head0 = hk * plan.group + rb * kRows;
  const uint16_t* qrow = a.Q + ((size_t)b * a.heads + head0 + min(col, rows - 1)) * D;
  v8h q[S::kSteps];
#pragma unroll
  for (int i = 0; i < S::kSteps; ++i) {
    const v8h x = *reinterpret_cast<const v8h*>(
        qrow + (kInt4 ? (D / 4) * quarter + 8 * i : 32 * i + 8 * quarter));
    if constexpr (kInt4) {
#pragma unroll
      for (int e = 0; e < 8; ++e) q[i][e] = x[code_order(e)];
    } else {
      q[i] = x;
    }
  }
  const float scale = a.scale * kLog2e;

  v4f o[S::kOut] = {};
  float m = -INFINITY, sum = 0.0f;
  uint8_t* tile = lds + wave * S::kLds;

  // Loads of one tile: keys as operands, values as contiguous pieces of their rows, scales of the
  // lane's four slots per block. Rows past the sequence's end read its last row.
  v4u key[S::kBlocks][(S::kKey + 15) / 16];
  v4u val[S::kBlocks][S::kPieces];
  uint2 ks[S::kBlocks], vs[S::kBlocks];
  const auto first_row = [&](int t) {  // of the block of 16 slots at t, and rows from there
    const int p = c.page_of(b, t >> c.log_page);
    return c.page_row(p, hk) + (t & ((1 << c.log_page) - 1));
  };
  const int last = (n - 1) & ~15;
  const auto load_keys = [&](int t0) {
#pragma unroll
    for (int u = 0; u < S::kBlocks; ++u) {
      const int t = min(t0 + 16 * u, last);
      const size_t row = first_row(t);
      const int slot = min(col, n - 1 - t);
      const uint8_t* p = c.k + row * S::kRow + slot * S::kRow + quarter * (kInt4 ? S::kKey : 16);
      if constexpr (S::kKey < 16) {
        const uint2 w = *reinterpret_cast<const uint2*>(p);
        key[u][0] = v4u{w.x, w.y, 0u, 0u};
      } else {
#pragma unroll
        for (int i = 0; i < S::kKey / 16; ++i)
          key[u][i] = *reinterpret_cast<const v4u*>(p + i * (kInt4 ? 16 : 64));
      }
      if constexpr (kInt4) {  // four slots: 8 bytes, inside the page
        ks[u] = *reinterpret_cast<const uint2*>(c.k_scale + row + 4 * quarter);
        vs[u] = *reinterpret_cast<const uint2*>(c.v_scale + row + 4 * quarter);
      }
    }
  };
  constexpr int kPerRow = S::kRow / S::kPiece;   // pieces of a row
  constexpr int kRowsPerLoad = 64 / kPerRow;     // rows that the wave loads at a time
  const auto load_values = [&](int t0) {
#pragma unroll
    for (int u = 0; u < S::kBlocks; ++u) {
      const int t = min(t0 + 16 * u, last);
      const uint8_t* p = c.v + first_row(t) * S::kRow + lane % kPerRow * S::kPiece;
#pragma unroll
      for (int i = 0; i < S::kPieces; ++i) {
        const int slot = min(i * kRowsPerLoad + lane / kPerRow, n - 1 - t);
        if constexpr (S::kPiece < 16) {
          const uint2 w = *reinterpret_cast<const uint2*>(p + slot * S::kRow);
          val[u][i] = v4u{w.x, w.y, 0u, 0u};
        } else {
          val[u][i] = *reinterpret_cast<const v4u*>(p + slot * S::kRow);
        }
      }
    }
  };

  int t0 = begin + wave * S::kTile;
  if (t0 < end) {
    load_keys(t0);
    load_values(t0);
  }
  for (; t0 < end; t0 += kWaves * S::kTile) {
    const int next = t0 + kWaves * S::kTile;
    // Logits, base 2.
    float l[S::kBlocks][4];
    bool live[S::kBlocks][4];
    float top = -INFINITY;
    float vscale[S::kBlocks][4];
#pragma unroll
    for (int u = 0; u < S::kBlocks; ++u) {
      v4f s = {};
#pragma unroll
      for (int i = 0; i < S::kSteps; ++i) {
        v8h k;
        if constexpr (kInt4)
          k = eight_codes(key[u][i / 4][i % 4]);
        else
          k = __builtin_bit_cast(v8h, key[u][i]);
        s = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, q[i], s, 0, 0, 0);
      }
      const int t = t0 + 16 * u + 4 * quarter;
      uint32_t mask = 0x01010101u;
      if (a.mask && t < end)  // four slots of one page: aligned, inside the row
        mask = *reinterpret_cast<const uint32_t*>(a.mask + (size_t)b * c.capacity() + t);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        live[u][r] = t + r < end && ((mask >> (8 * r)) & 255u) != 0;
        float x = s[r] * scale;
        float ref = 0.0f;
        if constexpr (kInt4) {
          const uint32_t wk = r < 2 ? ks[u].x : ks[u].y, wv = r < 2 ? vs[u].x : vs[u].y;
          x *= half_to_float((r & 1) ? wk >> 16 : wk & 0xFFFFu);
          vscale[u][r] = half_to_float((r & 1) ? wv >> 16 : wv & 0xFFFFu);
          ref = vscale[u][r] > 0.0f ? (float)__builtin_amdgcn_frexp_expf(vscale[u][r]) : -24.0f;
        }
        l[u][r] = live[u][r] ? x : -INFINITY;
        top = fmaxf(top, l[u][r] + ref);
      }
      if (plan.logits && t < end && col < rows)
        *reinterpret_cast<float4*>(plan.logits + ((size_t)b * a.heads + head0 + col) *
                                                     plan.ld_logits + t) =
            make_float4(l[u][0], l[u][1], l[u][2], l[u][3]);
    }
    if (next < end) load_keys(next);

    // The running maximum of the column, over the quarters too.
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    if (__any(top > m)) {
      const float up = fmaxf(m, top);
      const float shrink = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - up);
      m = up;
      sum *= shrink;
#pragma unroll
      for (int j = 0; j < S::kOut; ++j) o[j] *= shrink;
    }
    const float base = m == -INFINITY ? 0.0f : m;
    v8h p[S::kBlocks / 2];
#pragma unroll
    for (int u = 0; u < S::kBlocks; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float x = __builtin_amdgcn_exp2f(l[u][r] - base);
        sum += x;
        if constexpr (kInt4) x = live[u][r] ? x * vscale[u][r] : 0.0f;
        p[u / 2][4 * (u & 1) + r] = (_Float16)x;
      }

    // Values through LDS; the wave's own tile, so no barrier.
#pragma unroll
    for (int u = 0; u < S::kBlocks; ++u)
#pragma unroll
      for (int i = 0; i < S::kPieces; ++i) {
        const int t = 16 * u + i * kRowsPerLoad + lane / kPerRow;
        const int piece = lane % kPerRow;
        if constexpr (S::kPiece < 16)
          *reinterpret_cast<uint2*>(tile + S::at(t, piece >> 1) + 8 * (piece & 1)) =
              make_uint2(val[u][i][0], val[u][i][1]);
        else
          *reinterpret_cast<v4u*>(tile + S::at(t, piece)) = val[u][i];
      }
    if (next < end) load_values(next);
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < S::kOut; ++j) {
      if constexpr (kInt4) {
        // Lane i of a quarter names the row whose codes become nibble i of every lane: nibbles
        // x and x + 4 of a dword make one pair, slots 2 x and 2 x + 1 of p's order.
        const int i = col & 7;
        const int s = 2 * (i & 3) + (i >> 2);
        const int t = 32 * (col >> 3) + 16 * (s >> 2) + 4 * quarter + (s & 3);
        const v2i w = __builtin_amdgcn_ds_read_tr4_b64_v2i32(
            (lds_v2i)(tile + S::at(t, j >> 1) + 8 * (j & 1)));
        o[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(eight_codes((uint32_t)w[0]), p[0], o[j], 0,
                                                      0, 0);
        o[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(eight_codes((uint32_t)w[1]),
                                                      p[S::kBlocks / 2 - 1], o[j], 0, 0, 0);
      } else {
        // Lanes 4 r .. 4 r + 3 of a quarter name row r: 16 channels of 4 slots.
        v4s w[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int t = 16 * u + 4 * quarter + (col >> 2);
          w[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (lds_v4s)(tile + S::at(t, 2 * j + ((col & 3) >> 1)) + 8 * (col & 1)));
        }
        v8h v = __builtin_bit_cast(
            v8h, __builtin_shufflevector(w[0], w[1], 0, 1, 2, 3, 4, 5, 6, 7));
        if (a.mask) {  // 0 times what a masked row holds
          const bool alive[8] = {live[0][0], live[0][1], live[0][2], live[0][3],
                                 live[1][0], live[1][1], live[1][2], live[1][3]};
          v = mask_halves(v, alive);
        }
        o[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, p[0], o[j], 0, 0, 0);
      }
    }
    __builtin_amdgcn_wave_barrier();
  }

  // The waves' sums meet in LDS.
  sum += __shfl_xor(sum, 16);
  sum += __shfl_xor(sum, 32);
  float* mine = reinterpret_cast<float*>(tile);
#pragma unroll
  for (int j = 0; j < S::kOut; ++j)
    *reinterpret_cast<v4f*>(mine + col * S::kLdO + 16 * j + 4 * quarter) = o[j];
  if (quarter == 0) wave_stats[wave][col] = make_float2(m, sum);
  __syncthreads();
  for (int i = threadIdx.x; i < rows * D; i += kThreads) {
    const int r = i / D, d = i % D;
    float top = wave_stats[0][r].x;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) top = fmaxf(top, wave_stats[w][r].x);
    float acc = 0.0f, total = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float2 st = wave_stats[w][r];
      const float f = st.x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(st.x - top);
      acc += f * reinterpret_cast<const float*>(lds + w * S::kLds)[r * S::kLdO + d];
      total += f * st.y;
    }
    const size_t bh = (size_t)b * a.heads + head0 + r;
    if (whole) {
      const float x = total > 0.0f ? acc / total : 0.0f;
      a.out[bh * D + d] = __builtin_bit_cast(uint16_t, (_Float16)x);
      if (d == 0 && a.lse)
        a.lse[bh] = total > 0.0f ? (top + __builtin_amdgcn_logf(total)) / kLog2e : -INFINITY;
    } else {
      plan.part[(bh * plan.chunks + chunk) * D + d] = acc;
    }
    if (d == 0 && plan.stats) plan.stats[bh * plan.chunks + chunk] = make_float2(top, total);
  }
}

// The common maximum of a head's chunks and the sum relative to it.
__device__ __forceinline__ float2 join_stats(const float2* stats, int chunks) {
  float top = -INFINITY, total = 0.0f;
  for (int i = 0; i < chunks; ++i) top = fmaxf(top, stats[i].x);
  for (int i = 0; i < chunks; ++i)
    if (stats[i].x > -INFINITY) total += stats[i].y * __builtin_amdgcn_exp2f(stats[i].x - top);
  return make_float2(top, total);
}

// The first sequences x heads workgroups join the chunks of one head each (those of more than one
// chunk); the others turn the logits of 1024 slots of a (sequence, KV head) into weights.
template <int D>
__global__ void __launch_bounds__(kThreads)
    attention_join_kernel(AttentionArgs a, KvView c, Plan plan, int weight_blocks) {
  constexpr int kParts = kThreads / (D / 4);  // chunks read at a time, 4 channels per thread
  __shared__ float4 acc_of[kThreads];
  __shared__ float top_of[kThreads], inv_of[kThreads];
  const int joins = plan.chunks > 1 ? c.sequences * a.heads : 0;
  if ((int)blockIdx.x < joins) {
    const int bh = blockIdx.x, b = bh / a.heads;
    const int n = min(a.lengths[b], a.max_length);
    if (n <= plan.chunk) return;
    const int chunks = (n - 1) / plan.chunk + 1;
    const float2* stats = plan.stats + (size_t)bh * plan.chunks;
    const float2 all = join_stats(stats, chunks);
    const int d4 = threadIdx.x % (D / 4), part = threadIdx.x / (D / 4);
    const float4* src = reinterpret_cast<const float4*>(plan.part + (size_t)bh * plan.chunks * D);
    float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int i = part; i < chunks; i += kParts) {
      const float m = stats[i].x;
      if (m == -INFINITY) continue;
      const float f = __builtin_amdgcn_exp2f(m - all.x);
      const float4 x = src[(size_t)i * (D / 4) + d4];
      acc.x += f * x.x;
      acc.y += f * x.y;
      acc.z += f * x.z;
      acc.w += f * x.w;
    }
    acc_of[threadIdx.x] = acc;
    __syncthreads();
    if (part != 0) return;
    for (int i = 1; i < kParts; ++i) {
      const float4 x = acc_of[i * (D / 4) + d4];
      acc.x += x.x;
      acc.y += x.y;
      acc.z += x.z;
      acc.w += x.w;
    }
    const bool some = all.y > 0.0f;
    const float v[4] = {acc.x, acc.y, acc.z, acc.w};
    uint16_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      h[i] = __builtin_bit_cast(uint16_t, (_Float16)(some ? v[i] / all.y : 0.0f));
    *reinterpret_cast<uint2*>(a.out + (size_t)bh * D + 4 * d4) =
        make_uint2(h[0] | ((uint32_t)h[1] << 16), h[2] | ((uint32_t)h[3] << 16));
    if (d4 == 0 && a.lse)
      a.lse[bh] = some ? (all.x + __builtin_amdgcn_logf(all.y)) / kLog2e : -INFINITY;
    return;
  }
  const int id = blockIdx.x - joins;
  const int unit = id / weight_blocks, b = unit / c.heads, hk = unit % c.heads;
  const int n = min(a.lengths[b], a.max_length);
  const int s0 = id % weight_blocks * (4 * kThreads);
  if (s0 >= n) return;
  const int chunks = (n - 1) / plan.chunk + 1;
  const int s = s0 + 4 * threadIdx.x;
  float4 w = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  for (int g0 = 0; g0 < plan.group; g0 += kThreads) {
    const int heads = min(plan.group - g0, kThreads);
    const size_t bh0 = (size_t)b * a.heads + hk * plan.group + g0;
    __syncthreads();
    if ((int)threadIdx.x < heads) {
      const float2 all = join_stats(plan.stats + (bh0 + threadIdx.x) * plan.chunks, chunks);
      top_of[threadIdx.x] = all.x;
      inv_of[threadIdx.x] = all.y > 0.0f ? 1.0f / all.y : 0.0f;
    }
    __syncthreads();
    if (s < n)
      for (int g = 0; g < heads; ++g) {
        if (inv_of[g] == 0.0f) continue;
        const float4 l =
            *reinterpret_cast<const float4*>(plan.logits + (bh0 + g) * plan.ld_logits + s);
        const float t = top_of[g], f = inv_of[g];
        w.x += __builtin_amdgcn_exp2f(l.x - t) * f;
        w.y += __builtin_amdgcn_exp2f(l.y - t) * f;
        w.z += __builtin_amdgcn_exp2f(l.z - t) * f;
        w.w += __builtin_amdgcn_exp2f(l.w - t) * f;
      }
  }
  if (s >= n) return;
  float* out = a.weights + (size_t)unit * c.capacity() + s;
  const float add[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (s + i < n) out[i] += add[i];
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Chunks: enough workgroups for the card (256 compute units, three workgroups each) a few times
// over, since sequences are shorter than the longest; at least two tiles per wave.
Plan make_plan(const KvView& c, int heads, int max_length, bool with_weights, void* workspace,
               size_t* bytes) {
  Plan p{};
  p.group = heads / c.heads;
  p.row_blocks = (p.group + kRows - 1) / kRows;
  const long long units = (long long)c.sequences * c.heads * p.row_blocks;
  const int step = kWaves * (c.int4() ? 64 : 32);
  long long chunk = ((long long)max_length * units / 1536 + step - 1) / step * step;
  if (chunk < 2 * step) chunk = 2 * step;
  if (chunk > max_length) chunk = ((long long)max_length + step - 1) / step * step;
  p.chunk = (int)(chunk < (1 << 30) ? chunk : 1 << 30);
  p.chunks = (max_length - 1) / p.chunk + 1;
  p.ld_logits = (max_length + 15) & ~15;
  const size_t bh = (size_t)c.sequences * heads;
  const size_t stats = p.chunks > 1 || with_weights ? align256(bh * p.chunks * 8) : 0;
  const size_t part = p.chunks > 1 ? align256(bh * p.chunks * c.dim * 4) : 0;
  const size_t logits = with_weights ? align256(bh * (size_t)p.ld_logits * 4) : 0;
  *bytes = stats + part + logits;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  if (ws) {
    if (stats) p.stats = reinterpret_cast<float2*>(ws);
    if (part) p.part = reinterpret_cast<float*>(ws + stats);
    if (logits) p.logits = reinterpret_cast<float*>(ws + stats + part);
  }
  return p;
}

template <int D>
hipError_t launch(const AttentionArgs& a, const KvView& c, const Plan& p, hipStream_t stream) {
  const long long units = (long long)c.sequences * c.heads * p.chunks;
  const long long grid = p.row_blocks == 1 ? units : (units + 7) / 8 * 8 * p.row_blocks;
  if (grid >= (1ll << 31)) return hipErrorInvalidValue;
  if (c.int4())
    attention_kernel<D, true><<<(unsigned)grid, kThreads, 0, stream>>>(a, c, p);
  else
    attention_kernel<D, false><<<(unsigned)grid, kThreads, 0, stream>>>(a, c, p);
  if (hipError_t e = hipGetLastError()) return e;
  const int blocks = p.logits ? (a.max_length - 1) / (4 * kThreads) + 1 : 0;
  const long long joins = (p.chunks > 1 ? (long long)c.sequences * a.heads : 0) +
                          (long long)blocks * c.sequences * c.heads;
  if (joins >= (1ll << 31)) return hipErrorInvalidValue;
  if (joins > 0)
    attention_join_kernel<D><<<(unsigned)joins, kThreads, 0, stream>>>(a, c, p, blocks);
  return hipGetLastError();
}

}  // namespace

size_t attention_workspace_bytes(const KvView& c, int heads, int max_length, bool with_weights) {
  size_t bytes;
  make_plan(c, heads, max_length, with_weights, nullptr, &bytes);
  return bytes;
}

hipError_t launch_paged_attention(const AttentionArgs& a, const KvView& c, hipStream_t stream) {
  size_t bytes;
  const Plan p = make_plan(c, a.heads, a.max_length, a.weights != nullptr, a.workspace, &bytes);
  switch (c.dim) {
    case 64: return launch<64>(a, c, p, stream);
    case 128: return launch<128>(a, c, p, stream);
    default: return launch<256>(a, c, p, stream);
  }
}

}  // namespace rrs
