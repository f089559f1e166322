// Rotary positions and cache append in one pass over the QKV projection's output, and the
// cached values read back as float16. gfx950 only.
//
// Append. Row m of qkv is [heads queries | kv_heads keys | kv_heads values] of D channels. A
// workgroup takes one token; D / 16 lanes share a head's row, each with 16 of its channels: the
// 8 + 8 that make up eight rotary pairs (j and j + F, or 16 neighbours when interleaved), so the
// rotation needs no other lane. A lane's channels are the same in every head: its eight
// cosines and sines are loaded once per token and used for all heads. Bound by HBM: every
// byte of qkv is read once, 16 bytes per lane, and every result written once. Measured: 8192 tokens
// of 32 + 32 + 32 heads of 128, float16, 78.0 us (5.2 TB/s read and written; a copy of 400 MiB reaches
// 5.4); 1117 tokens of 32 + 8 + 8 into INT4, 9.0 to 10.4 us, one token 2.3 to 2.7 us (latency).
//
// Into FP8 a block of 16 slots shares a scale, so a block's new tokens belong to one wave, with the rows that they find
// there (rope_kv_append8_kernel). The same bytes bound it: 6113 tokens of 32 + 32 + 32 heads of 128 59 us (4.3
// TB/s read and written), one token 4.0 to 4.6 us (one more chain: the rows of its run, the block's scale).
//
// Read-back. One row of K and V per D / 8 lanes; bound by the writes, which go past the caches
// (134 MB from 2048 slots of 4 x 32 INT4 heads: 25.7 us, 40.8 with ordinary stores;
// 41 with both where inputs and outputs in use outgrow the last-level cache).
#include <algorithm>

#include "rrs_device.h"
#include "rrs_kv.h"

namespace rrs {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ uint4 pack_halves(const float (&v)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const _Float16 lo = (_Float16)v[2 * i], hi = (_Float16)v[2 * i + 1];
    w[i] = (uint32_t)__builtin_bit_cast(uint16_t, lo) |
           ((uint32_t)__builtin_bit_cast(uint16_t, hi) << 16);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ void unpack_halves(const uint4& w, float (&v)[8]) {
  const uint32_t d[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = half_to_float(d[i] & 0xFFFFu);
    v[2 * i + 1] = half_to_float(d[i] >> 16);
  }
}

// NaN if one of them is: it has to reach the row's scale.
__device__ __forceinline__ float larger(float a, float b) {
  return __builtin_elementwise_maximum(a, b);
}

__device__ __forceinline__ float max_abs(const float (&v)[8]) {
  float m = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = larger(m, fabsf(v[e]));
  return m;
}

// q = clamp(rint(x / s), -7, 7), eight codes of 4 bits. The division is the IEEE one: s has 11
// bits, so no quotient is close to a half integer without being one, and the code is
// that of the real quotient. Codes of 0 under a scale that is not finite: the row reads as NaN.
__device__ __forceinline__ uint32_t codes8(const float (&v)[8], float s) {
  if (!(s > 0.0f && s < INFINITY)) return 0u;
  uint32_t w = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float q = fminf(fmaxf(rintf(__fdiv_rn(v[e], s)), -7.0f), 7.0f);
    w |= ((uint32_t)(int)q & 15u) << (4 * e);
  }
  return w;
}

// Cosines and sines of frequencies [8 i, 8 i + 8) at token m's positions.
__device__ __forceinline__ void angles(const RopeArgs& a, int m, int i, float (&cs)[8],
                                       float (&sn)[8]) {
  const int F = a.rotary_dim / 2;
  int p[4];
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    p[x] = x < a.axes ? a.positions[(size_t)m * a.axes + x] : 0;
    p[x] = min(max(p[x], 0), a.rope_rows - 1);
  }
  const auto axis = [&](int j) {
    return (j >= a.bound[0]) + (j >= a.bound[1]) + (j >= a.bound[2]);
  };
  const auto position = [&](int j) {
    const int x = axis(j);
    return x == 0 ? p[0] : x == 1 ? p[1] : x == 2 ? p[2] : p[3];
  };
  const int j0 = 8 * i;
  if (axis(j0) == axis(j0 + 7)) {  // of one axis: neighbours in its row
    const float4* row =
        reinterpret_cast<const float4*>(a.rope + (size_t)position(j0) * a.rotary_dim + j0);
    const float4 c0 = row[0], c1 = row[1], s0 = row[F / 4], s1 = row[F / 4 + 1];
    const float cc[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w};
    const float ss[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      cs[e] = cc[e];
      sn[e] = ss[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float* row = a.rope + (size_t)position(j0 + e) * a.rotary_dim;
      cs[e] = row[j0 + e];
      sn[e] = row[F + j0 + e];
    }
  }
}

// Pairs (x, y) turned: (x c - y s, y c + x s).
__device__ __forceinline__ void turn(bool interleaved, const float (&cs)[8], const float (&sn)[8],
                                     float (&x)[8], float (&y)[8]) {
  if (interleaved) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float x0 = x[2 * e], x1 = x[2 * e + 1], y0 = y[2 * e], y1 = y[2 * e + 1];
      x[2 * e] = x0 * cs[e] - x1 * sn[e];
      x[2 * e + 1] = x1 * cs[e] + x0 * sn[e];
      y[2 * e] = y0 * cs[e + 4] - y1 * sn[e + 4];
      y[2 * e + 1] = y1 * cs[e + 4] + y0 * sn[e + 4];
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x0 = x[e], y0 = y[e];
      x[e] = x0 * cs[e] - y0 * sn[e];
      y[e] = y0 * cs[e] + x0 * sn[e];
    }
  }
}

template <int D, bool kInt4>
__global__ void __launch_bounds__(kThreads) rope_kv_append_kernel(RopeArgs a, KvView c) {
  constexpr int kLanes = D / 16;             // lanes per head row
  constexpr int kHeads = kThreads / kLanes;  // head rows per pass
  const int m = blockIdx.x;
  const int i = threadIdx.x % kLanes;
  const int F = a.rotary_dim / 2;
  const bool turns = 8 * i < F;

  // Channels of this lane: [o0, o0 + 8) and [o1, o1 + 8).
  int o0, o1;
  if (!turns || a.interleaved) {
    o0 = 16 * i;
    o1 = o0 + 8;
  } else {
    o0 = 8 * i;
    o1 = F + 8 * i;
  }
  // The first row is on its way while positions, cosines and the token's place are looked up.
  const int total = a.heads + 2 * c.heads;
  const uint16_t* src = a.qkv + (size_t)m * a.row_stride;
  const int step = kHeads * gridDim.y;
  int h = blockIdx.y * kHeads + threadIdx.x / kLanes;
  uint4 x_next = make_uint4(0, 0, 0, 0), y_next = x_next;
  const auto load = [&](int head) {
    if (head >= total) return;
    x_next = *reinterpret_cast<const uint4*>(src + (size_t)head * D + o0);
    y_next = *reinterpret_cast<const uint4*>(src + (size_t)head * D + o1);
  };
  load(h);

  float cs[8], sn[8];
  if (turns) angles(a, m, i, cs, sn);

  const int seq = a.seq[m], slot = a.slot[m];
  bool stored = seq >= 0 && seq < c.sequences && slot >= 0 && slot < c.capacity();
  size_t row0 = 0;  // the token's row in head 0's page
  if (stored) stored = c.find_row(seq, 0, slot, &row0);
  if (stored && blockIdx.y == 0)
    for (int h = threadIdx.x; h < c.heads; h += kThreads) {
      const size_t at = ((size_t)seq * c.heads + h) * c.capacity() + slot;
      if (a.weights) a.weights[at] = 0.0f;
      if (a.slot_pos) a.slot_pos[at] = a.positions[(size_t)m * a.axes];
    }

  for (; h < total; h += step) {
    const bool query = h < a.heads;
    const bool value = h >= a.heads + c.heads;
    uint4 xo = x_next, yo = y_next;
    load(h + step);
    if (!query && !stored) continue;
    float x[8], y[8];
    unpack_halves(xo, x);
    unpack_halves(yo, y);
    if (turns && !value) {
      turn(a.interleaved, cs, sn, x, y);
      xo = pack_halves(x);
      yo = pack_halves(y);
    }
    if (query) {
      uint16_t* q = a.Q + ((size_t)m * a.heads + h) * D;
      *reinterpret_cast<uint4*>(q + o0) = xo;
      *reinterpret_cast<uint4*>(q + o1) = yo;
      continue;
    }
    const int hk = h - a.heads - (value ? c.heads : 0);
    const size_t row = row0 + ((size_t)hk << c.log_page);
    if constexpr (!kInt4) {
      uint16_t* dst = reinterpret_cast<uint16_t*>(value ? c.v : c.k) + row * D;
      *reinterpret_cast<uint4*>(dst + o0) = xo;
      *reinterpret_cast<uint4*>(dst + o1) = yo;
    } else {
      // Quantized from the float16 values that a float16 cache would hold.
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[e] = (float)(_Float16)x[e];
        y[e] = (float)(_Float16)y[e];
      }
      float top = larger(max_abs(x), max_abs(y));
#pragma unroll
      for (int d = 1; d < kLanes; d <<= 1) top = larger(top, __shfl_xor(top, d));
      const _Float16 scale = (_Float16)__fdiv_rn(top, 7.0f);
      uint8_t* dst = (value ? c.v : c.k) + row * (D / 2);
      *reinterpret_cast<uint32_t*>(dst + o0 / 2) = codes8(x, (float)scale);
      *reinterpret_cast<uint32_t*>(dst + o1 / 2) = codes8(y, (float)scale);
      if (i == 0) (value ? c.v_scale : c.k_scale)[row] = __builtin_bit_cast(uint16_t, scale);
    }
  }
}

// Where a lane's 16 channels of a row lie: [o0, o0 + 8) and [o1, o1 + 8), whose pairs are the
// frequencies [8 i, 8 i + 8) if the lane has any.
struct Channels {
  int o0, o1;
  bool turns;
  __device__ __forceinline__ Channels(const RopeArgs& a, int i) {
    const int F = a.rotary_dim / 2;
    turns = 8 * i < F;
    const bool apart = turns && !a.interleaved;
    o0 = apart ? 8 * i : 16 * i;
    o1 = apart ? F + 8 * i : o0 + 8;
  }
};

// Largest |x| of the values that are finite.
__device__ __forceinline__ float max_finite(const float (&v)[8]) {
  float m = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(v[e]) < INFINITY ? fabsf(v[e]) : 0.0f);
  return m;
}

// The exponent of the smallest scale, 2^-15 or more, that brings `top` to 448 = 0.875 2^9 at most.
__device__ __forceinline__ int scale_exponent(float top) {
  if (top == 0.0f) return kLowest8;
  const int e = __builtin_amdgcn_frexp_expf(top) - 9;
  return max(__builtin_amdgcn_frexp_mantf(top) > 0.875f ? e + 1 : e, kLowest8);
}

// x 2^-e as four e4m3 codes, to nearest; at 2^8 up to 240, so that code times scale stays a float16
// (off by 2^-4 relative, as any rounding); NaN where x is not finite.
__device__ __forceinline__ uint32_t codes4(const float* x, float inv, float most) {
  float v[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[e] = fminf(fmaxf(x[e] * inv, -most), most);
    if (!(fabsf(x[e]) < INFINITY)) v[e] = __builtin_nanf("");
  }
  const int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], w, true);
}

// Four codes in a scale that is 1 / shrink times as large.
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float shrink, float most) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
  const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  const float x[4] = {lo[0], lo[1], hi[0], hi[1]};
  return codes4(x, shrink, most);
}

// FP8. The first workgroups write keys and values: blocks of 16 slots, whose tokens lie in a run of
// rows (one sequence, one slot after the other). `parts` workgroups look through the same 16 rows for those that
// begin a run, and share the runs' pairs of heads: a
// wave takes the keys, or the values, of a head of a run: 64 lanes hold 16 rows, so
// the block's largest value, its scale and its codes need nothing from another wave. Rows of the
// block that are not in the run keep their codes, or get new ones where the scale has grown: by a
// power of two, so that only codes below 2^-6 are rounded again. The other
// workgroups rotate queries, as above.
template <int D>
__global__ void __launch_bounds__(kThreads)
    rope_kv_append8_kernel(RopeArgs a, KvView c, int parts, int block_groups, int query_parts) {
  constexpr int kLanes = D / 16;             // lanes per head row
  constexpr int kHeads = kThreads / kLanes;  // head rows per pass
  constexpr int kRowsAtOnce = 64 / kLanes;   // rows of a block per wave and pass
  constexpr int kPasses = kSlots8 / kRowsAtOnce;
  const int lane = threadIdx.x & 63;
  const int i = threadIdx.x % kLanes;
  const Channels ch(a, i);

  if ((int)blockIdx.x >= block_groups) {
    const int id = blockIdx.x - block_groups;
    const int m = id / query_parts, part = id % query_parts;
    const uint16_t* src = a.qkv + (size_t)m * a.row_stride;
    const int step = kHeads * query_parts;
    int h = part * kHeads + threadIdx.x / kLanes;
    uint4 x_next = make_uint4(0, 0, 0, 0), y_next = x_next;
    const auto load = [&](int head) {
      if (head >= a.heads) return;
      x_next = *reinterpret_cast<const uint4*>(src + (size_t)head * D + ch.o0);
      y_next = *reinterpret_cast<const uint4*>(src + (size_t)head * D + ch.o1);
    };
    load(h);
    float cs[8], sn[8];
    if (ch.turns) angles(a, m, i, cs, sn);
    if (part == 0 && (a.weights || a.slot_pos)) {
      const int seq = a.seq[m], slot = a.slot[m];
      size_t row;
      if (seq >= 0 && seq < c.sequences && slot >= 0 && slot < c.capacity() &&
          c.find_row(seq, 0, slot, &row))
        for (int hk = threadIdx.x; hk < c.heads; hk += kThreads) {
          const size_t at = ((size_t)seq * c.heads + hk) * c.capacity() + slot;
          if (a.weights) a.weights[at] = 0.0f;
          if (a.slot_pos) a.slot_pos[at] = a.positions[(size_t)m * a.axes];
        }
    }
    for (; h < a.heads; h += step) {
      uint4 xo = x_next, yo = y_next;
      load(h + step);
      if (ch.turns) {
        float x[8], y[8];
        unpack_halves(xo, x);
        unpack_halves(yo, y);
        turn(a.interleaved, cs, sn, x, y);
        xo = pack_halves(x);
        yo = pack_halves(y);
      }
      uint16_t* q = a.Q + ((size_t)m * a.heads + h) * D;
      *reinterpret_cast<uint4*>(q + ch.o0) = xo;
      *reinterpret_cast<uint4*>(q + ch.o1) = yo;
    }
    return;
  }

  // Rows m0 .. m0 + 31: bit j of `joins`: row m0 + j goes on with the run of the row before it.
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m0 = blockIdx.x / parts * kSlots8, part = blockIdx.x % parts;
  bool stored = false, joined = false;
  int my_seq = 0, my_slot = 0;
  if (lane < 2 * kSlots8 - 1 && m0 + lane < a.M) {
    my_seq = a.seq[m0 + lane];
    my_slot = a.slot[m0 + lane];
    size_t row;
    stored = my_seq >= 0 && my_seq < c.sequences && my_slot >= 0 && my_slot < c.capacity() &&
             c.find_row(my_seq, 0, my_slot, &row);
    joined = stored && m0 + lane > 0 && my_slot % kSlots8 != 0 &&
             a.seq[m0 + lane - 1] == my_seq && a.slot[m0 + lane - 1] == my_slot - 1;
  }
  const uint64_t joins = __ballot(joined);
  uint64_t leads = __ballot(stored && !joined) & ((1ull << kSlots8) - 1);

  const bool value = wave >= 2;  // waves 0, 1: keys
  const int stride = 2 * parts;
  // Item n of the window, pair n % pairs of the heads of run n / pairs, is part n % parts's.
  const int pairs = (c.heads + 1) / 2;
  for (int own = part; leads; leads &= leads - 1) {
    const int pair = own;  // its first of this run
    if (pair >= pairs) {
      own -= pairs;
      continue;
    }
    own += (pairs - pair + parts - 1) / parts * parts - pairs;
    const int lead = __builtin_ctzll(leads);
    const int count = 1 + __builtin_ctzll(~(joins >> (lead + 1)));
    const int m = m0 + lead;
    const int seq = __builtin_amdgcn_readlane(my_seq, lead);
    const int slot = __builtin_amdgcn_readlane(my_slot, lead);
    const int first = slot % kSlots8;
    const size_t row0 = c.row_of(seq, 0, slot - first);  // of the block, in head 0's page
    float cs[kPasses][8], sn[kPasses][8];
    bool mine[kPasses];  // the lane's row of the pass is a token's
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      const int r = p * kRowsAtOnce + lane / kLanes;
      mine[p] = r >= first && r < first + count;
      if (!value && ch.turns && mine[p]) angles(a, m + r - first, i, cs[p], sn[p]);
    }
    uint4 x_next[kPasses], y_next[kPasses];
    uint16_t old_next = 0;
    const auto load = [&](int hk) {
      if (hk >= c.heads) return;
      const size_t row = row0 + ((size_t)hk << c.log_page);
      old_next = (value ? c.v_scale : c.k_scale)[row / kSlots8];
#pragma unroll
      for (int p = 0; p < kPasses; ++p)
        if (mine[p]) {
          const uint16_t* src =
              a.qkv + (size_t)(m + p * kRowsAtOnce + lane / kLanes - first) * a.row_stride +
              (size_t)(a.heads + (value ? c.heads : 0) + hk) * D;
          x_next[p] = *reinterpret_cast<const uint4*>(src + ch.o0);
          y_next[p] = *reinterpret_cast<const uint4*>(src + ch.o1);
        }
    };
    int hk = 2 * pair + (wave & 1);
    load(hk);
    for (; hk < c.heads; hk += stride) {
      const size_t row = row0 + ((size_t)hk << c.log_page);
      uint8_t* dst = (value ? c.v : c.k) + row * D;
      const uint16_t old_bits = old_next;
      float x[kPasses][8], y[kPasses][8];
      float top = 0.0f;
#pragma unroll
      for (int p = 0; p < kPasses; ++p)
        if (mine[p]) {
          unpack_halves(x_next[p], x[p]);
          unpack_halves(y_next[p], y[p]);
          if (!value && ch.turns) {
            // The float16 values that a float16 cache would hold.
            turn(a.interleaved, cs[p], sn[p], x[p], y[p]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              x[p][e] = (float)(_Float16)x[p][e];
              y[p][e] = (float)(_Float16)y[p][e];
            }
          }
          top = fmaxf(top, fmaxf(max_finite(x[p]), max_finite(y[p])));
        }
      load(hk + stride);
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
      // A scale so far that is none (of a block never written) counts as the smallest.
      const int bits = (old_bits >> 10) - 15;
      const int so_far = first == 0 || bits > kHighest8 ? kLowest8 : max(bits, kLowest8);
      const int e = max(scale_exponent(top), so_far);
      const float inv = __builtin_amdgcn_ldexpf(1.0f, -e);
      const float most = e == kHighest8 ? 240.0f : 448.0f;
      const bool grown = first != 0 && e > so_far;
      const float shrink = __builtin_amdgcn_ldexpf(1.0f, so_far - e);
#pragma unroll
      for (int p = 0; p < kPasses; ++p) {
        uint8_t* at = dst + (p * kRowsAtOnce + lane / kLanes) * D;
        if (mine[p]) {
          *reinterpret_cast<uint2*>(at + ch.o0) =
              make_uint2(codes4(x[p], inv, most), codes4(x[p] + 4, inv, most));
          *reinterpret_cast<uint2*>(at + ch.o1) =
              make_uint2(codes4(y[p], inv, most), codes4(y[p] + 4, inv, most));
        } else if (grown) {
          uint4* q = reinterpret_cast<uint4*>(at + 16 * i);
          uint4 w = *q;
          w.x = rescale4(w.x, shrink, most);
          w.y = rescale4(w.y, shrink, most);
          w.z = rescale4(w.z, shrink, most);
          w.w = rescale4(w.w, shrink, most);
          *q = w;
        }
      }
      if (lane == 0)
        (value ? c.v_scale : c.k_scale)[row / kSlots8] =
            __builtin_bit_cast(uint16_t, (_Float16)__builtin_amdgcn_ldexpf(1.0f, e));
    }
  }
}

// K and V rows of slots [0, max_length) of every (sequence, KV head), D / 8 lanes per row.
template <int D, int kFormat>
__global__ void __launch_bounds__(kThreads)
    kv_read_kernel(KvView c, const int32_t* lengths, int max_length, int blocks, uint16_t* K,
                   uint16_t* V) {
  constexpr int kLanes = D / 8;
  const int bh = blockIdx.x / blocks;
  const int t = (blockIdx.x % blocks) * (kThreads / kLanes) + threadIdx.x / kLanes;
  if (t >= max_length) return;
  const int b = bh / c.heads, h = bh % c.heads;
  const int i = threadIdx.x % kLanes;
  v4u k = {}, v = {};
  if (t < lengths[b]) {
    const size_t row = c.row_of(b, h, t);
    if constexpr (kFormat == kCacheFp8) {
      const float ks = block_unit(c.k_scale[row / kSlots8]);
      const float vs = block_unit(c.v_scale[row / kSlots8]);
      k = dequant8_fp8(reinterpret_cast<const uint2*>(c.k + row * D)[i], ks);
      v = dequant8_fp8(reinterpret_cast<const uint2*>(c.v + row * D)[i], vs);
    } else if constexpr (kFormat == kCacheInt4) {
      const float ks = half_to_float(c.k_scale[row]), vs = half_to_float(c.v_scale[row]);
      k = dequant8(reinterpret_cast<const uint32_t*>(c.k + row * (D / 2))[i], ks);
      v = dequant8(reinterpret_cast<const uint32_t*>(c.v + row * (D / 2))[i], vs);
    } else {
      k = reinterpret_cast<const v4u*>(c.k + row * (2 * D))[i];
      v = reinterpret_cast<const v4u*>(c.v + row * (2 * D))[i];
    }
  }
  const size_t out = ((size_t)bh * max_length + t) * D + 8 * i;
  __builtin_nontemporal_store(k, reinterpret_cast<v4u*>(K + out));
  __builtin_nontemporal_store(v, reinterpret_cast<v4u*>(V + out));
}

// Workgroups of an append into FP8. A window of 16 rows has work for one workgroup per pair of heads if its
// tokens are a prompt's, and for 16 if each is of another sequence, which the host does not know. Workgroups
// without work delay the others, so there are more than the pairs only up to two per CU (the append alone, from 32
// heads into 8 of 128: 500 tokens of a prompt 7.7 us, with four per CU 10.5, with none added 8.4, 2000 11.5, 15.4, 11.6; a
// token of each of 64 sequences 5.1, 5.8, 36.4, of 1000 23.6, 23.3, 36.5; of 800 into one head of 64 7.0, 6.4, 32), and
// fewer where windows alone are many (6113 tokens into 32 heads: 2048 in all 57 us, 1024 64, 4096 65).
struct Append8 {
  int parts, query_parts;
  int block_groups;
  long long grid;
};
Append8 append8_sizes(int M, int heads, const KvView& c) {
  Append8 s;
  const int per_pass = kThreads / (c.dim / 16);
  const int pairs = (c.heads - 1) / 2 + 1;  // of heads: a workgroup takes two at a time
  const int passes = (heads - 1) / per_pass + 1;
  const int windows = (M - 1) / kSlots8 + 1;
  const long long items = (long long)std::min(M, kSlots8) * pairs;  // of a window, at most
  s.parts = std::max({1, std::min(pairs, 2048 / windows), (int)std::min<long long>(items, 512 / windows)});
  s.query_parts = M < 768 ? std::min(passes, 65535) : 1;  // few tokens: as below
  const long long blocks = (long long)windows * s.parts;
  s.block_groups = (int)std::min<long long>(blocks, INT32_MAX);
  s.grid = blocks + (long long)M * s.query_parts;
  return s;
}

template <int D>
hipError_t append(const RopeArgs& a, const KvView& c, hipStream_t stream) {
  const int per_pass = kThreads / (D / 16);
  if (c.format == kCacheFp8) {
    const Append8 s = append8_sizes(a.M, a.heads, c);
    rope_kv_append8_kernel<D><<<(unsigned)s.grid, kThreads, 0, stream>>>(
        a, c, s.parts, s.block_groups, s.query_parts);
    return hipGetLastError();
  }
  const int passes = (a.heads + 2 * c.heads + per_pass - 1) / per_pass;
  // Few tokens: a workgroup per pass, so that all rows are in flight at once. More fill the card
  // by themselves, and a workgroup then looks up its token's cosines and place once. 32 + 32 + 32 heads of 128,
  // float16, passes against one: 1 token 3.3, 3.9 us; 256 4.4, 5.0; 512 6.4, 6.6; 1024 10.8, 9.9; 2047
  // 17.9, 16.9. 32 + 8 + 8: 512 4.6, 4.8; 1024 7.2, 6.7; 4096 18.7, 17.4 (into INT4 27.9, 24.7).
  const dim3 grid(a.M, a.M < 768 && passes <= 65535 ? passes : 1);
  if (c.int4())
    rope_kv_append_kernel<D, true><<<grid, kThreads, 0, stream>>>(a, c);
  else
    rope_kv_append_kernel<D, false><<<grid, kThreads, 0, stream>>>(a, c);
  return hipGetLastError();
}

int read_blocks(int dim, int max_length) {  // of a (sequence, KV head)
  return (max_length - 1) / (kThreads / (dim / 8)) + 1;
}

template <int D>
hipError_t read(const KvView& c, const int32_t* lengths, int max_length, uint16_t* K, uint16_t* V,
                hipStream_t stream) {
  const int blocks = read_blocks(D, max_length);
  const long long grid = (long long)blocks * c.sequences * c.heads;
  const auto run = [&](auto kernel) {
    kernel<<<(unsigned)grid, kThreads, 0, stream>>>(c, lengths, max_length, blocks, K, V);
  };
  c.format == kCacheFp8    ? run(kv_read_kernel<D, kCacheFp8>)
  : c.format == kCacheInt4 ? run(kv_read_kernel<D, kCacheInt4>)
                           : run(kv_read_kernel<D, kCacheF16>);
  return hipGetLastError();
}

}  // namespace

bool append_fits(int M, int heads, const KvView& c) {
  return fits_grid(c.format == kCacheFp8 ? append8_sizes(M, heads, c).grid : M, kThreads);
}

bool read_fits(const KvView& c, int max_length) {
  return fits_grid((long long)read_blocks(c.dim, max_length) * c.sequences * c.heads, kThreads);
}

hipError_t launch_rope_kv_append(const RopeArgs& a, const KvView& c, hipStream_t stream) {
  switch (c.dim) {
    case 64: return append<64>(a, c, stream);
    case 128: return append<128>(a, c, stream);
    default: return append<256>(a, c, stream);
  }
}

hipError_t launch_kv_read(const KvView& c, const int32_t* lengths, int max_length, uint16_t* K,
                          uint16_t* V, hipStream_t stream) {
  switch (c.dim) {
    case 64: return read<64>(c, lengths, max_length, K, V, stream);
    case 128: return read<128>(c, lengths, max_length, K, V, stream);
    default: return read<256>(c, lengths, max_length, K, V, stream);
  }
}

}  // namespace rrs
