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
// Read-back. One row of K and V per D / 8 lanes; bound by the writes, which go past the caches
// (134 MB from 2048 slots of 4 x 32 INT4 heads: 25.7 us, 40.8 with ordinary stores;
// 41 with both where inputs and outputs in use outgrow the last-level cache).
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
  if (turns) {
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
      if (a.interleaved) {
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

// K and V rows of slots [0, max_length) of every (sequence, KV head), D / 8 lanes per row.
template <int D, bool kInt4>
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
    if constexpr (kInt4) {
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

template <int D>
hipError_t append(const RopeArgs& a, const KvView& c, hipStream_t stream) {
  const int per_pass = kThreads / (D / 16);
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
  if (c.int4())
    kv_read_kernel<D, true>
        <<<(unsigned)grid, kThreads, 0, stream>>>(c, lengths, max_length, blocks, K, V);
  else
    kv_read_kernel<D, false>
        <<<(unsigned)grid, kThreads, 0, stream>>>(c, lengths, max_length, blocks, K, V);
  return hipGetLastError();
}

}  // namespace

bool append_fits(int M) { return fits_grid(M, kThreads); }

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
