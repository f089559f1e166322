// Attention of one new token per sequence over its paged cache. gfx950 only.
//
// One workgroup per (sequence, query head): 256 slots at a time, one logit per thread, the
// running maximum and sum of the softmax, then one output channel per thread over the 256 values.
#include "rrs_device.h"
#include "rrs_kv.h"

namespace rrs {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float wg_max(float v, float* red) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
}

__device__ __forceinline__ float wg_sum(float v, float* red) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

// Value d of a row.
template <int D>
__device__ __forceinline__ float value(const uint8_t* base, const uint16_t* scale, size_t row,
                                       int d) {
  if (!scale) return half_to_float(reinterpret_cast<const uint16_t*>(base)[row * D + d]);
  const uint32_t byte = base[row * (D / 2) + d / 2];
  const int q = (int)(byte << ((d & 1) ? 24 : 28)) >> 28;
  return (float)q * half_to_float(scale[row]);
}

// logits (nullptr: not wanted): sequences x heads x max_length.
template <int D>
__global__ void __launch_bounds__(kThreads)
    attention_kernel(AttentionArgs a, KvView c, float* logits, float* lse_out) {
  __shared__ float q[D], p[kThreads], red[4];
  const int bh = blockIdx.x;
  const int b = bh / a.heads, h = bh % a.heads;
  const int hk = h / (a.heads / c.heads);
  const int t = threadIdx.x;
  const int n = min(max(a.lengths[b], 0), a.max_length);
  if (t < D) q[t] = half_to_float(a.Q[(size_t)bh * D + t]);
  __syncthreads();
  float top = -INFINITY, total = 0.0f, acc = 0.0f;
  for (int t0 = 0; t0 < n; t0 += kThreads) {
    const int s = t0 + t;
    const bool live = s < n && !(a.mask && !a.mask[(size_t)b * c.capacity() + s]);
    float l = -INFINITY;
    if (live) {
      const size_t row = c.row_of(b, hk, s);
      float dot = 0.0f;
      for (int d = 0; d < D; ++d) dot += q[d] * value<D>(c.k, c.k_scale, row, d);
      l = dot * a.scale;
    }
    if (logits && s < n) logits[(size_t)bh * a.max_length + s] = l;
    const float new_top = fmaxf(top, wg_max(l, red));
    const float base = new_top == -INFINITY ? 0.0f : new_top;
    const float shrink = expf(top - base);
    p[t] = live ? expf(l - base) : 0.0f;
    total = total * shrink + wg_sum(p[t], red);  // its barrier publishes p
    acc *= shrink;
    if (t < D)
      for (int j = 0; j < min(kThreads, n - t0); ++j)
        if (p[j] != 0.0f) acc += p[j] * value<D>(c.v, c.v_scale, c.row_of(b, hk, t0 + j), t);
    top = new_top;
    __syncthreads();
  }
  const float lse = total > 0.0f ? top + logf(total) : -INFINITY;
  if (t < D)
    a.out[(size_t)bh * D + t] =
        __builtin_bit_cast(uint16_t, (_Float16)(total > 0.0f ? acc / total : 0.0f));
  if (t == 0 && a.lse) a.lse[bh] = lse;
  if (t == 0 && lse_out) lse_out[bh] = lse;
}

// weights[b, hk, s] += sum over the group's heads of exp(logit - lse).
__global__ void __launch_bounds__(kThreads)
    weights_kernel(AttentionArgs a, KvView c, const float* logits, const float* lse, int blocks) {
  const int bh = blockIdx.x / blocks;
  const int s = (blockIdx.x % blocks) * kThreads + threadIdx.x;
  const int b = bh / c.heads, hk = bh % c.heads;
  if (s >= min(a.lengths[b], a.max_length)) return;
  const int group = a.heads / c.heads;
  float sum = 0.0f;
  for (int g = 0; g < group; ++g) {
    const size_t at = (size_t)b * a.heads + hk * group + g;
    const float l = logits[at * a.max_length + s];
    if (l > -INFINITY) sum += expf(l - lse[at]);
  }
  a.weights[(size_t)bh * c.capacity() + s] += sum;
}

size_t lse_bytes(const KvView& c, int heads) {
  return ((size_t)c.sequences * heads * 4 + 255) & ~(size_t)255;
}

}  // namespace

size_t attention_workspace_bytes(const KvView& c, int heads, int max_length, bool with_weights) {
  if (!with_weights) return 0;
  return lse_bytes(c, heads) + (size_t)c.sequences * heads * max_length * 4;
}

hipError_t launch_paged_attention(const AttentionArgs& a, const KvView& c, hipStream_t stream) {
  float* lse = a.weights ? static_cast<float*>(a.workspace) : nullptr;
  float* logits = a.weights ? lse + lse_bytes(c, a.heads) / 4 : nullptr;
  const int grid = c.sequences * a.heads;
  switch (c.dim) {
    case 64: attention_kernel<64><<<grid, kThreads, 0, stream>>>(a, c, logits, lse); break;
    case 128: attention_kernel<128><<<grid, kThreads, 0, stream>>>(a, c, logits, lse); break;
    default: attention_kernel<256><<<grid, kThreads, 0, stream>>>(a, c, logits, lse); break;
  }
  if (a.weights) {
    const int blocks = (a.max_length - 1) / kThreads + 1;
    const long long wgs = (long long)blocks * c.sequences * c.heads;
    if (wgs >= (1ll << 31)) return hipErrorInvalidValue;
    weights_kernel<<<(unsigned)wgs, kThreads, 0, stream>>>(a, c, logits, lse, blocks);
  }
  return hipGetLastError();
}

}  // namespace rrs
