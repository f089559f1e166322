// Eviction from the cache by accumulated attention weight. gfx950 only.
//
// Slots are ordered by a 32-bit key that is larger for slots kept first: protected slots the
// largest, then the weight's bits with their order made unsigned; NaN lowest. One
// workgroup per (sequence, KV head) finds the key T of the budget-th slot digit by digit
// (four histograms of 8 bits), then walks the slots in order: those above T and the first of those at T
// are kept. A second launch copies the rows that kept names.
#include "rrs_device.h"
#include "rrs_kv.h"

namespace rrs {
namespace {

constexpr int kThreads = 1024;
constexpr int kMoveThreads = 256;

__device__ __forceinline__ uint32_t evict_key(float w, bool is_protected) {
  if (is_protected) return 0xFFFFFFFFu;
  if (w != w) return 0u;
  const uint32_t u = __builtin_bit_cast(uint32_t, w + 0.0f);  // -0 counts as 0
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// Exclusive prefix of `flag` over the workgroup and its total; red: 17 ints.
__device__ __forceinline__ int wg_prefix(bool flag, int* red, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint64_t ballot = __ballot(flag);
  __syncthreads();
  if (lane == 0) red[wave] = __popcll(ballot);
  __syncthreads();
  int before = 0, sum = 0;
  for (int w = 0; w < kThreads / 64; ++w) {
    before += w < wave ? red[w] : 0;
    sum += red[w];
  }
  *total = sum;
  return before + __popcll(ballot & ((1ull << lane) - 1));
}

__global__ void __launch_bounds__(kThreads) evict_select_kernel(EvictArgs a, KvView c) {
  __shared__ int hist[256], red[kThreads / 64], pick[2];
  const int bh = blockIdx.x;
  const int b = bh / c.heads;
  const int t = threadIdx.x;
  const int n = min(max(a.lengths[b], 0), a.max_length);
  const int C = a.budget;
  const int kept_n = min(n, C);
  const size_t base = (size_t)bh * c.capacity();
  const float* w = a.weights + base;
  const int32_t* pos = a.slot_pos + base;
  float* w_out = a.weights_out + base;
  int32_t* pos_out = a.pos_out + base;
  int32_t* kept = a.kept + (size_t)bh * C;
  const int keep_from = a.keep_from[b];
  if (bh % c.heads == 0 && t == 0) a.new_lengths[b] = kept_n;
  for (int j = kept_n + t; j < c.capacity(); j += kThreads) {
    w_out[j] = 0.0f;
    pos_out[j] = -1;
    if (j < C) kept[j] = -1;
  }
  if (n <= C) {
    for (int j = t; j < n; j += kThreads) {
      w_out[j] = w[j];
      pos_out[j] = pos[j];
      kept[j] = j;
    }
    return;
  }
  const auto key = [&](int j) { return evict_key(w[j], pos[j] >= keep_from); };

  // T, and how many slots at T are kept.
  uint32_t T = 0;
  int need = C;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int j = t; j < 256; j += kThreads) hist[j] = 0;
    __syncthreads();
    for (int j = t; j < n; j += kThreads) {
      const uint32_t k = key(j);
      if (shift == 24 || (k >> (shift + 8)) == (T >> (shift + 8)))
        atomicAdd(&hist[(k >> shift) & 255], 1);
    }
    __syncthreads();
    if (t == 0) {
      int d = 255, left = need;
      while (hist[d] < left) left -= hist[d--];
      pick[0] = d;
      pick[1] = left;
    }
    __syncthreads();
    T |= (uint32_t)pick[0] << shift;
    need = pick[1];
  }

  // Kept slots at or above C, in order, into kept[0..); ties counted from slot 0.
  int ties = 0, total, moved = 0;
  for (int j0 = 0; j0 < n; j0 += kThreads) {
    const int j = j0 + t;
    const uint32_t k = j < n ? key(j) : 0;
    const bool tie = j < n && k == T;
    const int rank = ties + wg_prefix(tie, red, &total);
    ties += total;
    const bool keep = j < n && (k > T || (tie && rank < need));
    const bool source = keep && j >= C;
    const int at = moved + wg_prefix(source, red, &total);
    moved += total;
    if (source) kept[at] = j;
    // A slot below C says in w_out whether it is kept; read back by the same thread.
    if (j < C) w_out[j] = keep ? 1.0f : 0.0f;
  }
  __syncthreads();
  // From the highest slot down: hole number r (r <= its slot) takes source r, which lies at
  // kept[r] and is overwritten only by a slot at or below this one.
  int after = 0;
  for (int j0 = (C - 1) / kThreads * kThreads; j0 >= 0; j0 -= kThreads) {
    const int j = j0 + t;
    const bool hole = j < C && w_out[j] == 0.0f;
    const int before = wg_prefix(hole, red, &total);
    const int r = moved - after - total + before;
    after += total;
    const int from = hole ? kept[r] : j;
    __syncthreads();
    if (j < C) {
      kept[j] = from;
      w_out[j] = w[from];
      pos_out[j] = pos[from];
    }
    __syncthreads();
  }
}

// Copies row kept[j] to row j where they differ. Sources are at or above the budget and
// targets below it, so no row is both. kRow: bytes of a row; 16 bytes per lane.
template <int kRow>
__global__ void __launch_bounds__(kMoveThreads)
    evict_move_kernel(const int32_t* kept, int budget, int blocks, KvView c) {
  constexpr int kLanes = kRow / 16;
  const int bh = blockIdx.x / blocks;
  const int j = (blockIdx.x % blocks) * (kMoveThreads / kLanes) + threadIdx.x / kLanes;
  if (j >= budget) return;
  const int from = kept[(size_t)bh * budget + j];
  if (from < 0 || from == j) return;
  const int i = threadIdx.x % kLanes;
  const int b = bh / c.heads, h = bh % c.heads;
  size_t src, dst;
  const bool exists = c.find_row(b, h, from, &src);
  if (!c.find_row(b, h, j, &dst) || !exists) return;
  const uint4 k = reinterpret_cast<const uint4*>(c.k + src * kRow)[i];
  const uint4 v = reinterpret_cast<const uint4*>(c.v + src * kRow)[i];
  reinterpret_cast<uint4*>(c.k + dst * kRow)[i] = k;
  reinterpret_cast<uint4*>(c.v + dst * kRow)[i] = v;
  if (c.int4() && i == 0) {
    c.k_scale[dst] = c.k_scale[src];
    c.v_scale[dst] = c.v_scale[src];
  }
}

template <int kRow>
hipError_t move(const EvictArgs& a, const KvView& c, hipStream_t stream) {
  const int rows = kMoveThreads / (kRow / 16);
  const int blocks = (a.budget - 1) / rows + 1;
  const long long grid = (long long)blocks * c.sequences * c.heads;
  if (grid >= (1ll << 31)) return hipErrorInvalidValue;
  evict_move_kernel<kRow><<<(unsigned)grid, kMoveThreads, 0, stream>>>(a.kept, a.budget, blocks, c);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_evict(const EvictArgs& a, const KvView& c, hipStream_t stream) {
  evict_select_kernel<<<c.sequences * c.heads, kThreads, 0, stream>>>(a, c);
  if (hipError_t e = hipGetLastError()) return e;
  if (a.max_length <= a.budget) return hipSuccess;  // nothing can move
  switch (c.int4() ? c.dim / 2 : 2 * c.dim) {
    case 32: return move<32>(a, c, stream);
    case 64: return move<64>(a, c, stream);
    case 128: return move<128>(a, c, stream);
    case 256: return move<256>(a, c, stream);
    default: return move<512>(a, c, stream);
  }
}

}  // namespace rrs
