// Eviction from the cache by accumulated attention weight. gfx950 only.
//
// Slots are ordered by a 32-bit key that is larger for slots kept first: protected slots the
// largest, then the weight's bits with their order made unsigned; NaN lowest. The key T of the
// budget-th slot is found digit by digit (histograms in LDS, 11 + 11 + 10 bits): slots above T are
// kept, and of those at T the first ones.
//
// Up to 16384 slots (evict_kernel) a workgroup takes a (sequence, KV head) and keeps its keys in
// registers: item k of lane l of wave w is slot (w items + k) 64 + l, so that ranks in slot order
// are ballots within a wave and one sum over the waves. The weights and positions are read once, from HBM;
// what is left is the time of a few passes over registers (latency, not bandwidth).
// Longer rows are cut into segments, one workgroup each, and the passes into launches
// that meet in the workspace.
//
// Measured: 64 rows of 2049 slots to 2048, 5.9 us; 128 rows of up to 8192 to 2048, 13.8 us, their moves
// (INT4 rows of 64 bytes) 14.7 us, or 12.4 where two sets of inputs in turn leave a part of them in the last
// cache; 16 rows of 131072 to 16384, three digits 8.6, 7.5 and 7.9 us, lists 15.0 us, moves 52 us
// (4.5 TB/s).
//
// Moves. The evicted slots below the budget (holes) take the kept slots above it, in order. No slot is
// both, so rows are copied in any order, 16 bytes per lane, bound by HBM: in the same kernel
// where there can be at most one round of them, else in a launch of their own.
#include "rrs_device.h"
#include "rrs_kv.h"

namespace rrs {
namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kMoveThreads = 256;
constexpr int kBins = 2048;  // of a digit
constexpr int kCopies = 4;   // of the first digit's histogram
constexpr int kDigits = 3;
constexpr int kShift[kDigits] = {21, 10, 0};
constexpr int kBits[kDigits] = {11, 11, 10};

__device__ __forceinline__ uint32_t evict_key(float w, bool is_protected) {
  if (is_protected) return 0xFFFFFFFFu;
  if (w != w) return 0u;
  const uint32_t u = __builtin_bit_cast(uint32_t, w + 0.0f);  // -0 counts as 0
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// Exclusive prefix over the waves of one number per wave, and the total; red: kWaves ints.
__device__ __forceinline__ int waves_prefix(int mine, int* red, int* total) {
  const int wave = threadIdx.x >> 6;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[wave] = mine;
  __syncthreads();
  int before = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const int x = red[w];
    before += w < wave ? x : 0;
    sum += x;
  }
  *total = sum;
  return before;
}

__device__ __forceinline__ int ballot_rank(uint64_t b) {  // set bits below this lane
  return __popcll(b & ((1ull << (threadIdx.x & 63)) - 1));
}

// The digit d of a histogram (2048 bins in LDS) such that the bins above it hold fewer than `need`
// slots and with it at least as many; its count, and what is left to take from it.
struct Pick {
  int digit, count, left;
};
__device__ __forceinline__ Pick pick_digit(const int* hist, int need, int* red, Pick* shared) {
  // Thread t sums the bins 2 (1023 - t), + 1: descending bins in ascending threads.
  const int lo = 2 * (kThreads - 1 - (int)threadIdx.x);
  const int a = hist[lo + 1], b = hist[lo];
  const int upto = wave_prefix(a + b);
  int total;
  const int above =
      waves_prefix(__builtin_amdgcn_readlane(upto, 63), red, &total) + upto - a - b;
  if (above < need && above + a >= need) *shared = Pick{lo + 1, a, need - above};
  if (above + a < need && above + a + b >= need) *shared = Pick{lo, b, need - above - a};
  __syncthreads();
  return *shared;
}

// Adds one to hist[digit] for the lanes with `in`; a wave whose digits are all the same adds once.
// kCopies: histograms that the lanes take in turn, since lanes that meet in a bin wait for each
// other (weights fill few bins of the first digit).
template <int kCopies>
__device__ __forceinline__ void count_digit(int* hist, uint32_t digit, bool in) {
  const uint64_t who = __ballot(in);
  if (!who) return;
  const uint32_t first = __builtin_amdgcn_readlane(digit, __builtin_ctzll(who));
  if (__ballot(in && digit == first) == who) {
    if ((int)(threadIdx.x & 63) == __builtin_ctzll(who)) atomicAdd(&hist[first], __popcll(who));
  } else if (in) {
    atomicAdd(&hist[(threadIdx.x & (kCopies - 1)) * kBins + digit], 1);
  }
}

// The copies summed into the first; barriers around it are the caller's.
template <int kCopies>
__device__ __forceinline__ void sum_copies(int* hist) {
#pragma unroll
  for (int i = 0; i < kBins / kThreads; ++i) {
    const int bin = threadIdx.x + i * kThreads;
    int sum = 0;
#pragma unroll
    for (int x = 0; x < kCopies; ++x) sum += hist[x * kBins + bin];
    hist[bin] = sum;
  }
}

// Copies row `from` of a head to row `to`, lane i of kRow / 16.
template <int kRow>
__device__ __forceinline__ void move_row(const KvView& c, int b, int h, int from, int to, int i) {
  size_t src, dst;
  const bool exists = c.find_row(b, h, from, &src);
  if (!c.find_row(b, h, to, &dst) || !exists) return;
  const uint4 k = reinterpret_cast<const uint4*>(c.k + src * kRow)[i];
  const uint4 v = reinterpret_cast<const uint4*>(c.v + src * kRow)[i];
  reinterpret_cast<uint4*>(c.k + dst * kRow)[i] = k;
  reinterpret_cast<uint4*>(c.v + dst * kRow)[i] = v;
  if (c.int4() && i == 0) {
    c.k_scale[dst] = c.k_scale[src];
    c.v_scale[dst] = c.v_scale[src];
  }
}

// Rows [j0, capacity) of the bookkeeping are empty.
__device__ __forceinline__ void clear_from(const EvictArgs& a, const KvView& c, int bh, int j0,
                                           int t, int threads) {
  const size_t base = (size_t)bh * c.capacity();
  for (int j = j0 + t; j < c.capacity(); j += threads) {
    a.weights_out[base + j] = 0.0f;
    a.pos_out[base + j] = -1;
    if (j < a.budget) a.kept[(size_t)bh * a.budget + j] = -1;
  }
}

// max_length <= 1024 kItems. kRow > 0: moves of at most kSources rows too.
template <int kItems, int kRow>
__global__ void __launch_bounds__(kThreads) evict_kernel(EvictArgs a, KvView c) {
  constexpr int kSlots = kItems * kThreads;
  constexpr int kSources = kRow > 0 ? 16 * kThreads / kRow : kSlots / 2;  // min(C, n - C)
  __shared__ int hist[kCopies * kBins > kSources ? kCopies * kBins : kSources];  // later sources
  __shared__ int red[kWaves];
  __shared__ Pick picked;
  const int bh = blockIdx.x;
  const int b = bh / c.heads, h = bh % c.heads;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int n = min(max(a.lengths[b], 0), a.max_length);
  const int C = a.budget;
  const size_t base = (size_t)bh * c.capacity();
  const float* w = a.weights + base;
  const int32_t* pos = a.slot_pos + base;
  float* w_out = a.weights_out + base;
  int32_t* pos_out = a.pos_out + base;
  int32_t* kept = a.kept + (size_t)bh * C;
  const int keep_from = a.keep_from[b];
  if (h == 0 && t == 0) a.new_lengths[b] = min(n, C);

  const int j0 = wave * kItems * 64 + lane;  // slot of item k: j0 + 64 k
  float wr[kItems];
  int32_t pr[kItems];
#pragma unroll
  for (int k = 0; k < kItems; ++k) {
    const int j = j0 + 64 * k;
    wr[k] = j < n ? w[j] : 0.0f;
    pr[k] = j < n ? pos[j] : 0;
  }
  clear_from(a, c, bh, min(n, C), t, kThreads);
  uint64_t keep = ~0ull;  // bit k: item k
  int sources = 0;
  uint32_t key[kItems];
#pragma unroll
  for (int k = 0; k < kItems; ++k) key[k] = evict_key(wr[k], pr[k] >= keep_from);
  if (n == C + 1) {
    // One slot too many, as at every step of a cache at its bound: the last in the order goes, the
    // lowest key's highest slot; slot C takes its place. One reduction instead of the digits
    // (2049 slots: 10.8 us with them).
    uint32_t low = 0xFFFFFFFFu;
    int victim = -1;
#pragma unroll
    for (int k = 0; k < kItems; ++k)
      if (j0 + 64 * k < n && key[k] <= low) {  // slots ascend with k
        low = key[k];
        victim = j0 + 64 * k;
      }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t other = __shfl_xor(low, d);
      const int slot = __shfl_xor(victim, d);
      if (other < low || (other == low && slot > victim)) {
        low = other;
        victim = slot;
      }
    }
    if (lane == 0) {
      hist[wave] = (int)low;
      red[wave] = victim;
    }
    __syncthreads();
    victim = -1;
    low = 0xFFFFFFFFu;
#pragma unroll
    for (int x = 0; x < kWaves; ++x) {
      const uint32_t other = (uint32_t)hist[x];
      const int slot = red[x];
      if (other < low || (other == low && slot > victim)) {
        low = other;
        victim = slot;
      }
    }
    __syncthreads();
    sources = victim < C;
#pragma unroll
    for (int k = 0; k < kItems; ++k)
      if (j0 + 64 * k == victim) keep &= ~(1ull << k);
    if (t == 0 && sources) {
      hist[0] = C;
      if constexpr (kRow > 0) hist[kSources] = victim;
      kept[victim] = C;
      w_out[victim] = w[C];
      pos_out[victim] = pos[C];
    }
  } else if (n > C) {
    // Every key above T is kept, and `need` of those equal to it.
    uint32_t T = 0;
    int need = C;
    bool exact = false;
#pragma unroll
    for (int p = 0; p < kDigits; ++p) {
      if (exact) break;
      for (int i = t; i < (p == 0 ? kCopies : 1) * kBins; i += kThreads) hist[i] = 0;
      __syncthreads();
      const uint32_t mask = (1u << kBits[p]) - 1;
#pragma unroll
      for (int k = 0; k < kItems; ++k) {
        const bool in = j0 + 64 * k < n &&
                        (p == 0 || (key[k] >> (kShift[p] + kBits[p])) ==
                                       (T >> (kShift[p] + kBits[p])));
        if (p == 0)
          count_digit<kCopies>(hist, (key[k] >> kShift[p]) & mask, in);
        else
          count_digit<1>(hist, (key[k] >> kShift[p]) & mask, in);
      }
      __syncthreads();
      if (p == 0) {
        sum_copies<kCopies>(hist);
        __syncthreads();
      }
      const Pick d = pick_digit(hist, need, red, &picked);
      T |= (uint32_t)d.digit << kShift[p];
      need = d.left;
      if (d.left == d.count) {  // all slots with these digits are kept: above T - 1
        T -= 1;  // T > 0: not every slot is kept
        need = 0;
        exact = true;
      }
    }
    // Slots kept among those at T: the first `need` of them.
    keep = 0;
    uint64_t tie = 0;
    int ties = 0;
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      const bool in = j0 + 64 * k < n;
      if (in && key[k] > T) keep |= 1ull << k;
      if (need > 0 && in && key[k] == T) tie |= 1ull << k;
    }
    int total;
    if (need > 0) {
#pragma unroll
      for (int k = 0; k < kItems; ++k) ties += __popcll(__ballot(tie >> k & 1));
      int rank = waves_prefix(ties, red, &total);
#pragma unroll
      for (int k = 0; k < kItems; ++k) {
        const uint64_t b64 = __ballot(tie >> k & 1);
        if ((tie >> k & 1) && rank + ballot_rank(b64) < need) keep |= 1ull << k;
        rank += __popcll(b64);
      }
    }
    // Kept slots at or above C, in order, into LDS.
    int count = 0;
#pragma unroll
    for (int k = 0; k < kItems; ++k)
      count += __popcll(__ballot((keep >> k & 1) && j0 + 64 * k >= C));
    int rank = waves_prefix(count, red, &sources);  // its barriers end the use of hist
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      const bool source = (keep >> k & 1) && j0 + 64 * k >= C;
      const uint64_t b64 = __ballot(source);
      if (source) hist[rank + ballot_rank(b64)] = j0 + 64 * k;
      rank += __popcll(b64);
    }
    // Holes below C, in order, take them.
    count = 0;
#pragma unroll
    for (int k = 0; k < kItems; ++k)
      count += __popcll(__ballot(!(keep >> k & 1) && j0 + 64 * k < C));
    rank = waves_prefix(count, red, &total);
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      const int j = j0 + 64 * k;
      const bool hole = !(keep >> k & 1) && j < C;
      const uint64_t b64 = __ballot(hole);
      if (hole) {
        const int from = hist[rank + ballot_rank(b64)];
        kept[j] = from;
        w_out[j] = w[from];
        pos_out[j] = pos[from];
        if constexpr (kRow > 0) hist[kSources + rank + ballot_rank(b64)] = j;
      }
      rank += __popcll(b64);
    }
  }
#pragma unroll
  for (int k = 0; k < kItems; ++k) {
    const int j = j0 + 64 * k;
    if ((keep >> k & 1) && j < min(n, C)) {
      kept[j] = j;
      w_out[j] = wr[k];
      pos_out[j] = pr[k];
    }
  }
  if constexpr (kRow > 0) {
    static_assert(2 * kSources <= kCopies * kBins, "sources and holes fit");
    constexpr int kLanes = kRow / 16;
    __syncthreads();
    const int i = t / kLanes;
    if (i < sources) move_row<kRow>(c, b, h, hist[i], hist[kSources + i], t % kLanes);
  }
}

// Copies row kept[j] to row j where they differ.
template <int kRow>
__global__ void __launch_bounds__(kMoveThreads)
    evict_move_kernel(const int32_t* kept, int budget, int blocks, KvView c) {
  constexpr int kLanes = kRow / 16;
  const int bh = blockIdx.x / blocks;
  const int j = (blockIdx.x % blocks) * (kMoveThreads / kLanes) + threadIdx.x / kLanes;
  if (j >= budget) return;
  const int from = kept[(size_t)bh * budget + j];
  if (from < 0 || from == j) return;
  move_row<kRow>(c, bh / c.heads, bh % c.heads, from, j, threadIdx.x % kLanes);
}

// ---------------------------------------------------------------------------------------------
// Rows of more than 16384 slots: segments of 8192, a workgroup each, and a launch per digit. A
// launch leaves every segment's histogram in the workspace; the next one sums them, each
// workgroup for itself, and knows the digit.
// ---------------------------------------------------------------------------------------------

constexpr int kSegItems = 8;
constexpr int kSegment = kSegItems * kThreads;

// Per (sequence, KV head) of the workspace.
struct LongRow {
  uint16_t* hist[2];  // segments x kBins; digits 0 and 2 in the first, 1 in the second
  int* above;    // segments: slots above the digits found so far
  int* state;    // T and need after digit 0, the same after digit 1, number of moves
  int* holes;    // evicted slots below the budget, ascending
  int* sources;  // kept slots at or above it, descending
};
constexpr int kStateInts = 8;

struct LongPlan {
  int segments;  // of max_length
  int moves;     // at most: min(budget, max_length - budget)
  int* ws;
  __host__ __device__ size_t ints() const {  // per row
    return (size_t)segments * (kBins + 1) + kStateInts + 2 * (size_t)moves;
  }
  __device__ LongRow row(int bh) const {
    int* p = ws + (size_t)bh * ints();
    LongRow r;
    r.hist[0] = reinterpret_cast<uint16_t*>(p);
    r.hist[1] = r.hist[0] + (size_t)segments * kBins;
    r.above = p + (size_t)segments * kBins;
    r.state = r.above + segments;
    r.holes = r.state + kStateInts;
    r.sources = r.holes + moves;
    return r;
  }
};

// The digit from the segments' histograms; hist: kBins ints of LDS.
__device__ __forceinline__ Pick pick_long(const uint16_t* slices, int segments, int need,
                                          int* hist, int* red, Pick* shared) {
  static_assert(kBins == 2 * kThreads && kSegment < 1 << 16, "two 16-bit counts per thread");
  const uint32_t* pairs = reinterpret_cast<const uint32_t*>(slices) + threadIdx.x;
  int lo = 0, hi = 0;
#pragma unroll 8
  for (int s = 0; s < segments; ++s) {
    const uint32_t x = pairs[(size_t)s * kThreads];
    lo += x & 0xFFFFu;
    hi += x >> 16;
  }
  hist[2 * threadIdx.x] = lo;
  hist[2 * threadIdx.x + 1] = hi;
  __syncthreads();
  return pick_digit(hist, need, red, shared);
}

// Launch p of 0 .. 2: digits below p are known, the histogram of digit p is made. Rows that
// keep everything, and segments past a row's end, have nothing to do.
template <int p>
__global__ void __launch_bounds__(kThreads) evict_digit_kernel(EvictArgs a, KvView c, LongPlan plan) {
  constexpr int kParts = p == 0 ? kCopies : 1;
  __shared__ int hist[kParts * kBins], red[kWaves];
  __shared__ Pick picked;
  const int bh = blockIdx.x / plan.segments, seg = blockIdx.x % plan.segments;
  const int b = bh / c.heads;
  const int n = min(max(a.lengths[b], 0), a.max_length);
  const int segments = (n + kSegment - 1) / kSegment;
  if (n <= a.budget || seg >= segments) return;
  const LongRow r = plan.row(bh);
  const int t = threadIdx.x;
  const size_t base = (size_t)bh * c.capacity();
  float wr[kSegItems];
  int32_t pr[kSegItems];
#pragma unroll
  for (int k = 0; k < kSegItems; ++k) {  // on their way while the digit is found
    const int j = min(seg * kSegment + k * kThreads + t, n - 1);
    wr[k] = a.weights[base + j];
    pr[k] = a.slot_pos[base + j];
  }
  uint32_t T = 0;
  if constexpr (p > 0) {
    const int need = p == 1 ? a.budget : r.state[1];
    if constexpr (p > 1) T = (uint32_t)r.state[0];
    const Pick d = pick_long(r.hist[p - 1], segments, need, hist, red, &picked);
    T |= (uint32_t)d.digit << kShift[p - 1];
    // Of this segment: slots above the digit.
    int mine = 0;
#pragma unroll
    for (int i = 0; i < kBins / kThreads; ++i) {
      const int bin = t + i * kThreads;
      if (bin > d.digit) mine += r.hist[p - 1][(size_t)seg * kBins + bin];
    }
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) mine += __shfl_xor(mine, x);
    int total;
    waves_prefix(mine, red, &total);
    if (t == 0) r.above[seg] = p == 1 ? total : r.above[seg] + total;
    if (t == 0 && seg == 0) {
      r.state[2 * (p - 1)] = (int)T;
      r.state[2 * (p - 1) + 1] = d.left;
    }
    __syncthreads();
  }
  for (int i = t; i < kParts * kBins; i += kThreads) hist[i] = 0;
  __syncthreads();
  const int keep_from = a.keep_from[b];
  const uint32_t mask = (1u << kBits[p]) - 1;
#pragma unroll
  for (int k = 0; k < kSegItems; ++k) {
    const uint32_t key = evict_key(wr[k], pr[k] >= keep_from);
    const bool match = seg * kSegment + k * kThreads + t < n &&
                       (p == 0 || (key >> (kShift[p] + kBits[p])) ==
                                            (T >> (kShift[p] + kBits[p])));
    count_digit<kParts>(hist, (key >> kShift[p]) & mask, match);
  }
  __syncthreads();
  if constexpr (kParts > 1) {
    sum_copies<kParts>(hist);
    __syncthreads();
  }
  reinterpret_cast<uint32_t*>(r.hist[p & 1])[(size_t)seg * kThreads + t] =
      (uint32_t)hist[2 * t] | ((uint32_t)hist[2 * t + 1] << 16);
}

// All digits are known: the kept slots, what the slots that stay look like, and the lists of holes and
// sources. How many slots the segments before this one keep follows from their histograms.
__global__ void __launch_bounds__(kThreads) evict_list_kernel(EvictArgs a, KvView c, LongPlan plan) {
  __shared__ int hist[kBins], red[kWaves];
  __shared__ Pick picked;
  const int bh = blockIdx.x / plan.segments, seg = blockIdx.x % plan.segments;
  const int b = bh / c.heads;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int n = min(max(a.lengths[b], 0), a.max_length);
  const int C = a.budget;
  const int segments = (n + kSegment - 1) / kSegment;
  const LongRow r = plan.row(bh);
  if (seg == 0) {
    if (t == 0 && bh % c.heads == 0) a.new_lengths[b] = min(n, C);
    if (t == 0 && n <= C) r.state[4] = 0;
  }
  const auto clear = [&] {
    clear_from(a, c, bh, min(n, C), seg * kThreads + t, plan.segments * kThreads);
  };
  if (seg >= segments) return clear();
  const size_t base = (size_t)bh * c.capacity();
  const int j0 = seg * kSegment + wave * kSegItems * 64 + lane;  // slot of item k: j0 + 64 k
  float wr[kSegItems];
  int32_t pr[kSegItems];
#pragma unroll
  for (int k = 0; k < kSegItems; ++k) {
    const int j = j0 + 64 * k;
    wr[k] = j < n ? a.weights[base + j] : 0.0f;
    pr[k] = j < n ? a.slot_pos[base + j] : 0;
  }
  uint32_t keep = ~0u;
  if (n > C) {
    const Pick d = pick_long(r.hist[0], segments, r.state[3], hist, red, &picked);
    const uint32_t T = (uint32_t)r.state[2] | (uint32_t)d.digit;
    const int need = d.left;
    // Slots above T and at T in the segments before this one (a wave per segment), and above T
    // in this one.
    int above = 0, at = 0, own = 0;
    for (int s = wave; s <= seg; s += kWaves) {
      const uint16_t* slice = r.hist[0] + (size_t)s * kBins;
      int x = 0;
#pragma unroll
      for (int i = 0; i < (1 << kBits[2]) / 64; ++i) {
        const int bin = 64 * i + lane;
        const int count = slice[bin];
        x += bin > d.digit ? count : 0;
      }
      if (lane == 0) x += r.above[s];
      if (s < seg) {
        above += x;
        if (lane == 0) at += slice[d.digit];
      } else {
        own += x;
      }
    }
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) {
      above += __shfl_xor(above, x);
      own += __shfl_xor(own, x);
    }
    at = __builtin_amdgcn_readfirstlane(at);
    int above_before, ties_before, above_own, total;
    waves_prefix(above, red, &above_before);
    waves_prefix(at, red, &ties_before);
    waves_prefix(own, red, &above_own);
    const int before = above_before + min(need, ties_before);  // kept below this segment

    const int keep_from = a.keep_from[b];
    keep = 0;
    uint32_t tie = 0;
    int ties = 0;
#pragma unroll
    for (int k = 0; k < kSegItems; ++k) {
      const bool in = j0 + 64 * k < n;
      const uint32_t key = evict_key(wr[k], pr[k] >= keep_from);
      if (in && key > T) keep |= 1u << k;
      const bool is = in && key == T;
      if (is) tie |= 1u << k;
      ties += __popcll(__ballot(is));
    }
    int rank = ties_before + waves_prefix(ties, red, &total);
    int count = 0;
#pragma unroll
    for (int k = 0; k < kSegItems; ++k) {
      const uint64_t b64 = __ballot(tie >> k & 1);
      if ((tie >> k & 1) && rank + ballot_rank(b64) < need) keep |= 1u << k;
      rank += __popcll(b64);
      count += __popcll(__ballot(keep >> k & 1));
    }
    // Kept slots before every slot: holes below C are counted up, sources at or above it down from
    // all C kept ones.
    rank = before + waves_prefix(count, red, &total);
#pragma unroll
    for (int k = 0; k < kSegItems; ++k) {
      const int j = j0 + 64 * k;
      const uint64_t b64 = __ballot(keep >> k & 1);
      const int kept_before = rank + ballot_rank(b64);
      const bool keeps = keep >> k & 1;
      if (j < C && !keeps) r.holes[j - kept_before] = j;
      if (j >= C && keeps) r.sources[C - 1 - kept_before] = j;
      // Slot C - 1 knows the number of holes.
      if (j == C - 1) r.state[4] = C - kept_before - (keeps ? 1 : 0);
      rank += __popcll(b64);
    }
  }
  int32_t* kept = a.kept + (size_t)bh * C;
#pragma unroll
  for (int k = 0; k < kSegItems; ++k) {
    const int j = j0 + 64 * k;
    if ((keep >> k & 1) && j < min(n, C)) {
      kept[j] = j;
      a.weights_out[base + j] = wr[k];
      a.pos_out[base + j] = pr[k];
    }
  }
  clear();  // last: loads issued after these stores would wait for them
}

// Move number i of a row: hole i takes source (moves - 1 - i) of the descending list.
template <int kRow>
__global__ void __launch_bounds__(kMoveThreads)
    evict_long_move_kernel(EvictArgs a, KvView c, LongPlan plan, int blocks) {
  constexpr int kLanes = kRow / 16;
  const int bh = blockIdx.x / blocks;
  const int i = (blockIdx.x % blocks) * (kMoveThreads / kLanes) + threadIdx.x / kLanes;
  const LongRow r = plan.row(bh);
  const int moves = r.state[4];
  if (i >= moves) return;
  const int to = r.holes[i], from = r.sources[moves - 1 - i];
  if (threadIdx.x % kLanes == 0) {
    const size_t base = (size_t)bh * c.capacity();
    a.kept[(size_t)bh * a.budget + to] = from;
    a.weights_out[base + to] = a.weights[base + from];
    a.pos_out[base + to] = a.slot_pos[base + from];
  }
  move_row<kRow>(c, bh / c.heads, bh % c.heads, from, to, threadIdx.x % kLanes);
}

// ---------------------------------------------------------------------------------------------

constexpr int kMostInRegisters = 16 * kThreads;

int most_moves(int max_length, int budget) {
  const int over = max_length - budget;
  return over <= 0 ? 0 : over < budget ? over : budget;
}

LongPlan long_plan(int max_length, int budget, void* workspace) {
  return LongPlan{(max_length - 1) / kSegment + 1, most_moves(max_length, budget),
                  static_cast<int*>(workspace)};
}

// The launches' workgroups: of the selection, and of the moves where they are a launch of their own.
struct Grids {
  long long select, move;
  int move_blocks;  // per (sequence, KV head)
};
Grids grids(const KvView& c, int max_length, int budget) {
  const int row = c.int4() ? c.dim / 2 : 2 * c.dim, per_block = kMoveThreads / (row / 16);
  const long long rows = (long long)c.sequences * c.heads;
  const int moves = most_moves(max_length, budget);
  const bool longer = max_length > kMostInRegisters;
  // One round of a workgroup's lanes moves so many rows; with no more, they are moved right there.
  const bool moves_too = !longer && moves <= 16 * kThreads / row;
  const int of = moves_too ? 0 : longer ? moves : budget;
  Grids g;
  g.move_blocks = (of + per_block - 1) / per_block;
  g.select = longer ? rows * ((max_length - 1) / kSegment + 1) : rows;
  g.move = rows * g.move_blocks;
  return g;
}

template <int kRow>
hipError_t launch(const EvictArgs& a, const KvView& c, void* workspace, hipStream_t stream) {
  const Grids g = grids(c, a.max_length, a.budget);
  const unsigned select = (unsigned)g.select, move = (unsigned)g.move;
  if (a.max_length > kMostInRegisters) {
    const LongPlan plan = long_plan(a.max_length, a.budget, workspace);
    if (move > 0) {
      evict_digit_kernel<0><<<select, kThreads, 0, stream>>>(a, c, plan);
      evict_digit_kernel<1><<<select, kThreads, 0, stream>>>(a, c, plan);
      evict_digit_kernel<2><<<select, kThreads, 0, stream>>>(a, c, plan);
    }
    evict_list_kernel<<<select, kThreads, 0, stream>>>(a, c, plan);
    if (move > 0)
      evict_long_move_kernel<kRow>
          <<<move, kMoveThreads, 0, stream>>>(a, c, plan, g.move_blocks);
    return hipGetLastError();
  }
  const bool moves_too = move == 0;
  const auto run = [&](auto kernel) { kernel<<<select, kThreads, 0, stream>>>(a, c); };
  if (a.max_length <= kThreads)
    moves_too ? run(evict_kernel<1, kRow>) : run(evict_kernel<1, 0>);
  else if (a.max_length <= 4 * kThreads)
    moves_too ? run(evict_kernel<4, kRow>) : run(evict_kernel<4, 0>);
  else if (a.max_length <= 8 * kThreads)
    moves_too ? run(evict_kernel<8, kRow>) : run(evict_kernel<8, 0>);
  else
    moves_too ? run(evict_kernel<16, kRow>) : run(evict_kernel<16, 0>);
  if (hipError_t e = hipGetLastError()) return e;
  if (moves_too) return hipSuccess;
  evict_move_kernel<kRow>
      <<<move, kMoveThreads, 0, stream>>>(a.kept, a.budget, g.move_blocks, c);
  return hipGetLastError();
}

}  // namespace

bool evict_fits(const KvView& c, int max_length, int budget) {
  const Grids g = grids(c, max_length, budget);
  return fits_grid(g.select, kThreads) && fits_grid(g.move, kMoveThreads);
}

size_t evict_workspace_bytes(const KvView& c, int max_length, int budget) {
  if (max_length <= kMostInRegisters) return 0;
  return (size_t)c.sequences * c.heads * long_plan(max_length, budget, nullptr).ints() * 4;
}

hipError_t launch_kv_evict(const EvictArgs& a, const KvView& c, void* workspace,
                           hipStream_t stream) {
  switch (c.int4() ? c.dim / 2 : 2 * c.dim) {
    case 32: return launch<32>(a, c, workspace, stream);
    case 64: return launch<64>(a, c, workspace, stream);
    case 128: return launch<128>(a, c, workspace, stream);
    case 256: return launch<256>(a, c, workspace, stream);
    default: return launch<512>(a, c, workspace, stream);
  }
}

}  // namespace rrs
