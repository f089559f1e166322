// Pages of a cache: rows of the page table forked, trimmed, freed and extended (kv_fork), pages in use
// moved to the front of the pool (kv_compact), and the pages themselves copied (kv_copy_pages). gfx950 only.
//
// No reference counts are kept: which pages are free follows from the table and the lengths, so
// every plan marks the pages that its rows keep, ranks the others by their numbers and hands
// them out in the order of rows. That is integer work on a few bytes per page and entry:
// latency bounds it. One workgroup does all of it where the table is small: pages are bits in LDS,
// ranks are popcounts. Larger tables are marked and written by the whole card, with the
// one workgroup between them.
//
// Copies: a page of a head is one run of memory, so a page is two runs of bytes (and two of scales),
// cut into pieces of 16 KB. Bound by HBM: 2019 pages of 2 x 128 KiB, with their plan, 197 us (5.36 TB/s
// read and written, as a plain copy of that size). Past the caches: 221 us with ordinary loads and stores.
#include <algorithm>

#include "rrs_device.h"
#include "rrs_kv.h"

namespace rrs {
namespace {

constexpr int kThreads = 256;
constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / 64;

// Tables up to so many rows and entries, and pools up to so many pages, are planned in one launch: forks of
// 16640 entries with their copies 25.3 us, in four launches 28.7; of 32000 28.1 and 26.2, of 58000 50 and 31.
constexpr int kSmallRows = 2048;
constexpr int kSmallEntries = 24576;
constexpr int kSmallPages = 65536;
constexpr int kMostPages = 1 << 20;  // bits in LDS
constexpr int kFar = 1 << 29;        // running sums stop here

__device__ __forceinline__ int load_agent(const int* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Inclusive prefix sum over the workgroup, and the total. scratch: kPlanWaves ints.
__device__ __forceinline__ int block_prefix(int x, int* scratch, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int mine = wave_prefix(x);
  __syncthreads();
  if (lane == 63) scratch[wave] = mine;
  __syncthreads();
  uint32_t before = mine, all = 0;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) {
    before += w < wave ? scratch[w] : 0;
    all += scratch[w];
  }
  *total = (int)all;
  return (int)before;
}

// Per page: entries that name it, rows that are about to write into it, and the first of these.
struct PageInfo {
  int* refs;
  int* writers;
  int* first;  // S - row, 0: none
};

// What is planned for a row of the new table.
struct RowPlan {
  int parent;  // row of the old table; -1: none
  int have;    // entries taken over
  int total;   // entries in the end
  int begin;   // rank of its first fresh page; bit 31: that one replaces entry have - 1
};

struct ForkPlan {
  uint32_t* used;  // bits of pages that rows keep; where a launch of its own marks them
  PageInfo info;
  RowPlan* rows;
  int* fresh;  // pages handed out, by rank
};

struct Row {
  int parent, kept, want, have, total, last;  // last: the shared page it may write into, or -1
};
__device__ __forceinline__ Row fork_row(const ForkArgs& a, int b) {
  Row r{-1, 0, 0, 0, 0, -1};
  const int p = a.parent ? a.parent[b] : b;
  if (p < 0 || p >= a.sequences) return r;
  const int P = 1 << a.log_page, capacity = a.max_pages << a.log_page;
  r.parent = p;
  r.want = min(max(a.room[b], 0), capacity);
  r.kept = min(min(max(a.lengths[p], 0), capacity), r.want);
  r.have = (r.kept + P - 1) >> a.log_page;
  r.total = (r.want + P - 1) >> a.log_page;
  if (r.want > r.kept && (r.kept & (P - 1)) != 0) {
    r.last = a.table[(size_t)p * a.max_pages + r.have - 1];
    if ((uint32_t)r.last >= (uint32_t)a.pages) r.last = -1;
  }
  return r;
}

// A row's fresh pages where the first writer of a page that has no reader keeps it, and where none does.
struct Need {
  bool copy, copy_tight;
  int some, tight;
};
__device__ __forceinline__ Need needs(const ForkArgs& a, const PageInfo& info, const Row& r, int b) {
  Need n{};
  if (r.last >= 0) {
    const int refs = load_agent(info.refs + r.last);
    const int writers = load_agent(info.writers + r.last);
    const int first = load_agent(info.first + r.last);
    n.copy_tight = refs > 1;
    n.copy = n.copy_tight && !(writers == refs && first == a.sequences - b);
  }
  const int grown = min(r.total - r.have, a.pages + 1);
  n.some = min(grown + n.copy, a.pages + 1);
  n.tight = min(grown + n.copy_tight, a.pages + 1);
  return n;
}

// Where an entry of the new table comes from; nullptr: there is none (-1).
__device__ __forceinline__ const int32_t* fork_entry(const ForkArgs& a, const RowPlan& r,
                                                     const int* fresh, int i) {
  const int copy = (uint32_t)r.begin >> 31, begin = r.begin & 0x7FFFFFFF;
  if (i < r.have - copy) return a.table + (size_t)r.parent * a.max_pages + i;
  return i < r.total ? fresh + begin + i - (r.have - copy) : nullptr;
}

// The entries of a small table that a thread has, kPlanThreads apart: use(k, n, row, column) for the k-th, number n of
// all (past the last: row 0, and n not below their count). Their pages stay in registers between the marks and the
// new table, all loads of a pass are under way at once, and offsets are 32 bits: with loads one after the other an
// entry per thread took 1 us; eight at a time, read twice, in 64 bits, a fork of 24000 entries with its copies took 30.0
// us, now 27.3, a compaction of 18000 41.6, now 37.3.
constexpr int kOwnEntries = kSmallEntries / kPlanThreads;
template <typename Use>
__device__ __forceinline__ void for_own(int rows, int columns, Use use) {
  const uint32_t all = rows * columns;
  const int down = kPlanThreads / columns, right = kPlanThreads % columns;
  int b = threadIdx.x / columns, i = threadIdx.x % columns;
#pragma unroll
  for (int k = 0; k < kOwnEntries; ++k) {
    if (k % 4 == 0 && k * kPlanThreads >= all) break;
    const uint32_t n = k * kPlanThreads + threadIdx.x;
    use(k, n, n < all ? b : 0, i);
    b += down;
    i += right;
    if (i >= columns) {
      i -= columns;
      ++b;
    }
  }
}
// The same without places.
template <typename Use>
__device__ __forceinline__ void for_own_numbers(uint32_t all, Use use) {
#pragma unroll
  for (int k = 0; k < kOwnEntries; ++k) {
    if (k % 4 == 0 && k * kPlanThreads >= all) break;
    use(k, k * kPlanThreads + threadIdx.x);
  }
}

// The plan, by one workgroup. kMarks: it marks the pages itself and writes the table, too, with the
// rows in LDS; else `used` and `info` hold the marks of another launch. kWords: of 32 pages.
template <int kWords, bool kMarks>
__global__ void __launch_bounds__(kPlanThreads) fork_plan_kernel(ForkArgs a, ForkPlan plan) {
  __shared__ uint32_t used[kWords];
  __shared__ uint32_t wanted[kMarks ? kWords : 1];  // pages that a row is about to write into
  __shared__ RowPlan in_lds[kMarks ? kSmallRows : 1];
  __shared__ int scratch[kPlanWaves];
  constexpr int kOwn = kSmallRows / kPlanThreads;  // rows of a thread
  const int t = threadIdx.x;
  const int words = (a.pages + 31) / 32;
  Row own[kOwn];
  int entry[kMarks ? kOwnEntries : 1];
  const uint32_t entries = kMarks ? a.sequences * a.max_pages : 0;
  if constexpr (kMarks) {
    for (int w = t; w < words; w += kPlanThreads) used[w] = wanted[w] = 0;
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
      const int b = k * kPlanThreads + t;
      own[k] = b < a.sequences ? fork_row(a, b) : Row{-1, 0, 0, 0, 0, -1};
      // (The row of entries in place of the parent.)
      if (b < a.sequences) in_lds[b] = RowPlan{own[k].parent * a.max_pages, own[k].have, 0, 0};
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
      const int page = own[k].last;
      if (page < 0) continue;
      atomicOr(&wanted[page / 32], 1u << (page % 32));
      // Atomics, as what follows on them: they meet in the L2.
      atomicExch(plan.info.refs + page, 0);
      atomicExch(plan.info.writers + page, 0);
      atomicExch(plan.info.first + page, 0);
    }
    __threadfence_block();
    __syncthreads();
    for_own(a.sequences, a.max_pages, [&](int k, uint32_t n, int b, int i) {
      const int row = in_lds[b].parent, have = in_lds[b].have;
      const bool there = n < entries && i < have;
      const int page = a.table[there ? (uint32_t)(row + i) : 0u];
      entry[k] = there ? page : -1;
    });
    for_own_numbers(entries, [&](int k, uint32_t) {
      const uint32_t page = entry[k];
      if (page >= (uint32_t)a.pages) return;
      const uint32_t bit = 1u << (page % 32);
      atomicOr(&used[page / 32], bit);
      if (wanted[page / 32] & bit) atomicAdd(plan.info.refs + page, 1);
    });
#pragma unroll
    for (int k = 0; k < kOwn; ++k)
      if (own[k].last >= 0) {
        atomicAdd(plan.info.writers + own[k].last, 1);
        atomicMax(plan.info.first + own[k].last, a.sequences - (k * kPlanThreads + t));
      }
    __threadfence_block();
  } else {
    for (int w = t; w < words; w += kPlanThreads) used[w] = plan.used[w];
  }
  __syncthreads();
  const auto row_of = [&](int b) { return kMarks ? own[b / kPlanThreads] : fork_row(a, b); };

  // Free pages of the thread's words, and of all.
  const int per_thread = (words + kPlanThreads - 1) / kPlanThreads;
  const int w0 = min(t * per_thread, words), w1 = min(w0 + per_thread, words);
  const auto free_bits = [&](int w) {
    const int left = a.pages - 32 * w;
    return ~used[w] & (left >= 32 ? ~0u : (1u << left) - 1);
  };
  int mine = 0, free_pages;
  for (int w = w0; w < w1; ++w) mine += __popc(free_bits(w));
  const int free_upto = block_prefix(mine, scratch, &free_pages);

  // Do all rows get what they need?
  Need own_need[kOwn];
  int sum = 0;
  if constexpr (kMarks) {
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
      own_need[k] = needs(a, plan.info, own[k], k * kPlanThreads + t);
      sum = min(sum + own_need[k].some, kMostPages + 1);
    }
  } else {
    for (int b = t; b < a.sequences; b += kPlanThreads)
      sum = min(sum + needs(a, plan.info, row_of(b), b).some, kMostPages + 1);
  }
  int all;
  block_prefix(sum, scratch, &all);
  const bool tight = all > free_pages;

  int carry = 0, copies = 0, taken = 0;
  const auto chunk = [&](int b, const Row& r, const Need& n) {
    const int need = tight ? n.tight : n.some;
    int here, more;
    const int upto = carry + block_prefix(need, scratch, &here);
    const bool served = need == 0 || upto <= free_pages;
    const bool copy = served && (tight ? n.copy_tight : n.copy);
    // Copies (up to 1024 here) and pages taken (up to 2^20 in all) as one sum.
    const uint32_t both = block_prefix((int)copy << 21 | (served ? need : 0), scratch, &more);
    const int rank = copies + (int)(both >> 21) - 1;
    if (b < a.sequences) {
      RowPlan out{r.parent, r.have, served ? r.total : r.have, served ? upto - need : 0};
      if (copy) {
        out.begin |= (int)0x80000000;
        a.src[rank] = r.last;
        a.dst[rank] = upto - need;  // a rank, for now
      }
      (kMarks ? in_lds : plan.rows)[b] = out;
      a.lengths_out[b] = r.kept;
      a.room_out[b] = served ? r.want : r.kept;
    }
    carry = min(carry + here, kFar);
    copies += (int)((uint32_t)more >> 21);
    taken += more & ((1 << 21) - 1);
  };
  if constexpr (kMarks) {
#pragma unroll
    for (int k = 0; k < kOwn; ++k)
      if (k * kPlanThreads < a.sequences) chunk(k * kPlanThreads + t, own[k], own_need[k]);
  } else {
    for (int b0 = 0; b0 < a.sequences; b0 += kPlanThreads) {
      const int b = b0 + t;
      Row r{-1, 0, 0, 0, 0, -1};
      Need n{};
      if (b < a.sequences) {
        r = fork_row(a, b);
        n = needs(a, plan.info, r, b);
      }
      chunk(b, r, n);
    }
  }
  if (t == 0) {
    a.count[0] = copies;
    a.count[1] = free_pages - taken;
  }
  // The pages of the first ranks.
  int rank = free_upto - mine;
  for (int w = w0; w < w1 && rank < taken; ++w)
    for (uint32_t bits = free_bits(w); bits && rank < taken; bits &= bits - 1)
      plan.fresh[rank++] = 32 * w + __builtin_ctz(bits);
  __threadfence_block();
  __syncthreads();
  for (int i = t; i < a.sequences; i += kPlanThreads) {
    if (i < copies) {
      a.dst[i] = plan.fresh[a.dst[i]];
    } else {
      a.src[i] = -1;
      a.dst[i] = -1;
    }
  }
  if constexpr (kMarks) {
    for_own(a.sequences, a.max_pages, [&](int k, uint32_t n, int b, int i) {
      const RowPlan r = in_lds[b];
      const int copy = (uint32_t)r.begin >> 31, kept = r.have - copy;
      const bool is_fresh = n < entries && i >= kept && i < r.total;
      const int page = plan.fresh[is_fresh ? (uint32_t)((r.begin & 0x7FFFFFFF) + i - kept) : 0u];
      entry[k] = is_fresh ? page : i < kept ? entry[k] : -1;
    });
    for_own_numbers(entries, [&](int k, uint32_t n) {
      if (n < entries) a.table_out[n] = entry[k];
    });
  }
}

// Units of work on the whole card: `kColumns` entries of a row, a wave each.
constexpr int kColumns = 512;
template <typename F>
__device__ __forceinline__ void for_rows(int sequences, int columns, F f) {
  const int per_row = (columns + kColumns - 1) / kColumns;
  const long long units = (long long)sequences * per_row;
  const int waves = kThreads / 64;
  for (long long u = (long long)blockIdx.x * waves + (threadIdx.x >> 6); u < units;
       u += (long long)gridDim.x * waves) {
    const int b = (int)(u / per_row), i0 = (int)(u % per_row) * kColumns;
    f(b, i0, min(i0 + kColumns, columns));
  }
}

__global__ void __launch_bounds__(kThreads) zero_kernel(int* p, int n) {
  for (int i = blockIdx.x * kThreads + threadIdx.x; i < n; i += gridDim.x * kThreads) p[i] = 0;
}

__global__ void __launch_bounds__(kThreads) fork_mark_kernel(ForkArgs a, ForkPlan plan) {
  const PageInfo info = plan.info;
  const int lane = threadIdx.x & 63;
  for_rows(a.sequences, a.max_pages, [&](int b, int i0, int i1) {
    const Row r = fork_row(a, b);
    for (int i = i0 + lane; i < min(i1, r.have); i += 64) {
      const int page = a.table[(size_t)r.parent * a.max_pages + i];
      if ((uint32_t)page >= (uint32_t)a.pages) continue;
      atomicOr(plan.used + page / 32, 1u << (page % 32));
      atomicAdd(info.refs + page, 1);
    }
    if (i0 == 0 && lane == 0 && r.last >= 0) {
      atomicAdd(info.writers + r.last, 1);
      atomicMax(info.first + r.last, a.sequences - b);
    }
  });
}

__global__ void __launch_bounds__(kThreads) fork_write_kernel(ForkArgs a, ForkPlan plan) {
  const int lane = threadIdx.x & 63;
  for_rows(a.sequences, a.max_pages, [&](int b, int i0, int i1) {
    const RowPlan r = plan.rows[b];
#pragma unroll 4
    for (int i = i0 + lane; i < i1; i += 64) {
      const int32_t* from = fork_entry(a, r, plan.fresh, i);
      a.table_out[(size_t)b * a.max_pages + i] = from ? *from : -1;
    }
  });
}

// ---------------------------------------------------------------------------------------------
// Compaction. U pages are in use; those from U on move, in order, to the unused ones below U.
// ---------------------------------------------------------------------------------------------

__device__ __forceinline__ int row_pages(const CompactArgs& a, int b) {
  const int capacity = a.max_pages << a.log_page;
  return (min(max(a.lengths[b], 0), capacity) + (1 << a.log_page) - 1) >> a.log_page;
}

// to: of a page that moves the new number.
__device__ __forceinline__ int compact_entry(const CompactArgs& a, const int* to, int used, int b,
                                             int i, int have) {
  if (i >= have) return -1;
  const int page = a.table[(size_t)b * a.max_pages + i];
  return page >= used && page < a.pages ? to[page] : page;
}

// marks: bits of another launch (else the kernel's own; it then writes the table, too).
template <int kWords, bool kMarks>
__global__ void __launch_bounds__(kPlanThreads)
    compact_plan_kernel(CompactArgs a, const uint32_t* marks, int* to) {
  __shared__ uint32_t used[kWords];
  __shared__ int have_of[kMarks ? kSmallRows : 1];
  __shared__ int scratch[kPlanWaves];
  const int t = threadIdx.x;
  const int words = (a.pages + 31) / 32;
  int entry[kMarks ? kOwnEntries : 1];
  const uint32_t entries = kMarks ? a.sequences * a.max_pages : 0;
  if constexpr (kMarks) {
    for (int w = t; w < words; w += kPlanThreads) used[w] = 0;
    for (int b = t; b < a.sequences; b += kPlanThreads) have_of[b] = row_pages(a, b);
    __syncthreads();
    for_own(a.sequences, a.max_pages, [&](int k, uint32_t n, int b, int i) {
      const bool there = n < entries && i < have_of[b];
      const int page = a.table[there ? n : 0u];
      entry[k] = there ? page : -1;
    });
    for_own_numbers(entries, [&](int k, uint32_t) {
      const uint32_t page = entry[k];
      if (page < (uint32_t)a.pages) atomicOr(&used[page / 32], 1u << (page % 32));
    });
  } else {
    for (int w = t; w < words; w += kPlanThreads) used[w] = marks[w];
  }
  __syncthreads();
  const int per_thread = (words + kPlanThreads - 1) / kPlanThreads;
  const int w0 = min(t * per_thread, words), w1 = min(w0 + per_thread, words);
  int mine = 0, U;
  for (int w = w0; w < w1; ++w) mine += __popc(used[w]);
  block_prefix(mine, scratch, &U);
  // Bits of a word below page U.
  const auto below = [&](int w) {
    const int n = U - 32 * w;
    return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1;
  };
  int movers = 0, holes = 0, moves, same;
  for (int w = w0; w < w1; ++w) {
    movers += __popc(used[w] & ~below(w));
    holes += __popc(~used[w] & below(w));
  }
  int mover = block_prefix(movers, scratch, &moves) - movers;
  int hole = block_prefix(holes, scratch, &same) - holes;
  for (int w = w0; w < w1; ++w) {
    for (uint32_t bits = used[w] & ~below(w); bits; bits &= bits - 1)
      a.src[mover++] = 32 * w + __builtin_ctz(bits);
    for (uint32_t bits = ~used[w] & below(w); bits; bits &= bits - 1)
      a.dst[hole++] = 32 * w + __builtin_ctz(bits);
  }
  if (t == 0) {
    a.count[0] = moves;
    a.count[1] = U;
  }
  __threadfence_block();
  __syncthreads();
  const int size = max(1, a.pages / 2);
  for (int i = t; i < size; i += kPlanThreads) {
    if (i < moves) {
      to[a.src[i]] = a.dst[i];
    } else {
      a.src[i] = -1;
      a.dst[i] = -1;
    }
  }
  if constexpr (kMarks) {
    __threadfence_block();
    __syncthreads();
    for_own_numbers(entries, [&](int k, uint32_t) {
      const bool moved = entry[k] >= U && entry[k] < a.pages;
      const int page = to[moved ? (uint32_t)entry[k] : 0u];
      entry[k] = moved ? page : entry[k];
    });
    for_own_numbers(entries, [&](int k, uint32_t n) {
      if (n < entries) a.table_out[n] = entry[k];
    });
  }
}

__global__ void __launch_bounds__(kThreads) compact_mark_kernel(CompactArgs a, uint32_t* marks) {
  const int lane = threadIdx.x & 63;
  for_rows(a.sequences, a.max_pages, [&](int b, int i0, int i1) {
    for (int i = i0 + lane; i < min(i1, row_pages(a, b)); i += 64) {
      const int page = a.table[(size_t)b * a.max_pages + i];
      if ((uint32_t)page < (uint32_t)a.pages) atomicOr(marks + page / 32, 1u << (page % 32));
    }
  });
}

__global__ void __launch_bounds__(kThreads) compact_write_kernel(CompactArgs a, const int* to) {
  const int lane = threadIdx.x & 63, used = a.count[1];
  for_rows(a.sequences, a.max_pages, [&](int b, int i0, int i1) {
    const int have = row_pages(a, b);
    for (int i = i0 + lane; i < i1; i += 64)
      a.table_out[(size_t)b * a.max_pages + i] = compact_entry(a, to, used, b, i, have);
  });
}

// ---------------------------------------------------------------------------------------------
// Copies
// ---------------------------------------------------------------------------------------------

constexpr int kAtOnce = 4;                             // loads in flight per thread
constexpr int kChunk = kThreads * kAtOnce * 16;        // bytes of a piece

// Units: pieces of k, then of v, then the scales of both, of each pair.
__global__ void __launch_bounds__(kThreads)
    copy_pages_kernel(KvView c, const int32_t* src, const int32_t* dst, const int32_t* count, int n,
                      size_t page_bytes, int pieces, int per_pair, int scale_rows) {
  const long long pairs = count ? min(max(*count, 0), n) : n;
  const long long units = pairs * per_pair;
  for (long long u = blockIdx.x; u < units; u += gridDim.x) {
    const int pair = (int)(u / per_pair), part = (int)(u % per_pair);
    const int from = src[pair], to = dst[pair];
    if ((uint32_t)from >= (uint32_t)c.pages || (uint32_t)to >= (uint32_t)c.pages) continue;
    if (part == 2 * pieces) {
      for (int i = threadIdx.x; i < scale_rows; i += kThreads) {
        c.k_scale[(size_t)to * scale_rows + i] = c.k_scale[(size_t)from * scale_rows + i];
        c.v_scale[(size_t)to * scale_rows + i] = c.v_scale[(size_t)from * scale_rows + i];
      }
      continue;
    }
    uint8_t* pool = part < pieces ? c.k : c.v;
    const size_t at = (size_t)(part % pieces) * kChunk;
    const size_t size = min(page_bytes - at, (size_t)kChunk);
    const v4u* in = reinterpret_cast<const v4u*>(pool + from * page_bytes + at);
    v4u* out = reinterpret_cast<v4u*>(pool + to * page_bytes + at);
    v4u x[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i)
      if ((size_t)(i * kThreads + threadIdx.x) * 16 < size)
        x[i] = __builtin_nontemporal_load(in + i * kThreads + threadIdx.x);
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i)
      if ((size_t)(i * kThreads + threadIdx.x) * 16 < size)
        __builtin_nontemporal_store(x[i], out + i * kThreads + threadIdx.x);
  }
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

unsigned row_grid(int sequences, int columns) {
  const long long units = (long long)sequences * ((columns - 1) / kColumns + 1);
  return (unsigned)std::min<long long>((units + 3) / 4, 2048);
}

bool small(int sequences, int max_pages, int pages) {
  return sequences <= kSmallRows && (long long)sequences * max_pages <= kSmallEntries &&
         pages <= kSmallPages;
}

// Clears n ints.
void zero(int* p, int n, hipStream_t stream) {
  zero_kernel<<<std::min((n - 1) / kThreads + 1, 1024), kThreads, 0, stream>>>(p, n);
}

int words_of(int pages) { return (pages + 31) / 32; }

}  // namespace

int most_pages() { return kMostPages; }

// Bits, three numbers per page, the pages handed out; the rows.
size_t fork_workspace_bytes(int sequences, int pages) {
  return align256(((size_t)words_of(pages) + 4 * (size_t)pages) * 4) +
         align256((size_t)sequences * sizeof(RowPlan));
}

hipError_t launch_kv_fork(const ForkArgs& a, void* workspace, hipStream_t stream) {
  int* bits = static_cast<int*>(workspace);
  const size_t n = (size_t)a.pages, words = (size_t)words_of(a.pages);
  int* info = bits + words;
  ForkPlan plan{reinterpret_cast<uint32_t*>(bits),
                {info, info + n, info + 2 * n},
                reinterpret_cast<RowPlan*>(static_cast<uint8_t*>(workspace) +
                                           align256((words + 4 * n) * 4)),
                info + 3 * n};
  if (small(a.sequences, a.max_pages, a.pages)) {
    fork_plan_kernel<kSmallPages / 32, true><<<1, kPlanThreads, 0, stream>>>(a, plan);
    return hipGetLastError();
  }
  const unsigned grid = row_grid(a.sequences, a.max_pages);
  zero(bits, (int)(words + 3 * n), stream);
  fork_mark_kernel<<<grid, kThreads, 0, stream>>>(a, plan);
  fork_plan_kernel<kMostPages / 32, false><<<1, kPlanThreads, 0, stream>>>(a, plan);
  fork_write_kernel<<<grid, kThreads, 0, stream>>>(a, plan);
  return hipGetLastError();
}

// Bits, and the new numbers.
size_t compact_workspace_bytes(int pages) {
  return align256(((size_t)words_of(pages) + (size_t)pages) * 4);
}

hipError_t launch_kv_compact(const CompactArgs& a, void* workspace, hipStream_t stream) {
  uint32_t* marks = static_cast<uint32_t*>(workspace);
  int* to = static_cast<int*>(workspace) + words_of(a.pages);
  if (small(a.sequences, a.max_pages, a.pages)) {
    compact_plan_kernel<kSmallPages / 32, true><<<1, kPlanThreads, 0, stream>>>(a, marks, to);
    return hipGetLastError();
  }
  const unsigned grid = row_grid(a.sequences, a.max_pages);
  zero(static_cast<int*>(workspace), words_of(a.pages), stream);
  compact_mark_kernel<<<grid, kThreads, 0, stream>>>(a, marks);
  compact_plan_kernel<kMostPages / 32, false><<<1, kPlanThreads, 0, stream>>>(a, marks, to);
  compact_write_kernel<<<grid, kThreads, 0, stream>>>(a, to);
  return hipGetLastError();
}

hipError_t launch_kv_copy_pages(const KvView& c, const int32_t* src, const int32_t* dst, int n,
                                const int32_t* count, hipStream_t stream) {
  const size_t rows = (size_t)c.heads << c.log_page;
  const size_t bytes = rows * c.row_bytes();
  const int pieces = (int)((bytes - 1) / kChunk + 1);
  const bool scales = c.format != kCacheF16;
  const int scale_rows = (int)(c.format == kCacheFp8 ? rows / kSlots8 : rows);
  const int per_pair = 2 * pieces + (scales ? 1 : 0);
  const long long units = (long long)n * per_pair;
  // Four rounds of workgroups, which balance each other (one: 217 us against 197).
  const unsigned grid = (unsigned)std::min<long long>(units, 256 * 32);
  copy_pages_kernel<<<grid, kThreads, 0, stream>>>(c, src, dst, count, n, bytes, pieces, per_pair,
                                                   scale_rows);
  return hipGetLastError();
}

}  // namespace rrs
