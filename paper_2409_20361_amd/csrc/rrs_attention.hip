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
// loads for the next tile are issued before the current one is done with.
//
// The slots of a sequence are cut into pieces, one workgroup each; its four waves
// take the piece's tiles in turn and are joined in LDS, pieces of one sequence by a second kernel
// in their order (so results repeat bit for bit). Where the attention weights are asked for, logits
// are kept in the workspace and turned into weights by that second kernel, or by the
// workgroup that has the whole sequence (15 x 3 KV heads of 65 slots: 9.7 -> 6.6 us).
//
// INT4. Codes become float16 exactly (an exponent is or-ed on, an offset taken off). A key's scale
// multiplies its logit; a value's scale multiplies its p before p is rounded to float16. m follows
// the largest of these products, not the largest p or scale: a slot whose values are large and
// whose weight is next to nothing, or the other way round, takes no bits from the others.
//
// p is rounded to float16 (as the matrix instruction needs it), in units that leave the largest
// weight 2^12 or more: off by 2^-11 relative, or by 2^-37 of the largest weight where that is more
// (INT4, with the value's scale: 2^-36 of the largest product). The matrix instruction and the sum of
// the rounded p keep float16's subnormals. Everything else is float32.
//
// Measured (kernel time; bytes of K, V and scales read): 256 sequences of 1 to 4096 slots, 8 KV
// heads of 128, float16, 383 us (5.7 TB/s); one of 131071 slots 94 us (5.7 TB/s); 49 sequences of
// 1 to 4096, INT4, 33.4 us (3.6 TB/s: half of the cycles issue vector instructions, two fifths of them the
// codes' way to float16, at three waves per SIMD; 64 of 1 to 8192 with 16 KV heads
// 127 us with the join, 4.4 TB/s); 8 x 40 heads over one KV head of 256 with a mask, 19 us (2.0 TB/s: latency of three or
// four tiles per wave, the rows read by three row blocks); one sequence of 117 slots, 32 heads, 5
// us (latency); 179 x 64 heads of up to 5 slots 14 us.
#include "rrs_device.h"
#include "rrs_kv.h"

namespace rrs {
namespace {

typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef _Float16 v4h __attribute__((ext_vector_type(4)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef int v2i __attribute__((ext_vector_type(2)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) v4s* lds_v4s;
typedef __attribute__((address_space(3))) v2i* lds_v2i;

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kRows = 16;  // query heads per workgroup: columns of the products
// Sequences up to which pieces follow the lengths: four lengths per lane of find_piece. Above it, as
// below, pieces of one size for all: 100 sequences of 1 to 8192 slots, one KV head of 128, 60.3 against
// 49.7 us; 256 of 1 to 4096 with eight 417 against 401; 65 of them 113 against 115. With eight lengths per
// lane 300 sequences of 1 to 4096 and eight KV heads take 474 instead of 513 us, but 512 with one
// KV head 124 instead of 115.
constexpr int kWidest = 256;
constexpr float kLog2e = 1.4426950408889634f;

// Sizes of a launch, and where its pieces lie in the workspace. A piece is a run of one sequence's
// slots, the work of one workgroup per KV head and row block; pieces of all sequences are
// numbered one after another.
struct Plan {
  int group;       // query heads per KV head
  int row_blocks;  // ceil(group / kRows)
  int step;        // slots that a workgroup takes at a time: pieces are whole numbers of them
  int target;      // workgroups to aim at; 0: pieces of `steps` steps each, `pieces` per sequence
  int steps;       // at least so many steps to a piece
  int pieces;
  int team;        // waves that share a piece: kWaves, or 1
  int ld_logits;   // row stride of the logits: max_length rounded up to whole blocks of 16
  int2* of_seq;    // sequences: first piece and number of pieces
  float* part;     // pieces x heads x dim: sums relative to the piece's m
  float2* stats;   // pieces x heads: m (base 2) and the sum of p
  float* logits;   // sequences x heads x ld_logits, base 2; nullptr: not wanted
  bool adds_weights;  // the first launch adds the weights: whole sequences, one row block
};

// A piece of a sequence: slots [begin, end) of it, number `index` of all pieces, `count` of which
// are the sequence's.
struct Piece {
  int b, n, begin, end, index, count, first;
};

// Which piece `index` is; false past the last. Every wave of every workgroup works this out for
// itself from the lengths, so that sequences of any lengths are cut into pieces of about the same
// size without the host knowing them.
__device__ __forceinline__ bool find_piece(const AttentionArgs& a, const KvView& c,
                                           const Plan& plan, int index, Piece* out) {
  const int lane = threadIdx.x & 63;
  const auto length = [&](int b) { return min(max(a.lengths[b], 0), a.max_length); };
  const auto all_steps = [&](int n) { return max(1, (n + plan.step - 1) / plan.step); };
  const auto steps_of = [&](int n) { return min(all_steps(n), 1 << 22); };  // sums fit an int
  int q = plan.steps, b = -1, first = 0;
  if (plan.target == 0) {
    b = index / plan.pieces;
    first = b * plan.pieces;
    if (b >= c.sequences) return false;
  } else if (c.sequences == 1) {
    const int want = max(plan.target / (c.heads * plan.row_blocks), 1);
    q = max(q, (all_steps(length(0)) + want - 1) / want);
    b = 0;
  } else {
    const int want = max(plan.target / (c.heads * plan.row_blocks), 1);  // pieces
    int steps[kWidest / 64] = {};  // of sequences lane, lane + 64, ...
    int total = 0;
#pragma unroll
    for (int i = 0; i < kWidest / 64; ++i)
      if (64 * i < c.sequences) {
        if (64 * i + lane < c.sequences) steps[i] = steps_of(length(64 * i + lane));
        total += steps[i];
      }
    q = max(q, (wave_total(total) + want - 1) / want);
    // Each sequence's last piece is short: larger pieces until they fit the target.
    for (int round = 0; round < 3; ++round) {
      int sum = 0;
#pragma unroll
      for (int i = 0; i < kWidest / 64; ++i)
        if (64 * i < c.sequences) sum += (steps[i] + q - 1) / q;
      sum = wave_total(sum);
      if (sum <= want || sum <= c.sequences) break;
      q += max(1, (int)((long long)q * (sum - want) / want));
    }
    // The sequence whose pieces contain the index.
#pragma unroll
    for (int i = 0; i < kWidest / 64; ++i)
      if (64 * i < c.sequences && b < 0) {
        const int mine = (steps[i] + q - 1) / q;
        const int upto = wave_prefix(mine);
        const uint64_t past = __ballot(first + upto > index);
        if (past) {
          const int l = __builtin_ctzll(past);
          b = 64 * i + l;
          first += __builtin_amdgcn_readlane(upto - mine, l);
        } else {
          first += __builtin_amdgcn_readlane(upto, 63);
        }
      }
    if (b < 0) return false;
  }
  const int n = __builtin_amdgcn_readfirstlane(length(b));
  const int steps = all_steps(n);
  const int count = ((c.sequences == 1 ? steps : steps_of(n)) + q - 1) / q;
  const int i = index - first;
  if (i >= count) return false;
  // Even pieces: the first steps % count of them are one step longer.
  const int base = steps / count, longer = steps % count;
  const int from = i * base + min(i, longer);
  const int to = from + base + (i < longer ? 1 : 0);
  out->b = b;
  out->n = n;
  out->begin = __builtin_amdgcn_readfirstlane(from * plan.step);
  out->end = __builtin_amdgcn_readfirstlane(min(n, to * plan.step));
  out->index = index;
  out->count = __builtin_amdgcn_readfirstlane(count);
  out->first = first;
  return true;
}

template <int D, bool kInt4, int kTeam = kWaves>
struct Shape {
  // Slots per wave and step. 16 where 32 rows would not leave registers for a second wave, and for
  // short sequences: more waves hide more of the chain of length, page and rows (179 x 64 heads of up to
  // 5 slots 26 -> 21 us, 200 x 64 of up to 64 within 3 %).
  static constexpr int kTile = kInt4 ? 64 : D == 256 || kTeam == 1 ? 16 : 32;
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
  // Waves: limits the registers.
  static constexpr int kPerSimd = D == 256 ? 2 : kTeam == 1 && !kInt4 ? 4 : 3;

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

// The T at byte `at` past an address that is the same for the wave: the address stays in scalar
// registers and the offset in one vector register (the compiler would else keep a 64-bit
// vector address for every such load of the loop).
template <typename T>
__device__ __forceinline__ T load_at(const void* base, uint32_t at) {
  typedef const __attribute__((address_space(1))) uint8_t* Global;
  Global p = (Global)base;
  asm("" : "+s"(p), "+v"(at));
  return *(const __attribute__((address_space(1))) T*)(p + at);
}

// Halves of x whose slot takes no part become 0.
template <typename V>
__device__ __forceinline__ V mask_halves(V x, const bool* live) {
  constexpr int kDwords = sizeof(V) / 4;
  typedef uint32_t W __attribute__((ext_vector_type(kDwords)));
  W w = __builtin_bit_cast(W, x);
#pragma unroll
  for (int i = 0; i < kDwords; ++i)
    w[i] &= (live[2 * i] ? 0xFFFFu : 0u) | (live[2 * i + 1] ? 0xFFFF0000u : 0u);
  return __builtin_bit_cast(V, w);
}

// NaN if one of them is (the column's result is NaN then, whatever its maximum): two of these are one
// instruction, where fmaxf first quiets its operands.
__device__ __forceinline__ float larger(float a, float b) {
  return __builtin_elementwise_maximum(a, b);
}

// The largest of x over the four lanes of a column.
__device__ __forceinline__ float column_max(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  x = larger(__builtin_bit_cast(float, (uint32_t)a[0]), __builtin_bit_cast(float, (uint32_t)a[1]));
  const uint32_t v = __builtin_bit_cast(uint32_t, x);
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return larger(__builtin_bit_cast(float, (uint32_t)b[0]),
               __builtin_bit_cast(float, (uint32_t)b[1]));
}

// float16 values: p is taken into the products as float16 of up to 2^15. A column's m is set kLift
// below its largest logit, and again where p would outgrow 2^kRoom: few tiles do that, and the largest
// p is 2^kLift at least, so that smaller ones are off by 2^-11 relative or half a subnormal
// step, 2^-25, at most: 2^-37 of the largest.
//
// INT4: the products of p and value scales are such float16 numbers. m is set so that
// the largest product lies in [2^(kLift - 1), 2^kLift), and again where one outgrows 2^15;
// smaller ones are off by 2^-11 relative or half a subnormal step, 2^-25, at most: 2^-36 of the largest.
// Where all products are small m is kDeepest below the largest logit, and what a product loses
// is at most 2^-25 2^-kDeepest of a weight of 1, times a code: 7 x 2^-45 of the output, which
// is float16. p itself stays below 2^kFar; its sum and that of the products are float32.
constexpr int kLift = 12;
constexpr float kRoom = 15.0f;
constexpr int kDeepest = 20;
constexpr float kFar = 24.0f;

// The weights of four slots: the sum over `rows` rows, ld apart, of 2^(logit - top) inv of the row;
// at(g): top and inv of row g.
template <typename At>
__device__ __forceinline__ float4 slot_weights(const float* logits, int ld, int rows, At at) {
  float4 w = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
  for (int g = 0; g < rows; ++g) {
    const float4 l = *reinterpret_cast<const float4*>(logits + (size_t)g * ld);
    const float2 r = at(g);
    w.x += __builtin_amdgcn_exp2f(l.x - r.x) * r.y;
    w.y += __builtin_amdgcn_exp2f(l.y - r.x) * r.y;
    w.z += __builtin_amdgcn_exp2f(l.z - r.x) * r.y;
    w.w += __builtin_amdgcn_exp2f(l.w - r.x) * r.y;
  }
  // Of a row with an inv of NaN the slots that take part get NaN; those under the mask (a logit of
  // -inf) got it, too. Summed again without them, since a condition in the loop above keeps its loads from
  // running ahead (40 heads over 6 x 1057 slots: 14.5 -> 22.5 us).
  if (w.x != w.x || w.y != w.y || w.z != w.z || w.w != w.w) {
    float x[4] = {};
    for (int g = 0; g < rows; ++g) {
      const float2 r = at(g);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float l = logits[(size_t)g * ld + i];
        if (l != -INFINITY) x[i] += __builtin_amdgcn_exp2f(l - r.x) * r.y;
      }
    }
    w = make_float4(x[0], x[1], x[2], x[3]);
  }
  return w;
}

// out[s .. s + 3] += w, up to slot n.
__device__ __forceinline__ void add_slots(float* out, int s, int n, const float4& w) {
  const float add[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (s + i < n) out[s + i] += add[i];
}

// log(2^m sum): the exponents are added before the logarithm, so that a sum far from 1 costs
// no digits.
__device__ __forceinline__ float log_sum(float m, float sum) {
  if (sum == 0.0f) return -INFINITY;
  const float e = m + (float)__builtin_amdgcn_frexp_expf(sum);
  return (e + __builtin_amdgcn_logf(__builtin_amdgcn_frexp_mantf(sum))) / kLog2e;
}

// top and inv of a row for slot_weights; a row without slots has logits of -inf only, one whose sum is
// NaN an inv of NaN.
__device__ __forceinline__ float2 weight_row(float top, float total) {
  return total != 0.0f ? make_float2(top, 1.0f / total) : make_float2(0.0f, 0.0f);
}

// Grid: pieces x KV heads x row blocks. The row blocks of a piece and head read the same rows: they
// are 8 apart, on one XCD, and share its L2.
// kTeam: waves that share a piece; 1: every wave takes a whole sequence by itself.
template <int D, bool kInt4, bool kMask, int kTeam>
__global__ void __launch_bounds__(kThreads, (Shape<D, kInt4, kTeam>::kPerSimd))
    attention_kernel(AttentionArgs a, KvView c, Plan plan) {
  using S = Shape<D, kInt4, kTeam>;
  constexpr int kLds = kTeam == 1 ? S::kValues : S::kLds;
  __shared__ __attribute__((aligned(16))) uint8_t lds[kWaves * kLds];
  __shared__ float2 wave_stats[kTeam][kRows], row_stats[kWaves / kTeam][kRows];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15;  // a slot of a block of 16, and a query head
  const int quarter = lane >> 4;

  int unit = blockIdx.x, rb = 0;
  if constexpr (kTeam == 1) unit = unit * kWaves + wave;
  if (plan.row_blocks > 1) {
    rb = unit / 8 % plan.row_blocks;
    unit = unit / (8 * plan.row_blocks) * 8 + unit % 8;
  }
  const int hk = unit % c.heads;
  Piece piece;
  if (!find_piece(a, c, plan, unit / c.heads, &piece)) return;
  const int b = piece.b, n = piece.n, begin = piece.begin, end = piece.end;
  const bool whole = piece.count == 1;  // the piece is the sequence
  if (plan.of_seq && (kTeam == 1 ? lane : threadIdx.x) == 0 && hk == 0 && rb == 0 &&
      piece.index == piece.first)
    plan.of_seq[b] = make_int2(piece.first, piece.count);

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
  // Logits are compared unscaled: a negative scale turns the queries around, and of no scale at
  // all every logit is 0.
  float scale = a.scale * kLog2e;
  if (!(scale > 0.0f)) {
    const _Float16 turn = (_Float16)(scale < 0.0f ? -1.0f : 0.0f);
#pragma unroll
    for (int i = 0; i < S::kSteps; ++i) q[i] *= turn;
    scale = scale < 0.0f ? -scale : 1.0f;
  }
  float* logits = nullptr;
  if (plan.logits && col < rows)
    logits = plan.logits + ((size_t)b * a.heads + head0 + col) * plan.ld_logits + 4 * quarter;

  v4f o[S::kOut] = {};
  float m = -INFINITY, sum = 0.0f;
  float rounded = 0.0f;  // float16 values: the sum of p as the products take it
  uint8_t* tile = lds + wave * kLds;

  // Pages: lane i holds page page0 + i of the sequence.
  const int last = (n - 1) & ~15;  // the last block of 16 slots
  int page0 = 0, pages = 0;
  const auto load_pages = [&](int first) {
    page0 = first;
    pages = c.page_of(b, min(first + lane, last >> c.log_page));
  };
  // Loads of one tile: keys as operands, values as contiguous pieces of their rows, scales of the
  // lane's four slots per block. Blocks past the sequence's end read its last one. Rows past the
  // end lie in that block, in a page of the cache; what they hold is dropped below.
  v4u key[S::kBlocks][(S::kKey + 15) / 16];
  v4u val[S::kBlocks][S::kPieces];
  v2u ks[S::kBlocks], vs[S::kBlocks];
  uint8_t mask = 0;  // of slot t0 + lane
  size_t row[S::kBlocks];  // the blocks' first rows
  // A block's last row, in whose place rows past it are not loaded: thousands of short sequences
  // would spend much of the bandwidth on those past their ends (200 x 64 heads of up to 30 slots 31 -> 23
  // us, of up to 100 76 -> 69). Longer sequences spare the instructions.
  int lim[S::kBlocks];
  const uint32_t quarter_at = quarter * (kInt4 ? S::kKey : 16);
  const uint32_t key_at0 = col * S::kRow + quarter_at;
  const auto load_keys = [&](int t0) {
    if ((min(t0 + S::kTile - 16, last) >> c.log_page) - page0 >= 64) load_pages(t0 >> c.log_page);
#pragma unroll
    for (int u = 0; u < S::kBlocks; ++u) {
      const int t = min(t0 + 16 * u, last);
      const int page = t >> c.log_page;
      row[u] = c.page_row(__builtin_amdgcn_readlane(pages, page - page0), hk) +
               (t & ((1 << c.log_page) - 1));
      lim[u] = kTeam == 1 ? min(n - 1 - t, 15) : 15;
      const uint32_t key_at =
          kTeam == 1 ? min(col, lim[u]) * S::kRow + quarter_at : key_at0;
      const uint8_t* p = c.k + row[u] * S::kRow;
      if constexpr (S::kKey < 16) {
        const v2u w = load_at<v2u>(p, key_at);
        key[u][0] = v4u{w[0], w[1], 0u, 0u};
      } else {
#pragma unroll
        for (int i = 0; i < S::kKey / 16; ++i)
          key[u][i] = load_at<v4u>(p + i * (kInt4 ? 16 : 64), key_at);
      }
      if constexpr (kInt4) {  // four slots: 8 bytes, inside the page
        ks[u] = load_at<v2u>(c.k_scale + row[u], 8 * quarter);
        vs[u] = load_at<v2u>(c.v_scale + row[u], 8 * quarter);
      }
    }
    if constexpr (kMask)  // up to the last block's end: inside the row
      mask = load_at<uint8_t>(a.mask + (size_t)b * c.capacity() + t0, min(lane, last + 15 - t0));
  };
  constexpr int kPerRow = S::kRow / S::kPiece;   // pieces of a row
  constexpr int kRowsPerLoad = 64 / kPerRow;     // rows that the wave loads at a time
  const uint32_t val_at = lane / kPerRow * S::kRow + lane % kPerRow * S::kPiece;
  const auto load_values = [&]() {
#pragma unroll
    for (int u = 0; u < S::kBlocks; ++u)
#pragma unroll
      for (int i = 0; i < S::kPieces; ++i) {
        const int first = min(i * kRowsPerLoad, lim[u] & -kRowsPerLoad);
        const uint8_t* p = c.v + (row[u] + first) * S::kRow;
        if constexpr (S::kPiece < 16) {
          const v2u w = load_at<v2u>(p, val_at);
          val[u][i] = v4u{w[0], w[1], 0u, 0u};
        } else {
          val[u][i] = load_at<v4u>(p, val_at);
        }
      }
  };

  int t0 = begin + (kTeam == 1 ? 0 : wave * S::kTile);
  if (t0 < end) {
    load_pages(t0 >> c.log_page);
    load_keys(t0);
    load_values();
  }
  for (; t0 < end; t0 += kTeam * S::kTile) {
    const int next = t0 + kTeam * S::kTile;
    // Logits, without the scale.
    float l[S::kBlocks][4];
    v4u vscale[(S::kBlocks + 1) / 2];  // INT4: the tile's value scales, two to a dword
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
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if constexpr (kInt4)
          l[u][r] = __builtin_fmaf(
              s[r], (float)__builtin_bit_cast(v2h, (uint32_t)ks[u][r / 2])[r & 1], 0.0f);
        else
          l[u][r] = s[r];
      }
      if constexpr (kInt4) {
        vscale[u / 2][2 * (u & 1)] = vs[u][0];
        vscale[u / 2][2 * (u & 1) + 1] = vs[u][1];
      }
    }
    // Slots that take no part: a logit of -inf, a value scale of 0 (whatever was there).
    bool live[S::kBlocks * 4];
    if (kMask || t0 + S::kTile > end) {
      uint64_t in_tile = end - t0 >= 64 ? ~0ull : (1ull << (end - t0)) - 1;  // bit: slot t0 + it
      if constexpr (kMask) in_tile &= __ballot(mask != 0);
      const uint64_t mine = in_tile >> (4 * quarter);
#pragma unroll
      for (int u = 0; u < S::kBlocks; ++u)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const bool in = mine >> (16 * u + r) & 1;
          live[4 * u + r] = in;
          l[u][r] = in ? l[u][r] : -INFINITY;
        }
      if constexpr (kInt4) {
#pragma unroll
        for (int u = 0; u < S::kBlocks / 2; ++u)
          vscale[u] = mask_halves(vscale[u], &live[8 * u]);
      }
    }
    if (logits) {
#pragma unroll
      for (int u = 0; u < S::kBlocks; ++u)
        if (t0 + 16 * u + 4 * quarter < end)
          *reinterpret_cast<float4*>(logits + t0 + 16 * u) =
              make_float4(l[u][0] * scale, l[u][1] * scale, l[u][2] * scale, l[u][3] * scale);
    }
    if (next < end) load_keys(next);

    // The running maximum of the column, over the quarters too.
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < S::kBlocks; ++u)
      top = larger(larger(larger(larger(top, l[u][0]), l[u][1]), l[u][2]), l[u][3]);
    bool fresh = false;  // INT4: m is to be set from the products
    if (__any(top * scale > m + (kInt4 ? kFar : kRoom))) {
      top = column_max(top) * scale;
      float up = fmaxf(m, top - kLift);
      if constexpr (kInt4) {
        fresh = top > m + kFar;
        up = fresh ? top : m;
      }
      const float shrink = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - up);
      m = up;
      sum *= shrink;
      rounded *= shrink;
#pragma unroll
      for (int j = 0; j < S::kOut; ++j) o[j] *= shrink;
    }
    const float base = m == -INFINITY ? 0.0f : m;
    _Float16 p[S::kBlocks * 4];
    float most = 0.0f;  // INT4: the lane's largest product
#pragma unroll
    for (int u = 0; u < S::kBlocks; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(l[u][r], scale, -base));
        sum += x;
        if constexpr (kInt4) {  // as a mixed fma, which takes the float16 factor as it is
          l[u][r] = __builtin_fmaf(
              x, (float)__builtin_bit_cast(v8h, vscale[u / 2])[4 * (u & 1) + r], 0.0f);
          most = larger(most, l[u][r]);
        } else {
          p[4 * u + r] = (_Float16)x;
        }
      }
    if constexpr (kInt4) {
      if (__any(fresh || most > 0x1p15f)) {
        const float all = column_max(most);
        int e = 0;
        if (fresh || all > 0x1p15f)
          e = all > 0.0f ? max(__builtin_amdgcn_frexp_expf(all) - kLift, -kDeepest) : -kDeepest;
        const float turn = __builtin_amdgcn_ldexpf(1.0f, -e);
        m += (float)e;
        sum *= turn;
#pragma unroll
        for (int j = 0; j < S::kOut; ++j) o[j] *= turn;
#pragma unroll
        for (int u = 0; u < S::kBlocks; ++u)
#pragma unroll
          for (int r = 0; r < 4; ++r) l[u][r] *= turn;
      }
#pragma unroll
      for (int u = 0; u < S::kBlocks; ++u)
#pragma unroll
        for (int r = 0; r < 4; ++r) p[4 * u + r] = (_Float16)l[u][r];
    }

    if constexpr (!kInt4) {
#pragma unroll
      for (int i = 0; i < S::kBlocks * 2; ++i)
        rounded = __builtin_amdgcn_fdot2(v2h{p[2 * i], p[2 * i + 1]},
                                         v2h{(_Float16)1.0f, (_Float16)1.0f}, rounded, false);
    }

    // Values through LDS; the wave's own tile, so no barrier. Rows past the end: 0 times what they
    // hold might not be 0 (INT4 codes are always finite).
    if (!kInt4 && t0 + S::kTile > end) {
#pragma unroll
      for (int u = 0; u < S::kBlocks; ++u)
#pragma unroll
        for (int i = 0; i < S::kPieces; ++i)
          if (t0 + 16 * u + i * kRowsPerLoad + lane / kPerRow >= end) val[u][i] = v4u{};
    }
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
    if (next < end) load_values();
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
#pragma unroll
        for (int h = 0; h < 2; ++h)
          o[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
              eight_codes((uint32_t)w[h]),
              v8h{p[8 * h], p[8 * h + 1], p[8 * h + 2], p[8 * h + 3], p[8 * h + 4], p[8 * h + 5],
                  p[8 * h + 6], p[8 * h + 7]},
              o[j], 0, 0, 0);
      } else {
        // Lanes 4 r .. 4 r + 3 of a quarter name row r: 16 channels of 4 slots.
        v4s w[S::kBlocks];
#pragma unroll
        for (int u = 0; u < S::kBlocks; ++u) {
          const int t = 16 * u + 4 * quarter + (col >> 2);
          w[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (lds_v4s)(tile + S::at(t, 2 * j + ((col & 3) >> 1)) + 8 * (col & 1)));
          if constexpr (kMask) w[u] = mask_halves(w[u], &live[4 * u]);  // 0 times what it holds
        }
        if constexpr (S::kBlocks == 2)
          o[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
              __builtin_bit_cast(v8h,
                                 __builtin_shufflevector(w[0], w[1], 0, 1, 2, 3, 4, 5, 6, 7)),
              v8h{p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7]}, o[j], 0, 0, 0);
        else
          o[j] = __builtin_amdgcn_mfma_f32_16x16x16f16(
              __builtin_bit_cast(v4h, w[0]), v4h{p[0], p[1], p[2], p[3]}, o[j], 0, 0, 0);
      }
    }
    __builtin_amdgcn_wave_barrier();
  }

  // The waves' sums meet in LDS. Float16 values: o is put in proportion to sum from the sum of the
  // rounded p, so that what rounding did to a weight it also did to the sum that divides it (one
  // weight that outgrows all others is then exact).
  sum += __shfl_xor(sum, 16);
  sum += __shfl_xor(sum, 32);
  float unit_o = 1.0f;
  if constexpr (!kInt4) {
    rounded += __shfl_xor(rounded, 16);
    rounded += __shfl_xor(rounded, 32);
    unit_o = rounded != 0.0f ? sum / rounded : 0.0f;
  }
  if constexpr (kTeam == 1) {
    unit_o = sum != 0.0f ? unit_o / sum : 0.0f;  // (NaN where the sum is)
    if (col < rows) {
      const size_t bh = (size_t)b * a.heads + head0 + col;
#pragma unroll
      for (int j = 0; j < S::kOut; ++j) {
        const v4f x = o[j] * unit_o;
        *reinterpret_cast<v4h*>(a.out + bh * D + 16 * j + 4 * quarter) =
            v4h{(_Float16)x[0], (_Float16)x[1], (_Float16)x[2], (_Float16)x[3]};
      }
      if (quarter == 0) {
        if (a.lse) a.lse[bh] = log_sum(m, sum);
        if (plan.stats)
          plan.stats[(size_t)piece.index * a.heads + head0 + col] = make_float2(m, sum);
      }
    }
    if (plan.adds_weights) {
      if (quarter == 0) row_stats[wave][col] = weight_row(m, sum);
      __threadfence_block();  // other lanes' logits and rows
      const float* of = plan.logits + ((size_t)b * a.heads + head0) * plan.ld_logits;
      for (int s = 4 * lane; s < n; s += 256)
        add_slots(a.weights + ((size_t)b * c.heads + hk) * c.capacity(), s, n,
                  slot_weights(of + s, plan.ld_logits, rows,
                               [&](int g) { return row_stats[wave][g]; }));
    }
    return;
  }
  if (quarter == 0) wave_stats[wave][col] = make_float2(m, sum);
  __syncthreads();
  float top = -INFINITY, total = 0.0f;  // of the column, over the waves
#pragma unroll
  for (int w = 0; w < kTeam; ++w) top = fmaxf(top, wave_stats[w][col].x);
  const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
  for (int w = 0; w < kTeam; ++w)
    total += wave_stats[w][col].y * __builtin_amdgcn_exp2f(wave_stats[w][col].x - base);
  unit_o *= __builtin_amdgcn_exp2f(m - base);
  if (whole) unit_o = total != 0.0f ? unit_o / total : 0.0f;
  float* mine = reinterpret_cast<float*>(tile);
#pragma unroll
  for (int j = 0; j < S::kOut; ++j)
    *reinterpret_cast<v4f*>(mine + col * S::kLdO + 16 * j + 4 * quarter) = o[j] * unit_o;
  if (wave == 0 && quarter == 0)  // rows, for the weights
    row_stats[0][col] = weight_row(top, total);
  if (threadIdx.x < rows) {
    const size_t bh = (size_t)b * a.heads + head0 + threadIdx.x;
    if (whole && a.lse) a.lse[bh] = log_sum(top, total);
    if (plan.stats)
      plan.stats[(size_t)piece.index * a.heads + head0 + threadIdx.x] = make_float2(top, total);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < rows * (D / 4); i += kThreads) {
    const int r = i / (D / 4), d = 4 * (i % (D / 4));
    v4f acc = {};
#pragma unroll
    for (int w = 0; w < kTeam; ++w)
      acc += *reinterpret_cast<const v4f*>(reinterpret_cast<const float*>(lds + w * kLds) +
                                           r * S::kLdO + d);
    const size_t bh = (size_t)b * a.heads + head0 + r;
    if (whole)
      *reinterpret_cast<v4h*>(a.out + bh * D + d) =
          v4h{(_Float16)acc[0], (_Float16)acc[1], (_Float16)acc[2], (_Float16)acc[3]};
    else
      *reinterpret_cast<v4f*>(plan.part +
                              ((size_t)piece.index * a.heads + head0 + r) * D + d) = acc;
  }
  if (plan.adds_weights) {
    const float* of = plan.logits + ((size_t)b * a.heads + head0) * plan.ld_logits;
    for (int s = 4 * threadIdx.x; s < n; s += 4 * kThreads)
      add_slots(a.weights + ((size_t)b * c.heads + hk) * c.capacity(), s, n,
                slot_weights(of + s, plan.ld_logits, rows, [&](int g) { return row_stats[0][g]; }));
  }
}

// The common maximum of a head's pieces and the sum relative to it, by `lanes` neighbouring lanes
// of a wave (a power of two). stats: the head's first piece; `heads` apart.
__device__ __forceinline__ float2 join_stats(const float2* stats, int count, int heads,
                                             int lanes) {
  const int lane = threadIdx.x & (lanes - 1);
  float top = -INFINITY, total = 0.0f;
#pragma unroll 4
  for (int i = lane; i < count; i += lanes) top = fmaxf(top, stats[(size_t)i * heads].x);
  for (int d = lanes / 2; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll 4
  for (int i = lane; i < count; i += lanes) {
    const float2 st = stats[(size_t)i * heads];
    total += st.y * __builtin_amdgcn_exp2f(st.x - base);
  }
  for (int d = lanes / 2; d > 0; d >>= 1) total += __shfl_xor(total, d);
  return make_float2(top, total);
}

// The first `joins` workgroups join the pieces of one head each (of sequences of more than one
// piece); the others turn the logits of 1024 slots of a (sequence, KV head) into weights.
template <int D>
__global__ void __launch_bounds__(kThreads)
    attention_join_kernel(AttentionArgs a, KvView c, Plan plan, int joins, int weight_blocks) {
  constexpr int kParts = kThreads / (D / 4);  // pieces read at a time, 4 channels per thread
  __shared__ float4 acc_of[kThreads];
  __shared__ float2 of_row[kThreads];
  if ((int)blockIdx.x < joins) {
    const int bh = blockIdx.x, b = bh / a.heads, h = bh % a.heads;
    const int2 at = plan.of_seq[b];  // first piece, pieces
    if (at.y == 1) return;
    const float2* stats = plan.stats + (size_t)at.x * a.heads + h;
    const int d4 = threadIdx.x % (D / 4), part = threadIdx.x / (D / 4);
    const float4* src =
        reinterpret_cast<const float4*>(plan.part + ((size_t)at.x * a.heads + h) * D) + d4;
    const size_t stride = (size_t)a.heads * (D / 4);
    // The thread's first pieces are on their way while the stats are joined.
    constexpr int kAhead = 4;
    float4 ahead[kAhead];
    float2 own[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int i = min(part + k * kParts, at.y - 1);
      ahead[k] = src[i * stride];
      own[k] = stats[(size_t)i * a.heads];
    }
    const float2 all = join_stats(stats, at.y, a.heads, 64);
    float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    const float base = all.x == -INFINITY ? 0.0f : all.x;
    const auto add = [&](float m, const float4& x) {
      const float f = __builtin_amdgcn_exp2f(m - base);  // 0 for a piece without slots
      acc.x += f * x.x;
      acc.y += f * x.y;
      acc.z += f * x.z;
      acc.w += f * x.w;
    };
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (part + k * kParts < at.y) add(own[k].x, ahead[k]);
#pragma unroll 4
    for (int i = part + kAhead * kParts; i < at.y; i += kParts)
      add(stats[(size_t)i * a.heads].x, src[i * stride]);
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
    const bool some = all.y != 0.0f;
    const float v[4] = {acc.x, acc.y, acc.z, acc.w};
    v4h y;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = (_Float16)(some ? v[i] / all.y : 0.0f);
    *reinterpret_cast<v4h*>(a.out + (size_t)bh * D + 4 * d4) = y;
    if (d4 == 0 && a.lse) a.lse[bh] = log_sum(all.x, all.y);
    return;
  }
  const int id = blockIdx.x - joins;
  const int unit = id / weight_blocks, b = unit / c.heads, hk = unit % c.heads;
  const int n = min(a.lengths[b], a.max_length);
  const int s0 = id % weight_blocks * (4 * kThreads);
  if (s0 >= n) return;
  const int2 at = plan.of_seq[b];
  const int s = s0 + 4 * threadIdx.x;
  float4 w = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  for (int g0 = 0; g0 < plan.group; g0 += kThreads) {
    const int heads = min(plan.group - g0, kThreads);
    const size_t bh0 = (size_t)b * a.heads + hk * plan.group + g0;
    __syncthreads();
    // All heads at once, as many lanes to each as there are: by whole waves in turn, 40 heads took
    // 20 us.
    int lanes = 64;
    while (lanes > 1 && lanes * heads > kThreads) lanes >>= 1;
    for (int g = threadIdx.x / lanes; g < heads; g += kThreads / lanes) {
      const float2 all = join_stats(
          plan.stats + (size_t)at.x * a.heads + hk * plan.group + g0 + g, at.y, a.heads, lanes);
      of_row[g] = weight_row(all.x, all.y);
    }
    __syncthreads();
    if (s < n) {
      const float4 x = slot_weights(plan.logits + bh0 * plan.ld_logits + s, plan.ld_logits, heads,
                                    [&](int g) { return of_row[g]; });
      w.x += x.x;
      w.y += x.y;
      w.z += x.z;
      w.w += x.w;
    }
  }
  if (s < n) add_slots(a.weights + (size_t)unit * c.capacity(), s, n, w);
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Pieces of the sequences, in numbers that a launch may reach.
long long max_pieces(const Plan& p, const KvView& c, int max_length) {
  if (p.target == 0) return (long long)c.sequences * p.pieces;
  const long long steps = (max_length - 1) / p.step + 1;
  const long long most = (long long)c.sequences * ((steps - 1) / p.steps + 1);
  const long long share = (long long)c.heads * p.row_blocks;
  const long long want = p.target > share ? p.target / share : 1;
  return most < want + c.sequences ? most : want + c.sequences;
}

Plan make_plan(const KvView& c, int heads, int max_length, bool with_weights, void* workspace,
               size_t* bytes) {
  Plan p{};
  p.group = heads / c.heads;
  p.row_blocks = (p.group + kRows - 1) / kRows;
  const long long share = (long long)c.heads * p.row_blocks;
  p.step = kWaves * (c.int4() ? 64 : c.dim == 256 ? 16 : 32);
  // Workgroups that run at the same time where cutting every sequence gives no more; else four
  // times as many, not too short, so that those that end last are a small part of the whole.
  const int resident = 256 * (c.dim == 256 ? 2 : 3);
  const bool one_round = c.sequences * share <= resident;
  p.target = one_round ? resident : 4 * resident;
  p.steps = one_round ? 2 : 8;
  const long long steps = (max_length - 1) / p.step + 1;
  // Sequences of a few steps stay whole, which spares them the second launch (17 x 3 KV heads
  // of 128, float16: 4 steps 8.6 against 11.1 us in two pieces, 6 steps 10.9 against 11.2, 8 steps 14.4
  // against 11.5; INT4, whose steps are longer, 10.5 against 11.8 at 4 and 13.7 against 11.8 at
  // 6); of up to 8 where whole ones already fill the card (60 x 8, 8 steps: 29 against 32 us).
  const long long units = c.sequences * share;
  if (steps <= (units >= 256 ? 8 : c.int4() ? 4 : 6)) p.steps = (int)steps;
  if (c.sequences > kWidest || steps <= p.steps) {  // many balance each other; or nothing to cut
    p.target = 0;
    long long q = steps * c.sequences * share / (4 * resident);
    q = q < p.steps ? p.steps : q;
    p.steps = (int)(q < steps ? q : steps);
    p.pieces = (int)((steps - 1) / p.steps + 1);
  }
  // Short sequences in more than one round of workgroups: a wave each, which saves the meeting of
  // the four. 250 x 32 heads of 30 slots, INT4, dim 64: 31.5 -> 14.3 us; 200 x 64 of 64,
  // float16: 77 -> 52 us. Longer ones gain from it with INT4 alone, which computes more per byte
  // (250 x 32 of 300: 66 -> 49 us; float16, of 250, 103 -> 108), or within one round not at all
  // (60 x 8 of 200, INT4: 7.3 -> 10.3 us).
  const long long team_steps = c.int4() && units > 4 * resident ? 2 : 1;
  p.team = p.pieces == 1 && units > resident && steps <= team_steps ? 1 : kWaves;
  p.ld_logits = (max_length + 15) & ~15;
  const size_t pieces = (size_t)max_pieces(p, c, max_length);
  const bool joined = pieces > (size_t)c.sequences;
  p.adds_weights = with_weights && !joined && p.target == 0 && p.row_blocks == 1;
  const bool second = joined || (with_weights && !p.adds_weights);  // a second launch
  const size_t of_seq = second ? align256((size_t)c.sequences * 8) : 0;
  const size_t stats = second ? align256(pieces * heads * 8) : 0;
  const size_t part = joined ? align256(pieces * heads * c.dim * 4) : 0;
  const size_t logits =
      with_weights ? align256((size_t)c.sequences * heads * (size_t)p.ld_logits * 4) : 0;
  *bytes = of_seq + stats + part + logits;
  if (uint8_t* ws = static_cast<uint8_t*>(workspace)) {
    if (of_seq) p.of_seq = reinterpret_cast<int2*>(ws);
    if (stats) p.stats = reinterpret_cast<float2*>(ws + of_seq);
    if (part) p.part = reinterpret_cast<float*>(ws + of_seq + stats);
    if (logits) p.logits = reinterpret_cast<float*>(ws + of_seq + stats + part);
  }
  return p;
}

// Workgroups of the first launch.
long long first_grid(const Plan& p, const KvView& c, int max_length) {
  const long long units = max_pieces(p, c, max_length) * c.heads;
  const long long grid = p.row_blocks == 1 ? units : (units + 7) / 8 * 8 * p.row_blocks;
  return p.team == 1 ? (grid + kWaves - 1) / kWaves : grid;
}

// Of the second those that join, and those per (sequence, KV head) that add the weights.
struct Second {
  int joins, blocks;
  long long grid;
};
Second second_grid(const Plan& p, const KvView& c, int heads, int max_length, bool with_weights) {
  Second s;
  s.joins = max_pieces(p, c, max_length) > c.sequences ? c.sequences * heads : 0;
  s.blocks = with_weights && !p.adds_weights ? (max_length - 1) / (4 * kThreads) + 1 : 0;
  s.grid = s.joins + (long long)s.blocks * c.sequences * c.heads;
  return s;
}

template <int D>
hipError_t launch(const AttentionArgs& a, const KvView& c, const Plan& p, hipStream_t stream) {
  const long long grid = first_grid(p, c, a.max_length);
  const auto run = [&](auto kernel) { kernel<<<(unsigned)grid, kThreads, 0, stream>>>(a, c, p); };
  if (p.team == 1) {
    if (c.int4())
      a.mask ? run(attention_kernel<D, true, true, 1>) : run(attention_kernel<D, true, false, 1>);
    else
      a.mask ? run(attention_kernel<D, false, true, 1>) : run(attention_kernel<D, false, false, 1>);
  } else {
    if (c.int4())
      a.mask ? run(attention_kernel<D, true, true, kWaves>)
             : run(attention_kernel<D, true, false, kWaves>);
    else
      a.mask ? run(attention_kernel<D, false, true, kWaves>)
             : run(attention_kernel<D, false, false, kWaves>);
  }
  if (hipError_t e = hipGetLastError()) return e;
  const Second s = second_grid(p, c, a.heads, a.max_length, a.weights != nullptr);
  if (s.grid > 0)
    attention_join_kernel<D><<<(unsigned)s.grid, kThreads, 0, stream>>>(a, c, p, s.joins, s.blocks);
  return hipGetLastError();
}

}  // namespace

bool attention_fits(const KvView& c, int heads, int max_length, bool with_weights) {
  size_t bytes;
  const Plan p = make_plan(c, heads, max_length, with_weights, nullptr, &bytes);
  return fits_grid(first_grid(p, c, max_length), kThreads) &&
         fits_grid(second_grid(p, c, heads, max_length, with_weights).grid, kThreads);
}

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
