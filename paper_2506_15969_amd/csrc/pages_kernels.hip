// Attention of tokens that share a context over its pages (lazyev_pages_attend): the rows of a unit (table row and KV
// head) are its tokens' query heads, token by token, and every row goes over the same entries.
//
// A wave keeps 32 rows: their queries, their output O^T (fp32) and, per row, a reference m and the sum l of the weights
// relative to it, exp2(s log2 e - m).  Entries come in stages of kKeys, fetched straight into LDS by the whole block while the
// stage before is worked on, by page numbers that the block keeps in LDS, kWindow at a time.  Of a stage each of the kWK waves that
// share 32 rows takes its own kKeys / kWK entries, 32 at a time:
//   S^T = K Q^T    v_mfma_f32_32x32x16_bf16 (fp32 rows: 32x32x2_f32): lane (c, h) = (l % 32, l / 32) holds, of row c, the
//                  logits of the entries 8 i + 4 h + j (i, j < 4)
//   P = exp2(S)    in place; for the product with bf16 values rounded to bf16 (128 x bf16: half a step, 2^-8, of each weight) or taken as two bf16 terms
//                  (64 x bf16: 2^-16), see kTerms; the sum l is that of the weights before, as it also is a result of its own
//   O^T += V^T P^T lane (c, h) already holds 8 entries of row c, in an order that the products take from V as well: V
//                  is read transposed (ds_read_b64_tr_b16), 4 entries of 16 columns to 16 lanes
// The reference is raised only when a lane's sum of weights relative to it in a stage (16 or, with 64 entries of a stage to a wave, 32 of
// them) exceeds 2^12 (never rescaled otherwise): a sum is as exact relative to any reference in the range of fp32, and with weights of 2^8 on average at
// most over 2^30 entries values of up to 2^89 stay in it.  Every decision that changes a row's arithmetic
// is taken for that row alone: what other rows see has no influence on it.  (But for tiles of tokens with lists of their own, see kPerTile: the lists of
// the others say which stage and split an entry of the joined list is in, and so move the roundings of a row's sums.)
// Entries that a row does not see (or that lead to no page) are masked to weight zero, which leaves a NaN of the output where V
// holds an infinity or NaN, as a weight's second term does.  A block that masked something, or has second terms, and ends up with such an output starts
// over, with those taken out of V in the stages where it masks (all of them); the rows that do see one get it at the end.
//
// Few rows: the entries are also cut into splits, which leave (m, l, O) in the workspace for a second kernel.
//
// Bound by memory where few rows read many entries: 80 rows over 100003 entries of each of 8 KV heads, 128 x bf16 (410 MB), 79 us, 5.2
// TB/s, the rate of a copy of 1 GiB.  Bound by the products and the vector instructions beside them where many do: 4096 tokens of 40 / 8 heads over
// their past (172 GFLOP) 193 - 198 us in a loop of passes, 870 - 890 TFLOP/s, against 1213 - 1358 of a bf16 product of 8192^3 on the same card.  By counters
// the matrix cores are busy in 45 % of the cycles (73 % in that product), vector instructions are issued in 44 %: together most of the time, as
// where the two waves of a SIMD seldom do both at once.  The clock is 2.24 GHz meanwhile, of 2.4, and 1.97 in the product, so power is not what binds (order and depth
// of the operands' reads, wave priorities and a third stage on its way change nothing).  Bound by its own length where both are
// few: one token's 28 heads over 8192 entries 13.3 us, of which the second launch 5.5, the products 1.3 and the entries' arrival 1.0.
#include "kernels.h"
#include "lazyev.h"
#include "rows.h"

#include <cfloat>
#include <climits>
#include <type_traits>

namespace lazyev {
namespace {

typedef unsigned short bf16_t;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(2))) float f32x2_t;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4_t;
typedef __attribute__((ext_vector_type(2))) unsigned u32x2_t;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kFar = 0x1p12f;         // a sum of weights beyond this raises the reference
constexpr float kHuge = 0x1p24f;        // of references beyond this the rounding exceeds 1 (see exponent_of)
constexpr int kSplitMax = 128;

template <typename T, int D>
struct Rows {
  static constexpr bool kF32 = sizeof(T) == 4;
  static constexpr int kChunks = D * static_cast<int>(sizeof(T)) / 16;   // 16-byte chunks of a row
  static constexpr int kOps = kChunks / 2;         // chunks of a row that a lane holds as an operand
  static constexpr int kTiles = D / 32;            // output tiles of 32 columns
  // Terms of a weight in the product with V.  128 x bf16 weights are rounded, as the decode step rounds them: two terms take a third longer where
  // products bind (4096 tokens of 40 / 8 heads over their past 207 -> 269 us, 80 rows over 100003 entries 81 -> 99) and lower the error against 64 bits from 0.0020 - 0.0022
  // to the 0.0016 - 0.0017 of the output's own rounding.  Listed entries the same: one token each of 16 sequences over 64 blocks of 32 of 8 KV heads 30.5 -> 31.5 us, 640
  // tokens of 28 / 4 heads over 32 of 512 blocks 128 -> 154 (weights kept in fp32 until they are needed; both terms at once 157, with registers spilled), error 0.0023 -> 0.0017.
  // 64 x bf16 rows the decode step keeps exact with three terms; two are as far below that rounding
  // here (the same calls with one / two / three terms 142 / 183 / 219 us, 52 / 56 - 61 / 71; 224 rows over 8192 entries 16.2 / 17.3 / 18.2).
  static constexpr int kTerms = kF32 || D == 128 ? 1 : 2;
  // Where chunk x of entry r of a stage lies among the entry's chunks: keys are read by 16 entries at a time, one chunk of
  // each; values by 4 (bf16) entries, 64 bytes of each, or (fp32) an entry and the one four further, 128 bytes of each.
  __device__ static int k_slot(int r, int x) { return x ^ (kChunks == 8 ? (r >> 1) & 7 : r & 15); }
  __device__ static int v_slot(int r, int x) { return x ^ (kF32 ? ((r >> 2) & 1) * 8 : kChunks == 8 ? ((r >> 1) & 1) * 4 : (r & 3) * 4); }
};

__device__ __forceinline__ unsigned pair_to_bf16(float lo, float hi) {
  return __builtin_bit_cast(unsigned, __builtin_convertvector(f32x2_t{lo, hi}, bf16x2_t));
}
__device__ __forceinline__ float bf16_low(unsigned w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(unsigned w) { return __uint_as_float(w & 0xFFFF0000u); }

// x of lane ^ 32 joined with x
__device__ __forceinline__ float max_of_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_of_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// What a row found in the pages (reference m in units of log 2, sum l relative to it; l = 0: nothing) and elsewhere:
// the factors of the pages' unnormalised output and of the other one, and the log-sum-exp over both.
struct Joined { float pages, other, lse; };
__device__ __forceinline__ Joined join(float m, float l, float lse_other) {
  const bool some = !(l <= 0.f);                   // (a NaN is something)
  const float lse = some ? fmaf(m, kLn2, logf(l)) : -INFINITY;
  Joined j;
  if (lse_other == -INFINITY) {
    j.pages = some ? 1.f / l : 0.f;
    j.other = 0.f;
    j.lse = lse;
    return j;
  }
  const float top = fmaxf(lse, lse_other);
  const float a = expf(lse - top), b = expf(lse_other - top);
  j.pages = some ? a / ((a + b) * l) : 0.f;
  j.other = b / (a + b);
  j.lse = top + logf(a + b);
  return j;
}

__device__ __forceinline__ bool takes_part(const AttendArgs &a, int token) {
  if (!a.slots.prompt_len) return true;
  return a.slots.prompt_len[token] >= 0 && a.t - a.slots.t0[token] >= 1;
}

// A row as the caller sees it.
struct RowPlace {
  int token;                        // of all sequences
  int head, kvh;                    // head: within the KV head's group
  long long row;                    // token * n_q_heads + query head
};
__device__ __forceinline__ RowPlace row_place(const AttendArgs &a, int unit, int r) {
  RowPlace p;
  const int seq = a.n_seqs == 1 ? 0 : unit / a.n_kv_heads, i = quotient(r, a.group);
  p.kvh = unit - seq * a.n_kv_heads;
  p.head = r - i * a.group;
  p.token = seq * a.n_tokens + i;
  p.row = static_cast<long long>(p.token) * a.n_q_heads + p.kvh * a.group + p.head;
  return p;
}

// Rows of tiles of tokens (see kPerTile): a place that row_place gave by the tile made that among all tokens; rows of the tile, of which a
// table row's last one may have fewer.
__device__ __forceinline__ int tile_token0(const AttendArgs &a, int tile, int &table_row) {
  table_row = tile / a.list.tiles;
  return (tile - table_row * a.list.tiles) * a.n_tokens;
}
__device__ __forceinline__ int tile_rows(const AttendArgs &a, int token0) { return min(a.n_tokens, a.list.tokens - token0) * a.group; }
__device__ __forceinline__ void place_in_tile(const AttendArgs &a, int tile, int table_row, int token0, RowPlace &p) {
  p.token += table_row * a.list.tokens + token0 - tile * a.n_tokens;
  p.row = static_cast<long long>(p.token) * a.n_q_heads + p.kvh * a.group + p.head;
}

// Four output elements of a row (columns e0 .. e0 + 3) joined with the other part and stored.
template <typename T, int D>
__device__ __forceinline__ void finish4(const AttendArgs &a, const RowPlace &p, int e0, f32x4_t o, const Joined &j) {
  T *to = static_cast<T *>(a.out) + p.row * D + e0;
  f32x4_t x = o * j.pages;
  if (j.pages == 0.f) x = f32x4_t{0.f, 0.f, 0.f, 0.f};      // (whatever lies there when nothing was seen)
  if (j.other != 0.f) {
    const T *from = static_cast<const T *>(a.joined_out) + p.row * D + e0;
    f32x4_t y;
    if constexpr (sizeof(T) == 4) {
      if (a.wide) y = *reinterpret_cast<const f32x4_t *>(from);
      else y = f32x4_t{from[0], from[1], from[2], from[3]};
    } else {
      u32x2_t w;
      if (a.wide) w = *reinterpret_cast<const u32x2_t *>(from);
      else w = u32x2_t{from[0] | static_cast<unsigned>(from[1]) << 16, from[2] | static_cast<unsigned>(from[3]) << 16};
      y = f32x4_t{bf16_low(w[0]), bf16_high(w[0]), bf16_low(w[1]), bf16_high(w[1])};
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = fmaf(j.other, y[e], x[e]);
  }
  if constexpr (sizeof(T) == 4) {
    if (a.wide) *reinterpret_cast<f32x4_t *>(to) = x;
    else
#pragma unroll
      for (int e = 0; e < 4; ++e) to[e] = x[e];
  } else {
    const u32x2_t w = {pair_to_bf16(x[0], x[1]), pair_to_bf16(x[2], x[3])};
    if (a.wide) *reinterpret_cast<u32x2_t *>(to) = w;
    else
#pragma unroll
      for (int e = 0; e < 4; ++e) to[e] = static_cast<bf16_t>(w[e / 2] >> (16 * (e % 2)));
  }
}

// Log-sum-exp of what the row is joined with (nothing: -inf).
__device__ __forceinline__ float lse_joined(const AttendArgs &a, const RowPlace &p) {
  if (a.joined_stat) {
    const float *st = a.joined_stat + (static_cast<size_t>(p.token) * a.n_kv_heads + p.kvh) * 16 + 2 * p.head;
    return st[0] - logf(st[1]);
  }
  return a.joined_lse ? a.joined_lse[p.row] : -INFINITY;
}
// Once for a row; both may be what lse_joined reads (of two kernels the first reads, the second writes).
__device__ __forceinline__ void finish_row(const AttendArgs &a, const RowPlace &p, const Joined &j) {
  if (a.lse) a.lse[p.row] = j.lse;
  if (a.joined_stat) a.joined_stat[(static_cast<size_t>(p.token) * a.n_kv_heads + p.kvh) * 16 + 2 * p.head + 1] *= j.other;
}

// A weight's exponent relative to the reference m: a multiply-add is exact but for one rounding of its result; where m, which
// is a rounded product itself, is so large that the difference of the two could leave the range, the product is rounded as well.
__device__ __forceinline__ float exponent_of(float s, float c2, float m) {
  float x = s * c2;
  __asm__("" : "+v"(x));                           // (not fused)
  return fabsf(m) > kHuge ? x - m : fmaf(s, c2, -m);
}

// Elements whose exponents are all ones taken out of a chunk of V.
template <bool kF32>
__device__ __forceinline__ unsigned odd_bits(unsigned w) {             // the sign bits of those elements
  return kF32 ? ((w & 0x7F800000u) + 0x00800000u) & 0x80000000u : ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u;
}
template <bool kF32>
__device__ __forceinline__ bool take_out_odd(u32x4_t &w) {
  unsigned any = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const unsigned odd = odd_bits<kF32>(w[e]);
    any |= odd;
    w[e] &= ~(kF32 ? 0u - (odd >> 31) : (odd >> 15) * 0xFFFFu);
  }
  return any != 0;
}

// The order of the products of a basic block (kMfma for each of kN operands) and the reads of their operands from LDS (kReads each):
// kDepth operands are on their way while one is multiplied.
template <int kN, int kMfma, int kReads, int kDepth>
__device__ __forceinline__ void ahead() {
  constexpr int kFirst = kDepth < kN ? kDepth : kN;
  __builtin_amdgcn_sched_group_barrier(0x100, kFirst * kReads, 0);
#pragma unroll
  for (int i = 0; i < kN - kFirst; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, kMfma, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, kReads, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, kFirst * kMfma, 0);
}

// kWR x kWK waves: kWR of 32 rows each, kWK that share the entries of a stage.
template <typename T, int D, int kWR, int kWK, int kKeys>
struct Shape {
  using R = Rows<T, D>;
  static constexpr int kWaves = kWR * kWK, kBlock = 64 * kWaves;
  static constexpr int kSub = kKeys / kWK / 32;    // sub-tiles of 32 entries that a wave takes of a stage
  static constexpr int kPerLoad = 64 / R::kChunks; // entries that a wave's load of 16 bytes a lane brings
  static constexpr int kLoads = kKeys / (kPerLoad * kWaves);   // of K and of V each, per wave and stage
  static_assert(kSub >= 1 && kLoads >= 1 && kLoads * kPerLoad * kWaves == kKeys, "whole loads");
  static constexpr int kPerSimd = D * sizeof(T) == 512 ? 1 : 2;   // (fp32 rows of 128: queries and output take 128 registers, the products' operands more)
  static constexpr int kWindow = 512;              // page numbers that a block keeps in LDS
  static constexpr int kHalf = kKeys * D * static_cast<int>(sizeof(T)), kStage = 2 * kHalf;   // bytes of a stage: of K, then of V
};

// Entries of listed blocks: entry x of the list is entry x % block of block list[x / block].  What a table of pages says of the others, the
// window says of runs of 1 << run_shift entries, which lie next to one another in a block and in a page: the row of the first one, and
//   kPerToken  (a unit is a token of a sequence and a KV head) how many of them the token sees; those beyond are holes, as pages that are none
//   kPerTile   (a unit is a tile of tokens and a KV head, the list one of pairs: a block that some of them read, and a bit for each that does)
//              the number of the first one in the table's row and the tokens' bits, by which every row is masked
enum Lists { kNoList, kPerToken, kPerTile };
constexpr int kNowhere = 1 << 30;       // beyond any entry that a token sees
template <typename T, int D, int kWR, int kWK, int kKeys, int kLists = kNoList>
__global__ __launch_bounds__(64 * kWR * kWK, (Shape<T, D, kWR, kWK, kKeys>::kPerSimd)) void attend_kernel(const AttendArgs a) {
  using R = Rows<T, D>;
  using S = Shape<T, D, kWR, kWK, kKeys>;
  constexpr int kSub = S::kSub, kOps = R::kOps, kTiles = R::kTiles, C = R::kChunks;
  constexpr bool kListed = kLists != kNoList, kPairs = kLists == kPerTile;
  constexpr int kWindow = kPairs ? S::kBlock : S::kWindow;   // (kPerTile: fewer registers on the way)
  __shared__ __align__(16) char stages[2 * S::kStage];
  __shared__ int window[kWindow];
  __shared__ float shared_ml[kWK][kWR][64];
  __shared__ int shared_most[S::kWaves], shared_least[S::kWaves], shared_hole[2], shared_odd;
  // of a run (kPerToken) entries that the token sees; (kPerTile) the first one's number, and the tokens' bits
  __shared__ int window_seen[kListed ? kWindow : 1], stage_seen[2][kListed ? kKeys : 1];
  __shared__ unsigned window_bits[kPairs ? kWindow : 1], stage_bits[2][kPairs ? kKeys : 1];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 31, h = lane >> 5;
  const int wr = wave % kWR, wk = wave / kWR;
  int M = a.n_tokens * a.group;
  // (blocks of one unit, split and so on are as far from one another as there are units: those of eight units, or four, share
  // an XCD and its L2.)  Late rows first: where a token sees its past only, they have the most to do
  const int unit = static_cast<int>(blockIdx.x), split = static_cast<int>(blockIdx.y), span = static_cast<int>(gridDim.z - 1 - blockIdx.z);
  const int seq = a.n_seqs == 1 ? 0 : unit / a.n_kv_heads, kvh = unit - seq * a.n_kv_heads;
  const int r0 = (span * kWR + wr) * 32;           // this wave's rows
  // (kPerTile: the table's row, the tile of its tokens, of which the last may be smaller, and the entries of the list)
  int table_row = kLists == kPerToken ? seq / a.list.tokens : seq, token0 = 0;
  if constexpr (kPairs) {
    token0 = tile_token0(a, seq, table_row);
    M = tile_rows(a, token0);
  }
  const bool have = r0 < M;
  RowPlace place = row_place(a, unit, min(r0 + c, M - 1));
  const int my_token = place.token - seq * a.n_tokens;       // of the tile
  if constexpr (kPairs) place_in_tile(a, seq, table_row, token0, place);
  const int length = kPairs ? a.list.counts[unit] << a.list.block_shift : a.length;

  // entries of this block: first .. last - 1
  // (kPerTile: lists are of lengths of their own, each cut into a.n_split parts)
  const int split_keys = kPairs ? ((length + kKeys - 1) / kKeys + a.n_split - 1) / a.n_split * kKeys : a.split_keys;
  const int first = kPairs ? min(split * split_keys, length) : split * split_keys, last = min(first + split_keys, length);
  const int32_t *table = a.pages.table + static_cast<long long>(table_row) * a.pages.stride;
  const int32_t *list = kLists == kPerToken ? a.list.list + static_cast<long long>(unit) * a.list.n_listed : nullptr;
  const int2 *pairs = kPairs ? a.list.pairs + static_cast<long long>(unit) * a.list.n_listed * a.n_tokens : nullptr;
  // (what the window goes by: a page, or a run)
  auto slot_of = [&](int entry) __attribute__((always_inline)) { return kListed ? entry >> a.list.run_shift : page_of(a.pages, entry); };
  // everything that is read before the first stage is worked on is asked for at once
  u32x4_t qb[kOps];
  {
    const T *q = static_cast<const T *>(a.q) + place.row * D + h * (16 / sizeof(T));
    if (a.wide) {
#pragma unroll
      for (int j = 0; j < kOps; ++j) qb[j] = *reinterpret_cast<const u32x4_t *>(q + j * (32 / sizeof(T)));
    } else {
#pragma unroll
      for (int j = 0; j < kOps; ++j) {
        T e[16 / sizeof(T)];
#pragma unroll
        for (int x = 0; x < static_cast<int>(16 / sizeof(T)); ++x) e[x] = q[j * (32 / sizeof(T)) + x];
        __builtin_memcpy(&qb[j], e, 16);
      }
    }
  }
  constexpr bool kLate = kPairs && kWK == 1;       // (nobody else of the block replaces it; fewer registers on the way)
  float lse_other = kLate ? 0.f : lse_joined(a, place);
  int seen = a.visible ? min(max(a.visible[place.token], 0), kListed ? a.list.entries : a.length) : kListed ? a.list.entries : a.length;
  const int reach = seen;                          // (kListed: entries of the table row that the row's token sees)
  if constexpr (kListed) seen = reach > 0 ? length : 0;

  // ---- stages on their way to LDS.  Loads go from memory to LDS, 1 KB a wave, in the order of the addresses there.  (Written out, as
  // the compiler has every read of LDS wait for all loads into it: they leave nothing in registers, and the waits for
  // them are in `arrived`.)
  const bool once = gridDim.z == 1 && (!kListed || a.list.tokens == 1);   // nobody else reads these entries (uniform): they need not stay in the caches
  const unsigned stages_at = static_cast<unsigned>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char *)stages));
  auto load_1k = [&](const char *from, unsigned to) __attribute__((always_inline)) {
    if (once) __asm__ volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off nt" ::"s"(to), "v"(from) : "memory", "m0");
    else __asm__ volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(from) : "memory", "m0");
  };
  const unsigned head_rows = static_cast<unsigned>(a.pages.page_size), page_rows = head_rows * static_cast<unsigned>(a.n_kv_heads);
  // The row of the pools that a run begins with, and of its entries those that are there and that the token sees, or (kPerTile) the first
  // one's number, beyond any that a token sees where they are not there, and the tokens' bits.
  auto run_at = [&](int slot, int &n, unsigned &bits) __attribute__((always_inline)) {
    const int shift = a.list.block_shift - a.list.run_shift, in_block = (slot & ((1 << shift) - 1)) << a.list.run_shift;
    const int limit = kPairs ? a.list.entries : reach;
    int b;
    if constexpr (kPairs) {
      const int2 pair = pairs[slot >> shift];
      b = pair.x;
      bits = static_cast<unsigned>(pair.y);
      n = kNowhere;
    } else {
      b = list[slot >> shift];
      n = 0;
    }
    if (b < 0 || b > (limit - 1) >> a.list.block_shift) return 0u;
    const int entry = (b << a.list.block_shift) + in_block;
    if (entry >= limit) return 0u;
    const int pg = page_of(a.pages, entry);
    const unsigned no = static_cast<unsigned>(table[pg]);
    if (no >= static_cast<unsigned>(a.pages.n_pages)) return 0u;
    n = kPairs ? entry : min(1 << a.list.run_shift, limit - entry);
    return no * page_rows + kvh * head_rows + static_cast<unsigned>(entry - pg * a.pages.page_size);
  };
  int window_at = slot_of(first);
  // Entries from e0 on, none beyond `limit`, to a stage's place; page numbers by number(page of the entry, load).  -> was one of them none?
  auto load_stage = [&](int e0, int limit, int buf, auto number) __attribute__((always_inline)) {
    bool hole = false;
#pragma unroll
    for (int u = 0; u < S::kLoads; ++u) {
      const int r = (u * S::kWaves + wave) * S::kPerLoad + lane / C;
      const int entry = min(e0 + r, limit), pg = slot_of(entry);
      unsigned no = static_cast<unsigned>(number(pg, u)), pool_row;
      if constexpr (kListed) {
        const int n = window_seen[pg - window_at], at = entry & ((1 << a.list.run_shift) - 1);
        if constexpr (kPairs) {                    // (every stage is masked; a run lies in one page as a whole)
          pool_row = n == kNowhere ? 0u : no + static_cast<unsigned>(at);
        } else {
          hole |= at >= n;
          pool_row = no + static_cast<unsigned>(max(min(at, n - 1), 0));
        }
      } else {
        if (no >= static_cast<unsigned>(a.pages.n_pages)) {   // no page: any row; its entries are masked
          hole = true;
          no = 0;
        }
        const unsigned in_page = kvh * head_rows + static_cast<unsigned>(entry - pg * a.pages.page_size);
        pool_row = no * page_rows + in_page;
      }
      const size_t row = static_cast<size_t>(pool_row) * (D * sizeof(T));
      const unsigned to = stages_at + buf * S::kStage + (u * S::kWaves + wave) * 1024;
      load_1k(static_cast<const char *>(a.k_pages) + row + R::k_slot(r, lane % C) * 16, to);
      load_1k(static_cast<const char *>(a.v_pages) + row + R::v_slot(r, lane % C) * 16, to + S::kHalf);
    }
    return hole;
  };
  // stage 0 before anything else is known of the block (last > first but for no entries at all), behind the first window of page
  // numbers: what the compiler waits for after a stage's loads would wait for them too
  const int page_last = last > first ? slot_of(last - 1) : 0;
  auto fill_window = [&]() __attribute__((always_inline)) {
    int no[kWindow / S::kBlock], runs[kListed ? kWindow / S::kBlock : 1];
    unsigned bits[kListed ? kWindow / S::kBlock : 1];
#pragma unroll
    for (int i = 0; i < kWindow / S::kBlock; ++i) {
      const int pg = window_at + i * S::kBlock + static_cast<int>(threadIdx.x);
      if constexpr (kListed) {
        no[i] = runs[i] = 0;
        bits[i] = 0;
        if (pg <= page_last) no[i] = static_cast<int>(run_at(pg, runs[i], bits[i]));
      } else {
        no[i] = pg <= page_last ? table[pg] : 0;
      }
    }
#pragma unroll
    for (int i = 0; i < kWindow / S::kBlock; ++i) {
      window[i * S::kBlock + threadIdx.x] = no[i];
      if constexpr (kListed) window_seen[i * S::kBlock + threadIdx.x] = runs[i];
      if constexpr (kPairs) window_bits[i * S::kBlock + threadIdx.x] = bits[i];
    }
  };
  // (kListed) what the token sees of a stage's runs, for the masks: the window may have moved on by then
  auto keep_runs = [&](int e0, int buf) __attribute__((always_inline)) {
    if (static_cast<int>(threadIdx.x) < kKeys >> a.list.run_shift) {
      const int x = (e0 >> a.list.run_shift) + static_cast<int>(threadIdx.x) - window_at;
      stage_seen[buf][threadIdx.x] = x < kWindow ? window_seen[x] : 0;
      if constexpr (kPairs) stage_bits[buf][threadIdx.x] = x < kWindow ? window_bits[x] : 0;
    }
  };
  bool hole_0 = false;
  if (kListed && last > first) {
    fill_window();
    __syncthreads();
    hole_0 = load_stage(first, last - 1, 0, [&](int pg, int) __attribute__((always_inline)) { return window[pg - window_at]; });
    keep_runs(first, 0);
  }
  if (!kListed && last > first) {
    int page[S::kLoads];
#pragma unroll
    for (int u = 0; u < S::kLoads; ++u) page[u] = table[page_of(a.pages, min(first + (u * S::kWaves + wave) * S::kPerLoad + lane / C, last - 1))];
    fill_window();
    hole_0 = load_stage(first, last - 1, 0, [&](int, int u) __attribute__((always_inline)) { return page[u]; });
  }

  // what the block's rows see of the entries
  if (!have) seen = 0;
  int most = seen, least = seen;
  if (a.visible) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      most = max(most, __shfl_xor(most, o));
      least = min(least, __shfl_xor(least, o));
    }
  }
  most = __builtin_amdgcn_readfirstlane(most);
  least = __builtin_amdgcn_readfirstlane(least);
  if (lane == 0) {
    shared_most[wave] = most;
    shared_least[wave] = have ? least : a.length;
  }
  if (threadIdx.x < 2) shared_hole[threadIdx.x] = 0;
  if (threadIdx.x == 0) shared_odd = 0;
  __syncthreads();
  if (hole_0) shared_hole[0] = 1;
  int end = 0, block_least = a.length;
#pragma unroll
  for (int w = 0; w < S::kWaves; ++w) {
    end = max(end, shared_most[w]);
    block_least = min(block_least, shared_least[w]);
  }
  end = __builtin_amdgcn_readfirstlane(min(end, last));
  const int n_stages = end > first ? (end - first + kKeys - 1) / kKeys : 0;
  // the first stage that some row does not see all of
  // (with weights in terms, of which the second may be negative or zero: as if it were the first of all)
  const int mask_from = R::kTerms > 1 || kPairs ? 0 : max(__builtin_amdgcn_readfirstlane(min(block_least, last)) - first, 0) / kKeys;
  int masked = INT_MAX;                            // ... and the first one with anything masked

  auto fetch = [&](int st, int buf) __attribute__((always_inline)) {
    const int e0 = first + st * kKeys;
    if (slot_of(min(e0 + kKeys, end) - 1) >= window_at + kWindow) {   // (uniform)
      window_at = slot_of(e0);
      __syncthreads();
      fill_window();
      __syncthreads();
    }
    const bool hole = load_stage(e0, end - 1, buf, [&](int pg, int) __attribute__((always_inline)) { return window[pg - window_at]; });
    if constexpr (kListed) keep_runs(e0, buf);
    if (!kPairs && hole) shared_hole[buf] = st + 1;   // (by the barrier before the stage is worked on)
  };
  // Waits for this wave's loads and for the other waves.
  auto arrived = [&]() __attribute__((always_inline)) {
    __asm__ volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(7 << 4);            // vmcnt(0), lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    __asm__ volatile("" ::: "memory");
  };

  const float c2 = a.scale * kLog2e;
  f32x16_t o[kTiles];
#pragma unroll
  for (int t = 0; t < kTiles; ++t)
#pragma unroll
    for (int x = 0; x < 16; ++x) o[t][x] = 0.f;
  float m = -FLT_MAX, l = 0.f;                     // l: over this lane's entries
  bool plain = true, fresh = true;                 // (of the wave) no reference beyond kHuge; none at all

  // Where this lane's operands lie in a stage: of K chunk 2 j + h of entry c of a sub-tile, of V the first entry's part of the
  // columns 32 t ..  All other entries lie at fixed distances (the places among an entry's chunks repeat).
  int k_at[kOps], v_at[kTiles];
#pragma unroll
  for (int j = 0; j < kOps; ++j) k_at[j] = (c * C + R::k_slot(c, 2 * j + h)) * 16;
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    const int r = R::kF32 ? 4 * h : 4 * h + (lane & 15) / 4, at = (R::kF32 ? 32 * t + c : 32 * t + (lane & 16) + (lane & 3) * 4) * static_cast<int>(sizeof(T));
    v_at[t] = (r * C + R::v_slot(r, at / 16)) * 16 + at % 16;
  }
  constexpr int kEntry = C * 16;                   // bytes of an entry

  // one sub-tile's logits
  auto logits = [&](const char *ks, int e0, f32x16_t &s) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < 16; ++x) s[x] = 0.f;
    int k_0 = k_at[0];                             // (kPerTile: the places of the others worked out rather than kept, an exclusive or each)
    if constexpr (kPairs) __asm__("" : "+v"(k_0));
#pragma unroll
    for (int j = 0; j < kOps; ++j) {
      const u32x4_t ka = *reinterpret_cast<const u32x4_t *>(ks + (kPairs ? k_0 ^ 32 * j : k_at[j]) + e0 * kEntry);
      if constexpr (R::kF32) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          s = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(ka[e]), __uint_as_float(qb[j][e]), s, 0, 0, 0);
      } else {
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, ka), __builtin_bit_cast(bf16x8_t, qb[j]), s, 0, 0, 0);
      }
    }
  };
  // The operand of V for a product: columns 32 t .., bf16: entries 16 g .. 16 g + 15 of the sub-tile; fp32: the entries
  // 8 i + 4 h + j with 4 i + j = g.
  auto values = [&](const char *vs, int e0, int t, int g) __attribute__((always_inline)) {
    if constexpr (R::kF32) {
      return *reinterpret_cast<const unsigned *>(vs + v_at[t] + (e0 + 8 * (g / 4) + g % 4) * kEntry);
    } else {
      typedef __attribute__((address_space(3))) s16x4_t *at_t;
      u32x4_t w;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const s16x4_t x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((at_t)(vs + v_at[t] + (e0 + 16 * g + 8 * u) * kEntry));
        const u32x2_t y = __builtin_bit_cast(u32x2_t, x);
        w[2 * u] = y[0];
        w[2 * u + 1] = y[1];
      }
      return w;
    }
  };
  constexpr int kProducts = R::kF32 ? 16 : 2;      // of a sub-tile and a tile of columns
  using Weights = std::conditional_t<R::kF32, f32x16_t, u32x4_t[R::kTerms][2]>;
  auto product = [&](auto v, const Weights &p, int g, f32x16_t &to) __attribute__((always_inline)) {
    if constexpr (R::kF32) to = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(v), p[g], to, 0, 0, 0);
    else
#pragma unroll
      for (int i = 0; i < R::kTerms; ++i)
        to = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, v), __builtin_bit_cast(bf16x8_t, p[i][g]), to, 0, 0, 0);
  };
  auto weights_of = [&](const f32x16_t &s, Weights &p, auto fast) __attribute__((always_inline)) {   // -> their sum
    float w[16], sum = 0.f;
#pragma unroll
    for (int x = 0; x < 16; ++x) w[x] = __builtin_amdgcn_exp2f(decltype(fast)::value ? fmaf(s[x], c2, -m) : exponent_of(s[x], c2, m));
#pragma unroll
    for (int x = 0; x < 16; x += 4) sum += (w[x] + w[x + 1]) + (w[x + 2] + w[x + 3]);
    if constexpr (R::kF32) {
#pragma unroll
      for (int x = 0; x < 16; ++x) p[x] = w[x];
    } else {
#pragma unroll
      for (int i = 0; i < R::kTerms; ++i)
#pragma unroll
        for (int x = 0; x < 16; x += 2) {
          const unsigned both = pair_to_bf16(w[x], w[x + 1]);
          p[i][x / 8][x % 8 / 2] = both;
          if (i + 1 < R::kTerms) {                 // what is left
            w[x] -= bf16_low(both);
            w[x + 1] -= bf16_high(both);
          }
        }
    }
    return sum;
  };
  auto weights = [&](const f32x16_t (&s)[kSub], Weights (&p)[kSub]) __attribute__((always_inline)) {
    float sum = 0.f;
    if (plain) {                                   // (wave-uniform)
#pragma unroll
      for (int x = 0; x < kSub; ++x) sum += weights_of(s[x], p[x], std::true_type{});
    } else {
#pragma unroll
      for (int x = 0; x < kSub; ++x) sum += weights_of(s[x], p[x], std::false_type{});
    }
    return sum;
  };

  auto work = [&](const char *ks, const char *vs, int st, int buf, bool holes) __attribute__((always_inline)) {
    const int key0 = first + st * kKeys + wk * (32 * kSub);   // this wave's entries
    ks += wk * (32 * kSub * kEntry);
    vs += wk * (32 * kSub * kEntry);
    if (key0 >= most) return;                      // (wave-uniform) nobody sees them
    // (kPerTile) what the lane's row sees of the entries of a run from one on, `left` at most
    const int shift = kPairs ? a.list.run_shift : 0, in_stage = wk * (32 * kSub) + 4 * h;
    const bool whole_runs = shift >= 5;            // (uniform) 32 entries are always of one run
    auto seen_of = [&](int key, int left) __attribute__((always_inline)) {
      const int run = key >> shift;
      const int n = (stage_bits[buf][kPairs ? run : 0] >> my_token & 1u) != 0 ? reach : 0;
      return min(n - stage_seen[buf][kListed ? run : 0] - (key & ((1 << shift) - 1)), left);
    };
    if constexpr (kPairs) {
      if (whole_runs) {
        bool some = false;
#pragma unroll
        for (int x = 0; x < kSub; ++x) some |= seen_of(in_stage + 32 * x, last - key0 - 4 * h - 32 * x) > 0;
        if (__builtin_amdgcn_ballot_w64(some) == 0) return;            // the wave's tokens read none of them
      }
    }
    f32x16_t s[kSub];
    Weights p[kSub];
#pragma unroll
    for (int x = 0; x < kSub; ++x) logits(ks, 32 * x, s[x]);
    ahead<kSub * kOps, R::kF32 ? 4 : 1, 1, R::kF32 || kPairs ? 2 : 4>();
    if constexpr (kPairs) {                        // each row by its token's bit and what it sees
#pragma unroll
      for (int x = 0; x < kSub; ++x) {
        if (whole_runs) {
          const int n = seen_of(in_stage + 32 * x, last - key0 - 4 * h - 32 * x);
          if (__builtin_amdgcn_ballot_w64(n < 28) == 0) continue;      // all of them, for every row
#pragma unroll
          for (int i = 0; i < 16; ++i) s[x][i] = 8 * (i / 4) + i % 4 < n ? s[x][i] : -INFINITY;
        } else {
          unsigned there = 0;
#pragma unroll 1
          for (int i = 0; i < 16; ++i) {
            const int key = 32 * x + 8 * (i / 4) + i % 4;
            there |= seen_of(in_stage + key, last - key0 - 4 * h - key) > 0 ? 1u << i : 0u;
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) s[x][i] = there >> i & 1u ? s[x][i] : -INFINITY;
        }
      }
    }
    const bool mask = !kPairs && (holes || key0 + 32 * kSub > min(least, last));
    if (mask) {
      const int limit = min(seen, last) - key0 - 4 * h;
      unsigned there[kSub];                        // bit i: the entry is on a page
#pragma unroll
      for (int x = 0; x < kSub; ++x) there[x] = 0xFFFFu;
      if (kLists == kPerToken && holes) {
        const int shift = a.list.run_shift, in_stage = wk * (32 * kSub) + 4 * h;
#pragma unroll
        for (int x = 0; x < kSub; ++x)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int key = in_stage + 32 * x + 8 * (i / 4) + i % 4;
            if ((key & ((1 << shift) - 1)) >= stage_seen[buf][key >> shift]) there[x] &= ~(1u << i);
          }
      }
      if (!kListed && holes) {
#pragma unroll
        for (int x = 0; x < kSub; ++x)
#pragma unroll 1
          for (int i = 0; i < 16; ++i) {
            const int key = min(key0 + 32 * x + 8 * (i / 4) + 4 * h + i % 4, end - 1);
            if (static_cast<unsigned>(table[page_of(a.pages, key)]) >= static_cast<unsigned>(a.pages.n_pages)) there[x] &= ~(1u << i);
          }
      }
#pragma unroll
      for (int x = 0; x < kSub; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          s[x][i] = 32 * x + 8 * (i / 4) + i % 4 < limit && (there[x] >> i & 1u) != 0 ? s[x][i] : -INFINITY;
    }
    auto top_of = [&]() __attribute__((always_inline)) {
      float top = s[0][0];
#pragma unroll
      for (int x = 0; x < kSub; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, s[x][i]);
      return max_of_halves(top) * c2;
    };
    auto look_for_huge = [&]() __attribute__((always_inline)) { plain = __builtin_amdgcn_ballot_w64(fabsf(m) > kHuge && m != -FLT_MAX) == 0; };
    if (fresh) {                                   // (wave-uniform) the first entries: no reference yet, and no output
      fresh = false;
      m = fmaxf(m, top_of());
      look_for_huge();
    }
    float sum = weights(s, p);
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(sum > kFar) != 0, 0)) {
      const bool far = max_of_halves(sum) > kFar;  // (of this row)
      const float up = far ? fmaxf(m, top_of()) : m;
      const float keep = __builtin_amdgcn_exp2f(m - up);
      m = up;
      l = far ? l * keep : l;
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int x = 0; x < 16; ++x) o[t][x] = far ? o[t][x] * keep : o[t][x];
      look_for_huge();
      sum = weights(s, p);
    }
    l += sum;
#pragma unroll
    for (int x = 0; x < kSub; ++x)
#pragma unroll
      for (int g = 0; g < kProducts; ++g)
#pragma unroll
        for (int t = 0; t < kTiles; ++t) product(values(vs, 32 * x, t, g), p[x], g, o[t]);
    ahead<kSub * kProducts * kTiles, R::kF32 ? 1 : R::kTerms, R::kF32 ? 1 : 2, kPairs ? 2 : 4>();
  };
  // (of a stage's values; the stage is complete and nobody's yet)
  auto take_out = [&](char *vs) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < S::kLoads; ++u) {
      u32x4_t *at = reinterpret_cast<u32x4_t *>(vs) + u * S::kBlock + threadIdx.x;
      u32x4_t w = *at;
      if (take_out_odd<R::kF32>(w)) {
        *at = w;
        shared_odd = 2;
      }
    }
    __syncthreads();
  };

  // One barrier a stage: behind it the stage is complete and the one before it, whose place the next load takes, no longer
  // read.  (A third place, with two stages on their way: 79.5 instead of 81.5 us for 80 rows over 100003 entries of 8 KV heads, the same elsewhere.)
  bool again = false;                              // (of the block)
  if (n_stages == 0) arrived();                    // (nobody sees an entry: stage 0 is not for a later block's LDS)
#pragma unroll 1
  for (int st = 0; st < n_stages; ++st) {
    arrived();
    if (st + 1 < n_stages) fetch(st + 1, (st + 1) & 1);
    char *at = stages + (st & 1) * S::kStage;
    const bool holes = !kPairs && __builtin_amdgcn_readfirstlane(shared_hole[st & 1]) == st + 1;
    if (holes || st >= mask_from) {
      masked = min(masked, st);
      if (__builtin_expect(again, 0)) take_out(at + S::kHalf);
    }
    work(at, at + S::kHalf, st, st & 1, holes);
    if (st + 1 < n_stages || masked == INT_MAX || again) continue;
    // what the masks met.  (A look at the outputs, once a block, in place of one at the values of every such stage: tokens that see parts of
    // 701 entries, 99 of 32 heads, 64 x fp32 22.4 -> 20.8 us, 64 x bf16 16.0 -> 13.4, 128 x bf16 16.7 -> 16.2; the same where little is masked.)
    float zero = 0.f;
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int x = 0; x < 16; ++x) zero = fmaf(o[t][x], 0.f, zero);
    if (!(zero == 0.f)) shared_odd = 1;
    __syncthreads();
    if (__builtin_expect(__builtin_amdgcn_readfirstlane(shared_odd) == 0, 1)) continue;
    again = true;
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int x = 0; x < 16; ++x) o[t][x] = 0.f;
    m = -FLT_MAX;
    l = 0.f;
    plain = fresh = true;
    window_at = slot_of(first);
    fill_window();
    __syncthreads();
    fetch(0, 0);
    st = -1;
  }
  l = sum_of_halves(l);

  // ---- the waves that share rows: their outputs go through LDS, and each of them ends up with a part of the columns, groups
  // of four per lane: group k of this wave is columns 32 t + 8 i + 4 h .. with 4 t + i = first_group + k
  constexpr int kOwn = 4 * kTiles / kWK;
  const int first_group = wk * kOwn;
  f32x4_t part[kOwn];
  if constexpr (kWK == 1) {
#pragma unroll
    for (int k = 0; k < kOwn; ++k) part[k] = f32x4_t{o[k / 4][k % 4 * 4], o[k / 4][k % 4 * 4 + 1], o[k / 4][k % 4 * 4 + 2], o[k / 4][k % 4 * 4 + 3]};
  } else {
    // (where the stages were, in rounds of what these hold)
    constexpr int kAll = S::kWaves * 32 * D * 4, kRounds = (kAll + 2 * S::kStage - 1) / (2 * S::kStage), kPer = kOwn / kRounds;
    static_assert(kPer * kRounds == kOwn, "whole rounds");
    static_assert(S::kWaves * kWK * kPer * 64 * 16 <= 2 * S::kStage, "every wave has a place");
    auto place_of_wave = [&](int w) __attribute__((always_inline)) { return reinterpret_cast<f32x4_t *>(stages) + w * (kWK * kPer * 64) + lane; };
    __syncthreads();                               // (every wave is past its last stage)
    shared_ml[wk][wr][lane] = h == 0 ? m : l;
    f32x4_t *mine = place_of_wave(wave);
    float x[kWK];
#pragma unroll
    for (int rnd = 0; rnd < kRounds; ++rnd) {
#pragma unroll
      for (int w = 0; w < kWK; ++w)                // for wave w: its groups of this round
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
          const int g = w * kOwn + rnd * kPer + k;
          mine[(w * kPer + k) * 64] = f32x4_t{o[g / 4][g % 4 * 4], o[g / 4][g % 4 * 4 + 1], o[g / 4][g % 4 * 4 + 2], o[g / 4][g % 4 * 4 + 3]};
        }
      __asm__ volatile("" ::"v"(lse_other));       // (read by all before one of them replaces it)
      __syncthreads();
      if (rnd == 0) {
        m = -FLT_MAX;
#pragma unroll
        for (int w = 0; w < kWK; ++w) m = fmaxf(m, shared_ml[w][wr][c]);
        l = 0.f;
#pragma unroll
        for (int w = 0; w < kWK; ++w) {
          x[w] = __builtin_amdgcn_exp2f(shared_ml[w][wr][c] - m);
          l = fmaf(shared_ml[w][wr][32 + c], x[w], l);
        }
      }
#pragma unroll
      for (int k = 0; k < kPer; ++k) {
        f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWK; ++w) sum += place_of_wave(w * kWR + wr)[(wk * kPer + k) * 64] * x[w];
        part[rnd * kPer + k] = sum;
      }
      if (rnd + 1 < kRounds) __syncthreads();
    }
  }
  if (!have) return;
  if constexpr (kPairs) {                          // (worked out anew rather than kept)
    int r = min(r0 + c, M - 1);
    __asm__("" : "+v"(r));
    place = row_place(a, unit, r);
    place_in_tile(a, seq, table_row, token0, place);
    if constexpr (kLate) lse_other = lse_joined(a, place);
  }

  if (__builtin_expect(again, 0) && __builtin_amdgcn_readfirstlane(shared_odd) == 2) {
    // the infinities and NaN that were taken out and that a row sees (with a weight above zero, however small)
    for (int key = first + masked * kKeys; key < min(last, most); ++key) {
      unsigned pool_row;
      bool sees = key < seen;
      if constexpr (kListed) {
        int n = 0;
        unsigned bits = 0;
        const int at = key & ((1 << a.list.run_shift) - 1);
        pool_row = run_at(key >> a.list.run_shift, n, bits) + static_cast<unsigned>(at);
        if constexpr (kPairs) {
          if (n == kNowhere) continue;
          sees = (bits >> my_token & 1u) != 0 && n + at < reach;
        } else if (at >= n) {
          continue;
        }
      } else {
        const int pg = page_of(a.pages, key), no = __builtin_amdgcn_readfirstlane(table[pg]);
        if (static_cast<unsigned>(no) >= static_cast<unsigned>(a.pages.n_pages)) continue;
        pool_row = no * page_rows + kvh * head_rows + static_cast<unsigned>(key - pg * a.pages.page_size);
      }
      const T *v = static_cast<const T *>(a.v_pages) + static_cast<size_t>(pool_row) * D + 4 * h;
#pragma unroll
      for (int k = 0; k < kOwn; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const T y = v[8 * (first_group + k) + e];
          float f;
          if constexpr (R::kF32) f = y;
          else f = __uint_as_float(static_cast<unsigned>(y) << 16);
          part[k][e] += sees && !(fabsf(f) <= FLT_MAX) ? f : 0.f;
        }
    }
  }

  if (a.n_split > 1) {
    // for the second kernel: [unit][32 rows][split][group][lane] float4, and (m, l) of the rows
    const int tiles = (a.n_tokens * a.group + 31) / 32;
    const size_t p = (static_cast<size_t>(unit) * tiles + r0 / 32) * a.n_split + split;
    f32x4_t *to = reinterpret_cast<f32x4_t *>(a.part_o) + p * (4 * kTiles * 64) + lane;
#pragma unroll
    for (int k = 0; k < kOwn; ++k) to[(first_group + k) * 64] = part[k];
    if (wk > 0) return;
    a.part_ml[p * 64 + lane] = h == 0 ? m : l;
    if (split == 0 && h == 0) a.part_lse[static_cast<size_t>(unit) * (tiles * 32) + r0 + c] = lse_other;
    return;
  }
  if (r0 + c >= M || !takes_part(a, place.token)) return;
  const Joined j = join(m, l, lse_other);
#pragma unroll
  for (int k = 0; k < kOwn; ++k) finish4<T, D>(a, place, 8 * (first_group + k) + 4 * h, part[k], j);
  if (wk == 0 && h == 0) finish_row(a, place, j);
}

// The splits of 32 rows joined: blocks = unit and 32 rows (x), 32 columns (y); kGroups groups of 256 threads take every kGroups-th
// of up to kMost splits each.
template <typename T, int D, int kGroups, int kMost>
__global__ __launch_bounds__(256 * kGroups) void attend_merge_kernel(const AttendArgs a) {
  constexpr int kTiles = D / 32, kBatch = kGroups == 1 ? kMost : 8;   // (one round trip)
  __shared__ float ml[kMost * 64];
  __shared__ f32x4_t sums[kGroups > 1 ? kGroups - 1 : 1][256];
  __shared__ float lsums[kGroups][32];
  const int lane = threadIdx.x & 63, i = threadIdx.x >> 6 & 3, g = threadIdx.x >> 8;
  const int c = lane & 31, h = lane >> 5;
  int M = a.n_tokens * a.group;
  const int tiles = (M + 31) / 32, n = a.n_split;
  const int t = static_cast<int>(blockIdx.y), ut = static_cast<int>(blockIdx.x);
  const size_t p0 = static_cast<size_t>(ut) * n;
  const f32x4_t *from = reinterpret_cast<const f32x4_t *>(a.part_o) + p0 * (4 * kTiles * 64) + (4 * t + i) * 64 + lane;
  f32x4_t x[kBatch];
  auto load = [&](int s0) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < kBatch; ++k)
      if (s0 + k * kGroups < n) x[k] = from[static_cast<size_t>(s0 + k * kGroups) * (4 * kTiles * 64)];   // (uniform)
  };
  for (int k = threadIdx.x; k < n * 64; k += 256 * kGroups) ml[k] = a.part_ml[p0 * 64 + k];
  load(g);
  const float lse_other = a.part_lse[static_cast<size_t>(ut) * 32 + c];
  __syncthreads();
  float m = -FLT_MAX;
  for (int s = 0; s < n; ++s) m = fmaxf(m, ml[s * 64 + c]);
  f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
  float l = 0.f;
  for (int s0 = g; s0 < n; s0 += kBatch * kGroups) {
    f32x4_t y[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) y[k] = x[k];
    if (s0 + kBatch * kGroups < n) load(s0 + kBatch * kGroups);
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int s = s0 + k * kGroups;
      if (s < n) {                                 // (uniform)
        const float w = __builtin_amdgcn_exp2f(ml[s * 64 + c] - m);
        l = fmaf(ml[s * 64 + 32 + c], w, l);
        sum += y[k] * w;
      }
    }
  }
  if constexpr (kGroups > 1) {
    if (i == 0 && h == 0) lsums[g][c] = l;
    if (g > 0) sums[g - 1][threadIdx.x & 255] = sum;
    __syncthreads();
    if (g > 0) return;
    l = 0.f;
#pragma unroll
    for (int k = 0; k < kGroups; ++k) l += lsums[k][c];
#pragma unroll
    for (int k = 0; k < kGroups - 1; ++k) sum += sums[k][threadIdx.x];
  }
  const int unit = tiles == 1 ? ut : ut / tiles, r0 = (ut - unit * tiles) * 32;
  RowPlace place = row_place(a, unit, min(r0 + c, M - 1));
  if (a.list.tiles > 0) {                          // (uniform)
    const int tile = unit / a.n_kv_heads;
    int table_row;
    const int token0 = tile_token0(a, tile, table_row);
    M = tile_rows(a, token0);
    place_in_tile(a, tile, table_row, token0, place);
  }
  if (r0 + c >= M || !takes_part(a, place.token)) return;
  const Joined j = join(m, l, lse_other);
  finish4<T, D>(a, place, 32 * t + 8 * i + 4 * h, sum, j);
  if (t == 0 && i == 0 && h == 0) finish_row(a, place, j);
}

// How a call is cut: rows of a block (32 wr), waves that share rows, entries of a stage, splits of the entries.
struct Plan { int wr, wk, keys, n_split, split_keys; };

// The shapes of blocks, and what a stage of theirs takes on a full chip of 256 compute units (us; the rule asks for no device, so that a workspace's
// size is the same everywhere; a part of the chip takes the same shapes).  More rows in a block
// share an entry's way to LDS, and a wave with 64 entries a stage has two chains of products; fewer rows make more blocks of few
// tokens without splits.  The cheapest by the sum of these is taken: stages one after the other, or the bytes where they take longer, a
// fixed part, and for splits a second launch that reads what the first left (16 KB for 32 rows and split).  Measured, us, 128 x bf16,
// (32 wr rows, wk) and splits:
//   4 KV heads,  224 rows,   8192 entries  (64, 4) x 16 21.5   (128, 2) x 32 22.8   (256, 1) x 32 25.2
//   4 KV heads,  512 rows,   8192          (64, 4) x  8 25.7   (128, 2) x 16 27.8   (256, 1) x 16 33.2
//   4 KV heads, 2048 rows,   4096          (64, 4) x  2 36.7   (128, 2) x  4 33.6   (256, 1) x  4 43.3
//   4 KV heads, 4480 rows,   4096          (64, 4) x  1 99.8   (128, 2) x  3 64.0   (256, 1) x  3 55.7
//   8 KV heads, 20480 rows, their past     (64, 4) x  1 299    (128, 2) x  1 214    (256, 1) x  1 193.5
//   8 KV heads,   80 rows, 100003          (64, 4) x 16 107    (128, 2) x 32 81.7   (256, 1) x 32 89.4
// Other rows, us of what the rule takes / of the best of all shapes and splits:
//                                                64 x bf16      64 x fp32      128 x fp32
//   4 KV heads,    7 rows, 8192 entries          11.6 / 11.6    16.3 / 16.2    25.2 / 25.2
//   8 KV heads,    8 rows, 4096                  10.4 / 10.4    15.0 / 13.5    22.0 / 22.0
//   4 KV heads,  224 rows, 8192                  17.6 / 17.6    32.5 / 32.3    55.4 / 51.6
//   8 KV heads,   80 rows, 100003 (fp32: 25000)  56.4 / 56.4    78.7 / 69.2    145 / 131
//   4 KV heads,  512 rows, 8192 (2048)           22.5 / 21.5    23.4 / 21.7    36.2 / 36.2
//   4 KV heads, 2048 rows, 4096 (1024)           28.6 / 27.9    33.3 / 31.0    55.9 / 54.0
//   4 KV heads, 4480 rows, 4096 (1024)           51.2 / 51.2    67.8 / 63.6    126 / 126
//   8 KV heads, 20480 (5120) rows, their past    174 / 174      85.5 / 74.2    153 / 148
//   4 KV heads, 7000 rows, their past            20.9 / 20.1    74.8 / 50.4    151 / 99.0
//   16 x 4 KV heads, 7 rows each, 8192           29.6 / 28.1    64.5 / 64.5    176 / 176
// (The last but one: the rule counts all entries where rows see half of them, and leaves out blocks of few rows, see plan_of.)
struct BlockShape { int wr, wk, keys; float stage_us; };
// (fp32 products run at a sixteenth of the rate of bf16 ones: a stage is a wave's products.  fp32 rows of 128: fewer entries a stage, and
// waves, than LDS and registers hold of the others.)
template <typename T, int D>
struct Shapes {
  static constexpr BlockShape kAll[] = {{1, 4, 128, D == 128 ? 2.0f : 1.2f}, {2, 4, 128, D == 128 ? 1.65f : 1.2f},
                                        {4, 2, 128, D == 128 ? 2.1f : 1.4f}, {8, 1, 64, D == 128 ? 1.9f : 1.3f}};
};
template <>
struct Shapes<float, 64> {
  static constexpr BlockShape kAll[] = {{1, 4, 128, 2.2f}, {2, 4, 128, 4.0f}, {4, 2, 128, 7.8f}, {8, 1, 64, 7.8f}};
};
template <>
struct Shapes<float, 128> {
  static constexpr BlockShape kAll[] = {{2, 2, 64, 4.0f}, {4, 1, 64, 7.8f}};
};

template <typename T, int D>
Plan plan_of(const AttendArgs &a) {
  constexpr const auto &shapes = Shapes<T, D>::kAll;
  constexpr int n_shapes = sizeof(shapes) / sizeof(shapes[0]);
  const int M = a.n_tokens * a.group, units = a.n_seqs * a.n_kv_heads, tiles = (M + 31) / 32;
  const float bytes_us = 2.f * units * a.length * (D * sizeof(T)) / 5.4e6f;
  Plan best = {0, 0, 0, 1, 0};
  float best_us = FLT_MAX;
  for (int i = 0; i < n_shapes; ++i) {
    const BlockShape &s = shapes[i];
    if (i > 0 && 32 * shapes[i - 1].wr >= M) break;            // (rows enough for the shape before)
    if (i + 1 < n_shapes && M > 32 * s.wr * 64) continue;      // (far more rows than blocks of few are for: 4480 and 20480 rows above)
    const long long blocks = static_cast<long long>(units) * ((M + 32 * s.wr - 1) / (32 * s.wr));
    const int stages = a.length > 0 ? (a.length + s.keys - 1) / s.keys : 1;
    const int fill = static_cast<int>(256 / blocks);
    for (int k = 0; k < 4; ++k) {                              // splits: none, half a chip of blocks, one chip, two
      int n = k == 0 ? 1 : k == 1 ? fill / 2 : k == 2 ? fill : static_cast<int>(512 / blocks);
      n = n > stages ? stages : n;
      n = n > kSplitMax ? kSplitMax : n;
      if (n < (k == 0 ? 1 : 2)) continue;
      const int each = (stages + n - 1) / n;
      n = (stages + each - 1) / each;
      const float full = static_cast<float>(blocks) * n / 256.f;
      const float rounds = full > 3.f ? full : full > 2.f ? 3.f : full > 1.f ? 2.f : 1.f;
      const float work = rounds * each * s.stage_us;
      const float join = n > 1 ? 4.f + 0.06f * n + 2.f * units * tiles * n * (32.f * D * 4.f) / 5e6f : 0.f;
      const float us = 7.f + (work > bytes_us ? work : bytes_us) + join;
      if (us < best_us) {
        best_us = us;
        best = {s.wr, s.wk, s.keys, n, each * s.keys};
      }
    }
  }
  return best;
}

size_t align_up(size_t x) { return (x + 255) / 256 * 256; }
size_t tiles_of(const AttendArgs &a) {
  return static_cast<size_t>(a.n_seqs) * a.n_kv_heads * ((static_cast<size_t>(a.n_tokens) * a.group + 31) / 32);
}
size_t bytes_of(const AttendArgs &a, const Plan &p) {
  if (p.n_split <= 1) return 0;
  const size_t parts = tiles_of(a) * p.n_split;
  return align_up(parts * 32 * a.head_dim * sizeof(float)) + align_up(parts * 64 * sizeof(float)) + align_up(tiles_of(a) * 32 * sizeof(float));
}

template <typename T, int D, int kWR, int kWK, int kKeys, int kLists = kNoList>
hipError_t launch_shape(const AttendArgs &a, hipStream_t stream) {
  const long long M = static_cast<long long>(a.n_tokens) * a.group, spans = (M + 32 * kWR - 1) / (32 * kWR);
  if (spans > 65535) return hipErrorInvalidValue;
  const dim3 grid(static_cast<unsigned>(a.n_seqs * a.n_kv_heads), static_cast<unsigned>(a.n_split), static_cast<unsigned>(spans));
  hipLaunchKernelGGL((attend_kernel<T, D, kWR, kWK, kKeys, kLists>), grid, dim3(64 * kWR * kWK), 0, stream, a);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_merge(const AttendArgs &a, hipStream_t stream) {
  if (a.n_split <= 1) return hipSuccess;
  const size_t blocks = tiles_of(a);
  if (blocks > 0x7FFFFFFFu) return hipErrorInvalidValue;
  const dim3 grid(static_cast<unsigned>(blocks), D / 32);
  if (a.n_split <= 4) hipLaunchKernelGGL((attend_merge_kernel<T, D, 1, 4>), grid, dim3(256), 0, stream, a);
  else if (a.n_split <= 16) hipLaunchKernelGGL((attend_merge_kernel<T, D, 1, 16>), grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((attend_merge_kernel<T, D, 4, kSplitMax>), grid, dim3(1024), 0, stream, a);
  return hipGetLastError();
}

template <typename T, int D, int kLists = kNoList>
hipError_t launch(AttendArgs a, hipStream_t stream) {
  constexpr bool kLong = D * sizeof(T) == 512;
  const Plan p = plan_of<T, D>(a);
  a.n_split = p.n_split;
  a.split_keys = p.split_keys;
  a.wide = (reinterpret_cast<uintptr_t>(a.q) | reinterpret_cast<uintptr_t>(a.out) | reinterpret_cast<uintptr_t>(a.joined_out)) % 16 == 0;
  if (bytes_of(a, p) > 0) {
    if (!a.workspace) return hipErrorInvalidValue;
    const size_t parts = tiles_of(a) * p.n_split;
    char *w = static_cast<char *>(a.workspace);
    a.part_o = reinterpret_cast<float *>(w);
    w += align_up(parts * 32 * D * sizeof(float));
    a.part_ml = reinterpret_cast<float *>(w);
    w += align_up(parts * 64 * sizeof(float));
    a.part_lse = reinterpret_cast<float *>(w);
  }
  hipError_t e = hipErrorInvalidValue;
  if constexpr (kLists == kPerToken) {             // (rows of one token: up to 64)
    if constexpr (kLong) e = launch_shape<T, D, 2, 2, 64, kPerToken>(a, stream);
    else if (p.wr == 1) e = launch_shape<T, D, 1, 4, 128, kPerToken>(a, stream);
    else if (p.wr == 2) e = launch_shape<T, D, 2, 4, 128, kPerToken>(a, stream);
  } else if constexpr (kLong) {
    if (p.wr == 2) e = launch_shape<T, D, 2, 2, 64>(a, stream);
    else if (p.wr == 4) e = launch_shape<T, D, 4, 1, 64>(a, stream);
  } else {
    if (p.wr == 1) e = launch_shape<T, D, 1, 4, 128>(a, stream);
    else if (p.wr == 2) e = launch_shape<T, D, 2, 4, 128>(a, stream);
    else if (p.wr == 4) e = launch_shape<T, D, 4, 2, 128>(a, stream);
    else if (p.wr == 8) e = launch_shape<T, D, 8, 1, 64>(a, stream);
  }
  return e == hipSuccess ? launch_merge<T, D>(a, stream) : e;
}

// The lists of a tile's tokens as one: blocks that some token reads, ascending, with a bit for each token that does.  A number that a
// token's list has had before is a pair of its own, behind the others: token by token (a wave each), in its list's order.  One block per unit.
// One such number of one token in each tile, us for the whole call: 640 tokens over 32 of 512 blocks each 128 as without, 300 over 200 of 938 179 and 174 without (one
// thread that goes over all tokens' numbers: 263, 1405).
constexpr int kListBlocks = 8192;       // of a table row, whose bits LDS holds (beyond: every token on its own.  640 tokens of 28 / 4 heads over 128 blocks of 16: 320 us of 8192, 386 of 8193)
__global__ __launch_bounds__(256) void join_lists_kernel(const AttendArgs a) {
  __shared__ unsigned bits[kListBlocks];
  __shared__ int counts[4], twice[32];             // (twice: numbers of a token that its list has had before)
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int unit = static_cast<int>(blockIdx.x), tile = unit / a.n_kv_heads, kvh = unit - tile * a.n_kv_heads;
  const int table_row = tile / a.list.tiles, token0 = (tile - table_row * a.list.tiles) * a.n_tokens;
  const int tokens = min(a.n_tokens, a.list.tokens - token0), n = tokens * a.list.n_listed;
  const int n_blocks = (a.list.entries + (1 << a.list.block_shift) - 1) >> a.list.block_shift;
  int2 *to = a.list.pairs + static_cast<long long>(unit) * a.list.n_listed * a.n_tokens;
  for (int b = threadIdx.x; b < n_blocks; b += 256) bits[b] = 0;
  if (threadIdx.x < 32) twice[threadIdx.x] = 0;
  __syncthreads();
  // number y of token i's list, -1 where it is no block that the token sees
  auto number = [&](int i, int y) __attribute__((always_inline)) {
    const long long token = static_cast<long long>(table_row) * a.list.tokens + token0 + i;
    const int b = a.list.list[(token * a.n_kv_heads + kvh) * a.list.n_listed + y];
    const int reach = a.visible ? min(max(a.visible[token], 0), a.list.entries) : a.list.entries;
    return b >= 0 && b <= (reach - 1) >> a.list.block_shift ? b : -1;
  };
  for (int x = threadIdx.x; x < n; x += 256) {
    const int i = x / a.list.n_listed, b = number(i, x - i * a.list.n_listed);
    if (b >= 0 && (atomicOr(&bits[b], 1u << i) >> i & 1u) != 0) atomicAdd(&twice[i], 1);
  }
  __syncthreads();
  int at = 0;
  for (int b0 = 0; b0 < n_blocks; b0 += 256) {
    const int b = b0 + static_cast<int>(threadIdx.x);
    const unsigned mine = b < n_blocks ? bits[b] : 0u;
    const unsigned long long m = __ballot(mine != 0);
    if (lane == 0) counts[wave] = __popcll(m);
    __syncthreads();
    int before = at;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      before += w < wave ? counts[w] : 0;
      at += counts[w];
    }
    if (mine) to[before + __popcll(m & ((1ull << lane) - 1))] = make_int2(b, static_cast<int>(mine));
    __syncthreads();
  }
  int all = at;
  for (int i = 0; i < tokens; ++i) all += twice[i];
  if (all > at) {                                  // (uniform)
    for (int b = threadIdx.x; b < n_blocks; b += 256) bits[b] = 0;
    __syncthreads();
    int next = at;                                 // the place of token i's first one
    for (int i = 0; i < tokens; next += twice[i++]) {
      if (i % 4 != wave || twice[i] == 0) continue;            // (wave-uniform)
      int place = next;
      for (int y0 = 0; y0 < a.list.n_listed; y0 += 64) {
        const int b = y0 + lane < a.list.n_listed ? number(i, y0 + lane) : -1;
        // had before these 64 (nobody else has this token's bits); then, of equal ones among them, all but the first
        bool had = b >= 0 && (*const_cast<volatile unsigned *>(&bits[max(b, 0)]) >> i & 1u) != 0;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const bool met = b >= 0 && (atomicOr(&bits[max(b, 0)], 1u << i) >> i & 1u) != 0;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (__ballot(met && !had) != 0) {          // (wave-uniform)
          bool later = false;
          for (unsigned long long rest = __ballot(b >= 0 && !had); rest != 0;) {
            const int first = __builtin_ctzll(rest);
            const unsigned long long same = rest & __ballot(b == __builtin_amdgcn_readlane(b, first));
            later |= lane != first && (same >> lane & 1u) != 0;
            rest &= ~same;
          }
          had |= later;
        }
        const unsigned long long m = __ballot(had);
        const int to_place = place + __popcll(m & ((1ull << lane) - 1));
        if (had && to_place < n) to[to_place] = make_int2(b, static_cast<int>(1u << i));   // (n: lists that change meanwhile, which no caller may do)
        place += __popcll(m);
      }
    }
  }
  if (threadIdx.x == 0) a.list.counts[unit] = min(all, n);
}

// Tokens that share a block's rows, by their lists as one (0: every token on its own), in tiles of a table row's; blocks of wr times 32 rows; splits of a
// tile's list.  Tokens next to one another read much the same blocks, and an entry's way to LDS and a stage's fixed part are shared by those that do; a wave
// none of whose 32 rows reads any of its entries passes them over, so that a wide tile costs little where they differ.  Measured, us, 128 x bf16,
// 640 tokens of 28 / 4 heads that read 32 of 512 blocks of 64 entries each (4 tokens 66 different ones, 9 90, 18 111), lists' kernel (5) and merge (8) left out:
//   every token on its own 378     tiles of 4 tokens, 32 rows 250     of 9, 64 rows 167     of 18, 128 rows 115 - 121
// the last one with 3 splits (2 167, 4 155, 5 135, 8 132: blocks come in rounds of 512), two blocks of four waves to a compute unit; with eight waves that
// share 128 rows, a block to a compute unit, 175.  More stages on their way make no difference, so their arrival does not bind: by counters waves wait for one another
// in 57 % of their time, at the barrier of a stage that some of them pass over, and matrix cores are busy in 16 %, vector units in 30 %.
// The other types, us for the whole call, every token on its own -> tiles: those 640 tokens 64 x bf16 146 -> 105, 64 x fp32 598 -> 336, 128 x fp32 1742 -> 1028; 300 tokens of 40 /
// 8 heads over 20 of 469 blocks of 64 157 -> 58 (64 x bf16 61 -> 48, 64 x fp32 219 -> 115, 128 x fp32 583 -> 246).  Lists of few entries lose: 2 x 100 tokens of 8 / 2 heads
// over 11 of 1250 blocks of 16 21 -> 29 (64 x bf16 10 -> 26, 64 x fp32 25 -> 35, 128 x fp32 45 -> 42), by the two more launches.
// Few units (at most one for each compute unit): every token on its own, as the latency of one's list is what counts.  Tokens of 28 / 4 heads over 32 blocks of 64, 128 x
// bf16 (64 x fp32), own -> tiles: 64 units 19 -> 28 us (24 -> 31), 128 28 -> 30 (38 -> 41), 192 41 -> 33 (62 -> 49), 256 42 -> 36 (63 -> 58), 260 76 -> 36 (118 -> 57), 512 80 -> 48
// (121 -> 89).  Of 2 / 1 heads: 32 15 -> 22, 128 28 -> 26, 256 42 -> 27, 260 78 -> 28: the second round of blocks is what tiles save.
struct TilePlan { int tokens, tiles, wr, n_split; };
TilePlan tile_plan_of(const AttendArgs &a) {
  TilePlan p = {0, 0, 0, 1};
  const int n = a.list.tokens, n_blocks = (a.list.entries + (1 << a.list.block_shift) - 1) >> a.list.block_shift;
  if (n < 2 || n_blocks > kListBlocks || n_blocks < 1 || static_cast<long long>(a.n_seqs) * a.n_kv_heads <= 256) return p;
  const bool long_rows = a.dtype == LAZYEV_DTYPE_FP32 && a.head_dim == 128;
  int most = (long_rows ? 64 : 128) / a.group;
  most = most < 32 ? most : 32;                    // (a bit each)
  p.tokens = n < most ? n : most;
  // (entries of a joined list have 32-bit numbers, and it may be as long as all of its tokens' together: numbers twice are pairs of their own)
  if (p.tokens < 2 || (static_cast<long long>(p.tokens) * a.list.n_listed << a.list.block_shift) > (1 << 30)) return TilePlan{0, 0, 0, 1};
  p.tiles = (n + p.tokens - 1) / p.tokens;
  const int rows = p.tokens * a.group;
  p.wr = rows <= 32 && !long_rows ? 1 : rows <= 64 ? 2 : 4;
  const long long units = static_cast<long long>(a.n_seqs / n) * p.tiles * a.n_kv_heads;
  // (of the joined list, at most: how much of it the tokens share is not known here.  Splits of eight stages or more, us for kernel and merge; by one token's list they
  // were fewer: 557 tokens of 8 / 2 heads, 11 of 6240 blocks of 16, one split 172, 11 42; 300 of 40 / 8, 20 of 938 blocks of 32, two 80, five 55;
  // every token on its own 79, 163)
  const long long joined = static_cast<long long>(p.tokens) * a.list.n_listed;
  const long long stages = ((joined < n_blocks ? joined : n_blocks) << a.list.block_shift) / (p.wr == 4 || long_rows ? 64 : 128);
  long long split = (p.wr == 4 ? 512 : 256) / units;
  if (split > stages / 8) split = stages / 8;
  p.n_split = static_cast<int>(split < 1 ? 1 : split > kSplitMax ? kSplitMax : split);
  return p;
}
struct TileBytes { size_t pairs, counts, part_o, part_ml, part_lse; };
TileBytes tile_bytes_of(const AttendArgs &a, const TilePlan &p) {
  const size_t units = static_cast<size_t>(a.n_seqs) / a.list.tokens * p.tiles * a.n_kv_heads, tiles = units * ((p.tokens * a.group + 31) / 32);
  TileBytes b = {align_up(units * p.tokens * a.list.n_listed * sizeof(int2)), align_up(units * sizeof(int32_t)), 0, 0, 0};
  if (p.n_split > 1) {
    b.part_o = align_up(tiles * p.n_split * 32 * a.head_dim * sizeof(float));
    b.part_ml = align_up(tiles * p.n_split * 64 * sizeof(float));
    b.part_lse = align_up(tiles * 32 * sizeof(float));
  }
  return b;
}

template <typename T, int D>
hipError_t launch_tiles(AttendArgs a, const TilePlan &p, hipStream_t stream) {
  const int rows = a.n_seqs / a.list.tokens;       // of the table
  const size_t units = static_cast<size_t>(rows) * p.tiles * a.n_kv_heads;
  const TileBytes bytes = tile_bytes_of(a, p);
  char *w = static_cast<char *>(a.workspace);
  if (!w) return hipErrorInvalidValue;
  a.list.pairs = reinterpret_cast<int2 *>(w);
  w += bytes.pairs;
  a.list.counts = reinterpret_cast<int32_t *>(w);
  w += bytes.counts;
  a.part_o = reinterpret_cast<float *>(w);
  w += bytes.part_o;
  a.part_ml = reinterpret_cast<float *>(w);
  w += bytes.part_ml;
  a.part_lse = reinterpret_cast<float *>(w);
  a.list.tiles = p.tiles;
  a.n_seqs = rows * p.tiles;
  a.n_tokens = p.tokens;
  a.n_split = p.n_split;
  a.split_keys = 0;
  a.wide = (reinterpret_cast<uintptr_t>(a.q) | reinterpret_cast<uintptr_t>(a.out) | reinterpret_cast<uintptr_t>(a.joined_out)) % 16 == 0;
  hipLaunchKernelGGL(join_lists_kernel, dim3(static_cast<unsigned>(units)), dim3(256), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if constexpr (D * sizeof(T) == 512) {
    e = launch_shape<T, D, 2, 2, 64, kPerTile>(a, stream);
  } else {
    e = p.wr == 1 ? launch_shape<T, D, 1, 4, 128, kPerTile>(a, stream)
        : p.wr == 2 ? launch_shape<T, D, 2, 4, 128, kPerTile>(a, stream) : launch_shape<T, D, 4, 1, 64, kPerTile>(a, stream);
  }
  return e == hipSuccess ? launch_merge<T, D>(a, stream) : e;
}

}  // namespace

size_t attend_workspace(const AttendArgs &a) {
  if (a.dtype == LAZYEV_DTYPE_FP32) return a.head_dim == 64 ? bytes_of(a, plan_of<float, 64>(a)) : bytes_of(a, plan_of<float, 128>(a));
  return a.head_dim == 64 ? bytes_of(a, plan_of<bf16_t, 64>(a)) : bytes_of(a, plan_of<bf16_t, 128>(a));
}

size_t attend_list_workspace(const AttendArgs &a) {
  const TilePlan p = tile_plan_of(a);
  if (p.tokens == 0) return attend_workspace(a);
  const TileBytes b = tile_bytes_of(a, p);
  return b.pairs + b.counts + b.part_o + b.part_ml + b.part_lse;
}

hipError_t launch_attend_list(const AttendArgs &a, hipStream_t stream) {
  if (a.n_tokens != 1 || a.group < 1 || a.group > 64 || a.list.tokens < 1 || a.list.run_shift > a.list.block_shift || a.list.run_shift > 6 ||
      a.length != a.list.n_listed << a.list.block_shift)
    return hipErrorInvalidValue;
  const TilePlan p = tile_plan_of(a);
  if (a.dtype == LAZYEV_DTYPE_FP32 && a.head_dim == 64) return p.tokens ? launch_tiles<float, 64>(a, p, stream) : launch<float, 64, kPerToken>(a, stream);
  if (a.dtype == LAZYEV_DTYPE_FP32 && a.head_dim == 128) return p.tokens ? launch_tiles<float, 128>(a, p, stream) : launch<float, 128, kPerToken>(a, stream);
  if (a.dtype == LAZYEV_DTYPE_BF16 && a.head_dim == 64) return p.tokens ? launch_tiles<bf16_t, 64>(a, p, stream) : launch<bf16_t, 64, kPerToken>(a, stream);
  if (a.dtype == LAZYEV_DTYPE_BF16 && a.head_dim == 128) return p.tokens ? launch_tiles<bf16_t, 128>(a, p, stream) : launch<bf16_t, 128, kPerToken>(a, stream);
  return hipErrorInvalidValue;
}

hipError_t launch_attend(const AttendArgs &a, hipStream_t stream) {
  const long long rows = static_cast<long long>(a.n_seqs) * a.n_tokens * a.n_q_heads;
  if (rows < 1 || rows > 0x7FFFFFFFLL || a.group < 1 || a.n_q_heads != a.n_kv_heads * a.group || a.length < 0 || !a.pages.table ||
      static_cast<long long>(a.pages.stride) * a.pages.page_size < a.length || (a.joined_stat && (a.n_seqs != 1 || a.group > 8)) ||
      ((a.joined_stat || a.joined_lse) && !a.joined_out) || !a.q || !a.out || !a.k_pages || !a.v_pages)
    return hipErrorInvalidValue;
  if (a.dtype == LAZYEV_DTYPE_FP32 && a.head_dim == 64) return launch<float, 64>(a, stream);
  if (a.dtype == LAZYEV_DTYPE_FP32 && a.head_dim == 128) return launch<float, 128>(a, stream);
  if (a.dtype == LAZYEV_DTYPE_BF16 && a.head_dim == 64) return launch<bf16_t, 64>(a, stream);
  if (a.dtype == LAZYEV_DTYPE_BF16 && a.head_dim == 128) return launch<bf16_t, 128>(a, stream);
  return hipErrorInvalidValue;
}

}  // namespace lazyev
