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
// is taken for that row alone: what other rows see has no influence on it.
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
  // to the 0.0016 - 0.0017 of the output's own rounding.  64 x bf16 rows the decode step keeps exact with three terms; two are as far below that rounding
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
// x / y for 0 <= x < 2^24, y > 0 (the rounded quotient is off by one at most).
__device__ __forceinline__ int quotient(int x, int y) {
  int q = static_cast<int>(static_cast<float>(x) * __builtin_amdgcn_rcpf(static_cast<float>(y)));
  const int r = x - q * y;
  q += r >= y ? 1 : 0;
  return q - (r < 0 ? 1 : 0);
}
__device__ __forceinline__ RowPlace row_place(const AttendArgs &a, int unit, int r) {
  RowPlace p;
  const int seq = a.n_seqs == 1 ? 0 : unit / a.n_kv_heads, i = quotient(r, a.group);
  p.kvh = unit - seq * a.n_kv_heads;
  p.head = r - i * a.group;
  p.token = seq * a.n_tokens + i;
  p.row = static_cast<long long>(p.token) * a.n_q_heads + p.kvh * a.group + p.head;
  return p;
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
  static constexpr int kHalf = kKeys * D * static_cast<int>(sizeof(T)), kStage = 2 * kHalf;   // bytes of a stage: of K, then of V
};
constexpr int kWindow = 512;            // page numbers that a block keeps in LDS

template <typename T, int D, int kWR, int kWK, int kKeys>
__global__ __launch_bounds__(64 * kWR * kWK, (Shape<T, D, kWR, kWK, kKeys>::kPerSimd)) void attend_kernel(const AttendArgs a) {
  using R = Rows<T, D>;
  using S = Shape<T, D, kWR, kWK, kKeys>;
  constexpr int kSub = S::kSub, kOps = R::kOps, kTiles = R::kTiles, C = R::kChunks;
  __shared__ __align__(16) char stages[2 * S::kStage];
  __shared__ int window[kWindow];
  __shared__ float shared_ml[kWK][kWR][64];
  __shared__ int shared_most[S::kWaves], shared_least[S::kWaves], shared_hole[2], shared_odd;

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 31, h = lane >> 5;
  const int wr = wave % kWR, wk = wave / kWR;
  const int M = a.n_tokens * a.group;
  // (blocks of one unit, split and so on are as far from one another as there are units: those of eight units, or four, share
  // an XCD and its L2.)  Late rows first: where a token sees its past only, they have the most to do
  const int unit = static_cast<int>(blockIdx.x), split = static_cast<int>(blockIdx.y), span = static_cast<int>(gridDim.z - 1 - blockIdx.z);
  const int seq = a.n_seqs == 1 ? 0 : unit / a.n_kv_heads, kvh = unit - seq * a.n_kv_heads;
  const int r0 = (span * kWR + wr) * 32;           // this wave's rows
  const bool have = r0 < M;
  const RowPlace place = row_place(a, unit, min(r0 + c, M - 1));

  // entries of this block: first .. last - 1
  const int first = split * a.split_keys, last = min(first + a.split_keys, a.length);
  const int32_t *table = a.pages.table + static_cast<long long>(seq) * a.pages.stride;
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
  const float lse_other = lse_joined(a, place);
  int seen = a.visible ? min(max(a.visible[place.token], 0), a.length) : a.length;

  // ---- stages on their way to LDS.  Loads go from memory to LDS, 1 KB a wave, in the order of the addresses there.  (Written out, as
  // the compiler has every read of LDS wait for all loads into it: they leave nothing in registers, and the waits for
  // them are in `arrived`.)
  const bool once = gridDim.z == 1;                // nobody else reads these entries (uniform): they need not stay in the caches
  const unsigned stages_at = static_cast<unsigned>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char *)stages));
  auto load_1k = [&](const char *from, unsigned to) __attribute__((always_inline)) {
    if (once) __asm__ volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off nt" ::"s"(to), "v"(from) : "memory", "m0");
    else __asm__ volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(from) : "memory", "m0");
  };
  const unsigned head_rows = static_cast<unsigned>(a.pages.page_size), page_rows = head_rows * static_cast<unsigned>(a.n_kv_heads);
  // Entries from e0 on, none beyond `limit`, to a stage's place; page numbers by number(page of the entry, load).  -> was one of them none?
  auto load_stage = [&](int e0, int limit, int buf, auto number) __attribute__((always_inline)) {
    bool hole = false;
#pragma unroll
    for (int u = 0; u < S::kLoads; ++u) {
      const int r = (u * S::kWaves + wave) * S::kPerLoad + lane / C;
      const int entry = min(e0 + r, limit), pg = page_of(a.pages, entry);
      unsigned no = static_cast<unsigned>(number(pg, u));
      if (no >= static_cast<unsigned>(a.pages.n_pages)) {   // no page: any row; its entries are masked
        hole = true;
        no = 0;
      }
      const unsigned in_page = kvh * head_rows + static_cast<unsigned>(entry - pg * a.pages.page_size);
      const size_t row = static_cast<size_t>(no * page_rows + in_page) * (D * sizeof(T));
      const unsigned to = stages_at + buf * S::kStage + (u * S::kWaves + wave) * 1024;
      load_1k(static_cast<const char *>(a.k_pages) + row + R::k_slot(r, lane % C) * 16, to);
      load_1k(static_cast<const char *>(a.v_pages) + row + R::v_slot(r, lane % C) * 16, to + S::kHalf);
    }
    return hole;
  };
  // stage 0 before anything else is known of the block (last > first but for no entries at all), behind the first window of page
  // numbers: what the compiler waits for after a stage's loads would wait for them too
  const int page_last = last > first ? page_of(a.pages, last - 1) : 0;
  int window_at = page_of(a.pages, first);
  auto fill_window = [&]() __attribute__((always_inline)) {
    int no[kWindow / S::kBlock];
#pragma unroll
    for (int i = 0; i < kWindow / S::kBlock; ++i) {
      const int pg = window_at + i * S::kBlock + static_cast<int>(threadIdx.x);
      no[i] = pg <= page_last ? table[pg] : 0;
    }
#pragma unroll
    for (int i = 0; i < kWindow / S::kBlock; ++i) window[i * S::kBlock + threadIdx.x] = no[i];
  };
  bool hole_0 = false;
  if (last > first) {
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
  const int mask_from = R::kTerms > 1 ? 0 : max(__builtin_amdgcn_readfirstlane(min(block_least, last)) - first, 0) / kKeys;
  int masked = INT_MAX;                            // ... and the first one with anything masked

  auto fetch = [&](int st, int buf) __attribute__((always_inline)) {
    const int e0 = first + st * kKeys;
    if (page_of(a.pages, min(e0 + kKeys, end) - 1) >= window_at + kWindow) {   // (uniform)
      window_at = page_of(a.pages, e0);
      __syncthreads();
      fill_window();
      __syncthreads();
    }
    const bool hole = load_stage(e0, end - 1, buf, [&](int pg, int) __attribute__((always_inline)) { return window[pg - window_at]; });
    if (hole) shared_hole[buf] = st + 1;           // (by the barrier before the stage is worked on)
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
#pragma unroll
    for (int j = 0; j < kOps; ++j) {
      const u32x4_t ka = *reinterpret_cast<const u32x4_t *>(ks + k_at[j] + e0 * kEntry);
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

  auto work = [&](const char *ks, const char *vs, int st, bool holes) __attribute__((always_inline)) {
    const int key0 = first + st * kKeys + wk * (32 * kSub);   // this wave's entries
    ks += wk * (32 * kSub * kEntry);
    vs += wk * (32 * kSub * kEntry);
    if (key0 >= most) return;                      // (wave-uniform) nobody sees them
    f32x16_t s[kSub];
    Weights p[kSub];
#pragma unroll
    for (int x = 0; x < kSub; ++x) logits(ks, 32 * x, s[x]);
    ahead<kSub * kOps, R::kF32 ? 4 : 1, 1, R::kF32 ? 2 : 4>();
    const bool mask = holes || key0 + 32 * kSub > min(least, last);
    if (mask) {
      const int limit = min(seen, last) - key0 - 4 * h;
      unsigned there[kSub];                        // bit i: the entry is on a page
#pragma unroll
      for (int x = 0; x < kSub; ++x) there[x] = 0xFFFFu;
      if (holes) {
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
    ahead<kSub * kProducts * kTiles, R::kF32 ? 1 : R::kTerms, R::kF32 ? 1 : 2, 4>();
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
    const bool holes = __builtin_amdgcn_readfirstlane(shared_hole[st & 1]) == st + 1;
    if (holes || st >= mask_from) {
      masked = min(masked, st);
      if (__builtin_expect(again, 0)) take_out(at + S::kHalf);
    }
    work(at, at + S::kHalf, st, holes);
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
    window_at = page_of(a.pages, first);
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

  if (__builtin_expect(again, 0) && __builtin_amdgcn_readfirstlane(shared_odd) == 2) {
    // the infinities and NaN that were taken out and that a row sees (with a weight above zero, however small)
    for (int key = first + masked * kKeys; key < min(last, most); ++key) {
      const int pg = page_of(a.pages, key), no = __builtin_amdgcn_readfirstlane(table[pg]);
      if (static_cast<unsigned>(no) >= static_cast<unsigned>(a.pages.n_pages)) continue;
      const T *v = static_cast<const T *>(a.v_pages) +
                   static_cast<size_t>(no * page_rows + kvh * head_rows + static_cast<unsigned>(key - pg * a.pages.page_size)) * D + 4 * h;
#pragma unroll
      for (int k = 0; k < kOwn; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const T y = v[8 * (first_group + k) + e];
          float f;
          if constexpr (R::kF32) f = y;
          else f = __uint_as_float(static_cast<unsigned>(y) << 16);
          part[k][e] += key < seen && !(fabsf(f) <= FLT_MAX) ? f : 0.f;
        }
    }
  }

  if (a.n_split > 1) {
    // for the second kernel: [unit][32 rows][split][group][lane] float4, and (m, l) of the rows
    const int tiles = (M + 31) / 32;
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
  const int M = a.n_tokens * a.group, tiles = (M + 31) / 32, n = a.n_split;
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
  const RowPlace place = row_place(a, unit, min(r0 + c, M - 1));
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

template <typename T, int D, int kWR, int kWK, int kKeys>
hipError_t launch_shape(const AttendArgs &a, hipStream_t stream) {
  const long long M = static_cast<long long>(a.n_tokens) * a.group, spans = (M + 32 * kWR - 1) / (32 * kWR);
  if (spans > 65535) return hipErrorInvalidValue;
  const dim3 grid(static_cast<unsigned>(a.n_seqs * a.n_kv_heads), static_cast<unsigned>(a.n_split), static_cast<unsigned>(spans));
  hipLaunchKernelGGL((attend_kernel<T, D, kWR, kWK, kKeys>), grid, dim3(64 * kWR * kWK), 0, stream, a);
  return hipGetLastError();
}

template <typename T, int D>
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
  if constexpr (kLong) {
    if (p.wr == 2) e = launch_shape<T, D, 2, 2, 64>(a, stream);
    else if (p.wr == 4) e = launch_shape<T, D, 4, 1, 64>(a, stream);
  } else {
    if (p.wr == 1) e = launch_shape<T, D, 1, 4, 128>(a, stream);
    else if (p.wr == 2) e = launch_shape<T, D, 2, 4, 128>(a, stream);
    else if (p.wr == 4) e = launch_shape<T, D, 4, 2, 128>(a, stream);
    else if (p.wr == 8) e = launch_shape<T, D, 8, 1, 64>(a, stream);
  }
  if (e != hipSuccess || p.n_split <= 1) return e;
  const size_t blocks = tiles_of(a);
  if (blocks > 0x7FFFFFFFu) return hipErrorInvalidValue;
  const dim3 grid(static_cast<unsigned>(blocks), D / 32);
  if (p.n_split <= 4) hipLaunchKernelGGL((attend_merge_kernel<T, D, 1, 4>), grid, dim3(256), 0, stream, a);
  else if (p.n_split <= 16) hipLaunchKernelGGL((attend_merge_kernel<T, D, 1, 16>), grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((attend_merge_kernel<T, D, 4, kSplitMax>), grid, dim3(1024), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

size_t attend_workspace(const AttendArgs &a) {
  if (a.dtype == LAZYEV_DTYPE_FP32) return a.head_dim == 64 ? bytes_of(a, plan_of<float, 64>(a)) : bytes_of(a, plan_of<float, 128>(a));
  return a.head_dim == 64 ? bytes_of(a, plan_of<bf16_t, 64>(a)) : bytes_of(a, plan_of<bf16_t, 128>(a));
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
