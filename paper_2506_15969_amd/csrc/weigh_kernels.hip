// The attention weight that every entry of a cache received (lazyev_pages_weigh): w[i] = (old) + sum over the rows r that see entry i of
// exp(scale q_r k_i - lse_r), rows being the tokens' heads of the entry's group.
//
// Both kernels have keys as the B operand and rows as A, so that a lane holds, of one entry, the logits of several rows, and the sum over rows is one in its
// register, then over the lanes of the same entry.  Rows that do not see all of the entries are masked, by the number of entries that they see; those past the
// last, and those that saw nothing (lse of -inf), see none.  The exponent is one multiply-add, logit scale log2 e - lse log2 e, of an lse that is
// rounded once more in these units: half a step, 2^-24, of it, as much as the lse's own rounding is; sums are fp32, two of a lane and sub-tile at most.
//   few   up to 32 rows (a decode step), as one or two operands of 16: 16x16x32_bf16 (fp32 rows: 16x16x4_f32), lane (c, g) = (l % 16, l / 16) holds the rows
//         4 g + j of each 16 for entry c.  A wave keeps them and goes over tiles of 32 entries, one on its way while another is worked on
//   many  32x32x16_bf16 (fp32 rows: 32x32x2_f32), lane (c, h) = (l % 32, l / 32) holds, of entry c, the rows 8 i + 4 h + j (i, j < 4) of each 32.
//         The waves of a block keep 32 kSubs entries each and go over stages of 64 rows, fetched straight into LDS while the stage before
//         is worked on.  A small kernel before it leaves, for every row, lse in units of log 2 and what it sees, and for every
//         stage the least and the most that a row of it sees: a block goes over the stages that see some of its entries alone.
// Few entries of many rows: the stages are also dealt out to splits in turn (where tokens see their past, late rows are seen by all entries,
// early ones by few), whose sums a last kernel adds in their order.
//
// few is bound by memory: 5 rows over 32768 entries of each of 128 units, 128 x bf16 (1.1 GB), 212 us, 5.2 TB/s, the rate of a large copy.  many is bound by the
// products and the multiply-add, exponential and addition beside each of their results: 4096 tokens of 40 / 8 heads over their past (86 GFLOP) 110 us with
// 5 + 5 for the kernels around it, 780 TFLOP/s, against 1220 of a bf16 product of 8192^3 on the same card; by counters the matrix cores are busy in 34 % of
// the cycles and vector units in 56, together most of the time.  Blocks in another order than that of their work: 181 us; 16 or 32 splits in place of 8: 115, 124;
// three blocks to a compute unit, of waves of 32 entries: 122.
#include "kernels.h"
#include "lazyev.h"
#include "rows.h"

#include <climits>

namespace lazyev {
namespace {

typedef unsigned short bf16_t;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(4))) int i32x4_t;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4_t;

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kStageRows = 64;
constexpr int kSplitMax = 64;

template <typename T, int D>
struct Rows {
  static constexpr bool kF32 = sizeof(T) == 4;
  static constexpr int kChunks = D * static_cast<int>(sizeof(T)) / 16;   // 16-byte chunks of a row
  static constexpr int kOps = kChunks / 2;         // chunks of a row that a lane holds as an operand
  static constexpr int kSubs = kF32 ? 1 : 2;       // (many) tiles of 32 entries that a wave keeps
  static constexpr int kEntries = 4 * 32 * kSubs;  // of a block
  // where chunk x of row r of a stage lies among the row's chunks: operands are read by 16 rows at a time, one chunk of each
  __device__ static int slot(int r, int x) { return x ^ (kChunks == 8 ? (r >> 1) & 7 : r & 15); }
};

// The row r of a unit among all rows of q; its token.
__device__ __forceinline__ long long row_of(const WeighArgs &a, int seq, int kvh, int r, long long &token) {
  const int i = quotient(r, a.group);
  token = static_cast<long long>(seq) * a.n_tokens + i;
  return token * a.n_q_heads + static_cast<long long>(kvh) * a.group + (r - i * a.group);
}

template <typename T, int D>
__device__ __forceinline__ void logits(const u32x4_t (&q)[Rows<T, D>::kOps], const u32x4_t (&k)[Rows<T, D>::kOps], f32x16_t &s) {
#pragma unroll
  for (int x = 0; x < 16; ++x) s[x] = 0.f;
#pragma unroll
  for (int j = 0; j < Rows<T, D>::kOps; ++j) {
    if constexpr (Rows<T, D>::kF32) {
#pragma unroll
      for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(q[j][e]), __uint_as_float(k[j][e]), s, 0, 0, 0);
    } else {
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, q[j]), __builtin_bit_cast(bf16x8_t, k[j]), s, 0, 0, 0);
    }
  }
}

// What an entry had before (known is 0 where decay is: nothing of it, whatever it holds).
__device__ __forceinline__ float before(const WeighArgs &a, long long at, int entry) { return entry < a.known ? a.decay * a.old[at] : 0.f; }

// The number of an entry's page, and where its keys lie there (any: some entry's).
__device__ __forceinline__ unsigned page_number(const WeighArgs &a, int seq, int entry) {
  return static_cast<unsigned>(a.pages.table[static_cast<long long>(seq) * a.pages.stride + page_of(a.pages, entry)]);
}
__device__ __forceinline__ size_t key_row(const WeighArgs &a, int kvh, int entry, unsigned no, bool &there) {
  const int pg = page_of(a.pages, entry);
  const unsigned head_rows = static_cast<unsigned>(a.pages.page_size), page_rows = head_rows * static_cast<unsigned>(a.n_kv_heads);
  there = no < static_cast<unsigned>(a.pages.n_pages);
  return (there ? no : 0u) * page_rows + kvh * head_rows + static_cast<unsigned>(entry - pg * a.pages.page_size);
}

// ------------------------------------------------------------------------------------ few rows

// Blocks of 256: wave w of block x of a unit has the tiles of 32 entries 4 x + w, and every 4 a.across further, in halves of 16: 16x16x32_bf16 (fp32
// rows: 16x16x4_f32), lane (c, g) = (l % 16, l / 16) holds the rows 4 g + j of each 16 for entry c, and a load of keys has 64 bytes
// of each of 16 entries.  kTiles: tiles of 16 rows.
template <typename T, int D, int kTiles>
__global__ __launch_bounds__(256) void weigh_few_kernel(const WeighArgs a) {
  using R = Rows<T, D>;
  constexpr int kOps = R::kChunks / 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = lane & 15, g = lane >> 4;
  const int unit = static_cast<int>(blockIdx.x) / a.across, x0 = static_cast<int>(blockIdx.x) - unit * a.across;
  const int seq = unit / a.n_kv_heads, kvh = unit - seq * a.n_kv_heads;
  const int M = a.n_tokens * a.group, tiles = (a.length + 31) / 32, step = 4 * a.across;
  int tile = 4 * x0 + wave;
  if (tile >= tiles) return;
  bool there[2][2];
  u32x4_t k[2][2][kOps];
  // (page numbers are asked for before the keys of the tile before: who waits for them does not wait for keys that are not needed yet.  32768
  // entries of 128 units, 5 rows each: 228 -> 212 us.  What the entries had before, asked for like that too: 219)
  unsigned no[2][2];
  auto numbers = [&](int tl, int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int y = 0; y < 2; ++y) no[buf][y] = page_number(a, seq, min(tl * 32 + 16 * y + c, a.length - 1));
  };
  auto fetch = [&](int tl, int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const char *from = static_cast<const char *>(a.k_pages) + key_row(a, kvh, min(tl * 32 + 16 * y + c, a.length - 1), no[buf][y], there[buf][y]) * (D * sizeof(T)) + g * 16;
#pragma unroll
      for (int j = 0; j < kOps; ++j) k[buf][y][j] = *reinterpret_cast<const u32x4_t *>(from + j * 64);
    }
  };
  numbers(tile, 0);
  numbers(min(tile + step, tiles - 1), 1);
  fetch(tile, 0);
  u32x4_t q[kTiles][kOps];
  long long token;
  float ref[kTiles][4];
  int sees[kTiles][4], least = INT_MAX;
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    const T *from = static_cast<const T *>(a.q) + row_of(a, seq, kvh, min(16 * t + c, M - 1), token) * D + g * (16 / sizeof(T));
#pragma unroll
    for (int j = 0; j < kOps; ++j) q[t][j] = load_chunk(from + j * (64 / sizeof(T)), a.wide);
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int r = 16 * t + 4 * g + x;
      const long long row = row_of(a, seq, kvh, min(r, M - 1), token);
      const float lse = a.lse[row];
      int n = a.visible ? min(max(a.visible[token], 0), a.length) : a.length;
      if (r >= M || lse == -INFINITY) n = 0;
      ref[t][x] = n > 0 ? lse * kLog2e : 0.f;
      sees[t][x] = n;
      least = min(least, r < M ? n : a.length);
    }
  }
  // (rows past the last do not add: the masks of a tile that all rows see leave out whole lanes)
  const float c2 = a.scale * kLog2e;
  auto work = [&](int tl, int buf) __attribute__((always_inline)) {
    const bool all = __builtin_amdgcn_ballot_w64(least < min(tl * 32 + 32, a.length)) == 0;   // (wave-uniform)
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int entry = tl * 32 + 16 * y + c;
      float w = 0.f;
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        f32x4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < kOps; ++j) {
          if constexpr (R::kF32) {
#pragma unroll
            for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(q[t][j][e]), __uint_as_float(k[buf][y][j][e]), s, 0, 0, 0);
          } else {
            s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, q[t][j]), __builtin_bit_cast(bf16x8_t, k[buf][y][j]), s, 0, 0, 0);
          }
        }
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const float p = __builtin_amdgcn_exp2f(fmaf(s[x], c2, -ref[t][x]));
          w += (all ? 16 * t + 4 * g + x < M : entry < sees[t][x]) ? p : 0.f;
        }
      }
      const auto r16 = __builtin_amdgcn_permlane16_swap(__float_as_uint(w), __float_as_uint(w), false, false);
      w = __uint_as_float(r16[0]) + __uint_as_float(r16[1]);
      const auto r32 = __builtin_amdgcn_permlane32_swap(__float_as_uint(w), __float_as_uint(w), false, false);
      w = there[buf][y] ? __uint_as_float(r32[0]) + __uint_as_float(r32[1]) : 0.f;
      if (g == 0 && entry < a.length) a.weights[static_cast<long long>(unit) * a.stride + entry] = before(a, static_cast<long long>(unit) * a.stride + entry, entry) + w;
    }
  };
  while (true) {
    numbers(min(tile + 2 * step, tiles - 1), 0);
    if (tile + step < tiles) fetch(tile + step, 1);
    work(tile, 0);
    tile += step;
    if (tile >= tiles) break;
    numbers(min(tile + 2 * step, tiles - 1), 1);
    if (tile + step < tiles) fetch(tile + step, 0);
    work(tile, 1);
    tile += step;
    if (tile >= tiles) break;
  }
}

// ------------------------------------------------------------------------------------ many rows

// Rows [units][stages][64]: lse in units of log 2, entries that the row sees; of a stage the least and the most that one sees.
__global__ __launch_bounds__(256) void weigh_rows_kernel(const WeighArgs a) {
  const int M = a.n_tokens * a.group;
  const long long at = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x, stage = at / kStageRows;
  const int unit = static_cast<int>(stage / a.stages);
  if (unit >= a.n_seqs * a.n_kv_heads) return;
  const int r = static_cast<int>(at - static_cast<long long>(unit) * a.stages * kStageRows);
  const int seq = unit / a.n_kv_heads, kvh = unit - seq * a.n_kv_heads;
  long long token;
  const long long row = row_of(a, seq, kvh, min(r, M - 1), token);
  const float lse = a.lse[row];
  int sees = a.visible ? min(max(a.visible[token], 0), a.length) : a.length;
  if (r >= M || lse == -INFINITY) sees = 0;
  a.row_lse[at] = sees > 0 ? lse * kLog2e : 0.f;
  a.row_sees[at] = sees;
  int least = sees, most = sees;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    least = min(least, __shfl_xor(least, o));
    most = max(most, __shfl_xor(most, o));
  }
  if ((threadIdx.x & 63) == 0) a.stage_sees[stage] = make_int2(least, most);
}

constexpr int kList = 1024;             // stages of a block's turn

template <typename T, int D>
__global__ __launch_bounds__(256, 2) void weigh_many_kernel(const WeighArgs a) {
  using R = Rows<T, D>;
  constexpr int kOps = R::kOps, C = R::kChunks, kSubs = R::kSubs;
  constexpr int kStage = kStageRows * C * 16;      // bytes
  constexpr int kPerLoad = 64 / C, kLoads = kStageRows / (kPerLoad * 4);   // rows of a wave's load of 1 KB, loads of a wave
  __shared__ __align__(16) char stages[2 * kStage];
  __shared__ __align__(16) float row_lse[2][kStageRows];
  __shared__ __align__(16) int row_sees[2][kStageRows];
  __shared__ int list[kList], list_least[kList], list_most[kList], counts[4][4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 31, h = lane >> 5;
  // early entries first: where tokens see their past, they have the most rows.  Units next: those of eight units share an XCD and its L2
  const int units = a.n_seqs * a.n_kv_heads, x0 = static_cast<int>(blockIdx.x / units), unit = static_cast<int>(blockIdx.x) - x0 * units;
  const int split = x0 % a.n_split, seq = unit / a.n_kv_heads, kvh = unit - seq * a.n_kv_heads;
  const int block_e0 = x0 / a.n_split * R::kEntries, e0 = block_e0 + wave * 32 * kSubs;
  const int M = a.n_tokens * a.group;
  bool there[kSubs];
  u32x4_t k[kSubs][kOps];
#pragma unroll
  for (int x = 0; x < kSubs; ++x) {
    const char *from = static_cast<const char *>(a.k_pages) + key_row(a, kvh, min(e0 + 32 * x + c, a.length - 1), page_number(a, seq, min(e0 + 32 * x + c, a.length - 1)), there[x]) * (D * sizeof(T)) + h * 16;
#pragma unroll
    for (int j = 0; j < kOps; ++j) k[x][j] = *reinterpret_cast<const u32x4_t *>(from + j * 32);
  }
  const unsigned stages_at = static_cast<unsigned>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char *)stages));
  const unsigned lse_at = static_cast<unsigned>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char *)row_lse));
  const unsigned sees_at = static_cast<unsigned>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char *)row_sees));
  // A stage's rows and what is known of them to LDS, straight from memory where the rows lie at multiples of 16 bytes.  (Written out, as the compiler
  // has every read of LDS wait for all loads into it: they leave nothing in registers, and the waits for them are in `arrived`.)
  const float *lse_from = a.row_lse + static_cast<size_t>(unit) * a.stages * kStageRows;
  const int *sees_from = a.row_sees + static_cast<size_t>(unit) * a.stages * kStageRows;
  auto fetch = [&](int stage, int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int r = (u * 4 + wave) * kPerLoad + lane / C;
      long long token;
      const T *row = static_cast<const T *>(a.q) + row_of(a, seq, kvh, min(stage * kStageRows + r, M - 1), token) * D + R::slot(r, lane % C) * (16 / sizeof(T));
      const unsigned at = buf * kStage + (u * 4 + wave) * 1024;
      if (a.wide) {
        __asm__ volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(stages_at + at), "v"(row) : "memory", "m0");
      } else {
        *reinterpret_cast<u32x4_t *>(stages + at + lane * 16) = load_chunk(row, false);
      }
    }
    if (wave < 2) {
      const void *from = wave == 0 ? static_cast<const void *>(lse_from + stage * kStageRows + lane) : sees_from + stage * kStageRows + lane;
      const unsigned at = (wave == 0 ? lse_at : sees_at) + buf * (kStageRows * 4);
      __asm__ volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(at), "v"(from) : "memory", "m0");
    }
  };
  auto arrived = [&]() __attribute__((always_inline)) {
    __asm__ volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(7 << 4);            // vmcnt(0), lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    __asm__ volatile("" ::: "memory");
  };
  const float c2 = a.scale * kLog2e;
  float sum[kSubs][2];
#pragma unroll
  for (int x = 0; x < kSubs; ++x) sum[x][0] = sum[x][1] = 0.f;
  int q_at[kOps];
#pragma unroll
  for (int j = 0; j < kOps; ++j) q_at[j] = (c * C + R::slot(c, 2 * j + h)) * 16;
  auto work = [&](int buf, bool mask) __attribute__((always_inline)) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      u32x4_t q[kOps];
#pragma unroll
      for (int j = 0; j < kOps; ++j) q[j] = *reinterpret_cast<const u32x4_t *>(stages + buf * kStage + half * 32 * C * 16 + q_at[j]);
      f32x4_t ref[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) ref[x] = *reinterpret_cast<const f32x4_t *>(&row_lse[buf][half * 32 + 8 * x + 4 * h]);
#pragma unroll
      for (int x = 0; x < kSubs; ++x) {
        f32x16_t s;
        logits<T, D>(q, k[x], s);
        if (mask) {                                // (what a row does not see has nothing of its lse either, a NaN for instance)
          const int entry = e0 + 32 * x + c;
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const i32x4_t limit = *reinterpret_cast<const i32x4_t *>(&row_sees[buf][half * 32 + 8 * y + 4 * h]);
#pragma unroll
            for (int z = 0; z < 4; ++z) sum[x][z & 1] += __builtin_amdgcn_exp2f(entry < limit[z] ? fmaf(s[4 * y + z], c2, -ref[y][z]) : -INFINITY);
          }
        } else {
#pragma unroll
          for (int y = 0; y < 16; ++y) sum[x][y & 1] += __builtin_amdgcn_exp2f(fmaf(s[y], c2, -ref[y / 4][y % 4]));
        }
      }
    }
  };
  const int mine = split < a.stages ? (a.stages - split + a.n_split - 1) / a.n_split : 0;   // stages of this split
  const int2 *stage_sees = a.stage_sees + static_cast<size_t>(unit) * a.stages;
#pragma unroll 1
  for (int w0 = 0; w0 < mine; w0 += kList) {
    // those of the next kList that see some of the block's entries, in their order
    int at = 0;
    __syncthreads();
#pragma unroll 1
    for (int x = 0; x < kList && w0 + x < mine; x += 256) {
      const int i = w0 + x + static_cast<int>(threadIdx.x), stage = split + i * a.n_split;
      const int2 s = i < mine ? stage_sees[stage] : make_int2(0, 0);
      const unsigned long long m = __builtin_amdgcn_ballot_w64(s.y > block_e0);
      if (lane == 0) counts[x / 256][wave] = __popcll(m);
      __syncthreads();
      int before_wave = at;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        before_wave += w < wave ? counts[x / 256][w] : 0;
        at += counts[x / 256][w];
      }
      if (s.y > block_e0) {
        const int to = before_wave + __popcll(m & ((1ull << lane) - 1));
        list[to] = stage;
        list_least[to] = s.x;
        list_most[to] = s.y;
      }
    }
    __syncthreads();
    const int n = __builtin_amdgcn_readfirstlane(at);
    if (n > 0) fetch(__builtin_amdgcn_readfirstlane(list[0]), 0);
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
      const int least = __builtin_amdgcn_readfirstlane(list_least[i]), most = __builtin_amdgcn_readfirstlane(list_most[i]);
      const int next = __builtin_amdgcn_readfirstlane(list[min(i + 1, n - 1)]);
      arrived();
      if (i + 1 < n) fetch(next, (i + 1) & 1);
      if (most <= e0) continue;                    // (wave-uniform)
      if (least >= e0 + 32 * kSubs) work(i & 1, false);
      else work(i & 1, true);
    }
  }
#pragma unroll
  for (int x = 0; x < kSubs; ++x) {
    float w = sum[x][0] + sum[x][1];
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(w), __float_as_uint(w), false, false);
    w = there[x] ? __uint_as_float(both[0]) + __uint_as_float(both[1]) : 0.f;
    const int entry = e0 + 32 * x + c;
    if (h != 0 || entry >= a.length) continue;
    if (a.n_split > 1) {
      a.part[(static_cast<size_t>(split) * a.n_seqs * a.n_kv_heads + unit) * a.length + entry] = w;
    } else {
      const long long at = static_cast<long long>(unit) * a.stride + entry;
      a.weights[at] = before(a, at, entry) + w;
    }
  }
}

__global__ __launch_bounds__(256) void weigh_join_kernel(const WeighArgs a) {
  const long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x, n = static_cast<long long>(a.n_seqs) * a.n_kv_heads * a.length;
  if (i >= n) return;
  const long long unit = i / a.length;
  const int entry = static_cast<int>(i - unit * a.length);
  float w = 0.f;
  for (int s = 0; s < a.n_split; ++s) w += a.part[static_cast<size_t>(s) * n + i];
  const long long at = unit * a.stride + entry;
  a.weights[at] = before(a, at, entry) + w;
}

// How a call is cut.
struct Plan { int many, across, stages, n_split; };
Plan plan_of(const WeighArgs &a) {
  Plan p = {0, 0, 0, 1};
  const int M = a.n_tokens * a.group, units = a.n_seqs * a.n_kv_heads;
  p.many = M > 32;
  if (!p.many) {                                   // (four blocks a compute unit, a few tiles a wave where there are so many)
    const int blocks = ((a.length + 31) / 32 + 3) / 4, most = (1024 + units - 1) / units;
    p.across = blocks < most ? blocks : most;
    return p;
  }
  const int entries = a.dtype == LAZYEV_DTYPE_FP32 ? Rows<float, 64>::kEntries : Rows<bf16_t, 64>::kEntries;
  p.across = (a.length + entries - 1) / entries;
  p.stages = (M + kStageRows - 1) / kStageRows;
  const long long blocks = static_cast<long long>(units) * p.across;
  long long n = 1024 / blocks;                     // (late blocks have less to do where tokens see their past: four for a compute unit)
  if (n > p.stages / 4) n = p.stages / 4;
  p.n_split = static_cast<int>(n < 1 ? 1 : n > kSplitMax ? kSplitMax : n);
  return p;
}

size_t align_up(size_t x) { return (x + 255) / 256 * 256; }
size_t rows_of(const WeighArgs &a, const Plan &p) { return static_cast<size_t>(a.n_seqs) * a.n_kv_heads * p.stages * kStageRows; }
size_t parts_of(const WeighArgs &a, const Plan &p) {
  return p.n_split > 1 ? align_up(static_cast<size_t>(p.n_split) * a.n_seqs * a.n_kv_heads * a.length * 4) : 0;
}

template <typename T, int D>
hipError_t launch(const WeighArgs &a, const Plan &p, hipStream_t stream) {
  const long long blocks = static_cast<long long>(a.n_seqs) * a.n_kv_heads * p.across * p.n_split;
  if (blocks < 1 || blocks >= (1ll << 24)) return hipErrorInvalidValue;
  const dim3 grid(static_cast<unsigned>(blocks));
  if (p.many) {
    hipLaunchKernelGGL((weigh_many_kernel<T, D>), grid, dim3(256), 0, stream, a);
    return hipGetLastError();
  }
  if (a.n_tokens * a.group <= 16) hipLaunchKernelGGL((weigh_few_kernel<T, D, 1>), grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((weigh_few_kernel<T, D, 2>), grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

size_t weigh_workspace(const WeighArgs &a) {
  const Plan p = plan_of(a);
  if (!p.many) return 0;
  return 2 * align_up(rows_of(a, p) * 4) + align_up(rows_of(a, p) / kStageRows * sizeof(int2)) + parts_of(a, p);
}

hipError_t launch_weigh(WeighArgs a, hipStream_t stream) {
  const Plan p = plan_of(a);
  a.across = p.across;
  a.stages = p.stages;
  a.n_split = p.n_split;
  a.wide = reinterpret_cast<uintptr_t>(a.q) % 16 == 0;
  const long long n = static_cast<long long>(a.n_seqs) * a.n_kv_heads * a.length;
  hipError_t e;
  if (a.n_tokens == 0) {                           // what there was before, alone
    a.n_split = 0;
    hipLaunchKernelGGL(weigh_join_kernel, dim3(static_cast<unsigned>((n + 255) / 256)), dim3(256), 0, stream, a);
    return hipGetLastError();
  }
  if (p.many) {
    const size_t rows = rows_of(a, p);
    char *w = static_cast<char *>(a.workspace);
    a.row_lse = reinterpret_cast<float *>(w);
    w += align_up(rows * 4);
    a.row_sees = reinterpret_cast<int32_t *>(w);
    w += align_up(rows * 4);
    a.stage_sees = reinterpret_cast<int2 *>(w);
    w += align_up(rows / kStageRows * sizeof(int2));
    a.part = reinterpret_cast<float *>(w);
    if ((rows + 255) / 256 >= (1u << 24)) return hipErrorInvalidValue;
    hipLaunchKernelGGL(weigh_rows_kernel, dim3(static_cast<unsigned>((rows + 255) / 256)), dim3(256), 0, stream, a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.dtype == LAZYEV_DTYPE_FP32) e = a.head_dim == 64 ? launch<float, 64>(a, p, stream) : launch<float, 128>(a, p, stream);
  else e = a.head_dim == 64 ? launch<bf16_t, 64>(a, p, stream) : launch<bf16_t, 128>(a, p, stream);
  if (e != hipSuccess || p.n_split <= 1) return e;
  hipLaunchKernelGGL(weigh_join_kernel, dim3(static_cast<unsigned>((n + 255) / 256)), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace lazyev
