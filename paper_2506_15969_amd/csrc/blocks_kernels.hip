// Blocks of a long cache: bounds of their keys (lazyev_blocks_bound) and the blocks that a token reads (lazyev_blocks_choose).
//
// Bounds.  lo[e], hi[e] = smallest and largest element e of the block's keys.  A wave takes a block: its rows in 16-byte chunks, 1 KB
// a load, minima and maxima in fp32 (exact), then over the lanes that hold the same chunk.  16384 keys of 8 heads (35 MB) 8.6 us: latency, as each of
// 2048 waves asks four times for four rows to a lane, one after the other (all at once, or four waves to a block: no faster; comparisons in place of
// three-operand minima: 11.7); a key each of 128 units 3.4 us.
//
// Choice.  score(b) = max over the heads g of the group of sum_e max(q_ge lo_be, q_ge hi_be): of the keys between the bounds none has a
// larger product with any of the queries.  The larger of the two terms is the one with hi where q_ge > 0 and with lo where q_ge < 0, so
// the sums are products of matrices, [q+ | q-] [hi | lo]^T with twice the length, on matrix instructions:
//   16x16x32_bf16 (fp32 rows: 16x16x4_f32), rows of q as A, blocks as B: lane (c, g) = (l % 16, l / 16) holds, of block c,
//   the sums of the rows 4 g + i (i < 4)
// Rows are heads, every token's filled up to a power of two of them with copies of its last, so that the maximum over a group is one of registers.
// Numbers that rank are to be the exact ones, whatever order a sum is taken in, and these sums are rounded: each of at most 128 terms that are not zero
// (the products of bf16 elements are exact) comes with an addition, off by at most 2^-22 of what is added up so far whichever way the
// matrix instruction rounds, fp32 products with another rounding: a score is within E = 2^-15 max_g |q_g| max_b |bound_b| (fp32 rows: 2^-14; Euclidean
// norms, of the larger bound of each element in size) of the exact one.
// With T the largest but k - 1 of the rounded scores, the exact score of a block
//   beyond T + 2 E is among the k best: it is above T + E, and so are only blocks whose rounded score is above T, at most k - 1
//   below T - 2 E is not: it is below T - E, and the k blocks from T on are not
// and those between, a few, are summed again in binary64, where products are exact and equal blocks give equal sums.
//
// Measured, us for scores and choice: a token each of 16 sequences, 40 / 8 heads, 3126 blocks of 128 x bf16 (205 MB of bounds) 41 + 14.8, the first at 5.0 TB/s; 640
// tokens of 28 / 4 heads, 512 blocks 17.4 + 14.9; 3 x 33 tokens of 32 / 8 heads of 64 x fp32, 313 blocks 12.5 + 10.6.  The second kernel is a chain of latencies: scores,
// border (6 us), places (3), and the sums in binary64 that the slowest row asks for (3 - 5).  Scores that stay in LDS, one kernel for a tile of tokens: 53 us
// in place of 36 for the 640 tokens.
#include "kernels.h"
#include "lanes.h"
#include "lazyev.h"
#include "rows.h"

#include <cfloat>
#include <climits>

namespace lazyev {
namespace {

typedef unsigned short bf16_t;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4_t;

__device__ __forceinline__ float bf16_low(unsigned w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(unsigned w) { return __uint_as_float(w & 0xFFFF0000u); }

// (a NaN stays: v_minimum3_f32, v_maximum3_f32)
__device__ __forceinline__ float lower(float m, float x) { return __builtin_elementwise_minimum(m, x); }
__device__ __forceinline__ float upper(float m, float x) { return __builtin_elementwise_maximum(m, x); }

// ------------------------------------------------------------------------------------ bounds

template <typename T, int D>
__global__ __launch_bounds__(256) void bound_kernel(const BoundArgs a) {
  constexpr bool kF32 = sizeof(T) == 4;
  constexpr int C = D * static_cast<int>(sizeof(T)) / 16, kRows = 64 / C, kElems = 16 / static_cast<int>(sizeof(T));
  constexpr int kAhead = 4;                        // loads of a wave on their way together
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const long long at = static_cast<long long>(blockIdx.x) * 4 + wave;
  if (at >= static_cast<long long>(a.units) * a.touched) return;
  const int unit = static_cast<int>(at / a.touched), b = a.first_block + static_cast<int>(at - static_cast<long long>(unit) * a.touched);
  const int seq = unit / a.n_kv_heads, kvh = unit - seq * a.n_kv_heads;
  const int32_t *table = a.pages.table + static_cast<long long>(seq) * a.pages.stride;
  const unsigned head_rows = static_cast<unsigned>(a.pages.page_size), page_rows = head_rows * static_cast<unsigned>(a.n_kv_heads);
  const int first = max(a.start, b * a.block), end = min(a.end, (b + 1) * a.block);
  const int chunk = lane % C;
  float lo[kElems], hi[kElems];
#pragma unroll
  for (int e = 0; e < kElems; ++e) {
    lo[e] = INFINITY;
    hi[e] = -INFINITY;
  }
  auto count = [&](u32x4_t w) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < kElems; ++e) {
      const float x = kF32 ? __uint_as_float(w[e % 4]) : e % 2 ? bf16_high(w[e / 2]) : bf16_low(w[e / 2]);
      lo[e] = lower(lo[e], x);
      hi[e] = upper(hi[e], x);
    }
  };
  for (int e0 = first + lane / C; e0 - lane / C < end; e0 += kRows * kAhead) {
    u32x4_t w[kAhead];
    bool there[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int entry = min(e0 + u * kRows, end - 1), pg = page_of(a.pages, entry);
      const unsigned no = static_cast<unsigned>(table[pg]);
      there[u] = e0 + u * kRows < end && no < static_cast<unsigned>(a.pages.n_pages);
      const unsigned row = (there[u] ? no : 0u) * page_rows + kvh * head_rows + static_cast<unsigned>(entry - pg * a.pages.page_size);
      w[u] = *reinterpret_cast<const u32x4_t *>(static_cast<const char *>(a.k_pages) + static_cast<size_t>(row) * (D * sizeof(T)) + chunk * 16);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (there[u]) count(w[u]);
  }
  char *to = static_cast<char *>(a.bounds) + (static_cast<size_t>(unit) * a.n_blocks + b) * (2 * D * sizeof(T)) + chunk * 16;
  if (b * a.block < a.start) {                     // entries before have been counted
    const u32x4_t l = *reinterpret_cast<const u32x4_t *>(to), u = *reinterpret_cast<const u32x4_t *>(to + D * sizeof(T));
#pragma unroll
    for (int e = 0; e < kElems; ++e) {
      lo[e] = lower(lo[e], kF32 ? __uint_as_float(l[e % 4]) : e % 2 ? bf16_high(l[e / 2]) : bf16_low(l[e / 2]));
      hi[e] = upper(hi[e], kF32 ? __uint_as_float(u[e % 4]) : e % 2 ? bf16_high(u[e / 2]) : bf16_low(u[e / 2]));
    }
  }
#pragma unroll
  for (int e = 0; e < kElems; ++e) {
    lo[e] = join_lanes<C, 32>(lo[e], lower);
    hi[e] = join_lanes<C, 32>(hi[e], upper);
  }
  if (lane >= 2 * C) return;                       // (the first C lanes store the lower bounds, the next ones the upper)
  const bool up = lane >= C;
  u32x4_t w;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (kF32) w[e] = __float_as_uint(up ? hi[e] : lo[e]);
    else w[e] = __float_as_uint(up ? hi[2 * e] : lo[2 * e]) >> 16 | (__float_as_uint(up ? hi[2 * e + 1] : lo[2 * e + 1]) & 0xFFFF0000u);
  }
  *reinterpret_cast<u32x4_t *>(to + (up ? D * sizeof(T) : 0)) = w;
}

// ------------------------------------------------------------------------------------ scores

// 16 bytes of a row of queries: its elements above zero, and those below.  (Of a NaN's two copies one is a NaN.)
template <bool kF32>
__device__ __forceinline__ void by_sign(u32x4_t w, u32x4_t &pos, u32x4_t &neg) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    unsigned minus;
    const unsigned high = static_cast<unsigned>(static_cast<int>(w[e]) >> 31), low = static_cast<unsigned>(static_cast<int>(w[e] << 16) >> 31);
    if constexpr (kF32) minus = high;
    else minus = (high & 0xFFFF0000u) | (low & 0xFFFFu);
    pos[e] = w[e] & ~minus;
    neg[e] = w[e] & minus;
  }
}

// Squares of the larger one of each pair of elements, in size.  (A NaN does not show here: it does in the score.)
template <bool kF32>
__device__ __forceinline__ float squares_of(u32x4_t lo, u32x4_t hi, float sum) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (kF32) {
      const float x = fmaxf(fabsf(__uint_as_float(lo[e])), fabsf(__uint_as_float(hi[e])));
      sum = fmaf(x, x, sum);
    } else {
      const float x = fmaxf(fabsf(bf16_low(lo[e])), fabsf(bf16_low(hi[e]))), y = fmaxf(fabsf(bf16_high(lo[e])), fabsf(bf16_high(hi[e])));
      sum = fmaf(y, y, fmaf(x, x, sum));
    }
  }
  return sum;
}
// Not below the norm whose squares sum up to this: 128 roundings and the root's, and elements too small to have a square in fp32.
__device__ __forceinline__ float norm_of(float squares) { return sqrtf(squares) * (1.f + 0x1p-10f) + 0x1p-50f; }

__device__ __forceinline__ float add(float x, float y) { return x + y; }

// A wave has 16 kCols blocks of a unit (x: the unit and 64 kCols blocks of it) and goes over the tokens of its share (y) of the launch's, 16 / kPad of
// them at a time, the next ones' queries on their way; a token's group of more than 16 heads comes in passes of 16.  (A load brings 64 bytes of each of 16
// rows: 32 rows to an operand, and 32 bytes of each, take the address units twice as long, which was what bound it.)
template <typename T, int D, int kPad, int kCols>
__global__ __launch_bounds__(256) void score_kernel(const ChooseArgs a) {
  constexpr bool kF32 = sizeof(T) == 4;
  constexpr int kOps = D * static_cast<int>(sizeof(T)) / 64, kTokens = 16 / kPad, kBlocks = 16 * kCols;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = lane & 15, g = lane >> 4;
  const int across = (a.scored + 4 * kBlocks - 1) / (4 * kBlocks), unit = static_cast<int>(blockIdx.x) / across;
  const int seq = unit / a.n_kv_heads, kvh = unit - seq * a.n_kv_heads;
  const int b0 = (static_cast<int>(blockIdx.x) - unit * across) * (4 * kBlocks) + wave * kBlocks;
  if (b0 >= a.scored) return;
  const int tiles = (a.tokens + kTokens - 1) / kTokens, passes = kPad == 16 ? (a.group + 15) / 16 : 1;
  const T *queries = static_cast<const T *>(a.q) + static_cast<size_t>(kvh) * a.group * D + g * (16 / sizeof(T));
  // (asked for together, before one is used)
  auto load_row = [&](int tile, int pass, u32x4_t (&w)[kOps]) __attribute__((always_inline)) {
    const size_t token = static_cast<size_t>(seq) * a.n_tokens + a.token0 + min(tile * kTokens + c / kPad, a.tokens - 1);
    const T *p = queries + (token * a.n_q_heads + min(pass * 16 + c % kPad, a.group - 1)) * D;
    if (a.wide) {
#pragma unroll
      for (int j = 0; j < kOps; ++j) w[j] = *reinterpret_cast<const u32x4_t *>(p + j * (64 / sizeof(T)));
    } else {
#pragma unroll
      for (int j = 0; j < kOps; ++j) w[j] = load_chunk(p + j * (64 / sizeof(T)), false);
    }
  };
  u32x4_t lo[kCols][kOps], hi[kCols][kOps], q[kOps];
#pragma unroll
  for (int x = 0; x < kCols; ++x) {
    const char *from = static_cast<const char *>(a.bounds) + (static_cast<size_t>(unit) * a.n_blocks + min(b0 + 16 * x + c, a.scored - 1)) * (2 * D * sizeof(T)) + g * 16;
#pragma unroll
    for (int j = 0; j < kOps; ++j) lo[x][j] = *reinterpret_cast<const u32x4_t *>(from + j * 64);
#pragma unroll
    for (int j = 0; j < kOps; ++j) hi[x][j] = *reinterpret_cast<const u32x4_t *>(from + D * sizeof(T) + j * 64);
  }
  int tile = static_cast<int>(blockIdx.y);
  if (tile < tiles) load_row(tile, 0, q);
  if (blockIdx.y == 0) {
#pragma unroll
    for (int x = 0; x < kCols; ++x) {
      float m = 0.f;
#pragma unroll
      for (int j = 0; j < kOps; ++j) m = squares_of<kF32>(lo[x][j], hi[x][j], m);
      m = norm_of(join_lanes<16, 32>(m, add));
      if (g == 0 && b0 + 16 * x + c < a.scored) a.peak[static_cast<size_t>(unit) * a.scored + b0 + 16 * x + c] = m;
    }
  }
  for (; tile < tiles; tile += static_cast<int>(gridDim.y)) {
    float top[kCols], out[kCols][4];
#pragma unroll
    for (int x = 0; x < kCols; ++x) top[x] = -INFINITY;
    for (int pass = 0; pass < passes; ++pass) {
      const bool last = pass + 1 == passes;
      u32x4_t next[kOps];
      load_row(last ? min(tile + static_cast<int>(gridDim.y), tiles - 1) : tile, last ? 0 : pass + 1, next);
      f32x4_t s[kCols];
#pragma unroll
      for (int x = 0; x < kCols; ++x) s[x] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < kOps; ++j) {
        u32x4_t pos, neg;
        by_sign<kF32>(q[j], pos, neg);
#pragma unroll
        for (int x = 0; x < kCols; ++x) {
          if constexpr (kF32) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              s[x] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(pos[e]), __uint_as_float(hi[x][j][e]), s[x], 0, 0, 0);
              s[x] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(neg[e]), __uint_as_float(lo[x][j][e]), s[x], 0, 0, 0);
            }
          } else {
            s[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, pos), __builtin_bit_cast(bf16x8_t, hi[x][j]), s[x], 0, 0, 0);
            s[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, neg), __builtin_bit_cast(bf16x8_t, lo[x][j]), s[x], 0, 0, 0);
          }
        }
      }
#pragma unroll
      for (int j = 0; j < kOps; ++j) q[j] = next[j];
      // rows 4 g + i in s[i]: the maxima of kPad rows next to one another
#pragma unroll
      for (int x = 0; x < kCols; ++x) {
        if constexpr (kPad == 1) {
#pragma unroll
          for (int i = 0; i < 4; ++i) out[x][i] = s[x][i];
        } else if constexpr (kPad == 2) {
          out[x][0] = upper(s[x][0], s[x][1]);
          out[x][1] = upper(s[x][2], s[x][3]);
        } else {
          float m = upper(upper(s[x][0], s[x][1]), upper(s[x][2], s[x][3]));
          if constexpr (kPad > 4) m = join_step<16>(m, upper);
          if constexpr (kPad > 8) m = join_step<32>(m, upper);
          out[x][0] = top[x] = upper(top[x], m);
        }
      }
    }
    auto put = [&](int t, int x, float y) __attribute__((always_inline)) {
      const int b = b0 + 16 * x + c;
      t += tile * kTokens;
      if (t < a.tokens && b < a.scored) a.score[((static_cast<size_t>(seq) * a.tokens + t) * a.n_kv_heads + kvh) * a.scored + b] = y;
    };
#pragma unroll
    for (int x = 0; x < kCols; ++x) {
      if constexpr (kPad == 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) put(4 * g + i, x, out[x][i]);
      } else if constexpr (kPad == 2) {
        put(2 * g, x, out[x][0]);
        put(2 * g + 1, x, out[x][1]);
      } else if constexpr (kPad == 4) {
        put(g, x, out[x][0]);
      } else if constexpr (kPad == 8) {
        if ((g & 1) == 0) put(g / 2, x, out[x][0]);
      } else {
        if (g == 0) put(0, x, out[x][0]);
      }
    }
  }
}

// ------------------------------------------------------------------------------------ choice

// Numbers in the order of the values (a NaN: the largest); 0 is below all of them.
__device__ __forceinline__ unsigned order_of(float x) {
  const unsigned u = __float_as_uint(x + 0.f);     // (-0 and 0 are one)
  return x != x ? 0xFFFFFFFFu : u ^ (static_cast<unsigned>(static_cast<int>(u) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(unsigned k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }
__device__ __forceinline__ unsigned long long order_of(double x) {
  const unsigned long long u = __double_as_longlong(x + 0.0);
  return x != x ? ~0ull : u ^ (static_cast<unsigned long long>(static_cast<long long>(u) >> 63) | 1ull << 63);
}

constexpr int kAgain = 512;             // blocks between the borders whose exact scores a row holds

// What a row's waves share.
template <int kWaves, int kRegs>
struct Room {
  int i[2][kWaves];
  unsigned u[2][kWaves];
  float f[2][kWaves];
  double exact[kAgain];
  int again[kAgain], look_count[kRegs > 0 ? kRegs * kWaves : 1];
};
// What the waves of a row have written is there for all of them.
template <int kWaves>
__device__ __forceinline__ void together() {
  if constexpr (kWaves > 1) {
    __syncthreads();
  } else {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }
}

// x of all waves, by `join`; LDS of one number a wave, of which two take turns.
template <int kWaves, typename V, typename F>
__device__ __forceinline__ V over_waves(V x, V (&room)[2][kWaves], int &turn, F join) {
  if constexpr (kWaves > 1) {
    if ((threadIdx.x & 63) == 0) room[turn][threadIdx.x >> 6] = x;
    __syncthreads();
    x = room[turn][0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) x = join(x, room[turn][w]);
    turn ^= 1;
  }
  return x;
}

// The choice of a token and KV head (row: of the launch's), by kWaves waves.  Its candidates' scores stay in registers, kRegs for a thread (candidate
// 64 (x kWaves + wave) + lane is x of a lane); 0: there are more of them, and they are read anew for every look.
// T is not needed to its last bit: an interval of T no wider than E does, so the bits of its order are settled from the first one in which candidates
// differ to about the fourteenth behind, by counts of the candidates from a number on.
template <typename T, int D, int kWaves, int kRegs>
__device__ __forceinline__ void choose_row(const ChooseArgs &a, unsigned row, Room<kWaves, kRegs> &room, const float *scores, const float *peaks) {
  constexpr bool kF32 = sizeof(T) == 4;
  constexpr int kBlock = 64 * kWaves, C = D * static_cast<int>(sizeof(T)) / 16, kElems = 16 / static_cast<int>(sizeof(T));
  constexpr int kLooks = kRegs * kWaves, kHeld = kRegs > 0 ? kRegs : 1;
  const int lane = threadIdx.x & 63, wave = kWaves > 1 ? threadIdx.x >> 6 : 0, thread = wave * 64 + lane;
  const unsigned its = row / a.n_kv_heads;         // (sequence, token of the launch)
  const int kvh = static_cast<int>(row - its * a.n_kv_heads), seq = static_cast<int>(its / a.tokens), t = static_cast<int>(its - seq * a.tokens);
  const long long token = static_cast<long long>(seq) * a.n_tokens + a.token0 + t;
  int32_t *to = a.chosen + (token * a.n_kv_heads + kvh) * a.n_chosen;
  const int seen = a.visible ? min(max(a.visible[token], 0), a.length) : a.length;
  const int nb = (seen + a.block - 1) / a.block;
  if (nb <= a.n_chosen) {
    for (int i = thread; i < a.n_chosen; i += kBlock) to[i] = i < nb ? i : -1;
    return;
  }
  // candidates are the blocks first .. first + n - 1, of which `want` go
  const int n = nb - a.n_last - a.n_first, want = a.n_chosen - a.n_last - a.n_first;
  const size_t unit = static_cast<size_t>(seq) * a.n_kv_heads + kvh;
  const auto score = [&](int i) __attribute__((always_inline)) { return scores[i + a.n_first]; };
  const auto peak = [&](int i) __attribute__((always_inline)) { return peaks[i + a.n_first]; };
  const T *q = static_cast<const T *>(a.q) + (token * a.n_q_heads + static_cast<long long>(kvh) * a.group) * D;
  for (int i = thread; i < a.n_first; i += kBlock) to[i] = i;
  for (int i = thread; i < a.n_last; i += kBlock) to[a.n_chosen - a.n_last + i] = nb - a.n_last + i;
  if (want == 0) return;

  // the scores, their range, and how far one may be off
  unsigned held[kHeld];
  const int looks = kRegs > 0 ? kRegs : (n + kBlock - 1) / kBlock;
  auto at_look = [&](int x) __attribute__((always_inline)) { return (x * kWaves + wave) * 64 + lane; };
  auto each = [&](auto f) __attribute__((always_inline)) {   // f(candidate, its order or 0)
    if constexpr (kRegs > 0) {
#pragma unroll
      for (int x = 0; x < kRegs; ++x) f(x, held[x]);
    } else {
      for (int x = 0; x < looks; ++x) f(x, at_look(x) < n ? order_of(score(min(at_look(x), n - 1))) : 0u);
    }
  };
  float most = 0.f, size = 0.f;                    // largest norm of a block's bounds, and of a query
  bool odd = false, none = true;                   // a score that is no finite number; no element of a query but zeros
  unsigned top = 0u, least = 0xFFFFFFFFu;
  if constexpr (kRegs > 0) {
    float s[kHeld], p[kHeld];
#pragma unroll
    for (int x = 0; x < kRegs; ++x) {
      s[x] = p[x] = 0.f;
      if (at_look(x) < n) {
        s[x] = score(at_look(x));
        p[x] = peak(at_look(x));
      }
    }
#pragma unroll
    for (int x = 0; x < kRegs; ++x) {
      const bool is = at_look(x) < n;
      most = upper(most, p[x]);
      odd |= !(fabsf(s[x]) <= FLT_MAX);
      held[x] = is ? order_of(s[x]) : 0u;
      top = max(top, held[x]);
      least = min(least, is ? held[x] : 0xFFFFFFFFu);
    }
  } else {
    for (int i = thread; i < n; i += kBlock) {
      const float s = score(i);
      most = upper(most, peak(i));
      odd |= !(fabsf(s) <= FLT_MAX);
      top = max(top, order_of(s));
      least = min(least, order_of(s));
    }
  }
  for (int g0 = 0; g0 < a.group; g0 += kBlock / C) {
    const int g = min(g0 + thread / C, a.group - 1);
    const u32x4_t w = load_chunk(q + g * D + lane % C * kElems, a.wide);
    none &= ((w[0] | w[1] | w[2] | w[3]) & (kF32 ? 0x7FFFFFFFu : 0x7FFF7FFFu)) == 0;
    size = upper(size, norm_of(join_lanes<1, C / 2>(squares_of<kF32>(w, w, 0.f), add)));
  }
  size = join_lanes<C, 32>(size, upper);
  most = join_lanes<1, 32>(most, upper);
  top = join_lanes<1, 32>(top, [](unsigned x, unsigned y) { return max(x, y); });
  least = join_lanes<1, 32>(least, [](unsigned x, unsigned y) { return min(x, y); });
  int turn_f = 0, turn_u = 0, turn_i = 0;
  most = over_waves<kWaves>(most, room.f, turn_f, upper);
  size = over_waves<kWaves>(size, room.f, turn_f, upper);
  top = over_waves<kWaves>(top, room.u, turn_u, [](unsigned x, unsigned y) { return max(x, y); });
  least = over_waves<kWaves>(least, room.u, turn_u, [](unsigned x, unsigned y) { return min(x, y); });
  if constexpr (kWaves > 1) {
    odd = __syncthreads_or(odd);
    none = __syncthreads_and(none);
  } else {
    odd = __ballot(odd) != 0;
    none = __ballot(!none) == 0;
  }
  // (2^-100: products too small for fp32; none of a row of zeros)
  const float off = none && most <= FLT_MAX ? 0.f : size * most * (kF32 ? 0x1p-14f : 0x1p-15f) + 0x1p-100f;
  const bool all_again = odd || !(size * most < 0x1p120f);
  auto count_from = [&](unsigned cand) __attribute__((always_inline)) {
    int have = 0;                                  // (of the lane: counts of ballots take scalar registers that there are too few of)
    each([&](int, unsigned k) __attribute__((always_inline)) { have += k >= cand ? 1 : 0; });
    have = join_lanes<1, 32>(have, [](int x, int y) { return x + y; });
    return over_waves<kWaves>(have, room.i, turn_i, [](int x, int y) { return x + y; });
  };

  // the borders: surely taken from `sure` on, surely not below `out`
  unsigned sure = 0xFFFFFFFFu, out = 1u;
  if (!all_again) {
    // at least `want` are from `border` on, and fewer beyond border + span (or, found, just `want` from border on)
    int bits = 32 - __clz(static_cast<int>(top ^ least));      // (__clz(0) = 32)
    unsigned border = bits == 32 ? 0u : top >> bits << bits;
    bool found = false;
    while (bits > 0 && !found && !(value_of(border | (bits == 32 ? 0xFFFFFFFFu : (1u << bits) - 1)) - value_of(border) <= off)) {
      --bits;
      const unsigned cand = border | 1u << bits;
      const int have = count_from(cand);
      if (have >= want) border = cand;
      found = have == want;
    }
    const float low = value_of(border), high = found ? low : value_of(border | ((1u << bits) - 1));
    // (both are moved outwards by a step of their own rounding; no error at all: above T surely, and equal scores by their numbers)
    sure = order_of(high + 2.f * off) + 1;
    out = order_of(low - 2.f * off) - (off > 0.f ? 1 : 0);
  }
  auto is_sure = [&](unsigned k) __attribute__((always_inline)) { return !all_again && k >= sure; };
  auto between = [&](unsigned k) __attribute__((always_inline)) { return k != 0u && (all_again || (k < sure && k >= out)); };
  int n_sure = 0, n_between = 0;
  each([&](int, unsigned k) __attribute__((always_inline)) {
    n_sure += is_sure(k) ? 1 : 0;
    n_between += between(k) ? 1 : 0;
  });
  n_sure = join_lanes<1, 32>(n_sure, [](int x, int y) { return x + y; });
  n_between = join_lanes<1, 32>(n_between, [](int x, int y) { return x + y; });
  n_sure = over_waves<kWaves>(n_sure, room.i, turn_i, [](int x, int y) { return x + y; });
  n_between = over_waves<kWaves>(n_between, room.i, turn_i, [](int x, int y) { return x + y; });
  const int rest = want - n_sure;                  // to take of those between, 0 .. n_between
  const bool ask = (off > 0.f || all_again) && rest > 0 && rest < n_between;

  // exact score of a block, for all lanes: a lane has D / 8 elements of one of eight heads
  auto exact_score = [&](int i) __attribute__((always_inline)) {
    constexpr int kPart = D / 8, kLoads = kPart / kElems;
    const T *bounds = static_cast<const T *>(a.bounds) + (unit * a.n_blocks + a.n_first + i) * (2 * D) + lane % 8 * kPart;
    u32x4_t lo[kLoads], hi[kLoads];
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      lo[j] = *reinterpret_cast<const u32x4_t *>(bounds + j * kElems);
      hi[j] = *reinterpret_cast<const u32x4_t *>(bounds + D + j * kElems);
    }
    double best = -INFINITY;
    for (int g0 = 0; g0 < a.group; g0 += 8) {
      const T *mine = q + min(g0 + lane / 8, a.group - 1) * D + lane % 8 * kPart;
      double s = 0.0;
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        const u32x4_t w = load_chunk(mine + j * kElems, a.wide);
#pragma unroll
        for (int e = 0; e < kElems; ++e) {
          auto of = [&](u32x4_t v) __attribute__((always_inline)) -> double {
            if constexpr (kF32) return __uint_as_float(v[e]);
            else return e % 2 ? bf16_high(v[e / 2]) : bf16_low(v[e / 2]);
          };
          const double x = of(w), y = x > 0.0 ? x * of(hi[j]) : x * of(lo[j]);   // (a NaN is a NaN)
          s += x == 0.0 ? 0.0 : y;
        }
      }
      s = join_lanes<1, 4>(s, [](double x, double y) { return x + y; });
      s = s != s ? INFINITY : s;
      best = s > best ? s : best;
    }
    return join_lanes<8, 32>(best, [](double x, double y) { return x > y ? x : y; });
  };

  if (kRegs == 0 || (ask && n_between > kAgain)) {
    // many: numbers of 64 bits in memory, those surely taken the largest, and the list by one wave
    unsigned long long *all = a.exact + static_cast<size_t>(row) * a.scored;
    for (int x = 0; x < looks; ++x) {
      const int i0 = (x * kWaves + wave) * 64, i = i0 + lane;
      unsigned k = i < n ? order_of(score(min(i, n - 1))) : 0u;
      const unsigned long long mid = __ballot(between(k));
      unsigned long long mine = is_sure(k) ? ~0ull : between(k) ? 1ull : 0ull;
      if (ask)
        for (unsigned long long m = mid; m; m &= m - 1) {
          const int b = __builtin_ctzll(m);
          const unsigned long long e = order_of(exact_score(i0 + b));
          mine = lane == b ? e : mine;
        }
      if (i < n) all[i] = mine;
    }
    together<kWaves>();
    unsigned long long border = 0;
    for (int bit = 63; bit >= 0; --bit) {
      const unsigned long long cand = border | 1ull << bit;
      int have = 0;
      for (int i0 = wave * 64; i0 < n; i0 += kBlock) have += __popcll(__ballot(i0 + lane < n && all[min(i0 + lane, n - 1)] >= cand));
      have = over_waves<kWaves>(have, room.i, turn_i, [](int x, int y) { return x + y; });
      if (have >= want) border = cand;
      if (have == want) break;
    }
    int above = 0;
    for (int i0 = wave * 64; i0 < n; i0 += kBlock) above += __popcll(__ballot(i0 + lane < n && all[min(i0 + lane, n - 1)] > border));
    above = over_waves<kWaves>(above, room.i, turn_i, [](int x, int y) { return x + y; });
    if (wave != 0) return;
    int at = a.n_first, met = 0;
    for (int i0 = 0; i0 < n; i0 += 64) {
      const unsigned long long k = i0 + lane < n ? all[i0 + lane] : 0ull, below = (1ull << lane) - 1;
      const unsigned long long same = __ballot(i0 + lane < n && k == border);
      const bool take = i0 + lane < n && (k > border || (k == border && met + __popcll(same & below) < want - above));
      const unsigned long long m = __ballot(take);
      if (take) to[at + __popcll(m & below)] = a.n_first + i0 + lane;
      at += __popcll(m);
      met += __popcll(same);
    }
    return;
  }
  if constexpr (kRegs > 0) {
    // numbers before a look of candidates with something: counts of all looks in LDS, added up by every wave
    const unsigned long long below = (1ull << lane) - 1;
    auto before_look = [&](const int (&mine)[kHeld], int (&before)[kHeld]) __attribute__((always_inline)) {
      if constexpr (kWaves == 1) {
        int sum = 0;
#pragma unroll
        for (int x = 0; x < kRegs; ++x) {
          before[x] = sum;
          sum += mine[x];
        }
      } else {
        constexpr int kPer = (kLooks + 63) / 64;
        together<kWaves>();
        if (lane == 0)
#pragma unroll
          for (int x = 0; x < kRegs; ++x) room.look_count[x * kWaves + wave] = mine[x];
        together<kWaves>();
        int part[kPer], sum = 0;
#pragma unroll
        for (int y = 0; y < kPer; ++y) {
          part[y] = sum;
          sum += lane * kPer + y < kLooks ? room.look_count[lane * kPer + y] : 0;
        }
        int run = sum;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
          const int y = __shfl_up(run, o);
          run += lane >= o ? y : 0;
        }
        run -= sum;
#pragma unroll
        for (int x = 0; x < kRegs; ++x) {
          const int look = x * kWaves + wave;
          int got = 0;
#pragma unroll
          for (int y = 0; y < kPer; ++y) {
            const int z = __shfl(run + part[y], look / kPer);
            got = look % kPer == y ? z : got;
          }
          before[x] = got;
        }
      }
    };
    int mine[kHeld], before[kHeld];
    unsigned taken = 0;                            // bit x: candidate x of this lane goes
    if (rest > 0 && rest < n_between) {            // some of those between
#pragma unroll
      for (int x = 0; x < kRegs; ++x) mine[x] = __popcll(__ballot(between(held[x])));
      before_look(mine, before);
      if (!ask) {                                  // (equal, as exact as they are: the lowest)
#pragma unroll
        for (int x = 0; x < kRegs; ++x) {
          const unsigned long long m = __ballot(between(held[x]));
          if (between(held[x]) && before[x] + __popcll(m & below) < rest) taken |= 1u << x;
        }
      } else {
#pragma unroll
        for (int x = 0; x < kRegs; ++x) {
          const unsigned long long m = __ballot(between(held[x]));
          if (between(held[x])) room.again[before[x] + __popcll(m & below)] = at_look(x);
        }
        together<kWaves>();
        for (int x = wave; x < n_between; x += kWaves) {
          const double s = exact_score(room.again[x]);
          if (lane == 0) room.exact[x] = s;
        }
        together<kWaves>();
#pragma unroll
        for (int x = 0; x < kRegs; ++x) {
          const unsigned long long m = __ballot(between(held[x]));
          if (!between(held[x])) continue;
          const int me = before[x] + __popcll(m & below);
          const double s = room.exact[me];
          int ahead = 0;
          for (int y = 0; y < n_between; ++y) ahead += room.exact[y] > s || (room.exact[y] == s && y < me) ? 1 : 0;
          if (ahead < rest) taken |= 1u << x;
        }
      }
    } else if (rest > 0) {                         // all of them
#pragma unroll
      for (int x = 0; x < kRegs; ++x) taken |= between(held[x]) ? 1u << x : 0u;
    }
#pragma unroll
    for (int x = 0; x < kRegs; ++x) taken |= is_sure(held[x]) ? 1u << x : 0u;
#pragma unroll
    for (int x = 0; x < kRegs; ++x) mine[x] = __popcll(__ballot(taken >> x & 1u));
    before_look(mine, before);
#pragma unroll
    for (int x = 0; x < kRegs; ++x) {
      const unsigned long long m = __ballot(taken >> x & 1u);
      if (taken >> x & 1u) to[a.n_first + before[x] + __popcll(m & below)] = a.n_first + at_look(x);
    }
  }
}

// One block for a row.
template <typename T, int D, int kWaves, int kRegs>
__global__ __launch_bounds__(64 * kWaves) void choose_kernel(const ChooseArgs a) {
  __shared__ Room<kWaves, kRegs> room;
  const unsigned row = blockIdx.x, its = row / a.n_kv_heads, seq = its / a.tokens;
  const size_t unit = static_cast<size_t>(seq) * a.n_kv_heads + (row - its * a.n_kv_heads);
  choose_row<T, D, kWaves, kRegs>(a, row, room, a.score + static_cast<size_t>(row) * a.scored, a.peak + unit * a.scored);
}

size_t align_up(size_t x) { return (x + 255) / 256 * 256; }

// Tokens of a launch: the scores of all of them stay in the on-chip cache (256 MB).
constexpr size_t kScoreBytes = 96u << 20;
int tokens_of(const ChooseArgs &a) {
  const size_t per_token = static_cast<size_t>(a.n_seqs) * a.n_kv_heads * a.scored * 12;
  const size_t most = (1u << 23) / (static_cast<size_t>(a.n_seqs) * a.n_kv_heads);   // (a launch has 2^32 threads at most)
  size_t n = per_token > 0 ? kScoreBytes / per_token : a.n_tokens;
  n = n < most ? n : most;
  return static_cast<int>(n < 1 ? 1 : n < static_cast<size_t>(a.n_tokens) ? n : a.n_tokens);
}

template <typename T, int D, int kPad>
hipError_t launch_scores(const ChooseArgs &a, hipStream_t stream) {
  constexpr int kCols = 2;                         // (one or four: 43 and 47 instead of 40 us for a token each of 128 units over 3126 blocks)
  const int tiles = (a.tokens + 16 / kPad - 1) / (16 / kPad);
  const long long blocks = static_cast<long long>(a.n_seqs) * a.n_kv_heads * ((a.scored + 64 * kCols - 1) / (64 * kCols));
  if (blocks > (1 << 22)) return hipErrorInvalidValue;
  int shares = 1;                                  // of the tokens: two blocks for a compute unit (one, four, eight: 26, 21, 33 instead of 17 us for 640 tokens)
  while (shares < tiles && shares * blocks < 512) shares *= 2;
  if (shares > tiles) shares = tiles;
  hipLaunchKernelGGL((score_kernel<T, D, kPad, kCols>), dim3(static_cast<unsigned>(blocks), static_cast<unsigned>(shares)), dim3(256), 0, stream, a);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch(ChooseArgs a, hipStream_t stream) {
  int pad = 1;
  while (pad < a.group && pad < 16) pad *= 2;
  a.wide = reinterpret_cast<uintptr_t>(a.q) % 16 == 0;
  const int each = tokens_of(a);
  const size_t rows = static_cast<size_t>(a.n_seqs) * each * a.n_kv_heads;
  if (a.scored > 0) {
    char *w = static_cast<char *>(a.workspace);
    a.peak = reinterpret_cast<float *>(w);
    w += align_up(static_cast<size_t>(a.n_seqs) * a.n_kv_heads * a.scored * 4);
    a.score = reinterpret_cast<float *>(w);
    w += align_up(rows * a.scored * 4);
    a.exact = reinterpret_cast<unsigned long long *>(w);
  }
  for (a.token0 = 0; a.token0 < a.n_tokens; a.token0 += each) {
    a.tokens = a.n_tokens - a.token0 < each ? a.n_tokens - a.token0 : each;
    if (a.scored > 0) {
      const hipError_t e = pad == 1 ? launch_scores<T, D, 1>(a, stream) : pad == 2 ? launch_scores<T, D, 2>(a, stream) : pad == 4 ? launch_scores<T, D, 4>(a, stream)
                           : pad == 8 ? launch_scores<T, D, 8>(a, stream) : launch_scores<T, D, 16>(a, stream);
      if (e != hipSuccess) return e;
    }
    const long long blocks = static_cast<long long>(a.n_seqs) * a.tokens * a.n_kv_heads;
    if (blocks > (1ll << 23)) return hipErrorInvalidValue;
    const dim3 grid(static_cast<unsigned>(blocks));
    // (registers that hold no candidate cost as much as others: 8 a thread rather than 16, us for 16 sequences' rows of 8 heads, and for 200 tokens': 500 blocks 16.2, 17.2 ->
    // 12.4, 14.0; 1000 15.4, 19.1 -> 11.8, 17.0; 2000 17.0, 34 -> 13.9, 24.6.  Beyond, many rows have less of eight waves that wait for one another
    // than of four: 4000 18.0, 36 -> 16.3, 43; 8000 by eight of 16 rather than sixteen of 16 30.6, 119 -> 20.0, 85, by sixteen of 8 21.5, 132.
    // More than 16384: read anew for every look.  Scores and choice for a token of 28 / 4 heads over 16000 and 17000 blocks 39 and 279, for 4 x 16 tokens 83 and 425)
    if (a.scored <= 4 * 64) hipLaunchKernelGGL((choose_kernel<T, D, 1, 4>), grid, dim3(64), 0, stream, a);
    else if (a.scored <= 8 * 64) hipLaunchKernelGGL((choose_kernel<T, D, 1, 8>), grid, dim3(64), 0, stream, a);
    else if (a.scored <= 8 * 128) hipLaunchKernelGGL((choose_kernel<T, D, 2, 8>), grid, dim3(128), 0, stream, a);
    else if (a.scored <= 8 * 256) hipLaunchKernelGGL((choose_kernel<T, D, 4, 8>), grid, dim3(256), 0, stream, a);
    else if (a.scored <= 8 * 512 && blocks <= 512) hipLaunchKernelGGL((choose_kernel<T, D, 8, 8>), grid, dim3(512), 0, stream, a);
    else if (a.scored <= 16 * 256) hipLaunchKernelGGL((choose_kernel<T, D, 4, 16>), grid, dim3(256), 0, stream, a);
    else if (a.scored <= 16 * 512) hipLaunchKernelGGL((choose_kernel<T, D, 8, 16>), grid, dim3(512), 0, stream, a);
    else if (a.scored <= 16 * 1024) hipLaunchKernelGGL((choose_kernel<T, D, 16, 16>), grid, dim3(1024), 0, stream, a);
    else hipLaunchKernelGGL((choose_kernel<T, D, 16, 0>), grid, dim3(1024), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_bound(const BoundArgs &a, hipStream_t stream) {
  const long long blocks = (static_cast<long long>(a.units) * a.touched + 3) / 4;
  if (blocks < 1 || blocks > (1ll << 23)) return hipErrorInvalidValue;
  const dim3 grid(static_cast<unsigned>(blocks));
  if (a.dtype == LAZYEV_DTYPE_FP32 && a.head_dim == 64) hipLaunchKernelGGL((bound_kernel<float, 64>), grid, dim3(256), 0, stream, a);
  else if (a.dtype == LAZYEV_DTYPE_FP32) hipLaunchKernelGGL((bound_kernel<float, 128>), grid, dim3(256), 0, stream, a);
  else if (a.head_dim == 64) hipLaunchKernelGGL((bound_kernel<bf16_t, 64>), grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((bound_kernel<bf16_t, 128>), grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

size_t choose_workspace(const ChooseArgs &a) {
  if (a.scored <= 0) return 0;
  const size_t rows = static_cast<size_t>(a.n_seqs) * tokens_of(a) * a.n_kv_heads;
  return align_up(static_cast<size_t>(a.n_seqs) * a.n_kv_heads * a.scored * 4) + align_up(rows * a.scored * 4) + align_up(rows * a.scored * 8);
}

hipError_t launch_choose(const ChooseArgs &a, hipStream_t stream) {
  if (a.dtype == LAZYEV_DTYPE_FP32) return a.head_dim == 64 ? launch<float, 64>(a, stream) : launch<float, 128>(a, stream);
  return a.head_dim == 64 ? launch<bf16_t, 64>(a, stream) : launch<bf16_t, 128>(a, stream);
}

}  // namespace lazyev
