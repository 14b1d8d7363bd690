// Eviction by the weights that entries received (lazyev_pages_evict): which entries of a unit (table row and KV head) stay, and their rows
// moved together.
//
// select  one block per unit, whose waves have the entries in 16 stretches.  Every entry has a key of 32 bits: the order of its weight (a NaN above
//         all), below it what is no entry, above it the newest and the first entries.  The key of the last entry that stays is
//         found by counts of 1024 equal parts of the keys' range, then of the part that it is in, and so on; of those equal to it the lowest
//         stay.  Entries that stay below `keep` keep their places; the places of the others there are free, and the n-th of them is the
//         source's of the n-th entry that stays from `keep` on: sums over words of 32 entries, or (too many entries for registers) along each wave's stretch.
// move    copies rows, weights and positions.  A row is read from `keep` on and written below it, so no two moves touch one another
//         and their order does not matter; moves in the entries' order (which would keep it) are as many as entries behind the first
//         one that goes: about `keep` of them where a window of 64 goes from 2112, instead of at most 64.
//
// Measured: 64 of 2112 entries of each of 128 units gone, 13.5 us in one launch (a chain of latencies: numbers 3, border 4, places 3, rows 3); 32 units of up to
// 32768 entries brought down to 4096 each 26 + 20, the first with 32 blocks on 256 compute units, of which each takes 1.8 us for a look at its 32768 keys, the
// second at 5.9 TB/s.
#include "kernels.h"
#include "lanes.h"
#include "lazyev.h"

#include <climits>

namespace lazyev {
namespace {

typedef __attribute__((ext_vector_type(4))) unsigned u32x4_t;

constexpr int kSelectBlock = 1024, kSelectWaves = kSelectBlock / 64, kBins = 1024;
constexpr int kOwnMoves = 256;          // moves of a unit that the selecting block makes itself

// The order of weights, above 0 (no entry) and below ~0 (stays whatever it weighs).
__device__ __forceinline__ unsigned weight_key(float w) {
  const unsigned u = __float_as_uint(w + 0.f);     // (-0 and 0 are one)
  return w != w ? 0xFFFFFFFEu : u ^ (static_cast<unsigned>(static_cast<int>(u) >> 31) | 0x80000000u);
}

// The row of an entry in the pools; false: it is in no page.
__device__ __forceinline__ bool pool_row(const WeightEvictArgs &a, const int32_t *table, int kvh, int entry, unsigned &row) {
  const int pg = page_of(a.pages, entry);
  const unsigned no = static_cast<unsigned>(table[pg]), head_rows = static_cast<unsigned>(a.pages.page_size);
  row = (no * static_cast<unsigned>(a.n_kv_heads) + kvh) * head_rows + static_cast<unsigned>(entry - pg * a.pages.page_size);
  return no < static_cast<unsigned>(a.pages.n_pages);
}

// Weight and position of a place, from its source.
__device__ __forceinline__ void put_numbers(const WeightEvictArgs &a, int unit, int place, int source) {
  const long long in = static_cast<long long>(unit) * a.stride, out = static_cast<long long>(unit) * a.to_stride + place;
  const float w = source >= 0 ? a.weights[in + source] : 0.f;
  const int p = source < 0 ? -1 : a.positions ? a.positions[in + source] : source;
  if (a.weights_to) a.weights_to[out] = w;
  if (a.positions_to) a.positions_to[out] = p;
}

// n rows from_row -> to_row (of the pools, LDS; the same number twice: none is moved), by kThreads threads in groups of kChunks, kTurns of a group's rows on their way together.
template <int kChunks, int kThreads, int kTurns>
__device__ __forceinline__ void move_rows(const WeightEvictArgs &a, const unsigned *from_row, const unsigned *to_row, int n) {
  constexpr int kRows = kThreads / kChunks;
  const int chunk = threadIdx.x % kChunks;
  for (int m0 = threadIdx.x / kChunks; m0 < n; m0 += kRows * kTurns) {
    u32x4_t k[kTurns], v[kTurns];
#pragma unroll
    for (int u = 0; u < kTurns; ++u) {
      const size_t at = static_cast<size_t>(from_row[min(m0 + u * kRows, n - 1)]) * (kChunks * 16) + chunk * 16;
      k[u] = *reinterpret_cast<const u32x4_t *>(static_cast<const char *>(a.k_pages) + at);
      v[u] = *reinterpret_cast<const u32x4_t *>(static_cast<const char *>(a.v_pages) + at);
    }
#pragma unroll
    for (int u = 0; u < kTurns; ++u) {
      if (m0 + u * kRows >= n || from_row[m0 + u * kRows] == to_row[m0 + u * kRows]) continue;
      const size_t at = static_cast<size_t>(to_row[m0 + u * kRows]) * (kChunks * 16) + chunk * 16;
      *reinterpret_cast<u32x4_t *>(static_cast<char *>(a.k_pages) + at) = k[u];
      *reinterpret_cast<u32x4_t *>(static_cast<char *>(a.v_pages) + at) = v[u];
    }
  }
}

// kRegs: keys that a lane keeps (of a stretch of 64 kRegs entries), 0: they are made anew from memory for every look.  kChunks: the block moves the rows
// too, of that many 16-byte chunks (at most kOwnMoves of them); 0: the next kernel does.
template <int kRegs, int kChunks>
__global__ __launch_bounds__(kSelectBlock) void select_kernel(const WeightEvictArgs a) {
  __shared__ int bins[kBins], waves_i[2][kSelectWaves];
  __shared__ unsigned waves_u[2][kSelectWaves];
  __shared__ int picked[3];                        // part of the range, keys of it, keys beyond it
  constexpr int kOwn = kChunks > 0 ? kOwnMoves : 1;
  __shared__ unsigned from_row[kOwn], to_row[kOwn];
  __shared__ int free_place[kOwn], late_entry[kOwn];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int unit = static_cast<int>(blockIdx.x), seq = unit / a.n_kv_heads, kvh = unit - seq * a.n_kv_heads;
  const int len = a.lengths ? min(max(a.lengths[seq], 0), a.length) : a.length;
  int32_t *sources = a.sources + static_cast<size_t>(unit) * a.keep;
  if (len <= a.keep) {
    for (int i = threadIdx.x; i < a.keep; i += kSelectBlock) {
      sources[i] = i < len ? i : -1;
      if constexpr (kChunks > 0) put_numbers(a, unit, i, i < len ? i : -1);
    }
    return;
  }
  const float *weights = a.weights + static_cast<long long>(unit) * a.stride;
  const int32_t *positions = a.positions ? a.positions + static_cast<long long>(unit) * a.stride : nullptr;
  const int looks = kRegs > 0 ? kRegs : (len + kSelectBlock - 1) / kSelectBlock;
  auto entry_of = [&](int x) __attribute__((always_inline)) { return (wave * looks + x) * 64 + lane; };

  // numbers over all waves; the two rooms take turns, so that one barrier does
  int turn = 0;
  auto before_wave = [&](int mine, int &all) __attribute__((always_inline)) {
    if (lane == 0) waves_i[turn][wave] = mine;
    __syncthreads();
    int before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < kSelectWaves; ++w) {
      const int n = waves_i[turn][w];
      before += w < wave ? n : 0;
      all += n;
    }
    turn ^= 1;
    return before;
  };

  // positions from `recent_from` on are the newest
  constexpr int kHeld = kRegs > 0 ? kRegs : 1;
  unsigned held[kHeld];
  constexpr bool kAnew = kRegs == 0 || kRegs > 32;  // positions are read twice, rather than kept
  int place[kAnew ? 1 : kHeld];
  int newest = len - 1;
  if (positions) {
    newest = INT_MIN;
    if constexpr (!kAnew) {
#pragma unroll
      for (int x = 0; x < kRegs; ++x) place[x] = entry_of(x) < len ? positions[entry_of(x)] : INT_MIN;
#pragma unroll
      for (int x = 0; x < kRegs; ++x) newest = max(newest, place[x]);
    } else {
      for (int x = 0; x < looks; ++x) newest = max(newest, entry_of(x) < len ? positions[entry_of(x)] : INT_MIN);
    }
    newest = join_lanes<1, 32>(newest, [](int x, int y) { return max(x, y); });
    if (lane == 0) waves_i[turn][wave] = newest;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kSelectWaves; ++w) newest = max(newest, waves_i[turn][w]);
    turn ^= 1;
  }
  const long long recent_from = static_cast<long long>(newest) - a.n_recent + 1;
  auto key_of = [&](int i, int p, float w) __attribute__((always_inline)) {
    return i >= len ? 0u : p >= recent_from || p < a.n_first ? 0xFFFFFFFFu : weight_key(w);
  };
  if constexpr (kRegs > 0) {
    if constexpr (kAnew) {                         // (a few at a time: there are no registers for all of them)
#pragma unroll
      for (int x0 = 0; x0 < kRegs; x0 += 8) {
        float w[8];
        int p[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          const int i = min(entry_of(x0 + x), len - 1);
          w[x] = weights[i];
          p[x] = positions ? positions[i] : entry_of(x0 + x);
        }
#pragma unroll
        for (int x = 0; x < 8; ++x) held[x0 + x] = key_of(entry_of(x0 + x), p[x], w[x]);
        __asm__ volatile("" ::: "memory");
      }
    } else {
      float w[kHeld];
#pragma unroll
      for (int x = 0; x < kRegs; ++x) w[x] = entry_of(x) < len ? weights[entry_of(x)] : 0.f;
#pragma unroll
      for (int x = 0; x < kRegs; ++x) held[x] = key_of(entry_of(x), positions ? place[x] : entry_of(x), w[x]);
    }
  }
  auto each = [&](auto f) __attribute__((always_inline)) {
    if constexpr (kRegs > 0) {
#pragma unroll
      for (int x = 0; x < kRegs; ++x) f(entry_of(x), held[x]);
    } else {
      for (int x = 0; x < looks; ++x) {
        const int i = entry_of(x), j = min(i, len - 1);
        f(i, key_of(i, positions ? positions[j] : j, weights[j]));
      }
    }
  };

  // the `keep`-th largest key: it is among those from low to high, of which `want` are to stay.  (The range is that of the keys in it: equal
  // keys are found to be so at once)
  unsigned low = 0u, high = 0xFFFFFFFFu;
  auto tighten = [&]() __attribute__((always_inline)) {
    unsigned least = 0xFFFFFFFFu, most = 0u;
    each([&](int i, unsigned k) __attribute__((always_inline)) {
      const bool in = i < len && k >= low && k <= high;
      least = min(least, in ? k : 0xFFFFFFFFu);
      most = max(most, in ? k : 0u);
    });
    least = join_lanes<1, 32>(least, [](unsigned x, unsigned y) { return min(x, y); });
    most = join_lanes<1, 32>(most, [](unsigned x, unsigned y) { return max(x, y); });
    if (lane == 0) {
      waves_u[0][wave] = least;
      waves_u[1][wave] = most;
    }
    __syncthreads();
    low = 0xFFFFFFFFu;
    high = 0u;
#pragma unroll
    for (int w = 0; w < kSelectWaves; ++w) {
      low = min(low, waves_u[0][w]);
      high = max(high, waves_u[1][w]);
    }
  };
  // Many weights may be alike: one such key, the most frequent of 64, is counted in registers, as additions to one place go one after the other.
  if (wave == 0) {
    unsigned k = 0;
    if constexpr (kRegs > 0) k = held[kRegs / 2];
    else k = key_of(lane, positions ? positions[lane] : lane, weights[lane]);
    int times = 0;
#pragma unroll 8
    for (int y = 0; y < 64; ++y) times += static_cast<unsigned>(__builtin_amdgcn_readlane(static_cast<int>(k), y)) == k ? 1 : 0;
    int best = times << 6 | lane;
    best = join_lanes<1, 32>(best, [](int x, int y) { return max(x, y); });
    const unsigned mode = static_cast<unsigned>(__shfl(static_cast<int>(k), best & 63));
    if (lane == 0) picked[0] = best >> 6 > 4 ? static_cast<int>(mode) : 0;
  }
  __syncthreads();
  const unsigned common = static_cast<unsigned>(picked[0]);
  __syncthreads();
  int want = a.keep, have = len;                   // of the keys in the range
  int had = 0;
  for (int pass = 0; pass < 8; ++pass) {           // (four do: 10 bits each)
    if (have > had / 4) tighten();                 // (the first time, and where a part has much of the range: many equal ones)
    had = have;
    if (low == high || want == have) break;        // (uniform)
    const int bits = 32 - __clz(static_cast<int>(high - low)), shift = bits > 10 ? bits - 10 : 0;
    bins[threadIdx.x] = 0;
    __syncthreads();
    int alike = 0;
    each([&](int, unsigned k) __attribute__((always_inline)) {
      if (k - low > high - low) return;            // (no entry: below all keys)
      if (k == common) ++alike;
      else atomicAdd(&bins[(k - low) >> shift], 1);
    });
    if (common - low <= high - low) {              // (uniform)
      alike = join_lanes<1, 32>(alike, [](int x, int y) { return x + y; });
      if (lane == 0) atomicAdd(&bins[(common - low) >> shift], alike);
    }
    __syncthreads();
    // parts from the top: thread t has part kBins - 1 - t
    const int part = kBins - 1 - static_cast<int>(threadIdx.x), mine = bins[part];
    int run = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(run, o);
      run += lane >= o ? y : 0;
    }
    int all;
    const int before = before_wave(__shfl(run, 63), all), above = before + run - mine;
    if (above < want && above + mine >= want) {
      picked[0] = part;
      picked[1] = mine;
      picked[2] = above;
    }
    __syncthreads();
    const unsigned from = low + (static_cast<unsigned>(picked[0]) << shift);
    have = picked[1];
    want -= picked[2];
    const unsigned to = from + ((1u << shift) - 1);
    high = to < from || to > high ? high : to;
    low = from;
    __syncthreads();
  }
  // keys beyond the range stay, and of those in it (all of them, or equal ones) `want`, the lowest
  const unsigned long long below = (1ull << lane) - 1;
  const int32_t *table = a.pages.table + static_cast<long long>(seq) * a.pages.stride;
  int32_t *list = kChunks > 0 ? free_place : a.free_places + static_cast<size_t>(unit) * a.keep;
  int all = 0;
  auto comes = [&](int i, int n, int place) __attribute__((always_inline)) {   // entry i to the n-th free place
    sources[place] = i;
    if constexpr (kChunks > 0) {
      put_numbers(a, unit, place, i);
      unsigned rf, rt;
      const bool both = pool_row(a, table, kvh, i, rf) & pool_row(a, table, kvh, place, rt);
      from_row[n] = both ? rf : 0u;
      to_row[n] = both ? rt : 0u;
    }
  };
  if constexpr (kRegs > 0) {
    // as bits, a word of 32 entries for a thread
    __shared__ unsigned beyond_bits[32 * kRegs], in_bits[32 * kRegs];
#pragma unroll
    for (int x = 0; x < kRegs; ++x) {
      const unsigned long long beyond = __ballot(held[x] > high), in = __ballot(held[x] - low <= high - low);
      if (lane < 2) {
        beyond_bits[(wave * kRegs + x) * 2 + lane] = static_cast<unsigned>(beyond >> (32 * lane));
        in_bits[(wave * kRegs + x) * 2 + lane] = static_cast<unsigned>(in >> (32 * lane));
      }
    }
    __syncthreads();
    constexpr int kWords = (32 * kRegs + kSelectBlock - 1) / kSelectBlock;   // of a thread, next to one another
    const int word0 = static_cast<int>(threadIdx.x) * kWords;
    auto before_words = [&](int mine, int &total) __attribute__((always_inline)) {
      int run = mine;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(run, o);
        run += lane >= o ? y : 0;
      }
      return before_wave(__builtin_amdgcn_readlane(run, 63), total) + run - mine;
    };
    unsigned kept[kWords], in[kWords], free[kWords], late[kWords];
    int n_in = 0, n_moves = 0;                     // (of no sign: __popc; room may be negative)
#pragma unroll
    for (int y = 0; y < kWords; ++y) {
      kept[y] = word0 + y < 32 * kRegs ? beyond_bits[word0 + y] : 0u;
      in[y] = word0 + y < 32 * kRegs ? in_bits[word0 + y] : 0u;
      n_in += static_cast<int>(__popc(in[y]));
    }
    int room = want - before_words(n_in, all);
#pragma unroll
    for (int y = 0; y < kWords; ++y) {
      const int n = static_cast<int>(__popc(in[y]));
      unsigned rest = room >= n ? 0u : in[y];
      if (room < n)
        for (int x = 0; x < room; ++x) rest &= rest - 1;
      kept[y] |= in[y] & ~rest;
      room -= n;
      const int left = a.keep - 32 * (word0 + y);  // entries of the word below `keep`
      const unsigned low_places = left >= 32 ? ~0u : left <= 0 ? 0u : (1u << left) - 1;
      free[y] = word0 + y < 32 * kRegs ? ~kept[y] & low_places : 0u;
      late[y] = kept[y] & ~low_places;
      // (numbers of 16 bits: as many of one as of the other, of at most 65536 entries)
      n_moves += static_cast<int>(__popc(free[y]) | __popc(late[y]) << 16);
    }
    int both = 0;
    const int before = before_words(n_moves, both);
    all = static_cast<int>(static_cast<unsigned>(both) >> 16);
    // (numbers alone: what has to be looked up for an entry is left to a thread of its own)
    int32_t *lates = kChunks > 0 ? late_entry : list + static_cast<size_t>(a.n_seqs) * a.n_kv_heads * a.keep;
    int at_free = before & 0xFFFF, at_late = static_cast<int>(static_cast<unsigned>(before) >> 16);
#pragma unroll
    for (int y = 0; y < kWords; ++y) {
      if (word0 + y < 32 * kRegs) beyond_bits[word0 + y] = kept[y];
      for (; free[y]; free[y] &= free[y] - 1) list[at_free++] = 32 * (word0 + y) + __builtin_ctz(free[y]);
      for (; late[y]; late[y] &= late[y] - 1) lates[at_late++] = 32 * (word0 + y) + __builtin_ctz(late[y]);
    }
    __threadfence_block();
    __syncthreads();
    for (int i = threadIdx.x; i < a.keep; i += kSelectBlock)
      if (beyond_bits[i / 32] >> (i % 32) & 1u) {
        sources[i] = i;
        if constexpr (kChunks > 0) put_numbers(a, unit, i, i);
      }
    for (int n = threadIdx.x; n < all; n += kSelectBlock) comes(lates[n], n, list[n]);
  } else {
    // along each wave's stretch.  (Numbers that change meanwhile, which no caller may do, find no place out of range)
    int mine = 0;
    each([&](int i, unsigned k) __attribute__((always_inline)) { mine += __popcll(__ballot(i < len && k >= low && k <= high)); });
    const int met_0 = before_wave(mine, all);
    int met = met_0;
    auto stays_of = [&](int i, unsigned k) __attribute__((always_inline)) {
      const bool in = i < len && k >= low && k <= high;
      const unsigned long long m = __ballot(in);
      const bool stays = i < len && (k > high || (in && met + __popcll(m & below) < want));
      met += __popcll(m);
      return stays;
    };
    int n_free = 0, n_late = 0;
    each([&](int i, unsigned k) __attribute__((always_inline)) {
      const bool stays = stays_of(i, k);
      n_free += __popcll(__ballot(i < a.keep && !stays));
      n_late += __popcll(__ballot(i >= a.keep && stays));
    });
    int at_free = before_wave(n_free, all), at_late = before_wave(n_late, all);
    met = met_0;
    each([&](int i, unsigned k) __attribute__((always_inline)) {
      const bool stays = stays_of(i, k), free = i < a.keep && !stays;
      const unsigned long long m = __ballot(free);
      const int n = at_free + __popcll(m & below);
      if (free && n < a.keep) list[n] = i;
      else if (i < a.keep) sources[i] = i;
      at_free += __popcll(m);
    });
    __threadfence_block();
    __syncthreads();
    met = met_0;
    each([&](int i, unsigned k) __attribute__((always_inline)) {
      const bool stays = stays_of(i, k), late = i >= a.keep && stays;
      const unsigned long long m = __ballot(late);
      const int n = at_late + __popcll(m & below);
      if (late && n < a.keep) {
        const int place = list[n];
        if (place >= 0 && place < a.keep) comes(i, n, place);
      }
      at_late += __popcll(m);
    });
  }
  if constexpr (kChunks > 0) {
    __syncthreads();
    move_rows<kChunks, kSelectBlock, 1>(a, from_row, to_row, all);
  }
}

constexpr int kMovePlaces = 64, kMoveBlock = 256;

// Places blockIdx.x * 64 .. of a unit; kChunks: 16-byte chunks of a row.
template <int kChunks>
__global__ __launch_bounds__(kMoveBlock) void move_kernel(const WeightEvictArgs a) {
  __shared__ unsigned from_row[kMovePlaces], to_row[kMovePlaces];
  __shared__ int n_moves;
  const int per_unit = (a.keep + kMovePlaces - 1) / kMovePlaces;
  const int unit = static_cast<int>(blockIdx.x / per_unit), place0 = (static_cast<int>(blockIdx.x) - unit * per_unit) * kMovePlaces;
  const int seq = unit / a.n_kv_heads, kvh = unit - seq * a.n_kv_heads;
  if (threadIdx.x < 64) {
    const int32_t *table = a.pages.table + static_cast<long long>(seq) * a.pages.stride;
    const int lane = threadIdx.x, place = place0 + lane;
    bool moves = false;
    unsigned from = 0, to = 0;
    if (place < a.keep) {
      const int source = a.sources[static_cast<size_t>(unit) * a.keep + place];
      put_numbers(a, unit, place, source);
      if (source > place) moves = pool_row(a, table, kvh, source, from) & pool_row(a, table, kvh, place, to);
    }
    const unsigned long long m = __ballot(moves);
    if (moves) {
      const int at = __popcll(m & ((1ull << lane) - 1));
      from_row[at] = from;
      to_row[at] = to;
    }
    if (lane == 0) n_moves = __popcll(m);
  }
  __syncthreads();
  constexpr int kTurns = kMovePlaces / (kMoveBlock / kChunks);
  move_rows<kChunks, kMoveBlock, kTurns < 4 ? kTurns : 4>(a, from_row, to_row, n_moves);
}

template <int kChunks>
void launch_select(const WeightEvictArgs &a, const dim3 &grid, hipStream_t stream) {
  const dim3 block(kSelectBlock);
  const int regs = (a.length + kSelectBlock - 1) / kSelectBlock;
  // (keys of up to three, rather than eight, a lane: 128 units of 2112 entries 14.7 us of the whole call, 17.1; 8 of 1500 14.9, 16.7.  8 units of 7000 entries 14.5 us by 8 keys a lane, 16000 21.4 by 16 and 29 by 32; 33205 to 60000 50 by 64 and 120 by none)
  if (regs <= 3) hipLaunchKernelGGL((select_kernel<3, kChunks>), grid, block, 0, stream, a);
  else if (regs <= 8) hipLaunchKernelGGL((select_kernel<8, kChunks>), grid, block, 0, stream, a);
  else if (regs <= 16) hipLaunchKernelGGL((select_kernel<16, kChunks>), grid, block, 0, stream, a);
  else if (regs <= 32) hipLaunchKernelGGL((select_kernel<32, kChunks>), grid, block, 0, stream, a);
  else if constexpr (kChunks == 0) {
    if (regs <= 64) hipLaunchKernelGGL((select_kernel<64, 0>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((select_kernel<0, 0>), grid, block, 0, stream, a);
  }
}

}  // namespace

size_t weight_evict_workspace(const WeightEvictArgs &a) {
  return (2 * static_cast<size_t>(a.n_seqs) * a.n_kv_heads * a.keep * 4 + 255) / 256 * 256;
}

hipError_t launch_weight_evict(WeightEvictArgs a, hipStream_t stream) {
  const long long units = static_cast<long long>(a.n_seqs) * a.n_kv_heads, blocks = units * ((a.keep + kMovePlaces - 1) / kMovePlaces);
  if (units >= (1 << 22) || blocks > (1ll << 24) - 1) return hipErrorInvalidValue;
  const dim3 grid(static_cast<unsigned>(units));
  const int chunks = a.head_dim * (a.dtype == LAZYEV_DTYPE_FP32 ? 4 : 2) / 16;
  const int moves = a.length - a.keep < a.keep ? a.length - a.keep : a.keep;   // of a unit, at most
  // (a block that keeps no keys makes them anew, from numbers that its moves may be changing)
  if (moves <= kOwnMoves && a.length <= 32 * kSelectBlock) {
    if (chunks == 8) launch_select<8>(a, grid, stream);
    else if (chunks == 16) launch_select<16>(a, grid, stream);
    else launch_select<32>(a, grid, stream);
    return hipGetLastError();
  }
  launch_select<0>(a, grid, stream);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 all(static_cast<unsigned>(blocks));
  if (chunks == 8) hipLaunchKernelGGL((move_kernel<8>), all, dim3(kMoveBlock), 0, stream, a);
  else if (chunks == 16) hipLaunchKernelGGL((move_kernel<16>), all, dim3(kMoveBlock), 0, stream, a);
  else hipLaunchKernelGGL((move_kernel<32>), all, dim3(kMoveBlock), 0, stream, a);
  return hipGetLastError();
}

}  // namespace lazyev
