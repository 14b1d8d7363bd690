// Eviction by the weights that entries received (lazyev_pages_evict): which entries of a unit (table row and KV head) stay, and their rows
// moved together.
//
// select  one block per unit.  Every entry has a key of 32 bits: the order of its weight (a NaN above all), below it what is no
//         entry, above it the newest and the first entries.  The key of the last entry that stays is found bit by bit from
//         the top, from counts of the keys that reach a candidate; of those equal to it the lowest stay.  Entries that stay below
//         `keep` keep their places; the places of the others there are free, and the n-th of them is the source's of the n-th
//         entry that stays from `keep` on.  All of these numbers are prefix sums over the entries in their order.
// move    copies rows, weights and positions.  A row is read from `keep` on and written below it, so no two moves touch one another
//         and their order does not matter; moves in the entries' order (which would keep it) are as many as entries behind the first
//         one that goes: about `keep` of them where a window of 64 goes from 2112, instead of at most 64.
#include "kernels.h"
#include "lazyev.h"

#include <climits>

namespace lazyev {
namespace {

typedef __attribute__((ext_vector_type(4))) unsigned u32x4_t;

constexpr int kSelectBlock = 1024, kSelectWaves = kSelectBlock / 64;

// The order of weights, above 0 (no entry) and below ~0 (stays whatever it weighs).
__device__ __forceinline__ unsigned weight_key(float w) {
  const unsigned u = __float_as_uint(w + 0.f);     // (-0 and 0 are one)
  return w != w ? 0xFFFFFFFEu : u ^ (static_cast<unsigned>(static_cast<int>(u) >> 31) | 0x80000000u);
}

// kRegs: keys that a thread keeps (entry x * kSelectBlock + thread), 0: the keys are made anew from memory for every look.
template <int kRegs>
__global__ __launch_bounds__(kSelectBlock) void select_kernel(const WeightEvictArgs a) {
  __shared__ int counts[2][kSelectWaves];
  __shared__ int wave_i[kSelectWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int unit = static_cast<int>(blockIdx.x), seq = unit / a.n_kv_heads;
  const int len = a.lengths ? min(max(a.lengths[seq], 0), a.length) : a.length;
  int32_t *sources = a.sources + static_cast<size_t>(unit) * a.keep;
  if (len <= a.keep) {
    for (int i = threadIdx.x; i < a.keep; i += kSelectBlock) sources[i] = i < len ? i : -1;
    return;
  }
  const float *weights = a.weights + static_cast<long long>(unit) * a.stride;
  const int32_t *positions = a.positions ? a.positions + static_cast<long long>(unit) * a.stride : nullptr;

  // positions from here on are the newest
  int newest = len - 1;
  if (positions) {
    newest = INT_MIN;
    for (int i = threadIdx.x; i < len; i += kSelectBlock) newest = max(newest, positions[i]);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) newest = max(newest, __shfl_xor(newest, o));
    if (lane == 0) wave_i[wave] = newest;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kSelectWaves; ++w) newest = max(newest, wave_i[w]);
  }
  const long long recent_from = static_cast<long long>(newest) - a.n_recent + 1;
  auto make_key = [&](int i) __attribute__((always_inline)) {
    if (i >= len) return 0u;
    const int p = positions ? positions[i] : i;
    return p >= recent_from || p < a.n_first ? 0xFFFFFFFFu : weight_key(weights[i]);
  };
  constexpr int kHeld = kRegs > 0 ? kRegs : 1;
  unsigned held[kHeld];
  const int looks = kRegs > 0 ? kRegs : (len + kSelectBlock - 1) / kSelectBlock;
  if constexpr (kRegs > 0) {
#pragma unroll
    for (int x = 0; x < kRegs; ++x) held[x] = make_key(x * kSelectBlock + static_cast<int>(threadIdx.x));
  }
  auto each = [&](auto f) __attribute__((always_inline)) {
    if constexpr (kRegs > 0) {
#pragma unroll
      for (int x = 0; x < kRegs; ++x) f(x, held[x]);
    } else {
      for (int x = 0; x < looks; ++x) f(x, make_key(x * kSelectBlock + static_cast<int>(threadIdx.x)));
    }
  };

  // the largest key that at least `keep` keys reach
  unsigned border = 0;
  int reach = len;                                 // keys that reach it
  for (int bit = 31; bit >= 0 && reach != a.keep; --bit) {
    const unsigned cand = border | 1u << bit;
    int have = 0;
    each([&](int, unsigned k) __attribute__((always_inline)) { have += __popcll(__ballot(k >= cand)); });
    if (lane == 0) counts[bit & 1][wave] = have;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int w = 0; w < kSelectWaves; ++w) all += counts[bit & 1][w];
    if (all >= a.keep) {
      border = cand;
      reach = all;
    }
  }
  __syncthreads();
  // of the keys equal to it this many stay, the lowest
  int above = 0;
  each([&](int, unsigned k) __attribute__((always_inline)) { above += __popcll(__ballot(k > border)); });
  if (lane == 0) counts[0][wave] = above;
  __syncthreads();
  above = 0;
#pragma unroll
  for (int w = 0; w < kSelectWaves; ++w) above += counts[0][w];
  const int equal = a.keep - above;

  // in the entries' order: those equal, free places, entries that stay from `keep` on.  Two sweeps, as the free places are to
  // be met before the entries that fill them: the first writes the numbers of the free places where the second looks them up
  auto sweep = [&](auto f) __attribute__((always_inline)) {
    int met = 0, nth = 0;                          // of all entries before this look
    for (int x = 0; x < looks; ++x) {
      const int i = x * kSelectBlock + static_cast<int>(threadIdx.x);
      unsigned k;
      if constexpr (kRegs > 0) {
        k = 0;
#pragma unroll
        for (int y = 0; y < kRegs; ++y) k = y == x ? held[y] : k;
      } else {
        k = make_key(i);
      }
      const unsigned long long below = (1ull << lane) - 1, eq = __ballot(k == border && i < len);
      __syncthreads();
      if (lane == 0) counts[0][wave] = __popcll(eq);
      __syncthreads();
      int before = met;
#pragma unroll
      for (int w = 0; w < kSelectWaves; ++w) {
        before += w < wave ? counts[0][w] : 0;
        met += counts[0][w];
      }
      const bool stays = i < len && (k > border || (k == border && before + __popcll(eq & below) < equal));
      const bool mine = f(i, stays);
      const unsigned long long m = __ballot(mine);
      if (lane == 0) counts[1][wave] = __popcll(m);
      __syncthreads();
      int at = nth;
#pragma unroll
      for (int w = 0; w < kSelectWaves; ++w) {
        at += w < wave ? counts[1][w] : 0;
        nth += counts[1][w];
      }
      at += __popcll(m & below);
      f.put(i, stays, mine, at);
    }
  };
  struct Free {
    int32_t *sources, *list;
    int keep;
    __device__ bool operator()(int i, bool stays) const { return i < keep && !stays; }
    __device__ void put(int i, bool, bool mine, int at) const {
      if (mine) list[at] = i;
      else if (i < keep) sources[i] = i;
    }
  };
  struct Late {
    int32_t *sources, *list;
    int keep;
    __device__ bool operator()(int i, bool stays) const { return i >= keep && stays; }
    __device__ void put(int i, bool, bool mine, int at) const {
      if (mine) sources[list[at]] = i;
    }
  };
  int32_t *list = a.free_places + static_cast<size_t>(unit) * a.keep;
  sweep(Free{sources, list, a.keep});
  __syncthreads();
  __threadfence_block();
  sweep(Late{sources, list, a.keep});
}

constexpr int kMovePlaces = 64, kMoveBlock = 256;

// Places blockIdx.x * 64 .. of a unit; kChunks: 16-byte chunks of a row.
template <int kChunks>
__global__ __launch_bounds__(kMoveBlock) void move_kernel(const WeightEvictArgs a) {
  __shared__ unsigned from_row[kMovePlaces], to_row[kMovePlaces];
  const int per_unit = (a.keep + kMovePlaces - 1) / kMovePlaces;
  const int unit = static_cast<int>(blockIdx.x / per_unit), place0 = (static_cast<int>(blockIdx.x) - unit * per_unit) * kMovePlaces;
  const int seq = unit / a.n_kv_heads, kvh = unit - seq * a.n_kv_heads;
  const int32_t *table = a.pages.table + static_cast<long long>(seq) * a.pages.stride;
  const unsigned head_rows = static_cast<unsigned>(a.pages.page_size), page_rows = head_rows * static_cast<unsigned>(a.n_kv_heads);
  __shared__ int n_moves;
  if (threadIdx.x < 64) {
    const int lane = threadIdx.x, place = place0 + lane;
    int source = -1;
    bool moves = false;
    unsigned from = 0, to = 0;
    if (place < a.keep) {
      source = a.sources[static_cast<size_t>(unit) * a.keep + place];
      const long long in = static_cast<long long>(unit) * a.stride, out = static_cast<long long>(unit) * a.to_stride + place;
      const float w = source >= 0 ? a.weights[in + source] : 0.f;
      const int p = source < 0 ? -1 : a.positions ? a.positions[in + source] : source;
      if (a.weights_to) a.weights_to[out] = w;
      if (a.positions_to) a.positions_to[out] = p;
      if (source > place) {
        const int pf = page_of(a.pages, source), pt = page_of(a.pages, place);
        const unsigned nf = static_cast<unsigned>(table[pf]), nt = static_cast<unsigned>(table[pt]);
        moves = nf < static_cast<unsigned>(a.pages.n_pages) && nt < static_cast<unsigned>(a.pages.n_pages);
        from = nf * page_rows + kvh * head_rows + static_cast<unsigned>(source - pf * a.pages.page_size);
        to = nt * page_rows + kvh * head_rows + static_cast<unsigned>(place - pt * a.pages.page_size);
      }
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
  constexpr int kRows = kMoveBlock / kChunks;      // rows of the block's turn, of K and of V
  const int n = n_moves, chunk = threadIdx.x % kChunks;
  constexpr int kTurns = kMovePlaces / kRows < 4 ? kMovePlaces / kRows : 4;
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
      if (m0 + u * kRows >= n) continue;
      const size_t at = static_cast<size_t>(to_row[m0 + u * kRows]) * (kChunks * 16) + chunk * 16;
      *reinterpret_cast<u32x4_t *>(static_cast<char *>(a.k_pages) + at) = k[u];
      *reinterpret_cast<u32x4_t *>(static_cast<char *>(a.v_pages) + at) = v[u];
    }
  }
}

}  // namespace

size_t weight_evict_workspace(const WeightEvictArgs &a) {
  return (static_cast<size_t>(a.n_seqs) * a.n_kv_heads * a.keep * 4 + 255) / 256 * 256;
}

hipError_t launch_weight_evict(WeightEvictArgs a, hipStream_t stream) {
  const long long units = static_cast<long long>(a.n_seqs) * a.n_kv_heads, blocks = units * ((a.keep + kMovePlaces - 1) / kMovePlaces);
  if (units > (1 << 22) || blocks > (1ll << 24) - 1) return hipErrorInvalidValue;
  const dim3 grid(static_cast<unsigned>(units)), block(kSelectBlock);
  const int regs = (a.length + kSelectBlock - 1) / kSelectBlock;
  if (regs <= 4) hipLaunchKernelGGL((select_kernel<4>), grid, block, 0, stream, a);
  else if (regs <= 32) hipLaunchKernelGGL((select_kernel<32>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((select_kernel<0>), grid, block, 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int chunks = a.head_dim * (a.dtype == LAZYEV_DTYPE_FP32 ? 4 : 2) / 16;
  const dim3 moves(static_cast<unsigned>(blocks));
  if (chunks == 8) hipLaunchKernelGGL((move_kernel<8>), moves, dim3(kMoveBlock), 0, stream, a);
  else if (chunks == 16) hipLaunchKernelGGL((move_kernel<16>), moves, dim3(kMoveBlock), 0, stream, a);
  else hipLaunchKernelGGL((move_kernel<32>), moves, dim3(kMoveBlock), 0, stream, a);
  return hipGetLastError();
}

}  // namespace lazyev
