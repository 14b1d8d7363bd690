// Norms of heads and their rotation by the token's position, in one pass over the rows, from any places to any
// places or into the pages of a cache (where the values go along as they are).
//
//   n = x / sqrt(mean(x^2) + eps) * w;   (n_a, n_b) -> (n_a cos - n_b sin, n_b cos + n_a sin), angle = position * inv_freq
//
// A head is L lanes of 16 bytes; the sum of squares is joined over the L lanes and the partner of an element that is
// turned with the other half's comes from its lane by a permutation, all on fp32 values that never leave the registers.
// The angle's sine and cosine are the same for all heads of a token: each is worked out once in the block, one pair per
// thread, and kept in LDS.  The angle is needed modulo a turn only: the product position * inv_freq / 2 pi in binary64 has
// 2^-52 of itself as its error, so that its fraction is good to 1e-9 at positions of millions, where an fp32 angle is off by a
// tenth of a turn.
//
// Bound by memory: 8192 tokens of 40 + 8 heads of 128 x bf16 (201 MB read and written) 40.6 us, 5.0 TB/s; 16384 tokens appended
// of 8 heads (134 MB) 25.0 us, 5.4 TB/s; a copy of 1 GiB reaches 5.2 on the same card.  32 tokens of 28 + 4 heads: 3.5 us, of
// which a kernel that does nothing takes 1.9.
#include "kernels.h"
#include "lazyev.h"

#include <type_traits>

namespace lazyev {
namespace {

constexpr int kBlock = 256;
constexpr int kWaves = kBlock / 64;
typedef unsigned short bf16_t;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4_t;
typedef __attribute__((ext_vector_type(2))) float f32x2_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;

// 16 bytes of a row and its elements as fp32.
template <typename T>
struct Chunk {
  static constexpr int kElems = 16 / static_cast<int>(sizeof(T));
  __device__ static void open(const u32x4_t &w, float (&x)[kElems]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (sizeof(T) == 4) {
        x[e] = __uint_as_float(w[e]);
      } else {
        x[2 * e] = __uint_as_float(w[e] << 16);
        x[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
      }
    }
  }
  __device__ static u32x4_t close(const float (&x)[kElems]) {
    u32x4_t w;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (sizeof(T) == 4) w[e] = __float_as_uint(x[e]);
      else w[e] = __builtin_bit_cast(unsigned, __builtin_convertvector(f32x2_t{x[2 * e], x[2 * e + 1]}, bf16x2_t));
    }
    return w;
  }
};

// kVec: every row starts at a multiple of 16 bytes.
template <typename T, bool kVec>
__device__ __forceinline__ u32x4_t load_chunk(const T *p) {
  if constexpr (kVec) return *reinterpret_cast<const u32x4_t *>(p);
  T e[16 / sizeof(T)];
#pragma unroll
  for (int i = 0; i < static_cast<int>(16 / sizeof(T)); ++i) e[i] = p[i];
  u32x4_t w;
  __builtin_memcpy(&w, e, 16);
  return w;
}
template <typename T, bool kVec, bool kPast>       // kPast: past the caches
__device__ __forceinline__ void store_chunk(T *p, const u32x4_t &w) {
  if constexpr (kVec) {
    if constexpr (kPast) __builtin_nontemporal_store(w, reinterpret_cast<u32x4_t *>(p));
    else *reinterpret_cast<u32x4_t *>(p) = w;
    return;
  }
  T e[16 / sizeof(T)];
  __builtin_memcpy(e, &w, 16);
#pragma unroll
  for (int i = 0; i < static_cast<int>(16 / sizeof(T)); ++i) p[i] = e[i];
}

// grid: x = spans of kTokens tokens (of all sequences in a row), y = shares of their heads.  A wave takes kBatch times its
// heads at once: their loads are on their way together, the first ones while the sines and cosines are worked out.  Up to
// four tokens a block: a wave's L-lane groups take heads of one token.  More: each group has a token of its own.
template <typename T, int D, int kTokens, int kBatch, bool kVec, bool kPast>
__global__ __launch_bounds__(kBlock) void rope_kernel(const RopeArgs a) {
  constexpr int E = Chunk<T>::kElems, L = D / E, kRows = 64 / L;   // elements and lanes of a chunk / a head, heads of a wave
  constexpr bool kOwnToken = kTokens > kWaves;     // a token for every group
  static_assert(!kOwnToken || kTokens == kWaves * kRows, "");
  constexpr int kWavesPerToken = kOwnToken ? 1 : kWaves / kTokens;
  __shared__ float2 turn[kTokens][D / 2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tokens = a.n_seqs * a.n_tokens;
  const int token0 = a.token0 + static_cast<int>(blockIdx.x) * kTokens;
  const int my_k = kOwnToken ? wave * kRows + lane / L : kTokens == 1 ? 0 : wave / kWavesPerToken;
  const int tk = min(token0 + my_k, tokens - 1);   // (a wave without a token works on the last one and leaves nothing)
  const int seq = a.n_seqs == 1 ? 0 : tk / a.n_tokens, token = tk - seq * a.n_tokens;
  const int li = lane % L, e0 = li * E;            // this lane's elements of a head: e0 .. e0 + E - 1
  const int n0 = a.rows[0].heads, n = n0 + a.rows[1].heads;
  const T *in[2];
  T *out[2];
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    in[s] = static_cast<const T *>(a.rows[s].in) + (seq * a.rows[s].in_seq + token * a.rows[s].in_token) + e0;
    out[s] = static_cast<T *>(a.rows[s].out) + (a.pages.table ? 0 : seq * a.rows[s].out_seq + token * a.rows[s].out_token) + e0;
  }
  constexpr int kStep = kOwnToken ? 1 : kRows * kWavesPerToken;
  const int step = kStep * static_cast<int>(gridDim.y);
  const int lane_head = kOwnToken ? 0 : lane / L;
  int h0 = kOwnToken ? static_cast<int>(blockIdx.y) : (static_cast<int>(blockIdx.y) * kWavesPerToken + wave % kWavesPerToken) * kRows + lane_head;   // this lane's head
  u32x4_t raw[kBatch];
  auto load = [&](int first) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int at = min(first + u * step, n - 1);
      const bool second = at >= n0;
      raw[u] = load_chunk<T, kVec>((second ? in[1] : in[0]) + (second ? at - n0 : at) * (second ? a.rows[1].in_head : a.rows[0].in_head));
    }
  };
  load(h0);
  float w[2][E];
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    if (a.rows[s].weight) Chunk<T>::open(load_chunk<T, kVec>(static_cast<const T *>(a.rows[s].weight) + e0), w[s]);
    else
#pragma unroll
      for (int e = 0; e < E; ++e) w[s][e] = 1.f;
  }
  if (a.half > 0) {
    for (int x = threadIdx.x; x < kTokens * a.half; x += kBlock) {
      const int k = x / a.half, j = x - k * a.half, at = min(token0 + k, tokens - 1);
      const long long p = a.start + (a.positions ? a.positions[at] : a.n_seqs == 1 ? at : at % a.n_tokens);
      constexpr double kPerTurn = 0.15915494309189533576888;
      const double turns = static_cast<double>(p) * static_cast<double>(a.inv_freq[j]) * kPerTurn;
      float s, c;
      sincospif(2.f * static_cast<float>(turns - rint(turns)), &s, &c);
      turn[k][j] = make_float2(c, s);
    }
    __syncthreads();
  }
  if (token0 + my_k >= tokens) return;
  // where the token's rows go in the pages
  if (a.pages.table) {
    const int entry = a.first_entry + token, pg = page_of(a.pages, entry);
    const int page = a.pages.table[static_cast<long long>(seq) * a.pages.stride + pg];
    if (page < 0 || page >= a.pages.n_pages) return;
    const long long row = static_cast<long long>(page) * n0 * a.pages.page_size + (entry - pg * a.pages.page_size);
    out[0] += row * D;
    out[1] += row * D;
  }
  const long long out_head[2] = {a.pages.table ? static_cast<long long>(a.pages.page_size) * D : a.rows[0].out_head,
                                 a.pages.table ? static_cast<long long>(a.pages.page_size) * D : a.rows[1].out_head};
  const bool halves = a.layout == LAZYEV_ROPE_HALVES;
  const bool turned = e0 < 2 * a.half;
  float cs[E], sn[E];                              // (pairs: of the first E / 2 places)
  {
    const int j0 = halves ? (e0 < a.half ? e0 : e0 - a.half) : e0 / 2;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float2 cv = turned ? turn[my_k][j0 + (halves ? e : e / 2)] : make_float2(1.f, 0.f);
      cs[e] = cv.x;
      sn[e] = (halves ? e0 < a.half : e % 2 == 0) ? -cv.y : cv.y;
    }
  }
  const int partner = halves && turned ? (e0 < a.half ? lane + a.half / E : lane - a.half / E) : lane;
  for (; h0 - lane_head < n; h0 += kBatch * step) {   // (the same in all lanes)
    u32x4_t done[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int at = h0 + u * step;
      const bool second = min(at, n - 1) >= n0;
      const bool normed = second ? a.rows[1].weight != nullptr : a.rows[0].weight != nullptr, turns = second ? a.rows[1].turn : a.rows[0].turn;
      float x[E], y[E];
      Chunk<T>::open(raw[u], x);
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) ss = fmaf(x[e], x[e], ss);
#pragma unroll
      for (int o = 1; o < L; o <<= 1) ss += __shfl_xor(ss, o);
      const float inv = normed ? 1.f / sqrtf(ss * (1.f / D) + a.eps) : 1.f;
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = x[e] * inv * (second ? w[1][e] : w[0][e]);
      if (halves) {
#pragma unroll
        for (int e = 0; e < E; ++e) y[e] = __shfl(x[e], partner);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) y[e] = x[e ^ 1];
      }
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = turned && turns ? fmaf(y[e], sn[e], x[e] * cs[e]) : x[e];
      done[u] = turns || normed ? Chunk<T>::close(x) : raw[u];
    }
    const int next = h0 + kBatch * step;
    if (next - lane_head < n) load(next);
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int at = h0 + u * step;
      const bool second = at >= n0;
      if (at < n) store_chunk<T, kVec, kPast>((second ? out[1] : out[0]) + (second ? at - n0 : at) * (second ? out_head[1] : out_head[0]), done[u]);
    }
  }
}

constexpr long long kPastBytes = 4ll << 20;        // (an XCD's L2)
// Blocks of a launch, which has fewer than 2^32 threads from one end to the other; calls of more tokens take several, one after the other.
constexpr long long kLaunchBlocks = 1ll << 23;

}  // namespace

RopeCut rope_cut(long long tokens, int heads, int elem, int head_dim) {
  const int row_lanes = head_dim * elem / 16, rows = 64 / row_lanes;   // of a head, heads of a wave
  // Three ways, us with one token a block (its heads dealt to four waves, and of few tokens to more blocks) / four (a wave each) / one
  // for every L lanes; query + key heads x tokens, or appended key and value heads, rows that no cache holds yet:
  //   128 x bf16  28 + 4 x 32     3.8 /  7.8 / 22.2    28 + 4 x 512   5.8 /  9.4 / 28.1    28 + 4 x 4096  20.0 / 17.7 / 34.8
  //               40 + 8 x 1024   9.1 / 14.1 / 43.0    40 + 8 x 4096 26.1 / 23.4 / 49.5    56 + 8 x 8192  58.6 / 57.5 / 69.0
  //               8 + 8 x 2048    8.7 /  7.8 / 17.3    8 + 8 x 65536  157 /  102 / 116     1 + 1 x 8192   16.4 /  9.3 /  6.8
  //               2 + 2 x 65536   116 / 55.1 / 35.5    1 + 1 x 65536  111 / 51.2 / 23.8
  //   64 x fp32   12 + 4 x 2048   6.5 /  6.9 /  -      12 + 4 x 4096 11.3 / 10.1 /  -      32 + 8 x 4096  18.1 / 19.8 / 33.9
  //   128 x fp32  8 + 2 x 2048    7.8 /  8.7 /  -      8 + 2 x 8192  21.7 / 20.2 /  -      32 + 8 x 8192  63.4 / 68.1 / 70.5
  // The first needs blocks for the whole chip, 256 compute units; the last leaves no lane without a head where these are
  // fewer than four times those of a wave, and shares a sine and cosine among fewer of them.  (Four loads of a wave at once instead of two: 46.6
  // instead of 45.6 for 40 + 8 x 8192, 32.1 instead of 30.8 for 8 + 8 x 16384.)
  // Results go past the caches: 28 + 4 x 4096 20.0 -> 17.8, 8 + 8 x 65536 106 -> 102, and an attention that reads them next takes no longer, also where they are
  // few (the two calls together, through the caches / past them: 2048 tokens of 1 + 1 heads, 1 MB, 17.0 / 16.9, 4096 17.8 / 17.5; 1600 of 4 + 4 16.5 / 16.4; 4096
  // of 1 + 1 of 64 x bf16 15.2 / 15.1; 2000 of 2 + 2 of 64 x fp32 17.0 / 17.1).  But not those of one token a block below an XCD's L2: 40 + 8 x 512, beyond
  // it, 8.3 -> 7.5, the attention over 300 rotated tokens 20.9 -> 21.4.
  const int lanes = heads * row_lanes;             // of a token
  RopeCut c;
  c.past = 1;
  c.shares = 1;
  if (heads < 4 * rows && tokens >= 1024ll * heads) {
    c.tokens = kWaves * rows;
  } else if (tokens >= 1536 && (elem == 2 ? tokens >= 4ll * lanes : tokens >= 8ll * lanes && lanes <= 384)) {
    c.tokens = 4;
  } else {
    c.tokens = 1;
    c.past = tokens * heads * (static_cast<long long>(head_dim) * elem) >= kPastBytes;
    const int shares = (heads + rows * kWaves - 1) / (rows * kWaves), want = static_cast<int>((512 + tokens - 1) / tokens);
    c.shares = shares < want ? shares : want;
  }
  c.launch = kLaunchBlocks * c.tokens;
  return c;
}

namespace {

template <typename T, int D, bool kVec>
hipError_t launch(RopeArgs a, hipStream_t stream) {
  constexpr int kRows = 64 / (D * static_cast<int>(sizeof(T)) / 16);
  const long long tokens = static_cast<long long>(a.n_seqs) * a.n_tokens;
  const RopeCut c = rope_cut(tokens, a.rows[0].heads + a.rows[1].heads, sizeof(T), D);
  for (long long first = 0; first < tokens; first += c.launch) {
    const long long n = tokens - first < c.launch ? tokens - first : c.launch;
    const dim3 grid(static_cast<unsigned>((n + c.tokens - 1) / c.tokens), static_cast<unsigned>(c.shares));
    a.token0 = static_cast<int32_t>(first);
    if (c.tokens == kWaves * kRows) hipLaunchKernelGGL((rope_kernel<T, D, kWaves * kRows, 2, kVec, true>), grid, dim3(kBlock), 0, stream, a);
    else if (c.tokens == 4) hipLaunchKernelGGL((rope_kernel<T, D, 4, 2, kVec, true>), grid, dim3(kBlock), 0, stream, a);
    else if (c.past) hipLaunchKernelGGL((rope_kernel<T, D, 1, 1, kVec, true>), grid, dim3(kBlock), 0, stream, a);
    else hipLaunchKernelGGL((rope_kernel<T, D, 1, 1, kVec, false>), grid, dim3(kBlock), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename T, int D>
hipError_t launch_any(const RopeArgs &a, hipStream_t stream) {
  // 16 bytes at a time where every row starts at a multiple of 16 bytes
  uintptr_t low = 0;
  for (const RopeRows &r : a.rows) {
    if (r.heads == 0) continue;
    low |= reinterpret_cast<uintptr_t>(r.in) | reinterpret_cast<uintptr_t>(r.out) | reinterpret_cast<uintptr_t>(r.weight);
    low |= static_cast<uintptr_t>(r.in_seq | r.in_token | r.in_head) * sizeof(T);
    if (!a.pages.table) low |= static_cast<uintptr_t>(r.out_seq | r.out_token | r.out_head) * sizeof(T);
  }
  return low % 16 == 0 ? launch<T, D, true>(a, stream) : launch<T, D, false>(a, stream);
}

}  // namespace

hipError_t launch_rope(const RopeArgs &a, int dtype, int head_dim, hipStream_t stream) {
  const long long tokens = static_cast<long long>(a.n_seqs) * a.n_tokens;
  if (tokens < 1 || tokens > (1ll << 30) || a.rows[0].heads < 1 || a.rows[1].heads < 0 || a.half < 0 || a.half > head_dim / 2 || a.half % 8 != 0 ||
      (a.half > 0 && !a.inv_freq) || (a.pages.table && a.rows[1].heads != 0 && a.rows[1].heads != a.rows[0].heads))
    return hipErrorInvalidValue;
  if (dtype == LAZYEV_DTYPE_FP32 && head_dim == 64) return launch_any<float, 64>(a, stream);
  if (dtype == LAZYEV_DTYPE_FP32 && head_dim == 128) return launch_any<float, 128>(a, stream);
  if (dtype == LAZYEV_DTYPE_BF16 && head_dim == 64) return launch_any<bf16_t, 64>(a, stream);
  if (dtype == LAZYEV_DTYPE_BF16 && head_dim == 128) return launch_any<bf16_t, 128>(a, stream);
  return hipErrorInvalidValue;
}

}  // namespace lazyev
