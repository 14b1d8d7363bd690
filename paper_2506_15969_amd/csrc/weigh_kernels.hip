// The attention weight that every entry of a cache received (lazyev_pages_weigh): w[i] = (old) + sum over the rows r that see entry i of
// exp(scale q_r k_i - lse_r), rows being the tokens' heads of the entry's group.
//
// A wave keeps 32 entries' keys as the B operand of 32 x 32 products (32x32x16_bf16; fp32 rows: 32x32x2_f32) and goes over the rows, 32 at a time as A:
// lane (c, h) = (l % 32, l / 32) holds, of entry c, the logits of the rows 8 i + 4 h + j (i, j < 4), so the sum over rows
// is one in its register.  Rows that do not see all of the entries are masked, by the number of entries that they see; those past the last, and those
// that saw nothing (lse of -inf), see none.
//
// Few entries: the rows are cut into splits too, every n-th tile of 32 to each (where tokens see their past, late rows are seen by
// all entries, early ones by few), whose sums a second kernel adds in their order.
#include "kernels.h"
#include "lazyev.h"

#include <climits>

namespace lazyev {
namespace {

typedef unsigned short bf16_t;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4_t;

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kEntries = 128;           // of a block
constexpr int kSplitMax = 64;

template <typename T>
__device__ __forceinline__ u32x4_t load_chunk(const T *p, bool wide) {
  if (wide) return *reinterpret_cast<const u32x4_t *>(p);
  T e[16 / sizeof(T)];
#pragma unroll
  for (int x = 0; x < static_cast<int>(16 / sizeof(T)); ++x) e[x] = p[x];
  u32x4_t w;
  __builtin_memcpy(&w, e, 16);
  return w;
}

// What an entry had before.
__device__ __forceinline__ float before(const WeighArgs &a, long long at, int entry) { return entry < a.known ? a.decay * a.old[at] : 0.f; }

template <typename T, int D>
__global__ __launch_bounds__(256) void weigh_kernel(const WeighArgs a) {
  constexpr bool kF32 = sizeof(T) == 4;
  constexpr int kOps = D * static_cast<int>(sizeof(T)) / 32;
  __shared__ __align__(16) float row_lse[4][32];
  __shared__ __align__(16) int row_sees[4][32];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = lane & 31, h = lane >> 5;
  const int across = (a.length + kEntries - 1) / kEntries;
  const int unit = static_cast<int>(blockIdx.x / across), split = static_cast<int>(blockIdx.y);
  const int seq = unit / a.n_kv_heads, kvh = unit - seq * a.n_kv_heads;
  const int e0 = (static_cast<int>(blockIdx.x) - unit * across) * kEntries + wave * 32;
  if (e0 >= a.length) return;
  const int entry = min(e0 + c, a.length - 1), end = min(e0 + 32, a.length);
  const int pg = page_of(a.pages, entry);
  const unsigned no = static_cast<unsigned>(a.pages.table[static_cast<long long>(seq) * a.pages.stride + pg]);
  const bool there = no < static_cast<unsigned>(a.pages.n_pages);
  const unsigned head_rows = static_cast<unsigned>(a.pages.page_size), page_rows = head_rows * static_cast<unsigned>(a.n_kv_heads);
  const unsigned k_row = (there ? no : 0u) * page_rows + kvh * head_rows + static_cast<unsigned>(entry - pg * a.pages.page_size);
  u32x4_t k[kOps];
  {
    const char *from = static_cast<const char *>(a.k_pages) + static_cast<size_t>(k_row) * (D * sizeof(T)) + h * 16;
#pragma unroll
    for (int j = 0; j < kOps; ++j) k[j] = *reinterpret_cast<const u32x4_t *>(from + j * 32);
  }
  const int M = a.n_tokens * a.group, tiles = (M + 31) / 32;
  const float c2 = a.scale * kLog2e;
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  for (int tile = split; tile < tiles; tile += a.n_split) {
    const int r = tile * 32 + c, rr = min(r, M - 1), i = rr / a.group;
    const long long token = static_cast<long long>(seq) * a.n_tokens + i;
    const long long row = token * a.n_q_heads + static_cast<long long>(kvh) * a.group + (rr - i * a.group);
    const float lse = a.lse[row];
    int sees = a.visible ? min(max(a.visible[token], 0), a.length) : a.length;
    if (r >= M || lse == -INFINITY) sees = 0;
    int most = sees, least = sees;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      most = max(most, __shfl_xor(most, o));
      least = min(least, __shfl_xor(least, o));
    }
    most = __builtin_amdgcn_readfirstlane(most);
    least = __builtin_amdgcn_readfirstlane(least);
    if (most <= e0) continue;                      // (wave-uniform) nobody sees them
    if (h == 0) {
      row_lse[wave][c] = lse * kLog2e;
      row_sees[wave][c] = sees;
    }
    const T *q = static_cast<const T *>(a.q) + row * D + h * (16 / sizeof(T));
    f32x16_t s;
#pragma unroll
    for (int x = 0; x < 16; ++x) s[x] = 0.f;
#pragma unroll
    for (int j = 0; j < kOps; ++j) {
      const u32x4_t w = load_chunk(q + j * (32 / sizeof(T)), a.wide);
      if constexpr (kF32) {
#pragma unroll
        for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(w[e]), __uint_as_float(k[j][e]), s, 0, 0, 0);
      } else {
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, w), __builtin_bit_cast(bf16x8_t, k[j]), s, 0, 0, 0);
      }
    }
    __builtin_amdgcn_wave_barrier();
    const bool mask = least < end;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const f32x4_t ref = *reinterpret_cast<const f32x4_t *>(&row_lse[wave][8 * x + 4 * h]);
      const int *limit = &row_sees[wave][8 * x + 4 * h];
      float p[4];
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        p[y] = __builtin_amdgcn_exp2f(fmaf(s[4 * x + y], c2, -ref[y]));
        if (mask) p[y] = e0 + c < limit[y] ? p[y] : 0.f;
      }
      sum[x] += (p[0] + p[1]) + (p[2] + p[3]);
    }
    __builtin_amdgcn_wave_barrier();
  }
  float w = (sum[0] + sum[1]) + (sum[2] + sum[3]);
  w += __shfl_xor(w, 32);
  if (h != 0 || e0 + c >= a.length) return;
  if (!there) w = 0.f;
  if (a.n_split > 1) {
    a.part[(static_cast<size_t>(split) * a.n_seqs * a.n_kv_heads + unit) * a.length + e0 + c] = w;
    return;
  }
  const long long at = static_cast<long long>(unit) * a.stride + e0 + c;
  a.weights[at] = before(a, at, e0 + c) + w;
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

// Splits of the rows: a few blocks for every compute unit.
int splits_of(const WeighArgs &a) {
  const long long blocks = static_cast<long long>(a.n_seqs) * a.n_kv_heads * ((a.length + kEntries - 1) / kEntries);
  const int tiles = (a.n_tokens * a.group + 31) / 32;
  long long n = blocks > 0 ? 1024 / blocks : 1;
  if (n > tiles / 4) n = tiles / 4;
  return static_cast<int>(n < 1 ? 1 : n > kSplitMax ? kSplitMax : n);
}

template <typename T, int D>
hipError_t launch(const WeighArgs &a, hipStream_t stream) {
  const long long blocks = static_cast<long long>(a.n_seqs) * a.n_kv_heads * ((a.length + kEntries - 1) / kEntries);
  if (blocks < 1 || blocks >= (1ll << 24)) return hipErrorInvalidValue;
  hipLaunchKernelGGL((weigh_kernel<T, D>), dim3(static_cast<unsigned>(blocks), static_cast<unsigned>(a.n_split)), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

size_t weigh_workspace(const WeighArgs &a) {
  const int n = splits_of(a);
  return n > 1 ? (static_cast<size_t>(n) * a.n_seqs * a.n_kv_heads * a.length * 4 + 255) / 256 * 256 : 0;
}

hipError_t launch_weigh(WeighArgs a, hipStream_t stream) {
  a.n_split = splits_of(a);
  a.wide = reinterpret_cast<uintptr_t>(a.q) % 16 == 0;
  hipError_t e;
  if (a.dtype == LAZYEV_DTYPE_FP32) e = a.head_dim == 64 ? launch<float, 64>(a, stream) : launch<float, 128>(a, stream);
  else e = a.head_dim == 64 ? launch<bf16_t, 64>(a, stream) : launch<bf16_t, 128>(a, stream);
  if (e != hipSuccess || a.n_split <= 1) return e;
  const long long n = static_cast<long long>(a.n_seqs) * a.n_kv_heads * a.length;
  hipLaunchKernelGGL(weigh_join_kernel, dim3(static_cast<unsigned>((n + 255) / 256)), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace lazyev
