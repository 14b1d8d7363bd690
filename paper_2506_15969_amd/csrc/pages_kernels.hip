// Attention of tokens that share a context over its pages (lazyev_pages_attend).  One wave per row (token and query
// head): every group of L lanes takes every 64 / L-th entry with a running maximum and sum; the groups are joined at the end.
#include "kernels.h"
#include "lazyev.h"

namespace lazyev {
namespace {

constexpr int kBlock = 256;
typedef unsigned short bf16_t;

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(bf16_t x) { return __uint_as_float(static_cast<unsigned>(x) << 16); }
__device__ __forceinline__ void put(float *p, float x) { *p = x; }
__device__ __forceinline__ void put(bf16_t *p, float x) { *p = __builtin_bit_cast(bf16_t, static_cast<__bf16>(x)); }

// What a row found in the pages (largest logit m, sum l relative to it; l = 0: nothing) and elsewhere: the shares of
// both in the output, the pages' one already divided by l, and the log-sum-exp over both.
struct Joined { float pages, other, lse; };
__device__ __forceinline__ Joined join(float m, float l, bool other, float lse_other) {
  const float lse = l > 0.f || l != l ? m + logf(l) : -INFINITY;
  Joined j;
  if (!other || lse_other == -INFINITY) {
    j.pages = l > 0.f || l != l ? 1.f / l : 0.f;
    j.other = 0.f;
    j.lse = lse;
    return j;
  }
  const float top = fmaxf(lse, lse_other);
  const float a = expf(lse - top), b = expf(lse_other - top);
  j.pages = l > 0.f || l != l ? a / ((a + b) * l) : 0.f;
  j.other = b / (a + b);
  j.lse = top + logf(a + b);
  return j;
}

__device__ __forceinline__ bool takes_part(const AttendArgs &a, int token) {
  if (!a.slots.prompt_len) return true;
  return a.slots.prompt_len[token] >= 0 && a.t - a.slots.t0[token] >= 1;
}

template <typename T, int D>
__global__ __launch_bounds__(kBlock) void attend_kernel(const AttendArgs a) {
  constexpr int E = 16 / static_cast<int>(sizeof(T)), L = D / E, kGroups = 64 / L;
  const int lane = threadIdx.x & 63;
  const long long row = static_cast<long long>(blockIdx.x) * (kBlock / 64) + (threadIdx.x >> 6);
  if (row >= static_cast<long long>(a.n_seqs) * a.n_tokens * a.n_q_heads) return;
  const long long tk = row / a.n_q_heads;
  const int head = static_cast<int>(row % a.n_q_heads), kvh = head / a.group, seq = static_cast<int>(tk / a.n_tokens);
  if (!takes_part(a, static_cast<int>(tk))) return;
  const int seen = a.visible ? min(max(a.visible[tk], 0), a.length) : a.length;
  const int e0 = lane % L * E;
  float q[E], acc[E], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    q[e] = to_float(static_cast<const T *>(a.q)[row * D + e0 + e]);
    acc[e] = 0.f;
  }
  for (int i = lane / L; i < seen; i += kGroups) {
    const int pg = page_of(a.pages, i), page = a.pages.table[static_cast<long long>(seq) * a.pages.stride + pg];
    if (page < 0 || page >= a.pages.n_pages) continue;
    const long long at = ((static_cast<long long>(page) * a.n_kv_heads + kvh) * a.pages.page_size + (i - pg * a.pages.page_size)) * D + e0;
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) s = fmaf(q[e], to_float(static_cast<const T *>(a.k_pages)[at + e]), s);
#pragma unroll
    for (int o = 1; o < L; o <<= 1) s += __shfl_xor(s, o);
    s *= a.scale;
    const float up = s > m ? s : m, keep = m == up ? 1.f : expf(m - up), p = expf(s - up);
    m = up;
    l = l * keep + p;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = fmaf(p, to_float(static_cast<const T *>(a.v_pages)[at + e]), acc[e] * keep);
  }
#pragma unroll
  for (int o = L; o < 64; o <<= 1) {
    const float mo = __shfl_xor(m, o), lo = __shfl_xor(l, o), up = fmaxf(m, mo);
    const float x = m == up ? 1.f : expf(m - up), y = mo == up ? 1.f : expf(mo - up);
    m = up;
    l = l * x + lo * y;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = acc[e] * x + __shfl_xor(acc[e], o) * y;
  }
  const bool other = a.joined_stat || a.joined_lse;
  float lse_other = 0.f;
  float *stat = a.joined_stat ? a.joined_stat + (tk * a.n_kv_heads + kvh) * 16 + 2 * (head % a.group) : nullptr;
  if (stat) lse_other = stat[0] - logf(stat[1]);
  else if (other) lse_other = a.joined_lse[row];
  const Joined j = join(m, l, other, lse_other);
  if (lane < L) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      float x = acc[e] * j.pages;
      if (other && j.other != 0.f) x = fmaf(j.other, to_float(static_cast<const T *>(a.joined_out)[row * D + e0 + e]), x);
      put(static_cast<T *>(a.out) + row * D + e0 + e, x);
    }
  }
  if (lane == 0) {
    if (a.lse) a.lse[row] = j.lse;
    if (stat) stat[1] *= j.other;
  }
}

template <typename T, int D>
hipError_t launch(const AttendArgs &a, hipStream_t stream) {
  const long long rows = static_cast<long long>(a.n_seqs) * a.n_tokens * a.n_q_heads;
  hipLaunchKernelGGL((attend_kernel<T, D>), dim3(static_cast<unsigned>((rows + kBlock / 64 - 1) / (kBlock / 64))), dim3(kBlock), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

size_t attend_workspace(const AttendArgs &) { return 0; }

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
