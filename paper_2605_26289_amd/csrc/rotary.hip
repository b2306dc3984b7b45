// Norms of queries and keys for each head and their rotation by position, into rows or into the pool's cells (gfx950).
//
// One wavefront per (token, head), elements through LDS, the plain way.
#include <hip/hip_runtime.h>

#include "kernels.hpp"

namespace dk {

namespace {

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(__bf16 x) { return (float)x; }
__device__ __forceinline__ void narrow(float* p, float x) { *p = x; }
__device__ __forceinline__ void narrow(__bf16* p, float x) { *p = (__bf16)x; }

// Where a token is: its position, and its cell (appends).
struct TokenAt {
  int64_t pos;
  int64_t cell;
};

typedef const __attribute__((address_space(4))) RotaryRuns* const_runs_ptr;
__device__ __forceinline__ TokenAt find_token(const_runs_ptr runs, int32_t n_runs, int32_t t) {
  int32_t lo = 0, hi = n_runs - 1;
  while (lo < hi) {
    const int32_t mid = (lo + hi + 1) >> 1;
    if (runs->tok[mid] <= t) lo = mid; else hi = mid - 1;
  }
  const int32_t d = t - runs->tok[lo];
  return {runs->pos[lo] + d, runs->cell[lo] + d};
}

template <typename T, int D>
__device__ __forceinline__ void turn_head(const RotaryArgs& a, const T* src, T* dst, const void* weight, bool turned, int64_t pos, float* buf) {
  const int lane = threadIdx.x & 63;
  float x[D / 64];
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < D / 64; ++j) {
    x[j] = widen(src[lane + 64 * j]);
    sum += x[j] * x[j];
  }
  if (turned && a.norm) {
#pragma unroll
    for (int off = 32; off; off >>= 1) sum += __shfl_xor(sum, off);
    const float inv = 1.f / sqrtf(sum * (1.f / D) + a.eps);
#pragma unroll
    for (int j = 0; j < D / 64; ++j) x[j] *= weight ? inv * widen(((const T*)weight)[lane + 64 * j]) : inv;
  }
#pragma unroll
  for (int j = 0; j < D / 64; ++j) buf[lane + 64 * j] = x[j];
  __syncthreads();
#pragma unroll
  for (int j = 0; j < D / 64; ++j) {
    const int e = lane + 64 * j, half = a.rotary_dim >> 1;
    float y = x[j];
    if (turned && e < a.rotary_dim) {
      const int i = a.pairs ? e >> 1 : (e < half ? e : e - half);
      const bool second = a.pairs ? (e & 1) != 0 : e >= half;
      const float other = buf[a.pairs ? e ^ 1 : (second ? e - half : e + half)];
      const double turns = (double)pos * (double)a.inv_freq[i] * 0.15915494309189535;
      float s, c;
      sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
      y = a.amplitude * (second ? y * c + other * s : y * c - other * s);
    }
    narrow(dst + e, y);
  }
}

template <typename T, int D>
__global__ __launch_bounds__(64) void rotate_append_kernel(RotaryRuns runs, int32_t n_runs, RotaryArgs a) {
  __shared__ float buf[D];
  (void)runs;
  const int32_t heads = a.n_q_heads + 2 * a.n_k_heads;
  const int32_t t = blockIdx.x / heads, h = blockIdx.x % heads;
  const TokenAt at = find_token((const_runs_ptr)__builtin_amdgcn_kernarg_segment_ptr(), n_runs, t);
  const T* src;
  T* dst;
  if (h < a.n_q_heads) {
    src = (const T*)a.q + t * a.q_stride + h * D;
    dst = (T*)a.q_out + ((int64_t)t * a.n_q_heads + h) * D;
  } else {
    const bool is_v = h >= a.n_q_heads + a.n_k_heads;
    const int32_t g = (h - a.n_q_heads) % a.n_k_heads;
    src = is_v ? (const T*)a.v + t * a.v_stride + g * D : (const T*)a.k + t * a.k_stride + g * D;
    dst = (T*)(is_v ? a.v_out : a.k_out) + (g * a.arena_cells + at.cell) * D;
  }
  turn_head<T, D>(a, src, dst, h < a.n_q_heads ? a.q_weight : a.k_weight, h < a.n_q_heads + a.n_k_heads, at.pos, buf);
}

template <typename T, int D>
__global__ __launch_bounds__(64) void rotate_table_kernel(const int32_t* table, int32_t tok_base, RotaryArgs a) {
  __shared__ float buf[D];
  const int32_t heads = a.n_q_heads + 2 * a.n_k_heads;
  const int32_t i = blockIdx.x / heads, h = blockIdx.x % heads;
  const int64_t t = (int64_t)tok_base + i;
  const TokenAt at{table[2 * i], table[2 * i + 1]};
  const T* src;
  T* dst;
  if (h < a.n_q_heads) {
    src = (const T*)a.q + t * a.q_stride + h * D;
    dst = (T*)a.q_out + (t * a.n_q_heads + h) * D;
  } else {
    const bool is_v = h >= a.n_q_heads + a.n_k_heads;
    const int32_t g = (h - a.n_q_heads) % a.n_k_heads;
    src = is_v ? (const T*)a.v + t * a.v_stride + g * D : (const T*)a.k + t * a.k_stride + g * D;
    dst = (T*)(is_v ? a.v_out : a.k_out) + (g * a.arena_cells + at.cell) * D;
  }
  turn_head<T, D>(a, src, dst, h < a.n_q_heads ? a.q_weight : a.k_weight, h < a.n_q_heads + a.n_k_heads, at.pos, buf);
}

template <typename T, int D>
__global__ __launch_bounds__(64) void rotate_rows_kernel(const int64_t* positions, RotaryArgs a) {
  __shared__ float buf[D];
  const int32_t heads = a.n_q_heads + a.n_k_heads;
  const int64_t t = blockIdx.x / heads;
  const int32_t h = blockIdx.x % heads;
  const bool is_q = h < a.n_q_heads;
  const int32_t g = is_q ? h : h - a.n_q_heads;
  const T* src = is_q ? (const T*)a.q + t * a.q_stride + g * D : (const T*)a.k + t * a.k_stride + g * D;
  T* dst = is_q ? (T*)a.q_out + (t * a.n_q_heads + g) * D : (T*)a.k_out + (t * a.n_k_heads + g) * D;
  turn_head<T, D>(a, src, dst, is_q ? a.q_weight : a.k_weight, true, positions[t], buf);
}

#define DK_SHAPES(KERNEL, GRID, ...)                                                                            \
  do {                                                                                                          \
    const dim3 grid((unsigned)(GRID));                                                                          \
    if (a.dtype == 0 && a.head_dim == 64) KERNEL<float, 64><<<grid, 64, 0, stream>>>(__VA_ARGS__);              \
    else if (a.dtype == 0 && a.head_dim == 128) KERNEL<float, 128><<<grid, 64, 0, stream>>>(__VA_ARGS__);       \
    else if (a.dtype == 1 && a.head_dim == 64) KERNEL<__bf16, 64><<<grid, 64, 0, stream>>>(__VA_ARGS__);        \
    else if (a.dtype == 1 && a.head_dim == 128) KERNEL<__bf16, 128><<<grid, 64, 0, stream>>>(__VA_ARGS__);      \
    else return hipErrorInvalidValue;                                                                           \
    return hipGetLastError();                                                                                   \
  } while (0)

}  // namespace

hipError_t launch_rotate_append(const RotaryArgs& a, const RotaryRuns& runs, int32_t n_runs, int32_t n_tok, hipStream_t stream) {
  if (n_tok <= 0) return hipSuccess;
  if (n_runs <= 0 || n_runs > ROTARY_INLINE_MAX_RUNS || runs.tok[n_runs] != n_tok) return hipErrorInvalidValue;
  DK_SHAPES(rotate_append_kernel, (int64_t)n_tok * (a.n_q_heads + 2 * a.n_k_heads), runs, n_runs, a);
}

hipError_t launch_rotate_append_table(const RotaryArgs& a, const int32_t* table_dev, int32_t tok_base, int32_t n_tok, hipStream_t stream) {
  if (n_tok <= 0) return hipSuccess;
  DK_SHAPES(rotate_table_kernel, (int64_t)n_tok * (a.n_q_heads + 2 * a.n_k_heads), table_dev, tok_base, a);
}

hipError_t launch_rotate_rows(const RotaryArgs& a, const int64_t* positions, int64_t n_tok, hipStream_t stream) {
  if (n_tok <= 0 || a.n_q_heads + a.n_k_heads == 0) return hipSuccess;
  DK_SHAPES(rotate_rows_kernel, n_tok * (a.n_q_heads + a.n_k_heads), positions, a);
}

}  // namespace dk
