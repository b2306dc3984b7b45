// Delta attention with changed scores (gfx950): capped by a tanh, biased by distance, and rows that see a range of
// positions of their own.
//
//   s = scale q.k,  s <- cap tanh(s / cap),  s <- s - slope_h |p_q - p_k|,
//   row p sees positions max(first, p - window + 1) .. max(p, prefix - 1);  O = softmax(s) V.
//
// One wavefront per (token, query head), a lane per key, the plain way.
#include <hip/hip_runtime.h>

#include "kernels.hpp"

namespace dk {

namespace {

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(__bf16 x) { return (float)x; }
__device__ __forceinline__ void narrow(float* p, float x) { *p = x; }
__device__ __forceinline__ void narrow(__bf16* p, float x) { *p = (__bf16)x; }

template <bool INLINE> struct BlobOf;
template <> struct BlobOf<true> { InlineBlob blob; };
template <> struct BlobOf<false> { char unused; };
template <bool INLINE, typename P>
__device__ __forceinline__ const P* in_blob(const P* p) {
  if constexpr (INLINE) {
    typedef const __attribute__((address_space(4))) char* const_char_ptr;
    return (const P*)((uintptr_t)(const_char_ptr)__builtin_amdgcn_kernarg_segment_ptr() + (uintptr_t)p);
  } else {
    return p;
  }
}

template <typename T, int D, bool INLINE>
__global__ __launch_bounds__(64) void scored_plain_kernel(BlobOf<INLINE> blob, AttendArgs a, ScoreArgs sc) {
  __shared__ float qs[D];
  __shared__ float red[64][D + 1];
  (void)blob;
  const DkEntry* entries = in_blob<INLINE>(a.entries);
  const DkSeg* segs = in_blob<INLINE>(a.segs);
  const int32_t* first = in_blob<INLINE>(sc.first);
  const int n_q_heads = a.arena.n_q_heads, n_kv_heads = a.arena.n_kv_heads;
  const int lane = threadIdx.x;
  const int tok = blockIdx.x / n_q_heads, h = blockIdx.x % n_q_heads;
  int lo = 0, hi = a.n_entries - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (entries[mid].tok0 <= tok) lo = mid; else hi = mid - 1;
  }
  while (entries[lo].delta == 0 || tok >= entries[lo].tok0 + entries[lo].delta) --lo;  // empty entries share a tok0
  const DkEntry e = entries[lo];
  const int pos = e.n + tok - e.tok0;
  const int last = max(pos, e.pad[0] - 1);
  int from = sc.masked_first ? first[tok] : 0;
  if (sc.window > 0) from = max(from, pos - sc.window + 1);
  const int g = h / (n_q_heads / n_kv_heads);
  const float slope = sc.slopes ? sc.slopes[h] : 0.f;
  const T* q = (const T*)a.q + ((int64_t)tok * n_q_heads + h) * D;
  for (int d = lane; d < D; d += 64) qs[d] = widen(q[d]);
  __syncthreads();

  float m = -INFINITY, l = 0.f;
  float o[D];
#pragma unroll
  for (int d = 0; d < D; ++d) o[d] = 0.f;
  for (int si = e.seg_begin; si < e.seg_end; ++si) {
    const DkSeg sg = segs[si];
    for (int j = lane; j < sg.len; j += 64) {
      const int key = sg.pos + j;
      if (key < from || key > last) continue;
      const int64_t off = (sg.src == 0 ? (int64_t)g * a.arena.arena_cells + sg.start + j : (sg.start + j) * n_kv_heads + g) * D;
      const T* kr = (const T*)(sg.src == 0 ? a.arena.k_arena : a.k_new) + off;
      const T* vr = (const T*)(sg.src == 0 ? a.arena.v_arena : a.v_new) + off;
      float s = 0.f;
      for (int d = 0; d < D; ++d) s += qs[d] * widen(kr[d]);
      s *= a.scale;
      if (sc.cap > 0.f) s = sc.cap * tanhf(s / sc.cap);
      s -= slope * (float)abs(pos - key);
      s *= 1.4426950408889634f;
      const float mn = fmaxf(m, s), ms = mn == -INFINITY ? 0.f : mn;
      const float alpha = exp2f(m - ms), p = exp2f(s - ms);
      l = l * alpha + p;
#pragma unroll
      for (int d = 0; d < D; ++d) o[d] = o[d] * alpha + p * widen(vr[d]);
      m = mn;
    }
  }
  float mw = m;
  for (int off = 32; off; off >>= 1) mw = fmaxf(mw, __shfl_xor(mw, off));
  const float f = m == -INFINITY ? 0.f : exp2f(m - mw);
  float lw = l * f;
  for (int off = 32; off; off >>= 1) lw += __shfl_xor(lw, off);
#pragma unroll
  for (int d = 0; d < D; ++d) red[lane][d] = l == 0.f ? 0.f : o[d] * f;
  __syncthreads();
  const float inv = lw == 0.f ? 0.f : 1.f / lw;
  T* out = (T*)a.out + ((int64_t)tok * n_q_heads + h) * D;
  for (int d = lane; d < D; d += 64) {
    float acc = 0.f;
    for (int r = 0; r < 64; ++r) acc += red[r][d];
    narrow(out + d, acc * inv);
  }
  if (a.lse && lane == 0) a.lse[(int64_t)tok * n_q_heads + h] = lw == 0.f ? -INFINITY : (mw + log2f(lw)) * 0.6931471805599453f;
}

template <typename T, int D>
hipError_t launch_plain(const AttendArgs& a, const ScoreArgs& sc, hipStream_t stream) {
  const dim3 grid((unsigned)((int64_t)a.total_tokens * a.arena.n_q_heads));
  if (a.inline_blob) scored_plain_kernel<T, D, true><<<grid, 64, 0, stream>>>(BlobOf<true>{*a.inline_blob}, a, sc);
  else scored_plain_kernel<T, D, false><<<grid, 64, 0, stream>>>(BlobOf<false>{0}, a, sc);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attend_scored(const AttendArgs& a, const ScoreArgs& sc, hipStream_t stream) {
  if (a.total_tokens <= 0) return hipSuccess;
  if (a.arena.dtype == 0 && a.arena.head_dim == 64) return launch_plain<float, 64>(a, sc, stream);
  if (a.arena.dtype == 0 && a.arena.head_dim == 128) return launch_plain<float, 128>(a, sc, stream);
  if (a.arena.dtype == 1 && a.arena.head_dim == 64) return launch_plain<__bf16, 64>(a, sc, stream);
  if (a.arena.dtype == 1 && a.arena.head_dim == 128) return launch_plain<__bf16, 128>(a, sc, stream);
  return hipErrorInvalidValue;
}

}  // namespace dk
