// Log probabilities of given tokens, their rank, the entropy and the best alternatives of logits rows (gfx950).
//
// One workgroup per row, the plain way: a pass for the maximum, one for the sums, one for every alternative.
#include <hip/hip_runtime.h>

#include "kernels.hpp"

namespace dk {

namespace {

constexpr int LOGPROB_THREADS = 256;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

__device__ __forceinline__ float logit_key(float x) { return x != x ? INFINITY : x; }
__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(uint16_t bits) { return __uint_as_float((uint32_t)bits << 16); }

struct Pick {
  float v;
  int32_t i;
};
// `a` comes before `b`: larger, or equal with the lower id
__device__ __forceinline__ bool before(Pick a, Pick b) { return a.v > b.v || (a.v == b.v && a.i < b.i); }

template <typename V, typename F>
__device__ V block_fold(V x, V* buf, F fold) {
  __syncthreads();
  buf[threadIdx.x] = x;
  __syncthreads();
  for (int half = LOGPROB_THREADS / 2; half > 0; half >>= 1) {
    if ((int)threadIdx.x < half) buf[threadIdx.x] = fold(buf[threadIdx.x], buf[threadIdx.x + half]);
    __syncthreads();
  }
  return buf[0];
}

template <typename T>
__global__ __launch_bounds__(LOGPROB_THREADS) void token_logprobs_kernel(LogprobArgs a) {
  __shared__ Pick picks[LOGPROB_THREADS];
  __shared__ float sums[LOGPROB_THREADS];
  const int64_t row = blockIdx.x;
  const T* p = (const T*)a.logits + row * a.row_stride;
  const auto earlier = [](Pick x, Pick y) { return before(x, y) ? x : y; };
  const auto add = [](float x, float y) { return x + y; };
  Pick best{-INFINITY, INT32_MAX};
  for (int64_t i = threadIdx.x; i < a.vocab; i += LOGPROB_THREADS) best = earlier(best, Pick{logit_key(widen(p[i])), (int32_t)i});
  best = block_fold(best, picks, earlier);
  const float m = best.v, c = a.scale * LOG2E;
  const int32_t token = a.tokens ? a.tokens[row] : -1;
  const bool given = token >= 0 && token < a.vocab;
  const float xt = given ? widen(p[token]) : 0.f, kt = logit_key(xt);
  float s0 = 0.f, s1 = 0.f, above = 0.f;
  for (int64_t i = threadIdx.x; i < a.vocab; i += LOGPROB_THREADS) {
    const float x = widen(p[i]);
    const float t = (x - m) * c;
    const float e = exp2f(t);
    s0 += e;
    s1 += e > 0.f || e != e ? e * t : 0.f;
    above += logit_key(x) > kt ? 1.f : 0.f;
  }
  s0 = block_fold(s0, sums, add);
  s1 = block_fold(s1, sums, add);
  above = block_fold(above, sums, add);
  const float lz = log2f(s0);
  if (threadIdx.x == 0) {
    if (a.logprob) a.logprob[row] = given ? (xt - m) * a.scale - lz * LN2 : -INFINITY;
    if (a.rank) a.rank[row] = given ? (int32_t)above : (int32_t)a.vocab;
    if (a.entropy) a.entropy[row] = (lz - s1 / s0) * LN2;
  }
  Pick last{INFINITY, -1};
  for (int32_t k = 0; k < a.n_top; ++k) {
    Pick next{-INFINITY, INT32_MAX};
    for (int64_t i = threadIdx.x; i < a.vocab; i += LOGPROB_THREADS) {
      const Pick x{logit_key(widen(p[i])), (int32_t)i};
      if (before(last, x)) next = earlier(next, x);
    }
    last = block_fold(next, picks, earlier);
    if (threadIdx.x == 0) {
      a.top_ids[row * a.n_top + k] = last.i;
      if (a.top_logprobs) a.top_logprobs[row * a.n_top + k] = (last.v - m) * a.scale - lz * LN2;
    }
  }
}

}  // namespace

int64_t logprobs_workspace_bytes(int32_t, int64_t, int32_t, int32_t) { return 256; }

hipError_t launch_token_logprobs(const LogprobArgs& a, void*, hipStream_t stream) {
  if (a.rows <= 0) return hipSuccess;
  if (a.dtype == 1) token_logprobs_kernel<uint16_t><<<dim3((unsigned)a.rows), LOGPROB_THREADS, 0, stream>>>(a);
  else token_logprobs_kernel<float><<<dim3((unsigned)a.rows), LOGPROB_THREADS, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace dk
