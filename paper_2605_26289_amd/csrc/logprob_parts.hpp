// What the kernels that go through logits rows chunk by chunk share: log probabilities (logprobs.hip) and beam selection (beam.hip).
#pragma once
#include <hip/hip_runtime.h>

#include "kernels.hpp"

namespace dk {

constexpr int LP_THREADS = 256;
constexpr int LP_WAVES = LP_THREADS / 64;
constexpr int LP_UNROLL = 8, LP_UNROLL_FEW = 2;  // 16-byte loads of a lane
constexpr int LP_CAP = 256;                      // candidates of a wavefront
constexpr int LP_MAX_CHUNKS = 2048;              // of a row: 2^24 logits of 4 bytes, LP_UNROLL loads a lane
static_assert(LP_MAX_CHUNKS * (LP_THREADS * LP_UNROLL * 4) >= LOGPROBS_MAX_VOCAB, "and so are 2^24 / 4 in shorter chunks, see cut_rows");
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// What a chunk says of its row.
struct Part {
  float m, s0, s1;  // largest logit; sum 2^y and sum 2^y y against it
  int32_t above;
};

__device__ __forceinline__ float logit_key(float x) { return x != x ? INFINITY : x; }
__device__ __forceinline__ float logit_at(const float* p, int64_t i) { return p[i]; }
__device__ __forceinline__ float logit_at(const uint16_t* p, int64_t i) { return __uint_as_float((uint32_t)p[i] << 16); }

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) x = fmaxf(x, __shfl_xor(x, off));
  return x;
}
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) x += __shfl_xor(x, off);
  return x;
}
// Whole numbers in the order of the floats (no NaN; both zeros alike).
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float from_ordered(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }
// A logit and its id as one whole number: the larger comes first, of equals the one with the lower id.  0: none.
typedef uint64_t Pick;
__device__ __forceinline__ Pick pick_of(float x, int32_t id) { return (uint64_t)ordered(x) << 32 | (uint32_t)~id; }
__device__ __forceinline__ float pick_value(Pick p) { return from_ordered((uint32_t)(p >> 32)); }
__device__ __forceinline__ int32_t pick_id(Pick p) { return (int32_t)~(uint32_t)p; }
// The n-th and the k-th largest of the lanes' values, or a little less: the first BITS bits of each, and the smallest value that
// begins with them.
template <int BITS>
__device__ __forceinline__ float2 nth_and_kth_largest(float x, int n, int k) {
  const uint32_t key = ordered(x);
  uint32_t tn = 0, tk = 0;
#pragma unroll
  for (int bit = 31; bit >= 32 - BITS; --bit) {
    const uint32_t un = tn | (1u << bit), uk = tk | (1u << bit);
    if (__builtin_popcountll(__builtin_amdgcn_ballot_w64(key >= un)) >= n) tn = un;
    if (__builtin_popcountll(__builtin_amdgcn_ballot_w64(key >= uk)) >= k) tk = uk;
  }
  // (below are no values, -infinity is the first)
  return make_float2(from_ordered(max(tn, 0x007fffffu)), from_ordered(max(tk, 0x007fffffu)));
}

// Chunks of a row.  Calls of few rows take short chunks, so that more compute units read and the lists of each are shorter.
struct Cut {
  int32_t unroll, n_chunks;
};
inline Cut cut_rows(int32_t rows, int64_t vocab, int32_t dtype) {
  const int64_t per = (int64_t)LP_THREADS * 16 / (dtype == 1 ? 2 : 4);
  const int64_t wide = (vocab + per * LP_UNROLL - 1) / (per * LP_UNROLL);
  if (rows * wide >= 256) return {LP_UNROLL, (int32_t)wide};
  return {LP_UNROLL_FEW, (int32_t)((vocab + per * LP_UNROLL_FEW - 1) / (per * LP_UNROLL_FEW))};
}
inline int64_t parts_bytes(int32_t rows, const Cut& cut) { return ((int64_t)rows * cut.n_chunks * (int64_t)sizeof(Part) + 255) / 256 * 256; }

}  // namespace dk
