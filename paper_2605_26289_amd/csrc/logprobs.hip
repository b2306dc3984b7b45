// Log probabilities of given tokens, their rank, the entropy and the best alternatives of logits rows (gfx950).
//
//   token_logprobs_chunk_kernel   one workgroup per (row, chunk): the logits of the chunk are read once, 16 bytes a lane and
//                                 UNROLL of them in flight, and stay in registers for everything that is asked of them.
//                                 With y = scale log2(e) (x - m), m the largest logit: sum 2^y and sum 2^y y, the number of
//                                 logits above the token's, and the n largest in order.
//   token_logprobs_finish_kernel  one workgroup per row folds the chunks:  ln p = scale (x - m) - ln sum 2^y,
//                                 H = ln sum 2^y - ln(2) (sum 2^y y) / sum 2^y.
//
// The n largest of a chunk.  Of the 64 lanes of a wavefront each has its largest logit; T, the n-th largest of those, is found bit
// by bit with ballots.  At least n of the wavefront's logits are T or more, and those above T are in less than n lanes: some n and a
// few candidates, at most 64 n.  The largest T of the four wavefronts does for all.  Candidates go to LDS -- all above T, and of
// those equal to T the first n in the order of their ids -- and are put in order by counting, for each, those before it.
//
// Ties go to the lowest id; a NaN counts as +infinity there and makes the sums NaN.
#include <hip/hip_runtime.h>

#include "kernels.hpp"

namespace dk {

namespace {

constexpr int LP_THREADS = 256;
constexpr int LP_WAVES = LP_THREADS / 64;
constexpr int LP_UNROLL = 8, LP_UNROLL_FEW = 2;  // 16-byte loads of a lane
constexpr int LP_CAP = 256;                      // candidates of a wavefront
constexpr int LP_MAX_CHUNKS = 2048;              // of a row: 2^24 logits of 4 bytes, LP_UNROLL loads a lane
static_assert(LP_MAX_CHUNKS * (LP_THREADS * LP_UNROLL * 4) >= LOGPROBS_MAX_VOCAB, "and so are 2^24 / 4 in shorter chunks, see cut_rows");
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct Pick {
  float v;
  int32_t i;
};
// `a` comes before `b`: larger, or equal with the lower id
__device__ __forceinline__ bool before(Pick a, Pick b) { return a.v > b.v || (a.v == b.v && a.i < b.i); }

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
// The n-th largest of the lanes' values.
__device__ __forceinline__ float nth_largest(float x, int n) {
  const uint32_t key = ordered(x);
  uint32_t t = 0;
#pragma unroll
  for (int bit = 31; bit >= 0; --bit) {
    const uint32_t trial = t | (1u << bit);
    if (__builtin_popcountll(__builtin_amdgcn_ballot_w64(key >= trial)) >= n) t = trial;
  }
  return from_ordered(t);
}

// The wavefront's n first logits in order, one after the other and from memory: where more logits lie above T than there is room for.
template <typename T, int UNROLL>
__device__ __forceinline__ int pick_rounds(const T* p, int32_t base, int32_t vocab, int n, Pick* out) {
  constexpr int VEC = 16 / (int)sizeof(T);
  const int lane = threadIdx.x & 63;
  Pick last{INFINITY, -1};
  int count = 0;
  for (int k = 0; k < n; ++k) {
    Pick best{-INFINITY, INT32_MAX};
#pragma unroll 1
    for (int u = 0; u < UNROLL; ++u) {
#pragma unroll 1
      for (int j = 0; j < VEC; ++j) {
        const int32_t id = base + u * (LP_THREADS * VEC) + j;
        if (id >= vocab) continue;
        const Pick x{logit_key(logit_at(p, id)), id};
        if (before(last, x) && before(x, best)) best = x;
      }
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) {
      const Pick o{__shfl_xor(best.v, off), __shfl_xor(best.i, off)};
      if (before(o, best)) best = o;
    }
    if (best.i == INT32_MAX) break;
    if (lane == 0) out[count] = best;
    ++count;
    last = best;
  }
  return count;
}

// A chunk is LP_THREADS * UNROLL * VEC logits; element VEC u + j of a thread is id base + (u LP_THREADS + thread) VEC + j.
template <typename T, int UNROLL, bool ONCE, bool STATS, bool TOP>
__global__ __launch_bounds__(LP_THREADS) void token_logprobs_chunk_kernel(LogprobArgs a, int32_t n_chunks, Part* __restrict__ parts,
                                                                          Pick* __restrict__ tops) {
  constexpr int VEC = 16 / (int)sizeof(T), N = UNROLL * VEC;
  __shared__ Part wave_parts[LP_WAVES];
  __shared__ float wave_t[LP_WAVES];
  __shared__ int32_t counts[LP_WAVES];
  __shared__ Pick cands[TOP ? LP_WAVES * LP_CAP : 1];
  const int32_t row = blockIdx.x / n_chunks, chunk = blockIdx.x - row * n_chunks;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const T* p = (const T*)a.logits + (int64_t)row * a.row_stride;
  const int32_t vocab = (int32_t)a.vocab;
  const int32_t base = chunk * (LP_THREADS * N) + (int32_t)threadIdx.x * VEC;  // (vocab < 2^31 - chunk: no overflow, see the host)
  const auto id_of = [&](int e) { return base + (e / VEC) * (LP_THREADS * VEC) + e % VEC; };

  typedef uint32_t words __attribute__((ext_vector_type(4)));
  words raw[UNROLL];  // (whole: the last of a row may hold what is behind it, up to the stride)
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    const int32_t e0 = min(base + u * (LP_THREADS * VEC), (vocab - 1) / VEC * VEC);
    raw[u] = ONCE ? __builtin_nontemporal_load((const words*)(p + e0)) : *(const words*)(p + e0);
  }
  const int32_t token = STATS && a.tokens ? a.tokens[row] : -1;
  const float given = token >= 0 && token < vocab ? logit_key(logit_at(p, token)) : INFINITY;
  float x[N];
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      if constexpr (sizeof(T) == 4) x[u * VEC + j] = __uint_as_float(raw[u][j]);
      else x[u * VEC + j] = __uint_as_float(j & 1 ? raw[u][j / 2] & 0xffff0000u : raw[u][j / 2] << 16);
    }
  }
  if ((int64_t)(chunk + 1) * (LP_THREADS * N) > vocab) {  // ragged end of the row: what lies behind it counts for nothing
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (id_of(e) >= vocab) x[e] = -INFINITY;
  }

  const auto lane_max = [&]() {
    float m = x[0];
#pragma unroll
    for (int e = 1; e < N; ++e) m = fmaxf(m, x[e]);
    return m;
  };
  float mine = lane_max();
  const float m = wave_max(mine);
  const float c = a.scale * LOG2E, mr = m == -INFINITY ? 0.f : m, mc = mr * c;
  float s0 = 0.f, s1 = 0.f;
  if (__builtin_fabsf(mc) <= 1048576.f) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float t = __builtin_fmaf(x[e], c, -mc);
      const float w = __builtin_amdgcn_exp2f(t);
      s0 += w;
      if constexpr (STATS) s1 = __builtin_fmaf(w, fmaxf(t, -200.f), s1);  // (2^-200 is no float: the weight is zero there)
    }
  } else {  // the difference first: it may be small against what is multiplied
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float t = (x[e] - mr) * c;
      const float w = __builtin_amdgcn_exp2f(t);
      s0 += w;
      if constexpr (STATS) s1 = __builtin_fmaf(w, fmaxf(t, -200.f), s1);
    }
  }
  if (__builtin_amdgcn_ballot_w64(s0 != s0) != 0) {  // a NaN or an infinity: from here on they count by their place
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = logit_key(x[e]);
    mine = lane_max();
  }
  int32_t above = 0;
  if constexpr (STATS) {
#pragma unroll
    for (int e = 0; e < N; ++e) above += __builtin_popcountll(__builtin_amdgcn_ballot_w64(x[e] > given));
  }
  s0 = wave_sum(s0);
  if constexpr (STATS) s1 = wave_sum(s1);
  // y = t - r: what rounding m c took off
  const float r = __builtin_fabsf(mc) <= 1048576.f ? __builtin_fmaf(mr, c, -mc) : 0.f;
  if (lane == 0) wave_parts[wave] = Part{m, s0 * __builtin_amdgcn_exp2f(-r), (s1 - r * s0) * __builtin_amdgcn_exp2f(-r), above};
  if constexpr (TOP) {
    const float t = nth_largest(mine, a.n_top);
    if (lane == 0) wave_t[wave] = t;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    Part q = wave_parts[0];
#pragma unroll
    for (int w = 1; w < LP_WAVES; ++w) q.m = fmaxf(q.m, wave_parts[w].m);
    q.s0 = q.s1 = 0.f;
    q.above = 0;
#pragma unroll
    for (int w = 0; w < LP_WAVES; ++w) {
      const Part o = wave_parts[w];
      const float d = o.m == q.m ? 0.f : (o.m - q.m) * c, f = __builtin_amdgcn_exp2f(d);
      q.s0 += f * o.s0;
      q.s1 += f * (o.s1 + fmaxf(d, -200.f) * o.s0);
      q.above += o.above;
    }
    parts[(int64_t)row * n_chunks + chunk] = q;
  }
  if constexpr (TOP) {
    float t = wave_t[0];
#pragma unroll
    for (int w = 1; w < LP_WAVES; ++w) t = fmaxf(t, wave_t[w]);
    t = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(t)));
    Pick* out = cands + wave * LP_CAP;
    int count = 0, ties = 0;
    if (__builtin_amdgcn_ballot_w64(mine >= t) != 0) {
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        uint64_t equal[VEC], any = 0;
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const float v = x[u * VEC + j];
          const uint64_t b = __builtin_amdgcn_ballot_w64(v > t);
          if (b != 0) {
            const int n = __builtin_popcountll(b);
            if (v > t && count + n <= LP_CAP - LOGPROBS_MAX_TOP)
              out[count + __builtin_amdgcn_mbcnt_hi((uint32_t)(b >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)b, 0))] = Pick{v, id_of(u * VEC + j)};
            count += n;
          }
          equal[j] = __builtin_amdgcn_ballot_w64(v == t && id_of(u * VEC + j) < vocab);
          any |= equal[j];
        }
        if (any != 0 && ties < a.n_top && count <= LP_CAP - LOGPROBS_MAX_TOP) {  // in the order of the ids: lane by lane
          int at = ties;
#pragma unroll
          for (int j = 0; j < VEC; ++j)
            at += __builtin_amdgcn_mbcnt_hi((uint32_t)(equal[j] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)equal[j], 0));
#pragma unroll
          for (int j = 0; j < VEC; ++j) {
            if (equal[j] >> lane & 1) {
              // (from the end of the wavefront's room, where those above T do not get to)
              if (at < a.n_top) out[LP_CAP - 1 - at] = Pick{t, id_of(u * VEC + j)};
              ++at;
            }
            ties += __builtin_popcountll(equal[j]);
          }
        }
      }
      if (count > LP_CAP - LOGPROBS_MAX_TOP) {
        count = pick_rounds<T, UNROLL>(p, base, vocab, a.n_top, out);
        ties = 0;
      }
      ties = min(ties, a.n_top);
      if (lane < ties) out[count + lane] = out[LP_CAP - 1 - lane];
    }
    if (lane == 0) counts[wave] = count + ties;
    __syncthreads();
    Pick* list = tops + ((int64_t)row * n_chunks + chunk) * a.n_top;
    int total = 0;
#pragma unroll
    for (int w = 0; w < LP_WAVES; ++w) total += counts[w];
    for (int k = threadIdx.x; k < total; k += LP_THREADS) {
      int w = 0, at = k;
      while (at >= counts[w]) at -= counts[w++];
      const Pick mypick = cands[w * LP_CAP + at];
      int rank = 0;
      for (int o = 0; o < LP_WAVES; ++o)
        for (int q = 0; q < counts[o]; ++q) rank += before(cands[o * LP_CAP + q], mypick);
      if (rank < a.n_top) list[rank] = mypick;
    }
    if ((int)threadIdx.x >= total && (int)threadIdx.x < a.n_top) list[threadIdx.x] = Pick{-INFINITY, INT32_MAX};  // a short last chunk
  }
}

template <typename V, typename F>
__device__ __forceinline__ V block_fold(V x, V* buf, F fold) {  // buf: one element a wavefront
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) x = fold(x, __shfl_xor(x, off));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = x;
  __syncthreads();
  V y = buf[0];
  for (int w = 1; w < (int)(blockDim.x >> 6); ++w) y = fold(y, buf[w]);
  return y;
}

// One workgroup per row, of one wavefront where no alternatives are asked for.  The row's n best are in the n lists with the
// best heads, and in the list with the r-th best head (r from 0) among the first n - r: n (n + 1) / 2 to be put in order, by counting.
template <bool TOP>
__global__ __launch_bounds__(LP_THREADS) void token_logprobs_finish_kernel(LogprobArgs a, int32_t n_chunks, const Part* __restrict__ parts,
                                                                           const Pick* __restrict__ tops) {
  __shared__ float fbuf[LP_WAVES];
  __shared__ int32_t ibuf[LP_WAVES];
  __shared__ Pick heads[TOP ? LP_MAX_CHUNKS : 1];
  __shared__ int32_t lists[TOP ? LOGPROBS_MAX_TOP : 1];
  __shared__ Pick cands[TOP ? LOGPROBS_MAX_TOP * (LOGPROBS_MAX_TOP + 1) / 2 : 1];
  const int32_t row = blockIdx.x;
  const int tid = threadIdx.x, threads = blockDim.x;
  const float c = a.scale * LOG2E;
  const Part* mine = parts + (int64_t)row * n_chunks;
  const Pick* top = tops + (int64_t)row * n_chunks * a.n_top;
  if constexpr (TOP)
    for (int k = tid; k < n_chunks; k += threads) heads[k] = top[(int64_t)k * a.n_top];
  const int32_t token = a.tokens ? a.tokens[row] : -1;
  const bool given = token >= 0 && token < a.vocab;
  const int64_t at = (int64_t)row * a.row_stride + (given ? token : 0);
  const float x = a.dtype == 1 ? logit_at((const uint16_t*)a.logits, at) : logit_at((const float*)a.logits, at);
  float m = -INFINITY;
  for (int k = tid; k < n_chunks; k += threads) m = fmaxf(m, mine[k].m);
  m = block_fold(m, fbuf, [](float p, float q) { return fmaxf(p, q); });
  float s0 = 0.f, s1 = 0.f;
  int32_t above = 0;
  for (int k = tid; k < n_chunks; k += threads) {
    const Part o = mine[k];
    const float d = o.m == m ? 0.f : (o.m - m) * c, f = __builtin_amdgcn_exp2f(d);
    s0 += f * o.s0;
    s1 += f * (o.s1 + fmaxf(d, -200.f) * o.s0);
    above += o.above;
  }
  const auto add = [](auto p, auto q) { return p + q; };
  s0 = block_fold(s0, fbuf, add);
  s1 = block_fold(s1, fbuf, add);
  above = block_fold(above, ibuf, add);
  const float lz = log2f(s0);
  const float ln_z = lz * LN2;
  if (tid == 0) {
    if (a.entropy) a.entropy[row] = (lz - s1 / s0) * LN2;
    if (a.logprob) a.logprob[row] = given ? (x - m) * a.scale - ln_z : -INFINITY;
    if (a.rank) a.rank[row] = given ? above : (int32_t)a.vocab;
  }
  if constexpr (TOP) {
    const int n = a.n_top, best = min(n, n_chunks);
    for (int k = tid; k < n_chunks; k += threads) {
      const Pick h = heads[k];
      int rank = 0;
      for (int l = 0; l < n_chunks && rank < n; ++l) rank += before(heads[l], h);
      if (rank < best) lists[rank] = k;
    }
    __syncthreads();
    const int total = best * n - best * (best - 1) / 2;
    for (int k = tid; k < total; k += threads) {
      int r = 0, e = k;
      while (e >= n - r) e -= n - r++;
      cands[k] = top[(int64_t)lists[r] * n + e];
    }
    __syncthreads();
    for (int k = tid; k < total; k += threads) {
      const Pick q = cands[k];
      int rank = 0;
      for (int l = 0; l < total; ++l) rank += before(cands[l], q);
      if (rank >= n || q.i == INT32_MAX) continue;
      a.top_ids[(int64_t)row * n + rank] = q.i;
      if (a.top_logprobs) a.top_logprobs[(int64_t)row * n + rank] = (q.v - m) * a.scale - ln_z;
    }
  }
}

// Chunks of a row.  Calls of few rows take short chunks, so that more compute units read and the lists of each are shorter.
struct Cut {
  int32_t unroll, n_chunks;
};
Cut cut_rows(int32_t rows, int64_t vocab, int32_t dtype) {
  const int64_t per = (int64_t)LP_THREADS * 16 / (dtype == 1 ? 2 : 4);
  const int64_t wide = (vocab + per * LP_UNROLL - 1) / (per * LP_UNROLL);
  if (rows * wide >= 256) return {LP_UNROLL, (int32_t)wide};
  return {LP_UNROLL_FEW, (int32_t)((vocab + per * LP_UNROLL_FEW - 1) / (per * LP_UNROLL_FEW))};
}
int64_t parts_bytes(int32_t rows, const Cut& cut) { return ((int64_t)rows * cut.n_chunks * (int64_t)sizeof(Part) + 255) / 256 * 256; }

template <typename T, int UNROLL>
void launch_chunks(const LogprobArgs& a, const Cut& cut, Part* parts, Pick* tops, hipStream_t stream) {
  const bool once = (int64_t)a.rows * a.vocab * (int64_t)sizeof(T) >= (int64_t)64 << 20;  // (as in verify.hip)
  const bool stats = a.rank || a.entropy;
  const dim3 grid((unsigned)a.rows * (unsigned)cut.n_chunks);
#define DK_CHUNKS(ONCE, STATS, TOP) token_logprobs_chunk_kernel<T, UNROLL, ONCE, STATS, TOP><<<grid, LP_THREADS, 0, stream>>>(a, cut.n_chunks, parts, tops)
  if (once) {
    if (stats) { if (a.n_top) DK_CHUNKS(true, true, true); else DK_CHUNKS(true, true, false); }
    else { if (a.n_top) DK_CHUNKS(true, false, true); else DK_CHUNKS(true, false, false); }
  } else {
    if (stats) { if (a.n_top) DK_CHUNKS(false, true, true); else DK_CHUNKS(false, true, false); }
    else { if (a.n_top) DK_CHUNKS(false, false, true); else DK_CHUNKS(false, false, false); }
  }
#undef DK_CHUNKS
}

}  // namespace

int64_t logprobs_workspace_bytes(int32_t rows, int64_t vocab, int32_t dtype, int32_t n_top) {
  const Cut cut = cut_rows(rows, vocab, dtype);
  return parts_bytes(rows, cut) + (int64_t)rows * cut.n_chunks * n_top * (int64_t)sizeof(Pick) + 256;
}

hipError_t launch_token_logprobs(const LogprobArgs& a, void* workspace, hipStream_t stream) {
  if (a.rows <= 0) return hipSuccess;
  const Cut cut = cut_rows(a.rows, a.vocab, a.dtype);
  if ((int64_t)a.rows * cut.n_chunks >= (int64_t(1) << 32) / LP_THREADS || cut.n_chunks > LP_MAX_CHUNKS) return hipErrorInvalidValue;
  Part* parts = (Part*)workspace;
  Pick* tops = (Pick*)((char*)workspace + parts_bytes(a.rows, cut));
  const bool wide = cut.unroll == LP_UNROLL;
  if (a.dtype == 1) wide ? launch_chunks<uint16_t, LP_UNROLL>(a, cut, parts, tops, stream) : launch_chunks<uint16_t, LP_UNROLL_FEW>(a, cut, parts, tops, stream);
  else wide ? launch_chunks<float, LP_UNROLL>(a, cut, parts, tops, stream) : launch_chunks<float, LP_UNROLL_FEW>(a, cut, parts, tops, stream);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (a.n_top > 0) token_logprobs_finish_kernel<true><<<dim3((unsigned)a.rows), LP_THREADS, 0, stream>>>(a, cut.n_chunks, parts, tops);
  else token_logprobs_finish_kernel<false><<<dim3((unsigned)a.rows), 64, 0, stream>>>(a, cut.n_chunks, parts, tops);
  return hipGetLastError();
}

}  // namespace dk
