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
// few candidates, at most 64 n.  The largest T of the four wavefronts does for all; so does the least of their (n / 4)-th largest
// lanes, since every wavefront has n / 4 logits from there on, and it lies higher where the large logits are spread: with n = 20 over
// chunks of 8192 some 30 candidates instead of 110.  The candidates --
// all from T on; where those are many, all above T and of those equal to T the first n in the order of their ids -- go to LDS and are
// put in order by counting, for each, those before it.
//
// Sums are in fp32: a thread's of at most 64 terms, then pairwise over the workgroup, then the chunks': 1e-7 of a log probability or an
// entropy against 64 bits (sums in fp64 would be 1e-8).
// Ties go to the lowest id; a NaN counts as +infinity there and makes the sums NaN.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "logprob_parts.hpp"

namespace dk {

namespace {

// The wavefront's n first logits in order, one after the other and from memory: where more logits lie above T than there is room for.
template <typename T, int UNROLL>
__device__ __forceinline__ int pick_rounds(const T* p, int32_t base, int32_t vocab, int n, Pick* out) {
  constexpr int VEC = 16 / (int)sizeof(T);
  const int lane = threadIdx.x & 63;
  Pick last = ~uint64_t(0);
  int count = 0;
  for (int k = 0; k < n; ++k) {
    Pick best = 0;
#pragma unroll 1
    for (int u = 0; u < UNROLL; ++u) {
#pragma unroll 1
      for (int j = 0; j < VEC; ++j) {
        const int32_t id = base + u * (LP_THREADS * VEC) + j;
        if (id >= vocab) continue;
        const Pick x = pick_of(logit_key(logit_at(p, id)), id);
        if (x < last && x > best) best = x;
      }
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) best = max(best, (Pick)__shfl_xor((unsigned long long)best, off));
    if (best == 0) break;
    if (lane == 0) out[count] = best;
    ++count;
    last = best;
  }
  return count;
}

// How many of list[0 .. n) come before q; the list is padded with none to whole eights, so that eight are on their way at a time.
__device__ __forceinline__ int count_before(const Pick* list, int n, Pick q) {
  int rank = 0;
  for (int k = 0; k < n; k += 8) {
#pragma unroll
    for (int j = 0; j < 8; ++j) rank += list[k + j] > q ? 1 : 0;
  }
  return rank;
}
__device__ __forceinline__ void pad_list(Pick* list, int n, int thread) {
  if (thread < 8) list[n + thread] = 0;
}

// x[AT + e], e below 32 and a lane's own: a tree of selections, by masks (the compiler would turn a tree of conditions into one
// that goes through the elements one by one, fifty times as long).
template <int AT, int N>
__device__ __forceinline__ float element(const float (&x)[N], int e) {
  uint32_t v[32];
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = AT + i < N ? __float_as_uint(x[AT + i < N ? AT + i : 0]) : 0u;
#pragma unroll
  for (int half = 16, bit = 0; half >= 1; half >>= 1, ++bit) {
    const uint32_t odd = 0u - ((uint32_t)e >> bit & 1u);
#pragma unroll
    for (int i = 0; i < half; ++i) v[i] = (v[2 * i + 1] & odd) | (v[2 * i] & ~odd);
  }
  return __uint_as_float(v[0]);
}

// A chunk is LP_THREADS * UNROLL * VEC logits; element VEC u + j of a thread is id base + (u LP_THREADS + thread) VEC + j.
template <typename T, int UNROLL, bool ONCE, bool STATS, bool TOP>
__global__ __launch_bounds__(LP_THREADS) void token_logprobs_chunk_kernel(LogprobArgs a, int32_t n_chunks, Part* __restrict__ parts,
                                                                          Pick* __restrict__ tops) {
  constexpr int VEC = 16 / (int)sizeof(T), N = UNROLL * VEC;
  __shared__ Part wave_parts[LP_WAVES];
  __shared__ float2 wave_t[LP_WAVES];
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
    for (int e = 0; e < N; e += 2) asm("v_max3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(m), "v"(x[e]), "v"(x[e + 1]));
    return m;
  };
  float mine = lane_max();
  const float m = wave_max(mine);
  const float c = a.scale * LOG2E, mr = m == -INFINITY ? 0.f : m, mc = mr * c;
  float s0 = 0.f, s1 = 0.f;
  // (eight at a time: an exponential's result may not be used by the very next instruction)
  const auto sums = [&](auto y) {
    float q0 = 0.f, q1 = 0.f;
#pragma unroll
    for (int e = 0; e < N; e += 8) {
      float t[8], w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) t[i] = y(x[e + i]);
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = __builtin_amdgcn_exp2f(t[i]);
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        s0 += w[i];
        q0 += w[i + 1];
        if constexpr (STATS) {
          s1 = __builtin_fmaf(w[i], fmaxf(t[i], -200.f), s1);  // (2^-200 is no float: the weight is zero there)
          q1 = __builtin_fmaf(w[i + 1], fmaxf(t[i + 1], -200.f), q1);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    s0 += q0;
    s1 += q1;
  };
  if (__builtin_fabsf(mc) <= 1048576.f) sums([&](float v) { return __builtin_fmaf(v, c, -mc); });
  else sums([&](float v) { return (v - mr) * c; });  // the difference first: it may be small against what is multiplied
  if (__builtin_amdgcn_ballot_w64(s0 != s0) != 0) {  // a NaN or an infinity: from here on they count by their place
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = logit_key(x[e]);
    mine = lane_max();
  }
  int32_t above = 0;
  if constexpr (STATS) {
#pragma unroll
    for (int e = 0; e < N; ++e) above += x[e] > given ? 1 : 0;
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) above += __shfl_xor(above, off);
  }
  s0 = wave_sum(s0);
  if constexpr (STATS) s1 = wave_sum(s1);
  // y = t - r: what rounding m c took off
  const float r = __builtin_fabsf(mc) <= 1048576.f ? __builtin_fmaf(mr, c, -mc) : 0.f;
  if (lane == 0) wave_parts[wave] = Part{m, s0 * __builtin_amdgcn_exp2f(-r), (s1 - r * s0) * __builtin_amdgcn_exp2f(-r), above};
  if constexpr (TOP) {
    const float2 t = nth_and_kth_largest<sizeof(T) == 2 ? 16 : 20>(mine, a.n_top, (a.n_top + LP_WAVES - 1) / LP_WAVES);
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
    float t = wave_t[0].x, every = wave_t[0].y;
#pragma unroll
    for (int w = 1; w < LP_WAVES; ++w) {
      t = fmaxf(t, wave_t[w].x);
      every = fminf(every, wave_t[w].y);
    }
    t = fmaxf(t, every);
    t = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(t)));
    Pick* out = cands + wave * LP_CAP;
    int count = 0;
    if (__builtin_amdgcn_ballot_w64(mine >= t) != 0) {
      uint32_t which[(N + 31) / 32];  // of the lane's logits; the last one in the lowest bit
      const auto mark = [&](auto take) {
#pragma unroll
        for (int k = 0; k < (N + 31) / 32; ++k) {
          which[k] = 0;
#pragma unroll
          for (int e = 32 * k; e < min(N, 32 * k + 32); ++e) which[k] = which[k] + which[k] + (take(x[e]) ? 1u : 0u);
        }
      };
      const auto collect_32 = [&](auto part) {  // false: more than there is room for
        constexpr int AT = 32 * decltype(part)::value;
        uint32_t w = which[AT / 32];
        for (uint64_t b; (b = __builtin_amdgcn_ballot_w64(w != 0)) != 0;) {
          const int n = __builtin_popcountll(b);
          if (count + n > LP_CAP - 8) return false;
          const int e = min(N - AT, 32) - 1 - __builtin_ctz(w | 0x80000000u);
          const Pick q = pick_of(element<AT>(x, e), id_of(AT + e));
          if (w != 0) out[count + __builtin_amdgcn_mbcnt_hi((uint32_t)(b >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)b, 0))] = q;
          w &= w - 1;
          count += n;
        }
        return true;
      };
      const auto collect = [&]() {
        if constexpr (N > 32) return collect_32(std::integral_constant<int, 0>()) && collect_32(std::integral_constant<int, 1>());
        else return collect_32(std::integral_constant<int, 0>());
      };
      mark([&](float v) { return v >= t; });
      if (t == -INFINITY || !collect()) {
        // Many logits are equal to T (a row held to a few tokens has -infinity everywhere else): all above it, and of those
        // equal the first n, in the order of the ids: lane by lane, 16 bytes by 16 bytes.
        count = 0;
        mark([&](float v) { return v > t; });
        if (collect() && count <= LP_CAP - 8 - LOGPROBS_MAX_TOP) {
          int ties = 0;
#pragma unroll
          for (int u = 0; u < UNROLL; ++u) {
            if (ties >= a.n_top) continue;
            uint64_t equal[VEC];
            int at = ties;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
              equal[j] = __builtin_amdgcn_ballot_w64(x[u * VEC + j] == t && id_of(u * VEC + j) < vocab);
              at += __builtin_amdgcn_mbcnt_hi((uint32_t)(equal[j] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)equal[j], 0));
            }
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
              if (equal[j] >> lane & 1) {
                if (at < a.n_top) out[count + at] = pick_of(t, id_of(u * VEC + j));
                ++at;
              }
              ties += __builtin_popcountll(equal[j]);
            }
          }
          count += min(ties, a.n_top);
        } else {
          count = pick_rounds<T, UNROLL>(p, base, vocab, a.n_top, out);
        }
      }
    }
    pad_list(out, count, lane);
    if (lane == 0) counts[wave] = count;
    __syncthreads();
    Pick* list = tops + ((int64_t)row * n_chunks + chunk) * a.n_top;
    int total = 0;
#pragma unroll
    for (int w = 0; w < LP_WAVES; ++w) total += counts[w];
    // a candidate's place is the number of those before it
    for (int k = threadIdx.x; k < total; k += LP_THREADS) {
      int w = 0, at = k;
      while (at >= counts[w]) at -= counts[w++];
      const Pick mypick = cands[w * LP_CAP + at];
      int rank = 0;
#pragma unroll
      for (int o = 0; o < LP_WAVES; ++o) rank += count_before(cands + o * LP_CAP, counts[o], mypick);
      if (rank < a.n_top) list[rank] = mypick;
    }
    if ((int)threadIdx.x >= total && (int)threadIdx.x < a.n_top) list[threadIdx.x] = 0;  // a short last chunk
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
  __shared__ Pick heads[TOP ? LP_MAX_CHUNKS + 8 : 1];
  __shared__ int32_t lists[TOP ? LOGPROBS_MAX_TOP : 1];
  __shared__ Pick cands[TOP ? LOGPROBS_MAX_TOP * (LOGPROBS_MAX_TOP + 1) / 2 + 8 : 1];
  const int32_t row = blockIdx.x;
  const int tid = threadIdx.x, threads = blockDim.x;
  const float c = a.scale * LOG2E;
  const Part* mine = parts + (int64_t)row * n_chunks;
  const Pick* top = tops + (int64_t)row * n_chunks * a.n_top;
  // (the thread's first chunk, asked for before all else: rows seldom have more chunks than threads)
  const Part own = tid < n_chunks ? mine[tid] : Part{-INFINITY, 0.f, 0.f, 0};
  if constexpr (TOP)
    for (int k = tid; k < n_chunks + 8; k += threads) heads[k] = k < n_chunks ? top[(int64_t)k * a.n_top] : 0;
  const int32_t token = a.tokens ? a.tokens[row] : -1;
  const bool given = token >= 0 && token < a.vocab;
  const int64_t at = (int64_t)row * a.row_stride + (given ? token : 0);
  const float x = a.dtype == 1 ? logit_at((const uint16_t*)a.logits, at) : logit_at((const float*)a.logits, at);
  float m = own.m;
  for (int k = tid + threads; k < n_chunks; k += threads) m = fmaxf(m, mine[k].m);
  m = block_fold(m, fbuf, [](float p, float q) { return fmaxf(p, q); });
  float s0 = 0.f, s1 = 0.f;
  int32_t above = 0;
  const auto take = [&](const Part& o) {
    const float d = o.m == m ? 0.f : (o.m - m) * c, f = __builtin_amdgcn_exp2f(d);
    s0 += f * o.s0;
    s1 += f * (o.s1 + fmaxf(d, -200.f) * o.s0);
    above += o.above;
  };
  take(own);
  for (int k = tid + threads; k < n_chunks; k += threads) take(mine[k]);
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
      const int rank = count_before(heads, n_chunks, heads[k]);
      if (rank < best) lists[rank] = k;
    }
    __syncthreads();
    const int total = best * n - best * (best - 1) / 2;
    for (int k = tid; k < total; k += threads) {
      int r = 0, e = k;
      while (e >= n - r) e -= n - r++;
      cands[k] = top[(int64_t)lists[r] * n + e];
    }
    pad_list(cands, total, tid);
    __syncthreads();
    for (int k = tid; k < total; k += threads) {
      const Pick q = cands[k];
      const int rank = count_before(cands, total, q);
      if (rank >= n || q == 0) continue;
      a.top_ids[(int64_t)row * n + rank] = pick_id(q);
      if (a.top_logprobs) a.top_logprobs[(int64_t)row * n + rank] = (pick_value(q) - m) * a.scale - ln_z;
    }
  }
}

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
  if (a.n_top > 0) token_logprobs_finish_kernel<true><<<dim3((unsigned)a.rows), a.n_top > 22 ? LP_THREADS : 64, 0, stream>>>(a, cut.n_chunks, parts, tops);
  else token_logprobs_finish_kernel<false><<<dim3((unsigned)a.rows), 64, 0, stream>>>(a, cut.n_chunks, parts, tops);
  return hipGetLastError();
}

}  // namespace dk
