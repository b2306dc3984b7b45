// The best continuations of each request's beams (gfx950): of every row r of a group and every token t
//
//   score(r, t) = scores[r] + scale x_rt - ln sum_u exp(scale x_ru),
//
// the n largest.  The rows' chunks are read by token_logprobs_chunk_kernel, which leaves each chunk's largest logit, its sum against that
// and its n best logits in order; beam_select_kernel, one workgroup per group, folds the sums of the group's rows and picks from the
// lists.  Scores are made and compared in fp64: rows of one group differ by sums of 10^5 terms, and two continuations may be close.
//
// The pick.  The first k entries of all lists (k so that there are 2 n of them, 1 where there are many lists) are n or more
// continuations, so T, the n-th largest of their scores by its upper 32 bits, is at most the n-th best of all.  Whatever reaches T --
// the beginning of some lists -- goes to LDS, a hundred or two, and each one's place is the number of those before it.  Where more do than there is room for
// (equal logits by the thousand), T is raised to the n-th of those that came and the lists are gone through again.
#include <hip/hip_runtime.h>

#include "logprob_parts.hpp"

namespace dk {

namespace {

constexpr int BEAM_THREADS = 256, BEAM_WAVES = BEAM_THREADS / 64;
constexpr int BEAM_ID_BITS = 20;
static_assert(BEAM_MAX_VOCAB <= 1 << BEAM_ID_BITS && BEAM_MAX_ROWS <= 1 << (64 - 32 - BEAM_ID_BITS), "row, logit and token in 64 bits");
constexpr int BEAM_MAX_LISTS = BEAM_MAX_ROWS * (int)((BEAM_MAX_VOCAB + LP_THREADS * LP_UNROLL * 4 - 1) / (LP_THREADS * LP_UNROLL * 4));
static_assert(BEAM_MAX_LISTS >= 1024, "calls of few rows have fewer than 4 x 256 chunks");
constexpr int BEAM_MAX_HEADS = BEAM_MAX_LISTS + 2 * BEAM_MAX_OUT;
constexpr int BEAM_CAP = 1024;  // continuations that reach T
constexpr int BEAM_OWN = 8;      // entries that a thread asks for before all else
constexpr int BEAM_ROW_SUMS = 16;

// Whole numbers in the order of the doubles (no NaN).  0: none.
__device__ __forceinline__ uint64_t ordered64(double x) {
  const uint64_t b = (uint64_t)__double_as_longlong(x + 0.0);
  return b ^ ((uint64_t)((int64_t)b >> 63) | 0x8000000000000000ull);
}
__device__ __forceinline__ double from_ordered64(uint64_t k) {
  return __longlong_as_double((int64_t)(k & 0x8000000000000000ull ? k ^ 0x8000000000000000ull : ~k));
}

// A continuation in the order wanted: by score, then the lower row, the larger logit, the lower token.
struct Found {
  uint64_t score, rest;
  __device__ __forceinline__ bool before(const Found& o) const { return score > o.score || (score == o.score && rest > o.rest); }
};
__device__ __forceinline__ uint64_t rest_of(int row, Pick p) {
  return (uint64_t)(BEAM_MAX_ROWS - 1 - row) << (32 + BEAM_ID_BITS) | (p >> 32) << BEAM_ID_BITS | (uint64_t)((1 << BEAM_ID_BITS) - 1 - pick_id(p));
}

}  // namespace

__global__ __launch_bounds__(BEAM_THREADS) void beam_select_kernel(BeamArgs a, int32_t n_chunks, const Part* __restrict__ parts,
                                                                   const Pick* __restrict__ tops) {
  __shared__ float2 sums[BEAM_MAX_ROWS * BEAM_ROW_SUMS];  // largest logit and sum of the rows' chunks, where they fit
  __shared__ uint32_t heads[BEAM_MAX_HEADS];
  __shared__ Found found[BEAM_CAP];
  __shared__ double base[BEAM_MAX_ROWS];  // of a row that takes part: its score less the log of its sum
  __shared__ float most[BEAM_MAX_ROWS];   // its largest logit; NaN: it takes no part
  __shared__ int32_t came;
  __shared__ Found bound;
  const int g = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = a.n_out;
  const int r0 = min(max(a.cu_rows[g], 0), a.rows);
  const int rows = min(min(max(a.cu_rows[g + 1], r0), a.rows) - r0, BEAM_MAX_ROWS);
  const int lists = rows * n_chunks, entries = lists * n;
  const Part* gp = parts + (int64_t)r0 * n_chunks;
  const Pick* gt = tops + (int64_t)r0 * n_chunks * n;

  // All that is read is asked for at once, as far as it fits the registers: the kernel is a chain of round trips.
  Pick own[BEAM_OWN];
#pragma unroll
  for (int j = 0; j < BEAM_OWN; ++j) own[j] = tid + j * BEAM_THREADS < entries ? gt[tid + j * BEAM_THREADS] : 0;
  const float own_score = tid < rows ? a.scores[r0 + tid] : 0.f;
  const bool fits = n_chunks <= BEAM_ROW_SUMS;
  if (fits) {
    for (int i = tid; i < lists; i += BEAM_THREADS) sums[i] = make_float2(gp[i].m, gp[i].s0);
  }
  if (tid < rows) most[tid] = own_score;
  __syncthreads();

  // the rows' sums, `per` lanes to a row
  int per = 1;
  while (per < 64 && per < n_chunks) per *= 2;
  const double c = a.scale * 1.4426950408889634;
  for (int at = 0; at < rows; at += BEAM_THREADS / per) {
    const int r = at + tid / per, sub = tid % per;
    const bool there = r < rows;
    const auto part = [&](int k) { return fits ? sums[r * n_chunks + k] : make_float2(gp[r * n_chunks + k].m, gp[r * n_chunks + k].s0); };
    float m = -INFINITY;
    for (int k = sub; there && k < n_chunks; k += per) m = fmaxf(m, part(k).x);
    for (int off = per / 2; off >= 1; off /= 2) m = fmaxf(m, __shfl_xor(m, off));
    double s = 0.0;
    for (int k = sub; there && k < n_chunks; k += per) {
      const float2 p = part(k);  // (of a chunk of nothing but -infinity the sum is 0, of one with a NaN it is one)
      s += p.x == -INFINITY ? (double)p.y : (double)p.y * exp2(((double)p.x - (double)m) * c);
    }
    for (int off = per / 2; off >= 1; off /= 2) s += __shfl_xor(s, off);
    if (there && sub == 0) {
      const float score = most[r];
      const bool live = __builtin_fabsf(score) < INFINITY && __builtin_fabsf(m) < INFINITY && s > 0.0 && s < (double)INFINITY;
      base[r] = live ? (double)score - log(s) : 0.0;
      most[r] = live ? m : __uint_as_float(0x7fc00000u);
    }
  }
  __syncthreads();
  // score of a list's entry, as a whole number; 0: none
  const auto score_of = [&](int row, Pick p) -> uint64_t {
    const float x = pick_value(p), m = most[row];
    if (p == 0 || m != m || x == -INFINITY) return 0;
    return ordered64(base[row] + ((double)x - (double)m) * a.scale);
  };

  const int k = lists > 0 ? min(n, (2 * n + lists - 1) / lists) : 0;
  const int n_heads = lists * k;
  uint64_t own_key[BEAM_OWN];
  int own_list[BEAM_OWN];
#pragma unroll
  for (int j = 0; j < BEAM_OWN; ++j) {
    const int i = tid + j * BEAM_THREADS;
    own_key[j] = 0;
    own_list[j] = 0;
    if (j * BEAM_THREADS >= entries || i >= entries) continue;
    own_list[j] = i / n;
    own_key[j] = score_of(own_list[j] / n_chunks, own[j]);
    const int e = i - own_list[j] * n;
    if (e < k) heads[own_list[j] * k + e] = (uint32_t)(own_key[j] >> 32);
  }
  for (int i = tid; i < n_heads && entries > BEAM_OWN * BEAM_THREADS; i += BEAM_THREADS) {
    const int list = i / k, e = i - list * k;
    if (list * n + e >= BEAM_OWN * BEAM_THREADS) heads[i] = (uint32_t)(score_of(list / n_chunks, gt[list * n + e]) >> 32);
  }
  if (tid == 0) came = 0;
  __syncthreads();
  // Every wavefront finds T by itself, bit by bit; its last bits (2^-10 of a score and less) do not matter.
  uint32_t t = 0;
  if (n_heads > n) {
    constexpr int KEEP = 4;
    uint32_t mine[KEEP];
#pragma unroll
    for (int i = 0; i < KEEP; ++i) mine[i] = lane + 64 * i < n_heads ? heads[lane + 64 * i] : 0u;
    for (int bit = 31; bit >= 10; --bit) {
      const uint32_t u = t | 1u << bit;
      int count = __builtin_popcountll(__builtin_amdgcn_ballot_w64(mine[0] >= u));
      if (n_heads > 64) {
#pragma unroll
        for (int i = 1; i < KEEP; ++i) count += __builtin_popcountll(__builtin_amdgcn_ballot_w64(mine[i] >= u));
        for (int i = 64 * KEEP; i < n_heads; i += 64) count += __builtin_popcountll(__builtin_amdgcn_ballot_w64(i + lane < n_heads && heads[i + lane] >= u));
      }
      if (count >= n) t = u;
    }
  }
  Found least = {(uint64_t)t << 32, 0};
  if (least.score == 0) least.score = 1;  // (0 is none)
  // what reaches T goes to LDS, a wavefront's at a time
  const auto collect = [&](uint64_t key, int row, Pick p) {
    const Found f = {key, rest_of(row, p)};
    const bool take = key != 0 && !least.before(f);
    const uint64_t b = __builtin_amdgcn_ballot_w64(take);
    if (b == 0) return;
    int at = 0;
    if (lane == __builtin_ctzll(b)) at = atomicAdd(&came, __builtin_popcountll(b));
    at = __shfl(at, __builtin_ctzll(b)) + __builtin_amdgcn_mbcnt_hi((uint32_t)(b >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)b, 0));
    if (take && at < BEAM_CAP) found[at] = f;
  };
  int total = 0;
  while (true) {
#pragma unroll
    for (int j = 0; j < BEAM_OWN; ++j)
      if (j * BEAM_THREADS < entries) collect(own_key[j], own_list[j] / n_chunks, own[j]);
    for (int at = BEAM_OWN * BEAM_THREADS; at < entries; at += BEAM_THREADS) {
      const int i = at + tid, list = min(i, entries - 1) / n;
      const bool look = i < entries && heads[list * k] >= (uint32_t)(least.score >> 32);
      const Pick p = look ? gt[i] : 0;
      collect(look ? score_of(list / n_chunks, p) : 0, list / n_chunks, p);
    }
    __syncthreads();
    total = came;
    if (total <= BEAM_CAP) break;
    // the n-th of those that came is the new bound
    for (int i = tid; i < BEAM_CAP; i += BEAM_THREADS) {
      const Found f = found[i];
      int rank = 0;
      for (int j = 0; j < BEAM_CAP; ++j) rank += found[j].before(f) ? 1 : 0;
      if (rank == n - 1) bound = f;
    }
    __syncthreads();
    least = bound;
    if (tid == 0) came = 0;
    __syncthreads();
  }
  const int64_t out0 = (int64_t)g * n;
  for (int i = tid; i < total; i += BEAM_THREADS) {
    const Found f = found[i];
    int rank = 0;
    for (int j = 0; j < total; ++j) rank += found[j].before(f) ? 1 : 0;
    if (rank >= n) continue;
    a.row_out[out0 + rank] = r0 + BEAM_MAX_ROWS - 1 - (int)(f.rest >> (32 + BEAM_ID_BITS));
    a.token_out[out0 + rank] = (1 << BEAM_ID_BITS) - 1 - (int)(f.rest & ((1 << BEAM_ID_BITS) - 1));
    a.score_out[out0 + rank] = (float)from_ordered64(f.score);
  }
  for (int i = total + tid; i < n; i += BEAM_THREADS) {
    a.row_out[out0 + i] = a.token_out[out0 + i] = -1;
    a.score_out[out0 + i] = -INFINITY;
  }
}

int64_t beam_workspace_bytes(int32_t rows, int64_t vocab, int32_t dtype, int32_t n_out) {
  return logprobs_workspace_bytes(rows, vocab, dtype, n_out);
}

hipError_t launch_beam_select(const BeamArgs& a, void* workspace, hipStream_t stream) {
  if (a.n_groups <= 0) return hipSuccess;
  const Cut cut = cut_rows(a.rows, a.vocab, a.dtype);
  Part* parts = (Part*)workspace;
  Pick* tops = (Pick*)((char*)workspace + parts_bytes(a.rows, cut));
  if ((int64_t)BEAM_MAX_ROWS * cut.n_chunks > BEAM_MAX_LISTS && (int64_t)a.rows * cut.n_chunks > BEAM_MAX_LISTS) return hipErrorInvalidValue;
  if (a.rows > 0) {
    LogprobArgs l{};
    l.logits = a.logits;
    l.dtype = a.dtype;
    l.rows = a.rows;
    l.vocab = a.vocab;
    l.row_stride = a.row_stride;
    l.scale = (float)a.scale;
    l.n_top = a.n_out;
    const hipError_t e = launch_logprob_chunks(l, cut, parts, tops, stream);
    if (e != hipSuccess) return e;
  }
  beam_select_kernel<<<dim3((unsigned)a.n_groups), BEAM_THREADS, 0, stream>>>(a, cut.n_chunks, parts, tops);
  return hipGetLastError();
}

}  // namespace dk
