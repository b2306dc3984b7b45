// The best continuations of each request's beams (gfx950): of every row r of a group and every token t
//
//   score(r, t) = scores[r] + scale x_rt - ln sum_u exp(scale x_ru),
//
// the n largest.
//
//   beam_chunk_kernel    one workgroup per (row, chunk): the logits are read once, 16 bytes a lane and UNROLL of them in flight.  It
//                        leaves the chunk's largest logit, its sum of exponentials against that, and a list of the lanes that may hold
//                        one of the chunk's n best, each with the largest of its logits: those that reach T, which n lanes of a
//                        wavefront reach, or n / 4 of every one (found bit by bit with ballots, as in token_logprobs_chunk_kernel).
//   beam_select_kernel   one workgroup per group: folds the sums of its rows, finds T -- the n-th largest score of the wavefronts' (or
//                        chunks', or lanes') largest logits, by how far it is from the best one of all: as many continuations are T or more, so the n best are --
//                        and reads the logits of the lanes that reach it once more, some n of them.  What reaches T there goes to LDS, and
//                        each one's place is the number of those before it.  Where more do than there is room for (equal logits by the
//                        thousand), T is raised to the n-th of those that came and the lists are gone through again.
// Scores are made and compared in fp64: rows of one group differ by the logs of sums of 10^5 terms, and two continuations may be close.
//
// Measured (kernel times): 64 groups of eight rows of 128 256 bf16 logits, n = 16: chunks 24.6 us (131 MB, 5.3 TB/s; some 450 vector
// instructions a wavefront keep the SIMDs busy three fifths of that, six wavefronts to a SIMD instead of five give 2 %), groups 12.3; with
// lists of the n best logits themselves, put in order, the chunks took 36.  One group of four such rows, n = 8: 3.5 and 10.2; 40 groups
// of up to ten rows of 50 003 fp32 logits, a third of them nearly all -infinity: 10.6 and 12.2.  The groups' kernel is a chain of round trips and of
// exchanges over LDS: load 1.1 us, sums 1.2 to 1.7, T 1.3, lists 1.8 to 2.6, logits 2 to 4, places 0.5 to 1; of 256 lanes instead
// of 512 it takes 10.3, 14.7 and 14.0, of 1024 10.8, 14.5 and 13.2.
#include <hip/hip_runtime.h>

#include "logprob_parts.hpp"

namespace dk {

namespace {

constexpr int BEAM_THREADS = 512;
constexpr int BEAM_ID_BITS = 20;
static_assert(BEAM_MAX_VOCAB <= 1 << BEAM_ID_BITS && BEAM_MAX_ROWS <= 1 << (64 - 32 - BEAM_ID_BITS), "row, logit and token in 64 bits");
constexpr int BEAM_MAX_LISTS = BEAM_MAX_ROWS * (int)((BEAM_MAX_VOCAB + LP_THREADS * LP_UNROLL * 4 - 1) / (LP_THREADS * LP_UNROLL * 4));
static_assert(BEAM_MAX_LISTS >= 1024, "calls of few rows have fewer than 4 x 256 chunks");
constexpr int BEAM_CAP = 1024;   // continuations that reach T
constexpr int BEAM_LANES = 1024;  // lanes that reach it, at a time
constexpr int BEAM_LISTS = BEAM_THREADS;  // lists that do, at a time
static_assert(BEAM_LANES >= LP_THREADS, "a list's");
constexpr int BEAM_LIST = LP_THREADS, BEAM_STEP = 64;  // a list: entries in any order, 0 behind the last up to the next multiple of BEAM_STEP
constexpr int BEAM_ROUNDS = 8;    // entries that a thread asks for at a time
constexpr int BEAM_ROW_SUMS = 16;

// What a chunk says of its row.
struct BeamPart {
  float m, s;     // largest logit, sum 2^(scale log2(e) (x - m))
  int32_t entries, pad;  // of its list
  float top[LP_WAVES];  // largest logits of its wavefronts
};
// A lane and the largest of its logits.  0: none.
typedef uint64_t Entry;

// Of a logit, in log2 units.  Rounded once: its error moves every term of a row's sum the same way, ln sum by up to as many times 2^-24 as
// the mean term is nats below the largest.
__device__ __forceinline__ float beam_factor(const BeamArgs& a) { return (float)(a.scale * 1.4426950408889634); }

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
__device__ __forceinline__ uint64_t rest_of(int row, float x, int id) {
  return (uint64_t)(BEAM_MAX_ROWS - 1 - row) << (32 + BEAM_ID_BITS) | (uint64_t)ordered(x) << BEAM_ID_BITS | (uint64_t)((1 << BEAM_ID_BITS) - 1 - id);
}

template <typename T>
__device__ __forceinline__ float element_of(const uint4& v, int j) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  if constexpr (sizeof(T) == 4) return __uint_as_float(w[j]);
  else return __uint_as_float(j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
}

}  // namespace

namespace {

// Over all lanes: quads, eights and sixteens by data-parallel moves, rows of sixteen and halves by swaps.  (By shuffles through LDS,
// six round trips of it each, and 16 steps for the thresholds, the chunks of 64 x 8 rows took 25.4 us instead of 24.6.)
template <int CTRL>
__device__ __forceinline__ float dpp_move(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
template <typename OP>
__device__ __forceinline__ float over_lanes(float x, OP op) {
  x = op(x, dpp_move<0xB1>(x));   // lanes 1, 0, 3, 2 of a quad
  x = op(x, dpp_move<0x4E>(x));   // lanes 2, 3, 0, 1
  x = op(x, dpp_move<0x141>(x));  // the other quad of eight lanes
  x = op(x, dpp_move<0x140>(x));  // the other eight of a row
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return op(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// nth_and_kth_largest, in fewer steps where the n largest are within two powers of two of the largest of all, `top` (uniform).
template <int BITS>
__device__ __forceinline__ float2 nth_and_kth_from(float x, float top, int n, int k) {
  const uint32_t key = ordered(x), from = ordered(top) >> 24 << 24;
  uint32_t tn = 0, tk = 0;
  const auto search = [&](int high) __attribute__((always_inline)) {
#pragma unroll
    for (int bit = high; bit >= 32 - BITS; --bit) {
      const uint32_t un = tn | (1u << bit), uk = tk | (1u << bit);
      if (__builtin_popcountll(__builtin_amdgcn_ballot_w64(key >= un)) >= n) tn = un;
      if (__builtin_popcountll(__builtin_amdgcn_ballot_w64(key >= uk)) >= k) tk = uk;
    }
  };
  if (__builtin_popcountll(__builtin_amdgcn_ballot_w64(key >= from)) >= max(n, k)) {
    tn = tk = (uint32_t)__builtin_amdgcn_readfirstlane((int)from);
    search(23);
  } else {
    search(31);
  }
  return make_float2(from_ordered(max(tn, 0x007fffffu)), from_ordered(max(tk, 0x007fffffu)));
}

}  // namespace

// A chunk is LP_THREADS * UNROLL * VEC logits; element VEC u + j of a thread is id base + (u LP_THREADS + thread) VEC + j.
template <typename T, int UNROLL, bool ONCE>
__global__ __launch_bounds__(LP_THREADS) void beam_chunk_kernel(BeamArgs a, int32_t n_chunks, BeamPart* __restrict__ parts,
                                                                Entry* __restrict__ lists) {
  constexpr int VEC = 16 / (int)sizeof(T), N = UNROLL * VEC;
  __shared__ float4 wave_part[LP_WAVES];  // largest logit, sum, the two thresholds
  __shared__ int32_t came;
  const int32_t row = blockIdx.x / n_chunks, chunk = blockIdx.x - row * n_chunks;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const T* p = (const T*)a.logits + (int64_t)row * a.row_stride;
  const int32_t vocab = (int32_t)a.vocab;
  const int32_t base = chunk * (LP_THREADS * N) + (int32_t)threadIdx.x * VEC;
  typedef uint32_t words __attribute__((ext_vector_type(4)));
  words raw[UNROLL];  // (whole: the last of a row may hold what is behind it, up to the stride)
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    const int32_t e0 = min(base + u * (LP_THREADS * VEC), (vocab - 1) / VEC * VEC);
    raw[u] = ONCE ? __builtin_nontemporal_load((const words*)(p + e0)) : *(const words*)(p + e0);
  }
  if (threadIdx.x == 0) came = 0;
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
      if (base + (e / VEC) * (LP_THREADS * VEC) + e % VEC >= vocab) x[e] = -INFINITY;
  }
  float mine = x[0];
#pragma unroll
  for (int e = 0; e < N; e += 2) asm("v_max3_f32 %0, %1, %2, %3" : "=v"(mine) : "v"(mine), "v"(x[e]), "v"(x[e + 1]));
  const float m = over_lanes(mine, [](float p, float q) { return fmaxf(p, q); });
  const float c = beam_factor(a), mr = m == -INFINITY ? 0.f : m, mc = mr * c;
  float s0 = 0.f, s1 = 0.f;
  // (eight at a time: an exponential's result may not be used by the very next instruction)
  const auto sums = [&](auto y) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < N; e += 8) {
      float w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = __builtin_amdgcn_exp2f(y(x[e + i]));
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        s0 += w[i];
        s1 += w[i + 1];
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  if (__builtin_fabsf(mc) <= 1048576.f) sums([&](float v) { return __builtin_fmaf(v, c, -mc); });
  else sums([&](float v) { return (v - mr) * c; });  // the difference first: it may be small against what is multiplied
  s0 = over_lanes(s0 + s1, [](float p, float q) { return p + q; });
  const float r = __builtin_fabsf(mc) <= 1048576.f ? __builtin_fmaf(mr, c, -mc) : 0.f;  // what rounding m c took off
  const float2 t = nth_and_kth_from<sizeof(T) == 2 ? 16 : 18>(mine, m, a.n_out, (a.n_out + LP_WAVES - 1) / LP_WAVES);
  if (lane == 0) wave_part[wave] = make_float4(m, s0 * __builtin_amdgcn_exp2f(-r), t.x, t.y);
  __syncthreads();
  float reach = wave_part[0].z, every = wave_part[0].w, top = wave_part[0].x;
#pragma unroll
  for (int w = 1; w < LP_WAVES; ++w) {
    reach = fmaxf(reach, wave_part[w].z);
    every = fminf(every, wave_part[w].w);
    top = fmaxf(top, wave_part[w].x);
  }
  reach = fmaxf(reach, every);
  const uint64_t b = __builtin_amdgcn_ballot_w64(mine >= reach && mine > -INFINITY);
  Entry* list = lists + (int64_t)blockIdx.x * BEAM_LIST;
  if (b != 0) {
    int at = 0;
    if (lane == 0) at = atomicAdd(&came, __builtin_popcountll(b));
    at = __builtin_amdgcn_readfirstlane(at) + __builtin_amdgcn_mbcnt_hi((uint32_t)(b >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)b, 0));
    if (b >> lane & 1) list[at] = (Entry)ordered(mine) << 32 | threadIdx.x;
  }
  __syncthreads();
  const int end = came, pad = end + (int)threadIdx.x;
  if (pad < min(BEAM_LIST, (end / BEAM_STEP + 1) * BEAM_STEP)) list[pad] = 0;
  if (threadIdx.x == 0) {
    BeamPart q{top, 0.f, end, 0, {}};
#pragma unroll
    for (int w = 0; w < LP_WAVES; ++w) {
      q.top[w] = wave_part[w].x;
      const float d = q.top[w] == top ? 0.f : (q.top[w] - top) * c;
      q.s += __builtin_amdgcn_exp2f(d) * wave_part[w].y;
    }
    parts[blockIdx.x] = q;
  }
}

template <typename T>
__global__ __launch_bounds__(BEAM_THREADS) void beam_select_kernel(BeamArgs a, int32_t n_chunks, int32_t unroll, const BeamPart* __restrict__ parts,
                                                                   const Entry* __restrict__ lists) {
  constexpr int VEC = 16 / (int)sizeof(T);
  __shared__ float2 sums[BEAM_MAX_ROWS * BEAM_ROW_SUMS];  // largest logit and sum of the rows' chunks, where they fit
  __shared__ uint32_t heads[BEAM_MAX_LISTS];
  __shared__ Found found[BEAM_CAP];
  __shared__ uint32_t lanes[BEAM_LANES];  // list * 256 + thread
  __shared__ uint32_t lane_key[BEAM_LANES];  // the largest logit's there, see key_of
  __shared__ double base[BEAM_MAX_ROWS];  // of a row that takes part: its score less the log of its sum
  __shared__ float most[BEAM_MAX_ROWS];   // its largest logit; NaN: it takes no part
  __shared__ int32_t lists_on[BEAM_LISTS];
  __shared__ int32_t came, reached, active;
  __shared__ uint32_t top_bits;  // upper bits of the best row's best score
  __shared__ Found bound;
  const int g = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int n = a.n_out;
  const int r0 = min(max(a.cu_rows[g], 0), a.rows);
  const int rows = min(min(max(a.cu_rows[g + 1], r0), a.rows) - r0, BEAM_MAX_ROWS);
  const int n_lists = rows * n_chunks;
  const BeamPart* gp = parts + (int64_t)r0 * n_chunks;
  const Entry* gl = lists + (int64_t)r0 * n_chunks * BEAM_LIST;

  constexpr int PER_ROUND = BEAM_THREADS / BEAM_STEP;  // lists
  const int sub = tid % BEAM_STEP;
  // T comes from one value of each list, of each wavefront of a list, or from the first entries of few lists
  const int kind = n_lists >= 4 * n ? 1 : LP_WAVES * n_lists >= n ? LP_WAVES : 0;
  const float own_score = tid < rows ? a.scores[r0 + tid] : 0.f;
  const bool fits = n_chunks <= BEAM_ROW_SUMS;
  if (fits) {
    for (int i = tid; i < n_lists; i += BEAM_THREADS) sums[i] = make_float2(gp[i].m, gp[i].s);
  }
  if (kind != 0) {
    for (int i = tid; i < n_lists * kind; i += BEAM_THREADS) heads[i] = __float_as_uint(kind == 1 ? gp[i].m : gp[i / LP_WAVES].top[i % LP_WAVES]);
  }
  if (tid < rows) most[tid] = own_score;
  if (tid == 0) came = reached = 0, top_bits = 0;
  __syncthreads();

  // the rows' sums, `per` lanes to a row
  int per = 1;
  while (per < 64 && per < n_chunks) per *= 2;
  const float c = beam_factor(a);  // (chunks' weights in fp32, as their sums: 2^-22 of the row's sum at the most)
  for (int at = 0; at < rows; at += BEAM_THREADS / per) {
    const int r = at + tid / per, s = tid % per;
    const bool there = r < rows;
    const auto part = [&](int k) { return fits ? sums[r * n_chunks + k] : make_float2(gp[r * n_chunks + k].m, gp[r * n_chunks + k].s); };
    float m = -INFINITY;
    for (int k = s; there && k < n_chunks; k += per) m = fmaxf(m, part(k).x);
    for (int off = per / 2; off >= 1; off /= 2) m = fmaxf(m, __shfl_xor(m, off));
    double z = 0.0;
    for (int k = s; there && k < n_chunks; k += per) {
      const float2 q = part(k);  // (of a chunk of nothing but -infinity the sum is 0, of one with a NaN it is one)
      z += q.x == -INFINITY ? (double)q.y : (double)(q.y * __builtin_amdgcn_exp2f((q.x - m) * c));
    }
    for (int off = per / 2; off >= 1; off /= 2) z += __shfl_xor(z, off);
    if (there && s == 0) {
      const float score = most[r];
      const bool live = __builtin_fabsf(score) < INFINITY && __builtin_fabsf(m) < INFINITY && z > 0.0 && z < (double)INFINITY;
      base[r] = live ? (double)score - log(z) : 0.0;
      most[r] = live ? m : __uint_as_float(0x7fc00000u);
      if (live) atomicMax(&top_bits, (uint32_t)(ordered64(base[r]) >> 32));
    }
  }
  __syncthreads();
  // score of a logit, as a whole number; 0: none
  const auto score_of = [&](int row, float x) -> uint64_t {
    const float m = most[row];
    if (m != m || !(x > -INFINITY)) return 0;
    return ordered64(base[row] + ((double)x - (double)m) * a.scale);
  };
  const auto entry_score = [&](int list, Entry e) -> uint64_t {
    return e == 0 ? 0 : score_of(list / n_chunks, from_ordered((uint32_t)(e >> 32)));
  };

  // Bounds are found among keys: how far a score is below `top`, which none is above, as a float in order.  (A score by itself grows with
  // the length of what has been said: of its 17 upper bits the last is 8 near -300 and 128 near -5000: bounds made of those
  // let so much through that a call took 1382 us there instead of 22.)  0: none, also of a bound that everything reaches.
  const double top = from_ordered64((uint64_t)top_bits << 32 | 0xffffffffu);
  const auto key_of = [&](uint64_t score) -> uint32_t { return score == 0 ? 0u : ordered(fminf((float)(from_ordered64(score) - top), -0x1p-126f)); };
  // a score that none with such a key or a larger one is below (the difference was rounded to fp64 and to fp32)
  const auto score_at = [&](uint32_t key) -> uint64_t {
    if (key <= 0x007fffffu) return 1;  // (-infinity is the first)
    return ordered64(top + (double)from_ordered(key) * (1.0 + 0x1p-20) - __builtin_fabs(top) * 0x1p-50);
  };
  int n_heads = n_lists * kind;
  if (kind != 0) {
    for (int i = tid; i < n_heads; i += BEAM_THREADS) heads[i] = key_of(score_of(i / (kind * n_chunks), __uint_as_float(heads[i])));
  } else {  // (fewer than BEAM_MAX_OUT / LP_WAVES lists)
    n_heads = n_lists * BEAM_STEP;
    for (int i = tid; i < n_heads; i += BEAM_THREADS) heads[i] = key_of(entry_score(i / BEAM_STEP, gl[i / BEAM_STEP * BEAM_LIST + i % BEAM_STEP]));
  }
  __syncthreads();
  // The n-th largest of some keys in LDS but for the last bits (2^-8 of the distance from `top`), 0 if there are fewer; every wavefront finds
  // it by itself.
  const auto nth_largest = [&](const uint32_t* of, int count_of) __attribute__((always_inline)) {
    constexpr int KEEP = 16;  // of a lane (where they were read again for every bit, 672 took 7 to 11 us)
    uint32_t mine[KEEP], t = 0;
#pragma unroll
    for (int i = 0; i < KEEP; ++i) mine[i] = 0;
#pragma unroll
    for (int i0 = 0; i0 < KEEP; i0 += 4) {
      if (64 * i0 >= count_of) break;
#pragma unroll
      for (int i = i0; i < i0 + 4; ++i) mine[i] = lane + 64 * i < count_of ? of[lane + 64 * i] : 0u;
    }
    for (int bit = 30; bit >= 15; --bit) {  // (the keys of negative floats)
      const uint32_t u = t | 1u << bit;
      int count = __builtin_popcountll(__builtin_amdgcn_ballot_w64(mine[0] >= u));
      if (count_of > 64) {
#pragma unroll
        for (int i = 1; i < 4; ++i) count += __builtin_popcountll(__builtin_amdgcn_ballot_w64(mine[i] >= u));
#pragma unroll
        for (int i0 = 4; i0 < KEEP; i0 += 4) {
          if (64 * i0 >= count_of) break;
#pragma unroll
          for (int i = i0; i < i0 + 4; ++i) count += __builtin_popcountll(__builtin_amdgcn_ballot_w64(mine[i] >= u));
        }
        for (int i = 64 * KEEP; i < count_of; i += 64) count += __builtin_popcountll(__builtin_amdgcn_ballot_w64(i + lane < count_of && of[i + lane] >= u));
      }
      if (count >= n) t = u;
    }
    return t;
  };
  Found least = {score_at(nth_largest(heads, n_heads)), 0};

  // places in LDS for those lanes of a wavefront that say so
  const auto places = [&](bool take, int32_t* counter) __attribute__((always_inline)) {
    const uint64_t b = __builtin_amdgcn_ballot_w64(take);
    if (b == 0) return 0;
    int at = 0;
    if (lane == 0) at = atomicAdd(counter, __builtin_popcountll(b));
    return __builtin_amdgcn_readfirstlane(at) + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(b >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)b, 0));
  };
  // reads the logits of the lanes that reach T
  const auto expand = [&]() __attribute__((always_inline)) {
    const int items = reached * unroll;
    for (int i0 = 0; i0 < items; i0 += BEAM_THREADS) {
      const int i = i0 + tid;
      const bool there = i < items;
      const uint32_t which = lanes[there ? i / unroll : 0];
      const int list = (int)(which / BEAM_LIST), row = list / n_chunks, chunk = list - row * n_chunks;
      const int id0 = (chunk * unroll + i % unroll) * (LP_THREADS * VEC) + (int)(which % BEAM_LIST) * VEC;
      uint4 v = make_uint4(0, 0, 0, 0);
      const bool in = there && id0 < (int)a.vocab;
      if (in) v = *(const uint4*)((const T*)a.logits + (int64_t)(r0 + row) * a.row_stride + id0);
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float x = element_of<T>(v, j);
        Found f = {in && id0 + j < (int)a.vocab ? score_of(row, x) : 0, 0};
        if (__builtin_amdgcn_ballot_w64(f.score >= least.score) == 0) continue;
        f.rest = rest_of(row, x, id0 + j);
        const bool take = f.score != 0 && !least.before(f);
        const int at = places(take, &came);
        if (take && at < BEAM_CAP) found[at] = f;
      }
    }
  };
  int total = 0;
  while (true) {
    // the lists whose largest logit reaches T, BEAM_LISTS of them at a time, a wavefront to a list
    for (int l0 = 0; l0 < n_lists; l0 += BEAM_LISTS) {
      if (tid == 0) active = 0;
      __syncthreads();
      const int list = l0 + tid;
      uint32_t head = 0;
      if (list < n_lists) {
        if (kind == 0) head = ~0u;
        else
          for (int w = 0; w < kind; ++w) head = max(head, heads[list * kind + w]);
      }
      const bool take = list < n_lists && head >= (least.score <= 1 ? 1u : key_of(least.score));
      const int at = places(take, &active);
      if (take) lists_on[at] = list;
      __syncthreads();
      const int n_active = active;
      for (int a0 = 0; a0 < n_active; a0 += PER_ROUND * BEAM_ROUNDS) {
        Entry q[BEAM_ROUNDS];
        int from[BEAM_ROUNDS];
#pragma unroll
        for (int j = 0; j < BEAM_ROUNDS; ++j) {
          const int k = a0 + j * PER_ROUND + tid / BEAM_STEP;
          from[j] = k < n_active ? lists_on[k] : -1;
          q[j] = k < n_active ? gl[(int64_t)from[j] * BEAM_LIST + sub] : 0;
        }
#pragma unroll
        for (int j = 0; j < BEAM_ROUNDS; ++j) {
          if (a0 + j * PER_ROUND >= n_active) continue;
          for (int e = sub;;) {
            // (a lane's largest logit: of equal scores any may come before the bound)
            const uint64_t key = q[j] != 0 ? entry_score(from[j], q[j]) : 0;
            const bool reaches = key >= least.score;
            const int to = places(reaches, &reached);
            if (reaches && to < BEAM_LANES) {
              lanes[to] = (uint32_t)(from[j] * BEAM_LIST) | (uint32_t)(q[j] & 0xffu);
              lane_key[to] = key_of(key);
            }
            // a list goes on where this step of it was full
            const bool more = __shfl((unsigned long long)q[j], lane | (BEAM_STEP - 1)) != 0 && e + BEAM_STEP < BEAM_LIST;
            if (__builtin_amdgcn_ballot_w64(more) == 0) break;
            e += BEAM_STEP;
            q[j] = more ? gl[(int64_t)from[j] * BEAM_LIST + e] : 0;
          }
        }
      }
      __syncthreads();
    }
    const int n_reached = reached;
    __syncthreads();
    if (n_reached <= BEAM_LANES) {
      // T by what they say themselves
      const auto raise = [&]() __attribute__((always_inline)) {
        const uint32_t higher = nth_largest(lane_key, n_reached);
        uint32_t which[BEAM_LANES / BEAM_THREADS];
        bool keep[BEAM_LANES / BEAM_THREADS];
#pragma unroll
        for (int i = 0; i < BEAM_LANES / BEAM_THREADS; ++i) {
          const int k = i * BEAM_THREADS + tid;
          keep[i] = k < n_reached && lane_key[k] >= higher;
          which[i] = keep[i] ? lanes[k] : 0;
        }
        if (score_at(higher) > least.score) least = {score_at(higher), 0};
        if (tid == 0) came = reached = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < BEAM_LANES / BEAM_THREADS; ++i) {
          const int to = places(keep[i], &reached);
          if (keep[i]) lanes[to] = which[i];
        }
        __syncthreads();
      };
      // At once where there is no T yet (few lists hold anything: a request's first step), or where they are many -- one row leads, and T came from
      // other rows' lists; 1.7 us, a round of `expand` takes 2.6.  Else where so much reached the T there is that the places would take
      // longer (without the second look one row of 6548 logits and 32 continuations took 70 us).
      const bool early = n_reached > n && (least.score <= 1 || n_reached * unroll > BEAM_THREADS);
      if (early) raise();
      expand();
      __syncthreads();
      const bool late = !early && n_reached > n && came > BEAM_CAP / 2;
      __syncthreads();
      if (late) {
        raise();
        expand();
      }
    } else {
      // more lanes than there is room for: T from those that came, and the lists again; if that is no higher, list by list (equal logits by the
      // thousand where the n-th best is one of them: four rows of 30 000 take 0.29 ms, eight of 128 256 1.74)
      const uint64_t higher = score_at(nth_largest(lane_key, BEAM_LANES));
      if (higher > least.score) {
        least = {higher, 0};
        __syncthreads();
        if (tid == 0) reached = 0;
        __syncthreads();
        continue;
      }
      for (int list = 0; list < n_lists; ++list) {
        __syncthreads();
        if (tid == 0) reached = 0;
        __syncthreads();
        const Entry q = tid < gp[list].entries ? gl[(int64_t)list * BEAM_LIST + tid] : 0;
        const bool reaches = q != 0 && entry_score(list, q) >= least.score;
        const int to = places(reaches, &reached);
        if (reaches) lanes[to] = (uint32_t)(list * BEAM_LIST) | (uint32_t)(q & 0xffu);
        __syncthreads();
        expand();
      }
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
    if (tid == 0) came = reached = 0;
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

namespace {

int64_t beam_parts_bytes(int32_t rows, const Cut& cut) { return ((int64_t)rows * cut.n_chunks * (int64_t)sizeof(BeamPart) + 255) / 256 * 256; }

template <typename T, int UNROLL>
void launch_beam(const BeamArgs& a, const Cut& cut, BeamPart* parts, Entry* lists, hipStream_t stream) {
  const bool once = (int64_t)a.rows * a.vocab * (int64_t)sizeof(T) >= (int64_t)64 << 20;  // (as in verify.hip)
  const dim3 grid((unsigned)a.rows * (unsigned)cut.n_chunks);
  if (a.rows > 0) {
    if (once) beam_chunk_kernel<T, UNROLL, true><<<grid, LP_THREADS, 0, stream>>>(a, cut.n_chunks, parts, lists);
    else beam_chunk_kernel<T, UNROLL, false><<<grid, LP_THREADS, 0, stream>>>(a, cut.n_chunks, parts, lists);
  }
  beam_select_kernel<T><<<dim3((unsigned)a.n_groups), BEAM_THREADS, 0, stream>>>(a, cut.n_chunks, UNROLL, parts, lists);
}

}  // namespace

int64_t beam_workspace_bytes(int32_t rows, int64_t vocab, int32_t dtype, int32_t) {
  const Cut cut = cut_rows(rows, vocab, dtype);
  return beam_parts_bytes(rows, cut) + (int64_t)rows * cut.n_chunks * BEAM_LIST * (int64_t)sizeof(Entry) + 256;
}

hipError_t launch_beam_select(const BeamArgs& a, void* workspace, hipStream_t stream) {
  if (a.n_groups <= 0) return hipSuccess;
  const Cut cut = cut_rows(a.rows, a.vocab, a.dtype);
  const int64_t most = a.rows < BEAM_MAX_ROWS ? a.rows : BEAM_MAX_ROWS;  // rows of a group
  if (most * cut.n_chunks > BEAM_MAX_LISTS || (int64_t)a.rows * cut.n_chunks >= (int64_t(1) << 32) / LP_THREADS) return hipErrorInvalidValue;
  BeamPart* parts = (BeamPart*)workspace;
  Entry* lists = (Entry*)((char*)workspace + beam_parts_bytes(a.rows, cut));
  const bool wide = cut.unroll == LP_UNROLL;
  if (a.dtype == 1) wide ? launch_beam<uint16_t, LP_UNROLL>(a, cut, parts, lists, stream) : launch_beam<uint16_t, LP_UNROLL_FEW>(a, cut, parts, lists, stream);
  else wide ? launch_beam<float, LP_UNROLL>(a, cut, parts, lists, stream) : launch_beam<float, LP_UNROLL_FEW>(a, cut, parts, lists, stream);
  return hipGetLastError();
}

}  // namespace dk
