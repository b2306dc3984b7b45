// Norms of queries and keys for each head and their rotation by position, into rows or into the pool's cells (gfx950).
//
//   y = x / sqrt(mean x^2 + eps) w;  pair i of the rotated part turns by position * inv_freq[i].
//
// A lane holds eight elements of a head: where the pairs lie in two halves of whole fours, four of the first half and the four that
// they turn with, so that nothing is exchanged; where neighbours turn, eight in a row.  A head of 128 takes 16 lanes, one of 64
// eight; its mean square is summed over them.  Every lane group has a token, works out its lanes' eight angles once and walks the
// token's heads, HEADS of them per workgroup, several requested at a time.  Angles are products in fp64, reduced to a part of a turn
// there: a position of 2^30 times a frequency leaves 2^-23 turns in fp64 and nothing in fp32.
// Bound by HBM: every element is read once and written once; an append of 8192 tokens of 32 + 2 x 8 heads of 128 in bf16, 201 MB,
// takes 35.2 us, 5.7 TB/s, where the Infinity Cache has the rows and 48.6 us, 4.1 TB/s, where it has not (a copy of 2 GiB on the same
// card 4.9 TB/s; one wavefront per head, as it was first, 178 us).  Loads past the caches 41.9 and 47.6, stores past them 35.1 and 46.3:
// the rows come from the projection just before and go to the attention just behind, so both go through the caches.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "kernels.hpp"

namespace dk {

namespace {

constexpr int ROT_THREADS = 256;
constexpr int ROT_AHEAD = 2;  // heads of a lane requested at a time

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Four elements as they lie in memory, and as floats.
template <typename T> struct Four;
template <> struct Four<float> {
  typedef f32x4 Raw;
  static __device__ __forceinline__ f32x4 widen(Raw r) { return r; }
  static __device__ __forceinline__ Raw narrow(f32x4 x) { return x; }
};
template <> struct Four<__bf16> {
  typedef u32x2 Raw;
  static __device__ __forceinline__ f32x4 widen(Raw r) {
    return f32x4{__uint_as_float(r[0] << 16), __uint_as_float(r[0] & 0xffff0000u), __uint_as_float(r[1] << 16), __uint_as_float(r[1] & 0xffff0000u)};
  }
  static __device__ __forceinline__ Raw narrow(f32x4 x) {
    typedef __bf16 quad __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(Raw, quad{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]});
  }
};

// How a head is laid over its lanes.  HALVES: quad a of lane i and quad b are elements that turn with one another (or two quads of
// the rest of the head); PAIRS: quads a and b follow each other; MIXED: halves of no whole fours, quads as in PAIRS and the
// partners through LDS.
enum Layout { HALVES, PAIRS, MIXED };

// Element of quad a and b of a head's lane.
template <int D, Layout L>
__device__ __forceinline__ void quads_of(int lane, int rotary_dim, int* a, int* b) {
  if constexpr (L == HALVES) {
    const int half = rotary_dim >> 1;  // whole fours
    *a = 4 * lane;
    if (4 * lane < half) {
      *b = 4 * lane + half;
    } else {  // the rest: quads of elements from rotary_dim on, in order
      const int k = 2 * (lane - half / 4);
      *a = rotary_dim + 4 * k;
      *b = rotary_dim + 4 * k + 4;
    }
  } else {
    *a = 8 * lane;
    *b = 8 * lane + 4;
  }
}

struct Turn {  // cosine and sine, times the amplitude, of a lane's pairs: HALVES and PAIRS four, MIXED one for each element
  float c[8], s[8];
};
__device__ __forceinline__ void angle(const RotaryArgs& a, int64_t pos, int pair, float* c, float* s) {
  const double turns = (double)pos * (double)a.inv_freq[pair] * 0.15915494309189535;
  sincospif((float)(2.0 * (turns - rint(turns))), s, c);
  *c *= a.amplitude;
  *s *= a.amplitude;
}
template <int D, Layout L>
__device__ __forceinline__ Turn turn_of(const RotaryArgs& a, int lane, int64_t pos) {
  Turn t{};
  const int half = a.rotary_dim >> 1;
  if constexpr (L == MIXED) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = 8 * lane + j;
      if (e >= a.rotary_dim) continue;
      angle(a, pos, e < half ? e : e - half, &t.c[j], &t.s[j]);
      if (e < half) t.s[j] = -t.s[j];  // the first of a pair takes the other's sine off
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int pair = 4 * lane + j;  // HALVES: elements pair and pair + half; PAIRS: elements 2 pair and 2 pair + 1
      if (pair < half) angle(a, pos, pair, &t.c[j], &t.s[j]);
    }
  }
  return t;
}

// (What is not turned stays as it is, whatever its neighbours hold.)
template <int D, Layout L>
__device__ __forceinline__ void turn(const RotaryArgs& args, const Turn& t, int lane, float* row, f32x4& a, f32x4& b) {
  const int half = args.rotary_dim >> 1;
  if constexpr (L == HALVES) {
    if (4 * lane >= half) return;
    const f32x4 x = a, y = b;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      a[j] = x[j] * t.c[j] - y[j] * t.s[j];
      b[j] = y[j] * t.c[j] + x[j] * t.s[j];
    }
  } else if constexpr (L == PAIRS) {
    const f32x4 x = a, y = b;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if (4 * lane + j < half) {
        a[2 * j] = x[2 * j] * t.c[j] - x[2 * j + 1] * t.s[j];
        a[2 * j + 1] = x[2 * j + 1] * t.c[j] + x[2 * j] * t.s[j];
      }
      if (4 * lane + 2 + j < half) {
        b[2 * j] = y[2 * j] * t.c[2 + j] - y[2 * j + 1] * t.s[2 + j];
        b[2 * j + 1] = y[2 * j + 1] * t.c[2 + j] + y[2 * j] * t.s[2 + j];
      }
    }
  } else {
    // (the lanes of a head are in one wavefront, whose LDS operations are in order)
    *(f32x4*)(row + 8 * lane) = a;
    *(f32x4*)(row + 8 * lane + 4) = b;
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = 8 * lane + j;
      if (e >= args.rotary_dim) continue;
      const float other = row[e < half ? e + half : e - half];
      if (j < 4) a[j & 3] = a[j & 3] * t.c[j] + other * t.s[j];
      else b[j & 3] = b[j & 3] * t.c[j] + other * t.s[j];
    }
    __builtin_amdgcn_wave_barrier();
  }
}

typedef const __attribute__((address_space(4))) RotaryRuns* const_runs_ptr;

enum Source { RUNS, TABLE, ROWS };  // where a token's position and cell come from

// Workgroup (token group, head group): ROT_THREADS / (D / 8) tokens, `heads_per` heads of each.  Heads are counted through: Q, K,
// and for appends V.
template <typename T, int D, Layout L, Source S>
__global__ __launch_bounds__(ROT_THREADS) void rotate_kernel(RotaryRuns runs, int32_t n_runs, const void* where, int64_t tok_base, int64_t n_tok,
                                                             RotaryArgs a, int32_t heads_per) {
  typedef Four<T> F;
  constexpr int LANES = D / 8, TOKENS = ROT_THREADS / LANES;
  __shared__ float rows[L == MIXED ? TOKENS * D : 1];
  (void)runs;
  const int lane = threadIdx.x % LANES, slot = threadIdx.x / LANES;
  const int64_t first = (int64_t)blockIdx.x * TOKENS;
  const int64_t i = min(first + slot, n_tok - 1);  // (groups past the end do the last token's work and store nothing)
  const bool live = first + slot < n_tok;
  const int64_t t = tok_base + i;
  const int n_heads = a.n_q_heads + (S == ROWS ? 1 : 2) * a.n_k_heads;
  const int h0 = blockIdx.y * heads_per, h1 = min(n_heads, h0 + heads_per);
  int ea, eb;
  quads_of<D, L>(lane, a.rotary_dim, &ea, &eb);

  const T* src_q = (const T*)a.q + t * a.q_stride;
  const T* src_k = (const T*)a.k + t * a.k_stride;
  const T* src_v = (const T*)a.v + t * a.v_stride;
  const auto source = [&](int h) {
    if (h < a.n_q_heads) return src_q + h * D;
    if (h < a.n_q_heads + a.n_k_heads) return src_k + (h - a.n_q_heads) * D;
    return src_v + (h - a.n_q_heads - a.n_k_heads) * D;
  };
  typename F::Raw ra[ROT_AHEAD], rb[ROT_AHEAD];
  const auto request = [&](int h) {
#pragma unroll
    for (int k = 0; k < ROT_AHEAD; ++k) {
      const T* p = source(min(h + k, h1 - 1));
      ra[k] = *(const typename F::Raw*)(p + ea);
      rb[k] = *(const typename F::Raw*)(p + eb);
    }
  };
  request(h0);

  int64_t pos, cell = 0;
  if constexpr (S == RUNS) {
    // (`runs` starts the kernel-argument segment and is read through it: an index of a lane's own would make a private copy of it)
    const_runs_ptr table = (const_runs_ptr)__builtin_amdgcn_kernarg_segment_ptr();
    const int32_t f = (int32_t)first;
    int32_t lo = 0, hi = n_runs - 1;  // the last run that starts at or before the workgroup's first token, by scalar loads
    while (lo < hi) {
      const int32_t mid = (lo + hi + 1) >> 1;
      if (table->tok[mid] <= f) lo = mid; else hi = mid - 1;
    }
    int32_t r = lo;
    while ((int32_t)i >= table->tok[r + 1]) ++r;
    const int32_t d = (int32_t)i - table->tok[r];
    pos = table->pos[r] + d;
    cell = table->cell[r] + d;
  } else if constexpr (S == TABLE) {
    pos = ((const int32_t*)where)[2 * i];
    cell = ((const int32_t*)where)[2 * i + 1];
  } else {
    pos = ((const int64_t*)where)[t];
  }
  const Turn turns = turn_of<D, L>(a, lane, pos);
  f32x4 wa[2], wb[2];  // norm weights of Q, of K
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    wa[k] = wb[k] = f32x4{1.f, 1.f, 1.f, 1.f};
    const T* w = (const T*)(k ? a.k_weight : a.q_weight);
    if (a.norm && w) {
      wa[k] = F::widen(*(const typename F::Raw*)(w + ea));
      wb[k] = F::widen(*(const typename F::Raw*)(w + eb));
    }
  }

  for (int h = h0; h < h1; h += ROT_AHEAD) {
    typename F::Raw xa[ROT_AHEAD], xb[ROT_AHEAD];
#pragma unroll
    for (int k = 0; k < ROT_AHEAD; ++k) {
      xa[k] = ra[k];
      xb[k] = rb[k];
    }
    if (h + ROT_AHEAD < h1) request(h + ROT_AHEAD);
#pragma unroll
    for (int k = 0; k < ROT_AHEAD; ++k) {
      const int head = h + k;
      if (head >= h1) continue;
      const bool is_q = head < a.n_q_heads, is_v = head >= a.n_q_heads + a.n_k_heads;
      if (!is_v) {
        f32x4 ya = F::widen(xa[k]), yb = F::widen(xb[k]);
        if (a.norm) {
          float sum = 0.f;
#pragma unroll
          for (int j = 0; j < 4; ++j) sum += ya[j] * ya[j] + yb[j] * yb[j];
#pragma unroll
          for (int off = LANES / 2; off >= 1; off >>= 1) sum += __shfl_xor(sum, off);
          const float inv = 1.f / sqrtf(sum * (1.f / D) + a.eps);
          ya *= inv * (is_q ? wa[0] : wa[1]);
          yb *= inv * (is_q ? wb[0] : wb[1]);
        }
        turn<D, L>(a, turns, lane, L == MIXED ? rows + slot * D : nullptr, ya, yb);
        xa[k] = F::narrow(ya);
        xb[k] = F::narrow(yb);
      }
      if (!live) continue;
      T* dst;
      if (is_q) dst = (T*)a.q_out + (t * a.n_q_heads + head) * D;
      else if (S == ROWS) dst = (T*)a.k_out + (t * a.n_k_heads + head - a.n_q_heads) * D;
      else dst = (T*)(is_v ? a.v_out : a.k_out) + ((head - a.n_q_heads - (is_v ? a.n_k_heads : 0)) * a.arena_cells + cell) * D;
      *(typename F::Raw*)(dst + ea) = xa[k];
      *(typename F::Raw*)(dst + eb) = xb[k];
    }
  }
}

template <typename T, int D, Layout L, Source S>
hipError_t launch_layout(const RotaryArgs& a, const RotaryRuns& runs, int32_t n_runs, const void* where, int64_t tok_base, int64_t n_tok,
                         hipStream_t stream) {
  constexpr int TOKENS = ROT_THREADS / (D / 8);
  const int n_heads = a.n_q_heads + (S == ROWS ? 1 : 2) * a.n_k_heads;
  const int64_t groups = (n_tok + TOKENS - 1) / TOKENS;
  // Heads of a workgroup: as many as leave eight workgroups to a compute unit.  8192 tokens of 48 heads, bf16, us a call (two heads
  // requested at a time / four): 1024 workgroups - / 36.9, 2048 35.2 / 35.3, 4096 35.1 / 36.0.
  int64_t per = std::max<int64_t>(ROT_AHEAD, groups * n_heads / 2048);
  per = std::min<int64_t>((per + ROT_AHEAD - 1) / ROT_AHEAD * ROT_AHEAD, n_heads);
  const int64_t y = (n_heads + per - 1) / per;
  if (y > 65535) return hipErrorInvalidValue;
  constexpr int64_t MOST = int64_t(1) << 22;  // workgroups of a launch along the tokens
  static_assert(MOST * TOKENS >= ROTARY_MAX_APPEND, "appends, whose places are counted from the launch's first token, take one launch");
  if (S != ROWS && groups > MOST) return hipErrorInvalidValue;
  for (int64_t g = 0; g < groups; g += MOST) {
    const int64_t some = std::min(MOST, groups - g);
    rotate_kernel<T, D, L, S><<<dim3((unsigned)some, (unsigned)y), ROT_THREADS, 0, stream>>>(
        runs, n_runs, where, tok_base + g * TOKENS, std::min<int64_t>(n_tok - g * TOKENS, some * TOKENS), a, (int32_t)per);
  }
  return hipGetLastError();
}

template <Source S>
hipError_t launch_rotate(const RotaryArgs& a, const RotaryRuns& runs, int32_t n_runs, const void* where, int64_t tok_base, int64_t n_tok,
                         hipStream_t stream) {
  const Layout layout = a.pairs ? PAIRS : a.rotary_dim % 8 == 0 ? HALVES : MIXED;
#define DK_LAYOUT(T, D, L) return launch_layout<T, D, L, S>(a, runs, n_runs, where, tok_base, n_tok, stream)
#define DK_SHAPE(T, D)                                \
  do {                                                \
    if (layout == HALVES) DK_LAYOUT(T, D, HALVES);    \
    if (layout == PAIRS) DK_LAYOUT(T, D, PAIRS);      \
    DK_LAYOUT(T, D, MIXED);                           \
  } while (0)
  if (a.dtype == 0 && a.head_dim == 64) DK_SHAPE(float, 64);
  if (a.dtype == 0 && a.head_dim == 128) DK_SHAPE(float, 128);
  if (a.dtype == 1 && a.head_dim == 64) DK_SHAPE(__bf16, 64);
  if (a.dtype == 1 && a.head_dim == 128) DK_SHAPE(__bf16, 128);
#undef DK_SHAPE
#undef DK_LAYOUT
  return hipErrorInvalidValue;
}

const RotaryRuns no_runs{};

}  // namespace

hipError_t launch_rotate_append(const RotaryArgs& a, const RotaryRuns& runs, int32_t n_runs, int32_t n_tok, hipStream_t stream) {
  if (n_tok <= 0) return hipSuccess;
  if (n_runs <= 0 || n_runs > ROTARY_INLINE_MAX_RUNS || runs.tok[n_runs] != n_tok) return hipErrorInvalidValue;
  return launch_rotate<RUNS>(a, runs, n_runs, nullptr, 0, n_tok, stream);
}

hipError_t launch_rotate_append_table(const RotaryArgs& a, const int32_t* table_dev, int32_t tok_base, int32_t n_tok, hipStream_t stream) {
  if (n_tok <= 0) return hipSuccess;
  return launch_rotate<TABLE>(a, no_runs, 0, table_dev, tok_base, n_tok, stream);
}

hipError_t launch_rotate_rows(const RotaryArgs& a, const int64_t* positions, int64_t n_tok, hipStream_t stream) {
  if (n_tok <= 0 || a.n_q_heads + a.n_k_heads == 0) return hipSuccess;
  return launch_rotate<ROWS>(a, no_runs, 0, positions, 0, n_tok, stream);
}

}  // namespace dk
