// Shared device code of the kernels for attention with changed scores and of those for shared prefixes: what a row sees, and the two
// products of a tile with the softmax between them.
#pragma once
#include "attend_common.hpp"

namespace dk {
namespace mfma {

// What a row sees: positions from .. last.
struct RowRange {
  int32_t pos, from, last;
};
__device__ __forceinline__ RowRange row_range(const ScoreParams& sp, const int32_t* first, const DkEntry& e, int tok) {
  RowRange r;
  r.pos = e.n + tok;
  r.last = max(r.pos, e.pad[0] - 1);
  r.from = sp.has_first ? first[e.tok0 + tok] : 0;
  if (sp.window > 0) r.from = max(r.from, r.pos - sp.window + 1);
  return r;
}

// What the non-finite elements of V that a row sees make of a sum of the finite ones, by their numbers.
__device__ __forceinline__ float with_non_finite(float sum, float nans, float plus, float minus) {
  if (nans > 0.f || (plus > 0.f && minus > 0.f)) return __uint_as_float(0x7fc00000u);
  return plus > 0.f ? INFINITY : minus > 0.f ? -INFINITY : sum;
}

// ---- bf16: 32 packed rows of a wavefront against tiles of keys
constexpr float SCORED_RESCALE_SLACK = 8.f;  // log2 units, as in the block kernel

// The largest of 16 values, raw products among them: the builtin would first make each of those canonical, an instruction a value.
__device__ __forceinline__ float max16(const f32x16& s) {
  float d;
  asm("v_max3_f32 %0, %1, %2, %3\n\tv_max3_f32 %0, %0, %4, %5\n\tv_max3_f32 %0, %0, %6, %7\n\tv_max3_f32 %0, %0, %8, %9\n\t"
      "v_max3_f32 %0, %0, %10, %11\n\tv_max3_f32 %0, %0, %12, %13\n\tv_max3_f32 %0, %0, %14, %15\n\tv_max_f32 %0, %0, %16"
      : "=&v"(d)
      : "v"(s[0]), "v"(s[1]), "v"(s[2]), "v"(s[3]), "v"(s[4]), "v"(s[5]), "v"(s[6]), "v"(s[7]), "v"(s[8]), "v"(s[9]), "v"(s[10]),
        "v"(s[11]), "v"(s[12]), "v"(s[13]), "v"(s[14]), "v"(s[15]));
  return d;
}

// A Q fragment, its signs turned where the scale is negative (the kernels work with the scale's size).
__device__ __forceinline__ bf16x8 signed_q(bf16x8 q, uint32_t flip) {
  typedef __attribute__((ext_vector_type(4))) uint32_t words;
  return __builtin_bit_cast(bf16x8, __builtin_bit_cast(words, q) ^ words{flip, flip, flip, flip});
}

// The kernels' first argument holds the descriptors if they fit; otherwise they are in the workspace.
template <typename T>
__device__ __forceinline__ const T* scored_desc(const T* p, bool in_args) {
  typedef const __attribute__((address_space(4))) char* const_char_ptr;
  const uintptr_t base = in_args ? (uintptr_t)(const_char_ptr)__builtin_amdgcn_kernarg_segment_ptr() : 0;
  return (const T*)(base + (uintptr_t)p);
}

// Of the rows of a wavefront (each in two lanes): the first and last position that any sees, and that all see.
struct WaveRange {
  int32_t any_from, any_last, all_from, all_last;
};
__device__ __forceinline__ WaveRange wave_range(const RowRange& r) {
  const bool empty = r.from > r.last;
  WaveRange w{empty ? INT32_MAX : r.from, empty ? -1 : r.last, r.from, r.last};
#pragma unroll
  for (int off = 16; off >= 1; off >>= 1) {
    w.any_from = min(w.any_from, __shfl_xor(w.any_from, off));
    w.any_last = max(w.any_last, __shfl_xor(w.any_last, off));
    w.all_from = max(w.all_from, __shfl_xor(w.all_from, off));
    w.all_last = min(w.all_last, __shfl_xor(w.all_last, off));
  }
  w.any_from = __builtin_amdgcn_readfirstlane(w.any_from);
  w.any_last = __builtin_amdgcn_readfirstlane(w.any_last);
  w.all_from = __builtin_amdgcn_readfirstlane(w.all_from);
  w.all_last = __builtin_amdgcn_readfirstlane(w.all_last);
  return w;
}

// Raw products of a 32-key block (accumulator r is key 8 (r / 4) + 4 h + r % 4) to scores in log2 units.  ahead: position of
// the block's key 4 h less the row's.
template <bool CAP, bool BIAS>
__device__ __forceinline__ void change_scores(const ScoreParams& sp, float slope, float ahead, f32x16& s) {
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    float t;
    if constexpr (CAP) {
      const float u = __builtin_amdgcn_exp2f(s[r] * sp.c);
      t = __builtin_fmaf(-2.f * sp.cap, __builtin_amdgcn_rcpf(1.f + u), sp.cap);
    } else {
      t = s[r] * sp.c;
    }
    if constexpr (BIAS) t = __builtin_fmaf(-slope, __builtin_fabsf(ahead + (float)(8 * (r >> 2) + (r & 3))), t);
    s[r] = t;
  }
}
// The keys of a 32-key block that a row does not see: those outside lo .. lo + span - 1 (relative to the block's key 4 h).
struct Seen {
  int32_t lo;
  uint32_t span;
  __device__ __forceinline__ bool hidden(int r) const { return (uint32_t)(8 * (r >> 2) + (r & 3) - lo) >= span; }
};
__device__ __forceinline__ Seen seen_of(const RowRange& rr, int at, int end) {  // at: the block's key 4 h; end: behind the tile's last
  const int lo = max(rr.from - at, 0);
  return {lo, (uint32_t)max(0, min(end, rr.last + 1) - at - lo)};
}
__device__ __forceinline__ void hide_scores(const Seen& seen, f32x16& s) {
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = seen.hidden(r) ? -INFINITY : s[r];
}

// One tile's raw products of 32 rows, KB blocks of 32 keys, to weights: packed pairs in the order of the second product's operand.
// Scores rise with the products (the scale is positive), so without a bias by distance the tile's largest score is that of its largest
// product, and a score and its distance from the reference maximum are one fused operation.  `rescale(alpha)` is called where the
// reference maximum is raised, which it only is when the tile outgrows it by more than the slack; `tick(i)` four times for every eight
// weights, i from 0 to 8 KB - 1, for matrix instructions of the caller's to stand between those of the vector unit.
template <bool CAP, bool BIAS, int KB, typename Rescale, typename Tick>
__device__ __forceinline__ void weigh(const ScoreParams& sp, const RowRange& rr, float slope, int tpos, int tcnt, int h, bool whole,
                                      f32x16 (&s)[KB], float& m, float& l, uint32_t (&pw)[KB][8], Rescale&& rescale, Tick&& tick) {
#pragma unroll
  for (int kb = 0; kb < KB; ++kb) {
    const int at = tpos + 32 * kb + 4 * h;
    if constexpr (BIAS) change_scores<CAP, BIAS>(sp, slope, (float)(at - rr.pos), s[kb]);
    if (!whole) hide_scores(seen_of(rr, at, tpos + tcnt), s[kb]);
    asm volatile("" : "+v"(s[kb]));  // (the way around the branch and the way through it meet in the same registers)
  }
  float mx = max16(s[0]);
  if constexpr (KB == 2) mx = fmaxf(mx, max16(s[KB - 1]));
  mx = fmaxf(mx, __shfl_xor(mx, 32));
  if constexpr (CAP && !BIAS) {
    // (A product of -infinity may well be one that the row sees, of score -cap: whether it sees any is a matter of positions.)
    const bool sees = max(rr.from, tpos) < min(rr.last + 1, tpos + tcnt);
    const float t = __builtin_fmaf(-2.f * sp.cap, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(mx * sp.c)), sp.cap);
    mx = sees ? t : -INFINITY;
  } else if constexpr (!BIAS) {
    mx *= sp.c;  // (the scale is positive: -infinity, of a row that sees nothing of the tile, stays what it is)
  }
  if (__builtin_amdgcn_ballot_w64(mx > m + SCORED_RESCALE_SLACK) != 0) {
    const float mn = fmaxf(m, mx);
    const float alpha = __builtin_amdgcn_exp2f(m - ((mn == -INFINITY) ? 0.f : mn));
    m = mn;
    l *= alpha;
    rescale(alpha);
  }
  const float ms = (m == -INFINITY) ? 0.f : m;
  const float top = sp.cap - ms;
  float sums[2] = {0.f, 0.f};
#pragma unroll
  for (int kb = 0; kb < KB; ++kb)
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const int at = 8 * kb + 4 * q;
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float raw = s[kb][8 * q + i];
        if constexpr (BIAS) x[i] = raw - ms;
        else if constexpr (CAP) x[i] = raw * sp.c;
        else x[i] = __builtin_fmaf(raw, sp.c, -ms);
      }
      tick(at);
      if constexpr (CAP && !BIAS) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __builtin_amdgcn_exp2f(x[i]);
        tick(at + 1);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __builtin_amdgcn_rcpf(1.f + x[i]);
        tick(at + 2);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __builtin_fmaf(-2.f * sp.cap, x[i], top);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = __builtin_amdgcn_exp2f(x[i]);
      if constexpr (!CAP || BIAS) {
        tick(at + 1);
        tick(at + 2);
      }
      if constexpr (CAP && !BIAS) {
        if (!whole) {  // (a hidden score has come out as -cap)
          Seen seen = seen_of(rr, tpos + 32 * kb + 4 * h, tpos + tcnt);
          asm volatile("" : "+v"(seen.lo), "+v"(seen.span));  // (compared anew: 32 masks do not fit the scalar registers)
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = seen.hidden(8 * q + i) ? 0.f : x[i];
        }
      }
      tick(at + 3);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        sums[0] += x[2 * w];
        sums[1] += x[2 * w + 1];
        pw[kb][4 * q + w] = pack_pair(x[2 * w], x[2 * w + 1]);
      }
    }
  l += sums[0] + sums[1];
}
// Fragment j (16 keys) of a tile's weights.
template <int KB>
__device__ __forceinline__ bf16x8 weight_frag(const uint32_t (&pw)[KB][8], int j) {
  typedef __attribute__((ext_vector_type(4))) uint32_t words;
  const uint32_t* w = &pw[j >> 1][4 * (j & 1)];
  return __builtin_bit_cast(bf16x8, words{w[0], w[1], w[2], w[3]});
}
// The two products of a tile, their LDS operands AHEAD fragments in front of the product that takes them: left to itself the compiler
// reads each fragment right before its product and waits, 16 times the latency of LDS for a tile.
// q_of(rb, ks): the Q fragment; S^T of RB row blocks of 32 against KB blocks of 32 keys.
template <int HD, int KB, int RB, int AHEAD, typename Q>
__device__ __forceinline__ void score_products(const char* k_lds, uint32_t koff, f32x16 (&s)[RB][KB], Q&& q_of) {
  constexpr int N = Geo<HD>::KS * KB;
  bf16x8 kf[AHEAD];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) kf[i] = read_k_frag<HD>(k_lds, koff, i % KB, i / KB);
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[rb][kb][r] = 0.f;
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int i = 0; i < N; ++i) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
      s[rb][i % KB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i % AHEAD], q_of(rb, i / KB), s[rb][i % KB], 0, 0, 0);
    if (i + AHEAD < N) kf[i % AHEAD] = read_k_frag<HD>(k_lds, koff, (i + AHEAD) % KB, (i + AHEAD) / KB);
    __builtin_amdgcn_sched_barrier(0);
  }
}
template <int HD, int AHEAD>
struct ValueFrags {
  bf16x8 vf[AHEAD];
  __device__ __forceinline__ void first(const char* v_lds, uint32_t voff) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) vf[i] = read_v_frag<HD>(v_lds, voff, i / Geo<HD>::DB, i % Geo<HD>::DB);
    __builtin_amdgcn_sched_barrier(0);
  }
  // O^T += V^T P^T of RB row blocks
  template <int KB, int RB>
  __device__ __forceinline__ void products(const char* v_lds, uint32_t voff, const uint32_t (&pw)[RB][KB][8], f32x16 (&o)[RB][Geo<HD>::DB]) {
    constexpr int DB = Geo<HD>::DB, N = 2 * KB * DB;
#pragma unroll
    for (int i = 0; i < N; ++i) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
        o[rb][i % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i % AHEAD], weight_frag<KB>(pw[rb], i / DB), o[rb][i % DB], 0, 0, 0);
      if (i + AHEAD < N) vf[i % AHEAD] = read_v_frag<HD>(v_lds, voff, (i + AHEAD) / DB, (i + AHEAD) % DB);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
};

template <typename F>
__device__ __forceinline__ uint32_t bad_rows(F&& any) {
  const uint64_t b = __builtin_amdgcn_ballot_w64(any);
  return (uint32_t)(b | b >> 32);
}

__device__ __forceinline__ void scored_barrier() {  // LDS reads of this wavefront have returned; K/V requests stay in flight
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

}  // namespace mfma
}  // namespace dk
