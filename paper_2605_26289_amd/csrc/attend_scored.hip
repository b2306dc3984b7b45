// bf16 MFMA delta attention with changed scores (gfx950): capped by a tanh, biased by distance, and rows that see a range of
// positions of their own.
//
//   s = scale q.k,  s <- cap tanh(s / cap),  s <- s - slope_h |p - k|,
//   row p sees positions max(first, p - window + 1) .. max(p, prefix - 1);  O = softmax(s) V.
//
// Scores are kept in log2 units t = s log2(e).  With u = 2^(2 log2(e) scale q.k / cap), tanh = 1 - 2 / (1 + u): one exponential,
// one reciprocal, and an infinite or vanishing u ends at the cap by itself.
// A weight is rounded once to bf16, the type of V, for the product with V; its row's sum is of the unrounded ones, in fp32.  That is off by
// at most half a step, 2^-8 of the weighted mean of |V|.  Keeping the rest of a weight for a second product with V, as the block kernel
// does for dk_delta_attend, would be half as many matrix instructions again, and in long turns those add to the time of the exponentials
// (see scored_rows_kernel).  Error against 64 bits, of the result's norm, normal inputs: bf16 store alone 1.6e-3; here one and nine
// tokens on 3000 1.7e-3 with 64-wide heads, 2.0e-3 with 128, 300 tokens on 2000 2.2e-3; dk_delta_attend 2.0e-3 to 2.3e-3 in the tile
// kernel, which rounds alike, 1.6e-3 to 1.7e-3 in the block kernel.
#include <hip/hip_runtime.h>

#include <mutex>
#include <type_traits>

#include "kernels.hpp"
#include "scored_common.hpp"

namespace dk {
namespace mfma {

namespace {

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
// Rows rl0 .. rl0 + 31 of the item, depth block db, done again without the non-finite elements of V (see redo_rows): what
// those make of a row is counted by products of their own, of one for every element and one for every key that a row sees.
// Of the block's four quads of depths, `quads` from quad0 on are this wavefront's to store.
template <int HD, bool CAP, bool BIAS>
__device__ __forceinline__ void redo_scored(const Ctx& c, const ScoreParams& sp, const int32_t* first, const DkEntry& e, const DkItem& it,
                                            int g, int rl0, uint32_t bad, float m, float l, int lane, int db, int quad0, int quads) {
  typedef Geo<HD> G;
  asm volatile("" : "+v"(lane));
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // after the ordinary store of the same rows
  const int col = lane & 31, h = lane >> 5;
  const int last_row = it.row0 + it.nrows - 1;
  const int row = min(it.row0 + rl0 + col, last_row);
  const int tok = row_token<true>(c, row);
  const int head = g * c.group + row_head<true>(c, row, tok);
  const RowRange rr = row_range(sp, first, e, tok);
  const float slope = BIAS ? sp.slopes[head] * 1.4426950408889634f : 0.f;
  const int64_t orow = (int64_t)(e.tok0 + tok) * c.n_q_heads + head;
  bf16x8 qf[G::KS];
#pragma unroll
  for (int ks = 0; ks < G::KS; ++ks) qf[ks] = signed_q(*(const bf16x8*)(c.q + orow * HD + ks * 16 + 8 * h), sp.flip);
  if (m == -INFINITY) m = 0.f;
  f32x16 o, odd[3];  // sums; counts of NaN, +infinity, -infinity
#pragma unroll
  for (int r = 0; r < 16; ++r) o[r] = odd[0][r] = odd[1][r] = odd[2][r] = 0.f;
  KvCursor<G::ROW> cur{c.segs, e.seg_begin, e.seg_end, it.kv_lo, it.kv_hi};
  KvTile t;
  while (cur.next(c, g, 32, t)) {
    const char* kp = t.k + (uint32_t)min(col, t.cnt - 1) * t.stride + 16 * h;
    f32x16 s;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
    for (int ks = 0; ks < G::KS; ++ks)
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8*)(kp + 32 * ks), qf[ks], s, 0, 0, 0);
    change_scores<CAP, BIAS>(sp, slope, (float)(t.pos + 4 * h - rr.pos), s);
    const Seen sees = seen_of(rr, t.pos + 4 * h, t.pos + t.cnt);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      bf16x8 p, seen, v, is[3];
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const int key = 16 * j + 8 * (x >> 2) + 4 * h + (x & 3);
        const uint32_t bits = *(const uint16_t*)(t.v + (uint32_t)min(key, t.cnt - 1) * t.stride + 64 * db + 2 * col);
        const bool fine = (bits & 0x7f80u) != 0x7f80u;
        v[x] = __builtin_bit_cast(__bf16, (uint16_t)(fine ? bits : 0u));
        is[0][x] = (__bf16)(!fine && (bits & 0x7fu) ? 1.f : 0.f);
        is[1][x] = (__bf16)(bits == 0x7f80u ? 1.f : 0.f);
        is[2][x] = (__bf16)(bits == 0xff80u ? 1.f : 0.f);
        const bool hidden = sees.hidden(8 * j + x);
        seen[x] = (__bf16)(hidden ? 0.f : 1.f);
        p[x] = (__bf16)(hidden ? 0.f : __builtin_amdgcn_exp2f(s[8 * j + x] - m));
      }
      o = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p, o, 0, 0, 0);
#pragma unroll
      for (int k = 0; k < 3; ++k) odd[k] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(is[k], seen, odd[k], 0, 0, 0);
    }
  }
  if ((bad >> col & 1) == 0 || rl0 + col >= it.nrows || l != l) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (i < quad0 || i >= quad0 + quads) continue;
    f32x4 x;
#pragma unroll
    for (int r = 0; r < 4; ++r) x[r] = with_non_finite(o[4 * i + r], odd[0][4 * i + r], odd[1][4 * i + r], odd[2][4 * i + r]);
    const int depth = 32 * db + 8 * i + 4 * h;
    if (it.part_row0 >= 0) {
      store_for_others((f32x4*)(c.parts + ((int64_t)(it.part_row0 + rl0 + col) * c.n_kv_heads + g) * HD + depth), x);
    } else {
      bf16x4 y;
#pragma unroll
      for (int r = 0; r < 4; ++r) y[r] = (__bf16)(x[r] * inv);
      *(bf16x4*)(c.out + orow * HD + depth) = y;
    }
  }
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

constexpr int ROWS_KT = 64;  // keys per tile of the rows kernel
template <int HD>
struct RowsGeo {
  static constexpr int TILE_BYTES = ROWS_KT * Geo<HD>::ROW;
  static constexpr int K_STAGES = 2, V_STAGES = 3;  // 80 KiB of LDS with 128-wide heads: two workgroups fill a compute unit's 160
  static constexpr int V_OFFSET = K_STAGES * TILE_BYTES;
  static constexpr int LDS_BYTES = V_OFFSET + V_STAGES * TILE_BYTES;
  static constexpr int LOADS = TILE_BYTES / 1024 / 4;  // 1 KiB requests per wavefront for a tile's K, as many for its V
};

}  // namespace

// Many rows: a workgroup owns 128 packed query rows of one KV head (4 wavefronts x 32) and walks the keys of its item in tiles
// of 64 that the wavefronts share through LDS, two workgroups to a compute unit.  Step t turns the products of tile t into weights with
// the products of tile t + 1 among the instructions of the vector unit, which with capped scores has more to do than the matrix
// cores: 28 of its cycles for a cap and 16 for the rest against 32 for a score's two products (128-wide heads).
// K of a tile is requested a step ahead, V two.  Workgroup w: item w / n_kv_heads, KV head w % n_kv_heads.
// 16 turns of 64 to 512 tokens on 1k to 8k keys, capped, 414 GFLOP: 545 to 572 us, 720 to 760 TFLOP/s (without a cap 460).  By counters
// the vector unit is busy 63 % of the SIMDs' cycles and the matrix pipe 34 %: the two run nearly one after the other.  Without the cap's
// and the weights' exponentials it took 488, without the first or the second products 462 and 457, without requests past the first
// tiles 498.  Weights of 32 keys between both products of their neighbours, in the same
// registers, took as long; 64 rows per wavefront, one wavefront per SIMD, 707.
template <int HD, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, 2) void scored_rows_kernel(InlineBlob blob, Ctx c, ScoreParams sp) {
  typedef Geo<HD> G;
  typedef RowsGeo<HD> B;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  (void)blob;
  c.entries = scored_desc(c.entries, sp.in_args);
  c.segs = scored_desc(c.segs, sp.in_args);
  c.items = scored_desc(c.items, sp.in_args);
  const int32_t* first = scored_desc(sp.first, sp.in_args);
  const int g = blockIdx.x % c.n_kv_heads;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane >> 5;
  const uint32_t koff = k_lane_off<HD>(lane), voff = v_lane_off<HD>(lane);

  const DkItem it = load_desc(c.items, blockIdx.x / c.n_kv_heads);
  const DkEntry e = load_desc(c.entries, it.entry);
  const int last_row = it.row0 + it.nrows - 1;
  const bool active = it.row0 + wave * 32 <= last_row;
  const int row = min(it.row0 + wave * 32 + (lane & 31), last_row);
  const int tok = row_token<true>(c, row);
  const int head = g * c.group + row_head<true>(c, row, tok);
  const RowRange rr = row_range(sp, first, e, tok);
  const WaveRange wr = wave_range(rr);
  const float slope = BIAS ? sp.slopes[head] * 1.4426950408889634f : 0.f;
  bf16x8 qf[G::KS];
  {
    const __bf16* qp = c.q + ((int64_t)(e.tok0 + tok) * c.n_q_heads + head) * HD + 8 * h;
#pragma unroll
    for (int ks = 0; ks < G::KS; ++ks) qf[ks] = signed_q(*(const bf16x8*)(qp + ks * 16), sp.flip);
  }

  KvCursor<G::ROW> cur{c.segs, e.seg_begin, e.seg_end, it.kv_lo, it.kv_hi};
  int cnt[3], pos[3];  // of tiles t, t + 1 and t + 2 (0 keys: none)
  int v_wr = 0;
  KvTile t;
  const auto request = [&](int slot, int k_stage) __attribute__((always_inline)) {
    cnt[slot] = 0;
    if (!cur.next(c, g, ROWS_KT, t)) return;
    cnt[slot] = t.cnt;
    pos[slot] = t.pos;
    char* kl = smem + k_stage * B::TILE_BYTES;
    char* vl = smem + B::V_OFFSET + v_wr * B::TILE_BYTES;
#pragma unroll
    for (int b = 0; b < B::LOADS; ++b) load_kib<false, HD>(t.k, t.stride, t.cnt, kl, b * 4 + wave, lane);
#pragma unroll
    for (int b = 0; b < B::LOADS; ++b) load_kib<true, HD>(t.v, t.stride, t.cnt, vl, b * 4 + wave, lane);
    v_wr = v_wr + 1 == B::V_STAGES ? 0 : v_wr + 1;
  };
  request(0, 0);
  request(1, 1);
#pragma unroll
  for (int ks = 0; ks < G::KS; ++ks) asm volatile("" ::"v"(qf[ks]));  // Q is waited for here, once
  asm volatile("" ::"v"(rr.from), "v"(slope));

  f32x16 o[1][G::DB];
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int db = 0; db < G::DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[0][db][r] = 0.f;
  const auto sees = [&](int slot) { return active && cnt[slot] > 0 && pos[slot] <= wr.any_last && pos[slot] + cnt[slot] - 1 >= wr.any_from; };

  // S^T of tile 0: behind its K come its V and tile 1
  f32x16 sa[1][2], sb[1][2];
  if (cnt[1] > 0) wait_vmcnt<3 * B::LOADS>();
  else wait_vmcnt<0>();
  scored_barrier();
  if (sees(0)) score_products<HD, 2, 1, 8>(smem, koff, sa, [&](int, int ks) { return qf[ks]; });

  int v_rd = 0;
  const auto step = [&](auto k_stage, f32x16 (&s)[1][2], f32x16 (&next)[1][2]) __attribute__((always_inline)) {
    constexpr int KST = decltype(k_stage)::value;  // where K of this tile was, and K of the tile after the next goes
    if (cnt[1] > 0) wait_vmcnt<B::LOADS>();  // only V of the next tile may be out
    else wait_vmcnt<0>();
    scored_barrier();  // landed for every wavefront; K of this tile and V of the one before have been read everywhere
    request(2, KST);
    const char* k_lds = smem + (1 - KST) * B::TILE_BYTES;
    const char* v_lds = smem + B::V_OFFSET + v_rd * B::TILE_BYTES;
    v_rd = v_rd + 1 == B::V_STAGES ? 0 : v_rd + 1;
    const int tcnt = cnt[0], tpos = pos[0];
    const bool has = sees(0), has_next = sees(1);
    cnt[0] = cnt[1];
    pos[0] = pos[1];
    cnt[1] = cnt[2];
    pos[1] = pos[2];
    if (!has) {
      if (has_next) score_products<HD, 2, 1, 8>(k_lds, koff, next, [&](int, int ks) { return qf[ks]; });
      return;
    }
    asm volatile("s_nop 11" : "+v"(s[0][0]), "+v"(s[0][1]));  // (inline assembly reads them, which the compiler does not wait for)
    const bool whole = tcnt == ROWS_KT && tpos >= wr.all_from && tpos + ROWS_KT - 1 <= wr.all_last;
    uint32_t pw[1][2][8];
    const auto rescale = [&](float alpha) {
#pragma unroll
      for (int db = 0; db < G::DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[0][db][r] *= alpha;
    };
    // (the next tile's products are computed whether a row sees it or not: a wavefront's tiles are nearly always all seen)
    constexpr int N = 2 * G::KS, AHEAD = 4;
    bf16x8 kf[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) kf[i] = read_k_frag<HD>(k_lds, koff, i % 2, i / 2);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) next[0][kb][r] = 0.f;
    // (a wavefront with a cap's exponentials to do goes before one in its second products: 16 capped turns 577 -> 557 us; without a cap
    // it does not pay, 467 -> 475)
    if constexpr (CAP && !BIAS) __builtin_amdgcn_s_setprio(1);
    weigh<CAP, BIAS, 2>(sp, rr, slope, tpos, tcnt, h, whole, s[0], m, l, pw[0], rescale, [&](int i) __attribute__((always_inline)) {
      if (16 / N * (i / (16 / N)) != i) return;  // (64-wide heads: every other time)
      const int n = i / (16 / N);
      __builtin_amdgcn_sched_barrier(0);
      next[0][n % 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[n % AHEAD], qf[n / 2], next[0][n % 2], 0, 0, 0);
      if (n + AHEAD < N) kf[n % AHEAD] = read_k_frag<HD>(k_lds, koff, (n + AHEAD) % 2, (n + AHEAD) / 2);
      __builtin_amdgcn_sched_barrier(0);
    });
    ValueFrags<HD, 4> values;
    values.first(v_lds, voff);
    if constexpr (CAP && !BIAS) __builtin_amdgcn_s_setprio(0);
    values.template products<2, 1>(v_lds, voff, pw, o);
  };
  while (cnt[0] > 0) {
    step(std::integral_constant<int, 0>(), sa, sb);
    if (cnt[0] <= 0) break;
    step(std::integral_constant<int, 1>(), sb, sa);
  }
  if (!active) return;
  const float lt = l + __shfl_xor(l, 32);
  float z = 0.f;  // NaN if any of the row's sums is not finite
#pragma unroll
  for (int db = 0; db < G::DB; ++db) {
    f32x4 quads[4];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      quads[r >> 2][r & 3] = o[0][db][r];
      z = __builtin_fmaf(o[0][db][r], 0.f, z);
    }
    store_quads<HD, true>(c, e, it, g, wave * 32 + (lane & 31), db * 32 + 4 * h, quads, lt == 0.f ? 1.f : lt);
  }
  const float lt1[1] = {lt}, mm[1] = {m};
  store_ml<1, true>(c, e, it, g, wave * 32, lane, mm, lt1);
  const uint32_t bad = bad_rows(z != 0.f);
  if (bad != 0) {
#pragma unroll 1
    for (int db = 0; db < G::DB; ++db)
      redo_scored<HD, CAP, BIAS>(c, sp, first, e, it, g, wave * 32, bad, m, lt, lane, db, 0, 4);
  }
}

namespace {

// Arrival counters, as those of the streaming kernel: zero whenever no kernel that uses them runs.
__device__ uint32_t g_scored_arrivals[ARRIVAL_SLICES * ARRIVALS_PER_SLICE];

template <int HD>
struct FewGeo {
  static constexpr int KT = 8192 / Geo<HD>::ROW;  // keys per tile: 8 KiB of K, 8 KiB of V
  static constexpr int KB = KT / 32;
  static constexpr int WAVE_BYTES = 4 * 8192;     // two stages of K and V
  static constexpr int ML_OFFSET = 4 * WAVE_BYTES;
  static constexpr int Q_OFFSET = ML_OFFSET + 4 * 32 * 8;
  static constexpr int lds_bytes(int rb) { return Q_OFFSET + (rb > 1 ? rb * Geo<HD>::KS * 1024 : 0); }
};

}  // namespace

// Few rows: at most 32 RB packed rows of one KV head to a workgroup, whose four wavefronts each walk a quarter of the item's keys
// through two private LDS stages, with no barrier until their sums are merged.  One workgroup to a compute unit.  K of tile t + 2
// is requested as soon as K of tile t has been read, V likewise: 16 to 32 KiB in flight per wavefront.  Two row blocks keep their Q
// in LDS, in the order of the fragments: registers are held to 256 (the bound on occupancy says so), since beyond that the
// accumulators move to the other half of the register file, and the compiler copies all of them back for every tile.
// 64 sessions verifying up to 9 tokens over 4096 visible keys each, 1.08 GB: 187 us with a cap, 179 without, 5.8 and 6.0 TB/s.
// One token on 3000 keys of 8 heads: 10.6 us a call, the merge inside (with a launch for it 12.2: 7.4 us and 3.4).
template <int HD, int RB, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, 2) void scored_few_kernel(InlineBlob blob, Ctx c, ScoreParams sp) {
  typedef Geo<HD> G;
  typedef FewGeo<HD> F;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  (void)blob;
  c.entries = scored_desc(c.entries, sp.in_args);
  c.segs = scored_desc(c.segs, sp.in_args);
  c.items = scored_desc(c.items, sp.in_args);
  const int32_t* first = scored_desc(sp.first, sp.in_args);
  const int g = blockIdx.x % c.n_kv_heads;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane >> 5;
  uint32_t koff = k_lane_off<HD>(lane), voff = v_lane_off<HD>(lane);
  char* mine = smem + wave * F::WAVE_BYTES;
  const uint32_t mine_addr = (uint32_t)(uintptr_t)(lds_void_ptr)mine;

  const DkItem it = load_desc(c.items, blockIdx.x / c.n_kv_heads);
  const DkEntry e = load_desc(c.entries, it.entry);
  const int last_row = it.row0 + it.nrows - 1;

  // this wavefront's share of the keys
  const int blocks = (it.kv_hi - it.kv_lo + F::KT - 1) / F::KT;
  const int per = (blocks + 3) / 4 * F::KT;
  const int lo = min(it.kv_hi, it.kv_lo + wave * per), hi = min(it.kv_hi, lo + per);
  KvCursor<G::ROW> cur{c.segs, e.seg_begin, e.seg_end, lo, hi};
  // tiles t (slot 0), t + 1 (slot 1) and, from the middle of step t on, t + 2
  KvTile tiles[3];
  // (the requests' offsets are the same for all whole tiles of a segment)
  uint32_t offk[8], offv[8], off_stride = 0;
  int off_cnt = 0;
  const auto offsets = [&](const KvTile& t) __attribute__((always_inline)) {
    if (t.stride == off_stride && t.cnt == off_cnt) return;
    off_stride = t.stride;
    off_cnt = t.cnt;
#pragma unroll
    for (int b = 0; b < 8; ++b) {
      offk[b] = kib_biased_off<false, HD>(t.stride, t.cnt, b, lane);
      offv[b] = kib_biased_off<true, HD>(t.stride, t.cnt, b, lane);
    }
  };
  const auto request = [&](auto is_v, const KvTile& t, int stage) __attribute__((always_inline)) {
    constexpr bool V = decltype(is_v)::value;
    if (t.cnt == 0) return;
    const char* from = V ? t.v : t.k;
    const uint32_t to = mine_addr + stage * 16384 + (V ? 8192 : 0);
    offsets(t);
    if (t.once) load_eight_kib<true>(from, V ? offv : offk, to);
    else load_eight_kib<false>(from, V ? offv : offk, to);
  };
  const auto request_k = [&](const KvTile& t, int stage) __attribute__((always_inline)) { request(std::false_type(), t, stage); };
  const auto request_v = [&](const KvTile& t, int stage) __attribute__((always_inline)) { request(std::true_type(), t, stage); };
  const auto take = [&](KvTile& t) __attribute__((always_inline)) {
    if (!cur.next(c, g, F::KT, t)) t.cnt = 0;
  };
  take(tiles[0]);
  request_k(tiles[0], 0);
  request_v(tiles[0], 0);

  RowRange rr[RB];
  WaveRange wr[RB];
  float slope[RB];
  constexpr bool Q_IN_LDS = RB > 1;
  bf16x8 qf[G::KS];
  bf16x8* q_lds = (bf16x8*)(smem + F::Q_OFFSET) + lane;  // [row block][depth step][lane]
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int row = min(it.row0 + rb * 32 + (lane & 31), last_row);
    const int tok = row_token<true>(c, row);
    const int head = g * c.group + row_head<true>(c, row, tok);
    rr[rb] = row_range(sp, first, e, tok);
    slope[rb] = BIAS ? sp.slopes[head] * 1.4426950408889634f : 0.f;
    const __bf16* qp = c.q + ((int64_t)(e.tok0 + tok) * c.n_q_heads + head) * HD + 8 * h;
#pragma unroll
    for (int ks = 0; ks < G::KS; ++ks) {
      if (!Q_IN_LDS) qf[ks] = signed_q(*(const bf16x8*)(qp + ks * 16), sp.flip);
      else if (ks % 4 == wave) q_lds[(rb * G::KS + ks) * 64] = signed_q(*(const bf16x8*)(qp + ks * 16), sp.flip);
    }
  }
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) wr[rb] = wave_range(rr[rb]);
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) asm volatile("" ::"v"(slope[rb]), "v"(rr[rb].from));  // waited for here, once
  if constexpr (Q_IN_LDS) {
    __syncthreads();
  } else {
#pragma unroll
    for (int ks = 0; ks < G::KS; ++ks) asm volatile("" ::"v"(qf[ks]));
  }
  take(tiles[1]);
  request_k(tiles[1], 1);
  request_v(tiles[1], 1);

  f32x16 o[RB][G::DB];
  float m[RB], l[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    m[rb] = -INFINITY;
    l[rb] = 0.f;
#pragma unroll
    for (int db = 0; db < G::DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[rb][db][r] = 0.f;
  }

  int stage = 0;
  while (tiles[0].cnt > 0) {
    const bool one_more = tiles[1].cnt > 0;
    // requests younger than K of this tile: its V, and K and V of the next one
    if (one_more) wait_vmcnt<24>();
    else wait_vmcnt<8>();
    const char* k_lds = mine + stage * 16384;
    const char* v_lds = k_lds + 8192;
    f32x16 s[RB][F::KB];
    // (computed anew from here on in every step: kept across steps, the addresses of the fragments cost more registers than there are)
    if constexpr (RB > 1) asm volatile("" : "+v"(koff), "+v"(voff));
    score_products<HD, F::KB, RB, 4>(k_lds, koff, s, [&](int rb, int ks) { return Q_IN_LDS ? q_lds[(rb * G::KS + ks) * 64] : qf[ks]; });
    // K has been read.  (The products are waited for here, on this side of the branches that follow: the compiler's own wait, on
    // the far side, counts the states of the longest way there.)
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int kb = 0; kb < F::KB; ++kb) asm volatile("s_nop %1" : "+v"(s[rb][kb]) : "n"(rb == RB - 1 && kb == F::KB - 1 ? 11 : 0));
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    take(tiles[2]);
    request_k(tiles[2], stage);
    const int tcnt = tiles[0].cnt, tpos = tiles[0].pos;
    uint32_t pw[RB][F::KB][8];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const bool whole = tcnt == F::KT && tpos >= wr[rb].all_from && tpos + F::KT - 1 <= wr[rb].all_last;
      weigh<CAP, BIAS, F::KB>(sp, rr[rb], slope[rb], tpos, tcnt, h, whole, s[rb], m[rb], l[rb], pw[rb], [&](float alpha) {
#pragma unroll
        for (int db = 0; db < G::DB; ++db)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[rb][db][r] *= alpha;
      }, [](int) {});
    }
    // requests younger than V of this tile: K and V of the next one, K of the one after
    if (one_more && tiles[2].cnt > 0) wait_vmcnt<24>();
    else if (one_more) wait_vmcnt<16>();
    else wait_vmcnt<0>();
    ValueFrags<HD, 4> values;
    values.first(v_lds, voff);
    values.template products<F::KB, RB>(v_lds, voff, pw, o);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // V has been read
    request_v(tiles[2], stage);
    tiles[0] = tiles[1];
    tiles[1] = tiles[2];
    stage ^= 1;
  }

  // Merge of the wavefronts' states, a block of 32 rows at a time: quad (db, r4) of a lane is depths 32 db + 8 r4 + 4 h .. + 3 of
  // its row; wavefront w stores quads w NQ .. of each row.
  constexpr int NQ = G::DB;  // of 4 DB quads
  f32x4* xo = (f32x4*)smem;  // [wave][quad][lane]
  float2* xml = (float2*)(smem + F::ML_OFFSET);
  const int quad0 = wave * NQ;
  uint32_t bad[RB];
  float mm[RB], lsum[RB];
  const bool merges = RB == 1 && sp.arrival_slice >= 0 && it.merge != 0;  // see merge_if_last
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const float lt = l[rb] + __shfl_xor(l[rb], 32);
    __syncthreads();
    if (lane < 32) xml[wave * 32 + lane] = make_float2(m[rb], lt);
#pragma unroll
    for (int db = 0; db < G::DB; ++db)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4)
        xo[(wave * 4 * G::DB + db * 4 + r4) * 64 + lane] =
            f32x4{o[rb][db][4 * r4], o[rb][db][4 * r4 + 1], o[rb][db][4 * r4 + 2], o[rb][db][4 * r4 + 3]};
    __syncthreads();
    float2 ml[4];
    mm[rb] = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      ml[w] = xml[w * 32 + (lane & 31)];
      mm[rb] = fmaxf(mm[rb], ml[w].x);
    }
    const float ms = (mm[rb] == -INFINITY) ? 0.f : mm[rb];
    lsum[rb] = 0.f;
    f32x4 acc[NQ];
#pragma unroll
    for (int i = 0; i < NQ; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = __builtin_amdgcn_exp2f(ml[w].x - ms);
      lsum[rb] += f * ml[w].y;
#pragma unroll
      for (int i = 0; i < NQ; ++i) acc[i] += f * xo[(w * 4 * G::DB + quad0 + i) * 64 + lane];
    }
    store_quads<HD, true>(c, e, it, g, rb * 32 + (lane & 31), quad0 * 8 + 4 * h, acc, lsum[rb] == 0.f ? 1.f : lsum[rb], merges);
    const float lt1[1] = {lsum[rb]}, m1[1] = {mm[rb]};
    if (wave == 0) store_ml<1, true>(c, e, it, g, rb * 32, lane, m1, lt1, merges);
    float z = 0.f;
#pragma unroll
    for (int i = 0; i < NQ; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) z = __builtin_fmaf(acc[i][r], 0.f, z);
    bad[rb] = bad_rows(z != 0.f);
  }
#pragma unroll 1
  for (int rb = 0; rb < RB; ++rb) {
    const uint32_t which = rb == 0 ? bad[0] : bad[RB - 1];
    if (which != 0)
      redo_scored<HD, CAP, BIAS>(c, sp, first, e, it, g, rb * 32, which, rb == 0 ? mm[0] : mm[RB - 1], rb == 0 ? lsum[0] : lsum[RB - 1], lane,
                                 quad0 / 4, quad0 % 4, NQ);
  }
  if constexpr (RB == 1) {
    if (merges)
      merge_if_last<HD, true, true>(c, e, it, g, g_scored_arrivals + sp.arrival_slice * ARRIVALS_PER_SLICE, smem, F::ML_OFFSET);
  }
}

// Merge of split key ranges, as attend_merge_kernel, with rows that no split has a key for.
template <int HD>
__global__ __launch_bounds__(256) void scored_merge_kernel(InlineBlob blob, Ctx c, ScoreParams sp, const DkMerge* merges) {
  constexpr int LANES = HD / 4, GROUPS = 256 / LANES;
  (void)blob;
  const DkMerge mg = load_desc(scored_desc(merges, sp.in_args), blockIdx.x);
  const int lane = threadIdx.x % LANES;
  const int rl = blockIdx.z * GROUPS + threadIdx.x / LANES;
  if (rl >= mg.nrows) return;
  const int g = blockIdx.y;
  const int64_t step = (int64_t)mg.nrows * c.n_kv_heads;
  const int64_t prow = (int64_t)(mg.part_row0 + rl) * c.n_kv_heads + g;
  float m = -INFINITY, l = 0.f;
  f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
  constexpr int AHEAD = 4;
  for (int s0 = 0; s0 < mg.nsplit; s0 += AHEAD) {
    float2 ml[AHEAD];
    f32x4 v[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int64_t at = prow + min(s0 + k, mg.nsplit - 1) * step;
      ml[k] = *(const float2*)(c.parts_ml + at * 2);
      v[k] = *(const f32x4*)(c.parts + at * HD + lane * 4);
    }
    float mn = m;
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      if (s0 + k >= mg.nsplit) ml[k] = make_float2(-INFINITY, 0.f);
      mn = fmaxf(mn, ml[k].x);
    }
    const float ms = mn == -INFINITY ? 0.f : mn;
    const float a = __builtin_amdgcn_exp2f(m - ms);
    m = mn;
    l *= a;
    acc *= piece_weight(a);
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      if (s0 + k >= mg.nsplit) continue;
      const float f = __builtin_amdgcn_exp2f(ml[k].x - ms);
      l += f * ml[k].y;
      acc += piece_weight(f) * v[k];
    }
  }
  const int row = mg.row0 + rl;
  const int tok = row_token<true>(c, row);
  const int64_t orow = (int64_t)(mg.tok0 + tok) * c.n_q_heads + g * c.group + row_head<true>(c, row, tok);
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if (sp.f32) {
    *(f32x4*)((float*)c.out + orow * HD + lane * 4) = acc * inv;
  } else {
    bf16x4 y;
#pragma unroll
    for (int r = 0; r < 4; ++r) y[r] = (__bf16)(acc[r] * inv);
    *(bf16x4*)(c.out + orow * HD + lane * 4) = y;
  }
  if (c.lse && lane == 0) c.lse[orow] = (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

namespace {

template <typename K>
hipError_t allow_lds(K kernel, int bytes) {
  return hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

template <int HD, bool CAP, bool BIAS>
hipError_t launch_scored(const InlineBlob& blob, const Ctx& c, const ScoreParams& sp, const ScoredItems& items, hipStream_t stream) {
  // once per process and instantiation, whatever thread or pool gets here first
  static std::once_flag once;
  static hipError_t status = hipSuccess;
  std::call_once(once, [] {
    status = allow_lds(scored_rows_kernel<HD, CAP, BIAS>, RowsGeo<HD>::LDS_BYTES);
    if (status == hipSuccess) status = allow_lds(scored_few_kernel<HD, 1, CAP, BIAS>, FewGeo<HD>::lds_bytes(1));
    if (status == hipSuccess) status = allow_lds(scored_few_kernel<HD, 2, CAP, BIAS>, FewGeo<HD>::lds_bytes(2));
  });
  if (status != hipSuccess) return status;
  Ctx d = c;
  const unsigned heads = (unsigned)c.n_kv_heads;
  if (items.n_rows > 0) {
    d.items = items.rows;
    scored_rows_kernel<HD, CAP, BIAS><<<dim3((unsigned)items.n_rows * heads), 256, RowsGeo<HD>::LDS_BYTES, stream>>>(blob, d, sp);
  }
  if (items.n_few > 0) {
    d.items = items.few;
    if (items.few_rows <= 32)
      scored_few_kernel<HD, 1, CAP, BIAS><<<dim3((unsigned)items.n_few * heads), 256, FewGeo<HD>::lds_bytes(1), stream>>>(blob, d, sp);
    else
      scored_few_kernel<HD, 2, CAP, BIAS><<<dim3((unsigned)items.n_few * heads), 256, FewGeo<HD>::lds_bytes(2), stream>>>(blob, d, sp);
  }
  return hipGetLastError();
}

template <int HD>
hipError_t launch_scored(const AttendArgs& a, const Ctx& c, const ScoreParams& sp, const ScoredItems& items, const InlineBlob& blob,
                         hipStream_t stream) {
  hipError_t e;
  if (sp.f32) e = launch_attend_f32_scored(a, sp, items.rows, items.n_rows, items.tile_rows, stream);
  else if (sp.capped) e = sp.slopes ? launch_scored<HD, true, true>(blob, c, sp, items, stream) : launch_scored<HD, true, false>(blob, c, sp, items, stream);
  else e = sp.slopes ? launch_scored<HD, false, true>(blob, c, sp, items, stream) : launch_scored<HD, false, false>(blob, c, sp, items, stream);
  if (e != hipSuccess || items.n_merges <= 0) return e;
  constexpr int rows = 1024 / HD;
  scored_merge_kernel<HD><<<dim3((unsigned)items.n_merges, (unsigned)c.n_kv_heads, (unsigned)((items.merge_rows + rows - 1) / rows)), 256, 0, stream>>>(
      blob, c, sp, items.merges);
  return hipGetLastError();
}

}  // namespace

}  // namespace mfma

hipError_t launch_attend_scored(const AttendArgs& a, const ScoreParams& sp, const ScoredItems& items, hipStream_t stream) {
  using namespace mfma;
  static const InlineBlob none{};
  const Ctx c = make_ctx(a, nullptr);
  const InlineBlob& blob = a.inline_blob ? *a.inline_blob : none;
  if (a.arena.head_dim == 64) return launch_scored<64>(a, c, sp, items, blob, stream);
  if (a.arena.head_dim == 128) return launch_scored<128>(a, c, sp, items, blob, stream);
  return hipErrorInvalidValue;
}

}  // namespace dk
