// bf16 MFMA delta attention with changed scores (gfx950): capped by a tanh, biased by distance, and rows that see a range of
// positions of their own.
//
//   s = scale q.k,  s <- cap tanh(s / cap),  s <- s - slope_h |p - k|,
//   row p sees positions max(first, p - window + 1) .. max(p, prefix - 1);  O = softmax(s) V.
//
// Scores are kept in log2 units t = s log2(e).  With u = 2^(2 log2(e) scale q.k / cap), tanh = 1 - 2 / (1 + u): one exponential,
// one reciprocal, and an infinite or vanishing u ends at the cap by itself.
#include <hip/hip_runtime.h>

#include <mutex>

#include "kernels.hpp"
#include "scored_common.hpp"

namespace dk {
namespace mfma {

namespace {

constexpr float SCORED_RESCALE_SLACK = 8.f;  // log2 units, as in the block kernel

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
  return d;
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
// Hides the keys of a 32-key block outside lo .. hi (relative to the block's key 4 h).
__device__ __forceinline__ void hide_scores(int lo, int hi, f32x16& s) {
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int key = 8 * (r >> 2) + (r & 3);
    if (key < lo || key > hi) s[r] = -INFINITY;
  }
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
  for (int ks = 0; ks < G::KS; ++ks) qf[ks] = *(const bf16x8*)(c.q + orow * HD + ks * 16 + 8 * h);
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
    hide_scores(rr.from - t.pos - 4 * h, min(t.cnt - 1, rr.last - t.pos) - 4 * h, s);
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
        const float score = s[8 * j + x];
        seen[x] = (__bf16)(score != -INFINITY ? 1.f : 0.f);
        p[x] = (__bf16)__builtin_amdgcn_exp2f(score - m);
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
      *(f32x4*)(c.parts + ((int64_t)(it.part_row0 + rl0 + col) * c.n_kv_heads + g) * HD + depth) = x;
    } else {
      bf16x4 y;
#pragma unroll
      for (int r = 0; r < 4; ++r) y[r] = (__bf16)(x[r] * inv);
      *(bf16x4*)(c.out + orow * HD + depth) = y;
    }
  }
}

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
  static constexpr int STAGE_BYTES = 2 * TILE_BYTES;
  static constexpr int STAGES = HD == 128 ? 2 : 4;  // 64 KiB of LDS either way
  static constexpr int LDS_BYTES = STAGES * STAGE_BYTES;
  static constexpr int LOADS = STAGE_BYTES / 1024 / 4;  // 1 KiB requests per wavefront and tile
};

}  // namespace

// Many rows: a workgroup owns 128 packed query rows of one KV head (4 wavefronts x 32) and walks the keys of its item in tiles
// of 64 that the wavefronts share through an LDS ring, two workgroups to a compute unit, as in the block kernel.
// Workgroup w: item w / n_kv_heads, KV head w % n_kv_heads.
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
    for (int ks = 0; ks < G::KS; ++ks) qf[ks] = *(const bf16x8*)(qp + ks * 16);
  }

  KvCursor<G::ROW> cur{c.segs, e.seg_begin, e.seg_end, it.kv_lo, it.kv_hi};
  int cnt[B::STAGES] = {}, pos[B::STAGES] = {};  // tiles requested and not yet computed, oldest first
  int stage_wr = 0;
  KvTile t;
  auto request = [&](int slot) {
    cnt[slot] = 0;
    if (!cur.next(c, g, ROWS_KT, t)) return;
    cnt[slot] = t.cnt;
    pos[slot] = t.pos;
    char* kl = smem + stage_wr * B::STAGE_BYTES;
    char* vl = kl + B::TILE_BYTES;
#pragma unroll
    for (int b = 0; b < B::LOADS / 2; ++b) load_kib<false, HD>(t.k, t.stride, t.cnt, kl, b * 4 + wave, lane);
#pragma unroll
    for (int b = 0; b < B::LOADS / 2; ++b) load_kib<true, HD>(t.v, t.stride, t.cnt, vl, b * 4 + wave, lane);
    stage_wr = stage_wr + 1 == B::STAGES ? 0 : stage_wr + 1;
  };
#pragma unroll
  for (int s = 0; s < B::STAGES - 1; ++s) request(s);
#pragma unroll
  for (int ks = 0; ks < G::KS; ++ks) asm volatile("" ::"v"(qf[ks]));  // Q is waited for here, once
  asm volatile("" ::"v"(rr.from), "v"(slope));

  f32x16 o[G::DB];
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int db = 0; db < G::DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[db][r] = 0.f;

  int stage_rd = 0;
  while (cnt[0] > 0) {
    int younger = 0;
#pragma unroll
    for (int s = 1; s < B::STAGES - 1; ++s) younger += cnt[s] > 0;
    if (B::STAGES > 3 && younger == 2) wait_vmcnt<2 * B::LOADS>();
    else if (B::STAGES > 2 && younger == 1) wait_vmcnt<B::LOADS>();
    else wait_vmcnt<0>();
    scored_barrier();  // landed for every wavefront, and the tile before it is finished everywhere
    request(B::STAGES - 1);
    const char* k_lds = smem + stage_rd * B::STAGE_BYTES;
    const char* v_lds = k_lds + B::TILE_BYTES;
    stage_rd = stage_rd + 1 == B::STAGES ? 0 : stage_rd + 1;
    const int tcnt = cnt[0], tpos = pos[0];
#pragma unroll
    for (int s = 0; s < B::STAGES - 1; ++s) {
      cnt[s] = cnt[s + 1];
      pos[s] = pos[s + 1];
    }
    if (!active || tpos > wr.any_last || tpos + tcnt - 1 < wr.any_from) continue;  // no row of this wavefront sees the tile

    f32x16 s[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[kb][r] = 0.f;
#pragma unroll
    for (int ks = 0; ks < G::KS; ++ks)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
        s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_k_frag<HD>(k_lds, koff, kb, ks), qf[ks], s[kb], 0, 0, 0);
    const bool whole = tcnt == ROWS_KT && tpos >= wr.all_from && tpos + ROWS_KT - 1 <= wr.all_last;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const int at = tpos + 32 * kb + 4 * h;
      change_scores<CAP, BIAS>(sp, slope, (float)(at - rr.pos), s[kb]);
      if (!whole) hide_scores(rr.from - at, min(tpos + tcnt - 1, rr.last) - at, s[kb]);
    }
    float mx = max3(s[0][0], s[1][0], s[0][1]);
    mx = fmaxf(mx, s[1][1]);
#pragma unroll
    for (int r = 2; r < 16; ++r) mx = max3(mx, s[0][r], s[1][r]);
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    // the reference maximum is only raised when the tile outgrows it by more than the slack
    if (__builtin_amdgcn_ballot_w64(mx > m + SCORED_RESCALE_SLACK) != 0) {
      const float mn = fmaxf(m, mx);
      const float alpha = __builtin_amdgcn_exp2f(m - ((mn == -INFINITY) ? 0.f : mn));
      m = mn;
      l *= alpha;
#pragma unroll
      for (int db = 0; db < G::DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[db][r] *= alpha;
    }
    const float ms = (m == -INFINITY) ? 0.f : m;
    float rs[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      typedef __attribute__((ext_vector_type(4))) uint32_t words;
      words p;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float p0 = __builtin_amdgcn_exp2f(s[j >> 1][8 * (j & 1) + 2 * w] - ms);
        const float p1 = __builtin_amdgcn_exp2f(s[j >> 1][8 * (j & 1) + 2 * w + 1] - ms);
        rs[w & 1] += p0 + p1;
        p[w] = pack_pair(p0, p1);
      }
      const bf16x8 pf = __builtin_bit_cast(bf16x8, p);
#pragma unroll
      for (int db = 0; db < G::DB; ++db)
        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_v_frag<HD>(v_lds, voff, j, db), pf, o[db], 0, 0, 0);
    }
    l += rs[0] + rs[1];
  }
  if (!active) return;
  const float lt = l + __shfl_xor(l, 32);
  float z = 0.f;  // NaN if any of the row's sums is not finite
#pragma unroll
  for (int db = 0; db < G::DB; ++db) {
    f32x4 quads[4];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      quads[r >> 2][r & 3] = o[db][r];
      z = __builtin_fmaf(o[db][r], 0.f, z);
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
  const uint32_t koff = k_lane_off<HD>(lane), voff = v_lane_off<HD>(lane);
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
  const auto take = [&](KvTile& t) __attribute__((always_inline)) {
    if (!cur.next(c, g, F::KT, t)) t.cnt = 0;
  };
  const auto request_k = [&](const KvTile& t, int stage) __attribute__((always_inline)) {
    if (t.cnt == 0) return;
    offsets(t);
    load_eight_kib<false>(t.k, offk, mine_addr + stage * 16384);
  };
  const auto request_v = [&](const KvTile& t, int stage) __attribute__((always_inline)) {
    if (t.cnt == 0) return;
    offsets(t);
    load_eight_kib<false>(t.v, offv, mine_addr + stage * 16384 + 8192);
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
      if (!Q_IN_LDS) qf[ks] = *(const bf16x8*)(qp + ks * 16);
      else if (ks % 4 == wave) q_lds[(rb * G::KS + ks) * 64] = *(const bf16x8*)(qp + ks * 16);
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
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int kb = 0; kb < F::KB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[rb][kb][r] = 0.f;
#pragma unroll
    for (int ks = 0; ks < G::KS; ++ks)
#pragma unroll
      for (int kb = 0; kb < F::KB; ++kb) {
        const bf16x8 kf = read_k_frag<HD>(k_lds, koff, kb, ks);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
          s[rb][kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, Q_IN_LDS ? q_lds[(rb * G::KS + ks) * 64] : qf[ks], s[rb][kb], 0, 0, 0);
      }
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
#pragma unroll
      for (int kb = 0; kb < F::KB; ++kb) {
        const int at = tpos + 32 * kb + 4 * h;
        change_scores<CAP, BIAS>(sp, slope[rb], (float)(at - rr[rb].pos), s[rb][kb]);
        if (!whole) hide_scores(rr[rb].from - at, min(tpos + tcnt - 1, rr[rb].last) - at, s[rb][kb]);
      }
      float mx = s[rb][0][0];
#pragma unroll
      for (int kb = 0; kb < F::KB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; r += 2) mx = max3(mx, s[rb][kb][r], s[rb][kb][r + 1]);
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      if (__builtin_amdgcn_ballot_w64(mx > m[rb] + SCORED_RESCALE_SLACK) != 0) {
        const float mn = fmaxf(m[rb], mx);
        const float alpha = __builtin_amdgcn_exp2f(m[rb] - ((mn == -INFINITY) ? 0.f : mn));
        m[rb] = mn;
        l[rb] *= alpha;
#pragma unroll
        for (int db = 0; db < G::DB; ++db)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[rb][db][r] *= alpha;
      }
      const float ms = (m[rb] == -INFINITY) ? 0.f : m[rb];
      float rs[2] = {0.f, 0.f};
#pragma unroll
      for (int kb = 0; kb < F::KB; ++kb)
#pragma unroll
        for (int w = 0; w < 8; ++w) {
          const float p0 = __builtin_amdgcn_exp2f(s[rb][kb][2 * w] - ms), p1 = __builtin_amdgcn_exp2f(s[rb][kb][2 * w + 1] - ms);
          rs[w & 1] += p0 + p1;
          pw[rb][kb][w] = pack_pair(p0, p1);
        }
      l[rb] += rs[0] + rs[1];
    }
    // requests younger than V of this tile: K and V of the next one, K of the one after
    if (one_more && tiles[2].cnt > 0) wait_vmcnt<24>();
    else if (one_more) wait_vmcnt<16>();
    else wait_vmcnt<0>();
#pragma unroll
    for (int j = 0; j < 2 * F::KB; ++j)
#pragma unroll
      for (int db = 0; db < G::DB; ++db) {
        const bf16x8 vf = read_v_frag<HD>(v_lds, voff, j, db);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          typedef __attribute__((ext_vector_type(4))) uint32_t words;
          const uint32_t* w = &pw[rb][j >> 1][4 * (j & 1)];
          o[rb][db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, __builtin_bit_cast(bf16x8, words{w[0], w[1], w[2], w[3]}), o[rb][db], 0, 0, 0);
        }
      }
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
    store_quads<HD, true>(c, e, it, g, rb * 32 + (lane & 31), quad0 * 8 + 4 * h, acc, lsum[rb] == 0.f ? 1.f : lsum[rb]);
    const float lt1[1] = {lsum[rb]}, m1[1] = {mm[rb]};
    if (wave == 0) store_ml<1, true>(c, e, it, g, rb * 32, lane, m1, lt1);
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
    acc *= a;
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      if (s0 + k >= mg.nsplit) continue;
      const float f = __builtin_amdgcn_exp2f(ml[k].x - ms);
      l += f * ml[k].y;
      acc += f * v[k];
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
