// Attention for batches whose sequences share cells (gfx950): keys that several sequences see are read once for the rows of all.
//
//   o = sum_j softmax_j(scale q.k_j) v_j over the positions up to the row's own.
//
// The planner cuts what the batch sees into nodes: ranges of positions with the rows that see all of them through the same cells
// (a prefix that sequences share, a longer one that some of these share, what a sequence has to itself).  A work item is a tile of
// a node's rows against a piece of its keys and leaves, per row, the largest score m, the sum of weights l and the weighted sum
// of values o; a second kernel joins a row's pieces: o = sum 2^(m_s - M) o_s / sum 2^(m_s - M) l_s.
//
// Scores are in log2 units.  bf16: a weight is rounded once to bf16 for the product with V (half a step, 2^-8 of the weighted mean of
// |V|); its row's sum is of the unrounded ones, in fp32.
#include <hip/hip_runtime.h>

#include <mutex>
#include <type_traits>

#include "kernels.hpp"
#include "scored_common.hpp"
#include "shared_kernels.hpp"

namespace dk {
namespace mfma {

namespace {

template <typename T>
__device__ __forceinline__ const T* shared_desc(const SharedArgs& a, const T* p) {
  return scored_desc(p, a.in_args != 0);
}

__device__ __forceinline__ int shared_token(const SharedArgs& a, int row) { return a.gmagic ? (int)__umulhi((uint32_t)row, a.gmagic) : row; }

// The last of n ascending numbers that is not above x (the first is not), 64 of them at a time by a vector load: a round trip up to 64, two up
// to 4096.  (Descriptors in the arguments are in host memory, and every cache line of them that a compute unit takes by scalar loads
// costs about as much again: the search by scalar loads, with the lines asked for beforehand, made the merge of 64 entries 9.4 us instead
// of 5.5.)
__device__ __forceinline__ int last_not_above(const int32_t* p, int n, int x, int lane) {
  int first = 0, range = n;
  while (true) {
    const int step = (range + 63) >> 6, at = first + lane * step;
    const int v = p[min(at, n - 1)];
    const int count = __builtin_popcountll(__builtin_amdgcn_ballot_w64(at < first + range && v <= x));
    first = __builtin_amdgcn_readfirstlane(first + max(count - 1, 0) * step);
    if (step == 1) return first;
    range = min(step, n - first);
  }
}

// A work item: rows row0 .. row0 + nrows - 1 of the node against positions kv_lo .. kv_hi - 1.
struct Job {
  DkShNode nd;
  int32_t seg_end;
  int32_t row0, nrows, kv_lo, kv_hi;
  int32_t part0;  // partial row of the node's row 0; < 0: output
};
__device__ __forceinline__ Job job_of(const SharedArgs& a, int unit, int tile_rows, int lane) {
  const int at = last_not_above(shared_desc(a, a.starts), a.n_nodes, unit, lane);
  const DkShNode* nodes = shared_desc(a, a.nodes);
  Job j;
  j.nd = load_desc(nodes, at);
  const DkShNode next = load_desc(nodes, at + 1);
  j.seg_end = next.seg0;
  const int first = load_desc(shared_desc(a, a.starts), at);
  const int tile = j.nd.rows <= SHARED_FEW && tile_rows == SHARED_TILE ? SHARED_FEW : tile_rows;
  const int tiles = (j.nd.rows + tile - 1) / tile;
  const int piece = (unit - first) / tiles;
  j.row0 = (unit - first - piece * tiles) * tile;
  j.nrows = min(tile, j.nd.rows - j.row0);
  j.kv_lo = j.nd.lo + piece * j.nd.chunk;
  j.kv_hi = min(min(j.nd.lo + j.nd.keys, j.kv_lo + j.nd.chunk), j.nd.n + shared_token(a, j.row0 + j.nrows - 1) + 1);
  j.part0 = j.nd.part0 < 0 ? -1 : j.nd.part0 + piece * j.nd.rows;
  return j;
}
// Packed token (row of Q and the output) of a node's token.
__device__ __forceinline__ int packed_token(const SharedArgs& a, const DkShNode& nd, int tok) {
  return nd.n == SHARED_ALL ? shared_desc(a, a.tokens)[nd.tok0 + tok] : nd.tok0 + tok;
}

// KvCursor over the segments of a node.
template <int ROW>
struct NodeCursor {
  const DkShSeg* segs;
  int32_t si, se, p, hi;
  int32_t seg_end = 0;
  const char* k = nullptr;
  const char* v = nullptr;
  uint32_t stride = 0;

  __device__ __forceinline__ void enter_segment(const SharedArgs& a, int g) {
    DkShSeg s = load_desc(segs, si);
    while (s.pos + s.len <= p && si + 1 < se) s = load_desc(segs, ++si);
    const int32_t off = p - s.pos;
    seg_end = s.pos + s.len;
    if (s.start >= 0) {
      const int64_t byte = ((int64_t)g * a.arena_cells + s.start + off) * ROW;
      k = (const char*)a.k_arena + byte;
      v = (const char*)a.v_arena + byte;
      stride = ROW;
    } else {
      const int64_t byte = (((int64_t)~s.start + off) * a.n_kv_heads + g) * (int64_t)ROW;
      k = (const char*)a.k_new + byte;
      v = (const char*)a.v_new + byte;
      stride = (uint32_t)a.n_kv_heads * ROW;
    }
  }
  __device__ __forceinline__ bool next(const SharedArgs& a, int g, int kt, KvTile& t) {
    if (p >= hi) return false;
    if (p >= seg_end) enter_segment(a, g);
    t.cnt = min(kt, min(seg_end, hi) - p);
    t.k = k;
    t.v = v;
    t.stride = stride;
    t.pos = p;
    t.once = 0;
    p += t.cnt;
    const uint32_t adv = (uint32_t)t.cnt * stride;
    k += adv;
    v += adv;
    return true;
  }
};
template <int ROW>
__device__ __forceinline__ NodeCursor<ROW> cursor_of(const SharedArgs& a, const Job& j, int lo, int hi) {
  return {shared_desc(a, a.segs), j.nd.seg0, j.seg_end, lo, hi};
}

// Where a row's results go: quad i of a lane holds depths depth0 + 8 i .. + 3.
template <int HD, int NQ>
__device__ __forceinline__ void store_sums(const SharedArgs& a, const Job& j, int g, int rl, int depth0, const f32x4 (&o)[NQ], float l) {
  if (rl >= j.nrows) return;
  const int row = j.row0 + rl;
  if (j.part0 >= 0) {
    float* p = a.parts + ((int64_t)(j.part0 + row) * a.n_kv_heads + g) * HD + depth0;
#pragma unroll
    for (int i = 0; i < NQ; ++i) *(f32x4*)(p + 8 * i) = o[i];
    return;
  }
  const int tok = shared_token(a, row);
  const float inv = 1.f / l;
  __bf16* dst = (__bf16*)a.out + ((int64_t)packed_token(a, j.nd, tok) * a.n_q_heads + g * a.group + row - tok * a.group) * HD + depth0;
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    bf16x4 v;
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = (__bf16)(o[i][u] * inv);
    *(bf16x4*)(dst + 8 * i) = v;
  }
}
__device__ __forceinline__ void store_maximum(const SharedArgs& a, const Job& j, int g, int rl, float m, float l) {
  if (rl >= j.nrows) return;
  const int row = j.row0 + rl;
  if (j.part0 >= 0) {
    *(float2*)(a.parts_ml + ((int64_t)(j.part0 + row) * a.n_kv_heads + g) * 2) = make_float2(m, l);
  } else if (a.lse) {
    const int tok = shared_token(a, row);
    a.lse[(int64_t)packed_token(a, j.nd, tok) * a.n_q_heads + g * a.group + row - tok * a.group] = (m + log2f(l)) * 0.6931471805599453f;
  }
}

// redo_rows for these items: rows rl0 .. rl0 + 31, depth block db, again without the non-finite elements of V, which are then put back
// by the first position of each kind.  Of the block's four quads of depths, `quads` from quad0 on are this wavefront's to store.
template <int HD>
__device__ __forceinline__ void redo_shared(const SharedArgs& a, const ScoreParams& sp, const Job& j, int g, int rl0, uint32_t bad, float m, float l,
                                            int lane, int db, int quad0, int quads) {
  typedef Geo<HD> G;
  asm volatile("" : "+v"(lane));
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // after the ordinary store of the same rows
  const int col = lane & 31, h = lane >> 5;
  const int row = j.row0 + min(rl0 + col, j.nrows - 1);
  const int tok = shared_token(a, row);
  const int limit = j.nd.n + tok;
  const int64_t orow = (int64_t)packed_token(a, j.nd, tok) * a.n_q_heads + g * a.group + row - tok * a.group;
  const float ms = m == -INFINITY ? 0.f : m;
  bf16x8 qf[G::KS];
#pragma unroll
  for (int ks = 0; ks < G::KS; ++ks) qf[ks] = signed_q(*(const bf16x8*)((const __bf16*)a.q + orow * HD + ks * 16 + 8 * h), sp.flip);
  f32x16 o;
  NonFinite nf;
#pragma unroll
  for (int r = 0; r < 16; ++r) o[r] = 0.f;
  NodeCursor<G::ROW> cur = cursor_of<G::ROW>(a, j, j.kv_lo, j.kv_hi);
  KvTile t;
  while (cur.next(a, g, 32, t)) {
    const char* kp = t.k + (uint32_t)min(col, t.cnt - 1) * t.stride + 16 * h;
    f32x16 s;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
    for (int ks = 0; ks < G::KS; ++ks) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8*)(kp + 32 * ks), qf[ks], s, 0, 0, 0);
    const int lim = min(t.cnt - 1, limit - t.pos) - 4 * h;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      bf16x8 p, v;
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const int key = 16 * i + 8 * (x >> 2) + 4 * h + (x & 3);
        const int at = min(key, t.cnt - 1);
        const uint32_t bits = *(const uint16_t*)(t.v + (uint32_t)at * t.stride + 64 * db + 2 * col);
        const bool odd = nf.see(bits << 16, t.pos + at);
        v[x] = __builtin_bit_cast(__bf16, (uint16_t)(odd ? 0u : bits));
        const bool hidden = 16 * i + 8 * (x >> 2) + (x & 3) > lim;
        p[x] = (__bf16)(hidden ? 0.f : __builtin_amdgcn_exp2f(__builtin_fmaf(s[8 * i + x], sp.c, -ms)));
      }
      o = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p, o, 0, 0, 0);
    }
  }
  nf.merge_lanes(32);
  const bool mine = (bad >> col & 1) != 0 && rl0 + col < j.nrows && l == l;
  const float inv = 1.f / l;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f32x4 x;
#pragma unroll
    for (int r = 0; r < 4; ++r) x[r] = nf.of_lane(8 * i + 4 * h + r).apply(o[4 * i + r], limit);
    if (!mine || i < quad0 || i >= quad0 + quads) continue;
    const int depth = 32 * db + 8 * i + 4 * h;
    if (j.part0 >= 0) {
      *(f32x4*)(a.parts + ((int64_t)(j.part0 + row) * a.n_kv_heads + g) * HD + depth) = x;
    } else {
      bf16x4 y;
#pragma unroll
      for (int r = 0; r < 4; ++r) y[r] = (__bf16)(x[r] * inv);
      *(bf16x4*)((__bf16*)a.out + orow * HD + depth) = y;
    }
  }
}

template <int HD>
struct SharedGeo {
  // tiles that the four wavefronts share: 64 keys, K in two stages, V in three
  static constexpr int ROWS_KT = 64;
  static constexpr int TILE_BYTES = ROWS_KT * Geo<HD>::ROW;
  static constexpr int K_STAGES = 2, V_STAGES = 3;
  static constexpr int V_OFFSET = K_STAGES * TILE_BYTES;
  static constexpr int LOADS = TILE_BYTES / 1024 / 4;  // 1 KiB requests per wavefront for a tile's K, as many for its V
  // a wavefront's own: 8 KiB of K, 8 KiB of V
  static constexpr int KT = 8192 / Geo<HD>::ROW;
  static constexpr int KB = KT / 32;
  static constexpr int WAVE_BYTES = 2 * 8192;
  static constexpr int Q_OFFSET = 4 * WAVE_BYTES;      // two row blocks keep their Q here; then maxima and sums
  static constexpr int LDS_BYTES = V_OFFSET + V_STAGES * TILE_BYTES > Q_OFFSET + 2 * Geo<HD>::KS * 1024 ? V_OFFSET + V_STAGES * TILE_BYTES
                                                                                                  : Q_OFFSET + 2 * Geo<HD>::KS * 1024;
  static_assert(LDS_BYTES <= 81920, "two workgroups to a compute unit");
};

// A tile of up to 128 rows: each wavefront has 32 of them, the keys go through LDS once for all, and the products of tile t + 1 stand among
// the instructions that turn those of tile t into weights, as in scored_rows_kernel.  Bound by the vector unit and the matrix pipe in turn:
// 2.2 to 2.6 us for 64 keys of 128-wide heads with two workgroups to a compute unit.  16 turns of 64 to 512 tokens behind one preamble, 326
// GFLOP: calls of 383 to 390 us, 840 to 850 TFLOP/s; one after the other for 25 ms, in a trace, 392 to 456, 411 on average.  32 drafts of up to nine tokens
// behind 30 000 keys, 72 GFLOP: 102 to 135 in such a trace, 119 on average.
// (128 rows rather than 256: a second workgroup's softmax runs beside the first one's products, and a group of a few sessions fills a tile.)
template <int HD>
__device__ __forceinline__ void many_rows(const SharedArgs& a, const ScoreParams& sp, const Job& j, int g, char* smem, int lane, int wave) {
  typedef Geo<HD> G;
  typedef SharedGeo<HD> B;
  const int h = lane >> 5;
  const uint32_t koff = k_lane_off<HD>(lane), voff = v_lane_off<HD>(lane);
  const bool active = wave * 32 < j.nrows;
  const int row = j.row0 + min(wave * 32 + (lane & 31), j.nrows - 1);
  const int tok = shared_token(a, row);
  const RowRange rr{j.nd.n + tok, 0, j.nd.n + tok};
  const int all_last = j.nd.n + shared_token(a, j.row0 + min(wave * 32, j.nrows - 1));
  const int any_last = j.nd.n + shared_token(a, j.row0 + min(wave * 32 + 31, j.nrows - 1));
  bf16x8 qf[G::KS];
  {
    const __bf16* qp = (const __bf16*)a.q + ((int64_t)packed_token(a, j.nd, tok) * a.n_q_heads + g * a.group + row - tok * a.group) * HD + 8 * h;
#pragma unroll
    for (int ks = 0; ks < G::KS; ++ks) qf[ks] = signed_q(*(const bf16x8*)(qp + ks * 16), sp.flip);
  }
  NodeCursor<G::ROW> cur = cursor_of<G::ROW>(a, j, j.kv_lo, j.kv_hi);
  int cnt[3], pos[3];  // of tiles t, t + 1 and t + 2 (0 keys: none)
  int v_wr = 0;
  KvTile t;
  const auto request = [&](int slot, int k_stage) __attribute__((always_inline)) {
    cnt[slot] = 0;
    if (!cur.next(a, g, B::ROWS_KT, t)) return;
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

  f32x16 o[1][G::DB];
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int db = 0; db < G::DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[0][db][r] = 0.f;
  const auto sees = [&](int slot) { return active && cnt[slot] > 0 && pos[slot] <= any_last; };

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
    const bool whole = tcnt == B::ROWS_KT && tpos + B::ROWS_KT - 1 <= all_last;
    uint32_t pw[1][2][8];
    const auto rescale = [&](float alpha) {
#pragma unroll
      for (int db = 0; db < G::DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[0][db][r] *= alpha;
    };
    // (the next tile's products are computed whether a row sees it or not)
    constexpr int N = 2 * G::KS, AHEAD = 4;
    bf16x8 kf[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) kf[i] = read_k_frag<HD>(k_lds, koff, i % 2, i / 2);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) next[0][kb][r] = 0.f;
    weigh<false, false, 2>(sp, rr, 0.f, tpos, tcnt, h, whole, s[0], m, l, pw[0], rescale, [&](int i) __attribute__((always_inline)) {
      if (16 / N * (i / (16 / N)) != i) return;  // (64-wide heads: every other time)
      const int n = i / (16 / N);
      __builtin_amdgcn_sched_barrier(0);
      next[0][n % 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[n % AHEAD], qf[n / 2], next[0][n % 2], 0, 0, 0);
      if (n + AHEAD < N) kf[n % AHEAD] = read_k_frag<HD>(k_lds, koff, (n + AHEAD) % 2, (n + AHEAD) / 2);
      __builtin_amdgcn_sched_barrier(0);
    });
    ValueFrags<HD, 4> values;
    values.first(v_lds, voff);
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
    store_sums<HD>(a, j, g, wave * 32 + (lane & 31), db * 32 + 4 * h, quads, lt);
  }
  if (lane < 32) store_maximum(a, j, g, wave * 32 + lane, m, lt);
  const uint32_t bad = bad_rows(z != 0.f);
  if (bad != 0) {
#pragma unroll 1
    for (int db = 0; db < G::DB; ++db) redo_shared<HD>(a, sp, j, g, wave * 32, bad, m, lt, lane, db, 0, 4);
  }
}

// A tile of up to 32 RB rows: each wavefront walks a quarter of the keys through LDS of its own, with no barrier until their
// sums are joined.  K of tile t + 1 is requested as soon as K of tile t has been read, V likewise.  Bound by HBM where the keys come from
// there: 16 requests of eight beams, 328 MB, 47 to 49 us on average (least 44), 6.7 to 7 TB/s; by latency where they are few: an item without its keys takes
// 5.5 us (descriptors 1, first requests and Q 1.5, four wavefronts' sums 1.5), four beams behind 3000 keys 7.3 in all.  One stage of K
// and V for a wavefront, and not two as in scored_few_kernel, so that two workgroups fit a compute unit: one's start and end
// are covered by the other.
template <int HD, int RB>
__device__ __forceinline__ void few_rows(const SharedArgs& a, const ScoreParams& sp, const Job& j, int g, char* smem, int lane, int wave) {
  typedef Geo<HD> G;
  typedef SharedGeo<HD> F;
  const int h = lane >> 5;
  uint32_t koff = k_lane_off<HD>(lane), voff = v_lane_off<HD>(lane);
  char* mine = smem + wave * F::WAVE_BYTES;
  const uint32_t mine_addr = (uint32_t)(uintptr_t)(lds_void_ptr)mine;
  const int blocks = (j.kv_hi - j.kv_lo + F::KT - 1) / F::KT;
  const int per = (blocks + 3) / 4 * F::KT;
  const int lo = min(j.kv_hi, j.kv_lo + wave * per), hi = min(j.kv_hi, lo + per);
  NodeCursor<G::ROW> cur = cursor_of<G::ROW>(a, j, lo, hi);
  KvTile tile, next;
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
  const auto request_k = [&](const KvTile& t) __attribute__((always_inline)) {
    if (t.cnt == 0) return;
    offsets(t);
    load_eight_kib<false>(t.k, offk, mine_addr);
  };
  const auto request_v = [&](const KvTile& t) __attribute__((always_inline)) {
    if (t.cnt == 0) return;
    offsets(t);
    load_eight_kib<false>(t.v, offv, mine_addr + 8192);
  };
  const auto take = [&](KvTile& t) __attribute__((always_inline)) {
    if (!cur.next(a, g, F::KT, t)) t.cnt = 0;
  };
  take(tile);
  request_k(tile);
  request_v(tile);

  RowRange rr[RB];
  int all_last[RB];
  constexpr bool Q_IN_LDS = RB > 1;
  bf16x8 qf[G::KS];
  bf16x8* q_lds = (bf16x8*)(smem + F::Q_OFFSET) + lane;  // [row block][depth step][lane]
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int row = j.row0 + min(rb * 32 + (lane & 31), j.nrows - 1);
    const int tok = shared_token(a, row);
    rr[rb] = {j.nd.n + tok, 0, j.nd.n + tok};
    all_last[rb] = j.nd.n + shared_token(a, j.row0 + min(rb * 32, j.nrows - 1));
    const __bf16* qp = (const __bf16*)a.q + ((int64_t)packed_token(a, j.nd, tok) * a.n_q_heads + g * a.group + row - tok * a.group) * HD + 8 * h;
#pragma unroll
    for (int ks = 0; ks < G::KS; ++ks) {
      if (!Q_IN_LDS) qf[ks] = signed_q(*(const bf16x8*)(qp + ks * 16), sp.flip);
      else if (ks % 4 == wave) q_lds[(rb * G::KS + ks) * 64] = signed_q(*(const bf16x8*)(qp + ks * 16), sp.flip);
    }
  }
  if constexpr (Q_IN_LDS) {
    __syncthreads();
  } else {
#pragma unroll
    for (int ks = 0; ks < G::KS; ++ks) asm volatile("" ::"v"(qf[ks]));
  }

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
  const char* k_lds = mine;
  const char* v_lds = mine + 8192;
  while (tile.cnt > 0) {
    wait_vmcnt<8>();  // younger than K of this tile: its V
    f32x16 s[RB][F::KB];
    // (computed anew from here on in every step: kept across steps, the addresses of the fragments cost more registers than there are)
    if constexpr (RB > 1) asm volatile("" : "+v"(koff), "+v"(voff));
    score_products<HD, F::KB, RB, 4>(k_lds, koff, s, [&](int rb, int ks) { return Q_IN_LDS ? q_lds[(rb * G::KS + ks) * 64] : qf[ks]; });
    // (the products are waited for here, on this side of the branches that follow)
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int kb = 0; kb < F::KB; ++kb) asm volatile("s_nop %1" : "+v"(s[rb][kb]) : "n"(rb == RB - 1 && kb == F::KB - 1 ? 11 : 0));
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // K has been read
    take(next);
    request_k(next);
    uint32_t pw[RB][F::KB][8];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const bool whole = tile.cnt == F::KT && tile.pos + F::KT - 1 <= all_last[rb];
      weigh<false, false, F::KB>(sp, rr[rb], 0.f, tile.pos, tile.cnt, h, whole, s[rb], m[rb], l[rb], pw[rb], [&](float alpha) {
#pragma unroll
        for (int db = 0; db < G::DB; ++db)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[rb][db][r] *= alpha;
      }, [](int) {});
    }
    if (next.cnt > 0) wait_vmcnt<8>();  // younger than V of this tile: K of the next
    else wait_vmcnt<0>();
    ValueFrags<HD, 4> values;
    values.first(v_lds, voff);
    values.template products<F::KB, RB>(v_lds, voff, pw, o);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // V has been read
    request_v(next);
    tile = next;
  }

  // Quad (db, r4) of a lane is depths 32 db + 8 r4 + 4 h .. + 3 of its row; wavefront w stores quads w NQ .. of each row.
  constexpr int NQ = G::DB;  // of 4 DB quads
  f32x4* xo = (f32x4*)smem;  // [wave][quad][lane]
  float2* xml = (float2*)(smem + F::Q_OFFSET);
  const int quad0 = wave * NQ;
#pragma unroll 1
  for (int rb = 0; rb < RB; ++rb) {
    if (rb * 32 >= j.nrows) break;
    const float lt0 = rb == 0 ? l[0] : l[RB - 1], mine_m = rb == 0 ? m[0] : m[RB - 1];
    const float lt = lt0 + __shfl_xor(lt0, 32);
    __syncthreads();
    if (lane < 32) xml[wave * 32 + lane] = make_float2(mine_m, lt);
#pragma unroll
    for (int db = 0; db < G::DB; ++db)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        f32x4 x;
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] = rb == 0 ? o[0][db][4 * r4 + r] : o[RB - 1][db][4 * r4 + r];
        xo[(wave * 4 * G::DB + db * 4 + r4) * 64 + lane] = x;
      }
    __syncthreads();
    float2 ml[4];
    float mm = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      ml[w] = xml[w * 32 + (lane & 31)];
      mm = fmaxf(mm, ml[w].x);
    }
    const float ms = (mm == -INFINITY) ? 0.f : mm;
    float lsum = 0.f;
    f32x4 acc[NQ];
#pragma unroll
    for (int i = 0; i < NQ; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = __builtin_amdgcn_exp2f(ml[w].x - ms);
      lsum += f * ml[w].y;
#pragma unroll
      for (int i = 0; i < NQ; ++i) acc[i] += f * xo[(w * 4 * G::DB + quad0 + i) * 64 + lane];
    }
    store_sums<HD>(a, j, g, rb * 32 + (lane & 31), quad0 * 8 + 4 * h, acc, lsum);
    if (wave == 0 && lane < 32) store_maximum(a, j, g, rb * 32 + lane, mm, lsum);
    float z = 0.f;
#pragma unroll
    for (int i = 0; i < NQ; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) z = __builtin_fmaf(acc[i][r], 0.f, z);
    const uint32_t bad = bad_rows(z != 0.f);
    if (bad != 0) redo_shared<HD>(a, sp, j, g, rb * 32, bad, mm, lsum, lane, quad0 / 4, quad0 % 4, NQ);
  }
}

}  // namespace

// bf16.  Workgroup w: work item w / n_kv_heads, KV head w % n_kv_heads, so that with eight KV heads each XCD reads the keys of one (runs of
// 4 to 64 items of one order on an XCD, the tiles of the same keys side by side, took as long or longer); two workgroups to a compute unit.
template <int HD>
__global__ __launch_bounds__(256, 2) void shared_attend_kernel(SharedBlob blob, SharedArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  (void)blob;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = blockIdx.x % a.n_kv_heads;
  const Job j = job_of(a, blockIdx.x / a.n_kv_heads, SHARED_TILE, lane);
  if (j.kv_lo >= j.kv_hi) return;  // a piece behind what the tile's rows see
  ScoreParams sp;
  sp.c = a.c;
  sp.flip = a.flip;
  if (j.nrows <= 32 && j.nd.rows <= SHARED_FEW) few_rows<HD, 1>(a, sp, j, g, smem, lane, wave);
  else if (j.nd.rows <= SHARED_FEW) few_rows<HD, 2>(a, sp, j, g, smem, lane, wave);
  else many_rows<HD>(a, sp, j, g, smem, lane, wave);
}

// Joins the partial rows of every row.  HD / 4 lanes take a row's depths; `spread` lane groups of a workgroup share its pieces.  Bound by
// latency, a chain of round trips: block, node and sources, partial rows (the first from the arguments, which are in host memory).  On average
// 4.9 us for four rows of 25 pieces (least 4.0), 6.7 to 7.2 for 64 to 128 beams, 10.6 for 32 drafts of up to nine tokens (least 9.1).
template <int HD, bool F32>
__global__ __launch_bounds__(256) void shared_merge_kernel(SharedBlob blob, SharedArgs a, SharedMergeArgs ma) {
  constexpr int LANES = HD / 4, GROUPS = 256 / LANES, AHEAD = 4;
  __shared__ f32x4 xo[256];
  __shared__ float2 xml[GROUPS];
  (void)blob;
  const int g = blockIdx.x % a.n_kv_heads, block = blockIdx.x / a.n_kv_heads;
  const int32_t *blocks = scored_desc(ma.blocks, ma.in_args != 0), *src0 = scored_desc(ma.src0, ma.in_args != 0);
  const DkShSource* sources = scored_desc(ma.sources, ma.in_args != 0);
  const int at = last_not_above(blocks, a.n_nodes, block, threadIdx.x & 63);
  const DkShNode nd = load_desc(scored_desc(ma.nodes, ma.nodes_in_args != 0), at);
  const int src_begin = load_desc(src0, at), src_end = load_desc(src0, at + 1);
  const int lane = threadIdx.x % LANES, grp = threadIdx.x / LANES;
  const int first = grp % ma.spread;
  const int row = (block - load_desc(blocks, at)) * (GROUPS / ma.spread) + grp / ma.spread;
  const bool there = row < nd.rows;
  const int r = min(row, nd.rows - 1);
  const int tok = shared_token(a, r);
  // of its own range, the pieces that some row of its tile sees
  const int tile_last = shared_token(a, min(nd.rows, (r / ma.tile_rows + 1) * ma.tile_rows) - 1);
  const int own = (min(nd.keys, nd.n + 1 - nd.lo + tile_last) + nd.chunk - 1) / nd.chunk;

  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  float l = 0.f, m = -INFINITY;
  const auto add = [&](float wm, float wl, const f32x4& v) __attribute__((always_inline)) {
    const float mn = fmaxf(m, wm);
    const float ms = (mn == -INFINITY) ? 0.f : mn;
    const float b = __builtin_amdgcn_exp2f(m - ms), f = __builtin_amdgcn_exp2f(wm - ms);
    m = mn;
    l = l * b + f * wl;
    acc = acc * piece_weight(b) + piece_weight(f) * v;
  };
  int skip = first;  // pieces until this lane group's next one
  const auto range = [&](int part0, int step, int pieces) __attribute__((always_inline)) {
    int s0 = skip;
    for (; s0 < pieces; s0 += ma.spread * AHEAD) {
      f32x4 v[AHEAD];
      float2 w[AHEAD];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {  // (a piece past the end repeats the last one and is left out below)
        const int64_t prow = ((int64_t)part0 + r + (int64_t)min(s0 + k * ma.spread, pieces - 1) * step) * a.n_kv_heads + g;
        w[k] = *(const float2*)(a.parts_ml + prow * 2);
        v[k] = *(const f32x4*)(a.parts + prow * HD + lane * 4);
      }
#pragma unroll
      for (int k = 0; k < AHEAD; ++k)
        if (s0 + k * ma.spread < pieces) add(w[k].x, w[k].y, v[k]);
    }
    const int done = pieces > skip ? (pieces - skip + ma.spread - 1) / ma.spread : 0;
    skip = skip + done * ma.spread - pieces;
  };
  for (int s = src_begin; s < src_end; ++s) {
    const DkShSource src = load_desc(sources, s);
    range(src.part0, src.step, src.pieces);
  }
  range(nd.part0, nd.rows, own);
  if (ma.spread > 1) {
    xo[threadIdx.x] = acc;
    if (lane == 0) xml[grp] = make_float2(m, l);
    __syncthreads();
    if (first == 0)
      for (int k = 1; k < ma.spread; ++k) add(xml[grp + k].x, xml[grp + k].y, xo[threadIdx.x + k * LANES]);
  }
  if (first != 0 || !there) return;
  const int64_t orow = (int64_t)(nd.tok0 + tok) * a.n_q_heads + g * a.group + r - tok * a.group;
  const float inv = 1.f / l;
  if constexpr (F32) {
    *(f32x4*)((float*)a.out + orow * HD + lane * 4) = acc * inv;
  } else {
    bf16x4 y;
#pragma unroll
    for (int u = 0; u < 4; ++u) y[u] = (__bf16)(acc[u] * inv);
    *(bf16x4*)((__bf16*)a.out + orow * HD + lane * 4) = y;
  }
  if (a.lse && lane == 0) a.lse[orow] = (m + log2f(l)) * 0.6931471805599453f;
}

// A piece of descriptors that do not fit a kernel's arguments, on its way to the workspace in the arguments of a launch of its own: 1.1 to
// 1.9 us of the device and 2.5 of the host, less than a copy from pinned memory and its event, and it needs neither.
__global__ __launch_bounds__(256) void shared_carry_kernel(SharedCarry piece, uint32_t* to, int32_t words) {
  typedef const __attribute__((address_space(4))) uint32_t* const_u32_ptr;
  const_u32_ptr from = (const_u32_ptr)__builtin_amdgcn_kernarg_segment_ptr();
  (void)piece;
  for (int i = threadIdx.x; i < words; i += 256) to[i] = from[i];
}

// fp32: 8 wavefronts split the keys of an item of 16 RB rows, as in attend_f32_kernel (operands straight from memory, products of
// 16 x 16 x 4, states joined through LDS); see there for the layout.  Bound by the fp32 matrix pipe, 1.7 us for 64 keys of 32 rows of 128, and
// by its start: 2.4 us a step with two wavefronts to a SIMD, and 8 without keys (the second wavefront of a SIMD gets to its keys 4 us after
// the first; wave priorities for what is not a product changed nothing).  Two groups of 6 to 12 samples, 2.1 GFLOP: 38 us.
namespace {
constexpr int SF_WAVES = 8, SF_KT = 16;
constexpr float SF_SLACK = 8.f;
template <int HD, int RB>
struct SharedF32Geo {
  static constexpr int ROW = 4 * HD, NI = HD / 16, NU = HD / 64, QUADS = RB * NI;
  static constexpr int ML_OFFSET = SF_WAVES * QUADS * 64 * 16;
  static constexpr int LDS_BYTES = ML_OFFSET + SF_WAVES * RB * 16 * 8;
};

template <int HD>
__device__ __forceinline__ void redo_shared_f32(const SharedArgs& a, const Job& j, int g, int rl0, uint32_t bad, float m, float l, int lane, int u, int r) {
  constexpr int ROW = 4 * HD, NI = HD / 16;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // after the ordinary store of the same rows
  const int col = lane & 15, h = lane >> 4;
  const int row = j.row0 + min(rl0 + col, j.nrows - 1);
  const int tok = shared_token(a, row);
  const int limit = j.nd.n + tok;
  const int64_t orow = (int64_t)packed_token(a, j.nd, tok) * a.n_q_heads + g * a.group + row - tok * a.group;
  const float ms = m == -INFINITY ? 0.f : m;
  f32x4 qf[NI], o[4];
  NonFinite nf[4];
#pragma unroll
  for (int i = 0; i < NI; ++i) qf[i] = *(const f32x4*)((const float*)a.q + orow * HD + 16 * i + 4 * h);
#pragma unroll
  for (int k = 0; k < 4; ++k) o[k] = f32x4{0.f, 0.f, 0.f, 0.f};
  NodeCursor<ROW> cur = cursor_of<ROW>(a, j, j.kv_lo, j.kv_hi);
  KvTile t;
  while (cur.next(a, g, SF_KT, t)) {
    const char* kp = t.k + (uint32_t)min(col, t.cnt - 1) * t.stride + 16 * h;
    f32x4 s[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const f32x4 kf = *(const f32x4*)(kp + 64 * i);
#pragma unroll
      for (int k = 0; k < 4; ++k) s[k & 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[k], qf[i][k], s[k & 1], 0, 0, 0);
    }
    const int lim = min(t.cnt - 1, limit - t.pos) - 4 * h;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int at = min(4 * h + k, t.cnt - 1);
      const f32x4 vf = *(const f32x4*)(t.v + (uint32_t)at * t.stride + 16 * col + 256 * u);
      const float p = k > lim ? 0.f : __builtin_amdgcn_exp2f(__builtin_fmaf(s[0][k] + s[1][k], a.c, -ms));
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const bool odd = nf[x].see(__float_as_uint(vf[x]), t.pos + at);
        o[x] = __builtin_amdgcn_mfma_f32_16x16x4f32(odd ? 0.f : vf[x], p, o[x], 0, 0, 0);
      }
    }
  }
  f32x4 y;
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    nf[x].merge_lanes(16);
    nf[x].merge_lanes(32);
    const float sum = r == 0 ? o[x][0] : r == 1 ? o[x][1] : r == 2 ? o[x][2] : o[x][3];
    y[x] = nf[x].of_lane(4 * h + r).apply(sum, limit);
  }
  if ((bad >> col & 1) == 0 || rl0 + col >= j.nrows || l != l) return;
  const int depth = 64 * u + 4 * (4 * h + r);
  if (j.part0 >= 0) *(f32x4*)(a.parts + ((int64_t)(j.part0 + row) * a.n_kv_heads + g) * HD + depth) = y;
  else *(f32x4*)((float*)a.out + orow * HD + depth) = y * (1.f / l);
}
}  // namespace

template <int HD, int RB>
__global__ __launch_bounds__(64 * SF_WAVES, 2) void shared_attend_f32_kernel(SharedBlob blob, SharedArgs a) {
  typedef SharedF32Geo<HD, RB> G;
  constexpr int NI = G::NI, NU = G::NU;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  (void)blob;
  const int g = blockIdx.x % a.n_kv_heads;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, h = lane >> 4;
  f32x4* xo = (f32x4*)smem;                      // [wave][quad][lane]
  float2* xml = (float2*)(smem + G::ML_OFFSET);  // [wave][row]: running maximum, weight sum
  const Job j = job_of(a, blockIdx.x / a.n_kv_heads, 16 * RB, lane);
  if (j.kv_lo >= j.kv_hi) return;
  const int min_limit = j.nd.n + shared_token(a, j.row0);
  f32x4 qf[RB][NI];
  int limit[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int row = j.row0 + min(rb * 16 + col, j.nrows - 1);
    const int tok = shared_token(a, row);
    limit[rb] = j.nd.n + tok;
    const float* qp = (const float*)a.q + ((int64_t)packed_token(a, j.nd, tok) * a.n_q_heads + g * a.group + row - tok * a.group) * HD + 4 * h;
#pragma unroll
    for (int i = 0; i < NI; ++i) qf[rb][i] = *(const f32x4*)(qp + 16 * i);
  }
  // this wavefront's share of the item's keys
  const int blocks = (j.kv_hi - j.kv_lo + SF_KT - 1) / SF_KT;
  const int per = (blocks + SF_WAVES - 1) / SF_WAVES * SF_KT;
  const int lo = min(j.kv_hi, j.kv_lo + wave * per);
  NodeCursor<G::ROW> cur = cursor_of<G::ROW>(a, j, lo, min(j.kv_hi, lo + per));
  KvTile t;
  f32x4 kf[NI], vf[4][NU];
  // rows past the end of a ragged block re-read the last valid one; their scores are masked
  const auto load_k = [&]() __attribute__((always_inline)) {
    const char* p = t.k + (uint32_t)min(col, t.cnt - 1) * t.stride + 16 * h;
#pragma unroll
    for (int i = 0; i < NI; ++i) kf[i] = *(const f32x4*)(p + 64 * i);
  };
  const auto load_v = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const char* p = t.v + (uint32_t)min(4 * h + r, t.cnt - 1) * t.stride + 16 * col;
#pragma unroll
      for (int u = 0; u < NU; ++u) vf[r][u] = *(const f32x4*)(p + 256 * u);
    }
  };
  bool have = cur.next(a, g, SF_KT, t);
  if (have) load_k();
  f32x4 o[RB][NI];
  float m[RB], l[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    m[rb] = -INFINITY;
    l[rb] = 0.f;
#pragma unroll
    for (int b = 0; b < NI; ++b) o[rb][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  while (have) {
    const int cnt = t.cnt, pos = t.pos;
    load_v();
    __builtin_amdgcn_sched_barrier(0);
    f32x4 s[RB][2];  // (two chains per score: shorter ones round less)
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) s[rb][0] = s[rb][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) s[rb][k & 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[i][k], qf[rb][i][k], s[rb][k & 1], 0, 0, 0);
    have = cur.next(a, g, SF_KT, t);
    load_k();  // (the same keys again where there are no more: a load that may not have been made is waited for at once)
    __builtin_amdgcn_sched_barrier(0);
    bool grow = false;
    float mx[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      s[rb][0] = (s[rb][0] + s[rb][1]) * a.c;
      if (cnt < SF_KT || pos + SF_KT - 1 > min_limit) {
        const int lim = min(cnt - 1, limit[rb] - pos) - 4 * h;
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (r > lim) s[rb][0][r] = -INFINITY;
      }
      mx[rb] = fmaxf(fmaxf(s[rb][0][0], s[rb][0][1]), fmaxf(s[rb][0][2], s[rb][0][3]));
      grow |= mx[rb] > m[rb] + SF_SLACK;
    }
    if (__builtin_amdgcn_ballot_w64(grow) != 0) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        float v = fmaxf(mx[rb], __shfl_xor(mx[rb], 16));
        v = fmaxf(v, __shfl_xor(v, 32));
        const float mn = fmaxf(m[rb], v);
        const float alpha = __builtin_amdgcn_exp2f(m[rb] - ((mn == -INFINITY) ? 0.f : mn));
        m[rb] = mn;
        l[rb] *= alpha;
#pragma unroll
        for (int b = 0; b < NI; ++b) o[rb][b] *= alpha;
      }
    }
    f32x4 p[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const float ms = (m[rb] == -INFINITY) ? 0.f : m[rb];  // no key seen yet: keep the arithmetic finite
#pragma unroll
      for (int r = 0; r < 4; ++r) p[rb][r] = __builtin_amdgcn_exp2f(s[rb][0][r] - ms);
      l[rb] += (p[rb][0] + p[rb][1]) + (p[rb][2] + p[rb][3]);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int rb = 0; rb < RB; ++rb)
            o[rb][4 * u + k] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[r][u][k], p[rb][r], o[rb][4 * u + k], 0, 0, 0);
  }
  // quad (rb, u, r) of a lane is depths 64 u + 4 (4 h + r) .. + 3 of row rb * 16 + col
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    float lt = l[rb] + __shfl_xor(l[rb], 16);
    lt += __shfl_xor(lt, 32);
    if (lane < 16) xml[(wave * RB + rb) * 16 + lane] = make_float2(m[rb], lt);
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        xo[((wave * RB + rb) * NI + u * 4 + r) * 64 + lane] = f32x4{o[rb][4 * u][r], o[rb][4 * u + 1][r], o[rb][4 * u + 2][r], o[rb][4 * u + 3][r]};
  }
  __syncthreads();
  for (int quad = wave; quad < G::QUADS; quad += SF_WAVES) {
    const int rb = quad / NI, u = (quad % NI) >> 2, r = quad & 3;
    const int rl = rb * 16 + col;
    float2 ml[SF_WAVES];
    float mm = -INFINITY;
#pragma unroll
    for (int w = 0; w < SF_WAVES; ++w) {
      ml[w] = xml[(w * RB + rb) * 16 + col];
      mm = fmaxf(mm, ml[w].x);
    }
    const float ms = (mm == -INFINITY) ? 0.f : mm;
    float lsum = 0.f;
    f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < SF_WAVES; ++w) {
      const float f = __builtin_amdgcn_exp2f(ml[w].x - ms);
      lsum += f * ml[w].y;
      acc += f * xo[(w * G::QUADS + quad) * 64 + lane];
    }
    const bool finite = acc[0] * 0.f + acc[1] * 0.f + acc[2] * 0.f + acc[3] * 0.f == 0.f;
    uint64_t bad = __builtin_amdgcn_ballot_w64(!finite && rl < j.nrows);
    const int depth = 64 * u + 4 * (4 * h + r);
    if (rl < j.nrows) {
      const int row = j.row0 + rl;
      if (j.part0 >= 0) {
        *(f32x4*)(a.parts + ((int64_t)(j.part0 + row) * a.n_kv_heads + g) * HD + depth) = acc;
      } else {
        const int tok = shared_token(a, row);
        *(f32x4*)((float*)a.out + ((int64_t)packed_token(a, j.nd, tok) * a.n_q_heads + g * a.group + row - tok * a.group) * HD + depth) = acc * (1.f / lsum);
      }
      if (u == 0 && r == 0 && h == 0) store_maximum(a, j, g, rl, mm, lsum);
    }
    if (bad != 0) {
      bad |= bad >> 32;
      redo_shared_f32<HD>(a, j, g, rb * 16, (uint32_t)(bad | bad >> 16) & 0xffffu, mm, lsum, lane, u, r);
    }
  }
}

namespace {

template <typename K>
hipError_t allow_lds(K kernel, int bytes) {
  return hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

template <int HD>
hipError_t launch_items(const SharedBlob& blob, const SharedArgs& a, int32_t tile_rows, unsigned grid, hipStream_t stream) {
  // once per process and instantiation, whatever thread or pool gets here first
  static std::once_flag once;
  static hipError_t status = hipSuccess;
  std::call_once(once, [] {
    status = allow_lds(shared_attend_kernel<HD>, SharedGeo<HD>::LDS_BYTES);
    if (status == hipSuccess) status = allow_lds(shared_attend_f32_kernel<HD, 1>, SharedF32Geo<HD, 1>::LDS_BYTES);
    if (status == hipSuccess) status = allow_lds(shared_attend_f32_kernel<HD, 2>, SharedF32Geo<HD, 2>::LDS_BYTES);
  });
  if (status != hipSuccess) return status;
  if (!a.f32) shared_attend_kernel<HD><<<grid, 256, SharedGeo<HD>::LDS_BYTES, stream>>>(blob, a);
  else if (tile_rows == 16) shared_attend_f32_kernel<HD, 1><<<grid, 64 * SF_WAVES, SharedF32Geo<HD, 1>::LDS_BYTES, stream>>>(blob, a);
  else if (tile_rows == 32) shared_attend_f32_kernel<HD, 2><<<grid, 64 * SF_WAVES, SharedF32Geo<HD, 2>::LDS_BYTES, stream>>>(blob, a);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace

}  // namespace mfma

hipError_t launch_shared_carry(const SharedCarry& piece, void* to, int32_t bytes, hipStream_t stream) {
  mfma::shared_carry_kernel<<<1, 256, 0, stream>>>(piece, (uint32_t*)to, bytes / 4);
  return hipGetLastError();
}

hipError_t launch_attend_shared(const SharedBlob* main, const SharedBlob* merge, const SharedArgs& a, const SharedMergeArgs& ma, int32_t head_dim,
                                int64_t items, int32_t merge_blocks, int32_t tile_rows, hipStream_t stream) {
  using namespace mfma;
  static const SharedBlob none{};
  if (head_dim != 64 && head_dim != 128) return hipErrorInvalidValue;
  const unsigned grid = (unsigned)items * (unsigned)a.n_kv_heads;
  hipError_t e = head_dim == 64 ? launch_items<64>(main ? *main : none, a, tile_rows, grid, stream) : launch_items<128>(main ? *main : none, a, tile_rows, grid, stream);
  if (e != hipSuccess || merge_blocks == 0) return e;
  const unsigned blocks = (unsigned)merge_blocks * (unsigned)a.n_kv_heads;
  const SharedBlob& blob = merge ? *merge : none;
  if (head_dim == 64) {
    if (a.f32) shared_merge_kernel<64, true><<<blocks, 256, 0, stream>>>(blob, a, ma);
    else shared_merge_kernel<64, false><<<blocks, 256, 0, stream>>>(blob, a, ma);
  } else {
    if (a.f32) shared_merge_kernel<128, true><<<blocks, 256, 0, stream>>>(blob, a, ma);
    else shared_merge_kernel<128, false><<<blocks, 256, 0, stream>>>(blob, a, ma);
  }
  return hipGetLastError();
}

}  // namespace dk
