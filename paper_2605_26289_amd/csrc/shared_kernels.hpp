// Launchers of attention for batches that share cells.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "shared_types.h"

namespace dk {

struct SharedBlob {
  uint32_t w[SHARED_BLOB_BYTES / 4];
};
struct SharedCarry {  // descriptors on their way to the workspace
  uint32_t w[960];
};

struct SharedArgs {
  // Descriptors: addresses, or offsets into the kernel's first argument where in_args says so.
  const int32_t* starts;
  const DkShNode* nodes;
  const DkShSeg* segs;
  const int32_t* tokens;
  const void* q;
  const void* k_arena;
  const void* v_arena;
  const void* k_new;
  const void* v_new;
  void* out;
  float* lse;
  float* parts;     // [partial row][KV head][head_dim]
  float* parts_ml;  // [partial row][KV head][2]: largest score in log2 units, sum of weights
  int64_t arena_cells;
  float c;          // raw product to score in log2 units (bf16: its size)
  uint32_t flip;    // bf16: the sign bits of a pair of Q's elements, where the scale is negative
  int32_t n_nodes, n_q_heads, n_kv_heads, group;
  uint32_t gmagic;  // ceil(2^32 / group), 0 for group 1
  int32_t in_args, f32;
};
// By node: its first workgroup (of a KV head; only nodes of one entry that leaves partial rows have any) and its first source, and behind
// the last.  The nodes are the attention kernel's where those are in the workspace, else a copy.
struct SharedMergeArgs {
  const int32_t* blocks;
  const int32_t* src0;
  const DkShSource* sources;
  const DkShNode* nodes;
  int32_t spread, tile_rows, in_args, nodes_in_args;
};
static_assert(sizeof(SharedBlob) + sizeof(SharedArgs) + sizeof(SharedMergeArgs) + 64 <= 4096, "kernel arguments are limited to 4 KiB");
static_assert(sizeof(SharedCarry) + 64 <= 4096, "likewise");

hipError_t launch_shared_carry(const SharedCarry& piece, void* to, int32_t bytes, hipStream_t stream);
// main, merge: the descriptors of the two kernels, where they travel in the arguments.  tile_rows: fp32, rows of an item.
// merge_blocks: of a KV head.
hipError_t launch_attend_shared(const SharedBlob* main, const SharedBlob* merge, const SharedArgs& a, const SharedMergeArgs& ma, int32_t head_dim,
                                int64_t items, int32_t merge_blocks, int32_t tile_rows, hipStream_t stream);

}  // namespace dk
