// Host-side planning of one dk_shared_attend call: which cells the batch's entries share, work items, partial rows and merges.
#pragma once
#include <cstddef>
#include <cstdint>
#include <vector>

#include "pool.hpp"
#include "shared_types.h"

namespace dk {

struct SharedConfig {
  int32_t n_q_heads = 0, n_kv_heads = 0, head_dim = 0;
  bool bf16 = true;
};

// May be reused from call to call: planning a batch like the previous one allocates next to nothing.
struct SharedPlan {
  struct Link {  // an entry's rows in a shared node: from row0 on; the node in front of it by `before` (-1: none)
    int32_t node, row0, before;
  };
  struct Member {  // an entry on its way down the tree of shared prefixes
    int32_t entry;
    int32_t part;   // the part of its chain that the position under consideration is in
    int32_t link;   // its innermost shared node so far
    int64_t key;    // first cell of the node in which it parts from others
  };
  struct Task {  // members [begin, end) whose cells are the same below `pos`; positions from `start` on are in no node yet
    int32_t begin, end;
    int64_t start, pos;
  };
  struct Node {
    DkShNode d;
    int32_t nsegs, seg0;   // in `segs` below (nodes are put in order when all are known)
    int32_t tiles, pieces;
    float per_key, fixed;  // cost of a work item
    int32_t entry, link;   // of one entry: which, and its innermost shared node; shared: -1
  };
  struct Load {  // of a node that is not cut: time of an item, of a key; row tiles, rows; 1: it leaves partial rows however it is cut
    double us, per_key, tiles, rows, part;
    double pieces, piece_us;  // of the cut that is looked at
  };
  std::vector<Load> loads;
  struct Level {  // places that are free from then on
    double us, places;
  };
  std::vector<Level> levels;
  std::vector<Extent> ext;
  std::vector<Pool::Part> parts;   // the entries' chains
  std::vector<int32_t> part0;      // first part of every entry
  std::vector<int64_t> n;          // cached tokens of every entry before the call
  std::vector<Member> members;
  std::vector<Task> tasks;
  std::vector<Link> links;
  std::vector<Node> nodes;
  std::vector<DkShSeg> node_segs;
  std::vector<int32_t> order;

  std::vector<int32_t> starts;     // first work item of every node, and behind the last
  std::vector<DkShNode> out_nodes;
  std::vector<DkShSeg> segs;
  std::vector<int32_t> tokens;
  // The merge: rows of entries that have more than one partial row.  By node, and behind the last: its first workgroup (of a KV head;
  // others than such entries' have none) and the first of its sources, the prefixes in front of it.
  std::vector<int32_t> blocks, src0;
  std::vector<DkShSource> sources;
  int64_t total_tokens = 0, part_rows = 0, items = 0, row_items = 0;
  int32_t tile_rows = 0;           // fp32: rows of an item
  int32_t spread = 1;              // lane groups that share the partial rows of a row in the merge
  int32_t merge_blocks = 0, n_merges = 0;
  // main kernel's descriptors, the merge's, its copy of the nodes where they travel in arguments, partial rows
  size_t off_nodes = 0, off_segs = 0, off_tokens = 0, main_bytes = 0;
  size_t off_src0 = 0, off_sources = 0, merge_bytes = 0;
  size_t off_merge = 0, off_parts = 0, total_bytes = 0;
  size_t node_bytes() const { return out_nodes.size() * sizeof(DkShNode); }
  bool in_args() const { return main_bytes <= (size_t)SHARED_BLOB_BYTES && (n_merges == 0 || merge_bytes + node_bytes() <= (size_t)SHARED_BLOB_BYTES); }
  bool merge_in_args() const { return merge_bytes <= (size_t)SHARED_BLOB_BYTES; }
};

// Caller holds pool.mutex().
int32_t build_shared_plan(Pool& pool, const SharedConfig& cfg, int32_t n_seqs, const int32_t* slots, const int32_t* cu_delta, bool staged,
                          SharedPlan* plan);

}  // namespace dk
