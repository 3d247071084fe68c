// plan.h -- host planner of the MSA library (no HIP calls).
#pragma once

#include <string>
#include <vector>

#include "append.h"
#include "msa.h"
#include "msa_internal.h"
#include "weights.h"

namespace msa {

struct HostPlan {
  msa_shape shape{};
  int32_t group = 1;        // G = Hq / Hkv
  int32_t tile_rows = 0;    // rows per tile: kTileRowsDecode, kTileRowsNarrow or kTileRowsWide
  int32_t item_rows = 0;    // rows per work item: tile_rows, or kTileRowsDecode in a 128-row plan of few tiles
  int32_t tile_tokens = 0;  // query tokens per work item
  bool precise_weights = false;  // MSA_PLAN_PRECISE_WEIGHTS: hi + lo weights on every step
  int64_t total_q = 0;
  std::vector<int32_t> row_pos;   // [total_q] absolute position of each packed row
  std::vector<int32_t> seq_blocks; // [num_seqs] block-table entries the plan reads per sequence
  std::vector<WorkItem> work;     // items grouped by workgroup (workgroup i: wg_ptr[i] .. wg_ptr[i+1]-1)
  std::vector<int32_t> wg_ptr;    // [num_workgroups + 1]; workgroup i runs on XCD i % 8
  std::vector<MergeItem> merge;
  std::vector<AppendItem> append; // one per (segment, cache block) slice
  std::vector<int32_t> seq_row0;  // [num_seqs + 1] first packed row of each sequence
  std::vector<WeightsItem> weights;      // key weights of sequences of more than kPairs pairs
  std::vector<WeightsJoin> weight_joins;
  int32_t weight_slots = 0;
  std::vector<StreamItem> streams;       // key weights of the others
  bool has_trees = false;         // built by msa_plan_tree (it may hold no tree all the same)
  std::vector<RowTree> row_tree;  // [total_q] if has_trees
  std::vector<TreeSpan> trees;    // one per tree segment
  int32_t tree_rows = 0;          // rows of all trees
  int32_t max_slots = 0;          // rows of the largest one
  int64_t num_tiles = 0;          // tiles x kv heads before splitting
  int64_t max_splits = 1;
  int32_t max_merge_rows = 0;     // rows (tokens x G) of the largest split tile
  int64_t num_slots = 0;          // workspace partial slots
  int64_t workspace_bytes = 0;
  int num_workgroups() const { return wg_ptr.empty() ? 0 : (int)wg_ptr.size() - 1; }
  double useful_flops = 0, tile_flops = 0, planned_bytes = 0, min_bytes = 0;
};

// The checks of a shape alone; a message in *err where it is refused.
msa_status check_shape(const msa_shape& shape, std::string* err);

// Validates the inputs and fills *out.  On error returns the status and a
// message in *err; *out is then unspecified.  with_trees: a plan of
// msa_plan_tree, seg_tree as there (null: every segment is a tree).
msa_status build_plan(const msa_shape* shape, const int32_t* seq_kv_len, const int32_t* seg_indptr,
                      const int32_t* seg_start, const int32_t* seg_len, const msa_plan_opts* opts,
                      bool with_trees, const int32_t* seg_tree, HostPlan* out, std::string* err);

}  // namespace msa
