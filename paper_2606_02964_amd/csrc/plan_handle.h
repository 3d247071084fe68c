// plan_handle.h -- what an msa_plan_t points to, shared by the entry points.
#pragma once

#include <cstdint>
#include <vector>

#include "plan.h"

struct msa_plan_s {
  msa::HostPlan hp;
  bool host_only = true;
  int device = -1;
  std::vector<char> staging;  // host image of the device buffer (kept alive for the async copy)
  char* dev = nullptr;        // device buffer: row_pos | work | merge | append | heads | seq rows | row trees | trees
                              // | weights | joins | streams
  const int32_t* d_row_pos = nullptr;
  const msa::WorkItem* d_work = nullptr;
  const msa::WgHead* d_heads = nullptr;
  const msa::MergeItem* d_merge = nullptr;
  const msa::AppendItem* d_append = nullptr;
  const int32_t* d_seq_row0 = nullptr;         // [num_seqs + 1] first packed row of each sequence
  const msa::RowTree* d_row_tree = nullptr;    // [total_q], plans of msa_plan_tree
  const msa::TreeSpan* d_trees = nullptr;      // [trees]
  const msa::WeightsItem* d_weights = nullptr;
  const msa::WeightsJoin* d_weight_joins = nullptr;
  const msa::StreamItem* d_streams = nullptr;
};
