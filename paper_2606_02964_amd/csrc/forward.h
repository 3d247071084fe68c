// forward.h -- msa_forward's parts, shared by the entry points that run it.
#pragma once

#include <cstddef>
#include <cstdint>

#include "msa.h"
#include "msa_internal.h"

namespace msa {

// Checks, then the attention launch and (for split tiles) the merge launch,
// with the given workspace.  `who` names the entry point in error messages.
msa_status forward_impl(const char* who, msa_plan_t plan, const void* q, const void* k_cache,
                        const void* v_cache, const int32_t* block_table, void* o, float* lse,
                        void* workspace, size_t workspace_bytes, void* hip_stream);

// The checks, and the attention kernel's arguments (left empty for a plan
// without rows: MSA_OK, nothing to launch).
msa_status forward_params(const char* who, msa_plan_t plan, const void* q, const void* k_cache,
                          const void* v_cache, const int32_t* block_table, void* o, float* lse,
                          void* workspace, size_t workspace_bytes, AttnParams* out);

// The same with the plan's window (hp.window > 0).
WindowAttnParams window_params(msa_plan_t plan, const AttnParams& base);

// The merge launch of the plan's split tiles, if it has any.
msa_status merge_splits(const char* who, msa_plan_t plan, void* o, float* lse, void* workspace,
                        void* hip_stream);

// MSA_OK, or MSA_ERR_DEVICE with a message, for the hipError_t of a launch.
msa_status launched(const char* who, const char* what, int rc);

// Whether a block's K and V, of `bytes` a number, span less than 4 GiB each: the kernels' offsets within one are 32 bits.
inline bool block_spans_fit(const msa_shape& s, int bytes) {
  const int64_t most = ((int64_t)1 << 32) / bytes;
  return s.k_stride_tok <= (most - s.head_dim) / (kBlockSize - 1) && s.v_stride_dim <= (most - kBlockSize) / (s.head_dim - 1);
}

// Workspace bytes a plan's msa_forward needs (plan non-null).
int64_t plan_workspace_bytes(msa_plan_t plan);

}  // namespace msa
