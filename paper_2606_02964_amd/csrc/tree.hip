// tree.hip -- attention of trees of drafted tokens over the paged cache, and
// the trees' ancestor masks.
//
// The attention kernels are those of attn.hip with a tree's visibility (see
// attn_device.h): a tree is a segment whose rows see the whole context and some
// of the segment's own slots, so nothing but the masked steps differs, of which
// a tree has one to three of its row's dozens or hundreds.  The merge of
// split tiles is msa_merge as it is.  Bound as those are: 48 trees of 16 slots over
// up to 6K keys each (32 query, 8 KV heads, d = 128) read K/V at 4.9 TB/s (154 us);
// 16 of 64 slots, each beside a chunk of 128 rows, over up to 30K keys (64 query heads)
// run at 934 TFLOP/s (599 us); one of 61 slots over 8K 21.4 us with its merge.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>

#include "attn_device.h"
#include "errors.h"
#include "forward.h"
#include "msa_tree.h"
#include "plan_handle.h"

namespace msa {
namespace {

template <int D, int W, bool kPrecise>
__global__ __launch_bounds__(64 * W, 2) void msa_tree_kernel(TreeAttnParams p) {
  using T = Tile<D>;
  __shared__ __attribute__((aligned(1024))) char smem[2 * T::kBytesK + 2 * T::kBytesV];
  const WgHead head = p.heads[blockIdx.x];
  WorkItem w = head.first;
  for (int it = head.rest;; w = p.work[it++]) {
    attn_item<D, W, kPrecise, false>(p, w, smem);
    if (it >= head.end) break;
  }
}

// 128-row tiles with a CU each: four further waves do the copies
template <int D, bool kPrecise>
__global__ __launch_bounds__(512, 2) void msa_tree_helped_kernel(TreeAttnParams p) {
  using T = Tile<D>;
  __shared__ __attribute__((aligned(1024))) char smem[2 * T::kBytesK + 2 * T::kBytesV];
  const WgHead head = p.heads[blockIdx.x];
  WorkItem w = head.first;
  for (int it = head.rest;; w = p.work[it++]) {
    attn_item<D, 4, kPrecise, true>(p, w, smem);
    if (it >= head.end) break;
  }
}

template <int D, bool kPrecise>
__global__ __launch_bounds__(256, 2) void msa_tree_narrow_kernel(TreeAttnParams p) {
  __shared__ __attribute__((aligned(16))) DecodeLds<D> lds;
  const WgHead head = p.heads[blockIdx.x];
  WorkItem w = head.first;
  for (int it = head.rest;; w = p.work[it++]) {
    decode_item<D, kPrecise>(p, w, lds);
    if (it >= head.end) break;
    __syncthreads();  // the item's merge reads are done
  }
}

template <int D, bool kPrecise>
int launch_tree(const TreeAttnParams& p, int item_rows, int num_wg, hipStream_t s) {
  if (item_rows == kTileRowsDecode)
    hipLaunchKernelGGL((msa_tree_narrow_kernel<D, kPrecise>), dim3(num_wg), dim3(256), 0, s, p);
  else if (item_rows == kTileRowsNarrow && num_wg <= kCUs)
    hipLaunchKernelGGL((msa_tree_helped_kernel<D, kPrecise>), dim3(num_wg), dim3(512), 0, s, p);
  else if (item_rows == kTileRowsNarrow)
    hipLaunchKernelGGL((msa_tree_kernel<D, 4, kPrecise>), dim3(num_wg), dim3(256), 0, s, p);
  else if (item_rows == kTileRowsWide)
    hipLaunchKernelGGL((msa_tree_kernel<D, 8, kPrecise>), dim3(num_wg), dim3(512), 0, s, p);
  else
    return (int)hipErrorInvalidValue;
  return (int)hipGetLastError();
}

// One workgroup per tree.  The mask of slot t is its own bit and the bits of
// its ancestors: each thread follows the parents of its slots up to the root
// through LDS, setting bits of one word at a time (a parent is a lower slot, so
// the walk ends, and it enters the words in descending order).
// A step's masks are a few KB; the launch is all there is to it (1.6 us).
__global__ __launch_bounds__(256) void msa_tree_mask_kernel(const TreeSpan* trees, const int32_t* parents,
                                                            uint64_t* mask, int64_t stride, int words) {
  __shared__ int16_t up[MSA_TREE_MAX_SLOTS];
  const TreeSpan tree = trees[blockIdx.x];
  for (int i = threadIdx.x; i < tree.n; i += blockDim.x) {
    const int32_t p = parents[tree.row0 + i];
    up[i] = (int16_t)(p >= 0 && p < i ? p : -1);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < tree.n; i += blockDim.x) {
    uint64_t* row = mask + (int64_t)(tree.row0 + i) * stride;
    int a = i;
    for (int w = words - 1; w >= 0; --w) {
      uint64_t bits = 0;
      for (; a >= 64 * w && a >= 0; a = up[a]) bits |= 1ull << (a & 63);
      row[w] = bits;
    }
  }
}

msa_status fail(const char* who, const std::string& msg) {
  set_last_error(std::string(who) + ": " + msg);
  return MSA_ERR_INVALID_ARG;
}

bool aligned(const void* p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

}  // namespace
}  // namespace msa

extern "C" msa_status msa_tree_mask(msa_plan_t plan, const int32_t* parents, uint64_t* mask, int64_t mask_stride,
                                    void* hip_stream) {
  const char* who = "msa_tree_mask";
  if (!plan) return msa::fail(who, "null plan");
  if (plan->host_only) return msa::fail(who, "plan was built with MSA_PLAN_HOST_ONLY");
  const msa::HostPlan& hp = plan->hp;
  if (hp.trees.empty()) return MSA_OK;
  const int words = (hp.max_slots + 63) / 64;
  if (!parents || !mask) return msa::fail(who, "parents and mask must be non-null");
  if (!msa::aligned(parents, 4) || !msa::aligned(mask, 8))
    return msa::fail(who, "parents must be 4-byte and mask 8-byte aligned");
  if (mask_stride < words)
    return msa::fail(who, "mask_stride must be at least " + std::to_string(words) + " words");
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev != plan->device)
    return msa::fail(who, "current device differs from the plan's device");
  hipLaunchKernelGGL(msa::msa_tree_mask_kernel, dim3((uint32_t)hp.trees.size()), dim3(256), 0,
                     static_cast<hipStream_t>(hip_stream), plan->d_trees, parents, mask, mask_stride, words);
  return msa::launched(who, "mask", (int)hipGetLastError());
}

extern "C" msa_status msa_tree_forward(msa_plan_t plan, const void* q, const void* k_cache, const void* v_cache,
                                       const int32_t* block_table, const uint64_t* mask, int64_t mask_stride,
                                       void* o, float* lse, void* workspace, size_t workspace_bytes,
                                       void* hip_stream) {
  const char* who = "msa_tree_forward";
  msa::TreeAttnParams p{};
  msa_status st = msa::forward_params(who, plan, q, k_cache, v_cache, block_table, o, lse, workspace,
                                      workspace_bytes, &p);
  if (st != MSA_OK) return st;
  const msa::HostPlan& hp = plan->hp;
  if (!hp.has_trees) return msa::fail(who, "the plan was not built by msa_plan_tree");
  if (hp.work.empty()) return MSA_OK;
  if (!hp.trees.empty()) {
    const int words = (hp.max_slots + 63) / 64;
    if (!mask || !msa::aligned(mask, 8)) return msa::fail(who, "mask must be non-null and 8-byte aligned");
    if (mask_stride < words)
      return msa::fail(who, "mask_stride must be at least " + std::to_string(words) + " words");
  }
  p.row_tree = plan->d_row_tree;
  p.mask = mask;
  p.mask_stride = mask_stride;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const int num_wg = hp.num_workgroups();
  const bool d128 = hp.shape.head_dim == 128, precise = hp.precise_weights;
  const int rc = d128 ? precise ? msa::launch_tree<128, true>(p, hp.item_rows, num_wg, s)
                                : msa::launch_tree<128, false>(p, hp.item_rows, num_wg, s)
                      : precise ? msa::launch_tree<64, true>(p, hp.item_rows, num_wg, s)
                                : msa::launch_tree<64, false>(p, hp.item_rows, num_wg, s);
  st = msa::launched(who, "attention", rc);
  return st != MSA_OK ? st : msa::merge_splits(who, plan, o, lse, workspace, hip_stream);
}
