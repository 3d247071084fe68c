// attn_launch.h -- the persistent launches of attn.hip for any of the attention's
// parameters (windows, 8-bit caches): the kernels differ in their work items alone,
// which attn_device.h and attn8_device.h choose by the parameters' type.
#pragma once

#include <hip/hip_runtime.h>

#include "attn8_device.h"
#include "attn_device.h"
#include "msa_internal.h"

namespace msa {
namespace {

template <class P, int D, int W, bool kPrecise, bool kHelp>
__global__ __launch_bounds__(kHelp ? 512 : 64 * W, 2) void msa_tiles_kernel(P p) {
  __shared__ __attribute__((aligned(1024))) char smem[Tile<D>::template lds_bytes<P>()];
  const WgHead head = p.heads[blockIdx.x];
  WorkItem w = head.first;
  for (int it = head.rest;; w = p.work[it++]) {
    attn_item<D, W, kPrecise, kHelp>(p, w, smem);
    if (it >= head.end) break;
  }
}

template <class P, int D, bool kPrecise>
__global__ __launch_bounds__(256, 2) void msa_rows_kernel(P p) {
  __shared__ __attribute__((aligned(16))) DecodeLds<D> lds;
  const WgHead head = p.heads[blockIdx.x];
  WorkItem w = head.first;
  for (int it = head.rest;; w = p.work[it++]) {
    if constexpr (P::kFp8) decode8_item<D, kPrecise>(p, w, lds);
    else decode_item<D, kPrecise>(p, w, lds);
    if (it >= head.end) break;
    __syncthreads();  // the item's merge reads are done
  }
}

// the forms by item width as launch_attn has them
template <class P, int D, bool kPrecise>
int launch_form(const P& p, int item_rows, int num_wg, hipStream_t s) {
  if (item_rows == kTileRowsDecode)
    hipLaunchKernelGGL((msa_rows_kernel<P, D, kPrecise>), dim3(num_wg), dim3(256), 0, s, p);
  else if (item_rows == kTileRowsNarrow && num_wg <= kCUs)
    hipLaunchKernelGGL((msa_tiles_kernel<P, D, 4, kPrecise, true>), dim3(num_wg), dim3(512), 0, s, p);
  else if (item_rows == kTileRowsNarrow)
    hipLaunchKernelGGL((msa_tiles_kernel<P, D, 4, kPrecise, false>), dim3(num_wg), dim3(256), 0, s, p);
  else if (item_rows == kTileRowsWide)
    hipLaunchKernelGGL((msa_tiles_kernel<P, D, 8, kPrecise, false>), dim3(num_wg), dim3(512), 0, s, p);
  else
    return (int)hipErrorInvalidValue;
  return (int)hipGetLastError();
}

template <class P>
int launch_tiles(const P& p, int head_dim, int item_rows, int num_wg, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (num_wg <= 0) return 0;
  if (head_dim == 128)
    return p.precise ? launch_form<P, 128, true>(p, item_rows, num_wg, s) : launch_form<P, 128, false>(p, item_rows, num_wg, s);
  if (head_dim == 64)
    return p.precise ? launch_form<P, 64, true>(p, item_rows, num_wg, s) : launch_form<P, 64, false>(p, item_rows, num_wg, s);
  return (int)hipErrorInvalidValue;
}

}  // namespace
}  // namespace msa
