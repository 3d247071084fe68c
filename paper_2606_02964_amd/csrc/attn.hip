// attn.hip -- gfx950 kernels of Multi-Segment Attention: the persistent launches
// around the work items of attn_device.h (which has the mathematics), and
// msa_merge, which combines the per-split partials of a split tile by
// log-sum-exp.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "attn_device.h"
#include "msa_internal.h"

namespace msa {
namespace {

// Persistent launch: workgroup i runs its first item, which lies in its head
// so that no second load has to wait for the list's bounds, then the items
// heads[i].rest .. heads[i].end-1.
template <int D, int W, bool kPrecise>
__global__ __launch_bounds__(64 * W, 2) void msa_attn_kernel(AttnParams p) {
  using T = Tile<D>;
  // K ring (2 steps) then V ring (2 steps); K runs one step ahead of V
  __shared__ __attribute__((aligned(1024))) char smem[2 * T::kBytesK + 2 * T::kBytesV];
  const WgHead head = p.heads[blockIdx.x];
  WorkItem w = head.first;
  for (int it = head.rest;; w = p.work[it++]) {
    attn_item<D, W, kPrecise, false>(p, w, smem);
    if (it >= head.end) break;
  }
}

// The same for 128-row tiles in a launch of no more workgroups than CUs: four
// further waves that only copy.  Alone on its CU, a 4-wave workgroup issues its
// copies (402 of a step's 2430 cycles) with nothing to run beside them; the
// helpers need the registers of a second workgroup, which such a launch does
// not place.  Suffix recompute at 1K, 144 tiles: 22.3 -> 20.4 us; 192 tiles at
// 0.8K keys 20.4 -> 18.7 us.
template <int D, bool kPrecise>
__global__ __launch_bounds__(512, 2) void msa_helped_kernel(AttnParams p) {
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
__global__ __launch_bounds__(256, 2) void msa_decode_kernel(AttnParams p) {
  __shared__ __attribute__((aligned(16))) DecodeLds<D> lds;
  const WgHead head = p.heads[blockIdx.x];
  WorkItem w = head.first;
  for (int it = head.rest;; w = p.work[it++]) {
    decode_item<D, kPrecise>(p, w, lds);
    if (it >= head.end) break;
    __syncthreads();  // the item's merge reads are done
  }
}

// msa_merge: one workgroup per (split tile, chunk of kRows rows), D / 4 threads
// to a row, 4 channels each.  Bound by reading the partials; a tile's rows are
// spread over workgroups because a plan may split few tiles into many pieces
// (58 tiles of 128 rows x 29 pieces, d = 128: 212 us with one workgroup per
// tile, about 16 us in this form; 688 tiles x 2-5 pieces: 71 us and 34 us).
// The lse and O of kBatch pieces load together, so that up to
// kBatch pieces cost one memory round trip.
template <int D>
__global__ __launch_bounds__(256) void msa_merge_kernel(MergeParams p) {
  constexpr int kThreadsPerRow = D / 4;
  constexpr int kRows = 256 / kThreadsPerRow;
  constexpr int kBatch = 8;
  const MergeItem mi = p.merge[blockIdx.x];
  const int G = p.group;
  const int r = blockIdx.y * kRows + threadIdx.x / kThreadsPerRow;
  if (r >= mi.nrows * G) return;
  const int sub = threadIdx.x % kThreadsPerRow;
  const int R = p.tile_rows;
  const int64_t slot_f = (int64_t)R * (D + 1);
  const int t = r / G, hh = r - t * G;
  const int tok = mi.row0 + t, head = mi.kv_head * G + hh;
  const float* base = p.ws + (int64_t)mi.slot0 * slot_f;
  float mx = -__builtin_inff(), L = 0.0f;
  f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s0 = 0; s0 < mi.nsplit; s0 += kBatch) {
    float ls[kBatch];
    f32x4 os[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const float* slot = base + (int64_t)min(s0 + u, mi.nsplit - 1) * slot_f;
      ls[u] = slot[(int64_t)R * D + r];
      os[u] = *reinterpret_cast<const f32x4*>(slot + r * D + sub * 4);
    }
    float m_new = mx;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) m_new = fmaxf(m_new, ls[u]);
    const float mu = m_new == -__builtin_inff() ? 0.0f : m_new;
    const float alpha = __builtin_amdgcn_exp2f((mx - mu) * kLog2e);  // 0 on the first batch
    L *= alpha;
    acc *= alpha;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const float wgt = s0 + u < mi.nsplit ? __builtin_amdgcn_exp2f((ls[u] - mu) * kLog2e) : 0.0f;
      L += wgt;
      acc += wgt * os[u];
    }
    mx = m_new;
  }
  const float inv = L > 0.0f ? 1.0f / L : 0.0f;
  bf16x4 v;
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = (__bf16)(acc[j] * inv);
  *reinterpret_cast<bf16x4*>(p.o + (int64_t)tok * p.o_st + (int64_t)head * p.o_sh + sub * 4) = v;
  if (p.lse && sub == 0)
    p.lse[(int64_t)tok * p.num_q_heads + head] = (mx == -__builtin_inff() ? 0.0f : mx) + __logf(L);
}

// The precise-weights forms are separate instantiations, so that the
// default kernels carry no test of the flag.
template <bool kPrecise>
int launch_attn_form(const AttnParams& p, int head_dim, int item_rows, int num_wg, hipStream_t s) {
  if (item_rows == kTileRowsNarrow && num_wg <= kCUs && head_dim == 128)
    hipLaunchKernelGGL((msa_helped_kernel<128, kPrecise>), dim3(num_wg), dim3(512), 0, s, p);
  else if (item_rows == kTileRowsNarrow && num_wg <= kCUs && head_dim == 64)
    hipLaunchKernelGGL((msa_helped_kernel<64, kPrecise>), dim3(num_wg), dim3(512), 0, s, p);
  else if (head_dim == 128 && item_rows == kTileRowsNarrow)
    hipLaunchKernelGGL((msa_attn_kernel<128, 4, kPrecise>), dim3(num_wg), dim3(256), 0, s, p);
  else if (head_dim == 128 && item_rows == kTileRowsWide)
    hipLaunchKernelGGL((msa_attn_kernel<128, 8, kPrecise>), dim3(num_wg), dim3(512), 0, s, p);
  else if (head_dim == 64 && item_rows == kTileRowsNarrow)
    hipLaunchKernelGGL((msa_attn_kernel<64, 4, kPrecise>), dim3(num_wg), dim3(256), 0, s, p);
  else if (head_dim == 64 && item_rows == kTileRowsWide)
    hipLaunchKernelGGL((msa_attn_kernel<64, 8, kPrecise>), dim3(num_wg), dim3(512), 0, s, p);
  else if (head_dim == 128 && item_rows == kTileRowsDecode)
    hipLaunchKernelGGL((msa_decode_kernel<128, kPrecise>), dim3(num_wg), dim3(256), 0, s, p);
  else if (head_dim == 64 && item_rows == kTileRowsDecode)
    hipLaunchKernelGGL((msa_decode_kernel<64, kPrecise>), dim3(num_wg), dim3(256), 0, s, p);
  else
    return (int)hipErrorInvalidValue;
  return (int)hipGetLastError();
}

}  // namespace

int launch_attn(const AttnParams& p, int head_dim, int item_rows, int num_wg, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (num_wg <= 0) return 0;
  return p.precise ? launch_attn_form<true>(p, head_dim, item_rows, num_wg, s)
                   : launch_attn_form<false>(p, head_dim, item_rows, num_wg, s);
}

int launch_merge(const MergeParams& p, int head_dim, int num_merge, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (num_merge <= 0) return 0;
  const int rows_per_wg = 1024 / head_dim;  // kRows of msa_merge_kernel
  const dim3 grid(num_merge, (p.max_rows + rows_per_wg - 1) / rows_per_wg);
  if (head_dim == 128)
    hipLaunchKernelGGL(msa_merge_kernel<128>, grid, dim3(256), 0, s, p);
  else if (head_dim == 64)
    hipLaunchKernelGGL(msa_merge_kernel<64>, grid, dim3(256), 0, s, p);
  else
    return (int)hipErrorInvalidValue;
  return (int)hipGetLastError();
}

}  // namespace msa
