// fp8.hip -- attention over the paged cache in 8 bits (msa_fp8_forward), with and
// without a window, and the 8-bit cache read back into a bf16 one (msa_fp8_read).
//
// The attention kernels are those of attn.hip; how the numbers get from the cache
// to the matrix products is in attn_device.h (tiles of 128 and 256 rows: turned
// into bf16 on their way into LDS) and attn8_device.h (items of up to 32 rows).
#include "attn_launch.h"

#include <cstdint>
#include <string>

#include "errors.h"
#include "forward.h"
#include "fp8.h"
#include "msa_fp8.h"
#include "plan.h"
#include "plan_handle.h"

namespace msa {
namespace {

struct ReadParams {
  const uint8_t* k;
  const uint8_t* v;
  const uint8_t* k_scale;
  const uint8_t* v_scale;
  const int32_t* table;
  const int32_t* to_table;
  const int32_t* start;  // null: 0
  const int32_t* end;
  uint16_t* k_out;
  uint16_t* v_out;
  int64_t k_sb, k_sh, k_st, v_sb, v_sh, v_sd;
  int64_t ko_sb, ko_sh, ko_st, vo_sb, vo_sh, vo_sd;
  int32_t max_blocks, num_blocks, to_max_blocks, to_num_blocks;
  int32_t num_kv_heads, max_len, seq_blocks, head_groups;
};

// One workgroup takes some heads of one block of one sequence.  A head's block is D
// 16-byte chunks of K and D of V, a chunk a thread: 16 channels of a token, or 16 tokens of a
// channel, to 32 bytes of bf16.  Bound by HBM: one byte read and two written for each number.
template <int D>
__global__ __launch_bounds__(256) void msa_fp8_read_kernel(ReadParams p) {
  const uint32_t item = blockIdx.x / (uint32_t)p.head_groups;
  const int group = (int)(blockIdx.x - item * (uint32_t)p.head_groups);
  const uint32_t b = item / (uint32_t)p.seq_blocks;
  const int i = (int)(item - b * (uint32_t)p.seq_blocks);
  const int lo = (p.start && p.start[b] > 0 ? p.start[b] : 0) - 16 * i;  // tokens lo .. hi - 1 of the block
  const int hi = (p.end[b] < p.max_len ? p.end[b] : p.max_len) - 16 * i;
  if (lo >= 16 || hi <= 0 || lo >= hi) return;
  const int32_t from = p.table[(int64_t)b * p.max_blocks + i], to = p.to_table[(int64_t)b * p.to_max_blocks + i];
  if (from < 0 || from >= p.num_blocks || to < 0 || to >= p.to_num_blocks) return;
  constexpr int kHeads = 256 / (2 * D);  // of a pass
  const int tid = threadIdx.x, c = tid % D;
  const bool is_v = tid / D % 2 != 0;
  const int h0 = p.num_kv_heads * group / p.head_groups, h1 = p.num_kv_heads * (group + 1) / p.head_groups;
  for (int h = h0 + tid / (2 * D); h < h1; h += kHeads) {
    const int64_t sb = ((int64_t)from * p.num_kv_heads + h) * kBlockSize;
    if (!is_v) {
      const int t = c / (D / 16), ch = c % (D / 16) * 16;
      const uint4 x = *reinterpret_cast<const uint4*>(p.k + from * p.k_sb + h * p.k_sh + t * p.k_st + ch);
      const float f = __uint_as_float((uint32_t)p.k_scale[sb + t] << 23);
      if (t < lo || t >= hi) continue;
      uint16_t* out = p.k_out + to * p.ko_sb + h * p.ko_sh + t * p.ko_st + ch;
      reinterpret_cast<uint4*>(out)[0] = make_uint4(fp8_pair<false>(x.x, f), fp8_pair<true>(x.x, f),
                                                    fp8_pair<false>(x.y, f), fp8_pair<true>(x.y, f));
      reinterpret_cast<uint4*>(out)[1] = make_uint4(fp8_pair<false>(x.z, f), fp8_pair<true>(x.z, f),
                                                    fp8_pair<false>(x.w, f), fp8_pair<true>(x.w, f));
    } else {
      const uint4 x = *reinterpret_cast<const uint4*>(p.v + from * p.v_sb + h * p.v_sh + c * p.v_sd);
      const uint4 s = *reinterpret_cast<const uint4*>(p.v_scale + sb);
      const uint32_t u[4] = {x.x, x.y, x.z, x.w}, f[4] = {s.x, s.y, s.z, s.w};
      uint32_t y[8];
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        y[2 * d] = fp8_pair2<0>(u[d], (f[d] & 0xff) << 23, (f[d] >> 8 & 0xff) << 23);
        y[2 * d + 1] = fp8_pair2<2>(u[d], (f[d] >> 16 & 0xff) << 23, f[d] >> 24 << 23);
      }
      uint16_t* out = p.v_out + to * p.vo_sb + h * p.vo_sh + c * p.vo_sd;
      if (lo <= 0 && hi >= 16) {
        reinterpret_cast<uint4*>(out)[0] = make_uint4(y[0], y[1], y[2], y[3]);
        reinterpret_cast<uint4*>(out)[1] = make_uint4(y[4], y[5], y[6], y[7]);
      } else {
#pragma unroll
        for (int t = 0; t < 16; ++t)
          if (t >= lo && t < hi) out[t] = (uint16_t)(y[t / 2] >> (16 * (t & 1)));
      }
    }
  }
}

msa_status refuse(const char* who, msa_status st, const std::string& what) {
  set_last_error(std::string(who) + ": " + what);
  return st;
}

bool aligned(const void* x, uintptr_t a) { return reinterpret_cast<uintptr_t>(x) % a == 0; }

}  // namespace
}  // namespace msa

extern "C" msa_status msa_fp8_forward(msa_plan_t plan, const void* q, const void* k_cache, const void* v_cache,
                                      const uint8_t* k_scale, const uint8_t* v_scale, const int32_t* block_table,
                                      void* o, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const char* who = "msa_fp8_forward";
  msa::AttnParams base;
  msa_status st = msa::forward_params(who, plan, q, k_cache, v_cache, block_table, o, lse, workspace, workspace_bytes, &base);
  if (st != MSA_OK) return st;
  const msa::HostPlan& hp = plan->hp;
  if (hp.has_trees) return msa::refuse(who, MSA_ERR_UNSUPPORTED, "plans of msa_plan_tree read bf16 caches");
  const std::string strides = msa::fp8_strides(hp.shape);
  if (!strides.empty()) return msa::refuse(who, MSA_ERR_INVALID_ARG, strides);
  if (hp.work.empty()) return MSA_OK;
  if (!k_scale || !v_scale || !msa::aligned(k_scale, 16) || !msa::aligned(v_scale, 16))
    return msa::refuse(who, MSA_ERR_INVALID_ARG, "k_scale and v_scale must be non-null and 16-byte aligned");
  auto run = [&](auto& p) {
    p.k_scale = k_scale;
    p.v_scale = v_scale;
    p.num_kv_heads = hp.shape.num_kv_heads;
    return msa::launch_tiles(p, hp.shape.head_dim, hp.item_rows, hp.num_workgroups(), hip_stream);
  };
  int rc;
  if (hp.window > 0) {
    msa::Fp8Params<msa::WindowAttnParams> p{};
    static_cast<msa::WindowAttnParams&>(p) = msa::window_params(plan, base);
    rc = run(p);
  } else {
    msa::Fp8Params<msa::AttnParams> p{};
    static_cast<msa::AttnParams&>(p) = base;
    rc = run(p);
  }
  st = msa::launched(who, "attention", rc);
  return st != MSA_OK ? st : msa::merge_splits(who, plan, o, lse, workspace, hip_stream);
}

extern "C" msa_status msa_fp8_read(const msa_shape* shape, const int32_t* start, const int32_t* end, int32_t max_len,
                                   const int32_t* block_table, const void* k_cache, const void* v_cache,
                                   const uint8_t* k_scale, const uint8_t* v_scale, const msa_shape* to,
                                   const int32_t* to_table, void* k_out, void* v_out, void* hip_stream) {
  const char* who = "msa_fp8_read";
  using msa::refuse;
  if (!shape || !to) return refuse(who, MSA_ERR_INVALID_ARG, "shape and to must be non-null");
  for (const msa_shape* s : {shape, to}) {
    std::string err;
    const msa_status st = msa::check_shape(*s, &err);
    if (st != MSA_OK) return refuse(who, st, err);
  }
  const msa_shape& s = *shape;
  const std::string strides = msa::fp8_strides(s);
  if (!strides.empty()) return refuse(who, MSA_ERR_INVALID_ARG, strides);
  if (s.num_seqs != to->num_seqs || s.num_kv_heads != to->num_kv_heads || s.head_dim != to->head_dim)
    return refuse(who, MSA_ERR_INVALID_ARG, "num_seqs, num_kv_heads and head_dim of both shapes must agree");
  const int64_t most = 16ll * (s.max_blocks_per_seq < to->max_blocks_per_seq ? s.max_blocks_per_seq : to->max_blocks_per_seq);
  if (max_len < 0) return refuse(who, MSA_ERR_INVALID_ARG, "max_len < 0");
  if (max_len > most) max_len = (int32_t)most;
  if (s.num_seqs == 0 || max_len == 0) return MSA_OK;
  if (!end || !block_table || !k_cache || !v_cache || !k_scale || !v_scale || !to_table || !k_out || !v_out)
    return refuse(who, MSA_ERR_INVALID_ARG, "a pointer that must be non-null is null");
  if (!msa::aligned(k_cache, 16) || !msa::aligned(v_cache, 16) || !msa::aligned(k_scale, 16) ||
      !msa::aligned(v_scale, 16) || !msa::aligned(k_out, 16) || !msa::aligned(v_out, 16))
    return refuse(who, MSA_ERR_INVALID_ARG, "caches and scales must be 16-byte aligned");
  if (!msa::aligned(start, 4) || !msa::aligned(end, 4) || !msa::aligned(block_table, 4) || !msa::aligned(to_table, 4))
    return refuse(who, MSA_ERR_INVALID_ARG, "start, end and tables must be 4-byte aligned");
  msa::ReadParams p{};
  p.k = static_cast<const uint8_t*>(k_cache);
  p.v = static_cast<const uint8_t*>(v_cache);
  p.k_scale = k_scale;
  p.v_scale = v_scale;
  p.table = block_table;
  p.to_table = to_table;
  p.start = start;
  p.end = end;
  p.k_out = static_cast<uint16_t*>(k_out);
  p.v_out = static_cast<uint16_t*>(v_out);
  p.k_sb = s.k_stride_block, p.k_sh = s.k_stride_head, p.k_st = s.k_stride_tok;
  p.v_sb = s.v_stride_block, p.v_sh = s.v_stride_head, p.v_sd = s.v_stride_dim;
  p.ko_sb = to->k_stride_block, p.ko_sh = to->k_stride_head, p.ko_st = to->k_stride_tok;
  p.vo_sb = to->v_stride_block, p.vo_sh = to->v_stride_head, p.vo_sd = to->v_stride_dim;
  p.max_blocks = s.max_blocks_per_seq;
  p.num_blocks = s.num_blocks;
  p.to_max_blocks = to->max_blocks_per_seq;
  p.to_num_blocks = to->num_blocks;
  p.num_kv_heads = s.num_kv_heads;
  p.max_len = max_len;
  p.seq_blocks = (max_len + 15) / 16;
  const int64_t items = (int64_t)s.num_seqs * p.seq_blocks;
  // (a launch counts its threads in 32 bits: at most 2^23 workgroups)
  if (items > (int64_t)1 << 23) return refuse(who, MSA_ERR_UNSUPPORTED, "more than 2^23 (sequence, block) pairs");
  p.head_groups = 1;
  const dim3 grid((uint32_t)(items * p.head_groups));
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (s.head_dim == 128)
    hipLaunchKernelGGL(msa::msa_fp8_read_kernel<128>, grid, dim3(256), 0, st, p);
  else
    hipLaunchKernelGGL(msa::msa_fp8_read_kernel<64>, grid, dim3(256), 0, st, p);
  return msa::launched(who, "read", (int)hipGetLastError());
}
