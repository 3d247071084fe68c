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
  int32_t num_kv_heads, max_len, seq_blocks;
};

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void put(uint16_t* to, const uint4& v) {
  const u32x4 x = {v.x, v.y, v.z, v.w};
  __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>(to));
}

// One workgroup takes one block of one sequence, all its heads, 8 bytes to 16 a thread.  Bound
// by HBM: one byte read and two written for each number (788 MB of 16 sequences of 8000, 8 heads,
// d = 128: 162 us, 4.9 TB/s; a device copy 5.2).  Stores of 16 bytes that lie side by side in a wave, as loads
// of 16 bytes would not give them (179 us), and past the caches: 43 us were 31 with 2 heads, 197 MB.
template <int D>
__global__ __launch_bounds__(256) void msa_fp8_read_kernel(ReadParams p) {
  const uint32_t b = blockIdx.x / (uint32_t)p.seq_blocks;
  const int i = (int)(blockIdx.x - b * (uint32_t)p.seq_blocks);
  const int lo = (p.start && p.start[b] > 0 ? p.start[b] : 0) - 16 * i;  // tokens lo .. hi - 1 of the block
  const int hi = (p.end[b] < p.max_len ? p.end[b] : p.max_len) - 16 * i;
  if (lo >= 16 || hi <= 0 || lo >= hi) return;
  const int32_t from = p.table[(int64_t)b * p.max_blocks + i], to = p.to_table[(int64_t)b * p.to_max_blocks + i];
  if (from < 0 || from >= p.num_blocks || to < 0 || to >= p.to_num_blocks) return;
  // a head's block is 2 D 8-byte pieces of K (8 channels of a token) and as many of V (8 tokens of a channel)
  constexpr int kPieces = 4 * D;
  for (int idx = threadIdx.x; idx < p.num_kv_heads * kPieces; idx += 256) {
    const int h = idx / kPieces, c = idx % (2 * D);
    const bool is_v = idx / (2 * D) % 2 != 0;  // uniform over a wave
    const int64_t sb = ((int64_t)from * p.num_kv_heads + h) * kBlockSize;
    if (!is_v) {
      const int t = c / (D / 8), ch = c % (D / 8) * 8;
      const uint2 x = *reinterpret_cast<const uint2*>(p.k + from * p.k_sb + h * p.k_sh + t * p.k_st + ch);
      const float f = __uint_as_float((uint32_t)p.k_scale[sb + t] << 23);
      if (t < lo || t >= hi) continue;
      put(p.k_out + to * p.ko_sb + h * p.ko_sh + t * p.ko_st + ch,
          make_uint4(fp8_pair<false>(x.x, f), fp8_pair<true>(x.x, f), fp8_pair<false>(x.y, f), fp8_pair<true>(x.y, f)));
    } else {
      const int ch = c / 2, t0 = c % 2 * 8;
      const uint2 x = *reinterpret_cast<const uint2*>(p.v + from * p.v_sb + h * p.v_sh + ch * p.v_sd + t0);
      const uint2 s = *reinterpret_cast<const uint2*>(p.v_scale + sb + t0);
      const uint4 y = make_uint4(fp8_pair2<0>(x.x, (s.x & 0xff) << 23, (s.x >> 8 & 0xff) << 23),
                                 fp8_pair2<2>(x.x, (s.x >> 16 & 0xff) << 23, s.x >> 24 << 23),
                                 fp8_pair2<0>(x.y, (s.y & 0xff) << 23, (s.y >> 8 & 0xff) << 23),
                                 fp8_pair2<2>(x.y, (s.y >> 16 & 0xff) << 23, s.y >> 24 << 23));
      uint16_t* out = p.v_out + to * p.vo_sb + h * p.vo_sh + ch * p.vo_sd + t0;
      if (lo <= t0 && hi >= t0 + 8) {
        put(out, y);
      } else {
        const uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int t = 0; t < 8; ++t)
          if (t0 + t >= lo && t0 + t < hi) out[t] = (uint16_t)(w[t / 2] >> (16 * (t & 1)));
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
  if (!msa::block_spans_fit(hp.shape, 1)) return msa::refuse(who, MSA_ERR_UNSUPPORTED, "K or V of a block spans 4 GiB or more");
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
  const dim3 grid((uint32_t)items);
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (s.head_dim == 128)
    hipLaunchKernelGGL(msa::msa_fp8_read_kernel<128>, grid, dim3(256), 0, st, p);
  else
    hipLaunchKernelGGL(msa::msa_fp8_read_kernel<64>, grid, dim3(256), 0, st, p);
  return msa::launched(who, "read", (int)hipGetLastError());
}
