// weights.hip -- the attention weight each cached key receives from a plan's
// query rows (msa_kv_weights).
//
//   w[j] = sum over the rows r that see key j, and the query heads h of a KV
//          head's group, of exp(scale q_rh k_j - lse_rh)
//
// The softmax's statistics are known (msa_forward's lse), so a key's sum needs
// one pass over the rows and no other key.  A wave takes 64 keys of one KV head
// and goes through the rows of their sequence, 32 (row, head) pairs at a time:
//   - S = Q K^T on v_mfma_f32_32x32x16_bf16 with Q as the A operand: each lane
//     then holds 16 rows of ONE key (a column of S), so a key's sum stays in its
//     lane; the lane pair (l, l + 32) of a key is joined once at the end;
//   - the subtraction of lse is one more MFMA: its A operand holds -lse / scale in
//     three bf16 terms (24 bits, as much as the fp32 lse has), its B operand
//     ones.  The score registers then hold (q k - lse / scale) and a weight is
//     exp2 of that times scale * log2(e).  A row that is to give no weight (no such
//     row, or lse = -inf) has -inf there, and costs nothing further;
//   - the causal limit is applied only on the tiles that hold a row before the
//     wave's last key.  Rows ascend in position, so the walk starts at the last
//     row and ends at the first tile whose rows all lie before the wave's keys.
// Sums are in fp32, 16 rows of a tile added pairwise and then to the running sum;
// no atomics, so equal calls give equal bits.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>

#include "errors.h"
#include "forward.h"
#include "msa_cache.h"
#include "plan_handle.h"

namespace msa {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kWaveKeys = 64;
constexpr int kGroupKeys = 4 * kWaveKeys;  // keys of a workgroup

struct WeightsParams {
  const uint16_t* q;
  const uint16_t* k;
  const int32_t* block_table;
  const int32_t* row_pos;
  const int32_t* seq_row0;
  const float* lse;
  float* weights;
  int64_t q_st, q_sh, k_sb, k_sh, k_st, w_sb, w_sh;
  int32_t num_seqs, num_q_heads, num_kv_heads, max_blocks, group;
  uint32_t group_inv;  // ceil(2^20 / G): r / G = r * group_inv >> 20 for r < 288
  float inv_scale, scale_log2;
  int32_t accumulate;
};

// x in three bf16 terms; infinities stay in the first
__device__ __forceinline__ bf16x8 three_terms(float x, bool here) {
  bf16x8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (__bf16)0.0f;
  if (here) {
    v[0] = (__bf16)x;
    const float r = __builtin_isinf(x) ? 0.0f : x - (float)v[0];
    v[1] = (__bf16)r;
    v[2] = (__bf16)(r - (float)v[1]);
  }
  return v;
}

template <int D>
__global__ __launch_bounds__(256, 2) void msa_kv_weights_kernel(WeightsParams p) {
  const int per_chunk = p.num_seqs * p.num_kv_heads;
  const int chunk = blockIdx.x / per_chunk, rest = blockIdx.x - chunk * per_chunk;
  const int seq = rest / p.num_kv_heads, kv_head = rest - seq * p.num_kv_heads;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, hl = lane >> 5, ln = lane & 31;
  const int row0 = p.seq_row0[seq], nrows = p.seq_row0[seq + 1] - row0;
  if (nrows == 0) return;
  const int last = p.row_pos[row0 + nrows - 1];
  const int k0 = chunk * kGroupKeys + wave * kWaveKeys;
  if (k0 > last) return;
  const int G = p.group;

  // B operand: key k0 + kt*32 + ln, channels kk*16 + hl*8 .. +8
  bf16x8 kf[2][D / 16], ones;
#pragma unroll
  for (int i = 0; i < 8; ++i) ones[i] = (__bf16)1.0f;
#pragma unroll
  for (int kt = 0; kt < 2; ++kt) {
    const int key = k0 + kt * 32 + ln;
    const int32_t blk = key <= last ? p.block_table[(int64_t)seq * p.max_blocks + (key >> 4)] : 0;
    const uint16_t* src = p.k + (int64_t)blk * p.k_sb + (int64_t)kv_head * p.k_sh + (int64_t)(key & 15) * p.k_st + hl * 8;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      if (key <= last) {
        kf[kt][kk] = *reinterpret_cast<const bf16x8*>(src + kk * 16);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) kf[kt][kk][j] = (__bf16)0.0f;
      }
    }
  }

  const int n = nrows * G;  // (row, head) pairs
  float sum[2] = {0.0f, 0.0f};
  for (int base = (n - 1) / 32 * 32; base >= 0; base -= 32) {
    const int t0 = base / G;  // uniform
    const uint32_t off = (uint32_t)(base - t0 * G + ln);
    const int dt = (int)(off * p.group_inv >> 20);
    const bool valid = base + ln < n;
    const int tok = row0 + t0 + dt, head = kv_head * G + (int)off - dt * G;
    const int pos = valid ? p.row_pos[tok] : 0x7fffffff;
    const int nvalid = n - base < 32 ? n - base : 32;
    if (__builtin_amdgcn_readlane(pos, nvalid - 1) < k0) break;
    bf16x8 qf[D / 16];
    float l = __builtin_inff();
    if (valid) {
      const uint16_t* src = p.q + (int64_t)tok * p.q_st + (int64_t)head * p.q_sh + hl * 8;
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) qf[kk] = *reinterpret_cast<const bf16x8*>(src + kk * 16);
      l = p.lse[(int64_t)tok * p.num_q_heads + head];
      if (l == -__builtin_inff()) l = __builtin_inff();
    } else {
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
        for (int j = 0; j < 8; ++j) qf[kk][j] = (__bf16)0.0f;
    }
    const bf16x8 lf = three_terms(-l * p.inv_scale, hl == 0);
    const bool masked = __builtin_amdgcn_readfirstlane(pos) < k0 + kWaveKeys - 1;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      f32x16 s = {};
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lf, ones, s, 0, 0, 0);
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[kk], kf[kt][kk], s, 0, 0, 0);
      // register i of a lane: pair base + (i/4)*8 + hl*4 + i%4, key k0 + kt*32 + ln
      float w[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) w[i] = __builtin_amdgcn_exp2f(s[i] * p.scale_log2);
      if (masked) {
        const int key = k0 + kt * 32 + ln;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int at = __shfl(pos, (i >> 2) * 8 + hl * 4 + (i & 3));
          w[i] = at >= key ? w[i] : 0.0f;
        }
      }
#pragma unroll
      for (int d = 8; d > 0; d >>= 1)
#pragma unroll
        for (int i = 0; i < d; ++i) w[i] += w[i + d];
      sum[kt] += w[0];
    }
  }
  // the two lanes of a key
#pragma unroll
  for (int kt = 0; kt < 2; ++kt) {
    const float total = sum[kt] + __shfl_xor(sum[kt], 32);
    const int key = k0 + kt * 32 + ln;
    if (hl == 0 && key <= last) {
      float* out = p.weights + (int64_t)seq * p.w_sb + (int64_t)kv_head * p.w_sh + key;
      *out = p.accumulate ? *out + total : total;
    }
  }
}

msa_status fail(const char* who, msa_status st, const std::string& msg) {
  set_last_error(std::string(who) + ": " + msg);
  return st;
}

bool aligned(const void* p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

}  // namespace
}  // namespace msa

extern "C" msa_status msa_kv_weights_workspace(msa_plan_t plan, size_t* bytes) {
  if (!plan || !bytes) return msa::fail("msa_kv_weights_workspace", MSA_ERR_INVALID_ARG, "null argument");
  *bytes = 0;
  return MSA_OK;
}

extern "C" msa_status msa_kv_weights(msa_plan_t plan, const void* q, const void* k_cache, const int32_t* block_table,
                                     const float* lse, float* weights, int64_t stride_seq, int64_t stride_head,
                                     int32_t accumulate, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const char* who = "msa_kv_weights";
  const auto invalid = [&](const std::string& msg) { return msa::fail(who, MSA_ERR_INVALID_ARG, msg); };
  (void)workspace, (void)workspace_bytes;
  if (!plan) return invalid("null plan");
  if (plan->hp.has_trees) return msa::fail(who, MSA_ERR_UNSUPPORTED, "the plan was built by msa_plan_tree");
  if (stride_seq < 0 || stride_head < 0) return invalid("strides must be >= 0");
  if (accumulate != 0 && accumulate != 1) return invalid("accumulate must be 0 or 1");
  if (plan->host_only) return invalid("plan was built with MSA_PLAN_HOST_ONLY");
  const msa::HostPlan& hp = plan->hp;
  if (hp.total_q == 0) return MSA_OK;
  if (!q || !k_cache || !block_table || !lse || !weights)
    return invalid("q, k_cache, block_table, lse, weights must be non-null");
  if (!msa::aligned(q, 16) || !msa::aligned(k_cache, 16) || !msa::aligned(block_table, 4) || !msa::aligned(lse, 4) ||
      !msa::aligned(weights, 4))
    return invalid("q and k_cache must be 16-byte, the others 4-byte aligned");
  const msa_shape& s = hp.shape;
  int64_t longest = 0;
  for (int32_t nb : hp.seq_blocks) longest = longest < nb ? nb : longest;
  const int64_t chunks = (longest * msa::kBlockSize + msa::kGroupKeys - 1) / msa::kGroupKeys;
  const int64_t groups = chunks * s.num_seqs * s.num_kv_heads;
  if (hp.total_q * hp.group >= ((int64_t)1 << 31) || groups >= ((int64_t)1 << 31))
    return msa::fail(who, MSA_ERR_UNSUPPORTED, "too many rows or keys for one launch");
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev != plan->device)
    return invalid("current device differs from the plan's device");
  msa::WeightsParams p{};
  p.q = static_cast<const uint16_t*>(q);
  p.k = static_cast<const uint16_t*>(k_cache);
  p.block_table = block_table;
  p.row_pos = plan->d_row_pos;
  p.seq_row0 = plan->d_seq_row0;
  p.lse = lse;
  p.weights = weights;
  p.q_st = s.q_stride_tok;
  p.q_sh = s.q_stride_head;
  p.k_sb = s.k_stride_block;
  p.k_sh = s.k_stride_head;
  p.k_st = s.k_stride_tok;
  p.w_sb = stride_seq;
  p.w_sh = stride_head;
  p.num_seqs = s.num_seqs;
  p.num_q_heads = s.num_q_heads;
  p.num_kv_heads = s.num_kv_heads;
  p.max_blocks = s.max_blocks_per_seq;
  p.group = hp.group;
  p.group_inv = ((1u << 20) + (uint32_t)hp.group - 1) / (uint32_t)hp.group;
  p.inv_scale = 1.0f / s.scale;
  p.scale_log2 = s.scale * 1.4426950408889634f;
  p.accumulate = accumulate;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (s.head_dim == 128)
    hipLaunchKernelGGL(msa::msa_kv_weights_kernel<128>, dim3((uint32_t)groups), dim3(256), 0, st, p);
  else
    hipLaunchKernelGGL(msa::msa_kv_weights_kernel<64>, dim3((uint32_t)groups), dim3(256), 0, st, p);
  return msa::launched(who, "weights", (int)hipGetLastError());
}
