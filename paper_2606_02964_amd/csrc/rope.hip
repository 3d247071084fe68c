// rope.hip -- gfx950 kernel that rotates the packed rows' queries and fresh keys
// by their positions and writes keys and values into the paged cache, in bf16 or
// quantised to 8 bits (msa_rope_append, msa_fp8_append).
//
// One workgroup takes some heads of one slice: the n <= 16 rows of one segment
// that fall into one cache block, as the cache write of append.hip does.
//   * Angles: position times frequency is taken in 64 bits, in turns, and reduced
//     to half a turn there; sine and cosine follow in 32 bits.  A row's pairs are
//     shared by all its heads, so a workgroup works them out once, a pair a thread,
//     and each thread then holds those of its 8 pairs in registers.
//   * D / 16 lanes hold a head's vector, 16 channels each, in two 16-byte chunks
//     that hold both sides of their 8 pairs: chunks c and c + rotary_dim / 16 where
//     pairs are halves apart, neighbours otherwise.  So nothing is exchanged
//     but the maximum of a vector that is quantised (three lane moves).
//   * Quantised rows: the power of two comes from the bits of the largest
//     magnitude (whole numbers, hence exact); scaling by it is exact too, so
//     v_cvt_pk_fp8_f32 rounds once.
//   * V is channel-major in the cache and goes through LDS, as in append.hip.
// Bound by HBM: each number is read once and written once.  8 x 1024 rows, 32 query and
// 8 KV heads, d = 128: 47 us, 4.3 TB/s (into 8 bits 42 us; K and V alone 11 us), 12K rows 59 to 68 us, 4.5 to
// 5.2 TB/s (a device copy: 5.2); single rows by launch and look-ups, 4.5 us, 2048 of them 33 us (8 bits 24),
// whose V numbers go to as many lines each.  (A pass's loads ahead of the angles and of the pass before: the
// same at 1024 rows, 5 to 10% slower at few, by their registers.)
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>

#include "append.h"
#include "errors.h"
#include "forward.h"
#include "fp8.h"
#include "msa_fp8.h"
#include "msa_rope.h"
#include "plan_handle.h"

namespace msa {
namespace {

struct RopeParams {
  const uint16_t* q;    // null: no query heads
  uint16_t* q_out;
  const uint16_t* k_new;
  const uint16_t* v_new;
  const int32_t* block_table;
  const AppendItem* items;
  const int32_t* positions;  // null: the rows' places
  const double* inv_freq;
  void* k_cache;
  void* v_cache;
  uint8_t* k_scale;
  uint8_t* v_scale;
  int64_t q_st, q_sh, qo_st, qo_sh;
  int64_t kn_st, kn_sh, vn_st, vn_sh;
  int64_t k_sb, k_sh, k_st;
  int64_t v_sb, v_sh, v_sd;
  int32_t num_q_heads;  // 0 if q is null
  int32_t num_kv_heads;
  int32_t max_blocks;
  int32_t num_blocks;
  int32_t half;         // pairs of a head: rotary_dim / 2
  int32_t head_groups;  // workgroups that share a slice's heads
  int32_t total_q;      // rows of all slices (launch_rope's choice of head_groups)
  float amplitude;
};

enum { kNoPairs, kHalves, kNeighbours };

// the two chunks of 8 channels of a lane in 32 bits
__device__ __forceinline__ void unpack(const uint4& u, float* x) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
typedef __bf16 bf16_pair __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint4 pack_bf16(const float* x) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bf16_pair v = {(__bf16)x[2 * i], (__bf16)x[2 * i + 1]};
    w[i] = __builtin_bit_cast(uint32_t, v);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint2 pack_fp8(const float* x, float inv) {
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i] * inv, x[4 * i + 1] * inv, 0, false);
    w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2] * inv, x[4 * i + 3] * inv, v, true);
  }
  return make_uint2(w[0], w[1]);
}

template <int kCtrl>
__device__ __forceinline__ float dpp_max(float x) {
  return fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), kCtrl, 0xf, 0xf, true)));
}
// byte of the power of two of the vector that these D / 16 lanes hold 16 numbers each of
template <int D>
__device__ __forceinline__ uint32_t scale_byte(const float* x) {
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) m = fmaxf(m, __builtin_fabsf(x[i]));
  m = dpp_max<0xB1>(m);                    // the neighbour
  m = dpp_max<0x4E>(m);                    // the other pair of four
  if (D == 128) m = dpp_max<0x141>(m);     // the other four of eight
  return fp8_scale_byte(__float_as_uint(m));
}

template <int D, int kPairs, bool kFp8>
__global__ __launch_bounds__(256) void msa_rope_kernel(RopeParams p) {
  constexpr int kLanes = D / 16;           // lanes of a head's vector
  constexpr int kVectors = 256 / kLanes;   // vectors a pass
  constexpr int kPitch = kFp8 ? D + 16 : D + 8;  // elements of a V row in LDS
  typedef typename std::conditional<kFp8, uint8_t, uint16_t>::type cache_t;
  __shared__ __align__(16) float s_cos[16][D / 2 + 4], s_sin[16][D / 2 + 4];  // (rows 16 bytes apart in the banks)
  __shared__ __align__(16) cache_t s_v[kVectors][kPitch];

  const uint32_t item = blockIdx.x / (uint32_t)p.head_groups;
  const int group = (int)(blockIdx.x - item * (uint32_t)p.head_groups);
  const AppendItem it = p.items[item];
  const int32_t blk = p.block_table[(int64_t)it.seq * p.max_blocks + it.pos0 / 16];
  const bool stored = blk >= 0 && blk < p.num_blocks;  // uniform over the workgroup
  const int off0 = it.pos0 % 16, n = it.n, tid = threadIdx.x;

  if constexpr (kPairs != kNoPairs) {
    constexpr int kPer = D / 2;  // threads of a row's angles
    for (int r = tid / kPer; r < n; r += 256 / kPer) {
      const int i = tid % kPer;
      if (i < p.half) {
        const int32_t pos = p.positions ? p.positions[it.row0 + r] : it.pos0 + r;
        double turns = (double)pos * p.inv_freq[i] * 0.15915494309189533577;
        turns -= __builtin_rint(turns);
        float s, c;
        sincospif(2.0f * (float)turns, &s, &c);
        s_cos[r][i] = c * p.amplitude;
        s_sin[r][i] = s * p.amplitude;
      }
    }
    __syncthreads();
  }

  // this workgroup's heads, K/V heads before query heads; a pass takes `per` of them
  const int kv0 = p.num_kv_heads * group / p.head_groups, kv1 = p.num_kv_heads * (group + 1) / p.head_groups;
  const int q0 = (int)((int64_t)p.num_q_heads * group / p.head_groups);
  const int q1 = (int)((int64_t)p.num_q_heads * (group + 1) / p.head_groups);
  const int nkv = kv1 - kv0, heads = nkv + q1 - q0;
  const int slots = n * kLanes, per = 256 / slots;
  const int first = tid / slots, slot = tid - first * slots;
  const int row = slot / kLanes, lane = slot % kLanes;
  const bool active = first < per;
  const int64_t r = (int64_t)it.row0 + row;
  const bool turned = kPairs != kNoPairs && 16 * lane < 2 * p.half;
  // channels of the lane's two chunks (V: neighbours)
  const int ca = turned && kPairs == kHalves ? 8 * lane : 16 * lane;
  const int cb = turned && kPairs == kHalves ? 8 * lane + p.half : 16 * lane + 8;
  float co[8], si[8];
  if constexpr (kPairs != kNoPairs) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      co[i] = turned ? s_cos[row][8 * lane + i] : 1.0f;
      si[i] = turned ? s_sin[row][8 * lane + i] : 0.0f;
    }
  }
  auto turn = [&](float* x) {
    if constexpr (kPairs == kNoPairs) return;
    if (!turned) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int u = kPairs == kHalves ? i : 2 * i, w = kPairs == kHalves ? i + 8 : 2 * i + 1;
      const float a = x[u], b = x[w];
      x[u] = a * co[i] - b * si[i];
      x[w] = b * co[i] + a * si[i];
    }
  };

  // the row's places (in vector registers: with all strides in scalar ones the loop spills them)
  const uint16_t* q_row = p.q + r * p.q_st + q0 * p.q_sh;
  uint16_t* qo_row = p.q_out + r * p.qo_st + q0 * p.qo_sh;
  const uint16_t* k_row = p.k_new + r * p.kn_st + kv0 * p.kn_sh;
  const uint16_t* v_row = p.v_new + r * p.vn_st + kv0 * p.vn_sh + 16 * lane;
  cache_t* kc_row = static_cast<cache_t*>(p.k_cache) + (int64_t)blk * p.k_sb + kv0 * p.k_sh + (int64_t)(off0 + row) * p.k_st;
  cache_t* vc = static_cast<cache_t*>(p.v_cache) + (int64_t)blk * p.v_sb + kv0 * p.v_sh;
  const int64_t powers = ((int64_t)blk * p.num_kv_heads + kv0) * 16 + off0 + row;
  for (int h0 = 0; h0 < heads; h0 += per) {
    const int h = h0 + first;
    if (active && h < heads && h >= nkv) {
      const int64_t g = h - nkv;
      const uint16_t* src = q_row + g * p.q_sh;
      uint16_t* dst = qo_row + g * p.qo_sh;
      const uint4 a = *reinterpret_cast<const uint4*>(src + ca), b = *reinterpret_cast<const uint4*>(src + cb);
      if (turned) {
        float x[16];
        unpack(a, x);
        unpack(b, x + 8);
        turn(x);
        *reinterpret_cast<uint4*>(dst + ca) = pack_bf16(x);
        *reinterpret_cast<uint4*>(dst + cb) = pack_bf16(x + 8);
      } else {
        *reinterpret_cast<uint4*>(dst + ca) = a;
        *reinterpret_cast<uint4*>(dst + cb) = b;
      }
    }
    if (h0 >= nkv || !stored) continue;  // (uniform: no K/V head in this pass)
    const int ng = nkv - h0 < per ? nkv - h0 : per;  // K/V heads of the pass
    if (active && h < nkv) {
      const int64_t g = h;
      const uint16_t* ks = k_row + g * p.kn_sh;
      const uint16_t* vs = v_row + g * p.vn_sh;
      const uint4 ka = *reinterpret_cast<const uint4*>(ks + ca), kb = *reinterpret_cast<const uint4*>(ks + cb);
      const uint4 va = *reinterpret_cast<const uint4*>(vs), vb = *reinterpret_cast<const uint4*>(vs + 8);
      cache_t* kd = kc_row + g * p.k_sh;
      cache_t* sv = s_v[first * n + row] + 16 * lane;
      float x[16];
      if constexpr (kFp8) {
        const int64_t at = powers + g * 16;
        unpack(ka, x);
        unpack(kb, x + 8);
        turn(x);
        uint32_t s = scale_byte<D>(x);
        if (lane == 0) p.k_scale[at] = (uint8_t)s;
        float inv = __uint_as_float((254u - s) << 23);
        const uint2 qa = pack_fp8(x, inv), qb = pack_fp8(x + 8, inv);
        if (cb == ca + 8) {
          *reinterpret_cast<uint4*>(kd + ca) = make_uint4(qa.x, qa.y, qb.x, qb.y);
        } else {
          *reinterpret_cast<uint2*>(kd + ca) = qa;
          *reinterpret_cast<uint2*>(kd + cb) = qb;
        }
        unpack(va, x);
        unpack(vb, x + 8);
        s = scale_byte<D>(x);
        if (lane == 0) p.v_scale[at] = (uint8_t)s;
        inv = __uint_as_float((254u - s) << 23);
        const uint2 wa = pack_fp8(x, inv), wb = pack_fp8(x + 8, inv);
        *reinterpret_cast<uint4*>(sv) = make_uint4(wa.x, wa.y, wb.x, wb.y);
      } else {
        if (turned) {
          unpack(ka, x);
          unpack(kb, x + 8);
          turn(x);
          *reinterpret_cast<uint4*>(kd + ca) = pack_bf16(x);
          *reinterpret_cast<uint4*>(kd + cb) = pack_bf16(x + 8);
        } else {
          *reinterpret_cast<uint4*>(kd + ca) = ka;
          *reinterpret_cast<uint4*>(kd + cb) = kb;
        }
        *reinterpret_cast<uint4*>(sv) = va;
        *reinterpret_cast<uint4*>(sv + 8) = vb;
      }
    }
    __syncthreads();
    // V out, one half block (8 tokens) at a time
    cache_t* vd = vc + (int64_t)h0 * p.v_sh;
#pragma unroll 1
    for (int hb = 0; hb < 2; ++hb) {
      const int lo = off0 > 8 * hb ? off0 : 8 * hb;
      const int hi = off0 + n < 8 * hb + 8 ? off0 + n : 8 * hb + 8;
      if (lo >= hi) continue;  // the slice misses this half
      const int w = hi - lo;
      if (w == 8) {
#pragma unroll 1
        for (int idx = tid; idx < ng * D; idx += 256) {
          const int c = idx % D, g = idx / D;
          cache_t e[8];
#pragma unroll
          for (int t = 0; t < 8; ++t) e[t] = s_v[g * n + lo - off0 + t][c];
          cache_t* to = vd + (int64_t)g * p.v_sh + (int64_t)c * p.v_sd + 8 * hb;
          if constexpr (kFp8) {
            uint32_t u[2];
#pragma unroll
            for (int t = 0; t < 2; ++t)
              u[t] = (uint32_t)e[4 * t] | (uint32_t)e[4 * t + 1] << 8 | (uint32_t)e[4 * t + 2] << 16 | (uint32_t)e[4 * t + 3] << 24;
            *reinterpret_cast<uint2*>(to) = make_uint2(u[0], u[1]);
          } else {
            uint32_t u[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) u[t] = (uint32_t)e[2 * t] | (uint32_t)e[2 * t + 1] << 16;
            *reinterpret_cast<uint4*>(to) = make_uint4(u[0], u[1], u[2], u[3]);
          }
        }
      } else {
#pragma unroll 1
        for (int idx = tid; idx < ng * D * w; idx += 256) {
          const int t = lo + idx % w, c = (idx / w) % D, g = idx / (w * D);
          vd[(int64_t)g * p.v_sh + (int64_t)c * p.v_sd + t] = s_v[g * n + t - off0][c];
        }
      }
    }
    __syncthreads();
  }
}

template <int D>
int launch_rope(RopeParams p, int pairs, bool fp8, int num_items, hipStream_t s) {
  // Workgroups that share a slice's heads: four passes each, since a workgroup's look-ups and angles cost as much as a
  // pass, but some 1024 in all where there is work for a pass each (32 query, 8 KV heads, d = 128, bf16, us, with
  // two KV heads and their queries each / by this rule: 1 row of 512 sequences 13.0 / 10.2, of 2048 46.4 / 33.3; 1024 rows
  // of 8 47.2 / 46.9; into 8 bits 13.7 / 9.5, 44.3 / 23.6, 42.1 / 46; d = 64, 16 heads: 2048 rows 64 / 23).
  // (Stores past the caches take a twentieth off this launch, and add as much to the attention behind it,
  // which then finds no q in them: 8 x 1024 rows 44.5 / 46.9, with msa_forward 225.3 / 223.2.)
  const int64_t passes = ((int64_t)p.total_q * (p.num_q_heads + p.num_kv_heads) * (D / 16) / num_items + 255) / 256;
  const int64_t most = std::max<int64_t>(1, std::min<int64_t>((1 << 23) / num_items, p.num_kv_heads));
  const int64_t groups = std::max<int64_t>(passes / 4, std::min<int64_t>(passes, 1024 / num_items));
  p.head_groups = (int32_t)std::max<int64_t>(1, std::min(groups, most));
  while (p.num_kv_heads % p.head_groups != 0) --p.head_groups;  // as many each (8 heads of 8 x 1024 rows, 8 bits: in 5 parts 46 us)
  const dim3 grid((uint32_t)num_items * (uint32_t)p.head_groups), block(256);
  if (fp8) {
    if (pairs == kNoPairs) hipLaunchKernelGGL((msa_rope_kernel<D, kNoPairs, true>), grid, block, 0, s, p);
    else if (pairs == kHalves) hipLaunchKernelGGL((msa_rope_kernel<D, kHalves, true>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((msa_rope_kernel<D, kNeighbours, true>), grid, block, 0, s, p);
  } else {
    if (pairs == kHalves) hipLaunchKernelGGL((msa_rope_kernel<D, kHalves, false>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((msa_rope_kernel<D, kNeighbours, false>), grid, block, 0, s, p);
  }
  return (int)hipGetLastError();
}

msa_status refuse(const char* who, msa_status st, const std::string& what) {
  set_last_error(std::string(who) + ": " + what);
  return st;
}

bool aligned(const void* x, uintptr_t a) { return reinterpret_cast<uintptr_t>(x) % a == 0; }

// the checks and the launch of both entry points; rope null: no rotation
msa_status write_rows(const char* who, msa_plan_t plan, const msa_rope* rope, const void* q, int64_t q_st, int64_t q_sh,
                      void* q_out, int64_t qo_st, int64_t qo_sh, const void* k_new, const void* v_new, int64_t kn_st,
                      int64_t kn_sh, int64_t vn_st, int64_t vn_sh, const int32_t* positions, const int32_t* block_table,
                      void* k_cache, void* v_cache, uint8_t* k_scale, uint8_t* v_scale, void* hip_stream) {
  if (!plan) return refuse(who, MSA_ERR_INVALID_ARG, "null plan");
  auto ok_stride = [](int64_t x) { return x > 0 && x % 8 == 0; };
  if (!ok_stride(kn_st) || !ok_stride(kn_sh) || !ok_stride(vn_st) || !ok_stride(vn_sh) ||
      (q && (!ok_stride(q_st) || !ok_stride(q_sh) || !ok_stride(qo_st) || !ok_stride(qo_sh))))
    return refuse(who, MSA_ERR_INVALID_ARG, "strides must be positive multiples of 8 elements");
  if (plan->host_only) return refuse(who, MSA_ERR_INVALID_ARG, "plan was built with MSA_PLAN_HOST_ONLY");
  const HostPlan& hp = plan->hp;
  const msa_shape& s = hp.shape;
  if (!k_scale != !v_scale) return refuse(who, MSA_ERR_INVALID_ARG, "k_scale and v_scale go together");
  if (rope) {
    if (rope->reserved != 0) return refuse(who, MSA_ERR_INVALID_ARG, "rope.reserved must be zero");
    if (rope->pairs != MSA_ROPE_HALF && rope->pairs != MSA_ROPE_INTERLEAVED)
      return refuse(who, MSA_ERR_INVALID_ARG, "rope.pairs is neither MSA_ROPE_HALF nor MSA_ROPE_INTERLEAVED");
    if (rope->rotary_dim < 2 || rope->rotary_dim > s.head_dim || rope->rotary_dim % 2 != 0)
      return refuse(who, MSA_ERR_INVALID_ARG, "rope.rotary_dim must be even and within [2, head_dim]");
    if (rope->rotary_dim % 16 != 0)
      return refuse(who, MSA_ERR_UNSUPPORTED, "rope.rotary_dim must be a multiple of 16");
    if (!std::isfinite(rope->amplitude)) return refuse(who, MSA_ERR_INVALID_ARG, "rope.amplitude must be finite");
  }
  const std::string strides = k_scale ? fp8_strides(s) : std::string();
  if (!strides.empty()) return refuse(who, MSA_ERR_INVALID_ARG, strides);
  if (hp.total_q == 0) return MSA_OK;
  if (!k_new || !v_new || !block_table || !k_cache || !v_cache || (q && !q_out) || (rope && !rope->inv_freq))
    return refuse(who, MSA_ERR_INVALID_ARG, "a pointer that must be non-null is null");
  if (!aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(q, 16) ||
      (q && !aligned(q_out, 16)) || !aligned(k_scale, 16) || !aligned(v_scale, 16))
    return refuse(who, MSA_ERR_INVALID_ARG, "q, k, v, caches and scales must be 16-byte aligned");
  if (!aligned(block_table, 4) || !aligned(positions, 4) || (rope && !aligned(rope->inv_freq, 8)))
    return refuse(who, MSA_ERR_INVALID_ARG, "block_table and positions must be 4-byte and inv_freq 8-byte aligned");
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev != plan->device)
    return refuse(who, MSA_ERR_INVALID_ARG, "current device differs from the plan's device");
  RopeParams p{};
  p.q = static_cast<const uint16_t*>(q);
  p.q_out = static_cast<uint16_t*>(q_out);
  p.k_new = static_cast<const uint16_t*>(k_new);
  p.v_new = static_cast<const uint16_t*>(v_new);
  p.block_table = block_table;
  p.items = plan->d_append;
  p.positions = positions;
  p.k_cache = k_cache;
  p.v_cache = v_cache;
  p.k_scale = k_scale;
  p.v_scale = v_scale;
  p.q_st = q_st, p.q_sh = q_sh, p.qo_st = qo_st, p.qo_sh = qo_sh;
  p.kn_st = kn_st, p.kn_sh = kn_sh, p.vn_st = vn_st, p.vn_sh = vn_sh;
  p.k_sb = s.k_stride_block, p.k_sh = s.k_stride_head, p.k_st = s.k_stride_tok;
  p.v_sb = s.v_stride_block, p.v_sh = s.v_stride_head, p.v_sd = s.v_stride_dim;
  p.num_q_heads = q ? s.num_q_heads : 0;
  p.num_kv_heads = s.num_kv_heads;
  p.max_blocks = s.max_blocks_per_seq;
  p.num_blocks = s.num_blocks;
  p.total_q = (int32_t)hp.total_q;
  int pairs = kNoPairs;
  if (rope) {
    p.inv_freq = rope->inv_freq;
    p.half = rope->rotary_dim / 2;
    p.amplitude = rope->amplitude;
    pairs = rope->pairs == MSA_ROPE_HALF ? kHalves : kNeighbours;
  }
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const int items = (int)hp.append.size();
  return launched(who, "write", s.head_dim == 128 ? launch_rope<128>(p, pairs, k_scale != nullptr, items, st)
                                                  : launch_rope<64>(p, pairs, k_scale != nullptr, items, st));
}

}  // namespace
}  // namespace msa

extern "C" msa_status msa_rope_append(msa_plan_t plan, const msa_rope* rope, const void* q, int64_t q_stride_tok,
                                      int64_t q_stride_head, void* q_out, int64_t q_out_stride_tok,
                                      int64_t q_out_stride_head, const void* k_new, const void* v_new,
                                      int64_t k_new_stride_tok, int64_t k_new_stride_head, int64_t v_new_stride_tok,
                                      int64_t v_new_stride_head, const int32_t* positions, const int32_t* block_table,
                                      void* k_cache, void* v_cache, uint8_t* k_scale, uint8_t* v_scale,
                                      void* hip_stream) {
  if (!rope) return msa::refuse("msa_rope_append", MSA_ERR_INVALID_ARG, "null rope");
  return msa::write_rows("msa_rope_append", plan, rope, q, q_stride_tok, q_stride_head, q_out, q_out_stride_tok,
                         q_out_stride_head, k_new, v_new, k_new_stride_tok, k_new_stride_head, v_new_stride_tok,
                         v_new_stride_head, positions, block_table, k_cache, v_cache, k_scale, v_scale, hip_stream);
}

extern "C" msa_status msa_fp8_append(msa_plan_t plan, const void* k_new, const void* v_new, int64_t k_new_stride_tok,
                                     int64_t k_new_stride_head, int64_t v_new_stride_tok, int64_t v_new_stride_head,
                                     const int32_t* block_table, void* k_cache, void* v_cache, uint8_t* k_scale,
                                     uint8_t* v_scale, void* hip_stream) {
  if (!k_scale || !v_scale) return msa::refuse("msa_fp8_append", MSA_ERR_INVALID_ARG, "k_scale and v_scale must be non-null");
  return msa::write_rows("msa_fp8_append", plan, nullptr, nullptr, 0, 0, nullptr, 0, 0, k_new, v_new, k_new_stride_tok,
                         k_new_stride_head, v_new_stride_tok, v_new_stride_head, nullptr, block_table, k_cache, v_cache,
                         k_scale, v_scale, hip_stream);
}
