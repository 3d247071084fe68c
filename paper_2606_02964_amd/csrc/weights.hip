// weights.hip -- the attention weight each cached key receives from a plan's
// query rows (msa_kv_weights).
//
//   w[j] = sum over the rows r that see key j, and the query heads h of a KV
//          head's group, of exp(scale q_rh k_j - lse_rh)
//
// The softmax's statistics are known (msa_forward's lse), so a key's sum needs
// one pass over the rows and no other key.  Rows are taken 32 (row, head) pairs of a
// KV head at a time:
//   - S = Q K^T on v_mfma_f32_32x32x16_bf16 with Q as the A operand: each lane
//     then holds 16 rows of ONE key (a column of S), so a key's sum stays in its
//     lane; the lane pair (l, l + 32) of a key is joined once at the end;
//   - the subtraction of lse is one more MFMA: its A operand holds -lse / scale in
//     three bf16 terms (24 bits, as much as the fp32 lse has), its B operand
//     ones.  The score registers then hold (q k - lse / scale) and a weight is
//     exp2 of that times scale * log2(e).  A row that is to give no weight (no such
//     row, or lse = -inf) has -inf there, and costs nothing further;
//   - the causal limit is applied only on the tiles that hold a row before the
//     wave's last key.
// Two kernels, by the pairs of a sequence's rows and a KV head's group:
//   msa_kv_weights_stream, up to 32 pairs (decoding): the rows stay in registers
//   and each wave streams a run of keys, the next 32 on their way while it
//   computes.  The plan deals out the runs, so that one long sequence among short
//   ones is spread as any other.  Bound by reading K: 64 rows over 1K to 8K keys each, 32
//   query and 8 KV heads of 128, 122 us, 5.1 TB/s; one row over 8K 6.1 us, over 32K
//   14.8 (by the other kernel 6.9 and 17.9; 16 rows over 8K at d = 64, 16 heads,
//   33.7 and 51.7).
//   msa_kv_weights_tiles, more: a workgroup holds 256 keys in registers, 64 a wave,
//   and streams the pairs' Q, lse and positions through a ring of four tiles in
//   LDS, filled by direct copies that run three tiles ahead (each wave its share,
//   one barrier a tile).  Read by every wave for itself, Q took four times the reads,
//   each over 32 cache lines.  The plan deals out the tiles (see plan_weights); where
//   keys have several items, their sums go through the workspace and are added in
//   order.  Prompts of 4099 and less, three of them, 32 heads: 94 us with the join;
//   one of 16384 1.06-1.11 ms, 990-1040 TFLOP/s.  Bound by vector instructions and
//   MFMAs: a tile of 32 pairs x 64 keys
//   takes a wave 17 MFMAs of 32 cycles and about 150 vector instructions, 32 of them
//   exponentials of 8 cycles, beside them.
// Sums are in fp32, 16 rows of a tile added pairwise and then to the running sum;
// no atomics, so equal calls give equal bits.
#include <hip/hip_runtime.h>

#include <algorithm>
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

typedef __attribute__((address_space(3))) void lds_void_t;

constexpr int kWaveKeys = kGroupKeys / 4;
constexpr int kRing = 4;  // tiles in LDS
constexpr int64_t kMostGroups = ((int64_t)1 << 32) / 256;  // workgroups of a launch: its threads are counted in 32 bits

struct WeightsParams {
  const uint16_t* q;
  const uint16_t* k;
  const int32_t* block_table;
  const int32_t* row_pos;
  const int32_t* seq_row0;
  const float* lse;
  float* weights;
  float* sums;  // [slots][KV heads][kGroupKeys]
  const StreamItem* streams;
  const WeightsItem* items;
  const WeightsJoin* joins;
  int64_t q_st, q_sh, k_sb, k_sh, k_st, w_sb, w_sh;
  int32_t num_q_heads, num_kv_heads, max_blocks, group;
  uint32_t group_inv; // ceil(2^20 / G): r / G = r * group_inv >> 20 for r < 288
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

__device__ __forceinline__ bf16x8 all_of(float x) {
  bf16x8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (__bf16)x;
  return v;
}

// the sum of a lane's 16 weights of one key; pos: position of pair `lane % 32` of the tile
__device__ __forceinline__ float key_sum(const f32x16& s, float scale_log2, bool masked, int pos, int key, int hl) {
  float w[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) w[i] = __builtin_amdgcn_exp2f(s[i] * scale_log2);
  if (masked) {
    // register i of a lane: pair (i/4)*8 + hl*4 + i%4
#pragma unroll
    for (int i = 0; i < 16; ++i) w[i] = __shfl(pos, (i >> 2) * 8 + hl * 4 + (i & 3)) >= key ? w[i] : 0.0f;
  }
#pragma unroll
  for (int d = 8; d > 0; d >>= 1)
#pragma unroll
    for (int i = 0; i < d; ++i) w[i] += w[i + d];
  return w[0];
}

// ---- up to 32 pairs ----

template <int D>
__global__ __launch_bounds__(256, 3) void msa_kv_weights_stream_kernel(WeightsParams p) {
  const uint32_t item = blockIdx.x / (uint32_t)p.num_kv_heads;
  const int kv_head = (int)(blockIdx.x - item * (uint32_t)p.num_kv_heads);
  const StreamItem it = p.streams[item];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, hl = lane >> 5, ln = lane & 31;
  const int seq = it.seq, row0 = it.row0, G = p.group, n = it.nrows * G;
  const int64_t begin = (int64_t)it.key0 + wave * it.wave_keys;
  if (begin > it.last) return;
  const int k0 = (int)begin, k1 = min(it.wave_keys, it.last + 1 - k0) + k0;

  // the wave's block ids, one a lane
  const int32_t* table = p.block_table + (int64_t)seq * p.max_blocks + (k0 >> 4);
  const int32_t ids = k0 + lane * kBlockSize < k1 ? table[lane] : 0;

  const int dt = (int)((uint32_t)ln * p.group_inv >> 20);
  const bool valid = ln < n;
  const int tok = row0 + (valid ? dt : 0), head = kv_head * G + (valid ? ln - dt * G : 0);
  const int pos = p.row_pos[tok];
  bf16x8 qf[D / 16];
  const uint16_t* src = p.q + (int64_t)tok * p.q_st + (int64_t)head * p.q_sh + hl * 8;
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) qf[kk] = *reinterpret_cast<const bf16x8*>(src + kk * 16);
  float l = p.lse[(int64_t)tok * p.num_q_heads + head];
  if (!valid || l == -__builtin_inff()) l = __builtin_inff();
  const bf16x8 lf = three_terms(-l * p.inv_scale, hl == 0), ones = all_of(1.0f);
  if (!valid) {  // (its scores are -inf whatever Q holds, but for NaN)
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) qf[kk] = all_of(0.0f);
  }
  const int first_pos = __builtin_amdgcn_readfirstlane(pos);
  float* out = p.weights + (int64_t)seq * p.w_sb + (int64_t)kv_head * p.w_sh;

  // B operand: key base + ln, channels kk*16 + hl*8 .. +8 (a key behind the last one reads the last one's row)
  const uint16_t* kbase = p.k + (int64_t)kv_head * p.k_sh + hl * 8;
  auto load = [&](bf16x8 (&kf)[D / 16], float& old, int base) __attribute__((always_inline)) {
    const int key = min(base + ln, k1 - 1);
    const int b = (base - k0) >> 4;
    const int32_t id0 = __builtin_amdgcn_readlane(ids, b), id1 = __builtin_amdgcn_readlane(ids, min(b + 1, 63));
    const int32_t blk = (key - base) >> 4 ? id1 : id0;
    const uint16_t* at = kbase + (int64_t)blk * p.k_sb + (int64_t)(key & 15) * p.k_st;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) kf[kk] = *reinterpret_cast<const bf16x8*>(at + kk * 16);
    old = p.accumulate ? out[key] : 0.0f;
  };
  bf16x8 kf[2][D / 16];
  float old[2];
  auto tile = [&](bf16x8 (&now)[D / 16], float was, bf16x8 (&then)[D / 16], float& next, int base)
      __attribute__((always_inline)) {
    if (base + 32 < k1) load(then, next, base + 32);
    f32x16 s = {};
    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lf, ones, s, 0, 0, 0);
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[kk], now[kk], s, 0, 0, 0);
    float sum = key_sum(s, p.scale_log2, first_pos < base + 31, pos, base + ln, hl);
    sum += __shfl_xor(sum, 32);
    if (hl == 0 && base + ln < k1) out[base + ln] = was + sum;
  };
  load(kf[0], old[0], k0);
  for (int base = k0; base < k1; base += 64) {
    tile(kf[0], old[0], kf[1], old[1], base);
    if (base + 32 < k1) tile(kf[1], old[1], kf[0], old[0], base + 32);
  }
}

// ---- more ----

// 16 or 4 bytes a lane from global memory straight into LDS at lds + 16 (4) * lane
// (M0 holds the wave's base); completion is tracked by vmcnt, which the
// kernel waits for itself
__device__ __forceinline__ void copy16(const void* src, void* lds) {
  const uint32_t l = (uint32_t)(uintptr_t)(lds_void_t*)lds;
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(src), "{m0}"(l) : "memory");
}
__device__ __forceinline__ void copy4(const void* src, void* lds) {
  const uint32_t l = (uint32_t)(uintptr_t)(lds_void_t*)lds;
  asm volatile("s_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(src), "{m0}"(l) : "memory");
}

// s_waitcnt's operand: at most n loads or copies outstanding
constexpr int wait_loads(int n) { return (n & 15) | (7 << 4) | (15 << 8) | ((n >> 4) << 14); }

template <int D>
struct QRing {
  static constexpr int kTile = kPairs * D * 2;
  char q[kRing][kTile];             // [pair][D], 16-byte chunks XOR-swizzled
  uint32_t more[kRing][4][64];      // for each wave: 32 lse, 32 positions
};

template <int D>
__global__ __launch_bounds__(256, 2) void msa_kv_weights_tiles_kernel(WeightsParams p) {
  __shared__ __attribute__((aligned(1024))) QRing<D> ring;
  const uint32_t item = blockIdx.x / (uint32_t)p.num_kv_heads;
  const int kv_head = (int)(blockIdx.x - item * (uint32_t)p.num_kv_heads);
  const WeightsItem it = p.items[item];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, hl = lane >> 5, ln = lane & 31;
  const int row0 = it.row0, last = it.last, t_begin = it.tile0, t_end = it.tile1;
  const int G = p.group, n = it.nrows * G, tiles_all = (n + kPairs - 1) / kPairs;
  const int32_t* row_pos = p.row_pos + row0;
  const int k0 = it.key0 + wave * kWaveKeys;

  // Copies: a wave's share of a tile is 8 pairs (two copies, or one at d = 64, of 16 bytes a
  // lane), and lse and position of all 32.  Pairs behind the last one read the last one's.
  constexpr int kChunks = D / 8;           // 16-byte chunks of a pair
  constexpr int kPerCopy = 64 / kChunks;   // pairs of a copy
  constexpr int kCopies = 8 / kPerCopy;
  auto swizzle = [](int r) { return (D == 128 ? r : r >> 1) & (kChunks - 1); };
  // Sources of the lane's copies from the next tile.  From tile to tile each moves on by 32 pairs,
  // that is step_rows rows and step_heads heads, and by one more row where the heads pass G.
  const int step_rows = kPairs / G, step_heads = kPairs - step_rows * G;
  int next = t_begin;
  const char* from[kCopies + 1];
  int head_at[kCopies + 1];
  const int64_t q_step = (step_rows * p.q_st + step_heads * p.q_sh) * 2, q_wrap = (p.q_st - G * p.q_sh) * 2;
  const int64_t l_step = hl ? step_rows * 4 : ((int64_t)step_rows * p.num_q_heads + step_heads) * 4;
  const int64_t l_wrap = hl ? 4 : ((int64_t)p.num_q_heads - G) * 4;
  auto aim = [&](int t, int most) __attribute__((always_inline)) {  // at tile t, pairs behind `most` at that one
#pragma unroll
    for (int c = 0; c <= kCopies; ++c) {
      const int r = c < kCopies ? wave * 8 + c * kPerCopy + lane / kChunks : ln;
      const int first_row = t * kPairs / G, off = t * kPairs - first_row * G + min(r, most);
      const int dt = (int)((uint32_t)off * p.group_inv >> 20), tok = first_row + dt;
      head_at[c] = off - dt * G;
      const int head = kv_head * G + head_at[c];
      if (c < kCopies)
        from[c] = reinterpret_cast<const char*>(p.q + (int64_t)(row0 + tok) * p.q_st + (int64_t)head * p.q_sh +
                                                ((lane % kChunks) ^ swizzle(r)) * 8);
      else
        from[c] = hl ? reinterpret_cast<const char*>(row_pos + tok)
                     : reinterpret_cast<const char*>(p.lse + (int64_t)(row0 + tok) * p.num_q_heads + head);
    }
  };
  auto copy = [&]() __attribute__((always_inline)) {
    const int slot = __builtin_amdgcn_readfirstlane(next & (kRing - 1));
    if (next == tiles_all - 1) aim(next, n - 1 - next * kPairs);  // the sequence's last tile may be short
#pragma unroll
    for (int c = 0; c < kCopies; ++c) copy16(from[c], ring.q[slot] + (wave * 8 + c * kPerCopy) * D * 2);
    copy4(from[kCopies], ring.more[slot][wave]);
    ++next;
    if (next >= t_end) return;  // (behind the last tile it is copied again, so that each step waits for as many)
#pragma unroll
    for (int c = 0; c <= kCopies; ++c) from[c] += c < kCopies ? q_step : l_step;
    if (step_heads != 0) {
#pragma unroll
      for (int c = 0; c <= kCopies; ++c) {
        head_at[c] += step_heads;
        const bool wraps = head_at[c] >= G;
        head_at[c] -= wraps ? G : 0;
        from[c] += wraps ? (c < kCopies ? q_wrap : l_wrap) : 0;
      }
    }
  };
  constexpr int kEach = kCopies + 1;  // copies of a wave and tile

  aim(t_begin, kPairs - 1);
  copy();
  copy();
  copy();

  // B operand: key k0 + kt*32 + ln, channels kk*16 + hl*8 .. +8 (behind the last one: that one, not written)
  bf16x8 kf[2][D / 16];
  const bf16x8 ones = all_of(1.0f);
  int32_t blk[2];
#pragma unroll
  for (int kt = 0; kt < 2; ++kt)
    blk[kt] = p.block_table[(int64_t)it.seq * p.max_blocks + (min(k0 + kt * 32 + ln, last) >> 4)];
#pragma unroll
  for (int kt = 0; kt < 2; ++kt) {
    const uint16_t* src = p.k + (int64_t)blk[kt] * p.k_sb + (int64_t)kv_head * p.k_sh +
                          (int64_t)(min(k0 + kt * 32 + ln, last) & 15) * p.k_st + hl * 8;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) kf[kt][kk] = *reinterpret_cast<const bf16x8*>(src + kk * 16);
  }
  float sum[2] = {0.0f, 0.0f};
  __builtin_amdgcn_s_waitcnt(wait_loads(0));  // K has arrived (the compiler would wait for it, and for all copies, in the loop)
  {
    // Tile t has arrived once no more than the copies of two tiles are outstanding; behind the
    // barrier every wave's share has, and tile t - 1 is read.
    auto advance = [&]() __attribute__((always_inline)) {
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(2 * kEach) : "memory");
      copy();
    };
    // the operands of tile t, -lse / scale and Q; and the positions of the lane's 16 score rows,
    // where some may not see all of the wave's keys
    int pos[16];
    auto read = [&](int t, bool masked, bf16x8& lf, bf16x8 (&qf)[D / 16]) __attribute__((always_inline)) {
      const int slot = t & (kRing - 1);
      float l = __uint_as_float(ring.more[slot][wave][ln]);
      if (masked) {
#pragma unroll
        for (int i = 0; i < 16; i += 4) {  // register i of a lane: pair (i/4)*8 + hl*4 + i%4
          const uint4 x = *reinterpret_cast<const uint4*>(&ring.more[slot][wave][32 + i * 2 + hl * 4]);
          pos[i] = (int)x.x;
          pos[i + 1] = (int)x.y;
          pos[i + 2] = (int)x.z;
          pos[i + 3] = (int)x.w;
        }
      }
      if (t * kPairs + ln >= n || l == -__builtin_inff()) l = __builtin_inff();
      lf = three_terms(-l * p.inv_scale, hl == 0);
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk)
        qf[kk] = *reinterpret_cast<const bf16x8*>(ring.q[slot] + ln * D * 2 + (((kk * 2 + hl) ^ swizzle(ln)) * 16));
    };
    auto position = [&](int t, int pair) {  // uniform
      return __builtin_amdgcn_readfirstlane((int)ring.more[t & (kRing - 1)][wave][32 + pair]);
    };
    auto is_masked = [&](int t) { return position(t, 0) < k0 + kWaveKeys - 1; };
    bf16x8 lf, qf[D / 16];
    f32x16 s[2][2];
    constexpr int kEl = 16 / (D / 16);  // scores of a key tile beside each pair of MFMAs
    float part_sum[2][4] = {};
    auto scores = [&](f32x16 (&to)[2], auto&& beside) __attribute__((always_inline)) {
      const f32x16 zero = {};
      to[0] = to[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lf, ones, zero, 0, 0, 0);
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
          to[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[kk], kf[kt][kk], to[kt], 0, 0, 0);
          beside(kt, kk);
          __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto weights = [&](const f32x16 (&of)[2], int kt, int kk) __attribute__((always_inline)) {
#pragma unroll
      for (int e = kk * kEl; e < (kk + 1) * kEl; e += 2) {
        part_sum[kt][e / 2 % 4] +=
            __builtin_amdgcn_exp2f(of[kt][e] * p.scale_log2) + __builtin_amdgcn_exp2f(of[kt][e + 1] * p.scale_log2);
        asm volatile("" : "+v"(part_sum[kt][e / 2 % 4]));  // (the compiler would move it all behind the MFMAs)
      }
    };
    auto hide = [&](f32x16 (&of)[2]) __attribute__((always_inline)) {
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int e = 0; e < 16; ++e) of[kt][e] = pos[e] >= k0 + kt * 32 + ln ? of[kt][e] : -__builtin_inff();
    };
    int t = t_begin;
    for (; t < t_end; ++t) {  // tiles of which no row sees any of the wave's keys
      advance();
      if (position(t, 31) >= k0) break;
    }
    // The MFMAs of tile t + 1 run beside the exponentials of tile t, two scores a key tile and MFMA
    // pair.  The first tiles are those whose rows do not all see all of the wave's keys.
    if (t < t_end) {
      bool masked = is_masked(t);
      read(t, masked, lf, qf);
      scores(s[0], [](int, int) {});
      ++t;
      while (t < t_end && masked) {
        hide(s[0]);
        advance();
        masked = is_masked(t);
        read(t, masked, lf, qf);
        scores(s[1], [&](int kt, int kk) __attribute__((always_inline)) { weights(s[0], kt, kk); });
        s[0][0] = s[1][0];
        s[0][1] = s[1][1];
        ++t;
      }
      auto step = [&](f32x16 (&now)[2], f32x16 (&then)[2]) __attribute__((always_inline)) {
        advance();
        read(t, false, lf, qf);
        scores(then, [&](int kt, int kk) __attribute__((always_inline)) { weights(now, kt, kk); });
        ++t;
      };
      while (t + 1 < t_end) {
        step(s[0], s[1]);
        step(s[1], s[0]);
      }
      if (t < t_end) {
        step(s[0], s[1]);
        s[0][0] = s[1][0];
        s[0][1] = s[1][1];
      }
      if (masked) hide(s[0]);
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) weights(s[0], kt, kk);
        sum[kt] = (part_sum[kt][0] + part_sum[kt][1]) + (part_sum[kt][2] + part_sum[kt][3]);
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // copies under way end before the workgroup's LDS does
  }
#pragma unroll
  for (int kt = 0; kt < 2; ++kt) {
    const float total = sum[kt] + __shfl_xor(sum[kt], 32);
    const int key = k0 + kt * 32 + ln;
    if (hl != 0 || key > last) continue;
    if (it.slot < 0) {
      float* out = p.weights + (int64_t)it.seq * p.w_sb + (int64_t)kv_head * p.w_sh + key;
      *out = p.accumulate ? *out + total : total;
    } else {
      p.sums[((int64_t)it.slot * p.num_kv_heads + kv_head) * kGroupKeys + (key - it.key0)] = total;
    }
  }
}

// adds up the sums of keys with several items, in order
__global__ __launch_bounds__(kGroupKeys) void msa_kv_weights_join_kernel(WeightsParams p) {
  const uint32_t item = blockIdx.x / (uint32_t)p.num_kv_heads;
  const int kv_head = (int)(blockIdx.x - item * (uint32_t)p.num_kv_heads);
  const WeightsJoin it = p.joins[item];
  const int key = it.key0 + (int)threadIdx.x;
  const int last = p.row_pos[p.seq_row0[it.seq + 1] - 1];
  if (key > last) return;
  float* out = p.weights + (int64_t)it.seq * p.w_sb + (int64_t)kv_head * p.w_sh + key;
  const float old = p.accumulate ? *out : 0.0f;
  const int64_t stride = (int64_t)p.num_kv_heads * kGroupKeys;
  const float* src = p.sums + (int64_t)it.slot0 * stride + (int64_t)kv_head * kGroupKeys + threadIdx.x;
  constexpr int kBatch = 16;
  float total = 0.0f;
  for (int i0 = 0; i0 < it.parts; i0 += kBatch) {
    float x[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) x[i] = src[min(i0 + i, it.parts - 1) * stride];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) total += i0 + i < it.parts ? x[i] : 0.0f;
  }
  *out = old + total;
}

size_t workspace_of(const HostPlan& hp) {
  return (size_t)hp.weight_slots * (size_t)hp.shape.num_kv_heads * kGroupKeys * sizeof(float);
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
  *bytes = msa::workspace_of(plan->hp);
  return MSA_OK;
}

extern "C" msa_status msa_kv_weights(msa_plan_t plan, const void* q, const void* k_cache, const int32_t* block_table,
                                     const float* lse, float* weights, int64_t stride_seq, int64_t stride_head,
                                     int32_t accumulate, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const char* who = "msa_kv_weights";
  const auto invalid = [&](const std::string& msg) { return msa::fail(who, MSA_ERR_INVALID_ARG, msg); };
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
  const size_t need = msa::workspace_of(hp);
  if (need > workspace_bytes || (need > 0 && (!workspace || !msa::aligned(workspace, 16))))
    return invalid("workspace must be 16-byte aligned and hold " + std::to_string(need) + " bytes");
  const int64_t streams = (int64_t)hp.streams.size() * s.num_kv_heads;
  const int64_t items = (int64_t)hp.weights.size() * s.num_kv_heads;
  const int64_t joins = (int64_t)hp.weight_joins.size() * s.num_kv_heads;
  if (hp.total_q * hp.group >= ((int64_t)1 << 31) - 64 || std::max(streams, items) >= msa::kMostGroups)
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
  p.num_q_heads = s.num_q_heads;
  p.num_kv_heads = s.num_kv_heads;
  p.max_blocks = s.max_blocks_per_seq;
  p.group = hp.group;
  p.group_inv = ((1u << 20) + (uint32_t)hp.group - 1) / (uint32_t)hp.group;
  p.inv_scale = 1.0f / s.scale;
  p.scale_log2 = s.scale * 1.4426950408889634f;
  p.accumulate = accumulate;
  p.streams = plan->d_streams;
  p.items = plan->d_weights;
  p.joins = plan->d_weight_joins;
  p.sums = static_cast<float*>(workspace);
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const bool d128 = s.head_dim == 128;
  if (streams > 0) {
    const dim3 grid((uint32_t)streams);
    if (d128)
      hipLaunchKernelGGL(msa::msa_kv_weights_stream_kernel<128>, grid, dim3(256), 0, st, p);
    else
      hipLaunchKernelGGL(msa::msa_kv_weights_stream_kernel<64>, grid, dim3(256), 0, st, p);
    const msa_status rc = msa::launched(who, "stream", (int)hipGetLastError());
    if (rc != MSA_OK) return rc;
  }
  if (items > 0) {
    const dim3 grid((uint32_t)items);
    if (d128)
      hipLaunchKernelGGL(msa::msa_kv_weights_tiles_kernel<128>, grid, dim3(256), 0, st, p);
    else
      hipLaunchKernelGGL(msa::msa_kv_weights_tiles_kernel<64>, grid, dim3(256), 0, st, p);
    const msa_status rc = msa::launched(who, "tiles", (int)hipGetLastError());
    if (rc != MSA_OK) return rc;
  }
  if (joins > 0) {
    hipLaunchKernelGGL(msa::msa_kv_weights_join_kernel, dim3((uint32_t)joins), dim3(msa::kGroupKeys), 0, st, p);
    return msa::launched(who, "join", (int)hipGetLastError());
  }
  return MSA_OK;
}
