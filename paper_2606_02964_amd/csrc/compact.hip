// compact.hip -- moves kept cache positions to the front, in place
// (msa_kv_compact).
//
// Position base + i of a sequence takes the K and V of position base + index[i],
// index strictly ascending, hence index[i] >= i: a source lies at or behind
// its destination and, for a run of moves, behind every destination of the moves
// before it.  One workgroup per (sequence, KV head, K or V) therefore goes through
// the list in runs: it reads a run's sources into registers, and writes
// them once every read of the run has arrived.  Runs need no further order: what a
// run writes lies before everything later runs read.
// A run is 64 moves.  K rows are copied in 16-byte pieces; the V of 8
// consecutive destination tokens of a channel is one 16-byte piece of the cache,
// gathered from 8 places and written whole where all 8 are moved to.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>

#include "errors.h"
#include "forward.h"
#include "msa_cache.h"
#include "plan.h"

namespace msa {
namespace {

constexpr int kRun = 64;
constexpr int kCompactThreads = 256;

struct CompactParams {
  const int32_t* base;  // may be null
  const int32_t* index;
  int64_t i_sb, i_sh;
  const int32_t* count;
  const int32_t* block_table;
  uint16_t* k;
  uint16_t* v;
  int64_t k_sb, k_sh, k_st, v_sb, v_sh, v_sd;
  int32_t num_kv_heads, max_blocks, num_blocks, max_count;
};

// Where the elements of a run's moves lie in the cache; -1: no such move.
struct RunPlaces {
  int64_t src[kRun], dst[kRun];
};

// every wave's reads have arrived (the barrier alone would not wait for them)
__device__ __forceinline__ void reads_arrived() { asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory"); }

template <int D>
__global__ __launch_bounds__(kCompactThreads) void msa_kv_compact_kernel(CompactParams p) {
  __shared__ RunPlaces at;
  const int head = blockIdx.x % p.num_kv_heads, rest = blockIdx.x / p.num_kv_heads;
  const bool is_v = rest & 1;
  const int seq = rest >> 1, tid = threadIdx.x;
  const int n = max(0, min(p.count[seq], p.max_count));
  const int64_t base = p.base ? p.base[seq] : 0;
  const int32_t* index = p.index + (int64_t)seq * p.i_sb + (int64_t)head * p.i_sh;
  const int32_t* table = p.block_table + (int64_t)seq * p.max_blocks;
  const int64_t end = (int64_t)p.max_blocks * kBlockSize;
  uint16_t* cache = is_v ? p.v + (int64_t)head * p.v_sh : p.k + (int64_t)head * p.k_sh;
  const int64_t sb = is_v ? p.v_sb : p.k_sb, st = is_v ? 1 : p.k_st;
  auto place = [&](int64_t pos) -> int64_t {
    if (pos < 0 || pos >= end) return -1;
    const int32_t blk = table[pos / kBlockSize];
    return blk < 0 || blk >= p.num_blocks ? -1 : blk * sb + pos % kBlockSize * st;
  };
  // runs end at multiples of 8 destination positions, so that V's 16-byte pieces lie in one run
  const int lead = (int)((base % 8 + 8) % 8);
  for (int i0 = -lead; i0 < n; i0 += kRun) {
    if (tid < kRun) {
      const int i = i0 + tid;
      int64_t src = -1, dst = -1;
      if (i >= 0 && i < n) {
        const int64_t from = index[i];
        if (from > i) {  // (a place kept where it is needs no move)
          src = place(base + from);
          dst = place(base + i);
        }
      }
      at.src[tid] = src >= 0 && dst >= 0 ? src : -1;
      at.dst[tid] = src >= 0 && dst >= 0 ? dst : -1;
    }
    __syncthreads();
    if (!is_v) {
      constexpr int kPieces = D / 8, kEach = kRun * kPieces / kCompactThreads;
      uint4 x[kEach];
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const int m = (e * kCompactThreads + tid) / kPieces, c = tid % kPieces;
        if (at.src[m] >= 0) x[e] = *reinterpret_cast<const uint4*>(cache + at.src[m] + c * 8);
      }
      reads_arrived();
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const int m = (e * kCompactThreads + tid) / kPieces, c = tid % kPieces;
        if (at.dst[m] >= 0) *reinterpret_cast<uint4*>(cache + at.dst[m] + c * 8) = x[e];
      }
    } else {
      constexpr int kEach = D * (kRun / 8) / kCompactThreads;
      uint32_t x[kEach][4];  // two tokens each
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const int c = (e * kCompactThreads + tid) % D, m = (e * kCompactThreads + tid) / D * 8;
#pragma unroll
        for (int t = 0; t < 8; t += 2) {
          const uint32_t a = at.src[m + t] >= 0 ? cache[at.src[m + t] + c * p.v_sd] : 0;
          const uint32_t b = at.src[m + t + 1] >= 0 ? cache[at.src[m + t + 1] + c * p.v_sd] : 0;
          x[e][t / 2] = a | b << 16;
        }
      }
      reads_arrived();
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const int c = (e * kCompactThreads + tid) % D, m = (e * kCompactThreads + tid) / D * 8;
        bool whole = true;
#pragma unroll
        for (int t = 0; t < 8; ++t) whole &= at.dst[m + t] >= 0;
        if (whole) {
          *reinterpret_cast<uint4*>(cache + at.dst[m] + c * p.v_sd) = make_uint4(x[e][0], x[e][1], x[e][2], x[e][3]);
        } else {
#pragma unroll
          for (int t = 0; t < 8; ++t)
            if (at.dst[m + t] >= 0) cache[at.dst[m + t] + c * p.v_sd] = (uint16_t)(x[e][t / 2] >> (t % 2 * 16));
        }
      }
    }
    __syncthreads();  // the places are read
  }
}

msa_status fail(msa_status st, const std::string& msg) {
  set_last_error("msa_kv_compact: " + msg);
  return st;
}

bool aligned(const void* p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

}  // namespace
}  // namespace msa

extern "C" msa_status msa_kv_compact(const msa_shape* shape, const int32_t* base, const int32_t* index,
                                     int64_t index_stride_seq, int64_t index_stride_head, int32_t max_count,
                                     const int32_t* count, const int32_t* block_table, void* k_cache, void* v_cache,
                                     void* hip_stream) {
  if (!shape) return msa::fail(MSA_ERR_INVALID_ARG, "shape must be non-null");
  std::string err;
  const msa_status st = msa::check_shape(*shape, &err);
  if (st != MSA_OK) return msa::fail(st, err);
  const msa_shape& s = *shape;
  if (max_count < 0 || index_stride_seq < 0 || index_stride_head < 0)
    return msa::fail(MSA_ERR_INVALID_ARG, "max_count and the index strides must be >= 0");
  if (s.num_seqs == 0 || max_count == 0) return MSA_OK;
  if (!index || !count || !block_table || !k_cache || !v_cache)
    return msa::fail(MSA_ERR_INVALID_ARG, "index, count, block_table, k_cache, v_cache must be non-null");
  if (!msa::aligned(k_cache, 16) || !msa::aligned(v_cache, 16) || !msa::aligned(base, 4) || !msa::aligned(index, 4) ||
      !msa::aligned(count, 4) || !msa::aligned(block_table, 4))
    return msa::fail(MSA_ERR_INVALID_ARG, "caches must be 16-byte, the others 4-byte aligned");
  const int64_t groups = (int64_t)s.num_seqs * s.num_kv_heads * 2;
  if (groups >= ((int64_t)1 << 31)) return msa::fail(MSA_ERR_UNSUPPORTED, "too many heads for one launch");
  msa::CompactParams p{};
  p.base = base;
  p.index = index;
  p.i_sb = index_stride_seq;
  p.i_sh = index_stride_head;
  p.count = count;
  p.block_table = block_table;
  p.k = static_cast<uint16_t*>(k_cache);
  p.v = static_cast<uint16_t*>(v_cache);
  p.k_sb = s.k_stride_block;
  p.k_sh = s.k_stride_head;
  p.k_st = s.k_stride_tok;
  p.v_sb = s.v_stride_block;
  p.v_sh = s.v_stride_head;
  p.v_sd = s.v_stride_dim;
  p.num_kv_heads = s.num_kv_heads;
  p.max_blocks = s.max_blocks_per_seq;
  p.num_blocks = s.num_blocks;
  p.max_count = max_count;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  if (s.head_dim == 128)
    hipLaunchKernelGGL(msa::msa_kv_compact_kernel<128>, dim3((uint32_t)groups), dim3(msa::kCompactThreads), 0, stream, p);
  else
    hipLaunchKernelGGL(msa::msa_kv_compact_kernel<64>, dim3((uint32_t)groups), dim3(msa::kCompactThreads), 0, stream, p);
  return msa::launched("msa_kv_compact", "compaction", (int)hipGetLastError());
}
