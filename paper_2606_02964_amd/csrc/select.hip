// select.hip -- the positions that a reduced cache keeps (msa_kv_select).
//
// One workgroup per list.  The kept positions outside the first and the latest
// ones are those of the largest scores: the bits of a float, flipped so that they
// order as unsigned numbers, are fixed from the top, some bits a pass, by
// counting (a histogram in LDS of the values that share the bits found so far).
// The last pass leaves the smallest kept value T and how many of the values equal to
// T stay; those of the lowest positions do.  One more pass over the positions
// in order writes the list.  Counts are whole numbers, so the result does not
// depend on the order of the LDS atomics.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>

#include "errors.h"
#include "forward.h"
#include "msa_cache.h"

namespace msa {
namespace {

constexpr int kSelectThreads = 1024;
constexpr int kSelectWaves = kSelectThreads / 64;
constexpr int kRadixBits = 11;
constexpr int kBins = 1 << kRadixBits;

struct SelectParams {
  const float* scores;
  int64_t s_sb, s_sl;
  const int32_t* seq_len;
  const int32_t* keep;
  int32_t* index;
  int64_t i_sb, i_sl;
  int32_t* count;
  int32_t num_lists, max_len, max_keep, first, recent;
};

// larger scores have larger keys; NaN as -inf, -0 as +0
__device__ __forceinline__ uint32_t order_key(float x) {
  if (x != x) x = -__builtin_inff();
  const uint32_t u = x == 0.0f ? 0u : __float_as_uint(x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__global__ __launch_bounds__(kSelectThreads) void msa_kv_select_kernel(SelectParams p) {
  __shared__ int hist[kBins];
  __shared__ int s_wave[2][kSelectWaves];
  __shared__ int s_bin, s_above;
  const int seq = blockIdx.x / p.num_lists, list = blockIdx.x - seq * p.num_lists;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = max(0, min(p.seq_len[seq], p.max_len));
  const int k = max(0, min(min(p.keep[seq], p.max_keep), n));
  if (list == 0 && tid == 0) p.count[seq] = k;
  if (k == 0) return;
  const float* scores = p.scores + (int64_t)seq * p.s_sb + (int64_t)list * p.s_sl;
  int32_t* out = p.index + (int64_t)seq * p.i_sb + (int64_t)list * p.i_sl;
  const int recent = min(p.recent, k), first = min(p.first, k - recent);
  const int lo = first, hi = n - recent;  // positions chosen by score lie in [lo, hi)
  int want = k - recent - first;          // of them stay

  // the key T of the last one that stays, and how many equal to it do
  uint32_t found = 0, known = 0;  // T's bits found so far, their mask
  int shift = 32, ties = 0;
  const bool all = want == hi - lo;
  if (!all && want > 0) {
    while (shift > 0) {
      const int bits = min(kRadixBits, shift);
      shift -= bits;
      for (int i = tid; i < kBins; i += kSelectThreads) hist[i] = 0;
      __syncthreads();
      for (int j = lo + tid; j < hi; j += kSelectThreads) {
        const uint32_t key = order_key(scores[j]);
        if ((key & known) == found) atomicAdd(&hist[key >> shift & ((1u << bits) - 1)], 1);
      }
      __syncthreads();
      // the bin, from the top, in which the want-th value lies: each thread has two bins
      const int b1 = kBins - 1 - 2 * tid, b0 = b1 - 1;
      const int c1 = hist[b1], c0 = hist[b0];
      int run = c0 + c1;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(run, d);
        if (lane >= d) run += y;
      }
      if (lane == 63) s_wave[0][wave] = run;
      __syncthreads();
      for (int i = 0; i < wave; ++i) run += s_wave[0][i];
      const int before = run - c0 - c1;
      if (before < want && want <= run) {
        const bool upper = want <= before + c1;
        s_bin = upper ? b1 : b0;
        s_above = before + (upper ? 0 : c1);
      }
      __syncthreads();
      found |= (uint32_t)s_bin << shift;
      known |= ((1u << bits) - 1) << shift;
      want -= s_above;
      __syncthreads();
    }
    ties = want;
  }

  // positions in order, one per thread at a time
  int placed = 0, equal = 0;  // before this round
  for (int base = 0; base < n; base += kSelectThreads) {
    const int j = base + tid;
    bool stays = j < n && (j < lo || j >= hi), tie = false;
    if (j >= lo && j < hi) {
      if (all) {
        stays = true;
      } else if (ties > 0) {
        const uint32_t key = order_key(scores[j]);
        stays = key > found;
        tie = key == found;
      }
    }
    const uint64_t below = (1ull << lane) - 1;
    const uint64_t tie_lanes = __ballot(tie);
    if (lane == 0) s_wave[0][wave] = __popcll(tie_lanes);
    __syncthreads();
    int eq = equal;
    for (int i = 0; i < kSelectWaves; ++i) {
      eq += i < wave ? s_wave[0][i] : 0;
      equal += s_wave[0][i];
    }
    if (tie && eq + __popcll(tie_lanes & below) < ties) stays = true;
    const uint64_t stay_lanes = __ballot(stays);
    if (lane == 0) s_wave[1][wave] = __popcll(stay_lanes);
    __syncthreads();
    int at = placed;
    for (int i = 0; i < kSelectWaves; ++i) {
      at += i < wave ? s_wave[1][i] : 0;
      placed += s_wave[1][i];
    }
    if (stays) out[at + __popcll(stay_lanes & below)] = j;
  }
}

msa_status fail(msa_status st, const std::string& msg) {
  set_last_error("msa_kv_select: " + msg);
  return st;
}

bool aligned4(const void* p) { return reinterpret_cast<uintptr_t>(p) % 4 == 0; }

}  // namespace
}  // namespace msa

extern "C" msa_status msa_kv_select(int32_t num_seqs, int32_t num_lists, const float* scores,
                                    int64_t score_stride_seq, int64_t score_stride_list, int32_t max_len,
                                    const int32_t* seq_len, const int32_t* keep, int32_t first, int32_t recent,
                                    int32_t max_keep, int32_t* index, int64_t index_stride_seq,
                                    int64_t index_stride_list, int32_t* count, void* hip_stream) {
  if (num_seqs < 0 || num_lists < 0 || max_len < 0 || max_keep < 0 || first < 0 || recent < 0)
    return msa::fail(MSA_ERR_INVALID_ARG, "sizes must be >= 0");
  if (score_stride_seq < 0 || score_stride_list < 0 || index_stride_seq < 0 || index_stride_list < 0)
    return msa::fail(MSA_ERR_INVALID_ARG, "strides must be >= 0");
  const int64_t lists = (int64_t)num_seqs * num_lists;
  if (lists == 0) return MSA_OK;
  if (lists >= ((int64_t)1 << 31)) return msa::fail(MSA_ERR_UNSUPPORTED, "too many lists for one launch");
  if (!scores || !seq_len || !keep || !index || !count)
    return msa::fail(MSA_ERR_INVALID_ARG, "scores, seq_len, keep, index, count must be non-null");
  if (!msa::aligned4(scores) || !msa::aligned4(seq_len) || !msa::aligned4(keep) || !msa::aligned4(index) ||
      !msa::aligned4(count))
    return msa::fail(MSA_ERR_INVALID_ARG, "pointers must be 4-byte aligned");
  msa::SelectParams p{};
  p.scores = scores;
  p.s_sb = score_stride_seq;
  p.s_sl = score_stride_list;
  p.seq_len = seq_len;
  p.keep = keep;
  p.index = index;
  p.i_sb = index_stride_seq;
  p.i_sl = index_stride_list;
  p.count = count;
  p.num_lists = num_lists;
  p.max_len = max_len;
  p.max_keep = max_keep;
  p.first = first;
  p.recent = recent;
  hipLaunchKernelGGL(msa::msa_kv_select_kernel, dim3((uint32_t)lists), dim3(msa::kSelectThreads), 0,
                     static_cast<hipStream_t>(hip_stream), p);
  return msa::launched("msa_kv_select", "selection", (int)hipGetLastError());
}
