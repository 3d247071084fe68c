// select.hip -- the positions that a reduced cache keeps (msa_kv_select).
//
// One workgroup per list.  Every position gets a 32-bit key that orders as its
// score does; the first and the latest positions, which stay whatever their
// score, get the largest key there is.  The k-th largest key T is found from
// its top bits down, 11 bits a pass, by counting (a histogram in LDS of the keys
// that share the bits found so far); with it comes how many of the keys equal to T
// stay, those of the lowest positions.  Each of the 16 waves holds a run of
// neighbouring positions: it counts what it keeps, learns from the other
// waves' counts where its own begin, and writes them in order.
// A list in a buffer of up to 64K scores is read once, into registers (32 or 64 keys
// a thread); others are read again by every pass.  One list of 9001 takes 9.0 us,
// 256 of 2K to 16K with half kept 16.6, one of 200 6.4: that is passes and barriers
// (waves wait 63% of the time; LDS is busy 15%, a third of it with conflicts).
// Reading is the smaller part: one instruction for each of 16K keys takes a CU 256
// cycles (16 waves, 16 keys a lane), so time goes by instructions per key.  (With the window and the list's end
// tested by position in every loop, and lanes that share a bin added up first, a
// list of 9001 took 13.7 us; ranking the values that share T's first 11 bits one
// against the other 19.6 us.)
// Counts are whole numbers, so the result does not depend on the order of
// the LDS atomics.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>

#include "errors.h"
#include "forward.h"
#include "msa_cache.h"
#include "wave_ops.h"

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

constexpr uint32_t kStays = 0xffffffffu;  // above every score's key

// larger scores have larger keys; NaN as -inf, -0 as +0.  No score's key is 0 or kStays.
__device__ __forceinline__ uint32_t order_key(float x) {
  if (x != x) x = -__builtin_inff();
  const int32_t u = __float_as_int(x + 0.0f);  // (-0 + 0 is +0)
  return (uint32_t)u ^ ((uint32_t)(u >> 31) | 0x80000000u);
}

// sum of the entries before `wave`'s
__device__ __forceinline__ int sum_before(const int (&x)[kSelectWaves], int wave) {
  int before = 0;
#pragma unroll
  for (int i = 0; i < kSelectWaves; ++i) before += i < wave ? x[i] : 0;
  return before;
}

// kEach: positions of a thread that registers hold, 0 where they do not
template <int kEach>
__global__ __launch_bounds__(kSelectThreads) void msa_kv_select_kernel(SelectParams p) {
  __shared__ __attribute__((aligned(16))) int hist[kBins];
  __shared__ __attribute__((aligned(16))) int s_bins[kSelectWaves], s_stay[kSelectWaves], s_tie[kSelectWaves];
  __shared__ int s_bin, s_above, s_in;
  const int seq = blockIdx.x / p.num_lists, list = blockIdx.x - seq * p.num_lists;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = __builtin_amdgcn_readfirstlane(max(0, min(p.seq_len[seq], p.max_len)));
  const int k = __builtin_amdgcn_readfirstlane(max(0, min(min(p.keep[seq], p.max_keep), n)));
  if (list == 0 && tid == 0) p.count[seq] = k;
  if (k == 0) return;
  const float* scores = p.scores + (int64_t)seq * p.s_sb + (int64_t)list * p.s_sl;
  int32_t* out = p.index + (int64_t)seq * p.i_sb + (int64_t)list * p.i_sl;
  const int recent = min(p.recent, k), first = min(p.first, k - recent);
  const uint32_t lo = (uint32_t)first, hi = (uint32_t)(n - recent);  // by score: [lo, hi); with k = n all stay

  // the wave's elements: element e of a lane is position first_of + 64 e
  const int each = (int)(((int64_t)n + kSelectThreads - 1) / kSelectThreads);
  const uint32_t first_of = (uint32_t)wave * (uint32_t)each * 64u + (uint32_t)lane;
  auto key_at = [&](uint32_t j) -> uint32_t {
    if (j >= (uint32_t)n) return 0u;
    if (j - lo >= hi - lo || k == n) return kStays;
    return order_key(scores[j]);
  };
  uint32_t held[kEach > 0 ? kEach : 1];
  if constexpr (kEach > 0) {
#pragma unroll
    for (int e0 = 0; e0 < kEach; e0 += 8) {
      if (e0 < each) {
#pragma unroll
        for (int e = e0; e < e0 + 8; ++e) held[e] = e < each ? key_at(first_of + (uint32_t)e * 64u) : 0u;
      }
    }
  }
  // f(position, key) for the wave's elements, in order
  auto for_each = [&](auto&& f) __attribute__((always_inline)) {
    uint32_t start = first_of;
    int count = each;
    asm volatile("" : "+v"(start), "+s"(count));  // (positions and bounds are not kept from one loop to the next)
    if constexpr (kEach > 0) {
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        if (e % 8 == 0 && e >= count) break;
        if (e < count) f(start + (uint32_t)e * 64u, held[e]);
      }
    } else {
      for (int e = 0; e < count; ++e) f(start + (uint32_t)e * 64u, key_at(start + (uint32_t)e * 64u));
    }
  };

  // Keys above `found` stay, and the first `ties` of those equal to it.
  uint32_t found = 0;
  int ties = 0;
  if (k < n) {
    int want = k, shift = 32;
    for (int i = tid; i < kBins; i += kSelectThreads) hist[i] = 0;
    __syncthreads();
    // counted: bits of a key from `shift` up are found, or in the histogram
    auto fix_bin = [&]() __attribute__((always_inline)) {
      __syncthreads();
      // the bin, from the top, in which the want-th key lies: each thread has two bins
      const int b1 = kBins - 1 - 2 * tid, b0 = b1 - 1;
      const int2 c = *reinterpret_cast<const int2*>(&hist[b0]);
      *reinterpret_cast<int2*>(&hist[b0]) = make_int2(0, 0);
      int run = wave_scan(c.x + c.y);
      if (lane == 63) s_bins[wave] = run;
      __syncthreads();
      run += sum_before(s_bins, wave);
      const int before = run - c.x - c.y;
      if (before < want && want <= run) {
        const bool upper = want <= before + c.y;
        s_bin = upper ? b1 : b0;
        s_above = before + (upper ? 0 : c.y);
        s_in = upper ? c.y : c.x;
      }
      __syncthreads();
      found |= (uint32_t)__builtin_amdgcn_readfirstlane(s_bin) << shift;
      want -= __builtin_amdgcn_readfirstlane(s_above);
      if (__builtin_amdgcn_readfirstlane(s_in) == want) {  // all that share the bits found so far stay
        found -= 1;                                        // (their bin is not 0: key 0 is no position's)
        want = 0;
      }
    };
    shift -= kRadixBits;
    for_each([&](uint32_t, uint32_t key) { atomicAdd(&hist[key >> (32 - kRadixBits)], 1); });
    fix_bin();
    while (shift > 0 && want > 0) {
      const uint32_t share = found >> shift, above_bits = (uint32_t)shift;
      const int bits = min(kRadixBits, shift);
      shift -= bits;
      for_each([&](uint32_t, uint32_t key) {
        if (key >> above_bits == share) atomicAdd(&hist[__builtin_amdgcn_ubfe(key, (uint32_t)shift, (uint32_t)bits)], 1);
      });
      fix_bin();
    }
    ties = want;
  }

  // what each wave keeps
  int stay = 0, tie = 0;
  for_each([&](uint32_t, uint32_t key) {
    stay += key > found;
    tie += key == found;
  });
  stay = wave_sum(stay);
  tie = ties > 0 ? wave_sum(tie) : 0;
  if (lane == 0) {
    s_stay[wave] = stay;
    s_tie[wave] = tie;
  }
  __syncthreads();
  int equal = sum_before(s_tie, wave);
  int32_t* at = out + sum_before(s_stay, wave) + min(equal, ties);
  if (tie == 0 || equal >= ties) {  // (uniform over the wave)
    for_each([&](uint32_t j, uint32_t key) {
      const uint64_t lanes = __ballot(key > found);
      if (key > found)
        at[__builtin_amdgcn_mbcnt_hi((uint32_t)(lanes >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)lanes, 0))] = (int32_t)j;
      at += __popcll(lanes);
    });
  } else {
    const uint64_t below = (1ull << lane) - 1;
    for_each([&](uint32_t j, uint32_t key) {
      const uint64_t tie_lanes = __ballot(key == found);
      const bool stays = key > found || (key == found && equal + __popcll(tie_lanes & below) < ties);
      const uint64_t lanes = __ballot(stays);
      if (stays) at[__popcll(lanes & below)] = (int32_t)j;
      equal += __popcll(tie_lanes);
      at += __popcll(lanes);
    });
  }
}

template <int kEach>
void launch_select(const SelectParams& p, int64_t lists, hipStream_t s) {
  hipLaunchKernelGGL(msa_kv_select_kernel<kEach>, dim3((uint32_t)lists), dim3(kSelectThreads), 0, s, p);
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
  if (lists >= ((int64_t)1 << 32) / msa::kSelectThreads) return msa::fail(MSA_ERR_UNSUPPORTED, "too many lists for one launch");
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
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  // What holds the longest list; its passes skip what a shorter one leaves empty, eight registers
  // at a time.  With 32 keys a thread a CU holds two workgroups, with 64 one (1024 lists of 8000 in
  // buffers of 32K: 26.8 and 39.4 us).  Held against read again in every pass: 256 lists of 30000
  // 27 against 46 us, of 65536 49 against 123.
  const int64_t each = ((int64_t)max_len + msa::kSelectThreads - 1) / msa::kSelectThreads;
  if (each <= 32)
    msa::launch_select<32>(p, lists, st);
  else if (each <= 64)
    msa::launch_select<64>(p, lists, st);
  else
    msa::launch_select<0>(p, lists, st);
  return msa::launched("msa_kv_select", "selection", (int)hipGetLastError());
}
