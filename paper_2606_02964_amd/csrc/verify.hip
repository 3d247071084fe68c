// verify.hip -- verification of trees of drafted tokens against the target's
// probabilities (msa_tree_verify; the rule is in include/msa_tree.h).
//
// A row of up to 32768 entries: one launch, a workgroup per tree that walks it and
// then sums the last node's weights (msa_verify_one).  Longer ones, whose reading one
// CU would take too long over, in two (in a captured graph, one launch and two: a
// row of 8000 6.5 and 8.7 us, of 32768 8.5 and 8.5, two rows of that 10.1 and 9.0; 64
// trees with two rows of 16000 9.0 and 10.2, of 32768 12.1 and 11.7; launched one by
// one, another launch takes the host 3.6 us):
// msa_verify_walk, one workgroup per tree: the walk reads two numbers a slot
// (p and q of the slot's token in its parent's row), all at once, and then
// takes one decision after the other in registers.  Where a node's children
// were drawn from q, the residual after n failed ones is max(a p - b q, 0) with
// two scalars a and b (max(max(x, 0) / P - q, 0) = max(x / P - q, 0), as q >= 0),
// so nothing of the vocabulary's length is stored; a second or later child's test
// needs that residual's mass, for which the workgroup reads the node's two rows.
// msa_verify_sums: the sum of r over each cell of 512 entries of the vocabulary, a wave
// a cell, 8 neighbouring entries a lane.  The tree's last workgroup to finish picks, by
// one wave: the cell, then the lane, then the entry at which the running sum passes u T.
// It learns the others' sums by accesses that go through to where the XCDs meet; as a
// launch of its own the pick took as long and the host 3.6 us more, and with fences
// that write back an XCD's whole L2, for every workgroup, 32 trees took 80 us.
// Bound by reading one or two rows of the vocabulary per tree, and for few trees by
// the chains of dependent reads in walk and pick (32 trees, two rows of 131072 fp32
// each: 16.5 us; the rows' 34 MB alone take 6.1 us; 32 trees of drawn slots over
// 128000, whose walks sum rows too: 46.5 us, 37 of them the walk).
// Sums are in 64 bits: with 10^5 tokens the borders between neighbouring tokens
// are about 10^-5 of the mass apart and a 32-bit running sum would pick a
// neighbour once in some hundred draws; and the tests' products (24 + 24 bits)
// are exact.  No floating-point atomics: sums run in a fixed order.
#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <string>

#include "errors.h"
#include "forward.h"
#include "msa_tree.h"
#include "plan_handle.h"
#include "wave_ops.h"

#pragma clang fp contract(off)  // a p - b q is 0 where both products are equal

namespace msa {
namespace {

constexpr int kWalkThreads = 1024;
constexpr int kWave = 64;
constexpr int kEach = 8;                // neighbouring entries of a lane
constexpr int kCell = kWave * kEach;    // entries of a cell
constexpr int kSumsThreads = 512;

// How the next token's weights follow from the last node's row(s).
enum Rest { kAsIs = 0, kResidual = 1, kWithout = 2 };

struct WalkResult {
  double a, b;       // kResidual: weights max(a p - b q, 0)
  int32_t tree_row;  // of the last node
  int32_t node;      // its slot
  int32_t rest;
  uint32_t done;     // workgroups of the sums that are finished
};

struct VerifyParams {
  const void* target;
  const void* draft;  // may be null
  int64_t target_stride, draft_stride;
  const int32_t* tokens;
  const int32_t* parents;
  const float* u_accept;
  const float* u_sample;
  int32_t* path;
  int64_t path_stride;
  int32_t* path_len;
  int32_t* next_token;
  const TreeSpan* trees;
  WalkResult* walk;  // [trees]
  double* sums;      // [trees][cells]
  int32_t vocab, max_slots;
  int32_t cells;     // of a row
  int32_t groups;    // sums: workgroups of a tree
};

__device__ __forceinline__ float clean(float x) { return x > 0.0f && x < __builtin_inff() ? x : 0.0f; }
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__hip_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }

// 4 entries from any element boundary
template <class T>
__device__ __forceinline__ void load4(const T* src, float (&x)[4]) {
  struct __attribute__((packed, aligned(sizeof(T)))) Raw {
    T v[4];
  };
  const Raw r = *reinterpret_cast<const Raw*>(src);
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = clean(to_float(r.v[i]));
}

template <class T>
__device__ __forceinline__ void load8(const T* src, float (&x)[8]) {
  float lo[4], hi[4];
  load4(src, lo);
  load4(src + 4, hi);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i] = lo[i];
    x[i + 4] = hi[i];
  }
}

// sum over the workgroup of max(a p - b q, 0) over the vocabulary
template <class T>
__device__ double residual_mass(const T* p, const T* q, double a, double b, int vocab, double* part) {
  const int tid = threadIdx.x;
  double sum = 0.0;
  const int whole = vocab & ~3;
  for (int t = tid * 4; t < whole; t += kWalkThreads * 4) {
    float x[4], y[4];
    load4(p + t, x);
    load4(q + t, y);
#pragma unroll
    for (int i = 0; i < 4; ++i) sum += fmax(a * (double)x[i] - b * (double)y[i], 0.0);
  }
  for (int t = whole + tid; t < vocab; t += kWalkThreads)
    sum += fmax(a * (double)clean(to_float(p[t])) - b * (double)clean(to_float(q[t])), 0.0);
  sum = wave_sum(sum);
  __syncthreads();  // part may still be read from the last call
  if ((tid & 63) == 0) part[tid >> 6] = sum;
  __syncthreads();
  double total = 0.0;
  for (int i = 0; i < kWalkThreads / kWave; ++i) total += part[i];
  return total;
}

struct WalkLds {
  int16_t parent[MSA_TREE_MAX_SLOTS];
  int32_t token[MSA_TREE_MAX_SLOTS];
  float p[MSA_TREE_MAX_SLOTS], q[MSA_TREE_MAX_SLOTS], u[MSA_TREE_MAX_SLOTS];
  double part[kWalkThreads / kWave];
};

// The walk of a tree; path and path_len are written.  Every wave of the workgroup
// takes the (uniform) decisions, so that all of them meet in residual_mass.
// Children lie behind their parent, so the walk is one pass over the slots, 64 at a time.
template <class T>
__device__ __forceinline__ WalkResult walk_tree(const VerifyParams& v, int tree_id, const TreeSpan& tree, WalkLds& s) {
  const T* target = static_cast<const T*>(v.target);
  const T* draft = static_cast<const T*>(v.draft);
  const int tid = threadIdx.x, lane = tid & 63;
  for (int i = tid; i < tree.n; i += kWalkThreads) {
    const int64_t row = (int64_t)tree.row0 + i;
    int32_t up = v.parents[row];
    up = up >= 0 && up < i ? up : -1;
    const int32_t token = v.tokens[row];
    const bool ok = up >= 0 && token >= 0 && token < v.vocab;
    const int64_t prow = (int64_t)tree.row0 + up;
    s.parent[i] = (int16_t)up;
    s.token[i] = token;
    s.p[i] = ok ? clean(to_float(target[prow * v.target_stride + token])) : 0.0f;
    s.q[i] = ok && draft ? clean(to_float(draft[prow * v.draft_stride + token])) : 0.0f;
    s.u[i] = v.u_accept[row];
  }
  __syncthreads();

  int32_t* path = v.path + (int64_t)tree_id * v.path_stride;
  int node = 0, len = 1;
  double a = 1.0, b = 0.0, mass = 1.0;
  bool known = true, dead = false, failed = false;  // mass known; no residual left; some child failed
  for (int base = 0; base < tree.n; base += kWave) {
    const int slot = base + lane;
    const bool in = slot < tree.n;
    const int up = in ? s.parent[slot] : -1;
    const int token = in ? s.token[slot] : -1;
    uint64_t children = __ballot(in && up == node);
    while (children) {
      const int l = __builtin_ctzll(children), i = base + l;
      children &= children - 1;
      double p = s.p[i], q = s.q[i];
      const double u = s.u[i];
      bool stays;
      if (draft) {
        if (!known && !dead) {
          mass = residual_mass(target + ((int64_t)tree.row0 + node) * v.target_stride,
                               draft + ((int64_t)tree.row0 + node) * v.draft_stride, a, b, v.vocab, s.part);
          known = true;
          dead = !(mass > 0.0);
        }
        stays = !dead && u * q * mass < fmax(a * p - b * q, 0.0);
      } else {
        // a token that failed before under this node has nothing left
        const int32_t x = s.token[i];
        bool twice = __any(in && up == node && slot < i && token == x);
        for (int e = node + 1 + lane; e < base; e += kWave) twice |= s.parent[e] == node && s.token[e] == x;
        if (__any(twice)) p = 0.0;
        stays = u * mass < p;
        if (!stays) mass -= p;
      }
      if (stays) {
        if (tid == 0) path[len] = i;
        node = i;
        ++len;
        a = 1.0, b = 0.0, mass = 1.0;
        known = true, dead = failed = false;
        children = __ballot(in && up == node);  // all behind slot i
      } else {
        failed = true;
        if (draft && !dead) {
          a = a / mass;
          b = b / mass + 1.0;
          known = false;
        }
      }
    }
  }
  for (int i = len + tid; i < v.max_slots; i += kWalkThreads) path[i] = -1;
  if (tid == 0) {
    path[0] = 0;
    v.path_len[tree_id] = len;
  }
  WalkResult r{};
  r.a = a;
  r.b = b;
  r.tree_row = tree.row0 + node;
  r.node = node;
  r.rest = !failed || dead ? kAsIs : draft ? kResidual : kWithout;
  return r;
}

template <class T>
__global__ __launch_bounds__(kWalkThreads) void msa_verify_walk_kernel(VerifyParams v) {
  __shared__ WalkLds s;
  const WalkResult r = walk_tree<T>(v, (int)blockIdx.x, v.trees[blockIdx.x], s);
  if (threadIdx.x == 0) v.walk[blockIdx.x] = r;
}

__device__ __forceinline__ double sum_of(const double (&w)[kEach]) {
  return ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
}

// 8 entries of a row from t0, 0 behind its end
template <class T>
__device__ __forceinline__ void load_entries(const T* row, int t0, int vocab, float (&x)[kEach]) {
  if (t0 + kEach <= vocab) {
    load8(row + t0, x);
  } else {
#pragma unroll
    for (int i = 0; i < kEach; ++i) x[i] = t0 + i < vocab ? clean(to_float(row[t0 + i])) : 0.0f;
  }
}

// Walk, sums and pick of a row of up to kOneCells * kOneCell entries in one
// workgroup.  A thread sums 8 neighbouring entries of each cell; the wave and cell, then the lane,
// then the entry at which the running sum passes u T follow one from the other, the entry from
// reading 8 of them again.
constexpr int kOneCell = kWalkThreads * kEach;
constexpr int kOneCells = 4;
constexpr int kWaves = kWalkThreads / kWave;

template <class T>
__global__ __launch_bounds__(kWalkThreads) void msa_verify_one_kernel(VerifyParams v) {
  __shared__ WalkLds s;
  __shared__ uint32_t gone[kOneCells * kOneCell / 32];
  __shared__ double part[kOneCells * kWaves];
  const int tree_id = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const TreeSpan tree = v.trees[tree_id];
  const double u = (double)fminf(fmaxf(v.u_sample[tree_id], 0.0f), 0x1.fffffep-1f);  // (fmaxf of NaN and 0 is 0)
  const WalkResult r = walk_tree<T>(v, tree_id, tree, s);
  const T* p = static_cast<const T*>(v.target) + (int64_t)r.tree_row * v.target_stride;
  const T* q = v.draft ? static_cast<const T*>(v.draft) + (int64_t)r.tree_row * v.draft_stride : nullptr;
  if (r.rest == kWithout) {
    for (int i = tid; i < kOneCells * kOneCell / 32; i += kWalkThreads) gone[i] = 0;
    __syncthreads();
    for (int i = r.node + 1 + tid; i < tree.n; i += kWalkThreads) {
      const int32_t t = s.token[i];
      if (s.parent[i] == r.node && t >= 0 && t < v.vocab) atomicOr(&gone[t >> 5], 1u << (t & 31));
    }
    __syncthreads();
  }
  // the thread's entries of a cell
  auto load = [&](int c, int rest, double (&w)[kEach]) __attribute__((always_inline)) {
    const int t0 = c * kOneCell + tid * kEach;
    float x[kEach], y[kEach];
    load_entries(p, t0, v.vocab, x);
    if (rest == kResidual) load_entries(q, t0, v.vocab, y);
    const uint32_t out = rest == kWithout ? gone[t0 >> 5] >> (t0 & 31) : 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      w[i] = rest == kResidual ? fmax(r.a * (double)x[i] - r.b * (double)y[i], 0.0) : out >> i & 1 ? 0.0 : (double)x[i];
  };
  int rest = r.rest;
  double run[kOneCells], running, total;
  for (;;) {
#pragma unroll 2
    for (int c = 0; c < kOneCells; ++c) {
      run[c] = 0.0;
      if (c * kOneCell < v.vocab) {  // (uniform)
        double w[kEach];
        load(c, rest, w);
        run[c] = wave_scan(sum_of(w));
      }
      if (lane == kWave - 1) part[c * kWaves + wave] = run[c];
    }
    __syncthreads();
    // the waves' sums, cell by cell: one of them a lane
    static_assert(kOneCells * kWaves == kWave, "a lane for each wave and cell");
    running = wave_scan(part[lane]);
    total = lane_value(running, kWave - 1);
    if (total > 0.0 || rest == kAsIs) break;  // (uniform)
    rest = kAsIs;  // nothing is left: the row itself
    __syncthreads();
  }
  if (!(total > 0.0)) {
    if (tid == 0) v.next_token[tree_id] = -1;
    return;
  }
  const double limit = u * total;
  // Where rounding leaves no sum above the limit, the last wave, lane and entry that hold any weight.
  // (Neighbouring sums of a scan are added up in another order, so one without any weight may
  // pass the limit where the one before it does not.)
  const uint64_t some = __ballot(part[lane] > 0.0), past = __ballot(running > limit) & some;
  const int at_wave = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(some);
  if (wave != at_wave % kWaves) return;  // (uniform)
  const int cell = at_wave / kWaves;
  double mine = 0.0;
#pragma unroll
  for (int c = 0; c < kOneCells; ++c) mine = c == cell ? run[c] : mine;
  const double before = lane_value(lane_below(running, 0.0), at_wave);
  double w[kEach];
  load(cell, rest, w);
  const double below = lane_below(mine, 0.0);
  const uint64_t some_lanes = __ballot(sum_of(w) > 0.0), past_lanes = __ballot(before + mine > limit) & some_lanes;
  const int at_lane = past_lanes ? __builtin_ctzll(past_lanes) : 63 - __builtin_clzll(some_lanes);
  if (lane != at_lane) return;
  double at = before + below;
  int found = -1, last = -1;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    at += w[i];
    if (w[i] > 0.0) {
      last = cell * kOneCell + tid * kEach + i;
      if (at > limit && found < 0) found = last;
    }
  }
  v.next_token[tree_id] = found >= 0 ? found : last;
}

// The last node's weights, a cell at a time, by one wave.
template <class T>
struct Rows {
  const T *p, *q;
  double a, b;
  int rest, vocab;
  const TreeSpan tree;
  int node;
  const int32_t *tokens, *parents;

  __device__ __forceinline__ Rows(const VerifyParams& v, int tree_id)
      : vocab(v.vocab), tree(v.trees[tree_id]), tokens(v.tokens + tree.row0), parents(v.parents + tree.row0) {
    const WalkResult r = v.walk[tree_id];
    p = static_cast<const T*>(v.target) + (int64_t)r.tree_row * v.target_stride;
    q = v.draft ? static_cast<const T*>(v.draft) + (int64_t)r.tree_row * v.draft_stride : nullptr;
    a = r.a;
    b = r.b;
    rest = r.rest;
    node = r.node;
  }

  // the lane's 8 entries of a cell, 0 behind the row's end; `gone` (the wave's own, in LDS) takes a
  // bit for each of the cell's tokens that failed under the last node
  __device__ __forceinline__ void load(int cell, uint32_t* gone, double (&w)[kEach]) const {
    const int lane = threadIdx.x & 63, lo = cell * kCell, t0 = lo + lane * kEach;
    float x[kEach], y[kEach];
    load_entries(p, t0, vocab, x);
    if (rest == kResidual) load_entries(q, t0, vocab, y);
    uint32_t out = 0;
    if (rest == kWithout) {  // (a wave's LDS accesses stay in order)
      volatile uint32_t* bits = gone;
      if (lane < kCell / 32) bits[lane] = 0;
      for (int i = node + 1 + lane; i < tree.n; i += kWave) {
        const int32_t t = tokens[i];
        if (parents[i] == node && t >= lo && t - lo < kCell) atomicOr(&gone[(t - lo) >> 5], 1u << ((t - lo) & 31));
      }
      out = bits[lane * kEach >> 5] >> (lane * kEach & 31);
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      w[i] = rest == kResidual ? fmax(a * (double)x[i] - b * (double)y[i], 0.0) : out >> i & 1 ? 0.0 : (double)x[i];
  }
};

// Sums on their way from one workgroup to another of the launch: written and read
// through to where all XCDs meet, so that no cache has to be written back or emptied.
__device__ __forceinline__ void shared_store(double* at, double x) {
  __hip_atomic_store(reinterpret_cast<uint64_t*>(at), __builtin_bit_cast(uint64_t, x), __ATOMIC_RELAXED,
                     __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ double shared_load(const double* at) {
  return __builtin_bit_cast(double, __hip_atomic_load(reinterpret_cast<const uint64_t*>(at), __ATOMIC_RELAXED,
                                                      __HIP_MEMORY_SCOPE_AGENT));
}

// The cell, then the lane, then the entry at which the running sum passes u T, by one wave.
template <class T>
__device__ __forceinline__ void pick(const VerifyParams& v, int tree_id, Rows<T> rows, uint32_t* gone) {
  const int lane = threadIdx.x & 63;
  const double* sums = v.sums + (int64_t)tree_id * v.cells;
  const double u = (double)fminf(fmaxf(v.u_sample[tree_id], 0.0f), 0x1.fffffep-1f);  // (fmaxf of NaN and 0 is 0)
  double w[kEach], total = 0.0;
  for (int c0 = 0; c0 < v.cells; c0 += kWave) total += wave_sum(c0 + lane < v.cells ? shared_load(sums + c0 + lane) : 0.0);
  const bool again = !(total > 0.0);  // nothing is left: the row itself, summed here (it hardly ever is)
  if (again) {
    rows.rest = kAsIs;
    total = 0.0;
    for (int c = 0; c < v.cells; ++c) {
      rows.load(c, gone, w);
      total += wave_sum(sum_of(w));
    }
    if (!(total > 0.0)) {
      if (lane == 0) v.next_token[tree_id] = -1;
      return;
    }
  }
  const double limit = u * total;
  // the first cell whose running sum passes the limit; where rounding leaves none, the
  // last one that holds any weight
  int found = -1, holds = 0;
  double before = 0.0, holds_before = 0.0, carry = 0.0;
  if (again) {
    for (int c = 0; c < v.cells && found < 0; ++c) {
      rows.load(c, gone, w);
      const double s = wave_sum(sum_of(w));
      if (s > 0.0 && carry + s > limit) {
        found = c;
        before = carry;
      } else if (s > 0.0) {
        holds = c;
        holds_before = carry;
      }
      carry += s;
    }
  }
  for (int c0 = 0; c0 < v.cells && found < 0 && !again; c0 += kWave) {
    const double s = c0 + lane < v.cells ? shared_load(sums + c0 + lane) : 0.0;
    const double run = carry + wave_scan(s);
    const uint64_t some = __ballot(s > 0.0), past = __ballot(run > limit) & some;
    const double prev = lane_below(run, carry);
    if (past) {
      const int l = __builtin_ctzll(past);
      found = c0 + l;
      before = lane_value(prev, l);
    } else if (some) {
      const int l = 63 - __builtin_clzll(some);
      holds = c0 + l;
      holds_before = lane_value(prev, l);
    }
    carry = lane_value(run, kWave - 1);
  }
  if (found < 0) {
    found = holds;
    before = holds_before;
  }
  rows.load(found, gone, w);
  const double own = sum_of(w), run = wave_scan(own);
  const uint64_t some = __ballot(own > 0.0), past = __ballot(before + run > limit) & some;
  const int at_lane = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(some);
  double at = before + lane_below(run, 0.0);
  int first = -1, last = -1;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    at += w[i];
    if (w[i] > 0.0) {
      last = found * kCell + lane * kEach + i;
      if (at > limit && first < 0) first = last;
    }
  }
  if (lane == at_lane) v.next_token[tree_id] = first >= 0 ? first : last;
}

template <class T>
__global__ __launch_bounds__(kSumsThreads) void msa_verify_sums_kernel(VerifyParams v) {
  __shared__ uint32_t gone[kSumsThreads / kWave][kCell / 32];
  __shared__ uint32_t before;
  const int tree_id = blockIdx.x / v.groups, group = blockIdx.x - tree_id * v.groups;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Rows<T> rows(v, tree_id);
  for (int cell = group * (kSumsThreads / kWave) + wave; cell < v.cells; cell += v.groups * (kSumsThreads / kWave)) {
    double w[kEach];
    rows.load(cell, gone[wave], w);
    const double sum = wave_sum(sum_of(w));
    if ((threadIdx.x & 63) == 0) shared_store(v.sums + (int64_t)tree_id * v.cells + cell, sum);
  }
  // The tree's last workgroup to arrive here picks: every wave's sums have arrived before its workgroup is counted.
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0)
    before = __hip_atomic_fetch_add(&v.walk[tree_id].done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (before + 1 == (uint32_t)v.groups && wave == 0) pick<T>(v, tree_id, rows, gone[0]);
}

template <class T>
int launch_verify(const VerifyParams& v, int trees, hipStream_t s) {
  if (v.vocab <= kOneCells * kOneCell) {
    hipLaunchKernelGGL(msa_verify_one_kernel<T>, dim3(trees), dim3(kWalkThreads), 0, s, v);
    return (int)hipGetLastError();
  }
  hipLaunchKernelGGL(msa_verify_walk_kernel<T>, dim3(trees), dim3(kWalkThreads), 0, s, v);
  int rc = (int)hipGetLastError();
  if (rc != 0) return rc;
  hipLaunchKernelGGL(msa_verify_sums_kernel<T>, dim3((uint32_t)trees * (uint32_t)v.groups), dim3(kSumsThreads), 0, s,
                     v);
  return (int)hipGetLastError();
}

int64_t cells_of(int64_t vocab) { return (vocab + kCell - 1) / kCell; }
size_t walk_bytes(int64_t trees) { return ((size_t)trees * sizeof(WalkResult) + 255) / 256 * 256; }
size_t workspace_of(int64_t trees, int64_t vocab) {
  return trees == 0 ? 0 : walk_bytes(trees) + (size_t)(trees * cells_of(vocab)) * sizeof(double);
}

msa_status fail(const char* who, msa_status st, const std::string& msg) {
  set_last_error(std::string(who) + ": " + msg);
  return st;
}

bool aligned(const void* p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

}  // namespace
}  // namespace msa

extern "C" msa_status msa_tree_verify_workspace(msa_plan_t plan, int32_t vocab, size_t* bytes) {
  const char* who = "msa_tree_verify_workspace";
  if (!plan || !bytes) return msa::fail(who, MSA_ERR_INVALID_ARG, "null argument");
  if (vocab < 1) return msa::fail(who, MSA_ERR_INVALID_ARG, "vocab < 1");
  *bytes = msa::workspace_of((int64_t)plan->hp.trees.size(), vocab);
  return MSA_OK;
}

extern "C" msa_status msa_tree_verify(msa_plan_t plan, int32_t prob_type, int32_t vocab, const void* target,
                                      int64_t target_stride, const void* draft, int64_t draft_stride,
                                      const int32_t* tokens, const int32_t* parents, const float* u_accept,
                                      const float* u_sample, int32_t* path, int64_t path_stride,
                                      int32_t* path_len, int32_t* next_token, void* workspace,
                                      size_t workspace_bytes, void* hip_stream) {
  const char* who = "msa_tree_verify";
  const auto invalid = [&](const std::string& msg) { return msa::fail(who, MSA_ERR_INVALID_ARG, msg); };
  if (!plan) return invalid("null plan");
  if (prob_type != MSA_PROB_F32 && prob_type != MSA_PROB_BF16 && prob_type != MSA_PROB_F16)
    return invalid("prob_type must be MSA_PROB_F32, MSA_PROB_BF16 or MSA_PROB_F16");
  if (vocab < 1) return invalid("vocab < 1");
  if (vocab > 0x7fff0000) return msa::fail(who, MSA_ERR_UNSUPPORTED, "vocab > 2^31 - 2^16");
  if (plan->host_only) return invalid("plan was built with MSA_PLAN_HOST_ONLY");
  const msa::HostPlan& hp = plan->hp;
  const int64_t trees = (int64_t)hp.trees.size();
  if (trees == 0) return MSA_OK;
  if (target_stride < vocab || (draft && draft_stride < vocab)) return invalid("row strides must be at least vocab");
  if (path_stride < hp.max_slots)
    return invalid("path_stride must be at least " + std::to_string(hp.max_slots));
  if (!target || !tokens || !parents || !u_accept || !u_sample || !path || !path_len || !next_token)
    return invalid("all pointers but draft must be non-null");
  const uintptr_t size = prob_type == MSA_PROB_F32 ? 4 : 2;
  if (!msa::aligned(target, size) || !msa::aligned(draft, size) || !msa::aligned(tokens, 4) ||
      !msa::aligned(parents, 4) || !msa::aligned(u_accept, 4) || !msa::aligned(u_sample, 4) ||
      !msa::aligned(path, 4) || !msa::aligned(path_len, 4) || !msa::aligned(next_token, 4))
    return invalid("pointers must be aligned to their elements");
  const size_t need = msa::workspace_of(trees, vocab);
  if (!workspace || !msa::aligned(workspace, 16) || workspace_bytes < need)
    return invalid("workspace must be 16-byte aligned and hold " + std::to_string(need) + " bytes");
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev != plan->device)
    return invalid("current device differs from the plan's device");
  msa::VerifyParams v{};
  v.target = target;
  v.draft = draft;
  v.target_stride = target_stride;
  v.draft_stride = draft_stride;
  v.tokens = tokens;
  v.parents = parents;
  v.u_accept = u_accept;
  v.u_sample = u_sample;
  v.path = path;
  v.path_stride = path_stride;
  v.path_len = path_len;
  v.next_token = next_token;
  v.trees = plan->d_trees;
  v.walk = static_cast<msa::WalkResult*>(workspace);
  v.sums = reinterpret_cast<double*>(static_cast<char*>(workspace) + msa::walk_bytes(trees));
  v.vocab = vocab;
  v.max_slots = hp.max_slots;
  v.cells = (int32_t)msa::cells_of(vocab);
  // a wave per cell, up to some 4096 workgroups of them
  constexpr int kCellsAtOnce = msa::kSumsThreads / msa::kWave;
  v.groups = (int32_t)std::min<int64_t>((v.cells + kCellsAtOnce - 1) / kCellsAtOnce, std::max<int64_t>(1, 4096 / trees));
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const int rc = prob_type == MSA_PROB_F32    ? msa::launch_verify<float>(v, (int)trees, s)
                 : prob_type == MSA_PROB_BF16 ? msa::launch_verify<__hip_bfloat16>(v, (int)trees, s)
                                              : msa::launch_verify<__half>(v, (int)trees, s);
  return msa::launched(who, "verification", rc);
}
