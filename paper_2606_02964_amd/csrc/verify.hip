// verify.hip -- verification of trees of drafted tokens against the target's
// probabilities (msa_tree_verify; the rule is in include/msa_tree.h).
//
// Two launches.
// msa_verify_walk, one workgroup per tree: the walk reads two numbers a slot
// (p and q of the slot's token in its parent's row), all at once, and then
// takes one decision after the other in registers.  Where a node's children
// were drawn from q, the residual after n failed ones is max(a p - b q, 0) with
// two scalars a and b (max(max(x, 0) / P - q, 0) = max(x / P - q, 0), as q >= 0),
// so nothing of the vocabulary's length is stored; a second or later child's test
// needs that residual's mass, for which the workgroup reads the node's two rows.
// msa_verify_sample, chunks of the vocabulary x trees: sums r over its chunk;
// the last chunk of a tree to finish finds the chunk, then the entry, at which the
// running sum passes u T.
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

#pragma clang fp contract(off)  // a p - b q is 0 where both products are equal

namespace msa {
namespace {

constexpr int kWalkThreads = 1024;
constexpr int kSampleThreads = 256;
constexpr int kChunkMin = 2048;   // entries of a sample workgroup, at least
constexpr int kChunkMax = 32768;  // and at most (its bitmap of failed tokens is in LDS)
constexpr int kWave = 64;

// How the next token's weights follow from the last node's row(s).
enum Rest { kAsIs = 0, kResidual = 1, kWithout = 2 };

struct WalkResult {
  double a, b;       // kResidual: weights max(a p - b q, 0)
  int32_t tree_row;  // of the last node
  int32_t node;      // its slot
  int32_t rest;
  int32_t arrived;   // chunks summed so far (msa_verify_sample)
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
  double* sums;      // [trees][chunks][2]: r, p
  int32_t vocab, max_slots, chunk, chunks;
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

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
  return x;
}
// inclusive running sum over the wave
__device__ __forceinline__ double wave_scan(double x, int lane) {
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const double y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  return x;
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

// Every wave of the workgroup takes the walk's (uniform) decisions, so that
// all of them meet in residual_mass.  Children lie behind their parent, so the
// walk is one pass over the slots, 64 at a time.
template <class T>
__global__ __launch_bounds__(kWalkThreads) void msa_verify_walk_kernel(VerifyParams v) {
  __shared__ int16_t s_parent[MSA_TREE_MAX_SLOTS];
  __shared__ int32_t s_token[MSA_TREE_MAX_SLOTS];
  __shared__ float s_p[MSA_TREE_MAX_SLOTS], s_q[MSA_TREE_MAX_SLOTS], s_u[MSA_TREE_MAX_SLOTS];
  __shared__ double part[kWalkThreads / kWave];
  const TreeSpan tree = v.trees[blockIdx.x];
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
    s_parent[i] = (int16_t)up;
    s_token[i] = token;
    s_p[i] = ok ? clean(to_float(target[prow * v.target_stride + token])) : 0.0f;
    s_q[i] = ok && draft ? clean(to_float(draft[prow * v.draft_stride + token])) : 0.0f;
    s_u[i] = v.u_accept[row];
  }
  __syncthreads();

  int32_t* path = v.path + (int64_t)blockIdx.x * v.path_stride;
  int node = 0, len = 1;
  double a = 1.0, b = 0.0, mass = 1.0;
  bool known = true, dead = false, failed = false;  // mass known; no residual left; some child failed
  for (int base = 0; base < tree.n; base += kWave) {
    const int slot = base + lane;
    const bool in = slot < tree.n;
    const int up = in ? s_parent[slot] : -1;
    const int token = in ? s_token[slot] : -1;
    uint64_t children = __ballot(in && up == node);
    while (children) {
      const int l = __builtin_ctzll(children), i = base + l;
      children &= children - 1;
      double p = s_p[i], q = s_q[i];
      const double u = s_u[i];
      bool stays;
      if (draft) {
        if (!known && !dead) {
          mass = residual_mass(target + ((int64_t)tree.row0 + node) * v.target_stride,
                               draft + ((int64_t)tree.row0 + node) * v.draft_stride, a, b, v.vocab, part);
          known = true;
          dead = !(mass > 0.0);
        }
        stays = !dead && u * q * mass < fmax(a * p - b * q, 0.0);
      } else {
        // a token that failed before under this node has nothing left
        const int32_t x = s_token[i];
        bool twice = __any(in && up == node && slot < i && token == x);
        for (int e = node + 1 + lane; e < base; e += kWave) twice |= s_parent[e] == node && s_token[e] == x;
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
    v.path_len[blockIdx.x] = len;
    WalkResult r{};
    r.a = a;
    r.b = b;
    r.tree_row = tree.row0 + node;
    r.node = node;
    r.rest = !failed || dead ? kAsIs : draft ? kResidual : kWithout;
    v.walk[blockIdx.x] = r;
  }
}

// The weights of the next token: entry t of a row is weight(t).
template <class T>
struct Weights {
  const T *p, *q;
  double a, b;
  int rest, lo;
  const uint32_t* gone;  // bit t - lo: token t failed under the last node
  __device__ __forceinline__ double of(float x, float y, int t) const {
    if (rest == kResidual) return fmax(a * (double)x - b * (double)y, 0.0);
    if (rest == kWithout && (gone[(t - lo) >> 5] >> ((t - lo) & 31) & 1)) return 0.0;
    return (double)x;
  }
  __device__ __forceinline__ double at(int t) const {
    return of(clean(to_float(p[t])), rest == kResidual ? clean(to_float(q[t])) : 0.0f, t);
  }
};

// marks the failed children's tokens inside [lo, hi) in `gone`
template <class T>
__device__ void mark_failed(const VerifyParams& v, const TreeSpan& tree, const WalkResult& r, int lo, int hi,
                            uint32_t* gone) {
  const int tid = threadIdx.x;
  __syncthreads();
  for (int i = tid; i < kChunkMax / 32; i += kSampleThreads) gone[i] = 0;
  __syncthreads();
  for (int i = r.node + 1 + tid; i < tree.n; i += kSampleThreads) {
    const int32_t t = v.tokens[tree.row0 + i];
    if (v.parents[tree.row0 + i] == r.node && t >= lo && t < hi)
      atomicOr(&gone[(t - lo) >> 5], 1u << ((t - lo) & 31));
  }
  __syncthreads();
}

template <class T>
__global__ __launch_bounds__(kSampleThreads) void msa_verify_sample_kernel(VerifyParams v) {
  __shared__ uint32_t gone[kChunkMax / 32];
  __shared__ double part[2][kSampleThreads / kWave];
  __shared__ int s_last, s_found;
  const int tree_id = blockIdx.x / v.chunks, chunk = blockIdx.x - tree_id * v.chunks;
  const TreeSpan tree = v.trees[tree_id];
  const WalkResult r = v.walk[tree_id];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  Weights<T> w;
  w.p = static_cast<const T*>(v.target) + (int64_t)r.tree_row * v.target_stride;
  w.q = r.rest == kResidual ? static_cast<const T*>(v.draft) + (int64_t)r.tree_row * v.draft_stride : nullptr;
  w.a = r.a;
  w.b = r.b;
  w.rest = r.rest;
  w.gone = gone;
  {
    const int lo = chunk * v.chunk, hi = min(lo + v.chunk, v.vocab);
    w.lo = lo;
    if (r.rest == kWithout) mark_failed<T>(v, tree, r, lo, hi, gone);
    double sr = 0.0, sp = 0.0;
    const int whole = lo + ((hi - lo) & ~3);
    for (int t = lo + tid * 4; t < whole; t += kSampleThreads * 4) {
      float x[4], y[4] = {0.0f, 0.0f, 0.0f, 0.0f};
      load4(w.p + t, x);
      if (r.rest == kResidual) load4(w.q + t, y);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sr += w.of(x[i], y[i], t + i);
        sp += (double)x[i];
      }
    }
    for (int t = whole + tid; t < hi; t += kSampleThreads) {
      sr += w.at(t);
      sp += (double)clean(to_float(w.p[t]));
    }
    sr = wave_sum(sr);
    sp = wave_sum(sp);
    if (lane == 0) {
      part[0][wave] = sr;
      part[1][wave] = sp;
    }
    __syncthreads();
    if (tid == 0) {
      double* out = v.sums + ((int64_t)tree_id * v.chunks + chunk) * 2;
      out[0] = part[0][0] + part[0][1] + part[0][2] + part[0][3];
      out[1] = part[1][0] + part[1][1] + part[1][2] + part[1][3];
      __threadfence();  // the sums are seen on every XCD before the arrival is
      s_last = atomicAdd(&v.walk[tree_id].arrived, 1) == v.chunks - 1;
    }
    __syncthreads();
    if (!s_last) return;
    __threadfence();
  }

  // The tree's last workgroup: total, chunk, entry.
  const volatile double* sums = v.sums + (int64_t)tree_id * v.chunks * 2;
  double total[2] = {0.0, 0.0};
  for (int c0 = 0; c0 < v.chunks; c0 += kWave) {
    const int c = c0 + lane;
    total[0] += __shfl(wave_scan(c < v.chunks ? sums[2 * c] : 0.0, lane), kWave - 1);
    total[1] += __shfl(wave_scan(c < v.chunks ? sums[2 * c + 1] : 0.0, lane), kWave - 1);
  }
  const int which = total[0] > 0.0 ? 0 : 1;  // nothing left: the row itself
  if (!(total[which] > 0.0)) {               // uniform over the workgroup
    if (tid == 0) v.next_token[tree_id] = -1;
    return;
  }
  if (which == 1) w.rest = kAsIs;
  const float u = fminf(fmaxf(v.u_sample[tree_id], 0.0f), 0x1.fffffep-1f);  // (fmaxf of NaN and 0 is 0)
  const double x = (double)u * total[which];
  // the first chunk whose running sum passes x; where rounding leaves none, the
  // last one that holds any weight
  double before = 0.0, carry = 0.0;
  int found = -1, holds = 0;
  double holds_before = 0.0;
  for (int c0 = 0; c0 < v.chunks && found < 0; c0 += kWave) {
    const int c = c0 + lane;
    const double s = c < v.chunks ? sums[2 * c + which] : 0.0;
    const double run = carry + wave_scan(s, lane);
    const uint64_t past = __ballot(run > x), some = __ballot(s > 0.0);
    double prev = __shfl_up(run, 1);
    if (lane == 0) prev = carry;
    if (past) {
      const int l = __builtin_ctzll(past);
      found = c0 + l;
      before = __shfl(prev, l);
    } else if (some) {
      const int l = 63 - __builtin_clzll(some);
      holds = c0 + l;
      holds_before = __shfl(prev, l);
    }
    carry = __shfl(run, kWave - 1);
  }
  if (found < 0) {
    found = holds;
    before = holds_before;
  }
  const int lo = found * v.chunk, hi = min(lo + v.chunk, v.vocab);
  w.lo = lo;
  if (w.rest == kWithout) mark_failed<T>(v, tree, r, lo, hi, gone);
  // inside it, each thread takes a run of entries
  const int each = (hi - lo + kSampleThreads - 1) / kSampleThreads;
  const int t0 = min(lo + tid * each, hi), t1 = min(t0 + each, hi);
  double own = 0.0;
  for (int t = t0; t < t1; ++t) own += w.at(t);
  const double run = wave_scan(own, lane);
  __syncthreads();
  if (lane == kWave - 1) part[0][wave] = run;
  if (tid == 0) s_found = 0x7fffffff, s_last = -1;
  __syncthreads();
  double at = before;
  for (int i = 0; i < wave; ++i) at += part[0][i];
  double prev = __shfl_up(run, 1);
  at += lane == 0 ? 0.0 : prev;
  for (int t = t0; t < t1; ++t) {
    const double y = w.at(t);
    at += y;
    if (y > 0.0) {
      if (at > x) {
        atomicMin(&s_found, t);
        break;
      }
      atomicMax(&s_last, t);
    }
  }
  __syncthreads();
  if (tid == 0) v.next_token[tree_id] = s_found != 0x7fffffff ? s_found : s_last;
}

template <class T>
int launch_verify(const VerifyParams& v, int trees, hipStream_t s) {
  hipLaunchKernelGGL(msa_verify_walk_kernel<T>, dim3(trees), dim3(kWalkThreads), 0, s, v);
  const int rc = (int)hipGetLastError();
  if (rc != 0) return rc;
  hipLaunchKernelGGL(msa_verify_sample_kernel<T>, dim3((uint32_t)trees * (uint32_t)v.chunks), dim3(kSampleThreads),
                     0, s, v);
  return (int)hipGetLastError();
}

// entries of a chunk: some 1024 workgroups in all, as the chunk's bounds allow
int chunk_of(int64_t trees, int64_t vocab) {
  const int64_t per_tree = std::max<int64_t>(1, 1024 / trees);
  const int64_t c = ((vocab + per_tree - 1) / per_tree + 1023) / 1024 * 1024;
  return (int)std::min<int64_t>(kChunkMax, std::max<int64_t>(kChunkMin, c));
}
int64_t chunks_of(int64_t trees, int64_t vocab) {
  const int64_t c = chunk_of(trees, vocab);
  return (vocab + c - 1) / c;
}
size_t walk_bytes(int64_t trees) { return ((size_t)trees * sizeof(WalkResult) + 255) / 256 * 256; }
size_t workspace_of(int64_t trees, int64_t vocab) {
  return trees == 0 ? 0 : walk_bytes(trees) + (size_t)(trees * chunks_of(trees, vocab)) * 2 * sizeof(double);
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
  const int64_t chunks = msa::chunks_of(trees, vocab);
  if (trees * chunks >= ((int64_t)1 << 31))
    return msa::fail(who, MSA_ERR_UNSUPPORTED, "trees x vocab too large for one launch");
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
  v.chunk = msa::chunk_of(trees, vocab);
  v.chunks = (int32_t)chunks;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const int rc = prob_type == MSA_PROB_F32    ? msa::launch_verify<float>(v, (int)trees, s)
                 : prob_type == MSA_PROB_BF16 ? msa::launch_verify<__hip_bfloat16>(v, (int)trees, s)
                                              : msa::launch_verify<__half>(v, (int)trees, s);
  return msa::launched(who, "verification", rc);
}
