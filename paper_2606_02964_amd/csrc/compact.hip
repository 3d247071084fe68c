// compact.hip -- moves kept cache positions to the front, in place
// (msa_kv_compact).
//
// Position base + i of a sequence takes the K and V of position base + index[i],
// index strictly ascending, hence index[i] >= i: a source lies at or behind
// its destination and, for a run of moves, behind every destination of the moves
// before it.  One workgroup per (sequence, KV head, 64 channels of K or of V)
// therefore goes through the list in runs of 128 moves, in order: what a run writes
// lies before everything that later runs read, so later runs' reads may be under way
// already, and the only wait is for the run's own reads, of all waves, before
// its writes (one barrier a run).
// The places of the moves (index, then two block-table entries) are entered three runs
// ahead by two waves of their own, and K and V are read two runs ahead.  Reads and
// writes of a wave are waited for by number, in the order of their issue, so every
// read is unconditional and so are the writes of a run whose places all move: else a
// wait for a run's reads would be one for the last writes too, or, in a wave that
// looks up places between them, for all reads (one sequence of 16K, half of it kept,
// 8 heads, d = 128: 124 us like that, 89 waiting by number, 75 with the two waves; of
// 128K: 1182, 680, 624 us).
//   K: rows of 128 bytes, in 16-byte pieces from register to register.
//   V: a block holds the 16 tokens of a channel side by side, and kept tokens
//   change their place in it.  The channel rows (32 bytes) of each source block
//   are read once, whole, and its kept tokens go to their place in a staging
//   buffer in LDS, from where full pieces of 8 tokens are written.  (Gathered
//   token by token in 2-byte reads, half of 16 x 16K tokens, 8 heads, d = 128, took
//   955 us; a 2-byte read of a wave touches 16 lines for 128 bytes.)
// Bound by HBM where there are enough sequences: each moved byte is read and written
// once, and whole blocks of V are read where half of their tokens stay (16 sequences
// of up to 16K, half kept: 183 us for 0.75 GB).  One sequence alone is bound by
// its runs, one after the other, 1.2 us each: the staging's 2-byte LDS writes and
// the barrier (three or four runs ahead, or more blocks of one, take as long).
// Lists of up to 64 entries (a tree's path) take a workgroup per (sequence, KV head,
// 32 channels), which holds them in LDS between reading and writing: 48 x 8 heads,
// 4 entries, 3.6 us; 128 x 8 heads, 8 and 64 entries 8.8 and 37 us, in runs 35 and
// 51; one sequence of 64 entries 5.6 and 5.4.  (A workgroup for all 128 channels:
// 10.2 us for the last, as 2-byte reads go one line each.)
#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>

#include "errors.h"
#include "forward.h"
#include "msa_cache.h"
#include "plan.h"

namespace msa {
namespace {

constexpr int kRun = 128;  // moves of a run: two waves' lanes hold one each
constexpr int kSlice = 64;   // channels of a workgroup
constexpr int kCompactThreads = 512;  // that move; kRun more look up places
constexpr int kRing = 5;     // runs whose places are held: the one written, three ahead, one slow waves still write
constexpr int kReadAhead = 2;  // runs
constexpr int kAhead = 3;    // V blocks of a run that a wave reads ahead
constexpr int kShort = 64;   // entries of a list that are held between reading and writing
constexpr int kShortSlice = 32;     // channels of a workgroup that does
constexpr int kShortThreads = 128;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));  // (stays in neighbouring registers)

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

// Where a run's moves lead, as element offsets in the head's cache.
struct PlacesK {
  int64_t src[kRun];
  int64_t dst[kRun];  // -1: no move
};
struct __attribute__((aligned(16))) PlacesV {
  // the distinct source blocks of each 64 moves, in order
  int64_t block[2][64];
  // by block and token: the run's move that takes it, kNoMove for none
  uint8_t slot[2][64][kBlockSize];
  // by 8 neighbouring moves: where their piece lies, and which of its tokens are moved to
  int64_t piece[kRun / 8];
  uint8_t moved[kRun / 8];
  int32_t blocks[2];
};
// s_waitcnt's operand: no loads or stores outstanding
constexpr int kNoLoads = 0x0f70;
constexpr int kNoMove = kRun;  // a column of the staging buffer that is not written out

// The list's positions, and where they are in the cache.
struct Moves {
  const int32_t* index;
  const int32_t* table;
  int64_t base, end, sb, st;
  int n, lead, num_blocks;

  // the move at entry i (of the list's entries shifted by lead): index[i], or -1; read, and tested
  __device__ __forceinline__ int32_t read_from(int i) const { return index[min(max(i, 0), n - 1)]; }
  __device__ __forceinline__ int32_t from(int i, int32_t read) const { return i >= 0 && i < n ? read : -1; }
  // the block of a position, or -1; likewise
  __device__ __forceinline__ int32_t read_block(int64_t pos) const {
    return table[min(max(pos, (int64_t)0), end - 1) / kBlockSize];
  }
  __device__ __forceinline__ int32_t block(int64_t pos, int32_t read) const {
    return pos >= 0 && pos < end && read < num_blocks ? read : -1;
  }
};

// What lane m of the last two waves knows of move m of a run on the way to its places.
struct Lookup {
  int32_t from = -1, src_blk = -1, dst_blk = -1;
};

__device__ __forceinline__ bool is_move(const Moves& mv, int i, const Lookup& l) {
  return l.from > i && l.from >= 0 && l.src_blk >= 0 && l.dst_blk >= 0;  // (a place kept where it is needs no move)
}
__device__ __forceinline__ void enter_places(PlacesK& at, const Moves& mv, int i, const Lookup& l) {
  const int m = threadIdx.x - kCompactThreads;
  const bool moves = is_move(mv, i, l);
  const int src_tok = (int)((mv.base + l.from) & (kBlockSize - 1)), dst_tok = (int)((mv.base + i) & (kBlockSize - 1));
  at.src[m] = moves ? l.src_blk * mv.sb + src_tok * mv.st : 0;  // (what is read where nothing moves is not used)
  at.dst[m] = moves ? l.dst_blk * mv.sb + dst_tok * mv.st : -1;
}
__device__ __forceinline__ void enter_places(PlacesV& at, const Moves& mv, int i, const Lookup& l) {
  const int m = threadIdx.x - kCompactThreads, lane = m & 63, half = m >> 6;
  const bool moves = is_move(mv, i, l);
  const int src_tok = (int)((mv.base + l.from) & (kBlockSize - 1)), dst_tok = (int)((mv.base + i) & (kBlockSize - 1));
  const int32_t blk = moves ? l.src_blk : -1;
  const int32_t below = __shfl_up(blk, 1);  // (by all lanes: one that does not take part would read as block 0)
  const bool leads = moves && (lane == 0 || blk != below);
  const uint64_t leaders = __ballot(leads), movers = __ballot(moves);
  const int g = __popcll(leaders & (~0ull >> (63 - lane))) - 1, blocks = __popcll(leaders);
  if (lane >= blocks) at.block[half][lane] = 0;
  if (leads) {
    at.block[half][g] = blk * mv.sb;
    *reinterpret_cast<uint4*>(at.slot[half][g]) = make_uint4(0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u);
  }
  if (moves) at.slot[half][g][src_tok] = (uint8_t)m;  // (a wave's LDS writes stay in order)
  if (lane % 8 == 0) {  // (runs start at block borders: dst_tok is 0 or 8)
    at.piece[m / 8] = l.dst_blk * mv.sb + dst_tok;
    at.moved[m / 8] = (uint8_t)(movers >> lane);
  }
  if (lane == 0) at.blocks[half] = blocks;
}
static_assert(kNoMove == 0x80, "the empty slot");

// The lookups, by the last two waves: each call enters one more run's places and issues
// the reads of the runs behind it, which arrive until the next call (each is used, and
// tested, there and not before: a wait here would be one for all reads under way).
struct Lookups {
  int32_t from = -1;             // index entry, of run `next`
  int32_t src_blk = 0, dst_blk = 0;  // as read from the table, of run `next`
  int32_t behind = 0;            // as read from the index, of run next + 1
  int next = 0;
  __device__ __forceinline__ int entry(const Moves& mv, int run) const {
    return run * kRun - mv.lead + (int)threadIdx.x - kCompactThreads;
  }
  __device__ __forceinline__ void start(const Moves& mv) {
    from = mv.from(entry(mv, 0), mv.read_from(entry(mv, 0)));
    read(mv);
  }
  __device__ __forceinline__ void read(const Moves& mv) {
    src_blk = mv.read_block(mv.base + from);
    dst_blk = mv.read_block(mv.base + entry(mv, next));
    behind = mv.read_from(entry(mv, next + 1));
  }
  template <class P>
  __device__ __forceinline__ void step(const Moves& mv, P (&ring)[kRing]) {
    const int i = entry(mv, next);
    const Lookup l{from, mv.block(mv.base + from, src_blk), mv.block(mv.base + i, dst_blk)};
    enter_places(ring[next % kRing], mv, i, l);
    ++next;
    from = mv.from(entry(mv, next), behind);
    read(mv);
  }
};

// the barrier that follows each run's reads: LDS writes of every wave are done
// (the reads have arrived: their registers were used before it)
__device__ __forceinline__ void run_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// The last two waves' part: as many barriers as the others meet.
template <class P>
__device__ __forceinline__ void look_up(const Moves& mv, P (&ring)[kRing], int runs) {
  Lookups look;
  look.start(mv);
  for (int r = 0; r < kReadAhead + 1; ++r) look.step(mv, ring);
  __syncthreads();
  for (int r = 0; r < (runs + 1) / 2 * 2; ++r) {
    look.step(mv, ring);
    run_barrier();
  }
}

__device__ __forceinline__ void compact_k(uint16_t* cache, const PlacesK (&ring)[kRing], int runs) {
  constexpr int kPieces = kSlice / 8, kEach = kRun * kPieces / kCompactThreads;
  const int tid = threadIdx.x;
  u32x4 x[kReadAhead][kEach];
  auto read = [&](u32x4 (&y)[kEach], int r) __attribute__((always_inline)) {
    const PlacesK& at = ring[r % kRing];
#pragma unroll
    for (int e = 0; e < kEach; ++e)
      y[e] = *reinterpret_cast<const u32x4*>(cache + at.src[(e * kCompactThreads + tid) / kPieces] + tid % kPieces * 8);
  };
  auto step = [&](u32x4 (&now)[kEach], int r) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < kEach; ++e) asm volatile("" : "+v"(now[e]));
    run_barrier();
    const PlacesK& at = ring[r % kRing];
    int64_t dst[kEach];
    bool all = true;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      dst[e] = at.dst[(e * kCompactThreads + tid) / kPieces];
      all = all && dst[e] >= 0;
    }
    if (__ballot(all) == ~0ull) {
#pragma unroll
      for (int e = 0; e < kEach; ++e) *reinterpret_cast<u32x4*>(cache + dst[e] + tid % kPieces * 8) = now[e];
    } else {
#pragma unroll
      for (int e = 0; e < kEach; ++e)
        if (dst[e] >= 0) *reinterpret_cast<u32x4*>(cache + dst[e] + tid % kPieces * 8) = now[e];
      __builtin_amdgcn_s_waitcnt(kNoLoads);
    }
    read(now, r + kReadAhead);  // (unconditional, so that the wait for the run before it can leave it out)
  };
  read(x[0], 0);
  read(x[1], 1);
  for (int r = 0; r < runs; r += 2) {
    step(x[0], r);
    step(x[1], r + 1);  // (behind the last run nothing moves)
  }
}

// Staged tokens of a run: [channel][move], rows of a multiple of 16 bytes, some
// columns for what does not stay
constexpr int kStagePitch = kRun + 8;

__device__ __forceinline__ void compact_v(uint16_t* cache, int64_t v_sd, const PlacesV (&ring)[kRing],
                                          uint16_t (&stage)[2][kSlice][kStagePitch], int runs) {
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = wave & 1, first_block = wave >> 1;  // four waves share a half run's blocks
  // a lane holds 8 tokens of one channel, and of the channel 32 further on
  const int c = lane >> 1, side = lane & 1;
  const uint16_t* from = cache + c * v_sd + side * 8;
  u32x4 x[kReadAhead][kAhead][2];
  auto read_block = [&](u32x4 (&y)[2], int64_t block) __attribute__((always_inline)) {
    y[0] = *reinterpret_cast<const u32x4*>(from + block);
    y[1] = *reinterpret_cast<const u32x4*>(from + block + 32 * v_sd);
  };
  auto read = [&](u32x4 (&y)[kAhead][2], int r) __attribute__((always_inline)) {
    const PlacesV& at = ring[r % kRing];
#pragma unroll
    for (int a = 0; a < kAhead; ++a) read_block(y[a], at.block[half][first_block + 4 * a]);
  };
  auto step = [&](u32x4 (&now)[kAhead][2], int r) __attribute__((always_inline)) {
    const PlacesV& at = ring[r % kRing];
    const int blocks = __builtin_amdgcn_readfirstlane(at.blocks[half]);
    uint16_t(&to)[kSlice][kStagePitch] = stage[r & 1];
    // each of a lane's tokens to the column of its move (most hold one), or to the spare one
    auto put = [&](const u32x4 a, const u32x4 b, int g) __attribute__((always_inline)) {
      const uint2 slot = *reinterpret_cast<const uint2*>(&at.slot[half][g][side * 8]);
      const uint32_t wa[4] = {a.x, a.y, a.z, a.w}, wb[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        const int m = (int)((t < 4 ? slot.x : slot.y) >> (t % 4 * 8) & 0xff);
        to[c][m] = (uint16_t)(wa[t / 2] >> (t % 2 * 16));
        to[c + 32][m] = (uint16_t)(wb[t / 2] >> (t % 2 * 16));
      }
    };
#pragma unroll
    for (int a = 0; a < kAhead; ++a)
#pragma unroll
      for (int h = 0; h < 2; ++h) asm volatile("" : "+v"(now[a][h]));
#pragma unroll
    for (int a = 0; a < kAhead; ++a)
      if (first_block + 4 * a < blocks) put(now[a][0], now[a][1], first_block + 4 * a);
    for (int g = first_block + 4 * kAhead; g < blocks; g += 4) {  // kept tokens far apart
      u32x4 y[2];
      read_block(y, at.block[half][g]);
      put(y[0], y[1], g);
    }
    run_barrier();
    // 32 channels of one destination block a wave
    constexpr int kOut = kSlice * (kRun / 8) / kCompactThreads;
    int moved[kOut], ch[kOut], piece[kOut];
    bool all = true;
#pragma unroll
    for (int e = 0; e < kOut; ++e) {
      const int unit = e * (kCompactThreads / 64) + wave;  // (block of the run, channel half)
      piece[e] = (unit >> 1) * 2 + side, ch[e] = (unit & 1) * 32 + c;
      moved[e] = at.moved[piece[e]];
      all = all && moved[e] == 0xff;
    }
    if (__ballot(all) == ~0ull) {
#pragma unroll
      for (int e = 0; e < kOut; ++e)
        *reinterpret_cast<u32x4*>(cache + at.piece[piece[e]] + ch[e] * v_sd) =
            *reinterpret_cast<const u32x4*>(&to[ch[e]][piece[e] * 8]);
    } else {
#pragma unroll
      for (int e = 0; e < kOut; ++e) {
        if (moved[e] == 0) continue;
        const u32x4 y = *reinterpret_cast<const u32x4*>(&to[ch[e]][piece[e] * 8]);
        uint16_t* dst = cache + at.piece[piece[e]] + ch[e] * v_sd;
        const uint32_t w[4] = {y.x, y.y, y.z, y.w};
        if (moved[e] == 0xff) {
          *reinterpret_cast<u32x4*>(dst) = y;
        } else {
#pragma unroll
          for (int t = 0; t < 8; ++t)
            if (moved[e] >> t & 1) dst[t] = (uint16_t)(w[t / 2] >> (t % 2 * 16));
        }
      }
      __builtin_amdgcn_s_waitcnt(kNoLoads);
    }
    read(now, r + kReadAhead);  // (unconditional, so that the wait for the run before it can leave it out)
  };
  read(x[0], 0);
  read(x[1], 1);
  for (int r = 0; r < runs; r += 2) {
    step(x[0], r);
    step(x[1], r + 1);  // (behind the last run nothing moves)
  }
}

template <int D>
__global__ __launch_bounds__(kCompactThreads + kRun, 5) void msa_kv_compact_kernel(CompactParams p) {
  __shared__ union {
    PlacesK k[kRing];
    PlacesV v[kRing];
  } ring;
  __shared__ __attribute__((aligned(16))) uint16_t stage[2][kSlice][kStagePitch];
  constexpr int kParts = 2 * D / kSlice;  // K slices, then V slices
  const int part = blockIdx.x % kParts, rest = blockIdx.x / kParts;
  const int seq = rest / p.num_kv_heads, head = rest - seq * p.num_kv_heads, tid = threadIdx.x;
  const bool is_v = part >= kParts / 2;
  const int slice = is_v ? part - kParts / 2 : part;
  Moves mv;
  // (entries from end - base on have no destination in the table; base may be negative, then the first ones have none)
  mv.end = (int64_t)p.max_blocks * kBlockSize;
  mv.base = p.base ? p.base[seq] : 0;
  mv.n = (int)max((int64_t)0, min((int64_t)min(p.count[seq], p.max_count), min(mv.end - mv.base, (int64_t)0x7ffff000)));
  if (mv.n == 0) return;
  mv.index = p.index + (int64_t)seq * p.i_sb + (int64_t)head * p.i_sh;
  mv.table = p.block_table + (int64_t)seq * p.max_blocks;
  mv.num_blocks = p.num_blocks;
  mv.sb = is_v ? p.v_sb : p.k_sb;
  mv.st = is_v ? 1 : p.k_st;
  mv.lead = (int)(mv.base & (kBlockSize - 1));  // runs end at block borders of the destination
  const int runs = (int)(((int64_t)mv.lead + mv.n + kRun - 1) / kRun);
  if (tid >= kCompactThreads) {
    if (is_v)
      look_up(mv, ring.v, runs);
    else
      look_up(mv, ring.k, runs);
    return;
  }
  __syncthreads();  // the first runs' places are entered
  if (is_v)
    compact_v(p.v + (int64_t)head * p.v_sh + slice * kSlice * p.v_sd, p.v_sd, ring.v, stage, runs);
  else
    compact_k(p.k + (int64_t)head * p.k_sh + slice * kSlice, ring.k, runs);
}

// Lists of up to kShort entries: everything is read before anything is written.
template <int D>
__global__ __launch_bounds__(kShortThreads) void msa_kv_compact_short_kernel(CompactParams p) {
  __shared__ __attribute__((aligned(16))) uint16_t s_k[kShort][kShortSlice], s_v[kShort][kShortSlice];
  __shared__ int64_t k_src[kShort], k_dst[kShort], v_src[kShort], v_dst[kShort];
  constexpr int kParts = D / kShortSlice;
  const int item = blockIdx.x / kParts, channel = (blockIdx.x - item * kParts) * kShortSlice;
  const int seq = item / p.num_kv_heads, head = item - seq * p.num_kv_heads, tid = threadIdx.x;
  const int n = max(0, min(min(p.count[seq], p.max_count), kShort));
  if (n == 0) return;
  Moves mv;
  mv.n = n;
  mv.base = p.base ? p.base[seq] : 0;
  mv.index = p.index + (int64_t)seq * p.i_sb + (int64_t)head * p.i_sh;
  mv.table = p.block_table + (int64_t)seq * p.max_blocks;
  mv.end = (int64_t)p.max_blocks * kBlockSize;
  mv.num_blocks = p.num_blocks;
  if (tid < n) {
    const int32_t from = mv.index[tid];
    const int64_t src = mv.base + from, dst = mv.base + tid;
    const int32_t sb = from > tid ? mv.block(src, mv.read_block(src)) : -1, db = mv.block(dst, mv.read_block(dst));
    const bool moves = sb >= 0 && db >= 0;
    const int st = (int)(src & (kBlockSize - 1)), dt = (int)(dst & (kBlockSize - 1));
    k_src[tid] = moves ? sb * p.k_sb + st * p.k_st : 0;  // (what is read where nothing moves is not used)
    v_src[tid] = moves ? sb * p.v_sb + st : 0;
    k_dst[tid] = moves ? db * p.k_sb + dt * p.k_st : -1;
    v_dst[tid] = moves ? db * p.v_sb + dt : -1;
  }
  __syncthreads();
  uint16_t* k = p.k + (int64_t)head * p.k_sh + channel;
  uint16_t* v = p.v + (int64_t)head * p.v_sh + channel * p.v_sd;
  constexpr int kPieces = kShortSlice / 8, kBatch = 8;  // reads of a thread under way together
  const int pieces = n * kPieces, tokens = n * kShortSlice;
  for (int e0 = tid; e0 < tokens; e0 += kShortThreads * kBatch) {
    uint16_t x[kBatch];
    uint4 y;
    const int ek = (e0 - tid) / kBatch + tid;  // a piece of K for 8 tokens of V
    if (ek < pieces) y = *reinterpret_cast<const uint4*>(k + k_src[ek / kPieces] + ek % kPieces * 8);
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int e = min(e0 + i * kShortThreads, tokens - 1);
      x[i] = v[v_src[e / kShortSlice] + e % kShortSlice * p.v_sd];
    }
    if (ek < pieces) *reinterpret_cast<uint4*>(&s_k[ek / kPieces][ek % kPieces * 8]) = y;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int e = min(e0 + i * kShortThreads, tokens - 1);
      s_v[e / kShortSlice][e % kShortSlice] = x[i];
    }
  }
  __syncthreads();
  for (int e = tid; e < pieces; e += kShortThreads) {
    const int64_t dst = k_dst[e / kPieces];
    if (dst >= 0) *reinterpret_cast<uint4*>(k + dst + e % kPieces * 8) = *reinterpret_cast<const uint4*>(&s_k[e / kPieces][e % kPieces * 8]);
  }
  for (int e = tid; e < tokens; e += kShortThreads) {
    const int64_t dst = v_dst[e / kShortSlice];
    if (dst >= 0) v[dst + e % kShortSlice * p.v_sd] = s_v[e / kShortSlice][e % kShortSlice];
  }
}

template <int D>
int launch_compact(const CompactParams& p, int64_t heads, hipStream_t s) {
  if (p.max_count <= kShort)
    hipLaunchKernelGGL(msa_kv_compact_short_kernel<D>, dim3((uint32_t)heads * (D / kShortSlice)), dim3(kShortThreads), 0,
                       s, p);
  else
    hipLaunchKernelGGL(msa_kv_compact_kernel<D>, dim3((uint32_t)heads * (2 * D / kSlice)), dim3(kCompactThreads + kRun), 0, s,
                       p);
  return (int)hipGetLastError();
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
  // (a table without entries has no position to move: the kernels read an entry for every list)
  if (s.num_seqs == 0 || max_count == 0 || s.num_blocks == 0 || s.max_blocks_per_seq == 0) return MSA_OK;
  if (!index || !count || !block_table || !k_cache || !v_cache)
    return msa::fail(MSA_ERR_INVALID_ARG, "index, count, block_table, k_cache, v_cache must be non-null");
  if (!msa::aligned(k_cache, 16) || !msa::aligned(v_cache, 16) || !msa::aligned(base, 4) || !msa::aligned(index, 4) ||
      !msa::aligned(count, 4) || !msa::aligned(block_table, 4))
    return msa::fail(MSA_ERR_INVALID_ARG, "caches must be 16-byte, the others 4-byte aligned");
  // (a launch counts its threads in 32 bits: up to 4 x 640 for each)
  if ((int64_t)s.num_seqs * s.num_kv_heads >= ((int64_t)1 << 20))
    return msa::fail(MSA_ERR_UNSUPPORTED, "too many heads for one launch");
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
  const int64_t heads = (int64_t)s.num_seqs * s.num_kv_heads;
  const int rc = s.head_dim == 128 ? msa::launch_compact<128>(p, heads, stream) : msa::launch_compact<64>(p, heads, stream);
  return msa::launched("msa_kv_compact", "compaction", rc);
}
