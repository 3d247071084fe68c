// attn8_device.h -- work items of up to 32 rows over an 8-bit cache (decode_item of
// attn_device.h, which has the mathematics, over bytes).
//
// The four waves of a workgroup hold the same rows and take 32-key half-steps in
// turn.  A wave copies its half-steps' pages into LDS of its own, two stages of 8 KB (in
// the area that its partial output takes at the end).  Where a (block, KV head) lies together, as in the layout
// that make_shape gives, every copy takes whole cache lines, so they can be
// non-temporal, which the caches' lines read in parts cannot.  64 rows over 8000 keys, 32 query
// heads on 8, d = 128: 164 us, 6.5 TB/s, where operands read straight into registers took 181 and these
// copies without the hint 182 (bf16 350); 8 rows 26.5 (29.4, bf16 51.0); one over 120000 keys 47
// (54.5), over 30000 18.0 with its merge (19.2, bf16 28.3); 48 rows with a window of 4096 keys 70.5 (without the
// hint 76.7; bf16 129).  The hint costs, us with / without, where sequences share all their blocks (16 over 30000
// keys, 16 heads of 64: 130 / 120; at d = 128 nothing), one short row (a window of 4096 keys: 11.2 / 10.6), and with
// strides that put several heads into a line (a token's and a channel's heads side by side), which take
// four times as long either way (64 over 8000, 8 heads of 128: 703 / 700, 16 of 64 790 / 745; windows of 4096 keys 302 /
// 250, 319 / 283, in bf16 326 / 281), most of all if their blocks are shared (520 / 191).
//   * QK: lane half hl holds channels 32 i + 16 hl .. + 15 of its key (and of Q): a
//     product does not mind the order of its terms, and a read from LDS is 16 bytes.  A key's
//     power of two goes into the conversion to bf16, which is exact.
//   * PV: a V chunk is 16 tokens of a channel, so lane half hl takes the tokens of
//     block hl of the half-step's two.  K's rows are ordered such that the lane's 16
//     scores are these tokens' too, in order: weights meet V without a move.  A
//     token's power of two multiplies its weight (exactly), not its d values.
// Bound by HBM where there are rows to fill it, else by the pieces' starts and the merge's launch.
#pragma once

#include "attn_device.h"

namespace msa {
namespace {

__device__ __forceinline__ bf16x8 fp8_octet(uint32_t lo, uint32_t hi, float scale) {
  return __builtin_bit_cast(bf16x8, make_uint4(fp8_pair<false>(lo, scale), fp8_pair<true>(lo, scale),
                                               fp8_pair<false>(hi, scale), fp8_pair<true>(hi, scale)));
}

// 4 bytes a lane straight into LDS, as dma16
__device__ __forceinline__ void stream4(const void* src, void* lds) {
  const uint32_t l = (uint32_t)(uintptr_t)(lds_void_t*)lds;
  asm volatile("s_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(src), "{m0}"(l) : "memory");
}

template <int D, bool kPrecise, class P>
__device__ __forceinline__ void decode8_item(const P& p, const WorkItem w, DecodeLds<D>& lds) {
  constexpr int kWaves = DecodeLds<D>::kWaves, kHalf = 32;
  if (w.nrows == 0) return;  // (uniform over the workgroup)

  // (an opaque copy of the thread id: lane-dependent set-up is computed per item)
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63, hl = lane >> 5, ln = lane & 31;
  const int G = p.group;
  const int t = div_group(ln, p), hh = ln - t * G;  // tile row ln <-> token t, head hh of the group
  const bool valid = t < w.nrows;
  const int tok = w.row0 + t;
  const int head = w.kv_head * G + hh;
  const auto axis = key_axis(p, w);

  // the two blocks of half-step h, as in decode_item
  const int32_t* bt = p.block_table + (int64_t)w.seq * p.max_blocks;
  const int nh = (w.kv_hi - w.kv_lo + kHalf - 1) / kHalf;
  auto table_blocks = [&](int h, int32_t& id0, int32_t& id1) {
    const int k0 = w.kv_lo + h * kHalf;
    id0 = bt[axis.block(k0)];
    id1 = k0 + kBlockSize < w.kv_hi ? bt[axis.next_block(k0)] : id0;
  };
  int32_t idv0 = 0, idv1 = 0;
  if (wave + kWaves * lane < nh) table_blocks(wave + kWaves * lane, idv0, idv1);

  const auto row_of = row_view(p, valid, tok);
  const int pos = row_of.pos;
  constexpr int kQk = D / 16;  // QK MFMAs per half-step
  bf16x8 qf[kQk];
  {
    const uint16_t* qrow = p.q + (int64_t)tok * p.q_st + (int64_t)head * p.q_sh + hl * 16;
#pragma unroll
    for (int kk = 0; kk < kQk; ++kk) {
      if (valid) {
        qf[kk] = *reinterpret_cast<const bf16x8*>(qrow + (kk >> 1) * 32 + (kk & 1) * 8);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) qf[kk][j] = (__bf16)0.0f;
      }
    }
  }

  // MFMA row m of K is token (m bits 4, 3, 1, 0) of block (m bit 2), so that lane half hl gets the
  // scores of block hl, register e those of token e
  const int kblk = (ln >> 2) & 1, ktok = ((ln >> 3) & 3) * 4 + (ln & 3);
  // copies of a half-step into the wave's part of LDS, whole cache lines of K and of V each: token t's 16-byte
  // chunk c goes to place c ^ swizzle(t), so that a chunk of all tokens lies over all banks
  constexpr int kRowChunks = D / 16, kCopyToks = 64 / kRowChunks, kCopies = 16 / kCopyToks;  // of a block's K
  constexpr int kStage = 2 * kHalf * D + 256, kOps = 4 * kCopies + 1;
  static_assert(2 * kStage <= (int)sizeof(lds.mo[0]), "the copies fit the wave's part of the merge area");
  char* const ring = reinterpret_cast<char*>(lds.mo[wave]);
  auto swizzle = [](int token) { return token / (16 / kRowChunks) % kRowChunks; };
  const char* kbase = reinterpret_cast<const char*>(p.k) + (int64_t)w.kv_head * p.k_sh;
  const char* vbase = reinterpret_cast<const char*>(p.v) + (int64_t)w.kv_head * p.v_sh;
  uint32_t koff[kCopies];
#pragma unroll
  for (int j = 0; j < kCopies; ++j) {
    int token = j * kCopyToks + lane / kRowChunks;
    asm volatile("" : "+v"(token));  // (else strides times constants are held in scalar registers over all items)
    koff[j] = (uint32_t)(token * p.k_st + (lane % kRowChunks ^ swizzle(token)) * 16);
  }
  uint32_t voff[D / 64];
#pragma unroll
  for (int j = 0; j < D / 64; ++j) {
    int channel = j * 64 + lane;
    asm volatile("" : "+v"(channel));
    voff[j] = (uint32_t)(channel * p.v_sd);
  }
  const uint8_t* sbase = (lane & 8 ? p.v_scale : p.k_scale) + w.kv_head * kBlockSize + (lane & 3) * 4;
  int32_t scales = p.num_kv_heads * kBlockSize;  // of a block
  asm volatile("" : "+v"(scales));  // (in vector registers: scalar ones are short)

  auto blocks = [&](int h, int64_t& id0, int64_t& id1) __attribute__((always_inline)) {
    const int i = (h - wave) / kWaves;  // wave-uniform
    if (i < 64) {
      id0 = __builtin_amdgcn_readlane(idv0, i);
      id1 = __builtin_amdgcn_readlane(idv1, i);
    } else {
      int32_t a, b;
      table_blocks(h, a, b);
      id0 = a;
      id1 = b;
    }
  };
  auto load = [&](int b, int h) __attribute__((always_inline)) {
    int64_t id[2];
    blocks(h, id[0], id[1]);
    char* const to = ring + b * kStage;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int j = 0; j < kCopies; ++j) stream16(kbase + id[u] * p.k_sb, koff[j], to + (u * kCopies + j) * 1024);
    stream4(sbase + (lane & 4 ? id[1] : id[0]) * scales, to + 2 * kHalf * D);
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int j = 0; j < D / 64; ++j)
        stream16(vbase + id[u] * p.v_sb, voff[j], to + kHalf * D + (u * D + j * 64) * 16);
  };

  const float c = p.scale_log2;
  float m_ref = -__builtin_inff(), l_run = 0.0f;
  f32x16 oacc[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) oacc[dt][i] = 0.0f;

  int pmin = 0, pmax = 0;  // positions of the tile's first and last row (set below, once loads are under way)
  auto half = [&](auto bsel, int h) __attribute__((always_inline)) {
    constexpr int b = decltype(bsel)::value;
    if (h + kWaves < nh) {
      __builtin_amdgcn_s_waitcnt(0xc07f);  // the reads of that stage, lgkmcnt(0)
      load(1 - b, h + kWaves);
      wait_dma<kOps>();
    } else {
      wait_dma<0>();
    }
    asm volatile("" ::: "memory");
    const char* const from = ring + b * kStage;
    const uint8_t* const sc8 = reinterpret_cast<const uint8_t*>(from + 2 * kHalf * D);
    const float kf = __uint_as_float((uint32_t)sc8[kblk * 16 + ktok] << 23);
    uint4 ka[D / 32], va[D / 32];
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
      ka[i] = *reinterpret_cast<const uint4*>(from + (kblk * 16 + ktok) * D + (2 * i + hl ^ swizzle(ktok)) * 16);
    const uint4 vs = *reinterpret_cast<const uint4*>(sc8 + 32 + hl * 16);
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
      va[i] = *reinterpret_cast<const uint4*>(from + kHalf * D + (hl * D + i * 32 + ln) * 16);
    f32x16 sc = {};
#pragma unroll
    for (int kk = 0; kk < kQk; ++kk) {
      const uint4& x = ka[kk >> 1];
      const bf16x8 a = kk & 1 ? fp8_octet(x.z, x.w, kf) : fp8_octet(x.x, x.y, kf);
      sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qf[kk], sc, 0, 0, 0);
    }
    // score e of a lane is token e of block hl
    const int k0 = axis.key(w.kv_lo + h * kHalf);
    const bool masked = k0 + kHalf - 1 >= pmin || before_window(p, k0, kHalf, pmax);
    const bool split = (k0 | (kKvStep - 1)) >= pmin || kPrecise;  // lo terms of the weights, as in decode_item
    if (masked) {
      const int lim = pos - k0 - hl * 16;
      if constexpr (P::kWindow) {
        const int low = lim - p.window, sink = p.sinks - k0 - hl * 16;
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[e] = e <= lim && (e > low || e < sink) ? sc[e] : -__builtin_inff();
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[e] = e <= lim ? sc[e] : -__builtin_inff();
      }
    }
    // weights and their sum; wv: times V's powers of two
    float wv[16], ls;
    auto weights = [&]() {
      const float nm = m_ref == -__builtin_inff() ? 0.0f : -m_ref;
      ls = 0.0f;
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        wv[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[e], c, nm));
        wv[e + 1] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[e + 1], c, nm));
        ls += wv[e] + wv[e + 1];
      }
    };
    weights();
    if (__any(!(ls < kSettleSum) || m_ref == -__builtin_inff())) {  // the lazy reference max
      float mx = -__builtin_inff();
#pragma unroll
      for (int e = 0; e < 16; ++e) mx = fmaxf(mx, sc[e]);
      const float m_blk = pair_max(mx) * c;
      const bool grow = m_blk > m_ref + kRescaleLog2;
      if (__any(grow)) {
        const float alpha = grow ? __builtin_amdgcn_exp2f(m_ref - m_blk) : 1.0f;
        m_ref = grow ? m_blk : m_ref;
        l_run *= alpha;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) oacc[dt] *= alpha;
        weights();
      }
    }
    l_run += ls;
    const uint32_t sv[4] = {vs.x, vs.y, vs.z, vs.w};
#pragma unroll
    for (int e = 0; e < 16; ++e) wv[e] *= __uint_as_float((sv[e >> 2] >> (8 * (e & 3)) & 0xff) << 23);
    uint32_t pk[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) pk[u] = pack_bf16x2(wv[2 * u], wv[2 * u + 1]);
    const bool own = (row_of.first | (kKvStep - 1)) <= (k0 | (kKvStep - 1)) &&
                     (k0 | (kKvStep - 1)) <= (pos | (kKvStep - 1));
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      const bf16x8 ph = __builtin_bit_cast(bf16x8, make_uint4(pk[4 * ks], pk[4 * ks + 1], pk[4 * ks + 2], pk[4 * ks + 3]));
      bf16x8 a[D / 32];
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt) {
        a[dt] = ks ? fp8_octet(va[dt].z, va[dt].w, 1.0f) : fp8_octet(va[dt].x, va[dt].y, 1.0f);
        oacc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[dt], ph, oacc[dt], 0, 0, 0);
      }
      if (split) {
        uint32_t lo[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const bf16x2 hv = __builtin_bit_cast(bf16x2, pk[4 * ks + u]);
          const uint32_t x = pack_bf16x2(wv[8 * ks + 2 * u] - (float)hv[0], wv[8 * ks + 2 * u + 1] - (float)hv[1]);
          lo[u] = kPrecise || own ? x : 0u;
        }
        const bf16x8 pl = __builtin_bit_cast(bf16x8, make_uint4(lo[0], lo[1], lo[2], lo[3]));
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
          oacc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[dt], pl, oacc[dt], 0, 0, 0);
      }
    }
  };
  if (wave < nh) load(0, wave);
  pmin = __builtin_amdgcn_readfirstlane(row_of.first);
  pmax = __builtin_amdgcn_readlane(pos, w.nrows * G - 1);
  for (int h = wave; h < nh; h += 2 * kWaves) {
    half(std::integral_constant<int, 0>{}, h);
    if (h + kWaves < nh) half(std::integral_constant<int, 1>{}, h + kWaves);
  }
  merge_waves<D>(p, w, lds, tid, wave, hl, ln, oacc, m_ref, l_run);
}

}  // namespace
}  // namespace msa
