// The inner step of the bf16 attention kernels (D = 128): eight score products and eight value products of 32 keys,
// interleaved with the probabilities of 32 others (gfx950 only).
#pragma once

#include "lds_dma.h"

namespace pc {

constexpr int kD = 128;
constexpr int kRowBytes = kD * 2;    // a K or V row in LDS: 256 bytes, unpadded, chunk-swizzled
constexpr float kRescaleTrigger = 1024.f;  // row sum of a half tile that forces a new reference maximum
constexpr float kLowestStart = -4096.f;    // lowest reference that products start from (see pipeline_phase)
constexpr int kRing = 4;

// ---- LDS tile layout ---------------------------------------------------------------------------
// K tiles use the fragment-read swizzle of lds_dma.h.  V is read with transposing loads
// (4 rows x 32 bytes per quarter wave): chunk c of row r is stored at position c ^ (4 (r & 3)).
__device__ __forceinline__ int v_chunk_pos(int row, int chunk) { return chunk ^ ((row & 3) << 2); }

// One phase of the software pipeline (see the kernel comment): 8 score products, then 8
// value products, with one element of the probability stage behind each.
// The probabilities are formed against the reference m_ref as it stands; no maximum is
// taken on the fast path.  If any row sum of the half tile comes out above kRescaleTrigger
// (a score outgrew the reference: rare, at most once per 2^10 of growth), the half tile is
// redone against its exact maximum and O, l are rescaled.
// kUnitC: the caller folded scale * log2(e) into Q (c == 1).  The score products then start
// from -m_ref instead of zero (neg_m: the reference in all 16 accumulator registers of the
// lane, which holds one query), so a score arrives as s - m_ref and the probability is a bare
// exp2: one vector instruction per element fewer.  When the reference moves, the scores that
// were started from the old one are shifted by the difference.
// Keys of a score -inf, or of a mask value far below the rest, weigh nothing, and a wave may see a half
// tile of nothing else before its first real key.  c general: a reference of -inf makes the row sum
// NaN or inf, so every half tile is redone until there is a finite one, and a redo without one adds
// zeros.  A far reference's probabilities (see far_exponent) are formed in the redo, so while any query of the
// wave has one (redo_all) every half tile is redone.  kUnitC: products must not start from a low reference
// (inf - inf, or a score lost in the rounding of -m_ref: an ulp at kLowestStart is 2^-11): they start from
// zero instead, and every half tile is redone for as long.
template <bool kUnitC>
__device__ __forceinline__ void pipeline_phase(
    const lds_u8* k_half, const int (&k_off)[8], const lds_u8* v_half, const int (&v_off)[4],
    const bf16x8 (&qf)[8], f32x16& s_nxt, const bf16x8 (&p_mm)[2], f32x16 (&o)[4], const f32x16& s_cur,
    bf16x8 (&p_cur)[2], float& m_ref, float& l_run, float c, f32x16& neg_m, bool& redo_all) {
  // fragment k: 0..7 -> K rows, contraction step k; 8..15 -> V^T (key step (k-8)/4, block (k-8)%4)
  auto frag = [&](int k) -> bf16x8 {
    if (k < 8) {
      return *reinterpret_cast<const __attribute__((address_space(3))) bf16x8*>(k_half + k_off[k]);
    }
    const int ks = (k - 8) >> 2, db = (k - 8) & 3;
    // keys ks*16 + g*4 + {0..3} and + 8: two transposing reads of 4 keys each
    const lds_u8* p = v_half + v_off[db] + ks * 16 * kRowBytes;
    const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
        reinterpret_cast<__attribute__((address_space(3))) bf16x4*>(const_cast<lds_u8*>(p)));
    const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
        reinterpret_cast<__attribute__((address_space(3))) bf16x4*>(const_cast<lds_u8*>(p + 8 * kRowBytes)));
    bf16x8 f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f[e] = lo[e];
      f[4 + e] = hi[e];
    }
    return f;
  };
  bf16x8 ring[kRing];
#pragma unroll
  for (int r = 0; r < kRing; ++r) ring[r] = frag(r);
  f32x16 zero;
#pragma unroll
  for (int i = 0; i < 16; ++i) zero[i] = 0.f;
  f32x16 s_acc = zero;
  float psum = 0.f;
  float pv[16];
  // The wave asks for issue priority over its SIMD neighbour while it is inside the interleaved
  // matrix / vector block, and gives it back for the bookkeeping behind it (measured: +0.5 %).
  __builtin_amdgcn_s_setprio(1);
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    const bf16x8 f = ring[k % kRing];
    if (k < 8) {
      s_acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, qf[k], k == 0 ? (kUnitC ? neg_m : zero) : s_acc, 0, 0, 0);
    } else {
      const int ks = (k - 8) >> 2, db = (k - 8) & 3;
      o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, p_mm[ks], o[db], 0, 0, 0);
    }
    if (k + kRing < 16) ring[k % kRing] = frag(k + kRing);
    pv[k] = kUnitC ? __builtin_amdgcn_exp2f(s_cur[k]) : __builtin_amdgcn_exp2f(fmaf(s_cur[k], c, -m_ref));
    psum += pv[k];
    if (k & 1) {
      p_cur[k >> 3][(k & 7) - 1] = static_cast<__bf16>(pv[k - 1]);
      p_cur[k >> 3][k & 7] = static_cast<__bf16>(pv[k]);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  __builtin_amdgcn_s_setprio(0);
  // keep the vector results in this basic block (otherwise they sink below the next branch)
#pragma unroll
  for (int half = 0; half < 2; ++half) asm volatile("" : "+v"(p_cur[half]));
  asm volatile("" : "+v"(psum));
  if (redo_all || __any(!(psum <= kRescaleTrigger))) {  // also catches inf and NaN
    float mx = s_cur[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s_cur[i]);
    mx = wave_half_max(mx);
    // unit c: s_cur holds s - start, and so do the scores just formed; start is the reference or zero
    const float start = kUnitC ? -neg_m[0] : 0.f;
    const float m_new = fmaxf(m_ref, kUnitC ? start + mx : mx * c);
    const bool none = m_new == -INFINITY;   // no key of a finite score yet
    const float alpha = none ? 1.f : __builtin_amdgcn_exp2f(m_ref - m_new);
    const float m_use = none ? 0.f : m_new - start;
    if constexpr (!kUnitC) redo_all = __any(far_ref(m_new));
    psum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      pv[i] = __builtin_amdgcn_exp2f(kUnitC ? s_cur[i] - m_use
                                            : far_ref(m_use) ? far_exponent(s_cur[i], c, m_use) : fmaf(s_cur[i], c, -m_use));
      psum += pv[i];
    }
    if constexpr (kUnitC) {
      const float start_new = m_new >= kLowestStart ? m_new : 0.f;
      redo_all = __any(!(m_new >= kLowestStart));
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s_acc[i] -= start_new - start;
        neg_m[i] = -start_new;
      }
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) p_cur[i >> 3][i & 7] = static_cast<__bf16>(pv[i]);
    l_run *= alpha;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
    m_ref = m_new;
  }
  l_run += psum;
  s_nxt = s_acc;
}

}  // namespace pc
