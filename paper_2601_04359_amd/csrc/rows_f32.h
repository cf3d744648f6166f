// The fp32 forms of the attention on several sequences (D = 64 or 128, gfx950 only), on the 16x16x4 fp32 MFMA: 16 kQ query rows
// per work-group, whose kW waves take the keys in steps of 16 by turns and merge their (O, m, l) through LDS once.
//   * S^T = K Q^T: lane (r = l % 16, kg = l / 16) holds key row r, dims 16 s + 4 kg .. + 3; the four products of step s contract
//     over (kg, element), the same permutation of the head dimension on both operands.
//   * The result leaves lane (q = l % 16, kg) with keys 4 kg .. + 3 of its query: P^T is the B operand of O^T += V^T P^T
//     (product e contracts over keys 4 kg + e), and row r of output block (db, e) stands for dim 64 db + 4 r + e, so that V
//     comes in 16-byte pieces and O leaves in them.
//   * A score is s (c + c_lo), and the reference is subtracted from the rounded product: the largest key's exponent is 0
//     however large the logits are.  c_lo > 0: a score of -inf stays one.
//   * A key that a row does not see has p = 0, and 0 times a NaN in V would reach the row: in steps where some row does not
//     see all keys, values that are not finite are taken out of the product and added to the rows that see them, behind the last
//     key: an infinity that went in earlier would meet the rescaling of what it stands in.
// K and V come straight from L2 to registers, the next step's K behind this one's scores and its V behind this one's
// products.  Bound: what a compute unit draws from L2 with 16 rows (16 KB per 2 x 32 products of 32 cycles and wave at D = 128),
// the products with 32; latency where there are few keys, which is why 16 rows come with eight waves.  Measured, D = 128: prompts of
// 40, 252, 333 and 1 rows, 8/2 heads, 15.4 us; 64 tokens with 1,000 rows each in pages, 16/4 heads, 45 us (5.8 TB/s).
#pragma once

#include <limits.h>

#include "seq_rows.h"

namespace pc {

constexpr int kF32Keys = 16;
template <int D, int kQ, int kW>
constexpr size_t kF32Smem = sizeof(float) * kW * kQ * 16 * (D + 2);

__device__ __forceinline__ f32x4 load_16B(const float* p) { return *reinterpret_cast<const f32x4*>(p); }

template <int D, bool kPages, int kQ, int kW>
__device__ __forceinline__ void rows_f32(const RowsArgs& a, const RowSet& r, float* smem) {
  constexpr int kSteps = D / 16, kBlocks = D / 64, kRows = 16 * kQ;
  float* o_lds = smem;                                                  // [kW][kRows][D]
  float2* ml_lds = reinterpret_cast<float2*>(smem + kW * kRows * D);    // [kW][kRows]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r16 = lane & 15, kg = lane >> 4;
  const int n_set = r.n_tok * a.rep;
  int lim[kQ], lim_max = 0, lim_min = INT_MAX;   // over the rows that see something
  // Queries stay in registers where there are 16, and in LDS (where O goes later) where there are 32: chunk c of row i lies at
  // place c ^ (i % 16), so that rows are written and fragments read with every bank.
  f32x4 qf[kQ == 1 ? kSteps : 1];
  auto q_row = [&](int i) {
    const int rho = min(r.tile * kRows + i, n_set - 1), tok = a.by_rep.of(rho), head = r.kvh * a.rep + rho - tok * a.rep;
    return static_cast<const float*>(a.Q) + head * a.q_stride + static_cast<int64_t>(r.t0 + tok) * D;
  };
  if constexpr (kQ == 1) {
    const float* q = q_row(r16) + kg * 4;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) qf[s] = load_16B(q + s * 16);
  } else {
    constexpr int kChunks = D / 4;
#pragma unroll
    for (int i = threadIdx.x; i < kRows * kChunks; i += kW * 64) {
      const int row = i / kChunks, c = i % kChunks;
      *reinterpret_cast<f32x4*>(o_lds + row * D + (c ^ (row & 15)) * 4) = load_16B(q_row(row) + c * 4);
    }
    __syncthreads();
  }
  auto q_frag = [&](int n, int s) -> f32x4 {
    if constexpr (kQ == 1) return qf[s];
    return *reinterpret_cast<const f32x4*>(o_lds + (n * 16 + r16) * D + ((4 * s + kg) ^ r16) * 4);
  };
#pragma unroll
  for (int n = 0; n < kQ; ++n) {
    lim[n] = limit_of(a, r, a.by_rep.of(min(r.tile * kRows + n * 16 + r16, n_set - 1)));
    lim_max = max(lim_max, lim[n]);
    if (lim[n] > 0) lim_min = min(lim_min, lim[n]);
  }
#pragma unroll
  for (int x = 1; x < 16; x *= 2) {
    lim_max = max(lim_max, __shfl_xor(lim_max, x));
    lim_min = min(lim_min, __shfl_xor(lim_min, x));
  }
  const int end = min(r.end, __builtin_amdgcn_readfirstlane(lim_max)), last = r.n_keys - 1;
  lim_min = __builtin_amdgcn_readfirstlane(lim_min);

  const float* Kh = static_cast<const float*>(a.K) + r.kvh * a.k_stride;
  const float* Vh = static_cast<const float*>(a.V) + r.kvh * a.v_stride;
  f32x4 acc[kQ][kBlocks][4];
  float m[kQ], l[kQ];
#pragma unroll
  for (int n = 0; n < kQ; ++n) {
    m[n] = kNothing, l[n] = 0.f;
#pragma unroll
    for (int db = 0; db < kBlocks; ++db)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[n][db][e] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  f32x4 kf[kSteps], vf[4][kBlocks];
  struct Place {
    int64_t base;   // of row 0 of what a step's keys lie in, elements
    int first;      // and the key that is row 0
    bool there;     // false: they are nobody's
  };
  // Loads are made for every step, with or without keys: rows that do not exist are read as the last one, those of a page that
  // is not there from page 0.
  auto place = [&](int kb) {
    Place t = {static_cast<int64_t>(r.k0) * D, 0, kb < end};
    if constexpr (kPages) {
      const int in_table = a.by_page.of(min(kb, last)), page = r.pages[in_table];
      const bool good = page >= 0 && page < a.n_pages;
      // (keys in front of the own rows: row_at must not reach another page)
      t.there = t.there && good && kb + kF32Keys > r.lo;
      t.base = (good ? page : 0) * a.page_stride, t.first = in_table * a.by_page.d;
    }
    return t;
  };
  // (rows in front of the own ones may lie in another page: within this one at least)
  const int page_last = kPages ? a.by_page.d - 1 : INT_MAX;
  auto row_at = [&](const Place& t, int j) {
    const int at = min(max(j, r.lo), last) - t.first;
    return t.base + static_cast<int64_t>(kPages ? min(at, page_last) : at) * D;
  };
  auto load_k = [&](const Place& t, int kb) {
    const float* p = Kh + row_at(t, kb + r16) + kg * 4;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) kf[s] = load_16B(p + s * 16);
  };
  auto load_v = [&](const Place& t, int kb) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float* p = Vh + row_at(t, kb + kg * 4 + e) + r16 * 4;
#pragma unroll
      for (int db = 0; db < kBlocks; ++db) vf[e][db] = load_16B(p + db * 64);
    }
  };

  int kb = r.begin + wave * kF32Keys;
  int odd_first = INT_MAX, odd_last = -1;   // first keys of steps with such values
  if (kb < end) {
    Place now = place(kb);
    load_k(now, kb);
    load_v(now, kb);
    do {
      const int kb_next = kb + kW * kF32Keys;
      const Place next = place(kb_next);
      float x[kQ][4];
#pragma unroll
      for (int n = 0; n < kQ; ++n) {
        f32x4 sc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};   // two chains
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
          const f32x4 q = q_frag(n, s);
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[s & 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[s][e], q[e], sc[s & 1], 0, 0, 0);
        }
        sc[0] += sc[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[n][e] = fmaf(sc[0][e], a.c, sc[0][e] * a.c_lo);
      }
      load_k(next, kb_next);
      if (now.there) {
        if (kb + kF32Keys > lim_min || kb < r.lo) {
          uint32_t odd = 0;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int j = kb + kg * 4 + e;
#pragma unroll
            for (int n = 0; n < kQ; ++n)
              if (j >= lim[n] || j < r.lo) x[n][e] = -INFINITY;
#pragma unroll
            for (int db = 0; db < kBlocks; ++db)
#pragma unroll
              for (int i = 0; i < 4; ++i) odd |= odd_mask(vf[e][db][i]);
          }
          if (__any(odd != 0)) {
            odd_first = min(odd_first, kb), odd_last = kb;
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int db = 0; db < kBlocks; ++db)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                  vf[e][db][i] = __uint_as_float(__float_as_uint(vf[e][db][i]) & ~odd_mask(vf[e][db][i]));
          }
        }
        float p[kQ][4];
#pragma unroll
        for (int n = 0; n < kQ; ++n) {
          float mx = fmaxf(fmaxf(x[n][0], x[n][1]), fmaxf(x[n][2], x[n][3]));
          mx = fmaxf(mx, __shfl_xor(mx, 16));
          mx = fmaxf(mx, __shfl_xor(mx, 32));
          if (__any(mx > m[n])) {
            const float m_new = fmaxf(m[n], mx), alpha = __builtin_amdgcn_exp2f(m[n] - m_new);
            l[n] *= alpha;
#pragma unroll
            for (int db = 0; db < kBlocks; ++db)
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[n][db][e] *= alpha;
            m[n] = m_new;
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            p[n][e] = __builtin_amdgcn_exp2f(x[n][e] - m[n]);
            l[n] += p[n][e];
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int db = 0; db < kBlocks; ++db)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int n = 0; n < kQ; ++n)
                acc[n][db][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[e][db][i], p[n][e], acc[n][db][i], 0, 0, 0);
      }
      load_v(next, kb_next);
      now = next;
      kb = kb_next;
    } while (kb < end);
#pragma unroll 1
    for (kb = odd_first; kb <= odd_last; kb += kW * kF32Keys) {
      const Place t = place(kb);
      if (!t.there || !(kb + kF32Keys > lim_min || kb < r.lo)) continue;
      for (int j = max(kb, r.lo); j < min(kb + kF32Keys, r.n_keys); ++j)
#pragma unroll
        for (int db = 0; db < kBlocks; ++db)
#pragma unroll
          for (int i = 0; i < 4; ++i) {   // this lane's dims 64 db + 16 kg + 4 i + e are rows 4 kg + i of block (db, e)
            const f32x4 v = load_16B(Vh + row_at(t, j) + db * 64 + kg * 16 + i * 4);
#pragma unroll
            for (int n = 0; n < kQ; ++n)
              if (j < lim[n]) {
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[n][db][e][i] += __uint_as_float(__float_as_uint(v[e]) & odd_mask(v[e]));
              }
          }
    }
  }

  if constexpr (kQ > 1) __syncthreads();   // the queries have been read by all
#pragma unroll
  for (int n = 0; n < kQ; ++n) {
    l[n] += __shfl_xor(l[n], 16);
    l[n] += __shfl_xor(l[n], 32);
    float* o = o_lds + ((wave * kQ + n) * 16 + r16) * D + kg * 16;
#pragma unroll
    for (int db = 0; db < kBlocks; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4*>(o + db * 64 + i * 4) = f32x4{acc[n][db][0][i], acc[n][db][1][i], acc[n][db][2][i], acc[n][db][3][i]};
    if (kg == 0) ml_lds[(wave * kQ + n) * 16 + r16] = make_float2(m[n], l[n]);
  }
  __syncthreads();
  constexpr int kThreads = D / 4, kPass = kW * 64 / kThreads;   // threads of a row, four dims each; rows at a time
  const int c = threadIdx.x % kThreads;
#pragma unroll
  for (int pass = 0; pass * kPass < kRows; ++pass) {
    const int row = pass * kPass + threadIdx.x / kThreads, rho = r.tile * kRows + row;
    if (row >= kRows || rho >= n_set) return;
    float M = kNothing, L = 0.f;
#pragma unroll
    for (int w = 0; w < kW; ++w) M = fmaxf(M, ml_lds[w * kRows + row].x);
    f32x4 out = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kW; ++w) {
      const float2 ml = ml_lds[w * kRows + row];
      const float by = __builtin_amdgcn_exp2f(ml.x - M);
      L += by * ml.y;
      out += by * *reinterpret_cast<const f32x4*>(o_lds + (w * kRows + row) * D + c * 4);
    }
    if (a.part_o != nullptr) {
      const int64_t at = static_cast<int64_t>(r.slot) * a.slot_rows + row;
      *reinterpret_cast<f32x4*>(a.part_o + at * D + c * 4) = out;
      if (c == 0) a.part_ml[at] = make_float2(M, L);
      continue;
    }
    const int tok = a.by_rep.of(rho), head = r.kvh * a.rep + rho - tok * a.rep;
    const int64_t t = r.t0 + tok;
    const bool none = sees_none(a, r, limit_of(a, r, tok), L);
    if (none) out = f32x4{0.f, 0.f, 0.f, 0.f};
    else out *= 1.f / L;
    *reinterpret_cast<f32x4*>(static_cast<float*>(a.O) + head * a.o_stride + t * D + c * 4) = out;
    if (a.lse != nullptr && c == 0) a.lse[head * static_cast<int64_t>(a.T) + t] = none ? -INFINITY : lse_of(M, L);
  }
}

template <int D, bool kPages, int kQ, int kW>
__global__ __launch_bounds__(kW * 64, 2) void rows_f32_kernel(RowsArgs a) {
  extern __shared__ __align__(16) float smem_f32[];
  constexpr size_t kAt = kF32Smem<D, kQ, kW> / sizeof(float);
  each_unit<16 * kQ, kPages>(a, (lds_int*)(smem_f32 + kAt), [&](const RowSet& r) { rows_f32<D, kPages, kQ, kW>(a, r, smem_f32); });
}

}  // namespace pc
