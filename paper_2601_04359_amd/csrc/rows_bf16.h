// The bf16 forms of the attention on several sequences (gfx950 only), on the 32x32x16 bf16 MFMA: one for D = 64 and 128, two for
// 128.
//
// Scores are formed transposed, S^T = K Q^T: a lane holds ONE query (column l % 32) and 16 of 32 keys (with g = l / 32, keys
// 8 i + 4 g .. + 3, i = 0 .. 3), so that a row's limit, reference and sum are per-lane numbers and the probabilities are
// the B operand of O^T += V^T P^T as they stand.  What a row does not see gets the score -inf, in the tiles where a row
// of the work-group does not see everything; a tile of keys lies in one page.
//
// Probabilities are rounded to bf16 for the second product, which the bf16 instructions take, and the normaliser sums them as they
// were: half a step per weight, in directions of their own, against the half step that O is rounded by anyway.  Against 64 bits the
// timed cases are off by 0.0008 to 0.0024 of O's norm, and with 32-bit probabilities by 0.0007 to 0.0017.
#pragma once

#include <limits.h>

#include <type_traits>

#include "attn_phase.h"
#include "seq_rows.h"

namespace pc {

typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef __attribute__((address_space(3))) u32x2 lds_u32x2;

// The sign bits of those halves of a dword that are bf16 numbers which are not finite: an exponent of ones carries into the
// sign.  By whole dwords, so that no comparison takes a pair of scalar registers of its own.
__device__ __forceinline__ uint32_t odd_halves(uint32_t w) { return ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u; }
__device__ __forceinline__ uint32_t odd_bf16(u32x4 v) { return odd_halves(v[0]) | odd_halves(v[1]) | odd_halves(v[2]) | odd_halves(v[3]); }
__device__ __forceinline__ u32x4 finite_bf16(u32x4 v) {   // those as zeros
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] &= ~((odd_halves(v[i]) >> 15) * 0xFFFFu);
  return v;
}
// Those of a row of V added to a lane's output, behind its last key: an infinity that went in earlier would meet the rescaling of
// what it stands in, and 0 times it is no number.  dims 32 db + 8 a + 4 g .. + 3 are accumulators 4 a .. of block db.
template <int kBlocks>
__device__ __forceinline__ void add_odd(f32x16 (&o)[kBlocks], const uint16_t* v, int g) {
#pragma unroll
  for (int db = 0; db < kBlocks; ++db)
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      const u32x2 w = *reinterpret_cast<const u32x2*>(v + db * 32 + a * 8 + g * 4);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t odd = w[e] & (odd_halves(w[e]) >> 15) * 0xFFFFu;
        o[db][a * 4 + e * 2] += __uint_as_float(odd << 16);
        o[db][a * 4 + e * 2 + 1] += __uint_as_float(odd & 0xFFFF0000u);
      }
    }
}
// Scores of keys `from` .. `upto` - 1, counted from a lane's first, stay; the others become -inf.
__device__ __forceinline__ int keys_below(int n) {   // the accumulators of keys below n
  int bits = 0;
#pragma unroll
  for (int q = 0; q < 4; ++q) bits |= ((1 << min(max(n - 8 * q, 0), 4)) - 1) << (4 * q);
  return bits;
}
__device__ __forceinline__ void hide(f32x16& sc, int from, int upto) {
  const int seen = keys_below(upto) & ~keys_below(from);
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const uint32_t keep = static_cast<uint32_t>(__builtin_amdgcn_sbfe(seen, i, 1));
    sc[i] = __uint_as_float((__float_as_uint(sc[i]) & keep) | (0xFF800000u & ~keep));
  }
}

// A pointer that is the same in every lane, in scalar registers (with page numbers in it, the compiler does not always see
// that it is).
template <bool kPages>
__device__ __forceinline__ const uint16_t* uniform(const uint16_t* p) {
  if constexpr (!kPages) return p;
  const uint64_t v = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v)), hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v >> 32));
  return reinterpret_cast<const uint16_t*>(static_cast<uint64_t>(hi) << 32 | lo);
}

// Where a work-group's keys lie.  The page of a tile (its number, -1: none) comes from the lanes' registers, 64 tiles at a
// time.
template <bool kPages, int kTile, int D = kD>
struct KeyTiles {
  const RowsArgs& a;
  const RowSet& r;
  const uint16_t *Kh, *Vh;
  int stride;      // tiles from one of this wave's to its next, and the first of them: key begin + (first + i * stride) kTile
  int first, ids, lane;
  __device__ __forceinline__ KeyTiles(const RowsArgs& args, const RowSet& set, int first_tile, int tile_stride, int l)
      : a(args), r(set), Kh(static_cast<const uint16_t*>(args.K) + set.kvh * args.k_stride),
        Vh(static_cast<const uint16_t*>(args.V) + set.kvh * args.v_stride), stride(tile_stride), first(first_tile), ids(-1), lane(l) {}
  __device__ __forceinline__ int key_of(int i) const { return r.begin + (first + i * stride) * kTile; }
  __device__ __forceinline__ void fetch(int i0, int end) {   // the pages of tiles i0 .. i0 + 63
    if constexpr (kPages) {
      const int k = key_of(i0 + lane);
      ids = -1;
      if (k < end) ids = r.pages[a.by_page.of(k)];
      if (ids >= a.n_pages || k + kTile <= r.lo) ids = -1;   // no page, or no row of it is asked for
    }
  }
  __device__ __forceinline__ int page(int i) const { return kPages ? __builtin_amdgcn_readlane(ids, i & 63) : 0; }
  // row `key` of the cache, in elements from Kh or Vh on
  __device__ __forceinline__ int64_t at(int key, int pg) const {
    if constexpr (kPages) return pg * a.page_stride + static_cast<int64_t>(key - a.by_page.of(key) * a.by_page.d) * D;
    return static_cast<int64_t>(r.k0 + key) * D;
  }
  // Values that are not finite of keys from .. from + 31 of the tile that begins with key0 are added to the rows that see them, if
  // some row does not (see all_below): they have been taken out of the tile.
  template <int kBlocks>
  __device__ __forceinline__ void add_odd_rows(f32x16 (&o)[kBlocks], int key0, int from, int all_below, int lim, int g) const {
    if (key0 + kTile <= all_below && key0 >= r.lo) return;
    const int pg = kPages ? r.pages[a.by_page.of(key0)] : 0;
    if (kPages && (pg < 0 || pg >= a.n_pages)) return;
    const uint16_t* rows = Vh + at(key0, pg);
    for (int k = max(from, r.lo); k < min(from + 32, r.n_keys); ++k)
      if (k < lim) add_odd(o, rows + static_cast<int64_t>(k - key0) * D, g);
  }
  // byte offset of chunk `chunk` of row key0 + row of a tile that begins with key0: rows that do not exist are read as the
  // nearest that does
  __device__ __forceinline__ uint32_t offset(int key0, int row, int chunk) const {
    return (min(max(key0 + row, r.lo), r.n_keys - 1) - key0) * (2 * D) + chunk * 16;
  }
};

// The end of a work-group whose waves share rows: wave w has (O, m, l) of rows 32 (w % kR) .. + 31 of the tile over its part of
// the keys.  Piece i of a wave's O = accumulators 4 i .. + 3 of every lane = dims 8 i + 4 g .. + 3 of its row, lanes permuted by
// i so that the reads use every bank; a thread adds up eight dims of a row, in the order of the waves, and rows leave whole.
template <int D>
constexpr int kWaveOBytes = 32 * D * 4;
template <int D, int kR, int kG>
__device__ __forceinline__ void merge_waves(const RowsArgs& a, const RowSet& r, lds_u8* smem, const f32x16 (&o)[D / 32], float m, float l,
                                            int wave, int lane) {
  constexpr int kWaves = kR * kG;
  auto piece = [&](int w, int i, int of_lane) {
    return reinterpret_cast<lds_f32x4*>(smem + w * kWaveOBytes<D> + i * 1024 + (of_lane ^ i) * 16);
  };
  auto* s_ml = reinterpret_cast<__attribute__((address_space(3))) float*>(smem + kWaves * kWaveOBytes<D>);
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *piece(wave, db * 4 + q, lane) = f32x4{o[db][q * 4], o[db][q * 4 + 1], o[db][q * 4 + 2], o[db][q * 4 + 3]};
  if (lane < 32) {
    s_ml[(wave * 32 + lane) * 2] = m;
    s_ml[(wave * 32 + lane) * 2 + 1] = l;
  }
  __syncthreads();
  constexpr int kThreads = D / 8, kPass = kWaves * 64 / kThreads;   // threads of a row, rows at a time
  const int i = threadIdx.x % kThreads, n_set = r.n_tok * a.rep;
#pragma unroll
  for (int pass = 0; pass * kPass < 32 * kR; ++pass) {
    const int in_tile = pass * kPass + threadIdx.x / kThreads, rg = in_tile >> 5, row = in_tile & 31;
    const int rho = r.tile * 32 * kR + in_tile;
    if (in_tile >= 32 * kR || rho >= n_set) return;
    float mw[kG], M = kNothing, L = 0.f;
#pragma unroll
    for (int w = 0; w < kG; ++w) {
      mw[w] = s_ml[((w * kR + rg) * 32 + row) * 2];
      M = fmaxf(M, mw[w]);
    }
    f32x4 acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int w = 0; w < kG; ++w) {
      const float by = __builtin_amdgcn_exp2f(mw[w] - M);
      L += by * s_ml[((w * kR + rg) * 32 + row) * 2 + 1];
#pragma unroll
      for (int t = 0; t < 2; ++t) acc[t] += by * *piece(w * kR + rg, i, t * 32 + row);
    }
    const int tok = a.by_rep.of(rho), head = r.kvh * a.rep + rho - tok * a.rep;
    const int64_t t = r.t0 + tok;
    if (a.part_o != nullptr) {
      const int64_t at = static_cast<int64_t>(r.slot) * a.slot_rows + in_tile;
#pragma unroll
      for (int h = 0; h < 2; ++h) *reinterpret_cast<f32x4*>(a.part_o + at * D + i * 8 + h * 4) = acc[h];
      if (i == 0) a.part_ml[at] = make_float2(M, L);
      continue;
    }
    const bool none = sees_none(a, r, limit_of(a, r, tok), L);
    const float inv = none ? 0.f : 1.f / L;
    u32x4 out = {0u, 0u, 0u, 0u};
    if (!none) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        out[h * 2] = pack_bf16x2(acc[h][0] * inv, acc[h][1] * inv);
        out[h * 2 + 1] = pack_bf16x2(acc[h][2] * inv, acc[h][3] * inv);
      }
    }
    *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(a.O) + head * a.o_stride + t * D + i * 8) = out;
    if (a.lse != nullptr && i == 0) a.lse[head * static_cast<int64_t>(a.T) + t] = none ? -INFINITY : lse_of(M, L);
  }
}

// ------------------------------------------------------------------------------------------
// Few rows: 32 query rows per work-group.  The eight waves take the keys in steps of 32 by turns, each through LDS of its
// own, so that the loop has no barrier (a step's fragments go to registers at once, the next step is fetched behind them);
// (O, m, l) of the waves are merged through LDS once.  Bound: the bytes of K and V, or latency.  Measured, D = 128: a token behind
// each of 16 sequences of 1 to 29,512 rows, 24/8 heads, 125 us with the join (649 MB, 5.2 TB/s); a prompt of 40 rows, 8/2 heads, 5.6 us.
// ------------------------------------------------------------------------------------------
constexpr int kFewRows = 32, kFewKeys = 32, kFewWaves = 8;
template <int D>
constexpr size_t kFewSmem = kFewWaves * (kWaveOBytes<D> + 32 * 8) + kFewRows * D * 2;

template <int D, bool kPages>
__device__ __forceinline__ void rows_few(const RowsArgs& a, const RowSet& r, lds_u8* smem) {
  constexpr int kRow = 2 * D, kTileBytes = kFewKeys * kRow;   // a row in LDS, a step's K or V
  constexpr int kChunks = kRow / 16, kRows = 64 / kChunks;    // 16-byte chunks of a row, rows of a load of 1 KB
  constexpr int kSteps = D / 16, kBlocks = D / 32;
  static_assert(2 * kTileBytes <= kWaveOBytes<D>, "a wave's K and V lie where its O goes");
  // Where chunk c of row r lies.  Rows of 128 bytes: two rows make 256 bytes, and what a quarter wave reads (one chunk of 16
  // rows of K, two chunks of four rows of V) uses every bank there too.
  auto k_pos = [](int row, int chunk) { return D == 128 ? k_chunk_pos(row, chunk) : chunk ^ ((row >> 1) & 7); };
  auto v_pos = [](int row, int chunk) { return D == 128 ? v_chunk_pos(row, chunk) : chunk ^ (((row >> 1) & 3) << 1); };
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l32 = lane & 31, g = lane >> 5;
  const int n_set = r.n_tok * a.rep;
  const lds_u8* lds = smem + wave * kWaveOBytes<D>;
  const uint32_t lds_w = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(lds));
  const lds_u8* q_tile = smem + kFewWaves * (kWaveOBytes<D> + 32 * 8);
  KeyTiles<kPages, kFewKeys, D> keys(a, r, wave, kFewWaves, lane);
  keys.fetch(0, r.end);

  if (wave * kRows < kFewRows) {   // four query rows per wave (D = 64: eight of each of the first four waves)
    const int row = wave * kRows + lane / kChunks, rho = min(r.tile * kFewRows + row, n_set - 1);
    const int tok = a.by_rep.of(rho), head = r.kvh * a.rep + rho - tok * a.rep;
    dma_16B(static_cast<const uint16_t*>(a.Q) + head * a.q_stride + static_cast<int64_t>(r.t0 + tok) * D + k_pos(row, lane % kChunks) * 8,
            static_cast<uint32_t>(reinterpret_cast<uintptr_t>(q_tile)) + wave * 1024);
  }
  auto stage = [&](int i) {   // step i of this wave: 32 rows of K and of V; false: they are nobody's
    const int pg = keys.page(i);
    if (pg < 0) return false;
    const int k0 = keys.key_of(i);
    const int64_t at = keys.at(k0, pg);
    const uint16_t *kb = keys.Kh + at, *vb = keys.Vh + at;
#pragma unroll
    for (int p = 0; p < kFewKeys / kRows; ++p) {
      const int row = p * kRows + lane / kChunks, pos = lane % kChunks;
      dma_16B_at(kb, keys.offset(k0, row, k_pos(row, pos)), __builtin_amdgcn_readfirstlane(lds_w + p * 1024));
      dma_16B_at(vb, keys.offset(k0, row, v_pos(row, pos)), __builtin_amdgcn_readfirstlane(lds_w + kTileBytes + p * 1024));
    }
    return true;
  };
  // the first step goes out before the rows' limits are known; it may turn out to be needed by none
  bool there = keys.key_of(0) < r.end && stage(0);

  const int tok = a.by_rep.of(min(r.tile * kFewRows + l32, n_set - 1));
  const int lim = limit_of(a, r, tok);
  int lim_max = lim, lim_min = lim > 0 ? lim : INT_MAX;   // over the rows that see something
#pragma unroll
  for (int x = 1; x < 32; x *= 2) {
    lim_max = max(lim_max, __shfl_xor(lim_max, x));
    lim_min = min(lim_min, __shfl_xor(lim_min, x));
  }
  const int end = min(r.end, __builtin_amdgcn_readfirstlane(lim_max));
  lim_min = __builtin_amdgcn_readfirstlane(lim_min);

  int k_off[kSteps], v_off[kBlocks];
#pragma unroll
  for (int s = 0; s < kSteps; ++s) k_off[s] = l32 * kRow + k_pos(l32, 2 * s + g) * 16;
  {
    const int r16 = lane & 15, G = (lane >> 4) & 1, row = g * 4 + (r16 >> 2);
#pragma unroll
    for (int db = 0; db < kBlocks; ++db) {
      const int dim = db * 32 + G * 16 + 4 * (r16 & 3);
      v_off[db] = kTileBytes + row * kRow + v_pos(row, dim >> 3) * 16 + (dim & 7) * 2;
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  bf16x8 qf[kSteps];
#pragma unroll
  for (int s = 0; s < kSteps; ++s) qf[s] = lds_frag(q_tile + k_off[s]);

  f32x16 o[kBlocks];
#pragma unroll
  for (int db = 0; db < kBlocks; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
  float m = kNothing, l = 0.f;
  int odd_first = INT_MAX, odd_last = -1;   // steps with values that are not finite and not seen by all
  for (int i = 0;; ++i) {
    const int k0 = keys.key_of(i);
    if (k0 >= end) break;
    const bool now = there;
    // This step's rows have landed (they are all that is in flight): every fragment goes to registers, so that the next
    // step's rows can be fetched into the same LDS at once.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    bf16x8 kf[kSteps], vf[2][kBlocks];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) kf[s] = lds_frag(lds + k_off[s]);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int db = 0; db < kBlocks; ++db) {
        const lds_u8* src = lds + v_off[db] + ks * 16 * kRow;
        const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
            reinterpret_cast<__attribute__((address_space(3))) bf16x4*>(const_cast<lds_u8*>(src)));
        const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
            reinterpret_cast<__attribute__((address_space(3))) bf16x4*>(const_cast<lds_u8*>(src + 8 * kRow)));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          vf[ks][db][e] = lo[e];
          vf[ks][db][4 + e] = hi[e];
        }
      }
#pragma unroll
    for (int s = 0; s < kSteps; ++s) asm volatile("" : "+v"(kf[s]));
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int db = 0; db < kBlocks; ++db) asm volatile("" : "+v"(vf[ks][db]));
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (kPages && (i & 63) == 63) keys.fetch(i + 1, r.end);
    there = keys.key_of(i + 1) < end && stage(i + 1);
    if (!now) continue;

    f32x16 sc;
#pragma unroll
    for (int e = 0; e < 16; ++e) sc[e] = 0.f;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[s], qf[s], sc, 0, 0, 0);
    if (k0 + kFewKeys > lim_min || k0 < r.lo) {
      hide(sc, r.lo - k0 - g * 4, lim - k0 - g * 4);
      uint32_t odd = 0;   // 0 times what is not finite would reach rows that do not see it
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int db = 0; db < kBlocks; ++db) odd |= odd_bf16(__builtin_bit_cast(u32x4, vf[ks][db]));
      if (__any(odd != 0)) {
        odd_first = min(odd_first, i), odd_last = i;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
          for (int db = 0; db < kBlocks; ++db) vf[ks][db] = __builtin_bit_cast(bf16x8, finite_bf16(__builtin_bit_cast(u32x4, vf[ks][db])));
      }
    }
    float mx = sc[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) mx = fmaxf(mx, sc[e]);
    mx = wave_half_max(mx) * a.c;
    float ref = m;
    if (__any(!(mx <= m + 8.f) || far_ref(m))) {     // the reference lags by at most 2^8
      const float m_new = fmaxf(m, mx), alpha = __builtin_amdgcn_exp2f(m - m_new);
      l *= alpha;
#pragma unroll
      for (int db = 0; db < kBlocks; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[db][e] *= alpha;
      ref = m = m_new;
      if (far_ref(m)) {      // its exponents come to the common fma as products of c, with 0 as their reference
        const float by = 1.f / a.c;
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[e] = far_exponent(sc[e], a.c, m) * by;
        ref = 0.f;
      }
    }
    bf16x8 p[2];
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float x = __builtin_amdgcn_exp2f(fmaf(sc[e], a.c, -ref));
      sum += x;
      p[e >> 3][e & 7] = static_cast<__bf16>(x);
    }
    l += sum;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int db = 0; db < kBlocks; ++db) o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[ks][db], p[ks], o[db], 0, 0, 0);
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");   // a first step that was needed by none may be in flight
  l = wave_half_sum(l);
  for (int i = odd_first; i <= odd_last; ++i) keys.add_odd_rows(o, keys.key_of(i), keys.key_of(i), lim_min, lim, g);

  merge_waves<D, 1, kFewWaves>(a, r, smem, o, m, l, wave, lane);
}

// ------------------------------------------------------------------------------------------
// Many rows: 128 query rows per work-group, 32 for each of four waves, two work-groups per compute unit.  Keys in tiles of
// 64, two of K and two of V in LDS (64 KB), processed as halves A and B of 32 keys; every wave runs
//     phase 1 of tile j:  S_B(j), O += V_B(j-1) P_B(j-1)  |  P_A(j)
//     phase 2 of tile j:  S_A(j+1), O += V_A(j) P_A(j)    |  P_B(j)
// (pipeline_phase).  One barrier per tile, after phase 1: behind it K(j+2) and V(j+1) are fetched into the slots just
// released.  Bound: the matrix pipe, which the other work-group of the unit keeps busy while one waits at its barrier.  Measured:
// a prompt of 16,384 rows, 24/8 heads, 1,503 to 1,591 us on several cards (1,036 to 1,097 TFLOP/s, 0.84 to 0.89 of a large product's rate).
// Eight waves with 128 or 256 rows were slower on causal prompts.
// ------------------------------------------------------------------------------------------
constexpr int kManyWaves = 4, kManyRows = 32 * kManyWaves, kManyKeys = 64;
constexpr int kManyTileBytes = kManyKeys * kRowBytes;
constexpr size_t kManySmem = 4 * kManyTileBytes + kManyWaves * 8;   // tiles, the waves' limits

template <bool kUnitC, bool kPages>
__device__ __forceinline__ void rows_many(const RowsArgs& a, const RowSet& r, lds_u8* smem) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t lds_mine = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(smem)) + wave * 4096;
  const int l32 = lane & 31, g = lane >> 5;
  const int n_set = r.n_tok * a.rep, row_first = r.tile * kManyRows + wave * 32;
  const bool active = row_first < n_set;   // wave-uniform
  const int rho = min(row_first + l32, n_set - 1);
  const int tok = a.by_rep.of(rho), head = r.kvh * a.rep + rho - tok * a.rep;

  KeyTiles<kPages, kManyKeys> keys(a, r, 0, 1, lane);
  auto k_slot = [](int t) { return (t & 1) * kManyTileBytes; };
  auto v_slot = [](int t) { return (2 + (t & 1)) * kManyTileBytes; };
  // a wave's 16 rows of a tile; rows that are nobody's are zeros
  auto stage = [&](auto is_v, int j, int pg, int slot) {
    if (pg < 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        reinterpret_cast<lds_u32x4*>(smem + slot + (wave * 4 + i) * 1024)[lane] = u32x4{0u, 0u, 0u, 0u};
      return;
    }
    const int k0 = keys.key_of(j);
    const uint16_t* base = (decltype(is_v)::value ? keys.Vh : keys.Kh) + keys.at(k0, pg);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = (wave * 4 + i) * 4 + (lane >> 4), pos = lane & 15;
      dma_16B_at(base, keys.offset(k0, row, decltype(is_v)::value ? v_chunk_pos(row, pos) : k_chunk_pos(row, pos)),
                 lds_mine + slot + i * 1024);
    }
  };
  keys.fetch(0, r.end);
  int pg = keys.page(0), pg_next = keys.page(1);   // pages of tiles j and j + 1
  if (r.begin < r.end) {   // the first tiles go out before it is known how many there are
    stage(std::false_type{}, 0, pg, k_slot(0));
    stage(std::true_type{}, 0, pg, v_slot(0));
    if (keys.key_of(1) < r.end) stage(std::false_type{}, 1, pg_next, k_slot(1));
  }
  // the slot of V(-1) is read once against zero probabilities: clear it
#pragma unroll
  for (int i = 0; i < 4; ++i) reinterpret_cast<lds_u32x4*>(smem + v_slot(1) + (wave * 4 + i) * 1024)[lane] = u32x4{0u, 0u, 0u, 0u};

  // the wave's queries, as fragments
  bf16x8 qf[8];
  {
    const uint16_t* q = static_cast<const uint16_t*>(a.Q) + head * a.q_stride + static_cast<int64_t>(r.t0 + tok) * kD + g * 8;
#pragma unroll
    for (int s = 0; s < 8; ++s) qf[s] = *reinterpret_cast<const bf16x8*>(q + s * 16);
  }
  // What the rows see.  One that sees none of these keys takes part as if it saw all, and its result is thrown away.
  const int lim_true = limit_of(a, r, tok);
  const bool sees = lim_true > max(r.lo, r.begin);
  const int lim = sees ? lim_true : INT_MAX;
  int lim_max = sees ? lim_true : 0, lim_min = lim;
#pragma unroll
  for (int x = 1; x < 32; x *= 2) {
    lim_max = max(lim_max, __shfl_xor(lim_max, x));
    lim_min = min(lim_min, __shfl_xor(lim_min, x));
  }
  lim_min = __builtin_amdgcn_readfirstlane(lim_min);   // of the wave
  auto* s_lim = reinterpret_cast<__attribute__((address_space(3))) int*>(smem + 4 * kManyTileBytes);   // behind the tiles
  if (lane == 0) s_lim[wave * 2] = active ? lim_max : 0, s_lim[wave * 2 + 1] = active ? lim_min : INT_MAX;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();   // K(0), V(0), K(1) and the limits
  int all_max = 0, all_min = INT_MAX;                  // of the work-group
#pragma unroll
  for (int w = 0; w < kManyWaves; ++w) all_max = max(all_max, s_lim[w * 2]), all_min = min(all_min, s_lim[w * 2 + 1]);
  all_max = __builtin_amdgcn_readfirstlane(all_max), all_min = __builtin_amdgcn_readfirstlane(all_min);
  const int end = min(r.end, all_max), n = (end - r.begin + kManyKeys - 1) / kManyKeys;

  int k_off[8], v_off[4];
#pragma unroll
  for (int s = 0; s < 8; ++s) k_off[s] = l32 * kRowBytes + k_chunk_pos(l32, 2 * s + g) * 16;
  {
    const int r16 = lane & 15, G = (lane >> 4) & 1, row = g * 4 + (r16 >> 2);
#pragma unroll
    for (int db = 0; db < 4; ++db) {
      const int dim = db * 32 + G * 16 + 4 * (r16 & 3);
      v_off[db] = row * kRowBytes + v_chunk_pos(row, dim >> 3) * 16 + (dim & 7) * 2;
    }
  }
  f32x16 o[4], sA, sB, neg_m;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
#pragma unroll
    for (int db = 0; db < 4; ++db) o[db][i] = 0.f;
    sA[i] = sB[i] = neg_m[i] = 0.f;
  }
  bf16x8 pA[2], pB[2];
#pragma unroll
  for (int ks = 0; ks < 2; ++ks)
#pragma unroll
    for (int e = 0; e < 8; ++e) pA[ks][e] = pB[ks][e] = static_cast<__bf16>(0.f);
  float m_ref = -INFINITY, l_run = 0.f;
  bool redo_all = false;   // wave-uniform
  int odd_first = INT_MAX, odd_last = -1;   // tiles with values that are not finite and not seen by all

  // hides what a row does not see of the 32 keys from key0 on; `there`: they have a page
  auto mask = [&](f32x16& sc, int key0, bool there) {
    if (key0 + 32 <= lim_min && key0 >= r.lo && there) return;
    hide(sc, r.lo - key0 - g * 4, there ? lim - key0 - g * 4 : 0);
  };
  if (n > 0) {
    if (active) {  // S_A of tile 0 and the first reference
      f32x16 zero;
#pragma unroll
      for (int i = 0; i < 16; ++i) zero[i] = 0.f;
#pragma unroll
      for (int s = 0; s < 8; ++s)
        sA = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lds_frag(smem + k_slot(0) + k_off[s]), qf[s], s == 0 ? zero : sA, 0, 0, 0);
      mask(sA, r.begin, pg >= 0);
      float mx = sA[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) mx = fmaxf(mx, sA[i]);
      m_ref = wave_half_max(mx) * a.c;
      if constexpr (!kUnitC) redo_all = __any(far_ref(m_ref));
      if constexpr (kUnitC) {
        const float start = m_ref >= kLowestStart ? m_ref : 0.f;
        redo_all = __any(!(m_ref >= kLowestStart));
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          sA[i] -= start;
          neg_m[i] = -start;
        }
      }
    }
    auto tile = [&](int j, auto parity) {
      constexpr int u = decltype(parity)::value;
      constexpr int k_cur = u * kManyTileBytes, k_nxt = (u ^ 1) * kManyTileBytes;
      constexpr int v_cur = (2 + u) * kManyTileBytes, v_prev = (2 + (u ^ 1)) * kManyTileBytes;
      const int key0 = r.begin + j * kManyKeys;
      if (active) {
        pipeline_phase<kUnitC>(smem + k_cur + 32 * kRowBytes, k_off, smem + v_prev + 32 * kRowBytes, v_off, qf, sB, pB, o, sA, pA, m_ref,
                               l_run, a.c, neg_m, redo_all);
        mask(sB, key0 + 32, pg >= 0);
      }
      // every wave is past K(j) and V(j-1); K(j+1) and V(j) have landed
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      if (kPages && ((j + 2) & 63) == 0) keys.fetch(j + 2, r.end);
      const int pg_after = keys.page(j + 2);
      if (j + 2 < n) stage(std::false_type{}, j + 2, pg_after, k_cur);
      if (j + 1 < n) stage(std::true_type{}, j + 1, pg_next, v_prev);
      if (key0 + kManyKeys > all_min || key0 < r.lo) {
        // Some row does not see all of this tile, and 0 times what is not finite would reach it: such values are taken out of
        // the tile and added to the rows that see them in the end.
        lds_u32x4* mine = reinterpret_cast<lds_u32x4*>(smem + v_cur) + threadIdx.x * 4;
        uint32_t odd = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) odd |= odd_bf16(mine[i]);
        if (__syncthreads_or(odd != 0)) {
          odd_first = min(odd_first, j), odd_last = j;
#pragma unroll
          for (int i = 0; i < 4; ++i) mine[i] = finite_bf16(mine[i]);
          __syncthreads();
        }
      }
      if (active) {
        pipeline_phase<kUnitC>(smem + k_nxt, k_off, smem + v_cur, v_off, qf, sA, pA, o, sB, pB, m_ref, l_run, a.c, neg_m, redo_all);
        mask(sA, key0 + kManyKeys, pg_next >= 0);
      }
      pg = pg_next, pg_next = pg_after;
    };
    for (int j = 0; j < n; j += 2) {
      tile(j, std::integral_constant<int, 0>{});
      if (j + 1 >= n) break;
      tile(j + 1, std::integral_constant<int, 1>{});
    }
    if (active) {  // O += V_B(n-1) P_B(n-1)
      const lds_u8* v_half = smem + v_slot(n - 1) + 32 * kRowBytes;
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int db = 0; db < 4; ++db) {
          const lds_u8* p = v_half + v_off[db] + ks * 16 * kRowBytes;
          const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
              reinterpret_cast<__attribute__((address_space(3))) bf16x4*>(const_cast<lds_u8*>(p)));
          const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
              reinterpret_cast<__attribute__((address_space(3))) bf16x4*>(const_cast<lds_u8*>(p + 8 * kRowBytes)));
          bf16x8 vf;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            vf[e] = lo[e];
            vf[4 + e] = hi[e];
          }
          o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pB[ks], o[db], 0, 0, 0);
        }
      for (int j = odd_first; j <= odd_last; ++j)
#pragma unroll 1
        for (int half = 0; half < 64; half += 32) keys.add_odd_rows(o, keys.key_of(j), keys.key_of(j) + half, all_min, lim, g);
    }
  }
  const float l_tot = wave_half_sum(l_run);
  __syncthreads();   // every wave has read its last tile; LDS takes the rows
  if (!active) return;
  const int rows_w = min(32, n_set - row_first);
  lds_u8* mine = smem + wave * kManyTileBytes;
  auto row_to = [&](int row, int* h) {   // token of a row of the wave, and its head
    const int rh = row_first + row, tk = a.by_rep.of(rh);
    *h = r.kvh * a.rep + rh - tk * a.rep;
    return static_cast<int64_t>(r.t0 + tk);
  };
  if (a.part_o != nullptr) {   // un-normalised, as fp32 rows
    const int64_t first = static_cast<int64_t>(r.slot) * a.slot_rows + wave * 32;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        f32x4 v = {o[db][q * 4], o[db][q * 4 + 1], o[db][q * 4 + 2], o[db][q * 4 + 3]};
        if (!sees) v = f32x4{0.f, 0.f, 0.f, 0.f};
        *reinterpret_cast<lds_f32x4*>(mine + l32 * 512 + ((db * 8 + q * 2 + g) ^ l32) * 16) = v;
      }
    wave_lds_sync();
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int row = i * 2 + g;
      const f32x4 v = *reinterpret_cast<const lds_f32x4*>(mine + row * 512 + l32 * 16);
      if (row < rows_w) *reinterpret_cast<f32x4*>(a.part_o + (first + row) * kD + (l32 ^ row) * 4) = v;
    }
    if (g == 0 && l32 < rows_w) a.part_ml[first + l32] = sees ? make_float2(fmaxf(m_ref, kNothing), l_tot) : make_float2(kNothing, 0.f);
    return;
  }
  const bool none = !sees || sees_none(a, r, lim, l_tot);
  const float inv = none ? 0.f : 1.f / l_tot;
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      u32x2 out = {pack_bf16x2(o[db][q * 4 + 0] * inv, o[db][q * 4 + 1] * inv), pack_bf16x2(o[db][q * 4 + 2] * inv, o[db][q * 4 + 3] * inv)};
      if (none) out = u32x2{0u, 0u};
      *reinterpret_cast<lds_u32x2*>(mine + l32 * kRowBytes + k_chunk_pos(l32, db * 4 + q) * 16 + g * 8) = out;
    }
  wave_lds_sync();
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int row = i * 4 + (lane >> 4), chunk = k_chunk_pos(row, lane & 15);
    const u32x4 v = *reinterpret_cast<const lds_u32x4*>(mine + row * kRowBytes + (lane & 15) * 16);
    int h;
    const int64_t t = row_to(min(row, rows_w - 1), &h);
    if (row < rows_w) *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(a.O) + h * a.o_stride + t * kD + chunk * 8) = v;
  }
  if (a.lse != nullptr && g == 0 && l32 < rows_w) a.lse[head * static_cast<int64_t>(a.T) + r.t0 + tok] = none ? -INFINITY : lse_of(m_ref, l_tot);
}

// ------------------------------------------------------------------------------------------
// Between the two: 64 query rows per work-group, a wave for each pair of one of two row groups and one of two key groups, two
// work-groups per compute unit; the keys are dealt to the key groups in tiles of 32, and the groups' (O, m, l) are merged through LDS.
//     phase j:  S(j+1), O += V(j-1) P(j-1)  |  P(j)
// One barrier behind it; then K(j+3) and V(j+1) are fetched into the slots just released.  The longest work-group has half of
// the products that it has with 128 rows, which is what a call of few work-groups waits for; where there are many, K and V
// come through L2 twice as often per product.  Measured: a prompt of 3,000 rows, 16/4 heads, 53 to 57 us (63 with 128 rows).
// ------------------------------------------------------------------------------------------
constexpr int kMidWaves = 4, kMidRows = 64;
constexpr size_t kMidSmem = kMidWaves * (kWaveOBytes<kD> + 32 * 8);

template <bool kUnitC, bool kPages>
__device__ __forceinline__ void rows_mid(const RowsArgs& a, const RowSet& r, lds_u8* smem) {
  constexpr int kR = 2, kG = 2, kS = 2;   // row groups, key groups, slots per operand and key group
  constexpr int kKeys = 32 * kG, kTile = kKeys * kRowBytes;   // of a phase
  static_assert(2 * kS * kTile <= kMidWaves * kWaveOBytes<kD>, "tiles");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l32 = lane & 31, g = lane >> 5, rg = wave % kR, kg = wave / kR;
  const int n_set = r.n_tok * a.rep, row_first = (r.tile * kR + rg) * 32;
  const bool active = row_first < n_set;   // wave-uniform
  const int rho = min(row_first + l32, n_set - 1);
  const int tok = a.by_rep.of(rho), head = r.kvh * a.rep + rho - tok * a.rep;

  const uint32_t lds_mine = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(smem)) + wave * 4096;
  KeyTiles<kPages, kKeys> keys(a, r, 0, 1, lane);
  auto k_slot = [](int t) { return (t & 1) * kTile; };
  auto v_slot = [](int t) { return (kS + (t & 1)) * kTile; };
  // a wave's 16 rows of a tile; rows that are nobody's are zeros
  auto stage = [&](auto is_v, int j, int pg, int slot) {
    if (pg < 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        reinterpret_cast<lds_u32x4*>(smem + slot + (wave * 4 + i) * 1024)[lane] = u32x4{0u, 0u, 0u, 0u};
      return;
    }
    const int k0 = keys.key_of(j);
    const uint16_t* base = uniform<kPages>((decltype(is_v)::value ? keys.Vh : keys.Kh) + keys.at(k0, pg));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = (wave * 4 + i) * 4 + (lane >> 4), pos = lane & 15;
      dma_16B_at(base, keys.offset(k0, row, decltype(is_v)::value ? v_chunk_pos(row, pos) : k_chunk_pos(row, pos)),
                 __builtin_amdgcn_readfirstlane(lds_mine + slot + i * 1024));
    }
  };
  keys.fetch(0, r.end);
  int pg = keys.page(0), pg_next = keys.page(1), pg_after = keys.page(2);   // of tiles j, j + 1, j + 2
  if (r.begin < r.end) {   // the first tiles go out before it is known how many there are
    stage(std::false_type{}, 0, pg, k_slot(0));
    stage(std::true_type{}, 0, pg, v_slot(0));
    if (keys.key_of(1) < r.end) stage(std::false_type{}, 1, pg_next, k_slot(1));
  }
  // the slot of V(-1) is read once against zero probabilities: clear it
#pragma unroll
  for (int i = 0; i < 4; ++i) reinterpret_cast<lds_u32x4*>(smem + v_slot(1) + (wave * 4 + i) * 1024)[lane] = u32x4{0u, 0u, 0u, 0u};

  // the wave's queries, as fragments
  bf16x8 qf[8];
  {
    const uint16_t* q = static_cast<const uint16_t*>(a.Q) + head * a.q_stride + static_cast<int64_t>(r.t0 + tok) * kD + g * 8;
#pragma unroll
    for (int s = 0; s < 8; ++s) qf[s] = *reinterpret_cast<const bf16x8*>(q + s * 16);
  }
  // What the rows see, as in rows_many.
  const int lim_true = limit_of(a, r, tok);
  const bool sees = lim_true > max(r.lo, r.begin);
  const int lim = sees ? lim_true : INT_MAX;
  int lim_max = sees ? lim_true : 0, lim_min = lim;
#pragma unroll
  for (int x = 1; x < 32; x *= 2) {
    lim_max = max(lim_max, __shfl_xor(lim_max, x));
    lim_min = min(lim_min, __shfl_xor(lim_min, x));
  }
  lim_min = __builtin_amdgcn_readfirstlane(lim_min);   // of the wave
  auto* s_lim = reinterpret_cast<__attribute__((address_space(3))) int*>(smem + kMidWaves * kWaveOBytes<kD>);   // behind the tiles
  if (lane == 0 && kg == 0) s_lim[rg * 2] = active ? lim_max : 0, s_lim[rg * 2 + 1] = active ? lim_min : INT_MAX;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();   // K(0), V(0), K(1) and the limits
  int all_max = 0, all_min = INT_MAX;                  // of the work-group
#pragma unroll
  for (int w = 0; w < kR; ++w) all_max = max(all_max, s_lim[w * 2]), all_min = min(all_min, s_lim[w * 2 + 1]);
  all_max = __builtin_amdgcn_readfirstlane(all_max), all_min = __builtin_amdgcn_readfirstlane(all_min);
  const int end = min(r.end, all_max), n = (end - r.begin + kKeys - 1) / kKeys;

  int k_off[8], v_off[4];
#pragma unroll
  for (int s = 0; s < 8; ++s) k_off[s] = (kg * 32 + l32) * kRowBytes + k_chunk_pos(l32, 2 * s + g) * 16;
  {
    const int r16 = lane & 15, G = (lane >> 4) & 1, row = g * 4 + (r16 >> 2);
#pragma unroll
    for (int db = 0; db < 4; ++db) {
      const int dim = db * 32 + G * 16 + 4 * (r16 & 3);
      v_off[db] = (kg * 32 + row) * kRowBytes + v_chunk_pos(row, dim >> 3) * 16 + (dim & 7) * 2;
    }
  }
  f32x16 o[4], sA, sB, neg_m;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
#pragma unroll
    for (int db = 0; db < 4; ++db) o[db][i] = 0.f;
    sA[i] = sB[i] = neg_m[i] = 0.f;
  }
  bf16x8 pA[2], pB[2];
#pragma unroll
  for (int ks = 0; ks < 2; ++ks)
#pragma unroll
    for (int e = 0; e < 8; ++e) pA[ks][e] = pB[ks][e] = static_cast<__bf16>(0.f);
  float m_ref = -INFINITY, l_run = 0.f;
  bool redo_all = false;   // wave-uniform
  int odd_first = INT_MAX, odd_last = -1;   // as in rows_many

  // hides what a row does not see of its half of tile j, whose page is pg
  auto mask = [&](f32x16& sc, int j, int pg) {
    const int key0 = keys.key_of(j) + kg * 32;
    if (key0 + 32 <= lim_min && key0 >= r.lo && pg >= 0) return;
    hide(sc, r.lo - key0 - g * 4, pg >= 0 ? lim - key0 - g * 4 : 0);
  };
  if (n > 0) {
    if (active) {  // scores of tile 0 and the first reference
      f32x16 zero;
#pragma unroll
      for (int i = 0; i < 16; ++i) zero[i] = 0.f;
#pragma unroll
      for (int s = 0; s < 8; ++s)
        sA = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lds_frag(smem + k_slot(0) + k_off[s]), qf[s], s == 0 ? zero : sA, 0, 0, 0);
      mask(sA, 0, pg);
      float mx = sA[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) mx = fmaxf(mx, sA[i]);
      m_ref = wave_half_max(mx) * a.c;
      if constexpr (!kUnitC) redo_all = __any(far_ref(m_ref));
      if constexpr (kUnitC) {
        const float start = m_ref >= kLowestStart ? m_ref : 0.f;
        redo_all = __any(!(m_ref >= kLowestStart));
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          sA[i] -= start;
          neg_m[i] = -start;
        }
      }
    }
    __syncthreads();               // K(0) has been read by all
    if (n > 2) stage(std::false_type{}, 2, pg_after, k_slot(2));
    auto phase = [&](int j, auto parity, const f32x16& s_cur, f32x16& s_nxt, const bf16x8 (&p_mm)[2], bf16x8 (&p_cur)[2]) {
      constexpr int u = decltype(parity)::value;   // of j
      constexpr int k_nxt = (u ^ 1) * kTile, v_cur = (kS + u) * kTile, v_prev = (kS + (u ^ 1)) * kTile;
      if (active) {
        pipeline_phase<kUnitC>(smem + k_nxt, k_off, smem + v_prev, v_off, qf, s_nxt, p_mm, o, s_cur, p_cur, m_ref, l_run, a.c, neg_m, redo_all);
        mask(s_nxt, j + 1, pg_next);
      }
      // every wave is past K(j+1) and V(j-1); K(j+2) and V(j) have landed
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      if (kPages && ((j + 3) & 63) == 0) keys.fetch(j + 3, r.end);
      const int pg_third = keys.page(j + 3);
      if (j + 3 < n) stage(std::false_type{}, j + 3, pg_third, k_nxt);
      if (j + 1 < n) stage(std::true_type{}, j + 1, pg_next, v_prev);
      const int key0 = r.begin + j * kKeys;
      if (key0 + kKeys > all_min || key0 < r.lo) {
        // as in rows_many; a wave adds what is in its half in the end
        lds_u32x4* mine = reinterpret_cast<lds_u32x4*>(smem + v_cur) + threadIdx.x * 4;
        uint32_t odd = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) odd |= odd_bf16(mine[i]);
        if (__syncthreads_or(odd != 0)) {
          odd_first = min(odd_first, j), odd_last = j;
#pragma unroll
          for (int i = 0; i < 4; ++i) mine[i] = finite_bf16(mine[i]);
          __syncthreads();
        }
      }
      pg = pg_next, pg_next = pg_after, pg_after = pg_third;
    };
    for (int j = 0; j < n; j += 2) {
      phase(j, std::integral_constant<int, 0>{}, sA, sB, pB, pA);
      if (j + 1 >= n) break;
      phase(j + 1, std::integral_constant<int, 1>{}, sB, sA, pA, pB);
    }
    if (active) {  // O += V(n-1) P(n-1)
      const lds_u8* v_last = smem + v_slot(n - 1);
      const bool odd = (n & 1) != 0;   // the last phase was an even one: its probabilities are pA
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int db = 0; db < 4; ++db) {
          const lds_u8* p = v_last + v_off[db] + ks * 16 * kRowBytes;
          const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
              reinterpret_cast<__attribute__((address_space(3))) bf16x4*>(const_cast<lds_u8*>(p)));
          const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
              reinterpret_cast<__attribute__((address_space(3))) bf16x4*>(const_cast<lds_u8*>(p + 8 * kRowBytes)));
          bf16x8 vf;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            vf[e] = lo[e];
            vf[4 + e] = hi[e];
          }
          o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, odd ? pA[ks] : pB[ks], o[db], 0, 0, 0);
        }
      for (int i = odd_first; i <= odd_last; ++i) keys.add_odd_rows(o, keys.key_of(i), keys.key_of(i) + kg * 32, all_min, lim, g);
    }
  }
  float l_tot = wave_half_sum(l_run), m_end = fmaxf(m_ref, kNothing);
  if (!sees) {
    l_tot = 0.f, m_end = kNothing;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
  }
  __syncthreads();   // every wave has read its last tile; LDS takes the rows
  merge_waves<kD, kR, kG>(a, r, smem, o, m_end, l_tot, wave, lane);
}

// ---- the kernels -----------------------------------------------------------------------------------------------------
template <int D, bool kPages>
__global__ __launch_bounds__(kFewWaves * 64, D == 64 ? 4 : 1) void rows_few_kernel(RowsArgs a) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  lds_u8* smem = (lds_u8*)smem_raw;
  each_unit<kFewRows, kPages>(a, (lds_int*)(smem + kFewSmem<D>), [&](const RowSet& r) { rows_few<D, kPages>(a, r, smem); });
}
template <bool kUnitC>
__global__ __launch_bounds__(kMidWaves * 64, 2) void rows_mid_kernel(RowsArgs a) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  lds_u8* smem = (lds_u8*)smem_raw;
  each_unit<kMidRows, true>(a, (lds_int*)(smem + kMidSmem), [&](const RowSet& r) { rows_mid<kUnitC, true>(a, r, smem); });
}
template <bool kUnitC>
__global__ __launch_bounds__(kManyWaves * 64, 2) void rows_many_kernel(RowsArgs a) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  lds_u8* smem = (lds_u8*)smem_raw;
  each_unit<kManyRows, true>(a, (lds_int*)(smem + kManySmem), [&](const RowSet& r) { rows_many<kUnitC, true>(a, r, smem); });
}
// Prompts take both forms in one launch: the n_heavy longest tiles of 128 rows as two of 64, the others whole.  All of them start
// early, the long ones end as early as 64 rows can, and most products still are those of 128.
template <bool kUnitC>
__global__ __launch_bounds__(kManyWaves * 64, 2) void rows_prompt_kernel(RowsArgs a) {
  static_assert(kMidWaves == kManyWaves && 2 * kMidRows == kManyRows, "one launch");
  extern __shared__ __align__(16) uint8_t smem_raw[];
  lds_u8* smem = (lds_u8*)smem_raw;
  const int lane = threadIdx.x & 63;
  const int u = a.by_hkv.of(blockIdx.x), kvh = blockIdx.x - u * a.by_hkv.d;
  const bool heavy = u < 2 * a.n_heavy;
  RowSet r = prompt_rows<kManyRows>(a, heavy ? u >> 1 : u - a.n_heavy, kvh, lane);
  if (heavy) {
    r.tile = r.tile * 2 + (u & 1);
    if (r.tile * kMidRows < r.n_tok * a.rep) rows_mid<kUnitC, false>(a, r, smem);
  } else {
    rows_many<kUnitC, false>(a, r, smem);
  }
}

}  // namespace pc
