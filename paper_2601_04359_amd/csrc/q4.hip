// The KV cache held in 4 bits: rows into it and out of it, and attention over it.
#include <limits.h>
#include <math.h>

#include <algorithm>

#include "q4.h"

namespace pc {
namespace {

constexpr float kNoRef = -3.402823466e38f;     // the reference of a row that has seen no score yet

// ------------------------------------------------------------------------------------------
// pc_q4_store, pc_q4_load.  Bound: bytes.  A lane owns eight elements, so four lanes are a group and agree on its
// largest magnitude by two lane exchanges; rows of K and V of all heads are one run of rows, so that one token of
// many heads fills a launch.
// ------------------------------------------------------------------------------------------
constexpr int kCopyThreads = 256;
// Threads of a launch along one axis fit 32 bits.  Rows of K and of V that one launch copies, in threads:
constexpr int64_t kMaxThreads = UINT32_MAX;
inline int64_t copy_threads(int64_t rows, int D) { return (rows * (D / 8) + kCopyThreads - 1) / kCopyThreads * kCopyThreads; }

struct RowsAt {          // rows 0 .. n - 1 of H heads of two tensors
  int H, D;
  Divisor by_n;
  int64_t k_stride_h, v_stride_h;
};

// the rows' bookkeeping that pc_q4_store writes as well (either pointer may be NULL)
struct Book {
  const int32_t* pos_new;
  int32_t* pos;
  float* weights;
  int64_t pos_stride_h, w_stride_h;
  int Hsel;
};

template <typename T, int D>
__global__ __launch_bounds__(kCopyThreads) void q4_store_kernel(const T* __restrict__ K, const T* __restrict__ V, RowsAt at,
                                                                Q4Rows cache, int row0, int n_units, Book book) {
  constexpr int kLanes = D / 8;      // lanes of a row
  const int n = at.by_n.d;
  const int64_t idx = static_cast<int64_t>(blockIdx.x) * kCopyThreads + threadIdx.x;
  const int unit = static_cast<int>(idx / kLanes), part = static_cast<int>(idx % kLanes);
  if (unit < n_units) {
    int rest = at.by_n.of(unit);
    const int i = unit - rest * n;
    const bool value = rest >= at.H;
    const int h = value ? rest - at.H : rest;
    const T* src = (value ? V + h * at.v_stride_h : K + h * at.k_stride_h) + static_cast<int64_t>(i) * D + part * 8;
    uint32_t top = 0, codes = 0;
    float scale;
    int byte;
    if constexpr (sizeof(T) == 2) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(src);
      for (int k = 0; k < 4; ++k) top = max(top, max(x[k] << 16 & 0x7fffffffu, x[k] & 0x7fff0000u));
      top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 1)));
      top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 2)));
      byte = q4_scale_byte(top);
      scale = q4_scale(byte);
      // (a vector's element is copied before its bits are taken as another type: the compiler takes element 0 of it otherwise)
      const uint32_t w0 = x[0], w1 = x[1], w2 = x[2], w3 = x[3];
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, w0), scale, 0);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, w1), scale, 1);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, w2), scale, 2);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, w3), scale, 3);
    } else {
      const f32x4 x = load_f32x4(reinterpret_cast<const float*>(src)), y = load_f32x4(reinterpret_cast<const float*>(src) + 4);
      for (int k = 0; k < 4; ++k)
        top = max(top, max(__float_as_uint(x[k]) & 0x7fffffffu, __float_as_uint(y[k]) & 0x7fffffffu));
      top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 1)));
      top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 2)));
      byte = q4_scale_byte(top);
      scale = q4_scale(byte);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[0], x[1], scale, 0);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[2], x[3], scale, 1);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, y[0], y[1], scale, 2);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, y[2], y[3], scale, 3);
    }
    if (byte == kQ4BadScale) codes = 0;
    const int64_t row = static_cast<int64_t>(row0) + i;
    uint8_t* out = const_cast<uint8_t*>(value ? cache.v_codes : cache.k_codes) + h * cache.code_stride_h + row * (D / 2);
    uint8_t* out_s = const_cast<uint8_t*>(value ? cache.v_scales : cache.k_scales) + h * cache.scale_stride_h + row * (D / 32);
    reinterpret_cast<uint32_t*>(out)[part] = codes;
    if (part % 4 == 0) out_s[part / 4] = static_cast<uint8_t>(byte);
  }
  // the rows' coordinates and their sums, which begin at zero
  if (book.pos == nullptr && book.weights == nullptr) return;
  for (int64_t t = idx; t < static_cast<int64_t>(book.Hsel) * n; t += static_cast<int64_t>(gridDim.x) * kCopyThreads) {
    const int h = at.by_n.of(static_cast<int>(t));
    const int i = static_cast<int>(t) - h * n;
    const int64_t row = static_cast<int64_t>(row0) + i;
    if (book.pos != nullptr)
      for (int k = 0; k < 3; ++k) book.pos[h * book.pos_stride_h + row * 3 + k] = book.pos_new[i * 3 + k];
    if (book.weights != nullptr) book.weights[h * book.w_stride_h + row] = 0.f;
  }
}

template <typename T, int D>
__global__ __launch_bounds__(kCopyThreads) void q4_load_kernel(T* __restrict__ K, T* __restrict__ V, RowsAt at, Q4Rows cache,
                                                               int row0, int first_unit, int n_units, int32_t* clear) {
  constexpr int kLanes = D / 8;
  const int n = at.by_n.d;
  const int64_t idx = static_cast<int64_t>(blockIdx.x) * kCopyThreads + threadIdx.x;
  if (clear != nullptr && idx == 0) *clear = 0;
  int unit = static_cast<int>(idx / kLanes);
  const int part = static_cast<int>(idx % kLanes);
  if (unit >= n_units) return;
  unit += first_unit;
  const int rest = at.by_n.of(unit);
  const int i = unit - rest * n;
  const bool value = rest >= at.H;
  const int h = value ? rest - at.H : rest;
  const int64_t row = static_cast<int64_t>(row0) + i;
  const uint8_t* codes = (value ? cache.v_codes : cache.k_codes) + h * cache.code_stride_h + row * (D / 2);
  const uint8_t* scales = (value ? cache.v_scales : cache.k_scales) + h * cache.scale_stride_h + row * (D / 32);
  const bf16x8 x = q4_to_bf16(reinterpret_cast<const uint32_t*>(codes)[part], q4_scale(scales[part / 4]));
  T* dst = (value ? V + h * at.v_stride_h : K + h * at.k_stride_h) + static_cast<int64_t>(i) * D + part * 8;
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<bf16x8*>(dst) = x;
  } else {
    f32x4 lo, hi;
    for (int k = 0; k < 4; ++k) lo[k] = static_cast<float>(x[k]), hi[k] = static_cast<float>(x[4 + k]);
    store_f32x4(reinterpret_cast<float*>(dst), lo);
    store_f32x4(reinterpret_cast<float*>(dst) + 4, hi);
  }
}

// ------------------------------------------------------------------------------------------
// Attention straight from the codes, for few query rows: 16 kRT rows per work-group, its eight waves deal the keys in
// steps of 32 (sixteen waves were 20 % faster per step where one compute unit does all, and 0.5 us slower to end).
//   * S^T = K Q^T by 16x16x32 products.  Which dims a product contracts is free as long as both operands agree: lane
//     (r = l % 16, g = l / 16) takes dims g D/4 .. of key row r, which lie in one scale group and are one load,
//     and its dwords of eight codes are the operands of the D/32 products after four conversions each.  K never
//     touches LDS.
//   * The result leaves lane (q, g) with keys 4 g .. 4 g + 3 of query q, of two tiles of 16: the eight k-slots of
//     O^T += V^T P^T.  V is converted by the lane that loads it (one scale for its 32 dims) and goes
//     through LDS of the wave's own as bf16 rows, read back by transposing loads.
//   * Softmax in base 2 against a reference that lags the maximum by at most 2^8; sums in fp32.  Far references take
//     exponents of their own (see far_exponent).
//   * bf16 queries: a probability is rounded to bf16 in front of the second product, half a step of its size, as in
//     pc_frame_attn; the sum it is divided by, the log-sum-exp and the weights are those of the unrounded ones.  Where one
//     key dominates, the output is off by that and its own rounding (0.0024 of its size, 0.0017 with fp32 probabilities).  A
//     second part would double the products of a loop whose registers are full at two tiles.
//   * fp32 queries and probabilities are three bf16 parts each: keys and values are exact in bf16, so the
//     products are exact and the sums are the fp32 ones.
// ------------------------------------------------------------------------------------------
constexpr int kWaves = 8, kThreads = 64 * kWaves;
constexpr int kStep = 32;                   // keys of a wave's step
constexpr int kMaxShares = 128;             // of the keys
// Rows per KV head up to which the weights come from logits that are kept (against 68 bytes and the products: 12 rows x
// 16,000 keys 13.1 us, 14.1 formed again; 16 rows 15.0 and 14.6).  Where the attention is not cut, that launch would be one
// more for it: up to 8 rows (12 rows x 300 keys 10.1 us, 8.5 formed again).
constexpr int kLogitRows = 12, kLogitRowsFewKeys = 8;
constexpr int kMaxJoinRows = 64;            // of a selection head, at a time

struct AttnArgs {
  Q4Rows cache;
  int rep, Nk;
  Divisor by_nq, by_tiles;                  // rows per head, row tiles per KV head
  int n_tiles, share_steps;                 // row tiles of all KV heads, steps of a key share
  int64_t q_stride_h, o_stride_h;
  float c;                                  // scale * log2(e)
  float* part_o;                            // NULL: one share
  float2* part_ml;
  float* lse;                               // natural logarithm, or NULL
  float* lse2;                              // base 2, for the weights, or NULL; of a row with a far reference: infinity
  float2* ref;                              // the same in its two terms: reference and log2 of the sum
  float* logits;                            // [rows_all][whole steps] for the weights of few rows, or NULL
  int64_t rows_all;
};

// What the scoring subtracts; infinity for a row of a far reference: probability 0 until its two terms are read.
__device__ __forceinline__ float lse2_of(float m, float log_l) {
  const float e2 = m + log_l;
  return far_ref(m) && e2 == e2 ? INFINITY : e2;
}

template <int D>
__device__ __forceinline__ int v_place(int key, int chunk) {      // a 32-byte chunk of a key's row in LDS
  return chunk ^ (D == 128 ? key & 7 : (key >> 1) & 3);
}

template <typename T, int D>
struct QueryFrags {
  static constexpr int kParts = sizeof(T) == 2 ? 1 : 3, kSteps = D / 32;
  bf16x8 f[kSteps][kParts];
  // the row's dims g D/4 + 8 b .. + 7, from its 16-byte chunks
  template <class Chunk>
  __device__ __forceinline__ void from(Chunk&& chunk, int g) {
#pragma unroll
    for (int b = 0; b < kSteps; ++b) {
      if constexpr (kParts == 1) {
        f[b][0] = __builtin_bit_cast(bf16x8, chunk(g * (D / 32) + b));
      } else {
        const f32x4 x = __builtin_bit_cast(f32x4, chunk(g * (D / 16) + 2 * b)), y = __builtin_bit_cast(f32x4, chunk(g * (D / 16) + 2 * b + 1));
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          __bf16 hi, mid, lo;
          split3(e < 4 ? x[e] : y[e - 4], hi, mid, lo);
          f[b][0][e] = hi, f[b][1][e] = mid, f[b][2][e] = lo;
        }
      }
    }
  }
  __device__ __forceinline__ void load(const T* row, int g) {
    from([&](int c) { return load_chunk(row + c * (16 / static_cast<int>(sizeof(T)))); }, g);
  }
  // fp32 rows only promise element alignment; the hardware takes 16-byte accesses at any dword
  static __device__ __forceinline__ u32x4 load_chunk(const T* p) {
    if constexpr (kParts == 1) return *reinterpret_cast<const u32x4*>(p);
    else return __builtin_bit_cast(u32x4, load_f32x4(p));
  }
};

// A lane's piece of a key row: D/8 bytes of codes, as D/32 dwords; `row` is counted from the bases.
template <int D>
struct KeyCodes {
  uint32_t w[D / 32];
  int byte;
  __device__ __forceinline__ void load(const uint8_t* codes, const uint8_t* scales, uint32_t row, int g) {
    const uint8_t* src = codes + (row * (D / 2) + g * (D / 8));
    if constexpr (D == 128) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(src);
      w[0] = x[0], w[1] = x[1], w[2] = x[2], w[3] = x[3];
      byte = scales[row * 4 + g];
    } else {
      const u32x2 x = *reinterpret_cast<const u32x2*>(src);
      w[0] = x[0], w[1] = x[1];
      byte = scales[row * 2 + g / 2];
    }
  }
};

// 16 keys by 16 queries: key rows of the lanes' pieces times the queries' fragments.  Small parts first.
template <typename T, int D>
__device__ __forceinline__ f32x4 scores(const bf16x8 (&k)[D / 32], const QueryFrags<T, D>& q) {
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int p = QueryFrags<T, D>::kParts - 1; p >= 0; --p)
#pragma unroll
    for (int b = 0; b < D / 32; ++b) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[b], q.f[b][p], s, 0, 0, 0);
  return s;
}

template <typename T, int D, int kRT>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 && kRT == 1 ? 4 : 2) void q4_attn_kernel(const T* __restrict__ Q, T* __restrict__ O, AttnArgs a) {
  using lds_byte = __attribute__((address_space(3))) uint8_t;
  constexpr int kParts = QueryFrags<T, D>::kParts;
  constexpr int kTileBytes = kStep * D * 2;                 // a wave's V rows; its partial output as well
  constexpr int kGroups = D / 32, kVRows = 64 / kGroups, kVLoads = kStep / kVRows;
  static_assert(16 * D * 4 == kTileBytes, "partial outputs take the place of the V rows");
  __shared__ __align__(16) uint8_t smem[kWaves * kTileBytes + kWaves * 16 * 8];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  int unit = xcd_contiguous_index(blockIdx.x, gridDim.x);
  const int split = unit / a.n_tiles;
  unit -= split * a.n_tiles;
  const int kvh = a.by_tiles.of(unit), tile = unit - kvh * a.by_tiles.d;
  const int n_rows = a.rep * a.by_nq.d;
  const uint8_t* kc = a.cache.k_codes + kvh * a.cache.code_stride_h;
  const uint8_t* ks = a.cache.k_scales + kvh * a.cache.scale_stride_h;
  const uint8_t* vc = a.cache.v_codes + kvh * a.cache.code_stride_h;
  const uint8_t* vs = a.cache.v_scales + kvh * a.cache.scale_stride_h;
  const int n_steps = (a.Nk + kStep - 1) / kStep;
  const int step_end = min((split + 1) * a.share_steps, n_steps);

  KeyCodes<D> raw_k[2];
  u32x4 raw_v[kVLoads];
  int raw_s[kVLoads];
  // From the step's first row by scalar bases; the lanes' offsets are the same in every step but the one with the last row,
  // which stands for those that are not there.
  auto fetch_rows = [&](const uint8_t* kcs, const uint8_t* kss, const uint8_t* vcs, const uint8_t* vss, uint32_t last) {
#pragma unroll
    for (int t = 0; t < 2; ++t) raw_k[t].load(kcs, kss, min(static_cast<uint32_t>(t * 16 + r), last), g);
#pragma unroll
    for (int i = 0; i < kVLoads; ++i) {
      const uint32_t row = min(static_cast<uint32_t>(i * kVRows + lane / kGroups), last);
      raw_v[i] = *reinterpret_cast<const u32x4*>(vcs + (row * (D / 2) + lane % kGroups * 16));
      raw_s[i] = vss[row * kGroups + lane % kGroups];
    }
  };
  auto fetch = [&](int step) {
    const int64_t k0 = static_cast<int64_t>(step) * kStep;
    const uint8_t *kcs = kc + k0 * (D / 2), *kss = ks + k0 * kGroups, *vcs = vc + k0 * (D / 2), *vss = vs + k0 * kGroups;
    if (k0 + kStep <= a.Nk) fetch_rows(kcs, kss, vcs, vss, kStep - 1);
    else fetch_rows(kcs, kss, vcs, vss, static_cast<uint32_t>(a.Nk - 1 - k0));
  };
  // The queries are fetched in front of the first codes: loads end in order, and a wait for queries behind codes would be a
  // wait for both (in the loop, where the compiler puts it, it made every step wait for the next one's codes).  Two tiles
  // of them go through LDS, a few chunks per thread: as fragments every wave would fetch both, 64 KB per work-group in
  // front of the codes (8/2 heads x 64 rows x 4,000 keys 12.6 -> 11.9 us); one tile is quicker without the barrier
  // (16/4 x 1 x 41,800 11.9 -> 11.4).
  auto row_of = [&](int i) {
    const int rho = min(tile * kRT * 16 + i, n_rows - 1), head = a.by_nq.of(rho);
    return Q + (kvh * a.rep + head) * a.q_stride_h + static_cast<int64_t>(rho - head * a.by_nq.d) * D;
  };
  QueryFrags<T, D> q[kRT];
  int step = split * a.share_steps + wave;
  if constexpr (kRT == 1) {
    q[0].load(row_of(r), g);
    asm volatile("" ::: "memory");
    if (step < step_end) fetch(step);
  } else {
    constexpr int kOfChunk = 16 / static_cast<int>(sizeof(T)), kRowChunks = D / kOfChunk, kChunks = 16 * kRT * kRowChunks;
    constexpr int kPerThread = kChunks / kThreads > 0 ? kChunks / kThreads : 1;
    static_assert(kChunks % kThreads == 0 || kChunks < kThreads, "whole rounds of chunks");
    __shared__ __align__(16) uint8_t smem_q[kChunks * 16];
    lds_byte* s_q = (lds_byte*)smem_q;
    auto place = [](int row, int c) { return (row * kRowChunks + (c ^ (row & (kRowChunks < 16 ? kRowChunks - 1 : 15)))) * 16; };
    u32x4 chunk[kPerThread];
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
      const int c = (static_cast<int>(threadIdx.x) + k * kThreads) % kChunks;
      chunk[k] = QueryFrags<T, D>::load_chunk(row_of(c / kRowChunks) + c % kRowChunks * kOfChunk);
    }
    asm volatile("" ::: "memory");
    if (step < step_end) fetch(step);
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
      const int c = static_cast<int>(threadIdx.x) + k * kThreads;
      if (c < kChunks) *reinterpret_cast<__attribute__((address_space(3))) u32x4*>(s_q + place(c / kRowChunks, c % kRowChunks)) = chunk[k];
    }
    __syncthreads();
#pragma unroll
    for (int rt = 0; rt < kRT; ++rt)
      q[rt].from([&](int c) { return *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(s_q + place(rt * 16 + r, c)); }, g);
  }
  f32x4 o[kRT][D / 16];
  float m[kRT], l[kRT];
#pragma unroll
  for (int rt = 0; rt < kRT; ++rt) {
    m[rt] = kNoRef, l[rt] = 0.f;
#pragma unroll
    for (int db = 0; db < D / 16; ++db) o[rt][db] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  lds_byte* mine = (lds_byte*)smem + wave * kTileBytes;
  // where a transposing load of 16 dims finds the four dims 4 (r % 4) of key 4 g + r / 4
  const int v_key = g * 4 + (r >> 2);
  lds_byte* v_at = mine + v_key * (D * 2) + (r & 3) * 8;

  for (; step < step_end; step += kWaves) {
    const int k0 = step * kStep;
    bf16x8 kf[2][D / 32];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int b = 0; b < D / 32; ++b) kf[t][b] = q4_to_bf16(raw_k[t].w[b], q4_scale(raw_k[t].byte));
    wave_lds_sync();       // the step before has read its values
#pragma unroll
    for (int i = 0; i < kVLoads; ++i) {
      const int key = i * kVRows + lane / kGroups, grp = lane % kGroups;
      const float scale = q4_scale(raw_s[i]);
#pragma unroll
      for (int b = 0; b < 4; ++b)
        *reinterpret_cast<__attribute__((address_space(3))) bf16x8*>(
            mine + key * (D * 2) + v_place<D>(key, grp * 2 + b / 2) * 32 + (b & 1) * 16) = q4_to_bf16(raw_v[i][b], scale);
    }
    wave_lds_sync();
    if (step + kWaves < step_end) fetch(step + kWaves);
    bf16x8 pf[kRT][kParts];
#pragma unroll
    for (int rt = 0; rt < kRT; ++rt) {
      f32x4 s[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) s[t] = scores<T, D>(kf[t], q[rt]);
      if (k0 + kStep > a.Nk) {
        asm volatile("" ::: "memory");     // a branch, not 24 selects in every step
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (k0 + t * 16 + g * 4 + i >= a.Nk) s[t][i] = -INFINITY;
      }
      if (kRT == 1 && a.logits != nullptr && r < n_rows) {
        float* to = a.logits + (static_cast<int64_t>(kvh) * n_rows + r) * (static_cast<int64_t>(n_steps) * kStep) + k0 + g * 4;
#pragma unroll
        for (int t = 0; t < 2; ++t) *reinterpret_cast<f32x4*>(to + t * 16) = s[t];
      }
      float mx = s[0][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) mx = fmaxf(mx, s[i >> 2][i & 3]);
      mx *= a.c;
      float ref = m[rt];
      if (__any(!(mx <= m[rt] + 8.f) || far_ref(m[rt]))) {
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float m_new = fmaxf(m[rt], mx), alpha = __builtin_amdgcn_exp2f(m[rt] - m_new);
        l[rt] *= alpha;
#pragma unroll
        for (int db = 0; db < D / 16; ++db) o[rt][db] *= alpha;
        ref = m[rt] = m_new;
        if (far_ref(m_new)) {     // its exponents come to the common fma as products of c, with 0 as their reference
          const float by = 1.f / a.c;
#pragma unroll
          for (int i = 0; i < 8; ++i) s[i >> 2][i & 3] = far_exponent(s[i >> 2][i & 3], a.c, m_new) * by;
          ref = 0.f;
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float p = __builtin_amdgcn_exp2f(fmaf(s[i >> 2][i & 3], a.c, -ref));
        l[rt] += p;
        if constexpr (kParts == 1) {
          pf[rt][0][i] = static_cast<__bf16>(p);
        } else {
          __bf16 hi, mid, lo;
          split3(p, hi, mid, lo);
          pf[rt][0][i] = hi, pf[rt][1][i] = mid, pf[rt][2][i] = lo;
        }
      }
    }
#pragma unroll
    for (int db = 0; db < D / 16; ++db) {
      lds_byte* src = v_at + v_place<D>(v_key, db) * 32;
      const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(reinterpret_cast<__attribute__((address_space(3))) bf16x4*>(src));
      const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
          reinterpret_cast<__attribute__((address_space(3))) bf16x4*>(src + 16 * D * 2));
      const bf16x8 vf = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
#pragma unroll
      for (int rt = 0; rt < kRT; ++rt)
#pragma unroll
        for (int p = kParts - 1; p >= 0; --p) o[rt][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[rt][p], o[rt][db], 0, 0, 0);
    }
  }

  // the waves' parts, 16 rows at a time: 16-byte unit u of row q lies at u ^ q
  constexpr int kUnits = D / 4;
  auto* s_ml = reinterpret_cast<__attribute__((address_space(3))) float*>((lds_byte*)smem + kWaves * kTileBytes);
#pragma unroll
  for (int rt = 0; rt < kRT; ++rt) {
    float sum = l[rt];
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    __syncthreads();
#pragma unroll
    for (int db = 0; db < D / 16; ++db)
      *reinterpret_cast<__attribute__((address_space(3))) f32x4*>(mine + r * (D * 4) + ((db * 4 + g) ^ r) * 16) = o[rt][db];
    if (lane < 16) {
      s_ml[(wave * 16 + lane) * 2] = m[rt];
      s_ml[(wave * 16 + lane) * 2 + 1] = sum;
    }
    __syncthreads();
    const int row = threadIdx.x / kUnits, u = threadIdx.x % kUnits;
    const int rho = (tile * kRT + rt) * 16 + row;
    if (row < 16 && rho < n_rows) {
      float M = kNoRef, lt = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) M = fmaxf(M, s_ml[(w * 16 + row) * 2]);
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float wt = __builtin_amdgcn_exp2f(s_ml[(w * 16 + row) * 2] - M);
        lt += wt * s_ml[(w * 16 + row) * 2 + 1];
        const f32x4 v = *reinterpret_cast<const __attribute__((address_space(3))) f32x4*>((lds_byte*)smem + w * kTileBytes +
                                                                                         row * (D * 4) + (u ^ row) * 16);
        acc += wt * v;
      }
      const int64_t at = static_cast<int64_t>(kvh) * n_rows + rho;
      if (a.part_o != nullptr) {
        const int64_t at_s = split * a.rows_all + at;
        *reinterpret_cast<f32x4*>(a.part_o + at_s * D + u * 4) = acc;
        if (u == 0) a.part_ml[at_s] = make_float2(M, lt);
      } else {
        const float inv = 1.f / lt;
        const int head = a.by_nq.of(rho);
        T* to = O + (kvh * a.rep + head) * a.o_stride_h + static_cast<int64_t>(rho - head * a.by_nq.d) * D + u * 4;
        if constexpr (kParts == 1) {
          *reinterpret_cast<u32x2*>(to) = u32x2{pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv)};
        } else {
          store_f32x4(to, f32x4{acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv});
        }
        if (u == 0) {
          const float log_l = log2f(lt), e2 = M + log_l;
          if (a.lse != nullptr) a.lse[at] = e2 * 0.6931471805599453f;
          if (a.lse2 != nullptr) {
            a.lse2[at] = lse2_of(M, log_l);
            a.ref[at] = make_float2(M, log_l);
          }
        }
      }
    }
  }
}

// ------------------------------------------------------------------------------------------
// What follows the attention of few rows, in one launch: a work-group per row that joins its key shares, and
// work-groups that form the weights of 1,024 keys each from the logits that the attention left (8 R bytes per key there
// and back for R rows, where forming them again reads 68 and multiplies).  Each work-group joins the shares'
// (reference, sum) pairs for itself.  Bound: two memory latencies.
// ------------------------------------------------------------------------------------------
constexpr int kJoinThreads = 256;

struct JoinArgs {
  int n_splits, rows, Hkv, Hsel, Nk;        // rows per KV head
  int row_blocks;                           // work-groups that join rows: all of them, or 0
  Divisor by_blocks;                        // key blocks of a selection head
  int64_t logit_stride, w_stride_h;
  float c, decay;
  float* weights;
};

// Reference and sum of a row over its shares, by one wave: in every lane.
__device__ __forceinline__ float2 join_ml(const float2* __restrict__ ml, int64_t stride, int n, int lane) {
  float M = kNoRef, l = 0.f;
  float2 x[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    x[k] = lane + k * 64 < n ? ml[(lane + k * 64) * stride] : make_float2(kNoRef, 0.f);
    M = fmaxf(M, x[k].x);
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) M = fmaxf(M, __shfl_xor(M, d));
#pragma unroll
  for (int k = 0; k < 2; ++k) l += __builtin_amdgcn_exp2f(x[k].x - M) * x[k].y;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) l += __shfl_xor(l, d);
  return make_float2(M, l);
}

template <typename T, int D>
__global__ __launch_bounds__(kJoinThreads) void q4_join_kernel(T* __restrict__ O, AttnArgs a, JoinArgs j) {
  constexpr int kUnits = D / 4, kLanes = kJoinThreads / kUnits;
  __shared__ f32x4 s_o[kLanes][kUnits];
  __shared__ float s_w[kMaxShares];
  __shared__ float2 s_ref[kMaxJoinRows];      // of a row: reference and log2 of its sum
  __shared__ int s_far;                       // a row with a far reference has been seen
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (static_cast<int>(blockIdx.x) < j.row_blocks) {
    const int64_t at = blockIdx.x;
    const int u = threadIdx.x % kUnits, part = threadIdx.x / kUnits;
    // the first partial rows are fetched in front of the pairs they are weighed by
    const float* from = a.part_o + at * D + u * 4;
    auto fetch = [&](f32x4 (&v)[8], int s0) {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = *reinterpret_cast<const f32x4*>(from + min(s0 + k * kLanes, j.n_splits - 1) * a.rows_all * D);
    };
    f32x4 v[8];
    fetch(v, part);
    const float own = static_cast<int>(threadIdx.x) < j.n_splits ? a.part_ml[threadIdx.x * a.rows_all + at].x : kNoRef;
    const float2 row = join_ml(a.part_ml + at, a.rows_all, j.n_splits, lane);
    static_assert(kMaxShares <= kJoinThreads, "a thread per share");
    if (static_cast<int>(threadIdx.x) < j.n_splits) s_w[threadIdx.x] = __builtin_amdgcn_exp2f(own - row.x);
    __syncthreads();
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = part;;) {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (s0 + k * kLanes < j.n_splits) acc += s_w[s0 + k * kLanes] * v[k];
      s0 += 8 * kLanes;
      if (s0 >= j.n_splits) break;
      fetch(v, s0);
    }
    s_o[part][u] = acc;
    __syncthreads();
    if (part != 0) return;
#pragma unroll
    for (int p = 1; p < kLanes; ++p) acc += s_o[p][u];
    const float inv = 1.f / row.y;
    const int head = a.by_nq.of(static_cast<int>(at));
    T* to = O + head * a.o_stride_h + (at - static_cast<int64_t>(head) * a.by_nq.d) * D + u * 4;
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<u32x2*>(to) = u32x2{pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv)};
    } else {
      store_f32x4(to, f32x4{acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv});
    }
    if (u == 0) {
      const float log_l = log2f(row.y), e2 = row.x + log_l;
      if (a.lse != nullptr) a.lse[at] = e2 * 0.6931471805599453f;
      if (a.lse2 != nullptr) {
        a.lse2[at] = lse2_of(row.x, log_l);
        a.ref[at] = make_float2(row.x, log_l);
      }
    }
    return;
  }
  // weights
  const int unit = blockIdx.x - j.row_blocks;
  const int sel = j.by_blocks.of(unit), block = unit - sel * j.by_blocks.d;
  const int per = j.Hkv / j.Hsel * j.rows;          // rows of the selection head
  const int64_t row0 = static_cast<int64_t>(sel) * per;
  const int k0 = block * (4 * kJoinThreads) + threadIdx.x * 4;
  const bool mine = k0 < j.Nk;
  const float* from = a.logits + row0 * j.logit_stride + (mine ? k0 : 0);
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  if (threadIdx.x == 0) s_far = 0;
  for (int r0 = 0; r0 < per; r0 += kMaxJoinRows) {
    const int n = min(per - r0, kMaxJoinRows);
    __syncthreads();
    for (int r = wave; r < n; r += kJoinThreads / 64) {
      float2 ref;
      if (j.n_splits > 1) {
        ref = join_ml(a.part_ml + row0 + r0 + r, a.rows_all, j.n_splits, lane);
        ref.y = log2f(ref.y);
      } else {
        ref = a.ref[row0 + r0 + r];
      }
      if (lane == 0) {
        s_ref[r] = ref;
        if (far_ref(ref.x)) s_far = 1;
      }
    }
    __syncthreads();
    if (s_far == 0) {
#pragma unroll 4
      for (int r = 0; r < n; ++r) {
        const f32x4 s = *reinterpret_cast<const f32x4*>(from + (r0 + r) * j.logit_stride);
        const float e2 = s_ref[r].x + s_ref[r].y;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] += __builtin_amdgcn_exp2f(fmaf(s[i], j.c, -e2));
      }
    } else {
      for (int r = 0; r < n; ++r) {
        const f32x4 s = *reinterpret_cast<const f32x4*>(from + (r0 + r) * j.logit_stride);
        const float2 ref = s_ref[r];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          sum[i] += __builtin_amdgcn_exp2f(far_ref(ref.x) ? far_exponent(s[i], j.c, ref.x) - ref.y
                                                          : fmaf(s[i], j.c, -(ref.x + ref.y)));
      }
    }
  }
  float* w = j.weights + sel * j.w_stride_h + k0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (k0 + i < j.Nk) w[i] = j.decay == 0.f ? sum[i] : fmaf(j.decay, w[i], sum[i]);
}

// ------------------------------------------------------------------------------------------
// The weights of more rows: weights[j] = decay * weights[j] + sum over the query rows of exp2(c s - lse2), the scores
// formed once more from the keys' codes.  A wave owns 64 or 128 keys as the second operand (a lane sums its keys' columns
// over the queries it sees) and walks the query rows in tiles of 16, the next one in flight.  Where keys are few, the
// waves of a work-group share 64 keys, deal the row tiles and are added up in their order; where they are many, each
// has keys of its own: dealing 16 row tiles of 60,000 keys over eight waves converted every key eight times (57 us
// instead of 35), and 128 keys per wave halve the queries' way through L2 (24).  With one sum for all heads a wave
// walks the KV heads as well.
// kRest: the last launch of the form for many rows.  pc_score's column pass has summed the rows' probabilities, but for rows
// of a far reference, which it leaves out; this adds its parts up (a wave per KV head of a shared sum) and, where there are
// such rows, their probabilities.
// ------------------------------------------------------------------------------------------
struct WeighArgs {
  Q4Rows cache;
  int rep, Nk, Hkv, Hsel;
  Divisor by_nq, by_blocks;                 // rows per head, key blocks of a selection head
  int dealt;                                // waves that share keys: 1, 2, 4 or 8
  int64_t q_stride_h, w_stride_h;
  float c, decay;
  const float* lse2;                        // see AttnArgs; kRest: natural log-sum-exps
  const float2* ref;
  float* weights;
  ScoreParts parts;                         // kRest
  const int32_t* any_far;
};
template <typename T, int D, int kTiles, bool kRest = false>
__global__ __launch_bounds__(kThreads) void q4_weigh_kernel(const T* __restrict__ Q, WeighArgs a) {
  constexpr int kKeys = 16 * kTiles;
  __shared__ float s_sum[kWaves][kKeys];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  const int unit = xcd_contiguous_index(blockIdx.x, gridDim.x);
  const int sel = a.by_blocks.of(unit), block = unit - sel * a.by_blocks.d;
  const int row_wave = wave & (a.dealt - 1), step = 16 * a.dealt;
  const int groups = blockDim.x / 64 / a.dealt;
  const int block0 = block * groups * kKeys, k0 = block0 + wave / a.dealt * kKeys;
  const int k_first = min(k0, a.Nk - 1);      // the last work-group's waves may lie behind the last key
  const int n_rows = a.rep * a.by_nq.d, per = a.Hkv / a.Hsel;
  float sum[kTiles] = {};
  float parts = 0.f, old = 0.f;
  int heads_end = (sel + 1) * per;
  if constexpr (kRest) {
    static_assert(kKeys == 64, "a lane per key");
    const int key = min(block0 + lane, a.Nk - 1);
    const int any_far = *a.any_far;
    if (a.decay != 0.f) old = a.weights[sel * a.w_stride_h + key];
    const float* from = a.parts.sums + key;
    for (int kvh = sel * per + wave; kvh < heads_end; kvh += a.dealt) {
      float v[kMaxScoreParts];
#pragma unroll
      for (int p = 0; p < kMaxScoreParts; ++p)
        v[p] = p < a.parts.n ? from[(static_cast<int64_t>(p) * a.Hkv + kvh) * a.Nk] : 0.f;
#pragma unroll
      for (int p = 0; p < kMaxScoreParts; ++p) parts += v[p];
    }
    if (any_far == 0) heads_end = 0;
  }
  for (int kvh = sel * per; kvh < heads_end; ++kvh) {
    bf16x8 kf[kTiles][D / 32];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      KeyCodes<D> raw;
      raw.load(a.cache.k_codes + (kvh * a.cache.code_stride_h + static_cast<int64_t>(k_first) * (D / 2)),
               a.cache.k_scales + (kvh * a.cache.scale_stride_h + static_cast<int64_t>(k_first) * (D / 32)),
               min(t * 16 + r, a.Nk - 1 - k_first), g);
#pragma unroll
      for (int b = 0; b < D / 32; ++b) kf[t][b] = q4_to_bf16(raw.w[b], q4_scale(raw.byte));
    }
    const float* lse2 = a.lse2 + static_cast<int64_t>(kvh) * n_rows;
    QueryFrags<T, D> next;
    float next_e2[4];
    auto scores_of = [](const QueryFrags<T, D>& q, const bf16x8 (&k)[D / 32]) {
      f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int p = QueryFrags<T, D>::kParts - 1; p >= 0; --p)
#pragma unroll
        for (int b = 0; b < D / 32; ++b) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q.f[b][p], k[b], s, 0, 0, 0);
      return s;
    };
    auto fetch = [&](int row0) {
      const int rho = min(row0 + r, n_rows - 1);
      const int head = a.by_nq.of(rho);
      next.load(Q + (kvh * a.rep + head) * a.q_stride_h + static_cast<int64_t>(rho - head * a.by_nq.d) * D, g);
#pragma unroll
      for (int i = 0; i < 4; ++i) next_e2[i] = lse2[min(row0 + g * 4 + i, n_rows - 1)];
    };
    if (!kRest && row_wave * 16 < n_rows) fetch(row_wave * 16);
    float top = kRest ? INFINITY : 0.f;            // infinity: a row of a far reference has been left out
    for (int row0 = row_wave * 16; !kRest && row0 < n_rows; row0 += step) {
      const QueryFrags<T, D> q = next;
      float e2[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        top = fmaxf(top, next_e2[i]);
        e2[i] = row0 + g * 4 + i < n_rows ? next_e2[i] : INFINITY;   // a row that is not there: probability 0
      }
      if (row0 + step < n_rows) fetch(row0 + step);
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        const f32x4 s = scores_of(q, kf[t]);
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[t] += __builtin_amdgcn_exp2f(fmaf(s[i], a.c, -e2[i]));
      }
    }
    if (!__any(top == INFINITY)) continue;
    // those rows: here the logarithm of the sum would be lost in the rounding of the reference's sum with it
    for (int row0 = row_wave * 16; row0 < n_rows; row0 += step) {
      fetch(row0);
      const float2* ref = a.ref + static_cast<int64_t>(kvh) * n_rows;
      float2 e2[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        // (kRest: as the column pass decided)
        const bool far = kRest ? fabsf(next_e2[i] * 1.4426950408889634f) >= kFarRef : next_e2[i] == INFINITY;
        e2[i] = row0 + g * 4 + i < n_rows && far ? ref[row0 + g * 4 + i] : make_float2(0.f, INFINITY);
      }
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        const f32x4 s = scores_of(next, kf[t]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          // (a score summed in another order than the reference's may lie an ulp above it, and that is no small number here)
          const float x = far_exponent(s[i], a.c, e2[i].x);
          sum[t] += __builtin_amdgcn_exp2f((x > 0.f ? 0.f : x) - e2[i].y);
        }
      }
    }
  }
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    sum[t] += __shfl_xor(sum[t], 16);
    sum[t] += __shfl_xor(sum[t], 32);
    if (g == 0) s_sum[wave][t * 16 + r] = sum[t];
  }
  if constexpr (kRest) {
    wave_lds_sync();
    s_sum[wave][lane] += parts;
  }
  __syncthreads();
  // key i of the work-group: of the waves from i / kKeys * dealt on
  for (int i = threadIdx.x; i < groups * kKeys && block0 + i < a.Nk; i += blockDim.x) {
    const int from = i / kKeys * a.dealt;
    float x = 0.f;
    for (int w = 0; w < a.dealt; ++w) x += s_sum[from + w][i % kKeys];
    float* w = a.weights + sel * a.w_stride_h + block0 + i;
    if (!kRest && a.decay != 0.f) old = *w;
    *w = a.decay == 0.f ? x : fmaf(a.decay, old, x);
  }
}

// ------------------------------------------------------------------------------------------
// host
// ------------------------------------------------------------------------------------------
constexpr size_t kWsAlign = 256;
// Query rows of a KV head from which on the cache is turned into bf16 rows first.
// 16/4 heads, direct and over expanded rows: 512 rows x 60,000 keys 96 and 120 us, 768 rows 163 and 144; x 16,000 38 and 46,
// 56 and 57; x 1,179 13.5 and 12.1, 16.1 and 12.5.  Short caches of three heads to a KV head lose by it (24/8, 768 rows x 4,000
// keys 30 and 36 us, x 60,000 301 and 255).  The rows are a workspace of 512 bytes per row and KV head.  A cache of more rows
// than one launch expands is read as it lies.
constexpr int kExpandRows = 768;

// How a call is made, and what lies where in its workspace (`base` may be NULL where only the size is asked for).
struct Q4Plan {
  bool expand, keep_logits;     // the cache as bf16 rows and pc_frame_attn; weights from kept logits
  int row_tiles, n_splits;      // tiles of 16 queries per work-group, key shares
  float *part_o, *lse, *logits;
  float2 *part_ml, *ref;
  int32_t* any_far;
  uint16_t *k_rows, *v_rows;
  void* attn_ws;
  size_t attn_bytes, bytes;    // of attn_ws, which the scoring takes after the attention
  Q4Plan(int dtype, int Hq, int Hkv, int Nq, int Nk, int D, bool weights, void* base) {
    *this = Q4Plan();
    const int rows = Hq / Hkv * Nq;
    const int64_t all = static_cast<int64_t>(Hkv) * rows;
    size_t at = 0;
    auto take = [&](int64_t n) {
      void* p = static_cast<uint8_t*>(base) + at;
      at += align_up(static_cast<size_t>(n), kWsAlign);
      return p;
    };
    expand = dtype == PC_BF16 && D == 128 && rows >= kExpandRows && copy_threads(2ll * Hkv * Nk, D) <= kMaxThreads;
    if (expand) {
      const int64_t bytes_kv = static_cast<int64_t>(Hkv) * Nk * D * 2;
      k_rows = static_cast<uint16_t*>(take(bytes_kv));
      v_rows = static_cast<uint16_t*>(take(bytes_kv));
      attn_bytes = pc_frame_attn_workspace_bytes_for(dtype, Hq, Hkv, Nq, Nk, D);
      if (weights) attn_bytes = std::max(attn_bytes, pc_score_workspace_bytes(Hq, Hkv, Nq, Nk, 1));
      attn_ws = take(attn_bytes);
    } else {
      row_tiles = rows <= 16 ? 1 : 2;
      const int64_t tiles = static_cast<int64_t>(ceil_div(rows, 16 * row_tiles)) * Hkv;
      const int steps = ceil_div(Nk, kStep);
      keep_logits = weights && rows <= (steps <= 3 * kWaves ? kLogitRowsFewKeys : kLogitRows);
      // One round of work-groups, each with a step per wave at least.  Joining shares is a launch (3.8 us), a step of all
      // waves 1.1 (bf16) to 2 us: up to three of them are not cut, unless the weights need that launch anyway.
      int64_t want = std::min<int64_t>(std::max<int64_t>(1, 256 / tiles), ceil_div(steps, kWaves));
      if (steps <= 3 * kWaves && !keep_logits) want = 1;
      n_splits = ceil_div(steps, ceil_div(steps, static_cast<int>(std::min<int64_t>(want, kMaxShares))));
      if (n_splits > 1) {
        part_o = static_cast<float*>(take(all * n_splits * D * 4));
        part_ml = static_cast<float2*>(take(all * n_splits * 8));
      }
      if (keep_logits) logits = static_cast<float*>(take(all * steps * kStep * 4));
    }
    if (weights) {
      lse = static_cast<float*>(take(all * 4));
      ref = static_cast<float2*>(take(all * 8));
      if (expand) any_far = static_cast<int32_t*>(take(4));
    }
    bytes = at;
  }

 private:
  Q4Plan() = default;
};

int check_kind(int dtype, int D, const char* who) {
  PC_REQUIRE(dtype == PC_F32 || dtype == PC_BF16, PC_ERR_DTYPE, "%s: dtype %d", who, dtype);
  PC_REQUIRE(D == 64 || D == 128, PC_ERR_UNSUPPORTED, "%s: needs D = 64 or 128, got %d", who, D);
  return PC_OK;
}

Q4Rows rows_of(const pc_q4_cache* c) {
  return {c->k_codes, c->k_scales, c->v_codes, c->v_scales, c->code_stride_h, c->scale_stride_h};
}

// Whether the `bytes` of some head of a share one with those of some head of b; strides in bytes, `bytes` at least.
bool heads_overlap(const void* a, int64_t a_stride, const void* b, int64_t b_stride, int H, int64_t bytes) {
  const int64_t gap = static_cast<int64_t>(reinterpret_cast<uintptr_t>(b) - reinterpret_cast<uintptr_t>(a));
  if (gap >= (H - 1) * a_stride + bytes || -gap >= (H - 1) * b_stride + bytes) return false;
  for (int i = 0; i < H; ++i) {      // heads may be interleaved: the two heads of b around head i of a
    const int64_t x = i * a_stride - gap, j = x >= 0 ? x / b_stride : -1;
    if (j >= 0 && j < H && x - j * b_stride < bytes) return true;
    if (j + 1 < H && (j + 1) * b_stride - x < bytes) return true;
  }
  return false;
}

bool aligned16(const void* p, int64_t stride, int dtype) {
  return dtype == PC_F32 ? reinterpret_cast<uintptr_t>(p) % 4 == 0
                         : reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % 8 == 0;
}

}  // namespace
}  // namespace pc

using namespace pc;

extern "C" int pc_q4_store(const void* K, const void* V, int dtype, int H, int n, int D, int64_t k_stride_h,
                           int64_t v_stride_h, const pc_q4_cache* cache, int row0, const int32_t* pos_new, int32_t* pos,
                           int64_t pos_stride_h, float* weights, int64_t weights_stride_h, int Hsel, void* stream) {
  const char* who = "pc_q4_store";
  if (int rc = check_kind(dtype, D, who)) return rc;
  PC_REQUIRE(H > 0 && n >= 0 && row0 >= 0, PC_ERR_SHAPE, "%s: H=%d n=%d row0=%d", who, H, n, row0);
  if (int rc = check_q4_cache(cache, D, who)) return rc;
  if (int rc = check_q4_span(cache, H, row0, n, D, who)) return rc;
  PC_REQUIRE((pos == nullptr) == (pos_new == nullptr), PC_ERR_NULL, "%s: pos and pos_new go together", who);
  const bool book = pos != nullptr || weights != nullptr;
  PC_REQUIRE(!book || (Hsel > 0 && Hsel <= H && H % Hsel == 0), PC_ERR_SHAPE, "%s: Hsel=%d for %d heads", who, Hsel, H);
  const int64_t end = static_cast<int64_t>(row0) + n;
  PC_REQUIRE(!book || Hsel == 1 || ((pos == nullptr || pos_stride_h >= end * 3) && (weights == nullptr || weights_stride_h >= end)),
             PC_ERR_SHAPE, "%s: rows up to %lld do not fit the strides of pos or weights", who, static_cast<long long>(end));
  if (n == 0) return PC_OK;
  PC_REQUIRE(K && V, PC_ERR_NULL, "%s: K or V is NULL", who);
  if (H == 1) k_stride_h = v_stride_h = static_cast<int64_t>(n) * D;      // one head has no stride that matters
  PC_REQUIRE(k_stride_h >= static_cast<int64_t>(n) * D && v_stride_h >= static_cast<int64_t>(n) * D, PC_ERR_SHAPE,
             "%s: a head stride is smaller than rows*D", who);
  PC_REQUIRE(aligned16(K, k_stride_h, dtype) && aligned16(V, v_stride_h, dtype), PC_ERR_SHAPE,
             "%s: bf16 rows and head strides must be 16-byte aligned", who);
  const int64_t units = 2ll * H * n;
  PC_REQUIRE(units <= INT_MAX - kCopyThreads && copy_threads(units, D) <= kMaxThreads, PC_ERR_SHAPE, "%s: %lld rows in one call", who,
             static_cast<long long>(units));
  const int blocks = static_cast<int>(copy_threads(units, D) / kCopyThreads);
  const RowsAt at = {H, D, Divisor(n), k_stride_h, v_stride_h};
  const Book b = {pos_new, pos, weights, pos_stride_h, weights_stride_h, book ? Hsel : 0};
  hipStream_t s = static_cast<hipStream_t>(stream);
  auto go = [&](auto kernel, auto* k, auto* v) {
    kernel<<<blocks, kCopyThreads, 0, s>>>(k, v, at, rows_of(cache), row0, static_cast<int>(units), b);
  };
  if (dtype == PC_BF16) {
    const auto *k = static_cast<const uint16_t*>(K), *v = static_cast<const uint16_t*>(V);
    D == 64 ? go(q4_store_kernel<uint16_t, 64>, k, v) : go(q4_store_kernel<uint16_t, 128>, k, v);
  } else {
    const auto *k = static_cast<const float*>(K), *v = static_cast<const float*>(V);
    D == 64 ? go(q4_store_kernel<float, 64>, k, v) : go(q4_store_kernel<float, 128>, k, v);
  }
  PC_CHECK_LAUNCH(who);
  return PC_OK;
}

namespace {
// clear: a word that is set to 0 as well, or NULL
int load_rows(const pc_q4_cache* cache, int H, int row0, int n, int D, int dtype, void* K, void* V, int64_t k_stride_h,
              int64_t v_stride_h, int32_t* clear, void* stream, const char* who) {
  if (int rc = check_kind(dtype, D, who)) return rc;
  PC_REQUIRE(H > 0 && n >= 0 && row0 >= 0, PC_ERR_SHAPE, "%s: H=%d n=%d row0=%d", who, H, n, row0);
  if (int rc = check_q4_cache(cache, D, who)) return rc;
  if (int rc = check_q4_span(cache, H, row0, n, D, who)) return rc;
  PC_REQUIRE(K || V, PC_ERR_NULL, "%s: K and V are NULL", who);
  if (n == 0) return PC_OK;
  if (H == 1) k_stride_h = v_stride_h = static_cast<int64_t>(n) * D;
  PC_REQUIRE((!K || k_stride_h >= static_cast<int64_t>(n) * D) && (!V || v_stride_h >= static_cast<int64_t>(n) * D), PC_ERR_SHAPE,
             "%s: a head stride is smaller than rows*D", who);
  PC_REQUIRE((!K || aligned16(K, k_stride_h, dtype)) && (!V || aligned16(V, v_stride_h, dtype)), PC_ERR_SHAPE,
             "%s: bf16 rows and head strides must be 16-byte aligned", who);
  const int64_t per = static_cast<int64_t>(H) * n, units = per * ((K != nullptr) + (V != nullptr));
  PC_REQUIRE(2 * per <= INT_MAX - kCopyThreads && copy_threads(units, D) <= kMaxThreads, PC_ERR_SHAPE, "%s: %lld rows in one call", who,
             static_cast<long long>(units));
  const int blocks = static_cast<int>(copy_threads(units, D) / kCopyThreads);
  const RowsAt at = {H, D, Divisor(n), k_stride_h, v_stride_h};
  const int first = K ? 0 : static_cast<int>(per);
  hipStream_t s = static_cast<hipStream_t>(stream);
  auto go = [&](auto kernel, auto* k, auto* v) {
    kernel<<<blocks, kCopyThreads, 0, s>>>(k, v, at, rows_of(cache), row0, first, static_cast<int>(units), clear);
  };
  if (dtype == PC_BF16) {
    auto *k = static_cast<uint16_t*>(K), *v = static_cast<uint16_t*>(V);
    D == 64 ? go(q4_load_kernel<uint16_t, 64>, k, v) : go(q4_load_kernel<uint16_t, 128>, k, v);
  } else {
    auto *k = static_cast<float*>(K), *v = static_cast<float*>(V);
    D == 64 ? go(q4_load_kernel<float, 64>, k, v) : go(q4_load_kernel<float, 128>, k, v);
  }
  PC_CHECK_LAUNCH(who);
  return PC_OK;
}
}  // namespace

extern "C" int pc_q4_load(const pc_q4_cache* cache, int H, int row0, int n, int D, int dtype, void* K, void* V,
                          int64_t k_stride_h, int64_t v_stride_h, void* stream) {
  return load_rows(cache, H, row0, n, D, dtype, K, V, k_stride_h, v_stride_h, nullptr, stream, "pc_q4_load");
}

namespace {
bool sizes_ok(int Hq, int Hkv, int Nq, int Nk) {
  return Hq > 0 && Hkv > 0 && Hq % Hkv == 0 && Nq >= 1 && Nk >= 1 && Nk <= kMaxRows && static_cast<int64_t>(Hq) * Nq <= INT_MAX / 2;
}
}  // namespace

extern "C" size_t pc_q4_attn_workspace_bytes(int dtype, int Hq, int Hkv, int Nq, int Nk, int D, int weights) {
  if (!sizes_ok(Hq, Hkv, Nq, Nk) || (dtype != PC_F32 && dtype != PC_BF16) || (D != 64 && D != 128)) return 0;
  return Q4Plan(dtype, Hq, Hkv, Nq, Nk, D, weights != 0, nullptr).bytes;
}

extern "C" int pc_q4_attn(const void* Q, const pc_q4_cache* cache, int dtype, int Hq, int Hkv, int Nq, int Nk, int D,
                          int64_t q_stride_h, int64_t o_stride_h, float scale, void* O, float* lse, float* weights,
                          int64_t weights_stride_h, int Hsel, float decay, void* ws, size_t ws_bytes, void* stream) {
  const char* who = "pc_q4_attn";
  if (int rc = check_kind(dtype, D, who)) return rc;
  PC_REQUIRE(sizes_ok(Hq, Hkv, Nq, Nk), PC_ERR_SHAPE,
             "%s: Hq=%d must be a positive multiple of Hkv=%d, Nq=%d and Nk=%d at least 1", who, Hq, Hkv, Nq, Nk);
  PC_REQUIRE(scale > 0.f && isfinite(scale), PC_ERR_SHAPE, "%s: scale %g must be > 0", who, scale);
  PC_REQUIRE(Q && O, PC_ERR_NULL, "%s: Q or O is NULL", who);
  if (int rc = check_q4_cache(cache, D, who)) return rc;
  if (int rc = check_q4_span(cache, Hkv, 0, Nk, D, who)) return rc;
  if (Hq == 1) q_stride_h = o_stride_h = static_cast<int64_t>(Nq) * D;    // one head has no stride that matters
  PC_REQUIRE(q_stride_h >= static_cast<int64_t>(Nq) * D && o_stride_h >= static_cast<int64_t>(Nq) * D, PC_ERR_SHAPE,
             "%s: a head stride is smaller than rows*D", who);
  PC_REQUIRE(aligned16(Q, q_stride_h, dtype) && aligned16(O, o_stride_h, dtype), PC_ERR_SHAPE,
             "%s: bf16 tensors and head strides must be 16-byte aligned", who);
  const int elt = dtype == PC_BF16 ? 2 : 4;
  PC_REQUIRE(!heads_overlap(Q, q_stride_h * elt, O, o_stride_h * elt, Hq, static_cast<int64_t>(Nq) * D * elt), PC_ERR_SHAPE,
             "%s: O may not overlap Q: queries are read again behind the first outputs", who);
  if (weights != nullptr) {
    PC_REQUIRE(Hsel == 1 || Hsel == Hkv, PC_ERR_SHAPE, "%s: weights of %d heads for %d KV heads", who, Hsel, Hkv);
    PC_REQUIRE(Hsel == 1 || weights_stride_h >= Nk, PC_ERR_SHAPE, "%s: weights' head stride is smaller than Nk", who);
    PC_REQUIRE(decay >= 0.f && isfinite(decay), PC_ERR_BUDGET, "%s: decay %g", who, decay);
  }
  const int rep = Hq / Hkv, rows = rep * Nq;
  const Q4Plan plan(dtype, Hq, Hkv, Nq, Nk, D, weights != nullptr, ws);
  PC_REQUIRE(plan.bytes == 0 || (ws != nullptr && ws_bytes >= plan.bytes && reinterpret_cast<uintptr_t>(ws) % 16 == 0),
             PC_ERR_WORKSPACE, "%s: needs %zu bytes of 16-byte aligned workspace, got %zu", who, plan.bytes, ws_bytes);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const float c = scale * 1.4426950408889634f;
  if (plan.expand) {
    // rows as they lie in the cache, so that one launch's worth of copying serves every query row
    const int64_t per = static_cast<int64_t>(Nk) * D;
    if (int rc = load_rows(cache, Hkv, 0, Nk, D, PC_BF16, plan.k_rows, plan.v_rows, per, per, plan.any_far, stream, who)) return rc;
    float* e = lse != nullptr ? lse : plan.lse;
    if (int rc = frame_attn(Q, plan.k_rows, plan.v_rows, dtype, Hq, Hkv, Nq, Nk, D, q_stride_h, per, o_stride_h, scale, O, e, plan.ref,
                            plan.attn_ws, plan.attn_bytes, stream))
      return rc;
    if (weights == nullptr) return PC_OK;
    ScoreParts parts;
    if (int rc = score_keys(Q, plan.k_rows, dtype, Hq, Hkv, Nq, Nk, D, q_stride_h, per, nullptr, scale, e, Nq, nullptr, 0, 0, 0, 0,
                            &parts, plan.any_far, plan.attn_ws, plan.attn_bytes, stream))
      return rc;
    int waves = 1;
    while (waves < kWaves && waves < Hkv / Hsel) waves *= 2;
    const WeighArgs w = {rows_of(cache), rep, Nk, Hkv, Hsel, Divisor(Nq), Divisor(ceil_div(Nk, 64)), waves, q_stride_h,
                         weights_stride_h, c, decay, e, plan.ref, weights, parts, plan.any_far};
    q4_weigh_kernel<uint16_t, 128, 4, true><<<w.by_blocks.d * Hsel, 64 * waves, 0, s>>>(static_cast<const uint16_t*>(Q), w);
    PC_CHECK_LAUNCH(who);
    return PC_OK;
  }
  auto run = [&](auto zero, auto dims) -> int {
    using T = decltype(zero);
    constexpr int kDims = decltype(dims)::value;
    const T* q = static_cast<const T*>(Q);
    const int tiles_q = ceil_div(rows, 16 * plan.row_tiles), steps = ceil_div(Nk, kStep);
    // 128 keys per wave of the scoring where that leaves most of the chip's 1,024 SIMDs one; else waves share keys until there
    // are two per SIMD.  Work-groups of few waves where keys are few: the chip has room for them side by side.
    const int64_t wide = static_cast<int64_t>(ceil_div(Nk, 128)) * Hsel, narrow = static_cast<int64_t>(ceil_div(Nk, 64)) * Hsel;
    const int keys = sizeof(T) == 2 && wide >= 448 ? 128 : 64;      // (fp32 queries in three parts leave no registers for it)
    int dealt = 1;
    while (keys == 64 && dealt < kWaves && 16 * dealt < rows && narrow * dealt < 2048) dealt *= 2;
    int groups = 1;           // powers of two: a compute unit holds eight waves of the widest form
    while (groups * dealt < kWaves && (keys == 128 ? wide : narrow) >= 1024 * groups) groups *= 2;
    PC_REQUIRE(static_cast<int64_t>(tiles_q) * Hkv * plan.n_splits * kThreads <= kMaxThreads &&
                   (weights == nullptr || static_cast<int64_t>(ceil_div(Nk, groups * keys)) * Hsel * 64 * groups * dealt <= kMaxThreads),
               PC_ERR_SHAPE, "%s: Hq=%d x Nq=%d rows over Nk=%d keys in one call", who, Hq, Nq, Nk);
    const AttnArgs a = {rows_of(cache), rep, Nk, Divisor(Nq), Divisor(tiles_q), tiles_q * Hkv, ceil_div(steps, plan.n_splits),
                        q_stride_h, o_stride_h, c, plan.part_o, plan.part_ml, lse, plan.lse, plan.ref, plan.logits,
                        static_cast<int64_t>(Hkv) * rows};
    const auto kernel = plan.row_tiles == 1 ? q4_attn_kernel<T, kDims, 1> : q4_attn_kernel<T, kDims, 2>;
    kernel<<<a.n_tiles * plan.n_splits, kThreads, 0, s>>>(q, static_cast<T*>(O), a);
    PC_CHECK_LAUNCH(who);
    const int blocks = ceil_div(Nk, 4 * kJoinThreads);
    const JoinArgs j = {plan.n_splits, rows, Hkv, Hsel, Nk, plan.n_splits > 1 ? static_cast<int>(a.rows_all) : 0, Divisor(blocks),
                        static_cast<int64_t>(steps) * kStep, weights_stride_h, c, decay, weights};
    const int grid = j.row_blocks + (plan.keep_logits ? blocks * Hsel : 0);
    if (grid > 0) {
      q4_join_kernel<T, kDims><<<grid, kJoinThreads, 0, s>>>(static_cast<T*>(O), a, j);
      PC_CHECK_LAUNCH(who);
    }
    if (weights != nullptr && !plan.keep_logits) {
      const WeighArgs w = {rows_of(cache), rep, Nk, Hkv, Hsel, Divisor(Nq), Divisor(ceil_div(Nk, groups * keys)), dealt,
                           q_stride_h, weights_stride_h, c, decay, plan.lse, plan.ref, weights, {}, nullptr};
      auto weigh = q4_weigh_kernel<T, kDims, 4>;
      if constexpr (sizeof(T) == 2)
        if (keys == 128) weigh = q4_weigh_kernel<T, kDims, 8>;
      weigh<<<w.by_blocks.d * Hsel, 64 * groups * dealt, 0, s>>>(q, w);
      PC_CHECK_LAUNCH(who);
    }
    return PC_OK;
  };
  using D64 = std::integral_constant<int, 64>;
  using D128 = std::integral_constant<int, 128>;
  if (dtype == PC_BF16) return D == 64 ? run(uint16_t{}, D64{}) : run(uint16_t{}, D128{});
  return D == 64 ? run(float{}, D64{}) : run(float{}, D128{});
}
