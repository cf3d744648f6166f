// The attention calls on several sequences: which rows a work-group has, what each of them sees, and what becomes of its
// results (gfx950 only).
//
// A work-group has a tile of query rows of one KV head and a range of keys.  The rows of a sequence (or of all of them, over
// the common rows) are numbered rho = i * rep + h through the rep query heads of the KV head, token by token, so that a
// tile holds few tokens and its rows see nearly the same keys.
#pragma once

#include "seq.h"

namespace pc {

constexpr float kNothing = -3.402823466e38f;   // the reference of a row that has seen no key: finite, so that sums merge

struct RowsArgs {
  const void *Q, *K, *V;
  void* O;
  float* lse;
  int64_t q_stride, k_stride, v_stride, o_stride;   // between heads, elements; pages: k_stride = v_stride
  // pages (pc_page_attn)
  const int32_t *table, *lens, *shared;
  int64_t table_stride, page_stride;
  int n_pages, n_shared, max_len;
  Divisor by_page;
  // rows
  int rep, T;                 // T: rows of O and lse
  int row0, n_rows;           // the launch's part of them
  Divisor by_rep, by_hkv;
  SeqTable seqs;
  int fold;                   // pc_prompt_attn: row tiles (of a KV head) that the chip's compute units get first; 0: no second ones
  int max_level;              // pc_prompt_attn, several sequences: above every tile's level
  int tiles_per_seq, n_tiles; // row tiles of one KV head: of a sequence (where all have as many), of all
  Divisor by_tiles_per_seq, by_tiles;
  // shares of the keys
  int n_common;               // work-groups of this launch that have common rows, per KV head
  int shared_tiles, shared_parts, shared_keys;   // row tiles over the common rows; their shares, keys of each
  Divisor by_shared_tiles;
  int own_parts, own_keys;                       // shares of the rows behind them, keys of each
  float* part_o;              // [parts][Hq][T][D], un-normalised; NULL: one share, the result itself
  float2* part_ml;            // [parts][Hq][T]: reference (base 2) and sum
  float c, c_lo;              // scale * log2(e) in two floats
};

// What a work-group has.
struct RowSet {
  int kvh, tile;        // rows tile * R .. of the set
  int t0, n_tok;        // the set's tokens
  int first;            // token i of the set sees keys below first + i; common: unused
  int lo, n_keys;       // keys that exist: lo .. n_keys - 1
  int begin, end;       // the work-group's
  int k0;               // pc_prompt_attn: row of key 0
  const int32_t* pages; // page numbers of the keys
  int part;
  bool common;
  bool idle;            // nothing to do, not even an empty result
};

// The keys that token i of the set sees: those below this (0: none).
__device__ __forceinline__ int limit_of(const RowsArgs& a, const RowSet& r, int i) {
  if (!r.common) return min(max(r.first + i, 0), r.n_keys);
  const int t = r.t0 + i, s = seq_of_row(a.seqs, t);
  if (s < 0) return 0;
  const bool even = a.seqs.per > 0;
  const int end = even ? (s + 1) * a.seqs.per : a.seqs.q0[s] + a.seqs.nq[s];
  const int len = min(a.lens[even ? s : a.seqs.k0[s]], a.max_len);
  return min(max(len - (end - t) + 1, 0), r.n_keys);
}

// pc_prompt_attn: work-groups in the order of what they have to do, longest first (a causal tile's work goes with where
// it ends, and the chip is filled from the front).  A tile's level is the number of row tiles' worth of keys in front of its
// own; tiles of one level follow each other, KV heads fastest, so that with 1, 2, 4, 8 or more heads an XCD's
// work-groups read few of them.  Where two work-groups share a compute unit, the second 256 come shortest first: unit i
// gets number i and number 256 + i, and in plain order the first units would have the longest of both.
template <int R>
__device__ __forceinline__ RowSet prompt_rows(const RowsArgs& a, int block, int lane) {
  RowSet r = {};
  int u = a.by_hkv.of(block);
  r.kvh = block - u * a.by_hkv.d;
  if (u >= a.fold && u < 2 * a.fold) u = min(2 * a.fold, a.n_tiles) - 1 - (u - a.fold);
  int s = 0;
  if (a.seqs.n == 1) {
    r.tile = a.n_tiles - 1 - u;
  } else {
    const int nq = lane < a.seqs.n ? a.seqs.nq[lane] : 0, nk = lane < a.seqs.n ? a.seqs.nk[lane] : 0;
    const int tiles = (nq * a.rep + R - 1) / R;
    const int base = nk > nq ? static_cast<int>(static_cast<int64_t>(nk - nq) * a.rep / R) : 0;
    auto above = [&](int x) {   // tiles of level x or more
      return __builtin_amdgcn_readlane(wave_prefix_sum(min(max(base + tiles - x, 0), tiles)), 63);
    };
    int at = 0, top = a.max_level;   // above(at) > u >= above(top)
    while (top - at > 1) {
      const int mid = (at + top) >> 1;
      if (above(mid) > u) at = mid;
      else top = mid;
    }
    const int rank = u - above(at + 1);
    const bool mine = at >= base && at < base + tiles;
    const uint64_t those = __ballot(mine && lanes_below(__ballot(mine), 0) == rank);
    s = __builtin_ctzll(those);
    r.tile = at - __builtin_amdgcn_readlane(base, s);
  }
  s = __builtin_amdgcn_readfirstlane(s);
  r.t0 = a.seqs.q0[s], r.n_tok = a.seqs.nq[s], r.k0 = a.seqs.k0[s];
  r.n_keys = a.seqs.nk[s], r.first = r.n_keys - r.n_tok + 1;
  r.end = r.n_keys;
  return r;
}

// pc_page_attn: first the work-groups over the common rows, then those over each sequence's own, shares slowest.
template <int R>
__device__ __forceinline__ RowSet page_rows(const RowsArgs& a, int block, int lane) {
  RowSet r = {};
  int u = a.by_hkv.of(block);
  r.kvh = block - u * a.by_hkv.d;
  if (u < a.n_common) {
    r.common = true;
    r.part = a.by_shared_tiles.of(u);
    r.tile = u - r.part * a.shared_tiles;
    r.t0 = a.row0, r.n_tok = a.n_rows;
    r.n_keys = a.n_shared;
    r.begin = r.part * a.shared_keys, r.end = min(r.begin + a.shared_keys, a.n_shared);
    r.pages = a.shared;
    return r;
  }
  u -= a.n_common;
  const int share = a.by_tiles.of(u);
  u -= share * a.n_tiles;
  int number, nq;
  if (a.seqs.per > 0) {
    number = a.by_tiles_per_seq.of(u);
    r.tile = u - number * a.tiles_per_seq;
    nq = a.seqs.per, r.t0 = number * nq;
  } else {
    const int tiles = lane < a.seqs.n ? (a.seqs.nq[lane] * a.rep + R - 1) / R : 0;
    const int upto = wave_prefix_sum(tiles);
    const int s = __builtin_ctzll(__ballot(upto > u));
    r.tile = u - (__builtin_amdgcn_readlane(upto, s) - __builtin_amdgcn_readlane(tiles, s));
    number = a.seqs.k0[s], nq = a.seqs.nq[s], r.t0 = a.seqs.q0[s];
  }
  r.n_tok = nq;
  const int len = min(a.lens[number], a.max_len);
  r.pages = a.table + number * a.table_stride;
  r.lo = a.n_shared, r.n_keys = max(len, 0), r.first = len - nq + 1;
  const int from = a.n_shared / kPageStep * kPageStep;
  r.begin = from + share * a.own_keys, r.end = min(r.begin + a.own_keys, r.n_keys);
  r.part = a.shared_parts + share;
  // a result of nothing is written only where nobody else writes the row
  if (len <= a.n_shared || r.begin >= r.n_keys) r.end = r.begin, r.idle = a.part_o != nullptr;
  return r;
}

// How many of the shares over a sequence's own rows have written something: those in front of its end.
__device__ __forceinline__ int own_parts_of(const RowsArgs& a, int len) {
  if (len <= a.n_shared) return 0;
  const int n = len - a.n_shared / kPageStep * kPageStep;
  return (n + a.own_keys - 1) / a.own_keys;
}

__device__ __forceinline__ bool not_finite(float v) { return (__float_as_uint(v) & 0x7F800000u) == 0x7F800000u; }

// ln(2^m l), rounded once: m may reach hundreds where l's logarithm is small
__device__ __forceinline__ float lse_of(float m, float l) {
  return l == 0.f ? -INFINITY : fmaf(m, 0.693147182464599609375f, fmaf(m, -1.90465429995776804525e-9f, logf(l)));
}

}  // namespace pc
