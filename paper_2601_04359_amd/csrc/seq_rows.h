// The attention calls on several sequences: which rows a work-group has, what each of them sees, and what becomes of its
// results (gfx950 only).
//
// A work-group has a tile of query rows of one KV head and a range of keys.  The rows of a sequence (or of all of them, over
// the common rows) are numbered rho = i * rep + h through the rep query heads of the KV head, token by token, so that a
// tile holds few tokens and its rows see nearly the same keys.
#pragma once

#include "seq.h"

namespace pc {

typedef __attribute__((address_space(3))) int lds_int;

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
  int row0, n_rows;           // the launch's part of them (one number of rows each: row0 = 0, tensors and tables begin there)
  Divisor by_rep, by_hkv;
  SeqTable seqs;
  int n_heavy;                // pc_prompt_attn: tiles of 128 rows (of a KV head), the longest, that are two work-groups' of 64
  int max_level;              // pc_prompt_attn, several sequences: above every tile's level
  int n_tiles;                // pc_prompt_attn: row tiles of one KV head
  // pc_page_attn: units of work per KV head, and where their results go
  int shared_tiles, shared_parts, shared_keys;   // row tiles over the common rows; their shares, keys of each
  Divisor by_shared_tiles, by_rest;   // by_rest: shares of all heads that eight do not divide
  int tiles_per_seq;          // row tiles of a sequence, where all have as many
  int own_parts, own_keys;    // > 0: shares of the own rows as the host has cut them; 0: the device does
  Divisor by_parts;
  int own_cap;                // units over the sequences' own rows at most
  float unit_us, key_us;      // what a unit and a key of its own rows cost a work-group
  int least_keys;             // of a share
  int slots;                  // work-groups that the chip takes at once
  int slot_rows;              // rows of a slot
  Divisor by_tile;            // rows of a tile
  float* part_o;              // [Hkv][n_common + own_cap][slot_rows][D], un-normalised; NULL: one share, the result itself
  float2* part_ml;            // [Hkv][..][slot_rows]: reference (base 2) and sum
  int* cut;                   // [1 + n_seq]: keys of a share of the own rows, the first unit of each sequence's
  float c, c_lo;              // scale * log2(e) in two floats, c_lo > 0 (fp32; bf16: c alone)
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
  int slot;             // where the result goes, if it is a share's
  bool common;
};

// Rows of sequence s of the launch; lens may hold anything.
__device__ __forceinline__ int len_of(const RowsArgs& a, int s) {
  return max(0, min(a.lens[a.seqs.per > 0 ? s : a.seqs.k0[s]], a.max_len));
}

// The keys that token i of the set sees: those below this (0: none).
__device__ __forceinline__ int limit_of(const RowsArgs& a, const RowSet& r, int i) {
  if (!r.common) return min(max(r.first + i, 0), r.n_keys);
  const int t = r.t0 + i, s = seq_of_row(a.seqs, t);
  if (s < 0) return 0;
  const bool even = a.seqs.per > 0;
  const int end = even ? (s + 1) * a.seqs.per : a.seqs.q0[s] + a.seqs.nq[s];
  return min(max(len_of(a, s) - (end - t) + 1, 0), r.n_keys);
}

// Whether any of keys from .. upto - 1 has a page.  Asked of rows whose weights add up to 0: they have seen nothing if none has (O = 0),
// and otherwise scores of -inf alone, which are no numbers.
__device__ __forceinline__ bool any_page(const RowsArgs& a, const int32_t* pages, int from, int upto) {
  for (int p = a.by_page.of(from), last = a.by_page.of(upto - 1); from < upto && p <= last; ++p)
    if (static_cast<uint32_t>(pages[p]) < static_cast<uint32_t>(a.n_pages)) return true;
  return false;
}
// The same of a row's limit in its set; prompts have no pages, and all of their keys.
__device__ __forceinline__ bool sees_none(const RowsArgs& a, const RowSet& r, int lim, float sum) {
  return lim <= r.lo || (r.pages != nullptr && sum == 0.f && !any_page(a, r.pages, r.lo, lim));
}

// pc_prompt_attn: work-groups in the order of what they have to do, longest first (a causal tile's work goes with where
// it ends, and the chip is filled from the front).  A tile's level is the number of row tiles' worth of keys in front of its
// own; tiles of one level follow each other, KV heads fastest, so that with 1, 2, 4, 8 or more heads an XCD's
// work-groups read few of them.
// (beyond 2^29 rows' worth the order no longer matters, and levels stay numbers of 32 bits)
__host__ __device__ inline int level_of(int nq, int nk, int rep, int rows) {
  const int64_t level = nk > nq ? static_cast<int64_t>(nk - nq) * rep / rows : 0;
  return static_cast<int>(level < (1 << 29) ? level : 1 << 29);
}
template <int R>
__device__ __forceinline__ RowSet prompt_rows(const RowsArgs& a, int u, int kvh, int lane) {   // tile u of a KV head
  RowSet r = {};
  r.kvh = kvh;
  int s = 0;
  if (a.seqs.n == 1) {
    r.tile = a.n_tiles - 1 - u;
  } else {
    const int nq = lane < a.seqs.n ? a.seqs.nq[lane] : 0, nk = lane < a.seqs.n ? a.seqs.nk[lane] : 0;
    const int tiles = (nq * a.rep + R - 1) / R;
    const int base = level_of(nq, nk, a.rep, R);
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

// pc_page_attn.  The lengths are known on the device only, and sequences may be of any lengths beside each other, so that every
// work-group cuts the work for itself, all alike: shares of `keys` keys of every sequence, and the units (sequence, share, row tile)
// numbered through.  plan_pages finds the length of a share among ten, from a third of what a work-group would have if all
// had the same up to three times that: the one with the shortest rounds of units (of equals the longest).  Mostly that is the
// one whose units just go into one round: 24/8 heads, 16 sequences of 1 to 27,575 keys (251 us of a copy), shares of 1, 1.4, 2 and
// 2.8 times the even one 266, 219, 247 and 295 us.  It is work of one wave, on sums over lanes.
constexpr int kPageSeqs = 256;                 // sequences of a launch at most, four per lane
struct PageUnits {
  int keys, total;    // keys of a share, units over own rows
  lds_int* first;     // [kPageSeqs]: units in front of each sequence; then their lengths
};
__device__ __forceinline__ int ceil_of(int x, int by, float inv) {   // ceil(x / by), 0 <= x < 2^30
  const int n = x + by - 1;
  int q = static_cast<int>(static_cast<float>(n) * inv);
  if (q * by > n) --q;
  else if (n - q * by >= by) ++q;
  return q;
}
// Keys of a sequence from where its own rows begin, whole steps.
__device__ __forceinline__ int own_keys_of(const RowsArgs& a, int len) {
  return len > a.n_shared ? len - a.n_shared / kPageStep * kPageStep : 0;
}
__device__ __forceinline__ int n_common(const RowsArgs& a) { return a.shared_tiles * a.shared_parts; }

__device__ __forceinline__ int wave_total(int x) { return __builtin_amdgcn_readlane(wave_prefix_sum(x), 63); }

template <int R, int kPer>   // sequences per lane
__device__ __forceinline__ void cut_pages(const RowsArgs& a, lds_int* plan, int lane) {
  int keys[kPer], tiles[kPer], lens[kPer], longest = 0, total = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int s = i * 64 + lane;
    const bool there = s < a.seqs.n;
    tiles[i] = !there ? 0 : a.seqs.per > 0 ? a.tiles_per_seq : (a.seqs.nq[s & (kSeqs - 1)] * a.rep + R - 1) / R;
    lens[i] = there ? len_of(a, s) : 0;
    keys[i] = tiles[i] > 0 ? own_keys_of(a, lens[i]) : 0;
    longest = max(longest, keys[i]);
    total += (keys[i] + kPageStep - 1) / kPageStep * tiles[i];   // (per steps of 64 keys)
  }
  longest = __builtin_amdgcn_readlane(wave_scan(longest, 0, [](int x, int y) { return max(x, y); }), 63);
  total = wave_total(total);
  const int whole = (max(longest, 1) + kPageStep - 1) / kPageStep * kPageStep;
  int best = whole;
  if (a.part_o != nullptr) {
    constexpr int kTries = 10;
    constexpr float kOf[kTries] = {0.35f, 0.5f, 0.7f, 1.f, 1.15f, 1.3f, 1.45f, 1.7f, 2.f, 2.8f};
    const float even = static_cast<float>(total) * kPageStep * a.by_hkv.d / a.slots;
    int share[kTries], units[kTries];
#pragma unroll
    for (int t = 0; t < kTries; ++t) {
      share[t] = min(max((static_cast<int>(even * kOf[t]) + kPageStep - 1) / kPageStep * kPageStep, a.least_keys), whole);
      units[t] = 0;
#pragma unroll
      for (int i = 0; i < kPer; ++i) units[t] += tiles[i] * ceil_of(keys[i], share[t], 1.f / share[t]);
    }
#pragma unroll
    for (int t = 0; t < kTries; ++t) units[t] = wave_total(units[t]);
    float best_us = 3e38f;
#pragma unroll
    for (int t = 0; t < kTries; ++t) {
      const float rounds = ceilf(static_cast<float>(units[t] + n_common(a)) * a.by_hkv.d / a.slots);
      const float us = rounds * (a.unit_us + a.key_us * share[t]);
      if (units[t] <= a.own_cap && us <= best_us) best_us = us, best = share[t];    // (whole sequences always fit)
    }
  }
  const float inv = 1.f / best;
  int base = 0;
#pragma unroll
  for (int i = 0; i < kPageSeqs / 64; ++i) {
    if (i < kPer) {
      const int units = tiles[i % kPer] * (a.part_o != nullptr ? ceil_of(keys[i % kPer], best, inv) : 1), upto = wave_prefix_sum(units);
      plan[i * 64 + lane] = base + upto - units;
      plan[kPageSeqs + 2 + i * 64 + lane] = lens[i % kPer];
      if (blockIdx.x == 0 && a.part_o != nullptr && i * 64 + lane < a.seqs.n) a.cut[1 + i * 64 + lane] = base + upto - units;
      base += __builtin_amdgcn_readlane(upto, 63);
    }
  }
  if (lane == 0) {
    plan[kPageSeqs] = best, plan[kPageSeqs + 1] = base;
    if (blockIdx.x == 0 && a.part_o != nullptr) a.cut[0] = best;
  }
}
template <int R>
__device__ __forceinline__ PageUnits plan_pages(const RowsArgs& a, lds_int* plan, int wave, int lane) {
  if (a.own_parts > 0) return {a.own_keys, a.own_cap, plan};
  if (wave == 0) {
    if (a.seqs.n <= 64) cut_pages<R, 1>(a, plan, lane);
    else cut_pages<R, kPageSeqs / 64>(a, plan, lane);
  }
  __syncthreads();
  return {__builtin_amdgcn_readfirstlane(plan[kPageSeqs]), __builtin_amdgcn_readfirstlane(plan[kPageSeqs + 1]), plan};
}
constexpr int kPlanBytes = (2 * kPageSeqs + 2) * 4;

// Unit `unit` of the launch, first those over the common rows; false: there are no more.  The row tiles over one share of a KV
// head's common rows read the same keys: they are dealt to one XCD (work-groups go to the eight in turn), so that its L2 reads
// them from memory once.  What does not go into eights, and the units over own rows, come with KV heads fastest.
template <int R>
__device__ __forceinline__ bool page_rows(const RowsArgs& a, const PageUnits& units, int unit, int lane, RowSet& r) {
  const int common = n_common(a), shares = a.by_hkv.d * a.shared_parts;
  r = {};
  if (unit < common * a.by_hkv.d) {
    const int in_eights = shares & ~7, rest = unit - in_eights * a.shared_tiles;
    int at;
    if (rest < 0) {
      const int i = unit >> 3, round = a.by_shared_tiles.of(i);
      r.tile = i - round * a.shared_tiles, at = round * 8 + (unit & 7);
    } else {
      r.tile = a.by_rest.of(rest), at = in_eights + rest - r.tile * a.by_rest.d;
    }
    const int share = a.by_hkv.of(at);
    r.kvh = at - share * a.by_hkv.d;
    r.slot = r.kvh * (common + a.own_cap) + share * a.shared_tiles + r.tile;
    r.common = true;
    r.t0 = a.row0, r.n_tok = a.n_rows;
    r.n_keys = a.n_shared;
    r.begin = share * a.shared_keys, r.end = min(r.begin + a.shared_keys, a.n_shared);
    r.pages = a.shared;
    return true;
  }
  unit -= common * a.by_hkv.d;
  int u = a.by_hkv.of(unit);
  r.kvh = unit - u * a.by_hkv.d;
  if (u >= units.total) return false;
  r.slot = r.kvh * (common + a.own_cap) + common + u;
  int s, tiles = a.tiles_per_seq, share = 0;
  if (a.own_parts > 0 && a.seqs.per > 0) {
    s = a.by_parts.of(u);     // (units of a sequence: its tiles times the shares)
    u -= s * a.by_parts.d;
  } else {
    s = -1;                   // the last sequence that begins at or in front of u
    if (a.own_parts > 0) {    // from a table's rows (64 sequences at most)
      const int units = lane < a.seqs.n ? (a.seqs.nq[lane] * a.rep + R - 1) / R * a.own_parts : 0, first = wave_prefix_sum(units) - units;
      s = __popcll(__ballot(lane < a.seqs.n && first <= u)) - 1;
      u -= __builtin_amdgcn_readlane(first, s);
    } else {
#pragma unroll
      for (int i = 0; i < kPageSeqs / 64; ++i)
        if (i * 64 < a.seqs.n) s += __popcll(__ballot(i * 64 + lane < a.seqs.n && units.first[i * 64 + lane] <= u));
      s = __builtin_amdgcn_readfirstlane(s);
      u -= __builtin_amdgcn_readfirstlane(units.first[s]);
    }
  }
  int number = s;
  if (a.seqs.per > 0) {
    r.n_tok = a.seqs.per, r.t0 = s * r.n_tok;
  } else {
    number = a.seqs.k0[s], r.n_tok = a.seqs.nq[s], r.t0 = a.seqs.q0[s];
    tiles = (r.n_tok * a.rep + R - 1) / R;
  }
  for (r.tile = u; r.tile >= tiles; r.tile -= tiles) ++share;
  const int len = a.own_parts > 0 ? len_of(a, s) : units.first[kPageSeqs + 2 + s];
  r.pages = a.table + number * a.table_stride;
  r.lo = a.n_shared, r.n_keys = len, r.first = len - r.n_tok + 1;
  r.begin = a.n_shared / kPageStep * kPageStep + share * units.keys;
  r.end = min(r.begin + units.keys, r.n_keys);
  if (len <= a.n_shared || r.end < r.begin) r.end = r.begin;
  // behind the sequence's end: an empty result is written only where nobody else writes the row
  return r.begin < r.end || a.part_o == nullptr;
}

// A work-group has one tile of a prompt, or one unit of pages; those behind the last unit end at once (a loop over units took
// 100 registers more, spilled).
template <int R, bool kPages, class Body>
__device__ __forceinline__ void each_unit(const RowsArgs& a, lds_int* plan, Body&& body) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if constexpr (!kPages) {
    const int u = a.by_hkv.of(blockIdx.x);
    body(prompt_rows<R>(a, u, blockIdx.x - u * a.by_hkv.d, lane));
  } else {
    const PageUnits units = plan_pages<R>(a, plan, wave, lane);
    RowSet r;
    if (!page_rows<R>(a, units, blockIdx.x, lane, r)) return;
    // the same in every lane, and in scalar registers: the compiler does not see it of what has gone through LDS
    for (int* v : {&r.kvh, &r.tile, &r.t0, &r.n_tok, &r.first, &r.lo, &r.n_keys, &r.begin, &r.end, &r.slot})
      *v = __builtin_amdgcn_readfirstlane(*v);
    const uint64_t at = reinterpret_cast<uint64_t>(r.pages);
    const uint32_t low = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(at)),
                   high = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(at >> 32));
    r.pages = reinterpret_cast<const int32_t*>(static_cast<uint64_t>(high) << 32 | low);
    body(r);
  }
}

// All ones for a number that is not finite, else 0: an exponent of ones carries into the sign.  (By whole words, so that no
// comparison takes a pair of scalar registers of its own.)
__device__ __forceinline__ uint32_t odd_mask(float v) {
  return static_cast<uint32_t>(static_cast<int32_t>((__float_as_uint(v) & 0x7F800000u) + 0x00800000u) >> 31);
}

// ln(2^m l), rounded once: m may reach hundreds where l's logarithm is small
__device__ __forceinline__ float lse_of(float m, float l) {
  return l == 0.f ? -INFINITY : fmaf(m, 0.693147182464599609375f, fmaf(m, -1.90465429995776804525e-9f, logf(l)));
}

}  // namespace pc
