// Eviction from a cache by accumulated attention weight, in place.
//
// Softmax attention does not depend on the order of its keys, and a cached row carries its own coordinates, so
// the rows that stay need no order either: an evicted row below n_keep is a hole, a kept row from n_keep on moves
// into one (holes and movers both ascending, so the result is a function of the inputs alone).  Sources lie at or
// above n_keep and destinations below it: the moves are in place without any order between them, and at
// most min(Nk - n_keep, n_keep) rows move where closing the gaps would move nearly all of them.
#include <limits.h>

#include <algorithm>

#include "q4.h"

namespace pc {
namespace {

constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / 64;
constexpr int kSlice = 4096, kMaxSlices = 512, kItemsOfSlice = kSlice / kSelThreads;     // of rows beyond one work-group's
constexpr int kTopBits = 11, kTopBins = 1 << kTopBits;     // of a rank, looked at first

struct Ranks {
  const float* weights;
  const int32_t* pos;        // NULL: no row is recent
  int64_t w_stride_h, pos_stride_h;
  int Nk, n_keep, n_anchor, recent_t;
};

// A weight as an integer of the same order: NaN below everything, -0 and 0 alike.
__device__ __forceinline__ uint32_t weight_rank(float w) {
  const uint32_t u = __float_as_uint(w + 0.f);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// One selection head's rows: anchors and recent rows rank above every weight.  What a row's rank is made of is
// fetched apart from the arithmetic, so that a thread has all its rows' loads in flight.
struct HeadRanks {
  const float* w;
  const int32_t* t;
  const int32_t* last;
  int n_anchor, recent_t;
  struct Row {
    float w;
    int32_t t;
  };
  __device__ HeadRanks(const Ranks& a, int sel)
      : w(a.weights + sel * a.w_stride_h), t(a.recent_t > 0 ? a.pos + sel * a.pos_stride_h : nullptr),
        last(t == nullptr ? nullptr : t + static_cast<int64_t>(a.Nk - 1) * 3), n_anchor(a.n_anchor), recent_t(a.recent_t) {}
  __device__ __forceinline__ Row fetch(int j) const { return {w[j], t == nullptr ? 0 : t[static_cast<int64_t>(j) * 3]}; }
  // the t above which a row is recent
  __device__ __forceinline__ int64_t border() const { return t == nullptr ? INT_MAX : static_cast<int64_t>(*last) - recent_t; }
  __device__ __forceinline__ uint32_t rank(const Row& row, int j, int64_t border) const {
    return j < n_anchor || row.t > border ? 0xffffffffu : weight_rank(row.w);
  }
};

// Counters of the top bits in four copies, a lane's by its number: weights crowd into few bins (a factor of two
// is four of them), and lanes of a wave that count in one bin take turns.
constexpr int kCopies = 4;
__device__ __forceinline__ void count_top(int* hist, uint32_t key) {
  atomicAdd(&hist[(key >> (32 - kTopBits)) * kCopies + (threadIdx.x & (kCopies - 1))], 1);
}
__device__ __forceinline__ int counted_top(const int* hist, int bin) {
  const u32x4 c = *reinterpret_cast<const u32x4*>(hist + bin * kCopies);
  return static_cast<int>(c[0] + c[1] + c[2] + c[3]);
}

// Sum of the first n waves' words, in every lane of the wave; s: a word per wave, n <= kSelWaves.
__device__ __forceinline__ int before_wave(const int* s, int n) {
  const int lane = threadIdx.x & 63;
  const int upto = wave_prefix_sum(lane < kSelWaves ? s[lane] : 0);
  return n == 0 ? 0 : __builtin_amdgcn_readlane(upto, n - 1);
}

// Where the left-th row from the top lies among kBins counted bins: s_found = (bin, rows still wanted of it, rows in it).
// Every thread calls it, between barriers; s_wave: a word per wave.
template <int kBins, class Count>
__device__ __forceinline__ void find_bin(Count&& count, int left, int* s_wave, int* s_found) {
  constexpr int kPer = kBins > kSelThreads ? kBins / kSelThreads : 1;
  constexpr int kUsed = kBins / kPer;            // threads with bins, from the top bin down
  static_assert(kUsed % 64 == 0 && kUsed <= kSelThreads, "whole waves");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int c[kPer], sum = 0;
  const bool mine = threadIdx.x < kUsed;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    c[k] = mine ? count(kBins - 1 - (static_cast<int>(threadIdx.x) * kPer + k)) : 0;
    sum += c[k];
  }
  const int upto = wave_prefix_sum(sum);
  if (mine && lane == 63) s_wave[wave] = upto;
  __syncthreads();
  if (mine) {
    int at = upto - sum + before_wave(s_wave, wave);
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      if (at < left && left <= at + c[k]) {
        s_found[0] = kBins - 1 - (static_cast<int>(threadIdx.x) * kPer + k);
        s_found[1] = left - at;
        s_found[2] = c[k];
      }
      at += c[k];
    }
  }
  __syncthreads();
}

// ------------------------------------------------------------------------------------------
// What moves: rows of whole 16-byte pieces of every head, and the small things beside them.
// ------------------------------------------------------------------------------------------
struct Moves {
  u32x4* rows[2];              // K and V, or their codes
  int64_t row_stride_h[2];     // in 16-byte pieces
  Divisor by_pieces, by_both;  // pieces of a row of one of them, and of both
  uint8_t* scales[2];          // of a 4-bit cache, else NULL
  int64_t scale_stride_h;
  int scale_bytes;             // of a row: 2 or 4
  int32_t* pos;                // of a selection head, may be NULL
  float* weights;
  int64_t pos_stride_h, w_stride_h;
  int32_t* idx;                // may be NULL
  int64_t idx_stride_h;
  int per;                     // heads of a selection head
};

// Units first, first + step, ... of the 16-byte pieces of head h's n moved rows, four loads in flight per thread
__device__ __forceinline__ void move_rows(const Moves& m, int h, int n, const int32_t* __restrict__ holes,
                                          const int32_t* __restrict__ movers, int first, int step) {
  const int n_units = n * m.by_both.d, pieces = m.by_pieces.d;
  for (int u0 = first; u0 < n_units; u0 += 4 * step) {
    u32x4 v[4];
    u32x4* to[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int u = u0 + k * step;
      if (u >= n_units) continue;
      const int i = m.by_both.of(u);
      const int both = u - i * m.by_both.d, second = both >= pieces;
      u32x4* base = m.rows[second] + h * m.row_stride_h[second] + (both - second * pieces);
      to[k] = base + static_cast<int64_t>(holes[i]) * pieces;
      v[k] = base[static_cast<int64_t>(movers[i]) * pieces];
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (u0 + k * step < n_units) *to[k] = v[k];
  }
}

// The small things of moved rows first, first + step, ...; the selection head's own with its first head
__device__ __forceinline__ void move_book(const Moves& m, int h, int sel, int n, const int32_t* __restrict__ holes,
                                          const int32_t* __restrict__ movers, int first, int step) {
  const bool own = h == sel * m.per;
  for (int i = first; i < n; i += step) {
    const int64_t to = holes[i], from = movers[i];
    if (m.scales[0] != nullptr)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        uint8_t* base = m.scales[k] + h * m.scale_stride_h;
        if (m.scale_bytes == 4) reinterpret_cast<uint32_t*>(base)[to] = reinterpret_cast<uint32_t*>(base)[from];
        else reinterpret_cast<uint16_t*>(base)[to] = reinterpret_cast<uint16_t*>(base)[from];
      }
    if (!own) continue;
    float* w = m.weights + sel * m.w_stride_h;
    const float was = w[from];
    if (m.pos != nullptr) {
      int32_t* p = m.pos + sel * m.pos_stride_h;
      const int32_t a = p[from * 3], b = p[from * 3 + 1], c = p[from * 3 + 2];
      p[to * 3] = a, p[to * 3 + 1] = b, p[to * 3 + 2] = c;
    }
    w[to] = was;
    if (m.idx != nullptr) m.idx[sel * m.idx_stride_h + to] = static_cast<int32_t>(from);
  }
}

__global__ __launch_bounds__(256) void evict_move_kernel(Moves m, int book_blocks, int room, const int32_t* __restrict__ counts,
                                                         const int32_t* __restrict__ lists) {
  const int h = blockIdx.y, sel = h / m.per, n = counts[sel];
  const int32_t* holes = lists + static_cast<int64_t>(sel) * 2 * room;
  const int block = static_cast<int>(blockIdx.x) - book_blocks;
  if (block < 0)
    move_book(m, h, sel, n, holes, holes + room, blockIdx.x * 256 + threadIdx.x, book_blocks * 256);
  else
    move_rows(m, h, n, holes, holes + room, block * 256 + threadIdx.x, (gridDim.x - book_blocks) * 256);
}

// ------------------------------------------------------------------------------------------
// Up to 24 x 1,024 rows: a work-group per selection head, the ranks in registers (wave w owns 64 kItems
// rows in a row, so that list places are a ballot per 64 of them and one sum over the waves).  The n_keep-th rank is
// found from the top bits down, 11, 11 and 10 at a time, in LDS counters; a step whose bin is wanted whole ends it.
// With `move` the same work-group moves the rows: a second launch costs more than it takes for few.
// Bound: latency, a chain of barriers behind one fetch.
// ------------------------------------------------------------------------------------------
template <int kItems>
__global__ __launch_bounds__(kSelThreads) void evict_select_kernel(Ranks a, int room, int32_t* __restrict__ counts,
                                                                   int32_t* __restrict__ lists, Moves m, int move) {
  __shared__ __align__(16) int hist[kTopBins * kCopies + 2048 + 1024];
  __shared__ int s_wave[3][kSelWaves], s_found[3];
  const int sel = blockIdx.x, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const HeadRanks head(a, sel);
  const int first = wave * 64 * kItems, j0 = first + lane;
  HeadRanks::Row row[kItems];
#pragma unroll
  for (int i = 0; i < kItems; ++i) row[i] = head.fetch(min(j0 + i * 64, a.Nk - 1));
  const int64_t border = head.border();
  for (int b = threadIdx.x * 4; b < kTopBins * kCopies + 2048 + 1024; b += kSelThreads * 4)
    *reinterpret_cast<u32x4*>(hist + b) = u32x4{0, 0, 0, 0};
  __syncthreads();
  uint32_t key[kItems];
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    key[i] = head.rank(row[i], j0 + i * 64, border);
    if (j0 + i * 64 < a.Nk) count_top(hist, key[i]);
  }
  __syncthreads();
  uint32_t prefix = 0;
  int left = a.n_keep, shift = 32 - kTopBits;
  bool whole = false;
  find_bin<kTopBins>([&](int b) { return counted_top(hist, b); }, left, s_wave[0], s_found);
  for (;;) {
    prefix |= static_cast<uint32_t>(s_found[0]) << shift;
    left = s_found[1];
    whole = s_found[2] == left;
    if (whole || shift == 0) break;
    const int upper = shift;
    shift = upper == 21 ? 10 : 0;
    int* h = hist + kTopBins * kCopies + (upper == 21 ? 0 : 2048);
#pragma unroll
    for (int i = 0; i < kItems; ++i)
      if (j0 + i * 64 < a.Nk && (key[i] ^ prefix) >> upper == 0) atomicAdd(&h[key[i] >> shift & ((1 << (upper - shift)) - 1)], 1);
    __syncthreads();
    if (upper == 21) find_bin<2048>([&](int b) { return h[b]; }, left, s_wave[0], s_found);
    else find_bin<1024>([&](int b) { return h[b]; }, left, s_wave[0], s_found);
  }
  // rows above the threshold stay; of those at it (not whole: several of one weight, left of them wanted) the first ones
  int ties_before = 0;
  if (!whole) {
    int mine = 0;
#pragma unroll
    for (int i = 0; i < kItems; ++i) mine += __popcll(__ballot(j0 + i * 64 < a.Nk && key[i] == prefix));
    if (lane == 0) s_wave[0][wave] = mine;
    __syncthreads();
    ties_before = before_wave(s_wave[0], wave);
  }
  uint32_t leaves = 0;         // a bit per row of the lane
  int n_holes = 0, n_movers = 0;
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    if (first + i * 64 >= a.Nk) break;
    const int j = j0 + i * 64;
    bool stays = key[i] > prefix || (whole && key[i] == prefix);
    if (!whole) {
      const bool tie = j < a.Nk && key[i] == prefix;
      const uint64_t tied = __ballot(tie);
      if (tied != 0) {
        stays |= tie && lanes_below(tied, ties_before) < left;
        ties_before += __popcll(tied);
      }
    }
    if (!stays) leaves |= 1u << i;
    if (first + i * 64 < a.n_keep) n_holes += __popcll(__ballot(!stays && j < a.n_keep));
    if (first + i * 64 + 63 >= a.n_keep) n_movers += __popcll(__ballot(stays && j >= a.n_keep && j < a.Nk));
    if (m.idx != nullptr && stays && j < a.n_keep) m.idx[sel * m.idx_stride_h + j] = j;
  }
  if (lane == 0) s_wave[1][wave] = n_holes, s_wave[2][wave] = n_movers;
  __syncthreads();
  int at_h = before_wave(s_wave[1], wave), at_m = before_wave(s_wave[2], wave);
  const int n = before_wave(s_wave[1], kSelWaves);
  int32_t* holes = lists + static_cast<int64_t>(sel) * 2 * room;
  int32_t* movers = holes + room;
  if (n_holes + n_movers > 0) {
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int j = j0 + i * 64;
      const bool gone = leaves >> i & 1;
      const bool hole = gone && j < a.n_keep, mover = !gone && j >= a.n_keep && j < a.Nk;
      const uint64_t bh = __ballot(hole), bm = __ballot(mover);
      if (hole) holes[lanes_below(bh, at_h)] = j;
      if (mover) movers[lanes_below(bm, at_m)] = j;
      at_h += __popcll(bh), at_m += __popcll(bm);
    }
  }
  if (!move) {
    if (threadIdx.x == 0) counts[sel] = n;
    return;
  }
  __threadfence_block();
  __syncthreads();
  for (int h = sel * m.per; h < (sel + 1) * m.per; ++h) {
    move_rows(m, h, n, holes, movers, threadIdx.x, kSelThreads);
    move_book(m, h, sel, n, holes, movers, threadIdx.x, kSelThreads);
  }
}

// ------------------------------------------------------------------------------------------
// Few rows leave (a cache at its budget that takes a token or a few per step): they are found one after another as
// the least of all, at one barrier each (0.56 us; 1.2 in two launches), where a threshold takes three counted passes:
// 4 heads losing one of 3,000 rows 8.1 -> 4.8 us, of 24,000 28 -> 8.1, of 193,792 50 -> 12.1; 112 heads one of 8,321 17.9 -> 13.2.
// Two launches, for caches beyond the registers and where work-groups of 4,096 rows are half of the chip at most: those
// find the least of theirs, and a work-group per selection head the least of these (8,321 rows of 4 heads 8.0 us, 8.7 in
// one launch, 24,000 rows 8.0 and 15.8, 5,000 rows 7.6 and 6.8; of 112 heads 15.1 and 13.1).
// ------------------------------------------------------------------------------------------
constexpr int kFew = 8;
// up to four rows of any cache, up to eight of more than 16,384 rows (eight of 1,180 rows 7.7 us one by one, 6.3 by a threshold, of
// 10,000 16.5 and 14.0, of 16,384 16.6 and 19.6; four of 3,000 6.6 and 8.1)
inline bool few_leave(int Nk, int n_keep) { return Nk - n_keep <= (Nk > 16 * kSelThreads ? kFew : kFew / 2); }

// The row that leaves first: lowest rank, of equal ones the highest row; row -1: none.
struct Least {
  uint32_t rank;
  int row;
  __device__ __forceinline__ void take(uint32_t other_rank, int other_row) {
    if (other_row >= 0 && (row < 0 || other_rank < rank || (other_rank == rank && other_row > row))) rank = other_rank, row = other_row;
  }
};
__device__ __forceinline__ Least wave_least(Least x) {
  auto least = [](int a, int b) { return static_cast<int>(min(static_cast<uint32_t>(a), static_cast<uint32_t>(b))); };
  // a lane without a row has the highest rank there is, and loses to any row of that rank
  const uint32_t rank = x.row < 0 ? 0xffffffffu : x.rank;
  const uint32_t lowest = __builtin_amdgcn_readlane(wave_scan(static_cast<int>(rank), -1, least), 63);
  const int row = wave_scan(rank == lowest ? x.row : -1, -1, [](int a, int b) { return max(a, b); });
  return {lowest, __builtin_amdgcn_readlane(row, 63)};
}
// of the work-group, in every thread; s: an entry per wave, not used by the call before
__device__ __forceinline__ Least block_least(Least x, Least* s) {
  const int lane = threadIdx.x & 63;
  x = wave_least(x);
  if (lane == 0) s[threadIdx.x >> 6] = x;
  __syncthreads();
  return wave_least(lane < kSelWaves ? s[lane] : Least{0, -1});
}

// The rows that leave, in any order, become holes and movers, both ascending; by one wave.  Returns how many.
__device__ __forceinline__ int pair_few(const int (&out)[kFew], int Nk, int n_keep, int32_t* holes, int32_t* movers) {
  const int lane = threadIdx.x & 63, n_out = Nk - n_keep;
  int mine = INT_MAX, before = 0;
#pragma unroll
  for (int k = 0; k < kFew; ++k)
    if (k == lane && k < n_out) mine = out[k];
  const bool hole = mine < n_keep;
  bool leaves = false;
#pragma unroll
  for (int k = 0; k < kFew; ++k) {
    before += k < n_out && out[k] < mine;
    leaves |= k < n_out && out[k] == n_keep + lane;
  }
  if (hole) holes[before] = mine;            // rows below a hole that leave are holes
  const uint64_t kept = __ballot(lane < n_out && !leaves);
  if (kept >> lane & 1) movers[lanes_below(kept, 0)] = n_keep + lane;
  return __popcll(__ballot(hole));
}

// Ends both forms: the pairs, and the rows' moves or what the launch that makes them reads.
__device__ __forceinline__ void finish_few(const int (&out)[kFew], const Ranks& a, int sel, int room, int32_t* counts,
                                           int32_t* lists, const Moves& m, int move) {
  __shared__ int32_t s_lists[2 * kFew], s_n;
  if (threadIdx.x < 64) {
    const int n = pair_few(out, a.Nk, a.n_keep, s_lists, s_lists + kFew);
    if (threadIdx.x == 0) s_n = n;
  }
  __threadfence_block();       // rows of idx that this work-group wrote lie before the ones that the moves write
  __syncthreads();
  const int n = s_n;
  if (!move) {
    int32_t* to = lists + static_cast<int64_t>(sel) * 2 * room;
    if (static_cast<int>(threadIdx.x) < n) {
      to[threadIdx.x] = s_lists[threadIdx.x];
      to[room + threadIdx.x] = s_lists[kFew + threadIdx.x];
    }
    if (threadIdx.x == 0) counts[sel] = n;
    return;
  }
  for (int h = sel * m.per; h < (sel + 1) * m.per; ++h) {
    move_rows(m, h, n, s_lists, s_lists + kFew, threadIdx.x, kSelThreads);
    move_book(m, h, sel, n, s_lists, s_lists + kFew, threadIdx.x, kSelThreads);
  }
}

// With `least` (slices of 64 kItems x 16 rows in grid.x) the slice's leavers go there, else they leave at once.
template <int kItems>
__global__ __launch_bounds__(kSelThreads) void evict_few_kernel(Ranks a, int room, int32_t* __restrict__ counts,
                                                                int32_t* __restrict__ lists, Moves m, int move, Least* least) {
  __shared__ Least s_least[kFew][kSelWaves];
  const int sel = blockIdx.y, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const HeadRanks head(a, sel);
  const int64_t j0 = (static_cast<int64_t>(blockIdx.x) * kSelWaves + wave) * 64 * kItems + lane;
  HeadRanks::Row row[kItems];
#pragma unroll
  for (int i = 0; i < kItems; ++i) row[i] = head.fetch(static_cast<int>(min(j0 + i * 64, static_cast<int64_t>(a.Nk) - 1)));
  const int64_t border = head.border();
  uint32_t key[kItems], there = 0;
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    const int64_t j = j0 + i * 64;
    key[i] = head.rank(row[i], static_cast<int>(j), border);
    if (j < a.Nk) there |= 1u << i;
    if (m.idx != nullptr && j < a.n_keep) m.idx[sel * m.idx_stride_h + j] = static_cast<int32_t>(j);
  }
  const int n_out = a.Nk - a.n_keep;
  int out[kFew] = {};
  Least mine = {0, -1};
  auto look = [&] {            // the lane's rows ascend: of equal ranks the last one wins
    mine = {0, -1};
#pragma unroll
    for (int i = 0; i < kItems; ++i)
      if ((there >> i & 1) && (mine.row < 0 || key[i] <= mine.rank)) mine = {key[i], static_cast<int>(j0) + i * 64};
  };
  look();
#pragma unroll
  for (int k = 0; k < kFew; ++k) {
    if (k >= n_out) break;
    const Least x = block_least(mine, s_least[k]);
    out[k] = x.row;
    if (least != nullptr && threadIdx.x == 0) least[(static_cast<int64_t>(sel) * gridDim.x + blockIdx.x) * n_out + k] = x;
    if (x.row >= 0 && x.row == mine.row) {      // its lane looks at its others
      there &= ~(1u << ((x.row - j0) >> 6));
      look();
    }
  }
  if (least == nullptr) finish_few(out, a, sel, room, counts, lists, m, move);
}

__global__ __launch_bounds__(kSelThreads) void evict_few_join_kernel(Ranks a, int room, int32_t* __restrict__ counts,
                                                                     int32_t* __restrict__ lists, Moves m, int move,
                                                                     const Least* __restrict__ least, int n_least) {
  __shared__ Least s_least[kFew][kSelWaves];
  const int sel = blockIdx.x, n_out = a.Nk - a.n_keep;
  const Least* from = least + static_cast<int64_t>(sel) * n_least;
  int out[kFew] = {};
  Least mine = {0, -1};
  auto look = [&](int n_gone) {
    mine = {0, -1};
    for (int c = threadIdx.x; c < n_least; c += kSelThreads) {
      const Least x = from[c];
      bool gone = false;
#pragma unroll
      for (int p = 0; p < kFew; ++p) gone |= p < n_gone && x.row == out[p];
      if (!gone) mine.take(x.rank, x.row);
    }
  };
  look(0);
#pragma unroll
  for (int k = 0; k < kFew; ++k) {
    if (k >= n_out) break;
    out[k] = block_least(mine, s_least[k]).row;
    if (out[k] == mine.row) look(k + 1);
  }
  finish_few(out, a, sel, room, counts, lists, m, move);
}

// ------------------------------------------------------------------------------------------
// More rows: slices of them, a work-group each, in four launches.
//   count    ranks (written out: the rows' t lies 12 bytes apart) and the slice's counts of the top bits
//   gather   the bin that the threshold lies in; rows above and below it are decided, rows in it are
//            appended to the selection head's candidates (their order does not matter: what is kept is a cut
//            through the order by rank, then row)
//   resolve  a work-group per selection head: the cut, and where every slice's holes and movers begin
//   place    the lists
// ------------------------------------------------------------------------------------------
struct Slices {
  int n, rows, rows_log2, row_bits;      // slices, rows of one (kSlice times a power of two), bits of a row number
  uint32_t* ranks;            // [Hsel][Nk]
  int32_t* hist;              // [Hsel][n][kTopBins]
  uint64_t* candidates;       // [Hsel][Nk]
  int32_t* decided;           // [Hsel][n][2]: holes and movers of the gather, then where a slice's begin
  int32_t* head;              // [Hsel][4]: the threshold's bin, rows wanted of it, rows in it
  uint32_t* cut;              // [Hsel][2]: rank and row: rows of a higher rank stay, of this rank up to this row
};

// A row whose rank lies in the threshold's bin, in the order by rank (its other 21 bits), then row, lower rows above;
// row_bits of them hold any row of the call.
constexpr int kRest = 32 - kTopBits;
__device__ __forceinline__ uint64_t candidate(uint32_t rank, int row, int row_bits) {
  return static_cast<uint64_t>(rank & ((1u << kRest) - 1)) << row_bits | static_cast<uint32_t>((1 << row_bits) - 1 - row);
}
__device__ __forceinline__ int row_of(uint64_t candidate, int row_bits) {
  return (1 << row_bits) - 1 - static_cast<int>(candidate & ((1u << row_bits) - 1));
}

__global__ __launch_bounds__(kSelThreads) void evict_count_kernel(Ranks a, Slices s) {
  __shared__ __align__(16) int hist[kTopBins * kCopies];
  const int sel = blockIdx.y, slice = blockIdx.x;
  const HeadRanks head(a, sel);
  const int64_t border = head.border();
  for (int b = threadIdx.x * 4; b < kTopBins * kCopies; b += kSelThreads * 4)
    *reinterpret_cast<u32x4*>(hist + b) = u32x4{0, 0, 0, 0};
  __syncthreads();
  const int64_t end = min(static_cast<int64_t>(slice + 1) * s.rows, static_cast<int64_t>(a.Nk));
  uint32_t* out = s.ranks + static_cast<int64_t>(sel) * a.Nk;
  for (int64_t r0 = static_cast<int64_t>(slice) * s.rows; r0 < end; r0 += kSlice) {
    HeadRanks::Row row[kItemsOfSlice];
#pragma unroll
    for (int i = 0; i < kItemsOfSlice; ++i)
      row[i] = head.fetch(static_cast<int>(min(r0 + i * kSelThreads + threadIdx.x, static_cast<int64_t>(a.Nk) - 1)));
#pragma unroll
    for (int i = 0; i < kItemsOfSlice; ++i) {
      const int64_t j = r0 + i * kSelThreads + threadIdx.x;
      const uint32_t key = head.rank(row[i], static_cast<int>(j), border);
      if (j < end) {
        out[j] = key;
        count_top(hist, key);
      }
    }
  }
  __syncthreads();
  int32_t* to = s.hist + (static_cast<int64_t>(sel) * s.n + slice) * kTopBins;
  for (int b = threadIdx.x; b < kTopBins; b += kSelThreads) to[b] = counted_top(hist, b);
}

__global__ __launch_bounds__(kSelThreads) void evict_gather_kernel(Ranks a, Slices s) {
  __shared__ __align__(16) int hist[kTopBins];
  __shared__ int s_wave[kSelWaves], s_found[3], s_count[2], s_at;
  const int sel = blockIdx.y, slice = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int32_t* all = s.hist + static_cast<int64_t>(sel) * s.n * kTopBins;
  const int64_t end = min(static_cast<int64_t>(slice + 1) * s.rows, static_cast<int64_t>(a.Nk));
  const uint32_t* in = s.ranks + static_cast<int64_t>(sel) * a.Nk;
  int64_t r0 = static_cast<int64_t>(slice) * s.rows;
  uint32_t key[kItemsOfSlice];
  auto fetch = [&] {
#pragma unroll
    for (int i = 0; i < kItemsOfSlice; ++i) key[i] = in[min(r0 + i * kSelThreads + threadIdx.x, end - 1)];
  };
  fetch();
  {
    // the slices' counts: half of the threads each, four bins per thread, twelve slices in flight
    static_assert(kTopBins == 2 * kSelThreads, "four bins per thread of a half");
    const int half = threadIdx.x >= kSelThreads / 2, quad = threadIdx.x % (kSelThreads / 2);
    const u32x4* from = reinterpret_cast<const u32x4*>(all) + quad;
    u32x4 c = {0, 0, 0, 0};
    for (int k0 = half; k0 < s.n; k0 += 24) {
      u32x4 v[12];
#pragma unroll
      for (int k = 0; k < 12; ++k) v[k] = from[static_cast<int64_t>(min(k0 + 2 * k, s.n - 1)) * (kTopBins / 4)];
#pragma unroll
      for (int k = 0; k < 12; ++k)
        if (k0 + 2 * k < s.n) c += v[k];
    }
    if (half) reinterpret_cast<u32x4*>(hist)[quad] = c;
    __syncthreads();
    if (!half) reinterpret_cast<u32x4*>(hist)[quad] += c;
  }
  if (threadIdx.x < 2) s_count[threadIdx.x] = 0;
  __syncthreads();
  find_bin<kTopBins>([&](int b) { return hist[b]; }, a.n_keep, s_wave, s_found);
  const uint32_t bin = s_found[0];
  // the slice's candidates begin behind those of the slices before it
  if (wave == 0) {
    int before = 0;
    for (int k = lane; k < slice; k += 64) before += all[static_cast<int64_t>(k) * kTopBins + bin];
    before = wave_prefix_sum(before);
    if (lane == 63) s_at = before;
  }
  if (slice == 0 && threadIdx.x < 3) s.head[sel * 4 + threadIdx.x] = s_found[threadIdx.x];
  __syncthreads();
  uint64_t* out = s.candidates + static_cast<int64_t>(sel) * a.Nk;
  int holes = 0, movers = 0;
  for (;;) {
#pragma unroll
    for (int i = 0; i < kItemsOfSlice; ++i) {
      const int64_t j = r0 + i * kSelThreads + threadIdx.x;
      const uint32_t top = key[i] >> kRest;
      holes += __popcll(__ballot(j < end && j < a.n_keep && top < bin));
      movers += __popcll(__ballot(j < end && j >= a.n_keep && top > bin));
      const bool open = j < end && top == bin;
      const uint64_t b = __ballot(open);
      if (b != 0) {      // the wave's place among the slice's candidates
        int at = 0;
        if (lane == 0) at = atomicAdd(&s_at, __popcll(b));
        at = __builtin_amdgcn_readfirstlane(at);
        if (open) out[lanes_below(b, at)] = candidate(key[i], static_cast<int>(j), s.row_bits);
      }
    }
    r0 += kSlice;
    if (r0 >= end) break;
    fetch();
  }
  if (lane == 0) {
    atomicAdd(&s_count[0], holes);
    atomicAdd(&s_count[1], movers);
  }
  __syncthreads();
  if (threadIdx.x < 2) s.decided[(static_cast<int64_t>(sel) * s.n + slice) * 2 + threadIdx.x] = s_count[threadIdx.x];
}

__global__ __launch_bounds__(kSelThreads) void evict_resolve_kernel(Ranks a, Slices s, int32_t* __restrict__ counts) {
  constexpr int kHeld = 12;          // candidates of a thread that stay in registers; more are read again each time
  __shared__ int hist[2048], s_wave[kSelWaves], s_found[3], s_holes[kMaxSlices], s_movers[kMaxSlices];
  const int sel = blockIdx.x, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint64_t* cand = s.candidates + static_cast<int64_t>(sel) * a.Nk;
  int32_t* decided = s.decided + static_cast<int64_t>(sel) * s.n * 2;
  const uint32_t bin = s.head[sel * 4];
  int left = s.head[sel * 4 + 1];
  const int n = s.head[sel * 4 + 2];
  uint64_t held[kHeld];
#pragma unroll
  for (int i = 0; i < kHeld; ++i) held[i] = cand[min(i * kSelThreads + static_cast<int>(threadIdx.x), n - 1)];
  auto each = [&](auto&& f) {
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
      if (i * kSelThreads + static_cast<int>(threadIdx.x) < n) f(held[i]);
    for (int c = kHeld * kSelThreads + threadIdx.x; c < n; c += kSelThreads) f(cand[c]);
  };
  for (int k = threadIdx.x; k < s.n; k += kSelThreads) s_holes[k] = decided[k * 2], s_movers[k] = decided[k * 2 + 1];
  uint64_t prefix = 0;
  bool whole = n == left;
  // 11 and 10 bits of the rank, up to 11 at a time of the row
  for (int shift = kRest + s.row_bits; !whole && shift > 0;) {
    const int bits = shift > s.row_bits ? (shift - s.row_bits > 10 ? 11 : 10) : min(11, shift), upper = shift;
    shift -= bits;
    __syncthreads();
    for (int b = threadIdx.x; b < 2048; b += kSelThreads) hist[b] = 0;
    __syncthreads();
    each([&](uint64_t o) {
      if ((o ^ prefix) >> upper == 0) atomicAdd(&hist[static_cast<int>(o >> shift) & ((1 << bits) - 1)], 1);
    });
    __syncthreads();
    find_bin<2048>([&](int b) { return hist[b]; }, left, s_wave, s_found);
    prefix |= static_cast<uint64_t>(s_found[0]) << shift;
    left = s_found[1];
    whole = s_found[2] == left;
  }
  __syncthreads();
  // candidates lie slice by slice, so a wave's are of one slice or two: one addition for all of a slice's
  auto tally = [&](uint64_t o, bool there) {
    const int row = row_of(o, s.row_bits), slice = row >> s.rows_log2;
    const bool stays = o >= prefix;
    const bool hole = there && row < a.n_keep && !stays, mover = there && row >= a.n_keep && stays;
    for (uint64_t todo = __ballot(hole || mover); todo != 0;) {
      const int at = __builtin_amdgcn_readlane(slice, __builtin_ctzll(todo));
      const uint64_t h = __ballot(hole && slice == at), m = __ballot(mover && slice == at);
      if (lane == 0 && h != 0) atomicAdd(&s_holes[at], __popcll(h));
      if (lane == 0 && m != 0) atomicAdd(&s_movers[at], __popcll(m));
      todo &= ~(h | m);
    }
  };
#pragma unroll
  for (int i = 0; i < kHeld; ++i)
    if (i * kSelThreads + wave * 64 < n) tally(held[i], i * kSelThreads + static_cast<int>(threadIdx.x) < n);
  for (int c = kHeld * kSelThreads + threadIdx.x; c - lane < n; c += kSelThreads) tally(cand[min(c, n - 1)], c < n);
  __syncthreads();
  // where the slices' holes and movers begin: a wave each, 64 slices at a time
  if (wave < 2) {
    const int* c = wave == 0 ? s_holes : s_movers;
    int before = 0;
    for (int k0 = 0; k0 < s.n; k0 += 64) {
      const int v = k0 + lane < s.n ? c[k0 + lane] : 0, upto = wave_prefix_sum(v);
      if (k0 + lane < s.n) decided[(k0 + lane) * 2 + wave] = before + upto - v;
      before += __builtin_amdgcn_readlane(upto, 63);
    }
    if (wave == 0 && lane == 0) {
      counts[sel] = before;
      s.cut[sel * 2] = bin << kRest | static_cast<uint32_t>(prefix >> s.row_bits);
      s.cut[sel * 2 + 1] = row_of(prefix, s.row_bits);
    }
  }
}

__global__ __launch_bounds__(kSelThreads) void evict_place_kernel(Ranks a, Slices s, int room, int32_t* __restrict__ lists,
                                                                  int32_t* __restrict__ idx, int64_t idx_stride_h) {
  __shared__ int s_wave[2][2][kSelWaves];
  const int sel = blockIdx.y, slice = blockIdx.x, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t* ranks = s.ranks + static_cast<int64_t>(sel) * a.Nk;
  const uint32_t cut = s.cut[sel * 2], cut_row = s.cut[sel * 2 + 1];
  const int32_t* begin = s.decided + (static_cast<int64_t>(sel) * s.n + slice) * 2;
  int at_h = begin[0], at_m = begin[1];
  int32_t* holes = lists + static_cast<int64_t>(sel) * 2 * room;
  int32_t* movers = holes + room;
  const int64_t end = min(static_cast<int64_t>(slice + 1) * s.rows, static_cast<int64_t>(a.Nk));
  int turn = 0;
  for (int64_t r0 = static_cast<int64_t>(slice) * s.rows; r0 < end; r0 += kSlice, turn ^= 1) {
    const int64_t j0 = r0 + wave * 64 * kItemsOfSlice + lane;
    uint32_t key[kItemsOfSlice];
    uint64_t bh[kItemsOfSlice], bm[kItemsOfSlice];
    int n_holes = 0, n_movers = 0;
#pragma unroll
    for (int i = 0; i < kItemsOfSlice; ++i) key[i] = ranks[min(j0 + i * 64, static_cast<int64_t>(a.Nk) - 1)];
#pragma unroll
    for (int i = 0; i < kItemsOfSlice; ++i) {
      const int64_t j = j0 + i * 64;
      const bool stays = j < end && (key[i] > cut || (key[i] == cut && j <= cut_row));
      bh[i] = __ballot(j < end && j < a.n_keep && !stays), bm[i] = __ballot(j >= a.n_keep && stays);
      n_holes += __popcll(bh[i]), n_movers += __popcll(bm[i]);
      if (idx != nullptr && stays && j < a.n_keep) idx[sel * idx_stride_h + j] = static_cast<int32_t>(j);
    }
    if (lane == 0) s_wave[turn][0][wave] = n_holes, s_wave[turn][1][wave] = n_movers;
    __syncthreads();
    int mine_h = at_h + before_wave(s_wave[turn][0], wave), mine_m = at_m + before_wave(s_wave[turn][1], wave);
    at_h += before_wave(s_wave[turn][0], kSelWaves), at_m += before_wave(s_wave[turn][1], kSelWaves);
#pragma unroll
    for (int i = 0; i < kItemsOfSlice; ++i) {
      const int j = static_cast<int>(j0) + i * 64;
      if (bh[i] >> lane & 1) holes[lanes_below(bh[i], mine_h)] = j;
      if (bm[i] >> lane & 1) movers[lanes_below(bm[i], mine_m)] = j;
      mine_h += __popcll(bh[i]), mine_m += __popcll(bm[i]);
    }
  }
}

// ------------------------------------------------------------------------------------------
// host
// ------------------------------------------------------------------------------------------
constexpr size_t kWsAlign = 256;
constexpr int kMaxInRegisters = 24 * kSelThreads;
constexpr int64_t kMoveWithSelect = 64 << 10;     // bytes that a work-group of the one-launch form moves at most

// What a call keeps in its workspace; `base` may be NULL where only the size is asked for.
struct EvictPlan {
  int room, n_slices, slice_rows;       // room: of a list; n_slices 0: one work-group per selection head
  bool few;                             // rows that leave are found one by one
  int32_t *counts, *lists;
  Least* least;                         // of few and several slices: [Hsel][n_slices][rows that leave]
  Slices s;
  size_t bytes;
  EvictPlan(int Hsel, int Nk, int n_keep, void* base) : room(std::min(Nk - n_keep, n_keep)), n_slices(0), slice_rows(0), few(few_leave(Nk, n_keep)), least(nullptr), s() {
    size_t at = 0;
    auto take = [&](size_t n) {
      void* p = static_cast<uint8_t*>(base) + at;
      at += align_up(n, kWsAlign);
      return p;
    };
    const size_t heads = Hsel;
    counts = static_cast<int32_t*>(take(heads * 4));
    lists = static_cast<int32_t*>(take(heads * 2 * room * 4));
    const int64_t pieces = ceil_div(Nk, kSlice);
    if (few && Nk > kSlice && (Nk > kMaxInRegisters || pieces * Hsel <= 128)) {
      n_slices = static_cast<int>(pieces);
      least = static_cast<Least*>(take(heads * n_slices * (Nk - n_keep) * sizeof(Least)));
    } else if (!few && Nk > kMaxInRegisters) {
      int rows_log2 = 12;
      static_assert(kSlice == 1 << 12, "the least slice");
      while (((Nk - 1) >> rows_log2) >= kMaxSlices) ++rows_log2;
      slice_rows = 1 << rows_log2;
      n_slices = ceil_div(Nk, slice_rows);
      int row_bits = 1;
      while ((1ll << row_bits) < Nk) ++row_bits;
      s = {n_slices, slice_rows, rows_log2, row_bits, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr};
      s.ranks = static_cast<uint32_t*>(take(heads * Nk * 4));
      s.hist = static_cast<int32_t*>(take(heads * n_slices * kTopBins * 4));
      s.candidates = static_cast<uint64_t*>(take(heads * Nk * 8));
      s.decided = static_cast<int32_t*>(take(heads * n_slices * 8));
      s.head = static_cast<int32_t*>(take(heads * 16));
      s.cut = static_cast<uint32_t*>(take(heads * 8));
    }
    bytes = at;
  }
};

int evict(const char* who, Moves m, int64_t row_bytes, int H, int32_t* pos, int64_t pos_stride_h, float* weights,
          int64_t w_stride_h, int Hsel, int Nk, int n_keep, int n_anchor, int recent_t, int32_t* idx_out, int64_t idx_stride_h,
          void* ws, size_t ws_bytes, void* stream) {
  PC_REQUIRE(H > 0 && Hsel > 0 && Hsel <= H && H % Hsel == 0, PC_ERR_SHAPE, "%s: %d selection heads for %d heads", who, Hsel, H);
  PC_REQUIRE(H <= 65535, PC_ERR_SHAPE, "%s: %d heads in one call", who, H);
  PC_REQUIRE(Nk >= 0 && Nk <= kMaxRows, PC_ERR_SHAPE, "%s: Nk=%d", who, Nk);
  PC_REQUIRE(n_keep >= 0 && n_anchor >= 0 && recent_t >= 0 && n_anchor <= n_keep, PC_ERR_BUDGET,
             "%s: n_keep=%d n_anchor=%d recent_t=%d", who, n_keep, n_anchor, recent_t);
  PC_REQUIRE(weights, PC_ERR_NULL, "%s: weights is NULL", who);
  PC_REQUIRE(recent_t == 0 || pos, PC_ERR_NULL, "%s: recent rows are found by pos, which is NULL", who);
  PC_REQUIRE(Hsel == 1 || (w_stride_h >= Nk && (!pos || pos_stride_h >= 3ll * Nk)), PC_ERR_SHAPE,
             "%s: the head stride of weights or pos is smaller than the rows", who);
  PC_REQUIRE(!idx_out || Hsel == 1 || idx_stride_h >= std::min(n_keep, Nk), PC_ERR_SHAPE, "%s: idx stride", who);
  if (Nk == 0) return PC_OK;
  if (n_keep >= Nk) {
    PC_REQUIRE(!idx_out, PC_ERR_BUDGET, "%s: nothing is evicted (n_keep=%d of %d rows), no index is written", who, n_keep, Nk);
    return PC_OK;
  }
  if (n_keep == 0) return PC_OK;
  const EvictPlan plan(Hsel, Nk, n_keep, ws);
  PC_REQUIRE(ws && ws_bytes >= plan.bytes && reinterpret_cast<uintptr_t>(ws) % 16 == 0, PC_ERR_WORKSPACE,
             "%s: needs %zu bytes of 16-byte aligned workspace, got %zu", who, plan.bytes, ws_bytes);
  m.pos = pos, m.weights = weights, m.pos_stride_h = pos_stride_h, m.w_stride_h = w_stride_h;
  m.idx = idx_out, m.idx_stride_h = idx_stride_h, m.per = H / Hsel;
  const int64_t units = static_cast<int64_t>(plan.room) * m.by_both.d;
  PC_REQUIRE(units <= INT_MAX - (1 << 22), PC_ERR_SHAPE, "%s: %d rows may move in one call", who, plan.room);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const Ranks a = {weights, pos, w_stride_h, pos_stride_h, Nk, n_keep, n_anchor, recent_t};
  const int move = plan.room * row_bytes * m.per <= kMoveWithSelect, items = ceil_div(Nk, kSelThreads);
  if (plan.few && plan.n_slices > 0) {
    evict_few_kernel<kItemsOfSlice><<<dim3(plan.n_slices, Hsel), kSelThreads, 0, s>>>(a, plan.room, plan.counts, plan.lists, m, 0, plan.least);
    PC_CHECK_LAUNCH(who);
    evict_few_join_kernel<<<Hsel, kSelThreads, 0, s>>>(a, plan.room, plan.counts, plan.lists, m, move, plan.least,
                                                       plan.n_slices * (Nk - n_keep));
    PC_CHECK_LAUNCH(who);
    if (move) return PC_OK;
  } else if (plan.few) {
    const auto kernel = items <= 2    ? evict_few_kernel<2>
                        : items <= 4  ? evict_few_kernel<4>
                        : items <= 8  ? evict_few_kernel<8>
                        : items <= 12 ? evict_few_kernel<12>
                        : items <= 16 ? evict_few_kernel<16>
                                      : evict_few_kernel<24>;
    kernel<<<dim3(1, Hsel), kSelThreads, 0, s>>>(a, plan.room, plan.counts, plan.lists, m, move, nullptr);
    PC_CHECK_LAUNCH(who);
    if (move) return PC_OK;
  } else if (plan.n_slices == 0) {
    // six and ten rows per thread beside eight and twelve: 4 heads x 5,500 rows 12.8 us, 13.4 with eight, x 9,500 16.3 and 17.2 with
    // twelve; 28 heads 10.7 and 11.3, 13.6 and 14.3; 112 heads 17.3 and 17.7, 25.1 and 25.7
    const auto kernel = items <= 2    ? evict_select_kernel<2>
                        : items <= 4  ? evict_select_kernel<4>
                        : items <= 6  ? evict_select_kernel<6>
                        : items <= 8  ? evict_select_kernel<8>
                        : items <= 10 ? evict_select_kernel<10>
                        : items <= 12 ? evict_select_kernel<12>
                        : items <= 16 ? evict_select_kernel<16>
                                      : evict_select_kernel<24>;
    kernel<<<Hsel, kSelThreads, 0, s>>>(a, plan.room, plan.counts, plan.lists, m, move);
    PC_CHECK_LAUNCH(who);
    if (move) return PC_OK;
  } else {
    const dim3 grid(plan.n_slices, Hsel);
    evict_count_kernel<<<grid, kSelThreads, 0, s>>>(a, plan.s);
    PC_CHECK_LAUNCH(who);
    evict_gather_kernel<<<grid, kSelThreads, 0, s>>>(a, plan.s);
    PC_CHECK_LAUNCH(who);
    evict_resolve_kernel<<<Hsel, kSelThreads, 0, s>>>(a, plan.s, plan.counts);
    PC_CHECK_LAUNCH(who);
    evict_place_kernel<<<grid, kSelThreads, 0, s>>>(a, plan.s, plan.room, plan.lists, idx_out, idx_stride_h);
    PC_CHECK_LAUNCH(who);
  }
  const int book = std::min(ceil_div(plan.room, 256), 64);
  const int rows = static_cast<int>(std::min<int64_t>((units + 1023) / 1024, 4096));
  evict_move_kernel<<<dim3(book + rows, H), 256, 0, s>>>(m, book, plan.room, plan.counts, plan.lists);
  PC_CHECK_LAUNCH(who);
  return PC_OK;
}

}  // namespace
}  // namespace pc

using namespace pc;

extern "C" size_t pc_evict_workspace_bytes(int Hsel, int Nk, int n_keep) {
  if (Hsel <= 0 || Nk <= 0 || n_keep <= 0 || n_keep >= Nk || Nk > kMaxRows) return 0;
  return EvictPlan(Hsel, Nk, n_keep, nullptr).bytes;
}

extern "C" int pc_evict(void* K, void* V, int dtype, int H, int D, int64_t k_stride_h, int64_t v_stride_h, int32_t* pos,
                        int64_t pos_stride_h, float* weights, int64_t weights_stride_h, int Hsel, int Nk, int n_keep,
                        int n_anchor, int recent_t, int32_t* idx_out, int64_t idx_stride_h, void* ws, size_t ws_bytes,
                        void* stream) {
  const char* who = "pc_evict";
  PC_REQUIRE(dtype == PC_F32 || dtype == PC_BF16, PC_ERR_DTYPE, "%s: dtype %d", who, dtype);
  PC_REQUIRE(D > 0 && D <= 1024 && D % 8 == 0, PC_ERR_UNSUPPORTED, "%s: D=%d must be a multiple of 8, at most 1024", who, D);
  PC_REQUIRE(K && V, PC_ERR_NULL, "%s: K or V is NULL", who);
  if (H == 1) k_stride_h = v_stride_h = static_cast<int64_t>(Nk) * D;     // one head has no stride that matters
  PC_REQUIRE(H <= 1 || (k_stride_h >= static_cast<int64_t>(Nk) * D && v_stride_h >= static_cast<int64_t>(Nk) * D), PC_ERR_SHAPE,
             "%s: a head stride is smaller than rows*D", who);
  const int elt = dtype == PC_BF16 ? 2 : 4;
  PC_REQUIRE((reinterpret_cast<uintptr_t>(K) | reinterpret_cast<uintptr_t>(V) | k_stride_h * elt | v_stride_h * elt) % 16 == 0,
             PC_ERR_SHAPE, "%s: K, V and their head strides must be 16-byte aligned", who);
  const int pieces = D * elt / 16;
  const Moves m = {{static_cast<u32x4*>(K), static_cast<u32x4*>(V)}, {k_stride_h * elt / 16, v_stride_h * elt / 16}, Divisor(pieces),
                   Divisor(2 * pieces)};
  return evict(who, m, 32ll * pieces, H, pos, pos_stride_h, weights, weights_stride_h, Hsel, Nk, n_keep, n_anchor, recent_t, idx_out,
               idx_stride_h, ws, ws_bytes, stream);
}

extern "C" int pc_q4_evict(const pc_q4_cache* cache, int H, int D, int32_t* pos, int64_t pos_stride_h, float* weights,
                           int64_t weights_stride_h, int Hsel, int Nk, int n_keep, int n_anchor, int recent_t,
                           int32_t* idx_out, int64_t idx_stride_h, void* ws, size_t ws_bytes, void* stream) {
  const char* who = "pc_q4_evict";
  PC_REQUIRE(D == 64 || D == 128, PC_ERR_UNSUPPORTED, "%s: needs D = 64 or 128, got %d", who, D);
  if (int rc = check_q4_cache(cache, D, who)) return rc;
  if (int rc = check_q4_span(cache, H, 0, Nk, D, who)) return rc;
  const int pieces = D / 32;
  const Moves m = {{reinterpret_cast<u32x4*>(cache->k_codes), reinterpret_cast<u32x4*>(cache->v_codes)},
                   {cache->code_stride_h / 16, cache->code_stride_h / 16}, Divisor(pieces), Divisor(2 * pieces),
                   {cache->k_scales, cache->v_scales}, cache->scale_stride_h, D / 32};
  return evict(who, m, 32ll * pieces, H, pos, pos_stride_h, weights, weights_stride_h, Hsel, Nk, n_keep, n_anchor, recent_t, idx_out,
               idx_stride_h, ws, ws_bytes, stream);
}
