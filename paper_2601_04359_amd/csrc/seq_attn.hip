// pc_prompt_attn and pc_page_attn: attention with a limit per row, over packed prompts and over a cache held in pages.
#include <limits.h>
#include <math.h>

#include <algorithm>
#include <vector>

#include "rows_bf16.h"
#include "rows_f32.h"

namespace pc {
namespace {

template <typename T>
__device__ __forceinline__ void store4(T* p, f32x4 v) {
  if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4*>(p) = v;
  else *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
}

// ------------------------------------------------------------------------------------------
// The shares of a row joined: O = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s with M = max_s m_s, over the shares that
// have written something.  A thread has four dims of a row; kSplit groups of them take the row's shares by turns and add
// up in LDS (few rows come in many shares, and one after the other they would wait for as many loads).  Bound: the launch and
// three loads one behind the other (64 rows of 6 shares 4 us), or the shares' bytes (8,192 rows of 9 shares, 38 MB, 9 us).
// ------------------------------------------------------------------------------------------
template <typename T, int D, int kSplit>
__global__ __launch_bounds__(256) void rows_join_kernel(RowsArgs a) {
  constexpr int kLanes = D / 4, kRows = 256 / (kLanes * kSplit), kBatch = 4;
  __shared__ f32x4 acc_lds[kSplit > 1 ? 256 : 1];
  __shared__ float2 ml_lds[kSplit > 1 ? 256 / kLanes : 1];
  const int group = threadIdx.x / kLanes, c = threadIdx.x % kLanes, turn = group % kSplit;
  const int n = blockIdx.x * kRows + group / kSplit;
  const int Hq = a.by_hkv.d * a.rep;
  const bool there = n < Hq * a.n_rows;
  const int head = there ? n / a.n_rows : 0, t = a.row0 + (there ? n - head * a.n_rows : 0);
  const int s = max(0, seq_of_row(a.seqs, t));
  const bool even = a.seqs.per > 0;
  const int len = len_of(a, s), q0 = even ? s * a.seqs.per : a.seqs.q0[s], nq = even ? a.seqs.per : a.seqs.nq[s];
  const int lim = len - (q0 + nq - t) + 1;
  bool none = lim <= 0;
  // where the shares of the row are: its row in the tiles over the common rows, and in those over its sequence's own
  const int kvh = a.by_rep.of(head), hh = head - kvh * a.rep, common = n_common(a);
  const int rho_c = (t - a.row0) * a.rep + hh, rho = (t - q0) * a.rep + hh;
  const int tile_c = a.by_tile.of(rho_c), tile = a.by_tile.of(rho), keys = own_keys_of(a, len);
  const bool fixed = a.own_parts > 0;
  const int share = fixed ? a.own_keys : keys > 0 ? a.cut[0] : 1, own = ceil_of(keys, share, 1.f / share);
  const int tiles = even ? a.tiles_per_seq : a.by_tile.of(nq * a.rep + a.by_tile.d - 1);
  const int64_t slots = static_cast<int64_t>(kvh) * (common + a.own_cap);
  const int64_t at_c = (slots + tile_c) * a.slot_rows + rho_c - tile_c * a.by_tile.d;
  int first = 0;     // the sequence's first unit
  if (!fixed) {
    if (keys > 0) first = a.cut[1 + s];
  } else if (even) {
    first = s * a.by_parts.d;
  } else {
    for (int q = 0; q < s; ++q) first += a.by_tile.of(a.seqs.nq[q] * a.rep + a.by_tile.d - 1) * a.own_parts;
  }
  const int64_t at_o = (slots + common + first + tile) * a.slot_rows + rho - tile * a.by_tile.d;
  const int parts = none ? 0 : a.shared_parts + own;
  auto place = [&](int p) {
    return p < a.shared_parts ? at_c + static_cast<int64_t>(p) * a.shared_tiles * a.slot_rows
                              : at_o + static_cast<int64_t>(p - a.shared_parts) * tiles * a.slot_rows;
  };
  // What a batch reads depends on the lengths only where the device has cut by them: the first one is on its way before they
  // are known, and what lies behind the shares that there are (it may be anything) does not count.
  const int last = (fixed ? a.shared_parts + a.own_parts : max(parts, 1)) - 1;
  float M = kNothing, L = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  int p0 = turn;
  do {
    f32x4 v[kBatch];
    float2 ml[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int64_t from = place(min(p0 + i * kSplit, last));
      ml[i] = a.part_ml[from];
      v[i] = *reinterpret_cast<const f32x4*>(a.part_o + from * D + c * 4);
    }
    float top = M;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      if (p0 + i * kSplit >= parts) ml[i] = {kNothing, 0.f}, v[i] = {0.f, 0.f, 0.f, 0.f};
      top = fmaxf(top, ml[i].x);
    }
    const float keep = __builtin_amdgcn_exp2f(M - top);
    M = top, L *= keep, acc *= keep;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const float by = __builtin_amdgcn_exp2f(ml[i].x - M);
      L += by * ml[i].y;
      acc += by * v[i];
    }
    p0 += kBatch * kSplit;
  } while (p0 < parts);
  if constexpr (kSplit > 1) {
    acc_lds[threadIdx.x] = acc;
    if (c == 0) ml_lds[group] = {M, L};
    __syncthreads();
    if (turn != 0) return;
    const float own_m = M;
#pragma unroll
    for (int i = 1; i < kSplit; ++i) M = fmaxf(M, ml_lds[group + i].x);
    const float keep = __builtin_amdgcn_exp2f(own_m - M);
    L *= keep, acc *= keep;
#pragma unroll
    for (int i = 1; i < kSplit; ++i) {
      const float by = __builtin_amdgcn_exp2f(ml_lds[group + i].x - M);
      acc += by * acc_lds[threadIdx.x + i * kLanes];
      L += by * ml_lds[group + i].y;
    }
  }
  if (!there) return;
  if (!none && L == 0.f)
    none = !any_page(a, a.shared, 0, min(lim, a.n_shared)) &&
           !any_page(a, a.table + (even ? s : a.seqs.k0[s]) * a.table_stride, a.n_shared, lim);
  if (!none) acc *= 1.f / L;
  else acc = f32x4{0.f, 0.f, 0.f, 0.f};
  store4(static_cast<T*>(a.O) + head * a.o_stride + static_cast<int64_t>(t) * D + c * 4, acc);
  if (a.lse != nullptr && c == 0) a.lse[static_cast<int64_t>(head) * a.T + t] = none ? -INFINITY : lse_of(M, L);
}

// ---- how a call is cut ---------------------------------------------------------------------------------------------
enum Form { kF32One, kF32Two, kFew, kMid, kMany };
int rows_of(Form f) { return f == kF32One ? 16 : f == kF32Two ? 32 : f == kFew ? kFewRows : f == kMid ? kMidRows : kManyRows; }

// Microseconds that `groups` work-groups of a bf16 form take, `steps` steps in all and `longest` in the one with the most (256
// keys for kFew, 64 for the others).  Either they fill the chip (what a work-group costs beside its steps, and a step, in time
// of a compute unit), or the longest is waited for; its steps take longer with a second work-group on its unit (`paired`).
struct Cost {
  double alone, per_step, paired, start, per_group, step;
  double operator()(double groups, double steps, double longest) const {
    return std::max(alone + (groups > 280 ? paired : per_step) * longest, start + (per_group * groups + step * steps) / 256);
  }
};
// Prompts: fitted to 40 to 16,384 rows in 8/2, 16/4 and 24/8 heads in all three forms, within 8 % from 1,000 rows on, all with a
// scale of its own (the folded one is 4 to 5 % faster on long prompts and is chosen for as these are).  Both sides, us:
//   few | mid    8/2 x 2,048: 23 | 32    16/4 x 1,024: 17 | 20    16/4 x 2,048: 42 | 34    24/8 x 1,024: 24 | 21
//   mid | many   8/2 x 8,192: 161 | 176  16/4 x 3,000: 53 | 63    16/4 x 4,288: 97 | 99    24/8 x 4,288: 140 | 118
constexpr Cost kPromptCost[3] = {{5.0, 1.75, 1.75, 2.5, 3.6, 1.25}, {7.5, 0.75, 0.84, 6.0, 2.9, 0.549}, {7.0, 1.07, 1.3, 5.0, 3.0, 0.953}};
// fp32, D = 128 and 64 (from prompts of 40 to 1,200 rows).  Both sides, 16 | 32 rows, us: 8/2 heads x 1,200 rows, D = 128, 51 | 62;
// two such prompts 94 | 84; 24/8 x 1,200 and 700 187 | 140.
constexpr Cost kF32Cost[2][2] = {{{5.5, 3.2, 3.75, 3.0, 2.0, 3.6}, {6.5, 2.7, 2.9, 3.0, 2.0, 2.8}},
                                 {{3.2, 2.1, 2.1, 3.0, 1.5, 1.6}, {5.3, 1.4, 1.5, 3.0, 1.5, 1.45}}};
const Cost& cost_of(Form f, int D) { return f <= kF32Two ? kF32Cost[D == 64][f] : kPromptCost[f - kFew]; }
int keys_per_step(Form f) { return f == kFew ? 256 : f == kF32One ? 128 : 64; }
// The forms that a call may take: first .. last.
Form first_form(int dtype) { return dtype == PC_F32 ? kF32One : kFew; }
Form last_form(int dtype, int D) { return dtype == PC_F32 ? kF32Two : D == kD ? kMany : kFew; }

int row_tiles(const int32_t* offs, int n_seq, int T, int rep, int rows) {
  if (offs == nullptr) return n_seq * ceil_div(T / n_seq * rep, rows);
  int n = 0;
  for (int s = 0; s < n_seq; ++s) n += ceil_div((offs[s + 1] - offs[s]) * rep, rows);
  return n;
}

// How pc_prompt_attn cuts a launch: the form with the lowest cost.  kMany: the n_heavy longest tiles (per KV head) are taken as two
// of 64 rows, those that would take longer than everything together.  16/4 heads, us, with none, all and these of the
// tiles: one prompt of 4,288 rows 98.6, 98.2, 90.9; nine of 1 to 2,049 rows 49.8, 50.9, 42.7; 6,000 rows 157.7, 180, 157.4.
struct Seq {
  int q0, nq, k0, nk;
};
struct PromptPlan {
  Form form;
  int n_heavy = 0;
  PromptPlan(int dtype, int D, int Hkv, int rep, const Seq* seqs, int n) {
    form = first_form(dtype);
    double best = 1e30, many_us = 0;
    for (int i = first_form(dtype); i <= last_form(dtype, D); ++i) {
      const Form f = static_cast<Form>(i);
      double groups = 0, steps = 0, longest = 0;
      for (int s = 0; s < n; ++s) {
        const double tiles = ceil_div(seqs[s].nq * rep, rows_of(f)), last = std::max(0, seqs[s].nk), first = std::max(0.0, last - seqs[s].nq);
        groups += tiles * Hkv;
        steps += tiles * Hkv * ((first + last) / 2 / keys_per_step(f) + 0.5);
        longest = std::max(longest, std::ceil(last / keys_per_step(f)));
      }
      const Cost& cost = cost_of(f, D);
      if (f == kMany) many_us = cost.start + (cost.per_group * groups + cost.step * steps) / 256;
      const double us = cost(groups, steps, longest);
      if (us < best) best = us, form = f;
    }
    if (form < kMid) return;
    // tiles with more keys than a work-group of 128 rows adds in the time that all of them take
    const Cost& cost = cost_of(kMany, D);
    const double x = (many_us - cost.alone) / cost.paired * keys_per_step(kMany);
    for (int s = 0; s < n; ++s) {
      const int tiles = ceil_div(seqs[s].nq * rep, kManyRows);
      const double light = std::floor((x - (seqs[s].nk - seqs[s].nq)) * rep / kManyRows);   // tile i ends at key nk - nq + (i + 1) 128 / rep
      n_heavy += static_cast<int>(tiles - std::min<double>(std::max(0.0, light), tiles));
    }
    form = kMany;
  }
};

// Microseconds of a launch of pc_page_attn: units over common rows of one length, and behind them units over own rows of
// another, go to the places that the chip has for a form's work-groups (`slots`; two on a compute unit take `paired` for a
// step, one alone takes `step`), each place taking the next unit when it is done with one.
struct PagesCost {
  double unit, step, paired, start;
  int slots;
  double operator()(int common, int common_steps, int own, int own_steps) const {
    const bool alone = slots == 256 || common + own <= 256;
    const double own_us = unit + own_steps * (alone ? step : paired);
    double us = start;
    int left = own;
    if (common > 0) {
      const double one = unit + common_steps * step, two = unit + common_steps * (slots == 256 ? step : paired);
      const int rounds = common / slots, rest = common - rounds * slots;
      us += rounds * two;
      if (rest > 0) {     // the last round: own rows' units go into the places left
        const double last = slots == 256 ? one : rest > 256 ? two : one + (two - one) * std::min(1.0, own * own_us / (256 * one));
        us += last;
        if (own > 0) left = std::max(0, own - (slots - rest) * static_cast<int>(std::min(last / own_us, 1e4)));
      }
    }
    return us + ceil_div(left, alone ? 256 : slots) * own_us;
  }
};
// Fitted to 3,800 launches (61 shapes of 1 to 256 sequences with 1 to 1,000 new rows, up to 41,800 common rows and 2,000 own ones, in
// each form, up to 25 lengths of a share): first the times, then the choice, which is 3 % off the best of a shape's launches
// at the mean, 15 % at most.  Both sides at the best share of each, 16/4 heads, 41,800 common rows, us:
//   few | mid | many   32 tokens: 35 | 36 | 37   64: 54 | 49 | 48   256: 168 | 139 | 131
// fp32 and D = 64: to 18 shapes each.  bf16 with D = 64 has one form, so that only its shares are chosen.
constexpr PagesCost kPagesCost[3] = {{3.2, 1.67, 1.67, 2.45, 256}, {2.1, 0.913, 1.064, 5.2, 512}, {0.0, 1.22, 1.45, 6.9, 512}};
constexpr PagesCost kPagesFew64 = {2.5, 0.89, 1.54, 2.1, 512};
// 16 | 32 rows, 16/4 heads, D = 128: 64 tokens with 1,000 rows each 45 | 65; 8 x 32 tokens behind 4,000 rows 117 | 108.
constexpr PagesCost kPagesF32[2][2] = {{{5.0, 2.95, 2.95, 4.9, 256}, {5.1, 3.14, 4.98, 6.7, 512}},
                                       {{2.7, 1.55, 2.83, 3.4, 512}, {0.1, 1.5, 2.74, 6.65, 512}}};
const PagesCost& pages_cost_of(Form f, int D) {
  return f <= kF32Two ? kPagesF32[D == 64][f] : D == 64 ? kPagesFew64 : kPagesCost[f - kFew];
}

// How pc_page_attn cuts a launch's work: a form, the shares of the common rows, and room for units over the sequences' own rows,
// which the device cuts (plan_pages); here their lengths are only known to be max_len at most, and taken to be that.  Beside
// the costs above there are the bytes of K and V (6.1 TB/s), and the shares' join: a launch, and the fp32 rows that are written
// and read (3.8 TB/s).  Candidates are the lengths that give 1, 2, 3, ... shares, and those whose units just fill the chip.
constexpr int kMostParts = 96;   // shares of a row
constexpr int kFixedKeys = 2048;
struct PagePlan {
  Form form = kF32One;
  int shared_tiles = 0, shared_parts = 0, shared_keys = kPageStep;
  int own_tiles = 0, own_parts = 0, own_cap = 0;   // own_parts 0: the device cuts
  int slot_rows = 0, slots = 0, least_keys = 4 * kPageStep;
  float unit_us = 0.f, key_us = 0.f;
  bool joined = false;           // results are shares
  PagePlan(int dtype, int D, int Hkv, int rep, int T, const int32_t* offs, int n_seq, int n_shared, int max_len) {
    const int n_rows = offs != nullptr ? offs[n_seq] - offs[0] : T;
    if (n_rows == 0) return;       // nothing is launched
    const int own = max_len > n_shared ? max_len - n_shared / kPageStep * kPageStep : 0;
    int most = offs == nullptr ? T / n_seq : 0;
    for (int s = 0; offs != nullptr && s < n_seq; ++s) most = std::max(most, offs[s + 1] - offs[s]);
    const int longest = std::max({n_shared, own, 1}), whole = ceil_div(longest, kPageStep) * kPageStep;
    const double bytes_us = 4.5 + (n_shared + static_cast<double>(own) * n_seq) * Hkv * 2.0 * D * (dtype == PC_BF16 ? 2 : 4) / 6.1e6;
    double best = 1e30;
    for (int i = first_form(dtype); i <= last_form(dtype, D); ++i) {
      const Form f = static_cast<Form>(i);
      const PagesCost& cost = pages_cost_of(f, D);
      const int step = keys_per_step(f), tiles_c = n_shared > 0 ? ceil_div(n_rows * rep, rows_of(f)) : 0,
                tiles_o = own > 0 ? row_tiles(offs, n_seq, T, rep, rows_of(f)) : 0;
      auto weigh = [&](int pieces) {
        const int share = std::min(whole, std::max(4 * kPageStep, ceil_div(ceil_div(longest, pieces), kPageStep) * kPageStep));
        const int parts_c = ceil_div(n_shared, share), parts_o = ceil_div(own, share);
        const double units = static_cast<double>(Hkv) * (static_cast<double>(tiles_c) * parts_c + static_cast<double>(tiles_o) * parts_o);
        if (parts_c + parts_o > kMostParts || (units > 1e6 && pieces > 1)) return;
        const double join = parts_c + parts_o > 1 ? 5.4 + static_cast<double>(n_rows) * rep * Hkv * (parts_c + parts_o) * (8.0 * D + 16) / 3.8e6 : 0.0;
        if (join + bytes_us >= best) return;
        const double us = join + std::max(bytes_us, units > 1e6 ? 1e12 + units : cost(Hkv * tiles_c * parts_c, ceil_div(std::min(share, n_shared), step),
                                                                                  Hkv * tiles_o * parts_o, ceil_div(std::min(share, own), step)));
        if (us >= best) return;
        best = us, form = f;
        shared_tiles = tiles_c, own_tiles = tiles_o, shared_keys = share, shared_parts = parts_c;
      };
      for (int pieces = 1; pieces <= kMostParts; pieces += 1 + pieces / 6) weigh(pieces);
      for (int fill = 256; fill <= 1536; fill += 256)
        if (const int pieces = fill / (Hkv * std::max({tiles_c, tiles_o, 1})); pieces > 1 && pieces <= kMostParts) weigh(pieces);
    }
    const PagesCost& cost = pages_cost_of(form, D);
    slots = form == kFew ? 256 : cost.slots;   // (D = 64: its longer shares cost less than the join of more)
    // a key of own rows comes from HBM: in 512 bytes a unit of kFew waits for them, not for its products
    unit_us = form == kFew ? 4.5f : 5.f;
    key_us = form == kFew ? (D == 64 ? 0.0054f : 0.0105f) : form == kF32One ? (D == 64 ? 0.0135f : 0.027f)
                          : static_cast<float>(cost.paired / keys_per_step(form));
    // The own rows' shares are as long as the common ones' while that bounds what a work-group has, whatever the lengths are:
    // it saves the work-groups 2 us of cutting.  Beyond kFixedKeys the device cuts by the lengths that there are.
    if (own > 0 && std::min(shared_keys, own) <= kFixedKeys) own_parts = ceil_div(own, shared_keys);
    joined = own > 0 && own_parts == 0 ? true : shared_parts + own_parts > 1;
    while (static_cast<int64_t>(own_tiles) * ceil_div(own, least_keys) > INT_MAX / 2) least_keys *= 2;   // sums of units are 32-bit numbers
    own_cap = own_parts > 0 ? own_tiles * own_parts
                            : static_cast<int>(std::min<int64_t>(static_cast<int64_t>(own_tiles) * ceil_div(own, 256), own_tiles + ceil_div(slots, Hkv)));
    slot_rows = std::min(rows_of(form), std::max(n_shared > 0 ? n_rows : 0, own > 0 ? most : 0) * rep);
  }
  int units() const { return shared_tiles * shared_parts + own_cap; }
  size_t o_bytes(int Hkv, int D) const { return align_up(static_cast<size_t>(Hkv) * units() * slot_rows * D * sizeof(float), 256); }
  size_t ml_bytes(int Hkv) const { return align_up(static_cast<size_t>(Hkv) * units() * slot_rows * sizeof(float2), 256); }
  size_t bytes(int Hkv, int D) const { return joined ? o_bytes(Hkv, D) + ml_bytes(Hkv) + (1 + kPageSeqs) * sizeof(int) : 0; }
};

// Calls f(first, count) for the launches that a call's sequences are dealt to; f returns a status.
template <class F>
int each_launch(const int32_t* offs, int n_seq, F&& f) {
  const int most = offs != nullptr ? kSeqs : kPageSeqs;
  for (int s0 = 0; s0 < n_seq; s0 += most)
    if (int rc = f(s0, std::min(most, n_seq - s0))) return rc;
  return PC_OK;
}

PagePlan plan_of(int dtype, int Hq, int Hkv, int T, int D, const int32_t* offs, int n_seq, int s0, int n, int max_len, int n_shared) {
  return PagePlan(dtype, D, Hkv, Hq / Hkv, offs != nullptr ? T : T / n_seq * n, offs != nullptr ? offs + s0 : nullptr, n,
                  std::min(n_shared, max_len), max_len);
}

// fp32: c is rounded down and c_lo above zero (by 2^-30 of c at least, which is far below a rounding), so that a score of -inf stays
// -inf in s c + s c_lo and is no NaN.  bf16 has c alone, to the nearest.
void set_scale(RowsArgs& a, int dtype, float scale) {
  const double c = static_cast<double>(scale) * 1.4426950408889634074;
  a.c = static_cast<float>(c);
  if (dtype == PC_F32 && a.c > c) a.c = nextafterf(a.c, 0.f);
  a.c_lo = std::max(static_cast<float>(std::max(c - a.c, c * 0x1p-30)), 0x1p-149f);
}

int check_attn(const char* who, int dtype, int Hq, int Hkv, int D, float scale) {
  PC_REQUIRE(dtype == PC_F32 || dtype == PC_BF16, PC_ERR_DTYPE, "%s: dtype %d", who, dtype);
  PC_REQUIRE(Hkv >= 1 && Hq >= 1 && Hq % Hkv == 0, PC_ERR_SHAPE, "%s: Hq=%d must be a multiple of Hkv=%d", who, Hq, Hkv);
  PC_REQUIRE(D == 64 || D == 128, PC_ERR_UNSUPPORTED, "%s: D=%d (64 or 128)", who, D);
  PC_REQUIRE(scale > 0.f && isfinite(scale), PC_ERR_SHAPE, "%s: scale %g must be > 0", who, scale);
  return PC_OK;
}

template <bool kPages>
int launch_rows(const char* who, Form form, int dtype, int D, const RowsArgs& a, int64_t blocks, hipStream_t s) {
  const int waves = form == kF32Two ? 4 : form == kF32One ? 8 : form == kFew ? kFewWaves : kManyWaves;
  PC_REQUIRE(blocks * waves * 64 <= kMaxThreads, PC_ERR_UNSUPPORTED, "%s: %lld work-groups in one launch", who, static_cast<long long>(blocks));
  if (form == kF32One || form == kF32Two) {
    static std::atomic<uint64_t> ok[4];
    const bool two = form == kF32Two;
    auto* kernel = D == 128 ? (two ? rows_f32_kernel<128, kPages, 2, 4> : rows_f32_kernel<128, kPages, 1, 8>)
                            : (two ? rows_f32_kernel<64, kPages, 2, 4> : rows_f32_kernel<64, kPages, 1, 8>);
    const size_t bytes = (D == 128 ? kF32Smem<128, 2, 4> : kF32Smem<64, 2, 4>) + kPlanBytes;
    static_assert(kF32Smem<128, 2, 4> == kF32Smem<128, 1, 8> && kF32Smem<64, 2, 4> == kF32Smem<64, 1, 8>, "the waves' O");
    if (int rc = allow_dynamic_lds(reinterpret_cast<const void*>(kernel), bytes, ok[(D == 128) * 2 + two], who)) return rc;
    kernel<<<blocks, waves * 64, bytes, s>>>(a);
  } else if (form == kFew) {
    static std::atomic<uint64_t> ok[2];
    auto* kernel = D == 128 ? rows_few_kernel<128, kPages> : rows_few_kernel<64, kPages>;
    const size_t bytes = (D == 128 ? kFewSmem<128> : kFewSmem<64>) + kPlanBytes;
    if (int rc = allow_dynamic_lds(reinterpret_cast<const void*>(kernel), bytes, ok[D == 128], who)) return rc;
    kernel<<<blocks, waves * 64, bytes, s>>>(a);
  } else {
    static std::atomic<uint64_t> ok[4];
    const bool unit_c = a.c == 1.0f, many = form == kMany;
    void (*kernel)(RowsArgs);
    if constexpr (kPages)
      kernel = many ? (unit_c ? rows_many_kernel<true> : rows_many_kernel<false>) : (unit_c ? rows_mid_kernel<true> : rows_mid_kernel<false>);
    else
      kernel = unit_c ? rows_prompt_kernel<true> : rows_prompt_kernel<false>;
    constexpr size_t kBytes = std::max(kManySmem, kMidSmem) + (kPages ? kPlanBytes : 0);
    if (int rc = allow_dynamic_lds(reinterpret_cast<const void*>(kernel), kBytes, ok[many * 2 + unit_c], who)) return rc;
    kernel<<<blocks, waves * 64, kBytes, s>>>(a);
  }
  PC_CHECK_LAUNCH(who);
  return PC_OK;
}

}  // namespace
}  // namespace pc

using namespace pc;

extern "C" int pc_prompt_attn(const void* Q, const void* K, const void* V, int dtype, int Hq, int Hkv, int Tq, int Tk,
                              int D, int64_t q_stride_h, int64_t k_stride_h, int64_t v_stride_h, int64_t o_stride_h,
                              float scale, const int32_t* offs_q, const int32_t* offs_k, int n_seq, void* O, float* lse,
                              void* stream) {
  const char* who = "pc_prompt_attn";
  if (int rc = check_attn(who, dtype, Hq, Hkv, D, scale)) return rc;
  PC_REQUIRE(Tq >= 0 && Tk >= 0 && n_seq >= 0, PC_ERR_SHAPE, "%s: Tq=%d Tk=%d n_seq=%d", who, Tq, Tk, n_seq);
  if (n_seq == 0) return PC_OK;
  PC_REQUIRE(offs_q != nullptr, PC_ERR_NULL, "%s: offs_q is NULL", who);
  if (int rc = check_offsets(who, "offs_q", offs_q, n_seq, Tq)) return rc;
  if (offs_k == nullptr) offs_k = offs_q;
  if (int rc = check_offsets(who, "offs_k", offs_k, n_seq, Tk)) return rc;
  if (offs_q[n_seq] == offs_q[0]) return PC_OK;
  const int rep = Hq / Hkv;
  PC_REQUIRE(static_cast<int64_t>(Hq) * Tq <= INT32_MAX / 2 && Tk <= INT32_MAX / 2, PC_ERR_UNSUPPORTED, "%s: %d heads x %d rows, %d keys",
             who, Hq, Tq, Tk);
  PC_REQUIRE(Q && O && (Tk == 0 || (K && V)), PC_ERR_NULL, "%s: Q, K, V or O is NULL", who);
  const int elt = dtype == PC_BF16 ? 2 : 4;
  const int64_t q_rows = static_cast<int64_t>(Tq) * D, k_rows = static_cast<int64_t>(Tk) * D;
  PC_REQUIRE((Hq == 1 || (q_stride_h >= q_rows && o_stride_h >= q_rows)) && (Hkv == 1 || (k_stride_h >= k_rows && v_stride_h >= k_rows)),
             PC_ERR_SHAPE, "%s: a head stride is smaller than the rows it must hold", who);
  PC_REQUIRE(aligned_16B(Q, q_stride_h, elt) && aligned_16B(K, k_stride_h, elt) && aligned_16B(V, v_stride_h, elt) &&
                 aligned_16B(O, o_stride_h, elt), PC_ERR_SHAPE, "%s: tensors and head strides must be 16-byte aligned", who);
  const Extent at_q = {Q, Hq, q_rows * elt, q_stride_h * elt}, at_o = {O, Hq, q_rows * elt, o_stride_h * elt}, at_lse = {lse, 1, 4ll * Hq * Tq, 0};
  for (const Extent& x : {at_q, Extent{Tk > 0 ? K : nullptr, Hkv, k_rows * elt, k_stride_h * elt},
                          Extent{Tk > 0 ? V : nullptr, Hkv, k_rows * elt, v_stride_h * elt}})
    PC_REQUIRE(!meet(at_o, x) && !meet(at_lse, x), PC_ERR_SHAPE, "%s: O and lse may not overlap Q, K or V", who);
  PC_REQUIRE(!meet(at_o, at_lse), PC_ERR_SHAPE, "%s: O and lse overlap", who);
  RowsArgs a = {};
  a.Q = Q, a.K = K, a.V = V, a.O = O, a.lse = lse;
  a.q_stride = q_stride_h, a.k_stride = k_stride_h, a.v_stride = v_stride_h, a.o_stride = o_stride_h;
  a.rep = rep, a.T = Tq, a.by_rep = Divisor(rep), a.by_hkv = Divisor(Hkv);
  set_scale(a, dtype, scale);
  hipStream_t st = static_cast<hipStream_t>(stream);
  // sequences without rows have nothing to do; the longest come first, so that those of a launch are about as long
  std::vector<Seq> seqs;
  try {
    for (int s = 0; s < n_seq; ++s)
      if (offs_q[s + 1] > offs_q[s]) seqs.push_back({offs_q[s], offs_q[s + 1] - offs_q[s], offs_k[s], offs_k[s + 1] - offs_k[s]});
    if (static_cast<int>(seqs.size()) > kSeqs) std::stable_sort(seqs.begin(), seqs.end(), [](const Seq& x, const Seq& y) { return x.nk > y.nk; });
  } catch (const std::bad_alloc&) {
    PC_FAIL(PC_ERR_SHAPE, "%s: no memory for a table of %d sequences", who, n_seq);
  }
  for (size_t s0 = 0; s0 < seqs.size(); s0 += kSeqs) {
    const int n = static_cast<int>(std::min<size_t>(kSeqs, seqs.size() - s0));
    a.seqs.n = n, a.seqs.per = 0;
    const PromptPlan plan(dtype, D, Hkv, rep, seqs.data() + s0, n);
    const int rows = rows_of(plan.form);
    a.n_tiles = 0, a.max_level = 0, a.n_heavy = plan.n_heavy;
    for (int s = 0; s < n; ++s) {
      const Seq& q = seqs[s0 + s];
      a.seqs.q0[s] = q.q0, a.seqs.nq[s] = q.nq, a.seqs.k0[s] = q.k0, a.seqs.nk[s] = q.nk;
      const int tiles = ceil_div(q.nq * rep, rows);
      a.n_tiles += tiles;
      a.max_level = std::max(a.max_level, level_of(q.nq, q.nk, rep, rows) + tiles);
    }
    if (int rc = launch_rows<false>(who, plan.form, dtype, D, a, static_cast<int64_t>(a.n_tiles + a.n_heavy) * Hkv, st)) return rc;
  }
  return PC_OK;
}

extern "C" size_t pc_page_attn_workspace_bytes(int dtype, int Hq, int Hkv, int T, int D, const int32_t* offs, int n_seq,
                                               int max_len, int n_shared) {
  if (dtype < 0 || dtype > 1 || Hkv < 1 || Hq < 1 || Hq % Hkv || T < 1 || n_seq < 1 || max_len < 1 || n_shared < 0 || (D != 64 && D != 128)) return 0;
  if (static_cast<int64_t>(Hq) * T > INT32_MAX / 64 || max_len > INT32_MAX / 2 || n_shared > INT32_MAX / 2) return 0;   // (refused by the call)
  if (offs == nullptr ? T % n_seq != 0 : check_offsets("pc_page_attn_workspace_bytes", "offs", offs, n_seq, T) != PC_OK) return 0;
  size_t most = 0;
  each_launch(offs, n_seq, [&](int s0, int n) {
    most = std::max(most, plan_of(dtype, Hq, Hkv, T, D, offs, n_seq, s0, n, max_len, n_shared).bytes(Hkv, D));
    return PC_OK;
  });
  return most;
}

extern "C" int pc_page_attn(const void* Q, const pc_pages* pages, int dtype, int Hq, int Hkv, int T, int D,
                            int64_t q_stride_h, int64_t o_stride_h, float scale, const int32_t* table, int table_width,
                            int64_t table_stride, const int32_t* lens, const int32_t* offs, int n_seq, int max_len,
                            const int32_t* shared, int n_shared, void* O, float* lse, void* ws, size_t ws_bytes,
                            void* stream) {
  const char* who = "pc_page_attn";
  if (int rc = check_attn(who, dtype, Hq, Hkv, D, scale)) return rc;
  PC_REQUIRE(T >= 0 && n_seq >= 0, PC_ERR_SHAPE, "%s: T=%d n_seq=%d", who, T, n_seq);
  const int elt = dtype == PC_BF16 ? 2 : 4;
  if (int rc = check_pages(who, pages, Hkv, D, elt)) return rc;
  if (T == 0 || n_seq == 0) return PC_OK;
  if (int rc = check_sequences(who, table, table_width, table_stride, lens, offs, n_seq, T)) return rc;
  const int64_t room = static_cast<int64_t>(table_width) * pages->page_rows;
  PC_REQUIRE(max_len >= 1 && max_len <= room && max_len <= INT32_MAX / 2, PC_ERR_SHAPE, "%s: max_len=%d, a table row holds %lld", who, max_len,
             static_cast<long long>(room));
  PC_REQUIRE(n_shared >= 0 && (n_shared == 0) == (shared == nullptr) && n_shared <= INT32_MAX / 2, PC_ERR_SHAPE,
             "%s: n_shared=%d goes with a list of pages", who, n_shared);
  PC_REQUIRE(Q && O, PC_ERR_NULL, "%s: Q or O is NULL", who);
  PC_REQUIRE(static_cast<int64_t>(Hq) * T <= INT32_MAX / 64, PC_ERR_UNSUPPORTED, "%s: %d heads x %d rows", who, Hq, T);
  const int64_t per_head = static_cast<int64_t>(T) * D;
  PC_REQUIRE(Hq == 1 || (q_stride_h >= per_head && o_stride_h >= per_head), PC_ERR_SHAPE, "%s: a head stride is smaller than T*D", who);
  PC_REQUIRE(aligned_16B(Q, q_stride_h, elt) && aligned_16B(O, o_stride_h, elt), PC_ERR_SHAPE,
             "%s: tensors and head strides must be 16-byte aligned", who);
  const Extent at_q = {Q, Hq, per_head * elt, q_stride_h * elt}, at_o = {O, Hq, per_head * elt, o_stride_h * elt}, at_lse = {lse, 1, 4ll * Hq * T, 0};
  PC_REQUIRE(!meet(at_o, at_q) && !meet(at_lse, at_q), PC_ERR_SHAPE,
             "%s: O and lse may not overlap Q: queries are read again behind the first outputs", who);
  const Extent at_k = extent_of(pages->K, *pages, Hkv, D, elt), at_v = extent_of(pages->V, *pages, Hkv, D, elt);
  for (const Extent& x : {at_k, at_v})
    PC_REQUIRE(!meet(at_o, x) && !meet(at_lse, x), PC_ERR_SHAPE, "%s: O and lse may not lie in the pages", who);
  PC_REQUIRE(!meet(at_o, at_lse), PC_ERR_SHAPE, "%s: O and lse overlap", who);
  n_shared = std::min(n_shared, max_len);   // nobody sees more
  // the plan of a call's only launch serves both its workspace and the launch
  const bool one = n_seq <= (offs != nullptr ? kSeqs : kPageSeqs);
  const PagePlan first = plan_of(dtype, Hq, Hkv, T, D, offs, n_seq, 0, std::min(n_seq, offs != nullptr ? kSeqs : kPageSeqs), max_len, n_shared);
  const size_t need = one ? first.bytes(Hkv, D) : pc_page_attn_workspace_bytes(dtype, Hq, Hkv, T, D, offs, n_seq, max_len, n_shared);
  PC_REQUIRE(need == 0 || (ws != nullptr && ws_bytes >= need && reinterpret_cast<uintptr_t>(ws) % 16 == 0), PC_ERR_WORKSPACE,
             "%s: needs %zu bytes of 16-byte aligned workspace, got %zu", who, need, ws_bytes);
  const Extent at_ws = {need > 0 ? ws : nullptr, 1, static_cast<int64_t>(need), 0};
  for (const Extent& x : {at_q, at_o, at_lse, at_k, at_v})
    PC_REQUIRE(!meet(at_ws, x), PC_ERR_WORKSPACE, "%s: the workspace overlaps Q, O, lse or the pages", who);
  const int rep = Hq / Hkv;
  RowsArgs a = {};
  a.Q = Q, a.K = pages->K, a.V = pages->V, a.O = O, a.lse = lse;
  a.q_stride = q_stride_h, a.k_stride = a.v_stride = pages->stride_h, a.o_stride = o_stride_h;
  a.table = table, a.lens = lens, a.shared = shared, a.table_stride = table_stride, a.page_stride = pages->stride_page;
  a.n_pages = pages->n_pages, a.n_shared = n_shared, a.max_len = max_len, a.by_page = Divisor(pages->page_rows);
  a.rep = rep, a.T = T, a.by_rep = Divisor(rep), a.by_hkv = Divisor(Hkv);
  set_scale(a, dtype, scale);
  hipStream_t st = static_cast<hipStream_t>(stream);
  return each_launch(offs, n_seq, [&](int s0, int n) -> int {
    const int32_t* o = offs != nullptr ? offs + s0 : nullptr;
    const int per = o != nullptr ? 0 : T / n_seq, rows = o != nullptr ? T : per * n;
    a.row0 = o != nullptr ? o[0] : 0, a.n_rows = o != nullptr ? o[n] - o[0] : rows;
    if (a.n_rows == 0) return PC_OK;
    a.seqs.n = n, a.seqs.per = per;
    if (o == nullptr) {   // the launch's rows and sequences begin at s0's
      const int64_t at = static_cast<int64_t>(s0) * per;
      a.Q = static_cast<const uint8_t*>(Q) + at * D * elt, a.O = static_cast<uint8_t*>(O) + at * D * elt;
      a.lse = lse != nullptr ? lse + at : nullptr;
      a.table = table + s0 * table_stride, a.lens = lens + s0;
      a.seqs.by_per = Divisor(per);
    } else {
      for (int s = 0; s < n; ++s) a.seqs.q0[s] = o[s], a.seqs.nq[s] = o[s + 1] - o[s], a.seqs.k0[s] = s0 + s;
    }
    const PagePlan plan = s0 == 0 ? first : plan_of(dtype, Hq, Hkv, T, D, offs, n_seq, s0, n, max_len, n_shared);
    a.tiles_per_seq = std::max(1, ceil_div(per * rep, rows_of(plan.form)));
    a.shared_tiles = plan.shared_tiles, a.shared_parts = plan.shared_parts, a.shared_keys = plan.shared_keys;
    a.by_shared_tiles = Divisor(std::max(1, plan.shared_tiles)), a.by_rest = Divisor(std::max(1, plan.shared_parts * Hkv % 8));
    a.own_parts = plan.own_parts, a.own_keys = plan.shared_keys, a.by_parts = Divisor(std::max(1, plan.own_parts * a.tiles_per_seq));
    a.own_cap = plan.own_cap, a.slots = plan.slots, a.slot_rows = plan.slot_rows, a.by_tile = Divisor(rows_of(plan.form));
    a.unit_us = plan.unit_us, a.key_us = plan.key_us;
    a.least_keys = plan.least_keys;
    a.part_o = nullptr, a.part_ml = nullptr, a.cut = nullptr;
    if (plan.joined) {
      auto* at = static_cast<uint8_t*>(ws);
      a.part_o = reinterpret_cast<float*>(at);
      a.part_ml = reinterpret_cast<float2*>(at + plan.o_bytes(Hkv, D));
      a.cut = reinterpret_cast<int*>(at + plan.o_bytes(Hkv, D) + plan.ml_bytes(Hkv));
    }
    if (int rc = launch_rows<true>(who, plan.form, dtype, D, a, static_cast<int64_t>(plan.units()) * Hkv, st)) return rc;
    if (!plan.joined) return PC_OK;
    // Few rows: one per work-group, its shares read by eight groups of threads at once; else eight rows (sixteen at D = 64).  Eight
    // at once | one, whole calls, 16/4 heads, us: 512 rows per head of 9 shares 151 | 142, 256 of 5 shares 53 | 47; 24/8 heads,
    // 64 of 10 shares 72.9 | 75.6.
    const bool few_rows = Hq * a.n_rows <= 2048;
    auto* join = dtype == PC_BF16 ? (D == 128 ? (few_rows ? rows_join_kernel<uint16_t, 128, 8> : rows_join_kernel<uint16_t, 128, 1>)
                                              : (few_rows ? rows_join_kernel<uint16_t, 64, 8> : rows_join_kernel<uint16_t, 64, 1>))
                                  : (D == 128 ? (few_rows ? rows_join_kernel<float, 128, 8> : rows_join_kernel<float, 128, 1>)
                                              : (few_rows ? rows_join_kernel<float, 64, 8> : rows_join_kernel<float, 64, 1>));
    join<<<ceil_div(Hq * a.n_rows, 256 / (D / 4) / (few_rows ? 8 : 1)), 256, 0, st>>>(a);
    PC_CHECK_LAUNCH(who);
    return PC_OK;
  });
}
