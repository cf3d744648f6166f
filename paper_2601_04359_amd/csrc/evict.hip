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

constexpr int kSelThreads = 1024;

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

// One selection head's rows: anchors and recent rows rank above every weight.
struct HeadRanks {
  const float* w;
  const int32_t* t;
  int64_t newest;
  int n_anchor, recent_t;
  __device__ HeadRanks(const Ranks& a, int sel)
      : w(a.weights + sel * a.w_stride_h), t(a.recent_t > 0 ? a.pos + sel * a.pos_stride_h : nullptr),
        newest(a.recent_t > 0 ? t[static_cast<int64_t>(a.Nk - 1) * 3] : 0), n_anchor(a.n_anchor), recent_t(a.recent_t) {}
  __device__ __forceinline__ uint32_t of(int j) const {
    const bool safe = j < n_anchor || (t != nullptr && t[static_cast<int64_t>(j) * 3] > newest - recent_t);
    return safe ? 0xffffffffu : weight_rank(w[j]);
  }
};

// exclusive sum over the work-group, and the total; s: one word per wave
__device__ __forceinline__ int block_scan(int v, int* s, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int x = v;
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  __syncthreads();
  if (lane == 63) s[wave] = x;
  __syncthreads();
  int before = 0;
  total = 0;
  for (int k = 0; k < kSelThreads / 64; ++k) {
    if (k < wave) before += s[k];
    total += s[k];
  }
  return before + x - v;
}

// lists: per selection head `room` holes, then `room` movers
__global__ __launch_bounds__(kSelThreads) void evict_select_kernel(Ranks a, int room, int32_t* __restrict__ counts,
                                                                   int32_t* __restrict__ lists, int32_t* __restrict__ idx,
                                                                   int64_t idx_stride_h) {
  __shared__ int hist[256];
  __shared__ int s_scan[kSelThreads / 64];
  __shared__ int s_bin, s_left;
  const int sel = blockIdx.x;
  const HeadRanks rank(a, sel);
  uint32_t prefix = 0;
  int left = a.n_keep;                    // rows to keep among those that share the prefix
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (threadIdx.x < 256) hist[threadIdx.x] = 0;
    __syncthreads();
    for (int j = threadIdx.x; j < a.Nk; j += kSelThreads) {
      const uint32_t k = rank.of(j);
      if (shift == 24 || k >> (shift + 8) == prefix >> (shift + 8)) atomicAdd(&hist[k >> shift & 255], 1);
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      int b = 255, n = left;
      while (hist[b] < n) n -= hist[b--];
      s_bin = b;
      s_left = n;
    }
    __syncthreads();
    prefix |= static_cast<uint32_t>(s_bin) << shift;
    left = s_left;
    __syncthreads();
  }
  int32_t* holes = lists + static_cast<int64_t>(sel) * 2 * room;
  int32_t* movers = holes + room;
  int ties = 0, n_holes = 0, n_movers = 0;
  for (int j0 = 0; j0 < a.Nk; j0 += kSelThreads) {
    const int j = j0 + threadIdx.x;
    const uint32_t k = j < a.Nk ? rank.of(j) : 0;
    const bool tie = j < a.Nk && k == prefix;
    int total;
    const int nth = ties + block_scan(tie, s_scan, total);
    ties += total;
    const bool keep = j < a.Nk && (k > prefix || (tie && nth < left));
    const bool hole = j < a.n_keep && !keep, mover = j >= a.n_keep && keep;
    const int at_h = n_holes + block_scan(hole, s_scan, total);
    n_holes += total;
    const int at_m = n_movers + block_scan(mover, s_scan, total);
    n_movers += total;
    if (hole) holes[at_h] = j;
    if (mover) movers[at_m] = j;
    if (idx != nullptr && keep && j < a.n_keep) idx[sel * idx_stride_h + j] = j;
  }
  if (threadIdx.x == 0) counts[sel] = n_holes;
}

// What moves with a row: planes of whole words, one run of words per row.
constexpr int kMaxPlanes = 6;
struct Planes {
  uint16_t* base[kMaxPlanes];
  int64_t stride_h[kMaxPlanes];     // in 2-byte units
  int words[kMaxPlanes];            // 2-byte units of a row
  int n_heads_planes, n;            // the first planes are of every head, the rest of a selection head
};

__global__ __launch_bounds__(256) void evict_move_kernel(Planes p, int per, int room, const int32_t* __restrict__ counts,
                                                         const int32_t* __restrict__ lists, int32_t* __restrict__ idx,
                                                         int64_t idx_stride_h) {
  const int lane = threadIdx.x & 63;
  const int h = blockIdx.y, sel = h / per;
  const bool first = h == sel * per;
  const int n = counts[sel];
  const int32_t* holes = lists + static_cast<int64_t>(sel) * 2 * room;
  for (int i = blockIdx.x * 4 + (threadIdx.x >> 6); i < n; i += gridDim.x * 4) {
    const int64_t to = holes[i], from = holes[room + i];
    for (int q = 0; q < p.n; ++q) {
      if (q >= p.n_heads_planes && !first) break;
      uint16_t* base = p.base[q] + (q < p.n_heads_planes ? h : sel) * p.stride_h[q];
      for (int w = lane; w < p.words[q]; w += 64) base[to * p.words[q] + w] = base[from * p.words[q] + w];
    }
    if (idx != nullptr && first && lane == 0) idx[sel * idx_stride_h + to] = static_cast<int32_t>(from);
  }
}

constexpr size_t kWsAlign = 256;
int list_room(int Nk, int n_keep) { return std::min(Nk - n_keep, n_keep); }

int evict(const char* who, Planes p, int H, int32_t* pos, int64_t pos_stride_h, float* weights, int64_t w_stride_h, int Hsel,
          int Nk, int n_keep, int n_anchor, int recent_t, int32_t* idx_out, int64_t idx_stride_h, void* ws, size_t ws_bytes,
          void* stream) {
  PC_REQUIRE(H > 0 && Hsel > 0 && Hsel <= H && H % Hsel == 0, PC_ERR_SHAPE, "%s: %d selection heads for %d heads", who, Hsel, H);
  PC_REQUIRE(H <= 65535, PC_ERR_SHAPE, "%s: %d heads in one call", who, H);
  PC_REQUIRE(Nk >= 0 && Nk <= (1 << 30), PC_ERR_SHAPE, "%s: Nk=%d", who, Nk);
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
  const int room = list_room(Nk, n_keep);
  const size_t lists_at = align_up(static_cast<size_t>(Hsel) * 4, kWsAlign);
  const size_t bytes = lists_at + static_cast<size_t>(Hsel) * 2 * room * 4;
  PC_REQUIRE(ws && ws_bytes >= bytes && reinterpret_cast<uintptr_t>(ws) % 16 == 0, PC_ERR_WORKSPACE,
             "%s: needs %zu bytes of 16-byte aligned workspace, got %zu", who, bytes, ws_bytes);
  auto plane = [&](void* base, int64_t stride_bytes, int row_bytes) {
    p.base[p.n] = static_cast<uint16_t*>(base);
    p.stride_h[p.n] = stride_bytes / 2;
    p.words[p.n++] = row_bytes / 2;
  };
  p.n_heads_planes = p.n;
  if (pos) plane(pos, pos_stride_h * 4, 12);
  plane(weights, w_stride_h * 4, 4);
  hipStream_t s = static_cast<hipStream_t>(stream);
  auto* counts = static_cast<int32_t*>(ws);
  auto* lists = reinterpret_cast<int32_t*>(static_cast<uint8_t*>(ws) + lists_at);
  const Ranks a = {weights, pos, w_stride_h, pos_stride_h, Nk, n_keep, n_anchor, recent_t};
  evict_select_kernel<<<Hsel, kSelThreads, 0, s>>>(a, room, counts, lists, idx_out, idx_stride_h);
  PC_CHECK_LAUNCH(who);
  evict_move_kernel<<<dim3(std::min(ceil_div(room, 4), 1024), H), 256, 0, s>>>(p, H / Hsel, room, counts, lists, idx_out,
                                                                             idx_stride_h);
  PC_CHECK_LAUNCH(who);
  return PC_OK;
}

}  // namespace
}  // namespace pc

using namespace pc;

extern "C" size_t pc_evict_workspace_bytes(int Hsel, int Nk, int n_keep) {
  if (Hsel <= 0 || Nk <= 0 || n_keep <= 0 || n_keep >= Nk) return 0;
  return align_up(static_cast<size_t>(Hsel) * 4, kWsAlign) + static_cast<size_t>(Hsel) * 2 * list_room(Nk, n_keep) * 4;
}

extern "C" int pc_evict(void* K, void* V, int dtype, int H, int D, int64_t k_stride_h, int64_t v_stride_h, int32_t* pos,
                        int64_t pos_stride_h, float* weights, int64_t weights_stride_h, int Hsel, int Nk, int n_keep,
                        int n_anchor, int recent_t, int32_t* idx_out, int64_t idx_stride_h, void* ws, size_t ws_bytes,
                        void* stream) {
  const char* who = "pc_evict";
  PC_REQUIRE(dtype == PC_F32 || dtype == PC_BF16, PC_ERR_DTYPE, "%s: dtype %d", who, dtype);
  PC_REQUIRE(D > 0 && D <= 1024 && D % 8 == 0, PC_ERR_UNSUPPORTED, "%s: D=%d must be a multiple of 8, at most 1024", who, D);
  PC_REQUIRE(K && V, PC_ERR_NULL, "%s: K or V is NULL", who);
  PC_REQUIRE(H <= 1 || (k_stride_h >= static_cast<int64_t>(Nk) * D && v_stride_h >= static_cast<int64_t>(Nk) * D), PC_ERR_SHAPE,
             "%s: a head stride is smaller than rows*D", who);
  const int elt = dtype == PC_BF16 ? 2 : 4;
  PC_REQUIRE((reinterpret_cast<uintptr_t>(K) | reinterpret_cast<uintptr_t>(V) | k_stride_h * elt | v_stride_h * elt) % 16 == 0,
             PC_ERR_SHAPE, "%s: K, V and their head strides must be 16-byte aligned", who);
  Planes p = {};
  p.base[0] = static_cast<uint16_t*>(K), p.base[1] = static_cast<uint16_t*>(V);
  p.stride_h[0] = k_stride_h * elt / 2, p.stride_h[1] = v_stride_h * elt / 2;
  p.words[0] = p.words[1] = D * elt / 2;
  p.n = 2;
  return evict(who, p, H, pos, pos_stride_h, weights, weights_stride_h, Hsel, Nk, n_keep, n_anchor, recent_t, idx_out,
               idx_stride_h, ws, ws_bytes, stream);
}

extern "C" int pc_q4_evict(const pc_q4_cache* cache, int H, int D, int32_t* pos, int64_t pos_stride_h, float* weights,
                           int64_t weights_stride_h, int Hsel, int Nk, int n_keep, int n_anchor, int recent_t,
                           int32_t* idx_out, int64_t idx_stride_h, void* ws, size_t ws_bytes, void* stream) {
  const char* who = "pc_q4_evict";
  PC_REQUIRE(D == 64 || D == 128, PC_ERR_UNSUPPORTED, "%s: needs D = 64 or 128, got %d", who, D);
  if (int rc = check_q4_cache(cache, D, who)) return rc;
  if (int rc = check_q4_span(cache, H, 0, Nk, D, who)) return rc;
  Planes p = {};
  uint8_t* const planes[4] = {cache->k_codes, cache->v_codes, cache->k_scales, cache->v_scales};
  for (int i = 0; i < 4; ++i) {
    p.base[i] = reinterpret_cast<uint16_t*>(planes[i]);
    p.stride_h[i] = (i < 2 ? cache->code_stride_h : cache->scale_stride_h) / 2;
    p.words[i] = (i < 2 ? D / 2 : D / 32) / 2;
  }
  p.n = 4;
  return evict(who, p, H, pos, pos_stride_h, weights, weights_stride_h, Hsel, Nk, n_keep, n_anchor, recent_t, idx_out,
               idx_stride_h, ws, ws_bytes, stream);
}
