// pc_page_store: the rows of a step go into a cache held in pages; keys and queries are turned by their (t, h, w) on the
// way (the operator R of Eq. 2).  Bound: HBM, every element is read once and written once (keys twice where the caller
// keeps them), and a launch where there are few rows.  Measured: 8,469 rows of eight prompts, 24/8 heads, bf16, 42 us (191 MB,
// 4.5 TB/s; the kernel alone 33); one row each of 64 sequences, 16/4 heads, 4.6 us.
#include <math.h>

#include <algorithm>

#include "rope.h"
#include "seq.h"

namespace pc {
namespace {

constexpr int kTokPerBlock = 4;
constexpr int kThreads = 256;
constexpr int kHeadsInFlight = 4;

struct StoreArgs {
  const void *K, *V, *Q;
  void *K_out, *Q_out, *K_pages, *V_pages;
  int64_t k_stride, v_stride, q_stride, k_out_stride, q_out_stride;   // between heads, elements
  int64_t page_stride, page_head_stride;
  const int32_t *table, *lens, *pos;
  int64_t table_stride;
  int table_rows, n_pages, Hkv, Hq;     // rows that a sequence's table has room for
  int row0, n_rows;                     // the launch's part of the T rows
  double q_scale;
  Divisor by_page, by_pairs, by_chunks;
  SeqTable seqs;
  RopeFreq freq;
};

// Four rows per work-group, each of all heads.  The places of the rows and the sines are formed first, one per thread,
// with the first elements already on their way; then a thread moves 16 bytes of four heads at a time, the heads in the
// order K, V, Q.
template <typename T, bool kTurn>
__global__ __launch_bounds__(kThreads) void page_store_kernel(StoreArgs a) {
  __shared__ float2 cs_k[kTokPerBlock][kMaxPairs / 2], cs_q[kTokPerBlock][kMaxPairs / 2];
  __shared__ int64_t place[kTokPerBlock];
  constexpr int kElems = 16 / sizeof(T);
  const int tok0 = blockIdx.x * kTokPerBlock;   // in front of row0
  const int chunks = a.by_chunks.d, D = chunks * kElems, pairs = a.by_pairs.d;
  const int groups_kv = (a.Hkv + kHeadsInFlight - 1) / kHeadsInFlight, groups_q = (a.Hq + kHeadsInFlight - 1) / kHeadsInFlight;
  const int total = kTokPerBlock * chunks * (2 * groups_kv + groups_q);

  u32x4 raw[kHeadsInFlight];
  struct Item {
    int kind, h0, t, c;   // 0 K, 1 V, 2 Q
  };
  auto item = [&](int e) {
    const int r = a.by_chunks.of(e);
    int g = r / kTokPerBlock, kind = 0;
    if (g >= groups_kv) g -= groups_kv, kind = 1;
    if (kind == 1 && g >= groups_kv) g -= groups_kv, kind = 2;
    return Item{kind, g * kHeadsInFlight, r % kTokPerBlock, e - r * chunks};
  };
  auto load = [&](int e) {   // what does not exist is read as what does, and never used
    const Item it = item(min(e, total - 1));
    const T* x = static_cast<const T*>(it.kind == 0 ? a.K : it.kind == 1 ? a.V : a.Q);
    const int64_t stride = it.kind == 0 ? a.k_stride : it.kind == 1 ? a.v_stride : a.q_stride;
    const int last = (it.kind == 2 ? a.Hq : a.Hkv) - 1;
    x += static_cast<int64_t>(a.row0 + min(tok0 + it.t, a.n_rows - 1)) * D + it.c * kElems;
#pragma unroll
    for (int i = 0; i < kHeadsInFlight; ++i) raw[i] = *reinterpret_cast<const u32x4*>(x + min(it.h0 + i, last) * stride);
  };
  int e = blockIdx.y * kThreads + threadIdx.x;
  load(e);

  if (threadIdx.x < kTokPerBlock) {
    const int t = a.row0 + min(tok0 + static_cast<int>(threadIdx.x), a.n_rows - 1);
    const int s = seq_of_row(a.seqs, t);
    int64_t at = -1;
    if (s >= 0) {
      const bool even = a.seqs.per > 0;
      const int number = even ? s : a.seqs.k0[s];
      const int end = even ? (s + 1) * a.seqs.per : a.seqs.q0[s] + a.seqs.nq[s];
      const int64_t r = static_cast<int64_t>(a.lens[number]) - (end - t);
      if (r >= 0 && r < a.table_rows) {
        const int in_table = a.by_page.of(static_cast<int>(r));
        const int page = a.table[number * a.table_stride + in_table];
        if (page >= 0 && page < a.n_pages)
          at = page * a.page_stride + static_cast<int64_t>(static_cast<int>(r) - in_table * a.by_page.d) * D;
      }
    }
    place[threadIdx.x] = at;
  }
  if constexpr (kTurn) {
    for (int i = threadIdx.x; i < kTokPerBlock * pairs; i += kThreads) {
      const int t = a.by_pairs.of(i), p = i - t * pairs;
      const int32_t* at = a.pos + static_cast<int64_t>(a.row0 + min(tok0 + t, a.n_rows - 1)) * 3;
      const int axis = a.freq.axis[p];
      double s, c;
      sincos_f64(static_cast<double>(at[axis]) * a.freq.inv_freq[p], &s, &c);
      cs_k[t][p] = make_float2(static_cast<float>(c), static_cast<float>(s));
      cs_q[t][p] = make_float2(static_cast<float>(c * a.q_scale), static_cast<float>(s * a.q_scale));
    }
  }
  __syncthreads();

  while (e < total) {
    const Item it = item(e);
    const bool there = tok0 + it.t < a.n_rows;
    const int64_t row = static_cast<int64_t>(a.row0 + tok0 + it.t) * D + it.c * kElems, to = place[it.t];
    if constexpr (kTurn) {
      if (it.kind != 1) {
#pragma unroll
        for (int i = 0; i < kHeadsInFlight; ++i) turn_16B<T>(raw[i], (it.kind == 0 ? cs_k : cs_q)[it.t] + it.c * (kElems / 2));
      }
    }
#pragma unroll
    for (int i = 0; i < kHeadsInFlight; ++i) {
      const int h = it.h0 + i;
      if (!there || h >= (it.kind == 2 ? a.Hq : a.Hkv)) continue;
      if (it.kind == 2) {
        *reinterpret_cast<u32x4*>(static_cast<T*>(a.Q_out) + h * a.q_out_stride + row) = raw[i];
        continue;
      }
      if (it.kind == 0 && a.K_out != nullptr) *reinterpret_cast<u32x4*>(static_cast<T*>(a.K_out) + h * a.k_out_stride + row) = raw[i];
      if (to >= 0)
        *reinterpret_cast<u32x4*>(static_cast<T*>(it.kind == 0 ? a.K_pages : a.V_pages) + h * a.page_head_stride + to + it.c * kElems) = raw[i];
    }
    e += gridDim.y * kThreads;
    if (e < total) load(e);
  }
}

}  // namespace
}  // namespace pc

using namespace pc;

extern "C" int pc_page_store(const void* K, const void* V, int dtype, int Hkv, int T, int D, int64_t k_stride_h,
                             int64_t v_stride_h, const pc_pages* pages, const int32_t* table, int table_width,
                             int64_t table_stride, const int32_t* lens, const int32_t* offs, int n_seq,
                             const int32_t* pos, int sec_t, int sec_h, int sec_w, double base, void* K_out,
                             int64_t k_out_stride_h, const void* Q, void* Q_out, int Hq, int64_t q_stride_h,
                             int64_t q_out_stride_h, double out_scale, void* stream) {
  const char* who = "pc_page_store";
  PC_REQUIRE(dtype == PC_F32 || dtype == PC_BF16, PC_ERR_DTYPE, "%s: dtype %d", who, dtype);
  PC_REQUIRE(Hkv >= 1 && T >= 0 && n_seq >= 0, PC_ERR_SHAPE, "%s: Hkv=%d T=%d n_seq=%d", who, Hkv, T, n_seq);
  PC_REQUIRE(D == 64 || D == 128, PC_ERR_UNSUPPORTED, "%s: D=%d (64 or 128)", who, D);
  PC_REQUIRE((Q == nullptr) == (Q_out == nullptr), PC_ERR_NULL, "%s: Q and Q_out go together", who);
  PC_REQUIRE(Q == nullptr || pos != nullptr, PC_ERR_NULL, "%s: queries are only turned, and there is no pos", who);
  if (pos != nullptr) {
    const int secs[3] = {sec_t, sec_h, sec_w};
    for (int i = 0; i < 3; ++i)
      PC_REQUIRE(secs[i] >= 0 && secs[i] % 2 == 0, PC_ERR_SHAPE, "%s: section %d has width %d (must be even, >= 0)", who, i, secs[i]);
    PC_REQUIRE(static_cast<int64_t>(sec_t) + sec_h + sec_w == D, PC_ERR_SHAPE, "%s: sections %d+%d+%d != D=%d", who, sec_t, sec_h, sec_w, D);
    PC_REQUIRE(base > 0.0, PC_ERR_SHAPE, "%s: base %g", who, base);
    PC_REQUIRE(out_scale > 0.0 && isfinite(out_scale), PC_ERR_SHAPE, "%s: out_scale %g must be > 0", who, out_scale);
  }
  const int elt = dtype == PC_BF16 ? 2 : 4;
  if (int rc = check_pages(who, pages, Hkv, D, elt)) return rc;
  if (T == 0 || n_seq == 0) return PC_OK;
  PC_REQUIRE(K && V, PC_ERR_NULL, "%s: K or V is NULL", who);
  if (int rc = check_sequences(who, table, table_width, table_stride, lens, offs, n_seq, T)) return rc;
  PC_REQUIRE(static_cast<int64_t>(table_width) * pages->page_rows <= INT32_MAX, PC_ERR_SHAPE, "%s: a table of %d pages of %d rows", who,
             table_width, pages->page_rows);
  const int64_t per_head = static_cast<int64_t>(T) * D;
  PC_REQUIRE(Hkv == 1 || (k_stride_h >= per_head && v_stride_h >= per_head && (K_out == nullptr || k_out_stride_h >= per_head)), PC_ERR_SHAPE,
             "%s: a head stride is smaller than T*D", who);
  PC_REQUIRE(aligned_16B(K, k_stride_h, elt) && aligned_16B(V, v_stride_h, elt) && aligned_16B(K_out, k_out_stride_h, elt), PC_ERR_SHAPE,
             "%s: tensors and head strides must be 16-byte aligned", who);
  if (Q != nullptr) {
    PC_REQUIRE(Hq >= 1 && (Hq == 1 || (q_stride_h >= per_head && q_out_stride_h >= per_head)), PC_ERR_SHAPE,
               "%s: Hq=%d, or a head stride smaller than T*D", who, Hq);
    PC_REQUIRE(aligned_16B(Q, q_stride_h, elt) && aligned_16B(Q_out, q_out_stride_h, elt), PC_ERR_SHAPE,
               "%s: tensors and head strides must be 16-byte aligned", who);
  }
  // what is written is nobody's input, but for rows that take the place of their own
  const int64_t bytes = per_head * elt;
  const Extent at_k = {K, Hkv, bytes, k_stride_h * elt}, at_v = {V, Hkv, bytes, v_stride_h * elt}, at_q = {Q, Hq, bytes, q_stride_h * elt},
               to_k = {K_out, Hkv, bytes, k_out_stride_h * elt}, to_q = {Q_out, Hq, bytes, q_out_stride_h * elt};
  PC_REQUIRE(to_k.is(at_k) || !meet(to_k, at_k), PC_ERR_SHAPE, "%s: K_out is neither K nor apart from it", who);
  PC_REQUIRE(to_q.is(at_q) || !meet(to_q, at_q), PC_ERR_SHAPE, "%s: Q_out is neither Q nor apart from it", who);
  PC_REQUIRE(!meet(to_k, at_v) && !meet(to_k, at_q) && !meet(to_q, at_k) && !meet(to_q, at_v) && !meet(to_k, to_q), PC_ERR_SHAPE,
             "%s: K_out or Q_out overlaps another input or each other", who);
  for (const void* p : {pages->K, pages->V}) {
    const Extent to = extent_of(p, *pages, Hkv, D, elt);
    PC_REQUIRE(!meet(to_k, to) && !meet(to_q, to), PC_ERR_SHAPE, "%s: K_out and Q_out may not lie in the pages", who);
  }
  const bool turn = pos != nullptr;
  StoreArgs a = {};
  a.K = K, a.V = V, a.Q = Q, a.K_out = K_out, a.Q_out = Q_out, a.K_pages = pages->K, a.V_pages = pages->V;
  a.k_stride = k_stride_h, a.v_stride = v_stride_h, a.q_stride = q_stride_h, a.k_out_stride = k_out_stride_h, a.q_out_stride = q_out_stride_h;
  a.page_stride = pages->stride_page, a.page_head_stride = pages->stride_h;
  a.table = table, a.lens = lens, a.pos = pos, a.table_stride = table_stride;
  a.table_rows = table_width * pages->page_rows, a.n_pages = pages->n_pages, a.Hkv = Hkv, a.Hq = Q != nullptr ? Hq : 0;
  a.q_scale = out_scale;
  a.by_page = Divisor(pages->page_rows), a.by_pairs = Divisor(D / 2), a.by_chunks = Divisor(D * elt / 16);
  if (turn) {
    const int secs[3] = {sec_t, sec_h, sec_w};
    a.freq = rope_freq(secs, base);
  }
  const int items = kTokPerBlock * a.by_chunks.d * (2 * ceil_div(Hkv, kHeadsInFlight) + ceil_div(a.Hq, kHeadsInFlight));
  hipStream_t st = static_cast<hipStream_t>(stream);
  auto launch = [&](int row0, int n_rows) -> int {
    constexpr int kMost = static_cast<int>(kMaxThreads / kThreads) * kTokPerBlock;   // rows of a launch
    for (int done = 0; done < n_rows; done += a.n_rows) {
      a.row0 = row0 + done, a.n_rows = std::min(n_rows - done, kMost);
      const int blocks = ceil_div(a.n_rows, kTokPerBlock);
      const dim3 grid(blocks, std::min(ceil_div(items, kThreads), ceil_div(512, blocks)));
      auto* kernel = dtype == PC_BF16 ? (turn ? page_store_kernel<uint16_t, true> : page_store_kernel<uint16_t, false>)
                                      : (turn ? page_store_kernel<float, true> : page_store_kernel<float, false>);
      kernel<<<grid, kThreads, 0, st>>>(a);
      PC_CHECK_LAUNCH(who);
    }
    return PC_OK;
  };
  if (offs == nullptr) {
    a.seqs.n = n_seq, a.seqs.per = T / n_seq, a.seqs.by_per = Divisor(T / n_seq);
    return launch(0, T);
  }
  for (int s0 = 0; s0 < n_seq; s0 += kSeqs) {
    const int n = std::min(kSeqs, n_seq - s0), rows = offs[s0 + n] - offs[s0];
    if (rows == 0) continue;
    a.seqs.n = n, a.seqs.per = 0;
    for (int s = 0; s < n; ++s) a.seqs.q0[s] = offs[s0 + s], a.seqs.nq[s] = offs[s0 + s + 1] - offs[s0 + s], a.seqs.k0[s] = s0 + s;
    if (int rc = launch(offs[s0], rows)) return rc;
  }
  return PC_OK;
}
