// Several sequences in one call (gfx950 only): whose rows are whose, pages, and the checks that the calls share.
#pragma once

#include "common.h"

namespace pc {

constexpr int kSeqs = 64;        // sequences of one launch's table: one per lane of a wave
constexpr int kPageStep = 64;    // pages are a multiple of this many rows: no tile of keys crosses one

constexpr int64_t kMaxThreads = UINT32_MAX;   // of a launch along one axis

// The sequences of a launch, by value.  per > 0: `n` sequences of `per` rows each, and the arrays are not looked at.
struct SeqTable {
  int n, per;
  Divisor by_per;
  int q0[kSeqs], nq[kSeqs];   // first row and rows
  int k0[kSeqs], nk[kSeqs];   // keys (pc_prompt_attn); pages: k0 is the sequence's number
  SeqTable() : n(0), per(0), by_per(1) {}
};

// The sequence that row t belongs to, among those of a launch; -1: none.
__device__ __forceinline__ int seq_of_row(const SeqTable& seqs, int t) {
  if (seqs.per > 0) {
    const int s = seqs.by_per.of(t);
    return s < seqs.n ? s : -1;
  }
  int at = -1;
  for (int s = 0; s < seqs.n; ++s) at = t >= seqs.q0[s] && t < seqs.q0[s] + seqs.nq[s] ? s : at;
  return at;
}

// offs as the calls take it: not descending, from 0 up to T at most.
inline int check_offsets(const char* who, const char* name, const int32_t* offs, int n_seq, int T) {
  PC_REQUIRE(offs[0] >= 0 && offs[n_seq] <= T, PC_ERR_SHAPE, "%s: %s from %d to %d of %d rows", who, name, offs[0], offs[n_seq], T);
  for (int s = 0; s < n_seq; ++s)
    PC_REQUIRE(offs[s] <= offs[s + 1], PC_ERR_SHAPE, "%s: %s[%d] = %d is above the next, %d", who, name, s, offs[s], offs[s + 1]);
  return PC_OK;
}

inline bool aligned_16B(const void* p, int64_t stride, int elt) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * elt % 16 == 0;
}

// What a tensor takes of the memory: n heads of `bytes` each, and where it is a cache in pages, as many of them `page_stride` apart.
// Strides in bytes.
struct Extent {
  const void* at;
  int n;
  int64_t bytes, stride;
  int pages = 1;
  int64_t page_stride = 0;
  int64_t span() const { return (n - 1) * stride + (pages - 1) * page_stride + bytes; }
  bool is(const Extent& y) const { return at == y.at && n == y.n && bytes == y.bytes && (n == 1 || stride == y.stride); }
};
// Whether two of them have a byte in common.  At most one is in pages.
inline bool meet(const Extent& x, const Extent& y) {
  if (x.pages > 1) return meet(y, x);
  if (x.at == nullptr || y.at == nullptr) return false;
  const int64_t gap = static_cast<int64_t>(reinterpret_cast<uintptr_t>(y.at) - reinterpret_cast<uintptr_t>(x.at));
  if (gap >= x.span() || -gap >= y.span()) return false;
  // whether for an r of 0 .. n - 1 the y.bytes from d + r step on meet the x.bytes from 0 on: the first r that ends behind 0
  auto any = [&](int64_t d, int64_t step, int n) {
    const int64_t r = d > -y.bytes || n == 1 ? 0 : (-y.bytes - d) / step + 1;
    return r < n && d + r * step > -y.bytes && d + r * step < x.bytes;
  };
  for (int i = 0; i < x.n; ++i) {
    const int64_t d = gap - i * x.stride;
    if (y.pages == 1) {
      if (any(d, y.stride, y.n)) return true;
    } else {
      for (int j = 0; j < y.n; ++j)
        if (any(d + j * y.stride, y.page_stride, y.pages)) return true;
    }
  }
  return false;
}

inline int check_pages(const char* who, const pc_pages* pages, int Hkv, int D, int elt) {
  PC_REQUIRE(pages != nullptr && pages->K != nullptr && pages->V != nullptr, PC_ERR_NULL, "%s: pages are NULL", who);
  const int64_t rows = static_cast<int64_t>(pages->page_rows) * D;
  PC_REQUIRE(pages->n_pages >= 1 && pages->page_rows >= kPageStep && pages->page_rows % kPageStep == 0, PC_ERR_SHAPE,
             "%s: %d pages of %d rows (at least one, rows a multiple of %d)", who, pages->n_pages, pages->page_rows, kPageStep);
  PC_REQUIRE((Hkv == 1 || pages->stride_h >= rows) && (pages->n_pages == 1 || pages->stride_page >= rows), PC_ERR_SHAPE,
             "%s: strides %lld, %lld of pages of %d x %d", who, static_cast<long long>(pages->stride_page),
             static_cast<long long>(pages->stride_h), pages->page_rows, D);
  PC_REQUIRE(aligned_16B(pages->K, pages->stride_page, elt) && aligned_16B(pages->V, pages->stride_h, elt), PC_ERR_SHAPE,
             "%s: pages and their strides must be 16-byte aligned", who);
  return PC_OK;
}

inline Extent extent_of(const void* pages_kv, const pc_pages& p, int Hkv, int D, int elt) {
  return {pages_kv, Hkv, static_cast<int64_t>(p.page_rows) * D * elt, p.stride_h * elt, p.n_pages, p.stride_page * elt};
}

// table, lens and offs of the two calls on pages
inline int check_sequences(const char* who, const int32_t* table, int table_width, int64_t table_stride, const int32_t* lens,
                           const int32_t* offs, int n_seq, int T) {
  PC_REQUIRE(table != nullptr && lens != nullptr, PC_ERR_NULL, "%s: table or lens is NULL", who);
  PC_REQUIRE(table_width >= 1 && (n_seq == 1 || table_stride >= table_width), PC_ERR_SHAPE, "%s: table of %d pages at stride %lld", who,
             table_width, static_cast<long long>(table_stride));
  if (offs != nullptr) return check_offsets(who, "offs", offs, n_seq, T);
  PC_REQUIRE(T % n_seq == 0, PC_ERR_SHAPE, "%s: %d rows of %d sequences, and no offsets", who, T, n_seq);
  return PC_OK;
}

}  // namespace pc
