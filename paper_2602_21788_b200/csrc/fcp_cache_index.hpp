// Where the tokens of a paged cache lie, and what of a batch's contents is usable.  Plain integer arithmetic, shared by the
// kernels and by host code that checks it without a GPU.
#pragma once
#include <cstdint>

#ifdef __CUDACC__
#define FCP_HD __host__ __device__ __forceinline__
#else
#define FCP_HD inline
#endif

namespace fcp {

// The new tokens of one sequence: rows [row0, row0 + n) of the call's tensors are its last n tokens of `length`.
struct SeqView {
  int32_t row0, n, length;
  int32_t bad;                 // 0, or the FCP_CACHE_BAD_* code that makes the sequence absent (n = length = 0 then)
};

FCP_HD SeqView seq_view(int32_t begin, int32_t end, int32_t length, int32_t rows, int32_t max_new, int32_t capacity) {
  SeqView s = {0, 0, 0, 0};
  if (begin < 0 || end < begin || end > rows || end - begin > max_new) s.bad = 1002;
  if (length < 0 || length > capacity) s.bad = 1001;
  if (!s.bad) {
    s.row0 = begin;
    s.n = end - begin;
    s.length = length;
  }
  return s;
}

// First row of a page's head in a [n_pages][hkv][page_tokens] array, or -1 for a page that does not exist.  The row count is
// below 2^31 (checked when the handle is made); byte offsets are formed in 64 bits from it.
FCP_HD int32_t page_row(int32_t page, int32_t n_pages, int32_t hkv, int32_t head, int32_t page_tokens) {
  return page < 0 || page >= n_pages ? -1 : (page * hkv + head) * page_tokens;
}

// Pages that new tokens touch are worked on as slots: sequence b owns the slots [append_slot(begin_b, b), append_slot(begin_{b+1}, b+1)).
// n tokens touch at most n / p + 2 pages of p tokens (one if there is one token), and the difference of two neighbouring
// values is at least that, because floor((x + n) / p) >= floor(x / p) + floor(n / p).
FCP_HD int32_t append_slot(int32_t row_offset, int32_t b, int32_t page_tokens) { return row_offset / page_tokens + 2 * b; }

// Tokens [lo, hi) (positions in the sequence) that slot `i` of a sequence adds, and the page they lie in; none if lo >= hi.
struct AppendSpan {
  int32_t page, lo, hi;        // index into the page table row
};
FCP_HD AppendSpan append_span(const SeqView& s, int32_t i, int32_t page_tokens) {
  int32_t start = s.length - s.n;
  if (start < 0) start = 0;    // rows in front of the sequence's first token are no tokens
  const int32_t page = start / page_tokens + i;
  const int64_t p0 = (int64_t)page * page_tokens, p1 = p0 + page_tokens;
  AppendSpan a;
  a.page = page;
  a.lo = p0 > start ? (int32_t)(p0 < s.length ? p0 : s.length) : start;
  a.hi = p1 < s.length ? (int32_t)p1 : s.length;
  if (s.n <= 0) a.hi = a.lo;
  return a;
}

}  // namespace fcp
