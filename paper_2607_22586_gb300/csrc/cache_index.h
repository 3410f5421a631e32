// Index arithmetic of the paged cache, for the host and the device: which request
// a row belongs to, where a position lies, which keys a row attends to, and how
// attention's work is shared out.
#pragma once

#include <stdint.h>

#if defined(__CUDACC__)
#define MMSHIFT_HD __host__ __device__ __forceinline__
#else
#define MMSHIFT_HD inline
#endif

namespace mmshift {

// The b with off[b] <= x < off[b + 1]; 0 <= x < off[n]. Empty ranges are passed over.
MMSHIFT_HD int range_of(const int32_t* off, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (off[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

// The pool's row of the position `t` whose table entry is `page`, -1 if the
// entry is outside the pool.
MMSHIFT_HD int32_t page_row(int32_t page, int32_t n_pages, int page_shift, int t) {
  if (page < 0 || page >= n_pages) return -1;
  return (page << page_shift) + (t & ((1 << page_shift) - 1));   // the pool's rows are below 2^31
}

// Keys that token i of a request's n tokens attends to in a sequence of len rows.
MMSHIFT_HD int keys_of(int causal, int len, int n, int i) {
  const int e = causal ? len - n + i + 1 : len;
  return e > 0 ? e : 0;
}

// W pieces of work are shared out to n workers in order: worker i takes
// [span_begin(W, n, i), span_begin(W, n, i + 1)), which differ by one piece at most.
MMSHIFT_HD int64_t span_begin(int64_t W, int n, int i) { return W * i / n; }

// The worker that has piece x.
MMSHIFT_HD int span_of(int64_t W, int n, int64_t x) { return (int)(((x + 1) * n - 1) / W); }

// Workers that W pieces occupy, each with `least` pieces where there are as many.
MMSHIFT_HD int span_workers(int64_t W, int most, int least) {
  const int64_t n = (W + least - 1) / least;
  return n < 1 ? 1 : n < most ? (int)n : most;
}

}  // namespace mmshift
