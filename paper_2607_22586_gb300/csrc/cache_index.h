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

// Where the rows of a call end in a sequence of which the device was told `len` rows: positions
// from the table's end on exist for no row, so a full sequence's rows stay what they are. A number
// that is no length (no table holds more than 2^30 rows) counts as the table's end.
MMSHIFT_HD int append_end(int len, int cap) { return len > 1 << 30 ? cap : len > 0 ? len : 0; }

// Keys that token i of a request's n tokens attends to in a sequence of len rows.
MMSHIFT_HD int keys_of(int causal, int len, int n, int i) {
  const int e = causal ? len - n + i + 1 : len;
  return e > 0 ? e : 0;
}

// Whether a block of the chunk kernel may wait for the V of key tile `s` of a run that
// begins at tile `s0` before it has waited for the tile's S. A wait by parity tells
// neighbouring fills of a stage apart and no others, so the fill before the wanted one has to be
// known to be complete. Behind a run's first tile it is: S of the tile before says that all
// fills up to that tile's K are. At the first tile the block may come from a run that it took no
// part in, many rounds ahead of the ring; then S of the tile itself says so.
MMSHIFT_HD bool v_before_s(int s, int s0) { return s > s0; }

// Division of 0 <= x < 2^31 by a number d >= 1 known on the host, as one high product:
// with L the least L such that d <= 2^L, m = ceil(2^(31 + L) / d) < 2^32 gives
// floor(x / d) = floor(x m / 2^(31 + L)) (Granlund and Montgomery, 1994).
struct Divisor {
  uint32_t m;      // 0: d = 1
  int32_t shift;   // L - 1
  MMSHIFT_HD int operator()(int x) const {
#if defined(__CUDA_ARCH__)
    return m ? (int)(__umulhi((uint32_t)x, m) >> shift) : x;
#else
    return m ? (int)((uint32_t)(((uint64_t)(uint32_t)x * m) >> 32) >> shift) : x;
#endif
  }
};

inline Divisor divisor_of(int32_t d) {
  Divisor r = {0, 0};
  if (d <= 1) return r;
  int L = 1;
  while (((int64_t)1 << L) < d) ++L;
  r.m = (uint32_t)((((uint64_t)1 << (31 + L)) + d - 1) / d);
  r.shift = L - 1;
  return r;
}

// x / y for 0 <= x, 0 < y; 64-bit division only where it is needed.
MMSHIFT_HD int64_t quotient(int64_t x, int64_t y) {
  if (((uint64_t)x | (uint64_t)y) >> 32) return x / y;
  return (uint32_t)x / (uint32_t)y;
}

// W pieces of work shared out in order to n workers, `most` at most and each with
// 2^least pieces where there are as many: the first `more` get base + 1, the others
// base. Worker i has [begin(i), begin(i + 1)); of(x) is the worker that has piece x.
struct Shares {
  int64_t base;
  int32_t n, more;
  MMSHIFT_HD int64_t begin(int i) const { return base * i + (i < more ? i : more); }
  MMSHIFT_HD int of(int64_t x) const {
    const int64_t t = (base + 1) * more;
    return (int)(x < t ? quotient(x, base + 1) : more + quotient(x - t, base));
  }
};

MMSHIFT_HD Shares shares_of(int64_t W, int most, int least) {
  const int64_t want = (W + (1 << least) - 1) >> least;
  Shares s;
  s.n = want < 1 ? 1 : want < most ? (int)want : most;
  s.base = quotient(W, s.n);
  s.more = (int)(W - s.base * s.n);
  return s;
}

}  // namespace mmshift
