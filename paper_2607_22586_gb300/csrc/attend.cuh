// Attention over the paged cache: how its work is cut and shared out.
//
// A unit is (request, KV head, tile of query rows); row rho of a request's
// head is token rho / r and query head h * r + rho % r. Its keys, up to its last
// row's, are cut into pieces of 2^step_shift, and the pieces of all units in
// their order are shared out evenly to the workers (CTAs), however long the
// sequences are: their lengths are read on the device, so every CTA adds up
// the pieces itself. A unit counts for some pieces more, before its first: its
// start and end take a worker about as long. A worker's range covers whole units,
// whose results it writes, and at most two parts of units, its first and its last,
// whose partial sums it leaves for the merge kernel.
#pragma once

#include "cache.cuh"

namespace mmshift {

// Where a worker's share begins: the unit with its first piece, the costs before that.
struct AttendStart {
  int64_t before;
  int32_t unit, unused;
};

struct AttendPlan {
  int32_t uoff[MMSHIFT_MAX_BATCH + 1];  // units, prefix over requests
  int32_t tiles[MMSHIFT_MAX_BATCH];     // a request's row tiles per KV head
  Divisor by_tiles[MMSHIFT_MAX_BATCH];
  int32_t rows;                         // query rows of a tile
  int32_t step_shift, extra, extra1;    // extra1: of units of at most 128 rows
  int32_t workers, least;               // workers at most; one has 2^least pieces where there are as many
  float* po;                            // [2 * workers][rows][d] sums of weights times values
  float2* pml;                          // [2 * workers][rows] their maximum (base 2) and sum of weights
  AttendStart* start;                   // [workers], and one more whose `before` is all units' cost
};

struct AttendUnit {
  int b, h, n;         // request, KV head, the request's tokens
  int row0, rows;      // the tile's first row, its rows
  int len, keys;       // rows of the sequence; keys that the tile's last row attends to
  int pieces, extra;   // its key pieces; what it counts for beside them
  int cost;            // both together, 0 without keys
};

// A sequence's length, from the L2: a merge reads it before its griddepcontrol.wait, when the
// L1 need not have what was written before the attention kernel began.
__device__ __forceinline__ int attend_len(const CacheJob& J, size_t u) {
  return min(max(__ldcg(J.lens + u), 0), J.cap);
}

// lens: the sequences' lengths (AttendScan::lengths), or null to read them from the cache.
__device__ __forceinline__ AttendUnit attend_unit(const AttendJob& A, const AttendPlan& P, const int32_t* lens, int u) {
  const CacheJob& J = A.c;
  AttendUnit x;
  x.b = range_of(P.uoff, J.B, u);
  x.n = J.off[x.b + 1] - J.off[x.b];
  const int all = x.n * J.r, tiles = P.tiles[x.b], rem = u - P.uoff[x.b];
  x.h = P.by_tiles[x.b](rem);
  x.row0 = (rem - x.h * tiles) * P.rows;
  x.rows = min(P.rows, all - x.row0);
  const int seq = x.b * J.Hkv + x.h;
  x.len = lens ? lens[seq] : attend_len(J, seq);
  x.keys = keys_of(A.causal, x.len, x.n, J.by_r(x.row0 + x.rows - 1));
  x.pieces = (x.keys + (1 << P.step_shift) - 1) >> P.step_shift;
  x.extra = x.rows <= 128 ? P.extra1 : P.extra;
  x.cost = x.pieces ? x.pieces + x.extra : 0;
  return x;
}

// A worker's place in the work: [begin, end) of all units' costs, the unit that
// holds the first of them and the costs before that unit.
struct AttendSpan {
  int64_t begin, end, before;
  int unit;
};

// LENS: up to so many sequences' lengths are kept in shared memory.
template <int NT, int LENS = 1024>
struct AttendScan {
  int64_t warp[NT / 32];
  AttendSpan span;
  int32_t lens[LENS];
  __device__ __forceinline__ const int32_t* lengths(const CacheJob& J) const {
    return J.B * J.Hkv <= LENS ? lens : nullptr;
  }
};

// Called by all NT threads of a CTA. Every thread adds up a run of units, [u0, u1);
// `before` are the costs before its run, `sum` the run's, W all units'.
struct AttendSums {
  int u0, u1;
  int64_t before, sum, W;
  template <int NT, int LENS>
  __device__ __forceinline__ AttendSums(const AttendJob& A, const AttendPlan& P, AttendScan<NT, LENS>* s) {
    const CacheJob& J = A.c;
    const int tid = threadIdx.x, lane = tid % 32, w = tid / 32, U = P.uoff[J.B];
    if (s->lengths(J))
      for (int i = tid; i < J.B * J.Hkv; i += NT) s->lens[i] = attend_len(J, i);
    __syncthreads();
    const int per = (U + NT - 1) / NT;
    u0 = min(tid * per, U);
    u1 = min(u0 + per, U);
    sum = 0;
    for (int u = u0; u < u1; ++u) sum += attend_unit(A, P, s->lengths(A.c), u).cost;
    int64_t x = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t y = __shfl_up_sync(0xffffffffu, x, d);
      if (lane >= d) x += y;
    }
    if (lane == 31) s->warp[w] = x;
    __syncthreads();
    W = 0;
    before = x - sum;
#pragma unroll
    for (int i = 0; i < NT / 32; ++i) {
      if (i < w) before += s->warp[i];
      W += s->warp[i];
    }
  }
};

// The CTA's share of the work, as a worker.
template <int NT, int LENS>
__device__ __forceinline__ AttendSpan attend_span(const AttendJob& A, const AttendPlan& P, AttendScan<NT, LENS>* s) {
  const AttendSums x(A, P, s);
  const Shares sh = shares_of(x.W, P.workers, P.least);
  const int i = blockIdx.x;
  const int64_t begin = i < sh.n ? sh.begin(i) : x.W, end = i < sh.n ? sh.begin(i + 1) : x.W;
  if (i == 0 && threadIdx.x == 0) P.start[P.workers].before = x.W;
  if (begin >= end) return AttendSpan{begin, end, 0, 0};
  if (begin >= x.before && begin < x.before + x.sum) {
    int u = x.u0;
    int64_t a = x.before;
    while (x.u1 - x.u0 > 1) {
      const int p = attend_unit(A, P, s->lengths(A.c), u).cost;
      if (a + p > begin) break;
      a += p;
      ++u;
    }
    s->span = AttendSpan{begin, end, a, u};
    P.start[i] = AttendStart{a, u, 0};
  }
  __syncthreads();
  return s->span;
}

// The unit's pieces [s0, s1) among a worker's [begin, end), with `before` before the unit.
__device__ __forceinline__ void attend_pieces(const AttendUnit& U, int64_t begin, int64_t end,
                                              int64_t before, int& s0, int& s1) {
  const int64_t first = before + U.extra;
  s0 = (int)(max(begin, first) - first);
  s1 = (int)max(min(end, first + U.pieces) - first, (int64_t)0);
}

// The partial sums' slot of a worker's part of the unit with `before` before it.
__device__ __forceinline__ int attend_slot(int worker, int64_t begin, int64_t before) {
  return 2 * worker + (before > begin);
}

// Four values of an output row from its sums; a row without weights is zeros.
// `row` counts the rows of the request's KV head.
template <typename T, int D>
__device__ __forceinline__ void attend_write(const AttendJob& A, int b, int h, int row, int d0, float4 v, float top,
                                             float z) {
  const CacheJob& J = A.c;
  const int tok = J.by_r(row);
  const size_t at = (size_t)(J.off[b] + tok) * J.Hq + h * J.r + row - tok * J.r;
  const float f = z == 0.f ? 0.f : 1.f / z;
  T* out = reinterpret_cast<T*>(A.out) + at * D + d0;
  if (z == 0.f) v = make_float4(0.f, 0.f, 0.f, 0.f);
  if constexpr (sizeof(T) == 2) {
    if (A.ovec) {
      *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16(v.x * f, v.y * f), pack_bf16(v.z * f, v.w * f));
    } else {
      out[0] = from_f32<T>(v.x * f);
      out[1] = from_f32<T>(v.y * f);
      out[2] = from_f32<T>(v.z * f);
      out[3] = from_f32<T>(v.w * f);
    }
  } else {
    if (A.ovec) {
      *reinterpret_cast<float4*>(out) = make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
    } else {
      out[0] = v.x * f;
      out[1] = v.y * f;
      out[2] = v.z * f;
      out[3] = v.w * f;
    }
  }
  if (d0 == 0 && A.lse) A.lse[at] = z == 0.f ? -INFINITY : (top + log2f(z)) * 0.6931471805599453f;
}

cudaError_t launch_attend_token(const AttendJob& A, const AttendPlan& P, bool cluster, cudaStream_t st);
cudaError_t launch_attend_simt(const AttendJob& A, const AttendPlan& P, cudaStream_t st);
cudaError_t launch_attend_chunk(const AttendJob& A, const AttendPlan& P, cudaStream_t st);

}  // namespace mmshift
