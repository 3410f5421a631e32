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
#include "prompt_index.h"

namespace mmshift {

static_assert(kPromptRequests == MMSHIFT_MAX_BATCH, "requests of a call");

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
// L1 need not have what was written before the attention kernel began. A prompt's is in the call.
__device__ __forceinline__ int attend_len(const CacheJob& J, int u) {
  const int b = J.lens ? 0 : J.by_heads(u);
  return J.lens ? min(max(__ldcg(J.lens + u), 0), J.cap) : J.off[b + 1] - J.off[b];
}

// The unit of a request's KV head and row tile. lens: the sequences' lengths (AttendScan::lengths), or
// null to read them from the cache.
__device__ __forceinline__ AttendUnit attend_unit(const AttendJob& A, const AttendPlan& P, const int32_t* lens, int b,
                                                  int h, int tile) {
  const CacheJob& J = A.c;
  AttendUnit x;
  x.b = b;
  x.h = h;
  x.n = J.off[b + 1] - J.off[b];
  const int all = x.n * J.r;
  x.row0 = tile * P.rows;
  x.rows = min(P.rows, all - x.row0);
  const int seq = x.b * J.Hkv + x.h;
  x.len = lens ? lens[seq] : attend_len(J, seq);
  x.keys = keys_of(A.causal, x.len, x.n, J.by_r(x.row0 + x.rows - 1));
  x.pieces = (x.keys + (1 << P.step_shift) - 1) >> P.step_shift;
  x.extra = x.rows <= 128 ? P.extra1 : P.extra;
  x.cost = x.pieces ? x.pieces + x.extra : 0;
  return x;
}
__device__ __forceinline__ AttendUnit attend_unit(const AttendJob& A, const AttendPlan& P, const int32_t* lens, int u) {
  const int b = range_of(P.uoff, A.c.B, u), rem = u - P.uoff[b], h = P.by_tiles[b](rem);
  return attend_unit(A, P, lens, b, h, rem - h * P.tiles[b]);
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
    return J.lens && J.B * J.Hkv <= LENS ? lens : nullptr;
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
// `row` counts the rows of the request's KV head. PART: by a kernel whose sums may be wanted as they are.
template <typename T, int D, bool PART = false>
__device__ __forceinline__ void attend_write(const AttendJob& A, int b, int h, int row, int d0, float4 v, float top,
                                             float z) {
  const CacheJob& J = A.c;
  const int tok = J.by_r(row);
  const size_t at = (size_t)(J.off[b] + tok) * J.Hq + h * J.r + row - tok * J.r;
  const float f = z == 0.f ? 0.f : 1.f / z;
  T* out = reinterpret_cast<T*>(A.out) + at * D + d0;
  if (z == 0.f) v = make_float4(0.f, 0.f, 0.f, 0.f);
  if (PART && A.part) {
    *reinterpret_cast<float4*>(A.part + at * D + d0) = v;
    if (d0 == 0) A.part_ml[at] = make_float2(top, z);
    return;
  }
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

// Which workers have a unit's parts: workers [i0, i1], the first one's slot.
struct Parts {
  int i0, i1, first;
  __device__ __forceinline__ Parts(const AttendPlan& P, const Shares& sh, const AttendUnit& U, int64_t before) {
    const int64_t a = before + U.extra;                // its pieces are at [a, a + pieces)
    i0 = sh.of(a);
    i1 = a + U.pieces <= sh.begin(i0 + 1) ? i0 : sh.of(a + U.pieces - 1);
    first = attend_slot(i0, sh.begin(i0), before);
  }
  // A worker's first part has an even slot; only the unit's first can be a worker's last.
  __device__ __forceinline__ size_t slot(const AttendPlan& P, int k, int r) const {
    return (size_t)(k ? 2 * (i0 + k) : first) * P.rows + r;
  }
};

// A warp's sum over the parts k0, k0 + STEP, ... of row r: its lane's D / 32 values.
template <int D, int STEP>
__device__ __forceinline__ void add_parts(const AttendPlan& P, const Parts& x, int r, int lane, int k0, float& top,
                                          float& z, float (&o)[D / 32]) {
  const int parts = x.i1 - x.i0 + 1;
  top = -INFINITY;
  for (int k = lane; k < parts; k += 32) top = fmaxf(top, P.pml[x.slot(P, k, r)].x);
#pragma unroll
  for (int s = 16; s; s >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
  z = 0.f;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) o[i] = 0.f;
#pragma unroll 8
  for (int k = k0; k < parts; k += STEP) {
    const size_t slot = x.slot(P, k, r);
    const float2 ml = P.pml[slot];
    const float f = ml.x == -INFINITY ? 1.f : fast_exp2(ml.x - top);
    z += ml.y * f;
    const float* p = P.po + slot * D + lane * (D / 32);
    if constexpr (D == 128) {
      const float4 v = *reinterpret_cast<const float4*>(p);
      o[0] += v.x * f;
      o[1] += v.y * f;
      o[2] += v.z * f;
      o[3] += v.w * f;
    } else {
      const float2 v = *reinterpret_cast<const float2*>(p);
      o[0] += v.x * f;
      o[1] += v.y * f;
    }
  }
}

// Attention whose sums are not merged yet: the plans of its few-row and of its other requests.
struct AttendParts {
  AttendJob A;
  AttendPlan t, c;
  int32_t few;         // rows of a request's KV head up to which it is in t
  int32_t whole;       // t's units are all in A.part
  int32_t common;      // c's keys are whole pages that all rows see
  int32_t behind;      // the kernel in front has tiles of other parts
};
// The plans of a call (few: 0 for what attention itself takes; common: of pages that a group's sequences
// share), and the call with or without its merges.
cudaError_t attend_parts(const AttendJob& A, void* scratch, int few, bool common, AttendParts* S);
cudaError_t launch_attend(const AttendParts& S, bool merge, cudaStream_t st);

// What a row's sum is found by: its request's first token and rows of a KV head, and of its plan.
struct AttendRows {
  int32_t tok0, rows, few, tile, units, tiles, unused[2];
};
inline AttendRows attend_rows(const AttendParts& S, int b) {
  const CacheJob& J = S.A.c;
  const int rows = (J.off[b + 1] - J.off[b]) * J.r, few = rows <= S.few;
  const AttendPlan& P = few ? S.t : S.c;
  return AttendRows{J.off[b], rows, few, P.rows, P.uoff[b], P.tiles[b], {0, 0}};
}

// A warp's: the sum of query row rho of KV head h of the request with rows R; its lane's D / 32 values.
template <int D>
__device__ __forceinline__ void sum_of_row(const AttendParts& S, const AttendRows& R, int b, int h, int rho, int lane,
                                           float& top, float& z, float (&o)[D / 32]) {
  const CacheJob& J = S.A.c;
  const AttendPlan& P = R.few ? S.t : S.c;
  const int tile = rho / R.tile, row = rho - tile * R.tile, u = R.units + h * R.tiles + tile;
  const int tok = J.by_r(rho);
  const size_t at = (size_t)(R.tok0 + tok) * J.Hq + h * J.r + rho - tok * J.r;
  top = -INFINITY;
  z = 0.f;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) o[i] = 0.f;
  if (!(R.few && S.whole)) {
    const int64_t W = P.start[P.workers].before;
    const int len = attend_len(J, b * J.Hkv + h), rows = min(R.tile, R.rows - tile * R.tile);
    AttendUnit U;
    U.rows = rows;
    U.keys = keys_of(S.A.causal, len, J.by_r(R.rows), J.by_r(tile * R.tile + rows - 1));
    U.pieces = (U.keys + (1 << P.step_shift) - 1) >> P.step_shift;
    U.extra = rows <= 128 ? P.extra1 : P.extra;
    if (!U.pieces) return;
    // If a worker's share begins in the unit, it says what is before the unit; else one worker had
    // all of it.
    const Shares sh = shares_of(W, P.workers, P.least);
    int lo = 0, hi = sh.n;                             // the first worker whose first unit is not before u
    while (lo < hi) {                                  // a lane a place in turn: a load's latency for 32
      const int step = (hi - lo + 31) / 32, i = lo + lane * step;
      const int less = __popc(__ballot_sync(0xffffffffu, i < hi && P.start[i].unit < u));
      if (less) {
        const int last = lo + (less - 1) * step;       // the last of them that is before u
        hi = min(hi, last + step);
        lo = last + 1;
      } else {
        hi = lo;
      }
    }
    if (lo < sh.n) {
      const AttendStart s = P.start[lo];
      if (s.unit == u) {
        const Parts parts(P, sh, U, s.before);
        if (parts.i0 < parts.i1) {
          add_parts<D, 1>(P, parts, row, lane, 0, top, z, o);
          return;
        }
      }
    }
  }
  const float2 ml = S.A.part_ml[at];
  top = ml.x;
  z = ml.y;
  const float* p = S.A.part + at * D + lane * (D / 32);
#pragma unroll
  for (int i = 0; i < D / 32; i += 2) {
    const float2 v = *reinterpret_cast<const float2*>(p + i);
    o[i] = v.x;
    o[i + 1] = v.y;
  }
}

cudaError_t launch_attend_token(const AttendJob& A, const AttendPlan& P, bool cluster, bool overlap, cudaStream_t st);
cudaError_t launch_attend_simt(const AttendJob& A, const AttendPlan& P, cudaStream_t st);
cudaError_t launch_attend_chunk(const AttendJob& A, const AttendPlan& P, cudaStream_t st);
cudaError_t launch_prompt_umma(const AttendJob& A, const AttendPlan& P, const PromptOrder& O, cudaStream_t st);
cudaError_t launch_common_umma(const AttendJob& A, const AttendPlan& P, cudaStream_t st);
cudaError_t launch_prompt_simt(const AttendJob& A, const AttendPlan& P, cudaStream_t st);

}  // namespace mmshift
