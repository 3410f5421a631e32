// Attention of new tokens over the paged cache (mmshift_cache_attention): which
// kernel takes which requests, and the merge of partial sums.
#include <algorithm>
#include <cstring>

#include "attend.cuh"

namespace mmshift {
namespace {

// Start of a merge: everything before it is done. The next kernel is not let in early:
// merges start early themselves, so it would come while the attention kernel still runs
// (178 to 285 us instead of 68 for a call behind another).
__device__ __forceinline__ void merge_start() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

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

// The merge of few units of many parts each (4 units of 114): a block a row, its warps
// on the row's parts. Zeros for units without keys. Which workers share the unit follows
// from the lengths, which were there before the attention kernel began: worked out while
// that still runs.
template <typename T, int D>
__global__ void __launch_bounds__(256) attend_merge_row_kernel(const __grid_constant__ AttendJob A,
                                                               const __grid_constant__ AttendPlan P) {
  __shared__ AttendScan<256> scan;
  __shared__ AttendStart place;
  __shared__ alignas(16) float so[8][D];
  __shared__ float sz[8];
  const int u = blockIdx.x, r = blockIdx.y, w = threadIdx.x / 32, lane = threadIdx.x % 32;
  const AttendSums x(A, P, &scan);
  if (u >= x.u0 && u < x.u1) {
    place.before = x.before;
    for (int k = x.u0; k < u; ++k) place.before += attend_unit(A, P, scan.lengths(A.c), k).cost;
  }
  __syncthreads();
  const AttendUnit U = attend_unit(A, P, scan.lengths(A.c), u);
  float top = -INFINITY, z = 0.f, o[D / 32] = {};
  if (U.pieces) {
    const Parts parts(P, shares_of(x.W, P.workers, P.least), U, place.before);
    merge_start();
    if (parts.i0 == parts.i1 || r >= U.rows) return;   // one worker had it all
    add_parts<D, 8>(P, parts, r, lane, w, top, z, o);
  } else {
    merge_start();
    if (r >= U.rows) return;
  }
#pragma unroll
  for (int i = 0; i < D / 32; ++i) so[w][lane * (D / 32) + i] = o[i];
  if (lane == 0) sz[w] = z;
  __syncthreads();
  if (threadIdx.x >= D / 4) return;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  z = 0.f;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const float4 y = *reinterpret_cast<const float4*>(&so[k][threadIdx.x * 4]);
    v.x += y.x;
    v.y += y.y;
    v.z += y.z;
    v.w += y.w;
    z += sz[k];
  }
  attend_write<T, D>(A, U.b, U.h, U.row0 + r, threadIdx.x * 4, v, top, z);
}

// The merge of many units: only those across a border of two workers' shares have
// parts, so a block takes a border (and 32 rows, kMergeRows a warp in turn), the first
// inside its unit's pieces. The blocks behind them write zeros for units without keys. Most
// blocks only find that they have nothing to do: with 8 rows each there are so many that
// ragged turns take 150 us instead of 145, with 64 rows a warp has too much (150).
constexpr int kEmptyBlocks = 16, kMergeRows = 4;

template <typename T, int D>
__global__ void __launch_bounds__(256) attend_merge_border_kernel(const __grid_constant__ AttendJob A,
                                                                  const __grid_constant__ AttendPlan P) {
  merge_start();
  const int w = threadIdx.x / 32, lane = threadIdx.x % 32, i = blockIdx.x + 1;
  if (i >= P.workers) {
    __shared__ int empty[256], n;
    if (blockIdx.y) return;
    const int units = P.uoff[A.c.B];
    for (int u0 = (i - P.workers) * 256; u0 < units; u0 += kEmptyBlocks * 256) {
      if (threadIdx.x == 0) n = 0;
      __syncthreads();
      const int u = u0 + threadIdx.x;
      if (u < units && !attend_unit(A, P, nullptr, u).pieces) empty[atomicAdd(&n, 1)] = u;
      __syncthreads();
      for (int k = 0; k < n; ++k) {
        const AttendUnit U = attend_unit(A, P, nullptr, empty[k]);
        for (int e = threadIdx.x; e < U.rows * (D / 4); e += 256)
          attend_write<T, D>(A, U.b, U.h, U.row0 + e / (D / 4), e % (D / 4) * 4, make_float4(0.f, 0.f, 0.f, 0.f),
                             -INFINITY, 0.f);
      }
      __syncthreads();
    }
    return;
  }
  const Shares sh = shares_of(P.start[P.workers].before, P.workers, P.least);
  if (i >= sh.n) return;
  const AttendStart s = P.start[i];
  const AttendUnit U = attend_unit(A, P, nullptr, s.unit);
  const Parts parts(P, sh, U, s.before);
  if (parts.i0 + 1 != i || parts.i0 == parts.i1) return;
  const int r0 = blockIdx.y * 8 * kMergeRows + w, r1 = min(U.rows, (int)(blockIdx.y + 1) * 8 * kMergeRows);
#pragma unroll 1
  for (int r = r0; r < r1; r += 8) {
    float top, z, o[D / 32];
    add_parts<D, 1>(P, parts, r, lane, 0, top, z, o);
    // four neighbouring values to one lane
    if constexpr (D == 128) {
      attend_write<T, D>(A, U.b, U.h, U.row0 + r, lane * 4, make_float4(o[0], o[1], o[2], o[3]), top, z);
    } else {
      const float a = __shfl_down_sync(0xffffffffu, o[0], 1), b = __shfl_down_sync(0xffffffffu, o[1], 1);
      if (lane % 2 == 0) attend_write<T, D>(A, U.b, U.h, U.row0 + r, lane * 2, make_float4(o[0], o[1], a, b), top, z);
    }
  }
}

template <typename T, int D>
cudaError_t launch_merge_t(const AttendJob& A, const AttendPlan& P, cudaStream_t st) {
  const unsigned units = P.uoff[A.c.B];
  if (8 * units <= (unsigned)P.workers)
    return launch_kernel(attend_merge_row_kernel<T, D>, dim3(units, P.rows), 256, 0, st, true, 0, A, P);
  constexpr int rows = 8 * kMergeRows;
  return launch_kernel(attend_merge_border_kernel<T, D>, dim3(P.workers - 1 + kEmptyBlocks, (P.rows + rows - 1) / rows),
                       256, 0, st, true, 0, A, P);
}

cudaError_t launch_merge(const AttendJob& A, const AttendPlan& P, cudaStream_t st) {
  if (A.c.bf16)
    return A.c.d == 128 ? launch_merge_t<__nv_bfloat16, 128>(A, P, st) : launch_merge_t<__nv_bfloat16, 64>(A, P, st);
  return A.c.d == 128 ? launch_merge_t<float, 128>(A, P, st) : launch_merge_t<float, 64>(A, P, st);
}

// Requests of few rows of a KV head have a plan of their own, of tiles of at most this
// many: bfloat16 rows go to the token kernel, float32 rows to tiles of 8 or 16 rows
// (requests of more rows to tiles of 256, or 128).
constexpr int kTokenRows = 16;
constexpr int kClusterSteps = 4;

// Rows of a request's KV head that go to the plan of tiles of kTokenRows. More than one
// tile reads the keys again, from the L2, but starts sooner than a chunk's tile and
// computes fewer rows that are not there: 16 requests of 32 heads, 300 to 750 rows,
// 32 tokens: bfloat16 68 us (chunk kernel 92), 8-bit 62 (95); 48 tokens: 96 (93), 87 (96);
// 64 tokens: 125 (95), 112 (98). float32 rows: 32 tokens 209 (tiles of 128: 474), 64
// tokens 407 (548), 96 tokens 616 (573); 8-bit pages 284 (463), 563 (537), 856 (560).
int few_rows(const CacheJob& J) { return J.bf16 ? 32 : 64; }

constexpr int kSMs = 152;              // the workspace is sized without asking the device

int sm_count() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return 0;
  return std::min(n, kSMs);
}

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

// The plan of the requests that `take`s, with tiles of at most `most` rows.
template <class Take>
AttendPlan plan_of(const CacheJob& J, int most, Take take) {
  AttendPlan P;
  std::memset(&P, 0, sizeof(P));
  int widest = 0;
  for (int b = 0; b < J.B; ++b) {
    const int rows = (J.off[b + 1] - J.off[b]) * J.r;
    if (rows && take(rows)) widest = std::max(widest, rows);
  }
  P.rows = std::min(widest, most);
  for (int b = 0; b < J.B; ++b) {
    const int rows = (J.off[b + 1] - J.off[b]) * J.r;
    P.tiles[b] = rows && take(rows) ? (rows + P.rows - 1) / P.rows : 0;
    P.by_tiles[b] = divisor_of(P.tiles[b]);
    P.uoff[b + 1] = P.uoff[b] + J.Hkv * P.tiles[b];
  }
  return P;
}

// Plans for `nsm` SMs; a CTA a worker, as many as fit.
AttendPlan token_plan(const CacheJob& J, int nsm) {
  AttendPlan P = plan_of(J, kTokenRows, [&](int rows) { return rows <= few_rows(J); });
  if (J.bf16) {
    const int row = J.i8 ? J.d : 2 * J.d;
    while ((row << P.step_shift) < 4096) ++P.step_shift;   // a warp's piece: 4 KB of K
    P.least = 2;
    P.workers = nsm * (P.rows <= 8 ? 3 : 2);
    P.extra = P.extra1 = 8;
  } else {
    P.step_shift = 5;
    P.workers = nsm * (J.d == 64 ? 8 : P.rows <= 8 ? 5 : 4);
  }
  return P;
}

AttendPlan chunk_plan(const CacheJob& J, int nsm) {
  AttendPlan P = plan_of(J, J.bf16 ? 256 : 128, [&](int rows) { return rows > few_rows(J); });
  P.step_shift = J.bf16 ? 7 : 6;
  P.workers = nsm;
  P.extra = !J.bf16 ? 0 : J.i8 ? 4 : 6;
  P.extra1 = !J.bf16 ? 0 : 3;
  return P;
}

// The plan's buffers from `at` on; where they end.
char* place(AttendPlan& P, const CacheJob& J, char* at) {
  P.po = reinterpret_cast<float*>(at);
  at += align256((size_t)2 * P.workers * P.rows * J.d * sizeof(float));
  P.pml = reinterpret_cast<float2*>(at);
  at += align256((size_t)2 * P.workers * P.rows * sizeof(float2));
  P.start = reinterpret_cast<AttendStart*>(at);
  return at + align256((size_t)(P.workers + 1) * sizeof(AttendStart));
}

}  // namespace

size_t attend_scratch_bytes(const CacheJob& J) {
  AttendPlan t = token_plan(J, kSMs), c = chunk_plan(J, kSMs);
  char* const base = reinterpret_cast<char*>(uintptr_t(256));
  return place(c, J, place(t, J, base)) - base;
}

cudaError_t launch_attend(const AttendJob& A, void* scratch, cudaStream_t st) {
  const CacheJob& J = A.c;
  const int nsm = sm_count();
  if (nsm <= 0) return cudaErrorInvalidDevice;
  AttendPlan t = token_plan(J, nsm), c = chunk_plan(J, nsm);
  place(c, J, place(t, J, static_cast<char*>(scratch)));
  cudaError_t e = cudaSuccess;
  if (c.uoff[J.B]) {
    e = J.bf16 ? launch_attend_chunk(A, c, st) : launch_attend_simt(A, c, st);
    if (e == cudaSuccess) e = launch_merge(A, c, st);
  }
  if (e == cudaSuccess && t.uoff[J.B]) {
    if (J.bf16) {
      // Clusters of eight CTAs where a warp has at most kClusterSteps steps even of a full
      // table, and all clusters fit at once: longer steps then cost less than another launch
      // and the reading of lengths. One token, 4 heads, bfloat16 rows: 513 rows 5.8 us (7.3
      // by the balanced form and its merge), 2049 (4 steps) 8.7 (8.9), 4097 13.0 (10.3);
      // 8-bit rows: 2049 8.1 (8.9), 4097 (4 steps) 10.3 (10.1).
      const bool cluster = J.cap >> t.step_shift <= 32 * kClusterSteps && 8 * t.uoff[J.B] <= t.workers;
      e = launch_attend_token(A, t, cluster, st);
      if (cluster) return e;
    } else {
      e = launch_attend_simt(A, t, st);
    }
    if (e == cudaSuccess) e = launch_merge(A, t, st);
  }
  return e;
}

}  // namespace mmshift
