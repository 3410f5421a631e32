// Attention over sequences that share pages (mmshift_cache_attention_shared).
//
// A group's rows attend twice: all of them to the pages that its sequences have in common, as if
// they were one request's, and each to the pages behind those. Both are the attention that
// the cache has anyway (attend.cu), over other lengths and beginnings of the page table, which
// common_pages_kernel works out on the device; both leave sums of weights times values with their
// maxima, in float32, as the workers left them, and join_kernel adds a row's up:
//   m = max m_k, z = sum z_k 2^(m_k - m), out = sum o_k 2^(m_k - m) / z.
// What the group has in common is read once instead of once a request, and its rows fill the
// tensor cores' tiles together.
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstring>

#include "attend.cuh"
#include "umma.cuh"

namespace mmshift {
mmshift_status noalloc_cuda_fail(cudaError_t e);

namespace {

using umma::cluster_arrive;
using umma::cluster_rank;
using umma::cluster_sync;
using umma::cluster_wait;
using umma::mapa;
using umma::smem_u32;
using umma::st_cluster_int;

constexpr int kCluster = 8;            // CTAs that compare a group's tables

struct SharedJob {
  CacheJob c;
  int32_t causal, n_groups;
  int64_t* at[2];                      // of the groups' common pages, of the requests' own
  int32_t* lens[2];                    // [n_groups][Hkv], [batch][Hkv]
  int32_t group[MMSHIFT_MAX_BATCH + 1];   // first requests
  int32_t lead[MMSHIFT_MAX_BATCH];     // of each group the first with rows, -1 where it is the only one
  AttendRows row[2][MMSHIFT_MAX_BATCH];   // of the groups, of the requests
  AttendRows* rows;                    // the same, in device memory
  int32_t* place;                      // [T] of each token: group << 16 | request
};

struct JoinJob {
  AttendParts part[2];                 // of the common pages, of the requests' own
  uint8_t* out;
  float* lse;
  int32_t ovec;
  const AttendRows* rows;
  const int32_t* place;
};

// Start: everything before in the stream is done, and the next kernel may take its place.
__device__ __forceinline__ void shared_start() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// A cluster a group and KV head: how many pages all its sequences with rows in the call have
// in common, up to an entry that is no page. Only keys that every row attends to count, and requests
// alone have none. Warps compare 32 places of the table at a time, eight requests at once (64
// requests of 375 pages, 8 heads: 15 us by one CTA each). It is a chain of loads that are not in the L2
// after a pass over the cache, so the first places are asked for together with the lengths, which say
// how many of them count (12.5 -> 6.4 us).
__global__ void __launch_bounds__(256) common_pages_kernel(const __grid_constant__ SharedJob S) {
  constexpr int AHEAD = 2, MOST = MMSHIFT_MAX_BATCH / 8;   // places of a lane at first; requests of a warp
  __shared__ int32_t common, keys, found[kCluster];
  const CacheJob& J = S.c;
  shared_start();
  const int rank = cluster_rank(), g = J.by_heads(blockIdx.x / kCluster), h = blockIdx.x / kCluster - g * J.Hkv;
  const int b0 = S.group[g], b1 = S.group[g + 1], lead = S.lead[g], first = max(lead, b0);
  const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
  if (tid == 0) common = keys = INT_MAX;
  __syncwarp();
  cluster_arrive();                                    // all CTAs are there before one writes to another
  const int own = b0 + tid;
  const bool mine = own < b1;
  const int len = mine ? cache_len(J, (size_t)own * J.Hkv + h) : 0;
  auto entry = [&](int b, int e) { return J.table[((size_t)b * J.Hkv + h) * J.max_pages + e]; };
  auto rows_in = [&](int b) { return J.off[b + 1] > J.off[b]; };
  int32_t is[AHEAD], other[AHEAD][MOST];
#pragma unroll
  for (int a = 0; a < AHEAD; ++a) {
    const int e = (a * kCluster + rank) * 32 + lane;
    const bool in = lead >= 0 && e < J.max_pages;
    is[a] = in ? entry(first, e) : 0;
#pragma unroll
    for (int k = 0; k < MOST; ++k) {
      const int b = first + 1 + warp + 8 * k;
      other[a][k] = in && b < b1 && rows_in(b) ? entry(b, e) : is[a];
    }
  }
  // what join_kernel would look up step by step
  if (h == 0) {
    for (int t = J.off[b0] + rank * 256 + tid; t < J.off[b1]; t += kCluster * 256) S.place[t] = g << 16 | range_of(J.off, J.B, t);
    if (g == 0 && rank == 0 && tid < 2 * MMSHIFT_MAX_BATCH)
      S.rows[tid] = S.row[tid / MMSHIFT_MAX_BATCH][tid % MMSHIFT_MAX_BATCH];
  }
  __syncthreads();
  if (mine && rows_in(own)) atomicMin(&keys, keys_of(S.causal, len, J.off[own + 1] - J.off[own], 0));
#pragma unroll
  for (int a = 0; a < AHEAD; ++a) {
    bool same = is[a] >= 0 && is[a] < J.n_pages;
#pragma unroll
    for (int k = 0; k < MOST; ++k) same &= other[a][k] == is[a];
    if (!same) atomicMin(&common, (a * kCluster + rank) * 32 + lane);
  }
  __syncthreads();
  const int most = lead >= 0 ? keys >> J.page_shift : 0;
  for (int e = (AHEAD * kCluster + rank) * 32 + lane; e < most; e += kCluster * 32) {
    const int32_t is_ = entry(first, e);
    bool same = is_ >= 0 && is_ < J.n_pages;
#pragma unroll 8
    for (int b = first + 1 + warp; b < b1; b += 8) same &= !rows_in(b) || entry(b, e) == is_;
    if (!same) {
      atomicMin(&common, e);
      break;                                           // what lies behind cannot be less
    }
  }
  __syncthreads();
  cluster_wait();
  if (tid == 0) st_cluster_int(mapa(smem_u32(&found[rank]), 0), common);
  __syncwarp();
  cluster_sync();
  if (rank) return;
  int pages = most;
#pragma unroll
  for (int r = 0; r < kCluster; ++r) pages = min(pages, found[r]);
  if (tid == 0) {
    S.at[0][g * J.Hkv + h] = ((int64_t)first * J.Hkv + h) * J.max_pages;
    S.lens[0][g * J.Hkv + h] = pages << J.page_shift;
  }
  if (mine) {
    const size_t u = (size_t)own * J.Hkv + h;
    const int less = rows_in(own) ? pages : 0;
    S.at[1][u] = (int64_t)u * J.max_pages + less;
    S.lens[1][u] = len - (less << J.page_shift);
  }
}

// Two warps a row: one adds up the common pages' sums, one the request's own.
template <typename T, int D>
__global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ JoinJob S) {
  constexpr int N = D / 32;                            // values of a lane
  __shared__ float2 ml[4];
  __shared__ alignas(16) float sum[4][D];
  const CacheJob& J = S.part[1].A.c;
  shared_start();
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, own = warp & 1;
  const int row = blockIdx.x * 4 + warp / 2;
  const bool in = row < J.off[J.B] * J.Hq;
  const int tok = in ? row / J.Hq : 0, hq = in ? row - tok * J.Hq : 0, h = J.by_r(hq), j = hq - h * J.r;
  const int at = S.place[tok], i = own ? at & 0xffff : at >> 16;
  const AttendRows R = S.rows[own * MMSHIFT_MAX_BATCH + i];
  float top, z, o[N];
  sum_of_row<D>(S.part[own], R, i, h, (tok - R.tok0) * J.r + j, lane, top, z, o);
  if (!own) {
#pragma unroll
    for (int k = 0; k < N; ++k) sum[warp / 2][lane * N + k] = o[k];
    if (lane == 0) ml[warp / 2] = make_float2(top, z);
  }
  __syncthreads();
  if (!own || !in) return;
  const float2 x = ml[warp / 2];
  const float most = fmaxf(top, x.x);
  const float fa = x.x == -INFINITY ? 1.f : fast_exp2(x.x - most), fb = top == -INFINITY ? 1.f : fast_exp2(top - most);
  const float all = x.y * fa + z * fb, f = all == 0.f ? 0.f : 1.f / all;
  float v[N];
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = all == 0.f ? 0.f : (sum[warp / 2][lane * N + k] * fa + o[k] * fb) * f;
  T* const out = reinterpret_cast<T*>(S.out) + (size_t)row * D + lane * N;
  if (S.ovec && N == 4) {
    if constexpr (sizeof(T) == 2)
      *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[N / 2], v[N - 1]));
    else
      *reinterpret_cast<float4*>(out) = make_float4(v[0], v[1], v[N / 2], v[N - 1]);
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) out[k] = from_f32<T>(v[k]);
  }
  if (lane == 0 && S.lse) S.lse[row] = all == 0.f ? -INFINITY : (most + log2f(all)) * 0.6931471805599453f;
}

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }
bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// The groups' requests as one each.
CacheJob groups_job(const CacheJob& J, int32_t n_groups, const int32_t* cu_groups) {
  CacheJob G = J;
  G.B = n_groups;
  for (int g = 0; g <= n_groups; ++g) G.off[g] = J.off[cu_groups[g]];
  return G;
}

// Buffers from `at` on; where they end.
struct SharedParts {
  int64_t* at[2];
  int32_t* lens[2];
  float* part[2];
  float2* ml[2];
  AttendRows* rows;
  int32_t* place;
  char* scratch[2];
};

// A request's own keys are few, so that one more tile of few rows costs less than a chunk's launch:
// up to this many rows of a KV head go to the tiles of few rows: drafts of 12 answers of seven heads a
// KV head, 5 tokens each, 47 us (60 by chunks).
constexpr int kOwnRows = 64;

char* place(const CacheJob& J, const CacheJob& G, char* at, SharedParts* P) {
  const size_t rows = (size_t)J.off[J.B] * J.Hq;
  for (int i = 0; i < 2; ++i) {
    const size_t units = (size_t)(i ? J.B : G.B) * J.Hkv;
    P->at[i] = reinterpret_cast<int64_t*>(at);
    at += align256(units * sizeof(int64_t));
    P->lens[i] = reinterpret_cast<int32_t*>(at);
    at += align256(units * sizeof(int32_t));
    P->part[i] = reinterpret_cast<float*>(at);
    at += align256(rows * J.d * sizeof(float));
    P->ml[i] = reinterpret_cast<float2*>(at);
    at += align256(rows * sizeof(float2));
  }
  P->rows = reinterpret_cast<AttendRows*>(at);
  at += align256(2 * MMSHIFT_MAX_BATCH * sizeof(AttendRows));
  P->place = reinterpret_cast<int32_t*>(at);
  at += align256(J.off[J.B] * sizeof(int32_t));
  P->scratch[0] = at;
  P->scratch[1] = at + attend_scratch_bytes(G);
  return P->scratch[1] + attend_scratch_bytes(J, kOwnRows);
}

mmshift_status shared_job(const mmshift_shape* s, const mmshift_cache* c, int32_t n_groups, const int32_t* cu_groups,
                          void* ws, CacheJob* J, CacheJob* G) {
  const mmshift_status st = rows_job(s, c, ws, J);
  if (st != MMSHIFT_OK) return st;
  if (J->L != 1) return MMSHIFT_ERR_UNSUPPORTED;
  if ((int64_t)J->B * J->Hkv * kCluster >= (int64_t)1 << 31) return MMSHIFT_ERR_UNSUPPORTED;   // blocks
  if (!cu_groups || n_groups < 1 || n_groups > J->B || cu_groups[0] != 0 || cu_groups[n_groups] != J->B)
    return MMSHIFT_ERR_INVALID_ARG;
  for (int g = 0; g < n_groups; ++g)
    if (cu_groups[g + 1] <= cu_groups[g]) return MMSHIFT_ERR_INVALID_ARG;
  *G = groups_job(*J, n_groups, cu_groups);
  return MMSHIFT_OK;
}

cudaError_t launch_join(const JoinJob& S, cudaStream_t st) {
  const CacheJob& J = S.part[1].A.c;
  const unsigned rows = (unsigned)J.off[J.B] * J.Hq;
  auto go = [&](auto kernel) { return launch_kernel(kernel, dim3((rows + 3) / 4), 256, 0, st, true, 0, S); };
  if (J.bf16) return J.d == 128 ? go(join_kernel<__nv_bfloat16, 128>) : go(join_kernel<__nv_bfloat16, 64>);
  return J.d == 128 ? go(join_kernel<float, 128>) : go(join_kernel<float, 64>);
}

}  // namespace
}  // namespace mmshift

using namespace mmshift;

extern "C" {

mmshift_status mmshift_cache_shared_workspace_size(const mmshift_shape* s, const mmshift_cache* c, int32_t n_groups,
                                                   const int32_t* cu_groups, size_t* bytes) {
  CacheJob J, G;
  const mmshift_status st = shared_job(s, c, n_groups, cu_groups, nullptr, &J, &G);
  if (st != MMSHIFT_OK) return st;
  if (!bytes) return MMSHIFT_ERR_INVALID_ARG;
  SharedParts P;
  char* const base = reinterpret_cast<char*>(uintptr_t(256));
  *bytes = 256 + (place(J, G, base, &P) - base);
  return MMSHIFT_OK;
}

mmshift_status mmshift_cache_attention_shared(const mmshift_shape* s, const mmshift_cache* c, int32_t n_groups,
                                              const int32_t* cu_groups, const void* Q, int64_t row_stride,
                                              int32_t causal, float softmax_scale, void* out, float* lse,
                                              void* workspace, size_t workspace_bytes, mmshift_stream_t stream) {
  AttendJob A[2];
  std::memset(A, 0, sizeof(A));
  mmshift_status st = shared_job(s, c, n_groups, cu_groups, workspace, &A[1].c, &A[0].c);
  if (st != MMSHIFT_OK) return st;
  const CacheJob& J = A[1].c;
  if ((st = attend_args(J, Q, row_stride, causal, softmax_scale, out, lse)) != MMSHIFT_OK) return st;
  SharedParts P;
  const size_t need = place(J, A[0].c, static_cast<char*>(workspace) + 256, &P) - static_cast<char*>(workspace) - 256;
  if ((st = check_workspace(workspace, workspace_bytes, need)) != MMSHIFT_OK) return st;
  if (!J.off[J.B]) return MMSHIFT_OK;
  SharedJob S;
  std::memset(&S, 0, sizeof(S));
  S.c = J;
  S.causal = causal;
  S.n_groups = n_groups;
  std::memcpy(S.group, cu_groups, (n_groups + 1) * sizeof(int32_t));
  for (int g = 0; g < n_groups; ++g) {
    int lead = -1, members = 0;
    for (int b = cu_groups[g + 1] - 1; b >= cu_groups[g]; --b) {
      if (J.off[b + 1] == J.off[b]) continue;
      lead = b;
      ++members;
    }
    S.lead[g] = members > 1 ? lead : -1;
  }
  JoinJob N;
  std::memset(&N, 0, sizeof(N));
  N.out = static_cast<uint8_t*>(out);
  N.lse = lse;
  N.ovec = aligned(out, 16);
  N.rows = S.rows = P.rows;
  N.place = S.place = P.place;
  for (int i = 0; i < 2; ++i) {
    S.at[i] = P.at[i];
    S.lens[i] = P.lens[i];
    attend_set(A[i], Q, row_stride, i ? causal : 0, softmax_scale);
    A[i].part = P.part[i];
    A[i].part_ml = P.ml[i];
    A[i].c.at = P.at[i];
    A[i].c.lens = P.lens[i];
    const cudaError_t e = attend_parts(A[i], P.scratch[i], i ? kOwnRows : 0, i == 0, &N.part[i]);
    if (e != cudaSuccess) return noalloc_cuda_fail(e);
    if (i) N.part[1].behind = N.part[0].c.uoff[A[0].c.B] > 0 && N.part[0].t.uoff[A[0].c.B] == 0;
    for (int b = 0; b < A[i].c.B; ++b) S.row[i][b] = attend_rows(N.part[i], b);
  }
  const cudaStream_t cs = (cudaStream_t)stream;
  cudaError_t e = launch_kernel(common_pages_kernel, dim3((unsigned)n_groups * J.Hkv * kCluster), 256, 0, cs, true, kCluster, S);
  for (int i = 0; e == cudaSuccess && i < 2; ++i) e = launch_attend(N.part[i], false, cs);
  if (e == cudaSuccess) e = launch_join(N, cs);
  return e == cudaSuccess ? MMSHIFT_OK : noalloc_cuda_fail(e);
}

}  // extern "C"
