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

namespace mmshift {
mmshift_status noalloc_cuda_fail(cudaError_t e);

namespace {

constexpr int kCommon = 1024;

struct SharedJob {
  CacheJob c;
  int32_t causal, n_groups;
  int64_t* at[2];                      // of the groups' common pages, of the requests' own
  int32_t* lens[2];                    // [n_groups][Hkv], [batch][Hkv]
  int32_t group[MMSHIFT_MAX_BATCH + 1];   // first requests
};

struct JoinJob {
  AttendParts part[2];                 // of the common pages, of the requests' own
  uint8_t* out;
  float* lse;
  int32_t ovec;
  int32_t group[MMSHIFT_MAX_BATCH + 1], n_groups;
};

// Start: everything before in the stream is done, and the next kernel may take its place.
__device__ __forceinline__ void shared_start() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// A block a group and KV head: how many pages all its sequences with rows in the call have
// in common. Only keys that every row attends to count, and requests alone have none.
__global__ void __launch_bounds__(kCommon) common_pages_kernel(const __grid_constant__ SharedJob S) {
  __shared__ int32_t common, first_, keys, members;
  const CacheJob& J = S.c;
  shared_start();
  const int g = blockIdx.x, h = blockIdx.y, b0 = S.group[g], b1 = S.group[g + 1], tid = threadIdx.x;
  if (tid == 0) {
    first_ = keys = INT_MAX;
    members = 0;
  }
  __syncthreads();
  if (b0 + tid < b1) {
    const int b = b0 + tid, n = J.off[b + 1] - J.off[b];
    if (n) {
      atomicMin(&first_, b);
      atomicMin(&keys, keys_of(S.causal, cache_len(J, (size_t)b * J.Hkv + h), n, 0));
      atomicAdd(&members, 1);
    }
  }
  __syncthreads();
  const int first = members ? first_ : b0, most = members > 1 ? keys >> J.page_shift : 0;
  if (tid == 0) common = most;
  __syncthreads();
  // places in order, 256 at a time, the requests behind the first shared out to four threads a place
  const int32_t* const lead = J.table + ((size_t)first * J.Hkv + h) * J.max_pages;
  for (int e0 = 0; e0 < most; e0 += 256) {
    const int e = e0 + tid % 256;
    bool same = true;
    if (e < most) {
      const int32_t is = lead[e];
#pragma unroll 8
      for (int b = first + 1 + tid / 256; b < b1; b += 4)
        same &= J.off[b + 1] == J.off[b] || J.table[((size_t)b * J.Hkv + h) * J.max_pages + e] == is;
    }
    if (!same) atomicMin(&common, e);
    __syncthreads();
    if (common < e0 + 256) break;                      // the same for all threads
    __syncthreads();
  }
  __syncthreads();
  const int pages = common;
  if (tid == 0) {
    S.at[0][g * J.Hkv + h] = ((int64_t)first * J.Hkv + h) * J.max_pages;
    S.lens[0][g * J.Hkv + h] = pages << J.page_shift;
  }
  for (int b = b0 + tid; b < b1; b += kCommon) {
    const size_t u = (size_t)b * J.Hkv + h;
    const bool rows = J.off[b + 1] > J.off[b];
    S.at[1][u] = (int64_t)u * J.max_pages + (rows ? pages : 0);
    S.lens[1][u] = cache_len(J, u) - (rows ? pages << J.page_shift : 0);
  }
}

// A warp a row.
template <typename T, int D>
__global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ JoinJob S) {
  const CacheJob& J = S.part[1].A.c;
  shared_start();
  const int row = blockIdx.x * 8 + threadIdx.x / 32, lane = threadIdx.x % 32;
  if (row >= J.off[J.B] * J.Hq) return;
  const int tok = row / J.Hq, hq = row - tok * J.Hq, h = J.by_r(hq), j = hq - h * J.r;
  const int b = range_of(J.off, J.B, tok), g = range_of(S.group, S.n_groups, b);
  float ta, za, oa[D / 32], tb, zb, ob[D / 32];
  sum_of_row<D>(S.part[0], g, h, (tok - S.part[0].A.c.off[g]) * J.r + j, lane, ta, za, oa);
  sum_of_row<D>(S.part[1], b, h, (tok - J.off[b]) * J.r + j, lane, tb, zb, ob);
  const float top = fmaxf(ta, tb);
  const float fa = ta == -INFINITY ? 1.f : fast_exp2(ta - top), fb = tb == -INFINITY ? 1.f : fast_exp2(tb - top);
  const float z = za * fa + zb * fb, f = z == 0.f ? 0.f : 1.f / z;
  T* const out = reinterpret_cast<T*>(S.out) + (size_t)row * D + lane * (D / 32);
  float v[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) v[i] = z == 0.f ? 0.f : (oa[i] * fa + ob[i] * fb) * f;
  if (S.ovec && D == 128) {
    if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[D / 64], v[D / 32 - 1]));
    else *reinterpret_cast<float4*>(out) = make_float4(v[0], v[1], v[D / 64], v[D / 32 - 1]);
  } else {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) out[i] = from_f32<T>(v[i]);
  }
  if (lane == 0 && S.lse) S.lse[row] = z == 0.f ? -INFINITY : (top + log2f(z)) * 0.6931471805599453f;
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
  char* scratch[2];
};
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
  P->scratch[0] = at;
  P->scratch[1] = at + attend_scratch_bytes(G);
  return P->scratch[1] + attend_scratch_bytes(J);
}

mmshift_status shared_job(const mmshift_shape* s, const mmshift_cache* c, int32_t n_groups, const int32_t* cu_groups,
                          void* ws, CacheJob* J, CacheJob* G) {
  const mmshift_status st = rows_job(s, c, ws, J);
  if (st != MMSHIFT_OK) return st;
  if (J->L != 1) return MMSHIFT_ERR_UNSUPPORTED;
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
  auto go = [&](auto kernel) { return launch_kernel(kernel, dim3((rows + 7) / 8), 256, 0, st, true, 0, S); };
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
  JoinJob N;
  std::memset(&N, 0, sizeof(N));
  N.out = static_cast<uint8_t*>(out);
  N.lse = lse;
  N.ovec = aligned(out, 16);
  N.n_groups = n_groups;
  std::memcpy(N.group, S.group, sizeof(N.group));
  for (int i = 0; i < 2; ++i) {
    S.at[i] = P.at[i];
    S.lens[i] = P.lens[i];
    attend_set(A[i], Q, row_stride, i ? causal : 0, softmax_scale);
    A[i].part = P.part[i];
    A[i].part_ml = P.ml[i];
    A[i].c.at = P.at[i];
    A[i].c.lens = P.lens[i];
  }
  const cudaStream_t cs = (cudaStream_t)stream;
  cudaError_t e = launch_kernel(common_pages_kernel, dim3(n_groups, J.Hkv), kCommon, 0, cs, true, 0, S);
  for (int i = 0; e == cudaSuccess && i < 2; ++i) e = launch_attend(A[i], P.scratch[i], cs, &N.part[i]);
  if (e == cudaSuccess) e = launch_join(N, cs);
  return e == cudaSuccess ? MMSHIFT_OK : noalloc_cuda_fail(e);
}

}  // extern "C"
