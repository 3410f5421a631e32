// Attention of new tokens over the paged cache (mmshift_cache_attention): one
// warp a row, one key at a time.
#include "cache.cuh"

namespace mmshift {
namespace {

template <typename T, int D, bool I8>
__device__ __forceinline__ float row_value(const uint8_t* pages, const float* scales, int64_t slot, int j) {
  if constexpr (I8) return (float)reinterpret_cast<const int8_t*>(pages)[slot * D + j] * scales[slot];
  else return to_f32(reinterpret_cast<const T*>(pages)[slot * D + j]);
}

template <typename T, int D, bool I8>
__global__ void __launch_bounds__(128) attend_row_kernel(const __grid_constant__ AttendJob A) {
  dependent_start();
  const CacheJob& J = A.c;
  const long long row = (long long)blockIdx.x * 4 + threadIdx.x / 32;
  const int lane = threadIdx.x % 32;
  if (row >= (long long)J.off[J.B] * J.Hq) return;
  const int tok = (int)(row / J.Hq), hq = (int)(row % J.Hq);
  const int b = cache_request(J, tok);
  const size_t u = (size_t)b * J.Hkv + hq / J.r;
  const int end = keys_of(A.causal, cache_len(J, u), J.off[b + 1] - J.off[b], tok - J.off[b]);
  float q[D / 32], o[D / 32] = {}, m = -INFINITY, z = 0.f;
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
    q[i] = to_f32(reinterpret_cast<const T*>(A.q)[(size_t)tok * J.stride + (size_t)hq * D + lane + 32 * i]);
  for (int t = 0; t < end; ++t) {
    const int64_t slot = cache_slot(J, u, t);
    if (slot < 0) {
      if (lane == 0) set_status(J.status, kStatusBadPage);
      continue;
    }
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) s += q[i] * row_value<T, D, I8>(J.kp, J.ks, slot, lane + 32 * i);
#pragma unroll
    for (int x = 16; x; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
    s *= A.alpha;
    if (s == -INFINITY) continue;
    const float mn = fmaxf(m, s);                    // a NaN stays out of the maximum
    const float c = m == -INFINITY ? 0.f : fast_exp2(m - mn), p = fast_exp2(s - mn);
    m = mn;
    z = z * c + p;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) o[i] = o[i] * c + p * row_value<T, D, I8>(J.vp, J.vs, slot, lane + 32 * i);
  }
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
    reinterpret_cast<T*>(A.out)[(size_t)row * D + lane + 32 * i] = from_f32<T>(z == 0.f ? 0.f : o[i] / z);
  if (A.lse && lane == 0) A.lse[row] = z == 0.f ? -INFINITY : (m + log2f(z)) * 0.6931471805599453f;
}

}  // namespace

size_t attend_scratch_bytes(const CacheJob&) { return 0; }

cudaError_t launch_attend(const AttendJob& A, void*, cudaStream_t st) {
  const CacheJob& J = A.c;
  const long long rows = (long long)J.off[J.B] * J.Hq;
  auto go = [&](auto kernel) {
    return launch_kernel(kernel, dim3((unsigned)((rows + 3) / 4)), 128, 0, st, true, 0, A);
  };
  if (J.bf16) {
    if (J.d == 128)
      return J.i8 ? go(attend_row_kernel<__nv_bfloat16, 128, true>) : go(attend_row_kernel<__nv_bfloat16, 128, false>);
    return J.i8 ? go(attend_row_kernel<__nv_bfloat16, 64, true>) : go(attend_row_kernel<__nv_bfloat16, 64, false>);
  }
  if (J.d == 128)
    return J.i8 ? go(attend_row_kernel<float, 128, true>) : go(attend_row_kernel<float, 128, false>);
  return J.i8 ? go(attend_row_kernel<float, 64, true>) : go(attend_row_kernel<float, 64, false>);
}

}  // namespace mmshift
