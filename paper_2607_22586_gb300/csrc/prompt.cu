// The entry point of attention over whole prompts (mmshift_prompt_attention).
#include <cstring>

#include "cache.cuh"

namespace mmshift {
mmshift_status noalloc_cuda_fail(cudaError_t e);

namespace {

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

mmshift_status prompt_job(const mmshift_shape* s, void* ws, CacheJob* J) {
  std::memset(J, 0, sizeof(*J));
  const mmshift_status st = check_rows(s);
  if (st != MMSHIFT_OK) return st;
  if (s->n_layers != 1) return MMSHIFT_ERR_UNSUPPORTED;
  J->B = s->batch;
  J->L = 1;
  J->Hq = s->n_q_heads;
  J->Hkv = s->n_kv_heads;
  J->r = s->n_q_heads / s->n_kv_heads;
  J->by_r = divisor_of(J->r);
  J->by_heads = divisor_of(J->Hkv);
  J->d = s->head_dim;
  J->bf16 = s->dtype == MMSHIFT_BF16;
  J->status = static_cast<int*>(ws);
  for (int b = 0; b <= s->batch; ++b) J->off[b] = s->cu_seqlens[b];
  return MMSHIFT_OK;
}

}  // namespace
}  // namespace mmshift

using namespace mmshift;

extern "C" {

mmshift_status mmshift_prompt_workspace_size(const mmshift_shape* s, size_t* bytes) {
  CacheJob J;
  const mmshift_status st = prompt_job(s, nullptr, &J);
  if (st != MMSHIFT_OK) return st;
  if (!bytes) return MMSHIFT_ERR_INVALID_ARG;
  *bytes = 256 + prompt_scratch_bytes(J);
  return MMSHIFT_OK;
}

mmshift_status mmshift_prompt_attention(const mmshift_shape* s, const void* Q, int64_t q_row_stride, const void* K,
                                        const void* V, int64_t kv_row_stride, int32_t causal, float softmax_scale,
                                        void* out, float* lse, void* workspace, size_t workspace_bytes,
                                        mmshift_stream_t stream) {
  AttendJob A;
  std::memset(&A, 0, sizeof(A));
  CacheJob& J = A.c;
  mmshift_status st = prompt_job(s, workspace, &J);
  if (st != MMSHIFT_OK) return st;
  if ((st = attend_args(J, Q, q_row_stride, causal, softmax_scale, out, lse)) != MMSHIFT_OK) return st;
  const int64_t dense = (int64_t)J.Hkv * J.d, esz = J.bf16 ? 2 : 4;
  if (kv_row_stride && kv_row_stride < dense) return MMSHIFT_ERR_INVALID_ARG;
  A.kv_stride = kv_row_stride ? kv_row_stride : dense;
  if (A.kv_stride * esz % 16 != 0 || A.kv_stride >= (int64_t)1 << 38) return MMSHIFT_ERR_INVALID_ARG;   // TMA's
  if (J.off[J.B] && (!K || !V)) return MMSHIFT_ERR_INVALID_ARG;
  if (!aligned(K, 16) || !aligned(V, 16)) return MMSHIFT_ERR_INVALID_ARG;
  if ((st = check_workspace(workspace, workspace_bytes, prompt_scratch_bytes(J))) != MMSHIFT_OK) return st;
  if (!J.off[J.B]) return MMSHIFT_OK;
  attend_set(A, Q, q_row_stride, causal, softmax_scale);
  J.kp = static_cast<uint8_t*>(const_cast<void*>(K));
  J.vp = static_cast<uint8_t*>(const_cast<void*>(V));
  A.out = static_cast<uint8_t*>(out);
  A.ovec = aligned(out, 32) ? 2 : aligned(out, 16);   // 2: 32 bytes at once
  A.lse = lse;
  const cudaError_t e = launch_prompt(A, static_cast<char*>(workspace) + 256, (cudaStream_t)stream);
  return e == cudaSuccess ? MMSHIFT_OK : noalloc_cuda_fail(e);
}

}  // extern "C"
