// Rotary positions of Q and K rows (mmshift_rope), and the frequencies of long contexts.
//
// A pair (x, y) of a row at position p turns by w = p f: x' = a (x cos w - y sin w),
// y' = a (y cos w + x sin w). The angle of a far position has to keep its fraction of a
// turn: f / 2 pi is held as a fraction of 2^64, so p f / 2 pi modulo 1 is one integer product's
// low 64 bits, exact but for the fraction's own rounding (p 2^-53 turns), and its upper 32 bits
// are the angle in [-1, 1) half turns, which float32 sine and cosine take without a reduction.
//
// Bound by the bytes it moves. A lane has 16 bytes of each half of a head (or 32 bytes
// in a row, interleaved), works its angles out once and goes through the token's heads.
#include <cmath>
#include <cstring>

#include "cache.cuh"

namespace mmshift {
mmshift_status noalloc_cuda_fail(cudaError_t e);

namespace {

constexpr int kPairs = 64;             // of the widest head

struct RopeSide {
  const uint8_t* in;
  uint8_t* out;
  int64_t in_row, in_layer, out_row, out_layer;   // bytes between tokens, layers
  int32_t heads, copy;                 // copy: rows move, so what is not rotated does too
};

struct RopeJob {
  RopeSide side[2];                    // Q, K
  const int32_t* pos;                  // [n_axes][T]
  int32_t T, heads, rot, warps;        // rotated dimensions; warps of a token
  int32_t axis1, axis2;                // first pairs of the second and third axis
  float amp, sine;                     // of the values, and with the angle's sign
  uint64_t turn[kPairs];               // turns a position, in 2^-64
};

// Start: everything before in the stream is done, and the next kernel may take its place.
__device__ __forceinline__ void rope_start() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

__device__ __forceinline__ void rope_angle(const RopeJob& J, int tok, int pair, float& c, float& s) {
  const int axis = (pair >= J.axis1) + (pair >= J.axis2);
  const uint64_t a = (uint64_t)(int64_t)J.pos[(size_t)axis * J.T + tok] * J.turn[pair];
  sincospif((float)(int32_t)(a >> 32) * 0x1p-31f, &s, &c);
  c *= J.amp;
  s *= J.sine;
}

template <typename T>
__device__ __forceinline__ void rope_unpack(const uint4& w, float* x) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) {
      x[2 * i] = bf16_lo(u[i]);
      x[2 * i + 1] = bf16_hi(u[i]);
    } else {
      x[i] = __uint_as_float(u[i]);
    }
  }
}
template <typename T>
__device__ __forceinline__ uint4 rope_pack(const float* x) {
  uint32_t u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2)
      u[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
    else
      u[i] = __float_as_uint(x[i]);
  }
  return make_uint4(u[0], u[1], u[2], u[3]);
}

// Rows whose addresses and rotated part go by 16 bytes. Lane `part` of a head has chunks
// ca and cb of it, whose values are pairs with one another (half), or both of which hold
// pairs of neighbours (interleaved). What is not rotated is copied by the lanes behind.
template <typename T, int D, bool INTER>
__global__ void __launch_bounds__(256) rope_rows_kernel(const __grid_constant__ RopeJob J) {
  constexpr int N = 16 / (int)sizeof(T), LANES = D / (2 * N), HEADS = 32 / LANES;
  rope_start();
  const int warp = blockIdx.x * 8 + threadIdx.x / 32, lane = threadIdx.x % 32;
  const int tok = warp / J.warps, part = lane % LANES;
  if (tok >= J.T) return;
  const bool turned = part * 2 * N < J.rot;
  const int at = turned ? part : part - J.rot / (2 * N);
  const int ca = turned ? (INTER ? 2 * part : part) : J.rot / N + 2 * at;
  const int cb = turned && !INTER ? part + J.rot / (2 * N) : ca + 1;
  // The warp's heads share their angles: each group of lanes works M of a lane's N out for all (with all
  // N by every lane, 32,768 tokens of 32 heads take 91 us).
  constexpr int M = N / HEADS;
  static_assert(M * HEADS == N, "angles of a group of lanes");
  float c[N], s[N], cm[M], sm[M];
#pragma unroll
  for (int i = 0; i < M; ++i) {
    cm[i] = 1.f;
    sm[i] = 0.f;
    if (turned) rope_angle(J, tok, part * N + lane / LANES * M + i, cm[i], sm[i]);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    c[i] = __shfl_sync(0xffffffffu, cm[i % M], i / M * LANES + part);
    s[i] = __shfl_sync(0xffffffffu, sm[i % M], i / M * LANES + part);
  }
#pragma unroll 2
  for (int h = warp % J.warps * HEADS + lane / LANES; h < J.heads; h += J.warps * HEADS) {
    const bool k = h >= J.side[0].heads;
    const RopeSide& S = J.side[k];
    if (!turned && !S.copy) continue;
    const int64_t head = (int64_t)(k ? h - J.side[0].heads : h) * (D * (int)sizeof(T));
    const uint8_t* in = S.in + tok * S.in_row + blockIdx.y * S.in_layer + head;
    uint8_t* out = S.out + tok * S.out_row + blockIdx.y * S.out_layer + head;
    uint4 a = *reinterpret_cast<const uint4*>(in + ca * 16), b = *reinterpret_cast<const uint4*>(in + cb * 16);
    if (turned) {
      float x[2 * N], y[2 * N];
      rope_unpack<T>(a, x);
      rope_unpack<T>(b, x + N);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int p = INTER ? 2 * i : i, q = INTER ? 2 * i + 1 : N + i;
        y[p] = fmaf(x[p], c[i], -(x[q] * s[i]));
        y[q] = fmaf(x[q], c[i], x[p] * s[i]);
      }
      a = rope_pack<T>(y);
      b = rope_pack<T>(y + N);
    }
    *reinterpret_cast<uint4*>(out + ca * 16) = a;
    *reinterpret_cast<uint4*>(out + cb * 16) = b;
  }
}

// Any addresses and any even number of rotated dimensions: a lane a pair.
template <typename T, bool INTER>
__global__ void __launch_bounds__(256) rope_pairs_kernel(const __grid_constant__ RopeJob J, int d) {
  rope_start();
  const int warp = blockIdx.x * 8 + threadIdx.x / 32, lane = threadIdx.x % 32, tok = warp / J.warps;
  if (tok >= J.T) return;
  for (int p = lane; p < d / 2; p += 32) {
    const bool turned = 2 * p < J.rot;
    const int a = INTER || !turned ? 2 * p : p, b = INTER || !turned ? 2 * p + 1 : p + J.rot / 2;
    float c = 1.f, s = 0.f;
    if (turned) rope_angle(J, tok, p, c, s);
    for (int h = warp % J.warps; h < J.heads; h += J.warps) {
      const bool k = h >= J.side[0].heads;
      const RopeSide& S = J.side[k];
      if (!turned && !S.copy) continue;
      const int64_t head = (int64_t)(k ? h - J.side[0].heads : h) * d;
      const T* in = reinterpret_cast<const T*>(S.in + tok * S.in_row + blockIdx.y * S.in_layer) + head;
      T* out = reinterpret_cast<T*>(S.out + tok * S.out_row + blockIdx.y * S.out_layer) + head;
      const T x = in[a], y = in[b];
      const float xf = to_f32(x), yf = to_f32(y);
      out[a] = turned ? from_f32<T>(fmaf(xf, c, -(yf * s))) : x;
      out[b] = turned ? from_f32<T>(fmaf(yf, c, xf * s)) : y;
    }
  }
}

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// Frequencies as fractions of 2^64 a position.
bool turns_of(const double* f, int n, uint64_t* turn) {
  constexpr double kTurn = 6.283185307179586476925;
  for (int j = 0; j < n; ++j) {
    if (!std::isfinite(f[j])) return false;
    const double x = f[j] / kTurn, frac = x - std::floor(x);
    turn[j] = frac < 1.0 ? (uint64_t)(frac * 0x1p64) : 0;
  }
  return true;
}

template <typename T>
cudaError_t launch_rope(RopeJob& J, int d, int L, bool inter, bool rows, cudaStream_t st) {
  constexpr int N = 16 / (int)sizeof(T);
  // A warp a token, its angles worked out once for all heads, where tokens alone fill the
  // SMs; else a token's heads are shared out to as many warps as keep eight on each SM: 16 tokens of
  // 32 + 8 heads 2.6 us (a warp a token 5.6), 512 tokens 4.2 (6.7; sixteen warps on each SM 5.8).
  const int at_once = rows ? 32 / (d / (2 * N)) : 1, most = (J.heads + at_once - 1) / at_once;
  const int64_t tokens = (int64_t)J.T * L;
  J.warps = 1;
  while (J.warps < most && tokens * J.warps < 152 * 8) J.warps *= 2;
  const int64_t blocks = ((int64_t)J.T * J.warps + 7) / 8;
  const dim3 grid((unsigned)blocks, L);
  // No programmatic dependent: what it is rotated after is a projection, whose SMs it would find
  // with little L1 (attend_token.cu). 2,048 tokens of 28/4 heads after a library product 8.3 us (11.1),
  // 32,768 86 (90); alone the same.
  if (!rows)
    return inter ? launch_kernel(rope_pairs_kernel<T, true>, grid, 256, 0, st, false, 0, J, d)
                 : launch_kernel(rope_pairs_kernel<T, false>, grid, 256, 0, st, false, 0, J, d);
  auto go = [&](auto kernel) { return launch_kernel(kernel, grid, 256, 0, st, false, 0, J); };
  if (d == 128) return inter ? go(rope_rows_kernel<T, 128, true>) : go(rope_rows_kernel<T, 128, false>);
  return inter ? go(rope_rows_kernel<T, 64, true>) : go(rope_rows_kernel<T, 64, false>);
}

}  // namespace
}  // namespace mmshift

using namespace mmshift;

extern "C" {

mmshift_status mmshift_rope_frequencies(int32_t rot_dims, double theta, const mmshift_rope_scaling* scaling,
                                        double* inv_freq, float* amplitude) {
  if (rot_dims < 2 || rot_dims > 2 * kPairs || rot_dims % 2 || !inv_freq) return MMSHIFT_ERR_INVALID_ARG;
  if (!(theta > 0.0) || !std::isfinite(theta)) return MMSHIFT_ERR_INVALID_ARG;
  const int n = rot_dims / 2;
  const int kind = scaling ? scaling->kind : MMSHIFT_ROPE_SCALE_NONE;
  const double factor = kind == MMSHIFT_ROPE_SCALE_NONE ? 1.0 : scaling->factor;
  if (kind < MMSHIFT_ROPE_SCALE_NONE || kind > MMSHIFT_ROPE_SCALE_PARTS) return MMSHIFT_ERR_INVALID_ARG;
  if (!(factor >= 1.0) || !std::isfinite(factor)) return MMSHIFT_ERR_INVALID_ARG;
  if (kind == MMSHIFT_ROPE_SCALE_BASE && n < 2) return MMSHIFT_ERR_INVALID_ARG;
  if (kind == MMSHIFT_ROPE_SCALE_PARTS &&
      !(scaling->original_length > 0.0 && std::isfinite(scaling->original_length) && scaling->low_turns >= 0.0 &&
        scaling->high_turns > scaling->low_turns && std::isfinite(scaling->high_turns)))
    return MMSHIFT_ERR_INVALID_ARG;
  if (kind == MMSHIFT_ROPE_SCALE_BASE) theta *= std::pow(factor, (double)n / (n - 1));
  for (int j = 0; j < n; ++j) {
    double f = std::pow(theta, -(double)j / n);
    if (kind == MMSHIFT_ROPE_SCALE_LINEAR) f /= factor;
    if (kind == MMSHIFT_ROPE_SCALE_PARTS) {
      const double turns = scaling->original_length * f / 6.283185307179586476925;
      double keep = (turns - scaling->low_turns) / (scaling->high_turns - scaling->low_turns);
      keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
      f = f * keep + f / factor * (1.0 - keep);
    }
    inv_freq[j] = f;
  }
  if (amplitude) *amplitude = kind == MMSHIFT_ROPE_SCALE_PARTS ? (float)(0.1 * std::log(factor) + 1.0) : 1.f;
  return MMSHIFT_OK;
}

mmshift_status mmshift_rope(const mmshift_shape* s, const mmshift_rotary* r, const void* Q, int64_t q_row_stride,
                            int64_t q_layer_stride, const void* K, int64_t k_row_stride, int64_t k_layer_stride,
                            void* out_Q, void* out_K, mmshift_stream_t stream) {
  const mmshift_status st = check_rows(s);
  if (st != MMSHIFT_OK) return st;
  if (!r || !r->inv_freq) return MMSHIFT_ERR_INVALID_ARG;
  const int d = s->head_dim, rot = r->rot_dims ? r->rot_dims : d, T = s->cu_seqlens[s->batch], L = s->n_layers;
  const int axes = r->n_axes ? r->n_axes : 1;
  if (rot < 2 || rot > d || rot % 2) return MMSHIFT_ERR_INVALID_ARG;
  if (r->layout != MMSHIFT_ROPE_HALF && r->layout != MMSHIFT_ROPE_INTERLEAVED) return MMSHIFT_ERR_INVALID_ARG;
  if (r->inverse != 0 && r->inverse != 1) return MMSHIFT_ERR_INVALID_ARG;
  if (!(r->amplitude >= 0.f) || !std::isfinite(r->amplitude)) return MMSHIFT_ERR_INVALID_ARG;
  RopeJob J;
  std::memset(&J, 0, sizeof(J));
  J.axis1 = J.axis2 = rot / 2;
  if (axes < 1 || axes > 3) return MMSHIFT_ERR_INVALID_ARG;
  if (axes > 1) {
    int sum = 0;
    for (int i = 0; i < axes; ++i) {
      if (r->sections[i] < 0 || r->sections[i] > rot / 2) return MMSHIFT_ERR_INVALID_ARG;
      sum += r->sections[i];
    }
    if (sum != rot / 2) return MMSHIFT_ERR_INVALID_ARG;
    J.axis1 = r->sections[0];
    if (axes > 2) J.axis2 = r->sections[0] + r->sections[1];
  }
  if (!turns_of(r->inv_freq, rot / 2, J.turn)) return MMSHIFT_ERR_INVALID_ARG;
  const int64_t esz = s->dtype == MMSHIFT_BF16 ? 2 : 4;
  // 16-byte chunks: whole ones are rotated, and start where they may
  bool rows = r->layout == MMSHIFT_ROPE_HALF ? rot / 2 * esz % 16 == 0 : rot * esz % 32 == 0;
  auto side = [&](RopeSide& S, const void* in, void* out, int heads, int64_t row, int64_t layer) {
    if (!in != !out) return false;
    if (!in) return true;
    const int64_t dense = (int64_t)heads * d;
    if (!row) row = dense;
    if (row < dense || !aligned(in, esz) || !aligned(out, esz)) return false;
    if (L > 1 && !layer) layer = T * row;
    // layers one behind another, or side by side in a token's row
    if (L > 1 && T && layer < dense) return false;
    if (L > 1 && T > 1 && row > (layer - dense) / (T - 1) && (row - dense) / layer < L - 1) return false;
    S.in = static_cast<const uint8_t*>(in);
    S.out = static_cast<uint8_t*>(out);
    S.in_row = row * esz;
    S.in_layer = layer * esz;
    S.heads = heads;
    S.copy = in != out;
    S.out_row = (S.copy ? dense : row) * esz;
    S.out_layer = (S.copy ? T * dense : layer) * esz;
    rows = rows && aligned(in, 16) && aligned(out, 16) && S.in_row % 16 == 0 && (L == 1 || S.in_layer % 16 == 0);
    return true;
  };
  if ((!Q && !K && T) || (T && !r->positions) || !aligned(r->positions, 4)) return MMSHIFT_ERR_INVALID_ARG;
  if (!side(J.side[0], Q, out_Q, s->n_q_heads, q_row_stride, q_layer_stride) ||
      !side(J.side[1], K, out_K, s->n_kv_heads, k_row_stride, k_layer_stride))
    return MMSHIFT_ERR_INVALID_ARG;
  // Blocks run in any order: a dense output may not lie on rows that are read, of either side, nor on the other
  // output; and rows that are turned in place are Q's or K's.
  auto on_rows = [&](const RopeSide& A, const RopeSide& B) {
    const int64_t out = (int64_t)A.out, end = out + L * A.out_layer, bytes = (int64_t)B.heads * d * esz;
    for (int l = 0; l < L; ++l) {
      const int64_t in = (int64_t)B.in + l * B.in_layer, before = out - in - bytes;
      const int64_t t = before < 0 ? 0 : before / B.in_row + 1;   // the first row that ends behind the output's start
      if (t < T && in + t * B.in_row < end) return true;
    }
    return false;
  };
  for (int i = 0; T && i < 2; ++i) {
    const RopeSide &A = J.side[i], &B = J.side[1 - i];
    if (A.heads && A.copy && on_rows(A, A)) return MMSHIFT_ERR_INVALID_ARG;
    if (!A.heads || !B.heads) continue;
    if (A.copy && on_rows(A, B)) return MMSHIFT_ERR_INVALID_ARG;
    const int64_t gap = (int64_t)B.out - (int64_t)A.out;
    if (A.copy == B.copy && gap >= 0 && gap < (A.copy ? L * A.out_layer : (int64_t)A.heads * d * esz))
      return MMSHIFT_ERR_INVALID_ARG;
  }
  if (!T) return MMSHIFT_OK;
  J.pos = r->positions;
  J.T = T;
  J.heads = J.side[0].heads + J.side[1].heads;
  J.rot = rot;
  J.amp = r->amplitude > 0.f ? r->amplitude : 1.f;
  J.sine = r->inverse ? -J.amp : J.amp;
  const bool inter = r->layout == MMSHIFT_ROPE_INTERLEAVED;
  const cudaError_t e = s->dtype == MMSHIFT_BF16 ? launch_rope<__nv_bfloat16>(J, d, L, inter, rows, (cudaStream_t)stream)
                                                 : launch_rope<float>(J, d, L, inter, rows, (cudaStream_t)stream);
  return e == cudaSuccess ? MMSHIFT_OK : noalloc_cuda_fail(e);
}

}  // extern "C"
