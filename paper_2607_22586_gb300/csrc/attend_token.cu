// Attention of few query rows (tiles of up to 16 of a request and KV head: single tokens
// under grouped heads, a few drafted tokens) over bfloat16 or 8-bit pages.
//
// Bound by the bytes of K and V, which pass once from global memory to the
// registers of the warp that uses them: no shared memory, no barrier in
// the loop. 64 requests of one token, 64 heads, 2 to 24 thousand rows: 260 us over 8-bit
// pages (6.0 TB/s; 53 % of the issue slots), 446 over bfloat16 ones (6.8 TB/s). Each warp takes pieces of KEYS keys of its own and keeps its own
// running maximum, sums and output. Both products are m16n8k16 MMAs with
// the keys (and then the dimensions) as M and the query rows as N, so eight
// rows cost one column block and no product is spent on padding beyond that:
//   S^T [keys x rows] = K Q^T,   O^T [dims x rows] += V^T P^T.
// An MMA sums over its k index in any order, and the order of output
// dimensions is free too, so both are chosen such that a lane's fragment is 16
// (or 8) consecutive bytes of a row: lane (g, c) holds key g's dimensions of
// chunk c for S, and, for O, the keys 2c, 2c + 1, 2c + 8, 2c + 9 of dimension
// chunk g, whose pairs of keys one byte permutation brings together.
//
// 8-bit pages: both products take float16. A code x becomes float16 without
// rounding, three instructions for two: with u = x + 128, 1024 + u is the pattern
// 0x6400 | u, less 1152. (bfloat16 holds no 8 bits beside a leading one: five
// instructions, and this kernel was bound by them, 468 us for 64 requests of 2 to 24
// thousand rows.) A query row is scaled by a power of two that brings its largest
// value to 2^14, so what float16 cannot hold of it is below 2^-39 of that. K's scale
// goes to the logit. V's goes into the weight, whose float16 form is relative to the
// row's largest such product: w = 2^7 e^(z + ln vs - M), while the sum of weights is
// taken of e^(z - m) as ever. With 2^7, weights reach 2^15 (the maximum is only raised by steps,
// below), the last power of two that float16 holds; its lower end, where a half step is 2^-25,
// then lies at 2^-32 of the largest product: rounding is off by at most 2^-11 of a weight or
// by that. (Without it, 3,000 weights of e^-18 beside one of 1 were all rounded to zero.)
//
// The maxima are only raised when a value passes them by 8 (base 2), so the common
// step has one vote and no reduction: weights then stay below 2^8 (2^15 in the
// form above). bfloat16 rows: a weight
// is rounded to bfloat16, the MMA's operand, its sum is not.
#include "attend.cuh"
#include "umma.cuh"

namespace mmshift {
namespace {

constexpr int NT = 128, NW = NT / 32;
constexpr int kCluster = 8;
constexpr float kRaise = 8.f, kUp = 7.f;   // kRaise + kUp: the exponent of float16's last power of two

__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                         uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The transpose of an 8 x 8 matrix of 16-bit values, two of a row in each lane.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

__device__ __forceinline__ void mma16816_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                             uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Bytes b0, b1 of x (codes + 128), picked by `sel` as b0 64 b1 64, as two float16 codes.
template <int SEL>
__device__ __forceinline__ uint32_t codes_f16(uint32_t x) {
  uint32_t y;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(y) : "r"(__byte_perm(x, 0x64646464u, SEL)), "r"(0x64806480u));
  return y;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float fast_log2(float x) {
  float y;
  asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ bool not_finite2(uint32_t w) {
  return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
}

__device__ __forceinline__ uint4 load_stream(const uint8_t* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ uint2 load_stream8(const uint8_t* p) {
  uint2 v;
  asm volatile("ld.global.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}

// NQ: blocks of eight query rows.
template <int D, bool I8, int NQ>
struct Token {
  static constexpr int ROWB = I8 ? D : 2 * D;
  static constexpr int NB = 256 / ROWB;        // 16-key blocks of a piece: 4 KB of K and of V
  static constexpr int KEYS = 16 * NB;
  static constexpr int KC = ROWB / 64;         // 16-byte chunks of a key per lane
  static constexpr int VW = ROWB / 32;         // words of a value row per lane
  static constexpr int KS = D / 16;            // k steps of S
  static constexpr int MT = D / 16;            // dimension blocks of O
  static constexpr int SROW = D + 4;           // floats between rows in shared memory

  struct alignas(16) Smem {
    float o[NW][8 * NQ][SROW];
    float2 ml[NW][8 * NQ], part[8 * NQ];
    AttendScan<NT> scan;
  };

  // 16 words of K and V rows of a block each: k[half][.] is key g + 8 * half,
  // v[.][.] the keys 2c, 2c + 1, 2c + 8, 2c + 9.
  struct KBlock { uint32_t w[2][4 * KC]; float s[2]; };
  struct VBlock { uint32_t w[4][VW]; float s[2]; };

  static __device__ __forceinline__ void load_k(const CacheJob& J, KBlock& x, int row, int t, int end, int g, int c) {
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const bool in = row >= 0 && t + 8 * hf + g < end;
      const uint8_t* p = J.kp + ((size_t)row + 8 * hf + g) * ROWB + c * 16;
#pragma unroll
      for (int i = 0; i < KC; ++i) {
        const uint4 v = in ? load_stream(p + i * 64) : make_uint4(0, 0, 0, 0);
        x.w[hf][4 * i] = v.x;
        x.w[hf][4 * i + 1] = v.y;
        x.w[hf][4 * i + 2] = v.z;
        x.w[hf][4 * i + 3] = v.w;
      }
      if constexpr (I8) x.s[hf] = in ? J.ks[(size_t)row + 8 * hf + g] : 0.f;
    }
  }

  static __device__ __forceinline__ void load_v(const CacheJob& J, VBlock& x, int row, int t, int end, int g, int c) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int key = 2 * c + (k & 1) + 8 * (k >> 1);
      const bool in = row >= 0 && t + key < end;
      if constexpr (VW >= 4) {
        const uint8_t* p = J.vp + ((size_t)row + key) * ROWB + g * 16;
#pragma unroll
        for (int i = 0; i < VW / 4; ++i) {
          const uint4 v = in ? load_stream(p + i * 128) : make_uint4(0, 0, 0, 0);
          x.w[k][4 * i] = v.x;
          x.w[k][4 * i + 1] = v.y;
          x.w[k][4 * i + 2] = v.z;
          x.w[k][4 * i + 3] = v.w;
        }
      } else {
        const uint2 v = in ? load_stream8(J.vp + ((size_t)row + key) * ROWB + g * 8) : make_uint2(0, 0);
        x.w[k][0] = v.x;
        x.w[k][1] = v.y;
      }
    }
    if constexpr (I8) {
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) x.s[hf] = row >= 0 && t + 8 * hf + g < end ? J.vs[(size_t)row + 8 * hf + g] : 0.f;
    }
  }

  // A fragments of k step `s` of S.
  static __device__ __forceinline__ void k_frag(const KBlock& x, int s, uint32_t (&a)[4]) {
    if constexpr (!I8) {
      a[0] = x.w[0][2 * s];
      a[1] = x.w[1][2 * s];
      a[2] = x.w[0][2 * s + 1];
      a[3] = x.w[1][2 * s + 1];
    } else {
      const uint32_t u0 = x.w[0][s] ^ 0x80808080u, u1 = x.w[1][s] ^ 0x80808080u;
      a[0] = codes_f16<0x4140>(u0);
      a[1] = codes_f16<0x4140>(u1);
      a[2] = codes_f16<0x4342>(u0);
      a[3] = codes_f16<0x4342>(u1);
    }
  }

  // A fragments of dimension blocks 2j and 2j + 1 of O^T: rows g and g + 8 of a block
  // are two neighbouring dimensions of chunk g.
  static __device__ __forceinline__ void v_frag(const VBlock& x, int j, uint32_t (&a)[2][4]) {
    if constexpr (!I8) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int m = 2 * j + e;
        a[e][0] = __byte_perm(x.w[0][m], x.w[1][m], 0x5410);
        a[e][1] = __byte_perm(x.w[0][m], x.w[1][m], 0x7632);
        a[e][2] = __byte_perm(x.w[2][m], x.w[3][m], 0x5410);
        a[e][3] = __byte_perm(x.w[2][m], x.w[3][m], 0x7632);
      }
    } else {
#pragma unroll
      for (int k = 0; k < 4; k += 2) {                 // keys 2c, 2c + 1, then 2c + 8, 2c + 9
        const uint32_t p = x.w[k][j] ^ 0x80808080u, q = x.w[k + 1][j] ^ 0x80808080u;
        const uint32_t lo = __byte_perm(p, q, 0x5140), hi = __byte_perm(p, q, 0x7362);
        a[0][k] = codes_f16<0x4140>(lo);
        a[0][k + 1] = codes_f16<0x4342>(lo);
        a[1][k] = codes_f16<0x4140>(hi);
        a[1][k + 1] = codes_f16<0x4342>(hi);
      }
    }
  }
  static __device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (I8) mma16816_f16(d, a[0], a[1], a[2], a[3], b0, b1);
    else mma16816(d, a[0], a[1], a[2], a[3], b0, b1);
  }

  // The first of the two dimensions of block m in lanes of chunk g.
  static __device__ __forceinline__ int dim_of(int m, int g) {
    if constexpr (!I8) return (m / 4) * 64 + g * 8 + (m % 4) * 2;
    else return g * (D / 8) + 2 * m;
  }
};

// CLUSTER: a cluster of kCluster CTAs has a unit, each an equal part of its pieces, and
// merges the parts through distributed shared memory: one launch, no lengths to add up.
// For calls of few units that can only be short (see launch_attend); others are
// balanced over all SMs, and merged by a kernel of their own.
template <int D, bool I8, int NQ, bool CLUSTER>
__global__ void __launch_bounds__(NT, NQ == 1 ? 3 : 2) attend_token_kernel(const __grid_constant__ AttendJob A,
                                                                           const __grid_constant__ AttendPlan P) {
  using T = Token<D, I8, NQ>;
  __shared__ typename T::Smem sm;
  cache_start();
  const CacheJob& J = A.c;
  const int lane = threadIdx.x % 32, w = threadIdx.x / 32, g = lane / 4, c = lane % 4;
  const int rank = CLUSTER ? blockIdx.x % kCluster : 0;
  const AttendSpan sp = CLUSTER ? AttendSpan{0, 1, 0, (int)blockIdx.x / kCluster} : attend_span(A, P, &sm.scan);
  int u = sp.unit;
  int64_t before = sp.before;
  for (int64_t at = sp.begin; at < sp.end;) {
    const AttendUnit U = attend_unit(A, P, CLUSTER ? nullptr : sm.scan.lengths(A.c), u);
    const int64_t last = before + U.cost, stop = min(sp.end, last);
    int s0, s1;
    if constexpr (CLUSTER) {
      s0 = U.pieces * rank / kCluster;
      s1 = U.pieces * (rank + 1) / kCluster;
    } else {
      if (last <= at) {                                // a unit without pieces
        before = last;
        ++u;
        continue;
      }
      attend_pieces(U, at, stop, before, s0, s1);
      if (s0 >= s1) {                                  // the unit's start alone
        at = stop;
        continue;
      }
    }
    const int32_t* table = cache_table(J, (size_t)U.b * J.Hkv + U.h);

    // Raises a maximum to its row's of the step; what sums relative to it have to be multiplied by.
    auto raise_max = [&](float& m, auto&& value) {
      float top = m;
#pragma unroll
      for (int nb = 0; nb < T::NB; ++nb) top = fmaxf(top, fmaxf(value(nb, 0), value(nb, 1)));
#pragma unroll
      for (int z = 4; z < 32; z <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, z));
      const float f = m == -INFINITY ? 0.f : fast_exp2(m - top);
      m = top;
      return f;
    };
    auto rows_of = [&](int s, int (&row)[T::NB]) {
#pragma unroll
      for (int nb = 0; nb < T::NB; ++nb) {
        const int t = s * T::KEYS + 16 * nb;
        row[nb] = s < s1 && t < U.keys ? page_row(table[t >> J.page_shift], J.n_pages, J.page_shift, t) : -1;
      }
    };
    typename T::KBlock kb[T::NB];
    typename T::VBlock vb[T::NB];
    int row[T::NB], next[T::NB];
    int s = s0 + w;
    rows_of(s, row);
    rows_of(s + NW, next);
#pragma unroll
    for (int nb = 0; nb < T::NB; ++nb) T::load_k(J, kb[nb], row[nb], s * T::KEYS + 16 * nb, U.keys, g, c);
#pragma unroll
    for (int nb = 0; nb < T::NB; ++nb) T::load_v(J, vb[nb], row[nb], s * T::KEYS + 16 * nb, U.keys, g, c);

    // query rows as B fragments: row 8 * nq + g
    uint32_t q[NQ][2 * T::KS];
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
      const int row = 8 * nq + g;
      const bool in = row < U.rows;
      const int all = in ? U.row0 + row : 0, tok = J.by_r(all), j = all - tok * J.r;
      const uint8_t* p = A.q + ((size_t)(J.off[U.b] + tok) * J.stride + (size_t)(U.h * J.r + j) * D) * 2;
#pragma unroll
      for (int i = 0; i < 2 * T::KS / 4; ++i) {
        // words of k steps 2i, 2i + 1: dimensions 8c.. of each 32 (bfloat16 pages), 16c.. of each 64 (codes)
        const int d0 = I8 ? (i / 2) * 64 + c * 16 + (i % 2) * 8 : i * 32 + c * 8;
        const uint4 v = in ? load_plain16(p + d0 * 2, A.qvec) : make_uint4(0, 0, 0, 0);
        q[nq][4 * i] = v.x;
        q[nq][4 * i + 1] = v.y;
        q[nq][4 * i + 2] = v.z;
        q[nq][4 * i + 3] = v.w;
      }
    }
    // rows 8 * nq + 2c and + 1 as columns of the products
    float m[NQ][2], l[NQ][2], o[NQ][T::MT][4];
    float mw[NQ][2], alpha[NQ][2];                     // 8-bit pages: M, and alpha over the row's power of two
    if constexpr (I8) {
#pragma unroll
      for (int nq = 0; nq < NQ; ++nq) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 2 * T::KS; ++i) top = max(top, max(q[nq][i] & 0x7fffu, (q[nq][i] >> 16) & 0x7fffu));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // 2^k with k = 14 - exponent of the largest, at most 126 (a largest below 2^-112 or a row of zeros)
        const int k = min(14 - ((int)(top >> 7) - 127), 126);
        const float f = __uint_as_float((uint32_t)(127 + k) << 23);
#pragma unroll
        for (int i = 0; i < 2 * T::KS; ++i) q[nq][i] = pack_f16(bf16_lo(q[nq][i]) * f, bf16_hi(q[nq][i]) * f);
        const float back = A.alpha * __uint_as_float((uint32_t)(127 - k) << 23);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          alpha[nq][e] = __shfl_sync(0xffffffffu, back, 4 * (2 * c + e));
          mw[nq][e] = -INFINITY;
        }
      }
    }
    int lim[NQ][2];
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        m[nq][e] = -INFINITY;
        l[nq][e] = 0.f;
        lim[nq][e] = keys_of(A.causal, U.len, U.n, J.by_r(U.row0 + min(8 * nq + 2 * c + e, U.rows - 1)));
#pragma unroll
        for (int mt = 0; mt < T::MT; ++mt) o[nq][mt][e] = o[nq][mt][2 + e] = 0.f;
      }
    const int least = keys_of(A.causal, U.len, U.n, J.by_r(U.row0));   // keys that every row attends to

    for (; s < s1; s += NW) {
      const int t0 = s * T::KEYS;
      float x[NQ][T::NB][4];                           // keys g, g | g + 8, g + 8; rows 2c, 2c + 1
#pragma unroll
      for (int nb = 0; nb < T::NB; ++nb) {
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
          for (int i = 0; i < 4; ++i) x[nq][nb][i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < T::KS; ++ks) {
          uint32_t a[4];
          T::k_frag(kb[nb], ks, a);
#pragma unroll
          for (int nq = 0; nq < NQ; ++nq) T::mma(x[nq][nb], a, q[nq][2 * ks], q[nq][2 * ks + 1]);
        }
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
          for (int i = 0; i < 4; ++i) x[nq][nb][i] *= I8 ? kb[nb].s[i / 2] * alpha[nq][i % 2] : A.alpha;
      }
      float y[I8 ? NQ : 1][T::NB][4];                  // 8-bit pages: with V's scales
      if constexpr (I8) {
#pragma unroll
        for (int nb = 0; nb < T::NB; ++nb) {
          const float lv[2] = {fast_log2(vb[nb].s[0]), fast_log2(vb[nb].s[1])};
#pragma unroll
          for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
            for (int i = 0; i < 4; ++i) y[nq][nb][i] = x[nq][nb][i] + lv[i / 2];
        }
      }
      const int tn = t0 + NW * T::KEYS;
#pragma unroll
      for (int nb = 0; nb < T::NB; ++nb) T::load_k(J, kb[nb], next[nb], tn + 16 * nb, U.keys, g, c);

      bool gone = false;
#pragma unroll
      for (int nb = 0; nb < T::NB; ++nb) gone |= row[nb] < 0 && t0 + 16 * nb < U.keys;
      const bool masked = t0 + T::KEYS > least || gone;
      if (masked) {
        if (gone && lane == 0) set_status(J.status, kStatusBadPage);
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
          for (int nb = 0; nb < T::NB; ++nb)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (row[nb] < 0 || t0 + 16 * nb + 8 * (i / 2) + g >= lim[nq][i % 2]) {
                x[nq][nb][i] = -INFINITY;
                if constexpr (I8) y[nq][nb][i] = -INFINITY;
              }
      }
      bool raise = false;
#pragma unroll
      for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
        for (int nb = 0; nb < T::NB; ++nb)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            raise |= x[nq][nb][i] > m[nq][i % 2] + kRaise;
            if constexpr (I8) raise |= y[nq][nb][i] > mw[nq][i % 2] + kRaise;
          }
      if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float f = raise_max(m[nq][e], [&](int nb, int hf) { return x[nq][nb][2 * hf + e]; });
            l[nq][e] *= f;
            if constexpr (I8) f = raise_max(mw[nq][e], [&](int nb, int hf) { return y[nq][nb][2 * hf + e]; });
#pragma unroll
            for (int mt = 0; mt < T::MT; ++mt) {
              o[nq][mt][e] *= f;
              o[nq][mt][2 + e] *= f;
            }
          }
      }
      uint32_t p[NQ][T::NB][2];
#pragma unroll
      for (int nq = 0; nq < NQ; ++nq) {
        const float m0 = m[nq][0] == -INFINITY ? 0.f : m[nq][0], m1 = m[nq][1] == -INFINITY ? 0.f : m[nq][1];
        float w0 = 0.f, w1 = 0.f;
        if constexpr (I8) {
          w0 = mw[nq][0] == -INFINITY ? 0.f : mw[nq][0] - kUp;
          w1 = mw[nq][1] == -INFINITY ? 0.f : mw[nq][1] - kUp;
        }
#pragma unroll
        for (int nb = 0; nb < T::NB; ++nb) {
          float e[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            e[i] = fast_exp2(x[nq][nb][i] - (i % 2 ? m1 : m0));
            l[nq][i % 2] += e[i];
            if constexpr (I8) e[i] = fast_exp2(y[nq][nb][i] - (i % 2 ? w1 : w0));
          }
          p[nq][nb][0] = transpose8(I8 ? pack_f16(e[0], e[1]) : pack_bf16(e[0], e[1]));
          p[nq][nb][1] = transpose8(I8 ? pack_f16(e[2], e[3]) : pack_bf16(e[2], e[3]));
        }
      }
      bool plain = true;
      if constexpr (!I8) {
        // A zero weight times a value that is not finite is a NaN. Where a tile has
        // such values behind some row's last key, the keys are multiplied one by one
        // and a row takes only those that it attends to.
        if (masked) {
          bool odd = false;
#pragma unroll
          for (int nb = 0; nb < T::NB; ++nb)
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
              for (int i = 0; i < T::VW; ++i) odd |= not_finite2(vb[nb].w[k][i]);
          plain = !__any_sync(0xffffffffu, odd);
        }
      }
      if (plain) {
#pragma unroll
        for (int nb = 0; nb < T::NB; ++nb)
#pragma unroll
          for (int j = 0; j < T::MT / 2; ++j) {
            uint32_t a[2][4];
            T::v_frag(vb[nb], j, a);
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
              for (int nq = 0; nq < NQ; ++nq) T::mma(o[nq][2 * j + e], a[e], p[nq][nb][0], p[nq][nb][1]);
          }
      } else {
#pragma unroll
        for (int nb = 0; nb < T::NB; ++nb)
#pragma unroll 1
          for (int k = 0; k < 16; ++k) {
            const uint32_t half = (k & 7) >> 1 == c ? (k & 1 ? 0xffff0000u : 0xffffu) : 0u;
            const uint32_t lo = k < 8 ? half : 0u, hi = k < 8 ? 0u : half;
#pragma unroll
            for (int j = 0; j < T::MT / 2; ++j) {
              uint32_t a[2][4];
              T::v_frag(vb[nb], j, a);
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const uint32_t b[4] = {a[e][0] & lo, a[e][1] & lo, a[e][2] & hi, a[e][3] & hi};
#pragma unroll
                for (int nq = 0; nq < NQ; ++nq) {
                  float d[4] = {};
                  T::mma(d, b, p[nq][nb][0], p[nq][nb][1]);
#pragma unroll
                  for (int i = 0; i < 4; ++i)
                    if (t0 + 16 * nb + k < lim[nq][i % 2]) o[nq][2 * j + e][i] += d[i];
                }
              }
            }
          }
      }
#pragma unroll
      for (int nb = 0; nb < T::NB; ++nb) T::load_v(J, vb[nb], next[nb], tn + 16 * nb, U.keys, g, c);
#pragma unroll
      for (int nb = 0; nb < T::NB; ++nb) row[nb] = next[nb];
      rows_of(s + 2 * NW, next);
    }

    // the warps' sums together
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float z = l[nq][e];
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) z += __shfl_xor_sync(0xffffffffu, z, d);
        const int r = 8 * nq + 2 * c + e;
        if constexpr (I8) {                            // O relative to m
          const float f = mw[nq][e] == -INFINITY ? 1.f : exp2f(mw[nq][e] - kUp - m[nq][e]);
#pragma unroll
          for (int mt = 0; mt < T::MT; ++mt) {
            o[nq][mt][e] *= f;
            o[nq][mt][2 + e] *= f;
          }
        }
        if (g == 0) sm.ml[w][r] = make_float2(m[nq][e], z);
#pragma unroll
        for (int mt = 0; mt < T::MT; ++mt)
          *reinterpret_cast<float2*>(&sm.o[w][r][T::dim_of(mt, g)]) = make_float2(o[nq][mt][e], o[nq][mt][2 + e]);
      }
    __syncthreads();
    const bool whole = s0 == 0 && s1 == U.pieces;
    const size_t slot = (size_t)attend_slot(blockIdx.x, sp.begin, before) * P.rows;
    for (int i = threadIdx.x; i < U.rows * (D / 4); i += NT) {
      const int r = i / (D / 4), d0 = i % (D / 4) * 4;
      float top = -INFINITY;
#pragma unroll
      for (int k = 0; k < NW; ++k) top = fmaxf(top, sm.ml[k][r].x);
      float z = 0.f;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < NW; ++k) {
        const float2 ml = sm.ml[k][r];
        // a warp without a maximum has zeros, or NaN that have to stay
        const float f = ml.x == -INFINITY ? 1.f : fast_exp2(ml.x - top);
        const float4 v = *reinterpret_cast<const float4*>(&sm.o[k][r][d0]);
        z += ml.y * f;
        acc.x += v.x * f;
        acc.y += v.y * f;
        acc.z += v.z * f;
        acc.w += v.w * f;
      }
      if constexpr (CLUSTER) {
        *reinterpret_cast<float4*>(&sm.o[0][r][d0]) = acc;   // read by this thread alone
        if (d0 == 0) sm.part[r] = make_float2(top, z);
      } else if (whole) {
        attend_write<__nv_bfloat16, D, true>(A, U.b, U.h, U.row0 + r, d0, acc, top, z);
      } else {
        *reinterpret_cast<float4*>(P.po + (slot + r) * D + d0) = acc;
        if (d0 == 0) P.pml[slot + r] = make_float2(top, z);
      }
    }
    if constexpr (CLUSTER) {
      umma::cluster_sync();
      for (int i = rank * NT + threadIdx.x; i < U.rows * (D / 4); i += kCluster * NT) {
        const int r = i / (D / 4), d0 = i % (D / 4) * 4;
        const uint32_t po = umma::smem_u32(&sm.o[0][r][d0]), pm = umma::smem_u32(&sm.part[r]);
        float2 ml[kCluster];
        float top = -INFINITY, z = 0.f;
#pragma unroll
        for (int k = 0; k < kCluster; ++k) {
          ml[k] = umma::ld_cluster_f2(umma::mapa(pm, k));
          top = fmaxf(top, ml[k].x);
        }
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < kCluster; ++k) {
          const float f = ml[k].x == -INFINITY ? 1.f : fast_exp2(ml[k].x - top);
          const uint32_t p = umma::mapa(po, k);
          const float2 a = umma::ld_cluster_f2(p), b = umma::ld_cluster_f2(p + 8);
          z += ml[k].y * f;
          acc.x += a.x * f;
          acc.y += a.y * f;
          acc.z += b.x * f;
          acc.w += b.y * f;
        }
        attend_write<__nv_bfloat16, D, true>(A, U.b, U.h, U.row0 + r, d0, acc, top, z);
      }
      umma::cluster_sync();                            // the others have read this CTA's part
      at = sp.end;
    } else {
      __syncthreads();
      at = stop;
      if (stop == last) {
        before = last;
        ++u;
      }
    }
  }
}

}  // namespace

cudaError_t launch_attend_token(const AttendJob& A, const AttendPlan& P, bool cluster, bool overlap, cudaStream_t st) {
  const CacheJob& J = A.c;
  // Not as a programmatic dependent (`overlap`) behind a kernel that has all of an SM's shared memory: its
  // CTAs would come to an SM that is never idle in between and seems to keep that split, with little L1
  // for loads in flight, whatever split the launch prefers. 64 requests of one token over 1,265 rows,
  // 64/8 heads, bfloat16, after the pages they share: 66 us (82); without such a kernel in front a
  // dependent saves 2 us.
  auto go = [&](auto whole, auto parts) {
    if (cluster)
      return launch_kernel(parts, dim3(P.uoff[J.B] * kCluster), NT, 0, st, overlap, kCluster, A, P);
    return launch_kernel(whole, dim3(P.workers), NT, 0, st, overlap, 0, A, P);
  };
#define MMSHIFT_TOKEN(D, I8, NQ) go(attend_token_kernel<D, I8, NQ, false>, attend_token_kernel<D, I8, NQ, true>)
  if (P.rows <= 8) {
    if (J.d == 128) return J.i8 ? MMSHIFT_TOKEN(128, true, 1) : MMSHIFT_TOKEN(128, false, 1);
    return J.i8 ? MMSHIFT_TOKEN(64, true, 1) : MMSHIFT_TOKEN(64, false, 1);
  }
  if (J.d == 128) return J.i8 ? MMSHIFT_TOKEN(128, true, 2) : MMSHIFT_TOKEN(128, false, 2);
  return J.i8 ? MMSHIFT_TOKEN(64, true, 2) : MMSHIFT_TOKEN(64, false, 2);
#undef MMSHIFT_TOKEN
}

}  // namespace mmshift
