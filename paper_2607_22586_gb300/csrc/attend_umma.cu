// Attention of chunks (more than 32 query rows of a request and KV head) on the
// 5th-generation tensor cores (tcgen05 + TMA + TMEM).
//
// Tiles of 256 query rows, two blocks of 128, over tiles of 128 keys:
//   S = Q K^T   [128 x 128]  both operands in shared memory, S in tensor memory;
//   O += P V    [128 x d]    P in tensor memory, over the columns of its S, V in
//               shared memory as it lies in the page (keys by dimensions: the
//               MN-major B operand), O in tensor memory for the whole run of keys.
// Roles (384 threads, 512 over 8-bit pages, one CTA per SM):
//   warps 0-7   softmax, one warpgroup a block, one thread a row (its maximum and
//               sum need no reduction across threads; over 8-bit pages four
//               threads have four rows). They read S, write P and, at the end of
//               the run, O;
//   warp 8      TMA producer: a ring of K and V tiles. A page is a box of up to
//               128 rows, so a tile is 1 to 8 boxes and 64 columns wide halves;
//   warp 9      MMA issuer;
//   warps 12-15 (8-bit pages) make codes bfloat16.
// The blocks alternate: while one block's softmax runs, the tensor cores have
// the other block's products. Tiles of at most 128 rows take the blocks in turn, so
// that one's results go out while the next one begins. A row's maximum is only raised
// when a logit passes it by 8 (base 2); then the thread rescales its row of O itself,
// which is idle at that point: S of a tile is complete only after the products of the
// tile before. 2048 tokens of 28 heads over 34816 rows: 620 us in short runs, 640 to 660 in long
// ones, 1.50 to 1.60 PFLOP/s (8-bit pages 1080: 2.3 times the instructions, for codes and scales;
// 54 % of the issue slots, the tensor pipe at 37 %). S in halves, its maximum checked against the
// one there is instead of read first, took 685 (1093). A run's start (lengths, Q) and end (O) take
// about 10 us, which is what short chunks wait for: 16 prompts of 1000 tokens on their own rows
// 273 us. P is rounded to bfloat16 (the tensor cores' operand type), its sum is not.
//
// Tiles that hold keys which some row of the tile does not attend to (the chunk's
// own keys under the causal mask, the last tile) are masked, and their V rows are
// cleaned first: behind the last key a page may hold anything, and a zero weight
// times a NaN is a NaN. Values that are not finite and that some rows do attend to
// are set to zero for the product and added to those rows at the end.
// Every wait is bounded; a role that gives up ends the CTA as score_umma.cu says.
#include <cudaTypedefs.h>

#include <algorithm>
#include <type_traits>

#include "attend_umma.cuh"

namespace mmshift {
namespace {

using namespace umma;

constexpr int PRODUCER = 8, ISSUER = 9, CONVERT = 12;   // first warps of the roles

template <int D, bool I8>
struct ChunkSmem {
  static constexpr int NT = I8 ? 512 : 384;
  static constexpr int HALVES = D / 64;
  static constexpr int HALF = BK * 128;              // 64 columns of 128 rows
  static constexpr int TILE = HALVES * HALF;         // a block of Q, a tile of K or V
  static constexpr int STAGES = D == 64 ? 8 : I8 ? 3 : 5;
  static_assert(STAGES >= 3, "v_before_s(): a tile's V is three positions behind the K of the tile before");
  static constexpr int RAW = BK * D;                 // a tile of codes
  // Tiles whose scales are kept: those of tile j + SCALES are written when its K has a
  // stage, which is after the V of tile j was freed, and so read by all.
  static constexpr int SCALES = 8;
  static_assert(2 * SCALES - STAGES >= 1, "scales would be overwritten while they are read");
  static constexpr int RAWS = I8 ? (D == 64 ? 6 : 3) : 0;
  static constexpr int BYTES = (2 + STAGES) * TILE + RAWS * RAW + 1024;
  static constexpr uint32_t O_COL = 256, O_STRIDE = D;
};

__device__ __forceinline__ void pin16(float* v) {
  asm volatile("" : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]),
                    "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]),
                    "+f"(v[15]));
}
// 16 lanes by 32 columns, spread as an MMA's accumulator: v[4k], v[4k + 1] are row
// lane / 4, columns 8k + 2 (lane % 4) and the next; v[4k + 2], v[4k + 3] row lane / 4 + 8.
__device__ __forceinline__ void ld_quads(uint32_t taddr, float* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
        "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
      : "r"(taddr));
}
// 16 lanes by 16 columns: w[2k] is row lane / 4, column 4k + lane % 4, w[2k + 1] row lane / 4 + 8.
__device__ __forceinline__ void st_quads(uint32_t taddr, const uint32_t* w) {
  asm volatile("tcgen05.st.sync.aligned.16x128b.x4.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(w[0]),
               "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}
// Two codes, in the low bytes of t's halves, as bfloat16.
__device__ __forceinline__ uint32_t codes_bf16(uint32_t t) {
  const uint32_t a = (t & 0x007f007fu) | 0x43004300u, c = (t & 0x00800080u) | 0x43004300u;
  uint32_t x;
  asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(x) : "r"(a), "r"(c));
  return x;
}
__device__ __forceinline__ uint64_t fmul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
// The part of a row's sums that comes from values that are not finite, of columns
// [d0, d0 + 32): added with the row's weights, key by key. Rare, so slow.
template <int D>
static __device__ __noinline__ void add_not_finite(const AttendJob& A, const Run& R, int row, int lim, float m, int d0,
                                                   float* o) {
  const CacheJob& J = A.c;
  const size_t seq = (size_t)R.U.b * J.Hkv + R.U.h;
  const int tok = J.by_r(row), j = row - tok * J.r;
  const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(A.q) +
                           (size_t)(J.off[R.U.b] + tok) * J.stride + (size_t)(R.U.h * J.r + j) * D;
  const int first = keys_of(A.causal, R.U.len, R.U.n, J.by_r(R.U.row0));
  for (int t = max(R.s0 * BK, first / BK * BK); t < min(R.s1 * BK, lim); ++t) {
    const int64_t slot = cache_slot(J, seq, t);
    if (slot < 0) continue;
    const __nv_bfloat16* v = reinterpret_cast<const __nv_bfloat16*>(J.vp) + (size_t)slot * D + d0;
    bool any = false;
    for (int i = 0; i < 32; ++i) any |= !isfinite(to_f32(v[i]));
    if (!any) continue;
    const __nv_bfloat16* k = reinterpret_cast<const __nv_bfloat16*>(J.kp) + (size_t)slot * D;
    float s = 0.f;
    for (int i = 0; i < D; ++i) s = fmaf(to_f32(q[i]), to_f32(k[i]), s);
    const float p = fast_exp2(fmaf(s, A.alpha, -m));
    for (int i = 0; i < 32; ++i) {
      const float x = to_f32(v[i]);
      if (!isfinite(x)) o[i] += p * x;
    }
  }
}

template <int D, bool I8>
__global__ void __launch_bounds__(ChunkSmem<D, I8>::NT, 1) attend_chunk_kernel(const __grid_constant__ CUtensorMap kmap,
                                                             const __grid_constant__ CUtensorMap vmap,
                                                             const __grid_constant__ AttendJob A,
                                                             const __grid_constant__ AttendPlan P) {
  using SM = ChunkSmem<D, I8>;
  constexpr int NT = SM::NT;
  extern __shared__ unsigned char smraw[];
  unsigned char* sm =
      reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smraw) + 1023) & ~uintptr_t(1023));
  unsigned char* ring = sm + 2 * SM::TILE;
  unsigned char* raw = ring + SM::STAGES * SM::TILE;
  __shared__ uint64_t rfull[I8 ? SM::RAWS : 1], rempty[I8 ? SM::RAWS : 1];
  __shared__ alignas(16) float scales[I8 ? SM::SCALES : 1][2][I8 ? BK : 1];   // K's (times alpha) and V's
  // Every wait is for the next fill of its stage that the waiting warp does not know to be complete,
  // or for one that is: producer, converters and issuer pass all positions of the ring, the softmax
  // blocks see v_before_s().
  __shared__ uint64_t full[SM::STAGES], empty[SM::STAGES], q_ready[2], s_ready[2], o_ready[2], o_free[2];
  __shared__ uint64_t p_ready[2], drain;
  __shared__ uint32_t tbase;
  __shared__ int abort_flag, odd_flag;
  __shared__ AttendScan<NT, 1> scan;
  __shared__ RunList<16> runs;
  volatile int* abort_ = &abort_flag;
  const CacheJob& J = A.c;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;

  if (threadIdx.x == 0) {
    abort_flag = odd_flag = 0;
    for (int s = 0; s < SM::STAGES; ++s) {
      mbar_init(&full[s], I8 ? 4 : 1);
      mbar_init(&empty[s], 1);
    }
    for (int s = 0; s < SM::RAWS; ++s) {
      mbar_init(&rfull[s], 1);
      mbar_init(&rempty[s], 4);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&q_ready[i], 4);     // a warpgroup's warps
      mbar_init(&s_ready[i], 1);
      mbar_init(&p_ready[i], 4);
      mbar_init(&o_ready[i], 1);
      mbar_init(&o_free[i], 4);
    }
    mbar_init(&drain, 1);
    fence_barrier_init();
    prefetch_tmap(&kmap);
    prefetch_tmap(&vmap);
  }
  if (warp == ISSUER) {
    tmem_alloc(&tbase, 512);
    tmem_relinquish();
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = tbase;
  cache_start();
  const AttendSpan sp = attend_span(A, P, &scan);
  if (warp == 0) list_runs(A, P, sp, lane, &runs);
  __syncthreads();
  Walk walk = {0, 0, 0, 0};
  Run R;
  if (warp == PRODUCER) {
    // bfloat16 rows go where the MMAs read them, codes to a ring of their own
    constexpr int NS = I8 ? SM::RAWS : SM::STAGES, BYTES = I8 ? SM::RAW : SM::TILE;
    uint64_t *const got = I8 ? rfull : full, *const room = I8 ? rempty : empty;
    int stage = 0;
    uint32_t phase = 0;
    ArmedStages armed;
    bool ok = true;
    const int shift = min(J.page_shift, 7), boxes = BK >> shift;
    const int outside = J.n_pages << J.page_shift;     // a box from there on reads zeros
    while (ok && next_run(A, P, sp, runs, walk, R)) {
      const int32_t* table = cache_table(J, (size_t)R.U.b * J.Hkv + R.U.h);
      // this lane's box of a tile: its row of the pool
      auto entry_of = [&](int s) {
        const int t = s * BK + (lane << shift);
        return lane < boxes && s < R.s1 && t < R.U.keys ? table[t >> J.page_shift] : -1;
      };
      int next = entry_of(R.s0);
      for (int s = R.s0; ok && s < R.s1; ++s) {
        const int got_row = page_row(next, J.n_pages, J.page_shift, s * BK + (lane << shift));
        const int row = got_row < 0 ? outside : got_row;
        next = entry_of(s + 1);                        // read a tile ahead
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          if (!wait_bar(&room[stage], phase ^ 1u, abort_)) { ok = false; break; }
          if (lane == 0) mbar_expect_tx(&got[stage], BYTES);
          armed.arm(stage, phase);
          __syncwarp();
          if (lane < boxes) {
            if constexpr (I8) {
              tma_load_3d(raw + stage * SM::RAW + (lane << shift) * D, kv ? &vmap : &kmap, &got[stage], 0, row, 0);
            } else {
#pragma unroll
              for (int c = 0; c < SM::HALVES; ++c)
                tma_load_3d(ring + stage * SM::TILE + c * SM::HALF + (lane << shift) * 128, kv ? &vmap : &kmap,
                            &got[stage], c * 64, row, 0);
            }
          }
          if (++stage == NS) { stage = 0; phase ^= 1u; }
        }
      }
    }
    if (!armed.drain(got)) *abort_ = 1;
  } else if (warp == ISSUER) {
    const uint32_t id_s = idesc_bf16_f32(BQ, BK), id_o = idesc_bf16_f32(BQ, D) | (1u << 16);   // V: MN-major
    const uint64_t qd = sdesc_k_sw128(smem_u32(sm)), kd = sdesc_k_sw128(smem_u32(ring));
    const uint64_t vd = sdesc_mn_sw128(smem_u32(ring), SM::HALF);
    int stage = 0;
    uint32_t phase = 0, qp = 0, pp = 0, of = 0;        // of the ring; bit i: of block i's barriers
    bool ok = true, issued = false;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      ok = ok && wait_bar(bar, parity & 1u, abort_);
      return ok;
    };
    auto step = [&] {
      if (++stage == SM::STAGES) { stage = 0; phase ^= 1u; }
    };
    auto commit = [&](uint64_t* bar) {
      if (elect_one()) mma_commit(bar);
      __syncwarp();
    };
    // S of block x with the K tile of the stage
    auto issue_s = [&](int x) {
      if (elect_one()) {
        const uint64_t k = kd + (uint64_t)(stage * (SM::TILE >> 4)), q = qd + (uint64_t)(x * (SM::TILE >> 4));
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          const uint64_t o = (uint64_t)(((ks / 4) * SM::HALF + (ks % 4) * 32) >> 4);
          mma_bf16(tmem + x * BK, q + o, k + o, id_s, ks > 0 ? 1u : 0u);
        }
        mma_commit(&s_ready[x]);
      }
      __syncwarp();
    };
    auto issue_o = [&](int x, int st, bool add) {
      if (elect_one()) {
        const uint64_t v = vd + (uint64_t)(st * (SM::TILE >> 4));
#pragma unroll
        for (int ks = 0; ks < BK / 16; ++ks)
          mma_p(tmem + SM::O_COL + x * SM::O_STRIDE, tmem + x * BK + ks * 8, v + (uint64_t)((ks * 2048) >> 4), id_o,
                add || ks > 0 ? 1u : 0u);
      }
      __syncwarp();
    };
    // What the loop goes by is the same in all lanes, and known to be: 2,048 tokens over 34,816 rows of
    // 28/4 heads 615 to 631 us (631 to 645).
    while (ok && __all_sync(0xffffffffu, next_run(A, P, sp, runs, walk, R))) {
      R.s0 = uniform(R.s0);
      R.s1 = uniform(R.s1);
      R.x = uniform(R.x);
      R.two = uniform(R.two) != 0;
      if (!wait(&full[stage], phase)) break;
      for (int x = 0; x < 2; ++x) {
        if (!R.has(x)) continue;
        if (!wait(&q_ready[x], qp >> x)) break;
        qp ^= 1u << x;
        fence_after();
        issue_s(x);
        issued = true;
      }
      if (!ok) break;
      commit(&empty[stage]);
      step();
      for (int x = 0; x < 2; ++x) {                    // the block's last O has been read
        if (!R.has(x)) continue;
        if (!wait(&o_free[x], (of >> x) ^ 1u)) break;
        of ^= 1u << x;
      }
      for (int s = R.s0; ok && s < R.s1; ++s) {
        // In order: P V of a tile reads P before S of the next tile takes its place. While
        // one block's products run, the other's softmax does.
        const int vst = stage;
        const bool more = s + 1 < R.s1;
        if (!wait(&full[vst], phase)) break;
        step();
        for (int x = 0; x < 2; ++x) {
          if (!R.has(x)) continue;
          if (!wait(&p_ready[x], pp >> x)) break;
          pp ^= 1u << x;
          fence_after();
          issue_o(x, vst, s > R.s0);
          if (x == 1 || !R.two) commit(&empty[vst]);
          if (more) {
            if ((x == 0 || !R.two) && !wait(&full[stage], phase)) break;
            issue_s(x);
          } else {
            commit(&o_ready[x]);
          }
        }
        if (!ok) break;
        if (more) {
          commit(&empty[stage]);
          step();
        }
      }
    }
    if (issued) {
      commit(&drain);
      if (!mbar_wait_drain(&drain, 0)) *abort_ = 1;
    }
  } else if (warp >= CONVERT) {
    if constexpr (I8) {
      // Codes to bfloat16, exactly: u = x & 127, x = (128 + u) - (128 or, below zero,
      // 256), eight at a time into the swizzled tile. Thread t has key t's scales.
      const int t = threadIdx.x - CONVERT * 32;
      int stage = 0, rs = 0, tile = 0;
      uint32_t phase = 0, rp = 0;
      bool ok = true;
      while (ok && next_run(A, P, sp, runs, walk, R)) {
        // what is read for the tiles ahead is worked on a tile later: page entries two
        // tiles ahead, scales one
        const int32_t* table = cache_table(J, (size_t)R.U.b * J.Hkv + R.U.h);
        auto entry_of = [&](int s) {
          const int k = s * BK + t;
          return s < R.s1 && k < R.U.keys ? table[k >> J.page_shift] : -1;
        };
        float ks, vs;
        auto read = [&](int s, int entry) {
          const int row = page_row(entry, J.n_pages, J.page_shift, s * BK + t);
          ks = row < 0 ? 0.f : J.ks[row];
          vs = row < 0 ? 0.f : J.vs[row];
        };
        read(R.s0, entry_of(R.s0));
        int entry = entry_of(R.s0 + 1);
        for (int s = R.s0; ok && s < R.s1; ++s) {
#pragma unroll 1
          for (int kv = 0; kv < 2; ++kv) {
            if (!wait_bar(&empty[stage], phase ^ 1u, abort_) || !wait_bar(&rfull[rs], rp, abort_)) {
              ok = false;
              break;
            }
            if (kv == 0) {
              scales[tile % SM::SCALES][0][t] = ks * A.alpha;
              scales[tile % SM::SCALES][1][t] = vs;
              read(s + 1, entry);
              entry = entry_of(s + 2);
            }
            const unsigned char* src = raw + rs * SM::RAW;
            unsigned char* dst = ring + stage * SM::TILE;
#pragma unroll
            for (int i = 0; i < BK * D / 8; i += 8 * 128) {
              uint2 w[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) w[e] = *reinterpret_cast<const uint2*>(src + (i + e * 128 + t) * 8);
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const int n = i + e * 128 + t, key = n / (D / 8), ch = n % (D / 8);
                *reinterpret_cast<uint4*>(dst + (ch / 8) * SM::HALF + key * 128 + ((ch % 8) ^ (key % 8)) * 16) =
                    make_uint4(codes_bf16(__byte_perm(w[e].x, 0, 0x1100)), codes_bf16(__byte_perm(w[e].x, 0, 0x3322)),
                               codes_bf16(__byte_perm(w[e].y, 0, 0x1100)), codes_bf16(__byte_perm(w[e].y, 0, 0x3322)));
              }
            }
            fence_async();
            __syncwarp();
            if (lane == 0) {
              mbar_arrive(&rempty[rs]);
              mbar_arrive(&full[stage]);
            }
            if (++stage == SM::STAGES) { stage = 0; phase ^= 1u; }
            if (++rs == SM::RAWS) { rs = 0; rp ^= 1u; }
          }
          ++tile;
        }
      }
    }
  } else if (warp < 8) {
    const int x = warp / 4, lrow = threadIdx.x % 128;   // block, its row
    const uint32_t lanes = (uint32_t)((warp % 4) * 32) << 16;
    const uint32_t scol = tmem + lanes + x * BK, ocol = tmem + lanes + SM::O_COL + x * SM::O_STRIDE;
    uint32_t sph = 0, oph = 0, vphase = 0;
    int vstage = 0, tile = 0;                            // ring stage of the next tile's K, tiles so far
    bool ok = true;
    while (ok && next_run(A, P, sp, runs, walk, R)) {
      const AttendUnit& U = R.U;
      const int ntiles = R.s1 - R.s0;
      if (!R.has(x)) {
        vstage += 2 * ntiles;
        vphase ^= (vstage / SM::STAGES) & 1;
        vstage %= SM::STAGES;
        tile += ntiles;
        continue;
      }
      const int32_t* table = cache_table(J, (size_t)U.b * J.Hkv + U.h);
      const int least = keys_of(A.causal, U.len, U.n, J.by_r(U.row0));   // keys that every row attends to
      // bit i: the tile's 16-key block i has no page
      auto entry_of = [&](int s) {
        const int t = s * BK + lane * 16;
        return lane < 8 && s < R.s1 && t < U.keys ? table[t >> J.page_shift] : 0;
      };
      int next = entry_of(R.s0);
      const int brow = R.first_row(x) + lrow, row = U.row0 + brow;
      const bool live = brow < U.rows;
      const int tok = J.by_r(row), j = row - tok * J.r;
      {
        // the warp's 32 rows, LPR lanes a row; a row's offset comes from the lane that owns it
        constexpr int LPR = D / 8, QN = I8 ? 8 : LPR;
        const int64_t off = live ? ((int64_t)(J.off[U.b] + tok) * J.stride + (int64_t)(U.h * J.r + j) * D) * 2 : -1;
        unsigned char* dst = sm + x * SM::TILE + warp % 4 * 32 * 128;
        auto offset = [&](int i) { return __shfl_sync(0xffffffffu, off, i * (32 / LPR) + lane / LPR); };
        auto put = [&](int i, const uint4& w) {
          const int r = i * (32 / LPR) + lane / LPR, ch = lane % LPR;
          *reinterpret_cast<uint4*>(dst + (ch / 8) * SM::HALF + r * 128 + ((ch % 8) ^ (r % 8)) * 16) = w;
        };
        if (A.qvec) {
#pragma unroll
          for (int i = 0; i < LPR; i += QN) {          // loads, then their stores
            uint4 w[QN];
#pragma unroll
            for (int e = 0; e < QN; ++e) {
              const int64_t o = offset(i + e);
              w[e] = o >= 0 ? *reinterpret_cast<const uint4*>(A.q + o + lane % LPR * 16) : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int e = 0; e < QN; ++e) put(i + e, w[e]);
          }
        } else {
#pragma unroll 1
          for (int i = 0; i < LPR; ++i) {
            const int64_t o = offset(i);
            put(i, o >= 0 ? load_plain16(A.q + o + lane % LPR * 16, false) : make_uint4(0, 0, 0, 0));
          }
        }
        fence_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(&q_ready[x]);
      }
      // bfloat16 pages: the thread's row. 8-bit pages: rows g + 8i of the warp's 32, with
      // the lanes of a quad sharing them (and their sums).
      constexpr int NR = I8 ? 4 : 1;
      const int g = lane / 4, c = lane % 4;
      float m[NR], l[NR];
      int lim[NR];
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        m[i] = -INFINITY;
        l[i] = 0.f;
        const int r = U.row0 + R.first_row(x) + (I8 ? warp % 4 * 32 + g + 8 * i : lrow);
        lim[i] = r < U.row0 + U.rows ? keys_of(A.causal, U.len, U.n, J.by_r(r)) : 0;
      }
      // a value of the thread's row, of those that the quads hold
      auto of_row = [&](const float* v) {
        if constexpr (!I8) return v[0];
        float got = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float w = __shfl_sync(0xffffffffu, v[I8 ? i : 0], lane % 8 * 4);
          if (lane / 8 == i) got = w;
        }
        return got;
      };
      for (int s = R.s0; s < R.s1; ++s) {
        const uint32_t gone = __ballot_sync(0xffffffffu, next < 0 || next >= J.n_pages);
        next = entry_of(s + 1);
        const int k0 = s * BK;
        const bool special = k0 + BK > least;
        // the tile's V, the stage behind its K; it stays there until P is ready
        int vs = vstage + 1;
        uint32_t vp = vphase;
        if (vs == SM::STAGES) { vs = 0; vp ^= 1u; }
        if (!I8 && special) {
          // Both blocks clean V, each before it reports its P: what one finds clean the
          // other has cleaned, after it set the flag. While S is computed, where the block is
          // known to be in step with the ring; else it waits for S here (and passes below).
          if (!v_before_s(s, R.s0) && !wait_bar(&s_ready[x], sph, abort_)) { ok = false; break; }
          if (!wait_bar(&full[vs], vp, abort_)) { ok = false; break; }
          unsigned char* vt = ring + vs * SM::TILE;
          constexpr int CH = SM::HALVES * 8;             // 16-byte chunks of a row
#pragma unroll 4
          for (int i = max(least - k0, 0) * CH + lrow; i < BK * CH; i += 128) {
            const int key = i / CH, ch = i % CH;
            uint4* p = reinterpret_cast<uint4*>(vt + (ch / 8) * SM::HALF + key * 128 + (ch % 8) * 16);
            const uint4 w = k0 + key < U.keys ? *p : make_uint4(0, 0, 0, 0);
            const bool bad = not_finite2(w.x) || not_finite2(w.y) || not_finite2(w.z) || not_finite2(w.w);
            if (bad) {
              *reinterpret_cast<volatile int*>(&odd_flag) = 1;
              __threadfence_block();
            }
            if (bad || k0 + key >= U.keys) *p = make_uint4(finite2(w.x), finite2(w.y), finite2(w.z), finite2(w.w));
          }
          fence_async();
        }
        if (!wait_bar(&s_ready[x], sph, abort_)) { ok = false; break; }
        sph ^= 1u;
        // 8-bit pages: the tile's scales were written before its V was
        if (I8 && !wait_bar(&full[vs], vp, abort_)) { ok = false; break; }
        fence_after();
        const bool masked = special || gone;
        if (gone && warp % 4 == 0 && lane == 0) set_status(J.status, kStatusBadPage);
        auto hidden = [&](int i, int r) { return k0 + i >= lim[r] || ((gone >> (i / 16)) & 1u); };
        // raises the maxima to `top` (base 2) where some row's passes them by enough
        auto raise = [&](float (&top)[NR]) {
          bool over = false;
#pragma unroll
          for (int i = 0; i < NR; ++i) over |= top[i] > m[i] + kRaise;
          if (!__any_sync(0xffffffffu, over)) return;
          float f[NR];
#pragma unroll
          for (int i = 0; i < NR; ++i) {
            if constexpr (I8) {
              top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 1));
              top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 2));
            }
            const float mn = fmaxf(m[i], top[i]);
            f[i] = m[i] == -INFINITY ? 0.f : fast_exp2(m[i] - mn);
            m[i] = mn;
            l[i] *= f[i];
          }
          if (s == R.s0) return;
          const float fr = of_row(f);
#pragma unroll 1
          for (int i = 0; i < D; i += 16) {
            float o[16];
            tmem_ld16(ocol + i, o);
            tmem_wait_ld16(o);
            uint32_t w[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) w[k] = __float_as_uint(o[k] * fr);
            st16(ocol + i, w);
          }
        };
        if constexpr (!I8) {
          uint64_t sum2[2] = {pk2(0.f, 0.f), pk2(0.f, 0.f)};
          const uint64_t al2 = pk2(A.alpha, A.alpha);
          auto weights = [&](const float* v, float mu, uint32_t* w) {   // 32 columns
            const uint64_t mu2 = pk2(-mu, -mu);
#pragma unroll
            for (int k = 0; k < 16; ++k) {
              float a, b;
              upk2(ffma2(pk2(v[2 * k], v[2 * k + 1]), al2, mu2), a, b);
              a = fast_exp2(a);
              b = fast_exp2(b);
              sum2[k % 2] = fadd2(sum2[k % 2], pk2(a, b));
              w[k] = pack_bf16(a, b);
            }
          };
          if (!masked) {
            // The second half is read again: 128 values and the rest do not fit in 168 registers
            // (spilled, a long chunk took 636 us instead of 616 on one GPU).
            float v[64];
            auto half = [&](int i) {
              ld32(scol + i, v);
              ld32(scol + i + 32, v + 32);
              tmem_wait_ld();
              pin32(v);
              pin32(v + 32);
            };
            half(64);
            float top[1] = {max_of<64>(v)};
            half(0);
            top[0] = fmaxf(top[0], max_of<64>(v)) * A.alpha;
            raise(top);
            const float mu = m[0] == -INFINITY ? 0.f : m[0];
#pragma unroll
            for (int i = 0; i < BK; i += 32) {
              if (i == 64) half(64);
              uint32_t w[16];
              weights(v + i % 64, mu, w);
              st16(scol + i / 2, w);
            }
          } else {
            // few tiles: a short loop, which reads S twice (its code is fetched once a call)
            float v[32], top[1] = {-INFINITY};
            auto load = [&](int i) {
              ld32(scol + i, v);
              tmem_wait_ld();
              pin32(v);
              const uint32_t none = gone >> (i / 16);
              const int n = lim[0] - (k0 + i);
#pragma unroll
              for (int k = 0; k < 32; ++k)
                if (k >= n || ((none >> (k / 16)) & 1u)) v[k] = -INFINITY;
            };
#pragma unroll 1
            for (int i = 0; i < BK; i += 32) {
              load(i);
              top[0] = fmaxf(top[0], max_of<32>(v) * A.alpha);
            }
            raise(top);
            const float mu = m[0] == -INFINITY ? 0.f : m[0];
#pragma unroll 1
            for (int i = 0; i < BK; i += 32) {
              load(i);
              uint32_t w[16];
              weights(v, mu, w);
              st16(scol + i / 2, w);
            }
          }
          float a, b;
          upk2(fadd2(sum2[0], sum2[1]), a, b);
          l[0] += a + b;
        } else {
          // A thread of a quad has a fourth of the columns of four rows, so it reads a fourth of
          // the scales from shared memory (with whole rows, 3 KB a thread and tile, that took
          // longer than the products). S is read twice, for the maxima and for the weights: 512
          // threads leave 128 registers. K's scales hold alpha; V's go with the weights.
          const float2* sk = reinterpret_cast<const float2*>(scales[tile % SM::SCALES][0]) + c;
          const float2* sv = reinterpret_cast<const float2*>(scales[tile % SM::SCALES][1]) + c;
          float v[2][16], top[NR];
          auto load = [&](int i) {
            ld_quads(scol + i, v[0]);
            ld_quads(scol + i + (16u << 16), v[1]);
            tmem_wait_ld();
            pin16(v[0]);
            pin16(v[1]);
          };
          auto pair = [&](int r, int k) { return pk2(v[r / 2][4 * k + 2 * (r % 2)], v[r / 2][4 * k + 2 * (r % 2) + 1]); };
          uint64_t mu2[NR], sum2[NR];
          auto maxima = [&](auto mask) {
#pragma unroll 1
            for (int i = 0; i < BK; i += 32) {
              load(i);
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const float2 f = sk[i / 2 + 4 * k];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                  float a, b;
                  upk2(fmul2(pair(r, k), pk2(f.x, f.y)), a, b);
                  if constexpr (decltype(mask)::value) {
                    if (hidden(i + 8 * k + 2 * c, r)) a = -INFINITY;
                    if (hidden(i + 8 * k + 2 * c + 1, r)) b = -INFINITY;
                  }
                  top[r] = fmaxf(top[r], fmaxf(a, b));
                }
              }
            }
          };
          auto weights = [&](auto mask) {
#pragma unroll 1
            for (int i = 0; i < BK; i += 32) {
              load(i);
              uint32_t w[2][8];
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const float2 f = sk[i / 2 + 4 * k], h = sv[i / 2 + 4 * k];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                  float a, b;
                  upk2(ffma2(pair(r, k), pk2(f.x, f.y), mu2[r]), a, b);
                  a = fast_exp2(a);
                  b = fast_exp2(b);
                  bool ha = false, hb = false;
                  if constexpr (decltype(mask)::value) {
                    ha = hidden(i + 8 * k + 2 * c, r);
                    hb = hidden(i + 8 * k + 2 * c + 1, r);
                    if (ha) a = 0.f;
                    if (hb) b = 0.f;
                  }
                  sum2[r] = fadd2(sum2[r], pk2(a, b));
                  upk2(fmul2(pk2(a, b), pk2(h.x, h.y)), a, b);
                  if (ha) a = 0.f;                     // a scale that no row may see can be a NaN
                  if (hb) b = 0.f;
                  w[r / 2][2 * k + r % 2] = pack_bf16(a, b);
                }
              }
              st_quads(scol + i / 2, w[0]);
              st_quads(scol + i / 2 + (16u << 16), w[1]);
            }
          };
#pragma unroll
          for (int r = 0; r < NR; ++r) top[r] = -INFINITY;
          if (masked) maxima(std::true_type());
          else maxima(std::false_type());
          raise(top);
#pragma unroll
          for (int r = 0; r < NR; ++r) {
            const float mu = m[r] == -INFINITY ? 0.f : m[r];
            mu2[r] = pk2(-mu, -mu);
            sum2[r] = pk2(0.f, 0.f);
          }
          if (masked) weights(std::true_type());
          else weights(std::false_type());
#pragma unroll
          for (int r = 0; r < NR; ++r) {
            float a, b;
            upk2(sum2[r], a, b);
            l[r] += a + b;
          }
        }
        ++tile;
        vstage = vs + 1;
        vphase = vp;
        if (vstage == SM::STAGES) { vstage = 0; vphase ^= 1u; }
        wait_st();
        fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_ready[x]);
      }
      if (!ok || !wait_bar(&o_ready[x], oph, abort_)) { ok = false; break; }
      oph ^= 1u;
      fence_after();
      if constexpr (I8) {
#pragma unroll
        for (int i = 0; i < NR; ++i) {
          l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
          l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
        }
      }
      const float lr = of_row(l), mr = of_row(m);
      const bool fix = !I8 && *reinterpret_cast<volatile int*>(&odd_flag) != 0;
      // sums, of a part of the unit's keys or to be joined with others, or the result
      const bool whole = R.s0 == 0 && R.s1 == U.pieces, sums = !whole || A.part;
      const float f = lr == 0.f ? 0.f : 1.f / lr;
      const int64_t orow = (int64_t)(J.off[U.b] + tok) * J.Hq + U.h * J.r + j;
      const int64_t slot = (int64_t)attend_slot(blockIdx.x, sp.begin, R.before) * P.rows + brow;
      // Rows leave by way of the block's place for Q, which no product reads any more: a
      // thread puts 16-byte chunks of its row there, then 2 * D bytes of a row at a time
      // (all of it, or half of its float32 sums) go out by consecutive lanes.
      constexpr int LPR = D / 8;
      unsigned char* mine = sm + x * SM::TILE + warp % 4 * 32 * 128;   // the warp's rows of Q
      auto chunk = [&](int r, int ch) {
        return reinterpret_cast<uint4*>(mine + (ch / 8) * SM::HALF + r * 128 + ((ch % 8) ^ (r % 8)) * 16);
      };
      float* const po = whole ? A.part : P.po;
      const int64_t to = live ? (whole ? orow : slot) : -1;
      auto flush = [&](int half) {
        __syncwarp();
        const int ch = lane % LPR;
        uint8_t* const base = sums ? reinterpret_cast<uint8_t*>(po) + half * (2 * D) + ch * 16 : A.out + ch * 16;
        const int64_t pitch = sums ? 4 * D : 2 * D;
        const bool vec = sums || A.ovec;
#pragma unroll 1
        for (int i = 0; i < LPR; i += 8) {
          uint4 w[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) w[e] = *chunk((i + e) * (32 / LPR) + lane / LPR, ch);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int64_t t = __shfl_sync(0xffffffffu, to, (i + e) * (32 / LPR) + lane / LPR);
            if (t >= 0) store_row16(base + t * pitch, w[e], vec);
          }
        }
        __syncwarp();
      };
#pragma unroll 1
      for (int i = 0; i < D; i += 32) {
        float o[32];
        ld32(ocol + i, o);
        tmem_wait_ld();
        pin32(o);
        if (fix && live) {
          float t[32];
#pragma unroll
          for (int c = 0; c < 32; ++c) t[c] = o[c];
          add_not_finite<D>(A, R, row, lim[0], mr == -INFINITY ? 0.f : mr, i, t);
#pragma unroll
          for (int c = 0; c < 32; ++c) o[c] = t[c];
        }
        if (!sums) {
          uint32_t w[16];
#pragma unroll
          for (int c = 0; c < 16; ++c) w[c] = lr == 0.f ? 0u : pack_bf16(o[2 * c] * f, o[2 * c + 1] * f);
#pragma unroll
          for (int c = 0; c < 4; ++c)
            *chunk(lane, i / 8 + c) = make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
        } else {
#pragma unroll
          for (int c = 0; c < 8; ++c)
            *chunk(lane, i % (D / 2) / 4 + c) =
                make_uint4(__float_as_uint(o[4 * c]), __float_as_uint(o[4 * c + 1]), __float_as_uint(o[4 * c + 2]),
                           __float_as_uint(o[4 * c + 3]));
          if ((i + 32) % (D / 2) == 0) flush(i >= D / 2);
        }
      }
      if (!sums) flush(0);
      if (live) {
        if (sums) (whole ? A.part_ml : P.pml)[to] = make_float2(mr, lr);
        else if (A.lse) A.lse[orow] = lr == 0.f ? -INFINITY : (mr + log2f(lr)) * 0.6931471805599453f;
      }
      fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&o_free[x]);
    }
  }

  fence_before();
  __syncthreads();
  if (warp == ISSUER) tmem_dealloc(tmem, 512);
  if (threadIdx.x == 0 && abort_flag) set_status(J.status, kStatusTimeout);
}

template <int D, bool I8>
cudaError_t launch(const AttendJob& A, const AttendPlan& P, cudaStream_t st) {
  using SM = ChunkSmem<D, I8>;
  const CacheJob& J = A.c;
  CUtensorMap kmap, vmap;
  const uint64_t rows = (uint64_t)J.n_pages << J.page_shift;
  const uint32_t box = std::min(1 << J.page_shift, BK);
  auto make = [&](CUtensorMap* m, const void* base) {
    return I8 ? make_tmap_u8_rows(m, base, D, rows, box) : make_tmap_bf16_3d(m, base, D, rows, 1, D * 2, rows * D * 2, box);
  };
  if (!make(&kmap, J.kp) || !make(&vmap, J.vp)) return cudaErrorInvalidValue;
  const cudaError_t e =
      cudaFuncSetAttribute(attend_chunk_kernel<D, I8>, cudaFuncAttributeMaxDynamicSharedMemorySize, SM::BYTES);
  if (e != cudaSuccess) return e;
  return launch_kernel(attend_chunk_kernel<D, I8>, dim3(P.workers), SM::NT, SM::BYTES, st, true, 0, kmap, vmap, A, P);
}

}  // namespace

cudaError_t launch_attend_chunk(const AttendJob& A, const AttendPlan& P, cudaStream_t st) {
  if (A.c.i8) return A.c.d == 128 ? launch<128, true>(A, P, st) : launch<64, true>(A, P, st);
  return A.c.d == 128 ? launch<128, false>(A, P, st) : launch<64, false>(A, P, st);
}

}  // namespace mmshift
