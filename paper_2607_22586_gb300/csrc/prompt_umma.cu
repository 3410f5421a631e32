// Attention over whole prompts of bfloat16 rows on the 5th-generation tensor cores
// (tcgen05 + TMA + TMEM).
//
// Tiles of 256 query rows (two blocks of 128, a token's heads next to one another) over tiles of
// 128 keys, S = Q K^T and O += P V as in the chunk kernel (attend_umma.cu): S and P in
// tensor memory, one softmax thread a row. Prompts have many tiles of few keys (a prompt of
// 1000 tokens and seven heads a KV head has 28 tiles, of 5 key tiles on average), so a
// run's start and end must not stop the products:
//   warps 0-7   softmax, a warpgroup a block; at a run's end they take O out;
//   warp 8      TMA producer of K and V tiles, across runs;
//   warp 9      MMA issuer: a block's first S of the next run follows its last P V of this one, so
//               that logits are there when its softmax warps have written O;
//   warps 10-11 load Q of the next blocks into a ring of three places (a block's place is
//               also where its O is put together for whole-line stores).
// K's and V's rows are tokens apart: a tile is one box of 128 rows. Rows behind a prompt's last
// are the next prompt's; masked tiles clean them as the chunk kernel does.
// Every wait is bounded; a role that gives up ends the CTA as score_umma.cu says.
#include <algorithm>

#include "attend_umma.cuh"

namespace mmshift {
namespace {

using namespace umma;

constexpr int PRODUCER = 8, ISSUER = 9, LOADER = 10;   // first warps of the roles

template <int D>
struct PromptSmem {
  static constexpr int NT = 384;
  static constexpr int HALVES = D / 64;
  static constexpr int HALF = BK * 128;              // 64 columns of 128 rows
  static constexpr int TILE = HALVES * HALF;         // a block of Q, a tile of K or V
  static constexpr int QS = 3;                       // blocks of Q
  static constexpr int STAGES = D == 64 ? 8 : 4;
  static_assert(STAGES >= 3, "v_before_s(): a tile's V is three positions behind the K of the tile before");
  static constexpr int BYTES = (QS + STAGES) * TILE + 1024;
  static constexpr uint32_t O_COL = 256, O_STRIDE = D;
};

// Start: everything before in the stream is done, and the next kernel may take its place.
__device__ __forceinline__ void prompt_start() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

__device__ __forceinline__ void copy_async16(uint32_t dst, const void* src, bool in) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// The part of a row's sums that comes from values that are not finite, of columns
// [d0, d0 + 32): added with the row's weights, key by key. Rare, so slow.
template <int D>
static __device__ __noinline__ void add_not_finite(const AttendJob& A, const Run& R, int row, int lim, float m, int d0,
                                                   float* o) {
  const CacheJob& J = A.c;
  const int tok = J.by_r(row), j = row - tok * J.r;
  const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(A.q) +
                           (size_t)(J.off[R.U.b] + tok) * J.stride + (size_t)(R.U.h * J.r + j) * D;
  const int first = keys_of(A.causal, R.U.len, R.U.n, J.by_r(R.U.row0));
  for (int t = max(R.s0 * BK, first / BK * BK); t < min(R.s1 * BK, lim); ++t) {
    const size_t at = (size_t)(J.off[R.U.b] + t) * A.kv_stride + (size_t)R.U.h * D;
    const __nv_bfloat16* v = reinterpret_cast<const __nv_bfloat16*>(J.vp) + at + d0;
    bool any = false;
    for (int i = 0; i < 32; ++i) any |= !isfinite(to_f32(v[i]));
    if (!any) continue;
    const __nv_bfloat16* k = reinterpret_cast<const __nv_bfloat16*>(J.kp) + at;
    float s = 0.f;
    for (int i = 0; i < D; ++i) s = fmaf(to_f32(q[i]), to_f32(k[i]), s);
    const float p = fast_exp2(fmaf(s, A.alpha, -m));
    for (int i = 0; i < 32; ++i) {
      const float x = to_f32(v[i]);
      if (!isfinite(x)) o[i] += p * x;
    }
  }
}

template <int D>
__global__ void __launch_bounds__(PromptSmem<D>::NT, 1) attend_prompt_kernel(const __grid_constant__ CUtensorMap kmap,
                                                              const __grid_constant__ CUtensorMap vmap,
                                                              const __grid_constant__ AttendJob A,
                                                              const __grid_constant__ AttendPlan P) {
  using SM = PromptSmem<D>;
  constexpr int NT = SM::NT;
  extern __shared__ unsigned char smraw[];
  unsigned char* sm =
      reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smraw) + 1023) & ~uintptr_t(1023));
  unsigned char* ring = sm + SM::QS * SM::TILE;
  // Every wait is for the next fill of its stage that the waiting warp does not know to be complete,
  // or for one that is: producer, loaders and issuer pass all positions of their rings, the softmax
  // blocks see v_before_s().
  __shared__ uint64_t full[SM::STAGES], empty[SM::STAGES], q_full[SM::QS], q_empty[SM::QS];
  __shared__ uint64_t s_ready[2], o_ready[2], o_free[2], p_ready[2], drain;
  __shared__ uint32_t tbase;
  __shared__ int abort_flag, odd_flag;
  __shared__ AttendScan<NT, 1> scan;
  __shared__ RunList runs;
  volatile int* abort_ = &abort_flag;
  const CacheJob& J = A.c;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;

  if (threadIdx.x == 0) {
    abort_flag = odd_flag = 0;
    for (int s = 0; s < SM::STAGES; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int s = 0; s < SM::QS; ++s) {
      mbar_init(&q_full[s], 2);      // both loaders
      mbar_init(&q_empty[s], 4);     // a warpgroup's warps
    }
    for (int i = 0; i < 2; ++i) {
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
  prompt_start();
  const AttendSpan sp = attend_span(A, P, &scan);
  if (warp == 0) list_runs(A, P, sp, lane, &runs);
  __syncthreads();
  Walk walk = {0, 0, 0, 0};
  Run R;
  // Blocks of Q are used in the order of the runs, a run's first block first: use n lies in
  // place n % QS.
  int use = 0;
  if (warp == PRODUCER) {
    int stage = 0;
    uint32_t phase = 0;
    ArmedStages armed;
    bool ok = true;
    while (ok && next_run(A, P, sp, runs, walk, R)) {
      const int row0 = J.off[R.U.b], col0 = R.U.h * D;
      for (int s = R.s0; ok && s < R.s1; ++s) {
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          if (!wait_bar(&empty[stage], phase ^ 1u, abort_)) { ok = false; break; }
          if (lane == 0) {
            mbar_expect_tx(&full[stage], SM::TILE);
#pragma unroll
            for (int c = 0; c < SM::HALVES; ++c)
              tma_load_3d(ring + stage * SM::TILE + c * SM::HALF, kv ? &vmap : &kmap, &full[stage], col0 + c * 64,
                          row0 + s * BK, 0);
          }
          armed.arm(stage, phase);
          __syncwarp();
          if (++stage == SM::STAGES) { stage = 0; phase ^= 1u; }
        }
      }
    }
    if (!armed.drain(full)) *abort_ = 1;
  } else if (warp == ISSUER) {
    const uint32_t id_s = idesc_bf16_f32(BQ, BK), id_o = idesc_bf16_f32(BQ, D) | (1u << 16);   // V: MN-major
    const uint64_t qd = sdesc_k_sw128(smem_u32(sm)), kd = sdesc_k_sw128(smem_u32(ring));
    const uint64_t vd = sdesc_mn_sw128(smem_u32(ring), SM::HALF);
    int stage = 0;
    uint32_t phase = 0, pp = 0, of = 0;                // of the ring; bit i: of block i's barriers
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
    // S of block x, whose Q is use n, with the K tile of the stage
    auto issue_s = [&](int x, int n) {
      if (elect_one()) {
        const uint64_t k = kd + (uint64_t)(stage * (SM::TILE >> 4)), q = qd + (uint64_t)(n % SM::QS * (SM::TILE >> 4));
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          const uint64_t o = (uint64_t)(((ks / 4) * SM::HALF + (ks % 4) * 32) >> 4);
          mma_bf16(tmem + x * BK, q + o, k + o, id_s, ks > 0 ? 1u : 0u);
        }
        mma_commit(&s_ready[x]);
      }
      __syncwarp();
      issued = true;
    };
    // the first S of a run
    auto first_s = [&](int x, int n) {
      if (!wait(&q_full[n % SM::QS], (uint32_t)(n / SM::QS))) return;
      fence_after();
      issue_s(x, n);
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
    bool have = next_run(A, P, sp, runs, walk, R);
    if (have && wait(&full[stage], phase)) {
      for (int x = 0; ok && x < 2; ++x)
        if (R.has(x)) first_s(x, use + (R.two ? x : 0));
      commit(&empty[stage]);
      step();
    }
    while (ok && have) {
      Run N;
      const bool next = next_run(A, P, sp, runs, walk, N);
      const int use_next = use + (R.two ? 2 : 1);
      for (int s = R.s0; ok && s < R.s1; ++s) {
        // In order: P V of a tile reads P before S of the next tile (of this run or the next) takes
        // its place. While one block's products run, the other's softmax does.
        const int vst = stage;
        const bool last = s + 1 == R.s1, more = !last || next;
        bool k_there = false;
        if (!wait(&full[vst], phase)) break;
        step();
        for (int x = 0; ok && x < 2; ++x) {
          if (R.has(x)) {
            if (s == R.s0) {                           // the block's last O has been read
              if (!wait(&o_free[x], (of >> x) ^ 1u)) break;
              of ^= 1u << x;
            }
            if (!wait(&p_ready[x], pp >> x)) break;
            pp ^= 1u << x;
            fence_after();
            issue_o(x, vst, s > R.s0);
            if (last) commit(&o_ready[x]);
            if (x == 1 || !R.two) commit(&empty[vst]);
          }
          if (last ? next && N.has(x) : R.has(x)) {
            if (!k_there && !wait(&full[stage], phase)) break;
            k_there = true;
            if (last) first_s(x, use_next + (N.two ? x : 0));
            else issue_s(x, use + (R.two ? x : 0));
          }
        }
        if (!ok) break;
        if (more) {
          commit(&empty[stage]);
          step();
        }
      }
      use = use_next;
      R = N;
      have = next;
    }
    if (issued) {
      commit(&drain);
      if (!mbar_wait_drain(&drain, 0)) *abort_ = 1;
    }
  } else if (warp >= LOADER) {
    // Rows [64 w, 64 w + 64) of each block, LPR lanes a row, 16 bytes a lane.
    constexpr int LPR = D / 8, PER = 32 / LPR;
    const int r0 = (warp - LOADER) * 64 + lane / LPR, ch = lane % LPR;
    bool ok = true;
    while (ok && next_run(A, P, sp, runs, walk, R)) {
      const AttendUnit& U = R.U;
      for (int x = 0; ok && x < 2; ++x) {
        if (!R.has(x)) continue;
        const int place = use % SM::QS;
        if (!wait_bar(&q_empty[place], (uint32_t)(use / SM::QS) & 1u ^ 1u, abort_)) { ok = false; break; }
        const uint32_t dst = smem_u32(sm + place * SM::TILE + (ch / 8) * SM::HALF);
#pragma unroll 4
        for (int i = 0; i < 64; i += PER) {
          const int r = r0 + i, brow = R.first_row(x) + r, row = U.row0 + brow;
          const bool in = brow < U.rows;
          const int tok = J.by_r(row), j = row - tok * J.r;
          const uint8_t* src =
              A.q + (in ? ((int64_t)(J.off[U.b] + tok) * J.stride + (int64_t)(U.h * J.r + j) * D) * 2 + ch * 16 : 0);
          const uint32_t to = dst + r * 128 + ((ch % 8) ^ (r % 8)) * 16;
          if (A.qvec) {
            copy_async16(to, src, in);
          } else {
            const uint4 w = in ? load_plain16(src, false) : make_uint4(0, 0, 0, 0);
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(w.x), "r"(w.y), "r"(w.z), "r"(w.w)
                         : "memory");
          }
        }
        copies_wait();
        fence_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(&q_full[place]);
        ++use;
      }
    }
  } else {
    const int x = warp / 4, lrow = threadIdx.x % 128;   // block, its row
    const uint32_t lanes = (uint32_t)((warp % 4) * 32) << 16;
    const uint32_t scol = tmem + lanes + x * BK, ocol = tmem + lanes + SM::O_COL + x * SM::O_STRIDE;
    uint32_t sph = 0, oph = 0, vphase = 0;
    int vstage = 0;                                      // ring stage of the next tile's K
    bool ok = true;
    for (; ok && next_run(A, P, sp, runs, walk, R); use += R.two ? 2 : 1) {
      const AttendUnit& U = R.U;
      const int ntiles = R.s1 - R.s0;
      if (!R.has(x)) {
        vstage += 2 * ntiles;
        vphase ^= (vstage / SM::STAGES) & 1;
        vstage %= SM::STAGES;
        continue;
      }
      const int place = (use + (R.two ? x : 0)) % SM::QS;
      const int least = keys_of(A.causal, U.len, U.n, J.by_r(U.row0));   // keys that every row attends to
      const int brow = R.first_row(x) + lrow, row = U.row0 + brow;
      const bool live = brow < U.rows;
      const int tok = J.by_r(row), j = row - tok * J.r;
      const int lim = live ? keys_of(A.causal, U.len, U.n, tok) : 0;
      float m = -INFINITY, l = 0.f;
      for (int s = R.s0; s < R.s1; ++s) {
        const int k0 = s * BK;
        const bool masked = k0 + BK > least;
        // the tile's V, the stage behind its K; it stays there until P is ready
        int vs = vstage + 1;
        uint32_t vp = vphase;
        if (vs == SM::STAGES) { vs = 0; vp ^= 1u; }
        if (masked) {
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
        fence_after();
        // raises the maximum to `top` (base 2) where some row's passes it by enough
        auto raise = [&](float top) {
          if (!__any_sync(0xffffffffu, top > m + kRaise)) return;
          const float mn = fmaxf(m, top), f = m == -INFINITY ? 0.f : fast_exp2(m - mn);
          m = mn;
          l *= f;
          if (s == R.s0) return;
#pragma unroll 1
          for (int i = 0; i < D; i += 16) {
            float o[16];
            tmem_ld16(ocol + i, o);
            tmem_wait_ld16(o);
            uint32_t w[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) w[k] = __float_as_uint(o[k] * f);
            st16(ocol + i, w);
          }
        };
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
          // The second half is read again: 128 values and the rest do not fit in 168 registers.
          float v[64];
          auto half = [&](int i) {
            ld32(scol + i, v);
            ld32(scol + i + 32, v + 32);
            tmem_wait_ld();
            pin32(v);
            pin32(v + 32);
          };
          half(64);
          float top = max_of<64>(v);
          half(0);
          top = fmaxf(top, max_of<64>(v)) * A.alpha;
          raise(top);
          const float mu = m == -INFINITY ? 0.f : m;
#pragma unroll
          for (int i = 0; i < BK; i += 32) {
            if (i == 64) half(64);
            uint32_t w[16];
            weights(v + i % 64, mu, w);
            st16(scol + i / 2, w);
          }
        } else {
          float v[32], top = -INFINITY;
          auto load = [&](int i) {
            ld32(scol + i, v);
            tmem_wait_ld();
            pin32(v);
            const int n = lim - (k0 + i);
#pragma unroll
            for (int k = 0; k < 32; ++k)
              if (k >= n) v[k] = -INFINITY;
          };
#pragma unroll 1
          for (int i = 0; i < BK; i += 32) {
            load(i);
            top = fmaxf(top, max_of<32>(v) * A.alpha);
          }
          raise(top);
          const float mu = m == -INFINITY ? 0.f : m;
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
        l += a + b;
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
      const bool fix = *reinterpret_cast<volatile int*>(&odd_flag) != 0;
      const bool whole = R.s0 == 0 && R.s1 == U.pieces;
      const float f = l == 0.f ? 0.f : 1.f / l;
      const int64_t orow = (int64_t)(J.off[U.b] + tok) * J.Hq + U.h * J.r + j;
      const int64_t slot = (int64_t)attend_slot(blockIdx.x, sp.begin, R.before) * P.rows + brow;
      // Rows leave by way of the block's place for Q, which no product reads any more: a
      // thread puts 16-byte chunks of its row there, then 2 * D bytes of a row at a time
      // (all of it, or half of its float32 sums) go out by consecutive lanes.
      constexpr int LPR = D / 8;
      unsigned char* mine = sm + place * SM::TILE + warp % 4 * 32 * 128;   // the warp's rows of Q
      auto chunk = [&](int r, int ch) {
        return reinterpret_cast<uint4*>(mine + (ch / 8) * SM::HALF + r * 128 + ((ch % 8) ^ (r % 8)) * 16);
      };
      const int64_t to = live ? (whole ? orow : slot) : -1;
      auto flush = [&](int half) {
        __syncwarp();
        const int ch = lane % LPR;
        uint8_t* const base = whole ? A.out + ch * 16 : reinterpret_cast<uint8_t*>(P.po) + half * (2 * D) + ch * 16;
        const int64_t pitch = whole ? 2 * D : 4 * D;
        const bool vec = !whole || A.ovec;
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
        if (i + 32 == D) {                               // the block's next products may take O's place
          fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&o_free[x]);
        }
        if (fix && live) {
          float t[32];
#pragma unroll
          for (int c = 0; c < 32; ++c) t[c] = o[c];
          add_not_finite<D>(A, R, row, lim, m == -INFINITY ? 0.f : m, i, t);
#pragma unroll
          for (int c = 0; c < 32; ++c) o[c] = t[c];
        }
        if (whole) {
          uint32_t w[16];
#pragma unroll
          for (int c = 0; c < 16; ++c) w[c] = l == 0.f ? 0u : pack_bf16(o[2 * c] * f, o[2 * c + 1] * f);
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
      if (whole) flush(0);
      if (lane == 0) mbar_arrive(&q_empty[place]);       // behind flush's barrier
      if (live) {
        if (!whole) P.pml[slot] = make_float2(m, l);
        else if (A.lse) A.lse[orow] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
      }
    }
  }

  fence_before();
  __syncthreads();
  if (warp == ISSUER) tmem_dealloc(tmem, 512);
  if (threadIdx.x == 0 && abort_flag) set_status(J.status, kStatusTimeout);
}

template <int D>
cudaError_t launch(const AttendJob& A, const AttendPlan& P, cudaStream_t st) {
  using SM = PromptSmem<D>;
  const CacheJob& J = A.c;
  CUtensorMap kmap, vmap;
  const uint64_t rows = J.off[J.B], cols = (uint64_t)J.Hkv * D, pitch = A.kv_stride * 2;
  if (!make_tmap_bf16_3d(&kmap, J.kp, cols, rows, 1, pitch, rows * pitch, BK) ||
      !make_tmap_bf16_3d(&vmap, J.vp, cols, rows, 1, pitch, rows * pitch, BK))
    return cudaErrorInvalidValue;
  const cudaError_t e =
      cudaFuncSetAttribute(attend_prompt_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, SM::BYTES);
  if (e != cudaSuccess) return e;
  return launch_kernel(attend_prompt_kernel<D>, dim3(P.workers), SM::NT, SM::BYTES, st, true, 0, kmap, vmap, A, P);
}

}  // namespace

cudaError_t launch_prompt_umma(const AttendJob& A, const AttendPlan& P, cudaStream_t st) {
  return A.c.d == 128 ? launch<128>(A, P, st) : launch<64>(A, P, st);
}

}  // namespace mmshift
