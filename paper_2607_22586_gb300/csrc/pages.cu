// The cache's pages: who holds them, which are free, and rows moved between them
// (mmshift_cache_reserve, _fork, _free, _compact).
//
// A page's count says how many sequences hold it; a page without a holder is free.
// Nothing else is kept (no list of free pages), so the state cannot disagree with itself,
// and which page a sequence gets follows from the counts alone: free pages go out by
// number, lowest first, in the order of the sequences and of their positions. Counting
// and taking is one CTA's work, or a cluster's: eight CTAs add up what their sequences need and
// which of their pages are free, and exchange sums through distributed shared memory.
// The counts of 200,000 pages are 0.8 MB, which the cluster reads from the L2 twice, and only
// where some sequence needs a page.
#include <algorithm>
#include <cstring>

#include "cache.cuh"
#include "umma.cuh"

namespace mmshift {
mmshift_status noalloc_cuda_fail(cudaError_t e);

namespace {

using umma::cluster_rank;
using umma::cluster_sync;
using umma::ld_cluster_int;
using umma::mapa;
using umma::smem_u32;

constexpr int kCluster = 8, kTake = 1024;

// A page taken: what it stands in for, and how many of that page's rows it is to have.
struct PageJob {
  int32_t from, to, rows, unused;      // from: -1 where there was no page
};

struct PagesJob {
  CacheJob c;
  int32_t* table;
  int32_t* refs;
  const int32_t* count;                // compact: kept rows, or null
  int32_t* taken;                      // number of jobs
  int32_t* list;                       // [most] free pages, lowest first
  PageJob* jobs;                       // [most]
  int32_t most;
  int32_t vec;                         // refs allow 16-byte loads
  int32_t group, once;                 // lanes of a sequence; they have all its pages at one go
  int32_t* old_table;                  // compact: the table and lengths before
  int32_t* old_lens;
};

// Start: everything before in the stream is done, and the next kernel may take its place.
__device__ __forceinline__ void pages_start() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

__device__ __forceinline__ bool is_page(const CacheJob& J, int32_t e) { return e >= 0 && e < J.n_pages; }

// The positions [start, stop) that a call writes in sequence u.
struct Written {
  int start, stop;
};
template <bool COMPACT>
__device__ __forceinline__ Written written(const PagesJob& G, int u) {
  const CacheJob& J = G.c;
  const int b = J.by_heads(u) % J.B, n = J.off[b + 1] - J.off[b];
  if (!n) return Written{0, 0};
  if constexpr (COMPACT) {
    const int held = cache_len(J, u);
    return Written{0, min(held, G.count ? min(max(G.count[u], 0), n) : n)};
  } else {
    const int end = append_end(J.lens[u], J.cap);
    return Written{max(end - n, 0), min(end, J.cap)};
  }
}

// The barrier of the kernel's CTAs, and the sums over all their threads before one, and over all.
template <int C>
__device__ __forceinline__ void sync_all() {
  if constexpr (C == 1) __syncthreads();
  else cluster_sync();
}
struct ClusterScan {
  int32_t warp[kTake / 32];
  int32_t total;
};
template <int C>
__device__ __forceinline__ void cluster_scan(ClusterScan& s, int x, int& before, int& all) {
  const int lane = threadIdx.x % 32, w = threadIdx.x / 32;
  int sum = x;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, sum, d);
    if (lane >= d) sum += y;
  }
  if (lane == 31) s.warp[w] = sum;
  __syncthreads();
  if (w == 0) {
    int t = s.warp[lane];
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, t, d);
      if (lane >= d) t += y;
    }
    s.warp[lane] = t;
    if (lane == 31) s.total = t;
  }
  sync_all<C>();
  before = sum - x + (w ? s.warp[w - 1] : 0);
  if constexpr (C == 1) {
    all = s.total;
  } else {
    all = 0;
    const int rank = cluster_rank();
#pragma unroll
    for (int r = 0; r < C; ++r) {
      const int t = ld_cluster_int(mapa(smem_u32(&s.total), r));
      if (r < rank) before += t;
      all += t;
    }
  }
}

// Every sequence's missing and shared pages among those that the call writes are replaced
// by free ones. COMPACT: of the first pages, which will hold the kept rows; the pages behind them
// are given back, and the lengths set.
template <bool COMPACT, int C>
__global__ void __launch_bounds__(kTake) take_pages_kernel(const __grid_constant__ PagesJob G) {
  __shared__ ClusterScan scan[2];
  const CacheJob& J = G.c;
  const int rank = C == 1 ? 0 : cluster_rank(), tid = rank * kTake + threadIdx.x, lane = threadIdx.x % 32;
  pages_start();
  // A sequence's lanes take its pages in turn; a group of lanes has a run of sequences.
  const int U = J.L * J.B * J.Hkv, groups = C * kTake / G.group, per = (U + groups - 1) / groups;
  const int g = tid / G.group, part = tid % G.group;
  const unsigned mine = (G.group == 32 ? 0xffffffffu : (1u << G.group) - 1u) << (lane / G.group * G.group);
  const int64_t u_first = (int64_t)g * per;
  const int u0 = (int)min(u_first, (int64_t)U), u1 = (int)min(u_first + per, (int64_t)U);
  const int page = 1 << J.page_shift;

  // Walks the pages that the group's sequences write: f(sequence, page's place in it, its entry
  // or -1, whether it has to be replaced, how many before it of the walk have to be). Warps stay
  // together: lanes that vote in groups of their own would go on one by one. Four pages a lane are
  // asked for at once; a walk of no more than those (`once`) is not read again.
  constexpr int K = 4;
  const bool once = per == 1 && G.once;
  Written w = {0, 0};
  int32_t e[K];
  bool need[K];
  auto walk = [&](bool read, auto f) {
    int n = 0;
    for (int k = 0; k < per; ++k) {
      const int u = u0 + k;
      if (read) w = u < u1 ? written<COMPACT>(G, u) : Written{0, 0};
      const int first = w.start >> J.page_shift, end = w.start < w.stop ? (w.stop + page - 1) >> J.page_shift : first;
      for (int i0 = first + part; __any_sync(0xffffffffu, i0 - part < end); i0 += K * G.group) {
        if (read) {
#pragma unroll
          for (int x = 0; x < K; ++x) {
            const int i = i0 + x * G.group;
            e[x] = i < end ? G.table[(size_t)u * J.max_pages + i] : -1;
            if (!is_page(J, e[x])) e[x] = -1;
          }
#pragma unroll
          for (int x = 0; x < K; ++x) need[x] = i0 + x * G.group < end && (e[x] < 0 || G.refs[e[x]] > 1);
        }
#pragma unroll
        for (int x = 0; x < K; ++x) {
          const unsigned all = __ballot_sync(0xffffffffu, need[x]) & mine;
          f(u, w, i0 + x * G.group, e[x], need[x], n + __popc(all & ((1u << lane) - 1u)));
          n += __popc(all);
        }
      }
    }
    return n;
  };
  const int warp = tid / 32, warps = C * kTake / 32;
  if constexpr (COMPACT) {                             // what is moved is found by way of the table before
    for (int64_t u = warp; u < U; u += warps) {
      const int b = J.by_heads((int)u) % J.B;
      if (J.off[b + 1] == J.off[b]) continue;
      const int held = cache_len(J, u), pages = (held + page - 1) >> J.page_shift;
#pragma unroll 4
      for (int i = lane; i < pages; i += 32) G.old_table[u * J.max_pages + i] = G.table[u * J.max_pages + i];
      if (lane == 0) G.old_lens[u] = held;
    }
  }
  const int needed = walk(true, [](int, Written, int, int32_t, bool, int) {});
  int before, all;
  cluster_scan<C>(scan[0], part ? 0 : needed, before, all);
  before = __shfl_sync(0xffffffffu, before, lane / G.group * G.group);
  if (all) {
    // Warps have a run of pages each, and count them before they number the free ones; a lane has
    // four in a row.
    const int run = ((J.n_pages + warps - 1) / warps + 127) / 128 * 128;
    const int64_t p_first = (int64_t)warp * run;
    const int p0 = (int)min(p_first, (int64_t)J.n_pages), p1 = (int)min(p_first + run, (int64_t)J.n_pages);
    auto free_of = [&](int p) {                        // bit i: page p + i is free
      int32_t r[4] = {1, 1, 1, 1};
      if (G.vec && p + 4 <= p1) {
        const int4 x = *reinterpret_cast<const int4*>(G.refs + p);
        r[0] = x.x, r[1] = x.y, r[2] = x.z, r[3] = x.w;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (p + i < p1) r[i] = G.refs[p + i];
      }
      return (r[0] == 0) | (r[1] == 0) << 1 | (r[2] == 0) << 2 | (r[3] == 0) << 3;
    };
    int free = 0;
#pragma unroll 8
    for (int p = p0 + 4 * lane; p < p1; p += 128) free += __popc(free_of(p));
#pragma unroll
    for (int s = 16; s; s >>= 1) free += __shfl_xor_sync(0xffffffffu, free, s);
    int at, found;
    cluster_scan<C>(scan[1], lane ? 0 : free, at, found);
    at = __shfl_sync(0xffffffffu, at, 0);
    const int end = min(all, G.most);
    for (int p = p0; p < p1 && at < end; p += 128) {
      const unsigned is = free_of(p + 4 * lane);
      int before_lane = 0, here = 0;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const unsigned lanes = __ballot_sync(0xffffffffu, is >> x & 1u);
        before_lane += __popc(lanes & ((1u << lane) - 1u));
        here += __popc(lanes);
      }
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int k = at + before_lane + __popc(is & ((1u << x) - 1u));
        if ((is >> x & 1u) && k < end) G.list[k] = p + 4 * lane + x;
      }
      at += here;
    }
    sync_all<C>();                                     // the list is there, and all counts have been read
    walk(!once, [&](int u, Written w, int i, int32_t e, bool need, int n) {
      if (!need) return;
      const int k = before + n;
      const int32_t to = k < min(found, G.most) ? G.list[k] : -1;
      if (to < 0) set_status(J.status, kStatusNoPage);
      else G.refs[to] = 1;
      if (k < G.most) {
        const int rows = min(max(w.start - (i << J.page_shift), 0), page);
        G.jobs[k] = PageJob{e, to, COMPACT || e < 0 || to < 0 ? 0 : rows, 0};
      }
      // the page of an entry behind the last job is noted in the entry: -2 - e, below -1
      G.table[(size_t)u * J.max_pages + i] = k < G.most || e < 0 ? to : -2 - e;
    });
    sync_all<C>();                                     // the counts are no longer asked for
    for (int k = tid; k < min(all, G.most); k += C * kTake) {
      const int32_t e = G.jobs[k].from;
      if (e >= 0) atomicSub(G.refs + e, 1);
    }
    // More wanted than the pool has pages: what had no job is given up by who noted it. Entries in what is
    // written are pages, -1 or notes by now; lengths that other warps have set give the same range.
    for (int k = 0; all > G.most && k < per && u0 + k < u1; ++k) {
      const Written x = written<COMPACT>(G, u0 + k);
      const int end = x.start < x.stop ? (x.stop + page - 1) >> J.page_shift : 0;
      for (int i = (x.start >> J.page_shift) + part; i < end; i += G.group) {
        int32_t* const at = G.table + (size_t)(u0 + k) * J.max_pages + i;
        const int32_t e = *at;
        if (e > -2) continue;
        atomicSub(G.refs + (-2 - e), 1);
        *at = -1;
      }
    }
  }
  if (tid == 0) *G.taken = min(all, G.most);
  if constexpr (COMPACT) {
    for (int64_t u = warp; u < U; u += warps) {
      const int b = J.by_heads((int)u) % J.B;
      if (J.off[b + 1] == J.off[b]) continue;
      const int kept = written<true>(G, (int)u).stop;
#pragma unroll 4
      for (int i = ((kept + page - 1) >> J.page_shift) + lane; i < J.max_pages; i += 32) {
        const int32_t e = G.table[u * J.max_pages + i];
        if (is_page(J, e)) atomicSub(G.refs + e, 1);
        G.table[u * J.max_pages + i] = -1;
      }
      __syncwarp();
      if (lane == 0) J.lens[u] = kept;
    }
  }
  if constexpr (C > 1) cluster_sync();                 // no CTA leaves while its sums are read
}

// The rows that were there already, into the pages that replace shared ones: a block a
// page in turn, 16 bytes a thread.
__global__ void __launch_bounds__(256) copy_pages_kernel(const __grid_constant__ PagesJob G) {
  const CacheJob& J = G.c;
  pages_start();
  const int row = J.i8 ? J.d : J.bf16 ? 2 * J.d : 4 * J.d, n = *G.taken;
  const int64_t bytes = (int64_t)row << J.page_shift;
  for (int k = blockIdx.x; k < n; k += gridDim.x) {
    const PageJob x = G.jobs[k];
    const int chunks = x.rows * row / 16;
#pragma unroll 4
    for (int i = threadIdx.x; i < 2 * chunks; i += 256) {
      const bool v = i >= chunks;
      uint8_t* const pool = v ? J.vp : J.kp;
      const int64_t at = (int64_t)(v ? i - chunks : i) * 16;
      *reinterpret_cast<uint4*>(pool + x.to * bytes + at) = *reinterpret_cast<const uint4*>(pool + x.from * bytes + at);
    }
    if (J.i8) {
      for (int i = threadIdx.x; i < 2 * x.rows; i += 256) {
        const bool v = i >= x.rows;
        float* const pool = v ? J.vs : J.ks;
        const int at = v ? i - x.rows : i;
        pool[((int64_t)x.to << J.page_shift) + at] = pool[((int64_t)x.from << J.page_shift) + at];
      }
    }
  }
}

// Sequences given back (src < 0) or made to hold another request's pages: a warp a sequence.
struct HoldJob {
  CacheJob c;
  int32_t* table;
  int32_t* refs;
  int32_t n;
  int32_t src[MMSHIFT_MAX_BATCH], dst[MMSHIFT_MAX_BATCH];
};

__global__ void __launch_bounds__(256) hold_pages_kernel(const __grid_constant__ HoldJob G) {
  const CacheJob& J = G.c;
  pages_start();
  const int lane = threadIdx.x % 32, i = blockIdx.x * 8 + threadIdx.x / 32;   // (pair, head)
  if (i >= G.n * J.Hkv) return;
  const int pair = J.by_heads(i), h = i - pair * J.Hkv, l = blockIdx.y;
  const size_t dst = ((size_t)l * J.B + G.dst[pair]) * J.Hkv + h;
  const size_t src = ((size_t)l * J.B + max(G.src[pair], 0)) * J.Hkv + h;
  const int len = G.src[pair] < 0 ? 0 : cache_len(J, src);
  const int pages = (len + (1 << J.page_shift) - 1) >> J.page_shift;
#pragma unroll 2
  for (int e = lane; e < J.max_pages; e += 32) {
    const int32_t was = G.table[dst * J.max_pages + e], is = e < pages ? G.table[src * J.max_pages + e] : -1;
    if (was == is) continue;
    if (is_page(J, was)) atomicSub(G.refs + was, 1);
    if (is_page(J, is)) atomicAdd(G.refs + is, 1);
    G.table[dst * J.max_pages + e] = is;
  }
  if (lane == 0) J.lens[dst] = len;
}

// Kept rows to the front of their sequences, K or V of a sequence by a cluster of CTAs (or
// one). Row i comes from position idx[i] >= i, so it can be moved in place: rows go in
// chunks, and a chunk is written once it has been read as a whole; what later chunks read lies
// behind it. While a chunk is written the next one is on its way, and the places of the
// one after it are looked up.
constexpr int kMoveThreads = 256;

template <int ROWB, bool I8>
struct MoveShape {
  static constexpr int LANES = ROWB / 16, HELD = 8;                  // lanes of a row; 16-byte pieces a thread
  static constexpr int ROWS = kMoveThreads / LANES * HELD;           // of a CTA's chunk
};

template <int ROWB, bool I8>
__global__ void __launch_bounds__(kMoveThreads) move_rows_kernel(const __grid_constant__ PagesJob G,
                                                                 const int32_t* idx, int ctas) {
  using S = MoveShape<ROWB, I8>;
  constexpr int PER = (S::ROWS + kMoveThreads - 1) / kMoveThreads;
  __shared__ int32_t from[3][S::ROWS], to[3][S::ROWS];
  const CacheJob& J = G.c;
  pages_start();
  const int rank = ctas > 1 ? cluster_rank() : 0;
  const int unit = blockIdx.x / ctas, l = blockIdx.z;
  // the requests that have rows, packed
  int b = 0, skip = J.by_heads(unit);
  const int h = unit - skip * J.Hkv;
  while (J.off[b + 1] == J.off[b] || skip-- > 0) ++b;
  const size_t u = ((size_t)l * J.B + b) * J.Hkv + h;
  const int kept = cache_len(J, u), held = G.old_lens[u];
  uint8_t* const pool = blockIdx.y ? J.vp : J.kp;
  float* const scales = blockIdx.y ? J.vs : J.ks;
  const int32_t* const sel = idx + ((size_t)l * J.off[J.B] + J.off[b]) * J.Hkv + h;
  const int tid = threadIdx.x, part = tid % S::LANES, step = ctas * S::ROWS;
  // from: the pool's row, -1 for one of zeros, -2 for none to write
  auto look_up = [&](int c) {
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int r = k * kMoveThreads + tid, i = c * step + rank * S::ROWS + r;
      if (r >= S::ROWS) continue;
      int32_t f = -2, t = -1;
      if (i < kept) {
        t = page_row(G.table[u * J.max_pages + (i >> J.page_shift)], J.n_pages, J.page_shift, i);
        const int p = sel[(size_t)i * J.Hkv];
        f = -1;
        if (p >= i && p < held) {
          f = page_row(G.old_table[u * J.max_pages + (p >> J.page_shift)], J.n_pages, J.page_shift, p);
          if (f < 0) set_status(J.status, kStatusBadPage);
        } else {
          set_status(J.status, kStatusBadIndex);
        }
        if (t < 0) f = -2;
        if (f == t) f = -2;                            // it stays where it is
      }
      from[c % 3][r] = f;
      to[c % 3][r] = t;
    }
  };
  uint4 w[2][S::HELD];
  float sc[2][PER] = {};
  auto load = [&](int c, uint4 (&x)[S::HELD], float (&s)[PER]) {
#pragma unroll
    for (int k = 0; k < S::HELD; ++k) {
      const int32_t f = from[c % 3][k * (kMoveThreads / S::LANES) + tid / S::LANES];
      x[k] = make_uint4(0, 0, 0, 0);
      if (f >= 0) x[k] = *reinterpret_cast<const uint4*>(pool + (size_t)f * ROWB + part * 16);
    }
    if constexpr (I8) {
#pragma unroll
      for (int k = 0; k < PER; ++k) {
        const int r = k * kMoveThreads + tid;
        s[k] = 0.f;
        if (r < S::ROWS && from[c % 3][r] >= 0) s[k] = scales[from[c % 3][r]];
      }
    }
  };
  auto store = [&](int c, const uint4 (&x)[S::HELD], const float (&s)[PER]) {
#pragma unroll
    for (int k = 0; k < S::HELD; ++k) {
      const int r = k * (kMoveThreads / S::LANES) + tid / S::LANES;
      if (from[c % 3][r] > -2) *reinterpret_cast<uint4*>(pool + (size_t)to[c % 3][r] * ROWB + part * 16) = x[k];
    }
    if constexpr (I8) {
#pragma unroll
      for (int k = 0; k < PER; ++k) {
        const int r = k * kMoveThreads + tid;
        if (r < S::ROWS && from[c % 3][r] > -2) scales[to[c % 3][r]] = s[k];
      }
    }
  };
  auto sync = [&] {                                    // every read before it is done, every place looked up
    if (ctas > 1) cluster_sync();
    else __syncthreads();
  };
  const int chunks = (kept + step - 1) / step;
  if (chunks == 0) return;                             // the same for all CTAs of the cluster
  look_up(0);
  __syncthreads();
  load(0, w[0], sc[0]);
  look_up(1);
#pragma unroll 1
  for (int c = 0; c < chunks; c += 2) {
    sync();
    load(c + 1, w[1], sc[1]);
    store(c, w[0], sc[0]);
    look_up(c + 2);
    if (c + 1 >= chunks) break;
    sync();
    load(c + 2, w[0], sc[0]);
    store(c + 1, w[1], sc[1]);
    look_up(c + 3);
  }
}

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }
bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
mmshift_status done(cudaError_t e) { return e == cudaSuccess ? MMSHIFT_OK : noalloc_cuda_fail(e); }

// Pages that a call with J's rows can take, and the most of one sequence.
int64_t most_pages(const CacheJob& J, int64_t* of_one) {
  int64_t sum = 0;
  *of_one = 0;
  for (int b = 0; b < J.B; ++b) {
    const int64_t n = J.off[b + 1] - J.off[b];
    const int64_t p = n ? std::min<int64_t>((n + (1 << J.page_shift) - 2 >> J.page_shift) + 1, J.max_pages) : 0;
    sum += p;
    *of_one = std::max(*of_one, p);
  }
  return std::min<int64_t>(sum * J.L * J.Hkv, J.n_pages);
}

size_t place(PagesJob* G, char* at) {
  char* const from = at;
  int64_t one;
  const int64_t most = most_pages(G->c, &one), U = (int64_t)G->c.L * G->c.B * G->c.Hkv;
  G->most = (int32_t)most;
  G->group = 1;
  while (G->group < 32 && 4 * G->group < one) G->group *= 2;   // a lane asks for four pages at once
  G->once = one <= 4 * G->group;
  G->taken = reinterpret_cast<int32_t*>(at);
  at += 256;
  G->list = reinterpret_cast<int32_t*>(at);
  at += align256(most * sizeof(int32_t));
  G->jobs = reinterpret_cast<PageJob*>(at);
  at += align256(most * sizeof(PageJob));
  G->old_table = reinterpret_cast<int32_t*>(at);
  at += align256(U * G->c.max_pages * sizeof(int32_t));
  G->old_lens = reinterpret_cast<int32_t*>(at);
  return at + align256(U * sizeof(int32_t)) - from;
}

mmshift_status pages_job(const mmshift_shape* s, const mmshift_cache* c, int32_t* refs, void* ws, size_t bytes,
                         PagesJob* G) {
  std::memset(G, 0, sizeof(*G));
  mmshift_status st = rows_job(s, c, ws, &G->c);
  if (st != MMSHIFT_OK) return st;
  if ((int64_t)G->c.L * G->c.B * G->c.Hkv > (int64_t)1 << 30) return MMSHIFT_ERR_UNSUPPORTED;
  if (!refs || !aligned(refs, 4)) return MMSHIFT_ERR_INVALID_ARG;
  G->table = const_cast<int32_t*>(c->page_table);
  G->refs = refs;
  G->vec = aligned(refs, 16);
  const size_t need = place(G, static_cast<char*>(ws) + 256);
  return check_workspace(ws, bytes, need);
}

template <bool COMPACT>
cudaError_t launch_take(const PagesJob& G, cudaStream_t st) {
  // One CTA where its threads see two sequences at most and a few pages: a cluster's barriers take
  // 1 to 2 us each. A page for each of 112 sequences, lengths and copies of the state with it: of
  // 8,000 pages 11.8 us by one CTA, 14.3 by a cluster; of 60,000 18.7 and 15.2; and for each of 12,288
  // sequences of 150,000 pages 107 and 28.
  const int64_t U = (int64_t)G.c.L * G.c.B * G.c.Hkv;
  if (U * G.group <= 2 * kTake && G.c.n_pages <= 32 * kTake)
    return launch_kernel(take_pages_kernel<COMPACT, 1>, dim3(1), kTake, 0, st, true, 0, G);
  return launch_kernel(take_pages_kernel<COMPACT, kCluster>, dim3(kCluster), kTake, 0, st, true, kCluster, G);
}

template <int ROWB, bool I8>
cudaError_t launch_move(const PagesJob& G, const int32_t* idx, cudaStream_t st) {
  const CacheJob& J = G.c;
  int requests = 0, longest = 0;
  for (int b = 0; b < J.B; ++b) {
    const int n = J.off[b + 1] - J.off[b];
    requests += n > 0;
    longest = std::max(longest, n);
  }
  const unsigned units = (unsigned)(requests * J.Hkv);
  // As many CTAs a sequence as find places at once (three an SM) and have a chunk each: 16,000 of
  // 32,000 rows of eight heads 53 us (a CTA a sequence 196), half of 4,100 rows of four heads and 28
  // layers 37 (40).
  int ctas = kCluster;
  while (ctas > 1 && ((int64_t)units * J.L * 2 * ctas > 3 * 152 || longest <= ctas / 2 * MoveShape<ROWB, I8>::ROWS))
    ctas /= 2;
  return launch_kernel(move_rows_kernel<ROWB, I8>, dim3(units * ctas, 2, J.L), kMoveThreads, 0, st, true,
                       ctas > 1 ? ctas : 0, G, idx, ctas);
}

// The pairs of a fork, or what is to be given back.
mmshift_status hold(const mmshift_shape* s, const mmshift_cache* c, int32_t* refs, int32_t n, const int32_t* src,
                    const int32_t* dst, void* ws, size_t bytes, cudaStream_t st) {
  HoldJob G;
  std::memset(&G, 0, sizeof(G));
  mmshift_status e = rows_job(s, c, ws, &G.c);
  if (e != MMSHIFT_OK) return e;
  const CacheJob& J = G.c;
  if (!refs || !aligned(refs, 4) || n < 0 || n > J.B || (n && !dst)) return MMSHIFT_ERR_INVALID_ARG;
  bool is_dst[MMSHIFT_MAX_BATCH] = {};
  for (int i = 0; i < n; ++i) {
    if (dst[i] < 0 || dst[i] >= J.B || is_dst[dst[i]]) return MMSHIFT_ERR_INVALID_ARG;
    is_dst[dst[i]] = true;
  }
  for (int i = 0; src && i < n; ++i)
    if (src[i] < 0 || src[i] >= J.B || is_dst[src[i]]) return MMSHIFT_ERR_INVALID_ARG;
  if ((e = check_workspace(ws, bytes)) != MMSHIFT_OK) return e;
  if (!n) return MMSHIFT_OK;
  G.table = const_cast<int32_t*>(c->page_table);
  G.refs = refs;
  G.n = n;
  for (int i = 0; i < n; ++i) {
    G.src[i] = src ? src[i] : -1;
    G.dst[i] = dst[i];
  }
  const int64_t warps = (int64_t)n * J.Hkv;
  return done(launch_kernel(hold_pages_kernel, dim3((unsigned)((warps + 7) / 8), J.L), 256, 0, st, true, 0, G));
}

}  // namespace
}  // namespace mmshift

using namespace mmshift;

extern "C" {

mmshift_status mmshift_cache_pages_workspace_size(const mmshift_shape* s, const mmshift_cache* c, size_t* bytes) {
  PagesJob G;
  std::memset(&G, 0, sizeof(G));
  const mmshift_status st = rows_job(s, c, nullptr, &G.c);
  if (st != MMSHIFT_OK) return st;
  if (!bytes) return MMSHIFT_ERR_INVALID_ARG;
  *bytes = 256 + place(&G, reinterpret_cast<char*>(uintptr_t(256)));
  return MMSHIFT_OK;
}

mmshift_status mmshift_cache_reserve(const mmshift_shape* s, const mmshift_cache* c, int32_t* refs, void* workspace,
                                     size_t workspace_bytes, mmshift_stream_t stream) {
  PagesJob G;
  const mmshift_status st = pages_job(s, c, refs, workspace, workspace_bytes, &G);
  if (st != MMSHIFT_OK) return st;
  if (!G.c.off[G.c.B]) return MMSHIFT_OK;
  cudaError_t e = launch_take<false>(G, (cudaStream_t)stream);
  // a block a page; a call's blocks take many pages in turn
  const unsigned blocks = (unsigned)std::min<int64_t>(G.most, 152 * 8);
  if (e == cudaSuccess)
    e = launch_kernel(copy_pages_kernel, dim3(blocks), 256, 0, (cudaStream_t)stream, true, 0, G);
  return done(e);
}

mmshift_status mmshift_cache_fork(const mmshift_shape* s, const mmshift_cache* c, int32_t* refs, int32_t n,
                                  const int32_t* src, const int32_t* dst, void* workspace, size_t workspace_bytes,
                                  mmshift_stream_t stream) {
  if (n > 0 && !src) return MMSHIFT_ERR_INVALID_ARG;
  return hold(s, c, refs, n, src, dst, workspace, workspace_bytes, (cudaStream_t)stream);
}

mmshift_status mmshift_cache_free(const mmshift_shape* s, const mmshift_cache* c, int32_t* refs, int32_t n,
                                  const int32_t* which, void* workspace, size_t workspace_bytes,
                                  mmshift_stream_t stream) {
  return hold(s, c, refs, n, nullptr, which, workspace, workspace_bytes, (cudaStream_t)stream);
}

mmshift_status mmshift_cache_compact(const mmshift_shape* s, const mmshift_cache* c, int32_t* refs, const int32_t* idx,
                                     const int32_t* count, void* workspace, size_t workspace_bytes,
                                     mmshift_stream_t stream) {
  PagesJob G;
  const mmshift_status st = pages_job(s, c, refs, workspace, workspace_bytes, &G);
  if (st != MMSHIFT_OK) return st;
  if ((G.c.off[G.c.B] && !idx) || !aligned(idx, 4) || !aligned(count, 4)) return MMSHIFT_ERR_INVALID_ARG;
  if (!G.c.off[G.c.B]) return MMSHIFT_OK;
  G.count = count;
  cudaError_t e = launch_take<true>(G, (cudaStream_t)stream);
  if (e == cudaSuccess) {
    const int row = G.c.i8 ? G.c.d : G.c.bf16 ? 2 * G.c.d : 4 * G.c.d;
    const cudaStream_t cs = (cudaStream_t)stream;
    if (G.c.i8) e = row == 128 ? launch_move<128, true>(G, idx, cs) : launch_move<64, true>(G, idx, cs);
    else if (row == 512) e = launch_move<512, false>(G, idx, cs);
    else if (row == 256) e = launch_move<256, false>(G, idx, cs);
    else e = launch_move<128, false>(G, idx, cs);
  }
  return done(e);
}

}  // extern "C"
