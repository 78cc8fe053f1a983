// Pages of a cache held in 4 bits: taking, sharing, letting go and moving them together (kvd_pages_*, kvd.h).  The pages' numbers
// are found by one CTA that looks through the reference counts, so the result does not depend on any order of arrival;
// the pages themselves are moved by a kernel over all SMs, bound by memory: 869 pages in use of 1024, of a
// Qwen3-4B layer's size in 4 layers, moved together in another pool 92 us (512 MB, 5.5 TB/s, the finding 5 of them), in place, 142 of 846 to move, 15
// (84 MB); 64 sequences forked and let go 18 us (47 MB: 9 for the copies, three launches); four forks of a small model's caches 8.2 us, the
// three launches; room for a token of each of 64 sequences 2.1 us in a graph.
#include <string.h>

#include <algorithm>

#include "kvd_internal.h"
#include "kvd_pages.h"
#include "kvd_ptx.cuh"

namespace kvd {

struct PgState {
  int32_t *table, *lens, *refs;
  int pages, seqs, max_pages;
};
template <int N>
struct PgGrow {
  PgState c;
  int32_t *first_out;
  int *status;
  int n;
  int32_t seq[N], count[N];
};
template <int N>
struct PgFork {
  PgState c;
  uint4 *pool;
  int *status;  // [1]: the copies are to be made
  int n, layers;
  int pieces, chunks;  // 16-byte pieces of a page, runs of PG_CHUNK pieces
  int32_t from[N], to[N];
};
template <int N>
struct PgFree {
  PgState c;
  int *status;
  int n;
  int32_t seq[N];
};
struct PgCompact {
  PgState in, out;
  const uint4 *pool;
  uint4 *pool_out;
  int32_t *map, *source, *hole, *used;  // scratch: [pages] each, then the pages in use (-1: nothing is moved) and the holes among them
  int32_t *used_out;
  int *status;
  int layers, pieces, chunks, in_place;
};

constexpr int PG_THREADS = 1024;       // the CTA that finds the pages
constexpr int PG_RUN = 4;              // reference counts a thread looks at in one go
constexpr int PG_COPY_THREADS = 288;   // pieces of a page are a multiple of that
constexpr int PG_COPY_UNROLL = 4;
constexpr int PG_CHUNK = PG_COPY_THREADS * PG_COPY_UNROLL;
constexpr int PG_COPY_CTAS = 6;        // per SM

constexpr int PG_LIST = PG_THREADS;    // free pages that are listed on the way
constexpr int PG_PLENTY = 1 << 29;     // sums stop here (more pages than there can be), so that they stay in 32 bits

// Exclusive sum over the CTA's threads in their order, of numbers up to PG_PLENTY; the total in `total`.  Sums that reach PG_PLENTY are
// only good for telling that they do.
__device__ __forceinline__ int pg_scan(int v, int (&warp_sum)[32], int &total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int s = v;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const int o = __shfl_up_sync(0xffffffffu, s, d);
    s = min(s + (lane >= d ? o : 0), PG_PLENTY);
  }
  __syncthreads();  // (the sums of the call before have been read)
  if (lane == 31) warp_sum[warp] = s;
  __syncthreads();
  int w = warp_sum[lane];
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const int o = __shfl_up_sync(0xffffffffu, w, d);
    w = min(w + (lane >= d ? o : 0), PG_PLENTY);
  }
  total = __shfl_sync(0xffffffffu, w, 31);
  return s - v + (warp > 0 ? __shfl_sync(0xffffffffu, w, warp - 1) : 0);
}

// The first `need` free pages in ascending order: take(k, page) for each.  Returns how many there are, `need` at most.  (Counts that
// this kernel changes by atomics are read past the first-level cache.)
template <class F>
__device__ __forceinline__ int pg_each_free(const PgState &c, int need, int (&warp_sum)[32], F take) {
  int found = 0;
  for (int base = 0; base < c.pages && found < need; base += PG_THREADS * PG_RUN) {
    const int p0 = base + static_cast<int>(threadIdx.x) * PG_RUN;
    bool is_free[PG_RUN];
    int mine = 0, total;
#pragma unroll
    for (int j = 0; j < PG_RUN; ++j) {
      is_free[j] = p0 + j < c.pages && __ldcg(c.refs + p0 + j) == 0;
      mine += is_free[j];
    }
    int k = found + pg_scan(mine, warp_sum, total);
#pragma unroll
    for (int j = 0; j < PG_RUN; ++j)
      if (is_free[j]) {
        if (k < need) take(k, p0 + j);
        ++k;
      }
    found += total;
  }
  return found < need ? found : need;
}

// A page number of a table, -1 where it is none.
__device__ __forceinline__ int pg_entry(const PgState &c, int seq, int j) {
  const int p = c.table[static_cast<long long>(seq) * c.max_pages + j];
  return p >= 0 && p < c.pages ? p : -1;
}
__device__ __forceinline__ int pg_held(const PgState &c, int len) { return len <= 0 ? 0 : min(pg_pages(min(len, INT32_MAX - PG_TOKENS)), c.max_pages); }

template <int N>
__global__ void __launch_bounds__(PG_THREADS) kvd_pages_grow_kernel(const __grid_constant__ PgGrow<N> P) {
  __shared__ int warp_sum[32];
  __shared__ int s_base[N + 1], s_len[N], s_free[PG_LIST];
  const int tid = threadIdx.x;
  grid_launch_dependents();
  grid_dependency_wait();
  int need = 0, len = 0, bad = 0;
  if (tid < P.n) {
    len = P.c.lens[P.seq[tid]];
    const long long grown = static_cast<long long>(len) + P.count[tid];
    bad = len < 0 || grown > static_cast<long long>(P.c.max_pages) * PG_TOKENS;
    if (!bad) need = pg_pages(static_cast<int>(grown)) - pg_pages(len);
    s_len[tid] = len;
  }
  int total;
  const int base = pg_scan(need, warp_sum, total);
  if (tid < P.n) s_base[tid] = base;
  bool ok = !__syncthreads_or(bad);
  // counted first: where the pages do not suffice nothing is written
  if (ok && total > 0) {
    ok = pg_each_free(P.c, total, warp_sum, [&](int k, int page) {
      if (k < PG_LIST) s_free[k] = page;
    }) == total;
    __syncthreads();
  }
  if (ok && total > 0) {
    auto take = [&](int k, int page) {
      int lo = 0, hi = P.n - 1;  // the last entry whose pages begin at or before k: entries without a page share their base with the next
      while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (s_base[mid] <= k) lo = mid;
        else hi = mid - 1;
      }
      const int j = pg_pages(s_len[lo]) + k - s_base[lo];
      if (!KVD_BOUNDS_OK(j >= 0 && j < P.c.max_pages, P.status)) return;
      P.c.table[static_cast<long long>(P.seq[lo]) * P.c.max_pages + j] = page;
      P.c.refs[page] = 1;
    };
    if (total <= PG_LIST) {
      if (tid < total) take(tid, s_free[tid]);
    } else {
      pg_each_free(P.c, total, warp_sum, take);
    }
  }
  if (tid < P.n) {
    if (ok) P.c.lens[P.seq[tid]] = len + P.count[tid];
    P.first_out[tid] = ok ? len : -1;
  }
  if (!ok && tid == 0) atomicOr(P.status, STATUS_CAPACITY);
}

template <int N>
__global__ void __launch_bounds__(PG_THREADS) kvd_pages_fork_kernel(const __grid_constant__ PgFork<N> P) {
  __shared__ int warp_sum[32];
  __shared__ int s_page[N];  // where the entry's last page is copied to, -1: it is full
  __shared__ int s_nth[N], s_free[N];
  __shared__ int s_held_to[N], s_held_from[N];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  grid_launch_dependents();
  grid_dependency_wait();
  int partial = 0, bad = 0, len = 0;
  if (tid < P.n) {
    len = P.c.lens[P.from[tid]];
    s_held_to[tid] = pg_held(P.c, P.c.lens[P.to[tid]]);
    s_held_from[tid] = pg_held(P.c, len);
    bad = len < 0 || len > static_cast<long long>(P.c.max_pages) * PG_TOKENS;
    partial = !bad && len % PG_TOKENS != 0;
  }
  int total;
  const int nth = pg_scan(partial, warp_sum, total);
  if (tid < P.n) {
    s_page[tid] = -1;
    if (partial) s_nth[nth] = tid;
  }
  bool ok = !__syncthreads_or(bad);
  // a warp for each list, four lists' entries asked for at once: visit(list, place, page)
  auto each_page = [&](const int32_t *seqs, const int *held, auto visit) {
    for (int i0 = warp; i0 < P.n; i0 += 128) {
      int most = 0;
#pragma unroll
      for (int q = 0; q < 4; ++q) most = max(most, i0 + 32 * q < P.n ? held[i0 + 32 * q] : 0);
      for (int j = lane; j < most; j += 32) {
        int page[4];
        bool some[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int i = i0 + 32 * q;
          some[q] = i < P.n && j < held[i];
          page[q] = some[q] ? pg_entry(P.c, seqs[i], j) : -1;
        }
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (some[q]) visit(i0 + 32 * q, j, page[q]);
      }
    }
    __syncthreads();
  };
  if (ok) {
    auto let_go = [&](int step) {
      each_page(P.to, s_held_to, [&](int, int, int p) {
        if (p >= 0) atomicAdd(P.c.refs + p, step);
      });
    };
    let_go(-1);
    ok = total == 0 || pg_each_free(P.c, total, warp_sum, [&](int k, int page) { s_free[k] = page; }) == total;
    if (!ok) let_go(1);
  }
  if (ok) {
    __syncthreads();
    if (tid < total && KVD_BOUNDS_OK(total <= N && s_nth[tid] >= 0 && s_nth[tid] < P.n, P.status)) s_page[s_nth[tid]] = s_free[tid];
    __syncthreads();
    each_page(P.from, s_held_from, [&](int i, int j, int p) {
      if (j == s_held_from[i] - 1 && s_page[i] >= 0) p = s_page[i];
      P.c.table[static_cast<long long>(P.to[i]) * P.c.max_pages + j] = p;
      if (p >= 0) atomicAdd(P.c.refs + p, 1);
    });
    if (tid < P.n) P.c.lens[P.to[tid]] = len;
  }
  if (tid == 0) {
    P.status[1] = ok;
    if (!ok) atomicOr(P.status, STATUS_CAPACITY);
  }
}

// A run of up to PG_CHUNK 16-byte pieces, four of a thread's in flight.
__device__ __forceinline__ void pg_copy_run(const uint4 *src, uint4 *dst, int pieces) {
  uint4 x[PG_COPY_UNROLL];
#pragma unroll
  for (int u = 0; u < PG_COPY_UNROLL; ++u)
    if (static_cast<int>(threadIdx.x) + u * PG_COPY_THREADS < pieces) x[u] = __ldcs(src + threadIdx.x + u * PG_COPY_THREADS);
#pragma unroll
  for (int u = 0; u < PG_COPY_UNROLL; ++u)
    if (static_cast<int>(threadIdx.x) + u * PG_COPY_THREADS < pieces) __stcs(dst + threadIdx.x + u * PG_COPY_THREADS, x[u]);
}

template <int N>
__global__ void __launch_bounds__(PG_COPY_THREADS) kvd_pages_fork_copy_kernel(const __grid_constant__ PgFork<N> P) {
  grid_launch_dependents();
  grid_dependency_wait();
  if (P.status[1] == 0) return;
  // a CTA keeps to a page and a run of its pieces, in some of the layers
  const int runs = P.n * P.chunks, parts = gridDim.x / runs;  // (as many CTAs as that makes, or fewer, one for all layers then)
  for (int u = blockIdx.x; u < runs * max(parts, 1); u += gridDim.x) {
    const int i = u % runs / P.chunks, chunk = u % P.chunks;
    const int len = P.c.lens[P.from[i]];
    if (len % PG_TOKENS == 0) continue;
    const int src = pg_entry(P.c, P.from[i], len / PG_TOKENS), dst = pg_entry(P.c, P.to[i], len / PG_TOKENS);
    if (src < 0 || dst < 0) continue;
    for (int layer = u / runs; layer < P.layers; layer += max(parts, 1)) {
      const long long slab = static_cast<long long>(layer) * P.c.pages;
      pg_copy_run(P.pool + (slab + src) * P.pieces + chunk * PG_CHUNK, P.pool + (slab + dst) * P.pieces + chunk * PG_CHUNK,
                  min(PG_CHUNK, P.pieces - chunk * PG_CHUNK));
    }
  }
}

// One CTA per sequence.
template <int N>
__global__ void __launch_bounds__(256) kvd_pages_free_kernel(const __grid_constant__ PgFree<N> P) {
  grid_launch_dependents();
  grid_dependency_wait();
  const int seq = P.seq[blockIdx.x], held = pg_held(P.c, P.c.lens[seq]);
  for (int j = threadIdx.x; j < held; j += 256) {
    const int p = pg_entry(P.c, seq, j);
    if (p >= 0) atomicSub(P.c.refs + p, 1);
    else atomicOr(P.status, STATUS_POSITION);
  }
  __syncthreads();
  if (threadIdx.x == 0) P.c.lens[seq] = 0;
}

__global__ void __launch_bounds__(PG_THREADS) kvd_pages_compact_kernel(const __grid_constant__ PgCompact P) {
  __shared__ int warp_sum[32];
  const int tid = threadIdx.x;
  grid_launch_dependents();
  grid_dependency_wait();
  int mine = 0, used;
  for (int p = tid; p < P.in.pages; p += PG_THREADS) mine += P.in.refs[p] != 0;
  pg_scan(mine, warp_sum, used);
  if (tid == 0 && P.used_out) *P.used_out = used;
  if (used > P.out.pages) {
    if (tid == 0) {
      *P.used = -1;
      atomicOr(P.status, STATUS_CAPACITY);
    }
    return;
  }
  if (tid == 0) *P.used = used;
  // below `used`: pages stay, the free ones are the holes; from there on, the k-th page goes to the k-th hole
  int holes = 0, movers = 0;
  for (int base = 0; base < P.in.pages; base += PG_THREADS) {
    const int p = base + tid;
    const bool held = p < P.in.pages && P.in.refs[p] != 0;
    int at, total;
    if (base < used) {
      const bool hole = p < used && !held;
      at = pg_scan(hole, warp_sum, total);
      if (hole) P.hole[holes + at] = p;
      holes += total;
      if (p < P.in.pages) P.map[p] = p < used && held ? p : -1;
      if (p < used && held) P.source[p] = p;
    }
    if (base + PG_THREADS > used) {
      const bool mover = p >= used && held;
      __syncthreads();  // the holes found so far can be read (there are as many as movers in all, and they come first)
      at = pg_scan(mover, warp_sum, total);
      if (mover && KVD_BOUNDS_OK(movers + at < holes, P.status)) {
        const int to = P.hole[movers + at];
        P.source[to] = p;
        P.map[p] = to;
      } else if (p >= used && p < P.in.pages) {
        P.map[p] = -1;
      }
      movers += total;
    }
  }
  if (tid == 0) P.used[1] = holes;
  __syncthreads();
  if (P.in_place) {
    for (int d = tid; d < used; d += PG_THREADS)
      if (P.source[d] != d) P.in.refs[d] = P.in.refs[P.source[d]];  // (read from above `used`, written below)
    __syncthreads();
    for (int p = used + tid; p < P.in.pages; p += PG_THREADS) P.in.refs[p] = 0;
  } else {
    for (int d = tid; d < P.out.pages; d += PG_THREADS) P.out.refs[d] = d < used ? P.in.refs[P.source[d]] : 0;
  }
}

__global__ void __launch_bounds__(PG_COPY_THREADS) kvd_pages_compact_copy_kernel(const __grid_constant__ PgCompact P) {
  grid_launch_dependents();
  grid_dependency_wait();
  const int used = *P.used;
  if (used < 0) return;
  // the tables
  const long long entries = static_cast<long long>(P.in.seqs) * P.in.max_pages;
  for (long long e = blockIdx.x * static_cast<long long>(PG_COPY_THREADS) + threadIdx.x; e < entries; e += static_cast<long long>(gridDim.x) * PG_COPY_THREADS) {
    const int seq = static_cast<int>(e / P.in.max_pages), j = static_cast<int>(e % P.in.max_pages);
    const int len = P.in.lens[seq];
    if (j == 0 && !P.in_place) P.out.lens[seq] = len;
    if (j < pg_held(P.in, len)) {
      const int p = pg_entry(P.in, seq, j);
      P.out.table[e] = p >= 0 ? P.map[p] : -1;
    }
  }
  // the pages: all of them, or those that fill the holes
  const long long units = static_cast<long long>(P.in_place ? P.used[1] : used) * P.layers * P.chunks;
  for (long long u = blockIdx.x; u < units; u += gridDim.x) {
    const int k = static_cast<int>(u / (P.layers * P.chunks)), rest = static_cast<int>(u % (P.layers * P.chunks)), layer = rest / P.chunks, chunk = rest % P.chunks;
    const int d = P.in_place ? P.hole[k] : k, s = P.source[d];
    if (!KVD_BOUNDS_OK(d >= 0 && d < P.out.pages && s >= 0 && s < P.in.pages, P.status)) continue;
    pg_copy_run(P.pool + (static_cast<long long>(layer) * P.in.pages + s) * P.pieces + chunk * PG_CHUNK,
                P.pool_out + (static_cast<long long>(layer) * P.out.pages + d) * P.pieces + chunk * PG_CHUNK, min(PG_CHUNK, P.pieces - chunk * PG_CHUNK));
  }
}

// ------------------------------------------------------------------------------------------------ host side
OnDevice::OnDevice(const kvd_ctx *ctx) {
  int now = -1;
  if (cudaGetDevice(&now) == cudaSuccess && now != ctx->device && cudaSetDevice(ctx->device) == cudaSuccess) back_ = now;
}
OnDevice::~OnDevice() {
  if (back_ >= 0) cudaSetDevice(back_);
}

kvd_status check_paged(const kvd_ctx *ctx, const kvd_paged_cache *c) {
  (void)ctx;
  if (!c || !c->pool || !c->table || !c->lens || !c->refs) return KVD_ERR_INVALID_ARG;
  if (c->layers < 1 || c->pages < 1 || c->seqs < 1 || c->max_pages < 1) return KVD_ERR_INVALID_ARG;
  if (c->max_pages > INT32_MAX / PG_TOKENS - 1) return KVD_ERR_SHAPE;  // positions are int32
  if ((reinterpret_cast<uintptr_t>(c->pool) & 127u) != 0 || !aligned4({c->table, c->lens, c->refs})) return KVD_ERR_ALIGNMENT;
  return KVD_OK;
}

kvd_status check_page_seqs(const kvd_paged_cache *c, int n, const int32_t *seqs, bool distinct) {
  for (int i = 0; i < n; ++i)
    if (seqs[i] < 0 || seqs[i] >= c->seqs) return KVD_ERR_INVALID_ARG;
  if (!distinct || n < 2) return KVD_OK;
  constexpr int BITS = 4096;
  uint64_t seen[BITS / 64] = {};
  bool low = true;
  for (int i = 0; i < n; ++i) {
    if (seqs[i] >= BITS) {
      low = false;
      break;
    }
    uint64_t &w = seen[seqs[i] / 64];
    const uint64_t bit = 1ull << (seqs[i] % 64);
    if (w & bit) return KVD_ERR_INVALID_ARG;
    w |= bit;
  }
  if (low) return KVD_OK;
  int32_t sorted[PG_MANY];
  memcpy(sorted, seqs, n * sizeof(int32_t));
  std::sort(sorted, sorted + n);
  for (int i = 1; i < n; ++i)
    if (sorted[i] == sorted[i - 1]) return KVD_ERR_INVALID_ARG;
  return KVD_OK;
}

static PgState state_of(const kvd_paged_cache *c) { return PgState{c->table, c->lens, c->refs, c->pages, c->seqs, c->max_pages}; }

static kvd_status pg_launched(kvd_ctx *ctx, cudaError_t e, const char *what) {
  if (e != cudaSuccess) return cuda_fail(ctx, e, what);
  ctx->launches += 1;
  return KVD_OK;
}

// The kernel behind the one that found the pages: its CTAs wait for it on the SMs that are free meanwhile.
template <typename P>
static cudaError_t launch_behind(const kvd_ctx *ctx, void (*kern)(P), unsigned grid, cudaStream_t stream, const P &params) {
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = dim3(grid, 1, 1);
  cfg.blockDim = dim3(PG_COPY_THREADS, 1, 1);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = serial_launch_mask() & 8 ? 0 : 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, params);
}

static unsigned copy_grid(const kvd_ctx *ctx, long long units) {
  const long long cap = static_cast<long long>(ctx->num_sms) * PG_COPY_CTAS;
  return static_cast<unsigned>(units < 1 ? 1 : units > cap ? cap : units);
}

template <int N>
static kvd_status launch_grow(kvd_ctx *ctx, const kvd_paged_cache *c, int n, const int32_t *seqs, const int32_t *counts, int32_t *first_out, cudaStream_t stream) {
  PgGrow<N> P;
  P.c = state_of(c);
  P.first_out = first_out;
  P.status = ctx->d_status;
  P.n = n;
  memcpy(P.seq, seqs, n * sizeof(int32_t));
  memcpy(P.count, counts, n * sizeof(int32_t));
  return pg_launched(ctx, launch_paged(ctx, kvd_pages_grow_kernel<N>, 1, PG_THREADS, stream, P), "launch pages_grow");
}

template <int N>
static kvd_status launch_fork(kvd_ctx *ctx, const kvd_paged_cache *c, int n, const int32_t *from, const int32_t *to, cudaStream_t stream) {
  PgFork<N> P;
  P.c = state_of(c);
  P.pool = static_cast<uint4 *>(c->pool);
  P.status = ctx->d_status;
  P.n = n;
  P.layers = c->layers;
  P.pieces = static_cast<int>(pg_page_bytes(ctx->desc.d_head, ctx->desc.n_kv_heads) / 16);
  P.chunks = (P.pieces + PG_CHUNK - 1) / PG_CHUNK;
  memcpy(P.from, from, n * sizeof(int32_t));
  memcpy(P.to, to, n * sizeof(int32_t));
  kvd_status st = pg_launched(ctx, launch_paged(ctx, kvd_pages_fork_kernel<N>, 1, PG_THREADS, stream, P), "launch pages_fork");
  if (st != KVD_OK) return st;
  return pg_launched(ctx, launch_behind(ctx, kvd_pages_fork_copy_kernel<N>, copy_grid(ctx, static_cast<long long>(n) * P.layers * P.chunks), stream, P),
                     "launch pages_fork (copies)");
}

template <int N>
static kvd_status launch_free(kvd_ctx *ctx, const kvd_paged_cache *c, int n, const int32_t *seqs, cudaStream_t stream) {
  PgFree<N> P;
  P.c = state_of(c);
  P.status = ctx->d_status;
  P.n = n;
  memcpy(P.seq, seqs, n * sizeof(int32_t));
  return pg_launched(ctx, launch_paged(ctx, kvd_pages_free_kernel<N>, n, 256, stream, P), "launch pages_free");
}

}  // namespace kvd

using namespace kvd;

extern "C" size_t kvd_page_bytes(const kvd_model_desc *desc) {
  if (kvd_workspace_bytes(desc) == 0) return 0;  // (a description the library does not take)
  return static_cast<size_t>(pg_page_bytes(desc->d_head, desc->n_kv_heads));
}

extern "C" size_t kvd_pages_scratch_bytes(int pages) { return pages < 1 ? 0 : (3 * static_cast<size_t>(pages) + 4) * sizeof(int32_t); }

extern "C" kvd_status kvd_pages_grow(kvd_ctx *ctx, const kvd_paged_cache *cache, int n, const int32_t *seqs, const int32_t *counts, int32_t *first_out,
                                     void *stream_) {
  if (!ctx || n < 0) return KVD_ERR_INVALID_ARG;
  kvd_status st = check_paged(ctx, cache);
  if (st != KVD_OK) return st;
  if (n == 0) return KVD_OK;
  if (!seqs || !counts || !first_out) return KVD_ERR_INVALID_ARG;
  if (n > KVD_MAX_PAGE_SEQS) return KVD_ERR_CAPACITY;
  if (!aligned4({first_out})) return KVD_ERR_ALIGNMENT;
  st = check_page_seqs(cache, n, seqs, true);
  if (st != KVD_OK) return st;
  for (int i = 0; i < n; ++i)
    if (counts[i] < 0) return KVD_ERR_INVALID_ARG;
  const OnDevice here(ctx);
  cudaStream_t stream = static_cast<cudaStream_t>(stream_);
  return n <= PG_FEW ? launch_grow<PG_FEW>(ctx, cache, n, seqs, counts, first_out, stream) : launch_grow<PG_MANY>(ctx, cache, n, seqs, counts, first_out, stream);
}

extern "C" kvd_status kvd_pages_fork(kvd_ctx *ctx, const kvd_paged_cache *cache, int n, const int32_t *from, const int32_t *to, void *stream_) {
  if (!ctx || n < 0) return KVD_ERR_INVALID_ARG;
  kvd_status st = check_paged(ctx, cache);
  if (st != KVD_OK) return st;
  if (n == 0) return KVD_OK;
  if (!from || !to) return KVD_ERR_INVALID_ARG;
  if (n > KVD_MAX_PAGE_SEQS) return KVD_ERR_CAPACITY;
  st = check_page_seqs(cache, n, from, false);
  if (st == KVD_OK) st = check_page_seqs(cache, n, to, true);
  if (st != KVD_OK) return st;
  for (int i = 0; i < n; ++i)
    for (int j = 0; j < n; ++j)
      if (from[i] == to[j]) return KVD_ERR_INVALID_ARG;
  const OnDevice here(ctx);
  cudaStream_t stream = static_cast<cudaStream_t>(stream_);
  return n <= PG_FEW ? launch_fork<PG_FEW>(ctx, cache, n, from, to, stream) : launch_fork<PG_MANY>(ctx, cache, n, from, to, stream);
}

extern "C" kvd_status kvd_pages_free(kvd_ctx *ctx, const kvd_paged_cache *cache, int n, const int32_t *seqs, void *stream_) {
  if (!ctx || n < 0) return KVD_ERR_INVALID_ARG;
  kvd_status st = check_paged(ctx, cache);
  if (st != KVD_OK) return st;
  if (n == 0) return KVD_OK;
  if (!seqs) return KVD_ERR_INVALID_ARG;
  if (n > KVD_MAX_PAGE_SEQS) return KVD_ERR_CAPACITY;
  st = check_page_seqs(cache, n, seqs, true);
  if (st != KVD_OK) return st;
  const OnDevice here(ctx);
  cudaStream_t stream = static_cast<cudaStream_t>(stream_);
  return n <= PG_FEW ? launch_free<PG_FEW>(ctx, cache, n, seqs, stream) : launch_free<PG_MANY>(ctx, cache, n, seqs, stream);
}

static bool ranges_meet(const void *a, size_t na, const void *b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}

extern "C" kvd_status kvd_pages_compact(kvd_ctx *ctx, const kvd_paged_cache *in, const kvd_paged_cache *out, void *scratch, size_t scratch_bytes,
                                        int32_t *used_out, void *stream_) {
  if (!ctx) return KVD_ERR_INVALID_ARG;
  kvd_status st = check_paged(ctx, in);
  if (st == KVD_OK) st = check_paged(ctx, out);
  if (st != KVD_OK) return st;
  if (!scratch || in->layers != out->layers || in->seqs != out->seqs || in->max_pages != out->max_pages) return KVD_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(scratch) & 15u) != 0 || !aligned4({used_out})) return KVD_ERR_ALIGNMENT;
  if (scratch_bytes < kvd_pages_scratch_bytes(in->pages)) return KVD_ERR_CAPACITY;
  const long long page = pg_page_bytes(ctx->desc.d_head, ctx->desc.n_kv_heads);
  const bool in_place = in->pool == out->pool && in->table == out->table && in->lens == out->lens && in->refs == out->refs && in->pages == out->pages;
  if (!in_place) {
    // nothing that is written may be read
    struct Range {
      const void *at;
      size_t bytes;
    };
    auto arrays = [&](const kvd_paged_cache *c, Range (&r)[4]) {
      r[0] = {c->pool, static_cast<size_t>(c->layers) * c->pages * page};
      r[1] = {c->table, static_cast<size_t>(c->seqs) * c->max_pages * 4};
      r[2] = {c->lens, static_cast<size_t>(c->seqs) * 4};
      r[3] = {c->refs, static_cast<size_t>(c->pages) * 4};
    };
    Range a[4], b[4];
    arrays(in, a);
    arrays(out, b);
    for (const Range &x : a)
      for (const Range &y : b)
        if (ranges_meet(x.at, x.bytes, y.at, y.bytes)) return KVD_ERR_INVALID_ARG;
  }
  const OnDevice here(ctx);
  cudaStream_t stream = static_cast<cudaStream_t>(stream_);
  PgCompact P;
  P.in = state_of(in);
  P.out = state_of(out);
  P.pool = static_cast<const uint4 *>(in->pool);
  P.pool_out = static_cast<uint4 *>(out->pool);
  P.map = static_cast<int32_t *>(scratch);
  P.source = P.map + in->pages;
  P.hole = P.source + in->pages;
  P.used = P.hole + in->pages;
  P.used_out = used_out;
  P.status = ctx->d_status;
  P.layers = in->layers;
  P.pieces = static_cast<int>(page / 16);
  P.chunks = (P.pieces + PG_CHUNK - 1) / PG_CHUNK;
  P.in_place = in_place;
  st = pg_launched(ctx, launch_paged(ctx, kvd_pages_compact_kernel, 1, PG_THREADS, stream, P), "launch pages_compact");
  if (st != KVD_OK) return st;
  return pg_launched(ctx, launch_behind(ctx, kvd_pages_compact_copy_kernel, copy_grid(ctx, static_cast<long long>(in->pages) * P.layers * P.chunks), stream, P),
                     "launch pages_compact (copies)");
}
