// Eviction from a cache by accumulated weight (include/kvd.h, kvd_cache_evict).
//
// Of the len slots of a sequence the `keep` largest stay, in the order (protected, weight, lower slot first).  Both parts of
// that order fit one 32-bit key, larger is better: the weight's bits mapped so that unsigned order is numeric order (a NaN
// counts as minus infinity, -0 as +0), and above all of them one value for protected slots.  The keep-th largest key T is
// found digit by digit (11, 11 and 10 bits from the top): a histogram of the keys that agree with T so far, and in it the
// digit at which the count from above passes what is still wanted.  Slots above T stay, and of those equal to T as many of
// the lowest as are wanted.
//
// One CTA per sequence of up to EV_RUN slots, a cluster beyond, its slots dealt out in contiguous runs that stay in shared
// memory, so that memory is read once.  Histograms of a cluster's CTAs are added up in the shared memory of rank 0 (integer
// additions: their order changes nothing), every CTA scans the sum itself; ranks among kept, evicted and moved slots are prefix
// counts: a warp owns a run of slots, keeps what concerns them as masks of a turn's 32 lanes, and counts bits.
//
// Selecting is a chain of barriers (8192 slots, 14 us before ranks were counted from masks: keys 2.3, digits 2.9, ranks 5,
// lists 3.6; 10 to 12 since): splitting it over a cluster's CTAs shortens the walks and lengthens the barriers.  us for the call, 8 x 8192
// slots of a Qwen3-4B layer to 2001, one CTA 35, clusters of 2 / 4 / 8 37 / 38 / 42; 1 x 32768 of a SmolLM2 layer, clusters of
// 2 / 4 / 8 31 / 25 / 27.  Moving rows is a copy, 5.8 TB/s (132 MB, 22.7 us).
//
// Slots below `keep` that stay keep their place; the r-th evicted slot below `keep` (a hole) receives the r-th kept slot
// from `keep` on (a mover).  So an eviction in place moves as few keys as possible, and no key is read that the same call
// overwrites: sources lie at `keep` and above, destinations below.  The second kernel copies the keys' rows.
#include <math_constants.h>
#include <string.h>

#include "kvd_internal.h"
#include "kvd_ptx.cuh"

namespace kvd {

constexpr int EV_THREADS = 1024;
constexpr int EV_WARPS = EV_THREADS / 32;
constexpr int EV_BINS = 2048;
constexpr int EV_BATCH = 8;                       // slots whose loads a thread has in flight
constexpr int EV_MAX_CTAS = 8;                    // a portable cluster
constexpr int EV_CTA_SLOTS = KVD_MAX_EVICT_SLOTS / EV_MAX_CTAS;
constexpr int EV_RUN = 8192;                      // slots that one CTA is enough for
constexpr int EV_SMALL = 2048;                    // slots up to which the rows are moved in the same launch
constexpr int EV_SMALL_BYTES = 128 << 10;         // ... if a CTA has no more to read than this
constexpr uint32_t EV_PROTECTED = 0xffffffffu;    // above the key of plus infinity, 0xff800000
constexpr uint32_t EV_GONE = 0x80000000u, EV_MOVES = 0x40000000u;
constexpr int EV_MAX_SEQS = 64;
constexpr int EV_ROW_THREADS = 256;

struct EvictParams {
  const float *weights;
  const int32_t *positions;  // or null: slot j holds position j
  float *weights_out;        // or null
  int32_t *positions_out;    // or null
  int32_t *slots_out, *evicted_out;
  long long cap_in, cap_out, evicted_stride;  // slots per sequence
  int keep, protect_below, run;  // run: slots per CTA of the cluster
  const uint4 *k, *v;
  uint4 *k_out, *v_out;
  long long row_in, row_out;  // 16-byte chunks between rows
  int row_chunks, rows_per_cta;
  int *status;
  int len[EV_MAX_SEQS], protect_from[EV_MAX_SEQS];
};

// (words: a single CTA's holes, at most half of its slots, follow its counts in hist; a small cache's places the unused ones in sum)
static_assert(3 * EV_BINS >= EV_SMALL, "places of a small cache");
static_assert(2 * 3 * EV_BINS >= EV_RUN, "a single CTA's holes");
struct EvictShared {
  uint32_t hist[3][EV_BINS];    // this CTA's counts, by pass; a single CTA's holes after that
  uint32_t sum[3][EV_BINS];     // rank 0: the cluster's, added up by remote atomics
  uint32_t warp_sum[EV_WARPS], part[2][EV_WARPS];
  uint32_t digit, above, through;  // found in the current pass: the digit, counts of the keys above it, and with it
  uint32_t count[2];            // of this CTA's run: slots equal to T; evicted ones and movers
};

__device__ __forceinline__ uint32_t evict_key(float w) {
  w = w == w ? w + 0.0f : -CUDART_INF_F;
  const uint32_t u = __float_as_uint(w);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void add_cluster_u32(uint32_t addr, uint32_t v) {
  asm volatile("red.relaxed.cluster.shared::cluster.add.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}

__global__ void __launch_bounds__(EV_THREADS, 1) kvd_evict_select_kernel(const __grid_constant__ EvictParams P, int ctas, int copies) {
  extern __shared__ __align__(16) uint8_t ev_smem[];
  EvictShared &S = *reinterpret_cast<EvictShared *>(ev_smem);
  uint32_t *ev_keys = reinterpret_cast<uint32_t *>(ev_smem + sizeof(EvictShared));  // [run], and the slots' positions behind them
  int32_t *ev_pos = reinterpret_cast<int32_t *>(ev_keys + P.run);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // (copies > 1: each CTA of the cluster takes all of the sequence's slots, comes to the same result, and moves a share of the rows)
  const int rank = ctas > 1 ? static_cast<int>(cluster_ctarank()) : 0, copy = copies > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  const int b = static_cast<int>(blockIdx.x) / (ctas * copies);
  const int len = P.len[b], keep = P.keep < len ? P.keep : len;
  const int slot0 = rank * P.run, n = max(0, min(P.run, len - slot0));
  auto all_sync = [&]() {
    if (ctas > 1) cluster_sync_all();
    else __syncthreads();
  };
  auto remote = [&](const void *p, int r) { return map_to_cta(smem_u32(p), static_cast<uint32_t>(r)); };  // (of a cluster)
  auto clear = [&]() {
    for (int i = tid; i < EV_BINS; i += EV_THREADS) {
      S.hist[0][i] = S.hist[1][i] = S.hist[2][i] = 0u;
      S.sum[0][i] = S.sum[1][i] = S.sum[2][i] = 0u;
    }
  };
  clear();
  grid_launch_dependents();
  grid_dependency_wait();
  const float *w = P.weights + b * P.cap_in;
  const int32_t *pos = P.positions ? P.positions + b * P.cap_in : nullptr;
  const int from = P.protect_from[b];
  auto is_protected = [&](int p) { return p < P.protect_below || p >= from; };
  all_sync();  // histograms are clear everywhere
  for (int at = tid; at < n; at += EV_BATCH * EV_THREADS) {
    int p[EV_BATCH];
    float x[EV_BATCH];
#pragma unroll
    for (int u = 0; u < EV_BATCH; ++u) {
      const int i = at + u * EV_THREADS;
      p[u] = i < n && pos ? pos[slot0 + i] : slot0 + i;
      x[u] = i < n ? w[slot0 + i] : 0.f;
    }
#pragma unroll
    for (int u = 0; u < EV_BATCH; ++u) {
      const int i = at + u * EV_THREADS;
      if (i < n) {
        const uint32_t key = is_protected(p[u]) ? EV_PROTECTED : evict_key(x[u]);
        ev_keys[i] = key;
        ev_pos[i] = p[u];
        if (keep < len) atomicAdd(&S.hist[0][key >> 21], 1u);
      }
    }
  }
  if (copies > 1) cluster_sync_all();  // everyone has read what the first of them may overwrite
  // ---- T: the keep-th largest key; need: how many of the slots equal to it stay
  uint32_t T, need;
  auto select = [&]() {
    T = 0u;
    need = static_cast<uint32_t>(keep);
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
      uint32_t *hist = S.hist[pass];
      __syncthreads();
      uint32_t *sum = S.sum[pass];
      if (ctas > 1) {
        const uint32_t dst = remote(sum, 0);
        for (int i = tid; i < EV_BINS; i += EV_THREADS)
          if (hist[i] != 0u) add_cluster_u32(dst + 4 * i, hist[i]);
        cluster_sync_all();
      }
      // counts from the top: thread t holds bins 2047 - 2t and 2046 - 2t
      uint32_t c0, c1;
      if (ctas > 1) {
        const uint32_t src = remote(sum, 0);
        c0 = ld_cluster_u32(src + 4 * (EV_BINS - 1 - 2 * tid));
        c1 = ld_cluster_u32(src + 4 * (EV_BINS - 2 - 2 * tid));
      } else {
        c0 = hist[EV_BINS - 1 - 2 * tid];
        c1 = hist[EV_BINS - 2 - 2 * tid];
      }
      uint32_t incl = c0 + c1;
#pragma unroll
      for (int k = 1; k < 32; k <<= 1) {
        const uint32_t o = __shfl_up_sync(0xffffffffu, incl, k);
        if (lane >= k) incl += o;
      }
      if (lane == 31) S.warp_sum[warp] = incl;
      __syncthreads();
      uint32_t before = 0;
      {
        const uint32_t v = lane < warp ? S.warp_sum[lane] : 0u;
        before = __reduce_add_sync(0xffffffffu, v);
      }
      const uint32_t a0 = before + incl - c0 - c1, a1 = a0 + c0, a2 = a1 + c1;  // keys above either bin, and through both
      if (a0 < need && need <= a1) {
        S.digit = EV_BINS - 1 - 2 * tid;
        S.above = a0;
        S.through = a1;
      } else if (a1 < need && need <= a2) {
        S.digit = EV_BINS - 2 - 2 * tid;
        S.above = a1;
        S.through = a2;
      }
      __syncthreads();
      T |= S.digit << shift;
      if (S.through == need) {  // all keys that agree with T so far stay: none of them is below it
        need = 0x7fffffffu;
        break;
      }
      need -= S.above;
      if (pass < 2) {
        const int next = pass == 0 ? 10 : 0;
        const uint32_t mask = pass == 0 ? 0x7ffu : 0x3ffu;
        uint32_t *nh = S.hist[pass + 1];
        for (int i = tid; i < n; i += EV_THREADS) {
          const uint32_t key = ev_keys[i];
          if ((key >> shift) == (T >> shift)) atomicAdd(&nh[(key >> next) & mask], 1u);
        }
      }
    }
  };
  T = need = 0u;
  if (keep < len && keep > 0) {
    select();
    if (T == EV_PROTECTED) {
      // Protected slots alone reach `keep`: once more among them, by their weights, with all others below minus infinity.
      all_sync();
      clear();
      all_sync();
      for (int i = tid; i < n; i += EV_THREADS) {
        const uint32_t key = is_protected(ev_pos[i]) ? evict_key(w[slot0 + i]) : 0u;
        ev_keys[i] = key;
        atomicAdd(&S.hist[0][key >> 21], 1u);
      }
      // (the weights were read again: once more everyone has to be done before the first CTA writes them.  T is the same in all
      // CTAs of a cluster, so all of them are here.)
      if (copies > 1) cluster_sync_all();
      select();
    }
  }
  __syncthreads();
  // ---- ranks.  A warp owns a contiguous part of the run, 32 slots to a turn, and lane t keeps what concerns turn t as masks:
  // counts of lanes, turns, warps and CTAs before a slot are then counts in slot order.  A slot's key gives way to what becomes
  // of it: its own index (stays), EV_MOVES | rank, EV_GONE | rank.
  const int turns = (n + EV_THREADS - 1) / EV_THREADS, i0 = min(n, warp * turns * 32), i1 = min(n, i0 + turns * 32);
  const uint32_t before_me = (1u << lane) - 1u;
  auto lower = [](int k) { return k >= 32 ? ~0u : k <= 0 ? 0u : (1u << k) - 1u; };
  auto lanes_before = [&](uint32_t mine, uint32_t *total) {
    uint32_t incl = mine;
#pragma unroll
    for (int k = 1; k < 32; k <<= 1) {
      const uint32_t o = __shfl_up_sync(0xffffffffu, incl, k);
      if (lane >= k) incl += o;
    }
    *total = __shfl_sync(0xffffffffu, incl, 31);
    return incl - mine;
  };
  auto warps_before = [&](uint32_t mine, uint32_t (&of_warp)[EV_WARPS], uint32_t *total) {  // (mine: the same in all lanes)
    if (lane == 0) of_warp[warp] = mine;
    __syncthreads();
    const uint32_t v = of_warp[lane];
    *total = __reduce_add_sync(0xffffffffu, v);
    return __reduce_add_sync(0xffffffffu, lane < warp ? v : 0u);
  };
  uint32_t same = 0, stay = 0, total, of_warp;  // of turn `lane`: slots whose key is T, and those above
#pragma unroll 4
  for (int t = 0; t < turns; ++t) {
    const int i = i0 + 32 * t + lane;
    const uint32_t key = i < i1 ? ev_keys[i] : 0u;
    const uint32_t eq = __ballot_sync(0xffffffffu, i < i1 && key == T), gt = __ballot_sync(0xffffffffu, i < i1 && key > T);
    if (lane == t) {
      same = eq;
      stay = gt;
    }
  }
  const int base = i0 + 32 * lane;
  const uint32_t there = lane < turns ? lower(i1 - base) : 0u, high = ~lower(keep - slot0 - base);
  uint32_t equal = lanes_before(__popc(same), &of_warp);
  equal += warps_before(of_warp, S.part[0], &total);
  if (ctas > 1) {
    if (tid == 0) S.count[0] = total;
    cluster_sync_all();
    for (int r = 0; r < rank; ++r) equal += ld_cluster_u32(remote(&S.count[0], r));
  }
  // of those equal to T the lowest `need` of the sequence
  if (keep == len) stay = there;
  else if (keep == 0) stay = 0u;
  else if (equal + __popc(same) <= need) stay |= same;
  else if (equal < need) stay |= same & lower(static_cast<int>(__fns(same, 0, static_cast<int>(need - equal) + 1)));
  // evicted slots, and movers in the upper half (a run has fewer than 2^16 slots)
  uint32_t both = lanes_before(__popc(there & ~stay) + (__popc(stay & high) << 16), &of_warp);
  both += warps_before(of_warp, S.part[1], &total);
  uint32_t gone = both & 0xffffu, moved = both >> 16;
  if (ctas > 1) {
    if (tid == 0) S.count[1] = total;
    cluster_sync_all();
    for (int r = 0; r < rank; ++r) {
      const uint32_t c = ld_cluster_u32(remote(&S.count[1], r));
      gone += c & 0xffffu;
      moved += c >> 16;
    }
  }
  // The r-th hole is the r-th evicted slot.  Its mover learns of it from shared memory (where the counts were), in a cluster from
  // the evicted list, which gets its positions once all have asked.
  uint32_t *holes = &S.hist[0][0], *source = &S.sum[0][0];  // (source: the slot that goes to a place, where rows are moved here)
  int32_t *ev = P.evicted_out + b * P.evicted_stride;
#pragma unroll 4
  for (int t = 0; t < turns; ++t) {
    const int i = i0 + 32 * t + lane, slot = slot0 + i;
    const uint32_t stay_t = __shfl_sync(0xffffffffu, stay, t), there_t = __shfl_sync(0xffffffffu, there, t), high_t = __shfl_sync(0xffffffffu, high, t);
    const uint32_t gone_t = __shfl_sync(0xffffffffu, gone, t), moved_t = __shfl_sync(0xffffffffu, moved, t);
    if (i < i1) {
      if ((stay_t >> lane) & 1u) {
        ev_keys[i] = slot < keep ? static_cast<uint32_t>(slot) : EV_MOVES | (moved_t + __popc(stay_t & high_t & before_me));
      } else {
        const uint32_t r = gone_t + __popc(there_t & ~stay_t & before_me);
        if (slot < keep && KVD_BOUNDS_OK(static_cast<int>(r) < len - keep, P.status)) {
          if (ctas > 1) ev[r] = slot;
          else holes[r] = static_cast<uint32_t>(slot);
        }
        ev_keys[i] = EV_GONE | r;
      }
    }
  }
  all_sync();
  // Kept slots.  In place nothing is overwritten that is still to be read: weights come from `keep` and above or go back to
  // where they are, the positions of the evicted are in shared memory.
  int32_t *so = P.slots_out + b * P.cap_out;
  for (int at = tid; at < n; at += EV_BATCH * EV_THREADS) {
    int dst[EV_BATCH];
    float x[EV_BATCH];
#pragma unroll
    for (int u = 0; u < EV_BATCH; ++u) {
      const int i = at + u * EV_THREADS;
      const uint32_t what = i < n ? ev_keys[i] : EV_GONE;
      const int r = static_cast<int>(what & ~(EV_MOVES | EV_GONE));
      dst[u] = static_cast<int>(what);  // (negative: gone)
      if ((what & (EV_GONE | EV_MOVES)) == EV_MOVES) dst[u] = !KVD_BOUNDS_OK(r < len - keep, P.status) ? keep : ctas > 1 ? __ldcg(ev + r) : static_cast<int>(holes[r]);
      if (i >= n) dst[u] = keep;
      x[u] = dst[u] >= 0 && i < n && P.weights_out && copy == 0 ? w[slot0 + i] : 0.f;
    }
#pragma unroll
    for (int u = 0; u < EV_BATCH; ++u) {
      const int i = at + u * EV_THREADS;
      if (copies > 1 && dst[u] >= 0 && dst[u] < keep) source[dst[u]] = static_cast<uint32_t>(i);
      if (copy != 0) continue;
      if (dst[u] < 0) {
        if (ctas == 1 && KVD_BOUNDS_OK((dst[u] & 0x7fffffff) < len - keep, P.status)) ev[dst[u] & 0x7fffffff] = ev_pos[i];
      } else if (dst[u] < keep) {
        so[dst[u]] = slot0 + i;
        if (P.positions_out) P.positions_out[b * P.cap_out + dst[u]] = ev_pos[i];
        if (P.weights_out) P.weights_out[b * P.cap_out + dst[u]] = x[u];
      }
    }
  }
  if (copies > 1) {
    // the rows: a warp for each, K and V, the CTAs of the sequence in turns
    __syncthreads();
    const uint4 *k = P.k + b * P.cap_in * P.row_in, *v = P.v + b * P.cap_in * P.row_in;
    uint4 *k_out = P.k_out + b * P.cap_out * P.row_out, *v_out = P.v_out + b * P.cap_out * P.row_out;
    for (int dst = copy + copies * warp; dst < keep; dst += copies * EV_WARPS) {
      const int src = static_cast<int>(source[dst]);
      if (P.k == P.k_out && src == dst) continue;
      if (!KVD_BOUNDS_OK(src >= 0 && src < len, P.status)) continue;
      for (int c0 = lane; c0 < P.row_chunks; c0 += 128) {
        uint4 x[2][4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (c0 + 32 * u < P.row_chunks) {
            x[0][u] = k[src * P.row_in + c0 + 32 * u];
            x[1][u] = v[src * P.row_in + c0 + 32 * u];
          }
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (c0 + 32 * u < P.row_chunks) {
            k_out[dst * P.row_out + c0 + 32 * u] = x[0][u];
            v_out[dst * P.row_out + c0 + 32 * u] = x[1][u];
          }
      }
    }
    return;
  }
  if (ctas == 1) return;
  cluster_sync_all();
#pragma unroll 4
  for (int i = tid; i < n; i += EV_THREADS) {
    const uint32_t what = ev_keys[i];
    if ((what & EV_GONE) && KVD_BOUNDS_OK(static_cast<int>(what & ~EV_GONE) < len - keep, P.status)) ev[what & ~EV_GONE] = ev_pos[i];
  }
}

// Rows of the kept keys to their slots, K and V: four 16-byte pieces of each in flight per thread.  Bound by memory: every
// kept row is read and written once (in place, only the movers').
__global__ void __launch_bounds__(EV_ROW_THREADS) kvd_evict_rows_kernel(const __grid_constant__ EvictParams P, int tiles) {
  grid_launch_dependents();
  grid_dependency_wait();
  const int b = static_cast<int>(blockIdx.x) / tiles, row0 = static_cast<int>(blockIdx.x) % tiles * P.rows_per_cta;
  const int kept = min(P.keep, P.len[b]), rows = min(P.rows_per_cta, kept - row0);
  if (rows <= 0) return;
  const int32_t *so = P.slots_out + b * P.cap_out + row0;
  const bool in_place = P.k == P.k_out;
  const uint4 *src_of[2] = {P.k + b * P.cap_in * P.row_in, P.v + b * P.cap_in * P.row_in};
  uint4 *dst_of[2] = {P.k_out + (b * P.cap_out + row0) * P.row_out, P.v_out + (b * P.cap_out + row0) * P.row_out};
  const int pieces = rows * P.row_chunks;
  for (int at = threadIdx.x; at < pieces; at += 4 * EV_ROW_THREADS) {
    uint4 x[2][4];
    long long to[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = at + u * EV_ROW_THREADS;
      to[u] = -1;
      if (i < pieces) {
        const int r = i / P.row_chunks, c = i % P.row_chunks, slot = so[r];
        if ((!in_place || slot != row0 + r) && KVD_BOUNDS_OK(slot >= 0 && slot < P.len[b], P.status)) {
          to[u] = r * P.row_out + c;
          x[0][u] = src_of[0][slot * P.row_in + c];
          x[1][u] = src_of[1][slot * P.row_in + c];
        }
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (to[u] >= 0) {
        dst_of[0][to[u]] = x[0][u];
        dst_of[1][to[u]] = x[1][u];
      }
  }
}

}  // namespace kvd

using namespace kvd;

static bool overlap(const void *a, size_t na, const void *b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}
// Rows of `width` bytes, `stride` apart.  Rows of one stride may lie between each other: keys and values as columns of one buffer.
struct EvictRows {
  const void *at;
  size_t rows, stride, width;
};
static bool overlap(const EvictRows &a, const EvictRows &b) {
  if (a.rows == 0 || b.rows == 0 || !overlap(a.at, (a.rows - 1) * a.stride + a.width, b.at, (b.rows - 1) * b.stride + b.width)) return false;
  if (a.stride != b.stride) return true;
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.at), y = reinterpret_cast<uintptr_t>(b.at);
  const size_t col = y >= x ? (y - x) % a.stride : (a.stride - (x - y) % a.stride) % a.stride;  // where b's columns begin in a's rows
  return col < a.width || col + b.width > a.stride;
}

extern "C" kvd_status kvd_cache_evict(kvd_ctx *ctx, int batch, const kvd_ranked_cache *in, const int32_t *lens, int keep, int32_t protect_below,
                                      const int32_t *protect_from, const kvd_ranked_cache *out, int32_t *slots_out, int32_t *evicted_out,
                                      int64_t evicted_stride, void *stream_) {
  if (!ctx || batch < 0 || keep < 0) return KVD_ERR_INVALID_ARG;
  if (batch == 0) return KVD_OK;
  if (!in || !out || !lens || !in->weights || !slots_out) return KVD_ERR_INVALID_ARG;
  const kvd_model_desc &d = ctx->desc;
  const int eb = ctx->dtype == KVD_DTYPE_F32 ? 4 : 2;
  const int64_t kdim = static_cast<int64_t>(d.n_kv_heads) * d.d_head;
  // rows are moved where there are rows: all four arrays, or none (the lists alone)
  const bool rows = in->k != nullptr;
  if ((in->v != nullptr) != rows || (out->k != nullptr) != rows || (out->v != nullptr) != rows) return KVD_ERR_INVALID_ARG;
  if (in->slots < 0 || out->slots < 0 || (out->positions && !in->positions && in->slots > INT32_MAX)) return KVD_ERR_INVALID_ARG;
  int max_len = 0, max_kept = 0, max_gone = 0;
  for (int b = 0; b < batch; ++b) {
    if (lens[b] < 0 || lens[b] > in->slots) return KVD_ERR_INVALID_ARG;
    const int kept = lens[b] < keep ? lens[b] : keep;
    max_len = lens[b] > max_len ? lens[b] : max_len;
    max_kept = kept > max_kept ? kept : max_kept;
    max_gone = lens[b] - kept > max_gone ? lens[b] - kept : max_gone;
  }
  if (max_len > KVD_MAX_EVICT_SLOTS || max_kept > out->slots || max_gone > evicted_stride) return KVD_ERR_CAPACITY;
  if (max_gone > 0 && !evicted_out) return KVD_ERR_INVALID_ARG;
  if (max_len == 0) return KVD_OK;
  if (!aligned4({in->weights, in->positions, out->weights, out->positions, slots_out, evicted_out})) return KVD_ERR_ALIGNMENT;
  if (rows) {
    if (in->row_stride < kdim || out->row_stride < kdim) return KVD_ERR_INVALID_ARG;
    const uintptr_t p = reinterpret_cast<uintptr_t>(in->k) | reinterpret_cast<uintptr_t>(in->v) | reinterpret_cast<uintptr_t>(out->k) | reinterpret_cast<uintptr_t>(out->v);
    if ((p & 15u) != 0 || in->row_stride * eb % 16 != 0 || out->row_stride * eb % 16 != 0) return KVD_ERR_ALIGNMENT;
    // in place: the same arrays with the same strides; otherwise nothing that is written may be read
    const size_t nin = static_cast<size_t>(batch - 1) * in->slots + max_len, nout = max_kept > 0 ? static_cast<size_t>(batch - 1) * out->slots + max_kept : 0;
    auto rows_of = [&](const void *p, const kvd_ranked_cache *c, size_t n) {
      return EvictRows{p, n, static_cast<size_t>(c->row_stride) * eb, static_cast<size_t>(kdim) * eb};
    };
    const EvictRows ik = rows_of(in->k, in, nin), iv = rows_of(in->v, in, nin), ok = rows_of(out->k, out, nout), ov = rows_of(out->v, out, nout);
    const bool same = in->k == out->k && in->v == out->v && in->row_stride == out->row_stride && in->slots == out->slots;
    if (!same && (overlap(ik, ok) || overlap(ik, ov) || overlap(iv, ok) || overlap(iv, ov))) return KVD_ERR_INVALID_ARG;
    if (overlap(ok, ov)) return KVD_ERR_INVALID_ARG;
  }
  const size_t win = (static_cast<size_t>(batch - 1) * in->slots + max_len) * 4, wout = (static_cast<size_t>(batch - 1) * out->slots + max_kept) * 4;
  if (out->weights && !(out->weights == in->weights && out->slots == in->slots) && overlap(in->weights, win, out->weights, wout)) return KVD_ERR_INVALID_ARG;
  if (out->positions && in->positions && !(out->positions == in->positions && out->slots == in->slots) && overlap(in->positions, win, out->positions, wout))
    return KVD_ERR_INVALID_ARG;
  cudaStream_t stream = static_cast<cudaStream_t>(stream_);
  // a cluster per sequence, of as many CTAs as its slots are worth
  int ctas = 1;
  while (ctas < EV_MAX_CTAS && max_len > ctas * EV_RUN) ctas *= 2;
  static thread_local EvictParams P;
  P.run = ((max_len + ctas - 1) / ctas + 3) / 4 * 4;
  const size_t smem = sizeof(EvictShared) + static_cast<size_t>(P.run) * 8;
  static std::atomic<bool> configured[64] = {};
  cudaError_t e = opt_in_smem(ctx, kvd_evict_select_kernel, sizeof(EvictShared) + EV_CTA_SLOTS * 8, configured);
  if (e != cudaSuccess) return cuda_fail(ctx, e, "cudaFuncSetAttribute(evict)");
  P.keep = keep;
  P.protect_below = protect_below;
  P.cap_in = in->slots;
  P.cap_out = out->slots;
  P.evicted_stride = evicted_stride;
  P.row_in = rows ? in->row_stride * eb / 16 : 0;
  P.row_out = rows ? out->row_stride * eb / 16 : 0;
  P.row_chunks = static_cast<int>(kdim * eb / 16);
  // Small caches: one launch instead of two, the selection made by every CTA of a cluster for itself, the rows shared out: as
  // long as a CTA's share is short, since a few CTAs' loads in flight are far from the memory's rate.  us, two launches / one,
  // three quarters kept: SmolLM2 layer 1 x 256 9.1 / 7.5, 1 x 1024 10.2 / 9.9, 1 x 2048 11.1 / 12.5, 8 x 1024 10.6 / 10.2, 40 x 256
  // 10.4 / 9.5, 40 x 1024 18.8 / 20.9, 8 x 3000 15.1 / 17.0; Qwen3-4B layer 8 x 256 9.8 / 9.4, 1 x 1024 9.9 / 16.2, 8 x 2048 26.0 / 27.4.
  int copies = 1;
  if (rows && max_len <= EV_SMALL)
    while (copies < EV_MAX_CTAS && 2 * copies * batch <= ctx->num_sms) copies *= 2;
  if (static_cast<int64_t>(max_kept) * kdim * eb * 2 > static_cast<int64_t>(copies) * EV_SMALL_BYTES) copies = 1;
  P.rows_per_cta = (4 * EV_ROW_THREADS + P.row_chunks - 1) / P.row_chunks;
  P.status = ctx->d_status;
  for (int b0 = 0; b0 < batch; b0 += EV_MAX_SEQS) {
    const int nb = batch - b0 < EV_MAX_SEQS ? batch - b0 : EV_MAX_SEQS;
    for (int i = 0; i < nb; ++i) {
      P.len[i] = lens[b0 + i];
      P.protect_from[i] = protect_from ? protect_from[b0 + i] : INT32_MAX;
    }
    P.weights = in->weights + static_cast<size_t>(b0) * in->slots;
    P.positions = in->positions ? in->positions + static_cast<size_t>(b0) * in->slots : nullptr;
    P.weights_out = out->weights ? out->weights + static_cast<size_t>(b0) * out->slots : nullptr;
    P.positions_out = out->positions ? out->positions + static_cast<size_t>(b0) * out->slots : nullptr;
    P.slots_out = slots_out + static_cast<size_t>(b0) * out->slots;
    P.evicted_out = evicted_out ? evicted_out + static_cast<size_t>(b0) * evicted_stride : nullptr;
    P.k = rows ? static_cast<const uint4 *>(in->k) + static_cast<size_t>(b0) * in->slots * P.row_in : nullptr;
    P.v = rows ? static_cast<const uint4 *>(in->v) + static_cast<size_t>(b0) * in->slots * P.row_in : nullptr;
    P.k_out = rows ? static_cast<uint4 *>(out->k) + static_cast<size_t>(b0) * out->slots * P.row_out : nullptr;
    P.v_out = rows ? static_cast<uint4 *>(out->v) + static_cast<size_t>(b0) * out->slots * P.row_out : nullptr;
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cudaLaunchAttribute attr[2];
    cfg.stream = stream;
    cfg.gridDim = dim3(nb * ctas * copies, 1, 1);
    cfg.blockDim = dim3(EV_THREADS, 1, 1);
    cfg.dynamicSmemBytes = smem;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = (serial_launch_mask() & 8) || 2 * nb * ctas > ctx->num_sms ? 0 : 1;  // (as launch_dependent)
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ctas * copies;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = ctas * copies > 1 ? 2 : 1;
    e = cudaLaunchKernelEx(&cfg, kvd_evict_select_kernel, P, ctas, copies);
    if (e != cudaSuccess) return cuda_fail(ctx, e, "launch evict (select)");
    ctx->launches += 1;
    if (!rows || max_kept == 0 || copies > 1) continue;
    const int tiles = (max_kept + P.rows_per_cta - 1) / P.rows_per_cta;
    cfg.gridDim = dim3(nb * tiles, 1, 1);
    cfg.blockDim = dim3(EV_ROW_THREADS, 1, 1);
    cfg.dynamicSmemBytes = 0;
    attr[0].val.programmaticStreamSerializationAllowed = serial_launch_mask() & 8 ? 0 : 1;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, kvd_evict_rows_kernel, P, tiles);
    if (e != cudaSuccess) return cuda_fail(ctx, e, "launch evict (rows)");
    ctx->launches += 1;
  }
  return KVD_OK;
}
