// Attention weights of a prompt's keys (include/kvd.h, kvd_prefill_attention_weights): w_j = sum over rows r of 2^(s_rj - z_r),
// z_r = log2 of the row's sum of 2^s (Eq. 6 in base 2), over the query rows of every head.  A row's statistic needs all of
// its scores, a key's weight the statistics of all its rows, so the scores are computed twice, on tcgen05.mma with fp32 sums
// in tensor memory, rather than kept (4 bytes per score and pass against d_head multiply-adds that take less time):
//
//   rows     S = Q K^T, 128 query rows x 128 keys: a thread has a row in its tensor-memory lane, and the row's reference
//            and sum in registers.  The query tile is the A operand in tensor memory, key tiles stream through shared memory.
//   columns  S^T = K Q^T, 128 keys x 128 query rows: a thread has a key, and adds up its weights in registers; the rows'
//            statistics come from shared memory, the same word for all lanes.  The query tile stays in shared memory as the B
//            operand while key tiles stream past it as A.  Sums of a tile's keys go to shared memory, one owner per word.
//   sum      partial columns of all KV heads and row ranges, added in a fixed order, to the weights so far.
//
// A row tile is 128 of the n_rows * G (token, head of the group) rows of a KV head; key tiles are aligned to absolute
// position.  In both passes eight warps in two groups take turns on the tiles, so that one group's exponentials cover the
// other's way to tensor memory and back; two warps gather keys from the segments with cp.async, one thread issues products.
// Every wait is bounded, as in the other tensor-core kernels.
#include <math_constants.h>
#include <string.h>

#include <type_traits>

#include "kvd_internal.h"
#include "kvd_ptx.cuh"

namespace kvd {

constexpr int PW_ROWS = 128;      // query rows per tile
constexpr int PW_KEYS = 128;      // keys per tile
constexpr int PW_LOADERS = 64;    // threads of warps 9 and 10
constexpr int PW_THREADS = 352;   // warps 0-7 exponentials, 8 products, 9 and 10 loads (168 registers a thread)
constexpr int PW_LAG = 2;         // tiles a loader thread keeps in flight behind the one it is issuing
constexpr int PW_RANGE = 64;      // row tiles one CTA of the columns pass can take
constexpr int PW_CHUNK = 8;       // key tiles of one (sums in shared memory)

struct PwParams {
  const __nv_bfloat16 *q;  // [n_rows][n_q][d_head]
  const int32_t *q_pos;    // DEVICE [n_rows]
  int n_rows, n_q, n_kv, window;
  float scale_log2e;
  int seg_lo, seg_hi;      // first and last position any segment holds
  const __nv_bfloat16 *k[KVD_MAX_SEGMENTS];
  long long stride[KVD_MAX_SEGMENTS];
  int first[KVD_MAX_SEGMENTS];
  int len[KVD_MAX_SEGMENTS];
  int rows, row_tiles;     // of a KV head
  int splits;              // rows pass: shares of a row tile's keys
  float2 *ml;              // [splits][n_kv][row_tiles * 128]: reference and sum
  float *neg_lse;          // [n_kv][row_tiles * 128]: -(m + log2 l); minus infinity: the row adds nothing
  int key_tile0, key_tiles, chunk, chunks, range, ranges;  // columns pass: key tiles per CTA, row tiles per CTA
  float *cols;             // [ranges][n_kv][key_tiles * 128]
  const float *in;
  float *out;
  int n_positions;
  int *status;
  unsigned long long timeout_ns;
};

template <int D_HEAD, bool COLUMNS>
struct PwCfg {
  static constexpr int TILE_BYTES = PW_KEYS * D_HEAD * 2;
  static constexpr int SLAB = PW_KEYS * 128;                   // 64 channels of a tile
  static constexpr int Q_SLOTS = COLUMNS ? (D_HEAD == 256 ? 1 : 2) : 0;
  static constexpr int SLOTS = D_HEAD == 256 ? (COLUMNS ? 2 : 3) : D_HEAD == 128 ? (COLUMNS ? 4 : 6) : 8;  // key tiles in the ring
  static constexpr int S_BUFS = COLUMNS ? 4 : 3;
  static constexpr int COL_S = 0, COL_Q = S_BUFS * PW_KEYS;    // rows: the query tile behind the scores, two elements per column
  static constexpr int COLS = 512;
  static_assert(COL_Q + (COLUMNS ? 0 : D_HEAD / 2) <= COLS, "tensor memory");
  static constexpr int N_BARS = 2 * SLOTS + 2 * S_BUFS + 10;
  static constexpr int SMEM_BYTES = 1024 + (SLOTS + Q_SLOTS) * TILE_BYTES + N_BARS * 8;
};

__device__ __forceinline__ bool pw_wait(uint32_t bar, uint32_t parity, const volatile int *abort_flag, unsigned long long timeout_ns) {
  if (mbar_try_wait(bar, parity)) return true;
  const unsigned long long t0 = globaltimer_ns();
  uint32_t it = 0;
  while (!mbar_try_wait(bar, parity)) {
    __nanosleep(20);
    if (((++it) & 31u) == 0u && (*abort_flag != 0 || globaltimer_ns() - t0 > timeout_ns)) return false;
  }
  return true;
}
__device__ __forceinline__ bool pw_warp_wait(uint32_t bar, uint32_t parity, const volatile int *abort_flag, unsigned long long timeout_ns, int lane) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  int ok = 1;
  if (lane == 0) ok = pw_wait(bar, parity, abort_flag, timeout_ns) ? 1 : 0;
  ok = __shfl_sync(0xffffffffu, ok, 0);
  __syncwarp();
  return ok != 0;
}

// Whether one segment holds all of n positions from pos on.
__device__ __forceinline__ bool pw_held(const PwParams &P, int pos, int n) {
  bool held = false;
#pragma unroll
  for (int sg = 0; sg < KVD_MAX_SEGMENTS; ++sg) held |= segment_holds(P.first[sg], P.len[sg], pos, n);
  return held;
}

// The keys that rows [row0, row0 + 128) can see, as key tiles (first, count); a warp's lanes go through the tokens.  Returns the
// smallest and the largest position of the rows' tokens as well.
template <int G>
__device__ __forceinline__ void pw_tile_range(const PwParams &P, int row0, int lane, int &tile, int &count, int &qmin, int &qmax) {
  const int tok0 = row0 / G, tok1 = min(P.n_rows - 1, (row0 + PW_ROWS - 1) / G);
  int lo = INT_MAX, hi = -1;
  qmin = INT_MAX;
  qmax = -1;
  for (int t = tok0 + lane; t <= tok1; t += 32) {
    const int qp = max(P.q_pos[t], -1);
    qmin = min(qmin, qp);
    qmax = max(qmax, qp);
    const int l = max(first_visible(qp, P.window), P.seg_lo), h = min(qp, P.seg_hi);
    if (h >= l) {
      lo = min(lo, l);
      hi = max(hi, h);
    }
  }
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  qmin = __reduce_min_sync(0xffffffffu, qmin);
  qmax = __reduce_max_sync(0xffffffffu, qmax);
  if (row0 + PW_ROWS > P.rows) qmin = -1;  // rows that are not there see nothing
  tile = hi >= 0 ? lo / PW_KEYS : 0;
  count = hi >= 0 ? hi / PW_KEYS - tile + 1 : 0;
}

// A loader thread's tiles: issued in order, published to the waiting roles once PW_LAG younger ones have been issued -- or
// all at once when the next would have to wait for a free slot.
struct PwFlight {
  uint32_t pend[PW_LAG + 1] = {};
  int n = 0;
  __device__ __forceinline__ void publish_all(int lane) {
    cp_async_wait_all();
    fence_proxy_async_smem();
    __syncwarp();
#pragma unroll
    for (int i = 0; i <= PW_LAG; ++i)
      if (i < n && lane == 0) mbar_arrive(pend[i]);
    n = 0;
  }
  __device__ __forceinline__ void issued(uint32_t bar, int lane) {
    cp_async_commit();
#pragma unroll
    for (int i = 0; i <= PW_LAG; ++i)
      if (i == n) pend[i] = bar;
    if (++n > PW_LAG) {
      cp_async_wait_group<PW_LAG>();
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(pend[0]);
#pragma unroll
      for (int i = 0; i < PW_LAG; ++i) pend[i] = pend[i + 1];
      --n;
    }
  }
  // the slot's last reader is done (parity of that phase); false: gave up
  __device__ __forceinline__ bool free_slot(uint32_t bar, uint32_t parity, int lane, const volatile int *s_abort, unsigned long long tmo) {
    int free_now = lane == 0 ? (mbar_try_wait(bar, parity) ? 1 : 0) : 0;
    if (__shfl_sync(0xffffffffu, free_now, 0)) return true;
    publish_all(lane);
    int got = lane == 0 ? (pw_wait(bar, parity, s_abort, tmo) ? 1 : 0) : 0;
    return __shfl_sync(0xffffffffu, got, 0) != 0;
  }
};
// 128 keys from position pos0 on into a tile at `base`: rows of 128 bytes per 64 channels, 128-byte swizzle; what no segment
// holds reads as zeros.
template <int D_HEAD>
__device__ __forceinline__ void pw_load_keys(const PwParams &P, uint32_t base, int pos0, int kvh, int ptid) {
  constexpr int CPR = D_HEAD / 8, RSTEP = PW_LOADERS / CPR, SLAB = PW_KEYS * 128;
  const int c = ptid % CPR, r0 = ptid / CPR;
  const uint32_t dst = base + static_cast<uint32_t>(c >> 3) * SLAB;
  const long long el = static_cast<long long>(kvh) * D_HEAD + c * 8;
  int whole = -1;
#pragma unroll
  for (int sg = 0; sg < KVD_MAX_SEGMENTS; ++sg)
    if (segment_holds(P.first[sg], P.len[sg], pos0, PW_KEYS)) whole = sg;
  if (whole >= 0) {
    const long long stride = P.stride[whole];
    const __nv_bfloat16 *src = P.k[whole] + static_cast<long long>(pos0 - P.first[whole] + r0) * stride + el;
#pragma unroll
    for (int pass = 0; pass < PW_KEYS / RSTEP; ++pass) {
      const int r = r0 + pass * RSTEP;
      cp_async16(dst + r * 128 + (((c & 7) ^ (r & 7)) << 4), src, true);
      src += RSTEP * stride;
    }
  } else {
#pragma unroll 1
    for (int pass = 0; pass < PW_KEYS / RSTEP; ++pass) {
      const int r = r0 + pass * RSTEP, pos = pos0 + r;
      const __nv_bfloat16 *src = P.q;
      bool have = false;
#pragma unroll
      for (int sg = 0; sg < KVD_MAX_SEGMENTS; ++sg)
        if (segment_holds(P.first[sg], P.len[sg], pos, 1)) {
          src = P.k[sg] + static_cast<long long>(pos - P.first[sg]) * P.stride[sg] + el;
          have = true;
        }
      cp_async16(dst + r * 128 + (((c & 7) ^ (r & 7)) << 4), src, have);
    }
  }
}
// Query row `row` of a KV head: element offset.
template <int D_HEAD, int G>
__device__ __forceinline__ long long pw_row(const PwParams &P, int row, int kvh) {
  return (static_cast<long long>(row / G) * P.n_q + kvh * G + row % G) * D_HEAD;
}

__device__ __forceinline__ float pw_max64(const uint32_t (&s0)[32], const uint32_t (&s1)[32]) {
  float mx[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
  for (int k = 0; k < 32; k += 4) {
    mx[0] = fmax3(mx[0], __uint_as_float(s0[k]), __uint_as_float(s0[k + 1]));
    mx[1] = fmax3(mx[1], __uint_as_float(s0[k + 2]), __uint_as_float(s0[k + 3]));
    mx[2] = fmax3(mx[2], __uint_as_float(s1[k]), __uint_as_float(s1[k + 1]));
    mx[3] = fmax3(mx[3], __uint_as_float(s1[k + 2]), __uint_as_float(s1[k + 3]));
  }
  return fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
}
// Sum of 2^(s * scale - m) over 64 scores, in four chains.
__device__ __forceinline__ float pw_sum64(const uint32_t (&s0)[32], const uint32_t (&s1)[32], uint64_t c2, uint64_t nm2) {
  const uint64_t one2 = pack2(1.0f, 1.0f);
  uint64_t l2[2] = {0ull, 0ull};
#pragma unroll
  for (int k = 0; k < 32; k += 2) {
    float e0, e1, e2, e3;
    unpack2(ffma2(pack2(__uint_as_float(s0[k]), __uint_as_float(s0[k + 1])), c2, nm2), e0, e1);
    unpack2(ffma2(pack2(__uint_as_float(s1[k]), __uint_as_float(s1[k + 1])), c2, nm2), e2, e3);
    l2[0] = ffma2(pack2(ex2_approx(e0), ex2_approx(e1)), one2, l2[0]);
    l2[1] = ffma2(pack2(ex2_approx(e2), ex2_approx(e3)), one2, l2[1]);
  }
  float a0, a1, a2, a3;
  unpack2(l2[0], a0, a1);
  unpack2(l2[1], a2, a3);
  return (a0 + a1) + (a2 + a3);
}

template <int D_HEAD, int G, int DT, bool COLUMNS>
__global__ void __launch_bounds__(PW_THREADS, 1) kvd_prefill_weights_kernel(const __grid_constant__ PwParams P) {
  using Cfg = PwCfg<D_HEAD, COLUMNS>;
  constexpr int SLOTS = Cfg::SLOTS, S_BUFS = Cfg::S_BUFS, Q_SLOTS = Cfg::Q_SLOTS;
  extern __shared__ uint8_t pw_smem_raw[];
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort_i;
  __shared__ int s_tile[PW_RANGE], s_count[PW_RANGE], s_qmin[PW_RANGE], s_qmax[PW_RANGE];  // per row tile of the CTA
  __shared__ float s_m[2][PW_ROWS], s_l[2][PW_ROWS];                   // rows: both groups' statistics
  __shared__ __align__(16) float s_nl[2][PW_ROWS];                     // columns: the rows' statistics and positions
  __shared__ __align__(16) int s_qp[2][PW_ROWS];
  __shared__ float s_sum[COLUMNS ? 2 : 1][COLUMNS ? PW_CHUNK * PW_KEYS : 1];
  volatile int *s_abort = &s_abort_i;
  const uint32_t ring = (smem_u32(pw_smem_raw) + 1023u) & ~1023u;  // the swizzle is a function of the address
  const uint32_t q_smem = ring + SLOTS * Cfg::TILE_BYTES;
  const uint32_t bar_base = q_smem + Q_SLOTS * Cfg::TILE_BYTES;
  auto bar_full = [&](int s) { return bar_base + 8u * s; };                          // a key tile has landed
  auto bar_empty = [&](int s) { return bar_base + 8u * (SLOTS + s); };               // its product is done
  auto bar_s_full = [&](int b) { return bar_base + 8u * (2 * SLOTS + b); };          // scores of a tile
  auto bar_s_free = [&](int b) { return bar_base + 8u * (2 * SLOTS + S_BUFS + b); };  // ... have been read
  const uint32_t bar_q = bar_base + 8u * (2 * SLOTS + 2 * S_BUFS);
  auto bar_q_full = [&](int s) { return bar_q + 8u * s; };                           // a query tile is in place
  auto bar_q_empty = [&](int s) { return bar_q + 8u * (2 + s); };                    // its products are done
  auto bar_nl_full = [&](int s) { return bar_q + 8u * (4 + s); };                    // statistics of a query tile's rows
  auto bar_nl_free = [&](int s) { return bar_q + 8u * (6 + s); };
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const unsigned long long tmo = P.timeout_ns;
  // ---- this CTA's work: long ones (late rows of a causal call, early keys) start first
  int kvh, tile0, n_tiles, part;  // row tiles [tile0, tile0 + n_tiles)
  int kt_lo = 0, kt_hi = INT_MAX;  // of its keys, the tiles it may take
  if constexpr (COLUMNS) {
    int at = static_cast<int>(blockIdx.x);
    kvh = at % P.n_kv;
    at /= P.n_kv;
    part = P.ranges - 1 - at % P.ranges;
    kt_lo = P.key_tile0 + at / P.ranges * P.chunk;
    kt_hi = min(P.key_tile0 + P.key_tiles, kt_lo + P.chunk);
    tile0 = part * P.range;
    n_tiles = min(P.range, P.row_tiles - tile0);
  } else {
    int at = static_cast<int>(blockIdx.x);
    part = at % P.splits;
    at /= P.splits;
    kvh = at % P.n_kv;
    tile0 = P.row_tiles - 1 - at / P.n_kv;
    n_tiles = 1;
  }
  if (tid == 0) {
    for (int s = 0; s < SLOTS; ++s) {
      mbar_init(bar_full(s), PW_LOADERS / 32);
      mbar_init(bar_empty(s), 1);
    }
    for (int b = 0; b < S_BUFS; ++b) {
      mbar_init(bar_s_full(b), 1);
      mbar_init(bar_s_free(b), 4);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(bar_q_full(s), COLUMNS ? PW_LOADERS / 32 : 8);
      mbar_init(bar_q_empty(s), 1);
      mbar_init(bar_nl_full(s), PW_LOADERS / 32);
      mbar_init(bar_nl_free(s), 8);
    }
    fence_mbar_init();
    s_abort_i = 0;
  }
  if (warp == 8) {
    tmem_claim(smem_u32(&s_tmem), Cfg::COLS);
  }
  __syncthreads();
  grid_launch_dependents();
  grid_dependency_wait();
  for (int i = warp; i < n_tiles; i += PW_THREADS / 32) {
    int t, n, qmin, qmax;
    pw_tile_range<G>(P, (tile0 + i) * PW_ROWS, lane, t, n, qmin, qmax);
    if constexpr (COLUMNS) {
      const int a = max(t, kt_lo), b = min(t + n, kt_hi);
      t = a;
      n = b > a ? b - a : 0;
    } else {
      // the split's share of the tiles
      const int a = static_cast<int>(static_cast<long long>(n) * part / P.splits), b = static_cast<int>(static_cast<long long>(n) * (part + 1) / P.splits);
      t += a;
      n = b - a;
    }
    if (lane == 0) {
      s_tile[i] = t;
      s_count[i] = n;
      s_qmin[i] = qmin;
      s_qmax[i] = qmax;
    }
  }
  if constexpr (COLUMNS)
    for (int i = tid; i < 2 * PW_CHUNK * PW_KEYS; i += PW_THREADS) (&s_sum[0][0])[i] = 0.f;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = s_tmem;

  if (warp < 8) {
    // ------------------------------------------------------------------ exponentials
    const int wg = warp >> 2, q4 = warp & 3, row = q4 * 32 + lane;
    const uint32_t lane_field = static_cast<uint32_t>(q4 * 32) << 16;
    const uint64_t c2 = pack2(P.scale_log2e, P.scale_log2e);
    bool ok = true;
    if constexpr (!COLUMNS) {
      const int r = tile0 * PW_ROWS + row, n_blk = s_count[0], t0 = s_tile[0];
      const bool valid = r < P.rows;
      const int qp = valid ? max(P.q_pos[r / G], -1) : -1, lo = first_visible(qp, P.window);
      if (n_blk > 0) {
        // the query row into tensor memory: element pairs (2c, 2c + 1) -> column c (zeros for padding rows)
        const uint4 *qsrc = reinterpret_cast<const uint4 *>(P.q + (valid ? pw_row<D_HEAD, G>(P, r, kvh) : 0));
#pragma unroll 1
        for (int c = wg; c < D_HEAD / 64; c += 2) {
          uint32_t x[32];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const uint4 w = valid ? qsrc[c * 8 + i] : make_uint4(0u, 0u, 0u, 0u);
            x[4 * i] = w.x;
            x[4 * i + 1] = w.y;
            x[4 * i + 2] = w.z;
            x[4 * i + 3] = w.w;
          }
          tmem_st_x32(tmem_base + lane_field + Cfg::COL_Q + c * 32, x);
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_q_full(0));
      }
      // range that every stored row of the warp sees
      const int all_lo = __reduce_max_sync(0xffffffffu, valid ? lo : INT_MIN), all_hi = __reduce_min_sync(0xffffffffu, valid ? qp : INT_MAX);
      // The reference m is the first finite maximum the row meets, rounded up to a whole number, and moves only if a sum
      // threatens to leave fp32's range: 2^(s - m) is as exact for any m.
      float m = -CUDART_INF_F, l = 0.f;
      for (int j = wg; j < n_blk; j += 2) {
        const int buf = j % S_BUFS, pos0 = (t0 + j) * PW_KEYS;
        if (!pw_warp_wait(bar_s_full(buf), (j / S_BUFS) & 1, s_abort, tmo, lane)) {
          raise(P.status, STATUS_TIMEOUT, s_abort);
          ok = false;
          break;
        }
        tc_fence_after();
        const bool whole = pos0 >= all_lo && pos0 + PW_KEYS - 1 <= all_hi && pw_held(P, pos0, PW_KEYS);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          uint32_t s0[32], s1[32];
          tmem_ld_x32(tmem_base + lane_field + Cfg::COL_S + buf * PW_KEYS + half * 64, s0);
          tmem_ld_x32(tmem_base + lane_field + Cfg::COL_S + buf * PW_KEYS + half * 64 + 32, s1);
          unsigned long long vis = ~0ull;
          if (!whole) {
            vis = 0ull;
#pragma unroll
            for (int sg = 0; sg < KVD_MAX_SEGMENTS; ++sg) vis |= segment_slots(P.first[sg], P.len[sg], pos0 + half * 64);
            vis &= visible_slots(lo, qp, pos0 + half * 64);
          }
          tmem_wait_ld();
          if (half == 1) {  // the scores are in registers: their columns may take another tile
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_s_free(buf));
          }
          if (!whole) {
            const uint32_t v0 = static_cast<uint32_t>(vis), v1 = static_cast<uint32_t>(vis >> 32);
#pragma unroll
            for (int k = 0; k < 32; ++k) {
              if (!((v0 >> k) & 1u)) s0[k] = 0xff800000u;  // -inf
              if (!((v1 >> k) & 1u)) s1[k] = 0xff800000u;
            }
          }
          if (__any_sync(0xffffffffu, m == -CUDART_INF_F)) {
            const float bm = ceilf(pw_max64(s0, s1) * P.scale_log2e);
            if (m == -CUDART_INF_F) m = bm;
          }
          float mu = m == -CUDART_INF_F ? 0.f : m;
          float sum = pw_sum64(s0, s1, c2, pack2(-mu, -mu));
          if (__any_sync(0xffffffffu, !(sum < 1e30f))) {  // (a NaN among them)
            const float bm = ceilf(pw_max64(s0, s1) * P.scale_log2e);
            if (bm > m) {
              l *= ex2_approx(m - bm);
              m = bm;
              mu = bm;
            }
            sum = pw_sum64(s0, s1, c2, pack2(-mu, -mu));
          }
          l += sum;
        }
      }
      // ---- both groups' parts, referred to the larger reference
      if (ok) {
        s_m[wg][row] = m;
        s_l[wg][row] = l;
      }
    } else {
      int j0 = 0;  // tiles before this row tile's
      for (int i = 0; ok && i < n_tiles; ++i) {
        const int n_blk = s_count[i];
        if (n_blk == 0) continue;
        const int t0 = s_tile[i], slot = i & 1;
        const int qmin = s_qmin[i], qmax = s_qmax[i];
        int used = 0;  // earlier row tiles with this parity
        for (int k = slot; k < i; k += 2) used += s_count[k] > 0;
        if (!pw_warp_wait(bar_nl_full(slot), used & 1, s_abort, tmo, lane)) {
          raise(P.status, STATUS_TIMEOUT, s_abort);
          ok = false;
          break;
        }
        for (int jj = (j0 & 1) ^ wg; jj < n_blk; jj += 2) {
          const int j = j0 + jj, buf = j % S_BUFS, pos0 = (t0 + jj) * PW_KEYS, kp = pos0 + row;
          if (!pw_warp_wait(bar_s_full(buf), (j / S_BUFS) & 1, s_abort, tmo, lane)) {
            raise(P.status, STATUS_TIMEOUT, s_abort);
            ok = false;
            break;
          }
          tc_fence_after();
          const bool whole = pos0 + PW_KEYS - 1 <= qmin && (P.window <= 0 || qmax - pos0 < P.window);
          const uint32_t window = P.window > 0 ? static_cast<uint32_t>(P.window) : 0x80000000u;
          uint64_t acc[2] = {0ull, 0ull};
#pragma unroll
          for (int quarter = 0; quarter < 4; ++quarter) {
            uint32_t s[32];
            tmem_ld_x32(tmem_base + lane_field + Cfg::COL_S + buf * PW_ROWS + quarter * 32, s);
            tmem_wait_ld();
            if (quarter == 3) {
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(bar_s_free(buf));
            }
            const uint64_t one2 = pack2(1.0f, 1.0f);
#pragma unroll
            for (int k = 0; k < 32; k += 4) {
              const float4 nl = *reinterpret_cast<const float4 *>(&s_nl[slot][quarter * 32 + k]);
              float e0, e1, e2, e3;
              unpack2(ffma2(pack2(__uint_as_float(s[k]), __uint_as_float(s[k + 1])), c2, pack2(nl.x, nl.y)), e0, e1);
              unpack2(ffma2(pack2(__uint_as_float(s[k + 2]), __uint_as_float(s[k + 3])), c2, pack2(nl.z, nl.w)), e2, e3);
              float p0 = ex2_approx(e0), p1 = ex2_approx(e1), p2 = ex2_approx(e2), p3 = ex2_approx(e3);
              if (!whole) {
                const int4 qp = *reinterpret_cast<const int4 *>(&s_qp[slot][quarter * 32 + k]);
                p0 = static_cast<uint32_t>(qp.x - kp) < window ? p0 : 0.f;
                p1 = static_cast<uint32_t>(qp.y - kp) < window ? p1 : 0.f;
                p2 = static_cast<uint32_t>(qp.z - kp) < window ? p2 : 0.f;
                p3 = static_cast<uint32_t>(qp.w - kp) < window ? p3 : 0.f;
              }
              acc[0] = ffma2(pack2(p0, p1), one2, acc[0]);
              acc[1] = ffma2(pack2(p2, p3), one2, acc[1]);
            }
          }
          float a0, a1, a2, a3;
          unpack2(acc[0], a0, a1);
          unpack2(acc[1], a2, a3);
          s_sum[wg][(t0 + jj - kt_lo) * PW_KEYS + row] += (a0 + a1) + (a2 + a3);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_nl_free(slot));
        j0 += n_blk;
      }
    }
  } else if (warp == 8) {
    // ------------------------------------------------------------------ products (one thread)
    constexpr uint32_t IDESC = DT == 0 ? umma_idesc_bf16_f32(128, 128) : umma_idesc_f16_f32(128, 128);
    if (lane == 0) {
      bool ok = true;
      int j = 0, tiles_used[2] = {0, 0}, nth = 0;
      for (int i = 0; ok && i < n_tiles; ++i) {
        const int n_blk = s_count[i];
        if (n_blk == 0) continue;
        const int qs = Q_SLOTS == 2 ? (nth & 1) : 0;
        ++nth;
        if (!pw_wait(bar_q_full(qs), tiles_used[qs] & 1, s_abort, tmo)) {
          ok = false;
          break;
        }
        tiles_used[qs] += 1;
        tc_fence_after();
        for (int jj = 0; jj < n_blk; ++jj, ++j) {
          const int slot = j % SLOTS, buf = j % S_BUFS;
          if (!pw_wait(bar_full(slot), (j / SLOTS) & 1, s_abort, tmo) || (j >= S_BUFS && !pw_wait(bar_s_free(buf), (j / S_BUFS - 1) & 1, s_abort, tmo))) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t d = tmem_base + Cfg::COL_S + buf * PW_KEYS;
          const uint64_t kdesc = umma_smem_desc_sw128(ring + slot * Cfg::TILE_BYTES), qdesc = umma_smem_desc_sw128(q_smem + qs * Cfg::TILE_BYTES);
#pragma unroll
          for (int ks = 0; ks < D_HEAD / 16; ++ks) {
            const uint64_t off = ((ks >> 2) * Cfg::SLAB + (ks & 3) * 32) >> 4;
            if constexpr (COLUMNS) umma_bf16(d, kdesc + off, qdesc + off, IDESC, ks > 0 ? 1u : 0u);
            else umma_f16_ts(d, tmem_base + Cfg::COL_Q + ks * 8, kdesc + off, IDESC, ks > 0 ? 1u : 0u);
          }
          umma_commit(bar_empty(slot));
          umma_commit(bar_s_full(buf));
        }
        if (COLUMNS && ok) umma_commit(bar_q_empty(qs));
      }
      if (!ok) raise(P.status, STATUS_TIMEOUT, s_abort);
    }
  } else {
    // ------------------------------------------------------------------ loads
    const int ptid = tid - 9 * 32;
    PwFlight fly;
    bool ok = true;
    int j = 0, used[2] = {0, 0}, nl_used[2] = {0, 0}, nth = 0;
    for (int i = 0; ok && i < n_tiles; ++i) {
      const int n_blk = s_count[i], t0 = s_tile[i];
      if (n_blk == 0) continue;
      if constexpr (COLUMNS) {
        const int qs = Q_SLOTS == 2 ? (nth & 1) : 0, row0 = (tile0 + i) * PW_ROWS;
        ++nth;
        if (used[qs] > 0) ok = fly.free_slot(bar_q_empty(qs), (used[qs] - 1) & 1, lane, s_abort, tmo);
        if (!ok) break;
        used[qs] += 1;
        constexpr int CPR = D_HEAD / 8, RSTEP = PW_LOADERS / CPR;
        const int c = ptid % CPR, r0 = ptid / CPR;
        const uint32_t dst = q_smem + qs * Cfg::TILE_BYTES + static_cast<uint32_t>(c >> 3) * Cfg::SLAB;
#pragma unroll 4
        for (int pass = 0; pass < PW_ROWS / RSTEP; ++pass) {
          const int r = r0 + pass * RSTEP;
          const bool have = row0 + r < P.rows;
          cp_async16(dst + r * 128 + (((c & 7) ^ (r & 7)) << 4), P.q + (have ? pw_row<D_HEAD, G>(P, row0 + r, kvh) + c * 8 : 0), have);
        }
        fly.issued(bar_q_full(qs), lane);
        // the rows' statistics and positions
        const int ns = i & 1;
        if (nl_used[ns] > 0) ok = fly.free_slot(bar_nl_free(ns), (nl_used[ns] - 1) & 1, lane, s_abort, tmo);
        if (!ok) break;
        nl_used[ns] += 1;
        const int r = row0 + ptid;
        for (int o = 0; o < PW_ROWS; o += PW_LOADERS) {
          s_nl[ns][ptid + o] = r + o < P.rows ? P.neg_lse[static_cast<long long>(kvh) * P.row_tiles * PW_ROWS + r + o] : -CUDART_INF_F;
          s_qp[ns][ptid + o] = r + o < P.rows ? max(P.q_pos[(r + o) / G], -1) : -1;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_nl_full(ns));
      }
      for (int jj = 0; jj < n_blk; ++jj, ++j) {
        const int slot = j % SLOTS;
        if (j >= SLOTS) ok = fly.free_slot(bar_empty(slot), (j / SLOTS - 1) & 1, lane, s_abort, tmo);
        if (!ok) break;
        pw_load_keys<D_HEAD>(P, ring + slot * Cfg::TILE_BYTES, (t0 + jj) * PW_KEYS, kvh, ptid);
        fly.issued(bar_full(slot), lane);
      }
    }
    if (ok) {
      fly.publish_all(lane);
    } else {
      cp_async_wait_all();
      raise(P.status, STATUS_TIMEOUT, s_abort);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 8) {
    tc_fence_after();
    tmem_dealloc(tmem_base, Cfg::COLS);
  }
  if constexpr (COLUMNS) {
    // (also the sums of a CTA that gave up: the status word says so)
    float *dst = P.cols + (static_cast<long long>(part) * P.n_kv + kvh) * P.key_tiles * PW_KEYS + (kt_lo - P.key_tile0) * PW_KEYS;
    for (int i = tid; i < (kt_hi - kt_lo) * PW_KEYS; i += PW_THREADS) dst[i] = pw_held(P, kt_lo * PW_KEYS + i, 1) ? s_sum[0][i] + s_sum[1][i] : 0.f;
  } else if (tid < PW_ROWS) {
    const float m0 = s_m[0][tid], m1 = s_m[1][tid], m = fmaxf(m0, m1), mu = m == -CUDART_INF_F ? 0.f : m;
    const bool none = s_count[0] == 0;
    const float l = none ? 0.f : s_l[0][tid] * ex2_approx(m0 - mu) + s_l[1][tid] * ex2_approx(m1 - mu);
    const long long at = static_cast<long long>(kvh) * P.row_tiles * PW_ROWS + tile0 * PW_ROWS + tid;
    if (P.splits == 1) P.neg_lse[at] = l == 0.f ? -CUDART_INF_F : -(mu + log2f(l));
    else P.ml[static_cast<long long>(part) * P.n_kv * P.row_tiles * PW_ROWS + at] = make_float2(none ? -CUDART_INF_F : m, l);
  }
}

// Row statistics of the splits put together, one thread per row.
__global__ void __launch_bounds__(128) kvd_prefill_weights_rows_kernel(const __grid_constant__ PwParams P) {
  grid_launch_dependents();
  grid_dependency_wait();
  const long long n = static_cast<long long>(P.n_kv) * P.row_tiles * PW_ROWS, at = blockIdx.x * 128ll + threadIdx.x;
  if (at >= n) return;
  float m = -CUDART_INF_F;
  for (int s = 0; s < P.splits; ++s) m = fmaxf(m, P.ml[s * n + at].x);
  const float mu = m == -CUDART_INF_F ? 0.f : m;
  float l = 0.f;
  for (int s = 0; s < P.splits; ++s) {
    const float2 v = P.ml[s * n + at];
    l += v.y * ex2_approx(v.x - mu);
  }
  P.neg_lse[at] = l == 0.f ? -CUDART_INF_F : -(mu + log2f(l));
}

// out_p = in_p + the partial columns of position p: 32 positions per CTA, eight warps over the partials, added in order.
__global__ void __launch_bounds__(256) kvd_prefill_weights_sum_kernel(const __grid_constant__ PwParams P) {
  grid_launch_dependents();
  grid_dependency_wait();
  __shared__ float s_part[8][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, p = static_cast<int>(blockIdx.x) * 32 + lane;
  const int n = P.ranges * P.n_kv;
  const long long width = static_cast<long long>(P.key_tiles) * PW_KEYS, col = p - static_cast<long long>(P.key_tile0) * PW_KEYS;
  float sum = 0.f;
  if (p < P.n_positions && col >= 0 && col < width) {
#pragma unroll 8
    for (int i = warp; i < n; i += 8) sum += __ldcg(P.cols + i * width + col);
  }
  s_part[warp][lane] = sum;
  __syncthreads();
  if (warp == 0 && p < P.n_positions) {
    float w = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) w += s_part[i][lane];
    P.out[p] = (P.in ? P.in[p] : 0.f) + w;
  }
}

// Shapes of a call's launches and the scratch they need, from the sizes alone: key tiles as if the keys filled all positions.
struct PwPlan {
  int row_tiles, splits, chunk, range, ranges;
  size_t ml_off, cols_off, bytes;
};
constexpr int PW_PLAN_SMS = 148;  // SMs of a B200 (the scratch is asked for without a device)
static PwPlan pw_plan(int n_kv, int group, int n_rows, int n_positions) {
  constexpr int num_sms = PW_PLAN_SMS;
  const int key_tiles = (n_positions + PW_KEYS - 1) / PW_KEYS;
  PwPlan s;
  const long long rows = static_cast<long long>(n_rows) * group;
  s.row_tiles = static_cast<int>((rows + PW_ROWS - 1) / PW_ROWS);
  const long long items = static_cast<long long>(s.row_tiles) * n_kv;
  long long splits = items >= num_sms ? 1 : num_sms / items;
  const long long most = key_tiles / 2 > 1 ? key_tiles / 2 : 1;
  s.splits = static_cast<int>(splits < most ? splits : most);
  // columns: about 32 tiles of work per CTA, fewer where that leaves SMs idle
  s.range = s.row_tiles < 4 ? s.row_tiles : 4;
  if ((s.row_tiles + PW_RANGE - 1) / PW_RANGE > s.range) s.range = (s.row_tiles + PW_RANGE - 1) / PW_RANGE;
  if (s.range > PW_RANGE) s.range = PW_RANGE;
  s.chunk = key_tiles < 8 ? key_tiles : 8;
  auto count = [&]() { return static_cast<long long>(n_kv) * ((key_tiles + s.chunk - 1) / s.chunk) * ((s.row_tiles + s.range - 1) / s.range); };
  while (s.chunk > 2 && count() < num_sms) s.chunk = (s.chunk + 1) / 2;
  while (s.range > 1 && count() < num_sms) s.range = (s.range + 1) / 2;
  while (s.chunk > 1 && count() < num_sms) s.chunk = (s.chunk + 1) / 2;
  s.ranges = (s.row_tiles + s.range - 1) / s.range;
  auto up = [](size_t v) { return (v + 255) / 256 * 256; };
  const size_t padded = static_cast<size_t>(n_kv) * s.row_tiles * PW_ROWS;
  s.ml_off = up(padded * sizeof(float));
  s.cols_off = s.ml_off + (s.splits > 1 ? up(padded * s.splits * sizeof(float2)) : 0);
  s.bytes = s.cols_off + up(static_cast<size_t>(s.ranges) * n_kv * key_tiles * PW_KEYS * sizeof(float));
  return s;
}

template <int D_HEAD, int G, int DT>
static kvd_status pw_launch(kvd_ctx *ctx, const PwParams &P, cudaStream_t stream) {
  auto rows = kvd_prefill_weights_kernel<D_HEAD, G, DT, false>;
  auto columns = kvd_prefill_weights_kernel<D_HEAD, G, DT, true>;
  using R = PwCfg<D_HEAD, false>;
  using C = PwCfg<D_HEAD, true>;
  static std::atomic<bool> rows_done[64] = {}, columns_done[64] = {};
  cudaError_t e = opt_in_smem(ctx, rows, R::SMEM_BYTES, rows_done);
  if (e == cudaSuccess) e = opt_in_smem(ctx, columns, C::SMEM_BYTES, columns_done);
  if (e != cudaSuccess) return cuda_fail(ctx, e, "cudaFuncSetAttribute(prefill weights)");
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof(cfg));
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  auto launch = [&](auto kern, long long grid, int threads, size_t smem) {
    if (e != cudaSuccess) return;
    cfg.gridDim = dim3(static_cast<unsigned>(grid), 1, 1);
    cfg.blockDim = dim3(threads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    attr[0].val.programmaticStreamSerializationAllowed = serial_launch_mask() & 8 ? 0 : 1;
    e = cudaLaunchKernelEx(&cfg, kern, P);
    if (e == cudaSuccess) ctx->launches += 1;
  };
  launch(rows, static_cast<long long>(P.row_tiles) * P.n_kv * P.splits, PW_THREADS, R::SMEM_BYTES);
  if (P.splits > 1) launch(kvd_prefill_weights_rows_kernel, static_cast<long long>(P.n_kv) * P.row_tiles, 128, 0);
  launch(columns, static_cast<long long>(P.chunks) * P.ranges * P.n_kv, PW_THREADS, C::SMEM_BYTES);
  launch(kvd_prefill_weights_sum_kernel, (P.n_positions + 31ll) / 32, 256, 0);
  return e == cudaSuccess ? KVD_OK : cuda_fail(ctx, e, "launch prefill weights");
}
template <int D_HEAD>
static kvd_status pw_group(kvd_ctx *ctx, const PwParams &P, int group, cudaStream_t stream) {
  switch (group * 2 + (ctx->dtype == KVD_DTYPE_F16)) {
    case 2: return pw_launch<D_HEAD, 1, 0>(ctx, P, stream);
    case 3: return pw_launch<D_HEAD, 1, 1>(ctx, P, stream);
    case 4: return pw_launch<D_HEAD, 2, 0>(ctx, P, stream);
    case 5: return pw_launch<D_HEAD, 2, 1>(ctx, P, stream);
    case 6: return pw_launch<D_HEAD, 3, 0>(ctx, P, stream);
    case 7: return pw_launch<D_HEAD, 3, 1>(ctx, P, stream);
    case 8: return pw_launch<D_HEAD, 4, 0>(ctx, P, stream);
    case 9: return pw_launch<D_HEAD, 4, 1>(ctx, P, stream);
    case 16: return pw_launch<D_HEAD, 8, 0>(ctx, P, stream);
    case 17: return pw_launch<D_HEAD, 8, 1>(ctx, P, stream);
    default: return KVD_ERR_SHAPE;
  }
}

}  // namespace kvd

using namespace kvd;

extern "C" size_t kvd_prefill_weights_scratch_bytes(const kvd_model_desc *d, int n_rows, int n_positions) {
  if (kvd_workspace_bytes(d) == 0 || n_rows <= 0 || n_positions <= 0 || n_positions > (1 << 30)) return 0;  // (checks the description)
  const int group = d->n_q_heads / d->n_kv_heads;
  if (static_cast<long long>(n_rows) * group > INT32_MAX - PW_ROWS) return 0;
  return pw_plan(d->n_kv_heads, group, n_rows, n_positions).bytes;
}

extern "C" kvd_status kvd_prefill_attention_weights(kvd_ctx *ctx, int layer, int n_rows, const void *q, const int32_t *q_pos,
                                                    const kvd_kv_segment *segs, int n_segs, float scale, const float *weights_in,
                                                    float *weights_out, int n_positions, void *scratch, size_t scratch_bytes,
                                                    void *stream_) {
  if (!ctx || n_rows < 0 || n_segs < 0 || n_segs > KVD_MAX_SEGMENTS || n_positions < 0) return KVD_ERR_INVALID_ARG;
  if (layer < 0 || layer >= ctx->desc.n_layers) return KVD_ERR_INVALID_ARG;
  const LayerState &ls = ctx->layers[layer];
  if (!ls.set) return KVD_ERR_STATE;
  if (ctx->dtype == KVD_DTYPE_F32) return KVD_ERR_UNSUPPORTED;
  if (n_positions == 0 && n_segs == 0) return KVD_OK;
  if (!weights_out || !scratch || (n_segs > 0 && !segs) || (n_rows > 0 && (!q || !q_pos))) return KVD_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(q) & 15u) != 0 || (reinterpret_cast<uintptr_t>(scratch) & 255u) != 0) return KVD_ERR_ALIGNMENT;
  if (n_positions > (1 << 30)) return KVD_ERR_CAPACITY;
  const kvd_model_desc &d = ctx->desc;
  const int kdim = d.n_kv_heads * d.d_head, group = d.n_q_heads / d.n_kv_heads;
  static thread_local PwParams P;
  P.seg_lo = INT32_MAX;
  P.seg_hi = -1;
  for (int s = 0; s < KVD_MAX_SEGMENTS; ++s) {
    P.k[s] = nullptr;
    P.stride[s] = 0;
    P.first[s] = 0;
    P.len[s] = 0;
    if (s >= n_segs) continue;
    const kvd_kv_segment &sg = segs[s];
    if (sg.len < 0 || sg.first_pos < 0) return KVD_ERR_INVALID_ARG;
    if (sg.len == 0) continue;
    if (!sg.k || sg.row_stride < kdim) return KVD_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(sg.k) & 15u) != 0 || sg.row_stride % 8 != 0) return KVD_ERR_ALIGNMENT;
    if (static_cast<int64_t>(sg.first_pos) + sg.len > n_positions) return KVD_ERR_CAPACITY;
    for (int s2 = 0; s2 < s; ++s2)
      if (P.len[s2] > 0 && sg.first_pos < P.first[s2] + P.len[s2] && P.first[s2] < sg.first_pos + sg.len) return KVD_ERR_INVALID_ARG;
    P.k[s] = static_cast<const __nv_bfloat16 *>(sg.k);
    P.stride[s] = sg.row_stride;
    P.first[s] = sg.first_pos;
    P.len[s] = sg.len;
    if (sg.first_pos < P.seg_lo) P.seg_lo = sg.first_pos;
    if (sg.first_pos + sg.len - 1 > P.seg_hi) P.seg_hi = sg.first_pos + sg.len - 1;
  }
  if (n_positions == 0) return KVD_OK;
  cudaStream_t stream = static_cast<cudaStream_t>(stream_);
  P.in = weights_in;
  P.out = weights_out;
  P.n_positions = n_positions;
  P.n_kv = d.n_kv_heads;
  if (n_rows == 0 || P.seg_hi < 0) {  // nothing weighs anything
    P.key_tile0 = P.key_tiles = P.ranges = 0;
    if (weights_in == weights_out) return KVD_OK;
    kvd_prefill_weights_sum_kernel<<<(n_positions + 31) / 32, 256, 0, stream>>>(P);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return cuda_fail(ctx, e, "launch prefill weights (sum)");
    ctx->launches += 1;
    return KVD_OK;
  }
  if (static_cast<long long>(n_rows) * group > INT32_MAX - PW_ROWS) return KVD_ERR_CAPACITY;
  P.key_tile0 = P.seg_lo / PW_KEYS;
  P.key_tiles = P.seg_hi / PW_KEYS - P.key_tile0 + 1;
  const PwPlan plan = pw_plan(d.n_kv_heads, group, n_rows, n_positions);
  if (plan.bytes > scratch_bytes) return KVD_ERR_CAPACITY;
  uint8_t *base = static_cast<uint8_t *>(scratch);
  P.neg_lse = reinterpret_cast<float *>(base);
  P.ml = reinterpret_cast<float2 *>(base + plan.ml_off);
  P.cols = reinterpret_cast<float *>(base + plan.cols_off);
  P.q = static_cast<const __nv_bfloat16 *>(q);
  P.q_pos = q_pos;
  P.n_rows = n_rows;
  P.n_q = d.n_q_heads;
  P.window = ls.window;
  P.scale_log2e = (scale > 0.f ? scale : 1.0f / sqrtf(static_cast<float>(d.d_head))) * 1.4426950408889634f;
  P.rows = n_rows * group;
  P.row_tiles = plan.row_tiles;
  P.splits = plan.splits;
  P.chunk = plan.chunk;
  P.chunks = (P.key_tiles + plan.chunk - 1) / plan.chunk;
  P.range = plan.range;
  P.ranges = plan.ranges;
  P.status = ctx->d_status;
  P.timeout_ns = ctx->timeout_ns;
  switch (d.d_head) {
    case 64: return pw_group<64>(ctx, P, group, stream);
    case 128: return pw_group<128>(ctx, P, group, stream);
    case 256: return pw_group<256>(ctx, P, group, stream);
    default: return KVD_ERR_SHAPE;
  }
}
