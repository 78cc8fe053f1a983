// Attention weights of a prompt's keys (include/kvd.h, kvd_prefill_attention_weights): w_j = sum over rows r of 2^(s_rj - z_r),
// z_r = log2 of the row's sum of 2^s (Eq. 6 in base 2), over the query rows of every head.  A row's statistic needs all of
// its scores, a key's weight the statistics of all its rows, so the scores are computed twice, on tcgen05.mma with fp32 sums
// in tensor memory, rather than kept (4 bytes per score and pass against d_head multiply-adds that take less time):
//
//   rows     S = Q K^T, 128 query rows x 128 keys: a thread has half of a row in its tensor-memory lane, and that half's
//            reference and sum in registers.
//   columns  S^T = K Q^T, 128 keys x 128 query rows: a thread has a key and half of the rows, and adds up the key's weights
//            in registers; the rows' statistics come from shared memory, the same word for all lanes.  Sums of a tile's keys go
//            to shared memory, one owner per word.
//   sum      partial columns of all KV heads and row ranges, added in a fixed order, to the weights so far.
//
// A row tile is 128 / G query tokens times the G heads of a KV head's group (G = 3: 42 tokens, two rows stay empty); key tiles
// are aligned to absolute position.  Either pass goes through row tiles and, for each, the key tiles it sees; both kinds of
// tiles share a ring of shared memory, filled by TMA (a key tile that touches more than one segment: piece by piece with
// cp.async).  A query tile keeps its slot until its last product, and the next one's comes in ahead of that.
//
// Two CTAs share an SM, so that one's start and end pass behind the other's work (d_head 256, whose tiles fill shared memory:
// one CTA with twice the warps).  In a CTA eight (sixteen) warps take exponentials, one issues products, one fetches tiles.
// Every wait is bounded, as in the other tensor-core kernels.
//
// Bound by exponentials and what surrounds them.  4096 tokens of a Qwen3-4B layer: rows 92, columns 120, sum 6 us; one product
// alone would be 42, a pass's exponentials at 16 per clock and SM 69 at 1.7 GHz (three quarters of them: 52).  With an eighth of the exponentials the passes take 65
// and 74.  One persistent CTA per SM instead, each key tile against two row tiles, with sixteen warps for exponentials and one or
// two for products, takes 59 and 68 then, but 94 and 127 with all of them.
#include <math_constants.h>
#include <string.h>

#include <type_traits>

#include "kvd_internal.h"
#include "kvd_ptx.cuh"

namespace kvd {

constexpr int PW_ROWS = 128;      // query rows per tile
constexpr int PW_KEYS = 128;      // keys per tile
constexpr int PW_RANGE = 64;      // row tiles one CTA of the columns pass can take
constexpr int PW_CHUNK = 8;       // key tiles of one (sums in shared memory)
// Of every eight pairs of scores, those that take the fp32 pipes.  Rows / columns pass of 4096 tokens of a Qwen3-4B layer with 0,
// 1, 2, 3 of them: 91 / 116, 89 / 119, 90 / 116, 96 / 126 us (special-function units busy 56 % / 43 % with two; issue slots 60 %).
constexpr int PW_POLY = 2;

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
  int row_tiles;           // of a KV head
  int splits;              // rows pass: shares of a row tile's keys
  float2 *ml;              // [splits][n_kv][row_tiles * 128]: reference and sum of a row's share; (-inf, 0): nothing seen
  int key_tile0, key_tiles, chunk, chunks, range, ranges;  // columns pass: key tiles per CTA, row tiles per CTA
  float *cols;             // [ranges][n_kv][key_tiles * 128]
  long long ml_size, cols_size;  // elements the scratch has room for (checking build)
  const float *in;
  float *out;
  int n_positions;
  int *status;
  unsigned long long timeout_ns;
};
struct PwMaps {
  CUtensorMap q;                    // [n_rows][n_q][d_head], boxes of 64 channels, a group's heads and a tile's tokens
  CUtensorMap k[KVD_MAX_SEGMENTS];  // [len][n_kv * d_head], boxes of 64 channels and a tile's keys
};

template <int D_HEAD, bool COLUMNS>
struct PwCfg {
  static constexpr int CTAS = D_HEAD == 256 ? 1 : 2;           // per SM
  static constexpr int SOFT = 16 / CTAS;                       // warps that take exponentials: pairs of groups of four share a
  static constexpr int TURNS = SOFT / 8;                       // tile, 64 columns each, and take turns on the tiles
  static constexpr int THREADS = SOFT * 32 + 64;
  static constexpr int TILE_BYTES = 128 * D_HEAD * 2, SLAB = 128 * 128;  // (64 channels)
  static constexpr int SLOTS = D_HEAD == 64 ? 6 : 3;
  static constexpr int COLS = 512 / CTAS, S_BUFS = COLS / 128;  // tensor memory: scores
  static constexpr int N_BARS = 2 * SLOTS + 2 * S_BUFS;
  static constexpr int SMEM_BYTES = 1024 + SLOTS * TILE_BYTES + N_BARS * 8;
  static_assert(SMEM_BYTES + (COLUMNS ? SOFT * 1024 : 0) + 4096 <= 232448 / CTAS - 1024, "does not fit");
};

// The ring's slots in the order in which they come free: a key tile's behind its own product, a query tile's behind its last
// one.  Whoever fills the slots and whoever empties them goes through the same sequence.
template <int SLOTS>
struct PwRing {
  uint32_t order = 0x543210u & ((1u << (4 * SLOTS)) - 1u);  // four bits each, the next one lowest
  int n = SLOTS;
  uint32_t phase = 0, used = 0;  // per slot: parity of the phase to be waited for, whether it has been filled at all
  __device__ __forceinline__ int take() {
    const int s = static_cast<int>(order & 15u);
    order >>= 4;
    --n;
    return s;
  }
  __device__ __forceinline__ void give(int s) {
    order |= static_cast<uint32_t>(s) << (4 * n);
    ++n;
  }
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

// The keys that the rows of a tile can see, as key tiles (first, count); a warp's lanes go through the tokens.  Returns the
// smallest and the largest position of the rows' tokens as well.
template <int G>
__device__ __forceinline__ void pw_tile_range(const PwParams &P, int row_tile, int lane, int &tile, int &count, int &qmin, int &qmax) {
  constexpr int TOK = PW_ROWS / G;
  const int tok0 = row_tile * TOK, tok1 = min(P.n_rows, tok0 + TOK);
  int lo = INT_MAX, hi = -1;
  qmin = INT_MAX;
  qmax = -1;
  for (int t = tok0 + lane; t < tok1; t += 32) {
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
  if (tok0 + TOK > P.n_rows) qmin = -1;  // rows that are not there see nothing
  tile = hi >= 0 ? lo / PW_KEYS : 0;
  count = hi >= 0 ? hi / PW_KEYS - tile + 1 : 0;
}

// A warp's 128 keys from position pos0 on into a tile at `base`: rows of 128 bytes per 64 channels, 128-byte swizzle; what no
// segment holds reads as zeros.
template <int D_HEAD>
__device__ __forceinline__ void pw_gather_keys(const PwParams &P, uint32_t base, int pos0, int kvh, int lane) {
  constexpr int CPR = D_HEAD / 8;
#pragma unroll 1
  for (int i = lane; i < PW_KEYS * CPR; i += 32) {
    const int r = i / CPR, c = i % CPR, pos = pos0 + r;
    const __nv_bfloat16 *src = P.q;
    bool have = false;
#pragma unroll
    for (int sg = 0; sg < KVD_MAX_SEGMENTS; ++sg)
      if (segment_holds(P.first[sg], P.len[sg], pos, 1)) {
        src = P.k[sg] + static_cast<long long>(pos - P.first[sg]) * P.stride[sg] + static_cast<long long>(kvh) * D_HEAD + c * 8;
        have = true;
      }
    cp_async16(base + (c >> 3) * (PW_KEYS * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4), src, have);
  }
  cp_async_commit();
  cp_async_wait_all();
  fence_proxy_async_smem();
  __syncwarp();
}

__device__ __forceinline__ float pw_max32(const uint32_t (&s)[32]) {
  float mx[2] = {-CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
  for (int k = 0; k < 32; k += 4) {
    mx[0] = fmax3(mx[0], __uint_as_float(s[k]), __uint_as_float(s[k + 1]));
    mx[1] = fmax3(mx[1], __uint_as_float(s[k + 2]), __uint_as_float(s[k + 3]));
  }
  return fmaxf(mx[0], mx[1]);
}

// 2^e for a pair, on the special-function unit.
__device__ __forceinline__ uint64_t pw_ex2(uint64_t e) {
  float e0, e1;
  unpack2(e, e0, e1);
  return pack2(ex2_approx(e0), ex2_approx(e1));
}
// The same on the fp32 pipes: e = n + f with n whole and |f| <= 1/2 (adding and taking away 1.5 * 2^23 rounds to whole numbers),
// 2^f by a polynomial of degree 5 with the constant term 1, n added to the exponent.  Over [-1/2, 1/2] the polynomial is off by
// -1.6e-7 to 1.5e-8 of the value (the degree's least error, to either side, with its constant term rounded to 1), with the steps'
// roundings by 2.5e-7 at most; ex2.approx by 2.4e-7.  From -126 down results lose bits, at and below -127 they are exactly 0.  UPPER:
// also for e that may be large -- the result is then at least 2^127; a NaN gives more than 1e30 or a NaN, and so does plus infinity.
template <bool UPPER>
__device__ __forceinline__ uint64_t pw_ex2_poly(uint64_t e) {
  float e0, e1, t0, t1, p0, p1;
  unpack2(e, e0, e1);
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(e0) : "f"(e0), "f"(-127.0f));
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(e1) : "f"(e1), "f"(-127.0f));
  if constexpr (UPPER) {
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(e0) : "f"(e0), "f"(127.0f));
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(e1) : "f"(e1), "f"(127.0f));
  }
  const uint64_t one2 = pack2(1.0f, 1.0f), x = pack2(e0, e1);
  const uint64_t t = ffma2(x, one2, pack2(12582912.0f, 12582912.0f)), n = ffma2(t, one2, pack2(-12582912.0f, -12582912.0f));
  const uint64_t f = ffma2(n, pack2(-1.0f, -1.0f), x);
  uint64_t p = pack2(0.001327647129073739f, 0.001327647129073739f);
  p = ffma2(p, f, pack2(0.009675540961325169f, 0.009675540961325169f));
  p = ffma2(p, f, pack2(0.05550713092088699f, 0.05550713092088699f));
  p = ffma2(p, f, pack2(0.24022120237350464f, 0.24022120237350464f));
  p = ffma2(p, f, pack2(0.6931469440460205f, 0.6931469440460205f));
  p = ffma2(p, f, one2);
  unpack2(t, t0, t1);
  unpack2(p, p0, p1);
  return pack2(__uint_as_float(__float_as_uint(p0) + (__float_as_uint(t0) << 23)), __uint_as_float(__float_as_uint(p1) + (__float_as_uint(t1) << 23)));
}
// Of the pairs of a thread's scores, those that take the fp32 pipes: PW_POLY of every eight.
template <bool UPPER>
__device__ __forceinline__ uint64_t pw_ex2_of(int pair, uint64_t e) {
  return (pair & 7) * PW_POLY % 8 < PW_POLY ? pw_ex2_poly<UPPER>(e) : pw_ex2(e);
}

template <int D_HEAD, int G, int DT, bool COLUMNS>
__global__ void __launch_bounds__(PwCfg<D_HEAD, COLUMNS>::THREADS, PwCfg<D_HEAD, COLUMNS>::CTAS)
    kvd_prefill_weights_kernel(const __grid_constant__ PwParams P, const __grid_constant__ PwMaps M) {
  using Cfg = PwCfg<D_HEAD, COLUMNS>;
  constexpr int SLOTS = Cfg::SLOTS, S_BUFS = Cfg::S_BUFS, SOFT = Cfg::SOFT, TURNS = Cfg::TURNS, GROUPS = SOFT / 4;
  constexpr int TOK = PW_ROWS / G;
  extern __shared__ uint8_t pw_smem_raw[];
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort_i;
  __shared__ int s_tile[PW_RANGE], s_count[PW_RANGE], s_qmin[PW_RANGE], s_qmax[PW_RANGE];  // per row tile of the CTA
  __shared__ float2 s_ml[COLUMNS ? 1 : GROUPS][COLUMNS ? 1 : PW_ROWS];  // rows: the groups' statistics
  __shared__ __align__(16) float s_nl[2][PW_ROWS];                      // columns: -(m + log2 l) of the rows, and their positions
  __shared__ __align__(16) int s_qp[2][PW_ROWS];
  __shared__ float s_sum[COLUMNS ? GROUPS : 1][COLUMNS ? PW_CHUNK * PW_KEYS : 1];
  volatile int *s_abort = &s_abort_i;
  const uint32_t ring = (smem_u32(pw_smem_raw) + 1023u) & ~1023u;  // the swizzle is a function of the address
  const uint32_t bar_base = ring + SLOTS * Cfg::TILE_BYTES;
  auto bar_full = [&](int s) { return bar_base + 8u * s; };                          // a tile has landed
  auto bar_empty = [&](int s) { return bar_base + 8u * (SLOTS + s); };               // its products are done
  auto bar_s_full = [&](int b) { return bar_base + 8u * (2 * SLOTS + b); };          // scores of a tile
  auto bar_s_free = [&](int b) { return bar_base + 8u * (2 * SLOTS + S_BUFS + b); };  // ... have been read
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
      mbar_init(bar_full(s), 1);
      mbar_init(bar_empty(s), 1);
    }
    for (int b = 0; b < S_BUFS; ++b) {
      mbar_init(bar_s_full(b), 1);
      mbar_init(bar_s_free(b), 8);
    }
    fence_mbar_init();
    s_abort_i = 0;
    prefetch_tensormap(&M.q);
    for (int sg = 0; sg < KVD_MAX_SEGMENTS; ++sg)
      if (P.len[sg] > 0) prefetch_tensormap(&M.k[sg]);
  }
  if (warp == SOFT) tmem_claim(smem_u32(&s_tmem), Cfg::COLS);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  grid_launch_dependents();
  grid_dependency_wait();
  const uint32_t tmem_base = s_tmem;
  if (warp >= SOFT) {
    for (int i = warp - SOFT; i < n_tiles; i += 2) {
      int t, n, qmin, qmax;
      pw_tile_range<G>(P, tile0 + i, lane, t, n, qmin, qmax);
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
      if (lane == 0 && KVD_BOUNDS_OK(i < PW_RANGE, P.status)) {
        s_tile[i] = t;
        s_count[i] = n;
        s_qmin[i] = qmin;
        s_qmax[i] = qmax;
      }
    }
  } else if constexpr (COLUMNS) {
    for (int i = tid; i < GROUPS * PW_CHUNK * PW_KEYS; i += SOFT * 32) (&s_sum[0][0])[i] = 0.f;
  }
  __syncthreads();

  if (warp < SOFT) {
    // ------------------------------------------------------------------ exponentials
    const int grp = warp >> 2, q4 = warp & 3, row = q4 * 32 + lane;
    const int half = grp / TURNS, turn = grp % TURNS;
    const uint64_t c2 = pack2(P.scale_log2e, P.scale_log2e), one2 = pack2(1.0f, 1.0f);
    const uint32_t s_col = tmem_base + (static_cast<uint32_t>(q4 * 32) << 16) + half * 64;
    bool ok = true;
    if constexpr (!COLUMNS) {
      const int tok = tile0 * TOK + row / G, n_blk = s_count[0], t0 = s_tile[0];
      const bool valid = row < TOK * G && tok < P.n_rows;
      const int qp = valid ? max(P.q_pos[tok], -1) : -1, lo = first_visible(qp, P.window);
      // range that every stored row of the warp sees
      const int all_lo = __reduce_max_sync(0xffffffffu, valid ? lo : INT_MIN), all_hi = __reduce_min_sync(0xffffffffu, valid ? qp : INT_MAX);
      // ... as far as the segment goes that held the last such piece
      int whole_lo = 1, whole_hi = 0;
      // The reference m is the first finite maximum the row meets, rounded up to a whole number, and moves only if a sum
      // threatens to leave fp32's range: 2^(s - m) is as exact for any m.
      float m = valid ? -CUDART_INF_F : 0.f, l = 0.f;  // (rows that nobody filled score anything)
      bool seen = false;  // every row of the warp has a reference
      for (int j = turn; j < n_blk; j += TURNS) {
        const int buf = j % S_BUFS, pos0 = (t0 + j) * PW_KEYS + half * 64;
        if (!pw_warp_wait(bar_s_full(buf), (j / S_BUFS) & 1, s_abort, tmo, lane)) {
          raise(P.status, STATUS_TIMEOUT, s_abort);
          ok = false;
          break;
        }
        tc_fence_after();
        if (pos0 < whole_lo || pos0 + 63 > whole_hi) {
#pragma unroll
          for (int sg = 0; sg < KVD_MAX_SEGMENTS; ++sg)
            if (segment_holds(P.first[sg], P.len[sg], pos0, 64)) {
              whole_lo = max(P.first[sg], all_lo);
              whole_hi = min(P.first[sg] + P.len[sg] - 1, all_hi);
            }
        }
        const bool whole = pos0 >= whole_lo && pos0 + 63 <= whole_hi;
        unsigned long long vis = ~0ull;
        if (!whole) {
          vis = 0ull;
#pragma unroll
          for (int sg = 0; sg < KVD_MAX_SEGMENTS; ++sg) vis |= segment_slots(P.first[sg], P.len[sg], pos0);
          vis &= visible_slots(lo, qp, pos0);
        }
#pragma unroll 1
        for (int chunk = 0; chunk < 2; ++chunk) {
          uint32_t s[32];
          tmem_ld_x32(s_col + buf * 128 + chunk * 32, s);
          tmem_wait_ld();
          if (chunk == 1) {  // the scores are in registers: their columns may take another tile
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_s_free(buf));
          }
          if (!whole) {
            const uint32_t v = static_cast<uint32_t>(vis >> (32 * chunk));
#pragma unroll
            for (int k = 0; k < 32; ++k)
              if (!((v >> k) & 1u)) s[k] = 0xff800000u;  // -inf
          }
          if (!seen) {  // (uniform)
            const float bm = ceilf(pw_max32(s) * P.scale_log2e);
            if (m == -CUDART_INF_F) m = bm;
            seen = !__any_sync(0xffffffffu, m == -CUDART_INF_F);
          }
          const float mu = m == -CUDART_INF_F ? 0.f : m;
          const uint64_t nm2 = pack2(-mu, -mu);
          uint64_t l2[2] = {0ull, 0ull};
#pragma unroll
          for (int k = 0; k < 32; k += 4) {
            l2[0] = ffma2(pw_ex2_of<true>(k / 2, ffma2(pack2(__uint_as_float(s[k]), __uint_as_float(s[k + 1])), c2, nm2)), one2, l2[0]);
            l2[1] = ffma2(pw_ex2_of<true>(k / 2 + 1, ffma2(pack2(__uint_as_float(s[k + 2]), __uint_as_float(s[k + 3])), c2, nm2)), one2, l2[1]);
          }
          float a0, a1, a2, a3;
          unpack2(l2[0], a0, a1);
          unpack2(l2[1], a2, a3);
          float sum = (a0 + a1) + (a2 + a3);
          const bool odd = valid && !(sum < 1e30f);  // (a NaN among them)
          if (__any_sync(0xffffffffu, odd)) {
            const float bm = ceilf(pw_max32(s) * P.scale_log2e);
            if (odd && bm > m) {
              l *= ex2_approx(m - bm);
              m = bm;
            }
            // (one by one: what is not a number, or is infinite, comes out as it does from the unit)
            float again = 0.f;
#pragma unroll 1
            for (int k = 0; k < 32; ++k) {
              uint32_t v = 0u;
#pragma unroll
              for (int u = 0; u < 32; ++u) v = u == k ? s[u] : v;
              again += ex2_approx(fmaf(__uint_as_float(v), P.scale_log2e, m == -CUDART_INF_F ? 0.f : -m));
            }
            if (odd) sum = again;
          }
          l += sum;
        }
      }
      if (ok) s_ml[grp][row] = make_float2(m, l);
    } else {
      // Statistics of row tile i's rows: two or four threads per row, the splits in turns (one split: the first thread alone)
      constexpr int PER = SOFT / 4;  // threads per row
      const int of = tid / PER, share = tid % PER;
      auto statistics = [&](int i) {
        const long long n = static_cast<long long>(P.n_kv) * P.row_tiles * PW_ROWS;
        const float2 *src = P.ml + static_cast<long long>(kvh) * P.row_tiles * PW_ROWS + (tile0 + i) * PW_ROWS + of;
        float m = -CUDART_INF_F, l = 0.f;
        for (int s0 = share; s0 < P.splits; s0 += 4 * PER) {
          float2 v[4];
#pragma unroll
          for (int u = 0; u < 4; ++u)
            v[u] = s0 + PER * u < P.splits && KVD_BOUNDS_OK(src + (s0 + PER * u) * n < P.ml + P.ml_size, P.status) ? __ldcg(src + (s0 + PER * u) * n)
                                                                                                                   : make_float2(-CUDART_INF_F, 0.f);
          const float mn = fmaxf(m, fmaxf(fmaxf(v[0].x, v[1].x), fmaxf(v[2].x, v[3].x))), mu = mn == -CUDART_INF_F ? 0.f : mn;
          l *= ex2_approx(m - mu);
#pragma unroll
          for (int u = 0; u < 4; ++u) l = fmaf(ex2_approx(v[u].x - mu), v[u].y, l);
          m = mn;
        }
#pragma unroll
        for (int k = 1; k < PER; k <<= 1) {
          const float mo = __shfl_xor_sync(0xffffffffu, m, k), lo = __shfl_xor_sync(0xffffffffu, l, k);
          const float mn = fmaxf(m, mo), mu = mn == -CUDART_INF_F ? 0.f : mn;
          l = l * ex2_approx(m - mu) + lo * ex2_approx(mo - mu);
          m = mn;
        }
        // a row that nothing weighs in (or that is not there) adds nothing
        return l == 0.f ? -CUDART_INF_F : -(m + log2f(l));
      };
      auto position = [&](int i) {
        const int tok = (tile0 + i) * TOK + of / G;
        return of < TOK * G && tok < P.n_rows ? max(P.q_pos[tok], -1) : -1;
      };
      auto next_of = [&](int i) {
        while (i < n_tiles && s_count[i] == 0) ++i;
        return i;
      };
      int j0 = 0, nth = 0;  // tiles before this row tile's
      int i = next_of(0);
      float nl = 0.f;
      int qp_of = 0;
      if (i < n_tiles) {
        nl = statistics(i);
        qp_of = position(i);
      }
      while (i < n_tiles) {
        const int n_blk = s_count[i], t0 = s_tile[i], slot = nth & 1, qmin = s_qmin[i], qmax = s_qmax[i];
        if (share == 0) {
          s_nl[slot][of] = nl;
          s_qp[slot][of] = qp_of;
        }
        asm volatile("bar.sync 1, %0;" ::"n"(SOFT * 32) : "memory");  // (two buffers: everyone has left the one written next)
        const int next = next_of(i + 1);
        if (next < n_tiles) {
          nl = statistics(next);
          qp_of = position(next);
        }
        for (int jj = (turn + TURNS - j0 % TURNS) % TURNS; ok && jj < n_blk; jj += TURNS) {
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
#pragma unroll 1
          for (int chunk = 0; chunk < 2; ++chunk) {
            const int at = half * 64 + chunk * 32;
            uint32_t s[32];
            tmem_ld_x32(s_col + buf * 128 + chunk * 32, s);
            tmem_wait_ld();
            if (chunk == 1) {
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(bar_s_free(buf));
            }
            if constexpr (TOK * G < PW_ROWS) {  // rows that nobody filled
#pragma unroll
              for (int k = 0; k < PW_ROWS - TOK * G; ++k) s[31 - k] = at == 96 ? 0u : s[31 - k];
            }
            uint64_t part[2] = {0ull, 0ull};
            auto add = [&](auto exact_c, auto whole_c) {
#pragma unroll
              for (int k = 0; k < 32; k += 4) {
                const ulonglong2 nl2 = *reinterpret_cast<const ulonglong2 *>(&s_nl[slot][at + k]);
                const uint64_t e[2] = {ffma2(pack2(__uint_as_float(s[k]), __uint_as_float(s[k + 1])), c2, nl2.x),
                                       ffma2(pack2(__uint_as_float(s[k + 2]), __uint_as_float(s[k + 3])), c2, nl2.y)};
                int4 qp = make_int4(0, 0, 0, 0);
                if constexpr (!whole_c) qp = *reinterpret_cast<const int4 *>(&s_qp[slot][at + k]);
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                  uint64_t p = exact_c ? pw_ex2(e[u]) : pw_ex2_of<false>(k / 2 + u, e[u]);
                  if constexpr (!whole_c) {
                    float p0, p1;
                    unpack2(p, p0, p1);
                    p0 = static_cast<uint32_t>((u ? qp.z : qp.x) - kp) < window ? p0 : 0.f;
                    p1 = static_cast<uint32_t>((u ? qp.w : qp.y) - kp) < window ? p1 : 0.f;
                    p = pack2(p0, p1);
                  }
                  part[u] = ffma2(p, one2, part[u]);
                }
              }
            };
            // (masked tiles are few, and a weight that is not a number comes out as one only from the unit)
            if (!whole) {
              add(std::true_type(), std::false_type());
            } else {
              add(std::false_type(), std::true_type());
              float a0, a1, a2, a3;
              unpack2(part[0], a0, a1);
              unpack2(part[1], a2, a3);
              const bool odd = !((a0 + a1) + (a2 + a3) < 1e30f);
              if (__any_sync(0xffffffffu, odd)) {
                const uint64_t was[2] = {part[0], part[1]};
                part[0] = part[1] = 0ull;
                add(std::true_type(), std::true_type());
                if (!odd) part[0] = was[0], part[1] = was[1];
              }
            }
            acc[0] = ffma2(part[0], one2, acc[0]);
            acc[1] = ffma2(part[1], one2, acc[1]);
          }
          float a0, a1, a2, a3;
          unpack2(acc[0], a0, a1);
          unpack2(acc[1], a2, a3);
          if (KVD_BOUNDS_OK(t0 + jj >= kt_lo && t0 + jj < kt_lo + PW_CHUNK, P.status))
            s_sum[grp][(t0 + jj - kt_lo) * PW_KEYS + row] += (a0 + a1) + (a2 + a3);
        }
        j0 += n_blk;
        ++nth;
        i = next;
      }
    }
  } else if (warp == SOFT) {
    // ------------------------------------------------------------------ products (one thread)
    constexpr uint32_t IDESC = DT == 0 ? umma_idesc_bf16_f32(128, 128) : umma_idesc_f16_f32(128, 128);
    if (lane == 0) {
      bool ok = true;
      int j = 0;
      PwRing<SLOTS> R;
      auto landed = [&](int s) {
        ok = ok && pw_wait(bar_full(s), (R.phase >> s) & 1u, s_abort, tmo);
        R.phase ^= 1u << s;
      };
      for (int i = 0; ok && i < n_tiles; ++i) {
        const int n_blk = s_count[i];
        if (n_blk == 0) continue;
        const int qs = R.take();
        landed(qs);
        for (int jj = 0; ok && jj < n_blk; ++jj, ++j) {
          const int slot = R.take(), buf = j % S_BUFS;
          R.give(slot);
          landed(slot);
          if (j >= S_BUFS) ok = ok && pw_wait(bar_s_free(buf), (j / S_BUFS - 1) & 1, s_abort, tmo);
          if (!ok) break;
          tc_fence_after();
          const uint64_t kdesc = umma_smem_desc_sw128(ring + slot * Cfg::TILE_BYTES), qdesc = umma_smem_desc_sw128(ring + qs * Cfg::TILE_BYTES);
          const uint64_t adesc = COLUMNS ? kdesc : qdesc, bdesc = COLUMNS ? qdesc : kdesc;
#pragma unroll
          for (int ks = 0; ks < D_HEAD / 16; ++ks) {
            const uint64_t off = ((ks >> 2) * Cfg::SLAB + (ks & 3) * 32) >> 4;
            umma_bf16(tmem_base + buf * 128, adesc + off, bdesc + off, IDESC, ks > 0 ? 1u : 0u);
          }
          umma_commit(bar_empty(slot));
          umma_commit(bar_s_full(buf));
        }
        if (ok) umma_commit(bar_empty(qs));
        R.give(qs);
      }
      if (!ok) raise(P.status, STATUS_TIMEOUT, s_abort);
    }
  } else {
    // ------------------------------------------------------------------ query and key tiles (a warp; TMA by its first lane)
    bool ok = true;
    PwRing<SLOTS> R;
    auto free_slot = [&](int s) {
      if ((R.used >> s) & 1u) {
        ok = ok && pw_warp_wait(bar_empty(s), (R.phase >> s) & 1u, s_abort, tmo, lane);
        if (ok) R.phase ^= 1u << s;
      }
      if (ok) R.used |= 1u << s;
    };
    for (int i = 0; ok && i < n_tiles; ++i) {
      const int n_blk = s_count[i], t0 = s_tile[i];
      if (n_blk == 0) continue;
      const int qs = R.take();
      free_slot(qs);
      if (!ok) break;
      if (lane == 0) {
        mbar_arrive_expect_tx(bar_full(qs), TOK * G * D_HEAD * 2);
#pragma unroll
        for (int c = 0; c < D_HEAD / 64; ++c)
          tma_load_3d(ring + qs * Cfg::TILE_BYTES + c * Cfg::SLAB, &M.q, bar_full(qs), c * 64, kvh * G, (tile0 + i) * TOK);
      }
      for (int jj = 0; ok && jj < n_blk; ++jj) {
        const int slot = R.take(), pos0 = (t0 + jj) * PW_KEYS;
        R.give(slot);
        free_slot(slot);
        if (!ok) break;
        // the segments that the tile touches; what lies outside of the one TMA reads as zeros
        int touched = 0, sg_of = 0;
#pragma unroll
        for (int sg = 0; sg < KVD_MAX_SEGMENTS; ++sg)
          if (P.len[sg] > 0 && pos0 < P.first[sg] + P.len[sg] && P.first[sg] - pos0 < PW_KEYS) {
            ++touched;
            sg_of = sg;
          }
        if (touched == 1) {
          if (lane == 0) {
            mbar_arrive_expect_tx(bar_full(slot), Cfg::TILE_BYTES);
#pragma unroll
            for (int c = 0; c < D_HEAD / 64; ++c)
              tma_load_2d(ring + slot * Cfg::TILE_BYTES + c * Cfg::SLAB, &M.k[sg_of], bar_full(slot), kvh * D_HEAD + c * 64, pos0 - P.first[sg_of]);
          }
        } else {
          pw_gather_keys<D_HEAD>(P, ring + slot * Cfg::TILE_BYTES, pos0, kvh, lane);
          if (lane == 0) mbar_arrive(bar_full(slot));
        }
      }
      R.give(qs);
    }
    if (!ok) {
      raise(P.status, STATUS_TIMEOUT, s_abort);
      // The copies in flight land before the CTA's shared memory goes to another.  (A slot that has been waited for n times has
      // been filled n + 1 times: its last copy completes phase n.)
      for (int s = 0; s < SLOTS; ++s) {
        const unsigned long long t0 = globaltimer_ns();
        while (((R.used >> s) & 1u) && !mbar_try_wait(bar_full(s), (R.phase >> s) & 1u) && globaltimer_ns() - t0 < tmo) __nanosleep(20);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == SOFT) {
    tc_fence_after();
    tmem_dealloc(tmem_base, Cfg::COLS);
  }
  if constexpr (COLUMNS) {
    // (also the sums of a CTA that gave up: the status word says so)
    const long long first = (static_cast<long long>(part) * P.n_kv + kvh) * P.key_tiles * PW_KEYS + (kt_lo - P.key_tile0) * PW_KEYS;
    float *dst = P.cols + first;
    for (int i = tid; i < (kt_hi - kt_lo) * PW_KEYS; i += Cfg::THREADS) {
      if (!KVD_BOUNDS_OK(i < PW_CHUNK * PW_KEYS && first + i < P.cols_size, P.status)) break;
      float w = 0.f;
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) w += s_sum[g][i];
      dst[i] = pw_held(P, kt_lo * PW_KEYS + i, 1) ? w : 0.f;
    }
  } else if (tid < PW_ROWS) {
    float m = -CUDART_INF_F, l = 0.f;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) m = fmaxf(m, s_ml[g][tid].x);
    const float mu = m == -CUDART_INF_F ? 0.f : m;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) l = fmaf(ex2_approx(s_ml[g][tid].x - mu), s_ml[g][tid].y, l);
    const bool there = tid < TOK * G && tile0 * TOK + tid / G < P.n_rows;
    const long long at = ((static_cast<long long>(part) * P.n_kv + kvh) * P.row_tiles + tile0) * PW_ROWS + tid;
    if (KVD_BOUNDS_OK(at < P.ml_size, P.status)) P.ml[at] = there ? make_float2(m, l) : make_float2(-CUDART_INF_F, 0.f);
  }
}

// The exponential on the fp32 pipes by itself (kvd_selftest_exp2), a pair per thread.
template <bool UPPER>
__global__ void kvd_selftest_exp2_kernel(const float2 *in, float2 *out, int pairs) {
  const int i = static_cast<int>(blockIdx.x * blockDim.x + threadIdx.x);
  if (i >= pairs) return;
  float2 v = in[i];
  unpack2(pw_ex2_poly<UPPER>(pack2(v.x, v.y)), v.x, v.y);
  out[i] = v;
}

// out_p = in_p + the partial columns of position p: 32 positions per CTA, PW_SUM warps over the partials, added in order.
constexpr int PW_SUM = 32;
__global__ void __launch_bounds__(PW_SUM * 32) kvd_prefill_weights_sum_kernel(const __grid_constant__ PwParams P) {
  grid_launch_dependents();
  grid_dependency_wait();
  __shared__ float s_part[PW_SUM][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, p = static_cast<int>(blockIdx.x) * 32 + lane, warps = static_cast<int>(blockDim.x) >> 5;
  const int n = P.ranges * P.n_kv;
  const long long width = static_cast<long long>(P.key_tiles) * PW_KEYS, col = p - static_cast<long long>(P.key_tile0) * PW_KEYS;
  float sum = 0.f;
  if (p < P.n_positions && col >= 0 && col < width) {
#pragma unroll 8
    for (int i = warp; i < n; i += warps) sum += KVD_BOUNDS_OK(i * width + col < P.cols_size, P.status) ? __ldcg(P.cols + i * width + col) : 0.f;
  }
  s_part[warp][lane] = sum;
  __syncthreads();
  if (warp == 0 && p < P.n_positions) {
    float w = 0.f;
    for (int i = 0; i < warps; ++i) w += s_part[i][lane];
    P.out[p] = (P.in ? P.in[p] : 0.f) + w;
  }
}

// Shapes of a call's launches and the scratch they need.  The shares a pass is cut into are those of least estimated time; the
// scratch is bounded by the sizes alone.  The estimate, in us, from the kernels' time lines: a CTA takes START before its first
// tile's scores are there, SWITCH between two row tiles and TILE for each pair of tiles; an SM that is full of CTAs takes TILE_SM.
struct PwPlan {
  int row_tiles, splits, chunk, range;
};
constexpr double PW_START = 4.0, PW_SWITCH = 0.6, PW_TILE = 1.3, PW_TILE_SM = 0.65, PW_TILE_256 = 0.85;
constexpr int PW_PLAN_SMS = 148;  // SMs of a B200 (the scratch is asked for without a device)
static int pw_row_tiles(int n_rows, int group) { return (n_rows + PW_ROWS / group - 1) / (PW_ROWS / group); }
static int pw_most_splits(long long items) { return static_cast<int>(items >= PW_PLAN_SMS ? 1 : 2 * PW_PLAN_SMS / items > 64 ? 64 : 2 * PW_PLAN_SMS / items); }
static int pw_most_ranges(int row_tiles) { return row_tiles <= PW_RANGE ? row_tiles : (row_tiles + PW_RANGE - 1) / PW_RANGE > PW_RANGE ? (row_tiles + PW_RANGE - 1) / PW_RANGE : PW_RANGE; }
// Time of `ctas` CTAs of `tiles` pairs of tiles in `rows` row tiles each, of which `share` are there to be done.
static double pw_estimate(int d_head, long long ctas, double rows, double tiles, double share) {
  const int per_sm = d_head == 256 ? 1 : 2;
  const double tile = d_head == 256 ? PW_TILE_256 : PW_TILE, tile_sm = d_head == 256 ? PW_TILE_256 : PW_TILE_SM;
  const double one = PW_START + rows * PW_SWITCH + tiles * tile;
  if (ctas <= PW_PLAN_SMS) return one;  // (the longest one has all of its tiles)
  const double full = one - tiles * tile + tiles * tile_sm * per_sm;  // beside another one
  if (share > 0.9) return full * ((ctas + per_sm * PW_PLAN_SMS - 1) / (per_sm * PW_PLAN_SMS));
  // uneven work (causal calls, windows): long CTAs start first, and a third of one is left when the others are done
  return ctas * share * ((PW_START + rows * PW_SWITCH) / per_sm + tiles * tile_sm) / PW_PLAN_SMS + 0.35 * full;
}
// seen_tiles: of the key tiles, those a row tile can see; share: of all pairs of tiles, those that see each other.
static PwPlan pw_plan(int d_head, int n_kv, int group, int n_rows, int key_tiles, int seen_tiles, double share) {
  PwPlan s;
  s.row_tiles = pw_row_tiles(n_rows, group);
  const long long items = static_cast<long long>(s.row_tiles) * n_kv;
  double best = 1e300;
  s.splits = 1;
  for (int n = 1; n <= pw_most_splits(items) && n <= seen_tiles; ++n) {
    const double t = pw_estimate(d_head, items * n, 1, (seen_tiles + n - 1) / n, 1.0) + 0.02 * n;
    if (t < best) best = t, s.splits = n;
  }
  best = 1e300;
  s.chunk = s.range = 1;
  for (int range = 1; range <= PW_RANGE; range = range < 4 ? range + 1 : range * 2) {
    const long long ranges = (s.row_tiles + range - 1) / range;
    if (ranges > pw_most_ranges(s.row_tiles) || (range > 1 && range > s.row_tiles)) continue;
    for (int chunk = 1; chunk <= PW_CHUNK && chunk <= key_tiles; ++chunk) {
      const double t = pw_estimate(d_head, ranges * n_kv * ((key_tiles + chunk - 1) / chunk), range, static_cast<double>(range) * chunk, share) + 0.01 * ranges;
      if (t < best) best = t, s.chunk = chunk, s.range = range;
    }
  }
  return s;
}
static size_t pw_up(size_t v) { return (v + 255) / 256 * 256; }
static size_t pw_ml_bytes(int n_kv, int row_tiles, int splits) { return pw_up(static_cast<size_t>(splits) * n_kv * row_tiles * PW_ROWS * sizeof(float2)); }

template <int D_HEAD, int G, int DT>
static kvd_status pw_launch(kvd_ctx *ctx, const PwParams &P, const PwMaps &M, cudaStream_t stream) {
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
  auto launch = [&](auto kern, long long grid, int threads, size_t smem, const auto &...args) {
    if (e != cudaSuccess) return;
    cfg.gridDim = dim3(static_cast<unsigned>(grid), 1, 1);
    cfg.blockDim = dim3(threads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    attr[0].val.programmaticStreamSerializationAllowed = serial_launch_mask() & 8 ? 0 : 1;
    e = cudaLaunchKernelEx(&cfg, kern, P, args...);
    if (e == cudaSuccess) ctx->launches += 1;
  };
  launch(rows, static_cast<long long>(P.row_tiles) * P.n_kv * P.splits, R::THREADS, R::SMEM_BYTES, M);
  launch(columns, static_cast<long long>(P.chunks) * P.ranges * P.n_kv, C::THREADS, C::SMEM_BYTES, M);
  // a warp for every eight partials, eight loads at once (fewer partials: eight warps)
  const int partials = P.ranges * P.n_kv, sum_warps = partials >= 8 * PW_SUM ? PW_SUM : partials >= 64 ? (partials + 7) / 8 : 8;
  launch(kvd_prefill_weights_sum_kernel, (P.n_positions + 31ll) / 32, 32 * sum_warps, 0);
  return e == cudaSuccess ? KVD_OK : cuda_fail(ctx, e, "launch prefill weights");
}
template <int D_HEAD>
static kvd_status pw_group(kvd_ctx *ctx, const PwParams &P, const PwMaps &M, int group, cudaStream_t stream) {
  switch (group * 2 + (ctx->dtype == KVD_DTYPE_F16)) {
    case 2: return pw_launch<D_HEAD, 1, 0>(ctx, P, M, stream);
    case 3: return pw_launch<D_HEAD, 1, 1>(ctx, P, M, stream);
    case 4: return pw_launch<D_HEAD, 2, 0>(ctx, P, M, stream);
    case 5: return pw_launch<D_HEAD, 2, 1>(ctx, P, M, stream);
    case 6: return pw_launch<D_HEAD, 3, 0>(ctx, P, M, stream);
    case 7: return pw_launch<D_HEAD, 3, 1>(ctx, P, M, stream);
    case 8: return pw_launch<D_HEAD, 4, 0>(ctx, P, M, stream);
    case 9: return pw_launch<D_HEAD, 4, 1>(ctx, P, M, stream);
    case 16: return pw_launch<D_HEAD, 8, 0>(ctx, P, M, stream);
    case 17: return pw_launch<D_HEAD, 8, 1>(ctx, P, M, stream);
    default: return KVD_ERR_SHAPE;
  }
}

}  // namespace kvd

using namespace kvd;

extern "C" kvd_status kvd_selftest_exp2(kvd_ctx *ctx, const float *in, float *out, int n, int upper, void *stream) {
  if (!ctx || n < 0 || n % 2 != 0) return KVD_ERR_INVALID_ARG;
  if (n == 0) return KVD_OK;
  if (!in || !out) return KVD_ERR_INVALID_ARG;
  if (((reinterpret_cast<uintptr_t>(in) | reinterpret_cast<uintptr_t>(out)) & 7u) != 0) return KVD_ERR_ALIGNMENT;
  const auto kern = upper ? kvd_selftest_exp2_kernel<true> : kvd_selftest_exp2_kernel<false>;
  kern<<<(n / 2 + 255) / 256, 256, 0, static_cast<cudaStream_t>(stream)>>>(reinterpret_cast<const float2 *>(in), reinterpret_cast<float2 *>(out), n / 2);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return cuda_fail(ctx, e, "launch selftest_exp2");
  ctx->launches += 1;
  return KVD_OK;
}

extern "C" size_t kvd_prefill_weights_scratch_bytes(const kvd_model_desc *d, int n_rows, int n_positions) {
  if (kvd_workspace_bytes(d) == 0 || n_rows <= 0 || n_positions <= 0 || n_positions > (1 << 30)) return 0;  // (checks the description)
  const int group = d->n_q_heads / d->n_kv_heads;
  if (n_rows > INT32_MAX - PW_ROWS || pw_row_tiles(n_rows, group) > INT32_MAX / PW_ROWS) return 0;
  const int row_tiles = pw_row_tiles(n_rows, group);
  const size_t width = (static_cast<size_t>(n_positions) + PW_KEYS - 1) / PW_KEYS * PW_KEYS;
  return pw_ml_bytes(d->n_kv_heads, row_tiles, pw_most_splits(static_cast<long long>(row_tiles) * d->n_kv_heads)) +
         pw_up(static_cast<size_t>(pw_most_ranges(row_tiles)) * d->n_kv_heads * width * sizeof(float));
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
  if ((reinterpret_cast<uintptr_t>(q) & 15u) != 0 || (reinterpret_cast<uintptr_t>(scratch) & 255u) != 0 || !aligned4({q_pos, weights_in, weights_out}))
    return KVD_ERR_ALIGNMENT;
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
    kvd_prefill_weights_sum_kernel<<<(n_positions + 31) / 32, 32, 0, stream>>>(P);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return cuda_fail(ctx, e, "launch prefill weights (sum)");
    ctx->launches += 1;
    return KVD_OK;
  }
  if (n_rows > INT32_MAX - PW_ROWS || pw_row_tiles(n_rows, group) > INT32_MAX / PW_ROWS) return KVD_ERR_CAPACITY;
  P.key_tile0 = P.seg_lo / PW_KEYS;
  P.key_tiles = P.seg_hi / PW_KEYS - P.key_tile0 + 1;
  // (a window hides all but so many tiles from a row tile whose tokens follow each other)
  const int row_span = (PW_ROWS + group - 1) / group;
  const int64_t reach = ls.window > 0 ? (static_cast<int64_t>(ls.window) + row_span) / PW_KEYS + 2 : P.key_tiles;  // (windows go up to INT32_MAX)
  const int seen = reach < P.key_tiles ? static_cast<int>(reach) : P.key_tiles;
  // (if the rows are the last of the keys' tokens)
  const double behind = n_rows < P.key_tiles * PW_KEYS ? static_cast<double>(n_rows) / (P.key_tiles * PW_KEYS) : 1.0;
  const double share = seen < P.key_tiles ? static_cast<double>(seen) / P.key_tiles : 1.0 - 0.5 * behind;
  const PwPlan plan = pw_plan(d.d_head, d.n_kv_heads, group, n_rows, P.key_tiles, seen, share);
  P.ranges = (plan.row_tiles + plan.range - 1) / plan.range;
  const size_t ml_bytes = pw_ml_bytes(d.n_kv_heads, plan.row_tiles, plan.splits);
  if (ml_bytes + static_cast<size_t>(P.ranges) * d.n_kv_heads * P.key_tiles * PW_KEYS * sizeof(float) > scratch_bytes) return KVD_ERR_CAPACITY;
  P.ml = static_cast<float2 *>(scratch);
  P.cols = reinterpret_cast<float *>(static_cast<uint8_t *>(scratch) + ml_bytes);
  P.ml_size = static_cast<long long>(ml_bytes / sizeof(float2));
  P.cols_size = static_cast<long long>((scratch_bytes - ml_bytes) / sizeof(float));
  static thread_local PwMaps M;
  {
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(d.d_head), static_cast<cuuint64_t>(d.n_q_heads), static_cast<cuuint64_t>(n_rows)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(d.d_head) * 2, static_cast<cuuint64_t>(d.n_q_heads) * d.d_head * 2};
    const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(group), static_cast<cuuint32_t>(PW_ROWS / group)}, ones[3] = {1, 1, 1};
    if (ctx->encode(&M.q, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(q), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return KVD_ERR_SHAPE;
  }
  for (int s = 0; s < KVD_MAX_SEGMENTS; ++s) {
    if (P.len[s] == 0) continue;
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(kdim), static_cast<cuuint64_t>(P.len[s])};
    const cuuint64_t strides[1] = {static_cast<cuuint64_t>(P.stride[s]) * 2};
    const cuuint32_t box[2] = {64, PW_KEYS}, ones[2] = {1, 1};
    if (P.stride[s] >= (1ll << 38) || ctx->encode(&M.k[s], CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<__nv_bfloat16 *>(P.k[s]), dims, strides, box, ones,
                                                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return KVD_ERR_SHAPE;  // (a tensor map's strides are below 2^40 bytes)
  }
  P.q = static_cast<const __nv_bfloat16 *>(q);
  P.q_pos = q_pos;
  P.n_rows = n_rows;
  P.n_q = d.n_q_heads;
  P.window = ls.window;
  P.scale_log2e = (scale > 0.f ? scale : 1.0f / sqrtf(static_cast<float>(d.d_head))) * 1.4426950408889634f;
  P.row_tiles = plan.row_tiles;
  P.splits = plan.splits;
  P.chunk = plan.chunk;
  P.chunks = (P.key_tiles + plan.chunk - 1) / plan.chunk;
  P.range = plan.range;
  P.status = ctx->d_status;
  P.timeout_ns = ctx->timeout_ns;
  switch (d.d_head) {
    case 64: return pw_group<64>(ctx, P, M, group, stream);
    case 128: return pw_group<128>(ctx, P, M, group, stream);
    case 256: return pw_group<256>(ctx, P, M, group, stream);
    default: return KVD_ERR_SHAPE;
  }
}
