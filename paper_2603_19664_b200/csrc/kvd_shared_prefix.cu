// Attention of a batch to the prefix that its sequences share (include/kvd.h, kvd_shared_prefix_attention): Eq. 6-7 with the
// prefix's keys and values read from memory once for the whole batch.
//
//   rows  = (sequence, head of the group) of one KV head, 128 per tile (G = 3: 42 sequences, two rows stay empty); a CTA takes NT tiles (two where there are two and
//           tensor memory holds both), a KV head and a share of the prefix, and leaves one partial (maximum, sum,
//           unnormalised output) per row, which the merge kernel of decode attention joins with those of the sequence's own
//           keys.
//   keys  = blocks of BK (128, at d_head 256 64), K and V in turns through a ring that TMA fills (64-channel slabs, 128-byte
//           swizzle; past the prefix's end it fills zeros, which are masked).  The query tiles come by TMA, too.
//   S     = Q K^T into tensor memory, four warps per row tile: a thread has a row, takes its maximum, then its weights, 32 columns
//           at a time, and puts the weights, in the element type, over the scores as the A operand of O += P V.
//   order = one thread issues all products.  One row tile: two score buffers, S runs a block ahead of the softmax.  Two row
//           tiles: one each, and a tile's products run during the other's softmax.
//
// Bound by reading the prefix as long as a block's arithmetic is shorter than its bytes take: per 128 keys of d_head 128 an
// SM's share of memory is 2900 clocks, the products of two row tiles 2048.  The weights' reference moves only when a
// block's maximum exceeds it by 2^8 (as in the prefill kernels), so O is rarely rescaled.
//
// The kernel leaves room on its SM -- registers, shared memory -- for CTAs of the streaming kernel that attends the sequences' own
// keys: that kernel is launched behind this one and starts beside it (AttnLaunchHead::beside), the merge behind both.
//
// Alone: 32749 keys of a Gemma-3-4B layer (fp16, 8 sequences) 30 us, 134 MB at 4.5 TB/s; 8192 keys of a Qwen3-4B layer (64 sequences)
// 26.5 us with 64 CTAs, 18.8 with 144, whose partials cost the merge more (13.2 against 5.6 us) than they save beside the own keys' 24.
#include <math_constants.h>
#include <string.h>

#include <type_traits>

#include "kvd_internal.h"
#include "kvd_ptx.cuh"

namespace kvd {

constexpr int SP_ROWS = 128;
constexpr float SP_TAU = 8.0f;

template <int D_HEAD, int NT>
struct SpCfg {
  static constexpr int BK = D_HEAD == 256 ? 64 : 128;    // keys per block
  static constexpr int THREADS = NT * 128 + 64;          // softmax warps, one that loads, one that issues products
  static constexpr int SLAB = BK * 128;                  // 64 channels of a block
  static constexpr int BLOCK_BYTES = BK * D_HEAD * 2;
  static constexpr int Q_BYTES = SP_ROWS * D_HEAD * 2;   // a row tile
  static constexpr int SLAB_Q = SP_ROWS * 128;
  static constexpr int S_BUFS = NT == 2 ? 1 : 2;         // per row tile
  static constexpr int COL_O = 0, COL_S = NT * D_HEAD;
  static constexpr int COLS_USED = COL_S + NT * S_BUFS * BK;
  static constexpr int COLS = COLS_USED <= 256 ? 256 : 512;
  static constexpr int SLOTS = D_HEAD == 64 ? 6 : NT == 2 ? 3 : 4;  // (about half of shared memory, 60 KB to spare at d_head 256)
  static constexpr int N_BARS = 2 * SLOTS + NT * (2 * S_BUFS + 3);
  static constexpr int SMEM_BYTES = 1024 + NT * Q_BYTES + SLOTS * BLOCK_BYTES + N_BARS * 8;
  static_assert(COLS_USED <= 512 && SLOTS >= 3, "does not fit");
};

__device__ __forceinline__ bool sp_wait(uint32_t bar, uint32_t parity, const volatile int *abort_flag, unsigned long long timeout_ns) {
  if (mbar_try_wait(bar, parity)) return true;
  const unsigned long long t0 = globaltimer_ns();
  uint32_t it = 0;
  while (!mbar_try_wait(bar, parity)) {
    __nanosleep(20);
    if (((++it) & 31u) == 0u && (*abort_flag != 0 || globaltimer_ns() - t0 > timeout_ns)) return false;
  }
  return true;
}
__device__ __forceinline__ bool sp_warp_wait(uint32_t bar, uint32_t parity, const volatile int *abort_flag, unsigned long long timeout_ns, int lane) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  int ok = 1;
  if (lane == 0) ok = sp_wait(bar, parity, abort_flag, timeout_ns) ? 1 : 0;
  ok = __shfl_sync(0xffffffffu, ok, 0);
  __syncwarp();
  return ok != 0;
}

struct SpMaps {
  CUtensorMap q;     // [sequences][n_q][d_head], boxes of 64 channels, a group's heads and a tile's sequences
  CUtensorMap k, v;  // [len][n_kv * d_head], boxes of 64 channels and a block's keys
};

// The unnormalised output of one row (its first query value at q) over the keys a .. b of the prefix that it sees, in fp32, by a warp:
// a lane has D_HEAD / 32 channels.  For rows whose tile has met a value that is not finite (below).
template <int D_HEAD, int DT>
__device__ __noinline__ void sp_redo_row(const SharedPrefixParams &P, const __nv_bfloat16 *q, int kvh, int a, int b, float mu, float *out, int lane) {
  constexpr int W = D_HEAD / 64;  // words of a lane's channels
  typedef typename std::conditional<W == 1, uint32_t, typename std::conditional<W == 2, uint2, uint4>::type>::type Words;
  union Piece {
    Words all;
    uint32_t w[W];
  };
  const long long first = static_cast<long long>(kvh) * D_HEAD + lane * 2 * W;
  Piece piece;
  uint64_t x[W], o[W];
  piece.all = *reinterpret_cast<const Words *>(q + lane * 2 * W);
#pragma unroll
  for (int i = 0; i < W; ++i) {
    x[i] = x2_to_f32x2<DT>(piece.w[i]);
    o[i] = 0ull;
  }
#pragma unroll 1
  for (int j = a; j <= b; ++j) {
    piece.all = *reinterpret_cast<const Words *>(P.k + j * P.stride + first);
    uint64_t dot = 0ull;
#pragma unroll
    for (int i = 0; i < W; ++i) dot = ffma2(x2_to_f32x2<DT>(piece.w[i]), x[i], dot);
    float s0, s1;
    unpack2(dot, s0, s1);
    s0 += s1;
#pragma unroll
    for (int i = 16; i >= 1; i >>= 1) s0 += __shfl_xor_sync(0xffffffffu, s0, i);
    const float p = ex2_approx(fmaf(s0, P.scale_log2e, -mu));
    piece.all = *reinterpret_cast<const Words *>(P.v + j * P.stride + first);
#pragma unroll
    for (int i = 0; i < W; ++i) o[i] = ffma2(pack2(p, p), x2_to_f32x2<DT>(piece.w[i]), o[i]);
  }
#pragma unroll
  for (int i = 0; i < W; ++i) {
    float2 f;
    unpack2(o[i], f.x, f.y);
    reinterpret_cast<float2 *>(out + lane * 2 * W)[i] = f;
  }
}

template <int D_HEAD, int G, int DT, int NT>
__global__ void __launch_bounds__(SpCfg<D_HEAD, NT>::THREADS, 1)
    kvd_shared_prefix_kernel(const __grid_constant__ SharedPrefixParams P, const __grid_constant__ SpMaps M) {
  using Cfg = SpCfg<D_HEAD, NT>;
  constexpr int BK = Cfg::BK, SLOTS = Cfg::SLOTS, S_BUFS = Cfg::S_BUFS;
  constexpr int SEQS = SP_ROWS / G;  // sequences of a row tile (G = 3: 42, and two rows stay empty)
  extern __shared__ uint8_t sp_smem_raw[];
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort_i;
  volatile int *s_abort = &s_abort_i;
  const uint32_t q_smem = (smem_u32(sp_smem_raw) + 1023u) & ~1023u;  // the swizzle is a function of the address
  const uint32_t ring = q_smem + NT * Cfg::Q_BYTES;
  const uint32_t bar_base = ring + SLOTS * Cfg::BLOCK_BYTES;
  auto bar_full = [&](int s) { return bar_base + 8u * s; };             // a block has landed
  auto bar_empty = [&](int s) { return bar_base + 8u * (SLOTS + s); };  // its products are done
  const uint32_t bar_t = bar_base + 8u * (2 * SLOTS);
  auto bar_s_full = [&](int t, int b) { return bar_t + 8u * (t * (2 * S_BUFS + 3) + b); };            // scores of a block
  auto bar_p_ready = [&](int t, int b) { return bar_t + 8u * (t * (2 * S_BUFS + 3) + S_BUFS + b); };  // weights in place
  auto bar_pv_done = [&](int t) { return bar_t + 8u * (t * (2 * S_BUFS + 3) + 2 * S_BUFS); };         // O += P V finished
  auto bar_o = [&](int t) { return bar_t + 8u * (t * (2 * S_BUFS + 3) + 2 * S_BUFS + 2); };           // the last one finished
  auto bar_q = [&](int t) { return bar_t + 8u * (t * (2 * S_BUFS + 3) + 2 * S_BUFS + 1); };           // the query tile is in place
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const unsigned long long tmo = P.timeout_ns;
  // row groups of one share are neighbours in the grid: the second one finds the blocks in L2
  const int groups = (P.row_tiles + NT - 1) / NT;
  const int group = static_cast<int>(blockIdx.x) % groups, kvh = static_cast<int>(blockIdx.x) / groups % P.n_kv, split = static_cast<int>(blockIdx.x) / groups / P.n_kv;
  const int blk_a = static_cast<int>(static_cast<long long>(P.n_blk) * split / P.splits), blk_b = static_cast<int>(static_cast<long long>(P.n_blk) * (split + 1) / P.splits);
  const int key0 = P.key0 + blk_a * BK, n_blk = blk_b - blk_a;  // (at least one)
  if (tid == 0) {
    for (int s = 0; s < SLOTS; ++s) {
      mbar_init(bar_full(s), 1);
      mbar_init(bar_empty(s), 1);
    }
    for (int t = 0; t < NT; ++t) {
      for (int b = 0; b < S_BUFS; ++b) {
        mbar_init(bar_s_full(t, b), 1);
        mbar_init(bar_p_ready(t, b), 4);
      }
      mbar_init(bar_pv_done(t), 1);
      mbar_init(bar_o(t), 1);
      mbar_init(bar_q(t), 1);
    }
    fence_mbar_init();
    s_abort_i = 0;
    prefetch_tensormap(&M.q);
    prefetch_tensormap(&M.k);
    prefetch_tensormap(&M.v);
  }
  if (warp == 4 * NT) {
    tmem_claim(smem_u32(&s_tmem), Cfg::COLS);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  // dependents are let in behind the wait: the streaming kernel relies on it that what precedes this kernel is complete
  grid_dependency_wait();
  grid_launch_dependents();
  const uint32_t tmem_base = s_tmem;

  if (warp < 4 * NT) {
    // ------------------------------------------------------------------ softmax: thread = row
    const int t = warp >> 2, q4 = warp & 3, in_tile = q4 * 32 + lane;
    const uint32_t lane_field = static_cast<uint32_t>(q4 * 32) << 16;
    const bool valid = in_tile < SEQS * G && (group * NT + t) * SEQS + in_tile / G < P.seqs;
    const int seq = valid ? (group * NT + t) * SEQS + in_tile / G : 0, head = kvh * G + (valid ? in_tile % G : 0);
    const int lo = valid ? P.lo[seq] : 0, hi = valid ? P.hi[seq] : -1;  // the prefix's keys that the row sees
    const int all_lo = __reduce_max_sync(0xffffffffu, valid ? lo : INT_MIN), all_hi = __reduce_min_sync(0xffffffffu, valid ? hi : INT_MAX);
    const uint64_t c2 = pack2(P.scale_log2e, P.scale_log2e), one2 = pack2(1.0f, 1.0f);
    float m = -CUDART_INF_F;
    uint64_t l2[2] = {0ull, 0ull};
    bool ok = true;
    for (int j = 0; j < n_blk; ++j) {
      const int buf = j % S_BUFS, k0 = key0 + j * BK;
      const uint32_t s_col = tmem_base + lane_field + Cfg::COL_S + (t * S_BUFS + buf) * BK;
      if (!sp_warp_wait(bar_s_full(t, buf), (j / S_BUFS) & 1, s_abort, tmo, lane)) {
        raise(P.status, STATUS_TIMEOUT, s_abort);
        ok = false;
        break;
      }
      tc_fence_after();
      const bool whole = k0 >= all_lo && k0 + BK - 1 <= all_hi;
      auto scores_of = [&](int i, uint32_t (&s)[32]) {
        tmem_ld_x32(s_col + i * 32, s);
        tmem_wait_ld();
        if (!whole) {
#pragma unroll
          for (int k = 0; k < 32; ++k)
            if (k0 + i * 32 + k < lo || k0 + i * 32 + k > hi) s[k] = 0xff800000u;  // -inf
        }
      };
      float mx[2] = {-CUDART_INF_F, -CUDART_INF_F};
#pragma unroll 1
      for (int i = 0; i < BK / 32; ++i) {
        uint32_t s[32];
        scores_of(i, s);
#pragma unroll
        for (int k = 0; k < 32; k += 4) {
          mx[0] = fmax3(mx[0], __uint_as_float(s[k]), __uint_as_float(s[k + 1]));
          mx[1] = fmax3(mx[1], __uint_as_float(s[k + 2]), __uint_as_float(s[k + 3]));
        }
      }
      const float bm = fmaxf(mx[0], mx[1]) * P.scale_log2e;  // (scale > 0)
      const float m_new = m == -CUDART_INF_F ? bm : (bm > m + SP_TAU ? bm : m);
      const float mu = m_new == -CUDART_INF_F ? 0.f : m_new;
      const float alpha = m == -CUDART_INF_F ? 1.0f : ex2_approx(m - mu);  // while nothing has been seen O and l are 0
      m = m_new;
      const uint64_t al2 = pack2(alpha, alpha), nm2 = pack2(-mu, -mu);
      l2[0] = fmul2(l2[0], al2);
      l2[1] = fmul2(l2[1], al2);
#pragma unroll 1
      for (int i = 0; i < BK / 32; ++i) {
        uint32_t s[32], w[16];
        scores_of(i, s);
#pragma unroll
        for (int k = 0; k < 32; k += 2) {
          float e0, e1;
          unpack2(ffma2(pack2(__uint_as_float(s[k]), __uint_as_float(s[k + 1])), c2, nm2), e0, e1);
          const float p0 = ex2_approx(e0), p1 = ex2_approx(e1);
          w[k >> 1] = pack_out<DT>(p0, p1);
          l2[(k >> 1) & 1] = ffma2(pack2(p0, p1), one2, l2[(k >> 1) & 1]);
        }
        tmem_st_x16(s_col + i * 16, w);  // over scores that have been read: columns 16 i .. of 32 i ..
      }
      if (__any_sync(0xffffffffu, alpha != 1.0f)) {
        // O holds the blocks before j; the last of those products must have finished (j >= 1 here: a maximum exists)
        if (!sp_warp_wait(bar_pv_done(t), (j - 1) & 1, s_abort, tmo, lane)) {
          raise(P.status, STATUS_TIMEOUT, s_abort);
          ok = false;
          break;
        }
        tc_fence_after();
#pragma unroll 1
        for (int c = 0; c < D_HEAD / 32; ++c) {
          uint32_t r[32];
          const uint32_t col = tmem_base + lane_field + Cfg::COL_O + t * D_HEAD + c * 32;
          tmem_ld_x32(col, r);
          tmem_wait_ld();
#pragma unroll
          for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * alpha);
          tmem_st_x32(col, r);
        }
      }
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_p_ready(t, buf));
    }
    // ---- the partial: unnormalised output, maximum, sum
    if (ok && !sp_warp_wait(bar_o(t), 0, s_abort, tmo, lane)) {
      raise(P.status, STATUS_TIMEOUT, s_abort);
      ok = false;
    }
    if (ok) {
      tc_fence_after();
      const long long slot = valid ? static_cast<long long>(P.slot[seq]) + split : 0;
      const bool store = valid && KVD_BOUNDS_OK(slot >= 0 && slot < P.max_parts, P.status);
      const long long at = slot * P.n_q + head;
      // A product takes in all keys of a block, those that a row does not see with weight 0: a value there that is not finite makes
      // the row's output a NaN (0 times infinity).  Rows that see less than the CTA's keys are looked through for it, and taken
      // again over the keys that they see.
      const int last = min(key0 + n_blk * BK, P.len) - 1;
      const bool in_part = valid && (lo > key0 || hi < last);
      bool odd = false;
#pragma unroll 1
      for (int c = 0; c < D_HEAD / 32; ++c) {
        uint32_t r[32];
        tmem_ld_x32(tmem_base + lane_field + Cfg::COL_O + t * D_HEAD + c * 32, r);
        tmem_wait_ld();
        if (in_part) {
#pragma unroll
          for (int i = 0; i < 32; ++i) odd |= (r[i] & 0x7f800000u) == 0x7f800000u;
        }
        if (store) {
          // (32 bytes at a time: whole sectors, whose halves would be written one by one otherwise)
          store_row_piece<8>(reinterpret_cast<__nv_bfloat16 *>(P.part_o + at * D_HEAD + c * 32), r, true);
        }
      }
      float a0, a1, a2, a3;
      unpack2(l2[0], a0, a1);
      unpack2(l2[1], a2, a3);
      if (store) *reinterpret_cast<float2 *>(P.part_ml + at * 2) = make_float2(m, (a0 + a1) + (a2 + a3));
      __syncwarp();
      for (uint32_t rows = __ballot_sync(0xffffffffu, odd && store); rows != 0u; rows &= rows - 1u) {
        const int of = __ffs(static_cast<int>(rows)) - 1;
        const int seq_of = __shfl_sync(0xffffffffu, seq, of), head_of = __shfl_sync(0xffffffffu, head, of);
        const float m_of = __shfl_sync(0xffffffffu, m, of);
        const int a = max(key0, __shfl_sync(0xffffffffu, lo, of)), b = min(last, __shfl_sync(0xffffffffu, hi, of));
        const long long at_of = __shfl_sync(0xffffffffu, at, of);
        sp_redo_row<D_HEAD, DT>(P, P.q + (static_cast<long long>(seq_of) * P.n_q + head_of) * D_HEAD, kvh, a, b, m_of == -CUDART_INF_F ? 0.f : m_of,
                                P.part_o + at_of * D_HEAD, lane);
      }
    }
  } else if (warp == 4 * NT) {
    // ------------------------------------------------------------------ products (one thread)
    constexpr uint32_t IDESC_BASE = (DT == 0 ? umma_idesc_bf16_f32(128, 8) : umma_idesc_f16_f32(128, 8)) & ~(1u << 17);
    constexpr uint32_t IDESC_S = IDESC_BASE | (static_cast<uint32_t>(BK >> 3) << 17);                   // N = keys, B K-major
    constexpr uint32_t IDESC_O = IDESC_BASE | (static_cast<uint32_t>(D_HEAD >> 3) << 17) | (1u << 16);  // N = d_head, B MN-major
    if (lane == 0) {
      bool ok = true;
      // ring entries: K of block j is 2 j, V of block j is 2 j + 1
      auto landed = [&](int e) { return sp_wait(bar_full(e % SLOTS), (e / SLOTS) & 1, s_abort, tmo); };
      auto scores = [&](int t, int j) {
        const uint64_t qdesc = umma_smem_desc_sw128(q_smem + t * Cfg::Q_BYTES), kdesc = umma_smem_desc_sw128(ring + (2 * j) % SLOTS * Cfg::BLOCK_BYTES);
        const uint32_t d = tmem_base + Cfg::COL_S + (t * S_BUFS + j % S_BUFS) * BK;
#pragma unroll
        for (int ks = 0; ks < D_HEAD / 16; ++ks)
          umma_bf16(d, qdesc + (((ks >> 2) * Cfg::SLAB_Q + (ks & 3) * 32) >> 4), kdesc + (((ks >> 2) * Cfg::SLAB + (ks & 3) * 32) >> 4), IDESC_S, ks > 0 ? 1u : 0u);
        if (t == NT - 1) umma_commit(bar_empty((2 * j) % SLOTS));
        umma_commit(bar_s_full(t, j % S_BUFS));
      };
      auto values = [&](int t, int j) {
        const uint64_t vdesc = umma_smem_desc_sw128_mn(ring + (2 * j + 1) % SLOTS * Cfg::BLOCK_BYTES, Cfg::SLAB);
        const uint32_t p = tmem_base + Cfg::COL_S + (t * S_BUFS + j % S_BUFS) * BK;
#pragma unroll
        for (int ks = 0; ks < BK / 16; ++ks)
          umma_f16_ts(tmem_base + Cfg::COL_O + t * D_HEAD, p + ks * 8, vdesc + ((ks * 16 * 128) >> 4), IDESC_O, (j > 0 || ks > 0) ? 1u : 0u);
        if (t == NT - 1) umma_commit(bar_empty((2 * j + 1) % SLOTS));
        umma_commit(bar_pv_done(t));
      };
      for (int t = 0; ok && t < NT; ++t) ok = sp_wait(bar_q(t), 0, s_abort, tmo);
      for (int j = 0; ok && j < S_BUFS && j < n_blk; ++j) {
        ok = landed(2 * j);
        if (ok) {
          tc_fence_after();
          for (int t = 0; t < NT; ++t) scores(t, j);
        }
      }
      for (int j = 0; ok && j < n_blk; ++j) {
        const int next = j + S_BUFS;  // its scores overwrite the weights of block j, behind the product that reads them
        ok = landed(2 * j + 1);
        for (int t = 0; ok && t < NT; ++t) {
          ok = sp_wait(bar_p_ready(t, j % S_BUFS), (j / S_BUFS) & 1, s_abort, tmo);
          if (!ok) break;
          tc_fence_after();
          values(t, j);
          if (next < n_blk) {
            ok = landed(2 * next);
            if (!ok) break;
            tc_fence_after();
            scores(t, next);
          }
        }
      }
      // (of pv_done a parity would not tell the last two phases apart: two blocks can be on their way at the end)
      for (int t = 0; ok && t < NT; ++t) umma_commit(bar_o(t));
      if (!ok) raise(P.status, STATUS_TIMEOUT, s_abort);
    }
  } else if (lane == 0) {
    // ------------------------------------------------------------------ blocks into the ring (one thread)
    bool ok = true;
    for (int t = 0; t < NT; ++t) {
      mbar_arrive_expect_tx(bar_q(t), SEQS * G * D_HEAD * 2);
#pragma unroll
      for (int c = 0; c < D_HEAD / 64; ++c)
        tma_load_3d(q_smem + t * Cfg::Q_BYTES + c * Cfg::SLAB_Q, &M.q, bar_q(t), c * 64, kvh * G, (group * NT + t) * SEQS);
    }
    int e = 0;
    for (; e < 2 * n_blk; ++e) {
      const int slot = e % SLOTS;
      if (e >= SLOTS && !sp_wait(bar_empty(slot), (e / SLOTS - 1) & 1, s_abort, tmo)) {
        ok = false;
        break;
      }
      mbar_arrive_expect_tx(bar_full(slot), Cfg::BLOCK_BYTES);
      const int key = key0 + (e >> 1) * BK;
#pragma unroll
      for (int c = 0; c < D_HEAD / 64; ++c)
        tma_load_2d(ring + slot * Cfg::BLOCK_BYTES + c * Cfg::SLAB, (e & 1) ? &M.v : &M.k, bar_full(slot), kvh * D_HEAD + c * 64, key);
    }
    if (!ok) {
      raise(P.status, STATUS_TIMEOUT, s_abort);
      // the copies in flight land before the CTA's shared memory goes to another
      const volatile int never = 0;
      for (int t = 0; t < NT; ++t) sp_wait(bar_q(t), 0, &never, tmo);
      for (int i = e < SLOTS ? 0 : e - SLOTS; i < e; ++i) {
        const unsigned long long t0 = globaltimer_ns();
        while (!mbar_try_wait(bar_full(i % SLOTS), (i / SLOTS) & 1) && globaltimer_ns() - t0 < tmo) __nanosleep(20);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 4 * NT) {
    tc_fence_after();
    tmem_dealloc(tmem_base, Cfg::COLS);
  }
}

// Merge of a launch of many rows with a few dozen partials each, a thread for four channels of a row: the partials in slot
// order, eight at a time, with a running maximum.  (The merge of decode attention gives a CTA to a head group and a slice of
// channels, whose registers leave three CTAs on an SM: 64 sequences of 32 heads of 128, 21 partials each, 13 us.)
constexpr int SP_MERGE_THREADS = 256;
template <int D_HEAD, int DT>
__global__ void __launch_bounds__(SP_MERGE_THREADS) kvd_shared_merge_kernel(const __grid_constant__ SharedMergeParams P) {
  grid_launch_dependents();
  grid_dependency_wait();
  constexpr int PER_ROW = D_HEAD / 4, BATCH = 8;
  const int at = static_cast<int>(blockIdx.x) * SP_MERGE_THREADS + static_cast<int>(threadIdx.x), row = at / PER_ROW, c = at % PER_ROW;
  if (row >= P.n_seqs * P.n_q) return;
  const int seq = row / P.n_q, head = row % P.n_q, count = P.count[seq];
  const size_t first = static_cast<size_t>(P.base[seq]) * P.n_q + head;
  const float2 *ml = reinterpret_cast<const float2 *>(P.part_ml) + first;
  const float4 *po = reinterpret_cast<const float4 *>(P.part_o + first * D_HEAD) + c;
  float m = -CUDART_INF_F, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int p0 = 0; p0 < count; p0 += BATCH) {
    float2 x[BATCH];
    float4 v[BATCH];
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const size_t off = static_cast<size_t>(p0 + i < count ? p0 + i : count - 1) * P.n_q;
      x[i] = __ldcg(ml + off);
      v[i] = __ldcg(po + off * PER_ROW);
      if (p0 + i >= count) x[i].x = -CUDART_INF_F;
    }
    float mn = m;
#pragma unroll
    for (int i = 0; i < BATCH; ++i) mn = fmaxf(mn, x[i].x);
    const float mu = mn == -CUDART_INF_F ? 0.f : mn, f = exp2f(m - mu);
    m = mn;
    l *= f;
    o.x *= f;
    o.y *= f;
    o.z *= f;
    o.w *= f;
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const float w = exp2f(x[i].x - mu);
      if (p0 + i >= count) continue;
      l = fmaf(w, x[i].y, l);
      o.x = fmaf(w, v[i].x, o.x);
      o.y = fmaf(w, v[i].y, o.y);
      o.z = fmaf(w, v[i].z, o.z);
      o.w = fmaf(w, v[i].w, o.w);
    }
  }
  const float r = l > 0.f ? 1.0f / l : 0.f;  // (nothing seen: zeros)
  reinterpret_cast<uint2 *>(P.out)[at] = make_uint2(pack_out<DT>(o.x * r, o.y * r), pack_out<DT>(o.z * r, o.w * r));
}
// Where a wave of such CTAs is there to be filled, and no live keys are left to the merge.
bool shared_prefix_merges(const kvd_ctx *ctx, const AttnLaunch &L, int d_head) {
  return !L.tail && static_cast<long long>(L.n_seqs) * L.n_q * (d_head / 4) >= static_cast<long long>(ctx->num_sms) * SP_MERGE_THREADS;
}
kvd_status launch_shared_merge(kvd_ctx *ctx, const AttnLaunch &L, int d_head, cudaStream_t stream) {
  static thread_local SharedMergeParams P;
  P.part_o = L.part_o;
  P.part_ml = L.part_ml;
  P.out = L.out;
  P.n_seqs = L.n_seqs;
  P.n_q = L.n_q;
  for (int i = 0; i < L.n_seqs; ++i) {
    if (L.seq[i].merge_base < 0 || L.seq[i].merge_base + L.seq[i].merge_count > L.max_parts) return KVD_ERR_CAPACITY;
    P.base[i] = L.seq[i].merge_base;
    P.count[i] = L.seq[i].merge_count;
  }
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof(cfg));
  cfg.stream = stream;
  cfg.gridDim = dim3((L.n_seqs * L.n_q * (d_head / 4) + SP_MERGE_THREADS - 1) / SP_MERGE_THREADS, 1, 1);
  cfg.blockDim = dim3(SP_MERGE_THREADS, 1, 1);
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = serial_launch_mask() & 4 ? 0 : 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const bool f16 = ctx->dtype == KVD_DTYPE_F16;
  cudaError_t e;
  switch (d_head) {
    case 64: e = f16 ? cudaLaunchKernelEx(&cfg, kvd_shared_merge_kernel<64, 1>, P) : cudaLaunchKernelEx(&cfg, kvd_shared_merge_kernel<64, 0>, P); break;
    case 128: e = f16 ? cudaLaunchKernelEx(&cfg, kvd_shared_merge_kernel<128, 1>, P) : cudaLaunchKernelEx(&cfg, kvd_shared_merge_kernel<128, 0>, P); break;
    case 256: e = f16 ? cudaLaunchKernelEx(&cfg, kvd_shared_merge_kernel<256, 1>, P) : cudaLaunchKernelEx(&cfg, kvd_shared_merge_kernel<256, 0>, P); break;
    default: return KVD_ERR_SHAPE;
  }
  if (e != cudaSuccess) return cuda_fail(ctx, e, "launch shared merge");
  ctx->launches += 1;
  return KVD_OK;
}

// Blocks of keys and the row tiles of a CTA, by head size.
int shared_prefix_block(int d_head) { return d_head == 256 ? 64 : 128; }
int shared_prefix_tiles(int d_head, int row_tiles) { return d_head <= 128 && row_tiles > 1 ? 2 : 1; }

template <int D_HEAD, int G, int DT, int NT>
static kvd_status sp_launch(kvd_ctx *ctx, const SharedPrefixParams &P, const SpMaps &M, cudaStream_t stream) {
  using Cfg = SpCfg<D_HEAD, NT>;
  auto kern = kvd_shared_prefix_kernel<D_HEAD, G, DT, NT>;
  static std::atomic<bool> configured[64] = {};
  cudaError_t e = opt_in_smem(ctx, kern, Cfg::SMEM_BYTES, configured);
  if (e != cudaSuccess) return cuda_fail(ctx, e, "cudaFuncSetAttribute(shared prefix)");
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof(cfg));
  cfg.stream = stream;
  cfg.gridDim = dim3(static_cast<unsigned>((P.row_tiles + NT - 1) / NT) * P.n_kv * P.splits, 1, 1);
  cfg.blockDim = dim3(Cfg::THREADS, 1, 1);
  cfg.dynamicSmemBytes = Cfg::SMEM_BYTES;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = serial_launch_mask() & 2 ? 0 : 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, kern, P, M);
  if (e != cudaSuccess) return cuda_fail(ctx, e, "launch shared prefix");
  ctx->launches += 1;
  return KVD_OK;
}
template <int D_HEAD, int G>
static kvd_status sp_dtype(kvd_ctx *ctx, const SharedPrefixParams &P, const SpMaps &M, cudaStream_t stream) {
  const bool f16 = ctx->dtype == KVD_DTYPE_F16;
  if constexpr (D_HEAD <= 128) {
    if (shared_prefix_tiles(D_HEAD, P.row_tiles) == 2) return f16 ? sp_launch<D_HEAD, G, 1, 2>(ctx, P, M, stream) : sp_launch<D_HEAD, G, 0, 2>(ctx, P, M, stream);
  }
  return f16 ? sp_launch<D_HEAD, G, 1, 1>(ctx, P, M, stream) : sp_launch<D_HEAD, G, 0, 1>(ctx, P, M, stream);
}
template <int D_HEAD>
static kvd_status sp_group(kvd_ctx *ctx, const SharedPrefixParams &P, int group, const SpMaps &M, cudaStream_t stream) {
  switch (group) {
    case 1: return sp_dtype<D_HEAD, 1>(ctx, P, M, stream);
    case 2: return sp_dtype<D_HEAD, 2>(ctx, P, M, stream);
    case 3: return sp_dtype<D_HEAD, 3>(ctx, P, M, stream);
    case 4: return sp_dtype<D_HEAD, 4>(ctx, P, M, stream);
    case 8: return sp_dtype<D_HEAD, 8>(ctx, P, M, stream);
    default: return KVD_ERR_SHAPE;
  }
}
kvd_status launch_shared_prefix(kvd_ctx *ctx, const SharedPrefixParams &P, const kvd_kv_segment &prefix, int d_head, int group, cudaStream_t stream) {
  static thread_local SpMaps M;
  const cuuint32_t ones[3] = {1, 1, 1};
  const cuuint64_t q_dims[3] = {static_cast<cuuint64_t>(d_head), static_cast<cuuint64_t>(P.n_q), static_cast<cuuint64_t>(P.seqs)};
  const cuuint64_t q_strides[2] = {static_cast<cuuint64_t>(d_head) * 2, static_cast<cuuint64_t>(P.n_q) * d_head * 2};
  const cuuint32_t q_box[3] = {64, static_cast<cuuint32_t>(group), static_cast<cuuint32_t>(SP_ROWS / group)};
  bool ok = ctx->encode(&M.q, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<__nv_bfloat16 *>(P.q), q_dims, q_strides, q_box, ones,
                        CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  for (int i = 0; ok && i < 2; ++i) {
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(P.n_kv) * d_head, static_cast<cuuint64_t>(prefix.len)};
    const cuuint64_t strides[1] = {static_cast<cuuint64_t>(prefix.row_stride) * 2};
    const cuuint32_t box[2] = {64, static_cast<cuuint32_t>(shared_prefix_block(d_head))};
    ok = ctx->encode(i ? &M.v : &M.k, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(i ? prefix.v : prefix.k), dims, strides, box, ones,
                     CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  }
  if (!ok) return KVD_ERR_SHAPE;
  switch (d_head) {
    case 64: return sp_group<64>(ctx, P, group, M, stream);
    case 128: return sp_group<128>(ctx, P, group, M, stream);
    case 256: return sp_group<256>(ctx, P, group, M, stream);
    default: return KVD_ERR_SHAPE;
  }
}

}  // namespace kvd
