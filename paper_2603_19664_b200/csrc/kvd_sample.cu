// Drawing tokens from a row's softmax under limits (kvd_scaffold_sample, kvd_scaffold.h).
//
// What stays under top-k, top-p and min-p is a prefix of the row in the order (logit descending, column ascending): everything above
// a threshold logit, and the first few columns of those equal to it.  A 16-bit logit has 65536 values at most, so the prefix is
// found without a sort: the CTAs of a cluster count the values of their shares of the row in shared memory, the values that occur are
// dealt out evenly, and running sums over them, from the largest, give the threshold; a value's mass is its count times one
// exponential.  A second walk over the row, in order of columns, adds the masses of what stays, looked up by value, and finds the column.
//
// 64 rows of 151936 bf16 logits, two CTAs a row: 41 us in a graph (19 MB, 3 us at the copy rate; fp16 52).  The counts take 17 of the 75 thousand clocks (a
// shared-memory atomic of random addresses 7 a warp: the banks' conflicts, twice), the second walk 20 where all columns stay
// (one look-up a column: 3.5 a warp, and as many issue slots), and some fifteen steps that end in a barrier over the CTA or the
// cluster 1 to 3 each: rows of 1000 take 18 us, and a single one of 49152 on eight CTAs 17 to 21.
//
// Masses are whole numbers, in units of 2^-44 of the largest logit's: sums of them are exact in any order, so that the token does not
// depend on how a row is cut, and a border between two tokens is off by 1e-11 of the mass (a token in a flat tail weighs
// 1e-5 of it; sums in 32 bits would take the wrong one of two neighbours once in some hundred rows).
#include <math_constants.h>
#include <string.h>

#include "../../include/kvd_scaffold.h"
#include "kvd_internal.h"
#include "kvd_pages.h"
#include "kvd_ptx.cuh"

namespace kvd {

constexpr int SM_THREADS = 1024, SM_WARPS = 32;
constexpr int SM_VALUES = 65536;             // of a 16-bit logit
constexpr int SM_HIST_BYTES = 2 * SM_VALUES;  // 16-bit counts
constexpr int SM_MAX_COUNT = 65535;
constexpr int SM_TURN = SM_MAX_COUNT / 8 * 8;  // columns that are counted without a count running over
constexpr int SM_RUN = 4096;                 // columns of a warp's run at most
static_assert(SM_RUN == 4 * SM_THREADS && SM_RUN * SM_WARPS >= 2 * SM_TURN, "a share is counted in two turns at most");
constexpr int SM_LIST = 14336;               // values of a CTA that its list holds: count, order key
constexpr unsigned SM_MANY = 1024;           // columns of a warp's run with one value that are counted apart
constexpr int SM_FEW = 256;                  // logits that stay whose exponentials are taken again instead
constexpr int SM_EIGHTS = SM_VALUES / 8 / 2;  // eights of counts of a CTA
constexpr int SM_SMEM = SM_HIST_BYTES + 6 * SM_LIST + 2 * SM_EIGHTS + 16;
constexpr int SM_MAGNITUDES = 24576;         // bits without the sign of what the table of masses has room for: fp16 below 512, bf16 below 2^65
static_assert(8 * SM_MAGNITUDES + 16 <= SM_SMEM - 2 * SM_LIST, "the table lies where counts were, below the list of keys");

struct SampleParams {
  const uint16_t *logits;
  long long stride;
  int n, share;  // columns, and those of a CTA
  const float *temperature, *top_p, *min_p, *u;
  const int32_t *top_k;
  int32_t *tokens;
  float *probs;
  int *status;
  unsigned long long timeout_ns;
};

// What the CTAs of a cluster tell each other; every CTA holds a copy.  Messages are 16 bytes (st.async) and counted by a barrier each.
struct SampleShared {
  unsigned char some[SM_VALUES / 64];  // which eights of 64 counts are not all zero
  unsigned full;                       // a count may have run over
  float best[8];                       // the largest logit of a CTA's share
  uint2 more[8];                       // a value of it that occurs more often than 65535 times (at most one does), and how much more
  unsigned any_more;                   // there is one
  uint64_t arrived[4];                 // barriers: sums, top-k, top-p, shares
  uint4 sums[8];                       // of a CTA's values: logits, the least value that min-p keeps and the entries of its list (16 bits
                                       // each; 65535: there is none), mass
  uint4 k, p;                          // the last value that stays, how many of those equal to it; the mass of what top-k keeps, the logits that
                                       // top-p does
  uint4 shares[8];                     // of a CTA's share: columns that equal the threshold, 0, mass of those above it
};
enum { SM_SUMS, SM_TOP_K, SM_TOP_P, SM_SHARES };

template <class T>
__device__ __forceinline__ T *peer(T *p, unsigned rank) {
  uint64_t a;
  asm("mapa.u64 %0, %1, %2;" : "=l"(a) : "l"(reinterpret_cast<uint64_t>(p)), "r"(rank));
  return reinterpret_cast<T *>(a);
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
// Until the other CTAs' threads have ended or come here too (of threads that have ended nothing is awaited); threads of a warp need not be together.
__device__ __forceinline__ void cluster_stay() { asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory"); }
// Until a barrier's messages have come; false: the time is up, or another thread's was.  Other CTAs complete it, so the wait acquires at
// cluster scope.
static __device__ __noinline__ bool await_slow(uint32_t bar, const volatile int *abort_flag, unsigned long long timeout_ns) {
  const unsigned long long t0 = globaltimer_ns();
  for (unsigned it = 1;; ++it) {
    if (mbar_try_wait_cluster(bar, 0)) return true;
    if ((it & 31u) == 0u && (*abort_flag != 0 || globaltimer_ns() - t0 > timeout_ns)) return false;
  }
}
__device__ __forceinline__ bool await(uint32_t bar, const volatile int *abort_flag, unsigned long long timeout_ns) {
#pragma unroll 1
  for (int i = 0; i < 16; ++i)
    if (mbar_try_wait_cluster(bar, 0)) return true;
  return await_slow(bar, abort_flag, timeout_ns);
}
// A message to all CTAs of the cluster
template <int CTAS>
__device__ __forceinline__ void tell(const uint4 *slot, const uint64_t *bar, unsigned a, unsigned b, uint64_t c) {
#pragma unroll
  for (int r = 0; r < CTAS; ++r)
    st_async_v4(map_to_cta(smem_u32(slot), r), map_to_cta(smem_u32(bar), r), a, b, static_cast<uint32_t>(c), static_cast<uint32_t>(c >> 32));
}
__device__ __forceinline__ uint64_t wide(const uint4 &m) { return m.z | static_cast<uint64_t>(m.w) << 32; }

// Order keys of values: unsigned order is numeric order.
template <int F16>
struct SampleKey {
  static constexpr unsigned INF = F16 ? 0x7c00u : 0x7f80u;
  static constexpr uint32_t NOTHING = (0x8000u | INF) * 0x10001u;  // two minus infinities: what is not there
  static constexpr unsigned LOWEST = 0xffffu ^ (0x8000u | INF);  // of minus infinity; NaN of either sign lie beyond the infinities
  static constexpr unsigned HIGHEST = 0x8000u | INF;
  static __device__ __forceinline__ unsigned bits(unsigned key) { return key & 0x8000u ? key ^ 0x8000u : 0xffffu ^ key; }
  static __device__ __forceinline__ float value(unsigned key) {
    if (F16) return __half2float(__ushort_as_half(static_cast<unsigned short>(bits(key))));
    return __uint_as_float(bits(key) << 16);
  }
};

// The masses of a row's values.
constexpr double SM_UNIT = 17592186044416.0;  // 2^44
// e^x, out of line: the kernel calls it from several places, and most warps pass them by
static __device__ __noinline__ double sample_exp(double x) { return exp(x); }
struct Weights {
  unsigned top_key;
  double top, inv_t;
  // e^((value - largest) / temperature)
  template <int F16>
  __device__ __forceinline__ double ratio(unsigned key) const {
    if (key == top_key) return 1.0;
    return top == CUDART_INF ? 0.0 : sample_exp((static_cast<double>(SampleKey<F16>::value(key)) - top) * inv_t);
  }
};
__device__ __forceinline__ uint64_t mass_of(double ratio) { return __double2ull_rn(ratio * SM_UNIT); }

// Masses by value, for walks over many columns: of what stays, 0 of what does not.  The table holds a mass's low 29 bits, in a direct order
// of the values (their bits with the sign behind them; a last entry, 0, for all beyond), so that a column costs one look into shared
// memory and eight of them add up in 32 bits.  What the high 16 are follows from an exponential that is good to 2^-18: 2^15 e^x less the
// low bits over 2^29 is a whole number up to 2^-3.  Few columns have any.
constexpr unsigned SM_BEYOND = 2 * SM_MAGNITUDES;
constexpr int SM_LOW = 29;
struct MassTable {
  const uint32_t *low;
  float top, scale;  // the largest logit, log2(e) / temperature
  // of two values
  static __device__ __forceinline__ uint32_t at2(uint32_t w) { return __vminu2((w * 2 & 0xfffefffeu) | (w >> 15 & 0x00010001u), SM_BEYOND * 0x10001u); }
  static __device__ __forceinline__ unsigned at(unsigned bits) { return min((bits << 1 | bits >> 15) & 0xffffu, SM_BEYOND); }
  __device__ __forceinline__ unsigned high(float x, uint32_t lo) const {
    const float lo_1 = __uint_as_float(0x3f800000u | lo >> (SM_LOW - 23));  // 1 + lo / 2^29
    return __float_as_uint(fmaf(ex2_approx((x - top) * scale), 32768.0f, 1.0f - lo_1) + 12582912.0f) - 0x4b400000u;  // (1.5 * 2^23: the sum is a whole number)
  }
};

// Inclusive running sums over the CTA's threads in their order; the total is that of the last thread.
__device__ __forceinline__ void running(unsigned &c, uint64_t &m, unsigned (&wc)[SM_WARPS], uint64_t (&wm)[SM_WARPS]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const unsigned a = __shfl_up_sync(0xffffffffu, c, d);
    const uint64_t b = __shfl_up_sync(0xffffffffu, m, d);
    if (lane >= d) {
      c += a;
      m += b;
    }
  }
  __syncthreads();  // (the sums of the call before have been read)
  if (lane == 31) {
    wc[warp] = c;
    wm[warp] = m;
  }
  __syncthreads();
  unsigned a = wc[lane];
  uint64_t b = wm[lane];
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const unsigned x = __shfl_up_sync(0xffffffffu, a, d);
    const uint64_t y = __shfl_up_sync(0xffffffffu, b, d);
    if (lane >= d) {
      a += x;
      b += y;
    }
  }
  if (warp > 0) {
    c += __shfl_sync(0xffffffffu, a, warp - 1);
    m += __shfl_sync(0xffffffffu, b, warp - 1);
  }
}
// the same of counts alone; returns the total
__device__ __forceinline__ unsigned running(unsigned &c, unsigned (&wc)[SM_WARPS]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const unsigned a = __shfl_up_sync(0xffffffffu, c, d);
    c += lane >= d ? a : 0;
  }
  __syncthreads();
  if (lane == 31) wc[warp] = c;
  __syncthreads();
  const unsigned w = wc[lane], total = __reduce_add_sync(0xffffffffu, w);
  c += __reduce_add_sync(0xffffffffu, lane < warp ? w : 0u);
  return total;
}

// Up to eight columns of a row, [at, end); minus infinities for those that are not there.
template <int F16>
__device__ __forceinline__ void load_eight(const uint16_t *row, int at, int end, uint32_t (&w)[4]) {
  if (at + 8 <= end && (reinterpret_cast<uintptr_t>(row + at) & 15u) == 0) {
    const uint4 x = *reinterpret_cast<const uint4 *>(row + at);
    w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      w[j] = SampleKey<F16>::NOTHING;
      if (at + 2 * j < end) w[j] = (w[j] & 0xffff0000u) | row[at + 2 * j];
      if (at + 2 * j + 1 < end) w[j] = (w[j] & 0xffffu) | static_cast<uint32_t>(row[at + 2 * j + 1]) << 16;
    }
  }
}
// Columns [c0, c1) of a row by a warp, eight to a lane and step, in order, four steps' loads at once: visit(their bits).  All lanes take
// part in every call.
template <int F16, class V>
__device__ __forceinline__ void walk(const uint16_t *row, int c0, int c1, int lane, V visit) {
#pragma unroll 1
  for (int c = c0; c < c1; c += 1024) {
    uint32_t w[4][4];
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (c + 256 * q < c1) load_eight<F16>(row, c + 256 * q + 8 * lane, c1, w[q]);
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (c + 256 * q < c1) visit(w[q]);
  }
}
__device__ __forceinline__ unsigned bits_of(const uint32_t (&w)[4], int j) { return j & 1 ? w[j / 2] >> 16 : w[j / 2] & 0xffffu; }
__device__ __forceinline__ unsigned pick_of(const uint32_t (&w)[4], int j) {  // (j not known at compile time)
  const uint32_t x = j < 4 ? (j < 2 ? w[0] : w[1]) : j < 6 ? w[2] : w[3];
  return x >> (16 * (j & 1)) & 0xffffu;
}
// the largest of eight columns; NaN is passed over
template <int F16>
__device__ __forceinline__ float largest_of(const uint32_t (&w)[4]) {
  if (F16) {
    const __half2 m = __hmax2(__hmax2(*reinterpret_cast<const __half2 *>(&w[0]), *reinterpret_cast<const __half2 *>(&w[1])),
                              __hmax2(*reinterpret_cast<const __half2 *>(&w[2]), *reinterpret_cast<const __half2 *>(&w[3])));
    return __half2float(__hmax(__low2half(m), __high2half(m)));
  }
  const __nv_bfloat162 m = __hmax2(__hmax2(*reinterpret_cast<const __nv_bfloat162 *>(&w[0]), *reinterpret_cast<const __nv_bfloat162 *>(&w[1])),
                                   __hmax2(*reinterpret_cast<const __nv_bfloat162 *>(&w[2]), *reinterpret_cast<const __nv_bfloat162 *>(&w[3])));
  return __bfloat162float(__hmax(__low2bfloat16(m), __high2bfloat16(m)));
}
template <int F16>
__device__ __forceinline__ float value_of(const uint32_t (&w)[4], int j) {
  if (F16) return __half2float(__ushort_as_half(static_cast<unsigned short>(bits_of(w, j))));
  return j & 1 ? bf16_hi(w[j / 2]) : bf16_lo(w[j / 2]);
}

template <int F16>
__device__ __forceinline__ float value_of_bits(unsigned b) {
  return F16 ? __half2float(__ushort_as_half(static_cast<unsigned short>(b))) : __uint_as_float(b << 16);
}

template <int F16, int CTAS>
__global__ void __launch_bounds__(SM_THREADS, 1) kvd_sample_kernel(const __grid_constant__ SampleParams P) {
  typedef SampleKey<F16> K;
  constexpr int EIGHTS = SM_VALUES / 8 / CTAS, EACH = EIGHTS / SM_THREADS, PER = 8 * EACH;  // a CTA's eights at most; a thread's without a list, and its values
  constexpr unsigned NONE = 0xffffffffu;
  extern __shared__ __align__(16) uint8_t smem[];
  uint32_t *hist = reinterpret_cast<uint32_t *>(smem);      // [bits / 2]: two 16-bit counts
  uint16_t *eights = reinterpret_cast<uint16_t *>(smem + SM_HIST_BYTES);  // eights of counts that are not all zero, the largest first
  uint32_t *list_count = reinterpret_cast<uint32_t *>(smem + SM_HIST_BYTES + 2 * SM_EIGHTS);  // the CTA's values that occur, the largest first
  uint16_t *list_key = reinterpret_cast<uint16_t *>(smem + SM_SMEM - 2 * SM_LIST);
  uint32_t *table = reinterpret_cast<uint32_t *>(smem);  // of masses, later
  __shared__ SampleShared S;
  __shared__ unsigned wc[SM_WARPS], s_ties[SM_WARPS];
  __shared__ uint64_t wm[SM_WARPS], s_above[SM_WARPS];
  __shared__ float s_best[SM_WARPS];
  __shared__ uint2 s_many[SM_WARPS];  // a value, and in how many columns of the warp's run
  __shared__ double s_inv_t;
  __shared__ uint64_t s_mass_t;
  __shared__ volatile int s_abort;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const unsigned rank = cluster_ctarank();
  const int r = blockIdx.x / CTAS;
  if (tid == 0) {
    s_abort = 0;
    for (int i = 0; i < 4; ++i) {
      mbar_init(smem_u32(&S.arrived[i]), 1);
      mbar_arrive_expect_tx(smem_u32(&S.arrived[i]), i == SM_SUMS || i == SM_SHARES ? 16 * CTAS : 16);
    }
    fence_mbar_init();
  }
  auto clear = [&]() {
#pragma unroll
    for (int i = 0; i < SM_HIST_BYTES / 16 / SM_THREADS; ++i) reinterpret_cast<uint4 *>(smem)[i * SM_THREADS + tid] = make_uint4(0, 0, 0, 0);
    if (tid < 8) S.more[tid] = make_uint2(0, 0);
    if (tid == 0) S.full = S.any_more = 0;
  };
  clear();
  grid_launch_dependents();
  grid_dependency_wait();
  const uint16_t *row = P.logits + static_cast<long long>(r) * P.stride;
  const float temp = P.temperature ? P.temperature[r] : 1.0f;
  const int asked_k = P.top_k ? P.top_k[r] : 0;
  const float asked_p = P.top_p ? P.top_p[r] : 1.0f, asked_m = P.min_p ? P.min_p[r] : 0.0f, u = P.u[r];
  const bool greedy = !(temp > 0.0f);
  const int share0 = min(P.n, static_cast<int>(rank) * P.share), share1 = min(P.n, share0 + P.share);
  // A CTA with a thread that has given up a wait keeps its memory until the others have ended: they still read it and send messages there.
  auto leave = [&]() {
    if (s_abort != 0) cluster_stay();
  };
  auto heard = [&](int what) {  // (a message that does not come: recorded, and the row has no token)
    if (await(smem_u32(&S.arrived[what]), &s_abort, P.timeout_ns)) return;
    raise(P.status, STATUS_TIMEOUT, &s_abort);
  };

  // ---- the counts: at once, or, where one of more than 65535 columns has run over all the same, in turns of so many.
  // Then the list of this CTA's values, from all CTAs' counts.
  // The eights of values whose counts are not all zero are dealt out evenly, in descending order over the cluster's CTAs.
  unsigned values = 0, n_eights = 0, cnt[PER];  // cnt: without a list
  // the values of eight `first / 8` in descending order
  auto bits_in = [](unsigned first, int o) { return first < 0x8000u ? first + 7 - o : first + o; };
  auto key_in = [&](unsigned first, int o) { return first < 0x8000u ? bits_in(first, o) | 0x8000u : 0xffffu ^ bits_in(first, o); };
  // all CTAs' counts of an eight; zeros of both signs are one value, NaN is none
  auto counts_of = [&](unsigned first, unsigned (&n)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) n[j] = 0;
#pragma unroll
    for (int p = 0; p < CTAS; ++p) {
      const uint4 x = reinterpret_cast<const uint4 *>(peer(hist, (rank + p) % CTAS))[first / 8];
      const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int j = 0; j < 8; ++j) n[j] += bits_of(w, j);
    }
    if (first == 0)
#pragma unroll
      for (int p = 0; p < CTAS; ++p) n[0] += peer(hist, p)[0x8000 / 2] & 0xffffu;
    if (S.any_more) {
#pragma unroll 1
      for (int p = 0; p < CTAS; ++p) {
        const uint2 x = S.more[p];
#pragma unroll
        for (int j = 0; j < 8; ++j) n[j] += first + j == x.x || (first + j == 0 && x.x == 0x8000u) ? x.y : 0u;
      }
    }
    if (first == 0x8000u) n[0] = 0;
    if ((first & 0x7fffu) + 7 > K::INF)
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (((first + j) & 0x7fffu) > K::INF) n[j] = 0;
  };
  bool has_list = true;
#pragma unroll 1
  for (int turns = 1;;) {
    const int turn_cols = turns == 1 ? P.share : SM_TURN;
#pragma unroll
    for (int j = 0; j < PER; ++j) cnt[j] = 0;
#pragma unroll 1
    for (int turn = 0; turn < turns; ++turn) {
      if (turns > 1) clear();
      cluster_arrive();  // (nobody writes here before it has begun and cleared)
      __syncthreads();
      const int t0 = min(share1, share0 + turn * turn_cols), t1 = min(share1, t0 + turn_cols);
      const int run = ((t1 - t0 + SM_WARPS - 1) / SM_WARPS + 7) / 8 * 8, r0 = min(t1, t0 + warp * run);
      unsigned counted = 0, common = NONE, same = 0;
      bool looked = false;
      float best = -CUDART_INF_F;
      // (minus infinity, which masks leave in numbers, is not counted.  A finite value that a mask leaves in numbers is counted in
      // registers: 32 atomics on one address take 32 turns.  64 rows with 140000 of 151936 columns masked 148 -> 49 us, others 39 -> 40.)
      walk<F16>(row, r0, min(t1, r0 + run), lane, [&](const uint32_t (&w)[4]) {
        best = fmaxf(best, largest_of<F16>(w));
        if (!looked) {
          looked = true;
          // (of the values of three lanes the one that most lanes have, if some do)
          const unsigned b = bits_of(w, 0);
          int most = 3;
#pragma unroll
          for (int l = 0; l < 32; l += 11) {
            const unsigned x = __shfl_sync(NONE, b, l);
            const int have = __popc(__ballot_sync(NONE, b == x));
            if (have > most && x != (0x8000u | K::INF)) {
              most = have;
              common = x;
            }
          }
        }
        if (common == NONE) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const unsigned b = bits_of(w, j);
            if (b != (0x8000u | K::INF)) {
              atomicAdd(hist + (b >> 1), 1u << ((b & 1u) * 16));
              ++counted;
            }
          }
        } else {
#pragma unroll 1
          for (int j = 0; j < 8; ++j) {  // (short code for the rarer case: tests in the other loop cost every call 3 %)
            const unsigned b = pick_of(w, j);
            if (b == common) {
              ++same;
            } else if (b != (0x8000u | K::INF)) {
              atomicAdd(hist + (b >> 1), 1u << ((b & 1u) * 16));
              ++counted;
            }
          }
        }
      });
#pragma unroll
      for (int d = 16; d >= 1; d /= 2) best = fmaxf(best, __shfl_xor_sync(NONE, best, d));
      same = __reduce_add_sync(NONE, same);
      if (lane == 0) {
        s_best[warp] = best;
        s_many[warp] = make_uint2(common, same >= SM_MANY ? same : 0u);
        counted += same;
        if (same > 0 && same < SM_MANY) atomicAdd(hist + (common >> 1), same << ((common & 1u) * 16));
      }
      uint2 more = make_uint2(0, 0);
      if (__syncthreads_or(same >= SM_MANY)) {
        if (warp == 0) {  // the warps' counts of a value come together; what does not fit 16 bits is kept apart
          const uint2 many = s_many[lane];
          const unsigned alike = __match_any_sync(NONE, many.y > 0 ? many.x : 0x10000u + lane);
          if (many.y > 0 && __ffs(alike) - 1 == lane) {
            uint16_t *count = reinterpret_cast<uint16_t *>(hist) + many.x;
            unsigned n = *count;
            for (unsigned m = alike; m; m &= m - 1) n += s_many[__ffs(m) - 1].y;
            *count = static_cast<uint16_t>(min(n, static_cast<unsigned>(SM_MAX_COUNT)));
            if (n > SM_MAX_COUNT) more = make_uint2(many.x, n - SM_MAX_COUNT);
          }
          more = make_uint2(__reduce_max_sync(NONE, more.x), __reduce_max_sync(NONE, more.y));
        }
        __syncthreads();
      }
      cluster_wait();
      if (warp == 0) {
        best = s_best[lane];
#pragma unroll
        for (int d = 16; d >= 1; d /= 2) best = fmaxf(best, __shfl_xor_sync(NONE, best, d));
        if (lane < CTAS) {
          peer(S.best, lane)[rank] = turn > 0 ? fmaxf(best, S.best[rank]) : best;
          if (more.y > 0) {
            peer(S.more, lane)[rank] = more;
            *peer(&S.any_more, lane) = 1;
          }
        }
      }
      // most of the values do not occur: what the others have to read of the counts
      unsigned some = 0, sum = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint4 x = reinterpret_cast<const uint4 *>(smem)[8 * tid + (j + tid) % 8];  // (in turns: no two lanes of eight on one bank)
        some |= (x.x | x.y | x.z | x.w) != 0 ? 1u << ((j + tid) % 8) : 0u;
        if (P.share > SM_MAX_COUNT)
          sum += (x.x & 0xffffu) + (x.x >> 16) + (x.y & 0xffffu) + (x.y >> 16) + (x.z & 0xffffu) + (x.z >> 16) + (x.w & 0xffffu) + (x.w >> 16);
      }
      S.some[tid] = static_cast<unsigned char>(some);
      if (turns == 1 && P.share > SM_MAX_COUNT) {
        // every count that runs over takes 65535 or 65536 off the sum
        const unsigned missing = __reduce_add_sync(NONE, counted - sum - (tid == 0 ? more.y : 0u));
        if (lane == 0) wc[warp] = missing;
        __syncthreads();
        if (warp == 0 && __reduce_add_sync(NONE, wc[lane]) != 0 && lane < CTAS) *peer(&S.full, lane) = 1;
      }
      cluster_arrive();
      if (turns == 1 && tid == 0) s_inv_t = greedy ? 0.0 : 1.0 / static_cast<double>(temp);  // (read behind later barriers)
      cluster_wait();
      if (turns == 1 && S.full == 0) {
        // the eights that are not all zero, from the largest values down: a thread looks at those of 64 values
        const unsigned key = SM_VALUES - 1 - 64 * tid, block = K::bits(key) / 64;
        unsigned mask = 0;
#pragma unroll
        for (int p = 0; p < CTAS; ++p) mask |= peer(S.some, p)[block];
        if (block == 0)  // (-0 counts as +0)
#pragma unroll
          for (int p = 0; p < CTAS; ++p) mask |= peer(S.some, p)[0x8000 / 64] & 1u;
        if (key >= 0x8000u) mask = __brev(mask) >> 24;  // positive values: the last eight is the largest
        unsigned to = __popc(mask);
        const unsigned mine = to, all_eights = running(to, wc), deal = (all_eights + CTAS - 1) / CTAS, from = min(all_eights, rank * deal);
        n_eights = min(all_eights, from + deal) - from;
        to -= mine + from;
        for (; mask; mask &= mask - 1, ++to) {
          const unsigned j = __ffs(mask) - 1;
          if (to < n_eights && KVD_BOUNDS_OK(to < EIGHTS, P.status)) eights[to] = static_cast<uint16_t>(block * 8 + (key >= 0x8000u ? 7 - j : j));
        }
        __syncthreads();
#pragma unroll 1
        for (unsigned e0 = 0; e0 < n_eights; e0 += SM_THREADS) {
          unsigned n[8] = {0, 0, 0, 0, 0, 0, 0, 0}, first = 0;
          if (e0 + tid < n_eights) {
            first = eights[e0 + tid] * 8;
            counts_of(first, n);
          }
          unsigned occurs = 0;
#pragma unroll
          for (int j = 0; j < 8; ++j) occurs |= n[j] ? 1u << j : 0u;
          unsigned at = __popc(occurs);
          const unsigned own = at, all = running(at, wc);
          at += values - own;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const unsigned before = first < 0x8000u ? occurs >> j >> 1 : occurs & ((1u << j) - 1);  // larger ones of the eight
            const unsigned to_j = at + __popc(before);
            if ((occurs >> j & 1u) && to_j < SM_LIST) {
              list_key[to_j] = static_cast<uint16_t>(first < 0x8000u ? (first + j) | 0x8000u : 0xffffu ^ (first + j));
              list_count[to_j] = n[j];
            }
          }
          values += all;
        }
        has_list = values <= SM_LIST;
      }
      if (turns > 1 || !has_list) {
        if (turns > 1) {  // (all eights of a fixed range: those that are zero differ from turn to turn)
          n_eights = EIGHTS;
#pragma unroll
          for (int j = 0; j < EACH; ++j) {
            const unsigned e = tid * EACH + j;
            eights[e] = static_cast<uint16_t>(K::bits(SM_VALUES - 1 - 8 * (rank * EIGHTS + e)) / 8);  // (its own thread's alone)
          }
        }
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
          unsigned n[8] = {0, 0, 0, 0, 0, 0, 0, 0}, first = 0;
          if (tid * EACH + j < n_eights) {
            first = eights[tid * EACH + j] * 8;
            counts_of(first, n);
          }
#pragma unroll
          for (int o = 0; o < 8; ++o) cnt[8 * j + o] += first < 0x8000u ? n[7 - o] : n[o];
        }
        has_list = false;
      }
      if (turn + 1 < turns) cluster_sync_all();
    }
    if (turns > 1 || S.full == 0) break;
    turns = (P.share + SM_TURN - 1) / SM_TURN;
    cluster_sync_all();
  }
  cluster_arrive();  // (this CTA's list can be read, and it reads no counts any more; the wait is ahead of the table)
  float top = S.best[0];
#pragma unroll
  for (int p = 1; p < CTAS; ++p) top = fmaxf(top, S.best[p]);
  if (top == -CUDART_INF_F) {  // nothing but minus infinities and NaN
    if (rank == 0 && tid == 0) {
      P.tokens[r] = 0;
      if (P.probs) P.probs[r] = 0.0f;
    }
    cluster_wait();
    return;
  }
  const unsigned top_bits = F16 ? __half_as_ushort(__float2half_rn(top)) : __float_as_uint(top) >> 16;
  const Weights W{top == 0.0f ? 0x8000u : top_bits & 0x8000u ? 0xffffu ^ top_bits : top_bits | 0x8000u, top, s_inv_t};
  __syncthreads();
  const int each = has_list ? (static_cast<int>(values) + SM_THREADS - 1) / SM_THREADS : 0, first = min(tid * each, static_cast<int>(values)),
            last = min(first + each, static_cast<int>(values));

  // ---- running counts and masses over the values, from the largest.  A thread has a few entries of the list, or, without one, its own values.
  const float min_p = greedy ? 0.0f : asked_m;
  unsigned c_own = 0, least = NONE;
  uint64_t m_own = 0;
  auto ratio_of = [&](unsigned key) { return greedy ? (key == W.top_key ? 1.0 : 0.0) : W.ratio<F16>(key); };
  auto count_at = [&](int j) {
    unsigned n = 0;
#pragma unroll
    for (int q = 0; q < PER; ++q) n = q == j ? cnt[q] : n;
    return n;
  };
  // the thread's values in order, until visit(key, count, ratio) answers true
  auto each_value = [&](auto visit) {
    const int n_own = has_list ? last - first : PER;
#pragma unroll 1
    for (int i = 0; i < n_own; ++i) {
      const unsigned n = has_list ? list_count[first + i] : count_at(i);
      const unsigned key = has_list ? list_key[first + i] : n > 0 ? key_in(eights[tid * EACH + i / 8] * 8u, i % 8) : 0u;
      if (n > 0 && visit(key, n, ratio_of(key))) return;
    }
  };
  each_value([&](unsigned key, unsigned n, double x) {
    c_own += n;
    m_own += n * mass_of(x);
    if (x >= static_cast<double>(min_p)) least = key;
    return false;
  });
  unsigned c_in = c_own;
  uint64_t m_in = m_own;
  least = __reduce_min_sync(NONE, least);
  if (lane == 0) s_ties[warp] = least;
  running(c_in, m_in, wc, wm);
  if (warp == SM_WARPS - 1) {
    least = __reduce_min_sync(NONE, s_ties[lane]);
    if (lane == 31) tell<CTAS>(&S.sums[rank], &S.arrived[SM_SUMS], c_in, (least & 0xffffu) | (has_list ? values : 0xffffu) << 16, m_in);
  }
  heard(SM_SUMS);
  unsigned c_all = 0;
  uint64_t m_all = 0;
  least = NONE;
#pragma unroll
  for (int p = 0; p < CTAS; ++p) {
    const uint4 x = S.sums[p];
    if (p == static_cast<int>(rank)) {
      c_in += c_all;
      m_in += m_all;
    }
    c_all += x.x;
    m_all += wide(x);
    if ((x.y & 0xffffu) != 0xffffu) least = min(least, x.y & 0xffffu);
  }
  const unsigned c_from = c_in - c_own;  // the thread's values are the logits c_from + 1 .. c_in, and the masses m_from + 1 .. m_in
  const uint64_t m_from = m_in - m_own;
  // ... with the mass of one, and the logits and the mass before it
  auto find = [&](auto visit) {
    unsigned c = c_from;
    uint64_t m = m_from;
    each_value([&](unsigned key, unsigned n, double ratio) {
      const uint64_t x = mass_of(ratio);
      if (visit(key, n, x, c, m)) return true;
      c += n;
      m += n * x;
      return false;
    });
  };

  // ---- top-k: the value that holds the k-th logit
  const int want_k = greedy ? 1 : asked_k;
  const bool some_k = want_k > 0 && static_cast<unsigned>(want_k) < c_all;
  uint64_t k_mass = m_all;
  unsigned key_t = 0, ties_t = NONE, stays = c_all;  // what stays: keys above key_t, ties_t of those equal to it; at most so many
  if (some_k) {
    const unsigned k = want_k;
    if (c_from < k && k <= c_in)
      find([&](unsigned key, unsigned n, uint64_t x, unsigned c, uint64_t m) {
        if (k > c + n) return false;
        tell<CTAS>(&S.k, &S.arrived[SM_TOP_K], key, k - c, m + (k - c) * x);
        return true;
      });
    heard(SM_TOP_K);
    const uint4 x = S.k;
    key_t = x.x;
    ties_t = x.y;
    k_mass = wide(x);
    stays = k;
  }

  // ---- top-p: the value at which the running mass reaches top_p of what top-k keeps
  if (!greedy && asked_p < 1.0f) {
    const uint64_t goal = __double2ull_ru(fmax(static_cast<double>(asked_p), 0.0) * __ull2double_rn(k_mass));
    const uint64_t target = goal > 1 ? goal : 1;
    if (m_from < target && target <= m_in)
      find([&](unsigned key, unsigned n, uint64_t x, unsigned c, uint64_t m) {
        if (target > m + n * x) return false;
        const unsigned ties = static_cast<unsigned>((target - m + x - 1) / x);
        tell<CTAS>(&S.p, &S.arrived[SM_TOP_P], key, ties, c + ties);
        return true;
      });
    heard(SM_TOP_P);
    const uint4 x = S.p;
    stays = min(stays, x.z);
    if (x.x > key_t) {
      key_t = x.x;
      ties_t = x.y;
    } else if (x.x == key_t) {
      ties_t = min(ties_t, x.y);
    }
  }

  // ---- min-p: the least value whose weight is min_p at least; one logit at least
  if (min_p > 0.0f) {
    if (least == NONE) {
      least = W.top_key;
      key_t = W.top_key;
      ties_t = 1;
    }
    if (least > key_t) {
      key_t = least;
      ties_t = NONE;
    }
  }

  // ---- what weighs less than 2^-45 is never drawn: it is at 32 temperatures below the largest one
  const bool usual = !greedy && top < CUDART_INF_F && temp > 0x1p-60f && temp < 0x1p+100f;  // (elsewhere the steps in 32 bits might leave their range)
  if (usual) {
    const float edge = fmaf(-32.0f, temp, top);
    const unsigned b = F16 ? __half_as_ushort(__float2half_rd(edge)) : __bfloat16_as_ushort(__float2bfloat16_rd(edge));
    const unsigned key = b & 0x8000u ? 0xffffu ^ b : b | 0x8000u;
    if (key > K::LOWEST && key > key_t) {
      key_t = key;
      ties_t = NONE;
    }
  }

  const bool all_ties = ties_t == NONE;
  // ---- where many stay, their masses go into a table, in every CTA (a few exponentials are taken again)
  bool tabled = usual && stays > SM_FEW;
#pragma unroll
  for (int p = 0; p < CTAS; ++p) tabled = tabled && S.sums[p].y >> 16 != 0xffffu;
  cluster_wait();
  // (one answer for all threads, and none of them reads counts any more: the table lies where they are)
  tabled = !__syncthreads_or(!tabled || s_abort != 0);
  if (tabled) {
    bool outside = false;
    // (the last value, where some of those equal to it do not stay, has no mass in the table)
#pragma unroll 1
    for (int p = 0; p < CTAS; ++p) {
      const uint16_t *keys = peer(list_key, (rank + p) % CTAS);
      const int n = S.sums[(rank + p) % CTAS].y >> 16;
#pragma unroll 1
      for (int i0 = tid; i0 < n; i0 += 4 * SM_THREADS) {
        unsigned key[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) key[q] = i0 + q * SM_THREADS < n ? keys[i0 + q * SM_THREADS] : 0u;
#pragma unroll 1
        for (int q = 0; q < 4; ++q) {
          const unsigned k = q < 2 ? (q == 0 ? key[0] : key[1]) : q == 2 ? key[2] : key[3];
          if (k == 0) break;
          const unsigned b = K::bits(k);
          const bool stay = k > key_t || (k == key_t && all_ties);
          if ((b & 0x7fffu) >= SM_MAGNITUDES) {
            outside |= stay;
            continue;
          }
          const uint32_t low = stay ? static_cast<uint32_t>(mass_of(W.ratio<F16>(k))) & ((1u << SM_LOW) - 1) : 0u;
          table[MassTable::at(b)] = low;
          if (b == 0) table[MassTable::at(0x8000u)] = low;
        }
      }
    }
    if (tid == 0) table[SM_BEYOND] = 0;
    tabled = !__syncthreads_or(outside);  // (all CTAs have seen the same lists)
  }
  const MassTable M{table, top, static_cast<float>(s_inv_t * 1.4426950408889634)};
  const float value_high = fmaf(-10.4f, temp, top);  // what is less weighs less than 2^-15: its high bits are zero
  const float value_t = key_t > K::LOWEST ? K::value(key_t) : -CUDART_INF_F;
  if (warp == SM_WARPS - 1) {
    const uint64_t x = key_t > K::LOWEST ? mass_of(greedy ? 1.0 : W.ratio<F16>(key_t)) : 0;
    if (lane == 0) s_mass_t = x;  // (read behind the next barrier)
  }
  auto mass_at = [&](unsigned b) -> uint64_t {  // of a logit above the threshold
    if (tabled) {
      const uint32_t lo = M.low[MassTable::at(b)];
      return lo + (static_cast<uint64_t>(M.high(value_of_bits<F16>(b), lo)) << SM_LOW);
    }
    const unsigned key = b == 0x8000u ? 0x8000u : b & 0x8000u ? 0xffffu ^ b : b | 0x8000u;
    return mass_of(greedy ? 1.0 : W.ratio<F16>(key));
  };

  // ---- masses of what stays, in order of columns: of the warps' runs, the shares ...
  const int run = ((share1 - share0 + SM_WARPS - 1) / SM_WARPS + 7) / 8 * 8, c0 = min(share1, share0 + warp * run), c1 = min(share1, c0 + run);
  uint64_t above = 0;
  unsigned ties = 0, above_high = 0;
  walk<F16>(row, c0, c1, lane, [&](const uint32_t (&w)[4]) {
    const float largest = largest_of<F16>(w);
    if (!__any_sync(NONE, largest >= value_t)) return;
    if (tabled) {
      uint32_t lo[8];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t at = MassTable::at2(w[j]);
        lo[2 * j] = M.low[at & 0xffffu];
        lo[2 * j + 1] = M.low[at >> 16];
      }
      above += ((lo[0] + lo[1]) + (lo[2] + lo[3])) + ((lo[4] + lo[5]) + (lo[6] + lo[7]));
      if (__any_sync(NONE, largest >= value_high)) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float x = value_of<F16>(w, j);
          if (x > value_t || (x == value_t && all_ties)) above_high += M.high(x, lo[j]);
        }
      }
      if (!all_ties) {
#pragma unroll
        for (int j = 0; j < 8; ++j) ties += value_of<F16>(w, j) == value_t;
      }
    } else {
      unsigned higher = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float x = value_of<F16>(w, j);
        if (x > value_t) higher |= 1u << j;
        if (x == value_t && x > -CUDART_INF_F) ++ties;
      }
#pragma unroll 1
      for (; higher; higher &= higher - 1) above += mass_at(pick_of(w, __ffs(higher) - 1));
    }
  });
  above += static_cast<uint64_t>(above_high) << SM_LOW;
#pragma unroll
  for (int d = 16; d >= 1; d /= 2) above += __shfl_xor_sync(NONE, above, d);
  ties = __reduce_add_sync(NONE, ties);
  if (lane == 0) {
    s_ties[warp] = ties;
    s_above[warp] = above;
  }
  __syncthreads();
  const uint64_t mass_t = s_mass_t;
  // (a warp's lanes look at all warps' sums)
  uint64_t above_in = s_above[lane];
  unsigned ties_in = s_ties[lane];
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const uint64_t x = __shfl_up_sync(NONE, above_in, d);
    const unsigned y = __shfl_up_sync(NONE, ties_in, d);
    above_in += lane >= d ? x : 0;
    ties_in += lane >= d ? y : 0;
  }
  if (tid == 31) tell<CTAS>(&S.shares[rank], &S.arrived[SM_SHARES], ties_in, 0, above_in);
  heard(SM_SHARES);
  // ... of those equal to the threshold the first ones stay; and where u of all falls
  uint64_t total = 0, share_from = 0;
  unsigned left = ties_t, share_left = 0;
  uint64_t reach[CTAS];
#pragma unroll
  for (int p = 0; p < CTAS; ++p) {
    const uint4 x = S.shares[p];
    if (p == static_cast<int>(rank)) {
      share_from = total;
      share_left = left;
    }
    const unsigned n = min(left, x.x);
    total += wide(x) + n * mass_t;
    reach[p] = total;
    left -= n;
  }
  // (below the total, so that the running mass exceeds it somewhere: at the last logit with a mass if u is 1)
  const uint64_t asked = __double2ull_rd(fmin(fmax(static_cast<double>(u), 0.0), 1.0) * __ull2double_rn(total)), target = asked < total ? asked : total - 1;
  // the share, and in it the run, where the running mass first exceeds the target
  int owner = -1;
#pragma unroll
  for (int p = CTAS - 1; p >= 0; --p) owner = reach[p] > target ? p : owner;
  if (owner != static_cast<int>(rank)) {
    leave();
    return;
  }
  const uint64_t run_in = share_from + above_in + min(ties_in, share_left) * mass_t;  // up to the end of run `lane`
  const int own = __ffs(__ballot_sync(NONE, run_in > target)) - 1;
  if (own < 0) {  // (a message did not come)
    leave();
    return;
  }
  uint64_t m = own > 0 ? __shfl_sync(NONE, run_in, own - 1) : share_from;
  unsigned quota = share_left;
  const unsigned ties_before = own > 0 ? __shfl_sync(NONE, ties_in, own - 1) : 0u;
  quota = quota > ties_before ? quota - ties_before : 0u;
  // all threads look at that run, a column each and turn
  const int o0 = min(share1, share0 + own * run), o1 = min(share1, o0 + run);
  uint32_t column[SM_RUN / SM_THREADS];
#pragma unroll
  for (int q = 0; q < SM_RUN / SM_THREADS; ++q) column[q] = o0 + q * SM_THREADS + tid < o1 ? row[o0 + q * SM_THREADS + tid] : K::NOTHING & 0xffffu;
#pragma unroll 1
  for (int q = 0; o0 + q * SM_THREADS < o1; ++q) {
    const unsigned b = q < 2 ? (q == 0 ? column[0] : column[1]) : q == 2 ? column[2] : column[3];
    const float x = value_of_bits<F16>(b);
    const bool tie = x == value_t && x > -CUDART_INF_F;
    const uint64_t mine = x > value_t ? mass_at(b) : 0;
    const unsigned tied = __ballot_sync(NONE, tie);
    unsigned ties_up = __popc(tied & (NONE >> (31 - lane)));
    uint64_t above_up = mine;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const uint64_t y = __shfl_up_sync(NONE, above_up, d);
      above_up += lane >= d ? y : 0;
    }
    __syncthreads();  // (the sums before have been read)
    if (lane == 31) {
      s_ties[warp] = ties_up;
      s_above[warp] = above_up;
    }
    __syncthreads();
    unsigned warp_ties = s_ties[lane];
    uint64_t warp_above = s_above[lane];
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const unsigned x = __shfl_up_sync(NONE, warp_ties, d);
      const uint64_t y = __shfl_up_sync(NONE, warp_above, d);
      warp_ties += lane >= d ? x : 0;
      warp_above += lane >= d ? y : 0;
    }
    if (warp > 0) {
      ties_up += __shfl_sync(NONE, warp_ties, warp - 1);
      above_up += __shfl_sync(NONE, warp_above, warp - 1);
    }
    // up to this column, and to the one before
    const uint64_t mass = tie && ties_up <= quota ? mass_t : mine, upto = m + above_up + min(ties_up, quota) * mass_t;
    if (upto > target && upto - mass <= target) {
      P.tokens[r] = o0 + q * SM_THREADS + tid;
      if (P.probs) P.probs[r] = static_cast<float>(__ull2double_rn(mass) / __ull2double_rn(total));
    }
    const unsigned n = min(__shfl_sync(NONE, warp_ties, 31), quota);
    const uint64_t all = __shfl_sync(NONE, warp_above, 31);
    m += all + n * mass_t;
    quota -= n;
  }
  leave();
}

}  // namespace kvd

using namespace kvd;

// A launch of m rows.  cudaFuncSetAttribute goes before it, and before the question how many clusters the device holds.
template <int F16, int CTAS>
struct SampleLaunch {
  cudaLaunchConfig_t cfg;
  cudaLaunchAttribute attr[2];
  cudaError_t error;
  SampleLaunch(const kvd_ctx *ctx, int m, cudaStream_t stream) {
    static std::atomic<bool> configured[64] = {};
    error = opt_in_smem(ctx, kvd_sample_kernel<F16, CTAS>, SM_SMEM, configured);
    memset(&cfg, 0, sizeof(cfg));
    cfg.gridDim = dim3(m * CTAS, 1, 1);
    cfg.blockDim = dim3(SM_THREADS, 1, 1);
    cfg.dynamicSmemBytes = SM_SMEM;
    cfg.stream = stream;
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = CTAS;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = (serial_launch_mask() & 8) || 2 * m * CTAS > ctx->num_sms ? 0 : 1;  // (as launch_dependent)
    cfg.attrs = attr;
    cfg.numAttrs = 2;
  }
};

template <int F16, int CTAS>
static cudaError_t launch_sample(kvd_ctx *ctx, const SampleParams &P, int m, cudaStream_t stream) {
  const SampleLaunch<F16, CTAS> L(ctx, m, stream);
  return L.error != cudaSuccess ? L.error : cudaLaunchKernelEx(&L.cfg, kvd_sample_kernel<F16, CTAS>, P);
}

// How many rows the device works on at once with that many CTAs each (asked once per device; 0 where it does not say).  A cluster lies within one of the
// device's groups of SMs, so these are fewer than SMs over CTAs: of 148 SMs 15 with eight, 33 with four.  One more row waits for a second turn: 16 rows of
// 49152 logits 41.3 us with eight CTAs each, 20.5 with four; 34 of 151936 53.9 with four, 39.6 with two.
template <int F16, int CTAS>
static int rows_at_once(const kvd_ctx *ctx) {
  static std::atomic<int> known[64] = {};  // one more than the answer
  std::atomic<int> &mine = known[ctx->device & 63];
  int n = mine.load(std::memory_order_relaxed);
  if (n == 0) {
    const SampleLaunch<F16, CTAS> L(ctx, 1, nullptr);
    if (L.error != cudaSuccess || cudaOccupancyMaxActiveClusters(&n, kvd_sample_kernel<F16, CTAS>, &L.cfg) != cudaSuccess) {
      cudaGetLastError();
      return 0;
    }
    mine.store(++n, std::memory_order_relaxed);
  }
  return n - 1;
}
template <int F16>
static int ctas_of_a_row(const kvd_ctx *ctx, int m) {
  return m <= rows_at_once<F16, 8>(ctx) ? 8 : m <= rows_at_once<F16, 4>(ctx) ? 4 : 2;
}

extern "C" kvd_status kvd_scaffold_sample(kvd_ctx *ctx, const void *logits, int64_t row_stride, int m, int n, const float *temperature, const int32_t *top_k,
                                          const float *top_p, const float *min_p, const float *u, int32_t *tokens_out, float *probs_out, void *stream_) {
  if (!ctx || m < 0 || n <= 0) return KVD_ERR_INVALID_ARG;
  if (ctx->dtype == KVD_DTYPE_F32) return KVD_ERR_UNSUPPORTED;
  if (m == 0) return KVD_OK;
  if (!logits || !u || !tokens_out || row_stride < n) return KVD_ERR_INVALID_ARG;
  if (m > 65535 || n > KVD_MAX_SAMPLE_VOCAB) return KVD_ERR_CAPACITY;
  if ((reinterpret_cast<uintptr_t>(logits) & 1u) != 0 || !aligned4({temperature, top_k, top_p, min_p, u, tokens_out, probs_out})) return KVD_ERR_ALIGNMENT;
  const OnDevice here(ctx);
  // eight CTAs per row, or four, where the device has room for all rows at once, else two; but no more columns for a CTA than two turns of counting
  // take
  const bool f16 = ctx->dtype == KVD_DTYPE_F16;
  int ctas = f16 ? ctas_of_a_row<1>(ctx, m) : ctas_of_a_row<0>(ctx, m);
  while (ctas < 8 && static_cast<int64_t>(ctas) * 2 * SM_TURN < n) ctas *= 2;
  SampleParams P;
  P.logits = static_cast<const uint16_t *>(logits);
  P.stride = row_stride;
  P.n = n;
  P.share = ((n + ctas - 1) / ctas + 7) / 8 * 8;
  P.temperature = temperature;
  P.top_p = top_p;
  P.min_p = min_p;
  P.u = u;
  P.top_k = top_k;
  P.tokens = tokens_out;
  P.probs = probs_out;
  P.status = ctx->d_status;
  P.timeout_ns = ctx->timeout_ns;
  cudaStream_t stream = static_cast<cudaStream_t>(stream_);
  cudaError_t e;
  if (ctas == 2) e = f16 ? launch_sample<1, 2>(ctx, P, m, stream) : launch_sample<0, 2>(ctx, P, m, stream);
  else if (ctas == 4) e = f16 ? launch_sample<1, 4>(ctx, P, m, stream) : launch_sample<0, 4>(ctx, P, m, stream);
  else e = f16 ? launch_sample<1, 8>(ctx, P, m, stream) : launch_sample<0, 8>(ctx, P, m, stream);
  if (e != cudaSuccess) return cuda_fail(ctx, e, "launch sample");
  ctx->launches += 1;
  return KVD_OK;
}
