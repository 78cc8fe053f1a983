// A cache held in 4 bits (kvd.h, kvd_pages.h): writing it, reading it back, and decode attention over it.
#include <string.h>

#include "kvd_internal.h"
#include "kvd_pages.h"
#include "kvd_ptx.cuh"

namespace kvd {

// ------------------------------------------------------------------------------------------------ codes
// Eight codes of +-{0, .5, 1, 1.5, 2, 3, 4, 6}, nearest, ties to the even code, saturating: that of f[j] in bits 4 j
__device__ __forceinline__ uint32_t e2m1_codes(const float (&f)[8]) {
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\tcvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\tmov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r)
      : "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]), "f"(f[5]), "f"(f[6]), "f"(f[7]));
  return r;
}
// the eight numbers of a word as four pairs of fp16
__device__ __forceinline__ void e2m1_word(uint32_t w, uint32_t (&h)[4]) {
  asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\tcvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(w));
}
__device__ __forceinline__ float2 h2f(uint32_t h) { return __half22float2(*reinterpret_cast<const __half2 *>(&h)); }

constexpr uint32_t C4_NAN = 0x7fffu;          // scale of a block with a value that is not finite
constexpr float C4_MAX_SCALE = 64512.0f;      // 63 * 2^10: the largest fp16 of 6 significant bits

// 18 significant bits of a quotient that was taken as the product with a rounded reciprocal (off by 2^-22 at most), so that one that lies on
// a border between two choices gets there.  One that does not is off the border by 2^-12 of itself at least: the dividend has 11 bits,
// a border times the divisor 10.  True divisions cost eight more instructions a value.
__device__ __forceinline__ float c4_quotient(float x, float inv) { return __uint_as_float((__float_as_uint(x * inv) + 0x20u) & ~0x3fu); }
// The scale of a block from its largest magnitude: max / 6 to 6 significant bits, ties to even.
__device__ __forceinline__ uint16_t c4_scale(float most) {
  const uint32_t u = __float_as_uint(c4_quotient(most, 1.0f / 6.0f));
  const float r = __uint_as_float((u + 0x1ffffu + ((u >> 18) & 1u)) & ~0x3ffffu);
  const uint16_t s = __half_as_ushort(__float2half_rn(fminf(r, C4_MAX_SCALE)));
  return most < INFINITY ? s : C4_NAN;
}
// the larger magnitude of two pairs of 16-bit numbers, NaN before all
template <int F16>
__device__ __forceinline__ uint32_t abs_max2(uint32_t a, uint32_t b) {
  if (F16) {
    const __half2 m = __hmax2_nan(__habs2(*reinterpret_cast<const __half2 *>(&a)), __habs2(*reinterpret_cast<const __half2 *>(&b)));
    return *reinterpret_cast<const uint32_t *>(&m);
  }
  const __nv_bfloat162 m = __hmax2_nan(__habs2(*reinterpret_cast<const __nv_bfloat162 *>(&a)), __habs2(*reinterpret_cast<const __nv_bfloat162 *>(&b)));
  return *reinterpret_cast<const uint32_t *>(&m);
}

template <int F16>
__device__ __forceinline__ float2 unpack16(uint32_t w) {
  if (F16) return h2f(w);
  return make_float2(bf16_lo(w), bf16_hi(w));
}
template <int F16>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
  if (F16) {
    const __half2 h = __floats2half2_rn(fminf(fmaxf(lo, -65504.0f), 65504.0f), fminf(fmaxf(hi, -65504.0f), 65504.0f));
    const uint32_t w = *reinterpret_cast<const uint32_t *>(&h);
    // (the limits swallow NaN)
    return (lo != lo ? 0x7fffu : w & 0xffffu) | (hi != hi ? 0x7fff0000u : w & 0xffff0000u);
  }
  return pack_bf16(lo, hi);
}

// ------------------------------------------------------------------------------------------------ writing and reading back
template <int N>
struct C4Rows {
  uint8_t *pool;             // of the layer
  const int32_t *table, *lens, *first;
  const uint4 *k, *v;        // rows in 16-byte pieces: 8 channels
  uint4 *k_out, *v_out;
  long long row_pieces;
  long long page_bytes;
  int *status;
  int n, n_kv, pages, max_pages;
  int splits;                // CTAs of a page
  uint32_t magic;            // item / (16-byte pieces of a row) as the high half of a product; 0: rows too long for it
  int32_t seq[N], count[N];
  int32_t page0[N];          // the entry's first page: c tokens touch (c + 62) / 64 + 1 pages at most
  int32_t row0[N];           // its first row
};

constexpr int C4_ROW_THREADS = 256;
constexpr int C4_ROW_UNROLL = 4;
constexpr int C4_ROW_ITEMS = C4_ROW_THREADS * C4_ROW_UNROLL;

// A CTA works on tokens of one page of one entry, in pairs (2 p, 2 p + 1 of the sequence).
struct C4Job {
  int pos0, pos1;  // the entry's tokens in the page
  int row;         // of the entry's position 0 (it may be negative)
  int pair0, pairs;
  int entry, page;
};
template <int N>
__device__ __forceinline__ bool c4_job(const C4Rows<N> &P, C4Job &J) {
  const int at = blockIdx.x / P.splits;
  int lo = 0;
  for (int hi = P.n - 1; lo < hi;) {
    const int mid = (lo + hi + 1) / 2;
    if (P.page0[mid] <= at) lo = mid;
    else hi = mid - 1;
  }
  const int first = P.first[lo];
  if (first < 0) return false;
  const long long page = first / PG_TOKENS + (at - P.page0[lo]), end = static_cast<long long>(first) + P.count[lo];
  const long long p0 = max(static_cast<long long>(first), page * PG_TOKENS), p1 = min(end, (page + 1) * PG_TOKENS);
  if (p0 >= p1 || page > INT32_MAX / PG_TOKENS - 1) {
    if (p0 < p1 && threadIdx.x == 0) atomicOr(P.status, STATUS_POSITION);  // (positions are int32)
    return false;
  }
  J.entry = lo;
  J.page = static_cast<int>(page);
  J.pos0 = static_cast<int>(p0);
  J.pos1 = static_cast<int>(p1);
  J.row = P.row0[lo] - first;
  J.pair0 = J.pos0 / 2;
  J.pairs = (J.pos1 + 1) / 2 - J.pair0;
  return true;
}
// The page, nullptr where there is none; tokens behind the sequence's end are cut off.
template <int N>
__device__ __forceinline__ uint8_t *c4_page(const C4Rows<N> &P, C4Job &J) {
  const int len = P.lens[P.seq[J.entry]];
  const int page = J.page < P.max_pages ? P.table[static_cast<long long>(P.seq[J.entry]) * P.max_pages + J.page] : -1;
  const bool bad = page < 0 || page >= P.pages;
  if ((len < J.pos1 || bad) && threadIdx.x == 0) atomicOr(P.status, STATUS_POSITION);
  J.pos1 = min(J.pos1, len);
  return bad || J.pos0 >= J.pos1 ? nullptr : P.pool + page * P.page_bytes;
}

// Four lanes take a block of both tokens of a pair, 16 bytes of each row apiece; its scale is the maximum over the four.  A thread takes
// up to four such pieces, whose rows it asks for before it knows the page.  2 bytes per value are read, 4.5 bits written: 16004 tokens
// of a Qwen3-4B layer 20 us, 84 MB (4.2 TB/s), issue slots at 72 % (14 instructions a value, 3.5 of them the quotient), and 15 to
// read them back (5.6 TB/s).  Rows, in both directions, are the first to leave the second-level cache (39.2 -> 36.9 us for both;
// attention of 256 rows over 4096 that were read back takes 38.9 us with the call either way).
// Packed fp32 arithmetic for the quotients: 3 % slower here, 4 % faster at 256 channels.
template <int DH, int F16, int N>
__global__ void __launch_bounds__(C4_ROW_THREADS) kvd_cache4_append_kernel(const __grid_constant__ C4Rows<N> P) {
  typedef PgTile<DH> T;
  grid_launch_dependents();
  grid_dependency_wait();
  C4Job J;
  if (!c4_job(P, J)) return;
  const int pieces = P.n_kv * T::NB * 4;  // of a row
  const int item0 = blockIdx.x % P.splits * C4_ROW_ITEMS;
  if (item0 >= J.pairs * pieces) return;
  uint8_t *page = nullptr;
  bool looked = false;
#pragma unroll 2
  for (int u = 0; u < C4_ROW_UNROLL; ++u) {
    const int item = item0 + u * C4_ROW_THREADS + threadIdx.x;
    if (item0 + u * C4_ROW_THREADS >= J.pairs * pieces) break;
    const int pair = P.magic ? static_cast<int>(__umulhi(item, P.magic)) : item / pieces, col = item - pair * pieces;  // col: 8 channels of a head
    const int pos = 2 * (J.pair0 + pair), t = col & 3, block = (col >> 2) % T::NB, head = (col >> 2) / T::NB;
    const bool some = pair < J.pairs;
    bool in[2];
    uint4 x[2][2];  // [K, V][token]
    const long long at = static_cast<long long>(J.row + pos) * P.row_pieces + col;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      in[e] = some && pos + e >= J.pos0 && pos + e < J.pos1;
      x[0][e] = x[1][e] = make_uint4(0, 0, 0, 0);
      if (in[e]) {
        x[0][e] = __ldcs(P.k + at + e * P.row_pieces);
        x[1][e] = __ldcs(P.v + at + e * P.row_pieces);
      }
    }
    if (!looked) {
      looked = true;
      page = c4_page(P, J);
      if (page == nullptr) return;
#pragma unroll
      for (int e = 0; e < 2; ++e) in[e] = in[e] && pos + e < J.pos1;
    }
    // the largest magnitudes of the four blocks (K, V, even and odd token), over the four lanes: lane t ends up with block t
    uint32_t most[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint4 &q = x[w >> 1][w & 1];
      most[w] = abs_max2<F16>(abs_max2<F16>(q.x, q.y), abs_max2<F16>(q.z, q.w));
    }
    // (halves of the lanes exchange two of the four blocks, then one of two)
    const uint32_t give0 = t & 2 ? most[0] : most[2], give1 = t & 2 ? most[1] : most[3];
    const uint32_t half0 = abs_max2<F16>(t & 2 ? most[2] : most[0], __shfl_xor_sync(0xffffffffu, give0, 2));
    const uint32_t half1 = abs_max2<F16>(t & 2 ? most[3] : most[1], __shfl_xor_sync(0xffffffffu, give1, 2));
    const float2 top = unpack16<F16>(abs_max2<F16>(t & 1 ? half1 : half0, __shfl_xor_sync(0xffffffffu, t & 1 ? half0 : half1, 1)));
    const uint16_t my_scale = c4_scale(top.x == top.x && top.y == top.y ? fmaxf(top.x, top.y) : INFINITY);
    const float s_own = __half2float(__ushort_as_half(my_scale));
    const float inv_own = s_own > 0.0f ? __fdividef(1.0f, s_own) : 0.0f;  // (no scale, or none that is a number: the codes do not matter, or are 0)
    uint32_t code[2][2];  // eight codes, channel j in bits 4 j
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint4 &q = x[w >> 1][w & 1];
      const float inv = __shfl_sync(0xffffffffu, inv_own, w, 4);
      const uint32_t u4[4] = {q.x, q.y, q.z, q.w};
      float f[8];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 x2 = unpack16<F16>(u4[j]);
        f[2 * j] = c4_quotient(x2.x, inv);
        f[2 * j + 1] = c4_quotient(x2.y, inv);
      }
      code[w >> 1][w & 1] = e2m1_codes(f);
    }
    if (!in[0] && !in[1]) continue;
    const int tok = pos % PG_TILE, p = tok / 2;
    uint8_t *tile = page + (head * PG_TILES + pos % PG_TOKENS / PG_TILE) * T::BYTES;
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (in[e]) *reinterpret_cast<uint32_t *>(tile + T::k_word(tok + e, block, t)) = code[0][e];
    // lane t has the scale of K or V (t / 2), of the even or odd token (t % 2)
    if (t & 1 ? in[1] : in[0]) *reinterpret_cast<uint16_t *>(tile + (t & 2 ? T::v_scale(p, block) + 2 * (t & 1) : T::k_scale(tok + (t & 1), block))) = my_scale;
    // values: byte i of a word is channel i of four, the even token below the odd one
    const uint32_t mine = (in[0] ? 0x0f0f0f0fu : 0u) | (in[1] ? 0xf0f0f0f0u : 0u);
    const uint32_t even = code[1][0], odd = code[1][1];
    // spread the four codes of a half over the bytes
    auto spread = [](uint32_t four) {
      const uint32_t x = (four | four << 8) & 0x00ff00ffu;
      return (x | x << 4) & 0x0f0f0f0fu;
    };
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      uint32_t *to = reinterpret_cast<uint32_t *>(tile + T::v_word(p, block, 2 * t + half));
      uint32_t w = spread(half ? even >> 16 : even & 0xffffu) | spread(half ? odd >> 16 : odd & 0xffffu) << 4;
      if (mine != 0xffffffffu) w = (w & mine) | (*to & ~mine);  // the other token's codes stay
      *to = w;
    }
  }
}

template <int DH, int F16, int N>
__global__ void __launch_bounds__(C4_ROW_THREADS) kvd_cache4_expand_kernel(const __grid_constant__ C4Rows<N> P) {
  typedef PgTile<DH> T;
  grid_launch_dependents();
  grid_dependency_wait();
  C4Job J;
  if (!c4_job(P, J)) return;
  const int pieces = P.n_kv * T::NB * 4;
  const int item0 = blockIdx.x % P.splits * C4_ROW_ITEMS;
  if (item0 >= J.pairs * pieces) return;
  const uint8_t *page = c4_page(P, J);
  if (page == nullptr) return;
  // what the thread's pieces need of the page is asked for at once
  uint32_t vw[C4_ROW_UNROLL][2], vs[C4_ROW_UNROLL], kw[C4_ROW_UNROLL][2];
  uint16_t ks[C4_ROW_UNROLL][2];
#pragma unroll
  for (int u = 0; u < C4_ROW_UNROLL; ++u) {
    const int item = min(item0 + u * C4_ROW_THREADS + static_cast<int>(threadIdx.x), J.pairs * pieces - 1);
    const int pair = P.magic ? static_cast<int>(__umulhi(item, P.magic)) : item / pieces, col = item - pair * pieces;
    const int pos = 2 * (J.pair0 + pair), t = col & 3, block = (col >> 2) % T::NB, head = (col >> 2) / T::NB;
    const uint8_t *tile = page + (head * PG_TILES + pos % PG_TOKENS / PG_TILE) * T::BYTES;
    const int tok = pos % PG_TILE, p = tok / 2;
    vw[u][0] = *reinterpret_cast<const uint32_t *>(tile + T::v_word(p, block, 2 * t));
    vw[u][1] = *reinterpret_cast<const uint32_t *>(tile + T::v_word(p, block, 2 * t + 1));
    vs[u] = *reinterpret_cast<const uint32_t *>(tile + T::v_scale(p, block));
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      kw[u][e] = *reinterpret_cast<const uint32_t *>(tile + T::k_word(tok + e, block, t));
      ks[u][e] = *reinterpret_cast<const uint16_t *>(tile + T::k_scale(tok + e, block));
    }
  }
#pragma unroll
  for (int u = 0; u < C4_ROW_UNROLL; ++u) {
    const int item = item0 + u * C4_ROW_THREADS + threadIdx.x;
    if (item >= J.pairs * pieces) return;
    const int pair = P.magic ? static_cast<int>(__umulhi(item, P.magic)) : item / pieces, col = item - pair * pieces, pos = 2 * (J.pair0 + pair);
    uint32_t h0[4], h1[4];
    e2m1_word(vw[u][0], h0);
    e2m1_word(vw[u][1], h1);
    const float2 s = h2f(vs[u]);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      if (pos + e < J.pos0 || pos + e >= J.pos1) continue;
      const long long at = static_cast<long long>(J.row + pos + e) * P.row_pieces + col;
      uint32_t h[4], o[4];
      e2m1_word(kw[u][e], h);
      const float sk = __half2float(__ushort_as_half(ks[u][e])), sv = e ? s.y : s.x;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 f = h2f(h[j]);
        o[j] = pack16<F16>(f.x * sk, f.y * sk);
      }
      __stcs(P.k_out + at, make_uint4(o[0], o[1], o[2], o[3]));
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 f0 = h2f(j < 2 ? h0[2 * j] : h1[2 * j - 4]), f1 = h2f(j < 2 ? h0[2 * j + 1] : h1[2 * j - 3]);
        o[j] = e ? pack16<F16>(f0.y * sv, f1.y * sv) : pack16<F16>(f0.x * sv, f1.x * sv);
      }
      __stcs(P.v_out + at, make_uint4(o[0], o[1], o[2], o[3]));
    }
  }
}

// ------------------------------------------------------------------------------------------------ decode attention
constexpr int C4_SEQS = 64;             // sequences per launch
constexpr int C4_MAX_CTAS = 320;        // of a launch: two for each of 160 SMs, more than any device of this kind has
constexpr uint32_t C4_TINY = 0x17ff;    // fp16 bits of the largest number below 2^-9 ...
constexpr uint32_t C4_USUAL = 0x3fff;   // ... and of that below 2
constexpr float C4_OFFSET = 12.0f;
constexpr int C4_RUN_COST = 28672;      // channels of a tile, over tiles
constexpr int C4_AHEAD = 6;             // parts that a thread of the last merge asks for at once (12: longer code, 1 to 2 % slower calls)
template <int DH>
struct C4Cfg {
  static constexpr int WARPS = DH == 128 ? 12 : 8;       // of a CTA
  static constexpr int CTAS = DH == 64 ? 2 : 1;          // per SM
  static constexpr int TILES = DH == 128 ? 2 : 1;        // tiles that are copied and attended at once: a part
  static constexpr int STAGES = DH == 128 ? 3 : DH == 256 ? 3 : 4;
  static constexpr int STAGE = TILES * PgTile<DH>::BYTES;
  static constexpr int RING = WARPS * STAGES * STAGE;
  static constexpr int QUERY = PgTile<DH>::NB * 512;     // fragments of a KV head's queries
  static constexpr int ROW = DH + 4;                     // floats of a head's sums in the merge: rows of head pairs 32 bytes apart in the banks
  static constexpr int HEADS = 4;                        // heads merged at once
  static constexpr int SUMS = WARPS * HEADS * ROW * 4, PARTS = 2 * 8 * (C4_MAX_CTAS + 1) * 4;  // of the warps; maxima and sums of a sequence's runs
  static constexpr int MERGE = SUMS > PARTS ? SUMS : PARTS;
  static constexpr int SMEM = RING + QUERY + MERGE + WARPS * STAGES * 8;
};

struct C4Attend {
  const uint8_t *pool;      // of the layer
  const int32_t *table, *lens;
  const uint16_t *q;
  uint16_t *out;
  float *part_o;            // [2 * CTAs][group][d_head]
  float *part_ml;           // [2 * CTAs][group][2]
  int *arrived;             // [seqs][n_kv]: runs of a sequence and KV head that are done; zero between launches
  long long page_bytes;
  int *status;
  unsigned long long timeout_ns;
  int n, n_q, n_kv, group, pages, max_pages;  // group: query heads of a KV head
  int window, sinks;
  float scale_log2e;
  float rounds, inv_grid;   // sequences and heads over CTAs, rounded up; 1 / CTAs
  int32_t seq[C4_SEQS];
};

// What a sequence's query sees: the tiles of pages [0, sink_pages) and of those from lo_page on, counted on; a tile at either's edge may
// hold no token that is seen.
struct C4Span {
  int len, lo, sinks, sink_pages, lo_page, tiles;
  int plain0, plain1;  // tiles of which every token is seen
  __device__ __forceinline__ int pos(int i) const {  // first position of tile i
    const int page = i / PG_TILES;
    return ((page < sink_pages ? page : lo_page + page - sink_pages) * PG_TILES + i % PG_TILES) * PG_TILE;
  }
};
__device__ __forceinline__ C4Span c4_span(const C4Attend &P, int b) {
  C4Span s;
  const int most = P.max_pages * PG_TOKENS;
  int len = P.lens[P.seq[b]];
  if (len < 0 || len > most) {
    if (blockIdx.x == 0) atomicOr(P.status, STATUS_POSITION);
    len = len < 0 ? 0 : most;
  }
  s.len = len;
  s.lo = P.window > 0 && len > P.window ? len - P.window : 0;
  s.sinks = min(P.sinks, s.lo);
  s.lo_page = s.lo / PG_TOKENS;
  s.sink_pages = min(pg_pages(s.sinks), s.lo_page);
  s.tiles = len > 0 ? (s.sink_pages - s.lo_page) * PG_TILES + (len + PG_TILE - 1) / PG_TILE : 0;
  s.plain0 = s.sink_pages * PG_TILES + (s.lo - s.lo_page * PG_TOKENS + PG_TILE - 1) / PG_TILE;
  s.plain1 = (s.sink_pages - s.lo_page) * PG_TILES + len / PG_TILE;
  return s;
}

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// Tiles are the first to leave the second-level cache.  (Most are read once.  Pages that sequences share are read by each of them, and no slower for it: 16
// continuations of one prompt of 8192 keys, Qwen3-4B layer, 31.2 us with and without, 37.5 and 37.2 behind other data.)
__device__ __forceinline__ uint64_t read_once() {
  uint64_t policy;
  asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
  return policy;
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar, uint64_t policy) {
  asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;" ::"r"(dst), "l"(src), "r"(bytes),
               "r"(bar), "l"(policy)
               : "memory");
}
__device__ __forceinline__ __half2 as_half2(uint32_t w) { return *reinterpret_cast<const __half2 *>(&w); }
__device__ __forceinline__ uint32_t as_word(__half2 h) { return *reinterpret_cast<const uint32_t *>(&h); }
template <int W>
__device__ __forceinline__ void lds_words(const uint8_t *p, uint32_t (&w)[W]) {
  if constexpr (W == 1) {
    w[0] = *reinterpret_cast<const uint32_t *>(p);
  } else if constexpr (W == 2) {
    const uint2 x = *reinterpret_cast<const uint2 *>(p);
    w[0] = x.x, w[1] = x.y;
  } else {
    const uint4 x = *reinterpret_cast<const uint4 *>(p);
    w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
  }
}

// The weights' reference for a largest score: 12 below, or less, but not more (times a scale below 2, a weight of 2^15 is all that fp16 holds).  From
// scores of 2^18 on, 12 below may round to something lower; no offset is taken then, and none from 2^27 on.
__device__ __forceinline__ float c4_reference(float top) {
  if (top == -INFINITY) return 0.f;
  const float r = top - C4_OFFSET;
  return top - r <= C4_OFFSET + 0x1p-6f ? r : top;
}

// A warp's sums over its chunk: lane (g, t) has heads 2 t, 2 t + 1.
template <int DH>
struct C4Sums {
  float o[PgTile<DH>::NB][2][4];  // [block][16 channels][C fragment]: channels 32 b + 4 g + i (i = 2 x, rows g and g + 8)
  float top0, top1, ref0, ref1, sum0, sum1;
  // Scales of values are taken 2^e times as large, and so is o: e = 10 while none is above C4_TINY, 0 while all are below 2.  Beyond, every block
  // has an e of its own: that, as long as its scales allow it, and what takes them below 2 then.  v_limit: fp16 bits, in both halves, of the
  // largest scale that e holds for, from which it follows; where blocks differ, a lane has those of the blocks that it looks at: `lane` modulo
  // the blocks, at 256 channels twice that and the next one.
  uint32_t v_limit[DH == 256 ? 2 : 1];
};
__device__ __forceinline__ int c4_exponent(uint32_t limit) { return 16 - static_cast<int>(((limit & 0xffffu) + 1) >> 10); }
// what the lane that has block b says of it
template <int DH, class X>
__device__ __forceinline__ X c4_of_block(const X (&own)[DH == 256 ? 2 : 1], int b) {
  if constexpr (DH == 256) return __shfl_sync(0xffffffffu, own[b & 1], b >> 1);
  else return __shfl_sync(0xffffffffu, own[0], b);
}
// two scales, those that are no numbers left out
__device__ __forceinline__ uint32_t c4_numbers(uint32_t w) { return ((w & 0xffffu) <= 0x7c00u ? w & 0xffffu : 0u) | (w >> 16 <= 0x7c00u ? w & 0xffff0000u : 0u); }

// NT tiles at once.  EDGE: tokens that are not seen are left out (the first one at `pos`); otherwise, and without `edge`, all are seen.  Without
// LARGE: false, and nothing done, where a scale of 2 or more is seen.  With it, scales times 2^e take their place in the tile.
template <int DH, int NT, bool EDGE, bool LARGE, int QB>
__device__ __forceinline__ bool c4_attend(uint8_t *tile0, const uint8_t *query, const uint32_t (&qf)[QB][4], float qs0, float qs1, const C4Span &sp,
                                          int pos, bool first, int lane, C4Sums<DH> &A, bool edge = true) {
  typedef PgTile<DH> T;
  constexpr int NB = T::NB, BH = T::BH;
  const int g = lane >> 2, t = lane & 3;
  auto seen = [&](int p) { return p < sp.len && (p >= sp.lo || p < sp.sinks); };
  // ---- scores of 16 keys (rows g, g + 8) and 8 heads (columns 2 t, 2 t + 1) a tile
  float s[NT][4];
#pragma unroll
  for (int x = 0; x < NT; ++x) {
    const uint8_t *tile = tile0 + x * T::BYTES;
    s[x][0] = s[x][1] = s[x][2] = s[x][3] = 0.f;
    uint32_t ks[2][NB / 2];  // fp16 scales of keys g and g + 8
    lds_words<NB / 2>(tile + T::KS + g * (NB * 2), ks[0]);
    lds_words<NB / 2>(tile + T::KS + (g + 8) * (NB * 2), ks[1]);
#pragma unroll
    for (int hf = 0; hf < T::HALVES; ++hf) {
      uint32_t kw[2][BH];
      lds_words<BH>(tile + T::K + hf * (64 * T::W) + lane * T::W, kw[0]);
      lds_words<BH>(tile + T::K + hf * (64 * T::W) + 32 * T::W + lane * T::W, kw[1]);
#pragma unroll
      for (int bb = 0; bb < BH; ++bb) {
        const int b = hf * BH + bb;
        uint32_t lo[4], hi[4], qb[4];
        if constexpr (QB == NB) {
#pragma unroll
          for (int j = 0; j < 4; ++j) qb[j] = qf[b][j];
        } else {
          lds_words<4>(query + b * 512 + lane * 16, qb);
        }
        e2m1_word(kw[0][bb], lo);
        e2m1_word(kw[1][bb], hi);
        float c[4] = {0.f, 0.f, 0.f, 0.f};
        mma_f16(c, lo[0], hi[0], lo[1], hi[1], qb[0], qb[1]);
        mma_f16(c, lo[2], hi[2], lo[3], hi[3], qb[2], qb[3]);
        const float2 s0 = h2f(ks[0][b / 2]), s1 = h2f(ks[1][b / 2]);
        const float a0 = b & 1 ? s0.y : s0.x, a1 = b & 1 ? s1.y : s1.x;
        s[x][0] = fmaf(c[0], a0, s[x][0]);
        s[x][1] = fmaf(c[1], a0, s[x][1]);
        s[x][2] = fmaf(c[2], a1, s[x][2]);
        s[x][3] = fmaf(c[3], a1, s[x][3]);
      }
    }
    s[x][0] *= qs0;
    s[x][1] *= qs1;
    s[x][2] *= qs0;
    s[x][3] *= qs1;
    if (EDGE && edge) {
      const int at = pos + x * PG_TILE;
      if (!seen(at + g)) s[x][0] = s[x][1] = -INFINITY;
      if (!seen(at + g + 8)) s[x][2] = s[x][3] = -INFINITY;
    }
  }
  // ---- whether a scale of the values is above its limit, as whole numbers (none is negative): a lane looks at two tokens of a block, or of two; at
  // an edge at those that are seen
  constexpr int VB = DH == 256 ? 2 : 1, LANES = DH == 64 ? 2 : 4;  // blocks of a lane; lanes that have different ones
  const int word0 = DH == 64 ? lane & 15 : VB * lane;
  uint32_t own[NT][VB], over = 0;
#pragma unroll
  for (int x = 0; x < NT; ++x) lds_words<VB>(tile0 + x * T::BYTES + T::VS + word0 * 4, own[x]);
  if (EDGE && edge) {
#pragma unroll
    for (int x = 0; x < NT; ++x) {
      const int token = pos + x * PG_TILE + word0 / NB * 2;
#pragma unroll
      for (int j = 0; j < VB; ++j) own[x][j] &= (seen(token) ? 0xffffu : 0u) | (seen(token + 1) ? 0xffff0000u : 0u);
    }
  }
#pragma unroll
  for (int j = 0; j < VB; ++j) {
    uint32_t most = A.v_limit[j];
#pragma unroll
    for (int x = 0; x < NT; ++x) most = __vmaxu2(most, own[x][j]);
    over |= most ^ A.v_limit[j];
  }
  // ---- the reference moves when a score exceeds it by 3, so that weights stay within 2^15; scales stay below 2
  float tm0 = fmaxf(s[0][0], s[0][2]), tm1 = fmaxf(s[0][1], s[0][3]);
#pragma unroll
  for (int x = 1; x < NT; ++x) {
    tm0 = fmax3(tm0, s[x][0], s[x][2]);
    tm1 = fmax3(tm1, s[x][1], s[x][3]);
  }
  if (__any_sync(0xffffffffu, tm0 > __fadd_rd(A.top0, 3.0f) || tm1 > __fadd_rd(A.top1, 3.0f) || over != 0)) {
    float n0 = tm0, n1 = tm1;
#pragma unroll
    for (int d = 4; d < 32; d *= 2) {
      n0 = fmaxf(n0, __shfl_xor_sync(0xffffffffu, n0, d));
      n1 = fmaxf(n1, __shfl_xor_sync(0xffffffffu, n1, d));
    }
    // (a NaN among the scales moves nothing, and hides nothing)
    auto largest = [&](int j, auto some) {
      uint32_t most = 0;
#pragma unroll
      for (int x = 0; x < NT; ++x) most = __vmaxu2(most, some(own[x][j]));
      return max(most & 0xffffu, most >> 16);
    };
    int shift[VB] = {};  // of the exponents
    if (LARGE) {
#pragma unroll
      for (int j = 0; j < VB; ++j) {
        uint32_t most = largest(j, c4_numbers);
#pragma unroll
        for (int d = LANES; d < 32; d *= 2) most = max(most, __shfl_xor_sync(0xffffffffu, most, d));
        const int e = c4_exponent(A.v_limit[j]);
        if (most > (A.v_limit[j] & 0xffffu)) A.v_limit[j] = ((max(static_cast<int>(most >> 10) - 14, 1) + 15) * 1024 - 1) * 0x10001u;  // (scales below 2^1, 2^2, ...)
        shift[j] = c4_exponent(A.v_limit[j]) - e;
      }
    } else {
      auto all = [&](auto some) { return __reduce_max_sync(0xffffffffu, VB == 2 ? max(largest(0, some), largest(VB - 1, some)) : largest(0, some)); };
      uint32_t most = all([](uint32_t w) { return w; });
      if (most > C4_USUAL) {
        most = all(c4_numbers);
        if (most > C4_USUAL) return false;
      }
      if (most > C4_TINY && A.v_limit[0] == C4_TINY * 0x10001u) {
#pragma unroll
        for (uint32_t &limit : A.v_limit) limit = C4_USUAL * 0x10001u;
        shift[0] = -10;
      }
    }
    n0 = fmaxf(n0, A.top0);
    n1 = fmaxf(n1, A.top1);
    const float r0 = c4_reference(n0), r1 = c4_reference(n1);
    const float c0 = A.top0 == -INFINITY ? 0.f : ex2_approx(A.ref0 - r0), c1 = A.top1 == -INFINITY ? 0.f : ex2_approx(A.ref1 - r1);
    A.top0 = n0;
    A.top1 = n1;
    A.ref0 = r0;
    A.ref1 = r1;
    if (!first) {
      A.sum0 *= c0;
      A.sum1 *= c1;
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const float back = __int_as_float((127 + (LARGE ? c4_of_block<DH>(shift, b) : shift[0])) << 23), o0 = c0 * back, o1 = c1 * back;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          A.o[b][x][0] *= o0;
          A.o[b][x][1] *= o1;
          A.o[b][x][2] *= o0;
          A.o[b][x][3] *= o1;
        }
      }
    }
  }
  // ---- weights, and the values times them
  __half2 w[NT][2];
#pragma unroll
  for (int x = 0; x < NT; ++x) {
    const float p0 = ex2_approx(s[x][0] - A.ref0), p1 = ex2_approx(s[x][1] - A.ref1), p2 = ex2_approx(s[x][2] - A.ref0), p3 = ex2_approx(s[x][3] - A.ref1);
    A.sum0 += p0 + p2;
    A.sum1 += p1 + p3;
    w[x][0] = as_half2(transpose8(as_word(__floats2half2_rn(p0, p1))));
    w[x][1] = as_half2(transpose8(as_word(__floats2half2_rn(p2, p3))));
  }
  const bool tiny = !LARGE && A.v_limit[0] != C4_USUAL * 0x10001u;
  auto add_values = [&]() {
#pragma unroll
    for (int x = 0; x < NT; ++x) {
      const uint8_t *tile = tile0 + x * T::BYTES;
      uint32_t keep0 = 0xffffffffu, keep1 = 0xffffffffu;
      if (EDGE && edge) {
        const int at = pos + x * PG_TILE;
        keep0 = (seen(at + 2 * t) ? 0xffffu : 0u) | (seen(at + 2 * t + 1) ? 0xffff0000u : 0u);
        keep1 = (seen(at + 2 * t + 8) ? 0xffffu : 0u) | (seen(at + 2 * t + 9) ? 0xffff0000u : 0u);
      }
#pragma unroll
      for (int hf = 0; hf < T::HALVES; ++hf) {
        uint32_t vw[2][BH], vs[2][BH];  // scales: fp16 of tokens 2 t, 2 t + 1 and of 2 t + 8, 2 t + 9
        lds_words<BH>(tile + T::VS + t * (NB * 4) + hf * (BH * 4), vs[0]);
        lds_words<BH>(tile + T::VS + (t + 4) * (NB * 4) + hf * (BH * 4), vs[1]);
        lds_words<BH>(tile + T::V + hf * (64 * T::W) + lane * T::W, vw[0]);
        lds_words<BH>(tile + T::V + hf * (64 * T::W) + 32 * T::W + lane * T::W, vw[1]);
        // Times the weights: here, or where they are used (16 x 8192 keys of 128 channels 30.3 and 31.3 us, 32768 of 256 channels 15.7 and 15.2).
        constexpr bool AHEAD = DH < 256;
        auto weigh = [&](int bb, __half2 up, bool scaled) {
          __half2 v0 = as_half2(vs[0][bb] & keep0), v1 = as_half2(vs[1][bb] & keep1);
          if (scaled) v0 = __hmul2(v0, up), v1 = __hmul2(v1, up);
          vs[0][bb] = as_word(AHEAD ? __hmul2(w[x][0], v0) : v0);
          vs[1][bb] = as_word(AHEAD ? __hmul2(w[x][1], v1) : v1);
        };
        if (!tiny) {
#pragma unroll
          for (int bb = 0; bb < BH; ++bb) weigh(bb, __half2(), false);
        } else {
#pragma unroll
          for (int bb = 0; bb < BH; ++bb) weigh(bb, __float2half2_rn(0x1p10f), true);
        }
#pragma unroll
        for (int bb = 0; bb < BH; ++bb) {
          const int b = hf * BH + bb;
          uint32_t lo[4], hi[4];
          e2m1_word(vw[0][bb], lo);
          e2m1_word(vw[1][bb], hi);
          const uint32_t b0 = AHEAD ? vs[0][bb] : as_word(__hmul2(w[x][0], as_half2(vs[0][bb])));
          const uint32_t b1 = AHEAD ? vs[1][bb] : as_word(__hmul2(w[x][1], as_half2(vs[1][bb])));
          mma_f16(A.o[b][0], lo[0], lo[1], hi[0], hi[1], b0, b1);
          mma_f16(A.o[b][1], lo[2], lo[3], hi[2], hi[3], b0, b1);
        }
      }
    }
  };
  if (!LARGE) {
    add_values();
    return true;
  }
  // Scales that have no room in fp16 times 2^e (with e < 0, below 2^-19: they have six bits) are left to a second turn, 2^16 times as
  // large and with weights 2^16 times as small, of which they lose 2^-28 at most.  A lane has its words to itself
  // (at 64 channels with another one, which writes the same).
  bool small = false;
  auto rescale = [&](bool second) {
    __syncwarp();  // (every lane has read the tile)
#pragma unroll
    for (int j = 0; j < VB; ++j) {
      const int e = c4_exponent(A.v_limit[j]);
      const uint32_t room = e >= 0 ? 0u : e > -6 ? 1u << (5 - e) : static_cast<uint32_t>(-4 - e) << 10;  // fp16 bits of 2^(-19 - e)
      const __half2 up = __float2half2_rn(__int_as_float((127 + (second ? min(e + 16, 15) : e)) << 23));
#pragma unroll
      for (int x = 0; x < NT; ++x) {
        const uint32_t low = ((own[x][j] & 0xffffu) < room ? 0xffffu : 0u) | (own[x][j] >> 16 < room ? 0xffff0000u : 0u);
        small = small || (own[x][j] & low) != 0;
        *reinterpret_cast<uint32_t *>(tile0 + x * T::BYTES + T::VS + (word0 + j) * 4) = as_word(__hmul2(as_half2(own[x][j] & (second ? low : ~low)), up));
      }
    }
    fence_proxy_async_smem();  // (the next copy into the stage comes behind this)
    __syncwarp();
  };
  rescale(false);
  add_values();
  if (__any_sync(0xffffffffu, small)) {
    rescale(true);
#pragma unroll
    for (int x = 0; x < NT; ++x)
#pragma unroll
      for (int h = 0; h < 2; ++h) w[x][h] = __hmul2(w[x][h], __float2half2_rn(0x1p-16f));
    add_values();
  }
  return true;
}

// A warp's tiles of a run, i .. end - 1 of the sequence and head, and their copies.  Parts are what it has of TILES aligned tiles; lane l knows the
// part that begins at or behind tile base + TILES l.
struct C4Feed {
  int i, end, base, bytes = 0;
  const uint8_t *src = nullptr;
  uint32_t bad = 0, unusable = 0;  // parts without a page, stages that hold one
  uint32_t attended = 0;           // parts, over all runs
  bool timed_out = false;
};
struct C4Place {
  int seq, head;   // of the launch
  uint32_t ring, bars;  // of the warp
  uint64_t policy;
};
template <int DH>
__device__ __forceinline__ void c4_look_up(const C4Attend &P, const C4Span *spans, const C4Place &W, int lane, C4Feed &F) {
  typedef PgTile<DH> T;
  constexpr int TP = C4Cfg<DH>::TILES;
  const int j = max(F.i, F.base + TP * lane), e = min(F.end, F.base + TP * lane + TP);
  bool bad = false;
  F.bytes = 0;
  if (j < e) {
    const int pos = spans[W.seq].pos(j);
    const int page = P.table[static_cast<long long>(P.seq[W.seq]) * P.max_pages + pos / PG_TOKENS];
    bad = page < 0 || page >= P.pages;
    F.bytes = bad ? 0 : (e - j) * T::BYTES;
    F.src = P.pool + (bad ? 0 : page) * P.page_bytes + (W.head * PG_TILES + j % PG_TILES) * T::BYTES;
    if (bad) atomicOr(P.status, STATUS_POSITION);
    if (!KVD_BOUNDS_OK(e - j <= TP && j % PG_TILES + e - j <= PG_TILES, P.status)) F.bytes = 0;  // (a part lies in one page, and in its stage)
  }
  F.bad = __ballot_sync(0xffffffffu, bad);
}
// the part that begins at or behind tile `at`, a multiple of TILES, if there is one
template <int DH>
__device__ __forceinline__ void c4_fetch(const C4Attend &P, const C4Span *spans, const C4Place &W, int lane, int at, uint32_t stage, C4Feed &F) {
  if (at >= F.end) return;
  int l = (at - F.base) / C4Cfg<DH>::TILES;
  if (l >= 32) {
    F.base = at;
    c4_look_up<DH>(P, spans, W, lane, F);
    l = 0;
  }
  F.unusable = (F.unusable & ~(1u << stage)) | (F.bad >> l & 1u) << stage;
  if (lane == l) {
    mbar_arrive_expect_tx(W.bars + 8 * stage, F.bytes);
    if (F.bytes > 0) bulk_load(W.ring + stage * C4Cfg<DH>::STAGE, F.src, F.bytes, W.bars + 8 * stage, W.policy);
  }
}
// A wait has run out.  The copies in flight land before the CTA's shared memory goes to another: each is waited for once more, whatever the abort flag
// says.  The warp goes on through the merges, whose barriers count it.
template <int DH>
__device__ __forceinline__ void c4_give_up(const C4Attend &P, const C4Place &W, int lane, volatile int *abort_flag, const volatile int *never, C4Feed &F) {
  constexpr int TP = C4Cfg<DH>::TILES, S = C4Cfg<DH>::STAGES;
  raise(P.status, STATUS_TIMEOUT, abort_flag);
  F.timed_out = true;
  for (int j = F.i / TP * TP; j < min(F.end, F.i / TP * TP + S * TP); j += TP, ++F.attended)
    warp_wait(W.bars + 8 * (F.attended % S), (F.attended / S) & 1, never, P.timeout_ns, lane);
}
// The rest of a run, from the first tile with a scale of 2 or more on; `ahead` tiles of its part have been attended
template <int DH, int QB>
__device__ __forceinline__ void c4_large(const C4Attend &P, const C4Span *spans, const C4Place &W, int lane, uint8_t *ring, const uint8_t *query, const uint32_t (&qf)[QB][4], float qs0,
                                         float qs1, volatile int *abort_flag, const volatile int *never, int ahead, bool first, C4Feed &F, C4Sums<DH> &A) {
  constexpr int TP = C4Cfg<DH>::TILES, S = C4Cfg<DH>::STAGES;
  constexpr bool PLAIN = DH == 128;  // one tile at a time for both kinds, but for 128 channels: two plain ones at once 32.6 us, one 40.6
  const int plain0 = spans[W.seq].plain0, plain1 = spans[W.seq].plain1;
#pragma unroll 1
  while (F.i < F.end) {
    const uint32_t stage = F.attended % S;
    if (!warp_wait(W.bars + 8 * stage, (F.attended / S) & 1, abort_flag, P.timeout_ns, lane)) {
      c4_give_up<DH>(P, W, lane, abort_flag, never, F);
      break;
    }
    const int next = min(F.end, F.i / TP * TP + TP);
    uint8_t *at = ring + stage * C4Cfg<DH>::STAGE + ahead * PgTile<DH>::BYTES;
    if (!(F.unusable >> stage & 1)) {
      if (PLAIN && next - F.i == TP && F.i >= plain0 && next <= plain1) {
        c4_attend<DH, TP, false, true>(at, query, qf, qs0, qs1, spans[W.seq], 0, first, lane, A);
      } else {
#pragma unroll 1
        for (int x = F.i; x < next; ++x)
          c4_attend<DH, 1, true, true>(at + (x - F.i) * PgTile<DH>::BYTES, query, qf, qs0, qs1, spans[W.seq], spans[W.seq].pos(x), first && x == F.i, lane, A,
                                       x < plain0 || x >= plain1);
      }
      first = false;
    }
    ahead = 0;
    F.i = next;
    __syncwarp();
    c4_fetch<DH>(P, spans, W, lane, next / TP * TP + (S - 1) * TP, stage, F);
    ++F.attended;
  }
}
// At 256 channels a function of its own, so that the code of the other runs lies together: inline, a call after other kernels' took 18.4 us instead of 16.4
// (Gemma-3-4B layer, window of 1024), and a step of two sequences of the 34-layer stack 2.74 ms instead of 2.66; runs with such scales take 25.0 us
// instead of 18.1 for it (32768 keys).  At 128 it would cost registers (31.7 us, 30.3).
template <int DH, int QB>
struct C4Large {
  const C4Span *spans;
  C4Place W;
  C4Feed F;
  C4Sums<DH> A;
  uint32_t qf[QB][4];
  float qs0, qs1;
  uint8_t *ring;
  const uint8_t *query;
  volatile int *abort_flag;
  const volatile int *never;
  int ahead;
  bool first;
};
template <int DH, int QB>
__device__ __noinline__ void c4_large_apart(const C4Attend &P, C4Large<DH, QB> &L, int lane) {
  C4Feed F = L.F;
  C4Sums<DH> A = L.A;
  const C4Place W = L.W;
  c4_large<DH, QB>(P, L.spans, W, lane, L.ring, L.query, L.qf, L.qs0, L.qs1, L.abort_flag, L.never, L.ahead, L.first, F, A);
  L.F = F;
  L.A = A;
}

// The tiles of a sequence and KV head are cut into equal runs, one a CTA, of at least a tile for each warp and not more of them than the
// launch has CTAs; where there are more sequences and heads than CTAs, a CTA has several whole ones.  Where either would leave a CTA with
// far more tiles than the average, all tiles one after the other are cut into equal pieces instead, and a CTA has several runs, the first
// and the last of them parts: that costs as much time as some 220 tiles of 128 channels (30 sequences of 2048 keys, Qwen3-4B layer:
// 29 us in equal pieces, 24 with whole ones).  A run's tiles go to the CTA's warps in equal parts, all query heads of the KV head at
// once; a warp streams its tiles through a ring of its own, one bulk copy for up to 4608 bytes, issued ahead over the ends of runs.
// The warps' sums of a run come together in shared memory; where a sequence's tiles of a head lie in several CTAs, the last of these
// to be done adds up what they left, in the order of the tiles.
//
// Codes become fp16 exactly and are multiplied as they are: keys (16 x 16 channels a step) with the queries, and the scores of every
// block of 32 channels with its scale in fp32; values, transposed by the way they are stored, with the softmax weights times
// their token's scale.  The weights are 2^(s - m'), m' = the reference maximum less 12 (c4_reference): fp16 rounds a weight like any other
// down to 2^-26 of the largest one.  So that it does the same to the products with scales, these are taken 2^10 times as large where none of the head
// is 2^-9 or more, and from the first one of 2 on each block's by a power of two that takes the largest below 2, in a loop of its own
// (values of deviation 30: 35.1 us for 16 x 8192 keys of a Qwen3-4B layer, 30.3 otherwise; 25.0 and 15.2 for 32768 of a Gemma-3-4B one; with one power for the
// whole head, which loses the small ones, 30.8 and 15.4).  One that this leaves below 2^-19 is left to a second turn over the tile.
//
// 16 x 8192 keys, 32 query on 8 KV heads of 128: 31.8 us for 146 MB (16-bit caches of the same keys take 106).  44 of 57 thousand clocks
// are the tiles, at 6.3 TB/s: bound by memory then, at 2 to 3 instructions a clock and SM (2 products, 8 conversions and some 6
// of scales for a block of 32 channels and 16 keys; with spilled registers, or with 16 warps of 128, the instructions were what bound it,
// 10 % longer).  6 are the start (lengths, page numbers, queries, the first copies: four latencies one after the other), 4 the merge
// of the warps.  One sequence of 32768 keys, 8 on 4 of 256: 16.2 us for 38 MB: start 5, tiles 12 (5.9 TB/s), merge of the warps 2,
// count 2, last merge 4.
template <int DH, int F16>
__global__ void __launch_bounds__(C4Cfg<DH>::WARPS * 32, C4Cfg<DH>::CTAS) kvd_cache4_attention_kernel(const __grid_constant__ C4Attend P) {
  typedef PgTile<DH> T;
  typedef C4Cfg<DH> C;
  constexpr int NB = T::NB, S = C::STAGES, TP = C::TILES, WARPS = C::WARPS;
  constexpr int QB = DH < 256 ? NB : 1;     // the queries' fragments stay in registers, or in shared memory
  constexpr int LANES = DH / 4;             // that share a head in the merge
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int s_tiles[C4_SEQS + 1];      // tiles before a sequence, over its KV heads
  __shared__ int s_runs[C4_SEQS + 1];       // runs before a sequence
  __shared__ int s_head_runs[C4_SEQS];      // runs of each of its heads
  __shared__ int s_cut;
  enum { ONE_RUN, WHOLE, EQUAL };
  __shared__ C4Span s_span[C4_SEQS];
  __shared__ float s_factor[8];             // of the KV head's queries: what a score is multiplied with
  __shared__ float2 s_ml[WARPS][8];         // maximum and sum of a warp and head
  __shared__ int2 s_parted[2];
  __shared__ int s_last[2];
  __shared__ volatile int s_abort, s_never;  // (a flag that nobody raises)
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int g = lane >> 2, t = lane & 3;
  uint8_t *ring = smem + warp * (S * C::STAGE), *query = smem + C::RING;
  float *merge = reinterpret_cast<float *>(smem + C::RING + C::QUERY);
  const uint32_t bars = smem_u32(smem) + C::RING + C::QUERY + C::MERGE + warp * (S * 8);
  if (lane == 0) {
    for (int i = 0; i < S; ++i) mbar_init(bars + 8 * i, 1);
    fence_mbar_init();
  }
  if (tid == 0) s_abort = s_never = 0;
  grid_launch_dependents();
  grid_dependency_wait();
  const int pairs = P.n * P.n_kv, grid = gridDim.x, spare = grid - pairs;
  if (warp == 0) {  // what the sequences' queries see, and how the tiles are cut: lanes have sequences `lane` and `lane + 32`
    C4Span sa, sc;
    sa.tiles = sc.tiles = 0;
    if (lane < P.n) s_span[lane] = sa = c4_span(P, lane);
    if (lane + 32 < P.n) s_span[lane + 32] = sc = c4_span(P, lane + 32);
    const int ta = sa.tiles, tc = sc.tiles;
    auto sums = [&](int a, int c, int *to) {  // running sums over the sequences; the last one
#pragma unroll
      for (int d = 1; d < 32; d *= 2) {
        const int x = __shfl_up_sync(0xffffffffu, a, d), y = __shfl_up_sync(0xffffffffu, c, d);
        a += lane >= d ? x : 0;
        c += lane >= d ? y : 0;
      }
      c += __shfl_sync(0xffffffffu, a, 31);
      if (lane == 0) to[0] = 0;
      if (lane < P.n) to[lane + 1] = a;
      if (lane + 32 < P.n) to[lane + 33] = c;
      return __shfl_sync(0xffffffffu, c, 31);
    };
    const int total = sums(ta * P.n_kv, tc * P.n_kv, s_tiles);
    // Runs of at most `most` tiles: no more of them than CTAs (the sum of tiles / most + 1 over the sequences and heads).  Quotients in fp32,
    // with most rounded up and the number of runs down.
    int ra = 0, rc = 0;  // of each head
    float run = 0.f;
    if (spare > 0) {
      const int most = max(WARPS, static_cast<int>(__fdividef(static_cast<float>(total), static_cast<float>(spare)) * (1.0f + 0x1p-18f)) + 1);
      const float per = __fdividef(1.0f - 0x1p-18f, static_cast<float>(most));
      if (ta > 0) ra = static_cast<int>(ta * per) + 1;
      if (tc > 0) rc = static_cast<int>(tc * per) + 1;
      run = fmaxf(ra > 0 ? __fdividef(static_cast<float>(ta), static_cast<float>(ra)) : 0.f, rc > 0 ? __fdividef(static_cast<float>(tc), static_cast<float>(rc)) : 0.f);
    }
    const float longest = __int_as_float(__reduce_max_sync(0xffffffffu, __float_as_int(run)));
    const float whole = static_cast<float>(__reduce_max_sync(0xffffffffu, max(ta, tc))) * P.rounds, limit = total * P.inv_grid + C4_RUN_COST / DH;
    sums(ra * P.n_kv, rc * P.n_kv, s_runs);
    if (lane < P.n) s_head_runs[lane] = ra;
    if (lane + 32 < P.n) s_head_runs[lane + 32] = rc;
    if (lane == 0) s_cut = spare > 0 && longest <= limit ? ONE_RUN : spare <= 0 && whole <= limit ? WHOLE : EQUAL;
  }
  __syncthreads();
  const int total = s_tiles[P.n];
  // a sequence without a token: zeros
  for (int b = blockIdx.x; b < P.n; b += gridDim.x)
    if (s_span[b].tiles == 0)
      for (int i = tid; i < P.n_q * DH / 8; i += WARPS * 32) reinterpret_cast<uint4 *>(P.out + static_cast<long long>(b) * P.n_q * DH)[i] = make_uint4(0, 0, 0, 0);
  const int cut = s_cut, ctas = cut == ONE_RUN ? s_runs[P.n] : cut == WHOLE ? grid : min(grid, (total + WARPS - 1) / WARPS);
  const int cta = blockIdx.x;
  if (cta >= ctas) return;
  // n in k parts, the first n % k of them one larger: where part j begins, and which one x is in
  auto part_of = [](int n, int k, int j) { return n / k * j + min(j, n % k); };
  auto part_with = [](int n, int k, int x) {
    const int q = n / k, r = n % k;
    return x < r * (q + 1) ? x / (q + 1) : r + (x - r * (q + 1)) / q;
  };
  auto last_before = [&](const int *sums, int x) {  // the last sequence with sums[.] <= x
    int lo = 0;
    for (int hi = P.n - 1; lo < hi;) {
      const int mid = (lo + hi + 1) / 2;
      if (sums[mid] <= x) lo = mid;
      else hi = mid - 1;
    }
    return lo;
  };
  int piece0, piece1, seq;
  if (cut == ONE_RUN) {
    seq = last_before(s_runs, cta);
    const int tiles = s_span[seq].tiles, runs = s_head_runs[seq], in = cta - s_runs[seq];
    const int h = static_cast<int>(__fdividef(in + 0.5f, static_cast<float>(runs))), k = in - h * runs;  // (both below 2^10: the quotient is off a whole number by 2^-11 at least)
    piece0 = s_tiles[seq] + h * tiles + part_of(tiles, runs, k);
    piece1 = s_tiles[seq] + h * tiles + part_of(tiles, runs, k + 1);
  } else if (cut == WHOLE) {
    auto begins = [&](int pair) { return pair == pairs ? total : s_tiles[pair / P.n_kv] + pair % P.n_kv * s_span[pair / P.n_kv].tiles; };
    piece0 = begins(part_of(pairs, grid, cta));
    piece1 = begins(part_of(pairs, grid, cta + 1));
    if (piece0 == piece1) return;
    seq = last_before(s_tiles, piece0);
  } else {
    piece0 = part_of(total, ctas, cta);
    piece1 = part_of(total, ctas, cta + 1);
    seq = last_before(s_tiles, piece0);
  }
  uint32_t qf[QB][4];  // block b, step h: registers 2 h, 2 h + 1
  // ---- a run: tiles run0 .. run1 - 1 of the launch, of a sequence and head that begin at `begin`
  int run0 = piece0, run1, begin;
  C4Feed F;
  C4Place W;
  W.ring = smem_u32(ring);
  W.bars = bars;
  W.policy = read_once();  // (3 to 5 % of the call: 32768 keys of a Gemma-3-4B layer 16.8 -> 16.1 us, 30 x 2048 of a Qwen3-4B one 23.4 -> 22.4)
  constexpr int CH = DH / 32;        // channels of a query that a lane has; a warp takes a head
  uint32_t qw[CH / 2];
  auto open_run = [&]() {  // the run that begins at run0: its queries and first parts are asked for
    while (s_tiles[seq + 1] <= run0) ++seq;
    const int tiles = s_span[seq].tiles;
    W.seq = seq;
    W.head = (run0 - s_tiles[seq]) / tiles;
    begin = s_tiles[seq] + W.head * tiles;
    run1 = min(piece1, begin + tiles);
    const bool some = warp < P.group;
    const uint16_t *src = P.q + (static_cast<long long>(seq) * P.n_q + W.head * P.group + (some ? warp : 0)) * DH + lane * CH;
#pragma unroll
    for (int j = 0; j < CH / 2; ++j) qw[j] = some ? reinterpret_cast<const uint32_t *>(src)[j] : 0u;
    F.i = run0 - begin + (run1 - run0) * warp / WARPS;
    F.end = F.timed_out ? F.i : run0 - begin + (run1 - run0) * (warp + 1) / WARPS;
    F.base = F.i / TP * TP;
    if (F.i < F.end) {  // (every copy that is issued is waited for)
      c4_look_up<DH>(P, s_span, W, lane, F);
#pragma unroll
      for (int j = 0; j < S; ++j) c4_fetch<DH>(P, s_span, W, lane, F.base + TP * j, (F.attended + j) % S, F);
    }
  };
  open_run();
  int parted = 0;  // runs that are not all of their sequence and head: the first one, the last one
#pragma unroll 1
  for (bool more = true; more;) {
    {
      // ... as fp16 in the order of the fragments: lane (g, t) of block b has channels 32 b + 8 t .. + 7 of head g.  bf16 becomes fp16 of the
      // same 8 bits times a power of two that takes the head's largest channel to 2^10 .. 2^11.
      // (heads that there are not, of eight: zeros)
      const int h = warp;
      float factor = P.scale_log2e;
      if (!F16) {
        uint32_t amax = 0;
#pragma unroll
        for (int j = 0; j < CH / 2; ++j) amax = max(amax, max(qw[j] & 0x7fffu, (qw[j] >> 16) & 0x7fffu));
        amax = __reduce_max_sync(0xffffffffu, amax);
        int e = static_cast<int>(amax >> 7) - 127 - 10;
        e = e < -126 ? -126 : e > 110 ? 110 : e;
        const float down = __int_as_float((127 - e) << 23);
#pragma unroll
        for (int j = 0; j < CH / 2; ++j) qw[j] = as_word(__floats2half2_rn(bf16_lo(qw[j]) * down, bf16_hi(qw[j]) * down));
        factor *= __int_as_float((127 + e) << 23);
      }
      if (h < 8) {
#pragma unroll
        for (int j = 0; j < CH / 2; ++j) {
          const int c = lane * CH + 2 * j;  // block c / 32, part c / 8 % 4, pair c / 2 % 4
          *reinterpret_cast<uint32_t *>(query + (c / 32) * 512 + (h * 4 + c / 8 % 4) * 16 + (c / 2 % 4) * 4) = qw[j];
        }
        if (lane == 0) s_factor[h] = factor;
      }
      __syncthreads();
      if constexpr (QB == NB) {
#pragma unroll
        for (int b = 0; b < NB; ++b) lds_words<4>(query + b * 512 + lane * 16, qf[b]);
      }
    }
    const float qs0 = s_factor[2 * t], qs1 = s_factor[2 * t + 1];

    C4Sums<DH> A;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i) A.o[b][x][i] = 0.f;
    A.top0 = A.top1 = -INFINITY;
    A.ref0 = A.ref1 = A.sum0 = A.sum1 = 0.f;
#pragma unroll
    for (uint32_t &limit : A.v_limit) limit = C4_TINY * 0x10001u;
    const int plain0 = s_span[seq].plain0, plain1 = s_span[seq].plain1;
    // the parts of the run, up to one with a scale of 2 or more
    bool first = true;
    int ahead = 0;
    auto usual_parts = [&]() {
#pragma unroll 1
      while (F.i < F.end) {
        const uint32_t stage = F.attended % S;
        if (!__all_sync(0xffffffffu, mbar_try_wait(bars + 8 * stage, (F.attended / S) & 1)) &&
            !warp_wait(bars + 8 * stage, (F.attended / S) & 1, &s_abort, P.timeout_ns, lane)) {
          c4_give_up<DH>(P, W, lane, &s_abort, &s_never, F);
          return true;
        }
        const int next = min(F.end, F.i / TP * TP + TP);
        uint8_t *at = ring + stage * C::STAGE;
        if (!(F.unusable >> stage & 1)) {
          if (next - F.i == TP && F.i >= plain0 && next <= plain1) {
            if (!c4_attend<DH, TP, false, false>(at, query, qf, qs0, qs1, s_span[seq], 0, first, lane, A)) return false;
          } else {
#pragma unroll 1
            for (int x = F.i; x < next; ++x) {
              if (!c4_attend<DH, 1, true, false>(at + (x - F.i) * T::BYTES, query, qf, qs0, qs1, s_span[seq], s_span[seq].pos(x), first && x == F.i, lane, A)) {
                ahead = x - F.i;
                F.i = x;
                first = first && ahead == 0;
                return false;
              }
            }
          }
          first = false;
        }
        F.i = next;
        __syncwarp();
        c4_fetch<DH>(P, s_span, W, lane, F.i / TP * TP + (S - 1) * TP, stage, F);
        ++F.attended;
      }
      return true;
    };
    const bool large = !usual_parts();
    if (large) {
      if constexpr (DH < 256) {
        c4_large<DH, QB>(P, s_span, W, lane, ring, query, qf, qs0, qs1, &s_abort, &s_never, ahead, first, F, A);
      } else {
        C4Large<DH, QB> L{s_span, W, F, A, {}, qs0, qs1, ring, query, &s_abort, &s_never, ahead, first};
        c4_large_apart<DH, QB>(P, L, lane);
        F = L.F;
        A = L.A;
      }
    }
    // ---- the next run is asked for before the warps' sums of this one come together
    const bool whole = run1 - run0 == s_span[seq].tiles;
    const long long out0 = static_cast<long long>(seq) * P.n_q + W.head * P.group;  // rows of the output
    const int slot = 2 * blockIdx.x + (run0 != piece0);
    if (!whole) {
      if (tid == 0) s_parted[parted] = make_int2(seq, W.head);
      ++parted;
    }
    more = run1 < piece1;
    if (more) {
      run0 = run1;
      open_run();
    }
#pragma unroll
    for (int d = 4; d < 32; d *= 2) {
      A.sum0 += __shfl_xor_sync(0xffffffffu, A.sum0, d);
      A.sum1 += __shfl_xor_sync(0xffffffffu, A.sum1, d);
    }
    if (g == 0) {
      s_ml[warp][2 * t] = make_float2(A.top0 == -INFINITY ? -INFINITY : A.ref0, A.sum0);
      s_ml[warp][2 * t + 1] = make_float2(A.top1 == -INFINITY ? -INFINITY : A.ref1, A.sum1);
    }
    if (large || A.v_limit[0] != C4_USUAL * 0x10001u) {
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const float down = __int_as_float((127 - c4_exponent(c4_of_block<DH>(A.v_limit, b))) << 23);
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int e = 0; e < 4; ++e) A.o[b][x][e] *= down;
      }
    }
#pragma unroll 1
    for (int h0 = 0; h0 < P.group; h0 += C::HEADS) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int h = 2 * t + e - h0;
        if (h >= 0 && h < C::HEADS && h0 + h < P.group) {
          float *row = merge + (warp * C::HEADS + h) * C::ROW + 4 * g;
#pragma unroll
          for (int b = 0; b < NB; ++b) *reinterpret_cast<float4 *>(row + 32 * b) = make_float4(A.o[b][0][e], A.o[b][0][e + 2], A.o[b][1][e], A.o[b][1][e + 2]);
        }
      }
      __syncthreads();
      const int heads = min(C::HEADS, P.group - h0);
#pragma unroll 1
      for (int at = tid; at < heads * LANES; at += WARPS * 32) {
        const int h = at / LANES, c = at % LANES * 4;
        float mh = -INFINITY, lh = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) mh = fmaxf(mh, s_ml[w][h0 + h].x);
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
          const float2 ml = s_ml[w][h0 + h];
          const float aw = ml.x == -INFINITY ? 0.f : ex2_approx(ml.x - mh);
          const float4 y = *reinterpret_cast<const float4 *>(merge + (w * C::HEADS + h) * C::ROW + c);
          lh = fmaf(aw, ml.y, lh);
          x.x = fmaf(aw, y.x, x.x);
          x.y = fmaf(aw, y.y, x.y);
          x.z = fmaf(aw, y.z, x.z);
          x.w = fmaf(aw, y.w, x.w);
        }
        if (whole) {
          const float inv = lh != 0.f ? 1.0f / lh : 0.f;  // (a NaN stays one)
          *reinterpret_cast<uint2 *>(P.out + (out0 + h0 + h) * DH + c) = make_uint2(pack16<F16>(x.x * inv, x.y * inv), pack16<F16>(x.z * inv, x.w * inv));
        } else {
          if (!KVD_BOUNDS_OK(slot < 2 * C4_MAX_CTAS, P.status)) continue;
          const long long row = static_cast<long long>(slot) * P.group + h0 + h;
          *reinterpret_cast<float4 *>(P.part_o + row * DH + c) = x;
          if (c == 0) *reinterpret_cast<float2 *>(P.part_ml + row * 2) = make_float2(mh, lh);
        }
      }
      __syncthreads();
    }
  }
  // ---- the runs of a sequence and head, one a CTA, are added up by the CTA that is done last
  struct Shared {
    int cta0, cta1, slot0;  // the CTAs that have its tiles, where the first one's sums are (the others': at their first place)
  };
  auto shared_by = [&](int seq, int head) {
    Shared w;
    const int tiles = s_span[seq].tiles, begin = s_tiles[seq] + head * tiles;
    if (cut == ONE_RUN) {
      const int runs = s_head_runs[seq];
      w.cta0 = s_runs[seq] + head * runs;
      w.cta1 = w.cta0 + runs - 1;
      w.slot0 = 2 * w.cta0;
    } else {
      w.cta0 = part_with(total, ctas, begin);
      w.cta1 = part_with(total, ctas, begin + tiles - 1);
      w.slot0 = 2 * w.cta0 + (part_of(total, ctas, w.cta0) != begin);
    }
    return w;
  };
  if (tid < parted) {
    const int2 x = s_parted[tid];
    const Shared w = shared_by(x.x, x.y);
    int *count = P.arrived + x.x * P.n_kv + x.y, before;
    asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(before) : "l"(count) : "memory");
    s_last[tid] = before == w.cta1 - w.cta0;
    if (before == w.cta1 - w.cta0) *count = 0;
  }
  __syncthreads();
#pragma unroll 1
  for (int x = 0; x < parted; ++x) {
    if (!s_last[x]) continue;
    const int head = s_parted[x].y;
    const long long out0 = static_cast<long long>(s_parted[x].x) * P.n_q + head * P.group;
    const Shared w = shared_by(s_parted[x].x, head);
    const int cta0 = w.cta0, cta1 = w.cta1, slot0 = w.slot0;
    const int parts = KVD_BOUNDS_OK(cta0 >= 0 && cta1 < static_cast<int>(gridDim.x) && slot0 < 2 * C4_MAX_CTAS, P.status) ? cta1 - cta0 + 1 : 0;
    // four channels of a head a thread; the parts in as many slices as there are threads for, some of a slice asked for at once, the first
    // ones ahead of the weights (the code is short on purpose: one CTA runs it, once, and fetches all of it)
    const int outs = P.group * LANES, slices = max(1, WARPS * 32 / outs), wide = min(outs, WARPS * 32), slice = tid / wide;
    const int odd = slot0 - 2 * cta0;  // the first part's place
    const float *part_o = P.part_o + static_cast<long long>(2 * cta0) * P.group * DH, *part_ml = P.part_ml + 4 * cta0 * P.group;
    float *weights = merge;  // [head][part]: what the parts' sums are multiplied with
#pragma unroll 1
    for (int o0 = 0; o0 < outs; o0 += WARPS * 32) {
      const int at = o0 + tid % wide, h = at / LANES, c = at % LANES * 4;
      const bool mine = slice < slices && at < outs;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
      for (int j0 = 0; j0 < parts; j0 += C4_AHEAD * slices) {
        float4 y[C4_AHEAD];
#pragma unroll
        for (int q = 0; q < C4_AHEAD; ++q) {
          const int j = j0 + slice + q * slices;
          y[q] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (mine && j < parts) y[q] = __ldcg(reinterpret_cast<const float4 *>(part_o + ((2 * j + (j == 0 ? odd : 0)) * P.group * DH + at * 4)));
        }
        if (o0 + j0 == 0) {
          for (int i = tid; i < parts * P.group; i += WARPS * 32) {
            const int j = i / P.group, head = i - j * P.group;
            const float2 ml = __ldcg(reinterpret_cast<const float2 *>(part_ml + (2 * j + (j == 0 ? odd : 0)) * P.group * 2 + head * 2));
            weights[head * parts + j] = ml.x;
            weights[(P.group + head) * parts + j] = ml.y;
          }
          __syncthreads();
          if (warp < P.group) {  // a warp for each head
            float m = -INFINITY, l = 0.f;
            for (int j = lane; j < parts; j += 32) m = fmaxf(m, weights[warp * parts + j]);
#pragma unroll
            for (int d = 16; d >= 1; d /= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
            for (int j = lane; j < parts; j += 32) {
              const float x = weights[warp * parts + j], a = x == -INFINITY ? 0.f : ex2_approx(x - m);
              weights[warp * parts + j] = a;
              l = fmaf(a, weights[(P.group + warp) * parts + j], l);
            }
#pragma unroll
            for (int d = 16; d >= 1; d /= 2) l += __shfl_xor_sync(0xffffffffu, l, d);
            if (lane == 0) s_factor[warp] = l != 0.f ? 1.0f / l : 0.f;
          }
          __syncthreads();
        }
#pragma unroll
        for (int q = 0; q < C4_AHEAD; ++q) {
          const int j = j0 + slice + q * slices;
          const float a = mine && j < parts ? weights[h * parts + j] : 0.f;
          x.x = fmaf(a, y[q].x, x.x);
          x.y = fmaf(a, y[q].y, x.y);
          x.z = fmaf(a, y[q].z, x.z);
          x.w = fmaf(a, y[q].w, x.w);
        }
      }
      if (slices > 1) {
        __syncthreads();  // (the weights have been read)
        float4 *sums = reinterpret_cast<float4 *>(merge);
        if (slice > 0 && slice < slices) sums[(slice - 1) * outs + at] = x;
        __syncthreads();
        for (int i = 1; slice == 0 && i < slices; ++i) {
          const float4 y = sums[(i - 1) * outs + at];
          x.x += y.x;
          x.y += y.y;
          x.z += y.z;
          x.w += y.w;
        }
      }
      if (slice == 0 && at < outs) {
        const float inv = s_factor[h];
        *reinterpret_cast<uint2 *>(P.out + (out0 + h) * DH + c) = make_uint2(pack16<F16>(x.x * inv, x.y * inv), pack16<F16>(x.z * inv, x.w * inv));
      }
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------------------------------------ launches
static kvd_status c4_launched(kvd_ctx *ctx, cudaError_t e, const char *what) {
  if (e != cudaSuccess) return cuda_fail(ctx, e, what);
  ctx->launches += 1;
  return KVD_OK;
}

template <int DH, int F16, int N, bool APPEND>
static kvd_status launch_rows4(kvd_ctx *ctx, C4Rows<N> &P, long long pages, int most, cudaStream_t stream) {
  const int pairs = most / 2 + 1 < PG_TOKENS / 2 ? most / 2 + 1 : PG_TOKENS / 2;  // of an entry in a page, at most
  const long long items = static_cast<long long>(pairs) * P.n_kv * (DH / PG_BLOCK) * 4;
  P.splits = static_cast<int>((items + C4_ROW_ITEMS - 1) / C4_ROW_ITEMS);
  // exact for items below 2^32 / pieces, and there are 32 * pieces of them at most
  const unsigned pieces = static_cast<unsigned>(P.n_kv) * (DH / PG_BLOCK) * 4;
  P.magic = pieces < 8192 ? static_cast<uint32_t>(((1ull << 32) + pieces - 1) / pieces) : 0;
  const long long grid = pages * P.splits;
  if (grid > INT32_MAX) return KVD_ERR_CAPACITY;
  if (APPEND) return c4_launched(ctx, launch_paged(ctx, kvd_cache4_append_kernel<DH, F16, N>, static_cast<unsigned>(grid), C4_ROW_THREADS, stream, P), "launch cache4_append");
  return c4_launched(ctx, launch_paged(ctx, kvd_cache4_expand_kernel<DH, F16, N>, static_cast<unsigned>(grid), C4_ROW_THREADS, stream, P), "launch cache4_expand");
}

template <int N, bool APPEND>
static kvd_status rows4(kvd_ctx *ctx, const kvd_paged_cache *c, int layer, int n, const int32_t *seqs, const int32_t *counts, const int32_t *first, const void *k,
                        const void *v, void *k_out, void *v_out, int64_t row_stride, cudaStream_t stream) {
  const kvd_model_desc &d = ctx->desc;
  C4Rows<N> P;
  P.page_bytes = pg_page_bytes(d.d_head, d.n_kv_heads);
  P.pool = static_cast<uint8_t *>(c->pool) + static_cast<long long>(layer) * c->pages * P.page_bytes;
  P.table = c->table;
  P.lens = c->lens;
  P.first = first;
  P.k = static_cast<const uint4 *>(k);
  P.v = static_cast<const uint4 *>(v);
  P.k_out = static_cast<uint4 *>(k_out);
  P.v_out = static_cast<uint4 *>(v_out);
  P.row_pieces = row_stride / 8;
  P.status = ctx->d_status;
  P.n = n;
  P.n_kv = d.n_kv_heads;
  P.pages = c->pages;
  P.max_pages = c->max_pages;
  long long pages = 0, rows = 0;
  int most = 0;
  for (int i = 0; i < n; ++i) {
    P.seq[i] = seqs[i];
    P.count[i] = counts[i];
    P.page0[i] = static_cast<int32_t>(pages);
    P.row0[i] = static_cast<int32_t>(rows);
    pages += counts[i] > 0 ? (static_cast<long long>(counts[i]) + PG_TOKENS - 2) / PG_TOKENS + 1 : 0;
    rows += counts[i];
    most = counts[i] > most ? counts[i] : most;
    if (rows > INT32_MAX / 2) return KVD_ERR_CAPACITY;
  }
  if (pages == 0) return KVD_OK;
  const bool f16 = ctx->dtype == KVD_DTYPE_F16;
  switch (d.d_head) {
    case 64: return f16 ? launch_rows4<64, 1, N, APPEND>(ctx, P, pages, most, stream) : launch_rows4<64, 0, N, APPEND>(ctx, P, pages, most, stream);
    case 128: return f16 ? launch_rows4<128, 1, N, APPEND>(ctx, P, pages, most, stream) : launch_rows4<128, 0, N, APPEND>(ctx, P, pages, most, stream);
    case 256: return f16 ? launch_rows4<256, 1, N, APPEND>(ctx, P, pages, most, stream) : launch_rows4<256, 0, N, APPEND>(ctx, P, pages, most, stream);
  }
  return KVD_ERR_SHAPE;
}

template <bool APPEND>
static kvd_status rows4_call(kvd_ctx *ctx, const kvd_paged_cache *c, int layer, int n, const int32_t *seqs, const int32_t *counts, const int32_t *first,
                             const void *k, const void *v, int64_t row_stride, void *stream) {
  if (!ctx || n < 0) return KVD_ERR_INVALID_ARG;
  kvd_status st = check_paged(ctx, c);
  if (st != KVD_OK) return st;
  if (layer < 0 || layer >= c->layers) return KVD_ERR_INVALID_ARG;
  if (ctx->dtype == KVD_DTYPE_F32) return KVD_ERR_UNSUPPORTED;
  if (n == 0) return KVD_OK;
  if (!seqs || !counts || !first || !k || !v) return KVD_ERR_INVALID_ARG;
  if (n > KVD_MAX_PAGE_SEQS) return KVD_ERR_CAPACITY;
  st = check_page_seqs(c, n, seqs, APPEND);
  if (st != KVD_OK) return st;
  for (int i = 0; i < n; ++i)
    if (counts[i] < 0) return KVD_ERR_INVALID_ARG;
  if (row_stride < static_cast<int64_t>(ctx->desc.n_kv_heads) * ctx->desc.d_head) return KVD_ERR_INVALID_ARG;
  if (((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & 15u) != 0 || row_stride % 8 != 0 || !aligned4({first})) return KVD_ERR_ALIGNMENT;
  const OnDevice here(ctx);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const void *in_k = APPEND ? k : nullptr, *in_v = APPEND ? v : nullptr;
  void *out_k = APPEND ? nullptr : const_cast<void *>(k), *out_v = APPEND ? nullptr : const_cast<void *>(v);
  if (n <= PG_FEW) return rows4<PG_FEW, APPEND>(ctx, c, layer, n, seqs, counts, first, in_k, in_v, out_k, out_v, row_stride, s);
  return rows4<PG_MANY, APPEND>(ctx, c, layer, n, seqs, counts, first, in_k, in_v, out_k, out_v, row_stride, s);
}

template <int DH, int F16>
static kvd_status launch_attend4(kvd_ctx *ctx, const C4Attend &P, cudaStream_t stream) {
  static std::atomic<bool> configured[64] = {};
  cudaError_t e = opt_in_smem(ctx, kvd_cache4_attention_kernel<DH, F16>, C4Cfg<DH>::SMEM, configured);
  if (e != cudaSuccess) return cuda_fail(ctx, e, "cudaFuncSetAttribute(cache4)");
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = dim3(C4Cfg<DH>::CTAS * ctx->num_sms, 1, 1);
  cfg.blockDim = dim3(C4Cfg<DH>::WARPS * 32, 1, 1);
  cfg.dynamicSmemBytes = C4Cfg<DH>::SMEM;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = serial_launch_mask() & 2 ? 0 : 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return c4_launched(ctx, cudaLaunchKernelEx(&cfg, kvd_cache4_attention_kernel<DH, F16>, P), "launch cache4_attention");
}

// Two runs of a CTA at most are parts of a sequence and head: its first and its last.
static size_t c4_scratch(const kvd_model_desc *d) {
  const size_t rows = 2 * C4_MAX_CTAS * static_cast<size_t>(d->n_q_heads / d->n_kv_heads);
  return (rows * (d->d_head + 2) * sizeof(float) + 255) & ~static_cast<size_t>(255);
}

}  // namespace kvd

using namespace kvd;

extern "C" kvd_status kvd_cache4_append(kvd_ctx *ctx, const kvd_paged_cache *cache, int layer, int n, const int32_t *seqs, const int32_t *counts,
                                        const int32_t *first, const void *k, const void *v, int64_t row_stride, void *stream) {
  return rows4_call<true>(ctx, cache, layer, n, seqs, counts, first, k, v, row_stride, stream);
}

extern "C" kvd_status kvd_cache4_expand(kvd_ctx *ctx, const kvd_paged_cache *cache, int layer, int n, const int32_t *seqs, const int32_t *counts,
                                        const int32_t *first, void *k_out, void *v_out, int64_t row_stride, void *stream) {
  return rows4_call<false>(ctx, cache, layer, n, seqs, counts, first, k_out, v_out, row_stride, stream);
}

extern "C" size_t kvd_cache4_scratch_bytes(const kvd_model_desc *desc, int batch) {
  if (kvd_workspace_bytes(desc) == 0 || batch < 1) return 0;
  return c4_scratch(desc);
}

extern "C" kvd_status kvd_decode_attention_cache4(kvd_ctx *ctx, const kvd_paged_cache *cache, int layer, int batch, const int32_t *seqs, const void *q, int sinks,
                                                  float scale, void *out, void *scratch, size_t scratch_bytes, void *stream_) {
  if (!ctx || batch < 0 || sinks < 0) return KVD_ERR_INVALID_ARG;
  kvd_status st = check_paged(ctx, cache);
  if (st != KVD_OK) return st;
  const kvd_model_desc &d = ctx->desc;
  if (layer < 0 || layer >= d.n_layers || layer >= cache->layers) return KVD_ERR_INVALID_ARG;
  // tiles are counted in 32 bits
  if (static_cast<int64_t>(C4_SEQS) * d.n_kv_heads * cache->max_pages * PG_TILES > INT32_MAX / 2) return KVD_ERR_SHAPE;
  const LayerState &ls = ctx->layers[layer];
  if (!ls.set) return KVD_ERR_STATE;
  if (ctx->dtype == KVD_DTYPE_F32) return KVD_ERR_UNSUPPORTED;
  if (batch == 0) return KVD_OK;
  if (!seqs || !q || !out || !scratch) return KVD_ERR_INVALID_ARG;
  if (((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) & 15u) != 0 || (reinterpret_cast<uintptr_t>(scratch) & 255u) != 0) return KVD_ERR_ALIGNMENT;
  if (scratch_bytes < c4_scratch(&d) || 2 * ctx->num_sms > C4_MAX_CTAS) return KVD_ERR_CAPACITY;
  st = check_page_seqs(cache, batch, seqs, false);
  if (st != KVD_OK) return st;
  const OnDevice here(ctx);
  cudaStream_t stream = static_cast<cudaStream_t>(stream_);
  C4Attend P;
  P.page_bytes = pg_page_bytes(d.d_head, d.n_kv_heads);
  P.pool = static_cast<const uint8_t *>(cache->pool) + static_cast<long long>(layer) * cache->pages * P.page_bytes;
  P.table = cache->table;
  P.lens = cache->lens;
  P.status = ctx->d_status;
  P.timeout_ns = ctx->timeout_ns;
  P.n_q = d.n_q_heads;
  P.n_kv = d.n_kv_heads;
  P.group = d.n_q_heads / d.n_kv_heads;
  P.pages = cache->pages;
  P.max_pages = cache->max_pages;
  P.window = ls.window;
  P.sinks = sinks;
  P.arrived = ctx->c4_arrived;
  const int grid = (d.d_head == 64 ? C4Cfg<64>::CTAS : d.d_head == 128 ? C4Cfg<128>::CTAS : C4Cfg<256>::CTAS) * ctx->num_sms;
  P.inv_grid = 1.0f / static_cast<float>(grid);
  P.scale_log2e = (scale > 0.f ? scale : 1.0f / sqrtf(static_cast<float>(d.d_head))) * 1.4426950408889634f;
  for (int b0 = 0; b0 < batch; b0 += C4_SEQS) {
    P.n = batch - b0 < C4_SEQS ? batch - b0 : C4_SEQS;
    const size_t row = static_cast<size_t>(b0) * d.n_q_heads * d.d_head;
    P.q = static_cast<const uint16_t *>(q) + row;
    P.out = static_cast<uint16_t *>(out) + row;
    P.part_o = static_cast<float *>(scratch);
    P.part_ml = P.part_o + 2 * C4_MAX_CTAS * static_cast<size_t>(P.group) * d.d_head;
    memcpy(P.seq, seqs + b0, P.n * sizeof(int32_t));
    P.rounds = static_cast<float>((P.n * d.n_kv_heads + grid - 1) / grid);
    const bool f16 = ctx->dtype == KVD_DTYPE_F16;
    switch (d.d_head) {
      case 64: st = f16 ? launch_attend4<64, 1>(ctx, P, stream) : launch_attend4<64, 0>(ctx, P, stream); break;
      case 128: st = f16 ? launch_attend4<128, 1>(ctx, P, stream) : launch_attend4<128, 0>(ctx, P, stream); break;
      case 256: st = f16 ? launch_attend4<256, 1>(ctx, P, stream) : launch_attend4<256, 0>(ctx, P, stream); break;
      default: st = KVD_ERR_SHAPE;
    }
    if (st != KVD_OK) return st;
  }
  return KVD_OK;
}
