// Attention of many new tokens per sequence over a paged cache of e4m3 codes:
//
//   s_r = scale q . k_r,  p_r = exp(s_r - max) / sum exp(s - max),  out = sum_r p_r v_r
//
// over the rows up to the token's own, in one pass over them with a running maximum
// and sum.
//
// What bounds it: 4 head_dim operations per token, query head and row, on the matrix
// cores; and beside them, per score, an exponential, a maximum, a sum and a rounding
// on the vector units, which is about as much for heads of 128 values and more for
// heads of 64; and LDS, from which every wave reads all of K and V for its 32 rows of q, at
// 128 bytes a cycle and CU as long as the matrix cores need for them.  With few tokens, a
// workgroup's beginning (its place, and pages, scales and rows, each read after the other) and
// the join.
//
// Work mapping.  A tile is 128 rows of q: as many tokens as fit, with all the query
// heads that share one key-value head, so that K and V are read once for them.  What a tile
// costs is the rows that it attends to; the tiles of all sequences and heads, one after
// the other, are cut into equal runs over as many workgroups as fit the GPU,
// between tiles or inside one.  The lengths are known to the device alone, so every
// workgroup finds its place from them, by closed sums.  What a workgroup finds
// for a tile, unless it has all of it, is joined by a second launch.  Consecutive
// runs go to one XCD, whose L2 then serves the tiles of a head.
//
// In a workgroup every wave has 32 rows of q, and all share 64 rows of K and V at a
// time, double buffered in LDS as f16.  Both products run on 32x32x16 MFMAs without
// moving anything between lanes:
//  * S^T = K Q^T: lane l holds the scores of q row l % 32 with rows 8 (i / 4) + 4 (l / 32)
//    + i % 4 of each half of 32.
//  * O^T = V^T P^T: eight probabilities of a lane are its P^T operand as they are; V is
//    written to LDS transposed, and with its rows in the order that this asks for.
//
// Precision.  e4m3 codes are exact in f16, and so are their products with powers of
// two down to 2^-15, which take the pages' scales.  Where the powers of a tile lie further apart,
// in a block or from block to block, a launch of its own (FAR) takes the rest of the workgroup's
// run: codes are operands as they are, the scores are multiplied by the powers of K's pages, and the
// probabilities by those of V's over the largest that the token itself has attended to (rounded at
// 2^-35 of that).  So rows that a token leaves out change nothing for it, however large they are.
// q is scaled by the power of two of its row's largest value: one f16 term holds all of bf16 and f16
// values (but for bits below 2^-25 of that largest), two 22 bits of fp32.  Probabilities, times 2^10,
// are one term for bf16 outputs (error 2^-11 of each at most, where the output's own rounding is 2^-8:
// 0.1 to 0.6% more error than that rounding alone), two for f16 and fp32 (with one, f16 outputs had 1.1
// to 1.5 times the error of their rounding; chunk of 2048 tokens on 30011 rows 1390 us with two against
// 1095, 6 prompts 91 against 80).  Scores, maxima, sums and outputs are fp32; the maximum is taken anew
// only when a score passes it by 2^5.
//
// Measured (kernel trace, then the join; an f16 product of 8192^3 reaches 1196 TFLOP/s):
//  * a chunk of 2048 tokens on 30011 rows, 32 heads over 8 of 128 values, bf16: 1110 to 1250 us
//    with the clock, and 16; 1.04 PFLOP at 830 to 940 TFLOP/s.  The matrix cores are busy for 41% of the
//    cycles, vector instructions issue in most of the rest.  Two rows of q per lane, which halve LDS's
//    part, left one wave per SIMD: 2208 us.
//  * 6 prompts of 100 to 2500 tokens, window 1024, 24 heads over 8 of 128 values: 78 and 10.6; a workgroup
//    has some two tiles of six blocks, 2.2 us for its place, some 10 us a tile beside its blocks.
//  * 16 drafts of 5 tokens on 1 to 6000 rows, 32 heads over 8 of 64 values, fp32: 22.4 and 7.6.
//  * 1024 tokens on 8000 rows, 32 heads over 8 (whole calls), 64, 128 and 256 values: bf16 125, 192 and 481 us, f16
//    153, 235 and 558, fp32, twice the products, 167, 325 and 845.
#include <type_traits>

#include "cache_internal.h"

#define SHERRY_INLINE __attribute__((always_inline))

namespace sherry {
namespace {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kQRows = 32 * kWaves;  // of a tile
constexpr int kRows = 64;            // of K and V at a time
constexpr int kCus = 256, kXcds = 8;
// What a tile costs besides its rows (its q, the first loads, the way out), in rows.  With 64 /
// 128 / 256 / 512: 16 drafts of 5 tokens 55.7 / 39.4 / 34.4 / 36.9 us, 6 prompts of 100 to 2500
// tokens 163 / 125 / 93 / 90 (a run's end near a tile's begin or end goes there, block_at).
constexpr int kTileCost = 256;
// The shortest run, in rows of cost.  With 128 / 256 / 512: the drafts 30.7 / 30.6 / 33.4 us, one
// sequence of 3000 rows and 5 tokens 22.6 / 22.7 / 27.1, one prompt of 500 tokens 36.4 / 34.9 / 38.2.
constexpr int kMinRun = 256;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kMinusInf = -__builtin_huge_valf();
constexpr float kUp = 10.0f;         // p is held times 2^kUp
// Scores may pass the maximum by this (with 0, where o is rescaled at every new maximum, 6
// prompts 94.4 us against 92.7).
constexpr float kLazy = 5.0f;
// From here on a score's own rounding is in the way: an exponent taken from the unrounded product is
// off from the maximum by a part of the rounding, without bound, and kUp would be rounded too.
constexpr float kLarge = 0x1p22f;
constexpr float kNowhere = -__FLT_MAX__;  // base where nothing is attended to yet
// A code times 2^0 .. 2^-15 is exact in f16: K's powers may differ by this in a block, V's in a block and
// from one block's largest to another's.
constexpr int kFarK = 15, kFarV = 8, kFarBlocks = 7;
// K's largest biased exponent that scores may be multiplied by at once (past it the factor of rows that
// a token leaves out could be infinite).
constexpr int kMostK = 127 + 64;

// A tile that workgroup w has the beginning of, and `last` the end: its tokens [first, first
// + tokens) and query heads.  tokens = 0: there is none.
struct Split {
  int first, tokens, head0, heads, last;
};

struct Tokens {
  Cache c;
  const void* q;
  void* out;
  const int32_t* first;
  const int32_t* length;
  const uint8_t* mask;
  // what workgroup w found for the tile that its run begins in (part 2 w), and for the
  // one that begins in its run and goes on behind it (2 w + 1)
  float2* stat;  // [part][part_rows]: where p is 1, in units of ln 2, and the sum of p
  float* sums;   // [part][part_rows][DP]: outputs of these rows
  Split* split;  // [workgroup]
  int64_t* rest;  // [workgroup]: the unit from which FAR takes its run, or -1
  int64_t q_stride, out_stride, mask_stride;
  int tokens, heads, group, gtiles, per_tile, hp, type, window, groups, part_rows;
  float scale;
  FastDiv by_hp, by_tile;
};

// ---- which tiles a workgroup takes -------------------------------------------

// A sequence's tokens [t0, t0 + n), its rows before them, and its tiles per head.
struct Seq {
  int t0, n, len, tiles;
};
__device__ __forceinline__ Seq seq_of(const Tokens& a, int b) {
  const int f0 = as_global(a.first)[b], f1 = as_global(a.first)[b + 1];
  const int t0 = f0 < 0 ? 0 : f0 < a.tokens ? f0 : a.tokens;
  const int t1 = f1 < t0 ? t0 : f1 < a.tokens ? f1 : a.tokens;
  return Seq{t0, t1 - t0, a.c.length(a.length, b), static_cast<int>(a.by_tile.div(t1 - t0 + a.per_tile - 1))};
}
// The rows that the first k tiles of a head attend to, and kTileCost each: tile t the
// rows from max(0, len + 1 - window + t r) to len + min(n, (t + 1) r), r = tokens per tile.
__device__ __forceinline__ int64_t cost_of(const Tokens& a, const Seq& s, int k) {
  const int64_t r = a.per_tile, kk = k;
  int64_t sum = kk * (s.len + kTileCost) + r * (kk * (kk + 1) / 2);
  if (k == s.tiles) sum -= kk * r - s.n;
  if (a.window) {
    const int64_t low = int64_t(s.len) + 1 - a.window;
    // (the first tile that leaves rows out)
    const int64_t from = low >= 0 ? 0 : int64_t(a.by_tile.div(static_cast<uint32_t>(-low - 1))) + 1;
    if (from < kk) sum -= (kk - from) * low + r * ((kk * (kk - 1) - from * (from - 1)) / 2);
  }
  return sum;
}

// What tile t alone costs.
__device__ __forceinline__ int64_t tile_cost(const Tokens& a, const Seq& s, int t) {
  const int64_t tok0 = int64_t(t) * a.per_tile, low = a.window ? s.len + 1 - a.window + tok0 : 0;
  return s.len + kTileCost + (t + 1 < s.tiles ? tok0 + a.per_tile : s.n) - (low > 0 ? low : 0);
}
// n / d for quotients below 2^50.  (A division of 64-bit integers is some 200 instructions,
// which every workgroup would have to fetch first.)
__device__ __forceinline__ int64_t divide(int64_t n, int64_t d) {
  int64_t q = static_cast<int64_t>(double(n) / double(d));
  if (q * d > n) --q;
  return (q + 1) * d <= n ? q + 1 : q;
}

struct Place {
  int b;    // -1: nowhere
  int head, t;    // key-value head and its tile of query heads; tile of tokens
  int64_t at;     // unit of the tile's cost
  Seq s;
};
__device__ __forceinline__ int64_t wave_scan64(int64_t v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t u = __shfl_up(v, o, 64);
    if (lane >= o) v += u;
  }
  return v;
}
__device__ __forceinline__ int64_t readlane64(int64_t v, int lane) {
  return int64_t(uint64_t(uint32_t(__builtin_amdgcn_readlane(int(v >> 32), lane))) << 32 |
                 uint32_t(__builtin_amdgcn_readlane(int(v), lane)));
}
// The first 64 sequences as the lanes have them, and what all sequences cost.
struct Costs {
  Seq s;
  int64_t head, upto, all;  // the lane's sequence: a head's tiles; the sequences' up to it
};
__device__ __forceinline__ Costs costs_from(const Tokens& a, int b0) {
  const int b = b0 + (threadIdx.x & 63);
  Costs c{{0, 0, 0, 0}, 0, 0, 0};
  if (b < a.c.batch) {
    c.s = seq_of(a, b);
    c.head = cost_of(a, c.s, c.s.tiles);
  }
  c.upto = wave_scan64(c.head * (int64_t(a.c.kv) * a.gtiles));
  c.all = readlane64(c.upto, 63);
  return c;
}
__device__ __forceinline__ Costs costs_of(const Tokens& a) {
  Costs c = costs_from(a, 0);
  for (int b0 = 64; b0 < a.c.batch; b0 += 64) c.all += costs_from(a, b0).all;
  return c;
}
// Where unit u of all tiles' cost lies.
__device__ __forceinline__ Place find_place(const Tokens& a, const Costs& first, int64_t u) {
  const int lane = threadIdx.x & 63;
  const int64_t heads = int64_t(a.c.kv) * a.gtiles;
  int64_t before = 0;
  for (int b0 = 0; b0 < a.c.batch; b0 += 64) {
    const Costs c = b0 == 0 ? first : costs_from(a, b0);
    const uint64_t past = __ballot(before + c.upto > u);
    if (!past) {
      before += readlane64(c.upto, 63);
      continue;
    }
    const int at = __builtin_ctzll(past);
    Place p;
    p.b = b0 + at;
    p.s = Seq{__builtin_amdgcn_readlane(c.s.t0, at), __builtin_amdgcn_readlane(c.s.n, at),
              __builtin_amdgcn_readlane(c.s.len, at), __builtin_amdgcn_readlane(c.s.tiles, at)};
    const int64_t head_cost = readlane64(c.head, at);
    int64_t in = u - before - (readlane64(c.upto, at) - head_cost * heads);
    const int64_t head = divide(in, head_cost);
    p.head = static_cast<int>(head);
    in -= head * head_cost;
    int lo = 0, n = p.s.tiles;  // the last tile that begins at or before `in`, by 64 probes a step
    for (;;) {
      const int step = (n + 63) / 64, probe = lane * step;
      const uint64_t not_past = __ballot(probe < n && cost_of(a, p.s, lo + (probe < n ? probe : 0)) <= in);
      const int k = __builtin_popcountll(not_past) - 1;  // (at least one: a tile begins at 0)
      lo += (k > 0 ? k : 0) * step;
      n = step < n - (k > 0 ? k : 0) * step ? step : n - (k > 0 ? k : 0) * step;
      if (step == 1) break;
    }
    p.t = lo;
    p.at = in - cost_of(a, p.s, lo);
    return p;
  }
  return Place{-1, 0, 0, 0, {0, 0, 0, 0}};
}
// The first tile of the next sequence from b on that has tokens (by find_place, whose scan begins
// at the first sequence: 4096 sequences of 100 rows and a token 469 us against 219, 6 prompts 86
// against 82, as its registers are not held then).
__device__ __forceinline__ Place next_place(const Tokens& a, int b) {
  const int lane = threadIdx.x & 63;
  for (; b < a.c.batch; b += 64) {
    const Seq s = b + lane < a.c.batch ? seq_of(a, b + lane) : Seq{0, 0, 0, 0};
    const uint64_t some = __ballot(s.n > 0);
    if (!some) continue;
    const int at = __builtin_ctzll(some);
    return Place{b + at, 0, 0, 0,
                 Seq{__builtin_amdgcn_readlane(s.t0, at), __builtin_amdgcn_readlane(s.n, at),
                     __builtin_amdgcn_readlane(s.len, at), __builtin_amdgcn_readlane(s.tiles, at)}};
  }
  return Place{-1, 0, 0, 0, {0, 0, 0, 0}};
}
__device__ __forceinline__ int64_t run_of(const Tokens& a, int64_t all) {
  const int64_t run = divide(all + a.groups - 1, a.groups);
  return run < kMinRun ? kMinRun : run;
}

// The rows of K and V that a tile reads: blocks [k0, k1) of kRows, up to row end.
struct Span {
  int k0, k1, end;
};
__device__ __forceinline__ Span span_of(const Tokens& a, const Seq& s, int t) {
  const int64_t tok0 = int64_t(t) * a.per_tile;
  const int64_t tok1 = tok0 + a.per_tile < s.n ? tok0 + a.per_tile : s.n;
  const int64_t end = s.len + tok1 < a.c.rows ? s.len + tok1 : a.c.rows;
  int64_t low = a.window ? s.len + tok0 + 1 - a.window : 0;
  low = low < 0 ? 0 : low < end ? low : end;
  return Span{static_cast<int>(low / kRows), static_cast<int>((end + kRows - 1) / kRows), static_cast<int>(end)};
}
// A run's end inside a tile, at unit `at` of its cost: the block of its rows that it stands
// for.  Near the tile's begin or end it is that (k0 or k1), so that no workgroup takes up a
// tile for a few rows of it.
__device__ __forceinline__ int block_at(const Span& sp, int64_t at, int64_t cost) {
  if (at < kTileCost) return sp.k0;
  if (cost - at < kTileCost) return sp.k1;
  const int64_t k = sp.k0 + (at - kTileCost / 2) / kRows;
  return k < sp.k1 ? static_cast<int>(k) : sp.k1;
}

// The kernel's arguments, to be read where this is called.
__device__ __forceinline__ const SHERRY_CONST Tokens* late_args() {
  uint64_t p = (uint64_t)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return (const SHERRY_CONST Tokens*)p;
}

// ---- operands -----------------------------------------------------------------

__device__ __forceinline__ v16f mfma(const u32x4& a, const u32x4& b, const v16f& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
}
__device__ __forceinline__ uint32_t pair_f16(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, v2h{static_cast<_Float16>(lo), static_cast<_Float16>(hi)});
}
__device__ __forceinline__ uint32_t pair_bf16(float lo, float hi) {
  typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, v2bf{static_cast<__bf16>(lo), static_cast<__bf16>(hi)});
}
// Two values as NT terms each: x = t[0] + t[1] up to the last one's rounding.
template <int NT>
__device__ __forceinline__ void split(float lo, float hi, uint32_t (&t)[NT]) {
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    t[n] = pair_f16(lo, hi);
    if (n + 1 < NT) {
      const v2h h = __builtin_bit_cast(v2h, t[n]);
      lo -= static_cast<float>(h[0]);
      hi -= static_cast<float>(h[1]);
    }
  }
}
// Codes 0 and 1, or 2 and 3, of a word, times a power of two (hi: known when compiled).
__device__ __forceinline__ uint32_t code_pair(uint32_t x, float times, bool hi) {
  return __builtin_bit_cast(uint32_t, hi ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(static_cast<int>(x), times, true)
                                         : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(static_cast<int>(x), times, false));
}
__device__ __forceinline__ float power(int biased) { return __uint_as_float(uint32_t(biased) << 23); }
// Biased exponent of a page's scale, 1 .. 254.
__device__ __forceinline__ int exponent(float scale) {
  const int e = static_cast<int>(__float_as_uint(scale) >> 23) & 0xFF;
  return e < 1 ? 1 : e < 254 ? e : 254;
}
// The larger of a value in the lanes n and n + 32.
__device__ __forceinline__ float max_of_halves(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ uint32_t max_of_halves(uint32_t v) {
  const auto a = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return a[0] > a[1] ? a[0] : a[1];
}
// The largest of two 16-bit values over the wave (steps inside 16 lanes, then across them).
__device__ __forceinline__ uint32_t wave_max_pairs(uint32_t v) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  auto with = [&](uint32_t u) {
    v = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, v), __builtin_bit_cast(u16x2, u)));
  };
  with(__builtin_amdgcn_update_dpp(v, v, 0x111, 0xF, 0xF, false));
  with(__builtin_amdgcn_update_dpp(v, v, 0x112, 0xF, 0xF, false));
  with(__builtin_amdgcn_update_dpp(v, v, 0x114, 0xF, 0xF, false));
  with(__builtin_amdgcn_update_dpp(v, v, 0x118, 0xF, 0xF, false));
  with(__builtin_amdgcn_update_dpp(v, v, 0x142, 0xA, 0xF, false));
  with(__builtin_amdgcn_update_dpp(v, v, 0x143, 0xC, 0xF, false));
  return __builtin_amdgcn_readlane(v, 63);
}

// K in LDS: rows of DP f16 values, 16 bytes further apart than they are long.
// V: DP rows of 64 f16 values, those of one step of 16 rows and lane half in a
// piece of 16 bytes (rows 4 g + 0..3 and 8 + 4 g + 0..3 of the 16); piece p of row d is
// at place p ^ (d / 2 % 8) ^ (d / 16 % 8), so that reads (16 rows at once) and writes (VB
// rows apart) spread over the banks.
template <int DP>
struct Lds {
  static constexpr int KW = DP * 2 + 16, K = kRows * KW, V = DP * kRows * 2;
  alignas(16) char k[2][K];
  alignas(16) char v[2][V];
  // of eight blocks:
  int64_t at[8][kRows];     // where a row begins in its pool (of no page: a place that can be read)
  float kx[8][kRows], vx[8][kRows];  // what its codes are multiplied by
  uint8_t ke[8][kRows], ve[8][kRows];  // FAR: the biased exponents of its page's scales
  // which rows there are (64 bits); kref | vref << 8 | part << 16, the biased exponents that
  // the products with kx and vx are over, and whether not every row of the tile attends to all
  u32x4 about[8];
  int vmax[8];              // the largest biased exponent of V's scales (0: no rows); 256 where some lie far below
  int nan[16];               // and some code of V is NaN:
  alignas(16) uint8_t odd[2][DP][16];  // of a value and four rows, a bit each
};

// Waves per SIMD that the registers allow.  One more, spilling: chunk of 2048 tokens on 30011
// rows of 128 values 1824 us against 1156, drafts of 64 values and two terms 59.0 against 34.4;
// one fewer 1753 and 32.8.
__host__ __device__ constexpr int waves_for(int dp, int terms) {
  return dp == 256 ? 1 : dp == 128 ? 2 : terms == 1 ? 3 : 2;
}

// Nothing is moved over this when compiled: operands are read from LDS a group ahead of
// their use.  (Left to itself the compiler read each right before its use, and waited for it.)
__device__ __forceinline__ void fence() { __builtin_amdgcn_sched_barrier(0); }

// A row of q as it lies (fp32 with two terms, else 16 bits), values 16 st + 8 g ...  (One
// address and fixed steps: with a condition and an address for each, the eight reads waited
// for each other's, 8 us.)
template <int DP, int NT>
__device__ __forceinline__ void load_q(const Tokens& a, int64_t at, u32x4 (&raw)[DP / 16][NT]) {
  const int g = (threadIdx.x & 63) >> 5;
  const SHERRY_GLOBAL u32x4* p =
      reinterpret_cast<const SHERRY_GLOBAL u32x4*>(as_global(static_cast<const char*>(a.q)) + (at + 8 * g) * (2 * NT));
#pragma unroll
  for (int st = 0; st < DP / 16; ++st)
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      raw[st][j] = u32x4{0, 0, 0, 0};
      if (16 * st < a.c.dim) raw[st][j] = p[2 * NT * st + j];
    }
}
// The same in terms, over the power of two of its largest value; returns the factor of its
// scores in units of ln 2 (the sign of scale goes into q).
template <int DP, int NT>
__device__ __forceinline__ float split_q(const Tokens& a, const u32x4 (&raw)[DP / 16][NT], u32x4 (&qf)[NT][DP / 16]) {
  constexpr int KS = DP / 16;
  const bool bf16 = a.type == SHERRY_BF16;
  auto pair = [&](int st, int i, float& lo, float& hi) {  // values 2 i, 2 i + 1 of a step
    if constexpr (NT == 2) {
      lo = __uint_as_float(raw[st][i >> 1][2 * (i & 1)]);
      hi = __uint_as_float(raw[st][i >> 1][2 * (i & 1) + 1]);
    } else {
      const uint32_t x = raw[st][0][i];
      const v2h h = __builtin_bit_cast(v2h, x);
      lo = bf16 ? __uint_as_float(x << 16) : static_cast<float>(h[0]);
      hi = bf16 ? __uint_as_float(x & 0xFFFF0000u) : static_cast<float>(h[1]);
    }
  };
  uint32_t most = 0;
#pragma unroll
  for (int st = 0; st < KS; ++st)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float lo, hi;
      pair(st, i, lo, hi);
      const uint32_t l = __float_as_uint(lo) & 0x7FFFFFFFu, h = __float_as_uint(hi) & 0x7FFFFFFFu;
      most = l > most ? l : most;
      most = h > most ? h : most;
    }
  most = max_of_halves(most);
  constexpr uint32_t kTiny = 0x00400000u;  // 2^-127
  const uint32_t e = most >> 23 < 254 ? most >> 23 : 254;
  const float down = __uint_as_float(e < 254 ? (254 - e) << 23 : kTiny) * (a.scale < 0 ? -1.0f : a.scale > 0 ? 1.0f : 0.0f);
#pragma unroll
  for (int st = 0; st < KS; ++st) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float lo, hi;
      pair(st, i, lo, hi);
      uint32_t t[NT];
      split<NT>(lo * down, hi * down, t);
#pragma unroll
      for (int j = 0; j < NT; ++j) qf[j][st][i] = t[j];
    }
    fence();
  }
  return fabsf(a.scale) * kLog2e * __uint_as_float(e > 0 ? e << 23 : kTiny);
}

// N times an MFMA and VALU other instructions.
template <int N, int VALU>
__device__ __forceinline__ void take_turns() {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x402, VALU, 0);
  }
}

// DP: head_dim rounded up to 64, 128 or 256; NT, NP: terms of q and p; QUADS: page_size % 4
// == 0, so that four rows of V together have one factor (6 prompts 92.7 us against 97.5 without,
// the chunk 1156 against 1169).  FAR: powers anywhere; takes what the launch without it has left (in one
// launch with both, a row's own powers in every block's loop: chunk of 2048 tokens on 30011 rows 1159 us against
// 1108, 6 prompts 89 against 80; a launch with nothing to take is 1 to 2 us).  1024 bf16 tokens on 8000 rows of 128
// values, powers of pages anywhere in 2^-30 .. 1: 362 us, where they are near each other 192 (64 values 274 and 125, 256 950
// and 480, fp32 of 128 650 and 317).
template <int DP, int NT, int NP, bool QUADS, bool FAR>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(waves_for(DP, NT)))) void tokens_kernel(
    Tokens a) {
  constexpr int KS = DP / 16;   // MFMA steps of a score
  constexpr int DB = DP / 32;   // blocks of 32 values of V
  constexpr int KP = DP / 64;   // 16-byte pieces of K per thread
  constexpr int KR = 4096 / DP; // rows from one to the next
  constexpr int VB = DP / 16;   // bytes of V per thread and row
  constexpr int VW = VB / 4;
  constexpr int KW = Lds<DP>::KW, VROW = 2 * kRows;
  __shared__ Lds<DP> lds;
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // consecutive runs on one XCD (workgroups go to them in turn)
  const int w = blockIdx.x % kXcds * (a.groups / kXcds) + blockIdx.x / kXcds;
  if constexpr (FAR) {
    if (as_const(a.rest)[w] < 0) return;
  }
  const Costs costs = costs_of(a);
  const int64_t run = run_of(a, costs.all);
  int64_t u = int64_t(w) * run;
  const int64_t u_end = u + run < costs.all ? u + run : costs.all;
  if constexpr (FAR) {
    u = as_const(a.rest)[w];
  } else if (tid == 0) {
    as_global_mut(a.split)[w] = Split{0, 0, 0, 0, 0};
    as_global_mut(a.rest)[w] = -1;
  }
  if (u >= u_end) return;
  Place pl = find_place(a, costs, u);
  if (pl.b < 0) return;  // (as below)

  // this thread's places: of K a piece of 16 codes, of V some codes of four rows.
  // (Values past head_dim are those at 0: q has zeros there, and outputs are not written.)
  const int k_row = tid / (DP / 16), k_dim = 16 * (tid % (DP / 16));
  const int k_d = k_dim < a.c.dim ? k_dim : 0, k_to = k_row * KW + 2 * k_dim;
  const int quad = tid / 16, col = tid % 16, v_d = VB * col < a.c.dim ? VB * col : 0;
  const int v_to = VB * col * VROW + 8 * (quad >> 1 & 1);
  const int v_piece = 16 * ((2 * (quad >> 2) + (quad & 1)) ^ (VB * col >> 1 & 7) ^ (VB * col >> 4 & 7));
  // and of the operands
  const int k_from = n * KW + 16 * g, v_from = n * VROW, v_swap = (n >> 1 & 7) ^ (n >> 4) ^ g;

  for (;;) {
    const Seq& s = pl.s;
    const int64_t cost = tile_cost(a, s, pl.t);
    const int64_t upto = cost - pl.at < u_end - u ? cost : pl.at + (u_end - u);
    if (upto <= pl.at) return;  // (first is not ascending, and the costs past 63 bits)
    const Span sp = span_of(a, s, pl.t);
    const int b = __builtin_amdgcn_readfirstlane(pl.b);
    const int kb0 = __builtin_amdgcn_readfirstlane(block_at(sp, pl.at, cost));
    const int kb1 = __builtin_amdgcn_readfirstlane(block_at(sp, upto, cost));
    const bool begins = kb0 == sp.k0, whole = begins && kb1 == sp.k1;
    const int end = __builtin_amdgcn_readfirstlane(sp.end);
    const int kvh = __builtin_amdgcn_readfirstlane(a.gtiles == 1 ? pl.head : pl.head / a.gtiles);
    const int head0 = kvh * a.group + (pl.head - kvh * a.gtiles) * a.hp;
    const int heads = (kvh + 1) * a.group - head0 < a.hp ? (kvh + 1) * a.group - head0 : a.hp;
    // a lane's row of q (where the tile has none for it: the first one, of which nothing comes)
    struct Row {
      int r, tok, token, head;
      bool mine;
    };
    auto row_of = [&](int lane_row) SHERRY_INLINE {
      const int r = wave * 32 + lane_row, tok = a.by_hp.div(r), hd = r - tok * a.hp;
      const int64_t in_seq = int64_t(pl.t) * a.per_tile + tok;
      const bool mine = tok < a.per_tile && in_seq < s.n && hd < heads;
      return Row{r, static_cast<int>(mine ? in_seq : 0), s.t0 + static_cast<int>(mine ? in_seq : 0),
                 head0 + (mine ? hd : 0), mine};
    };
    const Row row = row_of(n);
    const bool mine = row.mine;
    const int64_t own = int64_t(s.len) + row.tok + 1;  // rows up to its own
    const int lim = mine ? static_cast<int>(own < a.c.rows ? own : a.c.rows) : 0;
    const int64_t low64 = a.window ? own - a.window : 0;
    const int low = mine && low64 > 0 ? static_cast<int>(low64 < a.c.rows ? low64 : a.c.rows) : 0;
    const bool active = __any(mine);  // (the tile may have fewer rows than the workgroup)
    // the first token of the tile attends to rows before all_lim, the last to those from all_low
    const int64_t own0 = s.len + int64_t(pl.t) * a.per_tile + 1;
    const int all_lim = __builtin_amdgcn_readfirstlane(static_cast<int>(own0 < end ? own0 : end));
    const int64_t low1 = a.window ? own0 + a.per_tile - a.window : 0;
    const int all_low = __builtin_amdgcn_readfirstlane(static_cast<int>(low1 < 0 ? 0 : low1 < end ? low1 : end));

    u32x4 qraw[KS][NT], qf[NT][KS];
    float factor = 0.0f;

    v16f o[DB];
    float base = kNowhere, limit = kMinusInf, l = 0.0f;  // limit: scores past it move base
    int vrun = 1;  // o is over this power of two

    // ---- what the waves find out about blocks of rows, each about every fourth block:
    // its pages, their scales, the largest of these, and what follows for its rows ----
    int next_page = -1, next_mask = 1, seen_vref = 1, seen_vlow = 255, next_kref = 1;
    int stop = kb1;  // the first group of blocks that FAR has to take
    int64_t next_at = 0;
    float next_ks = 0, next_vs = 0;
    bool next_ok = false;
    auto look_page = [&](int kb) SHERRY_INLINE {
      const int row = (kb + wave) * kRows + lane;
      const bool in = kb + wave < kb1 && row < end;
      next_page = in ? as_global(a.c.table)[int64_t(b) * a.c.width + a.c.by_page.div(row)] : -1;
      next_mask = in && a.mask ? as_global(a.mask)[int64_t(b) * a.mask_stride + row] : 1;
    };
    auto look_scale = [&](int kb) SHERRY_INLINE {  // (rows of no page: any place that can be read)
      const int row = (kb + wave) * kRows + lane;
      const bool there = next_page >= 0 && next_page < a.c.pages;
      next_ok = there && next_mask != 0;
      const int page = there ? next_page : 0;
      const int off = there ? row - static_cast<int>(a.c.by_page.div(row)) * a.c.page_size : 0;
      next_at = a.c.at(page, kvh) + int64_t(off) * a.c.dim;
      next_ks = as_global(a.c.ks)[a.c.one_scale_at(page, kvh)];
      next_vs = as_global(a.c.vs)[a.c.one_scale_at(page, kvh)];
    };
    auto look_refs = [&](int kb) SHERRY_INLINE {
      if constexpr (!FAR) {
        // (largest of both at once; a row that is masked shares its factor with others of its page)
        const int ke = exponent(next_ks), ve = exponent(next_vs);
        const uint32_t top = wave_max_pairs(next_ok ? static_cast<uint32_t>(ke | ve << 16) : 0u);
        const int vref = top >> 16;
        next_kref = top & 0xFFFF;
        const bool far = __any(next_ok && (ke + kFarK < next_kref || ve + kFarV < vref)) || next_kref > kMostK;
        if (lane == 0) lds.vmax[(kb - kb0 + wave) & 7] = far ? vref | 256 : vref;
      }
    };
    auto publish = [&](int kb) SHERRY_INLINE {
      const int slot = (kb - kb0 + wave) & 7;
      if constexpr (!FAR) {
        bool far = false;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
          const int v = __builtin_amdgcn_readfirstlane(lds.vmax[(kb - kb0 + i) & 7]), top = v & 0xFF;
          seen_vref = top > seen_vref ? top : seen_vref;
          seen_vlow = top > 0 && top < seen_vlow ? top : seen_vlow;
          far = far || v > 255;
        }
        if (far || seen_vref > seen_vlow + kFarBlocks) stop = stop < kb ? stop : kb;
      }
      auto over = [](int ref, int e) { return power(ref - e < 0 ? 127 : ref - e < 126 ? 127 - (ref - e) : 1); };
      lds.at[slot][lane] = next_at;
      lds.kx[slot][lane] = FAR ? 1.0f : over(next_kref, exponent(next_ks));
      lds.vx[slot][lane] = FAR ? 1.0f : over(seen_vref, exponent(next_vs));
      if constexpr (FAR) {
        lds.ke[slot][lane] = static_cast<uint8_t>(exponent(next_ks));
        lds.ve[slot][lane] = static_cast<uint8_t>(exponent(next_vs));
      }
      const uint64_t valid = __ballot(next_ok);
      const int row0 = (kb + wave) * kRows;
      if (lane == 0) {
        const bool part = FAR || ~valid != 0 || row0 + kRows > all_lim || row0 < all_low;
        lds.about[slot] = u32x4{static_cast<uint32_t>(valid), static_cast<uint32_t>(valid >> 32),
                                static_cast<uint32_t>(next_kref | seen_vref << 8 | int(part) << 16), 0};
        lds.nan[(kb - kb0 + wave) & 15] = 0;
      }
    };

    // ---- a block's rows, from the pools to LDS ----
    u32x4 kr[KP];
    uint32_t vr[4][VW];
    auto load = [&](int slot) SHERRY_INLINE {
#pragma unroll
      for (int i = 0; i < KP; ++i)
        kr[i] = *reinterpret_cast<const SHERRY_GLOBAL u32x4*>(as_global(a.c.k) + lds.at[slot][k_row + KR * i] + k_d);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const SHERRY_GLOBAL char* from = as_global(a.c.v) + lds.at[slot][4 * quad + j] + v_d;
        if constexpr (VW == 4) {
          const u32x4 x = *reinterpret_cast<const SHERRY_GLOBAL u32x4*>(from);
#pragma unroll
          for (int i = 0; i < 4; ++i) vr[j][i] = x[i];
        } else if constexpr (VW == 2) {
          const u32x2 x = *reinterpret_cast<const SHERRY_GLOBAL u32x2*>(from);
          vr[j][0] = x[0];
          vr[j][1] = x[1];
        } else {
          vr[j][0] = *reinterpret_cast<const SHERRY_GLOBAL uint32_t*>(from);
        }
      }
    };
    auto fill = [&](int buf, int rel) SHERRY_INLINE {
      const int slot = rel & 7;
      if (__builtin_amdgcn_readfirstlane(lds.about[slot][2]) >> 16) {
        // NaN must not reach rows of q that do not attend to it: it is 0 here, and noted
        uint32_t any = 0;
#pragma unroll
        for (int i = 0; i < VW; ++i) {
          uint32_t bits = 0;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t t = ((vr[j][i] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
            bits |= t >> (7 - j);
            vr[j][i] &= ~(t | (t - (t >> 7)));
          }
          any |= bits;
#pragma unroll
          for (int e = 0; e < 4; ++e) lds.odd[buf][VB * col + 4 * i + e][quad] = static_cast<uint8_t>(bits >> (8 * e));
        }
        if (any) lds.nan[rel & 15] = 1;
      }
#pragma unroll
      for (int i = 0; i < KP; ++i) {
        const float times = lds.kx[slot][k_row + KR * i];
        u32x4 x[2];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[j >> 1][2 * (j & 1)] = code_pair(kr[i][j], times, false);
          x[j >> 1][2 * (j & 1) + 1] = code_pair(kr[i][j], times, true);
        }
        u32x4* to = reinterpret_cast<u32x4*>(lds.k[buf] + k_to + KR * i * KW);
        to[0] = x[0];
        to[1] = x[1];
      }
      float times[4] = {lds.vx[slot][4 * quad], 0, 0, 0};
      if constexpr (!QUADS)
#pragma unroll
        for (int j = 1; j < 4; ++j) times[j] = lds.vx[slot][4 * quad + j];
#pragma unroll
      for (int i = 0; i < VW; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          u32x2 x;
          if constexpr (QUADS) {
            const uint32_t sel = e & 2 ? 0x07030602u : 0x05010400u;  // (values e and e ^ 1 of two rows)
            x[0] = code_pair(__builtin_amdgcn_perm(vr[1][i], vr[0][i], sel), times[0], e & 1);
            x[1] = code_pair(__builtin_amdgcn_perm(vr[3][i], vr[2][i], sel), times[0], e & 1);
          } else {
            uint32_t y[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint32_t z = code_pair(vr[j][i], times[j], e & 2);
              y[j] = e & 1 ? z >> 16 : z & 0xFFFFu;
            }
            x[0] = y[0] | y[1] << 16;
            x[1] = y[2] | y[3] << 16;
          }
          constexpr int kSwap = VB / 2 < 8 ? VB / 2 : 8;
          const int d = 4 * i + e;
          *reinterpret_cast<u32x2*>(lds.v[buf] + v_to + (v_piece ^ 16 * (d / 2 % kSwap)) + d * VROW) = x;
        }
    };

    // ---- a block's scores, probabilities and outputs ----
    auto attend = [&](int kb, int buf) SHERRY_INLINE {
      const int row0 = kb * kRows;
      const char* kp = lds.k[buf] + k_from;
      const char* vp = lds.v[buf] + v_from;
      constexpr int GROUP = 4, GROUPS = 2 * KS / GROUP;
      u32x4 kf[2][GROUP], vf[2][DB];
      auto read_k = [&](int grp) {  // of 16 values after 16, both halves of the rows
#pragma unroll
        for (int i = 0; i < GROUP; ++i)
          kf[grp & 1][i] = *reinterpret_cast<const u32x4*>(kp + 32 * (i & 1) * KW + 32 * (grp * GROUP / 2 + i / 2));
      };
      auto read_v = [&](int st) {  // of 16 rows after 16
#pragma unroll
        for (int db = 0; db < DB; ++db)
          vf[st & 1][db] = *reinterpret_cast<const u32x4*>(vp + 16 * (2 * (st ^ (db & 3)) ^ v_swap) + 32 * db * VROW);
      };
      const u32x4 about = lds.about[(kb - kb0) & 7];
      read_k(0);
      v16f sc[2] = {v16f{}, v16f{}};
#pragma unroll
      for (int grp = 0; grp < GROUPS; ++grp) {
        if (grp + 1 < GROUPS) read_k(grp + 1);
        else read_v(0);
        fence();
#pragma unroll
        for (int i = 0; i < GROUP; ++i)
#pragma unroll
          for (int j = NT - 1; j >= 0; --j)
            sc[i & 1] = mfma(kf[grp & 1][i], qf[j][grp * GROUP / 2 + i / 2], sc[i & 1]);
        fence();
      }
      const uint32_t refs = __builtin_amdgcn_readfirstlane(about[2]);
      const bool part = refs >> 16;
      int vref = refs >> 8 & 0xFF;
      // (above 0, so that -infinity stays what it is)
      float f = fmaxf(FAR ? factor : factor * power(refs & 0xFF), 0x1p-126f);
      // the rows that this row of q attends to
      auto attended = [&](int h) {
        const int most = lim - row0 - 32 * h, least = low - row0 - 32 * h;
        const uint32_t bits = most >= 32 ? ~0u : most > 0 ? (1u << most) - 1 : 0u;
        return bits & (least >= 32 ? 0u : least > 0 ? ~0u << least : ~0u) & about[h];
      };
      if (part) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t ok = attended(h) >> (4 * g);
#pragma unroll
          for (int i = 0; i < 16; ++i) sc[h][i] = (ok >> (8 * (i / 4) + i % 4)) & 1 ? sc[h][i] : kMinusInf;
        }
      }
      auto exponent_of = [&](const uint8_t (&x)[8][kRows], int h, int i) SHERRY_INLINE {  // of a score's row
        const uint8_t* four = &x[(kb - kb0) & 7][32 * h + 8 * (i / 4) + 4 * g];
        return *reinterpret_cast<const uint32_t*>(four) >> (8 * (i % 4)) & 0xFF;
      };
      if constexpr (FAR) {
        uint32_t most = 1;  // of V's exponents in attended rows
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const uint32_t v = exponent_of(lds.ve, h, i);
            most = v > most && sc[h][i] != kMinusInf ? v : most;
            sc[h][i] = sc[h][i] * f * power(exponent_of(lds.ke, h, i));
          }
        f = 1.0f;
        vref = static_cast<int>(max_of_halves(most));
        vref = vref > vrun ? vref : vrun;
      }
      float top = sc[0][0];
#pragma unroll
      for (int i = 1; i < 32; ++i) top = fmaxf(top, sc[i >> 4][i & 15]);
      top = max_of_halves(top) * f;
      if (FAR ? __any(top > limit || vref > vrun) : __any(top > limit) || vref > vrun) {
        const float over = fabsf(top) < kLarge ? top - kUp : top, to = over > base ? over : base;
        float down = __builtin_amdgcn_exp2f(base - to);
        base = to;
        limit = fabsf(to) < kLarge ? to + (kUp + kLazy) : kMinusInf;
        l *= down;
        if constexpr (FAR) down = __builtin_amdgcn_ldexpf(down, vrun - vref);
        else down *= power(vref - vrun < 126 ? 127 - (vref - vrun) : 1);  // (so far only where o is 0)
        vrun = vref;
#pragma unroll
        for (int i = 0; i < DB; ++i)
#pragma unroll
          for (int j = 0; j < 16; ++j) o[i][j] *= down;
      }
      // (all scores rounded once, as top is.  A branch of its own: inside the one before, 1024 fp32 tokens on 8000
      // rows of 128 values took 338 us against 317)
      if (!FAR && __builtin_expect(__any(limit == kMinusInf && base > kNowhere), 0)) {
#pragma unroll
        for (int i = 0; i < 32; ++i) sc[i >> 4][i & 15] *= f;
        f = 1.0f;
      }
      float from = base;
      if constexpr (FAR) {  // p's sum, and the exponents of p times V's powers
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            // (over base first: a large score's rounding is more than V's exponent)
            const float x = sc[h][i] - base;
            l += __builtin_amdgcn_exp2f(x);
            sc[h][i] = x + static_cast<float>(static_cast<int>(exponent_of(lds.ve, h, i)) - vrun);
          }
        from = 0.0f;
      }
      float sum[2] = {0.0f, 0.0f};
      u32x4 pf[2][NP];
      auto probabilities = [&](int st) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float p[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            p[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[st >> 1][8 * (st & 1) + 2 * i + j], f, -from));
            sum[j] += p[j];
          }
          uint32_t t[NP];
          split<NP>(p[0], p[1], t);
#pragma unroll
          for (int j = 0; j < NP; ++j) pf[st & 1][j][i] = t[j];
        }
      };
      // (Of two workgroups on a CU the older one was served first, 2.1 us a block against 3.2, and
      // the other ended alone: chunk of 2048 tokens on 30011 rows 1183 us.  With what is half
      // done first 1146; with turns by a clock 1136.)
      __builtin_amdgcn_s_setprio(1);
      probabilities(0);
#pragma unroll
      for (int st = 0; st < 4; ++st) {
        if (st < 3) read_v(st + 1);
        fence();
        if (st < 3) probabilities(st + 1);
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int j = NP - 1; j >= 0; --j) o[db] = mfma(vf[st & 1][db], pf[st & 1][j], o[db]);
        if (st < 3) take_turns<DB * NP, (28 + 24 * (NP - 1)) / (DB * NP)>();
        fence();
      }
      __builtin_amdgcn_s_setprio(0);
      if constexpr (!FAR) l += sum[0] + sum[1];
      if (part && __builtin_amdgcn_readfirstlane(lds.nan[(kb - kb0) & 15])) {
        u32x4 mine_of;  // the attended rows, four a byte
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          const uint32_t x = attended(h >> 1) >> (16 * (h & 1));
          mine_of[h] = (x & 0xF) | (x & 0xF0) << 4 | (x & 0xF00) << 8 | (x & 0xF000) << 12;
        }
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const u32x4 x = *reinterpret_cast<const u32x4*>(lds.odd[buf][32 * db + 8 * (j / 4) + 4 * g + j % 4]) & mine_of;
            o[db][j] = (x[0] | x[1] | x[2] | x[3]) ? __uint_as_float(0x7FC00000u) : o[db][j];
          }
      }
    };

    // A block's rows are read two blocks before their turn, and put into LDS one before it; what
    // the blocks are is known from two to five blocks before they are read.
    // (first reads first: pages and q, then what the pages lead to)
    if (kb0 < kb1) {
      look_page(kb0 + kWaves);
      const int later_page = next_page, later_mask = next_mask;
      look_page(kb0);
      load_q<DP, NT>(a, int64_t(row.token) * a.q_stride + int64_t(row.head) * a.c.dim, qraw);
      look_scale(kb0);
      const int64_t at = next_at;
      const float ks = next_ks, vs = next_vs;
      const bool ok = next_ok;
      next_page = later_page;
      next_mask = later_mask;
      look_scale(kb0 + kWaves);
      const int64_t later_at = next_at;
      const float later_ks = next_ks, later_vs = next_vs;
      const bool later_ok = next_ok;
      next_at = at, next_ks = ks, next_vs = vs, next_ok = ok;
      __syncthreads();  // (the tile before has been read from LDS)
      lds.at[wave][lane] = next_at;
      look_refs(kb0);
      __syncthreads();
      load(0);
      publish(kb0);
      next_at = later_at, next_ks = later_ks, next_vs = later_vs, next_ok = later_ok;
      factor = split_q<DP, NT>(a, qraw, qf);
      __syncthreads();
      fill(0, 0);
      load(1);
      __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < DB; ++i) o[i] = v16f{};
    // (four turns written out: what one has asked memory for, a later one takes, and no
    // answer has to be there where turns would join)
    auto turn = [&](auto turn_c, int kb) SHERRY_INLINE {
      constexpr int t = decltype(turn_c)::value;
      const int rel = kb - kb0;
      if (active) attend(kb, t & 1);
      // (behind the last block: rows of no page, of which nothing comes)
      fill((t & 1) ^ 1, rel + 1);
      if constexpr (t == 0) look_refs(kb + kWaves);
      if constexpr (t == 1) publish(kb - 1 + kWaves);
      if constexpr (t == 2) look_page(kb - 2 + 2 * kWaves);
      if constexpr (t == 3) look_scale(kb - 3 + 2 * kWaves);
      load((rel + 2) & 7);
      __syncthreads();
    };
    for (int kb = kb0; kb < stop; kb += 4) {
      turn(std::integral_constant<int, 0>{}, kb);
      if (kb + 1 >= kb1) break;
      turn(std::integral_constant<int, 1>{}, kb + 1);
      if (kb + 2 >= kb1) break;
      turn(std::integral_constant<int, 2>{}, kb + 2);
      if (kb + 3 >= kb1) break;
      turn(std::integral_constant<int, 3>{}, kb + 3);
    }

    if constexpr (!FAR) {
      if (__builtin_expect(stop < kb1, 0)) {
        if (tid == 0) as_global_mut(late_args()->rest)[w] = u;
        return;
      }
    }

    // ---- the way out: o over p's sum ----
    l += __shfl_xor(l, 32, 64);
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    // (arguments that only this part needs, read here: kept, they would take registers all the way)
    const SHERRY_CONST Tokens& late = *late_args();
    int again = n;  // (found anew: it would take registers all the way)
    asm volatile("" : "+v"(again));
    const Row out = row_of(again);
    if (out.mine && (kb0 < kb1 || whole)) {
      const float times = power(vrun);
      const int64_t part = int64_t(2 * w + begins) * late.part_rows + out.r;
      const int64_t at = whole ? int64_t(out.token) * late.out_stride + int64_t(out.head) * a.c.dim : part * DP;
      if (!whole && g == 0) as_global_mut(late.stat)[part] = make_float2(base, l);
      SHERRY_GLOBAL char* to = as_global_mut(static_cast<char*>(whole ? late.out : late.sums)) +
                               (at + 4 * g) * (whole && NT == 1 ? 2 : 4);
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int d = 32 * db + 8 * j;  // (and 4 g)
          if (16 * (d / 16) >= a.c.dim) continue;
          v4f x;
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = o[db][4 * j + i] * inv * times;
          if (NT == 2 || !whole)
            *reinterpret_cast<SHERRY_GLOBAL v4f*>(to + 4 * d) = x;
          else
            *reinterpret_cast<SHERRY_GLOBAL u32x2*>(to + 2 * d) =
                late.type == SHERRY_BF16 ? u32x2{pair_bf16(x[0], x[1]), pair_bf16(x[2], x[3])}
                                      : u32x2{pair_f16(x[0], x[1]), pair_f16(x[2], x[3])};
        }
    }

    if (tid == 0 && begins && kb0 < kb1 && !whole) {  // (another workgroup ends it)
      const int tok0 = pl.t * a.per_tile;
      const int64_t from = u - pl.at;
      // the last run whose begin leaves it a block (block_at): not those near the tile's end, and, of a tile
      // whose tokens lie past the table, not those behind its rows, which its cost counts all the same
      const int64_t rows_end = kTileCost / 2 + int64_t(sp.k1 - sp.k0) * kRows - 1, tile_end = cost - kTileCost;
      const int64_t last = divide(from + (rows_end < tile_end ? rows_end : tile_end), run);
      as_global_mut(late.split)[w] = Split{s.t0 + tok0, s.n - tok0 < a.per_tile ? s.n - tok0 : a.per_tile, head0, heads,
                                        static_cast<int>(last)};
    }
    u += upto - pl.at;
    if (u >= u_end) return;
    pl.at = 0;
    if (pl.t + 1 < s.tiles) {
      ++pl.t;
    } else if (pl.head + 1 < a.c.kv * a.gtiles) {
      ++pl.head;
      pl.t = 0;
    } else {
      pl = next_place(a, pl.b + 1);
      if (pl.b < 0) return;
    }
  }
}

// Workgroup w joins the tile that begins in run w and goes on behind it; blockIdx.y: a
// share of its rows.
constexpr int kJoinThreads = 1024;
template <int DP>
__global__ __launch_bounds__(kJoinThreads) void tokens_join_kernel(Tokens a) {
  const int w = blockIdx.x;
  const SHERRY_CONST Split& sp = as_const(a.split)[w];
  const int tokens = sp.tokens, heads = sp.heads, last = sp.last;
  // Parts in flight (with 2: 16 drafts of 5 tokens 34.6 us against 31.8, 6 prompts the same; two or
  // four rows a thread, in smaller workgroups, were no faster).
  constexpr int LANES = DP / 4, AT = 4;
  const int d = 4 * (threadIdx.x % LANES), r = (blockIdx.y * kJoinThreads + threadIdx.x) / LANES;
  const int tok = a.by_hp.div(r), hd = r - tok * a.hp;
  if (tok >= tokens || hd >= heads || d >= a.c.dim) return;
  float base = kMinusInf, l = 0.0f;
  v4f sum = {0, 0, 0, 0};
  for (int i0 = w; i0 <= last; i0 += AT) {
    float2 st[AT];
    v4f x[AT];
#pragma unroll
    for (int j = 0; j < AT; ++j) {
      const int i = i0 + j <= last ? i0 + j : i0;
      const int64_t at = int64_t(2 * i + (i == w)) * a.part_rows + r;
      st[j] = as_global(a.stat)[at];
      x[j] = *reinterpret_cast<const SHERRY_GLOBAL v4f*>(as_global(a.sums) + at * DP + d);
      if (i0 + j > last) st[j].y = 0.0f;
    }
#pragma unroll
    for (int j = 0; j < AT; ++j) {
      if (st[j].y == 0.0f) continue;  // (nothing attended to)
      const float to = fmaxf(base, st[j].x);
      const float f0 = base == kMinusInf ? 0.0f : __builtin_amdgcn_exp2f(base - to);
      const float f1 = st[j].y * __builtin_amdgcn_exp2f(st[j].x - to);
      l = l * f0 + f1;
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] = sum[e] * f0 + x[j][e] * f1;
      base = to;
    }
  }
  const int64_t at = int64_t(sp.first + tok) * a.out_stride + int64_t(sp.head0 + hd) * a.c.dim + d;
  const v4f y = sum * (l == 0.0f ? 0.0f : 1.0f / l);
  if (a.type == SHERRY_F32)
    *reinterpret_cast<SHERRY_GLOBAL v4f*>(as_global_mut(static_cast<float*>(a.out)) + at) = y;
  else
    *reinterpret_cast<SHERRY_GLOBAL u32x2*>(as_global_mut(static_cast<uint16_t*>(a.out)) + at) =
        a.type == SHERRY_BF16 ? u32x2{pair_bf16(y[0], y[1]), pair_bf16(y[2], y[3])}
                              : u32x2{pair_f16(y[0], y[1]), pair_f16(y[2], y[3])};
}

int padded_dim(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

struct Shape {
  int group, gtiles, hp, per_tile, groups, part_rows;
  size_t split_bytes, rest_bytes, stat_bytes, sum_bytes;
};
Shape shape_of(const sherry_cache_desc& c, const sherry_attend_tokens_desc& d) {
  Shape s{};
  s.group = d.heads / c.kv_heads;
  s.hp = s.group < kQRows ? s.group : kQRows;
  s.gtiles = static_cast<int>(ceil_div(s.group, s.hp));
  s.per_tile = kQRows / s.hp;
  const int dp = padded_dim(c.head_dim);
  // as many workgroups as run at once, but no more than the shortest runs of the
  // most tiles that the tokens make, each over the whole table
  const int64_t fit = kCus * waves_for(dp, d.type == SHERRY_F32 ? 2 : 1);
  const int64_t split = d.tokens / s.per_tile + c.batch;
  const double tiles = double(split < d.tokens ? split : d.tokens) * c.kv_heads * s.gtiles;
  const double rows = double(c.table_width) * c.page_size + s.per_tile + kTileCost;
  const double most = tiles * rows / kMinRun / kXcds + 1;
  s.groups = static_cast<int>(most < fit / kXcds ? static_cast<int64_t>(most) * kXcds : fit);
  const int64_t part = int64_t(d.tokens) * s.hp;
  s.part_rows = static_cast<int>(part < kQRows ? part : kQRows);
  s.split_bytes = (s.groups * sizeof(Split) + 255) / 256 * 256;
  s.rest_bytes = (s.groups * sizeof(int64_t) + 255) / 256 * 256;
  s.stat_bytes = (size_t(2) * s.groups * s.part_rows * 8 + 255) / 256 * 256;
  s.sum_bytes = size_t(2) * s.groups * s.part_rows * dp * 4;
  return s;
}
template <int DP, int NT, int NP, bool QUADS>
int launch_both(const Tokens& a, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(a.groups));
  const int rc = launch(tokens_kernel<DP, NT, NP, QUADS, false>, grid, dim3(kThreads), 0, s, a);
  return rc != SHERRY_OK ? rc : launch(tokens_kernel<DP, NT, NP, QUADS, true>, grid, dim3(kThreads), 0, s, a);
}
template <int DP, bool QUADS>
int launch_terms(const Tokens& a, hipStream_t s) {
  switch (a.type) {
    case SHERRY_F32: return launch_both<DP, 2, 2, QUADS>(a, s);
    case SHERRY_F16: return launch_both<DP, 1, 2, QUADS>(a, s);
    default: return launch_both<DP, 1, 1, QUADS>(a, s);
  }
}
template <int DP>
int launch_dim(const Tokens& a, hipStream_t s) {
  const int rc = a.c.page_size % 4 == 0 ? launch_terms<DP, true>(a, s) : launch_terms<DP, false>(a, s);
  if (rc != SHERRY_OK) return rc;
  const dim3 join(static_cast<unsigned>(a.groups), static_cast<unsigned>(ceil_div(int64_t(a.part_rows) * (DP / 4), kJoinThreads)));
  return launch(tokens_join_kernel<DP>, join, dim3(kJoinThreads), 0, s, a);
}

}  // namespace

size_t attend_tokens_workspace(const sherry_cache_desc& c, const sherry_attend_tokens_desc& d) {
  const Shape s = shape_of(c, d);
  return s.split_bytes + s.rest_bytes + s.stat_bytes + s.sum_bytes;
}

int launch_attend_tokens(const sherry_cache_desc& c, const sherry_attend_tokens_desc& d, hipStream_t s) {
  const Shape sh = shape_of(c, d);
  char* ws = static_cast<char*>(d.workspace);
  const int64_t row = int64_t(d.heads) * c.head_dim;
  char* rest = ws + sh.split_bytes;
  char* stat = rest + sh.rest_bytes;
  const Tokens a{cache_of(c), d.q, d.out, d.first, d.length, d.mask, reinterpret_cast<float2*>(stat),
                 reinterpret_cast<float*>(stat + sh.stat_bytes), reinterpret_cast<Split*>(ws),
                 reinterpret_cast<int64_t*>(rest), d.q_stride ? d.q_stride : row, d.out_stride ? d.out_stride : row,
                 d.mask_stride, d.tokens, d.heads, sh.group, sh.gtiles, sh.per_tile, sh.hp, d.type, d.window, sh.groups,
                 sh.part_rows, d.scale, FastDiv::of(static_cast<uint32_t>(sh.hp)),
                 FastDiv::of(static_cast<uint32_t>(sh.per_tile))};
  switch (padded_dim(c.head_dim)) {
    case 64: return launch_dim<64>(a, s);
    case 128: return launch_dim<128>(a, s);
    default: return launch_dim<256>(a, s);
  }
}

}  // namespace sherry
