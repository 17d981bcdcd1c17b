// Attention of one new token per sequence over a paged cache:
//
//   s_r = scale q . k_r,  p_r = exp(s_r - max) / sum exp(s - max),  out = sum_r p_r v_r
//
// in one pass over the rows with a running maximum and sum, split over the
// rows and joined; and, when asked, weight_r += sum of p_r over the query heads
// that share the key-value head.
//
// What bounds it: every cached row is read once (2 head_dim values) for 4
// head_dim operations per query head, far below what the matrix cores do in
// that time, so the cache's bytes are the floor.
//
// Work mapping.  The 32-row tiles of all sequences, one after the other, are
// cut into as many equal runs as workgroups fit the GPU; a workgroup of four
// waves takes a run for one key-value head and up to 16 of its query heads.
// The lengths are known to the device alone, so every workgroup finds its
// place from them.  A run that passes the end of a sequence goes on with the
// next one; what a workgroup finds for a sequence, unless it has all of it, is
// joined by a second launch.  Wave w takes tiles w, w + 4, ... of its run.
// Both products run on 16x16x32 MFMAs without moving anything between lanes:
//  * S^T = K Q^T: lane l holds 8 values of row l % 16 of a 16-row half tile,
//    dims of block l / 16, so a row is read with 16-byte loads as it lies; the
//    result has in lane l the scores of query head l % 16 with rows 4 (l / 16)
//    + 0..3 of the half.
//  * O^T = V^T P^T: the sum over rows may take them in any order, so the eight
//    probabilities that a lane holds are its P^T operand as they are, and the
//    rows of V that it has to pair them with, 16 (j / 4) + 4 (l / 16) + j % 4,
//    are loaded whole, 16 lanes a row; a byte permute per two values turns
//    eight rows into the V^T operands.  The sums have query head l % 16 in lane
//    l again, so the running maximum rescales them lane by lane.
//
// Precision.  Cached values are exact in the operands (rows of int8 K as they
// are, of V as f16 integers; their scales are applied to the scores and the
// probabilities).  q and p are split into terms of bf16 (or, for f16 caches and p
// over int8 V, f16) whose products are summed in fp32: three bf16 terms hold all 24
// bits, two f16 terms 22 (p is scaled by 2^14 over the largest scale of V so far, so
// that its low term stays normal).  Over bf16 caches p takes three (with
// two the outputs of bf16 q were 1e-5 off before their own rounding) and q as many
// as hold it: one of bf16, two of f16, three of fp32.  Over f16 caches both take
// two.  Over int8 K q is three int8 digits, rounded at 2^-22 of its
// head's power of two, and their products are summed as integers (two f16 terms
// against K converted to f16 took 71 us instead of 64 for 64 sequences of 4000
// rows of 64 values, 119 instead of 100 for 256, 112 instead of 110 for 128).  e4m3
// codes become f16, exactly; their pages' powers of two are applied as int8's scales are, without
// rounding, and q takes one f16 term of bf16 and f16 (all of their bits, but for those below
// 2^-24 of the head's largest value), two of fp32; p takes two.  q is scaled by that power of two
// over every cache.
//
// Measured (kernel trace; a streaming read of 2 GiB reaches 7.05 TB/s):
//  * 4 sequences of 130000 rows, 32 query heads over 8 of 128 bf16 values, 2.13
//    GB: 322 us and 5 for the join, 6.6 TB/s of the first.  94% of that read.
//  * 32 sequences of 0 to 8000 rows, 24 heads over 8 of 128 f16 values, 119 MB:
//    27 us and 4.6.  One to eight sequences of one length and the same bytes take
//    23.5, 32 of 910 rows 27: the rest is sequences that begin and end inside a run.
//  * 16 sequences of 2000 to 9000 rows, 32 heads over 8 of 128 int8 values, a
//    window, a mask and weights: 40 us and 7.2, without the three 33.  Some 10 us are
//    a workgroup's beginning and end; conversions of V, scales, masks and stored
//    scores make more than twice the vector instructions per byte of the case before.
//    64 sequences of 4000 rows, 0.54 GB, without them: 98 to 104 us, 5.2 to 5.5 TB/s.
//  * the first case's sizes in e4m3, a mask, 1.07 GB: 170 to 181 us and 4.9, 5.9 to 6.3 TB/s; without
//    a mask, 24 heads, 184 with the join (5.8 TB/s), of 64 values 99 (5.4), of 256 327 (6.5).  32
//    sequences of 0 to 8000 rows, 24 heads over 8 of 128 values, 66 MB: 21.6 and 4.6; one of 300
//    rows of 64 values 8.2.
//  * one sequence of 300 rows: 7.2 to 7.7 us in one launch, all of it latency (length, table,
//    K, V, and the waves' sums, each after the other).
#include <type_traits>

#include "cache_internal.h"

namespace sherry {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kWaves = 4;
constexpr int kMinTiles = kWaves;  // tiles of the shortest run: one per wave
// Up to this many tiles of capacity a workgroup takes a sequence whole, and
// nothing is left to join (one sequence of 300 rows of 8 heads: 64 values 7.3 us
// against 6.3 and 3.0 for the join, 128 values 11.5 against 8.6 and 3.4; of 600
// rows 14.4 against 9.0 and 3.1, so no further).
constexpr int kWholeTiles = 16;
constexpr int kCus = 256;
constexpr int kTile = 32;          // rows per wave and step
constexpr int kMaxGroup = 256;       // query heads per key-value head
constexpr int kOutside = 0x7FFFFFF0;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kMinusInf = -__builtin_huge_valf();
constexpr float kLowest = -3.40282347e38f;  // the least finite value
// p is held times 2^kUp in f16, where its low term would be subnormal, its sum is
// not.  (In the exponent, exp2(x - (max - 14)), it was lost in the rounding of max -
// 14 where that is large.)
constexpr int kUp = 14;

struct Attend {
  Cache c;
  const void* q;
  void* out;
  const int32_t* length;
  const uint8_t* mask;
  const int32_t* position;
  const int32_t* q_pos;
  float* weight;
  // what workgroup column w found for sequence b is part w + b
  int2* parts;   // [batch]: a sequence's first part and how many it has
  float2* stat;  // [part][y][gmax]: maximum (of scores in units of ln 2) and sum
  float* sums;   // [part][y][gmax][DP]
  // [batch][heads][score_stride], in units of ln 2 (weight only): -infinity of rows
  // that are left out, and of these alone (kLowest of attended ones)
  float* score;
  int64_t q_stride, out_stride, mask_stride, row_stride, score_stride;
  int heads, group, gtiles, gmax, type, window, columns;
  bool whole;    // column w is sequence w
  float scale;
};

// ---- which rows a workgroup takes -------------------------------------------

// Rows [begin, end) of a sequence that can be attended to, and their tiles.
struct Span {
  int begin, end;
  __device__ __forceinline__ int tiles() const {
    return end > begin ? (end + kTile - 1) / kTile - begin / kTile : 0;
  }
};
__device__ __forceinline__ Span span_of(const Attend& a, int b) {
  const int n = a.c.length(a.length, b);
  const bool last = a.window > 0 && !a.position;
  return Span{last && n > a.window ? n - a.window : 0, n};
}

// What a sequence costs a workgroup besides its tiles (finding it, its q, the
// first loads, the sums' way out), in tiles of a cache type and padded head size: a
// workgroup that gets many short sequences would else end the launch.  Mean time with
// 0 / 3 / 8 / 10 / 16 / 24 / 32 tiles over that with 6, of four ragged batches each (32
// sequences of 1 to 8000 rows, 48 of 400 to 4000, 16 of 1 to 30000, 64 of 10 to 1500):
//   int8  64 values 1.64 / 1.03 / 0.99 / 1.00 / 0.95 / 0.99 / 1.01
//        128        1.79 / 1.15 / 0.94 / 0.95 / 0.90 / 0.96 / 1.04
//        256        1.70 / 1.25 / 0.93 / 0.86 / 0.83 / 0.83 / 0.87
//   bf16  64        1.53 / 1.00 / 1.00 / 1.03 / 1.06 / 1.09 / 1.10
//        128        1.70 / 1.14 / 1.00 / 1.03 / 1.06 / 1.15 / 1.23
//        256        1.76 / 1.23 / 0.95 / 0.96 / 1.03 / 1.12 / 1.20
// and f16 within 0.02 of bf16.  e4m3, with 6 / 10 / 24 tiles over that with 16:
//   64 values 1.03 / 1.01 / 1.02, 128 1.04 / 1.00 / 1.02, 256 1.08 / 1.04 / 1.00.
constexpr int sequence_cost(int type, int dp) {
  return type == SHERRY_I8 || type == SHERRY_F8 ? 16 : dp == 256 ? 8 : 6;
}

// Each workgroup column takes `run` of the sequences' costs, one after the
// other; a sequence's first SEQ units (sequence_cost) are no tiles.
struct Place {
  int b, at;  // sequence, and the unit of its cost, where a column starts; b = -1: nowhere
  int run;
};
template <int SEQ>
__device__ __forceinline__ Place find_place(const Attend& a, int w) {
  const int lane = threadIdx.x & 63;
  auto cost = [&](int b) {
    const int tiles = b < a.c.batch ? span_of(a, b).tiles() : 0;
    return tiles ? tiles + SEQ : 0;
  };
  const int n0 = cost(lane), upto0 = wave_scan(n0);
  int total = __builtin_amdgcn_readlane(upto0, 63);
  for (int b = 64; b < a.c.batch; b += 64)
    total += __builtin_amdgcn_readlane(wave_scan(cost(b + lane)), 63);
  int run = static_cast<int>((static_cast<uint32_t>(total) + a.columns - 1) / a.columns);
  run = run < kMinTiles ? kMinTiles : run;
  const int64_t start = int64_t(w) * run;
  if (start >= total) return Place{-1, 0, run};
  int before = 0;
  for (int b0 = 0; b0 < a.c.batch; b0 += 64) {
    const int n = b0 == 0 ? n0 : cost(b0 + lane);
    const int upto = b0 == 0 ? upto0 : wave_scan(n);
    const uint64_t past = __ballot(before + upto > start);
    if (past) {
      const int at = __builtin_ctzll(past);
      const int first = before + __builtin_amdgcn_readlane(upto - n, at);
      return Place{b0 + at, static_cast<int>(start) - first, run};
    }
    before += __builtin_amdgcn_readlane(upto, 63);
  }
  return Place{-1, 0, run};
}
// The next sequence from b on that has tiles (batch: none).
__device__ __forceinline__ int next_sequence(const Attend& a, int b) {
  const int lane = threadIdx.x & 63;
  for (; b < a.c.batch; b += 64) {
    const uint64_t some = __ballot(b + lane < a.c.batch && span_of(a, b + lane).tiles() > 0);
    if (some) return __builtin_amdgcn_readfirstlane(b + static_cast<int>(__builtin_ctzll(some)));
  }
  return a.c.batch;
}

// ---- operands -----------------------------------------------------------------

template <bool F16>
__device__ __forceinline__ v4f mfma(const u32x4& a, const u32x4& b, const v4f& c) {
  if constexpr (F16)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a),
                                                  __builtin_bit_cast(v8h, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a),
                                                   __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
}

__device__ __forceinline__ v4i mfma_i8(const u32x4& a, const u32x4& b, const v4i& c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(v4i, a), __builtin_bit_cast(v4i, b), c, 0, 0, 0);
}

// The upper (bf16: value) halves of two words.
__device__ __forceinline__ uint32_t upper(uint32_t hi, uint32_t lo) {
  return __builtin_amdgcn_perm(hi, lo, 0x07060302u);
}
__device__ __forceinline__ uint32_t lower(uint32_t hi, uint32_t lo) {
  return __builtin_amdgcn_perm(hi, lo, 0x05040100u);
}

// Eight values as NT terms: x = t[0] + t[1] + ... up to the last term's
// rounding (bf16 terms cut off, f16 terms round).
template <bool F16, int NT>
__device__ __forceinline__ void split(const float (&x)[8], u32x4 (&t)[NT]) {
  float r[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = x[i];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      float& lo = r[2 * w];
      float& hi = r[2 * w + 1];
      if constexpr (F16) {
        const _Float16 hl = static_cast<_Float16>(lo), hh = static_cast<_Float16>(hi);
        t[n][w] = uint32_t(__builtin_bit_cast(uint16_t, hl)) |
                  uint32_t(__builtin_bit_cast(uint16_t, hh)) << 16;
        if (n + 1 < NT) {
          lo -= static_cast<float>(hl);
          hi -= static_cast<float>(hh);
        }
      } else {
        const uint32_t bl = __float_as_uint(lo), bh = __float_as_uint(hi);
        t[n][w] = upper(bh, bl);
        if (n + 1 < NT) {
          lo -= __uint_as_float(bl & 0xFFFF0000u);
          hi -= __uint_as_float(bh & 0xFFFF0000u);
        }
      }
    }
}

typedef _Float16 v2h __attribute__((ext_vector_type(2)));
// int8 V: byte i of lo and of hi, x + 128 = u with its sign bit flipped, as the f16
// values x 2^-9 (exact): u alone is the subnormal u 2^-24, and u 2^-24 * 2^15 -
// 128 * 2^-9 is one operation.
constexpr int kByteDown = 9;
template <int i>
__device__ __forceinline__ uint32_t byte_pair_f16(uint32_t hi, uint32_t lo) {
  const uint32_t pair = __builtin_amdgcn_perm(hi, lo, 0x0C000C00u | (4 + i) << 16 | i);
  const v2h v = __builtin_elementwise_fma(__builtin_bit_cast(v2h, pair), v2h{32768, 32768},
                                          v2h{(_Float16)-0.25f, (_Float16)-0.25f});
  return __builtin_bit_cast(uint32_t, v);
}

// e4m3 codes: bytes 2 i and 2 i + 1 of a word as f16 values (exact).
template <int i>
__device__ __forceinline__ uint32_t code_pair_f16(uint32_t x) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(static_cast<int>(x), 1.0f, i != 0));
}
// A page's power of two: the exponent of its scale alone, 2^-126 .. 2^127.
__device__ __forceinline__ float power_of_page(float scale) {
  const uint32_t e = __float_as_uint(scale) & 0x7F800000u;
  return __uint_as_float(e < 0x00800000u ? 0x00800000u : e < 0x7F000000u ? e : 0x7F000000u);
}

// The largest of a value in the lanes n, n + 16, n + 32, n + 48.
__device__ __forceinline__ float max_over_blocks(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ uint32_t max_over_blocks(uint32_t v) {
  const auto a = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  v = a[0] > a[1] ? a[0] : a[1];
  const auto b = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  return b[0] > b[1] ? b[0] : b[1];
}
__device__ __forceinline__ float sum_over_blocks(float v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

// Waves per SIMD, and workgroups per CU, that the registers allow without
// spilling: 96 to 128 KB of loads per CU are then in flight.  More waves, spilling,
// were slower (16 sequences of 4000 to 8000 rows of 64 values: 32 us with three,
// 39 with four; 4 of 130000 rows of 128 values: 319 with two, 360 with three), and
// so were tiles of 64 rows (34 to 43 us, 341).
__host__ __device__ constexpr int waves_for(int dp) { return dp == 64 ? 3 : dp == 128 ? 2 : 1; }

// CT: cache type; QT, NT: terms of q and of p; DP: head_dim rounded up to 64, 128 or
// 256; ANY: pages of any size (else page_size % 16 == 0, so that a half tile
// lies in one page and its rows are read through one buffer resource).
// MORE: mask, position or weight are given.
// What each buys, against the general form on the same input: pages of multiples of
// 16 rows 7.5 us against 8.4 (one sequence of 300 rows), 321 against 330 (4 of
// 130000), 61 against 68 (16 of 4000 to 8000, 256 values), 61 against 95 (64 of
// 4000, int8, 64 values); no mask, position or weight 27.1 against 28.8 (32 short
// ones), 7.5 against 8.2 (the one of 300 rows), 61 against 72 (the 64 of int8).
template <int CT_, int QT_, int NT_, int DP_, bool ANY_, bool MORE_>
struct Cfg {
  static constexpr int CT = CT_, QT = QT_, NT = NT_, DP = DP_;
  static constexpr int EU = waves_for(DP), SEQ = sequence_cost(CT, DP);
  static constexpr bool ANY = ANY_, MORE = MORE_, F16 = CT != SHERRY_BF16, I8 = CT == SHERRY_I8, F8 = CT == SHERRY_F8;
  static constexpr bool BYTES = I8 || F8;
  static constexpr int E = BYTES ? 1 : 2;      // bytes per value
  static constexpr int KS = DP / 32;           // MFMA steps of a score
  static constexpr int KL = DP * E / 64;       // 16-byte loads per lane and half tile of K
  static constexpr int CH = DP / 16;           // values per lane and row of V
  static constexpr int VW = CH * E / 4;        // as words
  static constexpr int VP = VW > 4 ? 2 : 1;    // pieces (of 8 values) they are read in
  static constexpr int QS = I8 ? KL : KS;      // MFMA steps of q's operands
  // Tiles in flight per wave: int8 rows are half as many bytes, and leave the
  // registers for two (64 sequences of 4000 rows 100 us against 110 with 128 values,
  // 59 against 64 with 64, 95 against 100 with 256; with a mask 102 against 111).  So are rows of
  // e4m3 (4 sequences of 130000 rows 99 us against 106 with 64 values, 184 against 188 with 128,
  // 328 against 340 with 256; shorter ones within 3%).
  static constexpr int DEEP = BYTES && !ANY ? 2 : 1;
};

// d of value j of MFMA step s in the lanes of block g.
template <class G>
__device__ __forceinline__ int k_dim(int s, int g) {
  return G::BYTES ? 64 * (s >> 1) + 16 * g + 8 * (s & 1) : 32 * s + 8 * g;
}
// d of value e of the V values of lane column n.
template <class G>
__device__ __forceinline__ int v_dim(int n, int e) {
  return G::VP == 2 ? 128 * (e >> 3) + 8 * n + (e & 7) : G::CH * n + e;
}

// (Loads of K and V stream: each line is used once.  Left in the caches they took
// 354 us instead of 320 for 4 sequences of 130000 rows, 29.7 instead of 27.3 for the
// 32 short ones; with pages of 20 rows 66 instead of 61.)
template <int W>
__device__ __forceinline__ void buffer_words(uint32_t* to, __amdgpu_buffer_rsrc_t r, int off) {
  if constexpr (W == 4) {
    const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, kLoadStream);
#pragma unroll
    for (int i = 0; i < 4; ++i) to[i] = v[i];
  } else if constexpr (W == 2) {
    const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, kLoadStream);
    to[0] = v[0];
    to[1] = v[1];
  } else {
    to[0] = __builtin_amdgcn_raw_buffer_load_b32(r, off, 0, kLoadStream);
  }
}
template <int W>
__device__ __forceinline__ void global_words(uint32_t* to, const char* p, bool in) {
#pragma unroll
  for (int i = 0; i < W; ++i) to[i] = 0;
  if (!in) return;
  if constexpr (W == 4) {
    const u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const SHERRY_GLOBAL u32x4*>(as_global(p)));
#pragma unroll
    for (int i = 0; i < 4; ++i) to[i] = v[i];
  } else if constexpr (W == 2) {
    const u32x2 v = __builtin_nontemporal_load(reinterpret_cast<const SHERRY_GLOBAL u32x2*>(as_global(p)));
    to[0] = v[0];
    to[1] = v[1];
  } else {
    to[0] = __builtin_nontemporal_load(reinterpret_cast<const SHERRY_GLOBAL uint32_t*>(as_global(p)));
  }
}

// The rows of one sequence and key-value head, tile by tile.
template <class G>
struct Rows {
  const Attend& a;
  int b, h, begin, end;
  const uint8_t* mask = nullptr;      // of b; NULL: not given
  const int32_t* position = nullptr;  // of b and h; NULL: no window by them
  int qmin = 0;                       // rows with position <= qmin are left out (at least INT32_MIN)
  // the tile whose look-up finished last
  uint32_t valid = 0;       // bit r: row r of the tile is attended to
  int rows[2] = {0, 0};     // !ANY: rows of each half that are read
  int64_t at[2] = {0, 0};   // !ANY: element offset of each half
  int64_t srow[2] = {0, 0}; // !ANY, bytes: offset of the half's scales
  int64_t row = 0;          // ANY: element offset of row lane % 32
  int64_t sat = 0;          // ANY, bytes: offset of its scale
  // what a look-up has read of the tile after it
  int next_page[2] = {-1, -1}, next_pos = 0;
  uint32_t next_mask = 1;
  bool next_on = true;

  __device__ __forceinline__ Rows(const Attend& args, int b_, int h_, int begin_, int end_)
      : a(args), b(b_), h(h_), begin(begin_), end(end_) {
    if constexpr (G::MORE) {
      if (a.mask) mask = a.mask + int64_t(b) * a.mask_stride;
      if (a.position && a.window) {
        position = a.position + (int64_t(b) * a.c.kv + h) * a.row_stride;
        const int64_t from = int64_t(as_const(a.q_pos)[b]) - a.window;
        qmin = static_cast<int>(from < INT32_MIN ? INT32_MIN : from);
      }
    }
  }

  __device__ __forceinline__ int64_t scale_at(int page, int off) const {
    return G::F8 ? a.c.one_scale_at(page, h) : a.c.scale_at(page, h) + off;
  }
  __device__ __forceinline__ int page_of(int tile, int t) const {
    const int ph = tile * kTile + 16 * t;
    return ph < end ? as_const(a.c.table)[int64_t(b) * a.c.width + a.c.by_page.quotient(ph)] : -1;
  }
  // Reads what decides a tile's rows; finish() uses it a tile later, when it
  // has arrived.
  __device__ __forceinline__ void start(int tile) {
    const int l = threadIdx.x & 31, p0 = tile * kTile;
    if constexpr (G::ANY) {
      const int p = p0 + l;
      const bool in = p >= begin && p < end;
      next_page[0] = in ? as_global(a.c.table)[int64_t(b) * a.c.width + a.c.by_page.div(p)] : -1;
      next_on = in;
    } else {
      next_page[0] = page_of(tile, 0);
      next_page[1] = page_of(tile, 1);
    }
    if constexpr (G::MORE) {
      // (rows past the end read zeros, and are left out by it)
      const int n = end - p0 < kTile ? end - p0 : kTile;
      if (mask)
        next_mask = __builtin_amdgcn_raw_buffer_load_b8(
            __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(mask) + p0, 0, n, kBufferWord3), l, 0, 0);
      if (position)
        next_pos = __builtin_amdgcn_raw_buffer_load_b32(
            __builtin_amdgcn_make_buffer_rsrc(const_cast<int32_t*>(position) + p0, 0, 4 * n, kBufferWord3),
            4 * l, 0, 0);
    }
  }
  // (not on: a tile of no rows)
  __device__ __forceinline__ void finish(int tile, bool on) {
    const int p0 = tile * kTile;
    bool ok = next_on;
    if constexpr (G::MORE) {
      ok = ok && next_mask != 0 && (!position || next_pos > qmin);
    }
    if constexpr (G::ANY) {
      const int p = p0 + (threadIdx.x & 31);
      const int pid = next_page[0], off = p - a.c.by_page.div(p) * a.c.page_size;
      ok = ok && pid >= 0 && pid < a.c.pages;
      row = ok ? a.c.at(pid, h) + int64_t(off) * a.c.dim : 0;
      if constexpr (G::BYTES) sat = ok ? scale_at(pid, off) : 0;
      valid = static_cast<uint32_t>(__ballot(ok));
    } else {
      // (scalar: the rows from begin to end, and of pages that exist)
      const uint32_t from = begin > p0 ? ~0u << (begin - p0) : ~0u;
      const uint32_t to = end - p0 < kTile ? (1u << (end - p0)) - 1 : ~0u;
      valid = on ? from & to : 0;
      if constexpr (G::MORE) valid &= static_cast<uint32_t>(__ballot(ok));
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int ph = p0 + 16 * t;
        const bool in = static_cast<uint32_t>(next_page[t]) < static_cast<uint32_t>(a.c.pages);
        if (!in) valid &= t ? 0xFFFFu : 0xFFFF0000u;
        const int pid = in ? next_page[t] : 0;
        const int off = ph - a.c.by_page.quotient(ph) * a.c.page_size;
        rows[t] = valid >> (16 * t) & 0xFFFFu ? (end - ph < 16 ? end - ph : 16) : 0;
        at[t] = a.c.at(pid, h) + int64_t(off) * a.c.dim;
        if constexpr (G::BYTES) srow[t] = scale_at(pid, off);
      }
    }
  }

  __device__ __forceinline__ __amdgpu_buffer_rsrc_t half(const char* pool, int t) const {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(pool) + at[t] * G::E, 0,
                                             rows[t] * a.c.dim * G::E, kBufferWord3);
  }

  // K: row lane % 16 of each half, dims of block lane / 16.
  __device__ __forceinline__ void load_k(uint32_t (&k)[2][G::KL * 4]) const {
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if constexpr (G::ANY) {
        const int64_t from = __shfl(row, 16 * t + n, 64);
        const bool ok = (valid >> (16 * t + n)) & 1;
#pragma unroll
        for (int s = 0; s < G::KL; ++s) {
          const int d = (G::BYTES ? 64 : 32) * s + (G::BYTES ? 16 : 8) * g;
          global_words<4>(&k[t][4 * s], a.c.k + (from + d) * G::E, ok && d < a.c.dim);
        }
      } else {
        const __amdgpu_buffer_rsrc_t r = half(a.c.k, t);
#pragma unroll
        for (int s = 0; s < G::KL; ++s) {
          const int d = (G::BYTES ? 64 : 32) * s + (G::BYTES ? 16 : 8) * g;
          buffer_words<4>(&k[t][4 * s], r, d < a.c.dim ? (n * a.c.dim + d) * G::E : kOutside);
        }
      }
    }
  }
  // V: rows 4 (lane / 16) + 0..3 of each half, values of column lane % 16.
  __device__ __forceinline__ void load_v(uint32_t (&v)[8][G::VW]) const {
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    constexpr int PW = G::VW / G::VP;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      __amdgpu_buffer_rsrc_t r;
      if constexpr (!G::ANY) r = half(a.c.v, t);
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int c = 0; c < G::VP; ++c) {
          const int d = v_dim<G>(n, 8 * c), hr = 4 * g + j;
          uint32_t* to = &v[4 * t + j][PW * c];
          if constexpr (G::ANY) {
            const int64_t from = __shfl(row, 16 * t + hr, 64);
            const bool ok = (valid >> (16 * t + hr)) & 1;
            global_words<PW>(to, a.c.v + (from + d) * G::E, ok && d < a.c.dim);
          } else {
            buffer_words<PW>(to, r, d < a.c.dim ? (hr * a.c.dim + d) * G::E : kOutside);
          }
        }
    }
  }
  // Scales of rows 4 (lane / 16) + 0..3 of each half.
  __device__ __forceinline__ void load_scales(const float* pool, float (&s)[8]) const {
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if constexpr (G::ANY) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int r = 16 * t + 4 * g + j;
          const int64_t from = __shfl(sat, r, 64);
          s[4 * t + j] = (valid >> r) & 1 ? as_global(pool)[from] : 0.0f;
          if constexpr (G::F8) s[4 * t + j] = power_of_page(s[4 * t + j]);
        }
      } else if constexpr (G::F8) {
        // (one of the whole half, a scalar)
        const float one = power_of_page(as_const(pool)[srow[t]]);
#pragma unroll
        for (int j = 0; j < 4; ++j) s[4 * t + j] = one;
      } else {
        // (whole 16-byte pieces: those of rows past the last one lie in the page too)
        const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<float*>(pool) + srow[t], 0, ((rows[t] + 3) & ~3) * 4, kBufferWord3);
        const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(r, 16 * g, 0, 0);
#pragma unroll
        for (int j = 0; j < 4; ++j) s[4 * t + j] = __uint_as_float(v[j]);
      }
    }
  }
  // Whether rows that were read are left out: they hold anything, and their V
  // values become zeros (rows that were not read are zeros already).
  __device__ __forceinline__ bool holes() const {
    return valid != ((1u << rows[0]) - 1 | ((1u << rows[1]) - 1) << 16);
  }
};

template <class F, int... is>
__device__ __forceinline__ void for_each(F&& f, std::integer_sequence<int, is...>) {
  (f(std::integral_constant<int, is>{}), ...);
}

// This lane's values of a sequence's q as they lie (fp32, or pairs of 16 bits).
template <class G>
__device__ __forceinline__ void load_q(const Attend& a, int b, int head0, int heads,
                                       u32x4 (&q)[G::KS][2]) {
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const bool mine = n < heads;
  const int64_t at = int64_t(b) * a.q_stride + int64_t(head0 + (mine ? n : 0)) * a.c.dim;
#pragma unroll
  for (int s = 0; s < G::KS; ++s) {
    const int d = k_dim<G>(s, g);
    const bool in = mine && d < a.c.dim;
    const u32x4 zero = {0, 0, 0, 0};
    if (a.type == SHERRY_F32) {
      const SHERRY_GLOBAL u32x4* p =
          reinterpret_cast<const SHERRY_GLOBAL u32x4*>(as_global(static_cast<const float*>(a.q)) + at + d);
      q[s][0] = in ? p[0] : zero;
      q[s][1] = in ? p[1] : zero;
    } else {
      const SHERRY_GLOBAL u32x4* p =
          reinterpret_cast<const SHERRY_GLOBAL u32x4*>(as_global(static_cast<const uint16_t*>(a.q)) + at + d);
      q[s][0] = in ? *p : zero;
      q[s][1] = zero;
    }
  }
}
// The same in terms, and the factor of its scores in units of ln 2.
template <class G>
__device__ __forceinline__ float split_q(const Attend& a, const u32x4 (&raw)[G::KS][2],
                                         u32x4 (&qf)[G::QT][G::QS]) {
  float factor = a.scale * kLog2e;
  float q[G::KS][8];
  uint32_t most = 0;  // the largest magnitude's bits (of a NaN the most)
#pragma unroll
  for (int s = 0; s < G::KS; ++s)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (a.type == SHERRY_F32) {
        q[s][i] = __uint_as_float(raw[s][i >> 2][i & 3]);
      } else {
        const uint16_t x = static_cast<uint16_t>(raw[s][0][i >> 1] >> (16 * (i & 1)));
        q[s][i] = a.type == SHERRY_BF16 ? from_bf16(x) : from_f16(x);
      }
      const uint32_t bits = __float_as_uint(q[s][i]) & 0x7FFFFFFFu;
      most = bits > most ? bits : most;
    }
  // q / 2^e in [-2, 2): exact, and far from the terms' and the scores' limits
  most = max_over_blocks(most);
  constexpr uint32_t kTiny = 0x00400000u;  // 2^-127
  const uint32_t e = most >> 23 < 254 ? most >> 23 : 254;
  const float down = __uint_as_float(e < 254 ? (254 - e) << 23 : kTiny);
  factor *= __uint_as_float(e > 0 ? e << 23 : kTiny);
#pragma unroll
  for (int s = 0; s < G::KS; ++s)
#pragma unroll
    for (int i = 0; i < 8; ++i) q[s][i] *= down;
  if constexpr (G::I8) {
    // as integers over 2^21, in three signed digits of base 256: the bytes of
    // their sum with 128 in every place, less 128
    factor *= most < 0x7F800000u ? 0x1p-21f : __uint_as_float(0x7FC00000u);  // (not finite: NaN)
#pragma unroll
    for (int s = 0; s < G::QS; ++s)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        uint32_t u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)  // rounded in the last place of a float of 2^23
          u[i] = __float_as_uint(__builtin_fmaf(q[2 * s + (w >> 1)][4 * (w & 1) + i], 0x1p21f, 0x1.8p23f)) -
                 0x4B400000u + 0x00808080u;
        // bytes 0 and 1 of each pair, then byte by byte
        const uint32_t a01 = __builtin_amdgcn_perm(u[1], u[0], 0x05010400u);
        const uint32_t a23 = __builtin_amdgcn_perm(u[3], u[2], 0x05010400u);
        const uint32_t b01 = __builtin_amdgcn_perm(u[1], u[0], 0x0C0C0602u);
        const uint32_t b23 = __builtin_amdgcn_perm(u[3], u[2], 0x0C0C0602u);
        qf[2][s][w] = lower(a23, a01) ^ 0x80808080u;
        qf[1][s][w] = upper(a23, a01) ^ 0x80808080u;
        qf[0][s][w] = lower(b23, b01) ^ 0x80808080u;
      }
  } else {
#pragma unroll
    for (int s = 0; s < G::KS; ++s) {
      u32x4 t[G::QT];
      split<G::F16, G::QT>(q[s], t);
#pragma unroll
      for (int i = 0; i < G::QT; ++i) qf[i][s] = t[i];
    }
  }
  return factor;
}

// grid: x = key-value heads x tiles of 16 query heads, y = columns
template <class G>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(G::EU))) void attend_kernel(
    Attend a) {
  constexpr int DP = G::DP, NT = G::NT;
  __shared__ float red[kWaves * 16 * (DP + 4)];
  __shared__ float2 stat[kWaves][16];
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // (uniform values, which the compiler does not see through the wave's sums)
  const Place place = a.whole ? Place{static_cast<int>(blockIdx.y), 0, 1 << 30} : find_place<G::SEQ>(a, blockIdx.y);
  const int b_first = __builtin_amdgcn_readfirstlane(place.b);
  if (b_first < 0) return;
  const int h = blockIdx.x / a.gtiles, gt = blockIdx.x - h * a.gtiles;
  const int heads = a.group - 16 * gt < 16 ? a.group - 16 * gt : 16;  // of this workgroup
  const int head0 = h * a.group + 16 * gt;
  const int run = __builtin_amdgcn_readfirstlane(place.run);
  // of the run, and of b's cost before it
  int left = run, at_cost = __builtin_amdgcn_readfirstlane(place.at);
  for (int b = b_first; b < a.c.batch;) {
    const Span sp = span_of(a, b);
    const int begin = __builtin_amdgcn_readfirstlane(sp.begin);
    const int end = __builtin_amdgcn_readfirstlane(sp.end);
    const int tiles = __builtin_amdgcn_readfirstlane(sp.tiles());
    // units [at_cost, upto) of the sequence's cost: the tiles among them
    const int upto = tiles + G::SEQ < at_cost + left ? tiles + G::SEQ : at_cost + left;
    left = a.whole ? 0 : left - (upto - at_cost);
    const int n0 = at_cost > G::SEQ ? at_cost - G::SEQ : 0, n1 = upto - G::SEQ;
    if (n1 <= n0) {  // the run ends before the first tile; or there are none
      if (a.whole)
        for (int i = threadIdx.x; i < heads * a.c.dim; i += 64 * kWaves)
          store_from_f32(a.out, int64_t(b) * a.out_stride + int64_t(head0) * a.c.dim + i, a.type, 0.0f);
      return;
    }
    const int t0 = begin / kTile + n0, t1 = begin / kTile + n1;

    // q first, then the first tile's rows, so that their latencies overlap
    u32x4 qraw[G::KS][2], qf[G::QT][G::QS];
    load_q<G>(a, b, head0, heads, qraw);
    Rows<G> rows(a, b, h, begin, end);
    float* score = nullptr;  // of this lane's head, and its rows of a tile
    if (G::MORE && a.weight)
      score = a.score + (int64_t(b) * a.heads + head0 + (n < heads ? n : 0)) * a.score_stride + 4 * g;
    v4f o[G::CH];
#pragma unroll
    for (int e = 0; e < G::CH; ++e) o[e] = v4f{0, 0, 0, 0};
    float m = kMinusInf, l = 0.0f;
    // bytes: V's scales are held over 2^ve, the largest of them so far
    int ve = kUp - 126;  // (2^(kUp - ve) is a finite factor)

    // Tile i's rows are read into slot i % D while those of the D tiles before it
    // are used.  With D > 1 every load goes out (past t1 of no rows), so that a
    // wait counts the same loads on every path.
    constexpr int D = G::DEEP;
    uint32_t kr[D][2][G::KL * 4], vr[D][8][G::VW], valids[D];
    float kscs[D][8], vscs[D][8];
    bool hole[D];
    const int mine_first = t0 + wave;
    auto inside = [&](int i) { return D == 1 || i < t1 ? i : mine_first; };
    auto start = [&](int i) {
      if (D > 1 || i < t1) rows.start(inside(i));
    };
    auto fetch_k = [&](auto slot, int i) {
      constexpr int u = decltype(slot)::value;
      rows.finish(inside(i), D == 1 || i < t1);
      valids[u] = rows.valid;
      hole[u] = !G::I8 && !G::ANY && rows.holes();
      start(i + kWaves);
      rows.load_k(kr[u]);
      if constexpr (G::BYTES) rows.load_scales(a.c.ks, kscs[u]);
    };
    auto fetch_v = [&](auto slot) {
      constexpr int u = decltype(slot)::value;
      rows.load_v(vr[u]);
      if constexpr (G::BYTES) rows.load_scales(a.c.vs, vscs[u]);
    };
    if (mine_first < t1) {
      rows.start(mine_first);
      for_each([&](auto slot) {
        fetch_k(slot, mine_first + decltype(slot)::value * kWaves);
        fetch_v(slot);
      }, std::make_integer_sequence<int, D>{});
    }
    const float factor = split_q<G>(a, qraw, qf);
    auto step = [&](auto slot, int tile) {
      constexpr int u = decltype(slot)::value;
      auto& k = kr[u];
      auto& v = vr[u];
      float(&ksc)[8] = kscs[u];
      float(&vsc)[8] = vscs[u];
      const uint32_t valid = valids[u];
      const bool holes = hole[u];
      const int next = tile + D * kWaves;
      const bool more = D > 1 || next < t1;
      float x[8];
      if constexpr (G::I8) {
        // K's bytes as they lie, a product per digit of q: exact, up to 2^22
        static_assert(G::QT == 3, "digits");
        v4i s[3][2] = {};
#pragma unroll
        for (int st = 0; st < G::QS; ++st)
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            u32x4 kf;
#pragma unroll
            for (int i = 0; i < 4; ++i) kf[i] = k[t][4 * st + i];
#pragma unroll
            for (int i = 0; i < 3; ++i) s[i][t] = mfma_i8(kf, qf[i][st], s[i][t]);
          }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          auto digit = [&](int d) { return static_cast<float>(s[d][i >> 2][i & 3]); };
          x[i] = __builtin_fmaf(__builtin_fmaf(digit(0), 256.0f, digit(1)), 256.0f, digit(2)) * (factor * ksc[i]);
        }
      } else {
        v4f s[2] = {};
#pragma unroll
        for (int st = 0; st < G::KS; ++st)
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            u32x4 kf;
            if constexpr (G::F8) {
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                kf[2 * i] = code_pair_f16<0>(k[t][2 * st + i]);
                kf[2 * i + 1] = code_pair_f16<1>(k[t][2 * st + i]);
              }
            } else {
#pragma unroll
              for (int i = 0; i < 4; ++i) kf[i] = k[t][4 * st + i];
            }
#pragma unroll
            for (int i = G::QT - 1; i >= 0; --i) s[t] = mfma<G::F16>(kf, qf[i][st], s[t]);
          }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[i] = s[i >> 2][i & 3] * factor;
          if constexpr (G::F8) x[i] *= ksc[i];  // (last: the product of the factors may pass fp32 where the score is 0)
        }
      }
      if (more) fetch_k(slot, next);
      uint32_t mine = 0xFF;  // bit i: row of x[i] is attended to
      float kept[8];         // the scores as they are stored
      if constexpr (G::MORE) {
#pragma unroll
        for (int i = 0; i < 8; ++i) kept[i] = fmaxf(x[i], kLowest);  // (of a NaN its head's sum tells)
      }
      if (valid != 0xFFFFFFFFu) {
        mine = ((valid >> (4 * g)) & 0xF) | (((valid >> (16 + 4 * g)) & 0xF) << 4);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[i] = (mine >> i) & 1 ? x[i] : kMinusInf;
          if constexpr (G::MORE) kept[i] = (mine >> i) & 1 ? kept[i] : kMinusInf;
          if constexpr (G::BYTES) vsc[i] = (mine >> i) & 1 ? vsc[i] : 0.0f;
        }
      }
      if (G::MORE && a.weight && n < heads) {
        float* to = score + tile * kTile;
#pragma unroll
        for (int t = 0; t < 2; ++t)
          *reinterpret_cast<SHERRY_GLOBAL v4f*>(as_global_mut(to) + 16 * t) =
              v4f{kept[4 * t], kept[4 * t + 1], kept[4 * t + 2], kept[4 * t + 3]};
      }
      float top = x[0];
#pragma unroll
      for (int i = 1; i < 8; ++i) top = fmaxf(top, x[i]);
      top = fmaxf(m, max_over_blocks(top));
      const float base = top == kMinusInf ? 0.0f : top;
      int vt = ve;
      if constexpr (G::BYTES) {
        float big = 0.0f;  // of the tile's V scales
#pragma unroll
        for (int i = 0; i < 8; ++i) big = fmaxf(big, fabsf(vsc[i]));
        big = max_over_blocks(big);
        const int e = static_cast<int>(__float_as_uint(big) >> 23) - 127;
        vt = e > ve ? (e < 127 ? e : 127) : ve;
      }
      if (__any(top > m || vt > ve)) {
        float down = __builtin_amdgcn_exp2f(m - base);
        l *= down;
        if constexpr (G::BYTES) down = ldexpf(down, ve - vt);
#pragma unroll
        for (int e = 0; e < G::CH; ++e)
#pragma unroll
          for (int r = 0; r < 4; ++r) o[e][r] *= down;
        m = top;
        ve = vt;
      }
      if (holes) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int i = 0; i < G::VW; ++i) v[j][i] = (mine >> j) & 1 ? v[j][i] : 0;
      }
      const float scale_p = G::BYTES ? ldexpf(1.0f, kUp - ve) : ldexpf(1.0f, kUp);
      float p[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        p[i] = __builtin_amdgcn_exp2f(x[i] - base);
        l += p[i];
        if constexpr (G::BYTES) p[i] *= vsc[i] * scale_p;
        else if constexpr (G::F16) p[i] *= scale_p;
      }
      u32x4 pf[NT];
      split<G::F16, NT>(p, pf);
      if constexpr (G::I8) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int i = 0; i < G::VW; ++i) v[j][i] ^= 0x80808080u;
      }
      auto value = [&](auto ec) {
        constexpr int e = decltype(ec)::value;
        u32x4 vf;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (G::I8)
            vf[i] = byte_pair_f16<e & 3>(v[2 * i + 1][e >> 2], v[2 * i][e >> 2]);
          else if constexpr (G::F8)  // (the permuted word serves values e and e ^ 1)
            vf[i] = code_pair_f16<e & 1>(
                __builtin_amdgcn_perm(v[2 * i + 1][e >> 2], v[2 * i][e >> 2], e & 2 ? 0x07030602u : 0x05010400u));
          else
            vf[i] = e & 1 ? upper(v[2 * i + 1][e >> 1], v[2 * i][e >> 1])
                          : lower(v[2 * i + 1][e >> 1], v[2 * i][e >> 1]);
        }
#pragma unroll
        for (int i = NT - 1; i >= 0; --i) o[e] = mfma<G::F16>(vf, pf[i], o[e]);
      };
      for_each(value, std::make_integer_sequence<int, G::CH>{});
      if (more) fetch_v(slot);
    };
    for (int tile = mine_first; tile < t1; tile += D * kWaves) {
      step(std::integral_constant<int, 0>{}, tile);
      if constexpr (D > 1) {
        if (tile + kWaves >= t1) break;
        step(std::integral_constant<int, 1>{}, tile + kWaves);
      }
    }

    // the four waves' sums at their common maximum
    l = sum_over_blocks(l);
    if (m == kMinusInf && l != l) m = 0.0f;  // scores of NaN alone, which have no maximum
    if (g == 0) stat[wave][n] = make_float2(m, l);
    __syncthreads();
    float top = kMinusInf;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) top = fmaxf(top, stat[i][n].x);
    float down = m == kMinusInf ? 0.0f : __builtin_amdgcn_exp2f(m - top);
    if constexpr (G::BYTES) down = ldexpf(down, ve + (G::I8 ? kByteDown : 0) - kUp);
    else if constexpr (G::F16) down = ldexpf(down, -kUp);
    if (n < heads) {
#pragma unroll
      for (int e = 0; e < G::CH; ++e)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          red[(wave * 16 + n) * (DP + 4) + v_dim<G>(4 * g + r, e)] = m == kMinusInf ? 0.0f : o[e][r] * down;
    }
    __syncthreads();
    const bool whole = t1 - t0 == tiles;  // nothing to join
    const int64_t at = ((int64_t(blockIdx.y) + b) * gridDim.x + blockIdx.x) * a.gmax;
    auto sum_of = [&](int hd) {
      float mx = kMinusInf, sum = 0.0f;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) mx = fmaxf(mx, stat[i][hd].x);
#pragma unroll
      for (int i = 0; i < kWaves; ++i)
        if (stat[i][hd].x != kMinusInf) sum += stat[i][hd].y * __builtin_amdgcn_exp2f(stat[i][hd].x - mx);
      return make_float2(mx, sum);
    };
    for (int i = threadIdx.x; i < heads * DP; i += 64 * kWaves) {
      const int hd = i / DP, d = i % DP;
      float v = 0.0f;
#pragma unroll
      for (int j = 0; j < kWaves; ++j) v += red[(j * 16 + hd) * (DP + 4) + d];
      if (whole) {
        const float sum = sum_of(hd).y;
        if (d < a.c.dim)
          store_from_f32(a.out, int64_t(b) * a.out_stride + int64_t(head0 + hd) * a.c.dim + d, a.type,
                         sum == 0.0f ? 0.0f : v / sum);
      } else {
        as_global_mut(a.sums)[(at + hd) * DP + d] = v;
      }
    }
    if (a.whole) return;
    if (threadIdx.x < heads) as_global_mut(a.stat)[at + threadIdx.x] = sum_of(threadIdx.x);
    if (n0 == 0 && blockIdx.x == 0 && threadIdx.x == 0) {
      // the rest of the sequence is in whole runs and a last one
      const int more = tiles - n1;
      as_global_mut(a.parts)[b] = make_int2(static_cast<int>(blockIdx.y) + b, 1 + (more + run - 1) / run);
    }
    if (left <= 0) return;
    b = __builtin_amdgcn_readfirstlane(next_sequence(a, b + 1));
    at_cost = 0;
    __syncthreads();  // (the next sequence writes stat and red again)
  }
}

// Two maxima with their sums, as one (a maximum of -infinity: nothing yet).
__device__ __forceinline__ float factor_at(float m, float top) {
  return m == kMinusInf ? 0.0f : __builtin_amdgcn_exp2f(m - top);
}

constexpr int kWeightRows = 1024;  // rows of weight per workgroup

// Blocks [0, batch * heads): the query heads' outputs, the parts of their
// sequence joined; then, for weight, [batch][kv][rows / kWeightRows].
template <int DP>
__global__ __launch_bounds__(256) void attend_join_kernel(Attend a) {
  constexpr int PER = DP / 64;
  __shared__ float red[4][DP];
  __shared__ float2 st[4];
  __shared__ float2 lse[kMaxGroup];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int blk = blockIdx.x;
  const int64_t step = int64_t(a.c.kv) * a.gtiles * a.gmax;  // from part to part, in heads
  if (blk < a.c.batch * a.heads) {
    const int b = blk / a.heads, head = blk - b * a.heads;
    const int h = head / a.group, i = head - h * a.group;
    const int hd = (h * a.gtiles + i / 16) * a.gmax + i % 16;
    const int2 parts = as_global(a.parts)[b];  // (not set for an empty sequence)
    const bool none = span_of(a, b).tiles() == 0;
    if (!none && parts.y == 1) return;  // written already
    float m = kMinusInf, l = 0.0f, sum[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) sum[j] = 0.0f;
    if (!none) {
      constexpr int AT = 4;  // parts in flight per wave
      for (int p0 = wave; p0 < parts.y; p0 += 4 * AT) {
        float2 s[AT];
        float v[AT][PER];
#pragma unroll
        for (int u = 0; u < AT; ++u) {
          const int p = p0 + 4 * u < parts.y ? p0 + 4 * u : p0;
          const int64_t at = (parts.x + p) * step + hd;
          s[u] = as_global(a.stat)[at];
          if (p0 + 4 * u >= parts.y) s[u].x = kMinusInf;
#pragma unroll
          for (int j = 0; j < PER; ++j) v[u][j] = as_global(a.sums)[at * DP + 64 * j + lane];
        }
#pragma unroll
        for (int u = 0; u < AT; ++u) {
          if (s[u].x == kMinusInf) continue;
          const float top = fmaxf(m, s[u].x), f0 = factor_at(m, top), f1 = factor_at(s[u].x, top);
          l = l * f0 + s[u].y * f1;
#pragma unroll
          for (int j = 0; j < PER; ++j) sum[j] = sum[j] * f0 + v[u][j] * f1;
          m = top;
        }
      }
    }
    if (lane == 0) st[wave] = make_float2(m, l);
    __syncthreads();
    const float top = fmaxf(fmaxf(st[0].x, st[1].x), fmaxf(st[2].x, st[3].x));
    const float f = factor_at(m, top);
#pragma unroll
    for (int j = 0; j < PER; ++j) red[wave][64 * j + lane] = m == kMinusInf ? 0.0f : sum[j] * f;
    float total = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) total += st[i].x == kMinusInf ? 0.0f : st[i].y * factor_at(st[i].x, top);
    __syncthreads();
    for (int d = threadIdx.x; d < a.c.dim; d += 256) {
      const float v = red[0][d] + red[1][d] + red[2][d] + red[3][d];
      store_from_f32(a.out, int64_t(b) * a.out_stride + int64_t(head) * a.c.dim + d, a.type,
                     total == 0.0f ? 0.0f : v / total);
    }
    return;
  }
  blk -= a.c.batch * a.heads;
  const int chunks = (a.c.rows + kWeightRows - 1) / kWeightRows;
  const int ch = blk % chunks, bh = blk / chunks;
  const int b = bh / a.c.kv, h = bh - b * a.c.kv;
  const Span sp = span_of(a, b);
  const int r0 = ch * kWeightRows > sp.begin ? ch * kWeightRows : sp.begin;
  const int r1 = (ch + 1) * kWeightRows < sp.end ? (ch + 1) * kWeightRows : sp.end;
  if (r0 >= r1) return;
  const int2 parts = as_global(a.parts)[b];
  for (int i = wave; i < a.group; i += 4) {
    const int hd = (h * a.gtiles + i / 16) * a.gmax + i % 16;
    float m = kMinusInf, l = 0.0f;
    for (int p = lane; p < parts.y; p += 64) {
      const float2 s = as_global(a.stat)[(parts.x + p) * step + hd];
      if (s.x == kMinusInf) continue;
      const float top = fmaxf(m, s.x);
      l = l * factor_at(m, top) + s.y * factor_at(s.x, top);
      m = top;
    }
    const float top = wave_max_f32(m);
    l = m == kMinusInf ? 0.0f : l * factor_at(m, top);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) l += __shfl_xor(l, o, 64);
    // a row's probability is 2^(x - max) / sum; nothing attended to: 0 (a sum
    // that is NaN makes every attended row's weight NaN)
    if (lane == 0) lse[i] = l == 0.0f ? make_float2(0.0f, 0.0f) : make_float2(top, 1.0f / l);
  }
  // four rows per thread at once
  constexpr int AT = kWeightRows / 256;
  float* to = a.weight + (int64_t(b) * a.c.kv + h) * a.row_stride;
  const float* from = a.score + (int64_t(b) * a.heads + h * a.group) * a.score_stride;
  float p[AT], w[AT];
  int r[AT];
#pragma unroll
  for (int j = 0; j < AT; ++j) {
    r[j] = ch * kWeightRows + 256 * j + threadIdx.x;
    const bool in = r[j] >= r0 && r[j] < r1;
    if (!in) r[j] = r0;
    w[j] = as_global(to)[r[j]];
    p[j] = 0.0f;
    if (!in) r[j] = -1;
  }
  __syncthreads();  // lse
#pragma unroll 4
  for (int i = 0; i < a.group; ++i)
#pragma unroll
    for (int j = 0; j < AT; ++j) {
      const float x = as_global(from)[i * a.score_stride + (r[j] < 0 ? r0 : r[j])];
      const float add = __builtin_amdgcn_exp2f(x - lse[i].x) * lse[i].y;
      p[j] += x == kMinusInf ? 0.0f : add;  // (left out)
    }
#pragma unroll
  for (int j = 0; j < AT; ++j)
    if (r[j] >= 0) as_global_mut(to)[r[j]] = w[j] + p[j];
}

// Workgroups of the joining launch.
int64_t join_groups(int64_t batch, int64_t heads, int64_t kv, int64_t rows, bool weight) {
  return batch * (heads + (weight ? kv * ceil_div(rows, kWeightRows) : 0));
}

template <class G>
int launch_cfg(const Attend& a, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(a.c.kv * a.gtiles), static_cast<unsigned>(a.columns));
  const int rc = launch(attend_kernel<G>, grid, dim3(64 * kWaves), 0, s, a);
  if (rc != SHERRY_OK || a.whole) return rc;
  const int64_t blocks = join_groups(a.c.batch, a.heads, a.c.kv, a.c.rows, a.weight != nullptr);
  return launch(attend_join_kernel<G::DP>, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, s, a);
}
template <int CT, int QT, int NT, int DP>
int launch_pages(const Attend& a, hipStream_t s) {
  const bool more = a.mask || a.position || a.weight;
  if (a.c.page_size % 16 == 0)
    return more ? launch_cfg<Cfg<CT, QT, NT, DP, false, true>>(a, s) : launch_cfg<Cfg<CT, QT, NT, DP, false, false>>(a, s);
  return more ? launch_cfg<Cfg<CT, QT, NT, DP, true, true>>(a, s) : launch_cfg<Cfg<CT, QT, NT, DP, true, false>>(a, s);
}
template <int CT, int QT, int NT>
int launch_dim(const Attend& a, hipStream_t s) {
  if (a.c.dim <= 64) return launch_pages<CT, QT, NT, 64>(a, s);
  if (a.c.dim <= 128) return launch_pages<CT, QT, NT, 128>(a, s);
  return launch_pages<CT, QT, NT, 256>(a, s);
}

int padded_dim(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

// The columns of a launch and the parts of its workspace.
struct Shape {
  int group, gtiles, gmax, columns;
  bool whole;
  int64_t score_stride;
  size_t parts_bytes, stat_bytes, sum_bytes, score_bytes;
  size_t bytes() const { return parts_bytes + stat_bytes + sum_bytes + score_bytes; }
};
Shape shape_of(const sherry_cache_desc& c, const sherry_attend_desc& d) {
  Shape s{};
  s.group = d.heads / c.kv_heads;
  s.gtiles = static_cast<int>(ceil_div(s.group, 16));
  s.gmax = s.group < 16 ? s.group : 16;
  const int dp = padded_dim(c.head_dim);
  const int64_t y = int64_t(c.kv_heads) * s.gtiles;
  const int64_t rows = int64_t(c.table_width) * c.page_size, tiles = ceil_div(rows, kTile);
  // as many workgroups as run at once, but no more than full sequences make
  const int64_t groups = kCus * waves_for(dp), fit = y >= groups ? 1 : groups / y;
  const int64_t most = ceil_div(c.batch * (tiles + sequence_cost(c.type, dp)), kMinTiles);
  s.whole = !d.weight && tiles <= kWholeTiles;
  s.columns = s.whole ? c.batch : static_cast<int>(most < fit ? most : fit);
  auto up = [](int64_t n) { return static_cast<size_t>((n + 255) / 256 * 256); };
  const int64_t parts = int64_t(s.columns) + c.batch;
  s.parts_bytes = up(int64_t(c.batch) * 8);
  s.stat_bytes = up(parts * y * s.gmax * 8);
  s.sum_bytes = up(parts * y * s.gmax * dp * 4);
  s.score_stride = tiles * kTile;
  s.score_bytes = d.weight ? up(int64_t(c.batch) * d.heads * s.score_stride * 4) : 0;
  return s;
}

}  // namespace

int64_t attend_threads(const sherry_cache_desc& c, const sherry_attend_desc& d) {
  const Shape s = shape_of(c, d);  // (the first launch: at most 2^16 workgroups in x and in y)
  const int64_t rows = int64_t(c.table_width) * c.page_size;
  return s.whole ? 0 : 256 * join_groups(c.batch, d.heads, c.kv_heads, rows, d.weight != nullptr);
}

size_t attend_workspace(const sherry_cache_desc& c, const sherry_attend_desc& d) {
  return shape_of(c, d).bytes();
}

int launch_attend(const sherry_cache_desc& c, const sherry_attend_desc& d, hipStream_t s) {
  const Shape sh = shape_of(c, d);
  char* ws = static_cast<char*>(d.workspace);
  char* stat = ws + sh.parts_bytes;
  char* sums = stat + sh.stat_bytes;
  const int64_t row = int64_t(d.heads) * c.head_dim;
  const Attend a{cache_of(c), d.q, d.out, d.length, d.mask, d.position, d.q_pos, d.weight,
                 reinterpret_cast<int2*>(ws), reinterpret_cast<float2*>(stat),
                 reinterpret_cast<float*>(sums), reinterpret_cast<float*>(sums + sh.sum_bytes),
                 d.q_stride ? d.q_stride : row, d.out_stride ? d.out_stride : row, d.mask_stride,
                 d.row_stride, sh.score_stride, d.heads, sh.group, sh.gtiles, sh.gmax, d.type,
                 d.window, sh.columns, sh.whole, d.scale};
  if (c.type == SHERRY_F16) return launch_dim<SHERRY_F16, 2, 2>(a, s);
  if (c.type == SHERRY_I8) return launch_dim<SHERRY_I8, 3, 2>(a, s);
  if (c.type == SHERRY_F8) return d.type == SHERRY_F32 ? launch_dim<SHERRY_F8, 2, 2>(a, s) : launch_dim<SHERRY_F8, 1, 2>(a, s);
  switch (d.type) {
    case SHERRY_F32: return launch_dim<SHERRY_BF16, 3, 3>(a, s);
    case SHERRY_F16: return launch_dim<SHERRY_BF16, 2, 3>(a, s);
    default: return launch_dim<SHERRY_BF16, 1, 3>(a, s);
  }
}

}  // namespace sherry
