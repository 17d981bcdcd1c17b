// New tokens of a ragged batch into a paged cache of e4m3 codes with a power of two
// per page and head, and their rotary positions.
//
//   need = 2^e, the smallest e >= -100 with |y| <= 448 * 2^e for every finite new y
//   power = need for a page that holds nothing yet, else max(need, old)
//   code = e4m3(y / power); when power rises, the page's other codes = e4m3(code * old / power)
//
// A power of two keeps every step exact but the rounding to e4m3 itself: y / power
// only moves the exponent, a code that is rounded again loses at most the lowest bits
// of values near the subnormals, and a reader multiplies without rounding.
//
// What bounds it: the bytes of the tokens' q, k and v rows, read once, of q_out
// and the codes, written once; a decode batch costs a launch and the chain of
// dependent reads before its stores (lengths, table, rows and old power).
//
// Work mapping.  A page's power needs the largest new value of all of its rows, so
// one owner takes all new rows of a page and head, of K or of V: a wave, or, where
// that is much more than its registers hold, the four waves of a workgroup.  The rows stay
// in registers from the maximum to the stores (those past kKeep pieces a lane are read
// again, out of the caches).  Which page is a matter of the lengths, which the device alone
// knows: every workgroup finds its own by a scan over the sequences.  Further
// workgroups rotate q, some heads of one or several tokens each.
//
// Measured: 32 tokens of 32 sequences, 24 + 16 heads of 128 values, fp32 4.4 us, all of it a
// launch and its chain of reads; 8 prompts of 37 to 2048 tokens, 32 + 16 heads of 64 bf16
// values, 60 MB 20.5 us, 2.9 TB/s.
#include "rotary.h"

namespace sherry {
namespace {

constexpr int kKeep = 8;       // pieces of four values a lane that stay in registers
constexpr int kQGroups = 1024, kMostQ = 16;  // workgroups for q before they take several tokens; the most
constexpr int kLeast = -100;   // the smallest exponent that extend gives

struct Extend {
  Cache c;
  const void* q;
  const void* k;
  const void* v;
  void* q_out;
  const int32_t* first;
  const int32_t* length;
  const int32_t* pos;
  Rotary rope;
  int64_t q_stride, k_stride, v_stride, q_out_stride;
  int tokens, heads, units;   // units: most pages that the tokens reach
  int per_q;                  // tokens of a workgroup that turns q
  int both;                   // its lanes have both values of a pair
  FastDiv by_parts, by_qparts;  // workgroups per page, and per per_q tokens for q
};

// A sequence's tokens [t0, t0 + n) and its rows before them.
struct Tokens {
  int t0, n, len;
};
__device__ __forceinline__ Tokens tokens_of(const Extend& a, int b) {
  const int f0 = as_global(a.first)[b], f1 = as_global(a.first)[b + 1];
  const int t0 = f0 < 0 ? 0 : f0 < a.tokens ? f0 : a.tokens;
  const int t1 = f1 < t0 ? t0 : f1 < a.tokens ? f1 : a.tokens;
  const int len = a.c.length(a.length, b);
  const int room = a.c.rows - len;
  return Tokens{t0, t1 - t0 < room ? t1 - t0 : room, len};
}
__device__ __forceinline__ int pages_of(const Extend& a, const Tokens& t) {
  return t.n > 0 ? static_cast<int>(a.c.by_page.div(t.len + t.n - 1) - a.c.by_page.div(t.len)) + 1 : 0;
}

// Sequence and page (of its table) that the u-th reached page is; b = -1: there are fewer.
struct Unit {
  int b, j;
  Tokens t;
};
__device__ __forceinline__ Unit find_unit(const Extend& a, int u) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int b0 = 0; b0 < a.c.batch; b0 += 64) {
    const Tokens t = b0 + lane < a.c.batch ? tokens_of(a, b0 + lane) : Tokens{0, 0, 0};
    const int n = pages_of(a, t), upto = wave_scan(n);
    const uint64_t past = __ballot(before + upto > u);
    if (past) {
      const int at = __builtin_ctzll(past);
      const int own = u - before - (__builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(n, at));
      const Tokens mine{__builtin_amdgcn_readlane(t.t0, at), __builtin_amdgcn_readlane(t.n, at),
                        __builtin_amdgcn_readlane(t.len, at)};
      return Unit{b0 + at, static_cast<int>(a.c.by_page.div(mine.len)) + own, mine};
    }
    before += __builtin_amdgcn_readlane(upto, 63);
  }
  return Unit{-1, 0, {0, 0, 0}};
}
// The last sequence that begins at or before token t, by 64 probes a step (-1: none).
__device__ __forceinline__ int find_sequence(const Extend& a, int t) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = a.c.batch;
  for (;;) {
    const int step = (n + 63) / 64, at = lane * step;
    const int k = __builtin_popcountll(__ballot(at < n && as_global(a.first)[lo + (at < n ? at : 0)] <= t));
    if (k == 0) return -1;
    lo += (k - 1) * step;
    n = step < n - (k - 1) * step ? step : n - (k - 1) * step;
    if (step == 1) return lo;
  }
}

// Exponent (biased by 127) of the smallest power of two >= 2^kLeast with top <= 448 of it.
__device__ __forceinline__ int power_of(float top) {
  const uint32_t u = __float_as_uint(top);  // 448 = 1.75 * 2^8
  const int e = static_cast<int>(u >> 23) - 8 + ((u & 0x7FFFFFu) > 0x600000u);
  return e > 127 + kLeast ? e : 127 + kLeast;
}
__device__ __forceinline__ float power(int biased) { return __uint_as_float(uint32_t(biased) << 23); }
// Its reciprocal (2^-127, of the largest, is a subnormal number).
__device__ __forceinline__ float over_power(int biased) {
  return __uint_as_float(biased < 254 ? uint32_t(254 - biased) << 23 : 0x00400000u);
}

__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true));
}
__device__ __forceinline__ uint32_t requantized(uint32_t x, float ratio) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(x), false);
  const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(x), true);
  return codes4(lo[0] * ratio, lo[1] * ratio, hi[0] * ratio, hi[1] * ratio);
}

// WPP: waves per page, head and K or V.
template <int LPR, int WPP, int TYPE, bool VEC>
__device__ __forceinline__ void store_pages(const Extend& a, int blk) {
  constexpr int RPW = 64 / LPR, STEP = RPW * WPP;  // rows per wave and iteration, and of all waves
  __shared__ int most[4];
  const int u = a.by_parts.div(blk), part = blk - u * a.by_parts.d;
  const Unit unit = find_unit(a, u);
  const int b = __builtin_amdgcn_readfirstlane(unit.b);
  if (b < 0) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int j = __builtin_amdgcn_readfirstlane(unit.j), p0 = j * a.c.page_size;
  const int page = as_const(a.c.table)[int64_t(b) * a.c.width + j];
  if (page < 0 || page >= a.c.pages) return;
  const Tokens& t = unit.t;
  const int r0 = t.len > p0 ? t.len : p0;
  const int r1 = t.len + t.n - p0 < a.c.page_size ? t.len + t.n : p0 + a.c.page_size;
  const int pair = part * (4 / WPP) + (WPP == 1 ? wave : 0);
  if (pair >= 2 * a.c.kv) return;  // (with several waves a pair: the whole workgroup)
  const bool is_k = pair < a.c.kv;
  const int h = is_k ? pair : pair - a.c.kv;
  const int mine = WPP == 1 ? 0 : wave;  // of the waves of a pair
  const int d = 4 * (lane % LPR);
  const bool in = d < a.c.dim;

  auto position = [&](int row) { return a.pos ? as_global(a.pos)[t.t0 + row - t.len] : row; };
  auto value = [&](int row, float4& x) {
    const int tok = t.t0 + row - t.len, pos = position(row);
    if (!in || !a.rope.has(pos)) return false;
    x = is_k ? rotated<TYPE, VEC>(a.rope, a.k, int64_t(tok) * a.k_stride + h * a.c.dim, d, pos)
             : load4<TYPE, VEC>(a.v, int64_t(tok) * a.v_stride + h * a.c.dim + d);
    return true;
  };
  float top = 0.0f;
  auto see = [&](const float4& x) {
    auto one = [&](float v) { top = fmaxf(top, fabsf(v) < __builtin_huge_valf() ? fabsf(v) : 0.0f); };
    one(x.x), one(x.y), one(x.z), one(x.w);
  };
  // (a page that holds rows already: the power that they have)
  float* scale = (is_k ? a.c.ks : a.c.vs) + a.c.one_scale_at(page, h);
  const bool fresh = p0 >= t.len;
  int old = 0;
  if (!fresh) {
    old = static_cast<int>(__float_as_uint(as_global(scale)[0]) >> 23) & 0xFF;
    old = old < 1 ? 1 : old < 254 ? old : 254;
  }
  float4 kept[kKeep];
  uint32_t there = 0;
  bool some = false;  // rows past the kept ones are stored
  const int from = r0 + mine * RPW + lane / LPR;
#pragma unroll
  for (int i = 0; i < kKeep; ++i) {
    kept[i] = make_float4(0, 0, 0, 0);
    if (from + i * STEP < r1 && value(from + i * STEP, kept[i])) there |= 1u << i;
  }
#pragma unroll
  for (int i = 0; i < kKeep; ++i) see(kept[i]);
  for (int row = from + kKeep * STEP; row < r1; row += STEP) {
    float4 x = make_float4(0, 0, 0, 0);
    if (value(row, x)) some = true;
    see(x);
  }
  top = wave_max_f32(top);
  int now = 0;  // (none of these rows is stored)
  if (__any(there != 0 || some)) {
    now = power_of(top);
    now = now > old ? now : old;
  }
  if constexpr (WPP > 1) {
    if (lane == 0) most[wave] = now;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) now = now > most[i] ? now : most[i];
  }
  now = __builtin_amdgcn_readfirstlane(now);
  if (now == 0) return;  // (every token of the page is left out, and so is the page)

  char* rows = (is_k ? a.c.k : a.c.v) + a.c.at(page, h);
  auto store = [&](int row, const float4& x) {
    auto one = [&](float v) {
      return fabsf(v) < __builtin_huge_valf() ? v * over_power(now) : __uint_as_float(0x7FC00000u);
    };
    *reinterpret_cast<SHERRY_GLOBAL uint32_t*>(as_global_mut(rows) + int64_t(row - p0) * a.c.dim + d) =
        codes4(one(x.x), one(x.y), one(x.z), one(x.w));
  };
#pragma unroll
  for (int i = 0; i < kKeep; ++i)
    if ((there >> i) & 1) store(from + i * STEP, kept[i]);
  for (int row = from + kKeep * STEP; row < r1; row += STEP) {
    float4 x;
    if (value(row, x)) store(row, x);
  }
  if (!fresh && now > old) {
    // (a ratio below 2^-126 leaves nothing of any code)
    const float ratio = power(127 - (now - old < 126 ? now - old : 126));
    const int pieces = a.c.dim / 16;
    const int64_t before = int64_t(r0 - p0) * pieces, gap = int64_t(r1 - r0) * pieces;
    const int64_t all = int64_t(a.c.page_size) * pieces - gap;
    for (int64_t i = mine * 64 + lane; i < all; i += 64 * WPP) {
      SHERRY_GLOBAL u32x4* at = reinterpret_cast<SHERRY_GLOBAL u32x4*>(as_global_mut(rows)) + (i < before ? i : i + gap);
      u32x4 x = *at;
#pragma unroll
      for (int w = 0; w < 4; ++w) x[w] = requantized(x[w], ratio);
      *at = x;
    }
    for (int row = from; row < r1; row += STEP) {  // rows of tokens that are left out
      if (!in || a.rope.has(position(row))) continue;
      SHERRY_GLOBAL uint32_t* at = reinterpret_cast<SHERRY_GLOBAL uint32_t*>(as_global_mut(rows) + int64_t(row - p0) * a.c.dim + d);
      *at = requantized(*at, ratio);
    }
  }
  if (mine == 0 && lane == 0) as_global_mut(scale)[0] = power(now);
}

// per_q tokens one after the other, some of their heads.  With `both`, a lane has the four
// values d and their four partners (or, behind the rotated values, eight): x and the angles are
// read once for the two (8 prompts of 37 to 2048 tokens, 32 heads of 64 bf16 values: 22.6 us
// against 25.8; with the reads of four tokens together 21.0).
template <int LPR, int TYPE, bool VEC>
__device__ __forceinline__ void turn_q(const Extend& a, int blk) {
  const bool both = VEC && a.both;
  const int group = a.by_qparts.div(blk), part = blk - group * a.by_qparts.d;
  const int t0 = group * a.per_q, t1 = t0 + a.per_q < a.tokens ? t0 + a.per_q : a.tokens;
  const int lanes = both ? LPR / 2 : LPR;
  const int r = part * (256 / lanes) + threadIdx.x / lanes, i = threadIdx.x % lanes;
  const int half = a.rope.cos ? a.rope.rot >> 1 : 0;
  const bool turned = 4 * i < half;
  const int d = !both ? 4 * i : turned ? 4 * i : 2 * half + 8 * (i - half / 4), e = turned ? d + half : d + 4;
  const bool in = r < a.heads && d < a.c.dim;
  int b = __builtin_amdgcn_readfirstlane(find_sequence(a, t0));
  b = b < 0 ? 0 : b;
  Tokens s = tokens_of(a, b);
  for (int t4 = t0; t4 < t1; t4 += 4) {
    // (all reads of four tokens before the first is used; of those left out too)
    int pos[4];
    bool ok[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int t = t4 + j < t1 ? t4 + j : t1 - 1;
      while (b + 1 < a.c.batch && as_const(a.first)[b + 1] <= t) s = tokens_of(a, ++b);
      const bool here = t >= s.t0 && t - s.t0 < s.n;
      const int row = here ? s.len + (t - s.t0) : 0;
      const int page = as_const(a.c.table)[int64_t(b) * a.c.width + a.c.by_page.div(row)];
      pos[j] = a.pos ? as_const(a.pos)[t] : row;
      ok[j] = here && page >= 0 && page < a.c.pages && a.rope.has(pos[j]) && t4 + j < t1;
      pos[j] = ok[j] ? pos[j] : 0;
    }
    if (!in) continue;
    if (!both) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (ok[j])
          store4<TYPE, VEC>(a.q_out, int64_t(t4 + j) * a.q_out_stride + r * a.c.dim + d,
                            rotated<TYPE, VEC>(a.rope, a.q, int64_t(t4 + j) * a.q_stride + r * a.c.dim, d, pos[j]));
      continue;
    }
    float4 x[4], y[4], c[4], n[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t from = int64_t(t4 + j < t1 ? t4 + j : t1 - 1) * a.q_stride + r * a.c.dim;
      x[j] = load4<TYPE, VEC>(a.q, from + d);
      y[j] = load4<TYPE, VEC>(a.q, from + e);
      if (turned) {
        c[j] = *reinterpret_cast<const SHERRY_GLOBAL float4*>(as_global(a.rope.cos) + int64_t(pos[j]) * half + d);
        n[j] = *reinterpret_cast<const SHERRY_GLOBAL float4*>(as_global(a.rope.sin) + int64_t(pos[j]) * half + d);
      } else {
        c[j] = n[j] = make_float4(0, 0, 0, 0);  // (not used)
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (!ok[j]) continue;
      const int64_t to = int64_t(t4 + j) * a.q_out_stride + r * a.c.dim;
      float4 u = x[j], v = y[j];
      if (turned) {
        u = make_float4(u.x * c[j].x - v.x * n[j].x, u.y * c[j].y - v.y * n[j].y, u.z * c[j].z - v.z * n[j].z,
                        u.w * c[j].w - v.w * n[j].w);
        v = make_float4(v.x * c[j].x + x[j].x * n[j].x, v.y * c[j].y + x[j].y * n[j].y, v.z * c[j].z + x[j].z * n[j].z,
                        v.w * c[j].w + x[j].w * n[j].w);
      }
      store4<TYPE, VEC>(a.q_out, to + d, u);
      store4<TYPE, VEC>(a.q_out, to + e, v);
    }
  }
}

// Blocks [0, units * by_parts.d): pages; then [tokens / per_q][by_qparts.d]: q.
template <int LPR, int WPP, int TYPE, bool VEC>
__global__ __launch_bounds__(256) void extend_kernel(Extend a) {
  const int pages = a.units * static_cast<int>(a.by_parts.d);
  if (static_cast<int>(blockIdx.x) < pages) store_pages<LPR, WPP, TYPE, VEC>(a, blockIdx.x);
  else turn_q<LPR, TYPE, VEC>(a, blockIdx.x - pages);
}

struct Grid {
  int units;
  int per_q;              // tokens of a workgroup that turns q
  int64_t parts, qparts;  // workgroups per page, and per per_q tokens for q
  bool wide;              // four waves per page, head and K or V
  bool vec, both;
  int64_t blocks(int64_t tokens) const { return units * parts + ceil_div(tokens, per_q) * qparts; }
};
Grid grid_of(const sherry_cache_desc& c, const sherry_extend_desc& d) {
  Grid g{};
  const int lanes = lanes_per_row(c.head_dim);
  const int64_t batch = c.batch < d.tokens ? c.batch : d.tokens;
  const int64_t units = d.tokens / c.page_size + 2 * batch;  // n tokens reach n / page_size + 2 pages at most
  g.units = static_cast<int>(units < d.tokens ? units : d.tokens);
  // new rows of a page if the sequences have equally many
  const int64_t new_rows = ceil_div(d.tokens, c.batch) < c.page_size ? ceil_div(d.tokens, c.batch) : c.page_size;
  // (One wave / four for 8 x 1024 tokens of 8 heads, bf16, in us: 64 values with pages of 32 rows
  // 11.2 / 20.2, of 64 16.8 / 14.3; 128 values with 16 18.7 / 35.4, with 32 20.4 / 24.5, with 64
  // 35.1 / 18.8; 256 values with 16 37.9 / 42.5, with 32 40.9 / 36.7.)
  g.wide = new_rows > 32 || new_rows * lanes > 2 * 64 * kKeep;
  g.parts = g.wide ? 2 * c.kv_heads : ceil_div(2 * c.kv_heads, 4);
  const int64_t qrow = int64_t(d.heads) * c.head_dim, row = int64_t(c.kv_heads) * c.head_dim;
  auto whole = [&](const void* p, int64_t stride, int64_t least) { return whole_pieces(p, stride ? stride : least, d.type); };
  g.vec = whole(d.k, d.k_stride, row) && whole(d.v, d.v_stride, row) &&
          (!d.q || (whole(d.q, d.q_stride, qrow) && whole(d.q_out, d.q_out_stride, qrow))) &&
          reinterpret_cast<uintptr_t>(d.cos) % 16 == 0 && reinterpret_cast<uintptr_t>(d.sin) % 16 == 0;
  g.both = g.vec && (!d.cos || (d.pairing == SHERRY_ROPE_HALVES && d.rot_dim % 8 == 0));
  g.qparts = d.q ? ceil_div(d.heads, 256 / (g.both ? lanes / 2 : lanes)) : 0;
  // A workgroup finds its token's place by reads that wait for each other; past what runs at
  // once it takes several tokens, whose places follow from the first one's (8 prompts of 37 to
  // 2048 tokens, 32 heads of 64: 21.0 us against 29.4 with one each).
  const int64_t per = d.tokens * g.qparts / kQGroups;
  g.per_q = static_cast<int>(per < 1 ? 1 : per < kMostQ ? per : kMostQ);
  return g;
}

template <int LPR, int TYPE, bool VEC>
int launch_wide(const Extend& a, const Grid& g, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(g.blocks(a.tokens)));
  return g.wide ? launch(extend_kernel<LPR, 4, TYPE, VEC>, grid, dim3(256), 0, s, a)
                : launch(extend_kernel<LPR, 1, TYPE, VEC>, grid, dim3(256), 0, s, a);
}
template <int LPR>
int launch_type(const Extend& a, int type, bool vec, const Grid& g, hipStream_t s) {
  switch (type) {
    case SHERRY_F32:
      return vec ? launch_wide<LPR, SHERRY_F32, true>(a, g, s) : launch_wide<LPR, SHERRY_F32, false>(a, g, s);
    case SHERRY_F16:
      return vec ? launch_wide<LPR, SHERRY_F16, true>(a, g, s) : launch_wide<LPR, SHERRY_F16, false>(a, g, s);
    default:
      return vec ? launch_wide<LPR, SHERRY_BF16, true>(a, g, s) : launch_wide<LPR, SHERRY_BF16, false>(a, g, s);
  }
}

}  // namespace

int64_t extend_threads(const sherry_cache_desc& c, const sherry_extend_desc& d) {
  return 256 * grid_of(c, d).blocks(d.tokens);
}

int launch_extend(const sherry_cache_desc& c, const sherry_extend_desc& d, hipStream_t s) {
  const Grid g = grid_of(c, d);
  const int heads = d.q ? d.heads : 0;
  const int64_t qrow = int64_t(heads) * c.head_dim, row = int64_t(c.kv_heads) * c.head_dim;
  const Extend a{cache_of(c), d.q, d.k, d.v, d.q_out, d.first, d.length, d.pos,
                 Rotary{d.cos, d.sin, d.rope_rows, d.rot_dim, d.pairing == SHERRY_ROPE_PAIRS},
                 d.q_stride ? d.q_stride : qrow, d.k_stride ? d.k_stride : row, d.v_stride ? d.v_stride : row,
                 d.q_out_stride ? d.q_out_stride : qrow, d.tokens, heads, g.units, g.per_q, g.both,
                 FastDiv::of(static_cast<uint32_t>(g.parts)),
                 FastDiv::of(static_cast<uint32_t>(g.qparts ? g.qparts : 1))};
  switch (lanes_per_row(c.head_dim)) {
    case 16: return launch_type<16>(a, d.type, g.vec, g, s);
    case 32: return launch_type<32>(a, d.type, g.vec, g, s);
    default: return launch_type<64>(a, d.type, g.vec, g, s);
  }
}

}  // namespace sherry
