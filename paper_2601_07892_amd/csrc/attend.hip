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
// Work mapping.  A workgroup of four waves takes one key-value head, up to 16
// of its query heads and a run of 32-row tiles; wave w takes tiles w, w + 4, ...
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
// Precision.  Cached values are exact in the operands.  q and p are split
// into terms of bf16 (or, for f16 caches, f16) whose products are summed in
// fp32: three bf16 terms hold all 24 bits, two 16; two f16 terms 22 (q is
// scaled by a power of two per head, p by 2^14, so that their low terms stay
// normal).  fp32 inputs take three and two, 16-bit inputs two.
#include "cache_internal.h"

namespace sherry {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kWaves = 4;
constexpr int kTile = 32;            // rows per wave and step
constexpr int kMinTiles = 4;         // tiles of the shortest split: one per wave
constexpr int kTargetGroups = 1024;  // workgroups that a launch is split into
constexpr int kMaxGroup = 256;       // query heads per key-value head
constexpr int kOutside = 0x7FFFFFF0;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kMinusInf = -__builtin_huge_valf();

struct Attend {
  Cache c;
  const void* q;
  void* out;
  const int32_t* length;
  const uint8_t* mask;
  const int32_t* position;
  const int32_t* q_pos;
  float* weight;
  float* sums;   // partial sums [split][y][gmax][DP]
  float2* stat;  // their maximum (of the scores in units of ln 2) and sum
  float* score;  // [batch][heads][score_stride], in units of ln 2 (weight only)
  int64_t q_stride, out_stride, mask_stride, row_stride, score_stride;
  int heads, group, gtiles, gmax, type, window, target, splits;
  float scale;
};

// ---- which rows a workgroup takes -------------------------------------------

// Rows [begin, end) of a sequence that can be attended to, and their tiles.
struct Span {
  int begin, end;
  __device__ __forceinline__ int first_tile() const { return begin / kTile; }
  __device__ __forceinline__ int tiles() const {
    return end > begin ? (end + kTile - 1) / kTile - begin / kTile : 0;
  }
};
__device__ __forceinline__ Span span_of(const Attend& a, int b) {
  const int n = a.c.length(a.length, b);
  const bool last = a.window > 0 && !a.position;
  return Span{last && n > a.window ? n - a.window : 0, n};
}

__device__ __forceinline__ int wave_sum(int v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// Tiles per split: the launch's tiles over its target of splits, so that the
// lengths, which only the device knows, decide how many a sequence gets.
__device__ __forceinline__ int split_tiles(const Attend& a) {
  const int lane = threadIdx.x & 63;
  int total = 0;
  for (int b0 = 0; b0 < a.c.batch; b0 += 64)
    total += b0 + lane < a.c.batch ? span_of(a, b0 + lane).tiles() : 0;
  total = wave_sum(total);
  const int t = (total + a.target - 1) / a.target;
  return t <= kMinTiles ? kMinTiles : (t + kWaves - 1) / kWaves * kWaves;
}

// Sequence and part of split w; b = -1: there is no such split.
struct Part {
  int b, part;
};
__device__ __forceinline__ Part find_split(const Attend& a, int t, int w) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int b0 = 0; b0 < a.c.batch; b0 += 64) {
    const int n = b0 + lane < a.c.batch ? (span_of(a, b0 + lane).tiles() + t - 1) / t : 0;
    int upto = n;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(upto, o, 64);
      if (lane >= o) upto += v;
    }
    const uint64_t past = __ballot(before + upto > w);
    if (past) {
      const int at = __builtin_ctzll(past);
      const int first = before + __shfl(upto - n, at, 64);
      return Part{__builtin_amdgcn_readfirstlane(b0 + at),
                  __builtin_amdgcn_readfirstlane(w - first)};
    }
    before += __shfl(upto, 63, 64);
  }
  return Part{-1, 0};
}
// First split of sequence b, and how many it has.
struct Run {
  int first, count;
};
__device__ __forceinline__ Run splits_of(const Attend& a, int t, int b) {
  const int lane = threadIdx.x & 63;
  int before = 0, own = 0;
  for (int b0 = 0; b0 <= b; b0 += 64) {
    const int i = b0 + lane;
    const int n = i <= b && i < a.c.batch ? (span_of(a, i).tiles() + t - 1) / t : 0;
    if (i < b) before += n;
    if (i == b) own = n;
  }
  return Run{wave_sum(before), wave_sum(own)};
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

// Two words of int8 as eight bf16 values (exact).
__device__ __forceinline__ float byte_f32(uint32_t w, int i) {
  return static_cast<float>(static_cast<int8_t>(w >> (8 * i)));
}
__device__ __forceinline__ u32x4 bytes_bf16(uint32_t w0, uint32_t w1) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = i < 2 ? w0 : w1;
    r[i] = upper(__float_as_uint(byte_f32(w, 2 * (i & 1) + 1)),
                 __float_as_uint(byte_f32(w, 2 * (i & 1))));
  }
  return r;
}

__device__ __forceinline__ float max_over_blocks(float v) {
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float sum_over_blocks(float v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

// CT: cache type; NT: terms of q and p; DP: head_dim rounded up to 64, 128 or
// 256; ANY: pages of any size (else page_size % 16 == 0, so that a half tile
// lies in one page and its rows are read through one buffer resource).
template <int CT_, int NT_, int DP_, bool ANY_>
struct Cfg {
  static constexpr int CT = CT_, NT = NT_, DP = DP_;
  static constexpr bool ANY = ANY_, F16 = CT == SHERRY_F16, I8 = CT == SHERRY_I8;
  static constexpr int E = I8 ? 1 : 2;         // bytes per value
  static constexpr int KS = DP / 32;           // MFMA steps of a score
  static constexpr int KL = DP * E / 64;       // 16-byte loads per lane and half tile of K
  static constexpr int CH = DP / 16;           // values per lane and row of V
  static constexpr int VW = CH * E / 4;        // as words
  static constexpr int VP = VW > 4 ? 2 : 1;    // pieces (of 8 values) they are read in
};

// d of value j of MFMA step s in the lanes of block g.
template <class G>
__device__ __forceinline__ int k_dim(int s, int g) {
  return G::I8 ? 64 * (s >> 1) + 16 * g + 8 * (s & 1) : 32 * s + 8 * g;
}
// d of value e of the V values of lane column n.
template <class G>
__device__ __forceinline__ int v_dim(int n, int e) {
  return G::VP == 2 ? 128 * (e >> 3) + 8 * n + (e & 7) : G::CH * n + e;
}

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
    const u32x4 v = *reinterpret_cast<const SHERRY_GLOBAL u32x4*>(as_global(p));
#pragma unroll
    for (int i = 0; i < 4; ++i) to[i] = v[i];
  } else if constexpr (W == 2) {
    const u32x2 v = *reinterpret_cast<const SHERRY_GLOBAL u32x2*>(as_global(p));
    to[0] = v[0];
    to[1] = v[1];
  } else {
    to[0] = *reinterpret_cast<const SHERRY_GLOBAL uint32_t*>(as_global(p));
  }
}

// The rows of one sequence and key-value head, tile by tile.
template <class G>
struct Rows {
  const Attend& a;
  int b, h, begin, end, qmin;  // rows with position <= qmin are left out
  // the tile that was looked up last
  uint32_t valid = 0;      // bit r: row r of the tile is attended to
  int page[2] = {0, 0};    // !ANY: page of each half
  int64_t row = 0;         // ANY: element offset of row lane % 32
  int64_t srow = 0;        // ANY: the same of its scale

  __device__ __forceinline__ void look_up(int tile) {
    const int l = threadIdx.x & 31;
    const int p0 = tile * kTile, p = p0 + l;
    bool ok = p >= begin && p < end;
    if constexpr (G::ANY) {
      const int i = a.c.by_page.div(p);
      const int pid = ok ? as_global(a.c.table)[int64_t(b) * a.c.width + i] : -1;
      ok = ok && pid >= 0 && pid < a.c.pages;
      const int off = p - i * a.c.page_size;
      row = ok ? a.c.at(pid, h) + int64_t(off) * a.c.dim : 0;
      srow = ok ? a.c.scale_at(pid, h) + off : 0;
    } else {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int ph = p0 + 16 * t;
        const int i = a.c.by_page.div(ph);
        const int pid = ph < end ? as_const(a.c.table)[int64_t(b) * a.c.width + i] : -1;
        const bool in = pid >= 0 && pid < a.c.pages;
        page[t] = in ? pid : 0;
        if ((l >> 4) == t) ok = ok && in;
      }
    }
    if (a.mask && ok) ok = as_global(a.mask)[int64_t(b) * a.mask_stride + p] != 0;
    if (a.position && a.window && ok)
      ok = as_global(a.position)[(int64_t(b) * a.c.kv + h) * a.row_stride + p] > qmin;
    valid = static_cast<uint32_t>(__ballot(ok));
  }

  __device__ __forceinline__ int half_bits(int t) const { return (valid >> (16 * t)) & 0xFFFF; }
  // Rows of a half up to its last valid one.
  __device__ __forceinline__ int half_rows(int t) const {
    const int bits = half_bits(t);
    return bits ? 32 - __builtin_clz(bits) : 0;
  }
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t half(const char* pool, int tile, int t) const {
    const int ph = tile * kTile + 16 * t;
    const int off = ph - a.c.by_page.div(ph) * a.c.page_size;
    const char* base = pool + (a.c.at(page[t], h) + int64_t(off) * a.c.dim) * G::E;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0,
                                             half_rows(t) * a.c.dim * G::E, kBufferWord3);
  }
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t half_scales(const float* pool, int tile,
                                                                int t) const {
    const int ph = tile * kTile + 16 * t;
    const int off = ph - a.c.by_page.div(ph) * a.c.page_size;
    const float* base = pool + a.c.scale_at(page[t], h) + off;
    // (whole 16-byte pieces: those of rows past the last valid one lie in the page too)
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(base), 0,
                                             ((half_rows(t) + 3) & ~3) * 4, kBufferWord3);
  }

  // K: row lane % 16 of each half, dims of block lane / 16.
  __device__ __forceinline__ void load_k(int tile, uint32_t (&k)[2][G::KL * 4]) const {
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if constexpr (G::ANY) {
        const int64_t at = __shfl(row, 16 * t + n, 64);
        const bool ok = (valid >> (16 * t + n)) & 1;
#pragma unroll
        for (int s = 0; s < G::KL; ++s) {
          const int d = (G::I8 ? 64 : 32) * s + (G::I8 ? 16 : 8) * g;
          global_words<4>(&k[t][4 * s], a.c.k + (at + d) * G::E, ok && d < a.c.dim);
        }
      } else {
        const __amdgpu_buffer_rsrc_t r = half(a.c.k, tile, t);
#pragma unroll
        for (int s = 0; s < G::KL; ++s) {
          const int d = (G::I8 ? 64 : 32) * s + (G::I8 ? 16 : 8) * g;
          buffer_words<4>(&k[t][4 * s], r, d < a.c.dim ? (n * a.c.dim + d) * G::E : kOutside);
        }
      }
    }
  }
  // V: rows 16 (j / 4) + 4 (lane / 16) + j % 4, values of column lane % 16.
  __device__ __forceinline__ void load_v(int tile, uint32_t (&v)[8][G::VW]) const {
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    constexpr int PW = G::VW / G::VP;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      __amdgpu_buffer_rsrc_t r;
      if constexpr (!G::ANY) r = half(a.c.v, tile, t);
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int c = 0; c < G::VP; ++c) {
          const int d = v_dim<G>(n, 8 * c), hr = 4 * g + j;
          uint32_t* to = &v[4 * t + j][PW * c];
          if constexpr (G::ANY) {
            const int64_t at = __shfl(row, 16 * t + hr, 64);
            const bool ok = (valid >> (16 * t + hr)) & 1;
            global_words<PW>(to, a.c.v + (at + d) * G::E, ok && d < a.c.dim);
          } else {
            buffer_words<PW>(to, r, d < a.c.dim ? (hr * a.c.dim + d) * G::E : kOutside);
          }
        }
    }
  }
  // Scales of rows 16 t + 4 (lane / 16) + 0..3.
  __device__ __forceinline__ void load_scales(const float* pool, int tile, float (&s)[8]) const {
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if constexpr (G::ANY) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int hr = 16 * t + 4 * g + j;
          const int64_t at = __shfl(srow, hr, 64);
          s[4 * t + j] = (valid >> hr) & 1 ? as_global(pool)[at] : 0.0f;
        }
      } else {
        const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(half_scales(pool, tile, t), 16 * g, 0, 0);
#pragma unroll
        for (int j = 0; j < 4; ++j) s[4 * t + j] = __uint_as_float(v[j]);
      }
    }
  }
  // Rows left out inside a half hold anything: their V values become zeros
  // (those after its last valid row were not read, and are zeros already).
  __device__ __forceinline__ bool holes(uint32_t bits) const {
    const uint32_t lo = bits & 0xFFFF, hi = bits >> 16;
    return (lo & (lo + 1)) != 0 || (hi & (hi + 1)) != 0;
  }
};

// grid: x = key-value heads x tiles of 16 query heads, y = splits
template <class G>
__global__ __launch_bounds__(64 * kWaves) void attend_kernel(Attend a) {
  constexpr int DP = G::DP, NT = G::NT;
  __shared__ float red[kWaves * 16 * (DP + 4)];
  __shared__ float2 stat[kWaves][16];
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int T = __builtin_amdgcn_readfirstlane(split_tiles(a));
  const Part w = find_split(a, T, blockIdx.y);
  if (w.b < 0) return;
  const int b = w.b;
  const int h = blockIdx.x / a.gtiles, gt = blockIdx.x - h * a.gtiles;
  const int heads = a.group - 16 * gt < 16 ? a.group - 16 * gt : 16;  // of this workgroup
  const int head0 = h * a.group + 16 * gt;
  const Span sp = span_of(a, b);
  const int begin = __builtin_amdgcn_readfirstlane(sp.begin);
  const int end = __builtin_amdgcn_readfirstlane(sp.end);
  const int t0 = begin / kTile + w.part * T;
  const int all = (end + kTile - 1) / kTile;
  const int t1 = t0 + T < all ? t0 + T : all;

  // q in terms, and the factor of its scores in units of ln 2
  u32x4 qf[NT][G::KS];
  float factor = a.scale * kLog2e;
  {
    float q[G::KS][8];
    const bool mine = n < heads;
    const int64_t at = int64_t(b) * a.q_stride + int64_t(head0 + (mine ? n : 0)) * a.c.dim;
    float top = 0.0f;
#pragma unroll
    for (int s = 0; s < G::KS; ++s) {
      const int d = k_dim<G>(s, g);
      const bool in = mine && d < a.c.dim;
      if (a.type == SHERRY_F32) {
        const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(a.q) + at + d);
        const float4 lo = in ? p[0] : make_float4(0, 0, 0, 0), hi = in ? p[1] : make_float4(0, 0, 0, 0);
        q[s][0] = lo.x, q[s][1] = lo.y, q[s][2] = lo.z, q[s][3] = lo.w;
        q[s][4] = hi.x, q[s][5] = hi.y, q[s][6] = hi.z, q[s][7] = hi.w;
      } else {
        const u32x4* p = reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.q) + at + d);
        const u32x4 v = in ? *p : u32x4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint16_t x = static_cast<uint16_t>(v[i >> 1] >> (16 * (i & 1)));
          q[s][i] = a.type == SHERRY_BF16 ? from_bf16(x) : from_f16(x);
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(q[s][i]));
    }
    if constexpr (G::F16) {
      // q / 2^e in [-2, 2): exact, and far from f16's limits
      top = max_over_blocks(top);
      const int e = (__float_as_uint(top) >> 23) & 255;
      const bool use = e > 0 && e < 254;
      const float down = use ? __uint_as_float(static_cast<uint32_t>(254 - e) << 23) : 1.0f;
      factor *= use ? __uint_as_float(static_cast<uint32_t>(e) << 23) : 1.0f;
#pragma unroll
      for (int s = 0; s < G::KS; ++s)
#pragma unroll
        for (int i = 0; i < 8; ++i) q[s][i] *= down;
    }
#pragma unroll
    for (int s = 0; s < G::KS; ++s) {
      u32x4 t[NT];
      split<G::F16, NT>(q[s], t);
#pragma unroll
      for (int i = 0; i < NT; ++i) qf[i][s] = t[i];
    }
  }

  Rows<G> rows{a, b, h, begin, end,
               a.position && a.window ? as_global(a.q_pos)[b] - a.window : 0};
  constexpr float kUp = G::F16 ? 14.0f : 0.0f;  // p is held times 2^14 in f16
  v4f o[G::CH];
#pragma unroll
  for (int e = 0; e < G::CH; ++e) o[e] = v4f{0, 0, 0, 0};
  float m = kMinusInf, l = 0.0f;

  uint32_t kr[2][G::KL * 4], vr[8][G::VW];
  float ksc[8], vsc[8];
  int tile = t0 + wave;
  if (tile < t1) {
    rows.look_up(tile);
    rows.load_k(tile, kr);
    if constexpr (G::I8) rows.load_scales(a.c.ks, tile, ksc);
    rows.load_v(tile, vr);
    if constexpr (G::I8) rows.load_scales(a.c.vs, tile, vsc);
  }
  for (; tile < t1; tile += kWaves) {
    const uint32_t valid = rows.valid;
    const int next = tile + kWaves;
    v4f s[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) s[t] = v4f{0, 0, 0, 0};
#pragma unroll
    for (int st = 0; st < G::KS; ++st)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        u32x4 kf;
        if constexpr (G::I8) {
          kf = bytes_bf16(kr[t][2 * st], kr[t][2 * st + 1]);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) kf[i] = kr[t][4 * st + i];
        }
#pragma unroll
        for (int i = NT - 1; i >= 0; --i) s[t] = mfma<G::F16>(kf, qf[i][st], s[t]);
      }
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] = s[i >> 2][i & 3] * factor;
      if constexpr (G::I8) x[i] *= ksc[i];
    }
    if (next < t1) {
      rows.look_up(next);
      rows.load_k(next, kr);
      if constexpr (G::I8) rows.load_scales(a.c.ks, next, ksc);
    }
    uint32_t mine = 0xFF;  // bit i: row of x[i] is attended to
    if (valid != 0xFFFFFFFFu) {
      mine = ((valid >> (4 * g)) & 0xF) | (((valid >> (16 + 4 * g)) & 0xF) << 4);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = (mine >> i) & 1 ? x[i] : kMinusInf;
    }
    if (a.weight && n < heads) {
      float* to = a.score + (int64_t(b) * a.heads + head0 + n) * a.score_stride + tile * kTile + 4 * g;
#pragma unroll
      for (int t = 0; t < 2; ++t)
        *reinterpret_cast<float4*>(to + 16 * t) = make_float4(x[4 * t], x[4 * t + 1], x[4 * t + 2], x[4 * t + 3]);
    }
    float top = x[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) top = fmaxf(top, x[i]);
    top = fmaxf(m, max_over_blocks(top));
    const float base = top == kMinusInf ? 0.0f : top;
    if (__any(top > m)) {
      const float down = __builtin_amdgcn_exp2f(m - base);
      l *= down;
#pragma unroll
      for (int e = 0; e < G::CH; ++e)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[e][r] *= down;
      m = top;
    }
    float p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[i] = __builtin_amdgcn_exp2f(x[i] - base + kUp);
      l += p[i];
      if constexpr (G::I8) p[i] = (mine >> i) & 1 ? p[i] * vsc[i] : 0.0f;
    }
    u32x4 pf[NT];
    split<G::F16, NT>(p, pf);
    if (!G::I8 && !G::ANY && rows.holes(valid)) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int i = 0; i < G::VW; ++i) vr[j][i] = (mine >> j) & 1 ? vr[j][i] : 0;
    }
#pragma unroll
    for (int e = 0; e < G::CH; ++e) {
      u32x4 vf;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (G::I8)
          vf[i] = upper(__float_as_uint(byte_f32(vr[2 * i + 1][e >> 2], e & 3)),
                        __float_as_uint(byte_f32(vr[2 * i][e >> 2], e & 3)));
        else
          vf[i] = e & 1 ? upper(vr[2 * i + 1][e >> 1], vr[2 * i][e >> 1])
                        : lower(vr[2 * i + 1][e >> 1], vr[2 * i][e >> 1]);
      }
#pragma unroll
      for (int i = NT - 1; i >= 0; --i) o[e] = mfma<G::F16>(vf, pf[i], o[e]);
    }
    if (next < t1) {
      rows.load_v(next, vr);
      if constexpr (G::I8) rows.load_scales(a.c.vs, next, vsc);
    }
  }

  // the four waves' sums at their common maximum
  l = sum_over_blocks(l);
  if (g == 0) stat[wave][n] = make_float2(m, l);
  __syncthreads();
  float top = kMinusInf;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) top = fmaxf(top, stat[i][n].x);
  const float down = m == kMinusInf ? 0.0f : __builtin_amdgcn_exp2f(m - top);
  if (n < heads) {
#pragma unroll
    for (int e = 0; e < G::CH; ++e)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        red[(wave * 16 + n) * (DP + 4) + v_dim<G>(4 * g + r, e)] = m == kMinusInf ? 0.0f : o[e][r] * down;
  }
  __syncthreads();
  const int64_t at = (int64_t(blockIdx.y) * gridDim.x + blockIdx.x) * a.gmax;
  for (int i = threadIdx.x; i < heads * DP; i += 64 * kWaves) {
    const int hd = i / DP, d = i % DP;
    float v = 0.0f;
#pragma unroll
    for (int j = 0; j < kWaves; ++j) v += red[(j * 16 + hd) * (DP + 4) + d];
    a.sums[(at + hd) * DP + d] = v;
  }
  if (threadIdx.x < heads) {
    const int hd = threadIdx.x;
    float mx = kMinusInf, sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) mx = fmaxf(mx, stat[i][hd].x);
#pragma unroll
    for (int i = 0; i < kWaves; ++i)
      if (stat[i][hd].x != kMinusInf) sum += stat[i][hd].y * __builtin_amdgcn_exp2f(stat[i][hd].x - mx);
    a.stat[at + hd] = make_float2(mx, sum);
  }
}

// Maximum and sum of a query head over the splits of its sequence (every lane).
__device__ __forceinline__ float2 join_stat(const Attend& a, const Run& run, int y, int hd) {
  const int lane = threadIdx.x & 63;
  const int64_t step = int64_t(a.c.kv) * a.gtiles * a.gmax;
  const float2* st = a.stat + (int64_t(run.first) * a.c.kv * a.gtiles + y) * a.gmax + hd;
  float m = kMinusInf, l = 0.0f;
  for (int i = lane; i < run.count; i += 64) {
    const float2 s = st[i * step];
    const float top = fmaxf(m, s.x);
    if (top != kMinusInf) {
      l = l * (m == kMinusInf ? 0.0f : __builtin_amdgcn_exp2f(m - top)) +
          (s.x == kMinusInf ? 0.0f : s.y * __builtin_amdgcn_exp2f(s.x - top));
      m = top;
    }
  }
  const float top = wave_max_f32(m);
  l = m == kMinusInf ? 0.0f : l * __builtin_amdgcn_exp2f(m - top);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) l += __shfl_xor(l, o, 64);
  return make_float2(top, l);
}

constexpr int kWeightRows = 1024;  // rows of weight per workgroup

// Blocks [0, batch * heads): the query heads' outputs, their splits joined;
// then, for weight, [batch][kv][rows / kWeightRows].
template <int DP, bool F16>
__global__ __launch_bounds__(256) void attend_join_kernel(Attend a) {
  __shared__ float red[4][DP];
  __shared__ float2 lse[kMaxGroup];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int T = split_tiles(a);
  int blk = blockIdx.x;
  if (blk < a.c.batch * a.heads) {
    const int b = blk / a.heads, head = blk - b * a.heads;
    const int h = head / a.group, i = head - h * a.group;
    const int y = h * a.gtiles + i / 16, hd = i % 16;
    const Run run = splits_of(a, T, b);
    const float2 st = join_stat(a, run, y, hd);
    constexpr int PER = DP / 64;
    float sum[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) sum[j] = 0.0f;
    for (int w = wave; w < run.count; w += 4) {
      const int64_t at = (int64_t(run.first + w) * a.c.kv * a.gtiles + y) * a.gmax + hd;
      const float m = a.stat[at].x;
      if (m == kMinusInf) continue;
      const float f = __builtin_amdgcn_exp2f(m - st.x);
#pragma unroll
      for (int j = 0; j < PER; ++j) sum[j] += f * a.sums[at * DP + 64 * j + lane];
    }
#pragma unroll
    for (int j = 0; j < PER; ++j) red[wave][64 * j + lane] = sum[j];
    __syncthreads();
    for (int d = threadIdx.x; d < a.c.dim; d += 256) {
      const float v = red[0][d] + red[1][d] + red[2][d] + red[3][d];
      store_from_f32(a.out, int64_t(b) * a.out_stride + int64_t(head) * a.c.dim + d, a.type,
                     st.y == 0.0f ? 0.0f : v / st.y);
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
  const Run run = splits_of(a, T, b);
  constexpr float kUp = F16 ? 16384.0f : 1.0f;  // (f16: the sums are held times 2^14)
  for (int i = wave; i < a.group; i += 4) {
    const float2 st = join_stat(a, run, h * a.gtiles + i / 16, i % 16);
    // a row's probability is 2^(x - max) / sum; nothing attended to: 0
    if (lane == 0) lse[i] = st.y == 0.0f ? make_float2(0.0f, 0.0f) : make_float2(st.x, kUp / st.y);
  }
  __syncthreads();
  for (int r = r0 + threadIdx.x; r < r1; r += 256) {
    float p = 0.0f;
    for (int i = 0; i < a.group; ++i)
      p += __builtin_amdgcn_exp2f(a.score[(int64_t(b) * a.heads + h * a.group + i) * a.score_stride + r] - lse[i].x) *
           lse[i].y;
    a.weight[(int64_t(b) * a.c.kv + h) * a.row_stride + r] += p;
  }
}

template <int CT, int NT, int DP, bool ANY>
int launch_cfg(const Attend& a, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(a.c.kv * a.gtiles), static_cast<unsigned>(a.splits));
  const int rc = launch(attend_kernel<Cfg<CT, NT, DP, ANY>>, grid, dim3(64 * kWaves), 0, s, a);
  if (rc != SHERRY_OK) return rc;
  int64_t blocks = int64_t(a.c.batch) * a.heads;
  if (a.weight) blocks += int64_t(a.c.batch) * a.c.kv * ceil_div(a.c.rows, kWeightRows);
  return launch(attend_join_kernel<DP, CT == SHERRY_F16>, dim3(static_cast<unsigned>(blocks)),
                dim3(256), 0, s, a);
}
template <int CT, int NT, int DP>
int launch_pages(const Attend& a, hipStream_t s) {
  return a.c.page_size % 16 == 0 ? launch_cfg<CT, NT, DP, false>(a, s)
                                 : launch_cfg<CT, NT, DP, true>(a, s);
}
template <int CT, int NT>
int launch_dim(const Attend& a, hipStream_t s) {
  if (a.c.dim <= 64) return launch_pages<CT, NT, 64>(a, s);
  if (a.c.dim <= 128) return launch_pages<CT, NT, 128>(a, s);
  return launch_pages<CT, NT, 256>(a, s);
}

int padded_dim(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

// The split of a launch and the parts of its workspace.
struct Shape {
  int group, gtiles, gmax, target, splits;
  int64_t score_stride;
  size_t stat_bytes, sum_bytes, score_bytes;
};
Shape shape_of(const sherry_cache_desc& c, const sherry_attend_desc& d) {
  Shape s{};
  s.group = d.heads / c.kv_heads;
  s.gtiles = static_cast<int>(ceil_div(s.group, 16));
  s.gmax = s.group < 16 ? s.group : 16;
  const int64_t y = int64_t(c.kv_heads) * s.gtiles;
  s.target = static_cast<int>(y >= kTargetGroups ? 1 : kTargetGroups / y);
  const int64_t rows = int64_t(c.table_width) * c.page_size;
  const int64_t most = int64_t(c.batch) * ceil_div(ceil_div(rows, kTile) + 1, kMinTiles);
  s.splits = static_cast<int>(most < s.target + c.batch ? most : s.target + c.batch);
  auto up = [](int64_t n) { return static_cast<size_t>((n + 255) / 256 * 256); };
  s.stat_bytes = up(s.splits * y * s.gmax * 8);
  s.sum_bytes = up(s.splits * y * s.gmax * padded_dim(c.head_dim) * 4);
  s.score_stride = ceil_div(rows, kTile) * kTile;
  s.score_bytes = d.weight ? up(int64_t(c.batch) * d.heads * s.score_stride * 4) : 0;
  return s;
}

}  // namespace

size_t attend_workspace(const sherry_cache_desc& c, const sherry_attend_desc& d) {
  const Shape s = shape_of(c, d);
  return s.stat_bytes + s.sum_bytes + s.score_bytes;
}

int launch_attend(const sherry_cache_desc& c, const sherry_attend_desc& d, hipStream_t s) {
  const Shape sh = shape_of(c, d);
  char* ws = static_cast<char*>(d.workspace);
  const int64_t row = int64_t(d.heads) * c.head_dim;
  const Attend a{cache_of(c), d.q, d.out, d.length, d.mask, d.position, d.q_pos, d.weight,
                 reinterpret_cast<float*>(ws + sh.stat_bytes), reinterpret_cast<float2*>(ws),
                 reinterpret_cast<float*>(ws + sh.stat_bytes + sh.sum_bytes),
                 d.q_stride ? d.q_stride : row, d.out_stride ? d.out_stride : row, d.mask_stride,
                 d.row_stride, sh.score_stride, d.heads, sh.group, sh.gtiles, sh.gmax, d.type,
                 d.window, sh.target, sh.splits, d.scale};
  const bool f32 = d.type == SHERRY_F32;
  switch (c.type) {
    case SHERRY_F16: return launch_dim<SHERRY_F16, 2>(a, s);
    case SHERRY_BF16: return f32 ? launch_dim<SHERRY_BF16, 3>(a, s) : launch_dim<SHERRY_BF16, 2>(a, s);
    default: return f32 ? launch_dim<SHERRY_I8, 3>(a, s) : launch_dim<SHERRY_I8, 2>(a, s);
  }
}

}  // namespace sherry
