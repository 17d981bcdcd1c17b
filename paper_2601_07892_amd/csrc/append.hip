// New tokens into a paged cache: rotary positions on q and k, then k and v
// stored as bf16, f16, or int8 with one scale per row.
//
//   y_a = a c - b s,  y_b = b c + a s  in fp32, each operation rounded
//
// What bounds it: the bytes of the tokens' q, k and v rows, read and written
// once; a decode batch's few hundred rows cost one launch.  A row takes
// DP / 4 lanes of four values, so that its absolute maximum (int8) is a
// reduction inside a wave, and its rotation partner is read from the row
// again, out of the caches.
#include "cache_internal.h"

namespace sherry {
namespace {

struct Append {
  Cache c;
  const void* q;
  const void* k;
  const void* v;
  void* q_out;
  const int32_t* seq;
  const int32_t* slot;
  const int32_t* pos;
  const float* cos;
  const float* sin;
  float* weight;
  int32_t* position;
  int64_t row_stride, q_stride, k_stride, v_stride, q_out_stride;
  int tokens, heads, type, cache_type, rope_rows, rot, pairs;
};

template <bool VEC>
__device__ __forceinline__ float4 load4(const void* p, int64_t i, int type) {
  if constexpr (VEC) {
    if (type == SHERRY_F32)
      return *reinterpret_cast<const SHERRY_GLOBAL float4*>(as_global(static_cast<const float*>(p)) + i);
    typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
    const u16x4 h = *reinterpret_cast<const SHERRY_GLOBAL u16x4*>(as_global(static_cast<const uint16_t*>(p)) + i);
    return type == SHERRY_BF16
               ? make_float4(from_bf16(h[0]), from_bf16(h[1]), from_bf16(h[2]), from_bf16(h[3]))
               : make_float4(from_f16(h[0]), from_f16(h[1]), from_f16(h[2]), from_f16(h[3]));
  } else {
    return make_float4(load_as_f32(p, i, type), load_as_f32(p, i + 1, type),
                       load_as_f32(p, i + 2, type), load_as_f32(p, i + 3, type));
  }
}

// Values d .. d + 3 of a row at element `at`, rotated.
template <bool VEC>
__device__ __forceinline__ float4 rotated(const Append& a, const void* p, int64_t at, int d, int pos) {
  const float4 x = load4<VEC>(p, at + d, a.type);
  if (!a.cos || d >= a.rot) return x;
  const int half = a.rot >> 1;
  const float* cs = a.cos + int64_t(pos) * half;
  const float* sn = a.sin + int64_t(pos) * half;
  if (VEC && !a.pairs && half % 4 == 0) {
    // the four partners are together
    const int i = d < half ? d : d - half;
    const float4 w = load4<VEC>(p, at + (d < half ? d + half : i), a.type);
    const float4 c = *reinterpret_cast<const SHERRY_GLOBAL float4*>(as_global(cs) + i);
    const float4 s = *reinterpret_cast<const SHERRY_GLOBAL float4*>(as_global(sn) + i);
    return d < half ? make_float4(x.x * c.x - w.x * s.x, x.y * c.y - w.y * s.y, x.z * c.z - w.z * s.z,
                                  x.w * c.w - w.w * s.w)
                    : make_float4(x.x * c.x + w.x * s.x, x.y * c.y + w.y * s.y, x.z * c.z + w.z * s.z,
                                  x.w * c.w + w.w * s.w);
  }
  float r[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int j = d + e;
    if (j >= a.rot) break;
    const bool first = a.pairs ? (j & 1) == 0 : j < half;
    const int i = a.pairs ? j >> 1 : first ? j : j - half;
    const int other = a.pairs ? j ^ 1 : first ? j + half : i;
    const float w = load_as_f32(p, at + other, a.type) * as_global(sn)[i];
    const float v = r[e] * as_global(cs)[i];
    r[e] = first ? v - w : v + w;
  }
  return make_float4(r[0], r[1], r[2], r[3]);
}

template <bool VEC>
__device__ __forceinline__ void store4(void* p, int64_t i, int type, float4 v) {
  if (VEC && type == SHERRY_F32) {
    *reinterpret_cast<SHERRY_GLOBAL float4*>(as_global_mut(static_cast<float*>(p)) + i) = v;
  } else if (VEC) {
    typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
    const u16x4 h = type == SHERRY_BF16 ? u16x4{to_bf16(v.x), to_bf16(v.y), to_bf16(v.z), to_bf16(v.w)}
                                        : u16x4{to_f16(v.x), to_f16(v.y), to_f16(v.z), to_f16(v.w)};
    *reinterpret_cast<SHERRY_GLOBAL u16x4*>(as_global_mut(static_cast<uint16_t*>(p)) + i) = h;
  } else {
    store_from_f32(p, i, type, v.x);
    store_from_f32(p, i + 1, type, v.y);
    store_from_f32(p, i + 2, type, v.z);
    store_from_f32(p, i + 3, type, v.w);
  }
}

// One row (a head of q, k or v of one token) per LPR lanes.
template <int LPR, bool VEC>
__global__ __launch_bounds__(256) void append_kernel(Append a) {
  constexpr int RPB = 256 / LPR;
  const int per = a.heads + 2 * a.c.kv;  // rows of a token: q, k, v heads
  const int64_t row = int64_t(blockIdx.x) * RPB + threadIdx.x / LPR;
  const int d = 4 * (threadIdx.x % LPR);
  if (row >= int64_t(a.tokens) * per) return;
  const int t = static_cast<int>(row / per), r = static_cast<int>(row - int64_t(t) * per);
  const int seq = as_global(a.seq)[t], slot = as_global(a.slot)[t], pos = as_global(a.pos)[t];
  if (seq < 0 || seq >= a.c.batch || slot < 0 || slot >= a.c.rows) return;
  if (a.cos && (pos < 0 || pos >= a.rope_rows)) return;
  const int in_table = a.c.by_page.div(slot);
  const int page = as_global(a.c.table)[int64_t(seq) * a.c.width + in_table];
  if (page < 0 || page >= a.c.pages) return;
  // (all of a row's lanes are here or none)
  const bool in = d < a.c.dim;
  if (r < a.heads) {
    if (in)
      store4<VEC>(a.q_out, int64_t(t) * a.q_out_stride + int64_t(r) * a.c.dim + d, a.type,
                  rotated<VEC>(a, a.q, int64_t(t) * a.q_stride + int64_t(r) * a.c.dim, d, pos));
    return;
  }
  const bool is_k = r < a.heads + a.c.kv;
  const int h = r - a.heads - (is_k ? 0 : a.c.kv);
  float4 x = make_float4(0, 0, 0, 0);
  if (in)
    x = is_k ? rotated<VEC>(a, a.k, int64_t(t) * a.k_stride + int64_t(h) * a.c.dim, d, pos)
             : load4<VEC>(a.v, int64_t(t) * a.v_stride + int64_t(h) * a.c.dim + d, a.type);
  const int off = slot - in_table * a.c.page_size;
  char* pool = is_k ? a.c.k : a.c.v;
  const int64_t at = a.c.at(page, h) + int64_t(off) * a.c.dim + d;
  if (a.cache_type == SHERRY_I8) {
    float top = fmaxf(fmaxf(fabsf(x.x), fabsf(x.y)), fmaxf(fabsf(x.z), fabsf(x.w)));
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
    const float s = top / 127.0f;
    if (in)
      *reinterpret_cast<SHERRY_GLOBAL uint32_t*>(as_global_mut(pool) + at) =
          top == 0.0f ? 0u : quant4(x, s, 1.0f / s);
    if (d == 0) as_global_mut(is_k ? a.c.ks : a.c.vs)[a.c.scale_at(page, h) + off] = s;
  } else if (in) {
    store4<true>(pool, at, a.cache_type, x);
  }
  if (is_k && d == 0) {
    const int64_t w = (int64_t(seq) * a.c.kv + h) * a.row_stride + slot;
    if (a.weight) as_global_mut(a.weight)[w] = 0.0f;
    if (a.position) as_global_mut(a.position)[w] = pos;
  }
}

template <int LPR>
int launch_lanes(const Append& a, bool vec, hipStream_t s) {
  const int64_t rows = int64_t(a.tokens) * (a.heads + 2 * a.c.kv);
  const dim3 grid(static_cast<unsigned>(ceil_div(rows, 256 / LPR)));
  return vec ? launch(append_kernel<LPR, true>, grid, dim3(256), 0, s, a)
             : launch(append_kernel<LPR, false>, grid, dim3(256), 0, s, a);
}

}  // namespace

int launch_append(const sherry_cache_desc& c, const sherry_append_desc& d, hipStream_t s) {
  const int heads = d.q ? d.heads : 0;
  const int64_t qrow = int64_t(heads) * c.head_dim, row = int64_t(c.kv_heads) * c.head_dim;
  const Append a{cache_of(c), d.q, d.k, d.v, d.q_out, d.seq, d.slot, d.pos, d.cos, d.sin, d.weight,
                 d.position, d.row_stride, d.q_stride ? d.q_stride : qrow, d.k_stride ? d.k_stride : row,
                 d.v_stride ? d.v_stride : row, d.q_out_stride ? d.q_out_stride : qrow, d.tokens, heads,
                 d.type, c.type, d.rope_rows, d.rot_dim, d.pairing == SHERRY_ROPE_PAIRS};
  // four values at once where every row starts at a multiple of them
  const uintptr_t bytes = 4 * static_cast<uintptr_t>(type_bytes(d.type));
  auto whole = [&](const void* p, int64_t stride) {
    return reinterpret_cast<uintptr_t>(p) % bytes == 0 && stride % 4 == 0;
  };
  const bool vec = whole(a.k, a.k_stride) && whole(a.v, a.v_stride) &&
                   (!heads || (whole(a.q, a.q_stride) && whole(a.q_out, a.q_out_stride))) &&
                   reinterpret_cast<uintptr_t>(a.cos) % 16 == 0 && reinterpret_cast<uintptr_t>(a.sin) % 16 == 0;
  if (c.head_dim <= 64) return launch_lanes<16>(a, vec, s);
  if (c.head_dim <= 128) return launch_lanes<32>(a, vec, s);
  return launch_lanes<64>(a, vec, s);
}

}  // namespace sherry
