// New tokens into a paged cache: rotary positions on q and k, then k and v
// stored as bf16, f16, or int8 with one scale per row.
//
//   y_a = a c - b s,  y_b = b c + a s  in fp32, each operation rounded
//
// What bounds it: the bytes of the tokens' q, k and v rows, read and written
// once; a decode batch's few hundred rows cost one launch.  A workgroup takes
// rows of one token, whose place in the cache is then found by scalar loads; a
// row takes DP / 4 lanes of four values, so that its absolute maximum (int8) is a
// reduction inside a wave, and its rotation partner is read from the row
// again, out of the caches.
//
// Measured: 32 tokens of 24 + 16 heads of 128 values into f16 3.2 us, a launch's
// latency with two dependent reads; a prompt of 2048 tokens of 32 + 16 heads of 64
// values into int8, 45 MB, 11.6 to 13.0 us, 3.5 to 3.9 TB/s (the inputs are partly
// in the caches).  With rows of any token in a workgroup and the types as
// arguments these took 3.6 and 14.5; several rows per thread were slower.
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
  FastDiv by_parts;  // workgroups per token
};

typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));

// TYPE: SHERRY_F32, _F16 or _BF16 of q, k, v and q_out.  VEC: their rows and the
// angles' start at multiples of four values (the prompt above: 12 us against 18
// value by value).
template <int TYPE>
__device__ __forceinline__ float load1(const void* p, int64_t i) {
  return load_as_f32(p, i, TYPE);
}
template <int TYPE, bool VEC>
__device__ __forceinline__ float4 load4(const void* p, int64_t i) {
  if constexpr (!VEC) {
    return make_float4(load1<TYPE>(p, i), load1<TYPE>(p, i + 1), load1<TYPE>(p, i + 2), load1<TYPE>(p, i + 3));
  } else if constexpr (TYPE == SHERRY_F32) {
    return *reinterpret_cast<const SHERRY_GLOBAL float4*>(as_global(static_cast<const float*>(p)) + i);
  } else {
    const u16x4 h = *reinterpret_cast<const SHERRY_GLOBAL u16x4*>(as_global(static_cast<const uint16_t*>(p)) + i);
    return TYPE == SHERRY_BF16
               ? make_float4(from_bf16(h[0]), from_bf16(h[1]), from_bf16(h[2]), from_bf16(h[3]))
               : make_float4(from_f16(h[0]), from_f16(h[1]), from_f16(h[2]), from_f16(h[3]));
  }
}

// Values d .. d + 3 of a row at element `at`, rotated.
template <int TYPE, bool VEC>
__device__ __forceinline__ float4 rotated(const Append& a, const void* p, int64_t at, int d, int pos) {
  const float4 x = load4<TYPE, VEC>(p, at + d);
  if (!a.cos || d >= a.rot) return x;
  const int half = a.rot >> 1;
  const float* cs = a.cos + int64_t(pos) * half;
  const float* sn = a.sin + int64_t(pos) * half;
  if (VEC && !a.pairs && half % 4 == 0) {
    // the four partners are together; their products are added or subtracted,
    // which is the same as adding those of the negated sine
    const bool first = d < half;
    const int i = first ? d : d - half;
    const float4 w = load4<TYPE, VEC>(p, at + (first ? d + half : i));
    const float4 c = *reinterpret_cast<const SHERRY_GLOBAL float4*>(as_global(cs) + i);
    const float4 s = *reinterpret_cast<const SHERRY_GLOBAL float4*>(as_global(sn) + i);
    const float sg = first ? -1.0f : 1.0f;
    return make_float4(x.x * c.x + w.x * (sg * s.x), x.y * c.y + w.y * (sg * s.y),
                       x.z * c.z + w.z * (sg * s.z), x.w * c.w + w.w * (sg * s.w));
  }
  float r[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int j = d + e;
    if (j >= a.rot) break;
    const bool first = a.pairs ? (j & 1) == 0 : j < half;
    const int i = a.pairs ? j >> 1 : first ? j : j - half;
    const int other = a.pairs ? j ^ 1 : first ? j + half : i;
    const float w = load1<TYPE>(p, at + other) * as_global(sn)[i];
    const float v = r[e] * as_global(cs)[i];
    r[e] = first ? v - w : v + w;
  }
  return make_float4(r[0], r[1], r[2], r[3]);
}

__device__ __forceinline__ u16x4 to_16(int type, float4 v) {
  return type == SHERRY_BF16 ? u16x4{to_bf16(v.x), to_bf16(v.y), to_bf16(v.z), to_bf16(v.w)}
                             : u16x4{to_f16(v.x), to_f16(v.y), to_f16(v.z), to_f16(v.w)};
}
template <int TYPE, bool VEC>
__device__ __forceinline__ void store4(void* p, int64_t i, float4 v) {
  if constexpr (!VEC) {
    store_from_f32(p, i, TYPE, v.x);
    store_from_f32(p, i + 1, TYPE, v.y);
    store_from_f32(p, i + 2, TYPE, v.z);
    store_from_f32(p, i + 3, TYPE, v.w);
  } else if constexpr (TYPE == SHERRY_F32) {
    *reinterpret_cast<SHERRY_GLOBAL float4*>(as_global_mut(static_cast<float*>(p)) + i) = v;
  } else {
    *reinterpret_cast<SHERRY_GLOBAL u16x4*>(as_global_mut(static_cast<uint16_t*>(p)) + i) = to_16(TYPE, v);
  }
}

// 256 / LPR rows (heads of q, k, v) of one token per workgroup, one per LPR lanes.
template <int LPR, int TYPE, bool VEC>
__global__ __launch_bounds__(256) void append_kernel(Append a) {
  const int t = a.by_parts.div(blockIdx.x), part = blockIdx.x - t * a.by_parts.d;
  const int r = part * (256 / LPR) + threadIdx.x / LPR;
  const int d = 4 * (threadIdx.x % LPR);
  const int seq = as_const(a.seq)[t], slot = as_const(a.slot)[t], pos = as_const(a.pos)[t];
  if (seq < 0 || seq >= a.c.batch || slot < 0 || slot >= a.c.rows) return;
  if (a.cos && (pos < 0 || pos >= a.rope_rows)) return;
  const int in_table = a.c.by_page.div(slot);
  const int page = as_const(a.c.table)[int64_t(seq) * a.c.width + in_table];
  if (page < 0 || page >= a.c.pages || r >= a.heads + 2 * a.c.kv) return;
  const bool in = d < a.c.dim;
  if (r < a.heads) {
    if (in)
      store4<TYPE, VEC>(a.q_out, int64_t(t) * a.q_out_stride + r * a.c.dim + d,
                        rotated<TYPE, VEC>(a, a.q, int64_t(t) * a.q_stride + r * a.c.dim, d, pos));
    return;
  }
  const bool is_k = r < a.heads + a.c.kv;
  const int h = r - a.heads - (is_k ? 0 : a.c.kv);
  float4 x = make_float4(0, 0, 0, 0);
  if (in)
    x = is_k ? rotated<TYPE, VEC>(a, a.k, int64_t(t) * a.k_stride + h * a.c.dim, d, pos)
             : load4<TYPE, VEC>(a.v, int64_t(t) * a.v_stride + h * a.c.dim + d);
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
    *reinterpret_cast<SHERRY_GLOBAL u16x4*>(as_global_mut(reinterpret_cast<uint16_t*>(pool)) + at) =
        to_16(a.cache_type, x);
  }
  if (is_k && d == 0) {
    const int64_t w = (int64_t(seq) * a.c.kv + h) * a.row_stride + slot;
    if (a.weight) as_global_mut(a.weight)[w] = 0.0f;
    if (a.position) as_global_mut(a.position)[w] = pos;
  }
}

template <int LPR, int TYPE>
int launch_type(const Append& a, bool vec, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(int64_t(a.tokens) * a.by_parts.d));
  return vec ? launch(append_kernel<LPR, TYPE, true>, grid, dim3(256), 0, s, a)
             : launch(append_kernel<LPR, TYPE, false>, grid, dim3(256), 0, s, a);
}
int lanes_per_row(int dim) { return dim <= 64 ? 16 : dim <= 128 ? 32 : 64; }
// Workgroups per token.
int64_t parts_of(int heads, int kv, int lanes) { return ceil_div(heads + 2 * kv, 256 / lanes); }

template <int LPR>
int launch_lanes(Append a, bool vec, hipStream_t s) {
  a.by_parts = FastDiv::of(static_cast<uint32_t>(parts_of(a.heads, a.c.kv, LPR)));
  switch (a.type) {
    case SHERRY_F32: return launch_type<LPR, SHERRY_F32>(a, vec, s);
    case SHERRY_F16: return launch_type<LPR, SHERRY_F16>(a, vec, s);
    default: return launch_type<LPR, SHERRY_BF16>(a, vec, s);
  }
}

}  // namespace

int64_t append_threads(const sherry_cache_desc& c, const sherry_append_desc& d) {
  return 256 * d.tokens * parts_of(d.q ? d.heads : 0, c.kv_heads, lanes_per_row(c.head_dim));
}

int launch_append(const sherry_cache_desc& c, const sherry_append_desc& d, hipStream_t s) {
  const int heads = d.q ? d.heads : 0;
  const int64_t qrow = int64_t(heads) * c.head_dim, row = int64_t(c.kv_heads) * c.head_dim;
  const Append a{cache_of(c), d.q, d.k, d.v, d.q_out, d.seq, d.slot, d.pos, d.cos, d.sin, d.weight,
                 d.position, d.row_stride, d.q_stride ? d.q_stride : qrow, d.k_stride ? d.k_stride : row,
                 d.v_stride ? d.v_stride : row, d.q_out_stride ? d.q_out_stride : qrow, d.tokens, heads,
                 d.type, c.type, d.rope_rows, d.rot_dim, d.pairing == SHERRY_ROPE_PAIRS, FastDiv{1, 0, 0}};
  // four values at once where every row starts at a multiple of them
  const uintptr_t bytes = 4 * static_cast<uintptr_t>(type_bytes(d.type));
  auto whole = [&](const void* p, int64_t stride) {
    return reinterpret_cast<uintptr_t>(p) % bytes == 0 && stride % 4 == 0;
  };
  const bool vec = whole(a.k, a.k_stride) && whole(a.v, a.v_stride) &&
                   (!heads || (whole(a.q, a.q_stride) && whole(a.q_out, a.q_out_stride))) &&
                   reinterpret_cast<uintptr_t>(a.cos) % 16 == 0 && reinterpret_cast<uintptr_t>(a.sin) % 16 == 0;
  switch (lanes_per_row(c.head_dim)) {
    case 16: return launch_lanes<16>(a, vec, s);
    case 32: return launch_lanes<32>(a, vec, s);
    default: return launch_lanes<64>(a, vec, s);
  }
}

}  // namespace sherry
