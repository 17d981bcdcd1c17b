// Rows of new tokens as append and extend read, turn and write them:
//
//   y_a = a c - b s,  y_b = b c + a s  in fp32, each operation rounded
//
// four values a lane.
#pragma once

#include "cache_internal.h"

namespace sherry {

typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));

// TYPE: SHERRY_F32, _F16 or _BF16 of q, k, v and q_out.  VEC: their rows and the
// angles' start at multiples of four values (appending 2048 tokens of 32 + 16 heads of 64
// int8 values 12 us against 18 value by value, extending by 8 prompts 21 against 46).
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

// Angles of rotary positions (cos NULL: none), and which values are turned.
struct Rotary {
  const float* cos;
  const float* sin;
  int rows, rot, pairs;
  __device__ __forceinline__ bool has(int pos) const { return !cos || (pos >= 0 && pos < rows); }
};

// Values d .. d + 3 of a row at element `at`, turned (by cos, sin, rot and pairs of a Rotary or of
// what has them too).
template <int TYPE, bool VEC, class Angles>
__device__ __forceinline__ float4 rotated(const Angles& a, const void* p, int64_t at, int d, int pos) {
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

// A token's rows, 4 values a lane: lanes that a row takes.
inline int lanes_per_row(int dim) { return dim <= 64 ? 16 : dim <= 128 ? 32 : 64; }
// Whether every row at p starts at a multiple of four values of a type.
inline bool whole_pieces(const void* p, int64_t stride, int type) {
  return reinterpret_cast<uintptr_t>(p) % (4 * static_cast<uintptr_t>(type_bytes(type))) == 0 && stride % 4 == 0;
}

}  // namespace sherry
