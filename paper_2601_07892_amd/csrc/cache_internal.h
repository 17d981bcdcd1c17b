// What the kernels of the paged key-value cache share (not part of the ABI).
#pragma once

#include "sherry_internal.h"

namespace sherry {

// Division of 0 .. 2^31 - 1 by a fixed divisor: n / d = umulhi(n, mul) >> shift
// (mul = ceil(2^(32 + shift) / d) with 2^shift >= d / 2 fits 32 bits and is exact
// for 31-bit n; d = 1 is a pass-through).
struct FastDiv {
  uint32_t d, mul, shift;
  static FastDiv of(uint32_t d) {
    FastDiv f{d, 0, 0};
    if (d <= 1) return f;
    while ((2u << f.shift) < d) ++f.shift;
    f.mul = static_cast<uint32_t>(((1ull << (32 + f.shift)) + d - 1) / d);
    return f;
  }
  __device__ __forceinline__ uint32_t div(uint32_t n) const {
    return d <= 1 ? n : quotient(n);
  }
  // d >= 2
  __device__ __forceinline__ uint32_t quotient(uint32_t n) const { return __umulhi(n, mul) >> shift; }
};

// A sherry_cache_desc as the kernels take it.
struct Cache {
  char* k;
  char* v;
  float* ks;
  float* vs;
  const int32_t* table;
  int64_t page_stride;  // elements
  int pages, kv, page_size, dim, batch, width, rows;  // rows = width * page_size
  FastDiv by_page;
  // First row of head h in page p, in rows (scales) and in elements.
  __device__ __forceinline__ int64_t scale_at(int page, int h) const {
    return (int64_t(page) * kv + h) * page_size;
  }
  __device__ __forceinline__ int64_t at(int page, int h) const {
    return int64_t(page) * page_stride + int64_t(h) * page_size * dim;
  }
  // Rows of sequence b that a length asks for: 0 .. rows.
  __device__ __forceinline__ int length(const int32_t* lengths, int b) const {
    const int n = as_global(lengths)[b];
    return n < 0 ? 0 : n < rows ? n : rows;
  }
};

inline Cache cache_of(const sherry_cache_desc& d) {
  const int64_t whole = int64_t(d.kv_heads) * d.page_size * d.head_dim;
  return Cache{static_cast<char*>(d.k), static_cast<char*>(d.v), d.k_scale, d.v_scale, d.table,
               d.page_stride ? d.page_stride : whole, d.pages, d.kv_heads, d.page_size,
               d.head_dim, d.batch, d.table_width, d.table_width * d.page_size,
               FastDiv::of(static_cast<uint32_t>(d.page_size))};
}

inline int type_bytes(int type) { return type == SHERRY_F32 ? 4 : type == SHERRY_I8 ? 1 : 2; }

// fp32 -> 16 bits, to nearest even (NaN stays NaN).
__device__ __forceinline__ uint16_t to_bf16(float x) {
  const uint32_t u = __float_as_uint(x);
  if (x != x) return static_cast<uint16_t>((u >> 16) | 0x40u);
  return static_cast<uint16_t>((u + 0x7FFFu + ((u >> 16) & 1u)) >> 16);
}
__device__ __forceinline__ uint16_t to_f16(float x) {
  return __builtin_bit_cast(uint16_t, static_cast<_Float16>(x));
}
__device__ __forceinline__ float from_bf16(uint16_t h) { return __uint_as_float(uint32_t(h) << 16); }
__device__ __forceinline__ float from_f16(uint16_t h) {
  return static_cast<float>(__builtin_bit_cast(_Float16, h));
}

// Element i of a row of q, k, v or out of a type (SHERRY_F32, _F16, _BF16).
__device__ __forceinline__ float load_as_f32(const void* p, int64_t i, int type) {
  if (type == SHERRY_F32) return as_global(static_cast<const float*>(p))[i];
  const uint16_t h = as_global(static_cast<const uint16_t*>(p))[i];
  return type == SHERRY_BF16 ? from_bf16(h) : from_f16(h);
}
__device__ __forceinline__ void store_from_f32(void* p, int64_t i, int type, float x) {
  if (type == SHERRY_F32) as_global_mut(static_cast<float*>(p))[i] = x;
  else as_global_mut(static_cast<uint16_t*>(p))[i] = type == SHERRY_BF16 ? to_bf16(x) : to_f16(x);
}

// Inclusive sums over the lanes (steps inside 16 lanes, then across them).
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, true);  // from 1, 2, 4, 8 lanes below
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, true);  // lane 15 of the row below
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, true);  // lane 31
  return v;
}

// Threads of a call's largest launch; a grid holds 2^32 - 1.
int64_t append_threads(const sherry_cache_desc& c, const sherry_append_desc& a);
int64_t attend_threads(const sherry_cache_desc& c, const sherry_attend_desc& a);
int64_t evict_threads(const sherry_cache_desc& c, const sherry_evict_desc& a);
inline bool fits_grid(int64_t threads) { return threads <= int64_t(UINT32_MAX); }

size_t attend_workspace(const sherry_cache_desc& c, const sherry_attend_desc& a);
int launch_attend(const sherry_cache_desc& c, const sherry_attend_desc& a, hipStream_t s);
int launch_append(const sherry_cache_desc& c, const sherry_append_desc& a, hipStream_t s);
int launch_evict(const sherry_cache_desc& c, const sherry_evict_desc& a, hipStream_t s);

}  // namespace sherry
