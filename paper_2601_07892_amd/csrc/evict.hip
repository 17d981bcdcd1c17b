// A cache cut down to `keep` rows per sequence and key-value head, by
// accumulated attention weight.
//
// Two launches.  select: one workgroup per sequence and head finds the keep-th
// largest key (a radix select over the fp32 weights as ordered integers,
// protected rows above all) and writes, for every new row, its former slot:
// rows kept below the new length stay, the j-th kept row past it goes to the
// j-th slot given up below it.  move: copies those rows; sources lie past the
// new length and destinations below it, so the copies need no order.
//
// What bounds it: the rows that move are read and written once, the weights
// and positions read; below some thousand rows the two launches.
#include "cache_internal.h"

namespace sherry {
namespace {

struct Evict {
  Cache c;
  const int32_t* length;
  const float* weight;
  const int32_t* position;
  const int32_t* recent_from;
  int32_t* length_out;
  int32_t* kept;
  float* weight_out;
  int32_t* position_out;
  int64_t row_stride, out_stride;
  int keep, bytes;  // bytes per row of k or v
};

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kList = 16384;  // moves that are matched at a time

// fp32 weights as integers of the same order; NaN as -infinity, -0 as 0.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0x007FFFFFu;
  const uint32_t u = __float_as_uint(w == 0.0f ? 0.0f : w);
  return u >> 31 ? ~u : u | 0x80000000u;
}

struct Keys {
  const float* w;
  const int32_t* pos;
  int from;
  bool recent;
  __device__ __forceinline__ uint32_t at(int i) const {
    if (recent && (pos ? as_global(pos)[i] : i) >= from) return 0xFFFFFFFFu;
    return weight_key(as_global(w)[i]);
  }
};

// Exclusive sum of one value per wave, over the workgroup's waves in order;
// total: of all.
__device__ __forceinline__ int waves_before(int v, int* part, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  __syncthreads();
  if (lane == 0) part[wave] = v;
  __syncthreads();
  int before = 0;
  total = 0;
  for (int i = 0; i < kWaves; ++i) {
    if (i < wave) before += part[i];
    total += part[i];
  }
  return before;
}

__global__ __launch_bounds__(kThreads) void evict_select_kernel(Evict a) {
  __shared__ uint32_t hist[2048];
  __shared__ int part[kWaves];
  __shared__ uint32_t found[2];
  __shared__ int list[kList];
  const int b = blockIdx.x / a.c.kv, h = blockIdx.x - b * a.c.kv;
  const int n = a.c.length(a.length, b);
  const int m = n < a.keep ? n : a.keep;
  const int64_t row = int64_t(blockIdx.x) * a.row_stride, orow = int64_t(blockIdx.x) * a.out_stride;
  const float* w = a.weight + row;
  const int32_t* pos = a.position ? a.position + row : nullptr;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (h == 0 && tid == 0) as_global_mut(a.length_out)[b] = m;
  auto put = [&](int i, int src) {
    as_global_mut(a.kept)[orow + i] = src;
    if (a.weight_out) as_global_mut(a.weight_out)[orow + i] = as_global(w)[src];
    if (a.position_out) as_global_mut(a.position_out)[orow + i] = pos ? as_global(pos)[src] : src;
  };
  for (int i = m + tid; i < a.keep; i += kThreads) {
    as_global_mut(a.kept)[orow + i] = -1;
    if (a.weight_out) as_global_mut(a.weight_out)[orow + i] = 0.0f;
    if (a.position_out) as_global_mut(a.position_out)[orow + i] = 0;
  }
  if (n <= a.keep) {
    for (int i = tid; i < n; i += kThreads) put(i, i);
    return;
  }
  const Keys keys{w, pos, a.recent_from ? as_global(a.recent_from)[b] : 0, a.recent_from != nullptr};

  // the m-th largest key, 11, 11 and 10 bits at a time: of the keys with the
  // bits found so far, `want` are to be taken
  uint32_t prefix = 0;
  int want = m, shift = 32;
#pragma unroll
  for (int r = 0; r < 3; ++r) {
    const int bits = r < 2 ? 11 : 10;
    shift -= bits;
    hist[tid] = 0;
    hist[tid + 1024] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += kThreads) {
      const uint32_t k = keys.at(i);
      if (r == 0 || (k >> (shift + bits)) == prefix) atomicAdd(&hist[(k >> shift) & ((1u << bits) - 1)], 1u);
    }
    __syncthreads();
    // thread t: bins 2047 - 2 t and 2046 - 2 t, from the largest down
    const int c0 = hist[2047 - 2 * tid], c1 = hist[2046 - 2 * tid];
    int upto = c0 + c1;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(upto, o, 64);
      if (lane >= o) upto += v;
    }
    int total;
    const int before = waves_before(__shfl(upto, 63, 64), part, total) + upto - c0 - c1;
    if (before < want && before + c0 >= want) {
      found[0] = 2047 - 2 * tid;
      found[1] = want - before;
    } else if (before + c0 < want && before + c0 + c1 >= want) {
      found[0] = 2046 - 2 * tid;
      found[1] = want - before - c0;
    }
    __syncthreads();
    prefix = prefix << bits | found[0];
    want = found[1];
  }
  // kept: every key above prefix, and the first `want` that equal it.  Each
  // wave takes a run of slots, 64 at a time.
  const int seg = ((n + kWaves - 1) / kWaves + 63) / 64 * 64;
  const int s0 = wave * seg, s1 = s0 + seg < n ? s0 + seg : n;
  const uint64_t below = (1ull << lane) - 1;
  int equal = 0;
  for (int i = s0; i < s1; i += 64)
    equal += __popcll(__ballot(i + lane < s1 && keys.at(i + lane) == prefix));
  int total;
  const int equal0 = waves_before(equal, part, total);
  // holes (slots below m given up) and movers (kept slots past it)
  auto scan = [&](auto&& each) {
    int eq = equal0;
    for (int i = s0; i < s1; i += 64) {
      const bool in = i + lane < s1;
      const uint32_t k = in ? keys.at(i + lane) : 0;
      const uint64_t e = __ballot(in && k == prefix);
      const bool keep = in && (k > prefix || (k == prefix && eq + __popcll(e & below) < want));
      eq += __popcll(e);
      each(i + lane, in && !keep && i + lane < m, keep && i + lane >= m, keep && i + lane < m);
    }
  };
  int holes = 0, movers = 0;
  scan([&](int, bool hole, bool mover, bool) {
    holes += __popcll(__ballot(hole));
    movers += __popcll(__ballot(mover));
  });
  int moves, moves2;
  const int hole0 = waves_before(holes, part, moves);
  const int mover0 = waves_before(movers, part, moves2);
  for (int base = 0; base == 0 || base < moves; base += kList) {
    __syncthreads();
    int rank = mover0 - base;
    scan([&](int i, bool, bool mover, bool) {
      const uint64_t who = __ballot(mover);
      const int at = rank + __popcll(who & below);
      if (mover && at >= 0 && at < kList) list[at] = i;
      rank += __popcll(who);
    });
    __syncthreads();
    rank = hole0 - base;
    scan([&](int i, bool hole, bool, bool stays) {
      const uint64_t who = __ballot(hole);
      const int at = rank + __popcll(who & below);
      if (hole && at >= 0 && at < kList) put(i, list[at]);
      if (stays && base == 0) put(i, i);
      rank += __popcll(who);
    });
  }
}

constexpr int kMoveRows = 64;  // new rows per workgroup

// LPR lanes of 16 bytes per row (8-byte rows of 8 int8 values do not exist:
// head_dim is a multiple of 8, of 16 in int8).
__global__ __launch_bounds__(256) void evict_move_kernel(Evict a, int lpr) {
  const int chunks = (a.keep + kMoveRows - 1) / kMoveRows;
  const int ch = blockIdx.x % chunks, bh = blockIdx.x / chunks;
  const int b = bh / a.c.kv, h = bh - b * a.c.kv;
  const int n = a.c.length(a.length, b);
  if (n <= a.keep) return;
  const int end = (ch + 1) * kMoveRows < a.keep ? (ch + 1) * kMoveRows : a.keep;
  const int piece = threadIdx.x % lpr;
  for (int i = ch * kMoveRows + threadIdx.x / lpr; i < end; i += 256 / lpr) {
    const int src = as_global(a.kept)[int64_t(bh) * a.out_stride + i];
    if (src == i) continue;
    const int it = a.c.by_page.div(i), st = a.c.by_page.div(src);
    const int ip = as_global(a.c.table)[int64_t(b) * a.c.width + it];
    const int sp = as_global(a.c.table)[int64_t(b) * a.c.width + st];
    if (ip < 0 || ip >= a.c.pages || sp < 0 || sp >= a.c.pages) continue;
    const int io = i - it * a.c.page_size, so = src - st * a.c.page_size;
    const int64_t e = a.bytes / a.c.dim;
    const int64_t to = (a.c.at(ip, h) + int64_t(io) * a.c.dim) * e;
    const int64_t from = (a.c.at(sp, h) + int64_t(so) * a.c.dim) * e;
    for (int p = 16 * piece; p < a.bytes; p += 16 * lpr) {
      const u32x4 x = *reinterpret_cast<const SHERRY_GLOBAL u32x4*>(as_global(a.c.k) + from + p);
      const u32x4 y = *reinterpret_cast<const SHERRY_GLOBAL u32x4*>(as_global(a.c.v) + from + p);
      *reinterpret_cast<SHERRY_GLOBAL u32x4*>(as_global_mut(a.c.k) + to + p) = x;
      *reinterpret_cast<SHERRY_GLOBAL u32x4*>(as_global_mut(a.c.v) + to + p) = y;
    }
    if (a.c.ks && piece == 0) {
      const int64_t t = a.c.scale_at(ip, h) + io, f = a.c.scale_at(sp, h) + so;
      as_global_mut(a.c.ks)[t] = as_global(a.c.ks)[f];
      as_global_mut(a.c.vs)[t] = as_global(a.c.vs)[f];
    }
  }
}

}  // namespace

int launch_evict(const sherry_cache_desc& c, const sherry_evict_desc& d, hipStream_t s) {
  const Evict a{cache_of(c), d.length, d.weight, d.position, d.recent_from, d.length_out, d.kept,
                d.weight_out, d.position_out, d.row_stride, d.out_stride, d.keep,
                c.head_dim * type_bytes(c.type)};
  const int64_t heads = int64_t(c.batch) * c.kv_heads;
  const int rc = launch(evict_select_kernel, dim3(static_cast<unsigned>(heads)), dim3(kThreads), 0, s, a);
  if (rc != SHERRY_OK || d.keep >= a.c.rows) return rc;  // (a sequence that fits keep moves nothing)
  int lpr = 1;
  while (lpr < 32 && 16 * lpr < a.bytes) lpr *= 2;
  return launch(evict_move_kernel, dim3(static_cast<unsigned>(heads * ceil_div(d.keep, kMoveRows))),
                dim3(256), 0, s, a, lpr);
}

}  // namespace sherry
