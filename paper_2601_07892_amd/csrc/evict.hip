// A cache cut down to `keep` rows per sequence and key-value head, by
// accumulated attention weight.
//
// Two launches.  select: one workgroup per sequence and head finds the keep-th
// largest key (a radix select over the fp32 weights as ordered integers,
// protected rows above all) and writes, for every new row, its former slot:
// rows kept below the new length stay, the j-th kept row past it goes to the
// j-th slot given up below it.  move: copies those rows, and every new row's
// weight and position; sources lie past the new length and destinations below
// it, so the copies need no order.
//
// What bounds it: the rows that move are read and written once, the weights
// and positions read; below some thousand rows the two launches.
//
// Measured: 16 sequences of 1000 to 16384 rows cut to 4096, 8 heads of 128 f16
// values: select 20 us, most of it the longest sequence's passes over the keys in
// registers and LDS (a workgroup per sequence and head; several would need a
// launch between the passes); move 38 us for 150 MB read and written, 4.0 TB/s,
// where a copy reaches 4.9.  8 sequences of 2304 rows of 64 values cut to 2048:
// 7.4 and 5.5 us.
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
};

// Exclusive sum of one value per wave, over the workgroup's waves in order;
// total: of all.  part: kWaves integers that no other call uses.
__device__ __forceinline__ int waves_before(int v, int* part, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (lane == 0) part[wave] = v;
  __syncthreads();
  const int upto = wave_scan(lane < kWaves ? part[lane] : 0);
  total = __builtin_amdgcn_readlane(upto, kWaves - 1);
  return wave ? __builtin_amdgcn_readlane(upto, __builtin_amdgcn_readfirstlane(wave) - 1) : 0;
}

// Each wave takes a run of slots, in chunks of 64, and keeps their keys: J per
// lane, for sequences of up to 1024 J rows; J = 0 reads them again in every pass.
// Sequences of 2304 rows: 7.4 us with J = 4, 15.7 with 64, 14.6 with 0; of up to
// 16384 20 with 16, 27 with 64, 29 with 0; of 60000 63 with 64, of 100000 145 with 0.
template <int J>
struct Run {
  const Keys& keys;
  int first, end;  // of this wave
  int last;        // of the sequence
  uint32_t key[J > 0 ? J : 1];

  __device__ __forceinline__ Run(const Keys& k, int n) : keys(k), last(n - 1) {
    const int seg = ((n + kWaves - 1) / kWaves + 63) / 64 * 64;
    first = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6) * seg);
    end = __builtin_amdgcn_readfirstlane(first + seg < n ? first + seg : n);
    if constexpr (J > 0) {
      constexpr int AT = J < 16 ? J : 16;
#pragma unroll
      for (int j0 = 0; j0 < J; j0 += AT) {
        uint32_t k16[AT];
        load<AT>(first + 64 * j0, k16);
#pragma unroll
        for (int u = 0; u < AT; ++u) key[j0 + u] = k16[u];
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  // Keys of AT chunks from slot i0 on (past the last slot, that of the last):
  // every load goes out, so that none waits for another's branch.
  template <int AT>
  __device__ __forceinline__ void load(int i0, uint32_t (&k)[AT]) const {
    const int lane = threadIdx.x & 63;
    float w[AT];
    int32_t p[AT];
#pragma unroll
    for (int u = 0; u < AT; ++u) {
      const int i = i0 + 64 * u + lane;
      w[u] = as_global(keys.w)[i < last ? i : last];
      p[u] = i;
    }
    if (keys.recent && keys.pos) {
#pragma unroll
      for (int u = 0; u < AT; ++u) {
        const int i = i0 + 64 * u + lane;
        p[u] = as_global(keys.pos)[i < last ? i : last];
      }
    }
#pragma unroll
    for (int u = 0; u < AT; ++u)
      k[u] = keys.recent && p[u] >= keys.from ? 0xFFFFFFFFu : weight_key(w[u]);
  }
  // f(chunk, slot, whether it is of the run, its key): in order; every lane calls it.
  template <class F>
  __device__ __forceinline__ void each(F&& f) const {
    const int lane = threadIdx.x & 63;
    if constexpr (J > 0) {
#pragma unroll
      for (int j = 0; j < J; ++j) {
        if (first + 64 * j >= end) break;
        f(j, first + 64 * j + lane, first + 64 * j + lane < end, key[j]);
      }
    } else {
      constexpr int AT = 16;  // chunks whose loads go out together
      for (int i0 = first; i0 < end; i0 += 64 * AT) {
        uint32_t k[AT];
        load<AT>(i0, k);
#pragma unroll
        for (int u = 0; u < AT; ++u) {
          const int i = i0 + 64 * u;
          if (i >= end) break;
          f((i - first) / 64, i + lane, i + lane < end, k[u]);
        }
      }
    }
  }
};

template <int J>
__global__ __launch_bounds__(kThreads) void evict_select_kernel(Evict a) {
  __shared__ uint32_t hist[2048];
  __shared__ int part[6][kWaves];
  __shared__ uint32_t found[3];
  __shared__ int list[kList];
  const int b = blockIdx.x / a.c.kv, h = blockIdx.x - b * a.c.kv;
  const int n = a.c.length(a.length, b);
  const int m = n < a.keep ? n : a.keep;
  const int64_t row = int64_t(blockIdx.x) * a.row_stride, orow = int64_t(blockIdx.x) * a.out_stride;
  const float* w = a.weight + row;
  const int32_t* pos = a.position ? a.position + row : nullptr;
  const int tid = threadIdx.x, lane = tid & 63;
  if (h == 0 && tid == 0) as_global_mut(a.length_out)[b] = m;
  // past the end -1; a sequence that fits stays as it is
  for (int i = (n <= a.keep ? 0 : m) + tid; i < a.keep; i += kThreads)
    as_global_mut(a.kept)[orow + i] = i < m ? i : -1;
  if (n <= a.keep) return;
  const Keys keys{w, pos, a.recent_from ? as_global(a.recent_from)[b] : 0, a.recent_from != nullptr};
  const Run<J> run(keys, n);

  // the m-th largest key, 11, 11 and 10 bits at a time: of the keys with the
  // bits found so far, `want` are to be taken.  Where that is all of them, the
  // bits that follow decide nothing.
  uint32_t prefix = 0;
  int want = m, shift = 32;
#pragma unroll
  for (int r = 0; r < 3; ++r) {
    const int bits = r < 2 ? 11 : 10;
    const int above = shift;
    shift -= bits;
    hist[tid] = 0;
    hist[tid + 1024] = 0;
    __syncthreads();
    run.each([&](int, int, bool in, uint32_t k) {
      if (in && (r == 0 || (k >> (above & 31)) == prefix))
        atomicAdd(&hist[(k >> shift) & ((1u << bits) - 1)], 1u);
    });
    __syncthreads();
    // thread t: bins 2047 - 2 t and 2046 - 2 t, from the largest down
    const int c0 = hist[2047 - 2 * tid], c1 = hist[2046 - 2 * tid];
    const int upto = wave_scan(c0 + c1);
    int total;
    const int before = waves_before(__builtin_amdgcn_readlane(upto, 63), part[r], total) + upto - c0 - c1;
    const bool first = before < want && before + c0 >= want;
    if (first || (before + c0 < want && before + c0 + c1 >= want)) {
      found[0] = first ? 2047 - 2 * tid : 2046 - 2 * tid;
      found[1] = first ? want - before : want - before - c0;
      found[2] = first ? c0 : c1;
    }
    __syncthreads();
    prefix = prefix << bits | found[0];
    want = found[1];
    if (found[2] == static_cast<uint32_t>(want)) break;
  }
  // kept: every key above prefix (in its bits), and the first `want` that
  // equal it
  const uint64_t below = (1ull << lane) - 1;
  const bool ties = found[2] != static_cast<uint32_t>(want);
  int total, eq = 0;
  if (ties) {
    int equal = 0;
    run.each([&](int, int, bool in, uint32_t k) { equal += __popcll(__ballot(in && (k >> shift) == prefix)); });
    eq = waves_before(equal, part[3], total);
  }
  // f(chunk, slot of lane 0, lanes of the chunk that are kept)
  auto chunks = [&](auto&& f) {
    int seen = eq;
    run.each([&](int j, int i, bool in, uint32_t k) {
      const uint32_t top = k >> shift;
      bool keep = in && top >= prefix;
      if (ties) {
        const uint64_t e = __ballot(in && top == prefix);
        keep = keep && (top > prefix || seen + __popcll(e & below) < want);
        seen += __popcll(e);
      }
      f(j, i - lane, __ballot(keep));
    });
  };
  // Kept slots past m (movers) go to slots below m that are not (holes).  The
  // wave's kept lanes, one chunk a lane, give every chunk its first mover's and
  // first hole's number.
  auto below_m = [&](int i0) {  // lanes of a chunk whose slots are below m (and the run's end)
    const int k = (m < run.end ? m : run.end) - i0;
    return k <= 0 ? 0ull : k >= 64 ? ~0ull : (1ull << k) - 1;
  };
  int n_moves = 0, n_holes = 0;  // of the wave
  uint64_t mine = 0;             // J > 0: chunk lane's kept lanes
  chunks([&](int j, int i0, uint64_t kept) {
    const uint64_t low = below_m(i0);
    n_moves += __popcll(kept & ~low);
    n_holes += __popcll(~kept & low);
    if (J > 0 && lane == j) mine = kept;
  });
  int moves, holes;
  const int mover0 = waves_before(n_moves, part[4], moves);
  const int hole0 = waves_before(n_holes, part[5], holes);
  int my_moves = 0, my_holes = 0;  // J > 0: before chunk `lane` of the wave
  if constexpr (J > 0) {
    const uint64_t low = below_m(run.first + 64 * lane);
    const int c = __popcll(mine & ~low), d = __popcll(~mine & low);
    my_moves = wave_scan(c) - c;
    my_holes = wave_scan(d) - d;
  }
  // every chunk's kept lanes again, with the numbers of its first mover and hole
  auto again = [&](auto&& f) {
    if constexpr (J > 0) {
      const int count = (run.end - run.first + 63) / 64;
      for (int j = 0; j < count; ++j) {
        const uint32_t hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(mine >> 32), j);
        const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(mine), j);
        const uint64_t kept = uint64_t(hi) << 32 | lo;
        f(run.first + 64 * j, kept, mover0 + __builtin_amdgcn_readlane(my_moves, j),
          hole0 + __builtin_amdgcn_readlane(my_holes, j));
      }
    } else {
      int r = mover0, q = hole0;
      chunks([&](int, int i0, uint64_t kept) {
        f(i0, kept, r, q);
        const uint64_t low = below_m(i0);
        r += __popcll(kept & ~low);
        q += __popcll(~kept & low);
      });
    }
  };
  for (int base = 0; base == 0 || base < moves; base += kList) {
    __syncthreads();
    again([&](int i0, uint64_t kept, int r, int) {
      const uint64_t who = kept & ~below_m(i0);
      const int at = r - base + __popcll(who & below);
      if ((who >> lane & 1) && at >= 0 && at < kList) list[at] = i0 + lane;
    });
    __syncthreads();
    again([&](int i0, uint64_t kept, int, int q) {
      const uint64_t low = below_m(i0), who = ~kept & low;
      const int at = q - base + __popcll(who & below);
      int src = -1;
      if ((who >> lane & 1) && at >= 0 && at < kList) src = list[at];
      if ((kept & low) >> lane & 1) src = base == 0 ? i0 + lane : -1;
      if (src >= 0) as_global_mut(a.kept)[orow + i0 + lane] = src;
    });
  }
}

constexpr int kMoveAt = 4;  // rows in flight per thread (2 and 8: the same 37 to 39 us)

// LPR lanes of 16 bytes per row (rows of 8 bytes do not exist: head_dim is a
// multiple of 8, of 16 in int8), 256 / LPR * kMoveAt new rows per workgroup.
// Past `copies` workgroups, the new rows' weights and positions, 256 * kMoveAt of
// them per workgroup.
template <int LPR>
__global__ __launch_bounds__(256) void evict_move_kernel(Evict a, int copies) {
  constexpr int ROWS = 256 / LPR, PER = ROWS * kMoveAt;
  if (static_cast<int>(blockIdx.x) >= copies) {
    constexpr int ALL = 256 * kMoveAt;
    const int chunks = (a.keep + ALL - 1) / ALL, blk = static_cast<int>(blockIdx.x) - copies;
    const int bh = blk / chunks, i0 = (blk - bh * chunks) * ALL + threadIdx.x;
    const int64_t row = int64_t(bh) * a.row_stride, orow = int64_t(bh) * a.out_stride;
    int src[kMoveAt];
    float w[kMoveAt];
    int32_t pos[kMoveAt];
#pragma unroll
    for (int u = 0; u < kMoveAt; ++u) {
      const int i = i0 + 256 * u;
      src[u] = i < a.keep ? as_global(a.kept)[orow + i] : -1;
    }
#pragma unroll
    for (int u = 0; u < kMoveAt; ++u) {
      const int64_t at = row + (src[u] < 0 ? 0 : src[u]);
      w[u] = a.weight_out ? as_global(a.weight)[at] : 0.0f;
      pos[u] = a.position_out && a.position ? as_global(a.position)[at] : src[u];
    }
#pragma unroll
    for (int u = 0; u < kMoveAt; ++u) {
      const int i = i0 + 256 * u;
      if (i >= a.keep) break;
      if (a.weight_out) as_global_mut(a.weight_out)[orow + i] = src[u] < 0 ? 0.0f : w[u];
      if (a.position_out) as_global_mut(a.position_out)[orow + i] = src[u] < 0 ? 0 : pos[u];
    }
    return;
  }
  const int chunks = (a.keep + PER - 1) / PER;
  const int bh = blockIdx.x / chunks, ch = blockIdx.x - bh * chunks;
  const int b = bh / a.c.kv, h = bh - b * a.c.kv;
  const int n = a.c.length(a.length, b);
  const int p = 16 * (threadIdx.x % LPR), i0 = ch * PER + threadIdx.x / LPR;
  const int e = a.bytes / a.c.dim;
  const int64_t trow = int64_t(b) * a.c.width;
  const int64_t orow = int64_t(bh) * a.out_stride;
  int src[kMoveAt];
#pragma unroll
  for (int u = 0; u < kMoveAt; ++u) {
    const int i = i0 + u * ROWS;
    src[u] = i < a.keep ? as_global(a.kept)[orow + i] : i;
  }
  if (n <= a.keep) return;
  bool live[kMoveAt];
  int64_t to[kMoveAt], from[kMoveAt];  // elements
  u32x4 x[kMoveAt], y[kMoveAt];
  float sx[kMoveAt], sy[kMoveAt];
  int64_t sto[kMoveAt], sfrom[kMoveAt];
#pragma unroll
  for (int u = 0; u < kMoveAt; ++u) {
    const int i = i0 + u * ROWS;
    live[u] = src[u] != i;
    const int at = live[u] ? i : 0, was = live[u] ? src[u] : 0;
    const int it = a.c.by_page.div(at), st = a.c.by_page.div(was);
    int ip = as_global(a.c.table)[trow + it], sp = as_global(a.c.table)[trow + st];
    live[u] = live[u] && ip >= 0 && ip < a.c.pages && sp >= 0 && sp < a.c.pages;
    if (!live[u]) ip = sp = 0;
    const int io = at - it * a.c.page_size, so = was - st * a.c.page_size;
    to[u] = a.c.at(ip, h) + int64_t(io) * a.c.dim;
    from[u] = a.c.at(sp, h) + int64_t(so) * a.c.dim;
    sto[u] = a.c.scale_at(ip, h) + io;
    sfrom[u] = a.c.scale_at(sp, h) + so;
  }
  const bool in = p < a.bytes, scale = a.c.ks && p == 0;
#pragma unroll
  for (int u = 0; u < kMoveAt; ++u) {
    if (!live[u]) continue;
    if (in) {
      x[u] = *reinterpret_cast<const SHERRY_GLOBAL u32x4*>(as_global(a.c.k) + from[u] * e + p);
      y[u] = *reinterpret_cast<const SHERRY_GLOBAL u32x4*>(as_global(a.c.v) + from[u] * e + p);
    }
    if (scale) {
      sx[u] = as_global(a.c.ks)[sfrom[u]];
      sy[u] = as_global(a.c.vs)[sfrom[u]];
    }
  }
#pragma unroll
  for (int u = 0; u < kMoveAt; ++u) {
    if (!live[u]) continue;
    if (in) {
      *reinterpret_cast<SHERRY_GLOBAL u32x4*>(as_global_mut(a.c.k) + to[u] * e + p) = x[u];
      *reinterpret_cast<SHERRY_GLOBAL u32x4*>(as_global_mut(a.c.v) + to[u] * e + p) = y[u];
    }
    if (scale) {
      as_global_mut(a.c.ks)[sto[u]] = sx[u];
      as_global_mut(a.c.vs)[sto[u]] = sy[u];
    }
  }
}

int lanes_per_row(int bytes) { return bytes <= 64 ? 4 : bytes <= 128 ? 8 : bytes <= 256 ? 16 : 32; }
// Workgroups of the moving launch: those that copy rows (with room for every row
// nothing moves), and those that write weights and positions.
int64_t copy_groups(int64_t heads, int keep, int64_t rows, int lanes) {
  return keep < rows ? heads * ceil_div(keep, 256 / lanes * kMoveAt) : 0;
}
int64_t out_groups(int64_t heads, int keep, bool outs) {
  return outs ? heads * ceil_div(keep, 256 * kMoveAt) : 0;
}

template <int LPR>
int launch_move(const Evict& a, hipStream_t s) {
  const int64_t heads = int64_t(a.c.batch) * a.c.kv;
  const int64_t copies = copy_groups(heads, a.keep, a.c.rows, LPR);
  const int64_t outs = out_groups(heads, a.keep, a.weight_out || a.position_out);
  if (copies + outs == 0) return SHERRY_OK;
  return launch(evict_move_kernel<LPR>, dim3(static_cast<unsigned>(copies + outs)), dim3(256), 0, s, a,
                static_cast<int>(copies));
}

}  // namespace

int64_t evict_threads(const sherry_cache_desc& c, const sherry_evict_desc& d) {
  const int64_t heads = int64_t(c.batch) * c.kv_heads, rows = int64_t(c.table_width) * c.page_size;
  const int lanes = lanes_per_row(c.head_dim * type_bytes(c.type));
  const int64_t move = 256 * (copy_groups(heads, d.keep, rows, lanes) +
                              out_groups(heads, d.keep, d.weight_out || d.position_out));
  const int64_t select = kThreads * heads;
  return move > select ? move : select;
}

int launch_evict(const sherry_cache_desc& c, const sherry_evict_desc& d, hipStream_t s) {
  const Evict a{cache_of(c), d.length, d.weight, d.position, d.recent_from, d.length_out, d.kept,
                d.weight_out, d.position_out, d.row_stride, d.out_stride, d.keep,
                c.head_dim * type_bytes(c.type)};
  const dim3 grid(static_cast<unsigned>(int64_t(c.batch) * c.kv_heads)), block(kThreads);
  const int64_t rows = a.c.rows;
  const int rc = rows <= 4 * kThreads    ? launch(evict_select_kernel<4>, grid, block, 0, s, a)
                 : rows <= 16 * kThreads ? launch(evict_select_kernel<16>, grid, block, 0, s, a)
                 : rows <= 64 * kThreads ? launch(evict_select_kernel<64>, grid, block, 0, s, a)
                                         : launch(evict_select_kernel<0>, grid, block, 0, s, a);
  if (rc != SHERRY_OK) return rc;
  switch (lanes_per_row(a.bytes)) {
    case 4: return launch_move<4>(a, s);
    case 8: return launch_move<8>(a, s);
    case 16: return launch_move<16>(a, s);
    default: return launch_move<32>(a, s);
  }
}

}  // namespace sherry
