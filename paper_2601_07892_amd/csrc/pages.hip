// Pages that sequences share: a table for sequences that go on from others, with pages
// of their own where rows will be written (fork), and the pages in use moved to the
// front of the pool (compact).
//
// Nothing is kept about pages between calls: which are in use, and by how many, is
// counted from the tables each time.
//
// What bounds it: the pages that are copied, read once and written once in every
// layer.  Deciding what is copied is a few passes over the table and over one bit
// per page, too little for more than a workgroup while its answers depend on each
// other, so that is one launch of one workgroup, its bits in LDS; the copies, whose
// number the device alone knows, are a second one of as many workgroups as fill the
// GPU, each taking 16 KB at a time.
//
// Measured: 32 beams of 100 to 1500 rows go on from others, 16 layers of 8 heads of 64 bf16
// values 11.0 us, of which the plan is 7 to 8; 12 sequences get private copies of 2000 to 7000
// shared rows, 4 layers of 8 heads of 128 e4m3 values, 0.49 GB both ways 89 us, 5.5 TB/s (part of
// it in the caches); 32 compacted sequences, 0.98 GB 202 us, 4.8 TB/s, where a 4 GiB copy
// reaches 4.67.
#include "cache_internal.h"

namespace sherry {
namespace {

constexpr int kThreads = 1024, kPlanWaves = kThreads / 64;
constexpr int kSeqs = 1024;          // sequences whose place is kept in LDS
constexpr int kLdsWords = 10 * 1024;  // words of bits that are
constexpr int kLdsSmall = 24 * 1024;  // bytes of bits and last places that are in LDS beside the free pages
constexpr int kDeep = 4;             // strips of 64 entries in flight per wave
constexpr int kChunk = 16384;        // bytes that a workgroup copies at once
// (with 512 / 1024 / 2048 / 4096: 12 forked sequences 116 / 96 / 88 / 92 us, 32 compacted
// 250 / 213 / 202 / 202)
constexpr int kCopyGroups = 256 * 8;

struct Meta {
  int copies, live, ones_before_live;
};

struct Pages {
  Cache c;
  const int32_t* parent;
  const int32_t* length;
  const int32_t* add;
  const int32_t* from;
  int32_t* table_out;
  int32_t* length_out;
  int32_t* missing;
  int32_t* moved;
  int32_t* live;
  // workspace
  Meta* meta;
  int2* pairs;       // copies: from, to
  int32_t* free;     // fork: free pages in order; compact: pages in use before each word
  uint32_t* bits;    // fork: bits that are not in LDS; compact: pages in use
  int32_t* last;     // fork: the last place of a page, + 1
  int words;         // of one bit per page
  uint32_t entries;  // batch * width
  FastDiv by_width;
  int64_t layer_bytes, scale_layer_bytes, page_stride_bytes;
  int64_t page_bytes, scale_bytes, chunks;
  int layers;
};

// A sequence of the new table: the row of the old one that it goes on from, how many
// of its entries there are pages, and which entries [lo, hi) will be written.
struct Seq {
  int parent, pages, lo, hi, n;
};
__device__ __forceinline__ Seq seq_of(const Pages& a, int b) {
  const int p = a.parent ? as_global(a.parent)[b] : b;
  Seq s{p >= 0 && p < a.c.batch ? p : -1, 0, 0, 0, 0};
  s.n = s.parent < 0 ? 0 : a.c.length(a.length, s.parent);
  const int add = a.add ? as_global(a.add)[b] : 0;
  const uint32_t all = static_cast<uint32_t>(s.n) + static_cast<uint32_t>(add > 0 ? add : 0);
  const int total = all < static_cast<uint32_t>(a.c.rows) ? static_cast<int>(all) : a.c.rows;
  int begin = s.n;
  if (a.from) {
    const int f = as_global(a.from)[b];
    begin = f < 0 ? 0 : f < s.n ? f : s.n;
  }
  auto up = [&](int n) { return n > 0 ? static_cast<int>(a.c.by_page.div(n - 1)) + 1 : 0; };
  s.pages = up(s.n);
  if (total > begin) {
    s.lo = static_cast<int>(a.c.by_page.div(begin));
    s.hi = up(total);
  }
  return s;
}

// One bit per page, in LDS or in the workspace (read and written by one workgroup).
template <bool LDS>
struct Bits {
  uint32_t* w;
  __device__ __forceinline__ uint32_t set(int page) const {  // what the word was
    const uint32_t bit = 1u << (page & 31);
    if constexpr (LDS) return atomicOr(w + (page >> 5), bit) & bit;
    else return __hip_atomic_fetch_or(w + (page >> 5), bit, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) & bit;
  }
  __device__ __forceinline__ uint32_t word(int i) const {
    if constexpr (LDS) return w[i];
    else return __hip_atomic_load(w + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __device__ __forceinline__ void clear(int i) const {
    if constexpr (LDS) w[i] = 0;
    else __hip_atomic_store(w + i, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __device__ __forceinline__ bool operator[](int page) const { return (word(page >> 5) >> (page & 31)) & 1; }
};

// The last place of a page, + 1, in LDS or in the workspace (as Bits).
template <bool LDS>
struct Last {
  int32_t* p;
  __device__ __forceinline__ void clear(int page) const {
    if constexpr (LDS) p[page] = 0;
    else __hip_atomic_store(p + page, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __device__ __forceinline__ void raise(int page, int v) const {
    if constexpr (LDS) atomicMax(p + page, v);
    else __hip_atomic_fetch_max(p + page, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __device__ __forceinline__ int operator[](int page) const {
    if constexpr (LDS) return p[page];
    else return __hip_atomic_load(p + page, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
};

// Sums of v over the threads before this one, and over all.
struct Scan {
  int before, all;
};
__device__ __forceinline__ Scan block_scan(int v, int (&sums)[kPlanWaves]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int upto = wave_scan(v);
  __syncthreads();  // (sums of a scan before)
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  int before = upto - v, all = 0;
#pragma unroll
  for (int i = 0; i < kPlanWaves; ++i) {
    const int s = sums[i];
    if (i < wave) before += s;
    all += s;
  }
  return Scan{before, all};
}

// An entry of the new table.
struct Entry {
  uint32_t flat;
  int page;  // -1: none yet
  bool mine;
};

// The entries that this wave has: its share of the table, kDeep strips of 64 at a time.
// Once: they are no more than kDeep strips a wave, and stay in registers from one pass to
// the next (32 beams of up to 94 places 11.4 us in all against 15.6 with every pass over memory,
// 12 private prompts of up to 219 88 against 95).
template <bool ONCE, class Info>
struct Entries {
  const Pages& a;
  const Info& info;
  uint32_t s0, s1;
  Entry kept[kDeep];
  __device__ __forceinline__ Entries(const Pages& args, const Info& i) : a(args), info(i) {
    const uint32_t wave = threadIdx.x >> 6, strips = (a.entries + 63) / 64;
    const uint32_t share = (strips + kPlanWaves - 1) / kPlanWaves;
    s0 = wave * share;
    s1 = s0 + share < strips ? s0 + share : strips;
  }
  __device__ __forceinline__ void read(uint32_t s) {
#pragma unroll
    for (int i = 0; i < kDeep; ++i) {
      kept[i] = Entry{(s + i) * 64 + (threadIdx.x & 63), -1, false};
      if (s + i >= s1 || kept[i].flat >= a.entries) {
        kept[i].flat = ~0u;
        continue;
      }
      const int b = static_cast<int>(a.by_width.div(kept[i].flat));
      const int j = static_cast<int>(kept[i].flat - uint32_t(b) * a.c.width);
      const Seq q = info(b);
      kept[i].mine = j >= q.lo && j < q.hi;
      if (j < q.pages) kept[i].page = as_global(a.c.table)[int64_t(q.parent) * a.c.width + j];
    }
#pragma unroll
    for (int i = 0; i < kDeep; ++i)
      if (static_cast<uint32_t>(kept[i].page) >= static_cast<uint32_t>(a.c.pages)) kept[i].page = -1;
  }
  template <class F>
  __device__ __forceinline__ void each(F&& f) {
    if constexpr (ONCE) {
#pragma unroll
      for (int i = 0; i < kDeep; ++i) f(kept[i]);
    } else {
      for (uint32_t s = s0; s < s1; s += kDeep) {
        read(s);
#pragma unroll
        for (int i = 0; i < kDeep; ++i) f(kept[i]);
      }
    }
  }
  __device__ __forceinline__ void begin() {  // (after info is there)
    if constexpr (ONCE) read(s0);
  }
};

struct InfoOf {
  const Pages& a;
  const Seq* kept;
  __device__ __forceinline__ Seq operator()(int b) const { return b < kSeqs ? kept[b] : seq_of(a, b); }
};
__device__ __forceinline__ void keep_info(const Pages& a, Seq* kept) {
  for (int b = threadIdx.x; b < kSeqs && b < a.c.batch; b += kThreads) kept[b] = seq_of(a, b);
}

extern __shared__ uint32_t lds_bits[];

// ONCE: the entries stay in registers, and with LDS free pages and the places of shared ones
// in LDS too.
template <bool LDS, bool ONCE>
__global__ __launch_bounds__(kThreads) void fork_plan_kernel(Pages a) {
  __shared__ Seq kept[kSeqs];
  __shared__ int sums[kPlanWaves], needs[kPlanWaves], copies[kPlanWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  __shared__ int32_t free_lds[ONCE ? kThreads * kDeep : 1];
  uint32_t* base = LDS ? lds_bits : a.bits;
  // pages that the new table has, has more than once, and has where it is not written
  const Bits<LDS> used{base}, more{base + a.words}, other{base + 2 * a.words};
  const Last<LDS && ONCE> last{LDS && ONCE ? reinterpret_cast<int32_t*>(base + 3 * a.words) : a.last};
  for (int i = threadIdx.x; i < 3 * a.words; i += kThreads) Bits<LDS>{base}.clear(i);
  keep_info(a, kept);
  const InfoOf info{a, kept};
  __syncthreads();
  Entries<ONCE, InfoOf> entries(a, info);
  entries.begin();
  entries.each([&](const Entry& e) {
    if (e.page < 0) return;
    if (used.set(e.page)) more.set(e.page);
    if (!e.mine) other.set(e.page);
  });
  __syncthreads();
  // where all places of a shared page are written, the last of them keeps it
  auto contended = [&](const Entry& e) { return e.page >= 0 && e.mine && more[e.page] && !other[e.page]; };
  bool any = false;
  entries.each([&](const Entry& e) {
    if (!contended(e)) return;
    any = true;
    last.clear(e.page);
  });
  if (__syncthreads_or(any)) {
    entries.each([&](const Entry& e) {
      if (contended(e)) last.raise(e.page, static_cast<int>(e.flat) + 1);
    });
    __syncthreads();
  }
  auto need = [&](const Entry& e) {
    if (!e.mine) return false;
    if (e.page < 0) return true;
    if (!more[e.page]) return false;
    if (other[e.page]) return true;
    return last[e.page] != static_cast<int>(e.flat) + 1;
  };
  int n = 0, nc = 0;  // (uniform over the wave)
  entries.each([&](const Entry& e) {
    const bool y = need(e);
    n += __builtin_popcountll(__ballot(y));
    nc += __builtin_popcountll(__ballot(y && e.page >= 0));
  });
  if (lane == 0) {
    needs[wave] = n;
    copies[wave] = nc;
  }
  // free pages, by words in order
  const int per = (a.words + kThreads - 1) / kThreads;
  const int w0 = static_cast<int>(threadIdx.x) * per, w1 = w0 + per < a.words ? w0 + per : a.words;
  auto free_bits = [&](int i) {
    const int left = a.c.pages - 32 * i;
    return ~used.word(i) & (left < 32 ? (1u << left) - 1 : ~0u);
  };
  int mine = 0;
  for (int i = w0; i < w1; ++i) mine += __builtin_popcount(free_bits(i));
  const Scan free = block_scan(mine, sums);
  int all = 0, before = 0, all_copies = 0, copies_before = 0;
#pragma unroll
  for (int i = 0; i < kPlanWaves; ++i) {
    if (i < wave) {
      before += needs[i];
      copies_before += copies[i];
    }
    all += needs[i];
    all_copies += copies[i];
  }
  const int missing = all > free.all ? all - free.all : 0;
  if (threadIdx.x == 0) {
    as_global_mut(a.missing)[0] = missing;
    as_global_mut(&a.meta->copies)[0] = missing ? 0 : all_copies;
  }
  if (missing) return;
  int rank = free.before;
  for (int i = w0; i < w1 && rank < all; ++i)
    for (uint32_t f = free_bits(i); f && rank < all; f &= f - 1) {
      const int page = 32 * i + __builtin_ctz(f);
      if constexpr (ONCE) free_lds[rank++] = page;
      else as_global_mut(a.free)[rank++] = page;
    }
  __syncthreads();
  entries.each([&](const Entry& e) {
    const bool y = need(e), c = y && e.page >= 0;
    const uint64_t ys = __ballot(y), cs = __ballot(c), below = (1ull << lane) - 1;
    int to = e.page;
    if (y) {
      const int i = before + __builtin_popcountll(ys & below);
      to = ONCE ? free_lds[i] : as_global(a.free)[i];
    }
    if (c) as_global_mut(a.pairs)[copies_before + __builtin_popcountll(cs & below)] = make_int2(e.page, to);
    before += __builtin_popcountll(ys);
    copies_before += __builtin_popcountll(cs);
    if (e.flat != ~0u) as_global_mut(a.table_out)[e.flat] = to;
  });
  for (int b = threadIdx.x; b < a.c.batch; b += kThreads) as_global_mut(a.length_out)[b] = info(b).n;
}

template <bool LDS>
__global__ __launch_bounds__(kThreads) void compact_plan_kernel(Pages a) {
  __shared__ Seq kept[kSeqs];
  __shared__ int sums[kPlanWaves];
  __shared__ int ones_before_live;
  const Bits<LDS> used{LDS ? lds_bits : a.bits};
  for (int i = threadIdx.x; i < a.words; i += kThreads) used.clear(i);
  keep_info(a, kept);
  __syncthreads();
  const InfoOf info{a, kept};
  Entries<false, InfoOf> entries(a, info);
  entries.each([&](const Entry& e) {
    if (e.page >= 0) used.set(e.page);
  });
  __syncthreads();
  const int per = (a.words + kThreads - 1) / kThreads;
  const int w0 = static_cast<int>(threadIdx.x) * per, w1 = w0 + per < a.words ? w0 + per : a.words;
  int mine = 0;
  for (int i = w0; i < w1; ++i) mine += __builtin_popcount(used.word(i));
  const Scan ones = block_scan(mine, sums);
  const int live = ones.all;
  // holes before `live`, in order; the pages in use before each word, and before live
  int rank = ones.before;
  if (threadIdx.x == 0) ones_before_live = live;  // (all pages are in use)
  __syncthreads();
  for (int i = w0; i < w1; ++i) {
    const uint32_t u = used.word(i);
    as_global_mut(a.free)[i] = rank;
    if constexpr (LDS) as_global_mut(a.bits)[i] = u;
    const int left = live - 32 * i;  // pages of the word that lie before live
    if (left >= 0 && left < 32) ones_before_live = rank + __builtin_popcount(u & ((1u << left) - 1));
    if (left > 0)
      for (uint32_t f = ~u & (left < 32 ? (1u << left) - 1 : ~0u); f; f &= f - 1) {
        const int p = 32 * i + __builtin_ctz(f);
        as_global_mut(a.pairs)[p - rank - __builtin_popcount(u & ((1u << (p & 31)) - 1))].y = p;
      }
    rank += __builtin_popcount(u);
  }
  __syncthreads();
  const int before_live = ones_before_live;
  rank = ones.before;
  for (int i = w0; i < w1; ++i) {
    const uint32_t u = used.word(i);
    const int left = live - 32 * i;
    if (left < 32)
      for (uint32_t f = left > 0 ? u & (~0u << left) : u; f; f &= f - 1) {
        const int p = 32 * i + __builtin_ctz(f);
        as_global_mut(a.pairs)[rank + __builtin_popcount(u & ((1u << (p & 31)) - 1)) - before_live].x = p;
      }
    rank += __builtin_popcount(u);
  }
  if (threadIdx.x == 0) {
    as_global_mut(a.live)[0] = live;
    as_global_mut(&a.meta->copies)[0] = live - before_live;
    as_global_mut(&a.meta->live)[0] = live;
    as_global_mut(&a.meta->ones_before_live)[0] = before_live;
  }
}

// Copies the pairs' pages, in every layer, K and V, with their scales.
__device__ __forceinline__ void copy_pages(const Pages& a, uint32_t group, uint32_t groups) {
  const uint64_t per = a.chunks;  // of a page, of K or V, in one layer
  const uint64_t all = static_cast<uint64_t>(as_const(&a.meta->copies)[0]) * a.layers * 2 * per;
  for (uint64_t u = group; u < all; u += groups) {
    const uint64_t page = u / per;
    const int64_t chunk = u - page * per;
    const uint64_t pl = page >> 1;  // pair and layer; K and V take turns
    const int pair = static_cast<int>(pl / a.layers);
    const int layer = static_cast<int>(pl - uint64_t(pair) * a.layers);
    const bool is_k = (page & 1) == 0;
    const int from = as_const(&a.pairs[pair].x)[0], to = as_const(&a.pairs[pair].y)[0];
    char* pool = (is_k ? a.c.k : a.c.v) + layer * a.layer_bytes;
    const char* src = pool + from * a.page_stride_bytes;
    char* dst = pool + to * a.page_stride_bytes;
    const int64_t at = chunk * kChunk + 16 * threadIdx.x;
    u32x4 x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (at + 4096 * i < a.page_bytes)
        x[i] = *reinterpret_cast<const SHERRY_GLOBAL u32x4*>(as_global(src) + at + 4096 * i);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (at + 4096 * i < a.page_bytes)
        *reinterpret_cast<SHERRY_GLOBAL u32x4*>(as_global_mut(dst) + at + 4096 * i) = x[i];
    if (chunk == 0 && a.scale_bytes) {
      char* scales = reinterpret_cast<char*>(is_k ? a.c.ks : a.c.vs) + layer * a.scale_layer_bytes;
      const float* s = reinterpret_cast<const float*>(scales + from * a.scale_bytes);
      float* d = reinterpret_cast<float*>(scales + to * a.scale_bytes);
      for (int64_t i = threadIdx.x; i < a.scale_bytes / 4; i += 256) as_global_mut(d)[i] = as_global(s)[i];
    }
  }
}

__global__ __launch_bounds__(256) void copy_kernel(Pages a) { copy_pages(a, blockIdx.x, gridDim.x); }

// Copies; and every workgroup a share of the pages' new places and of the table.
__global__ __launch_bounds__(256) void move_kernel(Pages a) {
  const int live = as_const(&a.meta->live)[0], before_live = as_const(&a.meta->ones_before_live)[0];
  auto place = [&](int p) {  // -1: free
    const uint32_t u = as_global(a.bits)[p >> 5], bit = 1u << (p & 31);
    if (!(u & bit)) return -1;
    if (p < live) return p;
    return as_global(&a.pairs[as_global(a.free)[p >> 5] + __builtin_popcount(u & (bit - 1)) - before_live].y)[0];
  };
  const uint32_t t = blockIdx.x * 256 + threadIdx.x, step = gridDim.x * 256;
  if (a.moved)
    for (uint32_t p = t; p < static_cast<uint32_t>(a.c.pages); p += step)
      as_global_mut(a.moved)[p] = place(static_cast<int>(p));
  for (uint32_t f = t; f < a.entries; f += step) {
    const int b = static_cast<int>(a.by_width.div(f)), j = static_cast<int>(f - uint32_t(b) * a.c.width);
    const int n = a.c.length(a.length, b);
    int p = -1;
    if (n > 0 && j <= static_cast<int>(a.c.by_page.div(n - 1))) p = as_global(a.c.table)[f];
    as_global_mut(a.table_out)[f] = static_cast<uint32_t>(p) < static_cast<uint32_t>(a.c.pages) ? place(p) : -1;
  }
  copy_pages(a, blockIdx.x, gridDim.x);
}

struct Layout {
  size_t meta, pairs, free, bits, last;
  int words;
  int64_t most;  // copies
  size_t bytes() const { return meta + pairs + free + bits + last; }
};
inline size_t up(int64_t n) { return static_cast<size_t>((n + 255) / 256 * 256); }
Layout fork_layout(const sherry_cache_desc& c) {
  const int64_t entries = int64_t(c.batch) * c.table_width;
  Layout l{};
  l.words = static_cast<int>(ceil_div(c.pages, 32));
  l.most = entries < c.pages ? entries : c.pages;
  l.meta = up(sizeof(Meta));
  l.pairs = up(8 * l.most);
  l.free = up(4 * l.most);
  l.bits = 3 * int64_t(l.words) <= kLdsWords ? 0 : up(12 * int64_t(l.words));
  l.last = up(4 * int64_t(c.pages));
  return l;
}
Layout compact_layout(const sherry_cache_desc& c) {
  const int64_t entries = int64_t(c.batch) * c.table_width;
  Layout l{};
  l.words = static_cast<int>(ceil_div(c.pages, 32));
  l.most = entries < c.pages / 2 ? entries : c.pages / 2;  // (a place for each before live)
  l.meta = up(sizeof(Meta));
  l.pairs = up(8 * l.most);
  l.free = up(4 * int64_t(l.words));
  l.bits = up(4 * int64_t(l.words));
  return l;
}

template <class D>
Pages pages_of(const sherry_cache_desc& c, const D& d, const Layout& l) {
  Pages a{};
  a.c = cache_of(c);
  const int64_t e = type_bytes(c.type);
  a.length = d.length;
  a.table_out = d.table_out;
  char* ws = static_cast<char*>(d.workspace);
  a.meta = reinterpret_cast<Meta*>(ws);
  a.pairs = reinterpret_cast<int2*>(ws += l.meta);
  a.free = reinterpret_cast<int32_t*>(ws += l.pairs);
  a.bits = reinterpret_cast<uint32_t*>(ws += l.free);
  a.last = reinterpret_cast<int32_t*>(ws += l.bits);
  a.words = l.words;
  a.entries = static_cast<uint32_t>(int64_t(c.batch) * c.table_width);
  a.by_width = FastDiv::of(static_cast<uint32_t>(c.table_width));
  a.layer_bytes = d.layers > 1 ? d.layer_stride * e : 0;
  a.scale_layer_bytes = d.layers > 1 ? d.scale_layer_stride * 4 : 0;
  a.page_stride_bytes = a.c.page_stride * e;
  a.page_bytes = int64_t(c.kv_heads) * c.page_size * c.head_dim * e;
  a.scale_bytes = c.k_scale ? int64_t(c.kv_heads) * (c.type == SHERRY_F8 ? 1 : c.page_size) * 4 : 0;
  a.layers = d.layers;
  a.chunks = ceil_div(a.page_bytes, kChunk);
  return a;
}
// Workgroups of the copying launch.
unsigned copy_groups(const Pages& a, const Layout& l) {
  const double most = double(l.most) * a.layers * 2 * double(a.chunks);
  return most < 1 ? 1u : most < kCopyGroups ? static_cast<unsigned>(most) : unsigned(kCopyGroups);
}

}  // namespace

size_t fork_workspace(const sherry_cache_desc& c, const sherry_fork_desc&) { return fork_layout(c).bytes(); }

int launch_fork(const sherry_cache_desc& c, const sherry_fork_desc& d, hipStream_t s) {
  const Layout l = fork_layout(c);
  Pages a = pages_of(c, d, l);
  a.parent = d.parent;
  a.add = d.add;
  a.from = d.from_row;
  a.length_out = d.length_out;
  a.missing = d.missing;
  const bool once = a.entries <= kThreads * kDeep;
  const size_t bits = 12u * l.words, last = 4u * static_cast<size_t>(c.pages);
  const int rc = !l.bits && once && bits + last <= kLdsSmall
                     ? launch(fork_plan_kernel<true, true>, dim3(1), dim3(kThreads), bits + last, s, a)
                 : l.bits ? launch(fork_plan_kernel<false, false>, dim3(1), dim3(kThreads), 0, s, a)
                          : launch(fork_plan_kernel<true, false>, dim3(1), dim3(kThreads), bits, s, a);
  if (rc != SHERRY_OK) return rc;
  return launch(copy_kernel, dim3(copy_groups(a, l)), dim3(256), 0, s, a);
}

size_t compact_workspace(const sherry_cache_desc& c, const sherry_compact_desc&) { return compact_layout(c).bytes(); }

int launch_compact(const sherry_cache_desc& c, const sherry_compact_desc& d, hipStream_t s) {
  const Layout l = compact_layout(c);
  Pages a = pages_of(c, d, l);
  a.moved = d.moved;
  a.live = d.live;
  const int rc = l.words > kLdsWords ? launch(compact_plan_kernel<false>, dim3(1), dim3(kThreads), 0, s, a)
                                     : launch(compact_plan_kernel<true>, dim3(1), dim3(kThreads), 4u * l.words, s, a);
  if (rc != SHERRY_OK) return rc;
  // (the table and the pages' places: one workgroup per 1024 of them)
  const int64_t most = ceil_div(int64_t(a.entries) + c.pages, 1024), groups = copy_groups(a, l);
  return launch(move_kernel, dim3(static_cast<unsigned>(groups > most ? groups : most < kCopyGroups ? most : kCopyGroups)),
                dim3(256), 0, s, a);
}

}  // namespace sherry
