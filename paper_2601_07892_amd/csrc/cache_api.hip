// C ABI entry points of the paged key-value cache: argument validation.
// Every check happens on the host before anything is enqueued.
#include "cache_internal.h"

using namespace sherry;

// The descriptor layouts are part of the ABI (Python and C callers build them).
static_assert(sizeof(sherry_cache_desc) == 80, "sherry_cache_desc layout");
static_assert(sizeof(sherry_append_desc) == 152, "sherry_append_desc layout");
static_assert(sizeof(sherry_attend_desc) == 120, "sherry_attend_desc layout");
static_assert(sizeof(sherry_evict_desc) == 88, "sherry_evict_desc layout");

namespace {

constexpr int kMaxHeads = 4096, kMaxBatch = 65535, kMaxGroup = 256;

inline bool aligned(const void* p, uintptr_t a) {
  return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0;  // (NULL is)
}

inline bool float_type(int t) { return t == SHERRY_F32 || t == SHERRY_F16 || t == SHERRY_BF16; }

int check_cache(const sherry_cache_desc* c) {
  if (!c || !c->k || !c->v || !c->table) return SHERRY_E_INVALID;
  if (c->type != SHERRY_F16 && c->type != SHERRY_BF16 && c->type != SHERRY_I8) return SHERRY_E_INVALID;
  const bool i8 = c->type == SHERRY_I8;
  if (i8 != (c->k_scale != nullptr) || i8 != (c->v_scale != nullptr)) return SHERRY_E_INVALID;
  const int whole = i8 ? 16 : 8;
  if (c->pages < 1 || c->kv_heads < 1 || c->kv_heads > kMaxHeads || c->page_size < 1 ||
      c->head_dim < whole || c->head_dim > SHERRY_MAX_HEAD_DIM || c->head_dim % whole != 0 ||
      c->batch < 1 || c->batch > kMaxBatch || c->table_width < 1 ||
      int64_t(c->table_width) * c->page_size > SHERRY_MAX_CACHE_ROWS)
    return SHERRY_E_SHAPE;
  if (c->page_stride != 0 && (c->page_stride % whole != 0 ||
                              c->page_stride < int64_t(c->kv_heads) * c->page_size * c->head_dim))
    return SHERRY_E_SHAPE;
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->k_scale, 16) ||
      !aligned(c->v_scale, 16) || !aligned(c->table, 4))
    return SHERRY_E_ALIGN;
  return SHERRY_OK;
}
int64_t cache_rows(const sherry_cache_desc* c) { return int64_t(c->table_width) * c->page_size; }

int check_append(const sherry_cache_desc* c, const sherry_append_desc* a) {
  int st = check_cache(c);
  if (st != SHERRY_OK) return st;
  if (!a || !a->k || !a->v || !a->seq || !a->slot || !a->pos || !float_type(a->type) ||
      (a->q != nullptr) != (a->q_out != nullptr) || (a->cos != nullptr) != (a->sin != nullptr) ||
      (a->pairing != SHERRY_ROPE_HALVES && a->pairing != SHERRY_ROPE_PAIRS))
    return SHERRY_E_INVALID;
  if (a->tokens < 1 || a->tokens > SHERRY_MAX_M) return SHERRY_E_SHAPE;
  if (a->q && (a->heads < 1 || a->heads > kMaxHeads * kMaxGroup)) return SHERRY_E_SHAPE;
  if (a->cos && (a->rope_rows < 1 || a->rot_dim < 2 || a->rot_dim % 2 != 0 || a->rot_dim > c->head_dim))
    return SHERRY_E_SHAPE;
  if ((a->weight || a->position) && a->row_stride < cache_rows(c)) return SHERRY_E_SHAPE;
  const int64_t row = int64_t(c->kv_heads) * c->head_dim;
  const int64_t qrow = a->q ? int64_t(a->heads) * c->head_dim : 0;
  if ((a->k_stride && a->k_stride < row) || (a->v_stride && a->v_stride < row) ||
      (a->q && ((a->q_stride && a->q_stride < qrow) || (a->q_out_stride && a->q_out_stride < qrow))))
    return SHERRY_E_SHAPE;
  // in place every token's row has to lie where it is read: another stride would
  // write rows that other workgroups have yet to read
  if (a->q && a->q_out == a->q && a->tokens > 1 &&
      (a->q_stride ? a->q_stride : qrow) != (a->q_out_stride ? a->q_out_stride : qrow))
    return SHERRY_E_SHAPE;
  if (!fits_grid(append_threads(*c, *a))) return SHERRY_E_SHAPE;
  const uintptr_t e = static_cast<uintptr_t>(type_bytes(a->type));
  if (!aligned(a->q, e) || !aligned(a->k, e) || !aligned(a->v, e) || !aligned(a->q_out, e) ||
      !aligned(a->seq, 4) || !aligned(a->slot, 4) || !aligned(a->pos, 4) || !aligned(a->cos, 4) ||
      !aligned(a->sin, 4) || !aligned(a->weight, 4) || !aligned(a->position, 4))
    return SHERRY_E_ALIGN;
  return SHERRY_OK;
}

// Everything but the pointers' alignment and the workspace.
int check_attend_shape(const sherry_cache_desc* c, const sherry_attend_desc* a) {
  int st = check_cache(c);
  if (st != SHERRY_OK) return st;
  if (!a || !float_type(a->type) || a->window < 0) return SHERRY_E_INVALID;
  if (!(a->scale > -__builtin_huge_valf() && a->scale < __builtin_huge_valf())) return SHERRY_E_INVALID;
  if (a->position && a->window && !a->q_pos) return SHERRY_E_INVALID;
  if (a->heads < c->kv_heads || a->heads % c->kv_heads != 0 || a->heads / c->kv_heads > kMaxGroup)
    return SHERRY_E_SHAPE;
  const int64_t row = int64_t(a->heads) * c->head_dim;
  if (a->q_stride % 8 != 0 || a->out_stride % 8 != 0 || (a->q_stride && a->q_stride < row) ||
      (a->out_stride && a->out_stride < row))
    return SHERRY_E_SHAPE;
  if ((a->mask && a->mask_stride < cache_rows(c)) ||
      ((a->position || a->weight) && a->row_stride < cache_rows(c)))
    return SHERRY_E_SHAPE;
  // (all rows in tiles of 32, and up to 16 more per sequence, are counted in 31 bits)
  if (int64_t(c->batch) * (ceil_div(cache_rows(c), 32) + 16) > INT32_MAX) return SHERRY_E_SHAPE;
  if (!fits_grid(attend_threads(*c, *a))) return SHERRY_E_SHAPE;
  return SHERRY_OK;
}

int check_evict(const sherry_cache_desc* c, const sherry_evict_desc* a) {
  int st = check_cache(c);
  if (st != SHERRY_OK) return st;
  if (!a || !a->length || !a->weight || !a->length_out || !a->kept || a->length_out == a->length)
    return SHERRY_E_INVALID;
  if (a->keep < 1 || a->keep > SHERRY_MAX_CACHE_ROWS || a->row_stride < cache_rows(c) ||
      a->out_stride < a->keep)
    return SHERRY_E_SHAPE;
  if (!fits_grid(evict_threads(*c, *a))) return SHERRY_E_SHAPE;
  if (!aligned(a->length, 4) || !aligned(a->weight, 4) || !aligned(a->position, 4) ||
      !aligned(a->recent_from, 4) || !aligned(a->length_out, 4) || !aligned(a->kept, 4) ||
      !aligned(a->weight_out, 4) || !aligned(a->position_out, 4))
    return SHERRY_E_ALIGN;
  return SHERRY_OK;
}

}  // namespace

extern "C" int sherry_cache_append(const sherry_cache_desc* cache, const sherry_append_desc* args,
                                   void* stream) {
  const int st = check_append(cache, args);
  return st != SHERRY_OK ? st : launch_append(*cache, *args, static_cast<hipStream_t>(stream));
}

extern "C" size_t sherry_cache_attend_workspace(const sherry_cache_desc* cache,
                                                const sherry_attend_desc* args) {
  return check_attend_shape(cache, args) != SHERRY_OK ? 0 : attend_workspace(*cache, *args);
}

extern "C" int sherry_cache_attend(const sherry_cache_desc* cache, const sherry_attend_desc* args,
                                   void* stream) {
  const int st = check_attend_shape(cache, args);
  if (st != SHERRY_OK) return st;
  const sherry_attend_desc& a = *args;
  if (!a.q || !a.out || !a.length || !a.workspace) return SHERRY_E_INVALID;
  if (!aligned(a.q, 16) || !aligned(a.out, 16) || !aligned(a.workspace, 16) || !aligned(a.length, 4) ||
      !aligned(a.position, 4) || !aligned(a.q_pos, 4) || !aligned(a.weight, 4))
    return SHERRY_E_ALIGN;
  if (a.workspace_bytes < attend_workspace(*cache, a)) return SHERRY_E_BUFSIZE;
  return launch_attend(*cache, a, static_cast<hipStream_t>(stream));
}

extern "C" int sherry_cache_evict(const sherry_cache_desc* cache, const sherry_evict_desc* args,
                                  void* stream) {
  const int st = check_evict(cache, args);
  return st != SHERRY_OK ? st : launch_evict(*cache, *args, static_cast<hipStream_t>(stream));
}
