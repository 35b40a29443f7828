// What the calls of the paged cache share: checks of the descriptor (host), loads and running sums (device).
#pragma once
#include "../../include/lightkv.h"

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace lk {

constexpr int PAGE_MIN_TOKENS = 8, PAGE_MAX_TOKENS = 1024;
constexpr int64_t PAGE_MAX_SEQ = 1ll << 30;   // tokens of a table row: positions and a tile or page beyond them are ints

inline bool aligned_to(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline bool ints_ok(const void *p) { return p && aligned_to(p, 4); }
inline int log2_of(int v) { int l = 0; while ((1 << l) < v) ++l; return l; }

// Sizes and table.
inline lightkv_status check_page_table(const lightkv_pages *p) {
  if (!p || !p->table) return LIGHTKV_ERR_NULL;
  if (p->batch < 1 || p->n_pages < 1 || p->max_pages < 1 || p->page_tokens < 1 || p->table_stride < p->max_pages) return LIGHTKV_ERR_SHAPE;
  if (!aligned_to(p->table, 4) || p->batch > LIGHTKV_PAGED_MAX_BATCH) return LIGHTKV_ERR_UNSUPPORTED;
  if (p->page_tokens < PAGE_MIN_TOKENS || p->page_tokens > PAGE_MAX_TOKENS || (p->page_tokens & (p->page_tokens - 1))) return LIGHTKV_ERR_UNSUPPORTED;
  if ((int64_t)p->n_pages * p->page_tokens >= (1ll << 31) || (int64_t)p->max_pages * p->page_tokens > PAGE_MAX_SEQ) return LIGHTKV_ERR_UNSUPPORTED;
  return LIGHTKV_OK;
}

inline int page_elem_bytes(const lightkv_pages *p) { return p->dtype == LIGHTKV_BF16 ? 2 : 4; }

// Rows [.., heads, head_dim] at `base`: 16-byte pieces.  An axis of one entry has no stride to speak of.
inline lightkv_status check_strided(const void *base, int elem_bytes, int64_t outer, int64_t n_outer, int64_t head, int heads) {
  const int per = 16 / elem_bytes;
  if (!aligned_to(base, 16)) return LIGHTKV_ERR_UNSUPPORTED;
  if ((n_outer > 1 && outer < 0) || (heads > 1 && head < 0)) return LIGHTKV_ERR_SHAPE;
  if ((n_outer > 1 && outer % per) || (heads > 1 && head % per)) return LIGHTKV_ERR_UNSUPPORTED;
  return LIGHTKV_OK;
}

// Bytes from the first element of [n_outer, heads, head_dim] to behind its last one.
inline uint64_t strided_bytes(int elem_bytes, int64_t outer, int64_t n_outer, int64_t head, int heads, int head_dim) {
  if (n_outer < 1) return 0;
  return ((uint64_t)(n_outer > 1 ? outer : 0) * (uint64_t)(n_outer - 1) + (uint64_t)(heads > 1 ? head : 0) * (uint64_t)(heads - 1) + (uint64_t)head_dim) * (uint64_t)elem_bytes;
}

// Whether rows of `run` elements at the given strides (of axes with more than one entry) are apart, axis within axis.
inline bool apart(int64_t run, const int64_t *stride, const int64_t *count, int axes) {
  int64_t extent = run;
  bool done[3] = {};
  for (int k = 0; k < axes; ++k) {
    int next = -1;
    for (int i = 0; i < axes; ++i)
      if (!done[i] && count[i] > 1 && (next < 0 || stride[i] < stride[next])) next = i;
    if (next < 0) break;
    if (stride[next] < extent) return false;
    done[next] = true;
    extent += stride[next] * (count[next] - 1);
  }
  return true;
}

inline bool overlap(const void *a, uint64_t na, const void *b, uint64_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && x < y + nb && y < x + na;
}

// Head sizes, type and pools (either may be missing where need_both is false).
inline lightkv_status check_page_pools(const lightkv_pages *p, bool need_both) {
  const lightkv_status st = check_page_table(p);
  if (st != LIGHTKV_OK) return st;
  if (need_both && (!p->K || !p->V)) return LIGHTKV_ERR_NULL;
  if (p->kv_heads < 1 || p->heads < 1 || p->heads % p->kv_heads) return LIGHTKV_ERR_SHAPE;
  if (p->dtype != LIGHTKV_F32 && p->dtype != LIGHTKV_BF16) return LIGHTKV_ERR_UNSUPPORTED;
  if (p->head_dim != 32 && p->head_dim != 64 && p->head_dim != 128) return LIGHTKV_ERR_UNSUPPORTED;
  if (p->heads > 65535) return LIGHTKV_ERR_UNSUPPORTED;
  const int eb = page_elem_bytes(p);
  const void *pool[2] = {p->K, p->V};
  const int64_t pages[2] = {p->k_page_stride, p->v_page_stride}, toks[2] = {p->k_tok_stride, p->v_tok_stride}, heads[2] = {p->k_head_stride, p->v_head_stride};
  for (int i = 0; i < 2; ++i) {
    if (!pool[i]) continue;
    lightkv_status s = check_strided(pool[i], eb, pages[i], p->n_pages, heads[i], p->kv_heads);
    if (s == LIGHTKV_OK) s = check_strided(pool[i], eb, toks[i], p->page_tokens, heads[i], p->kv_heads);
    if (s != LIGHTKV_OK) return s;
  }
  return LIGHTKV_OK;
}

inline uint64_t pool_bytes(const lightkv_pages *p, int64_t page_stride, int64_t tok_stride, int64_t head_stride) {
  return strided_bytes(page_elem_bytes(p), page_stride, p->n_pages, head_stride, p->kv_heads, p->head_dim)
         + (uint64_t)tok_stride * (uint64_t)(p->page_tokens - 1) * (uint64_t)page_elem_bytes(p);
}

// Whether elements of V's rows, `delta` elements behind K's, are elements of K's rows.  Axes in the order of falling strides, each of them
// wider than what lies inside it (apart()); `stride` holds K's and V's.  Exact where both have the same strides; axes that differ
// count as filled.
inline bool rows_meet(int64_t delta, int64_t run, const int64_t (*stride)[2], const int64_t *count, int axes) {
  int64_t extent[2] = {run, run};
  for (int i = 0; i < axes; ++i)
    for (int k = 0; k < 2; ++k) extent[k] += stride[i][k] * (count[i] - 1);
  if (delta >= extent[0] || -delta >= extent[1]) return false;
  if (axes == 0 || stride[0][0] != stride[0][1]) return true;
  // entry i of K's axis against entry i + d of V's
  const int64_t s = stride[0][0], near = -delta / s;
  for (int64_t d = near - 2; d <= near + 2; ++d)
    if (d > -count[0] && d < count[0] && rows_meet(delta + d * s, run, stride + 1, count + 1, axes - 1)) return true;
  return false;
}

// Whether the pools of keys and values share elements (each of them apart in itself).
inline bool pools_meet(const lightkv_pages *p) {
  const int64_t all[3][2] = {{p->k_page_stride, p->v_page_stride}, {p->k_tok_stride, p->v_tok_stride}, {p->k_head_stride, p->v_head_stride}};
  const int64_t n[3] = {p->n_pages, p->page_tokens, p->kv_heads};
  int64_t stride[3][2], count[3];
  int axes = 0;
  for (int i = 0; i < 3; ++i) {
    if (n[i] < 2) continue;
    int at = axes++;
    for (; at > 0 && stride[at - 1][0] < all[i][0]; --at) {
      stride[at][0] = stride[at - 1][0]; stride[at][1] = stride[at - 1][1]; count[at] = count[at - 1];
    }
    stride[at][0] = all[i][0]; stride[at][1] = all[i][1]; count[at] = n[i];
  }
  const intptr_t bytes = reinterpret_cast<intptr_t>(p->V) - reinterpret_cast<intptr_t>(p->K);
  return rows_meet(bytes / page_elem_bytes(p), p->head_dim, stride, count, axes);
}

// ---- device ----
// Loads and stores of memory that is touched once: they do not stay in the caches.
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
__device__ __forceinline__ uint4 ld16_stream(const char *p) { return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p))); }
__device__ __forceinline__ void st16_stream(char *p, const uint4 &v) { __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), reinterpret_cast<u32x4 *>(p)); }

// Inclusive running result of `op` over the lanes of a wave, for an op with 0 as its neutral element.
template <typename Op> __device__ __forceinline__ int wave_running(int v, Op op) {
  v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false));   // row_shr 1, 2, 4, 8: inside rows of 16 lanes
  v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false));
  v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false));
  v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false));
  v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false));   // lane 15 of a row to the next row: rows 1 and 3
  v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false));   // lane 31 to rows 2 and 3
  return v;
}
__device__ __forceinline__ int wave_running_sum(int v) { return wave_running(v, [](int a, int b) { return a + b; }); }
__device__ __forceinline__ int wave_running_max(int v) { return wave_running(v, [](int a, int b) { return a > b ? a : b; }); }   // (not negative)

}  // namespace lk
