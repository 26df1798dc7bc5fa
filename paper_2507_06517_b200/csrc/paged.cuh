// What the kernels of the 8-bit paged cache share: device-side copies of the pool and the table, and the checks of both.
#pragma once

#include "args.cuh"
#include "common.cuh"

namespace skv {

constexpr int kPagedBlock = SPINDLEKV_PAGED_BLOCK;   // tokens that share a scale
constexpr int kPagedMaxUnits = 8192;                 // (layer, sequence) pairs of one call
constexpr int kPagedMaxPages = 1 << 20;                // sums of 1024 sequences' page numbers fit 32 bits

struct Pool {
  uint8_t *kc, *vc;
  float *ks, *vs;
  int32_t* ref;
  int n_pages, ps, heads, d;
  __host__ __device__ int per_page() const { return ps / kPagedBlock; }   // blocks of a page
};

struct Table {
  int32_t *pages, *lens;
  int n_layers, n_seqs, max_pages;
};

inline Pool make_pool(const spindlekv_page_pool& p) {
  return Pool{static_cast<uint8_t*>(p.k_codes), static_cast<uint8_t*>(p.v_codes), p.k_scale, p.v_scale, p.page_ref,
              p.n_pages, p.page_size, p.n_kv_heads, p.head_dim};
}
inline Table make_table(const spindlekv_page_table& t) { return Table{t.pages, t.lens, t.n_layers, t.n_seqs, t.max_pages}; }

// length of unit `u` = layer * n_seqs + seq, never more than its row of the table can hold
__device__ __forceinline__ int unit_len(const Table& t, const Pool& p, int u) {
  return (int)min((long long)max(t.lens[u], 0), (long long)t.max_pages * p.ps);
}

inline spindlekv_status pool_table_status(const spindlekv_page_pool* p, const spindlekv_page_table* t) {
  if (!p || !t) return SPINDLEKV_INVALID_ARG;
  if (!p->k_codes || !p->v_codes || !p->k_scale || !p->v_scale || !p->page_ref || !t->pages || !t->lens) return SPINDLEKV_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(p->k_codes) | reinterpret_cast<uintptr_t>(p->v_codes)) % 16) return SPINDLEKV_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(p->k_scale) | reinterpret_cast<uintptr_t>(p->v_scale) | reinterpret_cast<uintptr_t>(p->page_ref) |
       reinterpret_cast<uintptr_t>(t->pages) | reinterpret_cast<uintptr_t>(t->lens)) % 4)
    return SPINDLEKV_INVALID_ARG;
  if (p->n_pages <= 0 || p->n_kv_heads <= 0 || t->n_layers <= 0 || t->n_seqs <= 0 || t->max_pages <= 0) return SPINDLEKV_INVALID_ARG;
  if (p->page_size != 16 && p->page_size != 32 && p->page_size != 64 && p->page_size != 128) return SPINDLEKV_UNSUPPORTED;
  if (p->head_dim != 64 && p->head_dim != 128) return SPINDLEKV_UNSUPPORTED;
  if (p->format != SPINDLEKV_PAGED_INT8 && p->format != SPINDLEKV_PAGED_E4M3) return SPINDLEKV_UNSUPPORTED;
  if ((int64_t)t->n_layers * t->n_seqs > kPagedMaxUnits || p->n_kv_heads > 1024) return SPINDLEKV_UNSUPPORTED;
  if (p->n_pages > kPagedMaxPages) return SPINDLEKV_UNSUPPORTED;
  if ((int64_t)t->max_pages * p->page_size > 0x7FFFFF00) return SPINDLEKV_UNSUPPORTED;   // positions are 32-bit
  return SPINDLEKV_OK;
}

}  // namespace skv
