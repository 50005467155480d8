// paged.cuh -- the paged KV cache of the kernel-level entry points: where things stand in it.
//
// pages [n_pages][n_layers][2][n_kv_heads][page][head_dim]: a page is one piece of memory, so that
// copying or moving one is a single long copy, and the rows of a layer, side and head
// in a page (a slab) are another, so that an attention reads whole lines.
#pragma once

#include "kv8.cuh"

namespace ssd {

struct PagedView {
  char* pages;
  int32_t* table;
  int32_t* refs;
  int32_t n_seq, n_pages, max_pages, shift;  // page = 1 << shift
  int32_t n_kv_heads, slab, slabs;           // bytes of a slab, slabs of a page
  size_t bytes;                              // of a page
  __host__ __device__ __forceinline__ int cap() const { return max_pages << shift; }
  // The page of entry i of sequence b, or -1.
  __device__ __forceinline__ int entry(int b, int i) const {
    const int e = __ldg(table + (size_t)b * max_pages + i);
    return (unsigned)e < (unsigned)n_pages ? e : -1;
  }
  // Layer `layer`, side 0 (K) or 1 (V) of page 0, head 0.
  __host__ __device__ __forceinline__ size_t side(int layer, int side) const {
    return (size_t)(layer * 2 + side) * n_kv_heads * slab;
  }
};

// Checks of a cache that every entry point makes; null: fine.
const char* check_paged(const ssd_paged_cache* c, ssd_status* status) noexcept;
PagedView paged_view(const ssd_paged_cache* c) noexcept;

}  // namespace ssd
