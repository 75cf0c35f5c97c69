// Where a sequence's rows lie in the pool of pages.  Plain C++ so that a host program can try every row, table entry and pool
// at its limits (tests/host/page_row_check.cpp).
#pragma once
#include <stdint.h>
#ifndef __HIPCC__
#define __host__
#define __device__
#endif

struct PcPages {
  void* k;                        // [n_pages, H_kv, page, D], bf16 or (scales given) E4M3 codes with a scale a row
  void* v;
  float* k_scale;                 // [n_pages, H_kv, page] or nullptr
  float* v_scale;
  const int32_t* table;           // [B, max_pages]
  int n_pages, shift, max_pages;  // page = 1 << shift
};
// Entry of the table that row `row` needs; -1: there is none
__host__ __device__ inline int pc_page_entry(const PcPages& p, long long row) {
  return row < 0 || row >> p.shift >= p.max_pages ? -1 : (int)(row >> p.shift);
}
// The row as one of the pool ([n_pages, H_kv, page] flattened) for KV head g, given its page; -1: no page of the pool
__host__ __device__ inline long long pc_pool_row(const PcPages& p, int page, long long row, int g, int n_kv_heads) {
  if ((uint32_t)page >= (uint32_t)p.n_pages) return -1;
  return (((long long)page * n_kv_heads + g) << p.shift) + (row & ((1 << p.shift) - 1));
}
__host__ __device__ inline long long pc_page_row(const PcPages& p, long long b, long long row, int g, int n_kv_heads) {
  const int at = pc_page_entry(p, row);
  return at < 0 ? -1 : pc_pool_row(p, p.table[b * p.max_pages + at], row, g, n_kv_heads);
}
