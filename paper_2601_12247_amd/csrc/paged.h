// Keys and values in pages: launchers of pages.hip (tables, slots, stores) and paged_attention.hip.
//
// A cache is [pages][kv heads][tokens a page][d_head]; pages may lie further apart (a stride), what is in one is contiguous.  Table row b
// names the pages of request b in order; the slot of a token is page * tokens a page + place.
#pragma once

#include "common.h"

namespace pvf {

struct PageExtend {
  const int32_t *seq_len, *start, *n_rows, *n_free, *free_pages;
  int32_t *table;
  int32_t B, M, width, table_stride, page_size, free_cap;
  int32_t *seq_len_out, *n_free_out, *cu_rows, *admitted, *place, *pos, *slot;
};
pvf_status launch_page_extend(hipStream_t s, const PageExtend &a);

struct PageTrim {
  const int32_t *seq_len, *keep, *table, *n_free;
  int32_t *free_pages;
  int32_t B, width, table_stride, page_size, free_cap;
  int32_t *seq_len_out, *n_free_out, *place;
};
pvf_status launch_page_trim(hipStream_t s, const PageTrim &a);

struct PageStore {
  const void *qkv;
  const int32_t *pos, *slot;
  void *q_out, *k_cache, *v_cache;
  int64_t qkv_stride, q_stride, k_page_stride, v_page_stride;   // elements
  int32_t M, H, Hkv, dh, n_pages, page_size;
  double log2_theta;
};
pvf_status launch_page_store(hipStream_t s, int dtype, const PageStore &a);

struct PageAttention {
  const void *q, *k_cache, *v_cache;
  const int32_t *table, *seq_len, *cu_rows;                     // cu_rows NULL: row b is request b's
  void *out;
  float *ws;
  int64_t q_stride, out_stride, k_page_stride, v_page_stride;   // elements
  int32_t B, M, H, Hkv, dh, n_pages, page_size, width, table_stride, causal;
  float scale;
};
int64_t page_attention_workspace(int dtype, int B, int M, int H, int Hkv, int dh, int width, int page_size);
pvf_status launch_page_attention(hipStream_t s, int dtype, const PageAttention &a);

}  // namespace pvf
