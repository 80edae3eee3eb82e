// Keys and values in pages: launchers of pages.hip (tables, slots, stores) and paged_attention.hip.
//
// A cache is [pages][kv heads][tokens a page][d_head]; pages may lie further apart (a stride), what is in one is contiguous.  Table row b
// names the pages of request b in order; the slot of a token is page * tokens a page + place.
#pragma once

#include "common.h"

namespace pvf {
namespace page {

template <int N>
struct Const { static constexpr int value = N; };

// A wave's sums over lanes 0 .. i, at most 2^32 - 1.
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
  auto behind = [&](auto ctrl, auto rows) {
    x = __builtin_elementwise_add_sat(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, decltype(rows)::value, 0xf, false));
  };
  behind(Const<0x111>{}, Const<0xf>{});   // rows of 16: one, two, four, eight lanes back
  behind(Const<0x112>{}, Const<0xf>{});
  behind(Const<0x114>{}, Const<0xf>{});
  behind(Const<0x118>{}, Const<0xf>{});
  behind(Const<0x142>{}, Const<0xa>{});   // the row in front, both rows in front
  behind(Const<0x143>{}, Const<0xc>{});
  return x;
}
__device__ __forceinline__ uint32_t last_lane(uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)x, 63); }

}  // namespace page

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
