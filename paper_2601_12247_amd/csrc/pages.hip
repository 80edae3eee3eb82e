// Page tables of a paged K/V cache, and its rows: which page and slot the new rows of each request get (extend), pages behind the tokens
// that requests keep go back to the free list (trim), rotary embedding of fresh rows with their keys and values into the slots (store).
//
// Extend and trim are prefix sums over the requests and then independent writes.  One workgroup makes the sums; where there is little to write it does so
// itself (one launch: what a step of single tokens costs is latency), otherwise a second launch spreads the writes over the chip.  That launch reads the
// sums only, so lengths and free counts may be updated in place.
#include "paged.h"

#include <algorithm>

namespace pvf {
namespace {

using page::last_lane;
using page::wave_scan;

constexpr int kThreads = 1024, kWaves = kThreads / kWave;
// One launch and two, us, pages of 16 tokens:
//   extend: 64 requests by 1 row 3.6 and 5.8, by 32 4.9 and 6.1, by 128 9.6 and 6.1; 2048 by 1 7.5 and 9.1, by 4 14.0 and 9.1
//   trim: 64 by 64 tokens 3.1 and 5.4, by 1000 5.0 and 5.4; 512 by 5 3.3 and 4.9, by 900 25.3 and 5.6.  How much comes back is on the device: up to 64
//   requests are taken for a batch that returns a few tokens of long ones.
constexpr int kFusedRequests = 2048, kFusedRows = 2048;
constexpr int64_t kFusedPages = 65536, kFusedPagesOfMany = 16384;   // requests times the table's width

// Inclusive prefix sum, at most 2^32 - 1, over the workgroup's threads, or where all requests fit a wave over each wave's lanes; *total: the sum.
// part: kWaves words of LDS that the sum before this one did not use.
template <bool kOneWave>
__device__ __forceinline__ uint32_t scan(uint32_t x, uint32_t *part, uint32_t *total) {
  x = wave_scan(x);
  if (kOneWave) {
    *total = last_lane(x);
    return x;
  }
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (lane == 63) part[wid] = x;
  __syncthreads();
  const uint32_t upto = wave_scan(lane < kWaves ? part[lane] : 0);
  *total = last_lane(upto);
  return __builtin_elementwise_add_sat(x, wid > 0 ? (uint32_t)__builtin_amdgcn_readlane((int)upto, wid - 1) : 0u);
}

// of at most 2^30 tokens
__device__ __forceinline__ uint32_t few_pages(int tokens, int P) { return ((uint32_t)tokens + (uint32_t)P - 1) / (uint32_t)P; }

// The request that owns item x: the last r with first[r] <= x (first does not decrease).
__device__ __forceinline__ int owner(const int32_t *first, int B, int x) {
  int lo = 0, hi = B;                                         // first[lo] <= x < first[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

// ---- extend ------------------------------------------------------------------------------------
struct Grown { int32_t row0, rows, given, top, have, start; bool admitted; };

// The position of a request's first row waits in pos[] itself (a caller may update seq_len in place).
__device__ __forceinline__ void write_row(const PageExtend &a, int r, const Grown &g, int t) {
  const int p = (int)((uint32_t)g.start + (uint32_t)t);
  int slot = -1;
  if (g.admitted) {
    const int j = (int)((uint32_t)p / (uint32_t)a.page_size);
    const int page = j < g.have ? a.table[(int64_t)r * a.table_stride + j] : a.free_pages[g.top - 1 - (j - g.have)];
    const int64_t at = (int64_t)page * a.page_size + (p - j * a.page_size);
    slot = page < 0 || at > INT32_MAX ? -1 : (int)at;          // a table's or free list's entry that is no page
  }
  a.pos[g.row0 + t] = p;
  a.slot[g.row0 + t] = slot;
}
__device__ __forceinline__ void write_page(const PageExtend &a, int r, const Grown &g, int j) {
  a.table[(int64_t)r * a.table_stride + g.have + j] = a.free_pages[g.top - 1 - j];
}
__device__ __forceinline__ void write_padding(const PageExtend &a, int m) { a.pos[m] = 0; a.slot[m] = -1; }

// kMost requests at most: 64 (every wave makes the sums for itself: 64 requests by 1 row 3.6 us, 3.8 with the workgroup's sums; a trim of them 3.1 and 3.8),
// kFusedRequests, or 0 for any number and a second launch for the rows.
template <int kMost>
__global__ void __launch_bounds__(kThreads)
page_extend_kernel(PageExtend a) {
  constexpr bool kOneWave = kMost == kWave, kFused = kMost > 0;
  __shared__ uint32_t part[3][kWaves];
  __shared__ int32_t s_cu[kMost + 1], s_taken[kMost + 1], s_start[kFused ? kMost : 1], s_have[kFused ? kMost : 1];   // s_have < 0: not admitted
  const int tid = threadIdx.x, P = a.page_size, stride = kOneWave ? kWave : kThreads, me = kOneWave ? tid & 63 : tid, most = a.width * P;
  const bool writes = !kOneWave || tid < kWave;
  const uint32_t n_free = (uint32_t)min(max(*a.n_free, 0), a.free_cap);
  uint32_t rows_before = 0, asked_before = 0, given_before = 0;
  for (int b0 = 0; b0 < a.B; b0 += stride) {
    const int b = b0 + me;
    int len = 0, start = 0, n = 0;
    if (b < a.B) {
      len = a.seq_len[b];
      n = a.n_rows[b];
      start = a.start ? a.start[b] : len;
    }
    if (kOneWave) __syncthreads();                             // every wave has read what the first may write
    const bool sound = b < a.B && n >= 0 && start >= 0 && start <= len && len <= most && n <= most - start;
    const int new_len = sound ? max(len, start + n) : len;
    const uint32_t rows = (uint32_t)min(max(n, 0), a.M + 1);    // more than M is too many, however many
    uint32_t all;
    const uint32_t upto = __builtin_elementwise_add_sat(rows_before, scan<kOneWave>(rows, part[0], &all));
    rows_before = __builtin_elementwise_add_sat(rows_before, all);
    const bool fits = sound && upto <= (uint32_t)a.M;
    const uint32_t have = sound ? few_pages(len, P) : 0, need = fits ? few_pages(new_len, P) - have : 0;
    const uint32_t asked = __builtin_elementwise_add_sat(asked_before, scan<kOneWave>(need, part[1], &all));
    asked_before = __builtin_elementwise_add_sat(asked_before, all);
    const bool admitted = fits && (need == 0 || asked <= n_free);
    // what is asked for does not decrease, so the requests that get pages are the first of those that want some
    uint32_t taken = asked;
    if (asked_before <= n_free) {
      given_before = asked_before;
    } else {
      const uint32_t given = admitted ? need : 0;
      taken = given_before + scan<kOneWave>(given, part[2], &all);
      given_before += all;
    }
    if (b < a.B) {
      const int end = (int)min((uint32_t)a.M, upto), row0 = (int)min((uint32_t)a.M, upto - rows);
      if (writes) {
        a.seq_len_out[b] = admitted ? new_len : len;
        a.admitted[b] = admitted;
        a.cu_rows[b + 1] = end;
        a.place[b + 1] = (int)(n_free - taken);
        if (!kFused && row0 < a.M && rows > 0) a.pos[row0] = start;
      }
      if (kFused) {                                            // with one wave's requests, every wave writes the same
        s_cu[b + 1] = end;
        s_taken[b + 1] = (int)taken;
        s_start[b] = start;
        s_have[b] = admitted ? (int)have : -1;
      }
    }
    if (!kOneWave && b0 + stride < a.B) __syncthreads();       // part[] has been read
  }
  if (tid == 0) {
    a.cu_rows[0] = 0;
    a.place[0] = (int)n_free;
    if (kFused) s_cu[0] = s_taken[0] = 0;
  }
  __syncthreads();                                             // and every thread has read *n_free
  if (tid == 0) *a.n_free_out = (int)(n_free - given_before);
  if (!kFused) return;
  const int total_rows = a.B > 0 ? s_cu[a.B] : 0, total_pages = (int)given_before;
  auto grown = [&](int r) {
    return Grown{s_cu[r], s_cu[r + 1] - s_cu[r], s_taken[r + 1] - s_taken[r], (int)n_free - s_taken[r], s_have[r], s_start[r], s_have[r] >= 0};
  };
  for (int m = tid; m < a.M; m += kThreads) {
    if (m >= total_rows) { write_padding(a, m); continue; }
    const int r = owner(s_cu, a.B, m);
    const Grown g = grown(r);
    write_row(a, r, g, m - g.row0);
  }
  for (int x = tid; x < total_pages; x += kThreads) {
    const int r = owner(s_taken, a.B, x);
    write_page(a, r, grown(r), x - s_taken[r]);
  }
}

// Block (r, y) writes a part of the rows and pages of request r; block row B the rows behind the last request.
__global__ void __launch_bounds__(256)
page_extend_rows_kernel(PageExtend a) {
  const int r = blockIdx.x, first = blockIdx.y * 256 + threadIdx.x, step = gridDim.y * 256;
  if (r == a.B) {
    for (int m = a.cu_rows[a.B] + first; m < a.M; m += step) write_padding(a, m);
    return;
  }
  Grown g;
  g.row0 = a.cu_rows[r];
  g.rows = a.cu_rows[r + 1] - g.row0;
  g.top = a.place[r];
  g.given = g.top - a.place[r + 1];
  g.admitted = a.admitted[r] != 0;
  g.have = g.admitted ? (int)few_pages(a.seq_len_out[r], a.page_size) - g.given : 0;
  g.start = g.rows > 0 ? a.pos[g.row0] : 0;
  for (int t = first; t < g.rows; t += step) write_row(a, r, g, t);
  for (int j = first; j < g.given; j += step) write_page(a, r, g, j);
}

// ---- trim --------------------------------------------------------------------------------------
constexpr int kTrimEach = 4;               // requests of a thread where there are many

template <int kMost>
__global__ void __launch_bounds__(kThreads)
page_trim_kernel(PageTrim a) {
  constexpr bool kOneWave = kMost == kWave, kFused = kMost > 0;
  constexpr int kEach = kOneWave ? 1 : kTrimEach;
  __shared__ uint32_t part[2][kWaves];
  __shared__ int32_t s_place[kMost + 1], s_first[kFused ? kMost : 1];
  const int tid = threadIdx.x, P = a.page_size, me = kOneWave ? tid & 63 : tid, most = a.width * P, stride = (kOneWave ? kWave : kThreads) * kEach;
  const bool writes = !kOneWave || tid < kWave;
  const uint32_t n_free = (uint32_t)min(max(*a.n_free, 0), a.free_cap);
  uint32_t before = n_free;
  int turn = 0;
  for (int b0 = 0; b0 < a.B; b0 += stride, turn ^= 1) {
    int keep[kEach];
    uint32_t first[kEach], back[kEach], sum = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int b = b0 + me * kEach + i;
      int len = 0;
      keep[i] = 0;
      if (b < a.B) {
        len = min(max(a.seq_len[b], 0), most);
        keep[i] = min(max(a.keep[b], 0), len);
      }
      first[i] = few_pages(keep[i], P);
      back[i] = few_pages(len, P) - first[i];
      sum = __builtin_elementwise_add_sat(sum, back[i]);
    }
    if (kOneWave) __syncthreads();                             // every wave has read what the first may write
    uint32_t all, upto = __builtin_elementwise_add_sat(before, scan<kOneWave>(sum, part[turn], &all));
    before = __builtin_elementwise_add_sat(before, all);
    upto = upto == 0xffffffffu ? upto : upto - sum;            // beyond the list either way
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int b = b0 + me * kEach + i;
      upto = __builtin_elementwise_add_sat(upto, back[i]);
      if (b < a.B) {
        const int behind = (int)min((uint32_t)a.free_cap, upto);
        if (writes) {
          a.seq_len_out[b] = keep[i];
          a.place[b + 1] = behind;
        }
        if (kFused) {
          s_place[b + 1] = behind;
          s_first[b] = (int)first[i];
        }
      }
    }
  }
  const int top = (int)min((uint32_t)a.free_cap, before);
  if (tid == 0) {
    a.place[0] = (int)n_free;
    if (kFused) s_place[0] = (int)n_free;
  }
  __syncthreads();                                             // and every thread has read *n_free
  if (tid == 0) *a.n_free_out = top;
  if (!kFused) return;
  for (int x = (int)n_free + tid; x < top; x += kThreads) {
    const int r = owner(s_place, a.B, x);
    a.free_pages[x] = a.table[(int64_t)r * a.table_stride + s_first[r] + (x - s_place[r])];
  }
}

__global__ void __launch_bounds__(256)
page_trim_pages_kernel(PageTrim a) {
  const int r = blockIdx.x, at = a.place[r], n = a.place[r + 1] - at;
  if (n == 0) return;
  const int32_t *src = a.table + (int64_t)r * a.table_stride + few_pages(a.seq_len_out[r], a.page_size);
  for (int j = blockIdx.y * 256 + threadIdx.x; j < n; j += gridDim.y * 256) a.free_pages[at + j] = src[j];
}

// ---- store -------------------------------------------------------------------------------------
// One pass over the rows, bound by HBM.  A workgroup takes kRows rows; a thread takes units of 2 x VEC elements, i .. i + VEC - 1 of a head
// and their partners i + dh / 2 .., so that a rotation needs no other thread.  Heads of at most 128 bytes (kNarrow) would be written in pieces of half a
// line or less: there a unit is VEC elements and its partners are read as well (32 + 2 x 8 heads of 64 in bf16, 12000 rows: 27.4 us, 36.7 with pairs; of
// 256, 3000 rows: 33.4 and 27.3).  The lanes of a head are then in one wave, which has read all of it before it writes any: q_out may be qkv.  Angles are products in float64, brought to one turn there
// (off by 2^-28 radians at position 2^24 and 2^-21 at 2^31, where float32 is off by whole turns), their sine and cosine in float32, once for each row and pair.
// 11520 rows of 32 + 2 x 32 heads of 128, bf16: 117 us for 566 MB read and written (4.84 TB/s, a copy's 4.94).
template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) Pack { T v[VEC]; };

template <typename T, int VEC, int kRows, bool kNarrow>
__global__ void __launch_bounds__(256)
page_store_kernel(PageStore a) {
  __shared__ float2 s_cs[kRows * 128];
  __shared__ int64_t s_k[kRows], s_v[kRows];                   // where a row's first head goes, -1: nowhere
  typedef Pack<T, VEC> V;
  const int tid = threadIdx.x, half = a.dh / 2, m0 = blockIdx.x * kRows, rows = min(kRows, a.M - m0);
  if (tid < rows) {
    const int slot = a.slot[m0 + tid], page = slot / a.page_size, at = slot - page * a.page_size;
    const bool kept = slot >= 0 && page < a.n_pages;
    s_k[tid] = kept ? page * a.k_page_stride + (int64_t)at * a.dh : -1;
    s_v[tid] = kept ? page * a.v_page_stride + (int64_t)at * a.dh : -1;
  }
  for (int i = tid; i < rows * half; i += 256) {
    const int r = i / half, e = i - r * half;
    const double turns = a.pos[m0 + r] * (exp2(-2.0 * e / a.dh * a.log2_theta) * 0.15915494309189533577);   // 1 / (2 pi)
    float sn, cs;
    sincospif(2.0f * (float)(turns - rint(turns)), &sn, &cs);
    s_cs[i] = make_float2(cs, sn);
  }
  __syncthreads();
  const int per_head = (kNarrow ? a.dh : half) / VEC, heads = a.H + 2 * a.Hkv, units = rows * heads * per_head;
  const int64_t head_stride = (int64_t)a.page_size * a.dh;
  const T *qkv = (const T *)a.qkv;
  constexpr int kHeld = 4;                                     // units a thread has on the way (q_out may be the rows' own q part, so loads are not moved over stores)
  for (int u0 = tid; u0 < units; u0 += kHeld * 256) {
    V lo[kHeld], hi[kHeld];
    int row[kHeld], head[kHeld], c[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      const int u = min(u0 + i * 256, units - 1), x = u / per_head;
      c[i] = (u - x * per_head) * VEC;
      row[i] = x / heads;
      head[i] = x - row[i] * heads;
      const T *src = qkv + (int64_t)(m0 + row[i]) * a.qkv_stride + (int64_t)head[i] * a.dh + c[i];
      lo[i] = *(const V *)src;
      hi[i] = *(const V *)(kNarrow && c[i] >= half ? src - half : src + half);
    }
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      if (u0 + i * 256 >= units || s_k[row[i]] < 0) continue;
      if (head[i] < a.H + a.Hkv) {
        const bool upper = kNarrow && c[i] >= half;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float2 cs = s_cs[row[i] * half + (upper ? c[i] - half : c[i]) + e];
          const float x = to_float(lo[i].v[e]), y = to_float(hi[i].v[e]);
          const float2 t = rotate_pair(upper ? y : x, upper ? x : y, cs.x, cs.y);
          lo[i].v[e] = from_float<T>(upper ? t.y : t.x);
          hi[i].v[e] = from_float<T>(t.y);
        }
      }
      T *dst = head[i] < a.H ? (T *)a.q_out + (int64_t)(m0 + row[i]) * a.q_stride + (int64_t)head[i] * a.dh
               : head[i] < a.H + a.Hkv ? (T *)a.k_cache + s_k[row[i]] + (head[i] - a.H) * head_stride
                                       : (T *)a.v_cache + s_v[row[i]] + (head[i] - a.H - a.Hkv) * head_stride;
      *(V *)(dst + c[i]) = lo[i];
      if (!kNarrow) *(V *)(dst + c[i] + half) = hi[i];
    }
  }
}

// Four rows a workgroup keep more loads on the way, one spreads few rows over the chip: 512 rows of 32 + 2 x 8 heads of 128, bf16, 6.1 us with one and 8.3
// with four, 1024 8.7 and 9.1, 2048 14.0 and 13.1, 4096 22.3 and 19.3.
template <typename T, int VEC, bool kNarrow>
void store_rows(hipStream_t s, const PageStore &a) {
  if (a.M <= 1024) page_store_kernel<T, VEC, 1, kNarrow><<<a.M, 256, 0, s>>>(a);
  else page_store_kernel<T, VEC, 4, kNarrow><<<(a.M + 3) / 4, 256, 0, s>>>(a);
}

}  // namespace

pvf_status launch_page_extend(hipStream_t s, const PageExtend &a) {
  if (a.M <= kFusedRows && a.B <= kFusedRequests) {
    if (a.B <= kWave) page_extend_kernel<kWave><<<1, kThreads, 0, s>>>(a);
    else page_extend_kernel<kFusedRequests><<<1, kThreads, 0, s>>>(a);
    PVF_LAUNCH_CHECK(nullptr, "page_extend");
    return PVF_OK;
  }
  page_extend_kernel<0><<<1, kThreads, 0, s>>>(a);
  PVF_LAUNCH_CHECK(nullptr, "page_extend");
  const int y = (int)std::min<int64_t>(64, ((int64_t)a.M / 1024 + a.B) / (a.B + 1) + 1);
  page_extend_rows_kernel<<<dim3(a.B + 1, y), 256, 0, s>>>(a);
  PVF_LAUNCH_CHECK(nullptr, "page_extend_rows");
  return PVF_OK;
}

pvf_status launch_page_trim(hipStream_t s, const PageTrim &a) {
  if ((int64_t)a.B * a.width <= (a.B <= kWave ? kFusedPages : kFusedPagesOfMany) && a.B <= kFusedRequests) {
    if (a.B <= kWave) page_trim_kernel<kWave><<<1, kThreads, 0, s>>>(a);
    else page_trim_kernel<kFusedRequests><<<1, kThreads, 0, s>>>(a);
    PVF_LAUNCH_CHECK(nullptr, "page_trim");
    return PVF_OK;
  }
  page_trim_kernel<0><<<1, kThreads, 0, s>>>(a);
  PVF_LAUNCH_CHECK(nullptr, "page_trim");
  const int y = (int)std::min<int64_t>(64, ((int64_t)a.width / 1024) * 256 / std::max(a.B, 256) + 1);
  page_trim_pages_kernel<<<dim3(a.B, y), 256, 0, s>>>(a);
  PVF_LAUNCH_CHECK(nullptr, "page_trim_pages");
  return PVF_OK;
}

pvf_status launch_page_store(hipStream_t s, int dtype, const PageStore &a) {
  const int size = dtype == PVF_F32 ? 4 : 2, lanes = a.dh * size / 16;
  const bool narrow = a.dh * size % 32 == 0 && lanes <= 8 && (lanes & (lanes - 1)) == 0;      // whole heads in a wave
  if (dtype == PVF_F32 && narrow) store_rows<float, 4, true>(s, a);
  else if (dtype == PVF_F32) store_rows<float, 4, false>(s, a);
  else if (narrow) store_rows<bf16_t, 8, true>(s, a);
  else if (a.dh % 16 == 0) store_rows<bf16_t, 8, false>(s, a);
  else store_rows<bf16_t, 4, false>(s, a);
  PVF_LAUNCH_CHECK(nullptr, "page_store");
  return PVF_OK;
}

}  // namespace pvf
