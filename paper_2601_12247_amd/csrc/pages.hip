// Page tables of a paged K/V cache, and its rows: which page and slot the new rows of each request get (extend), pages behind the tokens
// that requests keep go back to the free list (trim), rotary embedding of fresh rows with their keys and values into the slots (store).
//
// Extend and trim are prefix sums over the requests and then independent writes.  One workgroup makes the sums; up to kFusedRows rows it
// writes everything itself (one launch: what a step of single tokens costs is latency), behind that a second launch spreads the writes over
// the chip.  That launch reads the sums only, so lengths and free counts may be updated in place.
#include "paged.h"

#include <algorithm>

namespace pvf {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / kWave;
constexpr int kFusedRequests = 2048, kFusedRows = 8192;
constexpr int64_t kFusedPages = 65536;

// Inclusive prefix sum over the workgroup's threads; *total: the sum.  part: kWaves elements of LDS.
__device__ __forceinline__ int64_t block_scan(int64_t x, int64_t *part, int64_t *total) {
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const int64_t y = __shfl_up(x, o, kWave);
    if (lane >= o) x += y;
  }
  __syncthreads();                                            // the last scan's reads of part are done
  if (lane == 63) part[wid] = x;
  __syncthreads();
  int64_t before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    const int64_t p = part[i];
    before += i < wid ? p : 0;
    all += p;
  }
  *total = all;
  return x + before;
}

__device__ __forceinline__ int64_t pages_of(int64_t tokens, int P) { return (tokens + P - 1) / P; }

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
    const int j = p / a.page_size;
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

template <bool kFused>
__global__ void __launch_bounds__(kThreads)
page_extend_kernel(PageExtend a) {
  __shared__ int64_t part[kWaves];
  __shared__ int32_t s_cu[kFused ? kFusedRequests + 1 : 1], s_taken[kFused ? kFusedRequests + 1 : 1];
  __shared__ int32_t s_start[kFused ? kFusedRequests : 1], s_have[kFused ? kFusedRequests : 1];   // s_have < 0: not admitted
  const int tid = threadIdx.x, P = a.page_size;
  const int64_t most = (int64_t)a.width * P;
  const int n_free = min(max(*a.n_free, 0), a.free_cap);
  int64_t rows_before = 0, asked_before = 0, given_before = 0;
  for (int b0 = 0; b0 < a.B; b0 += kThreads) {
    const int b = b0 + tid;
    int64_t len = 0, start = 0, n = 0;
    if (b < a.B) {
      len = a.seq_len[b];
      start = a.start ? a.start[b] : len;
      n = a.n_rows[b];
    }
    const bool sound = b < a.B && n >= 0 && start >= 0 && start <= len && len <= most;
    const int64_t rows = n > 0 ? n : 0, new_len = max(len, start + n);
    int64_t all;
    const int64_t upto = rows_before + block_scan(rows, part, &all);
    rows_before += all;
    const bool fits = sound && new_len <= most && upto <= a.M;
    const int64_t need = fits ? pages_of(new_len, P) - pages_of(len, P) : 0;
    const int64_t asked = asked_before + block_scan(need, part, &all);
    asked_before += all;
    const bool admitted = fits && (need == 0 || asked <= n_free);
    const int64_t given = admitted ? need : 0, taken = given_before + block_scan(given, part, &all);
    given_before += all;
    if (b < a.B) {
      const int row0 = (int)min((int64_t)a.M, upto - rows);
      a.seq_len_out[b] = (int)(admitted ? new_len : len);
      a.admitted[b] = admitted;
      a.cu_rows[b + 1] = (int)min((int64_t)a.M, upto);
      a.place[b + 1] = (int)(n_free - taken);
      if (row0 < a.M && rows > 0) a.pos[row0] = (int)start;
      if (kFused) {
        s_cu[b + 1] = (int)min((int64_t)a.M, upto);
        s_taken[b + 1] = (int)taken;
        s_start[b] = (int)start;
        s_have[b] = admitted ? (int)pages_of(len, P) : -1;
      }
    }
  }
  __syncthreads();
  if (tid == 0) {
    a.cu_rows[0] = 0;
    a.place[0] = n_free;
    *a.n_free_out = (int)(n_free - given_before);
    if (kFused) s_cu[0] = s_taken[0] = 0;
  }
  if (!kFused) return;
  __syncthreads();
  const int total_rows = s_cu[a.B], total_pages = s_taken[a.B];
  auto grown = [&](int r) {
    return Grown{s_cu[r], s_cu[r + 1] - s_cu[r], s_taken[r + 1] - s_taken[r], n_free - s_taken[r], s_have[r], s_start[r], s_have[r] >= 0};
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
  g.have = (int)pages_of(a.seq_len_out[r], a.page_size) - g.given;
  g.start = g.rows > 0 ? a.pos[g.row0] : 0;
  for (int t = first; t < g.rows; t += step) write_row(a, r, g, t);
  for (int j = first; j < g.given; j += step) write_page(a, r, g, j);
}

// ---- trim --------------------------------------------------------------------------------------
template <bool kFused>
__global__ void __launch_bounds__(kThreads)
page_trim_kernel(PageTrim a) {
  __shared__ int64_t part[kWaves];
  __shared__ int32_t s_place[kFused ? kFusedRequests + 1 : 1], s_first[kFused ? kFusedRequests : 1];
  const int tid = threadIdx.x, P = a.page_size;
  const int64_t most = (int64_t)a.width * P;
  const int n_free = min(max(*a.n_free, 0), a.free_cap);
  int64_t before = 0;
  for (int b0 = 0; b0 < a.B; b0 += kThreads) {
    const int b = b0 + tid;
    int64_t len = 0, keep = 0;
    if (b < a.B) {
      len = min(max((int64_t)a.seq_len[b], (int64_t)0), most);
      keep = min(max((int64_t)a.keep[b], (int64_t)0), len);
    }
    int64_t all;
    const int64_t back = pages_of(len, P) - pages_of(keep, P), upto = before + block_scan(back, part, &all);
    before += all;
    if (b < a.B) {
      const int behind = (int)min((int64_t)a.free_cap, n_free + upto);
      a.seq_len_out[b] = (int)keep;
      a.place[b + 1] = behind;
      if (kFused) {
        s_place[b + 1] = behind;
        s_first[b] = (int)pages_of(keep, P);
      }
    }
  }
  __syncthreads();
  const int top = (int)min((int64_t)a.free_cap, n_free + before);
  if (tid == 0) {
    a.place[0] = n_free;
    *a.n_free_out = top;
    if (kFused) s_place[0] = n_free;
  }
  if (!kFused) return;
  __syncthreads();
  for (int x = n_free + tid; x < top; x += kThreads) {
    const int r = owner(s_place, a.B, x);
    a.free_pages[x] = a.table[(int64_t)r * a.table_stride + s_first[r] + (x - s_place[r])];
  }
}

__global__ void __launch_bounds__(256)
page_trim_pages_kernel(PageTrim a) {
  const int r = blockIdx.x, at = a.place[r], n = a.place[r + 1] - at;
  if (n == 0) return;
  const int32_t *src = a.table + (int64_t)r * a.table_stride + pages_of(a.seq_len_out[r], a.page_size);
  for (int j = blockIdx.y * 256 + threadIdx.x; j < n; j += gridDim.y * 256) a.free_pages[at + j] = src[j];
}

// ---- store -------------------------------------------------------------------------------------
// One pass over the rows, bound by HBM.  A workgroup takes kRows rows; a thread takes units of 2 x VEC elements, i .. i + VEC - 1 of a head
// and their partners i + dh / 2 .., so that a rotation needs no other thread.  Angles are products in float64, brought to one turn there
// (position 2^31 is as exact as position 1), their sine and cosine in float32, once for each row and pair.
template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) Pack { T v[VEC]; };

template <typename T, int VEC, int kRows>
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
  const int per_head = half / VEC, heads = a.H + 2 * a.Hkv, units = rows * heads * per_head;
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
      hi[i] = *(const V *)(src + half);
    }
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      if (u0 + i * 256 >= units || s_k[row[i]] < 0) continue;
      if (head[i] < a.H + a.Hkv) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float2 cs = s_cs[row[i] * half + c[i] + e];
          const float2 t = rotate_pair(to_float(lo[i].v[e]), to_float(hi[i].v[e]), cs.x, cs.y);
          lo[i].v[e] = from_float<T>(t.x);
          hi[i].v[e] = from_float<T>(t.y);
        }
      }
      T *dst = head[i] < a.H ? (T *)a.q_out + (int64_t)(m0 + row[i]) * a.q_stride + (int64_t)head[i] * a.dh
               : head[i] < a.H + a.Hkv ? (T *)a.k_cache + s_k[row[i]] + (head[i] - a.H) * head_stride
                                       : (T *)a.v_cache + s_v[row[i]] + (head[i] - a.H - a.Hkv) * head_stride;
      *(V *)(dst + c[i]) = lo[i];
      *(V *)(dst + c[i] + half) = hi[i];
    }
  }
}

template <typename T, int VEC>
void store_rows(hipStream_t s, const PageStore &a) {
  if (a.M <= 512) page_store_kernel<T, VEC, 1><<<a.M, 256, 0, s>>>(a);
  else page_store_kernel<T, VEC, 4><<<(a.M + 3) / 4, 256, 0, s>>>(a);
}

}  // namespace

pvf_status launch_page_extend(hipStream_t s, const PageExtend &a) {
  if (a.M <= kFusedRows && a.B <= kFusedRequests) {
    page_extend_kernel<true><<<1, kThreads, 0, s>>>(a);
    PVF_LAUNCH_CHECK(nullptr, "page_extend");
    return PVF_OK;
  }
  page_extend_kernel<false><<<1, kThreads, 0, s>>>(a);
  PVF_LAUNCH_CHECK(nullptr, "page_extend");
  const int y = (int)std::min<int64_t>(64, ((int64_t)a.M / 1024 + a.B) / (a.B + 1) + 1);
  page_extend_rows_kernel<<<dim3(a.B + 1, y), 256, 0, s>>>(a);
  PVF_LAUNCH_CHECK(nullptr, "page_extend_rows");
  return PVF_OK;
}

pvf_status launch_page_trim(hipStream_t s, const PageTrim &a) {
  if ((int64_t)a.B * a.width <= kFusedPages && a.B <= kFusedRequests) {
    page_trim_kernel<true><<<1, kThreads, 0, s>>>(a);
    PVF_LAUNCH_CHECK(nullptr, "page_trim");
    return PVF_OK;
  }
  page_trim_kernel<false><<<1, kThreads, 0, s>>>(a);
  PVF_LAUNCH_CHECK(nullptr, "page_trim");
  const int y = (int)std::min<int64_t>(64, ((int64_t)a.width / 1024) * 256 / std::max(a.B, 256) + 1);
  page_trim_pages_kernel<<<dim3(a.B, y), 256, 0, s>>>(a);
  PVF_LAUNCH_CHECK(nullptr, "page_trim_pages");
  return PVF_OK;
}

pvf_status launch_page_store(hipStream_t s, int dtype, const PageStore &a) {
  if (dtype == PVF_F32) store_rows<float, 4>(s, a);
  else if (a.dh % 16 == 0) store_rows<bf16_t, 8>(s, a);
  else store_rows<bf16_t, 4>(s, a);
  PVF_LAUNCH_CHECK(nullptr, "page_store");
  return PVF_OK;
}

}  // namespace pvf
