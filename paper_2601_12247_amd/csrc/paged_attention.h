// What the kernels of attention over pages share: which worker takes which keys and rows, and how partial results travel.
//
// All (request, key head, tile of columns) triples lie behind each other, each with its steps of keys.  Workers (workgroups) take equal
// shares of that line, wherever they begin and end, so any mix of lengths fills the chip; every worker finds its place from the lengths by itself.
// A triple that more than one worker took is joined by a second launch, from partial results in the workspace.
#pragma once

#include "paged.h"

namespace pvf {
namespace page {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));

constexpr int kPageSlots = 1024;          // table entries in LDS

struct Args {
  PageAttention p;
  int32_t group, chunk_steps;             // heads a key head; steps whose pages fit kPageSlots
  uint32_t div_mul, div_shift;            // page of a key
  float c;                                // |scale| * log2(e), above zero: scores are compared before they are scaled,
  uint32_t q_xor;                         // and the sign of a negative scale goes into q
  int32_t whole;                          // 1: the line is of triples, not steps (host)
  int32_t *joins;                         // [workers][kJoinInts]: the triple that worker w begins and others end
};
constexpr int kJoinInts = 8;              // workers that took it (0: none), its first row, rows, length, key head, tile

struct Request {
  int row0, n, len, steps, tiles;         // its rows, visible keys, steps of keys and tiles of columns
  bool over;                              // longer than its table
  int64_t triples, items;                 // items: its length on the line, triples or steps of them
};

template <class I>
__device__ __forceinline__ Request request(const Args &a, int b, bool whole) {
  Request r;
  const int raw = a.p.seq_len[b];
  if (a.p.cu_rows) {
    const int from = a.p.cu_rows[b], to = a.p.cu_rows[b + 1];
    r.row0 = min(max(from, 0), a.p.M);
    r.n = max(min(to, a.p.M) - r.row0, 0);
  } else {
    r.row0 = b;
    r.n = 1;
  }
  const int len = max(raw, 0), most = a.p.width * a.p.page_size;
  r.len = min(len, most);
  r.over = len > most;
  r.steps = max((r.len - 1) / I::kStep + 1, 1);
  r.tiles = (int)(((uint32_t)(r.n * a.group) + I::QT - 1) / I::QT);
  r.triples = (int64_t)r.tiles * a.p.Hkv;
  r.items = whole ? r.triples : r.triples * r.steps;
  return r;
}

// Keys that row `row` of the request sees.
__device__ __forceinline__ int limit_of(const Args &a, int len, int n, int row) { return a.p.causal ? len - n + row + 1 : len; }

__device__ __forceinline__ int64_t wave_scan(int64_t x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const int64_t y = __shfl_up(x, o, kWave);
    if (lane >= o) x += y;
  }
  return x;
}
__device__ __forceinline__ int64_t uniform64(int64_t x) {
  return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)x));
}

// a / b, and *rest: exact below 2^52.
__device__ __forceinline__ int64_t divide(int64_t a, int b, int64_t *rest) {
  int64_t q = (int64_t)((double)a / (double)b), r = a - q * b;   // at most one off
  if (r < 0) { --q; r += b; }
  if (r >= b) { ++q; r -= b; }
  *rest = r;
  return q;
}

// A worker's place: items [at, end) of the line, `at` in request b, whose first item is `first`.
struct Place {
  int64_t at, end, first, share;
  int b;
  bool whole;                             // the line is of triples
};

// The request that item `at` belongs to, and its first item.
template <class I>
__device__ __forceinline__ int find_request(const Args &a, int64_t at, bool whole, int64_t *first) {
  const int lane = threadIdx.x & 63;
  int64_t base = 0;
  for (int b0 = 0;; b0 += kWave) {
    const int b = b0 + lane;
    const int64_t items = b < a.p.B ? request<I>(a, b, whole).items : 0, upto = base + wave_scan(items);
    const uint64_t beyond = __builtin_amdgcn_ballot_w64(upto > at);
    if (beyond || b0 + kWave >= a.p.B) {
      const int l = beyond ? __builtin_ctzll(beyond) : 63;
      *first = uniform64(__shfl(upto - items, l, kWave));
      return __builtin_amdgcn_readfirstlane(min(b0 + l, a.p.B - 1));
    }
    base = uniform64(__shfl(upto, 63, kWave));
  }
}

// Triples stay whole where the host says so, and on kSnap instances, whose partial results are large, where that divides the work well enough:
// none is longer than kSnap shares, and there are no more of them than workers, or several for each.
template <class I>
__device__ __forceinline__ Place place_of(const Args &a, int block, int workers, int *worker) {
  const int lane = threadIdx.x & 63;
  int64_t items = 0, triples = 0;
  int longest = 0;
  for (int b = lane; b < a.p.B; b += kWave) {
    const Request r = request<I>(a, b, a.whole);
    items += r.items;
    triples += r.triples;
    longest = max(longest, r.n > 0 ? r.steps : 0);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    items += __shfl_xor(items, o, kWave);
    if (I::kSnap > 0) triples += __shfl_xor(triples, o, kWave);
    if (I::kSnap > 0) longest = max(longest, __shfl_xor(longest, o, kWave));
  }
  items = uniform64(items);
  Place w;
  int64_t rest;
  w.share = divide(items + workers - 1, workers, &rest);
  w.whole = a.whole;
  if (I::kSnap > 0 && !a.whole) {
    triples = uniform64(triples);
    if (__builtin_amdgcn_readfirstlane(longest) <= I::kSnap * w.share && (triples <= workers || triples >= 4 * (int64_t)workers)) {
      w.whole = true;
      items = triples;
      w.share = divide(items + workers - 1, workers, &rest);
    }
  }
  // workers that follow each other read the same keys for other columns: where all take part, neighbours run on one XCD and share its L2
  *worker = workers % 8 == 0 && w.share * (workers - 1) < items ? block % 8 * (workers / 8) + block / 8 : block;
  w.at = w.share * *worker;
  w.end = min(w.at + w.share, items);
  if (w.at < w.end) w.b = find_request<I>(a, w.at, w.whole, &w.first);
  return w;
}

// The part of a triple that a worker takes next.
struct Piece {
  int step0, step1, head, tile, cols;
  bool done, begun;                       // all of it; from its first step on
};

// False: nothing is left (or lengths changed under the call).  b and r follow.
template <class I>
__device__ __forceinline__ bool next_piece(const Args &a, Place &w, Request &r, Piece &p) {
  if (w.at >= w.end) return false;
  while (w.at - w.first >= r.items) {
    w.first += r.items;
    if (++w.b >= a.p.B) return false;
    r = request<I>(a, w.b, w.whole);
  }
  int64_t triple = w.at - w.first;
  if (w.whole) {
    p.step0 = 0;
    p.step1 = r.steps;
    ++w.at;
  } else {
    int64_t step0;
    triple = divide(triple, r.steps, &step0);
    p.step0 = (int)step0;
    p.step1 = (int)min((int64_t)r.steps, p.step0 + (w.end - w.at));
    w.at += p.step1 - p.step0;
  }
  p.head = (int)((uint32_t)triple / (uint32_t)r.tiles);        // rows and heads together are below 2^31
  p.tile = (int)((uint32_t)triple - (uint32_t)p.head * r.tiles);
  if (p.head >= a.p.Hkv) return false;                         // cannot be, unless lengths change under the call
  p.cols = min(I::QT, r.n * a.group - p.tile * I::QT);
  p.begun = p.step0 == 0;
  p.done = p.begun && p.step1 == r.steps;
  return true;
}

// Where a column's row and head begin in q or out.
__device__ __forceinline__ int64_t row_place(const Args &a, int row0, int head, int pair, int64_t stride, int *row) {
  const uint32_t m = (uint32_t)pair / (uint32_t)a.group;
  const int sub = (int)((uint32_t)pair - m * (uint32_t)a.group);
  *row = (int)m;
  return (int64_t)(row0 + (int)m) * stride + (int64_t)(head * a.group + sub) * a.p.dh;
}

// Partial results: worker w has two, 2 w: of the triple that an earlier worker began, 2 w + 1: of the one that it begins itself.
template <class I>
__device__ __forceinline__ float *partial(const Args &a, int worker, bool begun) { return a.p.ws + (int64_t)(2 * worker + begun) * I::kSlotFloats; }

// How many workers take a triple that this one begins.
template <class I>
__device__ __forceinline__ void note_join(const Args &a, int worker, const Place &w, const Request &r, const Piece &p) {
  const int64_t behind = r.steps - p.step1;                    // items that other workers take, w.share each
  int32_t *j = a.joins + (int64_t)worker * kJoinInts;
  int64_t rest;
  *(int4 *)(j + 4) = make_int4(p.head, p.tile, 0, 0);
  *(int4 *)j = make_int4((int)divide(behind + w.share - 1, (int)w.share, &rest) + 1, r.row0, r.n, r.len);
}

template <typename T>
__device__ __forceinline__ void store4(T *dst, floatx4 x, float inv_total, bool none) {
  struct alignas(4 * sizeof(T)) { T v[4]; } y;
#pragma unroll
  for (int i = 0; i < 4; ++i) y.v[i] = from_float<T>(none ? 0.f : x[i] * inv_total);
  *(decltype(y) *)dst = y;
}

// A running maximum below which everything is zero, and how much a maximum m weighs beside it.
__device__ __forceinline__ float reference(float top) { return top == -INFINITY ? 0.f : top; }
__device__ __forceinline__ float weight(const Args &a, float m, float ref) { return __builtin_amdgcn_exp2f((m - ref) * a.c); }

// Where a key lies, from the table entries in LDS; *none: on no page (page 0 is read).
__device__ __forceinline__ int page_of(const Args &a, int key) { return (int)(__umulhi((uint32_t)(key >> 3) << 1, a.div_mul) >> a.div_shift); }

// Table entries of keys k0 .. k1 - 1 into LDS, -1 for what is no page; every thread's answer: whether one of its entries is.
__device__ __forceinline__ bool load_pages(const Args &a, int b, int k0, int k1, int first_page, int32_t *s_pages) {
  const int n = k1 > k0 ? page_of(a, k1 - 1) - first_page + 1 : 0;
  bool bad = false;
  for (int i = threadIdx.x; i < n; i += 256) {
    const int j = first_page + i;
    int id = -1;
    if (j < a.p.width) id = a.p.table[(int64_t)b * a.p.table_stride + j];
    const bool there = id >= 0 && id < a.p.n_pages;
    s_pages[i] = there ? id : -1;
    bad |= !there;
  }
  return bad;
}

__device__ __forceinline__ bool bf16s_not_finite(uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; }
__device__ __forceinline__ uint32_t bf16s_finite(uint32_t w) {   // what is not finite as zero
  if ((w & 0x7f800000u) == 0x7f800000u) w &= 0xffffu;
  if ((w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u;
  return w;
}

// y (float32 bits) where it is not finite, else zero: what a key adds whose probability is not zero
__device__ __forceinline__ float odd_part(uint32_t y) { return (y & 0x7f800000u) == 0x7f800000u ? __uint_as_float(y) : 0.f; }

// Two probabilities as bf16 in two parts: the upper halves, and the rest of 16 bits.  The rest is never zero beside p > 0 (2^-23 of p is added): zero
// times an infinite value would make NaN of infinity.
__device__ __forceinline__ uint32_t upper_parts(float x, float y) { return __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302); }
__device__ __forceinline__ uint32_t lower_parts(float x, float y) {
  auto low = [](float p) { return (bf16_t)__builtin_fmaf(p, 1.0f + 0x1p-23f, -__uint_as_float(__float_as_uint(p) & 0xffff0000u)); };
  const bf16x2 r = {low(x), low(y)};
  return __builtin_bit_cast(uint32_t, r);
}

// ---- the join: block w joins the triple that worker w begins, if others end it ----------------------
constexpr int kJoinThreads = 512;

template <typename T, class I>
__global__ void __launch_bounds__(kJoinThreads)
page_attention_join_kernel(Args a) {
  constexpr int DH = I::kDh, QT = I::QT, kLanes = kJoinThreads / QT < 64 ? kJoinThreads / QT : 64;
  __shared__ float s_top[QT], s_total[QT];
  __shared__ alignas(16) floatx4 s_part[kJoinThreads];
  const int tid = threadIdx.x;
  const int32_t *j = a.joins + (int64_t)blockIdx.x * kJoinInts;
  const int n = j[0];
  if (n == 0) return;
  const int row0 = j[1], rows = j[2], len = j[3], head = j[4], tile = j[5];
  const int cols = min(QT, rows * a.group - tile * QT);
  const float *first = partial<I>(a, blockIdx.x, true);
  auto slot = [&](int i) { return i == 0 ? first : first + (int64_t)(2 * i - 1) * I::kSlotFloats; };
  // a thread takes four dimensions of a column; where the workgroup has more threads than that, groups of them take every parts-th result
  const int per_col = a.p.dh / 4, elems = cols * per_col;
  int parts = 1;
  while (2 * parts * elems <= kJoinThreads && parts < n) parts *= 2;
  const int part = parts > 1 ? tid / elems : 0, e_first = parts > 1 ? tid - part * elems : tid;
  constexpr int kAhead = 4;
  floatx4 ahead[kAhead];                                       // the first results are on their way while the maxima are found
  {
    const int col = min(e_first / per_col, QT - 1), d = e_first % per_col * 4;
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      ahead[k] = e_first < elems && part + k * parts < n ? *(const floatx4 *)(slot(part + k * parts) + 2 * QT + col * DH + d) : floatx4{0.f, 0.f, 0.f, 0.f};
  }
  {
    const int col = tid / kLanes;
    float top = -INFINITY, total = 0.f;
    auto merge = [&](float m, float l) {
      const float t = fmaxf(top, m), ref = reference(t);
      total = total * weight(a, top, ref) + l * weight(a, m, ref);
      top = t;
    };
    if (col < cols)
      for (int i = tid % kLanes; i < n; i += kLanes) merge(slot(i)[col], slot(i)[QT + col]);
#pragma unroll
    for (int o = 1; o < kLanes; o <<= 1) merge(__shfl_xor(top, o, kWave), __shfl_xor(total, o, kWave));
    if (col < cols && tid % kLanes == 0) {
      s_top[col] = reference(top);
      s_total[col] = total;
    }
  }
  __syncthreads();
  for (int e0 = 0; e0 < elems; e0 += kJoinThreads) {
    const int e = e0 + e_first;
    const bool live = e < elems && part < parts;
    const int col = live ? e / per_col : 0, d = live ? e % per_col * 4 : 0;
    floatx4 sum = {0.f, 0.f, 0.f, 0.f};
    if (live) {
      int i = part;
      if (e0 == 0) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k, i += parts)
          if (i < n) sum += weight(a, slot(i)[col], s_top[col]) * ahead[k];
      }
#pragma unroll 4
      for (; i < n; i += parts) {
        const float *p = slot(i);
        sum += weight(a, p[col], s_top[col]) * *(const floatx4 *)(p + 2 * QT + col * DH + d);
      }
    }
    if (parts > 1) {
      s_part[tid] = sum;
      __syncthreads();
      if (live && part == 0)
        for (int k = 1; k < parts; ++k) sum += s_part[tid + k * elems];
    }
    if (live && part == 0) {
      int row;
      const int64_t at = row_place(a, row0, head, tile * QT + col, a.p.out_stride, &row);
      store4((T *)a.p.out + at + d, sum, 1.0f / s_total[col], limit_of(a, len, rows, row) <= 0);
    }
  }
}

// ---- host side -----------------------------------------------------------------------------------
struct Plan { int workers; bool whole; };
template <class I>
constexpr int64_t kPartialBytes = 2 * I::kSlotFloats * (int64_t)sizeof(float) + kJoinInts * (int64_t)sizeof(int32_t);   // a worker's

// Workers of a call: as many as the chip holds at once, or fewer where there is no more to do; whole triples where no request is long.
template <class I>
Plan plan(int B, int M, int Hkv, int group, int width, int page_size) {
  const int64_t tiles = (int64_t)M * group / I::QT + (B < M ? B : M), triples = tiles * Hkv;
  const int64_t steps = ((int64_t)width * page_size + I::kStep - 1) / I::kStep;
  // what fits the chip, and PVF_PAGE_WORKSPACE: a number that 8 divides, for the order of workers on the XCDs
  constexpr int64_t kRoom = PVF_PAGE_WORKSPACE / kPartialBytes<I> / 8 * 8, most = 256 * I::kPerCu < kRoom ? 256 * I::kPerCu : kRoom;
  Plan p;
  p.whole = steps <= I::kWholeSteps;
  const int64_t want = p.whole ? triples : triples * steps;
  p.workers = (int)(want < (p.whole ? 4 * most : most) ? want : (p.whole ? 4 * most : most));
  return p;
}
template <class I>
int64_t workspace_bytes(const Plan &p) {
  return p.whole || p.workers == 1 ? 0 : p.workers * kPartialBytes<I>;
}

// What a launch of instance I needs beside its arguments.
template <class I>
Plan prepare(Args &a) {
  const Plan p = plan<I>(a.p.B, a.p.M, a.p.Hkv, a.group, a.p.width, a.p.page_size);
  a.whole = p.whole || p.workers == 1;
  a.joins = a.whole ? nullptr : (int32_t *)(a.p.ws + (int64_t)p.workers * 2 * I::kSlotFloats);
  const int64_t chunk = (int64_t)(kPageSlots - 2) * a.p.page_size / I::kStep;
  a.chunk_steps = (int)(chunk < 1 << 20 ? chunk : 1 << 20);
  return p;
}

// more than 32 columns a tile, bf16 and d_head up to 128 (paged_attention_wide.hip)
pvf_status launch_wide(hipStream_t s, Args &a, int64_t pairs);
int64_t wide_workspace(int B, int M, int Hkv, int group, int dh, int width, int page_size, int64_t pairs);

}  // namespace page
}  // namespace pvf
