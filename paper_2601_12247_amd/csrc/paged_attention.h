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
constexpr int kCus = 256;

struct Args {
  PageAttention p;
  int32_t group, chunk_steps;             // heads a key head; steps whose pages fit kPageSlots
  uint32_t div_mul, div_shift;            // page of a key
  float c;                                // |scale| * log2(e), above zero: scores are compared before they are scaled,
  uint32_t q_xor;                         // and the sign of a negative scale goes into q
  int32_t whole;                          // 1: the line is of triples, not steps (host)
  int32_t workers;                        // workgroups between which triples may be divided: the grid's first
  int32_t *joins;                         // [workers][kJoinInts]: the triple that worker w begins and others end
};
constexpr int kJoinInts = 8;              // workers that took it (0: none), its first row, rows, length as told, key head, tile

struct Request {
  int row0, n, len, steps, tiles;         // its rows, keys in its table, steps of keys and tiles of columns
  int told;                               // its length, by which rows see: more than len if it is
  bool over;                              // longer than its table: keys are NaN, so every row is that sees one
};

// Keys that row `row` of a request sees whose length is `told`.
__device__ __forceinline__ int limit_of(const Args &a, int told, int n, int row) { return a.p.causal ? told - n + row + 1 : told; }

// The part of a triple that a worker takes next.
struct Piece {
  int step0, step1, head, tile, cols;
  bool done, begun;                       // all of it; from its first step on
};

// The line, 64 requests at a time, one a lane, and a worker's place on it.  Its items are `chunk` steps of a triple each, the last of a triple as many as are
// left: single steps, whole triples, or what gives each worker one item.  Triples are below 2^31 (rows and heads together are); a line of that many steps
// is one of whole triples.
template <class I>
struct Line {
  const Args &a;
  int row0, n, len;                       // this lane's; row0 with kOver set: longer than its table
  uint32_t upto, base;                    // items up to it and its own; in front of these 64
  int b0, b;                              // the first of these 64; the request of the last piece
  uint32_t chunk;
  uint32_t at, end, share;
  uint32_t rest_at, rest_end;             // the worker's items of steps behind those, of triples that are divided
  uint32_t left;                          // items of the last piece's triple behind it

  static constexpr int kOver = 1 << 30;
  static constexpr int kTogether = 4;     // times 64 requests on their way at once, where there are more than 64 (4096 of 16 keys: 84.3 -> 69.6 us)
  static constexpr uint32_t kWhole = 1u << 30;                 // more steps than a triple has

  __device__ __forceinline__ static int steps_of(int len) { return max((len + I::kStep - 1) / I::kStep, 1); }
  __device__ __forceinline__ int tiles_of(int rows) const { return (int)(((uint32_t)(rows * a.group) + I::QT - 1) / I::QT); }
  __device__ __forceinline__ uint32_t triples_of(int rows) const { return (uint32_t)tiles_of(rows) * (uint32_t)a.p.Hkv; }
  __device__ __forceinline__ uint32_t chunks_of(int keys) const { return chunk == 1 ? (uint32_t)steps_of(keys) : ((uint32_t)steps_of(keys) + chunk - 1) / chunk; }
  __device__ __forceinline__ uint32_t items_of(int rows, int keys) const { return triples_of(rows) * chunks_of(keys); }

  struct Raw { int len, r0, r1; };
  __device__ __forceinline__ Raw fetch(int from) const {
    const int i = from + (threadIdx.x & 63);
    Raw w = {0, 0, 0};
    if (i < a.p.B) {
      w = {a.p.seq_len[i], i, i + 1};
      if (a.p.cu_rows) {
        w.r0 = a.p.cu_rows[i];
        w.r1 = a.p.cu_rows[i + 1];
      }
    }
    return w;
  }
  __device__ __forceinline__ void take(int from, const Raw &w) {
    const int most = a.p.width * a.p.page_size;
    b0 = from;
    row0 = min(max(w.r0, 0), a.p.M);
    n = max(min(max(w.r1, 0), a.p.M) - row0, 0);   // (an offset far below zero less row0 would wrap)
    len = min(max(w.len, 0), most);
    if (w.len > most) row0 |= kOver;
  }
  __device__ __forceinline__ void load(int from) { take(from, fetch(from)); }

  // Triples stay whole where the host says so.  Else, unless one is longer than its share of all steps by more than kSplit (what dividing costs, in steps):
  // where they are fewer than workers, each CU takes one and the rest is divided between the workers that have none; where they are more, instances with
  // large partial results leave them whole, for the grid's workgroups as they come (a longest one at the end then costs less than dividing).  On the others
  // a few triples (half the CUs) are divided, too.
  //   bf16, 9 x 32 triples of 128 columns, 1280 keys: 65.4 us; 70.6 if none is divided, 81 with equal shares of all steps
  //   bf16, 20 x 32 of them: 126 us (94 with lengths from half of that on); 154 (124) with equal shares
  //   bf16, 32 x 8 triples of one column, 2048 keys: 45.8 us; 49.8 with equal shares
  __device__ __forceinline__ Line(const Args &args, int block, int grid, int *worker) : a(args) {
    const uint32_t workers = (uint32_t)a.workers;
    chunk = a.whole ? kWhole : 1;
    uint32_t sum = 0, all_triples = 0;
    int longest = 0;
    auto add = [&](int from, const Raw &w) {
      take(from, w);
      const uint32_t mine = items_of(n, len);
      sum = __builtin_elementwise_add_sat(sum, chunk == 1 && __umulhi(triples_of(n), (uint32_t)steps_of(len)) ? 0xffffffffu : mine);
      longest = max(longest, n > 0 ? steps_of(len) : 0);
      all_triples += triples_of(n);
    };
    if (a.p.B <= kWave) {
      add(0, fetch(0));
    } else {
      for (int from = 0; from < a.p.B; from += kTogether * kWave) {
        Raw w[kTogether];
#pragma unroll
        for (int k = 0; k < kTogether; ++k) w[k] = fetch(from + k * kWave);
#pragma unroll
        for (int k = 0; k < kTogether; ++k) add(from + k * kWave, w[k]);
      }
    }
    uint32_t all = last_lane(wave_scan(sum));
    share = (all + workers - 1) / workers;
    *worker = block;
    base = rest_at = rest_end = 0;
    const bool counted = chunk != 1 || all >> 31;
    auto longer = [&](uint32_t cus) { return __builtin_amdgcn_ballot_w64((uint32_t)longest > all / cus + I::kSplit) != 0; };
    if (!counted && !longer(kCus)) {
      const uint32_t t = last_lane(wave_scan(all_triples));
      const bool many = t >= workers - workers / 8;
      if (many ? I::kAsTheyCome && !longer(2 * kCus) : I::kAsTheyCome || t >= kCus / 2) {
        const uint32_t takers = many ? (uint32_t)grid : min(workers, (uint32_t)kCus), each = (t + takers - 1) / takers, dealt = many ? t : min(t, takers);
        if (dealt < t) {                  // steps of the triples that are dealt out lie in front of the others'
          if (a.p.B > kWave) load(0);
          uint32_t t0 = 0, s0 = 0;
          for (;;) {
            const uint32_t t1 = t0 + wave_scan(triples_of(n)), s1 = s0 + wave_scan(items_of(n, len));
            const uint64_t beyond = __builtin_amdgcn_ballot_w64(t1 > dealt);
            if (beyond || b0 + kWave >= a.p.B) {
              const int l = beyond ? __builtin_ctzll(beyond) : 63;
              const uint32_t behind = (uint32_t)__builtin_amdgcn_readlane((int)t1, l) - dealt;      // of this request's triples
              s0 = (uint32_t)__builtin_amdgcn_readlane((int)s1, l) - behind * (uint32_t)steps_of(__builtin_amdgcn_readlane(len, l));
              break;
            }
            t0 = last_lane(t1);
            s0 = last_lane(s1);
            load(b0 + kWave);
          }
          const uint32_t others = workers - takers;                                                 // more triples than CUs, fewer than workers
          share = (all - s0 + others - 1) / others;
          if ((uint32_t)block >= takers && (uint32_t)block < workers) {
            rest_at = min(s0 + share * ((uint32_t)block - takers), all);
            rest_end = min(rest_at + share, all);
          }
        }
        chunk = kWhole;
        const uint32_t of_each = many ? each : 1;
        at = (uint32_t)block < takers ? min((uint32_t)block * of_each, dealt) : dealt;
        end = min(at + of_each, dealt);
        begin();
        return;
      }
    }
    if (counted && chunk == 1) {
      chunk = kWhole;
      all = last_lane(wave_scan(all_triples));
      share = (all + workers - 1) / workers;
    }
    if (chunk == 1 && share > 1 && a.p.B <= kWave) {
      // A second piece costs a worker some steps (rows anew, its first keys, another result): each has one, if parts an eighth longer do.
      // 17 requests of up to 1411 keys, f32: 17.0 us, 19.8 with shares of steps that end anywhere.
      for (uint32_t more = 0; more < 3; ++more) {
        chunk = share + (more < 2 ? more : 1 + share / 8);
        const uint32_t items = last_lane(wave_scan(items_of(n, len)));
        if (items <= workers) {
          all = items;
          share = 1;
          break;
        }
        chunk = 1;
      }
    }
    // workers that follow each other read the same keys for other columns: where all take part, neighbours run on one XCD and share its L2
    if (workers % 8 == 0 && share * (workers - 1) < all && (uint32_t)block < workers) *worker = block % 8 * ((int)workers / 8) + block / 8;
    at = (uint32_t)block < workers ? min(share * (uint32_t)*worker, all) : all;
    end = min(at + share, all);
    begin();
  }

  __device__ __forceinline__ void begin() {
    base = 0;
    if (a.p.B > kWave) load(0);
    upto = wave_scan(items_of(n, len));
  }

  // False: nothing is left.  (A b that leaves the requests, or a head: lengths have changed under the call.)
  __device__ __forceinline__ bool next(Request &r, Piece &p) {
    if (at >= end) {
      if (rest_at >= rest_end) return false;
      at = rest_at;
      end = rest_end;
      rest_end = 0;
      chunk = 1;
      begin();
    }
    uint64_t beyond = __builtin_amdgcn_ballot_w64(upto > at);
    while (beyond == 0) {
      const int from = b0 + kWave;
      if (from >= a.p.B) return false;
      Raw w[kTogether];
#pragma unroll
      for (int k = 0; k < kTogether; ++k) w[k] = fetch(from + k * kWave);
#pragma unroll
      for (int k = 0; k < kTogether; ++k)
        if (beyond == 0) {
          base = last_lane(upto);
          take(from + k * kWave, w[k]);
          upto = base + wave_scan(items_of(n, len));
          beyond = __builtin_amdgcn_ballot_w64(upto > at);
        }
    }
    const int l = __builtin_ctzll(beyond);
    auto of = [&](int x) { return __builtin_amdgcn_readlane(x, l); };
    b = b0 + l;
    r.row0 = of(row0) & ~kOver;
    r.over = (of(row0) & kOver) != 0;
    r.n = of(n);
    r.len = r.told = of(len);
    if (r.over) r.told = max(a.p.seq_len[b], r.len);
    r.steps = steps_of(r.len);
    r.tiles = tiles_of(r.n);
    const uint32_t rel = at - ((uint32_t)of((int)upto) - items_of(r.n, r.len)), chunks = chunks_of(r.len), triple = chunks == 1 ? rel : rel / chunks;
    const uint32_t first = rel - triple * chunks, count = min(chunks - first, end - at);
    p.step0 = (int)(first * chunk);
    p.step1 = (int)min((uint32_t)r.steps, (first + count) * chunk);
    at += count;
    left = chunks - first - count;
    p.head = (int)(triple / (uint32_t)r.tiles);
    p.tile = (int)(triple - (uint32_t)p.head * (uint32_t)r.tiles);
    p.cols = min(I::QT, r.n * a.group - p.tile * I::QT);
    p.begun = p.step0 == 0;
    p.done = p.begun && p.step1 == r.steps;
    return p.head < a.p.Hkv;
  }

  // Notes how many workers take a triple that this one begins: others end it, `share` items each.
  __device__ __forceinline__ void note_join(int worker, const Request &r, const Piece &p) const {
    int32_t *j = a.joins + (int64_t)worker * kJoinInts;
    *(int4 *)(j + 4) = make_int4(p.head, p.tile, 0, 0);
    *(int4 *)j = make_int4((int)((left + share - 1) / share) + 1, r.row0, r.n, r.told);
  }
};

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

// Table entries of keys k0 .. k1 - 1 into LDS, -1 for what is no page; *s_bad (zero before, if given) becomes one if there is such.
__device__ __forceinline__ void load_pages(const Args &a, int b, int k0, int k1, int first_page, int32_t *s_pages, int32_t *s_bad) {
  const int n = k1 > k0 ? page_of(a, k1 - 1) - first_page + 1 : 0;
  const int32_t *row = a.p.table + (int64_t)b * a.p.table_stride + first_page;
  for (int i = threadIdx.x; i < n; i += 256) {
    int id = -1;
    if (first_page + i < a.p.width) id = row[i];
    const bool there = (uint32_t)id < (uint32_t)a.p.n_pages;
    s_pages[i] = there ? id : -1;
    if (s_bad && !there) *s_bad = 1;
  }
}
// Every wave's LDS accesses so far are done; loads from global memory stay on their way.
__device__ __forceinline__ void meet() {
  __builtin_amdgcn_s_waitcnt(0xc07f);     // lgkmcnt(0)
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

__device__ __forceinline__ bool bf16s_not_finite(uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; }
__device__ __forceinline__ uint32_t bf16s_finite(uint32_t w) {   // what is not finite as zero
  if ((w & 0x7f800000u) == 0x7f800000u) w &= 0xffffu;
  if ((w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u;
  return w;
}

// y (float32 bits) where it is not finite, else zero: what a key adds whose probability is not zero
__device__ __forceinline__ float odd_part(uint32_t y) { return (y & 0x7f800000u) == 0x7f800000u ? __uint_as_float(y) : 0.f; }

// Two probabilities as bf16 in two parts: the upper halves, and the rest of 16 bits.  The rest is never zero beside p > 2^-110 (2^-23 of p is added, and
// bf16 ends at 2^-133): zero times an infinite value would make NaN of infinity.
__device__ __forceinline__ uint32_t upper_parts(float x, float y) { return __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302); }
__device__ __forceinline__ uint32_t lower_parts(float x, float y) {
  auto low = [](float p) { return (bf16_t)__builtin_fmaf(p, 1.0f + 0x1p-23f, -__uint_as_float(__float_as_uint(p) & 0xffff0000u)); };
  const bf16x2 r = {low(x), low(y)};
  return __builtin_bit_cast(uint32_t, r);
}

// ---- the join: block w joins the triple that worker w begins, if others end it ----------------------
// A wait for the notes, one for the maxima and results, one sum over LDS: latency.  8 triples of 64 results of 4 columns 5.8 us, 68 of up to 8 results of 15
// columns 4.8, the 32 divided ones of 9 x 32 windows 8.2.  Sixteen or eight columns of a wide tile to a workgroup took 5 and 12 us more.
constexpr int kJoinThreads = 1024;
template <class I>
constexpr int kJoinCols = I::QT < 32 ? I::QT : 32;   // columns of a block

template <typename T, class I>
__global__ void __launch_bounds__(kJoinThreads)
page_attention_join_kernel(Args a) {
  constexpr int DH = I::kDh, QT = I::QT, kCols = kJoinCols<I>, kLanes = kJoinThreads / kCols;
  __shared__ float s_top[kCols], s_total[kCols];
  __shared__ alignas(16) floatx4 s_part[kJoinThreads];
  const int tid = threadIdx.x;
  const int32_t *j = a.joins + (int64_t)blockIdx.x * kJoinInts;
  const int n = min(j[0], (int)(gridDim.x + 1 - blockIdx.x));    // (more only if lengths have changed under the call)
  if (n == 0) return;
  const int row0 = j[1], rows = j[2], told = j[3], head = j[4], tile = j[5], col0 = blockIdx.y * kCols;
  const int cols = min(kCols, rows * a.group - tile * QT - col0);
  if (cols <= 0) return;
  const float *first = partial<I>(a, blockIdx.x, true) + col0;
  auto slot = [&](int i) { return i == 0 ? first : first + (int64_t)(2 * i - 1) * I::kSlotFloats; };       // m; l lies QT, O 2 QT + col0 (DH - 1) behind it
  // A thread takes four dimensions of a column; where the workgroup has more threads than that, groups of them take every parts-th result.  Eight
  // results at a time are on their way, the first eight while the maxima are found.
  const int per_col = a.p.dh / 4, elems = cols * per_col;      // at most kJoinThreads where d_head is at most 128
  int parts = 1;
  while (2 * parts * elems <= kJoinThreads && parts < n) parts *= 2;
  const int part = parts > 1 ? tid / elems : 0, e_first = parts > 1 ? tid - part * elems : tid;
  constexpr int kAhead = 8;
  floatx4 o[kAhead];
  float m[kAhead];
  auto fetch = [&](int i, int e) {
    const int col = e / per_col;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const float *p = slot(min(i + k * parts, n - 1));
      m[k] = p[col];
      o[k] = *(const floatx4 *)(p + 2 * QT + col0 * (DH - 1) + col * DH + e % per_col * 4);
    }
  };
  const bool any = e_first < elems && part < parts;
  if (any) fetch(part, e_first);
  {
    const int col = tid / kLanes;
    float top = -INFINITY, total = 0.f;
    auto merge = [&](float m1, float l1) {
      const float t = fmaxf(top, m1), ref = reference(t);
      total = total * weight(a, top, ref) + l1 * weight(a, m1, ref);
      top = t;
    };
    if (col < cols)
      for (int i = tid % kLanes; i < n; i += kLanes) merge(slot(i)[col], slot(i)[QT + col]);
#pragma unroll
    for (int off = 1; off < kLanes; off <<= 1) merge(__shfl_xor(top, off, kWave), __shfl_xor(total, off, kWave));
    if (col < cols && tid % kLanes == 0) {
      s_top[col] = reference(top);
      s_total[col] = total;
    }
  }
  __syncthreads();
  for (int e0 = 0; e0 < elems; e0 += kJoinThreads) {
    const int e = e0 + e_first;
    const bool live = e < elems && part < parts;
    const int col = live ? e / per_col : 0;
    floatx4 sum = {0.f, 0.f, 0.f, 0.f};
    if (live) {
      for (int i = part; i < n; i += kAhead * parts) {
        if (e0 > 0 || i > part) fetch(i, e);
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
          if (i + k * parts < n) sum += weight(a, m[k], s_top[col]) * o[k];
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
      const int64_t to = row_place(a, row0, head, tile * QT + col0 + col, a.p.out_stride, &row);
      store4((T *)a.p.out + to + e % per_col * 4, sum, 1.0f / s_total[col], limit_of(a, told, rows, row) <= 0);
    }
  }
}

// ---- host side -----------------------------------------------------------------------------------
struct Plan { int workers, grid; bool whole; };
template <class I>
constexpr int64_t kPartialBytes = 2 * I::kSlotFloats * (int64_t)sizeof(float) + kJoinInts * (int64_t)sizeof(int32_t);   // a worker's

// Workers of a call: as many as the chip holds at once, or fewer where there is no more to do.  Triples stay whole, which saves the second launch, where
// none can be long: up to kWholeSteps steps, or twice that where they fill half the chip.  (What a table has room for counts, lengths are on the device.)
//   bf16, one column, 128 keys a step: 8 triples of 4 steps 10.4 us whole, 10.5 divided, of 6 steps 12.6 and 10.7; 128 triples of 8 steps 16.8 and 21.6
//   f32, 64 keys a step: 8 triples of 4 steps 13.2 and 11.9, of 2 steps 9.8 and 11.6; 128 triples of 8 steps 22.5 and 24.1, of 12 steps 29.9 and 28.6
//   bf16, 128 columns, 64 keys a step: 8 triples of 8 steps 20.4 and 22.8, of 12 steps 27.0 and 18.9; 128 triples of 16 steps 34.8 and 38.9
template <class I>
Plan plan(int B, int M, int Hkv, int group, int width, int page_size) {
  const int64_t tiles = (int64_t)M * group / I::QT + (B < M ? B : M), triples = tiles * Hkv;
  const int64_t steps = ((int64_t)width * page_size + I::kStep - 1) / I::kStep;
  // what fits the chip, and PVF_PAGE_WORKSPACE: a number that 8 divides, for the order of workers on the XCDs
  constexpr int64_t kRoom = PVF_PAGE_WORKSPACE / kPartialBytes<I> / 8 * 8, most = kCus * I::kPerCu < kRoom ? kCus * I::kPerCu : kRoom, kGrid = 4 * kCus * I::kPerCu;
  const int64_t grid = triples < kGrid ? triples : kGrid;
  Plan p;
  p.whole = steps <= (triples < kCus / 2 ? 1 : 2) * I::kWholeSteps;
  // (every workgroup looks at all lengths: 256 x 8 triples of one column and 16 keys 20.6 us, 31.5 on four times as many)
  if (p.whole) p.workers = (int)(I::kAsTheyCome || grid < most ? grid : most);
  else p.workers = (int)(triples * steps < most ? triples * steps : most);
  p.grid = I::kAsTheyCome && grid > p.workers ? (int)grid : p.workers;
  return p;
}
template <class I>
int64_t workspace_bytes(int B, int M, int Hkv, int group, int width, int page_size) {
  const Plan p = plan<I>(B, M, Hkv, group, width, page_size);
  return p.whole || p.workers == 1 ? 0 : p.workers * kPartialBytes<I>;
}

// What a launch of instance I needs beside its arguments.
template <class I>
Plan prepare(Args &a) {
  const Plan p = plan<I>(a.p.B, a.p.M, a.p.Hkv, a.group, a.p.width, a.p.page_size);
  a.whole = p.whole || p.workers == 1;
  a.workers = p.workers;
  a.joins = a.whole ? nullptr : (int32_t *)(a.p.ws + (int64_t)p.workers * 2 * I::kSlotFloats);
  const int64_t chunk = (int64_t)(kPageSlots - 2) * a.p.page_size / I::kStep;
  a.chunk_steps = (int)(chunk < 1 << 20 ? chunk : 1 << 20);
  return p;
}

// many columns, bf16 (paged_attention_wide.hip)
pvf_status launch_wide(hipStream_t s, Args &a, int64_t pairs);
int64_t wide_workspace(int B, int M, int Hkv, int group, int dh, int width, int page_size, int64_t pairs);

}  // namespace page
}  // namespace pvf
