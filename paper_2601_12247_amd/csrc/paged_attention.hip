// Attention of rows against keys and values in pages: out = softmax(scale q k^T) v over the keys that a row sees, one pass with the running
// maximum and sum of the softmax (in units of log2).
//
// Matrix instructions compute S^T = K Q^T and O^T = V^T P^T, 16 columns a block: the (row, head) pairs that share a key head.  A lane of S^T holds
// one column and keys 4 g .. 4 g + 3 of every 16 (g = lane / 16), which is a lane's share of the operand P^T if the keys of V^T are taken in the
// same order, so scores never leave their lane.  Keys and values go from the pages straight into registers, a whole row of a value by 16 lanes:
// lane c holds dimensions VE c .. of four neighbouring keys, and operand j of the matrix instruction is made of dimension VE c + j of those.
//
// P enters the bf16 instruction as two bf16 parts (16 bits of it): the second instruction costs nothing beside the memory, and the result is
// rounded once, to its own type.
#include "paged.h"

#include <algorithm>
#include <cmath>

namespace pvf {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

constexpr int kPageSlots = 1024;          // table entries in LDS

struct Args {
  PageAttention p;
  int64_t share_min;
  int32_t group, chunk_steps;             // heads a key head; steps whose pages fit kPageSlots
  uint32_t div_mul, div_shift;            // page of a key
  float scale2;                           // scale * log2(e)
  int32_t whole;                          // 1: a worker takes whole (request, head, tile of columns) triples
};

// Sizes of an instance: T, d_head up to DH, 16 NQ columns a tile.
template <typename T, int DH, int NQ>
struct Inst {
  static constexpr bool kBf16 = sizeof(T) == 2;
  static constexpr int KT = kBf16 ? 32 : 16;            // keys a wave takes at once
  static constexpr int NU = KT / 16;
  static constexpr int KE = kBf16 ? 8 : 4;              // elements of a key row a lane loads at once
  static constexpr int KJ = DH / (4 * KE);
  static constexpr int VE = kBf16 && DH >= 128 ? 8 : 4;
  static constexpr int NB = DH / (16 * VE), NT = DH / 16;
  static constexpr int kStep = 4 * KT;                  // keys a workgroup takes at once
  static constexpr int QT = 16 * NQ;
  static constexpr int kOPad = DH + 4;
  static constexpr int kSlotFloats = QT * (DH + 2);     // a partial result: m[QT], l[QT], O[QT][DH]
  static constexpr int kRegs = (NT + KJ + 2) * 4 * NQ + NU * KJ * 4 + NU * 4 * NB * VE * (int)sizeof(T) / 4 + 64;   // about
  static constexpr int kPerCu = kRegs <= 256 ? 2 : 1;   // workgroups of 4 waves
};

// ---- which keys and columns belong to which worker ----------------------------------------------
struct Request {
  int row0, n, len, steps, tiles;         // its rows, visible keys, steps of keys and tiles of columns
  bool over;                              // longer than its table
  int64_t items;
};

template <class I>
__device__ __forceinline__ Request request(const Args &a, int b) {
  Request r;
  if (a.p.cu_rows) {
    r.row0 = min(max(a.p.cu_rows[b], 0), a.p.M);
    r.n = max(min(a.p.cu_rows[b + 1], a.p.M) - r.row0, 0);
  } else {
    r.row0 = b;
    r.n = 1;
  }
  const int len = max(a.p.seq_len[b], 0), most = a.p.width * a.p.page_size;
  r.len = min(len, most);
  r.over = len > most;
  r.steps = max((r.len - 1) / I::kStep + 1, 1);
  r.tiles = (int)(((int64_t)r.n * a.group + I::QT - 1) / I::QT);
  r.items = (int64_t)r.tiles * a.p.Hkv * (a.whole ? 1 : r.steps);
  return r;
}

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

// All items, and each worker's share of them.
template <class I>
__device__ __forceinline__ int64_t all_items(const Args &a) {
  const int lane = threadIdx.x & 63;
  int64_t sum = 0;
  for (int b = lane; b < a.p.B; b += kWave) sum += request<I>(a, b).items;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, kWave);
  return uniform64(sum);
}
__device__ __forceinline__ int64_t share_of(const Args &a, int64_t items, int workers) { return max(a.share_min, (items + workers - 1) / workers); }

// The request that item `at` (below all_items) belongs to, and its first item.
template <class I>
__device__ __forceinline__ int find_request(const Args &a, int64_t at, int64_t *first) {
  const int lane = threadIdx.x & 63;
  int64_t base = 0;
  for (int b0 = 0;; b0 += kWave) {
    const int b = b0 + lane;
    const int64_t items = b < a.p.B ? request<I>(a, b).items : 0, upto = base + wave_scan(items);
    const uint64_t beyond = __builtin_amdgcn_ballot_w64(upto > at);
    if (beyond || b0 + kWave >= a.p.B) {
      const int l = beyond ? __builtin_ctzll(beyond) : 63;
      *first = uniform64(__shfl(upto - items, l, kWave));
      return __builtin_amdgcn_readfirstlane(min(b0 + l, a.p.B - 1));
    }
    base = uniform64(__shfl(upto, 63, kWave));
  }
}

// Keys that a row sees.
__device__ __forceinline__ int limit_of(const Args &a, const Request &r, int row) { return a.p.causal ? r.len - r.n + row + 1 : r.len; }

// ---- the pass over the keys ----------------------------------------------------------------------
template <typename T, int DH, int NQ, bool kWhole>
struct Pass {
  typedef Inst<T, DH, NQ> I;
  struct alignas(I::VE * sizeof(T)) Val { uint32_t w[I::VE * sizeof(T) / 4]; };
  struct Tile {
    uint4 k[I::NU][I::KJ];
    Val v[I::NU][4][I::NB];
    bool bad[I::NU];                      // keys 4 g .. of these 16 lie on a page that is none
  };

  const Args &a;
  const int32_t *pages;                   // LDS: table entries from first_page on, -1: no page
  int first_page, len, lane, c, g;
  bool over;                              // keys lie behind the table
  const T *kbase, *vbase;                 // at the head
  uint4 q[NQ][I::KJ];
  int limit[NQ], least;                   // keys each column sees; the fewest of the wave's columns
  floatx4 o[NQ][I::NT];
  float m[NQ], l[NQ];
  Tile t;                                 // the tile under way

  __device__ __forceinline__ Pass(const Args &args, const int32_t *s_pages) : a(args), pages(s_pages) {
    lane = threadIdx.x & 63;
    c = lane & 15;
    g = lane >> 4;
  }

  __device__ __forceinline__ int64_t place(int key, int64_t page_stride, bool *none) const {
    const int page = (int)(__umulhi((uint32_t)(key >> 3) << 1, a.div_mul) >> a.div_shift);
    const int id = pages[page - first_page];
    *none = id < 0;
    return (int64_t)max(id, 0) * page_stride + (int64_t)((key - page * a.p.page_size) * a.p.dh);
  }

  // Keys kb .. kb + KT - 1, kb < len; the ones behind the last are read as copies of it.
  __device__ __forceinline__ void load_keys(int kb) {
#pragma unroll
    for (int u = 0; u < I::NU; ++u) {
      bool none;
      const T *p = kbase + place(min(kb + 16 * u + c, len - 1), a.p.k_page_stride, &none) + I::KE * g;
#pragma unroll
      for (int j = 0; j < I::KJ; ++j)
        t.k[u][j] = kWhole || j * 4 * I::KE + I::KE * g < a.p.dh ? *(const uint4 *)(p + j * 4 * I::KE) : make_uint4(0, 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  __device__ __forceinline__ void load_values(int kb) {
#pragma unroll
    for (int u = 0; u < I::NU; ++u) {
      const T *p = vbase + place(min(kb + 16 * u + 4 * g, (len - 1) & ~3), a.p.v_page_stride, &t.bad[u]) + I::VE * c;
      t.bad[u] |= over;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int nb = 0; nb < I::NB; ++nb) {
          Val v = {};
          if (kWhole || nb * 16 * I::VE + I::VE * c < a.p.dh) v = *(const Val *)(p + i * a.p.dh + nb * 16 * I::VE);
          t.v[u][i][nb] = v;
        }
    }
    __builtin_amdgcn_sched_barrier(0);
  }

  __device__ __forceinline__ static bool not_finite(uint32_t w) {
    return I::kBf16 ? (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u : (w & 0x7f800000u) == 0x7f800000u;
  }

  // What the values of this tile that are not finite add to column block nq: of the keys that a column sees, no others.  The values are read
  // again; p (what the tile's keys have in S^T's place) comes from the lane that holds it.
  __device__ __forceinline__ void add_not_finite(int nq, const floatx4 (&p)[I::NU], int kb) {
#pragma unroll 1
    for (int x = 0; x < I::KT; ++x) {
      const int key = kb + x;
      if (key >= len) break;
      float mine = 0.f;
#pragma unroll
      for (int u = 0; u < I::NU; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) mine = x / 16 == u && x % 4 == i ? p[u][i] : mine;
      const float px = __shfl(mine, x % 16 / 4 * 16 + c, kWave);
      bool none;
      const T *v = vbase + place(key, a.p.v_page_stride, &none);
#pragma unroll
      for (int nb = 0; nb < I::NB; ++nb)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < I::VE; ++j) {
            const int d = nb * 16 * I::VE + I::VE * (4 * g + i) + j;
            const float y = kWhole || d < a.p.dh ? to_float(v[d]) : 0.f;
            if (key < limit[nq] && !(fabsf(y) < INFINITY)) o[nq][nb * I::VE + j][i] += px * y;
          }
    }
  }

  // O^T += V^T P^T
  __device__ __forceinline__ void add_values(const uint4 (&ph)[NQ], const uint4 (&pl)[NQ], const floatx4 (&pf)[NQ]) {
#pragma unroll
    for (int nb = 0; nb < I::NB; ++nb)
#pragma unroll
      for (int j = 0; j < I::VE; ++j) {
        const int at = nb * I::VE + j;
        if constexpr (I::kBf16) {
          const uint32_t sel = j % 2 ? 0x07060302 : 0x05040100;
          auto two = [&](int u, int i) { return __builtin_amdgcn_perm(t.v[u][i + 1][nb].w[j / 2], t.v[u][i][nb].w[j / 2], sel); };
          const bf16x8 vt = __builtin_bit_cast(bf16x8, make_uint4(two(0, 0), two(0, 2), two(I::NU - 1, 0), two(I::NU - 1, 2)));
#pragma unroll
          for (int nq = 0; nq < NQ; ++nq) {
            o[nq][at] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, __builtin_bit_cast(bf16x8, ph[nq]), o[nq][at], 0, 0, 0);
            o[nq][at] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, __builtin_bit_cast(bf16x8, pl[nq]), o[nq][at], 0, 0, 0);
          }
        } else {
#pragma unroll
          for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[nq][at] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(t.v[0][i][nb].w[j]), pf[nq][i], o[nq][at], 0, 0, 0);
        }
      }
  }

  // The tile at kb, which is loaded; the one at `next` (-1: none) is asked for as soon as its registers are free.
  __device__ __forceinline__ void add(int kb, int next) {
    if (kb + I::KT > len) {               // what lies behind the last key is anything, NaN too
#pragma unroll
      for (int u = 0; u < I::NU; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int nb = 0; nb < I::NB; ++nb)
            if (kb + 16 * u + 4 * g + i >= len) t.v[u][i][nb] = Val{};
    }
    bool bad = t.bad[0];
    if (I::NU == 2) bad |= t.bad[I::NU - 1];
    const bool any_bad = __builtin_amdgcn_ballot_w64(bad) != 0, border = kb + I::KT > least;
    bool odd = false;
    if (border && least < len) {
      // A row's last keys end in this tile and other rows see further.  0 times an infinity is no zero, so values that are not finite leave the
      // products and are added to the columns that see them, by themselves.
      bool mine = false;
#pragma unroll
      for (int u = 0; u < I::NU; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int nb = 0; nb < I::NB; ++nb)
#pragma unroll
            for (int w = 0; w < (int)(sizeof(Val) / 4); ++w) mine |= not_finite(t.v[u][i][nb].w[w]);
      odd = __builtin_amdgcn_ballot_w64(mine) != 0;
      if (odd) {
#pragma unroll
        for (int u = 0; u < I::NU; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int nb = 0; nb < I::NB; ++nb)
#pragma unroll
              for (int w = 0; w < (int)(sizeof(Val) / 4); ++w) {
                uint32_t &x = t.v[u][i][nb].w[w];
                if ((x & 0x7f800000u) == 0x7f800000u) x &= I::kBf16 ? 0xffffu : 0u;
                if (I::kBf16 && (x & 0x7f80u) == 0x7f80u) x &= 0xffff0000u;
              }
      }
    }
    uint4 ph[NQ], pl[NQ];
    floatx4 pf[NQ], sc[NQ][I::NU];
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
      for (int u = 0; u < I::NU; ++u) {
        floatx4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < I::KJ; ++j) {
          if constexpr (I::kBf16) {
            x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, t.k[u][j]), __builtin_bit_cast(bf16x8, q[nq][j]), x, 0, 0, 0);
          } else {
            const floatx4 kf = __builtin_bit_cast(floatx4, t.k[u][j]), qf = __builtin_bit_cast(floatx4, q[nq][j]);
#pragma unroll
            for (int e = 0; e < 4; ++e) x = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[e], qf[e], x, 0, 0, 0);
          }
        }
        sc[nq][u] = x * a.scale2;
      }
    if (next >= 0) load_keys(next);
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
      floatx4 (&s)[I::NU] = sc[nq];
      if (any_bad) {
#pragma unroll
        for (int u = 0; u < I::NU; ++u)
          if (t.bad[u]) s[u] = floatx4{NAN, NAN, NAN, NAN};
      }
      if (border) {
#pragma unroll
        for (int u = 0; u < I::NU; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (kb + 16 * u + 4 * g + i >= limit[nq]) s[u][i] = -INFINITY;
      }
      float top = m[nq];
#pragma unroll
      for (int u = 0; u < I::NU; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, s[u][i]);
      top = fmaxf(top, __shfl_xor(top, 16, kWave));
      top = fmaxf(top, __shfl_xor(top, 32, kWave));
      const float ref = top == -INFINITY ? 0.f : top, alpha = __builtin_amdgcn_exp2f(m[nq] - ref);
      m[nq] = top;
      float sum = 0.f;
#pragma unroll
      for (int u = 0; u < I::NU; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s[u][i] = __builtin_amdgcn_exp2f(s[u][i] - ref);
          sum += s[u][i];
        }
      l[nq] = l[nq] * alpha + sum;
      if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
        for (int at = 0; at < I::NT; ++at) o[nq][at] *= alpha;
      }
      if (odd) add_not_finite(nq, s, kb);
      if constexpr (I::kBf16) {
        auto upper = [&](int u, int i) { return __builtin_amdgcn_perm(__float_as_uint(s[u][i + 1]), __float_as_uint(s[u][i]), 0x07060302); };
        auto rest = [&](int u, int i) {
          typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
          const float x = s[u][i], y = s[u][i + 1];
          // at least 2^-24 of p: a part that is zero would make NaN of an infinite value
          auto low = [](float p) { return (bf16_t)fmaxf(p - __uint_as_float(__float_as_uint(p) & 0xffff0000u), p * 0x1p-24f); };
          const bf16x2 r = {low(x), low(y)};
          return __builtin_bit_cast(uint32_t, r);
        };
        ph[nq] = make_uint4(upper(0, 0), upper(0, 2), upper(I::NU - 1, 0), upper(I::NU - 1, 2));
        pl[nq] = make_uint4(rest(0, 0), rest(0, 2), rest(I::NU - 1, 0), rest(I::NU - 1, 2));
      } else {
        pf[nq] = s[0];
      }
    }
    add_values(ph, pl, pf);
    if (next >= 0) load_values(next);
  }
};

template <typename T, int DH, int NQ, bool kWhole>
__global__ void __launch_bounds__(256, (Inst<T, DH, NQ>::kPerCu))
page_attention_kernel(Args a) {
  typedef Inst<T, DH, NQ> I;
  typedef Pass<T, DH, NQ, kWhole> P;
  __shared__ int32_t s_pages[kPageSlots];
  __shared__ float s_m[4][I::QT], s_l[4][I::QT];
  __shared__ alignas(16) float s_o[4][16][I::kOPad];
  const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t items = all_items<I>(a), share = share_of(a, items, gridDim.x);
  // workers that follow each other read the same keys for other columns: where all take part, neighbours run on one XCD and share its L2
  int worker = blockIdx.x;
  if (gridDim.x % 8 == 0 && share * (gridDim.x - 1) < items) worker = blockIdx.x % 8 * (gridDim.x / 8) + blockIdx.x / 8;
  int64_t at = share * worker;
  const int64_t end = min(at + share, items);
  if (at >= end) return;
  int64_t first;
  int b = find_request<I>(a, at, &first);
  Request r = request<I>(a, b);
  P pass(a, s_pages);
  while (at < end) {
    while (at - first >= r.items) {       // every item lies in a request, so b stays below B while the lengths are left alone
      first += r.items;
      if (++b >= a.p.B) return;
      r = request<I>(a, b);
    }
    int64_t seg;
    int step0, step1;
    if (a.whole) {
      seg = at - first;
      step0 = 0;
      step1 = r.steps;
      ++at;
    } else {
      seg = (at - first) / r.steps;
      step0 = (int)(at - first - seg * r.steps);
      step1 = (int)min((int64_t)r.steps, step0 + (end - at));
      at += step1 - step0;
    }
    const int head = (int)(seg / r.tiles), tile = (int)(seg - (int64_t)head * r.tiles);
    const int cols = (int)min((int64_t)I::QT, (int64_t)r.n * a.group - (int64_t)tile * I::QT);
    pass.len = r.len;
    pass.over = r.over;
    pass.kbase = (const T *)a.p.k_cache + (int64_t)head * a.p.page_size * a.p.dh;
    pass.vbase = (const T *)a.p.v_cache + (int64_t)head * a.p.page_size * a.p.dh;
    pass.least = INT32_MAX;
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
      const int col = 16 * nq + pass.c;
      const int64_t pair = (int64_t)tile * I::QT + col;
      const int row = (int)(pair / a.group), sub = (int)(pair - (int64_t)row * a.group);
      pass.limit[nq] = col < cols ? limit_of(a, r, row) : INT32_MAX;
      pass.least = min(pass.least, pass.limit[nq]);
      const T *src = (const T *)a.p.q + (r.row0 + row) * a.p.q_stride + (int64_t)(head * a.group + sub) * a.p.dh + I::KE * pass.g;
#pragma unroll
      for (int j = 0; j < I::KJ; ++j)
        pass.q[nq][j] = col < cols && (kWhole || j * 4 * I::KE + I::KE * pass.g < a.p.dh) ? *(const uint4 *)(src + j * 4 * I::KE) : make_uint4(0, 0, 0, 0);
      pass.m[nq] = -INFINITY;
      pass.l[nq] = 0.f;
#pragma unroll
      for (int t = 0; t < I::NT; ++t) pass.o[nq][t] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int off = 1; off < 16; off <<= 1) pass.least = min(pass.least, __shfl_xor(pass.least, off, kWave));
    pass.least = __builtin_amdgcn_readfirstlane(pass.least);

    for (int s0 = step0; s0 < step1; s0 += a.chunk_steps) {
      const int s1 = min(step1, s0 + min(a.chunk_steps, step1 - s0));
      const int k0 = s0 * I::kStep, k1 = (int)min((int64_t)r.len, (int64_t)s1 * I::kStep);
      __syncthreads();                    // the last chunk's pages, or the last piece's results, have been read
      pass.first_page = k0 / a.p.page_size;
      const int n = k1 > k0 ? (k1 - 1) / a.p.page_size - pass.first_page + 1 : 0;
      for (int i = tid; i < n; i += 256) {
        const int j = pass.first_page + i;
        int id = -1;
        if (j < a.p.width) id = a.p.table[(int64_t)b * a.p.table_stride + j];
        s_pages[i] = id >= 0 && id < a.p.n_pages ? id : -1;
      }
      __syncthreads();
      int kb = k0 + wid * I::KT;
      if (kb < k1) {
        pass.load_keys(kb);
        pass.load_values(kb);
      }
      while (kb < k1) {
        const int next = kb < k1 - I::kStep ? kb + I::kStep : -1;
        pass.add(kb, next);
        if (next < 0) break;
        kb = next;
      }
    }

    // the four waves' results, and the way out: the rows themselves, or a partial result for page_attention_join_kernel
    const bool done = step0 == 0 && step1 == r.steps;
    float *slot = done ? nullptr : a.p.ws + (int64_t)(2 * worker + (step0 == 0)) * I::kSlotFloats;
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
      float l = pass.l[nq];
      l += __shfl_xor(l, 16, kWave);
      l += __shfl_xor(l, 32, kWave);
      __syncthreads();
      if (pass.g == 0) {
        s_m[wid][16 * nq + pass.c] = pass.m[nq];
        s_l[wid][16 * nq + pass.c] = l;
      }
#pragma unroll
      for (int nb = 0; nb < I::NB; ++nb)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < I::VE; ++j) s_o[wid][pass.c][nb * 16 * I::VE + I::VE * (4 * pass.g + i) + j] = pass.o[nq][nb * I::VE + j][i];
      __syncthreads();
      for (int e = tid; e < 16 * (DH / 4); e += 256) {
        const int cq = e / (DH / 4), d = e % (DH / 4) * 4, col = 16 * nq + cq;
        if (col >= cols || (!kWhole && d >= a.p.dh)) continue;
        float top = s_m[0][col];
#pragma unroll
        for (int w = 1; w < 4; ++w) top = fmaxf(top, s_m[w][col]);
        const float ref = top == -INFINITY ? 0.f : top;
        float total = 0.f;
        floatx4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float f = __builtin_amdgcn_exp2f(s_m[w][col] - ref);
          total += f * s_l[w][col];
          sum += f * *(const floatx4 *)&s_o[w][cq][d];
        }
        if (done) {
          const int64_t pair = (int64_t)tile * I::QT + col;
          const int row = (int)(pair / a.group), sub = (int)(pair - (int64_t)row * a.group);
          const bool none = limit_of(a, r, row) <= 0;
          T *dst = (T *)a.p.out + (r.row0 + row) * a.p.out_stride + (int64_t)(head * a.group + sub) * a.p.dh + d;
          struct alignas(4 * sizeof(T)) { T v[4]; } res;
#pragma unroll
          for (int i = 0; i < 4; ++i) res.v[i] = from_float<T>(none ? 0.f : sum[i] / total);
          *(decltype(res) *)dst = res;
        } else {
          *(floatx4 *)(slot + 2 * I::QT + col * DH + d) = sum;
          if (d == 0) {
            slot[col] = top;
            slot[I::QT + col] = total;
          }
        }
      }
    }
  }
}

// Joins the partial results of every (request, head, tile of columns) that more than one worker took: block w looks at the border between
// workers w and w + 1 and does so if it is the first one in its triple.
template <typename T, int DH, int NQ>
__global__ void __launch_bounds__(256)
page_attention_join_kernel(Args a, int workers) {
  typedef Inst<T, DH, NQ> I;
  __shared__ float s_top[I::QT], s_total[I::QT];
  __shared__ alignas(16) floatx4 s_part[256];
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  const int64_t items = all_items<I>(a), share = share_of(a, items, workers), border = share * (blockIdx.x + 1);
  if (border >= items) return;
  int64_t first;
  const int b = find_request<I>(a, border, &first);
  const Request r = request<I>(a, b);
  const int64_t seg = (border - first) / r.steps, seg_first = first + seg * r.steps;
  if (border == seg_first || share * blockIdx.x > seg_first) return;
  const int head = (int)(seg / r.tiles), tile = (int)(seg - (int64_t)head * r.tiles);
  const int cols = (int)min((int64_t)I::QT, (int64_t)r.n * a.group - (int64_t)tile * I::QT);
  const int from = blockIdx.x, n = (int)((seg_first + r.steps - 1) / share) - from + 1;
  auto slot = [&](int i) { return a.p.ws + (int64_t)(2 * (from + i) + (i == 0)) * I::kSlotFloats; };
  for (int col = wid; col < cols; col += 4) {
    float top = -INFINITY;
    for (int i = lane; i < n; i += kWave) top = fmaxf(top, slot(i)[col]);
    top = wave_max(top);
    const float ref = top == -INFINITY ? 0.f : top;
    float total = 0.f;
    for (int i = lane; i < n; i += kWave) total += __builtin_amdgcn_exp2f(slot(i)[col] - ref) * slot(i)[I::QT + col];
    total = wave_sum(total);
    if (lane == 0) {
      s_top[col] = ref;
      s_total[col] = total;
    }
  }
  __syncthreads();
  // a thread takes four dimensions of a column; where the workgroup has more threads than that, groups of them take every parts-th result
  const int per_col = a.p.dh / 4, elems = cols * per_col;
  int parts = 1;
  while (2 * parts * elems <= 256 && parts < n) parts *= 2;
  for (int e0 = 0; e0 < elems; e0 += 256) {
    const int e = e0 + (parts > 1 ? tid % elems : tid), part = parts > 1 ? tid / elems : 0;
    const bool live = e < elems && part < parts;
    const int col = live ? e / per_col : 0, d = live ? e % per_col * 4 : 0;
    floatx4 sum = {0.f, 0.f, 0.f, 0.f};
    if (live) {
#pragma unroll 8
      for (int i = part; i < n; i += parts) {
        const float *p = slot(i);
        sum += __builtin_amdgcn_exp2f(p[col] - s_top[col]) * *(const floatx4 *)(p + 2 * I::QT + col * DH + d);
      }
    }
    if (parts > 1) {
      s_part[tid] = sum;
      __syncthreads();
      if (live && part == 0)
        for (int k = 1; k < parts; ++k) sum += s_part[tid + k * elems];
    }
    if (live && part == 0) {
      const int64_t pair = (int64_t)tile * I::QT + col;
      const int row = (int)(pair / a.group), sub = (int)(pair - (int64_t)row * a.group);
      const bool none = limit_of(a, r, row) <= 0;
      T *dst = (T *)a.p.out + (r.row0 + row) * a.p.out_stride + (int64_t)(head * a.group + sub) * a.p.dh + d;
      struct alignas(4 * sizeof(T)) { T v[4]; } res;
#pragma unroll
      for (int i = 0; i < 4; ++i) res.v[i] = from_float<T>(none ? 0.f : sum[i] / s_total[col]);
      *(decltype(res) *)dst = res;
    }
  }
}

// ---- choice of an instance -----------------------------------------------------------------------
struct Choice { int dh, nq, workers; bool whole; int64_t slot_floats; };

// Columns of a tile by the mean number of (row, head) pairs that share a key head; few enough workers that a partial result each fits.
template <class F>
auto with_instance(int dtype, int M, int B, int group, int dh, F f) {
  const int64_t pairs = ((int64_t)M + B - 1) / B * group;
  const int nq = pairs <= 16 ? 1 : pairs <= 32 ? 2 : 4;
  if (dtype == PVF_BF16) {
    if (dh <= 64) return nq == 1 ? f(Inst<bf16_t, 64, 1>{}) : nq == 2 ? f(Inst<bf16_t, 64, 2>{}) : f(Inst<bf16_t, 64, 4>{});
    if (dh <= 128) return nq == 1 ? f(Inst<bf16_t, 128, 1>{}) : nq == 2 ? f(Inst<bf16_t, 128, 2>{}) : f(Inst<bf16_t, 128, 4>{});
    return nq == 1 ? f(Inst<bf16_t, 256, 1>{}) : f(Inst<bf16_t, 256, 2>{});
  }
  if (dh <= 64) return nq == 1 ? f(Inst<float, 64, 1>{}) : f(Inst<float, 64, 2>{});
  if (dh <= 128) return nq == 1 ? f(Inst<float, 128, 1>{}) : f(Inst<float, 128, 2>{});
  return f(Inst<float, 256, 1>{});
}

struct Plan { int workers; bool whole; };

template <typename T, int DH, int NQ>
Plan plan(Inst<T, DH, NQ>, int B, int M, int Hkv, int group, int width, int page_size) {
  typedef Inst<T, DH, NQ> I;
  const int64_t tiles = (int64_t)M * group / I::QT + std::min(B, M), triples = tiles * Hkv;
  const int64_t steps = std::max<int64_t>(1, ((int64_t)width * page_size + I::kStep - 1) / I::kStep);
  const int64_t most = 256 * I::kPerCu;
  Plan p;
  p.whole = steps <= 4;
  p.workers = (int)std::min<int64_t>(p.whole ? 4 * most : most, triples * (p.whole ? 1 : steps));
  return p;
}

template <typename T, int DH, int NQ>
pvf_status launch(Inst<T, DH, NQ> inst, hipStream_t s, Args &a) {
  typedef Inst<T, DH, NQ> I;
  const Plan p = plan(inst, a.p.B, a.p.M, a.p.Hkv, a.group, a.p.width, a.p.page_size);
  a.whole = p.whole;
  a.share_min = 1;
  a.chunk_steps = (int)std::min<int64_t>((int64_t)(kPageSlots - 2) * a.p.page_size / I::kStep, 1 << 20);
  if (a.p.dh == DH) page_attention_kernel<T, DH, NQ, true><<<p.workers, 256, 0, s>>>(a);
  else page_attention_kernel<T, DH, NQ, false><<<p.workers, 256, 0, s>>>(a);
  PVF_LAUNCH_CHECK(nullptr, "page_attention");
  if (!p.whole && p.workers > 1) {
    page_attention_join_kernel<T, DH, NQ><<<p.workers - 1, 256, 0, s>>>(a, p.workers);
    PVF_LAUNCH_CHECK(nullptr, "page_attention_join");
  }
  return PVF_OK;
}

}  // namespace

int64_t page_attention_workspace(int dtype, int B, int M, int H, int Hkv, int dh, int width, int page_size) {
  return with_instance(dtype, M, B, H / Hkv, dh, [&](auto inst) {
    typedef decltype(inst) I;
    const Plan p = plan(inst, B, M, Hkv, H / Hkv, width, page_size);
    return p.whole || p.workers == 1 ? (int64_t)0 : (int64_t)p.workers * 2 * I::kSlotFloats * (int64_t)sizeof(float);
  });
}

pvf_status launch_page_attention(hipStream_t s, int dtype, const PageAttention &p) {
  Args a = {};
  a.p = p;
  a.group = p.H / p.Hkv;
  a.scale2 = (float)((double)p.scale * 1.4426950408889634);
  // page of a key = (key / 8) / (page_size / 8) by a product: exact below 2^28 (the multiplier's excess is at most 2^L / 2^(31 + L) of a step)
  const uint32_t d = (uint32_t)p.page_size / 8;
  uint32_t L = 0;
  while ((1u << L) < d) ++L;
  a.div_mul = (uint32_t)(((uint64_t)1 << (31 + L)) / d + 1);
  a.div_shift = L;
  return with_instance(dtype, p.M, p.B, a.group, p.dh, [&](auto inst) { return launch(inst, s, a); });
}

}  // namespace pvf
