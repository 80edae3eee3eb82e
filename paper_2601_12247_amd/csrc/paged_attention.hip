// Attention of rows against keys and values in pages: out = softmax(scale q k^T) v over the keys that a row sees, one pass with the running
// maximum and sum of the softmax (in units of log2).
//
// Matrix instructions compute S^T = K Q^T and O^T = V^T P^T, 16 columns a block: the (row, head) pairs that share a key head.  A lane of S^T holds
// one column and keys 4 g .. 4 g + 3 of every 16 (g = lane / 16), which is a lane's share of the operand P^T if the keys of V^T are taken in the
// same order, so scores never leave their lane.  Keys and values go from the pages straight into registers, a whole row of a value by 16 lanes:
// lane c holds dimensions VE c .. of four neighbouring keys, and operand j of the matrix instruction is made of dimension VE c + j of those.
//
// P enters the bf16 instruction as two bf16 parts (16 bits of it): the second instruction costs nothing beside the memory, and the result is
// rounded once, to its own type.  Beside probabilities of 32 bits that moves 0.4 % of results to the neighbouring bf16 (32768 keys: 0.42 and 0.46 % differ from 64 bits
// rounded once, 0.17 and 0.10 % with float32 arithmetic, on two inputs); the error against 64 bits is that of the one rounding, to four digits.
//
// Bound by reading keys and values.  bf16, 64 requests of up to 8192 tokens, 8 key heads, groups of 4: 191 us for 1.05 GB (5.5 TB/s; a copy, which writes
// as well, reaches 4.9), and 8 to join.  One request of 32768: 28.2 us for 134 MB (4.8 TB/s), and 6 to join.  Where there is little to read it is latency:
// f32, one request of 128 tokens, 6.5 us; 17 of up to 1411 with 5 rows, 16.9 us and 4.8 to join for 21 MB, of which the first keys take 6.
#include "paged_attention.h"

#include <cmath>

namespace pvf {
namespace page {
namespace {

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
  static constexpr int QT = 16 * NQ, kDh = DH, kSplit = 4, kWholeSteps = kBf16 ? 4 : 3;
  static constexpr bool kAsTheyCome = false;
  static constexpr int kOPad = DH + 4;
  static constexpr int kSlotFloats = QT * (DH + 2);     // a partial result: m[QT], l[QT], O[QT][DH]
  static constexpr int kRegs = (NT + KJ + 2) * 4 * NQ + NU * KJ * 4 + NU * 4 * NB * VE * (int)sizeof(T) / 4 + 64;   // about
  static constexpr int kPerCu = kRegs <= 256 ? 2 : 1;   // workgroups of 4 waves
};

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
    const int page = page_of(a, key);
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

  __device__ __forceinline__ static bool not_finite(uint32_t w) { return I::kBf16 ? bf16s_not_finite(w) : (w & 0x7f800000u) == 0x7f800000u; }

  // What the values of this tile that are not finite add to column block nq: of the keys that a column sees, no others.  They are read again.
  __device__ __forceinline__ void add_odd_values(int nq, int kb) {
#pragma unroll 1
    for (int x = 0; x < I::KT && kb + x < len; ++x) {
      bool none;
      const T *v = vbase + place(kb + x, a.p.v_page_stride, &none);
#pragma unroll
      for (int nb = 0; nb < I::NB; ++nb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int d = nb * 16 * I::VE + I::VE * (4 * g + i);
          Val y = {};
          if (kb + x < limit[nq] && (kWhole || d < a.p.dh)) y = *(const Val *)(v + d);
#pragma unroll
          for (int j = 0; j < I::VE; ++j)
            o[nq][nb * I::VE + j][i] += odd_part(I::kBf16 ? (j % 2 ? y.w[j / 2] & 0xffff0000u : y.w[j / 2] << 16) : y.w[j]);
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
                x = I::kBf16 ? bf16s_finite(x) : not_finite(x) ? 0u : x;
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
        sc[nq][u] = x;
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
      float top = s[0][0];
#pragma unroll
      for (int u = 0; u < I::NU; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, s[u][i]);
      top = fmaxf(top, __shfl_xor(top, 16, kWave));
      top = fmaxf(top, __shfl_xor(top, 32, kWave));
      // the maximum in use follows when it is passed by 2^8: sums stay far from overflow and are rarely scaled
      const bool up = (top - m[nq]) * a.c > 8.0f;               // the first time m = -inf
      const float now = up ? top : m[nq], ref = reference(now), alpha = up ? weight(a, m[nq], now) : 1.0f, less = -ref * a.c;
      m[nq] = now;
      float sum = 0.f;
#pragma unroll
      for (int u = 0; u < I::NU; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s[u][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][i], a.c, less));
          sum += s[u][i];
        }
      l[nq] = l[nq] * alpha + sum;
      if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
        for (int at = 0; at < I::NT; ++at) o[nq][at] *= alpha;
      }
      if (odd) add_odd_values(nq, kb);
      if constexpr (I::kBf16) {
        auto upper = [&](int u, int i) { return upper_parts(s[u][i], s[u][i + 1]); };
        auto rest = [&](int u, int i) { return lower_parts(s[u][i], s[u][i + 1]); };
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
  __shared__ int32_t s_pages[kPageSlots];
  __shared__ float s_m[4][I::QT], s_l[4][I::QT];
  __shared__ alignas(16) float s_o[4][16][I::kOPad];
  const int tid = threadIdx.x, wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  int worker;
  Line<I> line(a, blockIdx.x, gridDim.x, &worker);
  if (!a.whole && worker < a.workers && tid == 0) a.joins[(int64_t)worker * kJoinInts] = 0;
  Request r;
  Piece piece;
  Pass<T, DH, NQ, kWhole> pass(a, s_pages);
  while (line.next(r, piece)) {
    const int cols = piece.cols;
    pass.len = r.len;
    pass.over = r.over;
    pass.kbase = (const T *)a.p.k_cache + (int64_t)piece.head * a.p.page_size * a.p.dh;
    pass.vbase = (const T *)a.p.v_cache + (int64_t)piece.head * a.p.page_size * a.p.dh;
    pass.least = INT32_MAX;
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
      const int col = 16 * nq + pass.c;
      int row;
      const T *src = (const T *)a.p.q + row_place(a, r.row0, piece.head, piece.tile * I::QT + col, a.p.q_stride, &row) + I::KE * pass.g;
      pass.limit[nq] = col < cols ? limit_of(a, r.told, r.n, row) : INT32_MAX;
      pass.least = min(pass.least, pass.limit[nq]);
#pragma unroll
      for (int j = 0; j < I::KJ; ++j) {
        uint4 x = make_uint4(0, 0, 0, 0);
        if (col < cols && (kWhole || j * 4 * I::KE + I::KE * pass.g < a.p.dh)) x = *(const uint4 *)(src + j * 4 * I::KE);
        pass.q[nq][j] = make_uint4(x.x ^ a.q_xor, x.y ^ a.q_xor, x.z ^ a.q_xor, x.w ^ a.q_xor);
      }
      pass.m[nq] = -INFINITY;
      pass.l[nq] = 0.f;
#pragma unroll
      for (int t = 0; t < I::NT; ++t) pass.o[nq][t] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int off = 1; off < 16; off <<= 1) pass.least = min(pass.least, __shfl_xor(pass.least, off, kWave));
    pass.least = __builtin_amdgcn_readfirstlane(pass.least);

    for (int s0 = piece.step0; s0 < piece.step1; s0 += a.chunk_steps) {
      const int s1 = min(piece.step1, s0 + min(a.chunk_steps, piece.step1 - s0));
      const int k0 = s0 * I::kStep, k1 = (int)min((int64_t)r.len, (int64_t)s1 * I::kStep);
      meet();                             // the last chunk's pages, or the last piece's results, have been read
      pass.first_page = page_of(a, k0);
      load_pages(a, line.b, k0, k1, pass.first_page, s_pages, nullptr);
      meet();
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

    // the four waves' results, and the way out: the rows themselves, or a partial result
    float *slot = piece.done ? nullptr : partial<I>(a, worker, piece.begun);
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
        for (int k = 1; k < 4; ++k) top = fmaxf(top, s_m[k][col]);
        const float ref = reference(top);
        float total = 0.f;
        floatx4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float f = weight(a, s_m[k][col], ref);
          total += f * s_l[k][col];
          sum += f * *(const floatx4 *)&s_o[k][cq][d];
        }
        if (piece.done) {
          int row;
          const int64_t at = row_place(a, r.row0, piece.head, piece.tile * I::QT + col, a.p.out_stride, &row);
          store4((T *)a.p.out + at + d, sum, 1.0f / total, limit_of(a, r.told, r.n, row) <= 0);
        } else {
          *(floatx4 *)(slot + 2 * I::QT + col * DH + d) = sum;
          if (d == 0) {
            slot[col] = top;
            slot[I::QT + col] = total;
          }
        }
      }
    }
    if (!piece.done && piece.begun && tid == 0) line.note_join(worker, r, piece);
  }
}

// ---- choice of an instance -----------------------------------------------------------------------
// Columns of a tile by the mean number of (row, head) pairs that share a key head: two blocks, which leave one workgroup a CU, where one would read every
// key twice; in bf16 the wide kernel's.  64 requests of 2048 keys, 8 key heads, us:
//   f32, 16 and 32 columns: 16 pairs 103 and 109 (d_head 64), 195 and 233 (128); 24 pairs 190 and 109, 377 and 236
//   bf16, 16, 32 and the wide kernel's 64: 16 pairs 44.7, 46.6, 51.0 (64), 103, 117, 107 (128), 191, 259, - (256)
//                                          24 pairs 80.5, 46.8, 50.1,      189, 118, 107,       367, 264, 203;   40 pairs of d_head 64 116, 83.2, 49.6
template <class F>
auto with_instance(int dtype, int64_t pairs, int dh, F f) {
  const bool one = pairs <= 16;
  if (dtype == PVF_BF16) {
    if (dh <= 64) return one ? f(Inst<bf16_t, 64, 1>{}) : f(Inst<bf16_t, 64, 2>{});
    if (dh <= 128) return f(Inst<bf16_t, 128, 1>{});
    return f(Inst<bf16_t, 256, 1>{});
  }
  if (dh <= 64) return one ? f(Inst<float, 64, 1>{}) : f(Inst<float, 64, 2>{});
  if (dh <= 128) return one ? f(Inst<float, 128, 1>{}) : f(Inst<float, 128, 2>{});
  return f(Inst<float, 256, 1>{});
}
int64_t mean_pairs(int M, int B, int group) { return ((int64_t)M + B - 1) / B * group; }
bool is_wide(int dtype, int64_t pairs, int dh) { return dtype == PVF_BF16 && pairs > (dh <= 64 ? 32 : 16); }

template <typename T, int DH, int NQ>
pvf_status launch(Inst<T, DH, NQ>, hipStream_t s, Args &a) {
  typedef Inst<T, DH, NQ> I;
  const Plan p = prepare<I>(a);
  if (a.p.dh == DH) page_attention_kernel<T, DH, NQ, true><<<p.grid, 256, 0, s>>>(a);
  else page_attention_kernel<T, DH, NQ, false><<<p.grid, 256, 0, s>>>(a);
  PVF_LAUNCH_CHECK(nullptr, "page_attention");
  if (!a.whole) {
    page_attention_join_kernel<T, I><<<dim3(p.workers - 1, I::QT / kJoinCols<I>), kJoinThreads, 0, s>>>(a);
    PVF_LAUNCH_CHECK(nullptr, "page_attention_join");
  }
  return PVF_OK;
}

}  // namespace
}  // namespace page

int64_t page_attention_workspace(int dtype, int B, int M, int H, int Hkv, int dh, int width, int page_size) {
  const int group = H / Hkv;
  const int64_t pairs = page::mean_pairs(M, B, group);
  if (page::is_wide(dtype, pairs, dh)) return page::wide_workspace(B, M, Hkv, group, dh, width, page_size, pairs);
  return page::with_instance(dtype, pairs, dh, [&](auto inst) {
    typedef decltype(inst) I;
    return page::workspace_bytes<I>(B, M, Hkv, group, width, page_size);
  });
}

pvf_status launch_page_attention(hipStream_t s, int dtype, const PageAttention &p) {
  page::Args a = {};
  a.p = p;
  a.group = p.H / p.Hkv;
  a.c = std::fmax((float)(std::fabs((double)p.scale) * 1.4426950408889634), 0x1p-126f);   // zero, too: no score is then far from it
  if (p.scale < 0) a.q_xor = dtype == PVF_BF16 ? 0x80008000u : 0x80000000u;
  // page of a key = (key / 8) / (page_size / 8) by a product: exact below 2^28 (the multiplier's excess is at most 2^L / 2^(31 + L) of a step)
  const uint32_t d = (uint32_t)p.page_size / 8;
  uint32_t L = 0;
  while ((1u << L) < d) ++L;
  a.div_mul = (uint32_t)(((uint64_t)1 << (31 + L)) / d + 1);
  a.div_shift = L;
  const int64_t pairs = page::mean_pairs(p.M, p.B, a.group);
  if (page::is_wide(dtype, pairs, p.dh)) return page::launch_wide(s, a, pairs);
  return page::with_instance(dtype, pairs, p.dh, [&](auto inst) { return page::launch(inst, s, a); });
}

}  // namespace pvf
