// Products with block-scaled operands (mx.h) on the CDNA4 matrix cores: C[M,N] = A[M,K] * W[N,K]^T (+ residual), float32 accumulation.
//
//   rows      weights      result          arithmetic
//   e4m3      e4m3, e2m1   bfloat16        v_mfma_scale_f32_16x16x128_f8f6f4: codes and scale bytes as they lie in memory
//   e4m3      e4m3, e2m1   float32, e4m3   codes decoded to bfloat16, which holds them exactly, and v_mfma_f32_16x16x32_bf16
//   bfloat16  e2m1         bfloat16        weights decoded to bfloat16 (exact)
//   float32   e2m1         float32         rows as three bfloat16 whose sum they are (24 bits), weights decoded
//
// The scaled instruction adds 8 neighbouring products at a time, each cut off 13 bits below the largest of the eight (measured: 16 and 2^-8 1.27 in
// one group lose what lies below 2^-9), then those sums and the accumulator in float32.  On random operands that is 1.5e-5 of the
// result, a hundredth of a bfloat16 rounding: one result in 40 rounds to its other neighbour, and the error against 64 bits stays 1.66e-3.  An e4m3 element is itself rounded by up to
// 2^-4 of it, 70 times what its product can cost the others of its eight (7 2^-13 of it).  Float32 results do not take it (the bfloat16 instruction keeps float32 sums), nor does SwiGLU,
// whose 8-bit results would differ from the definition's in 0.3 % of the codes and here and there in a block's scale, where float32
// sums differ in one of 10^5; it would take half the time of the matrix instructions.
//
// Operands of the scaled 16 x 16 x 128 instruction: lane (r = lane % 16, g = lane / 16) holds row r; of e4m3 the 16 bytes at k = 16 g and
// the 16 at 64 + 16 g, of e2m1 the 32 elements from 32 g on; its scale byte is that of k = 32 g .. 32 g + 31.  The weights are the
// instruction's first operand, so that a lane ends up with 4 consecutive columns of C.
//
// Four kernels, from few results to many; choose() takes the instance whose fullest CU is done first.  Bounds: few rows by the launch (a kernel that
// does nothing takes 3 us) and the weights' bytes; tiles on the way by a CU's loads into LDS, 125-150 GB/s from L2 in any order, some 55 of what HBM
// delivers to all CUs; many rows by the matrix pipe and the power it takes (scaled) or by the instructions that decode (decoded).
//   gemm_mx_waves_kernel  tiles up to 80 x 64 or 32 x 128, a ring for each wave, no barrier
//   gemm_mx_kernel        tiles from 16 x 16 to 192 x 256, one ring; rows at any element
//   gemm_mx_steps_kernel  64 x 128 and 128 x 128, decoded operands
//   gemm_mx_quad_kernel   256 x 256, scaled instruction
#include "mx.h"

#include <algorithm>
#include <atomic>
#include <iterator>

namespace pvf {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef int intx4 __attribute__((ext_vector_type(4)));
typedef int intx8 __attribute__((ext_vector_type(8)));

enum Rows { kRowsMx, kRowsMxExact, kRowsBf16, kRowsF32 };   // what multiplies what (table above)
enum Out { kOutBf16, kOutF32, kOutSwiglu };

constexpr bool codes_in(int rows) { return rows == kRowsMx || rows == kRowsMxExact; }

// silu(g) within 2^-22: each rounding here moves codes of an 8-bit result that lie between two.  exp(-g) = 2^p with what p lost put back, its
// sum with one with what that lost, and a Newton step behind the reciprocal.  Past |g| = 80 the plain form: there a
// power may be 0 or infinite (to -256: far_act).  12288 x 4096 weights in 4 bits, 64 rows: 1 of 900000 codes differs from the definition in 64 bits, 1 of 120000 with the plain form; no time.
constexpr float kLog2e = 0x1.715476p+0f, kLog2eRest = 0x1.4ae0cp-26f, kLn2 = 0x1.62e43p-1f;
__device__ __forceinline__ float silu_f(float g) {
  const float p = -g * kLog2e, e = __builtin_amdgcn_exp2f(p), ec = fmaf(e, kLn2 * fmaf(-g, kLog2eRest, fmaf(-g, kLog2e, -p)), e);
  const float d = 1.0f + ec, b = d - 1.0f, lost = (1.0f - (d - b)) + (ec - b), r = __builtin_amdgcn_rcpf(d);
  const float near = fmaf(fmaf(-d, r, 1.0f) - lost * r, r, r);
  return g * (fabsf(g) < 80.f ? near : __builtin_amdgcn_rcpf(1.0f + e));
}

// silu(g) u for g of -256 to -80, where 1 + exp(-g) is exp(-g) in any type here: g exp(g) u with the power of two put on last.  silu(g) by itself is below
// float32's normal range from -92 on and its divisor above float32 from -89 on, while the product may be any code: a block's scale goes down to 2^-127.  (u 2^-64: what
// that loses is below 2^-168 in the product.)  Below -256 the product is less than 2^-230: zero.
__device__ __forceinline__ float far_act(float g, float u) {
  const float n = rintf(g * kLog2e), f = fmaf(g, kLog2eRest, fmaf(g, kLog2e, -n));      // g log2(e) - n, rounded to 2^-25
  return __builtin_ldexpf(g * __builtin_amdgcn_exp2f(f) * (u * 0x1p-64f), (int)n + 64);
}

// The four registers of 32 e2m1 codes; the instruction does not read the others.
__device__ __forceinline__ intx8 join(intx4 lo) { return __builtin_shufflevector(lo, lo, 0, 1, 2, 3, -1, -1, -1, -1); }
__device__ __forceinline__ intx8 join(intx4 lo, intx4 hi) { return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7); }

// Eight codes (two words of e4m3, one of e2m1) times 2^(b - 127) as bfloat16.
__device__ __forceinline__ bf16x8 decode_e4m3(int lo, int hi, float scale) {
#ifdef __HIP_DEVICE_COMPILE__
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true),
               c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
#else
  return bf16x8{};
#endif
}
__device__ __forceinline__ bf16x8 decode_e2m1(int w, float scale) {
#ifdef __HIP_DEVICE_COMPILE__
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1),
               c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
#else
  return bf16x8{};
#endif
}

// The conversions take the exponent bits of a float32 as their scale, which are the scale byte: 0 is 2^-127, 255 NaN.
__device__ __forceinline__ float byte_scale(int b) { return __uint_as_float((uint32_t)b << 23); }

// x = p[0] + p[1] + p[2] exactly, 8 bits of the mantissa each, cut off and not rounded so that nothing overflows.  What is not finite has to
// be in p[0] alone: a NaN makes NaN of the other parts, which is as good, an infinity is looked for in all eight at once (taking it out element by
// element was half of the instructions).
__device__ __forceinline__ void split3(const float *x, bf16x8 *p) {
  uint32_t hi[8], mid[8], lo[8];
  float top = fabsf(x[0]);
#pragma unroll
  for (int e = 1; e < 8; ++e) top = fmaxf(top, fabsf(x[e]));
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    hi[e] = __float_as_uint(x[e]);
    const float r = x[e] - __uint_as_float(hi[e] & 0xffff0000u);
    mid[e] = __float_as_uint(r);
    lo[e] = __float_as_uint(r - __uint_as_float(mid[e] & 0xffff0000u));
  }
  if (top == __builtin_inff()) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (fabsf(x[e]) == __builtin_inff()) mid[e] = lo[e] = 0;
  }
  intx4 w[3];
#pragma unroll
  for (int e = 0; e < 4; ++e) {                              // the upper halves of two words
    w[0][e] = (int)__builtin_amdgcn_perm(hi[2 * e + 1], hi[2 * e], 0x07060302u);
    w[1][e] = (int)__builtin_amdgcn_perm(mid[2 * e + 1], mid[2 * e], 0x07060302u);
    w[2][e] = (int)__builtin_amdgcn_perm(lo[2 * e + 1], lo[2 * e], 0x07060302u);
  }
#pragma unroll
  for (int q = 0; q < 3; ++q) p[q] = __builtin_bit_cast(bf16x8, w[q]);
}

// ---- results ------------------------------------------------------------------------------------------------------
// Columns n .. n + 3 of row m, those from n_from on.
template <typename T> __device__ __forceinline__ void store_row4(floatx4 v, int m, int n, const MxGemm &p, int n_from = 0) {
  const int N = p.N;
  T *row = (T *)p.C + (int64_t)m * N;
  const T *res = p.residual ? (const T *)p.residual + (int64_t)m * N : nullptr;
  if (N % 4 == 0 && n < N && n >= n_from) {                                 // a row begins as C does, at an element: unaligned vectors
    float x[4] = {v[0], v[1], v[2], v[3]};
    if constexpr (sizeof(T) == 2) {
      typedef uint32_t u2 __attribute__((ext_vector_type(2), aligned(2)));
      if (res) {
        const u2 q = *reinterpret_cast<const u2 *>(res + n);
#pragma unroll
        for (int e = 0; e < 2; ++e) { x[2 * e] += __uint_as_float(q[e] << 16); x[2 * e + 1] += __uint_as_float(q[e] & 0xffff0000u); }
      }
      u2 o;
#pragma unroll
      for (int e = 0; e < 2; ++e)
        o[e] = (uint32_t)__builtin_bit_cast(uint16_t, (bf16_t)x[2 * e]) | ((uint32_t)__builtin_bit_cast(uint16_t, (bf16_t)x[2 * e + 1]) << 16);
      *reinterpret_cast<u2 *>(row + n) = o;
    } else {
      typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
      if (res) {
        const f4 q = *reinterpret_cast<const f4 *>(res + n);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] += q[e];
      }
      *reinterpret_cast<f4 *>(row + n) = f4{x[0], x[1], x[2], x[3]};
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (n + e < N && n + e >= n_from) row[n + e] = from_float<T>(v[e] + (res ? to_float(res[n + e]) : 0.f));
}

// silu(gate) * up of 32 columns from c0 on, of which the lane has 4 g .. + 3 and 16 + 4 g .. + 3: a block, as codes and scale.  All 64 lanes.
__device__ __forceinline__ void store_act(floatx4 g0, floatx4 g1, floatx4 u0, floatx4 u1, bool live, int m, int c0, int g, const MxGemm &p, int Np) {
  float v[8], lowest = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[e] = silu_f(g0[e]) * u0[e];
    v[4 + e] = silu_f(g1[e]) * u1[e];
    lowest = fminf(lowest, fminf(g0[e], g1[e]));
  }
  if (__any(lowest <= -80.f)) {                              // hardly ever, so its instructions are jumped over (2560 x 12288 x 4096: 397 us with it, 396 without)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float gate = e < 4 ? g0[e & 3] : g1[e & 3], up = e < 4 ? u0[e & 3] : u1[e & 3];
      if (gate <= -80.f && gate >= -256.f) v[e] = far_act(gate, up);
    }
  }
  uint32_t am = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (c0 + (e & 4) * 4 + 4 * g + (e & 3) >= p.N) v[e] = 0.f;
    am = max(am, abs_bits(v[e]));
  }
  am = max(am, (uint32_t)__shfl_xor((int)am, 16, kWave));
  am = max(am, (uint32_t)__shfl_xor((int)am, 32, kWave));
  const int b = mx_scale_byte<PVF_MX_E4M3>(am);
  const float inv = mx_inverse(b);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = b == 255 ? 0.f : v[e] * inv;
  if (!live) return;
  uint8_t *row = (uint8_t *)p.C + (int64_t)m * Np + c0 + 4 * g;
  *reinterpret_cast<uint32_t *>(row) = pack_e4m3x4(v[0], v[1], v[2], v[3]);
  *reinterpret_cast<uint32_t *>(row + 16) = pack_e4m3x4(v[4], v[5], v[6], v[7]);
  if (g == 0) p.c_scales[((int64_t)(c0 / kMxStage) * p.M + m) * 4 + c0 / kMxBlock % 4] = (uint8_t)b;
}

// ---- the kernel ---------------------------------------------------------------------------------------------------
typedef __attribute__((address_space(1))) const void gptr_t;
typedef __attribute__((address_space(3))) void lptr_t;

// s_waitcnt vmcnt(n) only; n is a 6-bit field split 4 + 2
template <int N> __device__ __forceinline__ void wait_vmcnt() {
  static_assert(N >= 0 && N < 64, "vmcnt is a 6-bit counter");
  __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | ((N >> 4) << 14));
}

struct TileMap { int tiles_m, tiles_n, group_m; };

// Chunk c of a row lies at place c ^ swizzle(row) of an LDS row of R bytes, so that the reads of an operand (lane (r, g): row r, chunk c0 + X g) touch
// every bank once per 16 lanes.  ds_read_b128 takes lanes 0-3, 12-15 and 20-27 together, then 4-11, 16-19 and 28-31, and so on: rows whose
// bits 2 and 3 are equal with one g, the other rows with the next.  So the places of the first have to be those of the second moved by X.
template <int R, int X> __device__ __forceinline__ int swizzle(int row) {
  const int t = row >> 2 & 3;
  if (R == 64) return 0x78 >> 2 * t & 3;                     // 0, 2, 3, 1 (X = 1)
  if (R == 128) return X == 1 ? row >> 1 & 7 : (row >> 1 & 4) | (row >> 2 & 1) | (row & 2);      // X = 2: bits 0 and 1 of row / 2 exchanged
  return X <= 2 ? row & 15 : (row & 3) | (X == 4 ? 0x78 >> 2 * t & 3 : t ^ t >> 1) << 2;         // X = 8: 0, 1, 3, 2
}

// ---- operands of 128 k in registers -----------------------------------------------------------------------------------
// Lane (r, g) of a wave whose results are 16 MT rows x 16 NT columns.  Chunks of 16 bytes: of the scaled instruction's e4m3 rows the g-th and
// the 4 + g-th, of all others the kA (kW) from kA g on.
template <int ROWS, int WF, int MT, int NT> struct Operands {
  static constexpr bool kCodes = codes_in(ROWS), kW8 = WF == PVF_MX_E4M3;
  static constexpr int kA = kCodes ? 2 : ROWS == kRowsBf16 ? 4 : 8, kW = kW8 ? 2 : 1, kPlanes = ROWS == kRowsF32 ? 3 : 1;
  static constexpr int kAX = ROWS == kRowsMx ? 1 : kA, kWX = ROWS == kRowsMx ? 1 : kW;       // chunks from g to g + 1
  intx4 a[MT][kA], w[NT][kW];
  int as[kCodes ? MT : 1], ws[NT];

  // From LDS rows of RA and RW bytes (row am and row an are the lane's first), whose 128 k begin at chunks a_chunk and w_chunk; dwords of scales.
  // Of A there are AR rows: behind them (AR < 16) the first ones again, for columns of the instruction that are not stored.
  template <int RA, int RW, int AR>
  __device__ __forceinline__ void read(const unsigned char *la, int am, int a_chunk, const unsigned char *lw, int an, int w_chunk, const unsigned char *sa,
                                       const unsigned char *sw, int r, int g) {
#pragma unroll
    for (int q = 0; q < kPieces; ++q) read_piece<RA, RW, AR>(q, la, am, a_chunk, lw, an, w_chunk, sa, sw, r, g);
  }
  static constexpr int kAPieces = MT * (kA + kCodes), kPieces = kAPieces + NT * (kW + 1);
  template <int RA, int RW, int AR>
  __device__ __forceinline__ void read_piece(int q, const unsigned char *la, int am, int a_chunk, const unsigned char *lw, int an, int w_chunk, const unsigned char *sa,
                                             const unsigned char *sw, int r, int g) {
    const int ar = AR < 16 ? r % AR : am;
    if (q < kAPieces) {
      const int mt = q / (kA + kCodes), c = q % (kA + kCodes);
      if (c < kA) a[mt][c % kA] = *reinterpret_cast<const intx4 *>(la + (mt * 16 + ar) * RA + (((a_chunk + (ROWS == kRowsMx ? 4 * c + g : kA * g + c)) ^ swizzle<RA, kAX>(ar)) << 4));
      else as[kCodes ? mt : 0] = sa[(mt * 16 + ar) * 4 + g];
    } else {
      const int nt = (q - kAPieces) / (kW + 1), c = (q - kAPieces) % (kW + 1);
      if (c < kW) w[nt][c % kW] = *reinterpret_cast<const intx4 *>(lw + (nt * 16 + an) * RW + (((w_chunk + (ROWS == kRowsMx ? 4 * c + g : kW * g + c)) ^ swizzle<RW, kWX>(r)) << 4));
      else ws[nt] = sw[(nt * 16 + an) * 4 + g];
    }
  }

  // Matrix instructions of 128 k; multiply calls then(i) behind the i-th.  left: elements of a row of bf16 / float32 from the first of the 128 on;
  // what lies behind them is another chunk's.
  static constexpr int kInstrs = NT * MT * (ROWS == kRowsMx ? 1 : 4 * kPlanes);
  template <typename F> __device__ __forceinline__ void multiply(floatx4 (&acc)[NT][MT], int left, int g, F then) const {
    if constexpr (ROWS == kRowsMx) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
#ifdef __HIP_DEVICE_COMPILE__
          acc[nt][mt] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kW8 ? join(w[nt][0], w[nt][kW - 1]) : join(w[nt][0]), join(a[mt][0], a[mt][1]), acc[nt][mt], kW8 ? 0 : 4, 0,
                                                                         0, ws[nt], 0, as[kCodes ? mt : 0]);
#endif
          then(nt * MT + mt);
        }
    } else {
      // four steps of 32 k: lane g has elements 32 g + 8 j .. + 7 of its 128 in the j-th, all of one block
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        bf16x8 wf[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
          wf[nt] = kW8 ? decode_e4m3(w[nt][(j >> 1) % kW][j * 2 & 3], w[nt][(j >> 1) % kW][(j * 2 & 3) + 1], byte_scale(ws[nt])) : decode_e2m1(w[nt][0][j], byte_scale(ws[nt]));
        const int k = 32 * g + 8 * j;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          bf16x8 p[3];
          if constexpr (kCodes) {
            p[0] = decode_e4m3(a[mt][(j >> 1) % kA][j * 2 & 3], a[mt][(j >> 1) % kA][(j * 2 & 3) + 1], byte_scale(as[kCodes ? mt : 0]));
          } else if constexpr (ROWS == kRowsBf16) {
            p[0] = __builtin_bit_cast(bf16x8, k >= left ? intx4{0, 0, 0, 0} : a[mt][j % kA]);
          } else {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = k + (e & 4) >= left ? 0.f : __int_as_float(a[mt][(2 * j + e / 4) % kA][e % 4]);
            split3(v, p);
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int q = 0; q < kPlanes; ++q) {              // the least part first
              acc[nt][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[nt], p[kPlanes - 1 - q], acc[nt][mt], 0, 0, 0);
              then(((j * MT + mt) * NT + nt) * kPlanes + q);
            }
        }
      }
    }
  }
};

// Sizes of an instance.
template <int ROWS, int WF, int BM, int BN, int WM, int WN, int WK, int kStages, int AR = BM> struct Shape {
  static constexpr int kASize = codes_in(ROWS) ? 1 : ROWS == kRowsBf16 ? 2 : 4;
  static constexpr int kAX = ROWS == kRowsMx ? 1 : 2 * kASize, kWX = ROWS == kRowsMx || WF == PVF_MX_E2M1 ? 1 : 2;   // chunks from g to g + 1
  static constexpr int kThreads = 64 * WM * WN * WK, kWaves = WM * WN * WK, MT = BM / WM / 16, NT = BN / WN / 16;
  static constexpr int kARow = 128 * WK * kASize, kWRow = (WF == PVF_MX_E4M3 ? 128 : 64) * WK;           // LDS bytes of a row and stage
  static constexpr int kABytes = AR * kARow, kWBytes = BN * kWRow;
  static constexpr int kAUnits = codes_in(ROWS) ? (AR * WK + 63) / 64 : 0, kWUnits = (BN * WK + 63) / 64;   // scale dwords, 64 at a time
  static constexpr int kSBytes = (kAUnits + kWUnits) * 256, kStage = kABytes + kWBytes + kSBytes;
  static constexpr int kRing = kStages * kStage, kSums = WK > 1 ? WK * BM * BN * 4 : 0, kLds = kRing > kSums ? kRing : kSums;
};

// A workgroup computes BM x BN results.  A stage is 128 WK elements of k: wave (wm, wn, wk) multiplies the wk-th 128 of them for its
// BM / WM x BN / WN results, and with WK > 1 the waves' sums are added through LDS at the end.  Stages go through a ring of kStages slots of LDS, straight
// from memory (whole 128-byte lines per request: loads of 64-byte pieces straight into registers reached half the rate), one barrier
// a stage.  Rows of bf16 / float32 that do not begin at 16-byte chunks go through registers (kDirect = false).
// Bound by the CU's loads: a stage's BM + BN rows, not its BM BN results, so tiles are as square as the launch leaves them.  WK > 1 where there are fewer
// tiles than CUs: more loads in flight for the same tile.  1280 x 4096 x 12288, e4m3 weights, 160 x 128 tiles: 77-83 us, 1.6 PFLOP/s; one row of float32
// against 4-bit weights 12288 x 4096, 16 x 64 with k over 8 waves: 11.6 us (16 columns a workgroup 17: the row is split into its three parts
// for every 16 of them); 33 float32 rows that are not aligned, 4001 x 1411: 9.7 us, the latency of three stages.
template <int ROWS, int WF, int OUT, int BM, int BN, int WM, int WN, int WK, int kStages, int AR, bool kDirect>
__global__ void __launch_bounds__(64 * WM * WN * WK)
gemm_mx_kernel(MxGemm p, TileMap tm) {
  using S = Shape<ROWS, WF, BM, BN, WM, WN, WK, kStages, AR>;
  constexpr bool kSwiglu = OUT == kOutSwiglu, kCodes = codes_in(ROWS), kW8 = WF == PVF_MX_E4M3;
  constexpr int kThreads = S::kThreads, kWaves = S::kWaves, MT = S::MT, NT = S::NT, kASize = S::kASize;
  constexpr int kACpr = S::kARow / 16, kWCpr = S::kWRow / 16;                // chunks of a row
  constexpr int kAChunks = AR * kACpr, kWChunks = BN * kWCpr, LA = (kAChunks + kThreads - 1) / kThreads, LW = (kWChunks + kThreads - 1) / kThreads;
  constexpr int LS = (S::kAUnits + S::kWUnits + kWaves - 1) / kWaves;
  constexpr int kLoads = (kDirect ? LA : 0) + LW + LS;       // load instructions of a thread and stage that go straight to LDS
  static_assert(BM % (16 * WM) == 0 && BN % (16 * WN) == 0 && kAChunks % 64 == 0 && kWChunks % 64 == 0, "tile shape");
  static_assert(kDirect || !kCodes, "codes always go straight");
  static_assert(!kSwiglu || BN / WN == 64, "a wave has a block of gate and the same block of up");
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wk = wave / (WM * WN), wm = wave / WN % WM, wn = wave % WN, r = lane & 15, g = lane >> 4;
  const int M = p.M, N = p.N, K = p.K, Kp = (K + kMxStage - 1) / kMxStage * kMxStage, nk = Kp / kMxStage, ns = (nk + WK - 1) / WK;

  // the 32 workgroups that an XCD runs at a time cover a patch of tiles and share operands through its L2
  const int total = tm.tiles_m * tm.tiles_n, per_xcd = (total + 7) >> 3;
  const int block = mx_block(), L = (block & 7) * per_xcd + (block >> 3);
  if (block >> 3 >= per_xcd || L >= total) return;
  const int band = L / (tm.group_m * tm.tiles_n), within = L - band * (tm.group_m * tm.tiles_n);
  const int band_rows = min(tm.group_m, tm.tiles_m - band * tm.group_m);
  const int tile_n = within / band_rows, tile_m = band * tm.group_m + (within - tile_n * band_rows);
  const int m0 = tile_m * BM, n0 = tile_n * (kSwiglu ? BN / 2 : BN);
  const int w_rows = kSwiglu ? 2 * N : N;

  // row of W behind row t of the tile: SwiGLU has 32 gate rows and the 32 up rows of the same columns in every wave's 64
  auto w_row = [&](int t) -> int64_t {
    if (!kSwiglu) return min(n0 + t, N - 1);
    const int n = min(n0 + (t >> 6) * 32 + (t & 31), N - 1);
    return (t & 32) ? (int64_t)N + n : n;
  };
  // ---- loads: chunk i * kThreads + tid of an operand tile; behind the end of a row its last chunk again, which is not read.  Every wave has
  //      as many loads as the others: some repeat one, into the same place ----
  const uint32_t a_bytes = (uint32_t)((kCodes ? Kp : K) * kASize), w_bytes = kW8 ? Kp : Kp / 2;
  const uint8_t *a_src[LA], *w_src[LW], *s_src[LS];
  uint32_t a_at[LA], w_at[LW], s_rows[LS];
  int s_sub[LS], s_slot[LS];
#pragma unroll
  for (int i = 0; i < LA; ++i) {
    const int f = (i * kThreads + tid) % kAChunks, row = f / kACpr;
    a_at[i] = ((f % kACpr) ^ swizzle<S::kARow, S::kAX>(row)) * 16;
    a_src[i] = (const uint8_t *)p.A + (int64_t)min(m0 + row, M - 1) * a_bytes;
  }
#pragma unroll
  for (int i = 0; i < LW; ++i) {
    const int f = (i * kThreads + tid) % kWChunks, row = f / kWCpr;
    w_at[i] = ((f % kWCpr) ^ swizzle<S::kWRow, S::kWX>(row)) * 16;
    w_src[i] = (const uint8_t *)p.W + w_row(row) * w_bytes;
  }
#pragma unroll
  for (int i = 0; i < LS; ++i) {
    const int u = (i * kWaves + wave) % (S::kAUnits + S::kWUnits);
    const bool of_a = u < S::kAUnits;
    const int f = (of_a ? u : u - S::kAUnits) * 64 + lane;
    const int row = of_a ? f % AR : f % BN;
    s_slot[i] = u * 256;
    s_sub[i] = of_a ? f / AR : f / BN;
    s_rows[i] = of_a ? M : w_rows;
    s_src[i] = of_a ? p.a_scales + (int64_t)min(m0 + row, M - 1) * 4 : p.w_scales + w_row(row) * 4;
  }
  auto issue = [&](int st) {
    unsigned char *slot = lds + st % kStages * S::kStage;
    if constexpr (kDirect)
#pragma unroll
      for (int i = 0; i < LA; ++i)
        __builtin_amdgcn_global_load_lds((gptr_t *)(a_src[i] + min(a_at[i] + (uint32_t)st * S::kARow, a_bytes - 16)), (lptr_t *)(slot + (i * kThreads + (wave << 6)) % kAChunks * 16), 16, 0, 0);
#pragma unroll
    for (int i = 0; i < LW; ++i)
      __builtin_amdgcn_global_load_lds((gptr_t *)(w_src[i] + min(w_at[i] + (uint32_t)st * S::kWRow, w_bytes - 16)), (lptr_t *)(slot + S::kABytes + (i * kThreads + (wave << 6)) % kWChunks * 16), 16, 0, 0);
#pragma unroll
    for (int i = 0; i < LS; ++i)
      __builtin_amdgcn_global_load_lds((gptr_t *)(s_src[i] + (uint64_t)min(st * WK + s_sub[i], nk - 1) * s_rows[i] * 4), (lptr_t *)(slot + S::kABytes + S::kWBytes + s_slot[i]), 4, 0, 0);
  };
  // ---- rows through registers ----
  constexpr int LX = kDirect ? 1 : LA;
  uint4 x[LX];
  auto fetch = [&](int st) {
    if constexpr (!kDirect)
#pragma unroll
      for (int i = 0; i < LX; ++i) {
        const int k = (int)(a_at[i] + st * S::kARow) / kASize;
        if constexpr (ROWS == kRowsBf16) x[i] = load8_raw((const bf16_t *)a_src[i] + min(k, K), K - k);
        else x[i] = load4_raw((const float *)a_src[i] + min(k, K), K - k);
      }
  };
  auto stash = [&](int st) {
    if constexpr (!kDirect)
#pragma unroll
      for (int i = 0; i < LX; ++i) *reinterpret_cast<uint4 *>(lds + st % kStages * S::kStage + (i * kThreads + tid) % kAChunks * 16) = x[i];
  };

  floatx4 acc[NT][MT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) acc[nt][mt] = floatx4{0.f, 0.f, 0.f, 0.f};

  const int am = wm * (BM / WM) + r, an = wn * (BN / WN) + r;               // rows of the lane's operands in the tiles (but for 16 mt, 16 nt)
  using Ops = Operands<ROWS, WF, MT, NT>;
  auto read = [&](Ops &o, int st) {
    const unsigned char *slot = lds + st % kStages * S::kStage;
    o.template read<S::kARow, S::kWRow, AR>(slot, am, wk * (kACpr / WK), slot + S::kABytes, an, wk * (kWCpr / WK), slot + S::kABytes + S::kWBytes + wk * AR * 4,
                                            slot + S::kABytes + S::kWBytes + S::kAUnits * 256 + wk * BN * 4, r, g);
  };

  // ---- the ring ----
  fetch(0);
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s)
    if (s < ns) issue(s);
  stash(0);
  for (int st = 0; st < ns; ++st) {
    if (st + kStages - 2 < ns) wait_vmcnt<(kStages - 2) * kLoads>(); else wait_vmcnt<0>();    // my loads of this stage have landed
    __builtin_amdgcn_s_waitcnt(0xc07f);                      // lgkmcnt(0): my reads of the last stage and my rows of this one are done
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    if (!kDirect && st + 1 < ns) fetch(st + 1);
    if (st + kStages - 1 < ns) issue(st + kStages - 1);
    if (WK == 1 || st * WK + wk < nk) {
      Ops o;
      read(o, st);
      o.multiply(acc, K - (st * WK + wk) * 128, g, [](int) {});
    }
    if (!kDirect && st + 1 < ns) stash(st + 1);
  }

  // ---- results: lane has columns 4 g .. 4 g + 3 of row r of each 16 x 16 tile ----
  if constexpr (WK > 1) {
    floatx4 *sums = reinterpret_cast<floatx4 *>(lds);        // [wk][wm, wn][tile][lane]
    __syncthreads();                                         // every wave is done with the ring
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) sums[(wave * NT * MT + nt * MT + mt) * 64 + lane] = acc[nt][mt];
    __syncthreads();
  }
  auto result = [&](int nt, int mt) {                        // in the order of k
    if constexpr (WK == 1) return acc[nt][mt];
    const floatx4 *sums = reinterpret_cast<const floatx4 *>(lds) + ((wave % (WM * WN)) * NT * MT + nt * MT + mt) * 64 + lane;
    floatx4 s = sums[0];
#pragma unroll
    for (int k = 1; k < WK; ++k) s += sums[k * WM * WN * NT * MT * 64];
    return s;
  };
  if constexpr (kSwiglu) {
    const int Np = (N + kMxStage - 1) / kMxStage * kMxStage, c0 = n0 + wn * 32;
    if (c0 >= Np) return;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      if (WK > 1 && mt % WK != wk) continue;
      const int m = m0 + am + mt * 16;
      store_act(result(0, mt), result(1, mt), result(2, mt), result(3, mt), m < M, m, c0, g, p, Np);
    }
  } else {
    using T = std::conditional_t<OUT == kOutF32, float, bf16_t>;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        if (WK > 1 && (mt * NT + nt) % WK != wk) continue;
        const int m = m0 + am + mt * 16;
        if (m < M) store_row4<T>(result(nt, mt), m, n0 + wn * (BN / WN) + nt * 16 + 4 * g, p);
      }
  }
}

// Lets a kernel have so much LDS on the current device: asked for once a device (bits of `done`), by concurrent first callers perhaps twice.
pvf_status allow_lds(const void *kernel, int bytes, std::atomic<uint64_t> &done) {
  int device = 0;
  PVF_HIP_CHECK(nullptr, hipGetDevice(&device));
  const uint64_t bit = 1ull << (device & 63);
  if (done.load(std::memory_order_relaxed) & bit) return PVF_OK;
  PVF_HIP_CHECK(nullptr, hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes));
  done.fetch_or(bit, std::memory_order_relaxed);
  return PVF_OK;
}

template <int ROWS, int WF, int OUT, int BM, int BN, int WM, int WN, int WK, int kStages, int AR = BM, bool kDirect = true>
pvf_status run_as(hipStream_t s, const MxGemm &p) {
  using S = Shape<ROWS, WF, BM, BN, WM, WN, WK, kStages, AR>;
  static_assert(S::kLds <= 160 * 1024, "LDS");
  TileMap tm;
  const int64_t tiles_n = OUT == kOutSwiglu ? (mx_width(p.N) + BN / 2 - 1) / (BN / 2) : (p.N + BN - 1) / BN, tiles_m = (p.M + BM - 1) / BM;
  PVF_REQUIRE(nullptr, tiles_m * tiles_n < 1 << 28, PVF_ESHAPE, "%d x %d results are too many for a launch", p.M, p.N);
  tm.tiles_m = (int)tiles_m; tm.tiles_n = (int)tiles_n; tm.group_m = (int)std::min<int64_t>(tiles_m, 8);
  auto kernel = gemm_mx_kernel<ROWS, WF, OUT, BM, BN, WM, WN, WK, kStages, AR, kDirect>;
  static std::atomic<uint64_t> allowed{0};
  if (const pvf_status st = allow_lds((const void *)kernel, S::kLds, allowed)) return st;
  kernel<<<mx_grid((tiles_m * tiles_n + 7) / 8 * 8), S::kThreads, S::kLds, s>>>(p, tm);
  PVF_LAUNCH_CHECK(nullptr, "gemm_mx");
  return PVF_OK;
}

// ---- waves of their own -------------------------------------------------------------------------------------------------
// A workgroup computes BM x BN results for launches whose tiles make about one round over the chip: its kWaves waves take the 128s of k in turn, each
// with the whole tile and a ring of two slots of LDS of its own, so that the loop has no barrier and the waves' loads, reads and matrix
// instructions drift apart; a slot is loaded again as soon as it is in registers.  The sums are added through LDS at the end.
// Bound by the bytes in flight: 4 waves with two stages of 80 x 64 are all of a CU's LDS.  320 x 4096 x 12288, e4m3 weights: 25-26 us, 1.8 MB for each CU
// in 20 us behind 5 of launch and first loads (one ring with a barrier a stage: 30); splitting k over workgroups as well would need a workspace.  One
// row against 4-bit weights 12288 x 4096: 6.9 us with the call, 3.9 TB/s; 320 rows against 4096 x 4096: 18-19 us.
template <int ROWS, int WF, int OUT, int BM, int BN, int kWaves, int AR>
__global__ void __launch_bounds__(64 * kWaves)
gemm_mx_waves_kernel(MxGemm p, TileMap tm) {
  constexpr bool kSwiglu = OUT == kOutSwiglu, kCodes = codes_in(ROWS), kW8 = WF == PVF_MX_E4M3;
  using S = Shape<ROWS, WF, BM, BN, 1, 1, 1, 2, AR>;
  constexpr int MT = BM / 16, NT = BN / 16, kASize = S::kASize;
  constexpr int kACpr = S::kARow / 16, kWCpr = S::kWRow / 16, kAChunks = AR * kACpr;
  constexpr int LA = (kAChunks + 63) / 64, LW = BN * kWCpr / 64, LS = S::kAUnits + S::kWUnits, kLoads = LA + LW + LS;
  static_assert(kLoads < 64 && kAChunks % 64 == 0 && BN * kWCpr % 64 == 0, "whole load instructions");
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  const int M = p.M, N = p.N, K = p.K, Kp = (K + kMxStage - 1) / kMxStage * kMxStage, nk = Kp / kMxStage;
  const int total = tm.tiles_m * tm.tiles_n, per_xcd = (total + 7) >> 3;
  const int block = mx_block(), L = (block & 7) * per_xcd + (block >> 3);
  if (block >> 3 >= per_xcd || L >= total) return;
  const int band = L / (tm.group_m * tm.tiles_n), within = L - band * (tm.group_m * tm.tiles_n);
  const int band_rows = min(tm.group_m, tm.tiles_m - band * tm.group_m);
  const int tile_n = within / band_rows, tile_m = band * tm.group_m + (within - tile_n * band_rows);
  const int m0 = tile_m * BM, n0 = tile_n * (kSwiglu ? BN / 2 : BN), w_rows = kSwiglu ? 2 * N : N;
  auto w_row = [&](int t) -> int64_t {                       // SwiGLU: 32 gate rows, then the 32 up rows of the same columns
    if (!kSwiglu) return min(n0 + t, N - 1);
    const int n = min(n0 + (t >> 6) * 32 + (t & 31), N - 1);
    return (t & 32) ? (int64_t)N + n : n;
  };
  const uint32_t a_bytes = (uint32_t)((kCodes ? Kp : K) * kASize), w_bytes = kW8 ? Kp : Kp / 2;
  const uint8_t *a_src[LA], *w_src[LW], *s_src[LS];
  uint32_t a_at[LA];
#pragma unroll
  for (int i = 0; i < LA; ++i) {
    const int f = (i * 64 + lane) % kAChunks, row = f / kACpr;
    a_at[i] = ((f % kACpr) ^ swizzle<S::kARow, S::kAX>(row)) * 16;
    a_src[i] = (const uint8_t *)p.A + (int64_t)min(m0 + row, M - 1) * a_bytes + (kCodes ? a_at[i] : 0);
  }
#pragma unroll
  for (int i = 0; i < LW; ++i) {
    const int f = i * 64 + lane, row = f / kWCpr;
    w_src[i] = (const uint8_t *)p.W + w_row(row) * w_bytes + ((f % kWCpr) ^ swizzle<S::kWRow, S::kWX>(row)) * 16;
  }
#pragma unroll
  for (int i = 0; i < LS; ++i) {
    const int f = (i < S::kAUnits ? i : i - S::kAUnits) * 64 + lane;
    s_src[i] = i < S::kAUnits ? p.a_scales + (int64_t)min(m0 + min(f, AR - 1), M - 1) * 4 : p.w_scales + w_row(min(f, BN - 1)) * 4;
  }
  unsigned char *own = lds + wave * (2 * S::kStage);
  auto issue = [&](int kt, int slot, int l) {                // l-th load of a stage
    unsigned char *at = own + slot * S::kStage;
    if (l < LA) {
      const uint8_t *q = kCodes ? a_src[l % LA] + (int64_t)kt * S::kARow : a_src[l % LA] + min(a_at[l % LA] + (uint32_t)kt * S::kARow, a_bytes - 16);      // behind a row its last chunk
      __builtin_amdgcn_global_load_lds((gptr_t *)q, (lptr_t *)(at + l * 64 % kAChunks * 16), 16, 0, 0);
    } else if (l < LA + LW) {
      __builtin_amdgcn_global_load_lds((gptr_t *)(w_src[(l - LA) % LW] + (int64_t)kt * S::kWRow), (lptr_t *)(at + S::kABytes + (l - LA) * 1024), 16, 0, 0);
    } else {
      const int i = l - LA - LW;
      __builtin_amdgcn_global_load_lds((gptr_t *)(s_src[i % LS] + (int64_t)kt * (i < S::kAUnits ? M : w_rows) * 4), (lptr_t *)(at + S::kABytes + S::kWBytes + i * 256), 4, 0, 0);
    }
  };
  floatx4 acc[NT][MT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) acc[nt][mt] = floatx4{0.f, 0.f, 0.f, 0.f};
  const int mine = wave < nk ? (nk - wave + kWaves - 1) / kWaves : 0;       // stages of this wave: wave, wave + kWaves, ...
  using Ops = Operands<ROWS, WF, MT, NT>;
  Ops o[2];
  auto piece = [&](Ops &to, int slot, int q) {
    const unsigned char *at = own + slot * S::kStage;
    to.template read_piece<S::kARow, S::kWRow, AR>(q, at, r, 0, at + S::kABytes, r, 0, at + S::kABytes + S::kWBytes, at + S::kABytes + S::kWBytes + S::kAUnits * 256, r, g);
  };
  if (mine > 0) {
#pragma unroll
    for (int l = 0; l < kLoads; ++l) issue(wave, 0, l);
    if (mine > 1) {
#pragma unroll
      for (int l = 0; l < kLoads; ++l) issue(wave + kWaves, 1, l);
      wait_vmcnt<kLoads>();
    } else wait_vmcnt<0>();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int q = 0; q < Ops::kPieces; ++q) piece(o[0], 0, q);
  }
  // The n-th stage of the wave is multiplied from registers.  Behind its first instructions the stage after the next is asked for (its slot has
  // been read), in the middle the next one has landed, and behind the last instructions it is read.  Kind 0: all of that, 1: no stage after
  // the next, 2: the last stage.
  auto step = [&](int n, auto kind, auto parity) {
    constexpr int P = decltype(parity)::value, kKind = decltype(kind)::value, U = Ops::kInstrs, kHalf = (U + 1) / 2;
    if (kKind == 0) __builtin_amdgcn_s_waitcnt(0xc07f);      // lgkmcnt(0): the slot is in registers
    __builtin_amdgcn_sched_barrier(0);
    auto landed = [&]() {
      if (kKind == 0) wait_vmcnt<kLoads>(); else wait_vmcnt<0>();
      asm volatile("" ::: "memory");
    };
    o[P].multiply(acc, K - (wave + n * kWaves) * 128, g, [&](int i) {
      __builtin_amdgcn_sched_barrier(0);
      if (kKind == 0)
#pragma unroll
        for (int l = 0; l < kLoads; ++l)
          if (l * kHalf / kLoads == i) issue(wave + (n + 2) * kWaves, P, l);
      if (kKind < 2 && i == kHalf - 1) landed();
      if (kKind < 2)
#pragma unroll
        for (int q = 0; q < Ops::kPieces; ++q)
          if (U > kHalf ? i == kHalf + q * (U - kHalf) / Ops::kPieces : i == U - 1) piece(o[P ^ 1], P ^ 1, q);
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  constexpr std::integral_constant<int, 0> k0{};
  constexpr std::integral_constant<int, 1> k1{};
  constexpr std::integral_constant<int, 2> k2{};
  if (mine > 0) {
    int n = 0;
    for (; n + 3 < mine; n += 2) {
      step(n, k0, k0);
      step(n + 1, k0, k1);
    }
    if (mine - n == 3) { step(n, k0, k0); step(n + 1, k1, k1); step(n + 2, k2, k0); }
    else if (mine - n == 2) { step(n, k1, k0); step(n + 1, k2, k1); }
    else step(n, k2, k0);
  }
  // ---- results ----
  floatx4 *sums = reinterpret_cast<floatx4 *>(lds);          // [wave][tile][lane]
  __syncthreads();
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) sums[(wave * NT * MT + nt * MT + mt) * 64 + lane] = acc[nt][mt];
  __syncthreads();
  auto result = [&](int nt, int mt) {                        // in the order of the waves
    floatx4 s = sums[(nt * MT + mt) * 64 + lane];
#pragma unroll
    for (int k = 1; k < kWaves; ++k) s += sums[(k * NT * MT + nt * MT + mt) * 64 + lane];
    return s;
  };
  if constexpr (kSwiglu) {
    const int Np = (N + kMxStage - 1) / kMxStage * kMxStage;
    for (int t = wave; t < MT * (NT / 4); t += kWaves) {
      const int mt = t % MT, b = t / MT, m = m0 + mt * 16 + r, c0 = n0 + b * 32;
      if (c0 < Np) store_act(result(4 * b, mt), result(4 * b + 1, mt), result(4 * b + 2, mt), result(4 * b + 3, mt), m < M, m, c0, g, p, Np);
    }
  } else {
    using T = std::conditional_t<OUT == kOutF32, float, bf16_t>;
    for (int t = wave; t < MT * NT; t += kWaves) {
      const int m = m0 + t % MT * 16 + r;
      const floatx4 s = result(t / MT, t % MT);
      if (m < M) store_row4<T>(s, m, n0 + t / MT * 16 + 4 * g, p);
    }
  }
}

template <int ROWS, int WF, int OUT, int BM, int BN, int kWaves, int AR>
pvf_status run_waves(hipStream_t s, const MxGemm &p) {
  using S = Shape<ROWS, WF, BM, BN, 1, 1, 1, 2, AR>;
  constexpr int kLds = kWaves * (2 * S::kStage > BM * BN * 4 ? 2 * S::kStage : BM * BN * 4);
  static_assert(kLds <= 160 * 1024, "LDS");
  TileMap tm;
  const int64_t tiles_n = OUT == kOutSwiglu ? (mx_width(p.N) + BN / 2 - 1) / (BN / 2) : (p.N + BN - 1) / BN, tiles_m = (p.M + BM - 1) / BM;
  PVF_REQUIRE(nullptr, tiles_m * tiles_n < 1 << 28, PVF_ESHAPE, "%d x %d results are too many for a launch", p.M, p.N);
  tm.tiles_m = (int)tiles_m; tm.tiles_n = (int)tiles_n; tm.group_m = (int)std::min<int64_t>(tiles_m, 8);
  auto kernel = gemm_mx_waves_kernel<ROWS, WF, OUT, BM, BN, kWaves, AR>;
  static std::atomic<uint64_t> allowed{0};
  if (const pvf_status st = allow_lds((const void *)kernel, kLds, allowed)) return st;
  kernel<<<mx_grid((tiles_m * tiles_n + 7) / 8 * 8), 64 * kWaves, kLds, s>>>(p, tm);
  PVF_LAUNCH_CHECK(nullptr, "gemm_mx");
  return PVF_OK;
}

// ---- results of decoded operands, a step ahead ------------------------------------------------------------------------------
// 32 TM x 128 results, four waves of 16 TM x 64.  A stage is four steps of 32 k of 4 TM matrix instructions a wave.  Between the instructions of a step the operands of the next are decoded (two
// conversions a matrix instruction) and the codes after those are read from LDS; in the middle of a stage the next one has landed, every wave
// has read this one, one barrier, and its slot is loaded again.  Two workgroups fit a CU's registers.
// Bound by issue: a conversion beside a matrix instruction costs 2 cycles of its 16 (measured: 7.3 ns an instruction alone, 9.5 with two conversions), so
// 1.3 times the matrix time is the limit.  gate|up of 2560 rows, 12288 x 4096, e4m3 weights: 395-419 us, 1.3 PFLOP/s (bfloat16 products of
// a library, 16384 cube: 1.6; the same tile on one ring, decoding before the instructions: 441 us; this library's bfloat16 product with SwiGLU: 372-387).  64 rows, 4-bit weights, 64 x 128 tiles of four stages: 21-22 us, where the
// loads alone take 15: the conversions of 192 workgroups' weights do not all fit beside them.
template <int WF, int OUT, int TM, int kStages>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2)))
gemm_mx_steps_kernel(MxGemm p, TileMap tm) {
  constexpr bool kSwiglu = OUT == kOutSwiglu, kW8 = WF == PVF_MX_E4M3;
  constexpr int BM = 32 * TM, BN = 128, T = 4;               // T: tiles of 16 columns of a wave, TM of 16 rows
  using S = Shape<kRowsMxExact, WF, BM, BN, 2, 2, 1, kStages>;
  static_assert(kStages % 2 == 0, "the loop takes stages in pairs");
  constexpr int LA = TM, LW = kW8 ? 4 : 2, kLoads = LA + LW + 1, kUnits = BM / 64, CPR = S::kWRow / 16;
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave >> 1, wn = wave & 1, r = lane & 15, g = lane >> 4;
  const int M = p.M, N = p.N, Kp = (p.K + kMxStage - 1) / kMxStage * kMxStage, nk = Kp / kMxStage;
  const int total = tm.tiles_m * tm.tiles_n, per_xcd = (total + 7) >> 3;
  const int block = mx_block(), L = (block & 7) * per_xcd + (block >> 3);
  if (block >> 3 >= per_xcd || L >= total) return;
  const int band = L / (tm.group_m * tm.tiles_n), within = L - band * (tm.group_m * tm.tiles_n);
  const int band_rows = min(tm.group_m, tm.tiles_m - band * tm.group_m);
  const int tile_n = within / band_rows, tile_m = band * tm.group_m + (within - tile_n * band_rows);
  const int m0 = tile_m * BM, n0 = tile_n * (kSwiglu ? BN / 2 : BN), n_first = min(n0, N - 1);
  const uint32_t w_bytes = kW8 ? Kp : Kp / 2;
  // Rows by 32-bit offsets from the tile's first (128 rows of at most 2^22 bytes).  SwiGLU: of every 64 rows of the tile the lower 32 are gate, the
  // upper 32 up, which a wave's load has one of.
  const uint8_t *a_base = (const uint8_t *)p.A + (int64_t)m0 * Kp, *w_base = (const uint8_t *)p.W + (int64_t)n_first * w_bytes;
  uint32_t a_off[LA], w_off[LW];
#pragma unroll
  for (int i = 0; i < LA; ++i) {
    const int row = i * 32 + tid / 8;
    a_off[i] = (uint32_t)(min(m0 + row, M - 1) - m0) * (uint32_t)Kp + ((tid % 8) ^ swizzle<128, 2>(row)) * 16;
  }
#pragma unroll
  for (int i = 0; i < LW; ++i) {
    const int t = i * (256 / CPR) + tid / CPR, n = kSwiglu ? n0 + (t >> 6) * 32 + (t & 31) : n0 + t;
    w_off[i] = (uint32_t)(min(n, N - 1) - n_first) * w_bytes + ((tid % CPR) ^ swizzle<S::kWRow, S::kWX>(t)) * 16;
  }
  // scale dwords, 64 a wave: those of A, then those of W (64 rows of A: the fourth wave repeats the third's)
  const int unit = min(wave, kUnits + 1), s_t = (unit < kUnits ? unit : unit - kUnits) * 64 + lane;
  int64_t s_at = min(m0 + s_t, M - 1);
  if (unit >= kUnits) s_at = !kSwiglu ? min(n0 + s_t, N - 1) : min(n0 + (s_t >> 6) * 32 + (s_t & 31), N - 1) + ((s_t & 32) ? (int64_t)N : 0);
  const uint8_t *s_src = (unit < kUnits ? p.a_scales : p.w_scales) + s_at * 4;
  const int64_t s_step = (int64_t)(unit < kUnits ? M : kSwiglu ? 2 * N : N) * 4;
  auto issue = [&](int kt, int slot, int l) {
    unsigned char *at = lds + slot * S::kStage;
    if (l < LA) __builtin_amdgcn_global_load_lds((gptr_t *)(a_base + (int64_t)kt * 128 + a_off[l % LA]), (lptr_t *)(at + l * 4096 + wave * 1024), 16, 0, 0);
    else if (l < LA + LW) {
      const int i = l - LA;
      const bool up = kSwiglu && (kW8 ? i & 1 : wave >> 1);
      __builtin_amdgcn_global_load_lds((gptr_t *)(w_base + (int64_t)kt * S::kWRow + (up ? (int64_t)N * w_bytes : 0) + w_off[i % LW]), (lptr_t *)(at + S::kABytes + i * 4096 + wave * 1024), 16, 0, 0);
    } else
      __builtin_amdgcn_global_load_lds((gptr_t *)(s_src + kt * s_step), (lptr_t *)(at + S::kABytes + S::kWBytes + unit * 256), 4, 0, 0);
  };
  floatx4 acc[T][TM];
#pragma unroll
  for (int nt = 0; nt < T; ++nt)
#pragma unroll
    for (int mt = 0; mt < TM; ++mt) acc[nt][mt] = floatx4{0.f, 0.f, 0.f, 0.f};
  const int am = wm * (16 * TM) + r, an = wn * 64 + r;
  // codes: chunk h of A (and of e4m3 W) in set h; e2m1 W, one chunk a stage, in set kt % 2.  Scales in set kt % 2.
  intx4 ca[2][TM], cw[2][T];
  int as[2][TM], ws[2][T];
  bf16x8 da[2][TM], dw[2][T];                                 // decoded operands of step j in set j % 2
  auto read_a = [&](int slot, int h, int mt) {
    ca[h][mt] = *reinterpret_cast<const intx4 *>(lds + slot * S::kStage + (mt * 16 + am) * 128 + (((2 * g + h) ^ swizzle<128, 2>(r)) << 4));
  };
  auto read_w = [&](int slot, int h, int nt) {               // e2m1: h is the set
    const unsigned char *row = lds + slot * S::kStage + S::kABytes + (nt * 16 + an) * S::kWRow;
    cw[h][nt] = *reinterpret_cast<const intx4 *>(row + (((kW8 ? 2 * g + h : g) ^ swizzle<S::kWRow, S::kWX>(r)) << 4));
  };
  auto read_s = [&](int slot, int set, int q) {
    const unsigned char *at = lds + slot * S::kStage + S::kABytes + S::kWBytes + g;
    if (q < TM) as[set][q % TM] = at[(q * 16 + am) * 4]; else ws[set][(q - TM) % T] = at[BM * 4 + ((q - TM) * 16 + an) * 4];
  };
  auto decode = [&](int j, int set, int f) {                 // fragment f of step j of a stage whose scales are in `set`
    const int h = j >> 1, lo = j * 2 & 3;
    if (f < T) dw[j & 1][f % T] = kW8 ? decode_e4m3(cw[h][f % T][lo], cw[h][f % T][lo + 1], byte_scale(ws[set][f % T])) : decode_e2m1(cw[set][f % T][j], byte_scale(ws[set][f % T]));
    else da[j & 1][(f - T) % TM] = decode_e4m3(ca[h][(f - T) % TM][lo], ca[h][(f - T) % TM][lo + 1], byte_scale(as[set][(f - T) % TM]));
  };
#pragma unroll
  for (int st = 0; st < kStages; ++st)
    if (st < nk)
#pragma unroll
      for (int l = 0; l < kLoads; ++l) issue(st, st, l);
  if (kStages <= nk) wait_vmcnt<(kStages - 1) * kLoads>(); else wait_vmcnt<0>();
  __builtin_amdgcn_s_barrier();
#pragma unroll
  for (int q = 0; q < TM + T; ++q) read_s(0, 0, q);
#pragma unroll
  for (int q = 0; q < T; ++q) read_w(0, 0, q);
#pragma unroll
  for (int q = 0; q < TM; ++q) read_a(0, 0, q);
#pragma unroll
  for (int f = 0; f < T + TM; ++f) decode(0, 0, f);
  int slot = 0;                                              // of stage kt
  // kind 0: kStages more stages follow, 1: at least one, 2: none
  auto stage = [&](int kt, auto kind, auto parity) {
    constexpr int P = decltype(parity)::value, kKind = decltype(kind)::value, U = T * TM, kFrags = T + TM;
    const int next = kStages == 2 ? P ^ 1 : slot + 1 == kStages ? 0 : slot + 1, here = kStages == 2 ? P : slot;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (j == 2 && kKind < 2) {
        if (kKind == 0) wait_vmcnt<(kStages - 2) * kLoads>(); else wait_vmcnt<0>();      // my loads of the next stage have landed
        __builtin_amdgcn_s_waitcnt(0xc07f);                  // lgkmcnt(0): my reads of this one are done
        __builtin_amdgcn_s_barrier();
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int nt = i / TM, mt = i % TM;
        acc[nt][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(dw[j & 1][nt], da[j & 1][mt], acc[nt][mt], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int q = 0; q < kFrags; ++q)
          if (i == q * U / 2 / kFrags) {
            if (j == 0) { if (q < TM) read_a(here, 1, q % TM); else if (kW8) read_w(here, 1, (q - TM) % T); }
            if (j == 2 && kKind < 2) read_s(next, P ^ 1, q);
            if (j == 2 && kKind < 2) { if (q < T) read_w(next, kW8 ? 0 : P ^ 1, q % T); else read_a(next, 0, (q - T) % TM); }
          }
        if (kKind == 0 && j >= 2) {                          // loads of the stage that takes this one's slot
#pragma unroll
          for (int l = 0; l < kLoads; ++l)
            if ((j - 2) * U + i == 1 + l * (2 * U - 2) / kLoads) issue(kt + kStages, here, l);
        }
        if (j < 3 || kKind < 2)
#pragma unroll
          for (int f = 0; f < kFrags; ++f)
            if (i == (f + 1) * U / kFrags - 1) decode((j + 1) & 3, j < 3 ? P : P ^ 1, f);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    slot = next;
  };
  constexpr std::integral_constant<int, 0> k0{};
  constexpr std::integral_constant<int, 1> k1{};
  constexpr std::integral_constant<int, 2> k2{};
  int kt = 0;                                                // nk is even
  for (; kt + kStages + 1 < nk; kt += 2) {
    stage(kt, k0, k0);
    stage(kt + 1, k0, k1);
  }
  if constexpr (kStages > 2)
    for (; kt + 2 < nk; kt += 2) {
      stage(kt, k1, k0);
      stage(kt + 1, k1, k1);
    }
  stage(nk - 2, k1, k0);
  stage(nk - 1, k2, k1);

  if constexpr (kSwiglu) {
    const int Np = (N + kMxStage - 1) / kMxStage * kMxStage, c0 = n0 + wn * 32;
    if (c0 >= Np) return;
#pragma unroll
    for (int mt = 0; mt < TM; ++mt) store_act(acc[0][mt], acc[1][mt], acc[2][mt], acc[3][mt], m0 + am + mt * 16 < M, m0 + am + mt * 16, c0, g, p, Np);
  } else {
#pragma unroll
    for (int mt = 0; mt < TM; ++mt)
#pragma unroll
      for (int nt = 0; nt < T; ++nt)
        if (m0 + am + mt * 16 < M) store_row4<float>(acc[nt][mt], m0 + am + mt * 16, n0 + wn * 64 + nt * 16 + 4 * g, p);
  }
}

template <int WF, int OUT, int TM, int kStages> pvf_status run_steps(hipStream_t s, const MxGemm &p) {
  using S = Shape<kRowsMxExact, WF, 32 * TM, 128, 2, 2, 1, kStages>;
  static_assert(S::kLds <= 160 * 1024, "LDS");
  TileMap tm;
  const int64_t tiles_n = OUT == kOutSwiglu ? mx_width(p.N) / 64 : (p.N + 127) / 128, tiles_m = (p.M + 32 * TM - 1) / (32 * TM);
  PVF_REQUIRE(nullptr, tiles_m * tiles_n < 1 << 28, PVF_ESHAPE, "%d x %d results are too many for a launch", p.M, p.N);
  tm.tiles_m = (int)tiles_m; tm.tiles_n = (int)tiles_n; tm.group_m = (int)std::min<int64_t>(tiles_m, 8);
  auto kernel = gemm_mx_steps_kernel<WF, OUT, TM, kStages>;
  static std::atomic<uint64_t> allowed{0};
  if (const pvf_status st = allow_lds((const void *)kernel, S::kLds, allowed)) return st;
  kernel<<<mx_grid((tiles_m * tiles_n + 7) / 8 * 8), 256, S::kLds, s>>>(p, tm);
  PVF_LAUNCH_CHECK(nullptr, "gemm_mx");
  return PVF_OK;
}

// ---- 256 x 256 results: two stages of LDS, a wave's 128 x 64 results in quadrants --------------------------------------
// Row of the tile behind LDS row r: the lower halves of all wave tiles come first, then the upper ones, so that a half is a run of whole loads.
template <int BT, int WT> __device__ __forceinline__ int half_row(int r) {
  constexpr int kHalfTile = BT / 2, kHalfWave = WT / 2;
  const int h = r / kHalfTile, rr = r % kHalfTile;
  return (rr / kHalfWave) * WT + h * kHalfWave + rr % kHalfWave;
}

// A wave multiplies, stage by stage of 128 k, lower A x lower W, lower x upper, upper x upper, upper x lower.  The operands of a half are read
// from LDS one quadrant before their first use, which frees their rows early: each half of a stage's slot is refilled as soon as it is
// read, one barrier per half stage, so loads are issued evenly and have 1 to 1.5 stages to land.  Scale bytes have a ring of three stages.
// Bound by power: 11520 x 12288 x 4096, e4m3 weights, 435-459 us, 2.6 PFLOP/s at 1.8 GHz of 2.4 with the matrix pipe busy for 553 000 cycles, 0.7 of the
// time (a library's 8-bit product without block scales: 3.0 at 8192 cubed, 3.2 at 16384).  256 x 256 because a tile's operands are 1 / 128 of its work: 192 x 256 with one
// barrier a stage takes 586 us.  e2m1 weights: 493-514 us, ten registers spilled where one operand of the instruction is 4 registers wide and the other 8.
template <int WF>
__global__ void __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2)))
gemm_mx_quad_kernel(MxGemm p, TileMap tm) {
  constexpr bool kW8 = WF == PVF_MX_E4M3;
  constexpr int BM = 256, BN = 256, WTM = 128, WTN = 64, MH = 4, NH = 2, kPer = MH * NH;
  constexpr int kWRow = kW8 ? 128 : 64, kABytes = BM * 128, kWBytes = BN * kWRow, kScales = 2 * (kABytes + kWBytes), kScaleStage = (BM + BN) * 4;
  constexpr int LA = 4, LW = kW8 ? 4 : 2, kG1 = 1 + LA / 2 + LW / 2, kG2 = LA / 2 + LW / 2, kLoads = kG1 + kG2;
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 2, wn = wave & 3, r = lane & 15, g = lane >> 4;
  const int M = p.M, N = p.N, Kp = (p.K + kMxStage - 1) / kMxStage * kMxStage, nk = Kp / kMxStage;
  const int total = tm.tiles_m * tm.tiles_n, per_xcd = (total + 7) >> 3;
  const int block = mx_block(), L = (block & 7) * per_xcd + (block >> 3);
  if (block >> 3 >= per_xcd || L >= total) return;
  const int band = L / (tm.group_m * tm.tiles_n), within = L - band * (tm.group_m * tm.tiles_n);
  const int band_rows = min(tm.group_m, tm.tiles_m - band * tm.group_m);
  const int tile_n = within / band_rows, tile_m = band * tm.group_m + (within - tile_n * band_rows);
  const int m_own = tile_m * BM, n_own = tile_n * BN;        // the last tiles begin early, so that all of a tile exists, and store only what is theirs
  const int m0 = min(m_own, M - BM), n0 = min(n_own, N - BN);
  const uint32_t w_bytes = kW8 ? Kp : Kp / 2;

  // The i-th load of an operand lies a uniform distance behind the first: LDS rows 64 i are tile rows 128 i of the lower halves, then 64 (A)
  // or 32 (W) further on.  So a lane has one offset for each operand (32 bits: 256 rows of at most 2^22 bytes) and no address arithmetic.
  const uint32_t a_off = (tid / 8) * (uint32_t)Kp + ((tid % 8) ^ swizzle<128, 1>(tid / 8)) * 16;
  constexpr int CPR = kWRow / 16;
  const uint32_t w_off = half_row<BN, WTN>(tid / CPR) * w_bytes + ((tid % CPR) ^ swizzle<kWRow, 1>(tid / CPR)) * 16;
  const bool of_a = wave < 4;                                // waves 0-3 load the scale dwords of A, 4-7 those of W
  const uint32_t s_row = (wave & 3) * 64 + lane, s_off = (of_a ? half_row<BM, WTM>(s_row) : half_row<BN, WTN>(s_row)) * 4;
  const uint32_t s_step = (of_a ? M : N) * 4;
#ifdef __HIP_DEVICE_COMPILE__
  const __amdgpu_buffer_rsrc_t rsA = __builtin_amdgcn_make_buffer_rsrc((void *)((const uint8_t *)p.A + (int64_t)m0 * Kp), 0, BM * Kp, 0x00020000);
  const __amdgpu_buffer_rsrc_t rsW = __builtin_amdgcn_make_buffer_rsrc((void *)((const uint8_t *)p.W + (int64_t)n0 * w_bytes), 0, (int)(BN * w_bytes), 0x00020000);
  const __amdgpu_buffer_rsrc_t rsS = __builtin_amdgcn_make_buffer_rsrc((void *)(of_a ? p.a_scales + (int64_t)m0 * 4 : p.w_scales + (int64_t)n0 * 4), 0, (int)(s_step * nk - (of_a ? m0 : n0) * 4), 0x00020000);
#endif
  // q-th load of a stage: scales, lower A, lower W | upper W, upper A
  auto issue = [&](int kt, int q, int s3) {                  // s3: kt % 3
#ifdef __HIP_DEVICE_COMPILE__
    auto a = [&](int i) { __builtin_amdgcn_raw_ptr_buffer_load_lds(rsA, (lptr_t *)(lds + (kt & 1) * kABytes + i * 8192 + wave * 1024), 16, a_off, kt * 128 + ((i & 1) * 128 + (i >> 1) * 64) * Kp, 0, 0); };
    auto w = [&](int i) {
      const int first = kW8 ? (i & 1) * 128 + (i >> 1) * 32 : i * 32;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsW, (lptr_t *)(lds + 2 * kABytes + (kt & 1) * kWBytes + i * 8192 + wave * 1024), 16, w_off, kt * kWRow + first * w_bytes, 0, 0);
    };
    if (q == 0) __builtin_amdgcn_raw_ptr_buffer_load_lds(rsS, (lptr_t *)(lds + kScales + s3 * kScaleStage + wave * 256), 4, s_off, kt * s_step, 0, 0);
    else if (q < 1 + LA / 2) a(q - 1);
    else if (q < kG1) w(q - 1 - LA / 2);
    else if (q < kG1 + LW / 2) w(q - kG1 + LW / 2);
    else a(q - kG1 - LW / 2 + LA / 2);
#endif
  };
  floatx4 acc[2 * NH][2 * MH];
#pragma unroll
  for (int nt = 0; nt < 2 * NH; ++nt)
#pragma unroll
    for (int mt = 0; mt < 2 * MH; ++mt) acc[nt][mt] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int st = 0; st < 2; ++st)
    if (st < nk)
#pragma unroll
      for (int q = 0; q < kLoads; ++q) issue(st, q, st);

  intx8 a0[MH], a1[MH], b[2][NH];
  int as0[MH], as1[MH], bs[2][NH];
  const int a_row = wm * (WTM / 2) + r, w_row = wn * (WTN / 2) + r;
  const int a_c0 = a_row * 128 + ((g ^ swizzle<128, 1>(r)) << 4), a_c1 = a_row * 128 + (((4 + g) ^ swizzle<128, 1>(r)) << 4);
  const int w_c0 = 2 * kABytes + w_row * kWRow + ((g ^ swizzle<kWRow, 1>(r)) << 4), w_c1 = 2 * kABytes + w_row * kWRow + (((4 + g) ^ swizzle<128, 1>(r)) << 4);
  const int s_a = kScales + a_row * 4 + g, s_w = kScales + (BM + w_row) * 4 + g;
  auto rd_a = [&](int parity, int s3, int half, int j, intx8 &v, int &s) {
    const int at = parity * kABytes + half * (BM / 2 * 128) + j * 16 * 128;
    v = join(*reinterpret_cast<const intx4 *>(lds + a_c0 + at), *reinterpret_cast<const intx4 *>(lds + a_c1 + at));
    s = lds[s_a + s3 * kScaleStage + (half * (BM / 2) + j * 16) * 4];
  };
  auto rd_w = [&](int parity, int s3, int half, int j, intx8 &v, int &s) {
    const int at = parity * kWBytes + half * (BN / 2 * kWRow) + j * 16 * kWRow;
    v = kW8 ? join(*reinterpret_cast<const intx4 *>(lds + w_c0 + at), *reinterpret_cast<const intx4 *>(lds + w_c1 + at))
            : join(*reinterpret_cast<const intx4 *>(lds + w_c0 + at));
    s = lds[s_w + s3 * kScaleStage + (half * (BN / 2) + j * 16) * 4];
  };
  if (nk > 1) wait_vmcnt<kG2 + kLoads>(); else wait_vmcnt<kG2>();
  __builtin_amdgcn_s_barrier();
#pragma unroll
  for (int j = 0; j < NH; ++j) rd_w(0, 0, 0, j, b[0][j], bs[0][j]);
#pragma unroll
  for (int j = 0; j < MH; ++j) rd_a(0, 0, 0, j, a0[j], as0[j]);

  constexpr int kBarrierAt = 2, kSlots = 2 * kPer - kBarrierAt;
  int s3 = 0;                                                // kt % 3
  auto stage = [&](int kt, auto kind, auto parity) {         // kind 0: a stage that prefetches, 1: the last but one, 2: the last
    constexpr int P = decltype(parity)::value;
    constexpr bool kSteady = decltype(kind)::value == 0, more = decltype(kind)::value < 2;
    const int s3n = s3 == 2 ? 0 : s3 + 1, s3nn = s3n == 2 ? 0 : s3n + 1;
#pragma unroll
    for (int ph = 0; ph < 4; ++ph) {
      const int mh = ph >> 1, nh = ph == 1 || ph == 2;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int mt = i / NH, nt = i % NH;
        if (i == kBarrierAt && (ph == 0 || (ph == 2 && more))) {
          // ph 0: all of stage kt has landed; ph 2: the lower halves of stage kt + 1 have (my parts of them)
          if (ph == 0) { if (more) wait_vmcnt<kLoads>(); else wait_vmcnt<0>(); }
          else { if (kSteady) wait_vmcnt<kG2 + kG1>(); else wait_vmcnt<kG2>(); }
          __builtin_amdgcn_s_waitcnt(0xc07f);                // lgkmcnt(0): my reads of the rows that are refilled now are done
          __builtin_amdgcn_s_barrier();
          __builtin_amdgcn_sched_barrier(0);
        }
        floatx4 &c = acc[nh * NH + nt][mh * MH + mt];
#ifdef __HIP_DEVICE_COMPILE__
        c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b[nh ^ P][nt], mh ? a1[mt] : a0[mt], c, kW8 ? 0 : 4, 0, 0, bs[nh ^ P][nt], 0, mh ? as1[mt] : as0[mt]);
#endif
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < MH; ++j) {
          if (ph == 0 && j < NH && i == kBarrierAt + j * (kPer - kBarrierAt - 2) / NH) rd_w(P, s3, 1, j, b[P ^ 1][j], bs[P ^ 1][j]);
          if (ph == 1 && i == j * (kPer - 2) / MH) rd_a(P, s3, 1, j, a1[j], as1[j]);
          if (ph == 2 && more && i == kBarrierAt + j * (kPer - kBarrierAt) / MH) rd_a(P ^ 1, s3n, 0, j, a0[j], as0[j]);
          if (ph == 3 && more && j < NH && i == j * (kPer - 4) / NH) rd_w(P ^ 1, s3n, 0, j, b[P ^ 1][j], bs[P ^ 1][j]);
        }
        if (kSteady) {
          const int at = (ph & 1) * kPer + i - kBarrierAt;   // instructions since the half's barrier
#pragma unroll
          for (int q = 0; q < (ph < 2 ? kG1 : kG2); ++q)
            if (at == 1 + q * (kSlots - 1) / (ph < 2 ? kG1 : kG2)) issue(kt + 2, ph < 2 ? q : kG1 + q, s3nn);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    s3 = s3n;
  };
  constexpr std::integral_constant<int, 0> k0{};
  constexpr std::integral_constant<int, 1> k1{};
  constexpr std::integral_constant<int, 2> k2{};
  for (int kt = 0; kt + 2 < nk; kt += 2) {                   // nk is even
    stage(kt, k0, k0);
    stage(kt + 1, k0, k1);
  }
  stage(nk - 2, k1, k0);
  stage(nk - 1, k2, k1);

  // ---- results, 32 rows at a time through the wave's own piece of the free ring: stores of whole 128-byte lines ----
  // lane: column half * 32 + 16 nt + 4 g of row half * 64 + 16 mt + r of the wave's tile
  const int wave_m = m0 + wm * WTM, wave_n = n0 + wn * WTN;
  __syncthreads();
  if (N % 8 != 0) {
#pragma unroll
    for (int mt = 0; mt < 2 * MH; ++mt)
#pragma unroll
      for (int nt = 0; nt < 2 * NH; ++nt)
        if (wave_m + mt * 16 + r >= m_own) store_row4<bf16_t>(acc[nt][mt], wave_m + mt * 16 + r, wave_n + nt * 16 + 4 * g, p, n_own);
    return;
  }
  constexpr int kRow = WTN * 4 + 16;                         // float32, so that a residual is added before the rounding
  unsigned char *my = lds + wave * 32 * kRow;
#pragma unroll
  for (int mp = 0; mp < MH; ++mp) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int nt = 0; nt < 2 * NH; ++nt) *reinterpret_cast<floatx4 *>(my + (h * 16 + r) * kRow + (nt * 16 + 4 * g) * 4) = acc[nt][2 * mp + h];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int row = j * 8 + (lane >> 3), m = wave_m + mp * 32 + row, n = wave_n + (lane & 7) * 8;
      const floatx4 lo = *reinterpret_cast<const floatx4 *>(my + row * kRow + (lane & 7) * 32), hi = *reinterpret_cast<const floatx4 *>(my + row * kRow + (lane & 7) * 32 + 16);
      if (m < m_own || n < n_own) continue;
      float v[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) { v[e] = lo[e]; v[4 + e] = hi[e]; }
      if (p.residual) {
        float x[8];
        load8((const bf16_t *)p.residual + (int64_t)m * N + n, 8, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += x[e];
      }
      store8((bf16_t *)p.C + (int64_t)m * N + n, 8, v);
    }
  }
}

// M, N >= 256, an even number of stages, scales of less than 2^31 bytes.
template <int WF> pvf_status run_quad(hipStream_t s, const MxGemm &p) {
  constexpr int kLds = 2 * (256 * 128 + 256 * (WF == PVF_MX_E4M3 ? 128 : 64)) + 3 * 512 * 4;
  TileMap tm;
  const int64_t tiles_n = (p.N + 255) / 256, tiles_m = (p.M + 255) / 256;
  PVF_REQUIRE(nullptr, tiles_m * tiles_n < 1 << 28, PVF_ESHAPE, "%d x %d results are too many for a launch", p.M, p.N);
  tm.tiles_m = (int)tiles_m; tm.tiles_n = (int)tiles_n; tm.group_m = (int)std::min<int64_t>(tiles_m, 6);   // 8: 2 % slower at 8192 x 8192, nothing at 11520 x 12288
  auto kernel = gemm_mx_quad_kernel<WF>;
  static std::atomic<uint64_t> allowed{0};
  if (const pvf_status st = allow_lds((const void *)kernel, kLds, allowed)) return st;
  kernel<<<mx_grid((tiles_m * tiles_n + 7) / 8 * 8), 512, kLds, s>>>(p, tm);
  PVF_LAUNCH_CHECK(nullptr, "gemm_mx");
  return PVF_OK;
}

// ---- which instance -------------------------------------------------------------------------------------------------
// What a tile costs for 128 k, in microseconds, measured at K = 4096 and 12288 (launch time less 3 us, over the stages and the tiles of the fullest CU):
// where a CU has one tile, and per tile where it has several (those that fit its LDS run at a time and hide each other's barriers and
// latencies).  The launch takes the instance whose fullest CU is done first.  Of 188 launches of 1 to 11520 rows, against 4096 x 4096, 12288 x 4096 and 4096 x 12288 mostly, 181 take at
// most 1.05 times what the best of their list takes, the others up to 1.18.  Small tiles cost what their rows' loads cost, not their area.  Known to be off, because
// SwiGLU and float32 results have one cost for weights of either type, and one for stages whether weights come from HBM or a cache: SwiGLU of up to 16 rows against e4m3 weights 12288 x 4096
// takes 30 us on 16 x 64 tiles (64 x 64: 25); 11520 x 4096 x 12288 with e2m1 weights 547 on 256 x 256 (192 x 256: 472); 1280 x 4096 x 4096 of bfloat16 rows against 4-bit weights
// 56 on 32 x 128 (64 x 128: 50); 320 x 12288 x 4096 with e2m1 weights and float32 results 41 on 64 x 128 (80 x 64: 37).
struct Candidate {
  int BM, BN, most_rows;                                     // most_rows: rows of A that the instance loads (0: any number)
  float alone, among;
  pvf_status (*run)(hipStream_t, const MxGemm &);
  bool pairs = false;                                        // takes stages of 128 k in pairs
  int least = 0;                                             // rows and columns that there have to be
};

template <int ROWS, int WF, int OUT, bool kDirect> struct Candidates;
#define PVF_MX_TILE(BM, BN, WM, WN, WK, ST, AR, alone, among) \
  {BM, OUT == kOutSwiglu ? BN / 2 : BN, AR < BM ? AR : 0, alone, among, run_as<ROWS, WF, OUT, BM, BN, WM, WN, WK, ST, AR, kDirect>}

#define PVF_MX_WAVES(BM, BN, waves, AR, alone, among) \
  {BM, OUT == kOutSwiglu ? BN / 2 : BN, AR < BM ? AR : 0, alone, among, run_waves<ROWS, WF, OUT, BM, BN, waves, AR>}

template <int WF, bool kDirect> struct Candidates<kRowsMx, WF, kOutBf16, kDirect> {
  static constexpr int ROWS = kRowsMx, OUT = kOutBf16;
  static constexpr Candidate list[] = {
      PVF_MX_WAVES(16, 16, 4, 16, .079f, .070f),          PVF_MX_WAVES(32, 32, 4, 32, .115f, .112f),          PVF_MX_WAVES(64, 32, 4, 64, .17f, .186f),
      PVF_MX_WAVES(48, 64, 4, 48, .215f, .20f),           PVF_MX_WAVES(64, 64, 4, 64, .24f, .253f),           PVF_MX_TILE(64, 64, 2, 2, 2, 2, 64, .38f, .217f),   PVF_MX_WAVES(80, 64, 4, 80, .26f, .34f),
      PVF_MX_TILE(96, 64, 2, 2, 1, 3, 96, .39f, .28f),    PVF_MX_TILE(64, 128, 2, 4, 1, 3, 64, .44f, .375f), PVF_MX_TILE(128, 128, 2, 2, 1, 2, 128, .78f, .51f),
      PVF_MX_TILE(160, 128, 2, 4, 1, 2, 160, .83f, .74f), PVF_MX_TILE(192, 256, 2, 4, 1, 2, 192, 1.49f, 1.44f), {256, 256, 0, WF == PVF_MX_E4M3 ? 1.3f : 1.75f, WF == PVF_MX_E4M3 ? 1.5f : 1.62f, run_quad<WF>, true, 256}};
};
template <int WF, bool kDirect> struct Candidates<kRowsMxExact, WF, kOutF32, kDirect> {
  static constexpr int ROWS = kRowsMxExact, OUT = kOutF32;
  static constexpr Candidate list[] = {
      PVF_MX_WAVES(16, 16, 8, 16, .09f, .10f),           PVF_MX_WAVES(32, 32, 4, 32, .135f, .12f),           PVF_MX_WAVES(48, 64, 4, 48, .275f, .27f),
      PVF_MX_WAVES(64, 64, 4, 64, .325f, .35f),          PVF_MX_WAVES(80, 64, 4, 80, .425f, .45f),          PVF_MX_TILE(64, 128, 2, 4, 1, 3, 64, .74f, .61f),   PVF_MX_TILE(128, 128, 2, 2, 1, 2, 128, 1.2f, .91f), {128, 128, 0, 1.1f, .84f, run_steps<WF, OUT, 4, 2>, true},
      PVF_MX_TILE(160, 128, 2, 4, 1, 2, 160, 1.43f, 1.22f)};
};
template <int WF, bool kDirect> struct Candidates<kRowsMxExact, WF, kOutSwiglu, kDirect> {
  static constexpr int ROWS = kRowsMxExact, OUT = kOutSwiglu;
  static constexpr Candidate list[] = {
      PVF_MX_TILE(16, 64, 1, 1, 4, 2, 16, .18f, .14f),   PVF_MX_TILE(32, 64, 1, 1, 4, 2, 32, .25f, .20f),    PVF_MX_TILE(64, 128, 2, 2, 1, 2, 64, .67f, .57f),
      {64, 64, 0, .53f, .65f, run_steps<WF, OUT, 2, 4>, true}, PVF_MX_TILE(128, 128, 2, 2, 1, 2, 128, 1.2f, .90f), {128, 64, 0, 1.1f, .81f, run_steps<WF, OUT, 4, 2>, true}};
};
// rows that go through registers have the instances of one kernel only
template <> struct Candidates<kRowsBf16, PVF_MX_E2M1, kOutBf16, true> {
  static constexpr int ROWS = kRowsBf16, WF = PVF_MX_E2M1, OUT = kOutBf16;
  static constexpr bool kDirect = true;
  static constexpr Candidate list[] = {
      PVF_MX_WAVES(16, 16, 4, 4, .06f, .044f),           PVF_MX_WAVES(16, 16, 8, 16, .055f, .10f),
      PVF_MX_TILE(16, 16, 1, 1, 4, 2, 16, .095f, .058f), PVF_MX_WAVES(16, 64, 8, 16, .154f, .153f),          PVF_MX_WAVES(32, 32, 4, 32, .135f, .154f),
      PVF_MX_TILE(32, 64, 2, 1, 2, 2, 32, .35f, .205f),  PVF_MX_WAVES(48, 64, 4, 48, .27f, .27f),            PVF_MX_WAVES(32, 128, 4, 32, .327f, .33f),
      PVF_MX_WAVES(80, 64, 3, 80, .49f, .47f),           PVF_MX_TILE(64, 128, 2, 2, 1, 2, 64, .75f, .58f)};
};
template <> struct Candidates<kRowsBf16, PVF_MX_E2M1, kOutBf16, false> {
  static constexpr int ROWS = kRowsBf16, WF = PVF_MX_E2M1, OUT = kOutBf16;
  static constexpr bool kDirect = false;
  static constexpr Candidate list[] = {
      PVF_MX_TILE(16, 16, 1, 1, 8, 2, 1, .04f, .047f),   PVF_MX_TILE(16, 16, 1, 1, 8, 2, 4, .06f, .05f),     PVF_MX_TILE(16, 16, 1, 1, 4, 2, 16, .095f, .058f),
      PVF_MX_TILE(32, 32, 2, 1, 4, 2, 32, .19f, .20f),   PVF_MX_TILE(32, 64, 2, 1, 2, 2, 32, .35f, .215f),   PVF_MX_TILE(64, 128, 2, 2, 1, 2, 64, .75f, .58f)};
};
template <> struct Candidates<kRowsF32, PVF_MX_E2M1, kOutF32, true> {
  static constexpr int ROWS = kRowsF32, WF = PVF_MX_E2M1, OUT = kOutF32;
  static constexpr bool kDirect = true;
  static constexpr Candidate list[] = {
      PVF_MX_TILE(16, 16, 1, 1, 8, 2, 1, .16f, .14f),    PVF_MX_TILE(16, 64, 1, 1, 8, 2, 1, .25f, .24f),     PVF_MX_TILE(16, 16, 1, 1, 8, 2, 16, .18f, .225f),
      PVF_MX_WAVES(16, 64, 8, 4, .265f, .295f),          PVF_MX_WAVES(16, 64, 4, 16, .36f, .375f),           PVF_MX_WAVES(16, 128, 4, 16, .53f, .54f),
      PVF_MX_TILE(64, 128, 4, 1, 1, 2, 64, 1.92f, 1.98f)};
};
template <> struct Candidates<kRowsF32, PVF_MX_E2M1, kOutF32, false> {
  static constexpr int ROWS = kRowsF32, WF = PVF_MX_E2M1, OUT = kOutF32;
  static constexpr bool kDirect = false;
  static constexpr Candidate list[] = {
      PVF_MX_TILE(16, 16, 1, 1, 8, 2, 1, .20f, .16f),    PVF_MX_TILE(16, 64, 1, 1, 8, 2, 1, .32f, .33f),     PVF_MX_TILE(16, 64, 1, 1, 8, 2, 4, .36f, .36f),
      PVF_MX_TILE(16, 16, 1, 1, 8, 2, 16, .37f, .38f),   PVF_MX_TILE(16, 64, 1, 1, 4, 2, 16, .57f, .60f),    PVF_MX_TILE(32, 32, 2, 1, 4, 2, 32, .62f, .70f),
      PVF_MX_TILE(32, 64, 2, 1, 2, 2, 32, 1.0f, 1.1f),   PVF_MX_TILE(64, 128, 4, 1, 1, 2, 64, 2.9f, 2.5f),   PVF_MX_TILE(32, 128, 2, 1, 2, 2, 32, 1.45f, 1.45f)};
};

template <int ROWS, int WF, int OUT, bool kDirect = true> MxInstance choose(const MxGemm &p) {
  const int64_t columns = OUT == kOutSwiglu ? mx_width(p.N) : p.N;
  const int64_t stages = mx_width(p.K) / kMxStage;
  const Candidate *best = nullptr;
  float least = 0.f;
  for (const Candidate &c : Candidates<ROWS, WF, OUT, kDirect>::list) {
    if (c.most_rows && p.M > c.most_rows) continue;
    if ((c.pairs && stages % 2 != 0) || p.M < c.least || p.N < c.least || (c.least && stages * std::max(p.M, p.N) >= 1 << 29)) continue;      // (scales by 32-bit offsets)
    const int64_t tiles = ((p.M + c.BM - 1) / c.BM) * ((columns + c.BN - 1) / c.BN), fullest = (tiles + 255) / 256;
    const float cost = fullest == 1 ? c.alone : c.among * (float)fullest;
    if (!best || cost < least) { best = &c; least = cost; }
  }
  const auto &list = Candidates<ROWS, WF, OUT, kDirect>::list;
  return {best->run, (int)(best - list), (int)std::size(list)};
}

template <int WF> MxInstance choose_mx(const MxGemm &p) {
  if (p.c_scales) return choose<kRowsMxExact, WF, kOutSwiglu>(p);
  if (p.dtype == PVF_F32) return choose<kRowsMxExact, WF, kOutF32>(p);
  return choose<kRowsMx, WF, kOutBf16>(p);
}

}  // namespace

MxInstance gemm_mx_instance(const MxGemm &p) {
  if (!p.a_scales) {                                         // rows that begin at 16-byte chunks go straight to LDS
    const bool f32 = p.dtype == PVF_F32, direct = (uintptr_t)p.A % 16 == 0 && p.K % (f32 ? 4 : 8) == 0;
    if (f32) return direct ? choose<kRowsF32, PVF_MX_E2M1, kOutF32>(p) : choose<kRowsF32, PVF_MX_E2M1, kOutF32, false>(p);
    return direct ? choose<kRowsBf16, PVF_MX_E2M1, kOutBf16>(p) : choose<kRowsBf16, PVF_MX_E2M1, kOutBf16, false>(p);
  }
  return p.w_fmt == PVF_MX_E4M3 ? choose_mx<PVF_MX_E4M3>(p) : choose_mx<PVF_MX_E2M1>(p);
}

pvf_status launch_gemm_mx(hipStream_t s, const MxGemm &p) {
  if (p.M == 0 || p.N == 0) return PVF_OK;
  return gemm_mx_instance(p).run(s, p);
}

}  // namespace pvf
