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
// result, a hundredth of a bfloat16 rounding.  Float32 results do not take it (the bfloat16 instruction keeps float32 sums), nor does SwiGLU,
// whose 8-bit results would differ from the definition's in 0.3 % of the codes and here and there in a block's scale, where float32
// sums differ in one of 10^5; it would take half the time of the matrix instructions.
//
// Operands of the scaled 16 x 16 x 128 instruction: lane (r = lane % 16, g = lane / 16) holds row r; of e4m3 the 16 bytes at k = 16 g and
// the 16 at 64 + 16 g, of e2m1 the 32 elements from 32 g on; its scale byte is that of k = 32 g .. 32 g + 31.  The weights are the
// instruction's first operand, so that a lane ends up with 4 consecutive columns of C.
#include "mx.h"

#include <algorithm>

namespace pvf {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef int intx4 __attribute__((ext_vector_type(4)));
typedef int intx8 __attribute__((ext_vector_type(8)));

enum Rows { kRowsMx, kRowsMxExact, kRowsBf16, kRowsF32 };   // what multiplies what (table above)
enum Out { kOutBf16, kOutF32, kOutSwiglu };

template <int WF> constexpr int code_bytes(int elements) { return WF == PVF_MX_E4M3 ? elements : elements / 2; }

__device__ __forceinline__ float silu_f(float g) { return g * __builtin_amdgcn_rcpf(1.0f + __expf(-g)); }

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

// x = p[0] + p[1] + p[2] exactly, 8 bits of the mantissa each, cut off and not rounded so that nothing overflows; what is not finite is
// in p[0] alone.
__device__ __forceinline__ void split3(const float *x, bf16x8 *p) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t u = __float_as_uint(x[e]);
    const bool fine = (u & 0x7f800000u) != 0x7f800000u;
    const float r = fine ? x[e] - __uint_as_float(u & 0xffff0000u) : 0.f;
    const float b = __uint_as_float(__float_as_uint(r) & 0xffff0000u);
    p[0][e] = fine ? __builtin_bit_cast(bf16_t, (uint16_t)(u >> 16)) : (bf16_t)x[e];
    p[1][e] = __builtin_bit_cast(bf16_t, (uint16_t)(__float_as_uint(r) >> 16));
    p[2][e] = (bf16_t)(r - b);
  }
}

// ---- results ------------------------------------------------------------------------------------------------------
// Columns n .. n + 3 of row m.
template <typename T> __device__ __forceinline__ void store_row4(floatx4 v, int m, int n, const MxGemm &p) {
  const int N = p.N;
  T *row = (T *)p.C + (int64_t)m * N;
  const T *res = p.residual ? (const T *)p.residual + (int64_t)m * N : nullptr;
  if (N % 4 == 0 && n < N) {                                 // a row begins as C does, at an element: unaligned vectors
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
    if (n + e < N) row[n + e] = from_float<T>(v[e] + (res ? to_float(res[n + e]) : 0.f));
}

// silu(gate) * up of 32 columns from c0 on, of which the lane has 4 g .. + 3 and 16 + 4 g .. + 3: a block, as codes and scale.  All 64 lanes.
__device__ __forceinline__ void store_act(floatx4 g0, floatx4 g1, floatx4 u0, floatx4 u1, bool live, int m, int c0, int g, const MxGemm &p, int Np) {
  float v[8];
  uint32_t am = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[e] = c0 + 4 * g + e < p.N ? silu_f(g0[e]) * u0[e] : 0.f;
    v[4 + e] = c0 + 16 + 4 * g + e < p.N ? silu_f(g1[e]) * u1[e] : 0.f;
    am = max(am, max(abs_bits(v[e]), abs_bits(v[4 + e])));
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

// ---- few rows -----------------------------------------------------------------------------------------------------
// A workgroup computes 16 MT rows x 16 NT columns; its KW waves take the stages of 128 k in turn, operands straight from memory into the
// registers of the instruction, and add their sums through LDS.  Weights are read once for all rows of a workgroup.
template <int ROWS, int WF, int OUT, int MT, int NT, int KW>
__global__ void __launch_bounds__(64 * KW)
gemm_mx_rows_kernel(MxGemm p, uint32_t n_tiles) {
  constexpr bool kSwiglu = OUT == kOutSwiglu;
  constexpr int kPlanes = ROWS == kRowsF32 ? 3 : 1;
  static_assert(!kSwiglu || NT == 4, "SwiGLU: two column tiles of gate, two of up, a block of 32 outputs");
  __shared__ floatx4 sums[KW][NT * MT][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const int M = p.M, N = p.N, K = p.K, Kp = (K + kMxStage - 1) / kMxStage * kMxStage, nk = Kp / kMxStage;
  const int w_rows = kSwiglu ? 2 * N : N;
  const int n0 = (int)(blockIdx.x % n_tiles) * (kSwiglu ? 32 : 16 * NT), m0 = (int)(blockIdx.x / n_tiles) * (16 * MT);
  const uint8_t *w_ptr[NT], *a_ptr[MT];
  uint32_t w_s[NT], a_s[MT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int n = kSwiglu ? min(n0 + (nt & 1) * 16 + r, N - 1) + (nt >= 2 ? N : 0) : min(n0 + nt * 16 + r, N - 1);
    w_ptr[nt] = (const uint8_t *)p.W + (int64_t)n * code_bytes<WF>(Kp);
    w_s[nt] = n * 4 + g;
  }
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int m = min(m0 + mt * 16 + r, M - 1);
    a_ptr[mt] = (const uint8_t *)p.A + (ROWS == kRowsBf16 ? (int64_t)m * K * 2 : ROWS == kRowsF32 ? (int64_t)m * K * 4 : (int64_t)m * Kp);
    a_s[mt] = m * 4 + g;
  }
  floatx4 acc[NT][MT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) acc[nt][mt] = floatx4{0.f, 0.f, 0.f, 0.f};

  for (int kt = wave; kt < nk; kt += KW) {
    if constexpr (ROWS == kRowsMx) {
      intx8 w[NT], a[MT];
      int ws[NT], as[MT];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        if (WF == PVF_MX_E4M3) {
          const intx4 *q = reinterpret_cast<const intx4 *>(w_ptr[nt] + kt * 128 + 16 * g);
          w[nt] = join(q[0], q[4]);
        } else {
          const intx4 q = *reinterpret_cast<const intx4 *>(w_ptr[nt] + kt * 64 + 16 * g);
          w[nt] = join(q, intx4{0, 0, 0, 0});
        }
        ws[nt] = p.w_scales[(int64_t)kt * w_rows * 4 + w_s[nt]];
      }
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        const intx4 *q = reinterpret_cast<const intx4 *>(a_ptr[mt] + kt * 128 + 16 * g);
        a[mt] = join(q[0], q[4]);
        as[mt] = p.a_scales[(int64_t)kt * M * 4 + a_s[mt]];
      }
#ifdef __HIP_DEVICE_COMPILE__
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
          acc[nt][mt] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w[nt], a[mt], acc[nt][mt], WF == PVF_MX_E4M3 ? 0 : 4, 0, 0, ws[nt], 0, as[mt]);
#endif
    } else {
      // four instructions of 32 k: lane g has elements 32 g + 8 j .. + 7 of the stage in the j-th, all of one block
      intx4 w[NT][WF == PVF_MX_E4M3 ? 2 : 1];
      float ws[NT];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const intx4 *q = reinterpret_cast<const intx4 *>(w_ptr[nt] + code_bytes<WF>(kt * 128 + 32 * g));
        w[nt][0] = q[0];
        if (WF == PVF_MX_E4M3) w[nt][WF == PVF_MX_E4M3 ? 1 : 0] = q[1];
        ws[nt] = byte_scale(p.w_scales[(int64_t)kt * w_rows * 4 + w_s[nt]]);
      }
      bf16x8 a[MT][4][kPlanes];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        const int k = kt * 128 + 32 * g;
        if constexpr (ROWS == kRowsMxExact) {
          const intx4 *q = reinterpret_cast<const intx4 *>(a_ptr[mt] + k);
          const intx4 q0 = q[0], q1 = q[1];
          const float as = byte_scale(p.a_scales[(int64_t)kt * M * 4 + a_s[mt]]);
          a[mt][0][0] = decode_e4m3(q0[0], q0[1], as); a[mt][1][0] = decode_e4m3(q0[2], q0[3], as);
          a[mt][2][0] = decode_e4m3(q1[0], q1[1], as); a[mt][3][0] = decode_e4m3(q1[2], q1[3], as);
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int kj = k + 8 * j;
            if constexpr (ROWS == kRowsBf16) {
              a[mt][j][0] = __builtin_bit_cast(bf16x8, load8_raw((const bf16_t *)a_ptr[mt] + min(kj, K), K - kj));
            } else {
              float x[8];
              load8((const float *)a_ptr[mt] + min(kj, K), K - kj, x);
              split3(x, a[mt][j]);
            }
          }
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const bf16x8 wf = WF == PVF_MX_E4M3 ? decode_e4m3(w[nt][WF == PVF_MX_E4M3 ? j >> 1 : 0][j * 2 & 3], w[nt][WF == PVF_MX_E4M3 ? j >> 1 : 0][(j * 2 & 3) + 1], ws[nt])
                                              : decode_e2m1(w[nt][0][j], ws[nt]);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int q = kPlanes - 1; q >= 0; --q)
              acc[nt][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf, a[mt][j][q], acc[nt][mt], 0, 0, 0);
        }
    }
  }
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) sums[wave][nt * MT + mt][lane] = acc[nt][mt];
  __syncthreads();
  auto total = [&](int t, int l) {                           // in the order of the waves
    floatx4 s = sums[0][t][l];
#pragma unroll
    for (int w = 1; w < KW; ++w) s += sums[w][t][l];
    return s;
  };
  if constexpr (kSwiglu) {
    const int Np = (N + kMxStage - 1) / kMxStage * kMxStage;
    for (int mt = wave; mt < MT; mt += KW) {
      const int m = m0 + mt * 16 + r;
      store_act(total(mt, lane), total(MT + mt, lane), total(2 * MT + mt, lane), total(3 * MT + mt, lane), m < M, m, n0, g, p, Np);
    }
  } else {
    using T = std::conditional_t<OUT == kOutF32, float, bf16_t>;
    for (int t = wave; t < NT * MT; t += KW) {
      const int m = m0 + t % MT * 16 + r;
      const floatx4 s = total(t, lane);
      if (m < M) store_row4<T>(s, m, n0 + t / MT * 16 + 4 * g, p);
    }
  }
}

template <int ROWS, int WF, int OUT>
pvf_status run_rows(hipStream_t s, const MxGemm &p) {
  constexpr int NT = OUT == kOutSwiglu ? 4 : 1, KW = 4;
  const uint32_t n_tiles = OUT == kOutSwiglu ? (uint32_t)(mx_width(p.N) / 32) : (p.N + 16 * NT - 1) / (16 * NT);
  auto go = [&](auto mt) -> pvf_status {
    constexpr int MT = decltype(mt)::value;
    const int64_t grid = (int64_t)n_tiles * ((p.M + 16 * MT - 1) / (16 * MT));
    PVF_REQUIRE(nullptr, grid <= INT32_MAX, PVF_ESHAPE, "%d x %d results are too many for a launch", p.M, p.N);
    gemm_mx_rows_kernel<ROWS, WF, OUT, MT, NT, KW><<<(uint32_t)grid, 64 * KW, 0, s>>>(p, n_tiles);
    PVF_LAUNCH_CHECK(nullptr, "gemm_mx");
    return PVF_OK;
  };
  if (p.M <= 16) return go(std::integral_constant<int, 1>{});
  if (p.M <= 32 || ROWS == kRowsF32) return go(std::integral_constant<int, 2>{});
  return go(std::integral_constant<int, 4>{});
}


// ---- many rows ----------------------------------------------------------------------------------------------------
typedef __attribute__((address_space(1))) const void gptr_t;
typedef __attribute__((address_space(3))) void lptr_t;

// s_waitcnt vmcnt(n) only; n is a 6-bit field split 4 + 2
template <int N> __device__ __forceinline__ void wait_vmcnt() {
  static_assert(N >= 0 && N < 64, "vmcnt is a 6-bit counter");
  __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | ((N >> 4) << 14));
}

struct TileMap { int tiles_m, tiles_n, group_m; };

// Bytes of LDS that a stage of 128 k takes: operand rows, then their scale dwords.
template <int ROWS> constexpr int a_stage_bytes(int BM) { return ROWS == kRowsBf16 ? BM * 256 : ROWS == kRowsF32 ? BM * 768 : BM * 128; }
constexpr bool codes_in(int ROWS) { return ROWS == kRowsMx || ROWS == kRowsMxExact; }

// A workgroup computes BM x BN results, a wave BM / WM x BN / WN of them.  Stages of 128 k go through a ring of kStages slots of LDS: codes and scales
// straight from memory (a 16-byte chunk of a row sits at chunk position ^ swizzle(row), chosen by the lane's source address, so that the
// reads of 16 rows touch every bank once), rows of bf16 / float32 through registers, where float32 is split into its three parts.
template <int ROWS, int WF, int OUT, int BM, int BN, int WM, int WN, int kStages>
__global__ void __launch_bounds__(64 * WM * WN)
gemm_mx_tile_kernel(MxGemm p, TileMap tm) {
  constexpr bool kSwiglu = OUT == kOutSwiglu, kCodes = codes_in(ROWS), kW8 = WF == PVF_MX_E4M3;
  constexpr int kThreads = 64 * WM * WN, kWaves = WM * WN, WTM = BM / WM, WTN = BN / WN, MT = WTM / 16, NT = WTN / 16;
  constexpr int kPlanes = ROWS == kRowsF32 ? 3 : 1;
  constexpr int kABytes = a_stage_bytes<ROWS>(BM), kWRow = kW8 ? 128 : 64, kWBytes = BN * kWRow;
  constexpr int kASlots = kCodes ? kStages : 2;
  constexpr int kAScale = 0, kWScale = kCodes ? BM * 4 : 0, kScaleBytes = kWScale + BN * 4;
  constexpr int kWBase = kASlots * kABytes, kSBase = kWBase + kStages * kWBytes;
  // load instructions of a thread and stage
  constexpr int LA = kCodes ? BM * 8 / kThreads : 0, LW = kWBytes / 16 / kThreads;
  constexpr int kScaleUnits = kScaleBytes / 256, LS = (kScaleUnits + kWaves - 1) / kWaves, kLoads = LA + LW + LS;
  constexpr int LX = kCodes ? 0 : BM * 16 / kThreads;       // 8-element chunks of rows that a thread stages
  static_assert(BM % (16 * WM) == 0 && BN % (16 * WN) == 0 && (kCodes ? BM * 8 : BM * 16) % kThreads == 0 && kWBytes / 16 % kThreads == 0, "tile shape");
  static_assert(BM % 64 == 0 && BN % 64 == 0 && (!kSwiglu || WTN == 64), "scale dwords are loaded 64 at a time; a wave has a block of gate and of up");
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN, r = lane & 15, g = lane >> 4;
  const int M = p.M, N = p.N, K = p.K, Kp = (K + kMxStage - 1) / kMxStage * kMxStage, nk = Kp / kMxStage;

  // the 32 workgroups that an XCD runs at a time cover a patch of tiles and share operands through its L2
  const int total = tm.tiles_m * tm.tiles_n, chunk = (total + 7) >> 3;
  const int L = (int)(blockIdx.x & 7) * chunk + (int)(blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= chunk || L >= total) return;
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
  // ---- sources of this thread's direct loads ----
  const uint8_t *a_src = nullptr, *w_src[LW], *s_src[LS];
  int64_t a_step[LA > 0 ? LA : 1] = {};
  if (kCodes) {
    const int row = tid / 8, c = (tid % 8) ^ ((row >> 1) & 7);
    const int64_t first = min(m0 + row, M - 1);
    a_src = (const uint8_t *)p.A + first * Kp + c * 16;
#pragma unroll
    for (int i = 0; i < LA; ++i) a_step[i] = (min(m0 + i * (kThreads / 8) + row, M - 1) - first) * Kp;
  }
#pragma unroll
  for (int i = 0; i < LW; ++i) {
    constexpr int CPR = kWRow / 16;
    const int row = (i * kThreads + tid) / CPR, c = (tid % CPR) ^ (kW8 ? (row >> 1) & 7 : (row >> 2) & 3);
    w_src[i] = (const uint8_t *)p.W + w_row(row) * (Kp / (kW8 ? 1 : 2)) + c * 16;
  }
  int s_slot[LS];
  int64_t s_step[LS];
#pragma unroll
  for (int i = 0; i < LS; ++i) {                             // every wave has as many loads as the others: some repeat a unit
    const int u = (i * kWaves + wave) % kScaleUnits;
    s_slot[i] = u * 256;
    const bool of_a = kCodes && u < BM / 64;
    const int t = (of_a ? u : u - kWScale / 256) * 64 + lane;
    s_src[i] = of_a ? p.a_scales + (int64_t)min(m0 + t, M - 1) * 4 : p.w_scales + w_row(t) * 4;
    s_step[i] = (int64_t)(of_a ? M : w_rows) * 4;
  }
  auto issue = [&](int kt) {
    const int slot = kt % kStages;
#pragma unroll
    for (int i = 0; i < LA; ++i)
      __builtin_amdgcn_global_load_lds((gptr_t *)(a_src + a_step[i] + (int64_t)kt * 128), (lptr_t *)(lds + slot * kABytes + (i * kThreads + wave * 64) * 16), 16, 0, 0);
#pragma unroll
    for (int i = 0; i < LW; ++i)
      __builtin_amdgcn_global_load_lds((gptr_t *)(w_src[i] + (int64_t)kt * kWRow), (lptr_t *)(lds + kWBase + slot * kWBytes + (i * kThreads + wave * 64) * 16), 16, 0, 0);
#pragma unroll
    for (int i = 0; i < LS; ++i)
      __builtin_amdgcn_global_load_lds((gptr_t *)(s_src[i] + kt * s_step[i]), (lptr_t *)(lds + kSBase + slot * kScaleBytes + s_slot[i]), 4, 0, 0);
  };
  // ---- rows of bf16 / float32: chunk tid % 16 of rows tid / 16 + i * kThreads / 16 ----
  constexpr int kXRegs = LX > 0 ? LX : 1;
  uint4 xb[ROWS == kRowsBf16 ? kXRegs : 1];
  float xf[ROWS == kRowsF32 ? kXRegs : 1][8];
  auto fetch = [&](int kt) {
    const int k = kt * 128 + (tid & 15) * 8;
#pragma unroll
    for (int i = 0; i < LX; ++i) {
      const int64_t at = (int64_t)min(m0 + i * (kThreads / 16) + (tid >> 4), M - 1) * K + min(k, K);
      if constexpr (ROWS == kRowsBf16) xb[i] = load8_raw((const bf16_t *)p.A + at, K - k);
      if constexpr (ROWS == kRowsF32) load8((const float *)p.A + at, K - k, xf[i]);
    }
  };
  auto stash = [&](int kt) {                                 // plane, half of 64 k, row, chunk
    unsigned char *dst = lds + (kt & 1) * kABytes + (tid >> 3 & 1) * (BM * 128);
#pragma unroll
    for (int i = 0; i < LX; ++i) {
      const int row = i * (kThreads / 16) + (tid >> 4);
      unsigned char *q = dst + row * 128 + (((tid & 7) ^ (row >> 1 & 7)) << 4);
      if constexpr (ROWS == kRowsBf16) *reinterpret_cast<uint4 *>(q) = xb[i];
      if constexpr (ROWS == kRowsF32) {
        bf16x8 part[3];
        split3(xf[i], part);
#pragma unroll
        for (int e = 0; e < 3; ++e) *reinterpret_cast<bf16x8 *>(q + e * (BM * 256)) = part[e];
      }
    }
  };

  floatx4 acc[NT][MT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) acc[nt][mt] = floatx4{0.f, 0.f, 0.f, 0.f};

  if (!kCodes) { fetch(0); stash(0); }
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s)
    if (s < nk) issue(s);

  const int swz = (r >> 1) & 7, am = wm * WTM + r, an = wn * WTN + r;       // rows of the lane's operands in the tiles
  auto compute = [&](int kt) {
    const int slot = kt % kStages;
    const unsigned char *la = lds + (kCodes ? slot : kt & 1) * kABytes + am * 128, *lw = lds + kWBase + slot * kWBytes + an * kWRow;
    const unsigned char *sa = lds + kSBase + slot * kScaleBytes + am * 4 + g, *sw = lds + kSBase + slot * kScaleBytes + kWScale + an * 4 + g;
    auto chunk_of = [&](const unsigned char *row, int c) { return *reinterpret_cast<const intx4 *>(row + ((c ^ swz) << 4)); };
    auto w4_chunk = [&](int nt) { return *reinterpret_cast<const intx4 *>(lw + nt * 16 * 64 + ((g ^ (r >> 2 & 3)) << 4)); };
    if constexpr (ROWS == kRowsMx) {
      intx8 a[MT];
      int as[MT];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        a[mt] = join(chunk_of(la + mt * 16 * 128, g), chunk_of(la + mt * 16 * 128, 4 + g));
        as[mt] = sa[mt * 64];
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const intx8 w = kW8 ? join(chunk_of(lw + nt * 16 * 128, g), chunk_of(lw + nt * 16 * 128, 4 + g)) : join(w4_chunk(nt), intx4{0, 0, 0, 0});
        const int ws = sw[nt * 64];
#ifdef __HIP_DEVICE_COMPILE__
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
          acc[nt][mt] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, a[mt], acc[nt][mt], kW8 ? 0 : 4, 0, 0, ws, 0, as[mt]);
#endif
      }
    } else {
      float as[kCodes ? MT : 1];
      if (kCodes)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) as[mt] = byte_scale(sa[mt * 64]);
      float ws[NT];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) ws[nt] = byte_scale(sw[nt * 64]);
#pragma unroll
      for (int h = 0; h < 2; ++h) {                          // elements 32 g + 16 h .. + 15: two instructions
        bf16x8 a[MT][2][kPlanes];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          if constexpr (kCodes) {
            const intx4 c = chunk_of(la + mt * 16 * 128, 2 * g + h);
            a[mt][0][0] = decode_e4m3(c[0], c[1], as[mt]);
            a[mt][1][0] = decode_e4m3(c[2], c[3], as[mt]);
          } else {
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
              for (int q = 0; q < kPlanes; ++q)
                a[mt][j][q] = __builtin_bit_cast(bf16x8, chunk_of(la + mt * 16 * 128 + (g >> 1) * (BM * 128) + q * (BM * 256), (g & 1) * 4 + 2 * h + j));
          }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          bf16x8 w[2];
          if (kW8) {
            const intx4 c = chunk_of(lw + nt * 16 * 128, 2 * g + h);
            w[0] = decode_e4m3(c[0], c[1], ws[nt]);
            w[1] = decode_e4m3(c[2], c[3], ws[nt]);
          } else {
            const intx4 c = w4_chunk(nt);
            w[0] = decode_e2m1(c[2 * h], ws[nt]);
            w[1] = decode_e2m1(c[2 * h + 1], ws[nt]);
          }
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
              for (int q = kPlanes - 1; q >= 0; --q)
                acc[nt][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[j], a[mt][j][q], acc[nt][mt], 0, 0, 0);
        }
      }
    }
  };
  for (int kt = 0; kt < nk; ++kt) {
    if (kt + kStages - 2 < nk) wait_vmcnt<(kStages - 2) * kLoads>(); else wait_vmcnt<0>();    // my loads of stage kt have landed
    __builtin_amdgcn_s_waitcnt(0xc07f);                      // lgkmcnt(0): my reads of stage kt - 1 and my rows of stage kt are done
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    if (!kCodes && kt + 1 < nk) fetch(kt + 1);
    if (kt + kStages - 1 < nk) issue(kt + kStages - 1);
    compute(kt);
    if (!kCodes && kt + 1 < nk) stash(kt + 1);
  }

  // ---- results: lane has columns 4 g .. 4 g + 3 of row r of each 16 x 16 tile ----
  if constexpr (kSwiglu) {
    const int Np = (N + kMxStage - 1) / kMxStage * kMxStage, c0 = n0 + wn * 32;
    if (c0 >= Np) return;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const int m = m0 + wm * WTM + mt * 16 + r;
      store_act(acc[0][mt], acc[NT / 4][mt], acc[NT / 2][mt], acc[NT / 2 + NT / 4][mt], m < M, m, c0, g, p, Np);
    }
  } else {
    using T = std::conditional_t<OUT == kOutF32, float, bf16_t>;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const int m = m0 + wm * WTM + mt * 16 + r;
      if (m >= M) continue;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) store_row4<T>(acc[nt][mt], m, n0 + wn * WTN + nt * 16 + 4 * g, p);
    }
  }
}

template <int ROWS, int WF, int OUT, int BM, int BN, int WM, int WN, int kStages>
pvf_status run_tile(hipStream_t s, const MxGemm &p) {
  constexpr int kLds = (codes_in(ROWS) ? kStages : 2) * a_stage_bytes<ROWS>(BM) + kStages * (BN * (WF == PVF_MX_E4M3 ? 128 : 64) + (codes_in(ROWS) ? BM * 4 : 0) + BN * 4);
  static_assert(kLds <= 160 * 1024, "LDS");
  TileMap tm;
  const int64_t tiles_n = OUT == kOutSwiglu ? (mx_width(p.N) + BN / 2 - 1) / (BN / 2) : (p.N + BN - 1) / BN, tiles_m = (p.M + BM - 1) / BM;
  PVF_REQUIRE(nullptr, tiles_m * tiles_n < 1 << 28, PVF_ESHAPE, "%d x %d results are too many for a launch", p.M, p.N);
  tm.tiles_m = (int)tiles_m; tm.tiles_n = (int)tiles_n; tm.group_m = (int)std::min<int64_t>(tiles_m, 8);
  const int chunk = (int)((tiles_m * tiles_n + 7) / 8);
  auto kernel = gemm_mx_tile_kernel<ROWS, WF, OUT, BM, BN, WM, WN, kStages>;
  static const hipError_t allowed = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
  PVF_HIP_CHECK(nullptr, allowed);
  kernel<<<chunk * 8, 64 * WM * WN, kLds, s>>>(p, tm);
  PVF_LAUNCH_CHECK(nullptr, "gemm_mx");
  return PVF_OK;
}

template <int ROWS, int WF, int OUT> pvf_status run(hipStream_t s, const MxGemm &p) {
  if (p.M <= 64) return run_rows<ROWS, WF, OUT>(s, p);
  if constexpr (ROWS == kRowsMx) {
    if ((int64_t)p.M * p.N >= 256 * 256 * 192) return run_tile<ROWS, WF, OUT, 256, 256, 2, 4, 2>(s, p);
  }
  if constexpr (codes_in(ROWS)) {
    if ((int64_t)p.M * p.N * (OUT == kOutSwiglu ? 2 : 1) >= 128 * 128 * 192) return run_tile<ROWS, WF, OUT, 128, 128, 2, 2, 3>(s, p);
    return run_tile<ROWS, WF, OUT, 64, 64, 4, 1, 4>(s, p);
  } else {
    return run_tile<ROWS, WF, OUT, 64, 64, 2, 2, 3>(s, p);
  }
}

template <int WF> pvf_status run_mx(hipStream_t s, const MxGemm &p) {
  if (p.c_scales) return run<kRowsMxExact, WF, kOutSwiglu>(s, p);
  if (p.dtype == PVF_F32) return run<kRowsMxExact, WF, kOutF32>(s, p);
  return run<kRowsMx, WF, kOutBf16>(s, p);
}

}  // namespace

pvf_status launch_gemm_mx(hipStream_t s, const MxGemm &p) {
  if (p.M == 0 || p.N == 0) return PVF_OK;
  if (!p.a_scales)
    return p.dtype == PVF_F32 ? run<kRowsF32, PVF_MX_E2M1, kOutF32>(s, p) : run<kRowsBf16, PVF_MX_E2M1, kOutBf16>(s, p);
  return p.w_fmt == PVF_MX_E4M3 ? run_mx<PVF_MX_E4M3>(s, p) : run_mx<PVF_MX_E2M1>(s, p);
}

}  // namespace pvf
