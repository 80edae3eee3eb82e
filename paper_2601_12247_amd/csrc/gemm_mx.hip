// Products with block-scaled operands (mx.h) on the CDNA4 matrix cores: C[M,N] = A[M,K] * W[N,K]^T (+ residual), float32 accumulation.
//
//   rows      weights      result          arithmetic
//   e4m3      e4m3, e2m1   bfloat16, e4m3  v_mfma_scale_f32_16x16x128_f8f6f4: codes and scale bytes as they lie in memory
//   e4m3      e4m3, e2m1   float32         codes decoded to bfloat16, which holds them exactly, and v_mfma_f32_16x16x32_bf16
//   bfloat16  e2m1         bfloat16        weights decoded to bfloat16 (exact)
//   float32   e2m1         float32         rows as three bfloat16 whose sum they are (24 bits), weights decoded
//
// The scaled instruction adds 8 neighbouring products at a time, each cut off 13 bits below the largest of the eight (measured: 16 and 2^-8 1.27 in
// one group lose what lies below 2^-9), then those sums and the accumulator in float32.  On random operands that is 1.5e-5 of the
// result, a hundredth of a bfloat16 rounding, and far below the rounding of the codes themselves; float32 results do not take it (the
// bfloat16 instruction keeps float32 sums).
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
      float v[8];
      uint32_t am = 0;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const floatx4 gate = total(c * MT + mt, lane), up = total((2 + c) * MT + mt, lane);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[4 * c + e] = n0 + c * 16 + 4 * g + e < N ? silu_f(gate[e]) * up[e] : 0.f;
          am = max(am, abs_bits(v[4 * c + e]));
        }
      }
      am = max(am, (uint32_t)__shfl_xor((int)am, 16, kWave));
      am = max(am, (uint32_t)__shfl_xor((int)am, 32, kWave));
      const int b = mx_scale_byte<PVF_MX_E4M3>(am);
      const float inv = mx_inverse(b);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = b == 255 ? 0.f : v[e] * inv;
      if (m < M) {
        uint8_t *row = (uint8_t *)p.C + (int64_t)m * Np + n0 + 4 * g;
        *reinterpret_cast<uint32_t *>(row) = pack_e4m3x4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<uint32_t *>(row + 16) = pack_e4m3x4(v[4], v[5], v[6], v[7]);
        if (g == 0) p.c_scales[((int64_t)(n0 / kMxStage) * M + m) * 4 + n0 / kMxBlock % 4] = (uint8_t)b;
      }
    }
  } else {
    using T = std::conditional_t<OUT == kOutF32, float, bf16_t>;
    for (int t = wave; t < NT * MT; t += KW) {
      const int m = m0 + t % MT * 16 + r, n = n0 + t / MT * 16 + 4 * g;
      const floatx4 s = total(t, lane);
      if (m >= M) continue;
      T *row = (T *)p.C + (int64_t)m * N;
      const T *res = p.residual ? (const T *)p.residual + (int64_t)m * N : nullptr;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (n + e < N) row[n + e] = from_float<T>(s[e] + (res ? to_float(res[n + e]) : 0.f));
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

template <int WF> pvf_status run_mx(hipStream_t s, const MxGemm &p) {
  if (p.c_scales) return run_rows<kRowsMx, WF, kOutSwiglu>(s, p);
  if (p.dtype == PVF_F32) return run_rows<kRowsMxExact, WF, kOutF32>(s, p);
  return run_rows<kRowsMx, WF, kOutBf16>(s, p);
}

}  // namespace

pvf_status launch_gemm_mx(hipStream_t s, const MxGemm &p) {
  if (p.M == 0 || p.N == 0) return PVF_OK;
  if (!p.a_scales)
    return p.dtype == PVF_F32 ? run_rows<kRowsF32, PVF_MX_E2M1, kOutF32>(s, p) : run_rows<kRowsBf16, PVF_MX_E2M1, kOutBf16>(s, p);
  return p.w_fmt == PVF_MX_E4M3 ? run_mx<PVF_MX_E4M3>(s, p) : run_mx<PVF_MX_E2M1>(s, p);
}

}  // namespace pvf
