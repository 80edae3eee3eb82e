// Block-scaled rows: 32 consecutive elements of a row share a power of two, 2^(b - 127), b a byte; the elements are e4m3 (a byte,
// at most 448) or e2m1 (4 bits, the even element in the low half of a byte; 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives).  These
// are the formats that v_mfma_scale_f32_16x16x128_f8f6f4 multiplies.  Rows have mx_width(K) elements, zeros behind K; the scale
// bytes of 128 elements are one dword and the dwords of neighbouring rows lie side by side, scales[k / 128][row][k / 32 % 4], so
// that the scales of a tile's rows for one stage of k are one run of memory.
#pragma once

#include "common.h"

namespace pvf {

constexpr int kMxBlock = 32, kMxStage = 128;
inline int64_t mx_width(int64_t K) { return (K + kMxStage - 1) / kMxStage * kMxStage; }

pvf_status launch_quant_mx(hipStream_t s, int dtype, const void *x, int fmt, void *codes, void *scales, int M, int K);
pvf_status launch_add_rmsnorm_mx(hipStream_t s, int dtype, const void *x, const void *residual, const void *gain, void *sum,
                                 void *codes, void *scales, int M, int d, float eps);

// A product of rows with block-scaled weights W [N, mx_width(K)].
struct MxGemm {
  const void *A = nullptr;          // e4m3 codes [M, mx_width(K)], or rows [M, K] of `dtype` (a_scales == NULL)
  const uint8_t *a_scales = nullptr;
  const void *W = nullptr;
  const uint8_t *w_scales = nullptr;
  void *C = nullptr;                // [M, N] of `dtype`; SwiGLU: e4m3 codes [M, mx_width(N)]
  uint8_t *c_scales = nullptr;      // SwiGLU (W is [2 N, mx_width(K)], gate | up): scales of the codes in C
  const void *residual = nullptr;
  int M = 0, N = 0, K = 0, w_fmt = 0, dtype = 0;
};
pvf_status launch_gemm_mx(hipStream_t s, const MxGemm &g);

// The kernel instance that a product's launch takes: `index` of the `count` that products of this kind choose from.
struct MxInstance {
  pvf_status (*run)(hipStream_t, const MxGemm &);
  int index, count;
};
MxInstance gemm_mx_instance(const MxGemm &g);

#ifdef __HIPCC__
// A launch takes fewer than 2^32 threads along x: workgroups from the 2^22th on go on in y.
constexpr int kMxGridBits = 22;
inline dim3 mx_grid(int64_t n) {
  const int64_t x = n < 1 << kMxGridBits ? n : 1 << kMxGridBits;
  return dim3((uint32_t)x, (uint32_t)((n + x - 1) / x), 1);
}
__device__ __forceinline__ int mx_block() { return (int)(blockIdx.x + (blockIdx.y << kMxGridBits)); }

// Byte of a block's scale from the bits of its largest magnitude: the smallest power of two, from 2^-127 on, with amax <= top * 2^e
// (top = 448 = 1.75 2^8 or 6 = 1.5 2^2: the carry out of the mantissa decides), so that no element saturates.  NaN and infinities: 255.
template <int FMT> __device__ __forceinline__ int mx_scale_byte(uint32_t amax_bits) {
  constexpr uint32_t kTopMantissa = FMT == PVF_MX_E4M3 ? 0x600000u : 0x400000u;
  constexpr int kTopExp = FMT == PVF_MX_E4M3 ? 8 : 2;
  const int b = max((int)((amax_bits + (0x7fffffu - kTopMantissa)) >> 23) - kTopExp, 0);
  return amax_bits >= 0x7f800000u ? 255 : b;
}
// 2^(127 - b), what an element of the block is multiplied by (exact: a product that underflows is a zero code anyway); a block that
// holds a NaN or an infinity is NaN by its scale and its codes are zeros.
__device__ __forceinline__ float mx_inverse(int b) { return b == 255 ? 0.f : __uint_as_float((uint32_t)(254 - b) << 23); }
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// Four float32 values, already divided by their scale, to e4m3 codes (nearest, ties to even).
__device__ __forceinline__ uint32_t pack_e4m3x4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
  return (uint32_t)w;
}
// Eight values to e2m1 codes.
__device__ __forceinline__ uint32_t pack_e2m1x8(const float *v) {
  uint32_t w = 0;
#ifdef __HIP_DEVICE_COMPILE__
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], 1.f, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], 1.f, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], 1.f, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], 1.f, 3);
#endif
  return w;
}

// Eight consecutive elements from p on, those behind the first `left` as zeros.  Rows may begin anywhere: gfx950 loads 16 bytes from
// any element's address.
__device__ __forceinline__ void load8(const float *p, int left, float *v) {
  if (left >= 8) {
    typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
    const f4 a = *reinterpret_cast<const f4 *>(p), b = *reinterpret_cast<const f4 *>(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < left ? p[e] : 0.f;
  }
}
typedef uint32_t mx_u4 __attribute__((ext_vector_type(4), aligned(2)));
__device__ __forceinline__ uint4 load8_raw(const bf16_t *p, int left) {
  if (left >= 8) {
    const mx_u4 a = *reinterpret_cast<const mx_u4 *>(p);
    return make_uint4(a[0], a[1], a[2], a[3]);
  }
  uint32_t h[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) h[e] = e < left ? reinterpret_cast<const uint16_t *>(p)[e] : 0u;
  return make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
}
__device__ __forceinline__ uint4 load4_raw(const float *p, int left) {
  if (left >= 4) {
    typedef uint32_t u4 __attribute__((ext_vector_type(4), aligned(4)));
    const u4 a = *reinterpret_cast<const u4 *>(p);
    return make_uint4(a[0], a[1], a[2], a[3]);
  }
  return make_uint4(left > 0 ? __float_as_uint(p[0]) : 0u, left > 1 ? __float_as_uint(p[1]) : 0u, left > 2 ? __float_as_uint(p[2]) : 0u, 0u);
}
__device__ __forceinline__ void load8(const bf16_t *p, int left, float *v) {
  const uint4 a = load8_raw(p, left);
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) { v[2 * e] = __uint_as_float(w[e] << 16); v[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u); }
}
__device__ __forceinline__ void store8(float *p, int left, const float *v) {
  if (left >= 8) {
    typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
    *reinterpret_cast<f4 *>(p) = f4{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f4 *>(p + 4) = f4{v[4], v[5], v[6], v[7]};
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) if (e < left) p[e] = v[e];
  }
}
__device__ __forceinline__ void store8(bf16_t *p, int left, const float *v) {
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const bf16_t a = (bf16_t)v[2 * e], b = (bf16_t)v[2 * e + 1];
    w[e] = (uint32_t)__builtin_bit_cast(uint16_t, a) | ((uint32_t)__builtin_bit_cast(uint16_t, b) << 16);
  }
  if (left >= 8) {
    *reinterpret_cast<mx_u4 *>(p) = mx_u4{w[0], w[1], w[2], w[3]};
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) if (e < left) reinterpret_cast<uint16_t *>(p)[e] = (uint16_t)(w[e >> 1] >> (e & 1) * 16);
  }
}

// Quantises the 8 elements v of each of 16 neighbouring lanes (128 elements of a row): codes to `codes` (this lane's 8 or 4 bytes) and,
// from the first of the 16 lanes, the dword of scales.
template <int FMT>
__device__ __forceinline__ void quantise8(const float *v, bool live, uint8_t *codes, uint32_t *scale_word) {
  uint32_t am = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) am = max(am, abs_bits(v[e]));
  am = max(am, (uint32_t)__shfl_xor((int)am, 1, kWave));
  am = max(am, (uint32_t)__shfl_xor((int)am, 2, kWave));       // the block's four lanes agree
  const int b = mx_scale_byte<FMT>(am);
  const float inv = mx_inverse(b);
  uint32_t word = (uint32_t)b << (threadIdx.x >> 2 & 3) * 8;
  word |= (uint32_t)__shfl_xor((int)word, 4, kWave);
  word |= (uint32_t)__shfl_xor((int)word, 8, kWave);
  if (!live) return;
  float q[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) q[e] = b == 255 ? 0.f : v[e] * inv;
  if (FMT == PVF_MX_E4M3) {
    *reinterpret_cast<uint2 *>(codes) = make_uint2(pack_e4m3x4(q[0], q[1], q[2], q[3]), pack_e4m3x4(q[4], q[5], q[6], q[7]));
  } else {
    *reinterpret_cast<uint32_t *>(codes) = pack_e2m1x8(q);
  }
  if ((threadIdx.x & 15) == 0) *scale_word = word;
}
#endif

}  // namespace pvf
