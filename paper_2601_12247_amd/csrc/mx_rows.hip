// Rows to block-scaled codes (mx.h): the quantiser and the RMSNorm of the residual stream with codes as its output.
// Both are bound by HBM: one pass over the data.
#include "mx.h"

#include <algorithm>

namespace pvf {
namespace {

// A wave takes 512 neighbouring elements of a row, 8 a lane, and kRows rows below each other, so that the scale dwords of a
// workgroup's 4 kRows rows are one run for each 128 elements.  2443 x 1411 float32: 5.6 us, 3.1 TB/s; 320 x 4096 bfloat16: 3.8 us, of which an empty
// launch is 3; 24576 x 4096 float32 to e4m3 91 us, 5.6 TB/s, to e2m1 83 us, 5.5.
template <typename T, int FMT, int kRows>
__global__ void __launch_bounds__(256)
quant_mx_kernel(const T *__restrict__ x, uint8_t *__restrict__ codes, uint32_t *__restrict__ scales, int M, int K, int Kp) {
  const int strips = (Kp + 511) / 512, lane = threadIdx.x & 63, block = mx_block(), k = block % strips * 512 + lane * 8;
  const int m0 = (block / strips * 4 + (threadIdx.x >> 6)) * kRows;
  float v[kRows][8];
#pragma unroll
  for (int r = 0; r < kRows; ++r) load8(x + (int64_t)min(m0 + r, M - 1) * K + min(k, K), K - k, v[r]);
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    const int m = m0 + r;
    quantise8<FMT>(v[r], m < M && k < Kp, codes + ((int64_t)m * Kp + k) / (FMT == PVF_MX_E4M3 ? 1 : 2), scales + (int64_t)(k >> 7) * M + m);
  }
}

// h = x + residual, rounded to T; y = (h * inv) * gain in float32 with inv = float32(1 / sqrt(mean(h^2) + eps)), the sum in float64
// (products of two float32 are exact there, so inv does not depend on the order of the sum and equal rows have equal codes whatever
// the route).  One workgroup a row, the row in registers; rows that do not fit are read twice.  The float64 sum costs nothing beside the memory: 11520 x
// 4096 bfloat16 with a residual 63.5 us, 5.2 TB/s (a large copy 4.7; here 57 % are reads); one row 3.6 us, of which an empty launch is 3.
template <typename T, int kVec>
__global__ void __launch_bounds__(256)
add_rmsnorm_mx_kernel(const T *x, const T *residual, const T *__restrict__ gain, T *sum, uint8_t *__restrict__ codes,
                      uint32_t *__restrict__ scales, int M, int d, int dp, float eps) {
  constexpr bool kTwice = kVec == 0;
  constexpr int kHeld = kTwice ? 1 : kVec;
  __shared__ double part[4];
  __shared__ float row_inv;
  const int tid = threadIdx.x;
  const int64_t m = mx_block();
  if (m >= M) return;
  const T *xr = x + m * d, *rr = residual ? residual + m * d : nullptr;
  float h[kHeld][8];
  double ss = 0;
  auto add = [&](int k, float *v) {
    load8(xr + min(k, d), d - k, v);
    if (rr) {
      float r[8];
      load8(rr + min(k, d), d - k, r);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = to_float(from_float<T>(v[e] + r[e]));
    }
  };
  auto square = [&](const float *v) {
#pragma unroll
    for (int e = 0; e < 8; ++e) ss += (double)v[e] * (double)v[e];
  };
  if (kTwice) {
    for (int k = tid * 8; k < d; k += 2048) { add(k, h[0]); square(h[0]); }
  } else {
#pragma unroll
    for (int i = 0; i < kHeld; ++i) add((i * 256 + tid) * 8, h[i]);
#pragma unroll
    for (int i = 0; i < kHeld; ++i) square(h[i]);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) ss += __shfl_xor(ss, o, kWave);
  if ((tid & 63) == 0) part[tid >> 6] = ss;
  __syncthreads();
  if (tid == 0) row_inv = (float)(1.0 / sqrt(((part[0] + part[1]) + (part[2] + part[3])) / d + (double)eps));
  __syncthreads();
  const float inv = row_inv;
  auto out = [&](int k, float *v) {
    const int left = d - k;
    if (sum && left > 0) store8(sum + m * d + k, left, v);
    float g[8];
    load8(gain + min(k, d), left, g);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < left ? (v[e] * inv) * g[e] : 0.f;
    quantise8<PVF_MX_E4M3>(v, k < dp, codes + m * dp + k, scales + (int64_t)(k >> 7) * M + m);
  };
  if (kTwice) {
    for (int k = tid * 8; k - (tid & 15) * 8 < dp; k += 2048) { add(k, h[0]); out(k, h[0]); }
  } else {
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
      if ((i * 256 + (tid & ~63)) * 8 < dp) out((i * 256 + tid) * 8, h[i]);
  }
}

}  // namespace

pvf_status launch_quant_mx(hipStream_t s, int dtype, const void *x, int fmt, void *codes, void *scales, int M, int K) {
  if (M == 0) return PVF_OK;
  const int Kp = (int)mx_width(K);
  auto run = [&](auto t, auto f) -> pvf_status {
    using T = decltype(t);
    constexpr int F = decltype(f)::value;
    constexpr int kRows = 4;
    const int64_t grid = (int64_t)((Kp + 511) / 512) * ((M + 4 * kRows - 1) / (4 * kRows));
    PVF_REQUIRE(nullptr, grid < 1 << 28, PVF_ESHAPE, "quant_mx: %d x %d elements are too many for a launch", M, K);
    quant_mx_kernel<T, F, kRows><<<mx_grid(grid), 256, 0, s>>>((const T *)x, (uint8_t *)codes, (uint32_t *)scales, M, K, Kp);
    PVF_LAUNCH_CHECK(nullptr, "quant_mx");
    return PVF_OK;
  };
  using E4 = std::integral_constant<int, PVF_MX_E4M3>;
  using E2 = std::integral_constant<int, PVF_MX_E2M1>;
  if (dtype == PVF_BF16) return fmt == PVF_MX_E4M3 ? run(bf16_t{}, E4{}) : run(bf16_t{}, E2{});
  return fmt == PVF_MX_E4M3 ? run(float{}, E4{}) : run(float{}, E2{});
}

pvf_status launch_add_rmsnorm_mx(hipStream_t s, int dtype, const void *x, const void *residual, const void *gain, void *sum,
                                 void *codes, void *scales, int M, int d, float eps) {
  if (M == 0) return PVF_OK;
  const int dp = (int)mx_width(d);
  auto run = [&](auto t) {
    using T = decltype(t);
    auto go = [&](auto v) {
      add_rmsnorm_mx_kernel<T, decltype(v)::value><<<mx_grid(M), 256, 0, s>>>((const T *)x, (const T *)residual, (const T *)gain, (T *)sum,
                                                                     (uint8_t *)codes, (uint32_t *)scales, M, d, dp, eps);
    };
    if (dp <= 2048) go(std::integral_constant<int, 1>{});
    else if (dp <= 4096) go(std::integral_constant<int, 2>{});
    else if (dp <= 8192) go(std::integral_constant<int, 4>{});
    else go(std::integral_constant<int, 0>{});
  };
  if (dtype == PVF_BF16) run(bf16_t{}); else run(float{});
  PVF_LAUNCH_CHECK(nullptr, "add_rmsnorm_mx");
  return PVF_OK;
}

}  // namespace pvf
