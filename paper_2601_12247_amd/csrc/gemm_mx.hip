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

constexpr bool codes_in(int rows) { return rows == kRowsMx || rows == kRowsMxExact; }

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

// ---- the kernel ---------------------------------------------------------------------------------------------------
typedef __attribute__((address_space(1))) const void gptr_t;
typedef __attribute__((address_space(3))) void lptr_t;

// s_waitcnt vmcnt(n) only; n is a 6-bit field split 4 + 2
template <int N> __device__ __forceinline__ void wait_vmcnt() {
  static_assert(N >= 0 && N < 64, "vmcnt is a 6-bit counter");
  __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | ((N >> 4) << 14));
}

struct TileMap { int tiles_m, tiles_n, group_m; };

// Where 16-byte chunk c of a row lies in LDS rows of R bytes: the reads of an operand (16 rows, one chunk each) touch every bank once.
template <int R> __device__ __forceinline__ int swizzle(int row) { return R >= 256 ? row & 15 : R == 128 ? row >> 1 & 7 : row >> 2 & 3; }

// Sizes of an instance.
template <int ROWS, int WF, int BM, int BN, int WM, int WN, int WK, int kStages, int AR = BM> struct Shape {
  static constexpr int kASize = codes_in(ROWS) ? 1 : ROWS == kRowsBf16 ? 2 : 4;
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
  constexpr int kPlanes = ROWS == kRowsF32 ? 3 : 1;
  static_assert(BM % (16 * WM) == 0 && BN % (16 * WN) == 0 && kAChunks % 64 == 0 && kWChunks % 64 == 0, "tile shape");
  static_assert(kDirect || !kCodes, "codes always go straight");
  static_assert(!kSwiglu || BN / WN == 64, "a wave has a block of gate and the same block of up");
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wk = wave / (WM * WN), wm = wave / WN % WM, wn = wave % WN, r = lane & 15, g = lane >> 4;
  const int M = p.M, N = p.N, K = p.K, Kp = (K + kMxStage - 1) / kMxStage * kMxStage, nk = Kp / kMxStage, ns = (nk + WK - 1) / WK;

  // the 32 workgroups that an XCD runs at a time cover a patch of tiles and share operands through its L2
  const int total = tm.tiles_m * tm.tiles_n, per_xcd = (total + 7) >> 3;
  const int L = (int)(blockIdx.x & 7) * per_xcd + (int)(blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per_xcd || L >= total) return;
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
    a_at[i] = ((f % kACpr) ^ swizzle<S::kARow>(row)) * 16;
    a_src[i] = (const uint8_t *)p.A + (int64_t)min(m0 + row, M - 1) * a_bytes;
  }
#pragma unroll
  for (int i = 0; i < LW; ++i) {
    const int f = (i * kThreads + tid) % kWChunks, row = f / kWCpr;
    w_at[i] = ((f % kWCpr) ^ swizzle<S::kWRow>(row)) * 16;
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

  // ---- operands of a stage in registers ----
  const int am = wm * (BM / WM) + r, an = wn * (BN / WN) + r;               // rows of the lane's operands in the tiles (but for 16 mt, 16 nt)
  const int ar = AR < 16 ? r % AR : am;                      // behind AR rows the first ones again, for columns of the instruction that are not stored
  const int a_swz = swizzle<S::kARow>(ar), w_swz = swizzle<S::kWRow>(r);
  constexpr int kFA = kCodes ? 2 : ROWS == kRowsBf16 ? 4 : 8, kFW = kW8 ? 2 : 1;
  struct Operands { intx4 a[MT][kFA], w[NT][kFW]; int as[kCodes ? MT : 1], ws[NT]; };
  auto read = [&](Operands &o, int st) {
    const unsigned char *slot = lds + st % kStages * S::kStage;
    const unsigned char *la = slot + ar * S::kARow, *lw = slot + S::kABytes + an * S::kWRow;
    const unsigned char *sa = slot + S::kABytes + S::kWBytes + (wk * AR + ar) * 4 + g, *sw = slot + S::kABytes + S::kWBytes + S::kAUnits * 256 + (wk * BN + an) * 4 + g;
    // chunks of the lane: scaled instruction g and 4 + g; else kFA from kFA g on
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
      for (int c = 0; c < kFA; ++c)
        o.a[mt][c] = *reinterpret_cast<const intx4 *>(la + mt * 16 * S::kARow + (((wk * (kACpr / WK) + (ROWS == kRowsMx ? 4 * c + g : kFA * g + c)) ^ a_swz) << 4));
      if (kCodes) o.as[kCodes ? mt : 0] = sa[mt * 64];
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int c = 0; c < kFW; ++c)
        o.w[nt][c] = *reinterpret_cast<const intx4 *>(lw + nt * 16 * S::kWRow + (((wk * (kWCpr / WK) + (ROWS == kRowsMx ? 4 * c + g : kFW * g + c)) ^ w_swz) << 4));
      o.ws[nt] = sw[nt * 64];
    }
  };
  auto multiply = [&](const Operands &o, int st) {
    if constexpr (ROWS == kRowsMx) {
#ifdef __HIP_DEVICE_COMPILE__
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
          acc[nt][mt] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kW8 ? join(o.w[nt][0], o.w[nt][kFW - 1]) : join(o.w[nt][0], intx4{0, 0, 0, 0}),
                                                                         join(o.a[mt][0], o.a[mt][1]), acc[nt][mt], kW8 ? 0 : 4, 0, 0, o.ws[nt], 0, o.as[kCodes ? mt : 0]);
#endif
    } else {
      // four instructions of 32 k: lane g has elements 32 g + 8 j .. + 7 of its 128 in the j-th, all of one block
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        bf16x8 w[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
          w[nt] = kW8 ? decode_e4m3(o.w[nt][(j >> 1) % kFW][j * 2 & 3], o.w[nt][(j >> 1) % kFW][(j * 2 & 3) + 1], byte_scale(o.ws[nt]))
                      : decode_e2m1(o.w[nt][0][j], byte_scale(o.ws[nt]));
        const int k = (st * WK + wk) * 128 + 32 * g + 8 * j;                 // rows of bf16 / float32: what lies behind K is another chunk's
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          bf16x8 a[3];
          if constexpr (kCodes) {
            const float as = byte_scale(o.as[kCodes ? mt : 0]);
            a[0] = decode_e4m3(o.a[mt][j >> 1][j * 2 & 3], o.a[mt][j >> 1][(j * 2 & 3) + 1], as);
          } else if constexpr (ROWS == kRowsBf16) {
            a[0] = __builtin_bit_cast(bf16x8, k >= K ? intx4{0, 0, 0, 0} : o.a[mt][j]);
          } else {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = k + (e & 4) >= K ? 0.f : __int_as_float(o.a[mt][(2 * j + e / 4) % kFA][e % 4]);
            split3(v, a);
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int q = kPlanes - 1; q >= 0; --q) acc[nt][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[nt], a[q], acc[nt][mt], 0, 0, 0);
        }
      }
    }
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
      Operands o;
      read(o, st);
      multiply(o, st);
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

template <int ROWS, int WF, int OUT, int BM, int BN, int WM, int WN, int WK, int kStages, int AR = BM, bool kDirect = true>
pvf_status run_as(hipStream_t s, const MxGemm &p) {
  using S = Shape<ROWS, WF, BM, BN, WM, WN, WK, kStages, AR>;
  static_assert(S::kLds <= 160 * 1024, "LDS");
  TileMap tm;
  const int64_t tiles_n = OUT == kOutSwiglu ? (mx_width(p.N) + BN / 2 - 1) / (BN / 2) : (p.N + BN - 1) / BN, tiles_m = (p.M + BM - 1) / BM;
  PVF_REQUIRE(nullptr, tiles_m * tiles_n < 1 << 28, PVF_ESHAPE, "%d x %d results are too many for a launch", p.M, p.N);
  tm.tiles_m = (int)tiles_m; tm.tiles_n = (int)tiles_n; tm.group_m = (int)std::min<int64_t>(tiles_m, 8);
  auto kernel = gemm_mx_kernel<ROWS, WF, OUT, BM, BN, WM, WN, WK, kStages, AR, kDirect>;
  // once per kernel instance; a function-local static is initialised exactly once even with concurrent callers
  static const hipError_t allowed = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, S::kLds);
  PVF_HIP_CHECK(nullptr, allowed);
  kernel<<<(uint32_t)((tiles_m * tiles_n + 7) / 8 * 8), S::kThreads, S::kLds, s>>>(p, tm);
  PVF_LAUNCH_CHECK(nullptr, "gemm_mx");
  return PVF_OK;
}

// ---- which instance -------------------------------------------------------------------------------------------------
// What a tile costs for 128 k, in microseconds, measured at K = 4096 (launch time less 3 us, over 32 and the tiles of the fullest CU):
// where a CU has one tile, and per tile where it has several (those that fit its LDS run at a time and hide each other's barriers and
// latencies).  The launch takes the instance whose fullest CU is done first.  What bounds small tiles is a CU's loads on the way: some 60
// bytes a nanosecond, so a tile's rows count, not its area.
struct Candidate {
  int BM, BN, most_rows;                                     // most_rows: rows of A that the instance loads (0: any number)
  float alone, among;
  pvf_status (*run)(hipStream_t, const MxGemm &);
};

template <int ROWS, int WF, int OUT, bool kDirect> struct Candidates;
#define PVF_MX_TILE(BM, BN, WM, WN, WK, ST, AR, alone, among) \
  {BM, OUT == kOutSwiglu ? BN / 2 : BN, AR < BM ? AR : 0, alone, among, run_as<ROWS, WF, OUT, BM, BN, WM, WN, WK, ST, AR, kDirect>}

template <int WF, bool kDirect> struct Candidates<kRowsMx, WF, kOutBf16, kDirect> {
  static constexpr int ROWS = kRowsMx, OUT = kOutBf16;
  static constexpr Candidate list[] = {
      PVF_MX_TILE(16, 16, 1, 1, 4, 3, 16, .08f, .075f),   PVF_MX_TILE(32, 32, 1, 1, 4, 3, 32, .1375f, .153f), PVF_MX_TILE(64, 64, 2, 2, 2, 3, 64, .275f, .28f),
      PVF_MX_TILE(64, 64, 2, 2, 2, 2, 64, .38f, .217f),   PVF_MX_TILE(80, 64, 1, 2, 4, 2, 80, .29f, .33f),   PVF_MX_TILE(96, 64, 2, 2, 1, 3, 96, .39f, .28f),
      PVF_MX_TILE(64, 128, 2, 4, 1, 3, 64, .415f, .375f), PVF_MX_TILE(128, 128, 2, 2, 1, 2, 128, .78f, .51f), PVF_MX_TILE(160, 128, 2, 4, 1, 2, 160, .83f, .72f),
      PVF_MX_TILE(192, 256, 2, 4, 1, 2, 192, 1.49f, 1.44f), PVF_MX_TILE(256, 256, 2, 4, 1, 2, 256, 1.8f, 1.84f)};
};
template <int WF, bool kDirect> struct Candidates<kRowsMxExact, WF, kOutF32, kDirect> {
  static constexpr int ROWS = kRowsMxExact, OUT = kOutF32;
  static constexpr Candidate list[] = {
      PVF_MX_TILE(16, 16, 1, 1, 4, 3, 16, .10f, .10f),   PVF_MX_TILE(32, 32, 1, 1, 4, 3, 32, .19f, .20f),    PVF_MX_TILE(64, 64, 2, 2, 2, 2, 64, .42f, .36f),
      PVF_MX_TILE(64, 128, 2, 4, 1, 3, 64, .74f, .61f),  PVF_MX_TILE(128, 128, 2, 2, 1, 2, 128, 1.2f, .91f), PVF_MX_TILE(160, 128, 2, 4, 1, 2, 160, 1.43f, 1.22f)};
};
template <int WF, bool kDirect> struct Candidates<kRowsMxExact, WF, kOutSwiglu, kDirect> {
  static constexpr int ROWS = kRowsMxExact, OUT = kOutSwiglu;
  static constexpr Candidate list[] = {
      PVF_MX_TILE(16, 64, 1, 1, 4, 2, 16, .18f, .14f),   PVF_MX_TILE(32, 64, 1, 1, 4, 2, 32, .25f, .20f),    PVF_MX_TILE(64, 128, 2, 2, 2, 2, 64, .53f, .65f),
      PVF_MX_TILE(64, 128, 2, 2, 1, 2, 64, .67f, .55f),  PVF_MX_TILE(128, 128, 2, 2, 1, 2, 128, 1.2f, .90f)};
};
template <bool kDirect> struct Candidates<kRowsBf16, PVF_MX_E2M1, kOutBf16, kDirect> {
  static constexpr int ROWS = kRowsBf16, WF = PVF_MX_E2M1, OUT = kOutBf16;
  static constexpr Candidate list[] = {
      PVF_MX_TILE(16, 16, 1, 1, 8, 2, 1, .04f, .047f),   PVF_MX_TILE(16, 16, 1, 1, 8, 2, 4, .06f, .05f),     PVF_MX_TILE(16, 16, 1, 1, 4, 2, 16, .095f, .058f),
      PVF_MX_TILE(32, 32, 2, 1, 4, 2, 32, .19f, .20f),   PVF_MX_TILE(32, 64, 2, 1, 2, 2, 32, .35f, .215f),   PVF_MX_TILE(64, 64, 2, 2, 2, 2, 64, .41f, .42f),
      PVF_MX_TILE(64, 128, 2, 2, 1, 2, 64, .75f, .58f)};
};
template <bool kDirect> struct Candidates<kRowsF32, PVF_MX_E2M1, kOutF32, kDirect> {
  static constexpr int ROWS = kRowsF32, WF = PVF_MX_E2M1, OUT = kOutF32;
  static constexpr Candidate list[] = {
      PVF_MX_TILE(16, 16, 1, 1, 8, 2, 1, .07f, .10f),    PVF_MX_TILE(16, 16, 1, 1, 8, 2, 16, .27f, .30f),    PVF_MX_TILE(16, 32, 1, 1, 4, 2, 16, .35f, .37f),
      PVF_MX_TILE(32, 32, 2, 1, 4, 2, 32, .59f, .70f),   PVF_MX_TILE(32, 64, 2, 1, 2, 2, 32, .82f, .84f),    PVF_MX_TILE(64, 128, 4, 1, 1, 2, 64, 2.1f, 2.1f)};
};

template <int ROWS, int WF, int OUT, bool kDirect = true> pvf_status run(hipStream_t s, const MxGemm &p) {
  const int64_t columns = OUT == kOutSwiglu ? mx_width(p.N) : p.N;
  const Candidate *best = nullptr;
  float least = 0.f;
  for (const Candidate &c : Candidates<ROWS, WF, OUT, kDirect>::list) {
    if (c.most_rows && p.M > c.most_rows) continue;
    const int64_t tiles = ((p.M + c.BM - 1) / c.BM) * ((columns + c.BN - 1) / c.BN), fullest = (tiles + 255) / 256;
    const float cost = fullest == 1 ? c.alone : c.among * (float)fullest;
    if (!best || cost < least) { best = &c; least = cost; }
  }
  return best->run(s, p);
}

template <int WF> pvf_status run_mx(hipStream_t s, const MxGemm &p) {
  if (p.c_scales) return run<kRowsMxExact, WF, kOutSwiglu>(s, p);
  if (p.dtype == PVF_F32) return run<kRowsMxExact, WF, kOutF32>(s, p);
  return run<kRowsMx, WF, kOutBf16>(s, p);
}

}  // namespace

pvf_status launch_gemm_mx(hipStream_t s, const MxGemm &p) {
  if (p.M == 0 || p.N == 0) return PVF_OK;
  if (!p.a_scales) {                                         // rows that begin at 16-byte chunks go straight to LDS
    const bool f32 = p.dtype == PVF_F32, direct = (uintptr_t)p.A % 16 == 0 && p.K % (f32 ? 4 : 8) == 0;
    if (f32) return direct ? run<kRowsF32, PVF_MX_E2M1, kOutF32>(s, p) : run<kRowsF32, PVF_MX_E2M1, kOutF32, false>(s, p);
    return direct ? run<kRowsBf16, PVF_MX_E2M1, kOutBf16>(s, p) : run<kRowsBf16, PVF_MX_E2M1, kOutBf16, false>(s, p);
  }
  return p.w_fmt == PVF_MX_E4M3 ? run_mx<PVF_MX_E4M3>(s, p) : run_mx<PVF_MX_E2M1>(s, p);
}

}  // namespace pvf
