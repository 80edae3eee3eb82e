// Attention over pages for many rows a request (paged_attention.h): bf16, more (row, head) pairs a key head than 16, or 32 where
// d_head is at most 64.
//
// One workgroup = 128 columns of one (request, key head), 32 a wave, or 64, with the waves in two pairs that take alternate halves of the keys.
// 64 keys and their values at a time go from the pages into LDS (no detour over registers), one buffer ahead; S^T = K Q^T and O^T = V^T P^T on
// 32 x 32 x 16 matrix instructions.  A lane of S^T holds one column and keys 8 (e / 4) + 4 (lane / 32) + e % 4; P^T is multiplied as it is held, with V^T's
// keys in that order: transposing reads give a lane four keys of one dimension.
//
// Bound by what a step takes in turn: 64 keys of 128 columns are 3400 cycles, 1545 of the matrix unit and about 1800 of the vector unit, which overlap in
// part, and with the loads behind them.  bf16, 9 windows of 128 rows over up to 1280 tokens, 32 heads of 128: 60 us for 24 GFLOP (36 with P's second
// part: 0.60 PFLOP/s) and 200 MB (3.4 TB/s), and 9 to join.  Without the products 50 us, without the loads 54.  Eight waves a workgroup took 85 us, two
// workgroups of 64 columns 81.
//
// LDS rows are keys, in 16-byte chunks; chunk x of a key lies at x ^ turn(key), so that equal chunks of 8 keys (the operand K) and pairs of chunks of 4 keys
// (V^T) fall on different banks.
#include "paged_attention.h"

namespace pvf {
namespace page {
namespace {

typedef short short4v __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lptr_t;
typedef __attribute__((address_space(3))) short4v *trptr_t;

// Twice 16 bytes a lane from global memory to LDS, lane after lane from `at` and from 4096 bytes behind it on, counted by vmcnt alone: written out
// because the compiler, which cannot tell the tile on its way from the one that is read, waits for the builtin's loads before the next read of LDS.  There is
// no register that a load writes.  Every wait for them stands below.  The compiler does not count wait states into an asm block: addresses come from
// v_readlane, and a load may read a scalar register five states after a vector instruction wrote it (s_mov, s_nop 3), m0 one after.  m0, which the
// compiler reserves, is set by nothing else here.
__device__ __forceinline__ void load_to_lds(const void *src0, const void *src1, uint32_t lane_bytes, uint32_t at) {
  asm volatile(
      "s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %1, %2\n\t"
      "s_add_u32 m0, m0, 0x1000\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %3" ::"s"(at), "v"(lane_bytes), "s"(src0), "s"(src1) : "memory", "scc");
}
// at most N of this wave's loads are on the way; its LDS reads are done; then every wave's
template <int N>
__device__ __forceinline__ void wait_and_meet() {
  __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | (N >> 4) << 14);   // vmcnt(N) lgkmcnt(0)
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// CW: waves beside each other over columns; the 4 / CW groups of them share out the keys of a step.
template <int DH, int CW>
struct WideInst {
  static constexpr int kDh = DH, QT = 32 * CW, KW = 4 / CW, kStep = 64, kSubs = 2 / KW, kSplit = 8, kWholeSteps = 8, kPerCu = DH <= 128 ? 2 : 1;
  static constexpr bool kAsTheyCome = true;
  static constexpr int NT = DH / 32, KJ = DH / 16;
  static constexpr int kRow = DH * 2, kChunks = DH / 8, kTile = kStep * kRow;   // bytes of a key, its chunks, bytes of 64 keys
  static constexpr int kLoads = kTile / 4096, kKeys = 1024 / kRow;             // loads of 1 KB a wave and tile, keys of one
  static constexpr int kSlotFloats = QT * (DH + 2);
  static_assert(CW * KW == 4 && kSubs * KW == 2 && kLoads % 2 == 0, "four waves, two groups of 32 keys, loads by two");
};

template <int DH, int CW, bool kWhole>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(WideInst<DH, CW>::kPerCu, WideInst<DH, CW>::kPerCu)))
page_attention_wide_kernel(Args a) {
  typedef WideInst<DH, CW> I;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[4 * I::kTile];   // keys, values; twice
  __shared__ int32_t s_pages[kPageSlots];
  const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int cw = wid % CW, kw = wid / CW, fr = lane & 31, fh = lane >> 5;
  __shared__ int32_t s_bad;
  int worker;
  Line<I> line(a, blockIdx.x, gridDim.x, &worker);
  if (!a.whole && worker < a.workers && tid == 0) a.joins[(int64_t)worker * kJoinInts] = 0;
  Request r;
  Piece piece;

  auto turn = [](int key) { return (key & 3) << 1 | (key >> 2 & 1) | (I::kChunks == 16 ? key & 8 : 0); };
  // operand K: key fr of 32, chunk 2 j + fh.  Operand V^T: of 16 lanes, lane 4 k + x reads dimensions 4 x .. of key k; keys 4 fh .. (and 8 behind
  // them), dimensions 32 t + 16 (lane / 16 % 2) + ..
  int k_rd[I::KJ], v_rd[I::NT][2];
#pragma unroll
  for (int j = 0; j < I::KJ; ++j) k_rd[j] = fr * I::kRow + (((2 * j + fh) ^ turn(fr)) << 4);
#pragma unroll
  for (int t = 0; t < I::NT; ++t)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int s = lane & 15, key = 8 * e + 4 * fh + s / 4, dim = 32 * t + 16 * (lane >> 4 & 1) + 4 * (s & 3);
      v_rd[t][e] = key * I::kRow + ((dim / 8 ^ turn(key)) << 4) + dim % 8 * 2;
    }

  // a lane's part of a load: a chunk of one of its kKeys keys (turn() of a key is the same for every load of a wave)
  const int lane_key = wid * I::kKeys + lane / I::kChunks, lane_chunk = lane % I::kChunks ^ turn(lane_key);
  const uint32_t lane_bytes = (uint32_t)((lane / I::kChunks) * a.p.dh + lane_chunk * 8) * 2;

  while (line.next(r, piece)) {
    const int cols = piece.cols, len = r.len, col = 32 * cw + fr;
    const bf16_t *kbase = (const bf16_t *)a.p.k_cache + (int64_t)piece.head * a.p.page_size * a.p.dh;
    const bf16_t *vbase = (const bf16_t *)a.p.v_cache + (int64_t)piece.head * a.p.page_size * a.p.dh;
    int row;
    const int64_t q_at = row_place(a, r.row0, piece.head, piece.tile * I::QT + col, a.p.q_stride, &row);
    const int limit = col < cols ? limit_of(a, r.told, r.n, row) : INT32_MAX;
    const int least = limit_of(a, r.told, r.n, (int)((uint32_t)(piece.tile * I::QT) / (uint32_t)a.group));      // of the tile's columns: the first row's
    bf16x8 q[I::KJ];
#pragma unroll
    for (int j = 0; j < I::KJ; ++j) {
      uint4 x = make_uint4(0, 0, 0, 0);
      if (col < cols && (kWhole || 16 * j + 8 * fh < a.p.dh)) x = *(const uint4 *)((const bf16_t *)a.p.q + q_at + 16 * j + 8 * fh);
      q[j] = __builtin_bit_cast(bf16x8, x);
    }
    if (a.q_xor) {                        // not before it is needed: the rows are on their way
#pragma unroll
      for (int j = 0; j < I::KJ; ++j) {
        const uint4 x = __builtin_bit_cast(uint4, q[j]);
        q[j] = __builtin_bit_cast(bf16x8, make_uint4(x.x ^ a.q_xor, x.y ^ a.q_xor, x.z ^ a.q_xor, x.w ^ a.q_xor));
      }
    }
    floatx16 o[I::NT];
#pragma unroll
    for (int t = 0; t < I::NT; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[t][e] = 0.f;
    float m = -INFINITY, l = 0.f;
    meet();                               // the last piece's results have been read
    if (!kWhole) {                        // chunks behind d_head: nothing is loaded there, and q is zero beside them
      for (int i = tid; i < 4 * I::kTile / 16; i += 256) *(uint4 *)(lds + 16 * i) = make_uint4(0, 0, 0, 0);
    }

    for (int s0 = piece.step0; s0 < piece.step1; s0 += a.chunk_steps) {
      const int s1 = min(piece.step1, s0 + min(a.chunk_steps, piece.step1 - s0));
      const int k0 = s0 * I::kStep, k1 = (int)min((int64_t)len, (int64_t)s1 * I::kStep);
      if (tid == 0) s_bad = 0;
      meet();                             // the last chunk's pages and tiles have been read
      const int first_page = page_of(a, k0);
      load_pages(a, line.b, k0, k1, first_page, s_pages, &s_bad);
      meet();
      const bool bad = __builtin_amdgcn_readfirstlane(s_bad) != 0 || r.over;
      if (k1 <= k0) continue;             // a request without keys

      // 64 keys from kb on, or their values, kKeys neighbouring ones a load: they share a page.  Lane i finds where the wave's i-th load begins, for
      // keys and values at once.  What lies behind the last key comes along.
      const uint32_t lds_at = (uint32_t)(uintptr_t)(lptr_t *)lds + wid * 1024;
      int64_t values_at = 0;
      auto load = [&](int64_t at, uint32_t dst) {
#pragma unroll
        for (int i = 0; i < I::kLoads; i += 2) {
          auto from = [&](int l) {
            const uint32_t lo = __builtin_amdgcn_readlane((int)at, l), hi = __builtin_amdgcn_readlane((int)(at >> 32), l);
            return (const void *)((uint64_t)hi << 32 | lo);
          };
          const void *src0 = from(i), *src1 = from(i + 1);       // by all lanes: one that loads nothing may hold an address
          if (kWhole || lane_chunk * 8 < a.p.dh) load_to_lds(src0, src1, lane_bytes, dst + i * 4096);
        }
      };
      int64_t keys_at = 0;
      auto find = [&](int kb) {
        const int key = min(kb + (lane % I::kLoads * 4 + wid) * I::kKeys, (k1 - 1) & ~(I::kKeys - 1)), page = page_of(a, key);
        const int id = max(s_pages[page - first_page], 0), off = (key - page * a.p.page_size) * a.p.dh;
        keys_at = (int64_t)(kbase + (int64_t)id * a.p.k_page_stride + off);
        values_at = (int64_t)(vbase + (int64_t)id * a.p.v_page_stride + off);
      };
      auto load_keys = [&](int buf) { load(keys_at, lds_at + buf * 2 * I::kTile); };             // found last
      auto load_values = [&](int buf) { load(values_at, lds_at + (buf * 2 + 1) * I::kTile); };

      // Keys and values of a step are asked for two steps ahead, each when its buffer has been read: three tiles are on the way at most, and waits are
      // for the oldest (the last two steps': for all).  The keys of this step are awaited before it begins.
      auto step = [&](int kb, auto buf_c) {
        constexpr int kBuf = decltype(buf_c)::value;
        const unsigned char *ks = lds + kBuf * 2 * I::kTile;
        unsigned char *vs = lds + (kBuf * 2 + 1) * I::kTile;
        const bool more = kb < k1 - 2 * I::kStep;
        floatx16 s[I::kSubs];
#pragma unroll
        for (int u = 0; u < I::kSubs; ++u)
#pragma unroll
          for (int e = 0; e < 16; ++e) s[u][e] = 0.f;
        // operands of one part of a row are read while another is multiplied
        constexpr int kPart = I::KJ / 2 < 4 ? I::KJ / 2 : 4, kParts = I::KJ / kPart;
        bf16x8 kf[2][kPart][I::kSubs];
        auto read_keys = [&](int part) {
#pragma unroll
          for (int j = 0; j < kPart; ++j)
#pragma unroll
            for (int u = 0; u < I::kSubs; ++u) kf[part % 2][j][u] = *(const bf16x8 *)(ks + (u * I::KW + kw) * 32 * I::kRow + k_rd[part * kPart + j]);
          __builtin_amdgcn_sched_barrier(0);
        };
        read_keys(0);
        read_keys(1);
        find(kb + 2 * I::kStep);                               // beside the products
#pragma unroll
        for (int part = 0; part < kParts; ++part) {
#pragma unroll
          for (int j = 0; j < kPart; ++j)
#pragma unroll
            for (int u = 0; u < I::kSubs; ++u) s[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[part % 2][j][u], q[part * kPart + j], s[u], 0, 0, 0);
          if (part + 2 < kParts) read_keys(part + 2);
        }
        if (more) wait_and_meet<2 * I::kLoads>(); else wait_and_meet<0>();     // its values are there, its keys have been read
        if (more) load_keys(kBuf);
        bool odd = false;
        if (__builtin_expect(kb + I::kStep > least, 0)) {
          // The tile holds keys that a row does not see, or copies of the last one.  0 times an infinity is no zero: values that are not finite
          // leave it and are added to the columns that see them, by themselves.
          bool mine = false;
          for (int i = tid; i < I::kTile / 16; i += 256) {
            uint4 x = *(uint4 *)(vs + 16 * i);
            if (bf16s_not_finite(x.x) | bf16s_not_finite(x.y) | bf16s_not_finite(x.z) | bf16s_not_finite(x.w)) {
              mine = true;
              *(uint4 *)(vs + 16 * i) = make_uint4(bf16s_finite(x.x), bf16s_finite(x.y), bf16s_finite(x.z), bf16s_finite(x.w));
            }
          }
          odd = __syncthreads_or(mine) != 0;
        }
        auto key_of = [&](int u, int e) { return kb + 32 * (u * I::KW + kw) + 8 * (e / 4) + 4 * fh + e % 4; };
        if (__builtin_expect(bad, 0)) {                                             // four keys from a multiple of four on share a page
#pragma unroll
          for (int u = 0; u < I::kSubs; ++u)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
              const bool none = (s_pages[page_of(a, min(key_of(u, e), len - 1)) - first_page] < 0) | r.over;
#pragma unroll
              for (int i = 0; i < 4; ++i) s[u][e + i] = none ? NAN : s[u][e + i];
            }
        }
        if (__builtin_expect(kb + I::kStep > least, 0)) {
#pragma unroll
          for (int u = 0; u < I::kSubs; ++u)
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (key_of(u, e) >= min(limit, len)) s[u][e] = -INFINITY;
        }
        float top = s[0][0];
#pragma unroll
        for (int u = 0; u < I::kSubs; ++u)
#pragma unroll
          for (int e = 0; e < 16; ++e) top = fmaxf(top, s[u][e]);
        top = fmaxf(top, __shfl_xor(top, 32, kWave));
        // the maximum in use follows when it is passed by 2^8: sums stay far from overflow and are rarely scaled
        const bool up = (top - m) * a.c > 8.0f;                // the first time m = -inf
        const float now = up ? top : m, ref = reference(now), alpha = up ? weight(a, m, now) : 1.0f, less = -ref * a.c;
        m = now;
        l *= alpha;
        if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
          for (int t = 0; t < I::NT; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[t][e] *= alpha;
        }
        if (__builtin_expect(odd, 0)) {
#pragma unroll 1
          for (int x = 0; x < 64 && kb + x < len; ++x) {
            if (I::KW == 2 && x / 32 != kw) continue;
            const int key = kb + x, page = page_of(a, key), id = max(s_pages[page - first_page], 0);
            const bf16_t *v = vbase + (int64_t)id * a.p.v_page_stride + (key - page * a.p.page_size) * a.p.dh + 4 * fh;
#pragma unroll
            for (int t = 0; t < I::NT; ++t)
#pragma unroll
              for (int e = 0; e < 16; e += 4) {
                const int d = 32 * t + 2 * e;
                uint2 y = make_uint2(0, 0);
                if (key < limit && (kWhole || d + 4 * fh < a.p.dh)) y = *(const uint2 *)(v + d);
                o[t][e] += odd_part(y.x << 16);
                o[t][e + 1] += odd_part(y.x & 0xffff0000u);
                o[t][e + 2] += odd_part(y.y << 16);
                o[t][e + 3] += odd_part(y.y & 0xffff0000u);
              }
          }
        }
        // 16 keys at a time: while their values are multiplied, the next ones' operands are read and their probabilities computed, which takes the vector
        // unit as long as the products take the matrix unit
        constexpr int kBlocks = 2 * I::kSubs;
        bf16x8 vt[2][I::NT];
        auto read_values = [&](int k) {
          const int at = (32 * (k / 2 * I::KW + kw) + 16 * (k % 2)) * I::kRow;
#pragma unroll
          for (int t = 0; t < I::NT; ++t) {
            const short4v v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((trptr_t)(vs + at + v_rd[t][0]));
            const short4v v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((trptr_t)(vs + at + v_rd[t][1]));
            vt[k % 2][t] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
          }
        };
        float p[8];
        auto exponential = [&](int k, int i) { p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[k / 2][8 * (k % 2) + i], a.c, less)); };
        struct Parts { uint32_t w[4]; } hi[2], lo[2];          // P^T's two operands of 16 keys
        auto take = [&](int k, int i) {                        // the i-th of 8
          l += p[i];
          if (i % 2) {
            hi[k % 2].w[i / 2] = upper_parts(p[i - 1], p[i]);
            lo[k % 2].w[i / 2] = lower_parts(p[i - 1], p[i]);
          }
        };
        read_values(0);
#pragma unroll
        for (int i = 0; i < 8; ++i) exponential(0, i);
#pragma unroll
        for (int i = 0; i < 8; ++i) take(0, i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = 0; k < kBlocks; ++k) {
          const bool more_blocks = k + 1 < kBlocks;
          if (more_blocks) read_values(k + 1);
          constexpr int kProducts = 2 * I::NT;
#pragma unroll
          for (int i = 0; i < kProducts; ++i) {
            const int t = i % I::NT;
            o[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vt[k % 2][t], __builtin_bit_cast(bf16x8, i < I::NT ? hi[k % 2] : lo[k % 2]), o[t], 0, 0, 0);
            if (more_blocks) {
#pragma unroll
              for (int x = 8 * i / kProducts; x < 8 * (i + 1) / kProducts; ++x) {   // probabilities beside a product
                exponential(k + 1, x);
                if (x > 0) take(k + 1, x - 1);
              }
              __builtin_amdgcn_sched_barrier(0);
            }
          }
          if (more_blocks) take(k + 1, 7);
        }
      };
      __builtin_amdgcn_s_waitcnt(0x0f70);                      // vmcnt(0): nothing else is counted from here on
      find(k0);
      load_keys(0);
      load_values(0);
      const bool two = k0 < k1 - I::kStep;
      if (two) {
        find(k0 + I::kStep);
        load_keys(1);
        load_values(1);
        wait_and_meet<3 * I::kLoads>();
      } else {
        wait_and_meet<I::kLoads>();
      }
      for (int kb = k0;;) {               // two steps a turn, so that a buffer's place is a constant
        step(kb, std::integral_constant<int, 0>{});
        if (kb >= k1 - I::kStep) break;
        if (kb < k1 - 2 * I::kStep) {
          wait_and_meet<2 * I::kLoads>(); // the next step's keys are there, this one's values have been read
          load_values(0);
        } else {
          wait_and_meet<0>();
        }
        kb += I::kStep;
        step(kb, std::integral_constant<int, 1>{});
        if (kb >= k1 - I::kStep) break;
        if (kb < k1 - 2 * I::kStep) {
          wait_and_meet<2 * I::kLoads>();
          load_values(1);
        } else {
          wait_and_meet<0>();
        }
        kb += I::kStep;
      }
    }

    l += __shfl_xor(l, 32, kWave);
    if (I::KW == 2) {                     // the second pair's results, to the first
      __syncthreads();
      float *x = reinterpret_cast<float *>(lds) + cw * (I::NT * 16 + 2) * 64 + lane;
      if (kw == 1) {
#pragma unroll
        for (int t = 0; t < I::NT; ++t)
#pragma unroll
          for (int e = 0; e < 16; ++e) x[(t * 16 + e) * 64] = o[t][e];
        x[I::NT * 16 * 64] = m;
        x[(I::NT * 16 + 1) * 64] = l;
      }
      __syncthreads();
      if (kw == 0) {
        const float m1 = x[I::NT * 16 * 64], l1 = x[(I::NT * 16 + 1) * 64], top = fmaxf(m, m1), ref = reference(top);
        const float f0 = weight(a, m, ref), f1 = weight(a, m1, ref);
#pragma unroll
        for (int t = 0; t < I::NT; ++t)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[t][e] = f0 * o[t][e] + f1 * x[(t * 16 + e) * 64];
        l = f0 * l + f1 * l1;
        m = top;
      }
    }
    if (col < cols && kw == 0) {
      if (piece.done) {
        int r_;
        const float inv = 1.0f / l;
        bf16_t *dst = (bf16_t *)a.p.out + row_place(a, r.row0, piece.head, piece.tile * I::QT + col, a.p.out_stride, &r_);
#pragma unroll
        for (int t = 0; t < I::NT; ++t)
#pragma unroll
          for (int e = 0; e < 16; e += 4) {
            const int d = 32 * t + 2 * e + 4 * fh;
            if (kWhole || d < a.p.dh) store4(dst + d, floatx4{o[t][e], o[t][e + 1], o[t][e + 2], o[t][e + 3]}, inv, limit <= 0);
          }
      } else {
        float *slot = partial<I>(a, worker, piece.begun);
        if (fh == 0) {
          slot[col] = m;
          slot[I::QT + col] = l;
        }
#pragma unroll
        for (int t = 0; t < I::NT; ++t)
#pragma unroll
          for (int e = 0; e < 16; e += 4) {
            const int d = 32 * t + 2 * e + 4 * fh;
            if (kWhole || d < a.p.dh) *(floatx4 *)(slot + 2 * I::QT + col * DH + d) = floatx4{o[t][e], o[t][e + 1], o[t][e + 2], o[t][e + 3]};
          }
      }
    }
    if (!piece.done && piece.begun && tid == 0) line.note_join(worker, r, piece);
  }
}

// 128 columns where 64 would read every key twice.  64 requests of 2048 keys, 8 key heads, us with 64 and 128 columns: 64 pairs 50.0 and 68.0 (d_head 64),
// 110 and 133 (128); 72 pairs 88.6 and 68.2, 202 and 126; 128 pairs 90.3 and 71.9, 207 and 128.  d_head 256: 64 pairs 214, 128 pairs 277 (one workgroup a CU).
template <class F>
auto with_wide(int64_t pairs, int dh, F f) {
  if (dh <= 64) return pairs <= 64 ? f(WideInst<64, 2>{}) : f(WideInst<64, 4>{});
  if (dh <= 128) return pairs <= 64 ? f(WideInst<128, 2>{}) : f(WideInst<128, 4>{});
  return pairs <= 64 ? f(WideInst<256, 2>{}) : f(WideInst<256, 4>{});
}

template <int DH, int CW>
pvf_status launch(WideInst<DH, CW>, hipStream_t s, Args &a) {
  typedef WideInst<DH, CW> I;
  const Plan p = prepare<I>(a);
  if (a.p.dh == DH) page_attention_wide_kernel<DH, CW, true><<<p.grid, 256, 0, s>>>(a);
  else page_attention_wide_kernel<DH, CW, false><<<p.grid, 256, 0, s>>>(a);
  PVF_LAUNCH_CHECK(nullptr, "page_attention_wide");
  if (!a.whole) {
    page_attention_join_kernel<bf16_t, I><<<dim3(p.workers - 1, I::QT / kJoinCols<I>), kJoinThreads, 0, s>>>(a);
    PVF_LAUNCH_CHECK(nullptr, "page_attention_join");
  }
  return PVF_OK;
}

}  // namespace

pvf_status launch_wide(hipStream_t s, Args &a, int64_t pairs) {
  return with_wide(pairs, a.p.dh, [&](auto inst) { return launch(inst, s, a); });
}
int64_t wide_workspace(int B, int M, int Hkv, int group, int dh, int width, int page_size, int64_t pairs) {
  return with_wide(pairs, dh, [&](auto inst) {
    typedef decltype(inst) I;
    return workspace_bytes<I>(B, M, Hkv, group, width, page_size);
  });
}

}  // namespace page
}  // namespace pvf
