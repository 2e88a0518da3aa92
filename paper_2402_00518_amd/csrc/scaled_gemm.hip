// Products of 8-bit block-scaled matrices,
//
//   C[i][j] = sum_b sa[i][b] sb[j][b] sum_{k in block b} A[i][k] B[j][k],
//
// blocks of 128 values of K.  A block's dot products come from the matrix cores,
// are scaled and added in fp32.  Which instruction forms them goes by C's type:
//
//   bf16: v_mfma_f32_16x16x128_f8f6f4, one a block, 3.7 PFLOP/s from registers with
//     the scaling.  It adds eight neighbouring products at a time with a common
//     exponent, each cut to a multiple of 2^-13 of the power of two under the largest
//     (measured), so a sum is off by up to 7/8192 of each eight's largest product:
//     1.5e-5 of the result for random operands, a hundredth of C's own rounding.
//   fp32: that would be all of the error, so the codes are widened to bf16, which
//     holds both 8-bit types exactly, and v_mfma_f32_16x16x32_bf16 adds the (exact)
//     products in fp32, at the bf16 rate.
//
// B's rows (the weight's features) are the MFMA's rows, A's (tokens) its columns:
// a lane holds four consecutive features of one token, so C leaves in 16-byte
// stores, and a weight's 128 x 128 blocks give one scale a wave and block.
#include <hip/hip_runtime.h>

#include "ee_device.h"
#include "gemm.h"
#include "launch.h"
#include "ring.h"

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"

namespace ee {

namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef int i32x4_t __attribute__((ext_vector_type(4)));

// 4 bytes a lane from base + off to LDS, lane l's at lds + 4 l (see load_lds16).
__device__ __forceinline__ void load_lds4(const char *base, uint32_t off, uint32_t lds) {
  const uint64_t b = reinterpret_cast<uint64_t>(base);
  base = reinterpret_cast<const char *>(
      static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(b)))) |
      static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(b >> 32)))) << 32);
  lds = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(lds)));
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(off), "s"(base)
               : "memory", "m0");
}

// E5: the columns' codes are e5m2.
template <bool E5>
__device__ __forceinline__ f32x4_t mfma8(const i32x8_t &a, const i32x8_t &b) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, f32x4_t{0.0f, 0.0f, 0.0f, 0.0f}, 0, E5 ? 1 : 0, 0, 0, 0, 0);
}

// Eight codes as bf16.
template <bool E5>
__device__ __forceinline__ bf16x8_t widen(int lo, int hi) {
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  bf16x2_t p[4];
  if constexpr (E5) {
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(lo, 1.0f, false);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(lo, 1.0f, true);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(hi, 1.0f, false);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(hi, 1.0f, true);
  } else {
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
  }
  return __builtin_bit_cast(bf16x8_t, p);
}
template <bool E5>
__device__ __forceinline__ void widen32(const i32x8_t &v, bf16x8_t (&w)[4]) {
  w[0] = widen<E5>(v[0], v[1]);
  w[1] = widen<E5>(v[2], v[3]);
  w[2] = widen<E5>(v[4], v[5]);
  w[3] = widen<E5>(v[6], v[7]);
}
__device__ __forceinline__ f32x4_t mfma_wide(const bf16x8_t (&a)[4], const bf16x8_t (&b)[4]) {
  f32x4_t d = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  static_for<4>([&](auto q) EE_ALWAYS_INLINE {
    d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[decltype(q)::value], b[decltype(q)::value], d, 0, 0, 0);
  });
  return d;
}

// One operand of a stage of 128 values of K: ROWS rows of 128 bytes in LDS, 16-byte
// chunk c of row r at c ^ ((r / 2) mod 8).  A lane's 32 bytes of a row are chunks g
// and 4 + g (g = lane / 16); which values of K those are does not matter, as both
// operands take the same.
template <int ROWS, int THREADS>
struct Operand8 {
  static constexpr int LOADS = ROWS * 8 / THREADS;
  static constexpr int BYTES = ROWS * 128;
  static_assert(LOADS * THREADS == ROWS * 8, "every thread loads the same number of chunks");
  uint32_t off[LOADS];
  int ch[LOADS];
  const char *rd[2];
  const char *base;

  __device__ __forceinline__ void init(const ScaledMat &m, int row0, int tid, int wrow, int lane, const char *lds) {
    base = reinterpret_cast<const char *>(m.data) + static_cast<int64_t>(row0) * m.ld;
    const uint32_t ld = static_cast<uint32_t>(m.ld);
    static_for<LOADS>([&](auto e) EE_ALWAYS_INLINE {
      const int c = decltype(e)::value * THREADS + tid, lr = c >> 3;
      ch[e] = (c & 7) ^ ((lr >> 1) & 7);
      off[e] = static_cast<uint32_t>(min(row0 + lr, m.rows - 1) - row0) * ld + ch[e] * 16;
    });
    const int r = lane & 15, x = (r >> 1) & 7;
    static_for<2>([&](auto h) EE_ALWAYS_INLINE {
      rd[h] = lds + (wrow + r) * 128 + (((decltype(h)::value * 4 + (lane >> 4)) ^ x) << 4);
    });
  }
  // Stage t, of which `left` bytes a row (a multiple of 16) are in the matrix: a
  // chunk past them re-reads the row's first one, and zero_tail clears it.
  __device__ __forceinline__ void load(int t, int left, uint32_t lds_wave) const {
    const char *p = base + static_cast<int64_t>(t) * 128;
    static_for<LOADS>([&](auto e) EE_ALWAYS_INLINE {
      load_lds16(p, ch[e] * 16 < left ? off[e] : off[e] - ch[e] * 16, lds_wave + decltype(e)::value * THREADS * 16);
    });
  }
  __device__ __forceinline__ void zero_tail(int left, int tid, char *lds) const {
    static_for<LOADS>([&](auto e) EE_ALWAYS_INLINE {
      if (ch[e] * 16 >= left)
        *reinterpret_cast<u32x4_t *>(lds + (decltype(e)::value * THREADS + tid) * 16) = u32x4_t{0, 0, 0, 0};
    });
  }
  template <int NBLK>
  __device__ __forceinline__ void read(int stage, i32x8_t (&f)[NBLK]) const {
    static_for<NBLK>([&](auto i) EE_ALWAYS_INLINE {
      const i32x4_t lo = *reinterpret_cast<const i32x4_t *>(rd[0] + stage + decltype(i)::value * 2048);
      const i32x4_t hi = *reinterpret_cast<const i32x4_t *>(rd[1] + stage + decltype(i)::value * 2048);
      f[i] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    });
  }
};

struct StoreC {
  void *c;
  int64_t ld;
  int rows, features;
  bool accumulate, vec, vec8;  // vec, vec8: groups of four (eight) features are aligned
};

__device__ __forceinline__ u32x2_t pack4(f32x4_t v) {
  return u32x2_t{static_cast<uint32_t>(f32_to_bf16(v[0])) | (static_cast<uint32_t>(f32_to_bf16(v[1])) << 16),
                 static_cast<uint32_t>(f32_to_bf16(v[2])) | (static_cast<uint32_t>(f32_to_bf16(v[3])) << 16)};
}

// Four consecutive features of one row of C.
template <bool F32>
__device__ __forceinline__ void store_c(const StoreC &s, int row, int f, f32x4_t v) {
  if (row >= s.rows || f >= s.features) return;
  const int64_t o = static_cast<int64_t>(row) * s.ld + f;
  if constexpr (F32) {
    float *p = static_cast<float *>(s.c) + o;
    if (s.vec && f + 4 <= s.features) {
      if (s.accumulate) v += *reinterpret_cast<const f32x4_t *>(p);
      *reinterpret_cast<f32x4_t *>(p) = v;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (f + e < s.features) p[e] = s.accumulate ? p[e] + v[e] : v[e];
    }
  } else {
    bf16_t *p = static_cast<bf16_t *>(s.c) + o;
    if (s.vec && f + 4 <= s.features) {
      *reinterpret_cast<u32x2_t *>(p) = pack4(v);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (f + e < s.features) p[e] = f32_to_bf16(v[e]);
    }
  }
}

// Eight consecutive features of one row of a bf16 C.
__device__ __forceinline__ void store_row8(const StoreC &s, int row, int f, u32x4_t v) {
  if (row >= s.rows || f >= s.features) return;
  bf16_t *p = static_cast<bf16_t *>(s.c) + static_cast<int64_t>(row) * s.ld + f;
  if (s.vec8 && f + 8 <= s.features) {
    *reinterpret_cast<u32x4_t *>(p) = v;
  } else {
    static_for<8>([&](auto e) EE_ALWAYS_INLINE {
      constexpr int E = decltype(e)::value;
      if (f + E < s.features) p[E] = static_cast<bf16_t>(v[E / 2] >> (16 * (E % 2)));
    });
  }
}

// The 32 bytes of a row that a lane holds as two fragments of 16.
__device__ __forceinline__ i32x8_t fragment(const bf16x8_t (&f)[2]) { return __builtin_bit_cast(i32x8_t, f); }

// Ring of NS stages, the stage NS - 1 further on loaded while one is consumed, one
// barrier a stage (as Ring of ring.h).  W: the rows operand, Z: the columns.  ROW1: W's
// scales are one for each row, else one for each 128 (a wave's rows lie in one block).
// E5: Z's codes are e5m2.  WIDE: C is fp32.
template <int BM, int BN, int WM, int WN, int NS, bool ROW1, bool E5, bool WIDE>
__global__ __launch_bounds__(BM / WM * (BN / WN) * 64) void ring8_kernel(ScaledMat W, ScaledMat Z, int K, StoreC out) {
  constexpr int WAVES_N = BN / WN, THREADS = BM / WM * WAVES_N * 64;
  using TW = Operand8<BM, THREADS>;
  using TZ = Operand8<BN, THREADS>;
  constexpr int SL = (BM + BN + THREADS - 1) / THREADS;  // scale loads a thread and stage
  constexpr int S_OFF = TW::BYTES + TZ::BYTES, STAGE = S_OFF + SL * THREADS * 4;
  constexpr int LOADS = TW::LOADS + TZ::LOADS + SL;
  static_assert((NS - 2) * LOADS <= 63, "loads in flight past the waited-for stage");
  __shared__ __attribute__((aligned(128))) char smem[NS * STAGE];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int tiles_m = cdiv(W.rows, BM), tiles_n = cdiv(Z.rows, BN);
  int tile_m, tile_n;
  tile_of_block(blockIdx.x, gridDim.x, tiles_m, tiles_n, tile_m, tile_n);
  const int m0 = tile_m * BM, n0 = tile_n * BN;
  const int wm = (wave / WAVES_N) * WM, wn = (wave % WAVES_N) * WN;
  const int nk = cdiv(K, 128), bytes = (K + 15) & ~15;
  TW tw;
  TZ tz;
  tw.init(W, m0, tid, wm, lane, smem);
  tz.init(Z, n0, tid, wn, lane, smem + TW::BYTES);
  // scale e of this thread: of W's row, or, past BM, of Z's (past those, the last again)
  const char *sbase[SL];
  uint32_t soff[SL];
  int64_t sstep[SL];
  static_for<SL>([&](auto e) EE_ALWAYS_INLINE {
    const int i = decltype(e)::value * THREADS + wave * 64;  // a wave's 64 scales come from one side
    const bool w = i < BM;
    const ScaledMat &m = w ? W : Z;
    const int row = min((w ? m0 + i : n0 + i - BM) + lane, m.rows - 1);
    sbase[e] = reinterpret_cast<const char *>(m.scale);
    soff[e] = static_cast<uint32_t>(row >> m.shift) * 4;
    sstep[e] = m.scale_ld * 4;
  });
  static_assert(BM % 64 == 0, "a wave's scales come from one side");
  const uint32_t lds0 =
      static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char *)smem));
  auto load = [&](int t, int buf) EE_ALWAYS_INLINE {
    const uint32_t l = lds0 + buf * STAGE + wave * 1024;
    tw.load(t, bytes - t * 128, l);
    tz.load(t, bytes - t * 128, l + TW::BYTES);
    static_for<SL>([&](auto e) EE_ALWAYS_INLINE {
      load_lds4(sbase[e] + t * sstep[e], soff[e], lds0 + buf * STAGE + S_OFF + (decltype(e)::value * THREADS + wave * 64) * 4);
    });
  };
  f32x4_t acc[WM / 16][WN / 16];
  static_for<WM / 16>([&](auto i) EE_ALWAYS_INLINE {
    static_for<WN / 16>([&](auto j) EE_ALWAYS_INLINE { acc[i][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f}; });
  });
  static_for<NS - 1>([&](auto t) EE_ALWAYS_INLINE {
    if (decltype(t)::value < nk) load(decltype(t)::value, decltype(t)::value);
  });
  int cur = 0;
  for (int t = 0; t < nk; ++t) {
    const int later = min(nk - 1 - t, NS - 2);
    static_for<NS - 1>([&](auto l) EE_ALWAYS_INLINE {
      if (later == decltype(l)::value) wait_vm<decltype(l)::value * LOADS>();
    });
    const int left = bytes - t * 128;
    if (left < 128) {  // the last stage: each thread clears the chunks past K that it loaded itself
      tw.zero_tail(left, tid, smem + cur * STAGE);
      tz.zero_tail(left, tid, smem + cur * STAGE + TW::BYTES);
      wait_lgkm();
    }
    phase_barrier();
    if (t + NS - 1 < nk) load(t + NS - 1, cur == 0 ? NS - 1 : cur - 1);  // over stage t - 1, which every wave has read
    const int stage = cur * STAGE;
    const float *sc = reinterpret_cast<const float *>(smem + stage + S_OFF);
    i32x8_t fw[WM / 16], fz[WN / 16];
    float zs[WN / 16];
    tz.template read<WN / 16>(stage, fz);
    tw.template read<WM / 16>(stage, fw);
    static_for<WN / 16>([&](auto j) EE_ALWAYS_INLINE { zs[j] = sc[BM + wn + decltype(j)::value * 16 + (lane & 15)]; });
    if constexpr (!ROW1) {
      const float ws = sc[wm];
      static_for<WN / 16>([&](auto j) EE_ALWAYS_INLINE { zs[j] *= ws; });
    }
    bf16x8_t wz[WIDE ? WN / 16 : 1][4];
    if constexpr (WIDE) static_for<WN / 16>([&](auto j) EE_ALWAYS_INLINE { widen32<E5>(fz[j], wz[j]); });
    static_for<WM / 16>([&](auto i) EE_ALWAYS_INLINE {
      bf16x8_t ww[4];
      if constexpr (WIDE) widen32<false>(fw[i], ww);
      f32x4_t ws = f32x4_t{1.0f, 1.0f, 1.0f, 1.0f};
      if constexpr (ROW1) ws = *reinterpret_cast<const f32x4_t *>(sc + wm + decltype(i)::value * 16 + (lane >> 4) * 4);
      static_for<WN / 16>([&](auto j) EE_ALWAYS_INLINE {
        f32x4_t d;
        if constexpr (WIDE)
          d = mfma_wide(ww, wz[j]);
        else
          d = mfma8<E5>(fw[i], fz[j]);
        if constexpr (ROW1)
          acc[i][j] += d * (ws * zs[j]);
        else
          acc[i][j] += d * zs[j];
      });
    });
    wait_lgkm();
    cur = cur == NS - 1 ? 0 : cur + 1;
  }
  static_for<WM / 16>([&](auto i) EE_ALWAYS_INLINE {
    static_for<WN / 16>([&](auto j) EE_ALWAYS_INLINE {
      store_c<WIDE>(out, n0 + wn + decltype(j)::value * 16 + (lane & 15), m0 + wm + decltype(i)::value * 16 + (lane >> 4) * 4,
              acc[i][j]);
    });
  });
}

// bf16 C, weights with 128 x 128 blocks: 256 x 256 tiles on 8 waves of 128 features x 64
// tokens, the phases of GemmBlockBig (gemm.h) with stages of 128 codes in place of 64 bf16
// values.  A wave's 128 features are one block of the weight's scales, its lanes' tokens
// have one scale each, so a stage needs four scale products a lane.  The scales of a stage
// (256 features', 256 tokens') take one more load a thread, into one of four places in LDS.
constexpr int kBigStages = 131072, kBigScales = 2048;

template <bool E5>
__global__ __launch_bounds__(512, 1) void big8_kernel(ScaledMat W, ScaledMat Z, int K, StoreC out) {
  __shared__ __attribute__((aligned(128))) char smem[kBigStages + 4 * kBigScales];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wave_m = wave >> 2, wave_n = wave & 3;
  int tile_m, tile_n;
  tile_of_block(blockIdx.x, gridDim.x, cdiv(W.rows, 256), cdiv(Z.rows, 256), tile_m, tile_n);
  const int m0 = tile_m * 256, n0 = tile_n * 256;
  const int bytes = (K + 15) & ~15, nk = bytes / 128;  // whole stages
  constexpr int B_OFF = 32768;
  TileOperandB16<true, 128, false, false> ta;
  TileOperandB16<true, 64, false, false> tb;
  ta.init(Operand{W.data, W.ld / 2}, m0, W.rows, 0, tid, wave_m, lane, smem);
  tb.init(Operand{Z.data, Z.ld / 2}, n0, Z.rows, 0, tid, wave_n, lane, smem + B_OFF);
  const uint32_t lds0 =
      static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char *)smem));
  const uint32_t lds_wave = lds0 + wave * 1024;
  const ScaledMat &side = wave < 4 ? W : Z;  // whose scales this wave loads
  const char *sbase = reinterpret_cast<const char *>(side.scale);
  const uint32_t soff =
      static_cast<uint32_t>(min((wave < 4 ? m0 + tid : n0 + tid - 256), side.rows - 1) >> side.shift) * 4;
  const int64_t sstep = side.scale_ld * 4;
  auto load_s = [&](int t, int u) EE_ALWAYS_INLINE {  // stage u's, to stage t's place
    load_lds4(sbase + u * sstep, soff, lds0 + kBigStages + (t & 3) * kBigScales + wave * 256);
  };
  auto load_a = [&](auto q, auto buf, int t) EE_ALWAYS_INLINE {
    ta.template load<decltype(q)::value>(min(t, nk - 1), 64, lds_wave + decltype(buf)::value * 65536);
  };
  auto load_b = [&](auto q, auto buf, int t) EE_ALWAYS_INLINE {
    tb.template load<decltype(q)::value>(min(t, nk - 1), 64, lds_wave + decltype(buf)::value * 65536 + B_OFF);
  };
  f32x4_t acc[8][4];
  static_for<8>([&](auto i) EE_ALWAYS_INLINE {
    static_for<4>([&](auto j) EE_ALWAYS_INLINE { acc[i][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f}; });
  });
  bf16x8_t fa[4][2], fb[2][2][2];
  float zs[4];
  auto read_s = [&](int t) EE_ALWAYS_INLINE {
    const float *sc = reinterpret_cast<const float *>(smem + kBigStages + (t & 3) * kBigScales);
    const float ws = sc[wave_m * 128];
    static_for<4>([&](auto j) EE_ALWAYS_INLINE {
      zs[j] = ws * sc[256 + wave_n * 64 + decltype(j)::value * 16 + (lane & 15)];
    });
  };
  // One quadrant: eight products, each added two products later, so that the scaled adds
  // run under the matrix instructions.
  auto mma = [&](auto qa, auto qb) EE_ALWAYS_INLINE {
    f32x4_t d[8];
    static_for<10>([&](auto n) EE_ALWAYS_INLINE {
      constexpr int N = decltype(n)::value;
      if constexpr (N < 8) d[N] = mfma8<E5>(fragment(fa[N / 2]), fragment(fb[qb][N % 2]));
      if constexpr (N >= 2) {
        constexpr int P = N - 2, I = decltype(qa)::value * 4 + P / 2, J = decltype(qb)::value * 2 + P % 2;
        acc[I][J] += d[P] * zs[J];
      }
    });
  };
  using H0 = std::integral_constant<int, 0>;
  using H1 = std::integral_constant<int, 1>;
  load_s(0, 0);
  load_b(H0{}, H0{}, 0);
  load_a(H0{}, H0{}, 0);
  load_b(H1{}, H0{}, 0);
  load_a(H1{}, H0{}, 0);
  load_s(1, min(1, nk - 1));
  load_b(H1{}, H1{}, 1);
  load_a(H0{}, H1{}, 1);
  load_b(H0{}, H1{}, 1);
  load_a(H1{}, H1{}, 1);
  wait_vm<13>();  // stage 0's scales and first halves
  phase_barrier();
  tb.template read<0, 0>(fb[0]);
  wait_lgkm();
  phase_barrier();
  if (wave_m == 1) phase_barrier();  // waves 4..7 run one barrier behind
  // As GemmBlockBig's stage; the loads past which a wait lets none through are the last six
  // halves' and the scales' among them.
  auto stage = [&](auto buf, int t) EE_ALWAYS_INLINE {
    constexpr int BUF = decltype(buf)::value;
    using Cur = std::integral_constant<int, BUF>;
    using First = Cur;
    using Second = std::integral_constant<int, BUF ^ 1>;
    read_s(t);
    ta.template read<BUF, 0>(fa);
    load_b(First{}, Cur{}, t + 2);
    load_s(t + 2, min(t + 2, nk - 1));
    wait_vm<14>();
    wait_lgkm();
    phase_barrier();
    mma(H0{}, First{});
    phase_barrier();
    tb.template read<BUF, BUF ^ 1>(fb[BUF ^ 1]);
    load_a(H0{}, Cur{}, t + 2);
    wait_vm<14>();
    wait_lgkm();
    phase_barrier();
    mma(H0{}, Second{});
    phase_barrier();
    ta.template read<BUF, 1>(fa);
    load_b(Second{}, Cur{}, t + 2);
    wait_vm<13>();
    wait_lgkm();
    phase_barrier();
    mma(H1{}, Second{});
    phase_barrier();
    tb.template read<BUF ^ 1, BUF ^ 1>(fb[BUF ^ 1]);
    load_a(H1{}, Cur{}, t + 2);
    wait_vm<13>();
    wait_lgkm();
    phase_barrier();
    mma(H1{}, First{});
    phase_barrier();
  };
  int t = 0;
  for (; t + 1 < nk; t += 2) {
    stage(H0{}, t);
    stage(H1{}, t + 1);
  }
  if (t < nk) stage(H0{}, t);
  if (wave_m == 0) phase_barrier();
  wait_vm<0>();
  phase_barrier();
  const int left = bytes - nk * 128;
  if (left > 0) {  // codes past the last whole stage: a stage of its own, zero from there on
    const int ch = (tid & 7) ^ ((tid >> 4) & 7);
    const bool past = ch * 16 >= left;
    auto tail = [&](auto &op, int at) EE_ALWAYS_INLINE {
      static_for<2>([&](auto h) EE_ALWAYS_INLINE {
        static_for<2>([&](auto e) EE_ALWAYS_INLINE {
          constexpr int H = decltype(h)::value, E = decltype(e)::value;
          load_lds16(op.base + static_cast<int64_t>(nk) * 128, past ? op.off[H][E] - ch * 16 : op.off[H][E],
                     lds_wave + at + H * 16384 + E * 8192);
        });
      });
    };
    tail(ta, 0);
    tail(tb, B_OFF);
    load_s(0, nk);
    wait_vm<0>();
    if (past) {
      static_for<8>([&](auto e) EE_ALWAYS_INLINE {
        *reinterpret_cast<u32x4_t *>(smem + decltype(e)::value * 8192 + tid * 16) = u32x4_t{0, 0, 0, 0};
      });
    }
    wait_lgkm();
    phase_barrier();
    read_s(0);
    tb.template read<0, 0>(fb[0]);
    tb.template read<0, 1>(fb[1]);
    static_for<2>([&](auto qa) EE_ALWAYS_INLINE {
      ta.template read<0, decltype(qa)::value>(fa);
      mma(qa, H0{});
      mma(qa, H1{});
    });
    wait_lgkm();
    phase_barrier();
  }
  // C through LDS, a wave's 64 rows of 128 features (256 bytes) in 16 KB of its own: 16-byte
  // chunk c of row r at c ^ (r mod 16), so that it leaves in whole lines.
  char *mine = smem + wave * 16384;
  static_for<8>([&](auto i) EE_ALWAYS_INLINE {
    static_for<4>([&](auto j) EE_ALWAYS_INLINE {
      constexpr int I = decltype(i)::value, J = decltype(j)::value;
      const f32x4_t v = acc[I][J];
      const int r = J * 16 + (lane & 15), g = lane >> 4;
      *reinterpret_cast<u32x2_t *>(mine + r * 256 + (((2 * I + (g >> 1)) ^ (r & 15)) << 4) + (g & 1) * 8) = pack4(v);
    });
  });
  wait_lgkm();
  const int row0 = n0 + wave_n * 64, f0 = m0 + wave_m * 128;
  static_for<16>([&](auto it) EE_ALWAYS_INLINE {
    const int r = decltype(it)::value * 4 + (lane >> 4), c = lane & 15, f = f0 + c * 8;
    const u32x4_t v = *reinterpret_cast<const u32x4_t *>(mine + r * 256 + ((c ^ (r & 15)) << 4));
    store_row8(out, row0 + r, f, v);
  });
}

template <int BM, int BN, int WM, int WN, int NS>
hipError_t launch_ring8(const ScaledMat &W, const ScaledMat &Z, bool f32, const StoreC &out, hipStream_t stream) {
  const int64_t blocks = static_cast<int64_t>(cdiv(W.rows, BM)) * cdiv(Z.rows, BN);
  const dim3 grid(static_cast<unsigned>(blocks)), block(BM / WM * (BN / WN) * 64);
  auto go = [&](auto row1, auto e5, auto wide) {
    hipLaunchKernelGGL((ring8_kernel<BM, BN, WM, WN, NS, decltype(row1)::value, decltype(e5)::value, decltype(wide)::value>),
                       grid, block, 0, stream, W, Z, W.cols, out);
  };
  auto by = [&](auto row1, auto e5) {
    if (f32)
      go(row1, e5, std::true_type{});
    else
      go(row1, e5, std::false_type{});
  };
  if (W.shift == 0 && Z.e5m2)
    by(std::true_type{}, std::true_type{});
  else if (W.shift == 0)
    by(std::true_type{}, std::false_type{});
  else if (Z.e5m2)
    by(std::false_type{}, std::true_type{});
  else
    by(std::false_type{}, std::false_type{});
  return hipGetLastError();
}

}  // namespace

hipError_t scaled_matmul(const ScaledMat &a, const ScaledMat &b, void *c, bool c_f32, int64_t ldc, int accumulate,
                         hipStream_t stream) {
  if (a.rows <= 0 || b.rows <= 0) return hipSuccess;
  if (((a.cols + 15) & ~15) != ((b.cols + 15) & ~15) || b.e5m2) return hipErrorInvalidValue;
  const StoreC out{c, ldc, a.rows, b.rows, accumulate != 0, ldc % 4 == 0, ldc % 8 == 0};
  if (!c_f32 && b.shift != 0 && b.cols >= 256 && static_cast<int64_t>(cdiv(a.rows, 256)) * cdiv(b.rows, 256) > 128) {
    const dim3 grid(static_cast<unsigned>(cdiv(a.rows, 256)) * cdiv(b.rows, 256));
    if (a.e5m2)
      hipLaunchKernelGGL((big8_kernel<true>), grid, dim3(512), 0, stream, b, a, b.cols, out);
    else
      hipLaunchKernelGGL((big8_kernel<false>), grid, dim3(512), 0, stream, b, a, b.cols, out);
    return hipGetLastError();
  }
  if (a.rows <= 32) return launch_ring8<128, 32, 64, 32, 4>(b, a, c_f32, out, stream);
  if (a.rows <= 64) return launch_ring8<128, 64, 64, 32, 3>(b, a, c_f32, out, stream);
  return launch_ring8<128, 128, 64, 64, 2>(b, a, c_f32, out, stream);
}

}  // namespace ee

#pragma clang diagnostic pop
