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

#include <cmath>

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

// 4 bytes a lane from the lane's address to LDS, lane l's at lds + 4 l (see load_lds16).
__device__ __forceinline__ void load_lds4(const float *p, uint32_t lds) {
  lds = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(lds)));
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(p) : "memory", "m0");
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

// One operand of a stage of KW blocks of 128 values of K: for each block ROWS rows of 128 bytes
// in LDS, 16-byte chunk c of row r at c ^ ((r / 2) mod 8).  A lane's 32 bytes of a row are
// chunks g and 4 + g (g = lane / 16); which values of K those are does not matter, as both
// operands take the same.
template <int ROWS, int THREADS, int KW>
struct Operand8 {
  static constexpr int LOADS = KW * ROWS * 8 / THREADS;
  static constexpr int BYTES = KW * ROWS * 128;
  static_assert(LOADS * THREADS == KW * ROWS * 8, "every thread loads the same number of chunks");
  uint32_t off[LOADS];
  int at[LOADS];  // bytes of the chunk from the stage's first
  const char *rd[2];
  const char *base;

  // kw: the block of the stage that the wave takes
  __device__ __forceinline__ void init(const ScaledMat &m, int row0, int tid, int wrow, int kw, int lane, const char *lds) {
    base = reinterpret_cast<const char *>(m.data) + static_cast<int64_t>(row0) * m.ld;
    const uint32_t ld = static_cast<uint32_t>(m.ld);
    static_for<LOADS>([&](auto e) EE_ALWAYS_INLINE {
      const int c = decltype(e)::value * THREADS + tid, lr = (c >> 3) % ROWS;
      at[e] = (c / (ROWS * 8)) * 128 + ((c & 7) ^ ((lr >> 1) & 7)) * 16;
      off[e] = static_cast<uint32_t>(min(row0 + lr, m.rows - 1) - row0) * ld;
    });
    const int r = lane & 15, x = (r >> 1) & 7;
    static_for<2>([&](auto h) EE_ALWAYS_INLINE {
      rd[h] = lds + (kw * ROWS + wrow + r) * 128 + (((decltype(h)::value * 4 + (lane >> 4)) ^ x) << 4);
    });
  }
  // Stage t, of which `left` bytes a row (a multiple of 16) are in the matrix: a
  // chunk past them re-reads the row's first one, and zero_tail clears it.
  __device__ __forceinline__ void load(int t, int left, uint32_t lds_wave) const {
    const char *p = base + static_cast<int64_t>(t) * (128 * KW);
    static_for<LOADS>([&](auto e) EE_ALWAYS_INLINE {
      load_lds16(p, off[e] + (at[e] < left ? at[e] : 0), lds_wave + decltype(e)::value * THREADS * 16);
    });
  }
  __device__ __forceinline__ void zero_tail(int left, int tid, char *lds) const {
    static_for<LOADS>([&](auto e) EE_ALWAYS_INLINE {
      if (at[e] >= left)
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
  bool accumulate;
};

__device__ __forceinline__ u32x2_t pack4(f32x4_t v) {
  return u32x2_t{static_cast<uint32_t>(f32_to_bf16(v[0])) | (static_cast<uint32_t>(f32_to_bf16(v[1])) << 16),
                 static_cast<uint32_t>(f32_to_bf16(v[2])) | (static_cast<uint32_t>(f32_to_bf16(v[3])) << 16)};
}

// Four consecutive features of one row of C (whose rows need not be aligned).
template <bool F32>
__device__ __forceinline__ void store_c(const StoreC &s, int row, int f, f32x4_t v) {
  if (row >= s.rows || f >= s.features) return;
  const int64_t o = static_cast<int64_t>(row) * s.ld + f;
  if constexpr (F32) {
    float *p = static_cast<float *>(s.c) + o;
    if (f + 4 <= s.features) {
      if (s.accumulate) v += load_any<f32x4_t>(p);
      store_any(p, v);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (f + e < s.features) p[e] = s.accumulate ? p[e] + v[e] : v[e];
    }
  } else {
    bf16_t *p = static_cast<bf16_t *>(s.c) + o;
    if (f + 4 <= s.features) {
      store_any(p, pack4(v));
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
  if (f + 8 <= s.features) {
    store_any(p, v);
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
// barrier a stage (as Ring of ring.h).  W: the rows operand, Z: the columns.  KW waves share a
// wave's WM x WN outputs: a stage is KW blocks of K, one for each, and their sums meet in LDS.
// ROW1: W's scales are one for each row, else one for each 128 (a wave's rows lie in one
// block).  E5: Z's codes are e5m2.  WIDE: C is fp32.
//
// What bounds it, by K and tokens: the weights' trip from memory and the chain of load, barrier
// and sum (5120 x 13824, 48 tokens: 28 us, 2.6 TB/s, 160 blocks), or, for an fp32 C of
// thousands of tokens, the power that matrix and vector units draw together: 13824 x 5120, K
// 4016, scales by rows: 605 to 650 us, 0.9 PFLOP/s, with the matrix units busy 37% and the
// vector units 51% of the cycles (two instructions a product to widen, two to scale and add).
// Products and vector work interleaved by hand with the next stage's first reads under the
// last products took 656 us on the machine where this took 643, products of 32 x 32 outputs
// 685, a third stage 657.
template <int BM, int BN, int WM, int WN, int KW, int NS, bool ROW1, bool E5, bool WIDE>
__global__ __launch_bounds__(BM / WM * (BN / WN) * KW * 64) void ring8_kernel(ScaledMat W, ScaledMat Z, int K, StoreC out) {
  constexpr int WAVES_N = BN / WN, WAVES = BM / WM * WAVES_N, THREADS = WAVES * KW * 64;
  using TW = Operand8<BM, THREADS, KW>;
  using TZ = Operand8<BN, THREADS, KW>;
  constexpr int SROWS = KW * (BM + BN);  // scales of a stage: W's rows and Z's, block by block
  constexpr int SL = (SROWS + THREADS - 1) / THREADS;
  constexpr int S_OFF = TW::BYTES + TZ::BYTES, STAGE = S_OFF + SL * THREADS * 4;
  constexpr int LOADS = TW::LOADS + TZ::LOADS + SL;
  constexpr int RED = KW > 1 ? KW * BM * BN * 4 : 0;
  static_assert((NS - 2) * LOADS <= 63, "loads in flight past the waited-for stage");
  __shared__ __attribute__((aligned(128))) char smem[NS * STAGE > RED ? NS * STAGE : RED];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kw = wave / WAVES, ww = wave % WAVES;
  int tile_m, tile_n;
  tile_of_block(blockIdx.x, gridDim.x, cdiv(W.rows, BM), cdiv(Z.rows, BN), tile_m, tile_n);
  const int m0 = tile_m * BM, n0 = tile_n * BN;
  const int wm = (ww / WAVES_N) * WM, wn = (ww % WAVES_N) * WN;
  const int blocks = cdiv(K, 128), nk = cdiv(blocks, KW), bytes = (K + 15) & ~15;
  TW tw;
  TZ tz;
  tw.init(W, m0, tid, wm, kw, lane, smem);
  tz.init(Z, n0, tid, wn, kw, lane, smem + TW::BYTES);
  // Scale i of a stage: block i / (BM + BN), of W's row or, past BM, of Z's (past all, the
  // last again).  A block of K past the last repeats its scale: its codes are zeros.
  const float *sptr[SL];
  int sblk[SL];
  int64_t sld[SL];
  static_for<SL>([&](auto e) EE_ALWAYS_INLINE {
    const int i = min(decltype(e)::value * THREADS + tid, SROWS - 1), r = i % (BM + BN);
    const bool w = r < BM;
    const int row = w ? min(m0 + r, W.rows - 1) >> W.shift : min(n0 + r - BM, Z.rows - 1) >> Z.shift;
    sptr[e] = (w ? W.scale : Z.scale) + row;
    sld[e] = w ? W.scale_ld : Z.scale_ld;
    sblk[e] = i / (BM + BN);
  });
  const uint32_t lds0 =
      static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char *)smem));
  auto load = [&](int t, int buf) EE_ALWAYS_INLINE {
    const uint32_t l = lds0 + buf * STAGE + wave * 1024;
    tw.load(t, bytes - t * (128 * KW), l);
    tz.load(t, bytes - t * (128 * KW), l + TW::BYTES);
    static_for<SL>([&](auto e) EE_ALWAYS_INLINE {
      load_lds4(sptr[e] + min(t * KW + sblk[e], blocks - 1) * sld[e],
                lds0 + buf * STAGE + S_OFF + (decltype(e)::value * THREADS + wave * 64) * 4);
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
    const int left = bytes - t * (128 * KW);
    if (left < 128 * KW) {  // the last stage: each thread clears the chunks past K that it loaded itself
      tw.zero_tail(left, tid, smem + cur * STAGE);
      tz.zero_tail(left, tid, smem + cur * STAGE + TW::BYTES);
      wait_lgkm();
    }
    phase_barrier();
    if (t + NS - 1 < nk) load(t + NS - 1, cur == 0 ? NS - 1 : cur - 1);  // over stage t - 1, which every wave has read
    const int stage = cur * STAGE;
    const float *sc = reinterpret_cast<const float *>(smem + stage + S_OFF) + kw * (BM + BN);
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
  auto store = [&](int i, int j, f32x4_t v) EE_ALWAYS_INLINE {  // 16 x 16 block of the tile
    store_c<WIDE>(out, n0 + j * 16 + (lane & 15), m0 + i * 16 + (lane >> 4) * 4, v);
  };
  if constexpr (KW == 1) {
    static_for<WM / 16>([&](auto i) EE_ALWAYS_INLINE {
      static_for<WN / 16>([&](auto j) EE_ALWAYS_INLINE {
        store(wm / 16 + decltype(i)::value, wn / 16 + decltype(j)::value, acc[i][j]);
      });
    });
  } else {
    constexpr int ALL = (BM / 16) * (BN / 16);
    f32x4_t *red = reinterpret_cast<f32x4_t *>(smem);  // [kw][16 x 16 block][lane]
    __syncthreads();
    static_for<WM / 16>([&](auto i) EE_ALWAYS_INLINE {
      static_for<WN / 16>([&](auto j) EE_ALWAYS_INLINE {
        const int b = (wm / 16 + decltype(i)::value) * (BN / 16) + wn / 16 + decltype(j)::value;
        red[(kw * ALL + b) * 64 + lane] = acc[i][j];
      });
    });
    __syncthreads();
    for (int b = wave; b < ALL; b += WAVES * KW) {
      f32x4_t v = red[b * 64 + lane];
      static_for<KW - 1>([&](auto w) EE_ALWAYS_INLINE { v += red[((decltype(w)::value + 1) * ALL + b) * 64 + lane]; });
      store(b / (BN / 16), b % (BN / 16), v);
    }
  }
}

// bf16 C, weights with 128 x 128 blocks: 256 x 256 tiles on 8 waves of 128 features x 64
// tokens, the phases of GemmBlockBig (gemm.h) with stages of 128 codes in place of 64 bf16
// values.  A wave's 128 features are one block of the weight's scales, its lanes' tokens
// have one scale each, so a stage needs four scale products a lane.  The scales of a stage
// (256 features', 256 tokens') take one more load a thread, into one of four places in LDS.
// 4096 tokens, 32000 x 4096: 470 to 490 us, 2.2 to 2.3 PFLOP/s, the matrix units busy 54% of
// the cycles: 7.8 rounds of tiles, and the epilogue's 262 MB, which nothing hides.
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
  const float *sptr = side.scale + (min((wave < 4 ? m0 + tid : n0 + tid - 256), side.rows - 1) >> side.shift);
  auto load_s = [&](int t, int u) EE_ALWAYS_INLINE {  // stage u's, to stage t's place
    load_lds4(sptr + u * side.scale_ld, lds0 + kBigStages + (t & 3) * kBigScales + wave * 256);
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

// Few tokens, weights streamed once: a block has 16 RB features and up to 16 NB tokens, its
// waves share K and read both operands straight into MFMA fragments, U blocks of K at a
// time; their sums meet in LDS and each wave finishes some of the 16 x 16 blocks.  The weights'
// trip bounds it: 32000 x 4096, 1 token: 24 us, 5.5 TB/s (through an LDS ring 30 us).
template <int RB, int NB, int WAVES, int U, bool ROW1, bool E5, bool WIDE>
__global__ __launch_bounds__(64 * WAVES) void skinny8_kernel(ScaledMat W, ScaledMat Z, int K, StoreC out) {
  __shared__ f32x4_t red[WAVES][RB * NB][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m0 = blockIdx.x * 16 * RB, n0 = blockIdx.y * 16 * NB;
  const int bytes = (K + 15) & ~15, nk = cdiv(bytes, 128);
  const int k0 = wave * nk / WAVES, k1 = (wave + 1) * nk / WAVES, g = lane >> 4;
  const uint8_t *wp[RB], *zp[NB];
  const float *zsp[NB];
  static_for<RB>([&](auto i) EE_ALWAYS_INLINE {
    wp[i] = W.data + static_cast<int64_t>(min(m0 + decltype(i)::value * 16 + (lane & 15), W.rows - 1)) * W.ld + g * 16;
  });
  static_for<NB>([&](auto j) EE_ALWAYS_INLINE {
    const int row = min(n0 + decltype(j)::value * 16 + (lane & 15), Z.rows - 1);
    zp[j] = Z.data + static_cast<int64_t>(row) * Z.ld + g * 16;
    zsp[j] = Z.scale + (row >> Z.shift);
  });
  f32x4_t acc[RB][NB];
  static_for<RB>([&](auto i) EE_ALWAYS_INLINE {
    static_for<NB>([&](auto j) EE_ALWAYS_INLINE { acc[i][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f}; });
  });
  auto load = [&](const uint8_t *p, int k, int left) EE_ALWAYS_INLINE {
    // chunks g and 4 + g of the row's 128 bytes; past the matrix: zeros, read from its row's first
    const uint8_t *at = p + static_cast<int64_t>(k) * 128;
    i32x4_t lo = *reinterpret_cast<const i32x4_t *>(g * 16 < left ? at : at - g * 16);
    i32x4_t hi = *reinterpret_cast<const i32x4_t *>(64 + g * 16 < left ? at + 64 : at - g * 16);
    if (left < 128) {
      const i32x4_t zero = {0, 0, 0, 0};
      if (g * 16 >= left) lo = zero;
      if (64 + g * 16 >= left) hi = zero;
    }
    return i32x8_t(__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  // N blocks of K from k on, all loads ahead of the products
  auto step = [&](auto n, int k, int left) EE_ALWAYS_INLINE {
    constexpr int N = decltype(n)::value;
    i32x8_t fw[N][RB], fz[N][NB];
    float zs[N][NB];
    f32x4_t ws[N][ROW1 ? RB : 1];
    static_for<N>([&](auto q) EE_ALWAYS_INLINE {
      constexpr int Q = decltype(q)::value;
      const int l = Q == N - 1 ? left : 128;
      static_for<RB>([&](auto i) EE_ALWAYS_INLINE { fw[Q][i] = load(wp[i], k + Q, l); });
      static_for<NB>([&](auto j) EE_ALWAYS_INLINE { fz[Q][j] = load(zp[j], k + Q, l); });
      static_for<NB>([&](auto j) EE_ALWAYS_INLINE { zs[Q][j] = zsp[j][(k + Q) * Z.scale_ld]; });
      const float *s = W.scale + (k + Q) * W.scale_ld;
      if constexpr (ROW1) {
        static_for<RB>([&](auto i) EE_ALWAYS_INLINE {
          const int r = m0 + decltype(i)::value * 16 + g * 4;
          ws[Q][i] = f32x4_t{s[min(r, W.rows - 1)], s[min(r + 1, W.rows - 1)], s[min(r + 2, W.rows - 1)], s[min(r + 3, W.rows - 1)]};
        });
      } else {
        const float v = s[m0 >> 7];  // (16 RB features lie in one block of 128)
        ws[Q][0] = f32x4_t{v, v, v, v};
      }
    });
    __builtin_amdgcn_sched_barrier(0);
    static_for<N>([&](auto q) EE_ALWAYS_INLINE {
      constexpr int Q = decltype(q)::value;
      bf16x8_t wz[WIDE ? NB : 1][4];
      if constexpr (WIDE) static_for<NB>([&](auto j) EE_ALWAYS_INLINE { widen32<E5>(fz[Q][j], wz[j]); });
      static_for<RB>([&](auto i) EE_ALWAYS_INLINE {
        bf16x8_t ww[4];
        if constexpr (WIDE) widen32<false>(fw[Q][i], ww);
        static_for<NB>([&](auto j) EE_ALWAYS_INLINE {
          f32x4_t d;
          if constexpr (WIDE)
            d = mfma_wide(ww, wz[j]);
          else
            d = mfma8<E5>(fw[Q][i], fz[Q][j]);
          acc[i][j] += d * (ws[Q][ROW1 ? decltype(i)::value : 0] * zs[Q][j]);
        });
      });
    });
  };
  const int whole = min(k1, bytes / 128);  // blocks of K that the matrix fills
  int k = k0;
  for (; k + U <= whole; k += U) step(std::integral_constant<int, U>{}, k, 128);
  for (; k < k1; ++k) step(std::integral_constant<int, 1>{}, k, min(bytes - k * 128, 128));
  static_for<RB>([&](auto i) EE_ALWAYS_INLINE {
    static_for<NB>([&](auto j) EE_ALWAYS_INLINE { red[wave][decltype(i)::value * NB + decltype(j)::value][lane] = acc[i][j]; });
  });
  __syncthreads();
  for (int b = wave; b < RB * NB; b += WAVES) {
    f32x4_t v = red[0][b][lane];
    static_for<WAVES - 1>([&](auto w) EE_ALWAYS_INLINE { v += red[decltype(w)::value + 1][b][lane]; });
    store_c<WIDE>(out, n0 + (b % NB) * 16 + (lane & 15), m0 + (b / NB) * 16 + g * 4, v);
  }
}

// f(ROW1, E5, WIDE) for the matrices and C's type (of those that a tile is built for).
template <bool F32, bool BF16, class F>
hipError_t with_types(const ScaledMat &W, const ScaledMat &Z, bool f32, F &&f) {
  auto by = [&](auto row1, auto e5) {
    if constexpr (F32) {
      if (f32) return f(row1, e5, std::true_type{});
    }
    if constexpr (BF16) {
      if (!f32) return f(row1, e5, std::false_type{});
    }
    return hipErrorInvalidValue;
  };
  if (W.shift == 0) return Z.e5m2 ? by(std::true_type{}, std::true_type{}) : by(std::true_type{}, std::false_type{});
  return Z.e5m2 ? by(std::false_type{}, std::true_type{}) : by(std::false_type{}, std::false_type{});
}

template <int RB, int NB, int WAVES, int U>
hipError_t launch_skinny8(const ScaledMat &W, const ScaledMat &Z, bool f32, const StoreC &out, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(cdiv(W.rows, 16 * RB)), static_cast<unsigned>(cdiv(Z.rows, 16 * NB)));
  return with_types<true, true>(W, Z, f32, [&](auto row1, auto e5, auto wide) {
    hipLaunchKernelGGL((skinny8_kernel<RB, NB, WAVES, U, decltype(row1)::value, decltype(e5)::value, decltype(wide)::value>),
                       grid, dim3(64 * WAVES), 0, stream, W, Z, W.cols, out);
    return hipGetLastError();
  });
}

template <int BM, int BN, int WM, int WN, int KW, int NS, bool F32 = true, bool BF16 = true>
hipError_t launch_ring8(const ScaledMat &W, const ScaledMat &Z, bool f32, const StoreC &out, hipStream_t stream) {
  const int64_t blocks = static_cast<int64_t>(cdiv(W.rows, BM)) * cdiv(Z.rows, BN);
  return with_types<F32, BF16>(W, Z, f32, [&](auto row1, auto e5, auto wide) {
    hipLaunchKernelGGL((ring8_kernel<BM, BN, WM, WN, KW, NS, decltype(row1)::value, decltype(e5)::value, decltype(wide)::value>),
                       dim3(static_cast<unsigned>(blocks)), dim3(BM / WM * (BN / WN) * KW * 64), 0, stream, W, Z, W.cols, out);
    return hipGetLastError();
  });
}

// Which tile a product takes: the one of least time by a model, us with r rounds of T tiles
// (features by tokens) over `slots` at a time, r1 rounds of one a CU, n tokens and K:
//   rings and big8:  t0 + t1 r + t2 r K / 1000 + t3 T K / 1e5 + t4 r1 K / 1000
//   direct loads:    t0 + t1 T / 1000 + t2 r K / 1000 + t3 T K / 1e5 + t4 T K n / 1.6e6
// fitted to 36000 shapes (1 to 8192 tokens, 500 to 66000 features, K 320 to 16000), each
// timed on every tile that could matter.  Over those shapes the choice is 2 to 3% slower in
// the mean than the best of sixteen tiles, 16% in the worst twentieth.  What it weighs, us
// of the best against the next (bf16 C unless fp32 is said):
//   1 token: 32000 x 4096 direct 16 rows 23.7, 32 rows 24.9, ring 29.6; 8192 x 22016 16 rows
//   and 8 waves 34.1, 4 waves 39.0;
//   5120 x 13824: 16 tokens 32 x 16 shared by 8 waves 18.4, 32 x 32 20.0, direct 23.1; 48
//   tokens 32 x 64 by 4 waves 27.9 (fp32 32.0), 64 x 64 by 2 35.0, unshared 48.0;
//   13824 x 5120: 48 tokens 64 x 64 shared 19.4, unshared 22.6, 32 x 64 25.8; 200 tokens 128 x
//   64 45.1, 128 x 128 48.9, 64 x 128 51.3;
//   4096 tokens, 32000 x 4096: 256 x 256 470, 128 x 128 1156.
struct Tile8 {
  int bm, bn, slots;
  float bf16[5], f32[5];  // t0 .. t4 by C's type (t1 < 0: none)
};
enum { kBig, k128x256, k128x128, k128x64, k64x128, k64x64, k64x32, k32x64, k32x32, k32x16, kDirect16, kDirect32, kDirect16by8, kTiles8 };
constexpr Tile8 kTile8[kTiles8] = {
    {256, 256, 256, {0.0f, 17.716f, 0.0f, 1.982f, 8.948f}, {0.0f, -1.0f}},
    {128, 256, 256, {0.0f, -1.0f}, {0.0f, 11.229f, 11.484f, 2.039f, 0.0f}},
    {128, 128, 512, {0.0f, 7.793f, 5.655f, 0.457f, 2.18f}, {0.0f, 8.767f, 3.162f, 0.841f, 5.249f}},
    {128, 64, 512, {1.234f, 4.269f, 2.695f, 0.255f, 1.917f}, {0.949f, 5.15f, 1.486f, 0.284f, 3.935f}},
    {64, 128, 256, {1.45f, 3.649f, 3.261f, 0.469f, 0.0f}, {1.279f, 4.625f, 4.623f, 0.441f, 0.0f}},
    {64, 64, 256, {1.66f, 2.572f, 1.819f, 0.484f, 0.0f}, {1.327f, 3.333f, 0.0f, 0.358f, 2.425f}},
    {64, 32, 512, {0.312f, 3.792f, 0.0f, 0.406f, 1.589f}, {0.0f, 4.264f, 0.0f, 0.367f, 1.943f}},
    {32, 64, 256, {1.927f, 2.178f, 1.043f, 0.247f, 0.0f}, {1.608f, 2.541f, 1.596f, 0.225f, 0.0f}},
    {32, 32, 256, {2.359f, 1.686f, 0.816f, 0.199f, 0.0f}, {2.101f, 1.958f, 1.029f, 0.165f, 0.0f}},
    {32, 16, 256, {2.226f, 1.812f, 0.465f, 0.325f, 0.0f}, {1.919f, 2.141f, 0.637f, 0.28f, 0.0f}},
    {16, 16, 2048, {4.039f, 0.0f, 0.312f, 0.229f, 0.126f}, {4.132f, 0.0f, 0.263f, 0.231f, 0.132f}},
    {32, 16, 1024, {3.761f, 0.0f, 0.696f, 0.448f, 0.163f}, {3.774f, 0.0f, 0.792f, 0.456f, 0.169f}},
    {16, 16, 1024, {4.154f, 0.249f, 0.145f, 0.249f, 0.121f}, {4.095f, 0.429f, 0.174f, 0.25f, 0.133f}},
};

}  // namespace

int scaled_tile(bool c_f32, bool row_scales, int features, int tokens, int K) {
  int best = -1;
  double least = 0.0;
  for (int i = 0; i < kTiles8; ++i) {
    const Tile8 &t = kTile8[i];
    const float *c = c_f32 ? t.f32 : t.bf16;
    const bool direct = i >= kDirect16;
    // (below 1024 values of K the big tile's loads are mostly the first stages' again)
    if (c[1] < 0.0f || (i == kBig && (row_scales || K < 1024)) || (tokens > 16 ? direct : i < k32x32)) continue;
    const double T = static_cast<double>(cdiv(features, t.bm)) * cdiv(tokens, t.bn), k = K * 1e-3;
    const double r = std::ceil(T / t.slots), r1 = std::ceil(T / 256);
    const double us = direct ? c[0] + c[1] * T * 1e-3 + c[2] * r * k + (c[3] + c[4] * tokens / 16.0) * T * k * 1e-2
                             : c[0] + c[1] * r + c[2] * r * k + c[3] * T * k * 1e-2 + c[4] * r1 * k;
    if (best < 0 || us < least) {
      best = i;
      least = us;
    }
  }
  return best;
}

hipError_t scaled_matmul(const ScaledMat &a, const ScaledMat &b, void *c, bool c_f32, int64_t ldc, int accumulate,
                         hipStream_t stream) {
  if (a.rows <= 0 || b.rows <= 0) return hipSuccess;
  if (((a.cols + 15) & ~15) != ((b.cols + 15) & ~15) || b.e5m2) return hipErrorInvalidValue;
  const StoreC out{c, ldc, a.rows, b.rows, accumulate != 0};
  switch (scaled_tile(c_f32, b.shift == 0, b.rows, a.rows, b.cols)) {
    case kBig: {
      const dim3 grid(static_cast<unsigned>(cdiv(a.rows, 256)) * cdiv(b.rows, 256));
      if (a.e5m2)
        hipLaunchKernelGGL((big8_kernel<true>), grid, dim3(512), 0, stream, b, a, b.cols, out);
      else
        hipLaunchKernelGGL((big8_kernel<false>), grid, dim3(512), 0, stream, b, a, b.cols, out);
      return hipGetLastError();
    }
    case k128x256: return launch_ring8<128, 256, 64, 64, 1, 2, true, false>(b, a, c_f32, out, stream);
    case k128x128: return launch_ring8<128, 128, 64, 64, 1, 2>(b, a, c_f32, out, stream);
    case k128x64: return launch_ring8<128, 64, 64, 32, 1, 3>(b, a, c_f32, out, stream);
    case k64x128: return launch_ring8<64, 128, 32, 64, 2, 2>(b, a, c_f32, out, stream);
    case k64x64: return launch_ring8<64, 64, 64, 32, 4, 2>(b, a, c_f32, out, stream);
    case k64x32: return launch_ring8<64, 32, 32, 32, 2, 4>(b, a, c_f32, out, stream);
    case k32x64: return launch_ring8<32, 64, 32, 32, 4, 3>(b, a, c_f32, out, stream);
    case k32x32: return launch_ring8<32, 32, 32, 32, 4, 3>(b, a, c_f32, out, stream);
    case k32x16: return launch_ring8<32, 16, 32, 16, 8, 3>(b, a, c_f32, out, stream);
    case kDirect16: return launch_skinny8<1, 1, 4, 4>(b, a, c_f32, out, stream);
    case kDirect32: return launch_skinny8<2, 1, 4, 4>(b, a, c_f32, out, stream);
    default: return launch_skinny8<1, 1, 8, 4>(b, a, c_f32, out, stream);
  }
}

}  // namespace ee

#pragma clang diagnostic pop
