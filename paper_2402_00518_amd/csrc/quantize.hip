// 8-bit codes with block scales: a matrix, or the normalised rows of an exit.
//
// A block is 128 columns of 1 or 128 rows.  With M the largest code of the type
// (e4m3 448, e5m2 57344), s = max(max |x| / M, 2^-100) and the code of x is
// x * (1 / s) rounded to nearest even: 448 is reached, never passed (the
// products are at most M (1 + 2^-22), which rounds to M).  A NaN is left out of
// the maximum and keeps its own code; an infinity makes its block's scale
// infinite, so that products with the block are NaN.
//
// Memory bounds it: every value is read once, held in registers as one 128 x 128 tile a
// block (whose maxima need it whole, by rows, by columns or altogether) and its codes are
// written once or, with the transpose, twice.  32000 x 4096: fp32 weights (655 MB) 120 us,
// bf16 73 us, 5.4 TB/s; 4001 x 5120 bf16 with both outputs (82 MB): 21 us, 3.9 TB/s, 1280 tiles
// whose reading, barriers, LDS turn and writing follow each other, five tiles a CU; 8 rows of
// 4096: 4 us, one launch.
#include <hip/hip_runtime.h>

#include "ee_device.h"
#include "launch.h"

namespace ee {

namespace {

constexpr float kLeastScale = 0x1p-100f;

template <bool E5M2>
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  int r;
  if constexpr (E5M2) {
    r = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, 0, false);
    r = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, r, true);
  } else {
    r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
  }
  return static_cast<uint32_t>(r);
}

__device__ __forceinline__ float block_scale(float amax, bool e5m2) {
  return fmaxf(amax / (e5m2 ? 57344.0f : 448.0f), kLeastScale);
}

__device__ __forceinline__ float max16(float v) {  // over 16 consecutive lanes
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}

// Eight values of a row from column c on (0 past the last column).  Rows need not be aligned
// (4001 x 5124 bf16, both outputs: element by element 51 us, so 24).
template <typename T>
__device__ __forceinline__ void load8(const T *row, int c, int cols, float (&v)[8]) {
  if (c + 8 <= cols) {
    if constexpr (std::is_same<T, float>::value) {
      const f32x4_t a = load_any<f32x4_t>(row + c), b = load_any<f32x4_t>(row + c + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] = a[e];
        v[4 + e] = b[e];
      }
    } else {
      const u32x4_t a = load_any<u32x4_t>(row + c);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[2 * e] = __uint_as_float(a[e] << 16);
        v[2 * e + 1] = __uint_as_float(a[e] & 0xFFFF0000u);
      }
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = c + e < cols ? to_f32(row[c + e]) : 0.0f;
}

// Eight values as they are stored: bf16 ones in four registers, which leaves room for four
// blocks a CU in place of three (32000 x 4096 bf16 100 -> 73 us).
template <typename T>
struct Eight {
  float v[8];
  __device__ __forceinline__ float operator[](int e) const { return v[e]; }
  __device__ __forceinline__ void load(const float *row, int c, int cols) { load8(row, c, cols, v); }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.0f;
  }
};
template <>
struct Eight<bf16_t> {
  u32x4_t v;
  __device__ __forceinline__ float operator[](int e) const {
    return __uint_as_float(e % 2 == 0 ? v[e / 2] << 16 : v[e / 2] & 0xFFFF0000u);
  }
  __device__ __forceinline__ void load(const bf16_t *row, int c, int cols) {
    if (c + 8 <= cols) {
      v = load_any<u32x4_t>(row + c);
      return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      v[e] = (c + 2 * e < cols ? row[c + 2 * e] : 0u) | (c + 2 * e + 1 < cols ? static_cast<uint32_t>(row[c + 2 * e + 1]) << 16 : 0u);
  }
  __device__ __forceinline__ void clear() { v = u32x4_t{0, 0, 0, 0}; }
};

// One 128 x 128 tile a block of 256 threads: thread t holds columns 8 (t mod 16)
// .. + 7 of rows 4 (t / 16) .. + 3 and those + 64.  Four consecutive rows a thread, so that
// a column's codes pack into one 32-bit word on their way through LDS to the
// transposed output.
template <typename T, bool E5Q, bool E5T>
__global__ __launch_bounds__(256) void quantize_kernel(const T *__restrict__ x, int64_t ldx, int rows, int cols, bool apart,
                                                       ScaledMat q, ScaledMat qt) {
  __shared__ float colmax[4][128];
  __shared__ float wavemax[4];
  __shared__ uint32_t turned[128 * 32];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int across = (cols + 127) >> 7;  // (the grid is a multiple of 8)
  const int tile = apart ? (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3) : blockIdx.x;
  const int tc = tile % across, tr = tile / across;
  if (tr * 128 >= rows) return;
  const int c0 = tc * 128, r0 = tr * 128;
  const int c = (tid & 15) * 8, rg = tid >> 4;
  Eight<T> v[8];
  float rowmax[8], cm[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = r0 + rg * 4 + (i & 3) + (i >> 2) * 64;
    if (r < rows) {
      v[i].load(x + r * ldx, c0 + c, cols);
    } else {
      v[i].clear();
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) cm[e] = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float m = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      m = fmaxf(m, fabsf(v[i][e]));
      cm[e] = fmaxf(cm[e], fabsf(v[i][e]));
    }
    rowmax[i] = max16(m);
  }
  const bool tile_scale = (q.data != nullptr && q.shift != 0) || (qt.data != nullptr && qt.shift != 0);
  float tilemax = 0.0f;
  if (tile_scale) {
#pragma unroll
    for (int i = 0; i < 8; ++i) tilemax = fmaxf(tilemax, rowmax[i]);
    tilemax = fmaxf(tilemax, __shfl_xor(tilemax, 16));
    tilemax = fmaxf(tilemax, __shfl_xor(tilemax, 32));
    if (lane == 0) wavemax[wave] = tilemax;
  }
  const bool col_scale = qt.data != nullptr && qt.shift == 0;
  if (col_scale) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      cm[e] = fmaxf(cm[e], __shfl_xor(cm[e], 16));
      cm[e] = fmaxf(cm[e], __shfl_xor(cm[e], 32));
    }
    if (lane < 16) {
#pragma unroll
      for (int e = 0; e < 8; ++e) colmax[wave][c + e] = cm[e];
    }
  }
  if (tile_scale || col_scale) __syncthreads();
  if (tile_scale) tilemax = fmaxf(fmaxf(wavemax[0], wavemax[1]), fmaxf(wavemax[2], wavemax[3]));

  if (q.data != nullptr) {
    const int pad = (cols + 15) & ~15;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = r0 + rg * 4 + (i & 3) + (i >> 2) * 64;
      const float s = block_scale(q.shift != 0 ? tilemax : rowmax[i], E5Q), inv = 1.0f / s;
      if (r < rows) {
        if (c0 + c < pad)
          *reinterpret_cast<u32x2_t *>(q.data + r * q.ld + c0 + c) =
              u32x2_t{codes4<E5Q>(v[i][0] * inv, v[i][1] * inv, v[i][2] * inv, v[i][3] * inv),
                      codes4<E5Q>(v[i][4] * inv, v[i][5] * inv, v[i][6] * inv, v[i][7] * inv)};
        if ((tid & 15) == 0 && (q.shift == 0 || r == r0))
          q.scale[tc * q.scale_ld + (q.shift != 0 ? tr : r)] = s;
      }
    }
  }
  if (qt.data != nullptr) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float m = qt.shift != 0 ? tilemax
                                    : fmaxf(fmaxf(colmax[0][c + e], colmax[1][c + e]), fmaxf(colmax[2][c + e], colmax[3][c + e]));
      const float s = block_scale(m, E5T), inv = 1.0f / s;
      // row-quad words of a column, XORed with the column so that the 16 lanes of
      // a quad spread over the banks; the XOR keeps 16-byte pieces whole
      uint32_t *w = turned + (c + e) * 32;
      const int x4 = ((c >> 3) & 7) * 4;
      w[rg ^ x4] = codes4<E5T>(v[0][e] * inv, v[1][e] * inv, v[2][e] * inv, v[3][e] * inv);
      w[(rg + 16) ^ x4] = codes4<E5T>(v[4][e] * inv, v[5][e] * inv, v[6][e] * inv, v[7][e] * inv);
      if (rg == 0 && c0 + c + e < cols && (qt.shift == 0 || c + e == 0))
        qt.scale[tr * qt.scale_ld + (qt.shift != 0 ? tc : c0 + c + e)] = s;
    }
    __syncthreads();
    const int pad = (rows + 15) & ~15;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const int col = p * 32 + (tid >> 3), k = (tid & 7) * 16;
      if (c0 + col < cols && r0 + k < pad)
        *reinterpret_cast<u32x4_t *>(qt.data + (c0 + col) * qt.ld + r0 + k) =
            *reinterpret_cast<const u32x4_t *>(turned + col * 32 + (((tid & 7) * 4) ^ (((col >> 3) & 7) * 4)));
    }
  }
}

// The rows of an exit's norm as e4m3 codes, a scale for each 128 values: z = (x -
// mu) r gain (+ bias) as row_norm_kernel forms it, in fp32 up to the code (gain
// NULL: z = x).  One block a row; rows of up to IT * 2048 values stay in registers.
template <typename Tin, typename T, int IT>
__global__ __launch_bounds__(256) void norm_quantize_kernel(const Tin *__restrict__ x, int h, float eps, const T *__restrict__ gain,
                                                            const T *__restrict__ bias, int centre, uint8_t *__restrict__ q,
                                                            int64_t ldq, float *__restrict__ scale, int64_t scale_ld,
                                                            const float *__restrict__ extra, int n_extra) {
  __shared__ float red[2][4];
  const int tid = threadIdx.x;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * h, zs = static_cast<int64_t>(gridDim.x) * h;
  auto load_x = [&](int j, float (&v)[8]) EE_ALWAYS_INLINE {
    load8(x + row, j, h, v);
    for (int s = 0; s < n_extra; ++s) {
      float t[8];
      load8(extra + s * zs + row, j, h, t);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += t[e];
    }
  };
  constexpr int KEEP = IT > 0 ? IT : 1;
  float v[KEEP][8], g[KEEP][8], b[KEEP][8];
  auto load_gain = [&](int j, int c) EE_ALWAYS_INLINE {
    load8(gain, j, h, g[c]);
    if (bias != nullptr) {
      load8(bias, j, h, b[c]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) b[c][e] = 0.0f;
    }
  };
  if constexpr (IT > 0) {
#pragma unroll
    for (int c = 0; c < IT; ++c) {
      const int j = (c * 256 + tid) * 8;
      if (j < h) {
        load_x(j, v[c]);
        if (gain != nullptr) load_gain(j, c);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[c][e] = 0.0f;
      }
    }
  }
  auto each = [&](auto &&f) EE_ALWAYS_INLINE {
    if constexpr (IT > 0) {
#pragma unroll
      for (int c = 0; c < IT; ++c) {
        const int j = (c * 256 + tid) * 8;
        if (j < h) f(j, v[c], c);
      }
    } else {
      for (int j = tid * 8; j < h; j += 2048) {
        load_x(j, v[0]);
        f(j, v[0], 0);
      }
    }
  };
  auto block_sum = [&](float s, int slot) EE_ALWAYS_INLINE {
    s = warp_sum(s);
    if ((tid & 63) == 0) red[slot][tid >> 6] = s;
    __syncthreads();
    return (red[slot][0] + red[slot][1]) + (red[slot][2] + red[slot][3]);
  };
  float mean = 0.0f, r = 1.0f;
  if (gain != nullptr) {
    if (centre) {
      float t = 0.0f;
      each([&](int, const float (&w)[8], int) EE_ALWAYS_INLINE {
#pragma unroll
        for (int e = 0; e < 8; ++e) t += w[e];
      });
      mean = block_sum(t, 0) / static_cast<float>(h);
    }
    float s = 0.0f;
    each([&](int, const float (&w)[8], int) EE_ALWAYS_INLINE {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = w[e] - mean;
        s += d * d;
      }
    });
    r = 1.0f / sqrtf(block_sum(s, 1) / static_cast<float>(h) + eps);
  }
  // 16 threads hold a block of 128 values; a thread past the last value lends
  // its lane to the maximum.  h is a multiple of 64, so the last block may have 8.
  for (int c = 0, base = 0; base < h; ++c, base += 2048) {
    const int j = base + tid * 8;
    float o[8];
    float m = 0.0f;
    auto form = [&](const float (&w)[8], const float (&gc)[8], const float (&bc)[8]) EE_ALWAYS_INLINE {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        o[e] = gain != nullptr ? (w[e] - mean) * r * gc[e] + bc[e] : w[e];
        m = fmaxf(m, fabsf(o[e]));
      }
    };
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = 0.0f;
    if (j < h) {
      if constexpr (IT == 0) {
        load_x(j, v[0]);
        if (gain != nullptr) load_gain(j, 0);
        form(v[0], g[0], b[0]);
      } else {
        static_for<KEEP>([&](auto i) EE_ALWAYS_INLINE {
          if (c == decltype(i)::value) form(v[i], g[i], b[i]);
        });
      }
    }
    const float s = block_scale(max16(m), false), inv = 1.0f / s;
    if (j < h) {
      *reinterpret_cast<u32x2_t *>(q + blockIdx.x * ldq + j) =
          u32x2_t{codes4<false>(o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv),
                  codes4<false>(o[4] * inv, o[5] * inv, o[6] * inv, o[7] * inv)};
      if ((tid & 15) == 0) scale[(j >> 7) * scale_ld + blockIdx.x] = s;
    }
  }
}

}  // namespace

hipError_t launch_quantize(bool f32, const void *x, int64_t ldx, int rows, int cols, const ScaledMat *q, const ScaledMat *qt,
                           hipStream_t stream) {
  if (rows <= 0 || cols <= 0) return hipSuccess;
  const ScaledMat none{};
  const ScaledMat a = q != nullptr ? *q : none, b = qt != nullptr ? *qt : none;
  // Where a tile's pieces of rows end inside a cache line, the next tile along the row goes to the
  // same XCD, whose L2 has the line: 32003 x 4095 bf16 85 us, in plain order 154; 9000 x
  // 14000 fp32 131 and 155.  Else plain order spreads better: 32000 x 4096 bf16 73 us, so 77.
  const bool apart = ldx * (f32 ? 4 : 2) % 128 != 0;
  const dim3 grid(((cols + 127) / 128 * ((rows + 127) / 128) + 7) / 8 * 8);
  EE_DISPATCH(f32, {
    const T *xt = static_cast<const T *>(x);
    auto go = [&](auto eq, auto et) {
      hipLaunchKernelGGL((quantize_kernel<T, decltype(eq)::value, decltype(et)::value>), grid, dim3(256), 0, stream, xt, ldx,
                         rows, cols, apart, a, b);
    };
    if (a.e5m2 && b.e5m2)
      go(std::true_type{}, std::true_type{});
    else if (a.e5m2)
      go(std::true_type{}, std::false_type{});
    else if (b.e5m2)
      go(std::false_type{}, std::true_type{});
    else
      go(std::false_type{}, std::false_type{});
  });
  return hipGetLastError();
}

hipError_t launch_norm_quantize(bool x_f32, bool f32, const void *x, int n, int h, float eps, const void *gain, const void *bias,
                                bool centre, const ScaledMat &q, hipStream_t stream, const float *extra, int n_extra) {
  if (n <= 0) return hipSuccess;
  if (h % 64 != 0 || (n_extra > 0 && (!x_f32 || extra == nullptr))) return hipErrorInvalidValue;
  EE_DISPATCH(f32, {
    const T *g = static_cast<const T *>(gain), *b = static_cast<const T *>(bias);
    auto go = [&](auto it) {
      constexpr int IT = decltype(it)::value;
      if (x_f32)
        hipLaunchKernelGGL((norm_quantize_kernel<float, T, IT>), dim3(n), dim3(256), 0, stream, static_cast<const float *>(x), h,
                           eps, g, b, centre ? 1 : 0, q.data, q.ld, q.scale, q.scale_ld, extra, n_extra);
      else
        hipLaunchKernelGGL((norm_quantize_kernel<bf16_t, T, IT>), dim3(n), dim3(256), 0, stream, static_cast<const bf16_t *>(x), h,
                           eps, g, b, centre ? 1 : 0, q.data, q.ld, q.scale, q.scale_ld, extra, 0);
    };
    if (h <= 2048)
      go(std::integral_constant<int, 1>{});
    else if (h <= 4096)
      go(std::integral_constant<int, 2>{});
    else if (h <= 8192)
      go(std::integral_constant<int, 4>{});
    else
      go(std::integral_constant<int, 0>{});
  });
  return hipGetLastError();
}

}  // namespace ee
