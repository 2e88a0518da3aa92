// Sampling: one token a row of logits from a given random number.
//
// Tokens are ordered by falling logit, equal ones by rising id.  With mass_i =
// exp((x_i - max) / T), top-k keeps the first k of that order, top-p the shortest
// prefix whose mass reaches p times that of what top-k left, min-p those with mass_i
// >= min_p (the largest mass is 1); all three keep a prefix, so what is kept is known
// by its last logit and, among the tokens that share it, how many.  The token is
// the lowest id whose cumulated kept mass, in the order of ids, passes u times the
// whole.  Masses and their sums are 64 bits wide: a sum of 32 over a vocabulary
// would move its borders by more than the distance of neighbouring random numbers.
//
// One block of 16 waves a row.  Each wave holds a range of consecutive ids, so that
// everything in the order of ids is a prefix over waves, then inside one.
//   1. maximum;
//   2. sum of masses, and in LDS a histogram over (max - x) / T in 2047 bins of
//      1/64 and one for the rest: of counts for top-k, else of masses for top-p.
//      (Masses as multiples of 2^-43, so that the order of the atomics does not show.)
//   3. the bin in which the cut lies; its tokens and all above it, in the order of
//      ids, as a list in LDS; that list's logits sorted, their masses cumulated:
//      the cut; the list cumulated in the order of ids: the token.
// Where the list would not fit, top-p alone lists the cut's bin only and walks the
// row once more; what is left (a cut in the last bin, thousands of equal logits)
// finds the cut by the digits of the logits' bits, three passes over the row.
#include <hip/hip_runtime.h>

#include "ee_device.h"
#include "launch.h"

namespace ee {

namespace {

constexpr int kWaves = 16, kThreads = kWaves * 64;
constexpr int kBins = 2048;
constexpr float kBinsPerUnit = 64.0f;
constexpr int kList = 4096;
constexpr double kUnit = 0x1p43;  // masses in the histogram: at most 2^20 tokens of mass 1

// 2^t for t <= 0, relative error 1e-14: 2^f = sum (f ln 2)^k / k! on |f| <= 1/2.
__device__ __forceinline__ double pow2_neg(double t) {
  const double n = __builtin_rint(t), y = (t - n) * 0.69314718055994530942;
  double p = 1.0 / 479001600.0;
  p = __builtin_fma(p, y, 1.0 / 39916800.0);
  p = __builtin_fma(p, y, 1.0 / 3628800.0);
  p = __builtin_fma(p, y, 1.0 / 362880.0);
  p = __builtin_fma(p, y, 1.0 / 40320.0);
  p = __builtin_fma(p, y, 1.0 / 5040.0);
  p = __builtin_fma(p, y, 1.0 / 720.0);
  p = __builtin_fma(p, y, 1.0 / 120.0);
  p = __builtin_fma(p, y, 1.0 / 24.0);
  p = __builtin_fma(p, y, 1.0 / 6.0);
  p = __builtin_fma(p, y, 0.5);
  p = __builtin_fma(p, y, 1.0);
  p = __builtin_fma(p, y, 1.0);
  // (the clamp leaves 0 for -infinity and for what ldexp would underflow to)
  return t < -1022.0 ? 0.0 : __builtin_amdgcn_ldexp(p, static_cast<int>(n));
}

// Bits that order as the values do; -0 counts as 0.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) {
  return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key);
}

template <typename V>
__device__ __forceinline__ V wave_scan(V v, int lane) {  // inclusive
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const V t = __shfl_up(v, o);
    if (lane >= o) v += t;
  }
  return v;
}
template <typename V>
__device__ __forceinline__ V wave_sum(V v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

struct Shared {
  union {
    unsigned long long hist[kBins];
    uint32_t sorted[kList];
  };
  uint32_t key[kList];
  int32_t id[kList];
  double part[2][kWaves];
  int ipart[2][kWaves];
  unsigned long long upart[kWaves];
  int found;
  unsigned long long before;
  int token;
  double mass;
};

template <typename T, int IT>
struct Row {
  static constexpr int KEEP = IT > 0 ? IT : 1;
  const T *p;
  const uint32_t *allowed;
  int vocab, first, last;  // ids of the wave: [first, last)
  bool vec;
  int lane;
  float kept[KEEP][4];

  __device__ __forceinline__ void load4(int id, float (&x)[4]) const {
    if (vec && id + 4 <= vocab) {
      if constexpr (std::is_same<T, float>::value) {
        const f32x4_t v = *reinterpret_cast<const f32x4_t *>(p + id);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = v[e];
      } else {
        const u32x2_t v = *reinterpret_cast<const u32x2_t *>(p + id);
        x[0] = __uint_as_float(v[0] << 16);
        x[1] = __uint_as_float(v[0] & 0xFFFF0000u);
        x[2] = __uint_as_float(v[1] << 16);
        x[3] = __uint_as_float(v[1] & 0xFFFF0000u);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = id + e < vocab ? to_f32(p[id + e]) : -INFINITY;
    }
    if (allowed != nullptr && id < vocab) {
      const uint32_t w = allowed[id >> 5] >> (id & 31);  // id is a multiple of 4
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (((w >> e) & 1) == 0) x[e] = -INFINITY;
    }
  }
  __device__ __forceinline__ void init() {
    if constexpr (IT > 0) {
#pragma unroll
      for (int i = 0; i < IT; ++i) {
        const int id = first + i * 256 + lane * 4;
        if (id < last)
          load4(id, kept[i]);
        else
          kept[i][0] = kept[i][1] = kept[i][2] = kept[i][3] = -INFINITY;
      }
    }
  }
  // f(first id, values) for every four ids of this lane, in the order of ids.  Every
  // lane of the wave takes part (ids past the last have -infinity).
  template <class F>
  __device__ __forceinline__ void each(F &&f) const {
    if constexpr (IT > 0) {
#pragma unroll
      for (int i = 0; i < IT; ++i) {
        f(first + i * 256 + lane * 4, kept[i]);
        __builtin_amdgcn_sched_barrier(0);  // (one group's work at a time: mixed, they need more registers than there are)
      }
    } else {
      for (int i = first; i < last; i += 256) {
        float x[4];
        const int id = i + lane * 4;
        if (id < last)
          load4(id, x);
        else
          x[0] = x[1] = x[2] = x[3] = -INFINITY;
        f(id, x);
      }
    }
  }
};

template <typename T, int IT>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a) {
  __shared__ Shared sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = blockIdx.x;
  const float temp = a.temperature != nullptr ? a.temperature[n] : 1.0f;
  const int top_k = a.top_k != nullptr ? a.top_k[n] : 0;
  const float top_p = a.top_p != nullptr ? a.top_p[n] : 1.0f;
  const float min_p = a.min_p != nullptr ? a.min_p[n] : 0.0f;
  const float u = a.uniform[n];
  Row<T, IT> row;
  row.p = static_cast<const T *>(a.logits) + n * a.ld;
  row.allowed = a.allowed != nullptr ? a.allowed + n * a.allowed_ld : nullptr;
  row.vocab = a.vocab;
  const int chunk = (a.vocab + kWaves * 256 - 1) / (kWaves * 256) * 256;
  row.first = min(wave * chunk, a.vocab);
  row.last = min(row.first + chunk, a.vocab);
  row.vec = a.ld * sizeof(T) % (4 * sizeof(T)) == 0;
  row.lane = lane;
  row.init();

  int slot = 0;  // block sums alternate between two slots, one barrier each
  auto block_sum = [&](double v) EE_ALWAYS_INLINE {
    v = wave_sum(v);
    if (lane == 0) sh.part[slot][wave] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) s += sh.part[slot][w];
    slot ^= 1;
    return s;
  };

  // 1. the maximum, and whether the row has a distribution at all
  float mx = -INFINITY;
  bool bad = temp != temp || top_p != top_p || min_p != min_p || u != u;
  row.each([&](int, const float (&x)[4]) EE_ALWAYS_INLINE {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      mx = fmaxf(mx, x[e]);
      bad |= x[e] != x[e];
    }
  });
  mx = warp_max(mx);
  bad = __any(bad);
  if (lane == 0) {
    sh.part[0][wave] = mx;
    sh.ipart[0][wave] = bad;
  }
  __syncthreads();
  bad = false;
  mx = -INFINITY;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    mx = fmaxf(mx, static_cast<float>(sh.part[0][w]));
    bad |= sh.ipart[0][w] != 0;
  }
  slot = 1;
  if (bad || mx == INFINITY || mx == -INFINITY) {
    if (tid == 0) {
      a.token[n] = -1;
      if (a.prob != nullptr) a.prob[n] = 0.0f;
      if (a.confidence != nullptr) a.confidence[n] = 0.0f;
      if (a.exit_flag != nullptr) a.exit_flag[n] = 0;
    }
    return;
  }
  const bool greedy = !(temp > 0.0f);
  // (an infinite temperature still sends -infinity to mass 0)
  const double dmx = mx, c1 = 1.44269504088896340736, ct = greedy ? c1 : fmax(c1 / static_cast<double>(temp), 1e-300);
  auto mass_of = [&](float x) EE_ALWAYS_INLINE { return pow2_neg((static_cast<double>(x) - dmx) * ct); };
  const bool want_conf = a.confidence != nullptr || a.exit_flag != nullptr;
  const bool by_count = !greedy && top_k > 0 && top_k < a.vocab, by_mass = !greedy && top_p < 1.0f;
  const bool cut = by_count || by_mass;
  const bool same = ct == c1;  // one mass serves both

  // 2. sums of masses; the histogram
  const float bscale = static_cast<float>(kBinsPerUnit / (greedy ? 1.0 : static_cast<double>(temp)));
  auto bin_of = [&](float x) EE_ALWAYS_INLINE {  // monotone in x
    const float b = (mx - x) * bscale;
    return b < static_cast<float>(kBins - 1) ? static_cast<int>(b) : kBins - 1;
  };
  if (cut) {
    for (int i = tid; i < kBins; i += kThreads) sh.hist[i] = 0;
    __syncthreads();
  }
  double z = 0.0, z1 = 0.0;
  const bool need_z = (by_mass && !by_count) || (want_conf && same);
  if (need_z || cut || want_conf) {
    row.each([&](int, const float (&x)[4]) EE_ALWAYS_INLINE {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        double m = 0.0;
        if (need_z) {
          m = mass_of(x[e]);
          z += m;
        }
        if (want_conf && !same) z1 += pow2_neg((static_cast<double>(x[e]) - dmx) * c1);
        if (cut) {
          const int b = bin_of(x[e]);
          if (b < kBins - 1)
            atomicAdd(&sh.hist[b], by_count ? 1ull : static_cast<unsigned long long>(m * kUnit + 0.5));
        }
      }
    });
    z = block_sum(z);  // (its barrier also closes the histogram)
    if (want_conf && !same) z1 = block_sum(z1);
  }
  if (want_conf && tid == 0) {
    const float conf = static_cast<float>(1.0 / (same ? z : z1));
    if (a.confidence != nullptr) a.confidence[n] = conf;
    if (a.exit_flag != nullptr) a.exit_flag[n] = conf > a.threshold ? 1 : 0;
  }

  auto finish = [&](int token, double prob) EE_ALWAYS_INLINE {
    a.token[n] = token;
    if (a.prob != nullptr) a.prob[n] = static_cast<float>(prob);
  };
  if (greedy) {
    int at = 0x7FFFFFFF;
    row.each([&](int id, const float (&x)[4]) EE_ALWAYS_INLINE {
#pragma unroll
      for (int e = 3; e >= 0; --e)
        if (x[e] == mx) at = min(at, id + e);
    });
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) at = min(at, __shfl_xor(at, o));
    if (lane == 0) sh.ipart[1][wave] = at;
    __syncthreads();
    if (tid == 0) {
      for (int w = 0; w < kWaves; ++w) at = min(at, sh.ipart[1][w]);
      finish(at, 1.0);
    }
    return;
  }

  // What is kept: keys above `tau`, and the first `ties` of those equal to it; mass
  // at least `least`.  The largest logit's first token always is.
  uint32_t tau = 0;
  int ties = 0x7FFFFFFF;
  const double least = min_p > 0.0f ? (min_p < 1.0f ? static_cast<double>(min_p) : 1.0) : 0.0;
  const double p = top_p > 0.0f ? static_cast<double>(top_p) : 0.0;

  // Inclusive prefix of a value a thread over the block; returns it and the total.
  auto block_scan = [&](auto v, auto *parts, auto &total) EE_ALWAYS_INLINE {
    using V = decltype(v);
    const V mine = wave_scan(v, lane);
    if (lane == 63) parts[wave] = mine;
    __syncthreads();
    V before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const V t = parts[w];
      if (w < wave) before += t;
      total += t;
    }
    __syncthreads();
    return before + mine;
  };

  // Tokens whose bin satisfies lo <= bin <= hi, in the order of ids, as the list;
  // returns how many there are (the list holds them if no more than it has room for).
  auto make_list = [&](int lo, int hi) EE_ALWAYS_INLINE {
    int count = 0;
    auto in = [&](float x) EE_ALWAYS_INLINE {
      if (!(x > -INFINITY)) return false;
      const int b = bin_of(x);
      return b >= lo && b <= hi;
    };
    row.each([&](int, const float (&x)[4]) EE_ALWAYS_INLINE {
#pragma unroll
      for (int e = 0; e < 4; ++e) count += in(x[e]) ? 1 : 0;
    });
    count = wave_sum(count);
    if (lane == 0) sh.ipart[0][wave] = count;
    __syncthreads();
    int at = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) at += sh.ipart[0][w];
      total += sh.ipart[0][w];
    }
    if (total <= kList && count > 0) {
      row.each([&](int id, const float (&x)[4]) EE_ALWAYS_INLINE {
        int mine = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) mine += in(x[e]) ? 1 : 0;
        if (__any(mine > 0)) {
          const int upto = wave_scan(mine, lane);
          int o = at + upto - mine;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (in(x[e])) {
              sh.key[o] = key_of(x[e]);
              sh.id[o] = id + e;
              ++o;
            }
          }
          at += __shfl(upto, 63);
        }
      });
    }
    __syncthreads();
    return total;
  };

  // The list's keys by falling value in sh.sorted.
  auto sort_list = [&](int len) EE_ALWAYS_INLINE {
    int size = 64;
    while (size < len) size <<= 1;
    for (int i = tid; i < size; i += kThreads) sh.sorted[i] = i < len ? sh.key[i] : 0;
    __syncthreads();
    for (int k = 2; k <= size; k <<= 1) {
      for (int j = k >> 1; j > 0; j >>= 1) {
        for (int t = tid; t < size / 2; t += kThreads) {
          const int i = 2 * t - (t & (j - 1)), o = i + j;
          const uint32_t x = sh.sorted[i], y = sh.sorted[o];
          const bool falling = (i & k) == 0;
          if (falling ? x < y : x > y) {
            sh.sorted[i] = y;
            sh.sorted[o] = x;
          }
        }
        __syncthreads();
      }
    }
  };

  // tau and ties from the sorted list of `len` keys: of the first `most`, those
  // before which less than the target has gathered (share < 0: of p times the
  // mass of the first `most`; else `share`).
  auto cut_list = [&](int len, int most, double share) EE_ALWAYS_INLINE {
    double m[4], sum = 0.0, total;
    uint32_t k[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = tid * 4 + e;
      k[e] = i < len ? sh.sorted[i] : 0;
      m[e] = i < most ? mass_of(value_of(k[e])) : 0.0;
      sum += m[e];
    }
    double before = block_scan(sum, sh.part[0], total) - sum;
    const double target = !by_mass ? INFINITY : share < 0.0 ? p * total : share;
    int keep = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = tid * 4 + e;
      if (i < most && (i == 0 || before < target)) ++keep;
      before += m[e];
    }
    int kept;
    block_scan(keep, sh.ipart[0], kept);
    tau = sh.sorted[kept - 1];
    int above = 0, n_above;
#pragma unroll
    for (int e = 0; e < 4; ++e) above += tid * 4 + e < kept && k[e] > tau ? 1 : 0;
    block_scan(above, sh.ipart[0], n_above);
    ties = kept - n_above;
  };

  // tau by the digits of the keys: the largest key with at least `target` tokens, or
  // mass, at it and above; `above` is what lies above it.
  auto cut_digits = [&](bool count, double target, double &above) EE_ALWAYS_INLINE {
    uint32_t prefix = 0;
    double over = 0.0;
    const int bits[3] = {11, 11, 10};
    int shift = 32;
    for (int d = 0; d < 3; ++d) {
      const uint32_t mask = shift == 32 ? 0 : ~0u << shift;
      const int nb = 1 << bits[d];
      shift -= bits[d];
      for (int i = tid; i < nb; i += kThreads) sh.hist[i] = 0;
      __syncthreads();
      row.each([&](int, const float (&x)[4]) EE_ALWAYS_INLINE {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t key = key_of(x[e]);
          if (x[e] > -INFINITY && (key & mask) == (prefix & mask))
            atomicAdd(&sh.hist[(key >> shift) & (nb - 1)],
                      count ? 1ull : static_cast<unsigned long long>(mass_of(x[e]) * kUnit + 0.5));
        }
      });
      __syncthreads();
      // bins from the top: thread t has bins nb - 1 - 2 t and nb - 2 - 2 t
      const int hi = nb - 1 - 2 * tid;
      const unsigned long long v0 = hi >= 0 ? sh.hist[hi] : 0, v1 = hi >= 1 ? sh.hist[hi - 1] : 0;
      if (tid == 0) sh.found = -1;
      unsigned long long total;
      const unsigned long long upto = block_scan(v0 + v1, sh.upart, total);
      const double unit = count ? 1.0 : 1.0 / kUnit;
      const double b0 = over + static_cast<double>(upto - v0 - v1) * unit, b1 = over + static_cast<double>(upto - v1) * unit,
                   b2 = over + static_cast<double>(upto) * unit;
      if (hi >= 0 && v0 > 0 && b0 < target && b1 >= target) {
        sh.found = hi;
        sh.before = upto - v0 - v1;
      } else if (hi >= 1 && v1 > 0 && b1 < target && b2 >= target) {
        sh.found = hi - 1;
        sh.before = upto - v1;
      }
      __syncthreads();
      int f = sh.found;
      unsigned long long lower = sh.before;
      if (f < 0) {  // the whole row does not reach the target (or masses below the unit): its last bin
        __syncthreads();
        int low = 0x7FFFFFFF;
        if (hi >= 0 && v0 > 0) low = hi;
        if (hi >= 1 && v1 > 0) low = hi - 1;
        if (low != 0x7FFFFFFF) atomicMax(&sh.found, 0x7FFFFFFF - low);
        __syncthreads();
        f = sh.found < 0 ? 0 : 0x7FFFFFFF - sh.found;
        lower = total - sh.hist[f];
      }
      prefix |= static_cast<uint32_t>(f) << shift;
      over += static_cast<double>(lower) * unit;
      __syncthreads();
    }
    tau = prefix;
    above = over;
  };

  bool listed = false;  // the list holds all that is kept
  int len = 0;
  if (cut) {
    // 3. the bin of the cut: the first at which the gathered counts or masses reach the target
    const double target = by_count ? static_cast<double>(top_k) : p * z * kUnit;
    const unsigned long long v0 = sh.hist[2 * tid], v1 = 2 * tid + 1 < kBins - 1 ? sh.hist[2 * tid + 1] : 0;
    if (tid == 0) sh.found = kBins - 1;
    unsigned long long total;
    const unsigned long long upto = block_scan(v0 + v1, sh.upart, total);
    const double b0 = static_cast<double>(upto - v0 - v1), b1 = static_cast<double>(upto - v1), b2 = static_cast<double>(upto);
    if ((tid == 0 || b0 < target) && b1 >= target) {
      sh.found = 2 * tid;
      sh.before = upto - v0 - v1;
    } else if (b1 < target && b2 >= target) {
      sh.found = 2 * tid + 1;
      sh.before = upto - v1;
    }
    __syncthreads();
    const int bin = sh.found;
    const double lower = static_cast<double>(sh.before) / kUnit;
    len = make_list(0, bin);
    if (len <= kList) {
      listed = true;
      sort_list(len);
      cut_list(len, by_count ? min(top_k, len) : len, by_count ? -1.0 : p * z);
    } else if (!by_count && bin < kBins - 1 && (len = make_list(bin, bin)) <= kList) {
      sort_list(len);
      cut_list(len, len, p * z - lower);
    } else {
      double above;
      if (by_count) {
        cut_digits(true, static_cast<double>(top_k), above);
        ties = top_k - static_cast<int>(above);
      }
      if (by_mass) {
        double target_mass = fmax(p * z, 1e-300), mass_above = 0.0;
        bool inside = true;  // the cut lies among the keys above top-k's last
        if (by_count) {
          double m = 0.0;
          row.each([&](int, const float (&x)[4]) EE_ALWAYS_INLINE {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (key_of(x[e]) > tau) m += mass_of(x[e]);
          });
          mass_above = block_sum(m);
          target_mass = fmax(p * (mass_above + ties * mass_of(value_of(tau))), 1e-300);
          inside = mass_above >= target_mass;
        }
        const int most = by_count && !inside ? ties : 0x7FFFFFFF;
        if (inside) cut_digits(false, target_mass, mass_above);
        const double q = mass_of(value_of(tau));
        const double need = q > 0.0 ? ceil((target_mass - mass_above) / q) : INFINITY;
        ties = need < 1.0 ? 1 : need < static_cast<double>(most) ? static_cast<int>(need) : most;
      }
    }
  }

  if (listed) {
    // the token from the list, which is in the order of ids
    double m[4], sum = 0.0, total;
    int tie = 0, n_tie;
#pragma unroll
    for (int e = 0; e < 4; ++e) tie += tid * 4 + e < len && sh.key[tid * 4 + e] == tau ? 1 : 0;
    int rank = block_scan(tie, sh.ipart[0], n_tie) - tie;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = tid * 4 + e;
      m[e] = 0.0;
      if (i < len) {
        const uint32_t k = sh.key[i];
        const bool in = k > tau || (k == tau && rank < ties);
        if (k == tau) ++rank;
        if (in) {
          m[e] = mass_of(value_of(k));
          if (m[e] < least) m[e] = 0.0;
        }
      }
      sum += m[e];
    }
    double upto = block_scan(sum, sh.part[0], total) - sum;
    const double goal = static_cast<double>(u) * total;
    // the first that passes the goal; if none does (u of 1 and more), the last that has mass
    int first = 0x7FFFFFFF, last = -1;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      upto += m[e];
      if (m[e] > 0.0) {
        last = tid * 4 + e;
        if (upto > goal && first == 0x7FFFFFFF) first = tid * 4 + e;
      }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      first = min(first, __shfl_xor(first, o));
      last = max(last, __shfl_xor(last, o));
    }
    if (lane == 0) {
      sh.ipart[0][wave] = first;
      sh.ipart[1][wave] = last;
    }
    __syncthreads();
    if (tid == 0) {
      for (int w = 0; w < kWaves; ++w) {
        first = min(first, sh.ipart[0][w]);
        last = max(last, sh.ipart[1][w]);
      }
      const int at = first != 0x7FFFFFFF ? first : last;
      finish(sh.id[at], mass_of(value_of(sh.key[at])) / total);
    }
    return;
  }

  // the token from the row: kept mass and ties of each wave, then the wave that has it
  double m = 0.0;
  int tie = 0;
  const double q = mass_of(value_of(tau));
  row.each([&](int, const float (&x)[4]) EE_ALWAYS_INLINE {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t k = key_of(x[e]);
      if (x[e] > -INFINITY) {
        if (k > tau) {
          const double v = mass_of(x[e]);
          m += v >= least ? v : 0.0;
        } else if (k == tau) {
          ++tie;
        }
      }
    }
  });
  m = wave_sum(m);
  tie = wave_sum(tie);
  if (lane == 0) {  // (slots that no wave may still be reading)
    sh.part[slot][wave] = m;
    sh.ipart[1][wave] = tie;
  }
  __syncthreads();
  const double tie_mass = q >= least ? q : 0.0;
  double total = 0.0, wave_mass[kWaves];
  int seen = 0, ties_before = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const int mine = min(max(ties - seen, 0), sh.ipart[1][w]);
    wave_mass[w] = sh.part[slot][w] + mine * tie_mass;
    if (w == wave) ties_before = seen;
    seen += sh.ipart[1][w];
    total += wave_mass[w];
  }
  const double goal = static_cast<double>(u) * total;
  int pick = -1;
  double start = 0.0, sum = 0.0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (wave_mass[w] > 0.0 && (pick < 0 || sum <= goal)) {
      pick = w;
      start = sum;
    }
    sum += wave_mass[w];
  }
  if (wave != pick) return;
  double before = start, chosen_mass = 0.0;
  int rank = ties_before, chosen = -1;
  bool done = false;
  row.each([&](int id, const float (&x)[4]) EE_ALWAYS_INLINE {
    if (done) return;
    int mine = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) mine += x[e] > -INFINITY && key_of(x[e]) == tau ? 1 : 0;
    const int t_upto = wave_scan(mine, lane);
    int r = rank + t_upto - mine;
    double v[4], s = 0.0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t k = key_of(x[e]);
      v[e] = 0.0;
      if (x[e] > -INFINITY) {
        if (k > tau) v[e] = mass_of(x[e]);
        if (k == tau && r++ < ties) v[e] = q;
        if (v[e] < least) v[e] = 0.0;
      }
      s += v[e];
    }
    double upto = wave_scan(s, lane);
    const double iter = __shfl(upto, 63);
    upto += before - s;
    int hit = -1, last = -1;
    double hit_mass = 0.0, last_mass = 0.0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      upto += v[e];
      if (v[e] > 0.0) {
        last = id + e;
        last_mass = v[e];
        if (hit < 0 && upto > goal) {
          hit = id + e;
          hit_mass = v[e];
        }
      }
    }
    const uint64_t hits = __ballot(hit >= 0), lasts = __ballot(last >= 0);
    if (hits != 0) {
      const int l = __builtin_ctzll(hits);
      chosen = __shfl(hit, l);
      chosen_mass = __shfl(hit_mass, l);
      done = true;
    } else if (lasts != 0) {
      const int l = 63 - __builtin_clzll(lasts);
      chosen = __shfl(last, l);
      chosen_mass = __shfl(last_mass, l);
    }
    before += iter;
    rank += __shfl(t_upto, 63);
  });
  if (lane == 0) finish(chosen, chosen_mass / total);
}

}  // namespace

size_t sample_workspace(int, int) { return 256; }

hipError_t launch_sample(bool f32, const SampleArgs &a, void *, hipStream_t stream) {
  if (a.n <= 0) return hipSuccess;
  EE_DISPATCH(f32, {
    hipLaunchKernelGGL((sample_kernel<T, 0>), dim3(a.n), dim3(kThreads), 0, stream, a);
  });
  return hipGetLastError();
}

}  // namespace ee
