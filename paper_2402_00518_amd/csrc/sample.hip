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
// One block a row, of 16 waves (8 for more than 256 rows that LDS does not hold, two blocks a
// CU).  Each wave holds a range of consecutive ids, so that everything in the order of ids is
// a prefix over waves, then inside one.
//   1. maximum (the row goes into LDS on the way, if it fits);
//   2. sum of masses, and in LDS a histogram over (max - x) / T in 2047 bins of
//      1/64 and one for the rest: of counts for top-k, else of masses for top-p.
//      (Masses as multiples of 2^-43, so that the order of the atomics does not show.)
//   3. the bin in which the cut lies; its tokens and all above it, in the order of
//      ids, as a list in LDS; that list's logits sorted, their masses cumulated:
//      the cut; the list cumulated in the order of ids: the token.
// Where the list would not fit, top-p alone lists the cut's bin only and walks the
// row once more; what is left (a cut in the last bin, thousands of equal logits)
// finds the cut by the digits of the logits' bits, three passes over the row.
// Of up to 64 long rows that LDS does not hold, several blocks a row take steps 1 and 2.
//
// What bounds it: not the bytes.  A row's block walks its ids two to five times with some 45
// cycles of a SIMD for 64 exponentials and their histogram entries, and between the walks
// stand scans, a sort and about thirty barriers: 18 to 29 us for one row of 32000, where
// reading it takes well under one.  512 rows of 128000 fp32 logits (262 MB, a pass over which
// takes 46 us) with top-p 0.95: 231 us.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ee_device.h"
#include "launch.h"

namespace ee {

namespace {

constexpr int kBins = 2048;
constexpr float kBinsPerUnit = 64.0f;
constexpr int kSmallList = 128;  // one wave does the rest of a row with so few tokens listed
constexpr int kSorted = 2 * kBins;
constexpr double kUnit = 0x1p43; // masses in the histogram: at most 2^20 tokens of mass 1

// e^y by its series, for the compiler.
constexpr double series_exp(double y) {
  double sum = 1.0, term = 1.0;
  for (int k = 1; k < 24; ++k) {
    term *= y / k;
    sum += term;
  }
  return sum;
}
constexpr double kLn2 = 0.69314718055994530942;
struct Pow2Table {
  double v[64];  // 2^(i / 64)
  constexpr Pow2Table() : v() {
    for (int i = 0; i < 64; ++i) v[i] = series_exp(kLn2 * i / 64);
  }
};
__device__ constexpr Pow2Table kPow2{};

// 2^(t / 64) for t <= 0, relative error 4e-14: t = k + r with k whole and |r| <= 1/2, so it is
// 2^(k div 64) table[k mod 64] e^(r ln 2 / 64), the last by its series up to the fourth power.
// 0 below 2^-1000 (without CLEAN: 2^-1000 there, for sums in which that does not matter).
// A sum over a vocabulary is these exponentials, so rounding and scaling are integer
// operations on a sum with 1.5 2^52 (with the conversion and ldexp instructions, and a series
// of twelve terms in place of the table, 32000 tokens took 13 us in one block, so 6).
template <bool CLEAN = true>
__device__ __forceinline__ double pow2_neg(double t, const double *table) {
  constexpr double c1 = kLn2 / 64, c2 = c1 * c1 / 2, c3 = c1 * c2 / 3, c4 = c1 * c3 / 4;
  const double c = fmax(t, -64000.0), shifted = c + 0x1.8p52, r = c - (shifted - 0x1.8p52);
  const int k = static_cast<int>(static_cast<uint32_t>(__builtin_bit_cast(uint64_t, shifted)));
  const double p = __builtin_fma(__builtin_fma(__builtin_fma(__builtin_fma(c4, r, c3), r, c2), r, c1), r, 1.0);
  const uint64_t b = __builtin_bit_cast(uint64_t, p * table[k & 63]);
  const double v = __builtin_bit_cast(double, b + (static_cast<uint64_t>(static_cast<uint32_t>((k >> 6) << 20)) << 32));
  return CLEAN && !(t >= -64000.0) ? 0.0 : v;
}
__device__ __forceinline__ unsigned long long units_of(double mass) {  // of a mass <= 1
  return __builtin_bit_cast(uint64_t, __builtin_fma(mass, kUnit, 0x1p52)) & 0xFFFFFFFFFFFFFull;
}

// Bits that order as the values do; -0 counts as 0.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) {
  return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key);
}

// One step of a prefix sum: the value that a DPP pattern brings to each lane, 0 where
// it brings none.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, ROWS, 0xF, false));
}
template <int CTRL, int ROWS, typename V>
__device__ __forceinline__ V dpp_value(V v) {
  if constexpr (sizeof(V) == 4) {
    return __builtin_bit_cast(V, dpp<CTRL, ROWS>(__builtin_bit_cast(uint32_t, v)));
  } else {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint64_t lo = dpp<CTRL, ROWS>(static_cast<uint32_t>(b)), hi = dpp<CTRL, ROWS>(static_cast<uint32_t>(b >> 32));
    return __builtin_bit_cast(V, lo | hi << 32);
  }
}
// Inclusive prefix over the wave: within rows of 16 lanes, then the last lane of row 0
// (and 2) to row 1 (3), and of the first two rows to the others.
template <typename V>
__device__ __forceinline__ V wave_scan(V v) {
  v += dpp_value<0x111, 0xF>(v);
  v += dpp_value<0x112, 0xF>(v);
  v += dpp_value<0x114, 0xF>(v);
  v += dpp_value<0x118, 0xF>(v);
  v += dpp_value<0x142, 0xA>(v);
  v += dpp_value<0x143, 0xC>(v);
  return v;
}
template <typename V>
__device__ __forceinline__ V of_lane(V v, int lane) {  // lane: the same in all
  if constexpr (sizeof(V) == 4) {
    return __builtin_bit_cast(V, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
  } else {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint64_t lo = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(b), lane)),
                   hi = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(b >> 32), lane));
    return __builtin_bit_cast(V, lo | hi << 32);
  }
}
template <typename V>
__device__ __forceinline__ V wave_sum(V v) {
  return of_lane(wave_scan(v), 63);
}

// LIST: tokens that the list holds, a multiple of 64 for each wave.
template <int LIST>
struct Shared {
  union {
    unsigned long long hist[kBins];
    uint32_t sorted[kSorted];
  };
  uint32_t key[LIST];
  int32_t id[LIST];
  double table[64];
  double part[2][16];
  int ipart[2][16];
  unsigned long long upart[16];
  int found, n_sub;
  unsigned long long before;
};

// Beside a row in LDS the list is short; without one it is as long as two blocks a CU allow.
constexpr int list_of(bool cached) { return cached ? 2048 : 6144; }
constexpr size_t shared_bytes(bool cached) { return ((cached ? sizeof(Shared<list_of(true)>) : sizeof(Shared<list_of(false)>)) + 15) / 16 * 16; }

template <typename T> struct Quad;
template <> struct Quad<float> { using type = f32x4_t; };
template <> struct Quad<bf16_t> { using type = u32x2_t; };

// The logits of a row, four ids a lane and step.  CACHED: in LDS (tokens that are not
// allowed as -infinity), else read from memory again by every pass, four steps'
// loads at once (with one, a pass over 128000 tokens waited on memory for 31 of them
// in turn).
template <typename T, bool CACHED>
struct Row {
  using Q = typename Quad<T>::type;
  const T *p;
  const uint32_t *allowed;
  Q *cache;
  int vocab, first, last;  // ids of the wave: [first, last)
  int lane;
  mutable bool stop = false;  // set by a pass's function: no further step

  __device__ __forceinline__ static void unpack(const Q &v, float (&x)[4]) {
    if constexpr (std::is_same<T, float>::value) {
      static_for<4>([&](auto e) EE_ALWAYS_INLINE { x[decltype(e)::value] = v[decltype(e)::value]; });
    } else {
      x[0] = __uint_as_float(v[0] << 16);
      x[1] = __uint_as_float(v[0] & 0xFFFF0000u);
      x[2] = __uint_as_float(v[1] << 16);
      x[3] = __uint_as_float(v[1] & 0xFFFF0000u);
    }
  }
  __device__ __forceinline__ static Q pack(const float (&x)[4]) {
    if constexpr (std::is_same<T, float>::value)
      return Q{x[0], x[1], x[2], x[3]};
    else  // (values that are bf16 already)
      return Q{(__float_as_uint(x[0]) >> 16) | (__float_as_uint(x[1]) & 0xFFFF0000u),
               (__float_as_uint(x[2]) >> 16) | (__float_as_uint(x[3]) & 0xFFFF0000u)};
  }
  // Four ids from `id` < vocab on; past the vocabulary anything.
  __device__ __forceinline__ Q load(int id) const {
    if (id + 4 <= vocab) return load_any<Q>(p + id);
    float x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = to_f32(p[min(id + e, vocab - 1)]);
    return pack(x);
  }
  // -infinity for what is not allowed (bit e of w 0) or past the vocabulary.
  __device__ __forceinline__ void mask(int id, uint32_t w, float (&x)[4]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (((w >> e) & 1) == 0 || id + e >= vocab) x[e] = -INFINITY;
  }
  // f(first id, values) for every four ids of this lane, in the order of ids.  Every
  // lane of the wave takes part (ids past the last have -infinity).  FILL: the first pass.
  template <bool FILL = false, class F>
  __device__ __forceinline__ void each(F &&f) const {
    if constexpr (CACHED && !FILL) {
      for (int i = first; i < last && !stop; i += 256) {
        const int id = i + lane * 4;
        float x[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        if (id < last) unpack(cache[id >> 2], x);
        f(id, x);
      }
    } else {
      constexpr int U = 4;
      for (int i = first; i < last && !stop; i += 256 * U) {
        Q raw[U];
        uint32_t ok[U];
#pragma unroll
        for (int b = 0; b < U; ++b) {
          const int id = i + b * 256 + lane * 4;
          ok[b] = 0;
          if (id < last) {
            raw[b] = load(id);
            ok[b] = allowed != nullptr ? allowed[id >> 5] >> (id & 31) : 15u;  // (id is a multiple of 4)
          }
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int b = 0; b < U; ++b) {
          const int id = i + b * 256 + lane * 4;
          if (i + b * 256 < last && !stop) {
            float x[4];
            unpack(raw[b], x);
            mask(id, ok[b], x);
            if (CACHED && id < last) cache[id >> 2] = pack(x);
            f(id, x);
          }
          __builtin_amdgcn_sched_barrier(0);  // (one group at a time: mixed, they need more registers than there are)
        }
      }
    }
  }
};

// What a row's parameters ask for.
struct RowPlan {
  float temp, top_p, min_p, u;
  int top_k;
  bool valid, greedy, by_count, by_mass, cut, want_conf, same, need_z, need_z1;
  double c1, ct;   // 64 log2(e), and that over the temperature
  double least, p; // min-p and top-p
  float bscale;

  __device__ __forceinline__ RowPlan(const SampleArgs &a, int n) {
    temp = a.temperature != nullptr ? a.temperature[n] : 1.0f;
    top_k = a.top_k != nullptr ? a.top_k[n] : 0;
    top_p = a.top_p != nullptr ? a.top_p[n] : 1.0f;
    min_p = a.min_p != nullptr ? a.min_p[n] : 0.0f;
    u = a.uniform[n];
  }
  // (apart, as what is loaded is waited for here: before a row's own loads that took 0.8 us)
  __device__ __forceinline__ void derive(const SampleArgs &a) {
    valid = temp == temp && top_p == top_p && min_p == min_p && u == u;
    greedy = !(temp > 0.0f);
    by_count = !greedy && top_k > 0 && top_k < a.vocab;
    by_mass = !greedy && top_p < 1.0f;
    cut = by_count || by_mass;
    want_conf = a.confidence != nullptr || a.exit_flag != nullptr;
    // (an infinite temperature still sends -infinity to mass 0)
    c1 = 64.0 / kLn2;
    ct = greedy ? c1 : fmax(c1 / static_cast<double>(temp), 1e-300);
    same = ct == c1;  // one mass serves both
    least = min_p > 0.0f ? (min_p < 1.0f ? static_cast<double>(min_p) : 1.0) : 0.0;
    p = top_p > 0.0f ? static_cast<double>(top_p) : 0.0;
    need_z = (by_mass && !by_count) || (want_conf && same) || (!cut && !greedy && least == 0.0);
    need_z1 = want_conf && !same;
    bscale = static_cast<float>(kBinsPerUnit / (greedy ? 1.0 : static_cast<double>(temp)));
  }
  __device__ __forceinline__ int bin_of(float x, float mx) const {  // monotone in x
    const float b = (mx - x) * bscale;
    return b < static_cast<float>(kBins - 1) ? static_cast<int>(b) : kBins - 1;
  }
};

// Sums of masses at both temperatures over the wave's share of the row, and the histogram.
template <class R>
__device__ __forceinline__ void sum_masses(const R &row, const RowPlan &plan, float mx, const double *table,
                                           unsigned long long *hist, double &z, double &z1) {
  const double dmx = mx;
  auto pass = [&](auto with_z, auto with_z1, auto with_hist) EE_ALWAYS_INLINE {
    row.each([&](int, const float (&x)[4]) EE_ALWAYS_INLINE {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const double d = static_cast<double>(x[e]) - dmx;
        double m = 0.0;
        if constexpr (decltype(with_z)::value) {
          // (exact zeros where the sums are used to find the token)
          m = pow2_neg<!decltype(with_hist)::value>(d * plan.ct, table);
          z += m;
        }
        if constexpr (decltype(with_z1)::value) z1 += pow2_neg<false>(d * plan.c1, table);
        if constexpr (decltype(with_hist)::value) {
          const int b = plan.bin_of(x[e], mx);
          if (b < kBins - 1) atomicAdd(&hist[b], plan.by_count ? 1ull : units_of(m));
        }
      }
    });
  };
  with_flag(plan.need_z, [&](auto f) EE_ALWAYS_INLINE {
    with_flag(plan.need_z1, [&](auto g) EE_ALWAYS_INLINE { with_flag(plan.cut, [&](auto h) EE_ALWAYS_INLINE { pass(f, g, h); }); });
  });
}

// Few rows leave most CUs idle while one block of each walks a long row: the maximum and the
// sums with the histogram are then taken by `splits` blocks a row, in two launches ahead.
struct Part {
  float max;
  int bad;
  double z, z1;
};
constexpr int kPartWaves = 4;

__device__ __forceinline__ int first_of_part(int vocab, int split, int splits) {  // (whole steps of 256 ids)
  return static_cast<int>(static_cast<int64_t>((vocab + 255) / 256) * split / splits) * 256;
}

template <typename R>
__device__ __forceinline__ void share_part(R &row, const SampleArgs &a, int split, int splits, int wave) {
  const int from = first_of_part(a.vocab, split, splits), mine = (first_of_part(a.vocab, split + 1, splits) - from) / 256;
  row.first = min(from + mine * wave / kPartWaves * 256, a.vocab);
  row.last = min(from + mine * (wave + 1) / kPartWaves * 256, a.vocab);
}

template <typename T>
__device__ __forceinline__ Row<T, false> global_row(const SampleArgs &a, int n, int lane) {
  Row<T, false> row;
  row.p = static_cast<const T *>(a.logits) + n * a.ld;
  row.allowed = a.allowed != nullptr ? a.allowed + n * a.allowed_ld : nullptr;
  row.cache = nullptr;
  row.vocab = a.vocab;
  row.lane = lane;
  return row;
}

template <typename T>
__global__ __launch_bounds__(64 * kPartWaves) void part_max_kernel(SampleArgs a, Part *parts) {
  __shared__ float maxes[kPartWaves];
  __shared__ int bads[kPartWaves];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = blockIdx.y;
  Row<T, false> row = global_row<T>(a, n, lane);
  share_part(row, a, blockIdx.x, gridDim.x, wave);
  float mx = -INFINITY;
  bool bad = false;
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
    maxes[wave] = mx;
    bads[wave] = bad;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kPartWaves; ++w) {
      mx = fmaxf(mx, maxes[w]);
      bad |= bads[w] != 0;
    }
    Part &p = parts[n * gridDim.x + blockIdx.x];
    p.max = mx;
    p.bad = bad;
  }
}

// The row's maximum, and whether it has a NaN, from its parts (a part a lane).
__device__ __forceinline__ float max_of_parts(const Part *parts, int splits, int lane, bool &bad) {
  float mx = -INFINITY;
  for (int i = lane; i < splits; i += 64) {
    mx = fmaxf(mx, parts[i].max);
    bad |= parts[i].bad != 0;
  }
  bad = __any(bad);
  return warp_max(mx);
}

template <typename T>
__global__ __launch_bounds__(64 * kPartWaves) void part_sum_kernel(SampleArgs a, Part *parts, unsigned long long *hists) {
  __shared__ unsigned long long hist[kBins];
  __shared__ double table[64];
  __shared__ double sums[2][kPartWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = blockIdx.y;
  const int splits = gridDim.x, at = n * splits + blockIdx.x;
  RowPlan plan(a, n);
  plan.derive(a);
  bool bad = !plan.valid;
  const float mx = max_of_parts(parts + n * splits, splits, lane, bad);
  if (bad || mx == INFINITY || mx == -INFINITY || !(plan.need_z || plan.need_z1 || plan.cut)) return;
  for (int i = tid; i < kBins; i += 64 * kPartWaves) hist[i] = 0;
  if (tid < 64) table[tid] = kPow2.v[tid];
  __syncthreads();
  Row<T, false> row = global_row<T>(a, n, lane);
  share_part(row, a, blockIdx.x, splits, wave);
  double z = 0.0, z1 = 0.0;
  sum_masses(row, plan, mx, table, hist, z, z1);
  z = wave_sum(z);
  z1 = wave_sum(z1);
  if (lane == 0) {
    sums[0][wave] = z;
    sums[1][wave] = z1;
  }
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < kPartWaves; ++w) {
      z += sums[0][w];
      z1 += sums[1][w];
    }
    parts[at].z = z;
    parts[at].z1 = z1;
  }
  if (plan.cut)
    for (int i = tid; i < kBins; i += 64 * kPartWaves) hists[static_cast<int64_t>(at) * kBins + i] = hist[i];
}

// W: waves of the block.  splits > 0: steps 1 and 2 have been taken by the kernels above.
template <typename T, bool CACHED, int W>
__global__ __launch_bounds__(64 * W, 4) void sample_kernel(SampleArgs a, const Part *parts, const unsigned long long *hists,
                                                           int row_splits) {
  const int splits = CACHED ? 0 : row_splits;
  constexpr int kThreads = 64 * W, kList = list_of(CACHED);
  extern __shared__ __attribute__((aligned(16))) char smem[];
  auto &sh = *reinterpret_cast<Shared<kList> *>(smem);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = blockIdx.x;
  RowPlan plan(a, n);
  Row<T, CACHED> row;
  row.cache = reinterpret_cast<typename Quad<T>::type *>(smem + shared_bytes(CACHED));
  row.p = static_cast<const T *>(a.logits) + n * a.ld;
  row.allowed = a.allowed != nullptr ? a.allowed + n * a.allowed_ld : nullptr;
  row.vocab = a.vocab;
  // the waves' shares of ids [from, to), whole steps of 256 ids each
  auto share = [&](int from, int to) EE_ALWAYS_INLINE {
    const int chunk = (to - from + W * 256 - 1) / (W * 256) * 256;
    row.first = min(from + wave * chunk, to);
    row.last = min(row.first + chunk, to);
    return chunk;
  };
  const int chunk = share(0, a.vocab);
  row.lane = lane;

  int slot = 0;  // block sums alternate between two slots, one barrier each
  auto block_sum = [&](double v) EE_ALWAYS_INLINE {
    v = wave_sum(v);
    if (lane == 0) sh.part[slot][wave] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < W; ++w) s += sh.part[slot][w];
    slot ^= 1;
    return s;
  };

  // 1. the maximum, and whether the row has a distribution at all
  float mx = -INFINITY;
  bool bad = false;
  if (splits > 0) {
    plan.derive(a);
    parts += n * splits;
    hists += static_cast<int64_t>(n) * splits * kBins;
    mx = max_of_parts(parts, splits, lane, bad);
    if (plan.cut) {
      for (int i = tid; i < kBins; i += kThreads) {
        unsigned long long h = 0;
        if (!bad && mx < INFINITY && mx > -INFINITY) {
          for (int q = 0; q < splits; q += 8) {  // (eight loads in flight)
            unsigned long long v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = q + e < splits ? hists[static_cast<int64_t>(q + e) * kBins + i] : 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) h += v[e];
          }
        }
        sh.hist[i] = h;
      }
    }
  } else {
    for (int i = tid; i < kBins; i += kThreads) sh.hist[i] = 0;  // (closed by the barrier below, as is the table)
  }
  if (tid < 64) sh.table[tid] = kPow2.v[tid];
  if (splits == 0) {
    row.template each<true>([&](int, const float (&x)[4]) EE_ALWAYS_INLINE {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        mx = fmaxf(mx, x[e]);
        bad |= x[e] != x[e];
      }
    });
    mx = warp_max(mx);
    plan.derive(a);
  }
  bad = __any(bad) || !plan.valid;
  if (lane == 0) {
    sh.part[0][wave] = mx;
    sh.ipart[0][wave] = bad;
  }
  __syncthreads();
  bad = false;
  mx = -INFINITY;
#pragma unroll
  for (int w = 0; w < W; ++w) {
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
  const int top_k = plan.top_k;
  const float u = plan.u;
  const bool by_count = plan.by_count, by_mass = plan.by_mass, cut = plan.cut;
  const double dmx = mx, least = plan.least, p = plan.p;
  const float bscale = plan.bscale;
  auto mass_of = [&](float x) EE_ALWAYS_INLINE { return pow2_neg((static_cast<double>(x) - dmx) * plan.ct, sh.table); };
  auto bin_of = [&](float x) EE_ALWAYS_INLINE { return plan.bin_of(x, mx); };

  // 2. sums of masses; the histogram
  double z = 0.0, z1 = 0.0;
  if (splits > 0) {
    if (plan.need_z || plan.need_z1 || cut) {
      for (int q = lane; q < splits; q += 64) {
        z += parts[q].z;
        z1 += parts[q].z1;
      }
      z = wave_sum(z);
      z1 = wave_sum(z1);
    }
  } else if (plan.need_z || plan.need_z1 || cut) {
    sum_masses(row, plan, mx, sh.table, sh.hist, z, z1);
    z = block_sum(z);  // (its barrier also closes the histogram)
    if (plan.need_z1) z1 = block_sum(z1);
  }
  if (plan.want_conf && tid == 0) {
    const float conf = static_cast<float>(1.0 / (plan.same ? z : z1));
    if (a.confidence != nullptr) a.confidence[n] = conf;
    if (a.exit_flag != nullptr) a.exit_flag[n] = conf > a.threshold ? 1 : 0;
  }

  auto finish = [&](int token, double prob) EE_ALWAYS_INLINE {
    a.token[n] = token;
    if (a.prob != nullptr) a.prob[n] = static_cast<float>(prob);
  };
  if (plan.greedy) {
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
      for (int w = 0; w < W; ++w) at = min(at, sh.ipart[1][w]);
      finish(at, 1.0);
    }
    return;
  }

  // What is kept: keys above `tau`, and the first `ties` of those equal to it; mass
  // at least `least`.  The largest logit's first token always is.
  uint32_t tau = 0;
  int ties = 0x7FFFFFFF;

  // Inclusive prefix of a value a thread over the block; returns it and the total.
  auto block_scan = [&](auto v, auto *parts, auto &total) EE_ALWAYS_INLINE {
    using V = decltype(v);
    const V mine = wave_scan(v);
    if (lane == 63) parts[wave] = mine;
    __syncthreads();
    V before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const V t = parts[w];
      if (w < wave) before += t;
      total += t;
    }
    __syncthreads();
    return before + mine;
  };
  struct Block {};
  struct Wave {};
  // The same over the block or, where the first wave is alone, over that wave.
  auto scan = [&](auto scope, auto v, auto &total) EE_ALWAYS_INLINE {
    using V = decltype(v);
    if constexpr (std::is_same<decltype(scope), Block>::value) {
      if constexpr (std::is_same<V, double>::value)
        return block_scan(v, sh.part[0], total);
      else
        return block_scan(v, sh.ipart[0], total);
    } else {
      const V mine = wave_scan(v);
      total = of_lane(mine, 63);
      return mine;
    }
  };
  auto sync = [&](auto scope) EE_ALWAYS_INLINE {
    if constexpr (std::is_same<decltype(scope), Block>::value) {
      __syncthreads();
    } else {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  };

  // Tokens for which in(x) holds, in the order of ids, as the list; returns how many
  // there are (the list holds them if no more than it has room for).  `give_up`: as soon as
  // a wave has more than its part of the list, there count as too many.
  bool again = false;  // in() is asked a second time
  auto make_list = [&](bool give_up, auto &&in) EE_ALWAYS_INLINE {
    again = false;
    constexpr int SEG = kList / W, PER = SEG / 64;
    static_assert(PER * 64 * W == kList, "whole entries a lane");
    // The wave's from `at` on, as long as there is room up to `end`; returns how many.
    auto write = [&](int at, int end) EE_ALWAYS_INLINE {
      const int begin = at;
      row.each([&](int id, const float (&x)[4]) EE_ALWAYS_INLINE {
        const bool b0 = in(x[0]), b1 = in(x[1]), b2 = in(x[2]), b3 = in(x[3]);
        if (__any(b0 || b1 || b2 || b3)) {
          const bool b[4] = {b0, b1, b2, b3};
          const int upto = wave_scan(static_cast<int>(b0) + b1 + b2 + b3);
          int o = at + upto - (static_cast<int>(b0) + b1 + b2 + b3);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (b[e]) {
              if (o < end) {
                sh.key[o] = key_of(x[e]);
                sh.id[o] = id + e;
              }
              ++o;
            }
          }
          at += of_lane(upto, 63);
          row.stop = give_up && at > end;
        }
      });
      const int count = row.stop ? kList + 1 : at - begin;
      row.stop = false;
      return count;
    };
    // Each wave writes into a part of its own; the parts are then pushed together.
    const int count = write(wave * SEG, (wave + 1) * SEG);
    if (lane == 0) sh.ipart[0][wave] = count;
    __syncthreads();
    int at = 0, total = 0, most = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const int c = sh.ipart[0][w];
      if (w < wave) at += c;
      total += c;
      most = max(most, c);
    }
    if (total <= kList) {
      if (most <= SEG) {
        uint32_t k[PER];
        int d[PER];
#pragma unroll
        for (int e = 0; e < PER; ++e) {
          k[e] = sh.key[wave * SEG + e * 64 + lane];
          d[e] = sh.id[wave * SEG + e * 64 + lane];
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < PER; ++e) {
          if (e * 64 + lane < count) {
            sh.key[at + e * 64 + lane] = k[e];
            sh.id[at + e * 64 + lane] = d[e];
          }
        }
      } else {
        __syncthreads();  // (a part may reach into the next, whose wave writes it again)
        again = true;
        write(at, at + count);
      }
    }
    __syncthreads();
    return total;
  };

  // sh.sorted[0 .. len) by falling value: a bitonic network over the next power of two, whose
  // steps need the block only where they reach past a wave's own 128 keys.
  auto sort_block = [&](int len) EE_ALWAYS_INLINE {
    int size = 128;
    while (size < len) size <<= 1;
    for (int i = len + tid; i < size; i += kThreads) sh.sorted[i] = 0;
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
        const int next = j > 1 ? j >> 1 : k;
        if (j > 64 || next > 64)
          __syncthreads();
        else
          sync(Wave{});
      }
    }
    __syncthreads();
  };
  // The same for up to 128 keys of the list, by one wave: for each those before it counted.
  auto sort_wave = [&](int len) EE_ALWAYS_INLINE {
    for (int i = lane; i < len; i += 64) {
      const uint32_t mine = sh.key[i];
      int rank = 0;
      for (int j = 0; j < len; ++j) {
        const uint32_t k = sh.key[j];
        rank += k > mine || (k == mine && j < i) ? 1 : 0;
      }
      sh.sorted[rank] = mine;
    }
    sync(Wave{});
  };

  // tau and ties from `len` sorted keys: of the first `most`, those before which less than the
  // target has gathered (share_of < 0: of p times the mass of the first `most`; else share_of).
  auto cut_sorted = [&](auto scope, int len, int most, double share_of) EE_ALWAYS_INLINE {
    constexpr int PER = std::is_same<decltype(scope), Block>::value ? kSorted / kThreads : kSmallList / 64;
    double m[PER], sum = 0.0, total;
    uint32_t k[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const int i = tid * PER + e;
      k[e] = i < len ? sh.sorted[i] : 0;
      m[e] = by_mass && i < most ? mass_of(value_of(k[e])) : 0.0;
      sum += m[e];
    }
    double before = scan(scope, sum, total) - sum;
    const double target = !by_mass ? INFINITY : share_of < 0.0 ? p * total : share_of;
    int keep = 0;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const int i = tid * PER + e;
      if (i < most && (i == 0 || before < target)) ++keep;
      before += m[e];
    }
    int kept;
    scan(scope, keep, kept);
    tau = sh.sorted[kept - 1];
    int above = 0, n_above;
#pragma unroll
    for (int e = 0; e < PER; ++e) above += tid * PER + e < kept && k[e] > tau ? 1 : 0;
    scan(scope, above, n_above);
    ties = kept - n_above;
  };

  // The token from a list that holds all that is kept.
  auto pick_listed = [&](auto scope, int len) EE_ALWAYS_INLINE {
    constexpr bool BLOCK = std::is_same<decltype(scope), Block>::value;
    constexpr int PER = BLOCK ? kList / kThreads : kSmallList / 64;
    double m[PER], sum = 0.0, total;
    int tie = 0, n_tie;
#pragma unroll
    for (int e = 0; e < PER; ++e) tie += tid * PER + e < len && sh.key[tid * PER + e] == tau ? 1 : 0;
    int rank = scan(scope, tie, n_tie) - tie;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const int i = tid * PER + e;
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
    double upto = scan(scope, sum, total) - sum;
    const double goal = static_cast<double>(u) * total;
    // the first that passes the goal; if none does (u of 1 and more), the last that has mass
    int first = 0x7FFFFFFF, last = -1;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      upto += m[e];
      if (m[e] > 0.0) {
        last = tid * PER + e;
        if (upto > goal && first == 0x7FFFFFFF) first = tid * PER + e;
      }
    }
    const uint64_t firsts = __ballot(first != 0x7FFFFFFF), lasts = __ballot(last >= 0);
    first = firsts != 0 ? of_lane(first, __builtin_ctzll(firsts)) : 0x7FFFFFFF;
    last = lasts != 0 ? of_lane(last, 63 - __builtin_clzll(lasts)) : -1;
    if constexpr (BLOCK) {
      if (lane == 0) {
        sh.ipart[0][wave] = first;
        sh.ipart[1][wave] = last;
      }
      __syncthreads();
      if (tid != 0) return;
      for (int w = 0; w < W; ++w) {
        first = min(first, sh.ipart[0][w]);
        last = max(last, sh.ipart[1][w]);
      }
    }
    if (tid == 0) {
      const int at = first != 0x7FFFFFFF ? first : last;
      finish(sh.id[at], mass_of(value_of(sh.key[at])) / total);
    }
  };

  // tau by the digits of the keys: the largest key with at least `target` tokens, or
  // mass, at it and above; `above` is what lies above it.
  auto cut_digits = [&](bool count, double target, double &above) EE_ALWAYS_INLINE {
    uint32_t prefix = 0;
    double over = 0.0;
    int shift = 32;
    for (int d = 0; d < 3; ++d) {
      const uint32_t mask = shift == 32 ? 0 : ~0u << shift;
      const int nb = d < 2 ? 2048 : 1024;
      shift -= d < 2 ? 11 : 10;
      for (int i = tid; i < nb; i += kThreads) sh.hist[i] = 0;
      __syncthreads();
      row.each([&](int, const float (&x)[4]) EE_ALWAYS_INLINE {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t key = key_of(x[e]);
          if (x[e] > -INFINITY && (key & mask) == (prefix & mask))
            atomicAdd(&sh.hist[(key >> shift) & (nb - 1)], count ? 1ull : units_of(mass_of(x[e])));
        }
      });
      __syncthreads();
      // bins from the top: thread t has the PB bins from nb - 1 - PB t down
      constexpr int PB = kBins / kThreads;
      const int hi = nb - 1 - PB * tid;
      unsigned long long v[PB], sum = 0, total;
      int low = 0x7FFFFFFF;
#pragma unroll
      for (int e = 0; e < PB; ++e) {
        v[e] = hi - e >= 0 ? sh.hist[hi - e] : 0;
        sum += v[e];
        if (v[e] > 0) low = hi - e;
      }
      if (tid == 0) sh.found = -1;
      const double unit = count ? 1.0 : 1.0 / kUnit;
      unsigned long long before = block_scan(sum, sh.upart, total) - sum;
#pragma unroll
      for (int e = 0; e < PB; ++e) {
        if (v[e] > 0 && over + static_cast<double>(before) * unit < target && over + static_cast<double>(before + v[e]) * unit >= target) {
          sh.found = hi - e;
          sh.before = before;
        }
        before += v[e];
      }
      __syncthreads();
      int f = sh.found;
      unsigned long long lower = sh.before;
      if (f < 0) {  // the whole row does not reach the target (or masses below the unit): its last bin
        __syncthreads();
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

  bool in_bin = false;
  double above_bin = 0.0;
  if (cut) {
    // 3. the bin of the cut: the first at which the gathered counts or masses reach the target
    constexpr int PB = kBins / kThreads;
    const double target = by_count ? static_cast<double>(top_k) : p * z * kUnit;
    unsigned long long v[PB], sum = 0, total;
#pragma unroll
    for (int e = 0; e < PB; ++e) {
      v[e] = tid * PB + e < kBins - 1 ? sh.hist[tid * PB + e] : 0;
      sum += v[e];
    }
    if (tid == 0) sh.found = kBins - 1;
    unsigned long long before = block_scan(sum, sh.upart, total) - sum;
#pragma unroll
    for (int e = 0; e < PB; ++e) {
      const int b = tid * PB + e;
      if ((b == 0 || static_cast<double>(before) < target) && static_cast<double>(before + v[e]) >= target && b < kBins - 1) {
        sh.found = b;
        sh.before = before;
      }
      before += v[e];
    }
    __syncthreads();
    const int bin = sh.found;
    const double lower = static_cast<double>(sh.before) / kUnit;
    // All that lies in the bin and above, by one comparison: the bin's lower edge,
    // moved down past what its rounding may hide (a few tokens more do no harm).
    const float edge = (mx - static_cast<float>(bin + 1) / bscale), from = edge - 1e-5f * (fabsf(edge) + fabsf(mx));
    const bool all = bin == kBins - 1 || !(from > -INFINITY);
    // How many the list would have at least: counted, or from the masses, of which no token of
    // bin b has more than e^(-b / 64).  (512 rows of 128000: top-p 0.95 231 us, trying first 239;
    // top-k 20000 333, so 375.)
    bool too_many = false;
    if (bin < kBins - 1) {
      double tokens = static_cast<double>(sh.before + sh.hist[bin]);
      if (!by_count) {
        float mine = 0.0f;
#pragma unroll
        for (int e = 0; e < PB; ++e)
          if (tid * PB + e <= bin) mine += static_cast<float>(v[e]) * exp2f((tid * PB + e) * (1.0f / (kBinsPerUnit * static_cast<float>(kLn2))));
        tokens = block_sum(static_cast<double>(mine)) / kUnit;
      }
      too_many = tokens > kList * 1.001;
    }
    int len = too_many ? kList + 1 : make_list(!by_count, [&](float x) EE_ALWAYS_INLINE { return all ? x > -INFINITY : x >= from; });
    if (len <= kSmallList) {
      if (wave == 0) {
        sort_wave(len);
        cut_sorted(Wave{}, len, by_count ? min(top_k, len) : len, by_count ? -1.0 : p * z);
        pick_listed(Wave{}, len);
      }
      return;
    }
    if (len <= kList) {
      // With one criterion only the cut's bin has to be sorted: what lies above it is known.
      const bool whole = by_count && by_mass, tail = bin == kBins - 1;
      const int above_bin_count = static_cast<int>(sh.before);
      if (tid == 0) sh.n_sub = 0;
      __syncthreads();
      for (int i = tid; i < len; i += kThreads) {
        const uint32_t k = sh.key[i];
        if (whole || tail || bin_of(value_of(k)) == bin) {
          const int at = atomicAdd(&sh.n_sub, 1);  // (in any order: they are sorted next)
          if (at < kSorted) sh.sorted[at] = k;
        }
      }
      __syncthreads();
      const int n_sub = sh.n_sub;
      if (n_sub <= kSorted) {
        sort_block(n_sub);
        if (whole || tail)
          cut_sorted(Block{}, n_sub, by_count ? min(top_k, n_sub) : n_sub, by_count ? -1.0 : p * z);
        else
          cut_sorted(Block{}, n_sub, by_count ? min(top_k - above_bin_count, n_sub) : n_sub, p * z - lower);
        pick_listed(Block{}, len);
        return;
      }
    }
    if (!by_count && bin < kBins - 1) {
      // The bin's tokens, and on the way the mass that each wave has above it: its logits
      // gather in a queue (where the sorted list comes later) and are taken 64 at a time, as
      // few lanes have one (all lanes at every step: 60 us for 128000 tokens, so 30).
      float *queue = reinterpret_cast<float *>(sh.sorted) + wave * (kSorted / W);
      int queued = 0;
      len = make_list(false, [&](float x) EE_ALWAYS_INLINE {
        const int b = x > -INFINITY ? bin_of(x) : kBins;
        const bool above = b < bin && !again;
        const uint64_t mask = __ballot(above);
        if (mask != 0) {
          if (above)
            queue[queued + __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(mask >> 32),
                                                     __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(mask), 0))] = x;
          queued += __builtin_popcountll(mask);
          if (queued >= 64) {
            sync(Wave{});
            const float v = queue[lane], rest = queue[64 + lane];
            above_bin += mass_of(v);
            sync(Wave{});
            queued -= 64;
            if (lane < queued) queue[lane] = rest;
          }
        }
        return b == bin;
      });
      sync(Wave{});
      if (lane < queued) above_bin += mass_of(queue[lane]);
      __syncthreads();  // (the queues are overwritten next)
      in_bin = len <= min(kList, kSorted);
    }
    if (in_bin) {
      for (int i = tid; i < len; i += kThreads) sh.sorted[i] = sh.key[i];
      sort_block(len);
      cut_sorted(Block{}, len, len, p * z - lower);
      above_bin = wave_sum(above_bin);
      // the list is in the order of ids: the wave's part of it, and what of it is kept
      int lo = 0, hi = 0;
      for (int i = lane; i < len; i += 64) {
        lo += sh.id[i] < row.first ? 1 : 0;
        hi += sh.id[i] < row.last ? 1 : 0;
      }
      lo = wave_sum(lo);
      hi = wave_sum(hi);
      double m = 0.0;
      int tie = 0;
      for (int i = lo + lane; i < hi; i += 64) {
        const uint32_t k = sh.key[i];
        if (k > tau) m += mass_of(value_of(k));
        if (k == tau) ++tie;
      }
      m = wave_sum(m);
      tie = wave_sum(tie);
      if (lane == 0) {
        sh.part[0][wave] = above_bin + m;
        sh.ipart[0][wave] = tie;
      }
      __syncthreads();
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

  // The token from the row: each wave's kept mass, the wave in whose share the goal lies,
  // then the same once more with that share divided among all waves, and that wave's ids one
  // by one.
  const double q = mass_of(value_of(tau)), tie_mass = q >= least ? q : 0.0;
  // What the waves (or the parts taken ahead) have is known from step 2 (slot 1, no ties), or
  // from the list of the cut's bin, unless min-p takes some of it away again.
  const bool from_sums = !cut && least == 0.0, from_list = in_bin && least == 0.0;
  double before = 0.0, goal = 0.0, total = 0.0;
  int ties_before = 0, from = 0, width = chunk;
  for (int level = 0; level < 2; ++level) {
    const bool summed = level == 0 && from_sums;
    if (!summed && !(level == 0 && from_list)) {
      double m = 0.0;
      int tie = 0;
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
      __syncthreads();  // nobody reads the slots any more
      if (lane == 0) {
        sh.part[0][wave] = m;
        sh.ipart[0][wave] = tie;
      }
      __syncthreads();
    }
    // (step 2 left its sums, which have no ties, in slot 1)
    auto wave_of = [&](int w, int seen, int &t) EE_ALWAYS_INLINE {
      t = summed ? 0 : sh.ipart[0][w];
      if (summed && splits > 0) return parts[w].z;
      return sh.part[summed ? 1 : 0][w] + min(max(ties - seen, 0), t) * tie_mass;
    };
    int t;
    const int shares = summed && splits > 0 ? splits : W;
    if (level == 0) {
      for (int w = 0, seen = 0; w < shares; ++w) {
        total += wave_of(w, seen, t);
        seen += t;
      }
      goal = static_cast<double>(u) * total;
    }
    int pick = -1;
    double upto = before;
    for (int w = 0, seen = ties_before; w < shares; ++w) {
      const double mass = wave_of(w, seen, t);
      if (mass > 0.0 && (pick < 0 || upto <= goal)) {
        pick = w;
        before = upto;
        ties_before = seen;
      }
      upto += mass;
      seen += t;
    }
    int to;
    if (summed && splits > 0) {
      from = first_of_part(a.vocab, pick, splits);
      to = min(first_of_part(a.vocab, pick + 1, splits), a.vocab);
    } else {
      from = from + pick * width;
      to = min(from + width, a.vocab);
    }
    if (level == 0) {
      width = share(from, to);
    } else {
      if (wave != 0) return;
      row.first = from;
      row.last = to;
    }
  }
  int rank = ties_before, chosen = -1;
  bool done = false;
  row.each([&](int id, const float (&x)[4]) EE_ALWAYS_INLINE {
    if (done) return;
    int mine = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) mine += x[e] > -INFINITY && key_of(x[e]) == tau ? 1 : 0;
    const int t_upto = wave_scan(mine);
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
    double upto = wave_scan(s);
    const double iter = of_lane(upto, 63);
    upto += before - s;
    int hit = -1, last = -1;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      upto += v[e];
      if (v[e] > 0.0) {
        last = id + e;
        if (hit < 0 && upto > goal) hit = id + e;
      }
    }
    const uint64_t hits = __ballot(hit >= 0), lasts = __ballot(last >= 0);
    if (hits != 0) {
      chosen = of_lane(hit, __builtin_ctzll(hits));
      done = true;
    } else if (lasts != 0) {
      chosen = of_lane(last, 63 - __builtin_clzll(lasts));
    }
    before += iter;
    rank += of_lane(t_upto, 63);
  });
  if (lane == 0) finish(chosen, mass_of(to_f32(row.p[chosen])) / total);
}

}  // namespace

// The largest row that LDS holds beside what else is there: 32000 fp32 logits.
constexpr size_t kLds = 160 << 10;

// Blocks a row that take the first two steps ahead, or 0, for rows that LDS does not hold: up
// to 64 of them, one block of each with its own few waves reading, leave most of the card
// idle.  A part is at least 16000 ids, as the sampling block adds up the parts' histograms.
// fp32 logits, top-p 0.9: 4 rows of 128000 56 us, in one block a row 93; 33 rows 61 and 99; 64
// rows 80 and 101; 128 rows are slower so, 111 and 105, and rows in LDS too (64 bf16 rows of
// 50021: 53 and 47).
int sample_splits(int n, int vocab) {
  const int splits = std::min(256 / n, vocab / 16000);
  return n <= 64 && splits >= 2 ? splits : 0;
}

size_t sample_workspace(int n, int vocab) {
  const size_t parts = static_cast<size_t>(n) * sample_splits(n, vocab);
  return std::max<size_t>(256, (parts * sizeof(Part) + 255) / 256 * 256 + parts * kBins * 8);
}

hipError_t launch_sample(bool f32, const SampleArgs &a, void *ws, hipStream_t stream) {
  if (a.n <= 0) return hipSuccess;
  const size_t row = (static_cast<size_t>(a.vocab) + 3) / 4 * 4 * (f32 ? 4 : 2);
  const bool cached = shared_bytes(true) + row <= kLds;
  const size_t lds = shared_bytes(cached) + (cached ? row : 0);
  const int splits = cached ? 0 : sample_splits(a.n, a.vocab);
  Part *parts = static_cast<Part *>(ws);
  auto *hists = reinterpret_cast<unsigned long long *>(
      static_cast<char *>(ws) + (static_cast<size_t>(a.n) * splits * sizeof(Part) + 255) / 256 * 256);
  hipError_t e = hipSuccess;
  EE_DISPATCH(f32, {
    if (splits > 0) {
      const dim3 grid(splits, a.n), block(64 * kPartWaves);
      hipLaunchKernelGGL(part_max_kernel<T>, grid, block, 0, stream, a, parts);
      e = hipGetLastError();
      if (e != hipSuccess) return e;
      hipLaunchKernelGGL(part_sum_kernel<T>, grid, block, 0, stream, a, parts, hists);
      e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    auto go = [&](auto k, int waves) {
      e = hipFuncSetAttribute(reinterpret_cast<const void *>(k), hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(lds));
      if (e != hipSuccess) return;
      hipLaunchKernelGGL(k, dim3(a.n), dim3(64 * waves), lds, stream, a, parts, hists, splits);
      e = hipGetLastError();
    };
    if (cached)
      go(sample_kernel<T, true, 16>, 16);
    else if (a.n > 256)  // two blocks of 8 waves a CU; 512 rows of 128000 fp32 logits, top-p 0.9: 201 us, in blocks of 16 217
      go(sample_kernel<T, false, 8>, 8);
    else
      go(sample_kernel<T, false, 16>, 16);
  });
  return e;
}

}  // namespace ee
