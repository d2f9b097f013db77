// gfx950 kernels that draw indices from rows of scores with given random numbers, and that score such
// draws: the answers of networks with several outputs, and the parents of a generation. Weights
// and ranks: choice.h.
#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "choice.h"

namespace emr {
namespace {

constexpr int kWave = 64;
constexpr float kOne = 2147483648.0f;  // weight of the maximum

template <int TYPE>
struct Score;
template <>
struct Score<kTypeF32> {
  using T = float;
  static __device__ __forceinline__ float get(T v) { return v; }
  static __device__ __forceinline__ T put(float v) { return v; }
};
template <>
struct Score<kTypeBf16> {
  using T = uint16_t;
  static __device__ __forceinline__ float get(T v) { return __uint_as_float((uint32_t)v << 16); }
  static __device__ __forceinline__ T put(float v) {  // to nearest, ties to even; NaN stays one
    const uint32_t b = __float_as_uint(v);
    if ((b & 0x7FFFFFFFu) > 0x7F800000u) return (T)((b >> 16) | 0x40u);
    return (T)((b + 0x7FFFu + ((b >> 16) & 1u)) >> 16);
  }
};
template <>
struct Score<kTypeF16> {
  using T = _Float16;
  static __device__ __forceinline__ float get(T v) { return (float)v; }
  static __device__ __forceinline__ T put(float v) { return (T)v; }
};

__device__ __forceinline__ float capped(float x) { return x > 3.402823466e38f ? 3.402823466e38f : x; }
// A score as the draws take it: NaN as -inf, nothing above the largest float.
__device__ __forceinline__ float clean(float x) { return x != x ? -INFINITY : capped(x); }
__device__ __forceinline__ uint32_t key_of(float x) {  // rises with x; one zero
  const uint32_t b = __float_as_uint(x + 0.0f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_score(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
__device__ __forceinline__ uint64_t rank_of(float x, uint32_t i) {
  return (uint64_t)key_of(x) << 32 | (uint32_t)~i;
}

__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    const uint64_t w = (uint64_t)__shfl_xor((unsigned long long)v, o, kWave);
    v = w > v ? w : v;
  }
  return v;
}
__device__ __forceinline__ uint64_t wave_sum(uint64_t v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += (uint64_t)__shfl_xor((unsigned long long)v, o, kWave);
  return v;
}
__device__ __forceinline__ uint64_t wave_scan(uint64_t v, uint32_t lane) {  // inclusive
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const uint64_t w = (uint64_t)__shfl_up((unsigned long long)v, o, kWave);
    if (lane >= (uint32_t)o) v += w;
  }
  return v;
}

// Four entries of a row from i on (a multiple of four, at which the row's memory is aligned to four entries):
// those outside lo .. n - 1 as -inf; with `cap`, none above the largest float. A NaN stays one: every
// comparison below leaves it out, as it does -inf.
template <int TYPE>
__device__ __forceinline__ void load4(const typename Score<TYPE>::T* row, uint32_t i, uint32_t lo, uint32_t n,
                                      bool cap, float (&v)[4]) {
  using T = typename Score<TYPE>::T;
  struct alignas(4 * sizeof(T)) Four {
    T v[4];
  };
  if (i >= lo && i + 4u <= n) {
    const Four f = *reinterpret_cast<const Four*>(row + i);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = Score<TYPE>::get(f.v[j]);
  } else {
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j)
      v[j] = i + j >= lo && i + j < n ? Score<TYPE>::get(row[i + j]) : -INFINITY;
  }
  if (cap) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = capped(v[j]);
  }
}

// What a row's draws go by.
struct RowRule {
  float m, inv;      // maximum, 1 / temperature
  float per;         // bins of the exponent for a unit of score (negative)
  uint32_t first;    // index of the first maximum
  uint32_t k;        // entries that top-k leaves (0: all)
  double p;          // top-p (1: all)
  uint32_t least;    // least weight that min-p leaves
  bool greedy;
};
__device__ __forceinline__ RowRule row_rule(const SampleArgs& A, int64_t r, uint64_t best) {
  RowRule R;
  R.m = key_score((uint32_t)(best >> 32));
  R.first = ~(uint32_t)best;
  const float t = A.row_t ? A.row_t[r] : A.t;
  R.greedy = !(t >= 1.17549435e-38f);
  R.inv = R.greedy ? 1.0f : 1.0f / fminf(t, 3.402823466e38f);
  const int32_t k = A.row_k ? A.row_k[r] : A.k;
  R.k = k > 0 && (uint32_t)k < A.n ? (uint32_t)k : 0u;
  const float p = A.row_p ? A.row_p[r] : A.p;
  R.p = p < 1.0f ? (double)p : 1.0;
  const float mp = A.row_min_p ? A.row_min_p[r] : A.min_p;
  R.least = mp > 0.0f ? (uint32_t)ceil((double)fminf(mp, 1.0f) * (double)kOne) : 0u;
  return R;
}
__device__ __forceinline__ float exponent_of(float x, const RowRule& R) { return (x - R.m) * R.inv; }
// (x: not a NaN)
__device__ __forceinline__ uint32_t weight_of(float x, const RowRule& R) {
  return (uint32_t)(expf(exponent_of(x, R)) * kOne);
}
// Which part of the running sum u draws.
__device__ __forceinline__ uint64_t target_of(float u, uint64_t total) {
  const double t = (double)u * (double)total;
  const uint64_t k = t > 0.0 ? (t < 9.2e18 ? (uint64_t)t : ~0ull) : 0ull;
  return k < total ? k : total - 1;
}
__device__ __forceinline__ float logp_of(float x, const RowRule& R, uint64_t total) {
  return (float)((double)exponent_of(x, R) - log((double)total * (1.0 / 2147483648.0)));
}

// How many of the equal weights q, ranking after a sum of `before`, top-p's target needs (at least one).
__device__ __forceinline__ uint32_t ties_of(double target, uint64_t before, uint32_t q) {
  uint64_t m = (uint64_t)fmax((target - (double)before) / (double)q, 1.0);
  while ((double)(before + m * q) < target) ++m;
  while (m > 1 && (double)(before + (m - 1) * q) >= target) --m;
  return (uint32_t)m;
}

// ----------------------------------------------------------------------------- short rows

// Rows of up to G scores, G lanes each, a score to a lane. An entry's rank, and the weight before it by
// rank, come from comparing it with the G others. Bound by the launch: 4000 rows of 8 take 9.6 us a call. A row's
// draws are its lanes' alone: 300000 draws of one row of 50 take 2.35 ms, where a row of 1000 takes 16 us.
template <int TYPE, int G>
__global__ void __launch_bounds__(256) k_sample_short(SampleArgs A) {
  using T = typename Score<TYPE>::T;
  const uint32_t lane = threadIdx.x % G;
  const int64_t rows = (int64_t)gridDim.x * (256 / G);
  for (int64_t r0 = (int64_t)blockIdx.x * (256 / G); r0 < A.rows; r0 += rows) {
    const int64_t r = r0 + threadIdx.x / G < A.rows ? r0 + threadIdx.x / G : A.rows - 1;
    const bool mine = r == r0 + threadIdx.x / G;  // (lanes past the rows shadow the last one)
    const T* row = static_cast<const T*>(A.x) + r * A.stride;
    const float x = lane < A.n ? clean(Score<TYPE>::get(row[lane])) : -INFINITY;
    const uint32_t key = lane < A.n ? key_of(x) : 0u;
    uint32_t top = key;
#pragma unroll
    for (int o = G / 2; o >= 1; o >>= 1) {
      const uint32_t w = (uint32_t)__shfl_xor((int)top, o, G);
      top = w > top ? w : top;
    }
    RowRule R = row_rule(A, r, (uint64_t)top << 32);
    uint32_t q = x > -INFINITY ? weight_of(x, R) : 0u;
    if (R.greedy || R.k > 0 || R.p < 1.0) {
      uint32_t rank = 0;
      uint64_t above = 0;
#pragma unroll 8
      for (int j = 0; j < G; ++j) {
        const uint32_t kj = (uint32_t)__shfl((int)key, j, G), qj = (uint32_t)__shfl((int)q, j, G);
        const bool before = kj > key || (kj == key && (uint32_t)j < lane);
        rank += before ? 1u : 0u;
        above += before ? qj : 0u;
      }
      if (R.greedy) q = rank == 0 && x > -INFINITY ? (uint32_t)kOne : 0u;
      else if (R.k > 0 && rank >= R.k) q = 0;
      if (!R.greedy && R.p < 1.0) {
        uint64_t total = q;
#pragma unroll
        for (int o = G / 2; o >= 1; o >>= 1) total += (uint64_t)__shfl_xor((unsigned long long)total, o, G);
        if (above != 0 && !((double)above < R.p * (double)total)) q = 0;
      }
    }
    if (!R.greedy && q < R.least) q = 0;
    uint64_t run = q;
#pragma unroll
    for (int o = 1; o < G; o <<= 1) {
      const uint64_t w = (uint64_t)__shfl_up((unsigned long long)run, o, G);
      if (lane >= (uint32_t)o) run += w;
    }
    const uint64_t total = (uint64_t)__shfl((unsigned long long)run, G - 1, G);
    for (int64_t d0 = 0; d0 < A.draws; d0 += G) {
      const int64_t d = d0 + lane;
      const bool draws = d < A.draws;
      const uint64_t target = total > 0 && draws ? target_of(A.u[r * A.draws + d], total) : 0;
      uint32_t at = 0;  // entries whose running sum does not exceed the target
#pragma unroll
      for (int step = G / 2; step >= 1; step >>= 1)
        if ((uint64_t)__shfl((unsigned long long)run, (int)(at + step - 1), G) <= target) at += step;
      const float y = __shfl(x, (int)at, G);
      if (!draws || !mine) continue;
      A.index[r * A.draws + d] = total > 0 ? (int32_t)at : -1;
      if (A.logp)
        A.logp[r * A.draws + d] = total == 0 ? -INFINITY : (R.greedy ? 0.0f : logp_of(y, R, total));
    }
  }
}

// ----------------------------------------------------------------------------- a workgroup for a row

constexpr uint32_t kFew = 256;    // entries that threads rank among themselves, one each
constexpr uint32_t kPairs = 128;  // entries of a list that is short enough for that from the start
constexpr uint32_t kList = 2048;  // entries of a row that a list holds

// A workgroup's memory: NT threads, bins of scores, and the row's parts.
template <int NT, int PARTS>
struct RowShared {
  static constexpr int kBins = 2 * NT;
  uint64_t part[PARTS];       // the parts' sums, then their running sums
  uint64_t mass[kBins];       // the bins' weights and entries, then their running sums
  uint32_t count[kBins];
  uint64_t wave[NT / kWave];
  uint32_t wcount[NT / kWave];
  uint64_t list[kList];       // ranks
  uint64_t cand[kFew];
  uint32_t cq[kFew];
  uint32_t n, listed, bin, lo, hi;
  uint64_t cut, below;
};

template <int NT, typename SH>
__device__ __forceinline__ uint64_t block_max(uint64_t v, SH& S) {
  v = wave_max(v);
  if (threadIdx.x % kWave == 0) S.wave[threadIdx.x / kWave] = v;
  __syncthreads();
  uint64_t b = 0;
#pragma unroll
  for (int i = 0; i < NT / kWave; ++i) b = S.wave[i] > b ? S.wave[i] : b;
  __syncthreads();
  return b;
}
template <int NT, typename SH>
__device__ __forceinline__ float block_max(float v, SH& S) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, kWave));
  if (threadIdx.x % kWave == 0) S.wcount[threadIdx.x / kWave] = __float_as_uint(v);
  __syncthreads();
  float b = -INFINITY;
#pragma unroll
  for (int i = 0; i < NT / kWave; ++i) b = fmaxf(b, __uint_as_float(S.wcount[i]));
  __syncthreads();
  return b;
}

// PER sums of each thread to running sums over the workgroup; returns the total.
template <int NT, int PER, typename SH>
__device__ __forceinline__ uint64_t block_scan(uint64_t (&v)[PER], SH& S) {
  const uint32_t lane = threadIdx.x % kWave, wv = threadIdx.x / kWave;
  uint64_t sum = 0;
#pragma unroll
  for (int j = 0; j < PER; ++j) sum += v[j];
  const uint64_t in = wave_scan(sum, lane);
  if (lane == kWave - 1) S.wave[wv] = in;
  __syncthreads();
  uint64_t run = in - sum, total = 0;
#pragma unroll
  for (uint32_t i = 0; i < NT / kWave; ++i) {
    run += i < wv ? S.wave[i] : 0;
    total += S.wave[i];
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < PER; ++j) v[j] = run += v[j];
  return total;
}

// The parts' sums to running sums; returns the total.
template <int NT, int PARTS, typename SH>
__device__ __forceinline__ uint64_t scan_parts(SH& S, uint32_t parts) {
  constexpr int per = PARTS / NT;
  uint64_t v[per];
#pragma unroll
  for (int j = 0; j < per; ++j) {
    const uint32_t i = threadIdx.x * per + j;
    v[j] = i < parts ? S.part[i] : 0;
  }
  const uint64_t total = block_scan<NT, per>(v, S);
#pragma unroll
  for (int j = 0; j < per; ++j) {
    const uint32_t i = threadIdx.x * per + j;
    if (i < parts) S.part[i] = v[j];
  }
  __syncthreads();
  return total;
}

// The first part whose running sum exceeds `target`.
template <typename SH>
__device__ __forceinline__ uint32_t find_part(const SH& S, uint32_t parts, uint64_t target) {
  uint32_t lo = 0, hi = parts - 1;
  while (lo < hi) {
    const uint32_t mid = (lo + hi) / 2;
    if (S.part[mid] > target) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

// Even bins of the exponent, rising as a score falls, over the scores that weigh anything: 2^-31 of the largest
// weight is at an exponent of -31 ln 2 = -21.49. The bin of lower scores, of -inf and of NaN is BINS.
constexpr float kSpan = 21.5f;
template <int BINS>
__device__ __forceinline__ uint32_t bin_of(float x, const RowRule& R) {
  return (uint32_t)fminf((x - R.m) * R.per, (float)BINS);
}

// A register's value that the compiler does not follow: what a pass over a row in registers computes from it
// is not kept for the next pass, which would take more registers than the row.
template <typename T>
__device__ __forceinline__ T fresh(T v) {
  asm volatile("" : "+v"(v));
  return v;
}

// A row's scores, and their weights once the rule is known: in registers as J groups of four to a thread
// (part k is group k), or (J = 0) read again from memory each time (part k is A.part entries, a wave's).
// Groups lie where memory is aligned: the row's first entry is number `lo` (0 .. 3) here, its last n - 1.
template <int TYPE, int NT, int J>
struct Row {
  using T = typename Score<TYPE>::T;
  const SampleArgs& A;
  const T* row;
  uint32_t lo, n;
  bool cap = false;  // scores above the largest float count as that
  static constexpr bool kWeights = NT * J <= 2048;  // (more do not fit the registers beside the scores)
  RowRule R;
  float x[4 * J + 1];
  uint32_t q[kWeights ? 4 * J + 1 : 1];

  __device__ Row(const SampleArgs& a, const T* r) : A(a) {
    lo = (uint32_t)((uintptr_t)r / sizeof(T)) % 4u;
    row = r - lo;
    n = a.n + lo;
  }
  __device__ uint32_t parts() const { return J > 0 ? (n + 3u) / 4u : (n + A.part - 1u) / A.part; }
  // The thread's maximum (uncapped).
  __device__ __forceinline__ float load() {
    float best = -INFINITY;
    if constexpr (J > 0) {
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const uint32_t i = 4u * ((uint32_t)j * NT + threadIdx.x);
        float v[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        if (i < n) load4<TYPE>(row, i, lo, n, cap, v);
#pragma unroll
        for (int c = 0; c < 4; ++c) x[4 * j + c] = v[c];
      }
#pragma unroll
      for (int j = 0; j < 4 * J; ++j) best = fmaxf(best, x[j]);
    } else {
      each_score([&](uint32_t, const float (&v)[4]) {
        best = fmaxf(fmaxf(best, fmaxf(v[0], v[1])), fmaxf(v[2], v[3]));
      });
    }
    return best;
  }
  // The largest rank.
  __device__ __forceinline__ uint64_t first_best() {
    uint64_t best = 0;
    each_above(-INFINITY, [&](uint32_t i, float v) {
      const uint64_t k = rank_of(v, i);
      best = k > best ? k : best;
    });
    return best;
  }
  // f(i, score) for all entries, and places past them (-inf).
  template <typename F>
  __device__ __forceinline__ void each_entry(F&& f) {
    if constexpr (J > 0) {
      const uint32_t i = fresh(4u * threadIdx.x);
#pragma unroll
      for (int j = 0; j < J; ++j) {
        if ((uint32_t)j * 4u * NT >= n) break;
#pragma unroll
        for (int c = 0; c < 4; ++c) f(i + (uint32_t)(4 * j * NT + c), fresh(x[4 * j + c]));
      }
    } else {
      each_score([&](uint32_t i, const float (&v)[4]) {
#pragma unroll
        for (uint32_t c = 0; c < 4; ++c) f(i + c, v[c]);
      });
    }
  }
  // f(i, score) for the entries of at least `least` (and above -inf).
  template <typename F>
  __device__ __forceinline__ void each_above(float least, F&& f) {
    if constexpr (J > 0) {
      const uint32_t i = fresh(4u * threadIdx.x);
#pragma unroll
      for (int j = 0; j < J; ++j) {
        if ((uint32_t)j * 4u * NT >= n) break;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const float v = fresh(x[4 * j + c]);
          if (v >= least && v > -INFINITY) f(i + (uint32_t)(4 * j * NT + c), v);
        }
      }
    } else {
      each_score([&](uint32_t i, const float (&v)[4]) {
        if (!(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])) >= least)) return;
#pragma unroll
        for (uint32_t c = 0; c < 4; ++c)
          if (v[c] >= least && v[c] > -INFINITY) f(i + c, v[c]);
      });
    }
  }
  // (J = 0) f(i, four scores) from i on
  template <typename F>
  __device__ __forceinline__ void each_score(F&& f) {
    constexpr uint32_t U = 4, step = 4u * NT;
    uint32_t i = 4u * threadIdx.x;
    for (; (uint64_t)i + (U - 1) * step < n; i += U * step) {
      float v[U][4];
#pragma unroll
      for (uint32_t k = 0; k < U; ++k) load4<TYPE>(row, i + k * step, lo, n, cap, v[k]);
#pragma unroll
      for (uint32_t k = 0; k < U; ++k) f(i + k * step, v[k]);
    }
    for (; i < n; i += step) {
      float v[4];
      load4<TYPE>(row, i, lo, n, cap, v);
      f(i, v);
    }
  }
  __device__ __forceinline__ uint32_t weight(float v) const { return v > -INFINITY ? weight_of(v, R) : 0u; }
  __device__ __forceinline__ void cap_all() {
    cap = true;
    if constexpr (J > 0) {
#pragma unroll
      for (int j = 0; j < 4 * J; ++j) x[j] = capped(x[j]);
    }
  }
  __device__ __forceinline__ void weigh(const RowRule& rule) {
    R = rule;
    if constexpr (J > 0 && kWeights) {
#pragma unroll
      for (int j = 0; j < 4 * J; ++j) q[j] = weight(x[j]);
    }
  }
  // f(i, score, weight) for the entries in a bin of the exponent
  template <typename F>
  __device__ __forceinline__ void each(F&& f) {
    if constexpr (J > 0) {
      const uint32_t i = fresh(4u * threadIdx.x);
#pragma unroll
      for (int j = 0; j < J; ++j) {
        if ((uint32_t)j * 4u * NT >= n) break;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const float v = fresh(x[4 * j + c]);
          if (bin_of<2 * NT>(v, R) < 2 * NT)
            f(i + (uint32_t)(4 * j * NT + c), v, kWeights ? fresh(q[kWeights ? 4 * j + c : 0]) : weight_of(v, R));
        }
      }
    } else {
      each_score([&](uint32_t i, const float (&v)[4]) {
#pragma unroll
        for (uint32_t c = 0; c < 4; ++c)
          if (bin_of<2 * NT>(v[c], R) < 2 * NT) f(i + c, v[c], weight_of(v[c], R));
      });
    }
  }
  // The parts' sums of w(i, score) over the entries of at least the score `least`. Few lanes of a wave hold
  // such an entry at a time where most of a row is cut, so each takes its next one in turn.
  template <typename SH, typename F>
  __device__ __forceinline__ void sum_parts(SH& S, float least, F&& w) {
    auto four = [&](uint32_t i, const float (&v)[4]) {
      uint64_t sum = 0;
      uint32_t mask = (v[0] >= least ? 1u : 0u) | (v[1] >= least ? 2u : 0u) | (v[2] >= least ? 4u : 0u) |
                      (v[3] >= least ? 8u : 0u);
      while (mask != 0) {
        const uint32_t c = (uint32_t)__builtin_ctz(mask);
        mask &= mask - 1u;
        const float a = c & 1u ? v[1] : v[0], b = c & 1u ? v[3] : v[2];
        sum += w(i + c, c & 2u ? b : a);
      }
      return sum;
    };
    if constexpr (J > 0) {
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const uint32_t k = (uint32_t)j * NT + threadIdx.x;
        const float v[4] = {fresh(x[4 * j]), fresh(x[4 * j + 1]), fresh(x[4 * j + 2]), fresh(x[4 * j + 3])};
        S.part[k] = four(4u * k, v);
      }
    } else {
      // (a part of 256 entries is one group of four to a lane; four parts' loads in flight)
      const uint32_t lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, parts_ = parts();
      constexpr uint32_t U = 4, W = NT / kWave;
      if (A.part == 4u * kWave) {
        for (uint32_t p = wave; p < parts_; p += U * W) {
          float v[U][4];
#pragma unroll
          for (uint32_t k = 0; k < U; ++k) {
            const uint32_t i = (p + k * W) * A.part + 4u * lane;
            if (p + k * W < parts_ && i < n) {
              load4<TYPE>(row, i, lo, n, cap, v[k]);
            } else {
              v[k][0] = v[k][1] = v[k][2] = v[k][3] = NAN;
            }
          }
#pragma unroll
          for (uint32_t k = 0; k < U; ++k) {
            uint64_t sum = four((p + k * W) * A.part + 4u * lane, v[k]);
            if (__ballot(sum != 0) != 0) sum = wave_sum(sum);
            if (lane == 0 && p + k * W < parts_) S.part[p + k * W] = sum;
          }
        }
      } else {
        for (uint32_t p = wave; p < parts_; p += W) {
          uint64_t sum = 0;
          for (uint32_t b = 4u * lane; b < A.part && (uint64_t)p * A.part + b < n; b += 4u * kWave) {
            float v[4];
            load4<TYPE>(row, p * A.part + b, lo, n, cap, v);
            sum += four(p * A.part + b, v);
          }
          if (__ballot(sum != 0) != 0) sum = wave_sum(sum);
          if (lane == 0) S.part[p] = sum;
        }
      }
    }
    __syncthreads();
  }
  // The entry of part s at which the running sum of w first exceeds `target` (the part holds it): for J = 0
  // a wave's, else a lane's.
  template <typename F>
  __device__ __forceinline__ uint32_t find_entry(uint32_t s, uint64_t before, uint64_t target, F&& w) {
    if constexpr (J > 0) {
      float v[4];
      load4<TYPE>(row, 4u * s, lo, n, cap, v);
      uint32_t j = 0;
#pragma unroll
      for (uint32_t c = 0; c < 3; ++c) {
        before += v[c] > -INFINITY ? w(4u * s + c, v[c]) : 0;
        if (before <= target) j = c + 1;
      }
      return 4u * s + j;
    } else {
      const uint32_t lane = threadIdx.x % kWave;
      const uint32_t a = s * A.part;
      const uint32_t end = n - a < A.part ? n : a + A.part;
      for (uint32_t b = a; b < end; b += 4u * kWave) {
        float v[4];
        uint64_t p[4], sum = 0;
        const uint32_t i = b + 4u * lane;
        if (i < end) {
          load4<TYPE>(row, i, lo, n, cap, v);
        } else {
          v[0] = v[1] = v[2] = v[3] = -INFINITY;
        }
#pragma unroll
        for (uint32_t c = 0; c < 4; ++c) {
          p[c] = i < end && v[c] > -INFINITY ? w(i + c, v[c]) : 0;
          sum += p[c];
        }
        const uint64_t in = before + wave_scan(sum, lane);
        const uint64_t hit = __ballot(in > target);
        if (hit != 0) {
          const int l = __ffsll((unsigned long long)hit) - 1;
          uint64_t run = in - sum;
          uint32_t j = 0;
#pragma unroll
          for (uint32_t c = 0; c < 3; ++c) {
            run += p[c];
            if (run <= target) j = c + 1;
          }
          return (uint32_t)__shfl((int)(i + j), l, kWave);
        }
        before = (uint64_t)__shfl((unsigned long long)in, kWave - 1, kWave);
      }
      return end - 1;  // (not reached: the part's sum exceeds the target)
    }
  }
};

// Entries of a row in a list: what is left after most of the row is known to be cut.
template <int NT, typename SH>
struct List {
  SH& S;
  const RowRule& R;
  __device__ __forceinline__ uint32_t weight(float v) const { return v > -INFINITY ? weight_of(v, R) : 0u; }
  template <typename F>
  __device__ __forceinline__ void each(F&& f) {
    for (uint32_t k = threadIdx.x; k < S.listed; k += NT) {
      const uint64_t r = S.list[k];
      const float x = key_score((uint32_t)(r >> 32));
      if (bin_of<2 * NT>(x, R) < 2 * NT) f(~(uint32_t)r, x, weight_of(x, R));
    }
  }
  template <typename F>
  __device__ __forceinline__ void each_entry(F&& f) {
    each_above(-INFINITY, f);
  }
  template <typename F>
  __device__ __forceinline__ void each_above(float least, F&& f) {
    for (uint32_t k = threadIdx.x; k < S.listed; k += NT) {
      const uint64_t r = S.list[k];
      const float x = key_score((uint32_t)(r >> 32));
      if (x >= least) f(~(uint32_t)r, x);
    }
  }
};

// The entries in a bin of the exponent, in bins of falling score: entries and weights of each bin, as running
// sums (without MASS no weights, without COUNT weights alone). BIN(i, x): a bin, or kBins for none, rising as x
// falls.
template <bool MASS, bool COUNT, int NT, typename ROW, typename SH, typename BIN>
__device__ __forceinline__ void bin_row(ROW& row, SH& S, BIN&& bin) {
  for (uint32_t i = threadIdx.x; i < SH::kBins; i += NT) {
    if (COUNT) S.count[i] = 0;
    if (MASS) S.mass[i] = 0;
  }
  __syncthreads();
  if constexpr (MASS) {
    row.each([&](uint32_t i, float x, uint32_t q) {
      const uint32_t b = bin(i, x);
      if (b >= (uint32_t)SH::kBins) return;
      if (COUNT) atomicAdd(&S.count[b], 1u);
      atomicAdd((unsigned long long*)&S.mass[b], (unsigned long long)q);
    });
  } else {
    row.each_entry([&](uint32_t i, float x) {
      const uint32_t b = bin(i, x);
      if (b < (uint32_t)SH::kBins) atomicAdd(&S.count[b], 1u);
    });
  }
  __syncthreads();
  const uint32_t lane = threadIdx.x % kWave, wv = threadIdx.x / kWave, b = 2u * threadIdx.x;
  uint32_t c = 0, c1 = 0;
  if constexpr (COUNT) {
    c1 = S.count[b + 1];
    c = S.count[b] + c1;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const uint32_t w = (uint32_t)__shfl_up((int)c, o, kWave);
      if (lane >= (uint32_t)o) c += w;
    }
    if (lane == kWave - 1) S.wcount[wv] = c;
  }
  if constexpr (MASS) {
    uint64_t m[2] = {S.mass[b], S.mass[b + 1]};
    block_scan<NT, 2>(m, S);
    S.mass[b] = m[0];
    S.mass[b + 1] = m[1];
  }
  __syncthreads();
  if constexpr (COUNT) {
#pragma unroll
    for (uint32_t i = 0; i < NT / kWave; ++i) c += i < wv ? S.wcount[i] : 0u;
    S.count[b] = c - c1;
    S.count[b + 1] = c;
    __syncthreads();
  }
}

// The bin in which the running count (mass) reaches `target`, or the last one.
template <bool BY_MASS, int NT, typename SH>
__device__ __forceinline__ uint32_t reach_bin(SH& S, double target) {
  if (threadIdx.x == 0) S.bin = SH::kBins - 1;
  __syncthreads();
  auto run = [&](uint32_t b) { return BY_MASS ? (double)S.mass[b] : (double)S.count[b]; };
#pragma unroll
  for (uint32_t j = 0; j < 2; ++j) {
    const uint32_t b = 2u * threadIdx.x + j;
    if (run(b) >= target && (b == 0 || !(run(b - 1) >= target))) S.bin = b;
  }
  __syncthreads();
  const uint32_t b = S.bin;
  __syncthreads();
  return b;
}

// Among the S.n <= kFew entries of S.cand, which rank after `count` others of weight `mass`: the one at which the
// target is reached.
template <bool BY_MASS, typename SH>
__device__ __forceinline__ uint64_t rank_few(SH& S, uint64_t count, uint64_t mass, double target) {
  const uint32_t n = S.n < kFew ? S.n : kFew;
  if (threadIdx.x < n) {
    const uint64_t mine = S.cand[threadIdx.x];
    const uint32_t q = S.cq[threadIdx.x];
    uint64_t before = mass, rank = count;
    for (uint32_t j = 0; j < n; ++j) {
      const bool a = S.cand[j] > mine;
      if (BY_MASS) before += a ? S.cq[j] : 0u;
      else rank += a ? 1u : 0u;
    }
    if (BY_MASS ? (double)before < target && (double)(before + q) >= target : (double)(rank + 1) == target)
      S.cut = mine;
  }
  __syncthreads();
  const uint64_t cut = S.cut;
  __syncthreads();
  return cut;
}

// The rank at which the entries ranking at `from` or above reach `target` by count (by weight), counted by
// falling rank. The bins are filled by `first`; a bin of many entries is divided again, evenly over its scores'
// bits, until few are left or all are equal. `some`: the row, or a list that holds every entry ranking
// as high; `row`: the row.
template <bool BY_MASS, bool MASS, int NT, int PARTS, typename SOME, typename ROW, typename SH, typename BIN>
__device__ __forceinline__ uint64_t reach(SOME& some, ROW& row, SH& S, uint64_t from, double target, BIN&& first) {
  uint32_t b = reach_bin<BY_MASS, NT>(S, target);
  uint64_t count = b ? S.count[b - 1] : 0, mass = MASS && b ? S.mass[b - 1] : 0;  // before the bin
  uint32_t inside = S.count[b] - (uint32_t)count;
  uint32_t lo = 0, hi = 0xFFFFFFFFu, level = 0;  // keys of the bin, from the second level on
  auto in_bin = [&](uint32_t i, float x) {
    if (level == 0) {
      if (first(i, x) != b) return false;
    } else {
      const uint32_t k = key_of(x);
      if (k < lo || k > hi) return false;
    }
    return bin_of<2 * NT>(x, some.R) < 2 * NT && rank_of(x, i) >= from;
  };
  while (inside > kFew) {
    // the bin's least and largest keys
    if (threadIdx.x == 0) {
      S.lo = 0xFFFFFFFFu;
      S.hi = 0;
    }
    __syncthreads();
    uint32_t l = 0xFFFFFFFFu, h = 0;
    some.each_above(-INFINITY, [&](uint32_t i, float x) {
      if (!in_bin(i, x)) return;
      const uint32_t k = key_of(x);
      l = k < l ? k : l;
      h = k > h ? k : h;
    });
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
      const uint32_t a = (uint32_t)__shfl_xor((int)l, o, kWave), c = (uint32_t)__shfl_xor((int)h, o, kWave);
      l = a < l ? a : l;
      h = c > h ? c : h;
    }
    if (threadIdx.x % kWave == 0 && l <= h) {
      atomicMin(&S.lo, l);
      atomicMax(&S.hi, h);
    }
    __syncthreads();
    lo = S.lo;
    hi = S.hi;
    level = 1;
    __syncthreads();
    if (lo >= hi) {  // equal scores: the first of them by index
      const float same = key_score(hi);
      const uint32_t q = some.weight(same);
      const uint64_t m = BY_MASS ? ties_of(target, mass, q) : (uint64_t)target - count;
      auto is = [&](uint32_t i, float x) { return (uint64_t)(i < row.n && x == same ? 1 : 0); };
      row.sum_parts(S, same, is);
      scan_parts<NT, PARTS>(S, row.parts());
      const uint32_t s = find_part(S, row.parts(), m - 1);
      const uint32_t i = row.find_entry(s, s ? S.part[s - 1] : 0, m - 1, is);
      __syncthreads();
      return (uint64_t)hi << 32 | (uint32_t)~i;
    }
    const uint32_t at = lo, width = hi - lo + 1u;  // (0: all 2^32)
    auto bin = [&](uint32_t i, float x) {
      const uint32_t k = key_of(x);
      if (k < lo || k > hi || bin_of<2 * NT>(x, some.R) >= 2 * NT || rank_of(x, i) < from)
        return (uint32_t)SH::kBins;
      return SH::kBins - 1u - (uint32_t)((uint64_t)(k - at) * SH::kBins / (width ? width : 1ull << 32));
    };
    bin_row<MASS, true, NT>(some, S, bin);
    b = reach_bin<BY_MASS, NT>(S, BY_MASS ? target - (double)mass : target - (double)count);
    inside = S.count[b] - (b ? S.count[b - 1] : 0u);
    if (b) {
      count += S.count[b - 1];
      if (MASS) mass += S.mass[b - 1];
    }
    // the keys of that bin
    const uint64_t w = width ? width : 1ull << 32, j = SH::kBins - 1u - b;
    lo = at + (uint32_t)((j * w + SH::kBins - 1) / SH::kBins);
    hi = at + (uint32_t)(((j + 1) * w + SH::kBins - 1) / SH::kBins - 1);
    __syncthreads();
  }
  if (threadIdx.x == 0) S.n = 0;
  __syncthreads();
  some.each_above(-INFINITY, [&](uint32_t i, float x) {
    if (!in_bin(i, x)) return;
    const uint32_t at = atomicAdd(&S.n, 1u);
    if (at < kFew) {
      S.cand[at] = rank_of(x, i);
      S.cq[at] = some.weight(x);
    }
  });
  __syncthreads();
  return rank_few<BY_MASS>(S, count, mass, target);
}

// The draws of a row of which at most kPairs entries can be left by top-k: each thread holds one and compares
// it with all others, for its rank and the weight before it by rank, then for the weight before it by index.
template <int NT, typename SH>
__device__ __forceinline__ void draw_listed(const SampleArgs& A, const RowRule& R, SH& S, uint32_t lo, int64_t d0) {
  const uint32_t n = S.listed;
  const bool in = threadIdx.x < n;
  const uint64_t mine = in ? S.list[threadIdx.x] : 0;
  const float x = key_score((uint32_t)(mine >> 32));
  uint32_t q = in ? weight_of(x, R) : 0u, rank = 0;
  if (in) S.cq[threadIdx.x] = q;
  __syncthreads();
  uint64_t above = 0, total = 0;
  if (in)
    for (uint32_t j = 0; j < n; ++j) {
      const bool a = S.list[j] > mine;
      rank += a ? 1u : 0u;
      above += a ? S.cq[j] : 0u;
    }
  if (rank >= R.k) q = 0;
  __syncthreads();
  if (in) S.cq[threadIdx.x] = q;
  __syncthreads();
  if (R.p < 1.0) {
    for (uint32_t j = 0; j < n; ++j) total += S.cq[j];
    if (above != 0 && !((double)above < R.p * (double)total)) q = 0;
  }
  if (q < R.least) q = 0;
  __syncthreads();
  if (in) S.cq[threadIdx.x] = q;
  __syncthreads();
  uint64_t before = 0;
  total = 0;
  for (uint32_t j = 0; j < n; ++j) {
    const uint32_t w = S.cq[j];
    total += w;
    before += (uint32_t)~(uint32_t)S.list[j] < (uint32_t)~(uint32_t)mine ? w : 0u;
  }
  if (q == 0) return;
  for (int64_t d = blockIdx.y; d < A.draws; d += gridDim.y) {
    const uint64_t target = target_of(A.u[d0 + d], total);
    if (target < before || target >= before + q) continue;
    A.index[d0 + d] = (int32_t)(~(uint32_t)mine - lo);
    if (A.logp) A.logp[d0 + d] = logp_of(x, R, total);
  }
}

// A workgroup for a row (blockIdx.x, from A.first on), and for a share of its draws (blockIdx.y). Memory: the row once
// (J > 0); else for its maximum, for the limits' bins and for the parts' sums, and once more for each division of
// a crowded bin. 256 rows of 131072 float scores, top-p: 109 us, 1.2 TB/s of the scores read once (each is read
// three times, 200 MB of it from memory, and the VALU issues in 56 % of the cycles); 256 rows of 2485, all filters:
// 15 us, latency. Draws from a short list look at all of the workgroup's: one row, top-k of up to 128, 16384
// draws: 400 us.
template <int TYPE, int NT, int J>
__global__ void __launch_bounds__(NT) k_sample_row(SampleArgs A) {
  using T = typename Score<TYPE>::T;
  constexpr int PARTS = J > 0 ? J * NT : (int)kDrawSegs;
  __shared__ RowShared<NT, PARTS> S;
  constexpr int kBins = 2 * NT;
  const uint32_t lane = threadIdx.x % kWave;
  const int64_t r = A.first + blockIdx.x, d0 = r * A.draws;
  Row<TYPE, NT, J> row(A, static_cast<const T*>(A.x) + r * A.stride);
  float m = block_max<NT>(row.load(), S);
  if (m > 3.402823466e38f) {
    row.cap_all();
    m = capped(m);
  }
  RowRule R = row_rule(A, r, (uint64_t)key_of(m) << 32);
  // (bounded for the least temperatures, where it would be an infinity, and the maximum's difference of 0 times
  // that in no bin: the bins then cover more scores than weigh anything)
  R.per = fmaxf(-R.inv * ((float)kBins / kSpan), -3.402823466e38f);
  if (!(m > -INFINITY) || R.greedy) {
    const bool none = !(m > -INFINITY);
    if (!none) R.first = ~(uint32_t)block_max<NT>(row.first_best(), S);
    for (int64_t d = (int64_t)blockIdx.y * NT + threadIdx.x; d < A.draws; d += (int64_t)gridDim.y * NT) {
      A.index[d0 + d] = none ? -1 : (int32_t)(R.first - row.lo);
      if (A.logp) A.logp[d0 + d] = none ? -INFINITY : 0.0f;
    }
    return;
  }
  row.weigh(R);
  uint64_t from = 0;  // the least rank that is left
  bool listed = false, summed = false;
  auto bin = [&](uint32_t, float x) { return bin_of<kBins>(x, R); };
  // A score below any of bin b's, by more than the bins' rounding.
  auto below_bin = [&](uint32_t b) { return R.m + ((float)(b + 1u) + 0.5f) / R.per - fabsf(R.m) * 1e-6f; };
  List<NT, decltype(S)> list{S, R};
  if (R.k > 0) {
    bin_row<false, true, NT>(row, S, bin);
    if (S.count[kBins - 1] > R.k) {
      // what can be among the k: with few others, all that follows is done on a list of it
      const uint32_t b = reach_bin<false, NT>(S, (double)R.k);
      listed = S.count[b] <= kList;
      if (listed) {
        if (threadIdx.x == 0) S.listed = 0;
        __syncthreads();
        row.each_above(below_bin(b), [&](uint32_t i, float x) {
          if (bin(i, x) <= b) S.list[atomicAdd(&S.listed, 1u)] = rank_of(x, i);
        });
        __syncthreads();
        if (S.listed <= kPairs) {
          draw_listed<NT>(A, R, S, row.lo, d0);
          return;
        }
        from = reach<false, false, NT, PARTS>(list, row, S, 0, (double)R.k, bin);
      } else {
        from = reach<false, false, NT, PARTS>(row, row, S, 0, (double)R.k, bin);
      }
    }
  }
  auto kept = [&](uint32_t i, float x) {
    if (from != 0 && rank_of(x, i) < from) return (uint64_t)0;
    const uint32_t q = weight_of(x, R);
    return (uint64_t)(q >= R.least ? q : 0u);
  };
  if (R.p < 1.0) {
    auto left = [&](uint32_t i, float x) { return from != 0 && rank_of(x, i) < from ? (uint32_t)kBins : bin(i, x); };
    if (listed) {
      bin_row<true, true, NT>(list, S, left);
      from = reach<true, true, NT, PARTS>(list, row, S, from, fmax(R.p * (double)S.mass[kBins - 1], 1.0), bin);
    } else if constexpr (J == 0) {
      // with the limit's bin known, one more reading gives the parts' sums of the bins before it and the
      // entries in it, of which those that stay are added to their parts
      bin_row<true, false, NT>(row, S, left);
      const double target = fmax(R.p * (double)S.mass[kBins - 1], 1.0);
      const uint32_t b = reach_bin<true, NT>(S, target);
      const uint64_t mass = b ? S.mass[b - 1] : 0;
      if (threadIdx.x == 0) S.n = 0;
      __syncthreads();
      row.sum_parts(S, below_bin(b), [&](uint32_t i, float x) {
        const uint32_t at = left(i, x);
        if (at > b) return (uint64_t)0;
        const uint32_t q = weight_of(x, R);
        if (at < b) return (uint64_t)(q >= R.least ? q : 0u);
        const uint32_t k = atomicAdd(&S.n, 1u);
        if (k < kFew) {
          S.cand[k] = rank_of(x, i);
          S.cq[k] = q;
        }
        return (uint64_t)0;
      });
      summed = S.n <= kFew;
      __syncthreads();
      if (summed) {
        from = rank_few<true>(S, 0, mass, target);
        if (threadIdx.x < S.n && S.cand[threadIdx.x] >= from && S.cq[threadIdx.x] >= R.least)
          atomicAdd((unsigned long long*)&S.part[~(uint32_t)S.cand[threadIdx.x] / A.part],
                    (unsigned long long)S.cq[threadIdx.x]);
        __syncthreads();
      } else {
        bin_row<true, true, NT>(row, S, left);
        from = reach<true, true, NT, PARTS>(row, row, S, from, target, bin);
      }
    } else {
      bin_row<true, true, NT>(row, S, left);
      from = reach<true, true, NT, PARTS>(row, row, S, from, fmax(R.p * (double)S.mass[kBins - 1], 1.0), bin);
    }
  }
  if (!summed) row.sum_parts(S, from ? key_score((uint32_t)(from >> 32)) : -INFINITY, kept);
  const uint32_t parts = row.parts();
  const uint64_t total = scan_parts<NT, PARTS>(S, parts);
  if constexpr (J > 0) {
    for (int64_t d = (int64_t)blockIdx.y * NT + threadIdx.x; d < A.draws; d += (int64_t)gridDim.y * NT) {
      const uint64_t target = target_of(A.u[d0 + d], total);
      const uint32_t s = find_part(S, parts, target);
      const uint32_t i = row.find_entry(s, s ? S.part[s - 1] : 0, target, kept);
      A.index[d0 + d] = (int32_t)(i - row.lo);
      if (A.logp) A.logp[d0 + d] = logp_of(clean(Score<TYPE>::get(row.row[i])), R, total);
    }
  } else {
    const int64_t waves = (int64_t)gridDim.y * (NT / kWave);
    for (int64_t d = (int64_t)blockIdx.y * (NT / kWave) + threadIdx.x / kWave; d < A.draws; d += waves) {
      const uint64_t target = target_of(A.u[d0 + d], total);
      const uint32_t s = find_part(S, parts, target);
      const uint32_t i = row.find_entry(s, s ? S.part[s - 1] : 0, target, kept);
      if (lane == 0) {
        A.index[d0 + d] = (int32_t)(i - row.lo);
        if (A.logp) A.logp[d0 + d] = logp_of(clean(Score<TYPE>::get(row.row[i])), R, total);
      }
    }
  }
}

// ----------------------------------------------------------------------------- loss

// e^((x - m) / T) as a power of two, of (x - m) with the factor log2(e) / T: a rounding less than in steps.
__device__ __forceinline__ float power(float d, float factor) { return __builtin_amdgcn_exp2f(d * factor); }

// Sum (maximum) over groups of G lanes.
template <int G>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int o = G / 2; o >= 1; o >>= 1) v += __shfl_xor(v, o, G);
  return v;
}
template <int G>
__device__ __forceinline__ float lanes_max(float v) {
#pragma unroll
  for (int o = G / 2; o >= 1; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, G));
  return v;
}

// A row's answer: none for an index outside it, or scores that are all -inf (or NaN: the loss is one then).
__device__ __forceinline__ bool answers(const LossArgs& A, int32_t index, float m, float sum) {
  return index >= 0 && (uint32_t)index < A.n && (m > -INFINITY || sum != sum);
}
__device__ __forceinline__ float loss_of(const LossArgs& A, float x, float m, float sum, float c) {
  return (logf(sum) - (x - m) * A.inv_t) * c;
}

// Rows of up to G scores, G lanes each.
template <int TYPE, int G>
__global__ void __launch_bounds__(256) k_loss_short(LossArgs A) {
  using T = typename Score<TYPE>::T;
  const uint32_t lane = threadIdx.x % G;
  const int64_t rows = (int64_t)gridDim.x * (256 / G);
  const float factor = A.inv_t * 1.44269504f;
  for (int64_t r0 = (int64_t)blockIdx.x * (256 / G); r0 < A.rows; r0 += rows) {
    const int64_t r = r0 + threadIdx.x / G;
    if (r >= A.rows) return;  // (whole groups of lanes)
    const bool in = lane < A.n;
    const float x = in ? Score<TYPE>::get(static_cast<const T*>(A.x)[r * A.stride + lane]) : -INFINITY;
    const int32_t a = A.index[r];
    const float c = A.scale ? A.scale[r] : 1.0f;
    const float m = lanes_max<G>(x);
    const float e = x != -INFINITY ? power(x - m, factor) : 0.0f;
    const float sum = lanes_sum<G>(e);
    const bool some = answers(A, a, m, sum);
    if (A.loss && (some ? lane == (uint32_t)a : lane == 0)) A.loss[r] = some ? loss_of(A, x, m, sum, c) : 0.0f;
    if (A.grad && in) {
      const float p = e / sum, g = (lane == (uint32_t)a ? p - 1.0f : p) * (c * A.inv_t);
      static_cast<T*>(A.grad)[r * A.grad_stride + lane] = Score<TYPE>::put(some ? g : 0.0f);
    }
  }
}

// Sum (maximum) over a row's NT threads.
template <int NT>
__device__ __forceinline__ double row_sum(double v, double* part) {
#pragma unroll
  for (int o = kWave / 2; o >= 1; o >>= 1) v += __shfl_xor(v, o, kWave);
  if constexpr (NT > kWave) {
    if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int i = 0; i < NT / kWave; ++i) v += part[i];
  }
  return v;
}
template <int NT>
__device__ __forceinline__ float row_max(float v, float* part) {
  v = lanes_max<kWave>(v);
  if constexpr (NT > kWave) {
    if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int i = 1; i < NT / kWave; ++i) v = fmaxf(v, part[i]);
  }
  return v;
}

// A row for NT threads (a wave: four rows to a workgroup), its scores in registers as J groups of 16 bytes to
// a thread, or (J = 0) read for the maximum, the sum and the gradient. Groups lie where memory is aligned; the
// row's first entry is number `lo` of its first group. The sum is taken in doubles, so that its float does
// not depend on where the row lies. One read and one write of each row: 2047 rows of 32001 bfloat16 scores in
// 83.4 us, 3.1 TB/s, bound as much by arithmetic as by memory: the VALU issues in 67 % of the cycles, three
// waves to a SIMD (an entry is unpacked, its exponential taken, added in double, scaled and rounded).
template <int TYPE, int NT, int J>
__global__ void __launch_bounds__(NT == kWave ? 256 : NT) k_loss_row(LossArgs A) {
  using T = typename Score<TYPE>::T;
  constexpr uint32_t V = 16 / sizeof(T);
  struct alignas(16) Group {
    T v[V];
  };
  __shared__ float mpart[NT / kWave];
  __shared__ double spart[NT / kWave];
  const uint32_t tid = threadIdx.x % NT;
  const int64_t r = A.first + (int64_t)blockIdx.x * (NT == kWave ? 4 : 1) + threadIdx.x / NT;
  if (r >= A.rows) return;  // (a wave's row)
  const T* row = static_cast<const T*>(A.x) + r * A.stride;
  T* grad = A.grad ? static_cast<T*>(A.grad) + r * A.grad_stride : const_cast<T*>(row);  // (unused)
  const uint32_t lo = (uint32_t)((uintptr_t)row / sizeof(T)) % V, n = A.n + lo;
  // (stores of whole groups where the gradient's row lies like the scores')
  const bool same = (uint32_t)((uintptr_t)grad / sizeof(T)) % V == lo;
  row -= lo;
  grad -= lo;
  const int32_t a = A.index[r];
  const float c = A.scale ? A.scale[r] : 1.0f;
  const float factor = A.inv_t * 1.44269504f;
  auto load = [&](uint32_t i, float (&v)[V]) {
    if (i >= lo && i + V <= n) {
      const Group f = *reinterpret_cast<const Group*>(row + i);
#pragma unroll
      for (uint32_t k = 0; k < V; ++k) v[k] = Score<TYPE>::get(f.v[k]);
    } else {
#pragma unroll
      for (uint32_t k = 0; k < V; ++k)
        v[k] = i + k >= lo && i + k < n ? Score<TYPE>::get(row[i + k]) : -INFINITY;
    }
  };
  const uint32_t at = lo + (uint32_t)a;  // the answer's place
  auto store = [&](uint32_t i, const float (&e)[V], float sum, bool some) {
    const float g = some ? c * A.inv_t : 0.0f, inv = some ? 1.0f / sum : 0.0f, scaled = inv * g;
    Group f;
#pragma unroll
    for (uint32_t k = 0; k < V; ++k) {
      const float d = i + k == at ? (e[k] * inv - 1.0f) * g : e[k] * scaled;
      f.v[k] = Score<TYPE>::put(some ? d : 0.0f);
    }
    if (same && i >= lo && i + V <= n) {
      *reinterpret_cast<Group*>(grad + i) = f;
    } else {
#pragma unroll
      for (uint32_t k = 0; k < V; ++k)
        if (i + k >= lo && i + k < n) grad[i + k] = f.v[k];
    }
  };
  float x_at = 0.0f;
  if (a >= 0 && (uint32_t)a < A.n) x_at = Score<TYPE>::get(row[at]);  // (before a gradient over the scores)
  if constexpr (J > 0) {
    float x[J][V];
    float m = -INFINITY;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const uint32_t i = V * ((uint32_t)j * NT + tid);
      if ((uint32_t)j * NT * V < n) {  // (the row's)
        load(i, x[j]);
      } else {
#pragma unroll
        for (uint32_t k = 0; k < V; ++k) x[j][k] = -INFINITY;
      }
    }
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (uint32_t k = 0; k < V; ++k) m = fmaxf(m, x[j][k]);
    m = row_max<NT>(m, mpart);
    double all = 0.0;
#pragma unroll
    for (int j = 0; j < J; ++j) {
#pragma unroll
      for (uint32_t k = 0; k < V; ++k) {
        x[j][k] = x[j][k] != -INFINITY ? power(x[j][k] - m, factor) : 0.0f;
        all += (double)x[j][k];
      }
    }
    const float sum = (float)row_sum<NT>(all, spart);
    const bool some = answers(A, a, m, sum);
    if (A.loss && tid == 0) A.loss[r] = some ? loss_of(A, x_at, m, sum, c) : 0.0f;
    if (!A.grad) return;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const uint32_t i = V * ((uint32_t)j * NT + tid);
      if (i < n) store(i, x[j], sum, some);
    }
  } else {
    float m = -INFINITY;
    for (uint32_t i = V * tid; i < n; i += V * NT) {
      float v[V];
      load(i, v);
#pragma unroll
      for (uint32_t k = 0; k < V; ++k) m = fmaxf(m, v[k]);
    }
    m = row_max<NT>(m, mpart);
    double all = 0.0;
    for (uint32_t i = V * tid; i < n; i += V * NT) {
      float v[V];
      load(i, v);
#pragma unroll
      for (uint32_t k = 0; k < V; ++k) all += v[k] != -INFINITY ? (double)power(v[k] - m, factor) : 0.0;
    }
    const float sum = (float)row_sum<NT>(all, spart);
    const bool some = answers(A, a, m, sum);
    if (A.loss && tid == 0) A.loss[r] = some ? loss_of(A, x_at, m, sum, c) : 0.0f;
    if (!A.grad) return;
    for (uint32_t i = V * tid; i < n; i += V * NT) {
      float v[V];
      load(i, v);
#pragma unroll
      for (uint32_t k = 0; k < V; ++k) v[k] = power(v[k] - m, factor);
      store(i, v, sum, some);
    }
  }
}

// Workgroups of a launch, at most: its threads in a dimension are a 32-bit number.
constexpr int64_t most_groups(int threads) { return 0xFFFFFFFFll / threads; }

template <int TYPE, int G>
void launch_short(const SampleArgs& A, hipStream_t s) {
  const int64_t b = (A.rows + 256 / G - 1) / (256 / G);
  hipLaunchKernelGGL((k_sample_short<TYPE, G>), dim3((uint32_t)(b < 65536 ? b : 65536)), dim3(256), 0, s, A);
}
template <int TYPE, int NT, int J>
void launch_row(const SampleArgs& A, hipStream_t s) {
  // (every workgroup of a row finds its limits anew: shares of several draws for each thread, or wave)
  const int64_t per = J > 0 ? 8 * NT : 4 * NT, y = (A.draws + per - 1) / per, most = most_groups(NT);
  for (SampleArgs B = A; B.first < A.rows; B.first += most) {
    const int64_t rows = A.rows - B.first < most ? A.rows - B.first : most;
    hipLaunchKernelGGL((k_sample_row<TYPE, NT, J>), dim3((uint32_t)rows, (uint32_t)(y < 256 ? y : 256)), dim3(NT), 0,
                       s, B);
  }
}
// The smallest variant that holds a row. It is the faster one up to its border, with exceptions (us of it and of the
// next one, float scores, top-p 0.95; 4096 rows up to 8189 scores, then 1024): 64 scores: 11.9, 28.3; 1021: 33, 42;
// 4093: 67, 93; 8189: 136, 232 (but 256 rows, one to a CU: 24, 17); 16381: 80, 94; 32765: 146, 127, since the
// weights' registers spill there (without a filter 83, 89; with top-k 50 too 82, 92).
template <int TYPE>
void launch_sample(const SampleArgs& A, hipStream_t s) {
  if (A.n <= 8) launch_short<TYPE, 8>(A, s);
  else if (A.n <= 16) launch_short<TYPE, 16>(A, s);
  else if (A.n <= 32) launch_short<TYPE, 32>(A, s);
  else if (A.n <= 64) launch_short<TYPE, 64>(A, s);
  // (up to three entries more where a row is not aligned)
  else if (A.n <= 1024 - 3) launch_row<TYPE, 256, 1>(A, s);
  else if (A.n <= 4096 - 3) launch_row<TYPE, 256, 4>(A, s);
  else if (A.n <= 8192 - 3) launch_row<TYPE, 256, 8>(A, s);
  else if (A.n <= 16384 - 3) launch_row<TYPE, 1024, 4>(A, s);
  else if (A.n <= 32768 - 3) launch_row<TYPE, 1024, 8>(A, s);
  else launch_row<TYPE, 1024, 0>(A, s);
}
template <int TYPE, int G>
void launch_loss_short(const LossArgs& A, hipStream_t s) {
  const int64_t b = (A.rows + 256 / G - 1) / (256 / G);
  hipLaunchKernelGGL((k_loss_short<TYPE, G>), dim3((uint32_t)(b < 65536 ? b : 65536)), dim3(256), 0, s, A);
}
template <int TYPE, int NT, int J>
void launch_loss_row(const LossArgs& A, hipStream_t s) {
  constexpr int threads = NT == kWave ? 256 : NT, each = threads / NT;
  constexpr int64_t most = most_groups(threads) * each;
  for (LossArgs B = A; B.first < A.rows; B.first += most) {
    const int64_t rows = A.rows - B.first < most ? A.rows - B.first : most;
    hipLaunchKernelGGL((k_loss_row<TYPE, NT, J>), dim3((uint32_t)((rows + each - 1) / each)), dim3(threads), 0, s, B);
  }
}
// The smallest variant that holds a row (us of it and of the next one at its border, float scores, 4M of them up to
// rows of 64, then 32M): 8: 14.6, 25.6; 16: 14.2, 25.7; 32: 14.4, 26.9; 64: 15.2, 30.4; 1021: 42.6, 65.1; 4093: 42.7, 50.2;
// 16381: 40.9, 43.9; 32765: 43.3, 58.8; 65533: 50.2, 75.1 (bfloat16 rows of 65529: 40.4, 42.0).
template <int TYPE>
void launch_loss(const LossArgs& A, hipStream_t s) {
  constexpr uint32_t V = 16 / sizeof(typename Score<TYPE>::T);
  const uint32_t n = A.n + V - 1;  // (where a row is not aligned)
  if (A.n <= 8) launch_loss_short<TYPE, 8>(A, s);
  else if (A.n <= 16) launch_loss_short<TYPE, 16>(A, s);
  else if (A.n <= 32) launch_loss_short<TYPE, 32>(A, s);
  else if (A.n <= 64) launch_loss_short<TYPE, 64>(A, s);
  else if (n <= 16 * 64) launch_loss_row<TYPE, 64, 16 / V>(A, s);
  else if (n <= 16 * 256) launch_loss_row<TYPE, 256, 16 / V>(A, s);
  else if (n <= 64 * 256) launch_loss_row<TYPE, 256, 64 / V>(A, s);
  else if (n <= 64 * 512) launch_loss_row<TYPE, 512, 64 / V>(A, s);
  else if (n <= 64 * 1024) launch_loss_row<TYPE, 1024, 64 / V>(A, s);
  else launch_loss_row<TYPE, 1024, 0>(A, s);
}

}  // namespace
}  // namespace emr

// Kinds: 0 draws, 1 loss.
extern "C" hipError_t emr_launch_choice(int kind, const void* args, hipStream_t s) {
  using namespace emr;
  if (kind == 0) {
    const auto& A = *static_cast<const SampleArgs*>(args);
    if (A.rows <= 0 || A.draws <= 0) return hipSuccess;
    if (A.n == 0 || A.rows > 0x7FFFFFFF || A.part == 0 || A.part % kDrawPart != 0 ||
        ((uint64_t)A.n + 3 + A.part - 1) / A.part > kDrawSegs)
      return hipErrorInvalidValue;
    switch (A.type) {
      case kTypeF32: launch_sample<kTypeF32>(A, s); break;
      case kTypeBf16: launch_sample<kTypeBf16>(A, s); break;
      case kTypeF16: launch_sample<kTypeF16>(A, s); break;
      default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
  }
  if (kind == 1) {
    const auto& A = *static_cast<const LossArgs*>(args);
    if (A.rows <= 0 || A.n == 0) return hipSuccess;
    switch (A.type) {
      case kTypeF32: launch_loss<kTypeF32>(A, s); break;
      case kTypeBf16: launch_loss<kTypeBf16>(A, s); break;
      case kTypeF16: launch_loss<kTypeF16>(A, s); break;
      default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
  }
  return hipErrorInvalidValue;
}
