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

// A score as the draws take it: NaN as -inf, nothing above the largest float, one zero.
__device__ __forceinline__ float clean(float x) {
  x = x != x ? -INFINITY : (x > 3.402823466e38f ? 3.402823466e38f : x);
  return x + 0.0f;
}
__device__ __forceinline__ uint32_t key_of(float x) {  // rises with x
  const uint32_t b = __float_as_uint(x);
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

// Four entries of a row from i on (a multiple of four): those past the end as -inf.
template <int TYPE>
__device__ __forceinline__ void load4(const typename Score<TYPE>::T* row, uint32_t i, uint32_t n,
                                      bool vec, float (&v)[4]) {
  using T = typename Score<TYPE>::T;
  struct alignas(4 * sizeof(T)) Four {
    T v[4];
  };
  if (vec && i + 4u <= n) {
    const Four f = *reinterpret_cast<const Four*>(row + i);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = clean(Score<TYPE>::get(f.v[j]));
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      v[j] = i + (uint32_t)j < n ? clean(Score<TYPE>::get(row[i + j])) : -INFINITY;
  }
}

// What a row's draws go by.
struct RowRule {
  float m, inv;      // maximum, 1 / temperature
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
__device__ __forceinline__ uint32_t weight_of(float x, const RowRule& R) {
  return (uint32_t)(expf((x - R.m) * R.inv) * kOne);
}
// Which part of the running sum u draws.
__device__ __forceinline__ uint64_t target_of(float u, uint64_t total) {
  const double t = (double)u * (double)total;
  const uint64_t k = t > 0.0 ? (t < 9.2e18 ? (uint64_t)t : ~0ull) : 0ull;
  return k < total ? k : total - 1;
}
__device__ __forceinline__ float logp_of(float x, const RowRule& R, uint64_t total) {
  return (float)((double)((x - R.m) * R.inv) - log((double)total * (1.0 / 2147483648.0)));
}

// How many of the equal weights q, ranking after a sum of `before`, top-p's target needs (at least one).
__device__ __forceinline__ uint32_t ties_of(double target, uint64_t before, uint32_t q) {
  uint64_t m = (uint64_t)fmax((target - (double)before) / (double)q, 1.0);
  while ((double)(before + m * q) < target) ++m;
  while (m > 1 && (double)(before + (m - 1) * q) >= target) --m;
  return (uint32_t)m;
}

// A workgroup's memory.
struct RowShared {
  uint64_t part[kDrawSegs];        // the parts' sums, then their running sums
  uint64_t mass[256];
  uint32_t count[256];
  uint64_t wave[kDrawThreads / kWave];
  uint64_t out[2];
};

__device__ __forceinline__ uint64_t block_max(uint64_t v, RowShared& S) {
  v = wave_max(v);
  if (threadIdx.x % kWave == 0) S.wave[threadIdx.x / kWave] = v;
  __syncthreads();
  uint64_t b = 0;
  for (int i = 0; i < kDrawThreads / kWave; ++i) b = S.wave[i] > b ? S.wave[i] : b;
  __syncthreads();
  return b;
}

// The parts' sums to running sums; returns the total.
__device__ __forceinline__ uint64_t scan_parts(RowShared& S, uint32_t parts) {
  const uint32_t lane = threadIdx.x % kWave, wv = threadIdx.x / kWave;
  constexpr uint32_t per = kDrawSegs / kDrawThreads;
  uint64_t v[per], sum = 0;
#pragma unroll
  for (uint32_t j = 0; j < per; ++j) {
    const uint32_t i = threadIdx.x * per + j;
    v[j] = i < parts ? S.part[i] : 0;
    sum += v[j];
  }
  const uint64_t in = wave_scan(sum, lane);
  if (lane == kWave - 1) S.wave[wv] = in;
  __syncthreads();
  uint64_t run = in - sum, total = 0;
  for (uint32_t i = 0; i < kDrawThreads / kWave; ++i) {
    run += i < wv ? S.wave[i] : 0;
    total += S.wave[i];
  }
#pragma unroll
  for (uint32_t j = 0; j < per; ++j) {
    run += v[j];
    const uint32_t i = threadIdx.x * per + j;
    if (i < parts) S.part[i] = run;
  }
  __syncthreads();
  return total;
}

// The first part whose running sum exceeds `target`.
__device__ __forceinline__ uint32_t find_part(const RowShared& S, uint32_t parts, uint64_t target) {
  uint32_t lo = 0, hi = parts - 1;
  while (lo < hi) {
    const uint32_t mid = (lo + hi) / 2;
    if (S.part[mid] > target) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

// f(i, x) for every entry of the row, a wave to a part, four entries to a lane.
template <int TYPE, typename F>
__device__ __forceinline__ void each(const SampleArgs& A, const typename Score<TYPE>::T* row, F&& f) {
  const uint32_t lane = threadIdx.x % kWave;
  for (uint64_t a = (uint64_t)(threadIdx.x / kWave) * A.part; a < A.n;
       a += (uint64_t)(kDrawThreads / kWave) * A.part)
    for (uint32_t i = (uint32_t)a + 4u * lane; i < A.n && i - (uint32_t)a < A.part; i += 4u * kWave) {
      float v[4];
      load4<TYPE>(row, i, A.n, A.vec != 0, v);
#pragma unroll
      for (int j = 0; j < 4; ++j) f(i + (uint32_t)j, v[j]);
    }
}

// The part sums of w(i, x) over the row.
template <int TYPE, typename F>
__device__ __forceinline__ void sum_parts(const SampleArgs& A, const typename Score<TYPE>::T* row,
                                          RowShared& S, F&& w) {
  const uint32_t lane = threadIdx.x % kWave;
  for (uint64_t a = (uint64_t)(threadIdx.x / kWave) * A.part; a < A.n;
       a += (uint64_t)(kDrawThreads / kWave) * A.part) {
    uint64_t sum = 0;
    for (uint32_t i = (uint32_t)a + 4u * lane; i < A.n && i - (uint32_t)a < A.part; i += 4u * kWave) {
      float v[4];
      load4<TYPE>(row, i, A.n, A.vec != 0, v);
#pragma unroll
      for (int j = 0; j < 4; ++j) sum += w(i + (uint32_t)j, v[j]);
    }
    sum = wave_sum(sum);
    if (lane == 0) S.part[a / A.part] = sum;
  }
  __syncthreads();
}

// The entry of part `s` at which the running sum of w first exceeds `target` (a wave; the part
// holds it).
template <int TYPE, typename F>
__device__ __forceinline__ uint32_t find_entry(const SampleArgs& A, const typename Score<TYPE>::T* row,
                                               uint32_t s, uint64_t before, uint64_t target, F&& w) {
  const uint32_t lane = threadIdx.x % kWave;
  const uint32_t a = s * A.part;
  const uint32_t end = A.n - a < A.part ? A.n : a + A.part;
  for (uint32_t b = a; b < end; b += 4u * kWave) {
    float v[4];
    uint64_t q[4], sum = 0;
    const uint32_t i = b + 4u * lane;
    if (i < end) {
      load4<TYPE>(row, i, A.n, A.vec != 0, v);
    } else {
      v[0] = v[1] = v[2] = v[3] = -INFINITY;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      q[j] = i < end ? w(i + (uint32_t)j, v[j]) : 0;
      sum += q[j];
    }
    const uint64_t in = before + wave_scan(sum, lane);
    const uint64_t hit = __ballot(in > target);
    if (hit != 0) {
      const int l = __ffsll((unsigned long long)hit) - 1;
      uint64_t run = in - sum;
      uint32_t j = 0;
#pragma unroll
      for (int c = 0; c < 3; ++c) {
        run += q[c];
        if (run <= target) j = (uint32_t)c + 1u;
      }
      return (uint32_t)__shfl((int)(i + j), l, kWave);
    }
    before = (uint64_t)__shfl((unsigned long long)in, kWave - 1, kWave);
  }
  return end - 1;  // (not reached: the part's sum exceeds the target)
}

// Among the entries that rank at `from` or above: the score's key that the target-th entry (BY_MASS:
// the entry at which the sum of weights by rank reaches the target) has, eight bits at a time;
// *above receives the count (sum) that ranks before that key, *at the entries of that key.
template <int TYPE, bool BY_MASS>
__device__ uint32_t select_key(const SampleArgs& A, const typename Score<TYPE>::T* row, const RowRule& R,
                               RowShared& S, uint64_t from, double target, uint64_t* above) {
  uint32_t prefix = 0;
  uint64_t before = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (uint32_t i = threadIdx.x; i < 256u; i += kDrawThreads) {
      S.count[i] = 0;
      S.mass[i] = 0;
    }
    __syncthreads();
    each<TYPE>(A, row, [&](uint32_t i, float x) {
      const uint32_t key = key_of(x);
      if (shift < 24 && (key >> (shift + 8)) != (prefix >> (shift + 8))) return;
      if (!(x > -INFINITY) || rank_of(x, i) < from) return;
      const uint32_t q = weight_of(x, R);
      if (q == 0) return;
      const uint32_t d = (key >> shift) & 255u;
      if (BY_MASS) atomicAdd((unsigned long long*)&S.mass[d], (unsigned long long)q);
      else atomicAdd(&S.count[d], 1u);
    });
    __syncthreads();
    if (threadIdx.x == 0) {
      uint32_t d = 255;
      uint64_t sum = before;
      for (;; --d) {
        const uint64_t here = BY_MASS ? S.mass[d] : (uint64_t)S.count[d];
        if ((double)(sum + here) >= target || d == 0) break;
        sum += here;
      }
      S.out[0] = d;
      S.out[1] = sum;
    }
    __syncthreads();
    prefix |= (uint32_t)S.out[0] << shift;
    before = S.out[1];
    __syncthreads();
  }
  *above = before;
  return prefix;
}

// The rank of the m-th entry (from 1, by index) with this key.
template <int TYPE>
__device__ uint64_t rank_of_tie(const SampleArgs& A, const typename Score<TYPE>::T* row, RowShared& S,
                                uint32_t parts, uint32_t key, uint64_t m) {
  auto is = [&](uint32_t i, float x) { return (uint64_t)(i < A.n && key_of(x) == key ? 1 : 0); };
  sum_parts<TYPE>(A, row, S, is);
  scan_parts(S, parts);
  const uint32_t s = find_part(S, parts, m - 1);
  const uint32_t i = find_entry<TYPE>(A, row, s, s ? S.part[s - 1] : 0, m - 1, is);
  __syncthreads();
  return (uint64_t)key << 32 | (uint32_t)~i;
}

// A workgroup for a row (blockIdx.x), and for a share of its draws (blockIdx.y).
template <int TYPE>
__global__ void __launch_bounds__(kDrawThreads) k_sample_row(SampleArgs A) {
  using T = typename Score<TYPE>::T;
  __shared__ RowShared S;
  const uint32_t lane = threadIdx.x % kWave;
  const int64_t r = blockIdx.x;
  const T* row = static_cast<const T*>(A.x) + r * A.stride;
  const uint32_t parts = (A.n + A.part - 1) / A.part;
  uint64_t best = 0;
  each<TYPE>(A, row, [&](uint32_t i, float x) {
    const uint64_t k = i < A.n ? rank_of(x, i) : 0;
    best = k > best ? k : best;
  });
  best = block_max(best, S);
  const RowRule R = row_rule(A, r, best);
  const int64_t d0 = r * A.draws;
  if (!(R.m > -INFINITY) || R.greedy) {
    const bool none = !(R.m > -INFINITY);
    for (int64_t d = (int64_t)blockIdx.y * kDrawThreads + threadIdx.x; d < A.draws;
         d += (int64_t)gridDim.y * kDrawThreads) {
      A.index[d0 + d] = none ? -1 : (int32_t)R.first;
      if (A.logp) A.logp[d0 + d] = none ? -INFINITY : 0.0f;
    }
    return;
  }
  uint64_t from = 0;  // the least rank that is left
  if (R.k > 0) {
    uint64_t above;
    const uint32_t key = select_key<TYPE, false>(A, row, R, S, 0, (double)R.k, &above);
    // (fewer than k entries weigh anything: the last digits are 0, and all of them stay)
    if (key != 0) from = rank_of_tie<TYPE>(A, row, S, parts, key, R.k - above);
  }
  auto kept = [&](uint32_t i, float x) {
    if (!(x > -INFINITY) || rank_of(x, i) < from) return (uint64_t)0;
    const uint32_t q = weight_of(x, R);
    return (uint64_t)(q >= R.least ? q : 0);
  };
  if (R.p < 1.0) {
    const uint32_t least = R.least;
    sum_parts<TYPE>(A, row, S, [&](uint32_t i, float x) {
      return x > -INFINITY && rank_of(x, i) >= from ? (uint64_t)weight_of(x, R) : (uint64_t)0;
    });
    const uint64_t total = scan_parts(S, parts);
    const double target = fmax(R.p * (double)total, 1.0);
    uint64_t above;
    const uint32_t key = select_key<TYPE, true>(A, row, R, S, from, target, &above);
    const uint64_t cut =
        rank_of_tie<TYPE>(A, row, S, parts, key, ties_of(target, above, weight_of(key_score(key), R)));
    from = cut > from ? cut : from;
    (void)least;
  }
  sum_parts<TYPE>(A, row, S, kept);
  const uint64_t total = scan_parts(S, parts);
  const int64_t waves = (int64_t)gridDim.y * (kDrawThreads / kWave);
  for (int64_t d = (int64_t)blockIdx.y * (kDrawThreads / kWave) + threadIdx.x / kWave; d < A.draws;
       d += waves) {
    const uint64_t target = target_of(A.u[d0 + d], total);
    const uint32_t s = find_part(S, parts, target);
    const uint32_t i = find_entry<TYPE>(A, row, s, s ? S.part[s - 1] : 0, target, kept);
    if (lane == 0) {
      A.index[d0 + d] = (int32_t)i;
      if (A.logp) A.logp[d0 + d] = logp_of(clean(Score<TYPE>::get(row[i])), R, total);
    }
  }
}

// ----------------------------------------------------------------------------- loss

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, kWave);
  return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    const float w = __shfl_xor(v, o, kWave);
    v = w > v || w != w ? w : v;  // (a NaN stays)
  }
  return v;
}

// A wave for a row: maximum, sum, then the gradient, the row read three times.
template <int TYPE>
__global__ void __launch_bounds__(256) k_loss_row(LossArgs A) {
  using T = typename Score<TYPE>::T;
  const uint32_t lane = threadIdx.x % kWave;
  const int64_t waves = (int64_t)gridDim.x * (256 / kWave);
  for (int64_t r = (int64_t)blockIdx.x * (256 / kWave) + threadIdx.x / kWave; r < A.rows; r += waves) {
    const T* row = static_cast<const T*>(A.x) + r * A.stride;
    T* grad = A.grad ? static_cast<T*>(A.grad) + r * A.grad_stride : nullptr;
    const int32_t a = A.index[r];
    const float c = A.scale ? A.scale[r] : 1.0f;
    float m = -INFINITY;
    for (uint32_t i = lane; i < A.n; i += kWave) {
      const float v = Score<TYPE>::get(row[i]);
      m = v > m || v != v ? v : m;
    }
    m = wave_max(m);
    if (a < 0 || (uint32_t)a >= A.n || m == -INFINITY) {  // no answer
      if (A.loss && lane == 0) A.loss[r] = 0.0f;
      if (grad)
        for (uint32_t i = lane; i < A.n; i += kWave) grad[i] = Score<TYPE>::put(0.0f);
      continue;
    }
    float sum = 0.0f;
    for (uint32_t i = lane; i < A.n; i += kWave)
      sum += expf((Score<TYPE>::get(row[i]) - m) * A.inv_t);
    sum = wave_sum(sum);
    if (A.loss && lane == 0)
      A.loss[r] = (logf(sum) - (Score<TYPE>::get(row[a]) - m) * A.inv_t) * c;
    if (grad) {
      const float g = c * A.inv_t, inv = 1.0f / sum;
      for (uint32_t i = lane; i < A.n; i += kWave) {
        const float p = expf((Score<TYPE>::get(row[i]) - m) * A.inv_t) * inv;
        grad[i] = Score<TYPE>::put((i == (uint32_t)a ? p - 1.0f : p) * g);
      }
    }
  }
}

template <int TYPE>
void launch_sample(const SampleArgs& A, hipStream_t s) {
  const int64_t per = 4096;
  const uint32_t y = (uint32_t)((A.draws + per - 1) / per < 64 ? (A.draws + per - 1) / per : 64);
  hipLaunchKernelGGL(k_sample_row<TYPE>, dim3((uint32_t)A.rows, y), dim3(kDrawThreads), 0, s, A);
}
template <int TYPE>
void launch_loss(const LossArgs& A, hipStream_t s) {
  const int64_t b = (A.rows + 3) / 4;
  hipLaunchKernelGGL(k_loss_row<TYPE>, dim3((uint32_t)(b < 8192 ? b : 8192)), dim3(256), 0, s, A);
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
        (A.n + A.part - 1) / A.part > kDrawSegs)
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
