// gfx950 kernels of the gradients of activated networks: the derivatives of the edges' weights (and of
// the input patterns) from the states that an activation kept in 8 bits.
//
// With s_t the states after step t (s_0: the patterns at the input nodes, 0 elsewhere; inputs hold still) and
// z_t[i] the sum over i's incoming edges of w s_{t-1}, s_t = sigmoid(z_t). From the derivative d_T of the
// outputs backwards,
//   gz_t[i]    = d_t[i] s_t[i] (1 - s_t[i])                         (0 at input nodes)
//   gw[e]     += sum over patterns of gz_t[dst e] s_{t-1}[src e]
//   d_{t-1}[j] = sum over j's outgoing edges of w gz_t[dst]
// The states are the kept codes / 255, but for the outputs after the last step, which are given.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "emr_internal.h"
#include "learn.h"

namespace emr {
namespace {

__device__ __forceinline__ int64_t grid_thread() {
  return (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
}
__device__ __forceinline__ int64_t grid_threads() { return (int64_t)gridDim.x * blockDim.x; }

// ----------------------------------------------------------------------------- edges by source

// A wave for a node: its edges' destination, and their sort keys and values.
__global__ void __launch_bounds__(kNetThreads) k_turn_keys(NetTurnArgs A) {
  const uint32_t lane = threadIdx.x % kWave;
  for (int64_t i = grid_thread() / kWave; i < A.nodes; i += grid_threads() / kWave) {
    const int64_t e1 = A.in_offset[i + 1] < A.edges ? A.in_offset[i + 1] : A.edges;
    for (int64_t e = A.in_offset[i] + lane; e < e1; e += kWave) {
      A.key[e] = A.in_src[e];
      A.val[e] = (uint64_t)e | (uint64_t)i << 32;
      A.dst[e] = (uint32_t)i;
    }
  }
}

// The first sorted edge of every source.
__global__ void __launch_bounds__(kNetThreads) k_turn_offsets(NetTurnArgs A) {
  for (int64_t i = grid_thread(); i <= A.nodes; i += grid_threads()) {
    int64_t lo = 0, hi = A.edges;
    while (lo < hi) {
      const int64_t mid = (lo + hi) / 2;
      if ((int64_t)A.skey[mid] < i) lo = mid + 1;
      else hi = mid;
    }
    A.out_offset[i] = lo;
  }
}

// ----------------------------------------------------------------------------- stepwise

// The four codes of a node's state for pattern group pg, and their states.
__device__ __forceinline__ uint32_t code4(const NetKept& K, int64_t nodes, uint32_t plane, uint32_t pg,
                                          int64_t node) {
  const uint32_t b = pg / K.q;
  return *reinterpret_cast<const uint32_t*>(
      K.codes + (((int64_t)plane * K.blocks + b) * nodes + node) * (4 * K.q) + 4 * (pg % K.q));
}
__device__ __forceinline__ float4 states(uint32_t c) {
  constexpr float k = 1.0f / 255.0f;
  return make_float4((float)(c & 255u) * k, (float)((c >> 8) & 255u) * k,
                     (float)((c >> 16) & 255u) * k, (float)(c >> 24) * k);
}

// s (1 - s) of a code: c (255 - c) is exact, so states near 1 lose nothing to 1 - s.
__device__ __forceinline__ float slope_of(uint32_t c) {
  return (float)(c * (255u - c)) * (1.0f / 65025.0f);
}

__device__ __forceinline__ float4 pattern_of(const NetBackArgs& A, int32_t slot, uint32_t pb) {
  float c[4];
#pragma unroll
  for (uint32_t k = 0; k < 4; ++k) {
    const uint32_t p = 4u * pb + k;
    c[k] = p < A.n_patterns ? A.patterns[(int64_t)p * A.n_inputs + (uint32_t)slot] : 0.0f;
  }
  return make_float4(c[0], c[1], c[2], c[3]);
}

// A node's states before step A.step: the pattern's, the kept ones, or 0 before the first step.
__device__ __forceinline__ float4 state_before(const NetBackArgs& A, int64_t node, uint32_t pb) {
  const int32_t slot = A.node_in[node];
  if (slot >= 0) return pattern_of(A, slot, pb);
  if (A.step < 2) return make_float4(0.f, 0.f, 0.f, 0.f);
  return states(code4(A.kept, A.nodes, A.step - 2, pb, node));
}

// The derivatives by the output nodes' sums in the last step (the others are cleared before).
__global__ void __launch_bounds__(kNetThreads) k_back_outputs(NetBackArgs A) {
  float* gz = A.gz_before;
  const int64_t per = (int64_t)A.n_patterns * A.n_outputs;
  for (int64_t r = grid_thread(); r < per; r += grid_threads()) {
    const uint32_t p = (uint32_t)(r / A.n_outputs), o = (uint32_t)(r % A.n_outputs);
    const int64_t at = A.genome * per + r;
    const float v = A.outputs[at];
    gz[((int64_t)(p / 4u) * A.size + A.out_node[o]) * 4 + p % 4u] = A.grad_outputs[at] * v * (1.0f - v);
  }
}
__global__ void __launch_bounds__(kNetThreads) k_back_clear(LearnFillArgs A) {
  for (int64_t i = grid_thread(); i < A.n; i += grid_threads()) A.p[i] = 0.0f;
}

// The weights' derivatives in one step: a thread for an edge.
__global__ void __launch_bounds__(kNetThreads) k_back_edges(NetBackArgs A) {
  const float4* gz = reinterpret_cast<const float4*>(A.gz);
  for (int64_t e = A.edge0 + grid_thread(); e < A.edge1; e += grid_threads()) {
    const int64_t src = A.in_src[e], dst = A.dst[e];
    float sum = 0.0f;
    for (uint32_t pb = 0; pb < A.pblocks; ++pb) {
      const float4 d = gz[(int64_t)pb * A.size + dst - A.node0], s = state_before(A, src, pb);
      sum = fmaf(d.x, s.x, fmaf(d.y, s.y, fmaf(d.z, s.z, fmaf(d.w, s.w, sum))));
    }
    A.grad_w[e] = A.last ? sum : A.grad_w[e] + sum;
  }
}

// The derivatives before the step: a wave for a node, its outgoing edges over the lanes.
__global__ void __launch_bounds__(kNetThreads) k_back_nodes(NetBackArgs A) {
  const float4* gz = reinterpret_cast<const float4*>(A.gz);
  float4* before = reinterpret_cast<float4*>(A.gz_before);
  const uint32_t lane = threadIdx.x % kWave;
  for (int64_t i = grid_thread() / kWave; i < A.size; i += grid_threads() / kWave) {
    const int64_t j = A.node0 + i;
    const int32_t slot = A.node_in[j];
    const int64_t e0 = A.out_offset[j], e1 = A.out_offset[j + 1];
    for (uint32_t pb = blockIdx.z; pb < A.pblocks; pb += gridDim.z) {
      if (slot >= 0 && A.grad_inputs == nullptr) continue;
      float4 d = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int64_t k = e0 + lane; k < e1; k += kWave) {
        const uint64_t v = A.out_edge[k];
        const float w = A.in_w[(uint32_t)v];
        const float4 x = gz[(int64_t)pb * A.size + (int64_t)(v >> 32) - A.node0];
        d.x = fmaf(w, x.x, d.x);
        d.y = fmaf(w, x.y, d.y);
        d.z = fmaf(w, x.z, d.z);
        d.w = fmaf(w, x.w, d.w);
      }
#pragma unroll
      for (int o = 32; o >= 1; o >>= 1) {
        d.x += __shfl_xor(d.x, o, kWave);
        d.y += __shfl_xor(d.y, o, kWave);
        d.z += __shfl_xor(d.z, o, kWave);
        d.w += __shfl_xor(d.w, o, kWave);
      }
      if (slot >= 0) {
        const uint32_t p = 4u * pb + lane;
        if (lane < 4u && p < A.n_patterns) {
          float* g = A.grad_inputs + ((int64_t)A.genome * A.n_patterns + p) * A.n_inputs + (uint32_t)slot;
          const float v = lane == 0 ? d.x : (lane == 1 ? d.y : (lane == 2 ? d.z : d.w));
          *g = A.last ? v : *g + v;
        }
      } else if (lane == 0 && A.step > 1) {
        const uint32_t c = code4(A.kept, A.nodes, A.step - 2, pb, j);
        before[(int64_t)pb * A.size + i] =
            make_float4(d.x * slope_of(c & 255u), d.y * slope_of((c >> 8) & 255u),
                        d.z * slope_of((c >> 16) & 255u), d.w * slope_of(c >> 24));
      }
    }
  }
}

// ----------------------------------------------------------------------------- layouts

// Exclusive prefix sum over the workgroup (every thread must call it); *total receives the sum.
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t* part, uint32_t* total) {
  const uint32_t lane = threadIdx.x % kWave, wv = threadIdx.x / kWave;
  uint32_t x = v;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const uint32_t y = (uint32_t)__shfl_up((int)x, (unsigned)o, kWave);
    if (lane >= (uint32_t)o) x += y;
  }
  if (lane == kWave - 1) part[wv] = x;
  __syncthreads();
  uint32_t before = 0, tot = 0;
  for (uint32_t i = 0; i < blockDim.x / kWave; ++i) {
    before += i < wv ? part[i] : 0u;
    tot += part[i];
  }
  __syncthreads();
  *total = tot;
  return before + x - v;
}

__device__ __forceinline__ uint32_t padded(uint32_t len) {
  return (len + kLearnPad - 1u) / kLearnPad * kLearnPad;
}

constexpr int kLayoutThreads = 512;
constexpr uint32_t kAbsent = 0xFFFFFFFFu;

// One of a genome's four layouts (blockIdx.y).
__global__ void __launch_bounds__(kLayoutThreads) k_learn_layout(LearnLayoutArgs A) {
  __shared__ uint32_t key[kStepNodes];    // edges of a row (bit 31: an output's, always heavy), or kAbsent
  __shared__ uint16_t rank[kStepNodes];   // a row's place in the order
  __shared__ uint32_t part[kLayoutThreads / kWave];
  __shared__ uint32_t heavy, rows, places;
  const uint32_t g = A.genomes[blockIdx.x];
  const int which = (int)blockIdx.y;
  const LearnSet S = A.set[which];
  const bool by_in = which == kInHid || which == kInInp;
  const bool inputs = which == kInInp || which == kOutInp;
  const int64_t n0 = A.node_offset[g];
  const uint32_t n = (uint32_t)(A.node_offset[g + 1] - n0);
  if (n > kStepNodes) return;  // (host-checked)
  const uint32_t lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  constexpr uint32_t waves = kLayoutThreads / kWave;
  uint2* ent = S.ent + A.place[g];
  uint32_t* edge = S.edge + A.place[g];
  LearnSlice* slices = S.slices + A.slice[g];
  uint16_t* row_of = S.rows + 16 * A.slice[g];
  if (threadIdx.x == 0) heavy = rows = 0;
  __syncthreads();
  for (uint32_t i = wave; i < n; i += waves) {
    const int64_t node = n0 + i;
    const bool is_input = A.node_in[node] >= 0;
    uint32_t d = 0;
    if (by_in) {
      if (!is_input)
        for (int64_t e = A.in_offset[node]; e < A.in_offset[node + 1]; e += kWave) {
          const int64_t k = e + lane;
          const bool mine = k < A.in_offset[node + 1] && (A.node_in[A.in_src[k]] >= 0) == inputs;
          d += (uint32_t)__popcll(__ballot(mine));
        }
    } else if (is_input == inputs) {
      d = (uint32_t)(A.out_offset[node + 1] - A.out_offset[node]);
    }
    if (lane == 0) {
      const bool in = by_in ? !is_input : is_input == inputs;
      key[i] = in ? d : kAbsent;
    }
  }
  __syncthreads();
  if (which == kInHid) {
    for (uint32_t o = threadIdx.x; o < A.n_outputs; o += kLayoutThreads)
      key[A.out_node[o]] |= 0x80000000u;
    __syncthreads();
  }
  for (uint32_t i = threadIdx.x; i < n; i += kLayoutThreads) {
    const uint32_t k = key[i];
    if (k == kAbsent) continue;
    uint32_t r = 0;
    for (uint32_t j = 0; j < n; ++j) {
      const uint32_t o = key[j];
      r += o != kAbsent && (o > k || (o == k && j < i)) ? 1u : 0u;
    }
    rank[i] = (uint16_t)r;
    atomicAdd(&rows, 1u);
    if (k > kLightEdges) atomicAdd(&heavy, 1u);
  }
  __syncthreads();
  const uint32_t nh = heavy, ns = nh + (rows - nh + 15u) / 16u;
  // the slices' lengths, then their bases
  for (uint32_t i = threadIdx.x; i < n; i += kLayoutThreads) {
    const uint32_t k = key[i];
    if (k == kAbsent) continue;
    const uint32_t r = rank[i];
    if (r < nh) {
      slices[r] = {0, padded(((k & 0x7FFFFFFFu) + 15u) / 16u), 0, 1};
      for (uint32_t j = 0; j < 16; ++j) row_of[16u * r + j] = (uint16_t)i;
    } else {
      const uint32_t s = nh + (r - nh) / 16u;
      if ((r - nh) % 16u == 0) slices[s] = {0, padded(k), 0, 0};
      row_of[16u * s + (r - nh) % 16u] = (uint16_t)i;
    }
  }
  for (uint32_t r = rows + threadIdx.x; r < nh + 16u * (ns - nh); r += kLayoutThreads)
    row_of[16u * (nh + (r - nh) / 16u) + (r - nh) % 16u] = (uint16_t)kNoRow;
  __threadfence_block();
  __syncthreads();
  uint32_t base = 0;
  for (uint32_t s0 = 0; s0 < ns; s0 += kLayoutThreads) {
    const uint32_t s = s0 + threadIdx.x;
    uint32_t total;
    const uint32_t at = block_scan(s < ns ? 16u * slices[s].len : 0u, part, &total);
    if (s < ns) slices[s].base = base + at;
    base += total;
  }
  if (threadIdx.x == 0) {
    places = base;
    S.n_slices[g] = ns;
    S.n_places[g] = base;
  }
  __threadfence_block();
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < places; i += kLayoutThreads) {
    ent[i] = make_uint2(n, 0u);
    edge[i] = kNoEdge;
  }
  __threadfence_block();
  __syncthreads();
  for (uint32_t i = wave; i < n; i += waves) {
    if (key[i] == kAbsent) continue;
    const int64_t node = n0 + i;
    const uint32_t r = rank[i];
    const bool is_heavy = r < nh;
    const uint32_t s = is_heavy ? r : nh + (r - nh) / 16u;
    const uint32_t b = slices[s].base + (is_heavy ? 0u : (r - nh) % 16u), step = is_heavy ? 1u : 16u;
    const int64_t* off = by_in ? A.in_offset : A.out_offset;
    uint32_t done = 0, outs = 0;
    for (int64_t e = off[node]; e < off[node + 1]; e += kWave) {
      const int64_t k = e + lane;
      const bool in = k < off[node + 1];
      uint32_t other = 0, id = 0;
      bool mine = in;
      if (in) {
        if (by_in) {
          other = A.in_src[k];
          id = (uint32_t)k;
          mine = (A.node_in[other] >= 0) == inputs;
        } else {
          const uint64_t v = A.out_edge[k];
          other = (uint32_t)(v >> 32);
          id = (uint32_t)v;
        }
        other -= (uint32_t)n0;
      }
      const uint64_t m = __ballot(mine);
      if (mine) {
        const uint32_t at = b + step * (done + (uint32_t)__popcll(m & ((1ull << lane) - 1ull)));
        ent[at] = make_uint2(other, __float_as_uint(A.in_w[id]));
        edge[at] = id;
      }
      done += (uint32_t)__popcll(m);
      outs += (uint32_t)__popcll(__ballot(mine && other < A.n_sub));
    }
    if (lane == 0 && outs > 0) atomicMax(&slices[s].first, is_heavy ? (outs + 15u) / 16u : outs);
  }
}

__global__ void __launch_bounds__(kNetThreads) k_learn_weights(LearnWeightsArgs A) {
  const uint32_t g = A.genomes[blockIdx.y];
  for (int which = 0; which < kSets; ++which) {
    const LearnSet S = A.set[which];
    const uint32_t n = S.n_places[g];
    for (uint32_t i = blockIdx.x * kNetThreads + threadIdx.x; i < n; i += gridDim.x * kNetThreads) {
      const uint32_t e = S.edge[A.place[g] + i];
      if (e != kNoEdge) S.ent[A.place[g] + i].y = __float_as_uint(A.in_w[e]);
    }
  }
}

// ----------------------------------------------------------------------------- a genome in LDS

template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
  return v + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(
                 0, (int)__float_as_uint(v), CTRL, 0xF, 0xF, true));
}
constexpr int kDppXor2 = 0x4E, kDppXor1 = 0xB1;
// The sum over a row's LN lanes (of four patterns each).
template <int LN>
__device__ __forceinline__ float row_sum(float v) {
  if constexpr (LN >= 2) v = dpp_add<kDppXor1>(v);
  if constexpr (LN >= 4) v = dpp_add<kDppXor2>(v);
  return v;
}
__device__ __forceinline__ float dot4(const float4& a, const float4& b) {
  return fmaf(a.x, b.x, fmaf(a.y, b.y, fmaf(a.z, b.z, a.w * b.w)));
}
__device__ __forceinline__ void fma4(float4& a, float w, const float4& x) {
  a.x = fmaf(w, x.x, a.x);
  a.y = fmaf(w, x.y, a.y);
  a.z = fmaf(w, x.z, a.z);
  a.w = fmaf(w, x.w, a.w);
}
// The sum over the sixteen places of a heavy slice.
template <int LN>
__device__ __forceinline__ void heavy_sum(float4& a) {
#pragma unroll
  for (int o = LN; o < 16 * LN; o <<= 1) {
    a.x += __shfl_xor(a.x, o, kWave);
    a.y += __shfl_xor(a.y, o, kWave);
    a.z += __shfl_xor(a.z, o, kWave);
    a.w += __shfl_xor(a.w, o, kWave);
  }
}

// What a lane works on: group q of four patterns of the row at place r of a slice.
template <int LN>
struct Place {
  uint32_t q, r;
  uint32_t base, len, full;  // of the slice; `full` past the first edges too
  uint32_t most;             // the longest of the wave's slices
  uint32_t row;              // kNoRow: none
  bool heavy, any_heavy;
  bool writes;               // the lane holds its row's sum
};
// FIRST: only the edges that reach output nodes.
template <int LN, bool FIRST>
__device__ __forceinline__ Place<LN> place_of(const LearnSlice* slices, const uint16_t* rows, uint32_t at,
                                              uint32_t ns, uint32_t lane) {
  Place<LN> P;
  P.q = lane % LN;
  P.r = lane / LN % 16u;
  auto length = [](const LearnSlice& S) {
    return FIRST ? (S.first + kLearnPad - 1u) / kLearnPad * kLearnPad : S.len;
  };
  if constexpr (LN == 4) {  // the wave's slice
    const LearnSlice S = slices[at];
    P.base = S.base;
    P.len = P.most = length(S);
    P.full = S.len;
    P.heavy = P.any_heavy = S.heavy != 0;
    P.row = rows[16u * at + P.r];
  } else {
    P.most = 0;
    P.any_heavy = false;
    for (uint32_t j = 0; j < 4u / LN; ++j) {
      if (at + j >= ns) break;
      const uint32_t l = length(slices[at + j]);
      P.most = l > P.most ? l : P.most;
      P.any_heavy |= slices[at + j].heavy != 0;
    }
    const uint32_t s = at + lane / (16u * LN);
    const bool in = s < ns;
    const LearnSlice S = slices[in ? s : at];
    P.base = S.base;
    P.len = in ? length(S) : 0u;
    P.full = in ? S.len : 0u;
    P.heavy = in && S.heavy != 0;
    P.row = in ? rows[16u * s + P.r] : kNoRow;
  }
  P.writes = P.row != kNoRow && (!P.heavy || P.r == 0);
  return P;
}

// Four edges from the k-th of a lane's row on; a wave whose slices differ in length takes empty ones past
// its own slice's end (lengths are multiples of four).
template <int LN>
__device__ __forceinline__ void edges_at(const uint64_t* __restrict__ e, uint32_t k, const Place<LN>& P,
                                         uint32_t n, uint64_t (&v)[kLearnPad]) {
  if (LN == 4 || k < P.len) {
#pragma unroll
    for (uint32_t j = 0; j < kLearnPad; ++j) v[j] = e[16u * (k + j) + P.r];
  } else {
#pragma unroll
    for (uint32_t j = 0; j < kLearnPad; ++j) v[j] = n;
  }
}

// The weighted sums of a slice's rows over x (the values of the genome's nodes, LN float4 each).
template <int LN>
__device__ __forceinline__ float4 row_sums(const Place<LN>& P, const uint2* __restrict__ ent,
                                           const float4* x, uint32_t n) {
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  if (P.most > 0) {
    const uint64_t* e = reinterpret_cast<const uint64_t*>(ent) + P.base;
    uint64_t a[kLearnPad], b[kLearnPad];
    edges_at<LN>(e, 0, P, n, a);
    for (uint32_t k = kLearnPad;; k += kLearnPad) {
      const bool more = k < P.most;
      if (more) edges_at<LN>(e, k, P, n, b);
#pragma unroll
      for (uint32_t j = 0; j < kLearnPad; ++j)
        fma4(acc, __uint_as_float((uint32_t)(a[j] >> 32)), x[(uint32_t)a[j] * LN + P.q]);
      if (!more) break;
#pragma unroll
      for (uint32_t j = 0; j < kLearnPad; ++j) a[j] = b[j];
    }
  }
  if (P.any_heavy) {
    float4 h = acc;
    heavy_sum<LN>(h);
    if (P.heavy) acc = h;
  }
  return acc;
}

// The same for derivatives gz, and beside it the derivatives of the edges' weights, gz times the row's
// own states s summed over the patterns, added to `sum` at the edges' places (set: stored there, the first
// time; with FIRST, zeros at the places past those).
template <int LN>
__device__ __forceinline__ float4 row_grads(const Place<LN>& P, const uint2* __restrict__ ent,
                                            const float4* gz, uint32_t n, const float4& s,
                                            float* __restrict__ sum, bool set) {
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  if (P.most > 0) {
    const uint64_t* e = reinterpret_cast<const uint64_t*>(ent) + P.base;
    float* mine = sum + P.base;
    // each of a row's lanes adds the derivatives of one edge in LN
    constexpr int own = (int)kLearnPad / LN;
    uint64_t a[kLearnPad], b[kLearnPad];
    float had[own], next[own];
    auto sums_at = [&](uint32_t k, float (&v)[own]) {
#pragma unroll
      for (int c = 0; c < own; ++c)
        v[c] = !set && (LN == 4 || k < P.len) ? mine[16u * (k + (uint32_t)(c * LN) + P.q) + P.r] : 0.0f;
    };
    edges_at<LN>(e, 0, P, n, a);
    sums_at(0, had);
    for (uint32_t k = 0;; k += kLearnPad) {
      const bool more = k + kLearnPad < P.most;
      if (more) {
        edges_at<LN>(e, k + kLearnPad, P, n, b);
        sums_at(k + kLearnPad, next);
      }
      float d[kLearnPad];
#pragma unroll
      for (uint32_t j = 0; j < kLearnPad; ++j) {
        const float4 v = gz[(uint32_t)a[j] * LN + P.q];
        fma4(acc, __uint_as_float((uint32_t)(a[j] >> 32)), v);
        d[j] = row_sum<LN>(dot4(v, s));
      }
#pragma unroll
      for (int c = 0; c < own; ++c) {
        float v = d[c * LN];
#pragma unroll
        for (int j = 1; j < LN; ++j) v = P.q == (uint32_t)j ? d[c * LN + j] : v;
        if (LN == 4 || k < P.len) mine[16u * (k + (uint32_t)(c * LN) + P.q) + P.r] = had[c] + v;
      }
      if (!more) break;
#pragma unroll
      for (uint32_t j = 0; j < kLearnPad; ++j) a[j] = b[j];
#pragma unroll
      for (int c = 0; c < own; ++c) had[c] = next[c];
    }
  }
  if (set)
    for (uint32_t k = P.len + P.q; k < P.full; k += LN) sum[P.base + 16u * k + P.r] = 0.0f;
  if (P.any_heavy) {
    float4 h = acc;
    heavy_sum<LN>(h);
    if (P.heavy) acc = h;
  }
  return acc;
}

__device__ __forceinline__ float sigmoid_f(float z) { return 1.0f / (1.0f + expf(-z)); }
__device__ __forceinline__ uint32_t code_of(float s) { return (uint32_t)__float2uint_rn(255.0f * s); }
// The four codes of a node's state for pattern group pg.
__device__ __forceinline__ uint32_t* kept_at(const NetKept& K, int64_t nodes, uint32_t plane, uint32_t pg,
                                             int64_t node) {
  return reinterpret_cast<uint32_t*>(
      K.codes + (((int64_t)plane * K.blocks + pg / K.q) * nodes + node) * (4 * K.q) + 4 * (pg % K.q));
}
__device__ __forceinline__ float4 pattern4(const LearnArgs& A, int32_t slot, uint32_t pg) {
  float c[4];
#pragma unroll
  for (uint32_t k = 0; k < 4; ++k) {
    const uint32_t p = 4u * pg + k;
    c[k] = p < A.n_patterns ? A.patterns[(int64_t)p * A.n_inputs + (uint32_t)slot] : 0.0f;
  }
  return make_float4(c[0], c[1], c[2], c[3]);
}

// All steps of one genome for an item's blocks of 4 LN patterns: states in LDS as two halves that the steps
// swap and the sums of the input edges, which no step changes. A wave holds a slice of sixteen rows with
// LN lanes each (or 4 / LN slices).
template <int LN>
__device__ __forceinline__ void keep_item(const LearnArgs& A, const LearnItem& I, float4* lds) {
  const uint32_t g = I.genome;
  const int64_t n0 = A.node_offset[g];
  const uint32_t n = (uint32_t)(A.node_offset[g + 1] - n0);
  if (learn_lds(n, LN) > A.lds_bytes) return;  // (host-checked)
  const uint32_t lane = threadIdx.x % kWave;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), waves = blockDim.x / kWave;
  constexpr uint32_t per = 4 / LN;
  const LearnSet &H = A.set[kInHid], &E = A.set[kInInp];
  const uint2 *he = H.ent + A.place[g], *ie = E.ent + A.place[g];
  const LearnSlice *hs = H.slices + A.slice[g], *is = E.slices + A.slice[g];
  const uint16_t *hr = H.rows + 16 * A.slice[g], *ir = E.rows + 16 * A.slice[g];
  const uint32_t hn = H.n_slices[g], in = E.n_slices[g];
  float4 *cur = lds, *nxt = lds + (n + 1u) * LN, *held = nxt + (n + 1u) * LN;
  for (uint32_t b = I.b0; b < I.b1; ++b) {
    for (uint32_t i = threadIdx.x; i < (n + 1u) * LN; i += blockDim.x) {
      const uint32_t node = i / LN;
      const int32_t slot = node < n ? A.node_in[n0 + node] : -1;
      const float4 z = make_float4(0.f, 0.f, 0.f, 0.f);
      cur[i] = slot >= 0 ? pattern4(A, slot, b * LN + i % LN) : z;
      nxt[i] = z;
      held[i] = z;
      if (slot >= 0)
        for (uint32_t t = 0; t < A.kept.planes; ++t)
          *kept_at(A.kept, A.nodes, t, b * LN + i % LN, n0 + node) = 0;
    }
    __syncthreads();
    for (uint32_t at = wave * per; at < in; at += waves * per) {
      const Place<LN> P = place_of<LN, false>(is, ir, at, in, lane);
      const float4 z = row_sums<LN>(P, ie, cur, n);
      if (P.writes) held[P.row * LN + P.q] = z;
    }
    __syncthreads();
    for (uint32_t step = 1; step <= A.steps; ++step) {
      // the last step: output nodes alone, the first slices
      const uint32_t end = step == A.steps ? A.n_outputs : hn;
      for (uint32_t at = wave * per; at < end; at += waves * per) {
        Place<LN> P = place_of<LN, false>(hs, hr, at, end, lane);
        if (step == 1) P.most = 0;  // (hidden states are 0: their edges add nothing)
        float4 z = row_sums<LN>(P, he, cur, n);
        if (!P.writes) continue;
        const float4 y = held[P.row * LN + P.q];
        const float4 s = make_float4(sigmoid_f(z.x + y.x), sigmoid_f(z.y + y.y), sigmoid_f(z.z + y.z),
                                     sigmoid_f(z.w + y.w));
        nxt[P.row * LN + P.q] = s;
        if (step < A.steps)
          *kept_at(A.kept, A.nodes, step - 1, b * LN + P.q, n0 + P.row) =
              code_of(s.x) | code_of(s.y) << 8 | code_of(s.z) << 16 | code_of(s.w) << 24;
      }
      __syncthreads();
      float4* x = cur;
      cur = nxt;
      nxt = x;
    }
    const float* c = reinterpret_cast<const float*>(cur);
    const uint32_t p0 = b * 4u * LN, np = min(A.n_patterns - p0, 4u * LN);
    for (uint32_t i = threadIdx.x; i < np * A.n_outputs; i += blockDim.x) {
      const uint32_t p = i / A.n_outputs, o = i % A.n_outputs;
      A.outputs[((int64_t)g * A.n_patterns + p0 + p) * A.n_outputs + o] =
          c[(uint32_t)A.out_node[o] * 4u * LN + p];
    }
    __syncthreads();
  }
}

template <int LN>
__device__ __forceinline__ void back_item(const LearnArgs& A, const LearnItem& I, float4* lds) {
  const uint32_t g = I.genome;
  const int64_t n0 = A.node_offset[g];
  const uint32_t n = (uint32_t)(A.node_offset[g + 1] - n0);
  if (learn_lds(n, LN) > A.lds_bytes) return;  // (host-checked)
  const uint32_t lane = threadIdx.x % kWave;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), waves = blockDim.x / kWave;
  constexpr uint32_t per = 4 / LN;
  const LearnSet &H = A.set[kOutHid], &E = A.set[kOutInp];
  const uint2 *he = H.ent + A.place[g], *ie = E.ent + A.place[g];
  const LearnSlice *hs = H.slices + A.slice[g], *is = E.slices + A.slice[g];
  const uint16_t *hr = H.rows + 16 * A.slice[g], *ir = E.rows + 16 * A.slice[g];
  const uint32_t hn = H.n_slices[g], in = E.n_slices[g], hp = H.n_places[g], ip = E.n_places[g];
  float *hsum = A.partial + I.part, *isum = hsum + hp;
  float4 *cur = lds, *nxt = lds + (n + 1u) * LN, *all = nxt + (n + 1u) * LN;
  if (A.steps < 2)  // (no step of theirs)
    for (uint32_t i = threadIdx.x; i < hp; i += blockDim.x) hsum[i] = 0.0f;
  for (uint32_t b = I.b0; b < I.b1; ++b) {
    const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
    for (uint32_t i = threadIdx.x; i < (n + 1u) * LN; i += blockDim.x) cur[i] = nxt[i] = all[i] = zero;
    __syncthreads();
    const uint32_t p0 = b * 4u * LN, np = min(A.n_patterns - p0, 4u * LN);
    for (uint32_t i = threadIdx.x; i < np * A.n_outputs; i += blockDim.x) {
      const uint32_t p = i / A.n_outputs, o = i % A.n_outputs;
      const int64_t r = ((int64_t)g * A.n_patterns + p0 + p) * A.n_outputs + o;
      const float v = A.outputs[r], d = A.grad_outputs[r] * v * (1.0f - v);
      const uint32_t at = (uint32_t)A.out_node[o] * 4u * LN + p;
      reinterpret_cast<float*>(cur)[at] = d;
      reinterpret_cast<float*>(all)[at] = d;
    }
    __syncthreads();
    for (uint32_t step = A.steps; step >= 2; --step) {
      const bool last = step == A.steps;  // derivatives at the output nodes alone
      for (uint32_t at = wave * per; at < hn; at += waves * per) {
        const Place<LN> P = last ? place_of<LN, true>(hs, hr, at, hn, lane)
                                 : place_of<LN, false>(hs, hr, at, hn, lane);
        const uint32_t c =
            P.row != kNoRow ? *kept_at(A.kept, A.nodes, step - 2, b * LN + P.q, n0 + P.row) : 0u;
        const float4 d = row_grads<LN>(P, he, cur, n, states(c), hsum, last && b == I.b0);
        if (!P.writes) continue;
        const float4 v = make_float4(d.x * slope_of(c & 255u), d.y * slope_of((c >> 8) & 255u),
                                     d.z * slope_of((c >> 16) & 255u), d.w * slope_of(c >> 24));
        const uint32_t i = P.row * LN + P.q;
        nxt[i] = v;
        const float4 a = all[i];
        all[i] = make_float4(a.x + v.x, a.y + v.y, a.z + v.z, a.w + v.w);
      }
      __syncthreads();
      float4* x = cur;
      cur = nxt;
      nxt = x;
    }
    for (uint32_t at = wave * per; at < in; at += waves * per) {
      const Place<LN> P = place_of<LN, false>(is, ir, at, in, lane);
      const int32_t slot = P.row != kNoRow ? A.node_in[n0 + P.row] : -1;
      const float4 x = slot >= 0 ? pattern4(A, slot, b * LN + P.q) : zero;
      const float4 d = row_grads<LN>(P, ie, all, n, x, isum, b == I.b0);
      if (!A.grad_inputs || !P.writes) continue;
      const float v[4] = {d.x, d.y, d.z, d.w};
#pragma unroll
      for (uint32_t k = 0; k < 4; ++k) {
        const uint32_t p = p0 + 4u * P.q + k;
        if (p < A.n_patterns)
          A.grad_inputs[((int64_t)g * A.n_patterns + p) * A.n_inputs + (uint32_t)slot] = v[k];
      }
    }
    __syncthreads();
  }
  if (!I.alone) return;
  __threadfence_block();
  __syncthreads();
  const uint32_t *hi = H.edge + A.place[g], *ii = E.edge + A.place[g];
  for (uint32_t i = threadIdx.x; i < hp; i += blockDim.x)
    if (hi[i] != kNoEdge) A.grad_w[hi[i]] = hsum[i];
  for (uint32_t i = threadIdx.x; i < ip; i += blockDim.x)
    if (ii[i] != kNoEdge) A.grad_w[ii[i]] = isum[i];
}

template <bool BACK>
__global__ void __launch_bounds__(1024, 4) k_learn(LearnArgs A) {
  extern __shared__ float4 learn_lds_mem[];
  const LearnItem I = A.items[A.first_item + blockIdx.x];
  switch (I.groups) {
    case 1: BACK ? back_item<1>(A, I, learn_lds_mem) : keep_item<1>(A, I, learn_lds_mem); break;
    case 2: BACK ? back_item<2>(A, I, learn_lds_mem) : keep_item<2>(A, I, learn_lds_mem); break;
    default: BACK ? back_item<4>(A, I, learn_lds_mem) : keep_item<4>(A, I, learn_lds_mem); break;
  }
}

// One step of genomes too large for that, or too few to fill the chip: a workgroup holds all nodes' values of a
// block of patterns and takes a share of the slices.
template <int LN>
__device__ __forceinline__ void keep_step(const LearnArgs& A, const LearnStepItem& I, float4* lds) {
  const uint32_t g = I.genome;
  const int64_t n0 = A.node_offset[g];
  const uint32_t n = (uint32_t)(A.node_offset[g + 1] - n0);
  if (step_lds(n, LN) > A.lds_bytes) return;  // (host-checked)
  const uint32_t lane = threadIdx.x % kWave;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), waves = blockDim.x / kWave;
  constexpr uint32_t per = 4 / LN;
  const bool first = A.step == 1, last = A.step == A.steps;
  const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
  const float4* cur = A.cur + I.values;
  float4 *nxt = A.nxt + I.values, *held = A.held + I.values;
  const LearnSet& E = A.set[first ? kInInp : kInHid];
  const uint2* ent = E.ent + A.place[g];
  const LearnSlice* slices = E.slices + A.slice[g];
  const uint16_t* rows = E.rows + 16 * A.slice[g];
  for (uint32_t i = threadIdx.x; i < (n + 1u) * LN; i += blockDim.x) {
    const uint32_t node = i / LN;
    float4 v = zero;
    if (first) {  // the patterns; and what nodes without input edges hold
      const int32_t slot = node < n ? A.node_in[n0 + node] : -1;
      if (slot >= 0) v = pattern4(A, slot, I.block * LN + i % LN);
      if (I.chunk == 0 && slot >= 0)
        for (uint32_t t = 0; t < A.kept.planes; ++t)
          *kept_at(A.kept, A.nodes, t, I.block * LN + i % LN, n0 + node) = 0;
    } else if (node < n) {
      v = cur[i];
    }
    lds[i] = v;
  }
  __syncthreads();
  auto put = [&](uint32_t row, uint32_t q, const float4& z) {
    const float4 s = make_float4(sigmoid_f(z.x), sigmoid_f(z.y), sigmoid_f(z.z), sigmoid_f(z.w));
    nxt[row * LN + q] = s;
    if (!last)
      *kept_at(A.kept, A.nodes, A.step - 1, I.block * LN + q, n0 + row) =
          code_of(s.x) | code_of(s.y) << 8 | code_of(s.z) << 16 | code_of(s.w) << 24;
  };
  const uint32_t end = first ? E.n_slices[g] : (last ? A.n_outputs : E.n_slices[g]);
  for (uint32_t at = (wave * I.chunks + I.chunk) * per; at < end; at += waves * I.chunks * per) {
    const Place<LN> P = place_of<LN, false>(slices, rows, at, end, lane);
    const float4 z = row_sums<LN>(P, ent, lds, n);
    if (!P.writes) continue;
    const uint32_t i = P.row * LN + P.q;
    if (first) {
      held[i] = z;
      put(P.row, P.q, z);
    } else {
      const float4 y = held[i];
      put(P.row, P.q, make_float4(z.x + y.x, z.y + y.y, z.z + y.z, z.w + y.w));
    }
  }
}

template <int LN>
__device__ __forceinline__ void back_step(const LearnArgs& A, const LearnStepItem& I, float4* lds) {
  const uint32_t g = I.genome;
  const int64_t n0 = A.node_offset[g];
  const uint32_t n = (uint32_t)(A.node_offset[g + 1] - n0);
  if (step_lds(n, LN) > A.lds_bytes) return;  // (host-checked)
  const uint32_t lane = threadIdx.x % kWave;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), waves = blockDim.x / kWave;
  constexpr uint32_t per = 4 / LN;
  const bool inputs = A.step == 1, last = A.step == A.steps;
  const LearnSet &H = A.set[kOutHid], &E = A.set[inputs ? kOutInp : kOutHid];
  const uint2* ent = E.ent + A.place[g];
  const LearnSlice* slices = E.slices + A.slice[g];
  const uint16_t* rows = E.rows + 16 * A.slice[g];
  float* sum = A.partial + I.part + (inputs ? H.n_places[g] : 0u);
  const float4* from = (inputs ? A.held : A.cur) + I.values;
  float4 *nxt = A.nxt + I.values, *all = A.held + I.values;
  const uint32_t p0 = I.block * 4u * LN, np = min(A.n_patterns - p0, 4u * LN);
  // the derivatives after the step (of all steps); those after the last are at the output nodes alone
  for (uint32_t i = threadIdx.x; i < (n + 1u) * LN; i += blockDim.x)
    lds[i] = last || i >= n * LN ? make_float4(0.f, 0.f, 0.f, 0.f) : from[i];
  __syncthreads();
  if (last) {
    for (uint32_t i = threadIdx.x; i < np * A.n_outputs; i += blockDim.x) {
      const uint32_t p = i / A.n_outputs, o = i % A.n_outputs;
      const int64_t r = ((int64_t)g * A.n_patterns + p0 + p) * A.n_outputs + o;
      const float v = A.outputs[r];
      reinterpret_cast<float*>(lds)[(uint32_t)A.out_node[o] * 4u * LN + p] = A.grad_outputs[r] * v * (1.0f - v);
    }
    __syncthreads();
  }
  if (inputs && last)  // (one step: the other edges have no part)
    for (uint32_t i = I.chunk * blockDim.x + threadIdx.x; i < H.n_places[g]; i += I.chunks * blockDim.x)
      A.partial[I.part + i] = 0.0f;
  const uint32_t end = E.n_slices[g];
  for (uint32_t at = (wave * I.chunks + I.chunk) * per; at < end; at += waves * I.chunks * per) {
    const Place<LN> P = last && !inputs ? place_of<LN, true>(slices, rows, at, end, lane)
                                        : place_of<LN, false>(slices, rows, at, end, lane);
    if (inputs) {
      const int32_t slot = P.row != kNoRow ? A.node_in[n0 + P.row] : -1;
      const float4 x = slot >= 0 ? pattern4(A, slot, I.block * LN + P.q) : make_float4(0.f, 0.f, 0.f, 0.f);
      const float4 d = row_grads<LN>(P, ent, lds, n, x, sum, true);
      if (!A.grad_inputs || !P.writes) continue;
      const float v[4] = {d.x, d.y, d.z, d.w};
#pragma unroll
      for (uint32_t k = 0; k < 4; ++k) {
        const uint32_t p = p0 + 4u * P.q + k;
        if (p < A.n_patterns)
          A.grad_inputs[((int64_t)g * A.n_patterns + p) * A.n_inputs + (uint32_t)slot] = v[k];
      }
      continue;
    }
    const uint32_t c =
        P.row != kNoRow ? *kept_at(A.kept, A.nodes, A.step - 2, I.block * LN + P.q, n0 + P.row) : 0u;
    const float4 d = row_grads<LN>(P, ent, lds, n, states(c), sum, last);
    if (!P.writes) continue;
    const float4 v = make_float4(d.x * slope_of(c & 255u), d.y * slope_of((c >> 8) & 255u),
                                 d.z * slope_of((c >> 16) & 255u), d.w * slope_of(c >> 24));
    const uint32_t i = P.row * LN + P.q;
    nxt[i] = v;
    const float4 a = last ? lds[i] : all[i];
    all[i] = make_float4(a.x + v.x, a.y + v.y, a.z + v.z, a.w + v.w);
  }
}

template <bool BACK>
__global__ void __launch_bounds__(1024, 4) k_learn_step(LearnArgs A) {
  extern __shared__ float4 learn_lds_mem[];
  const LearnStepItem I = A.step_items[A.first_item + blockIdx.x];
  switch (I.groups) {
    case 1: BACK ? back_step<1>(A, I, learn_lds_mem) : keep_step<1>(A, I, learn_lds_mem); break;
    case 2: BACK ? back_step<2>(A, I, learn_lds_mem) : keep_step<2>(A, I, learn_lds_mem); break;
    default: BACK ? back_step<4>(A, I, learn_lds_mem) : keep_step<4>(A, I, learn_lds_mem); break;
  }
}

// The outputs of stepped genomes, from their states after the last step.
__global__ void __launch_bounds__(kNetThreads) k_step_outputs(LearnArgs A) {
  const LearnStepItem I = A.step_items[A.first_item + blockIdx.x];
  if (I.chunk != 0) return;
  const float* v = reinterpret_cast<const float*>(A.cur + I.values);
  const uint32_t wide = 4u * I.groups, p0 = I.block * wide, np = min(A.n_patterns - p0, wide);
  for (uint32_t i = threadIdx.x; i < np * A.n_outputs; i += kNetThreads) {
    const uint32_t p = i / A.n_outputs, o = i % A.n_outputs;
    A.outputs[((int64_t)I.genome * A.n_patterns + p0 + p) * A.n_outputs + o] =
        A.steps ? v[(uint32_t)A.out_node[o] * wide + p] : 0.0f;
  }
}

// The items' sums of genomes with more than one, in the items' order.
__global__ void __launch_bounds__(kNetThreads) k_learn_join(LearnArgs A) {
  const LearnJoin J = A.joins[blockIdx.y];
  const LearnSet &H = A.set[kOutHid], &E = A.set[kOutInp];
  const uint32_t hp = H.n_places[J.genome], all = hp + E.n_places[J.genome];
  const uint32_t *hi = H.edge + A.place[J.genome], *ii = E.edge + A.place[J.genome];
  for (uint32_t i = blockIdx.x * kNetThreads + threadIdx.x; i < all; i += gridDim.x * kNetThreads) {
    const uint32_t e = i < hp ? hi[i] : ii[i - hp];
    if (e == kNoEdge) continue;
    const float* p = A.partial + J.part + i;
    float sum = 0.0f;
    uint32_t k = 0;
    for (; k + 8 <= J.items; k += 8) {
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = p[(k + j) * J.stride];
#pragma unroll
      for (int j = 0; j < 8; ++j) sum += v[j];
    }
    for (; k < J.items; ++k) sum += p[k * J.stride];
    A.grad_w[e] = sum;
  }
}

uint32_t stride_blocks(int64_t n) {
  const int64_t b = (n + kNetThreads - 1) / kNetThreads;
  return (uint32_t)(b < 1 ? 1 : (b > 16384 ? 16384 : b));
}

}  // namespace
}  // namespace emr

// Steps: 0 the edges' keys by source, 1 their offsets (after the sort), 2 a layout, 3 its weights; all steps
// of the genomes in LDS: 4 activation, 5 gradients, 6 their joined sums; one step of others: 11 activation, 12
// gradients, 13 the outputs; a genome larger than the LDS: 7 the derivatives by
// the outputs' sums into gz_before (the other half behind it cleared), 8 one step's weight derivatives, 9 one
// step backwards; 10 zeros.
extern "C" hipError_t emr_launch_learn(int step, const void* args, hipStream_t s) {
  using namespace emr;
  const dim3 blk(kNetThreads);
  switch (step) {
    case 0: {
      const auto& A = *static_cast<const NetTurnArgs*>(args);
      hipLaunchKernelGGL(k_turn_keys, dim3(stride_blocks(A.nodes * kWave)), blk, 0, s, A);
      break;
    }
    case 1: {
      const auto& A = *static_cast<const NetTurnArgs*>(args);
      hipLaunchKernelGGL(k_turn_offsets, dim3(stride_blocks(A.nodes + 1)), blk, 0, s, A);
      break;
    }
    case 2: {
      const auto& A = *static_cast<const LearnLayoutArgs*>(args);
      if (A.count == 0) return hipSuccess;
      hipLaunchKernelGGL(k_learn_layout, dim3(A.count, kSets), dim3(kLayoutThreads), 0, s, A);
      break;
    }
    case 3: {
      const auto& A = *static_cast<const LearnWeightsArgs*>(args);
      for (uint32_t a = 0; a < A.count; a += 65535u) {
        LearnWeightsArgs B = A;
        B.genomes = A.genomes + a;
        hipLaunchKernelGGL(k_learn_weights, dim3(16, A.count - a < 65535u ? A.count - a : 65535u), blk, 0, s,
                           B);
      }
      break;
    }
    case 4:
    case 5: {
      const auto& A = *static_cast<const LearnArgs*>(args);
      if (A.n_items == 0) return hipSuccess;
      if (A.lds_bytes > kLearnLds || A.threads == 0 || A.threads > 1024u || A.threads % kWave != 0)
        return hipErrorInvalidValue;
      if (step == 4)
        hipLaunchKernelGGL(k_learn<false>, dim3(A.n_items), dim3(A.threads), A.lds_bytes, s, A);
      else
        hipLaunchKernelGGL(k_learn<true>, dim3(A.n_items), dim3(A.threads), A.lds_bytes, s, A);
      break;
    }
    case 6: {
      const auto& A = *static_cast<const LearnArgs*>(args);
      for (uint32_t a = 0; a < A.n_joins; a += 65535u) {
        LearnArgs B = A;
        B.joins = A.joins + a;
        hipLaunchKernelGGL(k_learn_join, dim3(64, A.n_joins - a < 65535u ? A.n_joins - a : 65535u), blk, 0, s,
                           B);
      }
      break;
    }
    case 7: {
      const auto& A = *static_cast<const NetBackArgs*>(args);
      const int64_t n = 8 * (int64_t)A.pblocks * A.size;  // (both halves: input nodes stay 0)
      hipLaunchKernelGGL(k_back_clear, dim3(stride_blocks(n)), blk, 0, s, LearnFillArgs{A.gz_before, n});
      hipLaunchKernelGGL(k_back_outputs, dim3(stride_blocks((int64_t)A.n_patterns * A.n_outputs)), blk, 0, s,
                         A);
      break;
    }
    case 8: {
      const auto& A = *static_cast<const NetBackArgs*>(args);
      if (A.edge1 <= A.edge0) return hipSuccess;
      hipLaunchKernelGGL(k_back_edges, dim3(stride_blocks(A.edge1 - A.edge0)), blk, 0, s, A);
      break;
    }
    case 9: {
      const auto& A = *static_cast<const NetBackArgs*>(args);
      hipLaunchKernelGGL(k_back_nodes,
                         dim3(stride_blocks(A.size * kWave), 1, A.pblocks < 64u ? A.pblocks : 64u), blk, 0, s,
                         A);
      break;
    }
    case 10: {
      const auto& A = *static_cast<const LearnFillArgs*>(args);
      if (A.n <= 0) return hipSuccess;
      hipLaunchKernelGGL(k_back_clear, dim3(stride_blocks(A.n)), blk, 0, s, A);
      break;
    }
    case 11:
    case 12:
    case 13: {
      const auto& A = *static_cast<const LearnArgs*>(args);
      if (A.n_items == 0) return hipSuccess;
      if (A.lds_bytes > kLearnLds || A.threads == 0 || A.threads > 1024u || A.threads % kWave != 0)
        return hipErrorInvalidValue;
      if (step == 11)
        hipLaunchKernelGGL(k_learn_step<false>, dim3(A.n_items), dim3(A.threads), A.lds_bytes, s, A);
      else if (step == 12)
        hipLaunchKernelGGL(k_learn_step<true>, dim3(A.n_items), dim3(A.threads), A.lds_bytes, s, A);
      else
        hipLaunchKernelGGL(k_step_outputs, dim3(A.n_items), blk, 0, s, A);
      break;
    }
    default:
      return hipErrorInvalidValue;
  }
  return hipGetLastError();
}
