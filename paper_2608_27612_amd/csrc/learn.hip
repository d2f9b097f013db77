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

__device__ __forceinline__ bool by_destination(int which) { return which == kInHid || which == kInInp; }
__device__ __forceinline__ bool of_inputs(int which) { return which == kInInp || which == kOutInp; }

// A wave for a node: the edges of its row.
__global__ void __launch_bounds__(kNetThreads) k_layout_degrees(LearnLayoutArgs A) {
  const uint32_t lane = threadIdx.x % kWave;
  const bool in = by_destination(A.which), inputs = of_inputs(A.which);
  for (int64_t i = grid_thread() / kWave; i < A.nodes; i += grid_threads() / kWave) {
    const bool is_input = A.node_in[i] >= 0;
    uint32_t d = kNoEdge;
    if (!in) {
      if (is_input == inputs) d = (uint32_t)(A.out_offset[i + 1] - A.out_offset[i]);
    } else if (!is_input) {
      const int64_t e1 = A.in_offset[i + 1];
      d = 0;
      for (int64_t e = A.in_offset[i]; e < e1; e += kWave) {
        const int64_t k = e + lane;
        d += (uint32_t)__popcll(__ballot(k < e1 && (A.node_in[A.in_src[k < e1 ? k : e]] >= 0) == inputs));
      }
    }
    if (lane == 0) A.key[i] = d;
  }
}

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
// (kLayoutBins: the last one holds the output nodes of kInHid, the one before it all longer rows)
// A workgroup for a genome: its rows ranked by falling edges (equal ones by node), its slices, and where each
// row's edges go.
__global__ void __launch_bounds__(kLayoutThreads) k_layout_slices(LearnLayoutArgs A) {
  __shared__ uint32_t bin[kLayoutBins];  // rows of it, then the rank of its next one
  __shared__ uint32_t key[kLayoutThreads];
  __shared__ uint32_t part[kLayoutThreads / kWave];
  __shared__ uint32_t edges;
  const uint32_t g = A.genomes[blockIdx.x];
  const LearnSet& S = A.set;
  if (threadIdx.x == 0) edges = 0;
  const int64_t n0 = A.node_offset[g];
  const uint32_t n = (uint32_t)(A.node_offset[g + 1] - n0);
  LearnSlice* slices = S.slices + A.slice[g];
  uint16_t* row_of = S.rows + 16 * A.slice[g];
  if (A.which == kInHid)
    for (uint32_t o = threadIdx.x; o < A.n_outputs; o += kLayoutThreads)
      A.key[n0 + A.out_node[o]] |= 0x80000000u;
  for (uint32_t i = threadIdx.x; i < kLayoutBins; i += kLayoutThreads) bin[i] = 0;
  __threadfence_block();
  __syncthreads();
  auto bin_of = [](uint32_t k) {
    return k & 0x80000000u ? kLayoutBins - 1u : (k < kLayoutBins - 2u ? k : kLayoutBins - 2u);
  };
  for (uint32_t i = threadIdx.x; i < n; i += kLayoutThreads) {
    const uint32_t k = A.key[n0 + i];
    if (k == kNoEdge) continue;
    atomicAdd(&bin[bin_of(k)], 1u);
    atomicAdd(&edges, k & 0x7FFFFFFFu);
  }
  __syncthreads();
  // ranks of the bins' first rows, from the last bin down
  uint32_t rows = 0, nh = 0;
  {
    static_assert(kLayoutBins == 2 * kLayoutThreads, "two bins to a thread");
    const uint32_t b = kLayoutBins - 1u - 2u * threadIdx.x;
    const uint32_t c0 = bin[b], c1 = bin[b - 1];
    const uint32_t at = block_scan(c0 + c1, part, &rows);
    bin[b] = at;
    bin[b - 1] = at + c0;
    __syncthreads();
    nh = bin[light_edges(edges, rows)];  // (rows of more edges)
    __syncthreads();
  }
  const uint32_t ns = nh + (rows - nh + 15u) / 16u;
  for (uint32_t i0 = 0; i0 < n; i0 += kLayoutThreads) {
    const uint32_t i = i0 + threadIdx.x;
    const uint32_t k = i < n ? A.key[n0 + i] : kNoEdge;
    const uint32_t mine = k == kNoEdge ? kNoEdge : bin_of(k);
    key[threadIdx.x] = mine;
    __syncthreads();
    uint32_t before = 0;
    for (uint32_t j = 0; j < threadIdx.x; ++j) before += key[j] == mine ? 1u : 0u;
    const uint32_t r = mine == kNoEdge ? kNoEdge : bin[mine] + before;
    __syncthreads();
    if (mine != kNoEdge) {
      atomicAdd(&bin[mine], 1u);
      if (r < nh) {
        slices[r] = {0, padded(((k & 0x7FFFFFFFu) + 15u) / 16u), 0, 1};
        for (uint32_t j = 0; j < 16; ++j) row_of[16u * r + j] = (uint16_t)i;
      } else {
        const uint32_t s = nh + (r - nh) / 16u;
        if ((r - nh) % 16u == 0) slices[s] = {0, padded(k), 0, 0};
        row_of[16u * s + (r - nh) % 16u] = (uint16_t)i;
      }
    }
    if (i < n) A.row[n0 + i] = {0, (uint32_t)n0, r};
    __syncthreads();
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
    S.n_slices[g] = ns;
    S.n_heavy[g] = nh;
    S.n_places[g] = base;
  }
  __threadfence_block();
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < n; i += kLayoutThreads) {
    const uint32_t r = A.row[n0 + i].slice;
    if (r == kNoEdge) continue;
    const uint32_t s = r < nh ? r : nh + (r - nh) / 16u;
    A.row[n0 + i] = {A.place[g] + slices[s].base + (r < nh ? 0u : (r - nh) % 16u), (uint32_t)n0,
                     s | (r < nh ? 0x80000000u : 0u)};
  }
  uint2* ent = S.ent + A.place[g];
  uint32_t* edge = S.edge + A.place[g];
  for (uint32_t i = threadIdx.x; i < base; i += kLayoutThreads) {
    ent[i] = make_uint2(n, 0u);
    edge[i] = kNoEdge;
  }
}

// A wave for a node: its row's edges to their places. (blockIdx.y: the genome's number in the list.)
__global__ void __launch_bounds__(kNetThreads) k_layout_fill(LearnLayoutArgs A) {
  const uint32_t lane = threadIdx.x % kWave;
  const bool by_in = by_destination(A.which), inputs = of_inputs(A.which);
  const uint32_t g = A.genomes[blockIdx.y];
  const int64_t end = A.node_offset[g + 1];
  LearnSlice* slices = A.set.slices + A.slice[g];
  const int64_t* off = by_in ? A.in_offset : A.out_offset;
  for (int64_t i = A.node_offset[g] + grid_thread() / kWave; i < end; i += grid_threads() / kWave) {
    const LearnRow R = A.row[i];
    if (R.slice == kNoEdge) continue;
    const bool heavy = R.slice >> 31;
    const uint32_t step = heavy ? 1u : 16u;
    uint32_t done = 0, outs = 0;
    for (int64_t e = off[i]; e < off[i + 1]; e += kWave) {
      const int64_t k = e + lane;
      uint32_t other = 0, id = 0;
      bool mine = k < off[i + 1];
      if (mine) {
        if (by_in) {
          other = A.in_src[k];
          id = (uint32_t)k;
          mine = (A.node_in[other] >= 0) == inputs;
        } else {
          const uint64_t v = A.out_edge[k];
          other = (uint32_t)(v >> 32);
          id = (uint32_t)v;
        }
        other -= R.node0;
      }
      const uint64_t m = __ballot(mine);
      if (mine) {
        const int64_t at = R.place + (int64_t)step * (done + (uint32_t)__popcll(m & ((1ull << lane) - 1ull)));
        A.set.ent[at] = make_uint2(other, __float_as_uint(A.in_w[id]));
        A.set.edge[at] = id;
      }
      done += (uint32_t)__popcll(m);
      outs += (uint32_t)__popcll(__ballot(mine && other < A.n_sub));
    }
    if (lane == 0 && outs > 0)
      atomicMax(&slices[R.slice & 0x7FFFFFFFu].first, heavy ? (outs + 15u) / 16u : outs);
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

// ----------------------------------------------------------------------------- rows

template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
  return v + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(
                 0, (int)__float_as_uint(v), CTRL, 0xF, 0xF, true));
}
constexpr int kDppXor2 = 0x4E, kDppXor1 = 0xB1, kDppHalfMirror = 0x141;
// The sum over a row's LN lanes. (The mirror of eight lanes pairs a lane with one of the other four.)
template <int LN>
__device__ __forceinline__ float row_sum(float v) {
  if constexpr (LN >= 2) v = dpp_add<kDppXor1>(v);
  if constexpr (LN >= 4) v = dpp_add<kDppXor2>(v);
  if constexpr (LN >= 8) v = dpp_add<kDppHalfMirror>(v);
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

// One of a genome's layouts.
struct Rows {
  const uint64_t* ent;
  const LearnSlice* slices;
  const uint16_t* rows;
  uint32_t n, heavy;  // slices
};
__device__ __forceinline__ Rows rows_of(const LearnArgs& A, int which, uint32_t g) {
  const LearnSet& S = A.set[which];
  return {reinterpret_cast<const uint64_t*>(S.ent + A.place[g]), S.slices + A.slice[g],
          S.rows + 16 * A.slice[g], S.n_slices[g], S.n_heavy[g]};
}
// A wave takes a heavy slice, or the rows of 64 / LN light places, at a time: units of work.
template <int LN>
__device__ __forceinline__ uint32_t units_of(const Rows& R) {
  const uint32_t light = R.n - R.heavy;
  return R.heavy + (LN > 4 ? light * (LN / 4) : (light + 4 / LN - 1) / (4 / LN));
}

// What a lane does of a unit: lane q of the LN of its row, edges off + step k, k < count.
template <int LN>
struct Place {
  uint32_t q, off, step;
  uint32_t count, most, full;  // the lane's edges, the most of the wave's lanes', those past the first too
  uint32_t row;                // kNoRow: none
  bool heavy;                  // (the wave's)
  bool writes;                 // the lane holds its row's sum
};
// FIRST: only the edges that reach output nodes.
template <int LN, bool FIRST>
__device__ __forceinline__ Place<LN> place_of(const Rows& R, uint32_t unit, uint32_t lane) {
  Place<LN> P;
  P.q = lane % LN;
  P.heavy = unit < R.heavy;
  if (P.heavy) {
    constexpr uint32_t each = kWave / LN;  // edges at a time
    const LearnSlice S = R.slices[unit];
    P.off = S.base + lane / LN;
    P.step = each;
    P.full = 16u * S.len / each;
    P.count = FIRST ? (16u * S.first + each - 1u) / each : P.full;
    if (LN >= 4) P.count = padded(P.count);
    P.most = P.count;
    P.row = R.rows[16u * unit];
    P.writes = lane < (uint32_t)LN;
    return P;
  }
  P.step = 16;
  if constexpr (LN >= 4) {  // the wave's slice (or half of one)
    constexpr uint32_t parts = LN / 4;
    const uint32_t s = R.heavy + (unit - R.heavy) / parts;
    const uint32_t r = (unit - R.heavy) % parts * (16u / parts) + lane / LN;
    const LearnSlice S = R.slices[s];
    P.off = S.base + r;
    P.full = S.len;
    P.count = P.most = FIRST ? padded(S.first) : S.len;
    P.row = R.rows[16u * s + r];
  } else {
    const uint32_t r = lane / LN % 16u;
    const uint32_t s0 = R.heavy + (unit - R.heavy) * (4u / LN);
    P.most = 0;
    for (uint32_t j = 0; j < 4u / LN && s0 + j < R.n; ++j) {
      const uint32_t l = FIRST ? R.slices[s0 + j].first : R.slices[s0 + j].len;
      P.most = l > P.most ? l : P.most;
    }
    const uint32_t s = s0 + lane / (16u * LN);
    const bool in = s < R.n;
    const LearnSlice S = R.slices[in ? s : s0];
    P.off = S.base + r;
    P.full = in ? S.len : 0u;
    P.count = in ? (FIRST ? S.first : S.len) : 0u;
    P.row = in ? R.rows[16u * s + r] : kNoRow;
  }
  P.writes = P.row != kNoRow;
  return P;
}

// Four of a lane's edges from the k-th on: from four lanes to a row on, all lanes of a wave have as many, a
// multiple of four; else empty ones past a lane's own. (The address is the wave's, but for a lane's constant
// offsets.)
template <int LN>
__device__ __forceinline__ void edges_at(const uint64_t* __restrict__ e, uint32_t k, const Place<LN>& P,
                                         uint32_t n, uint64_t (&v)[kLearnPad]) {
  const uint64_t* at = e + P.step * k;
#pragma unroll
  for (uint32_t j = 0; j < kLearnPad; ++j) {
    v[j] = n;
    if (LN >= 4 || k + j < P.count) v[j] = at[P.off + P.step * j];
  }
}

// The sum over the lanes of a heavy slice.
template <int LN>
__device__ __forceinline__ void heavy_sum(float4& a) {
#pragma unroll
  for (int o = LN; o < kWave; o <<= 1) {
    a.x += __shfl_xor(a.x, o, kWave);
    a.y += __shfl_xor(a.y, o, kWave);
    a.z += __shfl_xor(a.z, o, kWave);
    a.w += __shfl_xor(a.w, o, kWave);
  }
}

// The loops below hold kAhead fours of edges: while one is worked on, the loads of the others are under way.

// The weighted sums of a unit's rows over x (the values of the genome's nodes, LN float4 each).
template <int LN>
__device__ __forceinline__ float4 row_sums(const Place<LN>& P, const uint64_t* __restrict__ e, const float4* x,
                                           uint32_t n) {
  constexpr uint32_t kAhead = 3;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  uint64_t a[kAhead][kLearnPad];
#pragma unroll
  for (uint32_t i = 0; i < kAhead; ++i)
    if (i * kLearnPad < P.most) edges_at<LN>(e, i * kLearnPad, P, n, a[i]);
  for (uint32_t k = 0; k < P.most; k += kAhead * kLearnPad) {
#pragma unroll
    for (uint32_t i = 0; i < kAhead; ++i) {
      if (k + i * kLearnPad >= P.most) break;
#pragma unroll
      for (uint32_t j = 0; j < kLearnPad; ++j)
        fma4(acc, __uint_as_float((uint32_t)(a[i][j] >> 32)), x[(uint32_t)a[i][j] * LN + P.q]);
      if (k + (i + kAhead) * kLearnPad < P.most) edges_at<LN>(e, k + (i + kAhead) * kLearnPad, P, n, a[i]);
    }
  }
  if (P.heavy) heavy_sum<LN>(acc);
  return acc;
}

// The same for derivatives gz, and beside it the derivatives of the edges' weights, gz times the row's
// own states s summed over the patterns, added to `sum` at the edges' places (set: stored there, the first
// time; with FIRST, zeros at the places past those). An edge's derivative, read once from LDS, serves both.
template <int LN>
__device__ __forceinline__ float4 row_grads(const Place<LN>& P, const uint64_t* __restrict__ e, const float4* gz,
                                            uint32_t n, const float4& s, float* __restrict__ sum, bool set) {
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  constexpr int kAhead = 2;  // (three spill)
  // a row's lanes (four of them) share the adding of four edges' derivatives
  constexpr int four = LN < (int)kLearnPad ? LN : (int)kLearnPad, own = (int)kLearnPad / four;
  uint64_t a[kAhead][kLearnPad];
  float had[kAhead][own];
  const uint32_t mine = P.off + P.step * P.q;
  auto adds = [&](uint32_t k, int c) {
    return LN >= 4 ? P.q < (uint32_t)four : k + (uint32_t)(c * four) + P.q < P.count;
  };
  auto load = [&](uint32_t k, int i) {
    edges_at<LN>(e, k, P, n, a[i]);
#pragma unroll
    for (int c = 0; c < own; ++c)
      had[i][c] = !set && adds(k, c) ? (sum + P.step * k)[mine + P.step * (c * four)] : 0.0f;
  };
#pragma unroll
  for (int i = 0; i < kAhead; ++i)
    if ((uint32_t)i * kLearnPad < P.most) load((uint32_t)i * kLearnPad, i);
  for (uint32_t k0 = 0; k0 < P.most; k0 += kAhead * kLearnPad) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const uint32_t k = k0 + (uint32_t)i * kLearnPad;
      if (k >= P.most) break;
      float d[kLearnPad];
#pragma unroll
      for (uint32_t j = 0; j < kLearnPad; ++j) {
        const float4 v = gz[(uint32_t)a[i][j] * LN + P.q];
        fma4(acc, __uint_as_float((uint32_t)(a[i][j] >> 32)), v);
        d[j] = row_sum<LN>(dot4(v, s));
      }
#pragma unroll
      for (int c = 0; c < own; ++c) {
        float v = d[c * four];
#pragma unroll
        for (int j = 1; j < four; ++j) v = P.q == (uint32_t)j ? d[c * four + j] : v;
        if (adds(k, c)) (sum + P.step * k)[mine + P.step * (c * four)] = had[i][c] + v;
      }
      if (k + kAhead * kLearnPad < P.most) load(k + kAhead * kLearnPad, i);
    }
  }
  if (set)
    for (uint32_t k = P.count + P.q; k < P.full; k += LN) sum[P.off + P.step * k] = 0.0f;
  if (P.heavy) heavy_sum<LN>(acc);
  return acc;
}

__device__ __forceinline__ float sigmoid_f(float z) { return 1.0f / (1.0f + expf(-z)); }
__device__ __forceinline__ float4 sigmoid4(const float4& z) {
  return make_float4(sigmoid_f(z.x), sigmoid_f(z.y), sigmoid_f(z.z), sigmoid_f(z.w));
}
__device__ __forceinline__ float4 add4(const float4& a, const float4& b) {
  return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w);
}
__device__ __forceinline__ uint32_t code_of(float s) { return (uint32_t)__float2uint_rn(255.0f * s); }
__device__ __forceinline__ uint32_t codes_of(const float4& s) {
  return code_of(s.x) | code_of(s.y) << 8 | code_of(s.z) << 16 | code_of(s.w) << 24;
}
// d s (1 - s) for four codes.
__device__ __forceinline__ float4 slopes(const float4& d, uint32_t c) {
  return make_float4(d.x * slope_of(c & 255u), d.y * slope_of((c >> 8) & 255u), d.z * slope_of((c >> 16) & 255u),
                     d.w * slope_of(c >> 24));
}
// The four codes of a node's state for pattern group pg.
__device__ __forceinline__ uint32_t* kept_at(const NetKept& K, int64_t nodes, uint32_t plane, uint32_t pg,
                                             int64_t node) {
  return reinterpret_cast<uint32_t*>(
      K.codes + (((int64_t)plane * K.blocks + pg / K.q) * nodes + node) * (4 * K.q) + 4 * (pg % K.q));
}
// (a block's last groups may lie past the codes' blocks, whose patterns do not exist)
__device__ __forceinline__ bool kept_in(const NetKept& K, uint32_t pg) { return pg < K.blocks * K.q; }
__device__ __forceinline__ float4 pattern4(const LearnArgs& A, int32_t slot, uint32_t pg) {
  float c[4];
#pragma unroll
  for (uint32_t k = 0; k < 4; ++k) {
    const uint32_t p = 4u * pg + k;
    c[k] = p < A.n_patterns ? A.patterns[(int64_t)p * A.n_inputs + (uint32_t)slot] : 0.0f;
  }
  return make_float4(c[0], c[1], c[2], c[3]);
}
// A block's patterns at the input nodes, 0 elsewhere and past the last node; the input nodes' codes.
template <int W>
__device__ __forceinline__ void fill_patterns(const LearnArgs& A, int64_t n0, uint32_t n, uint32_t block,
                                              bool codes, float4* x) {
  for (uint32_t i = threadIdx.x; i < (n + 1u) * W; i += blockDim.x) {
    const uint32_t node = i / W, pg = block * W + i % W;
    const int32_t slot = node < n ? A.node_in[n0 + node] : -1;
    x[i] = slot >= 0 ? pattern4(A, slot, pg) : make_float4(0.f, 0.f, 0.f, 0.f);
    if (codes && slot >= 0 && kept_in(A.kept, pg))
      for (uint32_t t = 0; t < A.kept.planes; ++t) *kept_at(A.kept, A.nodes, t, pg, n0 + node) = 0;
  }
}
// A block's derivatives by the output nodes' sums in the last step, over zeros. (Every thread of the
// workgroup; a barrier before their use is the caller's.)
template <int W>
__device__ __forceinline__ void fill_outputs(const LearnArgs& A, uint32_t g, uint32_t n, uint32_t block,
                                             float4* x) {
  for (uint32_t i = threadIdx.x; i < (n + 1u) * W; i += blockDim.x) x[i] = make_float4(0.f, 0.f, 0.f, 0.f);
  __syncthreads();
  const uint32_t p0 = block * 4u * W, np = min(A.n_patterns - p0, 4u * W);
  for (uint32_t i = threadIdx.x; i < np * A.n_outputs; i += blockDim.x) {
    const uint32_t p = i / A.n_outputs, o = i % A.n_outputs;
    const int64_t r = ((int64_t)g * A.n_patterns + p0 + p) * A.n_outputs + o;
    const float v = A.outputs[r];
    reinterpret_cast<float*>(x)[(uint32_t)A.out_node[o] * 4u * W + p] = A.grad_outputs[r] * v * (1.0f - v);
  }
}
// A unit's rows of input nodes: their edges' derivatives, and their patterns'.
template <int LN>
__device__ __forceinline__ void input_rows(const LearnArgs& A, const Rows& R, uint32_t unit, uint32_t g,
                                           int64_t n0, uint32_t n, uint32_t block, const float4* gz, float* sum,
                                           bool set) {
  const Place<LN> P = place_of<LN, false>(R, unit, threadIdx.x % kWave);
  const int32_t slot = P.row != kNoRow ? A.node_in[n0 + P.row] : -1;
  const uint32_t pg = block * LN + P.q;
  const float4 x = slot >= 0 ? pattern4(A, slot, pg) : make_float4(0.f, 0.f, 0.f, 0.f);
  const float4 d = row_grads<LN>(P, R.ent, gz, n, x, sum, set);
  if (!A.grad_inputs || !P.writes) return;
  const float v[4] = {d.x, d.y, d.z, d.w};
#pragma unroll
  for (uint32_t j = 0; j < 4; ++j) {
    const uint32_t p = 4u * pg + j;
    if (p < A.n_patterns) A.grad_inputs[((int64_t)g * A.n_patterns + p) * A.n_inputs + (uint32_t)slot] = v[j];
  }
}

// ----------------------------------------------------------------------------- all steps of a genome

// The values after a step become those before the next.
template <int W, bool LOCAL>
__device__ __forceinline__ void advance(float4*& cur, float4*& nxt, uint32_t n) {
  if constexpr (LOCAL) {
    __syncthreads();
    float4* x = cur;
    cur = nxt;
    nxt = x;
  } else {
    __threadfence_block();
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < n * W; i += blockDim.x) cur[i] = nxt[i];
    __syncthreads();
  }
}

// All steps of one genome for an item's blocks of 4 LN patterns. Bound by waiting, with the four waves to a SIMD that
// the registers leave: an edge's entry, then the gathered 16 bytes of LDS for it and four patterns, then four fused
// adds. 150 networks of up to 773 hidden nodes, 1000 patterns, 4 steps take 638 us with the kept states as numbers:
// the waves wait in 57 % of their cycles, the VALU issues in 50 %, LDS serves in 29 % (a third of that bank
// conflicts). Their gradients (below) take 1013 us: 65 %, 49 % and 18 %, and 1.8 GB to and from memory, most of it the
// items' sums, read and added to in every step.
template <int LN, bool LOCAL>
__device__ __forceinline__ void keep_item(const LearnArgs& A, const LearnItem& I, float4* lds) {
  const uint32_t g = I.genome;
  const int64_t n0 = A.node_offset[g];
  const uint32_t n = (uint32_t)(A.node_offset[g + 1] - n0);
  if (learn_lds(n, {LN, LOCAL}) > A.lds_bytes) return;  // (host-checked)
  const uint32_t lane = threadIdx.x % kWave;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), waves = blockDim.x / kWave;
  const Rows H = rows_of(A, kInHid, g), E = rows_of(A, kInInp, g);
  float4 *cur = lds, *nxt = LOCAL ? lds + (n + 1u) * LN : A.values + I.values, *held = nxt + (n + 1u) * LN;
  if (LOCAL)
    for (uint32_t i = threadIdx.x; i < LN; i += blockDim.x) nxt[n * LN + i] = make_float4(0.f, 0.f, 0.f, 0.f);
  for (uint32_t b = I.b0; b < I.b1; ++b) {
    fill_patterns<LN>(A, n0, n, b, true, cur);
    __syncthreads();
    auto put = [&](uint32_t row, uint32_t q, uint32_t step, const float4& z) {
      const uint32_t pg = b * LN + q;
      const float4 s = sigmoid4(z);
      nxt[row * LN + q] = s;
      if (step < A.steps && kept_in(A.kept, pg)) *kept_at(A.kept, A.nodes, step - 1, pg, n0 + row) = codes_of(s);
    };
    // the first step: the inputs' edges alone, whose sums stay (hidden states are 0)
    if (A.steps > 0)
      for (uint32_t u = wave; u < units_of<LN>(E); u += waves) {
        const Place<LN> P = place_of<LN, false>(E, u, lane);
        const float4 z = row_sums<LN>(P, E.ent, cur, n);
        if (!P.writes) continue;
        held[P.row * LN + P.q] = z;
        put(P.row, P.q, 1, z);
      }
    for (uint32_t step = 2; step <= A.steps; ++step) {
      advance<LN, LOCAL>(cur, nxt, n);
      // the last step: output nodes alone, the first units
      const uint32_t end = step == A.steps ? A.n_outputs : units_of<LN>(H);
      for (uint32_t u = wave; u < end; u += waves) {
        const Place<LN> P = place_of<LN, false>(H, u, lane);
        const float4 z = row_sums<LN>(P, H.ent, cur, n);
        if (P.writes) put(P.row, P.q, step, add4(z, held[P.row * LN + P.q]));
      }
    }
    __threadfence_block();
    __syncthreads();
    const float* c = reinterpret_cast<const float*>(nxt);
    const uint32_t p0 = b * 4u * LN, np = min(A.n_patterns - p0, 4u * LN);
    for (uint32_t i = threadIdx.x; i < np * A.n_outputs; i += blockDim.x) {
      const uint32_t p = i / A.n_outputs, o = i % A.n_outputs;
      A.outputs[((int64_t)g * A.n_patterns + p0 + p) * A.n_outputs + o] =
          A.steps > 0 ? c[(uint32_t)A.out_node[o] * 4u * LN + p] : 0.0f;
    }
    __syncthreads();
  }
}

template <int LN, bool LOCAL>
__device__ __forceinline__ void back_item(const LearnArgs& A, const LearnItem& I, float4* lds) {
  const uint32_t g = I.genome;
  const int64_t n0 = A.node_offset[g];
  const uint32_t n = (uint32_t)(A.node_offset[g + 1] - n0);
  if (learn_lds(n, {LN, LOCAL}) > A.lds_bytes) return;  // (host-checked)
  const uint32_t lane = threadIdx.x % kWave;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), waves = blockDim.x / kWave;
  const Rows H = rows_of(A, kOutHid, g), E = rows_of(A, kOutInp, g);
  const uint32_t hp = A.set[kOutHid].n_places[g], ip = A.set[kOutInp].n_places[g];
  float *hsum = A.partial + I.part, *isum = hsum + hp;
  float4 *cur = lds, *nxt = LOCAL ? lds + (n + 1u) * LN : A.values + I.values, *all = nxt + (n + 1u) * LN;
  if (LOCAL)
    for (uint32_t i = threadIdx.x; i < LN; i += blockDim.x)
      nxt[n * LN + i] = all[n * LN + i] = make_float4(0.f, 0.f, 0.f, 0.f);
  if (A.steps < 2)  // (no step of theirs)
    for (uint32_t i = threadIdx.x; i < hp; i += blockDim.x) hsum[i] = 0.0f;
  for (uint32_t b = I.b0; b < I.b1; ++b) {
    fill_outputs<LN>(A, g, n, b, cur);
    __syncthreads();
    for (uint32_t step = A.steps; step >= 2; --step) {
      const bool last = step == A.steps;  // derivatives at the output nodes alone
      for (uint32_t u = wave; u < units_of<LN>(H); u += waves) {
        const Place<LN> P = last ? place_of<LN, true>(H, u, lane) : place_of<LN, false>(H, u, lane);
        const uint32_t pg = b * LN + P.q;
        const uint32_t c = P.row != kNoRow && kept_in(A.kept, pg)
                               ? *kept_at(A.kept, A.nodes, step - 2, pg, n0 + P.row) : 0u;
        const float4 d = row_grads<LN>(P, H.ent, cur, n, states(c), hsum, last && b == I.b0);
        if (!P.writes) continue;
        const uint32_t i = P.row * LN + P.q;
        const float4 v = slopes(d, c);
        nxt[i] = v;
        all[i] = add4(last ? cur[i] : all[i], v);
      }
      advance<LN, LOCAL>(cur, nxt, n);
    }
    const float4* sum_gz = A.steps < 2 ? cur : all;
    if (!LOCAL && A.steps >= 2) {
      for (uint32_t i = threadIdx.x; i < n * LN; i += blockDim.x) cur[i] = all[i];
      __syncthreads();
      sum_gz = cur;
    }
    for (uint32_t u = wave; u < units_of<LN>(E); u += waves)
      input_rows<LN>(A, E, u, g, n0, n, b, sum_gz, isum, b == I.b0);
    __syncthreads();
  }
  if (!I.alone) return;
  __threadfence_block();
  __syncthreads();
  const uint32_t *hi = A.set[kOutHid].edge + A.place[g], *ii = A.set[kOutInp].edge + A.place[g];
  for (uint32_t i = threadIdx.x; i < hp; i += blockDim.x)
    if (hi[i] != kNoEdge) A.grad_w[hi[i]] = hsum[i];
  for (uint32_t i = threadIdx.x; i < ip; i += blockDim.x)
    if (ii[i] != kNoEdge) A.grad_w[ii[i]] = isum[i];
}

template <bool BACK>
__global__ void __launch_bounds__(1024, 4) k_learn(LearnArgs A) {
  extern __shared__ float4 learn_lds_mem[];
  const LearnItem I = A.items[A.first_item + blockIdx.x];
  static_assert(sizeof kLearnShapes / sizeof kLearnShapes[0] == 8, "a case for each shape");
#define EMR_LEARN_CASE(i)                                                                                   \
  case i: {                                                                                                 \
    constexpr LearnShape S = kLearnShapes[i];                                                               \
    if constexpr (BACK) back_item<(int)S.lanes, S.local != 0>(A, I, learn_lds_mem);          \
    else keep_item<(int)S.lanes, S.local != 0>(A, I, learn_lds_mem);                         \
    break;                                                                                                  \
  }
  switch (__builtin_amdgcn_readfirstlane(I.shape)) {
    EMR_LEARN_CASE(0)
    EMR_LEARN_CASE(1)
    EMR_LEARN_CASE(2)
    EMR_LEARN_CASE(3)
    EMR_LEARN_CASE(4)
    EMR_LEARN_CASE(5)
    EMR_LEARN_CASE(6)
    EMR_LEARN_CASE(7)
    default: break;
  }
#undef EMR_LEARN_CASE
}

// ----------------------------------------------------------------------------- a step of a genome

// One step of genomes too large for that, or too few to fill the chip: a workgroup holds all nodes' values of a
// block of patterns and takes a share of the units.
template <int LN>
__device__ __forceinline__ void keep_step(const LearnArgs& A, const LearnStepItem& I, float4* lds) {
  const uint32_t g = I.genome;
  const int64_t n0 = A.node_offset[g];
  const uint32_t n = (uint32_t)(A.node_offset[g + 1] - n0);
  if (learn_lds(n, {LN, 0}) > A.lds_bytes) return;  // (host-checked)
  const uint32_t lane = threadIdx.x % kWave;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), waves = blockDim.x / kWave;
  const bool first = A.step == 1, last = A.step == A.steps;
  const Rows R = rows_of(A, first ? kInInp : kInHid, g);
  const uint32_t end = last && !first ? A.n_outputs : units_of<LN>(R);
  for (uint32_t b = I.b0; b < I.b1; ++b) {
    const int64_t v0 = I.values + (int64_t)b * n * LN;
    const float4* cur = A.cur + v0;
    float4 *nxt = A.nxt + v0, *held = A.held + v0;
    if (first) {
      fill_patterns<LN>(A, n0, n, b, I.chunk == 0, lds);
    } else {
      for (uint32_t i = threadIdx.x; i < (n + 1u) * LN; i += blockDim.x)
        lds[i] = i < n * LN ? cur[i] : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    __syncthreads();
    for (uint32_t u = wave * I.chunks + I.chunk; u < end; u += waves * I.chunks) {
      const Place<LN> P = place_of<LN, false>(R, u, lane);
      float4 z = row_sums<LN>(P, R.ent, lds, n);
      if (!P.writes) continue;
      const uint32_t i = P.row * LN + P.q, pg = b * LN + P.q;
      if (first) held[i] = z;
      else z = add4(z, held[i]);
      const float4 s = sigmoid4(z);
      nxt[i] = s;
      if (!last && kept_in(A.kept, pg)) *kept_at(A.kept, A.nodes, A.step - 1, pg, n0 + P.row) = codes_of(s);
    }
    __syncthreads();
  }
}

template <int LN>
__device__ __forceinline__ void back_step(const LearnArgs& A, const LearnStepItem& I, float4* lds) {
  const uint32_t g = I.genome;
  const int64_t n0 = A.node_offset[g];
  const uint32_t n = (uint32_t)(A.node_offset[g + 1] - n0);
  if (learn_lds(n, {LN, 0}) > A.lds_bytes) return;  // (host-checked)
  const uint32_t lane = threadIdx.x % kWave;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), waves = blockDim.x / kWave;
  const bool inputs = A.step == 1, last = A.step == A.steps;
  const uint32_t hp = A.set[kOutHid].n_places[g];
  const Rows R = rows_of(A, inputs ? kOutInp : kOutHid, g);
  float* sum = A.partial + I.part + (inputs ? hp : 0u);
  if (inputs && last)  // (one step: the other edges have no part)
    for (uint32_t i = I.chunk * blockDim.x + threadIdx.x; i < hp; i += I.chunks * blockDim.x)
      A.partial[I.part + i] = 0.0f;
  for (uint32_t b = I.b0; b < I.b1; ++b) {
    const int64_t v0 = I.values + (int64_t)b * n * LN;
    const float4* from = (inputs ? A.held : A.cur) + v0;
    float4 *nxt = A.nxt + v0, *all = A.held + v0;
    // the derivatives after the step (of all steps); those after the last are at the output nodes alone
    if (last) {
      fill_outputs<LN>(A, g, n, b, lds);
    } else {
      for (uint32_t i = threadIdx.x; i < (n + 1u) * LN; i += blockDim.x)
        lds[i] = i < n * LN ? from[i] : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    __syncthreads();
    for (uint32_t u = wave * I.chunks + I.chunk; u < units_of<LN>(R); u += waves * I.chunks) {
      if (inputs) {
        input_rows<LN>(A, R, u, g, n0, n, b, lds, sum, b == I.b0);
        continue;
      }
      const Place<LN> P = last ? place_of<LN, true>(R, u, lane) : place_of<LN, false>(R, u, lane);
      const uint32_t pg = b * LN + P.q;
      const uint32_t c = P.row != kNoRow && kept_in(A.kept, pg)
                             ? *kept_at(A.kept, A.nodes, A.step - 2, pg, n0 + P.row) : 0u;
      const float4 d = row_grads<LN>(P, R.ent, lds, n, states(c), sum, last && b == I.b0);
      if (!P.writes) continue;
      const uint32_t i = P.row * LN + P.q;
      const float4 v = slopes(d, c);
      nxt[i] = v;
      all[i] = add4(last ? lds[i] : all[i], v);
    }
    __syncthreads();
  }
}

template <bool BACK>
__global__ void __launch_bounds__(1024, 4) k_learn_step(LearnArgs A) {
  extern __shared__ float4 learn_lds_mem[];
  const LearnStepItem I = A.step_items[A.first_item + blockIdx.x];
  switch (__builtin_amdgcn_readfirstlane(I.lanes)) {
    case 1: BACK ? back_step<1>(A, I, learn_lds_mem) : keep_step<1>(A, I, learn_lds_mem); break;
    case 2: BACK ? back_step<2>(A, I, learn_lds_mem) : keep_step<2>(A, I, learn_lds_mem); break;
    case 4: BACK ? back_step<4>(A, I, learn_lds_mem) : keep_step<4>(A, I, learn_lds_mem); break;
    default: BACK ? back_step<8>(A, I, learn_lds_mem) : keep_step<8>(A, I, learn_lds_mem); break;
  }
}

// The outputs of stepped genomes, from their states after the last step.
__global__ void __launch_bounds__(kNetThreads) k_step_outputs(LearnArgs A) {
  const LearnStepItem I = A.step_items[A.first_item + blockIdx.x];
  if (I.chunk != 0) return;
  const int64_t n = A.node_offset[I.genome + 1] - A.node_offset[I.genome];
  const uint32_t wide = 4u * I.lanes;
  for (uint32_t b = I.b0; b < I.b1; ++b) {
    const float* v = reinterpret_cast<const float*>(A.cur + I.values + b * n * I.lanes);
    const uint32_t p0 = b * wide, np = min(A.n_patterns - p0, wide);
    for (uint32_t i = threadIdx.x; i < np * A.n_outputs; i += kNetThreads) {
      const uint32_t p = i / A.n_outputs, o = i % A.n_outputs;
      A.outputs[((int64_t)I.genome * A.n_patterns + p0 + p) * A.n_outputs + o] =
          A.steps ? v[(uint32_t)A.out_node[o] * wide + p] : 0.0f;
    }
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

// ----------------------------------------------------------------------------- kept states

// A state's number in a type: float, or 16 bits (bfloat16 to nearest, ties to even).
__device__ __forceinline__ float as(float v, float) { return v; }
__device__ __forceinline__ _Float16 as(float v, _Float16) { return (_Float16)v; }
__device__ __forceinline__ uint16_t as(float v, uint16_t) {
  const uint32_t b = __float_as_uint(v);
  return (uint16_t)((b + 0x7FFFu + ((b >> 16) & 1u)) >> 16);
}

// A lane for a node's block of codes; a wave for eight blocks of eight nodes, so that both the codes read and
// the numbers written lie side by side in runs of 128 bytes and more. (blockIdx.y: plane.)
template <typename T>
__global__ void __launch_bounds__(kNetThreads) k_kept_values(KeptValuesArgs A) {
  const uint32_t b = 4u * A.kept.q, tiles = (A.kept.blocks + 7u) / 8u;
  const int64_t groups = (A.nodes + 7) / 8, all = groups * tiles;
  const uint32_t lane = threadIdx.x % kWave;
  const bool wide = (uint64_t)A.n_patterns * sizeof(T) % 16 == 0 && (uintptr_t)A.out % 16 == 0;
  for (int64_t w = grid_thread() / kWave; w < all; w += grid_threads() / kWave) {
    const int64_t node = w / tiles * 8 + lane % 8u;
    const uint32_t block = (uint32_t)(w % tiles) * 8u + lane / 8u;
    if (node >= A.nodes || block >= A.kept.blocks) continue;
    const uint8_t* c = A.kept.codes + (((int64_t)blockIdx.y * A.kept.blocks + block) * A.nodes + node) * b;
    const uint32_t p0 = block * b, n = min(b, A.n_patterns - p0);
    T* out = static_cast<T*>(A.out) + ((int64_t)blockIdx.y * A.nodes + node) * A.n_patterns + p0;
    for (uint32_t k = 0; k < n; k += 4) {
      const float4 s = states(*reinterpret_cast<const uint32_t*>(c + k));
      struct alignas(4 * sizeof(T)) Four {
        T v[4];
      } f = {{as(s.x, T()), as(s.y, T()), as(s.z, T()), as(s.w, T())}};
      if (wide && k + 4 <= n) {
        *reinterpret_cast<Four*>(out + k) = f;
      } else {
        for (uint32_t j = 0; j < 4 && k + j < n; ++j) out[k + j] = f.v[j];
      }
    }
  }
}

// f(first, count) for shares of n workgroups: a launch's threads in a dimension are a 32-bit number.
template <typename F>
void launches(uint32_t n, uint32_t threads, F&& f) {
  const uint32_t most = 0xFFFFFFFFu / threads;
  for (uint64_t a = 0; a < n; a += most) f((uint32_t)a, n - (uint32_t)a < most ? n - (uint32_t)a : most);
}
uint32_t stride_blocks(int64_t n) {
  const int64_t b = (n + kNetThreads - 1) / kNetThreads;
  return (uint32_t)(b < 1 ? 1 : (b > 16384 ? 16384 : b));
}

}  // namespace
}  // namespace emr

// Steps: 0 the edges' keys by source, 1 their offsets (after the sort), 2 a layout, 3 its weights; all steps
// of the genomes in LDS: 4 activation, 5 gradients, 6 their joined sums; one step of others: 11 activation, 12
// gradients, 13 the outputs; 14 kept states as numbers; a genome larger than the LDS: 7 the derivatives by
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
      hipLaunchKernelGGL(k_layout_degrees, dim3(stride_blocks(A.nodes * kWave)), blk, 0, s, A);
      launches(A.count, kLayoutThreads, [&](uint32_t a, uint32_t n) {
        LearnLayoutArgs B = A;
        B.genomes = A.genomes + a;
        hipLaunchKernelGGL(k_layout_slices, dim3(n), dim3(kLayoutThreads), 0, s, B);
      });
      // (about 4096 workgroups over the genomes, a wave to a node)
      const uint32_t x = A.count < 4096u ? 4096u / A.count : 1u;
      for (uint32_t a = 0; a < A.count; a += 65535u) {
        LearnLayoutArgs B = A;
        B.genomes = A.genomes + a;
        hipLaunchKernelGGL(k_layout_fill, dim3(x < 512u ? x : 512u, A.count - a < 65535u ? A.count - a : 65535u),
                           blk, 0, s, B);
      }
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
      launches(A.n_items, A.threads, [&](uint32_t a, uint32_t n) {
        LearnArgs B = A;
        B.first_item = A.first_item + a;
        if (step == 4)
          hipLaunchKernelGGL(k_learn<false>, dim3(n), dim3(A.threads), A.lds_bytes, s, B);
        else
          hipLaunchKernelGGL(k_learn<true>, dim3(n), dim3(A.threads), A.lds_bytes, s, B);
      });
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
    case 14: {
      const auto& A = *static_cast<const KeptValuesArgs*>(args);
      const int64_t waves = (A.nodes + 7) / 8 * ((A.kept.blocks + 7) / 8);
      for (uint32_t a = 0; a < A.kept.planes; a += 65535u) {
        KeptValuesArgs B = A;
        const int64_t plane = (int64_t)A.kept.blocks * A.nodes * (4 * A.kept.q);
        B.kept.codes = A.kept.codes + a * plane;
        B.out = static_cast<char*>(A.out) + (int64_t)a * A.nodes * A.n_patterns * (A.type == 0 ? 4 : 2);
        const uint32_t y = A.kept.planes - a < 65535u ? A.kept.planes - a : 65535u;
        const dim3 grid(stride_blocks(waves * kWave), y);
        if (A.type == 0) hipLaunchKernelGGL(k_kept_values<float>, grid, blk, 0, s, B);
        else if (A.type == 1) hipLaunchKernelGGL(k_kept_values<uint16_t>, grid, blk, 0, s, B);
        else hipLaunchKernelGGL(k_kept_values<_Float16>, grid, blk, 0, s, B);
      }
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
