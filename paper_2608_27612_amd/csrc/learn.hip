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
#include "network.h"

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
  const int64_t per = (int64_t)A.n_patterns * A.n_outputs, all = per * A.n_genomes;
  for (int64_t r = grid_thread(); r < all; r += grid_threads()) {
    const int64_t g = r / per;
    const uint32_t p = (uint32_t)(r % per / A.n_outputs), o = (uint32_t)(r % A.n_outputs);
    const int64_t node = A.node_offset[g] + A.out_node[o];
    const float v = A.outputs[r];
    gz[((int64_t)(p / 4u) * A.nodes + node) * 4 + p % 4u] = A.grad_outputs[r] * v * (1.0f - v);
  }
}
__global__ void __launch_bounds__(kNetThreads) k_back_clear(float* p, int64_t n) {
  for (int64_t i = grid_thread(); i < n; i += grid_threads()) p[i] = 0.0f;
}

// The weights' derivatives in one step: a thread for an edge.
__global__ void __launch_bounds__(kNetThreads) k_back_edges(NetBackArgs A) {
  const float4* gz = reinterpret_cast<const float4*>(A.gz);
  for (int64_t e = grid_thread(); e < A.edges; e += grid_threads()) {
    const int64_t src = A.in_src[e], dst = A.dst[e];
    float sum = 0.0f;
    for (uint32_t pb = 0; pb < A.pblocks; ++pb) {
      const float4 d = gz[(int64_t)pb * A.nodes + dst], s = state_before(A, src, pb);
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
  for (int64_t j = grid_thread() / kWave; j < A.nodes; j += grid_threads() / kWave) {
    const int32_t slot = A.node_in[j];
    const int64_t e0 = A.out_offset[j], e1 = A.out_offset[j + 1];
    for (uint32_t pb = blockIdx.z; pb < A.pblocks; pb += gridDim.z) {
      if (slot >= 0 && A.grad_inputs == nullptr) continue;
      float4 d = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int64_t k = e0 + lane; k < e1; k += kWave) {
        const uint64_t v = A.out_edge[k];
        const float w = A.in_w[(uint32_t)v];
        const float4 x = gz[(int64_t)pb * A.nodes + (int64_t)(v >> 32)];
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
        int64_t lo = 0, hi = A.n_genomes;  // the node's genome
        while (hi - lo > 1) {
          const int64_t mid = (lo + hi) / 2;
          if (A.node_offset[mid] <= j) lo = mid;
          else hi = mid;
        }
        const uint32_t p = 4u * pb + lane;
        if (lane < 4u && p < A.n_patterns) {
          float* g = A.grad_inputs + (lo * A.n_patterns + p) * A.n_inputs + (uint32_t)slot;
          const float v = lane == 0 ? d.x : (lane == 1 ? d.y : (lane == 2 ? d.z : d.w));
          *g = A.last ? v : *g + v;
        }
      } else if (lane == 0 && A.step > 1) {
        const uint32_t c = code4(A.kept, A.nodes, A.step - 2, pb, j);
        before[(int64_t)pb * A.nodes + j] =
            make_float4(d.x * slope_of(c & 255u), d.y * slope_of((c >> 8) & 255u),
                        d.z * slope_of((c >> 16) & 255u), d.w * slope_of(c >> 24));
      }
    }
  }
}

uint32_t stride_blocks(int64_t n) {
  const int64_t b = (n + kNetThreads - 1) / kNetThreads;
  return (uint32_t)(b < 1 ? 1 : (b > 16384 ? 16384 : b));
}

}  // namespace
}  // namespace emr

// Steps: 0 the edges' keys by source, 1 their offsets (after the sort), 2 the derivatives by the outputs'
// sums into gz_before (the other half behind it cleared), 3 one step's weight derivatives, 4 one step
// backwards, 5 no derivatives at all.
extern "C" hipError_t emr_launch_learn(int step, const void* args, hipStream_t s) {
  using namespace emr;
  const dim3 blk(kNetThreads);
  if (step < 2) {
    const auto& A = *static_cast<const NetTurnArgs*>(args);
    if (step == 0)
      hipLaunchKernelGGL(k_turn_keys, dim3(stride_blocks(A.nodes * kWave)), blk, 0, s, A);
    else
      hipLaunchKernelGGL(k_turn_offsets, dim3(stride_blocks(A.nodes + 1)), blk, 0, s, A);
    return hipGetLastError();
  }
  const auto& A = *static_cast<const NetBackArgs*>(args);
  switch (step) {
    case 2: {
      const int64_t n = 8 * (int64_t)A.pblocks * A.nodes;  // (both halves: input nodes stay 0)
      hipLaunchKernelGGL(k_back_clear, dim3(stride_blocks(n)), blk, 0, s,
                         A.gz_before, n);
      hipLaunchKernelGGL(k_back_outputs,
                         dim3(stride_blocks((int64_t)A.n_genomes * A.n_patterns * A.n_outputs)), blk, 0,
                         s, A);
      break;
    }
    case 3:
      if (A.edges <= 0) return hipSuccess;
      hipLaunchKernelGGL(k_back_edges, dim3(stride_blocks(A.edges)), blk, 0, s, A);
      break;
    case 4:
      hipLaunchKernelGGL(k_back_nodes, dim3(stride_blocks(A.nodes * kWave), 1, A.pblocks < 64u ? A.pblocks : 64u),
                         blk, 0, s, A);
      break;
    case 5: {
      const int64_t n = (int64_t)A.n_genomes * A.n_patterns * A.n_inputs;
      if (A.edges > 0)
        hipLaunchKernelGGL(k_back_clear, dim3(stride_blocks(A.edges)), blk, 0, s, A.grad_w, A.edges);
      if (A.grad_inputs)
        hipLaunchKernelGGL(k_back_clear, dim3(stride_blocks(n)), blk, 0, s, A.grad_inputs, n);
      break;
    }
    default:
      return hipErrorInvalidValue;
  }
  return hipGetLastError();
}
