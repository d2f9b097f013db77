// Arguments of the kernels that draw from rows of scores and score the draws (choice.hip), shared with
// their host entry points (networks.cpp).
//
// Weights. A row's entry i with score x_i weighs q_i = floor(2^31 exp((x_i - m) / T)), m the row's
// maximum: a whole number of at most 31 bits and one, so that every sum of weights is a 64-bit
// whole number that no order of summation changes. An entry below 2^-31 of the maximum weighs
// nothing. Ranks go by (score falling, index rising): as one 64-bit number, the score's bits in an
// order that rises with it above the complement of the index (rank_of).
#pragma once
#include <stdint.h>

namespace emr {

constexpr int kTypeF32 = 0, kTypeBf16 = 1, kTypeF16 = 2;

constexpr uint32_t kDrawSegs = 4096;    // parts of a row with a sum each, at most
constexpr uint32_t kDrawPart = 256;     // a part's entries: a multiple of this

struct SampleArgs {
  const void* x;        // [rows] rows of n scores, stride entries apart
  int64_t stride, rows;
  uint32_t n;
  int32_t type;
  float t, p, min_p;    // for every row, where the pointer below is NULL
  int32_t k;
  const float* row_t;
  const int32_t* row_k;
  const float* row_p;
  const float* row_min_p;
  const float* u;       // [rows * draws]
  int64_t draws;
  int32_t* index;       // [rows * draws]
  float* logp;          // [rows * draws] or NULL
  uint32_t part;        // entries of a part of a row
  int64_t first;        // a launch's first row
};

struct LossArgs {
  const void* x;        // [rows] rows of n scores, stride entries apart
  int64_t stride, rows;
  uint32_t n;
  int32_t type;
  float inv_t;
  const int32_t* index;  // [rows]
  const float* scale;    // [rows] or NULL: 1
  float* loss;           // [rows] or NULL
  void* grad;            // [rows] rows of n, grad_stride entries apart, of x's type; or NULL
  int64_t grad_stride;
  int64_t first;         // a launch's first row
};

}  // namespace emr
