// Parameters and launchers of the kernels that normalise and rotate rows (implemented
// in norm.hip). Only host/norm.cpp calls them, after validating everything.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rope.hpp"

namespace fck {

// One tensor's rows: `rows` tokens of `heads` heads of d values.
struct NormRows {
  const void* in;          // forward: bf16 rows; backward: fp32 gradients of what it wrote
  void* out;
  const void* x;           // backward, normalised: the forward's bf16 rows
  int64_t in_stride, out_stride, x_stride;  // in elements
  const int32_t* in_gather;  // packed rows of `in`, of `x` (gpos); null: row r itself
  const int32_t* x_gather;
  const int32_t* gpos;     // as in RopeRows, for a row's position
  const int32_t* first;
  int32_t end;
  int32_t rows, heads;
  int32_t rotate;          // 0: not rotated
  int32_t norm;            // 0: not normalised
  int32_t centred;         // 1: the mean is subtracted first
  const void* weight;      // [d] (w_stride 0) or [heads, d] (w_stride d); null: ones
  int32_t w_stride, w_bf16;
  float offset, eps;       // added to the weights, to the mean square
  // a workgroup takes per_block rows, step_rows at a time, of group_heads of the heads
  int32_t group_heads, head_groups, step_rows, per_block;
  int32_t blocks;
  float* part;             // backward: null, or a row of partial weight gradients per
  int32_t part_width;      //   per_block rows: d, or heads * d floats
};

constexpr int kNormSets = 5;
// rows whose sines and cosines are in LDS at a time
constexpr int kNormRows = 16;
// the most rows of a workgroup
constexpr int kNormSteps = 4, kNormBlock = kNormSteps * kNormRows;
// threads of a head: two pieces of 8 (forward) or 4 (backward) values each
constexpr int norm_lanes(int d, bool back) { return d / (back ? 8 : 16); }

struct NormParams {
  NormRows set[kNormSets];
  int32_t n_sets;
  int32_t pairs, packed_pos;  // as in RopeParams
  float amplitude, sign;
  const int32_t* seg;
  uint64_t turn[64];
};

hipError_t launch_norm_fwd(const NormParams& p, int d, int layout, hipStream_t s);
hipError_t launch_norm_bwd(const NormParams& p, int d, int layout, bool out_f32, hipStream_t s);

// Sums of partial rows: dw[e] = sum of part[r * width + e] over n rows; of many rows
// (norm_slices over 1) first of `slices` of them, into a row of 64-bit sums each.
struct NormSum {
  const float* part;
  int32_t n, width;
  void* dw;
  int32_t bf16;
  int32_t slices;
  double* rows;
};
constexpr int kSumCols = 64, kSumRows = 128, kSumSlices = 64;
inline int32_t norm_slices(int64_t n) {
  const int64_t s = n / kSumRows;
  return int32_t(s < 1 ? 1 : s > kSumSlices ? kSumSlices : s);
}
// (one or two of them; width 0: none)
hipError_t launch_norm_sum(const NormSum& a, const NormSum& b, hipStream_t s);

}  // namespace fck
