// Internal interface between the C-ABI host code and the gfx950 kernels of head norms and rotations.
#pragma once
#include <hip/hip_runtime_api.h>
#include <stdint.h>

namespace ta {

constexpr int kRopeAxes = 4;
constexpr int kRopeWaves = 4;  // waves of a workgroup
// Tokens of a wave: a row of d values takes 8 lanes (d = 64) or 16, 8 values a lane.
constexpr int rope_tokens(int d) { return d == 64 ? 8 : 4; }

// Rows of a projection: strides in values.
struct Rows {
  uint16_t* p;
  int64_t batch, token, head;
};

struct RopeArgs {
  int B, S, d, norm, layout, axes;
  int dims[kRopeAxes];
  int start[kRopeAxes];  // first value of each axis; of those that are none, behind every value
  int turned;            // values that are turned: the sum of dims
  bool whole;            // partners of 8 values in a row, from a multiple of 8 on, are 8 such values again
  float eps;
  const float* weight[2];  // q's and k's, or null
  const float* bias[2];
  const double* freqs;
  const int32_t* positions;
  int64_t positions_batch;
  const int32_t* lens;  // or null
  int heads[3];         // of q, k, v; 0 for what is left out
  Rows x[3];            // what the projection gave (forward: q, k, v; gradients: q and k, with a norm)
  uint16_t* y[3];       // [B, heads, S, d]: the forward's results; gradients: their gradients, read only
  int heads_per;        // heads that a wave takes of a token
  // gradients
  Rows dx[3];
  int first[4];   // the first workgroup of q's, k's and v's rows, and their number
  float* part;    // fp32 [workgroups][weight, bias][d], or null: no sums are wanted
  float* sum[4];  // gradients of q's weight and bias, k's weight and bias, or null
};

hipError_t launch_head_rope(const RopeArgs& a, hipStream_t stream);
hipError_t launch_head_rope_grad(const RopeArgs& a, hipStream_t stream);

}  // namespace ta
