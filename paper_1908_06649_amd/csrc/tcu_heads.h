// Internal launchers of the heads' norms with rotation (host side).  Arguments are
// already validated by tcu_heads_abi.cpp.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tcu.h"

namespace tcu {

// tokens x heads x dim elements: pitches of tokens and of heads.
struct Heads {
  const void *p;
  int64_t ld, hd;
};

struct QkNormArgs {
  Heads x[2], dy[2], y[2];   // queries, keys; dy: the gradient's alone; y: out
  const void *w[2];
  const float *freq;
  const int32_t *pos;
  float *dw[2], *parts;
  int64_t tokens;
  int heads[2], dim, rot;
  float eps;
  bool adjacent;
};
hipError_t launch_qk_norm(int elem, const QkNormArgs &a, hipStream_t stream, int num_cus);
hipError_t launch_qk_norm_grad(int elem, const QkNormArgs &a, hipStream_t stream, int num_cus);

// Workgroups of a gradient, each with its tokens' sums of the weights' gradients.
constexpr int kHeadParts = 512;

}  // namespace tcu
