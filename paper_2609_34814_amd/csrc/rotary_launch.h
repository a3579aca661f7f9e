// Internal launch interface of the rotary-position kernel (not part of the ABI).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

struct WaRotaryLaunch {
  const void* in[2];      // q, k
  void* out[2];
  int64_t in_stride[2][3];   // elements: batch, head, token
  int64_t out_stride[2][3];
  int32_t heads[2];       // heads[1] = 0: one tensor
  int32_t copy[2];        // 1: columns past the rotated ones are copied (0 in place)
  const double* freq;     // [pairs] radians a position
  const int32_t* pos;     // [axes][pos_batch][tokens], null: the token's index
  int32_t pos_batch, axes;
  int32_t axis_end[3];    // first pair past each axis
  int32_t batch, tokens, head_dim, pairs, interleaved, dtype;
  float cos_scale, sin_scale;  // factor of the rotated values; the sine's is negative for the gradient
};

hipError_t wa_launch_rotary(const WaRotaryLaunch& a, hipStream_t stream);
