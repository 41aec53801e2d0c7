// What the rotation's kernel and the C-ABI share.
#pragma once

#include "rows.h"

namespace spc {

constexpr int kMostRotated = 256;  // columns of a head

struct RotateArgs {
  const void* x[2];  // queries, keys
  void* y[2];
  int64_t x_row[2], x_head[2], y_row[2], y_head[2];  // strides in elements
  const void* gamma[2];  // [d], or NULL: no norm
  const int32_t* pos;    // [n] places, or [n][4] voxels (b, x, y, z)
  const double* freq;    // [rot / 2] radians a position
  int64_t n;
  int heads[2];
  int d, rot, voxels;
  float eps, gain;
  int per, share;  // rows of a workgroup, and heads of a row (each share a workgroup of its own)
};

hipError_t launch_rotate(const RotateArgs& a, int dtype, bool interleaved, hipStream_t s);

}  // namespace spc
