// The second pass of the deterministic column reductions: adds the fp64
// partial sums that a grid of workgroups left per channel.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace sscn {

// Sums of the partials of the `blocks` workgroups for channel col: one
// workgroup of kFinThreads threads per 64 channels, wavefront w adding
// blocks w, w + 16, .. in order, then the sixteen wavefronts' sums added
// pairwise in a fixed tree (a fixed order: reproducible).  (One thread
// adding all blocks in turn took ~0.25 ms for 1024 blocks; four wavefronts
// ~15 us.)
constexpr int kFinThreads = 1024;
__device__ __forceinline__ bool sum_partials(const double* __restrict__ partial, int blocks, int c, double& s0,
                                             double& s1, int& col) {
  constexpr int NW = kFinThreads / 64;
  __shared__ double red[2][NW][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  col = blockIdx.x * 64 + lane;
  double a0 = 0.0, a1 = 0.0;
  if (col < c) {
#pragma unroll 4
    for (int b = wave; b < blocks; b += NW) {
      a0 += partial[((int64_t)b * 2) * c + col];
      a1 += partial[((int64_t)b * 2 + 1) * c + col];
    }
  }
  red[0][wave][lane] = a0;
  red[1][wave][lane] = a1;
  __syncthreads();
#pragma unroll
  for (int h = NW / 2; h >= 1; h /= 2) {
    if (wave < h) {
      red[0][wave][lane] += red[0][wave + h][lane];
      red[1][wave][lane] += red[1][wave + h][lane];
    }
    __syncthreads();
  }
  if (wave != 0 || col >= c) return false;
  s0 = red[0][0][lane];
  s1 = red[1][0][lane];
  return true;
}

static __global__ __launch_bounds__(kFinThreads) void k_two_sums(const double* __restrict__ partial, int blocks, int c,
                                                  float* __restrict__ out0, float* __restrict__ out1) {
  double s0, s1;
  int col;
  if (!sum_partials(partial, blocks, c, s0, s1, col)) return;
  out0[col] = (float)s0;
  if (out1) out1[col] = (float)s1;
}

}  // namespace sscn
