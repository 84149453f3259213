// Activation checkpoints in 8 bits: what a pre-activated unit's backward pass
// needs of its forward, the normalised input xhat = (x - mean) * invstd, kept
// as one byte per value and one exponent byte per 32 channels of a row in
// place of the unit's input and its activations (2 or 4 bytes a value each).
//
// A block of 32 consecutive channels of a row (the last may be shorter) shares
// the step 2^e, e the least integer from -126 up with max |xhat| <= 126 * 2^e;
// its byte is e + 127.  A code is xhat / 2^e rounded to the nearest whole
// number, ties to even: off by half a step at most, 2^-7 of the block's largest
// value.  Where rounding would carry a value over the ReLU's border, the code
// is moved by one towards the side of the forward (127 is kept free for that):
// the backward pass masks exactly what the forward masked.  A block that holds
// an infinity or a NaN has the byte 255 and codes 0: 0 * inf, it stands for NaN.
#include <algorithm>

#include "internal.h"
#include "numeric.h"
#include "partials.h"

namespace sscn {

namespace {

constexpr int kBlock = 32;          // channels that share an exponent
constexpr int kMaxPartials = 1024;  // workgroups over the rows

// Exponent byte of a block from the largest |xhat|'s bits (as numbers, NaN >
// inf > finite): 126 = 1.96875 * 2^6, so mantissas above 0x7c0000 take the
// next power.
__device__ __forceinline__ uint32_t exponent_byte(uint32_t most) {
  if (most >= 0x7f800000u) return 255;
  return (uint32_t)max(1, (int)((most + 0x3ffffu) >> 23) - 6);
}
__device__ __forceinline__ float power(uint32_t byte) { return __uint_as_float(byte << 23); }  // 2^(byte - 127)

// The ReLU's argument as the forward and as the backward pass forms it.
__device__ __forceinline__ float pre_forward(float d, float scale, float beta) { return fmaf(d, scale, beta); }
__device__ __forceinline__ float pre_restored(float v, float gamma, float beta) { return fmaf(v, gamma, beta); }

// relu that lets a NaN through.
__device__ __forceinline__ float relu_nan(float v) { return v <= 0.f ? 0.f : v; }

__device__ __forceinline__ int encode(float d, float v, uint32_t byte, float scale, float gamma, float beta) {
  if (byte == 255) return 0;
  const float q = rintf(v * power(254 - byte));
  const bool want = pre_forward(d, scale, beta) > 0.f;
  const bool have = pre_restored(q * power(byte), gamma, beta) > 0.f;
  const int way = gamma > 0.f ? 1 : gamma < 0.f ? -1 : 0;
  return max(-127, min(127, (int)q + ((int)want - (int)have) * way));
}

// One half wavefront per block, a lane per channel.
template <typename T>
__global__ __launch_bounds__(256) void k_apply_q8(const T* __restrict__ x, int64_t ldx, int64_t n, int c, int blocks,
                                                  const float* __restrict__ mean, const float* __restrict__ invstd,
                                                  const float* __restrict__ scale, const float* __restrict__ gamma,
                                                  const float* __restrict__ beta, T* __restrict__ y, int64_t ldy,
                                                  int8_t* __restrict__ codes, uint8_t* __restrict__ exponents) {
  const int lane = threadIdx.x & 31;
  const int64_t total = n * blocks, step = (int64_t)gridDim.x * 8;
  // every lane of a wavefront takes part in the maximum: the loop's count is the workgroup's
  for (int64_t i0 = (int64_t)blockIdx.x * 8; i0 < total; i0 += step) {
    const int64_t i = i0 + (threadIdx.x >> 5);
    const int64_t r = i / blocks;
    const int col = (int)(i - r * blocks) * kBlock + lane;
    const bool live = i < total && col < c;
    float d = 0.f, v = 0.f;
    if (live) {
      d = ld(x + r * ldx + col) - mean[col];
      v = d * invstd[col];
    }
    uint32_t most = __float_as_uint(v) & 0x7fffffffu;
#pragma unroll
    for (int s = 16; s >= 1; s >>= 1) most = max(most, (uint32_t)__shfl_xor(most, s, 32));
    const uint32_t byte = exponent_byte(most);
    if (live) {
      st(y + r * ldy + col, fmaxf(0.f, pre_forward(d, scale[col], beta[col])));
      codes[r * c + col] = (int8_t)encode(d, v, byte, scale[col], gamma[col], beta[col]);
      if (lane == 0) exponents[i] = (uint8_t)byte;
    }
  }
}

// The values that the codes stand for.
template <typename T>
__global__ __launch_bounds__(256) void k_q8_values(const int8_t* __restrict__ codes,
                                                   const uint8_t* __restrict__ exponents, int64_t n, int c, int blocks,
                                                   T* __restrict__ y, int64_t ldy) {
  const int64_t total = n * c;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / c;
    const int col = (int)(i - r * c);
    st(y + r * ldy + col, (float)codes[i] * power(exponents[r * blocks + col / kBlock]));
  }
}

// Per channel the fp64 sums of dz and dz * xhat, dz = dA where the restored
// ReLU passes, over the rows of this workgroup (a fixed set, added in a fixed
// order), and the restored activations.
template <typename T>
__global__ __launch_bounds__(256) void k_params_q8(const T* __restrict__ da, int64_t ldd,
                                                   const int8_t* __restrict__ codes,
                                                   const uint8_t* __restrict__ exponents, int64_t n, int c, int blocks,
                                                   const float* __restrict__ gamma, const float* __restrict__ beta,
                                                   T* __restrict__ a, int64_t lda, double* __restrict__ partial) {
  __shared__ double red[2][4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = blockIdx.y * 64 + lane;
  double a0 = 0.0, a1 = 0.0;
  if (col < c) {
    const float ga = gamma[col], be = beta[col];
    for (int64_t r = (int64_t)blockIdx.x * 4 + wave; r < n; r += (int64_t)gridDim.x * 4) {
      const float v = (float)codes[r * c + col] * power(exponents[r * blocks + col / kBlock]);
      const float pre = pre_restored(v, ga, be);
      const float dz = pre > 0.f ? ld(da + r * ldd + col) : 0.f;
      a0 += dz;
      a1 += (double)dz * (double)v;
      if (a) st(a + r * lda + col, relu_nan(pre));
    }
  }
  red[0][wave][lane] = a0;
  red[1][wave][lane] = a1;
  __syncthreads();
  if (wave == 0 && col < c) {
    partial[((int64_t)blockIdx.x * 2) * c + col] = (red[0][0][lane] + red[0][1][lane]) + (red[0][2][lane] + red[0][3][lane]);
    partial[((int64_t)blockIdx.x * 2 + 1) * c + col] = (red[1][0][lane] + red[1][1][lane]) + (red[1][2][lane] + red[1][3][lane]);
  }
}

// dx = gamma invstd (dz - dbeta / n - xhat dgamma / n) (+ add) for the columns
// [col0, col0 + cols) of the layer; dx and add hold just those.
template <typename T>
__global__ __launch_bounds__(256) void k_input_q8(const T* __restrict__ da, int64_t ldd,
                                                  const int8_t* __restrict__ codes,
                                                  const uint8_t* __restrict__ exponents, int64_t n, int c, int blocks,
                                                  int col0, int cols, const float* __restrict__ gamma,
                                                  const float* __restrict__ beta, const float* __restrict__ invstd,
                                                  const float* __restrict__ dgamma, const float* __restrict__ dbeta,
                                                  const T* __restrict__ add, int64_t lda, T* __restrict__ dx,
                                                  int64_t ldo) {
  const int64_t total = n * cols;
  const float inv_n = 1.f / (float)n;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / cols;
    const int k = (int)(i - r * cols), col = col0 + k;
    const float v = (float)codes[r * c + col] * power(exponents[r * blocks + col / kBlock]);
    const float dz = pre_restored(v, gamma[col], beta[col]) > 0.f ? ld(da + r * ldd + col) : 0.f;
    float out = gamma[col] * invstd[col] * (dz - dbeta[col] * inv_n - v * (dgamma[col] * inv_n));
    if (add) out += ld(add + r * lda + k);
    st(dx + r * ldo + k, out);
  }
}

int row_blocks(int64_t n) { return (int)std::max<int64_t>(1, std::min<int64_t>(ceil_div(n, 64), kMaxPartials)); }
unsigned grid_of(int64_t work) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>(work, 16384)); }

sscn_status check_dtype(sscn_dtype dtype) {
  if (dtype != SSCN_F32 && dtype != SSCN_BF16) return fail(SSCN_ERR_INVALID_ARG, "unknown dtype");
  return SSCN_OK;
}
sscn_status check_rows(const void* p, int64_t ld, int64_t n, int c, sscn_dtype dtype) {
  if (n < 0 || c < 1) return fail(SSCN_ERR_INVALID_ARG, "q8: n must be >= 0 and c >= 1");
  if (n > 0 && !p) return fail(SSCN_ERR_INVALID_ARG, "q8: NULL matrix");
  if (ld < c) return fail(SSCN_ERR_INVALID_ARG, "q8: row stride below the channel count");
  if (reinterpret_cast<uintptr_t>(p) % (dtype == SSCN_F32 ? 4 : 2) != 0)
    return fail(SSCN_ERR_INVALID_ARG, "q8: matrix not aligned to its elements");
  return SSCN_OK;
}
sscn_status check_codes(const void* codes, const void* exponents, int64_t n) {
  if (n > 0 && (!codes || !exponents)) return fail(SSCN_ERR_INVALID_ARG, "q8: NULL codes or exponents");
  return SSCN_OK;
}

}  // namespace
}  // namespace sscn

using namespace sscn;

extern "C" sscn_status sscn_batchnorm_relu_apply_q8(const void* x, int64_t ldx, int64_t n, int32_t c,
                                                    sscn_dtype dtype, const float* mean, const float* invstd,
                                                    const float* scale, const float* gamma, const float* beta, void* y,
                                                    int64_t ldy, int8_t* codes, uint8_t* exponents,
                                                    hipStream_t stream) {
  SSCN_TRY(check_dtype(dtype));
  SSCN_TRY(check_rows(x, ldx, n, c, dtype));
  SSCN_TRY(check_rows(y, ldy, n, c, dtype));
  SSCN_TRY(check_codes(codes, exponents, n));
  if (!mean || !invstd || !scale || !gamma || !beta)
    return fail(SSCN_ERR_INVALID_ARG, "q8: NULL mean, invstd, scale, gamma or beta");
  if (n == 0) return SSCN_OK;
  const int blocks = (int)ceil_div(c, kBlock);
  const unsigned g = grid_of(ceil_div(n * blocks, 8));
  if (dtype == SSCN_F32)
    k_apply_q8<float><<<g, 256, 0, stream>>>((const float*)x, ldx, n, c, blocks, mean, invstd, scale, gamma, beta,
                                             (float*)y, ldy, codes, exponents);
  else
    k_apply_q8<uint16_t><<<g, 256, 0, stream>>>((const uint16_t*)x, ldx, n, c, blocks, mean, invstd, scale, gamma,
                                                beta, (uint16_t*)y, ldy, codes, exponents);
  SSCN_HIP(hipGetLastError());
  return SSCN_OK;
}

extern "C" sscn_status sscn_q8_values(const int8_t* codes, const uint8_t* exponents, int64_t n, int32_t c,
                                      sscn_dtype dtype, void* y, int64_t ldy, hipStream_t stream) {
  SSCN_TRY(check_dtype(dtype));
  SSCN_TRY(check_rows(y, ldy, n, c, dtype));
  SSCN_TRY(check_codes(codes, exponents, n));
  if (n == 0) return SSCN_OK;
  const int blocks = (int)ceil_div(c, kBlock);
  const unsigned g = grid_of(ceil_div(n * c, 256));
  if (dtype == SSCN_F32)
    k_q8_values<float><<<g, 256, 0, stream>>>(codes, exponents, n, c, blocks, (float*)y, ldy);
  else
    k_q8_values<uint16_t><<<g, 256, 0, stream>>>(codes, exponents, n, c, blocks, (uint16_t*)y, ldy);
  SSCN_HIP(hipGetLastError());
  return SSCN_OK;
}

extern "C" sscn_status sscn_batchnorm_relu_backward_params_q8_workspace(int64_t n, int32_t c, int64_t* bytes) {
  if (n < 0 || c < 1) return fail(SSCN_ERR_INVALID_ARG, "q8: n must be >= 0 and c >= 1");
  if (!bytes) return fail(SSCN_ERR_INVALID_ARG, "q8: NULL bytes");
  *bytes = (int64_t)sizeof(double) * 2 * row_blocks(n) * c;
  return SSCN_OK;
}

extern "C" sscn_status sscn_batchnorm_relu_backward_params_q8(const void* da, int64_t ldd, const int8_t* codes,
                                                              const uint8_t* exponents, int64_t n, int32_t c,
                                                              sscn_dtype dtype, const float* gamma, const float* beta,
                                                              float* dgamma, float* dbeta, void* a, int64_t lda,
                                                              void* workspace, int64_t workspace_bytes,
                                                              hipStream_t stream) {
  SSCN_TRY(check_dtype(dtype));
  SSCN_TRY(check_rows(da, ldd, n, c, dtype));
  if (a) SSCN_TRY(check_rows(a, lda, n, c, dtype));
  SSCN_TRY(check_codes(codes, exponents, n));
  if (!gamma || !beta || !dgamma || !dbeta) return fail(SSCN_ERR_INVALID_ARG, "q8: NULL parameters or outputs");
  int64_t need = 0;
  SSCN_TRY(sscn_batchnorm_relu_backward_params_q8_workspace(n, c, &need));
  if (workspace_bytes < need || !workspace || reinterpret_cast<uintptr_t>(workspace) % sizeof(double) != 0)
    return fail(SSCN_ERR_INVALID_ARG, "q8: no workspace of the size that ..._params_q8_workspace says, 8-byte aligned");
  const int blocks = (int)ceil_div(c, kBlock), parts = row_blocks(n);
  const dim3 grid((unsigned)parts, (unsigned)ceil_div(c, 64));
  double* partial = (double*)workspace;
  if (dtype == SSCN_F32)
    k_params_q8<float><<<grid, 256, 0, stream>>>((const float*)da, ldd, codes, exponents, n, c, blocks, gamma, beta,
                                                 (float*)a, lda, partial);
  else
    k_params_q8<uint16_t><<<grid, 256, 0, stream>>>((const uint16_t*)da, ldd, codes, exponents, n, c, blocks, gamma,
                                                    beta, (uint16_t*)a, lda, partial);
  SSCN_HIP(hipGetLastError());
  k_two_sums<<<(unsigned)ceil_div(c, 64), kFinThreads, 0, stream>>>(partial, parts, c, dbeta, dgamma);
  SSCN_HIP(hipGetLastError());
  return SSCN_OK;
}

extern "C" sscn_status sscn_batchnorm_relu_backward_input_q8(const void* da, int64_t ldd, const int8_t* codes,
                                                             const uint8_t* exponents, int64_t n, int32_t c,
                                                             int32_t col0, int32_t cols, sscn_dtype dtype,
                                                             const float* gamma, const float* beta,
                                                             const float* invstd, const float* dgamma,
                                                             const float* dbeta, const void* add, int64_t ld_add,
                                                             void* dx, int64_t ldx_out, hipStream_t stream) {
  SSCN_TRY(check_dtype(dtype));
  SSCN_TRY(check_rows(da, ldd, n, c, dtype));
  if (col0 < 0 || cols < 1 || col0 > c - cols)
    return fail(SSCN_ERR_INVALID_ARG, "q8: the column range must lie in the layer's channels");
  SSCN_TRY(check_rows(dx, ldx_out, n, cols, dtype));
  if (add) SSCN_TRY(check_rows(add, ld_add, n, cols, dtype));
  SSCN_TRY(check_codes(codes, exponents, n));
  if (!gamma || !beta || !invstd || !dgamma || !dbeta)
    return fail(SSCN_ERR_INVALID_ARG, "q8: NULL parameters or statistics");
  if (n == 0) return SSCN_OK;
  const int blocks = (int)ceil_div(c, kBlock);
  const unsigned g = grid_of(ceil_div(n * cols, 256));
  if (dtype == SSCN_F32)
    k_input_q8<float><<<g, 256, 0, stream>>>((const float*)da, ldd, codes, exponents, n, c, blocks, col0, cols, gamma,
                                             beta, invstd, dgamma, dbeta, (const float*)add, ld_add, (float*)dx,
                                             ldx_out);
  else
    k_input_q8<uint16_t><<<g, 256, 0, stream>>>((const uint16_t*)da, ldd, codes, exponents, n, c, blocks, col0, cols,
                                                gamma, beta, invstd, dgamma, dbeta, (const uint16_t*)add, ld_add,
                                                (uint16_t*)dx, ldx_out);
  SSCN_HIP(hipGetLastError());
  return SSCN_OK;
}
