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
// an infinity or a NaN has the byte 255 and codes 0, and stands for NaN.
#include <algorithm>
#include <type_traits>

#include "internal.h"
#include "numeric.h"
#include "wave.h"

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
__device__ __forceinline__ float power(uint32_t byte) { return __uint_as_float(byte << 23); }  // 2^(byte - 127), byte 1 .. 254
// What a code of 1 stands for: 2^(byte - 127); the bit below the exponent makes
// the byte 0 that (a subnormal number) too, and the byte 255 a NaN, so that
// every code of its block is one.
__device__ __forceinline__ float unit(uint32_t byte) {
  return __uint_as_float(byte << 23 | (byte - 1 >= 254 ? 1u << 22 : 0));
}

// The ReLU's argument as the forward and as the backward pass forms it.
__device__ __forceinline__ float pre_forward(float d, float scale, float beta) { return fmaf(d, scale, beta); }
__device__ __forceinline__ float pre_restored(float v, float gamma, float beta) { return fmaf(v, gamma, beta); }

// relu that lets a NaN through.
__device__ __forceinline__ float relu_nan(float v) { return v <= 0.f ? 0.f : v; }

// How the row-wise kernels below share the work: a thread takes a piece of P
// consecutive channels (16 bytes of values, 4 in fp32 and 8 in bf16, at whatever
// alignment the row has; the hardware takes any) of every so many rows, so that
// the channels' constants stay in its registers; 32 / P threads make a block of
// 32 channels, a workgroup of 256 takes several rows at once, or (blockIdx.y)
// 8 P blocks of one.
//
// A row's last piece may be cut.  Where its block holds a whole piece's channels
// and nothing is computed in place it slides back over the piece before: the
// channels that they share are computed twice, to the same bits (the sums count
// them once).  Else it goes value by value (CUT; keeping 200,003 x 70 fp32: 49
// us that way, 34 sliding).
constexpr int kThreads = 256;
template <int P>
struct Place {
  static constexpr int kLanes = kBlock / P, kSpan = kThreads / kLanes;  // threads to a block, blocks to a workgroup
  int col, valid;     // first channel; channels of the piece (0: nothing to do)
  int twice = 0;      // of a piece that slid: channels of the piece before
  int block, sub;     // block of the row; piece of the block
  int64_t row, step;  // first row, and how many on to the next
  __device__ Place(int c, int blocks, bool slide) {
    const int lanes = kLanes * min(blocks - (int)blockIdx.y * kSpan, kSpan), rows = kThreads / lanes;
    const int in_row = (int)threadIdx.x % lanes, r = (int)threadIdx.x / lanes;
    block = (int)blockIdx.y * kSpan + in_row / kLanes;
    sub = in_row % kLanes;
    col = block * kBlock + sub * P;
    valid = max(0, min(P, c - col));
    if (slide && valid > 0 && valid < P) {
      twice = P - valid;
      col = c - P;
      valid = P;
    }
    row = r < rows ? (int64_t)blockIdx.x * rows + r : INT64_MAX;  // (threads beyond the last whole row take none)
    step = (int64_t)gridDim.x * rows;
  }
};
template <typename T>
constexpr int kPiece = 16 / (int)sizeof(T);

// A piece from memory, as it is stored; a short one (only where CUT says that
// there may be some) value by value.  Values past the row's end are 0.
template <typename T, bool CUT>
__device__ __forceinline__ void load_piece(const T* p, int valid, uint32_t (&w)[4]) {
  constexpr int P = kPiece<T>;
  if (valid == P) {
    __builtin_memcpy(w, p, 16);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = 0;
    if constexpr (CUT) {
#pragma unroll
      for (int i = 0; i < P - 1; ++i)
        if (i < valid) {
          if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(p[i]);
          else w[i / 2] |= (uint32_t)p[i] << 16 * (i % 2);
        }
    }
  }
}
template <int P>
__device__ __forceinline__ float value(const uint32_t (&w)[4], int i) {
  if constexpr (P == 4) return __uint_as_float(w[i]);
  else return __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
}
template <typename T, bool CUT>
__device__ __forceinline__ void store_piece(T* p, int valid, const float (&x)[kPiece<T>]) {
  constexpr int P = kPiece<T>;
  if (valid == P) {
    if constexpr (sizeof(T) == 4) {
      __builtin_memcpy(p, x, 16);
    } else {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
      __builtin_memcpy(p, w, 16);
    }
  } else if constexpr (CUT) {
#pragma unroll
    for (int i = 0; i < P - 1; ++i)
      if (i < valid) st(p + i, x[i]);
  }
}
// A piece's codes, and what they stand for: code * 2^e, exact, and infinite only
// where that is beyond fp32.
template <int P, bool CUT>
__device__ __forceinline__ void load_codes(const int8_t* p, int valid, uint32_t (&w)[P / 4]) {
  if (valid == P) {
    __builtin_memcpy(w, p, P);
  } else {
#pragma unroll
    for (int i = 0; i < P / 4; ++i) w[i] = 0;
    if constexpr (CUT) {
#pragma unroll
      for (int i = 0; i < P - 1; ++i)
        if (i < valid) w[i / 4] |= (uint32_t)(uint8_t)p[i] << 8 * (i % 4);
    }
  }
}
template <int P>
__device__ __forceinline__ void decode(const uint32_t (&w)[P / 4], uint32_t byte, float (&v)[P]) {
  const float s = unit(byte);
#pragma unroll
  for (int i = 0; i < P; ++i) v[i] = (float)(int8_t)(w[i / 4] >> 8 * (i % 4)) * s;
}
// Per-channel constants of a piece.
template <int P>
__device__ __forceinline__ void constants(const float* p, int valid, float (&k)[P]) {
  if (valid == P) {
    __builtin_memcpy(k, p, 4 * P);
  } else {
#pragma unroll
    for (int i = 0; i < P; ++i) k[i] = i < valid ? p[i] : 0.f;
  }
}

// Every kernel takes kRows of its rows a turn, so that their loads are in
// flight together (1,964,906 x 32 fp32, one row: 158 us for the parameter
// gradients with the activations, 115 with two).  All of them are bound by
// memory; at 1,964,906 x 32 bf16 (copy rate 5.5 TB/s): k_apply_q8 64 us for 317
// MB, 4.9 TB/s; k_q8_values 33 us for 191 MB, 5.8; k_params_q8 62 us for 317 MB,
// 5.1; k_input_q8_pieces 61 us for 317 MB, 5.2.
constexpr int kRows = 2;

template <typename T, bool CUT>
__global__ __launch_bounds__(kThreads) void k_apply_q8(const T* __restrict__ x, int64_t ldx, int64_t n, int c,
                                                       int blocks, bool slide, const float* __restrict__ mean,
                                                       const float* __restrict__ invstd,
                                                       const float* __restrict__ scale,
                                                       const float* __restrict__ gamma,
                                                       const float* __restrict__ beta, T* __restrict__ y, int64_t ldy,
                                                       int8_t* __restrict__ codes, uint8_t* __restrict__ exponents) {
  constexpr int P = kPiece<T>;
  const Place<P> w(c, blocks, slide);
  float mu[P], is[P], sc[P], ga[P], be[P];
  constants<P>(mean + w.col, w.valid, mu);
  constants<P>(invstd + w.col, w.valid, is);
  constants<P>(scale + w.col, w.valid, sc);
  constants<P>(gamma + w.col, w.valid, ga);
  constants<P>(beta + w.col, w.valid, be);
  // the threads of a block share its maximum: all of them take every turn
  for (int64_t r0 = w.row; r0 < n; r0 += kRows * w.step) {
    uint32_t in[kRows][4];
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      const int64_t r = r0 + u * w.step;
      load_piece<T, CUT>(x + r * ldx + w.col, r < n ? w.valid : 0, in[u]);
    }
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      const int64_t r = r0 + u * w.step;
      if (r >= n) break;
      float d[P], v[P], a[P], most = 0.f;
#pragma unroll
      for (int i = 0; i < P; ++i) {
        d[i] = value<P>(in[u], i) - mu[i];
        v[i] = d[i] * is[i];
        most = OpMax::of(most, fabsf(v[i]));  // 0 past the row's end
      }
      most = wave_reduce<OpMax, 1, Place<P>::kLanes>(most);
      const uint32_t byte = exponent_byte(__float_as_uint(most) & 0x7fffffffu);
      const float up = power(254 - byte), down = power(byte);
      uint32_t q8[P / 4] = {};
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const float pre = pre_forward(d[i], sc[i], be[i]);
        a[i] = fmaxf(0.f, pre);
        const float q = rintf(v[i] * up);
        const bool want = pre > 0.f, have = pre_restored(q * down, ga[i], be[i]) > 0.f;
        // towards the side of the forward
        const float way = want == have || ga[i] == 0.f ? 0.f : (ga[i] > 0.f) == want ? 1.f : -1.f;
        const int code = byte == 255 ? 0 : (int)fminf(fmaxf(q + way, -127.f), 127.f);
        q8[i / 4] |= (uint32_t)(uint8_t)code << 8 * (i % 4);
      }
      store_piece<T, CUT>(y + r * ldy + w.col, w.valid, a);
      int8_t* to = codes + r * c + w.col;
      if (w.valid == P) {
        __builtin_memcpy(to, q8, P);
      } else if constexpr (CUT) {
#pragma unroll
        for (int i = 0; i < P - 1; ++i)
          if (i < w.valid) to[i] = (int8_t)(q8[i / 4] >> 8 * (i % 4));
      }
      if (w.sub == 0) exponents[r * blocks + w.block] = (uint8_t)byte;
    }
  }
}

// The codes and exponent bytes of kRows rows, and the matrix piece of each.
template <typename T, bool CUT>
struct Turn {
  static constexpr int P = kPiece<T>;
  uint32_t q[kRows][P / 4], d[kRows][4], byte[kRows];
  __device__ __forceinline__ Turn(const Place<P>& w, int64_t r0, int64_t n, const int8_t* codes, int c,
                                  const uint8_t* exps, int blocks, const T* m, int64_t ldm) {
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      const int64_t r = r0 + u * w.step;
      const int valid = r < n ? w.valid : 0;
      if (m) load_piece<T, CUT>(m + r * ldm, valid, d[u]);
      load_codes<P, CUT>(codes + r * c, valid, q[u]);
      byte[u] = r < n ? exps[r * blocks] : 0;
    }
  }
};

// The values that the codes stand for.
template <typename T, bool CUT>
__global__ __launch_bounds__(kThreads) void k_q8_values(const int8_t* __restrict__ codes,
                                                        const uint8_t* __restrict__ exponents, int64_t n, int c,
                                                        int blocks, bool slide, T* __restrict__ y, int64_t ldy) {
  constexpr int P = kPiece<T>;
  const Place<P> w(c, blocks, slide);
  if (w.valid == 0) return;
  for (int64_t r0 = w.row; r0 < n; r0 += kRows * w.step) {
    const Turn<T, CUT> t(w, r0, n, codes + w.col, c, exponents + w.block, blocks, nullptr, 0);
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      const int64_t r = r0 + u * w.step;
      if (r >= n) break;
      float v[P];
      decode<P>(t.q[u], t.byte[u], v);
      store_piece<T, CUT>(y + r * ldy + w.col, w.valid, v);
    }
  }
}

// Per channel the fp64 sums of dz and dz * xhat, dz = dA where the restored
// ReLU passes, over the rows of this workgroup (a fixed set, added in a fixed
// order), and the restored activations.
template <typename T, bool CUT>
__global__ __launch_bounds__(kThreads) void k_params_q8(const T* __restrict__ da, int64_t ldd,
                                                        const int8_t* __restrict__ codes,
                                                        const uint8_t* __restrict__ exponents, int64_t n, int c,
                                                        int blocks, bool slide, const float* __restrict__ gamma,
                                                        const float* __restrict__ beta, T* __restrict__ a, int64_t lda,
                                                        double* __restrict__ partial) {
  constexpr int P = kPiece<T>;
  __shared__ double red[P][kThreads + 1];
  const Place<P> w(c, blocks, slide);
  float ga[P], be[P];
  constants<P>(gamma + w.col, w.valid, ga);
  constants<P>(beta + w.col, w.valid, be);
  double s0[P], s1[P];
#pragma unroll
  for (int i = 0; i < P; ++i) s0[i] = s1[i] = 0.0;
  if (w.valid > 0)
    for (int64_t r0 = w.row; r0 < n; r0 += kRows * w.step) {
      const Turn<T, CUT> t(w, r0, n, codes + w.col, c, exponents + w.block, blocks, da + w.col, ldd);
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        const int64_t r = r0 + u * w.step;
        if (r >= n) break;
        float v[P], out[P];
        decode<P>(t.q[u], t.byte[u], v);
#pragma unroll
        for (int i = 0; i < P; ++i) {
          const float pre = pre_restored(v[i], ga[i], be[i]);
          const float dz = pre > 0.f ? value<P>(t.d[u], i) : 0.f;
          s0[i] += dz;
          s1[i] = fma((double)dz, (double)v[i], s1[i]);
          out[i] = relu_nan(pre);
        }
        if (a) store_piece<T, CUT>(a + r * lda + w.col, w.valid, out);
      }
    }
  // thread t adds the workgroup's rows of channel t of its span, in order
  constexpr int kSpan = Place<P>::kSpan;
  const int here = min(blocks - (int)blockIdx.y * kSpan, kSpan), lanes = Place<P>::kLanes * here;
  const int rows = kThreads / lanes, c0 = (int)blockIdx.y * kSpan * kBlock;
#pragma unroll
  for (int kind = 0; kind < 2; ++kind) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < P; ++i)
      if (i >= w.twice) red[i - w.twice][threadIdx.x] = kind ? s1[i] : s0[i];
    __syncthreads();
    for (int t = threadIdx.x; t < min(c - c0, here * kBlock); t += kThreads) {
      double sum = 0.0;
      for (int q = 0; q < rows; ++q) sum += red[t % P][q * lanes + t / P];
      partial[((int64_t)blockIdx.x * 2 + kind) * c + c0 + t] = sum;
    }
  }
}

// Adds the parts, 16 channels to a workgroup: thread t the parts t / 16, + 64,
// .. of channel t % 16 in order, then the 64 threads of a channel in a fixed
// tree.  6 us for 1024 parts of 32 or 128 channels: latency.  (With 64 channels
// to a workgroup, too few for the CUs, and one row a turn above, the parameter
// gradients of 20,000 x 512 bf16 took 29 us, 18 now.)
__global__ __launch_bounds__(1024) void k_sum_parts(const double* __restrict__ partial, int parts, int c,
                                                    float* __restrict__ dbeta, float* __restrict__ dgamma) {
  __shared__ double red[2][64][16];
  const int k = threadIdx.x % 16, p0 = threadIdx.x / 16, col = blockIdx.x * 16 + k;
  double s0 = 0.0, s1 = 0.0;
  if (col < c) {
#pragma unroll 4
    for (int p = p0; p < parts; p += 64) {
      s0 += partial[((int64_t)p * 2) * c + col];
      s1 += partial[((int64_t)p * 2 + 1) * c + col];
    }
  }
  red[0][p0][k] = s0;
  red[1][p0][k] = s1;
  __syncthreads();
#pragma unroll
  for (int h = 32; h >= 1; h /= 2) {
    if (p0 < h) {
      red[0][p0][k] += red[0][p0 + h][k];
      red[1][p0][k] += red[1][p0 + h][k];
    }
    __syncthreads();
  }
  if (p0 == 0 && col < c) {
    dbeta[col] = (float)red[0][0][k];
    dgamma[col] = (float)red[1][0][k];
  }
}

// dx for the channels [col0, col0 + cols), col0 a multiple of the piece (so that
// one lies in one block).
template <typename T, bool CUT>
__global__ __launch_bounds__(kThreads) void k_input_q8_pieces(
    const T* __restrict__ da, int64_t ldd, const int8_t* __restrict__ codes, const uint8_t* __restrict__ exponents,
    int64_t n, int c, int blocks, int col0, int cols, bool slide, const float* __restrict__ gamma,
    const float* __restrict__ beta,
    const float* __restrict__ invstd, const float* __restrict__ dgamma, const float* __restrict__ dbeta,
    const T* __restrict__ add, int64_t lda, T* __restrict__ dx, int64_t ldo) {
  constexpr int P = kPiece<T>;
  const Place<P> w(cols, (cols + kBlock - 1) / kBlock, slide);
  if (w.valid == 0) return;
  const int col = col0 + w.col;  // of the layer
  const float inv_n = 1.f / (float)n;
  float ga[P], be[P], m0[P], m1[P], gi[P];
  constants<P>(gamma + col, w.valid, ga);
  constants<P>(beta + col, w.valid, be);
  constants<P>(dbeta + col, w.valid, m0);
  constants<P>(dgamma + col, w.valid, m1);
  constants<P>(invstd + col, w.valid, gi);
#pragma unroll
  for (int i = 0; i < P; ++i) {
    m0[i] *= inv_n;
    m1[i] *= inv_n;
    gi[i] *= ga[i];
  }
  for (int64_t r0 = w.row; r0 < n; r0 += kRows * w.step) {
    const Turn<T, CUT> t(w, r0, n, codes + col, c, exponents + col / kBlock, blocks, da + col, ldd);
    uint32_t more[kRows][4];
    if (add) {
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        const int64_t r = r0 + u * w.step;
        load_piece<T, CUT>(add + r * lda + w.col, r < n ? w.valid : 0, more[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      const int64_t r = r0 + u * w.step;
      if (r >= n) break;
      float v[P], out[P];
      decode<P>(t.q[u], t.byte[u], v);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const float dz = pre_restored(v[i], ga[i], be[i]) > 0.f ? value<P>(t.d[u], i) : 0.f;
        out[i] = gi[i] * (dz - m0[i] - v[i] * m1[i]);
        if (add) out[i] += value<P>(more[u], i);
      }
      store_piece<T, CUT>(dx + r * ldo + w.col, w.valid, out);
    }
  }
}

// dx = gamma invstd (dz - dbeta / n - xhat dgamma / n) (+ add) for the columns
// [col0, col0 + cols) of the layer; dx and add hold just those.  An element a
// lane: for ranges that start inside a piece.
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
    const float v = (float)codes[r * c + col] * unit(exponents[r * blocks + col / kBlock]);
    const float dz = pre_restored(v, gamma[col], beta[col]) > 0.f ? ld(da + r * ldd + col) : 0.f;
    float out = gamma[col] * invstd[col] * (dz - dbeta[col] * inv_n - v * (dgamma[col] * inv_n));
    if (add) out += ld(add + r * lda + k);
    st(dx + r * ldo + k, out);
  }
}

unsigned grid_of(int64_t work) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>(work, 16384)); }
int piece_of(sscn_dtype dtype) { return dtype == SSCN_F32 ? kPiece<float> : kPiece<uint16_t>; }
// Grid of the kernels that go by Place, `most` workgroups over the rows at most.
dim3 place_grid(int64_t n, int blocks, int64_t most, sscn_dtype dtype) {
  const int lanes = kBlock / piece_of(dtype), span = kThreads / lanes;
  const int rows = kThreads / (lanes * std::min(blocks, span));
  return dim3((unsigned)std::max<int64_t>(1, std::min<int64_t>(ceil_div(n, rows), most)),
              (unsigned)ceil_div(blocks, span));
}
// Workgroups over the rows of the row-wise kernels: 8 to a CU, which holds 4 to 8
// of them at once, by their registers.
constexpr int64_t kRowGroups = 2048;

// f(a value of the element type, whether pieces are cut, whether they slide) for
// the channels up to `end` of a layer, `cols` of them.
template <class F>
sscn_status by_type(sscn_dtype dtype, int cols, int end, bool in_place, const F& f) {
  const int piece = piece_of(dtype);
  const bool slide = cols % piece != 0 && end % kBlock >= piece && cols >= piece && !in_place;
  const bool cut = cols % piece != 0 && !slide;
  if (dtype == SSCN_F32) {
    if (cut) f(float{}, std::true_type{}, false);
    else f(float{}, std::false_type{}, slide);
  } else {
    if (cut) f(uint16_t{}, std::true_type{}, false);
    else f(uint16_t{}, std::false_type{}, slide);
  }
  SSCN_HIP(hipGetLastError());
  return SSCN_OK;
}

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
  if (x == y && ldx != ldy) return fail(SSCN_ERR_INVALID_ARG, "q8: y in x's place with another row stride");
  if (x != y && rows_share(x, ldx, c, y, ldy, c, n, dtype == SSCN_F32 ? 4 : 2))
    return fail(SSCN_ERR_INVALID_ARG, "q8: y shares memory with x, but is not x");
  const int blocks = (int)ceil_div(c, kBlock);
  const dim3 g = place_grid(n, blocks, kRowGroups, dtype);
  return by_type(dtype, c, c, x == y, [&](auto t, auto cut, bool slide) {
    using T = decltype(t);
    k_apply_q8<T, decltype(cut)::value><<<g, kThreads, 0, stream>>>((const T*)x, ldx, n, c, blocks, slide, mean, invstd,
                                                                    scale, gamma, beta, (T*)y, ldy, codes, exponents);
  });
}

extern "C" sscn_status sscn_q8_values(const int8_t* codes, const uint8_t* exponents, int64_t n, int32_t c,
                                      sscn_dtype dtype, void* y, int64_t ldy, hipStream_t stream) {
  SSCN_TRY(check_dtype(dtype));
  SSCN_TRY(check_rows(y, ldy, n, c, dtype));
  SSCN_TRY(check_codes(codes, exponents, n));
  if (n == 0) return SSCN_OK;
  const int blocks = (int)ceil_div(c, kBlock);
  const dim3 g = place_grid(n, blocks, kRowGroups, dtype);
  return by_type(dtype, c, c, false, [&](auto t, auto cut, bool slide) {
    using T = decltype(t);
    k_q8_values<T, decltype(cut)::value><<<g, kThreads, 0, stream>>>(codes, exponents, n, c, blocks, slide, (T*)y, ldy);
  });
}

extern "C" sscn_status sscn_batchnorm_relu_backward_params_q8_workspace(int64_t n, int32_t c, int64_t* bytes) {
  if (n < 0 || c < 1) return fail(SSCN_ERR_INVALID_ARG, "q8: n must be >= 0 and c >= 1");
  if (!bytes) return fail(SSCN_ERR_INVALID_ARG, "q8: NULL bytes");
  // (as many workgroups at least as either type's pieces give)
  *bytes = (int64_t)sizeof(double) * 2 * place_grid(n, (int)ceil_div(c, kBlock), kMaxPartials, SSCN_F32).x * c;
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
  if (n > 0 && (a == da || (a && rows_share(da, ldd, c, a, lda, c, n, dtype == SSCN_F32 ? 4 : 2))))
    return fail(SSCN_ERR_INVALID_ARG, "q8: a cannot replace dA");
  int64_t need = 0;
  SSCN_TRY(sscn_batchnorm_relu_backward_params_q8_workspace(n, c, &need));
  if (workspace_bytes < need || !workspace || reinterpret_cast<uintptr_t>(workspace) % sizeof(double) != 0)
    return fail(SSCN_ERR_INVALID_ARG, "q8: no workspace of the size that ..._params_q8_workspace says, 8-byte aligned");
  const int blocks = (int)ceil_div(c, kBlock);
  const dim3 grid = place_grid(n, blocks, kMaxPartials, dtype);
  const int parts = (int)grid.x;
  double* partial = (double*)workspace;
  SSCN_TRY(by_type(dtype, c, c, false, [&](auto t, auto cut, bool slide) {
    using T = decltype(t);
    k_params_q8<T, decltype(cut)::value><<<grid, kThreads, 0, stream>>>(
        (const T*)da, ldd, codes, exponents, n, c, blocks, slide, gamma, beta, (T*)a, lda, partial);
  }));
  k_sum_parts<<<(unsigned)ceil_div(c, 16), 1024, 0, stream>>>(partial, parts, c, dbeta, dgamma);
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
  const int64_t size = dtype == SSCN_F32 ? 4 : 2;
  if (dx == da || rows_share(da, ldd, c, dx, ldx_out, cols, n, size))
    return fail(SSCN_ERR_INVALID_ARG, "q8: dx cannot replace dA or columns of it");
  if (dx == add && ld_add != ldx_out) return fail(SSCN_ERR_INVALID_ARG, "q8: dx in add's place with another row stride");
  if (add && dx != add && rows_share(add, ld_add, cols, dx, ldx_out, cols, n, size))
    return fail(SSCN_ERR_INVALID_ARG, "q8: dx shares memory with add, but is not add");
  const int blocks = (int)ceil_div(c, kBlock);
  if (col0 % piece_of(dtype) == 0) {
    const dim3 g = place_grid(n, (int)ceil_div(cols, kBlock), kRowGroups, dtype);
    return by_type(dtype, cols, col0 + cols, add == dx, [&](auto t, auto cut, bool slide) {
      using T = decltype(t);
      k_input_q8_pieces<T, decltype(cut)::value><<<g, kThreads, 0, stream>>>(
          (const T*)da, ldd, codes, exponents, n, c, blocks, col0, cols, slide, gamma, beta, invstd, dgamma, dbeta,
          (const T*)add, ld_add, (T*)dx, ldx_out);
    });
  }
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
