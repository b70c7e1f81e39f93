// Microscaled 4-bit floating point: quantizing, expanding, and the product for any shape; see mx.cuh for the format.
#include "mx.cuh"

namespace aiq {
namespace {

// ---------------------------------------------------------------------------------------
// quantize
// ---------------------------------------------------------------------------------------
constexpr int kMxThreads = 256;
constexpr int kMxUnroll = 4;

// Rows that start on 16 bytes: a lane takes eight values (one word of codes), four lanes a block.
template <typename T>
__global__ void __launch_bounds__(kMxThreads)
mx_quantize_kernel(const T* __restrict__ x, int64_t x_stride, int K, uint32_t units, FastDiv words, int scale_row,
                   uint32_t* __restrict__ codes, uint8_t* __restrict__ scales) {
  const uint32_t u0 = blockIdx.x * (kMxThreads * kMxUnroll) + threadIdx.x;
  float f[kMxUnroll][8];
  uint32_t row[kMxUnroll], word[kMxUnroll];
#pragma unroll
  for (int i = 0; i < kMxUnroll; ++i) {
    const uint32_t u = u0 + i * kMxThreads;
    row[i] = words.div(u);
    word[i] = u - row[i] * words.d;
    const int k = (int)word[i] * 8;
    const T* src = x + (int64_t)row[i] * x_stride + k;
    if (u < units && k + 8 <= K) {
      load8(src, f[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) f[i][j] = u < units && k + j < K ? to_float(src[j]) : 0.f;
    }
  }
#pragma unroll
  for (int i = 0; i < kMxUnroll; ++i) {
    const uint32_t u = u0 + i * kMxThreads;
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(f[i][j]) & 0x7FFFFFFFu);
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const uint32_t s = mx_scale_byte(top);
    const float inv = mx_inverse_scale(s);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[i][j] *= inv;
    if (u < units) {
      codes[u] = s == 255 ? 0u : mx_codes8(f[i]);
      uint8_t* sr = scales + (int64_t)row[i] * scale_row;
      if ((word[i] & 3) == 0) sr[word[i] >> 2] = (uint8_t)s;
      if (word[i] + 1 == words.d)
        for (int b = (int)words.d / 4; b < scale_row; ++b) sr[b] = 0;
    }
  }
}

// Any row: a lane takes every 32nd value of 256, so that a load of the warp is one piece of memory wherever it starts and a
// block is one value per lane.  The eight 4-bit codes of a lane (one per block) then become one word of eight neighbours by a
// transposition among eight lanes.
template <typename T>
__global__ void __launch_bounds__(kMxThreads)
mx_quantize_any_kernel(const T* __restrict__ x, int64_t x_stride, int K, int64_t segments, FastDiv per_row, int words, int scale_row,
                       uint32_t* __restrict__ codes, uint8_t* __restrict__ scales) {
  const uint32_t seg = blockIdx.x * (kMxThreads / 32) + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (seg >= segments) return;
  const uint32_t row = per_row.div(seg);
  const int part = (int)(seg - row * per_row.d), k0 = part * 256;
  const T* src = x + (int64_t)row * x_stride;
  float f[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int k = k0 + j * 32 + lane;
    f[j] = k < K ? to_float(src[k]) : 0.f;
  }
  uint32_t packed = 0, my_scale = 0;
  float v[8];
  uint32_t dead = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t s = mx_scale_byte(__reduce_max_sync(0xffffffffu, __float_as_uint(f[j]) & 0x7FFFFFFFu));
    v[j] = f[j] * mx_inverse_scale(s);
    if (s == 255) dead |= 0xFu << (4 * j);
    if (lane == j) my_scale = s;
  }
  packed = mx_codes8(v) & ~dead;                       // nibble j: block j of this lane
  // 8 x 8 transposition of nibbles: afterwards lane 8g + i holds elements 8g .. 8g + 7 of block i
  const int i = lane & 7;
  uint32_t other = __shfl_xor_sync(0xffffffffu, packed, 4);
  packed = (i & 4) ? (packed & 0xFFFF0000u) | (other >> 16) : (packed & 0x0000FFFFu) | (other << 16);
  other = __shfl_xor_sync(0xffffffffu, packed, 2);
  packed = (i & 2) ? (packed & 0xFF00FF00u) | ((other >> 8) & 0x00FF00FFu) : (packed & 0x00FF00FFu) | ((other << 8) & 0xFF00FF00u);
  other = __shfl_xor_sync(0xffffffffu, packed, 1);
  packed = (i & 1) ? (packed & 0xF0F0F0F0u) | ((other >> 4) & 0x0F0F0F0Fu) : (packed & 0x0F0F0F0Fu) | ((other << 4) & 0xF0F0F0F0u);
  const int word = part * 32 + i * 4 + (lane >> 3);
  if (word < words) codes[(int64_t)row * words + word] = packed;
  uint8_t* sr = scales + (int64_t)row * scale_row + part * 8;
  if (lane < 8 && part * 8 + lane < scale_row) sr[lane] = (uint8_t)my_scale;       // blocks behind K: zero
  if (part + 1 == (int)per_row.d && lane >= 8 && part * 8 + lane < scale_row) sr[lane] = 0;
}

template <typename T>
aiq_status_t quantize_rows(const T* x, int64_t rows, int K, int64_t x_stride, uint8_t* codes, uint8_t* scales, cudaStream_t s) {
  const int64_t row_bytes = mx_row_bytes(K), scale_row = mx_scale_row_bytes(K);
  const bool aligned = (((uintptr_t)x) & 15) == 0 && (rows == 1 || x_stride * (int64_t)sizeof(T) % 16 == 0);
  const uint32_t per_row = (uint32_t)(aligned ? row_bytes / 4 : (row_bytes * 2 + 255) / 256);
  const int64_t step = max((int64_t)1, (int64_t)((1u << 30) / per_row));       // rows per launch: units below 2^31
  for (int64_t r = 0; r < rows; r += step) {
    const int64_t n = min(step, rows - r), units = n * per_row;
    const T* xr = x + r * x_stride;
    uint32_t* c = reinterpret_cast<uint32_t*>(codes + r * row_bytes);
    uint8_t* sc = scales + r * scale_row;
    LaunchScope scope(AIQ_KERNEL_QUANTIZE, s, 2.0 * n * K, (double)n * (sizeof(T) * (double)K + row_bytes + scale_row));
    if (aligned) {
      const int64_t per_block = kMxThreads * kMxUnroll;
      mx_quantize_kernel<T><<<(unsigned)((units + per_block - 1) / per_block), kMxThreads, 0, s>>>(
          xr, x_stride, K, (uint32_t)units, FastDiv(per_row), (int)scale_row, c, sc);
    } else {
      mx_quantize_any_kernel<T><<<(unsigned)((units + kMxThreads / 32 - 1) / (kMxThreads / 32)), kMxThreads, 0, s>>>(
          xr, x_stride, K, units, FastDiv(per_row), (int)(row_bytes / 4), (int)scale_row, c, sc);
    }
    AIQ_LAUNCH_CHECK("mx_quantize");
  }
  return AIQ_OK;
}

// ---------------------------------------------------------------------------------------
// dequantize
// ---------------------------------------------------------------------------------------
template <typename T>
__device__ __forceinline__ void store8(T* p, const float* f) {
  if (sizeof(T) == 4) {
    reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      T h[2] = {from_float<T>(f[2 * i]), from_float<T>(f[2 * i + 1])};
      w[i] = *reinterpret_cast<const uint32_t*>(h);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// A lane takes one word of codes.  Rows that start on 16 bytes are written eight values per lane.
template <typename T>
__global__ void __launch_bounds__(kMxThreads)
mx_dequantize_kernel(const uint32_t* __restrict__ codes, const uint8_t* __restrict__ scales, int scale_row, int K, uint32_t units,
                     FastDiv words, T* __restrict__ y, int64_t y_stride) {
  const uint32_t u0 = blockIdx.x * (kMxThreads * kMxUnroll) + threadIdx.x;
  uint32_t row[kMxUnroll], word[kMxUnroll], raw[kMxUnroll], sb[kMxUnroll];
#pragma unroll
  for (int i = 0; i < kMxUnroll; ++i) {
    const uint32_t u = u0 + i * kMxThreads;
    row[i] = words.div(u);
    word[i] = u - row[i] * words.d;
    raw[i] = u < units ? codes[u] : 0u;
    sb[i] = u < units ? scales[(int64_t)row[i] * scale_row + (word[i] >> 2)] : 0u;
  }
#pragma unroll
  for (int i = 0; i < kMxUnroll; ++i) {
    if (u0 + i * kMxThreads >= units) break;
    const int k = (int)word[i] * 8;
    const float s = mx_scale(sb[i]);
    float f[8];
    mx_expand8(raw[i], f);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] *= s;
    T* dst = y + (int64_t)row[i] * y_stride + k;
    if (k + 8 <= K) {
      store8(dst, f);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (k + j < K) dst[j] = from_float<T>(f[j]);
    }
  }
}

// Any row: a warp takes 256 values; a lane holds one word of codes and writes every 32nd value, so that a store of the warp is
// one piece of memory wherever it starts.
template <typename T>
__global__ void __launch_bounds__(kMxThreads)
mx_dequantize_any_kernel(const uint32_t* __restrict__ codes, const uint8_t* __restrict__ scales, int words, int scale_row, int K,
                         int64_t segments, FastDiv per_row, T* __restrict__ y, int64_t y_stride) {
  const uint32_t seg = blockIdx.x * (kMxThreads / 32) + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (seg >= segments) return;
  const uint32_t row = per_row.div(seg);
  const int part = (int)(seg - row * per_row.d), k0 = part * 256, word = part * 32 + lane;
  const uint32_t raw = word < words ? codes[(int64_t)row * words + word] : 0u;
  const float scale = word < words ? mx_scale(scales[(int64_t)row * scale_row + (word >> 2)]) : 0.f;
  T* dst = y + (int64_t)row * y_stride + k0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int from = j * 4 + (lane >> 3);                     // the lane that holds value 32 j + lane
    const uint32_t w = __shfl_sync(0xffffffffu, raw, from);
    const float s = __shfl_sync(0xffffffffu, scale, from);
    float f[8];
    mx_expand8((w >> (4 * (lane & 7))) & 0xFu, f);
    if (k0 + j * 32 + lane < K) dst[j * 32 + lane] = from_float<T>(f[0] * s);
  }
}

template <typename T>
aiq_status_t dequantize_rows(const uint8_t* codes, const uint8_t* scales, int64_t rows, int K, T* y, int64_t y_stride, cudaStream_t s) {
  const int64_t row_bytes = mx_row_bytes(K), scale_row = mx_scale_row_bytes(K);
  const bool aligned = (((uintptr_t)y) & 15) == 0 && (rows == 1 || y_stride * (int64_t)sizeof(T) % 16 == 0);
  const uint32_t per_row = (uint32_t)(aligned ? row_bytes / 4 : (row_bytes * 2 + 255) / 256);
  const int64_t step = max((int64_t)1, (int64_t)((1u << 30) / per_row));
  for (int64_t r = 0; r < rows; r += step) {
    const int64_t n = min(step, rows - r), units = n * per_row;
    const uint32_t* c = reinterpret_cast<const uint32_t*>(codes + r * row_bytes);
    const uint8_t* sc = scales + r * scale_row;
    T* yr = y + r * y_stride;
    LaunchScope scope(AIQ_KERNEL_QUANTIZE, s, (double)n * K, (double)n * (sizeof(T) * (double)K + row_bytes + scale_row));
    if (aligned) {
      const int64_t per_block = kMxThreads * kMxUnroll;
      mx_dequantize_kernel<T><<<(unsigned)((units + per_block - 1) / per_block), kMxThreads, 0, s>>>(
          c, sc, (int)scale_row, K, (uint32_t)units, FastDiv(per_row), yr, y_stride);
    } else {
      mx_dequantize_any_kernel<T><<<(unsigned)((units + kMxThreads / 32 - 1) / (kMxThreads / 32)), kMxThreads, 0, s>>>(
          c, sc, (int)(row_bytes / 4), (int)scale_row, K, units, FastDiv(per_row), yr, y_stride);
    }
    AIQ_LAUNCH_CHECK("mx_dequantize");
  }
  return AIQ_OK;
}

// ---------------------------------------------------------------------------------------
// the product, any shape
// ---------------------------------------------------------------------------------------
// A warp computes one output channel for MT rows of x; a lane takes every 32nd block of the weight row.  float32 throughout.
constexpr int kPlainRows = 4;

// eight values of x from k on (k a multiple of 8)
template <typename T>
struct PlainX {
  static constexpr bool kScaled = false;
  const T* x;
  int64_t stride;
  bool vec;
  __device__ __forceinline__ float block_scale(int64_t, int) const { return 1.f; }
  __device__ __forceinline__ void get8(int64_t m, int k, int K, float* f) const {
    const T* p = x + m * stride + k;
    if (vec && k + 8 <= K) {
      load8(p, f);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = k + j < K ? to_float(p[j]) : 0.f;
    }
  }
};
struct PlainMx {
  static constexpr bool kScaled = true;
  const uint8_t *codes, *scales;
  int64_t row_bytes, scale_row;
  __device__ __forceinline__ float block_scale(int64_t m, int b) const { return mx_scale(scales[m * scale_row + b]); }
  __device__ __forceinline__ void get8(int64_t m, int k, int, float* f) const {
    mx_expand8(*reinterpret_cast<const uint32_t*>(codes + m * row_bytes + (k >> 1)), f);
  }
};

template <typename X, typename T>
__global__ void __launch_bounds__(kMxThreads)
mx_product_plain_kernel(X x, const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t row_bytes, int64_t scale_row,
                        const float* __restrict__ bias, int N, int K, int M, T* __restrict__ y, int64_t y_stride) {
  const int n = blockIdx.x * (kMxThreads / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (n >= N) return;
  const int blocks = (K + MX_BLOCK - 1) / MX_BLOCK;
  for (int64_t m0 = (int64_t)blockIdx.y * kPlainRows; m0 < M; m0 += (int64_t)gridDim.y * kPlainRows) {
    float acc[kPlainRows] = {};
    for (int b = lane; b < blocks; b += 32) {
      const uint4 raw = *reinterpret_cast<const uint4*>(codes + n * row_bytes + (int64_t)b * 16);
      const float ws = mx_scale(scales[n * scale_row + b]);
      const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
      float sum[kPlainRows] = {};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float wf[8], xf[8];
        mx_expand8(w[j], wf);
        if (!X::kScaled) {                       // the weights' own values: x may be as large as its type allows
#pragma unroll
          for (int e = 0; e < 8; ++e) wf[e] *= ws;
        }
#pragma unroll
        for (int r = 0; r < kPlainRows; ++r) {
          if (m0 + r < M) {
            x.get8(m0 + r, b * MX_BLOCK + j * 8, K, xf);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[r] = fmaf(wf[e], xf[e], sum[r]);
          }
        }
      }
#pragma unroll
      for (int r = 0; r < kPlainRows; ++r)
        if (m0 + r < M) acc[r] = X::kScaled ? fmaf(sum[r], x.block_scale(m0 + r, b) * ws, acc[r]) : acc[r] + sum[r];
    }
#pragma unroll
    for (int r = 0; r < kPlainRows; ++r) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) acc[r] += __shfl_xor_sync(0xffffffffu, acc[r], o);
      if (lane == 0 && m0 + r < M) y[(m0 + r) * y_stride + n] = from_float<T>(acc[r] + (bias ? bias[n] : 0.f));
    }
  }
}

template <typename T>
aiq_status_t product_plain(const MxProduct& p, cudaStream_t s) {
  const int64_t row_bytes = mx_row_bytes(p.K), scale_row = mx_scale_row_bytes(p.K);
  const dim3 grid((p.N + kMxThreads / 32 - 1) / (kMxThreads / 32), min((p.M + kPlainRows - 1) / kPlainRows, 65535));
  LaunchScope scope(AIQ_KERNEL_QLINEAR, s, 2.0 * p.M * p.N * p.K,
                    (double)(p.N + (p.x ? 0 : p.M)) * (row_bytes + scale_row) + sizeof(T) * (double)p.M * (p.N + (p.x ? p.K : 0)));
  if (p.x) {
    const bool vec = (((uintptr_t)p.x) & 15) == 0 && (p.M == 1 || p.x_stride * (int64_t)sizeof(T) % 16 == 0);
    const PlainX<T> x = {static_cast<const T*>(p.x), p.x_stride, vec};
    mx_product_plain_kernel<<<grid, kMxThreads, 0, s>>>(x, p.w_codes, p.w_scales, row_bytes, scale_row, p.bias, p.N, p.K, p.M,
                                                        static_cast<T*>(p.y), p.y_stride);
  } else {
    const PlainMx x = {p.x_codes, p.x_scales, row_bytes, scale_row};
    mx_product_plain_kernel<<<grid, kMxThreads, 0, s>>>(x, p.w_codes, p.w_scales, row_bytes, scale_row, p.bias, p.N, p.K, p.M,
                                                        static_cast<T*>(p.y), p.y_stride);
  }
  AIQ_LAUNCH_CHECK("mx_product_plain");
  return AIQ_OK;
}

}  // namespace

aiq_status_t launch_mx_quantize(const void* x, int dtype, int rows, int K, int64_t x_stride, uint8_t* codes, uint8_t* scales,
                                cudaStream_t s) {
  switch (dtype) {
    case AIQ_DTYPE_F32: return quantize_rows(static_cast<const float*>(x), rows, K, x_stride, codes, scales, s);
    case AIQ_DTYPE_F16: return quantize_rows(static_cast<const __half*>(x), rows, K, x_stride, codes, scales, s);
    default: return quantize_rows(static_cast<const __nv_bfloat16*>(x), rows, K, x_stride, codes, scales, s);
  }
}

aiq_status_t launch_mx_dequantize(const uint8_t* codes, const uint8_t* scales, int rows, int K, int dtype, void* y,
                                  int64_t y_stride, cudaStream_t s) {
  switch (dtype) {
    case AIQ_DTYPE_F32: return dequantize_rows(codes, scales, rows, K, static_cast<float*>(y), y_stride, s);
    case AIQ_DTYPE_F16: return dequantize_rows(codes, scales, rows, K, static_cast<__half*>(y), y_stride, s);
    default: return dequantize_rows(codes, scales, rows, K, static_cast<__nv_bfloat16*>(y), y_stride, s);
  }
}

aiq_status_t launch_mx_product_plain(const MxProduct& p, cudaStream_t s) {
  switch (p.dtype) {
    case AIQ_DTYPE_F32: return product_plain<float>(p, s);
    case AIQ_DTYPE_F16: return product_plain<__half>(p, s);
    default: return product_plain<__nv_bfloat16>(p, s);
  }
}

}  // namespace aiq

// ---------------------------------------------------------------------------------------
// C entry points
// ---------------------------------------------------------------------------------------
using aiq::set_error;

// AIQ_OK, or what is wrong with the sizes and pointers that every entry point takes
static aiq_status_t mx_check(const char* what, const void* codes, const void* scales, int rows, int K) {
  if (!codes || !scales) return set_error(AIQ_ERR_INVALID_ARG, "%s: null pointer", what);
  if (rows <= 0 || K <= 0) return set_error(AIQ_ERR_INVALID_ARG, "%s: %d rows of K=%d", what, rows, K);
  if (((uintptr_t)codes) & 31) return set_error(AIQ_ERR_INVALID_ARG, "%s: codes not 32-byte aligned", what);
  if (((uintptr_t)scales) & 15) return set_error(AIQ_ERR_INVALID_ARG, "%s: scales not 16-byte aligned", what);
  return AIQ_OK;
}
static aiq_status_t mx_check_bias(const char* what, const float* bias) {
  return ((uintptr_t)bias) & 3 ? set_error(AIQ_ERR_INVALID_ARG, "%s: bias not aligned to its type", what) : AIQ_OK;
}
static aiq_status_t mx_check_rows(const char* what, const void* p, int dtype, int64_t stride) {
  if (!aiq::mx_dtype_ok(dtype)) return set_error(AIQ_ERR_INVALID_ARG, "%s: dtype=%d", what, dtype);
  if (!p) return set_error(AIQ_ERR_INVALID_ARG, "%s: null pointer", what);
  if (((uintptr_t)p) % aiq::mx_dtype_bytes(dtype)) return set_error(AIQ_ERR_INVALID_ARG, "%s: rows not aligned to their type", what);
  if (stride < 0 || stride > (int64_t)1 << 40) return set_error(AIQ_ERR_INVALID_ARG, "%s: row stride %lld", what, (long long)stride);
  return AIQ_OK;
}
// rows that are written may not overlap
static aiq_status_t mx_check_out(const char* what, const void* p, int dtype, int rows, int K, int64_t stride) {
  if (aiq_status_t st = mx_check_rows(what, p, dtype, stride)) return st;
  if (rows > 1 && stride < K) return set_error(AIQ_ERR_INVALID_ARG, "%s: output row stride %lld < %d", what, (long long)stride, K);
  return AIQ_OK;
}

extern "C" size_t aiq_mx_row_bytes(int K) { return K > 0 ? (size_t)aiq::mx_row_bytes(K) : 0; }
extern "C" size_t aiq_mx_scale_row_bytes(int K) { return K > 0 ? (size_t)aiq::mx_scale_row_bytes(K) : 0; }

extern "C" aiq_status_t aiq_mx_quantize(const void* x, int dtype, int rows, int K, int64_t x_stride, void* codes_out,
                                        void* scales_out, void* stream) {
  if (aiq_status_t st = mx_check("aiq_mx_quantize", codes_out, scales_out, rows, K)) return st;
  if (aiq_status_t st = mx_check_rows("aiq_mx_quantize", x, dtype, x_stride)) return st;
  if (aiq_status_t st = aiq::check_device_sm100()) return st;
  return aiq::launch_mx_quantize(x, dtype, rows, K, x_stride, static_cast<uint8_t*>(codes_out), static_cast<uint8_t*>(scales_out),
                                 (cudaStream_t)stream);
}

extern "C" aiq_status_t aiq_mx_dequantize(const void* codes, const void* scales, int rows, int K, int dtype, void* y, int64_t y_stride,
                                          void* stream) {
  if (aiq_status_t st = mx_check("aiq_mx_dequantize", codes, scales, rows, K)) return st;
  if (aiq_status_t st = mx_check_out("aiq_mx_dequantize", y, dtype, rows, K, y_stride)) return st;
  if (aiq_status_t st = aiq::check_device_sm100()) return st;
  return aiq::launch_mx_dequantize(static_cast<const uint8_t*>(codes), static_cast<const uint8_t*>(scales), rows, K, dtype, y, y_stride,
                                   (cudaStream_t)stream);
}

extern "C" size_t aiq_mx_linear_workspace_bytes(int N, int K, int M, int dtype) {
  if (N <= 0 || K <= 0 || M <= 0 || !aiq::mx_dtype_ok(dtype)) return 0;
  return aiq::mx_tc_workspace_bytes(K, M, dtype);
}

extern "C" aiq_status_t aiq_mx_linear(const void* codes, const void* scales, const float* bias, int N, int K, const void* x, int dtype,
                                      int M, int64_t x_stride, void* y, int64_t y_stride, void* workspace, size_t workspace_bytes,
                                      void* stream) {
  if (aiq_status_t st = mx_check("aiq_mx_linear", codes, scales, N, K)) return st;
  if (M <= 0) return set_error(AIQ_ERR_INVALID_ARG, "aiq_mx_linear: M=%d", M);
  if (aiq_status_t st = mx_check_rows("aiq_mx_linear", x, dtype, x_stride)) return st;
  if (aiq_status_t st = mx_check_out("aiq_mx_linear", y, dtype, M, N, y_stride)) return st;
  if (aiq_status_t st = mx_check_bias("aiq_mx_linear", bias)) return st;
  if (aiq_status_t st = aiq::check_device_sm100()) return st;
  aiq::MxProduct p = {};
  p.w_codes = static_cast<const uint8_t*>(codes);
  p.w_scales = static_cast<const uint8_t*>(scales);
  p.bias = bias;
  p.x = x; p.x_stride = x_stride;
  p.y = y; p.y_stride = y_stride;
  p.N = N; p.K = K; p.M = M; p.dtype = dtype;
  if (workspace) {
    if (((uintptr_t)workspace) & 15) return set_error(AIQ_ERR_INVALID_ARG, "aiq_mx_linear: workspace not 16-byte aligned");
    if (workspace_bytes < aiq::mx_tc_workspace_bytes(K, M, dtype))
      return set_error(AIQ_ERR_WORKSPACE_TOO_SMALL, "aiq_mx_linear: workspace of %zu bytes, %zu needed", workspace_bytes,
                       aiq::mx_tc_workspace_bytes(K, M, dtype));
    return aiq::launch_mx_product_tc(p, workspace, (cudaStream_t)stream);
  }
  return aiq::launch_mx_product_plain(p, (cudaStream_t)stream);
}

extern "C" aiq_status_t aiq_mx_matmul(const void* a_codes, const void* a_scales, int M, const void* b_codes, const void* b_scales, int N,
                                      const float* bias, int K, void* y, int dtype, int64_t y_stride, void* stream) {
  if (aiq_status_t st = mx_check("aiq_mx_matmul", a_codes, a_scales, M, K)) return st;
  if (aiq_status_t st = mx_check("aiq_mx_matmul", b_codes, b_scales, N, K)) return st;
  if (aiq_status_t st = mx_check_out("aiq_mx_matmul", y, dtype, M, N, y_stride)) return st;
  if (aiq_status_t st = mx_check_bias("aiq_mx_matmul", bias)) return st;
  if (aiq_status_t st = aiq::check_device_sm100()) return st;
  aiq::MxProduct p = {};
  p.w_codes = static_cast<const uint8_t*>(b_codes);
  p.w_scales = static_cast<const uint8_t*>(b_scales);
  p.bias = bias;
  p.x_codes = static_cast<const uint8_t*>(a_codes);
  p.x_scales = static_cast<const uint8_t*>(a_scales);
  p.y = y; p.y_stride = y_stride;
  p.N = N; p.K = K; p.M = M; p.dtype = dtype;
  return aiq::launch_mx_product_tc(p, nullptr, (cudaStream_t)stream);
}
