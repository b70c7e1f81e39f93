// Microscaled 4-bit floating point: quantizing, expanding, and the product for any shape; see mx.cuh for the format.
#include "mx.cuh"
#include "tc_ptx.cuh"

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
// the product, any shape; the kernel for a few rows of x and for small matrices
// ---------------------------------------------------------------------------------------
// A warp computes R output channels for MT rows of x, or a share of their k.  A lane takes a word of eight codes at a time, so that
// the loads of a warp are whole lines: 128 bytes of codes, and the 256 values of x that belong to them.  All loads of U words are
// under way before the first is used.  float32 throughout, two products per instruction.
constexpr int kRowChannels = 2;

// eight values of x from k on (k a multiple of 8), as they are loaded and as floats; zero behind K
template <typename T>
struct RowsOf {
  struct Raw { uint4 v[sizeof(T) / 2]; };
  const T* x;
  int64_t stride;
  bool vec;
  __device__ __forceinline__ Raw get(int64_t m, int k, int K) const {
    const T* p = x + m * stride + k;
    Raw r;
    if (vec && k + 8 <= K) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.v[i] = reinterpret_cast<const uint4*>(p)[i];
    } else {
      T v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = k + j < K ? p[j] : from_float<T>(0.f);
      memcpy(&r, v, sizeof(r));
    }
    return r;
  }
  static __device__ __forceinline__ Raw none() { return Raw{}; }
  static __device__ __forceinline__ void values(const Raw& r, float* f) {
    T v[8];
    memcpy(v, &r, sizeof(r));
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = to_float(v[j]);
  }
};
struct RowsHeld {
  struct Raw { uint32_t codes, scale; };
  const uint8_t *codes, *scales;
  int64_t row_bytes, scale_row;
  __device__ __forceinline__ Raw get(int64_t m, int k, int) const {
    return Raw{*reinterpret_cast<const uint32_t*>(codes + m * row_bytes + (k >> 1)), scales[m * scale_row + (k >> 5)]};
  }
  static __device__ __forceinline__ Raw none() { return Raw{0u, 0u}; }
  static __device__ __forceinline__ void values(const Raw& r, float* f) {
    mx_expand8(r.codes, f);
    const float s = mx_scale(r.scale);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] *= s;
  }
};

template <typename X, typename T, int MT, int U>
__global__ void __launch_bounds__(kMxThreads)
mx_product_rows_kernel(X x, const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t row_bytes, int64_t scale_row,
                       const float* __restrict__ bias, int N, int K, int M, int k_warps, T* __restrict__ y, int64_t y_stride) {
  constexpr int R = kRowChannels, WARPS = kMxThreads / 32;
  __shared__ float part[WARPS][R * MT];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, kw = warp % k_warps;
  const int n0 = (blockIdx.x * (WARPS / k_warps) + warp / k_warps) * R;
  const int words = (K + 7) / 8;
  for (int64_t m0 = (int64_t)blockIdx.y * MT; m0 < M; m0 += (int64_t)gridDim.y * MT) {
    uint64_t acc[R][MT];
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int r = 0; r < MT; ++r) acc[i][r] = 0;
    for (int w0 = kw * 32 * U + lane; w0 - lane < words && n0 < N; w0 += k_warps * 32 * U) {
      uint32_t raw[R][U], sb[R][U];
      typename X::Raw xr[MT][U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int w = w0 + u * 32;
#pragma unroll
        for (int i = 0; i < R; ++i) {
          const bool live = w < words && n0 + i < N;
          raw[i][u] = live ? *reinterpret_cast<const uint32_t*>(codes + (n0 + i) * row_bytes + (int64_t)w * 4) : 0u;
          sb[i][u] = live ? scales[(n0 + i) * scale_row + (w >> 2)] : 0u;
        }
#pragma unroll
        for (int r = 0; r < MT; ++r) {
          if (w < words && m0 + r < M) xr[r][u] = x.get(m0 + r, w * 8, K);
          else xr[r][u] = X::none();
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        uint64_t wf[R][4];
#pragma unroll
        for (int i = 0; i < R; ++i) {
          float f[8];
          mx_expand8(raw[i][u], f);
          const float s = mx_scale(sb[i][u]);
#pragma unroll
          for (int j = 0; j < 4; ++j) wf[i][j] = mul2(pack2(f[2 * j], f[2 * j + 1]), pack2(s, s));
        }
#pragma unroll
        for (int r = 0; r < MT; ++r) {
          float f[8];
          X::values(xr[r][u], f);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint64_t v = pack2(f[2 * j], f[2 * j + 1]);
#pragma unroll
            for (int i = 0; i < R; ++i) acc[i][r] = fma2(wf[i][j], v, acc[i][r]);
          }
        }
      }
    }
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int r = 0; r < MT; ++r) {
        const float2 a = unpack2(acc[i][r]);
        float v = a.x + a.y;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        if (lane == 0) part[warp][i * MT + r] = v;
      }
    if (k_warps > 1) __syncthreads(); else __syncwarp();
    if (kw == 0 && lane < R * MT) {
      const int i = lane / MT, r = lane % MT;
      float v = 0.f;
      for (int k = 0; k < k_warps; ++k) v += part[warp + k][lane];
      if (n0 + i < N && m0 + r < M) y[(m0 + r) * y_stride + n0 + i] = from_float<T>(v + (bias ? bias[n0 + i] : 0.f));
    }
    if (k_warps > 1) __syncthreads(); else __syncwarp();
  }
}

template <int MT, int U, typename X, typename T>
aiq_status_t product_rows(const MxProduct& p, X x, cudaStream_t s) {
  const int64_t row_bytes = mx_row_bytes(p.K), scale_row = mx_scale_row_bytes(p.K);
  // Warps along k until a warp's share is one round of loads, as long as that gives blocks to SMs without: one row, 4096 x 4096, 12.0 us
  // with 148 blocks at most, 9.9 with 296, 9.2 with 592 and more; 8192 x 8192 31.1, 31.1, 28.0, without a limit 30.7.
  int k_warps = 1;
  const int64_t m_blocks = (p.M + MT - 1) / MT;
  while (k_warps < kMxThreads / 32 && k_warps * 256 * U < p.K && (int64_t)p.N * k_warps / (kMxThreads / 32 * kRowChannels) * m_blocks < 592)
    k_warps *= 2;
  const int per_block = kMxThreads / 32 / k_warps * kRowChannels;
  const dim3 grid((p.N + per_block - 1) / per_block, min((p.M + MT - 1) / MT, 65535));
  mx_product_rows_kernel<X, T, MT, U><<<grid, kMxThreads, 0, s>>>(x, p.w_codes, p.w_scales, row_bytes, scale_row, p.bias, p.N, p.K, p.M,
                                                                 k_warps, static_cast<T*>(p.y), p.y_stride);
  AIQ_LAUNCH_CHECK("mx_product_rows");
  return AIQ_OK;
}
template <typename X, typename T>
aiq_status_t product_rows(const MxProduct& p, X x, cudaStream_t s) {
  LaunchScope scope(AIQ_KERNEL_QLINEAR, s, 2.0 * p.M * p.N * p.K,
                    (double)(p.N + (p.x ? 0 : p.M)) * (mx_row_bytes(p.K) + mx_scale_row_bytes(p.K)) + sizeof(T) * (double)p.M * (p.N + (p.x ? p.K : 0)));
  if (p.M == 1) return product_rows<1, 4, X, T>(p, x, s);
  if (p.M == 2) return product_rows<2, 2, X, T>(p, x, s);
  return product_rows<4, 2, X, T>(p, x, s);
}

template <typename T>
aiq_status_t product_rows(const MxProduct& p, cudaStream_t s) {
  if (p.x) {
    const bool vec = (((uintptr_t)p.x) & 15) == 0 && (p.M == 1 || p.x_stride * (int64_t)sizeof(T) % 16 == 0);
    return product_rows<RowsOf<T>, T>(p, RowsOf<T>{static_cast<const T*>(p.x), p.x_stride, vec}, s);
  }
  return product_rows<RowsHeld, T>(p, RowsHeld{p.x_codes, p.x_scales, mx_row_bytes(p.K), mx_scale_row_bytes(p.K)}, s);
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

aiq_status_t launch_mx_product_rows(const MxProduct& p, cudaStream_t s) {
  switch (p.dtype) {
    case AIQ_DTYPE_F32: return product_rows<float>(p, s);
    case AIQ_DTYPE_F16: return product_rows<__half>(p, s);
    default: return product_rows<__nv_bfloat16>(p, s);
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

// Whether the kernel for few rows and small matrices beats the tensor-core kernel, whose time below 2^22 products is its chain of
// set-up, first loads and last stores.  On the device, rows | tensor cores (linear layer: with its pre-pass, a second launch):
//   linear, bf16     1 row: 1280 x 320 2.6 | 7.0 us, 2000 x 2000 4.7 | 8.2, 4096 x 4096 9.2 | 9.7, 8192 x 8192 28 | 15.5
//                    4 rows: 724 x 724 4.9 | 7.5, 2000 x 2000 8.4 | 8.2;  8 rows, 724 x 724 5.6 | 7.4;  16 rows 9.4 | 7.6
//   both microscaled 1 row: 2000 x 2000 4.8 | 6.3, 4096 x 4096 10.0 | 7.6;  8 rows, 300 x 300 3.2 | 4.9;  4 rows, 2000 x 2000 8.0 | 6.4
static bool mx_rows_pay(int N, int K, int M, int log2_most) { return (double)N * K * M <= (double)(1ll << log2_most); }

extern "C" size_t aiq_mx_linear_workspace_bytes(int N, int K, int M, int dtype) {
  if (N <= 0 || K <= 0 || M <= 0 || !aiq::mx_dtype_ok(dtype)) return 0;
  return mx_rows_pay(N, K, M, M <= 4 ? 24 : 22) ? 0 : aiq::mx_tc_workspace_bytes(K, M, dtype);
}

extern "C" aiq_status_t aiq_mx_linear(const void* codes, const void* scales, const float* bias, int N, int K, const void* x, int dtype,
                                      int M, int64_t x_stride, void* y, int64_t y_stride, void* workspace, size_t workspace_bytes,
                                      void* stream) {
  if (aiq_status_t st = mx_check("aiq_mx_linear", codes, scales, N, K)) return st;
  if (M <= 0) return set_error(AIQ_ERR_INVALID_ARG, "aiq_mx_linear: M=%d", M);
  if (aiq_status_t st = mx_check_rows("aiq_mx_linear", x, dtype, x_stride)) return st;
  if (aiq_status_t st = mx_check_out("aiq_mx_linear", y, dtype, M, N, y_stride)) return st;
  if (aiq_status_t st = mx_check_bias("aiq_mx_linear", bias)) return st;
  aiq::MxProduct p = {};
  p.w_codes = static_cast<const uint8_t*>(codes);
  p.w_scales = static_cast<const uint8_t*>(scales);
  p.bias = bias;
  p.x = x; p.x_stride = x_stride;
  p.y = y; p.y_stride = y_stride;
  p.N = N; p.K = K; p.M = M; p.dtype = dtype;
  if (((uintptr_t)workspace) & 15) return set_error(AIQ_ERR_INVALID_ARG, "aiq_mx_linear: workspace not 16-byte aligned");
  const size_t needed = aiq_mx_linear_workspace_bytes(N, K, M, dtype);
  if (workspace && workspace_bytes < needed)
    return set_error(AIQ_ERR_WORKSPACE_TOO_SMALL, "aiq_mx_linear: workspace of %zu bytes, %zu needed", workspace_bytes, needed);
  if (aiq_status_t st = aiq::check_device_sm100()) return st;
  if (needed == 0 || !workspace) return aiq::launch_mx_product_rows(p, (cudaStream_t)stream);
  return aiq::launch_mx_product_tc(p, workspace, (cudaStream_t)stream);
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
  if (mx_rows_pay(N, K, M, M == 1 ? 23 : 22)) return aiq::launch_mx_product_rows(p, (cudaStream_t)stream);
  return aiq::launch_mx_product_tc(p, nullptr, (cudaStream_t)stream);
}
