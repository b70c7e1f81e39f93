// Microscaled 4-bit floating point: the stored format, shared by its kernels (internal; the public ABI is include/aiq.h).
//
// A row of K values is cut into blocks of 32.  A block is 32 four-bit codes (sign, two exponent bits, one mantissa bit: 0,
// 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) and one byte s, which scales them by 2^(s - 127); s = 255 makes the block NaN.
// Rows of codes are padded to 128 values (64 bytes: the unit in which a TMA copy expands 4-bit values to bytes), rows of
// scale bytes to 16 (one 16-byte TMA box holds the scales of 512 values); all padding is zero.
#pragma once

#include "common.cuh"

namespace aiq {

enum { MX_BLOCK = 32 };
inline bool mx_dtype_ok(int dtype) { return dtype == AIQ_DTYPE_F32 || dtype == AIQ_DTYPE_F16 || dtype == AIQ_DTYPE_BF16; }
inline size_t mx_dtype_bytes(int dtype) { return dtype == AIQ_DTYPE_F32 ? 4 : 2; }
inline int64_t mx_row_bytes(int K) { return ((int64_t)K + 127) / 128 * 64; }
inline int64_t mx_scale_row_bytes(int K) { return ((int64_t)K + 511) / 512 * 16; }

// One product: y[m][n] = sum_k x[m][k] W[n][k] + bias[n]
struct MxProduct {
  const uint8_t* w_codes;
  const uint8_t* w_scales;
  const float* bias;          // [N] or nullptr
  const void* x;              // [M] rows of `x_stride` elements of `dtype`, or nullptr:
  const uint8_t* x_codes;     //   x microscaled too
  const uint8_t* x_scales;
  void* y;                    // [M] rows of `y_stride` elements of `dtype`
  int64_t x_stride, y_stride;
  int N, K, M, dtype;
};

// ---- launchers ------------------------------------------------------------------------
aiq_status_t launch_mx_quantize(const void* x, int dtype, int rows, int K, int64_t x_stride, uint8_t* codes, uint8_t* scales,
                                cudaStream_t s);
aiq_status_t launch_mx_dequantize(const uint8_t* codes, const uint8_t* scales, int rows, int K, int dtype, void* y,
                                  int64_t y_stride, cudaStream_t s);
// any shape, no workspace: a few rows of x, small matrices
aiq_status_t launch_mx_product_rows(const MxProduct& p, cudaStream_t s);
// tensor cores (mx_tc.cu); with x not microscaled: needs the workspace, for x as eight-bit pieces
size_t mx_tc_workspace_bytes(int K, int M, int dtype);
aiq_status_t launch_mx_product_tc(const MxProduct& p, void* workspace, cudaStream_t s);
void mx_tc_expire_next(int64_t limit_cycles);      // see aiq_debug_mx_expire_wait

// ---- device helpers -------------------------------------------------------------------
// 2^(s - 127) as a float; NaN for 255
__device__ __forceinline__ float mx_scale(uint32_t s) {
  return __uint_as_float(s == 0 ? 0x00400000u : s == 255 ? 0x7FC00000u : s << 23);
}
// the scale byte of a block whose largest |x| has the float32 bits `top`, and the exact 2^(127 - s): floor(log2(top)) - 2, so
// that the largest value lies in [4, 8) of the codes' range and above 6 saturates.  NaN and infinity give 255.
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t top) {
  const uint32_t e = top >> 23;
  return e == 255 ? 255u : e < 2 ? 0u : e - 2;
}
__device__ __forceinline__ float mx_inverse_scale(uint32_t s) { return __uint_as_float((254u - s) << 23); }

// the eight codes of a word as floats (conversions to halves are exact)
__device__ __forceinline__ void mx_expand8(uint32_t w, float* f) {
  uint32_t h[4];
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "mov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\tcvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
    f[2 * i] = v.x;
    f[2 * i + 1] = v.y;
  }
}
// eight scaled values to codes, round to nearest even, saturating; the first in the lowest nibble
__device__ __forceinline__ uint32_t mx_codes8(const float* f) {
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r) : "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]), "f"(f[5]), "f"(f[6]), "f"(f[7]));
  return r;
}

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// eight consecutive values from a 16-byte aligned address (float: two loads)
template <typename T>
__device__ __forceinline__ void load8(const T* p, float* f) {
  if (sizeof(T) == 4) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  } else {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const T* h = reinterpret_cast<const T*>(&w[i]);
      f[2 * i] = to_float(h[0]);
      f[2 * i + 1] = to_float(h[1]);
    }
  }
}

// n / d for 0 <= n < 2^31 by a multiplication (Granlund and Montgomery, "Division by invariant integers using multiplication", 1994): q = (floor(n m / 2^32) + n) >> l with l = ceil(log2 d), m = floor(2^32 (2^l - d) / d) + 1
struct FastDiv {
  uint32_t d, m, l;
  explicit FastDiv(uint32_t divisor) : d(divisor), l(0) {
    while ((1ull << l) < d) ++l;
    m = (uint32_t)(((1ull << 32) * ((1ull << l) - d)) / d + 1);
  }
  __device__ __forceinline__ uint32_t div(uint32_t n) const { return (__umulhi(n, m) + n) >> l; }
};

}  // namespace aiq
