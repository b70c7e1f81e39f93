// Microscaled 4-bit floating point: quantizing, expanding, and the product for any shape; see mx.cuh for the format.
#include "mx.cuh"
#include "tc_ptx.cuh"

namespace aiq {
namespace {

// ---------------------------------------------------------------------------------------
// quantize
// ---------------------------------------------------------------------------------------
constexpr int kMxThreads = 256;
constexpr int kMxWarps = kMxThreads / 32;

// Eight values of a row as they lie in memory, and the largest |value| among them as float32 bits (0x7F800000 and above: not finite).
template <typename T>
struct Eight {
  uint4 raw[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) raw[i] = reinterpret_cast<const uint4*>(p)[i];
  }
  __device__ __forceinline__ void load_part(const T* p, int n) {       // zero from element n on
    T v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < n ? p[j] : from_float<T>(0.f);
    memcpy(raw, v, sizeof(raw));
  }
  // from `off` elements (less than 16 bytes) behind a 16-byte boundary: the aligned pieces around them, moved into place
  __device__ __forceinline__ void load_shifted(const T* p, int off) {
    constexpr int N = sizeof(T) == 4 ? 12 : 8;                 // words
    uint32_t w[N];
    const uint4* from = reinterpret_cast<const uint4*>(p - off);
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const uint4 c = from[i];
      w[4 * i] = c.x; w[4 * i + 1] = c.y; w[4 * i + 2] = c.z; w[4 * i + 3] = c.w;
    }
    const int words = sizeof(T) == 4 ? off : off >> 1, need = sizeof(T) == 4 ? 8 : 5;
    if (words & 2) {
#pragma unroll
      for (int i = 0; i < need + 1 && i + 2 < N; ++i) w[i] = w[i + 2];
    }
    if (words & 1) {
#pragma unroll
      for (int i = 0; i < need && i + 1 < N; ++i) w[i] = w[i + 1];
    }
    uint32_t* out = reinterpret_cast<uint32_t*>(raw);
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) * 2; ++i) out[i] = sizeof(T) == 4 ? w[i] : __funnelshift_r(w[i], w[i + 1], 16 * (off & 1));
  }
  __device__ __forceinline__ void values(float* f) const {
    T v[8];
    memcpy(v, raw, sizeof(raw));
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = to_float(v[j]);
  }
};
__device__ __forceinline__ uint32_t top_bits(const Eight<float>& e) {
  const uint32_t* w = reinterpret_cast<const uint32_t*>(e.raw);
  uint32_t t = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) t = max(t, w[j] & 0x7FFFFFFFu);
  return t;
}
// 16-bit types: the bits of |value| order like the values, two at a time
__device__ __forceinline__ uint32_t top_half(const uint4& r) {
  const uint32_t m = __vmaxu2(__vmaxu2(r.x & 0x7FFF7FFFu, r.y & 0x7FFF7FFFu), __vmaxu2(r.z & 0x7FFF7FFFu, r.w & 0x7FFF7FFFu));
  return max(m >> 16, m & 0xFFFFu);
}
__device__ __forceinline__ uint32_t top_bits(const Eight<__nv_bfloat16>& e) { return top_half(e.raw[0]) << 16; }
__device__ __forceinline__ uint32_t top_bits(const Eight<__half>& e) {
  return __float_as_uint(__half2float(__ushort_as_half((unsigned short)top_half(e.raw[0]))));
}

// A warp takes 256 U values of one row; a lane eight at a time (one word of codes), four lanes a block.  Where a value lies is decided
// once per warp, and the U loads of a lane are on their way together.  SHIFT: rows that do not start on 16 bytes.
// Bound by memory: 8192 x 8192, bfloat16, 27 us (170 MB, 95 % of the copy rate); 47 us with a division and bounds for every word
// (103 instructions a word).  Rows that start elsewhere: 42 us; 69 us with a value per lane and a transposition of the codes.
template <typename T, int U, bool SHIFT>
__global__ void __launch_bounds__(kMxThreads)
mx_quantize_kernel(const T* __restrict__ x, int64_t x_stride, int K, uint32_t segments, FastDiv per_row, int words, int scale_row,
                   uint32_t* __restrict__ codes, uint8_t* __restrict__ scales) {
  const uint32_t seg = blockIdx.x * kMxWarps + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (seg >= segments) return;
  const uint32_t row = per_row.div(seg);
  const int word0 = (int)(seg - row * per_row.d) * (32 * U) + lane;
  const T* src = x + (int64_t)row * x_stride + word0 * 8;
  const int off = SHIFT ? (int)((reinterpret_cast<uintptr_t>(src) & 15) / sizeof(T)) : 0;       // the same for all of the row
  uint32_t* out = codes + (int64_t)row * words + word0;
  uint8_t* sr = scales + (int64_t)row * scale_row;
  Eight<T> e[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int left = K - (word0 + 32 * i) * 8;
    if (SHIFT && off) {                                        // the pieces around the values have to lie in the row
      if (word0 + i > 0 && left >= 16) e[i].load_shifted(src + 256 * i, off);
      else e[i].load_part(src + 256 * i, left);
    } else if (left >= 8) {
      e[i].load(src + 256 * i);
    } else {
      e[i].load_part(src + 256 * i, left);
    }
  }
#pragma unroll
  for (int i = 0; i < U; ++i) {
    uint32_t top = top_bits(e[i]);
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const uint32_t s = mx_scale_byte(top);
    const float inv = mx_inverse_scale(s);
    float f[8];
    e[i].values(f);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] *= inv;
    const int word = word0 + 32 * i;
    if (word < words) out[32 * i] = s == 255 ? 0u : mx_codes8(f);
    if ((lane & 3) == 0 && (word >> 2) < scale_row) sr[word >> 2] = (uint8_t)s;          // blocks behind K: zero
  }
  // the row's last segment: scale bytes behind its own blocks
  const int end = (word0 - lane + 32 * U) >> 2;
  if ((word0 - lane) + 32 * U >= words && end + lane < scale_row) sr[end + lane] = 0;
}

template <typename T, int U>
aiq_status_t quantize_rows(const T* x, int64_t rows, int K, int64_t x_stride, uint8_t* codes, uint8_t* scales, bool aligned, cudaStream_t s) {
  const int64_t row_bytes = mx_row_bytes(K), scale_row = mx_scale_row_bytes(K), words = row_bytes / 4;
  const uint32_t per_row = (uint32_t)((words + 32 * U - 1) / (32 * U));
  const int64_t step = max((int64_t)1, (int64_t)((1u << 30) / per_row));       // rows per launch: segments below 2^31
  for (int64_t r = 0; r < rows; r += step) {
    const int64_t n = min(step, rows - r), segments = n * per_row;
    const T* xr = x + r * x_stride;
    uint32_t* c = reinterpret_cast<uint32_t*>(codes + r * row_bytes);
    uint8_t* sc = scales + r * scale_row;
    LaunchScope scope(AIQ_KERNEL_QUANTIZE, s, 2.0 * n * K, (double)n * (sizeof(T) * (double)K + row_bytes + scale_row));
    const unsigned grid = (unsigned)((segments + kMxWarps - 1) / kMxWarps);
    const auto kernel = aligned ? mx_quantize_kernel<T, U, false> : mx_quantize_kernel<T, U, true>;
    kernel<<<grid, kMxThreads, 0, s>>>(xr, x_stride, K, (uint32_t)segments, FastDiv(per_row), (int)words, (int)scale_row, c, sc);
    AIQ_LAUNCH_CHECK("mx_quantize");
  }
  return AIQ_OK;
}
// Words of eight values per lane (U): more loads on their way in a large matrix, more warps in a small one.  On the device, U = 1 | 2 | 4:
//   bfloat16, rows on 16 bytes  8192 x 8192 38.5 | 31.7 | 27.4 us, 8192 x 600 5.7 | 5.7 | 5.0;  others  8192 x 8191 45.4 | 41.8 | 43.3,
//     4099 x 1283 6.3 | 6.7 | 9.4;   float32  8192 x 8192 45.6 | 44.8 | 45.1, 2000 x 2000 4.9 | 5.1 | 5.7, 8192 x 8191 50 | 55 | 63,
//     724 x 724 2.4 | 2.5 | 2.7
template <typename T>
aiq_status_t quantize_rows(const T* x, int64_t rows, int K, int64_t x_stride, uint8_t* codes, uint8_t* scales, cudaStream_t s) {
  const bool aligned = (((uintptr_t)x) & 15) == 0 && (rows == 1 || x_stride * (int64_t)sizeof(T) % 16 == 0);
  const double n = (double)rows * K;
  const int most = K <= 256 ? 1 : K <= 512 ? 2 : 4;            // what a row fills
  const int u = sizeof(T) == 4 ? (!aligned || n <= 8e6 ? 1 : 2) : aligned ? (n <= 1e6 ? 1 : 4) : n <= 16e6 ? 1 : 2;
  if (u == 1 || most == 1) return quantize_rows<T, 1>(x, rows, K, x_stride, codes, scales, aligned, s);
  if (u == 2 || most == 2) return quantize_rows<T, 2>(x, rows, K, x_stride, codes, scales, aligned, s);
  return quantize_rows<T, 4>(x, rows, K, x_stride, codes, scales, aligned, s);
}

// ---------------------------------------------------------------------------------------
// dequantize
// ---------------------------------------------------------------------------------------
template <typename T>
__device__ __forceinline__ void store8(T* p, const float* f) {         // 32 bytes at a time for floats, 16 else, aligned to that
  uint32_t w[8];
  if (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(f[i]);
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]),
                 "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      T h[2] = {from_float<T>(f[2 * i]), from_float<T>(f[2 * i + 1])};
      w[i] = *reinterpret_cast<const uint32_t*>(h);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// A warp takes 256 U values of one row, a lane eight at a time.  With SHIFT a row of y may start anywhere: with `off` elements between a store
// boundary and the row's start, piece w of the row is its values 8 w - off to 8 w - off + 7, whose codes are a funnel shift of
// words w - 1 and w; the first `off` of them belong to word w - 1 and its scale.
// Bound by memory: 8192 x 8192 28 us to bfloat16 (170 MB, 91 % of the copy rate), 48 us to float32 (71 us in 16-byte stores 32 bytes
// apart); 8192 x 8191 36 us to bfloat16 (51 us by a value per lane).
template <typename T, int U, bool SHIFT>
__global__ void __launch_bounds__(kMxThreads)
mx_dequantize_kernel(const uint32_t* __restrict__ codes, const uint8_t* __restrict__ scales, int words, int scale_row, int K, uint32_t segments,
                     FastDiv per_row, T* __restrict__ y, int64_t y_stride) {
  constexpr int WIDTH = sizeof(T) == 4 ? 32 : 16;              // bytes of a store
  const uint32_t seg = blockIdx.x * kMxWarps + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (seg >= segments) return;
  const uint32_t row = per_row.div(seg);
  const int word0 = (int)(seg - row * per_row.d) * (32 * U) + lane;
  T* start = y + (int64_t)row * y_stride;
  const int off = SHIFT ? (int)((reinterpret_cast<uintptr_t>(start) & (WIDTH - 1)) / sizeof(T)) : 0;
  const uint32_t* cr = codes + (int64_t)row * words;
  const uint8_t* sr = scales + (int64_t)row * scale_row;
  uint32_t raw[U], before[U], sb[U], sb_before[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int w = word0 + 32 * i;
    raw[i] = w < words ? cr[w] : 0u;
    sb[i] = w < words ? sr[w >> 2] : 0u;
    before[i] = off && w > 0 && w <= words ? cr[w - 1] : 0u;
    sb_before[i] = off && w > 0 && w <= words ? sr[(w - 1) >> 2] : 0u;
  }
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int k = (word0 + 32 * i) * 8 - off;                  // first value
    if (k >= K) break;
    float f[8];
    mx_expand8(off ? __funnelshift_l(before[i], raw[i], 4 * off) : raw[i], f);
    const float s = mx_scale(sb[i]);
    if (off) {
      const float s0 = mx_scale(sb_before[i]);
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] *= j < off ? s0 : s;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] *= s;
    }
    T* dst = start + k;
    if (k >= 0 && k + 8 <= K) {
      store8(dst, f);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (k + j >= 0 && k + j < K) dst[j] = from_float<T>(f[j]);
    }
  }
}

template <typename T, int U>
aiq_status_t dequantize_rows(const uint8_t* codes, const uint8_t* scales, int64_t rows, int K, T* y, int64_t y_stride, cudaStream_t s) {
  const int64_t row_bytes = mx_row_bytes(K), scale_row = mx_scale_row_bytes(K), words = row_bytes / 4;
  constexpr int WIDTH = sizeof(T) == 4 ? 32 : 16;
  const bool aligned = (((uintptr_t)y) & (WIDTH - 1)) == 0 && (rows == 1 || y_stride * (int64_t)sizeof(T) % WIDTH == 0);
  const int64_t pieces = ((int64_t)K + 7) / 8 + (aligned ? 0 : 1);       // one more in a row that does not start on a store boundary
  const uint32_t per_row = (uint32_t)((pieces + 32 * U - 1) / (32 * U));
  const int64_t step = max((int64_t)1, (int64_t)((1u << 30) / per_row));
  for (int64_t r = 0; r < rows; r += step) {
    const int64_t n = min(step, rows - r), segments = n * per_row;
    LaunchScope scope(AIQ_KERNEL_QUANTIZE, s, (double)n * K, (double)n * (sizeof(T) * (double)K + row_bytes + scale_row));
    const auto kernel = aligned ? mx_dequantize_kernel<T, U, false> : mx_dequantize_kernel<T, U, true>;
    kernel<<<(unsigned)((segments + kMxWarps - 1) / kMxWarps), kMxThreads, 0, s>>>(
        reinterpret_cast<const uint32_t*>(codes + r * row_bytes), scales + r * scale_row, (int)words, (int)scale_row, K, (uint32_t)segments,
        FastDiv(per_row), y + r * y_stride, y_stride);
    AIQ_LAUNCH_CHECK("mx_dequantize");
  }
  return AIQ_OK;
}
// As above.  U = 1 | 2 | 4: 8192 x 8192, bfloat16 37.8 | 28.9 | 28.4 us, float32 52.4 | 48.2 | 48.8; 2000 x 2000, float32 5.1 | 4.5 | 4.8;
// rows off a store boundary: 8192 x 8191, bfloat16 46.0 | 37.1 | 36.0; 4099 x 1283, half 6.2 | 5.7 | 6.2; 1000 x 1281, float32 3.0 | 3.1 | 3.3
template <typename T>
aiq_status_t dequantize_rows(const uint8_t* codes, const uint8_t* scales, int64_t rows, int K, T* y, int64_t y_stride, cudaStream_t s) {
  const double n = (double)rows * K;
  if (K <= 248 || n <= 2e6) return dequantize_rows<T, 1>(codes, scales, rows, K, y, y_stride, s);
  if (K <= 504 || n <= 6e6) return dequantize_rows<T, 2>(codes, scales, rows, K, y, y_stride, s);
  return dequantize_rows<T, 4>(codes, scales, rows, K, y, y_stride, s);
}

// ---------------------------------------------------------------------------------------
// the product, any shape; the kernel for a few rows of x and for small matrices
// ---------------------------------------------------------------------------------------
// A warp computes R output channels for MT rows of x, or a share of their k.  A lane takes a word of eight codes at a time, so that
// the loads of a warp are whole lines: 128 bytes of codes, and the 256 values of x that belong to them.  All loads of U words are
// under way before the first is used.  float32 throughout, two products per instruction.
// An element times its scale reaches 6 * 2^127, which no float32 holds.  So a quarter of it is multiplied, exact at both ends (from
// 1.5 * 2^127 to 2^-130), and the sum is scaled back at the end: a sum that overflows would do so without it, too.  Below 2^-124 (2^-122 with two
// microscaled matrices) a sum has fewer than 24 bits.
constexpr int kRowChannels = 2;
__device__ __forceinline__ float mx_quarter_scale(uint32_t s) {        // 2^(s - 129); NaN for 255
  return __uint_as_float(s < 3 ? 0x00100000u << s : s == 255 ? 0x7FC00000u : (s - 2) << 23);
}

// eight values of x from k on (k a multiple of 8), as they are loaded and as floats; zero behind K
template <typename T>
struct RowsOf {
  static constexpr float UNIT = 1.f;               // of values()
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
  static constexpr float UNIT = 4.f;
  struct Raw { uint32_t codes, scale; };
  const uint8_t *codes, *scales;
  int64_t row_bytes, scale_row;
  __device__ __forceinline__ Raw get(int64_t m, int k, int) const {
    return Raw{*reinterpret_cast<const uint32_t*>(codes + m * row_bytes + (k >> 1)), scales[m * scale_row + (k >> 5)]};
  }
  static __device__ __forceinline__ Raw none() { return Raw{0u, 0u}; }
  static __device__ __forceinline__ void values(const Raw& r, float* f) {
    mx_expand8(r.codes, f);
    const float s = mx_quarter_scale(r.scale);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] *= s;
  }
};

// FUSED: an activation, a gate and a residual on the way out.  The residual may be y itself, so y is not __restrict__.  With a gate, channel n of a
// warp is row n / 2 of the weights' first half (n even) or second half (n odd), so that a gate and its factor are in the same warp.
struct MxTail {
  int act, gated;
  const void* residual;
  int64_t r_stride;
};
template <bool FUSED>
__device__ __forceinline__ int weight_row(const MxTail& tail, int n, int N) { return FUSED && tail.gated ? (n & 1) * (N >> 1) + (n >> 1) : n; }

template <typename X, typename T, int MT, int U, bool FUSED>
__global__ void __launch_bounds__(kMxThreads)
mx_product_rows_kernel(X x, const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t row_bytes, int64_t scale_row,
                       const float* __restrict__ bias, int N, int K, int M, int k_warps, T* y, int64_t y_stride, MxTail tail) {
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
          const int64_t row = weight_row<FUSED>(tail, n0 + i, N);
          raw[i][u] = live ? *reinterpret_cast<const uint32_t*>(codes + row * row_bytes + (int64_t)w * 4) : 0u;
          sb[i][u] = live ? scales[row * scale_row + (w >> 2)] : 0u;
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
          const float s = mx_quarter_scale(sb[i][u]);
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
      if constexpr (FUSED) {
        v = v * (4.f * X::UNIT) + (bias && n0 + i < N ? bias[weight_row<true>(tail, n0 + i, N)] : 0.f);
        int o = n0 + i;
        if (tail.gated) {                          // lanes below MT have the gates, MT lanes further on is what each multiplies
          const float up = __shfl_down_sync((1u << R * MT) - 1u, v, MT);
          mx_activate<1>(&v, tail.act);
          v *= up;
          o = i == 0 ? n0 >> 1 : N;
        } else {
          mx_activate<1>(&v, tail.act);
        }
        if (o < N >> tail.gated && m0 + r < M) {
          if (tail.residual) v += to_float(static_cast<const T*>(tail.residual)[(m0 + r) * tail.r_stride + o]);
          y[(m0 + r) * y_stride + o] = from_float<T>(v);
        }
      } else {
        if (n0 + i < N && m0 + r < M) y[(m0 + r) * y_stride + n0 + i] = from_float<T>(v * (4.f * X::UNIT) + (bias ? bias[n0 + i] : 0.f));
      }
    }
    if (k_warps > 1) __syncthreads(); else __syncwarp();
  }
}

template <int MT, int U, bool FUSED, typename X, typename T>
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
  mx_product_rows_kernel<X, T, MT, U, FUSED><<<grid, kMxThreads, 0, s>>>(x, p.w_codes, p.w_scales, row_bytes, scale_row, p.bias, p.N, p.K, p.M,
                                                                        k_warps, static_cast<T*>(p.y), p.y_stride,
                                                                        MxTail{p.act, p.gated, p.residual, p.r_stride});
  AIQ_LAUNCH_CHECK("mx_product_rows");
  return AIQ_OK;
}
template <bool FUSED, typename X, typename T>
aiq_status_t product_rows(const MxProduct& p, X x, cudaStream_t s) {
  LaunchScope scope(AIQ_KERNEL_QLINEAR, s, 2.0 * p.M * p.N * p.K,
                    (double)(p.N + (p.x ? 0 : p.M)) * (mx_row_bytes(p.K) + mx_scale_row_bytes(p.K)) + sizeof(T) * (double)p.M * (p.N + (p.x ? p.K : 0)));
  if (p.M == 1) return product_rows<1, 4, FUSED, X, T>(p, x, s);
  if (p.M == 2) return product_rows<2, 2, FUSED, X, T>(p, x, s);
  return product_rows<4, 2, FUSED, X, T>(p, x, s);
}

// ---------------------------------------------------------------------------------------
// the product, one row of x, in integers
// ---------------------------------------------------------------------------------------
// Twice an element is an integer of -12 to 12, and a block of x is P planes of bytes times a power of two, so a block's sum is 8 P
// four-product instructions.  A lane holds one block of x in registers; the warp passes 1,024 values of R channels by it, one 16-byte
// load per lane and channel.  The warps of a CTA share out k.
//   codes -> bytes: a permutation takes byte (code & 7) of a table of eight, or, where bit 3 of the code is set, that byte's top bit eight
//     times.  All table bytes have it set, so the table of 2 |element| - 64 gives 255 for negative codes, the one of -2 |element| - 64
//     with bit 3 inverted 255 for the others, and their AND is 2 element - 64.  The sums start at 64 times the block's sum of x.
//   x -> planes: rn(x 2^(8 P - 2 - e)) in two's complement, 2^e <= largest |x| < 2^(e + 1); top byte signed.  Three planes for bfloat16, four
//     for half, one (its own codes) for a microscaled x.  A block's sum is then an exact integer, below 2^41, and rounded once,
//     when it becomes a float32.
//   What the planes cannot hold, the last bits of values below 2^-15 (bfloat16) or 2^-20 (half) of the block's largest, is multiplied value
//     by value in float32 (one_rest): in normally distributed data one value in twenty thousand or fewer.
// Bound by instruction issue: 110 to 120 a block and lane, issue slots 59 % busy and the integer pipe 50 % (28000 x 8192, bfloat16, 46 us, where
// 438 CTAs go into 1.5 rounds), the multiply pipe's half that takes integers 50 %.  On the device,
// float kernel or tensor cores | this one, weights from memory: bfloat16 8192 x 1024 5.7 | 4.9 us, 4096 x 4096 8.7 | 6.5; half,
// 4096 x 4096 8.5 | 6.8; microscaled 2000 x 2000 3.7 | 2.7, 4096 x 4096 7.2 | 4.8.  Rounding what the planes cannot hold away instead took as long; finding it with
// float32 comparisons for every value, 0.3 to 0.6 us more.
// Two groups of channels on their way instead of one: 4096 x 4096 6.6 -> 6.9; 24 warps of 80 registers 6.9 instead of 6.8; default
// caching of the codes instead of streaming 6.5 -> 6.8.
// Float kernel | this: bfloat16 1100 x 1000 3.0 | 3.1 us, 2000 x 2000 3.7 | 3.7, 512 x 8192 3.6 | 3.6, 1500 x 3000 4.1 | 4.0, 1024 x 8192
// 5.6 | 4.9; half 1100 x 1000 2.9 | 3.2, 2000 x 2000 3.6 | 3.8, 1500 x 3000 4.4 | 4.3; 70 x 16500, too few channels for the SMs, 4.9 | 5.9.  So it
// gains above 2^22 and loses up to 0.3 us below (more with few channels); it starts at 2^20 because what an infinity in x gives changes there,
// and callers know it so.  Both microscaled it is faster at every size: 128 x 128 2.6 | 2.2.
constexpr int64_t kOneFrom = 1 << 20;
constexpr int kOneRow = 4;                       // channels at a time
constexpr int kOneWarps = 16, kOneChannels = 64; // at most, per CTA

// 2^(s - 127) of two scale bytes, NaN for 255
__device__ __forceinline__ float2 mx_scale2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("{\n\t.reg .b16 s;\n\tcvt.u16.u32 s, %1;\n\tcvt.rn.bf16x2.ue8m0x2 %0, s;\n\t}" : "=r"(r) : "r"(a | b << 8));
  return make_float2(__uint_as_float(r << 16), __uint_as_float(r & 0xFFFF0000u));
}
__device__ __forceinline__ uint32_t permute(uint32_t lo, uint32_t hi, uint32_t sel) {
  uint32_t r;
  asm("prmt.b32 %0, %1, %2, %3;" : "=r"(r) : "r"(lo), "r"(hi), "r"(sel));
  return r;
}
__device__ __forceinline__ int dot4(uint32_t a, uint32_t b, int c, bool b_signed) {
  int r;
  if (b_signed) asm("dp4a.s32.s32 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
  else asm("dp4a.s32.u32 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
  return r;
}
// eight codes as 2 element - 64, the first in the lowest byte
__device__ __forceinline__ uint2 biased8(uint32_t c) {
  const uint32_t n = c ^ 0x88888888u;
  return make_uint2(permute(0xC3C2C1C0u, 0xCCC8C6C4u, c) & permute(0xBDBEBFC0u, 0xB4B8BABCu, n),
                    permute(0xC3C2C1C0u, 0xCCC8C6C4u, c >> 16) & permute(0xBDBEBFC0u, 0xB4B8BABCu, n >> 16));
}

// a lane's block of x
template <int P>
struct OneBlock {
  uint32_t plane[P][8];
  int start[P];
  float low, last;                               // the block's sum is the planes' * low * weights' scale * last
  int up;                                        // the planes' values are x 2^up
  uint32_t rest;                                 // bit j: value j may not be all in the planes
  float first;                                   // what is left of the first of them
};
template <int P>
__device__ __forceinline__ void one_block_unit(OneBlock<P>& b, int e, bool dead) {
  // the block is plane sums times 2^e, |e| < 200: half of it on each side of the weights' scale, behind a common 2^-32, so that nothing
  // overflows or loses bits on the way that would not in the result
  const int a = (e + 32) >> 1, z = e + 32 - a;
  b.low = __uint_as_float((uint32_t)(a - 32 + 127) << 23);
  b.last = dead ? __uint_as_float(0x7FC00000u) : __uint_as_float((uint32_t)(z + 127) << 23);
#pragma unroll
  for (int q = 0; q < P; ++q) {
    int s = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) s = dot4(0x01010101u, b.plane[q][w], s, q == P - 1);
    b.start[q] = 64 * s;
  }
}

template <typename T>
struct OneOf {                                   // x in 16 bits
  static constexpr int P = std::is_same<T, __half>::value ? 4 : 3;
  const T* x;
  bool vec;
  __device__ __forceinline__ void get(OneBlock<P>& b, int k, int K) const {
    uint32_t raw[16];                              // two values each
    if (vec && k + 32 <= K) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint4 r = reinterpret_cast<const uint4*>(x + k)[i];
        raw[4 * i] = r.x; raw[4 * i + 1] = r.y; raw[4 * i + 2] = r.z; raw[4 * i + 3] = r.w;
      }
    } else {
      T t[32];
#pragma unroll
      for (int j = 0; j < 32; ++j) t[j] = k + j < K ? x[k + j] : from_float<T>(0.f);
      memcpy(raw, t, sizeof(raw));
    }
    // The largest |value|, and the least other than zero: with the sign bit set and one taken off, read as signed numbers, zero comes last.
    uint32_t top2 = 0, least2 = 0x7FFF7FFFu;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      top2 = __vmaxu2(top2, raw[i] & 0x7FFF7FFFu);
      least2 = __vmins2(least2, (raw[i] | 0x80008000u) - 0x00010001u);
    }
    const uint32_t least1 = __vmins2(least2, least2 >> 16 | least2 << 16);
    const uint32_t top = float_bits(max(top2 >> 16, top2 & 0xFFFFu)), least = float_bits((least1 + 1) & 0x7FFFu);
    const bool dead = top >= 0x7F800000u;
    const int e = max((int)(top >> 23) - 127, -126), up = dead ? 0 : 8 * P - 2 - e;
    float f[32];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const T* h = reinterpret_cast<const T*>(&raw[i]);
      f[2 * i] = to_float(h[0]);
      f[2 * i + 1] = to_float(h[1]);
    }
    int v[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = dead ? 0 : integer(f[j], up);
    b.up = up;
    b.rest = 0;
    // all bits of a value are in the planes where its last one is: at its exponent less 7 (bfloat16) or 10 (half)
    const int lowest = (P == 4 ? 10 : 7) + 127 - up;               // of a float32's exponent field
    if ((int)(least >> 23) < lowest && !dead && least != 0) {
#pragma unroll
      for (int j = 0; j < 32; ++j)
        if ((__float_as_uint(f[j]) & 0x7FFFFFFFu) - 1 < ((uint32_t)lowest << 23) - 1) b.rest |= 1u << j;
      b.first = left(to_float(x[k + __ffs(b.rest) - 1]), up);
    }
#pragma unroll
    for (int w = 0; w < 8; ++w)
#pragma unroll
      for (int q = 0; q < P; ++q) {
        const uint32_t sel = q | (4 + q) << 4;
        b.plane[q][w] = permute(permute(v[4 * w], v[4 * w + 1], sel), permute(v[4 * w + 2], v[4 * w + 3], sel), 0x5410);
      }
    one_block_unit(b, -up - 1, dead);
  }
  // |value| of 16 bits as the bits of a float32
  static __device__ __forceinline__ uint32_t float_bits(uint32_t a) {
    if (P == 3) return a << 16;
    return __float_as_uint(__half2float(__ushort_as_half((unsigned short)a)));
  }
  // f 2^up as an integer; the power of two is two factors, so that both are in range
  static __device__ __forceinline__ int integer(float f, int up) {
    const int half = up >> 1;
    return __float2int_rn(f * __uint_as_float((uint32_t)(half + 127) << 23) * __uint_as_float((uint32_t)(up - half + 127) << 23));
  }
  // what that leaves out of f, exactly
  static __device__ __forceinline__ float left(float f, int up) {
    const int half = up >> 1;
    return f - (float)integer(f, up) * __uint_as_float((uint32_t)(127 - half) << 23) * __uint_as_float((uint32_t)(127 - (up - half)) << 23);
  }
};
// one of a word's eight elements, from bit `shift` on
__device__ __forceinline__ float one_element(uint32_t word, int shift) {
  uint32_t h;
  asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, a;\n\t}" : "=r"(h) : "r"((word >> shift) & 0xFu));
  return __half2float(__ushort_as_half((unsigned short)(h & 0xFFFFu)));
}
// The sum of what the planes of a lane's block leave out, times its codes of R channels.  The values, save the first, come from memory again:
// nothing is held for them.
template <typename T>
__device__ __forceinline__ void one_rest(const OneOf<T>& x, const OneBlock<OneOf<T>::P>& b, int k, const uint4 (&c)[kOneRow], float (&sum)[kOneRow]) {
#pragma unroll
  for (int i = 0; i < kOneRow; ++i) sum[i] = 0.f;
  float r = b.first;
#pragma unroll 1
  for (uint32_t m = b.rest; m;) {
    const int at = __ffs(m) - 1;
#pragma unroll
    for (int i = 0; i < kOneRow; ++i) {
      const uint32_t word = at & 16 ? (at & 8 ? c[i].w : c[i].z) : (at & 8 ? c[i].y : c[i].x);
      sum[i] = fmaf(r, one_element(word, 4 * (at & 7)), sum[i]);
    }
    m &= m - 1;
    if (m) r = OneOf<T>::left(to_float(x.x[k + __ffs(m) - 1]), b.up);
  }
}
struct OneHeld {                                 // x microscaled
  static constexpr int P = 1;
  const uint8_t *codes, *scales;
  __device__ __forceinline__ void get(OneBlock<1>& b, int k, int K) const {
    uint4 c = make_uint4(0, 0, 0, 0);
    uint32_t s = 127;
    if (k < K) {
      c = *reinterpret_cast<const uint4*>(codes + (k >> 1));
      s = scales[k >> 5];
    }
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint2 u = biased8(w[i]);
      b.plane[0][2 * i] = __vadd4(u.x, 0x40404040u);
      b.plane[0][2 * i + 1] = __vadd4(u.y, 0x40404040u);
    }
    one_block_unit(b, s == 255 ? 0 : (int)s - 127 - 2, s == 255);
  }
};

template <typename X, typename T, bool FUSED>
__global__ void __launch_bounds__(32 * kOneWarps, X::P == 1 ? 2 : 1)
mx_product_row_kernel(X x, const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t row_bytes, int64_t scale_row,
                      const float* __restrict__ bias, int N, int K, int channels, T* y, MxTail tail) {
  constexpr int R = kOneRow, P = X::P;
  __shared__ float part[kOneChannels * kOneWarps];
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  const int n0 = blockIdx.x * channels, n_end = min(N - n0, channels);
  const int blocks = (int)(row_bytes >> 4);
  for (int b0 = warp * 32; b0 < blocks; b0 += warps * 32) {
    const int block = b0 + lane;
    // behind a row's end a lane reads the row's last block, and has zeros for x
    const uint32_t at = (uint32_t)min(block, blocks - 1), at16 = at * 16;
    uint4 next[R];
    uint32_t next_s[R];
    auto load = [&](int n) {
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const int64_t row = weight_row<FUSED>(tail, min(n0 + n + i, N - 1), N);
        next[i] = __ldcs(reinterpret_cast<const uint4*>(codes + row * row_bytes + at16));
        next_s[i] = *(scales + row * scale_row + at);
      }
    };
    load(0);
    OneBlock<P> xb;
    const int k = min(block, 0x3FFFFFF) * 32;
    x.get(xb, k, K);
    bool any_rest = false;
    if constexpr (P > 1) any_rest = __any_sync(0xffffffffu, xb.rest != 0);
    for (int n = 0; n < n_end; n += R) {
      uint4 c[R];
      float ws[R], v[R];
#pragma unroll
      for (int i = 0; i < R; i += 2) {
        const float2 two = mx_scale2(next_s[i], next_s[i + 1]);
        ws[i] = two.x; ws[i + 1] = two.y;
        c[i] = next[i]; c[i + 1] = next[i + 1];
      }
      if (n + R < n_end) load(n + R);
#pragma unroll
      for (int i = 0; i < R; ++i) {
        int s[P];
#pragma unroll
        for (int q = 0; q < P; ++q) s[q] = xb.start[q];
        const uint32_t w[4] = {c[i].x, c[i].y, c[i].z, c[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint2 u = biased8(w[j]);
#pragma unroll
          for (int q = 0; q < P; ++q)
            s[q] = dot4(u.y, xb.plane[q][2 * j + 1], dot4(u.x, xb.plane[q][2 * j], s[q], q == P - 1), q == P - 1);
        }
        float sum;
        if constexpr (P == 1) sum = (float)s[0] * xb.low;
        else if constexpr (P == 3) sum = (float)((int64_t)s[2] * 65536 + (s[1] * 256 + s[0])) * xb.low;
        else sum = (float)((int64_t)(s[3] * 256 + s[2]) * 65536 + (s[1] * 256 + s[0])) * xb.low;
        v[i] = sum * ws[i] * xb.last;
      }
      if constexpr (P > 1)
        if (any_rest) {
          float rest[R];
          one_rest(x, xb, k, c, rest);
#pragma unroll
          for (int i = 0; i < R; ++i) v[i] = fmaf(rest[i], ws[i], v[i]);
        }
      // the warp's sums of four channels at once: lanes 0, 8, 16 and 24 end up with one each
      const bool up = lane & 16, odd = lane & 8;
      const float a0 = (up ? v[2] : v[0]) + __shfl_xor_sync(0xffffffffu, up ? v[0] : v[2], 16);
      const float a1 = (up ? v[3] : v[1]) + __shfl_xor_sync(0xffffffffu, up ? v[1] : v[3], 16);
      float a = (odd ? a1 : a0) + __shfl_xor_sync(0xffffffffu, odd ? a0 : a1, 8);
#pragma unroll
      for (int o = 4; o > 0; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
      if ((lane & 7) == 0) {
        float* to = part + (n + (lane >> 3)) * warps + warp;
        *to = b0 == warp * 32 ? a : *to + a;
      }
    }
  }
  __syncthreads();
  if constexpr (FUSED) {
    // n0 and n_end are even with a gate: channels come in fours, and N is even
    for (int n = threadIdx.x << tail.gated; n < n_end; n += blockDim.x << tail.gated) {
      float v = bias ? bias[weight_row<true>(tail, n0 + n, N)] : 0.f;
      for (int w = 0; w < warps; ++w) v += part[n * warps + w];
      mx_activate<1>(&v, tail.act);
      if (tail.gated) {
        float up = bias ? bias[weight_row<true>(tail, n0 + n + 1, N)] : 0.f;
        for (int w = 0; w < warps; ++w) up += part[(n + 1) * warps + w];
        v *= up;
      }
      const int o = (n0 + n) >> tail.gated;
      if (tail.residual) v += to_float(static_cast<const T*>(tail.residual)[o]);
      y[o] = from_float<T>(v);
    }
    return;
  }
  for (int n = threadIdx.x; n < n_end; n += blockDim.x) {
    float v = 0.f;
    for (int w = 0; w < warps; ++w) v += part[n * warps + w];
    y[n0 + n] = from_float<T>(v + (bias ? bias[n0 + n] : 0.f));
  }
}

template <bool FUSED, typename X, typename T>
aiq_status_t product_row(const MxProduct& p, X x, cudaStream_t s) {
  DeviceProps props;
  if (aiq_status_t st = current_device_props(&props)) return st;
  const int64_t row_bytes = mx_row_bytes(p.K), scale_row = mx_scale_row_bytes(p.K);
  const int64_t slices = (row_bytes / 16 + 31) / 32;
  const int warps = (int)min(slices, (int64_t)kOneWarps), ctas = props.n_sms * ((X::P == 1 ? 32 : 16) / warps);   // as many warps as an SM holds
  const int channels = min(kOneChannels, ((p.N + ctas - 1) / ctas + kOneRow - 1) / kOneRow * kOneRow);
  LaunchScope scope(AIQ_KERNEL_QLINEAR, s, 2.0 * p.N * p.K,
                    (double)(p.N + (p.x ? 0 : 1)) * (row_bytes + scale_row) + sizeof(T) * (double)(p.N + (p.x ? p.K : 0)));
  mx_product_row_kernel<X, T, FUSED><<<(p.N + channels - 1) / channels, 32 * warps, 0, s>>>(x, p.w_codes, p.w_scales, row_bytes, scale_row, p.bias, p.N,
                                                                                           p.K, channels, static_cast<T*>(p.y),
                                                                                           MxTail{p.act, p.gated, p.residual, p.r_stride});
  AIQ_LAUNCH_CHECK("mx_product_row");
  return AIQ_OK;
}

template <typename T, bool FUSED>
aiq_status_t product_rows(const MxProduct& p, cudaStream_t s) {
  if (FUSED || p.x) {
    const bool vec = (((uintptr_t)p.x) & 15) == 0 && (p.M == 1 || p.x_stride * (int64_t)sizeof(T) % 16 == 0);
    if constexpr (sizeof(T) == 2)
      if (p.M == 1 && (int64_t)p.N * p.K > kOneFrom) return product_row<FUSED, OneOf<T>, T>(p, OneOf<T>{static_cast<const T*>(p.x), vec}, s);
    return product_rows<FUSED, RowsOf<T>, T>(p, RowsOf<T>{static_cast<const T*>(p.x), p.x_stride, vec}, s);
  }
  if constexpr (!FUSED) {
    if (p.M == 1) return product_row<false, OneHeld, T>(p, OneHeld{p.x_codes, p.x_scales}, s);
    return product_rows<false, RowsHeld, T>(p, RowsHeld{p.x_codes, p.x_scales, mx_row_bytes(p.K), mx_scale_row_bytes(p.K)}, s);
  }
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
    case AIQ_DTYPE_F32: return product_rows<float, false>(p, s);
    case AIQ_DTYPE_F16: return product_rows<__half, false>(p, s);
    default: return product_rows<__nv_bfloat16, false>(p, s);
  }
}
aiq_status_t launch_mx_linear_act_rows(const MxProduct& p, cudaStream_t s) {
  switch (p.dtype) {
    case AIQ_DTYPE_F32: return product_rows<float, true>(p, s);
    case AIQ_DTYPE_F16: return product_rows<__half, true>(p, s);
    default: return product_rows<__nv_bfloat16, true>(p, s);
  }
}

}  // namespace aiq

// ---------------------------------------------------------------------------------------
// C entry points
// ---------------------------------------------------------------------------------------
using aiq::set_error;

static const int kMxMost = 1 << 30;          // of any size: what rounds a size up stays an int

// AIQ_OK, or what is wrong with the sizes and pointers that every entry point takes
static aiq_status_t mx_check(const char* what, const void* codes, const void* scales, int rows, int K) {
  if (!codes || !scales) return set_error(AIQ_ERR_INVALID_ARG, "%s: null pointer", what);
  if (rows <= 0 || K <= 0 || rows > kMxMost || K > kMxMost) return set_error(AIQ_ERR_INVALID_ARG, "%s: %d rows of K=%d", what, rows, K);
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

static aiq_status_t mx_check_tail(const char* what, int activation, int gated, int N) {
  if (activation < AIQ_ACT_NONE || activation > AIQ_ACT_GELU_TANH) return set_error(AIQ_ERR_INVALID_ARG, "%s: activation=%d", what, activation);
  if (gated != 0 && gated != 1) return set_error(AIQ_ERR_INVALID_ARG, "%s: gated=%d", what, gated);
  if (gated && (N & 1)) return set_error(AIQ_ERR_INVALID_ARG, "%s: gated with N=%d", what, N);
  return AIQ_OK;
}

extern "C" size_t aiq_mx_row_bytes(int K) { return K > 0 ? (size_t)aiq::mx_row_bytes(K) : 0; }
extern "C" size_t aiq_mx_scale_row_bytes(int K) { return K > 0 ? (size_t)aiq::mx_scale_row_bytes(K) : 0; }

extern "C" aiq_status_t aiq_mx_quantize(const void* x, int dtype, int rows, int K, int64_t x_stride, void* codes_out,
                                        void* scales_out, void* stream) {
  if (rows == 1) x_stride = K;                 // ignored
  if (aiq_status_t st = mx_check("aiq_mx_quantize", codes_out, scales_out, rows, K)) return st;
  if (aiq_status_t st = mx_check_rows("aiq_mx_quantize", x, dtype, x_stride)) return st;
  if (aiq_status_t st = aiq::check_device_sm100()) return st;
  return aiq::launch_mx_quantize(x, dtype, rows, K, x_stride, static_cast<uint8_t*>(codes_out), static_cast<uint8_t*>(scales_out),
                                 (cudaStream_t)stream);
}

extern "C" aiq_status_t aiq_mx_dequantize(const void* codes, const void* scales, int rows, int K, int dtype, void* y, int64_t y_stride,
                                          void* stream) {
  if (rows == 1) y_stride = K;
  if (aiq_status_t st = mx_check("aiq_mx_dequantize", codes, scales, rows, K)) return st;
  if (aiq_status_t st = mx_check_out("aiq_mx_dequantize", y, dtype, rows, K, y_stride)) return st;
  if (aiq_status_t st = aiq::check_device_sm100()) return st;
  return aiq::launch_mx_dequantize(static_cast<const uint8_t*>(codes), static_cast<const uint8_t*>(scales), rows, K, dtype, y, y_stride,
                                   (cudaStream_t)stream);
}

// (Rows of x that do not start on 16 bytes are told by K: their stride and address are not known when the workspace is asked for.)
// Whether the kernel for few rows and small matrices beats the tensor-core kernel, whose time below 2^22 products is its chain of
// set-up, first loads and last stores.  On the device, rows | tensor cores (linear layer: with its pre-pass, a second launch):
//   linear, bf16     1 row (integers above 2^20): 1280 x 320 2.8 | 7.0 us, 2000 x 2000 3.7 | 8.2, 4096 x 4096 6.4 | 9.7, 8192 x 4096 9.4 | 10.8, 8192 x 8192 14.5 | 14.4,
//                    28000 x 8192 43 | 34;  float32 4096 x 4096 9.1 | 9.7, 8192 x 8192 25 | 15.5
//                    4 rows: 724 x 724 5.0 | 7.5, 2000 x 2000 7.4 | 8.2;  8 rows, 724 x 724 5.6 | 6.9, 720 x 720 4.3 | 7.0;
//                    16 rows, 724 x 724 (rows that do not start on 16 bytes) 9.4 | 7.0, 720 x 720 5.4 | 7.0, 300 x 2000 6.9 | 7.2
//   both microscaled 1 row: 2000 x 2000 2.7 | 6.3, 4096 x 4096 4.8 | 7.6, 8192 x 4096 6.8 | 10.0, 8192 x 8192 12.0 | 12.0, 28000 x 8192 29 | 26;  8 rows, 300 x 300 3.1 | 4.9;  4 rows, 2000 x 2000 8.0 | 6.4
static bool mx_rows_pay(int N, int K, int M, int log2_most) { return (double)N * K * M <= (double)(1ll << log2_most); }

extern "C" size_t aiq_mx_linear_workspace_bytes(int N, int K, int M, int dtype) {
  if (N <= 0 || K <= 0 || M <= 0 || N > kMxMost || K > kMxMost || M > kMxMost || !aiq::mx_dtype_ok(dtype)) return 0;
  return mx_rows_pay(N, K, M, M == 1 && dtype != AIQ_DTYPE_F32 ? 25 : M <= 4 ? 24 : K % 8 == 0 ? 23 : 22) ? 0 : aiq::mx_tc_workspace_bytes(K, M, dtype);
}

extern "C" aiq_status_t aiq_mx_linear(const void* codes, const void* scales, const float* bias, int N, int K, const void* x, int dtype,
                                      int M, int64_t x_stride, void* y, int64_t y_stride, void* workspace, size_t workspace_bytes,
                                      void* stream) {
  if (aiq_status_t st = mx_check("aiq_mx_linear", codes, scales, N, K)) return st;
  if (M <= 0 || M > kMxMost) return set_error(AIQ_ERR_INVALID_ARG, "aiq_mx_linear: M=%d", M);
  if (M == 1) { x_stride = K; y_stride = N; }
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

extern "C" aiq_status_t aiq_mx_linear_act(const void* codes, const void* scales, const float* bias, int N, int K, const void* x, int dtype,
                                          int M, int64_t x_stride, int activation, int gated, const void* residual, int64_t r_stride, void* y,
                                          int64_t y_stride, void* workspace, size_t workspace_bytes, void* stream) {
  if (aiq_status_t st = mx_check("aiq_mx_linear_act", codes, scales, N, K)) return st;
  if (M <= 0 || M > kMxMost) return set_error(AIQ_ERR_INVALID_ARG, "aiq_mx_linear_act: M=%d", M);
  if (aiq_status_t st = mx_check_tail("aiq_mx_linear_act", activation, gated, N)) return st;
  const int outputs = gated ? N / 2 : N;
  if (M == 1) { x_stride = K; y_stride = r_stride = outputs; }
  if (aiq_status_t st = mx_check_rows("aiq_mx_linear_act", x, dtype, x_stride)) return st;
  if (aiq_status_t st = mx_check_out("aiq_mx_linear_act", y, dtype, M, outputs, y_stride)) return st;
  if (aiq_status_t st = mx_check_bias("aiq_mx_linear_act", bias)) return st;
  if (residual)
    if (aiq_status_t st = mx_check_rows("aiq_mx_linear_act", residual, dtype, r_stride)) return st;
  aiq::MxProduct p = {};
  p.w_codes = static_cast<const uint8_t*>(codes);
  p.w_scales = static_cast<const uint8_t*>(scales);
  p.bias = bias;
  p.x = x; p.x_stride = x_stride;
  p.y = y; p.y_stride = y_stride;
  p.N = N; p.K = K; p.M = M; p.dtype = dtype;
  p.act = activation; p.gated = gated;
  p.residual = residual; p.r_stride = r_stride;
  if (((uintptr_t)workspace) & 15) return set_error(AIQ_ERR_INVALID_ARG, "aiq_mx_linear_act: workspace not 16-byte aligned");
  const size_t needed = aiq_mx_linear_workspace_bytes(N, K, M, dtype);
  if (workspace && workspace_bytes < needed)
    return set_error(AIQ_ERR_WORKSPACE_TOO_SMALL, "aiq_mx_linear_act: workspace of %zu bytes, %zu needed", workspace_bytes, needed);
  if (aiq_status_t st = aiq::check_device_sm100()) return st;
  if (needed == 0 || !workspace) return aiq::launch_mx_linear_act_rows(p, (cudaStream_t)stream);
  return aiq::launch_mx_linear_act_tc(p, workspace, (cudaStream_t)stream);
}

extern "C" aiq_status_t aiq_mx_matmul(const void* a_codes, const void* a_scales, int M, const void* b_codes, const void* b_scales, int N,
                                      const float* bias, int K, void* y, int dtype, int64_t y_stride, void* stream) {
  if (aiq_status_t st = mx_check("aiq_mx_matmul", a_codes, a_scales, M, K)) return st;
  if (aiq_status_t st = mx_check("aiq_mx_matmul", b_codes, b_scales, N, K)) return st;
  if (M == 1) y_stride = N;
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
  if (mx_rows_pay(N, K, M, M == 1 ? 25 : 22)) return aiq::launch_mx_product_rows(p, (cudaStream_t)stream);
  return aiq::launch_mx_product_tc(p, nullptr, (cudaStream_t)stream);
}

extern "C" aiq_status_t aiq_debug_mx_expire_wait(int64_t limit_cycles) {
  if (limit_cycles < 0 || limit_cycles > 2000000000ll)
    return set_error(AIQ_ERR_INVALID_ARG, "aiq_debug_mx_expire_wait: limit_cycles=%lld outside [0, 2e9]", (long long)limit_cycles);
  aiq::mx_tc_expire_next(limit_cycles);
  return AIQ_OK;
}
