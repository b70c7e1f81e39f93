// The linear layer with a way out (see mx_tc.cuh, MODE 1 and 2) for up to four rows of x, in one launch and without a workspace.
//
// With so few rows the tensor cores are idle whatever they multiply, and what takes time is the way there: a pre-pass, and weights that a copy expands
// to a byte each.  So x is cut into more and smaller pieces, which every CTA makes itself while its first weights are on their way, and both operands are
// four-bit codes: kind::mxf4, 64 k per MMA, weights as they are stored.
//   A value is a fixed-point number in units of 2^(e - 3(P - 1)), 2^e <= the largest |x| of its block of 32 < 2^(e + 1), and P digits of it, of -4 to 3, each an
//   element of the format: with 4 added in every place the digits are three bits each.  P rows of the B operand, with the scale bytes of a quarter of e's, of
//   that less 3, ... (a quarter, since the first digit of the largest floats is 2^128); sums are multiplied by 4.  8, 10 and 13 digits hold a bfloat16, half and
//   float exactly, but for what lies below 2^-22, 2^-28, 2^-37 of the block's largest value, or 2^-126.
//   D[128 channels][row of x, digit], rows of B to a multiple of 16; the digits' sums are added up smallest first.
// A CTA takes 128 channels of a layer (or of one expert), and with a cluster a part of K; sums meet in the first CTA of the cluster, in a fixed order.
//   warp 0      TMA: weights and their scale bytes
//   warp 1      MMA issuer
//   warps 4-11  x to digits, the warp's next 512 values of a row at a time, 16 a lane; then
//   warps 4-7   scale bytes: shared -> tensor memory
//   warps 8-11  sums -> y
// Two CTAs (of little K up to four: cluster_smem) share an SM, so that one's set-up and way out are covered by the other's stream.
// What bounds it.  One token through 4 of 32 experts of 4096 x 2048, bfloat16, 7.9 us a call, 8.6 in a graph with weights from memory: a launch, the plan and the first bytes of
// x and weights one after the other (5 us), then 17.8 MB of weights (2.7 us at the copy rate).  Gated 16384 x 4096, one row 10 us (5.4 for the weights).
// With the pre-pass and tiles of mx_tc.cuh in its place 12.8 and 14.3.
#include "mx_tc.cuh"

namespace aiq {
namespace {

constexpr int kFewThreads = 12 * 32;
constexpr int kFewRows = 4;                      // of x, at most
constexpr int kFewScaleStages = 4;
constexpr int kFewSupers = 64;                   // of 512 k that a CTA may have
constexpr int kFewStages = 6;

template <typename T> struct Digits { static constexpr int P = 13; };
template <> struct Digits<__half> { static constexpr int P = 10; };
template <> struct Digits<__nv_bfloat16> { static constexpr int P = 8; };

struct FewParams {
  int N, K, M;                                   // M: rows of x that are multiplied: all (`common`), or the most that a tile has
  int act, gated;
  int b_rows;                                    // rows of B, a multiple of 16
  int n_chunks, supers_per_split, cluster, cluster_log2, stages;
  int vec;
  int common;                                    // the rows of x are the same for every tile; else the tile's rows of the plan
  int top_k, tokens, plan_kind, width;
  int tmem_cols, sf_col;
  int hold, limit;
  int64_t x_stride, y_stride, r_stride;
};
__host__ __device__ inline int few_supers(const FewParams& p) { return p.supers_per_split; }
// ring of weights; digits of x; scale bytes of both; sums of a cluster
__host__ __device__ inline int few_smem_bytes(const FewParams& p) {
  return 1024 + p.stages * kMxATile + 2 * few_supers(p) * p.b_rows * 128 + kFewScaleStages * 2048 + few_supers(p) * 512 + kFewRows * 128 * 4 * (p.cluster - 1) +
         8 * (2 * p.stages + 2 * kFewScaleStages + few_supers(p) + 9) + 16;
}

// 16 values of a row as integers in units of 2^(e - 3(P - 1)), with 4 added in every place of three bits
template <typename T> struct FixedPoint { typedef uint32_t type; };
template <> struct FixedPoint<float> { typedef uint64_t type; };

template <typename T>
__device__ __forceinline__ void to_digits(const T* row, int k, int K, int vec, int lane, uint8_t* tile, int b_row, uint8_t* scales) {
  constexpr int P = Digits<T>::P;
  typedef typename FixedPoint<T>::type U;
  float f[16];
  load_x(row, k, K, vec, f);
  load_x(row, k + 8, K, vec, f + 8);
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < 16; ++j) top = max(top, __float_as_uint(f[j]) & 0x7FFFFFFFu);
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  const bool dead = (top >> 23) == 255;            // a NaN or an infinity: scale byte 255 makes the block NaN
  const int e = max((int)(top >> 23), 3 * (P - 1) + 2), up = 3 * (P - 1) + 127 - e;      // of the value's unit 2^-up
  // 2^up as two factors, both in range
  const float a = __uint_as_float((uint32_t)((up >> 1) + 127) << 23), b = __uint_as_float((uint32_t)(up - (up >> 1) + 127) << 23);
  constexpr U BIAS = (U)(0x4924924924924924ull & ((1ull << 3 * P) - 1));
  U u[16];
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    const float v = dead ? 0.f : f[j] * a * b;
    u[j] = (sizeof(U) == 8 ? (U)__float2ll_rn(v) : (U)__float2int_rn(v)) + BIAS;
  }
  const int unit = (lane & 15) >> 1;               // of 16 bytes in the row's 128
  uint8_t* to = tile + (lane & 1) * 8;
#pragma unroll
  for (int q = 0; q < P; ++q) {
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t even = 0, odd = 0;                  // selectors: four digits each
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        even |= ((uint32_t)(u[8 * h + 2 * j] >> 3 * (P - 1 - q)) & 7u) << 4 * j;
        odd |= ((uint32_t)(u[8 * h + 2 * j + 1] >> 3 * (P - 1 - q)) & 7u) << 4 * j;
      }
      // the codes of -4 -3 -2 -1 | 0 1 2 3
      uint32_t x, y;
      asm("prmt.b32 %0, %1, %2, %3;" : "=r"(x) : "r"(0x0A0C0D0Eu), "r"(0x05040200u), "r"(even));
      asm("prmt.b32 %0, %1, %2, %3;" : "=r"(y) : "r"(0x0A0C0D0Eu), "r"(0x05040200u), "r"(odd));
      w[h] = x | y << 4;
    }
    const int r = b_row + q;
    *reinterpret_cast<uint2*>(to + r * 128 + ((unit ^ (r & 7)) << 4)) = dead ? make_uint2(0u, 0u) : make_uint2(w[0], w[1]);
    if (!(lane & 1)) scales[r * 16 + (lane >> 1)] = (uint8_t)(dead ? 255 : e - 2 - 3 * q);
  }
}

template <typename T>
__global__ void __launch_bounds__(kFewThreads)
mx_few_kernel(const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap sa_map, const __grid_constant__ FewParams p, const T* x,
              const float* bias, const T* residual, T* y, const int* header, const ExpertBlock* blocks, const int* slots) {
  constexpr int P = Digits<T>::P;
  constexpr bool PROMOTE = sizeof(T) == 4;         // sums leave the accumulator every 512 k
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int rank = blockIdx.x & (p.cluster - 1), tile = blockIdx.x >> p.cluster_log2;
  const int row_blocks = (p.N + 127) / 128;
  const int c_begin = min(p.n_chunks, rank * p.supers_per_split * 2), chunks = min(p.n_chunks - c_begin, p.supers_per_split * 2), supers = (chunks + 1) / 2;

  uint8_t* aring = smem;
  uint8_t* digits = aring + p.stages * kMxATile;                             // [chunk][row][128]
  uint8_t* sa_ring = digits + 2 * few_supers(p) * p.b_rows * 128;
  uint8_t* sb = sa_ring + kFewScaleStages * 2048;                            // [super][32 rows][16]
  float* partial = reinterpret_cast<float*>(sb + few_supers(p) * 512);      // [cluster - 1][row][128]
  uint64_t* bars = reinterpret_cast<uint64_t*>(partial + kFewRows * 128 * (p.cluster - 1));
  const uint32_t a_full = smem_u32(bars), a_empty = a_full + 8 * p.stages, s_full = a_empty + 8 * p.stages, s_empty = s_full + 8 * kFewScaleStages;
  const uint32_t t_full = s_empty + 8 * kFewScaleStages, t_empty = t_full + 16, d_full = t_empty + 16, d_empty = d_full + 16, retired = d_empty + 16;
  const uint32_t x_full = retired + 8;                                       // a super's digits are there
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(bars + 2 * p.stages + 2 * kFewScaleStages + 9 + few_supers(p));
  volatile int* s_abort = reinterpret_cast<volatile int*>(s_tmem + 1);

  // What needs nothing from the kernels before runs beside them (programmatic dependent launch); no global memory is touched before the wait.
  if (warp == 0) {
    // arrivals: four warps for scale bytes read, scale words written and sums read, p.M for a super's digits, one for everything else
    const int total = 2 * p.stages + 2 * kFewScaleStages + 9;
    for (int i = lane; i < total + few_supers(p); i += 32) {
      const int j = i - 2 * p.stages;
      const bool four = (j >= kFewScaleStages && j < 2 * kFewScaleStages + 2) || (j >= 2 * kFewScaleStages + 6 && j < 2 * kFewScaleStages + 8);
      mbar_init(a_full + 8 * i, i >= total ? p.M : four ? 4 : 1);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncwarp();
    if (lane == 0) {
      s_abort[0] = 0; s_abort[1] = p.limit;
      asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&a_map)) : "memory");
      asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&sa_map)) : "memory");
    }
  } else if (warp == 1) {
    tmem_alloc(smem_u32(s_tmem), (uint32_t)p.tmem_cols);
    tmem_relinquish();
  }
  chain_wait();
  // which weights, and which rows of y: begin to stop - 1
  int expert = 0, n_block = tile, begin = 0, stop = p.M;
  bool none = false;
  if (header) {
    const int block = tile / row_blocks;
    const int4 h = ld_chain(reinterpret_cast<const int4*>(header)), at = ld_chain(reinterpret_cast<const int4*>(blocks + block));
    none = h.z != p.tokens || h.w != p.plan_kind || block >= h.y;             // of the whole cluster
    const int before = (block - at.w) * p.width;
    expert = at.x;
    begin = at.y + before;
    stop = none ? begin : begin + min(at.z - before, p.width);
    n_block = tile - block * row_blocks;
  }
  const int n0 = n_block * 128;

  // As many rows of x at a time as there are tokens.  (A second time only where tokens have the same expert twice.)
  // Rings and phases go on from one time to the next.
  RingCursor ar, sr;
  uint32_t times = 0, sets = 0, ring = 0, ring_phase = 0;                    // sets: of 512 k so far; ring: of the warp's own
  for (int m0 = begin; m0 < stop; m0 = p.common ? stop : m0 + p.M, ++times) {
  const int end = p.common ? stop : min(stop, m0 + p.M), x_rows = p.common ? p.M : end - m0;
  int sent = 0, scales_sent = 0;
  auto send_a = [&]() {
    tma_fill_4d(smem_u32(aring) + ar.stage * kMxATile, &a_map, a_full + 8 * ar.stage, kMxATile, (c_begin + sent) * 128, 0, n0 >> p.gated, expert);
    ar.sent(p.stages);
    ++sent;
  };
  auto send_scales = [&]() {
    tma_fill_4d(smem_u32(sa_ring) + sr.stage * 2048, &sa_map, s_full + 8 * sr.stage, 2048, (c_begin / 2 + scales_sent) * 16, 0, n0 >> p.gated, expert);
    sr.sent(kFewScaleStages);
    ++scales_sent;
  };
  if (warp == 0 && times == 0) {
    if (supers > 0) send_scales();
    while (sent < chunks && sent < p.stages) send_a();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  chain_release();                                 // (behind the tensor memory's allocation)
  // Before a CTA writes into another's shared memory, that one has to have started: arrived here, waited for at the first write.
  if (p.cluster > 1) asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
  const uint32_t tmem_base = __shfl_sync(0xffffffffu, *s_tmem, 0);
  bool alive = times == 0 || __shfl_sync(0xffffffffu, s_abort[0], 0) == 0;   // a wait that ran out the time before: nothing is waited for any more
  const bool began = alive;
  float sum[kFewRows] = {0.f, 0.f, 0.f, 0.f};      // warps 8-11: of this lane's channel

  if (warp == 0) {
    while (alive && (sent < chunks || scales_sent < supers)) {
      if (scales_sent < supers && scales_sent * 2 <= sent + 2) {
        alive = mx_wait(s_empty + 8 * sr.stage, sr.phase ^ 1u, s_abort);
        if (alive) send_scales();
      } else {
        alive = mx_wait(a_empty + 8 * ar.stage, ar.phase ^ 1u, s_abort);
        if (alive) send_a();
      }
    }
    ar.drain(a_full, p.stages);
    sr.drain(s_full, kFewScaleStages);
  } else if (warp == 1) {
    constexpr uint32_t DESC_HI = (uint32_t)(1024 >> 4) | (1u << 14) | (2u << 29);   // SBO 1024, version 1, 128-byte swizzle
    constexpr uint32_t LBO_FIELD = 1u << 16;
    const uint32_t idesc = (1u << 7) | (1u << 10) | (1u << 23) | (1u << 27) | ((uint32_t)(p.b_rows >> 3) << 17);
    uint32_t as = ring, aph = ring_phase;
    for (int s = 0; s < supers && alive; ++s, ++sets) {
      const uint32_t tb = sets & 1, tph = (sets >> 1) & 1;
      if (PROMOTE) alive = mbar_wait_uniform(d_empty + 8 * tb, tph ^ 1u, s_abort);
      alive = alive && mbar_wait_uniform(t_full + 8 * tb, tph, s_abort);       // behind the digits, too
      const uint32_t d = tmem_base + (PROMOTE ? tb * p.b_rows : 0), sf = tmem_base + p.sf_col + tb * 32;
      for (int c = 2 * s; c < min(chunks, 2 * s + 2) && alive; ++c) {
        alive = mbar_wait_uniform(a_full + 8 * as, aph, s_abort);
        if (!alive) break;
        tc_fence_after();
        const uint64_t adesc = ((uint64_t)DESC_HI << 32) | (uint64_t)(((smem_u32(aring) + as * kMxATile) >> 4) | LBO_FIELD);
        const uint64_t bdesc = ((uint64_t)DESC_HI << 32) | (uint64_t)(((smem_u32(digits) + c * p.b_rows * 128) >> 4) | LBO_FIELD);
        const uint32_t sfa = sf + (c & 1) * 16;
        mx_mma4<0>(d, adesc, bdesc, idesc, sfa, sfa + 4, 8, PROMOTE ? (uint32_t)(c & 1) : (uint32_t)(c > 0), a_empty + 8 * as, 0u);
        if (++as == (uint32_t)p.stages) { as = 0; aph ^= 1u; }
      }
      if (!alive) break;
      umma_commit(t_empty + 8 * tb);
      if (PROMOTE || s + 1 == supers) umma_commit(d_full + 8 * (PROMOTE ? tb : 0));
    }
    ring = as; ring_phase = aph;
    if (began && !alive) {                         // what was issued must end before the CTA does
      umma_commit(retired);
      const long long t0 = clock64();
      while (!mbar_try_wait(retired, 0) && clock64() - t0 < kWaitLimitCycles) {}
    }
  } else if (warp >= 4) {
    for (int i = warp - 4; i < supers * p.M; i += 8) {
      const int s = i / p.M, r = i - s * p.M;
      int64_t row = r;                             // of x
      if (header && !p.common) row = m0 + r;
      const int half = lane >> 4;                  // a super is two chunks, 16 lanes each
      if (r < x_rows) to_digits<T>(x + row * p.x_stride, (c_begin / 2 + s) * 512 + lane * 16, p.K, p.vec, lane, digits + (2 * s + half) * p.b_rows * 128, r * P, sb + s * 512);
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(x_full + 8 * s);
    }
    if (warp < 8) {
      // ---- scale bytes -> tensor memory: as in mx_tc.cuh, eight columns per 128 k -----------------------
      const uint32_t quarter = (uint32_t)(warp & 3) * 32;
      uint32_t stage = ring, phase = ring_phase;
      for (int s = 0; s < supers && alive; ++s, ++sets) {
        const uint32_t tb = sets & 1, tph = (sets >> 1) & 1;
        alive = mx_wait(s_full + 8 * stage, phase, s_abort) && mx_wait(x_full + 8 * s, times & 1, s_abort) && mx_wait(t_empty + 8 * tb, tph ^ 1u, s_abort);
        if (!alive) break;
        tc_fence_after();
        const uint32_t dst = tmem_base + p.sf_col + tb * 32 + (quarter << 16);
#pragma unroll
        for (int c = 0; c < 8; c += 4) {
          const uint32_t src = (c == 0 ? smem_u32(sa_ring) + stage * 2048 : smem_u32(sb) + s * 512) + lane * 16, next = c == 0 ? 512 : 0;   // (B: 32 rows)
          const uint4 v0 = lds128(src), v1 = lds128(src + next), v2 = lds128(src + 2 * next), v3 = lds128(src + 3 * next);
          tmem_st4(dst + c, v0.x, v1.x, v2.x, v3.x);
          tmem_st4(dst + 8 + c, v0.y, v1.y, v2.y, v3.y);
          tmem_st4(dst + 16 + c, v0.z, v1.z, v2.z, v3.z);
          tmem_st4(dst + 24 + c, v0.w, v1.w, v2.w, v3.w);
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(s_empty + 8 * stage);
          if (!p.hold) mbar_arrive(t_full + 8 * tb);
        }
        if (++stage == kFewScaleStages) { stage = 0; phase ^= 1u; }
      }
      ring = stage; ring_phase = phase;
    } else {
      // ---- sums: lane = channel ---------------------------------------------------------------------------
      const uint32_t taddr = tmem_base + ((uint32_t)((warp & 3) * 32) << 16);
      for (int s = PROMOTE ? 0 : supers - 1; s < supers && s >= 0 && alive; ++s, ++sets) {
        const uint32_t tb = PROMOTE ? sets & 1 : 0, tph = PROMOTE ? (sets >> 1) & 1 : times & 1;
        alive = mx_wait(d_full + 8 * tb, tph, s_abort);
        if (!alive) break;
        tc_fence_after();
#pragma unroll
        for (int r = 0; r < kFewRows; ++r) {
          if (r >= x_rows) break;
          uint32_t v[16];
          tmem_ld16(taddr + tb * p.b_rows + r * P, v);
          tmem_ld_wait();
          float part = 0.f;
#pragma unroll
          for (int q = P - 1; q >= 0; --q) part += __uint_as_float(v[q]);      // the smallest digits first
          sum[r] += part * 4.f;
        }
        tc_fence_before();
        __syncwarp();
        if (PROMOTE && lane == 0) mbar_arrive(d_empty + 8 * tb);
      }
      if (!alive) {
#pragma unroll
        for (int r = 0; r < kFewRows; ++r) sum[r] = __int_as_float(0x7FC00000);
      }
    }
  }

  if (p.cluster > 1) {
    asm volatile("barrier.cluster.wait;" ::: "memory");
    if (warp >= 8 && rank > 0) {
      const uint32_t mine = smem_u32(partial) + (((rank - 1) * kFewRows) * 128 + (warp & 3) * 32 + lane) * 4;
#pragma unroll
      for (int r = 0; r < kFewRows; ++r) {
        uint32_t to;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(mine + r * 512), "r"(0));
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to), "f"(sum[r]) : "memory");
      }
    }
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    if (warp >= 8 && rank == 0)
      for (int q = 0; q < p.cluster - 1; ++q) {
        const float* from = partial + (q * kFewRows) * 128 + (warp & 3) * 32 + lane;
#pragma unroll
        for (int r = 0; r < kFewRows; ++r) sum[r] += from[r * 128];
      }
  }
  if (warp >= 8 && rank == 0) {
    const int ch = (warp & 3) * 32 + lane, n = n0 + ch, outputs = p.N >> p.gated, o = n >> p.gated;
    const float b = bias && o < outputs ? bias[(int64_t)expert * p.N + (p.gated ? (ch & 1) * outputs + o : n)] : 0.f;
    const int last = o < outputs ? end : 0;
    for (int m = m0; m < end; m += kFewRows) {     // (once, but for experts that a token has twice)
      float f[kFewRows];
#pragma unroll
      for (int j = 0; j < kFewRows; ++j) {
        const int t = header && p.common ? (m + j < end ? slots[m + j] / p.top_k : 0) : j;         // the row's place among those of x
        f[j] = (t == 0 ? sum[0] : t == 1 ? sum[1] : t == 2 ? sum[2] : sum[3]) + b;
      }
      T r[kFewRows] = {};
      if (residual) load_residual<kFewRows, T>(r, p.gated, lane, m, last, residual, p.r_stride, o);
      finish_columns<kFewRows, T>(f, p.act, p.gated, lane, m, last, y, p.y_stride, r, residual != nullptr, o);
    }
  }
  __syncthreads();
  }
  tc_fence_before();
  __syncthreads();                                 // (a CTA without rows comes here at once)
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(*s_tmem, (uint32_t)p.tmem_cols);
  }
}

// false: not for this kernel
template <typename T>
bool few_shape(const MxProduct& g, int tiles, int rows, int n_sms, int smem_optin, FewParams* out) {
  FewParams p = {};
  p.N = g.N; p.K = g.K; p.M = rows;
  p.b_rows = (rows * Digits<T>::P + 15) / 16 * 16;
  p.n_chunks = (g.K + 255) / 256;
  const int n_super = (g.K + 511) / 512;
  // up to two CTAs for every SM, each with 512 k at least.  (Up to four for every SM: 10.1 -> 14.5 us.)
  p.cluster = 1;
  while (p.cluster < 8 && tiles * p.cluster * 2 <= 2 * n_sms && n_super >= p.cluster * 2) p.cluster *= 2;
  while ((1 << p.cluster_log2) < p.cluster) ++p.cluster_log2;
  p.supers_per_split = (n_super + p.cluster - 1) / p.cluster;
  if (p.supers_per_split > kFewSupers) return false;
  p.sf_col = (sizeof(T) == 4 ? 2 : 1) * p.b_rows;
  p.tmem_cols = 32;
  while (p.tmem_cols < p.sf_col + 64) p.tmem_cols <<= 1;
  // slots for the weights: as many as leave room for a second CTA.  (Three CTAs with two or three slots each: one row through 16384 x 4096 10.1 -> 11.4 us.)
  const int chunks = 2 * p.supers_per_split;
  for (int room : {smem_optin / 2 - 1024, smem_optin}) {
    for (p.stages = chunks < kFewStages ? chunks : kFewStages; p.stages > 2 && few_smem_bytes(p) > room;) --p.stages;
    if (few_smem_bytes(p) <= room && (p.stages > 2 || p.stages == chunks)) break;
  }
  if (few_smem_bytes(p) > smem_optin) return false;
  *out = p;
  return true;
}

template <typename T>
aiq_status_t launch_few(const MxProduct& g, int tiles, FewParams p, const int* slots, cudaStream_t s) {
  DeviceProps props;
  if (aiq_status_t st = current_device_props(&props)) return st;
  AIQ_ENSURE_DYNAMIC_SMEM((mx_few_kernel<T>), props.smem_optin);
  EncodeTiledFn enc = encode_tiled_fn();
  if (!enc) return set_error(AIQ_ERR_CUDA, "cuTensorMapEncodeTiled is not available from the driver");
  p.act = g.act; p.gated = g.gated;
  p.vec = x_vec<T>(g);
  p.top_k = g.top_k; p.tokens = g.tokens; p.plan_kind = g.plan_kind; p.width = g.width;
  p.x_stride = g.x_stride; p.y_stride = g.y_stride; p.r_stride = g.r_stride;
  const long long expire = mx_tc_expire_cycles();
  p.limit = (int)((expire ? expire : kWaitLimitCycles) >> 10);
  p.hold = expire != 0;
  CUtensorMap a_map, sa_map;
  const cuuint64_t w_row = (cuuint64_t)mx_row_bytes(g.K), s_row = (cuuint64_t)mx_scale_row_bytes(g.K), N = g.N, G = g.gated ? 2 : 1, E = g.experts ? g.experts : 1;
  // (the order of the strides: see launch_kind in mx_tc.cuh)
  const cuuint32_t box[4] = {128, (cuuint32_t)G, (cuuint32_t)(128 / G), 1}, sbox[4] = {16, (cuuint32_t)G, (cuuint32_t)(128 / G), 1};
  const cuuint64_t dims[4] = {w_row, G, N / G, E}, strides[3] = {N / G * w_row, w_row, N * w_row};
  const cuuint64_t sdims[4] = {s_row, G, N / G, E}, sstrides[3] = {N / G * s_row, s_row, N * s_row};
  if (aiq_status_t st = encode(enc, &a_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, g.w_codes, 4, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B)) return st;
  if (aiq_status_t st = encode(enc, &sa_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, g.w_scales, 4, sdims, sstrides, sbox, CU_TENSOR_MAP_SWIZZLE_NONE)) return st;
  LaunchScope scope(AIQ_KERNEL_QLINEAR, s, 2.0 * g.M * g.N * g.K, (double)tiles * 128 * (w_row + s_row) + sizeof(T) * (double)g.M * (g.N + g.K));
  const size_t smem = p.cluster > 1 ? cluster_smem(few_smem_bytes(p), p.tmem_cols, props.smem_optin) : (size_t)few_smem_bytes(p);
  AIQ_CUDA_TRY(launch_chained_cluster(true, p.cluster, mx_few_kernel<T>, dim3(tiles * p.cluster), dim3(kFewThreads), smem, s, a_map, sa_map, p,
                                      static_cast<const T*>(g.x), g.bias, static_cast<const T*>(g.residual), static_cast<T*>(g.y), g.header, g.blocks, slots));
  AIQ_LAUNCH_CHECK("mx_few");
  return AIQ_OK;
}

template <typename T>
aiq_status_t few(const MxProduct& g, cudaStream_t s, bool* done) {
  *done = false;
  // rows of B up to 32: four of bfloat16, three of half, two of float
  const int rows = g.header ? g.tokens : g.M, row_blocks = (g.N + 127) / 128;
  if (rows > kFewRows || rows * Digits<T>::P > 32 || mx_promote<0, T>(g.K) != (sizeof(T) == 4)) return AIQ_OK;
  DeviceProps props;
  if (aiq_status_t st = current_device_props(&props)) return st;
  const int64_t tiles = (int64_t)row_blocks * (g.header ? g.blocks_most : 1);
  FewParams p;
  if (tiles > 0xFFFFFF || !few_shape<T>(g, (int)tiles, rows, props.n_sms, props.smem_optin, &p)) return AIQ_OK;
  p.common = !g.header || g.positions != nullptr;
  *done = true;
  MxExpireOnce once;
  return launch_few<T>(g, (int)tiles, p, g.slots, s);
}

}  // namespace

aiq_status_t launch_mx_few(const MxProduct& p, cudaStream_t s, bool* done) {
  switch (p.dtype) {
    case AIQ_DTYPE_F32: return few<float>(p, s, done);
    case AIQ_DTYPE_F16: return few<__half>(p, s, done);
    default: return few<__nv_bfloat16>(p, s, done);
  }
}

}  // namespace aiq
