// Products of microscaled 4-bit matrices on the tcgen05 tensor cores, which multiply codes and block scales as they are stored.
//
//   y[m][n] = sum_k x[m][k] W[n][k] + bias[n]
//
// The weights are the MMA's M operand (128 output channels per CTA) and the rows of x its N operand, so that the packed weights
// - the bytes that bound a small batch - are read once and a single row of x costs one narrow MMA:
//   D[128 n][R] += (A[128 n][k] 2^sa) (B[R][k] 2^sb)^T
// KIND 0 (aiq_mx_matmul): both operands are four-bit codes, kind::mxf4, 64 k per MMA, rows of 128 bytes = 256 k.
// KIND 1 (aiq_mx_linear): x enters as a sum of eight-bit floats (1 + 4 + 3 bits) with a scale per block of 32, kind::mxf8f6f4,
//   32 k per MMA; TMA expands the weights' codes to a byte each on the way to shared memory.  Each such piece takes the next
//   five bits of the values (four, and the sign of what is left), so that 2 / 3 / 5 of them hold a bfloat16 / half / float
//   exactly, unless it lies far below the largest value of its block: 2^-(12 + 5 pieces) of that one, or 2^-137, is what is lost at
//   most.
//   The pieces are rows of the B operand beside each other while they fit into 256 (then each has columns of its own
//   in the sums), or further MMAs into the same columns.
//   A pre-pass writes them into the workspace; the product starts under programmatic dependent launch and loads weights meanwhile.
// Products are exact.  The tensor core drops what an addition has below the accumulator's last bit; with float32 results and over long K
// (mx_promote) the sums are therefore taken out every 512 k and added up in float32 registers (PROMOTE: two sets of columns, used in turn).
//
//   warp 0     TMA: weights            warp 2   TMA: rows of x
//   warp 1     MMA issuer              warp 3   TMA: scale bytes of both, 512 k at a time (16 bytes a row)
//   warps 4-7  scale bytes: shared memory -> tensor memory, where the MMA reads them: four k blocks of a row in a column's
//              32-bit word, rows 32 to a column, the same in each quarter of the lanes
//   warps 8-15 sums: tensor memory -> registers -> y (two warps to a quarter of the lanes, half of the columns each)
// Many tiles: one CTA per SM takes every gridDim-th; the sums leave tensor memory within microseconds and are written while
// the next tile's MMAs run.  Few tiles: the K range is split over the CTAs of a cluster, whose sums meet in shared memory in a
// fixed order.
//
// What bounds it.  2,048 rows, 8192 x 8192, calls in a row with inputs that change, under the power limit (a few calls by themselves): bfloat16
// 246 us (206; tensor pipe active 79 % of what follows the pre-pass), half 396 (355), float32 685 (580; tiles of 128 rows: shared memory feeds
// an MMA every 87 cycles instead of 64); both microscaled 76 us, 3.6 PFLOP/s (61 to 64; tensor pipe 62 %: an MMA every 120 cycles instead of
// 96; its 10 KB of operands are filled for it alone, 85 bytes a cycle and SM).  One row, 8192 x 8192,
// 14.2 us on the device: the weight stream takes 5.7 of them, pre-pass, set-up and first loads 3, the way out 1.5; some 4 have no owner.  Both
// microscaled, 4096 x 4096, 16 rows 7.2 us: set-up, the first loads and the cluster's exchange.
// What made the difference: operands of the MMAs in uniform registers (see mbar_wait_uniform and the broadcast of the warp index),
// scale bytes requested before the weights, code that runs once per tile kept in small loops, tiles by rounds over the SMs.
#include "mx.cuh"
#include "tc_ptx.cuh"

namespace aiq {
namespace {

constexpr int kMxTcThreads = 16 * 32;
constexpr int kMxATile = 128 * 128;          // bytes of 128 rows of weights in shared memory
constexpr int kMxACopied = 128 * 64;         // bytes that a copy counts which expands four-bit codes: those of the codes
constexpr int kMxSuper = 512;                // k per set of scale bytes
constexpr int kMxScaleStages = 3;            // sets of scale bytes in shared memory
constexpr int kMxMaxStages = 12;

template <int KIND>
struct MxKind {
  static constexpr int CHUNK = KIND == 0 ? 256 : 128;       // k per 128 bytes of a row in shared memory
  static constexpr int CPS = kMxSuper / CHUNK;
};

struct MxTcParams {
  int N, M;
  int y_vec;                // rows of y start on four values
  int Mt;                   // rows of x per tile
  int pieces;               // KIND 1: eight-bit pieces of x
  int stack;                // 1: the pieces' rows are one operand
  int rows;                 // rows of a B operand: Mt, stacked pieces * Mt
  int n_chunks, supers_per_split;
  int cluster, cluster_log2;
  int push;                 // bytes for sums that the cluster's CTAs write into each other's shared memory; 0: read from it afterwards
  int m_blocks, tiles;      // tiles: row blocks * m_blocks, then the halves of some of them:
  int full;                 // tiles from this one on are halves of tiles (Mt / 2 rows of x), two for each
  int box;                  // rows of x per copy: Mt, or Mt / 2 where there are halves
  int d_bufs;               // sets of sums in tensor memory, used in turn: 2 for float32 results and where they fit
  int a_stages, b_stages;
  int b_cols;               // scale columns of a B operand (a multiple of 4)
  int sf_col, sf_group;     // first scale column, columns per 128 k
  int tmem_cols;
  int hold;                 // 1: no scale words are reported as written, so that waits run out (aiq_debug_mx_expire_wait)
  int limit;                // of a wait, in units of 1024 cycles
};

// tile `t` of a launch
struct MxTile {
  int n0, m0, Mt;
};
__device__ __forceinline__ MxTile mx_tile(const MxTcParams& p, int t) {
  const bool half = t >= p.full;
  const int f = half ? p.full + ((t - p.full) >> 1) : t, n = f / p.m_blocks;
  return MxTile{n * 128, (f - n * p.m_blocks) * p.Mt + (half && ((t - p.full) & 1) ? p.Mt / 2 : 0), half ? p.Mt / 2 : p.Mt};
}

__host__ __device__ inline int mx_b_unit(int rows) { return rows * 128; }
// rings of codes; with a split K range the sums of the tile, [row of x][128 channels], in their place afterwards or behind them
__host__ __device__ inline int mx_ring_bytes(const MxTcParams& p) {
  const int rings = p.a_stages * kMxATile + p.b_stages * mx_b_unit(p.rows), sums = p.cluster > 1 && !p.push ? p.Mt * 128 * 4 : 0;
  return (rings > sums ? rings : sums) + p.push;
}
__host__ __device__ inline int mx_scale_tile(const MxTcParams& p) { return (128 + p.b_cols * 32 * (p.stack ? 1 : p.pieces)) * 16; }
inline int mx_smem_bytes(const MxTcParams& p) {
  return 1024 + mx_ring_bytes(p) + kMxScaleStages * mx_scale_tile(p) + 8 * (2 * p.a_stages + 2 * p.b_stages + 2 * kMxScaleStages + 10) + 16;
}

// The four MMAs of 128 bytes of the operands' rows, and the commits that free the operands; one election.  accumulate: the first
// one adds to what is there, too.  group: scale columns per 128 k.  bar_a: 0 = the weights stay.
template <int KIND>
__device__ __forceinline__ void mx_mma4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t group,
                                        uint32_t accumulate, uint32_t bar_b, uint32_t bar_a) {
  if (KIND == 0)
    asm volatile(
        "{\n\t.reg .pred p, q, r;\n\t.reg .b64 x, y;\n\t.reg .b32 i, u, v;\n\telect.sync _|q, 0xffffffff;\n\tsetp.ne.b32 p, %7, 0;\n\t"
        "setp.ne.and.b32 r, %9, 0, q;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t"
        "add.s64 x, %1, 2;\n\tadd.s64 y, %2, 2;\n\tadd.u32 i, %3, 0x40000020;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], x, y, i, [%4], [%5], 1;\n\t"
        "add.s64 x, %1, 4;\n\tadd.s64 y, %2, 4;\n\tadd.u32 u, %4, %6;\n\tadd.u32 v, %5, %6;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], x, y, %3, [u], [v], 1;\n\t"
        "add.s64 x, %1, 6;\n\tadd.s64 y, %2, 6;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], x, y, i, [u], [v], 1;\n\t"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%8];\n\t"
        "@r tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%9];\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(group), "r"(accumulate), "r"(bar_b), "r"(bar_a) : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p, q, r;\n\t.reg .b64 x, y;\n\t.reg .b32 i;\n\telect.sync _|q, 0xffffffff;\n\tsetp.ne.b32 p, %6, 0;\n\t"
        "setp.ne.and.b32 r, %8, 0, q;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t"
        "add.s64 x, %1, 2;\n\tadd.s64 y, %2, 2;\n\tadd.u32 i, %3, 0x20000010;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], x, y, i, [%4], [%5], 1;\n\t"
        "add.s64 x, %1, 4;\n\tadd.s64 y, %2, 4;\n\tadd.u32 i, %3, 0x40000020;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], x, y, i, [%4], [%5], 1;\n\t"
        "add.s64 x, %1, 6;\n\tadd.s64 y, %2, 6;\n\tadd.u32 i, %3, 0x60000030;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], x, y, i, [%4], [%5], 1;\n\t"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%7];\n\t"
        "@r tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%8];\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate), "r"(bar_b), "r"(bar_a) : "memory");
}
__device__ __forceinline__ void tmem_st4(uint32_t taddr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(taddr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ void tma_load_2d_elect(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1) {
  asm volatile(
      "{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\t"
      "@q cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];\n\t}"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1) : "memory");
}
__device__ __forceinline__ void tma_load_3d_elect(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2) {
  asm volatile(
      "{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\t"
      "@q cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];\n\t}"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1), "r"(c2) : "memory");
}

// The limit lies behind the abort flag in shared memory: read from there it costs a wait that does not run out nothing; as a kernel parameter
// it took 1.5 to 2 % (matmul 8192 x 8192, 2,048 rows 63.7 -> 64.7 us).
__device__ __forceinline__ long long mx_limit(volatile int* abort_flag) { return (long long)abort_flag[1] << 10; }

// Bounded wait of the issuing warp, in line and decided by votes: a call would have everything that lives across it moved out of
// the uniform registers, and an MMA whose operands are not in those takes 180 cycles to issue instead of 40.
__device__ __forceinline__ bool mbar_wait_uniform(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  const long long t0 = clock64();
  for (uint32_t i = 0; i < kSpinLimit; ++i) {
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    if ((i & 63u) == 63u) {
      const bool over = clock64() - t0 > mx_limit(abort_flag);
      if (__any_sync(0xffffffffu, over || *abort_flag != 0)) break;
    }
  }
  *abort_flag = 1;
  return false;
}

// The other warps'.
static __device__ __noinline__ bool mx_wait_slow(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  return mbar_wait_for(bar, parity, abort_flag, nullptr, mx_limit(abort_flag));
}
__device__ __forceinline__ bool mx_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  return __all_sync(0xffffffffu, mx_wait_slow(bar, parity, abort_flag));
}

// A ring of copies as its producer sees it: wait for the slot, remember the copy; drain() before the CTA may end.
struct RingCursor {
  uint32_t stage = 0, phase = 0, issued = 0, issued_phase = 0;
  __device__ __forceinline__ void sent(uint32_t stages) {
    issued |= 1u << stage;
    issued_phase = (issued_phase & ~(1u << stage)) | (phase << stage);
    if (++stage == stages) { stage = 0; phase ^= 1u; }
  }
  __device__ __forceinline__ void drain(uint32_t full, int stages) const {
    for (int i = 0; i < stages; ++i)
      if (issued & (1u << i)) {
        const long long t0 = clock64();
        while (!mbar_try_wait(full + 8 * i, (issued_phase >> i) & 1u) && clock64() - t0 < kWaitLimitCycles) {}
      }
  }
};

// 16 columns of a warp's 32 channels: 16 rows of y, a run of 32 values each.  dst: this lane's channel in the first row; live: rows
// left.  (Exchanging values among four lanes, so that each writes 8 bytes, costs more instructions than it saves: 850 cycles for 16
// columns instead of 700.)
template <typename T>
__device__ __forceinline__ void store_columns(T* dst, int64_t y_stride, const float* f, int live) {
#pragma unroll
  for (int c = 0; c < 16; ++c) {
    if (c < live) *dst = from_float<T>(f[c]);
    dst += y_stride;
  }
}

// ---- x as eight-bit pieces --------------------------------------------------------------------------
template <typename T> struct PieceCount { static constexpr int N = 5; };
template <> struct PieceCount<__half> { static constexpr int N = 3; };
template <> struct PieceCount<__nv_bfloat16> { static constexpr int N = 2; };

// eight values of a row from k on (a multiple of 8), zero from K on
template <typename T>
__device__ __forceinline__ void load_x(const T* row, int k, int K, int vec, float* f) {
  if (vec && k + 8 <= K) {
    load8(row + k, f);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = k + j < K ? to_float(row[k + j]) : 0.f;
  }
}

// A lane has eight values, four neighbours a block of 32; every lane of the warp takes part.  Piece 0 is the values times the power
// of two that brings the block's largest into [128, 256), rounded to four bits; what is left, at most 2^-5 of the unit above, times
// 32, is the next piece's input.  put(piece, eight codes, scale byte).
template <int PIECES, typename F>
__device__ __forceinline__ void to_pieces(float* f, F put) {
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(f[j]) & 0x7FFFFFFFu);
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
  const uint32_t e = top >> 23;
  const bool dead = e == 255;                      // a NaN or an infinity: scale byte 255 makes the block NaN
  uint32_t s = dead ? 255u : e < 7 ? 0u : e - 7;
  float up = mx_inverse_scale(s);
#pragma unroll
  for (int q = 0; q < PIECES; ++q) {
    uint32_t out[2] = {0u, 0u};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float a = f[2 * j] * up, b = f[2 * j + 1] * up;
      uint16_t c;
      uint32_t back;
      asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(c) : "f"(b), "f"(a));
      asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(back) : "h"(c));
      const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&back));
      f[2 * j] = a - v.x;
      f[2 * j + 1] = b - v.y;
      out[j >> 1] |= (uint32_t)c << ((j & 1) * 16);
    }
    put(q, dead ? make_uint2(0u, 0u) : make_uint2(out[0], out[1]), s);
    if (!dead) {
      const uint32_t next = s < 5 ? 0u : s - 5;
      up = (float)(1u << (s - next));
      s = next;
    }
  }
}

template <int KIND, typename T, bool PROMOTE>
__global__ void __launch_bounds__(kMxTcThreads, 1)
mx_tc_kernel(const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap b_map, const __grid_constant__ CUtensorMap sa_map,
             const __grid_constant__ CUtensorMap sb_map, const __grid_constant__ MxTcParams p, const float* __restrict__ bias,
             T* __restrict__ y, int64_t y_stride) {
  using Kd = MxKind<KIND>;
  constexpr bool CHAINED = KIND == 1;              // behind the pre-pass
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  // Broadcast, so that the compiler sees values that are the same in the whole warp and keeps what the tensor-core instructions take
  // in uniform registers: with plain tid >> 5 and the address as it lies in shared memory an MMA took 180 to 250 cycles to issue.
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int rank = blockIdx.x & (p.cluster - 1);
  const int first = blockIdx.x >> p.cluster_log2, step = gridDim.x >> p.cluster_log2;      // this CTA's tiles
  const int a_stages = p.a_stages, b_stages = p.b_stages, units = p.stack ? 1 : p.pieces;
  const int b_unit = mx_b_unit(p.rows), scale_tile = mx_scale_tile(p);
  const int c_begin = min(p.n_chunks, rank * p.supers_per_split * Kd::CPS);
  const int c_end = min(p.n_chunks, c_begin + p.supers_per_split * Kd::CPS);
  const int chunks = c_end - c_begin, supers = (chunks + Kd::CPS - 1) / Kd::CPS;

  uint8_t* aring = smem;
  uint8_t* bring = aring + a_stages * kMxATile;
  uint8_t* sring = smem + mx_ring_bytes(p);
  uint64_t* bars = reinterpret_cast<uint64_t*>(sring + kMxScaleStages * scale_tile);
  const uint32_t a_full = smem_u32(bars), a_empty = a_full + 8 * a_stages;
  const uint32_t b_full = a_empty + 8 * a_stages, b_empty = b_full + 8 * b_stages;
  const uint32_t s_full = b_empty + 8 * b_stages, s_empty = s_full + 8 * kMxScaleStages;    // scale bytes in shared memory
  const uint32_t t_full = s_empty + 8 * kMxScaleStages, t_empty = t_full + 16;              // scale words in tensor memory
  const uint32_t d_full = t_empty + 16, d_empty = d_full + 16;                              // sums
  const uint32_t retired = d_empty + 16;
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(bars + 2 * a_stages + 2 * b_stages + 2 * kMxScaleStages + 10);
  volatile int* s_abort = reinterpret_cast<volatile int*>(s_tmem + 1);

  // warp 0: the first copies leave before the other warps are set up, the scale bytes of the weights before the weights themselves
  RingCursor ar;
  int a_tile = first, a_chunk = c_begin, a_n0 = mx_tile(p, first).n0;
  auto send_a = [&]() {
    tma_fill_2d(smem_u32(aring) + ar.stage * kMxATile, &a_map, a_full + 8 * ar.stage, KIND == 0 ? kMxATile : kMxACopied, a_chunk * 128, a_n0);
    ar.sent(a_stages);
    if (++a_chunk == c_end) {
      a_chunk = c_begin;
      a_tile += step;
      a_n0 = mx_tile(p, a_tile).n0;
    }
  };
  if (warp == 0) {
    // arrivals: four warps for scale bytes read and words written, eight for sums read, one for everything else
    const int rings = 2 * (a_stages + b_stages) + kMxScaleStages;
    for (int i = lane; i < rings + kMxScaleStages + 9; i += 32)
      mbar_init(a_full + 8 * i, i >= rings && i < rings + kMxScaleStages + 2 ? 4 : i >= rings + kMxScaleStages + 6 && i < rings + kMxScaleStages + 8 ? 8 : 1);
    if (lane == 0) { s_abort[0] = 0; s_abort[1] = p.limit; }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncwarp();
    if (chunks > 0 && first < p.tiles) tma_fill_2d(smem_u32(sring), &sa_map, s_full, (uint32_t)((128 + (p.stack ? p.rows : mx_tile(p, first).Mt * units)) * 16), c_begin / Kd::CPS * 16, a_n0);
    if (chunks > 0)
      for (int i = 0; i < 2 && a_tile < p.tiles; ++i) send_a();
  } else if (warp == 1) {
    tmem_alloc(smem_u32(s_tmem), (uint32_t)p.tmem_cols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  // Before a CTA writes into another's shared memory, that one has to have started: arrived here, waited for at the first write.
  if (p.push) asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
  const uint32_t tmem_base = __shfl_sync(0xffffffffu, *s_tmem, 0);
  bool alive = true;

  if (warp == 0) {
    while (chunks > 0 && a_tile < p.tiles) {
      alive = mx_wait(a_empty + 8 * ar.stage, ar.phase ^ 1u, s_abort);
      if (!alive) break;
      send_a();
    }
    ar.drain(a_full, a_stages);
  } else if (warp == 2) {
    if (CHAINED) asm volatile("griddepcontrol.wait;" ::: "memory");
    RingCursor r;
    for (int tile = first; tile < p.tiles && alive; tile += step) {
      const MxTile at = mx_tile(p, tile);
      const int boxes = at.Mt > p.box ? 2 : 1, bytes = p.stack ? b_unit : at.Mt * 128;
      for (int c0 = c_begin; c0 < c_end && alive; c0 += Kd::CPS)
        for (int u = units - 1; u >= 0 && alive; --u)
          for (int c = c0; c < min(c0 + Kd::CPS, c_end); ++c) {
            alive = mx_wait(b_empty + 8 * r.stage, r.phase ^ 1u, s_abort);
            if (!alive) break;
            const uint32_t dst = smem_u32(bring) + r.stage * b_unit;
            tma_fill_3d(dst, &b_map, b_full + 8 * r.stage, (uint32_t)bytes, c * 128, at.m0, u);
            if (boxes == 2) tma_load_3d_elect(dst + p.box * 128, &b_map, b_full + 8 * r.stage, c * 128, at.m0 + p.box, u);
            r.sent(b_stages);
          }
    }
    r.drain(b_full, b_stages);
  } else if (warp == 3) {
    if (CHAINED) asm volatile("griddepcontrol.wait;" ::: "memory");
    RingCursor r;
    for (int tile = first; tile < p.tiles && alive; tile += step) {
      const MxTile at = mx_tile(p, tile);
      const int boxes = at.Mt > p.box ? 2 : 1, bytes = (128 + (p.stack ? p.rows : at.Mt * units)) * 16;
      for (int s = 0; s < supers; ++s) {
        alive = mx_wait(s_empty + 8 * r.stage, r.phase ^ 1u, s_abort);
        if (!alive) break;
        const uint32_t dst = smem_u32(sring) + r.stage * scale_tile, bar = s_full + 8 * r.stage;
        const int byte = (c_begin / Kd::CPS + s) * 16;
        if (tile != first || s != 0) {              // the very first by warp 0
          expect_tx_elect(bar, (uint32_t)bytes);
          tma_load_2d_elect(dst, &sa_map, bar, byte, at.n0);
        }
        for (int u = 0; u < units; ++u)
          for (int b = 0; b < boxes; ++b)
            tma_load_3d_elect(dst + (128 + u * p.b_cols * 32 + b * p.box) * 16, &sb_map, bar, byte, at.m0 + b * p.box, u);
        r.sent(kMxScaleStages);
      }
    }
    r.drain(s_full, kMxScaleStages);
  } else if (warp == 1) {
    // ---- MMA issuer: all 32 lanes converged, one elected lane issues --------------------------------
    // The answer of a look at a barrier takes about a hundred cycles, as long as several narrow MMAs: whether the next step's
    // operands are there is asked before this step's MMAs are issued.
    constexpr uint32_t DESC_HI = (uint32_t)(1024 >> 4) | (1u << 14) | (2u << 29);   // SBO 1024, version 1, 128-byte swizzle
    constexpr uint32_t LBO_FIELD = 1u << 16;
    // operand types, scales in powers of two, M = 128; N with each tile
    const uint32_t types = (KIND == 0 ? (1u << 7) | (1u << 10) : (5u << 7)) | (1u << 23) | (1u << 27);
    // The smallest pieces come first: while they are added up the sums are small, and so is what the additions drop.
    uint32_t as = 0, aph = 0, bs = 0, bph = 0, sets = 0, done = 0;               // sets, done: of all tiles so far
    bool ready = false, t_ready = false;
    for (int tile = first; tile < p.tiles && alive; tile += step, ++done) {
      const uint32_t idesc = types | ((uint32_t)((tile < p.full ? p.rows : p.Mt / 2) >> 3) << 17);
      const uint32_t db = p.d_bufs == 2 ? done & 1 : 0, dph = (p.d_bufs == 2 ? done >> 1 : done) & 1;
      if (!PROMOTE && supers > 0) alive = mbar_wait_uniform(d_empty + 8 * db, dph ^ 1u, s_abort);
      for (int s = 0; s < supers && alive; ++s, ++sets) {
        const uint32_t tb = sets & 1, tph = (sets >> 1) & 1;
        uint32_t accumulate = !PROMOTE && s > 0;
        if (PROMOTE) alive = mbar_wait_uniform(d_empty + 8 * tb, tph ^ 1u, s_abort);
        if (!t_ready) alive = alive && mbar_wait_uniform(t_full + 8 * tb, tph, s_abort);
        if (!alive) break;
        t_ready = false;
        const uint32_t d = tmem_base + (PROMOTE ? tb : db) * p.rows;
        const uint32_t sf = tmem_base + p.sf_col + tb * 4 * p.sf_group;
        const int n = min(Kd::CPS, chunks - s * Kd::CPS);
        for (int u = units - 1; u >= 0 && alive; --u) {
          uint32_t at = as, atph = aph;
          for (int cc = 0; cc < n; ++cc) {
            if (!ready) {
              alive = mbar_wait_uniform(a_full + 8 * at, atph, s_abort) && mbar_wait_uniform(b_full + 8 * bs, bph, s_abort);
              if (!alive) break;
            }
            tc_fence_after();
            const uint64_t adesc = ((uint64_t)DESC_HI << 32) | (uint64_t)(((smem_u32(aring) + at * kMxATile) >> 4) | LBO_FIELD);
            const uint64_t bdesc = ((uint64_t)DESC_HI << 32) | (uint64_t)(((smem_u32(bring) + bs * b_unit) >> 4) | LBO_FIELD);
            const uint32_t sfa = sf + (KIND == 0 ? 2 * cc : cc) * p.sf_group, sfb = sfa + 4 + u * p.b_cols;
            const uint32_t b_done = b_empty + 8 * bs, a_done = u == 0 ? a_empty + 8 * at : 0u;
            if (++bs == (uint32_t)b_stages) { bs = 0; bph ^= 1u; }
            if (++at == (uint32_t)a_stages) { at = 0; atph ^= 1u; }
            const bool last = cc + 1 == n;
            if (last && u == 0) { as = at; aph = atph; }
            const uint32_t na = last ? as : at, naph = last ? aph : atph;
            const bool next_ready = mbar_test(a_full + 8 * na, naph) & mbar_test(b_full + 8 * bs, bph);
            const bool next_t = last && u == 0 ? mbar_test(t_full + 8 * (tb ^ 1u), ((sets + 1) >> 1) & 1) : false;
            mx_mma4<KIND>(d, adesc, bdesc, idesc, sfa, sfb, p.sf_group, accumulate, b_done, a_done);
            accumulate = 1;
            ready = __all_sync(0xffffffffu, next_ready);
            t_ready = __all_sync(0xffffffffu, next_t);
          }
        }
        if (!alive) break;
        umma_commit(t_empty + 8 * tb);
        if (PROMOTE || s + 1 == supers) umma_commit(d_full + 8 * (PROMOTE ? tb : db));
      }
    }
    if (!alive) {                                  // what was issued must end before the CTA does
      umma_commit(retired);
      const long long t0 = clock64();
      while (!mbar_try_wait(retired, 0) && clock64() - t0 < kWaitLimitCycles) {}
    }
  } else if (warp < 8) {
    // ---- scale bytes -> tensor memory ----------------------------------------------------------------
    const uint32_t quarter = (uint32_t)(warp & 3) * 32;
    const int cols = p.b_cols * units;
    const int sets = first < p.tiles ? ((p.tiles - 1 - first) / step + 1) * supers : 0;
    uint32_t stage = 0, phase = 0;
    for (int s = 0; s < sets; ++s) {
      const uint32_t tb = s & 1, tph = (s >> 1) & 1;
      alive = mx_wait(s_full + 8 * stage, phase, s_abort) && mx_wait(t_empty + 8 * tb, tph ^ 1u, s_abort);
      if (!alive) break;
      tc_fence_after();
      const uint32_t src = smem_u32(sring) + stage * scale_tile + lane * 16;
      const uint32_t dst = tmem_base + p.sf_col + tb * 4 * p.sf_group + (quarter << 16);
      for (int c = 0; c < 4 + cols; c += 4) {
        const uint4 v0 = lds128(src + (c * 32) * 16), v1 = lds128(src + (c * 32 + 32) * 16), v2 = lds128(src + (c * 32 + 64) * 16),
                    v3 = lds128(src + (c * 32 + 96) * 16);
        tmem_st4(dst + c, v0.x, v1.x, v2.x, v3.x);
        tmem_st4(dst + p.sf_group + c, v0.y, v1.y, v2.y, v3.y);
        tmem_st4(dst + 2 * p.sf_group + c, v0.z, v1.z, v2.z, v3.z);
        tmem_st4(dst + 3 * p.sf_group + c, v0.w, v1.w, v2.w, v3.w);
      }
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(s_empty + 8 * stage);
        if (!p.hold) mbar_arrive(t_full + 8 * tb);
      }
      if (++stage == kMxScaleStages) { stage = 0; phase ^= 1u; }
    }
  } else {
    // ---- sums: lane = output channel, column = row of x --------------------------------------------------
    if (CHAINED) asm volatile("griddepcontrol.wait;" ::: "memory");
    if (p.push) asm volatile("barrier.cluster.wait;" ::: "memory");
    const int ch = (warp & 3) * 32 + lane;
    const int copies = p.stack ? p.pieces : 1;                 // columns that belong to one row of x, Mt apart
    uint32_t sets = 0, done = 0;
    for (int tile = first; tile < p.tiles && alive; tile += step, ++done) {
      const MxTile at = mx_tile(p, tile);
      const int split = (at.Mt / 16 + 1) / 2 * 16;             // columns of the lower four warps
      const int c_first = warp < 12 ? 0 : split, half = warp < 12 ? split : at.Mt - split;
      const uint32_t taddr = tmem_base + ((uint32_t)((warp & 3) * 32) << 16) + c_first;
      float* sums = reinterpret_cast<float*>(smem) + c_first * 128 + ch;
      // push: row r of the tile belongs to CTA r mod cluster, which gets a copy from every CTA: [CTA][row / cluster][128]
      const uint32_t mine = smem_u32(smem) + mx_ring_bytes(p) - p.push + ((rank * p.Mt) >> p.cluster_log2) * 512 + ch * 4;
      auto push = [&](int r, float v) {
        uint32_t to;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(mine + (uint32_t)(r >> p.cluster_log2) * 512), "r"(r & (p.cluster - 1)));
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to), "f"(v) : "memory");
      };
      const int n = at.n0 + ch, m0 = at.m0 + c_first;
      const bool direct = p.cluster == 1;
      const float b = direct && bias && n < p.N ? bias[n] : 0.f;
      const int live = n < p.N ? min(half, p.M - m0) : 0;      // this lane's columns that are rows of x
      T* dst = y + (int64_t)m0 * y_stride + n;
      if (PROMOTE) {
        float acc[64];
#pragma unroll
        for (int i = 0; i < 64; ++i) acc[i] = 0.f;
        for (int s = 0; s < supers; ++s, ++sets) {
          const uint32_t tb = sets & 1, tph = (sets >> 1) & 1;
          alive = mx_wait(d_full + 8 * tb, tph, s_abort);
          if (!alive) break;
          tc_fence_after();
          for (int q = copies - 1; q >= 0; --q) {              // the smallest pieces first
            const uint32_t from = taddr + tb * p.rows + q * p.Mt;
#pragma unroll
            for (int c0 = 0; c0 < 64; c0 += 8) {
              if (c0 >= half) break;
              uint32_t v[8];
              tmem_ld8(from + c0, v);
              tmem_ld_wait();
#pragma unroll
              for (int j = 0; j < 8; ++j) acc[c0 + j] += __uint_as_float(v[j]);
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(d_empty + 8 * tb);
        }
        if (direct) {
#pragma unroll
          for (int c = 0; c < 64; ++c) {
            if (c < live && alive) *dst = from_float<T>(acc[c] + b);
            dst += y_stride;
          }
        } else if (p.push) {
#pragma unroll
          for (int c = 0; c < 32; ++c)                         // Mt is 64 at most
            if (c < half) push(c_first + c, acc[c]);
        } else {
#pragma unroll
          for (int c = 0; c < 64; ++c)
            if (c < half) sums[c * 128] = acc[c];
        }
      } else {
        // Not unrolled: code that a block runs once per tile comes from far away (unrolled, 16 columns took 1,000 cycles).
        const uint32_t db = p.d_bufs == 2 ? done & 1 : 0, dph = (p.d_bufs == 2 ? done >> 1 : done) & 1;
        if (supers > 0) alive = mx_wait(d_full + 8 * db, dph, s_abort);
        if (!alive) break;
        tc_fence_after();
        T* out = dst;
        int left = n < p.N ? p.M - m0 : 0;
#pragma unroll 1
        for (int c0 = 0; c0 < half; c0 += 16) {
          float f[16];
#pragma unroll
          for (int j = 0; j < 16; ++j) f[j] = b;
          if (supers > 0) {
#pragma unroll 1
            for (int q = copies - 1; q >= 0; --q) {
              uint32_t v[16];
              tmem_ld16(taddr + db * p.rows + q * p.Mt + c0, v);
              tmem_ld_wait();
#pragma unroll
              for (int j = 0; j < 16; ++j) f[j] += __uint_as_float(v[j]);
            }
          }
          if (p.push) {
#pragma unroll
            for (int j = 0; j < 16; ++j) push(c_first + c0 + j, f[j]);
          } else if (!direct) {
#pragma unroll
            for (int j = 0; j < 16; ++j) sums[(c0 + j) * 128] = f[j];
          } else {
            store_columns<T>(out, y_stride, f, left);
            out += 16 * y_stride;
            left -= 16;
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(d_empty + 8 * db);
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, (uint32_t)p.tmem_cols);
  }
  if (p.cluster == 1) {
    if (*s_abort) {                                // a wait that ran out shows in the result
      for (int tile = first; tile < p.tiles; tile += step) {
        const MxTile at = mx_tile(p, tile);
        for (int i = tid; i < at.Mt * 128; i += kMxTcThreads)
          if (at.m0 + i / 128 < p.M && at.n0 + i % 128 < p.N) y[(int64_t)(at.m0 + i / 128) * y_stride + at.n0 + i % 128] = from_float<T>(__int_as_float(0x7FC00000));
      }
    }
    return;
  }

  // ---- sums of the cluster -> y, a row of 128 channels per warp -------------------------------------
  if (p.push && warp < 8) asm volatile("barrier.cluster.wait;" ::: "memory");
  if (*s_abort) {
    if (p.push) {                                  // the last word on every copy that this CTA owes the others
      const uint32_t mine = smem_u32(smem) + mx_ring_bytes(p) - p.push + ((rank * p.Mt) >> p.cluster_log2) * 512;
      for (int i = tid; i < p.Mt * 128; i += kMxTcThreads) {
        uint32_t to;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(mine + (uint32_t)((i >> 7) >> p.cluster_log2) * 512 + (i & 127) * 4), "r"((i >> 7) & (p.cluster - 1)));
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to), "f"(__int_as_float(0x7FC00000)) : "memory");
      }
    } else {
      for (int i = tid; i < p.Mt * 128; i += kMxTcThreads) reinterpret_cast<float*>(smem)[i] = __int_as_float(0x7FC00000);
    }
  }
  asm volatile("barrier.cluster.arrive.release;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
  if (CHAINED) asm volatile("griddepcontrol.wait;" ::: "memory");
  const MxTile at = mx_tile(p, first);
  const int n0 = at.n0, m0 = at.m0, rows = min(p.Mt, p.M - m0);
  const uint32_t copy = ((uint32_t)p.Mt >> p.cluster_log2) * 512;       // push: bytes of one CTA's sums here
  for (int r = rank + warp * p.cluster; r < rows; r += (kMxTcThreads / 32) * p.cluster) {
    T* dst = y + (int64_t)(m0 + r) * y_stride + n0;
    const uint32_t here = p.push ? smem_u32(smem) + mx_ring_bytes(p) - p.push + (uint32_t)(r >> p.cluster_log2) * 512 : smem_u32(smem) + (uint32_t)r * 512;
    // lane: four neighbouring channels where rows of y start on four values, else every 32nd
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    if (p.y_vec) {
      for (int q = 0; q < p.cluster; ++q) {
        float4 part;
        uint32_t from;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(from) : "r"(here + lane * 16 + (p.push ? q * copy : 0u)), "r"(p.push ? rank : q));
        asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(part.x), "=f"(part.y), "=f"(part.z), "=f"(part.w) : "r"(from) : "memory");
        sum[0] += part.x; sum[1] += part.y; sum[2] += part.z; sum[3] += part.w;
      }
    } else {
      for (int q = 0; q < p.cluster; ++q) {
        float part[4];
        uint32_t from;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(from) : "r"(here + lane * 4 + (p.push ? q * copy : 0u)), "r"(p.push ? rank : q));
#pragma unroll
        for (int j = 0; j < 4; ++j) asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(part[j]) : "r"(from + j * 128) : "memory");
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[j] += part[j];
      }
    }
    const int c0 = p.y_vec ? lane * 4 : lane, c_step = p.y_vec ? 1 : 32;
    if (bias) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (n0 + c0 + j * c_step < p.N) sum[j] += bias[n0 + c0 + j * c_step];
    }
    if (p.y_vec && n0 + c0 + 4 <= p.N) {
      if (sizeof(T) == 4) {
        *reinterpret_cast<float4*>(dst + c0) = make_float4(sum[0], sum[1], sum[2], sum[3]);
      } else {
        T h[4] = {from_float<T>(sum[0]), from_float<T>(sum[1]), from_float<T>(sum[2]), from_float<T>(sum[3])};
        *reinterpret_cast<uint2*>(dst + c0) = *reinterpret_cast<const uint2*>(h);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (n0 + c0 + j * c_step < p.N) dst[c0 + j * c_step] = from_float<T>(sum[j]);
    }
  }
  if (!p.push) {                                   // no CTA leaves while another reads its sums
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
  }
}

// ---------------------------------------------------------------------------------------
// x -> eight-bit pieces, for a large batch
// ---------------------------------------------------------------------------------------
constexpr int kSplitThreads = 256;
constexpr int kSplitWords = 2;               // words of eight values per lane
static_assert(kSplitWords % 2 == 0, "a warp takes whole groups of 512 k, as rows of scale bytes do: it writes all 16 of each");

// A warp takes 512 values of one row, a lane eight at a time.  2,048 x 8192, the profiler's times behind a write of 200 MB, so with old
// lines to write back on the way: bfloat16 18.3 us (68 MB; 18.9 with a 64-bit division for the row), half 22.7, float32 28.9.  With one word
// per lane a small x takes 2.5 us instead of 3.2, and a large one of float32 33.8; but the product's set-up and first loads of weights cover
// the small ones (8192 x 8192, one row 14.0 us either way; 5671 x 609, 37 rows, half 8.7 instead of 8.6).
template <typename T>
__global__ void __launch_bounds__(kSplitThreads)
mx_split_x_kernel(const T* __restrict__ x, int64_t x_stride, int K, int64_t M, int vec, uint32_t segments, FastDiv per_row, int words, int scale_row,
                  uint2* __restrict__ planes, uint8_t* __restrict__ scales) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const uint32_t seg = blockIdx.x * (kSplitThreads / 32) + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (seg >= segments) return;
  const uint32_t row_of = per_row.div(seg);
  const int64_t row = row_of;
  const int word0 = (int)(seg - row_of * per_row.d) * (32 * kSplitWords) + lane;
  float f[kSplitWords][8];
#pragma unroll
  for (int i = 0; i < kSplitWords; ++i) load_x(x + row * x_stride, (word0 + 32 * i) * 8, K, vec, f[i]);
  uint2* out = planes + row * words;
  uint8_t* sr = scales + row * scale_row;
  const int64_t piece_words = M * words, piece_scales = M * scale_row;
#pragma unroll
  for (int i = 0; i < kSplitWords; ++i) {
    const int word = word0 + 32 * i;
    to_pieces<PieceCount<T>::N>(f[i], [&](int q, uint2 codes, uint32_t s) {
      if (word < words) out[q * piece_words + word] = codes;
      if ((lane & 3) == 0 && (word >> 2) < scale_row) sr[q * piece_scales + (word >> 2)] = (uint8_t)s;       // blocks behind K: zero
    });
  }
}

inline int mx_pieces(int dtype) { return dtype == AIQ_DTYPE_F32 ? 5 : dtype == AIQ_DTYPE_F16 ? 3 : 2; }
inline int64_t mx_plane_row(int K) { return ((int64_t)K + 127) / 128 * 128; }

template <typename T>
int x_vec(const MxProduct& p) {
  return p.x && (((uintptr_t)p.x) & 15) == 0 && (p.M == 1 || p.x_stride * (int64_t)sizeof(T) % 16 == 0);
}

template <typename T>
aiq_status_t split_x(const MxProduct& p, uint8_t* planes, uint8_t* scales, cudaStream_t s) {
  const int words = (int)(mx_plane_row(p.K) / 8);
  const uint32_t per_row = (uint32_t)((words + 32 * kSplitWords - 1) / (32 * kSplitWords));
  const uint64_t segments = (uint64_t)p.M * per_row, blocks = (segments + kSplitThreads / 32 - 1) / (kSplitThreads / 32);
  if (segments > 0x7FFFFF00) return set_error(AIQ_ERR_SHAPE, "mx_split_x: M=%d K=%d", p.M, p.K);     // x and its pieces would be over 1.5 TB
  mx_split_x_kernel<T><<<(unsigned)blocks, kSplitThreads, 0, s>>>(static_cast<const T*>(p.x), p.x_stride, p.K, p.M, x_vec<T>(p), (uint32_t)segments,
                                                                   FastDiv(per_row), words, (int)mx_scale_row_bytes(p.K),
                                                                   reinterpret_cast<uint2*>(planes), scales);
  AIQ_LAUNCH_CHECK("mx_split_x");
  return AIQ_OK;
}

aiq_status_t encode(EncodeTiledFn enc, CUtensorMap* map, CUtensorMapDataType type, const void* base, int rank, const cuuint64_t* dims,
                    const cuuint64_t* strides, const cuuint32_t* box, CUtensorMapSwizzle swizzle) {
  const cuuint32_t ones[3] = {1, 1, 1};
  const CUresult r = enc(map, type, rank, const_cast<void*>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                         CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? AIQ_OK : set_error(AIQ_ERR_CUDA, "cuTensorMapEncodeTiled (microscaled product) failed with code %d", (int)r);
}

// Whether sums leave the accumulator every 512 k.  With 16-bit results they may stay while what the additions drop is little beside the
// result's own rounding.  All-positive sums lose 2^-27 of themselves an MMA: half, 640 channels, 2,100 rows, K = 2^20 (98,304 MMAs) 6.8e-4,
// where half a step is 2.4e-4 or more; K = 2^17 8.4e-5.  The limits keep it under a tenth of half a step: half up to K = 32,768 (both
// microscaled 196,608), bfloat16 up to 262,144 (1,048,576).  Above, tiles are 128 rows wide at most instead of 256: half, 640 channels, 2,100
// rows, K = 2^20 7.4 -> 8.6 ms; 2,048 channels, 520 rows, K = 2^17 0.48 -> 0.76.
template <int KIND, typename T>
bool mx_promote(int K) {
  if (sizeof(T) == 4) return true;
  const int64_t mmas = (int64_t)(KIND == 1 ? PieceCount<T>::N : 1) * K / (KIND == 0 ? 64 : 32);
  return mmas > (std::is_same<T, __half>::value ? 3072 : 16384);
}

thread_local long long mx_expire = 0;          // cycles: the next product of this thread holds an arrival back, 0: none does

template <int KIND, typename T, bool PROMOTE>
aiq_status_t launch_kind(const MxProduct& g, uint8_t* workspace, cudaStream_t s) {
  using Kd = MxKind<KIND>;
  DeviceProps props;
  if (aiq_status_t st = current_device_props(&props)) return st;
  AIQ_ENSURE_DYNAMIC_SMEM((mx_tc_kernel<KIND, T, PROMOTE>), props.smem_optin);
  EncodeTiledFn enc = encode_tiled_fn();
  if (!enc) return set_error(AIQ_ERR_CUDA, "cuTensorMapEncodeTiled is not available from the driver");

  MxTcParams p = {};
  p.N = g.N; p.M = g.M;
  p.limit = (int)((mx_expire ? mx_expire : kWaitLimitCycles) >> 10);
  p.hold = mx_expire != 0;
  p.pieces = KIND == 1 ? PieceCount<T>::N : 1;
  p.n_chunks = (g.K + Kd::CHUNK - 1) / Kd::CHUNK;
  const int n_super = (g.K + kMxSuper - 1) / kMxSuper, row_blocks = (g.N + 127) / 128, n_sms = props.n_sms;
  // Rows of x per tile (Mt): the sums of a tile and the scale words have to fit into 512 columns.
  const int widest = PROMOTE ? 128 : 256, stacked = p.pieces == 1 ? 0 : (PROMOTE ? 160 : 256) / p.pieces / 16 * 16;
  p.stack = g.M <= stacked;
  auto shape = [&](MxTcParams& q, int Mt) {
    q.Mt = Mt;
    q.rows = q.stack ? Mt * q.pieces : Mt;
    q.b_cols = ((q.rows + 31) / 32 + 3) / 4 * 4;
    q.sf_group = 4 + q.b_cols * (q.stack ? 1 : q.pieces);
    q.m_blocks = (g.M + Mt - 1) / Mt;
    const int64_t tiles = (int64_t)row_blocks * q.m_blocks;
    if (tiles > 0x3FFFFFFF) return false;
    q.full = q.tiles = (int)tiles;
    q.box = Mt;
    q.cluster = 1;
    while (q.cluster * 2 <= n_sms / q.tiles && q.cluster * 2 <= n_super && q.cluster < 8) q.cluster *= 2;
    // The tiles behind the last whole round over the SMs, where they are at most half a round, are cut in half.
    const int rest = q.tiles % n_sms;
    if (!q.stack && q.tiles > n_sms && rest > 0 && rest * 2 <= n_sms && Mt % 32 == 0) {
      q.full = q.tiles - rest;
      q.tiles = q.full + 2 * rest;
      q.box = Mt / 2;
    }
    q.d_bufs = PROMOTE || (tiles > n_sms && 2 * q.rows + 8 * q.sf_group <= 512) ? 2 : 1;
    q.sf_col = q.d_bufs * q.rows;
    q.tmem_cols = 32;
    while (q.tmem_cols < q.sf_col + 8 * q.sf_group) q.tmem_cols <<= 1;
    return q.tmem_cols <= 512;
  };
  if (p.stack) {
    if (!shape(p, (g.M + 15) / 16 * 16)) return set_error(AIQ_ERR_SHAPE, "mx_tc: N=%d M=%d", g.N, g.M);
  } else {
    // The width of the tiles decides how evenly they go into rounds over the SMs; a wide tile reads fewer operand bytes per product,
    // a narrow one leaves room for two sets of sums.  On the device, a few calls by themselves (below the power limit), 8192 x 8192, 2,048 rows, Mt 256 | 192 | 160 | 128: both
    // microscaled 65 | 61 | 65 | 68 us, bfloat16 207 | 219 | 227 | 240, half 367 | 351 | 356 | 360; 4096 x 4096, 2,048 rows, both
    // microscaled 23.5 | 21.4 | 21.6 | 23.7; 1,024 rows bfloat16 37 | 44 | 43 | 40 (one round of 128 tiles at 256).
    double best = 0;
    bool found = false;
    for (int Mt = (g.M + 15) / 16 * 16 < widest ? (g.M + 15) / 16 * 16 : widest; Mt >= 64; Mt = (Mt - 1) / 32 * 32) {
      MxTcParams q = p;
      if (!shape(q, Mt)) continue;
      const int rest = q.full == q.tiles ? q.tiles % n_sms : 0;
      const double rounds = q.full == q.tiles ? q.tiles / n_sms + (rest ? 1.0 : 0.0) : q.full / n_sms + 0.55;
      // columns' worth of time: KIND 0 a fixed part, and the sums' way out where it is not covered; KIND 1 the MMAs of at least 160
      const double tile = KIND == 0 ? Mt + 40 + (q.d_bufs == 1 ? 40 : 0) : Mt > 160 ? Mt : 160;
      const double cost = rounds * tile / q.cluster + (q.cluster > 1 ? 25 : 0);
      if (!found || cost < best) { best = cost; p = q; found = true; }
      if (PROMOTE || Mt <= 128) break;
    }
    if (!found) {
      if (!shape(p, g.M < 64 ? (g.M + 15) / 16 * 16 : 64)) return set_error(AIQ_ERR_SHAPE, "mx_tc: N=%d M=%d", g.N, g.M);
    }
  }
  while ((1 << p.cluster_log2) < p.cluster) ++p.cluster_log2;
  p.push = p.cluster > 1 && p.Mt <= 64 ? p.Mt * 512 : 0;       // Mt is a multiple of 16, the cluster has 2, 4 or 8 CTAs
  p.supers_per_split = (n_super + p.cluster - 1) / p.cluster;
  const int chunks = p.supers_per_split * Kd::CPS, units = p.stack ? 1 : p.pieces;
  p.a_stages = units > 1 ? Kd::CPS : 2;                        // the pieces of one set of chunks read the same weights
  p.b_stages = 2;
  auto fits = [&](int a, int b) { MxTcParams t = p; t.a_stages = a; t.b_stages = b; return mx_smem_bytes(t) <= props.smem_optin; };
  if (!fits(p.a_stages, p.b_stages)) return set_error(AIQ_ERR_SHAPE, "mx_tc: %d bytes of shared memory", mx_smem_bytes(p));
  for (bool more = true; more;) {
    const bool a_can = p.a_stages < kMxMaxStages && p.a_stages < chunks && fits(p.a_stages + 1, p.b_stages);
    const bool b_can = p.b_stages < kMxMaxStages * 2 && p.b_stages < chunks * units && fits(p.a_stages, p.b_stages + 1);
    if (a_can && (p.a_stages * units <= p.b_stages || !b_can)) ++p.a_stages;
    else if (b_can) ++p.b_stages;
    else more = false;
  }

  const cuuint64_t w_row = (cuuint64_t)mx_row_bytes(g.K), s_row = (cuuint64_t)mx_scale_row_bytes(g.K), N = g.N, M = g.M;
  CUtensorMap a_map, b_map, sa_map, sb_map;
  {
    const cuuint64_t dims[2] = {KIND == 0 ? w_row : 2 * w_row, N}, strides[1] = {w_row};
    const cuuint32_t box[2] = {128, 128};
    if (aiq_status_t st = encode(enc, &a_map, KIND == 0 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_16U4_ALIGN16B, g.w_codes, 2,
                                 dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B)) return st;
    const cuuint64_t sdims[2] = {s_row, N}, sstrides[1] = {s_row};
    const cuuint32_t sbox[2] = {16, 128};
    if (aiq_status_t st = encode(enc, &sa_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, g.w_scales, 2, sdims, sstrides, sbox, CU_TENSOR_MAP_SWIZZLE_NONE))
      return st;
  }
  {
    const cuuint64_t x_row = KIND == 0 ? w_row : (cuuint64_t)mx_plane_row(g.K), P = p.pieces;
    const uint8_t* codes = KIND == 0 ? g.x_codes : workspace;

    const uint8_t* scales = KIND == 0 ? g.x_scales : workspace + P * M * x_row;
    const cuuint64_t dims[3] = {x_row, M, P}, strides[2] = {x_row, x_row * M};
    const cuuint32_t box[3] = {128, (cuuint32_t)p.box, (cuuint32_t)(p.stack ? P : 1)};
    if (aiq_status_t st = encode(enc, &b_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, codes, 3, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B)) return st;
    const cuuint64_t sdims[3] = {s_row, M, P}, sstrides[2] = {s_row, s_row * M};
    const cuuint32_t sbox[3] = {16, (cuuint32_t)p.box, (cuuint32_t)(p.stack ? P : 1)};
    if (aiq_status_t st = encode(enc, &sb_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, scales, 3, sdims, sstrides, sbox, CU_TENSOR_MAP_SWIZZLE_NONE))
      return st;
  }
  const int y_step = 4 * (int)sizeof(T);                       // bytes a lane writes
  p.y_vec = (((uintptr_t)g.y) % y_step) == 0 && (g.M == 1 || g.y_stride * (int64_t)sizeof(T) % y_step == 0);
  LaunchScope scope(AIQ_KERNEL_QLINEAR, s, 2.0 * g.M * g.N * g.K,
                    (double)(g.N + (KIND == 0 ? g.M : 0)) * (w_row + s_row) + sizeof(T) * (double)g.M * (g.N + (KIND == 1 ? g.K : 0)));
  if (KIND == 1)
    if (aiq_status_t st = split_x<T>(g, workspace, workspace + (size_t)p.pieces * M * mx_plane_row(g.K), s)) return st;
  // The CTAs of a cluster wait for one another, and each waits for tensor memory, for as long as another CTA on its SM holds it.  If that
  // one belonged to a cluster of another stream with a CTA in the same position elsewhere, neither would ever go on.  So a CTA of a
  // cluster has its SM to itself: it asks for all of the shared memory.
  const size_t smem = p.cluster > 1 ? (size_t)props.smem_optin : (size_t)mx_smem_bytes(p);
  const int grid = p.cluster > 1 || p.tiles < n_sms ? p.tiles * p.cluster : n_sms;
  AIQ_CUDA_TRY(launch_chained_cluster(KIND == 1, p.cluster, mx_tc_kernel<KIND, T, PROMOTE>, dim3(grid), dim3(kMxTcThreads), smem, s, a_map, b_map, sa_map, sb_map, p,
                                      g.bias, static_cast<T*>(g.y), g.y_stride));
  AIQ_LAUNCH_CHECK("mx_tc");
  return AIQ_OK;
}

template <int KIND, typename T>
aiq_status_t launch_kind(const MxProduct& g, uint8_t* workspace, cudaStream_t s) {
  if constexpr (sizeof(T) == 2)
    if (!mx_promote<KIND, T>(g.K)) return launch_kind<KIND, T, false>(g, workspace, s);
  return launch_kind<KIND, T, true>(g, workspace, s);
}

}  // namespace

size_t mx_tc_workspace_bytes(int K, int M, int dtype) {
  return align_up((size_t)mx_pieces(dtype) * M * (size_t)(mx_plane_row(K) + mx_scale_row_bytes(K)), 16);
}

void mx_tc_expire_next(int64_t limit_cycles) { mx_expire = limit_cycles; }

aiq_status_t launch_mx_product_tc(const MxProduct& p, void* workspace, cudaStream_t s) {
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  struct Once { ~Once() { mx_expire = 0; } } once;
  switch (p.dtype) {
    case AIQ_DTYPE_F32: return p.x ? launch_kind<1, float>(p, ws, s) : launch_kind<0, float>(p, ws, s);
    case AIQ_DTYPE_F16: return p.x ? launch_kind<1, __half>(p, ws, s) : launch_kind<0, __half>(p, ws, s);
    default: return p.x ? launch_kind<1, __nv_bfloat16>(p, ws, s) : launch_kind<0, __nv_bfloat16>(p, ws, s);
  }
}

}  // namespace aiq
