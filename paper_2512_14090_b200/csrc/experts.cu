// A layer of experts: which experts a token goes to, the plan that sorts (token, expert) pairs by expert, and the weighted sum of what comes back.
#include <float.h>

#include "mx.cuh"

namespace aiq {
namespace {

constexpr int kMostExperts = 1024;
constexpr int kMostTopK = 31;                    // a warp's lanes hold the chosen and the first that is not
constexpr int kMostGroups = 32;

// ---------------------------------------------------------------------------------------
// the plan
// ---------------------------------------------------------------------------------------
// int32 words, each part on 16 bytes:
//   header     rows in all, blocks of rows, T, plan_kind(k, E): what a plan of other sizes, or none, is told by
//   offsets    [E + 1]  first row of each expert; the last is the number of rows
//   slots      [T k]    row -> t k + j; -1 behind the last row
//   positions  [T k]    t k + j -> row; -1 where token t has no expert in place j
//   blocks     ExpertBlock, of `width` rows
//   counts     [token blocks][E, rounded up to even], 16 bits: pairs of each expert in a token block (between the two launches of a large plan)
struct PlanLayout {
  int64_t offsets, slots, positions, blocks, counts, words;
  int pairs, width, blocks_most, token_blocks, block_tokens;
};
constexpr int kMostPairs = 65535;                // of a token block
__host__ __device__ inline int plan_kind(int top_k, int E) { return 0x41000000 | top_k << 16 | E; }
// Up to here one thread block does everything.  Choices and plan, in one launch and in two, calls in a graph: 16 tokens among 256 experts 7.9 us and 9.2, among
// 32 experts 6.2 and 8.2; 32 tokens 10.4 and 10.2, 5.6 and 8.1; 64 tokens among 256 experts 15.5 and 10.4.
constexpr int kOneBlockTokens = 16;
constexpr int kPlanThreads = 1024;
constexpr int kTokenBlocks = 148;                // as many as a B200 has SMs: a plan's size is asked for without a device; with up to kMostPairs each

PlanLayout plan_layout(int T, int top_k, int E) {
  PlanLayout l = {};
  l.pairs = T * top_k;
  // Rows per block: twice an expert's share, as long as it gets that many tokens.
  const int share = (l.pairs + E - 1) / E;
  l.width = 16;
  while (l.width < 128 && l.width / 2 < share && l.width < T) l.width *= 2;      // (twice the share may be 2^31)
  l.blocks_most = l.pairs / l.width + (l.pairs < E ? l.pairs : E);
  const int even = (T + kTokenBlocks - 1) / kTokenBlocks;
  l.block_tokens = T <= kOneBlockTokens ? T : even < 16 ? 16 : even;
  if (l.block_tokens > kMostPairs / top_k) l.block_tokens = kMostPairs / top_k;
  l.token_blocks = (T + l.block_tokens - 1) / l.block_tokens;
  auto part = [&](int64_t words) { const int64_t at = l.words; l.words += (words + 3) / 4 * 4; return at; };
  part(4);
  l.offsets = part(E + 1);
  l.slots = part(l.pairs);
  l.positions = part(l.pairs);
  l.blocks = part(4ll * l.blocks_most);
  l.counts = part(l.token_blocks > 1 ? (int64_t)l.token_blocks * ((E + 1) / 2) : 0);
  return l;
}

struct PlanParams {
  int T, top_k, E, pairs, width, token_blocks, block_tokens;
  int *header, *offsets, *slots, *positions, *counts;
  ExpertBlock* blocks;
};
PlanParams plan_params(const PlanLayout& l, int T, int top_k, int E, void* plan) {
  int* w = static_cast<int*>(plan);
  return PlanParams{T, top_k, E, l.pairs, l.width, l.token_blocks, l.block_tokens,
                    w, w + l.offsets, w + l.slots, w + l.positions, w + l.counts, reinterpret_cast<ExpertBlock*>(w + l.blocks)};
}

// Exclusive prefix sums of v[0 .. n) (pairs of numbers) in shared memory by one thread block; v[n] gets the sums.  part: 32 pairs.
__device__ void block_scan(int2* v, int n, int2* part) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
  int2 carry = make_int2(0, 0);
  for (int base = 0; base < n; base += blockDim.x) {
    const int i = base + tid;
    const int2 mine = i < n ? v[i] : make_int2(0, 0);
    int2 sum = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, sum.x, o), y = __shfl_up_sync(0xffffffffu, sum.y, o);
      if (lane >= o) { sum.x += x; sum.y += y; }
    }
    if (lane == 31) part[warp] = sum;
    __syncthreads();
    const int2 other = lane < warps ? part[lane] : make_int2(0, 0);
    const int before_x = __reduce_add_sync(0xffffffffu, lane < warp ? other.x : 0), before_y = __reduce_add_sync(0xffffffffu, lane < warp ? other.y : 0);
    const int all_x = __reduce_add_sync(0xffffffffu, other.x), all_y = __reduce_add_sync(0xffffffffu, other.y);
    if (i < n) v[i] = make_int2(carry.x + before_x + sum.x - mine.x, carry.y + before_y + sum.y - mine.y);
    carry.x += all_x; carry.y += all_y;
    if (base + (int)blockDim.x < n) __syncthreads();
  }
  if (tid == 0) v[n] = carry;
  __syncthreads();
}

// a token block's counts to where the second launch reads them
__device__ __forceinline__ void put_counts(const PlanParams& p, int b, const int* count) {
  const int words = (p.E + 1) / 2;
  for (int w = threadIdx.x; w < words; w += blockDim.x)
    p.counts[(int64_t)b * words + w] = count[2 * w] | (2 * w + 1 < p.E ? count[2 * w + 1] << 16 : 0);
}
__device__ __forceinline__ void write_header(const PlanParams& p, int rows, int blocks) {
  *reinterpret_cast<int4*>(p.header) = make_int4(rows, blocks, p.T, plan_kind(p.top_k, p.E));
}

// where `next` starts, on 16 bytes
__host__ __device__ inline int plan_next(int E, int threads) { return (2 * (E + 1) + 64 + E + threads + 3) / 4 * 4; }

__host__ __device__ inline size_t plan_smem(int E, int warps) { return sizeof(int) * ((size_t)plan_next(E, 32 * warps) + (size_t)warps * (E + 1)); }

// The share of thread block `b` in the plan.  ids: global or shared, of its tokens.  In shared memory: at[E + 1], the experts' first rows and
// first blocks of rows; next[warps][E], where each warp's next pair of an expert goes.
// count(at, before, scratch) fills in {pairs, blocks of rows} of every expert, and its pairs in the token blocks before this one; scratch: `next`, of 32 warps, and
// a little more.
template <typename F>
__device__ void plan_share(const PlanParams& p, int b, const int* ids, int* smem, F count) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
  int2* at = reinterpret_cast<int2*>(smem);
  int2* part = at + p.E + 1;
  int* before = reinterpret_cast<int*>(part + 32);
  int* quarters = before + p.E;
  int* next = smem + plan_next(p.E, blockDim.x);
  count(at, before, next);                         // (in the second launch of two, this waits for the first)
  for (int i = tid; i < warps * p.E; i += blockDim.x) next[i] = 0;
  __syncthreads();
  // each warp has a run of the block's pairs, in order
  const int slot0 = b * p.block_tokens * p.top_k, pairs = min(p.T - b * p.block_tokens, p.block_tokens) * p.top_k;
  const int run = (pairs + warps * 32 - 1) / (warps * 32) * 32, begin = min(pairs, warp * run), end = min(pairs, begin + run);
  for (int i = begin + lane; i < end; i += 32) {
    const int e = ids[i];
    if ((unsigned)e < (unsigned)p.E) atomicAdd(next + warp * p.E + e, 1);
  }
  block_scan(at, p.E, part);
  // warps' counts to where their first pair goes: four threads an expert, each for a quarter of the warps
  const int quarter = (warps + 3) / 4, w0 = tid / (blockDim.x / 4) * quarter, w1 = min(warps, w0 + quarter);
  for (int e0 = 0; e0 < p.E; e0 += blockDim.x / 4) {
    const int e = e0 + tid % (blockDim.x / 4);
    int sum = 0;
    if (e < p.E) {
#pragma unroll 8
      for (int w = w0; w < w1; ++w) sum += next[w * p.E + e];
      quarters[tid] = sum;
    }
    __syncthreads();
    if (e < p.E) {
      int row = at[e].x + before[e];
      for (int q = tid % (blockDim.x / 4); q < tid; q += blockDim.x / 4) row += quarters[q];
#pragma unroll 8
      for (int w = w0; w < w1; ++w) {
        const int n = next[w * p.E + e];
        next[w * p.E + e] = row;
        row += n;
      }
    }
    __syncthreads();
  }
  for (int i0 = begin; i0 < end; i0 += 32) {
    const int i = i0 + lane, e = i < end ? ids[i] : -1;
    const bool some = (unsigned)e < (unsigned)p.E;
    const uint32_t same = __match_any_sync(0xffffffffu, some ? e : -1);
    int row = -1;
    if (some) row = next[warp * p.E + e] + __popc(same & ((1u << lane) - 1u));
    __syncwarp();
    if (some && (same >> lane) == 1u) next[warp * p.E + e] = row + 1;        // the last of them
    __syncwarp();
    if (i < end) p.positions[slot0 + i] = row;
    if (some) p.slots[row] = slot0 + i;
  }
  // what is left is shared out over the thread blocks
  const int rows = at[p.E].x, blocks = at[p.E].y, stride = p.token_blocks * blockDim.x, mine = b * blockDim.x + tid;
  for (int i = rows + mine; i < p.pairs; i += stride) p.slots[i] = -1;
  for (int i = mine; i <= p.E; i += stride) p.offsets[i] = at[i].x;
  for (int i = mine; i < blocks; i += stride) {
    int lo = 0, hi = p.E - 1;                      // the last expert whose first block is i or before
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (at[mid].y <= i) lo = mid; else hi = mid - 1;
    }
    p.blocks[i] = ExpertBlock{lo, at[lo].x, at[lo + 1].x - at[lo].x, at[lo].y};
  }
  if (mine == 0) write_header(p, rows, blocks);
}

// A small plan, by one thread block: everything is counted by comparing with every pair.  ids: in shared memory, behind the last pair up to a
// multiple of four anything.  smem: two words a pair.
constexpr int kFewPairs = 64;
__device__ void plan_few(const PlanParams& p, const int* ids, int* smem) {
  const int tid = threadIdx.x;
  int* expert = smem;                              // of the first pair of an expert; else E
  int* blocks_of = smem + p.pairs;
  for (int i = tid; i < p.pairs; i += blockDim.x) {
    const int e = ids[i];
    const bool some = (unsigned)e < (unsigned)p.E;
    int less = 0, before = 0, same = 0;
    for (int j = 0; j < p.pairs; ++j) {
      const unsigned o = ids[j];
      less += o < (unsigned)e;
      same += o == (unsigned)e;
      before += o == (unsigned)e && j < i;
    }
    const int row = less + before;
    p.positions[i] = some ? row : -1;
    if (some) p.slots[row] = i;
    expert[i] = some && before == 0 ? e : p.E;
    blocks_of[i] = some && before == 0 ? (same + p.width - 1) / p.width : 0;
  }
  __syncthreads();
  for (int i = tid; i <= p.E; i += blockDim.x) {   // (all of them for i = E)
    int rows = 0;
    for (int j = 0; j < p.pairs; ++j) rows += (unsigned)ids[j] < (unsigned)i;
    p.offsets[i] = rows;
    if (i == p.E) {
      int blocks = 0;
      for (int j = 0; j < p.pairs; ++j) blocks += blocks_of[j];
      write_header(p, rows, blocks);
      for (int j = rows; j < p.pairs; ++j) p.slots[j] = -1;
    }
  }
  for (int i = tid; i < p.pairs; i += blockDim.x) {
    const int e = expert[i];
    if (e == p.E) continue;
    int first = 0, begin = 0, same = 0;
    for (int j = 0; j < p.pairs; ++j) {
      first += expert[j] < e ? blocks_of[j] : 0;
      begin += (unsigned)ids[j] < (unsigned)e;
      same += ids[j] == e;
    }
    for (int j = 0; j < blocks_of[i]; ++j) p.blocks[first + j] = ExpertBlock{e, begin, same, first};
  }
}
// All of a plan by one thread block, ids in shared memory.
__device__ void plan_whole(const PlanParams& p, const int* ids, int* smem) {
  if (p.pairs <= kFewPairs) {
    plan_few(p, ids, smem);
  } else {
    plan_share(p, 0, ids, smem, [&](int2* at, int* before, int*) {
      int* count = reinterpret_cast<int*>(at) + plan_smem(p.E, blockDim.x >> 5) / sizeof(int);
      for (int e = threadIdx.x; e < p.E; e += blockDim.x) count[e] = 0;
      __syncthreads();
      for (int i = threadIdx.x; i < p.pairs; i += blockDim.x)
        if ((unsigned)ids[i] < (unsigned)p.E) atomicAdd(count + ids[i], 1);
      __syncthreads();
      for (int e = threadIdx.x; e < p.E; e += blockDim.x) {
        at[e] = make_int2(count[e], (count[e] + p.width - 1) / p.width);
        before[e] = 0;
      }
    });
  }
}
inline size_t plan_whole_smem(const PlanParams& p, int warps) {
  return p.pairs <= kFewPairs ? sizeof(int) * 2 * (size_t)p.pairs : plan_smem(p.E, warps) + sizeof(int) * (size_t)p.E;
}

// The second launch of a large plan.  A thread adds up two experts' counts of every so-manieth token block: coalesced, and all on their way together.
// (Counts beside each other for an expert, so that a warp takes them at once, are written to as many lines as there are: 15 -> 18 us.)
__global__ void __launch_bounds__(kPlanThreads)
expert_plan_kernel(const __grid_constant__ PlanParams p, const int* ids) {
  extern __shared__ int2 plan_arrays[];
  chain_release();
  const int b = blockIdx.x;
  plan_share(p, b, ids + (int64_t)b * p.block_tokens * p.top_k, reinterpret_cast<int*>(plan_arrays), [&](int2* at, int* before, int* scratch) {
    const int words = (p.E + 1) / 2, groups = min(16, (int)blockDim.x / words), w = threadIdx.x % words, g = threadIdx.x / words;
    chain_wait();
    if (g < groups) {
      int all[2] = {0, 0}, earlier[2] = {0, 0};
#pragma unroll 8
      for (int q = g; q < p.token_blocks; q += groups) {
        const uint32_t two = p.counts[(int64_t)q * words + w], early = q < b ? two : 0u;
        all[0] += two & 0xFFFFu; all[1] += two >> 16;
        earlier[0] += early & 0xFFFFu; earlier[1] += early >> 16;
      }
      // scratch: [groups][words] of all four
      *reinterpret_cast<int4*>(scratch + (g * words + w) * 4) = make_int4(all[0], all[1], earlier[0], earlier[1]);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < p.E; e += blockDim.x) {
      int total = 0, sum = 0;
      for (int i = 0; i < groups; ++i) {
        const int* from = scratch + (i * words + (e >> 1)) * 4 + (e & 1);
        total += from[0];
        sum += from[2];
      }
      at[e] = make_int2(total, (total + p.width - 1) / p.width);
      before[e] = sum;
    }
    __syncthreads();
  });
}

// Given ids: their counts (first launch of a large plan), or all of a small one.
__global__ void __launch_bounds__(kPlanThreads)
expert_count_kernel(const __grid_constant__ PlanParams p, const int* ids) {
  extern __shared__ int2 plan_arrays[];
  int* smem = reinterpret_cast<int*>(plan_arrays);
  chain_release();
  chain_wait();
  const int b = blockIdx.x, slot0 = b * p.block_tokens * p.top_k, pairs = min(p.T - b * p.block_tokens, p.block_tokens) * p.top_k;
  if (p.token_blocks == 1) {
    for (int i = threadIdx.x; i < pairs; i += blockDim.x) smem[i] = ids[i];
    __syncthreads();
    plan_whole(p, smem, smem + ((p.pairs + 3) & ~3));
    return;
  }
  for (int e = threadIdx.x; e < p.E; e += blockDim.x) smem[e] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < pairs; i += blockDim.x) {
    const int e = ids[slot0 + i];
    if ((unsigned)e < (unsigned)p.E) atomicAdd(smem + e, 1);
  }
  __syncthreads();
  put_counts(p, b, smem);
}

// ---------------------------------------------------------------------------------------
// routing
// ---------------------------------------------------------------------------------------
struct RouteParams {
  const void* logits;
  int64_t stride;
  const float* bias;
  int sigmoid, groups, top_groups, group_best, renormalise;
  int group_size, group_shift;                     // 2^group_shift of a token's lanes score one group
  int run_shift;                                   // groups are 2^run_shift runs of eight, up to eight; else -1
  FastDiv group_of{1};
  int vec;                                         // rows are loaded eight logits at a time
  float scale;
  int* ids;
  float* weights;
  int with_plan;
};

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// over the L lanes of a token
template <int L, typename F, typename S>
__device__ __forceinline__ S join(S v, F f) {
#pragma unroll
  for (int o = 1; o < L; o <<= 1) v = f(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
template <int L> __device__ __forceinline__ float sum_of(float v) { return join<L>(v, [](float a, float b) { return a + b; }); }
template <int L> __device__ __forceinline__ float most_of(float v) { return join<L>(v, [](float a, float b) { return fmaxf(a, b); }); }
template <int L> __device__ __forceinline__ float least_of(float v) { return join<L>(v, [](float a, float b) { return fminf(a, b); }); }

// exp(x) by 2^x as the hardware has it
__device__ __forceinline__ float fast_exp(float v) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v * 1.4426950408889634f));
  return r;
}

__device__ __forceinline__ void larger_first(float& a, float& b) {
  const float x = a;
  a = fmaxf(x, b);
  b = fminf(x, b);
}
__device__ __forceinline__ void sort8(float (&v)[8]) {        // largest first: Batcher's odd-even merge sort
#pragma unroll
  for (int p = 1; p < 8; p <<= 1)
#pragma unroll
    for (int q = p; q >= 1; q >>= 1)
#pragma unroll
      for (int j = q % p; j + q < 8; j += 2 * q)
#pragma unroll
        for (int i = 0; i < q; ++i)
          if (j + i + q < 8 && (j + i) / (2 * p) == (j + i + q) / (2 * p)) larger_first(v[j + i], v[j + i + q]);
}
// The K largest of two falling runs, falling, where a[i] has become the larger of a[i] and the other run's [K - 1 - i]
template <int K>
__device__ __forceinline__ void merge_down(float (&a)[K]) {
#pragma unroll
  for (int q = K / 2; q >= 1; q >>= 1)
#pragma unroll
    for (int i = 0; i < K; ++i)
      if (!(i & q)) larger_first(a[i], a[i + q]);
}

struct __align__(16) Candidate {
  float choice, logit, bias;
  int expert;
};
constexpr int kFewTokens = kTokenBlocks * kPlanThreads / 32;       // a warp for each token at once
constexpr int kCandidates = 32;                  // of a token
// words of shared memory of a warp: choices, candidates, their values in 64 bits or before that the groups' scores, the chosen, counts
__host__ __device__ inline int route_row(int E) { return (E + 7) / 8 * 8; }
__host__ __device__ inline int route_warp_words(int E, int L) {
  return 32 / L * (route_row(E) + kCandidates * 4 + kCandidates * 2 + 32) + 4;
}

// Whether float32 tells two choices with a bias apart: by more than `base` for their scores and the rounding of the additions, at the larger one's size.
__device__ __forceinline__ bool apart(float x, float y, float base) { return fabsf(x - y) > base + 0x1p-22f * fmaxf(fabsf(x), fabsf(y)); }

// Where a token has more candidates than places (`many`): one after the other from all, by the comparisons that Router makes.  By itself, so that
// nothing of Router has to lie in memory for it.
template <typename T, int L>
__device__ __noinline__ void one_by_one(const T* row, int E, int top_k, bool sigmoid, const float* bias, float* choice, int* chosen, float top, float base, bool many) {
  const int sub = threadIdx.x & (L - 1);
  double sum = 0;
  if (!sigmoid) {
    for (int e = sub; e < E; e += L) sum += exp((double)to_float(row[e]) - (double)top);
    sum = join<L>(sum, [](double a, double b) { return a + b; });
  }
  auto exact = [&](int e) {
    const double l = to_float(row[e]);
    return (sigmoid ? 1.0 / (1.0 + exp(-l)) : exp(l - (double)top) / sum) + (double)bias[e];
  };
  auto before = [&](int a, int b) {                // experts that may be chosen
    const float x = choice[a], y = choice[b];
    if (!bias || apart(x, y, base)) return x != y ? x > y : a < b;
    if (to_float(row[a]) == to_float(row[b]) && bias[a] == bias[b]) return a < b;
    const double u = exact(a), v = exact(b);
    return u != v ? u > v : a < b;
  };
  for (int j = 0; j < top_k; ++j) {
    int best = -1;
    for (int c = sub; c * 8 < E; c += L)
      for (int e = c * 8; e < min(E, c * 8 + 8); ++e)
        if (choice[e] != -INFINITY && (best < 0 || before(e, best))) best = e;
    for (int o = 1; o < L; o <<= 1) {
      const int other = __shfl_xor_sync(0xffffffffu, best, o);
      if (other >= 0 && (best < 0 || before(other, best))) best = other;
    }
    __syncwarp();
    if (many && sub == 0) {
      if (best >= 0) choice[best] = -INFINITY;
      chosen[j] = best;
    }
    __syncwarp();
  }
}

// L lanes take a token: eight where there are many tokens, so that what is done once for a token is done for four at a time; 32 for the shortest way through
// one.  A lane has every L-th run of eight experts.
//   score of an expert: softmax or logistic function of its logit.  choice: score + bias; without a bias the logit itself, whose order it is.
//   -infinity: not to be chosen.
// The choices go to shared memory.  Each lane keeps the K (a power of two, top_k or more) largest, sorted, by merging sorted runs of eight; three
// exchanges (five) make them the token's.  All experts from the k-th largest on are candidates, which are ranked by comparing each with all.
// Float32 cannot tell choices apart that are closer than their rounding (equal logits and biases give equal choices): what is that close to
// the k-th is a candidate, too, and where two are that close, all candidates are ranked in float64; groups likewise, of which every taken one has to
// be clear of every other.  In steps of 2^-24, scores being at most 1, a logistic function is off by 4.3: by 0.22 for the
// rounding of the exponential's argument and 1 for the exponential (2^-22 of itself), by 3 for 1 + y and the reciprocal; two of them, and the additions of
// the bias, by 2^-20 + 2^-23 |choice|.  A softmax has an exponential (4.8), a sum of up to 1024 and a reciprocal: 2^-18.  A group's sum of two is off by as
// much, its numerators alone by 2^-20; but what counts of a bias is the size of the two choices, 2^-23 (|first| + |second|) for three roundings, of which the
// sum may have nothing left where they cancel.
// Bound by the length of the chain: every warp has one set of tokens, whose choices pass through shared memory five times, and issue is active for 34 % of the
// time.  16,384 tokens among 256 experts, 8 of them, in 8 groups, 22 us (8 MB of logits: 1.3), and 13 for the plan behind it; one token among 32 experts with its
// plan 4.5 us.  (64 registers, for blocks of 1,024 threads: 28 to 100 bytes a thread are spilt.)
template <typename T, int K, int L>
struct Router {
  const RouteParams& r;
  const int E, top_k;
  const float* bias;                               // shared, or nullptr
  float *choice, *group_score, *group_size_of;
  Candidate* candidate;
  double* precise;
  int *chosen, *found;
  const T* row;
  int sub;
  float top;
  double sum64;

  __device__ __forceinline__ float logit(int e) const { return to_float(row[e]); }
  __device__ __forceinline__ float score(float l, float inverse) const {
    return r.sigmoid ? fast_inverse(1.f + fast_exp(-l)) : fast_exp(l - top) * inverse;
  }
  __device__ __forceinline__ double score64(float l) const { return r.sigmoid ? 1.0 / (1.0 + exp(-(double)l)) : exp((double)l - (double)top) / sum64; }
  __device__ __forceinline__ void need64() {
    if (r.sigmoid || __all_sync(0xffffffffu, sum64 != 0.0)) return;
    double s = 0;
#pragma unroll 1
    for (int e = sub; e < E; e += L) s += exp((double)logit(e) - (double)top);
    sum64 = join<L>(s, [](double a, double b) { return a + b; });
  }

  // What a group counts as, of its best two choices (or logits), and the size of what was rounded on the way there.
  __device__ __forceinline__ void put_group(int g, float first, float second) {
    if (r.group_best == 2) {
      if (!bias) {                                 // of the softmax only the numerators: the rest is common to all
        first = first == -INFINITY ? first : score(first, 1.f);
        second = second == -INFINITY ? second : score(second, 1.f);
      }
      if (second == -INFINITY) second = 0.f;
    } else {
      second = 0.f;
    }
    // A finite sum beyond float32's range is the range's end, not the infinity that bars a group; its size is infinite then, so that float64 decides.
    const float most = fabsf(first) < INFINITY ? FLT_MAX : INFINITY;
    group_score[g] = fminf(fmaxf(first + second, -most), most);
    group_size_of[g] = fabsf(first) + fabsf(second);
  }
  // the groups' scores, of what is in `choice`
  __device__ __forceinline__ void score_groups() {
    const int lanes = 1 << r.group_shift, per = L >> r.group_shift, part = sub & (lanes - 1);
    const int begin = r.group_size * part >> r.group_shift, n = (r.group_size * (part + 1) >> r.group_shift) - begin;
    for (int g = sub >> r.group_shift; g < (r.groups + per - 1) / per * per; g += per) {
      float first = -INFINITY, second = -INFINITY;
      if (g < r.groups) {
        const int base = g * r.group_size + begin;
        int at = n > 0 ? (int)(threadIdx.x & 31) % n : 0;           // from different places on: other banks
        for (int i = 0; i < n; ++i) {
          const float v = choice[base + at];
          if (++at == n) at = 0;
          second = fmaxf(second, fminf(first, v));
          first = fmaxf(first, v);
        }
      }
      for (int o = 1; o < lanes; o <<= 1) {
        const float f = __shfl_xor_sync(0xffffffffu, first, o), t = __shfl_xor_sync(0xffffffffu, second, o);
        second = fmaxf(fmaxf(second, t), fminf(first, f));
        first = fmaxf(first, f);
      }
      if (g < r.groups && part == 0) put_group(g, first, second);
    }
  }
  // Groups of 8, 16, 32 or 64: beside each other lie the runs of eight of neighbouring lanes.
  __device__ __forceinline__ void score_groups_of_runs() {
    const int runs = 1 << r.run_shift;
#pragma unroll 1
    for (int c0 = 0; c0 * 8 < E; c0 += L) {
      const float* at = choice + (c0 + sub) * 8;
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = (c0 + sub) * 8 < E ? at[i] : -INFINITY;
      float first[4], second[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        first[i] = fmaxf(v[i], v[i + 4]);
        second[i] = fminf(v[i], v[i + 4]);
      }
#pragma unroll
      for (int n = 2; n >= 1; n >>= 1)
#pragma unroll
        for (int i = 0; i < n; ++i) {
          second[i] = fmaxf(fminf(first[i], first[i + n]), fmaxf(second[i], second[i + n]));
          first[i] = fmaxf(first[i], first[i + n]);
        }
      for (int o = 1; o < runs; o <<= 1) {
        const float f = __shfl_xor_sync(0xffffffffu, first[0], o), t = __shfl_xor_sync(0xffffffffu, second[0], o);
        second[0] = fmaxf(fmaxf(second[0], t), fminf(first[0], f));
        first[0] = fmaxf(first[0], f);
      }
      if ((sub & (runs - 1)) == 0 && (c0 + sub) * 8 < E) put_group((c0 + sub) >> r.run_shift, first[0], second[0]);
    }
  }
  // The groups that are taken, and of them and of the others those that float32 cannot put on either side.
  __device__ __forceinline__ void take_groups(uint32_t* taken, uint32_t* unclear) {
    __syncwarp();
    // A group's score in float64 is not further than this from what it is here.
    const float base = bias && !r.sigmoid ? 0x1p-18f : 0x1p-20f;
    auto off = [&](int g) { return base + 0x1p-22f * group_size_of[g]; };
    uint32_t in = 0;
    float last = INFINITY, next = -INFINITY;       // the least that a taken one, the most that another can be
    for (int g = sub; g < r.groups; g += L) {
      const float mine = group_score[g];
      int rank = 0;
      for (int o = 0; o < r.groups; ++o) {
        const float other = group_score[o];
        rank += other > mine || (other == mine && o < g);
      }
      if (rank < r.top_groups) {
        in |= 1u << g;
        last = fminf(last, mine == INFINITY ? mine : mine - off(g));
      } else {
        next = fmaxf(next, mine == -INFINITY ? mine : mine + off(g));
      }
    }
    *taken = join<L>(in, [](uint32_t a, uint32_t b) { return a | b; });
    *unclear = 0;
    if (!(bias || r.group_best == 2)) return;
    last = least_of<L>(last);
    next = most_of<L>(next);
    const bool clear = next == -INFINITY || last > next;                       // (of this token: its lanes stay with the others of the warp)
    uint32_t near = 0;
    for (int g = sub; g < r.groups; g += L) {
      const float mine = group_score[g];
      if (!clear && mine != -INFINITY && !(in >> g & 1u ? mine - off(g) > next : last > mine + off(g))) near |= 1u << g;
    }
    *unclear = join<L>(near, [](uint32_t a, uint32_t b) { return a | b; });
  }
  // Those again in float64, all lanes of a token at one group: the best of them get the places that the others leave.
  __device__ __forceinline__ uint32_t take_unclear(uint32_t taken, uint32_t unclear) {
    need64();
    __syncwarp();
    for (uint32_t m = unclear; __any_sync(0xffffffffu, m != 0); m &= m - 1) {
      const int g = __ffs(m) - 1;
      double first = -INFINITY, second = -INFINITY;
      if (g >= 0)
        for (int e = g * r.group_size + sub; e < (g + 1) * r.group_size; e += L)
          if (choice[e] != -INFINITY) {
            const double v = score64(logit(e)) + (bias ? (double)bias[e] : 0.0);
            second = fmax(second, fmin(first, v));
            first = fmax(first, v);
          }
#pragma unroll
      for (int o = 1; o < L; o <<= 1) {
        const double f = __shfl_xor_sync(0xffffffffu, first, o), t = __shfl_xor_sync(0xffffffffu, second, o);
        second = fmax(fmax(second, t), fmin(first, f));
        first = fmax(first, f);
      }
      if (g >= 0 && sub == 0) precise[g] = r.group_best == 2 && second != -INFINITY ? first + second : first;
    }
    __syncwarp();
    const int places = r.top_groups - __popc(taken & ~unclear);
    uint32_t in = taken & ~unclear;
    for (uint32_t m = unclear; m; m &= m - 1) {
      const int g = __ffs(m) - 1;
      int rank = 0;
      for (uint32_t o = unclear; o; o &= o - 1) {
        const int other = __ffs(o) - 1;
        rank += precise[other] > precise[g] || (precise[other] == precise[g] && other < g);
      }
      if (rank < places) in |= 1u << g;
    }
    __syncwarp();
    return in;
  }

  // rank by F's order; lanes share out the candidates
  template <typename F>
  __device__ __forceinline__ void rank(int n, F before) {
    for (int i = sub; i < n; i += L) {
      int at = 0;
      for (int j = 0; j < n; ++j) at += before(j, i);
      if (at < top_k) chosen[at] = candidate[i].expert;
    }
  }

  __device__ __forceinline__ void run(int t, bool live, bool bias_nan, int* count, int* ids_shared) {
    constexpr int J = (K + L - 1) / L;                 // chosen experts of a lane
    sum64 = 0;
    // logits to shared memory, their largest
    top = -INFINITY;
#pragma unroll 4
    for (int c = sub; c * 8 < E; c += L) {
      float f[8];
      if (r.vec) {
        load8(row + c * 8, f);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = c * 8 + i < E ? logit(c * 8 + i) : -INFINITY;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max_nan(top, f[i]);
      *reinterpret_cast<float4*>(choice + c * 8) = make_float4(f[0], f[1], f[2], f[3]);
      *reinterpret_cast<float4*>(choice + c * 8 + 4) = make_float4(f[4], f[5], f[6], f[7]);
    }
    top = join<L>(top, max_nan);
    const bool bad = top != top || bias_nan || (!r.sigmoid && top == INFINITY);
    // the softmax's sum, for choices with a bias and for weights that are not made to add up to 1
    float sum = 1.f;
    if (!r.sigmoid && (bias || !r.renormalise)) {
      float part = 0.f;
      for (int c = sub; c * 8 < E; c += L)
#pragma unroll
        for (int i = 0; i < 8; ++i) part += expf(choice[c * 8 + i] - top);
      sum = sum_of<L>(part);
    }
    if (bias) {
      const float inverse = fast_inverse(sum);
#pragma unroll 2
      for (int c = sub; c * 8 < E; c += L) {
        float* at = choice + c * 8;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = at[i] == -INFINITY ? -INFINITY : score(at[i], inverse) + bias[c * 8 + i];
#pragma unroll
        for (int i = 0; i < 8; ++i) at[i] = v[i];
      }
    }
    uint32_t open = 0xffffffffu;
    if (r.groups > 1) {
      __syncwarp();
      if (r.run_shift >= 0) score_groups_of_runs();
      else score_groups();
      uint32_t unclear;
      take_groups(&open, &unclear);
      if (bad || !live) unclear = 0;
      if (__any_sync(0xffffffffu, unclear != 0)) open = take_unclear(open, unclear);
    }
    float a[K];
#pragma unroll
    for (int i = 0; i < K; ++i) a[i] = -INFINITY;
    const bool whole = (r.group_size & 7) == 0;    // eight experts beside each other are of one group
#pragma unroll 1
    for (int c = sub; c * 8 < route_row(E); c += L) {
      float* at = choice + c * 8;
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = at[i];
      if (r.groups > 1) {
        if (whole) {
          const bool on = open >> r.group_of.div(c * 8) & 1u;
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = on ? v[i] : -INFINITY;
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = open >> (r.group_of.div(c * 8 + i) & 31) & 1u ? v[i] : -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) at[i] = v[i];
      }
      sort8(v);
#pragma unroll
      for (int i = 0; i < (K < 8 ? K : 8); ++i) a[K - 1 - i] = fmaxf(a[K - 1 - i], v[i]);
      merge_down<K>(a);
    }
#pragma unroll
    for (int o = 1; o < L; o <<= 1) {
      float other[K];
#pragma unroll
      for (int i = 0; i < K; ++i) other[i] = __shfl_xor_sync(0xffffffffu, a[i], o);
#pragma unroll
      for (int i = 0; i < K; ++i) a[i] = fmaxf(a[i], other[K - 1 - i]);
      merge_down<K>(a);
    }
    float least = a[0];
#pragma unroll
    for (int i = 1; i < K; ++i) least = i < top_k ? a[i] : least;
    const float base = !bias ? 0.f : r.sigmoid ? 0x1p-20f : 0x1p-18f, tolerance = bias ? base + 0x1p-22f * fabsf(least) : 0.f;
    float from = least - tolerance;
    if (!(from == from)) from = least;             // infinities
    if (bad || !live) from = INFINITY;
#pragma unroll
    for (int j = 0; j < J; ++j) chosen[sub + L * j] = -1;
    if (sub == 0) *found = 0;
    __syncwarp();
#pragma unroll 1
    for (int c = sub; c * 8 < E && !bad; c += L) {
      const float* at = choice + c * 8;
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) m |= at[i] >= from && at[i] != -INFINITY ? 1u << i : 0u;
      while (m) {
        const int e = c * 8 + __ffs(m) - 1;
        m &= m - 1;
        const int place = atomicAdd(found, 1);
        if (place < kCandidates) candidate[place] = Candidate{choice[e], logit(e), bias ? bias[e] : 0.f, e};
      }
    }
    __syncwarp();
    int n = *found;
    const bool many = n > kCandidates;
    if (many) n = 0;
    bool near = false;
    rank(n, [&](int j, int i) {
      const Candidate x = candidate[j], y = candidate[i];
      near = near || (bias && !apart(x.choice, y.choice, base) && (x.logit != y.logit || x.bias != y.bias));
      return x.choice > y.choice || (x.choice == y.choice && x.expert < y.expert);
    });
    near = join<L>((int)near, [](int x, int y) { return x | y; });
    if (__any_sync(0xffffffffu, near)) {
      need64();
      if (near) {
        for (int i = sub; i < n; i += L) precise[i] = score64(candidate[i].logit) + (double)candidate[i].bias;
#pragma unroll
        for (int j = 0; j < J; ++j) chosen[sub + L * j] = -1;
      }
      __syncwarp();
      if (near) rank(n, [&](int j, int i) { return precise[j] > precise[i] || (precise[j] == precise[i] && candidate[j].expert < candidate[i].expert); });
    }
    __syncwarp();
    if (__any_sync(0xffffffffu, many)) one_by_one<T, L>(row, E, top_k, r.sigmoid, bias, choice, chosen, top, base, many);
    // weights
    float w[J], high = -INFINITY, part = 0.f;
    int id[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
      id[j] = sub + L * j < top_k ? chosen[sub + L * j] : -1;
      w[j] = id[j] >= 0 ? logit(id[j]) : -INFINITY;
      high = fmaxf(high, w[j]);
    }
    if (r.renormalise) high = most_of<L>(high);
#pragma unroll
    for (int j = 0; j < J; ++j) {
      // Far left of zero logistic functions vanish, but their ratios are those of the exponentials.
      if (r.sigmoid && (!r.renormalise || high >= -40.f)) w[j] = 1.f / (1.f + expf(-w[j]));
      else w[j] = expf(w[j] - (r.renormalise ? high : top));
      part += id[j] >= 0 ? w[j] : 0.f;
    }
    if (r.renormalise) sum = sum_of<L>(part);
    else if (r.sigmoid) sum = 1.f;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int place = sub + L * j;
      if (place >= top_k || !live) continue;
      r.ids[(int64_t)t * top_k + place] = id[j];
      r.weights[(int64_t)t * top_k + place] = bad ? __int_as_float(0x7FC00000) : id[j] >= 0 ? w[j] / sum * r.scale : 0.f;
      if (ids_shared) ids_shared[place] = id[j];
      if (count && id[j] >= 0) atomicAdd(count + id[j], 1);
    }
    __syncwarp();
  }
};

template <typename T, int K, int L>
__global__ void __launch_bounds__(kPlanThreads)
route_experts_kernel(const __grid_constant__ RouteParams r, const __grid_constant__ PlanParams p) {
  extern __shared__ __align__(16) float route_smem[];
  chain_release();
  chain_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5, b = blockIdx.x, token = lane / L;
  // every warp's arrays; biases; the plan's arrays; counts or ids
  const int row = route_row(p.E);
  float* mine = route_smem + warp * route_warp_words(p.E, L);
  float* bias = route_smem + warps * route_warp_words(p.E, L);
  int* plan = reinterpret_cast<int*>(bias + row);
  const bool all = r.with_plan && p.token_blocks == 1;
  const int t0 = b * p.block_tokens, tokens = min(p.T - t0, p.block_tokens);
  bool nan = false;
  if (r.bias)
    for (int e = threadIdx.x; e < row; e += blockDim.x) {
      bias[e] = e < p.E ? r.bias[e] : 0.f;
      nan = nan || bias[e] != bias[e];
    }
  int* ids = plan;
  int* count = nullptr;
  if (all) {
    plan = ids + ((p.pairs + 3) & ~3);
  } else if (r.with_plan) {
    count = plan;
    for (int e = threadIdx.x; e < p.E; e += blockDim.x) count[e] = 0;
  }
  nan = __syncthreads_or(nan);
  float* at = mine + (32 / L) * row;
  Router<T, K, L> router{r, p.E, p.top_k, r.bias ? bias : nullptr, mine + token * row};
  router.sub = lane & (L - 1);
  router.candidate = reinterpret_cast<Candidate*>(at) + token * kCandidates;
  at += (32 / L) * kCandidates * 4;
  static_assert(kMostGroups <= kCandidates, "two words for each group lie where the candidates' values in 64 bits do");
  router.precise = reinterpret_cast<double*>(at) + token * kCandidates;
  router.group_score = reinterpret_cast<float*>(router.precise);
  router.group_size_of = router.group_score + kMostGroups;
  at += (32 / L) * kCandidates * 2;
  router.chosen = reinterpret_cast<int*>(at) + token * 32;
  router.found = reinterpret_cast<int*>(at) + (32 / L) * 32 + token;
  for (int base = warp * (32 / L); base < tokens; base += warps * (32 / L)) {
    const int t = base + token;
    const bool live = t < tokens;
    router.row = static_cast<const T*>(r.logits) + (t0 + min(t, tokens - 1)) * r.stride;
    router.run(t0 + t, live, nan, count, all ? ids + t * p.top_k : nullptr);
  }
  if (!r.with_plan) return;
  __syncthreads();
  if (all) {
    plan_whole(p, ids, plan);
  } else {
    put_counts(p, b, count);
  }
}

// bytes: ids in; slots, positions and offsets out
double plan_work(const PlanParams& p) { return 4.0 * (3.0 * p.pairs + p.E + 1); }

aiq_status_t launch_plan(const PlanParams& p, const int* ids, cudaStream_t s) {
  const size_t smem = plan_smem(p.E, kPlanThreads / 32);
  DeviceProps props;
  if (aiq_status_t st = current_device_props(&props)) return st;
  AIQ_ENSURE_DYNAMIC_SMEM(expert_plan_kernel, props.smem_optin);
  LaunchScope scope(AIQ_KERNEL_QLINEAR, s, 0.0, plan_work(p));
  AIQ_CUDA_TRY(launch_chained(true, expert_plan_kernel, dim3(p.token_blocks), dim3(kPlanThreads), smem, s, p, ids));
  AIQ_LAUNCH_CHECK("expert_plan");
  return AIQ_OK;
}

template <typename T, int K, int L>
aiq_status_t launch_route(RouteParams r, const PlanParams& p, cudaStream_t s) {
  DeviceProps props;
  if (aiq_status_t st = current_device_props(&props)) return st;
  AIQ_ENSURE_DYNAMIC_SMEM((route_experts_kernel<T, K, L>), props.smem_optin);
  const bool all = r.with_plan && p.token_blocks == 1;
  r.group_size = p.E / r.groups;
  r.group_of = FastDiv(r.group_size);
  while ((2 << r.group_shift) * r.groups <= L) ++r.group_shift;
  r.run_shift = -1;
  for (int i = 0; i < 4; ++i)
    if (r.group_size == 8 << i) r.run_shift = i;
  r.vec = p.E % 8 == 0 && ((uintptr_t)r.logits) % 16 == 0 && (p.T == 1 || r.stride * (int64_t)sizeof(T) % 16 == 0);
  // as many warps as the tokens take, or fit
  int warps = (p.block_tokens + 32 / L - 1) / (32 / L);
  if (warps > kPlanThreads / 32) warps = kPlanThreads / 32;
  size_t smem = 0;
  for (;; --warps) {
    smem = sizeof(int) * ((size_t)warps * route_warp_words(p.E, L) + route_row(p.E)) +
           (all ? sizeof(int) * (((size_t)p.pairs + 3) & ~(size_t)3) + plan_whole_smem(p, warps) : sizeof(int) * (size_t)p.E);
    if (smem <= (size_t)props.smem_optin) break;
    if (warps == 1) return set_error(AIQ_ERR_SHAPE, "route_experts: %zu bytes of shared memory", smem);
  }
  {
    LaunchScope scope(AIQ_KERNEL_QLINEAR, s, 10.0 * p.T * p.E, (double)p.T * (p.E * sizeof(T) + 8.0 * p.top_k));
    AIQ_CUDA_TRY(launch_chained(true, route_experts_kernel<T, K, L>, dim3(p.token_blocks), dim3(32 * warps), smem, s, r, p));
    AIQ_LAUNCH_CHECK("route_experts");
  }
  return r.with_plan && !all ? launch_plan(p, r.ids, s) : AIQ_OK;
}
template <typename T, int L>
aiq_status_t launch_route_lanes(const RouteParams& r, const PlanParams& p, cudaStream_t s) {
  if (p.top_k == 1) return launch_route<T, 1, L>(r, p, s);
  if (p.top_k == 2) return launch_route<T, 2, L>(r, p, s);
  if (p.top_k <= 4) return launch_route<T, 4, L>(r, p, s);
  if (p.top_k <= 8) return launch_route<T, 8, L>(r, p, s);
  if (p.top_k <= 16) return launch_route<T, 16, L>(r, p, s);
  return launch_route<T, 32, L>(r, p, s);
}

template <typename T>
aiq_status_t launch_route(const RouteParams& r, const PlanParams& p, cudaStream_t s) {
  // 4,096 tokens among 256 experts 10.9 us with a warp a token, 12.5 with eight lanes; 2,000 among 1,024 19 and 39; 16,384 among 256 27 and 23; up to 64
  // experts eight lanes have all of them.
  return p.T <= kFewTokens && p.E > 64 ? launch_route_lanes<T, 32>(r, p, s) : launch_route_lanes<T, 8>(r, p, s);
}

// ---------------------------------------------------------------------------------------
// the weighted sum
// ---------------------------------------------------------------------------------------
constexpr int kCombineThreads = 256;

// A thread has eight neighbouring values of a token (one where rows do not start on 16 bytes).  In float32: residual, then the experts in the
// token's order.  A place without an expert counts as a row of zeros.  Bound by memory: 4,096 tokens, 8 experts, rows of 4096, bfloat16, residual 61 us (336 MB, 84 %
// of the copy rate); one token a launch.
template <typename T, int C>
__global__ void __launch_bounds__(kCombineThreads)
combine_kernel(const T* z, int64_t z_stride, const float* weights, const int* header, int tokens, int kind, const int* positions, int top_k, int H,
               const T* residual, int64_t r_stride, T* y, int64_t y_stride) {
  chain_release();
  const int c = (blockIdx.y * kCombineThreads + threadIdx.x) * C;
  if (c >= H) return;
  chain_wait();
  {
    const int64_t t = blockIdx.x;
    const bool ours = header[2] == tokens && header[3] == kind;
    float acc[C];
    if (residual) {
      if constexpr (C == 8) load8(residual + t * r_stride + c, acc);
      else acc[0] = to_float(residual[t * r_stride + c]);
    } else {
#pragma unroll
      for (int j = 0; j < C; ++j) acc[j] = 0.f;
    }
    for (int i = 0; i < top_k; ++i) {
      const int row = ours ? positions[t * top_k + i] : -1;
      const float w = ours ? weights[t * top_k + i] : __int_as_float(0x7FC00000);
      float v[C];
      if (row < 0) {
#pragma unroll
        for (int j = 0; j < C; ++j) v[j] = 0.f;
      } else if constexpr (C == 8) {
        load8(z + row * z_stride + c, v);
      } else {
        v[0] = to_float(z[row * z_stride + c]);
      }
#pragma unroll
      for (int j = 0; j < C; ++j) acc[j] = fmaf(w, v[j], acc[j]);
    }
    T* out = y + t * y_stride + c;
    if constexpr (C == 8) {
      T h[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) h[j] = from_float<T>(acc[j]);
      uint4 raw[sizeof(T) / 2];
      memcpy(raw, h, sizeof(h));
#pragma unroll
      for (int j = 0; j < (int)sizeof(T) / 2; ++j) reinterpret_cast<uint4*>(out)[j] = raw[j];
    } else {
      *out = from_float<T>(acc[0]);
    }
  }
}

template <typename T>
aiq_status_t launch_combine(const void* z, int64_t z_stride, const float* weights, const PlanParams& p, int H, const void* residual, int64_t r_stride, void* y,
                            int64_t y_stride, cudaStream_t s) {
  const int tokens = p.T, top_k = p.top_k;
  auto aligned = [&](const void* q, int64_t stride, int rows) {
    return !q || ((((uintptr_t)q) & 15) == 0 && (rows == 1 || stride * (int64_t)sizeof(T) % 16 == 0));
  };
  const bool wide = H % 8 == 0 && aligned(z, z_stride, tokens * top_k) && aligned(residual, r_stride, tokens) && aligned(y, y_stride, tokens);
  const int per_block = kCombineThreads * (wide ? 8 : 1);
  const dim3 grid(tokens, (H + per_block - 1) / per_block);
  if (grid.y > 65535) return set_error(AIQ_ERR_SHAPE, "combine_experts: rows of %d", H);
  LaunchScope scope(AIQ_KERNEL_QLINEAR, s, 2.0 * tokens * top_k * H, (double)sizeof(T) * tokens * H * (top_k + (residual ? 2 : 1)));
  auto go = [&](auto kernel) {
    return launch_chained(true, kernel, grid, dim3(kCombineThreads), 0, s, static_cast<const T*>(z), z_stride, weights, p.header, tokens,
                          plan_kind(top_k, p.E), p.positions, top_k, H, static_cast<const T*>(residual), r_stride, static_cast<T*>(y), y_stride);
  };
  AIQ_CUDA_TRY(wide ? go(combine_kernel<T, 8>) : go(combine_kernel<T, 1>));
  AIQ_LAUNCH_CHECK("combine_experts");
  return AIQ_OK;
}

}  // namespace
}  // namespace aiq

// ---------------------------------------------------------------------------------------
// C entry points
// ---------------------------------------------------------------------------------------
using aiq::set_error;

static const int kMost = 1 << 30;

static aiq_status_t expert_check(const char* what, int T, int top_k, int E) {
  if (E <= 0 || E > aiq::kMostExperts) return set_error(AIQ_ERR_INVALID_ARG, "%s: %d experts (1 to %d)", what, E, aiq::kMostExperts);
  if (top_k <= 0 || top_k > aiq::kMostTopK || top_k > E) return set_error(AIQ_ERR_INVALID_ARG, "%s: top_k=%d of %d experts", what, top_k, E);
  if (T <= 0 || (int64_t)T * top_k > kMost) return set_error(AIQ_ERR_INVALID_ARG, "%s: %d tokens", what, T);
  return AIQ_OK;
}
static aiq_status_t plan_check(const char* what, const void* plan, size_t bytes, int T, int top_k, int E) {
  if (((uintptr_t)plan) & 15) return set_error(AIQ_ERR_INVALID_ARG, "%s: plan not 16-byte aligned", what);
  const size_t needed = aiq_expert_plan_bytes(T, top_k, E);
  if (bytes < needed) return set_error(AIQ_ERR_WORKSPACE_TOO_SMALL, "%s: plan of %zu bytes, %zu needed", what, bytes, needed);
  return AIQ_OK;
}
static aiq_status_t expert_check_rows(const char* what, const void* q, int dtype, int rows, int width, int64_t stride, bool out) {
  if (!aiq::mx_dtype_ok(dtype)) return set_error(AIQ_ERR_INVALID_ARG, "%s: dtype=%d", what, dtype);
  if (!q) return set_error(AIQ_ERR_INVALID_ARG, "%s: null pointer", what);
  if (((uintptr_t)q) % aiq::mx_dtype_bytes(dtype)) return set_error(AIQ_ERR_INVALID_ARG, "%s: rows not aligned to their type", what);
  if (rows > 1 && (stride < (out ? width : 0) || stride > (int64_t)1 << 40))
    return set_error(AIQ_ERR_INVALID_ARG, "%s: row stride %lld of rows of %d", what, (long long)stride, width);
  return AIQ_OK;
}

extern "C" size_t aiq_expert_plan_bytes(int T, int top_k, int E) {
  if (expert_check("aiq_expert_plan_bytes", T, top_k, E)) return 0;
  return (size_t)aiq::plan_layout(T, top_k, E).words * 4;
}
extern "C" aiq_status_t aiq_expert_plan_parts(int T, int top_k, int E, size_t* offsets, size_t* slots, size_t* positions) {
  if (aiq_status_t st = expert_check("aiq_expert_plan_parts", T, top_k, E)) return st;
  const aiq::PlanLayout l = aiq::plan_layout(T, top_k, E);
  if (offsets) *offsets = (size_t)l.offsets * 4;
  if (slots) *slots = (size_t)l.slots * 4;
  if (positions) *positions = (size_t)l.positions * 4;
  return AIQ_OK;
}

extern "C" aiq_status_t aiq_plan_experts(const int32_t* ids, int T, int top_k, int E, void* plan, size_t plan_bytes, void* stream) {
  const char* what = "aiq_plan_experts";
  if (aiq_status_t st = expert_check(what, T, top_k, E)) return st;
  if (!ids || !plan) return set_error(AIQ_ERR_INVALID_ARG, "%s: null pointer", what);
  if (((uintptr_t)ids) & 3) return set_error(AIQ_ERR_INVALID_ARG, "%s: ids not aligned to their type", what);
  if (aiq_status_t st = plan_check(what, plan, plan_bytes, T, top_k, E)) return st;
  if (aiq_status_t st = aiq::check_device_sm100()) return st;
  const aiq::PlanLayout l = aiq::plan_layout(T, top_k, E);
  const aiq::PlanParams p = aiq::plan_params(l, T, top_k, E, plan);
  cudaStream_t s = (cudaStream_t)stream;
  aiq::DeviceProps props;
  if (aiq_status_t st = aiq::current_device_props(&props)) return st;
  using namespace aiq;
  AIQ_ENSURE_DYNAMIC_SMEM(expert_count_kernel, props.smem_optin);
  const int threads = p.pairs <= kFewPairs ? (p.pairs + 31) / 32 * 32 : kPlanThreads;
  const size_t smem = p.token_blocks > 1 ? sizeof(int) * (size_t)E : sizeof(int) * (((size_t)p.pairs + 3) & ~(size_t)3) + plan_whole_smem(p, threads / 32);
  {
    LaunchScope scope(AIQ_KERNEL_QLINEAR, s, 0.0, p.token_blocks > 1 ? 4.0 * p.pairs : plan_work(p));
    AIQ_CUDA_TRY(launch_chained(true, expert_count_kernel, dim3(p.token_blocks), dim3(threads), smem, s, p, ids));
    AIQ_LAUNCH_CHECK("expert_count");
  }
  return p.token_blocks > 1 ? launch_plan(p, ids, s) : AIQ_OK;
}

extern "C" aiq_status_t aiq_route_experts(const void* logits, int dtype, int T, int E, int64_t stride, const float* bias, int scoring, int top_k,
                                          int groups, int top_groups, int group_best, int renormalise, float scale, int32_t* ids, float* weights,
                                          void* plan, size_t plan_bytes, void* stream) {
  const char* what = "aiq_route_experts";
  if (aiq_status_t st = expert_check(what, T, top_k, E)) return st;
  if (aiq_status_t st = expert_check_rows(what, logits, dtype, T, E, stride, false)) return st;
  if (!ids || !weights) return set_error(AIQ_ERR_INVALID_ARG, "%s: null pointer", what);
  if ((((uintptr_t)ids) | ((uintptr_t)weights) | ((uintptr_t)bias)) & 3)
    return set_error(AIQ_ERR_INVALID_ARG, "%s: ids, weights or bias not aligned to their type", what);
  if (scoring != AIQ_SCORE_SOFTMAX && scoring != AIQ_SCORE_SIGMOID) return set_error(AIQ_ERR_INVALID_ARG, "%s: scoring=%d", what, scoring);
  if (groups <= 0 || groups > aiq::kMostGroups || E % groups || top_groups <= 0 || top_groups > groups || group_best < 1 || group_best > 2)
    return set_error(AIQ_ERR_INVALID_ARG, "%s: %d of %d groups of %d experts, best %d", what, top_groups, groups, E, group_best);
  if (top_k > E / groups * top_groups) return set_error(AIQ_ERR_INVALID_ARG, "%s: top_k=%d of %d groups of %d", what, top_k, top_groups, E / groups);
  if (renormalise != 0 && renormalise != 1) return set_error(AIQ_ERR_INVALID_ARG, "%s: renormalise=%d", what, renormalise);
  if (!(scale - scale == 0.f)) return set_error(AIQ_ERR_INVALID_ARG, "%s: scale is not finite", what);
  if (plan)
    if (aiq_status_t st = plan_check(what, plan, plan_bytes, T, top_k, E)) return st;
  if (aiq_status_t st = aiq::check_device_sm100()) return st;
  const aiq::PlanParams p = aiq::plan_params(aiq::plan_layout(T, top_k, E), T, top_k, E, plan);
  aiq::RouteParams r = {};
  r.logits = logits;
  r.stride = T == 1 ? E : stride;
  r.bias = bias;
  r.sigmoid = scoring == AIQ_SCORE_SIGMOID;
  r.groups = groups; r.top_groups = top_groups; r.group_best = group_best;
  r.renormalise = renormalise;
  r.scale = scale;
  r.ids = ids;
  r.weights = weights;
  r.with_plan = plan != nullptr;
  cudaStream_t s = (cudaStream_t)stream;
  switch (dtype) {
    case AIQ_DTYPE_F32: return aiq::launch_route<float>(r, p, s);
    case AIQ_DTYPE_F16: return aiq::launch_route<__half>(r, p, s);
    default: return aiq::launch_route<__nv_bfloat16>(r, p, s);
  }
}

extern "C" aiq_status_t aiq_combine_experts(const void* z, int dtype, int T, int top_k, int E, int H, int64_t z_stride, const float* weights,
                                            const void* plan, size_t plan_bytes, const void* residual, int64_t r_stride, void* y, int64_t y_stride,
                                            void* stream) {
  const char* what = "aiq_combine_experts";
  if (aiq_status_t st = expert_check(what, T, top_k, E)) return st;
  if (H <= 0 || H > kMost) return set_error(AIQ_ERR_INVALID_ARG, "%s: rows of %d", what, H);
  if (aiq_status_t st = expert_check_rows(what, z, dtype, T * top_k, H, z_stride, false)) return st;
  if (aiq_status_t st = expert_check_rows(what, y, dtype, T, H, y_stride, true)) return st;
  if (residual)
    if (aiq_status_t st = expert_check_rows(what, residual, dtype, T, H, r_stride, false)) return st;
  if (!weights || !plan) return set_error(AIQ_ERR_INVALID_ARG, "%s: null pointer", what);
  if (((uintptr_t)weights) & 3) return set_error(AIQ_ERR_INVALID_ARG, "%s: weights not aligned to their type", what);
  if (aiq_status_t st = plan_check(what, plan, plan_bytes, T, top_k, E)) return st;
  if (aiq_status_t st = aiq::check_device_sm100()) return st;
  const aiq::PlanParams p = aiq::plan_params(aiq::plan_layout(T, top_k, E), T, top_k, E, const_cast<void*>(plan));
  if (T == 1) r_stride = y_stride = H;
  if (T * top_k == 1) z_stride = H;
  cudaStream_t s = (cudaStream_t)stream;
  switch (dtype) {
    case AIQ_DTYPE_F32: return aiq::launch_combine<float>(z, z_stride, weights, p, H, residual, r_stride, y, y_stride, s);
    case AIQ_DTYPE_F16: return aiq::launch_combine<__half>(z, z_stride, weights, p, H, residual, r_stride, y, y_stride, s);
    default: return aiq::launch_combine<__nv_bfloat16>(z, z_stride, weights, p, H, residual, r_stride, y, y_stride, s);
  }
}

extern "C" size_t aiq_mx_linear_experts_workspace_bytes(int E, int N, int K, int rows, int dtype) {
  if (E <= 0 || E > aiq::kMostExperts || N <= 0 || K <= 0 || rows <= 0 || N > kMost || K > kMost || rows > kMost || !aiq::mx_dtype_ok(dtype)) return 0;
  return aiq::mx_tc_workspace_bytes(K, rows, dtype);
}

extern "C" aiq_status_t aiq_mx_linear_experts(const void* codes, const void* scales, const float* bias, int E, int N, int K, const void* x, int dtype,
                                              int64_t x_stride, int x_sorted, const void* plan, size_t plan_bytes, int T, int top_k, int activation,
                                              int gated, void* y, int64_t y_stride, void* workspace, size_t workspace_bytes, void* stream) {
  const char* what = "aiq_mx_linear_experts";
  if (aiq_status_t st = expert_check(what, T, top_k, E)) return st;
  if (!codes || !scales || !plan || !workspace) return set_error(AIQ_ERR_INVALID_ARG, "%s: null pointer", what);
  if (N <= 0 || K <= 0 || N > kMost || K > kMost) return set_error(AIQ_ERR_INVALID_ARG, "%s: N=%d K=%d", what, N, K);
  if (((uintptr_t)codes) & 31) return set_error(AIQ_ERR_INVALID_ARG, "%s: codes not 32-byte aligned", what);
  if (((uintptr_t)scales) & 15) return set_error(AIQ_ERR_INVALID_ARG, "%s: scales not 16-byte aligned", what);
  if (((uintptr_t)bias) & 3) return set_error(AIQ_ERR_INVALID_ARG, "%s: bias not aligned to its type", what);
  if (((uintptr_t)workspace) & 15) return set_error(AIQ_ERR_INVALID_ARG, "%s: workspace not 16-byte aligned", what);
  if (x_sorted != 0 && x_sorted != 1) return set_error(AIQ_ERR_INVALID_ARG, "%s: x_sorted=%d", what, x_sorted);
  if (activation < AIQ_ACT_NONE || activation > AIQ_ACT_GELU_TANH) return set_error(AIQ_ERR_INVALID_ARG, "%s: activation=%d", what, activation);
  if ((gated != 0 && gated != 1) || (gated && (N & 1))) return set_error(AIQ_ERR_INVALID_ARG, "%s: gated=%d with N=%d", what, gated, N);
  const int rows = T * top_k, outputs = gated ? N / 2 : N;
  if (aiq_status_t st = expert_check_rows(what, x, dtype, x_sorted ? rows : T, K, x_stride, false)) return st;
  if (aiq_status_t st = expert_check_rows(what, y, dtype, rows, outputs, y_stride, true)) return st;
  if (aiq_status_t st = plan_check(what, plan, plan_bytes, T, top_k, E)) return st;
  const size_t needed = aiq_mx_linear_experts_workspace_bytes(E, N, K, rows, dtype);
  if (workspace_bytes < needed)
    return set_error(AIQ_ERR_WORKSPACE_TOO_SMALL, "%s: workspace of %zu bytes, %zu needed", what, workspace_bytes, needed);
  if (aiq_status_t st = aiq::check_device_sm100()) return st;
  const aiq::PlanLayout l = aiq::plan_layout(T, top_k, E);
  const int* w = static_cast<const int*>(plan);
  aiq::MxProduct p = {};
  p.w_codes = static_cast<const uint8_t*>(codes);
  p.w_scales = static_cast<const uint8_t*>(scales);
  p.bias = bias;
  p.x = x;
  p.x_stride = (x_sorted ? rows : T) == 1 ? K : x_stride;
  p.y = y;
  p.y_stride = rows == 1 ? outputs : y_stride;
  p.N = N; p.K = K; p.M = rows; p.dtype = dtype;
  p.act = activation; p.gated = gated;
  p.experts = E; p.top_k = top_k; p.width = l.width; p.blocks_most = l.blocks_most;
  p.header = w;
  p.plan_kind = aiq::plan_kind(top_k, E);
  p.tokens = T;
  p.blocks = reinterpret_cast<const aiq::ExpertBlock*>(w + l.blocks);
  p.positions = x_sorted ? nullptr : w + l.positions;
  p.slots = w + l.slots;
  return aiq::launch_mx_linear_experts(p, workspace, (cudaStream_t)stream);
}
