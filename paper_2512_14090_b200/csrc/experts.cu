// A layer of experts: which experts a token goes to, the plan that sorts (token, expert) pairs by expert, and the weighted sum of what comes back.
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
//   counts     [token blocks][E] pairs of each expert in a token block (between the two launches of a large plan)
struct PlanLayout {
  int64_t offsets, slots, positions, blocks, counts, words;
  int pairs, width, blocks_most, token_blocks, block_tokens;
};
__host__ __device__ inline int plan_kind(int top_k, int E) { return 0x41000000 | top_k << 16 | E; }
constexpr int kOneBlockTokens = 64;              // up to here one thread block does everything
constexpr int kPlanThreads = 1024;

PlanLayout plan_layout(int T, int top_k, int E) {
  PlanLayout l = {};
  l.pairs = T * top_k;
  // Rows per block: twice an expert's share, as long as it gets that many tokens.
  const int share = (l.pairs + E - 1) / E;
  l.width = 16;
  while (l.width < 128 && l.width < 2 * share && l.width < T) l.width *= 2;
  l.blocks_most = l.pairs / l.width + (l.pairs < E ? l.pairs : E);
  l.block_tokens = T <= kOneBlockTokens ? T : (T + 147) / 148 < 16 ? 16 : (T + 147) / 148;
  l.token_blocks = (T + l.block_tokens - 1) / l.block_tokens;
  auto part = [&](int64_t words) { const int64_t at = l.words; l.words += (words + 3) / 4 * 4; return at; };
  part(4);
  l.offsets = part(E + 1);
  l.slots = part(l.pairs);
  l.positions = part(l.pairs);
  l.blocks = part(4ll * l.blocks_most);
  l.counts = part(l.token_blocks > 1 ? (int64_t)l.token_blocks * E : 0);
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

// Exclusive prefix sums of v[0 .. n) in shared memory by one thread block; v[n] gets the sum.  part: 33 words.
__device__ void block_scan(int* v, int n, int* part) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int carry = 0;
  for (int base = 0; base < n; base += blockDim.x) {
    const int i = base + tid, mine = i < n ? v[i] : 0;
    int sum = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += up;
    }
    if (lane == 31) part[warp] = sum;
    __syncthreads();
    int before = 0, all = 0;
    for (int w = 0; w < (int)blockDim.x / 32; ++w) {
      before += w < warp ? part[w] : 0;
      all += part[w];
    }
    if (i < n) v[i] = carry + before + sum - mine;
    carry += all;
    __syncthreads();
  }
  if (tid == 0) v[n] = carry;
  __syncthreads();
}

// The share of thread block `b` in the plan.  ids: global or shared, of its tokens.  In shared memory: offset[E + 1], the experts' first rows;
// next[warps][E], where each warp's next pair of an expert goes; first[E + 1], the experts' first blocks of rows.
// total(e), before(e): pairs of expert e in all, and in the token blocks before this one.
template <typename F, typename G>
__device__ void plan_share(const PlanParams& p, int b, const int* __restrict__ ids, int* smem, F total, G before) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
  int* offset = smem;
  int* first = offset + p.E + 1;
  int* part = first + p.E + 1;
  int* next = part + 33;
  for (int e = tid; e < p.E; e += blockDim.x) {
    const int n = total(e);
    offset[e] = n;
    first[e] = (n + p.width - 1) / p.width;
  }
  for (int i = tid; i < warps * p.E; i += blockDim.x) next[i] = 0;
  __syncthreads();
  block_scan(offset, p.E, part);
  block_scan(first, p.E, part);
  // each warp has a run of the block's pairs, in order
  const int slot0 = b * p.block_tokens * p.top_k, pairs = min(p.T - b * p.block_tokens, p.block_tokens) * p.top_k;
  const int run = (pairs + warps * 32 - 1) / (warps * 32) * 32, begin = min(pairs, warp * run), end = min(pairs, begin + run);
  for (int i = begin + lane; i < end; i += 32) {
    const int e = ids[i];
    if ((unsigned)e < (unsigned)p.E) atomicAdd(next + warp * p.E + e, 1);
  }
  __syncthreads();
  for (int e = tid; e < p.E; e += blockDim.x) {
    int at = offset[e] + before(e);
    for (int w = 0; w < warps; ++w) {
      const int n = next[w * p.E + e];
      next[w * p.E + e] = at;
      at += n;
    }
  }
  __syncthreads();
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
  const int rows = offset[p.E], blocks = first[p.E], stride = p.token_blocks * blockDim.x, at = b * blockDim.x + tid;
  for (int i = rows + at; i < p.pairs; i += stride) p.slots[i] = -1;
  for (int i = at; i <= p.E; i += stride) p.offsets[i] = offset[i];
  for (int i = at; i < blocks; i += stride) {
    int lo = 0, hi = p.E - 1;                      // the last expert whose first block is i or before
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (first[mid] <= i) lo = mid; else hi = mid - 1;
    }
    const int n = offset[lo + 1] - offset[lo];
    p.blocks[i] = ExpertBlock{lo, offset[lo], n, first[lo]};
  }
  if (at == 0) *reinterpret_cast<int4*>(p.header) = make_int4(rows, blocks, p.T, plan_kind(p.top_k, p.E));
}
inline size_t plan_smem(int E, int warps) { return sizeof(int) * (2 * (size_t)(E + 1) + 33 + (size_t)warps * E); }

// The second launch of a large plan.
__global__ void __launch_bounds__(kPlanThreads)
expert_plan_kernel(const __grid_constant__ PlanParams p, const int* ids) {
  extern __shared__ int smem[];
  const int b = blockIdx.x;
  int* totals = smem + 2 * (p.E + 1) + 33 + (blockDim.x >> 5) * p.E;
  int* befores = totals + p.E;
  for (int e = threadIdx.x; e < p.E; e += blockDim.x) {
    int total = 0, before = 0;
    for (int q = 0; q < p.token_blocks; ++q) {
      const int n = p.counts[(int64_t)q * p.E + e];
      total += n;
      before += q < b ? n : 0;
    }
    totals[e] = total;
    befores[e] = before;
  }
  __syncthreads();
  plan_share(p, b, ids + (int64_t)b * p.block_tokens * p.top_k, smem, [&](int e) { return totals[e]; }, [&](int e) { return befores[e]; });
}

// Given ids: their counts (first launch of a large plan), or all of a small one.
__global__ void __launch_bounds__(kPlanThreads)
expert_count_kernel(const __grid_constant__ PlanParams p, const int* __restrict__ ids) {
  extern __shared__ int smem[];
  const int b = blockIdx.x, slot0 = b * p.block_tokens * p.top_k, pairs = min(p.T - b * p.block_tokens, p.block_tokens) * p.top_k;
  int* count = smem + (p.token_blocks > 1 ? 0 : 2 * (p.E + 1) + 33 + (blockDim.x >> 5) * p.E);
  for (int e = threadIdx.x; e < p.E; e += blockDim.x) count[e] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < pairs; i += blockDim.x) {
    const int e = ids[slot0 + i];
    if ((unsigned)e < (unsigned)p.E) atomicAdd(count + e, 1);
  }
  __syncthreads();
  if (p.token_blocks > 1) {
    for (int e = threadIdx.x; e < p.E; e += blockDim.x) p.counts[(int64_t)b * p.E + e] = count[e];
  } else {
    plan_share(p, 0, ids, smem, [&](int e) { return count[e]; }, [&](int) { return 0; });
  }
}

// ---------------------------------------------------------------------------------------
// routing
// ---------------------------------------------------------------------------------------
struct RouteParams {
  const void* logits;
  int64_t stride;
  const float* bias;
  int sigmoid, groups, top_groups, group_best, renormalise;
  float scale;
  int* ids;
  float* weights;
  int with_plan;
};

// Order-preserving keys: larger value, larger key; 0 is "not to be chosen".
template <typename S> struct Key;
template <> struct Key<float> {
  typedef uint32_t type;
  static __device__ __forceinline__ uint32_t of(float v) {
    const uint32_t b = __float_as_uint(v + 0.f);                             // -0 is 0
    return b & 0x80000000u ? ~b : b | 0x80000000u;
  }
  static __device__ __forceinline__ float value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }
  static __device__ __forceinline__ uint32_t most(uint32_t k) { return __reduce_max_sync(0xffffffffu, k); }
};
template <> struct Key<double> {
  typedef uint64_t type;
  static __device__ __forceinline__ uint64_t of(double v) {
    const uint64_t b = (uint64_t)__double_as_longlong(v + 0.0);
    return b >> 63 ? ~b : b | 0x8000000000000000ull;
  }
  static __device__ __forceinline__ double value(uint64_t k) { return __longlong_as_double((long long)(k >> 63 ? k & 0x7FFFFFFFFFFFFFFFull : ~k)); }
  static __device__ __forceinline__ uint64_t most(uint64_t k) {
    const uint32_t high = __reduce_max_sync(0xffffffffu, (uint32_t)(k >> 32));
    const uint32_t low = __reduce_max_sync(0xffffffffu, (uint32_t)(k >> 32) == high ? (uint32_t)k : 0u);
    return (uint64_t)high << 32 | low;
  }
};
__device__ __forceinline__ float route_exp(float v) { return expf(v); }
__device__ __forceinline__ double route_exp(double v) { return exp(v); }
template <typename S>
__device__ __forceinline__ S warp_sum(S v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// One token by one warp: lane holds experts lane, lane + 32, ...  Chooses in the arithmetic of S; lane j < top_k ends up with the j-th expert (-1:
// none).  Returns false where S = float cannot tell the order: two values in a row are closer than their rounding, and not equal because
// they come from equal logits and biases.  shared: E values of this warp, where groups have to be scored.
//   score of an expert: softmax or logistic function of its logit.  choice: score + bias; without a bias the logit itself, whose order it is.
// Float scores are off by less than 8 rounding steps of 2^-24 and, softmax, |l - max| p <= 0.37 times as much again; 2^-18 is beyond all that.
template <typename S, int V, typename T>
__device__ bool route_choose(const RouteParams& r, int E, int top_k, const float (&l)[V], const T* row, float top, S* shared, int* id_out) {
  typedef typename Key<S>::type K;
  const int lane = threadIdx.x & 31;
  const bool scored = r.bias || (r.groups > 1 && r.group_best == 2);
  K key[V];
  S score[V];
  if (scored) {
    if (r.sigmoid) {
#pragma unroll
      for (int i = 0; i < V; ++i) score[i] = S(1) / (S(1) + route_exp(-S(l[i])));
    } else {
      S sum = 0;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        score[i] = l[i] == -INFINITY ? S(0) : route_exp(S(l[i]) - S(top));
        sum += score[i];
      }
      const S inverse = S(1) / warp_sum(sum);
#pragma unroll
      for (int i = 0; i < V; ++i) score[i] *= inverse;
    }
    if (r.bias) {
#pragma unroll
      for (int i = 0; i < V; ++i) score[i] += S(lane + 32 * i < E ? r.bias[lane + 32 * i] : 0.f);
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) score[i] = S(l[i]);
  }
  bool clear = true;
  uint32_t open = 0xffffffffu;
  const int size = E / r.groups;
  if (r.groups > 1) {
    __syncwarp();
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int e = lane + 32 * i;
      if (e < E) shared[e] = l[i] == -INFINITY || score[i] == -INFINITY ? S(-INFINITY) : score[i];
    }
    __syncwarp();
    // as many lanes to a group as there are, each with every so-manieth of its experts
    int per = 32;
    while (per * r.groups > 32) per >>= 1;
    const int g = lane / per, sub = lane % per;
    S best = -INFINITY, second = -INFINITY;
    if (g < r.groups)
      for (int j = 0, at = (sub + g * per) % size; j < size; ++j, at = at + 1 == size ? 0 : at + 1)
        if (at % per == sub) {
          const S v = shared[g * size + at];
          second = v > best ? best : v > second ? v : second;
          best = v > best ? v : best;
        }
    for (int o = per >> 1; o > 0; o >>= 1) {
      const S b2 = __shfl_xor_sync(0xffffffffu, best, o), s2 = __shfl_xor_sync(0xffffffffu, second, o);
      const S low = b2 < best ? b2 : best;
      second = second > s2 ? second : s2;
      second = low > second ? low : second;
      best = b2 > best ? b2 : best;
    }
    K mine = best == S(-INFINITY) ? K(0) : Key<S>::of(r.group_best == 2 && second != S(-INFINITY) ? best + second : best);
    open = 0;
    S last = 0;
    for (int j = 0; j <= r.top_groups && j < r.groups; ++j) {
      const K most = Key<S>::most(mine);
      if (most == K(0)) break;
      const int at = __reduce_min_sync(0xffffffffu, mine == most ? (uint32_t)g : 32u);
      if (g == at) mine = K(0);
      const S v = Key<S>::value(most);
      if (sizeof(S) == 4 && scored && j == r.top_groups && !(last - v > S(0x1p-17f) + S(0x1p-22f) * fabsf((float)v))) clear = false;
      last = v;
      if (j < r.top_groups) open |= 1u << at;
    }
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int e = lane + 32 * i;
    const S v = r.bias ? score[i] : S(l[i]);
    bool on = e < E && l[i] != -INFINITY && v != S(-INFINITY);
    if (r.groups > 1 && on) on = open >> (e / size) & 1u;
    key[i] = on ? Key<S>::of(v) : K(0);
  }
  K mine = K(0);                                   // lane j: key of the j-th
  int id = -1;
  for (int j = 0; j <= top_k; ++j) {
    K best = key[0];
#pragma unroll
    for (int i = 1; i < V; ++i) best = key[i] > best ? key[i] : best;
    const K most = Key<S>::most(best);
    if (most == K(0)) break;
    uint32_t at = 0xffffu;
#pragma unroll
    for (int i = V - 1; i >= 0; --i)
      if (key[i] == most) at = lane + 32 * i;
    at = __reduce_min_sync(0xffffffffu, at);
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (at == (uint32_t)(lane + 32 * i)) key[i] = K(0);
    if (lane == j) { mine = most; id = (int)at; }
  }
  if (sizeof(S) == 4 && r.bias) {
    const float v = (float)Key<S>::value(mine), next = __shfl_down_sync(0xffffffffu, v, 1);
    const int next_id = __shfl_down_sync(0xffffffffu, id, 1);
    bool near = lane < top_k && id >= 0 && next_id >= 0 && !(v - next > 0x1p-18f + 0x1p-22f * fabsf(v));
    if (near) near = to_float(row[id]) != to_float(row[next_id]) || r.bias[id] != r.bias[next_id];
    if (__any_sync(0xffffffffu, near)) clear = false;
  }
  *id_out = lane < top_k ? id : -1;
  return clear;
}

template <typename T, int V>
__device__ void route_token(const RouteParams& r, int E, int top_k, int t, float* shared, int* count, int* ids_shared) {
  const int lane = threadIdx.x & 31;
  const T* row = static_cast<const T*>(r.logits) + t * r.stride;
  float l[V], top = -INFINITY;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < V; ++i) l[i] = lane + 32 * i < E ? to_float(row[lane + 32 * i]) : -INFINITY;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    top = fmaxf(top, l[i]);
    bad = bad || l[i] != l[i];
    if (r.bias && lane + 32 * i < E) bad = bad || r.bias[lane + 32 * i] != r.bias[lane + 32 * i];
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  bad = __any_sync(0xffffffffu, bad) || (!r.sigmoid && top == INFINITY);
  int id = -1;
  float w = 0.f;
  if (bad) {
    w = __int_as_float(0x7FC00000);
  } else if (top != -INFINITY) {
    if (!route_choose<float, V>(r, E, top_k, l, row, top, shared, &id))
      route_choose<double, V>(r, E, top_k, l, row, top, reinterpret_cast<double*>(shared), &id);
    const float mine = id >= 0 ? to_float(row[id]) : -INFINITY;
    float sum = 1.f;
    if (r.renormalise) {
      // Far left of zero logistic functions vanish, but their ratios are those of the exponentials.
      float high = mine;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) high = fmaxf(high, __shfl_xor_sync(0xffffffffu, high, o));
      w = r.sigmoid && high >= -40.f ? 1.f / (1.f + expf(-mine)) : expf(mine - high);
      sum = warp_sum(id >= 0 ? w : 0.f);
    } else if (r.sigmoid) {
      w = 1.f / (1.f + expf(-mine));
    } else {
      w = expf(mine - top);
      float part = 0.f;
#pragma unroll
      for (int i = 0; i < V; ++i) part += expf(l[i] - top);
      sum = warp_sum(part);
    }
    w = id >= 0 ? w / sum * r.scale : 0.f;
  }
  if (lane < top_k) {
    r.ids[(int64_t)t * top_k + lane] = id;
    r.weights[(int64_t)t * top_k + lane] = w;
    if (ids_shared) ids_shared[lane] = id;
    if (count && id >= 0) atomicAdd(count + id, 1);
  }
}

template <typename T, int V>
__global__ void __launch_bounds__(V > 8 ? kPlanThreads / 2 : kPlanThreads)
route_experts_kernel(const __grid_constant__ RouteParams r, const __grid_constant__ PlanParams p) {
  extern __shared__ double route_smem[];
  const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5, b = blockIdx.x;
  // scores of each warp, two words an expert (64 bits), where there are groups; the plan's arrays; counts and ids
  float* scores = reinterpret_cast<float*>(route_smem);
  int* plan = reinterpret_cast<int*>(route_smem) + (r.groups > 1 ? 2 * warps * p.E : 0);
  int* count = plan + (r.with_plan && p.token_blocks == 1 ? 2 * (p.E + 1) + 33 + warps * p.E : 0);
  int* ids = count + p.E;
  if (r.with_plan) {
    for (int e = threadIdx.x; e < p.E; e += blockDim.x) count[e] = 0;
    __syncthreads();
  }
  const int t0 = b * p.block_tokens, tokens = min(p.T - t0, p.block_tokens);
  for (int t = warp; t < tokens; t += warps)
    route_token<T, V>(r, p.E, p.top_k, t0 + t, scores + 2 * warp * p.E, r.with_plan ? count : nullptr,
                      r.with_plan && p.token_blocks == 1 ? ids + t * p.top_k : nullptr);
  if (!r.with_plan) return;
  __syncthreads();
  if (p.token_blocks > 1) {
    for (int e = threadIdx.x; e < p.E; e += blockDim.x) p.counts[(int64_t)b * p.E + e] = count[e];
  } else {
    plan_share(p, 0, ids, plan, [&](int e) { return count[e]; }, [&](int) { return 0; });
  }
}

aiq_status_t launch_plan(const PlanParams& p, const int* ids, cudaStream_t s) {
  const size_t smem = plan_smem(p.E, kPlanThreads / 32) + sizeof(int) * 2 * (size_t)p.E;
  DeviceProps props;
  if (aiq_status_t st = current_device_props(&props)) return st;
  AIQ_ENSURE_DYNAMIC_SMEM(expert_plan_kernel, props.smem_optin);
  expert_plan_kernel<<<p.token_blocks, kPlanThreads, smem, s>>>(p, ids);
  AIQ_LAUNCH_CHECK("expert_plan");
  return AIQ_OK;
}

template <typename T, int V>
aiq_status_t launch_route(const RouteParams& r, const PlanParams& p, cudaStream_t s) {
  DeviceProps props;
  if (aiq_status_t st = current_device_props(&props)) return st;
  AIQ_ENSURE_DYNAMIC_SMEM((route_experts_kernel<T, V>), props.smem_optin);
  const bool all = r.with_plan && p.token_blocks == 1;
  const int warps = V > 8 ? 16 : 32;               // registers
  const size_t smem = sizeof(int) * ((r.groups > 1 ? 2 * (size_t)warps * p.E : 0) + p.E + (all ? (size_t)p.block_tokens * p.top_k : 0)) +
                      (all ? plan_smem(p.E, warps) : 0);
  if (smem > (size_t)props.smem_optin) return set_error(AIQ_ERR_SHAPE, "route_experts: %zu bytes of shared memory", smem);
  {
    LaunchScope scope(AIQ_KERNEL_QLINEAR, s, 10.0 * p.T * p.E, (double)p.T * (p.E * sizeof(T) + 8.0 * p.top_k));
    route_experts_kernel<T, V><<<p.token_blocks, 32 * warps, smem, s>>>(r, p);
    AIQ_LAUNCH_CHECK("route_experts");
  }
  return r.with_plan && !all ? launch_plan(p, r.ids, s) : AIQ_OK;
}
template <typename T>
aiq_status_t launch_route(const RouteParams& r, const PlanParams& p, cudaStream_t s) {
  if (p.E <= 32) return launch_route<T, 1>(r, p, s);
  if (p.E <= 64) return launch_route<T, 2>(r, p, s);
  if (p.E <= 128) return launch_route<T, 4>(r, p, s);
  if (p.E <= 256) return launch_route<T, 8>(r, p, s);
  if (p.E <= 512) return launch_route<T, 16>(r, p, s);
  return launch_route<T, 32>(r, p, s);
}

// ---------------------------------------------------------------------------------------
// the weighted sum
// ---------------------------------------------------------------------------------------
constexpr int kCombineThreads = 256;

// A thread has eight neighbouring values of a token (one where rows do not start on 16 bytes).  In float32: residual, then the experts in the
// token's order.  A place without an expert counts as a row of zeros.
template <typename T, int C>
__global__ void __launch_bounds__(kCombineThreads)
combine_kernel(const T* __restrict__ z, int64_t z_stride, const float* __restrict__ weights, const int* __restrict__ header, int tokens, int kind,
               const int* __restrict__ positions, int top_k, int H, const T* residual, int64_t r_stride, T* y, int64_t y_stride) {
  const int c = (blockIdx.y * kCombineThreads + threadIdx.x) * C;
  if (c >= H) return;
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
    kernel<<<grid, kCombineThreads, 0, s>>>(static_cast<const T*>(z), z_stride, weights, p.header, tokens, plan_kind(top_k, p.E), p.positions, top_k, H,
                                            static_cast<const T*>(residual), r_stride, static_cast<T*>(y), y_stride);
  };
  if (wide) go(combine_kernel<T, 8>); else go(combine_kernel<T, 1>);
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
  const size_t smem = sizeof(int) * (size_t)E + (p.token_blocks > 1 ? 0 : plan_smem(E, kPlanThreads / 32));
  expert_count_kernel<<<p.token_blocks, kPlanThreads, smem, s>>>(p, ids);
  AIQ_LAUNCH_CHECK("expert_count");
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
  const aiq::RouteParams r = {logits, T == 1 ? E : stride, bias, scoring == AIQ_SCORE_SIGMOID, groups, top_groups, group_best, renormalise, scale,
                              ids, weights, plan != nullptr};
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
  return aiq::launch_mx_linear_experts(p, workspace, (cudaStream_t)stream);
}
