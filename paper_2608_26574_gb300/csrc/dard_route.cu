// dard_route.cu - dard_route: each token's experts and weights from its router logits, and the
// plan (the (token, slot) pairs sorted by expert) that dard_experts reads on the device.
//
// route_topk, one warp per token: lane l holds experts l, l + 32, ... in registers, as keys whose
// unsigned order is the order of the choice (see choose()). It is bound by instructions, not by
// HBM: 38912 x 256 fp32 logits (40 MB, 6 us of HBM) with a bias, 4 of 8 groups and 8 experts per token
// take 42 us, of which the scores and their order are 23, the groups 9 and seven more
// slots 9. So the work per expert is kept short: eight experts per lane, whose scores stay in
// registers, and no division before the choice where softmax needs none.
//
// The plan is a stable counting sort. A CTA owns a run of consecutive tokens; route_topk
// counts its pairs per expert, and plan_scatter (chained by programmatic dependent launch)
// adds up the counts of the CTAs before it and gives every pair its place. Counts are integers
// and places follow from them, so the plan does not depend on the order of execution. plan_scatter
// takes 10 us there: the sums of 152 CTAs' counts, 14 loads in flight, then the places in shared
// memory, each step waiting for the one before. Few tokens fit one CTA, which then writes the plan
// itself, in one launch.
#include <cuda_bf16.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdlib>

#include "dard_host.cuh"
#include "dard_internal.h"
#include "dard_ptx.cuh"

namespace dard {
namespace {

constexpr int kPlanWarps = 32;                 // plan_scatter
// One CTA routes and plans up to this many tokens. Beyond, more CTAs and a second launch
// are faster (256 experts: 64 tokens 12.5 against 14.5 us in one CTA, 128 tokens 12.6 against 20.8).
constexpr int kOneCtaTokens = 32;
constexpr uint32_t kNone = 0x007fffffu;        // key of -inf: an expert that cannot be chosen

// Ints of a CTA's counts in the workspace: 16-byte rows.
__host__ __device__ constexpr int count_row(int experts) { return (experts + 1 + 3) / 4 * 4; }

// Warps of a route_topk CTA with kPer experts per lane (its registers allow no more).
constexpr int route_warps(int per) { return per <= 8 ? 32 : 16; }

struct RouteParams {
  const void* logits;
  const float* bias;
  int32_t* ids;
  float* weights;
  int32_t* offsets;
  int32_t* rows;
  uint32_t* status;
  int32_t* counts;        // workspace [ctas][count_row]: experts, then slots without an expert
  int64_t logits_stride;
  int32_t tokens, experts, top_k, groups, top_groups, group_size;
  int32_t scoring, renormalise;
  int32_t cta_tokens;     // consecutive tokens of a CTA (both kernels)
  int32_t ctas;
  float scale;
};

// Unsigned order = float order; -inf gives kNone, every finite float more.
__device__ __forceinline__ uint32_t order_key(float f) {
  const int32_t b = __float_as_int(f);
  return static_cast<uint32_t>(b ^ ((b >> 31) | static_cast<int32_t>(0x80000000u)));
}

// Sorts v falling: Batcher's odd-even merge network.
template <int kN>
__device__ __forceinline__ void sort_falling(uint32_t (&v)[kN]) {
#pragma unroll
  for (int p = 1; p < kN; p *= 2) {
#pragma unroll
    for (int k = p; k >= 1; k /= 2) {
#pragma unroll
      for (int j = k % p; j <= kN - 1 - k; j += 2 * k) {
#pragma unroll
        for (int i = 0; i < k; ++i) {
          if (i + j + k < kN && (i + j) / (2 * p) == (i + j + k) / (2 * p)) {
            const uint32_t a = v[i + j], b = v[i + j + k];
            v[i + j] = max(a, b);
            v[i + j + k] = min(a, b);
          }
        }
      }
    }
  }
}

// v[j] for a j that is no constant.
template <int kN>
__device__ __forceinline__ uint32_t pick(const uint32_t (&v)[kN], int j) {
  uint32_t r = v[0];
#pragma unroll
  for (int i = 1; i < kN; ++i) r = i == j ? v[i] : r;
  return r;
}

// The top_k largest keys (expert j * 32 + lane: key[j]), ties to the lowest expert: the id of slot
// `lane`, -1 where no key above kNone is left. One slot after the other: the largest key of
// the warp, and the lowest index that reaches it.
template <int kPer>
__device__ int choose_exactly(uint32_t (&key)[kPer], int top_k, int lane) {
  int my_id = -1;
  for (int s = 0; s < top_k; ++s) {
    uint32_t best = key[0];
#pragma unroll
    for (int j = 1; j < kPer; ++j) best = max(best, key[j]);
    const uint32_t most = __reduce_max_sync(0xffffffffu, best);
    if (most <= kNone) break;
    int e = INT_MAX;
#pragma unroll
    for (int j = kPer - 1; j >= 0; --j)
      if (key[j] == most) e = j * 32 + lane;
    const int first = __reduce_min_sync(0xffffffffu, e);
    if (lane == s) my_id = first;
#pragma unroll
    for (int j = 0; j < kPer; ++j)
      if (first == j * 32 + lane) key[j] = 0;
  }
  return my_id;
}

// The same for fewer instructions where several slots repay the lists (38912 x 256, 8 slots: 42.0
// us against 47.9; 1 slot 22.8 against 19.8, so up to two are chosen above). A key's low bits
// give way to kLow - j, each lane sorts its keys once, and a slot is the largest head of the
// lanes' lists (the lowest lane that reaches it) popped. Equal keys come out by rising j, then
// lane: by rising expert, as they should. Keys that differ in the replaced bits alone could
// come out in the wrong order; they follow one another then, which is looked at, and the token
// is done again exactly.
template <int kPer>
__device__ __forceinline__ int choose(uint32_t (&key)[kPer], int top_k, int lane) {
  constexpr uint32_t kLow = kPer <= 1 ? 0 : kPer <= 2 ? 1 : kPer <= 4 ? 3 : kPer <= 8 ? 7 : 15;
  if (top_k <= 2) return choose_exactly<kPer>(key, top_k, lane);
  uint32_t list[kPer];
#pragma unroll
  for (int j = 0; j < kPer; ++j) list[j] = (key[j] & ~kLow) | (kLow - j);
  sort_falling(list);
  int my_id = -1;
  uint32_t last = 0;  // the slot before: its head and lane
  int last_lane = 0;
  for (int s = 0; s <= top_k; ++s) {  // (one more than is kept, for the look)
    const uint32_t most = __reduce_max_sync(0xffffffffu, list[0]);
    if (most <= kNone) break;
    const int from = __ffs(__ballot_sync(0xffffffffu, list[0] == most)) - 1;
    if (kPer > 1 && s > 0 && (most ^ last) <= kLow) {
      const uint32_t a = __shfl_sync(0xffffffffu, pick(key, kLow - (last & kLow)), last_lane);
      const uint32_t b = __shfl_sync(0xffffffffu, pick(key, kLow - (most & kLow)), from);
      if (a != b) return choose_exactly<kPer>(key, top_k, lane);
    }
    if (lane == s) my_id = static_cast<int>(kLow - (most & kLow)) * 32 + from;
    last = most;
    last_lane = from;
    if (lane == from) {
#pragma unroll
      for (int j = 0; j < kPer - 1; ++j) list[j] = list[j + 1];
      list[kPer - 1] = 0;
    }
  }
  return lane < top_k ? my_id : -1;
}

__device__ __forceinline__ float logit(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ float logit(const float* p) { return __ldg(p); }

// Which groups stay: the rank of a group is the sum of its two largest choices. A group's
// experts are read out of shared memory by 32 / (groups rounded up to a power of two) lanes.
__device__ __forceinline__ uint32_t kept_groups(const RouteParams& p, const float* choice,
                                                int lane) {
  int span = 32;  // lanes per group
  while (span * p.groups > 32) span >>= 1;
  const int g = lane / span, part = lane % span;
  float a = -INFINITY, b = -INFINITY;  // the two largest
  if (g < p.groups) {
    for (int i = part; i < p.group_size; i += span) {
      const float c = choice[g * p.group_size + i];
      b = fmaxf(b, fminf(a, c));
      a = fmaxf(a, c);
    }
  }
  for (int o = span >> 1; o > 0; o >>= 1) {
    const float a2 = __shfl_xor_sync(0xffffffffu, a, o), b2 = __shfl_xor_sync(0xffffffffu, b, o);
    b = fmaxf(fminf(a, a2), fmaxf(b, b2));
    a = fmaxf(a, a2);
  }
  const float rank = p.group_size > 1 ? a + b : a;
  // this lane's group (lane index = group) against every other
  const float mine = __shfl_sync(0xffffffffu, rank, (lane * span) & 31);
  int better = 0;
  for (int h = 0; h < p.groups; ++h) {
    const float other = __shfl_sync(0xffffffffu, rank, h * span);
    better += (other > mine || (other == mine && h < lane)) ? 1 : 0;
  }
  return __ballot_sync(0xffffffffu, lane < p.groups && better < p.top_groups);
}

// What a lane knows of its experts j * 32 + lane, whatever the token.
template <int kPer>
struct LaneExperts {
  float bias[kPer];      // 0 without a bias
  uint32_t group[kPer];  // bit of the expert's group; 0: no such expert
};

template <int kPer>
__device__ __forceinline__ LaneExperts<kPer> lane_experts(const RouteParams& p, int lane) {
  LaneExperts<kPer> x;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int e = j * 32 + lane;
    x.bias[j] = p.bias != nullptr && e < p.experts ? p.bias[e] : 0.f;
    x.group[j] = e < p.experts ? 1u << (e / p.group_size) : 0u;
  }
  return x;
}

// One token by one warp. kPer: experts per lane. Returns the id of slot `lane` (-1: none).
template <typename T, int kPer>
__device__ __forceinline__ int route_token(const RouteParams& p, const LaneExperts<kPer>& mine,
                                           int64_t token, float* choice_smem, int lane) {
  const T* l = static_cast<const T*>(p.logits) + token * p.logits_stride;
  const bool softmax = p.scoring == DARD_ROUTE_SOFTMAX;
  float choice[kPer];
  bool bad = false;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    choice[j] = mine.group[j] != 0 ? logit(l + j * 32 + lane) : -INFINITY;
    bad |= !(choice[j] < INFINITY);  // +inf or NaN
  }
  if (__any_sync(0xffffffffu, bad)) {
    if (lane == 0 && p.status) atomicOr(p.status, DARD_STATUS_INVALID_ROW);
    if (lane < p.top_k) {
      p.ids[token * p.top_k + lane] = -1;
      p.weights[token * p.top_k + lane] = 0.f;
    }
    return -1;
  }
  uint32_t on = 0;  // bit j: this lane's expert j exists and is on
#pragma unroll
  for (int j = 0; j < kPer; ++j) on |= choice[j] > -INFINITY ? 1u << j : 0u;
  float top = 0.f, total = 1.f;  // SOFTMAX: the largest logit, the sum of the exponentials
  if (softmax) {
    top = choice[0];
#pragma unroll
    for (int j = 1; j < kPer; ++j) top = fmaxf(top, choice[j]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (top == -INFINITY) top = 0.f;  // every expert is off
    total = 0.f;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      choice[j] = expf(choice[j] - top);
      total += choice[j];
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
    // Without a bias the exponentials are in the scores' order already (and the sums of two
    // in theirs), and only the chosen ones are divided, at the end.
    if (p.bias != nullptr) {
#pragma unroll
      for (int j = 0; j < kPer; ++j) choice[j] /= total;
    }
  } else {
#pragma unroll
    for (int j = 0; j < kPer; ++j) choice[j] = 1.f / (1.f + expf(-choice[j]));
  }
  uint32_t key[kPer];
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    choice[j] = on >> j & 1 ? choice[j] + mine.bias[j] : -INFINITY;  // (+ 0 without a bias)
    key[j] = order_key(choice[j]);
  }
  if (p.top_groups < p.groups) {
    __syncwarp();
#pragma unroll
    for (int j = 0; j < kPer; ++j)
      if (mine.group[j] != 0) choice_smem[j * 32 + lane] = choice[j];
    __syncwarp();
    const uint32_t keep = kept_groups(p, choice_smem, lane);
#pragma unroll
    for (int j = 0; j < kPer; ++j)
      if ((keep & mine.group[j]) == 0) key[j] = kNone;
  }
  const int my_id = choose<kPer>(key, p.top_k, lane);
  // the chosen experts' scores, from their logits again
  float weight = 0.f;
  if (my_id >= 0) {
    const float x = logit(l + my_id);
    weight = softmax ? expf(x - top) / total : 1.f / (1.f + expf(-x));
  }
  if (p.renormalise) {
    float sum = weight;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    weight = sum > 0.f ? weight / sum : 0.f;
  }
  if (lane < p.top_k) {
    p.ids[token * p.top_k + lane] = my_id;
    p.weights[token * p.top_k + lane] = weight * p.scale;
  }
  return my_id;
}

// Exclusive prefix sums over v[0 .. n) in shared memory, and their total in v[n], by the whole CTA
// (n at most its threads).
__device__ __forceinline__ void exclusive_scan(int32_t* v, int n, int32_t* warp_sums) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const int32_t x = static_cast<int>(threadIdx.x) < n ? v[threadIdx.x] : 0;
  int32_t s = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int32_t y = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += y;
  }
  if (lane == 31) warp_sums[warp] = s;
  __syncthreads();
  const int32_t w = lane < warps ? warp_sums[lane] : 0;
  const int32_t before = __reduce_add_sync(0xffffffffu, lane < warp ? w : 0);
  if (static_cast<int>(threadIdx.x) < n) v[threadIdx.x] = before + s - x;
  const int32_t all = __reduce_add_sync(0xffffffffu, w);
  if (threadIdx.x == 0) v[n] = all;
  __syncthreads();
}

// The pairs of `count` tokens from t0 on as warp w of kWarps sees them: the w-th run of `per` pairs (a
// multiple of 32). The ids of the first kHeld of 32 are held in registers, so that they can be
// on their way while something else is done.
constexpr int kHeld = 2;
struct WarpPairs {
  int64_t base;  // first pair of the CTA
  int i0, i1;    // this warp's, from there
  int id[kHeld];
};
template <int kWarps>
__device__ __forceinline__ WarpPairs warp_pairs(const RouteParams& p, int t0, int count) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  WarpPairs w;
  w.base = static_cast<int64_t>(t0) * p.top_k;
  const int pairs = count * p.top_k;
  const int per = ((pairs + kWarps - 1) / kWarps + 31) / 32 * 32;
  w.i0 = warp * per;
  w.i1 = min(pairs, w.i0 + per);
#pragma unroll
  for (int j = 0; j < kHeld; ++j) {
    const int i = w.i0 + 32 * j + lane;
    w.id[j] = i < w.i1 ? p.ids[w.base + i] : -1;
  }
  return w;
}

// Places of the CTA's pairs: next[b] is the place of its first pair of bucket b (expert, or
// `experts` for slots without one). Each warp counts its pairs (hist, zeros at the start), the counts
// are summed over the warps, then each warp places its pairs, 32 at a time, in order.
template <int kWarps>
__device__ __forceinline__ void place_pairs(const RouteParams& p, const WarpPairs& w,
                                            const int32_t* next, int32_t* hist) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, buckets = p.experts + 1;
  int32_t* mine = hist + warp * buckets;
  const auto id_of = [&](int step) {
    const int i = w.i0 + 32 * step + lane;
    return step == 0 ? w.id[0] : step == 1 ? w.id[1] : i < w.i1 ? p.ids[w.base + i] : -1;
  };
  const int steps = (w.i1 - w.i0 + 31) / 32;
  for (int s = 0; s < steps; ++s) {
    const int id = id_of(s);
    if (w.i0 + 32 * s + lane < w.i1) atomicAdd(&mine[id < 0 ? p.experts : id], 1);
  }
  __syncthreads();
  for (int b = threadIdx.x; b < buckets; b += blockDim.x) {
    int32_t at = next[b];
#pragma unroll 1
    for (int w0 = 0; w0 < kWarps; w0 += 8) {
      int32_t n[8];
#pragma unroll
      for (int v = 0; v < 8; ++v) n[v] = hist[(w0 + v) * buckets + b];
#pragma unroll
      for (int v = 0; v < 8; ++v) {
        hist[(w0 + v) * buckets + b] = at;
        at += n[v];
      }
    }
  }
  __syncthreads();
  for (int s = 0; s < steps; ++s) {
    const int i = w.i0 + 32 * s + lane;
    const bool in = i < w.i1;
    const int id = id_of(s);
    const int b = !in ? buckets : id < 0 ? p.experts : id;
    const uint32_t same = __match_any_sync(0xffffffffu, b);
    const int rank = __popc(same & ((1u << lane) - 1));
    if (in) p.rows[mine[b] + rank] = id < 0 ? -1 : static_cast<int32_t>(w.base) + i;
    __syncwarp();
    if (in && rank == 0) mine[b] += __popc(same);
    __syncwarp();
  }
}

template <typename T, int kPer>
__global__ void __launch_bounds__(32 * route_warps(kPer), 1)
    route_topk(const __grid_constant__ RouteParams p) {
  grid_dep_launch();  // what follows may be scheduled; it waits for this grid's end
  constexpr int kWarps = route_warps(kPer);
  extern __shared__ int32_t smem[];
  // choices of each warp's token (groups only), then the counts, then one CTA's buckets
  float* choice = reinterpret_cast<float*>(smem);
  int32_t* count = smem + (p.top_groups < p.groups ? kWarps * p.experts : 0);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int t0 = blockIdx.x * p.cta_tokens, count_t = min(p.cta_tokens, p.tokens - t0);
  const bool plan = p.rows != nullptr;
  if (plan) {
    for (int i = threadIdx.x; i <= p.experts; i += blockDim.x) count[i] = 0;
    __syncthreads();
  }
  const LaneExperts<kPer> mine = lane_experts<kPer>(p, lane);
  for (int t = warp; t < count_t; t += kWarps) {
    const int id = route_token<T, kPer>(p, mine, t0 + t, choice + warp * p.experts, lane);
    if (plan && lane < p.top_k) atomicAdd(&count[id < 0 ? p.experts : id], 1);
  }
  if (!plan) return;
  __syncthreads();
  if (p.ctas > 1) {
    const int row = count_row(p.experts);
    for (int i = threadIdx.x; i < row; i += blockDim.x)
      p.counts[static_cast<int64_t>(blockIdx.x) * row + i] = i <= p.experts ? count[i] : 0;
    return;
  }
  // one CTA: its counts are the totals
  __shared__ int32_t warp_sums[kWarps];
  int32_t* hist = count + p.experts + 1;
  for (int i = threadIdx.x; i < kWarps * (p.experts + 1); i += blockDim.x) hist[i] = 0;
  const WarpPairs pairs = warp_pairs<kWarps>(p, t0, count_t);
  exclusive_scan(count, p.experts, warp_sums);
  for (int i = threadIdx.x; i <= p.experts; i += blockDim.x) p.offsets[i] = count[i];
  place_pairs<kWarps>(p, pairs, count, hist);
}

// Every CTA adds up, per bucket, the counts of all CTAs and of those before it (each thread four
// buckets of every kRuns-th CTA, its loads in flight together), then places its own pairs.
__global__ void __launch_bounds__(32 * kPlanWarps)
    plan_scatter(const __grid_constant__ RouteParams p) {
  extern __shared__ int32_t smem[];
  __shared__ int32_t warp_sums[kPlanWarps];
  const int buckets = p.experts + 1, row = count_row(p.experts), quads = row / 4;
  int32_t* next = smem;          // [row] totals, then places
  int32_t* before = next + row;  // [row] pairs of the CTAs before this one
  int32_t* hist = before + row;  // [kPlanWarps][buckets]
  for (int i = threadIdx.x; i < 2 * row + kPlanWarps * buckets; i += blockDim.x) next[i] = 0;
  __syncthreads();
  grid_dep_launch();  // (what follows waits for this grid's end before it reads the plan)
  const int runs = blockDim.x / quads, run = threadIdx.x / quads, quad = threadIdx.x % quads;
  const int t0 = blockIdx.x * p.cta_tokens, count_t = min(p.cta_tokens, p.tokens - t0);
  grid_dep_wait();
  const WarpPairs pairs = warp_pairs<kPlanWarps>(p, t0, count_t);
  if (run < runs) {
    int4 total = make_int4(0, 0, 0, 0), prior = total;
    const int4* c = reinterpret_cast<const int4*>(p.counts) + quad;
#pragma unroll 16
    for (int i = run; i < p.ctas; i += runs) {
      const int4 n = c[static_cast<int64_t>(i) * quads];
      const bool b = i < static_cast<int>(blockIdx.x);
      total.x += n.x; total.y += n.y; total.z += n.z; total.w += n.w;
      prior.x += b ? n.x : 0; prior.y += b ? n.y : 0; prior.z += b ? n.z : 0; prior.w += b ? n.w : 0;
    }
    atomicAdd(&next[4 * quad], total.x);
    atomicAdd(&next[4 * quad + 1], total.y);
    atomicAdd(&next[4 * quad + 2], total.z);
    atomicAdd(&next[4 * quad + 3], total.w);
    atomicAdd(&before[4 * quad], prior.x);
    atomicAdd(&before[4 * quad + 1], prior.y);
    atomicAdd(&before[4 * quad + 2], prior.z);
    atomicAdd(&before[4 * quad + 3], prior.w);
  }
  __syncthreads();
  exclusive_scan(next, p.experts, warp_sums);
  if (static_cast<int>(threadIdx.x) < buckets) {
    if (blockIdx.x == 0) p.offsets[threadIdx.x] = next[threadIdx.x];
    next[threadIdx.x] += before[threadIdx.x];
  }
  __syncthreads();
  place_pairs<kPlanWarps>(p, pairs, next, hist);
}

// With no token at all every expert's run is empty.
__global__ void empty_plan(int32_t* offsets, int n) {
  for (int i = threadIdx.x; i < n; i += blockDim.x) offsets[i] = 0;
}

// (up to 2^31 - 1 tokens: no sum of two counts in 32 bits, here or in the kernels)
int ceil_div(int64_t n, int d) { return static_cast<int>((n + d - 1) / d); }

// Tokens per CTA: one CTA up to kOneCtaTokens; beyond, runs such that every SM gets one CTA of
// each kernel, so that plan_scatter's sums over the CTAs before it stay short.
int cta_tokens_for(int tokens) {
  if (tokens <= kOneCtaTokens) return std::max(tokens, 1);
  return std::max(32, ceil_div(tokens, sm_count()));
}

// The workspace of a plan that this many CTAs make.
size_t counts_bytes(int ctas, int experts) {
  return ctas <= 1 ? 0 : static_cast<size_t>(ctas) * count_row(experts) * 4;
}

template <typename T, int kPer>
cudaError_t launch_typed(const RouteParams& p, cudaStream_t s) {
  const size_t buckets = static_cast<size_t>(p.experts) + 1;
  const bool plan = p.rows != nullptr;
  constexpr int kWarps = route_warps(kPer);
  constexpr size_t kMost = 100 * 1024;  // 32 warps' choices and buckets of 256 experts: 67 KB
  size_t ints = p.top_groups < p.groups ? static_cast<size_t>(kWarps) * p.experts : 0;
  if (plan) ints += buckets;
  if (plan && p.ctas == 1) ints += kWarps * buckets;
  if (ints * 4 > 48 * 1024) {
    static std::atomic<uint64_t> done{0};
    const cudaError_t e = ensure_smem_attr(route_topk<T, kPer>, kMost, done);
    if (e != cudaSuccess) return e;
  }
  route_topk<T, kPer><<<p.ctas, 32 * kWarps, ints * 4, s>>>(p);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess || !plan || p.ctas == 1) return e;
  const size_t plan_smem = (2 * static_cast<size_t>(count_row(p.experts)) + kPlanWarps * buckets) * 4;
  if (plan_smem > 48 * 1024) {
    static std::atomic<uint64_t> done{0};
    e = ensure_smem_attr(plan_scatter, kMost, done);
    if (e != cudaSuccess) return e;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.ctas);
  cfg.blockDim = dim3(32 * kPlanWarps);
  cfg.dynamicSmemBytes = plan_smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, plan_scatter, p);
}

template <typename T>
cudaError_t launch_route(const RouteParams& p, cudaStream_t s) {
  // Experts per lane: empty ones cost as much as others (38912 tokens, 6 of 160: five per lane
  // 43.5 us, eight
  // 51.5; 5121 tokens: 16.6, 18.6; 20000 tokens, 8 of 384: twelve 60.5, sixteen 72.2).
  switch ((p.experts + 31) / 32) {
    case 1: return launch_typed<T, 1>(p, s);
    case 2: return launch_typed<T, 2>(p, s);
    case 3: return launch_typed<T, 3>(p, s);
    case 4: return launch_typed<T, 4>(p, s);
    case 5: return launch_typed<T, 5>(p, s);
    case 6: return launch_typed<T, 6>(p, s);
    case 7: return launch_typed<T, 7>(p, s);
    case 8: return launch_typed<T, 8>(p, s);
    case 9:
    case 10:
    case 11:
    case 12: return launch_typed<T, 12>(p, s);
    default: return launch_typed<T, 16>(p, s);
  }
}

bool sizes_ok(int64_t tokens, int64_t experts, int64_t top_k) {
  return tokens >= 0 && experts >= 1 && experts <= DARD_MAX_EXPERTS && top_k >= 1 &&
         top_k <= std::min<int64_t>(experts, DARD_MAX_TOP_K) && tokens * top_k <= 0x7fffffffll;
}

}  // namespace
}  // namespace dard

using namespace dard;

extern "C" {

size_t dard_route_workspace_size(int32_t tokens, int32_t experts, int32_t top_k) {
  if (!sizes_ok(tokens, experts, top_k) || tokens <= kOneCtaTokens) return 0;
  // The most CTAs of any count up to this one: past 32 tokens for each SM a CTA takes more, and
  // there may be fewer CTAs than for fewer tokens.
  return counts_bytes(std::min(ceil_div(tokens, 32), sm_count()), experts);
}

dard_status dard_route(const dard_route_args* a, void* stream) {
  report(DARD_OK, "%s", "");
  if (!a) return report(DARD_ERR_NULL, "args is NULL");
  if (a->experts < 1 || a->experts > DARD_MAX_EXPERTS)
    return report(DARD_ERR_SHAPE, "experts %d outside 1..%d", a->experts, DARD_MAX_EXPERTS);
  if (a->top_k < 1 || a->top_k > std::min(a->experts, DARD_MAX_TOP_K))
    return report(DARD_ERR_SHAPE, "top_k %d outside 1..min(experts, %d)", a->top_k, DARD_MAX_TOP_K);
  if (!sizes_ok(a->tokens, a->experts, a->top_k))
    return report(DARD_ERR_SHAPE, "tokens %d: below 0, or tokens * top_k above 2^31 - 1", a->tokens);
  if (a->groups < 1 || a->groups > DARD_MAX_GROUPS || a->experts % a->groups != 0)
    return report(DARD_ERR_SHAPE, "groups %d: outside 1..%d, or no divisor of experts %d", a->groups,
                  DARD_MAX_GROUPS, a->experts);
  if (a->top_groups < 1 || a->top_groups > a->groups)
    return report(DARD_ERR_SHAPE, "top_groups %d outside 1..groups %d", a->top_groups, a->groups);
  if (a->dtype != DARD_BF16 && a->dtype != DARD_F32)
    return report(DARD_ERR_VALUE, "dtype %d is neither DARD_F32 nor DARD_BF16", a->dtype);
  if (a->scoring != DARD_ROUTE_SOFTMAX && a->scoring != DARD_ROUTE_SIGMOID)
    return report(DARD_ERR_VALUE, "scoring %d is not a dard_route_scoring", a->scoring);
  if (a->renormalise != 0 && a->renormalise != 1)
    return report(DARD_ERR_VALUE, "renormalise must be 0 or 1");
  if (!std::isfinite(a->scale)) return report(DARD_ERR_VALUE, "scale must be finite");
  if (a->logits_stride < a->experts)
    return report(DARD_ERR_SHAPE, "logits_stride is below experts");
  if ((a->offsets == nullptr) != (a->rows == nullptr) && (a->tokens > 0 || !a->offsets))
    return report(DARD_ERR_NULL, "offsets and rows come together");
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool fail = std::getenv("DARD_TEST_FAIL_LAUNCH") != nullptr;  // test hook: no launch
  cudaError_t e = fail ? cudaErrorLaunchFailure : cudaSuccess;
  if (a->tokens == 0) {
    if (a->offsets && e == cudaSuccess) {
      empty_plan<<<1, 256, 0, s>>>(a->offsets, a->experts + 1);
      e = cudaGetLastError();
    }
    if (e != cudaSuccess)
      return report(DARD_ERR_CUDA, "routing launch failed: %s", cudaGetErrorString(e));
    return DARD_OK;
  }
  if (!a->logits || !a->ids || !a->weights)
    return report(DARD_ERR_NULL, "logits, ids or weights is NULL");
  if (reinterpret_cast<uintptr_t>(a->logits) % (a->dtype == DARD_BF16 ? 2 : 4) != 0)
    return report(DARD_ERR_ALIGN, "logits is not a multiple of the element size");
  const int cta_tokens = cta_tokens_for(a->tokens), ctas = ceil_div(a->tokens, cta_tokens);
  const size_t need = a->rows ? counts_bytes(ctas, a->experts) : 0;
  if (need > 0 && (!a->workspace || a->workspace_bytes < need))
    return report(DARD_ERR_WORKSPACE, "workspace of %zu bytes needed", need);
  if (need > 0 && reinterpret_cast<uintptr_t>(a->workspace) % 16 != 0)
    return report(DARD_ERR_ALIGN, "workspace must be 16-byte aligned");
  RouteParams p = {};
  p.logits = a->logits;
  p.bias = a->bias;
  p.ids = a->ids;
  p.weights = a->weights;
  p.offsets = a->offsets;
  p.rows = a->rows;
  p.status = a->status;
  p.counts = static_cast<int32_t*>(a->workspace);
  p.logits_stride = a->logits_stride;
  p.tokens = a->tokens;
  p.experts = a->experts;
  p.top_k = a->top_k;
  p.groups = a->groups;
  p.top_groups = a->top_groups;
  p.group_size = a->experts / a->groups;
  p.scoring = a->scoring;
  p.renormalise = a->renormalise;
  p.cta_tokens = cta_tokens;
  p.ctas = ctas;
  p.scale = a->scale;
  if (e == cudaSuccess)
    e = a->dtype == DARD_BF16 ? launch_route<__nv_bfloat16>(p, s) : launch_route<float>(p, s);
  if (e != cudaSuccess)
    return report(DARD_ERR_CUDA, "routing launch failed: %s", cudaGetErrorString(e));
  return DARD_OK;
}

}  // extern "C"
