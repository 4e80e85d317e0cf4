// dard_route.cu - dard_route: each token's experts and weights from its router logits, and the
// plan (the (token, slot) pairs sorted by expert) that dard_experts reads on the device.
//
// route_topk, one warp per token: lane l holds experts l, l + 32, ... in registers as keys
// whose unsigned order is the order of the choice; a slot is one warp-wide maximum of the keys
// and one minimum of the indices that reach it (ties to the lowest index). The largest
// call (38912 x 256 logits, 40 MB) is bound by these dependent rounds, not by HBM.
//
// The plan is a stable counting sort. A CTA owns a run of consecutive tokens; route_topk
// counts its pairs per expert, and plan_scatter (chained by programmatic dependent launch)
// adds up the counts of the CTAs before it and gives every pair its place. Counts are integers
// and places follow from them, so the plan does not depend on the order of execution. Few
// tokens fit one CTA, which then writes the plan itself, in one launch.
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

constexpr int kRouteWarps = 16;                // route_topk
constexpr int kRouteThreads = 32 * kRouteWarps;
constexpr int kPlanWarps = 8;                  // plan_scatter
constexpr int kOneCtaTokens = 64;              // one CTA routes and plans up to this many
constexpr uint32_t kNone = 0;                  // key of an expert that cannot be chosen

struct RouteParams {
  const void* logits;
  const float* bias;
  int32_t* ids;
  float* weights;
  int32_t* offsets;
  int32_t* rows;
  uint32_t* status;
  int32_t* counts;        // workspace [ctas][experts + 1]; the last: slots without an expert
  int64_t logits_stride;
  int32_t tokens, experts, top_k, groups, top_groups, group_size;
  int32_t scoring, renormalise;
  int32_t cta_tokens;     // consecutive tokens of a CTA (both kernels)
  int32_t ctas;
  float scale;
};

// Unsigned order = float order, every finite float above kNone.
__device__ __forceinline__ uint32_t order_key(float f) {
  const uint32_t b = __float_as_uint(f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
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

// One token by one warp. kPer: experts per lane. Returns the id of slot `lane` (-1: none).
template <typename T, int kPer>
__device__ __forceinline__ int route_token(const RouteParams& p, int64_t token, float* choice_smem,
                                           int lane) {
  const T* l = static_cast<const T*>(p.logits) + token * p.logits_stride;
  float score[kPer];
  uint32_t key[kPer];
  bool bad = false;
  float top = -INFINITY;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int e = j * 32 + lane;
    score[j] = e < p.experts ? logit(l + e) : -INFINITY;
    bad |= !(score[j] < INFINITY);  // +inf or NaN
    top = fmaxf(top, score[j]);
  }
  bad = __any_sync(0xffffffffu, bad);
  if (bad) {
    if (lane == 0 && p.status) atomicOr(p.status, DARD_STATUS_INVALID_ROW);
    if (lane < p.top_k) {
      p.ids[token * p.top_k + lane] = -1;
      p.weights[token * p.top_k + lane] = 0.f;
    }
    return -1;
  }
  float total = 0.f;  // SOFTMAX: the sum of the exponentials
  if (p.scoring == DARD_ROUTE_SOFTMAX) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (top == -INFINITY) top = 0.f;  // every expert is off
  }
  uint32_t off = 0;  // bit j: this lane's expert j is off (or does not exist)
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    if (score[j] == -INFINITY) off |= 1u << j;
    if (p.scoring == DARD_ROUTE_SOFTMAX) {
      score[j] = expf(score[j] - top);
      total += score[j];
    } else {
      score[j] = 1.f / (1.f + expf(-score[j]));
    }
  }
  if (p.scoring == DARD_ROUTE_SOFTMAX) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
    // Without a bias the exponentials are in the scores' order already (and the sums of two
    // in theirs), and the chosen ones are divided at the end.
    if (p.bias != nullptr) {
#pragma unroll
      for (int j = 0; j < kPer; ++j) score[j] /= total;
      total = 1.f;
    }
  } else {
    total = 1.f;
  }
  float choice[kPer];
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int e = j * 32 + lane;
    choice[j] = score[j];
    if (p.bias != nullptr && e < p.experts) choice[j] += __ldg(p.bias + e);
    if (off >> j & 1) choice[j] = -INFINITY;
    key[j] = choice[j] > -INFINITY ? order_key(choice[j]) : kNone;  // a NaN bias: never chosen
  }
  if (p.top_groups < p.groups) {
    __syncwarp();
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int e = j * 32 + lane;
      if (e < p.experts) choice_smem[e] = key[j] == kNone ? -INFINITY : choice[j];
    }
    __syncwarp();
    const uint32_t keep = kept_groups(p, choice_smem, lane);
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int e = j * 32 + lane;
      if (e < p.experts && !(keep >> (e / p.group_size) & 1)) key[j] = kNone;
    }
  }
  int my_id = -1;        // slot `lane`
  float my_weight = 0.f;
  for (int s = 0; s < p.top_k; ++s) {
    uint32_t best = key[0];
#pragma unroll
    for (int j = 1; j < kPer; ++j) best = max(best, key[j]);
    const uint32_t most = __reduce_max_sync(0xffffffffu, best);
    if (most == kNone) break;  // no expert is left
    int e = INT_MAX;
    float w = 0.f;
#pragma unroll
    for (int j = kPer - 1; j >= 0; --j) {
      if (key[j] == most) {
        e = j * 32 + lane;
        w = score[j];
      }
    }
    const int first = __reduce_min_sync(0xffffffffu, e);
    w = __shfl_sync(0xffffffffu, w, first & 31);
    if (lane == s) {
      my_id = first;
      my_weight = w;
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j)
      if (first == j * 32 + lane) key[j] = kNone;
  }
  if (p.renormalise) {  // the softmax's own division cancels
    float sum = my_weight;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    my_weight = sum > 0.f ? my_weight / sum : 0.f;
  } else if (my_id >= 0) {
    my_weight /= total;
  }
  if (lane < p.top_k) {
    p.ids[token * p.top_k + lane] = my_id;
    p.weights[token * p.top_k + lane] = my_weight * p.scale;
  }
  return my_id;
}

// Exclusive prefix sums over n <= 1024 values in shared memory, by the whole CTA.
__device__ void exclusive_scan(int32_t* v, int n, int32_t* warp_sums) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  int32_t carry = 0;
  for (int base = 0; base < n; base += blockDim.x) {
    const int i = base + threadIdx.x;
    const int32_t x = i < n ? v[i] : 0;
    int32_t s = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int32_t y = __shfl_up_sync(0xffffffffu, s, o);
      if (lane >= o) s += y;
    }
    if (lane == 31) warp_sums[warp] = s;
    __syncthreads();
    int32_t before = carry;
    for (int w = 0; w < warps; ++w) {
      const int32_t ws = warp_sums[w];
      if (w < warp) before += ws;
      carry += ws;
    }
    if (i < n) v[i] = before + s - x;
    __syncthreads();
  }
}

// Places of the pairs of tokens [t0, t1): next[b] is the place of the CTA's first pair of
// bucket b (expert, or `experts` for slots without one). Warp w takes the w-th run of pairs:
// it counts them (hist), the runs' counts are summed over the warps, then it places them, 32
// at a time, in order. Every warp of the CTA takes part; `warps` of them have pairs.
__device__ void place_pairs(const RouteParams& p, int t0, int t1, const int32_t* next,
                            int32_t* hist, int warps) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, buckets = p.experts + 1;
  for (int i = threadIdx.x; i < warps * buckets; i += blockDim.x) hist[i] = 0;
  __syncthreads();
  const int64_t base = static_cast<int64_t>(t0) * p.top_k;
  const int pairs = (t1 - t0) * p.top_k;
  const int per = ((pairs + warps - 1) / warps + 31) / 32 * 32;
  const int i0 = warp * per, i1 = min(pairs, i0 + per);
  int32_t* mine = hist + warp * buckets;
  if (warp < warps) {
    for (int i = i0 + lane; i < i1; i += 32) {
      const int id = p.ids[base + i];
      atomicAdd(&mine[id < 0 ? p.experts : id], 1);
    }
  }
  __syncthreads();
  for (int b = threadIdx.x; b < buckets; b += blockDim.x) {
    int32_t at = next[b];
    for (int w = 0; w < warps; ++w) {
      const int32_t n = hist[w * buckets + b];
      hist[w * buckets + b] = at;
      at += n;
    }
  }
  __syncthreads();
  if (warp < warps) {
    for (int i = i0; i < i1; i += 32) {
      const bool in = i + lane < i1;
      const int id = in ? p.ids[base + i + lane] : -1;
      const int b = !in ? buckets : id < 0 ? p.experts : id;
      const uint32_t same = __match_any_sync(0xffffffffu, b);
      const int rank = __popc(same & ((1u << lane) - 1));
      if (in) p.rows[mine[b] + rank] = id < 0 ? -1 : static_cast<int32_t>(base) + i + lane;
      __syncwarp();
      if (in && rank == 0) mine[b] += __popc(same);
      __syncwarp();
    }
  }
}

template <typename T, int kPer>
__global__ void __launch_bounds__(kRouteThreads) route_topk(const __grid_constant__ RouteParams p) {
  grid_dep_launch();  // plan_scatter may be scheduled; it waits for this grid's end
  extern __shared__ int32_t smem[];
  // choices of each warp's token (groups only), then the counts, then one_cta's buckets
  float* choice = reinterpret_cast<float*>(smem);
  const bool grouped = p.top_groups < p.groups;
  int32_t* count = smem + (grouped ? kRouteWarps * p.experts : 0);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int t0 = blockIdx.x * p.cta_tokens, t1 = min(p.tokens, t0 + p.cta_tokens);
  const bool plan = p.rows != nullptr;
  if (plan) {
    for (int i = threadIdx.x; i <= p.experts; i += kRouteThreads) count[i] = 0;
    __syncthreads();
  }
  for (int t = t0 + warp; t < t1; t += kRouteWarps) {
    const int id = route_token<T, kPer>(p, t, choice + warp * p.experts, lane);
    if (plan && lane < p.top_k) atomicAdd(&count[id < 0 ? p.experts : id], 1);
  }
  if (!plan) return;
  __syncthreads();
  if (p.ctas > 1) {
    for (int i = threadIdx.x; i <= p.experts; i += kRouteThreads)
      p.counts[static_cast<int64_t>(blockIdx.x) * (p.experts + 1) + i] = count[i];
    return;
  }
  // one CTA: its counts are the totals
  __shared__ int32_t warp_sums[kRouteWarps];
  exclusive_scan(count, p.experts + 1, warp_sums);
  for (int i = threadIdx.x; i <= p.experts; i += kRouteThreads) p.offsets[i] = count[i];
  place_pairs(p, t0, t1, count, count + p.experts + 1, kPlanWarps);
}

__global__ void __launch_bounds__(32 * kPlanWarps)
    plan_scatter(const __grid_constant__ RouteParams p) {
  extern __shared__ int32_t smem[];
  __shared__ int32_t warp_sums[kPlanWarps];
  const int buckets = p.experts + 1;
  int32_t* next = smem;             // [buckets] totals, then places
  int32_t* before = next + buckets; // [buckets] pairs of the CTAs before this one
  int32_t* hist = before + buckets; // [kPlanWarps][buckets]
  grid_dep_wait();
  for (int b = threadIdx.x; b < buckets; b += blockDim.x) {
    int32_t total = 0, prior = 0;
    const int32_t* c = p.counts + b;
#pragma unroll 8
    for (int i = 0; i < p.ctas; ++i) {
      const int32_t n = c[static_cast<int64_t>(i) * buckets];
      total += n;
      if (i < static_cast<int>(blockIdx.x)) prior += n;
    }
    next[b] = total;
    before[b] = prior;
  }
  __syncthreads();
  exclusive_scan(next, buckets, warp_sums);
  for (int b = threadIdx.x; b < buckets; b += blockDim.x) {
    if (blockIdx.x == 0) p.offsets[b] = next[b];
    next[b] += before[b];
  }
  __syncthreads();
  const int t0 = blockIdx.x * p.cta_tokens, t1 = min(p.tokens, t0 + p.cta_tokens);
  place_pairs(p, t0, t1, next, hist, kPlanWarps);
}

// With no token at all every expert's run is empty.
__global__ void empty_plan(int32_t* offsets, int n) {
  for (int i = threadIdx.x; i < n; i += blockDim.x) offsets[i] = 0;
}

// Tokens per CTA: one CTA up to kOneCtaTokens; beyond, runs such that every SM gets one CTA of
// each kernel, so that plan_scatter's sums over the CTAs before it stay short.
int cta_tokens_for(int tokens) {
  if (tokens <= kOneCtaTokens) return std::max(tokens, 1);
  const int sms = sm_count();
  return std::max(kRouteWarps, (tokens + sms - 1) / sms);
}

template <typename T, int kPer>
cudaError_t launch_typed(const RouteParams& p, cudaStream_t s) {
  const size_t buckets = static_cast<size_t>(p.experts) + 1;
  const bool plan = p.rows != nullptr;
  size_t ints = p.top_groups < p.groups ? static_cast<size_t>(kRouteWarps) * p.experts : 0;
  if (plan) ints += buckets;
  if (plan && p.ctas == 1) ints += kPlanWarps * buckets;
  if (ints * 4 > 48 * 1024) {
    static std::atomic<uint64_t> done{0};
    const cudaError_t e = ensure_smem_attr(route_topk<T, kPer>, 64 * 1024, done);
    if (e != cudaSuccess) return e;
  }
  route_topk<T, kPer><<<p.ctas, kRouteThreads, ints * 4, s>>>(p);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess || !plan || p.ctas == 1) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.ctas);
  cfg.blockDim = dim3(32 * kPlanWarps);
  cfg.dynamicSmemBytes = (2 + kPlanWarps) * buckets * 4;
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
  if (p.experts <= 32) return launch_typed<T, 1>(p, s);
  if (p.experts <= 64) return launch_typed<T, 2>(p, s);
  if (p.experts <= 128) return launch_typed<T, 4>(p, s);
  if (p.experts <= 256) return launch_typed<T, 8>(p, s);
  return launch_typed<T, 16>(p, s);
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
  if (!sizes_ok(tokens, experts, top_k)) return 0;
  const int per = cta_tokens_for(tokens);
  const size_t ctas = (static_cast<size_t>(tokens) + per - 1) / per;
  return ctas <= 1 ? 0 : ctas * (static_cast<size_t>(experts) + 1) * 4;
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
  const size_t need = a->rows ? dard_route_workspace_size(a->tokens, a->experts, a->top_k) : 0;
  if (need > 0 && (!a->workspace || a->workspace_bytes < need))
    return report(DARD_ERR_WORKSPACE, "workspace of %zu bytes needed", need);
  if (need > 0 && reinterpret_cast<uintptr_t>(a->workspace) % 4 != 0)
    return report(DARD_ERR_ALIGN, "workspace must be 4-byte aligned");
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
  p.cta_tokens = cta_tokens_for(a->tokens);
  p.ctas = (a->tokens + p.cta_tokens - 1) / p.cta_tokens;
  p.scale = a->scale;
  if (e == cudaSuccess)
    e = a->dtype == DARD_BF16 ? launch_route<__nv_bfloat16>(p, s) : launch_route<float>(p, s);
  if (e != cudaSuccess)
    return report(DARD_ERR_CUDA, "routing launch failed: %s", cudaGetErrorString(e));
  return DARD_OK;
}

}  // extern "C"
