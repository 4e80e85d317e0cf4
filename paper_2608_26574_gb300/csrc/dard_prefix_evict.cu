// dard_prefix_evict.cu - the keys of a shared prefix to keep, by their accumulated attention weight
// (dard_prefix_evict): per key/value head the largest weights between the fixed ends, in rising
// order of their index, and the kept rows of K and V moved together.
//
// evict_select: one cluster of CTAs per head; each warp owns a run of the candidates. Weights map
// to unsigned keys in the same order; three rounds of 11, 11 and 10 bits (a radix selection: count
// each digit's values among the candidates that share the digits so far, take the digit in which
// the count from the top passes the number wanted) find the smallest kept key and how many of its
// equals are kept. The CTAs of a cluster add their counts up in the shared memory of the first, which
// finds the digit with one scan over its threads. Then each warp counts its kept candidates, a scan
// over warps and CTAs places them, and ballots place each within its warp. Nothing depends on the
// order of the atomics: they only count. Bound by the barriers of the rounds (two of the cluster
// each) and, of long rows, by the passes over them (five; four loads of a lane in flight: 29 -> 26 us for
// 32 heads of 65537 weights, 8 MB), not by their bytes; 5 us for 704.
// evict_copy: 16 bytes of K and of V per thread and step, rows in the order of the outputs.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "dard_attn_common.cuh"

namespace dard {
namespace {

struct EvictParams {
  const float* w;
  const uint4* k;
  const uint4* v;
  int32_t* kept;
  uint4* k_out;
  uint4* v_out;
  float* w_out;
  int64_t w_stride;
  int64_t row, head, out_row, out_head;  // strides in 16-byte units
  int32_t hkv, prefix_len, keep, first, last;
  int32_t chunks;  // 16-byte chunks of a row
};

constexpr int kSelThreads = 1024, kSelWarps = 32;
constexpr int kBins = 2048;
constexpr int kMaxCluster = 8;
constexpr int kAhead = 4;  // a lane's weights in flight

// Order-preserving: a larger weight has a larger key; -0 as 0, NaN below everything.
__device__ __forceinline__ uint32_t key_of(float w) {
  if (w != w) return 0u;
  const uint32_t b = __float_as_uint(w == 0.f ? 0.f : w);
  return b & 0x80000000u ? ~b : b | 0x80000000u;  // at least 0x007fffff (-inf)
}

struct SelShared {
  uint32_t hist[2][kBins];        // one for every other round
  uint32_t warp_sum[kSelWarps];
  uint32_t warp_gt[kSelWarps], warp_eq[kSelWarps];
  uint32_t cta_gt, cta_eq;        // this CTA's counts
  uint32_t base_gt, base_eq;      // those of the cluster's earlier CTAs
  uint32_t digit, above;          // the round's result
};

__device__ __forceinline__ void add_cluster(uint32_t* p, uint32_t rank, uint32_t v) {
  asm volatile("red.relaxed.cluster.shared::cluster.add.u32 [%0], %1;" ::"r"(map_shared_rank(smem_u32(p), rank)),
               "r"(v)
               : "memory");
}
__device__ __forceinline__ void st_cluster(uint32_t* p, uint32_t rank, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(map_shared_rank(smem_u32(p), rank)), "r"(v) : "memory");
}
__device__ __forceinline__ uint32_t ld_cluster(const uint32_t* p, uint32_t rank) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(map_shared_rank(smem_u32(p), rank)) : "memory");
  return v;
}

// All threads of the cluster; shared memory written before is seen by all of them.
__device__ __forceinline__ void sync_head(int ctas) {
  __syncthreads();
  if (ctas > 1) cluster_sync();
}

__global__ void __launch_bounds__(kSelThreads, 1) evict_select(const __grid_constant__ EvictParams p,
                                                               int ctas) {
  __shared__ SelShared sh;
  grid_dep_launch();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int g = blockIdx.x / ctas, rank = blockIdx.x % ctas;
  const float* w = p.w + g * p.w_stride;
  int32_t* kept = p.kept + static_cast<int64_t>(g) * p.keep;
  float* w_out = p.w_out ? p.w_out + static_cast<int64_t>(g) * p.keep : nullptr;
  const int lo = p.first, hi = p.prefix_len - p.last;  // candidates
  const int want = p.keep - p.first - p.last;
  // the fixed ends
  for (int i = rank * kSelThreads + tid; i < p.first + p.last; i += ctas * kSelThreads) {
    const int at = i < p.first ? i : p.prefix_len - p.last + (i - p.first);
    const int to = i < p.first ? i : p.keep - p.last + (i - p.first);
    kept[to] = at;
    if (w_out) w_out[to] = w[at];
  }
  if (want == 0) return;  // (the same for the whole cluster)
  // this warp's run of candidates
  const long long n = hi - lo, units = static_cast<long long>(ctas) * kSelWarps;
  const long long unit = static_cast<long long>(rank) * kSelWarps + warp;
  const int a = lo + static_cast<int>(n * unit / units), b = lo + static_cast<int>(n * (unit + 1) / units);

  // f(index, weight, whether there is one) for the run, 32 at a time in order; kAhead loads in flight
  auto each = [&](auto f) {
    for (int i0 = a; i0 < b; i0 += 32 * kAhead) {
      float x[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int i = i0 + 32 * u + lane;
        x[u] = i < b ? __ldg(w + i) : 0.f;
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (i0 + 32 * u >= b) break;
        const int i = i0 + 32 * u + lane;
        f(i, x[u], i < b);
      }
    }
  };

  uint32_t prefix = 0, need = want;  // digits found so far; how many of their candidates are kept
  for (int i = tid; i < 2 * kBins; i += kSelThreads) sh.hist[0][i] = 0;
  sync_head(ctas);
#pragma unroll 1
  for (int round = 0; round < 3; ++round) {
    const int shift = round == 0 ? 21 : round == 1 ? 10 : 0, bins = round == 2 ? 1024 : 2048;
    const uint32_t done = round == 0 ? 0u : round == 1 ? 0xffe00000u : 0xfffffc00u;
    uint32_t* hist = sh.hist[round & 1];
    each([&](int, float x, bool in) {
      const uint32_t key = key_of(x);
      if (in && (key & done) == prefix) atomicAdd(&hist[key >> shift & (bins - 1)], 1u);
    });
    if (ctas > 1) {
      __syncthreads();
      if (rank != 0)
        for (int i = tid; i < bins; i += kSelThreads) {
          const uint32_t c = hist[i];
          if (c) add_cluster(&hist[i], 0, c);
        }
    }
    sync_head(ctas);
    if (rank == 0) {
      // thread t takes the two digits bins - 1 - 2t and bins - 2 - 2t: the first digit, from the
      // largest down, at which the count reaches `need`
      const int top = bins - 1 - 2 * tid;
      const uint32_t c0 = top > 0 ? hist[top] : 0u, c1 = top > 0 ? hist[top - 1] : 0u;
      uint32_t scan = c0 + c1;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t x = __shfl_up_sync(0xffffffffu, scan, o);
        if (lane >= o) scan += x;
      }
      if (lane == 31) sh.warp_sum[warp] = scan;
      __syncthreads();
      uint32_t before = lane < warp ? sh.warp_sum[lane] : 0u;
      before = __reduce_add_sync(0xffffffffu, before) + scan - c0 - c1;
      if (before < need && before + c0 + c1 >= need) {  // one thread
        const bool second = before + c0 < need;
        for (int c = 0; c < ctas; ++c) {
          st_cluster(&sh.digit, c, static_cast<uint32_t>(second ? top - 1 : top));
          st_cluster(&sh.above, c, second ? before + c0 : before);
        }
      }
    }
    // (the counts have been read or added up) room for the next round but one
    for (int i = tid; i < bins; i += kSelThreads) hist[i] = 0;
    sync_head(ctas);
    need -= sh.above;
    prefix |= sh.digit << shift;
  }
  // `prefix` is the smallest kept key, of which the first `need` are kept
  uint32_t gt = 0, eq = 0;
  each([&](int, float x, bool in) {
    const uint32_t key = key_of(x);
    gt += in && key > prefix;
    eq += in && key == prefix;
  });
  gt = __reduce_add_sync(0xffffffffu, gt);
  eq = __reduce_add_sync(0xffffffffu, eq);
  if (lane == 0) {
    sh.warp_gt[warp] = gt;
    sh.warp_eq[warp] = eq;
  }
  __syncthreads();
  if (warp == 0) {
    const uint32_t x = sh.warp_gt[lane], y = sh.warp_eq[lane];
    uint32_t sx = x, sy = y;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t ux = __shfl_up_sync(0xffffffffu, sx, o), uy = __shfl_up_sync(0xffffffffu, sy, o);
      if (lane >= o) { sx += ux; sy += uy; }
    }
    sh.warp_gt[lane] = sx - x;
    sh.warp_eq[lane] = sy - y;
    if (lane == 31) {
      sh.cta_gt = sx;
      sh.cta_eq = sy;
    }
  }
  sync_head(ctas);
  if (tid == 0) {
    uint32_t bx = 0, by = 0;
    for (int c = 0; c < rank; ++c) {
      bx += ld_cluster(&sh.cta_gt, c);
      by += ld_cluster(&sh.cta_eq, c);
    }
    sh.base_gt = bx;
    sh.base_eq = by;
  }
  sync_head(ctas);
  eq = sh.base_eq + sh.warp_eq[warp];
  int at = p.first + static_cast<int>(sh.base_gt + sh.warp_gt[warp] + min(eq, need));  // the next kept key's place
  const uint32_t below = (1u << lane) - 1;
  each([&](int i, float x, bool in) {
    const uint32_t key = key_of(x);
    bool take = in && key > prefix;
    const uint32_t equal = __ballot_sync(0xffffffffu, in && key == prefix);
    if (equal != 0) {
      take |= (equal >> lane & 1u) && eq + __popc(equal & below) < need;
      eq += __popc(equal);
    }
    const uint32_t taken = __ballot_sync(0xffffffffu, take);
    const int to = at + __popc(taken & below);
    if (take && to < p.keep - p.last) {  // (always, unless the weights change under the call)
      kept[to] = i;
      if (w_out) w_out[to] = x;
    }
    at += __popc(taken);
  });
}

// Each thread moves the same 16-byte chunk of kRowsPer consecutive output rows' K and V: kRowsPer
// independent loads of each in flight: 537 MB in 78 us, the copy's rate.
constexpr int kCopyThreads = 256, kRowsPer = 4;

__global__ void __launch_bounds__(kCopyThreads) evict_copy(const __grid_constant__ EvictParams p) {
  grid_dep_wait();
  const long long idx = static_cast<long long>(blockIdx.x) * kCopyThreads + threadIdx.x;
  const int c = static_cast<int>(idx % p.chunks);
  const long long rest = idx / p.chunks;
  const int g = static_cast<int>(rest % p.hkv);
  const long long i0 = rest / p.hkv * kRowsPer;
  if (i0 >= p.keep) return;
  const int32_t* kept = p.kept + static_cast<int64_t>(g) * p.keep;
  uint4 k[kRowsPer], v[kRowsPer];
#pragma unroll
  for (int u = 0; u < kRowsPer; ++u) {
    if (i0 + u >= p.keep) break;
    const int64_t row = min(max(kept[i0 + u], 0), p.prefix_len - 1);
    const int64_t at = row * p.row + g * p.head + c;
    k[u] = __ldcs(p.k + at);
    v[u] = __ldcs(p.v + at);
  }
#pragma unroll
  for (int u = 0; u < kRowsPer; ++u) {
    if (i0 + u >= p.keep) break;
    const int64_t to = (i0 + u) * p.out_row + g * p.out_head + c;
    p.k_out[to] = k[u];
    p.v_out[to] = v[u];
  }
}

// A tensor [rows, heads, d] in bytes: runs of `run` bytes, r * row + g * head from its start.
constexpr int64_t kMostBytes = 1ll << 60;  // more than any tensor has
struct Strided {
  int64_t rows, heads, row, head, run;
  bool fits() const {  // (rows times a stride may pass 64 bits)
    return rows == 0 || static_cast<double>(rows - 1) * row + static_cast<double>(heads - 1) * head < kMostBytes;
  }
  int64_t bytes() const { return rows == 0 ? 0 : (rows - 1) * row + (heads - 1) * head + run; }  // first to last
};
bool meet(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return na > 0 && nb > 0 && x < y + nb && y < x + na;
}
int64_t floor_div(int64_t a, int64_t b) { return a / b - (a % b < 0); }  // b > 0

// Whether a byte range [lo, hi) from the start of `t` meets one of its runs.
bool meets_run(const Strided& t, int64_t lo, int64_t hi) {
  for (int64_t g = 0; g < t.heads; ++g) {
    // rows r with lo - run < r * row + g * head < hi
    const int64_t at = g * t.head;
    const int64_t first = floor_div(lo - t.run - at, t.row) + 1, last = floor_div(hi - 1 - at, t.row);
    if (std::max<int64_t>(first, 0) <= std::min(last, t.rows - 1)) return true;
  }
  return false;
}
// Whether a run of `t` meets another one, or, with `at` bytes to a second tensor of the same form, one of that.
bool runs_meet(const Strided& t, int64_t at) {
  for (int64_t g = 1 - t.heads; g < t.heads; ++g) {
    // row differences r with |at + r * row + g * head| < run
    const int64_t off = at + g * t.head;
    const int64_t first = std::max(floor_div(-t.run - off, t.row) + 1, 1 - t.rows);
    const int64_t last = std::min(floor_div(t.run - 1 - off, t.row), t.rows - 1);
    if (at == 0 && g == 0 && first == 0 && last == 0) continue;  // a run and itself
    if (first <= last) return true;
  }
  return false;
}

dard_status prepare(const dard_prefix_evict_args* a, EvictParams& p) {
  memset(&p, 0, sizeof(p));
  if (!a) return report(DARD_ERR_NULL, "args is NULL");
  if (a->dtype != DARD_BF16 && a->dtype != DARD_F32)
    return report(DARD_ERR_VALUE, "dtype %d is neither DARD_F32 nor DARD_BF16", a->dtype);
  if (a->hkv < 1 || a->hkv > 65535) return report(DARD_ERR_SHAPE, "hkv %d outside 1..65535", a->hkv);
  if (a->head_dim != 64 && a->head_dim != 128)
    return report(DARD_ERR_UNSUPPORTED, "head_dim %d (supported: 64, 128)", a->head_dim);
  if (a->prefix_len < 0 || a->prefix_len > DARD_PREFIX_MAX_LEN)
    return report(DARD_ERR_SHAPE, "prefix_len %d outside 0..%d", a->prefix_len, DARD_PREFIX_MAX_LEN);
  if (a->keep_first < 0 || a->keep_last < 0 || a->keep > a->prefix_len ||
      static_cast<long long>(a->keep_first) + a->keep_last > a->keep)
    return report(DARD_ERR_SHAPE, "need 0 <= keep_first + keep_last <= keep <= prefix_len, got %d + %d, %d, %d",
                  a->keep_first, a->keep_last, a->keep, a->prefix_len);
  p.hkv = a->hkv;
  p.prefix_len = a->prefix_len;
  p.keep = a->keep;
  p.first = a->keep_first;
  p.last = a->keep_last;
  if (a->keep == 0) return DARD_OK;
  const int esz = a->dtype == DARD_BF16 ? 2 : 4;
  if (!a->weights || !a->kept) return report(DARD_ERR_NULL, "weights or kept is NULL");
  if (a->weights_stride < a->prefix_len) return report(DARD_ERR_SHAPE, "weights_stride is below prefix_len");
  if (static_cast<double>(a->hkv - 1) * a->weights_stride * 4 >= kMostBytes)
    return report(DARD_ERR_SHAPE, "rows times weights_stride exceed 2^60 bytes");
  if (((reinterpret_cast<uintptr_t>(a->weights) | reinterpret_cast<uintptr_t>(a->kept) |
        reinterpret_cast<uintptr_t>(a->weights_out)) & 3u) != 0)
    return report(DARD_ERR_ALIGN, "weights, kept and weights_out must be 4-byte aligned");
  const bool move = a->prefix_k || a->prefix_v || a->k_out || a->v_out;
  Strided in{0, 0, 0, 0, 0}, out{0, 0, 0, 0, 0};
  if (move) {
    if (!a->prefix_k || !a->prefix_v || !a->k_out || !a->v_out)
      return report(DARD_ERR_NULL, "prefix_k, prefix_v, k_out and v_out come together");
    const int64_t most = 1ll << 36;
    if (a->prefix_row_stride < a->head_dim || a->prefix_head_stride < a->head_dim ||
        a->out_row_stride < a->head_dim || a->out_head_stride < a->head_dim ||
        a->prefix_row_stride > most || a->prefix_head_stride > most || a->out_row_stride > most ||
        a->out_head_stride > most)
      return report(DARD_ERR_SHAPE, "strides outside head_dim..2^36");
    if (((reinterpret_cast<uintptr_t>(a->prefix_k) | reinterpret_cast<uintptr_t>(a->prefix_v) |
          reinterpret_cast<uintptr_t>(a->k_out) | reinterpret_cast<uintptr_t>(a->v_out) |
          static_cast<uintptr_t>(a->prefix_row_stride * esz) |
          static_cast<uintptr_t>(a->prefix_head_stride * esz) |
          static_cast<uintptr_t>(a->out_row_stride * esz) |
          static_cast<uintptr_t>(a->out_head_stride * esz)) & 15u) != 0)
      return report(DARD_ERR_ALIGN, "keys, values and their strides must be multiples of 16 bytes");
    const int64_t run = static_cast<int64_t>(a->head_dim) * esz;
    in = {a->prefix_len, a->hkv, a->prefix_row_stride * esz, a->prefix_head_stride * esz, run};
    out = {a->keep, a->hkv, a->out_row_stride * esz, a->out_head_stride * esz, run};
    if (!in.fits() || !out.fits()) return report(DARD_ERR_SHAPE, "rows times strides exceed 2^60 bytes");
  }
  const size_t w_in = static_cast<size_t>((a->hkv - 1) * a->weights_stride + a->prefix_len) * 4;
  const size_t list = static_cast<size_t>(a->hkv) * a->keep * 4;
  const void* const ins[3] = {a->weights, a->prefix_k, a->prefix_v};
  const size_t in_bytes[3] = {w_in, static_cast<size_t>(in.bytes()), static_cast<size_t>(in.bytes())};
  const void* const outs[4] = {a->kept, a->weights_out, a->k_out, a->v_out};
  const size_t out_bytes[4] = {list, a->weights_out ? list : 0, static_cast<size_t>(out.bytes()),
                               static_cast<size_t>(out.bytes())};
  for (int i = 0; i < 3; ++i)
    for (int o = 0; o < 4; ++o)
      if (meet(ins[i], in_bytes[i], outs[o], out_bytes[o]))
        return report(DARD_ERR_VALUE, "an output overlaps an input");
  // outputs and one another: by extent first; k_out and v_out may lie row by row beside each other
  if (meet(a->kept, list, a->weights_out, out_bytes[1]))
    return report(DARD_ERR_VALUE, "kept overlaps weights_out");
  for (int i = 0; i < 2; ++i)
    for (int o = 2; o < 4; ++o) {
      const int64_t lo = reinterpret_cast<intptr_t>(outs[i]) - reinterpret_cast<intptr_t>(outs[o]);
      if (meet(outs[i], out_bytes[i], outs[o], out_bytes[o]) &&
          meets_run(out, lo, lo + static_cast<int64_t>(out_bytes[i])))
        return report(DARD_ERR_VALUE, "kept or weights_out overlaps k_out or v_out");
    }
  if (move) {
    if (out.row < (out.heads - 1) * out.head + out.run && out.head < (out.rows - 1) * out.row + out.run &&
        runs_meet(out, 0))
      return report(DARD_ERR_VALUE, "rows of k_out and v_out overlap: strides %lld and %lld",
                    static_cast<long long>(a->out_row_stride), static_cast<long long>(a->out_head_stride));
    const int64_t at = static_cast<int64_t>(reinterpret_cast<intptr_t>(a->v_out) - reinterpret_cast<intptr_t>(a->k_out));
    if (at == 0 || (meet(a->k_out, out.bytes(), a->v_out, out.bytes()) && runs_meet(out, at)))
      return report(DARD_ERR_VALUE, "k_out overlaps v_out");
  }
  p.w = a->weights;
  p.w_stride = a->weights_stride;
  p.kept = a->kept;
  p.w_out = a->weights_out;
  if (move) {
    const int per = 16 / esz;
    p.k = static_cast<const uint4*>(a->prefix_k);
    p.v = static_cast<const uint4*>(a->prefix_v);
    p.k_out = static_cast<uint4*>(a->k_out);
    p.v_out = static_cast<uint4*>(a->v_out);
    p.row = a->prefix_row_stride / per;
    p.head = a->prefix_head_stride / per;
    p.out_row = a->out_row_stride / per;
    p.out_head = a->out_head_stride / per;
    p.chunks = a->head_dim / per;
  }
  return DARD_OK;
}

}  // namespace
}  // namespace dard

extern "C" dard_status dard_prefix_evict(const dard_prefix_evict_args* args, void* stream_ptr) {
  using namespace dard;
  report(DARD_OK, "%s", "");
  EvictParams p;
  const dard_status st = prepare(args, p);
  if (st != DARD_OK) return st;
  if (p.keep == 0) return DARD_OK;
  if (std::getenv("DARD_TEST_FAIL_LAUNCH") != nullptr)
    return report(DARD_ERR_CUDA, "prefix eviction launch failed: %s (DARD_TEST_FAIL_LAUNCH)",
                  cudaGetErrorString(cudaErrorLaunchFailure));
  const cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
  // CTAs of a head: one up to 8192 keys, as the cluster's barriers cost 3.5 us (8 heads of 4099 keys: 9.7 us
  // with one CTA, 13.3 with two), then one per 4096 (8 heads of 16384: 19.9 us with two, 17.6 with four)
  int ctas = 1;
  while (ctas < kMaxCluster && p.prefix_len > std::max(8192, 4096 * ctas) && 2ll * ctas * p.hkv <= sm_count())
    ctas *= 2;
  const AttnLaunch S(static_cast<unsigned>(p.hkv) * ctas, kSelThreads, 0, stream, ctas, false);
  cudaError_t e = cudaLaunchKernelEx(&S.cfg, evict_select, p, ctas);
  if (e == cudaSuccess && p.k) {
    const long long threads = (static_cast<long long>(p.keep) + kRowsPer - 1) / kRowsPer * p.hkv * p.chunks;
    const long long blocks = (threads + kCopyThreads - 1) / kCopyThreads;
    if (blocks > 0x7fffffffll) return report(DARD_ERR_SHAPE, "too many rows to move");
    const AttnLaunch C(static_cast<unsigned>(blocks), kCopyThreads, 0, stream, 1, true);
    e = cudaLaunchKernelEx(&C.cfg, evict_copy, p);
  }
  if (e != cudaSuccess)
    return report(DARD_ERR_CUDA, "prefix eviction launch failed: %s", cudaGetErrorString(e));
  return DARD_OK;
}
