// dard_prefix.cuh - pieces shared by the kernels of decoding behind a shared prefix: the launch
// parameters, the packing of query rows and heads into one run of queries, and the mask of a row
// over its own sequence (Sec. 3.2 of arXiv 2608.26574) from the block's data in global memory.
//
// Packed queries. The query rows of all sequences, in order, are numbered t = 0 .. T - 1; with G
// query heads to a key/value head, query m = t G + h stands for row t and head g G + h of the
// key/value head g. Tiles of consecutive m fill up whatever the sequences' lengths are. A tile's
// keys are the prefix, then the rows of the sequences that it touches, which lie back to back;
// a row's visibility bits leave only its own sequence's keys of those.
#pragma once
#include "dard_attn_common.cuh"

namespace dard {

constexpr int kTileTable = 1024;
static_assert(DARD_MAX_SEQS <= 256, "sequences fit in a byte");

struct PrefixParams {
  AttnParams a;               // the own rows (a.q, a.k, a.v, a.o and the sequences)
  const void* pk;
  const void* pv;
  int64_t row_stride, head_stride;  // of pk and pv, elements
  float* lse;                 // or null
  float* part;                // the parts of a split launch: see part_slot()
  int32_t prefix_len;
  int32_t group;              // query heads of a key/value head
  int32_t queries;            // packed queries of a key/value head
  int32_t tiles;              // query tiles of a key/value head
  int32_t nsplit;             // CTAs that share a tile's keys
  int32_t q_before[DARD_MAX_SEQS + 1];  // query rows of the sequences before each
  uint8_t tile_seq[kTileTable][2];      // first and last sequence of a query tile, if all fit in
};

// Parts of a split launch: one slot per (tile, part), rows x (D + 5) floats: the unnormalised
// output rows, then per row the reference maximum (times scale log2 e; -inf: no key), the sum of
// the weights, (8 bytes; the tile's last part counts) the output row, -1 for none, and the sum of
// the weights as the output has them (bf16: rounded; fp32: not used).
__host__ __device__ inline size_t part_slot_floats(int rows, int d) {
  return static_cast<size_t>(rows) * (d + 5);
}

struct JoinParams {
  const float* part;
  void* o;
  float* lse;
  int64_t rows;               // packed queries of all key/value heads
  int64_t out_rows;           // rows times heads of o
  int32_t queries, tiles, nsplit, tile_rows;
};

// The fp32 kernels on CUDA cores, with kF32FewRows or 128 packed queries per CTA.
constexpr int kF32FewRows = 8;
cudaError_t launch_prefix_f32(const PrefixParams& p, int rows, cudaStream_t stream);

namespace {

// One lane of a converged warp.
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r != 0;
}
// Whether a phase has completed, without waiting: its answer takes some 120 cycles, which a wait at
// the same place would too; asked ahead of the work before that place, it costs nothing.
__device__ __forceinline__ bool mbar_test(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(smem_u32(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}
// Bounded wait of a whole warp.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, long long limit) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, limit));
}
__device__ __forceinline__ void tma_load_3d(void* dst, const void* desc, uint64_t* bar, int32_t c0,
                                            int32_t c1, int32_t c2) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(desc)), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2)
      : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr),
               "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
// 32 or 16 columns of this warp's lanes.
__device__ __forceinline__ void tmem_load(uint32_t addr, uint32_t (&r)[32]) { tmem_ld32(addr, r); }
__device__ __forceinline__ void tmem_load(uint32_t addr, uint32_t (&r)[16]) { tmem_ld16(addr, r); }
__device__ __forceinline__ void tmem_store(uint32_t addr, const uint32_t (&r)[32]) { tmem_st32(addr, r); }
__device__ __forceinline__ void tmem_store(uint32_t addr, const uint32_t (&r)[16]) { tmem_st16(addr, r); }
__device__ __forceinline__ void tmem_store(uint32_t addr, const uint32_t (&r)[8]) { tmem_st8(addr, r); }

// Tensor map of bf16 elements [n2, n1, d], strides in elements, boxes of 64 x box1 x box2 with the
// 128-byte swizzle; elements outside read as zeros.
inline bool make_map3(CUtensorMap* m, const void* ptr, int d, long long n1, long long n2, int64_t stride1,
                      int64_t stride2, int box1, int box2) {
  auto fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(d), static_cast<cuuint64_t>(n1),
                              static_cast<cuuint64_t>(n2)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(stride1) * 2, static_cast<cuuint64_t>(stride2) * 2};
  const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(box1), static_cast<cuuint32_t>(box2)};
  const cuuint32_t estr[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(ptr), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Sequence of query row t, one of [lo, hi) (the last that starts at t or before: sequences without
// queries are passed over).
__device__ __forceinline__ int seq_of_query(const PrefixParams& p, int t, int lo, int hi) {
  while (hi - lo > 1) {  // q_before[lo] <= t < q_before[hi]
    const int mid = (lo + hi) >> 1;
    if (p.q_before[mid] <= t) lo = mid; else hi = mid;
  }
  return lo;
}
__device__ __forceinline__ int seq_of_query(const PrefixParams& p, int t) {
  return seq_of_query(p, t, 0, p.a.num_seqs);
}

// A tile's sequences [s0, s1] and its keys behind the prefix: rows [key0, key_end) of k and v. The
// same for every thread of a CTA, in a form that the compiler sees to be (results of ballots or
// selects would make the loop bounds that depend on it a thread's own: 5 % of a long call); from the
// launch's table where the tiles fit in (a search waits some 200 cycles for each of its reads).
__device__ __forceinline__ void own_range(const PrefixParams& p, int tile, int rows, int& s0, int& s1,
                                          int& key0, int& key_end) {
  if (p.tiles <= kTileTable) {
    s0 = p.tile_seq[tile][0];
    s1 = p.tile_seq[tile][1];
  } else {
    s0 = seq_of_query(p, tile * rows / p.group);
    s1 = seq_of_query(p, (min((tile + 1) * rows, p.queries) - 1) / p.group);
  }
  key0 = p.a.seq[s0].row_base;
  key_end = p.a.seq[s1].row_base + p.a.seq[s1].n_orig + p.a.seq[s1].slen;
}

// The masks of the rows of one warp over their sequences' blocks, read from global memory: what
// publish_block_info(), row_info() and row_masks() derive for a CTA whose rows are all of one
// sequence. Lane by lane: `seq` (-1: no row) and the sequence-relative row r; store = 0 for a
// shadow row whose shadow_src is invalid. Called by whole warps. The lanes fetch a sequence's block
// together, 32 positions each time; ballots make bit words of it, and the warp's scratch lets every
// lane read any position's confidence and any shadow row's position.
struct BlockScratch {
  float4 cf[DARD_MAX_BLOCK / 4];
  int4 pos[DARD_MAX_BLOCK / 4];  // block positions of the shadow rows (-1: none)
};
__device__ __forceinline__ RowMasks warp_query_masks(const AttnParams& p, BlockScratch& scratch, int seq,
                                                     int r, bool report, int& store) {
  constexpr uint32_t kAll = 0xffffffffu;
  const int lane = threadIdx.x & 31;
  float* cf = reinterpret_cast<float*>(scratch.cf);
  int* pos = reinterpret_cast<int*>(scratch.pos);
  RowMasks out{{0, 0}, {0, 0}};
  store = seq >= 0;
  uint32_t todo = __ballot_sync(kAll, seq >= 0);
  while (todo) {
    const int s = __shfl_sync(kAll, seq, __ffs(todo) - 1);
    const bool mine = seq == s;
    todo &= ~__ballot_sync(kAll, mine);
    const SeqDesc& sd = p.seq[s];
    const int blen = sd.blen, slen = sd.slen;
    if (blen == 0) continue;  // no block, no shadow rows: nothing is hidden
    // bit words over block positions (m, c: states; hs: a shadow copy exists) and over shadow rows
    // (valid: the position's lowest shadow row)
    uint32_t m[4] = {0, 0, 0, 0}, c[4] = {0, 0, 0, 0}, hs[4] = {0, 0, 0, 0}, valid[4] = {0, 0, 0, 0};
    int rows = 0, positions = 0;
    bool bad_state = false, identity = true;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (32 * i >= blen) break;
      const int j = 32 * i + lane;
      const int st = j < blen ? __ldg(p.state + sd.blk_off + j) : kStateU;
      const float x = j < blen ? __ldg(p.prev_conf + sd.blk_off + j) : 0.f;
      int at = j < slen ? __ldg(p.shadow_src + sd.sh_off + j) - sd.b0 : -1;
      if (at >= blen) at = -1;
      cf[j] = x;
      pos[j] = at;
      m[i] = __ballot_sync(kAll, st == kStateM || st > 2);
      c[i] = __ballot_sync(kAll, st == kStateC);
      valid[i] = __ballot_sync(kAll, at >= 0);
      bad_state |= st > 2;
      identity &= j >= slen || at == j;
      rows += __popc(valid[i]);
#pragma unroll
      for (int w = 0; w < 4; ++w)
        if (32 * w < blen) hs[w] |= __reduce_or_sync(kAll, at >= 0 && at >> 5 == w ? 1u << (at & 31) : 0u);
    }
#pragma unroll
    for (int w = 0; w < 4; ++w) positions += __popc(hs[w]);
    __syncwarp();
    if (positions != rows) {  // a repeated position: its lowest row alone is valid
      uint32_t seen[4] = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        for (int l = 0; l < 32 && 32 * i + l < slen; ++l) {
          const int x = pos[32 * i + l];
          if (x < 0) continue;
          bool again = false;
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const uint32_t bit = x >> 5 == w ? 1u << (x & 31) : 0u;
            again |= (seen[w] & bit) != 0;
            seen[w] |= bit;
          }
          if (again) valid[i] &= ~(1u << l);
        }
      }
    }
    identity = __all_sync(kAll, identity);
    if (report && p.status) {
      const uint32_t flags = (__any_sync(kAll, bad_state) ? DARD_STATUS_BAD_STATE : 0u) |
                             (positions != slen ? DARD_STATUS_BAD_SHADOW : 0u);
      if (lane == 0 && flags) atomicOr(p.status, flags);
    }
    if (mine) {  // this lane's row
      RowInfo q{0, kStateU, 0.f, -1, 1};
      const int kq = r - sd.n_orig, j = r - sd.b0;  // its shadow index, its block position
      if (kq >= 0) {
        const uint32_t word = kq < 64 ? (kq < 32 ? valid[0] : valid[1]) : (kq < 96 ? valid[2] : valid[3]);
        q.qs = q.store = word >> (kq & 31) & 1u;
        if (q.qs) q.i = pos[kq];
      } else if (j >= 0 && j < blen) {
        q.i = j;
      } else {
        q.si = j < 0 ? kStateU : kStateM;  // decoded context / still masked
      }
      if (q.i >= 0) {
        const int w = q.i >> 5;
        const uint32_t mw = w < 2 ? (w == 0 ? m[0] : m[1]) : (w == 2 ? m[2] : m[3]);
        const uint32_t cw = w < 2 ? (w == 0 ? c[0] : c[1]) : (w == 2 ? c[2] : c[3]);
        q.si = mw >> (q.i & 31) & 1u ? kStateM : cw >> (q.i & 31) & 1u ? kStateC : kStateU;
        q.ci = cf[q.i];
      }
      // positions taken from their shadow copy, as in row_masks()
      uint32_t ts[4], see[4] = {0, 0, 0, 0};
      const bool all_mc = q.si == kStateU || (q.si == kStateM && q.qs);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        ts[i] = all_mc ? m[i] | c[i] : 0u;
        if (q.si == kStateC && 32 * i < blen) {
          uint32_t lower = 0;  // C keys with !(c_i <= c_j) (Eq. 3)
#pragma unroll
          for (int l = 0; l < 8; ++l) {
            const float4 x = scratch.cf[8 * i + l];
            lower |= (static_cast<uint32_t>(!(q.ci <= x.x)) | static_cast<uint32_t>(!(q.ci <= x.y)) << 1 |
                      static_cast<uint32_t>(!(q.ci <= x.z)) << 2 | static_cast<uint32_t>(!(q.ci <= x.w)) << 3)
                     << (4 * l);
          }
          ts[i] = m[i] | (c[i] & lower);
        }
        if (q.qs && q.i >> 5 == i) ts[i] |= 1u << (q.i & 31);  // a shadow query takes its own copy
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (identity) {
          see[i] = ts[i];
        } else {
          for (int l = 0; l < 32 && 32 * i + l < slen; ++l) {
            const int x = pos[32 * i + l];
            const uint32_t word = x < 64 ? (x < 32 ? ts[0] : ts[1]) : (x < 96 ? ts[2] : ts[3]);
            see[i] |= (word >> (x & 31) & 1u) << l;
          }
        }
        see[i] &= valid[i];
      }
      store = q.store;
      const uint32_t hide[4] = {ts[0] & hs[0], ts[1] & hs[1], ts[2] & hs[2], ts[3] & hs[3]};
      out.hide_x = words128(hide);
      out.see_s = words128(see);
    }
    __syncwarp();
  }
  return out;
}

// Visibility of the 64 keys from sequence-relative row kt0 on (bit t = key kt0 + t); kt0 may lie
// before the sequence or behind it: keys outside it are hidden.
__device__ __forceinline__ uint64_t own_vis64(const SeqDesc& sd, int kt0, const RowMasks& m) {
  if (kt0 <= -64 || kt0 >= sd.n_orig + sd.slen) return 0;
  uint64_t vis = vis64(sd, kt0, m);
  if (kt0 < 0) vis &= ~0ull << -kt0;
  return vis;
}

// The first n of 64 keys.
__device__ __forceinline__ uint64_t first64(int n) {
  return n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1;
}

}  // namespace
}  // namespace dard
