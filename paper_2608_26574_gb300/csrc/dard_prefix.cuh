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
};

// Parts of a split launch: one slot per (tile, part), rows x (D + 3) floats: the unnormalised
// output rows, then per row the reference maximum (times scale log2 e; -inf: no key), the sum of
// the weights as the product uses them, and their sum unrounded (-1: a row that is not stored).
__host__ __device__ inline size_t part_slot_floats(int rows, int d) {
  return static_cast<size_t>(rows) * (d + 3);
}

// The fp32 kernel on CUDA cores.
int prefix_f32_rows(const PrefixParams& p, int sms);  // packed queries per CTA
cudaError_t launch_prefix_f32(const PrefixParams& p, int rows, cudaStream_t stream);

namespace {

// Sequence of query row t.
__device__ __forceinline__ int seq_of_query(const PrefixParams& p, int t) {
  int lo = 0, hi = p.a.num_seqs;  // q_before[lo] <= t < q_before[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (p.q_before[mid] <= t) lo = mid; else hi = mid;
  }
  return lo;
}

// A tile's keys behind the prefix: rows [key0, key_end) of k and v.
__device__ __forceinline__ void own_range(const PrefixParams& p, int m0, int rows, int& key0,
                                          int& key_end) {
  const int last = min(m0 + rows, p.queries) - 1;
  key0 = p.a.seq[seq_of_query(p, m0 / p.group)].row_base;
  const SeqDesc& s = p.a.seq[seq_of_query(p, last / p.group)];
  key_end = s.row_base + s.n_orig + s.slen;
}

// The masks of sequence-relative row r over its sequence's block, read from global memory by one
// thread: what publish_block_info(), row_info() and row_masks() derive for a CTA whose rows are
// all of one sequence. store = 0 for a shadow row whose shadow_src is invalid.
__device__ RowMasks query_masks(const AttnParams& p, const SeqDesc& sd, int r, bool report,
                                int& store) {
  Bits128 mb{0, 0}, cb{0, 0}, hs{0, 0}, valid{0, 0};
  uint32_t flags = 0;
  const uint8_t* st = p.state + sd.blk_off;
  for (int j0 = 0; j0 < sd.blen; j0 += 8) {
    int s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = j0 + e < sd.blen ? __ldg(st + j0 + e) : kStateU;
    uint64_t m8 = 0, c8 = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (s[e] > 2) flags |= DARD_STATUS_BAD_STATE;
      m8 |= static_cast<uint64_t>(s[e] == kStateM || s[e] > 2) << e;
      c8 |= static_cast<uint64_t>(s[e] == kStateC) << e;
    }
    if (j0 < 64) { mb.lo |= m8 << j0; cb.lo |= c8 << j0; }
    else { mb.hi |= m8 << (j0 - 64); cb.hi |= c8 << (j0 - 64); }
  }
  // shadow rows: a repeated position keeps its lowest row
  RowInfo q{0, kStateU, 0.f, -1, 1};
  const int32_t* src = p.shadow_src + sd.sh_off;
  const int kq = r - sd.n_orig;  // the row's shadow index, if it is one
  if (kq >= 0) q.store = 0;
  for (int k0 = 0; k0 < sd.slen; k0 += 8) {
    int pos[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) pos[e] = k0 + e < sd.slen ? __ldg(src + k0 + e) - sd.b0 : INT_MIN;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (k0 + e >= sd.slen) break;
      const bool ok = pos[e] >= 0 && pos[e] < sd.blen && !get_bit(hs, pos[e]);
      if (!ok) { flags |= DARD_STATUS_BAD_SHADOW; continue; }
      set_bit(hs, pos[e]);
      set_bit(valid, k0 + e);
      if (k0 + e == kq) { q.qs = 1; q.i = pos[e]; q.store = 1; }
    }
  }
  if (report && flags && p.status) atomicOr(p.status, flags);
  if (kq < 0) {
    const int j = r - sd.b0;
    if (j >= 0 && j < sd.blen) q.i = j;
    else q.si = j < 0 ? kStateU : kStateM;  // decoded context / still masked
  }
  if (q.i >= 0) {
    q.si = get_bit(mb, q.i) ? kStateM : get_bit(cb, q.i) ? kStateC : kStateU;
    q.ci = __ldg(p.prev_conf + sd.blk_off + q.i);
  }
  store = q.store;
  // positions taken from their shadow copy, as in row_masks()
  Bits128 ts{0, 0};
  if (q.si == kStateU || (q.si == kStateM && q.qs)) {
    ts = {mb.lo | cb.lo, mb.hi | cb.hi};
  } else if (q.si == kStateC) {
    Bits128 lower{0, 0};
    const float* cf = p.prev_conf + sd.blk_off;
    for (int j0 = 0; j0 < sd.blen; j0 += 8) {
      uint64_t l8 = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        l8 |= static_cast<uint64_t>(j0 + e < sd.blen && !(q.ci <= __ldg(cf + j0 + e))) << e;
      if (j0 < 64) lower.lo |= l8 << j0; else lower.hi |= l8 << (j0 - 64);
    }
    ts = {mb.lo | (cb.lo & lower.lo), mb.hi | (cb.hi & lower.hi)};
  }
  if (q.qs && q.i >= 0) set_bit(ts, q.i);
  RowMasks m;
  m.hide_x = {ts.lo & hs.lo, ts.hi & hs.hi};
  m.see_s = {0, 0};
  for (int k = 0; k < sd.slen; ++k)
    if (get_bit(valid, k) && get_bit(ts, __ldg(src + k) - sd.b0)) set_bit(m.see_s, k);
  return m;
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
