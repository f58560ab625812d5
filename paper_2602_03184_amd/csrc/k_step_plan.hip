// Tables of a step with several new tokens per sequence: packed starts, slot map, positions and ancestor masks from the
// sequences' lengths.  A few bytes a token and no arithmetic to speak of: latency for a decoding step, writes for prompts.
// One launch: every workgroup scans the B counts for itself (they are a cache line or two) instead of waiting for one that
// has, and then looks its own tokens up.  Ancestors are found by doubling: a node takes over what its parent has and then its
// parent's parent, so the rounds go with the logarithm of the depth (a walk from node to node, an LDS read each, took 5.8 us
// for eight trees of 64 nodes some 20 deep; this takes 5.3, most of it launch and the latency of three reads).
#include "dsk_common.hpp"
#include "dsk_internal.hpp"

namespace dsk {

constexpr int kPlanThreads = 256;
constexpr int kPlanWaves = kPlanThreads / DSK_WAVE;
constexpr int kPlanPerThread = 4;              // tokens of a thread where there is no tree

// a + b of 0..cap, at most cap: associative, so any order of a scan gives the same; a sum of two may pass 32 bits
__device__ __forceinline__ uint32_t add_sat(uint32_t a, uint32_t b, uint32_t cap) { return b < cap - a ? a + b : cap; }

// WORDS: mask words kept in registers (0: no masks), >= mask_words
template <int WORDS>
__global__ __launch_bounds__(kPlanThreads) void step_plan_kernel(dsk_step_plan_args a, int per_thread) {
  __shared__ uint32_t sm_base[kPlanThreads + 1];
  __shared__ uint32_t sm_wave[kPlanWaves];
  __shared__ int32_t sm_len[kPlanThreads], sm_row0[kPlanThreads];
  // The tile's nodes, and those of a sequence that begins before it.
  constexpr int kNodes = DSK_TREE_MAX_NODES + kPlanThreads, kPer = 2;
  static_assert(kNodes == kPer * kPlanThreads, "two nodes a thread");
  __shared__ int32_t sm_up[kNodes];                            // an ancestor that is not taken over yet, -1: none
  __shared__ int32_t sm_depth[kNodes];
  __shared__ uint32_t sm_bits[WORDS > 0 ? WORDS : 1][kNodes];
  const int tid = threadIdx.x, lane = tid & (DSK_WAVE - 1), wave = tid / DSK_WAVE;
  const bool tree = a.parent != nullptr, limited = tree || WORDS > 0;
  const uint32_t cap = (uint32_t)a.max_tokens + 1u;            // one more than fit: an overflow stays visible
  const int per = (a.B + kPlanThreads - 1) / kPlanThreads;     // sequences of a thread, in order
  const bool first_wg = blockIdx.x == 0;
  int32_t bad = 0;
  auto count_of = [&](int s) -> uint32_t {
    int n = a.n_new[s];
    if (n < 0) { n = 0; bad = DSK_ERR_SHAPE; }
    if (limited && n > a.max_nodes) { n = a.max_nodes; bad = DSK_ERR_SHAPE; }
    return (uint32_t)n < cap ? (uint32_t)n : cap;
  };
  const int64_t tile0 = (int64_t)blockIdx.x * per_thread * kPlanThreads;
  int parent[kPer];
  if (tree) {
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int64_t t = tile0 - DSK_TREE_MAX_NODES + k * kPlanThreads + tid;
      parent[k] = t >= 0 && t < a.max_tokens ? a.parent[t] : -1;
    }
  }
  uint32_t mine = 0, own = 0;
  if (per == 1) {                                              // a sequence a thread: all that it has is on its way at once
    if (tid < a.B) {
      sm_len[tid] = a.seq_len[tid];
      sm_row0[tid] = a.seq_row0[tid];
      mine = own = count_of(tid);
    }
  } else {
    for (int i = 0; i < per; ++i) {
      const int s = tid * per + i;
      if (s < a.B) mine = add_sat(mine, count_of(s), cap);
    }
  }
  // inclusive scan over the wavefront, as wave_incl_scan_i
  uint32_t incl = mine;
  incl = add_sat(incl, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)incl, kDppRowShr + 1, 0xF, 0xF, false), cap);
  incl = add_sat(incl, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)incl, kDppRowShr + 2, 0xF, 0xF, false), cap);
  incl = add_sat(incl, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)incl, kDppRowShr + 4, 0xF, 0xF, false), cap);
  incl = add_sat(incl, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)incl, kDppRowShr + 8, 0xF, 0xF, false), cap);
  incl = add_sat(incl, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)incl, kDppBcast15, 0xA, 0xF, false), cap);
  incl = add_sat(incl, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)incl, kDppBcast31, 0xC, 0xF, false), cap);
  if (lane == DSK_WAVE - 1) sm_wave[wave] = incl;
  uint32_t before = (uint32_t)__shfl_up((int)incl, 1, DSK_WAVE);
  if (lane == 0) before = 0;
  __syncthreads();
  uint32_t waves_before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) {
    if (w < wave) waves_before = add_sat(waves_before, sm_wave[w], cap);
    total = add_sat(total, sm_wave[w], cap);
  }
  before = add_sat(before, waves_before, cap);
  sm_base[tid] = before;
  if (tid == 0) sm_base[kPlanThreads] = total;
  const uint32_t fit = (uint32_t)a.max_tokens;
  if (first_wg) {
    uint32_t c = before;
    for (int i = 0; i < per; ++i) {
      const int s = tid * per + i;
      if (s < a.B) {
        a.cu_new[s] = (int32_t)(c < fit ? c : fit);
        c = add_sat(c, per == 1 ? own : count_of(s), cap);
        if (s == a.B - 1) a.cu_new[a.B] = (int32_t)(c < fit ? c : fit);
      }
    }
    if (bad) set_status(a.dev_status, bad);
    if (tid == 0 && total > fit) set_status(a.dev_status, DSK_ERR_CAPACITY);
  }
  __syncthreads();
  const uint32_t used = total < fit ? total : fit;
  // (threads without a sequence: sm_base is the total, above every t)
  int top = 1;                                                 // of the search: the largest power of two below the threads in use
  while (2 * top * per < a.B) top *= 2;
  // the sequence of a token below `used` and its first token
  auto find = [&](uint32_t t, int& s, uint32_t& base) {
    int lo = 0;                                                // the last thread whose sequences begin at or before t
    for (int step = top; step > 0; step /= 2)
      if (sm_base[lo + step] <= t) lo += step;
    s = lo * per;
    base = sm_base[lo];
    if (per > 1)
      for (uint32_t n; t >= base + (n = count_of(s)); ++s) base += n;
  };
  int seq = 0;
  uint32_t first = 0;                                          // of this thread's token
  if (tree) {
    const int64_t own_t = tile0 + tid;
    const bool real = own_t < used;
    if (real) find((uint32_t)own_t, seq, first);
    // the place in LDS of the first node of the sequence that the tile begins in; the same for every thread
    int s0 = 0;
    uint32_t first0 = 0;
    if (tile0 < used) find((uint32_t)tile0, s0, first0);
    const int start0 = (int)((int64_t)first0 - tile0) + DSK_TREE_MAX_NODES;
    int up[kPer], depth[kPer];
    uint32_t bits[kPer][WORDS > 0 ? WORDS : 1];
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int at = k * kPlanThreads + tid;
      const bool mine = k == kPer - 1;                         // of the tile; the others belong to its first sequence, or to none
      const int start = mine ? (int)((int64_t)first - tile0) + DSK_TREE_MAX_NODES : start0;
      const bool there = mine ? real : tile0 < used && at >= start0;
      const int node = there ? at - start : 0;
      bool ok = there && parent[k] >= -1 && parent[k] < node;
      if (there && !ok && mine) set_status(a.dev_status, DSK_ERR_ORDER);
      up[k] = ok && parent[k] >= 0 ? start + parent[k] : -1;
      depth[k] = up[k] >= 0 ? 1 : 0;                           // ancestors taken over, and the next one
#pragma unroll
      for (int w = 0; w < WORDS; ++w) bits[k][w] = there && (node >> 5) == w ? 1u << (node & 31) : 0u;
      sm_up[at] = up[k];
      sm_depth[at] = depth[k];
#pragma unroll
      for (int w = 0; w < WORDS; ++w) sm_bits[w][at] = bits[k][w];
    }
    // ends: a node's ancestors are below it, and a round leaves half of them at most
    while (__syncthreads_or(up[0] >= 0 || up[kPer - 1] >= 0)) {
#pragma unroll
      for (int k = 0; k < kPer; ++k) {
        if (up[k] < 0) continue;
        depth[k] += sm_depth[up[k]];
#pragma unroll
        for (int w = 0; w < WORDS; ++w) bits[k][w] |= sm_bits[w][up[k]];
        up[k] = sm_up[up[k]];
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < kPer; ++k) {
        const int at = k * kPlanThreads + tid;
        sm_up[at] = up[k];
        sm_depth[at] = depth[k];
#pragma unroll
        for (int w = 0; w < WORDS; ++w) sm_bits[w][at] = bits[k][w];
      }
    }
  }

  for (int k = 0; k < per_thread; ++k) {
    const int64_t t64 = tile0 + (int64_t)tid * per_thread + k;  // neighbours: the search is made once
    if (t64 >= a.max_tokens) break;
    const uint32_t t = (uint32_t)t64;
    uint32_t bits[WORDS > 0 ? WORDS : 1];
#pragma unroll
    for (int w = 0; w < WORDS; ++w) bits[w] = 0;
    if (t >= used) {
      a.tok_seq[t] = -1;
      a.tok_pos[t] = 0;
      a.tok_row[t] = -1;
    } else {
      if (!tree) {
        if (k == 0 || per > 1) {
          find(t, seq, first);
        } else {
          while (t >= sm_base[seq + 1]) first = sm_base[++seq];
        }
      }
      const int s = seq;
      const uint32_t base = first;
      int depth;
      const int i = (int)(t - base);
      if (tree) {
        const int at = DSK_TREE_MAX_NODES + tid;
        depth = sm_depth[at];
#pragma unroll
        for (int w = 0; w < WORDS; ++w) bits[w] = sm_bits[w][at];
      } else {
        depth = i;
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
          const int n = i + 1 - 32 * w;                        // nodes 0..i
          bits[w] = n >= 32 ? 0xFFFFFFFFu : (n > 0 ? (1u << n) - 1u : 0u);
        }
      }
      const int64_t len = per == 1 ? sm_len[s] : a.seq_len[s], row0 = per == 1 ? sm_row0[s] : a.seq_row0[s];
      const int64_t row = row0 + len + i, pos = len + depth;
      const bool ok = row0 >= 0 && len >= 0 && row < a.total_rows;
      if (!ok) set_status(a.dev_status, DSK_ERR_CAPACITY);
      a.tok_seq[t] = s;
      a.tok_pos[t] = (int32_t)(pos < 0x7FFFFFFF ? pos : 0x7FFFFFFF);
      a.tok_row[t] = ok ? (int32_t)row : -1;
    }
#pragma unroll
    for (int w = 0; w < WORDS; ++w)
      if (w < a.mask_words) a.mask[t64 * a.mask_words + w] = bits[w];
  }
}

hipError_t launch_step_plan(const dsk_step_plan_args& a, hipStream_t st) {
  // a tile of a tree is a node a thread, as its LDS; without a tree a thread makes one search for several tokens
  const int per_thread = a.parent != nullptr ? 1 : kPlanPerThread;
  const int tile = per_thread * kPlanThreads;
  const dim3 grid((unsigned)(((int64_t)a.max_tokens + tile - 1) / tile)), block(kPlanThreads);
  const int words = a.mask != nullptr ? a.mask_words : 0;
  if (words == 0) step_plan_kernel<0><<<grid, block, 0, st>>>(a, per_thread);
  else if (words <= 2) step_plan_kernel<2><<<grid, block, 0, st>>>(a, per_thread);
  else step_plan_kernel<DSK_TREE_MAX_NODES / 32><<<grid, block, 0, st>>>(a, per_thread);
  return hipGetLastError();
}

}  // namespace dsk
