// Tables of a step with several new tokens per sequence: packed starts, slot map, positions and ancestor masks from the
// sequences' lengths.  A few bytes a token and no arithmetic to speak of: latency for a decoding step, writes for prompts.
// One launch: every workgroup scans the B counts for itself (they are a cache line or two) instead of waiting for one that
// has, and then looks its own tokens up.
#include "dsk_common.hpp"
#include "dsk_internal.hpp"

namespace dsk {

constexpr int kPlanThreads = 256;
constexpr int kPlanWaves = kPlanThreads / DSK_WAVE;
constexpr int kPlanPerThread = 4;              // tokens of a thread where there is no tree to walk

// a + b, at most cap: associative on 0..cap, so any order of a scan gives the same, and it fits 32 bits
__device__ __forceinline__ uint32_t add_sat(uint32_t a, uint32_t b, uint32_t cap) { return a + b < cap ? a + b : cap; }

// WORDS: mask words kept in registers (0: no masks), >= mask_words
template <int WORDS>
__global__ __launch_bounds__(kPlanThreads) void step_plan_kernel(dsk_step_plan_args a, int per_thread) {
  __shared__ uint32_t sm_base[kPlanThreads + 1];
  __shared__ uint32_t sm_wave[kPlanWaves];
  __shared__ int32_t sm_len[kPlanThreads], sm_row0[kPlanThreads];
  __shared__ int32_t sm_parent[DSK_TREE_MAX_NODES + kPlanThreads];
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
  if (tree) {                                                  // the tile's parents, and those of a sequence that begins before it
    for (int i = tid; i < DSK_TREE_MAX_NODES + kPlanThreads; i += kPlanThreads) {
      const int64_t t = tile0 - DSK_TREE_MAX_NODES + i;
      sm_parent[i] = t >= 0 && t < a.max_tokens ? a.parent[t] : -1;
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

  for (int k = 0; k < per_thread; ++k) {
    const int64_t t64 = tile0 + (int64_t)k * kPlanThreads + tid;
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
      int lo = 0;                                              // the last thread whose sequences begin at or before t
#pragma unroll
      for (int step = kPlanThreads / 2; step > 0; step /= 2)
        if (sm_base[lo + step] <= t) lo += step;
      int s = lo * per;
      uint32_t base = sm_base[lo];
      if (per > 1)
        for (uint32_t n; t >= base + (n = count_of(s)); ++s) base += n;
      const int i = (int)(t - base);
      int depth = i;
      if (tree) {
        const int32_t* par = sm_parent + (int)(t64 - tile0) + DSK_TREE_MAX_NODES - i;   // the sequence's first node
        depth = 0;
        int node = i;
#pragma unroll
        for (int w = 0; w < WORDS; ++w) bits[w] |= (node >> 5) == w ? 1u << (node & 31) : 0u;
        for (;;) {                                             // ends: every parent taken is below its node
          const int up = par[node];
          if (up < -1 || up >= node) {
            set_status(a.dev_status, DSK_ERR_ORDER);
            break;
          }
          if (up < 0) break;
          node = up;
          ++depth;
#pragma unroll
          for (int w = 0; w < WORDS; ++w) bits[w] |= (node >> 5) == w ? 1u << (node & 31) : 0u;
        }
      } else {
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
  // walks take as long as a tree is deep, so a thread takes one node; without a tree it takes several tokens
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
