// The accepted path of every drafted tree and its K/V rows: a walk of a few steps and a copy of a few rows per layer and
// head, so latency bounds it.  Every wavefront makes the walk for itself (a sequence's nodes fit four registers), which
// spares a second launch and any wait between workgroups.  Eight trees of up to 64 nodes, 32 layers of 8 heads (6 MB) 5.9 us, of
// which some 2 are the launch's own; one tree of 8 nodes and two layers 3.3.  Calls of six accepted nodes a tree 6.0 us, in place 5.9;
// of 16 (two batches of rows, 34 MB) 12.4, in place 10.5.
#include "dsk_common.hpp"
#include "dsk_internal.hpp"

namespace dsk {

constexpr int kAcceptThreads = 256;
constexpr int kAcceptGroups = kAcceptThreads / 16;             // one head of K or V of one layer each
constexpr int kAcceptRegs = DSK_TREE_MAX_NODES / DSK_WAVE;
constexpr int kAcceptBatch = 8;                                // rows of a head on their way at once

__global__ __launch_bounds__(kAcceptThreads) void accept_kernel(dsk_accept_args a) {
  __shared__ int32_t sm_path[DSK_TREE_MAX_NODES];
  const int s = blockIdx.y, tid = threadIdx.x, lane = tid & (DSK_WAVE - 1);
  const bool first_wg = blockIdx.x == 0;
  const int64_t len = a.seq_len[s], row0 = a.seq_row0[s];
  int t0 = a.cu_new[s], n = a.cu_new[s + 1] - t0;
  if (t0 < 0 || n < 0 || t0 > a.n_tokens) {                     // malformed table: no nodes
    t0 = n = 0;
    if (first_wg && tid == 0) set_status(a.dev_status, DSK_ERR_SHAPE);
  }
  if (n > a.max_nodes || n > a.n_tokens - t0) {
    n = a.max_nodes < a.n_tokens - t0 ? a.max_nodes : a.n_tokens - t0;
    if (first_wg && tid == 0) set_status(a.dev_status, DSK_ERR_SHAPE);
  }
  // rows that the cache has left for this sequence; in place, the nodes from there on have none and end a path
  int64_t room = row0 >= 0 && len >= 0 ? a.total_rows - row0 - len : 0;
  if (room < 0) room = 0;
  const int placed = a.K != nullptr && a.Kd == nullptr && n > room ? (int)room : n;
  int parent[kAcceptRegs], draft[kAcceptRegs], target[kAcceptRegs];
#pragma unroll
  for (int r = 0; r < kAcceptRegs; ++r) {
    const int j = r * DSK_WAVE + lane;
    parent[r] = j < n ? a.parent[t0 + j] : -2;
    draft[r] = j < n ? a.draft_ids[t0 + j] : 0;
    target[r] = j < n ? a.target_ids[t0 + j] : 0;
  }
  const int most = room < a.max_path ? (int)room : a.max_path;
  int cur = n > 0 ? 0 : -1, taken = 0, choice = -1;
  while (cur >= 0) {                                            // ends: the next node is above the current one
    if (taken >= most || cur >= placed) {
      if (first_wg && tid == 0) set_status(a.dev_status, DSK_ERR_CAPACITY);
      break;
    }
    sm_path[taken++] = cur;                                     // all wavefronts write the same
    choice = 0;
#pragma unroll
    for (int r = 0; r < kAcceptRegs; ++r)
      if (cur / DSK_WAVE == r) choice = __builtin_amdgcn_readlane(target[r], cur & (DSK_WAVE - 1));
    int next = -1;
#pragma unroll
    for (int r = kAcceptRegs - 1; r >= 0; --r) {
      const int j = r * DSK_WAVE + lane;
      const uint64_t fits = __ballot(j > cur && j < n && parent[r] == cur && draft[r] == choice);
      if (fits) next = r * DSK_WAVE + __builtin_ctzll(fits);
    }
    cur = __builtin_amdgcn_readfirstlane(next);
  }
  __syncthreads();
  if (first_wg) {
    for (int i = tid; i < a.max_path; i += kAcceptThreads) {
      const int node = i < taken ? sm_path[i] : -1;
      a.path[(int64_t)s * a.max_path + i] = node;
      if (node >= 0 && a.token_ids != nullptr) a.token_ids[row0 + len + i] = a.draft_ids[t0 + node];
    }
    if (tid == 0) {
      a.n_accepted[s] = taken;
      a.len_new[s] = (int32_t)(len + taken);
      a.next_id[s] = choice;
    }
  }
  if (a.K == nullptr || taken == 0) return;
  // Rows are moved upwards in ascending order, each lane its own 16 bytes of every row: node path[i] >= i, so a row that is
  // overwritten has been read before (the batch is in registers when its first row is written).
  const int64_t item = (int64_t)blockIdx.x * kAcceptGroups + (tid >> 4);
  if (item >= (int64_t)a.n_layers * a.Hkv * 2) return;
  const bool is_v = item & 1;
  const int h = (int)((item >> 1) % a.Hkv);
  const int64_t l = (item >> 1) / a.Hkv;
  const int c = (tid & 15) * 8;
  const int64_t dst_tok = is_v ? a.v_stride_tok : a.k_stride_tok;
  uint16_t* dst = static_cast<uint16_t*>(is_v ? a.V : a.K) + l * (is_v ? a.v_stride_layer : a.k_stride_layer) +
                  h * (is_v ? a.v_stride_head : a.k_stride_head) + (row0 + len) * dst_tok + c;
  const uint16_t* src = dst;
  int64_t src_tok = dst_tok;
  if (a.Kd != nullptr) {
    src_tok = is_v ? a.vd_stride_tok : a.kd_stride_tok;
    src = static_cast<const uint16_t*>(is_v ? a.Vd : a.Kd) + l * (is_v ? a.vd_stride_layer : a.kd_stride_layer) +
          h * (is_v ? a.vd_stride_head : a.kd_stride_head) + t0 * src_tok + c;
  }
  for (int i0 = 0; i0 < taken; i0 += kAcceptBatch) {
    uint4 x[kAcceptBatch];
#pragma unroll
    for (int u = 0; u < kAcceptBatch; ++u) {
      const int i = i0 + u;
      x[u] = make_uint4(0, 0, 0, 0);
      if (i < taken) x[u] = *reinterpret_cast<const uint4*>(src + sm_path[i] * src_tok);
    }
#pragma unroll
    for (int u = 0; u < kAcceptBatch; ++u) {
      const int i = i0 + u;
      if (i < taken) *reinterpret_cast<uint4*>(dst + i * dst_tok) = x[u];
    }
  }
}

hipError_t launch_accept(const dsk_accept_args& a, hipStream_t st) {
  const int64_t items = a.K != nullptr ? (int64_t)a.n_layers * a.Hkv * 2 : 1;
  const int64_t wgs = (items + kAcceptGroups - 1) / kAcceptGroups;
  if (wgs > 0xFFFFFFFFll / kAcceptThreads) return hipErrorInvalidValue;
  accept_kernel<<<dim3((unsigned)wgs, (unsigned)a.B), dim3(kAcceptThreads), 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace dsk
