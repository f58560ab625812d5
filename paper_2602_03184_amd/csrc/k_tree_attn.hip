// Attention of the nodes of drafted trees over the cached prefix (or the selected slots of it) and their own ancestors.
#include "dsk_attn_fold.hpp"
#include "dsk_common.hpp"
#include "dsk_internal.hpp"

namespace dsk {

__global__ __launch_bounds__(DSK_WAVE) void tree_attn_simple_kernel(dsk_tree_attn_args a) {
  const int G = a.Hq / a.Hkv;
  const int i = blockIdx.x, h = blockIdx.y, s = blockIdx.z, hk = h / G;
  const int lane = threadIdx.x, grp = lane >> 4, c = lane & 15;
  int t0 = a.cu_new[s], n = a.cu_new[s + 1] - t0;
  if (t0 < 0 || n < 0 || t0 > a.n_tokens) return;
  if (n > a.max_nodes) n = a.max_nodes;
  if (n > a.n_tokens - t0) n = a.n_tokens - t0;
  if (i >= n) return;
  int64_t row0 = a.seq_row0[s], len = a.seq_len[s];
  if (row0 < 0 || row0 > a.total_rows || len < 0) row0 = len = 0;
  if (len > a.max_seqlen) len = a.max_seqlen;
  if (len > a.total_rows - row0) len = a.total_rows - row0;
  const float scale = a.scale != 0.0f ? a.scale : 0.08838834764831845f;
  const int64_t sh = (int64_t)(t0 + i) * a.Hq + h;
  const QRow q = make_qrow(*reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q) + sh * DSK_HEAD_DIM + c * 8));
  float m = -__builtin_inff(), l = 0.0f, acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  auto fold = [&](const uint16_t* K, const uint16_t* V) {       // one key of each lane group
    // the difference to the largest is taken before the scale: exact for the largest itself, however large it is
    const float z = group16_sum(dot8_bf16(q, *reinterpret_cast<const uint4*>(K)));
    const float mn = fmaxf(m, z), f = expf((m - mn) * scale), p = expf((z - mn) * scale);
    float x[8];
    unpack8(*reinterpret_cast<const uint4*>(V), x);
    l = l * f + p;
    for (int e = 0; e < 8; ++e) acc[e] = acc[e] * f + p * x[e];
    m = mn;
  };
  const uint16_t* K = static_cast<const uint16_t*>(a.K) + hk * a.k_stride_head + c * 8;
  const uint16_t* V = static_cast<const uint16_t*>(a.V) + hk * a.v_stride_head + c * 8;
  if (a.sel_start == nullptr) {
    for (int64_t t = row0 + grp; t < row0 + len; t += 4) fold(K + t * a.k_stride_tok, V + t * a.v_stride_tok);
  } else {
    const int64_t sk = (int64_t)s * a.Hkv + hk;
    const int count = a.sel_count[sk] < a.k ? a.sel_count[sk] : a.k;
    for (int j = 0; j < count; ++j) {
      const int st = a.sel_start[sk * a.k + j];
      int ln = a.sel_len[sk * a.k + j];
      if (ln > a.b) ln = a.b;
      if (st < 0 || ln <= 0 || st > a.total_rows - ln) continue;
      for (int64_t t = st + grp; t < st + ln; t += 4) fold(K + t * a.k_stride_tok, V + t * a.v_stride_tok);
    }
  }
  for (int j = grp; j < n; j += 4) {
    const bool sees = a.mask != nullptr ? (a.mask[(int64_t)(t0 + i) * a.mask_words + j / 32] >> (j & 31)) & 1 : j <= i;
    if (!sees) continue;
    if (a.Kd != nullptr)
      fold(static_cast<const uint16_t*>(a.Kd) + hk * a.kd_stride_head + (t0 + j) * a.kd_stride_tok + c * 8,
           static_cast<const uint16_t*>(a.Vd) + hk * a.vd_stride_head + (t0 + j) * a.vd_stride_tok + c * 8);
    else if (row0 + len + j < a.total_rows)
      fold(K + (row0 + len + j) * a.k_stride_tok, V + (row0 + len + j) * a.v_stride_tok);
  }
  float M = fmaxf(m, shfl_xor_f(m, 16));
  M = fmaxf(M, shfl_xor_f(M, 32));
  const float f = m == -__builtin_inff() ? 0.0f : expf((m - M) * scale);
  l *= f;
  l += shfl_xor_f(l, 16);
  l += shfl_xor_f(l, 32);
  for (int e = 0; e < 8; ++e) {
    float x = acc[e] * f;
    x += shfl_xor_f(x, 16);
    x += shfl_xor_f(x, 32);
    x = l > 0.0f ? x / l : 0.0f;
    if (grp == 0) {
      if (a.out != nullptr) a.out[sh * DSK_HEAD_DIM + c * 8 + e] = x;
      if (a.out_bf16 != nullptr)
        static_cast<uint16_t*>(a.out_bf16)[sh * DSK_HEAD_DIM + c * 8 + e] = (uint16_t)(__float_as_uint(bf16_round_rne(x)) >> 16);
    }
  }
  if (lane == 0 && a.lse != nullptr) a.lse[sh] = l > 0.0f ? M * scale + logf(l) : -__builtin_inff();
}

size_t tree_ws_bytes(const dsk_tree_attn_args&) { return 256; }

hipError_t launch_tree_attn(const dsk_tree_attn_args& a, hipStream_t st) {
  tree_attn_simple_kernel<<<dim3((unsigned)a.max_nodes, (unsigned)a.Hq, (unsigned)a.B), dim3(DSK_WAVE), 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace dsk
