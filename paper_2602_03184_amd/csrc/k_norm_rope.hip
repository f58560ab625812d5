// Per-head norm and position rotation of queries and keys, keys and values into the cache rows of a slot map.  Every byte is
// read once and written once, so HBM bounds long prompts and latency a decoding step.  A row of 128 channels is spread over
// 16 lanes x 8 channels, as everywhere in the library; a wavefront takes rows of one token, four at a time, so that it makes
// the token's angles once: a lane each, in 64 bits (an angle of position 131071 has 17 bits before the point), handed round
// through LDS.
// 32K tokens of 32 / 8 heads (805 MB) 143 to 156 us, 5.2 to 5.6 TB/s, a large copy's rate; 14K tokens of 40 / 40 heads (875 MB)
// 184 to 190 us, whatever part is rotated and how; eight tokens 3.6 us.
#include "dsk_internal.hpp"
#include "dsk_rope.hpp"

namespace dsk {

constexpr int kRopeWaves = 4;
constexpr int kRopeThreads = kRopeWaves * DSK_WAVE;
constexpr int kRopeBatch = 4;                 // quads of rows of a wavefront on their way at once

template <RopePairs PAIRS>
__global__ __launch_bounds__(kRopeThreads) void norm_rope_kernel(dsk_norm_rope_args a, int waves_per_token, int quads_per_wave) {
  __shared__ float sm_cos[kRopeWaves][kRopeHalf];
  __shared__ float sm_sin[kRopeWaves][kRopeHalf];
  const int lane = threadIdx.x & (DSK_WAVE - 1), wave = threadIdx.x / DSK_WAVE;
  const int grp = lane >> 4, c = lane & 15;
  const int64_t w = (int64_t)blockIdx.x * kRopeWaves + wave;
  const int64_t t64 = w / waves_per_token;
  if (t64 >= a.n_tokens) return;                               // wavefronts share nothing: no barrier follows
  const int t = (int)t64;
  const int part = (int)(w - t64 * waves_per_token);
  const int64_t row = a.tok_row != nullptr ? a.tok_row[t] : t;
  if (row < 0 || row >= a.total_rows) return;
  const int nq = a.q != nullptr ? a.Hq : 0, nk = a.k != nullptr ? a.Hkv : 0, nv = a.v != nullptr ? a.Hkv : 0;
  const int rows = nq + nk + nv;
  const uint16_t* q = static_cast<const uint16_t*>(a.q) + t * a.q_stride_tok + c * 8;
  const uint16_t* k = static_cast<const uint16_t*>(a.k) + t * a.k_stride_tok + c * 8;
  const uint16_t* v = static_cast<const uint16_t*>(a.v) + t * a.v_stride_tok + c * 8;

  float cs[8], sn[8];                                          // interleaved: four pairs of a lane, in the first half
  int partner = lane;
  bool inside = false;                                         // the lane's channels are rotated; the others keep what they hold
  if constexpr (PAIRS != RopePairs::kNone) {
    const int half = a.rot_dim / 2;
    if (lane < half) {
      // whole turns are taken off in 64 bits, the rest fits 32
      const double turns = (double)a.tok_pos[t] * ((double)a.inv_freq[lane] * 0.15915494309189535);
      float si, co;
      sincospif((float)(turns - rint(turns)) * 2.0f, &si, &co);
      sm_cos[wave][lane] = co;
      sm_sin[wave][lane] = si;
    }
    __builtin_amdgcn_wave_barrier();
    constexpr bool kInter = PAIRS == RopePairs::kInterleaved;
    const int chunks = a.rot_dim / 8, half_chunks = chunks / 2;
    inside = c < chunks;
    const bool upper = !kInter && c >= half_chunks;
    const int first = !inside ? 0 : (kInter ? c * 4 : (upper ? c - half_chunks : c) * 8);
#pragma unroll
    for (int e = 0; e < (kInter ? 4 : 8); ++e) {
      cs[e] = sm_cos[wave][first + e];
      sn[e] = sm_sin[wave][first + e];
      if (!kInter && !upper) sn[e] = -sn[e];                   // mine * cos + partner * (-sin), or + partner * sin
    }
    if (!kInter && inside) partner = upper ? lane - half_chunks : lane + half_chunks;
  }
  const int quad0 = part * quads_per_wave;
  const int quads = (rows + 3) / 4;
  const int quad1 = quad0 + quads_per_wave < quads ? quad0 + quads_per_wave : quads;
  for (int b0 = quad0; b0 < quad1; b0 += kRopeBatch) {
    uint4 x[kRopeBatch];
#pragma unroll
    for (int u = 0; u < kRopeBatch; ++u) {
      int r = 4 * (b0 + u) + grp;
      r = r < rows ? r : rows - 1;                             // padding rows re-read a real one and are not written
      const uint16_t* at = r < nq ? q + r * a.q_stride_head
                                  : (r < nq + nk ? k + (r - nq) * a.k_stride_head : v + (r - nq - nk) * a.v_stride_head);
      if (b0 + u < quad1) x[u] = load16<true>(at);
    }
#pragma unroll
    for (int u = 0; u < kRopeBatch; ++u) {
      if (b0 + u >= quad1) break;
      const int r = 4 * (b0 + u) + grp;
      const bool is_q = r < nq, is_v = r >= nq + nk;
      uint4 y = x[u];
      float f[8];
      unpack8(y, f);
      const float* weight = is_q ? a.q_weight : a.k_weight;
      if (a.q_weight != nullptr || a.k_weight != nullptr) {
        const float ss = rope_square_sum(f);
        if (weight != nullptr && !is_v) {
          rope_scale(f, ss, weight + c * 8, a.eps);
        }
      }
      rope_turn<PAIRS>(f, cs, sn, inside, partner);
      if (!is_v && (inside || weight != nullptr))
        y = make_uint4(pack_bf16_rne(f[0], f[1]), pack_bf16_rne(f[2], f[3]), pack_bf16_rne(f[4], f[5]), pack_bf16_rne(f[6], f[7]));
      if (r < rows) {
        uint16_t* to = is_q ? static_cast<uint16_t*>(a.q_out) + ((int64_t)t * a.Hq + r) * DSK_HEAD_DIM
                       : is_v ? static_cast<uint16_t*>(a.V) + row * a.vc_stride_tok + (r - nq - nk) * a.vc_stride_head
                              : static_cast<uint16_t*>(a.K) + row * a.kc_stride_tok + (r - nq) * a.kc_stride_head;
        store16<false>(to + c * 8, y);
      }
    }
  }
}

hipError_t launch_norm_rope(const dsk_norm_rope_args& a, hipStream_t st) {
  const int rows = (a.q != nullptr ? a.Hq : 0) + (a.k != nullptr ? a.Hkv : 0) + (a.v != nullptr ? a.Hkv : 0);
  const int quads = (rows + 3) / 4;
  // A wavefront takes all heads of a token and makes its angles once, but where that leaves too few wavefronts (16 a CU) it
  // takes fewer: what bounds those calls is latency, and the angles are made in all of them at the same time.
  int per_wave = quads;
  while (per_wave > 1 && (int64_t)a.n_tokens * ((quads + per_wave - 1) / per_wave) < 4096) per_wave = (per_wave + 1) / 2;
  const int waves = (quads + per_wave - 1) / per_wave;
  const int64_t wgs = ((int64_t)a.n_tokens * waves + kRopeWaves - 1) / kRopeWaves;
  if (wgs > 0xFFFFFFFFll / kRopeThreads) return hipErrorInvalidValue;
  const dim3 grid((unsigned)wgs), block(kRopeThreads);
  if (a.rot_dim == 0) norm_rope_kernel<RopePairs::kNone><<<grid, block, 0, st>>>(a, waves, per_wave);
  else if (a.flags & DSK_ROPE_INTERLEAVED) norm_rope_kernel<RopePairs::kInterleaved><<<grid, block, 0, st>>>(a, waves, per_wave);
  else if (a.rot_dim == DSK_HEAD_DIM) norm_rope_kernel<RopePairs::kHalfAll><<<grid, block, 0, st>>>(a, waves, per_wave);
  else norm_rope_kernel<RopePairs::kHalf><<<grid, block, 0, st>>>(a, waves, per_wave);
  return hipGetLastError();
}

}  // namespace dsk
