// New tokens into a cache of 8-bit codes with a scale per block of rows and head: queries and keys normed and rotated as in
// norm_rope_kernel, keys and values coded.  q, k, v come once and go once, K and V at half the bytes, so HBM bounds prompts and latency
// a decoding step.
//
// A scale is a power of two.  e4m3 has the same relative precision over 14 powers of two, so a finer scale would gain nothing but the
// last bit of the range below; in return a block's codes follow a larger scale exactly (but for those that become subnormal), and
// code * scale is a bf16 number, which the matrix instructions of the attention take as it is.
//
// A workgroup takes a block of rows of a sequence, all heads of it or some.  So that no scale has two writers, sequences begin with a
// block.  The angles of the block's tokens are made once, in LDS, for all heads; a wavefront takes 32 rows of a head of K or V at a time
// (blocks of 64 and 128 rows: two and four wavefronts, which exchange their largest values), or 32 rows of queries.  Its rows stay in
// registers between the largest value and the codes.
#include "dsk_internal.hpp"
#include "dsk_rope.hpp"

namespace dsk {

constexpr int kKv8Waves = 4;
constexpr int kKv8Threads = kKv8Waves * DSK_WAVE;
constexpr int kKv8Rows = 32;                   // of a wavefront
constexpr int kKv8Quads = kKv8Rows / 4;
constexpr int kKv8MinExp = -100, kKv8MaxExp = 120;
constexpr int kKv8Bias = 127;                  // of a scale's byte

// the least e with largest <= 448 * 2^e, 448 = 1.75 * 2^8
__device__ __forceinline__ int kv8_exponent(float largest) {
  const uint32_t u = __float_as_uint(largest);
  int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u);
  e = e > kKv8MinExp ? e : kKv8MinExp;         // (0 and subnormals too)
  return e < kKv8MaxExp ? e : kKv8MaxExp;
}

// eight values as codes; what is not finite becomes NaN
__device__ __forceinline__ uint2 kv8_encode(const float (&f)[8], float by) {
  int lo = 0, hi = 0;
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(f[0] * by, f[1] * by, lo, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(f[2] * by, f[3] * by, lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(f[4] * by, f[5] * by, hi, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(f[6] * by, f[7] * by, hi, true);
  return make_uint2((uint32_t)lo, (uint32_t)hi);
}

__device__ __forceinline__ void kv8_decode(const uint2& c, float (&f)[8]) {
  const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.x, true);
  const auto d = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.y, false), e = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.y, true);
  f[0] = a[0]; f[1] = a[1]; f[2] = b[0]; f[3] = b[1];
  f[4] = d[0]; f[5] = d[1]; f[6] = e[0]; f[7] = e[1];
}

// WPI wavefronts an item of K or V: blocks of 32 WPI rows
template <RopePairs PAIRS, int WPI>
__global__ __launch_bounds__(kKv8Threads) void kv8_append_kernel(dsk_kv8_append_args a, int groups) {
  constexpr int kBlock = WPI * kKv8Rows;
  constexpr bool kRotate = PAIRS != RopePairs::kNone, kInter = PAIRS == RopePairs::kInterleaved;
  __shared__ __align__(16) float sm_cos[kRotate ? kBlock : 1][kRopeHalf];
  __shared__ __align__(16) float sm_sin[kRotate ? kBlock : 1][kRopeHalf];
  __shared__ float sm_max[kKv8Waves];
  const int tid = threadIdx.x, lane = tid & (DSK_WAVE - 1), wave = __builtin_amdgcn_readfirstlane(tid / DSK_WAVE);
  const int grp = lane >> 4, c = lane & 15;
  const int s = blockIdx.z;

  // the sequence, and which of its new tokens are in this block: `count` from token `first` on, at rows `off` .. of the block
  const int tok0 = a.cu_new[s];
  int64_t n = (int64_t)a.cu_new[s + 1] - tok0;
  const int64_t row0 = a.seq_row0[s], len = a.seq_len[s];
  const bool report = blockIdx.x == 0 && blockIdx.y == 0 && tid == 0;
  if (tok0 < 0 || n < 0 || tok0 + n > a.n_tokens || n > a.max_new || row0 < 0 || len < 0) {
    if (report) set_status(a.dev_status, DSK_ERR_SHAPE);
    if (tok0 < 0 || row0 < 0 || len < 0) return;         // uniform, as all returns here
    n = n < a.n_tokens - (int64_t)tok0 ? n : a.n_tokens - (int64_t)tok0;
    n = n < a.max_new ? n : a.max_new;
  }
  if (n <= 0) return;
  if (row0 % kBlock != 0) {
    if (report) set_status(a.dev_status, DSK_ERR_ALIGN);
    return;
  }
  const int64_t begin = row0 + len;
  int64_t end = begin + n;
  if (end > a.total_rows) {
    if (report) set_status(a.dev_status, DSK_ERR_CAPACITY);
    end = a.total_rows;
  }
  const int64_t block = begin / kBlock + blockIdx.x, block_row = block * kBlock;
  const int64_t lo = begin > block_row ? begin : block_row, hi = end < block_row + kBlock ? end : block_row + kBlock;
  if (lo >= hi) return;
  const int off = (int)(lo - block_row), count = (int)(hi - lo);
  const int64_t tok = tok0 + (lo - begin);               // of the block's first new row

  int partner = lane, angle0 = 0;
  bool inside = false, upper = false;
  if constexpr (kRotate) {
    const int half = a.rot_dim / 2;
    for (int i = tid; i < count * half; i += kKv8Threads) {
      const int t = i / half, j = i - t * half;
      const int64_t pos = a.tok_pos != nullptr ? a.tok_pos[tok + t] : lo - row0 + t;
      // Whole turns are taken off in 64 bits.  What 32 bits then drop of the angle turns cos and sin on by as much.
      const double turns = (double)pos * ((double)a.inv_freq[j] * 0.15915494309189535);
      const double rest = 2.0 * (turns - rint(turns));
      const float near = (float)rest, left = (float)(rest - (double)near) * 3.14159265f;
      float si, co;
      sincospif(near, &si, &co);
      sm_cos[t][j] = fmaf(-si, left, co);
      sm_sin[t][j] = fmaf(co, left, si);
    }
    const int chunks = a.rot_dim / 8, half_chunks = chunks / 2;
    inside = c < chunks;
    upper = !kInter && c >= half_chunks;
    angle0 = !inside ? 0 : (kInter ? c * 4 : (upper ? c - half_chunks : c) * 8);
    if (!kInter && inside) partner = upper ? lane - half_chunks : lane + half_chunks;
    __syncthreads();
  }
  // a row of the block's token t, normed and rotated
  auto turn = [&](float (&f)[8], const float* weight, int t) {
    if (weight != nullptr) rope_scale(f, rope_square_sum(f), weight + c * 8, a.eps);
    if constexpr (kRotate) {
      float cs[8], sn[8];
#pragma unroll
      for (int e = 0; e < (kInter ? 4 : 8); e += 4) {
        const float4 x = *reinterpret_cast<const float4*>(&sm_cos[t][angle0 + e]);
        const float4 y = *reinterpret_cast<const float4*>(&sm_sin[t][angle0 + e]);
        cs[e] = x.x; cs[e + 1] = x.y; cs[e + 2] = x.z; cs[e + 3] = x.w;
        sn[e] = y.x; sn[e + 1] = y.y; sn[e + 2] = y.z; sn[e + 3] = y.w;
      }
      if (!kInter && !upper) {
#pragma unroll
        for (int e = 0; e < 8; ++e) sn[e] = -sn[e];
      }
      rope_turn<PAIRS>(f, cs, sn, inside, partner);
    }
  };

  // ---- keys and values: item 2 h is head h of K, item 2 h + 1 of V ----
  constexpr int kTogether = kKv8Waves / WPI;             // items of the workgroup at once
  const int part = wave % WPI;                           // of an item's rows
  for (int i0 = blockIdx.y * kTogether; i0 < 2 * a.Hkv; i0 += groups * kTogether) {   // uniform: barriers inside
    const int item = i0 + wave / WPI;
    const bool real = item < 2 * a.Hkv, is_v = item & 1;
    const int h = real ? item >> 1 : 0;
    uint8_t* scale = (is_v ? a.v_scale : a.k_scale) + h * a.scale_stride_head + block;
    const int before = real && off > 0 ? *scale : 0;
    const uint16_t* from = is_v ? static_cast<const uint16_t*>(a.v) + h * a.v_stride_head : static_cast<const uint16_t*>(a.k) + h * a.k_stride_head;
    const int64_t from_tok = is_v ? a.v_stride_tok : a.k_stride_tok;
    uint4 x[kKv8Quads];
#pragma unroll
    for (int u = 0; u < kKv8Quads; ++u) {
      const int r = part * kKv8Rows + 4 * u + grp - off;  // of the new rows
      x[u] = make_uint4(0, 0, 0, 0);
      if (real && r >= 0 && r < count) x[u] = load16<true>(from + (tok + r) * from_tok + c * 8);
    }
    float f[kKv8Quads][8], largest = 0.0f;
#pragma unroll
    for (int u = 0; u < kKv8Quads; ++u) {
      const int r0 = part * kKv8Rows + 4 * u - off;
      unpack8(x[u], f[u]);
      if (r0 + 3 < 0 || r0 >= count) continue;           // uniform: no row of the four is new
      if (!is_v) {
        int r = r0 + grp;
        r = r < 0 ? 0 : (r < count ? r : count - 1);     // lanes without a row turn zeros
        turn(f[u], a.k_weight, r);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float m = fabsf(f[u][e]);
        largest = fmaxf(largest, m < __builtin_inff() ? m : 0.0f);
      }
    }
    largest = wave_max(largest);
    if constexpr (WPI > 1) {
      if (lane == 0) sm_max[wave] = largest;
      __syncthreads();                                   // everybody has the scale as it was, too
#pragma unroll
      for (int w = 0; w < WPI; ++w) largest = fmaxf(largest, sm_max[wave - part + w]);
      __syncthreads();
    }
    if (!real) continue;
    int e = kv8_exponent(largest);
    const bool grows = off > 0 && e > before - kKv8Bias;
    if (off > 0 && !grows) e = before - kKv8Bias;
    const float by = ldexpf(1.0f, -e);
    unsigned char* to = (is_v ? static_cast<unsigned char*>(a.V) + h * a.vc_stride_head : static_cast<unsigned char*>(a.K) + h * a.kc_stride_head) + c * 8;
    const int64_t to_row = is_v ? a.vc_stride_tok : a.kc_stride_tok;
#pragma unroll
    for (int u = 0; u < kKv8Quads; ++u) {
      const int r = part * kKv8Rows + 4 * u + grp;
      if (r >= off && r < off + count) *reinterpret_cast<uint2*>(to + (block_row + r) * to_row) = kv8_encode(f[u], by);
    }
    if (grows) {                                         // uniform for the item
      const float less = ldexpf(1.0f, before - kKv8Bias - e);
      for (int u = 0; u < kKv8Quads; ++u) {
        const int r = part * kKv8Rows + 4 * u + grp;
        if (r >= off) continue;
        uint2* at = reinterpret_cast<uint2*>(to + (block_row + r) * to_row);
        float old[8];
        kv8_decode(*at, old);
        *at = kv8_encode(old, less);
      }
    }
    if (part == 0 && lane == 0 && (off == 0 || grows)) *scale = (uint8_t)(e + kKv8Bias);
  }

  // ---- queries: rows of the block's tokens and heads, one after the other ----
  if (a.q == nullptr) return;
  const int rows = count * a.Hq;
  for (int r0 = (blockIdx.y * kKv8Waves + wave) * kKv8Rows; r0 < rows; r0 += groups * kKv8Waves * kKv8Rows) {
    uint4 x[kKv8Quads];
#pragma unroll
    for (int u = 0; u < kKv8Quads; ++u) {
      const int r = r0 + 4 * u + grp, t = r / a.Hq, h = r - t * a.Hq;
      x[u] = make_uint4(0, 0, 0, 0);
      if (r < rows) x[u] = load16<true>(static_cast<const uint16_t*>(a.q) + (tok + t) * a.q_stride_tok + h * a.q_stride_head + c * 8);
    }
#pragma unroll
    for (int u = 0; u < kKv8Quads; ++u) {
      if (r0 + 4 * u >= rows) break;
      const int r = r0 + 4 * u + grp;
      float f[8];
      unpack8(x[u], f);
      turn(f, a.q_weight, r < rows ? r / a.Hq : 0);
      uint4 y = x[u];
      if (inside || a.q_weight != nullptr)
        y = make_uint4(pack_bf16_rne(f[0], f[1]), pack_bf16_rne(f[2], f[3]), pack_bf16_rne(f[4], f[5]), pack_bf16_rne(f[6], f[7]));
      if (r < rows) store16<false>(static_cast<uint16_t*>(a.q_out) + (tok * a.Hq + r) * DSK_HEAD_DIM + c * 8, y);
    }
  }
}

template <RopePairs PAIRS>
static void launch_pairs(const dsk_kv8_append_args& a, dim3 grid, int groups, hipStream_t st) {
  const dim3 block(kKv8Threads);
  if (a.scale_block == 32) kv8_append_kernel<PAIRS, 1><<<grid, block, 0, st>>>(a, groups);
  else if (a.scale_block == 64) kv8_append_kernel<PAIRS, 2><<<grid, block, 0, st>>>(a, groups);
  else kv8_append_kernel<PAIRS, 4><<<grid, block, 0, st>>>(a, groups);
}

hipError_t launch_kv8_append(const dsk_kv8_append_args& a, hipStream_t st) {
  // blocks that max_new tokens can meet, however the first of them lies
  const int64_t blocks = ((int64_t)a.max_new + a.scale_block - 2) / a.scale_block + 1;
  // Heads are spread over as many workgroups as it takes to have 16 wavefronts a CU; angles are made in each.
  const int64_t per_head = (int64_t)a.B * blocks * kKv8Waves;
  const int items = 2 * a.Hkv * (a.scale_block / kKv8Rows);
  const int most = (items + kKv8Waves - 1) / kKv8Waves;
  int64_t groups = (4096 + per_head - 1) / per_head;
  groups = groups < most ? groups : most;
  const dim3 grid((unsigned)blocks, (unsigned)groups, (unsigned)a.B);
  if (a.rot_dim == 0) launch_pairs<RopePairs::kNone>(a, grid, (int)groups, st);
  else if (a.flags & DSK_ROPE_INTERLEAVED) launch_pairs<RopePairs::kInterleaved>(a, grid, (int)groups, st);
  else if (a.rot_dim == DSK_HEAD_DIM) launch_pairs<RopePairs::kHalfAll>(a, grid, (int)groups, st);
  else launch_pairs<RopePairs::kHalf>(a, grid, (int)groups, st);
  return hipGetLastError();
}

}  // namespace dsk
