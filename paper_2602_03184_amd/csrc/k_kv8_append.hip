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
// (blocks of 64 and 128 rows: two and four wavefronts, which exchange their largest values), or 32 rows of queries.
// 32K tokens of 32 + 8 heads take 157 to 161 us whatever part is rotated and how, 168 to 177 with blocks of 64.  Both paths in one kernel
// leave 64 to 73 scalar registers in vector lanes.
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

// Under the scales 2^e from 2^120 on the codes from 2^(128 - e) on would stand for 2^128 and more: four codes with those as the one before.
__device__ __forceinline__ uint32_t kv8_finite(uint32_t codes, int e) {
  const uint32_t least = 0x78u - 8 * (uint32_t)(e - kKv8MaxExp), size = codes & 0x7F7F7F7Fu;
  const uint32_t nan = size + 0x01010101u, out = (size + (0x80u - least) * 0x01010101u) & ~nan & 0x80808080u;   // a code's top bit
  const uint32_t bits = out - (out >> 7);                // the others of it
  return (codes & ~bits) | (bits & ((least - 1) * 0x01010101u));
}

__device__ __forceinline__ void kv8_decode(const uint2& c, float (&f)[8]) {
  const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.x, true);
  const auto d = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.y, false), e = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.y, true);
  f[0] = a[0]; f[1] = a[1]; f[2] = b[0]; f[3] = b[1];
  f[4] = d[0]; f[5] = d[1]; f[6] = e[0]; f[7] = e[1];
}

// WPI wavefronts an item of K or V: blocks of 32 WPI rows.  Workgroups 0 .. kv_groups - 1 of a block take K and V, those from there on the
// queries, QUADS * 4 rows a wavefront at a time.
template <RopePairs PAIRS, int WPI, int QUADS>
__global__ __launch_bounds__(kKv8Threads) void kv8_append_kernel(dsk_kv8_append_args a, int kv_groups, uint32_t by_heads) {
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

  // ---- what is taken first is on its way while the angles are made ----
  const bool queries = (int)blockIdx.y >= kv_groups;
  const int group = queries ? (int)blockIdx.y - kv_groups : (int)blockIdx.y, groups = queries ? (int)gridDim.y - kv_groups : kv_groups;
  constexpr int kTogether = kKv8Waves / WPI;             // items of the workgroup at once
  const int part = wave % WPI;                           // of an item's rows
  uint4 x[kKv8Quads];
  // item h is head h of K, item Hkv + h of V: neighbours in the projection's output side by side
  auto load_kv = [&](int item) {
    const bool real = item < 2 * a.Hkv, is_v = item >= a.Hkv;
    const int h = is_v ? item - a.Hkv : item;
    const uint16_t* from = is_v ? static_cast<const uint16_t*>(a.v) + h * a.v_stride_head : static_cast<const uint16_t*>(a.k) + h * a.k_stride_head;
    const int64_t from_tok = is_v ? a.v_stride_tok : a.k_stride_tok;
#pragma unroll
    for (int u = 0; u < kKv8Quads; ++u) {
      const int r = part * kKv8Rows + 4 * u + grp - off;  // of the new rows
      x[u] = make_uint4(0, 0, 0, 0);
      if (real && r >= 0 && r < count) x[u] = load16<true>(from + (tok + r) * from_tok + c * 8);
    }
  };
  // queries: rows of the block's tokens and heads, one after the other
  const int rows = queries ? count * a.Hq : 0;
  constexpr int kQueryRows = 4 * QUADS;
  auto token_of = [&](int r) { return a.Hq == 1 ? r : (int)__umulhi((uint32_t)r, by_heads); };   // r / Hq: exact as r * Hq is below 2^32
  auto load_q = [&](int r0) {
#pragma unroll
    for (int u = 0; u < QUADS; ++u) {
      const int r = r0 + 4 * u + grp, t = token_of(r), h = r - t * a.Hq;
      x[u] = make_uint4(0, 0, 0, 0);
      if (r < rows) x[u] = load16<true>(static_cast<const uint16_t*>(a.q) + (tok + t) * a.q_stride_tok + h * a.q_stride_head + c * 8);
    }
  };
  if (queries) load_q((group * kKv8Waves + wave) * kQueryRows);
  else load_kv(group * kTogether + wave / WPI);

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
  const float* const weight = queries ? a.q_weight : a.k_weight;
  __align__(16) float wt[8];
  if (weight != nullptr) {
    const float4 w0 = *reinterpret_cast<const float4*>(weight + c * 8), w1 = *reinterpret_cast<const float4*>(weight + c * 8 + 4);
    wt[0] = w0.x; wt[1] = w0.y; wt[2] = w0.z; wt[3] = w0.w;
    wt[4] = w1.x; wt[5] = w1.y; wt[6] = w1.z; wt[7] = w1.w;
  }
  auto turn = [&](float (&f)[8], int t) {
    if (weight != nullptr) rope_scale(f, rope_square_sum(f), wt, a.eps);
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

  // ---- keys and values ----
  for (int i0 = group * kTogether; !queries && i0 < 2 * a.Hkv; i0 += groups * kTogether) {   // uniform: barriers inside
    const int item = i0 + wave / WPI;
    const bool real = item < 2 * a.Hkv, is_v = item >= a.Hkv;
    const int h = !real ? 0 : (is_v ? item - a.Hkv : item);
    uint8_t* scale = (is_v ? a.v_scale : a.k_scale) + h * a.scale_stride_head + block;
    const int before = real && off > 0 ? *scale : 0;
    // The rows stay in registers from their largest value to the codes: made twice they need 124 registers instead of 148 to 168
    // (three wavefronts a SIMD, but for blocks of 128 rows), but five prompts of 40 heads then take 180 us instead of 159.
    float f[kKv8Quads][8];
    auto any_new = [&](int u) { return part * kKv8Rows + 4 * u - off + 3 >= 0 && part * kKv8Rows + 4 * u - off < count; };   // of the four
    float largest = 0.0f;
#pragma unroll
    for (int u = 0; u < kKv8Quads; ++u) {
      unpack8(x[u], f[u]);
      if (!any_new(u)) continue;                         // uniform
      if (!is_v) {
        int r = part * kKv8Rows + 4 * u + grp - off;
        r = r < 0 ? 0 : (r < count ? r : count - 1);     // lanes without a row turn zeros
        turn(f[u], r);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float m = fabsf(f[u][e]);
        largest = fmaxf(largest, m < __builtin_inff() ? m : 0.0f);
      }
    }
    load_kv(item + groups * kTogether);
    largest = wave_max(largest);
    if constexpr (WPI > 1) {
      if (lane == 0) sm_max[wave] = largest;
      __syncthreads();                                   // everybody has the scale as it was, too
#pragma unroll
      for (int w = 0; w < WPI; ++w) largest = fmaxf(largest, sm_max[wave - part + w]);
      __syncthreads();
    }
    int e = kv8_exponent(largest);
    const bool grows = off > 0 && e > before - kKv8Bias;
    if (off > 0 && !grows) e = before - kKv8Bias;
    const float by = ldexpf(1.0f, -e);
    unsigned char* to = (is_v ? static_cast<unsigned char*>(a.V) + h * a.vc_stride_head : static_cast<unsigned char*>(a.K) + h * a.kc_stride_head) + c * 8;
    const int64_t to_row = is_v ? a.vc_stride_tok : a.kc_stride_tok;
#pragma unroll
    for (int u = 0; u < kKv8Quads; ++u) {
      const int r = part * kKv8Rows + 4 * u + grp;
      if (real && r >= off && r < off + count) {
        uint2 codes = kv8_encode(f[u], by);
        if (e >= kKv8MaxExp) codes = make_uint2(kv8_finite(codes.x, e), kv8_finite(codes.y, e));
        *reinterpret_cast<uint2*>(to + (block_row + r) * to_row) = codes;
      }
    }
    if (!real) continue;
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

  // ---- queries ----
  if (!queries) return;
  for (int r0 = (group * kKv8Waves + wave) * kQueryRows; r0 < rows; r0 += groups * kKv8Waves * kQueryRows) {
    uint4 y[QUADS];
#pragma unroll
    for (int u = 0; u < QUADS; ++u) y[u] = x[u];
    load_q(r0 + groups * kKv8Waves * kQueryRows);
#pragma unroll
    for (int u = 0; u < QUADS; ++u) {
      if (r0 + 4 * u >= rows) break;
      const int r = r0 + 4 * u + grp;
      float f[8];
      unpack8(y[u], f);
      turn(f, r < rows ? token_of(r) : 0);
      if (inside || weight != nullptr)
        y[u] = make_uint4(pack_bf16_rne(f[0], f[1]), pack_bf16_rne(f[2], f[3]), pack_bf16_rne(f[4], f[5]), pack_bf16_rne(f[6], f[7]));
      if (r < rows) store16<false>(static_cast<uint16_t*>(a.q_out) + (tok * a.Hq + r) * DSK_HEAD_DIM + c * 8, y[u]);
    }
  }
}

template <RopePairs PAIRS, int WPI>
static void launch_block(const dsk_kv8_append_args& a, int64_t blocks, hipStream_t st) {
  // Heads and queries are spread over as many workgroups as it takes to have 16 wavefronts a CU, angles are made in each; a wavefront then
  // takes 8 rows of queries at a time instead of 32 (a token of 8 sequences, 32 + 8 heads: 5.9 us, nearly all of it the wait for the
  // sequence, the rows and the angles, one after the other; with a workgroup a block 8.2).  With more blocks than that one workgroup takes
  // a block's K and V, and its queries go to so many that each has about as many rows: 32K tokens of 32 + 8 heads 155 us with two (4.8 TB/s
  // of 0.74 GB read and written), 161 with one, 160 with four; two for K and V 162.
  const int64_t most = ((int64_t)2 * a.Hkv * WPI + kKv8Waves - 1) / kKv8Waves;
  const int64_t wanted = (4096 / kKv8Waves + a.B * blocks - 1) / (a.B * blocks);
  const int kv_groups = (int)(wanted < most ? wanted : most);
  const bool few = wanted > 1;
  const int64_t rows = (int64_t)(a.max_new < a.scale_block ? a.max_new : a.scale_block) * (a.q != nullptr ? a.Hq : 0);
  const int64_t q_most = (rows + 8 * kKv8Waves - 1) / (8 * kKv8Waves);
  const int even = (a.Hq + 2 * a.Hkv - 1) / (2 * a.Hkv);
  const int q_groups = a.q == nullptr ? 0 : (int)(few ? (wanted < q_most ? wanted : q_most) : even);
  const dim3 grid((unsigned)blocks, (unsigned)(kv_groups + q_groups), (unsigned)a.B), block(kKv8Threads);
  const uint32_t by_heads = a.q == nullptr || a.Hq == 1 ? 0xFFFFFFFFu : (uint32_t)(((1ull << 32) + a.Hq - 1) / a.Hq);
  if (few) kv8_append_kernel<PAIRS, WPI, 2><<<grid, block, 0, st>>>(a, kv_groups, by_heads);
  else kv8_append_kernel<PAIRS, WPI, kKv8Quads><<<grid, block, 0, st>>>(a, kv_groups, by_heads);
}

// blocks that new tokens of a sequence can meet, however the first of them lies; more than all tokens says nothing more
static int64_t most_blocks(const dsk_kv8_append_args& a) {
  const int64_t most = a.max_new < a.n_tokens ? a.max_new : a.n_tokens;
  return (most + a.scale_block - 2) / a.scale_block + 1;
}

// a launch has fewer than 2^32 threads in x
bool kv8_append_fits(const dsk_kv8_append_args& a) { return a.n_tokens == 0 || most_blocks(a) * kKv8Threads <= 0xFFFFFFFF; }

template <RopePairs PAIRS>
static void launch_pairs(const dsk_kv8_append_args& a, hipStream_t st) {
  const int64_t blocks = most_blocks(a);
  if (a.scale_block == 32) launch_block<PAIRS, 1>(a, blocks, st);
  else if (a.scale_block == 64) launch_block<PAIRS, 2>(a, blocks, st);
  else launch_block<PAIRS, 4>(a, blocks, st);
}

hipError_t launch_kv8_append(const dsk_kv8_append_args& args, hipStream_t st) {
  dsk_kv8_append_args a = args;
  a.max_new = a.max_new < a.n_tokens ? a.max_new : a.n_tokens;
  if (a.rot_dim == 0) launch_pairs<RopePairs::kNone>(a, st);
  else if (a.flags & DSK_ROPE_INTERLEAVED) launch_pairs<RopePairs::kInterleaved>(a, st);
  else if (a.rot_dim == DSK_HEAD_DIM) launch_pairs<RopePairs::kHalfAll>(a, st);
  else launch_pairs<RopePairs::kHalf>(a, st);
  return hipGetLastError();
}

}  // namespace dsk
