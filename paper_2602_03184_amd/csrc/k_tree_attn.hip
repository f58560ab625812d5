// Attention of the nodes of drafted trees over the cached prefix (or the selected slots of it) and their own ancestors.
//
// All nodes of a sequence and all query heads of a KV head's group meet the same keys: R = nodes * G rows against one K/V
// stream, 512 bytes and 512 R flop a key.  Up to some 150 rows HBM bounds that, beyond it the matrix cores do, so both products
// run on them and K and V are read once per 32 * QW rows.
//
// Products are taken transposed: S^T = K Q^T, then O^T = V^T P^T, with 32x32x16 matrix instructions.  A lane then has one query
// (column lane % 32) and 16 of a tile's 32 keys, so the softmax needs one exchange between the two halves of the wavefront for the
// maximum, rescaling is a product by a lane's own factor, and the weights that S^T leaves in a lane are already those that the
// second product wants there: key 16 t + 8 (e / 4) + 4 (lane / 32) + e % 4 in place e of step t, if V^T is read with the same
// order of keys (two transposing LDS reads of four keys each).  No weight passes through LDS.
//
// K and V tiles go through registers to LDS (the loads of the next tile are under way during the products of this one), 16-byte
// chunks swizzled by row so that the reads of both products and the writes are free of bank conflicts.
#include "dsk_attn_fold.hpp"
#include "dsk_common.hpp"
#include "dsk_internal.hpp"

namespace dsk {

typedef __bf16 tree_bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 tree_bf16x2 __attribute__((ext_vector_type(2)));
typedef float tree_f32x16 __attribute__((ext_vector_type(16)));
typedef float tree_f32x2 __attribute__((ext_vector_type(2)));
typedef short tree_s16x4 __attribute__((ext_vector_type(4)));

constexpr int kTreeTile = 32;                   // keys and queries of a matrix tile
constexpr int kTreeRowBytes = 2 * DSK_HEAD_DIM;
constexpr int kTreeMaxSlots = 256;              // selected slots of a workgroup
constexpr int kTreeMaxListed = 2048;            // and their tokens
constexpr int kTreeMaxSplit = 64;               // parts of a sequence: a lane each in the merge

__device__ __forceinline__ uint32_t tree_pack(float lo, float hi) {   // nearest-even bf16 pair
  const tree_f32x2 f = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, tree_bf16x2));
}

// bits x of a node's mask row for nodes 32 w .. 32 w + 31, of those that exist
struct TreeMask {
  const uint32_t* row;   // nullptr: the node sees itself and what is before it
  int node, n;
  __device__ __forceinline__ uint32_t word(int w) const {
    const int left = n - 32 * w;
    if (left <= 0) return 0;
    uint32_t bits;
    if (row != nullptr) bits = row[w];
    else {
      const int upto = node + 1 - 32 * w;
      bits = upto >= 32 ? 0xFFFFFFFFu : (upto > 0 ? (1u << upto) - 1u : 0u);
    }
    return left >= 32 ? bits : bits & ((1u << left) - 1u);
  }
  // the 32 keys of which the first is node j0 (below 0: keys of the prefix come first)
  __device__ __forceinline__ uint32_t window(int j0) const {
    if (j0 <= -32) return 0xFFFFFFFFu;
    if (j0 < 0) return (word(0) << -j0) | ((1u << -j0) - 1u);
    const int w = j0 >> 5, s = j0 & 31;
    const uint32_t lo = word(w) >> s;
    return s == 0 ? lo : lo | (word(w + 1) << (32 - s));
  }
};

struct TreeSplit {
  int nsplit, keys_per_split;   // parts of a sequence and their keys (a selection: tokens)
  int slots_per_split;          // with a selection
};

// TERMS: bf16 terms that a weight is split into for the second product, 1 (bf16 result) or 3 (all 24 bits of it: fp32 result)
template <int QW, int KW, int NT, int TERMS, bool SEL>
__global__ __launch_bounds__(QW * KW * DSK_WAVE, QW * KW <= 4 ? 2 : 1) void tree_attn_kernel(
    dsk_tree_attn_args a, int G, int q_tiles, TreeSplit sp, float scale, float2* __restrict__ part_ml,
    float* __restrict__ part_acc) {
  constexpr int kThreads = QW * KW * DSK_WAVE;
  constexpr int kKeys = kTreeTile * KW * NT;             // keys of a stage
  constexpr int kLoads = kKeys * 16 / kThreads;          // 16-byte chunks of K (and of V) of a thread
  constexpr int kRowStep = kThreads / 16;
  __shared__ __align__(16) unsigned char sm_kv[2 * kKeys * kTreeRowBytes];
  __shared__ float2 sm_ml[KW > 1 ? (KW - 1) * QW * DSK_WAVE : 1];
  __shared__ uint32_t sm_bad[2][KW * NT];                // rows of V that hold values that are not finite
  __shared__ int32_t sm_rows[SEL ? kTreeMaxListed : 1];
  __shared__ int32_t sm_slot[SEL ? 3 : 1][SEL ? kTreeMaxSlots : 1];
  __shared__ int32_t sm_wave[SEL ? kTreeMaxSlots / DSK_WAVE : 1];

  unsigned char* const sm_k = sm_kv;
  unsigned char* const sm_v = sm_kv + kKeys * kTreeRowBytes;
  const int split = blockIdx.x, s = blockIdx.z;
  const int hk = blockIdx.y / q_tiles, q_tile = blockIdx.y - hk * q_tiles;
  const int tid = threadIdx.x, lane = tid & (DSK_WAVE - 1), wave = tid / DSK_WAVE;
  const int qw = wave % QW, kw = wave / QW;
  const int col = lane & 31, half = lane >> 5;

  int tok0 = a.cu_new[s], n = a.cu_new[s + 1] - tok0;
  if (tok0 < 0 || n <= 0 || tok0 > a.n_tokens) return;
  n = n < a.max_nodes ? n : a.max_nodes;
  n = n < a.n_tokens - tok0 ? n : a.n_tokens - tok0;
  const int R = n * G, r0 = (q_tile * QW + qw) * kTreeTile;
  if (q_tile * QW * kTreeTile >= R) return;              // uniform: no row of this pass
  int64_t row0 = a.seq_row0[s], len = a.seq_len[s];
  if (row0 < 0 || row0 > a.total_rows || len < 0) row0 = len = 0;
  len = len < a.max_seqlen ? len : a.max_seqlen;
  len = len < a.total_rows - row0 ? len : a.total_rows - row0;
  // nodes that have a K/V row
  const int n_keys = a.Kd != nullptr || n < a.total_rows - row0 - len ? n : (int)(a.total_rows - row0 - len);

  // Keys of this workgroup: t in [t_begin, t_end), of which those below P are the prefix's and t - P is a node's number.
  int P, t_begin, t_end, used;
  if constexpr (SEL) {
    const int64_t sk = (int64_t)s * a.Hkv + hk;
    int count = a.sel_count[sk];
    count = count < 0 ? 0 : (count < a.k ? count : a.k);
    used = (count + sp.slots_per_split - 1) / sp.slots_per_split;
    used = used > 0 ? used : 1;                          // the nodes go with the last slots
    if (split >= used) return;
    const int first = split * sp.slots_per_split;
    const int here = count - first < sp.slots_per_split ? count - first : sp.slots_per_split;
    int start = 0, ln = 0;
    if (tid < here) {
      start = a.sel_start[sk * a.k + first + tid];
      ln = a.sel_len[sk * a.k + first + tid];
      ln = ln < a.b ? ln : a.b;
      if (start < 0 || ln <= 0 || start > a.total_rows - ln) ln = 0;
    }
    if (tid < kTreeMaxSlots) {
      const int incl = wave_incl_scan_i(ln, lane);
      if (lane == DSK_WAVE - 1) sm_wave[wave] = incl;
      sm_slot[0][tid] = incl - ln;
      sm_slot[1][tid] = start;
      sm_slot[2][tid] = ln;
    }
    __syncthreads();
    P = 0;
#pragma unroll
    for (int w = 0; w < kTreeMaxSlots / DSK_WAVE; ++w) P += sm_wave[w];
    for (int i = tid; i < here * a.b; i += kThreads) {
      const int slot = i / a.b, off = i - slot * a.b;
      int base = sm_slot[0][slot];
      for (int w = 0; w < slot / DSK_WAVE; ++w) base += sm_wave[w];
      if (off < sm_slot[2][slot]) sm_rows[base + off] = sm_slot[1][slot] + off;
    }
    __syncthreads();
    t_begin = 0;
    t_end = P + (split == used - 1 ? n_keys : 0);
  } else {
    P = (int)len;
    const int64_t T = len + n_keys;
    used = (int)((T + sp.keys_per_split - 1) / sp.keys_per_split);
    used = used > 0 ? used : 1;
    used = used < sp.nsplit ? used : sp.nsplit;          // (never more: the host counts max_seqlen + max_nodes keys)
    if (split >= used) return;
    t_begin = split * sp.keys_per_split;
    t_end = (int)(T - t_begin < sp.keys_per_split ? T : t_begin + sp.keys_per_split);
  }

  // ---- queries: a lane's row, 8 channels of every 16 of its half --------------------------------------------
  const bool busy = r0 < R;                              // rows for this wavefront (uniform over it)
  const int r = r0 + col;
  const bool real = r < R;
  const int node = real ? r / G : 0, g = real ? r - node * G : 0;
  const int64_t out_row = (int64_t)(tok0 + node) * a.Hq + hk * G + g;
  tree_bf16x8 qf[8];
  {
    const uint16_t* q = static_cast<const uint16_t*>(a.q) + out_row * DSK_HEAD_DIM + half * 8;
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      uint4 x = make_uint4(0, 0, 0, 0);
      if (real) x = *reinterpret_cast<const uint4*>(q + t * 16);
      qf[t] = __builtin_bit_cast(tree_bf16x8, x);
    }
  }
  const TreeMask mask = {a.mask != nullptr ? a.mask + (int64_t)(tok0 + node) * a.mask_words : nullptr, node,
                         t_end > P ? t_end - P : 0};

  // ---- tiles ------------------------------------------------------------------------------------------------
  const int lrow = tid >> 4, lc = tid & 15;
  const uint16_t* Kh = static_cast<const uint16_t*>(a.K) + hk * a.k_stride_head + lc * 8;
  const uint16_t* Vh = static_cast<const uint16_t*>(a.V) + hk * a.v_stride_head + lc * 8;
  uint4 kx[kLoads], vx[kLoads];
  auto v_row = [&](int t, const uint16_t* prefix, int chunk) -> const uint16_t* {   // V of key t, nullptr: no such key
    if (t < P) return prefix + (int64_t)(SEL ? sm_rows[t] : row0 + t) * a.v_stride_tok;
    const int j = t - P;
    if (t >= t_end) return nullptr;
    if (a.Kd == nullptr) return prefix + (row0 + len + j) * a.v_stride_tok;
    return static_cast<const uint16_t*>(a.Vd) + hk * a.vd_stride_head + (int64_t)(tok0 + j) * a.vd_stride_tok + chunk * 8;
  };
  auto k_row = [&](int t) -> const uint16_t* {
    if (t < P) return Kh + (int64_t)(SEL ? sm_rows[t] : row0 + t) * a.k_stride_tok;
    const int j = t - P;
    if (t >= t_end) return nullptr;
    if (a.Kd == nullptr) return Kh + (row0 + len + j) * a.k_stride_tok;
    return static_cast<const uint16_t*>(a.Kd) + hk * a.kd_stride_head + (int64_t)(tok0 + j) * a.kd_stride_tok + lc * 8;
  };
  auto fetch = [&](int t0) {
    if (t0 + kKeys <= P) {
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        const int t = t0 + lrow + u * kRowStep;
        kx[u] = load16<false>(Kh + (int64_t)(SEL ? sm_rows[t] : row0 + t) * a.k_stride_tok);
      }
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        const int t = t0 + lrow + u * kRowStep;
        vx[u] = load16<false>(Vh + (int64_t)(SEL ? sm_rows[t] : row0 + t) * a.v_stride_tok);
      }
    } else {
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        const int t = t0 + lrow + u * kRowStep;
        kx[u] = vx[u] = make_uint4(0, 0, 0, 0);
        if (t < t_end) {
          kx[u] = load16<false>(k_row(t));
          vx[u] = load16<false>(v_row(t, Vh, lc));
        }
      }
    }
  };

  float m = -__builtin_inff(), l = 0.0f;                 // running maximum (of q.K, not scaled) and this half's sum of a query
  tree_f32x16 O[4];
#pragma unroll
  for (int ct = 0; ct < 4; ++ct)
#pragma unroll
    for (int i = 0; i < 16; ++i) O[ct][i] = 0.0f;
  const float scale_log2 = scale * kLog2e;

  if (tid < KW * NT) sm_bad[0][tid] = 0;
  if (t_begin < t_end) fetch(t_begin);
  __syncthreads();
  int flip = 0;
  for (int t0 = t_begin; t0 < t_end; t0 += kKeys, flip ^= 1) {
    const bool plain = t0 + kKeys <= P;                  // prefix only: nothing is masked
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int row = lrow + u * kRowStep;
      if (!plain) {
        // a masked row may hold anything, and 0 * NaN is NaN: such values stay out of the product, and their row is noted
        uint32_t* w = reinterpret_cast<uint32_t*>(&vx[u]);
        bool bad = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if ((w[i] & 0x7F80u) == 0x7F80u) { w[i] &= 0xFFFF0000u; bad = true; }
          if ((w[i] & 0x7F800000u) == 0x7F800000u) { w[i] &= 0xFFFFu; bad = true; }
        }
        if (bad) atomicOr(&sm_bad[flip][row / kTreeTile], 1u << (row % kTreeTile));
      }
      *reinterpret_cast<uint4*>(sm_k + row * kTreeRowBytes + ((lc ^ (row & 15)) << 4)) = kx[u];
      *reinterpret_cast<uint4*>(sm_v + row * kTreeRowBytes + ((lc ^ ((row & 3) << 2)) << 4)) = vx[u];
    }
    __syncthreads();
    if (tid < KW * NT) sm_bad[flip ^ 1][tid] = 0;
    if (t0 + kKeys < t_end) fetch(t0 + kKeys);
    if (busy) {
#pragma unroll 1
      for (int sub = 0; sub < NT; ++sub) {
        const int tile = kw * NT + sub, tt = t0 + tile * kTreeTile;
        if (tt >= t_end) break;
        // S^T: keys x queries
        tree_f32x16 z;
#pragma unroll
        for (int i = 0; i < 16; ++i) z[i] = 0.0f;
        const unsigned char* kt = sm_k + (tile * kTreeTile + col) * kTreeRowBytes;
#pragma unroll
        for (int t = 0; t < 8; ++t) {
          const tree_bf16x8 kf = *reinterpret_cast<const tree_bf16x8*>(kt + (((2 * t + half) ^ (col & 15)) << 4));
          z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[t], z, 0, 0, 0);
        }
        uint32_t allow = 0xFFFFFFFFu;
        if (!plain) {
          allow = real ? mask.window(tt - P) : 0u;
#pragma unroll
          for (int i = 0; i < 16; ++i)
            z[i] = (allow >> (8 * (i >> 2) + 4 * half + (i & 3))) & 1u ? z[i] : -__builtin_inff();
        }
        float mx = z[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) mx = fmaxf(mx, z[i]);
        mx = fmaxf(mx, shfl_xor_f(mx, 32));
        // The reference of the exponents only has to be near the maximum: it moves when a query's grows by more than 8 in
        // log2 units, so most tiles rescale nothing, and the weights stay below 2^8.
        if (__any((mx - m) * scale_log2 > 8.0f)) {       // m = -inf: true unless nothing has been seen
          const float m_new = fmaxf(m, mx);
          const float f = m == -__builtin_inff() ? 0.0f : exp2_small((m - m_new) * scale_log2);
          l *= f;
#pragma unroll
          for (int ct = 0; ct < 4; ++ct)
#pragma unroll
            for (int i = 0; i < 16; ++i) O[ct][i] *= f;
          m = m_new;
        }
        const float ref = m == -__builtin_inff() ? 0.0f : m;
        float p[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          // the difference before the scale: exact for the largest, however large it is
          p[i] = exp2_small((z[i] - ref) * scale_log2);
          l += p[i];
        }
        tree_bf16x8 pf[TERMS][2];
#pragma unroll
        for (int term = 0; term < TERMS; ++term) {
          uint32_t w[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            w[i] = tree_pack(p[2 * i], p[2 * i + 1]);
            if (term + 1 < TERMS) {                      // what the terms so far leave
              p[2 * i] -= bf16_lo(w[i]);
              p[2 * i + 1] -= bf16_hi(w[i]);
            }
          }
          pf[term][0] = __builtin_bit_cast(tree_bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
          pf[term][1] = __builtin_bit_cast(tree_bf16x8, make_uint4(w[4], w[5], w[6], w[7]));
        }
        // O^T: channels x queries
        const int quad = (lane & 15) >> 2;               // of the four keys of a transposing read
        const unsigned char* vt = sm_v + (tile * kTreeTile + 4 * half + quad) * kTreeRowBytes +
                                  ((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) << 4) + ((lane & 1) << 3);
#pragma unroll
        for (int ct = 0; ct < 4; ++ct) {
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const unsigned char* at = vt + ((ct ^ quad) << 6) + t * 16 * kTreeRowBytes;
            const tree_s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) tree_s16x4*)(at));
            const tree_s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) tree_s16x4*)(at + 8 * kTreeRowBytes));
            const tree_bf16x8 vf = __builtin_bit_cast(tree_bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
            for (int term = TERMS - 1; term >= 0; --term)
              O[ct] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[term][t], O[ct], 0, 0, 0);
          }
        }
        if (!plain) {                                    // the values left out above, for the nodes that see them
          for (uint32_t bad = __builtin_amdgcn_readfirstlane(sm_bad[flip][tile]); bad != 0; bad &= bad - 1) {
            const int j = __builtin_ctz(bad);
            if (!((allow >> j) & 1u)) continue;
            const uint16_t* v = v_row(tt + j, Vh - lc * 8, 0) + 4 * half;
#pragma unroll
            for (int ct = 0; ct < 4; ++ct)
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const uint16_t x = v[ct * 32 + 8 * (i >> 2) + (i & 3)];
                if ((x & 0x7F80u) == 0x7F80u) O[ct][i] += bf16_to_f32(x);
              }
          }
        }
      }
    }
    __syncthreads();
  }
  l += shfl_xor_f(l, 32);

  // ---- wavefronts that took other keys for the same queries, in order ---------------------------------------
  if constexpr (KW > 1) {
    float* const sm_o = reinterpret_cast<float*>(sm_kv);   // (KW - 1) * QW blocks of 64 values of 64 lanes
    if (kw > 0 && busy) {
      const int at = (kw - 1) * QW + qw;
      sm_ml[at * DSK_WAVE + lane] = make_float2(m, l);
#pragma unroll
      for (int ct = 0; ct < 4; ++ct)
#pragma unroll
        for (int i = 0; i < 16; ++i) sm_o[(at * 64 + ct * 16 + i) * DSK_WAVE + lane] = O[ct][i];
    }
    __syncthreads();
    if (kw > 0) return;
    if (busy) {
      float M = m;
#pragma unroll
      for (int o = 0; o < KW - 1; ++o) M = fmaxf(M, sm_ml[(o * QW + qw) * DSK_WAVE + lane].x);
      const float f = m == -__builtin_inff() ? 0.0f : exp2_small((m - M) * scale_log2);
      l *= f;
#pragma unroll
      for (int ct = 0; ct < 4; ++ct)
#pragma unroll
        for (int i = 0; i < 16; ++i) O[ct][i] *= f;
#pragma unroll
      for (int o = 0; o < KW - 1; ++o) {
        const int at = o * QW + qw;
        const float2 ml = sm_ml[at * DSK_WAVE + lane];
        const float fo = ml.x == -__builtin_inff() ? 0.0f : exp2_small((ml.x - M) * scale_log2);
        l = fmaf(ml.y, fo, l);
#pragma unroll
        for (int ct = 0; ct < 4; ++ct)
#pragma unroll
          for (int i = 0; i < 16; ++i) O[ct][i] = fmaf(sm_o[(at * 64 + ct * 16 + i) * DSK_WAVE + lane], fo, O[ct][i]);
      }
      m = M;
    }
  }
  if (!real) return;
  // a lane's channels: four in a row, at 32 ct + 8 i + 4 half
  if (used == 1) {
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 x = make_float4(O[ct][4 * i] * inv, O[ct][4 * i + 1] * inv, O[ct][4 * i + 2] * inv, O[ct][4 * i + 3] * inv);
        const int64_t at = out_row * DSK_HEAD_DIM + ct * 32 + 8 * i + 4 * half;
        if (a.out != nullptr) *reinterpret_cast<float4*>(a.out + at) = x;
        if (a.out_bf16 != nullptr)
          *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out_bf16) + at) = make_uint2(tree_pack(x.x, x.y), tree_pack(x.z, x.w));
      }
    if (half == 0 && a.lse != nullptr) a.lse[out_row] = l > 0.0f ? (m * scale_log2 + log2f(l)) * kLn2 : -__builtin_inff();
  } else {
    const int64_t part = out_row * sp.nsplit + split;
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<float4*>(part_acc + part * DSK_HEAD_DIM + ct * 32 + 8 * i + 4 * half) =
            make_float4(O[ct][4 * i], O[ct][4 * i + 1], O[ct][4 * i + 2], O[ct][4 * i + 3]);
    if (half == 0) part_ml[part] = make_float2(m, l);
  }
}

// The parts of a row put together in order: a wavefront a row, two channels a lane.  `used` as in the kernel above.
constexpr int kTreeMergeWaves = 4;
constexpr int kTreeMergeBatch = 8;             // partials on their way at once

template <bool SEL>
__global__ __launch_bounds__(kTreeMergeWaves * DSK_WAVE) void tree_merge_kernel(
    dsk_tree_attn_args a, int G, TreeSplit sp, float scale_log2, const float2* __restrict__ part_ml,
    const float* __restrict__ part_acc) {
  const int s = blockIdx.y, lane = threadIdx.x & (DSK_WAVE - 1);
  const int item = blockIdx.x * kTreeMergeWaves + threadIdx.x / DSK_WAVE;
  const int node = item / a.Hq, h = item - node * a.Hq;
  int tok0 = a.cu_new[s], n = a.cu_new[s + 1] - tok0;
  if (tok0 < 0 || n <= 0 || tok0 > a.n_tokens) return;
  n = n < a.max_nodes ? n : a.max_nodes;
  n = n < a.n_tokens - tok0 ? n : a.n_tokens - tok0;
  if (node >= n) return;
  int used;
  if constexpr (SEL) {
    int count = a.sel_count[(int64_t)s * a.Hkv + h / G];
    count = count < 0 ? 0 : (count < a.k ? count : a.k);
    used = (count + sp.slots_per_split - 1) / sp.slots_per_split;
  } else {
    int64_t row0 = a.seq_row0[s], len = a.seq_len[s];
    if (row0 < 0 || row0 > a.total_rows || len < 0) row0 = len = 0;
    len = len < a.max_seqlen ? len : a.max_seqlen;
    len = len < a.total_rows - row0 ? len : a.total_rows - row0;
    const int n_keys = a.Kd != nullptr || n < a.total_rows - row0 - len ? n : (int)(a.total_rows - row0 - len);
    used = (int)((len + n_keys + sp.keys_per_split - 1) / sp.keys_per_split);
    used = used < sp.nsplit ? used : sp.nsplit;
  }
  if (used <= 1) return;                                 // finished by the kernel above
  const int64_t row = (int64_t)(tok0 + node) * a.Hq + h;
  const float2* ml = part_ml + row * sp.nsplit;
  const float2* acc = reinterpret_cast<const float2*>(part_acc + row * sp.nsplit * DSK_HEAD_DIM) + lane;
  float M = -__builtin_inff(), l = 0.0f;
  for (int c = lane; c < used; c += DSK_WAVE) M = fmaxf(M, ml[c].x);
  M = wave_max(M);
  float2 o = make_float2(0.0f, 0.0f);
  for (int c0 = 0; c0 < used; c0 += kTreeMergeBatch) {
    float2 x[kTreeMergeBatch], v[kTreeMergeBatch];
#pragma unroll
    for (int u = 0; u < kTreeMergeBatch; ++u) {
      const int c = c0 + u < used ? c0 + u : used - 1;
      v[u] = ml[c];
      x[u] = acc[(int64_t)c * (DSK_HEAD_DIM / 2)];
    }
#pragma unroll
    for (int u = 0; u < kTreeMergeBatch; ++u) {
      if (c0 + u >= used || v[u].x == -__builtin_inff()) continue;
      const float f = exp2_small((v[u].x - M) * scale_log2);
      l = fmaf(v[u].y, f, l);
      o.x = fmaf(x[u].x, f, o.x);
      o.y = fmaf(x[u].y, f, o.y);
    }
  }
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;
  o.x *= inv;
  o.y *= inv;
  if (a.out != nullptr) *reinterpret_cast<float2*>(a.out + row * DSK_HEAD_DIM + 2 * lane) = o;
  if (a.out_bf16 != nullptr)
    *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out_bf16) + row * DSK_HEAD_DIM + 2 * lane) = tree_pack(o.x, o.y);
  if (lane == 0 && a.lse != nullptr) a.lse[row] = l > 0.0f ? (M * scale_log2 + log2f(l)) * kLn2 : -__builtin_inff();
}

// ---- geometry: follows the host's bounds alone ---------------------------------------------------------------
struct TreeLaunch {
  TreeSplit sp;
  int q_waves;        // QW
  int q_tiles;        // passes over a (sequence, KV head)'s keys
  size_t part_acc, total;
};

static int tree_stage_keys(int q_waves) { return q_waves == 1 ? 128 : 64; }

static TreeLaunch tree_layout(const dsk_tree_attn_args& a) {
  TreeLaunch t;
  const int rows = a.max_nodes * (a.Hq / a.Hkv);
  t.q_waves = rows <= 32 ? 1 : (rows <= 64 ? 2 : (rows <= 128 ? 4 : 8));
  t.q_tiles = (rows + t.q_waves * kTreeTile - 1) / (t.q_waves * kTreeTile);
  constexpr int64_t kWant = 512;                         // workgroups: two per CU
  const int64_t heads = (int64_t)a.Hkv * t.q_tiles;
  t.sp.keys_per_split = t.sp.slots_per_split = 0;
  if (a.sel_start != nullptr) {
    const int64_t slots = (int64_t)a.k * a.B * heads;
    int64_t per = (slots + kWant - 1) / kWant;
    const int64_t least = (128 + a.b - 1) / a.b, most = kTreeMaxListed / a.b < kTreeMaxSlots ? kTreeMaxListed / a.b : kTreeMaxSlots;
    per = per > least ? per : least;
    per = per < most ? per : most;
    t.sp.slots_per_split = (int)per;
    t.sp.nsplit = (int)((a.k + per - 1) / per);
  } else {
    const int stage = tree_stage_keys(t.q_waves);
    int64_t keys = (int64_t)a.B * a.max_seqlen;
    keys = (keys < a.total_rows ? keys : a.total_rows) + (int64_t)a.B * a.max_nodes;
    const int64_t longest = (int64_t)a.max_seqlen + a.max_nodes;
    int64_t per = (keys * heads + kWant - 1) / kWant;
    const int64_t least = 256, fewest = (longest + kTreeMaxSplit - 1) / kTreeMaxSplit;
    per = per > least ? per : least;
    per = per > fewest ? per : fewest;
    per = (per + stage - 1) / stage * stage;
    t.sp.keys_per_split = (int)per;
    t.sp.nsplit = (int)((longest + per - 1) / per);
  }
  const size_t parts = t.sp.nsplit > 1 ? (size_t)a.n_tokens * a.Hq * t.sp.nsplit : 0;
  t.part_acc = align_up(parts * sizeof(float2));
  t.total = t.part_acc + align_up(parts * DSK_HEAD_DIM * sizeof(float));
  t.total = t.total > 256 ? t.total : 256;
  return t;
}

size_t tree_ws_bytes(const dsk_tree_attn_args& a) { return tree_layout(a).total; }

template <int QW, int KW, int NT>
static void launch_tree(const dsk_tree_attn_args& a, const TreeLaunch& t, float scale, float2* ml, float* acc, hipStream_t st) {
  const int G = a.Hq / a.Hkv;
  const dim3 grid((unsigned)t.sp.nsplit, (unsigned)(a.Hkv * t.q_tiles), (unsigned)a.B), block(QW * KW * DSK_WAVE);
  if (a.sel_start != nullptr) {
    if (a.out != nullptr) tree_attn_kernel<QW, KW, NT, 3, true><<<grid, block, 0, st>>>(a, G, t.q_tiles, t.sp, scale, ml, acc);
    else tree_attn_kernel<QW, KW, NT, 1, true><<<grid, block, 0, st>>>(a, G, t.q_tiles, t.sp, scale, ml, acc);
  } else {
    if (a.out != nullptr) tree_attn_kernel<QW, KW, NT, 3, false><<<grid, block, 0, st>>>(a, G, t.q_tiles, t.sp, scale, ml, acc);
    else tree_attn_kernel<QW, KW, NT, 1, false><<<grid, block, 0, st>>>(a, G, t.q_tiles, t.sp, scale, ml, acc);
  }
}

hipError_t launch_tree_attn(const dsk_tree_attn_args& a, hipStream_t st) {
  const TreeLaunch t = tree_layout(a);
  if ((int64_t)a.Hkv * t.q_tiles > 65535) return hipErrorInvalidValue;
  const float scale = a.scale != 0.0f ? a.scale : 0.08838834764831845f;   // 128^-1/2
  float2* ml = static_cast<float2*>(a.workspace);
  float* acc = reinterpret_cast<float*>(static_cast<unsigned char*>(a.workspace) + t.part_acc);
  if (t.q_waves == 1) launch_tree<1, 4, 1>(a, t, scale, ml, acc, st);
  else if (t.q_waves == 2) launch_tree<2, 2, 1>(a, t, scale, ml, acc, st);
  else if (t.q_waves == 4) launch_tree<4, 1, 2>(a, t, scale, ml, acc, st);
  else launch_tree<8, 1, 2>(a, t, scale, ml, acc, st);
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess || t.sp.nsplit <= 1) return err;
  const dim3 grid((unsigned)((a.max_nodes * a.Hq + kTreeMergeWaves - 1) / kTreeMergeWaves), (unsigned)a.B);
  const dim3 block(kTreeMergeWaves * DSK_WAVE);
  const int G = a.Hq / a.Hkv;
  if (a.sel_start != nullptr) tree_merge_kernel<true><<<grid, block, 0, st>>>(a, G, t.sp, scale * kLog2e, ml, acc);
  else tree_merge_kernel<false><<<grid, block, 0, st>>>(a, G, t.sp, scale * kLog2e, ml, acc);
  return hipGetLastError();
}

}  // namespace dsk
