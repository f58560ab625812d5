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
// K and V tiles lie in LDS with their 16-byte chunks swizzled by row, so that the reads of both products and the writes are free
// of bank conflicts.  The general kernel copies stages of the prefix straight to LDS; the one for many rows has a schedule of its
// own and takes them through registers.  Stages that hold nodes go through registers in both, where what a mask
// may hide is looked at.
#include "dsk_attn_fold.hpp"
#include "dsk_common.hpp"
#include "dsk_internal.hpp"

#include <type_traits>

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
// Parts of a sequence at most.  One KV head (4 query heads, 16 nodes, 128K tokens): 36.1 us with 64, 29.5 with 128, 29.6 with 256;
// four sequences of 32K: 23.1, 25.9 and 33.6.
constexpr int kTreeMaxSplit = 128;
constexpr int kTreeMixedTiles = 16;             // tiles from the first one with a node on: 256 nodes, and a stage's other tiles
constexpr int kTreeTileBytes = kTreeTile * kTreeRowBytes;

__device__ __forceinline__ uint32_t tree_pack(float lo, float hi) {   // nearest-even bf16 pair
  const tree_f32x2 f = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, tree_bf16x2));
}

__device__ __forceinline__ uint32_t tree_pack_cut(float lo, float hi) {   // a bf16 pair, towards zero
  return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}

// 16 bytes at a uniform address and a lane's 32-bit offset, which is one instruction and no arithmetic; left to itself the
// compiler adds the parts the other way round, with a 64-bit product or sum per lane and load.
typedef const __attribute__((address_space(1))) char* tree_global;
template <bool STREAM>
__device__ __forceinline__ uint4 load16_at(tree_global base, uint32_t off) {
  asm("" : "+s"(base));
  typedef const __attribute__((address_space(1))) u32x4_t* at_t;
  const at_t at = (at_t)(base + off);
  u32x4_t v;
  if constexpr (STREAM) v = __builtin_nontemporal_load(at);
  else v = *at;
  return make_uint4(v.x, v.y, v.z, v.w);
}

// 16 bytes of each lane from its address to LDS, lane after lane from a uniform address on
template <bool STREAM>
__device__ __forceinline__ void lds_copy16(const void* from, unsigned char* to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)to, 16, 0,
                                   STREAM ? 2 : 0);
}
// every copy of this wavefront has arrived
__device__ __forceinline__ void lds_copies_done() { __builtin_amdgcn_s_waitcnt(0x0F70); }

// a bf16 pair with 0 for what is not finite
__device__ __forceinline__ uint32_t finite_bf16(uint32_t w) {
  if ((w & 0x7F80u) == 0x7F80u) w &= 0xFFFF0000u;
  if ((w & 0x7F800000u) == 0x7F800000u) w &= 0xFFFFu;
  return w;
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
  bool packed;                  // workgroups are numbered through the parts that there are, not by sequence
};

// What a sequence has in fact, malformed tables cut to the bounds that the host knows.
struct TreePlace {
  int tok0, n;          // its nodes' first token and their number; 0: nothing to do
  int64_t row0, len;    // prefix
  int n_keys;           // nodes that have a K/V row
  __device__ __forceinline__ TreePlace(const dsk_tree_attn_args& a, int s) {
    tok0 = a.cu_new[s];
    n = a.cu_new[s + 1] - tok0;
    if (tok0 < 0 || n <= 0 || tok0 > a.n_tokens) n = 0;
    n = n < a.max_nodes ? n : a.max_nodes;
    n = n < a.n_tokens - tok0 ? n : a.n_tokens - tok0;
    row0 = a.seq_row0[s];
    len = a.seq_len[s];
    const bool nowhere = row0 < 0 || row0 > a.total_rows || len < 0;
    if (nowhere) row0 = len = 0;
    len = len < a.max_seqlen ? len : a.max_seqlen;
    len = len < a.total_rows - row0 ? len : a.total_rows - row0;
    const int64_t left = nowhere ? 0 : a.total_rows - row0 - len;
    n_keys = a.Kd != nullptr || n < left ? n : (int)left;
  }
  // parts of its keys that have any; count: of the selection
  __device__ __forceinline__ int used(const TreeSplit& sp, bool selected, int count) const {
    int64_t u;
    if (selected) {
      u = (count + sp.slots_per_split - 1) / sp.slots_per_split;
    } else {
      u = (len + n_keys + sp.keys_per_split - 1) / sp.keys_per_split;
    }
    u = u > 0 ? u : 1;                                   // the nodes go with the last slots
    return (int)(u < sp.nsplit ? u : sp.nsplit);         // (never more: the host counts max_seqlen + max_nodes keys)
  }
};

// The p-th part of all sequences', those of a sequence one after the other; false: there are fewer.  Every wavefront for itself.
__device__ __forceinline__ bool tree_find(const dsk_tree_attn_args& a, const TreeSplit& sp, int p, int& s, int& split) {
  const int lane = threadIdx.x & (DSK_WAVE - 1);
  for (int s0 = 0; s0 < a.B; s0 += DSK_WAVE) {
    int parts = 0;
    if (s0 + lane < a.B) {
      const TreePlace at(a, s0 + lane);
      if (at.n > 0) parts = at.used(sp, false, 0);
    }
    const int incl = wave_incl_scan_i(parts, lane), total = __builtin_amdgcn_readlane(incl, DSK_WAVE - 1);
    if (p < total) {
      const int before = __builtin_popcountll(__ballot(incl <= p));    // sequences
      s = s0 + before;
      split = before > 0 ? p - __builtin_amdgcn_readlane(incl, before - 1) : p;
      return true;
    }
    p -= total;
  }
  return false;
}

// What a workgroup takes: part, sequence, KV head and pass; false: nothing.
struct TreeWork {
  int split, s, hk, q_tile;
  __device__ __forceinline__ bool find(const dsk_tree_attn_args& a, const TreeSplit& sp, int q_tiles) {
    const int y = sp.packed ? blockIdx.x : blockIdx.y;
    hk = y / q_tiles;
    q_tile = y - hk * q_tiles;
    if (sp.packed) return tree_find(a, sp, blockIdx.y, s, split);
    split = blockIdx.x;
    s = blockIdx.z;
    return true;
  }
};

__device__ __forceinline__ int tree_sel_count(const dsk_tree_attn_args& a, int s, int hk) {
  const int count = a.sel_count[(int64_t)s * a.Hkv + hk];
  return count < 0 ? 0 : (count < a.k ? count : a.k);
}

// A part of a selection: how many slots there are in all, and a thread's slot of the part (as the caller wrote it).  Read before
// anything is known about the sequence, so that it costs no round trip of its own.
template <bool SEL>
struct TreeSlots {
  int count = 0, start = 0, len = 0;
  __device__ __forceinline__ TreeSlots(const dsk_tree_attn_args& a, const TreeSplit& sp, int s, int hk, int split) {
    if constexpr (SEL) {
      const int tid = threadIdx.x, first = split * sp.slots_per_split;
      count = tree_sel_count(a, s, hk);
      if (tid < sp.slots_per_split && tid < a.k - first) {
        const int64_t at = ((int64_t)s * a.Hkv + hk) * a.k + first + tid;
        start = a.sel_start[at];
        len = a.sel_len[at];
      }
    }
  }
};

// The keys of a workgroup: t in [t_begin, t_end), of which those below P are the prefix's and t - P is a node's number.  A
// stage of LOADS * THREADS / 16 keys is copied to LDS, or fetched to registers and put there, a thread taking a 16-byte chunk of
// every THREADS / 16-th row.
template <int THREADS, int LOADS, bool SEL, bool STREAM>
struct TreeKeys {
  static constexpr int kRowStep = THREADS / 16;
  static constexpr int kKeys = LOADS * kRowStep;
  int P, t_begin, t_end;
  int t_mixed;                          // first stage that is not the prefix's alone
  int lrow, lc;
  int64_t kst, vst, row0;
  const uint16_t *K, *V, *Kn, *Vn;      // this lane's chunk of the prefix (of the whole cache with SEL) and of the nodes
  int64_t knst, vnst;
  tree_global Ku, Vu;                   // the prefix of the head, without the lane's part
  uint32_t k_off, v_off;                // the lane's part in bytes
  const int32_t* rows;                  // cache rows of the selected tokens, in LDS
  struct Regs {
    uint4 k[LOADS], v[LOADS];
  };

  __device__ __forceinline__ TreeKeys(const dsk_tree_attn_args& a, const TreeSplit& sp, const TreePlace& at, const TreeSlots<SEL>& slots,
                                      int hk, int split, int used, int32_t* sm_rows) {
    const int tid = threadIdx.x, lane = tid & (DSK_WAVE - 1), wave = tid / DSK_WAVE;
    lrow = tid >> 4;
    lc = tid & 15;
    kst = a.k_stride_tok;
    vst = a.v_stride_tok;
    row0 = SEL ? 0 : at.row0;
    rows = sm_rows;
    K = static_cast<const uint16_t*>(a.K) + hk * a.k_stride_head + row0 * kst;
    V = static_cast<const uint16_t*>(a.V) + hk * a.v_stride_head + row0 * vst;
    Ku = (tree_global)K;
    Vu = (tree_global)V;
    k_off = (uint32_t)(lrow * (int)kst + lc * 8) * 2u;   // 32 rows of 2^24 channels at most
    v_off = (uint32_t)(lrow * (int)vst + lc * 8) * 2u;
    K += lc * 8;
    V += lc * 8;
    if (a.Kd != nullptr) {
      knst = a.kd_stride_tok;
      vnst = a.vd_stride_tok;
      Kn = static_cast<const uint16_t*>(a.Kd) + hk * a.kd_stride_head + at.tok0 * knst + lc * 8;
      Vn = static_cast<const uint16_t*>(a.Vd) + hk * a.vd_stride_head + at.tok0 * vnst + lc * 8;
    } else {
      knst = kst;
      vnst = vst;
      Kn = K + (at.row0 - row0 + at.len) * kst;
      Vn = V + (at.row0 - row0 + at.len) * vst;
    }
    if constexpr (SEL) {
      __shared__ int32_t sm_slot[3][kTreeMaxSlots];
      __shared__ int32_t sm_wave[kTreeMaxSlots / DSK_WAVE];
      const int first = split * sp.slots_per_split;
      const int here = slots.count - first < sp.slots_per_split ? slots.count - first : sp.slots_per_split;
      const int start = slots.start;
      int ln = slots.len < a.b ? slots.len : a.b;
      if (tid >= here || start < 0 || ln <= 0 || start > a.total_rows - ln) ln = 0;
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
      for (int i = tid; i < here * a.b; i += THREADS) {
        const int slot = i / a.b, off = i - slot * a.b;
        int base = sm_slot[0][slot];
        for (int w = 0; w < slot / DSK_WAVE; ++w) base += sm_wave[w];
        if (off < sm_slot[2][slot]) sm_rows[base + off] = sm_slot[1][slot] + off;
      }
      __syncthreads();
      t_begin = 0;
      t_end = P + (split == used - 1 ? at.n_keys : 0);
    } else {
      P = (int)at.len;
      t_begin = split * sp.keys_per_split;
      t_end = P + at.n_keys - t_begin < sp.keys_per_split ? P + at.n_keys : t_begin + sp.keys_per_split;
    }
    t_mixed = P > t_begin ? t_begin + (P - t_begin) / kKeys * kKeys : t_begin;
  }
  __device__ __forceinline__ bool plain(int t0) const { return t0 + kKeys <= P; }   // a stage of the prefix alone: nothing is masked
  __device__ __forceinline__ int nodes() const { return t_end > P ? t_end - P : 0; }
  __device__ __forceinline__ const uint16_t* k_at(int t) const {
    return t < P ? K + (int64_t)(SEL ? rows[t] : t) * kst : Kn + (int64_t)(t - P) * knst;
  }
  __device__ __forceinline__ const uint16_t* v_at(int t) const {
    return t < P ? V + (int64_t)(SEL ? rows[t] : t) * vst : Vn + (int64_t)(t - P) * vnst;
  }
  // a stage of the prefix alone
  __device__ __forceinline__ void fetch_plain(Regs& x, int t0) const {
    static_assert(!SEL, "rows in order");
#pragma unroll
    for (int u = 0; u < LOADS; ++u) x.k[u] = load16_at<STREAM>(Ku + (t0 + u * kRowStep) * kst * 2, k_off);
#pragma unroll
    for (int u = 0; u < LOADS; ++u) x.v[u] = load16_at<STREAM>(Vu + (t0 + u * kRowStep) * vst * 2, v_off);
  }
  __device__ __forceinline__ void fetch_mixed(Regs& x, int t0) const {
#pragma unroll
    for (int u = 0; u < LOADS; ++u) {
      const int t = t0 + lrow + u * kRowStep;
      x.k[u] = x.v[u] = make_uint4(0, 0, 0, 0);
      if (t < t_end) {
        x.k[u] = load16<false>(k_at(t));
        x.v[u] = load16<false>(v_at(t));
      }
    }
  }
  // The same straight to LDS, with no register between.  A wavefront's 1 KB lies in LDS in the order of its lanes, so the
  // swizzle is in what a lane reads: chunk lc of a row is that chunk's place, K's or V's chunk lc ^ f(row) belongs there.
  __device__ __forceinline__ void copy_plain(int t0, unsigned char* sm_k, unsigned char* sm_v) const {
    const int w_row = (int)(threadIdx.x / DSK_WAVE) * 4;
#pragma unroll
    for (int u = 0; u < LOADS; ++u) {
      const int row = lrow + u * kRowStep, t = t0 + row;
      const int kc = (lc ^ (row & 15)) - lc, vc = (lc ^ ((row & 3) << 2)) - lc;
      const int64_t r = SEL ? rows[t] : t;
      lds_copy16<STREAM>(K + r * kst + kc * 8, sm_k + (u * kRowStep + w_row) * kTreeRowBytes);
      lds_copy16<STREAM>(V + r * vst + vc * 8, sm_v + (u * kRowStep + w_row) * kTreeRowBytes);
    }
  }
  // sm_bad: a word per tile from t_mixed on, zero before; rows of V that hold values that are not finite
  template <bool MIXED>
  __device__ __forceinline__ void put(Regs& x, int t0, unsigned char* sm_k, unsigned char* sm_v, uint32_t* sm_bad) const {
#pragma unroll
    for (int u = 0; u < LOADS; ++u) {
      const int row = lrow + u * kRowStep;
      uint4 v = x.v[u];
      if constexpr (MIXED) {
        // a masked row may hold anything, and 0 * NaN is NaN: such values stay out of the product, and their row is noted
        v = make_uint4(finite_bf16(v.x), finite_bf16(v.y), finite_bf16(v.z), finite_bf16(v.w));
        if (v.x != x.v[u].x || v.y != x.v[u].y || v.z != x.v[u].z || v.w != x.v[u].w)
          atomicOr(&sm_bad[(t0 - t_mixed + row) / kTreeTile], 1u << (row % kTreeTile));
      }
      *reinterpret_cast<uint4*>(sm_k + row * kTreeRowBytes + ((lc ^ (row & 15)) << 4)) = x.k[u];
      *reinterpret_cast<uint4*>(sm_v + row * kTreeRowBytes + ((lc ^ ((row & 3) << 2)) << 4)) = v;
    }
  }
};

// A wavefront's 32 queries: a lane has query lane % 32 and of a tile's 32 keys those at 8 (i / 4) + 4 (lane / 32) + i % 4.
struct TreeQueries {
  bool busy, real;      // the wavefront has rows; the lane's row exists
  int col, half, node;
  int64_t out_row;
  TreeMask mask;
  tree_bf16x8 q[8];     // channels 16 t + 8 half .. + 7

  __device__ __forceinline__ TreeQueries(const dsk_tree_attn_args& a, const TreePlace& at, int G, int hk, int r0) {
    const int lane = threadIdx.x & (DSK_WAVE - 1);
    col = lane & 31;
    half = lane >> 5;
    busy = r0 < at.n * G;
    const int r = r0 + col;
    real = r < at.n * G;
    node = real ? r / G : 0;
    out_row = (int64_t)(at.tok0 + node) * a.Hq + hk * G + (real ? r - node * G : 0);
    const uint16_t* from = static_cast<const uint16_t*>(a.q) + out_row * DSK_HEAD_DIM + half * 8;
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      uint4 x = make_uint4(0, 0, 0, 0);
      if (real) x = *reinterpret_cast<const uint4*>(from + t * 16);
      q[t] = __builtin_bit_cast(tree_bf16x8, x);
    }
    mask.row = a.mask != nullptr ? a.mask + (int64_t)(at.tok0 + node) * a.mask_words : nullptr;
    mask.node = node;
    mask.n = 0;                                          // until the keys are known
  }
  __device__ __forceinline__ uint32_t allowed(int t0, int P) const { return real ? mask.window(t0 - P) : 0u; }
};

// Fragments of a tile of 32 keys.
struct TreeKFrag {
  tree_bf16x8 k[8];
  template <int FROM, int TO>
  __device__ __forceinline__ void read(const unsigned char* sm_k, const TreeQueries& qs) {
    const unsigned char* at = sm_k + qs.col * kTreeRowBytes;
#pragma unroll
    for (int t = FROM; t < TO; ++t)
      k[t] = *reinterpret_cast<const tree_bf16x8*>(at + (((2 * t + qs.half) ^ (qs.col & 15)) << 4));
  }
  // logits: S^T = K Q^T
  template <int FROM, int TO>
  __device__ __forceinline__ void add(tree_f32x16& z, const TreeQueries& qs) const {
    if constexpr (FROM == 0) {
#pragma unroll
      for (int i = 0; i < 16; ++i) z[i] = 0.0f;
    }
#pragma unroll
    for (int t = FROM; t < TO; ++t) z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[t], qs.q[t], z, 0, 0, 0);
  }
};

__device__ __forceinline__ void tree_hide(tree_f32x16& z, uint32_t allow, int half) {
#pragma unroll
  for (int i = 0; i < 16; ++i)
    z[i] = (allow >> (8 * (i >> 2) + 4 * half + (i & 3))) & 1u ? z[i] : -__builtin_inff();
}

// the larger of a value and the other half's
__device__ __forceinline__ float tree_half_max(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ float tree_max(const tree_f32x16& z) {
  float m = z[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) m = fmaxf(m, z[i]);
  return tree_half_max(m);
}

// The weights of a tile, in TERMS bf16 terms.  A single term, or the last of two, is rounded to nearest.  The others are cut towards
// zero, 8 bits each, and what is left is made a little more each time, so that no term of a weight above 2^-80 is 0 or negative: an
// infinite value then stays infinite in the sum over them, where 0 * inf and inf - inf would make it NaN.  Two terms are off by 2^-16
// of the weight at most; three add up to 1.1 * 2^-24 .. 3 * 2^-24 more than it (2^-23 in the mean; taking what is left exactly and
// bounding the terms from below made fp32 calls 3 to 5 % slower).
template <int TERMS>
struct TreeWeights {
  tree_bf16x8 w[TERMS][2];
  __device__ __forceinline__ void set(float (&p)[16]) {
#pragma unroll
    for (int term = 0; term < TERMS; ++term) {
      uint32_t x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (TERMS == 1) {
          x[i] = tree_pack(p[2 * i], p[2 * i + 1]);
        } else {
          x[i] = TERMS == 2 && term == 1 ? tree_pack(p[2 * i], p[2 * i + 1]) : tree_pack_cut(p[2 * i], p[2 * i + 1]);
          if (term + 1 < TERMS) {                        // what the terms so far leave
            const float more = term == 0 ? 1.0f + 0x1p-23f : 1.0f + 0x1p-17f;
            p[2 * i] = fmaf(p[2 * i], more, -bf16_lo(x[i]));
            p[2 * i + 1] = fmaf(p[2 * i + 1], more, -bf16_hi(x[i]));
          }
        }
      }
      w[term][0] = __builtin_bit_cast(tree_bf16x8, make_uint4(x[0], x[1], x[2], x[3]));
      w[term][1] = __builtin_bit_cast(tree_bf16x8, make_uint4(x[4], x[5], x[6], x[7]));
    }
  }
};

struct TreeVFrag {
  tree_bf16x8 v[4][2];
  // a lane's place in a tile for channels 32 ct .. 32 ct + 31
  static __device__ __forceinline__ int place(int ct) {
    const int lane = threadIdx.x & (DSK_WAVE - 1), half = lane >> 5;
    const int quad = (lane & 15) >> 2;                   // of the four keys of a transposing read
    return (4 * half + quad) * kTreeRowBytes + ((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) << 4) + ((lane & 1) << 3) + ((ct ^ quad) << 6);
  }
  template <int T>                                       // 16 of the keys
  __device__ __forceinline__ void read(const unsigned char* sm_v) {
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) {
      const unsigned char* at = sm_v + place(ct) + T * 16 * kTreeRowBytes;
      const tree_s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) tree_s16x4*)(at));
      const tree_s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (__attribute__((address_space(3))) tree_s16x4*)(at + 8 * kTreeRowBytes));
      v[ct][T] = __builtin_bit_cast(tree_bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  }
  // All 32 keys while copies to other parts of LDS are under way: for the builtin the compiler would wait for those first, as it
  // does not see that they are other parts.
  __device__ __forceinline__ void read_beside_copies(const unsigned char* sm_v) {
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    const uint32_t at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const unsigned char*)sm_v;
    u32x2 x[4][4];
    static_assert(kTreeRowBytes == 256, "offsets: 8 rows");
    asm volatile(
        "ds_read_b64_tr_b16 %0, %16\n\tds_read_b64_tr_b16 %1, %16 offset:2048\n\t"
        "ds_read_b64_tr_b16 %4, %17\n\tds_read_b64_tr_b16 %5, %17 offset:2048\n\t"
        "ds_read_b64_tr_b16 %8, %18\n\tds_read_b64_tr_b16 %9, %18 offset:2048\n\t"
        "ds_read_b64_tr_b16 %12, %19\n\tds_read_b64_tr_b16 %13, %19 offset:2048\n\t"
        "ds_read_b64_tr_b16 %2, %16 offset:4096\n\tds_read_b64_tr_b16 %3, %16 offset:6144\n\t"
        "ds_read_b64_tr_b16 %6, %17 offset:4096\n\tds_read_b64_tr_b16 %7, %17 offset:6144\n\t"
        "ds_read_b64_tr_b16 %10, %18 offset:4096\n\tds_read_b64_tr_b16 %11, %18 offset:6144\n\t"
        "ds_read_b64_tr_b16 %14, %19 offset:4096\n\tds_read_b64_tr_b16 %15, %19 offset:6144\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[0][2]), "=&v"(x[0][3]), "=&v"(x[1][0]), "=&v"(x[1][1]), "=&v"(x[1][2]),
          "=&v"(x[1][3]), "=&v"(x[2][0]), "=&v"(x[2][1]), "=&v"(x[2][2]), "=&v"(x[2][3]), "=&v"(x[3][0]), "=&v"(x[3][1]),
          "=&v"(x[3][2]), "=&v"(x[3][3])
        : "v"(at + place(0)), "v"(at + place(1)), "v"(at + place(2)), "v"(at + place(3))
        : "memory");
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
      for (int t = 0; t < 2; ++t)
        v[ct][t] = __builtin_bit_cast(tree_bf16x8, make_uint4(x[ct][2 * t].x, x[ct][2 * t].y, x[ct][2 * t + 1].x, x[ct][2 * t + 1].y));
  }
  // O^T += V^T P^T
  template <int TERMS>
  __device__ __forceinline__ void add(tree_f32x16 (&O)[4], const TreeWeights<TERMS>& p, int t) const {   // 16 of the keys
#pragma unroll
    for (int term = TERMS - 1; term >= 0; --term)
#pragma unroll
      for (int ct = 0; ct < 4; ++ct)
        O[ct] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[ct][t], p.w[term][t], O[ct], 0, 0, 0);
  }
};

// The values that put() left out of a tile, for the nodes that see them.
template <class KEYS>
__device__ __forceinline__ void tree_values_left_out(tree_f32x16 (&O)[4], const KEYS& keys, const uint32_t* sm_bad,
                                                     uint32_t allow, int t0, int half) {
  for (uint32_t bad = __builtin_amdgcn_readfirstlane(sm_bad[(t0 - keys.t_mixed) / kTreeTile]); bad != 0; bad &= bad - 1) {
    const int j = __builtin_ctz(bad);
    if (!((allow >> j) & 1u)) continue;
    const uint16_t* v = keys.v_at(t0 + j) - keys.lc * 8 + 4 * half;
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const uint16_t x = v[ct * 32 + 8 * (i >> 2) + (i & 3)];
        if ((x & 0x7F80u) == 0x7F80u) O[ct][i] += bf16_to_f32(x);
      }
  }
}

__device__ __forceinline__ void tree_scale(tree_f32x16 (&O)[4], float f) {
#pragma unroll
  for (int ct = 0; ct < 4; ++ct)
#pragma unroll
    for (int i = 0; i < 16; ++i) O[ct][i] *= f;
}

// A query's running softmax: the reference of its exponents in log2 units (-inf: nothing seen) and this half's sum l - err.  A tile's
// weights are added up by themselves and join the sum with what rounding took from it carried along: added one after the other, equal
// weights are rounded alike, 1e-4 of the sum after 8192 of them.
struct TreeSoftmax {
  float m, l, err, scale_log2;
  FmaExponent exponent;
  __device__ __forceinline__ explicit TreeSoftmax(float scale) : m(-__builtin_inff()), l(0.0f), err(0.0f), scale_log2(scale), exponent(scale, 0.0f) {}
  // weights of a tile from its logits
  template <int TERMS>
  __device__ __forceinline__ void take(const tree_f32x16& z, tree_f32x16 (&O)[4], TreeWeights<TERMS>& w) {
    const float mx = tree_max(z) * scale_log2;
    // The reference only has to be near the maximum: it moves when a query's maximum grows by more than 8, so most tiles
    // rescale nothing, and the weights stay below 2^8.
    if (__any(mx - m > 8.0f)) {                          // m = -inf: true unless nothing has been seen
      const float m_new = fmaxf(m, mx);
      const float f = m == -__builtin_inff() ? 0.0f : exp2_small(m - m_new);
      l *= f;
      err *= f;
      tree_scale(O, f);
      m = m_new;
      exponent = FmaExponent(scale_log2, m == -__builtin_inff() ? 0.0f : m);
    }
    float p[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) p[i] = exp2_small(exponent.of(z[i]));
    const float tile = ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7])) +
                       (((p[8] + p[9]) + (p[10] + p[11])) + ((p[12] + p[13]) + (p[14] + p[15])));
    const float add = tile - err, sum = l + add;
    err = (sum - l) - add;
    l = sum;
    w.set(p);
  }
  // both halves' sum
  __device__ __forceinline__ void close() {
    l -= err;
    l += shfl_xor_f(l, 32);
  }
};

// The states of KW wavefronts that took other keys for the same queries, in order, into that of the first (kw = 0).
// sm_o: (KW - 1) * QW blocks of 64 values of 64 lanes.
template <int QW, int KW>
__device__ __forceinline__ void tree_join(TreeSoftmax& sm, tree_f32x16 (&O)[4], bool busy, int qw, int kw, float* sm_o, float2* sm_ml) {
  const int lane = threadIdx.x & (DSK_WAVE - 1);
  if (kw > 0 && busy) {
    const int blk = (kw - 1) * QW + qw;
    sm_ml[blk * DSK_WAVE + lane] = make_float2(sm.m, sm.l);
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
      for (int i = 0; i < 16; ++i) sm_o[(blk * 64 + ct * 16 + i) * DSK_WAVE + lane] = O[ct][i];
  }
  __syncthreads();
  if (kw > 0 || !busy) return;
  float M = sm.m;
#pragma unroll
  for (int o = 0; o < KW - 1; ++o) M = fmaxf(M, sm_ml[(o * QW + qw) * DSK_WAVE + lane].x);
  const float f = sm.m == -__builtin_inff() ? 0.0f : exp2_small(sm.m - M);
  sm.l *= f;
  tree_scale(O, f);
#pragma unroll
  for (int o = 0; o < KW - 1; ++o) {
    const int blk = o * QW + qw;
    const float2 ml = sm_ml[blk * DSK_WAVE + lane];
    const float fo = ml.x == -__builtin_inff() ? 0.0f : exp2_small(ml.x - M);
    sm.l = fmaf(ml.y, fo, sm.l);
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
      for (int i = 0; i < 16; ++i) O[ct][i] = fmaf(sm_o[(blk * 64 + ct * 16 + i) * DSK_WAVE + lane], fo, O[ct][i]);
  }
  sm.m = M;
}

// A lane's row: final, or this part's share.  Its channels lie four in a row, at 32 ct + 8 i + 4 half.
__device__ __forceinline__ void tree_store(const dsk_tree_attn_args& a, const TreeQueries& qs, const tree_f32x16 (&O)[4], float m,
                                           float l, int used, int nsplit, int split, float2* part_ml, float* part_acc) {
  if (!qs.real) return;
  if (used == 1) {
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 x = make_float4(O[ct][4 * i] * inv, O[ct][4 * i + 1] * inv, O[ct][4 * i + 2] * inv, O[ct][4 * i + 3] * inv);
        const int64_t at = qs.out_row * DSK_HEAD_DIM + ct * 32 + 8 * i + 4 * qs.half;
        if (a.out != nullptr) *reinterpret_cast<float4*>(a.out + at) = x;
        if (a.out_bf16 != nullptr)
          *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out_bf16) + at) = make_uint2(tree_pack(x.x, x.y), tree_pack(x.z, x.w));
      }
    if (qs.half == 0 && a.lse != nullptr) a.lse[qs.out_row] = l == 0.0f ? -__builtin_inff() : (m + log2f(l)) * kLn2;   // a NaN stays one
  } else {
    const int64_t part = qs.out_row * nsplit + split;
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<float4*>(part_acc + part * DSK_HEAD_DIM + ct * 32 + 8 * i + 4 * qs.half) =
            make_float4(O[ct][4 * i], O[ct][4 * i + 1], O[ct][4 * i + 2], O[ct][4 * i + 3]);
    if (qs.half == 0) part_ml[part] = make_float2(m, l);
  }
}

// TERMS: bf16 terms that a weight is split into for the second product: 3 for fp32 results, 2 for bf16 ones, 1 above 64 rows.
// KW wavefronts take other tiles of a stage for the same queries, NT of them each.  With two BUFS a stage is copied while the one
// before it is multiplied; with one (32 rows, whose products are short) that is left to the second workgroup of the CU.
// HBM bounds it: 40 / 40 heads, 128K tokens, 16 nodes (2.68 GB) 395 us, 6.8 TB/s; 32 / 8 heads, 16 nodes (0.54 GB) 88, 6.1; eight of
// 16K to 64K, 13 nodes, token-major (1.48 GB) 240 to 250, 5.9 to 6.2.  Where 4 wavefronts take 128 rows, their matrix instructions
// and exponentials, about as many cycles each, no longer hide entirely: 32 nodes, 0.54 GB at 5.0 TB/s.
template <int QW, int KW, int NT, int BUFS, int TERMS, bool SEL, bool STREAM>
__global__ __launch_bounds__(QW * KW * DSK_WAVE, 2) void tree_attn_kernel(
    dsk_tree_attn_args a, int G, int q_tiles, TreeSplit sp, float scale_log2, float2* __restrict__ part_ml,
    float* __restrict__ part_acc) {
  constexpr int kThreads = QW * KW * DSK_WAVE;
  constexpr int kTiles = KW * NT, kKeys = kTreeTile * kTiles;   // of a stage
  constexpr int kBufBytes = 2 * kTiles * kTreeTileBytes;
  __shared__ __align__(16) unsigned char sm_kv[BUFS * kBufBytes];
  __shared__ float2 sm_ml[KW > 1 ? (KW - 1) * QW * DSK_WAVE : 1];
  __shared__ uint32_t sm_bad[kTreeMixedTiles];
  static_assert(kTiles + DSK_TREE_MAX_NODES / kTreeTile + 1 <= kTreeMixedTiles, "words of sm_bad");
  __shared__ int32_t sm_rows[SEL ? kTreeMaxListed : 1];

  TreeWork work;
  if (!work.find(a, sp, q_tiles)) return;                // uniform, as all returns before the end
  const int split = work.split, s = work.s, hk = work.hk, q_tile = work.q_tile;
  const int tid = threadIdx.x, wave = tid / DSK_WAVE;
  const int qw = wave % QW, kw = wave / QW;

  const TreeSlots<SEL> slots(a, sp, s, hk, split);
  const TreePlace at(a, s);
  if (q_tile * QW * kTreeTile >= at.n * G) return;       // uniform: no row of this pass
  const int used = at.used(sp, SEL, slots.count);
  if (split >= used) return;
  TreeQueries qs(a, at, G, hk, (q_tile * QW + qw) * kTreeTile);
  const TreeKeys<kThreads, kKeys * 16 / kThreads, SEL, STREAM> keys(a, sp, at, slots, hk, split, used, sm_rows);
  qs.mask.n = keys.nodes();

  TreeSoftmax sm(scale_log2);
  tree_f32x16 O[4];
#pragma unroll
  for (int ct = 0; ct < 4; ++ct)
#pragma unroll
    for (int i = 0; i < 16; ++i) O[ct][i] = 0.0f;

  if (tid < kTreeMixedTiles) sm_bad[tid] = 0;
  auto tiles = [&](int t0, const unsigned char* sm_k, auto mixed) {   // this wavefront's tiles of the stage in LDS
    constexpr bool kMixed = decltype(mixed)::value;
    const unsigned char* const sm_v = sm_k + kTiles * kTreeTileBytes;
#pragma unroll
    for (int sub = 0; sub < NT; ++sub) {
      const int tile = kw * NT + sub, tt = t0 + tile * kTreeTile;
      if (kMixed && tt >= keys.t_end) break;
      TreeKFrag kf;
      kf.read<0, 8>(sm_k + tile * kTreeTileBytes, qs);
      tree_f32x16 z;
      kf.add<0, 8>(z, qs);
      uint32_t allow = 0;
      if constexpr (kMixed) {
        allow = qs.allowed(tt, keys.P);
        tree_hide(z, allow, qs.half);
      }
      TreeVFrag vf;
      if constexpr (BUFS > 1) {                          // during the products of K, whose results the weights wait for anyway
        __builtin_amdgcn_sched_barrier(0);
        vf.read_beside_copies(sm_v + tile * kTreeTileBytes);
        __builtin_amdgcn_sched_barrier(0);
      }
      TreeWeights<TERMS> w;
      sm.take(z, O, w);
      if constexpr (BUFS == 1) {
        vf.template read<0>(sm_v + tile * kTreeTileBytes);
        vf.template read<1>(sm_v + tile * kTreeTileBytes);
      }
      vf.add<TERMS>(O, w, 0);
      vf.add<TERMS>(O, w, 1);
      if constexpr (kMixed) tree_values_left_out(O, keys, sm_bad, allow, tt, qs.half);
    }
  };
  using Plain = std::integral_constant<bool, false>;
  using Mixed = std::integral_constant<bool, true>;
  int t0 = keys.t_begin;
  // stages of the prefix alone: nothing is masked
  auto some = [&](int t) { return keys.plain(t) && t < keys.t_end; };
  auto copy = [&](int t, unsigned char* to) { keys.copy_plain(t, to, to + kTiles * kTreeTileBytes); };
  unsigned char *here = sm_kv, *other = sm_kv + (BUFS - 1) * kBufBytes;
  if (BUFS > 1 && some(t0)) copy(t0, here);
  for (; some(t0); t0 += kKeys) {
    if (BUFS == 1) copy(t0, here);
    lds_copies_done();
    __syncthreads();                                     // the stage is here, and nobody reads the other one any more
    if (BUFS > 1 && some(t0 + kKeys)) copy(t0 + kKeys, other);
    if (qs.busy) tiles(t0, here, Plain());
    if (BUFS == 1) __syncthreads();
    unsigned char* const read = here;
    here = other;
    other = read;
  }
  if (BUFS > 1 || t0 == keys.t_begin) __syncthreads();   // (the latter: sm_bad)
  for (; t0 < keys.t_end; t0 += kKeys) {                 // its end and the nodes
    typename decltype(keys)::Regs x;
    keys.fetch_mixed(x, t0);
    keys.template put<true>(x, t0, sm_kv, sm_kv + kTiles * kTreeTileBytes, sm_bad);
    __syncthreads();
    if (qs.busy) tiles(t0, sm_kv, Mixed());
    __syncthreads();
  }
  sm.close();
  if constexpr (KW > 1) {
    static_assert((KW - 1) * QW <= BUFS * kTiles, "a block is as large as a tile of K and V");
    tree_join<QW, KW>(sm, O, qs.busy, qw, kw, reinterpret_cast<float*>(sm_kv), sm_ml);
    if (kw > 0) return;
  }
  tree_store(a, qs, O, sm.m, sm.l, used, sp.nsplit, split, part_ml, part_acc);
}

// The same for many rows, where the matrix cores bound it (bf16 results): eight wavefronts, two on a SIMD, of which one has the
// matrix cores while the other makes exponentials.  Time goes in slots with a barrier after each.  The first four wavefronts
// multiply step i in slot 2 i (V of step i - 1, then K of step i) and take its softmax in slot 2 i + 1; the other four do
// either a slot later.  A step is a tile of 32 keys, and every wavefront has 32 rows of its own.
// Steps go round four LDS buffers.  In the softmax slot of step i the first group puts its half of step i + 1 (slot 2 i + 1),
// the second its half of step i + 2 (slot 2 i + 2), so a step is whole one slot before its first use, and the step that it
// replaces was last read long before.  Loads are issued 64 KB before they are put.
// 32 / 8 heads, 64 nodes, 128K tokens: 137 GFLOP in 154 us while the chip is cool (0.89 PFLOP/s; a large library product reaches
// 1.15), 190 without pause, when the clock is lower.  As counted, a slot takes 1020 cycles of a CU, about what its 512 cycles of
// products and 490 to 600 of exponentials take one after the other (matrix cores 0.49 busy, LDS 0.30): the two groups take turns more
// than they overlap, and what holds them apart has not been found.  Taking tiles one after the other in every wavefront took 212.
constexpr int kWideWaves = 8;

template <bool STREAM>
__global__ __launch_bounds__(kWideWaves * DSK_WAVE, 2) void tree_wide_kernel(
    dsk_tree_attn_args a, int G, int q_tiles, TreeSplit sp, float scale_log2, float2* __restrict__ part_ml,
    float* __restrict__ part_acc) {
  constexpr int kThreads = kWideWaves * DSK_WAVE;
  constexpr int kKeys = kTreeTile;                       // of a step
  constexpr int kBufs = 4, kBufBytes = 2 * kTreeTileBytes;
  constexpr int kSets = 4;                               // steps on their way in registers: 64 KB
  __shared__ __align__(16) unsigned char sm_kv[kBufs * kBufBytes];
  __shared__ uint32_t sm_bad[kTreeMixedTiles];
  static_assert(1 + DSK_TREE_MAX_NODES / kTreeTile + 1 <= kTreeMixedTiles, "words of sm_bad");

  TreeWork work;
  if (!work.find(a, sp, q_tiles)) return;
  const int split = work.split, s = work.s, hk = work.hk, q_tile = work.q_tile;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / DSK_WAVE);
  const bool late = wave >= 4;

  const TreePlace at(a, s);
  if (q_tile * kWideWaves * kTreeTile >= at.n * G) return;       // uniform: no row of this pass
  const int used = at.used(sp, false, 0);
  if (split >= used) return;
  using Keys = TreeKeys<kThreads, kKeys * 16 / kThreads, false, STREAM>;
  const Keys keys(a, sp, at, TreeSlots<false>(a, sp, s, hk, split), hk, split, used, nullptr);
  TreeQueries qs(a, at, G, hk, (q_tile * kWideWaves + wave) * kTreeTile);
  qs.mask.n = keys.nodes();
  TreeSoftmax sm(scale_log2);
  tree_f32x16 O[4];
#pragma unroll
  for (int ct = 0; ct < 4; ++ct)
#pragma unroll
    for (int i = 0; i < 16; ++i) O[ct][i] = 0.0f;

  const int steps = keys.t_end > keys.t_begin ? (keys.t_end - keys.t_begin + kKeys - 1) / kKeys : 0;
  auto t_of = [&](int i) { return keys.t_begin + i * kKeys; };
  auto barrier = [] {
    __builtin_amdgcn_sched_barrier(0);
    __syncthreads();
    __builtin_amdgcn_sched_barrier(0);
  };
  // steps below `plain_steps` are of the prefix alone
  const int plain_steps = keys.P > keys.t_begin ? ((keys.P < keys.t_end ? keys.P : keys.t_end) - keys.t_begin) / kKeys : 0;
  // kPlain: what is put and fetched is known to be plain; beyond the last step it is put and fetched again, and not read.
  using Plain = std::integral_constant<bool, true>;
  using Any = std::integral_constant<bool, false>;
  auto put = [&](auto plain, typename Keys::Regs& x, int i, int buf) {
    unsigned char* to = sm_kv + buf * kBufBytes;
    if (decltype(plain)::value || i < plain_steps) keys.template put<false>(x, t_of(i), to, to + kTreeTileBytes, nullptr);
    else if (i < steps) keys.template put<true>(x, t_of(i), to, to + kTreeTileBytes, sm_bad);
  };
  auto fetch = [&](typename Keys::Regs& x, int i) {
    if (i < plain_steps) keys.fetch_plain(x, t_of(i));
    else if (i < steps) keys.fetch_mixed(x, t_of(i));
  };
  // Step i goes through set i % kSets of the first group, (i - 1) % kSets of the second, so that both put set (i + 1) % kSets
  // in their softmax slot of step i.
  typename Keys::Regs x[kSets];
  if (tid < kTreeMixedTiles) sm_bad[tid] = 0;
  // the first step multiplies weights of 0 by the values of "the step before" it: those have to be numbers
  for (int i = tid; i < kTreeTileBytes / 16; i += kThreads)
    *reinterpret_cast<uint4*>(sm_kv + (kBufs - 1) * kBufBytes + kTreeTileBytes + i * 16) = make_uint4(0, 0, 0, 0);
#pragma unroll
  for (int j = 0; j < kSets; ++j) fetch(x[j], late ? (j + 1) % kSets : j);
  __syncthreads();
  if (!late) {
    put(Any(), x[0], 0, 0);
    fetch(x[0], kSets);
  } else {
    put(Any(), x[kSets - 1], 0, 0);
    fetch(x[kSets - 1], kSets);
  }
  barrier();
  if (late) {
    put(Any(), x[0], 1, 1);
    fetch(x[0], kSets + 1);
    barrier();
  }
  const int ahead = late ? 2 : 1;
  // what the loop of plain steps fetches next, from the first step that is not fetched yet; the last one again when it is through
  int fetched = ahead + kSets < plain_steps ? ahead + kSets : (plain_steps > 0 ? plain_steps - 1 : 0);
  tree_global k_next = keys.Ku + t_of(fetched) * keys.kst * 2, v_next = keys.Vu + t_of(fetched) * keys.vst * 2;
  int64_t k_inc = kKeys * keys.kst * 2, v_inc = kKeys * keys.vst * 2;
  asm("" : "+s"(k_inc), "+s"(v_inc));                    // no more of the arguments is kept for them
  auto fetch_next = [&](typename Keys::Regs& x) {
    x.k[0] = load16_at<STREAM>(k_next, keys.k_off);
    x.v[0] = load16_at<STREAM>(v_next, keys.v_off);
    const bool more = fetched + 1 < plain_steps;
    fetched += more;
    k_next += more ? k_inc : 0;
    v_next += more ? v_inc : 0;
  };
  TreeVFrag vf;                                          // values and weights of the step before, for its product
  TreeWeights<1> w;
#pragma unroll
  for (int t = 0; t < 2; ++t) w.w[0][t] = __builtin_bit_cast(tree_bf16x8, make_uint4(0, 0, 0, 0));
#pragma unroll
  for (int ct = 0; ct < 4; ++ct) vf.v[ct][0] = w.w[0][0];
  // A wavefront without rows multiplies what is there: nothing reads its result.
  auto step = [&](auto plain, auto buffer, int i, typename Keys::Regs& regs) {
    constexpr bool kPlain = decltype(plain)::value;
    constexpr int kBuf = decltype(buffer)::value, kBefore = (kBuf + kBufs - 1) % kBufs;
    const unsigned char* from = sm_kv + kBuf * kBufBytes;
    // Fragments are read well ahead of their products; left to itself the compiler reads each one right before, and waits.
    TreeKFrag kf;
    tree_f32x16 z;
    vf.template read<1>(sm_kv + kBefore * kBufBytes + kTreeTileBytes);
    __builtin_amdgcn_sched_barrier(0);
    vf.template add<1>(O, w, 0);
    __builtin_amdgcn_sched_barrier(0);
    kf.template read<0, 4>(from, qs);
    __builtin_amdgcn_sched_barrier(0);
    vf.template add<1>(O, w, 1);
    __builtin_amdgcn_sched_barrier(0);
    kf.template read<4, 8>(from, qs);
    __builtin_amdgcn_sched_barrier(0);
    kf.template add<0, 4>(z, qs);
    kf.template add<4, 8>(z, qs);
    if (!kPlain && i > plain_steps) {
      tree_values_left_out(O, keys, sm_bad, qs.allowed(t_of(i - 1), keys.P), t_of(i - 1), qs.half);
    }
    barrier();
    put(plain, regs, i + ahead, late ? (kBuf + 2) % kBufs : (kBuf + 1) % kBufs);
    if constexpr (kPlain) fetch_next(regs);
    else fetch(regs, i + ahead + kSets);
    if (!kPlain && i >= plain_steps) tree_hide(z, qs.allowed(t_of(i), keys.P), qs.half);
    vf.template read<0>(from + kTreeTileBytes);
    __builtin_amdgcn_sched_barrier(0);
    sm.take(z, O, w);
    barrier();
  };
  // Steps of which all that they put and fetch is plain: the others only meet the end of the prefix.
  const int easy = steps == plain_steps ? steps : plain_steps - kSets - 2;
  int i = 0;
  using B0 = std::integral_constant<int, 0>;
  using B1 = std::integral_constant<int, 1>;
  using B2 = std::integral_constant<int, 2>;
  using B3 = std::integral_constant<int, 3>;
  for (; i + kBufs <= easy; i += kBufs) {
    step(Plain(), B0(), i, x[1]);
    step(Plain(), B1(), i + 1, x[2]);
    step(Plain(), B2(), i + 2, x[3]);
    step(Plain(), B3(), i + 3, x[0]);
  }
  for (; i < steps; i += kBufs) {
    step(Any(), B0(), i, x[1]);
    if (i + 1 < steps) step(Any(), B1(), i + 1, x[2]);
    if (i + 2 < steps) step(Any(), B2(), i + 2, x[3]);
    if (i + 3 < steps) step(Any(), B3(), i + 3, x[0]);
  }
  const int buf_before = (steps + kBufs - 1) % kBufs;
  vf.add<1>(O, w, 0);
  if (steps > 0) {
    vf.read<1>(sm_kv + buf_before * kBufBytes + kTreeTileBytes);
    vf.add<1>(O, w, 1);
  }
  if (steps > plain_steps) {
    tree_values_left_out(O, keys, sm_bad, qs.allowed(t_of(steps - 1), keys.P), t_of(steps - 1), qs.half);
  }
  if (!late) barrier();                                  // as many as the others
  sm.close();
  tree_store(a, qs, O, sm.m, sm.l, used, sp.nsplit, split, part_ml, part_acc);
}

// The parts of a row put together in order.  2048 rows of 32 parts (34 MB, L2 and memory-side cache) 8.4 to 11.8 us, 1024 of 16
// 4.2, the least 3.0 to 3.8: launch, lengths, maxima, partials, a round trip each.
// WAVES wavefronts a row, two channels a lane.  `used` as in the kernel above.
constexpr int kTreeMergeWaves = 4;
constexpr int kTreeMergeBatch = 8;             // partials of a wavefront on their way at once
// Parts from which on a row has all four: 64 parts of 16 rows 5.5 us less, 33 of 512 rows 1.9, 32 of 2048 none
constexpr int kTreeMergeMany = 16;

template <bool SEL, int WAVES>
__global__ __launch_bounds__(kTreeMergeWaves * DSK_WAVE) void tree_merge_kernel(
    dsk_tree_attn_args a, int G, TreeSplit sp, const float2* __restrict__ part_ml,
    const float* __restrict__ part_acc) {
  constexpr int kRows = kTreeMergeWaves / WAVES;
  const int s = blockIdx.y, lane = threadIdx.x & (DSK_WAVE - 1), wave = threadIdx.x / DSK_WAVE;
  const int item = blockIdx.x * kRows + wave / WAVES;
  const int node = item / a.Hq, h = item - node * a.Hq;
  const TreePlace at(a, s);
  if (node >= at.n) return;
  const int used = at.used(sp, SEL, SEL ? tree_sel_count(a, s, h / G) : 0);
  if (used <= 1) return;                                 // finished by the kernel above
  const int64_t row = (int64_t)(at.tok0 + node) * a.Hq + h;
  const float2* ml = part_ml + row * sp.nsplit;
  const float2* acc = reinterpret_cast<const float2*>(part_acc + row * sp.nsplit * DSK_HEAD_DIM) + lane;
  float M = -__builtin_inff(), l = 0.0f;
  for (int c = lane; c < used; c += DSK_WAVE) M = fmaxf(M, ml[c].x);
  M = wave_max(M);
  float2 o = make_float2(0.0f, 0.0f);
  for (int c0 = wave % WAVES * kTreeMergeBatch; c0 < used; c0 += WAVES * kTreeMergeBatch) {
    float2 x[kTreeMergeBatch], v[kTreeMergeBatch];
#pragma unroll
    for (int u = 0; u < kTreeMergeBatch; ++u) {
      const int c = c0 + u < used ? c0 + u : used - 1;
      v[u] = ml[c];
      x[u] = acc[(int64_t)c * (DSK_HEAD_DIM / 2)];
    }
#pragma unroll
    for (int u = 0; u < kTreeMergeBatch; ++u) {
      if (c0 + u >= used || v[u].y == 0.0f) continue;    // (not by the maximum: where every logit is NaN it is -inf)
      const float f = exp2_small(v[u].x - M);
      l = fmaf(v[u].y, f, l);
      o.x = fmaf(x[u].x, f, o.x);
      o.y = fmaf(x[u].y, f, o.y);
    }
  }
  if constexpr (WAVES > 1) {
    static_assert(kRows == 1, "all wavefronts of a workgroup have the same row, or none");
    __shared__ float sm_part[WAVES - 1][3][DSK_WAVE];
    if (wave > 0) {
      sm_part[wave - 1][0][lane] = o.x;
      sm_part[wave - 1][1][lane] = o.y;
      sm_part[wave - 1][2][lane] = l;
    }
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int w = 0; w < WAVES - 1; ++w) {
      o.x += sm_part[w][0][lane];
      o.y += sm_part[w][1][lane];
      l += sm_part[w][2][lane];
    }
  }
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;
  o.x *= inv;
  o.y *= inv;
  if (a.out != nullptr) *reinterpret_cast<float2*>(a.out + row * DSK_HEAD_DIM + 2 * lane) = o;
  if (a.out_bf16 != nullptr)
    *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out_bf16) + row * DSK_HEAD_DIM + 2 * lane) = tree_pack(o.x, o.y);
  if (lane == 0 && a.lse != nullptr) a.lse[row] = l == 0.0f ? -__builtin_inff() : (M + log2f(l)) * kLn2;
}

// K and V larger than the memory-side cache are hardly found there again by the next step, so they are read past it (one pass
// over them; several share its lines).  32 / 8 heads, 16 nodes: 128K tokens (512 MB) 116 us through it, 103 past it; 8 / 8 heads,
// 32 nodes, 32K tokens (128 MB) 40.3 and 42.8.
constexpr int64_t kTreeStreamBytes = 288ll << 20;

// ---- geometry: follows the host's bounds alone ---------------------------------------------------------------
struct TreeLaunch {
  TreeSplit sp;
  int q_waves;        // QW
  bool deep;          // tree_attn_kernel with eight wavefronts
  bool wide;          // tree_wide_kernel
  bool stream;        // K and V are read past the memory-side cache
  int q_tiles;        // passes over a (sequence, KV head)'s keys
  size_t part_acc;    // of the workspace
};

// Keys of a workgroup from which on the kernel for many rows gains (its first and last steps are slower), where the other has eight
// wavefronts a CU (one sequence) and where it has not.  32 / 8 heads: 64 nodes, 16K tokens (640 keys) 44.4 us with it and 40.6
// without, 32K (1152) 68.4 and 67.6, 128K (4224) 192 and 214; 40 nodes, 128K 170 and 176; 64 / 8 heads, 64 nodes, 32K (2176) 102.4
// and 105.9.  8 sequences of 2K, 64 nodes (768) 50.3 and 59.4, of 8K, 40 nodes 110.5 and 126; 64 nodes, 2K (256) 25.7 and 20.3.
constexpr int kTreeWideKeysOne = 2048, kTreeWideKeys = 512;
constexpr int kTreeLeastKeys = 256;            // of any: a shorter part costs more in partial results than it saves

constexpr int kTreeCus = 256;

static TreeLaunch tree_layout(const dsk_tree_attn_args& a, bool f32) {
  constexpr int stage = 128;                             // a multiple of the keys that the kernels take at once
  const int rows = a.max_nodes * (a.Hq / a.Hkv);
  const bool sel = a.sel_start != nullptr;
  const int64_t longest = (int64_t)a.max_seqlen + a.max_nodes;
  // the cache has no room for all sequences at max_seqlen: they differ in length
  const bool ragged = a.total_rows < (int64_t)a.B * a.max_seqlen;
  const int64_t keys = (ragged ? a.total_rows : (int64_t)a.B * a.max_seqlen) + (int64_t)a.B * a.max_nodes;
  TreeLaunch t;
  auto rows_of = [&](int q_waves) {
    t.q_waves = q_waves;
    t.q_tiles = (rows + q_waves * kTreeTile - 1) / (q_waves * kTreeTile);
  };
  // parts of `want` workgroups in all: keys of one
  auto keys_of = [&](int64_t want) {
    const int64_t heads = (int64_t)a.Hkv * t.q_tiles;
    // of all sequences together, the last of each a shorter one, which leaves room for one of each; or of each
    int64_t parts = ragged ? want / heads - (a.B - 1) : want / (heads * a.B);
    parts = parts > 1 ? parts : 1;
    int64_t per = ((ragged ? keys : longest) + parts - 1) / parts;
    const int64_t fewest = (longest + kTreeMaxSplit - 1) / kTreeMaxSplit;
    per = per > kTreeLeastKeys ? per : kTreeLeastKeys;
    per = per > fewest ? per : fewest;
    per = per < longest ? per : longest;                 // (of more sequences than workgroups)
    return (per + stage - 1) / stage * stage;
  };
  t.sp.keys_per_split = t.sp.slots_per_split = 0;
  t.deep = t.wide = t.stream = t.sp.packed = false;
  if (!sel) {
    if (rows > 128 && !f32) {
      rows_of(kWideWaves);
      t.sp.keys_per_split = (int)keys_of(kTreeCus);
      t.wide = t.sp.keys_per_split >= (a.B > 1 ? kTreeWideKeys : kTreeWideKeysOne);
    }
    if (!t.wide) {
      rows_of(rows <= 32 ? 1 : (rows <= 64 ? 2 : 4));
      t.sp.keys_per_split = (int)keys_of(2 * kTreeCus);  // two a CU, all there at once
      // One of eight wavefronts a CU instead, which halves the partial results, where that gives every CU a workgroup.  32 / 8 heads,
      // 16 nodes: 8K tokens 23.8 -> 21.6 us, 32K 39.5 -> 36.6, 128K 104.7 -> 99.9; fp32 32K 44.3 -> 40.8; 32 nodes: 32K 50.6 -> 44.6;
      // 4K (136 workgroups) 17.1 and 18.6; eight sequences of 32K 224 -> 177.  Sequences that are known to differ in length fill the
      // finer grain better: eight of 16K to 64K tokens, 13 nodes 246 and 269, four of up to 32K 75 and 74.
      t.deep = (a.B == 1 || !ragged) && t.q_waves > 1 && keys * a.Hkv * t.q_tiles >= (int64_t)kTreeCus * kTreeLeastKeys;
      if (t.deep) t.sp.keys_per_split = (int)keys_of(kTreeCus);
    }
    t.sp.nsplit = (int)(((int64_t)a.max_seqlen + a.max_nodes + t.sp.keys_per_split - 1) / t.sp.keys_per_split);
  } else {
    rows_of(rows <= 32 ? 1 : (rows <= 64 ? 2 : 4));
    const int64_t slots = (int64_t)a.k * a.B * a.Hkv * t.q_tiles;
    // (32 nodes, 4 heads a group, 4096 tokens: 26.2 us with at least 128 tokens, 23.6 with 256, 27.6 with 512)
    const int64_t least = (kTreeLeastKeys + a.b - 1) / a.b, most = kTreeMaxListed / a.b < kTreeMaxSlots ? kTreeMaxListed / a.b : kTreeMaxSlots;
    int64_t per = (slots + 511) / 512;
    per = per > least ? per : least;
    per = per < most ? per : most;
    t.sp.slots_per_split = (int)per;
    t.sp.nsplit = (int)((a.k + per - 1) / per);
  }
  // Where workgroups of four wavefronts' rows leave half the CUs idle or more, twice as many take two wavefronts' rows each and
  // split a stage's keys as well: K and V come from L2 once more, but every wavefront has half as much to do.  128 rows a
  // selection of 4K tokens (128 workgroups) 23.6 -> 20.9 us, of 2K 20.9 -> 18.0, a prefix of 600 tokens 16.0 -> 14.4; 4K tokens
  // (136 workgroups) would take 21.8 instead of 20.6.  (Halving two wavefronts' rows again gains nothing: 600 tokens 13.9 and
  // 14.1.)
  if (!t.wide && t.q_waves == 4 && (int64_t)a.B * a.Hkv * t.q_tiles * t.sp.nsplit <= kTreeCus / 2) rows_of(2);
  if (!sel) {
    // Workgroups go round XCDs and their shader engines by their number, whatever those have to do, and the parts that a shorter
    // sequence lacks end at once: numbered by sequence they leave some engines with two rounds of work and others with none.
    // Numbered through the parts that there are, each sequence's in turn and the heads fastest, all have the same: eight sequences
    // of 16K to 64K tokens, 13 nodes 283 -> 246 us, 32 nodes 319 -> 283, two of 32K and 64K 101 -> 85; what it costs is that a
    // workgroup looks its part up (16 sequences of 700 tokens 21.7 -> 22.3).  Several passes over the same keys stay as they are:
    // they have an XCD's L2 in common.  So do sequences of one part each, of which there may be many: each of their workgroups would
    // look at all before it (150 of 400 tokens 54.5 us by sequence and 56.8, 1024 of 500 363 and 450, 4096 of 60 0.56 and 1.82 ms).
    t.sp.packed = a.B > 1 && t.q_tiles == 1 && t.sp.nsplit > 1 && (int64_t)a.B * t.sp.nsplit <= 65535;
    t.stream = t.q_tiles == 1 && keys * a.Hkv * 2 * kTreeRowBytes >= kTreeStreamBytes;
  }
  const size_t parts = t.sp.nsplit > 1 ? (size_t)a.n_tokens * a.Hq * t.sp.nsplit : 0;
  t.part_acc = align_up(parts * sizeof(float2));
  return t;
}

// Parts of a sequence at most, under this max_seqlen and every smaller one: as in keys_of(), without its rounding.
static int64_t tree_most_parts(const dsk_tree_attn_args& a, int64_t want, int q_tiles) {
  const int64_t heads = (int64_t)a.Hkv * q_tiles;
  auto ceil_div = [](int64_t x, int64_t y) { return (x + y - 1) / y; };
  auto least = [](int64_t x, int64_t y) { return x < y ? x : y; };
  auto most = [](int64_t x, int64_t y) { return x > y ? x : y; };
  const int64_t even_seqlen = least(a.max_seqlen, a.total_rows / a.B);   // the largest that is not `ragged`
  int64_t n = least(most(want / (heads * a.B), 1), ceil_div(even_seqlen + a.max_nodes, kTreeLeastKeys));
  if (a.max_seqlen > even_seqlen) {
    const int64_t keys = a.total_rows + (int64_t)a.B * a.max_nodes, parts = most(want / heads - (a.B - 1), 1);
    n = most(n, ceil_div((int64_t)a.max_seqlen + a.max_nodes, most(ceil_div(keys, parts), kTreeLeastKeys)));
  }
  return least(n, kTreeMaxSplit);
}

// Whichever outputs the call will ask for, and no less than with a smaller max_seqlen: a workspace that is kept serves every length
// up to the one that it was made for.
size_t tree_ws_bytes(const dsk_tree_attn_args& a) {
  int64_t nsplit = 1;
  for (const bool f32 : {false, true}) {
    const TreeLaunch t = tree_layout(a, f32);
    nsplit = t.sp.nsplit > nsplit ? t.sp.nsplit : nsplit;
  }
  if (a.sel_start == nullptr) {
    const int rows = a.max_nodes * (a.Hq / a.Hkv);
    auto bound = [&](int64_t want, int q_waves) {
      const int64_t n = tree_most_parts(a, want, (rows + q_waves * kTreeTile - 1) / (q_waves * kTreeTile));
      nsplit = n > nsplit ? n : nsplit;
    };
    bound(2 * kTreeCus, rows <= 32 ? 1 : (rows <= 64 ? 2 : 4));
    if (rows > 128) bound(kTreeCus, kWideWaves);
  }
  const size_t parts = nsplit > 1 ? (size_t)a.n_tokens * a.Hq * nsplit : 0;
  const size_t total = align_up(parts * sizeof(float2)) + align_up(parts * DSK_HEAD_DIM * sizeof(float));
  return total > 256 ? total : 256;
}

static dim3 tree_grid(const dsk_tree_attn_args& a, const TreeLaunch& t) {
  const unsigned y = (unsigned)(a.Hkv * t.q_tiles);
  return t.sp.packed ? dim3(y, (unsigned)(a.B * t.sp.nsplit)) : dim3((unsigned)t.sp.nsplit, y, (unsigned)a.B);
}

// Rows of a KV head up to which a bf16 result's weights have two terms.  HBM or latency bounds those calls: 32 / 8 heads, 16 nodes: 128K
// tokens 91 us with one and 92 with two, 32K 31.6 and 32.2, 8K 18.3 and 19.3; eight of 16K to 64K, 13 nodes 201 and 204; 40 / 40 heads, 128K
// 402 and 402.  Beyond, products and their weights count: 32 nodes, 128K 113 and 136, eight of 16K to 64K 247 and 303, a selection of
// 4096 tokens 18.9 and 20.0, eight of them 45 and 52; 64 nodes, 128K 171 and 224.
constexpr int kTreeTwoTermRows = 64;

template <int QW, int KW, int NT, int BUFS, bool MAY_SELECT>
static void launch_tree(const dsk_tree_attn_args& a, const TreeLaunch& t, float scale_log2, float2* ml, float* acc, hipStream_t st) {
  const int G = a.Hq / a.Hkv;
  const dim3 grid = tree_grid(a, t), block(QW * KW * DSK_WAVE);
  auto go = [&](auto terms, auto may_stream) {
    constexpr int kTerms = decltype(terms)::value;
    constexpr bool kStream = decltype(may_stream)::value;
    if (MAY_SELECT && a.sel_start != nullptr)
      tree_attn_kernel<QW, KW, NT, BUFS, kTerms, MAY_SELECT, false>
          <<<grid, block, 0, st>>>(a, G, t.q_tiles, t.sp, scale_log2, ml, acc);
    else if (kStream && t.stream)
      tree_attn_kernel<QW, KW, NT, BUFS, kTerms, false, kStream><<<grid, block, 0, st>>>(a, G, t.q_tiles, t.sp, scale_log2, ml, acc);
    else
      tree_attn_kernel<QW, KW, NT, BUFS, kTerms, false, false><<<grid, block, 0, st>>>(a, G, t.q_tiles, t.sp, scale_log2, ml, acc);
  };
  using One = std::integral_constant<int, 1>;
  using Two = std::integral_constant<int, 2>;
  using Three = std::integral_constant<int, 3>;
  static_assert(kTreeTwoTermRows == 2 * kTreeTile, "one wavefront's rows always have two terms, four wavefronts' never");
  if (a.out != nullptr) {
    go(Three(), std::true_type());
  } else if constexpr (QW == 1) {
    go(Two(), std::true_type());
  } else if constexpr (QW == 2) {
    if (a.max_nodes * G <= kTreeTwoTermRows) go(Two(), std::true_type());
    else go(One(), std::false_type());                   // two passes and more
  } else {
    go(One(), std::true_type());
  }
}

hipError_t launch_tree_attn(const dsk_tree_attn_args& a, hipStream_t st) {
  const TreeLaunch t = tree_layout(a, a.out != nullptr);
  if ((int64_t)a.Hkv * t.q_tiles > 65535) return hipErrorInvalidValue;
  const float scale = a.scale != 0.0f ? a.scale : 0.08838834764831845f;   // 128^-1/2
  float2* ml = static_cast<float2*>(a.workspace);
  float* acc = reinterpret_cast<float*>(static_cast<unsigned char*>(a.workspace) + t.part_acc);
  const float scale_log2 = scale * kLog2e;
  const int G = a.Hq / a.Hkv;
  if (t.wide) {
    const dim3 grid = tree_grid(a, t), block(kWideWaves * DSK_WAVE);
    if (t.stream) tree_wide_kernel<true><<<grid, block, 0, st>>>(a, G, t.q_tiles, t.sp, scale_log2, ml, acc);
    else tree_wide_kernel<false><<<grid, block, 0, st>>>(a, G, t.q_tiles, t.sp, scale_log2, ml, acc);
  } else if (t.q_waves == 1) {
    launch_tree<1, 4, 1, 1, true>(a, t, scale_log2, ml, acc, st);
  } else if (t.q_waves == 2) {
    if (t.deep) launch_tree<2, 4, 1, 2, false>(a, t, scale_log2, ml, acc, st);
    else launch_tree<2, 2, 1, 2, true>(a, t, scale_log2, ml, acc, st);
  } else {
    if (t.deep) launch_tree<4, 2, 2, 2, false>(a, t, scale_log2, ml, acc, st);
    else launch_tree<4, 1, 2, 2, true>(a, t, scale_log2, ml, acc, st);
  }
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess || t.sp.nsplit <= 1) return err;
  const bool many = t.sp.nsplit >= kTreeMergeMany;
  const int rows = a.max_nodes * a.Hq, rows_per_wg = many ? 1 : kTreeMergeWaves;
  const dim3 grid((unsigned)((rows + rows_per_wg - 1) / rows_per_wg), (unsigned)a.B), block(kTreeMergeWaves * DSK_WAVE);
  if (a.sel_start != nullptr) {
    if (many) tree_merge_kernel<true, kTreeMergeWaves><<<grid, block, 0, st>>>(a, G, t.sp, ml, acc);
    else tree_merge_kernel<true, 1><<<grid, block, 0, st>>>(a, G, t.sp, ml, acc);
  } else {
    if (many) tree_merge_kernel<false, kTreeMergeWaves><<<grid, block, 0, st>>>(a, G, t.sp, ml, acc);
    else tree_merge_kernel<false, 1><<<grid, block, 0, st>>>(a, G, t.sp, ml, acc);
  }
  return hipGetLastError();
}

}  // namespace dsk
