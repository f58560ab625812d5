// Attention of a wavefront's 32 queries over tiles of 32 keys: fragments, softmax state and the join of states, shared by the
// kernels whose queries meet the same keys.
//
// Products are taken transposed: S^T = K Q^T, then O^T = V^T P^T, with 32x32x16 matrix instructions.  A lane then has one query
// (column lane % 32) and 16 of a tile's 32 keys, so the softmax needs one exchange between the two halves of the wavefront for the
// maximum, rescaling is a product by a lane's own factor, and the weights that S^T leaves in a lane are already those that the
// second product wants there: key 16 t + 8 (e / 4) + 4 (lane / 32) + e % 4 in place e of step t, if V^T is read with the same
// order of keys (two transposing LDS reads of four keys each).  No weight passes through LDS.
#pragma once

#include "dsk_attn_fold.hpp"
#include "dsk_common.hpp"

namespace dsk {

typedef __bf16 tile_bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 tile_bf16x2 __attribute__((ext_vector_type(2)));
typedef float tile_f32x16 __attribute__((ext_vector_type(16)));
typedef float tile_f32x2 __attribute__((ext_vector_type(2)));
typedef short tile_s16x4 __attribute__((ext_vector_type(4)));

constexpr int kAttnTile = 32;                   // keys and queries of a matrix tile
constexpr int kTileRowBytes = 2 * DSK_HEAD_DIM;

constexpr int kTileBytes = kAttnTile * kTileRowBytes;

__device__ __forceinline__ uint32_t tile_pack(float lo, float hi) {   // nearest-even bf16 pair
  const tile_f32x2 f = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, tile_bf16x2));
}

__device__ __forceinline__ uint32_t tile_pack_cut(float lo, float hi) {   // a bf16 pair, towards zero
  return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}

// 16 bytes at a uniform address and a lane's 32-bit offset, which is one instruction and no arithmetic; left to itself the
// compiler adds the parts the other way round, with a 64-bit product or sum per lane and load.
typedef const __attribute__((address_space(1))) char* tile_global;
template <bool STREAM>
__device__ __forceinline__ uint4 load16_at(tile_global base, uint32_t off) {
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

// A wavefront's 32 queries: a lane has query lane % 32 and of a tile's 32 keys those at 8 (i / 4) + 4 (lane / 32) + i % 4.
struct TileQueries {
  int col, half;
  tile_bf16x8 q[8];     // channels 16 t + 8 half .. + 7
};

// Fragments of a tile of 32 keys.
struct TileKFrag {
  tile_bf16x8 k[8];
  template <int FROM, int TO>
  __device__ __forceinline__ void read(const unsigned char* sm_k, const TileQueries& qs) {
    const unsigned char* at = sm_k + qs.col * kTileRowBytes;
#pragma unroll
    for (int t = FROM; t < TO; ++t)
      k[t] = *reinterpret_cast<const tile_bf16x8*>(at + (((2 * t + qs.half) ^ (qs.col & 15)) << 4));
  }
  // logits: S^T = K Q^T
  template <int FROM, int TO>
  __device__ __forceinline__ void add(tile_f32x16& z, const TileQueries& qs) const {
    if constexpr (FROM == 0) {
#pragma unroll
      for (int i = 0; i < 16; ++i) z[i] = 0.0f;
    }
#pragma unroll
    for (int t = FROM; t < TO; ++t) z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[t], qs.q[t], z, 0, 0, 0);
  }
};

__device__ __forceinline__ void tile_hide(tile_f32x16& z, uint32_t allow, int half) {
#pragma unroll
  for (int i = 0; i < 16; ++i)
    z[i] = (allow >> (8 * (i >> 2) + 4 * half + (i & 3))) & 1u ? z[i] : -__builtin_inff();
}

// the larger of a value and the other half's
__device__ __forceinline__ float tile_half_max(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ float tile_max(const tile_f32x16& z) {
  float m = z[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) m = fmaxf(m, z[i]);
  return tile_half_max(m);
}

// The weights of a tile, in TERMS bf16 terms.  A single term, or the last of two, is rounded to nearest.  The others are cut towards
// zero, 8 bits each, and what is left is made a little more each time, so that no term of a weight above 2^-80 is 0 or negative: an
// infinite value then stays infinite in the sum over them, where 0 * inf and inf - inf would make it NaN.  Two terms are off by 2^-16
// of the weight at most; three add up to 1.1 * 2^-24 .. 3 * 2^-24 more than it (2^-23 in the mean; taking what is left exactly and
// bounding the terms from below made fp32 calls 3 to 5 % slower).
template <int TERMS>
struct TileWeights {
  tile_bf16x8 w[TERMS][2];
  __device__ __forceinline__ void set(float (&p)[16]) {
#pragma unroll
    for (int term = 0; term < TERMS; ++term) {
      uint32_t x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (TERMS == 1) {
          x[i] = tile_pack(p[2 * i], p[2 * i + 1]);
        } else {
          x[i] = TERMS == 2 && term == 1 ? tile_pack(p[2 * i], p[2 * i + 1]) : tile_pack_cut(p[2 * i], p[2 * i + 1]);
          if (term + 1 < TERMS) {                        // what the terms so far leave
            const float more = term == 0 ? 1.0f + 0x1p-23f : 1.0f + 0x1p-17f;
            p[2 * i] = fmaf(p[2 * i], more, -bf16_lo(x[i]));
            p[2 * i + 1] = fmaf(p[2 * i + 1], more, -bf16_hi(x[i]));
          }
        }
      }
      w[term][0] = __builtin_bit_cast(tile_bf16x8, make_uint4(x[0], x[1], x[2], x[3]));
      w[term][1] = __builtin_bit_cast(tile_bf16x8, make_uint4(x[4], x[5], x[6], x[7]));
    }
  }
};

struct TileVFrag {
  tile_bf16x8 v[4][2];
  // a lane's place in a tile for channels 32 ct .. 32 ct + 31
  static __device__ __forceinline__ int place(int ct) {
    const int lane = threadIdx.x & (DSK_WAVE - 1), half = lane >> 5;
    const int quad = (lane & 15) >> 2;                   // of the four keys of a transposing read
    return (4 * half + quad) * kTileRowBytes + ((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) << 4) + ((lane & 1) << 3) + ((ct ^ quad) << 6);
  }
  template <int T>                                       // 16 of the keys
  __device__ __forceinline__ void read(const unsigned char* sm_v) {
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) {
      const unsigned char* at = sm_v + place(ct) + T * 16 * kTileRowBytes;
      const tile_s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) tile_s16x4*)(at));
      const tile_s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (__attribute__((address_space(3))) tile_s16x4*)(at + 8 * kTileRowBytes));
      v[ct][T] = __builtin_bit_cast(tile_bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  }
  // All 32 keys while copies to other parts of LDS are under way: for the builtin the compiler would wait for those first, as it
  // does not see that they are other parts.
  __device__ __forceinline__ void read_beside_copies(const unsigned char* sm_v) {
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    const uint32_t at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const unsigned char*)sm_v;
    u32x2 x[4][4];
    static_assert(kTileRowBytes == 256, "offsets: 8 rows");
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
        v[ct][t] = __builtin_bit_cast(tile_bf16x8, make_uint4(x[ct][2 * t].x, x[ct][2 * t].y, x[ct][2 * t + 1].x, x[ct][2 * t + 1].y));
  }
  // O^T += V^T P^T
  template <int TERMS>
  __device__ __forceinline__ void add(tile_f32x16 (&O)[4], const TileWeights<TERMS>& p, int t) const {   // 16 of the keys
#pragma unroll
    for (int term = TERMS - 1; term >= 0; --term)
#pragma unroll
      for (int ct = 0; ct < 4; ++ct)
        O[ct] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[ct][t], p.w[term][t], O[ct], 0, 0, 0);
  }
};

__device__ __forceinline__ void tile_scale(tile_f32x16 (&O)[4], float f) {
#pragma unroll
  for (int ct = 0; ct < 4; ++ct)
#pragma unroll
    for (int i = 0; i < 16; ++i) O[ct][i] *= f;
}

struct TileNoChange {
  __device__ __forceinline__ void operator()(float (&)[16]) const {}
};

// A query's running softmax: the reference of its exponents in log2 units (-inf: nothing seen) and this half's sum l - err.  A tile's
// weights are added up by themselves and join the sum with what rounding took from it carried along: added one after the other, equal
// weights are rounded alike, 1e-4 of the sum after 8192 of them.
struct TileSoftmax {
  float m, l, err, scale_log2;
  FmaExponent exponent;
  __device__ __forceinline__ explicit TileSoftmax(float scale) : m(-__builtin_inff()), l(0.0f), err(0.0f), scale_log2(scale), exponent(scale, 0.0f) {}
  // Weights of a tile from its logits.  APART: a query's reference moves by its own logits alone, so that no bit of its result depends
  // on the wavefront's other queries.  change: what else happens to the weights, once their sum is made.
  template <int TERMS, bool APART = false, class CHANGE = TileNoChange>
  __device__ __forceinline__ void take(const tile_f32x16& z, tile_f32x16 (&O)[4], TileWeights<TERMS>& w, const CHANGE& change = CHANGE()) {
    const float mx = tile_max(z) * scale_log2;
    // The reference only has to be near the maximum: it moves when a query's maximum grows by more than 8, so most tiles
    // rescale nothing, and the weights stay below 2^8.
    if (__any(mx - m > 8.0f)) {                          // m = -inf: true unless nothing has been seen
      const float m_new = !APART || mx - m > 8.0f ? fmaxf(m, mx) : m;
      const float f = m == -__builtin_inff() ? 0.0f : exp2_small(m - m_new);
      l *= f;
      err *= f;
      tile_scale(O, f);
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
    change(p);
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
__device__ __forceinline__ void tile_join(TileSoftmax& sm, tile_f32x16 (&O)[4], bool busy, int qw, int kw, float* sm_o, float2* sm_ml) {
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
  tile_scale(O, f);
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

}  // namespace dsk
