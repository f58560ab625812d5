// What the kernels have in common that attend to positions of a sequence or to listed rows of a cache in bf16 or 8 bits: the cache,
// fragments of codes, a wavefront's stream of key tiles, results and their parts.
#pragma once

#include "dsk_attn_tile.hpp"
#include "dsk_common.hpp"
#include "dsk_internal.hpp"

#include <type_traits>

namespace dsk {

constexpr int kWinMaxSplit = 128;              // parts of a sequence at most
constexpr int kWinLeastTiles = 4;              // of a part, a tile a wavefront (a head of 4096 tokens: 10.0 us; with 8 tiles 11.2)
constexpr int kWinLeastKeys = 8 * kAttnTile;   // of a part of selected slots (4096 tokens in each of 32 lists: 12.6 us; with half 13.8)
constexpr int kWinMaxSlots = 256;              // selected slots of a workgroup
constexpr int kWinMaxListed = 2048;            // and their tokens
constexpr int kWinTwoTermRows = 64;            // rows of a KV head up to which a bf16 result's weights have two terms
constexpr int kWinCus = 256;

// The cache with strides in bytes.
struct WinCache {
  const unsigned char *K, *V;
  int64_t k_tok, k_head, v_tok, v_head;
  const uint8_t *ks, *vs;
  int64_t s_head;
  int s_shift;                                 // log2 of the rows of a scale
};

struct WinOut {
  float* out;
  uint16_t* out_bf16;
  float* lse;
  float2* part_ml;
  float* part_acc;
};

// ---- fragments of codes ------------------------------------------------------------------------
// A row is eight chunks of 16 bytes; the two rows of 256 bytes of LDS, and the rows of a quarter wavefront's read, fall on different
// banks with chunk x of row r in place x ^ f(r).
__device__ __forceinline__ int win_swizzle8(int r) { return (r & 2) | ((r >> 1) & 4) | ((r >> 2) & 1); }

__device__ __forceinline__ uint32_t win_widen(uint32_t codes, float scale, bool upper) {
  return upper ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true))
               : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false));
}
__device__ __forceinline__ tile_bf16x8 win_widen8(uint32_t lo, uint32_t hi, float scale) {
  return __builtin_bit_cast(tile_bf16x8, make_uint4(win_widen(lo, scale, false), win_widen(lo, scale, true), win_widen(hi, scale, false),
                                                    win_widen(hi, scale, true)));
}

// 16 bytes of each lane from a uniform address and the lane's 32-bit offset to LDS, with no arithmetic (the asm keeps the compiler from
// making 64-bit addresses ahead, for which there are no registers)
template <bool STREAM>
__device__ __forceinline__ void lds_copy16_at(tile_global base, uint32_t off, unsigned char* to) {
  asm("" : "+s"(base), "+v"(off));
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(base + off), (__attribute__((address_space(3))) void*)to, 16,
                                   0, STREAM ? 2 : 0);
}
// a byte of each lane, four bytes apart in LDS and zeros between
__device__ __forceinline__ void lds_copy1(const uint8_t* from, unsigned char* to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)to, 1, 0, 0);
}

// Places of channels: with codes a lane reads 16 channels at once, those of two steps.
template <bool E4M3>
__device__ __forceinline__ int win_q_channel(int t, int half) {
  return E4M3 ? 32 * (t >> 1) + 16 * half + 8 * (t & 1) : 16 * t + 8 * half;
}

template <bool E4M3>
struct WinKFrag : TileKFrag {
  __device__ __forceinline__ void load(const unsigned char* sm_k, const TileQueries& qs, float scale) {
    if constexpr (!E4M3) {
      this->template read<0, 8>(sm_k, qs);
    } else {
      const unsigned char* at = sm_k + qs.col * DSK_HEAD_DIM;
      const int f = win_swizzle8(qs.col);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const uint4 x = *reinterpret_cast<const uint4*>(at + (((2 * u + qs.half) ^ f) << 4));
        k[2 * u] = win_widen8(x.x, x.y, scale);
        k[2 * u + 1] = win_widen8(x.z, x.w, scale);
      }
    }
  }
};

// A tile's values; load() reads all 32 keys while copies to other parts of LDS may be under way.
template <bool E4M3>
struct WinVFrag : TileVFrag {
  __device__ __forceinline__ void load(const unsigned char* sm_v) { read_beside_copies(sm_v); }
  // 0 for what is not finite; whether there was anything
  __device__ __forceinline__ bool keep_finite() {
    uint32_t found = 0;
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const uint4 x = __builtin_bit_cast(uint4, v[ct][t]);
        const uint4 y = make_uint4(finite_bf16(x.x), finite_bf16(x.y), finite_bf16(x.z), finite_bf16(x.w));
        found |= (x.x ^ y.x) | (x.y ^ y.y) | (x.z ^ y.z) | (x.w ^ y.w);
        v[ct][t] = __builtin_bit_cast(tile_bf16x8, y);
      }
    return __any(found != 0);
  }
  // O^T += V^T P^T
  template <int TERMS>
  __device__ __forceinline__ void multiply(tile_f32x16 (&O)[4], const TileWeights<TERMS>& p, float) const {
    this->template add<TERMS>(O, p, 0);
    this->template add<TERMS>(O, p, 1);
  }
};

template <>
struct WinVFrag<true> {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  u32x2 x[4][2];                                         // codes, widened when they are multiplied
  __device__ __forceinline__ void load(const unsigned char* sm_v) {
    const int lane = threadIdx.x & (DSK_WAVE - 1), half = lane >> 5, group = (lane >> 4) & 1, e = (lane & 15) >> 1;
    const int r = 4 * half + (e & 3) + 2 * (e & 4);      // the lane's key of a transposing read, of 16
    const int f = win_swizzle8(r) ^ group;               // (the same for row r + 16)
    const uint32_t at = ((uint32_t)(uintptr_t)(__attribute__((address_space(3))) const unsigned char*)sm_v + r * DSK_HEAD_DIM + ((lane & 1) << 3)) ^ (f << 4);
    static_assert(16 * DSK_HEAD_DIM == 2048, "offset: 16 rows");
    asm volatile(
        "ds_read_b64_tr_b8 %0, %8\n\tds_read_b64_tr_b8 %1, %8 offset:2048\n\t"
        "ds_read_b64_tr_b8 %2, %9\n\tds_read_b64_tr_b8 %3, %9 offset:2048\n\t"
        "ds_read_b64_tr_b8 %4, %10\n\tds_read_b64_tr_b8 %5, %10 offset:2048\n\t"
        "ds_read_b64_tr_b8 %6, %11\n\tds_read_b64_tr_b8 %7, %11 offset:2048\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[1][0]), "=&v"(x[1][1]), "=&v"(x[2][0]), "=&v"(x[2][1]), "=&v"(x[3][0]), "=&v"(x[3][1])
        : "v"(at), "v"(at ^ 32u), "v"(at ^ 64u), "v"(at ^ 96u)
        : "memory");
  }
  // 0 for the codes from `least` on, whatever their sign; whether there were any
  __device__ __forceinline__ bool keep_below(uint32_t least) {
    const uint32_t add = (0x80u - least) * 0x01010101u;  // sets the top bit of such a code, and passes nothing on to the next one
    uint32_t found = 0;
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t out = ((x[ct][t][i] & 0x7F7F7F7Fu) + add) & 0x80808080u;
          found |= out;
          x[ct][t][i] &= ~((out << 1) - (out >> 7));
        }
    return __any(found != 0);
  }
  __device__ __forceinline__ bool keep_finite() { return keep_below(0x7F); }
  template <int TERMS>
  __device__ __forceinline__ void multiply(tile_f32x16 (&O)[4], const TileWeights<TERMS>& p, float scale) const {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int ct = 0; ct < 4; ++ct) {
        const tile_bf16x8 v = win_widen8(x[ct][t].x, x[ct][t].y, scale);
#pragma unroll
        for (int term = TERMS - 1; term >= 0; --term) O[ct] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p.w[term][t], O[ct], 0, 0, 0);
      }
  }
};

// ---- rows and keys -------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t win_below(int64_t n) {   // bits 0 .. n - 1 of 32
  return n >= 32 ? 0xFFFFFFFFu : (n > 0 ? (1u << (int)n) - 1u : 0u);
}

struct WinRows : TileQueries {
  bool busy, real;      // the wavefront has rows; the lane's row exists
  int pos;
  int64_t out_row;
  template <bool E4M3>
  __device__ __forceinline__ void load(const uint16_t* q) {
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      uint4 x = make_uint4(0, 0, 0, 0);
      if (real) x = *reinterpret_cast<const uint4*>(q + out_row * DSK_HEAD_DIM + win_q_channel<E4M3>(t, half));
      this->q[t] = __builtin_bit_cast(tile_bf16x8, x);
    }
  }
};

// The values that were left out of a tile, for the rows that see them: of key j, four channels at a time.  Of codes: what has no finite
// value in bf16, and all under a scale that is no number.
template <bool E4M3, class KEYS>
__device__ __forceinline__ void win_add_left_out(tile_f32x16 (&O)[4], const WinCache& c, const KEYS& keys, int hk, int v, uint32_t allow, int half) {
  for (int j = 0; j < kAttnTile; ++j) {
    if (!((allow >> j) & 1u)) continue;
    const int64_t row = keys.row0 + keys.row_of(v, j);
    const unsigned char* at = c.V + hk * c.v_head + row * c.v_tok + half * (E4M3 ? 4 : 8);
    float scale = 1.0f;
    if constexpr (E4M3) {
      const uint32_t b = c.vs[hk * c.s_head + (row >> c.s_shift)];
      scale = b == 255 ? __builtin_nanf("") : __uint_as_float(b << 23);
    }
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (E4M3) {
          const uint32_t x = *reinterpret_cast<const uint32_t*>(at + ct * 32 + 8 * i);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float y = __builtin_amdgcn_cvt_f32_fp8((int)(x >> (8 * e)), 0) * scale;
            if (!(fabsf(y) < 0x1.ffp127f)) O[ct][4 * i + e] += y;
          }
        } else {
          const uint2 x = *reinterpret_cast<const uint2*>(at + 2 * (ct * 32 + 8 * i));
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t y = (e < 2 ? x.x : x.y) >> (16 * (e & 1)) & 0xFFFFu;
            if ((y & 0x7F80u) == 0x7F80u) O[ct][4 * i + e] += bf16_to_f32((uint16_t)y);
          }
        }
        __builtin_amdgcn_sched_barrier(0);               // few registers, not speed
      }
  }
}

// ---- a wavefront's stream of tiles -----------------------------------------------------------------------------
// Where a workgroup's rows fit one wavefront (32), its wavefronts take other tiles each and share nothing until the end: a wavefront
// copies the tile that it will multiply into LDS of its own, a ring of two tiles, and waits for its own copies alone.  The next tile
// and, once the fragments of this one are in registers, the one after it are on their way while it is multiplied: 64 KB a workgroup
// in 8 bits, of which two fit a CU, 128 KB in bf16.
constexpr int kStreamWaves = 4;
constexpr int kStreamRing = 2;

template <bool E4M3>
struct WinStreamLds {
  static constexpr int kRowBytes = E4M3 ? DSK_HEAD_DIM : 2 * DSK_HEAD_DIM;
  static constexpr int kTile = kAttnTile * kRowBytes;
  static constexpr int kSlot = 2 * kTile;
  __align__(256) unsigned char ring[kStreamWaves][kStreamRing][kSlot];
  __align__(16) uint32_t scale[E4M3 ? kStreamWaves : 1][kStreamRing][2][kAttnTile];   // of a tile's keys and values
  float2 ml[kStreamWaves][DSK_WAVE];
  static_assert(kStreamRing * kSlot >= 64 * DSK_WAVE * 4, "a wavefront's state is left in its ring's place");
};

__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}

template <int N>
__device__ __forceinline__ void win_copies_but(bool last) {   // this wavefront's copies are here but for the N last ones, or all
  if (last) __builtin_amdgcn_s_waitcnt(0x0F70);
  else __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14));
}

template <int TERMS, bool E4M3, bool STREAM, class KEYS>
__device__ __forceinline__ void win_stream(WinStreamLds<E4M3>& sh, const WinCache& c, const KEYS& keys, int hk, const WinRows& rows,
                                           TileSoftmax& sm, tile_f32x16 (&O)[4]) {
  using Lds = WinStreamLds<E4M3>;
  constexpr int kChunks = Lds::kRowBytes / 16, kRows = DSK_WAVE / kChunks, kCopies = kAttnTile / kRows;   // of a copy: 64 chunks
  constexpr int kPlaces = E4M3 ? 2 : 4;                  // swizzles of K that a lane meets
  constexpr int kOps = 2 * kCopies + (E4M3 ? 1 : 0);
  const int lane = threadIdx.x & (DSK_WAVE - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / DSK_WAVE);
  const int left = keys.end - keys.begin - wave, count = left > 0 ? (left + kStreamWaves - 1) / kStreamWaves : 0;
  const unsigned char *K = c.K + hk * c.k_head, *V = c.V + hk * c.v_head;
  const uint8_t* scales = nullptr;
  if constexpr (E4M3) scales = (lane < kAttnTile ? c.ks : c.vs) + hk * c.s_head;
  // a lane's chunk of a copy, whose order is that of the lanes: the swizzle is in what a lane reads
  const int first = lane / kChunks, place = lane % kChunks;
  uint32_t k_off[kPlaces], v_off[kPlaces];
#pragma unroll
  for (int x = 0; x < kPlaces; ++x) {
    const int r = first + x * kRows;
    const int kc = E4M3 ? place ^ win_swizzle8(r) : place ^ r, vc = E4M3 ? kc : place ^ ((r & 3) << 2);
    k_off[x] = (uint32_t)(first * (int)c.k_tok + kc * 16);   // 8 rows of 2^25 bytes at most
    v_off[x] = (uint32_t)(first * (int)c.v_tok + vc * 16);
  }
  auto issue = [&](int j) {
    const int v = keys.begin + wave + j * kStreamWaves;
    unsigned char* to = sh.ring[wave][j % kStreamRing];
    if constexpr (KEYS::kRun) {                          // rows one after the other: uniform addresses and a lane's offset
      const int64_t start = keys.start(v);
      const int last = keys.last(v);                       // of the tile's rows, those behind it are this one again
      tile_global kb = (tile_global)(K + start * c.k_tok), vb = (tile_global)(V + start * c.v_tok);
      if (last == kAttnTile - 1) {
#pragma unroll
        for (int u = 0; u < kCopies; ++u) {
          lds_copy16_at<STREAM>(kb, k_off[u % kPlaces], to + u * 1024);
          lds_copy16_at<STREAM>(vb, v_off[u % kPlaces], to + Lds::kTile + u * 1024);
          kb += kRows * c.k_tok;
          vb += kRows * c.v_tok;
        }
      } else {
#pragma unroll
        for (int u = 0; u < kCopies; ++u) {
          const int r = first + u * kRows, back = (r < last ? r : last) - first;
          lds_copy16_at<STREAM>(kb, k_off[u % kPlaces] + back * (int)c.k_tok, to + u * 1024);
          lds_copy16_at<STREAM>(vb, v_off[u % kPlaces] + back * (int)c.v_tok, to + Lds::kTile + u * 1024);
        }
      }
      const int r_scale = lane % kAttnTile < last ? lane % kAttnTile : last;
      if constexpr (E4M3) lds_copy1(scales + ((start + r_scale) >> c.s_shift), reinterpret_cast<unsigned char*>(sh.scale[wave][j % kStreamRing]));
    } else {
#pragma unroll
      for (int u = 0; u < kCopies; ++u) {
        const int64_t row = keys.row_of(v, first + u * kRows) - first;
        uint32_t ko = k_off[u % kPlaces], vo = v_off[u % kPlaces];
        asm("" : "+v"(ko), "+v"(vo));
        lds_copy16<STREAM>(K + row * c.k_tok + ko, to + u * 1024);
        lds_copy16<STREAM>(V + row * c.v_tok + vo, to + Lds::kTile + u * 1024);
      }
      if constexpr (E4M3)
        lds_copy1(scales + (keys.row_of(v, lane % kAttnTile) >> c.s_shift), reinterpret_cast<unsigned char*>(sh.scale[wave][j % kStreamRing]));
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  // places of the fragments in a slot; the chunk of step t, or of channels 32 t on, is a xor away
  const int f = E4M3 ? win_swizzle8(rows.col) : rows.col & 15;
  const uint32_t k_at = rows.col * Lds::kRowBytes + ((rows.half ^ f) << 4);
  if (count > 0) issue(0);
  if (count > 1) issue(1);
  for (int j = 0; j < count; ++j) {
    const int v = keys.begin + wave + j * kStreamWaves;
    const unsigned char* const slot = sh.ring[wave][j % kStreamRing];
    const uint32_t scales_at = lds_address(sh.scale[E4M3 ? wave : 0][j % kStreamRing]);
    win_copies_but<kOps>(j + 1 >= count);
    __builtin_amdgcn_sched_barrier(0);
    // Fragments are read by hand: for plain reads the compiler would wait for all copies first, as it does not see that those under
    // way go elsewhere.
    TileKFrag kf;
    u32x4_t x[8];
    uint32_t ks = 0, vs = 0;
    const uint32_t at = lds_address(slot) + k_at;
    if constexpr (E4M3) {
      const uint32_t scale_at = scales_at + rows.col * 4;
      asm volatile(
          "ds_read_b128 %0, %6\n\tds_read_b128 %1, %7\n\tds_read_b128 %2, %8\n\tds_read_b128 %3, %9\n\t"
          "ds_read_b32 %4, %10\n\tds_read_b32 %5, %10 offset:128\n\t"
          "s_waitcnt lgkmcnt(0)"
          : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(ks), "=&v"(vs)
          : "v"(at), "v"(at ^ 32u), "v"(at ^ 64u), "v"(at ^ 96u), "v"(scale_at)
          : "memory");
      const float scale = __uint_as_float(ks << 23);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        kf.k[2 * u] = win_widen8(x[u].x, x[u].y, scale);
        kf.k[2 * u + 1] = win_widen8(x[u].z, x[u].w, scale);
      }
    } else {
      asm volatile(
          "ds_read_b128 %0, %8\n\tds_read_b128 %1, %9\n\tds_read_b128 %2, %10\n\tds_read_b128 %3, %11\n\t"
          "ds_read_b128 %4, %12\n\tds_read_b128 %5, %13\n\tds_read_b128 %6, %14\n\tds_read_b128 %7, %15\n\t"
          "s_waitcnt lgkmcnt(0)"
          : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]), "=&v"(x[7])
          : "v"(at), "v"(at ^ 32u), "v"(at ^ 64u), "v"(at ^ 96u), "v"(at ^ 128u), "v"(at ^ 160u), "v"(at ^ 192u), "v"(at ^ 224u)
          : "memory");
#pragma unroll
      for (int t = 0; t < 8; ++t) kf.k[t] = __builtin_bit_cast(tile_bf16x8, x[t]);
    }
    tile_f32x16 z;
    kf.template add<0, 8>(z, rows);
    __builtin_amdgcn_sched_barrier(0);
    WinVFrag<E4M3> vf;
    vf.load(slot + Lds::kTile);
    __builtin_amdgcn_sched_barrier(0);
    if (j + kStreamRing < count) issue(j + kStreamRing);   // this tile's place is free
    const bool plain = keys.plain(v);
    uint32_t allow = 0;
    bool left_out = false;
    if (!plain) {
      allow = rows.real ? keys.allowed(v, rows.pos) : 0u;
      tile_hide(z, allow >> (4 * rows.half), 0);
      left_out = vf.keep_finite();                       // a masked row may hold anything, and 0 * NaN is NaN
      if constexpr (E4M3) {                              // and so may its scale
        left_out |= __any(vs == 255);
        vs = vs == 255 ? 0 : vs;
      }
    }
    // values are widened with their scale where the tile has one for all; otherwise it goes into the weights
    float v_scale = 1.0f;
    bool one = true;
    if constexpr (E4M3) {
      const uint32_t v0 = __builtin_amdgcn_readfirstlane(vs);
      one = __all(vs == v0);
      if (one) v_scale = __uint_as_float(v0 << 23);
      // a masked row may also hold codes whose value is beyond bf16: from 2^(128 - e) on under the scale 2^e, e >= 120
      if (!plain && one && v0 >= 247) left_out |= vf.keep_below(0x78u - 8 * (v0 - 247));
    }
    TileWeights<TERMS> w;
    sm.template take<TERMS, true>(z, O, w, [&](float (&p)[16]) {
      if (one) return;
      int lane4 = 16 * rows.half;                        // (the asm: sixteen sums are not kept from tile to tile)
      asm("" : "+v"(lane4));
#pragma unroll
      for (int i = 0; i < 16; ++i)
        p[i] *= __uint_as_float((uint32_t)__builtin_amdgcn_ds_bpermute(lane4 + 32 * (i >> 2) + 4 * (i & 3), (int)vs) << 23);
    });
    vf.template multiply<TERMS>(O, w, v_scale);
    if (left_out) win_add_left_out<E4M3>(O, c, keys, hk, v, allow, rows.half);
  }
  __syncthreads();                                       // the ring is free for what follows
}

__device__ __forceinline__ void win_clear(tile_f32x16 (&O)[4]) {
#pragma unroll
  for (int ct = 0; ct < 4; ++ct)
#pragma unroll
    for (int i = 0; i < 16; ++i) O[ct][i] = 0.0f;
}

// A lane's row, channels 32 ct on: final, or part `part` of `parts`.  They lie four in a row, at 32 ct + 8 i + 4 half.
__device__ __forceinline__ void win_store(const WinOut& to, const WinRows& rows, const tile_f32x16& O, int ct, float m, float l, bool last,
                                          int part, int parts) {
  if (!rows.real) return;
  if (last) {
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 x = make_float4(O[4 * i] * inv, O[4 * i + 1] * inv, O[4 * i + 2] * inv, O[4 * i + 3] * inv);
      const int64_t at = rows.out_row * DSK_HEAD_DIM + ct * 32 + 8 * i + 4 * rows.half;
      if (to.out != nullptr) *reinterpret_cast<float4*>(to.out + at) = x;
      if (to.out_bf16 != nullptr) *reinterpret_cast<uint2*>(to.out_bf16 + at) = make_uint2(tile_pack(x.x, x.y), tile_pack(x.z, x.w));
    }
    if (ct == 0 && rows.half == 0 && to.lse != nullptr) to.lse[rows.out_row] = l == 0.0f ? -__builtin_inff() : (m + log2f(l)) * kLn2;   // a NaN stays one
  } else {
    const int64_t p = rows.out_row * parts + part;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<float4*>(to.part_acc + p * DSK_HEAD_DIM + ct * 32 + 8 * i + 4 * rows.half) =
          make_float4(O[4 * i], O[4 * i + 1], O[4 * i + 2], O[4 * i + 3]);
    if (ct == 0 && rows.half == 0) to.part_ml[p] = make_float2(m, l);
  }
}

// ---- long runs in 32 bits --------------------------------------------------------------------------------------
// Equal terms that are added up one after the other are rounded alike: 4.8e-5 of a sum over V after 2048 steps of 16 keys, 9.2e-5 after
// 4096, where a result in 32 bits has room for 1e-5.  For such results a run is taken in segments, whose sums join those of the segments
// before in memory, in the place of the result or of the part's, each lane its own: 4.5e-6 with 64 tiles a wavefront (128 steps), 1.05e-5
// with 128, and up to 2^-25 for each segment.  Prompts of 8K and 32K tokens take 3 and 5 % longer, one token a sequence 0 to 2 %.
constexpr int kWinSegment = 64;                // tiles of a wavefront

struct WinKept {
  bool any = false;     // there is a sum in memory,
  float m;              // and the reference of its weights
  // O, whose reference is m_now, and what is there
  __device__ __forceinline__ void join(const float* at, tile_f32x16& O, int ct, float m_now) const {
    const float f = m == -__builtin_inff() ? 0.0f : exp2_small(m - m_now);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 x = *reinterpret_cast<const float4*>(at + ct * 32 + 8 * i);
      O[4 * i] = fmaf(x.x, f, O[4 * i]);
      O[4 * i + 1] = fmaf(x.y, f, O[4 * i + 1]);
      O[4 * i + 2] = fmaf(x.z, f, O[4 * i + 2]);
      O[4 * i + 3] = fmaf(x.w, f, O[4 * i + 3]);
    }
  }
  static __device__ __forceinline__ void put(float* at, const tile_f32x16& O, int ct) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<float4*>(at + ct * 32 + 8 * i) = make_float4(O[4 * i], O[4 * i + 1], O[4 * i + 2], O[4 * i + 3]);
  }
  // a lane's channels of its row, or of its part
  static __device__ __forceinline__ float* place(const WinOut& to, const WinRows& rows, bool last, int part, int parts) {
    return (last ? to.out + rows.out_row * DSK_HEAD_DIM : to.part_acc + (rows.out_row * parts + part) * DSK_HEAD_DIM) + 4 * rows.half;
  }
};

// The states of a stream's wavefronts, in order: each of them puts 32 channels together.  more: of a segment that is not the last one.
template <bool E4M3>
__device__ __forceinline__ void win_stream_store(WinStreamLds<E4M3>& sh, const WinOut& to, const WinRows& rows, const TileSoftmax& sm,
                                                 const tile_f32x16 (&O)[4], bool last, int part, int parts, WinKept& kept, bool more) {
  const int lane = threadIdx.x & (DSK_WAVE - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / DSK_WAVE);
  auto at = [&](int w, int ct, int i) { return reinterpret_cast<float*>(sh.ring[w]) + (ct * 16 + i) * DSK_WAVE + lane; };
  sh.ml[wave][lane] = make_float2(sm.m, sm.l);
#pragma unroll
  for (int ct = 0; ct < 4; ++ct)
#pragma unroll
    for (int i = 0; i < 16; ++i) *at(wave, ct, i) = O[ct][i];
  __syncthreads();
  float2 ml[kStreamWaves];
  float M = -__builtin_inff(), l = 0.0f;
#pragma unroll
  for (int w = 0; w < kStreamWaves; ++w) {
    ml[w] = sh.ml[w][lane];
    M = fmaxf(M, ml[w].x);
  }
  tile_f32x16 o;
#pragma unroll
  for (int w = 0; w < kStreamWaves; ++w) {
    const float f = ml[w].x == -__builtin_inff() ? 0.0f : exp2_small(ml[w].x - M);
    l = fmaf(ml[w].y, f, l);
#pragma unroll
    for (int i = 0; i < 16; ++i) o[i] = w == 0 ? *at(w, wave, i) * f : fmaf(*at(w, wave, i), f, o[i]);
  }
  if (kept.any && rows.real) kept.join(WinKept::place(to, rows, last, part, parts), o, wave, M);
  if (!more) {
    win_store(to, rows, o, wave, M, l, last, part, parts);
    return;
  }
  if (rows.real) WinKept::put(WinKept::place(to, rows, last, part, parts), o, wave);
  kept.any = true;
  kept.m = M;
  __syncthreads();                                       // the ring is free again
}

// ---- the parts of a row put together in order ------------------------------------------------------------------
// WAVES wavefronts a row, two channels a lane.
constexpr int kWinMergeWaves = 4;            // (eight take 3.5 us instead of 3.0 for a row of 32 parts)
constexpr int kWinMergeBatch = 8;              // partials of a wavefront on their way at once
constexpr int kWinMergeMany = 16;              // parts from which on a row has all four

// The first partials are on their way before it is known which of them there are.
template <int WAVES, class USED>
__device__ __forceinline__ void win_merge(const WinOut& to, int64_t row, int parts, int wave, const USED& used_parts) {
  const int lane = threadIdx.x & (DSK_WAVE - 1);
  const float2* ml = to.part_ml + row * parts;
  const float2* acc = reinterpret_cast<const float2*>(to.part_acc + row * parts * DSK_HEAD_DIM) + lane;
  float2 x[kWinMergeBatch], v[kWinMergeBatch];
  auto load = [&](int c0) {
#pragma unroll
    for (int u = 0; u < kWinMergeBatch; ++u) {
      const int c = c0 + u < parts ? c0 + u : parts - 1;
      v[u] = ml[c];
      x[u] = acc[(int64_t)c * (DSK_HEAD_DIM / 2)];
    }
  };
  int c0 = wave % WAVES * kWinMergeBatch;
  load(c0);
  const float2 mine = ml[lane < parts ? lane : parts - 1];
  const int used = used_parts();
  if (used <= 1) return;                                 // finished by the kernel before; uniform for a row
  float M = lane < used ? mine.x : -__builtin_inff(), l = 0.0f;
  for (int c = lane + DSK_WAVE; c < used; c += DSK_WAVE) M = fmaxf(M, ml[c].x);
  M = wave_max(M);
  float2 o = make_float2(0.0f, 0.0f);
  for (; c0 < used; c0 += WAVES * kWinMergeBatch, load(c0)) {
#pragma unroll
    for (int u = 0; u < kWinMergeBatch; ++u) {
      if (c0 + u >= used || v[u].y == 0.0f) continue;    // (not by the maximum: where every logit is NaN it is -inf)
      const float f = exp2_small(v[u].x - M);
      l = fmaf(v[u].y, f, l);
      o.x = fmaf(x[u].x, f, o.x);
      o.y = fmaf(x[u].y, f, o.y);
    }
  }
  if constexpr (WAVES > 1) {
    static_assert(WAVES == kWinMergeWaves, "all wavefronts of a workgroup have the same row");
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
  if (to.out != nullptr) *reinterpret_cast<float2*>(to.out + row * DSK_HEAD_DIM + 2 * lane) = o;
  if (to.out_bf16 != nullptr) *reinterpret_cast<uint32_t*>(to.out_bf16 + row * DSK_HEAD_DIM + 2 * lane) = tile_pack(o.x, o.y);
  if (lane == 0 && to.lse != nullptr) to.lse[row] = l == 0.0f ? -__builtin_inff() : (M + log2f(l)) * kLn2;
}

// ---- host ----------------------------------------------------------------------------------------------------
constexpr float kWinScale = 0.08838834764831845f;   // 128^-1/2


inline int64_t ceil_div(int64_t x, int64_t y) { return (x + y - 1) / y; }

template <class ARGS>
inline WinCache win_cache(const ARGS& a) {
  const int width = a.k_scale != nullptr ? 1 : 2;        // bytes of a channel
  WinCache c;
  c.K = static_cast<const unsigned char*>(a.K);
  c.V = static_cast<const unsigned char*>(a.V);
  c.k_tok = a.k_stride_tok * width;
  c.k_head = a.k_stride_head * width;
  c.v_tok = a.v_stride_tok * width;
  c.v_head = a.v_stride_head * width;
  c.ks = a.k_scale;
  c.vs = a.v_scale;
  c.s_head = a.scale_stride_head;
  c.s_shift = a.k_scale == nullptr ? 0 : (a.scale_block == 32 ? 5 : (a.scale_block == 64 ? 6 : 7));
  return c;
}

template <class ARGS>
inline WinOut win_out(const ARGS& a, size_t parts) {
  WinOut o;
  o.out = a.out;
  o.out_bf16 = static_cast<uint16_t*>(a.out_bf16);
  o.lse = a.lse;
  o.part_ml = static_cast<float2*>(a.workspace);
  o.part_acc = reinterpret_cast<float*>(static_cast<unsigned char*>(a.workspace) + align_up(parts * sizeof(float2)));
  return o;
}

inline size_t win_part_bytes(size_t parts) {
  const size_t total = align_up(parts * sizeof(float2)) + align_up(parts * DSK_HEAD_DIM * sizeof(float));
  return total > 256 ? total : 256;
}

}  // namespace dsk
