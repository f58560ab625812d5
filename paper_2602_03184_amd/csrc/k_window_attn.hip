// Attention of new tokens that see what is near and a few first tokens, over a cache in bf16 or 8 bits: causal with a sliding window
// (dsk_window_attn), and one token a sequence with the selected slots as well (dsk_window_sparse_decode_attn).
//
// The new tokens of a sequence and the query heads of a KV head's group are the rows of one product over the same keys, as in
// dsk_attn_tile.hpp.  Keys come in tiles of 32 positions; what a workgroup's rows see is a run of tiles for the first tokens and one
// for the window, and a tile is masked only if some row does not see all of it.  Long runs are split over workgroups, whose results
// a second launch puts together in a fixed order.
//
// A cache in 8 bits goes to LDS as it is, half the bytes of bf16 all the way, and is widened when fragments are read: K's codes with
// their scale, which gives bf16 numbers without rounding; V's as they are, with the scale in the weights instead, since the eight keys
// of a lane's fragment need not have one scale.
#include "dsk_attn_tile.hpp"
#include "dsk_common.hpp"
#include "dsk_internal.hpp"

#include <type_traits>

namespace dsk {

constexpr int kWinMaxSplit = 128;              // parts of a sequence at most
constexpr int kWinLeastTiles = 8;              // of a part: a shorter one costs more in partial results than it saves
constexpr int kWinLeastKeys = kWinLeastTiles * kAttnTile;
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

template <bool E4M3>
struct WinVFrag : TileVFrag {
  // all 32 keys while copies to other parts of LDS may be under way
  __device__ __forceinline__ void load(const unsigned char* sm_v) {
    if constexpr (!E4M3) {
      read_beside_copies(sm_v);
    } else {
      const int lane = threadIdx.x & (DSK_WAVE - 1), half = lane >> 5, group = (lane >> 4) & 1, e = (lane & 15) >> 1;
      const int r = 4 * half + (e & 3) + 2 * (e & 4);    // the lane's key of a transposing read, of 16
      const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const unsigned char*)sm_v + r * DSK_HEAD_DIM + ((lane & 1) << 3);
      const int f = win_swizzle8(r) ^ group;             // (the same for row r + 16)
      typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
      u32x2 x[4][2];
      static_assert(16 * DSK_HEAD_DIM == 2048, "offset: 16 rows");
      asm volatile(
          "ds_read_b64_tr_b8 %0, %8\n\tds_read_b64_tr_b8 %1, %8 offset:2048\n\t"
          "ds_read_b64_tr_b8 %2, %9\n\tds_read_b64_tr_b8 %3, %9 offset:2048\n\t"
          "ds_read_b64_tr_b8 %4, %10\n\tds_read_b64_tr_b8 %5, %10 offset:2048\n\t"
          "ds_read_b64_tr_b8 %6, %11\n\tds_read_b64_tr_b8 %7, %11 offset:2048\n\t"
          "s_waitcnt lgkmcnt(0)"
          : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[1][0]), "=&v"(x[1][1]), "=&v"(x[2][0]), "=&v"(x[2][1]), "=&v"(x[3][0]), "=&v"(x[3][1])
          : "v"(base + ((0 ^ f) << 4)), "v"(base + ((2 ^ f) << 4)), "v"(base + ((4 ^ f) << 4)), "v"(base + ((6 ^ f) << 4))
          : "memory");
#pragma unroll
      for (int ct = 0; ct < 4; ++ct)
#pragma unroll
        for (int t = 0; t < 2; ++t) v[ct][t] = win_widen8(x[ct][t].x, x[ct][t].y, 1.0f);
    }
  }
  // 0 for what is not finite; whether there was anything
  __device__ __forceinline__ bool keep_finite() {
    uint32_t found = 0;
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        uint4 x = __builtin_bit_cast(uint4, v[ct][t]);
        const uint4 y = make_uint4(finite_bf16(x.x), finite_bf16(x.y), finite_bf16(x.z), finite_bf16(x.w));
        found |= (x.x ^ y.x) | (x.y ^ y.y) | (x.z ^ y.z) | (x.w ^ y.w);
        v[ct][t] = __builtin_bit_cast(tile_bf16x8, y);
      }
    return __any(found != 0);
  }
};

// ---- which keys ------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t win_below(int64_t n) {   // bits 0 .. n - 1 of 32
  return n >= 32 ? 0xFFFFFFFFu : (n > 0 ? (1u << (int)n) - 1u : 0u);
}

// What a sequence has in fact, malformed tables cut to the bounds that the host knows.
struct WinPlace {
  int tok0, n;          // its new tokens; 0: nothing to do
  int64_t row0;
  int len, there;       // tokens before them; positions that have a row
  __device__ __forceinline__ WinPlace(const dsk_window_attn_args& a, int s) {
    tok0 = a.cu_new[s];
    int64_t m = (int64_t)a.cu_new[s + 1] - tok0;
    if (tok0 < 0 || tok0 > a.n_tokens || m < 0) m = 0;
    m = m < a.max_new ? m : a.max_new;
    m = m < a.n_tokens - tok0 ? m : a.n_tokens - tok0;
    n = (int)m;
    row0 = a.seq_row0[s];
    len = a.seq_len[s];
    const bool nowhere = row0 < 0 || row0 >= a.total_rows || len < 0;
    if (nowhere) row0 = len = 0;
    len = len < a.max_seqlen ? len : a.max_seqlen;
    const int64_t left = nowhere ? 0 : a.total_rows - row0;
    there = (int)(len + (int64_t)n < left ? len + (int64_t)n : left);
  }
};

// The tiles that rows [r0, r1) of a sequence see: `first` of the first tokens, then those from position lo on.
struct WinTiles {
  int p0, p1;           // positions of the first and the last row
  int first, lo, n;
  __device__ __forceinline__ WinTiles(const dsk_window_attn_args& a, const WinPlace& at, int G, int r0, int r1) {
    p0 = at.len + r0 / G;
    p1 = at.len + (r1 - 1) / G;
    const int w = p0 - a.window + 1 > 0 ? p0 - a.window + 1 : 0;
    const int hi = p1 + 1 < at.there ? p1 + 1 : at.there;
    int sinks = a.n_sink < w ? a.n_sink : w;
    sinks = sinks < at.there ? sinks : at.there;         // (no row, no tile)
    first = (int)(((int64_t)sinks + kAttnTile - 1) / kAttnTile);
    lo = w / kAttnTile * kAttnTile;
    if (first > 0 && lo <= first * kAttnTile) first = lo = 0;
    n = first + (hi > lo ? (hi - lo + kAttnTile - 1) / kAttnTile : 0);
  }
  __device__ __forceinline__ int t0(int v) const { return v < first ? v * kAttnTile : lo + (v - first) * kAttnTile; }
  __device__ __forceinline__ int used(int tiles_per_split) const {
    const int u = (n + tiles_per_split - 1) / tiles_per_split;
    return u > 0 ? u : 1;
  }
};

// Keys of a workgroup that are positions of its sequence: tiles [begin, end).
struct WinRun {
  WinTiles tiles;
  int begin, end;
  int64_t row0;
  int there, window, sinks;
  __device__ __forceinline__ int row_of(int v, int r) const {   // of the sequence; cut to what there is
    const int t = tiles.t0(v) + r;
    return t < there ? t : there - 1;
  }
  // every row sees all of the tile
  __device__ __forceinline__ bool plain(int v) const {
    const int t = tiles.t0(v);
    return t + kAttnTile <= (tiles.p0 + 1 < there ? tiles.p0 + 1 : there) && (t > tiles.p1 - window || t + kAttnTile <= sinks);
  }
  // keys of the tile that a row at position p sees
  __device__ __forceinline__ uint32_t allowed(int v, int p) const {
    const int64_t t = tiles.t0(v);
    const int64_t gone = (int64_t)p - window + 1;        // positions that have left the window
    return win_below((p + 1 < there ? p + 1 : there) - t) & (~win_below((gone > 0 ? gone : 0) - t) | win_below(sinks - t));
  }
};

// Keys of a workgroup that are listed in LDS as rows of the cache: every row of the product sees all of them.
struct WinList {
  const int32_t* rows;
  int count;
  int begin, end;
  int64_t row0;         // 0
  __device__ __forceinline__ int row_of(int v, int r) const {
    const int t = v * kAttnTile + r;
    return rows[t < count ? t : count - 1];
  }
  __device__ __forceinline__ bool plain(int v) const { return (v + 1) * kAttnTile <= count; }
  __device__ __forceinline__ uint32_t allowed(int v, int) const { return win_below(count - v * kAttnTile); }
};

// ---- a workgroup's keys folded into its rows -----------------------------------------------------------------
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

// QW wavefronts have 32 rows each, KW take other tiles of a stage for the same rows, NT of them each.  With two BUFS a stage is copied
// while the one before it is multiplied; with one that is left to the second workgroup of the CU.  TERMS: bf16 terms of a weight.
template <int QW, int KW, int NT, int BUFS, int TERMS, bool E4M3>
struct WinFold {
  static constexpr int kThreads = QW * KW * DSK_WAVE;
  static constexpr int kTiles = KW * NT, kKeys = kAttnTile * kTiles;   // of a stage
  static constexpr int kRowBytes = E4M3 ? DSK_HEAD_DIM : 2 * DSK_HEAD_DIM;
  static constexpr int kTile = kAttnTile * kRowBytes;
  static constexpr int kBuf = 2 * kTiles * kTile;
  static constexpr int kChunks = kRowBytes / 16, kRowsAtOnce = DSK_WAVE / kChunks;   // of a wavefront's copy
  static constexpr int kCopies = kKeys / (kRowsAtOnce * QW * KW);
  static_assert(kKeys <= kThreads && kCopies >= 1, "a thread a scale, every wavefront copies");
  static_assert(KW == 1 || BUFS * kBuf >= (KW - 1) * QW * 64 * DSK_WAVE * 4, "states are joined in the stages' place");
  struct Shared {
    __align__(16) unsigned char kv[BUFS * kBuf];
    float2 ml[KW > 1 ? (KW - 1) * QW * DSK_WAVE : 1];
    __align__(16) float scale[E4M3 ? BUFS * 2 * kKeys : 4];
  };

  template <class KEYS>
  static __device__ __forceinline__ void copy(const WinCache& c, const KEYS& keys, int hk, int v0, unsigned char* sm) {
    const int lane = threadIdx.x & (DSK_WAVE - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / DSK_WAVE);
    const unsigned char *K = c.K + hk * c.k_head, *V = c.V + hk * c.v_head;
#pragma unroll
    for (int u = 0; u < kCopies; ++u) {
      const int first = (u * QW * KW + wave) * kRowsAtOnce, at = first + lane / kChunks;   // rows of the stage, of one tile
      const int v = v0 + first / kAttnTile;
      const int64_t row = keys.row0 + keys.row_of(v < keys.end ? v : keys.end - 1, at % kAttnTile);
      const int place = lane % kChunks;                  // a wavefront's copy lies lane after lane: the swizzle is in what it reads
      const int kc = E4M3 ? place ^ win_swizzle8(at) : place ^ (at & 15), vc = E4M3 ? kc : place ^ ((at & 3) << 2);
      lds_copy16<false>(K + row * c.k_tok + kc * 16, sm + first * kRowBytes);
      lds_copy16<false>(V + row * c.v_tok + vc * 16, sm + kTiles * kTile + first * kRowBytes);
    }
  }
  template <class KEYS>
  static __device__ __forceinline__ uchar2 scales(const WinCache& c, const KEYS& keys, int hk, int v0) {
    uchar2 b = make_uchar2(0, 0);
    if (E4M3 && threadIdx.x < kKeys) {
      const int v = v0 + threadIdx.x / kAttnTile;
      const int64_t at = hk * c.s_head + ((keys.row0 + keys.row_of(v < keys.end ? v : keys.end - 1, threadIdx.x % kAttnTile)) >> c.s_shift);
      b.x = c.ks[at];
      b.y = c.vs[at];
    }
    return b;
  }

  // The values that were left out of a tile, for the rows that see them.
  template <class KEYS>
  static __device__ __forceinline__ void add_left_out(tile_f32x16 (&O)[4], const WinCache& c, const KEYS& keys, int hk, int v, uint32_t allow, int half) {
    for (int j = 0; j < kAttnTile; ++j) {
      if (!((allow >> j) & 1u)) continue;
      const unsigned char* at = c.V + hk * c.v_head + (keys.row0 + keys.row_of(v, j)) * c.v_tok;
#pragma unroll
      for (int ct = 0; ct < 4; ++ct)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int ch = ct * 32 + 8 * (i >> 2) + 4 * half + (i & 3);
          if constexpr (E4M3) {
            if ((at[ch] & 0x7Fu) == 0x7Fu) O[ct][i] += __builtin_nanf("");
          } else {
            const uint16_t x = reinterpret_cast<const uint16_t*>(at)[ch];
            if ((x & 0x7F80u) == 0x7F80u) O[ct][i] += bf16_to_f32(x);
          }
        }
    }
  }

  template <class KEYS>
  static __device__ __forceinline__ void run(Shared& sh, const WinCache& c, const KEYS& keys, int hk, const WinRows& rows, int kw, TileSoftmax& sm,
                                             tile_f32x16 (&O)[4]) {
    const int tid = threadIdx.x;
    auto tiles = [&](int v0, int buf) {
      const unsigned char *sm_k = sh.kv + buf * kBuf, *sm_v = sm_k + kTiles * kTile;
      const float* scale = sh.scale + buf * 2 * kKeys;
#pragma unroll
      for (int sub = 0; sub < NT; ++sub) {
        const int tile = kw * NT + sub, v = v0 + tile;
        if (v >= keys.end) break;
        WinKFrag<E4M3> kf;
        kf.load(sm_k + tile * kTile, rows, E4M3 ? scale[tile * kAttnTile + rows.col] : 1.0f);
        tile_f32x16 z;
        kf.template add<0, 8>(z, rows);
        const bool plain = keys.plain(v);
        uint32_t allow = 0;
        if (!plain) {
          allow = rows.real ? keys.allowed(v, rows.pos) : 0u;
          tile_hide(z, allow, rows.half);
        }
        WinVFrag<E4M3> vf;
        __builtin_amdgcn_sched_barrier(0);
        vf.load(sm_v + tile * kTile);
        __builtin_amdgcn_sched_barrier(0);
        // a masked row may hold anything, and 0 * NaN is NaN: such values stay out of the product
        const bool left_out = !plain && vf.keep_finite();
        TileWeights<TERMS> w;
        if constexpr (E4M3) sm.template take<TERMS, true>(z, O, w, scale + kKeys + tile * kAttnTile + 4 * rows.half);
        else sm.template take<TERMS, true>(z, O, w);
        vf.template add<TERMS>(O, w, 0);
        vf.template add<TERMS>(O, w, 1);
        if (left_out) add_left_out(O, c, keys, hk, v, allow, rows.half);
      }
    };
    uchar2 b = make_uchar2(0, 0);
    int buf = 0;
    if (BUFS > 1 && keys.begin < keys.end) {
      copy(c, keys, hk, keys.begin, sh.kv);
      b = scales(c, keys, hk, keys.begin);
    }
    for (int v0 = keys.begin; v0 < keys.end; v0 += kTiles) {
      if (BUFS == 1) {
        copy(c, keys, hk, v0, sh.kv);
        b = scales(c, keys, hk, v0);
      }
      lds_copies_done();
      if (E4M3 && tid < kKeys) {
        sh.scale[buf * 2 * kKeys + tid] = __uint_as_float((uint32_t)b.x << 23);
        sh.scale[buf * 2 * kKeys + kKeys + tid] = __uint_as_float((uint32_t)b.y << 23);
      }
      __syncthreads();                                   // the stage is here, and nobody reads the other one any more
      if (BUFS > 1 && v0 + kTiles < keys.end) {
        copy(c, keys, hk, v0 + kTiles, sh.kv + (buf ^ 1) * kBuf);
        b = scales(c, keys, hk, v0 + kTiles);
      }
      if (rows.busy) tiles(v0, buf);
      if (BUFS == 1) __syncthreads();
      else buf ^= 1;
    }
    if (BUFS > 1) __syncthreads();
    sm.close();
  }
};

__device__ __forceinline__ void win_clear(tile_f32x16 (&O)[4]) {
#pragma unroll
  for (int ct = 0; ct < 4; ++ct)
#pragma unroll
    for (int i = 0; i < 16; ++i) O[ct][i] = 0.0f;
}

// A lane's row: final, or part `part` of `parts`.  Its channels lie four in a row, at 32 ct + 8 i + 4 half.
__device__ __forceinline__ void win_store(const WinOut& to, const WinRows& rows, const tile_f32x16 (&O)[4], float m, float l, bool last,
                                          int part, int parts) {
  if (!rows.real) return;
  if (last) {
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 x = make_float4(O[ct][4 * i] * inv, O[ct][4 * i + 1] * inv, O[ct][4 * i + 2] * inv, O[ct][4 * i + 3] * inv);
        const int64_t at = rows.out_row * DSK_HEAD_DIM + ct * 32 + 8 * i + 4 * rows.half;
        if (to.out != nullptr) *reinterpret_cast<float4*>(to.out + at) = x;
        if (to.out_bf16 != nullptr)
          *reinterpret_cast<uint2*>(to.out_bf16 + at) = make_uint2(tile_pack(x.x, x.y), tile_pack(x.z, x.w));
      }
    if (rows.half == 0 && to.lse != nullptr) to.lse[rows.out_row] = l == 0.0f ? -__builtin_inff() : (m + log2f(l)) * kLn2;   // a NaN stays one
  } else {
    const int64_t p = rows.out_row * parts + part;
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<float4*>(to.part_acc + p * DSK_HEAD_DIM + ct * 32 + 8 * i + 4 * rows.half) =
            make_float4(O[ct][4 * i], O[ct][4 * i + 1], O[ct][4 * i + 2], O[ct][4 * i + 3]);
    if (rows.half == 0) to.part_ml[p] = make_float2(m, l);
  }
}

struct WinSplit {
  int parts, tiles_per_part;
};

template <int QW, int KW, int NT, int BUFS, int TERMS, bool E4M3>
__global__ __launch_bounds__(QW * KW * DSK_WAVE, 2) void window_attn_kernel(dsk_window_attn_args a, WinCache c, WinOut to, int G, int q_tiles,
                                                                            WinSplit sp, float scale_log2) {
  using Fold = WinFold<QW, KW, NT, BUFS, TERMS, E4M3>;
  __shared__ typename Fold::Shared sh;
  const int part = blockIdx.y, s = blockIdx.z;
  const int hk = blockIdx.x / q_tiles, q_tile = blockIdx.x - hk * q_tiles;
  const int lane = threadIdx.x & (DSK_WAVE - 1), wave = threadIdx.x / DSK_WAVE, qw = wave % QW, kw = wave / QW;

  const WinPlace at(a, s);
  const int64_t r0 = (int64_t)q_tile * QW * kAttnTile, all = (int64_t)at.n * G;   // this workgroup's first row
  if (r0 >= all) return;                                 // uniform, as all returns before the end
  const int r1 = (int)(r0 + QW * kAttnTile < all ? r0 + QW * kAttnTile : all);
  const WinTiles tiles(a, at, G, (int)r0, r1);
  const int used = tiles.used(sp.tiles_per_part);
  if (part >= used) return;
  WinRun keys{tiles, part * sp.tiles_per_part, 0, at.row0, at.there, a.window, a.n_sink};
  keys.end = tiles.n - keys.begin < sp.tiles_per_part ? tiles.n : keys.begin + sp.tiles_per_part;

  WinRows rows;
  rows.col = lane & 31;
  rows.half = lane >> 5;
  const int r = (int)r0 + qw * kAttnTile + rows.col;
  rows.busy = r0 + qw * kAttnTile < all;
  rows.real = r < all;
  const int i = rows.real ? r / G : 0;
  rows.pos = at.len + i;
  rows.out_row = (int64_t)(at.tok0 + i) * a.Hq + hk * G + (rows.real ? r - i * G : 0);
  rows.template load<E4M3>(static_cast<const uint16_t*>(a.q));
  TileSoftmax sm(scale_log2);
  tile_f32x16 O[4];
  win_clear(O);
  Fold::run(sh, c, keys, hk, rows, kw, sm, O);
  if constexpr (KW > 1) {
    tile_join<QW, KW>(sm, O, rows.busy, qw, kw, reinterpret_cast<float*>(sh.kv), sh.ml);
    if (kw > 0) return;
  }
  win_store(to, rows, O, sm.m, sm.l, used == 1, part, sp.parts);
}

// ---- selected slots and what is near ---------------------------------------------------------------------------
struct WinSparse {
  int G, heads;               // query heads of a KV head; lists of a sequence
  int slots_per_part, slot_parts;
  int near_per_part, near_parts;
  int row_tiles;              // workgroups for the query heads of a KV head, 32 each
};

// Parts 0 .. slot_parts - 1 of a list are its slots'; the others, of a KV head, are what is near.  Every part leaves a result.
template <int KW, int NT, int TERMS, bool E4M3>
__global__ __launch_bounds__(KW * DSK_WAVE, 2) void window_sparse_kernel(dsk_window_sparse_args a, WinCache c, WinOut to, WinSparse sp,
                                                                         float scale_log2) {
  using Fold = WinFold<1, KW, NT, 1, TERMS, E4M3>;
  __shared__ typename Fold::Shared sh;
  __shared__ int32_t sm_rows[kWinMaxListed];
  __shared__ int32_t sm_slot[3][kWinMaxSlots];
  __shared__ int32_t sm_wave[kWinMaxSlots / DSK_WAVE];
  constexpr int kThreads = KW * DSK_WAVE;
  static_assert(kThreads == kWinMaxSlots, "a thread a slot");
  const int part = blockIdx.x, s = blockIdx.z;
  const int list = blockIdx.y / sp.row_tiles, g0 = (blockIdx.y - list * sp.row_tiles) * kAttnTile;   // the first of its query heads
  const int tid = threadIdx.x, lane = tid & (DSK_WAVE - 1), wave = tid / DSK_WAVE;
  const bool shared = sp.heads != a.Hq, near = part >= sp.slot_parts;
  if (!shared && (near ? list % sp.G != 0 : g0 != 0)) return;          // uniform, as all returns before the end
  const int hk = shared ? list : list / sp.G;

  // slots and lengths on their way together
  const int first = part * sp.slots_per_part;
  int slots = 0, start = 0, ln = 0;
  if (!near) {
    const int64_t at = (int64_t)s * sp.heads + list;
    slots = a.sel_count[at];
    if (tid < sp.slots_per_part && tid < a.k - first) {
      start = a.sel_start[at * a.k + first + tid];
      ln = a.sel_len[at * a.k + first + tid];
    }
  }
  int64_t row0 = a.seq_row0[s], len = a.seq_len[s];
  if (row0 < 0 || row0 >= a.total_rows || len < 0) row0 = len = 0;
  len = len < a.max_seqlen ? len : a.max_seqlen;
  len = len < a.total_rows - row0 ? len : a.total_rows - row0;
  const int64_t lo = len > a.window ? len - a.window : 0;              // first position of the window
  const int64_t few = a.n_sink < lo ? a.n_sink : lo;                   // first tokens before it

  WinRows rows;
  rows.col = lane & 31;
  rows.half = lane >> 5;
  rows.real = g0 + rows.col < (shared || near ? sp.G : 1);
  rows.busy = true;
  rows.pos = 0;
  rows.out_row = (int64_t)s * a.Hq + (shared || near ? hk * sp.G + g0 : list) + (rows.real ? rows.col : 0);
  rows.template load<E4M3>(static_cast<const uint16_t*>(a.q));

  int count = 0;
  if (near) {
    const int64_t all = few + (len - lo), begin = (int64_t)(part - sp.slot_parts) * sp.near_per_part;
    const int64_t left = all - begin;
    count = left > 0 ? (int)(left < sp.near_per_part ? left : sp.near_per_part) : 0;
    for (int i = tid; i < count; i += kThreads) {
      const int64_t t = begin + i;
      sm_rows[i] = (int)(row0 + (t < few ? t : lo + (t - few)));
    }
  } else {
    // what is near is not taken from the slots: a span stays a span
    slots = slots < a.k ? slots : a.k;
    if (tid >= slots - first || tid >= sp.slots_per_part || ln <= 0 || start < 0) ln = 0;
    ln = ln < a.b ? ln : a.b;
    int64_t from = start, upto = (int64_t)start + ln;
    from = from > row0 + few ? from : row0 + few;
    upto = upto < row0 + lo ? upto : row0 + lo;
    ln = upto > from ? (int)(upto - from) : 0;
    const int incl = wave_incl_scan_i(ln, lane);
    if (lane == DSK_WAVE - 1) sm_wave[wave] = incl;
    sm_slot[0][tid] = incl - ln;
    sm_slot[1][tid] = (int)from;
    sm_slot[2][tid] = ln;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWinMaxSlots / DSK_WAVE; ++w) count += sm_wave[w];
    const int here = slots - first < sp.slots_per_part ? slots - first : sp.slots_per_part;
    for (int i = tid; i < here * a.b; i += kThreads) {
      const int slot = i / a.b, off = i - slot * a.b;
      int base = sm_slot[0][slot];
      for (int w = 0; w < slot / DSK_WAVE; ++w) base += sm_wave[w];
      if (off < sm_slot[2][slot]) sm_rows[base + off] = sm_slot[1][slot] + off;
    }
  }
  __syncthreads();

  const WinList keys{sm_rows, count, 0, (count + kAttnTile - 1) / kAttnTile, 0};
  TileSoftmax sm(scale_log2);
  tile_f32x16 O[4];
  win_clear(O);
  Fold::run(sh, c, keys, hk, rows, wave, sm, O);
  tile_join<1, KW>(sm, O, true, 0, wave, reinterpret_cast<float*>(sh.kv), sh.ml);
  if (wave > 0) return;
  const int parts = sp.slot_parts + sp.near_parts;
  win_store(to, rows, O, sm.m, sm.l, parts == 1, part, parts);
}

// ---- the parts of a row put together in order ------------------------------------------------------------------
// WAVES wavefronts a row, two channels a lane.
constexpr int kWinMergeWaves = 4;
constexpr int kWinMergeBatch = 8;              // partials of a wavefront on their way at once
constexpr int kWinMergeMany = 16;              // parts from which on a row has all four

template <int WAVES>
__device__ __forceinline__ void win_merge(const WinOut& to, int64_t row, int used, int parts, int wave) {
  const int lane = threadIdx.x & (DSK_WAVE - 1);
  const float2* ml = to.part_ml + row * parts;
  const float2* acc = reinterpret_cast<const float2*>(to.part_acc + row * parts * DSK_HEAD_DIM) + lane;
  float M = -__builtin_inff(), l = 0.0f;
  for (int c = lane; c < used; c += DSK_WAVE) M = fmaxf(M, ml[c].x);
  M = wave_max(M);
  float2 o = make_float2(0.0f, 0.0f);
  for (int c0 = wave % WAVES * kWinMergeBatch; c0 < used; c0 += WAVES * kWinMergeBatch) {
    float2 x[kWinMergeBatch], v[kWinMergeBatch];
#pragma unroll
    for (int u = 0; u < kWinMergeBatch; ++u) {
      const int c = c0 + u < used ? c0 + u : used - 1;
      v[u] = ml[c];
      x[u] = acc[(int64_t)c * (DSK_HEAD_DIM / 2)];
    }
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

// q_rows: rows of a workgroup of the kernel above
template <int WAVES>
__global__ __launch_bounds__(kWinMergeWaves * DSK_WAVE) void window_merge_kernel(dsk_window_attn_args a, WinOut to, int G, int q_rows, WinSplit sp) {
  constexpr int kRows = kWinMergeWaves / WAVES;
  const int s = blockIdx.y, wave = threadIdx.x / DSK_WAVE;
  const int64_t item = (int64_t)blockIdx.x * kRows + wave / WAVES;
  const int i = (int)(item / a.Hq), h = (int)(item - (int64_t)i * a.Hq);
  const WinPlace at(a, s);
  if (i >= at.n) return;
  const int all = at.n * G, r0 = (i * G + h % G) / q_rows * q_rows;
  const WinTiles tiles(a, at, G, r0, r0 + q_rows < all ? r0 + q_rows : all);
  const int used = tiles.used(sp.tiles_per_part);
  if (used <= 1) return;                                 // finished by the kernel above
  win_merge<WAVES>(to, (int64_t)(at.tok0 + i) * a.Hq + h, used, sp.parts, wave);
}

template <int WAVES>
__global__ __launch_bounds__(kWinMergeWaves * DSK_WAVE) void window_sparse_merge_kernel(int64_t rows, WinOut to, int parts) {
  const int wave = threadIdx.x / DSK_WAVE;
  const int64_t row = (int64_t)blockIdx.x * (kWinMergeWaves / WAVES) + wave / WAVES;
  if (row < rows) win_merge<WAVES>(to, row, parts, parts, wave);
}

// ---- geometry: follows the host's bounds alone ---------------------------------------------------------------
static int64_t ceil_div(int64_t x, int64_t y) { return (x + y - 1) / y; }

template <class ARGS>
static WinCache win_cache(const ARGS& a) {
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
static WinOut win_out(const ARGS& a, size_t parts) {
  WinOut o;
  o.out = a.out;
  o.out_bf16 = static_cast<uint16_t*>(a.out_bf16);
  o.lse = a.lse;
  o.part_ml = static_cast<float2*>(a.workspace);
  o.part_acc = reinterpret_cast<float*>(static_cast<unsigned char*>(a.workspace) + align_up(parts * sizeof(float2)));
  return o;
}

static size_t win_part_bytes(size_t parts) {
  const size_t total = align_up(parts * sizeof(float2)) + align_up(parts * DSK_HEAD_DIM * sizeof(float));
  return total > 256 ? total : 256;
}

struct WinLaunch {
  int q_waves, q_tiles;
  WinSplit sp;
};

// Parts of a sequence at most, whatever max_seqlen up to the given one is: a workspace that is kept serves a growing cache.
static int win_most_parts(const dsk_window_attn_args& a, int q_tiles, int64_t tiles) {
  const int64_t want = 2 * kWinCus / ((int64_t)a.Hkv * q_tiles), by_length = ceil_div(tiles, kWinLeastTiles);
  int64_t n = want < by_length ? want : by_length;
  n = n < kWinMaxSplit ? n : kWinMaxSplit;
  return (int)(n > 1 ? n : 1);
}

static WinLaunch win_layout(const dsk_window_attn_args& a) {
  const int G = a.Hq / a.Hkv;
  const int64_t rows = (int64_t)a.max_new * G;
  WinLaunch t;
  t.q_waves = rows <= kAttnTile ? 1 : (rows <= kWinTwoTermRows ? 2 : 4);
  t.q_tiles = (int)ceil_div(rows, t.q_waves * kAttnTile);
  // tiles that a workgroup's rows see at most: the window of all its tokens, the first ones, a tile begun at either end
  const int64_t tokens = a.max_new < t.q_waves * kAttnTile / G + 2 ? a.max_new : t.q_waves * kAttnTile / G + 2;
  const int64_t longest = (int64_t)a.max_seqlen + a.max_new;
  const int64_t near = ceil_div((int64_t)a.window + tokens, kAttnTile) + 1 + ceil_div(a.n_sink, kAttnTile);
  const int64_t tiles = near < ceil_div(longest, kAttnTile) ? near : ceil_div(longest, kAttnTile);
  const int most = win_most_parts(a, t.q_tiles, tiles);
  int64_t parts = 2 * kWinCus / ((int64_t)a.Hkv * t.q_tiles * a.B);
  parts = parts > 1 ? (parts < most ? parts : most) : 1;
  t.sp.tiles_per_part = (int)ceil_div(tiles, parts);
  t.sp.tiles_per_part = t.sp.tiles_per_part > 1 ? t.sp.tiles_per_part : 1;
  t.sp.parts = (int)ceil_div(tiles, t.sp.tiles_per_part);
  t.sp.parts = t.sp.parts > 1 ? t.sp.parts : 1;
  return t;
}

size_t window_ws_bytes(const dsk_window_attn_args& a) {
  const WinLaunch t = win_layout(a);
  const int most = win_most_parts(a, t.q_tiles, ceil_div((int64_t)a.max_seqlen + a.max_new, kAttnTile));
  return win_part_bytes(most > 1 ? (size_t)a.n_tokens * a.Hq * most : 0);
}

template <int QW, int KW, int NT8, int NT16, int BUFS>
static void launch_window(const dsk_window_attn_args& a, const WinLaunch& t, const WinCache& c, const WinOut& to, float scale_log2, hipStream_t st) {
  const int G = a.Hq / a.Hkv;
  const dim3 grid((unsigned)(a.Hkv * t.q_tiles), (unsigned)t.sp.parts, (unsigned)a.B), block(QW * KW * DSK_WAVE);
  auto go = [&](auto terms) {
    constexpr int kTerms = decltype(terms)::value;
    if (a.k_scale != nullptr)
      window_attn_kernel<QW, KW, NT8, BUFS, kTerms, true><<<grid, block, 0, st>>>(a, c, to, G, t.q_tiles, t.sp, scale_log2);
    else
      window_attn_kernel<QW, KW, NT16, BUFS, kTerms, false><<<grid, block, 0, st>>>(a, c, to, G, t.q_tiles, t.sp, scale_log2);
  };
  static_assert(kWinTwoTermRows == 2 * kAttnTile, "one and two wavefronts' rows always have two terms, four wavefronts' never");
  if (a.out != nullptr) go(std::integral_constant<int, 3>());
  else go(std::integral_constant<int, QW <= 2 ? 2 : 1>());
}

constexpr float kWinScale = 0.08838834764831845f;   // 128^-1/2

hipError_t launch_window_attn(const dsk_window_attn_args& a, hipStream_t st) {
  const WinLaunch t = win_layout(a);
  const int G = a.Hq / a.Hkv;
  const WinCache c = win_cache(a);
  const WinOut to = win_out(a, t.sp.parts > 1 ? (size_t)a.n_tokens * a.Hq * t.sp.parts : 0);
  const float scale_log2 = (a.scale != 0.0f ? a.scale : kWinScale) * kLog2e;
  if (t.q_waves == 1) launch_window<1, 4, 2, 1, 1>(a, t, c, to, scale_log2, st);
  else if (t.q_waves == 2) launch_window<2, 2, 2, 1, 2>(a, t, c, to, scale_log2, st);
  else launch_window<4, 1, 4, 2, 2>(a, t, c, to, scale_log2, st);
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess || t.sp.parts <= 1) return err;
  const bool many = t.sp.parts >= kWinMergeMany;
  const int64_t rows = (int64_t)a.max_new * a.Hq, wgs = ceil_div(rows, many ? 1 : kWinMergeWaves);
  const dim3 grid((unsigned)wgs, (unsigned)a.B), block(kWinMergeWaves * DSK_WAVE);
  if (many) window_merge_kernel<kWinMergeWaves><<<grid, block, 0, st>>>(a, to, G, t.q_waves * kAttnTile, t.sp);
  else window_merge_kernel<1><<<grid, block, 0, st>>>(a, to, G, t.q_waves * kAttnTile, t.sp);
  return hipGetLastError();
}

static int64_t win_most_slots(int b) { return kWinMaxListed / b < kWinMaxSlots ? kWinMaxListed / b : kWinMaxSlots; }
static int64_t win_least_slots(int b) { return kWinLeastKeys / b > 1 ? kWinLeastKeys / b : 1; }

static WinSparse win_sparse_layout(const dsk_window_sparse_args& a) {
  WinSparse sp;
  const bool shared = a.flags & DSK_ATTN_SHARED_SELECTION;
  sp.G = a.Hq / a.Hkv;
  sp.heads = shared ? a.Hkv : a.Hq;
  const int64_t least = win_least_slots(a.b), most = win_most_slots(a.b);
  int64_t per = ceil_div((int64_t)a.k * a.B * sp.heads, 2 * kWinCus);
  per = per > least ? per : least;
  per = per < most ? per : most;
  sp.slots_per_part = (int)per;
  sp.slot_parts = (int)ceil_div(a.k, per);
  const int64_t near = (int64_t)a.window + a.n_sink < a.max_seqlen ? (int64_t)a.window + a.n_sink : a.max_seqlen;
  int64_t near_per = ceil_div(near * a.B * a.Hkv, 2 * kWinCus);
  near_per = near_per > kWinLeastKeys ? near_per : kWinLeastKeys;
  sp.near_per_part = (int)(near_per < kWinMaxListed ? near_per : kWinMaxListed);
  sp.near_parts = (int)ceil_div(near, sp.near_per_part);
  sp.row_tiles = (int)ceil_div(sp.G, kAttnTile);
  return sp;
}

// No less than with a smaller k, window or max_seqlen: parts of n things that are at least `least` and at most `most` each and
// otherwise shared out to 2 * kWinCus / lists parts.
size_t window_sparse_ws_bytes(const dsk_window_sparse_args& a) {
  const WinSparse sp = win_sparse_layout(a);
  auto bound = [&](int64_t n, int64_t least, int64_t most, int64_t lists) {
    const int64_t by_length = ceil_div(n, least), shared_out = ceil_div(2 * kWinCus, lists), fewest = ceil_div(n, most);
    const int64_t parts = by_length < shared_out ? by_length : shared_out;
    return (size_t)(parts > fewest ? parts : fewest);
  };
  const int64_t near = (int64_t)a.window + a.n_sink < a.max_seqlen ? (int64_t)a.window + a.n_sink : a.max_seqlen;
  const size_t parts = bound(a.k, win_least_slots(a.b), win_most_slots(a.b), (int64_t)a.B * sp.heads) +
                       bound(near, kWinLeastKeys, kWinMaxListed, (int64_t)a.B * a.Hkv);
  return win_part_bytes((size_t)a.B * a.Hq * parts);
}

hipError_t launch_window_sparse(const dsk_window_sparse_args& a, hipStream_t st) {
  const WinSparse sp = win_sparse_layout(a);
  const int parts = sp.slot_parts + sp.near_parts;
  const int64_t rows = (int64_t)a.B * a.Hq;
  const WinCache c = win_cache(a);
  const WinOut to = win_out(a, parts > 1 ? (size_t)rows * parts : 0);
  const float scale_log2 = (a.scale != 0.0f ? a.scale : kWinScale) * kLog2e;
  const dim3 grid((unsigned)parts, (unsigned)(sp.heads * sp.row_tiles), (unsigned)a.B), block(4 * DSK_WAVE);
  if (a.k_scale != nullptr) {
    if (a.out != nullptr) window_sparse_kernel<4, 2, 3, true><<<grid, block, 0, st>>>(a, c, to, sp, scale_log2);
    else window_sparse_kernel<4, 2, 2, true><<<grid, block, 0, st>>>(a, c, to, sp, scale_log2);
  } else {
    if (a.out != nullptr) window_sparse_kernel<4, 1, 3, false><<<grid, block, 0, st>>>(a, c, to, sp, scale_log2);
    else window_sparse_kernel<4, 1, 2, false><<<grid, block, 0, st>>>(a, c, to, sp, scale_log2);
  }
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess || parts <= 1) return err;
  const bool many = parts >= kWinMergeMany;
  const dim3 merge((unsigned)ceil_div(rows, many ? 1 : kWinMergeWaves)), merge_block(kWinMergeWaves * DSK_WAVE);
  if (many) window_sparse_merge_kernel<kWinMergeWaves><<<merge, merge_block, 0, st>>>(rows, to, parts);
  else window_sparse_merge_kernel<1><<<merge, merge_block, 0, st>>>(rows, to, parts);
  return hipGetLastError();
}

}  // namespace dsk
