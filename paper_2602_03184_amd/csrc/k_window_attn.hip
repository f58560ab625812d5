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
#include "dsk_window_fold.hpp"

namespace dsk {

// ---- which keys ------------------------------------------------------------------------------------------
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
  WinTiles() = default;
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
  static constexpr bool kRun = true;
  WinTiles tiles;
  int begin, end;
  int64_t row0;
  int there, window, sinks;
  // row of the cache of the tile's first position, which there always is, and the last of its positions that there is
  __device__ __forceinline__ int64_t start(int v) const { return row0 + tiles.t0(v); }
  __device__ __forceinline__ int last(int v) const {
    const int left = there - tiles.t0(v);
    return (left < kAttnTile ? left : kAttnTile) - 1;
  }
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

// ---- a workgroup's keys folded into its rows -----------------------------------------------------------------
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
          tile_hide(z, allow >> (4 * rows.half), 0);
        }
        WinVFrag<E4M3> vf;
        __builtin_amdgcn_sched_barrier(0);
        vf.load(sm_v + tile * kTile);
        __builtin_amdgcn_sched_barrier(0);
        // a masked row may hold anything, and 0 * NaN is NaN: such values stay out of the product
        const bool left_out = !plain && vf.keep_finite();
        TileWeights<TERMS> w;
        sm.template take<TERMS, true>(z, O, w, [&](float (&p)[16]) {
          if constexpr (E4M3) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float4 f = *reinterpret_cast<const float4*>(scale + kKeys + tile * kAttnTile + 4 * rows.half + 8 * j);
              p[4 * j] *= f.x; p[4 * j + 1] *= f.y; p[4 * j + 2] *= f.z; p[4 * j + 3] *= f.w;
            }
          }
        });
        vf.template multiply<TERMS>(O, w, 1.0f);
        if (left_out) win_add_left_out<E4M3>(O, c, keys, hk, v, allow, rows.half);
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

struct WinSplit {
  int parts, tiles_per_part;
};

// What a workgroup takes: rows from r0 on of KV head hk, and a part of the tiles that they see; false: nothing.
struct WinWork {
  int s, hk, part, used;
  int64_t r0, all;      // first row; rows of the sequence
  __device__ __forceinline__ bool find(const dsk_window_attn_args& a, const WinSplit& sp, int G, int q_tiles, int q_rows, WinRun& keys, int& tok0, int& len) {
    part = blockIdx.y;
    s = blockIdx.z;
    hk = blockIdx.x / q_tiles;
    const WinPlace at(a, s);
    r0 = (int64_t)(blockIdx.x - hk * q_tiles) * q_rows;
    all = (int64_t)at.n * G;
    if (r0 >= all) return false;
    const WinTiles tiles(a, at, G, (int)r0, (int)(r0 + q_rows < all ? r0 + q_rows : all));
    used = tiles.used(sp.tiles_per_part);
    if (part >= used) return false;
    const int begin = part * sp.tiles_per_part;
    keys = WinRun{tiles, begin, tiles.n - begin < sp.tiles_per_part ? tiles.n : begin + sp.tiles_per_part, at.row0, at.there, a.window, a.n_sink};
    tok0 = at.tok0;
    len = at.len;
    return true;
  }
  // the rows of a wavefront from r0 + first on
  template <bool E4M3>
  __device__ __forceinline__ void rows(WinRows& rows, const dsk_window_attn_args& a, int G, int first, int tok0, int len) const {
    const int lane = threadIdx.x & (DSK_WAVE - 1);
    rows.col = lane & 31;
    rows.half = lane >> 5;
    const int r = (int)r0 + first + rows.col;
    rows.busy = r0 + first < all;
    rows.real = r < all;
    const int i = rows.real ? r / G : 0;
    rows.pos = len + i;
    rows.out_row = (int64_t)(tok0 + i) * a.Hq + hk * G + (rows.real ? r - i * G : 0);
    rows.template load<E4M3>(static_cast<const uint16_t*>(a.q));
  }
};

template <int QW, int KW, int NT, int BUFS, int TERMS, bool E4M3>
__global__ __launch_bounds__(QW * KW * DSK_WAVE, 2) void window_attn_kernel(dsk_window_attn_args a, WinCache c, WinOut to, int G, int q_tiles,
                                                                            WinSplit sp, float scale_log2) {
  using Fold = WinFold<QW, KW, NT, BUFS, TERMS, E4M3>;
  __shared__ typename Fold::Shared sh;
  const int wave = threadIdx.x / DSK_WAVE, qw = wave % QW, kw = wave / QW;
  WinWork work;
  WinRun keys;
  int tok0 = 0, len = 0;
  if (!work.find(a, sp, G, q_tiles, QW * kAttnTile, keys, tok0, len)) return;   // uniform, as all returns before the end
  WinRows rows;
  work.rows<E4M3>(rows, a, G, qw * kAttnTile, tok0, len);
  TileSoftmax sm(scale_log2);
  tile_f32x16 O[4];
  win_clear(O);
  Fold::run(sh, c, keys, work.hk, rows, kw, sm, O);
  if constexpr (KW > 1) {
    tile_join<QW, KW>(sm, O, rows.busy, qw, kw, reinterpret_cast<float*>(sh.kv), sh.ml);
    if (kw > 0) return;
  }
#pragma unroll
  for (int ct = 0; ct < 4; ++ct) win_store(to, rows, O[ct], ct, sm.m, sm.l, work.used == 1, work.part, sp.parts);
}

// The same where the rows fit one wavefront: HBM bounds it.
template <int TERMS, bool E4M3, bool STREAM>
__global__ __launch_bounds__(kStreamWaves * DSK_WAVE, E4M3 ? 2 : 1) void window_stream_kernel(dsk_window_attn_args a, WinCache c, WinOut to, int G,
                                                                                             WinSplit sp, float scale_log2) {
  __shared__ WinStreamLds<E4M3> sh;
  WinWork work;
  WinRun keys;
  int tok0 = 0, len = 0;
  if (!work.find(a, sp, G, 1, kAttnTile, keys, tok0, len)) return;     // uniform
  WinRows rows;
  work.rows<E4M3>(rows, a, G, 0, tok0, len);
  TileSoftmax sm(scale_log2);
  tile_f32x16 O[4];
  win_clear(O);
  win_stream<TERMS, E4M3, STREAM>(sh, c, keys, work.hk, rows, sm, O);
  win_stream_store<E4M3>(sh, to, rows, sm, O, work.used == 1, work.part, sp.parts);
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

// ---- geometry: follows the host's bounds alone ---------------------------------------------------------------
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
  // two workgroups a CU; of those that stream bf16 tiles, whose rings are twice as large, one
  const int64_t want = t.q_waves == 1 && a.k_scale == nullptr ? kWinCus : 2 * kWinCus;
  int64_t parts = want / ((int64_t)a.Hkv * t.q_tiles * a.B);
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
  static_assert(kWinTwoTermRows == 2 * kAttnTile, "two wavefronts' rows always have two terms, four wavefronts' never");
  if (a.out != nullptr) go(std::integral_constant<int, 3>());
  else go(std::integral_constant<int, QW <= 2 ? 2 : 1>());
}

static void launch_stream(const dsk_window_attn_args& a, const WinLaunch& t, const WinCache& c, const WinOut& to, float scale_log2, hipStream_t st) {
  const int G = a.Hq / a.Hkv;
  const dim3 grid((unsigned)a.Hkv, (unsigned)t.sp.parts, (unsigned)a.B), block(kStreamWaves * DSK_WAVE);
  auto go = [&](auto terms, auto stream) {
    constexpr int kTerms = decltype(terms)::value;
    constexpr bool kStream = decltype(stream)::value;
    if (a.k_scale != nullptr) window_stream_kernel<kTerms, true, kStream><<<grid, block, 0, st>>>(a, c, to, G, t.sp, scale_log2);
    else window_stream_kernel<kTerms, false, kStream><<<grid, block, 0, st>>>(a, c, to, G, t.sp, scale_log2);
  };
  if (a.out != nullptr) go(std::integral_constant<int, 3>(), std::false_type());
  else go(std::integral_constant<int, 2>(), std::false_type());
}

hipError_t launch_window_attn(const dsk_window_attn_args& a, hipStream_t st) {
  const WinLaunch t = win_layout(a);
  const int G = a.Hq / a.Hkv;
  const WinCache c = win_cache(a);
  const WinOut to = win_out(a, t.sp.parts > 1 ? (size_t)a.n_tokens * a.Hq * t.sp.parts : 0);
  const float scale_log2 = (a.scale != 0.0f ? a.scale : kWinScale) * kLog2e;
  if (t.q_waves == 1) launch_stream(a, t, c, to, scale_log2, st);
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

}  // namespace dsk
