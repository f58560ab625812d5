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
#include "dsk_window_run.hpp"

namespace dsk {

// ---- a workgroup's keys folded into its rows -----------------------------------------------------------------
// QW wavefronts have 32 rows each, KW take other tiles of a stage for the same rows, NT of them each.  A stage is copied while the one
// before it is multiplied.  TERMS: bf16 terms of a weight.  131K tokens of 8 heads in 8 bits: 64 rows a head 78 us (two wavefronts of rows,
// two of tiles; 3.4 TB/s and 0.44 PFLOP/s), 128 rows 100 us (0.69 PFLOP/s), in bf16 94 and 110, without the merge; whole calls 85, 117, 106
// and 117, with a result in 32 bits 95, 160, 108 and 164.  Here products, exponentials and LDS take turns, and only the second workgroup
// of a CU fills in.
template <int QW, int KW, int NT, int TERMS, bool E4M3>
struct WinFold {
  static constexpr int kThreads = QW * KW * DSK_WAVE;
  static constexpr int kTiles = KW * NT, kKeys = kAttnTile * kTiles;   // of a stage
  static constexpr int kRowBytes = E4M3 ? DSK_HEAD_DIM : 2 * DSK_HEAD_DIM;
  static constexpr int kTile = kAttnTile * kRowBytes;
  static constexpr int kBuf = 2 * kTiles * kTile;
  static constexpr int kChunks = kRowBytes / 16, kRowsAtOnce = DSK_WAVE / kChunks;   // of a wavefront's copy
  static constexpr int kCopies = kKeys / (kRowsAtOnce * QW * KW);
  static_assert(kKeys <= kThreads && kCopies >= 1, "a thread a scale, every wavefront copies");
  static_assert(KW == 1 || 2 * kBuf >= (KW - 1) * QW * 64 * DSK_WAVE * 4, "states are joined in the stages' place");
  struct Shared {
    __align__(16) unsigned char kv[2 * kBuf];
    float2 ml[KW > 1 ? (KW - 1) * QW * DSK_WAVE : 1];
    __align__(16) float scale[E4M3 ? 4 * kKeys : 4];
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
        bool left_out = !plain && vf.keep_finite();
        bool no_scale = false;                           // nor is every scale a number
        if constexpr (E4M3) {
          no_scale = !plain && __any(scale[kKeys + tile * kAttnTile + rows.col] == __builtin_inff());
          left_out |= no_scale;
        }
        TileWeights<TERMS> w;
        sm.template take<TERMS, true>(z, O, w, [&](float (&p)[16]) {
          if constexpr (E4M3) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              float4 f = *reinterpret_cast<const float4*>(scale + kKeys + tile * kAttnTile + 4 * rows.half + 8 * j);
              if (no_scale) {
                f.x = f.x == __builtin_inff() ? 0.0f : f.x;
                f.y = f.y == __builtin_inff() ? 0.0f : f.y;
                f.z = f.z == __builtin_inff() ? 0.0f : f.z;
                f.w = f.w == __builtin_inff() ? 0.0f : f.w;
              }
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
    if (keys.begin < keys.end) {
      copy(c, keys, hk, keys.begin, sh.kv);
      b = scales(c, keys, hk, keys.begin);
    }
    for (int v0 = keys.begin; v0 < keys.end; v0 += kTiles) {
      lds_copies_done();
      if (E4M3 && tid < kKeys) {
        sh.scale[buf * 2 * kKeys + tid] = __uint_as_float((uint32_t)b.x << 23);
        sh.scale[buf * 2 * kKeys + kKeys + tid] = __uint_as_float((uint32_t)b.y << 23);
      }
      __syncthreads();                                   // the stage is here, and nobody reads the other one any more
      if (v0 + kTiles < keys.end) {
        copy(c, keys, hk, v0 + kTiles, sh.kv + (buf ^ 1) * kBuf);
        b = scales(c, keys, hk, v0 + kTiles);
      }
      if (rows.busy) tiles(v0, buf);
      buf ^= 1;
    }
    __syncthreads();
  }
};

template <int QW, int KW, int NT, int TERMS, bool E4M3>
__global__ __launch_bounds__(QW * KW * DSK_WAVE, 2) void window_attn_kernel(dsk_window_attn_args a, WinCache c, WinOut to, int G, int q_tiles,
                                                                            WinSplit sp, float scale_log2) {
  using Fold = WinFold<QW, KW, NT, TERMS, E4M3>;
  __shared__ typename Fold::Shared sh;
  const int wave = threadIdx.x / DSK_WAVE, qw = wave % QW, kw = wave / QW;
  WinWork work;
  WinRun keys;
  int tok0 = 0, len = 0;
  if (!work.find(a, sp, G, blockIdx.x / q_tiles, blockIdx.x % q_tiles, QW * kAttnTile, keys, tok0, len)) return;   // uniform, as all returns before the end
  WinRows rows;
  work.rows<E4M3>(rows, a, G, qw * kAttnTile, tok0, len);
  TileSoftmax sm(scale_log2);
  tile_f32x16 O[4];
  win_clear(O);
  WinKept kept;
  for (;;) {
    const int end = keys.end;
    const bool more = TERMS == 3 && end - keys.begin > KW * kWinSegment;   // uniform
    if (more) keys.end = keys.begin + KW * kWinSegment;
    Fold::run(sh, c, keys, work.hk, rows, kw, sm, O);
    if (!more) break;
    TileSoftmax so_far = sm;                             // (its sum of weights is not used)
    if constexpr (KW > 1) tile_join<QW, KW>(so_far, O, rows.busy, qw, kw, reinterpret_cast<float*>(sh.kv), sh.ml);
    if (kw == 0 && rows.real) {
      float* const at = WinKept::place(to, rows, work.used == 1, work.part, sp.parts);
#pragma unroll
      for (int ct = 0; ct < 4; ++ct) {
        if (kept.any) kept.join(at, O[ct], ct, so_far.m);
        WinKept::put(at, O[ct], ct);
      }
    }
    kept.any = true;
    kept.m = so_far.m;
    win_clear(O);
    if constexpr (KW > 1) __syncthreads();               // the stages' place is free again
    keys.begin = keys.end;
    keys.end = end;
  }
  sm.close();
  if constexpr (KW > 1) {
    tile_join<QW, KW>(sm, O, rows.busy, qw, kw, reinterpret_cast<float*>(sh.kv), sh.ml);
    if (kw > 0) return;
  }
#pragma unroll
  for (int ct = 0; ct < 4; ++ct) {
    if (kept.any && rows.real) kept.join(WinKept::place(to, rows, work.used == 1, work.part, sp.parts), O[ct], ct, sm.m);
    win_store(to, rows, O[ct], ct, sm.m, sm.l, work.used == 1, work.part, sp.parts);
  }
}

// The same where the rows fit one wavefront: HBM bounds it.  268 MB of codes take 51 us (5.3 TB/s; with stages that the wavefronts share,
// and so wait for together, 65), 1.34 GB 199 us (6.7 TB/s); 269 MB in bf16 52.
template <int TERMS, bool E4M3, bool STREAM>
__global__ __launch_bounds__(kStreamWaves * DSK_WAVE, E4M3 ? 2 : 1) void window_stream_kernel(dsk_window_attn_args a, WinCache c, WinOut to, int G,
                                                                                             WinSplit sp, float scale_log2) {
  __shared__ WinStreamLds<E4M3> sh;
  WinWork work;
  WinRun keys;
  int tok0 = 0, len = 0;
  if (!work.find(a, sp, G, blockIdx.x, 0, kAttnTile, keys, tok0, len)) return;     // uniform
  WinRows rows;
  work.rows<E4M3>(rows, a, G, 0, tok0, len);
  TileSoftmax sm(scale_log2);
  tile_f32x16 O[4];
  win_clear(O);
  WinKept kept;
  for (;;) {
    const int end = keys.end;
    const bool more = TERMS == 3 && end - keys.begin > kStreamWaves * kWinSegment;   // uniform
    if (more) keys.end = keys.begin + kStreamWaves * kWinSegment;
    win_stream<TERMS, E4M3, STREAM>(sh, c, keys, work.hk, rows, sm, O);
    if (!more) sm.close();
    win_stream_store<E4M3>(sh, to, rows, sm, O, work.used == 1, work.part, sp.parts, kept, more);
    if (!more) break;
    win_clear(O);
    keys.begin = keys.end;
    keys.end = end;
  }
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
  win_merge<WAVES>(to, (int64_t)(at.tok0 + i) * a.Hq + h, sp.parts, wave, [&] {
    const int all = at.n * G, r0 = (i * G + h % G) / q_rows * q_rows;
    return WinTiles(a, at, G, r0, r0 + q_rows < all ? r0 + q_rows : all).used(sp.tiles_per_part);
  });
}

// ---- geometry: follows the host's bounds alone ---------------------------------------------------------------
// K and V larger than the memory-side cache (256 MB) push each other out before the next step, so they are read past it: the same 302 MB
// again and again 50 us instead of 52, 335 MB 54 and 61, 470 MB 74 and 85; 201 to 268 MB take as long either way.
constexpr int64_t kWinStreamBytes = 288ll << 20;

struct WinLaunch {
  int q_waves, q_rows, q_tiles;   // wavefronts' rows of a workgroup, its rows, workgroups for all of them
  bool wide;                      // window_wide_kernel
  bool stream;                    // K and V are read past the memory-side cache
  WinSplit sp;
};

// Parts of a sequence at most, whatever max_seqlen up to the given one is: a workspace that is kept serves a growing cache.
static int win_most_parts(const dsk_window_attn_args& a, int q_tiles, int64_t tiles) {
  const int64_t want = 2 * kWinCus / ((int64_t)a.Hkv * q_tiles), by_length = ceil_div(tiles, kWinLeastTiles);
  int64_t n = want < by_length ? want : by_length;
  n = n < kWinMaxSplit ? n : kWinMaxSplit;
  return (int)(n > 1 ? n : 1);
}

static WinLaunch win_layout(const dsk_window_attn_args& a, bool f32) {
  const int G = a.Hq / a.Hkv;
  const int64_t rows = (int64_t)a.max_new * G;
  WinLaunch t;
  t.q_waves = rows <= kAttnTile ? 1 : (rows <= kWinTwoTermRows ? 2 : 4);
  // Rows of a KV head, over 131K tokens of 8 heads in 8 bits, whole calls: 128 rows take four wavefronts 108 us, the eight that fit many rows 167, as
  // half of them have none; 256 rows 193 and 177 (in bf16 116 and 167, 179 and 167).  A result in 32 bits has weights of three terms,
  // which those have no registers for.
  t.wide = rows > 128 && !f32;
  t.q_rows = t.wide ? kWideRows : t.q_waves * kAttnTile;
  t.q_tiles = (int)ceil_div(rows, t.q_rows);
  // tiles that a workgroup's rows see at most: the window of all its tokens, the first ones, a tile begun at either end
  const int64_t tokens = a.max_new < t.q_rows / G + 2 ? a.max_new : t.q_rows / G + 2;
  const int64_t longest = (int64_t)a.max_seqlen + a.max_new;
  const int64_t near = ceil_div((int64_t)a.window + tokens, kAttnTile) + 1 + ceil_div(a.n_sink, kAttnTile);
  const int64_t tiles = near < ceil_div(longest, kAttnTile) ? near : ceil_div(longest, kAttnTile);
  // Tiles of all sequences.  Where the cache has no room for all of them at their longest they differ in length, and the parts are cut to
  // fill the chip with those that there are: eight sequences of 16K to 64K tokens in 8 bits, four new tokens 174 -> 142 us.  The lengths
  // are not known here: the same sequences in regions of 64K rows each are split as if they were as long, 159 us a call instead of 146.
  const int64_t rows_tiles = (int64_t)a.total_rows / kAttnTile + 2 * (int64_t)a.B, all = a.B * tiles < rows_tiles ? a.B * tiles : rows_tiles;
  const bool ragged = all < a.B * tiles;
  const int most = win_most_parts(a, t.q_tiles, tiles);
  // two workgroups a CU; one of those for many rows, and of those that stream bf16 tiles, whose rings are twice as large
  const int64_t want = (t.wide || (t.q_waves == 1 && a.k_scale == nullptr) ? kWinCus : 2 * kWinCus) / ((int64_t)a.Hkv * t.q_tiles);
  int64_t parts = ragged ? want - (a.B - 1) : want / a.B;  // of all sequences together, the last of each a shorter one; of each
  parts = parts > 1 ? parts : 1;
  int64_t per = ceil_div(ragged ? all : tiles, parts);
  const int64_t least = ceil_div(tiles, most);
  per = per > least ? per : least;
  t.sp.tiles_per_part = (int)(per > 1 ? per : 1);
  t.sp.parts = (int)ceil_div(tiles, t.sp.tiles_per_part);
  t.sp.parts = t.sp.parts > 1 ? t.sp.parts : 1;
  t.sp.packed = ragged && t.q_tiles == 1 && t.sp.parts > 1 && (int64_t)a.B * t.sp.parts <= 65535;
  t.stream = !t.wide && t.q_tiles == 1 && all * a.Hkv * kAttnTile * DSK_HEAD_DIM * (a.k_scale != nullptr ? 2 : 4) >= kWinStreamBytes;
  return t;
}

// A launch has fewer than 2^32 threads in x.  (Rows whose parts are put together are 65536 at most, as more are not split.)
bool window_attn_fits(const dsk_window_attn_args& a) {
  const WinLaunch t = win_layout(a, a.out != nullptr);
  return (int64_t)a.Hkv * t.q_tiles * (t.wide ? kWideWaves : 4) * DSK_WAVE <= 0xFFFFFFFF;
}

// Whichever outputs the call will ask for, and no less than with a smaller max_seqlen.
size_t window_ws_bytes(const dsk_window_attn_args& a) {
  int most = 1;
  for (const bool f32 : {false, true}) {
    const int n = win_most_parts(a, win_layout(a, f32).q_tiles, ceil_div((int64_t)a.max_seqlen + a.max_new, kAttnTile));
    most = n > most ? n : most;
  }
  return win_part_bytes(most > 1 ? (size_t)a.n_tokens * a.Hq * most : 0);
}

static dim3 win_grid(const dsk_window_attn_args& a, const WinLaunch& t, int x) {
  return t.sp.packed ? dim3((unsigned)x, (unsigned)(a.B * t.sp.parts)) : dim3((unsigned)x, (unsigned)t.sp.parts, (unsigned)a.B);
}

template <int QW, int KW, int NT8, int NT16>
static void launch_window(const dsk_window_attn_args& a, const WinLaunch& t, const WinCache& c, const WinOut& to, float scale_log2, hipStream_t st) {
  const int G = a.Hq / a.Hkv;
  const dim3 grid = win_grid(a, t, a.Hkv * t.q_tiles), block(QW * KW * DSK_WAVE);
  auto go = [&](auto terms) {
    constexpr int kTerms = decltype(terms)::value;
    if (a.k_scale != nullptr)
      window_attn_kernel<QW, KW, NT8, kTerms, true><<<grid, block, 0, st>>>(a, c, to, G, t.q_tiles, t.sp, scale_log2);
    else
      window_attn_kernel<QW, KW, NT16, kTerms, false><<<grid, block, 0, st>>>(a, c, to, G, t.q_tiles, t.sp, scale_log2);
  };
  static_assert(kWinTwoTermRows == 2 * kAttnTile, "two wavefronts' rows always have two terms, four wavefronts' never");
  if (a.out != nullptr) go(std::integral_constant<int, 3>());
  else go(std::integral_constant<int, QW <= 2 ? 2 : 1>());
}

static void launch_stream(const dsk_window_attn_args& a, const WinLaunch& t, const WinCache& c, const WinOut& to, float scale_log2, hipStream_t st) {
  const int G = a.Hq / a.Hkv;
  const dim3 grid = win_grid(a, t, a.Hkv), block(kStreamWaves * DSK_WAVE);
  auto go = [&](auto terms, auto stream) {
    constexpr int kTerms = decltype(terms)::value;
    constexpr bool kStream = decltype(stream)::value;
    if (a.k_scale != nullptr) window_stream_kernel<kTerms, true, kStream><<<grid, block, 0, st>>>(a, c, to, G, t.sp, scale_log2);
    else window_stream_kernel<kTerms, false, kStream><<<grid, block, 0, st>>>(a, c, to, G, t.sp, scale_log2);
  };
  auto terms = [&](auto stream) {
    if (a.out != nullptr) go(std::integral_constant<int, 3>(), stream);
    else go(std::integral_constant<int, 2>(), stream);
  };
  if (t.stream) terms(std::true_type());
  else terms(std::false_type());
}

hipError_t launch_window_attn(const dsk_window_attn_args& a, hipStream_t st) {
  const WinLaunch t = win_layout(a, a.out != nullptr);
  const int G = a.Hq / a.Hkv;
  const WinCache c = win_cache(a);
  const WinOut to = win_out(a, t.sp.parts > 1 ? (size_t)a.n_tokens * a.Hq * t.sp.parts : 0);
  const float scale_log2 = (a.scale != 0.0f ? a.scale : kWinScale) * kLog2e;
  if (t.wide) {
    const hipError_t err = launch_window_wide(a, c, to, win_grid(a, t, a.Hkv * t.q_tiles), t.q_tiles, t.sp, scale_log2, st);
    if (err != hipSuccess) return err;
  } else if (t.q_waves == 1) launch_stream(a, t, c, to, scale_log2, st);
  else if (t.q_waves == 2) launch_window<2, 2, 2, 1>(a, t, c, to, scale_log2, st);
  else launch_window<4, 1, 4, 2>(a, t, c, to, scale_log2, st);
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess || t.sp.parts <= 1) return err;
  const bool many = t.sp.parts >= kWinMergeMany;
  const int64_t rows = (int64_t)a.max_new * a.Hq, wgs = ceil_div(rows, many ? 1 : kWinMergeWaves);
  const dim3 grid((unsigned)wgs, (unsigned)a.B), block(kWinMergeWaves * DSK_WAVE);
  if (many) window_merge_kernel<kWinMergeWaves><<<grid, block, 0, st>>>(a, to, G, t.q_rows, t.sp);
  else window_merge_kernel<1><<<grid, block, 0, st>>>(a, to, G, t.q_rows, t.sp);
  return hipGetLastError();
}

}  // namespace dsk
