// Which positions of a sequence the rows of a workgroup of dsk_window_attn see.
#pragma once

#include "dsk_window_fold.hpp"

namespace dsk {

constexpr int kWideWaves = 8, kWideRows = kWideWaves * kAttnTile;   // of a workgroup of the kernel for many rows

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
  // Every row sees all of the tile: plain(v) as an interval of tiles and those of first tokens before it.
  struct Plain {
    int few, from, to;
    __device__ __forceinline__ bool operator()(int v) const { return v < few || (v >= from && v < to); }
  };
  __device__ __forceinline__ Plain plain_tiles() const {
    const int end = tiles.p0 + 1 < there ? tiles.p0 + 1 : there;       // of what the first row sees
    const int gone = tiles.p1 - window + 1 - tiles.lo;                 // positions of the run that the last row does not see
    Plain p;
    p.few = 0;
    if (tiles.first > 0 || tiles.lo == 0) {
      const int most = tiles.first > 0 ? tiles.first : tiles.n, upto = sinks < end ? sinks : end;
      p.few = upto / kAttnTile < most ? upto / kAttnTile : most;
    }
    p.from = tiles.first + (gone > 0 ? (int)(((int64_t)gone + kAttnTile - 1) / kAttnTile) : 0);
    p.to = end > tiles.lo ? tiles.first + (end - tiles.lo) / kAttnTile : tiles.first;
    return p;
  }
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

struct WinSplit {
  int parts, tiles_per_part;   // of a sequence at most; of a part
  bool packed;                 // workgroups are numbered through the parts that there are, not by sequence
};

// The p-th part of all sequences', those of a sequence one after the other; false: there are fewer.  Every wavefront for itself.
__device__ __forceinline__ bool win_find_part(const dsk_window_attn_args& a, const WinSplit& sp, int G, int p, int& s, int& part) {
  const int lane = threadIdx.x & (DSK_WAVE - 1);
  for (int s0 = 0; s0 < a.B; s0 += DSK_WAVE) {
    int parts = 0;
    if (s0 + lane < a.B) {
      const WinPlace at(a, s0 + lane);
      if (at.n > 0) parts = WinTiles(a, at, G, 0, at.n * G).used(sp.tiles_per_part);
    }
    const int incl = wave_incl_scan_i(parts, lane), total = __builtin_amdgcn_readlane(incl, DSK_WAVE - 1);
    if (p < total) {
      const int before = __builtin_popcountll(__ballot(incl <= p));    // sequences
      s = __builtin_amdgcn_readfirstlane(s0 + before);
      part = before > 0 ? p - __builtin_amdgcn_readlane(incl, before - 1) : p;
      return true;
    }
    p -= total;
  }
  return false;
}

// What a workgroup takes: rows from r0 on of KV head hk, and a part of the tiles that they see; false: nothing.
struct WinWork {
  int s, hk, part, used;
  int64_t r0, all;      // first row; rows of the sequence
  __device__ __forceinline__ bool find(const dsk_window_attn_args& a, const WinSplit& sp, int G, int head, int q_tile, int q_rows, WinRun& keys, int& tok0, int& len) {
    part = blockIdx.y;
    s = blockIdx.z;
    if (sp.packed && !win_find_part(a, sp, G, blockIdx.y, s, part)) return false;
    hk = head;
    const WinPlace at(a, s);
    r0 = (int64_t)q_tile * q_rows;
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

hipError_t launch_window_wide(const dsk_window_attn_args& a, const WinCache& c, const WinOut& to, dim3 grid, int q_tiles, const WinSplit& sp,
                              float scale_log2, hipStream_t st);

}  // namespace dsk
