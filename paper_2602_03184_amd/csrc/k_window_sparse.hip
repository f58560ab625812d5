// Attention of one new token a sequence to selected slots and to what is near: the newest tokens and the first ones
// (dsk_window_sparse_decode_attn).
#include "dsk_window_fold.hpp"

namespace dsk {

// Keys of a workgroup that are listed in LDS as rows of the cache: every row of the product sees all of them.
struct WinList {
  static constexpr bool kRun = false;
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

// ---- selected slots and what is near ---------------------------------------------------------------------------
struct WinSparse {
  int G, heads;               // query heads of a KV head; lists of a sequence
  int slots_per_part, slot_parts;
  int near_per_part, near_parts;
  int row_tiles;              // workgroups for the query heads of a KV head, 32 each
};

// Parts 0 .. slot_parts - 1 of a list are its slots'; the others, of a KV head, are what is near.  Every part leaves a result.  Latency
// bounds it: lengths and slots, the list of rows in LDS, their scales and codes, two tiles a wavefront.  32 lists of 4096 tokens in 8 bits
// and 8 windows of 128 take 11.7 us (25 MB), 64 lists of 4096 tokens and 64 windows of 1024 19.3 us (67 MB at 3.5 TB/s).
template <int TERMS, bool E4M3>
__global__ __launch_bounds__(kStreamWaves * DSK_WAVE, E4M3 ? 2 : 1) void window_sparse_kernel(dsk_window_sparse_args a, WinCache c, WinOut to, WinSparse sp,
                                                                         float scale_log2) {
  __shared__ WinStreamLds<E4M3> sh;
  __shared__ int32_t sm_rows[kWinMaxListed];
  __shared__ int32_t sm_slot[3][kWinMaxSlots];
  __shared__ int32_t sm_wave[kWinMaxSlots / DSK_WAVE];
  constexpr int kThreads = kStreamWaves * DSK_WAVE;
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
    slots = slots < 0 ? 0 : (slots < a.k ? slots : a.k);
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
  win_stream<TERMS, E4M3, false>(sh, c, keys, hk, rows, sm, O);
  sm.close();
  const int parts = sp.slot_parts + sp.near_parts;
  static_assert(kWinMaxListed <= kStreamWaves * kWinSegment * kAttnTile, "one segment");
  WinKept none;
  win_stream_store<E4M3>(sh, to, rows, sm, O, parts == 1, part, parts, none, false);
}

template <int WAVES>
__global__ __launch_bounds__(kWinMergeWaves * DSK_WAVE) void window_sparse_merge_kernel(int64_t rows, WinOut to, int parts) {
  const int wave = threadIdx.x / DSK_WAVE;
  const int64_t row = (int64_t)blockIdx.x * (kWinMergeWaves / WAVES) + wave / WAVES;
  if (row < rows) win_merge<WAVES>(to, row, parts, wave, [&] { return parts; });
}

// ---- geometry: follows the host's bounds alone ---------------------------------------------------------------
static int64_t win_most_slots(int b) { return kWinMaxListed / b < kWinMaxSlots ? kWinMaxListed / b : kWinMaxSlots; }
static int64_t win_least_slots(int b) { return kWinLeastKeys / b > 1 ? kWinLeastKeys / b : 1; }

static WinSparse win_sparse_layout(const dsk_window_sparse_args& a) {
  WinSparse sp;
  const bool shared = a.flags & DSK_ATTN_SHARED_SELECTION;
  sp.G = a.Hq / a.Hkv;
  sp.heads = shared ? a.Hkv : a.Hq;
  const int64_t near = (int64_t)a.window + a.n_sink < a.max_seqlen ? (int64_t)a.window + a.n_sink : a.max_seqlen;
  // Tokens of a part: as few as leave all parts in one round of workgroups, two a CU in 8 bits and one in bf16, whose rings are twice as
  // large.
  const int64_t want = a.k_scale != nullptr ? 2 * kWinCus : kWinCus, lists = (int64_t)a.B * sp.heads, groups = (int64_t)a.B * a.Hkv;
  int64_t tokens = (lists * a.k * a.b + groups * near) / want / kAttnTile * kAttnTile;
  tokens = tokens > kWinLeastKeys ? tokens : kWinLeastKeys;
  for (;; tokens += kAttnTile) {
    tokens = tokens < kWinMaxListed ? tokens : kWinMaxListed;
    int64_t per = tokens / a.b > 1 ? tokens / a.b : 1;
    per = per < win_most_slots(a.b) ? per : win_most_slots(a.b);
    sp.slots_per_part = (int)per;
    sp.slot_parts = (int)ceil_div(a.k, per);
    sp.near_per_part = (int)tokens;
    sp.near_parts = (int)ceil_div(near, tokens);
    if (tokens == kWinMaxListed || lists * sp.slot_parts + groups * sp.near_parts <= want) break;
  }
  sp.row_tiles = (int)ceil_div(sp.G, kAttnTile);
  return sp;
}

// A launch has fewer than 2^32 threads in x and at most 65535 workgroups in y.
bool window_sparse_fits(const dsk_window_sparse_args& a) {
  const WinSparse sp = win_sparse_layout(a);
  const int64_t parts = (int64_t)sp.slot_parts + sp.near_parts, rows = (int64_t)a.B * a.Hq;
  const int64_t merge = parts <= 1 ? 0 : ceil_div(rows, parts >= kWinMergeMany ? 1 : kWinMergeWaves);
  return (int64_t)sp.heads * sp.row_tiles <= 65535 && parts * kStreamWaves * DSK_WAVE <= 0xFFFFFFFF && merge * kWinMergeWaves * DSK_WAVE <= 0xFFFFFFFF;
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
    if (a.out != nullptr) window_sparse_kernel<3, true><<<grid, block, 0, st>>>(a, c, to, sp, scale_log2);
    else window_sparse_kernel<2, true><<<grid, block, 0, st>>>(a, c, to, sp, scale_log2);
  } else {
    if (a.out != nullptr) window_sparse_kernel<3, false><<<grid, block, 0, st>>>(a, c, to, sp, scale_log2);
    else window_sparse_kernel<2, false><<<grid, block, 0, st>>>(a, c, to, sp, scale_log2);
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
