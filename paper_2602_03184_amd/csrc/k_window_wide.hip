// dsk_window_attn for many rows (prompts): the matrix cores bound it.
//
// Eight wavefronts of 32 rows make a workgroup, two a SIMD, and read each tile of K and V from LDS.  A wavefront's step begins with its
// products, of K for the logits of the next tile and of V with the weights of the one before, and among them the exponentials of this
// one; then it reads the fragments that come next, which the other wavefront of the SIMD covers.  What is rare (masks, a reference that
// moves, the ends of a run) lies on branches that a step in the middle of a run does not take: 624 us for a prompt of 8191 tokens of 32
// heads in bf16 (880 TFLOP/s; 670 where every step asks for all of it), 184 for 2048 tokens over windows of 4096 in 8 bits.  A step takes
// about 2300 cycles: 1024 of the matrix core for two wavefronts, 1000 of the vector ALU, the rest waits, mostly for LDS.  Four wavefronts
// of 64 rows read LDS half as often, but nothing fills in where a lone one waits (702 us); two wavefronts kept half a step apart by a
// second barrier take 613 us in bf16 and 199 in 8 bits, where widening makes their halves unequal.  (Each compared side by side; whole
// calls take 560 to 617 us and 159 to 171, as the card's clock allows.)
//
// A weight has one bf16 term: it is off by 2^-8 of itself at most, and results by 0.0022 (root mean square) where rounding them
// to bf16 alone gives 0.0016.  A second term would be half as many products again.
//
// K and V come to LDS through registers, a ring of four tiles in bf16: codes are widened on the way, once for all wavefronts.  In step i
// tile i + 3 is written where tile i - 1 was, while K of tile i + 2 and V of tile i are read: one barrier a step.  All 256 registers of a
// wavefront are taken, and four to six more go through scratch.
#include "dsk_window_run.hpp"

namespace dsk {

// What a thread has of a tile on its way: a 16-byte chunk of a row of K and of V in bf16, or the eight codes that make one.
template <bool E4M3>
struct WideStage {
  static constexpr int kBytes = E4M3 ? 8 : 16;
  typename std::conditional<E4M3, uint2, uint4>::type k, v;
  uint32_t ks, vs;      // scales of the row
};

// BYTES of each lane from a uniform address and the lane's 32-bit offset (the asm keeps the compiler from making 64-bit addresses)
template <int BYTES>
__device__ __forceinline__ auto wide_load(tile_global base, uint32_t off) {
  asm("" : "+s"(base), "+v"(off));
  typedef uint32_t words __attribute__((ext_vector_type(BYTES / 4)));
  return __builtin_bit_cast(typename std::conditional<BYTES == 8, uint2, uint4>::type, *(const __attribute__((address_space(1))) words*)(base + off));
}

// Tiles on their way, one after the other from the run's first on.  Loads lie on no branch: where one does, the compiler waits for more
// of them than it has to.
template <bool E4M3>
struct WideLoader {
  using Stage = WideStage<E4M3>;
  static constexpr int kChunks = DSK_HEAD_DIM / 8;       // of a row
  static_assert(kWideWaves * DSK_WAVE == kAttnTile * kChunks, "a thread a chunk of a tile");
  const WinCache& c;
  const WinRun& keys;
  const WinRun::Plain plain;
  int hk, row, chunk;
  int v;                // the next tile
  int64_t at;           // its first row, and its addresses
  tile_global k, w;
  uint32_t k_off, v_off;   // of the thread
  int64_t scale;        // with codes: where the scale of the thread's row is
  __device__ __forceinline__ WideLoader(const WinCache& cache, const WinRun& run, int head) : c(cache), keys(run), plain(run.plain_tiles()), hk(head) {
    row = threadIdx.x / kChunks;
    chunk = threadIdx.x % kChunks;
    go(keys.begin);
  }
  __device__ __forceinline__ void go(int tile) {
    v = tile;
    at = keys.start(v);
    k = (tile_global)(c.K + hk * c.k_head + at * c.k_tok);
    w = (tile_global)(c.V + hk * c.v_head + at * c.v_tok);
    const int last = keys.last(v), n = row < last ? row : last;   // rows behind the last one that there is are that one again
    k_off = (uint32_t)(n * (int)c.k_tok + chunk * Stage::kBytes);
    v_off = (uint32_t)(n * (int)c.v_tok + chunk * Stage::kBytes);
    scale = E4M3 ? at + n : 0;
  }
  // the next tile; quiet: it is whole, and neither the last one nor the last of the first tokens'
  __device__ __forceinline__ void fetch(Stage& x, bool quiet) {
    x.k = wide_load<Stage::kBytes>(k, k_off);
    x.v = wide_load<Stage::kBytes>(w, v_off);
    if constexpr (E4M3) {
      const int64_t block = hk * c.s_head + (scale >> c.s_shift);
      x.ks = c.ks[block];
      x.vs = c.vs[block];
    }
    if (__builtin_expect(quiet, 1)) {
      v += 1;
      at += kAttnTile;
      k += kAttnTile * c.k_tok;
      w += kAttnTile * c.v_tok;
      if constexpr (E4M3) scale += kAttnTile;
    } else if (v + 1 < keys.end) {                       // beyond the last one that comes again, and is not read
      go(v + 1);
    }
  }
  // Tile v into its buffer.  A masked row may hold anything, and 0 * NaN is NaN: where not every row sees all of the tile, values that are
  // not finite (of codes: with their scale) are left out and the tile is noted.
  __device__ __forceinline__ void put(const Stage& x, int tile, bool quiet, unsigned char* sm_k, int* sm_left_out) const {
    uint4 a, b;
    if constexpr (!E4M3) {
      a = x.k;
      b = x.v;
    } else {
      a = __builtin_bit_cast(uint4, win_widen8(x.k.x, x.k.y, __uint_as_float(x.ks << 23)));
      b = __builtin_bit_cast(uint4, win_widen8(x.v.x, x.v.y, __uint_as_float(x.vs << 23)));
    }
    if (__builtin_expect(!quiet && !plain(tile), 0)) {   // (nor of what lies behind the last one)
      uint4 y = make_uint4(finite_bf16(b.x), finite_bf16(b.y), finite_bf16(b.z), finite_bf16(b.w));
      if (E4M3 && x.vs == 255) y = make_uint4(0, 0, 0, 0);
      if ((y.x ^ b.x) | (y.y ^ b.y) | (y.z ^ b.z) | (y.w ^ b.w)) *sm_left_out = tile;
      b = y;
    }
    unsigned char* const sm_v = sm_k + kTileBytes;
    *reinterpret_cast<uint4*>(sm_k + row * kTileRowBytes + ((chunk ^ (row & 15)) << 4)) = a;
    *reinterpret_cast<uint4*>(sm_v + row * kTileRowBytes + ((chunk ^ ((row & 3) << 2)) << 4)) = b;
  }
};

// A wavefront's rows.  The softmax is that of TileSoftmax, taken apart: exponents are made from the reference as it is when the
// logits come, and again in the rare case that it has to move.
struct WideRows {
  WinRows rows;
  TileSoftmax sm;
  tile_f32x16 O[4];
  tile_f32x16 z;        // logits of a tile,
  float x[16];          // their exponents, in log2 units above the reference,
  float mx;             // and the largest of these
  TileWeights<1> w;
  __device__ __forceinline__ explicit WideRows(float scale_log2) : sm(scale_log2) { win_clear(O); }
  __device__ __forceinline__ void exponents() {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = sm.exponent.of(z[i]);
    float a = fmaxf(fmaxf(x[0], x[1]), x[2]), b = fmaxf(fmaxf(x[3], x[4]), x[5]);
    a = fmaxf(fmaxf(a, x[6]), x[7]);
    b = fmaxf(fmaxf(b, x[8]), x[9]);
    a = fmaxf(fmaxf(a, x[10]), x[11]);
    b = fmaxf(fmaxf(b, x[12]), x[13]);
    mx = tile_half_max(fmaxf(fmaxf(fmaxf(a, x[14]), x[15]), b));
  }
  __device__ __forceinline__ uint32_t allowed(const WinRun& keys, int v) const { return rows.real ? keys.allowed(v, rows.pos) : 0u; }
  // what comes between the logits of tile v and their weights
  __device__ __forceinline__ void look(const WinRun& keys, int v, bool plain, WinVFrag<false>& vf) {
    if (__builtin_expect(!plain, 0)) {
      tile_hide(z, allowed(keys, v) >> (4 * rows.half), 0);
      exponents();
    }
    if (__builtin_expect(__any(mx > 8.0f || sm.m == -__builtin_inff()), 0)) {
      vf.template add<1>(O, w, 0);                       // weights that wait for their product still go by the old reference
      vf.template add<1>(O, w, 1);
      // It is taken: what the next step multiplies is 0 in both factors, as 0 times an infinity that all rows see is NaN.
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        w.w[0][t] = __builtin_bit_cast(tile_bf16x8, make_uint4(0, 0, 0, 0));
#pragma unroll
        for (int ct = 0; ct < 4; ++ct) vf.v[ct][t] = w.w[0][t];
      }
      const float top = tile_max(z) * sm.scale_log2;
      const bool move = mx > 8.0f || sm.m == -__builtin_inff();
      const float m_new = move ? fmaxf(sm.m, top) : sm.m;
      const float f = sm.m == -__builtin_inff() ? 0.0f : exp2_small(sm.m - m_new);
      sm.l *= f;
      sm.err *= f;
      tile_scale(O, f);
      sm.m = m_new;
      sm.exponent = FmaExponent(sm.scale_log2, sm.m == -__builtin_inff() ? 0.0f : sm.m);
      exponents();
    }
  }
};

// The weights of a tile, and meanwhile products: of K for the logits of the next one, of V with the weights of the one before.
__device__ __forceinline__ void wide_products(WideRows& h, const TileKFrag& kf, const WinVFrag<false>& vf) {
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int i = 0; i < 16; ++i) asm volatile("" : "+v"(h.x[i]));   // what is made of them is made here
  kf.template add<0, 8>(h.z, h.rows);
  vf.template add<1>(h.O, h.w, 0);
  vf.template add<1>(h.O, h.w, 1);
#pragma unroll
  for (int i = 0; i < 16; ++i) h.x[i] = exp2_small(h.x[i]);
  const float (&e)[16] = h.x;
  const float tile = ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7])) +
                     (((e[8] + e[9]) + (e[10] + e[11])) + ((e[12] + e[13]) + (e[14] + e[15])));
  const float add = tile - h.sm.err, sum = h.sm.l + add;
  h.sm.err = (sum - h.sm.l) - add;
  h.sm.l = sum;
  h.w.set(h.x);
  __builtin_amdgcn_iglp_opt(3);                          // a matrix instruction, an exponential, and what else there is
  asm volatile("" : "+v"(h.sm.l), "+v"(h.sm.err));
  __builtin_amdgcn_sched_barrier(0);
}

template <bool E4M3>
__global__ __launch_bounds__(kWideWaves * DSK_WAVE, 2) void window_wide_kernel(dsk_window_attn_args a, WinCache c, WinOut to, int G, int q_tiles,
                                                                              WinSplit sp, float scale_log2) {
  constexpr int kRing = 4, kBuf = 2 * kTileBytes;
  __shared__ __align__(16) unsigned char sm_kv[kRing * kBuf];
  __shared__ int sm_left_out[kRing];                     // the tile of which values were left out, -1 none
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / DSK_WAVE);
  // the last rows of a prompt see the most: they come first, and the workgroups of an XCD have few heads among them
  const int hk = blockIdx.x % a.Hkv, q_tile = q_tiles - 1 - blockIdx.x / a.Hkv;
  WinWork work;
  WinRun keys;
  int tok0 = 0, len = 0;
  if (!work.find(a, sp, G, hk, q_tile, kWideRows, keys, tok0, len)) return;     // uniform
  WideRows h(scale_log2);
  work.rows<false>(h.rows, a, G, wave * kAttnTile, tok0, len);

  const int begin = keys.begin, count = keys.end - keys.begin;
  if (threadIdx.x < kRing) sm_left_out[threadIdx.x] = -1;
  __syncthreads();
  WideStage<E4M3> x[2];
  TileKFrag kf;
  WinVFrag<false> vf;
  auto buffer = [&](int b) { return sm_kv + b * kBuf; };
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    h.w.w[0][t] = __builtin_bit_cast(tile_bf16x8, make_uint4(0, 0, 0, 0));
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) vf.v[ct][t] = h.w.w[0][t];
  }
  if (count > 0) {
    WideLoader<E4M3> loader(c, keys, hk);
    loader.fetch(x[0], false);
    loader.fetch(x[1], false);
    loader.put(x[0], begin, false, buffer(0), sm_left_out);
    loader.fetch(x[0], false);
    loader.put(x[1], begin + 1, false, buffer(1), sm_left_out + 1);
    loader.fetch(x[1], false);
    loader.put(x[0], begin + 2, false, buffer(2), sm_left_out + 2);
    loader.fetch(x[0], false);
    __syncthreads();
    kf.template read<0, 8>(buffer(0), h.rows);
    kf.template add<0, 8>(h.z, h.rows);
    kf.template read<0, 8>(buffer(1), h.rows);
    h.exponents();
    h.look(keys, begin, loader.plain(begin), vf);
    // Tile i in buffer B = i % 4: its exponents in h.x, K of tile i + 1 in kf, V of tile i - 1 in vf and its weights in h.w; set (i + 1) % 2 of
    // x has tile i + 3.
    const int quiet_from = loader.plain.from - begin, quiet_to = (loader.plain.to < keys.end ? loader.plain.to : keys.end) - begin - 7;
    auto step = [&](auto buf, int i) {
      const bool quiet = i >= quiet_from && i <= quiet_to;   // tiles i to i + 6 are plain
      constexpr int B = decltype(buf)::value, kPut = (B + 3) % kRing, kSet = (B + 1) % 2;
      const int v = begin + i;
      wide_products(h, kf, vf);
      kf.template read<0, 8>(buffer((B + 2) % kRing), h.rows);
      vf.template read<0>(buffer(B) + kTileBytes);
      vf.template read<1>(buffer(B) + kTileBytes);
      loader.put(x[kSet], v + 3, quiet, buffer(kPut), sm_left_out + kPut);
      loader.fetch(x[kSet], quiet);
      h.exponents();
      if (quiet || i + 1 < count) h.look(keys, v + 1, quiet || loader.plain(v + 1), vf);   // (behind the last tile the logits are another one's and nobody's)
      if (__builtin_expect(!quiet && !loader.plain(v) && sm_left_out[B] == v, 0))
        win_add_left_out<E4M3>(h.O, c, keys, hk, v, h.allowed(keys, v), h.rows.half);
      __syncthreads();
    };
    using B0 = std::integral_constant<int, 0>;
    using B1 = std::integral_constant<int, 1>;
    using B2 = std::integral_constant<int, 2>;
    using B3 = std::integral_constant<int, 3>;
    for (int i = 0; i < count; i += kRing) {
      step(B0(), i);
      if (i + 1 < count) step(B1(), i + 1);
      if (i + 2 < count) step(B2(), i + 2);
      if (i + 3 < count) step(B3(), i + 3);
    }
    vf.template add<1>(h.O, h.w, 0);
    vf.template add<1>(h.O, h.w, 1);
  }
  h.sm.close();
#pragma unroll
  for (int ct = 0; ct < 4; ++ct) win_store(to, h.rows, h.O[ct], ct, h.sm.m, h.sm.l, work.used == 1, work.part, sp.parts);
}

hipError_t launch_window_wide(const dsk_window_attn_args& a, const WinCache& c, const WinOut& to, dim3 grid, int q_tiles, const WinSplit& sp,
                              float scale_log2, hipStream_t st) {
  const int G = a.Hq / a.Hkv;
  const dim3 block(kWideWaves * DSK_WAVE);
  if (a.k_scale != nullptr) window_wide_kernel<true><<<grid, block, 0, st>>>(a, c, to, G, q_tiles, sp, scale_log2);
  else window_wide_kernel<false><<<grid, block, 0, st>>>(a, c, to, G, q_tiles, sp, scale_log2);
  return hipGetLastError();
}

}  // namespace dsk
