// Norm and rotation of a row of 128 channels spread over 16 lanes x 8 channels, shared by the kernels that bring queries and keys
// into the cache.
#pragma once

#include "dsk_common.hpp"

namespace dsk {

constexpr int kRopeHalf = DSK_HEAD_DIM / 2;

enum class RopePairs { kNone, kHalfAll, kHalf, kInterleaved };   // kHalfAll: channels i and i + 64, a fixed lane move

typedef __bf16 rope_bf16x2 __attribute__((ext_vector_type(2)));
typedef float rope_f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_bf16_rne(float lo, float hi) {
  const rope_f32x2 f = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, rope_bf16x2));
}

// sum of the row's squares, in every lane of it
__device__ __forceinline__ float rope_square_sum(const float (&f)[8]) {
  float ss = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) ss = fmaf(f[e], f[e], ss);
  return group16_sum(ss);
}

// the norm of a row of that sum of squares; weight: of the lane's channels, 16-byte aligned if it is in memory
__device__ __forceinline__ void rope_scale(float (&f)[8], float ss, const float* weight, float eps) {
  const float inv = 1.0f / sqrtf(ss * (1.0f / DSK_HEAD_DIM) + eps);
  const float4 w0 = *reinterpret_cast<const float4*>(weight);
  const float4 w1 = *reinterpret_cast<const float4*>(weight + 4);
  f[0] *= inv * w0.x; f[1] *= inv * w0.y; f[2] *= inv * w0.z; f[3] *= inv * w0.w;
  f[4] *= inv * w1.x; f[5] *= inv * w1.y; f[6] *= inv * w1.z; f[7] *= inv * w1.w;
}

// Rotation of a lane's channels.  inside: they are rotated at all; kHalf: partner is the lane with the other channels of the pairs, and
// sn has its sign turned where the lane has the first ones.  kInterleaved: cs and sn hold four pairs.
template <RopePairs PAIRS>
__device__ __forceinline__ void rope_turn(float (&f)[8], const float (&cs)[8], const float (&sn)[8], bool inside, int partner) {
  if constexpr (PAIRS == RopePairs::kInterleaved) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float lo = f[2 * e], hi = f[2 * e + 1];
      f[2 * e] = inside ? fmaf(lo, cs[e], -hi * sn[e]) : lo;
      f[2 * e + 1] = inside ? fmaf(lo, sn[e], hi * cs[e]) : hi;
    }
  } else if constexpr (PAIRS != RopePairs::kNone) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float o = PAIRS == RopePairs::kHalfAll ? dpp_f<0x128>(f[e]) : __shfl(f[e], partner, DSK_WAVE);   // 0x128: 8 lanes on in the row of 16
      f[e] = PAIRS == RopePairs::kHalfAll || inside ? fmaf(f[e], cs[e], o * sn[e]) : f[e];
    }
  }
}

}  // namespace dsk
